"""AdamW over lists of tensors against the definition in 64 bits.

Bars, u = 2^-24: m and v are sums of two products of rounded factors, off by at most 4 u of the sum of the magnitudes (and of grad_scale g: 6 u).  The
update's quotient carries those of m and half of v's, and five roundings of its own: with |m| for the magnitude of m's terms, 12 u |m| /
(1 - beta1^t) / (sqrt(v) / sqrt(1 - beta2^t) + eps), beside 3 u of the parameter.  8-bit states lie within one unit of the format of the exact value; the
exact value may itself be off by the bar above, so that a neighbour one further is allowed where it is that near to a number of the format."""
import numpy as np
import pytest

from oracle import student as S
from rounding import hold

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
U = 2.0 ** -24
SIZES = [1, 2, 3, 4, 5, 255, 256, 257, 1023, 1024, 1025, 70001, 0, 64]


def _api():
    import paper_2604_06596_amd as P

    return P


def _random(rng, n, dtype, size, odd=0):
    """n values on the GPU, beginning `odd` elements behind an aligned address."""
    t = torch.zeros(n + odd, dtype=dtype, device="cuda")[odd:]
    t.copy_(torch.from_numpy(size * rng.standard_normal(n)))
    return t


def _wide(t):
    return t.double().cpu().numpy() if t.dtype != torch.float8_e4m3fn else t.float().double().cpu().numpy()


@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("param, grad, copy", [("float32", "float32", None), ("float32", "bfloat16", "bfloat16"), ("bfloat16", "bfloat16", None),
                                               ("float16", "float32", "float32"), ("float32", "float16", "float16")])
def test_states_in_32_bits(param, grad, copy, odd):
    P = _api()
    rng = np.random.default_rng(1)
    sizes = SIZES * 7  # more tensors than one launch takes
    params = [_random(rng, n, TYPES[param], 0.1, odd) for n in sizes]
    copies = [_random(rng, n, TYPES[copy], 0.1, odd) for n in sizes] if copy else None
    states = [(_random(rng, n, torch.float32, 0.01, odd), _random(rng, n, torch.float32, 0.01, odd).square_()) for n in sizes]
    decay = [0.1 * (k % 3) for k in range(len(sizes))]
    gs = torch.tensor([0.37], device="cuda")
    for step in (1, 2, 1000):
        grads = [_random(rng, n, TYPES[grad], 0.02, odd) for n in sizes]
        before = [(_wide(p), _wide(g), _wide(s[0]), _wide(s[1])) for p, g, s in zip(params, grads, states)]
        P.adamw_step(params, grads, states, step=step, lr=0.01, betas=(0.8, 0.99), eps=1e-7, weight_decay=decay, copies=copies, grad_scale=gs)
        for k, (p, g, m, v) in enumerate(before):
            scale = float(np.float32(0.37))
            want, m1, v1 = S.adamw(p, g, m, v, step, 0.01, 0.8, 0.99, 1e-7, float(np.float32(decay[k])), scale)
            terms = 0.8 * np.abs(m) + 0.2 * np.abs(scale * g)
            assert np.all(np.abs(_wide(states[k][0]) - m1) <= 6 * U * terms)
            assert np.all(np.abs(_wide(states[k][1]) - v1) <= 8 * U * v1)
            bar = 3 * U * np.abs(p) + 0.01 * 12 * U * terms / (1 - 0.8 ** step) / (np.sqrt(v1) / np.sqrt(1 - 0.99 ** step) + 1e-7)
            for out in (params[k],) + ((copies[k],) if copy else ()):  # a copy is rounded from the unrounded parameter
                hold(out, want, bar)


def _states8(P, rng, n):
    """States in 8 bits as an earlier step left them."""
    p = torch.zeros(n, device="cuda")
    state = P.adamw_state(p, bits=8)
    P.adamw_step([p], [_random(rng, n, torch.float32, 0.02)], [state], step=1, lr=0.01)
    return state


@pytest.mark.parametrize("odd", [0, 3])
@pytest.mark.parametrize("grad", ["float32", "bfloat16"])
def test_states_in_8_bits(grad, odd):
    P = _api()
    rng = np.random.default_rng(2)
    sizes = SIZES * 4
    params = [_random(rng, n, torch.float32, 0.1, odd) for n in sizes]
    copies = [_random(rng, n, torch.bfloat16, 0.1, odd) for n in sizes]
    states = [_states8(P, rng, n) for n in sizes]
    for step in (1, 2, 1000):
        grads = [_random(rng, n, TYPES[grad], 0.02 * 10.0 ** (step % 3 - 1), odd) for n in sizes]
        before = [(_wide(p), _wide(g), S.state_values(s[0].view(torch.uint8).cpu().numpy(), _wide(s[2])),
                   S.state_values(s[1].view(torch.uint8).cpu().numpy(), _wide(s[3])) ** 2) for p, g, s in zip(params, grads, states)]
        P.adamw_step(params, grads, states, step=step, lr=0.01, weight_decay=0.05, copies=copies, seed=step)
        for k, (p, g, m, v) in enumerate(before):
            want, m1, v1 = S.adamw(p, g, m, v, step, 0.01, 0.9, 0.999, 1e-8, float(np.float32(0.05)))
            if not len(p):
                continue
            terms = 0.9 * np.abs(m) + 0.1 * np.abs(g)
            bar = 3 * U * np.abs(p) + 0.01 * 12 * U * terms / (1 - 0.9 ** step) / (np.sqrt(v1) / np.sqrt(1 - 0.999 ** step) + 1e-8)
            hold(params[k], want, bar)
            assert torch.equal(copies[k], params[k].to(torch.bfloat16))
            codes = [s.view(torch.uint8).cpu().numpy() for s in states[k][:2]]
            for exact, slack, code, scale in ((m1, 6 * U * terms, codes[0], _wide(states[k][2])), (np.sqrt(v1), 8 * U * np.sqrt(v1), codes[1], _wide(states[k][3]))):
                top = [np.abs(exact[a:a + S.STATE_BLOCK]).max() for a in range(0, len(exact), S.STATE_BLOCK)]
                assert np.all((np.array(top) * (1 + 1e-6) >= 128 * scale) & (np.array(top) * (1 - 1e-6) < 256 * scale))
                unit = np.repeat(scale, S.STATE_BLOCK)[:len(exact)]
                low = S.state_neighbours(np.maximum(np.abs(exact) - slack, 0.0) / unit)[0] * unit
                high = S.state_neighbours((np.abs(exact) + slack) / unit)[1] * unit
                got = S.state_values(code, scale)
                assert np.all((np.abs(got) >= low) & (np.abs(got) <= high))
                assert np.all((got == 0) | (np.sign(got) == np.sign(exact)))
            assert np.all((codes[1] > 0) == (v1 > 0)) and np.all(codes[1] < 128)


def test_rounding_to_8_bits_is_right_on_average():
    """Of many equal values, as many are rounded up as lie between: 65,536 draws of a probability are off by 5 / 512 at most (five standard
    deviations); with another seed, step or tensor others are."""
    P = _api()
    n = 256 * 257
    for value in (0.71, 0.013, 3.1e-4, 2e-6):
        g = torch.full((n,), value, device="cuda")
        g[::256] = 1.0  # the block's largest: m = 0.1 of it
        seen = []
        for seed, step in ((0, 1), (0, 2), (1, 1)):
            states = [P.adamw_state(g, bits=8) for _ in range(2)]
            P.adamw_step([torch.zeros(n, device="cuda")] * 2, [g, g], states, step=step, lr=0.0, seed=seed)
            seen += [s[0].view(torch.uint8) for s in states]
            m = S.state_values(seen[-1].cpu().numpy(), _wide(states[1][2])).reshape(-1, 256)[:, 1:].ravel()
            exact = float(np.float32(np.float32(value) * np.float32(0.1)))
            low, high = (x[0] * states[1][2][0].item() for x in S.state_neighbours(np.array([exact / states[1][2][0].item()])))
            assert set(np.unique(m)) <= {low, high}
            assert abs((m == high).mean() - (exact - low) / (high - low)) <= 5 / 512
        assert all(not torch.equal(a, b) for i, a in enumerate(seen) for b in seen[:i])


def test_a_running_mean_in_8_bits_does_not_stand_still():
    """Gradients stop: after 3,000 steps v has fallen by 0.999^3000 = 0.05, r by 0.22, in the mean over many elements."""
    P = _api()
    n = 65536
    p, zero = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    g = torch.ones(n, device="cuda")
    g[::256] = 4.0
    state = P.adamw_state(p, bits=8)
    P.adamw_step([p], [g], [state], step=1, lr=0.0)
    first = S.state_values(state[1].view(torch.uint8).cpu().numpy(), _wide(state[3])).mean()
    for step in range(2, 3002):
        zero[::256] = 4.0  # the largest of each block stays, and so does the scale
        P.adamw_step([p], [zero], [state], step=step, lr=0.0, seed=9)
    r = S.state_values(state[1].view(torch.uint8).cpu().numpy(), _wide(state[3])).reshape(-1, 256)[:, 1:].mean()
    assert 0.1 * first < r < 0.45 * first


def test_zeros_infinities_and_tiny_values_in_8_bits():
    P = _api()
    n = 1024
    p = torch.ones(n, device="cuda")
    state = P.adamw_state(p, bits=8)
    zero = torch.zeros(n, device="cuda")
    P.adamw_step([p], [zero], [state], step=1, lr=0.1)
    assert torch.equal(p, torch.ones_like(p)) and not any(s.view(torch.uint8).any() for s in state)
    g = zero.clone()
    g[3] = float("inf")
    g[300] = float("nan")
    g[600] = 1e-30  # v = 1e-63 is below float32: r is 0, m is not
    g[900] = 1e-3
    P.adamw_step([p], [g], [state], step=2, lr=0.1)
    assert torch.isnan(state[2][:2]).all() and torch.isnan(state[3][:2]).all()
    assert torch.isfinite(state[2][2:]).all() and torch.isfinite(state[3][2:]).all() and float(state[3][2]) == 0.0
    good = torch.ones(n, dtype=torch.bool, device="cuda")
    good[:512] = False
    assert torch.isfinite(p[good]).all()
    untouched = torch.ones(n, dtype=torch.bool, device="cuda")
    untouched[[3, 300, 600, 900]] = False
    assert torch.equal(p[untouched], torch.ones_like(p)[untouched])
    P.adamw_step([p], [zero], [state], step=3, lr=0.1)
    assert torch.isnan(p[:512]).all() and torch.isfinite(p[512:]).all()


def test_the_same_bits_every_time_and_in_any_list():
    """A step over a list gives what the same seed gives again, and with 32 bits what each tensor gives alone."""
    P = _api()
    rng = np.random.default_rng(4)
    for bits in (8, 32):
        params = [_random(rng, n, torch.float32, 0.1) for n in (1000, 70, 4096)]
        grads = [_random(rng, p.numel(), torch.float32, 0.1) for p in params]
        results = []
        for turn in range(3):
            ps = [p.clone() for p in params]
            states = [P.adamw_state(p, bits) for p in ps]
            if turn < 2 or bits == 8:
                P.adamw_step(ps, grads, states, step=3, lr=0.1, seed=5)
            else:
                for p, g, s in zip(ps, grads, states):
                    P.adamw_step([p], [g], [s], step=3, lr=0.1)
            results.append(ps + [t.view(torch.uint8) if bits == 8 and t.dtype == torch.float8_e4m3fn else t for s in states for t in s])
        for other in results[1:]:
            assert all(torch.equal(a, b) for a, b in zip(results[0], other))


@pytest.mark.parametrize("bits", [8, 32])
def test_arrays_larger_than_the_caches(bits):
    """What is done past them is what is done through them: the first elements of a long tensor, and a tensor of these alone."""
    P = _api()
    rng = np.random.default_rng(6)
    n, few = 20_000_003, 1_000_003
    p, g = (torch.randn(n, device="cuda") for _ in range(2))
    state = P.adamw_state(p, bits)
    short = p[:few].clone()
    short_state = P.adamw_state(short, bits)
    for step in (1, 2):
        g.mul_(1.1)
        P.adamw_step([p], [g], [state], step=step, lr=0.1, seed=5)
        P.adamw_step([short], [g[:few]], [short_state], step=step, lr=0.1, seed=5)
    whole = few // 256 * 256  # the short tensor's last block has another scale
    assert torch.equal(p[:few], short)
    for a, b in zip(state[:2], short_state[:2]):
        assert torch.equal(a.view(torch.uint8)[:whole * a.element_size()], b.view(torch.uint8)[:whole * a.element_size()])


def test_replays_of_a_graph():
    P = _api()
    rng = np.random.default_rng(5)
    p, g = _random(rng, 5000, torch.float32, 0.1), _random(rng, 5000, torch.float32, 0.1)
    state = P.adamw_state(p, 8)
    P.adamw_step([p.clone()], [g], [P.adamw_state(p, 8)], step=1, lr=0.1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.adamw_step([p], [g], [state], step=7, lr=0.1, seed=3)
    q, other = p.clone(), tuple(s.clone() for s in state)
    for k in range(4):
        g.mul_(-0.7)
        graph.replay()
        P.adamw_step([q], [g], [other], step=7, lr=0.1, seed=3)
        torch.cuda.synchronize()
        assert torch.equal(p, q) and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(state, other))


def test_the_binding_refuses():
    P = _api()
    p = torch.zeros(300, device="cuda")
    s = P.adamw_state(p)
    s8 = P.adamw_state(p, 8)
    ok = dict(step=1, lr=0.1)
    for call in (lambda: P.adamw_step([p], [], [s], **ok), lambda: P.adamw_step([p], [p[:4]], [s], **ok), lambda: P.adamw_step([p], [p.double()], [s], **ok),
                 lambda: P.adamw_step([p, p], [p, p], [s, s8], **ok), lambda: P.adamw_step([p], [p], [s[:1] + (p[:3],)], **ok),
                 lambda: P.adamw_step([p], [p], [s8[:2] + (p[:1], p[:1])], **ok), lambda: P.adamw_step([p], [p], [(s8[0], s8[1])], **ok),
                 lambda: P.adamw_step([p[::2]], [p[::2]], [(p[:150], p[:150])], **ok), lambda: P.adamw_step([p], [p], [s], step=0, lr=0.1),
                 lambda: P.adamw_step([p], [p], [s], step=1, lr=float("nan")), lambda: P.adamw_step([p], [p], [s], weight_decay=[0.1, 0.2], **ok),
                 lambda: P.adamw_step([p], [p], [s], copies=[p[:5]], **ok), lambda: P.adamw_step([p], [p.cpu()], [s], **ok),
                 lambda: P.adamw_step([p], [p], [s], grad_scale=p, **ok)):
        with pytest.raises(P.DynLPError):
            call()
