"""Scores of rows and of the head against the definitions in 64 bits.

Bars, u = 2^-24.  A row's sums are made by 64 lanes at least and then joined: n = 2 ceil(C / 64) + 64 roundings each (a sum is rescaled when a
larger value comes).  s is off by n u and what rounding the exponents x - m does, u sum p |x - m|; log p by that, 3 u (|x - m| + |log s|) and its own rounding.
Entropy log s - t / s: the same for log s, and for t the n u and the exponents' rounding of sum p |x - m| (1 + |x - m|).  Of probabilities, log x stands for x - m, and is off by 2 u of
itself.  Logits of the head are off by (D + 3) u (sum |h||W| + |b|), of heads in 32 bits, whose products are made of six of 16 bits, by (6 D + 8) u of it, which
moves log p by up to twice the row's largest and the entropy by that times 2 + 2 max |log p|."""
import numpy as np
import pytest

from oracle import student as S
from rounding import hold

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
U = 2.0 ** -24


def _api():
    import paper_2604_06596_amd as P

    return P


def _bars(x, probabilities):
    """Errors of log probabilities [N, C] and entropy [N] of finite rows."""
    x = np.asarray(x, dtype=np.float64)
    n = 2 * -(-x.shape[1] // 64) + 64
    with np.errstate(divide="ignore", invalid="ignore"):
        z = np.log(x) if probabilities else x
        log_p = S.scores(x, probabilities)[0]
        p = np.exp(log_p)
        d = np.abs(z) if probabilities else np.abs(z - z.max(axis=1, keepdims=True))
        d0 = np.where(p == 0.0, 0.0, np.where(np.isfinite(d), d, 0.0))
        log_s = np.abs(np.log(x.sum(axis=1, keepdims=True))) if probabilities else np.abs(np.max(log_p, axis=1, keepdims=True))
        mean = (p * d0).sum(axis=1, keepdims=True)
        s = n * U + U * mean
        log_bar = s + 3 * U * (d0 + log_s) + 2 * U * np.where(np.isfinite(log_p), np.abs(log_p), 0.0) + 2.0 ** -140
        entropy = s[:, 0] + 4 * U * log_s[:, 0] + n * U * (1 + 2 * mean[:, 0]) + 4 * U * (p * d0 * (1 + d0)).sum(axis=1) + 2.0 ** -140
    return log_bar, entropy


def _check(out, x, probabilities, given, top, log_bar=None, entropy_bar=None):
    log_p, entropy, order = S.scores(x, probabilities)
    if log_bar is None:
        log_bar, entropy_bar = _bars(x, probabilities)
    rows = np.arange(len(x))[:, None]
    if out.entropy is not None:
        hold(out.entropy, entropy, entropy_bar, "entropy")
    if given is not None:
        real = (given >= 0) & (given < x.shape[1])
        at = np.where(real, given, 0)
        exact, bar = np.where(real, log_p[rows, at], 0.0), np.where(real, log_bar[rows, at], 0.0)
        _hold("log_given", out.log_given, exact, bar)
    if top:
        np.testing.assert_array_equal(out.top.cpu().numpy(), order[:, :top])
        _hold("log_top", out.log_top, log_p[rows, order[:, :top]], log_bar[rows, order[:, :top]])


def _hold(name, got, exact, bar):
    """-infinity has to be itself."""
    value = got.double().cpu().numpy()
    low = np.isneginf(exact)
    assert np.array_equal(np.isneginf(value), low), name
    if (~low).any():
        hold(torch.from_numpy(value[~low]).float(), exact[~low], bar[~low], name)


ROWS = [  # rows, classes, top, given
    (0, 5, 2, 1), (1, 1, 1, 1), (1, 2, 2, 0), (3, 2, 1, 5), (1, 1000, 5, 1), (5, 63, 63, 2), (4, 64, 64, 1), (7, 65, 64, 1), (300, 50, 4, 0), (129, 50, 9, 3),
    (2, 255, 128, 1), (3, 256, 100, 1), (5, 257, 7, 0), (33, 511, 32, 1), (2, 2049, 128, 1), (9, 4100, 16, 4), (3, 10007, 33, 1), (2, 100003, 32, 1),
    (1, 131072, 128, 1), (1025, 17, 17, 1), (2000, 8, 3, 1),
]


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16", "probabilities"])
@pytest.mark.parametrize("rows, classes, top, given", ROWS)
def test_rows(rows, classes, top, given, kind):
    P = _api()
    rng = np.random.default_rng(rows * 131 + classes)
    probabilities = kind == "probabilities"
    dtype = TYPES.get(kind, torch.float32)
    x = 3.0 * rng.standard_normal((rows, classes))
    if probabilities:
        x = np.exp(x - x.max(axis=1, keepdims=True, initial=-99.0))
        x /= x.sum(axis=1, keepdims=True)
        x[:, classes // 2:classes // 2 + classes // 5] = 0.0
    else:
        x[:, classes // 2:classes // 2 + classes // 5] = -np.inf
    wide = torch.zeros(max(rows, 1), classes + rows % 5, dtype=dtype, device="cuda")
    wide[:rows, :classes] = torch.from_numpy(x).to(dtype).cuda()
    t = wide[:rows, :classes]
    ids = rng.integers(-1, classes, size=(rows, given)).astype(np.int32) if given else None
    out = P.row_scores(t, given=None if ids is None else torch.from_numpy(ids).cuda(), top=top, probabilities=probabilities)
    _check(out, t.double().cpu().numpy(), probabilities, ids, top)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("pattern", ["equal", "rising", "falling", "few", "signs", "late"])
@pytest.mark.parametrize("classes", [5, 50, 64, 300, 5000, 40000])
def test_order(classes, pattern, kind):
    """Rows that make an order hard: equal values, rising ones, few different ones, zeros of both signs, all the large ones at the end."""
    P = _api()
    c = np.arange(classes)
    x = {"equal": np.zeros(classes), "rising": c / 64.0, "falling": -c / 64.0, "few": (c * 7 % 5).astype(float),
         "signs": np.where(c % 3 == 0, -0.0, np.where(c % 3 == 1, 0.0, -1.0)), "late": np.where(c > classes - 200, 5.0 + c % 7, -1.0)}[pattern]
    t = torch.from_numpy(np.stack([x, x[::-1]])).to(TYPES[kind]).cuda()
    top = min(classes, 128)
    out = P.row_scores(t, top=top)
    _check(out, t.double().cpu().numpy(), False, None, top)


@pytest.mark.parametrize("classes", [3, 50, 64, 65, 700, 9000])
def test_rows_without_numbers(classes):
    P = _api()
    x = np.random.default_rng(3).standard_normal((6, classes)).astype(np.float32)
    x[1] = -np.inf
    x[2, classes // 2] = np.nan
    x[3, classes - 1] = np.inf
    x[4] = np.nan
    x[5, 0] = -np.inf
    given = torch.zeros(6, dtype=torch.int32, device="cuda")
    out = P.row_scores(torch.from_numpy(x).cuda(), given=given, top=3)
    assert np.array_equal(np.isnan(out.entropy.cpu().numpy()), [False, False, True, True, True, False])
    assert np.isnan(out.log_top[2:5].cpu().numpy()).all() and np.isnan(out.log_given[2:5].cpu().numpy()).all()
    order = S.scores(x)[2][:, :3]
    assert np.array_equal(out.top.cpu().numpy(), order)
    uniform = torch.tensor(-np.log(classes)).float()
    assert torch.allclose(out.log_top[1].cpu(), uniform.expand(3), rtol=4 * U, atol=0) and abs(float(out.entropy[1]) - np.log(classes)) <= 4 * U * np.log(classes)
    assert float(out.log_given[5]) == -np.inf
    empty = P.row_scores(torch.zeros(2, classes, device="cuda"), top=2, probabilities=True)
    assert empty.top.tolist() == [[0, 1], [0, 1]] and torch.allclose(empty.log_top.cpu(), uniform.expand(2, 2), rtol=4 * U, atol=0)


def test_given_classes_that_are_not_there():
    P = _api()
    x = torch.randn(3, 20, device="cuda")
    given = torch.tensor([[0, 20, -1], [19, -5, 2 ** 31 - 1], [3, 21, -2 ** 31]], dtype=torch.int32, device="cuda")
    weight = torch.randn(20, 8, device="cuda")
    h = torch.randn(3, 8, device="cuda")
    for call in (lambda r: P.row_scores(x, given=given, rejected=r), lambda r: P.head_scores(h, weight, given=given, rejected=r)):
        rejected = torch.full((1,), 7, dtype=torch.int32, device="cuda")
        out = call(rejected)
        assert int(rejected) == 10
        assert (out.log_given[given.cpu() < 0] == 0).all() and (out.log_given[given.cpu() >= 20] == 0).all() and (out.log_given[:, 0] < 0).all()
    assert P.row_scores(x, given=given[:, 0].contiguous()).log_given.shape == (3,)
    assert P.row_scores(x, entropy=False) == (None, None, None, None)


HEADS = [  # rows, dim, classes, top, given
    (0, 8, 3, 1, 1), (1, 1, 1, 1, 1), (1, 64, 10, 3, 1), (2, 3, 2, 2, 0), (15, 33, 17, 5, 2), (16, 32, 64, 64, 1), (17, 64, 65, 10, 1), (63, 40, 300, 8, 1),
    (65, 96, 257, 128, 1), (64, 32, 256, 1, 1), (130, 200, 29, 3, 1), (300, 100, 1000, 16, 1), (257, 64, 50, 4, 0), (5, 1030, 70, 3, 7), (1000, 16, 129, 9, 1),
    (3, 256, 10007, 5, 1), (200, 48, 3001, 20, 1),
]


def _head(rng, rows, dim, classes, dtype, grid, stride=0, shift=0):
    """h, weight, bias on the GPU and in 64 bits; with a grid, every sum is exact in 32 bits."""
    def matrix(n, m, size, step):
        v = size * rng.standard_normal((n, m))
        v = np.round(v / step) * step if grid else v
        flat = torch.zeros(max(n, 1) * (m + stride) + shift, dtype=dtype, device="cuda")
        t = flat[shift:].view(max(n, 1), m + stride)[:n, :m]
        t.copy_(torch.from_numpy(v).to(dtype))
        return t, t.double().cpu().numpy()

    h, eh = matrix(rows, dim, 1.0, 1 / 8)
    W, eW = matrix(classes, dim, 2.0 / np.sqrt(dim), 1 / 256)
    b = (np.round(rng.standard_normal(classes) * 64) / 256).astype(np.float32)
    return h, W, torch.from_numpy(b).cuda(), eh, eW, b.astype(np.float64)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows, dim, classes, top, given", HEADS)
def test_head(rows, dim, classes, top, given, kind):
    """On a grid the logits are exact, and so is the order; without one the order is right up to the logits' error."""
    P = _api()
    rng = np.random.default_rng(rows + 7 * dim + classes)
    ids = rng.integers(-1, classes, size=(rows, given)).astype(np.int32) if given else None
    for grid in (True, False):
        h, W, b, eh, eW, eb = _head(rng, rows, dim, classes, TYPES[kind], grid, stride=rows % 3, shift=dim % 2)
        bias = b if rows % 2 else None
        out = P.head_scores(h, W, bias, given=None if ids is None else torch.from_numpy(ids).cuda(), top=top)
        z = eh @ eW.T + (0.0 if bias is None else eb)
        magnitude = np.abs(eh) @ np.abs(eW).T + (0.0 if bias is None else np.abs(eb))
        off = ((6 * dim + 8) if kind == "float32" else (dim + 3)) * U * magnitude.max(axis=1, initial=0.0)[:, None]
        log_bar, entropy_bar = _bars(z, False)
        if grid:
            _check(out, z, False, ids, top, log_bar, entropy_bar)
            continue
        log_p, entropy, order = S.scores(z)
        log_bar = log_bar + 2 * off
        hold(out.entropy, entropy, entropy_bar + off[:, 0] * (2 + 2 * np.abs(log_p).max(axis=1, initial=0.0)), "entropy")
        if not rows:
            continue
        got = out.top.cpu().numpy()
        at = np.arange(rows)[:, None]
        assert (np.sort(got, axis=1)[:, 1:] != np.sort(got, axis=1)[:, :-1]).all()
        assert (np.abs(z[at, got] - z[at, order[:, :top]]) <= 2 * off).all()
        hold(out.log_top, log_p[at, got], log_bar[at, got], "log_top")
        if given:
            hold(out.log_given, np.where(ids >= 0, log_p[at, np.maximum(ids, 0)], 0.0), np.where(ids >= 0, log_bar[at, np.maximum(ids, 0)], 0.0), "log_given")


def test_head_with_classes_that_are_shut():
    P = _api()
    rng = np.random.default_rng(5)
    h, W, b, eh, eW, eb = _head(rng, 40, 32, 300, torch.bfloat16, True)
    W[7] = float("nan")
    h[3] = float("inf")
    shut = np.zeros(300, bool)
    shut[[0, 7, 255, 256, 299]] = True
    b[torch.from_numpy(shut).cuda()] = -float("inf")
    out = P.head_scores(h, W, b, top=128)
    z = np.where(shut, -np.inf, eh @ np.where(np.isnan(eW), 0.0, eW).T + eb)
    fine = np.arange(40) != 3
    _check(type(out)(None, out.entropy[fine], out.top[fine], out.log_top[fine]), z[fine], False, None, 128)
    assert torch.isnan(out.entropy[3])
    all_shut = P.head_scores(h[:2], W, torch.full_like(b, -float("inf")), top=2)
    assert all_shut.top.tolist() == [[0, 1], [0, 1]] and torch.allclose(all_shut.log_top, torch.tensor(-np.log(300.0)).float().cuda(), rtol=4 * U, atol=0)


def test_large_and_tiny_values_in_32_bits():
    """Terms of values that rounding to bfloat16 would make infinite, and of those that have no third term."""
    P = _api()
    h = torch.tensor([[3.4028234e38, 1.0, 0.0], [1e-30, 2.0 ** -100, 1.0], [float("inf"), 0.0, 0.0]], device="cuda")
    W = torch.tensor([[1.0, 2.0, 3.0], [-1.0, 0.0, 1.0]], device="cuda")
    out = P.head_scores(h, W, top=2)
    assert out.top.tolist() == [[0, 1], [0, 1], [0, 1]]
    assert float(out.log_top[0, 0]) == 0.0 and float(out.log_top[0, 1]) < -1e38
    assert abs(float(out.log_top[1, 0]) + np.log1p(np.exp(-2.0))) < 1e-6
    assert torch.isnan(out.log_top[2]).all()


def test_many_rows_by_turns():
    """More logits than are in memory at a time: the turns meet at no row."""
    P = _api()
    rng = np.random.default_rng(1)
    h, W, b, *_ = _head(rng, 3000, 32, 40000, torch.bfloat16, True)
    out = P.head_scores(h, W, b, top=4)
    for at in (0, 1500, 1535, 1536, 1663, 1664, 1677, 1678, 2999):
        one = P.head_scores(h[at:at + 1], W, b, top=4)
        assert torch.equal(one.top[0], out.top[at]) and torch.allclose(one.log_top[0], out.log_top[at], rtol=1e-5)


def test_streams_and_graphs():
    P = _api()
    rng = np.random.default_rng(2)
    h, W, b, *_ = _head(rng, 100, 64, 1000, torch.bfloat16, True)
    given = torch.randint(0, 1000, (100,), dtype=torch.int32, device="cuda")
    want = P.head_scores(h, W, b, given=given, top=8)
    x = torch.randn(100, 1000, device="cuda")
    want_rows = P.row_scores(x, given=given, top=8)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = P.head_scores(h, W, b, given=given, top=8)
        got_rows = P.row_scores(x, given=given, top=8)
    torch.cuda.current_stream().wait_stream(stream)
    for a, c in zip((*want, *want_rows), (*got, *got_rows)):
        assert torch.equal(a, c)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = P.head_scores(h, W, b, given=given, top=8)
        got_rows = P.row_scores(x, given=given, top=8)
    for turn in range(3):
        h.copy_(h.roll(1, 0))
        x.mul_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip((*P.head_scores(h, W, b, given=given, top=8), *P.row_scores(x, given=given, top=8)), (*got, *got_rows)):
            assert torch.equal(a, c), turn


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16", "probabilities"])
@pytest.mark.parametrize("classes, top", [(1, 1), (5, 2), (29, 4), (50, 8), (63, 3), (64, 5), (64, 0)])
def test_many_short_rows(classes, top, kind):
    """So many that each has a lane: a row count that is no multiple of 64, rows with padding behind them, rows that have fewer numbers than classes asked for."""
    P = _api()
    g = torch.Generator(device="cuda").manual_seed(classes * 10 + top)
    rows = 1024 * 64 + 37
    dtype = TYPES.get(kind, torch.float32)
    probabilities = kind == "probabilities"
    x = 3.0 * torch.randn(rows, classes, generator=g, device="cuda")
    if probabilities:
        x = torch.softmax(x, 1)
        x[::7] = torch.nn.functional.one_hot(x[::7].argmax(1), classes).float()
    else:
        x[::5, classes // 2:] = -float("inf")
        x[3] = -float("inf")
        x[::11] = 1.0
    wide = torch.full((rows, classes + 3), 9.0, dtype=dtype, device="cuda")
    wide[:, :classes] = x.to(dtype)
    t = wide[:, :classes]
    given = torch.randint(-1, classes, (rows, 2), generator=g, device="cuda", dtype=torch.int32)
    out = P.row_scores(t, given=given, top=top, probabilities=probabilities)
    _check(out, t.double().cpu().numpy(), probabilities, given.cpu().numpy(), top)
    if not probabilities and classes > 2:
        odd = t[:rows].clone()
        odd[100, 1], odd[200, 0] = float("nan"), float("inf")
        got = P.row_scores(odd, top=top)
        assert torch.isnan(got.entropy[[100, 200]]).all()
        keep = torch.ones(rows, dtype=torch.bool, device="cuda")
        keep[[100, 200]] = False
        assert torch.equal(got.entropy[keep], P.row_scores(t.contiguous(), top=top).entropy[keep])
        if top:
            assert torch.isnan(got.log_top[[100, 200]]).all()
            assert np.array_equal(got.top[[100, 200]].cpu().numpy(), S.scores(odd[[100, 200]].double().cpu().numpy())[2][:, :top])
            assert torch.equal(got.top[keep], out.top[keep])


@pytest.mark.parametrize("lowest", [-3.4028234663852886e38, -1e30])
def test_masks_of_the_lowest_value(lowest):
    """Masked classes that hold the type's lowest value: nothing of them is left; where all are, they are equal."""
    P = _api()
    for classes in (7, 64, 300, 5000):
        x = torch.randn(3, classes, device="cuda")
        x[0, ::2] = lowest
        x[1] = lowest
        out = P.row_scores(x, top=2)
        _check(out, x.double().cpu().numpy(), False, None, 2)
        h, W = torch.zeros(3, 8, device="cuda"), torch.zeros(classes, 8, device="cuda")
        b = torch.where(torch.arange(classes, device="cuda") % 2 == 0, torch.full((classes,), lowest, device="cuda"), torch.randn(classes, device="cuda"))
        _check(P.head_scores(h, W, b, top=2), b.double().cpu().numpy()[None].repeat(3, 0), False, None, 2)


@pytest.mark.parametrize("rows, dim, classes", [(20, 40, 100000), (3, 64, 600000), (70, 33, 1100000)])
def test_heads_of_many_classes(rows, dim, classes):
    """Groups of groups, and more of them than 64 lanes hold at a time."""
    P = _api()
    rng = np.random.default_rng(classes)
    h, W, b, eh, eW, eb = _head(rng, rows, dim, classes, torch.bfloat16, True)
    given = rng.integers(0, classes, size=(rows, 3)).astype(np.int32)
    out = P.head_scores(h, W, b, given=torch.from_numpy(given).cuda(), top=100)
    z = eh @ eW.T + eb
    _check(out, z, False, given, 100)
