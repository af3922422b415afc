"""Learning from a teacher's first classes where the numbers themselves are hard.  Bars as in test_gpu_distill."""
import numpy as np
import pytest

from oracle import student as S
from rounding import hold
from test_gpu_distill import _bars, _lists, _run
from test_gpu_scores import TYPES, U, _api, _head

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows, classes", [(5, 10), (40, 64), (5, 100), (300, 400)])
def test_a_class_that_is_named_twice_is_one_class(rows, classes, kind):
    """The loss is a divergence of distributions over classes: of [c, c] it is that of [c], whichever logits share its probability; nothing where the head is certain of c."""
    P = _api()
    rng = np.random.default_rng(rows)
    h, W, b, eh, eW, eb = _head(rng, rows, 32, classes, TYPES[kind], False)
    y = rng.integers(0, classes, size=(rows, 1)).astype(np.int32)
    for kept in (2, 5, 33):
        u = rng.standard_normal((rows, kept)).astype(np.float32)
        many = np.repeat(y, kept, axis=1)
        got = _run(P, h, W, b, many, u)
        ref = S.distill(eh, eW, eb, y, u[:, :1])
        bars = _bars(ref, eh, eW, eb, np.ones(rows), 1.0, 1.0, kind, "float32", u)
        for name, value in zip(("loss", "dh", "dweight", "dbias"), got):
            hold(value, ref[name], bars[name], name)
        # two classes, the first of them several times: its probabilities' sum
        other = np.concatenate([many, (y + 1) % classes], axis=1)
        v = np.concatenate([u, rng.standard_normal((rows, 1)).astype(np.float32)], axis=1)
        both = np.concatenate([np.log(np.exp(v[:, :-1].astype(np.float64)).sum(axis=1, keepdims=True)), v[:, -1:]], axis=1)
        got = _run(P, h, W, b, other, v)
        ref = S.distill(eh, eW, eb, np.concatenate([y, (y + 1) % classes], axis=1), both)
        bars = _bars(ref, eh, eW, eb, np.ones(rows), 1.0, 1.0, kind, "float32", v)
        for name, value in zip(("loss", "dh", "dweight", "dbias"), got):
            hold(value, ref[name], bars[name], name)
    sure = torch.full((classes,), -float("inf"), device="cuda")
    sure[1] = 0.0
    one = torch.ones(rows, 2, dtype=torch.int32, device="cuda")
    loss = P.head_distill(torch.zeros_like(h), W, sure, one, torch.randn(rows, 2, device="cuda"))[0]
    assert float(loss.abs().max()) <= 4 * U


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("classes", [50, 100, 700])
@pytest.mark.parametrize("size", [1e3, 1e5, 1e7])
def test_logits_that_share_a_large_part(size, classes, kind):
    """Logits on a grid far from zero, exact in 32 bits: the softmax is that of their differences, whose size d is all that it is rounded at.  p is off by (C + 64) u + 4 u d
    of itself, the loss by T^2 (C + K + 64) u (1 + d + log C)."""
    P = _api()
    rng = np.random.default_rng(classes)
    rows, kept = 70, 3
    h, W, b, eh, eW, eb = _head(rng, rows, 32, classes, TYPES[kind], True)
    h.copy_((h * 8).round().clamp(-2, 2))  # integers: the logits' differences are, too
    W.copy_((W * 8).round().clamp(-3, 3))
    eh, eW = h.double().cpu().numpy(), W.double().cpu().numpy()
    for equal in (True, False):
        if equal:
            h.zero_()
            eb = np.full(classes, size)
        else:
            h.copy_(torch.from_numpy(eh))
            eb = size + rng.integers(-3, 3, size=classes)
        b.copy_(torch.from_numpy(eb))
        at, u = _lists(rng, rows, classes, kept, pad=False)
        for temperature in (1.0, 2.0):
            loss, dh, dweight, dbias = _run(P, h, W, b, at, u, temperature=temperature)
            ref = S.distill(np.zeros_like(eh) if equal else eh, eW, eb, at, u, temperature)
            z = ref["logits"]
            d = (z.max(axis=1) - z.min(axis=1)).max()
            spread = float(u.max() - u.min()) / temperature
            p, q = ref["soft"], ref["target"]
            dp = temperature * (p * ((classes + 64) * U + 4 * U * (d + np.log(classes))) + q * ((kept + 16 + 2 * spread) * U)) + 4 * U * np.abs(ref["dz"])
            hold(dbias, ref["dbias"], (dp + (rows + 64) * U * np.abs(ref["dz"])).sum(axis=0), "dbias")
            hold(loss, ref["loss"], temperature ** 2 * (classes + kept + 64) * U * (1 + d + spread + np.log(classes)) * np.ones(rows), "loss")


@pytest.mark.parametrize("rows, dim, classes", [(40, 64, 200), (300, 64, 130000)])
def test_rows_of_little_weight_in_16_bits(rows, dim, classes):
    """A row's dh is as exact as with a call to itself.  Weights that are powers of two change no digit of what it is made from: dh is that of weights of 1 times them, wherever
    float16 holds both without loss."""
    P = _api()
    rng = np.random.default_rng(rows)
    h, W, b, eh, eW, eb = _head(rng, rows, dim, classes, torch.float16, False)
    at, u = _lists(rng, rows, classes, 3, pad=False)
    r = 2.0 ** -torch.from_numpy(rng.integers(0, 25, size=rows)).cuda().float()
    r[3] = 1.0
    for grad in (torch.float16, torch.float32):
        want = _run(P, h, W, b, at, u, grad_scale=8192.0, dtype=grad)[1].float() * r[:, None]
        got = _run(P, h, W, b, at, u, grad_scale=8192.0, dtype=grad, row_weight=r)[1].float()
        normal = want.abs() >= 2.0 ** -14
        assert float(normal.float().mean()) > 0.5
        assert torch.equal(got[normal], want[normal])


@pytest.mark.parametrize("rows", [40, 200])
def test_sums_over_rows_of_all_weights_in_16_bits(rows):
    """dweight and dbias beside the largest weight: what float16 terms leave out is 2^-22 of dz and 2^-39 of that weight."""
    P = _api()
    rng = np.random.default_rng(rows)
    h, W, b, eh, eW, eb = _head(rng, rows, 64, 200, torch.float16, False)
    at, u = _lists(rng, rows, 200, 3, pad=False)
    r = (2.0 ** -rng.integers(0, 25, size=rows) * rng.random(rows)).astype(np.float32)
    for grad in ("float16", "float32"):
        got = _run(P, h, W, b, at, u, row_weight=torch.from_numpy(r).cuda(), grad_scale=4096.0, dtype=TYPES[grad])
        ref = S.distill(eh, eW, eb, at, u, 1.0, r, 4096.0)
        bars = _bars(ref, eh, eW, eb, r.astype(np.float64), 1.0, 4096.0, "float32", "float32", u)
        dz = np.abs(ref["dz"])
        weight = 4096.0 * r.astype(np.float64)[:, None]
        for name, value, more in (("loss", got[0], 0.0), ("dh", got[1], (2.0 ** -22 * dz + 2.0 ** -39 * weight) @ np.abs(eW)),
                                  ("dweight", got[2], (2.0 ** -22 * dz + np.where(dz > 0, 2.0 ** -39 * weight.max(), 0.0)).T @ np.abs(eh)), ("dbias", got[3], 0.0)):
            hold(value, ref[name], bars[name] + more, name)


def test_the_largest_number_of_classes():
    """2^22 classes, whose tiles' counts alone take 64 KB of shared memory.  Sums of the softmax: 2,114 roundings one after the other at most (32 values of a lane, two joins of lanes,
    65,536 parts by 32 threads and those joined), n u of it; products over classes: 131,072 steps, whose roundings are 2^-7 of the sum of magnitudes; dz in two terms."""
    P = _api()
    rows, dim, classes, kept = 20, 32, 1 << 22, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.randn(rows, dim, generator=g, device="cuda").to(torch.bfloat16)
    W = (0.3 * torch.randn(classes, dim, generator=g, device="cuda")).to(torch.bfloat16)
    at = torch.randint(0, classes, (rows, kept), generator=g, device="cuda", dtype=torch.int32)
    at[0] = torch.tensor([classes - 1, 0, classes], dtype=torch.int32)
    u = torch.randn(rows, kept, generator=g, device="cuda")
    rejected = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, dh, dweight, dbias = P.head_distill(h, W, None, at, u, rejected=rejected)
    assert int(rejected) == 1
    u = torch.where(at < classes, u, -float("inf")).double()
    q = torch.softmax(u, 1)
    z = h.double() @ W.double().t()
    lse = torch.logsumexp(z, 1, keepdim=True)
    picked = z.gather(1, at.long().clamp(max=classes - 1))
    want = torch.where(q > 0, q * (q.log() - picked + lse), 0.0).sum(1)
    n = 2114 * U
    assert ((loss.double() - want).abs() <= n + 64 * U * 20).all()
    p = z.sub_(lse).exp_()
    sums = p.sum(0)
    dz = p.scatter_add_(1, at.long().clamp(max=classes - 1), -q)
    want = dz.sum(0)
    assert ((dbias.double() - want).abs() <= (2 * n + 128 * U) * sums + 64 * U * dz.abs().sum(0)).all()
    want = dz @ W.double()
    assert ((dh.double() - want).abs() <= (2.0 ** -7 + n) * (dz.abs() @ W.double().abs()) + 2.0 ** -8 * want.abs()).all()
    want = dz.t().contiguous() @ h.double()
    bar = (2 * n + 2.0 ** -16) * (dz.abs().t().contiguous() @ h.double().abs())
    assert ((dweight.double() - want).abs() <= bar + U * want.abs()).all()


@pytest.mark.parametrize("classes", [10, 64, 70, 300])
def test_lists_with_what_is_no_number(classes):
    """All of the row's gradients are none then, whatever the head's size."""
    P = _api()
    rng = np.random.default_rng(classes)
    h, W, b, eh, eW, eb = _head(rng, 20, 16, classes, torch.float32, False)
    for bad in (np.nan, np.inf):
        at, u = _lists(rng, 20, classes, 3, pad=False)
        u[4, 1] = bad
        loss, dh, dweight, dbias = _run(P, h, W, b, at, u)
        keep = np.arange(20) != 4
        assert torch.isnan(loss[4]) and torch.isnan(dh[4]).all() and torch.isnan(dweight).all() and torch.isnan(dbias).all()
        assert torch.isfinite(loss[keep]).all() and torch.isfinite(dh[keep]).all()


@pytest.mark.filterwarnings("ignore::RuntimeWarning")  # bars of gradients, which are not looked at
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("classes", [50, 100])
@pytest.mark.parametrize("temperature", [1e-15, 1e-21, 1e-25, 1e-30])
def test_losses_at_small_temperatures(temperature, classes, kind):
    """T^2 leaves 32 bits long before T^2 times the divergence does, which is then about T times a difference of logits."""
    P = _api()
    rng = np.random.default_rng(classes)
    h, W, b, eh, eW, eb = _head(rng, 30, 32, classes, TYPES[kind], False)
    at, u = _lists(rng, 30, classes, 4, pad=False)
    temperature = float(np.float32(temperature))
    loss = _run(P, h, W, b, at, u, temperature=temperature, grads=False)[0]
    ref = S.distill(eh, eW, eb, at, u, temperature)
    bars = _bars(ref, eh, eW, eb, np.ones(30), temperature, 1.0, kind, "float32", u)
    hold(loss, ref["loss"], bars["loss"] - 2.0 ** -140 + 2.0 ** -149, "loss")


@pytest.mark.parametrize("rows", [3, 20, 150])
def test_large_and_tiny_values_of_wide_heads(rows):
    """Operands in 32 bits become bfloat16 terms: values that rounding to bfloat16 would make infinite, and those that have no second or third term."""
    P = _api()
    classes = 80
    h = torch.zeros(rows, 3, device="cuda")
    W = torch.zeros(classes, 3, device="cuda")
    h[0] = torch.tensor([3.4028234e38, 1.0, 0.0])
    h[1] = torch.tensor([1e-30, 2.0 ** -100, 1.0])
    h[2] = torch.tensor([2.0 ** -60, 1.0 + 2.0 ** -20, 3.0])
    W[:2] = torch.tensor([[1.0, 2.0, 3.0], [-1.0, 0.0, 1.0]])
    b = torch.full((classes,), -100.0, device="cuda")
    b[:2] = 0.0
    at, u = np.ones((rows, 1), dtype=np.int32), np.zeros((rows, 1), dtype=np.float32)
    r = np.ones(rows, dtype=np.float32)
    r[0] = 0.0
    got = _run(P, h, W, b, at, u, row_weight=torch.from_numpy(r).cuda())
    eh, eW, eb = (x.double().cpu().numpy() for x in (h, W, b))
    ref = S.distill(eh, eW, eb, at, u, 1.0, r)
    # the power of two of a logit 87 to 104 below the largest, a denormal number, is 0: each p is off by 2^-126, of up to `rows` and `classes`, times 3 at most of h or W
    below = 2.0 ** -126 * rows * classes * 3
    bars = _bars(ref, eh, eW, eb, r.astype(np.float64), 1.0, 1.0, "float32", "float32", u)
    for name, value in zip(("loss", "dh", "dweight", "dbias"), got):
        hold(value, ref[name], bars[name] + below, name)
    # the row of the large value alone: the head is certain of class 0, and its loss is beyond 32 bits
    r[:] = 0.0
    r[0] = 1.0
    loss, dh, dweight, dbias = _run(P, h, W, b, at, u, row_weight=torch.from_numpy(r).cuda())
    assert float(loss[0]) == float("inf") and dh[0].tolist() == [2.0, 2.0, 2.0] and dbias[:3].tolist() == [1.0, -1.0, 0.0]
    assert torch.equal(dweight[0], h[0]) and torch.equal(dweight[1], -h[0]) and (dweight[2:] == 0).all() and (dh[1:] == 0).all() and (loss[1:] == 0).all()


@pytest.mark.parametrize("kind, grad, rows", [("float16", "float16", 16001), ("float16", "float32", 16001), ("bfloat16", "float32", 16001), ("float32", "float32", 11003)])
def test_turns_of_all_types(kind, grad, rows):
    """More of dz than is in memory at a time (4 GiB), a shorter last turn: rows are those of calls that are done at once, sums over rows the sum of theirs.  Weights of
    the first half are far below those of the second, so that the turns' powers of two differ."""
    P = _api()
    classes, dim, kept = 70000, 32, 3
    g = torch.Generator(device="cuda").manual_seed(rows)
    dtype = TYPES[kind]
    h = torch.randn(rows, dim, generator=g, device="cuda").to(dtype)
    W = (0.3 * torch.randn(classes, dim, generator=g, device="cuda")).to(dtype)
    b = torch.randn(classes, generator=g, device="cuda")
    at = torch.randint(-1, classes + 1, (rows, kept), generator=g, device="cuda", dtype=torch.int32)
    u = torch.randn(rows, kept, generator=g, device="cuda")
    r = torch.rand(rows, generator=g, device="cuda") + 0.5
    r[torch.rand(rows, generator=g, device="cuda") < 0.1] = 0.0
    r[:rows // 2] *= 2.0 ** -9
    rejected = torch.zeros(1, dtype=torch.int32, device="cuda")
    loss, dh, dweight, dbias = P.head_distill(h, W, b, at, u, row_weight=r, grad_scale=64.0, dtype=TYPES[grad], rejected=rejected)
    assert int(rejected) == int((at == classes).sum())
    third = -(-rows // 3)
    parts = [P.head_distill(h[s], W, b, at[s], u[s], row_weight=r[s], grad_scale=64.0, dtype=torch.float32) for s in (slice(k, min(k + third, rows)) for k in range(0, rows, third))]
    assert torch.equal(loss, torch.cat([x[0] for x in parts]))
    # the same dz in the same terms; the order of its sums, of up to 70,000 products with |W| up to 1.5, is what the tiles give: 2^-16 of the row's weight beside a rounding
    want = torch.cat([x[1] for x in parts]).double()
    step = {"float32": U, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
    assert ((dh.double() - want).abs() <= 2 * step[kind] * want.abs() + 2.0 ** -15 * 64.0 * r[:, None] + 2.0 ** -24).all()
    assert (dh[r == 0] == 0).all()
    for got, want, error in ((dweight.double(), sum(x[2].double() for x in parts), step[grad] + (2.0 ** -16 if grad == "float32" else step[kind])),
                             (dbias.double(), sum(x[3].double() for x in parts), 2.0 ** -16)):
        assert float((got - want).norm() / want.norm()) <= error


@pytest.mark.parametrize("kind", list(TYPES))
def test_calls_on_two_streams_at_once(kind):
    """Each with a workspace of its own, over and over, none waiting for the other: the same bits as alone."""
    P = _api()
    rng = np.random.default_rng(12)
    sets = []
    for rows, classes in ((700, 1500), (90, 5000)):
        h, W, b, *_ = _head(rng, rows, 64, classes, TYPES[kind], False)
        at, u = (torch.from_numpy(x).cuda() for x in _lists(rng, rows, classes, 8))
        sets.append((h, W, b, at, u))
    call = lambda s: (*P.head_distill(*s), *P.head_scores(*s[:3], given=s[3], top=9), *P.row_scores(s[4], top=3)[1:])  # noqa: E731
    want = [call(s) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = []
    for _ in range(8):
        for s, stream in zip(sets, streams):
            with torch.cuda.stream(stream):
                got.append(call(s))
    torch.cuda.synchronize()
    for k, outs in enumerate(got):
        for a, c in zip(outs, want[k % 2]):
            assert torch.equal(a, c), k


@pytest.mark.parametrize("kind", list(TYPES))
def test_a_batch_with_padding(kind):
    """A buffer of more rows than there are: rows behind the last one, whose lists are empty or whose weight is 0, change nothing, whatever they hold."""
    P = _api()
    rng = np.random.default_rng(13)
    for rows, classes in ((45, 30), (45, 90), (300, 1000)):
        h, W, b, eh, eW, eb = _head(rng, rows, 48, classes, TYPES[kind], False)
        at, u = _lists(rng, rows, classes, 4, pad=False)
        r = rng.random(rows).astype(np.float32) + 0.5
        ref = S.distill(eh, eW, eb, at, u, 1.0, r)
        bars = _bars(ref, eh, eW, eb, r.astype(np.float64), 1.0, 1.0, kind, "float32", u)
        more = 83
        big = torch.full((rows + more, 48), float("nan"), dtype=TYPES[kind], device="cuda")
        big[:rows] = h
        at = np.concatenate([at, np.full((more, 4), -1, dtype=np.int32)])
        at[rows + 40:] = 3
        u = np.concatenate([u, np.full((more, 4), np.nan, dtype=np.float32)])
        r = np.concatenate([r, np.ones(more, dtype=np.float32)])
        r[rows + 40:] = 0.0
        loss, dh, dweight, dbias = _run(P, big, W, b, at, u, row_weight=torch.from_numpy(r).cuda())
        assert (loss[rows:] == 0).all() and (dh[rows:] == 0).all()
        for name, value in (("loss", loss[:rows]), ("dh", dh[:rows]), ("dweight", dweight), ("dbias", dbias)):
            hold(value, ref[name], bars[name], name)


@pytest.mark.parametrize("rows, dim, classes", [(100, 32, 300), (300, 40, 200000)])
def test_float16_gradients_one_at_a_time(rows, dim, classes):
    """dh has terms of its own there: each gradient by itself is what it is with the others, in one term and in two."""
    from paper_2604_06596_amd import train as T

    P = _api()
    rng = np.random.default_rng(14)
    L = T._library()
    h, W, b, *_ = _head(rng, rows, dim, classes, torch.float16, False)
    at, u = (torch.from_numpy(x).cuda() for x in _lists(rng, rows, classes, 4))
    r = 2.0 ** -torch.from_numpy(rng.integers(0, 12, size=rows)).cuda().float()
    m, w = T._matrix(h, "h", h.device), T._matrix(W, "W", h.device)
    t = T._Teacher(at.data_ptr(), u.data_ptr(), r.data_ptr(), None, 4, 1.0, 512.0)
    for dtype in (torch.float16, torch.float32):
        _, dh, dweight, dbias = P.head_distill(h, W, b, at, u, row_weight=r, grad_scale=512.0, dtype=dtype)
        outs = [torch.full((rows + 1, dim), 7.0, dtype=torch.float16, device="cuda"), torch.full((classes + 1, dim), 7.0, dtype=dtype, device="cuda"),
                torch.full((classes + 1,), 7.0, device="cuda")]
        for which in range(3):
            grad = T._TYPES[dtype]
            call, space = T._call(h.device, L.dynlp_head_distill_workspace(rows, dim, classes, 4, m.type, grad))
            T._check(L.dynlp_head_distill(m, w, b.data_ptr(), t, None, T._Matrix(outs[0].data_ptr(), rows, dim, dim, m.type) if which == 0 else None,
                                          T._Matrix(outs[1].data_ptr(), classes, dim, dim, grad) if which == 1 else None, outs[2].data_ptr() if which == 2 else None, call))
            value, want = outs[which], (dh, dweight, dbias)[which]
            assert torch.equal(value[:-1], want) and (value[-1] == 7).all()


@pytest.mark.parametrize("kind", ["bfloat16", "float32"])
def test_rows_that_lie_far_apart(kind):
    """Strides of more than 2^22 elements, of inputs and outputs: offsets within a tile of rows pass 32 bits."""
    from paper_2604_06596_amd import train as T

    P = _api()
    rng = np.random.default_rng(15)
    rows, dim, classes, stride = 140, 64, 90, (1 << 22) + (1 << 20) + 8
    h, W, b, *_ = _head(rng, rows, dim, classes, TYPES[kind], False)
    at, u = (torch.from_numpy(x).cuda() for x in _lists(rng, rows, classes, 4))
    want = P.head_distill(h, W, b, at, u, dtype=TYPES[kind])
    scores = P.head_scores(h, W, b, top=5)
    far = torch.zeros(rows * stride, dtype=TYPES[kind], device="cuda").view(rows, stride)
    far_h, far_w = far[:, :dim], far[:classes, dim:2 * dim]
    far_h.copy_(h)
    far_w.copy_(W)
    got = P.head_distill(far_h, far_w, b, at, u, dtype=TYPES[kind])
    for a, c in zip(want, got):
        assert torch.equal(a, c)
    for a, c in zip(scores[1:], P.head_scores(far_h, far_w, b, top=5)[1:]):
        assert torch.equal(a, c)
    for a, c in zip(P.row_scores(h, top=5)[1:], P.row_scores(far_h, top=5)[1:]):
        assert torch.equal(a, c)
    # outputs there, too
    L = T._library()
    m = T._matrix(far_h, "h", h.device)
    out_h, out_w = far[:, 2 * dim:3 * dim], far[:classes, 3 * dim:4 * dim]
    call, space = T._call(h.device, L.dynlp_head_distill_workspace(rows, dim, classes, 4, m.type, m.type))
    t = T._Teacher(at.data_ptr(), u.data_ptr(), None, None, 4, 1.0, 1.0)
    T._check(L.dynlp_head_distill(m, T._matrix(far_w, "weight", h.device), b.data_ptr(), t, None, T._matrix(out_h, "dh", h.device), T._matrix(out_w, "dweight", h.device), None, call))
    assert torch.equal(out_h, want[1]) and torch.equal(out_w, want[2])
    assert (far[:, 4 * dim:] == 0).all() and (far[classes:, 3 * dim:4 * dim] == 0).all()


@pytest.mark.parametrize("kind, grad", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32")])
@pytest.mark.parametrize("rows, dim, classes", [(1, 1, 65), (18, 1, 66), (33, 2, 200), (260, 31, 70), (20, 65, 4097)])
def test_heads_of_few_columns(rows, dim, classes, kind, grad):
    P = _api()
    rng = np.random.default_rng(rows + dim)
    h, W, b, eh, eW, eb = _head(rng, rows, dim, classes, TYPES[kind], False)
    at, u = _lists(rng, rows, classes, 3)
    got = _run(P, h, W, b, at, u, dtype=TYPES[grad])
    ref = S.distill(eh, eW, eb, at, u)
    bars = _bars(ref, eh, eW, eb, np.ones(rows), 1.0, 1.0, kind, grad, u)
    for name, value in zip(("loss", "dh", "dweight", "dbias"), got):
        hold(value, ref[name], bars[name], name)
