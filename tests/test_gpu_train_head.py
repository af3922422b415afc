"""The class head, its loss and gradients against the definitions in 64 bits.

Bars, u = 2^-24.  A logit is a float32 sum of D products and a bias: off by at most dz = (D + 3) u (sum |h||W| + |b|).  Probabilities:
exp and the division add a few u, the sum of C of them C u: |dp| <= p (exp(2 dz) - 1 + (C + 16) u), dz the row's largest.  The loss is a sum over
classes of q (lse - z): r sum q (2 dz + (C + 16) u (1 + |lse - z|)).  dz = g r (S p - q): g r (S |dp| + 4 u (S p + q)); sums over classes (dh) and rows
(dweight, dbias) carry those and (terms + 4) u of their magnitudes; dh in bfloat16 works with dz to 2^-16 of it; all of which is then rounded to the result's type."""
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


def _matrix(rng, rows, dim, dtype, size=1.0, stride=None):
    t = torch.zeros(max(rows, 1), stride or dim, dtype=dtype, device="cuda")
    t[:rows, :dim] = torch.from_numpy(size * rng.standard_normal((rows, dim))).to(dtype).cuda()
    t = t[:rows, :dim]
    return t, t.double().cpu().numpy()


def _bars(h, W, b, ref, r, grad_scale):
    """Largest errors of logits' rows, soft labels, loss, dz, dh, dweight, dbias."""
    n, classes = len(h), len(W)
    h, W = np.where(np.isfinite(h), h, 0.0), np.asarray(W)
    z = (h.shape[1] + 3) * U * (np.abs(h) @ np.abs(W).T + (0.0 if b is None else np.where(np.isfinite(b), np.abs(b), 0.0)))
    row = z.max(axis=1, initial=0.0)
    p, q = ref["soft"], ref["target"]
    total = np.abs(q.sum(axis=1, keepdims=True))
    dp = p * (np.exp(2 * row)[:, None] - 1 + (classes + 16) * U) + 2.0 ** -140
    finite = np.where(q != 0, ref["logits"], 0.0)
    lse = np.log(np.exp(ref["logits"] - ref["logits"].max(axis=1, keepdims=True)).sum(axis=1)) + ref["logits"].max(axis=1)
    loss = np.abs(r) * (np.abs(q) * (2 * row[:, None] + (classes + 16) * U * (1 + np.abs(lse[:, None] - finite)))).sum(axis=1)
    scale = np.abs(grad_scale * r)[:, None]
    ddz = scale * (total * dp + 4 * U * (total * p + np.abs(q)) + (classes + 4) * U * np.abs(q).sum(axis=1, keepdims=True) * p) + 2.0 ** -140
    ddz[ref["left_out"]] = 0.0
    dz = np.abs(ref["dz"])
    dh = (ddz + ((classes + 4) * U + 2.0 ** -16) * dz) @ np.abs(W)
    dweight = (ddz + (n + 4) * U * dz).T @ np.where(ref["left_out"][:, None], 0.0, np.abs(h)) + 2.0 ** -140
    dbias = (ddz + (n + 4) * U * dz).sum(axis=0)
    return {"soft": dp, "loss": loss + 2.0 ** -140, "dh": dh, "dweight": dweight, "dbias": dbias}


def _hold(name, got, exact, bar):
    hold(got, exact, bar, name)


SHAPES = [  # rows, dim, classes
    (0, 8, 3), (1, 64, 10), (1, 1, 1), (2, 3, 2), (15, 8, 16), (16, 33, 17), (17, 64, 4), (31, 7, 31), (33, 100, 32), (127, 65, 33), (128, 128, 48),
    (129, 200, 29), (130, 257, 50), (257, 301, 64), (300, 16, 63), (1000, 1030, 20), (2000, 64, 10),
]


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows, dim, classes", SHAPES)
def test_answers(rows, dim, classes, kind):
    P = _api()
    rng = np.random.default_rng(rows + dim)
    h, eh = _matrix(rng, rows, dim, TYPES[kind], stride=dim + rows % 3)
    W, eW = _matrix(rng, classes, dim, TYPES[kind], 2.0 / np.sqrt(dim))
    b = rng.standard_normal(classes).astype(np.float32) if rows % 2 else None
    bias = None if b is None else torch.from_numpy(b).cuda()
    soft, hard = P.head_labels(h, W, bias)
    z, p, label = S.head(eh, eW, b)
    off = (dim + 3) * U * (np.abs(eh) @ np.abs(eW).T + (0.0 if b is None else np.abs(b)))
    _hold("soft", soft, p, p * (np.exp(2 * off.max(axis=1, initial=0.0))[:, None] - 1 + (classes + 16) * U) + 2.0 ** -140)
    ordered = np.sort(z, axis=1)
    clear = np.ones(rows, bool) if classes == 1 else ordered[:, -1] - ordered[:, -2] > 2 * off.max(axis=1, initial=0.0)
    assert np.array_equal(hard.cpu().numpy()[clear], label[clear]) and clear.sum() >= 0.9 * rows
    only, none = P.head_labels(h, W, bias, hard=False)
    assert none is None and torch.equal(only, soft)
    none, only = P.head_labels(h, W, bias, soft=False)
    assert none is None and torch.equal(only, hard)


def test_ties_go_to_the_lowest_class():
    P = _api()
    for classes in (2, 5, 16, 17, 40, 64):
        W = torch.ones(classes, 8, device="cuda")
        h = torch.ones(70, 8, device="cuda")
        soft, hard = P.head_labels(h, W)
        assert not hard.any()
        bias = torch.zeros(classes, device="cuda")
        bias[classes // 2:] = 1.0
        assert torch.equal(P.head_labels(h, W, bias)[1], torch.full((70,), classes // 2, dtype=torch.int32, device="cuda"))


def test_classes_that_are_masked_out():
    P = _api()
    rng = np.random.default_rng(2)
    for classes in (3, 20, 50):
        h, eh = _matrix(rng, 40, 24, torch.float32)
        W, eW = _matrix(rng, classes, 24, torch.float32)
        b = np.where(np.arange(classes) % 3 == 1, -np.inf, rng.standard_normal(classes)).astype(np.float32)
        soft, hard = P.head_labels(h, W, torch.from_numpy(b).cuda())
        _, p, label = S.head(eh, eW, b)
        assert np.all(soft.cpu().numpy()[:, np.isinf(b)] == 0.0) and np.array_equal(hard.cpu().numpy(), label)
        assert np.abs(soft.cpu().numpy() - p).max() <= np.exp(2 * 27 * U * (np.abs(eh) @ np.abs(eW).T + 4).max()) - 1 + (classes + 16) * U
        lowest = torch.where(torch.from_numpy(np.isinf(b)).cuda(), torch.finfo(torch.float32).min, torch.from_numpy(b).cuda())
        assert torch.equal(P.head_labels(h, W, lowest)[0], soft)
        nothing = torch.full((classes,), -float("inf"), device="cuda")
        soft, hard = P.head_labels(h, W, nothing)
        assert torch.equal(soft, torch.full_like(soft, 1.0 / classes)) and not hard.any()
        q = torch.full((40, classes), 1.0 / classes, device="cuda")
        for out in P.head_loss(h, W, nothing, q):
            assert not out.any()


def test_not_a_numbers_stay_in_their_rows():
    P = _api()
    rng = np.random.default_rng(3)
    h, _ = _matrix(rng, 100, 40, torch.float32)
    W, _ = _matrix(rng, 10, 40, torch.float32)
    clean = P.head_labels(h, W)
    h[37, 5] = float("nan")
    soft, hard = P.head_labels(h, W)
    assert torch.isnan(soft[37]).all() and 0 <= int(hard[37]) < 10
    keep = torch.arange(100, device="cuda") != 37
    assert torch.equal(soft[keep], clean[0][keep]) and torch.equal(hard[keep], clean[1][keep])


@pytest.mark.parametrize("targets", ["soft", "hard", "weighted"])
@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows, dim, classes", SHAPES)
def test_loss_and_gradients(rows, dim, classes, kind, targets):
    P = _api()
    rng = np.random.default_rng(7 * rows + dim)
    h, eh = _matrix(rng, rows, dim, TYPES[kind], stride=dim + rows % 5)
    W, eW = _matrix(rng, classes, dim, TYPES[kind], 2.0 / np.sqrt(dim), stride=dim + 1)
    b = rng.standard_normal(classes).astype(np.float32)
    soft = hard = r = None
    if targets == "hard":
        hard = rng.integers(-1, classes, rows).astype(np.int32)
    else:
        soft = rng.random((rows, classes)).astype(np.float32) * (rng.random((rows, classes)) < 0.7)
        soft = (soft / np.maximum(soft.sum(axis=1, keepdims=True), 1e-3) * (1.0 if targets == "soft" else 1.7)).astype(np.float32)
    if targets == "weighted":
        r = np.where(rng.random(rows) < 0.2, 0.0, 2.0 * rng.random(rows)).astype(np.float32)
        # what is left out is not looked at
        h[torch.from_numpy(r == 0).cuda()] = float("nan")
        soft[r == 0] = np.nan
    scale = 1.0 / max(rows, 1) if rows % 2 else 3.0
    ref = S.head_loss(eh, eW, b, soft, hard, r, float(np.float32(scale)))
    bars = _bars(eh, eW, b, ref, np.ones(rows) if r is None else r.astype(np.float64), scale)
    target = torch.from_numpy(soft if hard is None else hard).cuda()
    args = (h, W, torch.from_numpy(b).cuda(), target)
    kw = dict(row_weight=None if r is None else torch.from_numpy(r).cuda(), grad_scale=scale)
    got = dict(zip(("loss", "dh", "dweight", "dbias"), P.head_loss(*args, **kw)))
    for name, x in got.items():
        _hold(name, x, ref[name], bars[name])
    alone = P.head_loss(*args, **kw, grads=False)
    assert torch.equal(alone[0], got["loss"]) and alone[1:] == (None, None, None)
    again = P.head_loss(*args, **kw)
    assert all(torch.equal(x, y) for x, y in zip(got.values(), again))


def test_many_rows_and_their_splits():
    """Rows beyond what one set of workgroups takes in one go; the bars as above."""
    P = _api()
    rng = np.random.default_rng(11)
    for kind, dim, classes in (("float32", 50, 10), ("bfloat16", 136, 50), ("float16", 24, 29)):
        rows = 70001
        h, eh = _matrix(rng, rows, dim, TYPES[kind])
        W, eW = _matrix(rng, classes, dim, TYPES[kind], 2.0 / np.sqrt(dim))
        b = rng.standard_normal(classes).astype(np.float32)
        soft = rng.random((rows, classes)).astype(np.float32)
        soft /= soft.sum(axis=1, keepdims=True)
        ref = S.head_loss(eh, eW, b, soft, None, None, 1.0 / 65536)
        bars = _bars(eh, eW, b, ref, np.ones(rows), 1.0 / 65536)
        got = P.head_loss(h, W, torch.from_numpy(b).cuda(), torch.from_numpy(soft).cuda(), grad_scale=1.0 / 65536)
        for name, x in zip(("loss", "dh", "dweight", "dbias"), got):
            _hold(name, x, ref[name], bars[name])


@pytest.mark.parametrize("kind, rows, dim, classes", [("float32", 140001, 20, 17), ("bfloat16", 33001, 1000, 64), ("float16", 140001, 33, 29)])
def test_many_answers(kind, rows, dim, classes):
    """Rows enough for workgroups that keep a copy of W, of more than 64 KB too: the same as of a few rows at a time, which are held to the bars."""
    P = _api()
    rng = np.random.default_rng(rows)
    h, _ = _matrix(rng, rows, dim, TYPES[kind])
    W, _ = _matrix(rng, classes, dim, TYPES[kind], 2.0 / np.sqrt(dim))
    b = torch.from_numpy(rng.standard_normal(classes).astype(np.float32)).cuda()
    soft, hard = P.head_labels(h, W, b)
    for at in (0, 4097, rows // 2, rows - 300):
        few = P.head_labels(h[at:at + 300], W, b)
        assert torch.equal(few[0], soft[at:at + 300]) and torch.equal(few[1], hard[at:at + 300])


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows, dim, classes, stride", [(300, 520, 50, 520), (200, 700, 64, 701), (70, 512, 64, 512), (5, 40, 20, 1 << 22), (3, 24, 3, 1 << 23)])
def test_heads_that_do_not_fit_a_workgroup(rows, dim, classes, stride, kind):
    """More columns than one pass keeps, W larger than shared memory (64 x 512 float32), rows further apart than 32 bits hold a tile of."""
    P = _api()
    rng = np.random.default_rng(rows + dim)
    h, eh = _matrix(rng, rows, dim, TYPES[kind], stride=stride)
    W, eW = _matrix(rng, classes, dim, TYPES[kind], 2.0 / np.sqrt(dim))
    b = rng.standard_normal(classes).astype(np.float32)
    soft = rng.random((rows, classes)).astype(np.float32)
    r = np.where(rng.random(rows) < 0.3, 0.0, rng.random(rows)).astype(np.float32)
    ref = S.head_loss(eh, eW, b, soft, None, r, 0.5)
    bars = _bars(eh, eW, b, ref, r.astype(np.float64), 0.5)
    got = P.head_loss(h, W, torch.from_numpy(b).cuda(), torch.from_numpy(soft).cuda(), row_weight=torch.from_numpy(r).cuda(), grad_scale=0.5)
    for name, x in zip(("loss", "dh", "dweight", "dbias"), got):
        _hold(name, x, ref[name], bars[name])


def test_classes_out_of_range_leave_rows_out_and_are_counted():
    P = _api()
    rng = np.random.default_rng(12)
    h, eh = _matrix(rng, 90, 20, torch.float32)
    W, eW = _matrix(rng, 7, 20, torch.float32)
    hard = rng.integers(-2, 10, 90).astype(np.int32)
    rejected = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = P.head_loss(h, W, None, torch.from_numpy(hard).cuda(), rejected=rejected)
    assert int(rejected) == (hard >= 7).sum()
    ref = S.head_loss(eh, eW, None, None, hard)
    bars = _bars(eh, eW, None, ref, np.ones(90), 1.0)
    for name, x in zip(("loss", "dh", "dweight", "dbias"), got):
        _hold(name, x, ref[name], bars[name])


def test_gradients_against_differences():
    """Central differences of the loss in 64 bits, step 1e-4: off by its third derivative times 1e-9, with |h|, |W| below 8, and by rounding."""
    P = _api()
    rng = np.random.default_rng(13)
    h, eh = _matrix(rng, 9, 6, torch.float32)
    W, eW = _matrix(rng, 5, 6, torch.float32)
    b = rng.standard_normal(5).astype(np.float32)
    soft = rng.random((9, 5)).astype(np.float32)
    r = rng.random(9).astype(np.float32)
    _, dh, dweight, dbias = P.head_loss(h, W, torch.from_numpy(b).cuda(), torch.from_numpy(soft).cuda(), row_weight=torch.from_numpy(r).cuda())
    ref = S.head_loss(eh, eW, b, soft, None, r)
    bars = _bars(eh, eW, b, ref, r.astype(np.float64), 1.0)
    point = [eh, eW, b.astype(np.float64)]
    for at, (got, bar) in enumerate(((dh, bars["dh"]), (dweight, bars["dweight"]), (dbias, bars["dbias"]))):
        got = got.double().cpu().numpy()
        for k in np.ndindex(got.shape):
            sides = []
            for step in (1e-4, -1e-4):
                args = [x.copy() for x in point]
                args[at][k] += step
                sides.append(S.head_loss(*args, soft, None, r)["loss"].sum())
            assert abs((sides[0] - sides[1]) / 2e-4 - got[k]) <= bar[k] + 1e-6


def test_replays_of_a_graph():
    P = _api()
    rng = np.random.default_rng(14)
    h, _ = _matrix(rng, 5000, 72, torch.bfloat16)
    W, _ = _matrix(rng, 12, 72, torch.bfloat16)
    q = torch.softmax(torch.randn(5000, 12, device="cuda"), 1)
    P.head_loss(h, W, None, q), P.head_labels(h, W)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = P.head_loss(h, W, None, q) + P.head_labels(h, W)
    for k in range(4):
        h.mul_(0.9)
        q.copy_(torch.roll(q, k + 1, 0))
        graph.replay()
        want = P.head_loss(h, W, None, q) + P.head_labels(h, W)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_the_binding_refuses():
    P = _api()
    h, W, b = torch.zeros(5, 8, device="cuda"), torch.zeros(3, 8, device="cuda"), torch.zeros(3, device="cuda")
    q = torch.zeros(5, 3, device="cuda")
    for call in (lambda: P.head_labels(h, W.half()), lambda: P.head_labels(h, W[:, :7]), lambda: P.head_labels(h, torch.zeros(65, 8, device="cuda")),
                 lambda: P.head_labels(h, W, b[:2]), lambda: P.head_labels(h, W, b.double()), lambda: P.head_labels(h, W.cpu()),
                 lambda: P.head_loss(h, W, b, q[:4]), lambda: P.head_loss(h, W, b, q.t()), lambda: P.head_loss(h, W, b, q.half()),
                 lambda: P.head_loss(h, W, b, torch.zeros(5, dtype=torch.int64, device="cuda")),
                 lambda: P.head_loss(h, W, b, q, row_weight=b), lambda: P.head_loss(h[:, ::2], W[:, ::2], b, q)):
        with pytest.raises(P.DynLPError):
            call()
