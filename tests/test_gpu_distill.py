"""Learning from a teacher's first classes against the definition in 64 bits.

Bars, u = 2^-24, K entries, T the temperature.  Logits: e = (D + 3) u (sum |h||W| + |b|), heads in 32 bits (6 D + 8) u of it; the row's largest, over T, moves p by
p (exp(2 e / T) - 1 + (C + 64) u + 4 u y), y the largest |z| / T in use (z and its logarithm are rounded at that size).  q is off by (K + 16) u + 2 u of the spread of the list.  The loss, r T^2 (sum q log q + log sum - sum q z / T):
by r T^2 (2 e / T + (C + K + 64) u (1 + y + log C)).  dz: g r T (|dp| + |dq|), and what its terms leave out: 2^-8 of it in one bfloat16 term, 2^-11 in one of
float16, 2^-22 in two of float16, 2^-23 in three of bfloat16; float16 is scaled so that the largest weight lies in 2^14 .. 2^15 and is off by 2^-25 of that scale at least.
Sums over classes and rows carry those and (6 terms + 8) u of their magnitudes; results are rounded to their type."""
import numpy as np
import pytest

from oracle import student as S
from rounding import hold
from test_gpu_scores import TYPES, U, _api, _head

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _lists(rng, rows, classes, kept, pad=True):
    at = np.stack([rng.permutation(max(classes, kept))[:kept] for _ in range(rows)]) if rows else np.zeros((0, kept), dtype=np.int64)
    at = np.where(at < classes, at, -1)
    if pad and kept > 1:
        at[rng.random(at.shape) < 0.1] = -1
    return at.astype(np.int32), (5.0 + 2.0 * rng.standard_normal((rows, kept))).astype(np.float32)


def _left_out(kind, grad, to_h):
    """What dz's terms leave out, relative and (of the largest weight) absolute."""
    if kind == "float32":
        return 2.0 ** -22, 0.0
    one = to_h or grad != "float32"
    if kind == "bfloat16":
        return (2.0 ** -8 if one else 2.0 ** -23), 0.0
    return (2.0 ** -11 if one else 2.0 ** -22), 2.0 ** -25 * 2.0 ** -14


def _bars(ref, eh, eW, eb, r, temperature, grad_scale, kind, grad, logits):
    n, classes = ref["dz"].shape
    dim, kept = eh.shape[1], logits.shape[1]
    u_z = ((6 * dim + 8) if kind == "float32" else (dim + 3)) * U
    eh = np.where(ref["left_out"][:, None], 0.0, eh)
    e = u_z * (np.abs(eh) @ np.abs(eW).T + np.abs(eb)).max(axis=1, initial=0.0) / temperature
    y = np.abs(ref["logits"]).max(axis=1, initial=0.0)
    y = np.where(ref["left_out"], 0.0, y)
    spread = (logits.max(axis=1, initial=-99) - logits.min(axis=1, initial=99)) / temperature
    loss = np.abs(r) * temperature ** 2 * (2 * e + (classes + kept + 64) * U * (1 + y + spread + np.log(classes + 1)))
    p, q = ref["soft"], ref["target"]
    ddz = p * (np.exp(2 * e)[:, None] - 1 + (classes + 64) * U + 4 * U * (y[:, None] + np.log(classes + 1))) + q * ((kept + 16 + 2 * spread[:, None]) * U)
    scale = np.abs(grad_scale * r * temperature)[:, None]
    most = np.abs(grad_scale * temperature) * np.abs(r).max(initial=0.0)
    ddz = np.where(ref["left_out"][:, None], 0.0, scale * ddz + 4 * U * np.abs(ref["dz"]))
    dz = np.abs(ref["dz"])
    out = {"loss": loss + 2.0 ** -140, "dbias": (ddz + (n + 64) * U * dz).sum(axis=0) + 2.0 ** -140}
    for name, to_h, terms in (("dh", True, classes), ("dweight", False, n)):
        rel, absolute = _left_out(kind, grad, to_h)
        all_dz = ddz + (rel + (6 * terms + 8) * U) * dz + np.where(dz > 0, absolute * most, 0.0)
        out[name] = (all_dz @ np.abs(eW) if to_h else all_dz.T @ np.abs(eh)) + 2.0 ** -140
    return out


def _run(P, h, W, b, classes, logits, **more):
    return P.head_distill(h, W, b, torch.from_numpy(classes).cuda(), torch.from_numpy(logits).cuda(), **more)


CASES = [  # rows, dim, classes, kept
    (0, 8, 3, 1), (1, 1, 1, 1), (1, 64, 10, 3), (2, 3, 2, 2), (15, 33, 17, 5), (16, 32, 64, 64), (17, 64, 65, 64), (63, 40, 300, 8), (64, 96, 256, 1),
    (65, 100, 257, 128), (129, 200, 50, 7), (100, 64, 1000, 33), (300, 16, 129, 65), (513, 64, 10, 4), (40, 1030, 70, 3), (200, 300, 513, 16), (130, 31, 700, 2),
    (20, 24, 5000, 32),
]


@pytest.mark.parametrize("kind, grad", [("float32", "float32"), ("bfloat16", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32"), ("float16", "float16")])
@pytest.mark.parametrize("rows, dim, classes, kept", CASES)
def test_distill(rows, dim, classes, kept, kind, grad):
    P = _api()
    rng = np.random.default_rng(rows + 3 * dim + classes + kept)
    h, W, b, eh, eW, eb = _head(rng, rows, dim, classes, TYPES[kind], False, stride=rows % 3, shift=dim % 2)
    bias, eb = (b, eb) if rows % 2 else (None, np.zeros(classes))
    at, u = _lists(rng, rows, classes, kept)
    r = np.where(rng.random(rows) < 0.1, 0.0, rng.random(rows) * 3.0).astype(np.float32) if rows % 4 != 1 else None
    temperature, grad_scale = (1.0, 2.0, 0.5)[rows % 3], 1.0 / max(rows, 1)
    got = _run(P, h, W, bias, at, u, temperature=temperature, grad_scale=grad_scale, row_weight=None if r is None else torch.from_numpy(r).cuda(), dtype=TYPES[grad])
    ref = S.distill(eh, eW, eb, at, u, temperature, r, grad_scale)
    r = np.ones(rows) if r is None else r.astype(np.float64)
    bars = _bars(ref, eh, eW, eb, r, temperature, grad_scale, kind, grad, u)
    for name, value in zip(("loss", "dh", "dweight", "dbias"), got):
        hold(value, ref[name], bars[name], name)
    assert got[1].dtype == TYPES[kind] and got[2].dtype == TYPES[grad]
    alone = _run(P, h, W, bias, at, u, temperature=temperature, row_weight=None if r is None else torch.from_numpy(r.astype(np.float32)).cuda(), grads=False)
    assert torch.equal(alone[0], got[0]) and alone[1:] == (None, None, None)


@pytest.mark.parametrize("rows, classes", [(12, 10), (40, 300)])
def test_rows_that_are_left_out(rows, classes):
    """Whatever their h and lists hold: nothing of them is anywhere."""
    P = _api()
    rng = np.random.default_rng(1)
    h, W, b, eh, eW, eb = _head(rng, rows, 32, classes, torch.bfloat16, False)
    at, u = _lists(rng, rows, classes, 5, pad=False)
    r = np.ones(rows, dtype=np.float32)
    r[0], r[rows - 1] = 0.0, 0.0
    at[1] = -1
    u[2] = -np.inf
    at[3] = classes + 5
    out = [0, 1, 2, 3, rows - 1]
    h[out[0]], h[out[1]], h[out[2]], h[rows - 1] = float("nan"), float("inf"), float("nan"), float("nan")
    u[0] = np.nan
    rejected = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = _run(P, h, W, b, at, u, row_weight=torch.from_numpy(r).cuda(), rejected=rejected)
    assert int(rejected) == 5
    assert (got[0][out] == 0).all() and (got[1][out] == 0).all()
    keep = np.setdiff1d(np.arange(rows), out)
    ref = S.distill(eh[keep], eW, eb, at[keep], u[keep])
    bars = _bars(ref, eh[keep], eW, eb, np.ones(len(keep)), 1.0, 1.0, "bfloat16", "float32", u[keep])
    for name, value in zip(("loss", "dh", "dweight", "dbias"), (got[0][keep], got[1][keep], got[2], got[3])):
        hold(value, ref[name], bars[name], name)
    # nothing at all to learn
    none = _run(P, h, W, b, np.full_like(at, -1), u)
    assert all((v == 0).all() for v in none)
    none = _run(P, h[4:6], W, torch.full_like(b, -float("inf")), at[4:6], u[4:6])
    assert all((v == 0).all() for v in none)


@pytest.mark.parametrize("kind", list(TYPES))
def test_lists_with_the_same_class_twice(kind):
    P = _api()
    rng = np.random.default_rng(2)
    for rows, classes, kept in ((9, 20, 6), (33, 400, 70)):
        h, W, b, eh, eW, eb = _head(rng, rows, 32, classes, TYPES[kind], False)
        at = rng.integers(-1, 12, size=(rows, kept)).astype(np.int32)
        u = rng.standard_normal((rows, kept)).astype(np.float32)
        got = _run(P, h, W, b, at, u)
        ref = S.distill(eh, eW, eb, at, u)
        bars = _bars(ref, eh, eW, eb, np.ones(rows), 1.0, 1.0, kind, "float32", u)
        for name, value in zip(("loss", "dh", "dweight", "dbias"), got):
            hold(value, ref[name], bars[name], name)


def test_one_class_is_a_hard_label():
    P = _api()
    h = torch.randn(70, 32, device="cuda")
    W = torch.randn(40, 32, device="cuda")
    y = torch.randint(0, 40, (70,), dtype=torch.int32, device="cuda")
    got = P.head_distill(h, W, None, y[:, None].contiguous(), torch.randn(70, 1, device="cuda"))
    want = P.head_loss(h, W, None, y)
    for a, b in zip(got, want):
        assert torch.allclose(a, b, rtol=1e-4, atol=1e-5)


def test_impossible_classes():
    """A listed class whose logit is -infinity: infinite loss, finite gradients; entries without probability ask for nothing of their class."""
    P = _api()
    rng = np.random.default_rng(4)
    h, W, b, eh, eW, eb = _head(rng, 5, 32, 100, torch.float32, False)
    b[7] = -float("inf")
    at = np.array([[7, 3], [3, 7], [7, 7], [1, 2], [9, 9]], dtype=np.int32)
    u = np.array([[0, 0], [0, -np.inf], [0, 0], [np.nan, 0], [np.inf, 0]], dtype=np.float32)
    loss, dh, dweight, dbias = _run(P, h, W, b, at, u, row_weight=torch.tensor([1.0, 1.0, 1.0, 0.0, 0.0], device="cuda"))
    assert loss[0] == float("inf") and loss[2] == float("inf") and torch.isfinite(loss[[1, 3, 4]]).all()
    assert torch.isfinite(dh).all() and torch.isfinite(dweight).all()
    assert float(dbias[7]) == -1.5
    loss, dh, dweight, dbias = _run(P, h, W, b, at, u)
    assert torch.isnan(loss[3]) and torch.isnan(loss[4]) and torch.isnan(dh[3]).all() and torch.isfinite(dh[:3]).all()


def test_weights_of_all_sizes_in_16_bits():
    """The scale that float16 gradients are made with follows the largest weight."""
    P = _api()
    rng = np.random.default_rng(6)
    for kind in ("float16", "bfloat16"):
        for size in (1e-30, 1e-6, 1.0, 1e6):
            h, W, b, eh, eW, eb = _head(rng, 30, 32, 90, TYPES[kind], False)
            at, u = _lists(rng, 30, 90, 4)
            r = (size * rng.random(30)).astype(np.float32)
            for grad in (kind, "float32"):
                scale = 1.0 / size if grad == kind else 1.0
                got = _run(P, h, W, b, at, u, row_weight=torch.from_numpy(r).cuda(), grad_scale=scale, dtype=TYPES[grad])
                scale = float(np.float32(scale))
                ref = S.distill(eh, eW, eb, at, u, 1.0, r, scale)
                bars = _bars(ref, eh, eW, eb, r.astype(np.float64), 1.0, scale, kind, grad, u)
                for name, value in zip(("loss", "dh", "dweight", "dbias"), got):
                    hold(value, ref[name], bars[name], name)


def test_gradients_are_those_of_the_loss():
    """Differences of the 64-bit loss along random directions against the gradients of a float32 head: both sides of a step of 1e-4, whose error is of the step's square."""
    P = _api()
    rng = np.random.default_rng(8)
    h, W, b, eh, eW, eb = _head(rng, 20, 24, 80, torch.float32, False)
    at, u = _lists(rng, 20, 80, 6)
    r = rng.random(20).astype(np.float32)
    loss, dh, dweight, dbias = _run(P, h, W, b, at, u, temperature=2.0, row_weight=torch.from_numpy(r).cuda())
    for g, k in ((dh, 0), (dweight, 1), (dbias, 2)):
        v = rng.standard_normal(tuple(g.shape))
        at_step = lambda t: S.distill(*(x + t * v if j == k else x for j, x in enumerate((eh, eW, eb))), at, u, 2.0, r)["loss"].sum()  # noqa: E731
        want = (at_step(1e-4) - at_step(-1e-4)) / 2e-4
        assert abs(float((g.double().cpu().numpy() * v).sum()) - want) < 1e-4 * (1 + abs(want))


def test_the_same_bits_every_time_and_on_other_streams():
    P = _api()
    rng = np.random.default_rng(9)
    for rows, classes in ((300, 50), (700, 1000)):
        h, W, b, *_ = _head(rng, rows, 64, classes, torch.bfloat16, False)
        at, u = (torch.from_numpy(x).cuda() for x in _lists(rng, rows, classes, 8))
        want = P.head_distill(h, W, b, at, u)
        for _ in range(5):
            for x, y in zip(want, P.head_distill(h, W, b, at, u)):
                assert torch.equal(x, y)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            other = P.head_distill(h, W, b, at, u)
        torch.cuda.current_stream().wait_stream(stream)
        for x, y in zip(want, other):
            assert torch.equal(x, y)


@pytest.mark.parametrize("kind", ["bfloat16", "float16", "float32"])
def test_captured_steps(kind):
    """Two graphs and eager calls in between, replayed on new inputs."""
    P = _api()
    rng = np.random.default_rng(10)
    sets = []
    for rows, classes in ((100, 40), (90, 600)):
        h, W, b, *_ = _head(rng, rows, 64, classes, TYPES[kind], False)
        at, u = (torch.from_numpy(x).cuda() for x in _lists(rng, rows, classes, 8))
        sets.append((h, W, b, at, u))
    for s in sets:
        P.head_distill(*s)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(P.head_distill(*s, dtype=TYPES[kind]))
        graphs.append(g)
    for turn in range(4):
        for s in sets:
            s[0].copy_(s[0].roll(1, 0))
            s[4].add_(torch.randn_like(s[4]))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, o in zip(sets, outs):
            for x, y in zip(P.head_distill(*s, dtype=TYPES[kind]), o):
                assert torch.equal(x, y), turn


def test_outputs_one_at_a_time():
    """Through the C entry point: each output without the others is what it is with them, and rows behind a padded dh stay as they were."""
    from paper_2604_06596_amd import train as T

    P = _api()
    rng = np.random.default_rng(11)
    L = T._library()
    for kind, rows, classes in (("bfloat16", 100, 300), ("float32", 40, 20)):
        h, W, b, *_ = _head(rng, rows, 32, classes, TYPES[kind], False)
        at, u = (torch.from_numpy(x).cuda() for x in _lists(rng, rows, classes, 4))
        loss, dh, dweight, dbias = P.head_distill(h, W, b, at, u)
        m, w = T._matrix(h, "h", h.device), T._matrix(W, "W", h.device)
        t = T._Teacher(at.data_ptr(), u.data_ptr(), None, None, 4, 1.0, 1.0)
        for which in range(4):
            pad = torch.full((rows + 1, 40), 7.0, dtype=TYPES[kind], device="cuda")
            wide = torch.full((classes + 1, 37), 7.0, device="cuda")
            flat = [torch.full((n,), 7.0, device="cuda") for n in (rows + 1, classes + 1)]
            grad = 0 if which == 2 else -1 if which == 0 else m.type
            call, space = T._call(h.device, L.dynlp_head_distill_workspace(rows, 32, classes, 4, m.type, grad))
            T._check(L.dynlp_head_distill(m, w, b.data_ptr(), t, flat[0].data_ptr() if which == 0 else None,
                                          T._Matrix(pad.data_ptr(), rows, 40, 32, m.type) if which == 1 else None,
                                          T._Matrix(wide.data_ptr(), classes, 37, 32, 0) if which == 2 else None, flat[1].data_ptr() if which == 3 else None, call))
            if which == 0:
                assert torch.equal(flat[0][:rows], loss) and float(flat[0][rows]) == 7.0
            if which == 1:
                assert torch.allclose(pad[:rows, :32], dh) and (pad[rows:] == 7).all() and (pad[:, 32:] == 7).all()
            if which == 2:
                assert torch.equal(wide[:classes, :32], dweight) and (wide[classes:] == 7).all() and (wide[:, 32:] == 7).all()
            if which == 3:
                assert torch.equal(flat[1][:classes], dbias) and float(flat[1][classes]) == 7.0


def test_a_step_by_turns():
    """More of dz than is in memory at a time: 40,000 x 70,000 in 16 bits; the rows' sums meet, whichever turn they were in."""
    P = _api()
    rows, classes, dim = 40000, 70000, 32
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.randn(rows, dim, generator=g, device="cuda").to(torch.bfloat16)
    W = (0.3 * torch.randn(classes, dim, generator=g, device="cuda")).to(torch.bfloat16)
    at = torch.randint(0, classes, (rows, 2), generator=g, device="cuda", dtype=torch.int32)
    u = torch.randn(rows, 2, generator=g, device="cuda")
    loss, dh, dweight, dbias = P.head_distill(h, W, None, at, u, dtype=torch.bfloat16)
    half = [P.head_distill(h[s], W, None, at[s], u[s], dtype=torch.float32) for s in (slice(0, 20000), slice(20000, rows))]
    assert torch.allclose(loss, torch.cat([x[0] for x in half]), rtol=1e-5) and torch.allclose(dh.float(), torch.cat([x[1] for x in half]).float(), rtol=2.0 ** -7, atol=1e-6)
    both = half[0][2] + half[1][2]
    assert float((dweight.float() - both).norm() / both.norm()) < 2.0 ** -8
    bias = half[0][3] + half[1][3]
    assert float((dbias - bias).norm() / bias.norm()) < 1e-5


@pytest.mark.parametrize("classes, kept", [(50, 8), (500, 20)])
def test_a_teacher_and_its_student(classes, kept):
    """As they are used together: a teacher's first classes, a student that learns them through its table, and its own scores."""
    P = _api()
    g = torch.Generator(device="cuda").manual_seed(3)
    items, words, dim = 400, 300, 32
    ids = torch.randint(0, words, (items * 6,), generator=g, device="cuda", dtype=torch.int32)
    offsets = torch.arange(0, items * 6 + 1, 6, device="cuda")
    soft = torch.softmax(3.0 * torch.randn(items, classes, generator=g, device="cuda"), 1)
    lists = P.row_scores(soft, top=kept, probabilities=True)
    table = (0.3 * torch.randn(words, dim, generator=g, device="cuda")).to(torch.bfloat16)
    weight = torch.zeros(classes, dim, dtype=torch.bfloat16, device="cuda")
    bias = torch.zeros(classes, device="cuda")
    h = P.embed(table, ids, offsets)
    loss, dh, dweight, dbias = P.head_distill(h, weight, bias, lists.top, lists.log_top, grad_scale=1.0 / items)
    dtable = P.embed_grad(dh, ids, words, offsets)
    assert dtable.shape == table.shape
    q = torch.softmax(lists.log_top.double(), 1)
    want = (q * q.log()).sum(1) + np.log(classes)  # a head of zeros says 1/C
    assert torch.allclose(loss.double(), want, rtol=1e-5, atol=1e-5)
    dense = torch.full((items, classes), 1.0 / classes, device="cuda", dtype=torch.float64).scatter_add_(1, lists.top.long(), -q)
    assert torch.allclose(dbias.double(), dense.mean(0), rtol=1e-4, atol=1e-7)
    assert torch.allclose(dweight.double(), dense.t().contiguous() @ h.double() / items, rtol=1e-3, atol=1e-6)
    answer = P.head_scores(h, weight, bias, given=lists.top[:, 0].contiguous(), top=2)
    assert torch.allclose(answer.log_given, torch.full((items,), -float(np.log(classes)), device="cuda")) and (answer.top == torch.tensor([0, 1], device="cuda")).all()


@pytest.mark.parametrize("rows, dim, classes, kept", [(70, 16, 70, 5), (1, 301, 20011, 16), (3000, 48, 900, 3), (1500, 130, 66, 128), (33, 20, 100003, 2), (5000, 17, 100, 9),
                                                      (260, 64, 8200, 64)])
@pytest.mark.parametrize("kind", list(TYPES))
def test_other_shapes_of_heads(rows, dim, classes, kept, kind):
    """Few rows and many classes, many rows and few classes: each has tiles and joins of its own."""
    P = _api()
    rng = np.random.default_rng(rows + dim)
    h, W, b, eh, eW, eb = _head(rng, rows, dim, classes, TYPES[kind], False)
    at = rng.integers(0, classes, size=(rows, kept)).astype(np.int32)
    u = rng.standard_normal((rows, kept)).astype(np.float32)
    r = np.where(rng.random(rows) < 0.2, 0.0, rng.random(rows)).astype(np.float32)
    got = _run(P, h, W, b, at, u, temperature=3.0, row_weight=torch.from_numpy(r).cuda(), dtype=TYPES[kind])
    ref = S.distill(eh, eW, eb, at, u, 3.0, r)
    bars = _bars(ref, eh, eW, eb, r.astype(np.float64), 3.0, 1.0, kind, kind, u)
    for name, value in zip(("loss", "dh", "dweight", "dbias"), got):
        hold(value, ref[name], bars[name], name)


def test_the_example_learns_from_lists():
    """It runs, its numbers are numbers; unsure() is the entropy of labels()."""
    import importlib.util
    import os

    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "student.py")
    spec = importlib.util.spec_from_file_location("student_example", at)
    E = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(E)
    results = E.run(items=2000, steps=3, words=2000, dim=32, keep=3, verbose=True)
    assert np.isfinite(results).all()
    student = E.Student(500, 32, 10, 32, 1)
    student.weight.normal_()
    texts = E.make_texts(torch.arange(40, device="cuda") % 10, 10, 500, 8.0, 3)
    soft = student.labels(*texts)[0].double()
    assert torch.allclose(student.unsure(*texts).double(), -torch.xlogy(soft, soft).sum(1), rtol=1e-4, atol=1e-5)


@pytest.mark.parametrize("rows, dim, classes", [(3, 64, 70), (40, 64, 200), (256, 48, 1000)])
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
def test_small_calls_are_off_by_their_own_rounding(rows, dim, classes, kind):
    """dz in two terms: what they leave out, 2^-16 of it in bfloat16 and 2^-22 in float16, is little beside the result's rounding."""
    P = _api()
    rng = np.random.default_rng(rows)
    h, W, b, eh, eW, eb = _head(rng, rows, dim, classes, TYPES[kind], False)
    at, u = _lists(rng, rows, classes, 2)
    got = _run(P, h, W, b, at, u, dtype=TYPES[kind])
    ref = S.distill(eh, eW, eb, at, u)
    bars = _bars(ref, eh, eW, eb, np.ones(rows), 1.0, 1.0, "float32", "float32", u)
    dz = np.abs(ref["dz"])
    rel, absolute = (2.0 ** -16, 0.0) if kind == "bfloat16" else (2.0 ** -22, 2.0 ** -25 * 2.0 ** -14)
    more = rel * dz + np.where(dz > 0, absolute, 0.0)
    hold(got[1], ref["dh"], bars["dh"] + more @ np.abs(eW), "dh")
    hold(got[2], ref["dweight"], bars["dweight"] + more.T @ np.abs(eh), "dweight")
