"""The student's operators where lists, rows and arguments are unlike those of a batch of texts: offsets that miss the list, long runs of items
without tokens, more items than one launch has workgroups, outputs in the inputs' memory, factors that are not finite.

Bars as in test_gpu_train_embed.py and test_gpu_train_head.py."""
import numpy as np
import pytest

from oracle import student as S
from rounding import hold
from test_gpu_train_head import SHAPES, _bars

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
U = 2.0 ** -24


def _api():
    import paper_2604_06596_amd as P

    return P


def _random(rng, rows, dim, dtype, size=1.0):
    """(matrix on the GPU, its values in 64 bits)"""
    t = torch.from_numpy(size * rng.standard_normal((rows, dim))).to(dtype).cuda()
    return t, t.double().cpu().numpy()


def _ids(rng, count, rows):
    """ids, a tenth of them padding."""
    return np.where(rng.random(count) < 0.1, -1, rng.integers(0, rows, count)).astype(np.int32)


def _gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _hold_sum(got, exact, magnitude, terms):
    hold(got, exact, (terms[:, None] + 2) * U * magnitude)


def _embed_into(out, table, ids, offsets, weights=None, scale=1.0):
    """dynlp_embed into `out`, so that what is not written is seen."""
    from paper_2604_06596_amd import train as T

    L = T._library()
    t = T._tokens(ids, offsets, weights, scale, None, table.device)
    call, space = T._call(table.device, L.dynlp_embed_workspace(t.count, t.items, table.shape[1]))
    T._check(L.dynlp_embed(T._matrix(table, "table", table.device), t, T._matrix(out, "out", table.device), call))
    return out


@pytest.mark.parametrize("kind, dim", [("float32", 64), ("float32", 24), ("bfloat16", 128), ("float16", 200), ("bfloat16", 520)])
@pytest.mark.parametrize("count", [500, 2049, 9001])
def test_items_that_begin_before_the_list_or_end_behind_it(count, kind, dim):
    """Such an item has the tokens that are in the list, whatever the length of list and rows; every row is written."""
    P = _api()
    rng = np.random.default_rng(count + dim)
    table, exact = _random(rng, 50, dim, TYPES[kind])
    ids, w = _ids(rng, count, 50), rng.standard_normal(count).astype(np.float32)
    for offsets in ([-5, 2 ** 40], [-5, count // 2, count], [-9, -7, 300, count + 1], [-2 ** 40, 1, 1, count - 3, count + 9, count + 9], [-3, 0, 0, 40, 40]):
        out = torch.full((len(offsets) - 1, dim), float("nan"), dtype=TYPES[kind], device="cuda")
        _embed_into(out, table, _gpu(ids), _gpu(np.array(offsets)), _gpu(w), 0.5)
        _hold_sum(out, *S.embed(exact, ids, offsets, w, 0.5))
        grad, exact_grad = _random(rng, len(offsets) - 1, dim, TYPES[kind])
        _hold_sum(P.embed_grad(grad, _gpu(ids), 50, _gpu(np.array(offsets)), _gpu(w), 0.5), *S.embed_grad(exact_grad, ids, 50, offsets, w, 0.5))


def _loss_into(dh, h, weight, target, dweight=None):
    """dynlp_head_loss with a dh of the caller's; returns (status, loss)."""
    from paper_2604_06596_amd import train as T

    L = T._library()
    m, w = T._matrix(h, "h", h.device), T._matrix(weight, "weight", h.device)
    loss = torch.empty(len(h), device="cuda")
    call, space = T._call(h.device, L.dynlp_head_loss_workspace(m.rows, m.dim, w.rows, m.type))
    t = T._Targets(target.data_ptr(), None, None, None, 1.0)
    status = L.dynlp_head_loss(m, w, None, t, loss.data_ptr(), T._matrix(dh, "dh", h.device), None if dweight is None else dweight.data_ptr(), None, call)
    return status, loss


@pytest.mark.parametrize("kind, rows, dim, classes", [("float32", 700, 64, 10), ("bfloat16", 700, 200, 50), ("float16", 300, 520, 20)])
def test_a_gradient_of_h_beside_it_or_in_its_place(kind, rows, dim, classes):
    """Rows of h and dh may take turns in one array, by columns or by rows.  Where no dweight is asked for, dh may take h's place; where it is,
    that is refused, and so is an overlap that is not the same place."""
    rng = np.random.default_rng(3)
    h, _ = _random(rng, rows, dim, TYPES[kind])
    W, _ = _random(rng, classes, dim, TYPES[kind], 2.0 / np.sqrt(dim))
    q = torch.softmax(_random(rng, rows, classes, torch.float32)[0], 1)
    want, dweight, other = torch.empty_like(h), torch.empty(classes, dim, device="cuda"), torch.empty(classes, dim, device="cuda")
    status, loss = _loss_into(want, h, W, q, dweight)
    assert status == 0
    both = torch.zeros(rows, 2 * dim, dtype=h.dtype, device="cuda")
    for a, b in ((both[:, :dim], both[:, dim:]), (both.view(2 * rows, dim)[::2], both.view(2 * rows, dim)[1::2]), (both[:, dim:], both[:, :dim])):
        a.copy_(h)
        status, again = _loss_into(b, a, W, q, other)
        assert status == 0 and torch.equal(again, loss) and torch.equal(b, want) and torch.equal(other, dweight)
    alone = torch.empty_like(h)
    assert _loss_into(alone, h, W, q)[0] == 0
    same = h.clone()
    status, again = _loss_into(same, same, W, q)
    assert status == 0 and torch.equal(again, loss) and torch.equal(same, alone)
    same = torch.cat([h, h[:1]])
    before = same.clone()
    assert _loss_into(same[:rows], same[:rows], W, q, other)[0] == -1
    assert _loss_into(same[1:], same[:rows], W, q, other)[0] == -1 and _loss_into(same[1:], same[:rows], W, q)[0] == -1
    torch.cuda.synchronize()
    assert torch.equal(same, before)


@pytest.mark.parametrize("dim", [8, 128])
@pytest.mark.parametrize("count", [37, 2048, 2049, 8192, 8193])
def test_every_rejected_id_of_the_list_is_counted(count, dim):
    """Whether an item has it or not, and also where there is no item, or no row, at all."""
    P = _api()
    rng = np.random.default_rng(count)
    ids = rng.integers(-3, 60, count).astype(np.int32)
    bad = int((ids >= 50).sum())
    assert bad > 0
    table = torch.ones(50, dim, device="cuda")
    for offsets in ([0, 5, count], [7, 20], [count // 2, count // 2], [0]):
        o = torch.tensor(offsets, device="cuda")
        rejected = torch.tensor([3], dtype=torch.int32, device="cuda")
        P.embed(table, _gpu(ids), o, rejected=rejected)
        assert int(rejected) == 3 + bad
        P.embed_grad(torch.ones(len(offsets) - 1, dim, device="cuda"), _gpu(ids), 50, o, rejected=rejected)
        assert int(rejected) == 3 + 2 * bad
        P.embed_grad(torch.ones(len(offsets) - 1, dim, device="cuda"), _gpu(ids), 0, o, rejected=rejected)
        assert int(rejected) == 3 + 2 * bad + int((ids >= 0).sum())


@pytest.mark.parametrize("count", [0, 37, 2048])
def test_more_items_than_a_launch_has_workgroups(count):
    """2^24 + 1 items with few tokens: 2^32 threads, where an item has a workgroup."""
    rng = np.random.default_rng(count)
    items = 2 ** 24 + 1
    table, exact = _random(rng, 40, 4, torch.float32)
    ids = _ids(rng, count, 40)
    with_tokens = np.unique(np.concatenate([[0, items - 1], rng.integers(0, items, 20)]))
    cuts = np.concatenate([[0], np.sort(rng.integers(0, count + 1, len(with_tokens) - 1)), [count]])
    offsets = torch.zeros(items + 1, dtype=torch.int64, device="cuda")
    offsets[_gpu(with_tokens + 1)] = _gpu(np.diff(cuts))
    torch.cumsum(offsets, 0, out=offsets)
    out = torch.full((items, 4), float("nan"), device="cuda")
    _embed_into(out, table, _gpu(ids), offsets)
    want, magnitude, terms = S.embed(exact, ids, cuts)
    _hold_sum(out[_gpu(with_tokens)], want, magnitude, terms)
    out[_gpu(with_tokens)] = 0.0
    assert not out.any()


def _least_ms(f, turns=4):
    f()
    times = []
    for _ in range(turns):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        f()
        end.record()
        end.synchronize()
        times.append(begin.elapsed_time(end))
    return min(times)


@pytest.mark.parametrize("kind, dim, empty, most_ms", [("bfloat16", 128, 1_000_000, 20.0), ("float32", 16, 8_000_000, 5.0)])
def test_a_long_run_of_items_without_tokens(kind, dim, empty, most_ms):
    """Two texts with a million or more empty items between them.  The zeros are 256 and 512 MB, 0.1 ms; a search for the next text takes some tens of reads
    one after the other.  A look at one item after the other by a wave takes 0.2 us and more each (200 ms), by a workgroup 256 at a time 15 ms."""
    P = _api()
    rng = np.random.default_rng(dim)
    count = 9001
    ids, w = _ids(rng, count, 300), rng.standard_normal(count).astype(np.float32)
    table, exact = _random(rng, 300, dim, TYPES[kind])
    offsets = torch.full((empty + 3,), 4003, dtype=torch.int64, device="cuda")
    offsets[0], offsets[-1] = 0, count
    args = _gpu(ids), offsets, _gpu(w)
    out = P.embed(table, *args)
    assert out.shape == (empty + 2, dim) and not out[1:-1].any()
    _hold_sum(out[[0, -1]], *S.embed(exact, ids, [0, 4003, count], w))
    assert _least_ms(lambda: P.embed(table, *args)) < most_ms
    out.normal_()
    g = P.embed_grad(out, args[0], 300, *args[1:])
    _hold_sum(g, *S.embed_grad(out[[0, -1]].double().cpu().numpy(), ids, 300, [0, 4003, count], w))
    assert _least_ms(lambda: P.embed_grad(out, args[0], 300, *args[1:])) < most_ms


@pytest.mark.parametrize("dim", [16, 128])
@pytest.mark.parametrize("count", [60, 9001])
def test_items_without_tokens_are_zeros_whatever_the_scale(count, dim):
    P = _api()
    table = torch.ones(5, dim, device="cuda")
    ids = torch.zeros(count, dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 0, 30, 30, count, count], device="cuda")
    for scale in (float("inf"), float("nan"), -2.0):
        out = P.embed(table, ids, offsets, None, scale)
        assert torch.equal(out[[0, 2, 4]], torch.zeros(3, dim, device="cuda"))
        want = torch.full((2, dim), scale, device="cuda") * torch.tensor([[30.0], [count - 30.0]], device="cuda")
        assert torch.equal(out[[1, 3]].nan_to_num(7.0), want.nan_to_num(7.0))


@pytest.mark.parametrize("bits", [8, 32])
def test_a_step_is_a_change_of_its_tensors(bits):
    """torch counts changes of a tensor, and refuses a backward pass through one that has changed since: a step is such a change, of copies too."""
    P = _api()
    p, c = torch.ones(300, device="cuda", requires_grad=True), torch.ones(300, device="cuda", requires_grad=True)
    state = P.adamw_state(p, bits)
    before = [t._version for t in (p, c) + state]
    saved = [(p * p).sum(), (c * c).sum()]
    P.adamw_step([p], [torch.ones(300, device="cuda")], [state], step=1, lr=0.1, copies=[c])
    assert all(t._version > v for t, v in zip((p, c) + state, before))
    for s in saved:
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            s.backward()
    with torch.inference_mode():
        q = torch.ones(300, device="cuda")
        P.adamw_step([q], [torch.ones(300, device="cuda")], [P.adamw_state(q, bits)], step=1, lr=0.1)
    assert torch.equal(q, p)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows, dim", [(200, 24), (200, 64), (64, 520)])
def test_gradients_of_classes_that_cancel(rows, dim, kind):
    """W's rows are 64 and a little, and dz sums to nothing: 64 of dz must cancel to what float32 holds.  All logits are 0, so that exponentials and their sum
    are exact: dz is a division, a product and a difference away from the definition, 3 u (p + q), and dh's products and sums add (C + 4) u |dz| |W|."""
    P = _api()
    rng = np.random.default_rng(dim)
    classes = 3
    W = 64.0 + 0.5 * rng.integers(0, 2, (classes, dim))
    q = rng.random((rows, classes)).astype(np.float32)
    q /= q.sum(axis=1, keepdims=True)
    h = torch.zeros(rows, dim, dtype=TYPES[kind], device="cuda")
    dh = P.head_loss(h, _gpu(W).to(TYPES[kind]), None, _gpu(q))[1]
    exact = q.astype(np.float64)
    p = 1.0 / classes
    dz = exact.sum(axis=1, keepdims=True) * p - exact
    hold(dh, dz @ W, (3 * U * (exact.sum(axis=1, keepdims=True) * p + exact) + (classes + 4) * U * np.abs(dz)) @ W)


def test_a_tensor_of_more_workgroups_than_a_launch_has():
    """2^34 + 1,030 elements, 2^24 + 2 workgroups: a step changes what has a gradient, at the ends of the launches too, and nothing else."""
    if torch.cuda.mem_get_info()[0] < 140e9:
        pytest.skip("103 GB of states, gradients and parameters, and room to look at them")
    P = _api()
    n, launch = 2 ** 34 + 1030, (2 ** 24 - 1) * 1024
    at = torch.tensor([0, 5, 2 ** 32 + 3, launch - 1, launch, launch + 1024, 2 ** 34 - 1, 2 ** 34, n - 1], device="cuda")
    params, grads = ([torch.zeros(k, dtype=torch.bfloat16, device="cuda") for k in (n, 300)] for _ in range(2))
    states = [P.adamw_state(p, bits=8) for p in params]
    grads[0][at] = grads[1][:len(at)] = torch.linspace(-0.5, 0.75, len(at), device="cuda").bfloat16()
    P.adamw_step(params, grads, states, step=1, lr=0.01, seed=3)

    def others(t):
        return sum(int(c.count_nonzero()) for c in t.split(2 ** 30)) - int(t[torch.unique(at if len(t) == n else at // 256)].count_nonzero())

    assert torch.equal(params[0][at], params[1][:len(at)]) and bool((params[0][at] != 0).all()) and others(params[0]) == 0
    for codes, scales in (states[0][::2], states[0][1::2]):
        codes = codes.view(torch.uint8)
        assert bool((codes[at] != 0).all()) and others(codes) == 0 and bool((scales[at // 256] != 0).all()) and others(scales) == 0
    del params, grads, states, codes, scales
    torch.cuda.empty_cache()


def test_a_head_of_four_million_columns():
    """dweight's 2^28 elements and more are joined 16 to a workgroup: 2^32 threads.  h is zero but for 16 columns, so that a logit has 17 roundings."""
    P = _api()
    rng = np.random.default_rng(8)
    dim, classes = 2 ** 22 + 70, 64
    some = _gpu(np.concatenate([np.arange(8), dim - 8 + np.arange(8)]))
    h = torch.zeros(2, dim, device="cuda")
    h[:, some] = _random(rng, 2, 16, torch.float32)[0]
    W = torch.randn(classes, dim, device="cuda")
    label = np.array([3, 63])
    got = dict(zip(("loss", "dh", "dweight", "dbias"), P.head_loss(h, W, None, _gpu(label.astype(np.int32)))))
    eh, eW = (x[:, some].double().cpu().numpy() for x in (h, W))
    ref = S.head_loss(eh, eW, None, hard=label)
    off = 19 * U * (np.abs(eh) @ np.abs(eW).T).max(axis=1, keepdims=True)
    p, dz = ref["soft"], np.abs(ref["dz"])
    ddz = p * (np.exp(2 * off) - 1 + (classes + 16) * U) + 4 * U * (p + ref["target"]) + (classes + 4) * U * dz
    hold(got["dbias"], ref["dbias"], (ddz + 2 * U * dz).sum(axis=0))
    hold(got["dweight"][:, some], ref["dweight"], (ddz + 2 * U * dz).T @ np.abs(eh))
    got["dweight"][:, some] = 0.0
    assert not got["dweight"].any()
    wide = W.double()
    hold(got["dh"], (_gpu(ref["dz"]) @ wide).cpu().numpy(), (_gpu(ddz) @ wide.abs()).cpu().numpy())


def test_the_loss_of_as_many_rows_as_there_may_be():
    """2^31 - 2 rows: 2^24 workgroups of 128 rows.  2 (D + 3) u |h W| + (C + 16) u (1 + |lse - z|) is below 40 u for the last row."""
    P = _api()
    rows = 2 ** 31 - 2
    h, hard = torch.zeros(rows, 1, dtype=torch.float16, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    h[-1], hard[-1] = 2.0, 1
    loss = P.head_loss(h, torch.tensor([[0.0], [1.0]], dtype=torch.float16, device="cuda"), None, hard, grads=False)[0]
    hold(loss[-1:], np.log1p(np.exp([-2.0])), 40 * U)
    loss[-1] = loss[0]
    hold(torch.stack([loss.min(), loss.max()]), np.full(2, np.log(2.0)), 40 * U)


def test_rows_of_sixteen_million_columns():
    """A wave has 256 columns of a piece of the list, and so has a wave that joins runs: 65,538 of them side by side."""
    P = _api()
    rng = np.random.default_rng(9)
    count, dim = 2049, 2 ** 24 + 300
    table = torch.randn(3, dim, device="cuda")
    ids, w = _ids(rng, count, 3), rng.random(count).astype(np.float32)
    offsets = np.array([0, 1001, count])
    args = _gpu(ids), _gpu(offsets), _gpu(w)
    factor, _, terms = S.embed(np.eye(3), ids, offsets, w)  # a row's factor in an item
    out = P.embed(table, *args)
    for part in (slice(0, 4096), slice(2 ** 23, 2 ** 23 + 4096), slice(dim - 4096, dim)):
        rows = table[:, part].double().cpu().numpy()
        _hold_sum(out[:, part], factor @ rows, factor @ np.abs(rows), terms)


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("rows, dim, classes", SHAPES)
def test_gradients_of_h_are_those_of_32_bits(rows, dim, classes, kind):
    """dh of every type within the bars of a float32 dz: those of test_gpu_train_head.py without the 2^-16 of dz that it leaves to bfloat16."""
    P = _api()
    rng = np.random.default_rng(5 * rows + dim)
    (h, eh), (W, eW) = _random(rng, rows, dim, TYPES[kind]), _random(rng, classes, dim, TYPES[kind], 2.0 / np.sqrt(dim))
    q = rng.random((rows, classes)).astype(np.float32)
    ref = S.head_loss(eh, eW, None, q)
    bar = _bars(eh, eW, None, ref, np.ones(rows), 1.0)["dh"] - 2.0 ** -16 * np.abs(ref["dz"]) @ np.abs(eW)
    hold(P.head_loss(h, W, None, _gpu(q))[1], ref["dh"], bar)


def test_matrices_without_rows():
    """Whatever their strides, which numpy's are zeros of."""
    P = _api()
    none = torch.from_numpy(np.zeros((0, 8), dtype=np.float32)).cuda()
    W = torch.ones(3, 8, device="cuda")
    no_ids, no_offsets = torch.empty(0, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    for empty in (none, torch.empty_strided((0, 8), (1, 4), device="cuda"), W[:0]):
        soft, hard = P.head_labels(empty, W)
        assert soft.shape == (0, 3) and hard.shape == (0,)
        loss, dh, dweight, dbias = P.head_loss(empty, W, None, soft)
        assert loss.shape == (0,) and dh.shape == (0, 8) and torch.equal(dweight, torch.zeros_like(W)) and not dbias.any()
        assert P.embed(empty, no_ids).shape == (0, 8) and P.embed(empty, no_ids, no_offsets).shape == (0, 8)
        assert torch.equal(P.embed_grad(empty, no_ids, 5, no_offsets), torch.zeros(5, 8, device="cuda"))


@pytest.mark.parametrize("kind, rows, dim, classes", [("float32", 700, 64, 10), ("bfloat16", 700, 200, 50), ("float16", 300, 520, 20)])
def test_dbias_alone_with_a_gradient_in_the_place_of_h(kind, rows, dim, classes):
    """The kernels that make dbias read h again for a dweight that nobody asked for; dbias and dh are what they are apart from h."""
    from paper_2604_06596_amd import train as T

    rng = np.random.default_rng(4)
    h, _ = _random(rng, rows, dim, TYPES[kind])
    W, _ = _random(rng, classes, dim, TYPES[kind], 2.0 / np.sqrt(dim))
    q = torch.softmax(_random(rng, rows, classes, torch.float32)[0], 1)
    _, dh, _, dbias = _api().head_loss(h, W, None, q)
    L, got = T._library(), torch.empty(classes, device="cuda")
    m, w = T._matrix(h, "h", h.device), T._matrix(W, "weight", h.device)
    call, space = T._call(h.device, L.dynlp_head_loss_workspace(m.rows, m.dim, w.rows, m.type))
    T._check(L.dynlp_head_loss(m, w, None, T._Targets(q.data_ptr(), None, None, None, 1.0), None, m, None, got.data_ptr(), call))
    assert torch.equal(h, dh) and torch.equal(got, dbias)
