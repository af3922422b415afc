"""Rows of items and the table's gradient against plain sums in 64 bits.

Bars: a float32 sum of k products differs from the exact one by at most (k + 2) 2^-24 times the sum of the magnitudes, whatever the order, and
the result is that sum rounded to its type."""
import numpy as np
import pytest

from oracle import student as S
from rounding import hold

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def _api():
    import paper_2604_06596_amd as P

    return P


def _matrix(rng, rows, dim, dtype, stride=None):
    """(tensor with the given row stride on the GPU, its values in 64 bits)"""
    t = torch.zeros(max(rows, 1), stride or dim, dtype=dtype, device="cuda")
    t[:rows, :dim] = torch.from_numpy(rng.standard_normal((rows, dim))).to(dtype).cuda()
    t = t[:rows, :dim]
    return t, t.double().cpu().numpy()


def _list(rng, count, items, rows, weights=True, bags=True, law="even"):
    """ids with padding and ids out of range, offsets with items of no tokens, weights."""
    if law == "even":
        ids = rng.integers(0, max(rows, 1), count)
    elif law == "one":
        ids = np.full(count, rows // 2)
    else:
        ids = np.minimum((rows * rng.random(count) ** 4).astype(np.int64), rows - 1)
    if law != "one":
        ids = np.where(rng.random(count) < 0.1, -1 - rng.integers(0, 5, count), ids)
    offsets = None
    if bags:
        cuts = np.sort(rng.integers(0, count + 1, max(items - 1, 0)))
        offsets = np.concatenate([[0], cuts, [count]]) if items else np.array([0])
    w = rng.standard_normal(count).astype(np.float32) if weights else None
    return ids, offsets, w


def _gpu(a, dtype=None):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda() if dtype else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _hold(got, exact, magnitude, terms):
    hold(got, exact, (terms[:, None] + 2) * 2.0 ** -24 * magnitude)


# count: nothing, one, a workgroup's list, just beyond what one workgroup holds, several tiles of the sort, pieces that end amid an item
CASES = [
    # count, items, rows, dim, type, weights, bags, law
    (0, 3, 5, 16, "float32", True, True, "even"),
    (1, 1, 1, 1, "float32", False, False, "even"),
    (1, 1, 7, 8, "bfloat16", True, True, "even"),
    (5, 0, 7, 8, "float32", True, True, "even"),
    (37, 1, 301, 64, "float32", True, True, "even"),
    (255, 40, 64, 3, "bfloat16", True, True, "even"),
    (257, 257, 300, 100, "float16", False, False, "even"),
    (2048, 300, 1000, 33, "float32", True, True, "skew"),
    (2049, 300, 1000, 33, "float16", False, True, "skew"),
    (2500, 2000, 50, 257, "bfloat16", True, True, "even"),
    (4099, 1, 500, 64, "float32", True, True, "even"),
    (8192, 100, 40, 20, "float32", True, True, "skew"),
    (8193, 100, 40, 20, "float32", True, True, "skew"),
    (8193, 8193, 9000, 7, "bfloat16", True, False, "even"),
    (9000, 700, 1, 16, "float32", True, True, "even"),
    (12289, 900, 70000, 24, "float16", True, True, "skew"),
    (20001, 37, 255, 520, "bfloat16", True, True, "skew"),
    (20001, 37, 256, 264, "float32", False, True, "even"),
    (30011, 5000, 16777300, 4, "float32", True, True, "even"),
    (40000, 3, 100, 16, "bfloat16", True, True, "one"),
    (70001, 6000, 65536, 16, "float32", True, True, "skew"),
]


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("count, items, rows, dim, kind, weights, bags, law", CASES)
def test_rows_of_items(count, items, rows, dim, kind, weights, bags, law, wide):
    P = _api()
    rng = np.random.default_rng(count + dim)
    rows = min(rows, 70000)
    ids, offsets, w = _list(rng, count, items, rows, weights, bags, law)
    table, exact_table = _matrix(rng, rows, dim, TYPES[kind])
    out = P.embed(table, _gpu(ids, torch.int64 if wide else torch.int32), _gpu(offsets), _gpu(w), 0.75)
    _hold(out, *S.embed(exact_table, ids, offsets, w, 0.75))


@pytest.mark.parametrize("same_type", [False, True])
@pytest.mark.parametrize("count, items, rows, dim, kind, weights, bags, law", CASES)
def test_gradient_of_the_table(count, items, rows, dim, kind, weights, bags, law, same_type):
    P = _api()
    rng = np.random.default_rng(count + dim)
    ids, offsets, w = _list(rng, count, items, rows, weights, bags, law)
    grad, exact_grad = _matrix(rng, items if bags else count, dim, TYPES[kind])
    out = P.embed_grad(grad, _gpu(ids, torch.int32), rows, _gpu(offsets), _gpu(w), 0.75, dtype=TYPES[kind] if same_type else torch.float32)
    some = np.unique(np.concatenate([ids[(ids >= 0) & (ids < rows)], rng.integers(0, rows, 50)]))  # of a very long table: what occurs, and more
    if rows > 100000:
        back = np.full(rows, -1)
        back[some] = np.arange(len(some))
        assert int((out != 0).any(1).sum()) <= len(some)
        out, ids, rows = out[torch.from_numpy(some).cuda()], np.where(ids >= 0, back[np.clip(ids, 0, rows - 1)], -1), len(some)
    _hold(out, *S.embed_grad(exact_grad, ids, rows, offsets, w, 0.75))


@pytest.mark.parametrize("count", [100, 9001])
@pytest.mark.parametrize("kind", list(TYPES))
def test_strides_and_odd_addresses(count, kind):
    """Rows that begin at any multiple of the element's size."""
    P = _api()
    rng = np.random.default_rng(3)
    dtype = TYPES[kind]
    ids, offsets, w = _list(rng, count, 60, 90, True, True)
    i = _gpu(np.concatenate([[0], ids]), torch.int32)[1:]
    wide_w = _gpu(np.concatenate([[0.0], w]).astype(np.float32))[1:]
    table, exact = _matrix(rng, 90, 45, dtype, stride=47)
    odd = torch.zeros(90 * 47 + 1, dtype=dtype, device="cuda")[1:].as_strided((90, 45), (47, 1))
    odd.copy_(table)
    out = P.embed(odd, i, _gpu(offsets), wide_w, 1.0)
    _hold(out, *S.embed(exact, ids, offsets, w, 1.0))
    grad, exact = _matrix(rng, 60, 45, dtype, stride=53)
    _hold(P.embed_grad(grad, i, 90, _gpu(offsets), wide_w), *S.embed_grad(exact, ids, 90, offsets, w))


@pytest.mark.parametrize("count, bags", [(50, True), (50, False), (3000, True), (9001, True), (9001, False)])
def test_what_is_left_out_is_not_looked_at(count, bags):
    """Padding and ids beyond the table: not-a-number weights and rows next to them change nothing; the latter are counted."""
    P = _api()
    rng = np.random.default_rng(4)
    ids, offsets, w = _list(rng, count, 30, 40, True, bags)
    bad = rng.random(count) < 0.05
    ids = np.where(bad, 40 + rng.integers(0, 2 ** 30, count), ids)
    w = np.where((ids < 0) | (ids >= 40), np.nan, w).astype(np.float32)
    table, exact_table = _matrix(rng, 41, 24, torch.float32)
    table[40] = float("nan")
    rejected = torch.tensor([5], dtype=torch.int32, device="cuda")
    out = P.embed(table[:40], _gpu(ids, torch.int32), _gpu(offsets), _gpu(w), 2.0, rejected=rejected)
    exact = S.embed(exact_table[:40], ids, offsets, w, 2.0)
    _hold(out, *exact)
    assert int(rejected) == 5 + bad.sum()
    grad, exact_grad = _matrix(rng, out.shape[0], 24, torch.float32)
    g = P.embed_grad(grad, _gpu(ids, torch.int64), 40, _gpu(offsets), _gpu(w), 2.0, rejected=rejected)
    _hold(g, *S.embed_grad(exact_grad, ids, 40, offsets, w, 2.0))
    assert int(rejected) == 5 + 2 * bad.sum()
    huge = torch.full((count,), 2 ** 40, dtype=torch.int64, device="cuda")
    assert not P.embed(table[:40], huge, _gpu(offsets), _gpu(w)).any()
    assert not P.embed_grad(grad, huge, 40, _gpu(offsets), _gpu(w)).any()


@pytest.mark.parametrize("count", [600, 9001])
def test_infinities_and_not_a_numbers_stay_in_their_rows(count):
    P = _api()
    rng = np.random.default_rng(5)
    ids, offsets, w = _list(rng, count, 50, 300, False, True)
    table, exact = _matrix(rng, 300, 16, torch.float32)
    table[7], exact[7] = float("nan"), np.nan
    table[9], exact[9] = float("inf"), np.inf
    out = P.embed(table, _gpu(ids, torch.int32), _gpu(offsets)).cpu().numpy()
    want = S.embed(exact, ids, offsets)[0]
    assert np.array_equal(np.isnan(out), np.isnan(want)) and np.array_equal(np.isinf(out), np.isinf(want))


@pytest.mark.parametrize("count", [500, 9001])
def test_tokens_outside_the_offsets_belong_to_no_item(count):
    P = _api()
    rng = np.random.default_rng(6)
    ids, _, w = _list(rng, count, 1, 80, True, False)
    offsets = np.array([13, 13, 200, 430, 430])
    table, exact = _matrix(rng, 80, 12, torch.float32)
    _hold(P.embed(table, _gpu(ids, torch.int32), _gpu(offsets), _gpu(w)), *S.embed(exact, ids, offsets, w))
    grad, exact = _matrix(rng, 4, 12, torch.float32)
    _hold(P.embed_grad(grad, _gpu(ids, torch.int32), 80, _gpu(offsets), _gpu(w)), *S.embed_grad(exact, ids, 80, offsets, w))


def test_offsets_beyond_the_list_touch_nothing_outside_it():
    """Offsets are the caller's; wrong ones give wrong sums, but reads stay inside the list."""
    P = _api()
    for count in (500, 9001):
        ids = torch.zeros(count, dtype=torch.int32, device="cuda")
        table = torch.ones(3, 8, device="cuda")
        for offsets in ([-5, 2 ** 40], [2 ** 40, 2 ** 40], [0, count + 1000]):
            out = P.embed(table, ids, torch.tensor(offsets, device="cuda"))
            assert out.shape == (1, 8) and float(out.max()) <= count
            P.embed_grad(torch.ones(1, 8, device="cuda"), ids, 3, torch.tensor(offsets, device="cuda"))
    torch.cuda.synchronize()


@pytest.mark.parametrize("count", [3000, 100003])
def test_the_same_bits_every_time_and_on_another_stream(count):
    P = _api()
    rng = np.random.default_rng(7)
    ids, offsets, w = _list(rng, count, 500, 900, True, True, "skew")
    table, _ = _matrix(rng, 900, 40, torch.bfloat16)
    grad, _ = _matrix(rng, 500, 40, torch.bfloat16)
    args = (_gpu(ids, torch.int32), _gpu(offsets), _gpu(w))
    first = P.embed(table, *args), P.embed_grad(grad, args[0], 900, *args[1:])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = P.embed(table, *args), P.embed_grad(grad, args[0], 900, *args[1:])
    side.synchronize()
    for a, b in zip(first, again):
        assert torch.equal(a, b)


@pytest.mark.parametrize("count", [700, 20011])
def test_replays_of_a_graph(count):
    """Captured once, replayed over new inputs with other work and synchronizations in between."""
    P = _api()
    rng = np.random.default_rng(8)
    ids, offsets, w = _list(rng, count, 200, 1000, True, True, "skew")
    table, _ = _matrix(rng, 1000, 32, torch.float32)
    grad, _ = _matrix(rng, 200, 32, torch.float32)
    i, o, x = _gpu(ids, torch.int32), _gpu(offsets), _gpu(w)
    P.embed_grad(P.embed(table, i, o, x), i, 1000, o, x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = P.embed(table, i, o, x)
        g = P.embed_grad(grad, i, 1000, o, x)
    for k in range(4):
        i.copy_(torch.roll(i, 17 * k + 1))
        table.mul_(1.01)
        grad.add_(0.1)
        graph.replay()
        want = P.embed(table, i, o, x), P.embed_grad(grad, i, 1000, o, x)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(g, want[1])


def test_gradient_against_differences():
    """d/dE of <embed(E), G> by central differences of the definition in 64 bits: the sum is linear, so they are exact up to 1e-9."""
    P = _api()
    rng = np.random.default_rng(9)
    ids, offsets, w = _list(rng, 60, 9, 12, True, True)
    E = rng.standard_normal((12, 5))
    G, exact_G = _matrix(rng, 9, 5, torch.float32)
    got = P.embed_grad(G, _gpu(ids, torch.int32), 12, _gpu(offsets), _gpu(w), 0.5).double().cpu().numpy()
    magnitude, terms = S.embed_grad(exact_G, ids, 12, offsets, w, 0.5)[1:]
    for k in np.ndindex(E.shape):
        up, down = E.copy(), E.copy()
        up[k] += 1e-3
        down[k] -= 1e-3
        d = ((S.embed(up, ids, offsets, w, 0.5)[0] - S.embed(down, ids, offsets, w, 0.5)[0]) * exact_G).sum() / 2e-3
        assert abs(d - got[k]) <= 1e-9 + (terms[k[0]] + 3) * 2.0 ** -24 * magnitude[k]


def test_a_table_beyond_32_bit_offsets():
    """Element offsets of a table of 2.3e9 elements, and of its gradient, pass 32 bits."""
    P = _api()
    rows, dim = 1_100_000, 2048
    table = torch.zeros(rows, dim, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([rows - 1, 5, rows - 1, 1_048_577], dtype=torch.int32, device="cuda")
    table[ids.long()] = torch.tensor([[3.0], [1.0], [3.0], [2.0]], dtype=torch.bfloat16, device="cuda")
    out = P.embed(table, ids, torch.tensor([0, 2, 4], device="cuda"))
    assert float(out[0].min()) == float(out[0].max()) == 4.0 and float(out[1].min()) == float(out[1].max()) == 5.0
    del table
    many = ids.repeat(3000)
    for i in (ids, many):
        g = P.embed_grad(torch.ones(len(i), dim, dtype=torch.bfloat16, device="cuda"), i, rows, dtype=torch.bfloat16)
        n = len(i) // 4
        want = torch.tensor([2.0 * n, n, n], dtype=torch.bfloat16, device="cuda")
        assert torch.equal(g[[rows - 1, 5, 1_048_577]].amax(1), want) and torch.equal(g[[rows - 1, 5, 1_048_577]].amin(1), want)
        assert int((g[:, 0] != 0).sum()) == 3 and int((g[:, -1] != 0).sum()) == 3
        del g


@pytest.mark.parametrize("count, items, rows, dim, kind", [(300007, 21000, 70003, 8, "float32"), (300007, 900, 1500000, 130, "bfloat16")])
def test_long_lists(count, items, rows, dim, kind):
    """Lists long enough for the sort's long tiles, rows narrower and wider than a wave."""
    P = _api()
    rng = np.random.default_rng(count + dim)
    ids, offsets, w = _list(rng, count, items, min(rows, 70003), True, True, "skew")
    table, exact_table = _matrix(rng, 70003, dim, TYPES[kind])
    args = _gpu(ids, torch.int32), _gpu(offsets), _gpu(w)
    _hold(P.embed(table, *args, 0.75), *S.embed(exact_table, ids, offsets, w, 0.75))
    grad, exact_grad = _matrix(rng, items, dim, TYPES[kind])
    out = P.embed_grad(grad, args[0], rows, *args[1:], 0.75)
    assert not out[70003:].any()
    _hold(out[:70003], *S.embed_grad(exact_grad, ids, 70003, offsets, w, 0.75))


def test_a_gradient_larger_than_the_caches():
    """What is written past them is what is written through them (a table of fewer rows)."""
    P = _api()
    rng = np.random.default_rng(21)
    ids, offsets, w = _list(rng, 12000, 700, 5000, True, True, "skew")
    grad, _ = _matrix(rng, 700, 256, torch.float32)
    args = _gpu(ids, torch.int32), _gpu(offsets), _gpu(w)
    small, large = (P.embed_grad(grad, args[0], rows, *args[1:]) for rows in (5000, 150000))
    assert torch.equal(large[:5000], small) and not large[5000:].any()


def test_the_binding_refuses():
    P = _api()
    table = torch.zeros(5, 8, device="cuda")
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    offsets = torch.zeros(2, dtype=torch.int64, device="cuda")
    for call in (lambda: P.embed(table.double(), ids), lambda: P.embed(table.t(), ids), lambda: P.embed(table[0], ids),
                 lambda: P.embed(table, ids.float()), lambda: P.embed(table, ids, offsets.int()), lambda: P.embed(table, ids, offsets[:0]),
                 lambda: P.embed(table, ids, offsets, torch.zeros(2, device="cuda")), lambda: P.embed(table, ids.cpu()),
                 lambda: P.embed(table, ids, rejected=torch.zeros(1, device="cuda")), lambda: P.embed(table[:, ::2], ids),
                 lambda: P.embed_grad(table, ids, 5), lambda: P.embed_grad(table[:3], ids, -1),
                 lambda: P.embed_grad(table[:3], ids, 5, dtype=torch.float16), lambda: P.embed_grad(table[:3], ids, 5, dtype=torch.float64)):
        with pytest.raises(P.DynLPError):
            call()
