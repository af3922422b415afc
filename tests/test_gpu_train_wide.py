"""Rows of 256 bytes and more in lists beyond one workgroup's, where a wave has a piece of the list: every type and number of columns per lane, at the
edges that the shorter rows are tested at.  Bars as in test_gpu_train_embed.py."""
import numpy as np
import pytest

from oracle import student as S
from rounding import hold

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
# one, two and four words per lane, a length that is no multiple of a lane's columns, more columns than a wave takes at once
WIDTHS = [("float32", 64), ("float32", 65), ("float32", 100), ("float32", 128), ("float32", 131), ("float32", 300),
          ("bfloat16", 128), ("bfloat16", 129), ("bfloat16", 256), ("bfloat16", 333), ("bfloat16", 520),
          ("float16", 128), ("float16", 131), ("float16", 200), ("float16", 333), ("float16", 520), ("float16", 1030)]


def _api():
    import paper_2604_06596_amd as P

    return P


def _matrix(rng, rows, dim, dtype, stride, odd=0):
    """Matrix on the GPU with rows `stride` apart, `odd` elements behind an aligned address, and its values in 64 bits."""
    t = torch.zeros(rows * stride + odd, dtype=dtype, device="cuda")[odd:].as_strided((rows, dim), (stride, 1))
    t.copy_(torch.from_numpy(rng.standard_normal((rows, dim))))
    return t, t.double().cpu().numpy()


def _list(rng, count, items, rows):
    """ids of which few are frequent, a tenth padding; offsets with empty items; weights."""
    ids = np.where(rng.random(count) < 0.1, -1 - rng.integers(0, 5, count), (rows * rng.random(count) ** 3).astype(np.int64))
    offsets = np.concatenate([[0], np.sort(rng.integers(0, count + 1, items - 1)), [count]])
    return ids.astype(np.int32), offsets, rng.standard_normal(count).astype(np.float32)


def _gpu(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _hold(got, exact, magnitude, terms):
    hold(got, exact, (terms[:, None] + 2) * 2.0 ** -24 * magnitude)


@pytest.mark.parametrize("count, items, odd", [(2049, 300, 0), (9001, 70, 1)])
@pytest.mark.parametrize("kind, dim", WIDTHS)
def test_rows_and_gradients(kind, dim, count, items, odd):
    """odd: rows begin at multiples of the element's size only, ids and weights at those of theirs."""
    P = _api()
    rng = np.random.default_rng(count + dim)
    dtype, rows = TYPES[kind], 90
    ids, offsets, w = _list(rng, count, items, rows)
    args = _gpu(np.concatenate([[0] * odd, ids]).astype(np.int32))[odd:], _gpu(offsets), _gpu(np.concatenate([[0] * odd, w]).astype(np.float32))[odd:]
    table, exact = _matrix(rng, rows, dim, dtype, dim + 3 * odd, odd)
    _hold(P.embed(table, *args, 0.75), *S.embed(exact, ids, offsets, w, 0.75))
    grad, exact = _matrix(rng, items, dim, dtype, dim + 5 * odd, odd)
    want = S.embed_grad(exact, ids, rows, offsets, w, 0.75)
    for out_type in {torch.float32, dtype}:
        _hold(P.embed_grad(grad, args[0], rows, *args[1:], 0.75, dtype=out_type), *want)


SOME = [("float32", 100), ("bfloat16", 256), ("float16", 200)]


@pytest.mark.parametrize("bags", [True, False])
@pytest.mark.parametrize("kind, dim", SOME)
def test_what_is_left_out_is_not_looked_at(kind, dim, bags):
    P = _api()
    rng = np.random.default_rng(4)
    count = 9001
    ids, offsets, w = _list(rng, count, 30, 40)
    bad = rng.random(count) < 0.05
    ids = np.where(bad, 40 + rng.integers(0, 2 ** 30, count), ids).astype(np.int32)
    w = np.where((ids < 0) | (ids >= 40), np.nan, w).astype(np.float32)
    if not bags:
        offsets = None
    table, exact = _matrix(rng, 41, dim, TYPES[kind], dim)
    table[40] = float("nan")
    rejected = torch.zeros(1, dtype=torch.int32, device="cuda")
    o = None if offsets is None else _gpu(offsets)
    out = P.embed(table[:40], _gpu(ids), o, _gpu(w), 2.0, rejected=rejected)
    _hold(out, *S.embed(exact[:40], ids, offsets, w, 2.0))
    grad, exact = _matrix(rng, len(out), dim, TYPES[kind], dim)
    _hold(P.embed_grad(grad, _gpu(ids), 40, o, _gpu(w), 2.0, rejected=rejected), *S.embed_grad(exact, ids, 40, offsets, w, 2.0))
    assert int(rejected) == 2 * bad.sum()


@pytest.mark.parametrize("kind, dim", SOME)
def test_infinities_and_not_a_numbers_stay_in_their_rows(kind, dim):
    P = _api()
    rng = np.random.default_rng(5)
    ids, offsets, _ = _list(rng, 9001, 700, 3000)
    table, exact = _matrix(rng, 3000, dim, TYPES[kind], dim)
    for row, value in ((7, np.nan), (900, np.inf)):
        table[row], exact[row] = float(value), value
    out = P.embed(table, _gpu(ids), _gpu(offsets)).double().cpu().numpy()
    want = S.embed(exact, ids, offsets)[0]
    assert np.array_equal(np.isnan(out), np.isnan(want)) and np.array_equal(np.isinf(out), np.isinf(want)) and 0 < np.isfinite(out).all(axis=1).sum() < 700
    grad, exact = _matrix(rng, 700, dim, TYPES[kind], dim)
    for row, value in ((3, np.nan), (90, -np.inf)):
        grad[row], exact[row] = float(value), value
    out = P.embed_grad(grad, _gpu(ids), 3000, _gpu(offsets)).double().cpu().numpy()
    want = S.embed_grad(exact, ids, 3000, offsets)[0]
    assert np.array_equal(np.isnan(out), np.isnan(want)) and np.array_equal(np.isinf(out), np.isinf(want)) and 0 < np.isfinite(out).all(axis=1).sum() < 3000


@pytest.mark.parametrize("kind, dim", SOME)
def test_tokens_outside_the_offsets_belong_to_no_item(kind, dim):
    P = _api()
    rng = np.random.default_rng(6)
    ids, _, w = _list(rng, 9001, 5, 80)
    offsets = np.array([130, 130, 2000, 4300, 4300])
    table, exact = _matrix(rng, 80, dim, TYPES[kind], dim)
    _hold(P.embed(table, _gpu(ids), _gpu(offsets), _gpu(w)), *S.embed(exact, ids, offsets, w))
    grad, exact = _matrix(rng, 4, dim, TYPES[kind], dim)
    _hold(P.embed_grad(grad, _gpu(ids), 80, _gpu(offsets), _gpu(w)), *S.embed_grad(exact, ids, 80, offsets, w))


@pytest.mark.parametrize("kind, dim", SOME)
def test_the_same_bits_every_time_on_another_stream_and_in_a_graph(kind, dim):
    P = _api()
    rng = np.random.default_rng(7)
    ids, offsets, w = _list(rng, 50003, 500, 900)
    table, _ = _matrix(rng, 900, dim, TYPES[kind], dim)
    grad, _ = _matrix(rng, 500, dim, TYPES[kind], dim)
    i, o, x = _gpu(ids), _gpu(offsets), _gpu(w)

    def both():
        return P.embed(table, i, o, x), P.embed_grad(grad, i, 900, o, x)

    first = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for k in range(4):
        i.copy_(torch.roll(i, 17 * k + 1))
        table.mul_(1.01)
        grad.add_(0.1)
        graph.replay()
        want = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
