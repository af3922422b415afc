"""The student's operators where lists, rows and arguments are unlike those of a batch of texts: offsets that miss the list, long runs of items
without tokens, more items than one launch has workgroups, outputs in the inputs' memory, factors that are not finite.

Bars as in test_gpu_train_embed.py and test_gpu_train_head.py."""
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
