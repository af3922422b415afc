"""Scores where the numbers themselves are hard.  Bars as in test_gpu_scores."""
import numpy as np
import pytest

from oracle import student as S
from rounding import hold
from test_gpu_scores import TYPES, U, _api, _bars, _check, _head

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

PATHS = [(65536 + 5, 50, 4), (40, 50, 4), (40, 50, 20), (5, 3, 1), (40, 300, 5), (40, 1500, 70), (600, 3001, 5), (9, 9000, 5)]  # a lane, 16 lanes, 1, 4 and 16 waves for a row


@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows, classes, top", PATHS)
def test_probabilities_of_all_sizes(rows, classes, top, kind):
    """Denormal ones beside others (a softmax of logits that lie up to 100 apart), rows of nothing but denormal ones, rows of tiny sums and of huge ones, which 32 bits do
    not hold: the scores are those of x over the sum of x, whatever that is."""
    P = _api()
    rng = np.random.default_rng(classes + top)
    x = rng.random((8, classes)) + 0.01
    x[0] = np.exp(-100.0 * np.arange(classes) / max(classes - 1, 1))
    x[1] = np.where(np.arange(classes) % 3 == 0, 1e-40, 1.0 / classes)
    x[2] *= 1e-39
    x[3] = 0.0
    x[3, classes // 2:] = 2e-40
    x[4] *= 1e-38
    x[5] *= 1e-25
    x[6] *= 1e37
    x[7] *= 3e30
    t = torch.from_numpy(x).to(TYPES[kind]).cuda()
    t = t.repeat(-(-rows // 8), 1)[:rows].contiguous()
    given = rng.integers(-1, classes, size=(rows, 2)).astype(np.int32)
    out = P.row_scores(t, given=torch.from_numpy(given).cuda(), top=top, probabilities=True)
    assert torch.isfinite(out.entropy).all()
    _check(out, t.double().cpu().numpy(), True, given, top)


@pytest.mark.parametrize("rows, classes, top", PATHS)
def test_infinite_probabilities(rows, classes, top):
    """A row with one says nothing; the others beside it are what they are without it."""
    P = _api()
    x = torch.rand(rows, classes, generator=torch.Generator(device="cuda").manual_seed(classes), device="cuda")
    given = torch.zeros(rows, dtype=torch.int32, device="cuda")
    want = P.row_scores(x, given=given, top=top, probabilities=True)
    x[2, classes - 1] = float("inf")
    got = P.row_scores(x, given=given, top=top, probabilities=True)
    assert torch.isnan(got.entropy[2]) and torch.isnan(got.log_given[2]) and torch.isnan(got.log_top[2]).all()
    keep = torch.arange(rows, device="cuda") != 2
    for a, b in zip(got, want):
        assert torch.equal(a[keep], b[keep])


@pytest.mark.parametrize("rows", [16, 17, 60, 300])
def test_infinite_elements_of_heads_in_32_bits(rows):
    """Up to 16 rows an infinite element makes logits that are infinite, as in the definition; from 17 rows on every logit that it meets is not a number, whatever the
    other element is, and its row has no scores."""
    P = _api()
    rng = np.random.default_rng(rows)
    classes, dim = 100, 40
    h, W, b, eh, eW, eb = _head(rng, rows, dim, classes, torch.float32, False)
    given = torch.full((rows,), 5, dtype=torch.int32, device="cuda")
    for at in (1.0 + 2.0 ** -9 + 2.0 ** -18, 1.0, 1.0 + 2.0 ** -9, -1.5):  # three terms of one sign, one, two; another sign
        h[1:, 7], h[2, 7] = 0.5, at
        W[5, 7] = -float("inf")
        out = P.head_scores(h, W, b, given=given, top=3)
        if rows <= 16:
            fine = [1] + list(range(3, rows)) + ([2] if at > 0 else [])
            assert torch.isfinite(out.entropy[fine]).all() and (out.log_given[fine] == -float("inf")).all()
        else:
            assert torch.isnan(out.entropy).all() and torch.isnan(out.log_given).all() and torch.isnan(out.log_top).all()
        W[:, 7] = at
        h[2, 7] = float("inf")
        out = P.head_scores(h, W, b, given=given, top=3)
        assert torch.isfinite(out.entropy[3:]).all()
        if rows > 16 or at > 0:
            assert torch.isnan(out.entropy[2]) and torch.isnan(out.log_top[2]).all() and out.top[2].tolist() == [0, 1, 2]
