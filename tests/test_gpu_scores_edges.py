"""Scores where the numbers themselves are hard.  Bars as in test_gpu_scores."""
import numpy as np
import pytest

from oracle import student as S
from rounding import hold
from test_gpu_scores import TYPES, U, _api, _bars, _check, _head

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

PATHS = [(65536 + 5, 50, 4), (40, 50, 4), (40, 50, 20), (5, 3, 1), (40, 300, 5), (40, 1500, 70), (600, 3001, 5), (9, 9000, 5), (2050, 4100, 40)]  # a lane, 16 lanes, 1, 4, 16 waves and 1 for a row


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


@pytest.mark.parametrize("rows", [3, 20, 150])
def test_large_and_tiny_values_of_wide_heads(rows):
    """More than 64 classes and 16 rows, where operands in 32 bits become bfloat16 terms: values that rounding to bfloat16 would make infinite, and those that have no
    second or third term."""
    P = _api()
    classes = 80
    h = torch.zeros(rows, 3, device="cuda")
    W = torch.zeros(classes, 3, device="cuda")
    h[0] = torch.tensor([3.4028234e38, 1.0, 0.0])
    h[1] = torch.tensor([1e-30, 2.0 ** -100, 1.0])
    h[2] = torch.tensor([2.0 ** -60, 1.0 + 2.0 ** -20, 3.0])
    W[:2] = torch.tensor([[1.0, 2.0, 3.0], [-1.0, 0.0, 1.0]])
    W[2] = torch.tensor([2.0 ** 60, 2.0 ** -120, 0.0])
    b = torch.full((classes,), -100.0, device="cuda")
    b[:3] = torch.tensor([0.0, 0.0, -float("inf")])
    z = h.double() @ W.double().t() + b.double()
    z[:, 2] = -float("inf")
    z = z.cpu().numpy()
    out = P.head_scores(h, W, b, top=3)
    assert out.top[0].tolist()[:1] == [0] and float(out.log_top[0, 0]) == 0.0 and float(out.log_top[0, 1]) < -1e38
    log_bar, entropy_bar = _bars(z[1:], False)
    off = 26 * U * (np.abs(h.double().cpu().numpy()[1:]) @ np.abs(W.double().cpu().numpy())[[0, 1]].T).max(axis=1)
    log_p, entropy, order = S.scores(z[1:])
    at = np.arange(rows - 1)[:, None]
    assert np.array_equal(out.top[1:].cpu().numpy(), order[:, :3])
    hold(out.log_top[1:], log_p[at, order[:, :3]], log_bar[at, order[:, :3]] + 2 * off[:, None], "log_top")
    hold(out.entropy[1:], entropy, entropy_bar + off * (2 + 2 * np.abs(np.where(np.isfinite(log_p), log_p, 0.0)).max(axis=1)), "entropy")


@pytest.mark.parametrize("kind, rows, dim, classes", [("bfloat16", 3000, 32, 131072), ("float32", 2300, 20, 131000), ("float16", 500, 40, 1500000)])
def test_turns(kind, rows, dim, classes):
    """More logits than are in memory at a time (1 GiB), a shorter last turn: every row's scores against the definition, on a grid on which logits are exact."""
    P = _api()
    from paper_2604_06596_amd import train as T

    rng = np.random.default_rng(rows)
    assert T._library().dynlp_head_scores_workspace(rows, dim, classes, T._TYPES[TYPES[kind]]) < 4 * rows * classes  # logits of some rows at a time
    h, W, b, eh, eW, eb = _head(rng, rows, dim, classes, TYPES[kind], True)
    given = torch.from_numpy(rng.integers(-1, classes, size=(rows, 2)).astype(np.int32)).cuda()
    out = P.head_scores(h, W, b, given=given, top=4)
    w64, b64 = W.double().t().contiguous(), b.double()
    n = (2 * -(-classes // 64) + 64) * U
    for at in range(0, rows, 100):
        some = slice(at, at + 100)
        z = h[some].double() @ w64 + b64
        order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :4]
        assert torch.equal(out.top[some].long(), order)
        d = z.amax(1, keepdim=True) - z
        z -= torch.logsumexp(z, 1, keepdim=True)
        p = z.exp()
        mean, square, log_s = (p * d).sum(1), (p * d * d).sum(1), -z.amax(1)
        log_bar = (n + U * mean + 3 * U * log_s)[:, None] + U * (3 * d - 2 * z)
        g = given[some].long()
        real = g >= 0
        for got, want, bar in ((out.log_top[some], z.gather(1, order), log_bar.gather(1, order)),
                               (out.log_given[some][real], z.gather(1, g.clamp(min=0))[real], log_bar.gather(1, g.clamp(min=0))[real]),
                               (out.entropy[some], -(p * z).sum(1), n * (2 + 2 * mean) + U * (5 * mean + 4 * square + 4 * log_s))):
            assert ((got.double() - want).abs() <= bar + U * want.abs()).all(), at
        assert (out.log_given[some][~real] == 0).all()


@pytest.mark.parametrize("rows", [3, 20])
def test_the_largest_number_of_classes(rows):
    """2^22 classes, few rows by themselves and a tile of them, on a grid on which logits are exact; the last classes among the first."""
    P = _api()
    classes, dim = 1 << 22, 16
    g = torch.Generator(device="cuda").manual_seed(rows)
    h = (torch.randint(-8, 9, (rows, dim), generator=g, device="cuda") / 8.0).to(torch.bfloat16)
    W = (torch.randint(-32, 33, (classes, dim), generator=g, device="cuda") / 64.0).to(torch.bfloat16)
    b = torch.randint(-64, 65, (classes,), generator=g, device="cuda") / 64.0
    b[[0, classes - 1]] = 30.0
    given = torch.tensor([0, classes - 1, classes, -1], dtype=torch.int32, device="cuda").repeat(rows, 1)
    rejected = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = P.head_scores(h, W, b, given=given, top=128, rejected=rejected)
    assert int(rejected) == rows and (out.log_given[:, 2:] == 0).all()
    z = h.double() @ W.double().t() + b.double()
    order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :128]
    assert torch.equal(out.top.long(), order)
    d = z.amax(1, keepdim=True) - z
    z -= torch.logsumexp(z, 1, keepdim=True)
    p = z.exp()
    n = (2 * classes // 64 + 64) * U
    mean, square, log_s = (p * d).sum(1), (p * d * d).sum(1), -z.amax(1)
    log_bar = (n + U * mean + 3 * U * log_s)[:, None] + U * (3 * d - 3 * z)
    for got, at in ((out.log_top, order), (out.log_given[:, :2], given[:, :2].long())):
        assert ((got.double() - z.gather(1, at)).abs() <= log_bar.gather(1, at)).all()
    assert ((out.entropy.double() + (p * z).sum(1)).abs() <= n * (2 + 2 * mean) + U * (6 * mean + 4 * square + 5 * log_s)).all()


@pytest.mark.parametrize("kind", ["float32", "bfloat16", "float16", "probabilities"])
@pytest.mark.parametrize("rows, classes, top, given", [(2048, 2049, 128, 1), (2050, 5003, 9, 2), (2047, 5003, 32, 0)])
def test_many_long_rows(rows, classes, top, given, kind):
    """A wave for each row that takes several turns through it (2,047 rows: four waves): equal values, rising and falling ones, masks, rows of nothing."""
    P = _api()
    g = torch.Generator(device="cuda").manual_seed(rows + classes)
    probabilities = kind == "probabilities"
    dtype = TYPES.get(kind, torch.float32)
    x = 3.0 * torch.randn(rows, classes, generator=g, device="cuda")
    at = torch.arange(classes, device="cuda").float()
    x[0], x[1], x[2] = 0.0, at / 64.0, -at / 64.0
    x[3] = torch.where(at > classes - 300, 5.0 + at % 7, -1.0)
    x[4] = at * 7 % 5
    if probabilities:
        x = torch.softmax(x, 1)
        x[5] = 0.0
    else:
        x[5:300, classes // 3:classes // 2] = -float("inf")
        x[6] = -float("inf")
        x[7, :-1] = -float("inf")
    wide = torch.zeros(rows, classes + 3, dtype=dtype, device="cuda")
    wide[:, :classes] = x.to(dtype)
    t = wide[:, :classes]
    ids = torch.randint(-1, classes, (rows, given), generator=g, device="cuda", dtype=torch.int32) if given else None
    out = P.row_scores(t, given=ids, top=top, probabilities=probabilities)
    some = np.concatenate([np.arange(310), np.arange(310, rows, 29), [rows - 1]])
    e = t[torch.from_numpy(some).cuda()].double().cpu().numpy()
    keep = some != 5 if probabilities else np.ones(len(some), bool)  # a row of zeros has bars of no size
    pick = torch.from_numpy(some[keep]).cuda()
    _check(type(out)(None if ids is None else out.log_given[pick], out.entropy[pick], out.top[pick], out.log_top[pick]), e[keep], probabilities,
           None if ids is None else ids[pick].cpu().numpy(), top)
    if probabilities:
        assert out.top[5].tolist() == list(range(top)) and torch.allclose(out.entropy[5], torch.tensor(float(np.log(classes)), device="cuda"), rtol=4 * U, atol=0)
