"""What scores and learning from a teacher refuse before anything is enqueued, and their definitions against differences.  Addresses are never
looked at: these run without a GPU, and none of the calls would be accepted."""
import numpy as np
import pytest

from oracle import student as S
from paper_2604_06596_amd import train as T

A = 1 << 20  # an address that is aligned to everything


def _refused(status, word):
    assert status == -1
    assert word in T._lib.dynlp_last_error(None).decode()


def _scores(**more):
    s = dict(given=1, top=2, classes=A << 4, log_given=A << 5, entropy=A << 6, top_classes=A << 7, log_top=A << 8, rejected=None)
    s.update(more)
    return T._Scores(**s)


@pytest.mark.parametrize("more, word", [(dict(given=-1), "given"), (dict(given=(1 << 20) + 1), "given"), (dict(top=-1), "first"), (dict(top=129), "first"),
                                        (dict(top=11), "first 11 of 10"), (dict(classes=None), "without classes"), (dict(log_given=None), "without log_given")])
def test_scores(more, word):
    L = T._library()
    call = T._Call(None, A << 10, 1 << 40)
    x = T._Matrix(A, 5, 10, 10, 0)
    _refused(L.dynlp_row_scores(x, 0, _scores(**more), call), word)
    _refused(L.dynlp_head_scores(T._Matrix(A, 5, 8, 8, 0), T._Matrix(A << 1, 10, 8, 8, 0), None, _scores(**more), call), word)


def test_heads():
    L = T._library()
    call = T._Call(None, A << 10, 1 << 50)
    h, w = T._Matrix(A, 5, 8, 8, 1), T._Matrix(A << 1, 10, 8, 8, 1)
    teacher = T._Teacher(A << 4, A << 5, None, None, 3, 1.0, 1.0)
    bad = [(T._Matrix(A << 1, 10, 8, 8, 0), "type"), (T._Matrix(A << 1, 10, 9, 9, 1), "rows of 9"), (T._Matrix(A << 1, 0, 8, 8, 1), "classes"),
           (T._Matrix(A << 1, (1 << 22) + 1, 8, 8, 1), "classes"), (None, "weight is NULL")]
    for weight, word in bad:
        _refused(L.dynlp_head_scores(h, weight, None, _scores(), call), word)
        _refused(L.dynlp_head_distill(h, weight, None, teacher, A << 6, None, None, None, call), word)
    long = (1 << 16) + 1
    _refused(L.dynlp_head_scores(T._Matrix(A, 5, long, long, 1), T._Matrix(A << 8, 10, long, long, 1), None, _scores(), call), "elements")
    wide = T._Matrix(A << 1, 100, 8, 8, 1)  # up to 64 classes take no workspace
    _refused(L.dynlp_head_scores(h, wide, None, _scores(), T._Call(None, None, 0)), "workspace")
    _refused(L.dynlp_head_scores(h, wide, None, _scores(), T._Call(None, (A << 10) + 16, 1 << 50)), "aligned")
    _refused(L.dynlp_head_distill(h, wide, None, teacher, A << 6, None, None, None, T._Call(None, A << 10, 1)), "workspace")
    _refused(L.dynlp_head_scores(h, w, None, _scores(), None), "call is NULL")
    _refused(L.dynlp_head_scores(h, w, None, None, call), "scores is NULL")
    _refused(L.dynlp_head_distill(h, w, None, None, A << 6, None, None, None, call), "teacher is NULL")


@pytest.mark.parametrize("change, word", [(dict(kept=0), "lists of 0"), (dict(kept=129), "lists of 129"), (dict(classes=None), "without classes"), (dict(logits=None), "without logits"),
                                          (dict(temperature=0.0), "temperature"), (dict(temperature=-1.0), "temperature"), (dict(temperature=float("nan")), "temperature"),
                                          (dict(temperature=float("inf")), "temperature"), (dict(temperature=1e-39), "temperature"), (dict(temperature=1e25), "temperature"),
                                          (dict(grad_scale=float("inf")), "grad_scale"), (dict(grad_scale=1e30, temperature=1e15), "grad_scale")])
def test_teachers(change, word):
    L = T._library()
    t = dict(classes=A << 4, logits=A << 5, row_weight=None, rejected=None, kept=3, temperature=1.0, grad_scale=1.0)
    t.update(change)
    _refused(L.dynlp_head_distill(T._Matrix(A, 5, 8, 8, 1), T._Matrix(A << 1, 10, 8, 8, 1), None, T._Teacher(**t), A << 6, None, None, None,
                                  T._Call(None, A << 10, 1 << 40)), word)


def test_outputs_in_the_memory_of_inputs():
    L = T._library()
    h, w = T._Matrix(A, 5, 8, 8, 1), T._Matrix(A << 1, 10, 8, 8, 1)
    teacher = T._Teacher(A << 4, A << 5, None, None, 3, 1.0, 1.0)

    def call(dh=None, dweight=None):
        return L.dynlp_head_distill(h, w, None, teacher, A << 6, dh, dweight, None, T._Call(None, A << 10, 1 << 40))

    _refused(call(T._Matrix(A, 5, 8, 8, 1)), "dh overlaps h")
    _refused(call(T._Matrix((A << 1) + 16, 5, 8, 8, 1)), "dh overlaps weight")
    _refused(call(T._Matrix(A << 2, 5, 8, 8, 0)), "dh has another")
    _refused(call(T._Matrix(A << 2, 4, 8, 8, 1)), "dh has another")
    _refused(call(None, T._Matrix(A + 32, 10, 8, 8, 0)), "dweight overlaps h")
    _refused(call(None, T._Matrix(A << 1, 10, 8, 8, 1)), "dweight overlaps weight")
    _refused(call(T._Matrix(A << 2, 5, 8, 8, 1), T._Matrix(A << 2, 10, 8, 8, 0)), "dweight overlaps dh")
    _refused(call(None, T._Matrix(A << 2, 10, 8, 8, 2)), "dweight has type 2")
    _refused(call(None, T._Matrix(A << 2, 11, 8, 8, 1)), "dweight has another")


def test_workspaces_of_sizes_that_no_call_takes():
    L = T._library()
    assert L.dynlp_head_scores_workspace(0, 8, 10, 0) == 0 and L.dynlp_head_scores_workspace(5, 8, (1 << 22) + 1, 0) == 0
    assert L.dynlp_head_distill_workspace(0, 8, 10, 1, 0, 0) == 0 and L.dynlp_head_distill_workspace(5, 8, 10, 0, 0, 0) == 0
    assert 0 < L.dynlp_head_distill_workspace(5, 8, 100, 1, 1, -1) < L.dynlp_head_distill_workspace(5, 8, 100, 1, 1, 1)
    # up to 64 classes: none for scores and the loss, that of head_loss for gradients
    assert L.dynlp_head_scores_workspace(5, 8, 64, 1) == 0 and L.dynlp_head_distill_workspace(5, 8, 64, 1, 1, -1) == 0
    assert L.dynlp_head_distill_workspace(500, 8, 64, 1, 1, 1) == L.dynlp_head_loss_workspace(500, 8, 64, 1) > 0
    # whatever the rows, no more than some GiB, the head itself apart
    for rows, classes in ((1, 1 << 22), (1 << 20, 1 << 22), ((1 << 31) - 2, 65)):
        for t in (0, 1, 2):
            assert 0 < L.dynlp_head_scores_workspace(rows, 64, classes, t) < 8 << 30
            assert 0 < L.dynlp_head_distill_workspace(rows, 64, classes, 8, t, 0) < 32 << 30


def test_the_definition_of_scores():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((4, 9))
    log_p, entropy, order = S.scores(x)
    p = np.exp(x) / np.exp(x).sum(axis=1, keepdims=True)
    np.testing.assert_allclose(log_p, np.log(p), atol=1e-14)
    np.testing.assert_allclose(entropy, -(p * np.log(p)).sum(axis=1), atol=1e-14)
    np.testing.assert_allclose(S.scores(3.0 * p, True)[0], np.log(p), atol=1e-14)
    assert (order == np.argsort(-x, axis=1)).all()
    log_p, entropy, order = S.scores([[-np.inf, -np.inf], [0.0, -np.inf], [np.nan, 1.0]])
    np.testing.assert_allclose(log_p[0], -np.log(2.0))
    assert entropy[1] == 0.0 and log_p[1, 1] == -np.inf and np.isnan(log_p[2]).all() and order[2].tolist() == [1, 0]


def test_the_definition_of_learning_from_lists():
    """Its gradients against differences, one class against the cross entropy of a hard label."""
    rng = np.random.default_rng(1)
    h, W, b = rng.standard_normal((5, 4)), rng.standard_normal((7, 4)), rng.standard_normal(7)
    at = np.array([[0, 3, 6], [1, 1, -1], [2, 9, 4], [5, 0, 1], [6, 2, 3]])
    u, r = rng.standard_normal((5, 3)), rng.random(5)
    ref = S.distill(h, W, b, at, u, 1.7, r, 0.3)
    for k, name in enumerate(("dh", "dweight", "dbias")):
        v = rng.standard_normal(ref[name].shape)
        f = lambda t: 0.3 * S.distill(*(x + t * v if j == k else x for j, x in enumerate((h, W, b))), at, u, 1.7, r)["loss"].sum()  # noqa: E731
        np.testing.assert_allclose((f(1e-5) - f(-1e-5)) / 2e-5, (ref[name] * v).sum(), rtol=1e-7, atol=1e-9)
    one, want = S.distill(h, W, b, at[:, :1], u[:, :1]), S.head_loss(h, W, b, hard=at[:, 0])
    for name in ("loss", "dh", "dweight", "dbias"):
        np.testing.assert_allclose(one[name], want[name], atol=1e-12)
