"""The definition of learning from lists, held to its formula where a list names a class several times."""
import numpy as np
import pytest

from oracle import student as S


@pytest.mark.parametrize("temperature", [1.0, 2.5])
def test_a_class_that_is_named_several_times_has_the_sum_of_its_probabilities(temperature):
    """The divergence of one distribution over classes from another: never below zero, zero where they are the same, and that of the list with each class once."""
    rng = np.random.default_rng(0)
    h, W, b = rng.standard_normal((6, 4)), rng.standard_normal((5, 4)), rng.standard_normal(5)
    at = rng.integers(0, 5, size=(6, 7))
    u = rng.standard_normal((6, 7))
    ref = S.distill(h, W, b, at, u, temperature)
    q, p = ref["target"], ref["soft"]
    np.testing.assert_allclose(q.sum(axis=1), 1.0)
    with np.errstate(divide="ignore", invalid="ignore"):
        want = temperature ** 2 * np.where(q > 0, q * (np.log(q) - np.log(p)), 0.0).sum(axis=1)
    np.testing.assert_allclose(ref["loss"], want, rtol=1e-12)
    assert (ref["loss"] > 0).all()
    once = S.distill(h, W, b, np.tile(np.arange(5), (6, 1)), temperature * np.log(np.maximum(q, 1e-300)), temperature)
    for name in ("loss", "dh", "dweight", "dbias"):
        np.testing.assert_allclose(ref[name], once[name], rtol=1e-9, atol=1e-12)
    sure = np.array([-np.inf, 0.0, -np.inf, -np.inf, -np.inf])
    assert abs(S.distill(np.zeros((1, 4)), W, sure, np.array([[1, 1, 1]]), rng.standard_normal((1, 3)))["loss"][0]) < 1e-15


@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_a_list_with_what_is_no_number(bad):
    """Its row's dz is none for every class; others are what they are without it."""
    rng = np.random.default_rng(1)
    h, W, b = rng.standard_normal((3, 4)), rng.standard_normal((6, 4)), rng.standard_normal(6)
    at, u = np.array([[0, 1], [2, 3], [4, 5]]), rng.standard_normal((3, 2))
    want = S.distill(h, W, b, at, u)
    u[1, 0] = bad
    ref = S.distill(h, W, b, at, u)
    assert np.isnan(ref["dz"][1]).all() and np.isnan(ref["loss"][1]) and np.isnan(ref["dh"][1]).all() and np.isnan(ref["dweight"]).all()
    np.testing.assert_array_equal(ref["dz"][[0, 2]], want["dz"][[0, 2]])


@pytest.mark.parametrize("temperature", [2.95e-39, 3.5e-39, 4.2e-39])
def test_temperatures_that_make_powers_of_two_infinite_are_refused(temperature):
    """Exponents are multiplied by log2(e) / T, which 32 bits do not hold here although they do 1 / T.  No GPU is needed to be refused."""
    from paper_2604_06596_amd import train as T

    a = 1 << 20
    L = T._library()
    assert np.isfinite(np.float32(1.0) / np.float32(temperature))
    for classes in (10, 100):
        status = L.dynlp_head_distill(T._Matrix(a, 5, 8, 8, 1), T._Matrix(a << 1, classes, 8, 8, 1), None, T._Teacher(a << 4, a << 5, None, None, 3, temperature, 1.0), a << 6,
                                      None, None, None, T._Call(None, a << 10, 0))
        assert status == -1 and ("temperature" in T._lib.dynlp_last_error(None).decode())
