"""What the student's operators refuse before anything is enqueued: outputs in the memory of inputs, numbers that 32 bits do not hold.  Addresses are
never looked at: these run without a GPU, and none of them is a call that would be accepted."""
import itertools

import numpy as np
import pytest

from paper_2604_06596_amd import train as T

A = 1 << 20  # an address that is aligned to everything


def _refused(status, word):
    assert status == -1
    assert word in T._lib.dynlp_last_error(None).decode()


def _rows(data, rows, stride, width):
    """The bytes of a float32 matrix."""
    return {data + 4 * (i * stride + k) + b for i in range(rows) for k in range(width) for b in range(4)}


def _loss(h, dh, weight=None, dweight=None, classes=3):
    L = T._library()
    w = weight or T._Matrix(A << 10, classes, h.dim, h.dim, 0)
    call = T._Call(None, A << 12, L.dynlp_head_loss_workspace(h.rows, h.dim, w.rows, 0))
    return L.dynlp_head_loss(h, w, None, T._Targets(A << 14, None, None, None, 1.0), A << 16, dh, dweight, None, call)


@pytest.mark.parametrize("stride", [8, 11, 16, 24])
def test_dh_that_meets_h_is_refused_wherever_it_lies(stride):
    """Every place of a dh of the same stride around h: refused if a byte of it is one of h's."""
    rows, dim = 5, 8
    h = T._Matrix(A, rows, stride, dim, 0)
    own = _rows(A, rows, stride, dim)
    met = 0
    for shift in range(-(rows + 1) * stride, (rows + 1) * stride + 1):
        at = A + 4 * shift
        if own & _rows(at, rows, stride, dim):
            met += 1
            _refused(_loss(h, T._Matrix(at, rows, stride, dim, 0), dweight=A << 18), "dh overlaps h")
            if shift:
                _refused(_loss(h, T._Matrix(at, rows, stride, dim, 0)), "dh overlaps h")
    assert met >= rows + 4


def test_dh_of_another_stride_that_meets_h_is_refused():
    rows, dim = 4, 6
    for a, b, shift in itertools.product((6, 9, 12), (6, 8, 12, 30), range(-40, 41)):
        h, at = T._Matrix(A, rows, a, dim, 0), A + 4 * shift
        if a != b and _rows(A, rows, a, dim) & _rows(at, rows, b, dim):
            _refused(_loss(h, T._Matrix(at, rows, b, dim, 0), dweight=A << 18), "dh overlaps h")


def test_one_row_has_no_stride():
    h = T._Matrix(A, 1, 8, 8, 0)
    _refused(_loss(h, T._Matrix(A, 1, 1 << 40, 8, 0), dweight=A << 18), "dh overlaps h")
    _refused(_loss(h, T._Matrix(A + 4, 1, 1 << 40, 8, 0)), "dh overlaps h")


def test_other_outputs_in_the_memory_of_inputs_are_refused():
    L = T._library()
    h = T._Matrix(A, 5, 8, 8, 0)
    _refused(_loss(h, T._Matrix((A << 10) + 64, 5, 8, 8, 0)), "overlaps weight")
    tokens = T._Tokens(7, 5, A << 10, A << 11, None, None, 1.0, 0)
    call = T._Call(None, None, 0)
    table = T._Matrix(A, 50, 16, 16, 0)
    _refused(L.dynlp_embed(table, tokens, T._Matrix(A + 49 * 64, 5, 16, 16, 0), call), "out overlaps the table")
    _refused(L.dynlp_embed_grad(T._Matrix(A, 5, 16, 16, 1), tokens, T._Matrix(A + 64, 50, 16, 16, 0), call), "out overlaps grad")
    huge = T._Matrix(A, 2 ** 31 - 2, 1 << 40, 16, 0)  # rows times stride pass 64 bits
    _refused(L.dynlp_embed(huge, tokens, T._Matrix(A + (1 << 50), 5, 1 << 40, 16, 0), call), "out overlaps the table")


@pytest.mark.parametrize("option, decay, word", [(dict(eps=1e-50), 0.0, "eps"), (dict(eps=1e39), 0.0, "eps"), (dict(lr=1e39), 0.0, "lr"),
                                                 (dict(lr=1e35, beta1=0.99999), 0.0, "lr"), (dict(lr=1e30), 1e30, "weight_decay")])
def test_adamw_refuses_what_32_bits_do_not_hold(option, decay, word):
    """eps that is nothing in 32 bits would divide a zero gradient's step by zero; a step or a decay that is infinite leaves no parameter."""
    table = np.zeros(1, dtype=T._ADAMW_TENSOR)
    for name, value in dict(n=10, param=A, grad=A << 1, m=A << 2, v=A << 3, weight_decay=decay).items():
        table[name] = value
    o = dict(dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, grad_scale=None, seed=0, state_bits=32), **option)
    _refused(T._library().dynlp_adamw_step(1, table.ctypes.data, T._AdamwOptions(**o), T._Call(None, None, 0)), word)
