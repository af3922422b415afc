"""Whether a result that is rounded once to its type may have come from a 64-bit one with a known error before the rounding."""
import numpy as np


def rounded(x, dtype):
    """64-bit values rounded to a torch type, in 64 bits again."""
    import torch

    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float64)).to(dtype).double().numpy()


def hold(got, exact, error, name=""):
    """got (a tensor on any device): its type's rounding of something within `error` of `exact`.  Rounding keeps order, so that got lies between
    the rounded ends of that interval."""
    values = got.double().cpu().numpy()
    assert values.shape == np.shape(exact), name
    low, high = rounded(exact - error, got.dtype), rounded(exact + error, got.dtype)
    wrong = ~((values >= low) & (values <= high))
    assert not wrong.any(), (name, int(wrong.sum()), values[wrong][:3], np.asarray(exact)[wrong][:3], np.broadcast_to(error, values.shape)[wrong][:3])
