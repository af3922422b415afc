"""DynLP on AMD MI355X: dynamic batched label propagation behind a C-ABI HIP library.

``build()`` compiles ``csrc/dynlp.hip`` and ``csrc/dynlp_train.hip`` for gfx950 into ``libdynlp.so`` next to this file;
``DynLP`` (see ``binding``) is a thin ctypes wrapper with the same call names as the C ABI in
``include/dynlp.h``; ``embed``, ``embed_grad``, ``head_labels``, ``head_loss`` and ``adamw_step`` (see ``train``) are those of
``include/dynlp_train.h``, which train and ask a student of the labels.  All computation happens in the HIP kernels; there is no CPU path, and
loading fails loudly if the library has not been built.
"""
from .build import build, library_path  # noqa: F401
from .binding import (DynLP, DynLPError, Stats, InitInfo, INIT_UNIFORM, INIT_SUPERNODE, UPDATE_SYNCHRONOUS, UPDATE_IN_PLACE,
                      load_library, release_kept_memory,  # noqa: F401
                      STATUS)

_TRAIN = ("embed", "embed_grad", "head_labels", "head_loss", "adamw_state", "adamw_step")


def __getattr__(name):
    # on first use: unlike the rest of the package, these need torch
    if name in _TRAIN:
        from . import train

        globals().update((n, getattr(train, n)) for n in _TRAIN)
        return globals()[name]
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
