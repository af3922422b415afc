"""Compile the HIP library for gfx950 (cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess
import tempfile

_HERE = os.path.dirname(os.path.abspath(__file__))
_ROOT = os.path.dirname(_HERE)
_SRC = [os.path.join(_HERE, "csrc", name) for name in ("dynlp.hip", "dynlp_train.hip", "dynlp_teach.hip")]
_SO = os.path.join(_HERE, "libdynlp.so")


def library_path() -> str:
    return _SO


def _run(commands, verbose):
    """All at once; the first that fails is raised."""
    jobs = [subprocess.Popen(c, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for c in commands]
    said = [j.communicate()[0] for j in jobs]
    for job, text in zip(jobs, said):
        if verbose or job.returncode != 0:
            print(text)
    for job, text in zip(jobs, said):
        if job.returncode != 0:
            raise RuntimeError("hipcc failed:\n" + text[-4000:])


def build(verbose: bool = False) -> str:
    """hipcc -> paper_2604_06596_amd/libdynlp.so.  Always recompiles; the sources at the same time."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    flags = [
        "-O3", "--offload-arch=gfx950", "-std=c++17", "-fPIC", "-pthread",
        # packed-FP32 instruction selection is switched off for all device code
        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
        "-I", os.path.join(_ROOT, "include"), "-I", os.path.join(_HERE, "csrc"),
    ]
    with tempfile.TemporaryDirectory(prefix="dynlp_build_") as space:
        objects = [os.path.join(space, os.path.basename(s) + ".o") for s in _SRC]
        _run([[hipcc, *flags, "-c", s, "-o", o] for s, o in zip(_SRC, objects)], verbose)
        _run([[hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-pthread", "-o", _SO + ".tmp", *objects]], verbose)
    os.replace(_SO + ".tmp", _SO)
    return _SO


if __name__ == "__main__":
    print(build(verbose=True))
