"""Compile the HIP libraries for gfx950 in-tree (hipcc cross-compiles without a GPU)."""
from __future__ import annotations

import os
import subprocess

_HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(_HERE, "csrc")
LIB_PATH = os.path.join(_HERE, "libchicle_round.so")
CSRC_TRAIN = os.path.join(_HERE, "csrc_train")
TRAIN_LIB_PATH = os.path.join(_HERE, "libchicle_train.so")

HIPCC_FLAGS = [
    "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-shared",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-munsafe-fp-atomics", "-Wall", "-Wno-unused-function",
]


def sources():
    return [os.path.join(CSRC, "chicle_round.hip")]


def train_sources():
    return [os.path.join(CSRC_TRAIN, name) for name in ("chicle_train.hip", "sequence.hip")]


def _compile(path: str, files, verbose: bool) -> str:
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    tmp = path + ".tmp%d" % os.getpid()
    cmd = [hipcc] + HIPCC_FLAGS + ["-o", tmp] + files
    if verbose:
        print(" ".join(cmd))
    subprocess.check_call(cmd)
    os.replace(tmp, path)
    return path


def build_library(verbose: bool = False) -> str:
    """Run hipcc unconditionally and return the path of the round's shared library."""
    return _compile(LIB_PATH, sources(), verbose)


def build_train_library(verbose: bool = False) -> str:
    """The same for the library of the training operators."""
    return _compile(TRAIN_LIB_PATH, train_sources(), verbose)
