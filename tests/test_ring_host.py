"""What a product's block waits for after a wait of it has run out, against a model of barriers:
every copy on its way, whichever thread asked for it, and nothing that does not come."""
import ctypes
import os
import subprocess

import pytest

from paper_2607_23115_gb300 import binding as B
from paper_2607_23115_gb300 import build as G

SRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "native", "ring_model.cpp")


@pytest.fixture(scope="module")
def ring_run(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("ring") / "ring.so")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-I", G.CSRC, SRC,
                           "-o", out])
    f = ctypes.CDLL(out).ring_run
    f.argtypes = [ctypes.c_uint32] * 4
    return f


# threads that fill a stage together; stages of the rings (2 to 12)
@pytest.mark.parametrize("threads", [1, 2])
@pytest.mark.parametrize("n", [1, 2, 3, 4, 6, 7, 12])
def test_copies_on_their_way_are_waited_for(ring_run, n, threads):
    for steps in (0, 1, 2, 5, 20, 60, 200, 1000):
        for seed in range(200):
            assert ring_run(n, threads, steps, seed) == 0, (steps, seed)


def test_hooks_refuse():
    G.build()
    for what, value in [(B.GLEAM_DEBUG_WAIT_LIMIT_NS, 0), (B.GLEAM_DEBUG_SKIP_ARRIVE, 0),
                        (B.GLEAM_DEBUG_SKIP_ARRIVE, 1 << 32), (9, 1)]:
        assert B.gleam_operators_debug_set(what, value) == B.GLEAM_ERR_INVALID_ARG
