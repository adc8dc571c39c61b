"""CPU-only: calls of pc_token_logprobs by two threads at a time, on the library's own objects and a CUDA runtime that keeps a kernel's attribute as the real one does."""
import ctypes
import itertools
import os
import subprocess
import threading
from ctypes import byref

import pytest

from tests.test_cache_builds import ROOT, _objects
from tests.test_tree_host import _typed, logprobs

ROWS = [1, 148, 149, 296, 297, 444, 445, 592, 593, 5000]                 # one to four CTAs an SM, and more than there is room for


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    from paper_2502_14317_b200 import build
    tmp = tmp_path_factory.mktemp("attributes")
    out = str(tmp / "libpc_attributes.so")
    subprocess.run([build._nvcc(), "-shared", "-cudart", "none", "-gencode", "arch=compute_100a,code=sm_100a", "-Xcompiler", "-fPIC", "-Xlinker", "-Bsymbolic",
                    "-Xlinker", "--no-undefined", os.path.join(ROOT, "tests", "fake_attributes.cpp"), *_objects(tmp), "-o", out], check=True)
    return _typed(ctypes.CDLL(out))


def _together(lib, calls):
    got = [None] * len(calls)

    def one(i):
        got[i] = lib.pc_token_logprobs(byref(calls[i]), None)             # (ctypes lets go of the interpreter's lock)

    lib.fake_meet(len(calls))
    threads = [threading.Thread(target=one, args=(i,)) for i in range(len(calls))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    lib.fake_meet(0)
    return got


@pytest.mark.parametrize("type", [0, 1, 2])
def test_calls_of_any_rows_go_together(lib, type):
    for rows in itertools.combinations(ROWS, 2):
        assert _together(lib, [logprobs(type=type, N=n) for n in rows]) == [0, 0], rows
