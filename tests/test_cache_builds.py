"""CPU-only: the kernels that pc_cache_attn launches for the calls of cache_builds.py, on the library's own objects and a CUDA runtime that notes names."""
import ctypes
import os
import re
import subprocess
from ctypes import POINTER, byref, c_size_t, c_void_p

import pytest

from tests.cache_builds import CALLS, FORMATS, Call
from tests.test_cache_host import AT, Args, args, cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _objects(tmp):
    """the library's objects: those of the build where they are of these sources, else made here"""
    from paper_2502_14317_b200 import build
    build.build_library()
    made = [os.path.join(build.HERE, "_build", s.replace(".cu", ".o")) for s in build.SOURCES]
    inputs = [os.path.join(build.CSRC, f) for f in os.listdir(build.CSRC)] + [os.path.join(ROOT, "include", "pc.h")]
    if all(os.path.exists(o) and os.path.getmtime(o) > max(map(os.path.getmtime, inputs)) for o in made):
        return made
    made = [str(tmp / s.replace(".cu", ".o")) for s in build.SOURCES]
    procs = [subprocess.Popen([build._nvcc(), *build.NVCC_FLAGS, "-c", os.path.join(build.CSRC, s), "-o", o]) for s, o in zip(build.SOURCES, made)]
    assert not any(p.wait() for p in procs)
    return made


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    from paper_2502_14317_b200 import build
    tmp = tmp_path_factory.mktemp("names")
    out = str(tmp / "libpc_names.so")
    subprocess.run([build._nvcc(), "-shared", "-cudart", "none", "-gencode", "arch=compute_100a,code=sm_100a", "-Xcompiler", "-fPIC", "-Xlinker", "-Bsymbolic",
                    "-Xlinker", "--no-undefined", os.path.join(ROOT, "tests", "fake_launches.cpp"), *_objects(tmp), "-o", out], check=True)
    lib = ctypes.CDLL(out)
    lib.pc_cache_attn_workspace_bytes.restype = c_size_t
    lib.pc_cache_attn_workspace_bytes.argtypes = [POINTER(Args)]
    lib.pc_cache_attn.argtypes = [POINTER(Args), c_void_p]
    lib.fake_launched.restype = lib.fake_known.restype = ctypes.c_char_p
    return lib


def _short(name):
    few, wide = re.search(r"3FewILi(\d+)ELi(\d)ELi(\d)ELb(\d)ELb(\d)E", name), re.search(r"cache_wide_kernelILi(\d+)ELi(\d)ELb(\d)E", name)
    if few:
        d, fmt, groups, short, causal = map(int, few.groups())
        return ("short " * short + "causal") if causal else ("short" if short else "few") + str(8 * groups)
    if wide:
        return "pair" if wide.group(3) == "1" else "wide"
    return "rows" if "cache_rows_kernel" in name else "merge" if "cache_merge_kernel" in name else name


def launched(lib, c, fmt, **more):
    kept = {}
    if c.n_prefix:
        kept["prefix"] = cache(FORMATS.index(fmt), 1, c.Hkv, c.d, c.n_prefix)
    if c.n_own:
        kept["own"] = cache(FORMATS.index(fmt), c.B, c.Hkv, c.d, c.n_own)
    a = args(**kept, B=c.B, w=c.w, Hq=c.Hq, Hkv=c.Hkv, d=c.d, n_prefix=c.n_prefix, n_own=c.n_own, own_len=AT if c.ragged else None, lse=AT, status_word=AT,
             **({} if c.window else dict(k_win=None, v_win=None)), **more)
    a.workspace_bytes = lib.pc_cache_attn_workspace_bytes(byref(a))
    lib.fake_clear()
    assert lib.pc_cache_attn(byref(a), None) == 0
    return lib.fake_launched().decode().split("\n")[:-1]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("call", CALLS, ids=str)
def test_kernels_of_a_call(lib, call, fmt):
    want = call.kernels["bf16" if fmt == "bf16" else "8 bits"] if isinstance(call.kernels, dict) else call.kernels
    assert [_short(n) for n in launched(lib, call, fmt)] == want


def test_the_calls_reach_every_build(lib):
    seen = {n for c in CALLS for fmt in FORMATS for n in launched(lib, c, fmt)}
    every = {n for n in lib.fake_known().decode().split("\n") if re.search("cache_(few|wide|rows|merge)_kernel", n)}
    assert len(every) >= 41 and every == seen, sorted(every - seen)


@pytest.mark.parametrize("w,phase", [(24, False), (25, True), (40, True)])
def test_new_tokens_that_are_a_phase(lib, w, phase):
    """More than 24, through strides that TMA has: 0 in no dimension of more than one entry."""
    c = Call(4, w, 4, 2, 64, 200, 0, False, True, None)
    row = w * 2 * 64
    names = lambda *s: [_short(n) for n in launched(lib, c, "int8", k_win_stride=s, v_win_stride=s)]                     # noqa: E731
    for s in ((0, 0, 0), (row, 128, 64), (2 * row, 256, 64)):
        assert any("causal" in n for n in names(*s)) == phase, s
    for s in ((row, 128, 0), (0, 128, 64), (row, 0, 64)):
        assert not any("causal" in n for n in names(*s)), s
