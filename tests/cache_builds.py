"""Calls of cache_attn that between them reach every build of its kernels: the GPU tests compare them with the answer in 64 bits, and the tests without a GPU
look at the kernels that are launched for them on 148 SMs, so that no threshold moves one away unseen."""
from collections import namedtuple

# sequences, new tokens, heads, kv-heads, head size; entries of the prefix and of the own caches (lengths: ragged), whether the new tokens' keys are there;
# kernels: what is launched, by short names, and where bf16 and the 8-bit formats differ both ("few8": groups of 8 rows, "short8": their short build, "causal", "short causal", "wide", "pair", "rows", "merge")
Call = namedtuple("Call", "B w Hq Hkv d n_prefix n_own ragged window kernels")


def _calls():
    for d in (64, 128):
        # few rows: one group, two groups, splits as a cluster or as slots
        yield Call(1, 1, 8, 2, d, 0, 20000, False, True, ["few8", "merge"])
        yield Call(3, 2, 16, 2, d, 0, 700, True, True, ["few16"])
        yield Call(2, 5, 8, 2, d, 0, 130, True, False, ["few16"])
        # short builds: more than a round of long CTAs, with rows made by the CTAs and ahead
        for n in (60, 1000):
            for ragged in (False, True):
                yield Call(160, 1, 8, 2, d, 0, n, ragged, True, ["short8"])
                yield Call(160, 2, 16, 2, d, 0, n, ragged, True, ["short16"])
        yield Call(310, 1, 4, 2, d, 0, 90, True, True, ["rows", "short8"])
        yield Call(300, 2, 16, 2, d, 0, 90, True, True, ["rows", "short16"])
        yield Call(160, 2, 16, 2, d, 150, 70, True, True, ["rows", "pair" if d == 128 else "wide", "short16"])
        # many rows: blocks of one CTA and of two, one split and several
        many = "pair" if d == 128 else "wide"
        yield Call(40, 2, 8, 2, d, 200, 0, False, True, ["rows", many, "merge"])
        yield Call(3, 60, 2, 2, d, 0, 400, False, True, ["rows", "wide", "causal"])
        yield Call(2, 70, 4, 2, d, 0, 3000, False, False, ["rows", many, "merge"])
        # new tokens as a phase: alone, behind a prefix and behind own caches; long and short builds, with rows made by the CTAs and ahead
        yield Call(1, 25, 8, 2, d, 0, 0, False, True, ["causal"])
        yield Call(5, 30, 8, 4, d, 40, 0, False, True, ["rows", many, "causal"])
        yield Call(1, 64, 64, 8, d, 0, 0, False, True, ["short causal"])
        yield Call(2, 64, 64, 8, d, 0, 0, False, True, ["rows", "short causal"])
        yield Call(3, 128, 16, 4, d, 0, 50, True, True, {"bf16": ["rows", "short16", "short causal"], "8 bits": ["rows", many, "short causal"]})
        yield Call(40, 25, 8, 4, d, 0, 33, True, True, {"bf16": ["rows", "short16", "short causal"], "8 bits": ["rows", "wide", "short causal"]})
        yield Call(2, 37, 24, 8, d, 200, 60, True, True, {"bf16": ["rows", many, "few16", "causal"], "8 bits": ["rows", many, "wide", "causal"]})


CALLS = list(_calls())
FORMATS = ["bf16", "int8", "e4m3"]
