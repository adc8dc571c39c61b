"""Calls of tree_attn that between them reach every build of its kernels: the GPU tests compare them with the answer in 64 bits, and the tests without a GPU look at
the kernels that are launched for them on 148 SMs, so that no threshold moves one away unseen."""
from collections import namedtuple

# sequences, new tokens, heads, kv-heads, head size, entries of a page, entries before the new tokens (ragged: at most); kernels: what is launched, by short
# names, and where bf16 and the 8-bit formats differ both ("few8": groups of 8 rows, "short8": their short build, "wide": many rows, "rows", "merge")
Call = namedtuple("Call", "B w Hq Hkv d page n ragged kernels")


def _calls():
    for d in (64, 128):
        yield Call(1, 1, 8, 2, d, 16, 20000, False, ["few8", "merge"])                   # splits as slots
        yield Call(3, 1, 8, 2, d, 64, 700, True, ["few8"])                               # splits as a cluster
        yield Call(2, 5, 8, 2, d, 48, 130, True, ["few16"])
        yield Call(160, 1, 8, 2, d, 16, 60, True, ["short8"])                            # more than a round of long CTAs
        yield Call(160, 2, 16, 2, d, 32, 100, True, ["short16"])
        yield Call(310, 1, 4, 2, d, 16, 90, True, ["rows", "short8"])
        yield Call(300, 2, 16, 2, d, 16, 90, True, ["rows", "short16"])
        slots = ["rows", "few8", "merge"]
        yield Call(40, 1, 32, 4, d, 128, 3000, True, slots if d == 128 else {"bf16": ["few8"], "8 bits": slots})
        yield Call(4, 40, 8, 2, d, 64, 6000, True, ["rows", "wide", "merge"])            # two blocks of rows
        yield Call(8, 30, 8, 2, d, 16, 5000, False, ["rows", "wide", "merge"])           # one
        yield Call(6, 64, 12, 2, d, 256, 2500, True, ["rows", "wide", "merge"])          # three
        yield Call(10, 64, 16, 2, d, 64, 1500, True, ["rows", "wide", "merge"])          # more rows than the join takes one a warp


CALLS = list(_calls())
FORMATS = ["bf16", "int8", "e4m3"]
