"""CPU-only: what page_append hands to the C entry point for parents of one tree for all sequences, on host memory, with an entry point that notes its arguments."""
import ctypes

import pytest
import torch

from tests.test_tree_host import Append


@pytest.fixture(scope="module")
def append():
    import paper_2502_14317_b200 as pc
    from paper_2502_14317_b200 import binding, build
    build.build_library()
    seen = []
    run = ctypes.CFUNCTYPE(ctypes.c_int32, ctypes.POINTER(Append), ctypes.c_void_p)(lambda a, s: seen.append((a.contents.parents, a.contents.parents_stride)) or 0)
    cache, x, table = pc.kv_cache(6, 2, 16, 64, "bf16", device="cpu"), torch.zeros(3, 4, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 2, dtype=torch.int32)

    def call(parents):
        del seen[:]
        got = binding._host_module().page_append(ctypes.cast(run, ctypes.c_void_p).value, 0, False, cache, x, x, table, 0, None, None, None, parents, None, 0, 1e4)
        return seen[0] if got == 0 else got

    return call


def test_one_tree_for_all(append):
    tree = torch.tensor([-1, 0, 0, 1, 9, 9], dtype=torch.int32)
    assert append(tree[:4]) == (tree.data_ptr(), 0) == append(tree[:4].expand(3, -1))
    each = tree[:4].repeat(3, 1)
    assert append(each) == (each.data_ptr(), 4) and append(None) == (None, 0)


@pytest.mark.parametrize("parents", [torch.zeros(3, dtype=torch.int32), torch.zeros(5, dtype=torch.int32), torch.zeros(4, dtype=torch.int64), torch.zeros(8, dtype=torch.int32)[::2],
                                     torch.zeros(1, 4, dtype=torch.int32), torch.zeros(3, 4, 1, dtype=torch.int32), torch.zeros((), dtype=torch.int32)])
def test_parents_that_are_refused(append, parents):
    assert isinstance(append(parents), str)
