"""The example of many answers over one compressed prompt: its last step against plain PyTorch."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "many_answers.py")
    spec = importlib.util.spec_from_file_location("many_answers", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("answers,steps,question,Hq,Hkv,d", [(1, 3, 1, 8, 2, 64), (5, 4, 12, 8, 2, 128), (40, 3, 5, 4, 4, 64)])
def test_last_step_is_the_plain_one(example, fmt, answers, steps, question, Hq, Hkv, d):
    r = example.run(answers, steps, fmt, chunks=3, chunk_len=256, question=question, Hq=Hq, Hkv=Hkv, d=d, m=2, k_keep=100)
    assert r["own_entries"] == question + steps                   # a step outside the graph, the rest replayed
    assert r["cache_bytes"] < r["bf16_cache_bytes"] * 0.54        # 1 + 4 / d bytes a value against 2
    # a step of bf16 in the output (2^-8), the roundings of P (2^-9), of the dequantised values that the plain form reads (2^-9) and
    # of q's rotation (logits of a few units: 2^-8), with a factor of 2
    assert r["relative_difference"] <= 2 * (2.0 ** -8 + 2.0 ** -9 + 2.0 ** -9 + 2.0 ** -8)
