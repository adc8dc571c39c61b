"""The example of drafted tokens over pages: all calls together, the last step against plain PyTorch from a record of what was kept."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "drafted_tokens.py")
    spec = importlib.util.spec_from_file_location("drafted_tokens", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("answers,steps,Hq,Hkv,d,page", [(1, 2, 4, 2, 64, 16), (5, 6, 16, 2, 128, 32), (3, 9, 8, 8, 64, 64)])
def test_last_step_is_the_plain_one(example, fmt, answers, steps, Hq, Hkv, d, page):
    r = example.run(answers, steps, fmt, chunks=4, chunk_len=200, w=16, Hq=Hq, Hkv=Hkv, d=d, page=page, m=2, k_keep=96, vocabulary=1000)
    assert r["entries"] == [2 * 96 + n for n in r["kept"]]
    assert r["chunks"] == sorted(sorted(range(4), key=lambda c: r["chunk_score"][c])[:2])
    assert steps < 3 or max(r["kept"]) >= steps - 2              # the guess that holds is kept each time, whatever else is
    # a step of bf16 in the output (2^-8), the roundings of P (2^-9) and of q's and the keys' rotation (logits of a few units: 2^-8 each); in 8 bits the keys' and
    # values' codes: half a step of the row's largest, 1 / 254 for int8 and 1 / 16 for e4m3, of values of which dozens are averaged, and in logits of a few units
    # the same of 128 products of either sign (a tenth of it); with a factor of 2
    codes = {"bf16": 0.0, "int8": 1.5 / 254, "e4m3": 1.5 / 16}[fmt]
    assert r["relative_difference"] <= 2 * (2.0 ** -8 + 2.0 ** -9 + 2 * 2.0 ** -8 + codes)
