"""examples/attention_layer.py at a small size: the served outputs lie where a 4-bit cache puts them.

What a 4-bit group may lose: a code is off by at most half a step of (max - min) / 15.  A uniform
error of that width is 1 / (15 sqrt 12) of the range, and 64 normal values span about 4.8 of their
deviations on average: 0.092 of the norm of K and of V.  Values average over the tokens that a query
sees like the signal does, so the outputs differ by that and what the scores add; 0.3 is far above
both, and far below an output that read a wrong token or a wrong page (1 and more).
"""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example(qe):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_layer.py")
    spec = importlib.util.spec_from_file_location("attention_layer", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("group,page", [(64, 32), (32, 64)])
def test_served_layer(example, dtype, group, page):
    r = example.run(hidden=256, heads=8, kv_heads=2, dim=64, prompts=(70, 1, 33), steps=5, chunk=32, calibration=1024,
                    group=group, page=page, dtype=dtype)
    assert r["held"] == [75, 6, 38]
    assert r["bytes_per_token"] < 0.32 * r["bytes_per_token_16_bit"]
    assert all(0.0 < e < 0.3 for e in r["cache"]), r["cache"]
    assert all(0.0 < e < 0.6 for e in r["both"]), r["both"]
