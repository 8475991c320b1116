"""The example of a layer of experts: router, gated experts, second products, sums."""
import importlib.util
import os

import pytest
import torch

from test_abi import ROOT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_example_layer(dtype):
    spec = importlib.util.spec_from_file_location("expert_layer", os.path.join(ROOT, "examples", "expert_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    errors, same = m.main(tokens=(130, 1, 9), dtype=dtype, say=lambda *_: None)
    assert same
    # 8 bits with the step of a row's largest value, 3.5 deviations of 1024: a rounding is 3.5 / 127 / sqrt(12) = 0.8 % of a deviation on each side of a product;
    # gate and up 1.1 % each, the hidden rows' largest 8 deviations or so: 1.8 %, the second weights 0.8 %: 2.6 % together, half as much again for single tokens
    assert all(2e-3 < e < 6e-2 for e in errors), errors
