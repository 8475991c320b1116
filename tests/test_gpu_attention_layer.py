"""The example of the whole path: expanded projections, planned pages, 4-bit cache, prompts and single tokens."""
import importlib.util
import os

import pytest

from test_abi import ROOT

pytestmark = pytest.mark.gpu


def test_example_layer():
    spec = importlib.util.spec_from_file_location("attention_layer", os.path.join(ROOT, "examples", "attention_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    prompt, full, held = m.main(steps=6, say=lambda *_: None)
    # The attentions are fp32; the projection behind them rounds its input to 8 bits with the scale of the largest value, in both: an output of the
    # attention that lies on the edge between two codes may fall either way, one step of 1/127 of the largest in one of 1024 features.
    assert prompt < 2e-3 and max(held) < 2e-3
    # 4 bits: half a step of 1/15 of a row's range (about 5 deviations) in each value is 10 % of a deviation, a third of it on average in keys
    # and values, and the sums over many tokens average the values' share
    assert 1e-3 < max(full) < 0.2
