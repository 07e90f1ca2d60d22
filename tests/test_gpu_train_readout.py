"""The example that fits a readout, run as a user would (needs a GB300): the loss
falls, the readout gives more of the full model's answers on the rows it was fitted
to, and an engine takes the result."""
import importlib.util
import os

import pytest

import synth

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("train_readout", os.path.join(ROOT, "examples", "train_readout.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_fit_a_readout():
    import paper_2609_14144_gb300 as ee

    shape = synth.CONFIGS["tiny"]
    model = synth.make_model(shape)
    out = example().fit(shape, model, tokens=400, steps=25, report=None)
    assert all(b < a for a, b in zip(out["losses"][:10], out["losses"][1:11])), out["losses"]
    assert out["losses"][-1] < 0.7 * out["losses"][0]
    assert out["after"]["training"][0] > out["before"]["training"][0]
    assert out["after"]["training"][1] > out["before"]["training"][1]
    eng = ee.Engine(shape, out["model"])
    eng.prefill(synth.prompt(shape))
    eng.decode_n(16, taus=[0.5])
    assert eng.stats()["steps"] == 16
    eng.close()
