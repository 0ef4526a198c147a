"""The example that keeps both records of a small data-parallel policy loop."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_policy_step_example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("policy_step", os.path.join(ROOT, "examples", "policy_step.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    rec = example.run(ranks=3, steps=12, vocab=1031)
    assert torch.isfinite(rec["terms"]).all() and torch.isfinite(rec["norm"]).all()
    assert (rec["norm"] > 0).all() and not rec["wrong"].any() and rec["status"] == 0
    # the first step is on-policy: no KL, nothing clipped; then the loss falls
    assert abs(rec["terms"][0, 2]) < 1e-9 and rec["terms"][0, 3] == 0
    assert rec["terms"][-1, 0] < rec["terms"][0, 0] and rec["terms"][-1, 2] > 0
    assert rec["exposed"].sum() > 0 and rec["exposed"].numel() == len(example.STAGES)
