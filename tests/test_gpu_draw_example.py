"""The example's answers that the policy draws itself, and its dropout."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("policy_step", os.path.join(ROOT, "examples", "policy_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("options", [dict(drafts=True), dict(dropout=0.1), dict(drafts=True, dropout=0.2)])
def test_policy_step_draws(example, options):
    rec = example.run(ranks=3, steps=6, vocab=1031, **options)
    assert torch.isfinite(rec["terms"]).all() and torch.isfinite(rec["norm"]).all()
    assert (rec["norm"] > 0).all() and not rec["wrong"].any() and rec["status"] == 0
    if "dropout" not in options:
        # the first step is on-policy by the log-probabilities that the draws had
        assert abs(rec["terms"][0, 2]) < 1e-9 and rec["terms"][0, 3] == 0
    again = example.run(ranks=3, steps=6, vocab=1031, **options)
    assert torch.equal(rec["terms"][0], again["terms"][0])  # drawn by counter


def test_answers(example):
    """What the ranks train on: drafts up to the first refused, one token more,
    with the policy's log-probabilities."""
    from paper_2606_06751_amd import train
    dev = "cuda:0"
    g = torch.Generator().manual_seed(1)
    start = torch.tensor([0, 5, 6, 30, 41])
    d = dict(x=torch.randn(41, 16, generator=g).to(dev), start=start.to(dev))
    weight = (torch.randn(301, 16, generator=g) * 0.5).to(dev)
    small = weight + (torch.randn(301, 16, generator=g) * 0.05).to(dev)
    example.answer(d, weight, small, torch.tensor([4, 0], device=dev), 0)
    for b in range(4):
        t = d["t"][start[b]:start[b + 1]]
        n = int((t >= 0).sum())
        assert n >= 1 and (t[:n] >= 0).all() and (t[n:] == -1).all()
    logp, _, _ = train.sf_token_logp(d["x"] @ weight.t(), d["t"], entropy=False)
    assert (logp - d["old"]).abs().max() < 1e-5 and torch.equal(d["mask"], d["t"] >= 0)
