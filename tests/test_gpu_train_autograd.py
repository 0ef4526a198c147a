"""What the calls of the second header write, as autograd sees it."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def tr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_06751_amd import train
    return train


def test_writes_count_as_writes(tr):
    """What a call writes into a caller's tensor, autograd knows of: a tensor
    that it saved and that was written since is refused in the backward pass."""
    x = torch.randn(6, 301, device=DEV)
    t = torch.randint(0, 301, (6,), device=DEV)
    f, w = lambda *s: torch.zeros(s, device=DEV), torch.ones(1, device=DEV, requires_grad=True)  # noqa: E731
    o = [f(6), f(6), f(6)]
    _, lse, _ = tr.sf_token_logp(x, t, out_logp=o[0], out_lse=o[1], out_entropy=o[2])
    terms, gl, start = f(4), f(6), torch.tensor([0, 2, 6], device=DEV)
    tr.sf_policy_loss(o[0], o[0], torch.ones(2, device=DEV), start, out_terms=terms, out_grad=gl)
    saved = (x * w).relu()  # saves its result
    tr.sf_token_logp_grad(saved.detach(), t, lse, gl, out_grad=saved.detach())
    grads = [torch.ones(50, device=DEV), torch.ones(3, device=DEV)]
    out = [g.clone() for g in grads]
    norms, total, wrong = f(2), f(1), torch.zeros(2, dtype=torch.int64, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    tr.sf_grad_norm(grads, norms, total, wrong)
    tr.sf_grad_clip(grads, total, 1.0, out=out, status=status)
    for v in o + [terms, gl, norms, total, wrong, status] + out:
        assert v._version == 1
    assert x._version == t._version == start._version == 0 and all(g._version == 0 for g in grads)
    tr.sf_grad_clip(tr.GradSet(grads), total, 1.0)
    assert all(g._version == 1 for g in grads)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        saved.sum().backward()
