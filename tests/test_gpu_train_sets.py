"""Sets of gradients: what their calls owe a rank that has none, layouts that are
alike, tensors that moved."""
import math

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


@pytest.mark.parametrize("norms,wrong", [([2.0, math.inf], True), ([math.nan], True), ([2.0, 1e38], False), ([0.5], False)])
def test_status_without_gradients(tr, norms, wrong):
    """A rank that owns no gradients learns as the others do that the norm over
    all ranks is not finite."""
    for grads in ([], [torch.zeros(0, device=DEV)], [torch.ones(5, device=DEV)]):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        made = tr.sf_grad_clip(grads, torch.tensor(norms, device=DEV), 1.0, status=status)
        assert len(made) == len(grads) and status.item() == (tr.SF_ERANGE if wrong else 0)
        status.zero_()
        tr.sf_grad_clip(tr.GradSet(grads), torch.tensor(norms, device=DEV), 1.0, out=tr.GradSet([g.clone() for g in grads]),
                        status=status)
        assert status.item() == (tr.SF_ERANGE if wrong else 0)
    tr.sf_grad_clip([], torch.tensor(norms, device=DEV), 1.0)


def test_dimensions_of_one_entry_have_any_stride(tr):
    """Layouts that differ in the stride of a dimension of size 1 alone are one."""
    base = torch.randn(4, 6, device=DEV)
    g = torch.as_strided(base, (6, 1, 4), (1, 77, 6))
    o = torch.as_strided(torch.zeros(4, 6, device=DEV), (6, 1, 4), (1, 1, 6))
    assert not g.is_contiguous() and g.stride() != o.stride()
    tr.sf_grad_clip([g], torch.tensor([4.0], device=DEV), 1.0, eps=0.0, out=[o])
    assert torch.equal(o, g * 0.25)
    with pytest.raises(ValueError):
        tr.sf_grad_clip([g], torch.tensor([4.0], device=DEV), 1.0, out=[torch.zeros(6, 1, 4, device=DEV)])


def test_tensors_that_moved_are_refused(tr):
    """A set stands for the memory that its tensors had: given other memory, or
    freed, they are no longer that."""
    grads = [torch.ones(50, device=DEV), torch.ones(4, 6, device=DEV), torch.zeros(0, device=DEV)]
    norm = torch.tensor([2.0], device=DEV)

    def refused(s, other=None):
        for call in (lambda: tr.sf_grad_norm(s), lambda: tr.sf_grad_clip(s, norm, 1.0),
                     lambda: tr.sf_grad_clip(s, norm, 1.0, out=other), lambda: tr.sf_grad_clip(other, norm, 1.0, out=s)):
            with pytest.raises(ValueError, match="gradient 1"):
                call()

    other = tr.GradSet([g.clone() for g in grads])
    for move in (lambda g: setattr(g, "data", torch.full((4, 6), 3.0, device=DEV)),
                 lambda g: setattr(g, "data", g.data[:2]),
                 lambda g: g.resize_(8, 6),
                 lambda g: g.untyped_storage().resize_(0),
                 lambda g: g.set_(torch.zeros(4, 6, device=DEV))):
        s = tr.GradSet([grads[0], torch.ones(4, 6, device=DEV), grads[2]])
        assert abs(tr.sf_grad_norm(s)[1].item() - math.sqrt(74.0)) < 1e-5
        move(s.tensors[1])
        refused(s, other)
    torch.cuda.synchronize()
    assert all((g == 1).all() for g in grads[:2]) and (other.tensors[1] == 1).all()
    # the same memory in another order: of weight only where the order of two sets is
    s = tr.GradSet([grads[0], torch.ones(4, 6, device=DEV), grads[2]])
    s.tensors[1].t_()
    assert abs(tr.sf_grad_norm(s)[1].item() - math.sqrt(74.0)) < 1e-5
    for a, b in ((s, other), (other, s)):
        with pytest.raises(ValueError, match="gradient 1"):
            tr.sf_grad_clip(a, norm, 1.0, out=b)
    # values that change in place are the same tensors
    s = tr.GradSet(grads)
    grads[1].mul_(2.0)
    assert abs(tr.sf_grad_norm(s)[1].item() - math.sqrt(50 + 4 * 24.0)) < 1e-5
