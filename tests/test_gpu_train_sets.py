"""Sets of gradients: what their calls owe a rank that has none, and layouts
that are alike."""
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
