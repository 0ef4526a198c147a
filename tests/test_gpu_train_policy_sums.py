"""What the policy loss promises of its numbers: tokens summed in 64 bits."""
import numpy as np
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


def loss(tr, lp, old, adv, start, ref=None, mask=None, **kw):
    dev = [None if v is None else torch.tensor(v).to(DEV) for v in (lp, old, adv, start, ref, mask)]
    terms, grad = tr.sf_policy_loss(*dev[:4], ref_logp=dev[4], mask=dev[5], **kw)
    return terms.double().cpu().numpy(), grad.cpu().numpy()


# one workgroup with one round and two, chunks by many, chunks that meet more
# sequences than a workgroup keeps
PATHS = [(8, 1), (4096, 9), (8192, 1000), (40000, 11), (40000, 2000), (40000, 80000)]


def starts(N, B):
    return (np.arange(B + 1) * N // B).astype(np.int64)


@pytest.mark.parametrize("N,B", PATHS)
def test_terms_of_opposite_sign_cancel(tr, N, B):
    """-A r of tokens with r = 1: of each four, neighbours or 64 apart, two of
    2^30 with opposite signs and two of 1.  All sums are exact in 64 bits."""
    i = np.arange(N)
    adv = np.array([2.0 ** 30, 1.0, -2.0 ** 30, 1.0], np.float32)[(i + i // 64) % 4]
    zero = np.zeros(N, np.float32)
    terms, grad = loss(tr, zero, zero, adv, starts(N, B), advantage_per_token=True, reduction=2)
    np.testing.assert_array_equal(grad, -adv)
    exact = -adv.astype(np.float64).sum()
    assert terms[1] == exact and terms[0] == exact


@pytest.mark.parametrize("N,B", PATHS)
def test_large_terms_do_not_overflow(tr, N, B):
    """e^x - x - 1 of 1.65e38 a token: any three pass the largest float; the loss,
    with its small share of their sum, does not."""
    zero = np.zeros(N, np.float32)
    x = np.full(N, 88.0, np.float32)
    terms, _ = loss(tr, zero, zero, np.zeros(B, np.float32), starts(N, B), ref=x, reduction=2, kl_coef=1e-11)
    each = np.expm1(np.float64(x[0])) - np.float64(x[0])
    beta = np.float64(np.float32(1e-11))
    # one value for all tokens, within 2 units in the last place and 2 roundings
    # of the term, and the loss's own rounding
    assert abs(terms[0] - beta * N * each) <= 8 * 2.0 ** -24 * beta * N * each
    assert terms[2] == np.inf and terms[1] == 0
