"""What the policy loss promises of its numbers: tokens summed in 64 bits,
weights rounded once, e^x right over the whole range of floats."""
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


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("reduction", [0, 1])
@pytest.mark.parametrize("N,B", PATHS + [(30000, 200), (30000, 3000), (8191, 77)])
def test_weights_round_once(tr, N, B, reduction, masked):
    """On-policy tokens with advantage -1 have their weight as gradient."""
    rng = np.random.default_rng(N + B)
    start = np.concatenate([[0], np.sort(rng.integers(0, N + 1, B - 1)), [N]]).astype(np.int64)
    mask = (rng.random(N) < 0.7).astype(np.uint8) if masked else None
    on = np.ones(N, bool) if mask is None else mask != 0
    zero = np.zeros(N, np.float32)
    _, grad = loss(tr, zero, zero, np.full(B, -1.0, np.float32), start, mask=mask, reduction=reduction, scale=0.7)
    scale = float(np.float32(0.7))
    seq = np.searchsorted(start, np.arange(N), side="right") - 1
    count = np.bincount(seq[on], minlength=B)
    share = on.sum() if reduction == 0 else (count > 0).sum() * count[seq]
    want = np.where(on, scale / np.maximum(share, 1), 0.0).astype(np.float32)
    np.testing.assert_array_equal(grad, want)


def within_ulps(got, want, n, what):
    off = np.abs(got.astype(np.float64) - want) / np.spacing(np.abs(want).astype(np.float32)).astype(np.float64)
    assert (off <= n).all(), "%s: %.1f units in the last place at %d" % (what, off.max(), np.argmax(off))


@pytest.mark.parametrize("N,B", PATHS[2:4])
def test_ratio_over_the_whole_range(tr, N, B):
    """r = e^d within 2 units in the last place wherever it is a float."""
    d = np.concatenate([np.linspace(-103.0, 88.72, N - 2000), np.linspace(88.0, 88.7228, 1000),
                        np.linspace(-103.2, -87.0, 1000)]).astype(np.float32)
    adv = np.where(d <= 0, 1.0, -1.0).astype(np.float32)  # never clipped
    _, grad = loss(tr, d, np.zeros(N, np.float32), adv, starts(N, B), advantage_per_token=True, reduction=2)
    within_ulps(-grad * adv, np.exp(d.astype(np.float64)), 2.0, "ratio")
    far = np.array([-1e30, -np.inf, -200.0, 88.73, 100.0, 1e30, np.inf] + [0.0] * (N - 7), np.float32)
    adv = np.where(far <= 0, 1.0, -1.0).astype(np.float32)
    _, grad = loss(tr, far, np.zeros(N, np.float32), adv, starts(N, B), advantage_per_token=True, reduction=2)
    assert not grad[:3].any() and (grad[3:7] == np.finfo(np.float32).max).all()


def test_kl_near_the_largest_float(tr):
    N = 4000
    x = np.linspace(85.0, 88.7228, N).astype(np.float32)
    zero = np.zeros(N, np.float32)
    _, grad = loss(tr, zero, zero, zero[:1], starts(N, 1), ref=x, reduction=2, kl_coef=1.0)
    within_ulps(-grad, np.expm1(x.astype(np.float64)), 3.0, "e^x - 1")  # and the difference's own rounding
