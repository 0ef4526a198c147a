"""Equal inputs give equal bits wherever the buffers lie, if they begin alike
modulo 128 bytes; from other places 32-bit sums may round differently."""
import numpy as np
import pytest

import train_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def tr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_06751_amd import train
    return train


def placed(x, at):
    """A copy of x that begins ``at`` entries after a 512-byte boundary."""
    buf = torch.zeros(x.numel() + at, dtype=x.dtype, device=DEV)
    assert buf.data_ptr() % 512 == 0
    buf[at:] = x.reshape(-1)
    return buf[at:].view(x.shape)


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V", [(3, 515), (5, 9001), (300, 20011), (2, 131073)])
def test_rows_at_any_place(tr, N, V, kind):
    gen = torch.Generator().manual_seed(V)
    x = (torch.randn(N, V, generator=gen) * 3.0).to(kind).to(DEV)
    t = torch.randint(0, V, (N,), generator=gen).to(DEV)
    g, h = torch.randn(N, generator=gen).to(DEV), torch.randn(N, generator=gen).to(DEV)
    line = 128 // x.element_size()
    first = tr.sf_token_logp(x, t)
    grad = tr.sf_token_logp_grad(x, t, first[1], g, entropy=first[2], grad_entropy=h)
    bounds = np.array([ref.token_logp(x[i].float().cpu().numpy(), int(t[i]), 1.0)[1] for i in range(N)]).T
    for at in (line, 5 * line, 1, 7, line - 1):
        y = placed(x, at)
        got = tr.sf_token_logp(y, t)
        for a, b, e in zip(first, got, bounds):
            if at % line == 0:
                assert torch.equal(a, b)
            assert ((a - b).abs().double().cpu().numpy() <= 2 * e).all()  # each within e of the truth
        # element by element: the place says nothing
        assert torch.equal(grad, tr.sf_token_logp_grad(y, t, first[1], g, entropy=first[2], grad_entropy=h,
                                                       out_grad=placed(torch.zeros_like(x), at + 3)))


@pytest.mark.parametrize("n", [1000, 100003, 1 << 21])
def test_norms_at_any_place(tr, n):
    x = torch.randn(n, generator=torch.Generator().manual_seed(n)).to(DEV)
    first = tr.sf_grad_norm([x, x[:n // 3]])
    for at in (32, 96, 1, 31):
        y = placed(x, at)
        for a, b in zip(first, tr.sf_grad_norm([y, y[:n // 3]])):
            if at % 32 == 0:
                assert torch.equal(a, b)
            # 64-bit sums, rounded once: the place can move that rounding alone
            assert ((a - b).abs() <= 2.0 ** -23 * a.abs()).all()


@pytest.mark.parametrize("N,B", [(5003, 8), (70001, 11), (70001, 4000)])
def test_policy_loss_at_any_place(tr, N, B):
    gen = torch.Generator().manual_seed(N + B)
    v = [torch.randn(N, generator=gen).to(DEV) for _ in range(3)]
    adv, mask = torch.randn(B, generator=gen).to(DEV), (torch.rand(N, generator=gen) < 0.7).to(DEV)
    start = (torch.arange(B + 1) * N // B).to(DEV)
    for red in (0, 1, 2):
        first = tr.sf_policy_loss(v[0], v[1], adv, start, ref_logp=v[2], mask=mask, reduction=red, kl_coef=0.1)
        for at in (32, 1, 3, 17):
            got = tr.sf_policy_loss(placed(v[0], at), placed(v[1], at + 1), placed(adv, at), placed(start, at),
                                    ref_logp=placed(v[2], at + 2), mask=placed(mask, at), reduction=red, kl_coef=0.1,
                                    out_grad=placed(torch.zeros(N, device=DEV), at))
            assert all(torch.equal(a, b) for a, b in zip(first, got))
