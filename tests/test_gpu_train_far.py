"""Gradients of rows whose logits lie far from 0, against the softmax of the
logits themselves in 64 bits (not against the 32-bit lse of the forward call)."""
import numpy as np
import pytest

import train_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda:0"
KINDS = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FAR = 65536.0  # |lse| from which the gradient takes its normaliser from the logits


@pytest.fixture(scope="module")
def tr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_06751_amd import train
    return train


def gradient(x, t, inv_t, g, h, kind):
    """The gradient of one row and its bound, u = 2^-24: log p = (x - max) / T -
    log s has 6 u of the distance and 4 u of log s from its own roundings and
    the exponential's argument, and the sum's V / 64 + 72; where lse is
    nearer to 0 than FAR, the rounding of lse, u |lse|, besides.  Then the formula's
    products, 12 u, and the error of the entropy that it is given."""
    x = np.asarray(x, np.float64)
    top = x.max()
    d = (x - top) * inv_t
    s = np.exp(d).sum()
    q = d - np.log(s)
    p = np.exp(q)
    live = p > 0
    d, q = np.where(live, d, 0.0), np.where(live, q, 0.0)
    ent = -(p * q).sum()
    e_ent = ref.token_logp(x, t, inv_t)[1][2]
    hot = np.zeros(len(x))
    hot[t] = g
    y = inv_t * (hot - p * (g + h * (q + ent)))
    lse = top * inv_t + np.log(s)
    e_q = ref.U * (6 * np.abs(d) + 4 * abs(np.log(s)) + len(x) / 64 + 72 + (abs(lse) if abs(lse) < FAR else 0.0))
    size = p * (abs(g) + abs(h) * (np.abs(q) + ent))
    err = inv_t * (size * (e_q + 12 * ref.U) + p * abs(h) * (e_q + e_ent) + 6 * ref.U * np.abs(hot))
    return y, err + ref.HALF_ULP[kind] * (np.abs(y) + err) + ref.TINY[kind]


def check(got, want, bound, kind, what):
    got = got.double().cpu().numpy()
    beyond = np.abs(want) >= torch.finfo(KINDS[kind]).max * (1 + 2.0 ** -8)  # rounds to an infinity of the type
    assert (got[beyond] == np.copysign(np.inf, want[beyond])).all(), what
    off = np.abs(got - want)[~beyond]
    assert (off <= bound[~beyond]).all(), "%s: worst %g against %g for %g" % (
        what, off.max(), bound[~beyond][np.argmax(off)], want[~beyond][np.argmax(off)])


def far_rows(kind, V):
    info = torch.finfo(KINDS[kind])
    rng = np.random.default_rng(V)
    far = 1e9 if kind != "f16" else 60000.0
    step = {"f32": 64.0, "bf16": 4194304.0, "f16": 32.0}[kind]  # of the type's numbers there
    rows = np.zeros((7, V))
    rows[0] = info.min                                  # masked alike throughout
    rows[1] = -far
    rows[2] = -far + step * rng.integers(0, 3, V)       # the type's neighbours
    rows[3] = far + step * rng.integers(0, 3, V)
    rows[4] = info.min
    rows[4, V // 3] = 0.5                               # one left
    rows[5] = -far
    rows[5, ::2] = -np.inf
    rows[6] = info.max
    x = torch.tensor(rows, dtype=torch.float64).to(KINDS[kind])
    x[0] = x[4, 1] = info.min
    x[6] = info.max
    assert torch.isfinite(x[[0, 1, 2, 3, 4, 6]]).all()
    return x


@pytest.mark.parametrize("T", [1.0, 0.9, 1.3, 0.7, 50.0, 1e-6])
@pytest.mark.parametrize("V", [5, 515, 9000, 40001])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_gradient_of_far_rows(tr, kind, V, T):
    x = far_rows(kind, V)
    targets = torch.tensor([1, V - 1, 2, 3, V // 3, 1, V // 2])
    inv_t = float(np.float32(1.0 / T))
    logits = x.to(DEV)
    t = targets.to(DEV)
    logp, lse, ent = tr.sf_token_logp(logits, t, inv_temperature=inv_t)
    assert torch.isfinite(lse).all()  # held within the largest floats
    rng = np.random.default_rng(5)
    g, h = rng.normal(size=7).astype(np.float32), (0.1 * rng.normal(size=7)).astype(np.float32)
    dev = [torch.tensor(v).to(DEV) for v in (g, h)]
    got = tr.sf_token_logp_grad(logits, t, lse, dev[0], entropy=ent, grad_entropy=dev[1], inv_temperature=inv_t)
    torch.cuda.synchronize()
    wide = x.double().numpy()
    for i in range(7):
        (w_logp, _, w_ent), (b_logp, _, b_ent) = ref.token_logp(wide[i], int(targets[i]), inv_t)
        assert abs(logp[i].item() - w_logp) <= b_logp and abs(ent[i].item() - w_ent) <= b_ent, i
        want, bound = gradient(wide[i], int(targets[i]), inv_t, float(g[i]), float(h[i]), kind)
        check(got[i], want, bound, kind, "row %d" % i)
    # the same in place, among padding that stays
    buf = torch.full((7, V + 3), 7.0, dtype=KINDS[kind], device=DEV)
    buf[:, 1:V + 1] = logits
    inside = buf[:, 1:V + 1]
    tr.sf_token_logp_grad(inside, t, lse, dev[0], entropy=ent, grad_entropy=dev[1], inv_temperature=inv_t, out_grad=inside)
    out = tr.sf_token_logp_grad(logits, t, lse, dev[0], inv_temperature=inv_t)
    torch.cuda.synchronize()
    assert (buf[:, 0] == 7).all() and (buf[:, V + 1:] == 7).all()
    for i in range(7):
        want, bound = gradient(wide[i], int(targets[i]), inv_t, float(g[i]), float(h[i]), kind)
        check(inside[i], want, bound, kind, "row %d in place" % i)
        want, bound = gradient(wide[i], int(targets[i]), inv_t, float(g[i]), 0.0, kind)
        check(out[i], want, bound, kind, "row %d without entropy" % i)


def test_far_rows_among_others(tr):
    """Far rows, ordinary ones, masked ones and empty ones in turn, over more rows
    than the grid's workgroups of one chunk."""
    V, N = 1031, 900
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(N, V, generator=gen)
    x[::3] -= 2.0 ** 20
    x[5::10] = -float("inf")
    t = torch.randint(0, V, (N,), generator=gen)
    t[7::11] = -1
    logits, td = x.to(DEV), t.to(DEV)
    _, lse, _ = tr.sf_token_logp(logits, td)
    g = torch.randn(N, generator=gen)
    got = tr.sf_token_logp_grad(logits, td, lse, g.to(DEV))
    wide = x.double().numpy()
    for i in range(N):
        if t[i] < 0 or i % 10 == 5:
            assert not got[i].any(), i
        else:
            want, bound = gradient(wide[i], int(t[i]), 1.0, g[i].item(), 0.0, "f32")
            check(got[i], want, bound, "f32", "row %d" % i)
