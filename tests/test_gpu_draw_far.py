"""Draws where a row's entries lie far apart, where a uniform number is exactly 0,
where a token is all but certain, and where next to nothing is left of a target's
distribution: each by every way that a row is taken, against the definitions
(draw_ref.py)."""
import math

import numpy as np
import pytest

import draw_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda:0"
KINDS = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INF, NAN = math.inf, math.nan

# Row lengths and copies of a few rows that are taken by a workgroup of 1024, by one
# of 256, by a wave, by many workgroups, and (bfloat16) by a table of powers.
WAYS = [(kind, V, copies) for kind in KINDS
        for V, copies in ((9000, 1), (9000, 150), (9000, 900), (70001, 1))] + [("bf16", 40000, 100)]


@pytest.fixture(scope="module")
def dr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2606_06751_amd import draw
    return draw


def f64(t):
    return t.double().cpu().numpy()


def repeated(dr, target, drafts, draft, start, u, times, **kw):
    """The sequences of a batch ``times`` over: [accepted, token, logp], a row for
    each time."""
    n = int(start[-1])
    starts = (start[:-1][None, :] + torch.arange(times, device=DEV)[:, None] * n).reshape(-1)
    starts = torch.cat([starts, torch.tensor([n * times], device=DEV)])
    got = dr.sf_draft_verify(target.repeat(times, 1), None if drafts is None else drafts.repeat(times, 1), draft.repeat(times),
                             starts, u.repeat(times), **kw)
    return [t.view(times, -1) for t in got]


# -- a uniform number of 0 -----------------------------------------------------

@pytest.mark.parametrize("kind,times", [("f32", 1), ("f32", 300), ("bf16", 1), ("bf16", 300), ("bf16", 2200), ("f16", 1),
                                        ("f16", 300)])
def test_residual_of_low_logits_at_zero(dr, kind, times):
    """Entries that both rows mask leave nothing, however small the sums that their
    powers are divided by: the first token that p has more of than q is drawn."""
    V, masked, d = 8192, 2048, 2050
    p, q, last = (torch.full((1, V), v) for v in (-82.0, -62.0, 0.0))
    p[0, masked:d + 1], q[0, masked:d + 1] = -92.0, -60.0   # q has more of these
    p[0, :masked] = q[0, :masked] = -INF
    target, drafts = torch.cat([p, last]).to(DEV, KINDS[kind]), q.to(DEV, KINDS[kind])
    u = torch.tensor([0.99, 0.0], device=DEV)
    k, near, logp, _ = ref.verify(f64(target), f64(drafts), [d], [float(np.float32(0.99)), 0.0], 1.0, 1.0)
    assert k == 0 and d + 1 in near
    got = repeated(dr, target, drafts, torch.tensor([d], device=DEV), torch.tensor([0, 1], device=DEV), u, times)
    assert not got[0].any()
    assert (got[1] == torch.tensor([d + 1, -1], device=DEV)).all()
    assert ((got[2][:, 0].double() - logp(d + 1)).abs() <= ref.logp_bound(logp(d + 1))).all() and not got[2][:, 1].any()
