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


def far_rows(kind, V, what):
    """Rows of ordinary logits beside others that lie far above them, the tokens
    that a uniform number of 0 may draw, and the temperature's inverse."""
    low, high, inv_t = {"beyond": (-80.0, 656.0, 1.0), "within": (620.0, 720.0, 1.0), "cold": (-8.0, 65.5, 10.0)}[what]
    x = torch.full((6, V), -INF)
    x[:, :2048], x[:, V - 3] = low, high
    x[1, 2048:4096] = high                       # a whole part that is as high
    x[2, 7] = NAN
    x[3, 1:2048] = -INF                          # one entry alone
    x[4, :2048], x[4, 2048:4096] = high, low     # the other way round
    x[5, 2048:] = -INF                           # nothing above
    # 2^-144 of the largest has its probability; 2^-1062 may count as 0
    allowed = [{0}] * 6 if what == "within" else [{0, V - 3}, {0, 2048}, {0}, {0, V - 3}, {0}, {0}]
    allowed[2] = {-1}
    return x.to(DEV, KINDS[kind]), allowed, inv_t


def check_drawn(x, inv_t, allowed, token, logp):
    """Copies of the rows: the same token in each, one of those allowed, and its
    log-probability."""
    token, logp = token.view(-1, len(allowed)), logp.view(-1, len(allowed)).double()
    assert (token == token[:1]).all()
    for i, (t, want) in enumerate(zip(token[0].tolist(), allowed)):
        assert t in want, (i, t)
        if t < 0:
            assert torch.isnan(logp[:, i]).all()
        else:
            v = ref.log_p(ref.softmax(f64(x[i]), inv_t)[t])
            assert ((logp[:, i] - v).abs() <= ref.logp_bound(v)).all(), (i, logp[0, i].item(), v)


@pytest.mark.parametrize("kind,V,copies", WAYS)
@pytest.mark.parametrize("what", ["beyond", "within", "cold"])
def test_sample_far_apart_at_zero(dr, kind, V, copies, what):
    """What has 2^-144 of the largest's probability is drawn, what has 2^-1062 of it
    or not, and neither leaves a row without a token."""
    x, want, inv_t = far_rows(kind, V, what)
    u = torch.zeros(6 * copies, device=DEV)
    check_drawn(x, inv_t, want, *dr.sf_token_sample(x.repeat(copies, 1), u, inv_temperature=inv_t))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("what", ["beyond", "within", "cold"])
@pytest.mark.parametrize("copies", [1, 60, 400])
def test_verify_far_apart_at_zero(dr, kind, what, copies):
    """The same as a sequence's last token: without drafts, and behind a draft
    without logits that the target forbids."""
    x, want, inv_t = far_rows(kind, 9000, what)
    u, start = torch.zeros(6, device=DEV), torch.zeros(7, dtype=torch.int64, device=DEV)
    none = torch.zeros(0, dtype=torch.int64, device=DEV)
    for drafts in (None, x[:0]):
        acc, token, logp = repeated(dr, x, drafts, none, start, u, copies, inv_temperature=inv_t)
        assert not acc.any()
        check_drawn(x, inv_t, want, token, logp)
    # a draft of a token with no probability before each, and rows behind that are not reached
    target = torch.stack([x, torch.zeros_like(x)], 1).view(12, 9000)
    draft = torch.full((6,), 8999, device=DEV)
    u = torch.tensor([0.5, 0.0], device=DEV).repeat(6)
    acc, token, logp = repeated(dr, target, None, draft, torch.arange(7, device=DEV), u, copies, inv_temperature=inv_t)
    token, logp = token.view(-1, 6, 2), logp.view(-1, 6, 2)
    assert not acc.any() and (token[:, :, 1] == -1).all() and not logp[:, :, 1].any()
    check_drawn(x, inv_t, want, token[:, :, 0], logp[:, :, 0])


@pytest.mark.parametrize("kind,V,copies", WAYS)
def test_sample_any_distance_at_zero(dr, kind, V, copies):
    """Between what is drawn and what counts as 0 either is right; a token is."""
    g = torch.Generator().manual_seed(V + copies)
    x = torch.full((60, V), -INF)
    at = torch.rand(60, generator=g) * -130.0 - 10.0
    x[:, :2048] = at[:, None]
    x[:, V - 3] = at + torch.linspace(100.0, 800.0, 60)
    x = x.to(DEV, KINDS[kind])
    rows = (copies * 6 + 59) // 60
    token, logp = dr.sf_token_sample(x.repeat(rows, 1), torch.zeros(60 * rows, device=DEV))
    token, logp = token.view(rows, 60), logp.view(rows, 60)
    apart = (x[:, V - 3].double() - x[:, 0].double()) * math.log2(math.e)
    assert ((token == 0) | (token == V - 3)).all() and torch.isfinite(logp).all()
    assert (token[:, apart < 700] == 0).all()


# -- temperatures at which masked entries alone are far -------------------------

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("inv_t,iq", [(1e-37, 1e-37), (1e-37, 1.0), (1.0, 1e-37), (2.0 ** -149, 2.0 ** -149)])
@pytest.mark.parametrize("times", [1, 700])
def test_residual_at_nearly_infinite_temperatures(dr, kind, inv_t, iq, times):
    """Rows of 0 and -inf: what the draft's row masks is left to the target's."""
    V = 3000
    target, drafts = torch.zeros(2, V), torch.zeros(1, V)
    target[0, 2000:], drafts[0, 1000:] = -INF, -INF
    target, drafts = target.to(DEV, KINDS[kind]), drafts.to(DEV, KINDS[kind])
    for v, want in ((0.0, 1000), (0.3003, 1300), (0.9999, 1999)):
        u = torch.tensor([0.9, v], device=DEV)
        got = repeated(dr, target, drafts, torch.tensor([3], device=DEV), torch.tensor([0, 1], device=DEV), u, times,
                       inv_temperature=inv_t, draft_inv_temperature=iq)
        assert not got[0].any() and (got[1] == torch.tensor([want, -1], device=DEV)).all(), got[1][0].tolist()
        assert ((got[2][:, 0].double() + math.log(2000)).abs() <= ref.logp_bound(math.log(2000))).all()


# -- tokens that are all but certain ----------------------------------------------

def near_bound(v):
    """One rounding; powers within 2^-39.7, farther than 1/8 from 0 the logarithm
    within 2^-39, 2^-38.5 in all and 8 times that relative to it; and nearer the sums,
    of at most 64 additions to the longest of these rows, 2^-53 each."""
    return ref.U * abs(v) + 2.0 ** -35 * abs(v) + 2.0 ** -46


def certain_rows(kind, V):
    """Rows with one token left, or with one that takes almost all, and that token."""
    g = torch.Generator().manual_seed(V)
    tops = [0.0, 1.5, -7.25, 80.0, -200.0, 640.0, -640.0, 2000.0, -2000.0, 2.0 ** -46, -2.0 ** -46, 0.3, 5e-7]
    x, at = torch.full((52, V), -INF), torch.randint(0, V, (52,), generator=g)
    at[:4] = torch.tensor([0, V - 1, 2047, 2048]).clamp(max=V - 1)
    for i in range(52):
        top = tops[i % 13]
        if i >= 13:
            # others below it, few or many, until it is no longer the likeliest
            gap = [40.0, 30.0, 24.0, 20.0, 16.0, 12.0, 9.0, 7.0, 5.0, 3.0, 2.5, 2.0, 1.0][(i * 5 + i // 13) % 13]
            n = [1, 3, 200, V][i // 13]
            if n == V:
                x[i] = top - gap - 2.0 * torch.rand(V, generator=g)
            else:
                x[i, torch.randint(0, V, (n,), generator=g)] = top - gap
        x[i, at[i]] = top
    return x.to(KINDS[kind]), at


@pytest.mark.parametrize("kind,V,copies", [(k, V, (c + 7) // 8) for k, V, c in WAYS] + [(k, V, 1) for k in KINDS for V in (3, 500, 900)])
@pytest.mark.parametrize("inv_t", [1.0, 0.37, 3.0])
def test_log_probabilities_near_0(dr, kind, V, copies, inv_t):
    """0 where nothing else is left, never above it, and near it as exact as a
    float is."""
    x, at = certain_rows(kind, V)
    u = torch.full((52 * copies,), 0.5, device=DEV)
    token, logp = dr.sf_token_sample(x.to(DEV).repeat(copies, 1), u, inv_temperature=inv_t)
    token, logp = token.view(copies, 52), logp.view(copies, 52)
    assert (token >= 0).all() and (token[:, :13] == at[:13].to(DEV)).all()
    assert (logp <= 0).all() and not logp[:, :13].any(), logp[0, :13].tolist()
    for i in range(13, 52):
        p = ref.softmax(f64(x[i]), inv_t)
        for t, lp in set(zip(token[:, i].tolist(), logp[:, i].tolist())):
            v = ref.log_p(p[t])
            assert abs(lp - v) <= near_bound(v), (i, lp, v)


@pytest.mark.parametrize("kind,V,times", [("f32", 900, 1), ("bf16", 900, 1), ("f16", 9000, 1), ("f32", 9000, 4), ("bf16", 9000, 4),
                                          ("bf16", 40000, 20), ("f16", 40000, 40)])
@pytest.mark.parametrize("lookup", [False, True])
def test_verified_log_probabilities_near_0(dr, kind, V, times, lookup):
    """The same of drafts that are accepted, and of the last token."""
    x, at = certain_rows(kind, V)
    # sequences of three drafts, each the token that takes almost all
    start, draft = torch.arange(0, 40, 3, device=DEV), at.view(13, 4)[:, :3].reshape(-1).to(DEV)
    drafts = None if lookup else x.view(13, 4, V)[:, :3].reshape(39, V).to(DEV)
    u = torch.full((52,), 0.25, device=DEV)
    acc, token, logp = repeated(dr, x.to(DEV), drafts, draft, start, u, times)
    for b in range(13):
        for k in range(int(acc[0, b]) + 1):
            i = 4 * b + k
            p = ref.softmax(f64(x[i]), 1.0)
            for t, lp in set(zip(token[:, i].tolist(), logp[:, i].tolist())):
                v = ref.log_p(p[t])
                assert t >= 0 and lp <= 0 and abs(lp - v) <= near_bound(v), (i, t, lp, v)
                assert i >= 13 or lp == 0
    assert (acc[0] > 0).sum() > 5 and (acc == acc[:1]).all()


@pytest.mark.parametrize("kind", KINDS)
def test_no_log_probability_above_0(dr, kind):
    """One token left, of any size."""
    N, V = 4000, 700
    g = torch.Generator().manual_seed(9)
    x, at = torch.full((N, V), -INF), torch.randint(0, V, (N,), generator=g)
    x[torch.arange(N), at] = torch.randn(N, generator=g) * torch.logspace(-18, 3, N)
    token, logp = dr.sf_token_sample(x.to(DEV, KINDS[kind]), torch.rand(N, generator=g).to(DEV))
    assert (token == at.to(DEV)).all() and not logp.any()


def test_powers_from_a_table_are_the_same_numbers(dr):
    """Rows of many bfloat16 numbers near 0, whose powers are all but 1, and of one
    such number alone: the same bits as of a few rows."""
    V, N = 33000, 30
    g = torch.Generator().manual_seed(4)
    x = torch.randn(N, V, generator=g) * 2.0 ** (-60.0 + torch.arange(N)[:, None])
    at = torch.randint(0, V, (N,), generator=g)
    x[::2] = -INF
    x[torch.arange(N), at] = torch.randn(N, generator=g) * 2.0 ** (-60.0 + torch.arange(N))
    x = x.to(DEV, torch.bfloat16)
    u = torch.rand(N, generator=g).to(DEV)
    one = dr.sf_token_sample(x, u)
    many = dr.sf_token_sample(x.repeat(20, 1), u.repeat(20))
    assert (many[0].view(20, N) == one[0]).all() and (many[1].view(20, N) == one[1]).all()


# -- what p leaves of q, or next to nothing -----------------------------------------

def swapped(V, share, kind="f32"):
    """A target's and a draft's row that are the same but for two unlikely tokens, j
    and d, which change places: the draft has d where the target has j, and ``share``
    of its distribution is left.  Nothing else is: p = q there, bit for bit."""
    j, d = V // 3, V // 2
    p = torch.zeros(1, V, dtype=torch.float64)
    p[0, j], p[0, d] = math.log(share * (V - 2) / (1 - share)), -80.0
    q = p.clone()
    q[0, j], q[0, d] = p[0, d], p[0, j]
    target = torch.cat([p, torch.zeros(1, V)]).to(KINDS[kind])
    return target.to(DEV), q.to(KINDS[kind]).to(DEV), j, d


@pytest.mark.parametrize("V,times", [(1000, 1), (1000, 1500), (9000, 1), (9000, 300), (70001, 1), (70001, 40)])
@pytest.mark.parametrize("share", [2.0 ** -20, 2.0 ** -28, 2.0 ** -29, 1.02 * 2.0 ** -30, 0.98 * 2.0 ** -30, 2.0 ** -32, 2.0 ** -50])
def test_residual_of_next_to_nothing(dr, V, times, share):
    """A refused draft's token is drawn from what is left down to 2^-30, below that
    from p."""
    target, drafts, j, d = swapped(V, share)
    for v in (0.25, 0.9):
        u = [0.5, float(np.float32(v))]
        k, near, logp, _ = ref.verify(f64(target), f64(drafts), [d], u, 1.0, 1.0)
        assert k == 0 and (near == {j} if share > ref.LEAST else j not in near)
        got = repeated(dr, target, drafts, torch.tensor([d], device=DEV), torch.tensor([0, 1], device=DEV), torch.tensor(u, device=DEV),
                       times)
        t = int(got[1][0, 0])
        assert not got[0].any() and t in near and (got[1] == torch.tensor([t, -1], device=DEV)).all()
        assert ((got[2][:, 0].double() - logp(t)).abs() <= ref.logp_bound(logp(t))).all()


@pytest.mark.parametrize("kind,V,times", [("bf16", 9000, 1), ("bf16", 9000, 300), ("bf16", 9000, 1700), ("f16", 9000, 300)])
@pytest.mark.parametrize("share", [2.0 ** -16, 2.0 ** -28, 2.0 ** -32])
def test_residual_of_next_to_nothing_in_16_bits(dr, kind, V, times, share):
    """The same where logits are coarse, among them the sums by table."""
    target, drafts, j, d = swapped(V, share, kind)
    p, q = ref.softmax(f64(target)[0], 1.0), ref.softmax(f64(drafts)[0], 1.0)
    left = float(np.maximum(p - q, 0).sum())
    assert (left > 1.5 * ref.LEAST) == (share > ref.LEAST) and abs(left / ref.LEAST - 1) > 0.5
    u = torch.tensor([0.5, 0.25], device=DEV)
    got = repeated(dr, target, drafts, torch.tensor([d], device=DEV), torch.tensor([0, 1], device=DEV), u, times)
    want = j if share > ref.LEAST else ref.sample(f64(target)[0], 0.25, 1.0)[1]
    t = int(got[1][0, 0])
    assert not got[0].any() and (t == want if share > ref.LEAST else t in want)
    assert (got[1] == torch.tensor([t, -1], device=DEV)).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("times", [1, 400])
def test_certain_draft_that_takes_almost_all(dr, kind, times):
    """A draft without logits that is refused although it has all but 2^-23 or so of
    the probability: the token is another."""
    V, d = 9000, 5000
    target = torch.full((2, V), -4.0)
    target[0, d] = -4.0 + math.log(V) + 23 * math.log(2.0)
    target[0, :40] = -INF
    target = target.to(DEV, KINDS[kind])
    if kind == "bf16":
        target[0, d] = 21.125   # (a step of 1/8)
    p = ref.softmax(f64(target)[0], 1.0)
    assert 2.0 ** -24 < 1.0 - float(p[d]) < 2.0 ** -22
    for v in (0.0, 0.6):
        u = [1 - 2.0 ** -24, float(np.float32(v))]
        k, near, logp, _ = ref.verify(f64(target), None, [d], u, 1.0, 1.0)
        assert k == 0 and d not in near
        got = repeated(dr, target, None, torch.tensor([d], device=DEV), torch.tensor([0, 1], device=DEV), torch.tensor(u, device=DEV),
                       times)
        t = int(got[1][0, 0])
        assert not got[0].any() and t in near and (got[1][:, 0] == t).all()


# -- memory -------------------------------------------------------------------------

def test_dropout_at_large_offsets(dr):
    """Rows that begin beyond 2^31 entries of their buffer, in place: every entry
    that the mask keeps is there."""
    C, N, stride = 1031, 5, 600000000
    buf = torch.empty(stride * (N - 1) + C, dtype=torch.bfloat16, device=DEV)
    x = buf.as_strided((N, C), (stride, 1))
    g = torch.Generator().manual_seed(3)
    values = (torch.randn(N, C, generator=g) * 3.0).to(torch.bfloat16)
    values[values == 0] = 1.0
    x.copy_(values)
    keep = ref.kept(1, 1, 0, 0.5, np.arange(N * C).reshape(N, C))
    dr.sf_dropout(x, 0.5, torch.tensor([1, 1], device=DEV), out=x)
    want, bound = ref.dropout(f64(values), keep, 0.5, None, "bf16")
    assert (np.abs(f64(x) - want) <= bound).all()
    np.testing.assert_array_equal(f64(x) != 0, keep)


@pytest.mark.parametrize("lookup", [False, True])
@pytest.mark.parametrize("V,B", [(300, 2), (9000, 60), (40000, 200)])
def test_starts_outside_touch_nothing_else(dr, lookup, V, B):
    """Starts that the contract rules out: what lies around every output and the
    workspace stays."""
    D, g = 3 * B, torch.Generator().manual_seed(1)
    for kind in ("bf16", "f16"):
        target, drafts = (torch.randn(n, V, generator=g).to(DEV, KINDS[kind]) for n in (D + B, D))
        draft, u = torch.randint(0, V, (D,), generator=g).to(DEV), torch.rand(D + B, generator=g).to(DEV)
        need = dr.sf_draft_verify_workspace(KINDS[kind], D, B, V)
        for bad in ([-5, 3, 6], [0, 900000, 6], [0, 1 << 62, -(1 << 62)], [D, 0, D], [3, 3, 3], [D, D, 0]):
            start = torch.tensor((bad * B)[:B + 1], device=DEV)
            guards = [torch.full((n + 128,), 7, dtype=t, device=DEV) for n, t in
                      ((B, torch.int64), (D + B, torch.int64), (D + B, torch.float32), (need, torch.uint8))]
            acc, token, logp, space = (t[64:-64] for t in guards)
            dr.sf_draft_verify(target, None if lookup else drafts, draft, start, u, out_accepted=acc, out_token=token, out_logp=logp,
                               workspace=space)
            for t in guards:
                assert (t[:64] == 7).all() and (t[-64:] == 7).all()
