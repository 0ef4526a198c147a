"""The oracle of the draws against published values and cases by hand (CPU)."""
import math

import numpy as np
import pytest

import draw_ref as ref


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((ref.WORD,) * 4, (ref.WORD,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_philox_known_answers(counter, key, want):
    """The generator's published answers (Random123's kat_vectors)."""
    assert tuple(ref.philox(counter, key)) == want


def test_uniform_and_mask():
    u = ref.uniform(-5, 7, 3, 1, 4000)
    assert (u >= 0).all() and (u < 1).all() and (u * 2 ** 24 == np.round(u * 2 ** 24)).all()
    assert abs(u.mean() - 0.5) < 4 / math.sqrt(12 * 4000)
    assert ref.uniform(-5, 7, 3, 2, 3999).tolist() == u[1:].tolist()
    assert ref.uniform(-5, 7 + (1 << 32), 3, 1, 4).tolist() == u[:4].tolist()
    keep = ref.kept(9, 0, 0, 0.25, np.arange(8000).reshape(8, 1000))
    assert abs(keep.mean() - 0.75) < 4 * math.sqrt(0.1875 / 8000)
    assert ref.kept(9, 0, 0, 0.0, np.arange(99)).all() and not ref.kept(9, 0, 0, 1.0, np.arange(99)).any()
    assert ref.threshold(1e-6) == 0 and ref.threshold(0.5) == 32768 and ref.threshold(0.1) == 6554


def test_sample_by_hand():
    x = np.log([0.25, 0.5, 0.0 + 1e-300, 0.25]).tolist()
    x[2] = -math.inf
    for u, t in ((0.0, 0), (0.2, 0), (0.26, 1), (0.74, 1), (0.76, 3), (1 - 2.0 ** -24, 3)):
        token, near, logp = ref.sample(x, u, 1.0)
        assert token == t and near == {t} and abs(logp(t) - x[t]) < 1e-12
    assert ref.sample(x, 0.25, 1.0)[1] == {0, 1}
    assert ref.sample(x, 1.0, 1.0)[0] == ref.sample(x, math.nan, 1.0)[0] == -1
    assert ref.sample([-math.inf] * 3, 0.5, 1.0)[0] == -1 and ref.sample([-math.inf] * 3, 0.5, 1.0)[2](-1) == -math.inf
    assert math.isnan(ref.sample([1.0, math.nan], 0.5, 1.0)[2](-1)) and math.isnan(ref.sample([1.0, math.inf], 0.5, 1.0)[2](-1))


def test_verify_by_hand():
    p, q = np.log([0.5, 0.25, 0.25]), np.log([0.25, 0.5, 0.25])
    run = lambda d, u, **k: ref.verify([p, p], [q], [d], u, 1.0, 1.0, **k)  # noqa: E731
    assert run(0, [0.9, 0.1])[:2] == (1, {0})          # p > q: accepted, then from p
    assert run(0, [0.9, 0.6])[1] == {1}
    assert run(1, [0.4, 0.1])[0] == 1 and run(1, [0.6, 0.9])[:2] == (0, {0})  # only token 0 is left
    assert run(2, [0.99, 0.1])[0] == 1
    assert run(1, [0.5, 0.1]) is None                   # at the border
    assert ref.verify([p, p], None, [0], [0.4, 0.3], 1.0, 1.0)[:2] == (1, {0})
    assert ref.verify([p, p], None, [0], [0.6, 0.6], 1.0, 1.0)[:2] == (0, {2})
    assert run(-1, [0.6, 0.6])[:2] == (0, {1})          # no draft: from p
    assert run(0, [1.5, 0.6])[:2] == (0, {-1})


@pytest.mark.parametrize("lookup", [False, True])
def test_verified_tokens_are_the_targets(lookup):
    """Drafts from q, verified against p, leave p: summed over all drafts and
    outcomes, exactly."""
    rng = np.random.default_rng(3)
    p, q = rng.dirichlet(np.ones(6)), rng.dirichlet(np.ones(6))
    if lookup:
        q = np.eye(6)[2]
    accept = np.where(q > 0, np.minimum(1, p / np.where(q > 0, q, 1)), 0)
    residual = np.maximum(p - q, 0)
    got = q * accept + (1 - (q * accept).sum()) * residual / residual.sum()
    np.testing.assert_allclose(got, p, atol=1e-15)


@pytest.mark.parametrize("share,left", [(2.0 ** -29, True), (1.01 * 2.0 ** -30, True), (0.99 * 2.0 ** -30, False), (2.0 ** -33, False)])
def test_verify_next_to_nothing_by_hand(share, left):
    """A refused draft's token comes from what p has more of than q, here token 3
    alone, down to a share of 2^-30; below that from p."""
    p = np.log([0.5, 0.25, 0.25, share, 1e-100])
    q = np.log([0.5, 0.25, 0.25, 1e-100, share])
    for u, t in ((0.3, 0), (0.6, 1), (0.9, 2)):
        assert ref.verify([p, p], [q], [4], [0.5, u], 1.0, 1.0)[:2] == (0, {3 if left else t})
    # without the draft's distribution only its own share is taken from p
    assert ref.verify([p, p], None, [4], [0.5, 0.6], 1.0, 1.0)[:2] == (0, {1})
