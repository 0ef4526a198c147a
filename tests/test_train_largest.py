"""The largest sizes that the second header accepts: every launch stays below
2^32 threads in a dimension (CPU only: launch_recorder.c stands in for the HIP
runtime)."""
import os

import pytest

from launches import build_recorder
from train_launches import launches

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_06751_amd",
                   "libstagefrontier.so")


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    recorder = build_recorder(tmp_path_factory.mktemp("recorder"))
    return lambda calls: launches(recorder, LIB, calls)


def fits(got):
    assert got and all(0 < grid * block < 1 << 32 for call in got for _, grid, block in call)


N_MOST = (1 << 34) - (1 << 11)


@pytest.mark.parametrize("reduction", [0, 1, 2])
@pytest.mark.parametrize("B", [1, 300, 5000, (1 << 31) - 1])
def test_policy_of_most_tokens(run, B, reduction):
    got = run([["sf_policy_loss", ["p0", "p1", "p2", "p3", ["i", 0], "p4", "p5", ["l", N_MOST], ["l", B], ["i", reduction],
                                   ["f", 1.0], ["f", 0.2], ["f", 0.2], ["f", 0.1], "p6", "p7", "p8", ["l", 1 << 45],
                                   ["l", 0]]]])
    assert [name for name, _, _ in got[0]][-2:] == ["k_policy_loss", "k_policy_join"]
    fits(got)


def test_policy_of_more_tokens_is_refused():
    torch = pytest.importorskip("torch")  # noqa: F841  (its HIP runtime comes first)
    from paper_2606_06751_amd import stagefrontier, train
    lib = stagefrontier.raw_library()
    p = [k << 46 for k in range(1, 10)]
    for N in (N_MOST + 1, (1 << 34) - 1):
        assert lib.sf_policy_loss_workspace(N, 8) == -1
        assert lib.sf_policy_loss(*p[:4], 0, p[4], p[5], N, 8, 0, 1.0, 0.2, 0.2, 0.1, p[6], p[7], p[8], 1 << 45,
                                  None) == train.SF_EINVAL
    assert lib.sf_policy_loss_workspace(N_MOST, 8) > 0


@pytest.mark.parametrize("sizes", [[(1 << 40) - 1], [(1 << 39) + 1], [1, (1 << 40) - 5000] + [3] * 1000, [1 << 30] * 1000])
def test_norm_and_clip_of_most_entries(run, sizes):
    grads, out = ["list", [[9, n, 1] for n in sizes]], ["list", [[20 + 60 * k, n, 1] for k, n in enumerate(sizes[:1])]]
    calls = [["sf_grad_norm", [grads, "p0", "p1", "p2", "p3", ["l", 1 << 44], ["l", 0]]],
             ["sf_grad_clip", [grads, grads, "p0", ["l", 4], ["f", 1.0], ["f", 0.0], "p1", ["l", 0]]]]
    if len(sizes) == 1:
        calls.append(["sf_grad_clip", [grads, out, "p0", ["l", 4], ["f", 1.0], ["f", 0.0], "p1", ["l", 0]]])
    fits(run(calls))


@pytest.mark.parametrize("N,V", [(1, 1 << 30), (1 << 14, 1 << 30), (1 << 30, 1 << 14), (1 << 40, 5), (1 << 24, 100003)])
def test_rows_of_most_logits(run, N, V):
    ld = ["l", V]
    fits(run([["sf_token_logp", ["p0", ["i", 1], ["l", N], ["l", V], ld, "p1", ["f", 1.0], "p2", "p3", "p4", "p5",
                                 ["l", 1 << 44], ["l", 0]]],
              ["sf_token_logp_grad", ["p0", ["i", 1], ["l", N], ["l", V], ld, "p1", ["f", 1.0], "p2", "p3", "p4", "p5",
                                      "p6", ld, ["l", 0]]]]))
