"""Which kernels the entry points of stagefrontier_train.h launch, at the edges
of their rules, and the registers of those kernels (CPU only: launch_recorder.c
stands in for the HIP runtime)."""
import os

import pytest

from launches import build_recorder, spilled_vgprs
from train_launches import launches

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_06751_amd",
                   "libstagefrontier.so")
BF16, F32 = 1, 0


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    recorder = build_recorder(tmp_path_factory.mktemp("recorder"))
    return lambda calls: launches(recorder, LIB, calls)


def logp(N, V, dtype=BF16):
    return ["sf_token_logp", ["p0", ["i", dtype], ["l", N], ["l", V], ["l", V], "p1", ["f", 1.0], "p2", "p3", "p4", "p5",
                              ["l", 1 << 40], ["l", 0]]]


@pytest.mark.parametrize("N,V,dtype,kernels", [
    (1, 2048, BF16, ["<1, 256, 1>"]), (1, 2049, BF16, ["<1, 1024, 16>"]), (1, 65536, BF16, ["<1, 1024, 16>"]),
    (1, 65537, BF16, ["<1, 256, 4>", "join<1>"]), (64, 65537, BF16, ["<1, 256, 4>", "join<1>"]),
    (65, 65537, BF16, ["<1, 1024, 16>"]), (256, 65537, BF16, ["<1, 1024, 16>"]), (257, 65537, BF16, ["<1, 256, 4>"]),
    (2047, 32768, BF16, ["<1, 256, 4>"]), (2048, 32768, BF16, ["<1, 256, 1>"]), (2048, 32769, BF16, ["<1, 256, 4>"]),
    (8191, 32768, BF16, ["<1, 256, 1>"]), (8192, 10240, BF16, ["<1, 256, 1>"]), (8192, 10241, BF16, ["<1, 256, 4>"]),
    (2048, 16384, F32, ["<0, 256, 1>"]), (2048, 16385, F32, ["<0, 256, 4>"]), (1, 32769, F32, ["<0, 256, 4>", "join<0>"])])
def test_rows(run, N, V, dtype, kernels):
    got = run([logp(N, V, dtype)])[0]
    assert len(got) == len(kernels)
    for (name, grid, block), want in zip(got, kernels):
        assert name.endswith(want), (name, want)
    if len(kernels) == 1:  # rows of a workgroup
        per = 4 if kernels[0].endswith("256, 1>") else 1
        assert got[0][1] == -(-N // per)


def grad(N, V):
    return ["sf_token_logp_grad", ["p0", ["i", BF16], ["l", N], ["l", V], ["l", V], "p1", ["f", 1.0], "p2", "p3", "p4",
                                   "p5", "p6", ["l", V], ["l", 0]]]


@pytest.mark.parametrize("V,kernel,chunks", [(1, "64>", 1), (1031, "64>", 1), (1032, "256>", 1), (4096, "256>", 1),
                                             (4104, "256>", 2), (131072, "256>", 32)])
def test_gradient_chunks(run, V, kernel, chunks):
    (name, grid, block), = run([grad(10, V)])[0]
    assert name.endswith(kernel) and grid == chunks and block == 256


def policy(N, B, reduction, mask):
    return ["sf_policy_loss", ["p0", "p1", "p2", "p3", ["i", 0], "p4" if mask else ["l", 0], "p5", ["l", N], ["l", B],
                               ["i", reduction], ["f", 1.0], ["f", 0.2], ["f", 0.2], ["f", 0.1], "p6", "p7", "p8",
                               ["l", 1 << 40], ["l", 0]]]


@pytest.mark.parametrize("N,B,reduction,mask,kernels", [
    (8192, 1024, 1, True, ["small"]), (0, 0, 0, False, ["small"]),
    (8193, 1024, 2, True, ["loss", "join"]), (8193, 1024, 0, False, ["loss", "join"]),
    (8193, 1024, 0, True, ["count<0>", "loss", "join"]),
    (8193, 1024, 1, True, ["count<1>", "loss", "join"]), (8192, 1025, 1, False, ["count<1>", "loss", "join"]), (8193, 256, 1, False, ["loss", "join"]),
    (8193, 257, 1, False, ["count<1>", "loss", "join"]), (8193, 2048, 1, True, ["count<1>", "loss", "join"]),
    (8193, 2049, 1, True, ["count<2>", "loss", "join"]),
    (100000, 5000, 1, True, ["count<2>", "loss", "join"]), (100000, 5000, 0, False, ["loss", "join"]),
    (100000, 0, 1, True, ["loss", "join"]), (0, 2000, 0, True, ["join"])])
def test_policy_launches(run, N, B, reduction, mask, kernels):
    got = run([policy(N, B, reduction, mask)])[0]
    assert [g[0] for g in got] == ["k_policy_" + k for k in kernels]


def norm(sizes, dtype=BF16):
    return ["sf_grad_norm", [["list", [[9, n, dtype] for n in sizes]], "p0", "p1", "p2", "p3", ["l", 1 << 40], ["l", 0]]]


@pytest.mark.parametrize("sizes,kernels", [
    ([], ["norm_empty"]), ([0], ["norm", "norm_join"]), ([5] * 192, ["norm", "norm_join"]),
    ([5] * 193, ["norm", "norm", "norm_join"]), ([5] * 1025, ["norm"] * 6 + ["norm_item", "norm_total"]),
    ([4096 * 256], ["norm", "norm_join"]), ([4096 * 256 + 1], ["norm", "norm_item", "norm_total"])])
def test_norm_launches(run, sizes, kernels):
    got = run([norm(sizes)])[0]
    assert [g[0] for g in got] == ["k_grad_" + k for k in kernels]


def test_norm_chunks(run):
    """Batches of equal numbers of tensors, chunks that span no two of them."""
    got = run([norm([5] * 193), norm([4096, 4097, 0, 1]), norm([1 << 30])])
    assert [g[1] for g in got[0][:2]] == [97, 96]
    assert got[1][0][1] == 1 + 2 + 0 + 1
    assert got[2][0][1] == (1 << 30) // (1 << 16)


@pytest.mark.parametrize("n,grids", [(1, [3]), (128, [384]), (129, [195, 192]), (0, [])])
def test_clip_launches(run, n, grids):
    sizes = [[9, 8192 * 2 + 1, F32]] * n
    out = [[20, 8192 * 2 + 1, F32]] * n
    got = run([["sf_grad_clip", [["list", sizes], ["list", out], "p0", ["l", 4], ["f", 1.0], ["f", 0.0], "p1", ["l", 0]]]])[0]
    assert [g[0] for g in got] == ["k_grad_clip"] * len(grids) and [g[1] for g in got] == grids


def test_kernels_spill_nothing(tmp_path):
    mine = {k: n for k, n in spilled_vgprs(tmp_path).items() if k.startswith(("k_token_", "k_policy_", "k_grad_"))}
    assert len(mine) >= 20 and not any(mine.values()), mine
