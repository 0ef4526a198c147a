"""Which kernels the entry points of stagefrontier_draw.h launch, at the edges of
their rules and at the largest sizes, and the registers of those kernels (CPU only:
launch_recorder.c stands in for the HIP runtime)."""
import os
import subprocess

import pytest

from launches import LLVM, build_recorder, spilled_vgprs
from train_launches import launches

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_06751_amd",
                   "libstagefrontier.so")
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    recorder = build_recorder(tmp_path_factory.mktemp("recorder"))
    return lambda calls: launches(recorder, LIB, calls)


def uniform(n, first=0):
    return ["sf_uniform", ["p0", ["i", 0], ["l", first], ["l", n], "p1", ["l", 0]]]


def dropout(N, C, x=BF16, out=BF16, residual=True, pad=0, stride=0):
    ld = ["l", C + pad]
    return ["sf_dropout", ["p0", ["i", x], ["l", N], ["l", C], ld, ["f", 0.1], "p1", ["i", 0], ["l", 0], ["l", stride or C],
                           "p2" if residual else ["l", 0], ld, "p3", ["i", out], ld, ["l", 0]]]


def sample(N, V, dtype=BF16):
    return ["sf_token_sample", ["p0", ["i", dtype], ["l", N], ["l", V], ["l", V], "p1", ["f", 1.0], "p2", "p3", "p4",
                                ["l", 1 << 50], ["l", 0]]]


def verify(D, B, V, dtype=BF16, lookup=False):
    return ["sf_draft_verify", ["p0", ["l", 0] if lookup else "p1", ["i", dtype], ["l", D], ["l", B], ["l", V], ["l", V],
                                ["l", V], "p2", "p3", "p4", ["f", 1.0], ["f", 1.0], "p5", "p6", "p7", "p8",
                                ["l", 1 << 58], ["l", 0]]]


def fits(got):
    assert got and all(0 < grid * block < 1 << 32 for call in got for _, grid, block in call)


@pytest.mark.parametrize("N,V,dtype,kernels", [
    (1, 1, BF16, ["short<1, 1>"]), (1, 519, BF16, ["short<1, 1>"]), (1, 520, BF16, ["short<1, 2>"]),
    (1, 1031, F16, ["short<2, 2>"]), (1, 1032, F16, ["short<2, 4>"]), (9, 2048, F16, ["short<2, 4>"]),
    (9, 259, F32, ["short<0, 1>"]), (9, 1024, F32, ["short<0, 4>"]), (9, 1025, F32, ["sample<0, 1024, 16>"]),
    (1, 2049, BF16, ["sample<1, 1024, 16>"]), (255, 65536, BF16, ["sample<1, 1024, 16>"]),
    (256, 65536, BF16, ["row_table", "draw<1>"]), (255, 65537, BF16, ["row_table", "draw<1>"]),
    (248, 65537, BF16, ["row_segments<1>", "draw<1>"]), (1024, 30700, BF16, ["sample<1, 256, 4>"]),
    (1024, 30750, BF16, ["row_table", "draw<1>"]), (512, 30750, BF16, ["row_table", "draw<1>"]),
    (511, 30750, BF16, ["sample<1, 1024, 16>"]), (9000, 30700, BF16, ["sample<1, 256, 1>"]),
    (511, 65536, F16, ["sample<2, 1024, 16>"]), (511, 65537, F16, ["row_segments<2>", "draw<2>"]),
    (512, 65537, F16, ["sample<2, 256, 4>"]), (512, 2097152, F16, ["sample<2, 256, 4>"]),
    (512, 2097153, F16, ["row_segments<2>", "draw<2>"]), (4095, 524288, F16, ["sample<2, 256, 4>"]),
    (4096, 524288, F16, ["sample<2, 256, 1>"]), (4096, 524289, F16, ["sample<2, 256, 4>"]),
    (1 << 20, 1 << 22, BF16, ["row_segments<1>", "draw<1>"])])
def test_sample_launches(run, N, V, dtype, kernels):
    got = run([sample(N, V, dtype)])[0]
    assert [g[0].split("k_", 1)[1].replace("token_", "") for g in got] == kernels


@pytest.mark.parametrize("D,B,V,lookup,kernels", [
    (0, 1, 5, False, ["row_segments<1>", "draft_few<1>", "draft_draw<1>"]),
    (5, 1, 65536, False, ["row_segments<1>", "draft_few<1>", "draft_draw<1>"]),
    (5, 1, 65536, True, ["row_segments<1>", "draft_decide<1, true>"]),
    (32, 32, 65536, False, ["row_segments<1>", "draft_few<1>", "draft_draw<1>"]),
    (32, 33, 65536, False, ["row_segments<1>", "draft_decide<1, false>", "draft_residual<1>", "draft_draw<1>"]),
    (1024, 256, 131072, False, ["row_table", "draft_decide<1, false>", "residual_table", "draft_draw<1>"]),
    (511, 256, 131072, False, ["row_table", "draft_decide<1, false>", "residual_table", "draft_draw<1>"]),
    (128, 128, 131072, False, ["row_table", "draft_decide<1, false>", "residual_table", "draft_draw<1>"]),
    (128, 127, 131072, False, ["row_table", "draft_decide<1, false>", "draft_residual<1>", "draft_draw<1>"]),
    (127, 128, 131072, False, ["row_segments<1>", "draft_decide<1, false>", "residual_table", "draft_draw<1>"]),
    (900, 200, 50001, True, ["draft_segments<1>", "draft_alive<1>", "draft_segments<1>", "draft_decide<1, true>"]),
    (900, 200, 20000, True, ["row_table", "draft_decide<1, true>"]),
    (300, 200, 50001, True, ["row_table", "draft_decide<1, true>"])])
def test_verify_launches(run, D, B, V, lookup, kernels):
    got = run([verify(D, B, V, BF16, lookup)])[0]
    assert [g[0].split("k_", 1)[1] for g in got] == kernels


@pytest.mark.parametrize("D,B,V,kernels", [
    (1024, 256, 131072, ["draft_segments<2>", "draft_alive<2>", "draft_segments<2>", "draft_decide<2, false>",
                         "draft_residual<2>", "draft_draw<2>"]),
    (511, 256, 131072, ["row_segments<2>", "draft_decide<2, false>", "draft_residual<2>", "draft_draw<2>"]),
    (512, 256, 105000, ["draft_segments<2>", "draft_alive<2>", "draft_segments<2>", "draft_decide<2, false>",
                        "draft_residual<2>", "draft_draw<2>"]),
    (512, 256, 104000, ["row_segments<2>", "draft_decide<2, false>", "draft_residual<2>", "draft_draw<2>"])])
def test_verify_launches_without_a_table(run, D, B, V, kernels):
    assert [g[0].split("k_", 1)[1] for g in run([verify(D, B, V, F16)])[0]] == kernels


@pytest.mark.parametrize("inv_t,iq,kernels", [
    (1.0, 1.0, ["row_table", "draft_decide<1, false>", "residual_table", "draft_draw<1>"]),
    (1.0, 0.5, ["row_table", "row_table", "draft_decide<1, false>", "draft_residual<1>", "draft_draw<1>"]),
    (2.0 ** 100, 1.0, ["row_segments<1>", "draft_decide<1, false>", "draft_residual<1>", "draft_draw<1>"]),
    (2.0 ** -110, 2.0 ** -110, ["row_table", "draft_decide<1, false>", "residual_table", "draft_draw<1>"]),
    (2.0 ** -120, 2.0 ** -120, ["draft_segments<1>", "draft_alive<1>", "draft_segments<1>", "draft_decide<1, false>",
                                "draft_residual<1>", "draft_draw<1>"])])
def test_tables_of_temperatures(run, inv_t, iq, kernels):
    """A table serves one temperature, whose range of powers a bfloat16 has."""
    call = verify(1024, 256, 131072)
    call[1][11:13] = [["f", inv_t], ["f", iq]]
    assert [g[0].split("k_", 1)[1] for g in run([call])[0]] == kernels


@pytest.mark.parametrize("N,C,kw,far,grid", [
    (1, 1, {}, False, 1), (4096, 2048, {}, False, 4097), (16384, 8192, {}, True, 65537),
    (5000, 5, dict(pad=1), False, 1), (5000, 8000, dict(pad=1), False, 4), (16384, 8192, dict(residual=False, x=F32), True, 65537),
    (10922, 4096, {}, False, 21845), (10923, 4096, {}, True, 21847), (10923, 4096, dict(residual=False), False, 21847)])
def test_dropout_launches(run, N, C, kw, far, grid):
    (name, got, block), = run([dropout(N, C, **kw)])[0]
    assert name.startswith("k_dropout") and name.endswith("true>" if far else "false>") and block == 256
    assert got == grid


def test_largest(run):
    fits(run([uniform((1 << 44) - 1), uniform(5, (1 << 60) - 5)]))
    fits(run([dropout(1 << 20, 1 << 20), dropout(1 << 40, 3, pad=1), dropout(1, 1 << 40), dropout(5, 1 << 36, pad=7)]))
    fits(run([sample(N, V, d) for N, V in ((1, 1 << 30), (1 << 14, 1 << 30), (1 << 30, 1 << 14), (1 << 40, 5), (1 << 24, 100003))
              for d in (F32, BF16)]))
    fits(run([verify(D, B, V, d, lookup) for D, B, V in ((0, 1, 1 << 30), (1 << 12, 1, 1 << 30), (1 << 12, 1 << 12, 1 << 30),
                                                        ((1 << 31) - 1, (1 << 31) - 1, 5), ((1 << 31) - 1, 1, 1000),
                                                        ((1 << 31) - 1, 1 << 20, 1000), (0, (1 << 31) - 1, 100),
                                                        (1 << 19, 1 << 19, 1 << 20))
              for d in (F32, BF16) for lookup in (False, True)]))


def test_kernels_keep_nothing_in_memory(tmp_path):
    """No kernel of the library's third part has a stack of its own in memory."""
    data, held = open(LIB, "rb").read(), {}
    at = data.find(b"\x7fELF", 4)
    while at >= 0:
        if int.from_bytes(data[at + 18:at + 20], "little") == 224:  # an AMDGPU code object
            end = data.find(b"\x7fELF", at + 4)
            path = tmp_path / "object.elf"
            path.write_bytes(data[at:end if end > 0 else len(data)])
            notes = subprocess.run([LLVM + "llvm-readelf", "--notes", str(path)], capture_output=True, text=True).stdout
            name = None
            for line in notes.split("\n"):
                key, _, value = line.strip().lstrip("- ").partition(":")
                if key == ".name" and value.strip().startswith("_Z"):
                    name = value.strip()
                elif key == ".private_segment_fixed_size" and name:
                    held[name] = int(value)
        at = data.find(b"\x7fELF", at + 4)
    mine = {n: v for n, v in held.items() if any(k in n for k in ("k_uniform", "k_dropout", "k_token_short", "k_token_sample",
                                                                 "k_token_draw", "k_row_", "k_draft", "k_residual"))}
    assert len(mine) >= 50 and not any(mine.values()), mine


def test_kernels_spill_nothing(tmp_path):
    mine = {k: n for k, n in spilled_vgprs(tmp_path).items()
            if k.startswith(("k_uniform", "k_dropout", "k_token_short", "k_token_sample", "k_token_draw", "k_row_", "k_draft", "k_residual"))}
    assert len(mine) >= 50 and not any(mine.values()), mine
