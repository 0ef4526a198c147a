"""The third header: plain C, every declared entry point exported and bound, bad
arguments refused on the host before any device work (CPU only: no call here
reaches a kernel)."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "stagefrontier_draw.h")
A, B, C, D, E, F, G, W, X = (k << 44 for k in range(1, 10))  # device addresses that nothing reads


def declared():
    with open(HEADER) as fh:
        text = re.sub(r"/\*.*?\*/", "", fh.read(), flags=re.S)
    return sorted(set(re.findall(r"\b(sf_[a-z0-9_]+)\s*\(", text)))


@pytest.fixture(scope="module")
def dr():
    import torch  # noqa: F401
    from paper_2606_06751_amd import draw
    return draw


@pytest.fixture(scope="module")
def sf():
    from paper_2606_06751_amd import stagefrontier
    return stagefrontier


@pytest.fixture(scope="module")
def lib(dr):
    return dr._lib


def test_declared_and_exported(lib):
    assert declared() == ["sf_draft_verify", "sf_draft_verify_workspace", "sf_dropout", "sf_token_sample",
                          "sf_token_sample_workspace", "sf_uniform"]
    for name in declared():
        assert getattr(lib, name).argtypes is not None


def test_package_names(dr):
    import paper_2606_06751_amd as pkg
    assert sorted(pkg._DRAW_NAMES) == declared()
    for name in pkg._DRAW_NAMES:
        assert getattr(pkg, name) is getattr(dr, name)


def test_header_is_plain_c(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "use.c"
    src.write_text('#include "stagefrontier_draw.h"\n'
                   "int use(void) { return SF_BF16 + (int)sf_token_sample_workspace(0, 1, 1); }\n")
    p = subprocess.run([cc, "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"),
                        "-c", str(src), "-o", str(tmp_path / "use.o")], capture_output=True, text=True)
    assert p.returncode == 0, p.stderr


def test_uniform_refusals(sf, lib):
    def call(**k):
        a = dict(dict(key=A, site=0, first=0, n=100, out=B), **k)
        return lib.sf_uniform(a["key"], a["site"], a["first"], a["n"], a["out"], None)

    assert call(n=0, key=None, out=None) == sf.SF_OK
    for bad in (dict(n=-1), dict(first=-1), dict(first=1 << 60), dict(n=(1 << 60) + 1), dict(first=(1 << 62)), dict(key=None), dict(out=None),
                dict(key=A + 4), dict(out=B + 2), dict(out=A + 8), dict(out=A - 8)):
        assert call(**bad) == sf.SF_EINVAL, bad


def test_dropout_refusals(sf, lib):
    def call(**k):
        a = dict(dict(x=A, dt=1, N=10, C=100, xs=100, p=0.1, key=B, site=0, first=0, istr=100, r=C, rs=100, o=D, odt=1,
                      os=100), **k)
        return lib.sf_dropout(a["x"], a["dt"], a["N"], a["C"], a["xs"], a["p"], a["key"], a["site"], a["first"], a["istr"],
                              a["r"], a["rs"], a["o"], a["odt"], a["os"], None)

    for none in (dict(N=0), dict(C=0, xs=0, istr=0, r=None, os=0)):
        assert call(x=None, key=None, o=None, **none) == sf.SF_OK
    for bad in (dict(dt=3), dict(odt=-1), dict(N=-1), dict(C=-1), dict(N=(1 << 40) + 1), dict(xs=99), dict(os=99), dict(rs=99),
                dict(p=-0.01), dict(p=1.01), dict(p=float("nan")), dict(first=-1), dict(istr=99), dict(first=(1 << 60) - 500),
                dict(istr=1 << 60), dict(N=1 << 30, xs=1 << 30, istr=1 << 30), dict(x=None), dict(key=None), dict(o=None),
                dict(x=A + 1), dict(key=B + 4), dict(o=D + 1), dict(r=C + 1),
                dict(o=A + 2), dict(o=A, xs=120), dict(o=A, odt=0), dict(o=A + 1998), dict(o=C + 200), dict(o=C, rs=101),
                dict(o=B - 8), dict(r=A, o=A, dt=0)):
        assert call(**bad) == sf.SF_EINVAL, bad


def test_token_sample_refusals(sf, lib):
    def call(**k):
        a = dict(dict(x=A, dt=1, N=10, V=100, ld=100, u=B, it=1.0, t=C, lp=D, ws=W, wb=1 << 30), **k)
        return lib.sf_token_sample(a["x"], a["dt"], a["N"], a["V"], a["ld"], a["u"], a["it"], a["t"], a["lp"], a["ws"],
                                   a["wb"], None)

    assert call(N=0, x=None, u=None, t=None, lp=None, ws=None) == sf.SF_OK
    V = 1 << 20  # one row of many logits is split, and needs its workspace
    need = lib.sf_token_sample_workspace(1, 1, V)
    assert need > 0 and need % 4 == 0
    for bad in (dict(dt=3), dict(dt=-1), dict(N=-1), dict(V=0), dict(V=(1 << 30) + 1, ld=1 << 31), dict(ld=99), dict(it=0.0),
                dict(it=-1.0), dict(it=float("inf")), dict(it=float("nan")), dict(x=None), dict(u=None), dict(t=None),
                dict(lp=None), dict(x=A + 1), dict(u=B + 2), dict(t=C + 4), dict(lp=D + 1), dict(t=A + 8), dict(lp=B + 8),
                dict(lp=C + 16), dict(N=1 << 50, ld=1 << 20), dict(N=1, V=V, ld=V, ws=None),
                dict(N=1, V=V, ld=V, wb=need - 1), dict(N=1, V=V, ld=V, ws=W + 4), dict(N=1, V=V, ld=V, ws=A + 64),
                dict(N=1, V=V, ld=V, ws=C)):
        assert call(**bad) == sf.SF_EINVAL, bad
    for bad in ((1, 1, 0), (1, -1, 5), (3, 1, 5), (0, 1, 1 << 31)):
        assert lib.sf_token_sample_workspace(*bad) == -1, bad
    assert lib.sf_token_sample_workspace(0, 0, 5) == 0 and lib.sf_token_sample_workspace(2, 100000, 32000) == 0


def test_draft_verify_refusals(sf, lib):
    need = lib.sf_draft_verify_workspace(2, 30, 10, 1000)
    assert need > 0

    def call(**k):
        a = dict(dict(x=A, q=B, dt=2, D=30, B=10, V=1000, ld=1000, lq=1000, d=C, s=D, u=E, it=1.0, iq=1.0, acc=F, t=G,
                      lp=X, ws=W, wb=need), **k)
        return lib.sf_draft_verify(a["x"], a["q"], a["dt"], a["D"], a["B"], a["V"], a["ld"], a["lq"], a["d"], a["s"], a["u"],
                                   a["it"], a["iq"], a["acc"], a["t"], a["lp"], a["ws"], a["wb"], None)

    assert call(B=0, D=0, x=None, q=None, d=None, s=None, u=None, acc=None, t=None, lp=None, ws=None) == sf.SF_OK
    for bad in (dict(dt=3), dict(D=-1), dict(B=-1), dict(D=1 << 31), dict(B=1 << 31), dict(V=0), dict(V=(1 << 30) + 1),
                dict(ld=999), dict(lq=999), dict(it=0.0), dict(iq=0.0), dict(iq=float("nan")), dict(it=float("inf")),
                dict(x=None), dict(d=None), dict(s=None), dict(u=None), dict(acc=None), dict(t=None), dict(lp=None),
                dict(ws=None), dict(wb=need - 1), dict(x=A + 1), dict(q=B + 1), dict(d=C + 4), dict(s=D + 4), dict(u=E + 2),
                dict(acc=F + 4), dict(t=G + 4), dict(lp=X + 2), dict(ws=W + 8), dict(t=C), dict(acc=D), dict(lp=E + 8),
                dict(ws=A + 1600), dict(ws=B + 1600), dict(t=F + 8), dict(lp=G + 8), dict(ws=X - 16)):
        assert call(**bad) == sf.SF_EINVAL, bad
    for bad in ((3, 1, 1, 5), (0, -1, 1, 5), (0, 1, -1, 5), (0, 1, 1, 0), (0, 1 << 31, 1, 5), (0, 1, 1 << 31, 5)):
        assert lib.sf_draft_verify_workspace(*bad) == -1, bad
    assert lib.sf_draft_verify_workspace(0, 5, 0, 5) == 0
