"""The second header: plain C, every declared entry point exported and bound,
bad arguments refused on the host before any device work (CPU only: no call
here reaches a kernel)."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "stagefrontier_train.h")
A, B, C, D, E, F, G, W = (k << 40 for k in range(1, 9))  # device addresses that nothing reads


def declared():
    with open(HEADER) as fh:
        text = re.sub(r"/\*.*?\*/", "", fh.read(), flags=re.S)
    return sorted(set(re.findall(r"\b(sf_[a-z0-9_]+)\s*\(", text)))


@pytest.fixture(scope="module")
def tr():
    import torch  # noqa: F401
    from paper_2606_06751_amd import train
    return train


@pytest.fixture(scope="module")
def lib(tr):
    from paper_2606_06751_amd import stagefrontier
    return stagefrontier.raw_library()


def test_declared_and_exported(lib):
    assert declared() == ["sf_grad_clip", "sf_grad_list_bytes", "sf_grad_list_init", "sf_grad_norm",
                          "sf_grad_norm_workspace", "sf_policy_loss", "sf_policy_loss_workspace", "sf_token_logp",
                          "sf_token_logp_grad", "sf_token_logp_workspace"]
    for name in declared():
        assert getattr(lib, name).argtypes is not None


def test_package_names(tr):
    import paper_2606_06751_amd as pkg
    for name in pkg._TRAIN_NAMES:
        assert getattr(pkg, name) is getattr(tr, name)


def test_header_is_plain_c(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "use.c"
    src.write_text('#include "stagefrontier_train.h"\n'
                   "int use(void) { return SF_BF16 + SF_SUM_TOKENS + (int)sf_grad_list_bytes(0); }\n")
    p = subprocess.run([cc, "-std=c99", "-Wall", "-Wextra", "-pedantic", "-Werror", "-I", os.path.join(ROOT, "include"),
                        "-c", str(src), "-o", str(tmp_path / "use.o")], capture_output=True, text=True)
    assert p.returncode == 0, p.stderr


def test_token_logp_refusals(tr, lib):
    def call(**k):
        a = dict(dict(x=A, dt=1, N=10, V=100, ld=100, t=B, it=1.0, lp=C, lse=D, h=E, ws=W, wb=1 << 30), **k)
        return lib.sf_token_logp(a["x"], a["dt"], a["N"], a["V"], a["ld"], a["t"], a["it"], a["lp"], a["lse"], a["h"],
                                 a["ws"], a["wb"], None)

    assert call(N=0, x=None, t=None, lp=None, lse=None, h=None, ws=None) == tr.SF_OK
    for bad in (dict(dt=3), dict(dt=-1), dict(N=-1), dict(V=0), dict(V=(1 << 30) + 1, ld=1 << 31), dict(ld=99),
                dict(it=0.0), dict(it=-1.0), dict(it=float("inf")), dict(it=float("nan")), dict(x=None), dict(t=None),
                dict(lp=None), dict(lse=None), dict(x=A + 1), dict(t=B + 4), dict(lp=C + 2), dict(lse=D + 1),
                dict(h=E + 2), dict(lp=D + 8), dict(lp=A + 8), dict(h=B + 16), dict(N=1 << 50, ld=1 << 20)):
        assert call(**bad) == tr.SF_EINVAL, bad
    # one row of many logits is split, and needs its workspace
    V = 1 << 20
    need = lib.sf_token_logp_workspace(1, 1, V)
    assert need > 0 and need % 4 == 0
    for bad in (dict(ws=None), dict(wb=need - 1), dict(ws=W + 4), dict(ws=A + 64)):
        assert call(N=1, V=V, ld=V, **bad) == tr.SF_EINVAL, bad
    for bad in ((1, 1, 0), (1, -1, 5), (3, 1, 5), (0, 1, 1 << 31)):
        assert lib.sf_token_logp_workspace(*bad) == -1, bad
    assert lib.sf_token_logp_workspace(0, 0, 5) == 0 and lib.sf_token_logp_workspace(2, 100000, 32000) == 0


def test_token_logp_grad_refusals(tr, lib):
    def call(**k):
        a = dict(dict(x=A, dt=2, N=10, V=100, ld=128, t=B, it=1.0, lse=C, g=D, h=E, gh=F, o=G, lo=128), **k)
        return lib.sf_token_logp_grad(a["x"], a["dt"], a["N"], a["V"], a["ld"], a["t"], a["it"], a["lse"], a["g"],
                                      a["h"], a["gh"], a["o"], a["lo"], None)

    assert call(N=0, x=None, t=None, lse=None, g=None, h=None, gh=None, o=None) == tr.SF_OK
    for bad in (dict(dt=9), dict(V=0), dict(ld=99), dict(lo=99), dict(it=0.0), dict(x=None), dict(t=None), dict(lse=None),
                dict(g=None), dict(o=None), dict(h=None), dict(x=A + 1), dict(o=G + 1), dict(g=D + 2), dict(gh=F + 2),
                dict(o=A + 2), dict(o=A, lo=100), dict(o=C - 100), dict(o=B - 2000)):
        assert call(**bad) == tr.SF_EINVAL, bad


def test_policy_refusals(tr, lib):
    nan, inf = float("nan"), float("inf")

    def call(**k):
        a = dict(dict(lp=A, old=B, ref=C, adv=D, per=0, mask=E, start=F, N=100000, B=10, red=0, sc=1.0, lo=0.2, hi=0.2,
                      kl=0.1, terms=G, grad=G + (1 << 30), ws=W, wb=1 << 30), **k)
        return lib.sf_policy_loss(a["lp"], a["old"], a["ref"], a["adv"], a["per"], a["mask"], a["start"], a["N"], a["B"],
                                  a["red"], a["sc"], a["lo"], a["hi"], a["kl"], a["terms"], a["grad"], a["ws"], a["wb"],
                                  None)

    need = lib.sf_policy_loss_workspace(100000, 10)
    assert need > 0
    for bad in (dict(N=-1), dict(B=-1), dict(N=1 << 34), dict(B=1 << 31), dict(red=-1), dict(red=3), dict(sc=nan),
                dict(sc=inf), dict(lo=1.0), dict(lo=-0.1), dict(lo=nan), dict(hi=-0.1), dict(hi=inf), dict(kl=nan),
                dict(lp=None), dict(old=None), dict(adv=None), dict(start=None), dict(terms=None), dict(grad=None),
                dict(ws=None), dict(wb=need - 1), dict(ws=W + 8), dict(lp=A + 2), dict(start=F + 4), dict(terms=G + 2),
                dict(grad=A), dict(grad=G + 8), dict(N=20, terms=A + 40, ws=None), dict(terms=D), dict(ws=F), dict(ws=E), dict(grad=C + 400)):
        assert call(**bad) == tr.SF_EINVAL, bad
    assert lib.sf_policy_loss_workspace(-1, 0) == -1 and lib.sf_policy_loss_workspace(0, 0) == 0


def make_list(lib, items):
    n = len(items)
    size = lib.sf_grad_list_bytes(n)
    buf = (ctypes.c_int64 * (size // 8 + 1))()
    rc = lib.sf_grad_list_init(buf, size, (ctypes.c_void_p * n)(*(i[0] for i in items)),
                               (ctypes.c_int64 * n)(*(i[1] for i in items)), (ctypes.c_int32 * n)(*(i[2] for i in items)),
                               n)
    return rc, buf


def test_grad_list_refusals(tr, lib):
    assert lib.sf_grad_list_bytes(-1) == -1 and lib.sf_grad_list_bytes((1 << 20) + 1) == -1
    assert make_list(lib, [])[0] == tr.SF_OK
    assert make_list(lib, [(A, 10, 0), (None, 0, 1), (B, 7, 2)])[0] == tr.SF_OK
    for bad in ((A, -1, 0), (A, 1 << 40, 0), (A, 10, 3), (A, 10, -1), (None, 1, 0), (A + 2, 1, 0), (A + 1, 1, 1)):
        assert make_list(lib, [(C, 4, 0), bad])[0] == tr.SF_EINVAL, bad
    size = lib.sf_grad_list_bytes(1)
    buf = (ctypes.c_int64 * (size // 8 + 1))()
    arrays = ((ctypes.c_void_p * 1)(A), (ctypes.c_int64 * 1)(5), (ctypes.c_int32 * 1)(0))
    assert lib.sf_grad_list_init(buf, size - 1, *arrays, 1) == tr.SF_EINVAL
    assert lib.sf_grad_list_init(None, size, *arrays, 1) == tr.SF_EINVAL
    assert lib.sf_grad_list_init(buf, size, None, None, None, 1) == tr.SF_EINVAL
    assert lib.sf_grad_list_init(ctypes.addressof(buf) + 4, size, *arrays, 1) == tr.SF_EINVAL


def test_grad_norm_refusals(tr, lib):
    rc, l = make_list(lib, [(A, 1000, 0), (B, 33, 1)])
    assert rc == tr.SF_OK
    need = lib.sf_grad_norm_workspace(l)
    assert need > 0 and lib.sf_grad_norm_workspace(None) == -1
    assert lib.sf_grad_norm_workspace((ctypes.c_int64 * 64)()) == -1  # not a list

    def call(**k):
        a = dict(dict(l=l, n=C, t=D, f=E, ws=W, wb=need), **k)
        return lib.sf_grad_norm(a["l"], a["n"], a["t"], a["f"], a["ws"], a["wb"], None)

    for bad in (dict(l=None), dict(l=(ctypes.c_int64 * 64)()), dict(n=None), dict(t=None), dict(f=None), dict(ws=None),
                dict(wb=need - 1), dict(n=C + 2), dict(t=D + 1), dict(f=E + 4), dict(ws=W + 8), dict(n=A + 8),
                dict(t=B + 32), dict(ws=A - 16), dict(n=D), dict(f=W)):
        assert call(**bad) == tr.SF_EINVAL, bad


def test_grad_clip_refusals(tr, lib):
    items = [(A, 1000, 0), (B, 33, 1), (None, 0, 0)]
    l = make_list(lib, items)[1]
    other = make_list(lib, [(E, 1000, 0), (F, 33, 1), (None, 0, 2)])[1]  # another type of an empty tensor

    def call(**k):
        a = dict(dict(l=l, o=l, n=C, m=8, mx=1.0, eps=1e-6, st=D), **k)
        return lib.sf_grad_clip(a["l"], a["o"], a["n"], a["m"], a["mx"], a["eps"], a["st"], None)

    def out(*its):
        rc, b = make_list(lib, list(its))
        assert rc == tr.SF_OK
        return b

    empty = (None, 0, 0)
    for bad in (dict(l=None), dict(o=None), dict(n=None), dict(m=0), dict(m=65537), dict(mx=0.0), dict(mx=float("inf")),
                dict(mx=float("nan")), dict(eps=-1.0), dict(eps=float("nan")), dict(n=C + 2), dict(st=D + 2),
                dict(n=A), dict(st=B), dict(st=C + 4), dict(o=other),
                dict(o=out((E, 1000, 0), (F, 33, 1))),                    # another count of tensors
                dict(o=out((E, 999, 0), (F, 33, 1), empty)),              # another size
                dict(o=out((E, 1000, 0), (F, 33, 2), empty)),             # another type
                dict(o=out((E, 1000, 0), (E + 8, 33, 1), empty)),         # outputs that overlap
                dict(o=out((A + 4, 1000, 0), (F, 33, 1), empty)),         # a shifted gradient
                dict(o=out((A - 3996, 1000, 0), (F, 33, 1), empty)),
                dict(o=out((E, 1000, 0), (A + 40, 33, 1), empty))):       # inside another gradient
        assert call(**bad) == tr.SF_EINVAL, bad
    # a gradient listed twice, kept in place by one of its two outputs
    twice = out((A, 10, 0), (A, 10, 0))
    assert call(l=twice, o=out((A, 10, 0), (E, 10, 0))) == tr.SF_EINVAL
    assert call(l=twice, o=twice) == tr.SF_EINVAL
    assert lib.sf_grad_clip(make_list(lib, [])[1], make_list(lib, [])[1], C, 1, 1.0, 0.0, None, None) == tr.SF_OK
