"""Argument checks of the gated delta rule and of the norms between two blocks, without a GPU: everything that is refused is refused
before anything is launched."""
import ctypes

import pytest
import torch

import __graft_entry__ as entry
from paper_2307_14995_b200 import binding as la

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def lib():
    entry.build()
    return la.load()


def delta(**kw):
    base = dict(B=1, H=4, N=200, d=64, e=64, in_dtype=F32, out_dtype=F32, Hk=2)
    base.update(kw)
    return la.make_delta_shape(**base)


def norm(**kw):
    base = dict(rows=10, D=64, dtype=BF16, res_dtype=F32, eps=1e-6)
    base.update(kw)
    return la.make_block_norm_shape(**base)


PLENTY = 1 << 40


def fwd(lib, s, ws=4096, size=PLENTY, **bad):
    a = dict(q=256, k=256, v=256, g=256, beta=256, o=256, kv_in=None, kv_out=None)
    a.update(bad)
    return lib.la_delta_fwd(ctypes.byref(s), *a.values(), ws, size, None)


def bwd(lib, s, ws=1 << 41, size=PLENTY, fws=None, **bad):
    a = dict(q=256, k=256, v=256, g=256, beta=256, do=256, dq=256, dk=256, dv=256, dg=256, dbeta=256, kv_in=None, out=None, gin=None)
    a.update(bad)
    return lib.la_delta_bwd(ctypes.byref(s), *a.values(), fws, ws, size, None)


def steps(lib, s, **bad):
    a = dict(q=256, k=256, v=256, g=256, beta=256, kv=256, o=256)
    a.update(bad)
    return lib.la_delta_steps(ctypes.byref(s), *a.values(), None)


@pytest.mark.parametrize("bad,status", [
    (dict(N=0), INVALID), (dict(N=-1), INVALID), (dict(B=0), INVALID), (dict(H=0), INVALID), (dict(Hk=0), INVALID), (dict(Hk=3), INVALID),
    (dict(Hk=8), INVALID), (dict(d=48, e=48), UNSUPPORTED), (dict(e=128), UNSUPPORTED), (dict(out_dtype=BF16), UNSUPPORTED),
    (dict(B=65536), UNSUPPORTED), (dict(N=1 << 30), UNSUPPORTED), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(path=3), INVALID), (dict(layout=2), INVALID), (dict(path=la.LA_PATH_TENSOR), UNSUPPORTED)])
def test_shapes_that_are_refused(lib, bad, status):
    s = delta(**bad)
    assert fwd(lib, s) == status and bwd(lib, s) == status
    if "path" not in bad or bad["path"] == 3:
        assert steps(lib, s) == status
    assert lib.la_delta_workspace_bytes(la.LA_OP_FWD, ctypes.byref(s)) == ctypes.c_size_t(-1).value


@pytest.mark.parametrize("call", [fwd, bwd, steps])
def test_pointers_that_are_refused(lib, call):
    s = delta()
    for name in ("q", "k", "v", "g", "beta"):
        assert call(lib, s, **{name: None}) == INVALID
        assert call(lib, s, **{name: 264}) == INVALID  # not 16-byte aligned
    if call is fwd:
        assert call(lib, s, o=None) == INVALID and call(lib, s, kv_in=8) == INVALID
    elif call is bwd:
        for name in ("do", "dq", "dk", "dv", "dg", "dbeta"):
            assert call(lib, s, **{name: None}) == INVALID
        assert call(lib, s, gin=8) == INVALID
    else:
        assert call(lib, s, kv=None) == INVALID and call(lib, s, o=None) == INVALID


def test_workspaces_that_are_refused(lib):
    s = delta()
    one, both = la.delta_workspace_bytes(la.LA_OP_FWD, s), la.delta_workspace_bytes(la.LA_OP_BWD, s)
    assert one > 0 and both > one and la.delta_workspace_bytes(la.LA_OP_DECODE, s) == 0
    assert fwd(lib, s, ws=None) == WORKSPACE and fwd(lib, s, size=one - 1) == WORKSPACE and fwd(lib, s, ws=4096 + 16) == INVALID
    assert bwd(lib, s, ws=None) == WORKSPACE and bwd(lib, s, size=both - 1) == WORKSPACE
    assert bwd(lib, s, fws=4096, size=both - one - 1) == WORKSPACE
    ws = 1 << 41
    for fws in (ws, ws + 256, ws - one + 256, ws + (both - one) - 256):  # one inside the other
        assert bwd(lib, s, ws=ws, size=both - one, fws=fws) == INVALID
    assert bwd(lib, s, ws=ws, size=both - one, fws=ws + 128) == INVALID
    assert la.delta_workspace_bytes(la.LA_OP_FWD, delta(N=64 * 1000)) == 250 * la.delta_workspace_bytes(la.LA_OP_FWD, delta(N=256))


def norm_fwd(lib, s, **bad):
    a = dict(x=256, y=256, u=256, w_post=256, s=256, w_pre=256, h=256, n=256)
    a.update(bad)
    return lib.la_block_norm_fwd(ctypes.byref(s), *a.values(), None)


def norm_bwd(lib, s, ws=4096, size=PLENTY, **bad):
    a = dict(x=256, y=256, u=256, w_post=256, s=256, w_pre=256, dh=256, dn=256, dx=256, dy=256, du=256, dwp=256, ds=256, dwn=256)
    a.update(bad)
    return lib.la_block_norm_bwd(ctypes.byref(s), *a.values(), ws, size, None)


@pytest.mark.parametrize("bad,status", [
    (dict(rows=0), INVALID), (dict(D=0), INVALID), (dict(D=16385), UNSUPPORTED), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(gate=3), INVALID), (dict(dtype=F32, res_dtype=BF16), UNSUPPORTED), (dict(rows=1 << 40, D=8192), UNSUPPORTED)])
def test_norm_shapes_that_are_refused(lib, bad, status):
    s = norm(**bad)
    assert norm_fwd(lib, s) == status and norm_bwd(lib, s) == status
    assert lib.la_block_norm_workspace_bytes(ctypes.byref(s)) == ctypes.c_size_t(-1).value


def test_norm_arguments_that_are_refused(lib):
    s = norm()
    for name in ("x", "y"):
        assert norm_fwd(lib, s, **{name: None}) == INVALID and norm_bwd(lib, s, **{name: None}) == INVALID
        assert norm_fwd(lib, s, **{name: 8}) == INVALID
    assert norm_fwd(lib, s, h=None, n=None) == INVALID
    assert norm_bwd(lib, s, dh=None, dn=None) == INVALID
    assert norm_bwd(lib, s, du=None) == INVALID and norm_bwd(lib, s, u=None) == INVALID
    assert norm_bwd(lib, s, dx=None) == INVALID and norm_bwd(lib, s, dy=None) == INVALID
    need = la.block_norm_workspace_bytes(s)
    assert norm_bwd(lib, s, ws=None) == WORKSPACE and norm_bwd(lib, s, size=need - 1) == WORKSPACE and norm_bwd(lib, s, ws=4096 + 64) == INVALID


@pytest.mark.skipif(torch.cuda.is_available(), reason="needs a host without a CUDA device")
def test_no_cpu_fallback_without_a_device(lib):
    assert fwd(lib, delta()) in (4, 5) and bwd(lib, delta()) in (4, 5) and steps(lib, delta()) in (4, 5)
    assert norm_fwd(lib, norm()) in (4, 5) and norm_bwd(lib, norm()) in (4, 5)


def test_argument_kinds_are_those_of_the_header(monkeypatch):
    import inspect
    import os
    import re
    header = open(os.path.join(os.path.dirname(la.LIB_PATH), "..", "include", "la.h")).read()
    header = re.sub(r"/\*.*?\*/|//[^\n]*", "", header, flags=re.S)
    got = []
    monkeypatch.setattr(la, "_enter", lambda name, kinds, *args: got.append((name, kinds, len(args))))
    for name in ("la_delta_fwd", "la_delta_bwd", "la_delta_steps", "la_block_norm_fwd", "la_block_norm_bwd"):
        args = re.search(r"la_status\s+%s\(([^;]*?)\);" % name, header, re.S).group(1)
        want = ""
        for a in (" ".join(x.split()) for x in args.split(",")):
            want += "d" if "la_delta_shape" in a else "n" if "la_block_norm_shape" in a else "r" if a == "void* stream" else "t" if "*" in a else "i"
        f = getattr(la, name)
        f(**{p: (delta() if "delta" in name else norm()) if p == "shape" else None for p in inspect.signature(f).parameters})
        kinds = "".join("t" if c in "QPVOGSXYFw" else c for c in got[-1][1])  # (tensors that are held to the shape)
        assert (got[-1][0], kinds, got[-1][2]) == (name, want, len(want))


@pytest.mark.parametrize("wrong", [la.make_shape(1, 1, 1, 64, 64, BF16, F32), 5, None])
def test_shapes_of_other_calls_are_refused(monkeypatch, wrong):
    monkeypatch.setattr(la, "_current_device", lambda: 0)
    with pytest.raises(TypeError):
        la.la_delta_steps(wrong, None, None, None, None, None, None, None)
    with pytest.raises(TypeError):
        la.la_block_norm_fwd(wrong, None, None)
    with pytest.raises(TypeError):
        la._enter("la_fwd", "sttthttttir", delta(), None, None, None, la._lam([1.0]), None, None, None, None, 0, None)


def test_tensors_that_do_not_match_are_refused(monkeypatch):
    """Types and sizes follow from the shape, argument by argument.  (Tensors on the CPU say that they are on device -1.)"""
    la.load()
    s = delta(N=3)
    q, v, g = torch.zeros(1, 2, 3, 64), torch.zeros(1, 4, 3, 64), torch.zeros(1, 4, 3)
    kv = torch.zeros(1, 4, 64, 64)
    for args, word in (((q.bfloat16(), q, v, g, g, kv, v), "argument 1 has to be torch.float32 with 384 elements"), ((q, v, v, g, g, kv, v), "argument 2 has to be torch.float32 with 384"),
                       ((q, q, q, g, g, kv, v), "argument 3 has to be torch.float32 with 768"), ((q, q, v, g.double(), g, kv, v), "argument 4 has to be torch.float32 with 12 "),
                       ((q, q, v, g, g, q, v), "argument 6 has to be torch.float32 with 16384"),
                       ((q, q, v, g, g, kv, q), "argument 7 has to be torch.float32 with 768"),
                       ((q.transpose(1, 2), q, v, g, g, kv, v), "argument 1 has to be contiguous"),
                       ((q, q, v, g, g, kv, v), "on the current CUDA device")):
        monkeypatch.setattr(la, "_current_device", lambda: 0 if "device" in word else -1)
        with pytest.raises(ValueError, match=word):
            la.la_delta_steps(s, *args)
    n, x, w = norm(rows=2), torch.zeros(2, 64), torch.zeros(64)
    y = x.bfloat16()
    monkeypatch.setattr(la, "_current_device", lambda: -1)
    for args, word in (((y, y, y, w, w, w, x, y), "argument 1 has to be torch.float32 with 128"), ((x, x, y, w, w, w, x, y), "argument 2 has to be torch.bfloat16"),
                       ((x, y, y, x, w, w, x, y), "argument 4 has to be torch.float32 with 64"), ((x, y, y, w, w, w, x, x), "argument 8 has to be torch.bfloat16")):
        with pytest.raises(ValueError, match=word):
            la.la_block_norm_fwd(n, *args)
