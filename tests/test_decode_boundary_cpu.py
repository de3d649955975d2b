"""Host-side checks of the operators of albireo_decode.h that need no GPU: the library exports what the header
declares, and argument errors come back as status codes (or ValueError from the binding) before any launch."""
from __future__ import annotations

import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def alb():
    if not os.path.exists(os.path.join(ROOT, "paper_2606_01927_amd", "libalbireo.so")):
        pytest.skip("library not built")
    import paper_2606_01927_amd

    return paper_2606_01927_amd


def test_header_and_exports(alb):
    text = open(os.path.join(ROOT, "include", "albireo_decode.h")).read()
    names = re.findall(r"^\s*albireo_status_t\s+(albireo_\w+)\s*\(", text, re.M)
    assert sorted(names) == sorted(alb.DECODE_EXPORTED)
    lib = ctypes.CDLL(alb.LIB_PATH)
    assert all(hasattr(lib, n) for n in names)
    assert "ALBIREO_MAX_NORM_WIDTH %d" % alb.MAX_NORM_WIDTH in text


def test_norm_validates(alb):
    f = alb.raw_call("albireo_rms_norm")
    base = dict(x=0x10000, dtype=alb.BF16, T=4, D=64, ldx=64, res=None, ldr=0, w=0x20000, wd=alb.F32, eps=1e-6, ro=None,
                ldro=0, out=0x30000, ldo=64, q=None, ldq=0, s=None, stream=None)

    def call(**kw):
        return f(*{**base, **kw}.values())

    E, U = alb.E_INVALID, alb.E_UNSUPPORTED
    assert call(T=0) == alb.OK
    for bad in (dict(dtype=2), dict(wd=5), dict(T=-1), dict(D=0), dict(ldx=63), dict(eps=0.0), dict(eps=-1.0),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(res=0x40000, ldr=63), dict(ro=0x40000, ldro=1),
                dict(ldo=63), dict(q=0x50000, ldq=64), dict(s=0x50000), dict(q=0x50000, s=0x60000, ldq=63),
                dict(x=0x10001), dict(w=0x20002), dict(out=0x30001), dict(x=None), dict(out=None),
                dict(out=0x10000, ldo=72), dict(ro=0x30000, ldro=64), dict(s=0x50002, q=0x50000, ldq=64)):
        assert call(**bad) == E, bad
    assert call(D=alb.MAX_NORM_WIDTH + 1, ldx=1 << 20, ldo=1 << 20) == U
    assert call(T=1 << 31) == U


def test_matmul_validates(alb):
    from paper_2606_01927_amd.decode import ROWS_BF16, ROWS_I8, _W4

    f = alb.raw_call("albireo_matmul_w4")
    wbase = dict(N=100, K=256, group=128, q=0x10000, ldq=128, scales=0x20000, scale_dtype=alb.BF16, lds=2, zeros=None, ldz=0)
    base = dict(x=0x30000, xt=ROWS_BF16, B=4, ldx=256, xs=None, w=True, out=0x40000, od=alb.F32, ldo=100, stream=None)

    def call(w=None, **kw):
        a = {**base, **kw}
        if w is not None or a["w"] is True:
            a["w"] = ctypes.pointer(_W4(**{**wbase, **(w or {})}))
        return f(*a.values())

    E, U = alb.E_INVALID, alb.E_UNSUPPORTED
    assert call(B=0) == alb.OK
    assert call(w=dict(N=0)) == alb.OK
    a = {**base, "w": None}
    assert f(*a.values()) == E
    for bad in (dict(xt=0), dict(xt=3), dict(od=2), dict(B=-1), dict(ldx=255), dict(ldo=99), dict(xs=0x50000),
                dict(xt=ROWS_I8), dict(x=None), dict(out=None), dict(x=0x30001), dict(out=0x40002),
                dict(xt=ROWS_I8, xs=0x50001)):
        assert call(**bad) == E, bad
    for bad in (dict(scale_dtype=7), dict(group=16), dict(group=0), dict(group=256), dict(K=200), dict(K=0), dict(N=-1),
                dict(ldq=127), dict(lds=1), dict(zeros=0x60000, ldz=1), dict(q=None), dict(scales=None),
                dict(scales=0x20001)):
        assert call(w=bad) == E, bad
    assert call(w=dict(N=1 << 31), ldo=1 << 31) == U
    assert call(w=dict(K=1 << 25, ldq=1 << 24, lds=1 << 18), ldx=1 << 25) == U


def test_adjust_validates(alb):
    from paper_2606_01927_amd.decode import _Constraints

    f = alb.raw_call("albireo_adjust_logits")
    base = dict(x=0x10000, dtype=alb.BF16, B=4, V=100, ld=100, p=None, c=None, out=0x20000, od=alb.F32, ldo=100, fl=None,
                stream=None)

    def call(c=None, **kw):
        a = {**base, **kw}
        if c is not None:
            a["c"] = ctypes.pointer(_Constraints(**c))
        return f(*a.values())

    E = alb.E_INVALID
    assert call(B=0) == alb.OK
    for bad in (dict(dtype=3), dict(od=9), dict(B=-1), dict(V=0), dict(ld=99), dict(ldo=99), dict(x=None), dict(out=None),
                dict(x=0x10001), dict(out=0x20002), dict(fl=0x30001), dict(out=0x10000), dict(out=0x10000, od=alb.BF16, ldo=104)):
        assert call(**bad) == E, bad
    bias = dict(bias_offsets=0x30000, bias_ids=0x40000, bias_values=0x50000, bias_len=5)
    mask = dict(mask=0x60000, mask_rows=4, mask_ld=4)
    for bad in ({**bias, "bias_len": -1}, {**bias, "bias_ids": None}, {**bias, "bias_values": None},
                {**mask, "mask_rows": 3}, {**mask, "mask_ld": 3}, {**mask, "mask_rows": -1}, {**mask, "mask": 0x60002}):
        assert call(c=bad) == E, bad
    assert call(B=1 << 20) == alb.E_UNSUPPORTED
    p = alb.Params()
    p.hist_offsets, p.hist_len = 0x5000, 10
    assert call(p=ctypes.pointer(p)) == E


def test_binding_refuses(alb):
    import torch

    x = torch.zeros((4, 64))
    for bad in (lambda: alb.PreparedNorm(x.double()), lambda: alb.PreparedNorm(x[0]), lambda: alb.PreparedNorm(x.t()),
                lambda: alb.PreparedNorm(x, torch.zeros(63)), lambda: alb.PreparedNorm(x, residual=torch.zeros((4, 63))),
                lambda: alb.PreparedNorm(x, residual=x.bfloat16()), lambda: alb.PreparedNorm(x, quant=True, out=alb.NormOut(y=x)),
                lambda: alb.PreparedNorm(x, out=alb.NormOut())):
        with pytest.raises(ValueError):
            bad()
    q, s = torch.zeros((10, 64), dtype=torch.uint8), torch.zeros((10, 1))
    w = alb.W4Weight(q, s)
    assert (w.N, w.K, w.group) == (10, 128, 128)
    for bad in (lambda: alb.W4Weight(q, torch.zeros((10, 3))), lambda: alb.W4Weight(q, torch.zeros((9, 1))),
                lambda: alb.W4Weight(q.int(), s), lambda: alb.W4Weight(q, s.double()), lambda: alb.W4Weight(q, torch.zeros((10, 8))),
                lambda: alb.W4Weight(q, s, zeros=s)):
        with pytest.raises(ValueError):
            bad()
    xb = torch.zeros((3, 128), dtype=torch.bfloat16)
    for bad in (lambda: alb.PreparedMatmulW4(xb.float(), w), lambda: alb.PreparedMatmulW4(xb[:, :64], w),
                lambda: alb.PreparedMatmulW4(xb, w, x_scale=torch.ones(3)), lambda: alb.PreparedMatmulW4(xb.char(), w),
                lambda: alb.PreparedMatmulW4(xb, w, out=torch.zeros((3, 11))),
                lambda: alb.PreparedMatmulW4(xb, w, out=torch.zeros((3, 10)).double())):
        with pytest.raises(ValueError):
            bad()
    y = torch.zeros((2, 100))
    C = alb.Constraints
    i32 = torch.zeros(3, dtype=torch.int32)
    for bad in (lambda: alb.PreparedAdjust(y.half()), lambda: alb.PreparedAdjust(y, out=torch.zeros((2, 99))),
                lambda: alb.PreparedAdjust(y, constraints=C(mask=torch.zeros((2, 3), dtype=torch.int32))),
                lambda: alb.PreparedAdjust(y, constraints=C(mask=torch.zeros((1, 4), dtype=torch.int32))),
                lambda: alb.PreparedAdjust(y, constraints=C(mask=torch.zeros((2, 4)))),
                lambda: alb.PreparedAdjust(y, constraints=C(bias_offsets=torch.zeros(3, dtype=torch.int64))),
                lambda: alb.PreparedAdjust(y, constraints=C(bias_offsets=torch.zeros(3, dtype=torch.int64), bias_ids=i32,
                                                            bias_values=torch.zeros(2))),
                lambda: alb.PreparedAdjust(y, constraints=C(bias_offsets=torch.zeros(2, dtype=torch.int64), bias_ids=i32,
                                                            bias_values=torch.zeros(3)))):
        with pytest.raises(ValueError):
            bad()
