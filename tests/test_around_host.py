"""Host checks of the operators around the split layer that need no GPU: what they refuse, before any HIP call."""
import array
import ctypes
import os
import re

import numpy as np
import pytest

from tests import mx_formats as mx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000          # fake, 16-byte aligned "device" addresses: validation never dereferences them


@pytest.fixture(scope="module")
def ws():
    from paper_2011_09208_amd import buildlib
    if buildlib.is_stale():
        buildlib.build()
    from paper_2011_09208_amd import binding
    return binding


@pytest.fixture(scope="module")
def E(ws):
    return {ws.status_string(i)[7:] or "OK": i for i in range(8)}


def test_limits_are_the_headers(ws):
    text = open(os.path.join(ROOT, "include", "whalesplit.h")).read()
    assert int(re.search(r"#define\s+WS_RMS_NORM_MAX_D\s+(\d+)", text).group(1)) == ws.RMS_NORM_MAX_D
    power, less = re.search(r"#define\s+WS_W4_MAX_CLASSES\s+\(\(1 << (\d+)\) - (\d+)\)", text).groups()
    assert (1 << int(power)) - int(less) == ws.W4_MAX_CLASSES


def test_norm_refusals(ws, E):
    def fwd(x=A, ldx=64, r=A, ldr=64, es=4, gamma=A, eps=1e-6, B=4, D=64, h=A, ldh=64, y=A, ldy=64, rstd=A):
        return ws.lib.ws_rms_norm_fwd(x, ldx, r, ldr, es, gamma, eps, B, D, h, ldh, y, ldy, rstd, None)

    def mx8(x=A, ldx=64, r=None, ldr=0, es=2, gamma=A, eps=1e-6, B=4, D=64, h=None, ldh=0, y=A, ldy=64, s=A, lds=2, rstd=None):
        return ws.lib.ws_rms_norm_fwd_mx8(x, ldx, r, ldr, es, gamma, eps, B, D, h, ldh, y, ldy, s, lds, rstd, None)

    for f in (fwd, mx8):
        assert f(x=None) == E["NULL"] and f(gamma=None) == E["NULL"] and f(y=None) == E["NULL"]
        assert f(B=0) == E["SHAPE"] and f(D=96) == E["SHAPE"] and f(D=0) == E["SHAPE"] and f(es=3) == E["SHAPE"]
        assert f(D=16448, ldx=16448, ldr=16448, ldh=16448, ldy=16448) == E["SHAPE"]               # more than a row may have
        assert f(ldx=56) == E["SHAPE"] and f(r=A, ldr=56) == E["SHAPE"] and f(h=A, ldh=0) == E["SHAPE"] and f(ldy=48) == E["SHAPE"]
        assert f(eps=0.0) == E["RANGE"] and f(eps=-1.0) == E["RANGE"] and f(eps=float("nan")) == E["RANGE"] and f(eps=float("inf")) == E["RANGE"]
        assert f(x=A + 8) == E["ALIGN"] and f(ldx=68) == E["ALIGN"] and f(gamma=A + 4) == E["ALIGN"] and f(y=A + 8) == E["ALIGN"]
        assert f(r=A + 8, ldr=64) == E["ALIGN"] and f(h=A + 4, ldh=64) == E["ALIGN"] and f(rstd=A + 2) == E["ALIGN"] and f(ldy=68) == E["ALIGN"]
    assert fwd(ldr=66) == E["ALIGN"] and fwd(ldh=66) == E["ALIGN"] and fwd(es=2, ldr=68) == E["ALIGN"]
    assert mx8(s=None) == E["NULL"] and mx8(lds=1) == E["SHAPE"] and mx8(s=A + 1) == E["ALIGN"] and mx8(lds=3) == E["ALIGN"]


def test_norm_back_refusals(ws, E):
    def bwd(dY=A, lddy=64, h=A, ldh=64, d=A, ldd=64, es=4, gamma=A, rstd=A, B=4, D=64, dh=A, lddh=64, dg=A, wsp=A, wsb=1 << 20):
        return ws.lib.ws_rms_norm_bwd(dY, lddy, h, ldh, d, ldd, es, gamma, rstd, B, D, dh, lddh, dg, wsp, wsb, None)

    for k in ("dY", "h", "gamma", "rstd", "dh"):
        assert bwd(**{k: None}) == E["NULL"]
    assert bwd(B=0) == E["SHAPE"] and bwd(D=72) == E["SHAPE"] and bwd(es=8) == E["SHAPE"] and bwd(D=16448) == E["SHAPE"]
    for k in ("lddy", "ldh", "ldd", "lddh"):
        assert bwd(**{k: 60}) == E["SHAPE"] and bwd(**{k: 66}) == E["ALIGN"]
    assert bwd(es=2, ldh=68) == E["ALIGN"] and bwd(dY=A + 4) == E["ALIGN"] and bwd(h=A + 8) == E["ALIGN"] and bwd(d=A + 8) == E["ALIGN"]
    assert bwd(dg=A + 2) == E["ALIGN"] and bwd(rstd=A + 1) == E["ALIGN"] and bwd(wsp=A + 8) == E["ALIGN"]
    assert bwd(wsp=None) == E["WORKSPACE"] and bwd(wsb=16) == E["WORKSPACE"]
    assert ws.rms_norm_bwd_workspace_bytes(0, 64) == 0 and ws.rms_norm_bwd_workspace_bytes(4, 65) == 0 and ws.rms_norm_bwd_workspace_bytes(4, 16448) == 0
    assert ws.rms_norm_bwd_workspace_bytes(100000, 16384) <= 64 << 20


def test_packing_and_w4_refusals(ws, E):
    def pack(W=A, ldw=64, C=8, D=64, W4=A, ldw4=32, s=A, lds=2):
        return ws.lib.ws_quantize_mx4(W, ldw, C, D, W4, ldw4, s, lds, None)

    assert pack(W=None) == E["NULL"] and pack(W4=None) == E["NULL"] and pack(s=None) == E["NULL"]
    assert pack(C=0) == E["SHAPE"] and pack(D=32) == E["SHAPE"] and pack(ldw=56) == E["SHAPE"] and pack(ldw4=16) == E["SHAPE"] and pack(lds=1) == E["SHAPE"]
    assert pack(W=A + 8) == E["ALIGN"] and pack(ldw=68) == E["ALIGN"] and pack(W4=A + 4) == E["ALIGN"] and pack(ldw4=40) == E["ALIGN"]
    assert pack(s=A + 1) == E["ALIGN"] and pack(lds=3) == E["ALIGN"]

    def logits(X=A, ldx=64, xs=None, ldxs=0, W4=A, ldw4=32, s=A, lds=2, b=None, B=4, D=64, C=8, Z=A, ldz=8):
        return ws.lib.ws_split_fc_w4_logits(X, ldx, xs, ldxs, W4, ldw4, s, lds, b, B, D, C, Z, ldz, None)

    def top1(X=A, ldx=64, xs=None, ldxs=0, W4=A, ldw4=32, s=A, lds=2, b=None, B=4, D=64, C=8, off=0, v=A, c=A, wsp=A, wsb=1 << 20):
        return ws.lib.ws_split_fc_w4_top1(X, ldx, xs, ldxs, W4, ldw4, s, lds, b, B, D, C, off, v, c, wsp, wsb, None)

    for f in (logits, top1):
        assert f(X=None) == E["NULL"] and f(W4=None) == E["NULL"] and f(s=None) == E["NULL"]
        assert f(B=0) == E["SHAPE"] and f(D=96) == E["SHAPE"] and f(C=0) == E["SHAPE"] and f(B=(1 << 20) + 1) == E["SHAPE"]
        assert f(ldx=56) == E["SHAPE"] and f(ldw4=16) == E["SHAPE"] and f(lds=1) == E["SHAPE"] and f(xs=A, ldxs=1) == E["SHAPE"]
        assert f(X=A + 8) == E["ALIGN"] and f(ldx=68) == E["ALIGN"] and f(W4=A + 8) == E["ALIGN"] and f(ldw4=36) == E["ALIGN"]
        assert f(xs=A, ldxs=2, ldx=72) == E["ALIGN"] and f(xs=A + 1, ldxs=2) == E["ALIGN"] and f(xs=A, ldxs=3) == E["ALIGN"]
        assert f(s=A + 1) == E["ALIGN"] and f(lds=3) == E["ALIGN"] and f(b=A + 2) == E["ALIGN"]
        assert f(C=2**31 - 1) == E["RANGE"] and f(C=(1 << 30) - 65535) == E["RANGE"]
        assert f(ldw4=(1 << 26) + 16) == E["SHAPE"] and f(lds=(1 << 26) + 2) == E["SHAPE"]
    assert logits(Z=None) == E["NULL"] and logits(ldz=4) == E["SHAPE"] and logits(ldz=9) == E["ALIGN"] and logits(Z=A + 4) == E["ALIGN"]
    assert top1(v=None) == E["NULL"] and top1(c=None) == E["NULL"] and top1(v=A + 1) == E["ALIGN"] and top1(off=-1) == E["RANGE"]
    assert top1(off=2**31 - 4) == E["RANGE"] and top1(wsp=None) == E["WORKSPACE"] and top1(wsb=8) == E["WORKSPACE"] and top1(wsp=A + 8) == E["ALIGN"]
    assert ws.w4_top1_workspace_bytes(0, 8) == 0 and ws.w4_top1_workspace_bytes(4, 0) == 0
    assert ws.w4_top1_workspace_bytes(256, 10**8) <= 64 << 20


def _ptr(values, code="q"):
    a = array.array(code, values)
    return a.buffer_info()[0], a


def test_gradient_refusals(ws, E):
    def tables(data=(A, A), rows=(1, 4), cols=(8, 8), lds=(8, 8), es=(2, 4)):
        return [_ptr(data), _ptr(rows), _ptr(cols), _ptr(lds), _ptr(es, "i")]

    def sumsq(out=A, wsp=A, wsb=1 << 20, n=2, null=None, **kw):
        t = tables(**kw)
        p = [None if i == null else v[0] for i, v in enumerate(t)]
        return ws.lib.ws_grad_sumsq(*p, n, out, wsp, wsb, None)

    def clip(ss=A, S=1, limit=1.0, norm=None, n=2, **kw):
        t = tables(**kw)
        return ws.lib.ws_grad_clip(*[v[0] for v in t], n, ss, S, limit, norm, None)

    def sgd(ss=A, S=1, limit=1.0, lr=0.1, norm=None, n=2, pdata=(A, A), ldp=(8, 8), pes=(2, 2), pnull=False, **kw):
        t, (pd, _1), (pl, _2), (pb, _3) = tables(**kw), _ptr(pdata), _ptr(ldp), _ptr(pes, "i")
        return ws.lib.ws_grad_clip_sgd(None if pnull else pd, pl, pb, *[v[0] for v in t], n, ss, S, limit, lr, norm, None)

    for f in (sumsq, clip, sgd):
        assert f(data=(A, 0)) == E["NULL"] and f(n=-1) == E["RANGE"]
        assert f(rows=(1, -1)) == E["SHAPE"] and f(cols=(-8, 8)) == E["SHAPE"] and f(es=(2, 8)) == E["SHAPE"] and f(lds=(8, 4)) == E["SHAPE"]
        assert f(rows=(1, 2**31)) == E["SHAPE"] and f(cols=(2**43, 8)) == E["RANGE"]
        assert f(data=(A + 1, A)) == E["ALIGN"] and f(data=(A, A + 2)) == E["ALIGN"]
    assert sumsq(out=None) == E["NULL"] and sumsq(out=A + 4) == E["ALIGN"] and all(sumsq(null=i) == E["NULL"] for i in range(5))
    assert sumsq(wsp=None) == E["WORKSPACE"] and sumsq(wsb=8) == E["WORKSPACE"] and sumsq(wsp=A + 8) == E["ALIGN"]
    for f in (clip, sgd):
        assert f(ss=None) == E["NULL"] and f(ss=A + 4) == E["ALIGN"] and f(norm=A + 2) == E["ALIGN"]
        assert f(S=0) == E["RANGE"] and f(S=65) == E["RANGE"] and f(limit=0.0) == E["RANGE"] and f(limit=-1.0) == E["RANGE"] and f(limit=float("nan")) == E["RANGE"]
    assert sgd(lr=float("nan")) == E["RANGE"] and sgd(lr=float("inf")) == E["RANGE"] and sgd(pnull=True) == E["NULL"] and sgd(pdata=(A, 0)) == E["NULL"]
    assert sgd(ldp=(8, 4)) == E["SHAPE"] and sgd(pes=(2, 1)) == E["SHAPE"] and sgd(pdata=(A, A + 1)) == E["ALIGN"]
    assert ws.grad_workspace_bytes(-1) == 0 and ws.grad_workspace_bytes(100) > ws.grad_workspace_bytes(0) > 0


def test_binding_refuses_tensors_that_are_not_what_a_call_takes(ws):
    """Tensors of the host, of another type, shape or order: refused before a pointer is passed on."""
    import torch
    x, g = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros(64)
    with pytest.raises(AssertionError):
        ws.rms_norm_fwd(x, None, g, 1e-6, None, x.clone(), None)
    with pytest.raises(AssertionError):
        ws.quantize_mx4(x, torch.zeros((4, 32), dtype=torch.uint8), torch.zeros((4, 2), dtype=torch.uint8))
    with pytest.raises(AssertionError):
        ws.grad_sumsq([g], torch.zeros(1, dtype=torch.float64), torch.zeros(1 << 20, dtype=torch.uint8))
    with pytest.raises(AssertionError):
        ws.grad_table([torch.zeros((4, 64)).t()])
    with pytest.raises(KeyError):
        ws.grad_table([torch.zeros(4, dtype=torch.float16, device="meta")])


def test_formats_of_the_oracle():
    """The tests' own forms of the 8- and 4-bit formats: known values, and every value comes back from packing."""
    import torch
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(mx.E4M3, t, equal_nan=True)
    assert np.array_equal(mx.scale_bytes(np.array([0.0, 6.0, 6.0001, 448.0, np.inf, np.nan, 2.0 ** -140]), 6.0), [0, 127, 128, 134, 255, 255, 0])
    codes = np.arange(256, dtype=np.uint8).reshape(16, 16)
    codes[:, 0] = (codes[:, 0] & 0x88) | 0x77                      # a 6 in every group: the scale comes back, too
    scales = np.arange(100, 116, dtype=np.uint8).reshape(16, 1)
    c, s = mx.quantize4(mx.values4(codes, scales))
    assert np.array_equal(c, codes) and np.array_equal(s, scales)


def test_a_library_with_these_entry_points_has_a_version_of_its_own(ws):
    assert ws.version() >= 1221                            # 1220 was without them
