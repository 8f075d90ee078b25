"""GPU: the root-mean-square norm with the residual's addition and its way back, against the formulas in 64 bits."""
import numpy as np
import pytest

from tests import mx_formats as mx

pytestmark = pytest.mark.gpu
U = 2.0 ** -24                                            # half a step of fp32, relative
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}            # of the types that results are rounded to
# D: one piece per lane and an eighth to a whole wave, each number of pieces, a ragged last piece, a workgroup for a row, a large one, the largest
SIZES = [(1, 64), (3, 64), (5, 512), (2, 576), (7, 1024), (9, 1088), (4, 2048), (1, 2112), (3, 4096), (2, 4160), (3, 8192), (2, 8256), (2, 16384), (531, 320),
         (5, 128), (37, 192), (19, 256), (1000, 256)]


@pytest.fixture(scope="module")
def G():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU; there is no CPU fallback")
    from tests import gpu_harness
    return gpu_harness


def _inputs(B, D, stream, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if stream == "bf16" else torch.float32
    x = torch.randn((B, D), device="cuda", generator=g).to(torch.bfloat16)
    res = (3 * torch.randn((B, D), device="cuda", generator=g)).to(dt)
    gamma = 1 + 0.3 * torch.randn(D, device="cuda", generator=g)
    return x, res, gamma, dt


def _f64(t):
    return t.double().cpu().numpy()


def _check_y(y, want, half):
    """A sum of D squares, at most 32 in a row per lane and then a tree of 6 + 16, off by 56 half steps; half of that on rstd, and
    six roundings of its own: 40 half steps of fp32.  Then the rounding to the output's type."""
    assert np.all(np.abs(y - want) <= (half + 40 * U) * np.abs(want) + 1e-30)


@pytest.mark.parametrize("stream", ["bf16", "fp32"])
@pytest.mark.parametrize("B,D", SIZES)
def test_norm(G, B, D, stream):
    import torch
    from paper_2011_09208_amd import binding as ws
    print(f"[norm] B={B} D={D} {stream}", flush=True)
    x, res, gamma, dt = _inputs(B, D, stream, B + D)
    eps = 1e-5
    for residual in (None, res):
        h = G.Guarded(B, D, dt, pad_cols=8)
        y, rstd = G.Guarded(B, D, torch.bfloat16, pad_cols=16), G.Guarded(1, B, torch.float32)
        ws.rms_norm_fwd(x, residual, gamma, eps, h.t, y.t, rstd.vec())
        torch.cuda.synchronize()
        assert h.intact_outside_payload() and y.intact_outside_payload() and rstd.intact_outside_payload()
        want_h = x.to(dt) if residual is None else (x.float() + res.float()).to(dt)
        assert torch.equal(h.t, want_h)                   # one fp32 addition, rounded once
        hd = _f64(want_h)
        want_r = 1 / np.sqrt((hd * hd).mean(1) + eps)
        assert np.all(np.abs(_f64(rstd.vec()) - want_r) <= 34 * U * want_r)
        _check_y(_f64(y.t), hd * want_r[:, None] * _f64(gamma), HALF["bf16"])
        # without h and rstd, and in place
        y2 = torch.empty_like(x)
        ws.rms_norm_fwd(x, residual, gamma, eps, None, y2, None)
        if residual is not None:
            assert torch.equal(y2, y.t)
            r2 = res.clone()
            y2.zero_()
            ws.rms_norm_fwd(x, r2, gamma, eps, r2, y2, None)
            assert torch.equal(r2, want_h)
        assert torch.equal(y2, y.t)


@pytest.mark.parametrize("stream", ["bf16", "fp32"])
@pytest.mark.parametrize("B,D", SIZES)
def test_norm_in_eight_bits(G, B, D, stream):
    import torch
    from paper_2011_09208_amd import binding as ws
    print(f"[norm mx8] B={B} D={D} {stream}", flush=True)
    x, res, gamma, dt = _inputs(B, D, stream, 3 * B + D)
    gamma[:: 37] = 0.0
    if D >= 128:
        gamma[64:128] = 0.0                               # two whole groups of zeros
    h = torch.empty((B, D), device="cuda", dtype=dt)
    y, s, rstd = G.Guarded(B, D, torch.uint8, pad_cols=16), G.Guarded(B, D // 32, torch.uint8, pad_cols=2), torch.empty(B, device="cuda")
    ws.rms_norm_fwd_mx8(x, res, gamma, 1e-6, h, y.t, s.t, rstd)
    torch.cuda.synchronize()
    assert y.intact_outside_payload() and s.intact_outside_payload()
    hd = _f64(h)
    want = hd / np.sqrt((hd * hd).mean(1, keepdims=True) + 1e-6) * _f64(gamma)
    q, sb = y.t.cpu().numpy(), s.t.cpu().numpy()
    sv = mx.scale_values(sb)
    top = np.abs(want).reshape(B, -1, 32).max(2)
    # the smallest power of two that holds the group, but for the 40 half steps that y is off
    assert np.all(top <= 448 * sv * (1 + 40 * U)) and np.all((top >= 224 * sv * (1 - 40 * U)) | (sb == 0))
    assert np.all(sb[top == 0] == 0)
    step = np.repeat(sv, 32, 1)
    # half a step: 2^-4 of the value, or 2^-10 of the scale below the smallest normal number
    assert np.all(np.abs(mx.values8(q, sb) - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * step) + 40 * U * np.abs(want))


def test_rows_with_infinities_and_nans(G):
    import torch
    from paper_2011_09208_amd import binding as ws
    B, D = 6, 192
    x, res, gamma, _ = _inputs(B, D, "fp32", 5)
    res[1, 7] = float("inf")
    res[2, 9] = float("nan")
    res[3] = 0.0
    x[3] = 0.0                                            # a row of zeros: y = 0, rstd = 1 / sqrt(eps)
    h, y, rstd = torch.empty_like(res), torch.empty_like(x), torch.empty(B, device="cuda")
    ws.rms_norm_fwd(x, res, gamma, 1e-6, h, y, rstd)
    q, s = torch.empty((B, D), device="cuda", dtype=torch.uint8), torch.empty((B, D // 32), device="cuda", dtype=torch.uint8)
    ws.rms_norm_fwd_mx8(x, res, gamma, 1e-6, None, q, s, None)
    y, q, s = y.float().cpu().numpy(), q.cpu().numpy(), s.cpu().numpy()
    assert np.isfinite(y[[0, 3, 4, 5]]).all() and np.all(y[3] == 0)
    assert abs(float(rstd[3]) - 1e3) <= 1e3 * 40 * U + 1e3 * 2e-8       # eps itself is rounded to fp32
    assert np.isnan(y[2]).all()
    assert np.isnan(y[1, 7]) and np.all(np.delete(y[1], 7) == 0)        # 1 / sqrt(inf) = 0
    assert np.all(s[2] == 255) and s[1, 0] == 255 and np.all(s[1, 1:] == 0) and np.all(q[3] == 0) and np.all(s[3] == 0)


@pytest.mark.parametrize("stream", ["bf16", "fp32"])
def test_more_rows_than_a_launch_takes(G, stream):
    """2^21 + 70 rows, 64 that come again and again: the result of a row does not depend on where it is."""
    import torch
    from paper_2011_09208_amd import binding as ws
    B, D = (1 << 21) + 70, 64
    x, res, gamma, dt = _inputs(64, D, stream, 12)
    many = lambda t: t.repeat(B // 64 + 1, *[1] * (t.dim() - 1))[:B].contiguous()        # noqa: E731
    h, y, rstd = torch.empty((64, D), device="cuda", dtype=dt), torch.empty_like(x), torch.empty(64, device="cuda")
    ws.rms_norm_fwd(x, res, gamma, 1e-6, h, y, rstd)
    H, Y, R = torch.empty((B, D), device="cuda", dtype=dt), torch.empty((B, D), device="cuda", dtype=torch.bfloat16), torch.empty(B, device="cuda")
    ws.rms_norm_fwd(many(x), many(res), gamma, 1e-6, H, Y, R)
    assert torch.equal(H, many(h)) and torch.equal(Y, many(y)) and torch.equal(R, many(rstd))
    q, s = torch.empty((64, D), device="cuda", dtype=torch.uint8), torch.empty((64, 2), device="cuda", dtype=torch.uint8)
    ws.rms_norm_fwd_mx8(x, res, gamma, 1e-6, None, q, s, None)
    Q, S = torch.empty((B, D), device="cuda", dtype=torch.uint8), torch.empty((B, 2), device="cuda", dtype=torch.uint8)
    ws.rms_norm_fwd_mx8(many(x), many(res), gamma, 1e-6, H, Q, S, R)
    assert torch.equal(Q, many(q)) and torch.equal(S, many(s)) and torch.equal(H, many(h)) and torch.equal(R, many(rstd))


def test_tensors_of_another_device_are_refused(G, monkeypatch):
    import torch
    from paper_2011_09208_amd import binding as ws
    x, res, gamma, _ = _inputs(4, 64, "bf16", 1)
    y, work = torch.empty_like(x), torch.empty(1 << 16, device="cuda", dtype=torch.uint8)
    sumsq = torch.empty(1, device="cuda", dtype=torch.float64)
    ws.rms_norm_fwd(x, res, gamma, 1e-6, None, y, None)
    ws.grad_sumsq([x, gamma], sumsq, work)
    torch.cuda.synchronize()
    table = ws.grad_table([x, gamma])
    monkeypatch.setattr(ws, "_device", lambda: 1)
    for call in (lambda: ws.rms_norm_fwd(x, res, gamma, 1e-6, None, y, None), lambda: ws.grad_table([x]), lambda: ws.grad_sumsq(table, sumsq, work),
                 lambda: ws.quantize_mx4(x, torch.empty((4, 32), device="cuda", dtype=torch.uint8), torch.empty((4, 2), device="cuda", dtype=torch.uint8)),
                 lambda: ws.grad_clip(table, sumsq, 1.0)):
        with pytest.raises(AssertionError):
            call()
    monkeypatch.undo()
    table.device = 1                                      # built while another device was the current one
    with pytest.raises(AssertionError):
        ws.grad_sumsq(table, sumsq, work)
    with pytest.raises(AssertionError):
        ws.grad_table([x, gamma.cpu()])


@pytest.mark.parametrize("stream", ["bf16", "fp32"])
@pytest.mark.parametrize("B,D", SIZES + [(4099, 64), (2500, 2048)])
def test_way_back(G, B, D, stream):
    import torch
    from paper_2011_09208_amd import binding as ws
    print(f"[norm back] B={B} D={D} {stream}", flush=True)
    _, h, gamma, dt = _inputs(B, D, stream, 7 * B + D)
    g = torch.Generator(device="cuda").manual_seed(B)
    dY = torch.randn((B, D), device="cuda", generator=g) * 1e-2
    dres = (torch.randn((B, D), device="cuda", generator=g) * 1e-2).to(dt)
    rstd = 1 / torch.sqrt(h.float().square().mean(1) + 1e-6)
    nws = ws.rms_norm_bwd_workspace_bytes(B, D)
    hd, gd, dd, rd = _f64(h), _f64(gamma), _f64(dY), _f64(rstd)[:, None]
    xh = hd * rd
    gy = dd * gd
    mean = (gy * xh).mean(1, keepdims=True)
    want = rd * (gy - xh * mean)
    # the mean: at most 32 products in a row per lane and a tree of 6 + 16, each product off by 3; the rest a few roundings
    slack = rd * (6 * np.abs(gy) + np.abs(xh) * (64 * np.abs(gy * xh).mean(1, keepdims=True) + 6 * np.abs(mean))) * U
    want_g = (dd * xh).sum(0)
    # rows one after the other in a wave, then four waves, 32 workgroups in a row and 32 sums of those; two roundings of the product
    steps = B // 512 + 1 + 4 + 16 + 32 + 3
    slack_g = steps * U * np.abs(dd * xh).sum(0)
    for through in (None, dres):
        dh, dg, work = G.Guarded(B, D, dt, pad_cols=8), G.Guarded(1, D, torch.float32), G.Guarded(1, nws, torch.uint8)
        ws.rms_norm_bwd(dY, h, through, gamma, rstd, dh.t, dg.vec(), work.vec())
        torch.cuda.synchronize()
        assert dh.intact_outside_payload() and dg.intact_outside_payload() and work.intact_outside_payload()
        total = want if through is None else want + _f64(dres)
        assert np.all(np.abs(_f64(dh.t) - total) <= HALF[stream] * np.abs(total) + (slack + U * np.abs(total)) * (1 + 2.0 ** -7))
        assert np.all(np.abs(_f64(dg.vec()) - want_g) <= slack_g)
        again = torch.empty_like(dg.vec())
        out = dres.clone() if through is not None else torch.empty_like(dres)       # in place, without dgamma and its workspace
        ws.rms_norm_bwd(dY, h, None if through is None else out, gamma, rstd, out, None, None)
        assert torch.equal(out, dh.t)
        ws.rms_norm_bwd(dY, h, through, gamma, rstd, out, again, work.vec())
        assert torch.equal(again, dg.vec())                                         # the same order of the sums


def test_gradient_against_differences(G):
    """Central differences of the 64-bit norm, along random directions."""
    import torch
    from paper_2011_09208_amd import binding as ws
    B, D, eps = 3, 128, 1e-3
    rng = np.random.default_rng(0)
    h, gamma, dY = rng.normal(size=(B, D)), 1 + 0.3 * rng.normal(size=D), rng.normal(size=(B, D))

    def loss(hh, gg):
        return (dY * hh / np.sqrt((hh * hh).mean(1, keepdims=True) + eps) * gg).sum()

    dev = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()                     # noqa: E731
    rstd = dev(1 / np.sqrt((h * h).mean(1) + eps))
    dh, dg = torch.empty((B, D), device="cuda"), torch.empty(D, device="cuda")
    work = torch.empty(ws.rms_norm_bwd_workspace_bytes(B, D), device="cuda", dtype=torch.uint8)
    ws.rms_norm_bwd(dev(dY), dev(h), None, dev(gamma), rstd, dh, dg, work)
    for _ in range(4):
        u, v, t = rng.normal(size=(B, D)), rng.normal(size=D), 1e-4
        diff = (loss(h + t * u, gamma + t * v) - loss(h - t * u, gamma - t * v)) / (2 * t)
        got = (_f64(dh) * u).sum() + (_f64(dg) * v).sum()
        size = np.abs(_f64(dh) * u).sum() + np.abs(_f64(dg) * v).sum()
        assert abs(got - diff) <= 1e-5 * size             # t^2 of the differences, and fp32 inputs
