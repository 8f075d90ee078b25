"""GPU: packing to 4 bits, and the logits and arg-max of a layer with 4-bit weights, against the formats' definitions in 64 bits."""
import numpy as np
import pytest

from paper_2011_09208_amd import inputs
from tests import mx_formats as mx

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU; there is no CPU fallback")
    from tests import gpu_harness
    return gpu_harness


def _dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def test_packing_every_value(G):
    """Every bf16 value, as the largest of its group (31 zeros) and beside others: codes and scales are determined to the bit."""
    import torch
    from paper_2011_09208_amd import binding as ws
    bits = np.arange(65536, dtype=np.uint16)
    alone = np.zeros((512, 128, 32), np.uint16)
    alone[:, :, 5] = bits.reshape(512, 128)
    mixed = bits.reshape(16, 64, 64).transpose(1, 0, 2).copy().reshape(64, 1024)         # neighbours in magnitude
    rng = np.random.default_rng(1)
    order = rng.permutation(bits).reshape(64, 1024)                                      # magnitudes far apart
    for w in (alone.reshape(512, 4096), mixed, order):
        C, D = w.shape
        W4, s = G.Guarded(C, D // 2, torch.uint8, pad_cols=16), G.Guarded(C, D // 32, torch.uint8, pad_cols=2)
        ws.quantize_mx4(G.dev_bf16(w), W4.t, s.t)
        torch.cuda.synchronize()
        assert W4.intact_outside_payload() and s.intact_outside_payload()
        codes, scales = mx.quantize4(inputs.bf16_bits_to_f64(w))
        assert np.array_equal(s.t.cpu().numpy(), scales)
        fine = np.repeat(scales != 255, 16, 1)                                           # a NaN group's codes stand for nothing
        assert np.array_equal(W4.t.cpu().numpy()[fine], codes[fine])


@pytest.mark.parametrize("C,D", [(1, 64), (3, 192), (1001, 64), (77, 1088), (515, 4160)])
def test_packing(G, C, D):
    import torch
    from paper_2011_09208_amd import binding as ws
    p = inputs.make_inputs("w4-pack", 1, D, C, w_sigma=0.05, seed=C)
    wide = torch.zeros((C, D + 72), device="cuda", dtype=torch.bfloat16)
    wide[:, 64:64 + D] = G.dev_bf16(p.W_bits)
    W4, s = torch.empty((C, D // 2), device="cuda", dtype=torch.uint8), torch.empty((C, D // 32), device="cuda", dtype=torch.uint8)
    ws.quantize_mx4(wide[:, 64:64 + D], W4, s)                                           # rows with a pitch
    codes, scales = mx.quantize4(inputs.bf16_bits_to_f64(p.W_bits))
    assert np.array_equal(s.cpu().numpy(), scales) and np.array_equal(W4.cpu().numpy(), codes)


def _layer(B, D, C, x_kind, seed):
    """Random codes and scales of some spread, features in either form; values in 64 bits beside them."""
    rng = np.random.default_rng(seed)
    W4 = rng.integers(0, 256, (C, D // 2), dtype=np.uint8)
    ws_ = rng.integers(119, 124, (C, D // 32), dtype=np.uint8)
    bias = rng.normal(size=C).astype(np.float32)
    if x_kind == "bf16":
        xb = inputs.f32_to_bf16_bits(rng.normal(size=(B, D)).astype(np.float32))
        return W4, ws_, bias, xb, None, inputs.bf16_bits_to_f64(xb)
    q = rng.integers(0, 256, (B, D), dtype=np.uint8)
    q[(q & 127) == 127] = 0                                                              # no NaNs
    xs = rng.integers(116, 121, (B, D // 32), dtype=np.uint8)
    return W4, ws_, bias, q, xs, mx.values8(q, xs)


def _slack(X, W, D):
    """Products are exact; a matrix instruction adds 32 of them to a sum with at most 32 roundings of a step each, of at most the sum
    of the magnitudes, and the sum passes D / 32 instructions, the waves' shares and the bias."""
    return (D / 32 + 32 + 16) * 2.0 ** -23 * (np.abs(X) @ np.abs(W).T + 4.0)


# one row, rows of one tile and more than one; D in a part of a span, whole spans and a rest, more than a chunk of features; few classes
SHAPES = [(1, 64, 1), (1, 64, 5), (2, 128, 63), (1, 2048, 1001), (3, 192, 64), (5, 320, 65), (16, 512, 130), (17, 576, 100), (1, 8192, 77), (15, 8256, 70),
          (32, 1088, 257), (33, 640, 129), (64, 2112, 260), (65, 704, 131), (100, 4160, 67), (201, 1088, 515), (129, 64, 1000), (256, 448, 64), (300, 1600, 190)]


@pytest.mark.parametrize("x_kind", ["bf16", "mx8"])
@pytest.mark.parametrize("B,D,C", SHAPES)
def test_logits_and_top1(G, B, D, C, x_kind):
    import torch
    from paper_2011_09208_amd import binding as ws
    print(f"[w4] B={B} D={D} C={C} {x_kind}", flush=True)
    W4, s, bias, x, xs, X = _layer(B, D, C, x_kind, B + D + C)
    W = mx.values4(W4, s)
    dx = G.dev_bf16(x) if xs is None else _dev(x)
    dxs = None if xs is None else _dev(xs)
    d4, ds, db = _dev(W4), _dev(s), _dev(bias)
    z = X @ W.T
    slack = _slack(X, W, D)
    for b in (None, db):
        want = z if b is None else z + bias.astype(np.float64)
        Z = G.Guarded(B, C, torch.float32, pad_cols=(-C) % 4 + 4)
        ws.split_fc_w4_logits(dx, dxs, d4, ds, b, Z.t)
        torch.cuda.synchronize()
        assert Z.intact_outside_payload()
        got = Z.t.double().cpu().numpy()
        assert np.all(np.abs(got - want) <= slack), np.max(np.abs(got - want) / slack)
        top, cls, work = G.Guarded(1, B, torch.float32), G.Guarded(1, B, torch.int32), G.Guarded(1, ws.w4_top1_workspace_bytes(B, C), torch.uint8)
        ws.split_fc_w4_top1(dx, dxs, d4, ds, b, 1000, top.vec(), cls.vec(), work.vec())
        torch.cuda.synchronize()
        assert top.intact_outside_payload() and cls.intact_outside_payload() and work.intact_outside_payload()
        at = cls.vec().cpu().numpy().astype(np.int64) - 1000
        assert np.all((at >= 0) & (at < C))
        r = np.arange(B)
        assert np.all(np.abs(top.vec().double().cpu().numpy() - want[r, at]) <= slack[r, at])
        assert np.all(want[r, at] >= want.max(1) - 2 * slack.max(1))


# Every way of dividing the work, at sizes where it is taken: rows that stream (short and long ones), contractions shared out among waves (by every
# number of steps), tiles of rows and classes (narrow and wide ones of every height)
LARGE = [(1, 512, 20000), (9, 2048, 17000), (32, 1984, 17000), (1, 4224, 9000), (3, 1024, 2000), (20, 1088, 3100), (5, 2048, 1000), (64, 2048, 5000),
         (7, 4096, 8000), (31, 4096, 500), (1, 4224, 300), (40, 8192, 2000), (20, 8256, 300), (20, 8256, 42000), (50, 576, 1000), (64, 512, 42001),
         (40, 1024, 2000), (33, 2048, 12500), (5, 2048, 12400), (31, 4096, 8000), (2, 4096, 300), (17, 1984, 300), (64, 4160, 500), (100, 2048, 3000), (200, 1024, 4000), (129, 8192, 1000),
         (2000, 1024, 200), (70, 4096, 1500), (40, 64, 45000), (96, 576, 83000), (100, 128, 90003), (73, 128, 90003), (128, 320, 83001), (250, 64, 45000)]


def _device_layer(B, D, C, x_kind, seed):
    """As _layer, on the device, with the 64-bit values."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    W4 = torch.randint(0, 256, (C, D // 2), device="cuda", dtype=torch.uint8, generator=gen)
    s = torch.randint(119, 124, (C, D // 32), device="cuda", dtype=torch.uint8, generator=gen)
    codes = torch.stack((W4 & 15, W4 >> 4), 2).reshape(C, D).long()
    W = _dev(mx.E2M1)[codes] * torch.exp2(s.double() - 127).repeat_interleave(32, 1)
    if x_kind == "bf16":
        x, xs = torch.randn((B, D), device="cuda", generator=gen).bfloat16(), None
        X = x.double()
    else:
        x = torch.randint(0, 256, (B, D), device="cuda", dtype=torch.uint8, generator=gen)
        x[(x & 127) == 127] = 0
        xs = torch.randint(116, 121, (B, D // 32), device="cuda", dtype=torch.uint8, generator=gen)
        X = _dev(mx.E4M3)[x.long()] * torch.exp2(xs.double() - 127).repeat_interleave(32, 1)
    return W4, s, torch.randn(C, device="cuda", generator=gen), x, xs, X, W


@pytest.mark.parametrize("x_kind", ["bf16", "mx8"])
@pytest.mark.parametrize("B,D,C", LARGE)
def test_every_division_of_the_work(G, B, D, C, x_kind):
    import torch
    from paper_2011_09208_amd import binding as ws
    print(f"[w4] B={B} D={D} C={C} {x_kind}", flush=True)
    W4, s, bias, x, xs, X, W = _device_layer(B, D, C, x_kind, B + D + C)
    want = X @ W.T + bias.double()
    slack = (D / 32 + 32 + 16) * 2.0 ** -23 * (X.abs() @ W.abs().T + 4.0)                # as _slack
    Z = G.Guarded(B, C, torch.float32, pad_cols=(-C) % 4 + 4)
    ws.split_fc_w4_logits(x, xs, W4, s, bias, Z.t)
    torch.cuda.synchronize()
    assert Z.intact_outside_payload()
    assert bool(((Z.t.double() - want).abs() <= slack).all())
    top, cls, work = G.Guarded(1, B, torch.float32), G.Guarded(1, B, torch.int32), G.Guarded(1, ws.w4_top1_workspace_bytes(B, C), torch.uint8)
    ws.split_fc_w4_top1(x, xs, W4, s, bias, 7, top.vec(), cls.vec(), work.vec())
    torch.cuda.synchronize()
    assert top.intact_outside_payload() and cls.intact_outside_payload() and work.intact_outside_payload()
    at = (cls.vec().long() - 7)[:, None]
    assert bool(((at >= 0) & (at < C)).all())
    assert bool(((top.vec().double()[:, None] - want.gather(1, at)).abs() <= slack.gather(1, at)).all())
    assert bool((want.gather(1, at)[:, 0] >= want.max(1).values - 2 * slack.max(1).values).all())
    # both calls add the products of a logit in one order
    assert torch.equal(top.vec(), Z.t.max(1).values) and torch.equal(Z.t.gather(1, at)[:, 0], top.vec())


def test_as_many_rows_as_there_may_be(G):
    """2^20 rows against several groups of classes; every row is one of 64 that come again and again."""
    import torch
    from paper_2011_09208_amd import binding as ws
    B, D, C = 1 << 20, 64, 17000
    W4, s, bias, x, _, X, W = _device_layer(64, D, C, "bf16", 3)
    want = X @ W.T + bias.double()
    top, cls = torch.empty(B, device="cuda"), torch.empty(B, device="cuda", dtype=torch.int32)
    work = torch.empty(ws.w4_top1_workspace_bytes(B, C), device="cuda", dtype=torch.uint8)
    ws.split_fc_w4_top1(x.repeat(B // 64, 1), None, W4, s, bias, 0, top, cls, work)
    at = cls[:64].long()[:, None]
    slack = (D / 32 + 32 + 16) * 2.0 ** -23 * (X.abs() @ W.abs().T + 4.0)
    assert bool((want.gather(1, at)[:, 0] >= want.max(1).values - 2 * slack.max(1).values).all())
    assert torch.equal(cls.view(-1, 64), cls[:64].expand(B // 64, 64)) and torch.equal(top.view(-1, 64), top[:64].expand(B // 64, 64))


def test_pitches_and_slices_of_a_packed_layer(G):
    """A slice of the rows of the packed layer is the shard; pitched codes, scales and features."""
    import torch
    from paper_2011_09208_amd import binding as ws
    B, D, C = 21, 320, 700
    for kind in ("bf16", "mx8"):
        W4, s, bias, x, xs, X = _layer(B, D, C, kind, 4)
        big4 = torch.full((C, D // 2 + 48), 0x77, device="cuda", dtype=torch.uint8)
        bigs = torch.full((C, D // 32 + 6), 255, device="cuda", dtype=torch.uint8)
        big4[:, 16:16 + D // 2], bigs[:, 2:2 + D // 32] = _dev(W4), _dev(s)
        bigx = torch.full((B, D + 48), float("nan"), device="cuda", dtype=torch.bfloat16) if xs is None else torch.full((B, D + 48), 127, device="cuda", dtype=torch.uint8)
        bigx[:, 16:16 + D] = G.dev_bf16(x) if xs is None else _dev(x)
        bxs = None
        if xs is not None:
            bxs = torch.full((B, D // 32 + 4), 255, device="cuda", dtype=torch.uint8)
            bxs[:, 2:2 + D // 32] = _dev(xs)
            bxs = bxs[:, 2:2 + D // 32]
        W = mx.values4(W4, s)
        for a, e in ((0, 333), (333, 700)):
            Z = torch.full((B, 400), float("nan"), device="cuda")
            ws.split_fc_w4_logits(bigx[:, 16:16 + D], bxs, big4[a:e, 16:16 + D // 2], bigs[a:e, 2:2 + D // 32], _dev(bias)[a:e], Z[:, :e - a])
            got = Z.double().cpu().numpy()
            assert np.all(np.abs(got[:, :e - a] - (X @ W[a:e].T + bias[a:e])) <= _slack(X, W[a:e], D)) and np.isnan(got[:, e - a:]).all()


def test_equal_logits_and_nan(G):
    """The lowest class of equal ones wins, within a tile, across waves and workgroups; a NaN logit never wins."""
    import torch
    from paper_2011_09208_amd import binding as ws
    B, D, C = 19, 128, 1500
    W4, s, _, x, _, _ = _layer(B, D, C, "bf16", 8)
    W4[:] = W4[7]
    s[:] = s[7]
    bias = np.zeros(C, np.float32)
    bias[:11] = -5
    bias[400], bias[900] = np.float32("nan"), np.float32("-inf")
    top, cls = torch.empty(B, device="cuda"), torch.empty(B, device="cuda", dtype=torch.int32)
    work = torch.empty(ws.w4_top1_workspace_bytes(B, C), device="cuda", dtype=torch.uint8)
    ws.split_fc_w4_top1(G.dev_bf16(x), None, _dev(W4), _dev(s), _dev(bias), 0, top, cls, work)
    assert torch.equal(cls.cpu(), torch.full((B,), 11, dtype=torch.int32))
    bias[:] = float("-inf")
    bias[1333] = -1e30
    ws.split_fc_w4_top1(G.dev_bf16(x), None, _dev(W4), _dev(s), _dev(bias), 0, top, cls, work)
    assert torch.equal(cls.cpu(), torch.full((B,), 1333, dtype=torch.int32))


@pytest.mark.parametrize("byte", [1, 10, 100, 127, 200, 240])
def test_scales_of_every_size(G, byte):
    """One group far from the others; features of 1."""
    import torch
    from paper_2011_09208_amd import binding as ws
    D, C = 128, 32
    W4, s = np.full((C, D // 2), 0x22, np.uint8), np.full((C, D // 32), byte, np.uint8)          # codes of 1
    s[3, 2] = 255
    Z = torch.empty((1, C), device="cuda")
    ws.split_fc_w4_logits(torch.ones((1, D), device="cuda", dtype=torch.bfloat16), None, _dev(W4), _dev(s), None, Z)
    got = Z.double().cpu().numpy()[0]
    assert np.isnan(got[3]) and np.all(np.delete(got, 3) == D * 2.0 ** (byte - 127))


def test_codes_beyond_four_gigabytes(G):
    """The last classes of a layer whose codes pass 32-bit offsets."""
    import torch
    from paper_2011_09208_amd import binding as ws
    D, C = 64, (1 << 27) + 77                                                            # 4.3 GB of codes, 0.27 of scales
    W4 = torch.zeros((C, D // 2), device="cuda", dtype=torch.uint8)
    s = torch.full((C, D // 32), 127, device="cuda", dtype=torch.uint8)
    W4[C - 3] = 0x22
    X = torch.ones((1, D), device="cuda", dtype=torch.bfloat16)
    top, cls = torch.empty(1, device="cuda"), torch.empty(1, device="cuda", dtype=torch.int32)
    work = torch.empty(ws.w4_top1_workspace_bytes(1, C), device="cuda", dtype=torch.uint8)
    ws.split_fc_w4_top1(X, None, W4, s, None, 5, top, cls, work)
    assert float(top) == 64.0 and int(cls) == C - 3 + 5
    Z = torch.empty((1, 80), device="cuda")
    ws.split_fc_w4_logits(X, None, W4[C - 80:], s[C - 80:], None, Z)
    assert float(Z[0, 77]) == 64.0 and float(Z.abs().sum()) == 64.0


@pytest.mark.parametrize("B", [1, 40])
def test_as_many_classes_as_there_may_be(G, B):
    """2^30 - 65 536 classes: 34 GB of codes, 4 GB of biases; rows of 1, codes of 0 but for one class, the bias of another one outside its part."""
    import torch
    from paper_2011_09208_amd import binding as ws
    D, C = 64, ws.W4_MAX_CLASSES
    W4 = torch.zeros((C, D // 2), device="cuda", dtype=torch.uint8)
    s = torch.full((C, D // 32), 127, device="cuda", dtype=torch.uint8)
    bias = torch.zeros(C, device="cuda")
    X = torch.ones((B, D), device="cuda", dtype=torch.bfloat16)
    top, cls = torch.empty(B, device="cuda"), torch.empty(B, device="cuda", dtype=torch.int32)
    work = torch.empty(ws.w4_top1_workspace_bytes(B, C), device="cuda", dtype=torch.uint8)
    W4[C - 3] = 0x22                                                                     # codes of 1
    ws.split_fc_w4_top1(X, None, W4, s, bias, 9, top, cls, work)
    assert bool((top == 64).all()) and bool((cls == C - 3 + 9).all())
    bias[C - 1], bias[(1 << 29) + 5] = 65, 64.5
    ws.split_fc_w4_top1(X, None, W4, s, bias, 9, top, cls, work)
    assert bool((top == 65).all()) and bool((cls == C - 1 + 9).all())
    bias[C - 1] = 0
    ws.split_fc_w4_top1(X, None, W4, s, bias, 9, top, cls, work)
    assert bool((top == 64.5).all()) and bool((cls == (1 << 29) + 5 + 9).all())
    if B == 1:
        Z = torch.full((B, C), -1.0, device="cuda")
        ws.split_fc_w4_logits(X, None, W4, s, bias, Z)
        assert float(Z[0, C - 3]) == 64 and float(Z[0, (1 << 29) + 5]) == 64.5 and int((Z != 0).sum()) == 2
