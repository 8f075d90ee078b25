"""GPU: rows without a logit that compares, in the arg-max of the 4-bit layer and in the merge over shards."""
import numpy as np
import pytest

from tests import mx_formats as mx

pytestmark = pytest.mark.gpu
INF, NAN, NONE = float("inf"), float("nan"), 2**31 - 1


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU; there is no CPU fallback")
    return torch


def _layer(torch, B, D, C, seed):
    """Features of 8 bits, codes and scales without NaNs, on the device."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randint(0, 256, (B, D), device="cuda", dtype=torch.uint8, generator=g)
    q[(q & 127) == 127] = 0
    u8 = lambda n, lo, hi: torch.randint(lo, hi, (n[0], n[1]), device="cuda", dtype=torch.uint8, generator=g)          # noqa: E731
    return q, u8((B, D // 32), 116, 121), u8((C, D // 2), 0, 256), u8((C, D // 32), 119, 124)


def _top1(torch, q, qs, W4, s, bias, offset):
    from paper_2011_09208_amd import binding as ws
    B, C = q.shape[0], W4.shape[0]
    top, cls = torch.full((B,), 5.0, device="cuda"), torch.full((B,), -5, device="cuda", dtype=torch.int32)
    work = torch.empty(ws.w4_top1_workspace_bytes(B, C), device="cuda", dtype=torch.uint8)
    ws.split_fc_w4_top1(q, qs, W4, s, bias, offset, top, cls, work)
    return top, cls


def _combine(torch, tops, classes):
    from paper_2011_09208_amd import binding as ws
    top, cls = torch.stack(tops).contiguous(), torch.stack(classes).contiguous()
    best, best_cls = torch.full_like(top[0], 5.0), torch.full_like(cls[0], -5)
    ws.combine_top1(top, cls, best, best_cls)
    return best, best_cls


# one row and more, by each way of dividing the work: streams, shared contractions, tiles of rows and classes
@pytest.mark.parametrize("B,D,C", [(1, 128, 1500), (9, 64, 70), (1, 2048, 1001), (20, 1088, 3100), (40, 128, 1500), (201, 1088, 515), (300, 64, 45000)])
def test_rows_of_nan(torch, B, D, C):
    q, qs, W4, s = _layer(torch, B, D, C, B + D)
    cut = C // 3
    part = lambda scales, a, e: _top1(torch, q, scales, W4[a:e], s[a:e], None, a)                                      # noqa: E731
    clean, bad = [part(qs, 0, cut), part(qs, cut, C)], qs.clone()
    rows = sorted({0, B // 2, B - 1})
    bad[rows] = 255                                       # what the norm in 8 bits makes of a row with a NaN
    got = [part(bad, 0, cut), part(bad, cut, C)]
    for (top, cls), (top0, cls0), offset in zip(got, clean, (0, cut)):
        top0[rows], cls0[rows] = NAN, offset
        assert torch.equal(cls, cls0) and torch.equal(top.isnan(), top0.isnan()) and torch.equal(top.nan_to_num(), top0.nan_to_num())
    best, best_cls = _combine(torch, [t for t, _ in got], [c for _, c in got])
    assert bool(best[rows].isnan().all()) and bool((best_cls[rows] == 0).all())
    others = [r for r in range(B) if r not in rows]
    want, want_cls = _combine(torch, [t for t, _ in clean], [c for _, c in clean])
    assert torch.equal(best[others], want[others]) and torch.equal(best_cls[others], want_cls[others])


@pytest.mark.parametrize("B,D,C", [(1, 128, 1500), (3, 2048, 1001), (40, 128, 1500)])
def test_a_shard_of_nan_beside_one_that_compares(torch, B, D, C):
    """Biases of NaN, of -infinity and of neither: what compares wins, -infinity included, and the class lies in its shard."""
    q, qs, W4, s = _layer(torch, B, D, C, 5)
    dead, low = torch.full((C,), NAN, device="cuda"), torch.full((C,), -INF, device="cuda")
    nan, ninf, fine = (_top1(torch, q, qs, W4, s, b, o) for b, o in ((dead, 0), (low, C), (None, 2 * C)))
    assert bool(nan[0].isnan().all()) and bool((nan[1] == 0).all())
    assert bool((ninf[0] == -INF).all()) and bool((ninf[1] == C).all())
    for shards, want in (((nan, ninf, fine), fine), ((nan, ninf), ninf), ((fine, nan), fine)):
        best, cls = _combine(torch, [t for t, _ in shards], [c for _, c in shards])
        assert torch.equal(best, want[0]) and torch.equal(cls, want[1])
    Z = torch.empty((B, (C + 3) // 4 * 4), device="cuda")[:, :C]                         # pitches are multiples of 4
    from paper_2011_09208_amd import binding as ws
    ws.split_fc_w4_logits(q, qs, W4, s, None, Z)
    assert torch.equal(fine[0], Z.max(1).values)


@pytest.mark.parametrize("S", [1, 2, 12, 13, 64, 200])
@pytest.mark.parametrize("B", [1, 17, 70])
def test_merge_of_candidates_that_do_not_compare(torch, S, B):
    """A candidate that compares, then the NaN of the lowest class, then none at all (-infinity and the largest int32), in every order."""
    rng = np.random.default_rng(S * 100 + B)
    kind = rng.integers(0, 3, (S, B))                     # none, NaN, a number
    kind[:, ::2] = np.minimum(kind[:, ::2], 1)            # columns without a number
    kind[:, ::3] = 0
    classes = rng.permuted(np.arange(S * B, dtype=np.int32).reshape(S, B), axis=0)
    top = np.where(kind == 2, rng.integers(-2, 3, (S, B)), np.where(kind == 1, NAN, -INF)).astype(np.float32)
    classes[kind == 0] = NONE
    best, cls = _combine(torch, list(torch.from_numpy(top).cuda()), list(torch.from_numpy(classes).cuda()))
    best, cls = best.cpu().numpy(), cls.cpu().numpy()
    for i in range(B):
        k = kind[:, i].max()
        among = [(-top[j, i] if k == 2 else 0, classes[j, i]) for j in range(S) if kind[j, i] == k]
        want, want_cls = min(among)
        assert cls[i] == want_cls
        assert (np.isnan(best[i]) if k == 1 else best[i] == (-want if k == 2 else -INF))


def test_norm_in_eight_bits_to_a_class(torch):
    """A token whose stream holds a NaN, from the norm to the answer: its class may be looked up."""
    from paper_2011_09208_amd import binding as ws
    B, D, C = 5, 192, 600
    _, _, W4, s = _layer(torch, B, D, C, 2)
    x = torch.randn((B, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.bfloat16)
    x[3, 100] = NAN
    q, qs = torch.empty((B, D), device="cuda", dtype=torch.uint8), torch.empty((B, D // 32), device="cuda", dtype=torch.uint8)
    ws.rms_norm_fwd_mx8(x, None, torch.ones(D, device="cuda"), 1e-6, None, q, qs, None)
    assert bool((qs[3] == 255).all())
    top, cls = _top1(torch, q, qs, W4, s, None, 100)
    assert torch.equal(top.isnan().cpu(), torch.tensor([False, False, False, True, False])) and int(cls[3]) == 100
    names = torch.arange(100 + C, device="cuda")
    assert bool((names[cls.long()] == cls).all())
    X, W = mx.values8(q.cpu().numpy(), qs.cpu().numpy())[[0, 1, 2, 4]], mx.values4(W4.cpu().numpy(), s.cpu().numpy())
    z, at = X @ W.T, cls.cpu().numpy()[[0, 1, 2, 4]] - 100
    slack = (D / 32 + 48) * 2.0 ** -23 * (np.abs(X) @ np.abs(W).T).max()                # fp32 sums of exact products
    assert np.all(z[range(4), at] >= z.max(1) - 2 * slack)
