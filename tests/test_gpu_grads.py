"""GPU: the norm over many gradients, clipping in place and into the update, against the formulas in 64 bits."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {2: 2.0 ** -8, 4: 2.0 ** -24}


@pytest.fixture(scope="module")
def G():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU; there is no CPU fallback")
    from tests import gpu_harness
    return gpu_harness


def _tensors(G, shapes, seed, scale=1e-2):
    """Guarded tensors: (rows, cols, type, elements by which the start is moved off a 16-byte boundary, padding columns)."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    guards, views = [], []
    for rows, cols, kind, off, pad in shapes:
        dt = torch.bfloat16 if kind == "bf16" else torch.float32
        g = G.Guarded(rows, off + cols, dt, pad_cols=pad)
        v = g.t[:, off:]
        v.copy_((torch.randn((rows, cols), device="cuda", generator=gen) * scale).to(dt))
        guards.append((g, off))
        views.append(v if rows > 1 else v[0])
    return guards, views


def _outside_intact(G, guard, off):
    g = guard
    r = g.raw.clone()
    if off:
        import torch
        as_int = {2: torch.int16, 4: torch.int32}[g.es]
        fill = {2: int(np.int16(np.uint16(0xA5A5))), 4: int(np.int32(np.uint32(0xA5A5A5A5)))}[g.es]
        p = g._payload(r, as_int)
        if not bool((p[:, :off] == fill).all()):
            return False
    return g.intact_outside_payload()


MIXED = [(5, 64, "bf16", 0, 0), (1, 1, "fp32", 0, 0), (1, 7, "bf16", 3, 0), (1, 1001, "fp32", 1, 0), (13, 33, "bf16", 1, 8), (300, 257, "fp32", 0, 3),
         (1, 30000, "bf16", 5, 0), (7, 9001, "bf16", 0, 7), (3, 8192, "fp32", 2, 0), (1000, 1, "fp32", 0, 4), (64, 8193, "bf16", 0, 1)]



@pytest.mark.parametrize("limit", [0.3, 1.0 - 1e-6, 1.0 + 1e-6, 5.0, float("inf")])
def test_norm_and_clipping_in_place(G, limit):
    import torch
    from paper_2011_09208_amd import binding as ws
    guards, views = _tensors(G, MIXED, 1)
    before = [v.clone() for v in views]
    want = math.sqrt(sum((v.double() ** 2).sum().item() for v in views))
    n = ws.grad_workspace_bytes(len(views))
    work, sumsq, norm = G.Guarded(1, n, torch.uint8), torch.full((1,), float("nan"), device="cuda", dtype=torch.float64), torch.empty(1, device="cuda")
    table = ws.grad_table(views)
    ws.grad_sumsq(table, sumsq, work.vec())
    torch.cuda.synchronize()
    assert work.intact_outside_payload()
    # 64-bit sums of exact squares; at most some thousands of additions in a row
    assert abs(sumsq.item() - want * want) <= 1e-12 * want * want
    ws.grad_clip(table, sumsq, limit * want, norm)
    torch.cuda.synchronize()
    assert abs(norm.item() - want) <= U * want * (1 + 1e-6)
    m = float(np.float32(limit * want)) if math.isfinite(limit) else math.inf
    k = min(1.0, m / want)
    for (g, off), v, b in zip(guards, views, before):
        assert _outside_intact(G, g, off)
        if k == 1.0:
            assert torch.equal(v, b)
            continue
        w = b.double() * k                                # the factor is rounded, then the product, then to the type
        assert ((v.double() - w).abs() <= (HALF[v.element_size()] + 2.1 * U) * w.abs() + 1e-38).all()


@pytest.mark.parametrize("limit", [0.3, 2.0])
def test_clipping_into_the_update(G, limit):
    import torch
    from paper_2011_09208_amd import binding as ws
    _, grads = _tensors(G, MIXED, 2)
    other = {"bf16": "fp32", "fp32": "bf16"}
    for kinds in ("same", "other"):
        shapes = [(r, c, k if kinds == "same" else other[k], (o + i) % 4, 5 - i % 5) for i, (r, c, k, o, _) in enumerate(MIXED)]
        guards, params = _tensors(G, shapes, 3, 1.0)
        before, gbefore = [p.double() for p in params], [g.clone() for g in grads]
        work, sumsq, norm = (torch.empty(ws.grad_workspace_bytes(len(grads)), device="cuda", dtype=torch.uint8),
                             torch.empty(1, device="cuda", dtype=torch.float64), torch.empty(1, device="cuda"))
        ws.grad_sumsq(grads, sumsq, work)
        want = math.sqrt(sumsq.item())
        lr = 0.3
        ws.grad_clip_sgd(params, grads, sumsq, limit * want, lr, norm)
        torch.cuda.synchronize()
        k, lr = min(1.0, float(np.float32(limit * want)) / want), float(np.float32(lr))
        for (g, off), p, b, gr, gb in zip(guards, params, before, grads, gbefore):
            assert _outside_intact(G, g, off) and torch.equal(gr, gb)
            step = lr * k * gr.double()
            w = b - step
            # k and k g are rounded, then the result to fp32 and to its type
            assert ((p.double() - w).abs() <= HALF[p.element_size()] * w.abs() * (1 + 2.0 ** -7) + 1.01 * U * w.abs() + 2.1 * U * step.abs()).all()


def test_many_tensors_and_parts(G):
    """More tensors than a launch takes, some of them empty, in two parts as two devices hold them."""
    import torch
    from paper_2011_09208_amd import binding as ws
    gen = torch.Generator(device="cuda").manual_seed(9)
    grads = [torch.randn((int(n),), device="cuda", generator=gen).to(torch.bfloat16 if i % 3 else torch.float32)
             for i, n in enumerate(np.random.default_rng(0).integers(0, 5000, 301))]
    grads[5], grads[100], grads[300] = (torch.empty(0, device="cuda") for _ in range(3))
    grads.append(torch.empty((0, 8), device="cuda", dtype=torch.bfloat16))
    sumsq = torch.empty(2, device="cuda", dtype=torch.float64)
    work = torch.empty(ws.grad_workspace_bytes(len(grads)), device="cuda", dtype=torch.uint8)
    ws.grad_sumsq(grads[:120], sumsq[:1], work)
    ws.grad_sumsq(grads[120:], sumsq[1:], work)
    want = [sum((g.double() ** 2).sum().item() for g in part) for part in (grads[:120], grads[120:])]
    assert np.all(np.abs(sumsq.cpu().numpy() - want) <= 1e-12 * np.array(want))
    whole, norm = torch.empty(1, device="cuda", dtype=torch.float64), torch.empty(1, device="cuda")
    ws.grad_sumsq(grads, whole, work)
    again = torch.empty_like(whole)
    ws.grad_sumsq(grads, again, work)
    assert torch.equal(whole, again)                       # the same order of the sums
    before = [g.clone() for g in grads]
    ws.grad_clip(grads, sumsq, 1.0, norm)
    assert abs(norm.item() - math.sqrt(sum(want))) <= 2 * U * norm.item()
    k = 1.0 / math.sqrt(sum(want))
    for g, b in zip(grads, before):
        w = b.double() * k
        assert ((g.double() - w).abs() <= (HALF[g.element_size()] + 2.1 * U) * w.abs()).all()


def test_nothing_at_all(G):
    """No tensors, or none with elements: the sum is 0, the norm is 0."""
    import torch
    from paper_2011_09208_amd import binding as ws
    work = torch.empty(ws.grad_workspace_bytes(0), device="cuda", dtype=torch.uint8)
    for grads in ([], [torch.empty(0, device="cuda")]):
        sumsq, norm = torch.full((1,), 7.0, device="cuda", dtype=torch.float64), torch.full((1,), 7.0, device="cuda")
        ws.grad_sumsq(grads, sumsq, torch.empty(ws.grad_workspace_bytes(len(grads)), device="cuda", dtype=torch.uint8))
        assert sumsq.item() == 0.0
        ws.grad_clip(grads, sumsq, 1.0, norm)
        assert norm.item() == 0.0
        norm.fill_(7.0)
        ws.grad_clip_sgd(grads, grads, sumsq, 1.0, 0.1, norm)
        assert norm.item() == 0.0
    del work


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_a_norm_that_is_not_finite_leaves_the_step_out(G, bad, kind):
    import torch
    from paper_2011_09208_amd import binding as ws
    _, grads = _tensors(G, [(9, 777, kind, 0, 0), (1, 50, "fp32", 0, 0)], 4)
    grads[0][4, 300] = bad
    params = [torch.ones_like(g) for g in grads]
    sumsq, norm = torch.empty(1, device="cuda", dtype=torch.float64), torch.empty(1, device="cuda")
    work = torch.empty(ws.grad_workspace_bytes(2), device="cuda", dtype=torch.uint8)
    ws.grad_sumsq(grads, sumsq, work)
    ws.grad_clip_sgd(params, grads, sumsq, 1.0, 0.1, norm)
    assert not math.isfinite(norm.item()) and math.isnan(norm.item()) == math.isnan(bad)
    assert all((p == 1).all() for p in params)
    ws.grad_clip(grads, sumsq, float("inf"), norm)
    assert all((g == 0).all() for g in grads)


def test_sizes_that_overflow_or_vanish_in_32_bits(G):
    import torch
    from paper_2011_09208_amd import binding as ws
    work = torch.empty(ws.grad_workspace_bytes(1), device="cuda", dtype=torch.uint8)
    sumsq, norm = torch.empty(1, device="cuda", dtype=torch.float64), torch.empty(1, device="cuda")
    for size in (1e30, 1e-30):
        g = torch.full((4096,), size, device="cuda")
        want = float(g[0]) * 64
        ws.grad_sumsq([g], sumsq, work)
        ws.grad_clip([g], sumsq, want / 4, norm)
        assert abs(norm.item() - want) <= 2 * U * want and abs(g[5].item() / (want / 256) - 1) <= 4 * U


def test_more_elements_than_31_bits(G):
    """One gradient of 2^31 + 77 values and one behind it."""
    import torch
    from paper_2011_09208_amd import binding as ws
    n = (1 << 31) + 77
    g = torch.zeros(n, device="cuda", dtype=torch.bfloat16)
    g[-1], g[0], g[1 << 30] = 3.0, 4.0, 12.0
    tail = torch.full((1,), 84.0, device="cuda")
    sumsq, norm = torch.empty(1, device="cuda", dtype=torch.float64), torch.empty(1, device="cuda")
    ws.grad_sumsq([g, tail], sumsq, torch.empty(ws.grad_workspace_bytes(2), device="cuda", dtype=torch.uint8))
    assert sumsq.item() == 85.0 ** 2
    ws.grad_clip([g, tail], sumsq, 42.5, norm)
    assert (float(g[-1]), float(g[0]), float(g[1 << 30]), float(tail)) == (1.5, 2.0, 6.0, 42.0) and norm.item() == 85.0
