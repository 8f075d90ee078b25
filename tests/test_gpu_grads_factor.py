"""GPU: clipping factors far below fp32's range, whose products with large gradients are ordinary numbers."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {2: 2.0 ** -8, 4: 2.0 ** -24}
LEAST = {2: 2.0 ** -134, 4: 2.0 ** -150}                  # half a step among the subnormal numbers


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU; there is no CPU fallback")
    return torch


def _grads(torch, size):
    """Whole chunks, a piece of one, a pitch; both types."""
    g = torch.Generator(device="cuda").manual_seed(3)
    make = lambda *s: torch.rand(s, device="cuda", generator=g).sub_(0.5).mul_(2.0).mul_(size)                      # noqa: E731
    return [make(8192 * 3 + 17), make(20000).bfloat16(), make(9, 40)[:, :33], make(5).bfloat16(), make(7, 9000).bfloat16()[:, 1:]]


def _norm(torch, grads):
    from paper_2011_09208_amd import binding as ws
    sumsq = torch.empty(1, device="cuda", dtype=torch.float64)
    ws.grad_sumsq(grads, sumsq, torch.empty(ws.grad_workspace_bytes(len(grads)), device="cuda", dtype=torch.uint8))
    return sumsq


# factors around 1e-39, where fp32 has lost bits, and far below; the last one is the smallest that fp32 holds in full
CASES = [(1e30, 1e-20), (1e38, 1e-3), (3e38, 1e-30), (1e20, 1e-19), (1e36, 1e-2), (1e30, 1e-7), (1e30, 1e-5)]


@pytest.mark.parametrize("size,limit", CASES)
def test_clipping_in_place(torch, size, limit):
    from paper_2011_09208_amd import binding as ws
    grads = _grads(torch, size)
    before = [g.double() for g in grads]
    want = math.sqrt(sum((g * g).sum().item() for g in before))
    sumsq, norm = _norm(torch, grads), torch.empty(1, device="cuda")
    ws.grad_clip(grads, sumsq, limit, norm)
    k = float(np.float32(limit)) / want
    assert k < 2.0 ** -119
    for g, b in zip(grads, before):
        w = b * k
        assert ((g.double() - w).abs() <= (HALF[g.element_size()] + 2.1 * U) * w.abs() + LEAST[g.element_size()] + LEAST[4]).all()
    assert bool((torch.stack([g.abs().max().double() for g in grads]) > 0).all())


@pytest.mark.parametrize("size,limit", CASES)
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_clipping_into_the_update(torch, size, limit, kind):
    from paper_2011_09208_amd import binding as ws
    grads, lr = _grads(torch, size), 0.5
    dt = torch.bfloat16 if kind == "bf16" else torch.float32
    params = [(torch.rand(g.shape, device="cuda") * (limit / 100)).to(dt) for g in grads]
    before, sumsq = [p.double() for p in params], _norm(torch, grads)
    k = float(np.float32(limit)) / math.sqrt(sumsq.item())
    ws.grad_clip_sgd(params, grads, sumsq, limit, lr)
    for p, b, g in zip(params, before, grads):
        step = lr * k * g.double()
        w = b - step
        # k and k g are rounded, then the result to fp32 and to its type
        bound = HALF[p.element_size()] * w.abs() * (1 + 2.0 ** -7) + 1.01 * U * w.abs() + 2.1 * U * step.abs() + 2 * LEAST[4] + LEAST[p.element_size()]
        assert ((p.double() - w).abs() <= bound).all()
        assert not torch.equal(p.double(), b)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_a_norm_that_is_not_finite_still_leaves_the_step_out(torch, bad):
    from paper_2011_09208_amd import binding as ws
    grads = _grads(torch, 1e30)
    grads[0][77] = bad
    params = [torch.ones_like(g) for g in grads]
    sumsq = _norm(torch, grads)
    ws.grad_clip_sgd(params, grads, sumsq, 1e-20, 0.5)
    assert all(bool((p == 1).all()) for p in params)
    ws.grad_clip(grads, sumsq, 1e-20)
    assert all(bool((g == 0).all()) for g in grads)
