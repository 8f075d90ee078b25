"""The operators around the class-split layer of a language model, measured: what makes its features out of the residual
stream (root-mean-square norm), the way back through it, the layer with 4-bit weights as it answers tokens, the packing of
those weights, and the norm and clipping of a training step's gradients with the update that follows.

Where `own` is false each is computed in its plain form, of elementary torch operations; where it is true, by the library.

A case is a dict of plain values; `kind` is
  norm    h = residual + x, y = h / rms(h) * gamma        B rows, D features; res: type of the residual stream, or "none";
                                                          out: y in "bf16", or "mx8" (e4m3 with a power of two for 32 values)
  back    the gradient of the stream and of gamma         B, D, res (bf16 or fp32); through: a gradient arrives beside the norm too
  pack    W in bf16 to 4 bits with scales                 C classes, D features
  w4      the layer with 4-bit weights                    B, D, C; x: features in "bf16" or "mx8"; out: "logits" or "top1"; bias
  clip    norm over all gradients, then clipping          head: classes of the layer, D; blocks: layers of the trunk; sgd: the
                                                          clipped update of the weights instead of clipping in place;
                                                          limit: the largest norm allowed, in units of the norm there is
"""
import math

import torch

own = False

EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # one token on its way to the layer: launch and latency
        dict(name="norm_b1", kind="norm", B=1, D=2048, res="bf16", out="bf16"),
        # a training step's token rows, residual stream in fp32
        dict(name="norm_rows", kind="norm", B=8192, D=1024, res="fp32", out="bf16"),
        # a serving batch, straight to the 8-bit features that the 4-bit layer reads
        dict(name="norm8_b32", kind="norm", B=32, D=2048, res="bf16", out="mx8"),
        # the way back of the ordinary batch
        dict(name="back_b1024", kind="back", B=1024, D=2048, res="bf16", through=False),
        # the way back of the token rows, in the middle of a trunk
        dict(name="back_rows", kind="back", B=8192, D=1024, res="fp32", through=True),
        # packing a ragged share of a layer for serving
        dict(name="pack_ragged", kind="pack", C=14450, D=1088),
        # packing the whole 100K-class layer
        dict(name="pack_layer", kind="pack", C=100000, D=2048),
        # the class of one token among 100K
        dict(name="w4_top1_b1", kind="w4", B=1, D=2048, C=100000, x="bf16", out="top1", bias=True),
        # logits of a serving batch over one GPU's share
        dict(name="w4_logits_b32", kind="w4", B=32, D=2048, C=12500, x="mx8", out="logits", bias=False),
        # many sequences at once, nothing a multiple of any tile
        dict(name="w4_ragged", kind="w4", B=201, D=1088, C=50001, x="bf16", out="logits", bias=True),
        # many small gradients of a trunk, their norm below the limit: most steps of a run
        dict(name="clip_trunk", kind="clip", head=1001, D=512, blocks=12, sgd=False, limit=1.5),
        # the whole layer's gradients, clipped into the update
        dict(name="clip_head", kind="clip", head=100000, D=2048, blocks=0, sgd=True, limit=0.5),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "back", "pack", "w4", "w4", "w4", "clip"])
    D = 64 * _log(rng, 1, 128)
    if kind == "norm":
        return dict(kind=kind, B=_log(rng, 1, min(16384, (1 << 23) // D)), D=D, res=rng.choice(["none", "bf16", "bf16", "fp32"]),
                    out=rng.choice(["bf16", "mx8"]))
    if kind == "back":
        return dict(kind=kind, B=_log(rng, 1, min(16384, (1 << 23) // D)), D=D, res=rng.choice(["bf16", "fp32"]), through=rng.random() < 0.5)
    if kind == "pack":
        return dict(kind=kind, C=_log(rng, 100, min(400000, 204800000 // D)), D=D)
    if kind == "w4":
        B = _log(rng, 1, 256)
        return dict(kind=kind, B=B, D=D, C=_log(rng, 100, min(200000, 204800000 // D, 10900000000 // (B * D))), x=rng.choice(["bf16", "mx8"]),
                    out=rng.choice(["logits", "logits", "top1"]) if B <= 32 else "logits", bias=rng.random() < 0.5)
    D = 64 * _log(rng, 1, 32)
    # clipping in place leaves gradients that the next pass would find clipped: only the update is drawn above the limit
    sgd = rng.random() < 0.7
    return dict(kind=kind, head=_log(rng, 100, min(200000, 60000000 // D)), D=D, blocks=_log(rng, 1, max(1, min(48, 100000000 // (12 * D * D)))),
                sgd=sgd, limit=rng.choice([0.1, 0.5, 0.9, 1.5]) if sgd else 1.5)


# ---- the plain forms -------------------------------------------------------------------------------------------------

def _rounded_up(amax, whole, exponent):
    """The byte e of the smallest power of two 2^(e - 127) with amax <= whole * 2^exponent * 2^(e - 127), whole in [0.5, 1)."""
    m, e = torch.frexp(amax)
    e = e + 127 - exponent + (m > whole).to(e.dtype)
    return torch.where(amax == 0, 0, e.clamp(min=0)).to(torch.uint8)


def _mx8(y):
    """e4m3 (largest value 448) and a scale for every 32 values."""
    blocks = y.unflatten(1, (-1, 32))
    s = _rounded_up(blocks.abs().amax(2), 0.875, 9)
    q = (blocks / s.view(torch.float8_e8m0fnu).float().unsqueeze(2)).flatten(1)
    return q.to(torch.float8_e4m3fn), s


def _mx4(w):
    """e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign), two to a byte, the first in the low bits, and a scale for every 32 values."""
    blocks = w.float().unflatten(1, (-1, 32))
    s = _rounded_up(blocks.abs().amax(2), 0.75, 3)
    v = (blocks / s.view(torch.float8_e8m0fnu).float().unsqueeze(2)).flatten(1)
    a = v.abs()
    # halfway values go to the even code
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
            + 8 * torch.signbit(v).to(torch.uint8))
    return code[:, 0::2] | (code[:, 1::2] << 4), s


def _values4(codes, s):
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    table = torch.cat((table, -table))
    v = table[torch.stack((codes & 15, codes >> 4), 2).flatten(1).int()]
    return (v.unflatten(1, (-1, 32)) * s.view(torch.float8_e8m0fnu).float().unsqueeze(2)).flatten(1)


def _values8(q, s):
    return (q.float().unflatten(1, (-1, 32)) * s.view(torch.float8_e8m0fnu).float().unsqueeze(2)).flatten(1)


def _norm(st):
    h = st["x"].float()
    if st["residual"] is not None:
        h = (h + st["residual"].float()).to(st["residual"].dtype)
    f = h.float()
    rstd = torch.rsqrt(f.square().mean(1) + EPS)
    y = f * rstd.unsqueeze(1) * st["gamma"]
    out = [] if st["h"] is None else [h]
    if st["out"] == "mx8":
        q, s = _mx8(y)
        return out + [q, s.view(torch.float8_e8m0fnu)]
    return out + [y.to(torch.bfloat16), rstd]


def _back(st):
    xhat = st["h"].float() * st["rstd"].unsqueeze(1)
    gy = st["dY"] * st["gamma"]
    dh = st["rstd"].unsqueeze(1) * (gy - xhat * (gy * xhat).mean(1, keepdim=True))
    if st["dres"] is not None:
        dh = dh + st["dres"].float()
    return [dh.to(st["h"].dtype), (st["dY"] * xhat).sum(0)]


def _w4(st):
    X = st["X"].float() if st["X_scales"] is None else _values8(st["X"], st["X_scales"])
    z = X @ _values4(st["W4"], st["W_scales"]).t()
    if st["bias"] is not None:
        z = z + st["bias"]
    if st["out"] == "logits":
        return [z]
    best, at = z.max(1)
    return [best, (at + st["offset"]).to(torch.int32)]


def _clip(st):
    norm = torch.stack([g.float().square().sum() for g in st["grads"]]).sum().sqrt()
    scale = torch.where(norm > st["limit"], st["limit"] / norm, 1.0)
    if st["params"] is None:
        [g.copy_(g.float() * scale) for g in st["grads"]]
    else:
        [p.copy_(p.float() - st["lr"] * (scale * g.float())) for p, g in zip(st["params"], st["grads"])]
    return [norm.reshape(1)] + (st["flat_g"] if st["params"] is None else st["flat_p"])


# ---- the library's operators -----------------------------------------------------------------------------------------

def _norm_own(st, ws):
    out = [] if st["h"] is None else [st["h"]]
    if st["out"] == "mx8":
        ws.rms_norm_fwd_mx8(st["x"], st["residual"], st["gamma"], EPS, st["h"], st["y"], st["y_scales"], None)
        return out + [st["y"].view(torch.float8_e4m3fn), st["y_scales"].view(torch.float8_e8m0fnu)]
    ws.rms_norm_fwd(st["x"], st["residual"], st["gamma"], EPS, st["h"], st["y"], st["rstd"])
    return out + [st["y"], st["rstd"]]


def _back_own(st, ws):
    ws.rms_norm_bwd(st["dY"], st["h"], st["dres"], st["gamma"], st["rstd"], st["dh"], st["dgamma"], st["work"])
    return [st["dh"], st["dgamma"]]


def _pack_own(st, ws):
    ws.quantize_mx4(st["W"], st["W4"], st["W_scales"])
    return [st["W4"], st["W_scales"]]


def _w4_own(st, ws):
    if st["out"] == "logits":
        ws.split_fc_w4_logits(st["X"], st["X_scales"], st["W4"], st["W_scales"], st["bias"], st["Z"])
        return [st["Z"]]
    ws.split_fc_w4_top1(st["X"], st["X_scales"], st["W4"], st["W_scales"], st["bias"], st["offset"], st["top"], st["cls"], st["work"])
    return [st["top"], st["cls"]]


def _clip_own(st, ws):
    grads = ws.grad_table(st["grads"])
    ws.grad_sumsq(grads, st["sumsq"], st["work"])
    if st["params"] is None:
        ws.grad_clip(grads, st["sumsq"], st["limit"], st["norm"])
        return [st["norm"]] + st["flat_g"]
    ws.grad_clip_sgd(ws.grad_table(st["params"]), grads, st["sumsq"], st["limit"], st["lr"], st["norm"])
    return [st["norm"]] + st["flat_p"]


PLAIN = {"norm": _norm, "back": _back, "pack": lambda st: list(_mx4(st["W"])), "w4": _w4, "clip": _clip}
OWN = {"norm": _norm_own, "back": _back_own, "pack": _pack_own, "w4": _w4_own, "clip": _clip_own}


def run(st):
    if own:
        from paper_2011_09208_amd import binding as ws
        return OWN[st["kind"]](st, ws)
    return PLAIN[st["kind"]](st)


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _stream(B, D, g):
    """Hidden states: a spread that differs from row to row and a few features that stand out, as they do in trained models."""
    h = torch.empty((B, D), device="cuda").normal_(generator=g)
    rows = torch.empty((B, 1), device="cuda").uniform_(0.5, 4.0, generator=g)
    features = 1.0 + 7.0 * (torch.rand(D, generator=g, device="cuda") < 0.02)
    return h * rows * features


def _gamma(D, g):
    return torch.empty(D, device="cuda").normal_(1.0, 0.2, generator=g)


def _shapes(case):
    """(rows, columns, type) of every gradient: the layer's W and bias, its norm's gamma, and the trunk's blocks of four square
    matrices, two that widen and narrow fourfold, and two gammas."""
    D = case["D"]
    head = [(case["head"], D, torch.bfloat16), (1, case["head"], torch.float32), (1, D, torch.float32)]
    block = [(D, D, torch.bfloat16)] * 4 + [(4 * D, D, torch.bfloat16), (D, 4 * D, torch.bfloat16)] + [(1, D, torch.float32)] * 2
    return head + block * case["blocks"]


def _cut(flat, shapes):
    """Views of the flat buffers, one for each shape, as a bucketed all-reduce keeps its gradients."""
    at, views = {t: 0 for t in flat}, []
    for rows, cols, t in shapes:
        v = flat[t][at[t]:at[t] + rows * cols]
        views.append(v.view(rows, cols) if rows > 1 else v)
        at[t] += rows * cols
    return views


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    kind = case["kind"]
    st = dict(kind=kind)
    if kind in ("norm", "back"):
        B, D = case["B"], case["D"]
        st["gamma"] = _gamma(D, g)
        stream = TYPES.get(case["res"], torch.bfloat16)
        if kind == "norm":
            st.update(out=case["out"], x=torch.empty((B, D), device=dev).normal_(generator=g).to(torch.bfloat16), residual=None, h=None)
            if case["res"] != "none":
                st.update(residual=_stream(B, D, g).to(stream), h=torch.empty((B, D), device=dev, dtype=stream))
            st["y"] = torch.empty((B, D), device=dev, dtype=torch.bfloat16 if case["out"] == "bf16" else torch.uint8)
            if case["out"] == "bf16":
                st["rstd"] = torch.empty(B, device=dev)
            else:
                st["y_scales"] = torch.empty((B, D // 32), device=dev, dtype=torch.uint8)
            return st
        h = _stream(B, D, g).to(stream)
        st.update(h=h, rstd=torch.rsqrt(h.float().square().mean(1) + EPS), dY=torch.empty((B, D), device=dev).normal_(0.0, 1e-3, generator=g),
                  dres=torch.empty((B, D), device=dev).normal_(0.0, 1e-3, generator=g).to(stream) if case["through"] else None,
                  dh=torch.empty((B, D), device=dev, dtype=stream), dgamma=torch.empty(D, device=dev),
                  work=torch.empty(64 << 20, device=dev, dtype=torch.uint8))
        return st
    if kind in ("pack", "w4"):
        C, D = case["C"], case["D"]
        W = torch.empty((C, D), device=dev, dtype=torch.bfloat16).normal_(0.0, 0.02, generator=g)
        if kind == "pack":
            st.update(W=W, W4=torch.empty((C, D // 2), device=dev, dtype=torch.uint8),
                      W_scales=torch.empty((C, D // 32), device=dev, dtype=torch.uint8))
            return st
        B = case["B"]
        st["W4"], st["W_scales"] = _mx4(W)
        X = torch.empty((B, D), device=dev).normal_(generator=g) * _gamma(D, g)
        if case["x"] == "mx8":
            q, st["X_scales"] = _mx8(X)
            st["X"] = q
        else:
            st.update(X=X.to(torch.bfloat16), X_scales=None)
        st.update(out=case["out"], bias=torch.empty(C, device=dev).normal_(0.0, 0.1, generator=g) if case["bias"] else None)
        if case["out"] == "logits":
            st["Z"] = torch.empty((B, (C + 3) // 4 * 4), device=dev)[:, :C]
        else:
            st.update(offset=C, top=torch.empty(B, device=dev), cls=torch.empty(B, device=dev, dtype=torch.int32),
                      work=torch.empty(64 << 20, device=dev, dtype=torch.uint8))
        return st
    shapes = _shapes(case)
    many = {t: sum(r * c for r, c, u in shapes if u == t) for t in (torch.bfloat16, torch.float32)}
    # gradients of a mean loss: small, and of a scale that differs from tensor to tensor
    flat = {t: torch.empty(n, device=dev, dtype=t).normal_(0.0, 1e-3, generator=g) for t, n in many.items()}
    st["grads"] = _cut(flat, shapes)
    sizes = torch.rand(len(shapes), generator=g, device=dev).mul_(3.0).exp_()
    for v, k in zip(st["grads"], sizes):
        v.mul_(k)
    norm = math.sqrt(sum(float(torch.linalg.vector_norm(v, dtype=torch.float64)) ** 2 for v in st["grads"]))
    st.update(flat_g=list(flat.values()), params=None, limit=case["limit"] * norm, lr=0.05, sumsq=torch.empty(1, device=dev, dtype=torch.float64),
              norm=torch.empty(1, device=dev), work=torch.empty(1 << 20, device=dev, dtype=torch.uint8))
    if case["sgd"]:
        flat_p = {t: torch.empty(n, device=dev, dtype=t).normal_(0.0, 0.02, generator=g) for t, n in many.items()}
        st.update(params=_cut(flat_p, shapes), flat_p=list(flat_p.values()))
    return st


def work(case):
    kind, D = case["kind"], case["D"]
    if kind == "norm":
        B, r = case["B"], {"none": 0, "bf16": 2, "fp32": 4}[case["res"]]
        y = 2.0 * D + 4 if case["out"] == "bf16" else D + D / 32
        return {"bytes": B * (2.0 * D + 2 * r * D + y) + 4.0 * D, "flops": 5.0 * B * D}
    if kind == "back":
        B, r = case["B"], {"bf16": 2, "fp32": 4}[case["res"]]
        return {"bytes": B * (4.0 * D + (3 if case["through"] else 2) * r * D + 4) + 8.0 * D, "flops": 9.0 * B * D}
    if kind == "pack":
        return {"bytes": case["C"] * D * (2.0 + 0.5 + 1 / 32), "flops": 2.0 * case["C"] * D}
    if kind == "w4":
        B, C = case["B"], case["C"]
        x = B * D * (2.0 if case["x"] == "bf16" else 1 + 1 / 32)
        out = 4.0 * B * C if case["out"] == "logits" else 8.0 * B
        return {"bytes": C * D * (0.5 + 1 / 32) + x + (4.0 * C if case["bias"] else 0) + out, "flops": 2.0 * B * C * D}
    once = sum(float(r) * c * (2 if t == torch.bfloat16 else 4) for r, c, t in _shapes(case))
    n = sum(float(r) * c for r, c, t in _shapes(case))
    if case["sgd"]:                                            # gradients and weights in, weights out
        return {"bytes": 3 * once + 4, "flops": 5.0 * n}
    return {"bytes": (2 if case["limit"] < 1 else 1) * once + 4, "flops": (3.0 if case["limit"] < 1 else 2.0) * n}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------

def _exact_values4(codes, s):
    """A sign, two bits of exponent (0: subnormal) and one of fraction."""
    c = torch.stack((codes % 16, codes // 16), 2).reshape(codes.shape[0], -1)
    e, m = (c // 2) % 4, (c % 2).double()
    v = torch.where(e == 0, m / 2, (1 + m / 2) * torch.exp2((e - 1.0).double())) * (1 - 2 * (c // 8).double())
    return v * torch.exp2(s.double() - 127).repeat_interleave(32, 1)


def _exact_round8(v):
    """The nearest e4m3 value, ties to even: steps of an eighth of the power of two below, at least 2^-9."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(v / step) * step


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "pack":
        return None                                            # codes: every bit of them is determined, they have to be equal
    if kind == "norm":
        h = st["x"].double()
        if st["residual"] is not None:
            # what the stream stores is rounded: the norm is of what it holds
            h = (h + st["residual"].double()).to(st["residual"].dtype).double()
        rstd = 1 / torch.sqrt((h * h).sum(1) / case["D"] + EPS)
        y = h * rstd[:, None] * st["gamma"].double()
        out = [] if st["h"] is None else [h]
        if case["out"] == "bf16":
            return out + [y, rstd]
        blocks = y.reshape(case["B"], -1, 32)
        top = blocks.abs().max(2).values
        s = torch.exp2(torch.ceil(torch.log2(top / 448)).clamp(min=-127.0))
        return out + [_exact_round8(blocks / s[:, :, None]).reshape(case["B"], -1), s]
    if kind == "back":
        h, dy, gamma, rstd = st["h"].double(), st["dY"].double(), st["gamma"].double(), st["rstd"].double()[:, None]
        c = (dy * gamma * h).sum(1, keepdim=True) / case["D"]
        dh = rstd * dy * gamma - rstd ** 3 * c * h
        if st["dres"] is not None:
            dh = dh + st["dres"].double()
        return [dh, (dy * h * rstd).sum(0)]
    if kind == "w4":
        X = st["X"].double()
        if case["x"] == "mx8":
            X = X * torch.exp2(st["X_scales"].double() - 127).repeat_interleave(32, 1)
        z = torch.mm(X, _exact_values4(st["W4"], st["W_scales"]).t().contiguous())
        if st["bias"] is not None:
            z = z + st["bias"].double()
        return [z] if case["out"] == "logits" else [z.max(1).values, None]
    norm = torch.sqrt(sum((v.double() ** 2).sum() for v in st["grads"]))
    scale = min(1.0, st["limit"] / float(norm))
    if case["sgd"]:
        flat = [p.double() - st["lr"] * scale * v.double() for p, v in zip(st["flat_p"], st["flat_g"])]
    else:
        flat = [v.double() * scale for v in st["flat_g"]]
    return [norm.reshape(1)] + flat
