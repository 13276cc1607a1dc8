"""The operators around the quantised layer of a decoder block, over the sizes,
data types and options in use: the layer with bias, activation (gated or not)
and residual in its epilogue, the router of a mixture of experts, the layer
grouped by expert, and the combination of the experts' rows.

The kinds of call:

* ``layer``    the whole modality-aware layer (smoothing, per-token int8
               quantisation, shared weight, rank-r compensation), then bias,
               activation, the product of gate and up channels, residual.
* ``route``    the k best experts of every token, their weights, and the
               choices sorted by expert.
* ``experts``  the modality-aware layer with a weight and factors per expert,
               over the rows sorted by expert.
* ``combine``  a token's expert rows, weighted and summed, onto the residual.

``run`` makes the framework's calls where ``own`` is true, else the same
mathematics in elementary torch operations.  ``exact`` is the definition in 64
bits.  ``work`` counts what a call cannot do without: each input read once,
each output written once, and the multiply-adds of its products.

A gated layer's weight holds gate channel i at row 2 i and up channel i at row
2 i + 1.  A 4-bit weight is packed two codes a byte: byte b of a 4-byte word
holds code b of its eight in the low half and code b + 4 in the high half.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
TEXT_RANGE, RANGES = 1.0, (1.0, 30.0, 2.0, 5.0)      # row scale by modality id
EPS = 1e-5


def _layer(name, T, K, N, rank, mods, act="none", gated=False, bias=False, residual=False,
           io="bf16", bits=8):
    return dict(name=name, kind="layer", T=T, K=K, N=N, rank=rank, mods=mods, act=act, gated=gated,
                bias=bias, residual=residual, io=io, bits=bits)


def _experts(name, T, E, top_k, K, N, rank, mods, act="none", gated=False, bias=False, gather=True,
             io="bf16", bits=8):
    return dict(name=name, kind="experts", T=T, E=E, top_k=top_k, K=K, N=N, rank=rank, mods=mods,
                act=act, gated=gated, bias=bias, gather=gather, io=io, bits=bits)


def listed():
    return [
        # decoding one sequence: the joint q/k/v projection with its bias
        _layer("layer_t1_3584_4608_bias", 1, 3584, 4608, 64, 2, bias=True),
        # decoding 64 sequences: the down projection from a 4-bit weight,
        # onto the residual stream
        _layer("layer_w4_t64_18944_3584_residual", 64, 18944, 3584, 64, 2, residual=True, bits=4),
        # an fp32 encoder block of odd length and width: bias, GELU, residual
        _layer("layer_fp32_t333_1040_2000_gelu", 333, 1040, 2000, 16, 2, act="gelu", bias=True,
               residual=True, io="f32"),
        # prefill of an image-text prompt: gate and up projections in one
        # product, the gated activation in its epilogue
        _layer("layer_t4096_3584_37888_gated", 4096, 3584, 37888, 64, 2, act="silu", gated=True),
        # routing a decode batch of four sequences
        dict(name="route_t4_e64_k8", kind="route", T=4, E=64, top_k=8, io="bf16", norm=True,
             masked=0.0),
        # routing a long prompt, one row in sixteen padding
        dict(name="route_t8192_e128_k8", kind="route", T=8192, E=128, top_k=8, io="f32", norm=True,
             masked=1 / 16),
        # decoding one token: eight experts' gate and up weights are streamed
        _experts("experts_t1_e64_k8_2048_2048_gated", 1, 64, 8, 2048, 2048, 32, 2, act="silu",
                 gated=True),
        # decoding 32 sequences: the experts' down projection from 4-bit weights
        _experts("experts_w4_t32_e64_k8_1024_2048", 32, 64, 8, 1024, 2048, 32, 2, gather=False,
                 bits=4),
        # fp32, sizes that fill no tile, biases, GELU (tanh form)
        _experts("experts_fp32_t333_e10_k3_1040_720_gelu", 333, 10, 3, 1040, 720, 16, 3,
                 act="gelu_tanh", bias=True, io="f32"),
        # prefill: 32768 rows over 64 experts, gate and up in one product
        _experts("experts_t4096_e64_k8_2048_2816_gated", 4096, 64, 8, 2048, 2816, 32, 2,
                 act="silu", gated=True),
        # the end of the block while decoding 16 sequences
        dict(name="combine_t16_k8_2048", kind="combine", T=16, top_k=8, N=2048, io="bf16",
             residual=True, masked=0.0),
        # the end of the block for a prompt, some tokens with fewer experts
        dict(name="combine_t4096_k8_2048", kind="combine", T=4096, top_k=8, N=2048, io="bf16",
             residual=True, masked=1 / 16),
    ]


_MOST = 4096 * 3584 * 37888          # multiply-adds of the largest listed call
_MOST_WEIGHT = 64 * 2048 * 2816      # codes of the largest listed set of experts


def _log(rng, lo, hi, unit=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(unit, int(round(v / unit)) * unit)


def draw(rng):
    """One more case: a layer or a set of experts mostly."""
    kind = rng.choice(["layer"] * 3 + ["experts"] * 3 + ["route", "combine"])
    io = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "route":
        E = rng.randint(2, 256)
        return dict(kind=kind, T=_log(rng, 1, 8192), E=E, top_k=rng.randint(1, min(E, 8)), io=io,
                    norm=rng.random() < 0.7, masked=rng.choice([0.0, 0.0, 0.1]))
    if kind == "combine":
        return dict(kind=kind, T=_log(rng, 1, 4096), top_k=rng.randint(1, 8),
                    N=_log(rng, 256, 2048, 16), io=io, residual=rng.random() < 0.7,
                    masked=rng.choice([0.0, 0.0, 0.1]))
    bits = 4 if rng.random() < 0.3 else 8
    mods = rng.choice([1, 2, 2, 3])
    rank = 0 if mods == 1 else rng.choice([16, 32, 64, 64])
    gated = rng.random() < 0.5
    act = rng.choice(["silu", "gelu", "gelu_tanh"]) if gated else \
        rng.choice(["none", "none", "silu", "gelu", "gelu_tanh"])
    unit = 64 if bits == 4 else 16
    bias = rng.random() < 0.4
    if kind == "layer":
        T, K = _log(rng, 1, 4096), _log(rng, 512, 18944, unit)
        if rng.random() < 0.25:
            T = _log(rng, 1, 16)                          # decoding
        N = _log(rng, 256, 37888, 32)
        while T * K * N > _MOST or K * N > 3584 * 37888:
            K, N = max(512, K // 2 // unit * unit), max(256, N * 3 // 4 // 32 * 32)
        if io == "f32":
            T = min(T, 1024)
        return dict(kind=kind, T=T, K=K, N=N, rank=rank, mods=mods, act=act, gated=gated, bias=bias,
                    residual=rng.random() < 0.5, io=io, bits=bits)
    E = _log(rng, 4, 64)
    top_k = rng.randint(1, min(E, 8))
    T, K, N = _log(rng, 1, 4096), _log(rng, 256, 4096, unit), _log(rng, 256, 4096, 32)
    if rng.random() < 0.3:
        T = _log(rng, 1, 32)
    while E * K * N > _MOST_WEIGHT:
        K, N = max(256, K // 2 // unit * unit), max(256, N * 3 // 4 // 32 * 32)
    if io == "f32":
        T = min(T, 1024)
    return dict(kind=kind, T=T, E=E, top_k=top_k, K=K, N=N, rank=rank, mods=mods, act=act,
                gated=gated, bias=bias, gather=rng.random() < 0.6, io=io, bits=bits)


# ------------------------------------------------------------------ inputs
def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * int(seed) + salt)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _dtype(io):
    return torch.bfloat16 if io == "bf16" else torch.float32


def _modality(g, T, mods):
    """Runs of tokens of one modality: 64 to 512 tokens in a prompt, shorter
    ones in a decode batch."""
    if mods == 1:
        return torch.zeros(T, device=DEV, dtype=torch.int32)
    t = torch.arange(T, device=DEV)
    if T <= 256:
        length = torch.randint(1, max(2, T // 4 + 1), (2 * T + 2,), generator=g, device=DEV)
    else:
        length = torch.randint(64, 513, (T // 64 + 2,), generator=g, device=DEV)
    start = torch.randint(0, mods, (1,), generator=g, device=DEV)
    run_of = torch.searchsorted(torch.cumsum(length, 0), t, right=True)
    return ((run_of + start) % mods).to(torch.int32)


def _activations(g, rows, K, modality, io):
    """Normal rows scaled by modality, one channel in a hundred an outlier."""
    x = _randn(g, rows, K)
    scale = torch.tensor(RANGES, device=DEV)[modality.long()]
    out = torch.randperm(K, generator=g, device=DEV)[:max(1, K // 100)]
    x *= scale[:, None]
    x[:, out] *= 20.0
    return x.to(_dtype(io))


def _inv_smooth(g, x, modality, mods):
    """Reciprocal smoothing factors sqrt(range of x / range of w)."""
    K = x.shape[1]
    wmax = (4.0 / math.sqrt(K)) * (0.8 + 0.4 * torch.rand((K,), generator=g, device=DEV))
    r = torch.zeros((mods, K), device=DEV)
    for m in range(mods):
        masked = torch.where((modality == m)[:, None], x.abs(), torch.zeros_like(x))
        r[m] = masked.amax(0).float()
    return (1.0 / torch.sqrt(r.clamp(min=EPS) / wmax)).contiguous()


def _codes(g, rows, K, bits):
    """Codes of normal weights, the largest of a channel at the last code
    (packed two a byte for 4 bits)."""
    top = 127 if bits == 8 else 7
    out = torch.empty((rows, K * bits // 8), device=DEV,
                      dtype=torch.int8 if bits == 8 else torch.uint8)
    for i in range(0, rows, 8192):
        n = min(8192, rows - i)
        c = (_randn(g, n, K) * (top / 4.0)).round_().clamp_(-top, top).to(torch.int8)
        if bits == 4:
            w = c.view(n, K // 8, 2, 4).to(torch.int16) & 15
            c = (w[:, :, 0] | (w[:, :, 1] << 4)).to(torch.uint8).reshape(n, K // 2)
        out[i:i + n] = c
    return out


def _unpacked(wq, bits):
    """The codes as float32 [rows][K]."""
    if bits == 8:
        return wq.float()
    b = wq.view(wq.shape[0], -1, 1, 4).to(torch.int16)
    v = torch.cat([b & 15, b >> 4], dim=2)
    return torch.where(v > 7, v - 16, v).reshape(wq.shape[0], -1).float()


def _logits(g, T, E, io, masked):
    """Router outputs: normal, each expert with its own offset in a prompt;
    padding rows hold the lowest value throughout."""
    l = _randn(g, T, E)
    if T >= 64:
        l += 0.5 * _randn(g, 1, E)
    if masked:
        pad = torch.rand((T,), generator=g, device=DEV) < masked
        l = torch.where(pad[:, None], torch.full_like(l, -math.inf), l)
    return l.to(_dtype(io))


def _routed(logits, top_k, norm, modality=None):
    """The router in elementary operations: the k largest finite logits of a
    row (the first of equals first), softmax weights over them (norm) or over
    all experts, and the choices in stable order of expert."""
    T, E = logits.shape
    l = logits.float()
    l = torch.where(torch.isnan(l), torch.full_like(l, -math.inf), l)
    v, ids = torch.sort(l, dim=1, descending=True, stable=True)
    top = v[:, :1]
    p = torch.where(v == top, torch.ones_like(v), torch.exp(v - top))
    p = torch.where(v == -math.inf, torch.zeros_like(p), p)
    total = (p[:, :top_k] if norm else p).sum(1, keepdim=True)
    live = v[:, :top_k] > -math.inf
    w = torch.where(live, p[:, :top_k] / torch.where(total > 0, total, torch.ones_like(total)),
                    torch.zeros_like(p[:, :top_k]))
    ids = torch.where(live, ids[:, :top_k], torch.full_like(ids[:, :top_k], -1))
    flat = torch.where(live, ids, torch.full_like(ids, E)).reshape(-1)
    key, order = torch.sort(flat, stable=True)
    edges = torch.arange(E + 1, device=logits.device)
    offsets = torch.searchsorted(key, edges).to(torch.int32)
    used = key < E
    rows = torch.where(used, order // top_k, torch.full_like(order, -1)).to(torch.int32)
    slots = torch.empty_like(order)
    slots[order] = torch.arange(T * top_k, device=logits.device)
    slots = torch.where(live, slots.view(T, top_k), torch.full_like(ids, -1)).to(torch.int32)
    out = dict(experts=ids.to(torch.int32), weights=w, offsets=offsets, rows=rows, slots=slots)
    if modality is not None:
        out["modality"] = torch.where(used, modality[rows.clamp(min=0).long()],
                                      torch.zeros_like(rows))
    return out


def _layer_inputs(g, c, experts, rows):
    """Weights, factors and biases of `experts` layers (a leading axis where
    there is more than one) and the rows' operands."""
    K, N, E, mods, r = c["K"], c["N"], experts or 1, c["mods"], c["rank"]
    lead = (E,) if experts else ()
    wq = _codes(g, E * N, K, c["bits"])
    top = 127 if c["bits"] == 8 else 7
    scale = (4.0 / top / math.sqrt(K)) * (0.75 + 0.5 * torch.rand((E * N,), generator=g, device=DEV))
    s = dict(wq=wq.view(*lead, N, -1), scale=scale.view(*lead, N), l_down=None, r_up=None,
             bias=None)
    if r and mods > 1:
        lr = _dtype(c["io"])
        s["l_down"] = (_randn(g, *lead, mods - 1, r, K) / math.sqrt(K)).to(lr)
        s["r_up"] = (_randn(g, *lead, mods - 1, N, r) * 0.2).to(lr)
    if c["bias"]:
        s["bias"] = 0.5 * _randn(g, *lead, N)
    s["x"] = _activations(g, rows.shape[0], K, rows, c["io"])
    s["inv"] = _inv_smooth(g, s["x"], rows, mods)
    s["mod"] = rows
    return s


def prepare(case, seed):
    c = case
    kind, T = c["kind"], c["T"]
    g = _gen(seed, 17 * c.get("K", c.get("N", c.get("E", 0))) + T)
    if kind == "route":
        s = dict(logits=_logits(g, T, c["E"], c["io"], c["masked"]), mod=_modality(g, T, 3))
    elif kind == "combine":
        # rows in the order of their experts, some choices without one
        n = T * c["top_k"]
        perm = torch.randperm(n, generator=g, device=DEV).to(torch.int32).view(T, c["top_k"])
        gone = torch.rand((T, c["top_k"]), generator=g, device=DEV) < c["masked"]
        w = torch.softmax(_randn(g, T, c["top_k"]), 1)
        s = dict(d=_randn(g, n, c["N"]).to(_dtype(c["io"])),
                 slots=torch.where(gone, torch.full_like(perm, -1), perm),
                 weights=torch.where(gone, torch.zeros_like(w), w),
                 res=_randn(g, T, c["N"]).to(_dtype(c["io"])) if c["residual"] else None)
    elif kind == "layer":
        s = _layer_inputs(g, c, 0, _modality(g, T, c["mods"]))
        width = c["N"] // 2 if c["gated"] else c["N"]
        s["res"] = _randn(g, T, width).to(_dtype(c["io"])) if c["residual"] else None
    else:
        mod = _modality(g, T, c["mods"])
        r = _routed(_logits(g, T, c["E"], "f32", 0.0), c["top_k"], True, mod)
        s = _layer_inputs(g, c, c["E"], mod if c["gather"] else r["modality"])
        s["offsets"] = r["offsets"]
        s["rows"] = r["rows"] if c["gather"] else None
    s["case"] = c
    if own:
        _handles(s)
    elif kind == "experts":
        s["edges"] = s["offsets"].tolist()                # the groups' places, for the loop over them
    return s


def _handles(s):
    """What a serving loop keeps: the layer, its output and the bound call."""
    from paper_2603_04800_amd import ops
    c = s["case"]
    if c["kind"] == "route":
        s["call"] = ops.bind_route_experts(s["logits"], c["top_k"], renormalize=c["norm"],
                                           modality=s["mod"])
    elif c["kind"] == "combine":
        s["call"] = ops.bind_combine_experts(s["d"], s["slots"], s["weights"], residual=s["res"])
    elif c["kind"] == "layer":
        lin = ops.Linear(s["inv"], s["wq"], s["scale"], s["l_down"], s["r_up"])
        s["call"] = lin.bind_fused(s["x"], s["mod"], bias=s["bias"], act=c["act"], gated=c["gated"],
                                   residual=s["res"])
    else:
        lin = ops.ExpertLinear(s["inv"], s["wq"], s["scale"], s["l_down"], s["r_up"],
                               bias=s["bias"], act=c["act"], gated=c["gated"])
        s["call"] = lin.bind(s["x"], s["mod"], s["offsets"], rows=s["rows"])


# ------------------------------------------------------------------ a pass
def _quantised(x, mod, inv):
    """The smoothed rows, their int8 codes (as float32) and steps."""
    xs = x.float() * inv[mod.long()]
    amax = xs.abs().amax(1)
    ok = amax > 0
    top = torch.full_like(amax, 127.0)                    # (a scalar divisor is multiplied by
    dx = torch.where(ok, amax / top, torch.zeros_like(amax))     # its rounded reciprocal)
    rq = torch.where(ok, top / amax, torch.zeros_like(amax))
    return xs, torch.round(xs * rq[:, None]).clamp(-127, 127), dx


def _activated(z, act, gated):
    """act(z), or act(gate) * up for channels in pairs."""
    a = z[:, 0::2] if gated else z
    if act == "silu":
        h = a / (1.0 + torch.exp(-a))
    elif act == "gelu":
        h = 0.5 * a * (1.0 + torch.erf(a * (1.0 / math.sqrt(2.0))))
    elif act == "gelu_tanh":
        h = 0.5 * a * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (a + 0.044715 * (a * a * a))))
    else:
        h = a
    return h * z[:, 1::2] if gated else h


def _plain_rows(xs, q, dx, mod, wq, scale, l_down, r_up, bias, c):
    """The layer on quantised rows, up to the activation."""
    y = q @ _unpacked(wq, c["bits"]).T
    y = y * dx[:, None] * scale[None, :]
    if l_down is not None:
        for m in range(1, c["mods"]):
            u = torch.where((mod == m)[:, None], xs, torch.zeros_like(xs)) @ l_down[m - 1].float().T
            y += u @ r_up[m - 1].float().T
    if bias is not None:
        y += bias[None, :]
    return _activated(y, c["act"], c["gated"])


def _plain(s):
    c = s["case"]
    if c["kind"] == "route":
        return _routed(s["logits"], c["top_k"], c["norm"], s["mod"])
    if c["kind"] == "combine":
        picked = s["d"][s["slots"].clamp(min=0).long()].float()
        w = torch.where(s["slots"] >= 0, s["weights"], torch.zeros_like(s["weights"]))
        y = (picked * w[:, :, None]).sum(1)
        if s["res"] is not None:
            y = y + s["res"].float()
        return y.to(s["d"].dtype)
    xs, q, dx = _quantised(s["x"], s["mod"], s["inv"])
    if c["kind"] == "layer":
        y = _plain_rows(xs, q, dx, s["mod"], s["wq"], s["scale"], s["l_down"], s["r_up"], s["bias"], c)
        if s["res"] is not None:
            y = y + s["res"].float()
        return y.to(s["x"].dtype)
    width = c["N"] // 2 if c["gated"] else c["N"]
    y = torch.empty((c["T"] * c["top_k"], width), device=DEV, dtype=s["x"].dtype)
    rows = s["rows"].long() if s["rows"] is not None else None
    for e in range(c["E"]):
        a, b = s["edges"][e], s["edges"][e + 1]
        if a == b:
            continue
        at = rows[a:b] if rows is not None else slice(a, b)
        y[a:b] = _plain_rows(xs[at], q[at], dx[at], s["mod"][at], s["wq"][e], s["scale"][e],
                             s["l_down"][e] if s["l_down"] is not None else None,
                             s["r_up"][e] if s["r_up"] is not None else None,
                             s["bias"][e] if s["bias"] is not None else None, c).to(y.dtype)
    return y


def run(s):
    if not own:
        return _plain(s)
    out = s["call"]()
    if s["case"]["kind"] == "route":
        return dict(experts=out.experts, weights=out.weights, offsets=out.offsets, rows=out.rows,
                    slots=out.slots, modality=out.modality)
    return out


# ------------------------------------------------------------------ work
def _hit(c):
    """Experts that at least one of the tokens' choices reaches."""
    return c["E"] * (1.0 - (1.0 - c["top_k"] / c["E"]) ** c["T"])


def work(case):
    c = case
    T = c["T"]
    xb = 2 if c["io"] == "bf16" else 4
    if c["kind"] == "route":
        # logits and modalities in; ids, weights, rows, slots, modalities out
        return dict(bytes=T * c["E"] * xb + 4 * T + T * c["top_k"] * 20 + 4 * (c["E"] + 1),
                    flops=3 * T * c["E"])
    if c["kind"] == "combine":
        n = T * c["top_k"] * (1.0 - c["masked"])
        return dict(bytes=int(n * c["N"] * xb) + T * c["top_k"] * 8 +
                    T * c["N"] * xb * (2 if c["residual"] else 1),
                    flops=int(2 * n * c["N"]))
    K, N, mods = c["K"], c["N"], c["mods"]
    r = c["rank"] if mods > 1 else 0
    width = N // 2 if c["gated"] else N
    if c["kind"] == "layer":
        rows, sets, x_rows = T, 1, T
        extra = T * width * xb if c["residual"] else 0
    else:
        rows, sets = T * c["top_k"], _hit(c)
        x_rows = T if c["gather"] else rows
        extra = 4 * (c["E"] + 1) + (4 * rows if c["gather"] else 0)
    other = rows * (mods - 1) // mods
    weight = sets * (N * K * c["bits"] // 8 + 4 * N * (2 if c["bias"] else 1))
    factors = min(sets * (mods - 1), rows) * r * (K + N) * xb
    byte = x_rows * (K * xb + 4) + mods * K * 4 + weight + factors + rows * width * xb + extra
    return dict(bytes=int(byte), flops=2 * rows * K * N + 2 * other * r * (K + N))


# ------------------------------------------------------------------ 64 bits
def _exact_activated(z, act, gated):
    a = z[:, 0::2] if gated else z
    if act == "silu":
        a = a * torch.sigmoid(a)
    elif act == "gelu":
        a = a * 0.5 * torch.special.erfc(-a / math.sqrt(2.0))
    elif act == "gelu_tanh":                              # (1 + tanh t) / 2 = sigmoid(2 t)
        a = a * torch.sigmoid(math.sqrt(8.0 / math.pi) * a * (1.0 + 0.044715 * a ** 2))
    return a * z[:, 1::2] if gated else a


def _exact_rows(s, c, at, e):
    """Rows `at` of the input through layer e (None: the only one).  The codes
    are what the rounding of the quantiser makes them: products and quotients
    of 32-bit numbers formed in 64 bits and rounded to 32 once."""
    pick = (lambda t: t) if e is None else (lambda t: t[e])
    mod = s["mod"][at].long()
    xs = (s["x"][at].double() * s["inv"][mod].double()).float().double()
    amax = xs.abs().max(1).values
    safe = torch.where(amax > 0, amax, torch.ones_like(amax))
    dx = (amax / 127.0).float().double()
    q = ((xs * (127.0 / safe).float().double()[:, None]).float().round().clamp(-127, 127)).double()
    w = pick(s["wq"])
    if c["bits"] == 4:
        word = w.to(torch.int64).view(w.shape[0], -1, 4)
        code = torch.stack([(word[:, :, j % 4] >> (4 * (j // 4))) & 15 for j in range(8)], 2)
        w = ((code + 8) % 16 - 8).reshape(w.shape[0], -1)
    y = (q @ w.double().T.contiguous()) * dx[:, None] * pick(s["scale"]).double()
    if s["l_down"] is not None:
        for m in range(1, c["mods"]):
            i = torch.nonzero(mod == m).flatten()
            if i.numel():
                u = xs[i] @ pick(s["l_down"])[m - 1].double().T.contiguous()
                y[i] += u @ pick(s["r_up"])[m - 1].double().T.contiguous()
    if s["bias"] is not None:
        y += pick(s["bias"]).double()
    return _exact_activated(y, c["act"], c["gated"])


def _exact_route(c, s):
    l = s["logits"].double().cpu().numpy()
    mod = s["mod"].cpu().numpy()
    T, E = l.shape
    k = c["top_k"]
    l = np.where(np.isnan(l), -np.inf, l)
    order = np.lexsort((np.broadcast_to(np.arange(E), l.shape), -l), axis=1)[:, :k]
    v = np.take_along_axis(l, order, 1)
    live = v > -np.inf
    with np.errstate(invalid="ignore"):
        p = np.where(l == -np.inf, 0.0, np.exp(l - np.where(live[:, :1], v[:, :1], 0.0)))
    chosen = np.take_along_axis(p, order, 1)
    total = (chosen if c["norm"] else p).sum(1)
    w = np.where(live, chosen / np.where(total > 0, total, 1.0)[:, None], 0.0)
    experts = np.where(live, order, -1)
    rows, slot_mod = np.full(T * k, -1), np.zeros(T * k, np.int64)
    slots, offsets, n = np.full((T, k), -1), np.zeros(E + 1, np.int64), 0
    for e in range(E):
        t, j = np.nonzero(experts == e)
        rows[n:n + len(t)], slot_mod[n:n + len(t)] = t, mod[t]
        slots[t, j] = np.arange(n, n + len(t))
        n += len(t)
        offsets[e + 1] = n
    back = {k_: torch.from_numpy(np.ascontiguousarray(a)).to(DEV) for k_, a in dict(
        experts=experts, offsets=offsets, rows=rows, slots=slots, modality=slot_mod).items()}
    back["weights"] = torch.from_numpy(w).to(DEV)
    return {n_: back[n_] for n_ in ("experts", "weights", "offsets", "rows", "slots", "modality")}


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["kind"] == "route":
        return _exact_route(c, s)
    if c["kind"] == "combine":
        y = s["res"].double() if s["res"] is not None else torch.zeros((c["T"], c["N"]), device=DEV,
                                                                      dtype=torch.float64)
        for j in range(c["top_k"]):
            at, w = s["slots"][:, j].long(), s["weights"][:, j].double()
            here = (at >= 0)[:, None]
            y = y + torch.where(here, w[:, None] * s["d"][at.clamp(min=0)].double(),
                                torch.zeros_like(y))
        return y
    if c["kind"] == "layer":
        y = _exact_rows(s, c, slice(0, c["T"]), None)
        return y + s["res"].double() if s["res"] is not None else y
    edges = s["offsets"].tolist()
    y = torch.zeros((c["T"] * c["top_k"], c["N"] // 2 if c["gated"] else c["N"]), device=DEV,
                    dtype=torch.float64)
    for e in range(c["E"]):
        a, b = edges[e], edges[e + 1]
        if a < b:
            at = s["rows"][a:b].long() if s["rows"] is not None else slice(a, b)
            y[a:b] = _exact_rows(s, c, at, e)
    return y
