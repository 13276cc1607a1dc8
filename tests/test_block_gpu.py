"""The operators around the quantised layer on the GPU, against 64 bits: the
layer's epilogue, routing, the experts' layer, the combination, and all of
them as one block."""
import math

import pytest
import torch

import block_reference as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def ops():
    from paper_2603_04800_amd import ops as o
    return o


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _pack(codes):
    """[..][K] codes in [-7, 7] -> [..][K / 2] bytes."""
    w = codes.to(torch.int16).unflatten(-1, (-1, 2, 4)) & 15
    return (w[..., 0, :] | (w[..., 1, :] << 4)).to(torch.uint8).flatten(-2).contiguous()


class Case:
    """Operands of E layers (0: one, without the axis)."""

    def __init__(self, seed, T, K, N, E=0, rank=0, mods=1, io="bf16", bits=8, bias=False, out_rows=None,
                 width=None, residual=False, lr=None):
        g = _gen(seed)
        lead = (E,) if E else ()
        top = 127 if bits == 8 else 7
        self.x = (_randn(g, T, K) * (1 + 4 * torch.rand((T, 1), generator=g, device="cuda"))).to(DT[io])
        self.mod = torch.randint(0, mods, (T,), generator=g, device="cuda").to(torch.int32)
        self.inv = (0.5 + torch.rand((mods, K), generator=g, device="cuda")).contiguous()
        self.codes = torch.randint(-top, top + 1, (*lead, N, K), generator=g, device="cuda").to(torch.int8)
        self.wq = _pack(self.codes) if bits == 4 else self.codes
        self.scale = (0.5 + torch.rand((*lead, N), generator=g, device="cuda")) * (2.0 / top / math.sqrt(K))
        self.ld = self.ru = self.bias = self.res = None
        if rank and mods > 1:
            t = DT[lr or io]
            self.ld = (_randn(g, *lead, mods - 1, rank, K) / math.sqrt(K)).to(t)
            self.ru = (_randn(g, *lead, mods - 1, N, rank) * 0.2).to(t)
        if bias:
            self.bias = _randn(g, *lead, N)
        if residual:
            self.res = _randn(g, T, width).to(DT[io])


# ------------------------------------------------------------------ the layer's epilogue
LAYERS = [
    # T, K, N, rank, mods, io, bits, act, gated, bias, residual
    (1, 64, 32, 0, 1, "bf16", 8, "none", False, True, False),
    (1, 3584, 4608, 64, 2, "bf16", 8, "none", False, True, True),
    (3, 128, 96, 16, 2, "f32", 8, "silu", True, True, True),
    (5, 80, 48, 16, 2, "bf16", 8, "gelu", False, True, True),          # a small batch with K % 64 != 0
    (16, 8192, 224, 32, 3, "bf16", 8, "gelu", False, True, True),      # decode GEMM, split rows
    (16, 512, 18944, 16, 2, "bf16", 4, "silu", True, False, True),
    (15, 4096, 64, 64, 4, "f32", 4, "gelu_tanh", True, True, False),
    (17, 528, 48, 16, 2, "bf16", 8, "silu", False, True, True),        # 32 x 64 tiles, K % 64 = 16
    (32, 4096, 96, 16, 2, "f32", 8, "gelu", True, True, True),         # split into slices
    (33, 1040, 2000, 16, 2, "f32", 8, "gelu", False, True, True),
    (70, 512, 992, 32, 3, "bf16", 8, "silu", True, True, True),
    (100, 8192, 2048, 16, 2, "bf16", 4, "gelu", True, False, True),    # 32 x 64 tiles in slices
    (48, 6160, 528, 32, 3, "f32", 8, "silu", False, True, True),
    (64, 18944, 512, 64, 2, "bf16", 4, "none", False, False, True),
    (333, 1040, 720, 128, 2, "bf16", 8, "gelu_tanh", False, True, True),
    (300, 768, 13248, 16, 2, "f32", 8, "silu", True, True, False),     # 128 x 128 tiles
    (1000, 640, 4096, 64, 3, "bf16", 8, "silu", True, True, True),
    (2048, 256, 8192, 16, 2, "bf16", 4, "gelu", True, False, True),
    (2500, 192, 8480, 0, 1, "bf16", 8, "silu", True, True, True),      # past the 128 x 128 rounds
    (2304, 320, 6176, 64, 3, "bf16", 8, "gelu_tanh", False, True, True),
]


@pytest.mark.parametrize("T,K,N,rank,mods,io,bits,act,gated,bias,residual", LAYERS)
def test_layer_epilogue(ops, T, K, N, rank, mods, io, bits, act, gated, bias, residual):
    width = N // 2 if gated else N
    c = Case(T + K + N, T, K, N, rank=rank, mods=mods, io=io, bits=bits, bias=bias, width=width,
             residual=residual)
    lin = ops.Linear(c.inv, c.wq, c.scale, c.ld, c.ru)
    got = lin.fused(c.x, c.mod, bias=c.bias, act=act, gated=gated, residual=c.res)
    z, e = ref.layer(c.x, c.mod, c.inv, c.codes, c.scale, c.ld, c.ru, c.bias)
    ref.assert_close(got, *ref.finish(z, e, act, gated, c.res, DT[io]))


@pytest.mark.parametrize("T,K,N,rank,mods,io,lr", [
    # down-projections of fp32 factors and of ranks past 64: batches and rows on
    # both sides of the choice between the two first stages, odd batches
    (17, 64, 64, 16, 2, "f32", "f32"), (1, 1040, 48, 32, 3, "f32", "f32"), (100, 8192, 64, 16, 2, "f32", "f32"),
    (99, 8256, 64, 16, 2, "f32", "f32"), (33, 2048, 96, 64, 2, "bf16", "f32"), (33, 2112, 96, 64, 2, "bf16", "f32"),
    (255, 1040, 272, 48, 4, "f32", "f32"), (257, 1040, 272, 48, 4, "f32", "f32"),
    (301, 4160, 64, 256, 2, "bf16", "bf16"),
    (77, 4096, 80, 80, 3, "f32", "bf16"), (77, 4160, 80, 80, 3, "f32", "bf16"), (2049, 128, 32, 128, 2, "bf16", "bf16"),
    (4097, 64, 48, 256, 2, "f32", "f32"), (301, 18944, 32, 16, 2, "bf16", "f32"),
])
def test_compensations_of_fp32_factors_and_high_ranks(ops, T, K, N, rank, mods, io, lr):
    c = Case(T + K + rank, T, K, N, rank=rank, mods=mods, io=io, lr=lr, bias=True, residual=True, width=N)
    lin = ops.Linear(c.inv, c.wq, c.scale, c.ld, c.ru)
    ws = torch.full((ops.workspace_bytes(T, K, N, rank, mods),), 255, dtype=torch.uint8, device="cuda")  # dirty
    got = lin.fused(c.x, c.mod, bias=c.bias, act="silu", residual=c.res, workspace=ws)
    z, e = ref.layer(c.x, c.mod, c.inv, c.codes, c.scale, c.ld, c.ru, c.bias)
    ref.assert_close(got, *ref.finish(z, e, "silu", False, c.res, DT[io]))
    assert torch.equal(got, lin.fused(c.x, c.mod, bias=c.bias, act="silu", residual=c.res, workspace=ws))


@pytest.mark.parametrize("T,K,N", [(1, 512, 256), (16, 2048, 512), (40, 512, 512), (400, 1024, 4096),
                                   (50, 8192, 528), (128, 18944, 512), (2304, 320, 6176)])
def test_epilogue_of_nothing_is_the_layer(ops, T, K, N):
    c = Case(T, T, K, N, rank=16, mods=2)
    c.mod.zero_()
    lin = ops.Linear(c.inv, c.wq, c.scale, c.ld, c.ru)
    assert torch.equal(lin.fused(c.x, c.mod), lin(c.x, c.mod))


@pytest.mark.parametrize("T", [2, 16, 48, 600])
@pytest.mark.parametrize("gated", [False, True])
def test_residual_in_place(ops, T, gated):
    N = 512
    c = Case(T, T, 512, N, rank=16, mods=2, residual=True, width=N // 2 if gated else N)
    lin = ops.Linear(c.inv, c.wq, c.scale, c.ld, c.ru)
    want = lin.fused(c.x, c.mod, act="silu", gated=gated, residual=c.res)
    buf = c.res.clone()
    got = lin.fused(c.x, c.mod, act="silu", gated=gated, residual=buf, out=buf)
    assert got.data_ptr() == buf.data_ptr() and torch.equal(got, want)


@pytest.mark.parametrize("T,K,N", [(7, 256, 96), (60, 512, 512), (400, 320, 4096), (2500, 192, 8480)])
@pytest.mark.parametrize("xt,yt,lr", [("bf16", "f32", "bf16"), ("f32", "bf16", "f32"), ("bf16", "bf16", "f32")])
def test_mixed_types(ops, T, K, N, xt, yt, lr):
    c = Case(T, T, K, N, rank=32, mods=3, io=xt, lr=lr, bias=True)
    c.mod[::5] = 9                                          # no modality: text
    c.mod[1::7] = -1
    res = _randn(_gen(1), T, N // 2).to(DT[yt])
    lin = ops.Linear(c.inv, c.wq, c.scale, c.ld, c.ru)
    ws = torch.full((ops.workspace_bytes(T, K, N, 32, 3),), 255, dtype=torch.uint8, device="cuda")   # dirty
    out = torch.empty((T, N // 2), dtype=DT[yt], device="cuda")
    got = lin.fused(c.x, c.mod, bias=c.bias, act="gelu_tanh", gated=True, residual=res, out=out, workspace=ws)
    mod = torch.where((c.mod < 0) | (c.mod > 2), torch.zeros_like(c.mod), c.mod)
    z, e = ref.layer(c.x, mod, c.inv, c.codes, c.scale, c.ld, c.ru, c.bias)
    ref.assert_close(got, *ref.finish(z, e, "gelu_tanh", True, res, DT[yt]))


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_activations_over_their_range(ops, act, io):
    # codes of +-127 and steps that put z from -1e6 to 1e6, zeros among them
    K, N, T = 64, 4096, 8
    x = torch.ones((T, K), device="cuda", dtype=DT[io])
    x[3] = 0
    codes = torch.full((N, K), 127, device="cuda", dtype=torch.int8)
    codes[::2] = -127
    scale = (10.0 ** torch.linspace(-9, 3, N, device="cuda")).float()
    scale[:2048] = torch.linspace(0, 15, 2048, device="cuda") / (127 * 64)
    inv, mod = torch.ones((1, K), device="cuda"), torch.zeros(T, device="cuda", dtype=torch.int32)
    got = ops.Linear(inv, codes, scale).fused(x, mod, act=act)
    z, e = ref.layer(x, mod, inv, codes, scale, None, None)
    assert torch.isfinite(got).all() and (got[3] == 0).all()
    ref.assert_close(got, *ref.finish(z, e, act, False, None, DT[io]))


# ------------------------------------------------------------------ routing
def _check_route(ops, logits, k, renorm, mod=None):
    r = ops.route_experts(logits, k, renormalize=renorm, modality=mod)
    experts, weights, offsets, rows, slots = ref.route(logits, k, renorm)
    assert r.experts.tolist() == experts
    assert r.offsets.tolist() == offsets
    assert r.rows.tolist() == rows
    assert r.slots.tolist() == slots
    want = torch.tensor(weights, dtype=torch.float64, device="cuda").view(r.weights.shape)
    # exp of a difference d (rounded once, so off by |d| u) and E sums, one quotient
    spread = logits.double()[logits.double().abs() < math.inf]
    d = float(spread.max() - spread.min()) if spread.numel() else 0.0
    ref.assert_close(r.weights, want, want * ref.U * (2 * d + logits.shape[1] + 8) + 1e-37)
    if mod is not None:
        m = mod.tolist()
        assert r.modality.tolist() == [m[t] if t >= 0 else 0 for t in rows]
    return r


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 2, 1), (1, 64, 8), (4, 64, 8), (31, 10, 3), (33, 65, 16),
                                   (256, 128, 8), (257, 128, 8), (300, 512, 16), (64, 9, 2), (65, 510, 3), (1000, 7, 7), (2049, 60, 4),
                                   (8192, 6, 2), (8225, 13, 2)])
@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_route(ops, T, E, k, io):
    g = _gen(T + E)
    logits = (2 * _randn(g, T, E)).to(DT[io])               # (bf16: ties)
    mod = torch.randint(0, 3, (T,), generator=g, device="cuda").to(torch.int32)
    _check_route(ops, logits, k, renorm=bool(T % 2), mod=mod)


@pytest.mark.parametrize("T", [7, 300])
def test_route_ties_masks_and_extremes(ops, T):
    E, k = 70, 4
    g = _gen(T)
    l = _randn(g, T, E)
    inf = math.inf
    l[0] = 0.0                                              # ties throughout
    l[1] = -inf                                             # nothing left
    l[2] = math.nan
    l[3] = -inf
    l[3, 68] = -3e38                                        # one left, of the lowest value
    l[4, 5] = l[4, 66] = inf                                # infinities share the weight
    l[5, :] = -0.0
    l[5, 1::2] = 0.0                                        # -0 and +0 are a tie
    l[6, :3] = math.nan
    l[6, 3:] = torch.finfo(torch.float32).min
    if T > 64:
        l[64:96] = -inf                                     # a whole group of 32 tokens
    for renorm in (False, True):
        r = ops.route_experts(l, k, renormalize=renorm)
        experts, weights, offsets, rows, slots = ref.route(l, k, renorm)
        assert r.experts.tolist() == experts and r.slots.tolist() == slots
        assert r.rows.tolist() == rows and r.offsets.tolist() == offsets
        assert r.experts[0].tolist() == [0, 1, 2, 3] and r.experts[5].tolist() == [0, 1, 2, 3]
        assert r.experts[3].tolist() == [68, -1, -1, -1] and r.weights[3].tolist() == [1, 0, 0, 0]
        assert r.weights[4].tolist() == [0.5, 0.5, 0, 0] and not r.weights[1:3].any()
        want = torch.tensor(weights, dtype=torch.float64, device="cuda")
        ref.assert_close(r.weights[7:], want[7:], want[7:] * ref.U * (2 * 12 + E + 8) + 1e-37)


def test_route_of_an_empty_batch(ops):
    r = ops.route_experts(torch.empty((0, 8), device="cuda"), 2)
    assert r.offsets.tolist() == [0] * 9 and r.rows.numel() == 0 and r.slots.shape == (0, 2)


# ------------------------------------------------------------------ the experts' layer
def _offsets(counts):
    return torch.tensor([0, *torch.tensor(counts).cumsum(0).tolist()], dtype=torch.int32, device="cuda")


def _check_experts(ops, c, counts, rows, act, gated, io, extra=0):
    """rows: None or the row of x of each slot; extra: slots past the last."""
    E, N = c.scale.shape
    lin = ops.ExpertLinear(c.inv, c.wq, c.scale, c.ld, c.ru, bias=c.bias, act=act, gated=gated)
    n = sum(counts)
    slots = n + extra
    x_rows = rows if rows is not None else torch.arange(slots, device="cuda", dtype=torch.int32)
    out = torch.full((slots, lin.width), 7.25, device="cuda", dtype=DT[io])
    got = lin(c.x, c.mod, _offsets(counts), rows=rows, out=out)
    at = 0
    for e, cnt in enumerate(counts):
        if cnt:
            i = x_rows[at:at + cnt].long()
            z, err = ref.layer(c.x[i], c.mod[i], c.inv, c.codes[e], c.scale[e],
                               c.ld[e] if c.ld is not None else None,
                               c.ru[e] if c.ru is not None else None,
                               c.bias[e] if c.bias is not None else None)
            ref.assert_close(got[at:at + cnt], *ref.finish(z, err, act, gated, None, DT[io]))
        at += cnt
    assert (got[n:] == 7.25).all()                          # rows past the last slot stay


EXPERTS = [
    # counts, T (0: slot order), K, N, rank, mods, io, bits, act, gated, bias
    ([1], 1, 64, 32, 0, 1, "bf16", 8, "none", False, True),
    ([0, 1, 0, 2, 1], 4, 256, 96, 16, 2, "bf16", 8, "silu", True, True),
    ([3, 0, 33, 5, 0, 0, 31, 1, 64, 0], 40, 528, 208, 32, 3, "f32", 8, "gelu", False, True),
    ([16] * 8, 0, 512, 128, 16, 2, "bf16", 4, "silu", True, False),
    ([0] * 70 + [9, 0, 40] + [1] * 60, 30, 192, 64, 16, 2, "bf16", 8, "none", False, False),
    ([130, 0, 1, 257], 200, 320, 288, 80, 2, "bf16", 8, "gelu_tanh", True, True),
    ([500, 20, 400, 0, 129], 0, 448, 416, 64, 4, "bf16", 4, "silu", True, True),
    ([1500, 3], 700, 1040, 160, 16, 2, "f32", 8, "silu", False, True),
    ([0, 0, 0, 700], 300, 512, 512, 256, 2, "f32", 8, "silu", True, False),
    # 256 x 256 tiles: gathered rows, rows in slot order
    ([1500, 0, 601, 33, 1], 800, 192, 3104, 16, 3, "bf16", 8, "silu", True, True),
    ([1500, 0, 601, 33, 1], 0, 192, 3104, 64, 2, "bf16", 4, "gelu", False, True),
    ([1, 1400, 700, 0, 129], 700, 128, 3104, 16, 2, "f32", 8, "gelu_tanh", True, True),
    ([2000], 1999, 64, 4096, 128, 4, "bf16", 8, "none", False, False),
    ([900, 300], 0, 64, 4112, 0, 1, "bf16", 8, "silu", False, True),
    ([0, 0, 4300, 0] + [0] * 3 + [100], 1024, 320, 1440, 48, 2, "bf16", 4, "silu", True, False),
]


@pytest.mark.parametrize("counts,T,K,N,rank,mods,io,bits,act,gated,bias", EXPERTS)
def test_experts(ops, counts, T, K, N, rank, mods, io, bits, act, gated, bias):
    n, E = sum(counts), len(counts)
    c = Case(n + K, T or n, K, N, E=E, rank=rank, mods=mods, io=io, bits=bits, bias=bias)
    rows = None
    if T:
        rows = torch.randint(0, T, (n,), generator=_gen(n), device="cuda").to(torch.int32)
    _check_experts(ops, c, counts, rows, act, gated, io)


@pytest.mark.parametrize("lr,io", [("f32", "bf16"), ("bf16", "f32")])
def test_experts_factor_types(ops, lr, io):
    counts = [5, 0, 40, 2]
    c = Case(3, 30, 256, 96, E=4, rank=32, mods=3, io=io, bias=True, lr=lr)
    rows = torch.randint(0, 30, (47,), generator=_gen(5), device="cuda").to(torch.int32)
    _check_experts(ops, c, counts, rows, "silu", True, io)


def test_experts_leave_rows_past_the_last_slot(ops):
    counts = [4, 0, 9]
    c = Case(1, 20, 128, 64, E=3, rank=16, mods=2)
    rows = torch.cat([torch.randint(0, 20, (13,), generator=_gen(1), device="cuda").to(torch.int32),
                      torch.full((7,), -1, device="cuda", dtype=torch.int32)])
    _check_experts(ops, c, counts, rows, "silu", False, "bf16", extra=7)
    # in slot order, whatever the unused rows of x hold
    c = Case(2, 20, 128, 64, E=3, rank=16, mods=2)
    c.x[13:] = math.nan
    _check_experts(ops, c, counts, None, "silu", True, "bf16", extra=7)


@pytest.mark.parametrize("hit", [{0: 1}, {63: 2, 64: 3}, {511: 40}, {5: 1, 127: 20, 128: 33, 300: 7, 511: 1}])
def test_many_experts(ops, hit):
    counts = [hit.get(e, 0) for e in range(512)]
    n = sum(counts)
    c = Case(n, 50, 64, 96, E=512, rank=16, mods=2, bias=True)
    rows = torch.randint(0, 50, (n,), generator=_gen(n), device="cuda").to(torch.int32)
    _check_experts(ops, c, counts, rows, "silu", True, "bf16")


def test_experts_mixed_types_and_modalities(ops):
    c = Case(9, 40, 256, 96, E=3, rank=16, mods=4, io="bf16", lr="f32")
    c.mod[::3] = 77                                         # no modality: text
    rows = torch.randint(0, 40, (90,), generator=_gen(9), device="cuda").to(torch.int32)
    got = ops.ExpertLinear(c.inv, c.wq, c.scale, c.ld, c.ru)(c.x, c.mod, _offsets([50, 0, 40]), rows=rows,
                                                              out_dtype=torch.float32)
    mod = torch.where(c.mod > 3, torch.zeros_like(c.mod), c.mod)
    for e, a, b in ((0, 0, 50), (2, 50, 90)):
        i = rows[a:b].long()
        z, err = ref.layer(c.x[i], mod[i], c.inv, c.codes[e], c.scale[e], c.ld[e], c.ru[e])
        ref.assert_close(got[a:b], *ref.finish(z, err, "none", False, None, torch.float32))


@pytest.mark.parametrize("n", [6, 700])
def test_rows_and_offsets_outside_their_range_are_clamped(ops, n):
    c = Case(n, 20, 128, 64, E=2, rank=16, mods=2)
    rows = torch.randint(0, 20, (n,), generator=_gen(n), device="cuda").to(torch.int32)
    bad = rows.clone()
    bad[::4] = torch.tensor([-1, 20, 2 ** 31 - 1, -2 ** 31], device="cuda")[torch.arange(len(bad[::4])) % 4].int()
    lin = ops.ExpertLinear(c.inv, c.wq, c.scale, c.ld, c.ru)
    first = torch.where((bad < 0) | (bad >= 20), torch.zeros_like(bad), bad)
    want = lin(c.x, c.mod, _offsets([2, n - 2]), rows=first)
    off = torch.tensor([-5, 2, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    assert torch.equal(lin(c.x, c.mod, off, rows=bad), want)


def test_experts_without_any_row(ops):
    c = Case(1, 8, 128, 64, E=3, rank=16, mods=2)
    rows = torch.full((8,), -1, device="cuda", dtype=torch.int32)
    _check_experts(ops, c, [0, 0, 0], rows, "none", False, "bf16", extra=8)


def test_an_infinite_factor_stays_with_its_expert_and_modality(ops):
    c = Case(4, 24, 128, 64, E=3, rank=16, mods=3)
    c.ld[1, 0, 3, 5] = math.inf                             # expert 1, modality 1
    rows = torch.arange(24, device="cuda", dtype=torch.int32)
    lin = ops.ExpertLinear(c.inv, c.wq, c.scale, c.ld, c.ru)
    got = lin(c.x, c.mod, _offsets([8, 8, 8]), rows=rows)
    hit = torch.zeros(24, dtype=torch.bool, device="cuda")
    hit[8:16] = c.mod[8:16] == 1
    assert torch.isfinite(got[~hit]).all()


def test_one_expert_is_the_layer(ops):
    for T, N in ((9, 96), (300, 512)):
        c = Case(T, T, 512, N, E=1, rank=16, mods=2, bias=True)
        c.mod.zero_()
        one = ops.ExpertLinear(c.inv, c.wq, c.scale, c.ld, c.ru, bias=c.bias, act="silu")
        lin = ops.Linear(c.inv, c.wq[0], c.scale[0], c.ld[0], c.ru[0])
        assert torch.equal(one(c.x, c.mod, _offsets([T])), lin.fused(c.x, c.mod, bias=c.bias[0], act="silu"))


# ------------------------------------------------------------------ combination
@pytest.mark.parametrize("T,N,k", [(1, 16, 1), (5, 48, 3), (33, 2048, 8), (700, 3584, 5), (64, 528, 16)])
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_combine(ops, T, N, k, io):
    g = _gen(T + N)
    n = T * k
    d = _randn(g, n, N).to(DT[io])
    slots = torch.randint(0, n, (T, k), generator=g, device="cuda").to(torch.int32)   # slots may recur
    slots[torch.rand((T, k), generator=g, device="cuda") < 0.2] = -1
    slots[0, 0] = n                                         # outside: nothing
    w = _randn(g, T, k)
    for res in (None, _randn(g, T, N).to(DT[io])):
        y = torch.zeros((T, N), dtype=torch.float64, device="cuda")
        a = torch.zeros_like(y)
        for j in range(k):
            s = slots[:, j].long()
            ok = ((s >= 0) & (s < n))[:, None]
            term = torch.where(ok, w[:, j:j + 1].double() * d[s.clamp(0, n - 1)].double(), torch.zeros_like(y))
            y, a = y + term, a + term.abs()
        if res is not None:
            y, a = y + res.double(), a + res.double().abs()
        err = ref.U * (k + 2) * a
        err = err + torch.finfo(DT[io]).eps / 2 * (y.abs() + err) + 1e-37
        ref.assert_close(ops.combine_experts(d, slots, w, residual=res), y, err)
        if res is not None:
            buf = res.clone()
            ref.assert_close(ops.combine_experts(d, slots, w, residual=buf, out=buf), y, err)


def test_combine_of_no_slots_is_the_residual(ops):
    res = _randn(_gen(1), 5, 64)
    slots = torch.full((5, 2), -1, dtype=torch.int32, device="cuda")
    w = torch.ones((5, 2), device="cuda")
    assert torch.equal(ops.combine_experts(torch.empty((0, 64), device="cuda"), slots, w, residual=res), res)


def test_combine_skips_what_unused_slots_hold(ops):
    d = torch.full((4, 32), math.nan, device="cuda")
    d[2] = 1.5
    slots = torch.tensor([[2, -1], [-1, -1]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[2.0, math.nan], [math.nan, 1.0]], device="cuda")
    y = ops.combine_experts(d, slots, w)
    assert (y[0] == 3.0).all() and (y[1] == 0).all()


# ------------------------------------------------------------------ the block
class Block:
    def __init__(self, ops, seed, T, E, k, K, inner, io="bf16", bits=8, rank=16, mods=2):
        self.up = Case(seed, T, K, 2 * inner, E=E, rank=rank, mods=mods, io=io, bits=bits, bias=True)
        self.dn = Case(seed + 1, 1, inner, K, E=E, rank=rank, mods=mods, io=io, bits=bits)
        g = _gen(seed + 2)
        self.logits = _randn(g, T, E)
        self.logits[T // 2] = -math.inf                     # a padding row
        self.res = _randn(g, T, K).to(DT[io])
        u, d = self.up, self.dn
        self.gate_up = ops.ExpertLinear(u.inv, u.wq, u.scale, u.ld, u.ru, bias=u.bias, act="silu", gated=True)
        self.down = ops.ExpertLinear(d.inv, d.wq, d.scale, d.ld, d.ru)
        self.mlp = ops.ExpertMLP(self.gate_up, self.down, k)
        self.k, self.io = k, io

    def __call__(self):
        return self.mlp(self.up.x, self.up.mod, self.logits, residual=self.res)

    def check(self, got, ops):
        """Each layer against 64 bits on the rows it is given (the down layer
        quantises the rows that the gate/up layer rounded)."""
        x, mod, dt = self.up.x, self.up.mod, DT[self.io]
        experts, weights, offsets, rows, slots = ref.route(self.logits, self.k, True)
        r = ops.route_experts(self.logits, self.k, modality=mod)
        h = self.gate_up(x, mod, r.offsets, rows=r.rows)
        y, a = self.res.double(), self.res.double().abs()
        total = offsets[-1]
        d = torch.zeros((total, self.dn.scale.shape[1]), dtype=torch.float64, device="cuda")
        de = torch.zeros_like(d)
        for e in range(len(offsets) - 1):
            lo, hi = offsets[e], offsets[e + 1]
            if lo == hi:
                continue
            i = torch.tensor(rows[lo:hi], device="cuda")
            u, n = self.up, self.dn
            z, err = ref.layer(x[i], mod[i], u.inv, u.codes[e], u.scale[e], u.ld[e], u.ru[e], u.bias[e])
            ref.assert_close(h[lo:hi], *ref.finish(z, err, "silu", True, None, dt))
            z, err = ref.layer(h[lo:hi], mod[i], n.inv, n.codes[e], n.scale[e], n.ld[e], n.ru[e])
            d[lo:hi], de[lo:hi] = ref.finish(z, err, "none", False, None, dt)
        err = torch.zeros_like(y)
        for t, row in enumerate(slots):
            for j, s in enumerate(row):
                if s >= 0:
                    w = weights[t][j]
                    y[t] += w * d[s]
                    a[t] += w * (d[s].abs() + de[s])
                    err[t] += w * (de[s] + 64 * ref.U * d[s].abs())
        err = err + ref.U * (self.k + 2) * a
        ref.assert_close(got, y, err + torch.finfo(dt).eps / 2 * (y.abs() + err))
        assert torch.equal(got[len(slots) // 2], self.res[len(slots) // 2])   # the padding row


@pytest.mark.parametrize("T,E,k,K,inner,io,bits", [(1, 4, 2, 64, 64, "bf16", 8), (6, 16, 4, 256, 128, "bf16", 4),
                                                   (70, 10, 3, 528, 208, "f32", 8),
                                                   (400, 8, 2, 512, 320, "bf16", 8)])
def test_block(ops, T, E, k, K, inner, io, bits):
    b = Block(ops, T + E, T, E, k, K, inner, io=io, bits=bits)
    b.check(b(), ops)


def test_block_captured_and_replayed(ops):
    blocks = [Block(ops, s, T, 8, 2, 256, 128) for s, T in ((1, 9), (20, 300))]
    lin = [ops.Linear(b.dn.inv, b.dn.wq[0], b.dn.scale[0], b.dn.ld[0], b.dn.ru[0]) for b in blocks]
    eager = [b() for b in blocks]
    graphs, outs = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for b, l in zip(blocks, lin):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=side):
            y = b()
            z = l.fused(y[:, :128].contiguous(), b.up.mod, act="silu", residual=b.res)
        graphs.append(gr)
        outs.append((y, z))
    for rep in range(3):
        for b in blocks:                                    # new inputs in the same buffers
            b.up.x.copy_(_randn(_gen(100 + rep), *b.up.x.shape))
            b.logits.copy_(_randn(_gen(200 + rep), *b.logits.shape))
            b.logits[b.logits.shape[0] // 2] = -math.inf
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        for b, l, (y, z) in zip(blocks, lin, outs):
            want = b()
            assert torch.equal(y, want)
            assert torch.equal(z, l.fused(want[:, :128].contiguous(), b.up.mod, act="silu", residual=b.res))
    assert len(eager) == 2


def test_calls_on_two_streams_at_once(ops):
    blocks = [Block(ops, s, 200, 8, 2, 256, 128) for s in (1, 2)]
    want = [b() for b in blocks]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    got = []
    for _ in range(5):
        for b, s in zip(blocks, streams):
            got.append(b.mlp(b.up.x, b.up.mod, b.logits, residual=b.res, stream=s))
    torch.cuda.synchronize()
    for i, y in enumerate(got):
        assert torch.equal(y, want[i % 2])


# ------------------------------------------------------------------ past 2^31 elements
def test_rows_past_2_31_elements(ops):
    T, K, N = 70000, 64, 32768
    c = Case(5, T, K, N, bias=True, residual=True, width=N)
    lin = ops.Linear(c.inv, c.wq, c.scale)
    y = lin.fused(c.x, c.mod, bias=c.bias, act="silu", residual=c.res)
    at = slice(T - 40, T)
    part = lin.fused(c.x[at].contiguous(), c.mod[at], bias=c.bias, act="silu", residual=c.res[at].contiguous())
    assert torch.equal(y[at], part)
    # the same rows as two experts' (the last slots are the second one's)
    two = ops.ExpertLinear(c.inv, c.wq[None].expand(2, -1, -1).contiguous(), c.scale[None].repeat(2, 1),
                           bias=c.bias[None].repeat(2, 1), act="silu")
    z = two(c.x, c.mod, _offsets([T - 100, 100]), out=y)
    assert torch.equal(z[at], lin.fused(c.x[at].contiguous(), c.mod[at], bias=c.bias, act="silu"))
    # and combined: token t takes row T - 1 - t
    slots = torch.arange(T - 1, -1, -1, device="cuda", dtype=torch.int32)[:, None].contiguous()
    w = torch.ones((T, 1), device="cuda")
    s = ops.combine_experts(z, slots, w, out=c.res)
    assert torch.equal(s[:40].flip(0), z[at]) and torch.equal(s[T - 40:].flip(0), z[:40])


def test_weights_past_2_31_bytes(ops):
    E, N, K = 34, 8192, 8192
    g = _gen(2)
    wq = torch.zeros((E, N, K), dtype=torch.int8, device="cuda")
    wq[-1] = torch.randint(-127, 128, (N, K), generator=g, device="cuda").to(torch.int8)
    scale = torch.full((E, N), 1e-4, device="cuda")
    x = _randn(g, 9, K).to(torch.bfloat16)
    mod, inv = torch.zeros(9, dtype=torch.int32, device="cuda"), torch.ones((1, K), device="cuda")
    got = ops.ExpertLinear(inv, wq, scale)(x, mod, _offsets([0] * (E - 2) + [2, 7]))
    want = ops.Linear(inv, wq[-1], scale[-1])(x, mod)
    assert torch.equal(got[2:], want[2:]) and not got[:2].any()


def test_results_do_not_vary(ops):
    b = Block(ops, 3, 500, 16, 4, 256, 128)
    first = b()
    for _ in range(3):
        assert torch.equal(b(), first)
