"""The operators around the quantised layer on the GPU, where test_block_gpu.py does
not reach."""
import math

import pytest
import torch

import block_reference as ref
from test_block_gpu import DT, Block, Case, _gen, _offsets, _randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2603_04800_amd import ops as o
    return o


# ------------------------------------------------------------------ activations
# |z| from where every activation is z or 0 to fp32 working precision, past 7e12,
# where z^3 leaves fp32, to past 2.4e38, where z log2 e does
FAR = [200.0, 1e3, 1e7, 6.5e12, 8e12, 1e13, 1e20, 1e30, 2.3e38, 2.5e38, 3e38]


@pytest.mark.parametrize("T", [8, 300])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_activations_far_from_zero(ops, act, io, gated, T):
    """act(z) is z for z far above zero and 0 far below.  z carries 3 u of the
    product; logistic and erfc are within 8 u of 1 there (exp, reciprocal, their
    products); gating and the output round once more.  The last pair of channels
    overflows fp32: the infinity above stays one."""
    K, per = 64, 2 if gated else 1
    far = FAR + [1e42]
    z = torch.tensor([s * v for v in far for s in (1.0, -1.0)] + [0.0] * 8, dtype=torch.float64, device="cuda")
    N = per * z.numel()
    x = torch.ones((T, K), device="cuda", dtype=DT[io])
    x[-1] = 0                                               # a row of zeros beside them
    codes = torch.full((N, K), 127, device="cuda", dtype=torch.int8)
    codes[per:per * len(far) * 2:2 * per] = -127            # (a gate's negative; its up channel stays positive)
    scale = torch.full((N,), 0.5 / (127 * K), device="cuda")
    scale[::per] = (z.abs() / (127 * K)).clamp(max=1e38).float()
    inv, mod = torch.ones((1, K), device="cuda"), torch.zeros(T, device="cuda", dtype=torch.int32)
    got = ops.Linear(inv, codes, scale).fused(x, mod, act=act, gated=gated).double()
    want, _ = ref.layer(x, mod, inv, codes, scale, None, None)
    want = torch.where(want[:, ::per] > 0, want[:, ::per], torch.zeros_like(want[:, ::per])) * (0.5 if gated else 1.0)
    n = 2 * len(FAR)
    want, over = want[:, :n], got[:, n:n + 2]
    # (codes 127 and steps of 1 / 127: the up channel is 0.5 to 3 u)
    err = want * (ref.U * 16 + torch.finfo(DT[io]).eps / 2 * 1.01) + 1e-37
    want, err = want[:-1], err[:-1]
    ref.assert_close(got[:-1, :n], want, err)
    assert (over[:-1, 0] == math.inf).all()
    assert not got[-1].isnan().any() and not got[-1].any()
    assert not got[:, n + 2:].any()


# ------------------------------------------------------------------ routing and offsets
def test_empty_routing_writes_its_offsets_on_the_calls_stream(ops):
    logits = torch.empty((0, 8), device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):                              # memory of s that s itself fills, late
        torch.cuda._sleep(200_000_000)
        junk = torch.full((9,), -1, dtype=torch.int32, device="cuda")
        at = junk.data_ptr()
        del junk
    r = ops.route_experts(logits, 2, stream=s)
    assert r.offsets.data_ptr() == at
    s.synchronize()
    torch.cuda.synchronize()
    assert r.offsets.tolist() == [0] * 9


@pytest.mark.parametrize("n,K,N", [(400, 128, 64), (3000, 64, 3104)])
def test_offsets_that_do_not_ascend_stay_within_the_rows(ops, n, K, N):
    """Experts that claim the same slots make more tiles than the slots can: no
    row is written, and none past them."""
    c = Case(n, 20, K, N, E=6, rank=16, mods=2)
    rows = torch.randint(0, 20, (n,), generator=_gen(n), device="cuda").to(torch.int32)
    off = torch.tensor([0, n, 0, n, 0, n, 0], dtype=torch.int32, device="cuda")
    buf = torch.full((n + 64, N), 7.25, dtype=torch.bfloat16, device="cuda")
    ops.ExpertLinear(c.inv, c.wq, c.scale, c.ld, c.ru)(c.x, c.mod, off, rows=rows, out=buf[:n])
    assert (buf == 7.25).all()


# ------------------------------------------------------------------ the first stage's forms
def _dirty(ops, T, n, K, rank, mods):
    need = ops.raw().masq_expert_linear_workspace_bytes(T, n, K, rank, mods)
    return torch.full((need,), 255, dtype=torch.uint8, device="cuda")           # NaN throughout


@pytest.mark.parametrize("counts,T,K,rank,mods,io,lr", [
    # slots in groups of 32 (past 512 groups of 16) and of 64 (past 1024), one and
    # two rank blocks, then four; experts that end inside a group, rows that end
    # inside a step
    ([4001, 0, 17, 5003], 500, 96, 16, 2, "bf16", "bf16"), ([3000, 33, 6100], 0, 80, 32, 3, "bf16", "bf16"),
    ([9100, 1], 300, 144, 16, 4, "f32", "f32"), ([2222, 7001], 0, 64, 32, 2, "bf16", "f32"),
    ([8200, 9001, 40], 700, 80, 16, 3, "bf16", "bf16"), ([16999, 0, 31], 0, 96, 32, 4, "bf16", "bf16"),
    ([5, 17001], 400, 112, 32, 2, "f32", "f32"), ([17100], 200, 64, 16, 2, "f32", "bf16"),
    ([700, 16900], 0, 80, 16, 3, "bf16", "f32"),
    ([9001, 70], 333, 80, 48, 3, "bf16", "bf16"), ([10, 9300], 0, 96, 64, 2, "f32", "f32"),
])
def test_every_form_of_the_first_stage(ops, counts, T, K, rank, mods, io, lr):
    E, n, N = len(counts), sum(counts), 32
    c = Case(n + K, T or n, K, N, E=E, rank=rank, mods=mods, io=io, lr=lr, bias=True)
    rows = torch.randint(0, T, (n,), generator=_gen(n), device="cuda").to(torch.int32) if T else None
    at = rows.long() if T else torch.arange(n, device="cuda")
    lin = ops.ExpertLinear(c.inv, c.wq, c.scale, c.ld, c.ru, bias=c.bias, act="silu")
    got = lin(c.x, c.mod, _offsets(counts), rows=rows, workspace=_dirty(ops, T or n, n, K, rank, mods))
    lo = 0
    for e, cnt in enumerate(counts):
        i = at[lo:lo + cnt]
        if cnt:
            z, err = ref.layer(c.x[i], c.mod[i], c.inv, c.codes[e], c.scale[e], c.ld[e], c.ru[e], c.bias[e])
            ref.assert_close(got[lo:lo + cnt], *ref.finish(z, err, "silu", False, None, DT[io]))
        lo += cnt


@pytest.mark.parametrize("T,K,rank,mods,io,lr", [
    # the same forms over a layer's own rows (one expert)
    (9001, 80, 16, 3, "f32", "f32"), (8999, 96, 32, 2, "bf16", "f32"), (17003, 64, 16, 2, "bf16", "f32"),
    (17001, 144, 32, 4, "f32", "f32"), (9003, 80, 80, 3, "bf16", "bf16"),
])
def test_every_form_of_the_first_stage_over_a_layers_rows(ops, T, K, rank, mods, io, lr):
    N = 32
    c = Case(T, T, K, N, rank=rank, mods=mods, io=io, lr=lr, bias=True, residual=True, width=N)
    ws = torch.full((ops.workspace_bytes(T, K, N, rank, mods),), 255, dtype=torch.uint8, device="cuda")
    got = ops.Linear(c.inv, c.wq, c.scale, c.ld, c.ru).fused(c.x, c.mod, bias=c.bias, act="silu", residual=c.res,
                                                             workspace=ws)
    z, err = ref.layer(c.x, c.mod, c.inv, c.codes, c.scale, c.ld, c.ru, c.bias)
    ref.assert_close(got, *ref.finish(z, err, "silu", False, c.res, DT[io]))


# ------------------------------------------------------------------ layers that split K over 256 x 256 tiles
@pytest.mark.parametrize("T,K,N,rank,mods,io,bits,act,gated", [
    (257, 18944, 3584, 64, 2, "bf16", 8, "none", False), (300, 18944, 3584, 16, 3, "f32", 8, "silu", True),
    (384, 18944, 3584, 64, 2, "bf16", 4, "gelu", False), (401, 28672, 2048, 32, 2, "bf16", 8, "gelu_tanh", True),
])
def test_layers_whose_own_product_splits_k(ops, T, K, N, rank, mods, io, bits, act, gated):
    width = N // 2 if gated else N
    c = Case(T + K, T, K, N, rank=rank, mods=mods, io=io, bits=bits, bias=True, residual=True, width=width)
    lin = ops.Linear(c.inv, c.wq, c.scale, c.ld, c.ru)
    got = lin.fused(c.x, c.mod, bias=c.bias, act=act, gated=gated, residual=c.res)
    z, e = ref.layer(c.x, c.mod, c.inv, c.codes, c.scale, c.ld, c.ru, c.bias)
    ref.assert_close(got, *ref.finish(z, e, act, gated, c.res, DT[io]))
    text = c.mod == 0
    assert torch.equal(lin.fused(c.x, c.mod)[text], lin(c.x, c.mod)[text])


# ------------------------------------------------------------------ replays on the inputs captured
def test_replays_repeat_the_eager_result(ops):
    blocks = [Block(ops, s, T, 8, 2, 256, 128) for s, T in ((3, 9), (30, 300))]
    lin = [ops.Linear(b.dn.inv, b.dn.wq[0], b.dn.scale[0], b.dn.ld[0], b.dn.ru[0]) for b in blocks]
    c = Case(5, 64, 4096, 96, rank=16, mods=2, bias=True, residual=True, width=96)   # slices and their counters
    split = ops.Linear(c.inv, c.wq, c.scale, c.ld, c.ru)

    def all_of(b, l):
        y = b()
        return (y, l.fused(y[:, :128].contiguous(), b.up.mod, act="silu", residual=b.res),
                split.fused(c.x, c.mod, bias=c.bias, act="gelu", residual=c.res))

    eager = [all_of(b, l) for b, l in zip(blocks, lin)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs, outs = [], []
    for b, l in zip(blocks, lin):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=side):
            outs.append(all_of(b, l))
        graphs.append(gr)
    for _ in range(3):
        for gr, o, want, b, l in zip(graphs, outs, eager, blocks, lin):
            for t in o:
                t.fill_(math.nan)
            gr.replay()
            again = all_of(b, l)                            # eager work between the replays
            torch.cuda.synchronize()
            for got, w, a in zip(o, want, again):
                assert torch.equal(got, w) and torch.equal(a, w)
