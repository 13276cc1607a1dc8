"""The operators around the quantised layer on the GPU, where test_block_gpu.py does
not reach."""
import math

import pytest
import torch

import block_reference as ref
from test_block_gpu import DT, Case, _gen

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
