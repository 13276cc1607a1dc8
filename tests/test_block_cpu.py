"""What the operators around the quantised layer refuse, without a GPU:
every check runs before any HIP call."""
import pytest
import torch

from paper_2603_04800_amd import ops

P = 1 << 20          # a fake, 256-byte aligned "device" address; never dereferenced


@pytest.fixture(scope="module")
def lib():
    return ops.raw()


def _epilogue(lib, **kw):
    a = dict(x=P, x_dt=1, mod=P, inv=P, wq=P, bits=8, ws=P, ld=P, ru=P, lr_dt=1, T=16, K=64, N=64,
             rank=16, n_mod=2, bias=P, act=0, res=P, y=P, y_dt=1, work=P, work_bytes=1 << 30, stream=None)
    a.update(kw)
    return lib.masq_linear_epilogue(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), 1), (dict(wq=None), 1), (dict(y=None), 1), (dict(ld=None), 1), (dict(work=None), 1),
    (dict(K=40), 2), (dict(N=24), 2), (dict(T=-1), 2), (dict(rank=8), 2), (dict(n_mod=5), 2),
    (dict(bits=3), 2), (dict(bits=4, K=80), 2), (dict(act=16, N=48), 2), (dict(K=133152), 2),
    (dict(x_dt=7), 3), (dict(y_dt=2), 3),
    (dict(x=P + 8), 4), (dict(bias=P + 4), 4), (dict(res=P + 8), 4), (dict(work=P + 16), 4),
    (dict(work_bytes=100), 5),
    (dict(act=4), 7), (dict(act=-1), 7), (dict(act=32), 7), (dict(act=20), 7),
])
def test_epilogue_refuses(lib, kw, code):
    assert _epilogue(lib, **kw) == code


def test_epilogue_of_an_empty_batch(lib):
    assert _epilogue(lib, T=0, x=None, y=None, work=None, work_bytes=0, bias=None, res=None, act=17) == 0


def _route(lib, **kw):
    a = dict(logits=P, dt=0, mod=P, T=1000, E=64, k=8, norm=1, experts=P, weights=P, offsets=P, rows=P,
             slots=P, slot_mod=P, work=P, work_bytes=1 << 30, stream=None)
    a.update(kw)
    return lib.masq_route_experts(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(logits=None), 1), (dict(slots=None), 1), (dict(mod=None), 1), (dict(slot_mod=None), 1),
    (dict(work=None), 1),
    (dict(T=-1), 2), (dict(E=0), 2), (dict(E=513), 2), (dict(k=0), 2), (dict(k=17), 2), (dict(E=4, k=5), 2),
    (dict(T=1 << 31, k=1), 2), (dict(T=1 << 28, k=8), 2),
    (dict(dt=2), 3), (dict(rows=P + 4), 4), (dict(work=P + 16), 4), (dict(work_bytes=64), 5),
])
def test_route_refuses(lib, kw, code):
    assert _route(lib, **kw) == code


def test_route_workspace(lib):
    f = lib.masq_route_experts_workspace_bytes
    assert _route(lib, T=0, logits=None, work=None, work_bytes=0) == 0
    assert f(-1, 8) == 0 and f(100, 0) == 0 and f(0, 8) == 0
    assert f(8192, 128) >= 256 * 128 * 4 and f(9000, 128) > f(8192, 128)


def _experts(lib, **kw):
    a = dict(x=P, x_dt=1, T=16, mod=P, inv=P, wq=P, bits=8, ws=P, ld=P, ru=P, lr_dt=1, rows=P, offsets=P,
             n=32, E=4, K=64, N=64, rank=16, n_mod=2, bias=P, act=0, y=P, y_dt=1, work=P,
             work_bytes=1 << 30, stream=None)
    a.update(kw)
    return lib.masq_expert_linear(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), 1), (dict(offsets=None), 1), (dict(ru=None), 1), (dict(y=None), 1), (dict(work=None), 1),
    (dict(K=40), 2), (dict(N=24), 2), (dict(E=0), 2), (dict(E=513), 2), (dict(n=-1), 2), (dict(n=1 << 31), 2),
    (dict(rows=None), 2), (dict(bits=5), 2), (dict(bits=4, K=80), 2), (dict(act=17, N=80), 2),
    (dict(rank=8), 2), (dict(n=(1 << 31) - 1, N=1 << 20), 2),
    (dict(lr_dt=3), 3), (dict(rows=P + 4), 4), (dict(bias=P + 4), 4), (dict(work=P + 16), 4),
    (dict(work_bytes=64), 5), (dict(act=9), 7),
])
def test_experts_refuse(lib, kw, code):
    assert _experts(lib, **kw) == code


def test_experts_of_nothing(lib):
    assert _experts(lib, T=0, x=None, work=None, work_bytes=0) == 0
    assert _experts(lib, n=0, x=None, work=None, work_bytes=0) == 0
    f = lib.masq_expert_linear_workspace_bytes
    assert f(16, 32, 64, 16, 2) >= 16 * 64 + 16 * 4 + 32 * 16 * 4
    assert f(16, 32, 64, 16, 1) < f(16, 32, 64, 16, 2) and f(-1, 1, 64, 0, 1) == 0


def _combine(lib, **kw):
    a = dict(d=P, dt=1, slots=P, weights=P, T=8, n=16, N=64, k=2, res=P, y=P, stream=None)
    a.update(kw)
    return lib.masq_combine_experts(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(d=None), 1), (dict(slots=None), 1), (dict(y=None), 1), (dict(N=24), 2), (dict(k=0), 2),
    (dict(k=17), 2), (dict(T=-1), 2), (dict(n=-1), 2), (dict(dt=5), 3), (dict(res=P + 8), 4), (dict(d=P + 2), 4),
])
def test_combine_refuses(lib, kw, code):
    assert _combine(lib, **kw) == code


def test_combine_of_an_empty_batch(lib):
    assert _combine(lib, T=0, d=None, y=None) == 0


# ------------------------------------------------------------------ the Python entry points
def _lin(gated=False):
    return ops.Linear(torch.ones(1, 64), torch.zeros(32, 64, dtype=torch.int8), torch.ones(32))


def test_python_checks():
    x, mod = torch.ones(4, 64), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        _lin().fused(x, mod)
    with pytest.raises(ValueError, match="activation"):
        _lin().fused(x, mod, act="relu6")
    with pytest.raises(ValueError, match=r"\[T\]\[64\]"):
        _lin().fused(torch.ones(4, 32), mod)
    with pytest.raises(ValueError, match="GPU"):
        ops.route_experts(torch.ones(4, 8), 2)
    with pytest.raises(ValueError, match="GPU"):
        ops.combine_experts(torch.ones(4, 16), torch.zeros(2, 2, dtype=torch.int32), torch.ones(2, 2))


def test_expert_layer_checks_its_weights():
    inv, wq, sc = torch.ones(2, 64), torch.zeros(3, 32, 64, dtype=torch.int8), torch.ones(3, 32)
    lin = ops.ExpertLinear(inv, wq, sc, act="silu", gated=True)
    assert lin.width == 16 and lin.rank == 0 and not lin.w4
    with pytest.raises(ValueError, match="width"):
        ops.ExpertLinear(torch.ones(2, 48), wq, sc)
    with pytest.raises(ValueError, match="w_scale"):
        ops.ExpertLinear(inv, wq, torch.ones(3, 31))
    with pytest.raises(ValueError, match="bias"):
        ops.ExpertLinear(inv, wq, sc, bias=torch.ones(32))
    with pytest.raises(ValueError, match="r_up"):
        ops.ExpertLinear(inv, wq, sc, l_down=torch.ones(3, 1, 16, 64))
    with pytest.raises(ValueError, match="l_down"):
        ops.ExpertLinear(inv, wq, sc, torch.ones(3, 2, 16, 64), torch.ones(3, 2, 32, 16))
    with pytest.raises(ValueError, match="fit"):
        ops.ExpertMLP(lin, lin, 2)


def test_interleaved_channels():
    g, u = torch.arange(6).view(1, 3, 2), 10 + torch.arange(6).view(1, 3, 2)
    w = ops.interleave_gate_up(g, u, axis=1)
    assert w.shape == (1, 6, 2) and torch.equal(w[:, 0::2], g) and torch.equal(w[:, 1::2], u)
    assert ops.interleave_gate_up(torch.tensor([1, 2]), torch.tensor([3, 4])).tolist() == [1, 3, 2, 4]
    with pytest.raises(ValueError):
        ops.interleave_gate_up(torch.ones(2), torch.ones(3))
