"""Host-only checks of the operators around the expert GEMMs: what they refuse, before they touch a device."""
import ctypes as C

import pytest

from paper_2605_05607_amd import binding as B

A = 4096  # an aligned address that is never dereferenced: validation fails first
INV, UNS, WSP = B.MOE_ERR_INVALID_ARG, B.MOE_ERR_UNSUPPORTED, B.MOE_ERR_WORKSPACE
NORM = dict(rows=4, cols=64, dtype=B.MOE_BF16, x=A, residual=2 * A, weight=3 * A, eps=1e-6, sum=4 * A, y=5 * A, codes=6 * A,
            scales=7 * A, rstd=8 * A, stream=None)
BACK = dict(rows=4, cols=64, dtype=B.MOE_BF16, sum=A, weight=2 * A, rstd=3 * A, dy=4 * A, dsum=5 * A, dx=6 * A, dweight=7 * A,
            workspace=8 * A, workspace_bytes=1 << 20, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), INV), (dict(rows=1 << 31), INV), (dict(cols=0), INV), (dict(cols=60), INV), (dict(cols=32776), UNS),
    (dict(dtype=2), UNS), (dict(x=None), INV), (dict(weight=None), INV), (dict(y=None, codes=None, scales=None), INV),
    (dict(codes=None), INV), (dict(scales=None), INV), (dict(residual=None), INV), (dict(eps=0.0), INV), (dict(eps=-1.0), INV),
    (dict(eps=float("nan")), INV), (dict(eps=float("inf")), INV), (dict(y=A), INV), (dict(y=2 * A), INV), (dict(y=4 * A), INV),
    (dict(x=A + 8), INV), (dict(residual=A + 8), INV), (dict(weight=A + 8), INV), (dict(sum=4 * A + 8), INV),
    (dict(y=5 * A + 8), INV), (dict(codes=6 * A + 4), INV), (dict(scales=7 * A + 2), INV), (dict(rstd=8 * A + 2), INV)])
def test_norm_refusals(change, status):
    assert B.lib().moe_rmsnorm(*{**NORM, **change}.values()) == status


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), INV), (dict(cols=12), INV), (dict(cols=32776), UNS), (dict(dtype=7), UNS), (dict(sum=None), INV),
    (dict(weight=None), INV), (dict(rstd=None), INV), (dict(dy=None), INV), (dict(dx=None), INV), (dict(workspace=None), WSP),
    (dict(workspace_bytes=4 * 64 * 4 - 1), WSP), (dict(sum=A + 8), INV), (dict(dy=A + 8), INV), (dict(dsum=A + 8), INV),
    (dict(dx=6 * A + 8), INV), (dict(workspace=A + 8), INV), (dict(dx=A), INV), (dict(rstd=A + 2), INV),
    (dict(dweight=7 * A + 2), INV)])
def test_norm_backward_refusals(change, status):
    assert B.lib().moe_rmsnorm_backward(*{**BACK, **change}.values()) == status


def test_norm_of_no_rows_and_workspace_sizes():
    assert B.lib().moe_rmsnorm(*{**NORM, "rows": 0}.values()) == 0
    assert B.lib().moe_rmsnorm_backward(*{**BACK, "rows": 0, "dweight": None}.values()) == 0
    size = B.moe_rmsnorm_backward_workspace_bytes
    assert size(-1, 64) == 0 and size(4, 60) == 0 and size(4, 32776) == 0
    assert 0 < size(0, 64) <= size(1, 64) <= size(5, 64) <= size(1 << 20, 64) and size(9, 7168) % 4 == 0


def good_shape(**kw):
    return B.make_shape(**{**dict(T=64, d=64, f=128, E=8, k=2, R=4, local_rank_begin=0, local_rank_end=1, dtype=B.MOE_BF16),
                           **kw})


TABLES = B.moe_dispatch(*([A] * 9))


def rows_calls(s, tables=TABLES, **kw):
    p = {**dict(rows=A, dy=2 * A, idx=3 * A, w=4 * A, out=5 * A, dw=6 * A), **kw}
    L, s, tb = B.lib(), C.byref(s), None if tables is None else C.byref(tables)
    return (L.moe_combine_weighted(s, p["rows"], p["idx"], p["w"], tb, p["out"], None),
            L.moe_combine_weighted_backward(s, p["rows"], p["dy"], p["idx"], p["w"], tb, p["out"], p["dw"], None),
            L.moe_dispatch_gather_backward(s, p["rows"], p["idx"], tb, p["out"], None))


def test_rows_refusals():
    assert rows_calls(good_shape(E=10)) == (INV,) * 3 and rows_calls(good_shape(dtype=5)) == (UNS,) * 3
    assert rows_calls(good_shape(d=60)) == (INV,) * 3
    for missing in ("rows", "idx", "out"):
        assert rows_calls(good_shape(), **{missing: None}) == (INV,) * 3, missing
    assert rows_calls(good_shape(T=0), w=None) == (INV, INV, 0)
    assert rows_calls(good_shape(T=0), dy=None) == (0, INV, 0) and rows_calls(good_shape(T=0), dw=None) == (0, INV, 0)
    assert rows_calls(good_shape(), tables=None) == (INV,) * 3
    for n in ("offsets", "inv_perm"):
        tb = B.moe_dispatch(*([A] * 9))
        setattr(tb, n, None)
        assert rows_calls(good_shape(), tables=tb) == (INV,) * 3, n
    assert rows_calls(good_shape(), rows=A + 8) == (INV,) * 3 and rows_calls(good_shape(), out=A + 8) == (INV,) * 3
    assert rows_calls(good_shape(T=0), dy=2 * A + 8) == (0, INV, 0)
    assert rows_calls(good_shape(T=0), out=A) == (INV, 0, INV)  # (d_rows may be rows)
    assert rows_calls(good_shape(T=0), out=2 * A) == (0, INV, 0)
    assert rows_calls(good_shape(T=0)) == (0, 0, 0) and rows_calls(good_shape(T=1 << 24)) == (UNS,) * 3
    assert rows_calls(good_shape(d=(1 << 30) + 8)) == (UNS,) * 3


def adamw(tensor=None, device=None, count=1, **config):
    now = B.moe_adamw_device(config.pop("lr", 1e-3), config.pop("grad_scale", 1.0), config.pop("step", 1), 0)
    c = B.moe_adamw_config(*{**dict(beta1=0.9, beta2=0.99, eps=1e-8, bits=32), **config}.values(), now)
    t = B.moe_adamw_tensor(*{**dict(param=A, copy=2 * A, grad=3 * A, m=4 * A, v=5 * A, m_scale=6 * A, v_scale=7 * A, n=0,
                                    decay=0.0, grad_dtype=B.MOE_BF16), **(tensor or {})}.values())
    return B.lib().moe_adamw_step(C.byref(c), C.byref(t), count, device, None)


def test_adamw_refusals():
    assert adamw() == 0 and adamw(count=0) == 0 and adamw(dict(param=None, grad=None, m=None, v=None)) == 0  # empty tensors
    assert adamw(count=-1) == INV and B.lib().moe_adamw_step(None, None, 0, None, None) == INV
    for bad in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=0.0), dict(eps=1e-60),
                dict(eps=float("inf")), dict(lr=-1.0), dict(lr=float("nan")), dict(step=0), dict(step=-3), dict(device=A + 2)):
        assert adamw(**bad) == INV, bad
    assert adamw(device=A, step=0, lr=-1.0) == 0  # (those of the device count)
    assert adamw(bits=16) == UNS and adamw(dict(grad_dtype=4)) == UNS and adamw(dict(n=1 << 35)) == UNS
    for bad in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(param=A + 8), dict(copy=A + 8),
                dict(grad=A + 8), dict(m=A + 8), dict(v=A + 8), dict(n=-1), dict(decay=-0.1), dict(decay=float("nan"))):
        assert adamw({"n": 4, **bad}) == INV, bad
    for bad in (dict(m_scale=None), dict(v_scale=None), dict(m_scale=A + 2)):
        assert adamw({"n": 4, **bad}, bits=8) == INV, bad


def test_adamw_eps_is_a_normal_number():
    assert adamw(eps=1e-39) == INV and adamw(eps=2.0 ** -127) == INV  # (their reciprocals leave fp32: 0 / eps would be NaN)
    assert adamw(eps=2.0 ** -126) == 0 and adamw(eps=1e-30) == 0


def test_adamw_class_checks_its_tensors():
    import torch

    from paper_2605_05607_amd import layer as L
    p, g = torch.zeros(10), torch.zeros(10, dtype=torch.bfloat16)
    L.AdamW([p], [g], 1e-3)
    for args, kw in ((([p], []), {}), (([p.bfloat16()], [g]), {}), (([p], [g[:5]]), {}), (([p], [g.half()]), {}),
                     (([p], [g]), dict(copies=[p])), (([p], [g]), dict(bits=16)), (([p], [g]), dict(weight_decay=[0.1, 0.1])),
                     (([torch.zeros(4, 4).t()[:2]], [torch.zeros(8)]), {}),
                     (([p], [g]), dict(bits=8, states=[(p, p, None, None)])), (([p, p], [g, g]), {}),
                     (([p], [g]), dict(states=[(p, torch.zeros(10), None, None)]))):
        with pytest.raises((ValueError, AttributeError)):
            L.AdamW(*args, 1e-3, **kw)
    opt = L.AdamW([p], [g], 1e-3, bits=8, seed=0xFFFFFFFF, device_scalars=True)
    assert opt.scalars.tolist()[2:] == [0, -1] and opt.states[0][2].numel() == 1
    with pytest.raises(ValueError):
        opt.step(lr=1.0)


def test_layer_asks_for_what_comes_first():
    import torch

    from paper_2605_05607_amd import layer as L
    from paper_2605_05607_amd import workloads as wl
    lay = L.MoELayer(wl.CONFIGS["tiny"].scaled(T=4, dtype=wl.BF16), device="cpu")
    with pytest.raises(ValueError):
        lay.enable_optimizer(None, None, None, 1e-3)
    for w in (torch.ones(512), torch.ones(504, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            lay.enable_norm(w)
    lay.enable_norm(torch.ones(512, dtype=torch.bfloat16))
    assert lay.x.shape == (4, 512) and lay.x_codes.dtype == torch.uint8 and lay.rstd.numel() == 4
