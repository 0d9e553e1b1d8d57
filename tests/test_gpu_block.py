"""The operators around the expert GEMMs as they are used together: the norm in front of the layer and its codes in the FP8
forward, a whole training step with the optimizer, and experts of the caller's own between the sorting copy and the way back."""
import pytest
import torch

from paper_2605_05607_amd import binding as B
from paper_2605_05607_amd import layer as L
from paper_2605_05607_amd import workloads as wl

pytestmark = pytest.mark.gpu


def layer_of(T, d, f, E, k, R, lo, hi, seed=1, **kw):
    cfg = wl.MoEConfig("block", T=T, d=d, f=f, E=E, k=k, R=R, local_rank_begin=lo, local_rank_end=hi, dtype=wl.BF16,
                       router="normal", seed=seed)
    return cfg, L.MoELayer(cfg), wl.make_workload(cfg)


# weight-streaming kernels; codes beside the tile table; no room for them there (1024 local experts); two launches; no tokens
FP8_SHAPES = [(1, 512, 512, 16, 2, 4), (24, 1024, 512, 16, 4, 4), (700, 272, 128, 64, 8, 8), (300, 32, 64, 4096, 2, 4),
              (2100, 512, 256, 8, 2, 1), (0, 512, 512, 16, 2, 4)]


@pytest.mark.parametrize("T,d,f,E,k,R", FP8_SHAPES)
def test_fp8_forward_from_codes(T, d, f, E, k, R):
    print(f"fp8 codes T={T} d={d} f={f} E={E}", flush=True)
    cfg, lay, w = layer_of(T, d, f, E, k, R, 0, 1)
    lay.load_weights_fp8(w.W_gate, w.W_up, w.W_down, wl.fp8_h_scale(cfg))
    x, logits = (L.to_device(a) if T else torch.zeros(8, device="cuda") for a in (w.x, w.logits))
    lay.route(logits)
    lay.build_dispatch()
    lay.y.fill_(7.0)
    lay.forward_fp8(x)
    want = lay.y.clone()
    codes = torch.empty((max(1, T), d), dtype=torch.uint8, device="cuda")
    scales = torch.empty(max(1, T), device="cuda")
    if T:
        B.moe_fp8_quantize_rows(T, d, x, codes, scales)
    held = codes.clone(), scales.clone()
    for fill in (0xFF, 0x5A):
        lay.fp8_ws.fill_(fill)
        lay.y.fill_(7.0)
        lay.forward_fp8_codes(codes, scales)
        torch.cuda.synchronize()
        assert torch.equal(lay.y, want)
    assert torch.equal(codes, held[0]) and torch.equal(scales, held[1])
    for bad in (dict(scales=None), dict(codes=None), dict(codes=codes.data_ptr() + 8), dict(scales=scales.data_ptr() + 2)):
        a = {"codes": codes, "scales": scales, **bad}
        with pytest.raises(B.MoeError) as err:
            lay.forward_fp8_codes(a["codes"], a["scales"])
        assert err.value.status == B.MOE_ERR_INVALID_ARG


@pytest.mark.parametrize("T", [1, 33, 600])
def test_serving_step_from_the_residual_stream(T):
    """Norm with codes, gate network on its x, tables, FP8 forward from the codes; the bf16 forward on x is 0.5 to 10 % away, as the
    FP8 form from x itself is, and nearer to that form than to it."""
    d, f, E, k, R = 1024, 512, 32, 4, 4
    cfg, lay, w = layer_of(T, d, f, E, k, R, 1, 3, seed=T)
    gen = torch.Generator(device="cuda").manual_seed(T)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    lay.load_weights(w.W_gate, w.W_up, w.W_down)
    lay.load_weights_fp8(w.W_gate, w.W_up, w.W_down, wl.fp8_h_scale(cfg))
    lay.enable_norm(1 + 0.1 * r(d))
    h, res, W_r = r(T, d), 3 * r(T, d), r(E, d) * d ** -0.5
    ws = torch.empty(B.moe_route_from_x_workspace_bytes(lay.shape), dtype=torch.uint8, device="cuda")
    lay.norm(h, res, codes=True)
    assert torch.equal(lay.norm_sum[:T], (h.float() + res.float()).bfloat16())
    B.moe_route_from_x(lay.shape, lay.x, W_r, None, lay.topk_idx, lay.topk_w, ws)
    lay.build_dispatch()
    lay.forward_fp8_codes(lay.x_codes, lay.x_scales)
    own = lay.y_host()
    lay.forward_fp8(lay.x)
    by_x = lay.y_host()
    lay.forward(lay.x)
    full = lay.y_host()
    import numpy as np
    size = np.linalg.norm(full)
    if size == 0:
        assert not own.any()
        return
    off = np.linalg.norm(own - full) / size
    assert 0.005 <= off <= 0.1, off
    # the two sets of codes come from x before and after its rounding to bf16 (2^-8 of it against a code's 2^-4): most agree
    assert np.linalg.norm(own - by_x) / size < off


def plain_block(h, res, wn, Wr, Wg, Wu, Wd, idx, first, eps):
    """The block in torch, differentiable: norm, gate weights of the given picks, local experts, weighted sum."""
    s = h + res
    x = s * (s.square().mean(1, keepdim=True) + eps).rsqrt() * wn
    w = torch.softmax((x @ Wr.t()).gather(1, idx), 1)
    y = torch.zeros_like(x)
    for e in range(len(Wg)):
        t, j = (idx == first + e).nonzero(as_tuple=True)
        if len(t):
            g, u = x[t] @ Wg[e], x[t] @ Wu[e]
            y = y.index_add(0, t, (torch.nn.functional.silu(g) * u) @ Wd[e] * w[t, j][:, None])
    return s, x, y


@pytest.mark.parametrize("bits", [32, 8])
def test_training_step_with_norm_and_optimizer(bits):
    T, d, f, E, k, R = 300, 256, 128, 16, 4, 4
    cfg, lay, w = layer_of(T, d, f, E, k, R, 1, 3, seed=bits)
    gen = torch.Generator(device="cuda").manual_seed(5)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    lay.load_weights(w.W_gate, w.W_up, w.W_down)
    lay.enable_training(w.W_gate, w.W_up, w.W_down)
    lay.enable_norm(1 + 0.1 * r(d))
    lay.enable_optimizer(w.W_gate, w.W_up, w.W_down, 1e-2, weight_decay=0.1, bits=bits, seed=3)
    wn = lay.norm_weight.float()
    opt_n = L.AdamW([wn], [lay.d_norm_weight], 1e-2, copies=[lay.norm_weight], bits=bits)
    W_r = r(E, d) * d ** -0.5
    ws = torch.empty(B.moe_route_from_x_workspace_bytes(lay.shape), dtype=torch.uint8, device="cuda")
    dlogits, dh = torch.empty((T, E), device="cuda"), torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    for step in range(3):
        h, res, dy, dsum = r(T, d), r(T, d), r(T, d), r(T, d)
        lay.norm(h, res)
        B.moe_route_from_x(lay.shape, lay.x, W_r, None, lay.topk_idx, lay.topk_w, ws)
        lay.build_dispatch()
        lay.forward_train(lay.x)
        lay.backward(lay.x, dy)
        B.moe_route_backward(lay.shape, lay.topk_idx, lay.topk_w, lay.d_topk_w, dlogits)
        dx = (lay.dx.float() + dlogits @ W_r.float()).bfloat16()
        lay.norm_backward(dx, dsum, dh)
        torch.cuda.synchronize()
        # the same in fp32 on the host (products of a few hundred terms; bf16 rounds x, h, y and the gradients' way: the layer's
        # own bar, 2e-2 of the largest and 5e-3 of the mean, doubled for the two layers of roundings that a gradient passes)
        leaf = [t.detach().float().cpu().requires_grad_() for t in (h, res, lay.norm_weight, W_r, *lay.weights)]
        idx = lay.topk_idx[: T * k].view(T, k).long().cpu()
        s, _, y = plain_block(*leaf, idx, cfg.first_local_expert, lay.norm_eps)
        ((y * dy.float().cpu()).sum() + (s * dsum.float().cpu()).sum()).backward()
        for name, got, want in (("y", lay.y, y.detach()), ("dh", dh, leaf[0].grad), ("dw", lay.d_norm_weight, leaf[2].grad),
                                ("dW_gate", lay.dW_gate, leaf[4].grad), ("dW_up", lay.dW_up, leaf[5].grad),
                                ("dW_down", lay.dW_down, leaf[6].grad)):
            err = (got.float().cpu() - want).abs()
            assert err.max() <= 4e-2 * want.abs().max() and err.mean() <= 1e-2 * want.abs().mean(), (step, name)
        before = [t.clone() for t in lay.weights]
        lay.optimizer_step()
        opt_n.step()
        assert all(not torch.equal(a, b) for a, b in zip(before, lay.weights))
        assert all(torch.equal(m.bfloat16(), c) for m, c in zip(lay.masters, lay.weights))
        # the packed weights are those of a layer that loads the copies
        other = L.MoELayer(cfg)
        host = [L.from_device_bf16_bits(t) for t in lay.weights]
        other.load_weights(*host)
        other.enable_training(*host)
        for n in ("packed_gate_up", "packed_down", "packed_down_t", "packed_gate_up_t"):
            assert torch.equal(getattr(other, n), getattr(lay, n)), n


def test_captured_training_step():
    """Norm, layer, gradients and both optimizer steps in one graph, replayed with new inputs: the bits of the eager step."""
    T, d, f, E, k, R = 200, 256, 128, 16, 4, 4
    sides = []
    for _ in range(2):
        cfg, lay, w = layer_of(T, d, f, E, k, R, 0, 2, seed=4)
        lay.load_weights(w.W_gate, w.W_up, w.W_down)
        lay.enable_training(w.W_gate, w.W_up, w.W_down)
        lay.enable_norm(torch.ones(d, dtype=torch.bfloat16, device="cuda"))
        lay.enable_optimizer(w.W_gate, w.W_up, w.W_down, 1e-2, bits=8, seed=3, device_scalars=True)
        h, res, dy = (torch.zeros((T, d), dtype=torch.bfloat16, device="cuda") for _ in range(3))
        logits, dh = L.to_device(w.logits), torch.empty_like(h)

        def step(lay=lay, h=h, res=res, dy=dy, logits=logits, dh=dh):
            lay.norm(h, res)
            lay.route(logits)
            lay.build_dispatch()
            lay.forward_train(lay.x)
            lay.backward(lay.x, dy)
            lay.norm_backward(lay.dx, dy, dh)
            lay.optimizer_step()
        step()
        sides.append((lay, (h, res, dy), dh, step))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sides[0][3]()
    gen = torch.Generator(device="cuda").manual_seed(2)
    for turn in range(4):
        for t in range(3):
            v = torch.randn((T, d), generator=gen, device="cuda").bfloat16()
            for s in sides:
                s[1][t].copy_(v)
        torch.cuda.synchronize()
        graph.replay()
        sides[1][3]()
        torch.cuda.synchronize()
        a, b = sides
        for p, q in zip([a[2], a[0].y, a[0].d_norm_weight, *a[0].masters, *a[0].weights, a[0].packed_down, a[0].packed_gate_up_t],
                        [b[2], b[0].y, b[0].d_norm_weight, *b[0].masters, *b[0].weights, b[0].packed_down, b[0].packed_gate_up_t]):
            assert torch.equal(p, q), turn
        assert a[0].y.float().abs().max() > 0


@pytest.mark.parametrize("dtype", [wl.BF16, wl.F32])
def test_own_experts_between_sorting_and_the_way_back(dtype):
    """Experts of the caller's own (a product and a relu), forward and backward, against torch's gradients in fp64 on the host."""
    T, d, E, k, R = 400, 192, 16, 3, 4
    cfg = wl.MoEConfig("own", T=T, d=d, f=8, E=E, k=k, R=R, local_rank_begin=1, local_rank_end=3, dtype=dtype, router="zipf", seed=6)
    lay, w = L.MoELayer(cfg), wl.make_workload(cfg, weights=False)
    dt, first, El = lay.elt_dtype, cfg.first_local_expert, cfg.E_loc
    x = L.to_device(w.x)
    gen = torch.Generator(device="cuda").manual_seed(7)
    W = (torch.randn((El, d, d), generator=gen, device="cuda") * d ** -0.5).to(dt)
    dy = torch.randn((T, d), generator=gen, device="cuda").to(dt)
    lay.route(L.to_device(w.logits))
    lay.build_dispatch()
    off = (lay.tables.offsets[first: first + El + 1] - lay.tables.offsets[first]).tolist()
    new = lambda: torch.zeros((T * min(k, El), d), dtype=dt, device="cuda")  # noqa: E731
    xs, rows, d_rows, d_xs, dW = new(), new(), new(), new(), torch.zeros_like(W)
    y, dx, d_w = torch.empty_like(dy), torch.empty_like(dy), torch.empty((T, k), device="cuda")
    B.moe_dispatch_gather(lay.shape, x, lay.tables, xs)
    for e in range(El):
        rows[off[e]: off[e + 1]] = torch.relu(xs[off[e]: off[e + 1]] @ W[e])
    B.moe_combine_weighted(lay.shape, rows, lay.topk_idx, lay.topk_w, lay.tables, y)
    B.moe_combine_weighted_backward(lay.shape, rows, dy, lay.topk_idx, lay.topk_w, lay.tables, d_rows, d_w)
    for e in range(El):
        s = slice(off[e], off[e + 1])
        g = d_rows[s] * (rows[s] > 0)
        d_xs[s] = g @ W[e].t().contiguous()
        dW[e] = xs[s].t().contiguous() @ g
    B.moe_dispatch_gather_backward(lay.shape, d_xs, lay.topk_idx, lay.tables, dx)
    torch.cuda.synchronize()
    X, V, gate = (t.double().cpu().requires_grad_() for t in (x, W, lay.topk_w[: T * k].view(T, k)))
    idx = lay.topk_idx[: T * k].view(T, k).cpu()
    Y = torch.zeros((T, d), dtype=torch.float64)
    for e in range(El):
        t, j = (idx == first + e).nonzero(as_tuple=True)
        Y = Y.index_add(0, t, torch.relu(X[t] @ V[e]) * gate[t, j][:, None])
    (Y * dy.double().cpu()).sum().backward()
    # bf16: each array on the way rounds by 2^-8, three or four of them in a chain; fp32: sums of some hundred products
    bar = 3e-2 if dtype == wl.BF16 else 1e-5
    for name, got, want in (("y", y, Y.detach()), ("dx", dx, X.grad), ("d_w", d_w, gate.grad), ("dW", dW, V.grad)):
        err = (got.double().cpu() - want).abs()
        assert err.max() <= bar * want.abs().max() and err.mean() <= bar / 4 * want.abs().mean(), name
