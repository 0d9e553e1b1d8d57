"""The layer's optimizer step: every packed form of the weights is that of a layer that has loaded the new ones."""
import pytest
import torch

from paper_2605_05607_amd import layer as L
from paper_2605_05607_amd import workloads as wl

pytestmark = pytest.mark.gpu
T, D, F_, E, K = 96, 256, 128, 16, 4


def layer_of(fp8, **kw):
    cfg = wl.MoEConfig("optimizer", T=T, d=D, f=F_, E=E, k=K, R=4, local_rank_begin=0, local_rank_end=2, dtype=wl.BF16,
                       router="normal", seed=8)
    lay, w = L.MoELayer(cfg), wl.make_workload(cfg)
    lay.load_weights(w.W_gate, w.W_up, w.W_down)
    if fp8:
        lay.load_weights_fp8(w.W_gate, w.W_up, w.W_down, wl.fp8_h_scale(cfg))
    lay.enable_training(w.W_gate, w.W_up, w.W_down)
    lay.enable_norm(torch.ones(D, dtype=torch.bfloat16, device="cuda"))
    lay.enable_optimizer(w.W_gate, w.W_up, w.W_down, 1e-2, bits=8, **kw)
    lay.route(L.to_device(w.logits))
    lay.build_dispatch()
    gen = torch.Generator(device="cuda").manual_seed(1)
    h, dy = (torch.randn((T, D), generator=gen, device="cuda").bfloat16() for _ in range(2))
    return cfg, lay, w, h, dy


def train(lay, h, dy):
    lay.norm(h, codes=True)
    lay.forward_train(lay.x)
    lay.backward(lay.x, dy)
    lay.optimizer_step()


def fp8_of_loaded(cfg, lay):
    """y of the FP8 forward of a layer that loads the present weights."""
    other = L.MoELayer(cfg)
    other.load_weights_fp8(*[L.from_device_bf16_bits(t) for t in lay.weights], wl.fp8_h_scale(cfg))
    other.topk_idx.copy_(lay.topk_idx)
    other.topk_w.copy_(lay.topk_w)
    other.build_dispatch()
    other.forward_fp8_codes(lay.x_codes, lay.x_scales)
    torch.cuda.synchronize()
    assert torch.equal(other.fp8_gate_up, lay.fp8_gate_up) and torch.equal(other.fp8_down, lay.fp8_down)
    return other.y


def test_fp8_forward_after_a_step():
    cfg, lay, _, h, dy = layer_of(True)
    lay.norm(h, codes=True)
    lay.forward_fp8_codes(lay.x_codes, lay.x_scales)
    before = lay.y.clone()
    for _ in range(2):
        train(lay, h, dy)
        lay.forward_fp8_codes(lay.x_codes, lay.x_scales)
        torch.cuda.synchronize()
        assert torch.equal(lay.y, fp8_of_loaded(cfg, lay))
    assert not torch.equal(lay.y, before)


def test_fp8_weights_loaded_behind_the_optimizer():
    cfg, lay, w, h, dy = layer_of(False)
    lay.load_weights_fp8(w.W_gate, w.W_up, w.W_down, wl.fp8_h_scale(cfg))
    train(lay, h, dy)
    lay.forward_fp8_codes(lay.x_codes, lay.x_scales)
    torch.cuda.synchronize()
    assert torch.equal(lay.y, fp8_of_loaded(cfg, lay))


def test_fp8_weights_in_a_captured_step():
    cfg, lay, _, h, dy = layer_of(True, device_scalars=True)
    train(lay, h, dy)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        train(lay, h, dy)
    for turn in range(3):
        graph.replay()
        torch.cuda.synchronize()
        lay.forward_fp8_codes(lay.x_codes, lay.x_scales)
        torch.cuda.synchronize()
        same = torch.equal(lay.y, fp8_of_loaded(cfg, lay))
        assert same, turn


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("captured", [False, True])
def test_first_steps_that_are_skipped(bits, captured):
    """Steps skipped for a scale that is not finite, at the start and between others: the bits of a run without them."""
    gen = torch.Generator(device="cuda").manual_seed(bits)
    r = lambda n: torch.randn(n, generator=gen, device="cuda")  # noqa: E731
    sizes = [70000, 33]
    start, grads = [r(n) for n in sizes], [[r(n) for n in sizes] for _ in range(4)]
    runs = []
    for skips in (False, True):
        params, g = [p.clone() for p in start], [torch.empty(n, device="cuda") for n in sizes]
        opt = L.AdamW(params, g, 1e-2, bits=bits, seed=9, device_scalars=captured and skips)
        step = opt.step
        if opt.scalars is not None:
            opt.step()  # (with whatever the gradients hold: undone below)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                opt.step()
            for t, p in zip(params, start):
                t.copy_(p)
            for s in opt.states:
                for t in s[:2]:
                    t.zero_()
                for t in s[2:] if bits == 8 else ():
                    t.fill_(1)
            opt._device[2:5:2] = 0
            words = opt.scalars.view(torch.float32)

            def step(grad_scale=1.0, words=words, graph=graph):
                words[1] = grad_scale
                graph.replay()
        for turn, values in enumerate(grads):
            for t, v in zip(g, values):
                t.copy_(v)
            if skips and turn != 2:
                for scale in (float("inf"), float("nan"))[: 1 + turn % 2]:
                    step(grad_scale=scale)
            step()
        torch.cuda.synchronize()
        assert opt.steps == 4
        runs.append(params + [t for s in opt.states for t in s if t is not None])
    for a, b in zip(*runs):
        same = torch.equal(a, b)
        assert same


def test_first_step_behind_skipped_ones_has_its_size():
    """A fresh state's first step is lr g / (|g| + eps), here lr, whatever was skipped before it.  Tolerance: 64 steps of fp32 in the
    update, half a step in the parameter (1 at most)."""
    for bits in (32, 8):
        for device in (False, True):
            p, g = torch.zeros(1000, device="cuda"), torch.full((1000,), -3.0, device="cuda")
            opt = L.AdamW([p], [g], 1e-3, bits=bits, device_scalars=device)
            for scale in (float("inf"),) * 5 + (1.0,):
                if device:
                    opt.scalars.view(torch.float32)[1] = scale
                    opt.step()
                else:
                    opt.step(grad_scale=scale)
            off = (p.double() - 1e-3).abs().max().item()
            assert off <= 1e-3 * 64 * 2.0 ** -24, (bits, device, off)
            assert opt.steps == 1
