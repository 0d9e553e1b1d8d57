"""What the optimizers refuse, and what a refused or skipped call leaves, without a GPU."""
import ctypes as C

import pytest
import torch

from paper_2605_05607_amd import binding as B
from paper_2605_05607_amd import layer as L
from paper_2605_05607_amd import workloads as wl


@pytest.fixture
def packs(monkeypatch):
    """The library's calls that a layer on the CPU cannot make, by name."""
    calls = []
    for name in ("moe_pack_weights", "moe_pack_weights_backward", "moe_adamw_step"):
        monkeypatch.setattr(B, name, lambda *a, _n=name, **k: calls.append(_n))
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: None)
    return calls


def layer_and_weights():
    cfg = wl.CONFIGS["tiny"].scaled(T=4, dtype=wl.BF16)
    w = wl.make_workload(cfg)
    return L.MoELayer(cfg, device="cpu"), (w.W_gate, w.W_up, w.W_down)


def test_optimizer_asks_for_both_packings(packs):
    lay, w = layer_and_weights()
    lay.enable_training(*w)
    with pytest.raises(ValueError):  # no forward weights to pack a step into
        lay.enable_optimizer(*w, 1e-3)
    with pytest.raises(ValueError):
        lay.optimizer_step()
    lay.load_weights(*w)
    lay.enable_optimizer(*w, 1e-3)
    lay.optimizer_step()
    assert packs[-3:] == ["moe_adamw_step", "moe_pack_weights", "moe_pack_weights_backward"]


def test_optimizer_ends_with_the_weights_and_gradients_that_it_was_made_for(packs):
    """Other weights, or other buffers for the gradients: a step would bring the old weights back, or read gradients that no backward
    pass writes any more."""
    for other in ("load_weights", "enable_training"):
        lay, w = layer_and_weights()
        lay.load_weights(*w)
        lay.enable_training(*w)
        lay.enable_optimizer(*w, 1e-3)
        getattr(lay, other)(*w)
        packs.clear()
        with pytest.raises(ValueError):
            lay.optimizer_step()
        assert not packs
        lay.enable_optimizer(*w, 1e-3)
        lay.optimizer_step()
        assert "moe_adamw_step" in packs


def test_skipped_steps_do_not_count(packs):
    p, g = torch.zeros(10), torch.zeros(10)
    opt = L.AdamW([p], [g], 1e-3, steps=4)
    for scale, steps in ((1.0, 5), (float("inf"), 5), (float("nan"), 5), (0.5, 6), (1e39, 6)):  # (1e39 is infinite in fp32)
        opt.step(grad_scale=scale)
        assert opt.steps == steps
    opt = L.AdamW([p], [g], 1e-3, steps=4, device_scalars=True)
    words = opt.scalars.view(torch.float32)
    for scale, steps in ((1.0, 5), (float("inf"), 5), (float("-inf"), 5), (float("nan"), 5), (0.5, 6)):
        words[1] = scale
        opt.step()
        assert opt.steps == steps
    assert opt.scalars.tolist()[2] == 9  # calls


def test_numbers_of_steps_that_cannot_be():
    t = B.moe_adamw_tensor(None, None, None, None, None, None, None, 0, 0.0, B.MOE_F32)
    for step, skipped, ok in ((1, 0, True), (3, 2, True), (3, 3, False), (1, 1, False), (2, -1, False), (-2 ** 31, 2 ** 31 - 1, False)):
        c = B.moe_adamw_config(0.9, 0.99, 1e-8, 32, B.moe_adamw_device(1e-3, 1.0, step, 0, skipped))
        assert (B.lib().moe_adamw_step(C.byref(c), C.byref(t), 1, None, None) == B.MOE_OK) == ok, (step, skipped)


def test_norm_weight_is_the_layer_s_own_kind_of_memory():
    """The library is given its address: elsewhere or strided it would be read wrongly."""
    lay, _ = layer_and_weights()
    d = lay.shape.d
    for w in (torch.ones(d, dtype=torch.bfloat16, device="meta"), torch.ones((d, 2), dtype=torch.bfloat16)[:, 0]):
        with pytest.raises(ValueError):
            lay.enable_norm(w)
    lay.enable_norm(torch.ones(1, d, dtype=torch.bfloat16))


def test_arrays_of_an_optimizer_do_not_overlap():
    flat, g = torch.zeros(100), torch.zeros(60)
    for p in ([flat[:60], flat[40:]], [flat[40:], flat[:60]], [flat, flat[20:80]]):
        with pytest.raises(ValueError):
            L.AdamW(p, [torch.zeros(t.numel()) for t in p], 1e-3)
    halves = [flat[:50], flat[50:]]
    with pytest.raises(ValueError):  # a gradient that the step of another tensor writes
        L.AdamW(halves, [flat[50:], torch.zeros(50)], 1e-3)
    L.AdamW(halves, [g[:50], g[:50]], 1e-3)  # (one gradient for both is only read)
    L.AdamW([flat[:0], flat[50:50], flat], [g[:0], g[:0], flat + 0], 1e-3)
    state = torch.zeros(100)
    with pytest.raises(ValueError):
        L.AdamW(halves, [g[:50], g[:50]], 1e-3, states=[(state[:50], state[50:], None, None), (state[25:75], flat + 0, None, None)])


def test_refused_step_leaves_the_rate(packs, monkeypatch):
    p, g = torch.zeros(10), torch.zeros(10)
    opt = L.AdamW([p], [g], 1e-3)

    def refuse(*a, **k):
        raise B.MoeError(B.MOE_ERR_INVALID_ARG, "moe_adamw_step")
    with monkeypatch.context() as m:
        m.setattr(B, "moe_adamw_step", refuse)
        with pytest.raises(B.MoeError):
            opt.step(lr=-1.0)
    opt.step()
    assert opt.steps == 1 and abs(opt.config.now.lr - 1e-3) < 1e-9


def test_refused_norm_leaves_what_its_gradient_reads(monkeypatch):
    lay, _ = layer_and_weights()
    lay.enable_norm(torch.ones(lay.shape.d, dtype=torch.bfloat16))
    seen = []
    monkeypatch.setattr(B, "moe_rmsnorm", lambda *a, **k: None)
    monkeypatch.setattr(B, "moe_rmsnorm_backward", lambda rows, cols, dtype, s, *a, **k: seen.append(s))
    h = torch.zeros_like(lay.x)
    lay.norm(h)

    def refuse(*a, **k):
        raise B.MoeError(B.MOE_ERR_INVALID_ARG, "moe_rmsnorm")
    monkeypatch.setattr(B, "moe_rmsnorm", refuse)
    with pytest.raises(B.MoeError):
        lay.norm(h, residual=lay.x)
    lay.norm_backward(lay.x, None, lay.x)
    assert seen[0] is h


def test_steps_can_be_set(packs):
    for device in (False, True):
        opt = L.AdamW([torch.zeros(10)], [torch.zeros(10)], 1e-3, device_scalars=device)
        opt.step()
        opt.steps = 41
        opt.step()
        assert opt.steps == 42
