"""8-bit states of AdamW bit for bit: the formulas evaluated in fp32, one rounding an operation, on the host.  Scales are largest
magnitude times fp32's 1/448; codes take the hash's bits.  Nothing is left to a tolerance."""
import numpy as np
import pytest
import torch

from paper_2605_05607_amd import binding as B
from paper_2605_05607_amd import layer as L

pytestmark = pytest.mark.gpu
BLOCK = B.MOE_ADAMW_BLOCK
F = np.float32


def mix(z):
    z = ((z ^ (z >> np.uint64(16))) * np.uint64(0x6A09E667)) & np.uint64(0xFFFFFFFF)
    z = ((z ^ (z >> np.uint64(15))) * np.uint64(0xBB67AE85)) & np.uint64(0xFFFFFFFF)
    return z ^ (z >> np.uint64(16))


def hash_of(n, seed, step, tensor):
    u = lambda v: np.uint64(v & 0xFFFFFFFF)  # noqa: E731
    key = int(mix(u(seed + int(mix(u(step + int(mix(u(tensor + 0x9E3779B9)))))))))
    return mix(np.arange(n, dtype=np.uint64) ^ mix(u(key)))


def decode(codes, scale):
    v = torch.from_numpy(codes).view(torch.float8_e4m3fn).float().numpy()
    return v * np.repeat(scale, BLOCK)[: len(v)]


def encode(v, bits16, least):
    blocks = np.pad(np.abs(v), (0, -len(v) % BLOCK)).reshape(-1, BLOCK)
    top = blocks.max(1)
    scale = np.where(top > 0, top * (F(1) / F(448)), F(1)).astype(F)
    q = np.abs(v) / np.repeat(scale, BLOCK)[: len(v)]
    bits = np.minimum(q * F(2.0 ** -120), F(448 * 2.0 ** -120)).view(np.uint32)
    code = (bits + (bits16.astype(np.uint32) << np.uint32(4))) >> np.uint32(20)
    if least:
        code = np.where(v > 0, np.maximum(code, 1), code)
    return (code | (np.signbit(v).astype(np.uint32) << np.uint32(7))).astype(np.uint8), scale


@pytest.mark.parametrize("grads", [torch.bfloat16, torch.float32])
def test_states_are_those_of_the_formulas_in_fp32(grads):
    sizes, b1, b2, seed, first = [70001, 1, 300, 0, 4096, 1 << 18], 0.9, 0.99, 99, 5
    rng = np.random.default_rng(3)
    new = lambda n: (rng.standard_normal(n) * np.exp(2 * rng.standard_normal(n))).astype(F)  # noqa: E731
    params = [torch.zeros(n, device="cuda") for n in sizes]
    g = [torch.from_numpy(new(n) * F(1e-3)).cuda().to(grads) for n in sizes]
    opt = L.AdamW(params, g, 1e-3, b1, b2, bits=8, seed=seed, steps=first - 1)
    held = [[t.cpu().numpy() for t in s] for s in opt.states]
    for step in range(first, first + 4):
        for t, n in zip(g, sizes):
            t.copy_(torch.from_numpy(new(n) * F(1e-3)).to(grads))
        opt.step()
        for k, n in enumerate(sizes):
            grad, rnd = g[k].float().cpu().numpy(), hash_of(n, seed, step, k)
            m, root = decode(held[k][0], held[k][2]), decode(held[k][1], held[k][3])
            m = F(b1) * m + F(1 - b1) * grad
            v = F(b2) * (root * root) + F(1 - b2) * grad * grad
            want = [None] * 4
            want[0], want[2] = encode(m, rnd & np.uint64(0xFFFF), False)
            want[1], want[3] = encode(np.sqrt(v), rnd >> np.uint64(16), True)
            for name, a, b in zip(("m", "v", "m_scale", "v_scale"), opt.states[k], want):
                off = int((a.cpu().numpy() != b).sum())
                assert off == 0, (step, k, name)
            held[k] = want
