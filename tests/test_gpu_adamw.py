"""AdamW steps over lists of tensors with states in 32 and in 8 bits, against float64.

Tolerances, derived (u = 2^-24, half an fp32 step): a new m or v is two products and an addition, 3 u of the terms' magnitudes; the
square root and the reciprocal of the step are one step each (2 u), with the products around them and the two bias corrections
(each a few u of 1 - b^t) below 32 u of the update; the parameter adds 3 u of itself.   8-bit codes: see codes_of."""
import pytest
import torch

from paper_2605_05607_amd import binding as B
from paper_2605_05607_amd import layer as L

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BLOCK = B.MOE_ADAMW_BLOCK
M32 = 0xFFFFFFFF


def mix(z):
    z = (z ^ (z >> 16)) * 0x6A09E667 & M32
    z = (z ^ (z >> 15)) * 0xBB67AE85 & M32
    return z ^ (z >> 16)


def hash_of(i, seed, step, tensor):
    key = mix((seed + mix((step + mix((tensor + 0x9E3779B9) & M32)) & M32)) & M32)
    return mix((i & M32) ^ mix((i >> 32) + key & M32))


def blocks_of(v):
    return torch.nn.functional.pad(v, (0, -v.numel() % BLOCK)).view(-1, BLOCK)


def decode(codes, scale):
    return codes.view(torch.float8_e4m3fn).double() * scale.double().repeat_interleave(BLOCK)[: codes.numel()]


def codes_of(v, scale, bits16, least, off):
    """Codes of float64 values, rounded stochastically, and which of them fp32 arithmetic may see otherwise.  off: how far the
    quotient v / scale may be off, relative to itself; a code's step is 1/16 to 1/8 of the quotient, so that moves what is cut off by
    16 off of the 2^20 parts of a step at most: off / u of them."""
    q = (v / scale.double().repeat_interleave(BLOCK)[: v.numel()]).abs().clamp(max=448.0)
    exp = torch.floor(torch.log2(q.clamp(min=2.0 ** -6)))
    exp = torch.where(2.0 ** exp > q.clamp(min=2.0 ** -6), exp - 1, exp)
    steps = q / 2.0 ** (exp - 3)  # 8 to 16, or 0 to 8 below 2^-6
    low = torch.floor(steps)
    cut = (steps - low) * 2 ** 20 + bits16.double() * 16 - 2 ** 20
    near = 1 + off / U
    unsure = (cut.abs() <= near) | ((steps - low) * 2 ** 20 <= near) | ((1 - (steps - low)) * 2 ** 20 <= near)
    unsure &= v != 0  # (zero is exact)
    code = ((exp + 6) * 8 + low + (cut >= 0)).long()
    if least:
        code = torch.where(v > 0, code.clamp(min=1), code)
    return code | ((v < 0).long() << 7), unsure


def check_state(codes, scale, value, tol, rnd, least):
    """One state's codes and scales against its float64 values, which fp32 knows to within tol (an array)."""
    n = value.numel()
    top = blocks_of(value).abs().amax(1)
    want = torch.where(top > 0, top / 448, torch.ones_like(top))
    tol_scale = blocks_of(tol).amax(1) / 448 + 4 * U * want  # two blocks' maxima differ by no more than their values do
    assert ((scale.double() - want).abs() <= tol_scale).all()
    off = tol / value.abs().clamp(min=1e-300) + (tol_scale / want).repeat_interleave(BLOCK)[:n] + 4 * U
    ref, unsure = codes_of(value, want, rnd, least, off)
    assert torch.equal(codes.long()[~unsure], ref[~unsure])
    assert unsure.double().mean() < 0.05 or n < 1000  # (nearly all are compared)


def make(sizes, bits, gdt, copy, seed=0, fresh=False, device="cuda"):
    gen = torch.Generator(device=device).manual_seed(seed)
    r = lambda n: torch.randn(n, generator=gen, device=device)  # noqa: E731
    params, grads, copies, states = [], [], [], []
    for n in sizes:
        size = 1e-3 * torch.exp(2 * r(n))
        params.append(0.02 * r(n))
        g = size * r(n)
        g[::7] = 0
        grads.append(g.to(gdt))
        copies.append(torch.full((n,), 7.0, dtype=torch.bfloat16, device=device) if copy else None)
        m, root = 0.3 * size * r(n), size * (0.2 + torch.rand(n, generator=gen, device=device))
        root[5::11], m[5::11] = 0, 0
        if bits == 32:
            states.append((m, root.square(), None, None))
        else:
            st = []
            for t in (m, root):
                b = blocks_of(t)
                top = b.abs().amax(1)
                sc = torch.where(top > 0, top / 448, torch.ones_like(top))
                st.append(((b / sc[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).view(-1)[:n].contiguous(), sc))
            states.append((st[0][0], st[1][0], st[0][1], st[1][1]))
    return params, grads, copies, None if fresh else states


def reference(p, g, m, v, step, lr, b1, b2, eps, decay, scale=1.0):
    """float64 step; the new values and the tolerances of m, v and the parameter."""
    g = g.double() * scale
    m2, v2 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    tol_m, tol_v = 4 * U * (b1 * m.abs() + (1 - b1) * g.abs()), 5 * U * v2
    down = (v2 / (1 - b2 ** step)).sqrt() + eps
    rate = lr / (1 - b1 ** step)
    update = rate * m2 / down
    new = p.double() * (1 - lr * decay) - update
    return m2, v2, new, tol_m, tol_v, 3 * U * p.double().abs() + 32 * U * update.abs() + rate * tol_m / down + 2.0 ** -140


LISTS = [[1], [3, 0, 255], [256, 257, 4095, 4096, 4097], [8191, 1, 70001, 12], [5] * 39 + [4096] * 2 + [1 << 20, 7] + [300] * 45]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: f"{len(s)}x{max(s)}")
def test_steps_against_float64(sizes, bits):
    print("adamw", bits, len(sizes), max(sizes), flush=True)
    lr, b1, b2, eps, seed = 1e-3, 0.9, 0.99, 1e-8, 12345
    for gdt, copy, first in ((torch.bfloat16, True, 1), (torch.float32, False, 700)):
        params, grads, copies, states = make(sizes, bits, gdt, copy, 3, fresh=first == 1)
        decay = [0.1 * (i % 3) for i in range(len(sizes))]
        opt = L.AdamW(params, grads, lr, b1, b2, eps, decay, copies, bits, seed, states, steps=first - 1)
        for step in (first, first + 1, first + 2):
            old = [p.clone() for p in params]
            held = [[None if t is None else t.clone() for t in s] for s in opt.states]
            opt.step()
            torch.cuda.synchronize()
            assert opt.steps == step
            for k, (p, g, o, h, now) in enumerate(zip(params, grads, old, held, opt.states)):
                if p.numel() == 0:
                    continue
                m = h[0].double() if bits == 32 else decode(h[0], h[2])
                v = h[1].double() if bits == 32 else decode(h[1], h[3]).square()
                m2, v2, new, tol_m, tol_v, tol_p = reference(o, g, m, v, step, lr, b1, b2, eps, decay[k])
                assert ((p.double() - new).abs() <= tol_p).all(), (k, step)
                if copy:
                    assert torch.equal(copies[k], p.to(torch.bfloat16))
                if bits == 32:
                    assert ((now[0].double() - m2).abs() <= tol_m).all() and ((now[1].double() - v2).abs() <= tol_v).all()
                    continue
                h32 = hash_of(torch.arange(p.numel(), device="cuda"), seed, step, k)
                for value, codes, scale, rnd, least in ((m2, now[0], now[2], h32 & 0xFFFF, False),
                                                        (v2.sqrt(), now[1], now[3], h32 >> 16, True)):
                    check_state(codes, scale, value, 16 * U * value if least else tol_m, rnd, least)


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_and_copies_of_both_kinds_in_one_list(bits):
    """Each tensor gets what it gets in a list of its own kind (32 bits), or at its own place of the list (8: the hash)."""
    sizes = [700, 4097, 256, 9000, 0, 31]
    sets = []
    for kinds in (("b", "f", "b", "f", "f", "b"), "bbbbbb", "ffffff"):
        params, grads, _, states = make(sizes, bits, torch.bfloat16, False, 12)
        grads = [g if k == "b" else g.float() for g, k in zip(grads, kinds)]  # (the same values)
        copies = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") if k == "b" else None for n, k in zip(sizes, kinds)]
        L.AdamW(params, grads, 1e-3, copies=copies, bits=bits, states=states, steps=5, seed=2).step()
        assert all(c is None or torch.equal(c, p.bfloat16()) for c, p in zip(copies, params))
        sets.append(params + [t for s in states for t in s if t is not None])
    for other in sets[1:]:
        assert all(torch.equal(a, b) for a, b in zip(sets[0], other))


def test_lists_without_values():
    L.AdamW([], [], 1e-3).step()
    for bits in (32, 8):
        p = torch.zeros(0, device="cuda")
        L.AdamW([p], [p], 1e-3, bits=bits).step()
    torch.cuda.synchronize()


def test_rounding_has_no_bias():
    """Values between two codes: the mean of what is held is the value.  n draws of a part f of a step d: standard deviation
    d sqrt(f (1 - f) / n), and the 16 bits are off by at most d 2^-16."""
    n = BLOCK * 4000
    for part in (0.5, 0.1, 0.93):
        for base in (16.0, 0.0009765625):  # codes 8/8 of an octave, and half a step of the subnormal codes
            value = base * (1 + part / 8) if base >= 1 else 2.0 ** -9 * (3 + part)
            g = torch.full((n,), value, device="cuda")
            g[::BLOCK] = 448.0
            p = torch.zeros(n, device="cuda")
            opt = L.AdamW([p], [g], 0.0, 0.0, 0.0, 1e-8, bits=8, seed=77)  # beta 0: m = g and sqrt(v) = |g|
            opt.step()
            d = base / 8 if base >= 1 else 2.0 ** -9
            keep = torch.arange(n, device="cuda") % BLOCK != 0
            for codes, scale in (opt.states[0][::2], opt.states[0][1::2]):
                held = decode(codes, scale)[keep]
                assert ((held - value).abs() < d * 1.001).all()
                sd = d * (part * (1 - part) / held.numel()) ** 0.5
                assert abs(held.mean().item() - value) <= 5 * sd + d * 2.0 ** -15, (part, base)


def test_states_in_8_bits_keep_moving():
    """A gradient that shrinks tenfold: sqrt(v) falls by 0.05 % a step, far less than half a code, and has to follow.
    Every element of a block but the first; tolerance: the mean over 65000 elements of walks whose steps are rounded without bias
    (each rounding at most d / 2 off, 200 steps: sd of one walk below sqrt(200) d / 2, of the mean below it / sqrt(65000) = d / 36),
    and 1 % for the curvature of the square (sqrt(v) is rounded without bias, v is not: d^2 / 4 of v = 0.4 % a step at most,
    taken in by 1 - b2 = 0.1 % of... the bound below is checked against the same walk in float64)."""
    n, b2, steps = 1 << 16, 0.999, 200
    g = torch.full((n,), 0.01, device="cuda")
    g[::BLOCK] = 1.0
    p = torch.zeros(n, device="cuda")
    root = torch.full((n,), 0.1, device="cuda")
    root[::BLOCK] = 1.0
    sc = torch.full((n // BLOCK,), 1 / 448.0, device="cuda")
    codes = (root * 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    opt = L.AdamW([p], [g], 0.0, 0.9, b2, 1e-8, bits=8, seed=5,
                  states=[(torch.zeros(n, dtype=torch.uint8, device="cuda"), codes.clone(), sc.clone(), sc.clone())], steps=1000)
    start = decode(codes, sc)[1].item()
    # the same walk in float64 on the CPU with numpy's random numbers
    import numpy as np
    rng = np.random.default_rng(1)
    w = np.full(n, start)
    for _ in range(steps):
        x = np.sqrt(b2 * w * w + (1 - b2) * 1e-4) * 448.0
        d = 2.0 ** (np.floor(np.log2(x)) - 3)
        low = np.floor(x / d)
        w = (low + (rng.random(n) < x / d - low)) * d / 448.0
        opt.step()
    held = decode(opt.states[0][1], opt.states[0][3])
    keep = torch.arange(n, device="cuda") % BLOCK != 0
    mean = held[keep].mean().item()
    free = (b2 ** steps * start ** 2 + (1 - b2 ** steps) * 1e-4) ** 0.5
    assert abs(mean - w.mean()) <= 6 * w.std() / (n ** 0.5) * 1.5  # two samples of the same walk
    assert start - mean > 0.5 * (start - free)  # and it has moved


def test_small_gradients_with_a_small_eps():
    """Gradients whose second state is subnormal in fp32 (below 1.2e-38), and zeros: a fresh state's first step is -lr g / (|g| + eps),
    which for these is lr away from 0.  Tolerance: v = (1 - b2) g^2 is off by half a subnormal step, 2^-150, its root by half of that relative to
    v (below 2e-3: 1 % for what is left out of the series); else the 32 u of an update."""
    n, lr, eps = 4096, 1e-3, 1e-30
    grad = 10 ** (torch.rand(n, generator=torch.Generator().manual_seed(5), dtype=torch.float64) * 4.7 - 19.7)
    grad = (grad * (1 - 2 * (torch.arange(n) % 2))).float()
    grad[::7] = 0
    grad = grad.cuda()
    p = torch.zeros(n, device="cuda")
    L.AdamW([p], [grad], lr, 0.9, 0.999, eps).step()
    g = grad.double()
    off = 2.0 ** -150 / (1e-3 * g * g).clamp(min=1e-43) / 2 * 1.01 + 32 * U
    assert ((p.double() + lr * g / (g.abs() + eps)).abs() <= lr * off).all()
    assert (p[::7] == 0).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_skipped_step_changes_nothing(bits):
    sizes = [5000, 33]
    params, grads, copies, states = make(sizes, bits, torch.bfloat16, True, 9)
    opt = L.AdamW(params, grads, 1e-3, copies=copies, bits=bits, states=states, steps=10)
    everything = params + copies + [t for s in states for t in s if t is not None]
    before = [t.clone() for t in everything]
    for scale in (float("nan"), float("inf"), float("-inf")):
        opt.step(grad_scale=scale)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(everything, before))
    opt.step(grad_scale=0.5)
    assert not torch.equal(params[0], before[0])


def test_gradient_scale_is_that_of_scaled_gradients():
    for bits in (32, 8):
        sets = []
        for scale in (1.0, 0.25):  # a power of two: the same bits
            params, grads, _, states = make([3001], bits, torch.float32, False, 4)
            grads = [g / scale for g in grads]
            opt = L.AdamW(params, grads, 1e-3, bits=bits, states=states, steps=3, seed=8)
            opt.step(grad_scale=scale)
            sets.append(params + [t for t in states[0] if t is not None])
        assert all(torch.equal(a, b) for a, b in zip(*sets))


def test_gradients_that_are_not_finite_stay_in_their_block():
    for bits in (32, 8):
        out = []
        for bad in (False, True):
            params, grads, _, states = make([20 * BLOCK + 9], bits, torch.float32, False, 4)
            if bad:
                grads[0][3 * BLOCK + 5] = float("nan")
                grads[0][7 * BLOCK + 1] = float("inf")
            opt = L.AdamW(params, grads, 1e-3, bits=bits, states=states, steps=3)
            opt.step()
            opt.step()
            out.append((params[0], *(states[0][:2] if bits == 32 else (decode(states[0][0], states[0][2]),
                                                                      decode(states[0][1], states[0][3])))))
        keep = torch.ones(20 * BLOCK + 9, dtype=torch.bool, device="cuda")
        if bits == 32:
            keep[[3 * BLOCK + 5, 7 * BLOCK + 1]] = False
        else:
            keep[3 * BLOCK: 4 * BLOCK] = keep[7 * BLOCK: 8 * BLOCK] = False
        for a, b in zip(*out):
            assert torch.equal(a[keep], b[keep])
        assert torch.isnan(out[1][0][3 * BLOCK + 5]) and not torch.isfinite(out[1][2][~keep]).any()
        if bits == 8:  # the whole block shows it after the next step
            assert torch.isnan(out[1][0][3 * BLOCK: 4 * BLOCK]).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_values_between_the_tensors_are_left_alone(bits):
    sizes = [1, 5, 250, 300, 4099]
    gap = 512
    flat = [torch.full((sum(-(-n // BLOCK) * BLOCK + gap for n in sizes),), 7.0, device="cuda", dtype=dt)
            for dt in (torch.float32, torch.bfloat16, *((torch.float32,) * 2 if bits == 32 else (torch.uint8,) * 2))]
    grads = torch.randn(flat[0].numel(), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    at, pieces = gap // 2, []
    for n in sizes:
        pieces.append((at, n))
        at += -(-n // BLOCK) * BLOCK + gap
    cut = lambda t: [t[a: a + n] for a, n in pieces]  # noqa: E731
    scales = [tuple(torch.ones(-(-n // BLOCK), device="cuda") if bits == 8 else None for _ in range(2)) for n in sizes]
    states = [(m, v, *s) for m, v, s in zip(cut(flat[2]), cut(flat[3]), scales)]
    opt = L.AdamW(cut(flat[0]), cut(grads), 1e-2, copies=cut(flat[1]), bits=bits, states=states)
    opt.step()
    torch.cuda.synchronize()
    inside = torch.zeros(flat[0].numel(), dtype=torch.bool, device="cuda")
    for a, n in pieces:
        inside[a: a + n] = True
    for t in flat:
        assert (t[~inside] == 7).all()
    # an update below half a step of 7.0 (2.4e-7 of lr = 1e-2: a new m below 2.4e-5 of its size, one in 10^4) leaves it as it is
    assert (flat[0][inside] != 7).double().mean() > 0.99


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_advance(bits):
    """Device scalars: replays take the next step each, with a rate and a scale written between them; the same bits as steps
    whose numbers come from the host."""
    sizes = [70000, 256, 3]
    a, b = (make(sizes, bits, torch.bfloat16, True, 6, fresh=True) for _ in range(2))
    host = L.AdamW(*a[:2], 1e-3, copies=a[2], bits=bits, seed=(1 << 32) - 5, weight_decay=0.1)
    dev = L.AdamW(*b[:2], 1e-3, copies=b[2], bits=bits, seed=(1 << 32) - 5, weight_decay=0.1, device_scalars=True)
    dev.step()
    host.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        dev.step()
    torch.cuda.synchronize()
    words = dev.scalars.view(torch.float32)
    for turn in range(5):
        lr, scale = 1e-3 / (1 + turn), 1.0 if turn != 3 else float("nan")
        words[:2] = torch.tensor([lr, scale], device="cuda")
        fresh = torch.randn(sizes[0], device="cuda").bfloat16()
        a[1][0].copy_(fresh)
        b[1][0].copy_(fresh)
        torch.cuda.synchronize()
        graph.replay()
        host.step(lr=float(torch.tensor(lr)), grad_scale=scale)
        torch.cuda.synchronize()
        for s, t in zip(a[0] + a[2] + [x for st in host.states for x in st if x is not None],
                        b[0] + b[2] + [x for st in dev.states for x in st if x is not None]):
            assert torch.equal(s, t), turn
    assert dev.scalars[2].item() == 6 + 0 * turn


def test_elements_past_32_bits_of_index():
    n = (1 << 32) + 4096 + 3
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(8195, device="cuda") * 1e-3
    at = n - 8195
    g[at:] = tail.bfloat16()
    opt = L.AdamW([p], [g], 1e-3, 0.9, 0.99, 1e-8, bits=8, seed=4)
    opt.step()
    torch.cuda.synchronize()
    m2, v2, new, *_, tol = reference(torch.zeros(8195, device="cuda"), g[at:], torch.zeros((), device="cuda").double(),
                                     torch.zeros((), device="cuda").double(), 1, 1e-3, 0.9, 0.99, 1e-8, 0.0)
    assert ((p[at:].double() - new).abs() <= tol).all() and not p[:1 << 20].any() and not p[at - (1 << 20): at].any()
    start = (1 << 32)  # a block's edge
    h = hash_of(torch.arange(start, n, device="cuda"), 4, 1, 0)
    for value, codes, scale, rnd, least in ((m2, opt.states[0][0], opt.states[0][2], h & 0xFFFF, False),
                                            (v2.sqrt(), opt.states[0][1], opt.states[0][3], h >> 16, True)):
        check_state(codes[start:], scale[start // BLOCK:], value[start - at:], 16 * U * value[start - at:].abs(), rnd, least)
