"""8-bit lists of more than 2^22 values, whose waves take four blocks of 256 values each: states to go on from, tensors that end at
and around a workgroup's 4096 values and in each of a wave's blocks, and lists of which one launch takes this form and one the other.
Against float64 with the tolerances of test_gpu_adamw."""
import pytest
import torch

import test_gpu_adamw as A
from paper_2605_05607_amd import layer as L

pytestmark = pytest.mark.gpu
C = 4096
ENDS = [3 * C - 1, 3 * C, 3 * C + 1, C + 255, C + 256, C + 300, 2 * C + 511, 2 * C + 600, 2 * C + 767, C + 900, 5 * C + 1024, 5 * C + 1025,
        5 * C + 2048 + 257, 5 * C + 3 * 1024 + 513, 5 * C + 4095, 1, 0, 3, 255]
LISTS = {"one": [(1 << 22) + 1], "at the line": [1 << 22], "ends": ENDS + [1 << 22] + ENDS,
         "many first": [200000 + 7 * i for i in range(40)] + [300, 4097, 70001, 0, 9], "few first": [5000 + i for i in range(40)] + [(1 << 22) + 777, 513]}


@pytest.mark.parametrize("gdt,copy", [(torch.bfloat16, True), (torch.float32, False)])
@pytest.mark.parametrize("name", LISTS)
def test_steps_against_float64(name, gdt, copy):
    sizes, lr, b1, b2, eps, seed, first = LISTS[name], 1e-3, 0.9, 0.99, 1e-8, 777, 30
    print("adamw", name, len(sizes), sum(sizes), gdt, flush=True)
    params, grads, copies, states = A.make(sizes, 8, gdt, copy, 4)
    decay = [0.1 * (i % 3) for i in range(len(sizes))]
    opt = L.AdamW(params, grads, lr, b1, b2, eps, decay, copies, 8, seed, states, steps=first - 1)
    for step in (first, first + 1):
        old, held = [p.clone() for p in params], [[t.clone() for t in s] for s in opt.states]
        opt.step()
        torch.cuda.synchronize()
        for k, (p, g, o, h, now) in enumerate(zip(params, grads, old, held, opt.states)):
            if p.numel() == 0:
                continue
            m2, v2, new, tol_m, _, tol_p = A.reference(o, g, A.decode(h[0], h[2]), A.decode(h[1], h[3]).square(), step, lr, b1, b2,
                                                       eps, decay[k])
            assert bool(((p.double() - new).abs() <= tol_p).all()), (k, step)
            assert copies[k] is None or torch.equal(copies[k], p.to(torch.bfloat16)), (k, step)
            rnd = A.hash_of(torch.arange(p.numel(), device="cuda"), seed, step, k)
            A.check_state(now[0], now[2], m2, tol_m, rnd & 0xFFFF, False)
            A.check_state(now[1], now[3], v2.sqrt(), 16 * A.U * v2.sqrt(), rnd >> 16, True)


def test_both_forms_write_the_same():
    """A tensor at its place in a list gets the same bits whichever form its launch takes."""
    small = [70001, 4097, 300]
    out = []
    for rest in ([], [(1 << 22) + 5]):
        params, grads, copies, states = A.make(small, 8, torch.bfloat16, True, 5)
        more = A.make(rest, 8, torch.bfloat16, True, 6)
        opt = L.AdamW(params + more[0], grads + more[1], 1e-3, copies=copies + more[2], bits=8, states=states + more[3], steps=3)
        opt.step()
        torch.cuda.synchronize()
        out.append(params + copies + [t for s in states for t in s])
    for a, b in zip(*out):
        same = torch.equal(a, b)
        assert same


def test_values_around_large_tensors_are_left_alone():
    sizes, gap = [(1 << 22) + 300, 3 * C + 1, 5 * C + 1025], 512
    whole = [-(-n // A.BLOCK) * A.BLOCK + gap for n in sizes]
    starts = [gap // 2 + sum(whole[:i]) for i in range(len(sizes))]
    flat = [torch.full((sum(whole),), 7.0, device="cuda", dtype=dt) for dt in (torch.float32, torch.bfloat16, torch.uint8, torch.uint8)]
    scales = [torch.full((sum(whole) // A.BLOCK,), 1.0, device="cuda") for _ in range(2)]
    grads = torch.randn(sum(whole), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    cut = lambda t: [t[a: a + n] for a, n in zip(starts, sizes)]  # noqa: E731
    at = [0]
    for n in sizes:
        at.append(at[-1] + -(-n // A.BLOCK) + 1)
    states = [(m, v, scales[0][a: a + -(-n // A.BLOCK)], scales[1][a: a + -(-n // A.BLOCK)])
              for m, v, a, n in zip(cut(flat[2]), cut(flat[3]), at, sizes)]
    L.AdamW(cut(flat[0]), cut(grads), 1e-2, copies=cut(flat[1]), bits=8, states=states, steps=9).step()
    torch.cuda.synchronize()
    inside = torch.zeros(sum(whole), dtype=torch.bool, device="cuda")
    for a, n in zip(starts, sizes):
        inside[a: a + n] = True
    for t in flat:
        assert bool((t[~inside] == 7).all())
    for t in scales:  # one between two tensors' scales
        assert all(float(t[a - 1]) == 1 for a in at[1:])
