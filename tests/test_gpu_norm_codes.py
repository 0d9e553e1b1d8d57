"""The norm's E4M3 codes bit for bit: scale = largest magnitude / 448, code = cvt(y / scale), both divisions in fp32, of the y that
the row's rstd gives.  Nothing is left to a tolerance: y is two fp32 products, and the divisions are rounded correctly."""
import pytest
import torch

from paper_2605_05607_amd import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": (torch.bfloat16, B.MOE_BF16), "f32": (torch.float32, B.MOE_F32)}


def codes_of(s, rstd, w):
    """On the host, where a division by a number is one."""
    y = (s.float().cpu() * rstd.cpu()[:, None]) * w.float().cpu()
    top = y.abs().amax(1)
    scales = torch.where(top > 0, (top / torch.full_like(top, 448.0)).clamp(min=2.0 ** -126), torch.ones_like(top))
    return (y / scales[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), scales


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 7168), (3, 8), (40, 2880), (300, 1000), (300, 4096), (257, 7168), (260, 16384)])
def test_codes_are_those_of_the_divisions(rows, cols, dtype):
    """Values of eight bits: their quotients are exact ties between two codes for four elements of 10^4, which the last bit decides."""
    print("norm codes", rows, cols, dtype, flush=True)
    dt, code = DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    r = lambda *a: torch.randn(a, generator=gen, device="cuda").bfloat16().to(dt)  # noqa: E731
    # rows of every size, down to where a scale is the smallest there is and a quotient's remainder is no normal number
    size = 2.0 ** torch.tensor([0, 40, -30, -62, -80, -88, -96, -104, -118, -130, 60], device="cuda")
    for w in (1 + 0.3 * r(cols), torch.full((cols,), 2.0 ** -6, device="cuda", dtype=dt)):
        x = (r(rows, cols).float() * size[torch.arange(rows, device="cuda") % len(size)][:, None]).to(dt)
        x[rows // 2, 3] = -0.0
        for eps in (1e-6, 1.0):
            q, sc = torch.empty((rows, cols), dtype=torch.uint8, device="cuda"), torch.empty(rows, device="cuda")
            rstd = torch.empty(rows, device="cuda")
            B.moe_rmsnorm(rows, cols, code, x, None, w.to(dt), eps, None, None, q, sc, rstd)
            want, scales = codes_of(x, rstd, w.to(dt))
            off = (q.cpu() != want).sum(1)
            plain, every, of_scales = int(off[:: len(size)].sum()), int(off.sum()), int((sc.cpu() != scales).sum())
            assert plain == 0 and every == 0 and of_scales == 0  # (plain: rows of size 1)


def test_fp32_rows_of_several_launches():
    """More than 2^21 rows: the second launch's rows, codes and scales, and their gradients.  Tolerances: half a step (u = 2^-24) for
    each operation, eight products and nine additions a row; dx has three such terms."""
    rows, cols, u = (1 << 21) + 7, 8, 2.0 ** -24
    gen = torch.Generator(device="cuda").manual_seed(2)
    r = lambda *a: torch.randn(a, generator=gen, device="cuda")  # noqa: E731
    x, res, w, dy, dsum = r(rows, cols), r(rows, cols), r(cols), r(rows, cols), r(rows, cols)
    s, y, dx, q = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty((rows, cols), dtype=torch.uint8, device="cuda")
    sc, rstd, dw = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(B.moe_rmsnorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.moe_rmsnorm(rows, cols, B.MOE_F32, x, res, w, 1e-6, s, y, q, sc, rstd)
    B.moe_rmsnorm_backward(rows, cols, B.MOE_F32, s, w, rstd, dy, dsum, dx, dw, ws)
    torch.cuda.synchronize()
    assert torch.equal(s, x + res)
    s64, w64, g = s.double(), w.double(), dy.double()
    k = (s64.square().mean(1) + 1e-6).rsqrt()
    assert bool(((rstd.double() - k).abs() <= 16 * u * k).all())
    ref = s64 * k[:, None] * w64
    assert bool(((y.double() - ref).abs() <= 24 * u * ref.abs()).all())
    tail = slice((1 << 21) - 1000, rows)
    want, scales = codes_of(s[tail], rstd[tail], w)
    same = torch.equal(q[tail].cpu(), want) and torch.equal(sc[tail].cpu(), scales)
    assert same
    k = rstd.double()[:, None]
    a = g * w64
    ref = k * (a - s64 * k * k * (a * s64).mean(1, keepdim=True)) + dsum.double()
    size = k * (a.abs() + s64.abs() * k * k * (a * s64).abs().mean(1, keepdim=True)) + dsum.double().abs()
    assert bool(((dx.double() - ref).abs() <= 32 * u * size).all())
    size = (g * s64 * k).abs().sum(0)  # a chain of rows / 2048 in a register, then the partial rows
    assert bool(((dw.double() - (g * s64 * k).sum(0)).abs() <= (rows / 2048 + 64) * u * size).all())
