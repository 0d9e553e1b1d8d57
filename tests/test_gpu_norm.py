"""The root-mean-square norm with the residual's addition and E4M3 codes, and its gradients, against float64.

Tolerances, derived: u = 2^-24 is half an fp32 step.  A row's sum of squares is a chain of at most 32 products in a thread and
at most 22 additions over threads and waves, all of one sign: relative error below 64 u, half of that in rstd, and five more
roundings to y: 2^-18 covers 64 u.  What is stored in the element type adds half a step of it (eps / 2).  E4M3 codes: half a
step, 2^-4 of a normal value, 2^-10 scales of a subnormal one."""
import pytest
import torch

from paper_2605_05607_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": (torch.bfloat16, B.MOE_BF16), "f32": (torch.float32, B.MOE_F32)}
EPS = 1e-6


def half(dt):
    return torch.finfo(dt).eps / 2 if dt != torch.float32 else U


def guarded(shape, dtype, fill):
    """An array with a line of `fill` on either side of it; the view and a check that the lines are as they were."""
    import math
    n, pad = math.prod(shape), 256 // torch.empty(0, dtype=dtype).element_size()
    flat = torch.empty(n + 2 * pad, dtype=dtype, device="cuda").fill_(fill)
    edges = torch.cat([flat[:pad], flat[pad + n:]]).clone()
    return flat[pad: pad + n].view(shape), lambda: torch.equal(torch.cat([flat[:pad], flat[pad + n:]]), edges)


def inputs(rows, cols, dt, seed, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    return ((r(rows, cols) * scale).to(dt), (r(rows, cols) * 2 * scale).to(dt), (1 + 0.3 * r(cols)).to(dt), r(rows, cols).to(dt),
            r(rows, cols).to(dt))


def forward64(s, w, eps=EPS):
    s, w = s.double(), w.double()
    rstd = (s.square().mean(1) + eps).rsqrt()
    return s * rstd[:, None] * w, rstd


def backward64(s, w, rstd, dy, dsum):
    s, w, dy = s.double(), w.double(), dy.double()
    a, r = dy * w, rstd.double()[:, None]
    dx = r * (a - s * r * r * (a * s).mean(1, keepdim=True))
    return dx + (0 if dsum is None else dsum.double()), (dy * s * r).sum(0)


def check_codes(codes, scales, y, dt):
    top = y.abs().amax(1)
    want = torch.where(top > 0, top / 448, torch.ones_like(top))
    assert ((scales.double() - want).abs() <= want * 2.0 ** -18).all()
    sc = scales.double()[:, None]
    err = (codes.view(torch.float8_e4m3fn).double() * sc - y).abs()
    assert (err <= torch.maximum(y.abs() * 2.0 ** -4, sc * 2.0 ** -10) + y.abs() * 2.0 ** -17).all()


# one wave, four and sixteen waves a row; every count of pieces a thread; columns that end inside a piece's wave; few rows
SIZES = [(1, 8), (3, 8), (1, 7168), (2, 512), (5, 520), (300, 8), (257, 512), (301, 1000), (256, 2048), (259, 2056), (270, 2880), (512, 136), (513, 136),
         (1025, 4096), (300, 7168), (256, 8192), (257, 8200), (3, 16384), (261, 16392), (2, 32768), (256, 32768), (4099, 264)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward_and_gradients(rows, cols, dtype):
    print(f"norm {rows} x {cols} {dtype}", flush=True)
    dt, code = DT[dtype]
    x, res, w, dy, dsum = inputs(rows, cols, dt, rows * 7 + cols)
    x[0] = 0
    res[0] = 0  # a row of zeros: y 0, scale 1
    for residual in (res, None):
        s, s_ok = guarded((rows, cols), dt, 7.0)
        y, y_ok = guarded((rows, cols), dt, 7.0)
        q, q_ok = guarded((rows, cols), torch.uint8, 7)
        sc, sc_ok = guarded((rows,), torch.float32, 7.0)
        rstd, r_ok = guarded((rows,), torch.float32, 7.0)
        B.moe_rmsnorm(rows, cols, code, x, residual, w, EPS, None if residual is None else s, y, q, sc, rstd)
        torch.cuda.synchronize()
        assert s_ok() and y_ok() and q_ok() and sc_ok() and r_ok()
        want_s = x if residual is None else (x.float() + residual.float()).to(dt)  # (one rounding: equal)
        assert residual is None or torch.equal(s, want_s)
        ref, r64 = forward64(want_s, w)
        assert ((rstd.double() - r64).abs() <= r64 * 2.0 ** -18).all()
        assert ((y.double() - ref).abs() <= ref.abs() * (half(dt) + 2.0 ** -18)).all()
        check_codes(q, sc, ref, dt)
        assert sc[0] == 1 and not (q[0] & 127).any() and not y[0].any()  # (a negative weight makes its zero -0)
        # y alone, and codes alone, give the same
        y2, q2, sc2 = torch.empty_like(y), torch.empty_like(q), torch.empty_like(sc)
        B.moe_rmsnorm(rows, cols, code, x, residual, w, EPS, None, y2, None, None, None)
        B.moe_rmsnorm(rows, cols, code, x, residual, w, EPS, None, None, q2, sc2, None)
        assert torch.equal(y2, y) and torch.equal(q2, q) and torch.equal(sc2, sc)

        dx, dx_ok = guarded((rows, cols), dt, 7.0)
        dw, dw_ok = guarded((cols,), torch.float32, 7.0)
        ws, ws_ok = guarded((B.moe_rmsnorm_backward_workspace_bytes(rows, cols),), torch.uint8, 7)
        direct = dsum if residual is not None else None
        B.moe_rmsnorm_backward(rows, cols, code, want_s, w, rstd, dy, direct, dx, dw, ws)
        torch.cuda.synchronize()
        assert dx_ok() and dw_ok() and ws_ok()
        ref_dx, ref_dw = backward64(want_s, w, rstd, dy, direct)
        a, r = dy.double() * w.double(), rstd.double()[:, None]
        s64 = want_s.double()
        # roundings of the three terms; the mean's chain is that of the sum of squares, its error relative to the magnitudes
        size = (r * a).abs() + r ** 3 * s64.abs() * (a * s64).abs().mean(1, keepdim=True)
        assert ((dx.double() - ref_dx).abs() <= size * 2.0 ** -18 + ref_dx.abs() * (half(dt) + 4 * U)).all()
        # a column's sum: rows / (partial sums) in a register, eight registers, then 256 partial sums in sixteen chains
        # (up to 512 rows: at most 16 rows in a register and 64 registers)
        chain = max(rows / min(rows, 256) + 8 + 256 / 16 + 16, 80)
        assert ((dw.double() - ref_dw).abs() <= chain * U * (dy.double() * s64 * r).abs().sum(0) + 1e-300).all()
        # without the weight's gradient; into dy or the direct gradient itself; again: the same bits
        for target in (dy.clone(), None if direct is None else direct.clone()):
            if target is None:
                continue
            own_dy = target if direct is None or not torch.equal(target, direct) else dy
            own_ds = direct if own_dy is target or direct is None else target
            B.moe_rmsnorm_backward(rows, cols, code, want_s, w, rstd, own_dy, own_ds, target, None, None)
            assert torch.equal(target, dx)
        over = dy.clone()
        B.moe_rmsnorm_backward(rows, cols, code, want_s, w, rstd, over, direct, over, dw, ws)
        size = (dy.double() * s64 * r).abs().sum(0)
        assert torch.equal(over, dx) and ((dw.double() - ref_dw).abs() <= chain * U * size + 1e-300).all()
        B.moe_rmsnorm_backward(rows, cols, code, want_s, w, rstd, dy, direct, torch.empty_like(dx), dw, ws)
        again = torch.empty_like(dw)
        ws.fill_(0xFF)
        B.moe_rmsnorm_backward(rows, cols, code, want_s, w, rstd, dy, direct, torch.empty_like(dx), again, ws)
        assert torch.equal(again, dw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sum_in_place_and_shared_inputs(dtype):
    dt, code = DT[dtype]
    for rows, cols in ((2, 7168), (300, 1000), (300, 4096)):
        x, res, w, _, _ = inputs(rows, cols, dt, 3)
        want, y0 = torch.empty_like(x), torch.empty_like(x)
        B.moe_rmsnorm(rows, cols, code, x, res, w, EPS, want, y0, None, None, None)
        for alias in ("x", "residual"):
            a, b, y = x.clone(), res.clone(), torch.empty_like(x)
            B.moe_rmsnorm(rows, cols, code, a, b, w, EPS, a if alias == "x" else b, y, None, None, None)
            assert torch.equal(a if alias == "x" else b, want) and torch.equal(y, y0)
        twice, y = torch.empty_like(x), torch.empty_like(x)
        B.moe_rmsnorm(rows, cols, code, x, x, w, EPS, twice, y, None, None, None)  # the same array as both
        assert torch.equal(twice, (2 * x.float()).to(dt))


def test_gradients_against_differences():
    rows, cols = 6, 264
    x, res, w, dy, dsum = inputs(rows, cols, torch.float32, 5)
    s, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda")
    B.moe_rmsnorm(rows, cols, B.MOE_F32, x, res, w, EPS, s, y, None, None, rstd)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(B.moe_rmsnorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.moe_rmsnorm_backward(rows, cols, B.MOE_F32, s, w, rstd, dy, dsum, dx, dw, ws)

    def loss(s64, w64):
        return ((forward64(s64, w64)[0] * dy.double()).sum() + (s64 * dsum.double()).sum()).item()
    gen = torch.Generator(device="cuda").manual_seed(9)
    h = 1e-5
    for _ in range(4):
        u = torch.randn((rows, cols), generator=gen, device="cuda").double()
        v = torch.randn((cols,), generator=gen, device="cuda").double()
        s64, w64 = s.double(), w.double()
        ds = (loss(s64 + h * u, w64) - loss(s64 - h * u, w64)) / (2 * h)
        dv = (loss(s64, w64 + h * v) - loss(s64, w64 - h * v)) / (2 * h)
        # fp32 gradients: 2^-18 of the terms' magnitudes; the differences' own error is h^2 and 1e-16 / h
        assert abs(ds - (dx.double() * u).sum().item()) <= 2.0 ** -17 * (dx.double().abs() * u.abs()).sum().item() + 1e-6
        assert abs(dv - (dw.double() * v).sum().item()) <= 2.0 ** -17 * (dw.double().abs() * v.abs()).sum().item() + 1e-6


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e-4, 1e4, 1e12])
def test_rows_of_extreme_size(scale, dtype):
    dt, code = DT[dtype]
    for cols in (512, 2880, 7168):
        rows = 260
        x, _, w, _, _ = inputs(rows, cols, dt, 11, scale)
        y, q, sc = torch.empty_like(x), torch.empty((rows, cols), dtype=torch.uint8, device="cuda"), torch.empty(rows, device="cuda")
        B.moe_rmsnorm(rows, cols, code, x, None, w, EPS, None, y, q, sc, None)
        ref, _ = forward64(x, w)
        least = torch.finfo(torch.float32).tiny  # (what falls under the normal range is off by its own step)
        assert ((y.double() - ref).abs() <= ref.abs() * (half(dt) + 2.0 ** -18) + least).all()
        check_codes(q, sc, ref, dt)


def test_rows_that_are_not_finite_stay_rows_of_their_own():
    for cols in (512, 2880, 7168):
        rows = 300
        x, res, w, _, _ = inputs(rows, cols, torch.bfloat16, 4)
        clean = [torch.empty_like(x), torch.empty((rows, cols), dtype=torch.uint8, device="cuda"), torch.empty(rows, device="cuda")]
        B.moe_rmsnorm(rows, cols, B.MOE_BF16, x, res, w, EPS, None, *clean, None)
        bad = {5: float("nan"), 17: float("inf"), 299: float("-inf")}
        for r, v in bad.items():
            x[r, cols - 3] = v
        y, q, sc = (torch.empty_like(t) for t in clean)
        B.moe_rmsnorm(rows, cols, B.MOE_BF16, x, res, w, EPS, None, y, q, sc, None)
        keep = torch.ones(rows, dtype=torch.bool, device="cuda")
        keep[list(bad)] = False
        for a, b in zip((y, q, sc), clean):
            assert torch.equal(a[keep], b[keep])
        assert not torch.isfinite(sc[~keep]).any() and torch.isnan(y[~keep][:, cols - 3]).all()


def test_no_rows_and_no_tokens():
    w, dw = torch.ones(64, dtype=torch.bfloat16, device="cuda"), torch.full((64,), 7.0, device="cuda")
    x = torch.full((1, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(B.moe_rmsnorm_backward_workspace_bytes(0, 64), dtype=torch.uint8, device="cuda")
    y, r = x.clone(), torch.full((1,), 7.0, device="cuda")
    B.moe_rmsnorm(0, 64, B.MOE_BF16, x, None, w, EPS, None, y, None, None, r)
    B.moe_rmsnorm_backward(0, 64, B.MOE_BF16, x, w, r, x, None, y, dw, ws)
    torch.cuda.synchronize()
    assert (y == 7).all() and (r == 7).all() and not dw.any()


def test_replays_from_a_graph_on_another_stream():
    rows, cols = 700, 2880
    x, res, w, dy, dsum = inputs(rows, cols, torch.bfloat16, 21)
    new = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
    ws = new(B.moe_rmsnorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8)

    def call():
        out = [new(rows, cols), new(rows, cols), new(rows, cols, dtype=torch.uint8), new(rows, dtype=torch.float32),
               new(rows, dtype=torch.float32), new(rows, cols), new(cols, dtype=torch.float32)]
        s, y, q, sc, rstd, dx, dw = out
        B.moe_rmsnorm(rows, cols, B.MOE_BF16, x, res, w, EPS, s, y, q, sc, rstd)
        B.moe_rmsnorm_backward(rows, cols, B.MOE_BF16, s, w, rstd, dy, dsum, dx, dw, ws)
        return out
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for turn in range(4):
        x.copy_(inputs(rows, cols, torch.bfloat16, 30 + turn)[0])
        for t in held:
            t.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = call()
        torch.cuda.synchronize()
        for a, b in zip(held, eager):
            assert torch.equal(a, b), turn


def test_rows_of_several_launches():
    rows, cols = (1 << 21) + 5, 8
    x, res, w, dy, _ = inputs(rows, cols, torch.bfloat16, 13)
    s, y, q = torch.empty_like(x), torch.empty_like(x), torch.empty((rows, cols), dtype=torch.uint8, device="cuda")
    sc, rstd = (torch.full((rows,), 7.0, device="cuda") for _ in range(2))
    B.moe_rmsnorm(rows, cols, B.MOE_BF16, x, res, w, EPS, s, y, q, sc, rstd)
    assert torch.equal(s, (x.float() + res.float()).bfloat16())
    ref, r64 = forward64(s, w)
    assert ((rstd.double() - r64).abs() <= r64 * 2.0 ** -18).all()
    assert ((y.double() - ref).abs() <= ref.abs() * (half(torch.bfloat16) + 2.0 ** -18)).all()
    check_codes(q, sc, ref, torch.bfloat16)
    dx, dw = torch.empty_like(x), torch.empty(cols, device="cuda")
    ws = torch.empty(B.moe_rmsnorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.moe_rmsnorm_backward(rows, cols, B.MOE_BF16, s, w, rstd, dy, None, dx, dw, ws)
    ref_dx, ref_dw = backward64(s, w, rstd, dy, None)
    assert (dx.double() - ref_dx).abs().max() <= 2.0 ** -7 * ref_dx.abs().max()
    # a chain of rows / 256 / 8 in a register
    size = (dy.double() * s.double() * rstd.double()[:, None]).abs().sum(0)
    assert ((dw.double() - ref_dw).abs() <= (rows / 2048 + 64) * U * size).all()


def test_two_streams_at_once():
    rows, cols = 900, 4096
    sets = [inputs(rows, cols, torch.bfloat16, 40 + i) for i in range(2)]

    def call(a, ws):
        x, res, w, dy, dsum = a
        s, y, dx = (torch.empty_like(x) for _ in range(3))
        rstd, dw = torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda")
        for _ in range(5):
            B.moe_rmsnorm(rows, cols, B.MOE_BF16, x, res, w, EPS, s, y, None, None, rstd)
            B.moe_rmsnorm_backward(rows, cols, B.MOE_BF16, s, w, rstd, dy, dsum, dx, dw, ws)
        return s, y, dx, rstd, dw
    size = B.moe_rmsnorm_backward_workspace_bytes(rows, cols)
    spaces = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    want = [call(a, ws) for a, ws in zip(sets, spaces)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for a, ws, st in zip(sets, spaces, streams):
        with torch.cuda.stream(st):
            got.append(call(a, ws))
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(g, w))


def test_more_than_2_to_the_31_values():
    rows, cols = 65600, 32768  # 2.15e9 values: offsets past 32 bits
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    few = [0, 40000, 65535, rows - 1]
    part, _, w, dyp, _ = inputs(len(few), cols, torch.bfloat16, 8)
    x[few] = part
    y, rstd = torch.empty_like(x), torch.empty(rows, device="cuda")
    B.moe_rmsnorm(rows, cols, B.MOE_BF16, x, None, w, EPS, None, y, None, None, rstd)
    ref, _ = forward64(part, w)
    assert ((y[few].double() - ref).abs() <= ref.abs() * (half(torch.bfloat16) + 2.0 ** -18)).all()
    y.zero_()
    y[few] = dyp  # as dy, and dx over it
    dw = torch.empty(cols, device="cuda")
    ws = torch.empty(B.moe_rmsnorm_backward_workspace_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    B.moe_rmsnorm_backward(rows, cols, B.MOE_BF16, x, w, rstd, y, None, y, dw, ws)
    ref_dx, ref_dw = backward64(part, w, rstd[few], dyp, None)
    assert (y[few].double() - ref_dx).abs().max() <= 2.0 ** -7 * ref_dx.abs().max()
    size = (dyp.double() * part.double() * rstd[few].double()[:, None]).abs().sum(0)
    assert ((dw.double() - ref_dw).abs() <= 200 * U * size).all()
