"""The experts' rows back to their tokens with the gate weights, and the gradients of that and of the sorting copy, against
float64.

Tolerances, derived: u = 2^-24 is half an fp32 step.  A sum over k slots is k products and additions: k u of the magnitudes, and
half a step of the element type at the write.  A dot product over d columns is a chain of d / (columns in flight) products in a
thread, at most d / 32 of them, and at most 16 additions over lanes and waves: (d / 32 + 16) u of the magnitudes."""
import pytest
import torch

from paper_2605_05607_amd import binding as B
from paper_2605_05607_amd import layer as L
from paper_2605_05607_amd import workloads as wl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


class Batch:
    def __init__(self, T, d, E, k, R, lo, hi, dtype, router="normal", seed=1):
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.half = torch.finfo(self.dt).eps / 2 if dtype == "bf16" else U
        cfg = wl.MoEConfig("rows", T=T, d=d, f=8, E=E, k=k, R=R, local_rank_begin=lo, local_rank_end=hi,
                           dtype=wl.BF16 if dtype == "bf16" else wl.F32, router=router, seed=seed)
        self.lay = L.MoELayer(cfg)
        gen = torch.Generator(device="cuda").manual_seed(seed + T)
        self.randn = lambda *s: torch.randn(s, generator=gen, device="cuda").to(self.dt)
        w = wl.make_workload(cfg, weights=False)
        self.lay.route(L.to_device(w.logits))
        self.tables()

    def tables(self):
        c, lay = self.lay.cfg, self.lay
        lay.build_dispatch()
        self.shape, self.idx, self.w, self.tb = lay.shape, lay.topk_idx, lay.topk_w, lay.tables
        T, k = c.T, c.k
        off = self.tb.offsets.cpu()
        first = c.first_local_expert
        self.P = int(off[first + c.E_loc] - off[first])
        self.cap = max(1, T * min(k, c.E_loc))
        n = T * k
        e = self.idx[:n].view(T, k).long()
        self.local = (e >= first) & (e < first + c.E_loc)
        self.row = torch.where(self.local, self.tb.inv_perm[:n].view(T, k).long() - int(off[first]), 0)
        self.w64 = self.w[:n].view(T, k).double() * self.local

    def rows(self, fill=float("nan")):
        """Layout rows: values up to the last local row, `fill` behind it (never read)."""
        r = torch.full((self.cap, self.lay.cfg.d), fill, dtype=self.dt, device="cuda")
        r[: self.P] = self.randn(self.P, self.lay.cfg.d)
        return r

    def pairs(self, rows):
        """Rows of every (token, slot) in float64, zeros where the slot is not local."""
        return torch.where(self.local[:, :, None], rows[: max(1, self.P)].double()[self.row] if self.P else 0.0, 0.0)


SHAPES = [
    # T, d, E, k, R, local ranks, router
    (1, 8, 8, 2, 8, 0, 1, "normal"), (1, 7168, 256, 8, 8, 0, 8, "normal"), (2, 520, 8, 8, 1, 0, 1, "normal"),
    (16, 2048, 64, 8, 8, 0, 1, "normal"), (5, 7168, 256, 8, 8, 4, 5, "zipf"), (67, 264, 16, 1, 4, 1, 3, "normal"),
    (333, 2880, 128, 4, 4, 0, 1, "forced"), (257, 1000, 64, 32, 2, 1, 2, "normal"), (1025, 512, 32, 6, 8, 2, 5, "zipf"),
    (500, 4096, 8, 2, 8, 7, 8, "normal"), (300, 16, 4096, 4, 64, 3, 4, "normal"), (4100, 104, 16, 3, 4, 0, 4, "normal"),
    (40, 20488, 8, 3, 2, 0, 1, "normal"), (2049, 2056, 64, 8, 8, 0, 1, "normal"),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_back_and_gradients(shape, dtype):
    print("rows", shape, dtype, flush=True)
    T, d, E, k, R, lo, hi, router = shape
    b = Batch(T, d, E, k, R, lo, hi, dtype, router)
    picks = b.idx[: T * k].clone()
    for form in ("as routed", "picks outside", "one expert twice", "no local row"):
        if form == "one expert twice" and k > b.lay.cfg.E_loc:
            continue  # (more rows than picks of distinct experts have room for)
        if form != "as routed":
            p = picks.view(T, k).clone()
            if form == "picks outside":
                p[1::3] = -1
                p[2::3, 0] = E + 5
            elif form == "one expert twice":
                p[:, -1] = p[:, 0]
                p[::4] = b.lay.cfg.first_local_expert
            else:
                p[:] = (b.lay.cfg.first_local_expert + b.lay.cfg.E_loc) % E if b.lay.cfg.E_loc < E else -1
            b.idx[: T * k].copy_(p.view(-1))
            b.tables()
        rows, dy = b.rows(), b.randn(T, d)
        y = torch.full((T, d), 7.0, dtype=b.dt, device="cuda")
        B.moe_combine_weighted(b.shape, rows, b.idx, b.w, b.tb, y)
        g = b.pairs(rows)
        ref, size = (b.w64[:, :, None] * g).sum(1), (b.w64[:, :, None] * g).abs().sum(1)
        assert ((y.double() - ref).abs() <= ref.abs() * b.half + (k + 1) * U * size).all(), form
        none = ~b.local.any(1)
        assert not y[none].any()
        # the sorting copy's gradient: the same sums without weights
        dx = torch.full((T, d), 7.0, dtype=b.dt, device="cuda")
        B.moe_dispatch_gather_backward(b.shape, rows, b.idx, b.tb, dx)
        ref, size = g.sum(1), g.abs().sum(1)
        assert ((dx.double() - ref).abs() <= ref.abs() * b.half + (k + 1) * U * size).all(), form
        assert not dx[none].any()
        # the weighted way's gradient
        d_rows = torch.full((b.cap, d), 7.0, dtype=b.dt, device="cuda")
        d_w = torch.full((T, k), 7.0, device="cuda")
        B.moe_combine_weighted_backward(b.shape, rows, dy, b.idx, b.w, b.tb, d_rows, d_w)
        assert (d_rows[b.P:] == 7).all()  # rows behind the last local one
        ref = b.w64[:, :, None] * dy.double()[:, None, :]
        got = b.pairs(d_rows)
        assert ((got - ref).abs() <= ref.abs() * (b.half + U)).all(), form
        dots = g * dy.double()[:, None, :]
        assert ((d_w.double() - dots.sum(2)).abs() <= (d / 32 + 16) * U * dots.abs().sum(2)).all(), form
        assert not d_w[~b.local].any()
        again, d_w2 = rows.clone(), torch.empty_like(d_w)  # over the rows themselves: the same bits
        B.moe_combine_weighted_backward(b.shape, again, dy, b.idx, b.w, b.tb, again, d_w2)
        assert torch.equal(again[: b.P], d_rows[: b.P]) and torch.equal(d_w2, d_w)
        assert torch.isnan(again[b.P:]).all()


def test_gradients_against_differences():
    b = Batch(37, 136, 16, 4, 4, 1, 3, "f32", seed=6)
    T, k, d = 37, 4, 136
    rows, dy, x, dxs = b.rows(0.0), b.randn(T, d), b.randn(T, d), b.rows(0.0)
    d_rows, d_w, dx = torch.zeros_like(rows), torch.empty((T, k), device="cuda"), torch.empty_like(x)
    B.moe_combine_weighted_backward(b.shape, rows, dy, b.idx, b.w, b.tb, d_rows, d_w)
    B.moe_dispatch_gather_backward(b.shape, dxs, b.idx, b.tb, dx)
    y = torch.empty_like(x)

    def back(r, w):  # the operator itself, linear in either argument: differences are exact up to rounding
        B.moe_combine_weighted(b.shape, r, b.idx, w.contiguous(), b.tb, y)
        return (y.double() * dy.double()).sum().item()

    def sort(v):
        xs = torch.zeros_like(rows)
        B.moe_dispatch_gather(b.shape, v, b.tb, xs)
        return (xs.double() * dxs.double())[: b.P].sum().item()
    u, v, z = b.rows(0.0), torch.randn((T, k), device="cuda"), b.randn(T, d)
    w = b.w[: T * k].view(T, k)
    # every product and sum of the two fp32 evaluations and of the gradient rounds once: below 16 u of the terms' magnitudes
    most = (b.pairs(rows).abs() + b.pairs(u).abs() + b.pairs(dxs).abs()) * (1 + v.abs().max())
    size = 16 * U * (most * (dy.abs() + x.abs() + z.abs()).double()[:, None, :]).sum().item()
    assert abs((back(rows + u, w) - back(rows - u, w)) / 2 - (d_rows.double() * u.double())[: b.P].sum().item()) <= size
    assert abs((back(rows, w + v) - back(rows, w - v)) / 2 - (d_w.double() * v.double()).sum().item()) <= size
    assert abs((sort(x + z) - sort(x - z)) / 2 - (dx.double() * z.double()).sum().item()) <= size


def test_zero_weight_and_rows_that_are_not_finite():
    """A row reaches its own token alone; weight 0 times an infinity is NaN there, as the formula says."""
    b = Batch(300, 512, 16, 4, 4, 0, 2, "bf16", seed=3)
    rows = b.rows()
    clean = torch.empty((300, 512), dtype=b.dt, device="cuda")
    B.moe_combine_weighted(b.shape, rows, b.idx, b.w, b.tb, clean)
    t, j = (int(v) for v in b.local.nonzero()[20])
    rows[b.row[t, j], 100] = float("inf")
    y = torch.empty_like(clean)
    B.moe_combine_weighted(b.shape, rows, b.idx, b.w, b.tb, y)
    assert torch.isinf(y[t, 100])
    y[t, 100] = clean[t, 100]
    assert torch.equal(y, clean)


def test_no_tokens_touch_nothing():
    b = Batch(1, 64, 8, 2, 2, 0, 1, "bf16")
    s = B.make_shape(0, 64, 8, 8, 2, 2, 0, 1, B.MOE_BF16)
    y, d_w = torch.full((1, 64), 7.0, dtype=b.dt, device="cuda"), torch.full((1, 2), 7.0, device="cuda")
    rows, out = torch.zeros((2, 64), dtype=b.dt, device="cuda"), torch.full((2, 64), 7.0, dtype=b.dt, device="cuda")
    B.moe_combine_weighted(s, rows, b.idx, b.w, b.tb, y)
    B.moe_dispatch_gather_backward(s, rows, b.idx, b.tb, y)
    B.moe_combine_weighted_backward(s, rows, y, b.idx, b.w, b.tb, out, d_w)
    torch.cuda.synchronize()
    assert (y == 7).all() and (d_w == 7).all() and (out == 7).all()


def test_replays_from_a_graph():
    b = Batch(700, 1000, 32, 4, 4, 1, 2, "bf16", seed=12)
    x, rows, dy, dxs = b.randn(700, 1000), b.rows(), b.randn(700, 1000), b.rows()

    def call():
        xs, y, d_rows, d_w, dx = (torch.zeros_like(rows), torch.empty_like(x), torch.zeros_like(rows),
                                  torch.empty((700, 4), device="cuda"), torch.empty_like(x))
        B.moe_dispatch_gather(b.shape, x, b.tb, xs)
        B.moe_combine_weighted(b.shape, rows, b.idx, b.w, b.tb, y)
        B.moe_combine_weighted_backward(b.shape, rows, dy, b.idx, b.w, b.tb, d_rows, d_w)
        B.moe_dispatch_gather_backward(b.shape, dxs, b.idx, b.tb, dx)
        return xs, y, d_rows, d_w, dx
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for turn in range(4):
        dy.copy_(b.randn(700, 1000))
        rows[: b.P].copy_(b.randn(b.P, 1000))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for p, q in zip(held, call()):
            assert torch.equal(p, q), turn


def test_rows_past_32_bit_offsets():
    T, d = 66000, 32776  # 2.16e9 values
    b = Batch(T, d, 4, 1, 1, 0, 1, "bf16", seed=2)
    rows = torch.zeros((T, d), dtype=b.dt, device="cuda")
    few = [0, 65535, 65536, T - 1]
    val = b.randn(len(few), d)
    at = b.row[few, 0]
    rows[at] = val
    y = torch.empty((T, d), dtype=b.dt, device="cuda")
    B.moe_dispatch_gather_backward(b.shape, rows, b.idx, b.tb, y)
    assert torch.equal(y[few], val)  # (one slot a token: a copy)
    assert int(torch.count_nonzero(y.view(torch.int16).view(-1)[:: 8])) == int(torch.count_nonzero(rows.view(torch.int16).view(-1)[:: 8]))
    d_w = torch.empty((T, 1), device="cuda")
    B.moe_combine_weighted_backward(b.shape, rows, y, b.idx, b.w, b.tb, rows, d_w)
    assert torch.equal(rows[at], val)  # (weight 1)
    want = val.double().square().sum(1)
    assert ((d_w[few, 0].double() - want).abs() <= (d / 32 + 16) * U * want).all()
