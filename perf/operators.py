"""The operators around the expert GEMMs of an MoE layer, as a list of cases: what each computes in elementary torch
operations, and the calls that a user of this framework makes for it.

  norm    root-mean-square norm in front of the layer.  serve: s = x + residual, y = s rstd w and the E4M3 codes of y with a
          scale per row, for the gate network and the FP8 layer; train: forward, then the gradients of x and w
  sort    token rows to layout rows sorted by expert and the experts' rows back, with the gate weights applied; train: the
          gradients of both as well
  adamw   one AdamW step over a list of tensors, with both states in 32 bits, or in 8 bits: E4M3 codes of m and of sqrt(v) in
          blocks of 256 values with a scale each, rounded stochastically by a hash of seed, step, tensor and element

Shapes are those of the package's layer configurations and generic ones between them; batches run from a single token to
16384, lists of tensors from one norm weight to all expert weights of a layer.
"""
import math

import numpy as np
import torch

own = False

# hidden size, expert width, experts, picks, ranks of the layers the cases are drawn from
LAYERS = {
    "deepseek_v3": (7168, 2048, 256, 8, 8),
    "qwen3": (4096, 1536, 128, 8, 8),
    "gpt_oss": (2880, 2880, 128, 4, 4),
    "mixtral": (4096, 14336, 8, 2, 8),
    "table1_s": (2048, 512, 64, 8, 8),
    "table1_m": (4096, 1024, 128, 8, 8),
}
MAX_TOKENS = 16384
BLOCK = 256  # values that share a scale in the 8-bit states
E4M3_MAX = 448.0
LR, BETA1, BETA2, EPS, DECAY = 3e-4, 0.9, 0.95, 1e-8, 0.1
NORM_EPS = 1e-6


def _norm(name, mode, rows, cols, dtype="bf16", residual=True):
    return {"name": name, "kind": "norm", "mode": mode, "rows": rows, "cols": cols, "dtype": dtype, "residual": residual}


def _sort(name, mode, layer, T, router):
    d, _, E, k, R = LAYERS[layer]
    return {"name": name, "kind": "sort", "mode": mode, "T": T, "d": d, "E": E, "k": k, "R": R, "dtype": "bf16",
            "router": router}


def _adamw(name, sizes, bits, grads, copy, step):
    return {"name": name, "kind": "adamw", "sizes": ",".join(str(n) for n in sizes), "bits": bits, "grads": grads,
            "copy": copy, "step": step}


def _experts(layer):
    d, f, E, _, R = LAYERS[layer]
    return [E // R * d * f] * 3


def listed():
    return [
        # decode of one token of the largest hidden size: latency
        _norm("norm_one_token", "serve", 1, 7168),
        # prefill in front of the FP8 layer: residual, norm and codes in one pass
        _norm("norm_prefill", "serve", 4096, 7168),
        # a training step's norm and its gradients, with the gradient that comes down the residual stream
        _norm("norm_train", "train", 8192, 4096),
        # the fp32 layer's small batch, odd in number, without a residual
        _norm("norm_train_f32", "train", 255, 512, "f32", False),
        # decode batch of a small layer, one rank of eight local: most tokens have one local row, some none
        _sort("sort_decode_16", "serve", "table1_s", 16, "normal"),
        # prefill with the skewed load of inference: one expert with nearly all rows
        _sort("sort_prefill_skewed", "serve", "deepseek_v3", 4096, "zipf"),
        # one training step's sorting, weighting and their gradients, even load
        _sort("sort_train", "train", "qwen3", 8192, "normal"),
        # the same for an odd number of tokens of an odd size, a tenth of them with all their picks on one rank
        _sort("sort_train_ragged", "train", "gpt_oss", 5003, "forced"),
        # gate network, norm weights and biases of a small layer: many tensors, the smallest of a few values
        _adamw("adamw_small_tensors", [64 * 2048, 64, 1, 257, 100003] + [2048] * 30 + [2880, 7], 32, "f32", False, 700),
        # the expert weights of a small layer, states in 32 bits, bf16 gradients in and bf16 weights out
        _adamw("adamw_experts", _experts("table1_s"), 32, "bf16", True, 700),
        # all expert weights of one rank of a large layer with 8-bit states
        _adamw("adamw_experts_8bit", _experts("qwen3"), 8, "bf16", True, 2500),
        # first step of a fine-tuning run on ragged tensors, 8-bit states, fp32 gradients
        _adamw("adamw_first_step_8bit", [1500001, 262147, 4099, 2880 * 128, 2880], 8, "f32", False, 1),
    ]


def _log_int(rng, lo, hi, step=1):
    return max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))) // step * step)


def draw(rng):
    kind = rng.choice(["norm", "sort", "adamw"])
    if kind == "norm":
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        cols = rng.choice([LAYERS[rng.choice(sorted(LAYERS))][0], _log_int(rng, 256, 16384, 8)])
        case = {"kind": "norm", "mode": rng.choice(["serve", "train"]), "rows": _log_int(rng, 1, MAX_TOKENS), "cols": cols,
                "dtype": dtype, "residual": rng.random() < 0.75}
        while _cost(case) > _MOST["norm"]:
            case["rows"] = case["rows"] * 2 // 3
        return case
    if kind == "sort":
        if rng.random() < 0.6:
            d, _, E, k, R = LAYERS[rng.choice(sorted(LAYERS))]
        else:
            d, E, R = _log_int(rng, 256, 7168, 8), rng.choice([8, 16, 32, 64, 128, 256]), rng.choice([1, 2, 4, 8])
            k = rng.choice([n for n in (1, 2, 3, 4, 6, 8, 16) if n <= E])
        mode = rng.choice(["serve", "train"])
        case = {"kind": "sort", "mode": mode, "T": _log_int(rng, 1, MAX_TOKENS), "d": d, "E": E, "k": k, "R": R,
                "dtype": rng.choice(["bf16", "bf16", "bf16", "f32"]), "router": rng.choice(["normal", "zipf", "forced"])}
        while case["T"] > 1 and _cost(case) > _MOST["sort"]:
            case["T"] = case["T"] * 2 // 3
        return case
    if rng.random() < 0.4:
        sizes = _experts(rng.choice(["table1_s", "table1_m"]))
    else:
        sizes = [_log_int(rng, 1, 1 << 22) for _ in range(_log_int(rng, 1, 60))]
    return {"kind": "adamw", "sizes": ",".join(str(n) for n in sizes), "bits": rng.choice([8, 32]),
            "grads": rng.choice(["bf16", "f32"]), "copy": rng.random() < 0.5, "step": rng.choice([1, 2, 40, 5000])}


# ---- inputs ----
class State:
    pass


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, dtype=torch.float32, device="cuda")


def _prepare_norm(s, gen):
    c = s.case
    n, cols, dt = c["rows"], c["cols"], _dtype(c["dtype"])
    # a residual stream: most columns near one, a few of them many times as large
    loud = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.01, 20.0, 1.0)
    s.x = (_randn(gen, n, cols) * (loud if not c["residual"] else 1.0)).to(dt)
    s.residual = (_randn(gen, n, cols) * 2 * loud).to(dt) if c["residual"] else None
    s.w = (1.0 + 0.2 * _randn(gen, cols)).to(dt)
    new = lambda *a, dtype=dt: torch.empty(a, dtype=dtype, device="cuda")  # noqa: E731
    s.sum = new(n, cols) if c["residual"] else s.x
    s.y = new(n, cols)
    if c["mode"] == "serve":
        s.codes, s.scales = new(n, cols, dtype=torch.uint8), new(n, dtype=torch.float32)
    else:
        s.dy = _randn(gen, n, cols).to(dt)
        s.dsum = _randn(gen, n, cols).to(dt) if c["residual"] else None
        s.rstd, s.dx, s.dw = new(n, dtype=torch.float32), new(n, cols), new(cols, dtype=torch.float32)
        if own:  # scratch of the call, sized by the library
            from paper_2605_05607_amd import binding as B
            s.ws = new(max(1, B.moe_rmsnorm_backward_workspace_bytes(n, cols)), dtype=torch.uint8)


def _bias(case):
    """Per-expert addend of the logits (the load model, a property of the layer) and the local rank: the one that hosts the
    most popular expert of a skewed load."""
    E = case["E"]
    if case["router"] != "zipf":
        return np.zeros(E, dtype=np.float32), 0
    pi = np.random.default_rng([E, case["T"], case["d"]]).permutation(E)
    return (-1.1 * np.log1p(pi)).astype(np.float32), int(np.argmin(pi)) // (E // case["R"])


def _prepare_sort(s, gen):
    c = s.case
    T, d, E, k, R, dt = c["T"], c["d"], c["E"], c["k"], c["R"], _dtype(c["dtype"])
    bias, rank = _bias(c)
    logits = _randn(gen, T, E) + torch.from_numpy(bias).cuda()
    if c["router"] == "forced":  # a tenth of the tokens sends all its picks to one rank, where that has enough experts
        hit = torch.rand((T,), generator=gen, device="cuda") < 0.1
        to = torch.randint(0, R, (T,), generator=gen, device="cuda")
        on = (torch.arange(E, device="cuda") // (E // R))[None, :] == to[:, None]
        logits += 16.0 * (on & hit[:, None])
    val, idx = torch.topk(logits, k, dim=1)
    s.w = torch.softmax(val, dim=1).contiguous()
    s.idx = idx.to(torch.int32).contiguous()
    # the dispatch tables (all experts, all ranks), as the layer has built them for this batch
    flat, pair = idx.reshape(-1), torch.arange(T * k, device="cuda")
    perm = torch.argsort(flat, stable=True)
    inv = torch.empty_like(perm)
    inv[perm] = pair
    counts = torch.bincount(flat, minlength=E)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    key = flat // (E // R) * T + pair // k  # (rank, token) of every pair
    entries, to_entry = torch.unique(key, return_inverse=True)
    mask = torch.zeros(len(entries), dtype=torch.int64, device="cuda").scatter_add_(0, to_entry, 1 << (pair % k))
    rank_counts = torch.bincount(entries // T, minlength=R)
    tables = {"counts": counts, "offsets": offsets, "perm": perm, "inv_perm": inv, "rank_counts": rank_counts,
              "rank_offsets": torch.cat([rank_counts.new_zeros(1), rank_counts.cumsum(0)]), "dedup_tok": entries % T,
              "dedup_mask": mask, "pair_to_dedup": to_entry}
    s.tables = {n: t.to(torch.int32) for n, t in tables.items()}
    s.lo, s.hi = rank * (E // R), (rank + 1) * (E // R)
    first, s.P = int(offsets[s.lo]), int(offsets[s.hi] - offsets[s.lo])
    s.perm, s.first = perm, first
    cap = max(1, T * min(k, E // R))
    rows = lambda: torch.zeros((cap, d), dtype=dt, device="cuda")  # noqa: E731  (room for the most local rows there can be)
    s.x = _randn(gen, T, d).to(dt)
    s.xs, s.rows = rows(), rows()
    s.rows[: s.P] = _randn(gen, s.P, d).to(dt)
    s.y = torch.empty((T, d), dtype=dt, device="cuda")
    if c["mode"] == "train":
        s.dy = _randn(gen, T, d).to(dt)
        s.dxs, s.drows = rows(), rows()
        s.dxs[: s.P] = _randn(gen, s.P, d).to(dt)
        s.dx = torch.empty_like(s.y)
        s.dw = torch.empty((T, k), dtype=torch.float32, device="cuda")
    if own:  # the same tables in the arrays that the calls take
        from paper_2605_05607_amd import binding as B
        s.shape = B.make_shape(T, d, d, E, k, R, rank, rank + 1, B.MOE_F32 if c["dtype"] == "f32" else B.MOE_BF16)
        s.handle = B.DispatchTables(s.shape)
        for n, t in s.tables.items():
            getattr(s.handle, n)[: t.numel()].copy_(t)


def _codes_nearest(v):
    """E4M3 codes and block scales of a flat tensor, to the nearest code."""
    blocks = torch.nn.functional.pad(v, (0, -v.numel() % BLOCK)).view(-1, BLOCK)
    amax = blocks.abs().amax(1)
    scale = torch.where(amax > 0, amax / E4M3_MAX, 1.0)
    q = (blocks / scale[:, None]).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return q.view(torch.uint8).reshape(-1)[: v.numel()].contiguous(), scale


def _prepare_adamw(s, gen):
    """Every kind of array is one flat buffer, as for a data-parallel reduction; the tensors are pieces of it that start at
    whole blocks, with zeros between them."""
    c = s.case
    s.step = c["step"]
    s.seed = int(torch.randint(0, 1 << 31, (1,), generator=gen, device="cuda"))
    sizes = [int(v) for v in c["sizes"].split(",")]
    starts = [0]
    for n in sizes:
        starts.append(starts[-1] + -(-n // BLOCK) * BLOCK)
    s.pieces = list(zip(starts, sizes))
    total = starts[-1]
    within = torch.zeros(total, device="cuda")
    for at, n in s.pieces:
        within[at: at + n] = 1
    # gradients whose size varies along the buffer, and a last eighth without any (experts that had no rows)
    size = within * 1e-3 * torch.exp(_randn(gen, -(-total // 1024))).repeat_interleave(1024)[:total]
    grads = size * _randn(gen, total)
    grads[total - total // 8:] = 0
    s.flat = {"params": 0.02 * _randn(gen, total) * within, "grads": grads.to(_dtype(c["grads"]))}
    if c["copy"]:
        s.flat["copies"] = s.flat["params"].to(torch.bfloat16)
    m, r = torch.zeros(total, device="cuda"), torch.zeros(total, device="cuda")
    if s.step > 1:
        m = 0.3 * size * _randn(gen, total)
        r = size * (0.5 + torch.rand(total, generator=gen, device="cuda"))
    if c["bits"] == 32:
        s.flat.update(m=m, v=r * r)
    else:
        s.flat["m"], s.flat["m_scale"] = _codes_nearest(m)
        s.flat["v"], s.flat["v_scale"] = _codes_nearest(r)
    piece = lambda name: [s.flat[name][at: at + n] if name in s.flat else None for at, n in s.pieces]  # noqa: E731
    blocks = lambda name: [s.flat[name][at // BLOCK: at // BLOCK + -(-n // BLOCK)] if name in s.flat else None  # noqa: E731
                           for at, n in s.pieces]
    s.params, s.grads, s.copies = piece("params"), piece("grads"), piece("copies")
    s.states = list(zip(piece("m"), piece("v"), blocks("m_scale"), blocks("v_scale")))
    if own:
        from paper_2605_05607_amd import layer as L
        s.opt = L.AdamW(s.params, s.grads, lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY,
                        copies=s.copies if c["copy"] else None, bits=c["bits"], seed=s.seed, states=s.states,
                        steps=s.step - 1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = State()
    s.case = case
    {"norm": _prepare_norm, "sort": _prepare_sort, "adamw": _prepare_adamw}[case["kind"]](s, gen)
    return s


# ---- one pass: the framework's calls ----
def _norm_own(s):
    from paper_2605_05607_amd import binding as B
    c = s.case
    dt = B.MOE_F32 if c["dtype"] == "f32" else B.MOE_BF16
    stored = s.sum if c["residual"] else None
    if c["mode"] == "serve":
        B.moe_rmsnorm(c["rows"], c["cols"], dt, s.x, s.residual, s.w, NORM_EPS, stored, s.y, s.codes, s.scales, None)
        return {"sum": s.sum, "y": s.y, "codes": s.codes.view(torch.float8_e4m3fn), "scales": s.scales}
    B.moe_rmsnorm(c["rows"], c["cols"], dt, s.x, s.residual, s.w, NORM_EPS, stored, s.y, None, None, s.rstd)
    B.moe_rmsnorm_backward(c["rows"], c["cols"], dt, s.sum, s.w, s.rstd, s.dy, s.dsum, s.dx, s.dw, s.ws)
    return {"sum": s.sum, "y": s.y, "rstd": s.rstd, "dx": s.dx, "dw": s.dw}


def _sort_own(s):
    from paper_2605_05607_amd import binding as B
    B.moe_dispatch_gather(s.shape, s.x, s.handle, s.xs)
    B.moe_combine_weighted(s.shape, s.rows, s.idx, s.w, s.handle, s.y)
    out = {"xs": s.xs, "y": s.y}
    if s.case["mode"] == "train":
        B.moe_combine_weighted_backward(s.shape, s.rows, s.dy, s.idx, s.w, s.handle, s.drows, s.dw)
        B.moe_dispatch_gather_backward(s.shape, s.dxs, s.idx, s.handle, s.dx)
        out.update(drows=s.drows, dw=s.dw, dx=s.dx)
    return out


def _adamw_out(s):
    """The updated buffers: parameters, their bf16 copies and both states (8-bit codes as the values they stand for in units of
    their block's scale)."""
    out = {n: t for n, t in s.flat.items() if n != "grads"}
    if s.case["bits"] == 8:
        out.update(m=out["m"].view(torch.float8_e4m3fn), v=out["v"].view(torch.float8_e4m3fn))
    return out


def _adamw_own(s):
    s.opt.step()
    return _adamw_out(s)


# ---- one pass: the plain forms ----
def _norm_plain(s):
    c = s.case
    dt = s.x.dtype
    stored = (s.x.float() + s.residual.float()).to(dt) if c["residual"] else s.x
    v, w = stored.float(), s.w.float()
    rstd = 1.0 / torch.sqrt((v * v).mean(1) + NORM_EPS)
    y = v * rstd[:, None] * w
    if c["mode"] == "serve":
        amax = y.abs().amax(1)
        scales = torch.where(amax > 0, amax / E4M3_MAX, 1.0)
        codes = (y / scales[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        return {"sum": stored, "y": y.to(dt), "codes": codes, "scales": scales}
    dy = s.dy.float()
    a = dy * w
    dx = rstd[:, None] * (a - v * (rstd * rstd * (a * v).mean(1))[:, None])
    if s.dsum is not None:
        dx = dx + s.dsum.float()
    return {"sum": stored, "y": y.to(dt), "rstd": rstd, "dx": dx.to(dt), "dw": (dy * v * rstd[:, None]).sum(0)}


def _sort_plain(s):
    T, k, d = s.case["T"], s.case["k"], s.case["d"]
    dt = s.x.dtype
    pairs = s.perm[s.first: s.first + s.P]  # pair of every local row
    tok, w = pairs // k, s.w.reshape(-1)[pairs]
    # local row of every pair, one behind the last for a pair that has none
    row = torch.full((T * k,), s.P, dtype=torch.int64, device=s.x.device)
    row[pairs] = torch.arange(s.P, device=s.x.device)
    row = row.view(T, k)
    none = torch.zeros((1, d), dtype=torch.float32, device=s.x.device)
    rows = torch.cat([s.rows[: s.P].float(), none])
    s.xs[: s.P] = s.x[tok]  # (what lies behind the last local row stays as it was)
    out = {"xs": s.xs, "y": (rows[row] * s.w[:, :, None]).sum(1).to(dt)}
    if s.case["mode"] == "train":
        dy = s.dy.float()[tok]
        dw = torch.zeros(T * k, dtype=torch.float32, device=s.x.device)
        dw[pairs] = (rows[: s.P] * dy).sum(1)
        dxs = torch.cat([s.dxs[: s.P].float(), none])
        s.drows[: s.P] = w[:, None] * dy
        out.update(drows=s.drows, dw=dw.view(T, k), dx=dxs[row].sum(1).to(dt))
    return out


M32 = 0xFFFFFFFF


def _mix(z):
    z = (z ^ (z >> 16)) * 0x6A09E667 & M32
    z = (z ^ (z >> 15)) * 0xBB67AE85 & M32
    return z ^ (z >> 16)


def _hash(n, seed, step, tensor, device):
    key = _mix(seed + _mix(step + _mix(tensor + 0x9E3779B9 & M32) & M32) & M32)
    return _mix(torch.arange(n, dtype=torch.int64, device=device) ^ _mix(key))


def _decode(codes, scale):
    n = codes.numel()
    return codes.view(torch.float8_e4m3fn).float() * scale.repeat_interleave(BLOCK)[:n]


def _encode(v, bits16, least):
    """E4M3 codes of v over its block's scale, rounded up with the probability of what is cut off (16 random bits)."""
    n = v.numel()
    blocks = torch.nn.functional.pad(v, (0, -n % BLOCK)).view(-1, BLOCK)
    amax = blocks.abs().amax(1)
    scale = torch.where(amax > 0, amax / E4M3_MAX, 1.0)
    q = (blocks / scale[:, None]).reshape(-1)[:n]
    a = q.abs().clamp_(max=E4M3_MAX)
    small = a < 2.0 ** -6  # codes below 8 are multiples of 2^-9
    a = torch.where(small, a + 2.0 ** -6, a).view(torch.int32) + (bits16 << 4).to(torch.int32)
    code = (a >> 20) - 960 - 8 * small.to(torch.int32)
    if least:
        code = torch.where(v > 0, code.clamp(min=1), code)
    return (code | ((q < 0).to(torch.int32) << 7)).to(torch.uint8), scale


def _adamw_plain(s):
    bits = s.case["bits"]
    c1, c2 = 1.0 - BETA1 ** s.step, 1.0 - BETA2 ** s.step
    for i, (p, grad, (m, v, ms, vs)) in enumerate(zip(s.params, s.grads, s.states)):
        g = grad.float()
        m_old = m if bits == 32 else _decode(m, ms)
        v_old = v if bits == 32 else _decode(v, vs).square()
        m_new = BETA1 * m_old + (1.0 - BETA1) * g
        v_new = BETA2 * v_old + (1.0 - BETA2) * g * g
        root = torch.sqrt(v_new)
        p.mul_(1.0 - LR * DECAY).sub_((LR / c1) * m_new / (root / math.sqrt(c2) + EPS))
        if s.copies[i] is not None:
            s.copies[i].copy_(p)
        if bits == 32:
            m.copy_(m_new)
            v.copy_(v_new)
        else:
            h = _hash(p.numel(), s.seed, s.step, i, p.device)
            for state, scale, (codes, scales) in ((m, ms, _encode(m_new, h & 0xFFFF, False)),
                                                  (v, vs, _encode(root, h >> 16, True))):
                state.copy_(codes)
                scale.copy_(scales)
    s.step += 1
    return _adamw_out(s)


def run(s):
    if own:
        return {"norm": _norm_own, "sort": _sort_own, "adamw": _adamw_own}[s.case["kind"]](s)
    return {"norm": _norm_plain, "sort": _sort_plain, "adamw": _adamw_plain}[s.case["kind"]](s)


# ---- what a pass cannot do without ----
def _local(case):
    """Expected local rows and tokens with a local row: a sample of the load model's routing."""
    rng = np.random.default_rng(12345)
    bias, rank = _bias(case)
    T, E, R, k = case["T"], case["E"], case["R"], case["k"]
    n = min(T, 512)
    lg = rng.standard_normal((n, E)) + bias
    if case["router"] == "forced":
        on = np.arange(E)[None, :] // (E // R) == rng.integers(0, R, size=n)[:, None]
        lg += 16.0 * (on & (rng.random(n) < 0.1)[:, None])
    idx = np.argpartition(-lg, k - 1, axis=1)[:, :k] if k < E else np.tile(np.arange(E), (n, 1))
    local = idx // (E // R) == rank
    return local.sum() / n * T, local.any(axis=1).mean() * T


def work(case):
    if case["kind"] == "norm":
        n, cols, b = case["rows"], case["cols"], 4 if case["dtype"] == "f32" else 2
        e, res = float(n * cols), 1 if case["residual"] else 0
        forward = e * b * (2 + 2 * res) + cols * b  # x, y; the residual in and the sum out
        if case["mode"] == "serve":
            return {"bytes": forward + e + 4.0 * n, "flops": 8.0 * e}
        # the sum, dy and the gradient of the residual stream in, dx out
        return {"bytes": forward + e * b * (3 + res) + 8.0 * n + cols * (b + 4.0), "flops": 15.0 * e}
    if case["kind"] == "sort":
        T, d, k, b = case["T"], case["d"], case["k"], 4 if case["dtype"] == "f32" else 2
        P, tokens = _local(case)
        table = 12.0 * T * k  # picks, weights, rows of the pairs
        moved = (tokens + P + P + T) * d * b + table  # x, xs, rows, y
        if case["mode"] == "serve":
            return {"bytes": moved, "flops": 2.0 * P * d}
        moved += (tokens + P + P + P + T) * d * b + table + 4.0 * T * k  # dy, rows, drows, dxs, dx
        return {"bytes": moved, "flops": 6.0 * P * d}
    n = float(sum(int(v) for v in case["sizes"].split(",")))
    state = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / BLOCK
    return {"bytes": n * (8 + state + (4 if case["grads"] == "f32" else 2) + (2 if case["copy"] else 0)), "flops": 15.0 * n}


def _cost(case):
    return work(case)["bytes"]


_MOST = {kind: max(_cost(c) for c in listed() if c["kind"] == kind) for kind in ("norm", "sort", "adamw")}


# ---- in 64 bits ----
def _norm_exact(s):
    c = s.case
    total = s.x.double() + s.residual.double() if c["residual"] else s.x.double()
    z = total.to(s.x.dtype).double()  # the norm is that of the stored sum
    n, g = c["cols"], s.w.double()
    r = ((z * z).sum(1, keepdim=True) / n + NORM_EPS).rsqrt()
    y = z * r * g
    if c["mode"] == "serve":
        top = y.abs().max(1, keepdim=True).values
        unit = torch.where(top > 0, top / 448, torch.ones_like(top))
        return {"sum": total, "y": y, "codes": y / unit, "scales": unit[:, 0]}
    dy = s.dy.double()
    xhat = z * r
    dxhat = dy * g
    dx = r * (dxhat - xhat * (dxhat * xhat).sum(1, keepdim=True) / n)
    if c["residual"]:
        dx = dx + s.dsum.double()
    return {"sum": total, "y": y, "rstd": r[:, 0], "dx": dx, "dw": (dy * xhat).sum(0)}


def _sort_exact(s):
    T, d, k = s.case["T"], s.case["d"], s.case["k"]
    pair = s.perm.narrow(0, s.first, s.P)
    token = torch.div(pair, k, rounding_mode="floor")
    gate = s.w.double().flatten().index_select(0, pair).unsqueeze(1)
    back = lambda rows: torch.zeros((T, d), dtype=torch.float64, device="cuda").index_add_(0, token, rows)  # noqa: E731
    rows = s.rows.narrow(0, 0, s.P).double()
    whole = lambda rows: torch.nn.functional.pad(rows, (0, 0, 0, len(s.xs) - s.P))  # noqa: E731
    out = {"xs": whole(s.x.double().index_select(0, token)), "y": back(rows * gate)}
    if s.case["mode"] == "train":
        dy = s.dy.double().index_select(0, token)
        dw = torch.zeros(T * k, dtype=torch.float64, device="cuda").index_copy_(0, pair, (rows * dy).sum(1))
        out.update(drows=whole(gate * dy), dw=dw.reshape(T, k), dx=back(s.dxs.narrow(0, 0, s.P).double()))
    return out


def _adamw_exact(s):
    # over the whole buffers: what lies between two tensors is zero and stays so; states in 8 bits: the values before they are
    # rounded, in units of their block's scale
    eight = s.case["bits"] == 8
    p, g = s.flat["params"].double(), s.flat["grads"].double()
    m, v = s.flat["m"], s.flat["v"]
    if eight:
        block = torch.arange(p.numel(), device="cuda") // BLOCK
        m = m.view(torch.float8_e4m3fn).double() * s.flat["m_scale"].double()[block]
        v = (v.view(torch.float8_e4m3fn).double() * s.flat["v_scale"].double()[block]) ** 2
    m, v = m.double(), v.double()
    m, v = m + (1 - BETA1) * (g - m), v + (1 - BETA2) * (g * g - v)
    step = (m / (1 - BETA1 ** s.step)) / ((v / (1 - BETA2 ** s.step)).sqrt() + EPS)
    new = p - LR * (DECAY * p + step)
    out = {"params": new}
    if s.case["copy"]:
        out["copies"] = new
    if not eight:
        return {**out, "m": m, "v": v}
    for name, t in (("m", m), ("v", v.sqrt())):
        top = t.abs().view(-1, BLOCK).amax(1)
        unit = torch.where(top > 0, top / 448, torch.ones_like(top))
        out[name], out[name + "_scale"] = t / unit[block], unit
    return out


def exact(case, seed):
    with torch.no_grad():
        s = prepare(case, seed)
        return {"norm": _norm_exact, "sort": _sort_exact, "adamw": _adamw_exact}[case["kind"]](s)
