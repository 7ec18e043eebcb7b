"""Operators of layers with experts, and norms of queries and keys, as a serving program uses them.

Kinds of case, each through the package's public entry points:

``route``    the scores of E experts per token -> the k best, their weights, and the plan that lays the
             token-expert pairs out by expert (mxq.route).
``product``  the tokens quantized to MXINT by that plan (mxq.quantize_act_experts), and multiplied with
             their experts' MXINT weights, groups of ragged sizes (mxq.gemm_experts).
``down``     SiLU(gate) * up of every pair quantized by the plan (mxq.quantize_act_swiglu_experts), the
             experts' down projections (mxq.gemm_experts), and the weighted sum of a token's experts on
             top of the residual (mxq.combine_experts).
``layer``    all of them in one sequence: route, gate and up, SiLU * up, down, combine.
``norm``     queries and keys normalised per head and rotated in one pass (mxq.rope_qk).
``append``   the same on the way into the paged cache (mxq.kv_append with gains), the cached rows read
             back (mxq.kv_read).

Pair p = t * k + j is expert ids[t, j] of token t.  A plan lays the pairs out by expert, each expert's from
a multiple of 16 rows on: ``first`` [E + 1] those rows, ``pair`` [rows] the pair of each row, -1 for none.
Activations carry outlier channels; the column permutation ranks the channels by scale, so that the widest
blocks hold them.  The experts of a layer share a width map; they may each have a permutation of their own.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 32
ROWS = 16
DEVICE = "cuda"


# --------------------------------------------------------------------------
# the cases

def _product(name, T, E, k, K, N, p6=0.10, p8=0.05, low=4, out="bf16", perms="shared", kind="product"):
    c = {"kind": kind, "T": T, "E": E, "k": k, "K": K, "N": N, "p6": p6, "p8": p8, "low": low, "out": out,
         "perms": perms}
    if name:
        c["name"] = name
    return c


def _norm(name, T, Hq, Hk, D, rot, interleaved, positions, kind="norm", **more):
    c = {"kind": kind, "T": T, "Hq": Hq, "Hk": Hk, "D": D, "rot": rot, "interleaved": interleaved,
         "positions": positions}
    c.update(more)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token among 64 experts: the smallest call, latency counts
        {"name": "route_m1", "kind": "route", "T": 1, "E": 64, "k": 6, "score": "softmax", "bias": False,
         "normalise": False, "logits": "f32"},
        # a large prefill batch, sigmoid scores, a bias that balances the experts' load, bf16 logits
        {"name": "route_m8191_bias", "kind": "route", "T": 8191, "E": 256, "k": 8, "score": "sigmoid",
         "bias": True, "normalise": True, "logits": "bf16"},
        # one token through gate and up of 6 among 64 small experts: weights of 6 are streamed
        _product("gate_up_m1", 1, 64, 6, 2048, 2816),
        # 64 sequences decoding: about 4 rows for each of 128 experts, all weights are streamed
        _product("gate_up_m64", 64, 128, 8, 2048, 1536, perms="each"),
        # a short ragged prompt chunk, the 3-6-8 template, an odd column count, float32 results
        _product("up_m333_368", 333, 8, 2, 4096, 4000, 0.10, 0.10, low=3, out="f32"),
        # a 4096-token prefill through gate and up of 8 large experts: the most work
        _product("gate_up_m4096", 4096, 8, 2, 4096, 28672, 0.15, 0.15),
        # 48 sequences decoding through the down projections
        _product("down_m48", 48, 16, 4, 1408, 2048, kind="down"),
        # a 2048-token prefill through the down projections, all 4-bit but one block
        _product("down_m2048", 2048, 64, 6, 1408, 2048, 0.0, 0.01, kind="down", perms="each"),
        # a whole layer of experts on a ragged batch of 1000 tokens
        {"name": "layer_m1000", "kind": "layer", "T": 1000, "E": 32, "k": 4, "K": 2048, "F": 1792,
         "p6": 0.10, "p8": 0.05, "low": 4},
        # queries and keys of a single token
        _norm("norm_m1", 1, 32, 8, 128, 128, False, 4096),
        # a 4001-token prompt, half of the head turned in pairs, far positions, a view of fused rows
        _norm("norm_m4001_part", 4001, 40, 8, 128, 64, True, 131072),
        # one token of each of 64 sequences into the cache of a layer
        _norm("append_b64", 64, 64, 8, 128, 128, False, 8192, kind="append", widths="4444", page=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["route", "product", "product", "product", "product", "down", "down", "layer", "norm",
                       "append"])
    E = rng.choice([4, 8, 16, 32, 60, 64, 128])
    k = min(E, rng.choice([1, 2, 2, 4, 6, 8]))
    p6, p8 = rng.choice([(0.10, 0.05), (0.10, 0.10), (0.15, 0.15), (0.10, 0.30), (0.0, 0.01)])
    low = rng.choice([4, 4, 4, 3])
    if kind == "route":
        E = rng.choice([E, 96, 160, 256])
        return {"kind": kind, "T": _log(rng, 1, 8191), "E": E, "k": k, "score": rng.choice(["softmax", "sigmoid"]),
                "bias": rng.random() < 0.4, "normalise": rng.random() < 0.6,
                "logits": rng.choice(["f32", "bf16"])}
    if kind in ("product", "down", "layer"):
        K = BLOCK * _log(rng, 16, 160)
        N = _log(rng, 256, 8192)
        while E * K * N > 1 << 29:                       # (half of the largest listed case's weights)
            E //= 2
        k = min(k, E)
        T = rng.choice([_log(rng, 1, 64), _log(rng, 65, 1024), _log(rng, 1025, 8192)])
        T = max(1, min(T, (1 << 38) // (K * N * k)))
        perms = rng.choice(["shared", "each"])
        if kind == "layer":
            F = BLOCK * _log(rng, 8, 64)
            return {"kind": kind, "T": min(T, 2000), "E": E, "k": k, "K": min(K, 4096), "F": F, "p6": p6,
                    "p8": p8, "low": low}
        return _product(None, T, E, k, K, N, p6, p8, low, rng.choice(["bf16", "bf16", "f32"])
                        if kind == "product" else "bf16", perms, kind)
    Hk = rng.choice([1, 2, 4, 8, 8])
    Hq = Hk * rng.choice([1, 2, 4, 5, 8])
    T = _log(rng, 1, 8192 if Hq <= 32 else 4001)
    far = rng.choice([4096, 32768, 131072])
    pairs = rng.random() < 0.5
    if kind == "append":
        return _norm(None, min(T, 2048), Hq, Hk, 128, rng.choice([128, 128, 64, 32]), pairs, far, kind,
                     widths=rng.choice(["4444", "4468", "8888", "3368"]), page=rng.choice([16, 64, 256]))
    D = rng.choice([64, 80, 96, 128, 128, 256])
    return _norm(None, min(T, 4001 * 48 * 128 // ((Hq + Hk) * D)), Hq, Hk, D, rng.choice([D, D, D // 2]), pairs,
                 far)


# --------------------------------------------------------------------------
# inputs, made on the device from the seed alone

def _gen(seed, k):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(1000003 * (seed + 1) + k)
    return g


def _randn(shape, seed, k):
    return torch.randn(shape, generator=_gen(seed, k), device=DEVICE)


def _logits(T, E, seed, k):
    """Scores of a router: some experts are liked more than others."""
    return 1.5 * _randn((T, E), seed, k) + 0.5 * _randn((E,), seed, k + 1)


def _widths(K, p6, p8, low):
    nb = K // BLOCK
    n8 = max(1, round(p8 * nb))
    n6 = min(nb - n8, round(p6 * nb))
    return [low] * (nb - n6 - n8) + [6] * n6 + [8] * n8


def _scales(K, seed, k):
    """Per-channel scales: 1 % of the channels x20 to x100, 5 % x2 to x5."""
    u = torch.rand((K,), generator=_gen(seed, k), device=DEVICE)
    f = torch.rand((K,), generator=_gen(seed, k + 1), device=DEVICE)
    return torch.where(u < 0.01, 20 + 80 * f, torch.where(u < 0.06, 2 + 3 * f, torch.ones_like(f)))


def _perm(scales):
    return torch.argsort(scales).int()


def _perms(c, scales, E, seed, k):
    """One permutation for all experts, or one each: calibrated apart, their scales differ a little."""
    if c.get("perms", "shared") == "shared":
        return _perm(scales)
    return torch.argsort(scales * (1 + 0.2 * torch.rand((E, scales.numel()), generator=_gen(seed, k),
                                                        device=DEVICE)), dim=-1).int()


def _weights(E, N, K, seed, k):
    w = torch.empty((E, N, K), dtype=torch.bfloat16, device=DEVICE)
    for e in range(E):
        w[e] = 0.02 * _randn((N, K), seed, k + 1000 * (e + 1))
    return w


def _chosen(T, E, k, seed, at):
    """A batch's experts and weights, as a router gives them."""
    w, ids = torch.softmax(_logits(T, E, seed, at), dim=-1).topk(k, dim=-1)
    return ids.int(), w / w.sum(-1, keepdim=True)


def prepare(case, seed):
    c, kind = dict(case), case["kind"]
    s = {"case": c}
    if kind == "route":
        s["logits"] = _logits(c["T"], c["E"], seed, 1)
        if c["logits"] == "bf16":
            s["logits"] = s["logits"].to(torch.bfloat16)
        s["bias"] = 0.1 * _randn((c["E"],), seed, 3) if c["bias"] else None
        return s
    if kind in ("product", "down", "layer"):
        T, E, k, K = c["T"], c["E"], c["k"], c["K"]
        scales = _scales(K, seed, 10)
        s["widths"] = _widths(K, c["p6"], c["p8"], c["low"])
        s["perm"] = _perms(c, scales, E, seed, 12)
        if kind == "layer":
            F = c["F"]
            s["logits"] = _logits(T, E, seed, 1)
            s["x"] = (_randn((T, K), seed, 20) * scales).to(torch.bfloat16)
            s["residual"] = _randn((T, K), seed, 21).to(torch.bfloat16)
            s["w"] = _weights(E, 2 * F, K, seed, 30)
            s["widths2"] = _widths(F, c["p6"], c["p8"], c["low"])
            s["perm2"] = _perm(_scales(F, seed, 14))
            s["w2"] = _weights(E, K, F, seed, 40)
            return s
        s["ids"], s["weights"] = _chosen(T, E, k, seed, 1)
        s["first"], s["pair"] = _plan(s["ids"], E)
        s["w"] = _weights(E, c["N"], K, seed, 30)
        if kind == "product":
            s["x"] = (_randn((T, K), seed, 20) * scales).to(torch.bfloat16)
            return s
        rows = _randn((T * k, 2 * K), seed, 20)                    # gate and up of every pair, one product's rows
        rows[:, K:] *= scales
        s["gate"], s["up"] = rows.to(torch.bfloat16).split(K, dim=1)
        s["residual"] = _randn((T, c["N"]), seed, 21).to(torch.bfloat16)
        return s
    T, Hq, Hk, D = c["T"], c["Hq"], c["Hk"], c["D"]
    rows = 2 * _randn((T, Hq + 2 * Hk, D), seed, 1)                # a fused projection's rows
    rows[:, Hq:Hq + Hk, 5] *= 8
    s["q"], s["k"], s["v"] = rows.to(torch.bfloat16).split([Hq, Hk, Hk], dim=1)
    s["q_gain"], s["k_gain"] = ((1 + 0.2 * _randn((D,), seed, i)).to(torch.bfloat16) for i in (2, 3))
    s["pos"] = torch.randint(0, c["positions"], (T,), generator=_gen(seed, 4), device=DEVICE).int()
    f = 10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64, device=DEVICE) / c["rot"])
    a = torch.arange(c["positions"], dtype=torch.float64, device=DEVICE)[:, None] * f
    s["table"] = torch.stack([a.cos(), a.sin()], dim=-1).float()
    s["eps"] = 1e-6
    if kind == "append":
        s["pages"] = -(-T // c["page"]) + 3
        s["slots"] = torch.randperm(s["pages"] * c["page"], generator=_gen(seed, 5), device=DEVICE)[:T]
    return s


# --------------------------------------------------------------------------
# the framework's calls

def _own_linear(s, mxq, at=""):
    """The format and the packed weights of the experts' linear: laid out once, at model load."""
    if "packed" + at not in s:
        perm = s["perm" + at]
        each = perm if perm.dim() == 2 else None
        fmt = mxq.Format(s["w" + at].shape[2], s["widths" + at], None if each is not None else perm)
        s["packed" + at] = (fmt, each, mxq.pack_experts(s["w" + at], fmt, perms=each))
    return s["packed" + at]


def _own_plan(s, mxq):
    if "plan" not in s:
        c = s["case"]
        s["plan"] = mxq.ExpertPlan(c["T"] * c["k"], c["E"], first=s["first"], pair=s["pair"])
    return s["plan"]


def _own_image(s, mxq, fmt, plan, at=""):
    """The activations' buffers, which a serving program keeps."""
    if "image" + at not in s:
        s["image" + at] = tuple(torch.empty(n, dtype=torch.uint8, device=DEVICE)
                                for n in (fmt.act_bytes(plan.rows), fmt.act_exp_bytes(plan.rows)))
    return s["image" + at]


def _own_route(s, mxq, **more):
    c = s["case"]
    if "routed" not in s:                                          # the router's buffers, kept too
        ids = torch.empty((c["T"], c["k"]), dtype=torch.int32, device=DEVICE)
        s["routed"] = ids, torch.empty(ids.shape, dtype=torch.float32, device=DEVICE), mxq.ExpertPlan(
            ids.numel(), c["E"], device=DEVICE)
    return mxq.route(s["logits"], c["k"], out=s["routed"], **more)


def _own_run(s):
    from paper_2607_17733_amd import mxq
    c, kind = s["case"], s["case"]["kind"]
    if kind == "route":
        ids, weights, plan = _own_route(s, mxq, score=c["score"], normalise=c["normalise"], scale=2.5,
                                        bias=s["bias"])
        return ids, weights, plan.first, plan.pair
    if kind in ("product", "down", "layer"):
        fmt, perms, (wm, we) = _own_linear(s, mxq)
        ids, weights, plan = _own_route(s, mxq) if kind == "layer" else (s["ids"], s["weights"],
                                                                         _own_plan(s, mxq))
        image = _own_image(s, mxq, fmt, plan)
        if kind == "down":
            am, ae = mxq.quantize_act_swiglu_experts(s["gate"], s["up"], fmt, plan, perms=perms, out=image)
            # (float32 rows: the weighted sum's, which is rounded once, as the result)
            y = mxq.gemm_experts(am, ae, wm, we, fmt, plan, c["N"], dtype=torch.float32)
            return mxq.combine_experts(y, ids, weights, plan, residual=s["residual"])
        am, ae = mxq.quantize_act_experts(s["x"], fmt, plan, perms=perms, out=image)
        if kind == "product":
            return mxq.gemm_experts(am, ae, wm, we, fmt, plan, c["N"],
                                    dtype=torch.float32 if c["out"] == "f32" else torch.bfloat16)
        F = c["F"]
        h = mxq.gemm_experts(am, ae, wm, we, fmt, plan, 2 * F)
        fmt2, perms2, (wm2, we2) = _own_linear(s, mxq, "2")
        am, ae = mxq.quantize_act_swiglu_experts(h[:, :F], h[:, F:], fmt2, plan, perms=perms2,
                                                 out=_own_image(s, mxq, fmt2, plan, "2"))
        y = mxq.gemm_experts(am, ae, wm2, we2, fmt2, plan, c["K"], dtype=torch.float32)
        return ids, mxq.combine_experts(y, ids, weights, plan, residual=s["residual"])
    if kind == "norm":
        return mxq.rope_qk(s["q"], s["k"], s["pos"], s["table"], s["q_gain"], s["k_gain"], s["eps"],
                           interleaved=c["interleaved"])
    if "cache" not in s:                                           # the handle that a program keeps
        s["cache"] = mxq.PagedCache(mxq.Format(c["D"], [int(w) for w in c["widths"]]), c["Hk"], s["pages"],
                                    c["page"])
    q = mxq.kv_append(s["cache"], s["k"], s["v"], s["slots"], pos=s["pos"], rope=s["table"],
                      interleaved=c["interleaved"], q=s["q"], q_gain=s["q_gain"], k_gain=s["k_gain"],
                      eps=s["eps"])
    return (q,) + tuple(mxq.kv_read(s["cache"], s["slots"]))


# --------------------------------------------------------------------------
# the plain forms

def _plan(ids, E):
    """(first [E + 1], pair [rows]) of the chosen experts."""
    f = ids.flatten().long()
    P = f.numel()
    rows = (P + (ROWS - 1) * min(E, P)) // ROWS * ROWS
    count = torch.zeros(E, dtype=torch.long, device=f.device).scatter_add_(0, f, torch.ones_like(f))
    first = torch.zeros(E + 1, dtype=torch.long, device=f.device)
    first[1:] = torch.cumsum((count + ROWS - 1) // ROWS * ROWS, 0)
    order = torch.argsort(f, stable=True)
    rank = torch.arange(P, device=f.device) - (torch.cumsum(count, 0) - count)[f[order]]
    pair = torch.full((rows,), -1, dtype=torch.int32, device=f.device)
    pair[first[f[order]] + rank] = order.int()
    return first.int(), pair


def _plain_route(logits, k, score, bias, normalise, scale):
    x = logits.float()
    if score == "softmax":
        p = torch.exp(x - x.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
    else:
        p = 1 / (1 + torch.exp(-x))
    rank = x.double()                                              # (both scores rise with the logits)
    if bias is not None:                                           # next to a border 64 bits decide
        y = x.double()
        e = torch.exp(y - y.amax(-1, keepdim=True))
        rank = (e / e.sum(-1, keepdim=True) if score == "softmax" else 1 / (1 + torch.exp(-y))) + bias.double()
    ids = torch.sort(rank, dim=-1, descending=True, stable=True)[1][:, :k]
    w = p.gather(1, ids)
    if normalise:
        w = w / w.sum(-1, keepdim=True)
    return ids.int(), w * scale


def _pow2(e):
    """2^e in 32 bits for e in [-149, 254], as two factors that are both in range."""
    h = e // 2
    return torch.exp2(h.float()), torch.exp2((e - h).float())


def _quantized(x, widths):
    """bf16 [..., K], columns in order -> the values that their quantization stands for, in 32 bits."""
    y = x.unflatten(-1, (len(widths), BLOCK)).contiguous()
    E = (y.view(torch.int16).int() & 0x7FFF).amax(-1) >> 7
    m = torch.tensor(widths, device=x.device)
    a, b = _pow2(127 + m - 2 - E)
    lim = (2 ** (m - 1) - 1).float()[:, None]
    q = torch.minimum(torch.maximum(torch.round(y.float() * a[..., None] * b[..., None]), -lim), lim)
    a, b = _pow2(E - 127 - (m - 2))
    return (q * a[..., None] * b[..., None]).flatten(-2)


def _laid_out(s, at=""):
    """The experts' quantized weights, columns in the permuted order (their values are exact in bf16): once."""
    if "values" + at not in s:
        w, perm = s["w" + at], s["perm" + at].long()
        w = w[:, :, perm] if perm.dim() == 1 else w.gather(2, perm[:, None].expand(w.shape))
        s["values" + at] = _quantized(w, s["widths" + at]).to(torch.bfloat16)
    return s["values" + at]


def _plain_product(s, rows, ids, at=""):
    """rows bf16 [pairs, K] -> float32 [pairs, N]: each group padded to the longest, one batched product."""
    values, perm = _laid_out(s, at), s["perm" + at].long()
    f = ids.flatten().long()
    P, E = f.numel(), values.shape[0]
    x = rows[:, perm] if perm.dim() == 1 else rows.gather(1, perm[f])
    x = _quantized(x, s["widths" + at])
    count = torch.zeros(E, dtype=torch.long, device=f.device).scatter_add_(0, f, torch.ones_like(f))
    order = torch.argsort(f, stable=True)
    rank = torch.empty_like(f)
    rank[order] = torch.arange(P, device=f.device) - (torch.cumsum(count, 0) - count)[f[order]]
    active = torch.nonzero(count)[:, 0]                            # the groups' sizes size the product
    slot = torch.zeros_like(count)
    slot[active] = torch.arange(active.numel(), device=f.device)
    padded = x.new_zeros((active.numel(), int(count.max()), x.shape[1]))
    padded[slot[f], rank] = x
    w = values if active.numel() == E else values[active]
    return torch.bmm(padded, w.float().transpose(1, 2))[slot[f], rank]


def _plain_swiglu(gate, up):
    g = gate.float()
    return ((g / (1 + torch.exp(-g))).to(torch.bfloat16).float() * up.float()).to(torch.bfloat16)


def _plain_combine(y, weights, residual):
    T, k = weights.shape
    return (residual.float() + (weights[..., None] * y.unflatten(0, (T, k))).sum(1)).to(torch.bfloat16)


def _plain_norm(x, gain, eps, pos, table, interleaved):
    y = x.float()
    y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * gain.float()
    R = 2 * table.shape[1]
    cs = table[pos.long()]
    c, sn = cs[:, None, :, 0], cs[:, None, :, 1]
    if interleaved:
        x1, x2 = y[..., 0:R:2], y[..., 1:R:2]
        r = torch.stack([x1 * c - x2 * sn, x2 * c + x1 * sn], dim=-1).flatten(-2)
    else:
        x1, x2 = y[..., :R // 2], y[..., R // 2:R]
        r = torch.cat([x1 * c - x2 * sn, x2 * c + x1 * sn], dim=-1)
    return torch.cat([r, y[..., R:]], dim=-1).to(x.dtype)


def _plain_append(s):
    """The cache as the values that it stands for, [slots, heads, 128]."""
    c, widths = s["case"], [int(w) for w in s["case"]["widths"]]
    if "kept" not in s:
        s["kept"] = torch.zeros((2, s["pages"] * c["page"], c["Hk"], c["D"]), dtype=torch.bfloat16, device=DEVICE)
    q, k = (_plain_norm(s[x], s[x + "_gain"], s["eps"], s["pos"], s["table"], c["interleaved"]) for x in "qk")
    s["kept"][0][s["slots"]] = _quantized(k, widths).to(torch.bfloat16)
    s["kept"][1][s["slots"]] = _quantized(s["v"], widths).to(torch.bfloat16)
    return q, s["kept"][0][s["slots"]], s["kept"][1][s["slots"]]


def run(state):
    if own:
        return _own_run(state)
    s, c = state, state["case"]
    kind = c["kind"]
    if kind == "route":
        ids, w = _plain_route(s["logits"], c["k"], c["score"], s["bias"], c["normalise"], 2.5)
        return (ids, w) + _plan(ids, c["E"])
    if kind == "product":
        y = _plain_product(s, s["x"].repeat_interleave(c["k"], dim=0), s["ids"])
        return y if c["out"] == "f32" else y.to(torch.bfloat16)
    if kind == "down":
        y = _plain_product(s, _plain_swiglu(s["gate"], s["up"]), s["ids"])
        return _plain_combine(y, s["weights"], s["residual"])
    if kind == "layer":
        ids, w = _plain_route(s["logits"], c["k"], "softmax", None, True, 1.0)
        # gate and up are bf16 rows: the quantizer's input
        h = _plain_product(s, s["x"].repeat_interleave(c["k"], dim=0), ids).to(torch.bfloat16)
        y = _plain_product(s, _plain_swiglu(h[:, :c["F"]], h[:, c["F"]:]), ids, "2")
        return ids, _plain_combine(y, w, s["residual"])
    if kind == "norm":
        return tuple(_plain_norm(s[x], s[x + "_gain"], s["eps"], s["pos"], s["table"], c["interleaved"])
                     for x in "qk")
    return _plain_append(s)


# --------------------------------------------------------------------------
# what a pass cannot do without

def _linear_work(T, E, k, K, N, p6, p8, low):
    """Weights of the experts that a batch is expected to choose, and the products."""
    active = E * (1 - (1 - k / E) ** T)
    bits = sum(w * BLOCK + 8 for w in _widths(K, p6, p8, low))
    return active * N * bits / 8, 2 * T * k * N * K


def work(case):
    c, kind = case, case["kind"]
    T = c["T"]
    if kind == "route":
        P, E = T * c["k"], c["E"]
        return {"bytes": T * E * (4 if c["logits"] == "f32" else 2) + 12 * P + 4 * E, "flops": 8 * T * E}
    if kind in ("product", "down"):
        E, k, K, N = c["E"], c["k"], c["K"], c["N"]
        w, flops = _linear_work(T, E, k, K, N, c["p6"], c["p8"], c["low"])
        if kind == "product":
            return {"bytes": w + 2 * T * K + 4 * T * k + T * k * N * (4 if c["out"] == "f32" else 2),
                    "flops": flops}
        return {"bytes": w + 4 * T * k * K + 8 * T * k + 4 * T * N, "flops": flops + 2 * T * k * N}
    if kind == "layer":
        E, k, K, F = c["E"], c["k"], c["K"], c["F"]
        w1, f1 = _linear_work(T, E, k, K, 2 * F, c["p6"], c["p8"], c["low"])
        w2, f2 = _linear_work(T, E, k, F, K, c["p6"], c["p8"], c["low"])
        return {"bytes": w1 + w2 + 4 * T * E + 6 * T * K + 4 * T * k, "flops": f1 + f2 + 2 * T * k * K}
    heads, D = c["Hq"] + c["Hk"], c["D"]
    total = {"bytes": T * (heads * 4 * D + 4 + 4 * c["rot"]) + 4 * D, "flops": T * heads * (4 * D + 3 * c["rot"])}
    if kind == "append":                                           # the keys' rows are the cache's; values too
        row = sum(4 * int(m) for m in c["widths"]) + 4
        total["bytes"] += T * (8 + c["Hk"] * (4 * row + 4 * D))
    return total


# --------------------------------------------------------------------------
# the operators' values in 64 bits, from their definitions

def _exact_quantized(x, widths):
    """Values -> those that their quantization stands for, from powers of two and whole numbers in 64 bits."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    at = 0
    for m in sorted(set(widths)):                                  # the blocks of one width are adjacent
        n = widths.count(m) * BLOCK
        y = x[..., at:at + n].double().unflatten(-1, (-1, BLOCK))
        _, e = torch.frexp(y.abs().amax(-1, keepdim=True))
        unit = torch.exp2((e - 1 - (m - 2)).double())
        most = 2 ** (m - 1) - 1
        out[..., at:at + n] = ((y / unit).round().clamp(-most, most) * unit).flatten(-2)
        at += n
    return out


def _exact_product(s, rows, ids, at=""):
    f, w, perm = ids.flatten(), s["w" + at], s["perm" + at].long()
    y = torch.zeros((f.numel(), w.shape[1]), dtype=torch.float64, device=w.device)
    for e in range(w.shape[0]):
        here = torch.nonzero(f == e)[:, 0]
        if here.numel():
            p = perm if perm.dim() == 1 else perm[e]
            y[here] = _exact_quantized(rows[here][:, p], s["widths" + at]) @ _exact_quantized(
                w[e][:, p], s["widths" + at]).T
    return y


def _exact_swiglu(gate, up):
    """SiLU and the product are bf16 values by definition: those roundings are part of it."""
    g = gate.double()
    return ((g * torch.sigmoid(g)).to(torch.bfloat16).double() * up.double()).to(torch.bfloat16)


def _exact_choice(x, k, score, bias, normalise, scale):
    y = x.double()
    p = torch.softmax(y, dim=-1) if score == "softmax" else torch.sigmoid(y)
    rank = y if bias is None else p + bias.double()
    ids = torch.argsort(rank, dim=-1, descending=True, stable=True)[:, :k]
    w = p.gather(1, ids)
    return ids, scale * (w / w.sum(-1, keepdim=True) if normalise else w)


def _exact_sum(y, w, residual):
    out = residual.double()
    for j in range(w.shape[1]):
        out = out + w[:, j:j + 1].double() * y[j::w.shape[1]]
    return out


def _exact_norm(s, x):
    """Angles from the positions themselves; the table holds their cosines and sines in 32 bits."""
    c = s["case"]
    y = s[x].double()
    y = y * torch.rsqrt((y * y).sum(-1, keepdim=True) / c["D"] + s["eps"]) * s[x + "_gain"].double()
    i = torch.arange(c["rot"] // 2, device=y.device, dtype=torch.float64)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=y.device),
                       s["pos"].double()[:, None] * torch.pow(torch.full_like(i, 10000.0), -2 * i / c["rot"]))
    a = 2 * i.long() if c["interleaved"] else i.long()
    b = a + 1 if c["interleaved"] else a + c["rot"] // 2
    z = torch.complex(y[..., a].contiguous(), y[..., b].contiguous()) * turn[:, None]
    y[..., a], y[..., b] = z.real.contiguous(), z.imag.contiguous()
    return y


def exact(case, seed):
    s = prepare(case, seed)
    c, kind = s["case"], s["case"]["kind"]
    if kind == "route":
        ids, w = _exact_choice(s["logits"], c["k"], c["score"], s["bias"], c["normalise"], 2.5)
        return (ids, w) + _plan(ids, c["E"])
    if kind == "product":
        return _exact_product(s, s["x"].repeat_interleave(c["k"], dim=0), s["ids"])
    if kind == "down":
        y = _exact_product(s, _exact_swiglu(s["gate"], s["up"]), s["ids"])
        return _exact_sum(y, s["weights"], s["residual"])
    if kind == "layer":
        ids, w = _exact_choice(s["logits"], c["k"], "softmax", None, True, 1.0)
        h = _exact_product(s, s["x"].repeat_interleave(c["k"], dim=0), ids).to(torch.bfloat16)
        y = _exact_product(s, _exact_swiglu(h[:, :c["F"]], h[:, c["F"]:]), ids, "2")
        return ids, _exact_sum(y, w, s["residual"])
    if kind == "norm":
        return _exact_norm(s, "q"), _exact_norm(s, "k")
    widths = [int(w) for w in c["widths"]]
    # the turned keys are bf16 values before they are quantized: that rounding is part of the definition
    return (_exact_norm(s, "q"), _exact_quantized(_exact_norm(s, "k").to(torch.bfloat16), widths),
            _exact_quantized(s["v"], widths))
