"""Routing, plans, the quantizers by a plan, the grouped products and their weighted
sum against the oracle, and a layer's step of them together.

Bounds.  Choices and plans are whole numbers and have to be equal.  A weight's
relative error is documented as below 1e-6.  A product sums K exact digit products
in float32: each of at most K / 64 + 16 additions (64 at least to an instruction;
the waves' sums) rounds by 2^-24 of what the terms add up to, and an instruction
aligns its terms to the largest, 2^-24 of it each: (K / 64 + 16) 2^-23 of the terms'
absolute sum.  bf16 results are off by half a step, 2^-8, more.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import experts as oe
from oracle.paged import to_bf16, to_f32
from paper_2607_17733_amd import mxq
from parity_util import say, to_dev_bf16

pytestmark = pytest.mark.gpu


def bits_of(t):
    return t.cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


def _randn(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def _widths(nb, mix):
    """About a tenth of the blocks each of the wider widths of the mix."""
    n = max(1, nb // 10)
    rest = [m for m in mix[1:]]
    rest = rest[-max(0, nb - 1) // n:] if nb > 1 else []
    w = [m for m in rest for _ in range(n)][-(nb - 1):] if nb > 1 else []
    return [mix[0]] * (nb - len(w)) + w


# --------------------------------------------------------------------------
# routing and plans

def _check_route(x, k, **kw):
    ids, w, plan = mxq.route(x.cuda(), k, **{n: v.cuda() if isinstance(v, torch.Tensor) else v
                                            for n, v in kw.items()})
    torch.cuda.synchronize()
    ref = {n: v.numpy() if isinstance(v, torch.Tensor) else v for n, v in kw.items()}
    want, ww = oe.route(x.float().numpy(), k, **ref)
    assert np.array_equal(ids.cpu().numpy(), want)
    got = w.cpu().numpy().astype(np.float64)
    assert np.all(np.abs(got - ww) <= 1e-6 * np.abs(ww) + 1e-37)
    first, pair = oe.plan(want, x.shape[1])
    assert np.array_equal(plan.first.cpu().numpy(), first)
    assert np.array_equal(plan.pair.cpu().numpy(), pair)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 6), (3, 3, 3), (17, 65, 7), (33, 8, 2), (130, 200, 8),
                                   (257, 256, 8), (64, 128, 8), (9, 512, 32), (5, 1000, 10), (4, 1024, 32)])
def test_route(T, E, k, score, bias):
    say("route", T, E, k, score, bias)
    x = 2 * _randn((T, E), T + E)
    b = 0.3 * _randn((E,), E) if bias else None
    _check_route(x, k, score=score, bias=b, normalise=T % 2 == 0, scale=2.5)
    _check_route(x.to(torch.bfloat16), k, score=score, bias=b, normalise=T % 2 == 1)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [False, True])
def test_route_ties_masks_and_infinities(score, bias):
    inf, nan = float("inf"), float("nan")
    rows = [[0.0] * 70, [-inf] * 70, [nan] * 70, [-inf] * 69 + [1.0], [nan] * 30 + [2.0, 2.0] + [-inf] * 38,
            [inf] * 3 + [0.0] * 67, [3e38] * 2 + [inf] + [-3e38] * 67, [-200.0] * 70, [200.0] * 70,
            [-0.0, 0.0] * 35, [1e-45, -1e-45] * 35, [-3e38] * 70]
    x = torch.tensor(rows)
    b = torch.zeros(70) if bias else None
    for k in (1, 4, 32):
        for normalise in (False, True):
            _check_route(x, k, score=score, bias=b, normalise=normalise)


def test_route_bias_that_rules_experts_out():
    inf, nan = float("inf"), float("nan")
    x = _randn((20, 40), 1)
    b = 0.1 * _randn((40,), 2)
    b[3], b[7], b[11], b[12], b[39] = -inf, nan, inf, inf, 1e30
    for score in ("softmax", "sigmoid"):
        _check_route(x, 6, score=score, bias=b)
    b[:] = -inf
    b[5] = 0.0
    _check_route(x, 3, score="sigmoid", bias=b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_route_strided_and_odd_rows(dtype):
    full = _randn((37, 101), 5).to(dtype).cuda()
    x = full[:, 3:96]
    ids, w, plan = mxq.route(x, 5)
    want, ww = oe.route(x.float().cpu().numpy(), 5)
    assert np.array_equal(ids.cpu().numpy(), want)
    assert np.all(np.abs(w.cpu().numpy() - ww) <= 1e-6 * ww)


@pytest.mark.parametrize("T,E,k,how", [(0, 5, 2, "any"), (1, 1, 1, "any"), (1, 1024, 4, "any"), (5, 4, 3, "one"),
                                       (100, 7, 3, "any"), (333, 128, 8, "any"), (4096, 8, 2, "any"),
                                       (4099, 300, 8, "any"), (700, 16, 4, "none"), (700, 16, 4, "one"),
                                       (70000, 64, 1, "any"), (16, 1024, 32, "any")])
def test_expert_plan(T, E, k, how):
    say("plan", T, E, k, how)
    g = torch.Generator().manual_seed(T + E)
    ids = torch.randint(-2, E + 3, (T, k), generator=g).int()
    if how == "one":
        ids[:] = E - 1
    if how == "none":
        ids[:] = -1
        ids[::2] = 2 ** 31 - 1
    plan = mxq.expert_plan(ids.cuda(), E)
    first, pair = oe.plan(ids.numpy(), E)
    assert np.array_equal(plan.first.cpu().numpy(), first)
    assert np.array_equal(plan.pair.cpu().numpy(), pair)


def test_plan_is_written_again():
    g = torch.Generator().manual_seed(3)
    plan = None
    for i in range(4):
        ids = torch.randint(-1, 9, (50, 3), generator=g).int()
        plan = mxq.expert_plan(ids.cuda(), 9, out=plan)
        first, pair = oe.plan(ids.numpy(), 9)
        assert np.array_equal(plan.first.cpu().numpy(), first) and np.array_equal(plan.pair.cpu().numpy(), pair)


# --------------------------------------------------------------------------
# the quantizers by a plan

def _byte_rows(widths, rows):
    """The image row that each byte of the mantissas and of the scales belongs to."""
    n = [sum(1 for w in widths if w == m) for m in (3, 4, 6, 8)]
    S = [-(-n[0] // 4), -(-n[1] // 4), -(-n[2] // 2), -(-n[3] // 2)]
    lane = np.arange(64) % 16
    tile = np.concatenate([np.tile(lane.repeat(24), S[0] + S[1] + S[2]), np.tile(lane.repeat(32), S[3])])
    scale = np.tile(lane.repeat(4), sum(-(-s // 4) for s in S))
    at = np.arange(rows // 16)[:, None] * 16
    return (at + tile).reshape(-1), (at + scale).reshape(-1)


def _image_case(T, E, k, K, mix, perms, swiglu=False, per_pair=False, seed=0, clamp="sym", round_="rne", ld=0,
                skip=0.1):
    g = torch.Generator().manual_seed(seed + T + E + K)
    widths = _widths(K // 32, mix)
    ids = torch.randint(0, E, (T, k), generator=g).int()
    ids[torch.rand((T, k), generator=g) < skip] = -1
    plan = mxq.expert_plan(ids.cuda(), E)
    order = torch.stack([torch.randperm(K, generator=g) for _ in range(E)]).int().cuda()
    fmt = mxq.Format(K, widths, order[0].clone() if perms == "shared" else None, round=round_, clamp=clamp)
    n = T * k if per_pair or swiglu else T
    x = (torch.randn((n, K + ld), generator=g) * 3).to(torch.bfloat16).cuda()[:, :K]
    u = torch.randn((n, K + ld), generator=g).to(torch.bfloat16).cuda()[:, :K]
    return ids, plan, fmt, order if perms == "each" else None, x, u


@pytest.mark.parametrize("perms", ["none", "shared", "each"])
@pytest.mark.parametrize("T,E,k,K,mix", [(1, 4, 1, 32, (4,)), (1, 64, 6, 512, (4, 6, 8)),
                                         (7, 3, 2, 96, (3, 6, 8)), (40, 16, 4, 1408, (4, 6, 8)),
                                         (300, 8, 2, 1024, (4, 8)), (64, 128, 8, 640, (3, 8)),
                                         (2000, 5, 3, 160, (6,)), (129, 2, 2, 4096, (4, 6, 8)),
                                         (3, 2, 2, 20480, (4, 6, 8))])
@pytest.mark.parametrize("kind", ["tokens", "pairs", "swiglu"])
def test_images_are_those_of_the_plain_quantizers(T, E, k, K, mix, perms, kind):
    say("image", T, E, k, K, mix, perms, kind)
    ids, plan, fmt, each, x, u = _image_case(T, E, k, K, mix, perms, kind == "swiglu", kind == "pairs",
                                             ld=8 if T % 2 else 3)
    pair = plan.pair.cpu().numpy()
    first = plan.first.cpu().numpy()
    live = pair >= 0
    noise = [torch.randint(0, 256, (n,), dtype=torch.uint8).cuda()
             for n in (fmt.act_bytes(plan.rows), fmt.act_exp_bytes(plan.rows))]
    out = tuple(t.clone() for t in noise)
    if kind == "swiglu":
        got = mxq.quantize_act_swiglu_experts(x, u, fmt, plan, perms=each, out=out)
    else:
        got = mxq.quantize_act_experts(x, fmt, plan, perms=each, out=out)
    # the same rows, gathered by hand, through the plain quantizers (one expert's at a time)
    src = torch.from_numpy(np.where(live, pair, 0) // (1 if x.shape[0] == ids.numel() else k)).cuda()
    rows = x[src].contiguous()
    ups = u[src].contiguous()
    want = tuple(t.clone() for t in noise)
    tb, sb = fmt.act_bytes(16), fmt.act_exp_bytes(16)
    for e in range(E):
        a, b = int(first[e]), int(first[e + 1])
        if a == b:
            continue
        f = fmt if each is None else mxq.Format(K, fmt.widths, each[e])
        part = (want[0][a // 16 * tb:b // 16 * tb], want[1][a // 16 * sb:b // 16 * sb])
        if kind == "swiglu":
            mxq.quantize_act_swiglu(rows[a:b], ups[a:b], f, out=part)
        else:
            mxq.quantize_act(rows[a:b], f, out=part)
    torch.cuda.synchronize()
    for g, w, z, at in zip(got, want, noise, _byte_rows(list(fmt.widths), plan.rows)):
        g, w, z = g.cpu().numpy(), w.cpu().numpy(), z.cpu().numpy()
        assert np.array_equal(g[live[at]], w[live[at]])
        assert np.array_equal(g[~live[at]], z[~live[at]])


# --------------------------------------------------------------------------
# the grouped products

def _product_case(T, E, k, K, N, mix=(4, 6, 8), perms="none", out=torch.float32, clamp="sym", round_="rne",
                  how="any", ldy=0, seed=0, skip=0.1, sample=None):
    say("product", T, E, k, K, N, mix, perms, out, clamp, how)
    g = torch.Generator().manual_seed(seed + T + E + K + N)
    widths = _widths(K // 32, mix)
    ids = torch.randint(0, E, (T, k), generator=g).int()
    if how == "one":
        ids[:] = E - 1
    elif how == "skewed":
        ids = (ids.float() ** 2 / max(1, E - 1)).int()
    if skip:
        ids[torch.rand((T, k), generator=g) < skip] = -1
    x = torch.randn((T, K), generator=g)
    x[:, 5] *= 20
    x = x.to(torch.bfloat16)
    w = (0.02 * torch.randn((E, N, K), generator=g)).to(torch.bfloat16)
    order = torch.stack([torch.randperm(K, generator=g) for _ in range(E)]).int()
    shared = order[0].clone().cuda() if perms == "shared" else None
    fmt = mxq.Format(K, widths, shared, round=round_, clamp=clamp)
    each = order.cuda() if perms == "each" else None
    plan = mxq.expert_plan(ids.cuda(), E)
    wm, we = mxq.pack_experts(w.cuda(), fmt, perms=each)
    am, ae = mxq.quantize_act_experts(x.cuda(), fmt, plan, perms=each)
    y = torch.full((T * k, N + ldy), 7.0, dtype=out, device="cuda")
    got = mxq.gemm_experts(am, ae, wm, we, fmt, plan, N, out=y)
    torch.cuda.synchronize()
    p = None if perms == "none" else order[0].numpy() if perms == "shared" else order.numpy()
    f = ids.reshape(-1).numpy().copy()
    if sample is not None:                               # the oracle of some of the pairs
        keep = np.zeros(f.size, bool)
        keep[np.random.RandomState(seed).permutation(f.size)[:sample]] = True
        chosen = f >= 0
        f[~keep] = -1
    want, big = oe.product(bits_of(x).repeat(k, axis=0), bits_of(w), f, p, widths,
                           1 if round_ == "rna" else 0, 1 if clamp == "full" else 0)
    y = got.float().cpu().numpy().astype(np.float64)
    here = f >= 0
    tol = (K / 64 + 16) * 2.0 ** -23 * big[here]
    if out is torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(want[here]) + tol)
    d = np.abs(y[here][:, :N] - want[here])
    assert np.all(d <= tol), (float(d.max()), float(tol.min()), np.unravel_index(np.argmax(d - tol), d.shape))
    gone = f < 0 if sample is None else ~chosen
    assert np.all(y[gone] == 7.0) and np.all(y[:, N:] == 7.0)
    return got


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,E,k,K,N", [(1, 1, 1, 32, 1), (1, 64, 6, 512, 130), (2, 3, 2, 96, 16), (5, 4, 4, 128, 40),
                                       (16, 8, 2, 1408, 100), (64, 128, 8, 256, 96), (33, 5, 1, 160, 257),
                                       (100, 7, 3, 640, 200), (300, 4, 2, 512, 384), (512, 2, 1, 256, 1000),
                                       (1500, 8, 2, 128, 300), (2100, 3, 2, 384, 520), (40, 1024, 32, 64, 33)])
def test_product(T, E, k, K, N, out):
    _product_case(T, E, k, K, N, out=out, perms=("none", "shared", "each")[T % 3])


@pytest.mark.parametrize("mix", [(3,), (4,), (6,), (8,), (3, 6, 8), (4, 6), (3, 8), (3, 4, 6, 8)])
@pytest.mark.parametrize("clamp", ["sym", "full"])
@pytest.mark.parametrize("T", [3, 70, 700])
def test_product_of_width_mixes(T, mix, clamp):
    _product_case(T, 3, 2, 32 * 23, 150, mix=mix, clamp=clamp, round_="rna" if T == 70 else "rne", perms="each")


@pytest.mark.parametrize("how", ["one", "skewed"])
@pytest.mark.parametrize("T,E,k", [(20, 6, 2), (70, 40, 3), (900, 6, 2), (1300, 70, 2)])
def test_product_of_uneven_groups(T, E, k, how):
    _product_case(T, E, k, 256, 200, how=how, out=torch.bfloat16)


@pytest.mark.parametrize("T,E,k,K,N", [(9, 6, 2, 256, 100), (90, 6, 2, 256, 129), (1000, 3, 2, 256, 260)])
@pytest.mark.parametrize("ldy", [1, 4, 8, 100])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_product_into_strided_rows(T, E, k, K, N, ldy, out):
    _product_case(T, E, k, K, N, ldy=ldy, out=out)


@pytest.mark.parametrize("T,E,k,K,N", [(64, 16, 4, 2048, 2816), (4096, 8, 2, 1024, 2048), (777, 32, 4, 4096, 1000),
                                       (16, 8, 2, 4096, 28672)])
def test_product_at_size(T, E, k, K, N):
    _product_case(T, E, k, K, N, sample=150, perms="shared", skip=0.0)


def test_products_repeat_bit_for_bit_and_do_not_depend_on_other_rows():
    a = _product_case(50, 4, 2, 512, 200, skip=0.0)
    b = _product_case(50, 4, 2, 512, 200, skip=0.0)
    assert torch.equal(a, b)


def test_product_without_rows():
    fmt = mxq.Format(64, [4, 4])
    w = torch.zeros((3, 20, 64), dtype=torch.bfloat16, device="cuda")
    wm, we = mxq.pack_experts(w, fmt)
    for ids in (torch.empty((0, 2), dtype=torch.int32), torch.full((5, 2), -1, dtype=torch.int32)):
        plan = mxq.expert_plan(ids.cuda(), 3)
        x = torch.ones((max(1, ids.shape[0]), 64), dtype=torch.bfloat16, device="cuda")[:ids.shape[0]]
        am, ae = mxq.quantize_act_experts(x, fmt, plan)
        y = torch.full((ids.numel(), 20), 3.0, device="cuda")
        mxq.gemm_experts(am, ae, wm, we, fmt, plan, 20, out=y)
        assert bool((y == 3.0).all())
        o = mxq.combine_experts(y, ids.cuda(), torch.ones(ids.shape, device="cuda"), plan)
        assert o.shape == (ids.shape[0], 20) and bool((o == 0).all())


def test_nan_and_infinite_rows_stay_their_own():
    fmt = mxq.Format(128, [4, 4, 6, 8])
    g = torch.Generator().manual_seed(0)
    x = torch.randn((40, 128), generator=g).to(torch.bfloat16)
    w = torch.randn((2, 50, 128), generator=g).to(torch.bfloat16).cuda()
    ids = torch.randint(0, 2, (40, 1), generator=g).int().cuda()
    plan = mxq.expert_plan(ids, 2)
    wm, we = mxq.pack_experts(w, fmt)
    y = mxq.gemm_experts(*mxq.quantize_act_experts(x.cuda(), fmt, plan), wm, we, fmt, plan, 50,
                         dtype=torch.float32)
    z = x.clone()
    z[3, 7], z[17, 100] = float("nan"), float("inf")
    yz = mxq.gemm_experts(*mxq.quantize_act_experts(z.cuda(), fmt, plan), wm, we, fmt, plan, 50,
                          dtype=torch.float32)
    rest = torch.ones(40, dtype=torch.bool, device="cuda")
    rest[[3, 17]] = False
    assert torch.equal(y[rest], yz[rest]) and bool(yz[~rest].isnan().all())


# --------------------------------------------------------------------------
# the weighted sum

@pytest.mark.parametrize("T,k,N", [(1, 1, 1), (1, 6, 2048), (7, 2, 33), (64, 8, 256), (301, 3, 1000), (3, 32, 8)])
@pytest.mark.parametrize("y32,o32,residual,pad", [(False, False, "own", 0), (True, True, None, 0),
                                                  (False, True, "own", 8), (True, False, "in place", 3),
                                                  (False, False, None, 1), (False, False, "in place", 16)])
def test_combine(T, k, N, y32, o32, residual, pad):
    say("combine", T, k, N, y32, o32, residual, pad)
    g = torch.Generator().manual_seed(T + k + N)
    E = 5
    ids = torch.randint(-1, E + 1, (T, k), generator=g).int()
    w = torch.randn((T, k), generator=g)
    y = torch.randn((T * k, N + pad), generator=g)
    y = y if y32 else y.to(torch.bfloat16)
    out = (ids.reshape(-1) < 0) | (ids.reshape(-1) >= E)
    y[out] = float("nan")                                # nobody's rows
    w[(ids < 0) | (ids >= E)] = float("nan")
    res = None if residual is None else torch.randn((T, N + pad), generator=g).to(torch.bfloat16)
    plan = mxq.ExpertPlan(T * k, E)
    r = None if res is None else res.cuda()[:, :N]
    got = mxq.combine_experts(y.cuda()[:, :N], ids.cuda(), w.cuda(), plan, residual=r,
                              out=r if residual == "in place" else None,
                              dtype=torch.float32 if o32 else torch.bfloat16)
    want, big = oe.combine(y[:, :N].double().numpy(), ids.numpy(), w.numpy(), E,
                           None if res is None else res[:, :N].float().numpy())
    d = np.abs(got.double().cpu().numpy() - want)
    f32 = got.dtype is torch.float32
    assert (got.dtype is torch.float32) == (o32 and residual != "in place")
    # a rounding to float32 per term, then the result's
    tol = k * 2.0 ** -24 * big
    assert np.all(d <= (tol if f32 else tol + 2.0 ** -8 * (np.abs(want) + tol)))


# --------------------------------------------------------------------------
# a layer's step

class Layer:
    """Router, gate and up, SiLU * up, down, weighted sum, as a serving program runs them."""

    def __init__(self, T, E, k, K, F, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.T, self.E, self.k, self.K, self.F = T, E, k, K, F
        self.fmt1 = mxq.Format(K, _widths(K // 32, (4, 6, 8)), torch.randperm(K, generator=g).int().cuda())
        self.fmt2 = mxq.Format(F, _widths(F // 32, (4, 6, 8)))
        self.perms2 = torch.stack([torch.randperm(F, generator=g) for _ in range(E)]).int().cuda()
        self.w1 = (0.05 * torch.randn((E, 2 * F, K), generator=g)).to(torch.bfloat16)
        self.w2 = (0.05 * torch.randn((E, K, F), generator=g)).to(torch.bfloat16)
        self.p1 = mxq.pack_experts(self.w1.cuda(), self.fmt1)
        self.p2 = mxq.pack_experts(self.w2.cuda(), self.fmt2, perms=self.perms2)
        self.inputs(seed)

    def inputs(self, seed):
        g = torch.Generator().manual_seed(1000 + seed)
        x = torch.randn((self.T, self.K), generator=g).to(torch.bfloat16)
        logits = torch.randn((self.T, self.E), generator=g)
        if hasattr(self, "x"):
            self.x.copy_(x)
            self.logits.copy_(logits)
        else:
            self.x, self.logits = x.cuda(), logits.cuda()
        return self

    def run(self):
        F = self.F
        ids, w, plan = mxq.route(self.logits, self.k)
        h = mxq.gemm_experts(*mxq.quantize_act_experts(self.x, self.fmt1, plan), *self.p1, self.fmt1, plan, 2 * F)
        a2 = mxq.quantize_act_swiglu_experts(h[:, :F], h[:, F:], self.fmt2, plan, perms=self.perms2)
        y = mxq.gemm_experts(*a2, *self.p2, self.fmt2, plan, self.K, dtype=torch.float32)
        return ids, w, h, y, mxq.combine_experts(y, ids, w, plan, residual=self.x)

    def check(self):
        from oracle import fused
        ids, w, h, y, o = (t.cpu() for t in self.run())
        want, _ = oe.route(self.logits.cpu().numpy(), self.k)
        assert np.array_equal(ids.numpy(), want)
        K, F, k = self.K, self.F, self.k
        xb = bits_of(self.x).repeat(k, axis=0)
        hr, big = oe.product(xb, bits_of(self.w1), want, self.fmt1.perm.cpu().numpy(), list(self.fmt1.widths))
        tol = (K / 64 + 16) * 2.0 ** -23 * big
        assert np.all(np.abs(h.double().numpy() - hr) <= tol + 2.0 ** -8 * (np.abs(hr) + tol))
        # from the framework's own rows on, so that a rounding does not count twice
        hb = bits_of(h)
        act = fused.swiglu_bf16(hb[:, :F], hb[:, F:])
        yr, big = oe.product(act, bits_of(self.w2), want, self.perms2.cpu().numpy(), list(self.fmt2.widths))
        assert np.all(np.abs(y.double().numpy() - yr) <= (F / 64 + 16) * 2.0 ** -23 * big)
        orf, big = oe.combine(y.double().numpy(), want, w.numpy(), self.E, self.x.float().cpu().numpy())
        tol = k * 2.0 ** -24 * big
        assert np.all(np.abs(o.double().numpy() - orf) <= tol + 2.0 ** -8 * (np.abs(orf) + tol))
        return o


@pytest.mark.parametrize("T,E,k,K,F", [(1, 8, 2, 256, 96), (5, 16, 4, 512, 160), (64, 8, 2, 256, 256),
                                       (700, 4, 2, 256, 128)])
def test_layer(T, E, k, K, F):
    Layer(T, E, k, K, F).check()


def test_layer_captured_and_replayed():
    """One capture serves other inputs (and so other groups); eager work in between."""
    a, eager = Layer(40, 8, 2, 256, 128), Layer(33, 8, 2, 256, 128, seed=1)
    a.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = a.run()
    for seed in range(4):
        a.inputs(seed)
        graph.replay()
        other = eager.run()
        got = [t.clone() for t in out]
        torch.cuda.synchronize()
        for g, w in zip(got, a.run()):
            assert torch.equal(g, w)
        for g, w in zip(other, eager.run()):
            assert torch.equal(g, w)


def test_layers_on_two_streams():
    a, b = Layer(30, 8, 2, 256, 128), Layer(300, 4, 2, 256, 96, seed=2)
    want = a.run(), b.run()
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(s):
            x = a.run()
        with torch.cuda.stream(t):
            y = b.run()
        torch.cuda.synchronize()
        for got, ref in zip((x, y), want):
            for g, w in zip(got, ref):
                assert torch.equal(g, w)


# --------------------------------------------------------------------------
# where it can go wrong

@pytest.mark.parametrize("T,E,k", [(0, 8, 2), (31, 64, 8), (32, 64, 8), (32, 1024, 8), (33, 64, 8), (16, 64, 16),
                                   (17, 64, 16), (8, 64, 32), (9, 64, 32), (256, 5, 1), (2048, 4, 1), (2049, 4, 1)])
def test_route_at_the_borders_of_its_launches(T, E, k):
    _check_route(_randn((T, E), T + k), k)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_neighbours_that_32_bits_cannot_tell_apart(score):
    """Scores one unit of the logits apart, in an order that only 64 bits show."""
    g = np.random.RandomState(0)
    x = np.zeros((64, 96), np.float32)
    for t in range(64):
        steps = g.permutation(96)
        v = np.float32(0.5 + t / 16)
        x[t] = (np.full(96, v, np.float32).view(np.int32) + steps.astype(np.int32)).view(np.float32)
    b = torch.zeros(96)
    for bias in (None, b, b + 0.25, 1e-9 * torch.from_numpy(g.randn(96).astype(np.float32))):
        _check_route(torch.from_numpy(x), 7, score=score, bias=bias)


def test_products_past_2_to_the_32_elements_of_y():
    """140000 pairs of 32768 columns: 9.2 GB of bf16 results."""
    T, N, K = 140000, 32768, 32
    g = torch.Generator().manual_seed(0)
    x = torch.randn((T, K), generator=g).to(torch.bfloat16)
    w = torch.randn((2, N, K), generator=g).to(torch.bfloat16)
    ids = torch.randint(0, 2, (T, 1), generator=g).int()
    fmt = mxq.Format(K, [4])
    plan = mxq.expert_plan(ids.cuda(), 2)
    wm, we = mxq.pack_experts(w.cuda(), fmt)
    y = mxq.gemm_experts(*mxq.quantize_act_experts(x.cuda(), fmt, plan), wm, we, fmt, plan, N)
    at = np.array([0, 1, 65535, 131071, 131072, 131073, T - 2, T - 1])
    want, big = oe.product(bits_of(x)[at], bits_of(w), ids.numpy()[at], None, [4])
    got = y[torch.from_numpy(at).cuda()].double().cpu().numpy()
    tol = 17 * 2.0 ** -23 * big
    assert np.all(np.abs(got - want) <= tol + 2.0 ** -8 * (np.abs(want) + tol))
    o = mxq.combine_experts(y, ids.cuda(), torch.full((T, 1), 0.5, device="cuda"), plan)
    assert torch.equal(o[-5:], (y[-5:].float() * 0.5).to(torch.bfloat16))


def test_source_rows_past_2_to_the_32_elements():
    """Rows 65536 elements apart, the last ones 9 GB behind the first."""
    T, ld, K = 70000, 65536, 512
    x = torch.zeros((T, ld), dtype=torch.bfloat16, device="cuda")
    view = x[:, 64:64 + K]
    view.copy_(torch.randn((T, K), device="cuda"))
    fmt = mxq.Format(K, [4] * 12 + [6] * 2 + [8] * 2)
    ids = torch.zeros((T, 1), dtype=torch.int32)
    ids[:-40] = -1                                       # the last 40 tokens alone choose
    plan = mxq.expert_plan(ids.cuda(), 1)
    near = torch.zeros((40, 1), dtype=torch.int32)
    small = mxq.expert_plan(near.cuda(), 1)
    last = view[-40:].contiguous()
    for u in (None, x[:, 1024:1024 + K]):
        if u is None:
            a = mxq.quantize_act_experts(view, fmt, plan)
            b = mxq.quantize_act_experts(last, fmt, small)
        else:
            u.copy_(torch.randn((T, K), device="cuda"))
            a = mxq.quantize_act_swiglu_experts(view, u, fmt, plan)
            b = mxq.quantize_act_swiglu_experts(last, u[-40:].contiguous(), fmt, small)
        for s, t, rows in zip(a, b, _byte_rows(list(fmt.widths), 48)):
            s, t = s[:t.numel()].cpu().numpy(), t.cpu().numpy()
            assert np.array_equal(s[rows < 40], t[rows < 40])


def test_weights_past_4_gb():
    """The last of 80 experts of 62 MB each."""
    E, N, K = 80, 28672, 4096
    fmt = mxq.Format(K, [4] * 128)
    w = (0.02 * torch.randn((1, N, K), device="cuda")).to(torch.bfloat16)
    one = mxq.pack_experts(w, fmt)
    many = [torch.zeros((E, t.shape[1]), dtype=torch.uint8, device="cuda") for t in one]
    for m, t in zip(many, one):
        m[-1:] = t
    x = torch.randn((20, K), device="cuda").to(torch.bfloat16)
    ids = torch.full((20, 1), E - 1, dtype=torch.int32, device="cuda")
    plan = mxq.expert_plan(ids, E)
    y = mxq.gemm_experts(*mxq.quantize_act_experts(x, fmt, plan), *many, fmt, plan, N, dtype=torch.float32)
    first = mxq.expert_plan(torch.zeros_like(ids), E)
    many[0][0], many[1][0] = one[0][0], one[1][0]
    z = mxq.gemm_experts(*mxq.quantize_act_experts(x, fmt, first), *many, fmt, first, N, dtype=torch.float32)
    assert torch.equal(y, z) and bool((y != 0).any())


def test_permutations_with_entries_out_of_range():
    """They read as zeros, as in the plain quantizer."""
    g = torch.Generator().manual_seed(4)
    K, E = 96, 3
    perms = torch.stack([torch.randperm(K, generator=g) for _ in range(E)]).int()
    perms[0, 5], perms[1, 40], perms[2, 95] = -1, K, 2 ** 31 - 1
    x = torch.randn((30, K), generator=g).to(torch.bfloat16).cuda()
    ids = torch.randint(0, E, (30, 1), generator=g).int()
    plan = mxq.expert_plan(ids.cuda(), E)
    fmt = mxq.Format(K, [4, 6, 8])
    w = torch.randn((E, 40, K), generator=g).to(torch.bfloat16).cuda()
    wm, we = mxq.pack_experts(w, fmt, perms=perms.cuda())
    am, ae = mxq.quantize_act_experts(x, fmt, plan, perms=perms.cuda())
    y = mxq.gemm_experts(am, ae, wm, we, fmt, plan, 40, dtype=torch.float32)
    for e in range(E):
        here = torch.nonzero(ids[:, 0] == e)[:, 0].cuda()
        f = mxq.Format(K, [4, 6, 8], perms[e].cuda())
        want = mxq.gemm(*mxq.quantize_act(x[here].contiguous(), f), *mxq.pack_weights(w[e], f), f, len(here), 40)
        assert torch.allclose(y[here], want, rtol=1e-5, atol=1e-5)


def test_refused_tensors():
    """Checks of the binding that need device tensors."""
    fmt = mxq.Format(64, [4, 4])
    x = torch.zeros((6, 64), dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros((6, 2), dtype=torch.int32, device="cuda")
    plan = mxq.expert_plan(ids, 4)
    am, ae = mxq.quantize_act_experts(x, fmt, plan)
    w = torch.zeros((4, 20, 64), dtype=torch.bfloat16, device="cuda")
    wm, we = mxq.pack_experts(w, fmt)
    y = torch.zeros((12, 20), device="cuda")
    weights = torch.zeros((6, 2), device="cuda")
    for f in (lambda: mxq.route(x, 65), lambda: mxq.route(x, 2, score="max"), lambda: mxq.route(x.half(), 2),
              lambda: mxq.route(x, 2, bias=torch.zeros(63, device="cuda")),
              lambda: mxq.route(x, 2, out=(ids, weights, plan)),            # a plan of 4 experts, not 64
              lambda: mxq.route(x, 2, scale=float("nan")), lambda: mxq.route(x.expand(6, 64)[:, ::2], 2),
              lambda: mxq.expert_plan(ids.long(), 4), lambda: mxq.expert_plan(ids[:, :1], 4),
              lambda: mxq.expert_plan(ids, 5, out=plan),
              lambda: mxq.expert_plan(ids, 4, out=mxq.ExpertPlan(12, 4, first=plan.first, pair=plan.pair)),
              lambda: mxq.quantize_act_experts(x[:5], fmt, plan), lambda: mxq.quantize_act_experts(x[:, :32], fmt, plan),
              lambda: mxq.quantize_act_experts(x, fmt, plan, perms=torch.zeros((3, 64), dtype=torch.int32, device="cuda")),
              lambda: mxq.quantize_act_experts(x, fmt, plan, out=(am[:-1], ae)),
              lambda: mxq.gemm_experts(am, ae, wm[:3].contiguous(), we, fmt, plan, 20),
              lambda: mxq.gemm_experts(am, ae, wm, we, fmt, plan, 200), lambda: mxq.gemm_experts(am, ae, wm, we, fmt, plan, -1),
              lambda: mxq.gemm_experts(am, ae, wm, we, fmt, plan, 20, out=y[:11]),
              lambda: mxq.gemm_experts(am, ae, wm, we, fmt, plan, 20, dtype=torch.float16),
              lambda: mxq.combine_experts(y[:10], ids, weights, plan), lambda: mxq.combine_experts(y, ids, weights[:5], plan),
              lambda: mxq.combine_experts(y, ids, weights, plan, residual=y[:6]),
              lambda: mxq.combine_experts(y, ids, weights, plan, out=y[:5]),
              lambda: mxq.pack_experts(w.float(), fmt), lambda: mxq.pack_experts(w[0], fmt)):
        with pytest.raises(mxq.MxqError):
            f()


# --------------------------------------------------------------------------
# the tiled kernel: groups of 32 rows and more, 1.4 tiles of 128 rows per CU and more

@pytest.mark.parametrize("clamp", ["sym", "full"])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,E,k,K,N,how", [(1400, 4, 2, 32, 5000, "any"), (1400, 4, 2, 736, 4999, "skewed"),
                                           (700, 9, 2, 160, 9000, "any"), (300, 4, 2, 96, 20000, "skewed"),
                                           (257, 2, 1, 1408, 33000, "one"), (2000, 40, 2, 352, 3001, "skewed")])
def test_product_on_tiles(T, E, k, K, N, how, out, clamp):
    _product_case(T, E, k, K, N, how=how, out=out, clamp=clamp, sample=120, perms="shared",
                  mix=(4, 6, 8) if K > 32 else (4,), ldy=T % 8)


@pytest.mark.parametrize("clamp", ["sym", "full"])
@pytest.mark.parametrize("mix", [(3,), (4,), (6,), (8,), (3, 6, 8), (4, 6), (3, 8), (3, 4, 6, 8)])
def test_product_on_tiles_of_width_mixes(mix, clamp):
    for blocks in (1, 5, 23):
        _product_case(450, 5, 2, 32 * blocks, 9000, mix=mix, clamp=clamp, sample=60, how="skewed",
                      round_="rna" if blocks == 5 else "rne")


def test_rows_do_not_depend_on_the_other_groups():
    """The same pairs beside other ones, in a call of the same size: bit for bit."""
    g = torch.Generator().manual_seed(0)
    T, E, K, N = 600, 6, 256, 9000
    x = torch.randn((T, K), generator=g).to(torch.bfloat16).cuda()
    w = torch.randn((E, N, K), generator=g).to(torch.bfloat16).cuda()
    fmt = mxq.Format(K, [4] * 6 + [6, 8])
    wm, we = mxq.pack_experts(w, fmt)
    ids = torch.randint(0, E, (T, 1), generator=g).int()
    other = torch.randint(0, E, (T, 1), generator=g).int()
    other[:50] = ids[:50]
    ys = []
    for i in (ids, other):
        plan = mxq.expert_plan(i.cuda(), E)
        ys.append(mxq.gemm_experts(*mxq.quantize_act_experts(x, fmt, plan), wm, we, fmt, plan, N, dtype=torch.float32))
    assert torch.equal(ys[0][:50], ys[1][:50])
    same = (ids == other)[:, 0].cuda()
    assert torch.equal(ys[0][same], ys[1][same])


# --------------------------------------------------------------------------
# the bits of a layer's results

def test_the_cases_sum_rows_of_32_bits(monkeypatch):
    """A term of a token's sum is not rounded before it is added: the measured calls give the
    one rounding of the result, and the product's and the sum's in float32."""
    import perf.more_operators as cases
    from oracle import fused
    monkeypatch.setattr(cases, "own", True)
    T, E, k, K, N = 40, 6, 3, 256, 200
    s = cases.prepare(cases._product("down", T, E, k, K, N, kind="down", perms="each"), 0)
    got = cases.run(s).double().cpu().numpy()
    ids, w = s["ids"].cpu().numpy(), s["weights"].cpu().numpy()
    act = fused.swiglu_bf16(bits_of(s["gate"]), bits_of(s["up"]))
    y, big = oe.product(act, bits_of(s["w"]), ids, s["perm"].cpu().numpy(), list(s["widths"]))
    tol = (K / 64 + 16) * 2.0 ** -23 * big
    want, sums = oe.combine(y, ids, w, E, s["residual"].float().cpu().numpy())
    # (what the product's error adds to a sum, and a rounding to float32 for each term)
    more, _ = oe.combine(tol, ids, np.abs(w), E)
    more = more + k * 2.0 ** -24 * (sums + more)
    assert np.all(np.abs(got - want) <= more + 2.0 ** -8 * (np.abs(want) + more))

    # a layer's rows on their way into the sum
    seen = []
    combine = mxq.combine_experts
    monkeypatch.setattr(mxq, "combine_experts", lambda y, *a, **kw: (seen.append(y.dtype), combine(y, *a, **kw))[1])
    cases.run(cases.prepare({"kind": "layer", "T": 5, "E": 4, "k": 2, "K": 128, "F": 64, "p6": 0.1, "p8": 0.05,
                             "low": 4}, 0))
    assert seen == [torch.float32]


def test_rows_of_another_number_of_tokens_are_refused():
    """Row counts that divide the pairs; the plan of ids, of a router, written again, or brought with k."""
    fmt = mxq.Format(64, [4, 4])
    x = torch.ones((12, 64), dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros((6, 2), dtype=torch.int32, device="cuda")
    plan = mxq.expert_plan(ids, 4)
    routed = mxq.route(torch.randn((6, 4), device="cuda"), 2)[2]
    brought = mxq.ExpertPlan(12, 4, first=plan.first, pair=plan.pair, k=2)
    for p in (plan, routed, brought):
        for f in (lambda r: mxq.quantize_act_experts(x[:r], fmt, p),
                  lambda r: mxq.quantize_act_swiglu_experts(x[:r], x[:r], fmt, p)):
            for rows in (1, 2, 3, 4):
                with pytest.raises(mxq.MxqError):
                    f(rows)
            f(6), f(12)
    weights = torch.ones((4, 3), device="cuda")
    y = torch.ones((12, 8), device="cuda")
    with pytest.raises(mxq.MxqError):                   # three pairs a token, of a plan of two
        mxq.combine_experts(y, ids.view(4, 3), weights, plan)
    mxq.expert_plan(ids.view(4, 3), 4, out=plan)        # now of three
    mxq.quantize_act_experts(x[:4], fmt, plan)
    mxq.combine_experts(y, ids.view(4, 3), weights, plan)
    with pytest.raises(mxq.MxqError):
        mxq.quantize_act_experts(x[:6], fmt, plan)
    mxq.quantize_act_experts(x[:4], fmt, mxq.ExpertPlan(12, 4, first=plan.first, pair=plan.pair))
    torch.cuda.synchronize()


# --------------------------------------------------------------------------
# SiLU * up of large batches: 16-byte pieces, the table, several row groups to a workgroup

@pytest.mark.parametrize("perms", ["none", "shared", "each"])
@pytest.mark.parametrize("T,E,k,K,skip,round_", [(2001, 64, 6, 1408, 0.1, "rne"), (1001, 32, 4, 1792, 0.0, "rna"),
                                                 (4003, 60, 6, 1408, 0.0, "rne"), (1500, 3, 8, 2048, 0.3, "rne")])
def test_swiglu_images_of_many_groups(T, E, k, K, skip, round_, perms):
    """Workgroups that go from one live group to the next: the table stays, the rows, the expert and its
    permutation are others.  512 workgroups at 256 CUs, and about 700, 530, 1530 and 530 groups with rows."""
    say("swiglu groups", T, E, k, K, skip, perms)
    ids, plan, fmt, each, gate, up = _image_case(T, E, k, K, (4, 6, 8), perms, True, ld=8, skip=skip, round_=round_)
    gate[::7] *= 1000                                    # gates that the table does not hold
    gate[3::11] *= 1e-6
    pair, first = plan.pair.cpu().numpy(), plan.first.cpu().numpy()
    live = pair >= 0
    noise = [torch.randint(0, 256, (n,), dtype=torch.uint8).cuda()
             for n in (fmt.act_bytes(plan.rows), fmt.act_exp_bytes(plan.rows))]
    got = mxq.quantize_act_swiglu_experts(gate, up, fmt, plan, perms=each, out=tuple(t.clone() for t in noise))
    src = torch.from_numpy(np.where(live, pair, 0)).cuda()
    rows, ups = gate[src].contiguous(), up[src].contiguous()
    want = tuple(t.clone() for t in noise)
    tb, sb = fmt.act_bytes(16), fmt.act_exp_bytes(16)
    for e in range(E):
        a, b = int(first[e]), int(first[e + 1])
        f = fmt if each is None else mxq.Format(K, fmt.widths, each[e], round=round_)
        if a < b:
            mxq.quantize_act_swiglu(rows[a:b], ups[a:b], f, out=(want[0][a // 16 * tb:b // 16 * tb],
                                                                 want[1][a // 16 * sb:b // 16 * sb]))
    torch.cuda.synchronize()
    for g, w, z, at in zip(got, want, noise, _byte_rows(list(fmt.widths), plan.rows)):
        g, w, z = g.cpu().numpy(), w.cpu().numpy(), z.cpu().numpy()
        assert np.array_equal(g[live[at]], w[live[at]])
        assert np.array_equal(g[~live[at]], z[~live[at]])


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [False, True])
def test_route_scores_below_float32_and_a_large_scale(score, bias):
    """A weight is good to 1e-6 wherever it is a normal float32, also where its score is not one."""
    x = torch.tensor([[0.0, -40.0, -79.9, -80.1, -87.0, -90.0, -95.5, -103.0, -104.5, -110.25, -120.0, -150.0, -170.0, -400.0],
                      [30.0, 29.0, -50.0, -51.0, -60.0, -70.0, -73.0, -75.0, -80.0, -90.0, -100.0, -110.0, -140.0, -3e38],
                      [-100.0, -101.0, -180.0, -181.0, -186.5, -190.0, -200.0, -210.0, -250.0, -270.0, -280.0, -3e38, -3e38,
                       -3e38]])
    b = torch.zeros(14) if bias else None
    for scale in (1.5, 1e10, 1e25, 3e38, -1e30):
        for normalise in (False, True):
            for k in (2, 14):
                _check_route(x, k, score=score, bias=b, normalise=normalise, scale=scale)


@pytest.mark.parametrize("T,E,K,N", [(50, 4, 512, 200), (7, 3, 1408, 130), (300, 16, 256, 400), (90, 40, 96, 1000)])
@pytest.mark.parametrize("clamp", ["sym", "full"])
def test_rows_of_shared_steps_do_not_depend_on_the_other_groups(T, E, K, N, clamp):
    """The shares of K (groups of a few rows): the same pairs beside other ones, and beside other values, in
    calls of the same size, bit for bit."""
    g = torch.Generator().manual_seed(T)
    x = torch.randn((T, K), generator=g).to(torch.bfloat16).cuda()
    w = torch.randn((E, N, K), generator=g).to(torch.bfloat16).cuda()
    fmt = mxq.Format(K, _widths(K // 32, (4, 6, 8)), clamp=clamp)
    wm, we = mxq.pack_experts(w, fmt)
    ids = torch.randint(0, E, (T, 1), generator=g).int()
    other = torch.randint(-1, E, (T, 1), generator=g).int()
    other[::3] = ids[::3]
    same = (ids == other)[:, 0].cuda()
    z = torch.where(same[:, None], x, torch.randn((T, K), device="cuda").to(torch.bfloat16) * 50)
    ys = []
    for i, v in ((ids, x), (other, x), (other, z)):
        plan = mxq.expert_plan(i.cuda(), E)
        ys.append(mxq.gemm_experts(*mxq.quantize_act_experts(v, fmt, plan), wm, we, fmt, plan, N, dtype=torch.float32))
    assert torch.equal(ys[0][same], ys[1][same]) and torch.equal(ys[0][same], ys[2][same])


# --------------------------------------------------------------------------
# the largest counts: 2^26 pairs

def _check_plan_on_device(ids, E, plan):
    """first and pair against a stable sort on the device."""
    f = ids.flatten().long()
    f = torch.where((f >= 0) & (f < E), f, torch.full_like(f, E))
    count = torch.bincount(f, minlength=E + 1)[:E]
    first = torch.zeros(E + 1, dtype=torch.long, device=f.device)
    first[1:] = torch.cumsum((count + 15) // 16 * 16, 0)
    assert torch.equal(plan.first.long(), first)
    order = torch.argsort(f, stable=True)[:int(count.sum())]
    e = f[order]
    del f
    rank = torch.arange(order.numel(), device=e.device) - (torch.cumsum(count, 0) - count)[e]
    want = torch.full((plan.rows,), -1, dtype=torch.int32, device=e.device)
    want[first[e] + rank] = order.int()
    assert torch.equal(plan.pair, want)


@pytest.mark.parametrize("T,k,E", [(2 ** 26, 1, 1024), (2 ** 23, 8, 60), (2 ** 21, 32, 1000)])
def test_plans_of_the_most_pairs(T, k, E):
    say("plan", T, k, E)
    g = torch.Generator(device="cuda").manual_seed(k)
    ids = torch.randint(-1, E + 1, (T, k), generator=g, device="cuda", dtype=torch.int32)
    plan = mxq.expert_plan(ids, E)
    _check_plan_on_device(ids, E, plan)


@pytest.mark.parametrize("T,k,E", [(2 ** 24, 4, 6), (2 ** 21, 32, 70)])
def test_routing_of_the_most_pairs(T, k, E):
    say("route", T, k, E)
    g = torch.Generator(device="cuda").manual_seed(E)
    x = torch.randn((T, E), generator=g, device="cuda").to(torch.bfloat16)
    ids, w, plan = mxq.route(x, k, score="sigmoid", normalise=False)
    order = torch.sort(x.float(), dim=-1, descending=True, stable=True)[1][:, :k]
    assert torch.equal(ids, order.int())
    s = torch.sigmoid(x.gather(1, order).double())
    assert bool(((w.double() - s).abs() <= 1e-6 * s).all())
    _check_plan_on_device(ids, E, plan)


def test_products_and_sums_of_the_most_pairs():
    """2^26 pairs of 2^25 tokens: an image of 6.4 GB, a row of y for each."""
    T, k, E, K, N = 2 ** 25, 2, 3, 32, 8
    say("product", T, k, E, K, N)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((T, K), generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randn((E, N, K), generator=g, device="cuda").to(torch.bfloat16)
    ids = torch.randint(-1, E, (T, k), generator=g, device="cuda", dtype=torch.int32)
    fmt = mxq.Format(K, [8])
    plan = mxq.expert_plan(ids, E)
    wm, we = mxq.pack_experts(w, fmt)
    y = torch.full((T * k, N), 7.0, device="cuda")
    mxq.gemm_experts(*mxq.quantize_act_experts(x, fmt, plan), wm, we, fmt, plan, N, out=y)
    chosen = ids.flatten() >= 0
    assert bool((y[~chosen] == 7.0).all()) and not bool((y[chosen] == 7.0).all(dim=1).any())
    at = torch.cat([torch.arange(64), torch.randint(0, T * k, (400,), generator=torch.Generator().manual_seed(2)),
                    torch.arange(T * k - 64, T * k)]).cuda()
    f = ids.flatten()[at].cpu().numpy()
    want, big = oe.product(bits_of(x[at // k]), bits_of(w), f, None, [8])
    here = f >= 0
    got = y[at].double().cpu().numpy()
    assert np.all(np.abs(got[here] - want[here]) <= (K / 64 + 16) * 2.0 ** -23 * big[here])
    weights = torch.rand((T, k), generator=g, device="cuda")
    o = mxq.combine_experts(y, ids, weights, plan, residual=torch.ones((T, N), dtype=torch.bfloat16, device="cuda"),
                            dtype=torch.float32)
    terms = torch.where(chosen[:, None], weights.flatten()[:, None] * y, torch.zeros((), device="cuda")).view(T, k, N)
    # (a rounding for each of three sums and the products')
    assert bool(((o - (1 + terms.sum(1))).abs() <= 5 * 2.0 ** -24 * (1 + terms.abs().sum(1))).all())
