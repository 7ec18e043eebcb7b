"""Layers with experts, and norms of queries and keys, on the CPU: the C ABI's status
for every refused argument (nothing is launched: each call fails its checks), the
binding's checks, and pins of the oracle."""
import ctypes
import math
import types

import numpy as np
import pytest
import torch

import oracle
from oracle import experts as oe
from oracle.paged import to_bf16
from paper_2607_17733_amd import mxq

NULL, SHAPE, WIDTHS, ALIGN, UNSUPPORTED = 1, 2, 3, 5, 6
FAKE = 1 << 20                                     # aligned, never dereferenced


@pytest.fixture(scope="module")
def L():
    return mxq.lib()


def ref(x):
    return None if x is None else ctypes.byref(x)


def plan(**kw):
    c = dict(pairs=12, experts=4, reserved=0, first=FAKE, pair=FAKE, work=FAKE)
    c.update(kw)
    return mxq._Experts(*[c[n] for n, _ in mxq._Experts._fields_])


def opts(**kw):
    c = dict(k=3, score=0, normalise=1, scale=1.0, bias=None)
    c.update(kw)
    return mxq._RouteOpts(*[c[n] for n, _ in mxq._RouteOpts._fields_])


BAD_PLANS = [(dict(pairs=-1), SHAPE), (dict(pairs=2 ** 26 + 4), SHAPE), (dict(experts=0), SHAPE),
             (dict(experts=-3), SHAPE), (dict(experts=1025), SHAPE), (dict(reserved=1), UNSUPPORTED),
             (dict(first=0), NULL), (dict(pair=0), NULL), (dict(first=FAKE + 8), ALIGN),
             (dict(pair=FAKE + 4), ALIGN)]
BAD_WORK = [(dict(work=0), NULL), (dict(work=FAKE + 8), ALIGN)]        # of the calls that write a plan


def test_rows(L):
    for pairs in (0, 1, 2, 15, 16, 17, 100, 512, 2 ** 26):
        for E in (1, 2, 7, 128, 1024):
            rows = L.mxq_expert_rows(pairs, E)
            assert rows == oe.rows_of(pairs, E) and rows % 16 == 0
    # as many as the worst choice needs: one pair with each of 128 experts, the rest with one
    ids = np.concatenate([np.arange(127), np.full(385, 127)])
    assert oe.plan(ids, 128)[0][-1] <= L.mxq_expert_rows(512, 128) == 2432
    assert L.mxq_expert_rows(-1, 4) == -SHAPE and L.mxq_expert_rows(2 ** 26 + 1, 4) == -SHAPE
    assert L.mxq_expert_rows(4, 0) == -SHAPE and L.mxq_expert_rows(4, 1025) == -SHAPE


def test_route_refusals(L):
    def call(o=None, p=None, logits=FAKE, f32=1, T=4, ld=4, ids=FAKE, w=FAKE, none=False):
        return L.mxq_route(None if none else ref(o or opts()), logits, f32, T, ld, ids, w, ref(p or plan()), None)

    for kw, want in ([(dict(p=plan(**k)), w) for k, w in BAD_PLANS + BAD_WORK] +
                     [(dict(none=True), NULL), (dict(logits=0), NULL), (dict(ids=0), NULL), (dict(w=0), NULL),
                      (dict(o=opts(k=0), p=plan(pairs=0)), SHAPE), (dict(o=opts(k=5), p=plan(pairs=20)), SHAPE),
                      (dict(o=opts(k=33), p=plan(pairs=132, experts=100), ld=100), SHAPE),
                      (dict(o=opts(score=2)), UNSUPPORTED), (dict(o=opts(score=-1)), UNSUPPORTED),
                      (dict(o=opts(scale=math.inf)), SHAPE), (dict(o=opts(scale=math.nan)), SHAPE),
                      (dict(T=-1), SHAPE), (dict(T=5), SHAPE), (dict(T=2 ** 62), SHAPE), (dict(ld=3), SHAPE),
                      (dict(logits=FAKE + 2), ALIGN), (dict(logits=FAKE + 1, f32=0), ALIGN),
                      (dict(ids=FAKE + 4), ALIGN), (dict(w=FAKE + 8), ALIGN), (dict(o=opts(bias=FAKE + 2)), ALIGN)]):
        assert call(**kw) == want, kw
    assert L.mxq_route(ref(opts()), FAKE, 1, 4, 4, FAKE, FAKE, None, None) == NULL


def test_plan_refusals(L):
    for k, want in BAD_PLANS + BAD_WORK:
        assert L.mxq_expert_plan(FAKE, ref(plan(**k)), None) == want, k
    assert L.mxq_expert_plan(FAKE, None, None) == NULL
    assert L.mxq_expert_plan(0, ref(plan()), None) == NULL
    assert L.mxq_expert_plan(FAKE + 4, ref(plan()), None) == ALIGN


def test_quantize_refusals(L):
    f = mxq.Format(128, [4, 4, 6, 8])
    odd = mxq.Format(128, [4, 4, 6, 8])
    odd.widths[0] = 5

    def call(f=f, p=None, perms=None, a=FAKE, per=3, ld=128, mant=FAKE, exp=FAKE, up=None):
        if up is not None:
            return L.mxq_quantize_act_swiglu_experts(f.ref, ref(p or plan()), perms, a, up, per, ld, mant, exp, None)
        return L.mxq_quantize_act_experts(f.ref, ref(p or plan()), perms, a, per, ld, mant, exp, None)

    for up in (None, FAKE):
        for kw, want in ([(dict(p=plan(**k)), w) for k, w in BAD_PLANS] +
                         [(dict(f=odd), WIDTHS), (dict(a=0), NULL), (dict(mant=0), NULL), (dict(exp=0), NULL),
                          (dict(per=0), SHAPE), (dict(per=-1), SHAPE), (dict(per=5), SHAPE), (dict(per=2 ** 40), SHAPE),
                          (dict(ld=127), SHAPE), (dict(a=FAKE + 8), ALIGN), (dict(mant=FAKE + 4), ALIGN),
                          (dict(exp=FAKE + 1), ALIGN), (dict(perms=FAKE + 4), ALIGN)]):
            assert call(up=up, **kw) == want, (up, kw)
    assert call(up=0) == NULL and call(up=FAKE + 8) == ALIGN
    assert call(p=plan(pairs=0, pair=0), a=0, mant=0, exp=0, per=1) == 0
    # a row too long for a workgroup's LDS
    long = mxq.Format(81920, [4] * 2560)
    assert call(f=long, ld=81920) == UNSUPPORTED


def test_product_refusals(L):
    f = mxq.Format(128, [4, 4, 6, 8])

    def call(p=None, N=40, am=FAKE, ae=FAKE, wm=FAKE, we=FAKE, y=FAKE, f32=0, ldy=40):
        return L.mxq_gemm_experts(f.ref, ref(p or plan()), N, am, ae, wm, we, y, f32, ldy, None)

    for kw, want in ([(dict(p=plan(**k)), w) for k, w in BAD_PLANS] +
                     [(dict(N=-1), SHAPE), (dict(ldy=39), SHAPE), (dict(N=2 ** 31, ldy=2 ** 31), SHAPE)] +
                     [(dict([(n, 0)]), NULL) for n in ("am", "ae", "wm", "we", "y")] +
                     [(dict([(n, FAKE + 8)]), ALIGN) for n in ("am", "ae", "wm", "we", "y")]):
        assert call(**kw) == want, kw
    assert L.mxq_gemm_experts(f.ref, None, 40, FAKE, FAKE, FAKE, FAKE, FAKE, 0, 40, None) == NULL
    assert call(N=0) == 0 and call(p=plan(pairs=0, pair=0), am=0) == 0
    # more tiles than a dispatch holds
    assert call(p=plan(pairs=2 ** 26, experts=1024), N=2 ** 31 - 1, ldy=2 ** 31) == SHAPE


def test_combine_refusals(L):
    def call(y=FAKE, f32=0, ldy=40, ids=FAKE, w=FAKE, T=4, k=3, E=4, N=40, res=FAKE, ldr=40, out=FAKE + 4096, of32=0,
             ldo=40):
        return L.mxq_combine_experts(y, f32, ldy, ids, w, T, k, E, N, res, ldr, out, of32, ldo, None)

    for kw, want in ([(dict([(n, 0)]), NULL) for n in ("y", "ids", "w", "out")] +
                     [(dict([(n, -1)]), SHAPE) for n in ("T", "N", "k", "E")] +
                     [(dict(k=0), SHAPE), (dict(E=0), SHAPE), (dict(ldy=39), SHAPE), (dict(ldr=39), SHAPE),
                      (dict(ldo=39), SHAPE), (dict(T=2 ** 26, k=2), SHAPE), (dict(T=2 ** 62, k=4), SHAPE),
                      (dict(T=2 ** 20, k=1, N=2 ** 31, ldy=2 ** 31, ldr=2 ** 31, ldo=2 ** 31), SHAPE),
                      (dict(y=FAKE + 1), ALIGN), (dict(y=FAKE + 2, f32=1), ALIGN), (dict(out=FAKE + 1), ALIGN),
                      (dict(out=FAKE + 2, of32=1), ALIGN), (dict(ids=FAKE + 2), ALIGN), (dict(w=FAKE + 2), ALIGN),
                      (dict(res=FAKE + 1), ALIGN),
                      # in place: the same type, the same rows
                      (dict(res=FAKE + 4096, ldr=48), SHAPE), (dict(res=FAKE + 4096, of32=1), SHAPE)]):
        assert call(**kw) == want, kw
    assert call(T=0, y=0) == 0 and call(N=0, y=0) == 0


def rotary(**kw):
    c = dict(table=FAKE, positions=100, rot=64, layout=0)
    c.update(kw)
    return mxq._Rotary(*[c[n] for n, _ in mxq._Rotary._fields_])


def norm(q=FAKE, k=FAKE, eps=1e-6):
    return mxq._QkNorm(q, k, eps)


def test_rope_qk_refusals(L):
    def call(r=None, n=None, pos=FAKE, T=4, D=128, q=FAKE, Hq=2, qs=(512, 128), qo=FAKE + 65536, qos=(256, 128),
             k=FAKE + 512, Hk=1, ks=(512, 128), ko=FAKE + 131072, kos=(128, 128), none=()):
        return L.mxq_rope_qk(None if "r" in none else ref(r or rotary()), None if "n" in none else ref(n or norm()), pos,
                             T, D, q, Hq, *qs, qo, *qos, k, Hk, *ks, ko, *kos, None)

    for kw, want in ((dict(none="r"), NULL), (dict(none="n"), NULL), (dict(r=rotary(table=0)), NULL), (dict(q=0), NULL),
                     (dict(qo=0), NULL), (dict(k=0), NULL), (dict(ko=0), NULL), (dict(pos=0), NULL),
                     (dict(n=norm(q=0)), NULL), (dict(n=norm(k=0)), NULL), (dict(n=norm(eps=-1.0)), SHAPE),
                     (dict(n=norm(eps=math.nan)), SHAPE), (dict(n=norm(eps=math.inf)), SHAPE),
                     (dict(n=norm(q=FAKE + 8)), ALIGN), (dict(r=rotary(rot=63)), SHAPE),
                     (dict(r=rotary(layout=2)), UNSUPPORTED), (dict(T=-1), SHAPE), (dict(Hq=-1), SHAPE),
                     (dict(Hk=65536), SHAPE), (dict(D=62), SHAPE), (dict(D=129), SHAPE), (dict(D=4098), SHAPE),
                     (dict(T=2 ** 31), SHAPE), (dict(T=2 ** 30, Hq=60), SHAPE), (dict(q=FAKE + 2), ALIGN),
                     (dict(ko=FAKE + 131074), ALIGN), (dict(qs=(511, 128)), ALIGN), (dict(kos=(128, 129)), ALIGN),
                     (dict(qo=FAKE), SHAPE), (dict(qos=(128, 128)), SHAPE), (dict(kos=(64, 128)), SHAPE)):
        assert call(**kw) == want, kw
    assert call(T=0, q=0, k=0, pos=0) == 0 and call(Hq=0, Hk=0, q=0, k=0) == 0


def test_append_norm_refusals(L):
    f = mxq.Format(128, [4, 4, 6, 8])
    c = mxq._PagedKv(4, 2, 16, 0, FAKE, FAKE, FAKE, FAKE)

    def call(n=norm(), r=rotary(), q=FAKE, qo=FAKE + 65536, slots=FAKE):
        return L.mxq_kv_append_norm(f.ref, ref(c), ref(n), FAKE, 256, 128, FAKE, 256, 128, 4, slots, FAKE, ref(r), q, 4,
                                    512, 128, qo, None)

    for kw, want in ((dict(n=None), NULL), (dict(r=None), NULL), (dict(n=norm(k=0)), NULL), (dict(n=norm(q=0)), NULL),
                     (dict(n=norm(eps=-1.0)), SHAPE), (dict(n=norm(k=FAKE + 8)), ALIGN), (dict(slots=0), NULL),
                     (dict(r=rotary(rot=24)), SHAPE), (dict(qo=0), NULL)):
        assert call(**kw) == want, kw


def test_binding_refuses_host_tensors():
    x, ids = torch.zeros((4, 8)), torch.zeros((4, 2), dtype=torch.int32)
    for f in (lambda: mxq.route(x, 2), lambda: mxq.expert_plan(ids, 4), lambda: mxq.ExpertPlan(8, 4, device="cpu"),
              lambda: mxq.ExpertPlan(8, 4, first=ids), lambda: mxq.ExpertPlan(-8, 4), lambda: mxq.ExpertPlan(8, 0),
              lambda: mxq.pack_experts(torch.zeros((2, 4, 32)), mxq.Format(32, [4])),
              lambda: mxq.rope_qk(None, None, ids, x, x, x, 1e-6),
              lambda: mxq.rope_qk(torch.zeros((4, 2, 8)), None, ids, x, x, x, 1e-6)):
        with pytest.raises(mxq.MxqError):
            f()


# --------------------------------------------------------------------------
# pins of the oracle

def test_oracle_route_against_torch():
    g = torch.Generator().manual_seed(0)
    x = torch.randn((50, 33), generator=g)
    ids, w = oe.route(x.numpy(), 5)
    p, at = torch.softmax(x.double(), -1).topk(5)
    assert np.array_equal(ids, at.numpy()) and np.allclose(w, (p / p.sum(-1, keepdim=True)).numpy(), rtol=1e-12)
    ids, w = oe.route(x.numpy(), 5, "sigmoid", False, 2.0)
    assert np.array_equal(ids, at.numpy())
    assert np.allclose(w, 2 * torch.sigmoid(x.double()).gather(1, at).numpy(), rtol=1e-12)
    ids, w = oe.route(np.array([[1.0, 1.0, -np.inf, np.nan]], np.float32), 3)
    assert ids.tolist() == [[0, 1, -1]] and w.tolist() == [[0.5, 0.5, 0.0]]


def test_oracle_plan_by_hand():
    first, pair = oe.plan(np.array([[2, 0], [2, -1], [0, 2]]), 4)
    assert first.tolist() == [0, 16, 16, 32, 32]
    want = np.full(64, -1)                         # 6 + 15 * 4 rows, in sixteens
    want[[0, 1, 16, 17, 18]] = [1, 4, 0, 2, 5]
    assert pair.tolist() == want.tolist()


def test_oracle_product_is_the_linear_of_each_expert():
    g = np.random.RandomState(0)
    widths = [4, 4, 6, 8]
    x, w = to_bf16(g.randn(7, 128).astype(np.float32)), to_bf16(g.randn(3, 9, 128).astype(np.float32))
    ids = np.array([0, 2, 2, -1, 0, 5, 1])
    y, _ = oe.product(x, w, ids, None, widths)
    for p, e in enumerate(ids):
        if 0 <= e < 3:
            qa, ea = oracle.quantize(x[p:p + 1], widths=widths)
            qw, ew = oracle.quantize(w[e], widths=widths)
            assert np.allclose(y[p], oracle.gemm(qa, ea, qw, ew, widths)[0], rtol=1e-12, atol=1e-12)
        else:
            assert np.isnan(y[p]).all()


def test_oracle_norm_has_unit_mean_square_and_keeps_lengths():
    g = np.random.RandomState(1)
    x = to_bf16(g.randn(5, 3, 64).astype(np.float32))
    table = np.stack([np.cos(np.arange(40.0)), np.sin(np.arange(40.0))], -1).reshape(1, 40, 2)[:, :32].repeat(6, 0)
    one = to_bf16(np.ones(64, np.float32))
    y, _ = oe.norm_rope(x, np.arange(5), table, one, 0.0, True)
    assert np.allclose((y * y).mean(-1), 1.0, rtol=1e-12)
    z, _ = oe.norm_rope(x, np.arange(5), table * 0 + [1.0, 0.0], one, 0.0, False)
    assert np.allclose((z * z).mean(-1), 1.0, rtol=1e-12)
    assert not oe.norm_rope(np.zeros((1, 1, 64), np.uint16), [0], table, one, 0.0, False)[0].any()


def test_source_rows_are_those_of_the_tokens_or_of_the_pairs():
    """Rows that divide the pairs but are not the tokens would be other tokens' rows."""
    plan = types.SimpleNamespace(pairs=12, experts=4, k=2, device="here")
    assert mxq._per_row(6, plan, "x", "here") == 2 and mxq._per_row(12, plan, "x", "here") == 1
    for rows in (0, 1, 2, 3, 4, 5, 7, 24):
        with pytest.raises(mxq.MxqError):
            mxq._per_row(rows, plan, "x", "here")
    plan.k = None                                      # of a plan that came without it: as many as divide
    assert mxq._per_row(6, plan, "x", "here") == 2 and mxq._per_row(4, plan, "x", "here") == 3
    with pytest.raises(mxq.MxqError):
        mxq._per_row(5, plan, "x", "here")
    none = types.SimpleNamespace(pairs=0, experts=4, k=2, device="here")
    assert mxq._per_row(0, none, "x", "here") == 1
    with pytest.raises(mxq.MxqError):
        mxq._per_row(5, none, "x", "here")
    for k in (0, -1, 5):
        with pytest.raises(mxq.MxqError):
            mxq.ExpertPlan(12, 4, k=k)


def test_images_of_more_threads_than_a_dispatch_holds(L):
    """Long rows of as many pairs as a plan allows: a group of rows to a workgroup, 2^32 threads and more."""
    for blocks, pairs in ((640, 2 ** 23), (640, 2 ** 26), (128, 2 ** 26)):
        f = mxq.Format(32 * blocks, [4] * blocks)
        p = plan(pairs=pairs)
        assert L.mxq_quantize_act_experts(f.ref, ref(p), None, FAKE, 2, 32 * blocks, FAKE, FAKE, None) == SHAPE
