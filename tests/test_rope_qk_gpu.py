"""Norms of queries and keys with the rotation in the same pass, alone and on the way
into the cache.

Bounds, in units of 2^-24: the squares' sum rounds at most 7 times in a lane (D / 64 beyond
D = 512) and 6 times over the lanes, the mean and eps twice, which the root halves, and the
root's own unit counts two: 12 for the factor (40 up to D = 4096).  The normalised value x
r takes one rounding, the gain another, a rotation's products and their sum three more: 18
(46) of what the terms add up to; the result is off by half a bf16 step, 2^-8, more
(subnormal results by half of 2^-133).
"""
import numpy as np
import pytest
import torch

from oracle import experts as oe
from paper_2607_17733_amd import mxq
from parity_util import say

pytestmark = pytest.mark.gpu


def bits_of(t):
    return t.cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


def _check(y, x, pos, table, gain, eps, interleaved):
    want, big = oe.norm_rope(bits_of(x), pos.cpu().numpy(), table.cpu().numpy(), bits_of(gain), eps, interleaved)
    got = y.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    tol = (18 if x.shape[2] <= 512 else 46) * 2.0 ** -24 * big
    tol = tol + 2.0 ** -8 * (np.abs(want) + tol) + 2.0 ** -134
    d = np.abs(got - want)
    assert np.all(d[ok] <= tol[ok]), float((d[ok] - tol[ok]).max())


def _inputs(T, Hq, Hk, D, rot, P=500, view=None, seed=0):
    g = torch.Generator().manual_seed(seed + T + 7 * Hq + D + rot)
    rows = (2 * torch.randn((T, Hq + Hk + 2, D + 8), generator=g)).to(torch.bfloat16).cuda()
    q, k = rows[:, :Hq], rows[:, Hq:Hq + Hk]
    cut = {None: lambda x: x[..., :D].contiguous(), "fused": lambda x: x[..., :D], "odd": lambda x: x[..., 2:D + 2],
           "heads": lambda x: x[..., :D].transpose(0, 1).contiguous().transpose(0, 1)}[view]
    gains = [(1 + 0.3 * torch.randn((D,), generator=g)).to(torch.bfloat16).cuda() for _ in range(2)]
    pos = torch.randint(0, P, (T,), generator=g).int().cuda()
    table = mxq.rope_table(mxq.rope_inv_freq(rot)[0], P)
    return cut(q), cut(k), gains, pos, table


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,Hq,Hk,D,rot", [(1, 1, 1, 128, 128), (1, 32, 8, 128, 128), (17, 5, 1, 128, 64),
                                           (33, 4, 2, 64, 64), (3, 6, 3, 256, 256), (5, 2, 2, 80, 80),
                                           (5, 2, 2, 80, 20), (4, 3, 1, 96, 96), (2, 2, 2, 66, 66), (3, 1, 1, 2, 2),
                                           (2, 1, 1, 512, 512), (2, 2, 1, 520, 64), (1, 1, 1, 4096, 256),
                                           (301, 3, 2, 128, 32), (7, 3, 0, 128, 128), (7, 0, 3, 128, 128),
                                           (9, 1, 1, 8, 8), (9, 2, 1, 16, 16)])
def test_rope_qk(T, Hq, Hk, D, rot, interleaved):
    say("rope_qk", T, Hq, Hk, D, rot, interleaved)
    q, k, gains, pos, table = _inputs(T, Hq, Hk, D, rot)
    q, k = q if Hq else None, k if Hk else None
    yq, yk = mxq.rope_qk(q, k, pos, table, gains[0], gains[1], 1e-6, interleaved)
    for y, x, g in ((yq, q, gains[0]), (yk, k, gains[1])):
        if x is None:
            assert y is None
        else:
            _check(y, x, pos, table, g, 1e-6, interleaved)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("view", ["fused", "odd", "heads"])
@pytest.mark.parametrize("inplace", [False, True])
def test_strided_rows_and_in_place(view, inplace, interleaved):
    q, k, gains, pos, table = _inputs(19, 4, 2, 128, 64, view=view)
    q0, k0 = q.clone(), k.clone()
    yq, yk = mxq.rope_qk(q, k, pos, table, *gains, 1e-5, interleaved, q_out=q if inplace else None,
                         k_out=k if inplace else None)
    _check(yq, q0, pos, table, gains[0], 1e-5, interleaved)
    _check(yk, k0, pos, table, gains[1], 1e-5, interleaved)


@pytest.mark.parametrize("D", [128, 66])
def test_extreme_rows(D):
    """Rows of zeros, tiny, huge and subnormal values; positions without an angle; infinities and NaN."""
    x = torch.ones((9, 1, D), dtype=torch.bfloat16)
    x[:, :, ::3] = -2.0
    for i, f in enumerate((0.0, 1e-30, 1e-39, 1e38, 1.0, 1.0, 1.0)):
        x[i] = (x[i].double() * f).to(torch.bfloat16)
    x[7, 0, 5], x[8, 0, 1] = float("nan"), float("inf")
    pos = torch.tensor([0, 1, 2, 3, -1, 100, 99, 4, 5], dtype=torch.int32).cuda()
    gain = torch.ones(D, dtype=torch.bfloat16).cuda()
    table = mxq.rope_table(mxq.rope_inv_freq(D)[0], 100)
    for eps in (0.0, 1e-6):
        yq, yk = mxq.rope_qk(x.cuda(), x.cuda(), pos, table, gain, gain, eps)
        assert torch.equal(yq.view(torch.int16), yk.view(torch.int16))
        with np.errstate(all="ignore"):
            _check(yq[:7], x[:7].cuda(), pos[:7], table, gain, eps, False)
        assert bool(yq[7].isnan().all())                 # its mean is a NaN
        assert bool(yq[8].isnan().any())                 # Inf / Inf; the others are zeros or turn with it


@pytest.mark.parametrize("widths,rot,interleaved", [((4, 4, 4, 4), 128, False), ((4, 4, 6, 8), 64, True),
                                                    ((3, 3, 6, 8), 32, False), ((8, 8, 8, 8), 128, True)])
@pytest.mark.parametrize("T", [1, 15, 16, 70])
@pytest.mark.parametrize("with_q", [True, False])
def test_append_is_rope_qk_then_append(T, widths, rot, interleaved, with_q):
    """Bit for bit, from strided rows, with padding slots."""
    q, k, gains, pos, table = _inputs(T, 5, 2, 128, rot, view="fused")
    v = torch.randn((T, 2, 128)).to(torch.bfloat16).cuda()
    pages = T // 16 + 3
    slots = torch.randperm(pages * 16)[:T].cuda()
    slots[T // 2] = -1
    caches = [mxq.PagedCache(mxq.Format(128, list(widths)), 2, pages, 16) for _ in range(2)]
    q1 = mxq.kv_append(caches[0], k, v, slots, pos=pos, rope=table, interleaved=interleaved, k_gain=gains[1],
                       q=q if with_q else None, q_gain=gains[0] if with_q else None, eps=1e-6)
    q2, k2 = mxq.rope_qk(q, k, pos, table, *gains, 1e-6, interleaved)
    mxq.kv_append(caches[1], k2, v, slots)
    for a, b in zip(caches[0].k + caches[0].v, caches[1].k + caches[1].v):
        assert torch.equal(a, b)
    assert torch.equal(q1, q2) if with_q else q1 is None


def test_both_paths_of_rope_qk_agree():
    """Rows that the 16-byte accesses can and cannot take give the same bits."""
    q, k, gains, pos, table = _inputs(11, 3, 2, 128, 64)
    wide = torch.zeros((11, 3, 130), dtype=torch.bfloat16, device="cuda")
    wide[..., 2:] = q
    for interleaved in (False, True):
        a = mxq.rope_qk(q, None, pos, table, gains[0], None, 1e-6, interleaved)[0]
        b = mxq.rope_qk(wide[..., 2:], None, pos, table, gains[0], None, 1e-6, interleaved)[0]
        assert torch.equal(a, b)


def test_captured_and_replayed_in_place():
    q, k, gains, pos, table = _inputs(20, 4, 2, 128, 128)
    q0, k0 = q.clone(), k.clone()
    want = mxq.rope_qk(q, k, pos, table, *gains, 1e-6)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mxq.rope_qk(q, k, pos, table, *gains, 1e-6, q_out=qo, k_out=ko)
    for _ in range(3):
        qo.zero_()
        ko.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
    assert torch.equal(q, q0) and torch.equal(k, k0)


@pytest.mark.parametrize("D,rot,interleaved", [(128, 128, False), (128, 64, True), (66, 66, False)])
def test_captured_with_the_results_in_place_of_other_inputs(D, rot, interleaved):
    """One capture that overwrites q and k, replayed on other values (and positions), between eager calls."""
    q, k, gains, pos, table = _inputs(20, 4, 2, D, rot)
    mxq.rope_qk(q.clone(), k.clone(), pos, table, *gains, 1e-6, interleaved)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mxq.rope_qk(q, k, pos, table, *gains, 1e-6, interleaved, q_out=q, k_out=k)
    for seed in range(1, 5):
        q1, k1, _, pos1, _ = _inputs(20, 4, 2, D, rot, seed=seed)
        want = mxq.rope_qk(q1, k1, pos1, table, *gains, 1e-6, interleaved)
        q.copy_(q1)
        k.copy_(k1)
        pos.copy_(pos1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q, want[0]) and torch.equal(k, want[1])
        _check(q, q1, pos1, table, gains[0], 1e-6, interleaved)


@pytest.mark.parametrize("D", [128, 66])
def test_the_largest_eps(D):
    """The mean and eps add up beyond float32's largest."""
    x = torch.full((3, 1, D), 2.0 ** 56, dtype=torch.bfloat16)
    x[1] *= 2.0 ** -40
    x[2] *= 2.0 ** 4
    x[:, :, ::3] *= -1.5
    pos = torch.tensor([0, 7, 99], dtype=torch.int32).cuda()
    gain = torch.full((D,), 1.5, dtype=torch.bfloat16).cuda()
    table = mxq.rope_table(mxq.rope_inv_freq(D)[0], 100)
    for eps in (float(np.finfo(np.float32).max), 2.0 ** 127, 2.0 ** 100):
        y, _ = mxq.rope_qk(x.cuda(), None, pos, table, gain, None, eps)
        _check(y, x.cuda(), pos, table, gain, eps, False)
