"""Rotary positions (mxq_rope, mxq_rope_table) against the oracle.

The rotation is defined operation by operation in float32, so its bf16 results
are compared bit for bit.  The table's entries are float64 cosines and sines
rounded to float32: half a step is eps / 2 of the value, and a cosine whose
angle is off by 2^-53 of itself (positions below 2^20, frequencies at most 1) by
2^-33, so |c - c_ref| <= 2^-24 |c_ref| + 2^-32.
"""
import numpy as np
import pytest
import torch

from oracle import paged as opaged
from paper_2607_17733_amd import mxq
from parity_util import say

pytestmark = pytest.mark.gpu


def bits_of(t):
    return t.cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


def _same(a, b):
    """bf16 bits, any NaN equal to any other."""
    na, nb = np.isnan(opaged.to_f32(a)), np.isnan(opaged.to_f32(b))
    return np.array_equal(na, nb) and np.array_equal(a[~na], b[~nb])


def _run(T, H, D, rot, interleaved, P=700, view=None, inplace=False, seed=0):
    say("rope", T, H, D, rot, interleaved, view, inplace)
    g = torch.Generator().manual_seed(seed + T + 7 * H + D + rot)
    x = torch.randn((T, H + 3, D + 8), generator=g).to(torch.bfloat16).cuda()
    x = {None: lambda: x[:, :H, :D].contiguous(), "fused": lambda: x[:, 1:H + 1, :D],
         "heads": lambda: x[:, :H, :D].transpose(0, 1).contiguous().transpose(0, 1),
         "odd": lambda: x[:, :H, 2:D + 2]}[view]()
    pos = torch.randint(0, P, (T,), generator=g).int().cuda()
    f, ms = mxq.rope_inv_freq(rot)
    table = mxq.rope_table(f, P, ms)
    want = opaged.rope(bits_of(x), pos.cpu().numpy(), table.cpu().numpy(), interleaved)
    y = mxq.rope(x, pos, table, interleaved, out=x if inplace else None)
    torch.cuda.synchronize()
    assert _same(bits_of(y), want)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,D,rot", [(1, 1, 128, 128), (1, 64, 128, 128), (17, 5, 128, 64),
                                       (33, 3, 128, 96), (5, 2, 64, 64), (3, 7, 256, 256),
                                       (4, 3, 80, 20), (2, 2, 66, 66), (3, 1, 2, 2),
                                       (2, 3, 130, 32), (301, 2, 128, 32), (2, 1, 512, 512)])
def test_rotation_bit_for_bit(T, H, D, rot, interleaved):
    _run(T, H, D, rot, interleaved)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("view", ["fused", "heads", "odd"])
@pytest.mark.parametrize("inplace", [False, True])
def test_strided_rows_and_in_place(view, inplace, interleaved):
    _run(19, 4, 128, 64, interleaved, view=view, inplace=inplace)


def test_in_place_leaves_the_neighbours():
    g = torch.Generator().manual_seed(4)
    rows = torch.randn((9, 6, 128), generator=g).to(torch.bfloat16).cuda()
    before = rows.clone()
    pos = torch.arange(9, dtype=torch.int32, device="cuda")
    table = mxq.rope_table(mxq.rope_inv_freq(128)[0], 16)
    mxq.rope(rows[:, 2:4], pos, table, out=rows[:, 2:4])
    torch.cuda.synchronize()
    assert torch.equal(rows[:, :2], before[:, :2]) and torch.equal(rows[:, 4:], before[:, 4:])
    assert torch.equal(rows[0, 2:4], before[0, 2:4])           # position 0 turns by nothing
    assert not torch.equal(rows[1:, 2:4], before[1:, 2:4])


def test_special_values_and_positions_outside_the_table():
    x = torch.zeros((6, 1, 32), dtype=torch.bfloat16)
    x[0, 0, 3], x[1, 0, 4], x[2, 0, 20] = float("inf"), float("nan"), float("-inf")
    x[5] = 3.0
    pos = torch.tensor([3, 2, 9, -1, 10, 2 ** 31 - 1], dtype=torch.int32)
    table = mxq.rope_table(mxq.rope_inv_freq(16)[0], 10)
    for interleaved in (False, True):
        y = mxq.rope(x.cuda(), pos.cuda(), table, interleaved)
        torch.cuda.synchronize()
        want = opaged.rope(bits_of(x), pos.numpy(), table.cpu().numpy(), interleaved)
        assert _same(bits_of(y), want)
        assert y[3:, :, :16].isnan().all() and torch.equal(y[3:, :, 16:].cpu(), x[3:, :, 16:])


@pytest.mark.parametrize("scaling,kw", [(None, {}), ("linear", dict(factor=8.0)),
                                        ("base", dict(factor=4.0)),
                                        ("ramp", dict(factor=16.0, orig_positions=4096)),
                                        ("bands", dict(factor=8.0, orig_positions=8192, low=1.0,
                                                       high=4.0))])
def test_table_of_far_positions(scaling, kw):
    P = 200001
    f, ms = mxq.rope_inv_freq(128, base=500000.0, scaling=scaling, **kw)
    table = mxq.rope_table(f, P, ms).cpu().double().numpy()
    for p in (0, 1, 77, 4095, 131071, P - 1):
        a = np.float64(p) * f
        for k, want in ((0, ms * np.cos(a)), (1, ms * np.sin(a))):
            assert np.all(np.abs(table[p, :, k] - want) <= 2.0 ** -24 * np.abs(want) + 2.0 ** -32)


def test_rotation_keeps_products_of_equal_distance():
    # q . k depends on the distance of the positions alone: the float32 rotation
    # and the bf16 rounding of both rows bound the difference by
    # 4 * 2^-8 * |q| |k| (half a bf16 step each, on both sides of the comparison)
    g = torch.Generator().manual_seed(9)
    q, k = (torch.randn((1, 1, 128), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    table = mxq.rope_table(mxq.rope_inv_freq(128)[0], 3000)

    def at(x, p):
        return mxq.rope(x, torch.tensor([p], dtype=torch.int32, device="cuda"), table).double()

    bound = 4 * 2.0 ** -8 * float(q.double().norm() * k.double().norm())
    first = float((at(q, 40) * at(k, 7)).sum())
    for shift in (1, 500, 2900):
        assert abs(float((at(q, 40 + shift) * at(k, 7 + shift)).sum()) - first) <= bound


def test_no_rows_and_another_stream():
    table = mxq.rope_table(mxq.rope_inv_freq(128)[0], 64)
    x = torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda")
    assert mxq.rope(x, torch.empty(0, dtype=torch.int32, device="cuda"), table).shape == (0, 4, 128)
    x = torch.randn((40, 4, 128), device="cuda").to(torch.bfloat16)
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    want = mxq.rope(x, pos, table)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = mxq.rope(x, pos, table)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rows_past_four_billion_elements(interleaved):
    # 70001 tokens of 512 heads of 128 values: 4.6e9 elements, in place; sampled rows against the oracle
    T, H, D, rot = 70001, 512, 128, 64
    x = torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 2 ** 32
    small = torch.randn((1001, H, D), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    for t in range(0, T, 1001):
        n = min(1001, T - t)
        x[t:t + n] = small[:n]
    pos = torch.randint(0, 700, (T,), generator=torch.Generator().manual_seed(3)).int()
    table = mxq.rope_table(mxq.rope_inv_freq(rot)[0], 700)
    at = [0, 1, 32767, 32768, 65535, 65536, 65537, T - 1]          # (2^31 elements are 32768 tokens)
    before = bits_of(x[at])
    say("rope of 9 GB", interleaved)
    y = mxq.rope(x, pos.cuda(), table, interleaved, out=x)
    torch.cuda.synchronize()
    assert y is x
    assert _same(bits_of(x[at]), opaged.rope(before, pos.numpy()[at], table.cpu().numpy(), interleaved))
