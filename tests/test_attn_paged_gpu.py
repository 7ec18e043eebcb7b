"""Attention over the paged MXINT cache (mxq_attn_paged) against the float64
oracle; the bounds are derived in paged_util.  Every cache is noise outside the
appended rows, E = 255 with mantissas among it, so that a place behind a
sequence's last token, or another sequence's page, shows at once."""
import numpy as np
import pytest
import torch

from paged_util import D, Batch
from paper_2607_17733_amd import mxq
from parity_util import say

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16]
MIXES = [(n4, n6, 4 - n4 - n6) for n4 in range(4, -1, -1) for n6 in range(4 - n4, -1, -1)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300])
def test_single_tokens(n, dtype):
    say("decode", n, dtype)
    Batch(n, [(1, n), (1, max(1, n // 2)), (1, n)], 8, 2).check(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 33, 64, 65, 130, 257])
def test_whole_prompts(n, dtype):
    say("prompt", n, dtype)
    Batch(100 + n, [(n, n), (max(1, n // 3), max(1, n // 3))], 4, 2).check(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("q,n", [(2, 300), (5, 131), (7, 64), (20, 333), (40, 200), (130, 259)])
def test_chunks_after_a_cached_part(q, n, dtype):
    say("chunk", q, n, dtype)
    Batch(200 + q, [(q, n), (q, q), (q, q + 1)], 8, 2, widths=(4, 4, 6, 8)).check(dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_mixed_batch_with_empty_sequences(dtype):
    # sequences without new tokens, without any token, with one, with a chunk
    lens = [(0, 40), (1, 77), (33, 90), (0, 0), (1, 1), (70, 70), (3, 500), (0, 5)]
    Batch(300, lens, 8, 2, widths=(3, 4, 6, 8), page=32).check(dtype)


@pytest.mark.parametrize("mix", MIXES)
@pytest.mark.parametrize("low", [3, 4])
def test_every_width_mix(mix, low):
    w = [low] * mix[0] + [6] * mix[1] + [8] * mix[2]
    if mix[0] == 2 and low == 3:
        w[1] = 4
    say("widths", w)
    Batch(400 + sum(w), [(1, 70), (21, 70)], 8, 2, widths=w).check(torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (5, 5), (6, 2), (12, 4), (16, 1), (17, 1), (40, 2), (64, 1)])
def test_head_groupings(Hq, Hkv, dtype):
    say("heads", Hq, Hkv, dtype)
    Batch(500 + Hq, [(1, 130), (9, 75)], Hq, Hkv).check(dtype)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 512, 1024])
def test_page_sizes(page):
    Batch(600 + page, [(1, 1030), (37, 500), (1, 15)], 4, 2, page=page, extra_pages=1).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window", [1, 2, 16, 50, 64, 100, 1000])
def test_windows(window, dtype):
    Batch(700 + window, [(1, 300), (90, 200), (200, 200)], 4, 2, window=window).check(dtype)


@pytest.mark.parametrize("window", [0, 1, 40])
def test_prefixes(window):
    # a prefix of nothing, of some tokens, past the rows' own positions, past the end
    lens = [(1, 200), (60, 200), (100, 100), (100, 100), (30, 90), (5, 5)]
    Batch(800 + window, lens, 4, 2, window=window, prefix=[3, 17, 0, 64, 90, 1000]).check()
    Batch(801 + window, lens, 4, 2, window=window, prefix=[-5, 130, 99, 100, 0, 2]).check(torch.bfloat16)


@pytest.mark.parametrize("dtype", TYPES)
def test_capped_and_biased_scores(dtype):
    lens = [(1, 333), (50, 210), (128, 128)]
    slopes = [2.0 ** -(i + 1) for i in range(8)]
    Batch(900, lens, 8, 2, softcap=5.0).check(dtype)
    Batch(901, lens, 8, 2, slopes=slopes).check(dtype)
    Batch(902, lens, 8, 2, softcap=20.0, slopes=slopes, window=70, prefix=[2, 0, 60]).check(dtype)


@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0, 4.0])
def test_scales(scale):
    Batch(950, [(1, 150), (40, 90)], 4, 2, scale=scale).check()


def test_rows_that_see_nothing_are_zero():
    # more new tokens than cached ones (positions below zero), no token at all
    b = Batch(960, [(5, 5), (1, 40)], 4, 2)
    b.kv_len.copy_(torch.tensor([2, 0]))
    for dtype in TYPES:
        o = b.run(dtype)
        assert not o[:3].any() and not o[5].any() and bool(o[3:5].any(dim=2).all())
    b = Batch(961, [(40, 40)], 4, 2, prefix=[3])
    b.kv_len.copy_(torch.tensor([6]))                      # rows at -34 .. 5: the prefix is seen by all
    o = b.run()
    assert bool(o.any(dim=2).all())
    assert torch.allclose(o[0].isnan(), torch.zeros_like(o[0], dtype=torch.bool))


def test_rows_outside_every_sequence_stay_as_they_are():
    for lens in ([(1, 60), (1, 9)], [(40, 60), (3, 9)]):
        for dtype in TYPES:
            b = Batch(970, lens, 8, 2, tail_rows=37)
            out = torch.full((b.T, 8, D), 7.0, dtype=dtype, device="cuda")
            b.q[-37:] = float("nan")
            b.run(dtype, out=out)
            assert bool((out[-37:] == 7.0).all()) and not out[:-37].isnan().any()


def test_table_entries_outside_the_pool_read_as_zero_rows():
    b = Batch(980, [(1, 100), (30, 64)], 4, 2, page=16)
    kk, vv = mxq.kv_read(b.cache, b.slots)
    zero = torch.zeros_like(kk[:16])
    mxq.kv_append(b.cache, zero, zero, b.slots[16:32])     # the second page of the first sequence
    mxq.kv_append(b.cache, zero[:16], zero[:16], b.slots[148:164])   # the last page of the second
    want = [b.run(t) for t in TYPES]
    for hole in (-1, 2 ** 31 - 1, -2 ** 31, b.cache.pages):
        b.table[0, 1] = hole
        b.table[1, 3] = hole
        for t, w in zip(TYPES, want):
            assert torch.equal(b.run(t), w)


def test_strided_queries_and_table():
    b = Batch(990, [(1, 100), (30, 64)], 6, 2)
    want = b.run()
    fused = torch.randn((b.T, 10, D), device="cuda").to(torch.bfloat16)
    fused[:, 2:8] = b.q
    assert torch.equal(b.run(q=fused[:, 2:8]), want)
    heads = b.q.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(b.run(q=heads), want)
    wide = torch.full((2, b.table.shape[1] + 9), -7, dtype=torch.int32, device="cuda")
    wide[:, 4:4 + b.table.shape[1]] = b.table
    b.table = wide[:, 4:4 + b.table.shape[1]]
    assert torch.equal(b.run(), want)


def test_lengths_end_at_the_table_and_at_max_kv():
    b = Batch(995, [(1, 100)], 4, 2, page=16)
    b.kv_len.fill_(48)
    want = b.run()
    b.kv_len.fill_(2 ** 31 - 1)
    full = b.table
    b.table = full[:, :3].contiguous()
    assert torch.equal(b.run(), want)
    b.table, b.max_kv = full, 48
    assert torch.equal(b.run(), want)


@pytest.mark.parametrize("spread", [12, 40])
def test_blocks_of_unlike_size(spread):
    # block scales far apart: K's and V's from 2^-spread to 2^spread
    Batch(1000 + spread, [(1, 90), (20, 60)], 4, 2, widths=(4, 4, 6, 8), spread=spread,
          scale=2.0 ** -(spread + 3)).check()


@pytest.mark.parametrize("widths", [(3, 4, 6, 8), (4, 4, 4, 4), (8, 8, 8, 8), (6, 6, 6, 6)])
def test_values_at_the_ends_of_the_range(widths):
    # V blocks near 2^110 (sums of them stay in range) and below 2^-126, K zero (uniform weights)
    b = Batch(1100, [(1, 40), (20, 40)], 4, 2, widths=widths)
    g = torch.Generator().manual_seed(5)
    n = b.slots.numel()
    v = torch.rand((n, 2, D), generator=g) * 0.75 + 0.25
    v[:, 0] *= 2.0 ** 110
    v[:, 1] *= 2.0 ** -126
    k = torch.zeros((n, 2, D), dtype=torch.bfloat16)
    mxq.kv_append(b.cache, k.cuda(), v.to(torch.bfloat16).cuda(), b.slots)
    _, vv = mxq.kv_read(b.cache, b.slots)
    for dtype in TYPES:
        o = b.run(dtype).double().cpu()
        assert bool(torch.isfinite(o).all())
        for s, (rows, at) in enumerate(((range(0, 1), 0), (range(1, 21), 40))):
            for r in rows:
                L = 40 if s == 0 else 21 + (r - 1)
                mean = vv[at:at + L].double().cpu().mean(dim=0).repeat_interleave(2, dim=0)
                tol = (2.0 ** -7 if dtype is torch.bfloat16 else 2.0 ** -18)
                # (values near 2^-126 may lose up to 2^-133 to bf16's subnormal steps)
                assert bool(((o[r] - mean).abs() <= tol * mean.abs() + 2.0 ** -132).all())


def test_infinite_and_nan_queries_stay_in_their_rows():
    b = Batch(1200, [(1, 60), (40, 100)], 4, 2)
    want = {t: b.run(t) for t in TYPES}
    b.q[0, 1, 3] = float("nan")
    b.q[7, 2, 9] = float("inf")
    keep = torch.ones((b.T, 4), dtype=torch.bool, device="cuda")
    keep[0, 1] = keep[7, 2] = False
    for t in TYPES:
        o = b.run(t)
        assert bool(o[0, 1].isnan().all()) and torch.equal(o[keep], want[t][keep])


def test_keys_that_held_infinities_count_as_zero():
    b = Batch(1210, [(1, 50), (17, 50)], 4, 2)
    x = torch.randn((100, 2, D), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    y = x.clone()
    y[::7, :, 40] = float("inf")
    y[3::7, :, 100] = float("nan")
    z = x.clone()
    z[::7, :, 32:64] = 0
    z[3::7, :, 96:] = 0
    out = []
    for rows in (y, z):
        mxq.kv_append(b.cache, rows.cuda(), rows.cuda(), b.slots)
        out.append([b.run(t) for t in TYPES])
    for a, c in zip(*out):
        assert torch.equal(a, c) and bool(torch.isfinite(a).all())


def test_repeats_and_work_contents_do_not_matter():
    for lens in ([(1, 3000), (1, 700)], [(300, 900), (1, 40)]):
        b = Batch(1300, lens, 8, 2)
        n = mxq.attn_paged_work_bytes(b.cache, b.S, b.T, 8, b.max_q, b.max_kv)
        work = torch.full((max(n, 16),), 255, dtype=torch.uint8, device="cuda")
        for t in TYPES:
            first = b.run(t, work=work)
            assert torch.equal(first, b.run(t, work=work)) and torch.equal(first, b.run(t))


def test_long_caches():
    Batch(1400, [(1, 20000), (1, 1)], 8, 1).check(seqs=[0])
    Batch(1401, [(5, 9001)], 8, 1, page=256, widths=(4, 4, 4, 8)).check(torch.bfloat16)


def test_serving_batch_sampled():
    # 24 sequences of unlike length, one of them far longer
    lens = [(1, 50 + 61 * i) for i in range(23)] + [(1, 12000)]
    Batch(1402, lens, 32, 8, page=64).check(seqs=[0, 7, 22, 23])


def test_prompt_chunk_sampled():
    Batch(1403, [(150, 2100), (1, 700), (400, 400)], 16, 2, page=64, widths=(4, 4, 4, 6)).check(
        torch.bfloat16, seqs=[0, 1])


def test_graph_replays_with_other_lengths():
    # a decode step captured once, replayed as the sequences grow; and a chunk
    for q, lens in ((1, [(1, 700), (1, 64)]), (20, [(20, 300), (20, 64)])):
        b = Batch(1500 + q, lens, 8, 2)
        work = torch.empty(max(16, mxq.attn_paged_work_bytes(b.cache, 2, b.T, 8, b.max_q, 1024)),
                           dtype=torch.uint8, device="cuda")
        b.max_kv = 1024
        out = torch.empty((b.T, 8, D), dtype=torch.float32, device="cuda")
        b.run(out=out, work=work)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.run(out=out, work=work)
        first = b.kv_len.clone()
        for step in (0, 5, 41, 20):
            b.kv_len.copy_(first - step)
            want = b.run()
            out.fill_(float("nan"))
            work.fill_(0xA5)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)


def test_another_stream():
    b = Batch(1600, [(1, 500), (40, 80)], 8, 2)
    want = b.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = b.run()
    side.synchronize()
    assert torch.equal(got, want)


def test_a_layers_steps_together():
    # a prompt in two chunks, then tokens one by one, appended and attended through one cache,
    # against the whole prompt at once: the same rows, whatever the chunks
    Hq, Hkv, page, N = 8, 2, 16, 75
    g = torch.Generator().manual_seed(8)
    rows = torch.randn((N, Hq + 2 * Hkv, D), generator=g).to(torch.bfloat16).cuda()
    q, k, v = rows.split([Hq, Hkv, Hkv], dim=1)
    table = mxq.rope_table(mxq.rope_inv_freq(128)[0], 128)
    pages = torch.randperm(6, generator=g).int().cuda()[None]
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    slots = pages[0].long()[pos.long() // page] * page + pos.long() % page

    def step(cache, a, b):
        cu = torch.tensor([0, b - a], dtype=torch.int32, device="cuda")
        n = torch.tensor([b], dtype=torch.int32, device="cuda")
        qr = mxq.kv_append(cache, k[a:b], v[a:b], slots[a:b], pos=pos[a:b], rope=table, q=q[a:b])
        assert torch.equal(qr, mxq.rope(q[a:b], pos[a:b], table))
        return mxq.attn_paged(qr, cache, cu, n, pages, b - a, b, D ** -0.5, dtype=torch.float32)

    fmt = mxq.Format(D, [4, 4, 6, 8])
    whole = step(mxq.PagedCache(fmt, Hkv, 6, page), 0, N)
    cache = mxq.PagedCache(fmt, Hkv, 6, page)
    cuts = [0, 33, 70] + list(range(71, N + 1))
    parts = torch.cat([step(cache, a, b) for a, b in zip(cuts, cuts[1:])])
    # two float32 evaluations of the same mean, each within 2^-24 (131 + 4 + 64) of the values'
    # largest (scores are of the order of 1 here; see paged_util)
    bound = 2 * 2 * 2.0 ** -24 * (131 * 16 + 4 + 64 * 4) * float(v.float().abs().max()) * 1.1
    assert float((whole - parts).abs().max()) <= bound
    # the rotated, quantized first token attends to itself alone
    _, vv = mxq.kv_read(cache, slots[:1])
    assert torch.equal(whole[0], vv[0].float().repeat_interleave(Hq // Hkv, dim=0))


# Batches whose tiles are as many as the CUs (16 x 128 new tokens of 8 query heads for each of 4 KV
# heads are 256 tiles of 256 rows): the kernel with eight waves
def _wide(seed, **kw):
    lens = [(128, 128 + 37 * i) for i in range(15)] + [(128, 128)]
    kw = {"widths": (4, 4, 6, 8), "page": 64, **kw}
    b = Batch(seed, lens, 32, 4, **kw)
    assert b.T * 8 // 256 * 4 >= torch.cuda.get_device_properties(0).multi_processor_count
    return b


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("widths", [(4, 4, 6, 8), (4, 4, 4, 4), (3, 3, 6, 8), (8, 8, 8, 8)])
def test_many_tiles(widths, dtype):
    say("many tiles", widths, dtype)
    _wide(2000 + sum(widths), widths=widths).check(dtype, seqs=[3, 15])


@pytest.mark.parametrize("dtype", TYPES)
def test_many_tiles_with_masks_caps_and_biases(dtype):
    slopes = [2.0 ** (-8.0 * (h + 1) / 32) for h in range(32)]
    _wide(2010, window=70, prefix=[5 * i for i in range(16)]).check(dtype, seqs=[0, 9])
    _wide(2011, softcap=8.0, slopes=slopes, prefix=[600] * 16).check(dtype, seqs=[6])
    _wide(2012, slopes=slopes, window=100).check(dtype, seqs=[15])


def test_many_tiles_holes_nans_and_repeats():
    b = _wide(2020, page=16)
    want = {t: b.run(t) for t in TYPES}
    for t in TYPES:
        assert torch.equal(b.run(t), want[t])
    zero = torch.zeros((16, 4, D), dtype=torch.bfloat16, device="cuda")
    mxq.kv_append(b.cache, zero, zero, b.slots[16:32])
    want = {t: b.run(t) for t in TYPES}
    b.table[0, 1] = -1
    for t in TYPES:
        assert torch.equal(b.run(t), want[t])
    b.q[130, 3, 5] = float("nan")
    b.q[700, 20, 9] = float("-inf")
    keep = torch.ones((b.T, 32), dtype=torch.bool, device="cuda")
    keep[130, 3] = keep[700, 20] = False
    for t in TYPES:
        o = b.run(t)
        assert bool(o[130, 3].isnan().all()) and torch.equal(o[keep], want[t][keep])


@pytest.mark.parametrize("dtype", TYPES)
def test_both_kernels_split_and_merged(dtype):
    # long caches and few sequences: the decoding ones and the chunk are both split, into unlike counts
    lens = [(1, 5000), (40, 4000), (0, 100), (1, 33), (2, 2600), (1, 1)]
    b = Batch(2100, lens, 8, 1, widths=(4, 4, 4, 8), page=128)
    b.check(dtype)
    # and G = 20 query heads: two groups of sixteen rows beside the tiles
    Batch(2101, [(1, 1500), (17, 900), (1, 40)], 20, 1).check(dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,q", [(8, 4), (8, 3), (32, 1), (24, 1), (1, 32), (1, 17), (5, 6)])
def test_up_to_32_rows(Hq, q, dtype):
    say("rows", Hq, q, dtype)
    Batch(2200 + 10 * Hq + q, [(q, 300), (q, q), (q, 1000)], Hq, 1, widths=(3, 4, 6, 8), window=0).check(dtype)


def test_many_sequences():
    # more than 64: the search of a tile's sequence takes two steps; some have no rows
    lens = [(3 + (i % 40), 3 + (i % 40) + i) if i % 7 else (0, i) for i in range(150)]
    Batch(2300, lens, 4, 2).check(seqs=[1, 63, 64, 65, 128, 149])
    Batch(2301, [(1, 1 + i) for i in range(130)], 8, 1).check(torch.bfloat16, seqs=[0, 64, 129])


def test_two_calls_at_once_on_two_streams():
    b = [Batch(2400 + i, [(1, 900), (30, 400)], 8, 2) for i in range(2)]
    want = [x.run() for x in b]
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        for x, s in zip(b, side):
            with torch.cuda.stream(s):
                got.append(x.run())
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert torch.equal(g, want[i % 2])


def test_pages_past_four_gigabytes():
    # K's mantissas alone take 4.6 GB: page 0 and the last ones hold the sequences
    Hkv, page, pages = 16, 1024, 2200
    assert pages * page * Hkv * 128 > 2 ** 32
    mk = lambda m: torch.empty(pages * page * Hkv * m, dtype=torch.uint8, device="cuda")  # noqa: E731
    fmt = mxq.Format(D, [8, 8, 8, 8])
    far = mxq.PagedCache(fmt, Hkv, pages, page, k=(mk(128), mk(4)), v=(mk(128), mk(4)))
    near = mxq.PagedCache(fmt, Hkv, 3, page)
    g = torch.Generator().manual_seed(12)
    n = 1500
    k, v = (torch.randn((n, Hkv, D), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    t = torch.arange(n, device="cuda")
    tables = {}
    for c, at in ((far, [pages - 1, 0]), (near, [2, 0])):
        tables[c] = torch.tensor([at], dtype=torch.int32, device="cuda")
        mxq.kv_append(c, k, v, tables[c][0].long()[t // page] * page + t % page)
    for q in (1, 70):
        x = torch.randn((q, 2 * Hkv, D), generator=g).to(torch.bfloat16).cuda()
        cu = torch.tensor([0, q], dtype=torch.int32, device="cuda")
        kv = torch.tensor([n], dtype=torch.int32, device="cuda")
        a, b = (mxq.attn_paged(x, c, cu, kv, tables[c], q, n, 0.1) for c in (far, near))
        assert torch.equal(a, b) and bool(a.any())


def test_odd_counts_of_partial_results():
    # one query head, one row, an odd number of splits
    for n in (400, 700, 1000):
        Batch(2500 + n, [(1, n)], 1, 1).check()
    Batch(2600, [(1, 900), (1, 500), (1, 77)], 1, 1).check(torch.bfloat16)


@pytest.mark.parametrize("S", [63, 64, 65, 130])
def test_counts_of_sequences_with_tiles(S):
    # empty, single, few and many rows in turn
    kinds = [(0, 9), (1, 30), (40, 40), (9, 60), (0, 0), (65, 70), (17, 17)]
    b = Batch(1600 + S, [kinds[(3 * s) % 7] for s in range(S)], 8, 2, tail_rows=3)
    b.check(seqs=[0, 1, 2, 3, 4, 5, 6, 61, 62, S - 3, S - 2, S - 1])
    empty = Batch(1700 + S, [(0, 5)] * (S - 1) + [(50, 90)], 8, 2)
    empty.check(torch.bfloat16)


@pytest.mark.parametrize("lens,kw", [([(256, 2100)], {}),
                                     ([(300, 2100), (5, 900), (200, 700)], dict(widths=(4, 4, 6, 8))),
                                     ([(256, 2200)], dict(window=900, prefix=[70])),
                                     ([(300, 2100), (0, 4), (205, 700)], dict(softcap=30.0))])
def test_tiles_of_all_rows_with_their_tokens_split(lens, kw):
    # full tiles of 256 rows, several splits of each
    for dtype in TYPES:
        Batch(1800 + len(lens), lens, 32, 8, page=64, **kw).check(dtype, seqs=[0])


@pytest.mark.parametrize("cap", [40.0, 300.0, 1e4, 1e6, 1e9, 1e20, 3e38])
def test_caps_far_above_the_scores(cap):
    # almost the identity; what is lost has to be a part of the score, not of the cap.
    # (A bf16 result's tanh: its exponential and reciprocal are good to 5.2 x 2^-24 of the cap from an
    # eighth of the cap on, 42 x 2^-24 of the score; the score's own sum is allowed 131 in tol32.)
    lens = [(1, 333), (50, 210), (5, 64)]
    for Hq, scale in ((8, D ** -0.5), (2, 1.0)):
        b = Batch(3000, lens, Hq, 2, softcap=cap, scale=scale)
        b.check(torch.float32)
        o, tol32, tol16 = b.expected()
        d = np.abs(b.run(torch.bfloat16).double().cpu().numpy() - o)
        assert np.all(d <= tol16 + tol32 * (42 / 131))
    slopes = [2.0 ** -(i + 1) for i in range(8)]
    Batch(3001, lens, 8, 2, softcap=cap, slopes=slopes, window=70, prefix=[2, 0, 60]).check(torch.bfloat16)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,Hq,Hkv,max_q", [
    ([(3, 100), (1, 50), (0, 20), (40, 200)], 16, 2, 1),             # the kernel for few rows alone
    ([(3, 5000), (1, 2050), (7, 7)], 8, 1, 2),                       # and its splits
    ([(60, 300), (1, 200), (5, 90), (41, 41)], 8, 2, 40),            # both kernels
    ([(60, 3000), (1, 2000), (5, 90)], 8, 1, 33),                    # and the splits of both
    ([(60, 300), (3, 90)], 40, 1, 20),                               # tiles alone
    ([(60, 3000), (20, 500)], 8, 1, 40),                             # as many rows as 2 x max_q: tiles, split
    ([(5 + i % 50, 60 + i) for i in range(70)], 4, 2, 17)])          # more than 64 sequences
def test_rows_past_max_q_are_not_computed(lens, Hq, Hkv, max_q, dtype):
    say("max_q", len(lens), Hq, Hkv, max_q, dtype)
    b = Batch(3100 + max_q, lens, Hq, Hkv)
    assert b.max_q > max_q
    b.max_q = max_q
    out = torch.full((b.T, Hq, D), 7.0, dtype=dtype, device="cuda")
    work = torch.full((max(16, mxq.attn_paged_work_bytes(b.cache, b.S, b.T, Hq, max_q, b.max_kv)),), 0x41,
                      dtype=torch.uint8, device="cuda")
    b.run(dtype, out=out, work=work)
    o, tol32, tol16 = b.expected()
    got = out.double().cpu().numpy()
    first = np.concatenate([np.arange(n) < max_q for n, _ in lens])
    assert np.all(got[~first] == 7.0)
    # (the others stand where they stood: at their own positions)
    assert np.all(np.abs(got - o)[first] <= (tol32 if dtype is torch.float32 else tol16)[first])


@pytest.mark.parametrize("widths", [(3, 3, 3, 3), (4, 4, 4, 4), (6, 6, 6, 6), (8, 8, 8, 8), (3, 4, 6, 8)])
def test_lowest_values_of_the_full_clamp_stay_out_of_rows_that_do_not_see_them(widths):
    # -2^128, which the full clamp's lowest mantissa stands for with E = 254, has no bf16: in a token that
    # a row does not see it must not reach the row (0 x infinity)
    b = Batch(3200, [(1, 60), (40, 100), (5, 40)], 4, 2, widths=widths, window=9)
    fmt = mxq.Format(D, list(widths), clamp="full")
    cache = mxq.PagedCache(fmt, 2, b.cache.pages, b.page)
    g = torch.Generator().manual_seed(3)
    x = torch.randn((200, 2, D), generator=g).to(torch.bfloat16)
    y = x.clone()
    low = torch.tensor([5, 59, 60, 120, 159, 160 + 39, 160])     # the batch's rows in the cache, by sequence
    y[low] = torch.finfo(torch.bfloat16).min
    b.cache = cache
    rows = torch.arange(b.T)
    pos = torch.cat([torch.tensor([59]), torch.arange(60, 100), torch.arange(35, 40)])
    seq = torch.tensor([0] + [1] * 40 + [2] * 5)
    sees = torch.zeros(b.T, dtype=torch.bool)
    for t in low.tolist():
        s = 0 if t < 60 else 1 if t < 160 else 2
        j = t - (0, 60, 160)[s]
        sees |= (seq == s) & (j <= pos) & (pos - j < 9)
    assert sees.any() and not sees.all()
    for dtype in TYPES:
        mxq.kv_append(cache, x.cuda(), x.cuda(), b.slots)
        want = b.run(dtype)
        mxq.kv_append(cache, x.cuda(), y.cuda(), b.slots)
        got = b.run(dtype)
        keep = rows[~sees].cuda()
        assert torch.equal(got[keep], want[keep])
        assert not got.isnan().any()


@pytest.mark.parametrize("q", [1, 40])
def test_the_longest_cache(q):
    # 2^31 - 1 tokens, every table entry the same page, a window that ends at the last one: the places are
    # those of 1023 tokens, and so is the result, bit for bit; the place behind them holds infinities
    n, short = 2 ** 31 - 1, 1023
    cache = mxq.PagedCache(mxq.Format(D, [4, 4, 6, 8]), 1, 2, 1024)
    for t in cache.k + cache.v:
        t.fill_(0x77)
    cache.k[1].fill_(255)
    cache.v[1].fill_(255)
    g = torch.Generator().manual_seed(7)
    x = torch.randn((short, 1, D), generator=g).to(torch.bfloat16).cuda()
    mxq.kv_append(cache, x, x.flip(0), torch.arange(1024, 1024 + short, device="cuda"))
    table = torch.ones((1, 2 ** 21), dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, q], dtype=torch.int32, device="cuda")
    xq = torch.randn((q, 8, D), generator=g).to(torch.bfloat16).cuda()
    for dtype in TYPES:
        got, want = (mxq.attn_paged(xq, cache, cu, torch.tensor([L], dtype=torch.int32, device="cuda"), table,
                                    q, n, 0.1, window=50, dtype=dtype) for L in (n, short))
        assert torch.equal(got, want) and bool(torch.isfinite(got).all()) and bool(got.any())


@pytest.mark.parametrize("q", [1, 64])
def test_float32_results_use_all_bits_of_the_probabilities(q):
    # Two tokens, both in the prefix that every row sees.  Scores 0 and x, x a value of q itself (the key is
    # one in a single place: an exact product); the values 0 and 1: o = e^x / (1 + e^x).  The exponential: a
    # few units and one of its argument, as in paged_util, on each side; one rounding each of the sum, the
    # reciprocal and the product.  The value product is exact with three bf16 terms of the probability; with
    # two it would be off by up to 2^-18 of it.
    cache = mxq.PagedCache(mxq.Format(D, [4, 4, 4, 8]), 1, 1, 16)
    k = torch.zeros((2, 1, D), dtype=torch.bfloat16)
    v = k.clone()
    k[1, 0, 40], v[1] = 1.0, 1.0
    mxq.kv_append(cache, k.cuda(), v.cuda(), torch.arange(2, device="cuda"))
    xq = torch.zeros((q, 16, D), dtype=torch.bfloat16)
    g = torch.Generator().manual_seed(11)
    x = -(torch.rand((q, 16), generator=g) * 2).to(torch.bfloat16)
    xq[:, :, 40] = x
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    got = mxq.attn_paged(xq.cuda(), cache, i32(0, q), i32(2), i32(0).view(1, 1), q, 2, 1.0, prefix=i32(2),
                         dtype=torch.float32).double().cpu()
    e = x.double().exp()
    ref = e / (1 + e)
    u = 2.0 ** -24
    bound = ref * u * ((4 + 4 * x.double().abs()) + 3)
    assert bool(((got - ref[..., None]).abs() <= bound[..., None]).all())
    # (the inputs tell two terms from three)
    p = e.float()
    hi = p.to(torch.bfloat16).float()
    two = (hi + (p - hi).to(torch.bfloat16).float()).double()
    assert bool(((two - e).abs() / (1 + e) > 2 * bound).any())


def _waves(T, G, Hkv, max_kv, cus):
    """Waves per tile and splits of the tiles, by the plan's rule for an uneven batch."""
    steps, t4, t8 = -(-max_kv // 64), T * G // 128 + 1, T * G // 256 + 1
    n4, n8 = (max(1, min(w // (t * Hkv), steps // 4, 256)) for w, t in ((2 * cus, t4), (cus, t8)))
    wgs = t8 * Hkv * n8
    eight = G >= 4 and 16 * wgs >= 15 * cus * -(-wgs // cus) and 12 * t8 <= 7 * t4
    return (8, n8) if eight else (4, n4)


@pytest.mark.parametrize("S,T,kv,Hq,Hkv,waves,split", [
    (65, 1940, 1500, 32, 4, 8, False),              # whole rounds of full tiles
    (130, 1290, 1500, 16, 2, 8, True),              # and split
    (100, 580, 3000, 8, 1, 4, True)])               # few rows over long caches
def test_more_than_64_sequences_in_every_kind_of_tile(S, T, kv, Hq, Hkv, waves, split):
    say("many sequences", S, T, kv, Hq, Hkv)
    # two chunks among sequences that decode, draft or bring nothing
    lens = [((1, 30 + s), (0, 9), (3, 50), (0, 0), (17, 70))[s % 5] for s in range(S)]
    rest = T - sum(n for s, (n, _) in enumerate(lens) if s not in (3, S - 2))
    lens[3], lens[S - 2] = (rest // 8, kv), (rest - rest // 8, rest)
    b = Batch(3300 + S, lens, Hq, Hkv, page=64, widths=(4, 4, 6, 8))
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    got, n = _waves(T, Hq // Hkv, Hkv, b.max_kv, cus)
    if cus == 256:
        assert got == waves and (n > 1) == split, (got, n)
    for dtype in TYPES:
        b.check(dtype, seqs=[0, 1, 2, 3, 4, 34, 63, 64, S - 1])


def test_a_few_rows_among_many_empty_sequences():
    # tiles are launched for all 65536 of them, with as many splits as a dispatch has room for
    lens = [(0, 0)] * 65536
    lens[7], lens[40000], lens[65535] = (1, 20), (34, 60), (5, 300)
    b = Batch(3400, lens, 8, 1)
    b.max_kv = 65536
    n = mxq.attn_paged_work_bytes(b.cache, b.S, b.T, 8, b.max_q, b.max_kv) // (4 * b.T * 8 * (D + 2))
    assert n > 100
    for dtype in TYPES:
        b.check(dtype, seqs=[7, 40000, 65535])


def test_a_layers_step_captured_and_replayed_with_other_inputs():
    # append (queries rotated by the same launch), attention, rows read back, all in one graph with its own
    # allocations, replayed with other rows, positions, slots and lengths, beside eager calls
    Hq, Hkv, page, S, most = 8, 2, 16, 3, 400
    g = torch.Generator().manual_seed(21)
    fmt = mxq.Format(D, [3, 4, 6, 8])
    pages = S * most // page
    table = torch.randperm(pages, generator=g).int().view(S, -1).cuda()
    rope = mxq.rope_table(mxq.rope_inv_freq(D)[0], most)
    new = [1, 40, 5]
    T = sum(new)
    cu = torch.tensor([0, 1, 41, 46], dtype=torch.int32, device="cuda")
    rows = torch.empty((T, Hq + 2 * Hkv, D), dtype=torch.bfloat16, device="cuda")
    slots, pos = torch.empty(T, dtype=torch.int64, device="cuda"), torch.empty(T, dtype=torch.int32, device="cuda")
    kv_len = torch.empty(S, dtype=torch.int32, device="cuda")

    def fill(lens):
        rows.copy_(torch.randn(rows.shape, generator=g))
        at = torch.cat([torch.arange(L - n, L) for L, n in zip(lens, new)])
        seq = torch.repeat_interleave(torch.arange(S), torch.tensor(new))
        pos.copy_(at.int())
        slots.copy_(table.cpu()[seq, at // page].long() * page + at % page)
        kv_len.copy_(torch.tensor(lens, dtype=torch.int32))

    def step(cache):
        q, k, v = rows.split([Hq, Hkv, Hkv], dim=1)
        qr = mxq.kv_append(cache, k, v, slots, pos=pos, rope=rope, q=q)
        o = mxq.attn_paged(qr, cache, cu, kv_len, table, max(new), most, D ** -0.5, window=150, prefix=cu[1:])
        return (qr, o, mxq.rope(qr, pos, rope)) + tuple(mxq.kv_read(cache, slots))

    eager, graphed = (mxq.PagedCache(fmt, Hkv, pages, page) for _ in range(2))
    fill([1, 40, 5])
    for c in (eager, graphed):
        step(c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(graphed)
    for lens in ([2, 80, 10], [3, 120, 15], [390, 333, 400], [4, 41, 16]):
        fill(lens)
        want = step(eager)
        for t in got:
            t.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        for a, b in zip(eager.k + eager.v, graphed.k + graphed.v):
            assert torch.equal(a, b)
