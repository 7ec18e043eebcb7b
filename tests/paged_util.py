"""Shared by the tests of attention over the paged cache: a ragged batch in
permuted pages of a cache that is noise elsewhere, the oracle's answer, and the
bound on their difference."""
from __future__ import annotations

import numpy as np
import torch

from oracle import paged as opaged
from paper_2607_17733_amd import mxq

D = 128


class Batch:
    def __init__(self, seed, lens, Hq, Hkv, widths=(4, 4, 4, 4), page=16, window=0, prefix=None,
                 softcap=0.0, slopes=None, scale=D ** -0.5, extra_pages=3, tail_rows=0, spread=0):
        """lens: (new tokens, cached tokens) of each sequence; tail_rows: rows of q
        that belong to no sequence; spread: block scales 2^-spread .. 2^spread."""
        g = torch.Generator().manual_seed(seed)
        self.lens, self.Hq, self.Hkv, self.widths, self.page = list(lens), Hq, Hkv, list(widths), page
        self.window, self.softcap, self.scale = window, softcap, scale
        S = len(self.lens)
        T = sum(n for n, _ in self.lens)
        self.S, self.T = S, T + tail_rows
        need = [-(-n // page) for _, n in self.lens]
        pages = sum(need) + extra_pages
        most = max(max(need, default=0), 1)
        order = torch.randperm(pages, generator=g).int()
        table = torch.full((S, most), 2 ** 31 - 1, dtype=torch.int32)
        at = 0
        for s, k in enumerate(need):
            table[s, :k] = order[at:at + k]
            at += k
        self.cpu_table = table
        self.table = table.cuda()
        cu = np.concatenate([[0], np.cumsum([n for n, _ in self.lens])])
        self.cu_q = torch.tensor(cu, dtype=torch.int32).cuda()
        self.kv_len = torch.tensor([n for _, n in self.lens], dtype=torch.int32).cuda()
        self.max_q = max((n for n, _ in self.lens), default=0)
        self.max_kv = max((n for _, n in self.lens), default=0)
        self.prefix = None if prefix is None else torch.tensor(prefix, dtype=torch.int32).cuda()
        self.slopes = None if slopes is None else torch.tensor(slopes, dtype=torch.float32).cuda()
        self.cache = mxq.PagedCache(mxq.Format(D, self.widths), Hkv, pages, page)
        for t in self.cache.k + self.cache.v:                   # noise, E = 255 with mantissas among it
            t.copy_(torch.randint(0, 256, (t.numel(),), dtype=torch.uint8, generator=g))
            t[::3] = 255

        def rows(n, H):
            x = torch.randn((n, H, D), generator=g)
            if spread:
                e = torch.randint(-spread, spread + 1, (n, H, D // 32), generator=g).float()
                x = x * torch.exp2(e).repeat_interleave(32, dim=2)
            return x

        total = sum(n for _, n in self.lens)
        k, v = rows(total, Hkv), rows(total, Hkv)
        k[..., 5] *= 8
        k[..., 77] *= 8
        self.q = torch.randn((self.T, Hq, D), generator=g).to(torch.bfloat16).cuda()
        slots = [self.cpu_table[s].long()[torch.arange(n) // page] * page + torch.arange(n) % page
                 for s, (_, n) in enumerate(self.lens)]
        self.slots = torch.cat(slots).cuda()
        mxq.kv_append(self.cache, k.to(torch.bfloat16).cuda(), v.to(torch.bfloat16).cuda(), self.slots)

    def run(self, dtype=torch.float32, q=None, **kw):
        a = dict(softcap=self.softcap, window=self.window, prefix=self.prefix, slopes=self.slopes)
        a.update(kw)
        return mxq.attn_paged(self.q if q is None else q, self.cache, self.cu_q, self.kv_len, self.table,
                              self.max_q, self.max_kv, self.scale, dtype=dtype, **a)

    def expected(self, seqs=None):
        """(o, bound of a float32 result, bound of a bf16 result), float64 [T, Hq, 1 or D];
        rows of sequences outside `seqs` (None: all) are NaN."""
        kk, vv = mxq.kv_read(self.cache, self.slots)
        kk, vv = kk.cpu().double().numpy(), vv.cpu().double().numpy()
        q = self.q.cpu().double().numpy()
        o = np.full(q.shape, np.nan)
        tol32, tol16 = np.zeros(q.shape), np.zeros(q.shape)
        at = r = 0
        pre = [0] * self.S if self.prefix is None else self.prefix.tolist()
        sl = None if self.slopes is None else self.slopes.cpu().numpy()
        for s, (n, L) in enumerate(self.lens):
            if seqs is None or s in seqs:
                k, v = kk[at:at + L], vv[at:at + L]
                ref, absv, big, bias = opaged.attention(q[r:r + n], k, v, n, self.scale, self.softcap,
                                                        self.window, pre[s], sl)
                # A score: 128 exact products summed in float32 (128 roundings), the scale, the
                # tanh (a few units of its value, at most the cap) and the bias (product and
                # difference), the subtraction of the maximum.  The exponential: a few units, and
                # one of its argument (at most twice the largest score).  An error x of every
                # score or weight moves the output by at most 2 x max|v|.  The sums: at most a
                # rounding per 16 tokens and one per merged part (64 of them at most).
                u = 2.0 ** -24
                x = u * (131 * big + 8 * min(self.softcap or 0.0, big) + 4 * bias)
                e = u * (4 + 4 * (big + bias))
                acc = u * (64 + L / 16)
                vmax = np.abs(v).max(axis=(0, 2)) if L else np.zeros(self.Hkv)
                vmax = np.repeat(vmax, self.Hq // self.Hkv)[None, :, None]
                t = 2 * (x + e + acc) * vmax + np.zeros(ref.shape)
                o[r:r + n], tol32[r:r + n] = ref, t
                # bf16: half a step (2^-8) of the result and of each probability
                tol16[r:r + n] = t + 2.0 ** -8 * (1 + 2.0 ** -8) * (np.abs(ref) + absv)
            at += L
            r += n
        return o, tol32, tol16

    def check(self, dtype=torch.float32, seqs=None, **kw):
        got = self.run(dtype, **kw)
        o, tol32, tol16 = self.expected(seqs)
        g = got.double().cpu().numpy()
        rows = ~np.isnan(o)
        d = np.abs(g - o)[rows]
        t = (tol32 if dtype is torch.float32 else tol16)[rows]
        bad = ~(d <= t)
        assert not bad.any(), (int(bad.sum()), float(d[bad].max()) if bad.any() else 0, float(t.max()))
        return got
