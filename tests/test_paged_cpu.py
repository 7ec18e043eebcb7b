"""Rotary positions, the paged cache and its attention on the CPU: the C ABI's
status for every refused argument (nothing is launched: each call fails its
checks), the binding's checks, the frequencies of long contexts, and pins of
the oracle."""
import ctypes
import math
from unittest import mock

import numpy as np
import pytest
import torch

import oracle
from oracle import paged as opaged
from paper_2607_17733_amd import mxq

NULL, SHAPE, WIDTHS, ALIGN, UNSUPPORTED = 1, 2, 3, 5, 6
FAKE = 1 << 20                                     # aligned, never dereferenced


@pytest.fixture(scope="module")
def L():
    return mxq.lib()


def fmt(widths=(4, 4, 6, 8), K=128):
    return mxq.Format(K, list(widths))


def cache(**kw):
    c = dict(pages=4, Hkv=2, page_tokens=16, reserved=0, k_mant=FAKE, k_exp=FAKE, v_mant=FAKE, v_exp=FAKE)
    c.update(kw)
    return mxq._PagedKv(*[c[n] for n, _ in mxq._PagedKv._fields_])


def rotary(**kw):
    c = dict(table=FAKE, positions=100, rot=64, layout=0)
    c.update(kw)
    return mxq._Rotary(*[c[n] for n, _ in mxq._Rotary._fields_])


def ref(x):
    return None if x is None else ctypes.byref(x)


BAD_CACHES = [(dict(pages=0), SHAPE), (dict(pages=-1), SHAPE), (dict(Hkv=0), SHAPE), (dict(Hkv=65536), SHAPE),
              (dict(page_tokens=8), SHAPE), (dict(page_tokens=48), SHAPE), (dict(page_tokens=2048), SHAPE),
              (dict(page_tokens=0), SHAPE), (dict(pages=2 ** 28), SHAPE), (dict(pages=2 ** 62), SHAPE),
              (dict(reserved=1), UNSUPPORTED), (dict(k_mant=0), NULL), (dict(v_exp=0), NULL),
              (dict(k_exp=FAKE + 8), ALIGN), (dict(v_mant=FAKE + 4), ALIGN)]


def test_page_sizes(L):
    for widths, row in (((4, 4, 4, 4), 64), ((3, 3, 6, 8), 80), ((8, 8, 8, 8), 128), ((3, 4, 6, 8), 84)):
        f = fmt(widths)
        for Hkv in (1, 8):
            for page in (16, 64, 1024):
                assert L.mxq_kv_page_bytes(f.ref, Hkv, page) == Hkv * page * row
                assert L.mxq_kv_page_exp_bytes(f.ref, Hkv, page) == Hkv * page * 4
    assert L.mxq_kv_page_bytes(fmt().ref, 0, 16) == -SHAPE
    assert L.mxq_kv_page_bytes(fmt().ref, 1, 17) == -SHAPE
    assert L.mxq_kv_page_bytes(fmt((4, 4), 64).ref, 1, 16) == -SHAPE
    assert L.mxq_kv_page_bytes(None, 1, 16) == -NULL
    bad = fmt()
    bad.widths[1] = 5
    assert L.mxq_kv_page_exp_bytes(bad.ref, 1, 16) == -WIDTHS
    perm = fmt()
    perm._c.perm = FAKE
    assert L.mxq_kv_page_bytes(perm.ref, 1, 16) == -UNSUPPORTED


def test_rope_refusals(L):
    def call(r=None, x=FAKE, T=4, H=2, D=128, xs=(256, 128), pos=FAKE, y=FAKE + 4096, ys=(256, 128), null=False):
        return L.mxq_rope(None if null else ref(r or rotary()), x, T, H, D, *xs, pos, y, *ys, None)

    for kw, want in ((dict(null=True), NULL), (dict(r=rotary(table=0)), NULL), (dict(x=0), NULL),
                     (dict(y=0), NULL), (dict(pos=0), NULL), (dict(r=rotary(rot=63)), SHAPE),
                     (dict(r=rotary(rot=0)), SHAPE), (dict(r=rotary(rot=514), D=1024), SHAPE),
                     (dict(r=rotary(positions=0)), SHAPE), (dict(r=rotary(positions=2 ** 31)), SHAPE),
                     (dict(r=rotary(layout=2)), UNSUPPORTED), (dict(r=rotary(table=FAKE + 4)), ALIGN),
                     (dict(T=-1), SHAPE), (dict(H=-1), SHAPE), (dict(H=65536), SHAPE), (dict(D=63), SHAPE),
                     (dict(D=62), SHAPE), (dict(D=129), SHAPE), (dict(D=4098), SHAPE), (dict(T=2 ** 31), SHAPE),
                     (dict(x=FAKE + 2), ALIGN), (dict(y=FAKE + 4098), ALIGN), (dict(xs=(255, 128)), ALIGN),
                     (dict(ys=(256, 127)), ALIGN), (dict(y=FAKE, ys=(512, 128)), SHAPE),
                     (dict(T=2 ** 31 - 1, H=65535, D=4096), SHAPE), (dict(T=2 ** 20, H=64, D=128), SHAPE)):
        assert call(**kw) == want, kw
    assert call(T=0, x=0, y=0, pos=0) == 0 and call(H=0, x=0) == 0


def test_rope_refuses_output_rows_that_overlap(L):
    def call(T=4, H=2, ys=(256, 128), x=FAKE, xs=None):
        return L.mxq_rope(ref(rotary()), x, T, H, 128, *(xs or ys), FAKE, FAKE, *ys, None)

    for kw in (dict(ys=(0, 128)), dict(ys=(256, 0)), dict(ys=(256, 64)), dict(ys=(64, 256)),
               dict(ys=(-64, 256)), dict(ys=(256, 126), x=FAKE + 2 ** 20), dict(T=1, ys=(0, 0)),
               dict(H=1, ys=(126, 0))):
        assert call(**kw) == SHAPE, kw


def _overlap(T, ts, H, hs, D):
    at = sorted(t * ts + h * hs for t in range(T) for h in range(H))
    return any(b - a < D for a, b in zip(at, at[1:]))


def test_rope_refuses_rows_that_overlap_across_tokens_and_heads(L):
    # each stride alone keeps its rows apart, both together do not: token 1's first head is token 0's second
    def call(T, ts, H, hs, x=FAKE, D=128):
        return L.mxq_rope(ref(rotary()), x, T, H, D, ts, hs, FAKE, FAKE, ts, hs, None)

    assert call(2, 128, 2, 128) == SHAPE and call(2, 128, 2, 128, x=FAKE + 2 ** 20) == SHAPE
    far = 2 ** 62
    for T, ts, H, hs in ((2, far, 2, far + 126), (3, far, 3, -far), (2 ** 20, 130, 3, 130 * 2 ** 19 + 2),
                         (9, 256, 40, 896), (2, 384, 4, 128)):
        assert call(T, ts, H, hs) == SHAPE, (T, ts, H, hs)
    # every pair of small strides: refused exactly where rows overlap (the others pass every check,
    # which shows in what comes after them: nothing here has a device to launch on)
    steps = [-512, -390, -384, -256, -254, -128, -126, 0, 126, 128, 130, 254, 256, 258, 320, 384, 512, 640, 1024]
    ok = 0
    for T, H in ((2, 2), (2, 3), (3, 2), (4, 5), (7, 3)):
        for ts in steps:
            for hs in steps:
                want = SHAPE if _overlap(T, ts, H, hs, 128) else None
                if want is None and torch.cuda.is_available():
                    continue                           # (the address is not memory)
                got = call(T, ts, H, hs)
                assert (got == SHAPE) == (want == SHAPE), (T, ts, H, hs)
                ok += want is None
    assert ok > 100 or torch.cuda.is_available()


def test_rope_table_refusals(L):
    f = (ctypes.c_double * 256)(*[1.0] * 256)
    p = ctypes.cast(f, ctypes.c_void_p)
    assert L.mxq_rope_table(None, 64, 10, 1.0, FAKE, None) == NULL
    assert L.mxq_rope_table(p, 64, 10, 1.0, None, None) == NULL
    for rot, P, ms in ((63, 10, 1.0), (0, 10, 1.0), (514, 10, 1.0), (64, 0, 1.0), (64, -5, 1.0),
                       (64, 10, math.inf), (64, 10, math.nan)):
        assert L.mxq_rope_table(p, rot, P, ms, FAKE, None) == SHAPE
    assert L.mxq_rope_table(p, 512, 2 ** 25, 1.0, FAKE, None) == SHAPE
    f[5] = math.nan
    assert L.mxq_rope_table(p, 64, 10, 1.0, FAKE, None) == SHAPE
    f[5] = 1.0
    assert L.mxq_rope_table(p, 64, 10, 1.0, FAKE + 8, None) == ALIGN


def test_append_and_read_refusals(L):
    def call(c=None, f=None, k=FAKE, ks=(256, 128), v=FAKE, vs=(256, 128), T=4, slots=FAKE, pos=FAKE, r=None,
             q=None, Hq=0, qs=(0, 0), qo=None, null=False):
        return L.mxq_kv_append((f or fmt()).ref, None if null else ref(c or cache()), k, *ks, v, *vs, T, slots,
                               pos, ref(r), q, Hq, *qs, qo, None)

    good_q = dict(q=FAKE, Hq=4, qs=(512, 128), qo=FAKE + 8192)
    cases = [(dict(c=cache(**kw)), want) for kw, want in BAD_CACHES]
    cases += [(dict(null=True), NULL), (dict(f=fmt((4, 4), 64)), SHAPE), (dict(k=0), NULL), (dict(v=0), NULL),
              (dict(slots=0), NULL), (dict(r=rotary(), pos=0), NULL), (dict(r=rotary(rot=24)), SHAPE),
              (dict(r=rotary(rot=144)), SHAPE), (dict(r=rotary(layout=-1)), UNSUPPORTED),
              (dict(r=rotary(table=0)), NULL), (dict(T=-1), SHAPE), (dict(T=2 ** 31), SHAPE),
              (dict(k=FAKE + 8), ALIGN), (dict(ks=(260, 128)), ALIGN), (dict(vs=(256, 124)), ALIGN),
              (dict(good_q, qo=None), NULL), (dict(good_q, Hq=0), SHAPE), (dict(good_q, Hq=-1), SHAPE),
              (dict(good_q, qs=(516, 128)), ALIGN), (dict(good_q, qo=FAKE + 8), ALIGN),
              (dict(good_q, qo=FAKE, qs=(1024, 128)), SHAPE), (dict(good_q, Hq=65536), SHAPE),
              (dict(good_q, T=2 ** 31 - 1, Hq=65535), SHAPE), (dict(good_q, T=2 ** 24, Hq=64), SHAPE)]
    for kw, want in cases:
        assert call(**kw) == want, kw
    assert call(T=0, k=0, v=0, slots=0) == 0

    def read(c=None, slots=FAKE, n=4, k=FAKE, v=FAKE):
        return L.mxq_kv_read(fmt().ref, ref(c or cache()), slots, n, k, v, None)

    for kw, want in BAD_CACHES:
        assert read(cache(**kw)) == want, kw
    assert read(slots=0) == NULL and read(n=-1) == SHAPE and read(n=2 ** 31) == SHAPE
    assert read(k=FAKE + 8) == ALIGN and read(v=FAKE + 4) == ALIGN
    assert read(n=0, slots=0) == 0 and read(k=None, v=None) == 0


def test_attention_refusals(L):
    big = 1 << 40

    def call(c=None, f=None, q=FAKE, Hq=8, qs=(1024, 128), o=FAKE, work=FAKE, wb=big, b=None, p=None, null=()):
        batch = dict(S=2, T=4, max_q=3, max_kv=40, cu_q=FAKE, kv_len=FAKE, table=FAKE, ld_table=3, table_pages=3)
        batch.update(b or {})
        opts = dict(scale=0.1, softcap=0.0, window=0, prefix=None, slopes=None)
        opts.update(p or {})
        bb = mxq._PagedBatch(*[batch[n] for n, _ in mxq._PagedBatch._fields_])
        oo = mxq._AttnOpts(*[opts[n] for n, _ in mxq._AttnOpts._fields_])
        return L.mxq_attn_paged((f or fmt()).ref, ref(c or cache()), None if "batch" in null else ref(bb),
                                None if "opts" in null else ref(oo), q, Hq, *qs, o, 0, work, wb, None)

    cases = [(dict(c=cache(**kw)), want) for kw, want in BAD_CACHES]
    cases += [(dict(null=("batch",)), NULL), (dict(null=("opts",)), NULL), (dict(f=fmt((4, 4), 64)), SHAPE),
              (dict(q=0), NULL), (dict(o=0), NULL), (dict(q=FAKE + 8), ALIGN), (dict(o=FAKE + 8), ALIGN),
              (dict(work=FAKE + 8), ALIGN), (dict(qs=(1028, 128)), ALIGN), (dict(Hq=7), SHAPE), (dict(Hq=0), SHAPE),
              (dict(Hq=130), SHAPE), (dict(Hq=-8), SHAPE)]
    cases += [(dict(b=b), SHAPE) for b in (dict(S=-1), dict(T=-1), dict(max_q=-1), dict(max_kv=-1), dict(S=2 ** 31),
                                           dict(T=2 ** 31), dict(max_kv=2 ** 31), dict(max_q=2 ** 40),
                                           dict(table_pages=-1), dict(table_pages=2 ** 31), dict(ld_table=2),
                                           dict(T=2 ** 27), dict(S=2 ** 22))]
    cases += [(dict(b=dict(cu_q=0)), NULL), (dict(b=dict(kv_len=0)), NULL), (dict(b=dict(table=0)), NULL)]
    cases += [(dict(p=p), SHAPE) for p in (dict(scale=math.inf), dict(scale=math.nan), dict(softcap=-1.0),
                                           dict(softcap=math.inf), dict(softcap=math.nan), dict(softcap=1e-40),
                                           dict(window=-1))]
    for kw, want in cases:
        assert call(**kw) == want, kw
    for b in (dict(S=0), dict(T=0), dict(max_q=0)):
        assert call(b=b, q=0, o=0) == 0

    def work(c=None, S=2, T=4, Hq=8, max_q=3, max_kv=40):
        return L.mxq_attn_paged_work_bytes(fmt().ref, ref(c or cache()), S, T, Hq, max_q, max_kv)

    assert work() >= 0 and work(S=0) >= 0 and work(T=0) >= 0 and work(max_kv=0) >= 0
    assert work(Hq=7) == -SHAPE and work(S=-1) == -SHAPE and work(max_kv=-1) == -SHAPE
    for kw, want in BAD_CACHES:
        assert work(cache(**kw)) == -want


def test_work_size_is_what_the_call_asks_for(L):
    # one byte less is refused, for sizes that need partial results
    for S, T, Hq, max_q, max_kv in ((1, 1, 8, 1, 100000), (3, 60, 64, 20, 50000), (2, 300, 8, 200, 30000)):
        n = L.mxq_attn_paged_work_bytes(fmt().ref, ref(cache()), S, T, Hq, max_q, max_kv)
        if n == 0:
            continue
        b = mxq._PagedBatch(S, T, max_q, max_kv, FAKE, FAKE, FAKE, 3, 3)
        o = mxq._AttnOpts(0.1, 0.0, 0, None, None)
        assert L.mxq_attn_paged(fmt().ref, ref(cache()), ref(b), ref(o), FAKE, Hq, 128 * Hq, 128, FAKE, 0,
                                FAKE, n - 1, None) == SHAPE
        assert L.mxq_attn_paged(fmt().ref, ref(cache()), ref(b), ref(o), FAKE, Hq, 128 * Hq, 128, FAKE, 0,
                                None, n, None) == NULL


def test_splits_of_many_sequences_stay_in_a_dispatch(L):
    # a few rows among many sequences that are mostly empty: tiles are launched for all of them, and
    # with the splits they have to stay below 2^32 threads.  (The work size tells the splits.)
    for S, T, Hkv in ((0, 40, 1), (65536, 40, 1), (2 ** 19, 40, 8), (2 ** 22, 40, 1), (300, 40, 8)):
        c = cache(pages=100, Hkv=Hkv, page_tokens=1024)
        n = L.mxq_attn_paged_work_bytes(fmt().ref, ref(c), S, T, Hkv, 40, 65536)
        assert n >= 0
        splits = max(1, n // (4 * T * Hkv * (128 + 2)))
        assert (T // 128 + S) * Hkv * splits * 256 < 2 ** 32, (S, splits)
    assert splits > 8                                  # where there is room they are kept


# --------------------------------------------------------------------------
# the binding

class _NoLaunch:
    def __init__(self, real):
        self._real = real

    def __getattr__(self, name):
        if name in ("mxq_rope", "mxq_rope_table", "mxq_kv_append", "mxq_kv_read", "mxq_attn_paged"):
            def fail(*_a, **_k):
                raise AssertionError("%s reached a launch" % name)
            return fail
        return getattr(self._real, name)


@pytest.fixture
def host():
    """Host tensors presented as device tensors; a launch fails the test."""
    real = mxq.lib()
    with mock.patch.object(torch.Tensor, "is_cuda", new_callable=mock.PropertyMock, return_value=True), \
            mock.patch.object(mxq, "_current", lambda dev, what: None), \
            mock.patch.object(mxq, "lib", lambda path=mxq.LIB_PATH: _NoLaunch(real)):
        yield


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def test_binding_refuses_rope(host):
    x, pos, t = bf(4, 2, 128), i32(4), torch.zeros(10, 32, 2)
    for a in ((bf(4, 256), pos, t), (x.float(), pos, t), (x.transpose(1, 2), pos, t), (x, pos.long(), t),
              (x, i32(3), t), (x, i32(4, 1), t), (x, i32(8)[::2], t), (x, pos, t.double()), (x, pos, t[:, :, 0]),
              (x, pos, t.transpose(0, 1)), (x, None, t), (x, pos, None)):
        with pytest.raises(mxq.MxqError):
            mxq.rope(*a)
    for out in (bf(4, 2, 64), bf(5, 2, 128), x.float(), bf(4, 128, 2).transpose(1, 2)):
        with pytest.raises(mxq.MxqError):
            mxq.rope(x, pos, t, out=out)
    with pytest.raises(mxq.MxqError):
        mxq.rope_table(np.ones(300), 10, device="cpu")
    with pytest.raises(mxq.MxqError):
        mxq.rope_table(np.ones(4), 0, device="cpu")
    with pytest.raises(mxq.MxqError):
        mxq.rope_table(np.ones(4), 10, out=torch.zeros(79))


def test_binding_refuses_caches(host):
    f = fmt()
    with pytest.raises(mxq.MxqError):
        mxq.PagedCache(fmt((4, 4), 64), 2, 4, 16, device="cpu")
    for a in ((0, 4, 16), (2, 0, 16), (2, 4, 17), (2, 4, 8), (2, 4, 2048), (2, 2 ** 27, 16), (2, 4, 2 ** 33)):
        with pytest.raises(mxq.MxqError):
            mxq.PagedCache(f, *a, device="cpu")
    u8 = lambda n: torch.zeros(n, dtype=torch.uint8)  # noqa: E731
    n, e = 4 * 2 * 16 * 88, 4 * 2 * 16 * 4
    assert mxq.PagedCache(f, 2, 4, 16, k=(u8(n), u8(e)), v=(u8(n), u8(e))).page_bytes == n // 4
    for k in ((u8(n - 1), u8(e)), (u8(n), u8(e - 1)), (u8(n).float(), u8(e)), (u8(2 * n)[::2], u8(e))):
        with pytest.raises(mxq.MxqError):
            mxq.PagedCache(f, 2, 4, 16, k=k, v=(u8(n), u8(e)))


def test_a_cache_keeps_its_own_widths(host):
    f = fmt((4, 4, 4, 4))
    c = mxq.PagedCache(f, 2, 4, 16, device="cpu")
    f.widths[:] = 8                                    # the buffers were sized for 4 bits
    assert c.fmt.widths.tolist() == [4, 4, 4, 4]
    assert mxq.lib().mxq_kv_page_bytes(c.fmt.ref, 2, 16) == c.page_bytes
    with pytest.raises(ValueError):
        c.fmt.widths[0] = 8


def test_binding_refuses_append_and_read(host):
    c = mxq.PagedCache(fmt(), 2, 4, 16, device="cpu")
    k, slots, t = bf(5, 2, 128), torch.zeros(5, dtype=torch.int64), torch.zeros(10, 32, 2)
    for a, kw in (((bf(5, 3, 128), k, slots), {}), ((k, bf(4, 2, 128), slots), {}), ((k, bf(5, 2, 64), slots), {}),
                  ((k, k, slots.int()), {}), ((k, k, slots[:4]), {}), ((k.half(), k, slots), {}),
                  ((k, k, slots), dict(rope=t)), ((k, k, slots), dict(rope=t, pos=i32(4))),
                  ((k, k, slots), dict(q=bf(4, 8, 128))), ((k, k, slots), dict(q=bf(5, 8, 64))),
                  ((k, k, slots), dict(q=bf(5, 8, 128), q_out=bf(5, 4, 128))),
                  ((k, k, slots), dict(q=bf(5, 8, 128), q_out=bf(8, 5, 128).transpose(0, 1))),
                  ((k, k, slots), dict(q_out=bf(5, 8, 128)))):
        with pytest.raises(mxq.MxqError):
            mxq.kv_append(c, *a, **kw)
    for s, out in ((slots.int(), None), (slots.view(5, 1), None), ([1, 2], None), (slots, (k, bf(4, 2, 128))),
                   (slots, (k.float(), k)), (slots, (bf(5, 128, 2).transpose(1, 2), k))):
        with pytest.raises(mxq.MxqError):
            mxq.kv_read(c, s, out=out)


def test_binding_refuses_attention(host):
    c = mxq.PagedCache(fmt(), 2, 4, 16, device="cpu")
    good = dict(q=bf(5, 8, 128), cache=c, cu_q=i32(3), kv_len=i32(2), table=i32(2, 3), max_q=4, max_kv=40, scale=0.1)
    for bad in (dict(q=bf(5, 8, 64)), dict(q=bf(5, 1024)), dict(cu_q=i32(2)), dict(cu_q=i32(3).long()),
                dict(kv_len=i32(2, 1)), dict(kv_len=[1, 2]), dict(table=i32(3, 3)), dict(table=i32(2, 3).long()),
                dict(table=i32(3, 2).t()), dict(table=i32(6)), dict(prefix=i32(3)), dict(prefix=i32(2).float()),
                dict(slopes=torch.zeros(2)), dict(slopes=torch.zeros(8).double()), dict(out=bf(5, 8, 64)),
                dict(out=bf(5, 8, 128).half()), dict(out=bf(8, 5, 128).transpose(0, 1)), dict(dtype=torch.float16),
                dict(work=torch.zeros(64)), dict(q=bf(5, 7, 128)), dict(max_q=-1)):
        with pytest.raises(mxq.MxqError):
            mxq.attn_paged(**{**good, **bad})


def test_calls_on_another_device_are_refused():
    with mock.patch.object(torch._C, "_cuda_getDevice", lambda: 0, create=True), \
            mock.patch.object(torch._C, "_cuda_getCurrentRawStream", lambda i: 77 + i, create=True):
        assert mxq._current(torch.device("cuda:0"), "x") == 77
        with pytest.raises(mxq.MxqError, match="current device"):
            mxq._current(torch.device("cuda:1"), "x")


# --------------------------------------------------------------------------
# frequencies

def test_frequencies():
    f, ms = mxq.rope_inv_freq(8, base=10000.0)
    assert ms == 1.0 and np.allclose(f, [1, 0.1, 0.01, 0.001], rtol=1e-15)
    assert np.allclose(mxq.rope_inv_freq(8, scaling="linear", factor=4.0)[0], f / 4, rtol=1e-15)
    g, _ = mxq.rope_inv_freq(8, scaling="base", factor=5.0)
    assert g[0] == 1.0 and math.isclose(g[-1], f[-1] / 5, rel_tol=1e-12)
    assert mxq.rope_inv_freq(2, scaling="base", factor=5.0)[0].tolist() == [1.0]
    for kind, lo, hi in (("ramp", 1.0, 32.0), ("bands", 1.0, 4.0)):
        f, _ = mxq.rope_inv_freq(128, base=500000.0)
        g, ms = mxq.rope_inv_freq(128, base=500000.0, scaling=kind, factor=8.0, orig_positions=8192, low=lo, high=hi)
        turns = 8192 * f / (2 * math.pi)
        ratio = f / g
        assert np.all(ratio[turns >= hi * 1.3] == 1) and np.allclose(ratio[turns <= lo / 1.3], 8)
        assert np.all(np.diff(ratio) >= -1e-12) and 1 < ratio[np.abs(turns - (lo + hi) / 2).argmin()] < 8
        assert ms == (1.0 if kind == "bands" else 1 + 0.1 * math.log(8.0))
    # the band between: at three quarters of the way down from `high` turns to `low`
    g, _ = mxq.rope_inv_freq(128, base=500000.0, scaling="bands", factor=8.0, orig_positions=8192, low=1.0, high=4.0)
    for x, y, n in zip(f, g, turns):
        if 1 < n < 4:
            k = (n - 1) / 3
            assert math.isclose(y, x * (k + (1 - k) / 8), rel_tol=1e-12)
    # factor 1 changes nothing
    for kind in ("linear", "base", "ramp", "bands"):
        g, ms = mxq.rope_inv_freq(64, scaling=kind, factor=1.0, orig_positions=4096)
        assert ms == 1.0 and np.allclose(g, mxq.rope_inv_freq(64)[0], rtol=1e-14)
    for kw in (dict(rot=3), dict(rot=0), dict(rot=8, base=-1.0), dict(rot=8, factor=0.5),
               dict(rot=8, scaling="other"), dict(rot=8, scaling="ramp", factor=2.0),
               dict(rot=8, scaling="bands", factor=2.0, orig_positions=100, low=4.0, high=1.0),
               dict(rot=8, scaling="ramp", base=1.0, orig_positions=100)):
        with pytest.raises(mxq.MxqError):
            mxq.rope_inv_freq(**kw)


def test_scalings_without_a_result_are_refused():
    # a ramp over frequencies that rise with the index, lengths and turns that are no numbers
    ok = dict(rot=8, scaling="ramp", factor=2.0, orig_positions=100)
    assert np.isfinite(mxq.rope_inv_freq(**ok, base=1.5)[0]).all()
    for kw in (dict(base=0.5), dict(base=1.0), dict(orig_positions=math.nan), dict(orig_positions=math.inf),
               dict(high=math.inf), dict(high=math.nan), dict(low=math.nan)):
        with pytest.raises(mxq.MxqError):
            mxq.rope_inv_freq(**{**ok, **kw})
        if "base" not in kw:
            with pytest.raises(mxq.MxqError):
                mxq.rope_inv_freq(**{**ok, **kw, "scaling": "bands"})


@pytest.mark.parametrize("rot,positions", [(128, 131072), (64, 65536), (128, 4096), (128, 16384), (16, 10 ** 6)])
def test_ramp_by_its_definition(rot, positions):
    # also where the last frequency makes more than `low` turns in the trained range (2.4 and 1.4 of
    # them in the first two): the mix goes on to the index that would make `low`
    factor, low, high = 4.0, 1.0, 32.0
    g, _ = mxq.rope_inv_freq(rot, scaling="ramp", factor=factor, orig_positions=positions, low=low, high=high)

    def index(turns):                                  # positions base^(-2 i / rot) / 2 pi = turns
        return rot / 2 * math.log(positions / (2 * math.pi * turns), 10000.0)

    a, b = max(math.floor(index(high)), 0), math.ceil(index(low))
    for i in range(rot // 2):
        f = 10000.0 ** (-2.0 * i / rot)
        new = min(max((i - a) / (b - a), 0.0), 1.0)    # the share of f / factor
        assert math.isclose(g[i], f * (1 - new) + f / factor * new, rel_tol=1e-12), i
        if positions * f / (2 * math.pi) > low:
            assert g[i] > f / factor * (1 + 1e-9), i   # divided in full only from `low` turns down


# --------------------------------------------------------------------------
# the oracle's pins

def _bf16(x):
    return torch.as_tensor(x, dtype=torch.float32).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


def test_oracle_rotation_pins():
    x = np.zeros((2, 1, 4), dtype=np.float32)
    x[:, 0] = [1, 2, 3, 4]
    table = np.zeros((2, 1, 2), dtype=np.float32)
    table[0, 0] = [1, 0]
    table[1, 0] = [0, 1]                                   # a quarter turn
    for inter, turned in ((False, [-2, 1, 3, 4]), (True, [-2, 1, 3, 4])):
        y = opaged.to_f32(opaged.rope(_bf16(x), [0, 1], table, inter))
        assert y[0, 0].tolist() == [1, 2, 3, 4] and y[1, 0].tolist() == turned
    table = np.tile(np.array([[0, 1]], dtype=np.float32), (2, 2, 1))
    y = opaged.to_f32(opaged.rope(_bf16(x), [0, 5], table, False))
    assert y[0, 0].tolist() == [-3, -4, 1, 2] and np.isnan(y[1]).all()
    y = opaged.to_f32(opaged.rope(_bf16(x), [0, -1], table, True))
    assert y[0, 0].tolist() == [-2, 1, -4, 3] and np.isnan(y[1]).all()
    # against complex arithmetic in float64: half a bf16 step, and three float32 roundings
    rng = np.random.default_rng(3)
    x = opaged.to_f32(_bf16(rng.standard_normal((5, 2, 16))))
    a = rng.uniform(-50, 50, (5, 8))
    table = np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)
    y = opaged.to_f32(opaged.rope(_bf16(x), np.arange(5), table, False)).astype(np.float64)
    z = (x[..., :8].astype(np.float64) + 1j * x[..., 8:]) * np.exp(1j * a)[:, None]
    ref = np.concatenate([z.real, z.imag], -1)
    mag = np.concatenate([np.abs(z)] * 2, -1)
    assert np.all(np.abs(y - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -21 * mag)


def test_oracle_bf16_pins():
    x = torch.randn(4096, generator=torch.Generator().manual_seed(1)) * torch.exp2(
        torch.randint(-130, 120, (4096,), generator=torch.Generator().manual_seed(2)).float())
    assert np.array_equal(opaged.to_bf16(x.numpy()), _bf16(x))
    assert opaged.to_bf16(np.array([np.inf, -np.inf, np.nan], np.float32)).tolist() == [0x7F80, 0xFF80, 0xFFFF]


def test_oracle_place_covers_a_pool_once():
    for widths in ([4, 4, 4, 4], [3, 4, 6, 8], [3, 3, 6, 8]):
        Hkv, page, pages = 3, 16, 2
        row = sum(4 * m for m in widths)
        m_seen, e_seen = np.zeros(pages * Hkv * page * row, int), np.zeros(pages * Hkv * page * 4, int)
        for slot in range(pages * page):
            for h in range(Hkv):
                for b, m in enumerate(widths):
                    pm, pe = opaged.place(widths, Hkv, page, slot, h, b)
                    m_seen[pm:pm + 4 * m] += 1
                    e_seen[pe] += 1
        assert np.all(m_seen == 1) and np.all(e_seen == 1)
    # consecutive tokens of a page adjoin, block by block
    assert opaged.place([4, 4, 4, 4], 2, 16, 17, 1, 2) == ((1 * 2 + 1) * 16 * 64 + 16 * 32 + 16, (3 * 16 + 1) * 4 + 2)


def test_oracle_append_round_trip():
    widths, Hkv, page, pages = [3, 4, 6, 8], 2, 16, 2
    rng = np.random.default_rng(4)
    bits = _bf16(rng.standard_normal((7, Hkv, 128)))
    mant = np.zeros(pages * Hkv * page * 84, np.uint8)
    exp = np.zeros(pages * Hkv * page * 4, np.uint8)
    slots = [3, 31, -1, 16, 0, 32, 9]
    opaged.append(mant, exp, bits, slots, widths, Hkv, page, pages)
    ref = opaged.values(bits, widths)
    for t, s in enumerate(slots):
        if not 0 <= s < 32:
            continue
        for h in range(Hkv):
            pm, pe = opaged.place(widths, Hkv, page, s, h, 3)          # the 8-bit block, byte by byte
            got = mant[pm:pm + 32].view(np.int8) * 2.0 ** (int(exp[pe]) - 127 - 6)
            assert np.array_equal(got, ref[t, h, 96:])
            pm, pe = opaged.place(widths, Hkv, page, s, h, 1)          # the 4-bit block, nibble by nibble
            n = np.stack([mant[pm:pm + 16] & 15, mant[pm:pm + 16] >> 4], -1).reshape(-1).astype(int)
            assert np.array_equal(np.where(n > 7, n - 16, n) * 2.0 ** (int(exp[pe]) - 127 - 2), ref[t, h, 32:64])
    q, e = oracle.quantize(bits.reshape(-1, 128), widths=widths)
    d = oracle.dequantize(q, e, widths)
    assert np.array_equal(d.reshape(ref.shape), ref)


def test_oracle_attention_pins():
    rng = np.random.default_rng(5)
    k, v = rng.standard_normal((9, 2, 128)), rng.standard_normal((9, 2, 128))
    q = rng.standard_normal((3, 4, 128))
    o, a, big, bias = opaged.attention(q, k, v, 3, 0.1)
    # by brute force, with the whole score matrix and an additive mask
    for h in range(4):
        s = q[:, h] @ k[:, h // 2].T * 0.1
        s[np.arange(9)[None] > np.arange(6, 9)[:, None]] = -np.inf
        w = np.exp(s) / np.exp(s).sum(1, keepdims=True)
        assert np.allclose(o[:, h], w @ v[:, h // 2], rtol=1e-12)
        assert np.allclose(a[:, h], w @ np.abs(v[:, h // 2]), rtol=1e-12)
    assert bias == 0 and big >= np.abs(q[0, 0] @ k[0, 0]) * 0.1
    # a window of one token is that token's value; with a prefix of one, the mean of two
    o, _, _, _ = opaged.attention(q, k, v, 3, 0.0, window=1)
    assert np.allclose(o[1, 2], v[7, 1])
    o, _, _, _ = opaged.attention(q, k, v, 3, 0.0, window=1, prefix=1)
    assert np.allclose(o[1, 2], (v[7, 1] + v[0, 1]) / 2)
    # a steep bias leaves the nearest token, a tiny cap makes all weights equal
    o, _, _, bias = opaged.attention(q, k, v, 3, 0.1, slopes=[1e4] * 4)
    assert np.allclose(o[2, 0], v[8, 0]) and bias == 8e4
    o, _, _, _ = opaged.attention(q, k, v, 3, 0.1, softcap=1e-9)
    assert np.allclose(o[2, 0], v[:, 0].mean(0))
    # no visible token
    o, _, _, _ = opaged.attention(q, k[:2], v[:2], 3, 0.1)
    assert not o[0].any() and np.allclose(o[1, 0], v[0, 0])
