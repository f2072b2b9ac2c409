"""Host-side checks of the attention side that need no GPU: frequencies, index arithmetic, refusals before any launch."""
import ctypes
import math
import os

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def hbl():
    from paper_2504_18415_amd import hbl as H
    if not os.path.exists(H.LIB_PATH):
        from paper_2504_18415_amd import build
        build.build_library()
    H.lib()
    return H


def test_frequencies(hbl):
    f = hbl.rope_frequencies(128, device="cpu")
    assert f.dtype == torch.float32 and f.shape == (64,) and f[0] == 1.0
    for i in range(64):
        assert abs(float(f[i]) - 10000.0 ** (-i / 64)) <= 2.0 ** -23 * float(f[i])
    assert torch.equal(hbl.rope_frequencies(128, scaling="linear", factor=4.0, device="cpu"), f / 4)
    b = hbl.rope_frequencies(128, scaling="base", factor=4.0, device="cpu")
    assert b[0] == 1.0 and abs(float(b[-1]) * 4 / float(f[-1]) - 1) < 1e-6   # the slowest pair slows by the factor
    p = hbl.rope_frequencies(128, scaling="parts", factor=8.0, trained_len=8192, slow=1.0, fast=4.0, device="cpu")
    for i in range(64):
        turns = 8192 * 10000.0 ** (-i / 64) / (2 * math.pi)
        g = min(1.0, max(0.0, (turns - 1) / 3))
        want = 10000.0 ** (-i / 64) * (g + (1 - g) / 8)
        assert abs(float(p[i]) - want) <= 2.0 ** -22 * want
    assert p[0] == f[0] and abs(float(p[-1]) * 8 / float(f[-1]) - 1) < 1e-6
    for bad in (dict(rot_dim=3), dict(rot_dim=2), dict(rot_dim=514), dict(base=1.0), dict(base=float("nan")), dict(factor=0.5),
                dict(scaling="parts", trained_len=0.0), dict(scaling="parts", trained_len=1.0, slow=2.0, fast=2.0)):
        with pytest.raises(hbl.HblError) as e:
            hbl.rope_frequencies(**{"rot_dim": 64, "device": "cpu", **bad})
        assert e.value.status == hbl.E_SHAPE
    with pytest.raises(ValueError):
        hbl.rope_frequencies(64, scaling="other", device="cpu")


def rows_of(hbl, starts, lens, table, T, seq, n, n_pages=10, page=16, heads=2, page_rows=None, width=None):
    starts, lens = (ctypes.c_int32 * len(starts))(*starts), (ctypes.c_int32 * len(lens))(*lens)
    stride = len(table[0])
    flat = (ctypes.c_int32 * (len(table) * stride))(*[e for r in table for e in r])
    cache = hbl._Cache(0, 0, 0, 0, n_pages, page_rows or heads * page, 16, page, heads, 64)
    at = lambda a: ctypes.cast(a, ctypes.c_void_p)
    batch = hbl._Batch(at(starts), at(lens), at(flat), stride, len(lens), stride if width is None else width)
    rows, span = (ctypes.c_int64 * n)(), (ctypes.c_int * 4)()
    assert hbl.lib().hbl_test_kv_rows(ctypes.byref(cache), ctypes.byref(batch), T, seq, rows, n, span) == 0
    return list(span), list(rows)


def test_rows_and_pages_that_are_not_there(hbl):
    big = 2 ** 31 - 1
    table = [[3, 9, -1, 10], [big, -big - 1, 0, 5]]
    span, rows = rows_of(hbl, [0, 4, 6], [60, 70], table, 6, 0, 64)
    assert span == [0, 4, 60, 60]
    assert rows[:16] == [3 * 32 + 16 + i for i in range(16)] and rows[16:32] == [9 * 32 + 16 + i for i in range(16)]
    assert rows[32:60] == [-1] * 28 and rows[60:] == [-2] * 4
    span, rows = rows_of(hbl, [0, 4, 6], [60, 70], table, 6, 1, 70)
    assert span == [4, 2, 64, 70]                       # the table ends before the length does
    assert rows[:32] == [-1] * 32 and rows[32] == 16 and rows[63] == 5 * 32 + 31 and rows[64:] == [-2] * 6
    # rows beyond 32 bits
    span, rows = rows_of(hbl, [0, 1], [2], [[9]], 1, 0, 2, page_rows=1 << 30)
    assert rows == [9 * (1 << 30) + 16, 9 * (1 << 30) + 17]
    # starts that make no sense stay inside the call's tokens
    for starts, want in (([5, 2], [5, 0]), ([-7, 3], [0, 3]), ([4, 100], [4, 4]), ([big, big], [8, 0]), ([-big - 1, -5], [0, 0])):
        span, _ = rows_of(hbl, starts, [-3], [[0]], 8, 0, 1)
        assert span == want + [0, 0]


def test_visible_keys(hbl):
    lo, hi = ctypes.c_int(), ctypes.c_int()

    def see(*a):
        assert hbl.lib().hbl_test_visible_keys(*a, ctypes.byref(lo), ctypes.byref(hi)) == 0
        return lo.value, hi.value

    for p in (-3, 0, 1, 7, 40):
        for keys in (0, 1, 8, 30):
            for window in (0, 1, 5, 2 ** 31 - 1):
                for prefix in (0, 3, 100, -4, 2 ** 31 - 1):
                    want = [j for j in range(keys) if p >= 0 and (j <= p or j < prefix) and (window == 0 or j > p - window)]
                    a, b = see(p, keys, window, prefix)
                    assert list(range(a, b)) == want, (p, keys, window, prefix)
    assert see(2 ** 31 - 2, 2 ** 31 - 1, 2, 0) == (2 ** 31 - 3, 2 ** 31 - 1)


def test_refusals_before_any_launch(hbl):
    """Every refused argument, on pointers that no kernel could follow."""
    L, B = hbl.lib(), ctypes.byref
    ok, null = ctypes.c_void_p(4096), None

    def cache(**kw):
        c = dict(k=4096, v=4096, k_scales=4096, v_scales=4096, n_pages=4, page_rows=64, bits=16, page_size=16, n_kv_heads=4, d=64)
        return hbl._Cache(*{**c, **kw}.values())

    def batch(**kw):
        b = dict(q_starts=4096, kv_lens=4096, block_table=4096, table_stride=4, n_seqs=2, table_width=4)
        return hbl._Batch(*{**b, **kw}.values())

    def rope(x=ok, dt=1, T=4, H=2, d=64, xs=128, pos=ok, fr=ok, rot=32, layout=0, out=ok, odt=1, os_=128):
        return L.hbl_rope(x, dt, T, H, d, xs, pos, fr, rot, layout, 1.0, 0, out, odt, os_, None)

    S, N, D, A, BI = hbl.E_SHAPE, hbl.E_NULL, hbl.E_DTYPE, hbl.E_ALIGN, hbl.E_BITS
    for kw, want in ((dict(T=0), 0), (dict(dt=2), D), (dict(odt=-1), D), (dict(T=-1), S), (dict(T=(1 << 24) + 1), S), (dict(H=0), S),
                     (dict(d=72, xs=144), S), (dict(d=528, H=1, xs=528), S), (dict(rot=0), S), (dict(rot=24), S), (dict(rot=80), S),
                     (dict(layout=2), S), (dict(xs=127), S), (dict(os_=64), S), (dict(x=null), N), (dict(out=null), N), (dict(pos=null), N),
                     (dict(fr=null), N), (dict(x=ctypes.c_void_p(4104)), A), (dict(xs=132), A), (dict(out=ctypes.c_void_p(4098)), A),
                     (dict(odt=0), S), (dict(os_=136), S)):   # (the last two: in place, but not the same layout)
        assert rope(**kw) == want, kw

    def append(c=None, b=None, k=ok, ks=256, v=ok, vs=256, dt=1, T=4, q=null, Hq=0, qs=0, qo=null, qdt=1, qos=0, fr=ok, rot=32, layout=0):
        return L.hbl_kv_append(B(c or cache()), B(b or batch()), k, ks, v, vs, dt, T, q, Hq, qs, qo, qdt, qos, fr, rot, layout, 1.0, 1e-5, None)

    shapes = [(dict(c=cache(bits=5)), BI), (dict(c=cache(d=32)), S), (dict(c=cache(d=512)), S), (dict(c=cache(page_size=24)), S),
              (dict(c=cache(page_size=8)), S), (dict(c=cache(page_size=2048, page_rows=8192)), S), (dict(c=cache(n_kv_heads=0)), S),
              (dict(c=cache(page_rows=63)), S), (dict(c=cache(n_pages=-1)), S), (dict(c=cache(n_pages=1 << 31)), S),
              (dict(c=cache(n_pages=1 << 20, page_rows=1 << 20)), S), (dict(c=cache(k=0)), N), (dict(c=cache(v=None)), N),
              (dict(c=cache(bits=8, k_scales=None)), N), (dict(c=cache(k=4100)), A), (dict(b=batch(n_seqs=-1)), S), (dict(b=batch(n_seqs=0)), 0),
              (dict(b=batch(table_width=5)), S), (dict(b=batch(q_starts=None)), N), (dict(b=batch(kv_lens=None)), N), (dict(b=batch(block_table=None)), N),
              (dict(T=0), 0), (dict(T=-1), S), (dict(T=(1 << 24) + 1), S)]
    for kw, want in shapes + [(dict(dt=7), D), (dict(k=null), N), (dict(v=null), N), (dict(ks=255), S), (dict(vs=260), A), (dict(rot=80), S), (dict(rot=8), S),
                              (dict(layout=-1), S), (dict(q=ok, Hq=0), S), (dict(q=ok, Hq=4, qs=256, qos=256), N), (dict(q=ok, Hq=4, qs=256, qo=ok, qdt=3), D),
                              (dict(q=ok, Hq=4, qs=128, qo=ok, qos=256), S), (dict(q=ok, Hq=4, qs=256, qo=ok, qos=512), S),
                              (dict(q=ok, Hq=4, qs=256, qo=ok, qos=256, qdt=0), S)]:
        assert append(**kw) == want, kw
    assert L.hbl_kv_append(None, B(batch()), ok, 256, ok, 256, 1, 4, None, 0, 0, None, 1, 0, None, 0, 0, 1.0, 1e-5, None) == N
    assert L.hbl_kv_append(B(cache()), None, ok, 256, ok, 256, 1, 4, None, 0, 0, None, 1, 0, None, 0, 0, 1.0, 1e-5, None) == N

    def attend(c=None, b=None, q=ok, T=4, Hq=8, qs=512, m=1, scale=0.1, cap=0.0, window=0, out=ctypes.c_void_p(1 << 20), os_=512, ws=ok, wb=1 << 40):
        return L.hbl_paged_attention(q, T, Hq, qs, B(c or cache()), B(b or batch()), m, scale, cap, window, None, None, out, os_, ws, wb, None)

    for kw, want in shapes + [(dict(b=batch(n_seqs=1 << 20, table_width=1 << 14, table_stride=1 << 14)), S), (dict(T=1 << 24, Hq=128, qs=8192, os_=8192), S), (dict(Hq=6), S), (dict(Hq=0), S), (dict(m=0), S), (dict(window=-1), S), (dict(window=1 << 31), S), (dict(cap=-1.0), S), (dict(cap=1e-7), S), (dict(out=ok), S),
                              (dict(cap=float("nan")), S), (dict(cap=float("inf")), S), (dict(scale=float("nan")), S), (dict(scale=float("inf")), S),
                              (dict(q=null), N), (dict(out=null), N), (dict(ws=null), N), (dict(qs=511), S), (dict(os_=516), A),
                              (dict(q=ctypes.c_void_p(4097)), A), (dict(ws=ctypes.c_void_p(4096 + 128)), A), (dict(wb=16), hbl.E_WORKSPACE)]:
        assert attend(**kw) == want, kw
    size = lambda c, b, T, Hq, m: L.hbl_paged_attention_workspace_bytes(B(c), B(b), T, Hq, m)
    assert size(cache(), batch(), 4, 8, 1) >= 256 and size(cache(), batch(), 4, 8, 1) % 256 == 0
    assert size(cache(), batch(), 4, 6, 1) == 0 and size(cache(bits=7), batch(), 4, 8, 1) == 0 and size(cache(), batch(n_seqs=-1), 4, 8, 1) == 0


def test_binding_refuses_host_tensors(hbl):
    x = torch.zeros((2, 2, 64))
    with pytest.raises(ValueError):
        hbl.rope(x, torch.zeros(2, dtype=torch.int32), torch.zeros(32))
    with pytest.raises(ValueError):
        hbl.KvCache(torch.zeros((2, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((2, 2, 16, 64), dtype=torch.bfloat16))
