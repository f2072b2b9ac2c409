"""GPU tests of rotary positions, the paged cache's append and paged attention, against their definitions in 64 bits
(paged_reference.py), through the Python binding."""
import math

import pytest

torch = pytest.importorskip("torch")

import paged_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hbl():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2504_18415_amd import hbl as H
    H.lib()
    return H


def note(text):
    print("[gpu-case] " + text, flush=True)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# --- rotary positions -------------------------------------------------------------------------------------------

ROPE = [  # T, H, d, rot, extra stride
    (1, 1, 64, 64, 0), (1, 32, 128, 128, 0), (7, 3, 80, 32, 16), (33, 8, 128, 64, 128), (5, 12, 16, 16, 0), (130, 2, 256, 256, 0),
    (3, 5, 512, 512, 0), (257, 1, 16, 16, 0), (64, 7, 96, 48, 8 * 96), (1000, 4, 64, 32, 0), (18, 1, 512, 16, 0)]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype,out_dtype", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32),
                                             (torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("T,H,d,rot,extra", ROPE)
def test_rope(hbl, T, H, d, rot, extra, dtype, out_dtype, layout):
    note(f"rope T={T} H={H} d={d} rot={rot} extra={extra} {dtype}->{out_dtype} {layout}")
    g = gen(T * 131 + d)
    rows = torch.randn((T, H * d + extra), generator=g).to(dtype).cuda()
    x = rows[:, extra // 2:extra // 2 + H * d].unflatten(-1, (H, d))
    positions = torch.randint(0, 1 << 20, (T,), generator=g).to(torch.int32).cuda()
    positions[0] = 0
    positions[-1] = -12345 if T > 2 else 2 ** 31 - 1
    freqs = R.frequencies(rot).cuda()
    for backward in (False, True):
        m = 1.25 if backward else 1.0
        y = hbl.rope(x, positions, freqs, layout=layout, magnitude=m, backward=backward, out_dtype=out_dtype)
        want = R.rotate(x, positions, freqs, layout, m, backward)
        tol = R.rotate_bound(x, freqs, layout, m) + (want.abs() * R.U16 * 1.001 if out_dtype == torch.bfloat16 else 0.0)
        assert y.dtype == out_dtype and ((y.double() - want).abs() <= tol).all()
        if T > 2:
            assert torch.equal(y[0, :, rot:].float(), x[0, :, rot:].to(out_dtype).float())


def test_rope_and_append_of_outputs_beyond_l2(hbl):
    """Outputs of more than 32 MiB leave by other stores: the same values as in parts that do not."""
    note("rope and append, large outputs")
    T, H, d = 5000, 32, 128
    x = torch.randn((T, H, d), generator=gen(2)).bfloat16().cuda()
    positions, freqs = torch.arange(T, dtype=torch.int32, device="cuda"), R.frequencies(d).cuda()
    for layout in ("half", "interleaved"):
        parts = [hbl.rope(x[i:i + 1000], positions[i:i + 1000], freqs, layout=layout) for i in range(0, T, 1000)]
        assert torch.equal(hbl.rope(x, positions, freqs, layout=layout).view(torch.int16), torch.cat(parts).view(torch.int16))
        cache = hbl.KvCache.empty(80, 1, 64, d)
        q = hbl.kv_append(cache, x[:, :1], x[:, 1:2], ints([0, T]), ints([T]), ints([list(range(80))]), freqs=freqs, layout=layout, q=x)
        assert torch.equal(q.view(torch.int16), torch.cat(parts).view(torch.int16))


def test_rope_in_place_in_a_fused_output(hbl):
    """Queries and keys turned where the projection left them; values and what lies beside untouched."""
    note("rope in place")
    T, H, d = 37, 4, 64
    qkv = torch.randn((T, 3 * H * d), generator=gen(3)).bfloat16().cuda()
    before, positions, freqs = qkv.clone(), torch.arange(T, dtype=torch.int32, device="cuda") + 100, R.frequencies(d).cuda()
    for part in (0, 1):
        x = qkv[:, part * H * d:(part + 1) * H * d].unflatten(-1, (H, d))
        assert hbl.rope(x, positions, freqs, out=x).data_ptr() == x.data_ptr()
    want = hbl.rope(before[:, :2 * H * d].unflatten(-1, (2 * H, d)), positions, freqs)
    assert torch.equal(qkv[:, :2 * H * d].view(torch.int16), want.flatten(1).view(torch.int16))
    assert torch.equal(qkv[:, 2 * H * d:], before[:, 2 * H * d:])


def test_rope_backward_is_the_gradient(hbl):
    """<rope(x), g> and <x, backward(g)> agree, and differences of the forward map give the same."""
    note("rope gradient")
    T, H, d, rot = 9, 2, 64, 32
    g0 = gen(11)
    x, g = (torch.randn((T, H, d), generator=g0).cuda() for _ in range(2))
    positions, freqs = torch.arange(T, dtype=torch.int32, device="cuda") * 1001, R.frequencies(rot).cuda()
    for layout in ("half", "interleaved"):
        y = hbl.rope(x, positions, freqs, layout=layout, magnitude=0.75)
        dx = hbl.rope(g, positions, freqs, layout=layout, magnitude=0.75, backward=True)
        a, b = (y.double() * g.double()).sum(), (x.double() * dx.double()).sum()
        slack = (R.rotate_bound(x, freqs, layout, 0.75) * g.abs()).sum() + (R.rotate_bound(g, freqs, layout, 0.75) * x.abs()).sum()
        assert (a - b).abs() <= slack
        step = torch.zeros_like(x)
        step[4, 1, 3] = 1.0   # the map is linear: one step gives a column of it
        column = hbl.rope(step, positions, freqs, layout=layout, magnitude=0.75)
        tol = (R.rotate_bound(step, freqs, layout, 0.75) * g.abs()).sum() + R.rotate_bound(g, freqs, layout, 0.75)[4, 1, 3]
        assert ((column.double() * g.double()).sum() - dx[4, 1, 3].double()).abs() <= tol


# --- append -----------------------------------------------------------------------------------------------------

APPEND = [  # new tokens, lengths, Hq, Hkv, page
    ([1], [1], 1, 1, 16), ([1, 1, 1], [5, 64, 65], 8, 2, 16), ([130], [130], 4, 4, 64), ([0, 7, 0, 33, 1], [9, 7, 0, 100, 3], 6, 2, 32),
    ([1] * 70, list(range(1, 71)), 2, 1, 16), ([5, 4], [3, 4], 3, 3, 128)]   # (the last: two tokens before the first position)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bits", [16, 8, 4, 3])
@pytest.mark.parametrize("d,rot", [(64, 32), (128, 128), (256, 64)])
@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append(hbl, case, d, rot, bits, dtype, layout):
    new, lens, Hq, Hkv, page = APPEND[case]
    note(f"append case={case} d={d} rot={rot} bits={bits} {dtype} {layout}")
    g = gen(case * 7 + bits)
    T = sum(new) + 2   # two tokens behind the last sequence
    qkv = torch.randn((T, (Hq + 2 * Hkv) * d), generator=g).to(dtype).cuda()
    q, k, v = (p.unflatten(-1, (-1, d)) for p in qkv.split((Hq * d, Hkv * d, Hkv * d), -1))
    table, n_pages = R.page_table(g, lens, page, spare=2)
    (kp, ks), (vp, vs) = (R.random_pages(g, n_pages, Hkv, page, d, bits, "cuda") for _ in range(2))
    was = [None if t is None else t.clone() for t in (kp, vp, ks, vs)]
    cache = hbl.KvCache(kp, vp, bits, ks, vs)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    freqs = R.frequencies(rot).cuda()
    q_out = torch.full((T, Hq, d), 7.0, dtype=dtype, device="cuda")
    got = hbl.kv_append(cache, k, v, ints(starts), ints(lens), table.cuda(), freqs=freqs, layout=layout, q=q, q_out=q_out)
    assert got is q_out
    # once more, the queries where they are: the same rows again
    own = qkv.clone()[:, :Hq * d].unflatten(-1, (Hq, d))
    hbl.kv_append(cache, k, v, ints(starts), ints(lens), table.cuda(), freqs=freqs, layout=layout, q=own, q_out=own)
    assert torch.equal(own[:starts[-1]], q_out[:starts[-1]]) and torch.equal(own[starts[-1]:], q[starts[-1]:])
    torch.cuda.synchronize()
    position = torch.zeros(T, dtype=torch.int32)
    where = []
    for s, n in enumerate(new):
        for i in range(n):
            p = lens[s] - n + i
            position[starts[s] + i] = p
            if p >= 0:
                where.append((starts[s] + i, int(table[s, p // page]), p % page))
    # what rope and kv_quant_absmax give, bit for bit
    live = starts[-1]
    k32 = hbl.rope(k, position.cuda(), freqs, layout=layout, out_dtype=torch.float32)
    want_q = hbl.rope(q, position.cuda(), freqs, layout=layout)
    assert torch.equal(q_out[:live], want_q[:live]) and (q_out[live:] == 7.0).all()
    want = [None if t is None else t.clone() for t in was]
    for side, x in ((0, k32), (1, v.float())):
        if bits == 16:
            rows, scales = x.bfloat16(), None
        else:
            rows, scales = hbl.kv_quant_absmax(x.contiguous().view(T * Hkv, d), bits)
            rows, scales = rows.view(T, Hkv, -1), scales.view(T, Hkv)
        for t, p, slot in where:
            want[side][p, :, slot] = rows[t]
            if bits != 16:
                want[2 + side][p, :, slot] = scales[t]
    for a, b in zip((kp, vp, ks, vs), want):   # every other row as it was
        assert a is None or torch.equal(a.view(torch.int16) if a.dtype == torch.bfloat16 else a, b.view(torch.int16) if b.dtype == torch.bfloat16 else b)


def test_append_without_rotation_queries_or_pages(hbl):
    note("append: no rotation, entries that name no page, a table that ends early, an interleaved pool")
    d, page, H = 64, 16, 2
    pool = torch.zeros((6, 2, H, page, d), dtype=torch.bfloat16, device="cuda")   # keys and values side by side
    cache = hbl.KvCache(pool[:, 0], pool[:, 1])
    k, v = (torch.randn((60, H, d), generator=gen(5)).bfloat16().cuda() for _ in range(2))
    table = ints([[3, -1, 6, 0], [2 ** 31 - 1, 4, 1, 5]])[:, :3]
    # sequence 0: 30 tokens at 20..49: slots 4.. of no page, of a page that is not there (6), beyond the table's three pages
    assert hbl.kv_append(cache, k, v, ints([0, 30, 60]), ints([50, 47]), table) is None
    torch.cuda.synchronize()
    want = torch.zeros_like(pool)
    for i in range(30):   # sequence 1: tokens at 17..46
        p = 17 + i
        if p // page < 3 and [None, 4, 1][p // page] is not None:
            want[[None, 4, 1][p // page], 0, :, p % page], want[[None, 4, 1][p // page], 1, :, p % page] = k[30 + i], v[30 + i]
    assert torch.equal(pool, want)


# --- attention --------------------------------------------------------------------------------------------------

def check_attention(hbl, new, lens, Hq, Hkv, d, bits, page, seed=0, tail=0, pad_table=0, table_edit=None, q_scale=2.0, max_q_len=None,
                    **options):
    g = gen(seed + 1000 * bits + d)
    T = sum(new) + tail
    table, n_pages = R.page_table(g, lens, page, spare=1, width=pad_table)
    if table_edit is not None:
        table_edit(table)
    (kp, ks), (vp, vs) = (R.random_pages(g, n_pages, Hkv, page, d, bits, "cuda") for _ in range(2))
    vp = vp if bits != 16 else (vp.float() + 0.5).bfloat16()
    # fused layout: the queries are a slice of wider rows
    q = (q_scale * torch.randn((T, (Hq + 2) * d), generator=g)).bfloat16().cuda()[:, d:-d].unflatten(-1, (Hq, d))
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    slopes, prefix = options.get("slopes"), options.get("prefix_lens")
    cache = hbl.KvCache(kp, vp, bits, ks, vs)
    out = torch.full((T, Hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
    kw = {**options, "slopes": None if slopes is None else torch.tensor(slopes, device="cuda"), "prefix_lens": None if prefix is None else ints(prefix)}
    got = hbl.paged_attention(q, cache, ints(starts), ints(lens), table.cuda(), max_q_len or max(max(new, default=1), 1), out=out, **kw)
    assert got is out
    torch.cuda.synchronize()
    kw["prefix_lens"] = prefix
    scale = kw.pop("scale", None)
    want, bound = R.attention(q, kp, vp, ks, vs, bits, starts, lens, table.tolist(), d ** -0.5 if scale is None else scale,
                              **{k: v for k, v in kw.items() if k in ("softcap", "window", "slopes", "prefix_lens")})
    live = starts[-1]
    error = (out[:live].double() - want[:live]).abs()
    tol = bound[:live] + (want[:live].abs() + bound[:live]) * R.U16 * 1.001
    assert torch.isfinite(out.float()).all()
    worst = (error - tol).max() if live else torch.tensor(0.0)
    assert (error <= tol).all(), f"worst excess {float(worst):.3e}, largest error {float(error.max()):.3e}"
    assert (out[live:] == 7.0).all()
    return out


DECODE = [  # new, lens, Hq, Hkv, page
    ([1], [1], 1, 1, 16), ([1], [17], 2, 1, 16), ([1, 1], [33, 1000], 8, 2, 64), ([1] * 5, [1, 15, 16, 31, 32], 4, 4, 16),
    ([1, 0, 1, 1], [64, 10, 0, 700], 32, 8, 128), ([1], [4097], 7, 1, 32), ([2, 3, 1], [2, 259, 600], 8, 4, 64),
    ([1, 4], [2500, 4], 16, 2, 256), ([1] * 3, [130, 65, 300], 64, 2, 1024), ([1] * 40, [37 * i + 1 for i in range(40)], 4, 2, 64)]


@pytest.mark.parametrize("bits", [16, 8, 4, 3])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("case", range(len(DECODE)))
def test_attention_decode(hbl, case, d, bits):
    new, lens, Hq, Hkv, page = DECODE[case]
    note(f"attention decode case={case} d={d} bits={bits}")
    check_attention(hbl, new, lens, Hq, Hkv, d, bits, page, seed=case, tail=case % 3)


CHUNK = [  # new, lens, Hq, Hkv, page
    ([33], [33], 2, 2, 16), ([64], [64], 4, 2, 64), ([65, 1], [130, 77], 4, 1, 16), ([200], [1000], 2, 1, 128), ([17, 90, 0, 3], [17, 300, 5, 4], 3, 3, 32),
    ([257], [300], 5, 1, 64), ([40, 300], [30, 300], 2, 2, 16), ([128], [2100], 8, 8, 256), ([511], [511], 1, 1, 1024)]


@pytest.mark.parametrize("bits", [16, 8, 4, 3])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("case", range(len(CHUNK)))
def test_attention_chunk(hbl, case, d, bits):
    new, lens, Hq, Hkv, page = CHUNK[case]
    note(f"attention chunk case={case} d={d} bits={bits}")
    check_attention(hbl, new, lens, Hq, Hkv, d, bits, page, seed=50 + case, tail=case % 2)


OPTIONS = [
    dict(softcap=30.0), dict(softcap=1.5, scale=0.3), dict(window=1), dict(window=100), dict(slopes=True), dict(prefix_lens=[70, 3, 0]),
    dict(prefix_lens=[1000, 1000, 2], window=50), dict(softcap=20.0, window=333, slopes=True, prefix_lens=[0, 5, 9]), dict(scale=0.0),
    dict(scale=-0.05), dict(softcap=55.0), dict(slopes=True, prefix_lens=[300, 0, 4], window=120)]


@pytest.mark.parametrize("bits,d", [(16, 128), (4, 64), (8, 256), (3, 128)])
@pytest.mark.parametrize("new,lens", [([1, 1, 1], [500, 1, 77]), ([50, 130, 1], [400, 130, 9])])
@pytest.mark.parametrize("option", range(len(OPTIONS)))
def test_attention_options(hbl, option, new, lens, bits, d):
    note(f"attention option={option} new={new} bits={bits} d={d}")
    kw = dict(OPTIONS[option])
    if kw.get("slopes"):
        kw["slopes"] = [2.0 ** (-i - 1) for i in range(4)]
    check_attention(hbl, new, lens, 4, 2, d, bits, 32, seed=90 + option, **kw)


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("new", [[1, 1, 1], [60, 70, 80]])
def test_attention_with_pages_that_are_not_there(hbl, new, bits):
    """Entries that name no page leave their keys out; a row that sees nothing else gets zeros."""
    note(f"attention: absent pages new={new} bits={bits}")

    def edit(table):
        table[0, :] = -1                       # nothing at all
        table[1, 0] = 2 ** 31 - 1
        table[1, 2] = -2 ** 31
        table[2, 3:] = 10 ** 6

    check_attention(hbl, new, [100, 300, 200], 4, 2, 128, bits, 32, seed=7, table_edit=edit)
    check_attention(hbl, new, [100, 300, 200], 4, 2, 128, bits, 32, seed=8, table_edit=edit, window=20)


def test_attention_lengths_beyond_the_table(hbl):
    note("attention: lengths beyond the table")
    g = gen(4)
    (kp, _), (vp, _) = (R.random_pages(g, 4, 1, 16, 64, 16, "cuda") for _ in range(2))
    q = torch.randn((5, 2, 64), generator=g).bfloat16().cuda()
    table = ints([[0, 1], [2, 3]])
    starts, lens = [0, 2, 5], [90, 32]
    out = hbl.paged_attention(q, hbl.KvCache(kp, vp), ints(starts), ints(lens), table, 3)
    want, bound = R.attention(q, kp, vp, None, None, 16, starts, lens, table.tolist(), 64 ** -0.5)
    assert ((out.double() - want).abs() <= bound + (want.abs() + bound) * R.U16 * 1.001).all()


@pytest.mark.parametrize("bits", [16, 8, 4, 3])
@pytest.mark.parametrize("new,lens", [([1, 1], [90, 300]), ([70, 40], [90, 300])])
def test_what_masked_places_hold_does_not_count(hbl, new, lens, bits):
    """NaN and infinities behind the last key, in pages of nobody and in scales of unused slots leave no trace."""
    note(f"attention: NaN in masked places new={new} bits={bits}")
    d, page, H = 128, 64, 2
    g = gen(12)
    table, n_pages = R.page_table(g, lens, page, spare=2)
    (kp, ks), (vp, vs) = (R.random_pages(g, n_pages, H, page, d, bits, "cuda") for _ in range(2))
    q = torch.randn((sum(new), 4, d), generator=g).bfloat16().cuda()
    starts = ints([0, new[0], sum(new)])
    args = (starts, ints(lens), table.cuda(), max(new))
    clean = hbl.paged_attention(q, hbl.KvCache(kp, vp, bits, ks, vs), *args)
    used = torch.zeros((n_pages, page), dtype=torch.bool)
    for s, n in enumerate(lens):
        for j in range(n):
            used[int(table[s, j // page]), j % page] = True
    for t in (kp, vp, ks, vs):
        if t is not None and t.dtype != torch.uint8:
            m = (~used).cuda()[:, None, :].expand(n_pages, H, page)
            for i, bad in enumerate((float("nan"), float("inf"), -float("inf"))):
                pick = m & ((torch.arange(page, device="cuda") % 3) == i)
                t[pick] = bad
    dirty = hbl.paged_attention(q, hbl.KvCache(kp, vp, bits, ks, vs), *args)
    assert torch.equal(clean.view(torch.int16), dirty.view(torch.int16))


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new", [1, 64])
def test_attention_of_large_scores(hbl, new, bits):
    """Scores of thousands: one key takes all, and nothing overflows."""
    note(f"attention: large scores new={new} bits={bits}")
    check_attention(hbl, [new, new], [300, 400], 4, 2, 128, bits, 32, seed=3, q_scale=512.0)


@pytest.mark.parametrize("bits", [8, 4, 3])
def test_attention_of_scales_far_apart(hbl, bits):
    """Rows of zeros (scale 0), tiny and huge scales of values side by side."""
    note(f"attention: scales far apart bits={bits}")
    d, page, H = 64, 16, 1
    g = gen(21)
    lens, new = [200, 33], [40, 1]
    table, n_pages = R.page_table(g, lens, page)
    (kp, ks), (vp, vs) = (R.random_pages(g, n_pages, H, page, d, bits, "cuda") for _ in range(2))
    vs[:, :, 0::4] = 0.0
    vs[:, :, 1::4] *= 1e-20
    vs[:, :, 2::4] *= 1e20
    ks[:, :, 3::5] = 0.0
    q = torch.randn((41, 2, d), generator=g).bfloat16().cuda()
    out = hbl.paged_attention(q, hbl.KvCache(kp, vp, bits, ks, vs), ints([0, 40, 41]), ints(lens), table.cuda(), 40)
    want, bound = R.attention(q, kp, vp, ks, vs, bits, [0, 40, 41], lens, table.tolist(), d ** -0.5)
    assert ((out.double() - want).abs() <= bound + (want.abs() + bound) * R.U16 * 1.001).all()


def test_attention_same_bits_every_time(hbl):
    """No result depends on the order in which workgroups finish, nor on what the workspace held."""
    note("attention: repeated")
    g = gen(31)
    lens, new, d, page = [3000, 800, 1], [1, 1, 1], 128, 64
    table, n_pages = R.page_table(g, lens, page)
    (kp, _), (vp, _) = (R.random_pages(g, n_pages, 4, page, d, 16, "cuda") for _ in range(2))
    cache, q = hbl.KvCache(kp, vp), torch.randn((3, 8, d), generator=g).bfloat16().cuda()
    args = (ints([0, 1, 2, 3]), ints(lens), table.cuda(), 1)
    n = hbl.paged_attention_workspace_bytes(cache, 3, 3, 8, 1)
    first = hbl.paged_attention(q, cache, *args)
    for fill in (0, 255, 127):
        again = hbl.paged_attention(q, cache, *args, workspace=torch.full((n,), fill, dtype=torch.uint8, device="cuda"))
        assert torch.equal(first.view(torch.int16), again.view(torch.int16))


MANY = [100, 300]


@pytest.mark.parametrize("S", MANY)
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("chunk", [False, True])
def test_attention_of_many_sequences(hbl, S, bits, chunk):
    """More sequences than a wave, and than a workgroup, has lanes; empty ones among them."""
    note(f"attention: {S} sequences bits={bits} chunk={chunk}")
    new = [(i * 7 % 5 if i % 9 else 40) if chunk else int(i % 10 != 3) for i in range(S)]
    lens = [n + (i * 37) % 90 for i, n in enumerate(new)]
    check_attention(hbl, new, lens, 4, 2, 64, bits, 16, seed=S, tail=1)


@pytest.mark.parametrize("bits", [16, 8])
def test_attention_with_more_row_tiles_than_are_cut(hbl, bits):
    note(f"attention: whole row tiles bits={bits}")
    check_attention(hbl, [1500], [1600], 128, 128, 64, bits, 64, seed=5)


@pytest.mark.parametrize("new", [1, 3, 200])
def test_tokens_beyond_max_q_len_stay(hbl, new):
    note(f"attention: max_q_len smaller than a sequence's {new}")
    d, page = 64, 16
    g = gen(81)
    lens = [new + 60, 30]
    table, n = R.page_table(g, lens, page)
    (kp, _), (vp, _) = (R.random_pages(g, n, 2, page, d, 16, "cuda") for _ in range(2))
    q = torch.randn((new + 1, 4, d), generator=g).bfloat16().cuda()
    starts, most = [0, new, new + 1], max(1, new - 2)
    out = torch.full_like(q, 7.0)
    hbl.paged_attention(q, hbl.KvCache(kp, vp), ints(starts), ints(lens), table.cuda(), most, out=out)
    want, bound = R.attention(q, kp, vp, None, None, 16, starts, lens, table.tolist(), d ** -0.5)
    seen = torch.ones(new + 1, dtype=torch.bool, device="cuda")
    seen[most:new] = False
    assert ((out.double() - want).abs() <= bound + (want.abs() + bound) * R.U16 * 1.001)[seen].all() and (out[~seen] == 7.0).all()


@pytest.mark.parametrize("bits", [16, 8, 4, 3])
@pytest.mark.parametrize("new", [1, 70])
def test_pools_side_by_side_and_beyond_32_bits(hbl, new, bits):
    """Keys and values of one pool, pages far apart (more than 2^31 values, and bytes, from the first one): as in pools of their own."""
    note(f"attention: far pages new={new} bits={bits}")
    d, page, H, n_pages = 256, 64, 2, 4
    g = gen(91)
    lens, table = [200], ints([[3, 1, 0, 2]])
    (kp, ks), (vp, vs) = (R.random_pages(g, n_pages, H, page, d, bits, "cuda") for _ in range(2))
    q = torch.randn((new, 4, d), generator=g).bfloat16().cuda()
    k, v = (torch.randn((new, H, d), generator=g).bfloat16().cuda() for _ in range(2))
    # rows of d * bits / 8 bytes: the last page begins beyond byte 2^32 of the pool (16, 8 bits) or row 2^22 times 3
    page_rows = ((1 << 32) // 3 // (d * bits // 8) + 64) if bits >= 8 else 1 << 22
    row = tuple(kp.shape[1:])
    far = torch.zeros((3 * page_rows + 2 * H * page) * kp.shape[-1], dtype=kp.dtype, device="cuda")
    width = kp.shape[-1]
    pools = [far[i * H * page * width:].as_strided((n_pages, *row), (page_rows * width, page * width, width, 1)) for i in (0, 1)]
    scales = [None, None]
    if bits != 16:
        far_scales = torch.zeros(3 * page_rows + 2 * H * page, device="cuda")
        scales = [far_scales[i * H * page:].as_strided((n_pages, H, page), (page_rows, page, 1)) for i in (0, 1)]
        for a, b in zip(scales, (ks, vs)):
            a.copy_(b)
    for a, b in zip(pools, (kp, vp)):
        a.copy_(b)
    batch = (ints([0, new]), ints(lens), table)
    near, apart = hbl.KvCache(kp, vp, bits, ks, vs), hbl.KvCache(*pools, bits, *scales)
    freqs = hbl.rope_frequencies(128)
    for cache in (near, apart):
        hbl.kv_append(cache, k, v, *batch, freqs=freqs)
    got = [hbl.paged_attention(q, c, *batch, new) for c in (near, apart)]
    assert torch.equal(got[0].view(torch.int16), got[1].view(torch.int16))
    assert torch.equal(pools[0].contiguous().view(torch.uint8), kp.view(torch.uint8)) and torch.equal(pools[1].contiguous().view(torch.uint8), vp.view(torch.uint8))


def test_chunks_in_a_graph(hbl):
    """A captured chunk whose keys are cut into parts, replayed at other lengths with eager work between."""
    note("chunks in a graph")
    d, page, n, H = 128, 64, 100, 2
    g = gen(95)
    table, n_pages = R.page_table(g, [6000], page)
    (kp, ks), (vp, vs) = (R.random_pages(g, n_pages, H, page, d, 4, "cuda") for _ in range(2))
    cache, q = hbl.KvCache(kp, vp, 4, ks, vs), torch.randn((n, 8, d), generator=g).bfloat16().cuda()
    lens, starts, table = ints([500]), ints([0, n]), table.cuda()
    workspace = torch.empty(hbl.paged_attention_workspace_bytes(cache, n, 1, 8, n), dtype=torch.uint8, device="cuda")
    hbl.paged_attention(q, cache, starts, lens, table, n, workspace=workspace)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = hbl.paged_attention(q, cache, starts, lens, table, n, workspace=workspace)
    for length in (100, 6000, 777, 50, 4096):
        lens.fill_(length)
        graph.replay()
        got = y.clone()
        want = hbl.paged_attention(q, cache, starts, lens, table, n)
        torch.cuda.synchronize()
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))


# --- together ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [16, 8, 4, 3])
def test_generation_in_steps_equals_one_prompt(hbl, bits):
    """A prompt in one call, and the same tokens in chunks and single steps over the growing cache: append, attend."""
    note(f"generation in steps bits={bits}")
    T, Hq, Hkv, d, page = 150, 8, 2, 128, 16
    g = gen(41)
    qkv = torch.randn((T, (Hq + 2 * Hkv) * d), generator=g).bfloat16().cuda()
    parts = lambda x: [p.unflatten(-1, (-1, d)) for p in x.split((Hq * d, Hkv * d, Hkv * d), -1)]
    freqs = hbl.rope_frequencies(d, scaling="parts", factor=4.0, trained_len=64.0)
    table = torch.randperm(10, generator=g).to(torch.int32).cuda().view(1, 10)

    def go(steps):
        cache, outs, at = hbl.KvCache.empty(10, Hkv, page, d, bits), [], 0
        for n in steps:
            q, k, v = parts(qkv[at:at + n])
            at += n
            batch = (ints([0, n]), ints([at]), table)
            q = hbl.kv_append(cache, k, v, *batch, freqs=freqs, q=q)
            outs.append(hbl.paged_attention(q, cache, *batch, n))
        return torch.cat(outs), cache

    whole, cache = go([T])
    steps, other = go([64, 1, 1, 33, 2, 1, 40, 8])
    assert torch.equal(cache.k[table[0, :9].long()].view(torch.uint8), other.k[table[0, :9].long()].view(torch.uint8))
    q = hbl.rope(parts(qkv)[0], torch.arange(T, dtype=torch.int32, device="cuda"), freqs)
    want, bound = R.attention(q, cache.k, cache.v, cache.k_scales, cache.v_scales, bits, [0, T], [T], table.tolist(), d ** -0.5)
    tol = bound + (want.abs() + bound) * R.U16 * 1.001
    assert ((whole.double() - want).abs() <= tol).all() and ((steps.double() - want).abs() <= tol).all()


def test_decode_steps_in_a_graph(hbl):
    """A captured step (append and attend) replayed while lengths grow on the device, against eager calls."""
    note("decode steps in a graph")
    S, Hq, Hkv, d, page, bits = 3, 8, 4, 64, 16, 4
    g = gen(51)
    cache, twin = (hbl.KvCache.empty(S * 8, Hkv, page, d, bits) for _ in range(2))
    table = torch.randperm(S * 8, generator=g).to(torch.int32).cuda().view(S, 8)
    freqs, starts = hbl.rope_frequencies(d), ints([0, 1, 2, 3])
    new = [torch.randn((S, (Hq + 2 * Hkv) * d), generator=g).bfloat16().cuda() for _ in range(40)]
    hold, lens = new[0].clone(), ints([0, 0, 0])
    lens_now = ints([0, 0, 0])
    workspace = torch.empty(hbl.paged_attention_workspace_bytes(cache, S, S, Hq, 1), dtype=torch.uint8, device="cuda")

    def step(x, c, lens, workspace):
        q, k, v = (p.unflatten(-1, (-1, d)) for p in x.split((Hq * d, Hkv * d, Hkv * d), -1))
        q = hbl.kv_append(c, k, v, starts, lens, table, freqs=freqs, q=q)
        return hbl.paged_attention(q, c, starts, lens, table, 1, workspace=workspace)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(hold, cache, lens + 1, workspace)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lens.add_(1)
        y = step(hold, cache, lens, workspace)
    lens.zero_()
    for x in new:
        hold.copy_(x)
        graph.replay()
        lens_now += 1
        want = step(x, twin, lens_now, None)
        torch.cuda.synchronize()
        assert torch.equal(y.view(torch.int16), want.view(torch.int16))


def test_two_streams_at_once(hbl):
    note("two streams")
    d, page = 128, 64
    work = []
    for i, bits in enumerate((16, 4)):
        g = gen(60 + i)
        lens = [700 + 100 * i, 50]
        table, n = R.page_table(g, lens, page)
        (kp, ks), (vp, vs) = (R.random_pages(g, n, 2, page, d, bits, "cuda") for _ in range(2))
        q = torch.randn((2, 8, d), generator=g).bfloat16().cuda()
        work.append((q, hbl.KvCache(kp, vp, bits, ks, vs), ints([0, 1, 2]), ints(lens), table.cuda(), 1))
    want = [hbl.paged_attention(*w) for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    got = [[], []]
    for _ in range(20):
        for i, w in enumerate(work):
            with torch.cuda.stream(streams[i]):
                got[i].append(hbl.paged_attention(*w))
    torch.cuda.synchronize()
    for i in range(2):
        for y in got[i]:
            assert torch.equal(y.view(torch.int16), want[i].view(torch.int16))


# --- the binding ------------------------------------------------------------------------------------------------

def test_native_and_python_marshalling_agree(hbl, monkeypatch):
    """Both ways of making the calls: the same outputs bit for bit, and the same refusals."""
    note("native and Python marshalling")
    native = hbl._call
    assert native is not None, "_host_call is not built"
    g = gen(71)
    T, Hq, Hkv, d, page, bits = 20, 4, 2, 64, 16, 8
    qkv = torch.randn((T, (Hq + 2 * Hkv) * d), generator=g).bfloat16().cuda()
    q, k, v = (p.unflatten(-1, (-1, d)) for p in qkv.split((Hq * d, Hkv * d, Hkv * d), -1))
    table, starts, lens = torch.randperm(8, generator=g).to(torch.int32).cuda().view(2, 4), ints([0, 13, 20]), ints([40, 7])
    freqs, positions = hbl.rope_frequencies(d), torch.arange(T, dtype=torch.int32, device="cuda")
    slopes, prefix = torch.tensor([0.5, 0.25, 0.125, 0.0], device="cuda"), ints([20, 0])

    def outputs():
        cache = hbl.KvCache.empty(8, Hkv, page, d, bits)
        for t in (cache.k, cache.v, cache.k_scales, cache.v_scales):
            t.zero_()
        yield hbl.rope(q, positions, freqs)
        yield hbl.rope(q, positions, freqs, "interleaved", 1.5, True, torch.float32)
        kept = torch.zeros((T, 2 * Hq, d), dtype=torch.float32, device="cuda")
        assert hbl.rope(q, positions, freqs, out=kept[:, Hq:]).data_ptr() == kept[:, Hq:].data_ptr()
        yield kept
        turned = hbl.kv_append(cache, k, v, starts, lens, table, freqs=freqs, q=q)
        yield turned
        assert hbl.kv_append(cache, k, v, starts, lens, table) is None
        yield hbl.kv_append(cache, k, v, starts, lens, table, freqs=freqs, layout="interleaved", q=q, q_out=torch.zeros_like(kept[:, :Hq]))
        yield from (cache.k, cache.v, cache.k_scales, cache.v_scales)
        yield hbl.paged_attention(turned, cache, starts, lens, table, 13)
        n = hbl.paged_attention_workspace_bytes(cache, T, 2, Hq, 13)
        yield hbl.paged_attention(turned, cache, starts, lens, table, 13, scale=0.2, softcap=5.0, window=9, slopes=slopes, prefix_lens=prefix,
                                  out=torch.zeros_like(turned), workspace=torch.empty(n, dtype=torch.uint8, device="cuda"))

    mine = list(outputs())
    monkeypatch.setattr(hbl, "_call", None)
    for a, b in zip(mine, outputs(), strict=True):
        assert a.dtype == b.dtype and torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    cache = hbl.KvCache.empty(8, Hkv, page, d, bits)
    for call in (native, None):
        monkeypatch.setattr(hbl, "_call", call)
        refused = [
            (ValueError, lambda: hbl.rope(q.transpose(0, 1), positions, freqs)), (ValueError, lambda: hbl.rope(q, positions[:5], freqs)),
            (ValueError, lambda: hbl.rope(q, positions.long(), freqs)), (ValueError, lambda: hbl.rope(q, positions, freqs.double())),
            (ValueError, lambda: hbl.rope(q, positions, freqs.cpu())), (ValueError, lambda: hbl.rope(q, positions, freqs, layout="both")),
            (TypeError, lambda: hbl.rope(q.half(), positions, freqs)), (TypeError, lambda: hbl.rope(q, positions, freqs, out_dtype=torch.float16)),
            (ValueError, lambda: hbl.rope(q, positions, freqs, out=torch.empty_like(q)[:, :2])),
            (hbl.HblError, lambda: hbl.rope(q, positions, freqs[:4].clone())), (hbl.HblError, lambda: hbl.rope(q, positions, hbl.rope_frequencies(128))),
            (ValueError, lambda: hbl.kv_append(cache, k[:, :1], v[:, :1], starts, lens, table)), (ValueError, lambda: hbl.kv_append(cache, k, v[:5], starts, lens, table)),
            (ValueError, lambda: hbl.kv_append(cache, k, v, starts[:2], lens, table, q=q)), (ValueError, lambda: hbl.kv_append(cache, k, v, starts, lens, table.t(), q=q)),
            (ValueError, lambda: hbl.kv_append(cache, k, v, starts, lens, table, q=q.float())), (ValueError, lambda: hbl.kv_append(cache, k, v, starts, lens, table, q_out=q)),
            (ValueError, lambda: hbl.kv_append(cache, k, v, starts, lens, table[:1], q=q)),
            (TypeError, lambda: hbl.paged_attention(q.float(), cache, starts, lens, table, 13)), (ValueError, lambda: hbl.paged_attention(q, cache, starts, lens.long(), table, 13)),
            (ValueError, lambda: hbl.paged_attention(q, cache, starts, lens, table, 13, slopes=slopes[:3])),
            (ValueError, lambda: hbl.paged_attention(q, cache, starts, lens, table, 13, prefix_lens=prefix[:1])),
            (hbl.HblError, lambda: hbl.paged_attention(q[:, :3].contiguous(), cache, starts, lens, table, 13)),
            (hbl.HblError, lambda: hbl.paged_attention(q, cache, starts, lens, table, 0)), (hbl.HblError, lambda: hbl.paged_attention(q, cache, starts, lens, table, 13, window=-1)),
            (hbl.HblError, lambda: hbl.paged_attention(q, cache, starts, lens, table, 13, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))),
            (ValueError, lambda: hbl.KvCache(cache.k, cache.v, 16)), (ValueError, lambda: hbl.KvCache(cache.k, cache.v, 8)),
            (ValueError, lambda: hbl.KvCache(cache.k, cache.v[:4], 8, cache.k_scales, cache.v_scales)),
            (ValueError, lambda: hbl.KvCache(cache.k, cache.v, 5, cache.k_scales, cache.v_scales)),
            (ValueError, lambda: hbl.KvCache(cache.k.transpose(1, 2), cache.v, 8, cache.k_scales, cache.v_scales))]
        for i, (error, f) in enumerate(refused):
            with pytest.raises(error):
                f()
                print("not refused:", i)


def test_empty_calls(hbl):
    note("empty calls")
    cache, table = hbl.KvCache.empty(2, 2, 16, 64), torch.zeros((0, 3), dtype=torch.int32, device="cuda")
    x = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert hbl.rope(x, ints([]), hbl.rope_frequencies(64)).shape == (0, 2, 64)
    assert hbl.kv_append(cache, x, x, ints([0]), ints([]), table, q=x).shape == (0, 2, 64)
    assert hbl.paged_attention(x, cache, ints([0]), ints([]), table, 1).shape == (0, 2, 64)
    # tokens of nobody, a cache without pages, a table without columns
    y = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(y, 7.0)
    hbl.paged_attention(y, cache, ints([0]), ints([]), table, 1, out=out)
    assert (out == 7.0).all()
    none, narrow = hbl.KvCache.empty(0, 2, 16, 64), torch.zeros((1, 0), dtype=torch.int32, device="cuda")
    for c, t in ((none, torch.zeros((1, 3), dtype=torch.int32, device="cuda")), (cache, narrow)):
        hbl.kv_append(c, y, y, ints([0, 3]), ints([3]), t)
        assert (hbl.paged_attention(y, c, ints([0, 3]), ints([3]), t, 3) == 0).all()
        wide = torch.ones((50, 2, 64), dtype=torch.bfloat16, device="cuda")   # (a chunk)
        assert (hbl.paged_attention(wide, c, ints([0, 50]), ints([50]), t, 50) == 0).all()
