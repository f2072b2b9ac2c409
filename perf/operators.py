"""Performance cases of the library's attention side: what a program that serves a model with low-bit head states does
around its projections.

Kinds of case (key "kind"):
  rope       rotary positions of the heads of a batch of tokens, or the gradient through them ("backward")
  append     the new tokens' keys (rotated on the way) and values into a paged cache, with the queries rotated by the same call
  attention  the new tokens' queries against the paged cache: one token a sequence, or a chunk

A cache is pages of "page" tokens, [pages, heads, page, d] in bf16 ("bits" 16) or in codes of 8, 4 or 3 bits with one fp32
scale a row.  A batch is ragged: sequence s has q_starts[s+1] - q_starts[s] new tokens, the last ones of its kv_lens[s] keys.
"""
import math

import torch

own = False   # True: the library's operators, else their plain form

EPS = 1e-5
BASE = 10000.0


def listed():
    return [
        # one decode step's queries, eight sequences: a launch and little else
        {"name": "rope_decode_b8", "kind": "rope", "T": 8, "H": 32, "d": 128, "rot": 128, "layout": "half", "backward": False,
         "dtype": "bfloat16", "stride": 4096, "first": 4000, "stretch": 1.0},
        # the queries of an 8192-token prompt, read in place from the fused QKV output of the 7B layer
        {"name": "rope_prompt_qkv7b", "kind": "rope", "T": 8192, "H": 32, "d": 128, "rot": 128, "layout": "interleaved",
         "backward": False, "dtype": "bfloat16", "stride": 3 * 4096, "first": 0, "stretch": 1.0},
        # gradient through a partial rotation, fp32, an odd count of tokens far out in a stretched context
        {"name": "rope_backward_far", "kind": "rope", "T": 5003, "H": 32, "d": 64, "rot": 32, "layout": "half",
         "backward": True, "dtype": "float32", "stride": 32 * 64, "first": 900000, "stretch": 8.0},
        # one decode step of 64 sequences into a 16-bit cache, heads of the 7B layer
        {"name": "append_decode_b64", "kind": "append", "S": 64, "new": 1, "context": 1021, "ragged": True, "Hq": 32, "Hkv": 32,
         "d": 128, "rot": 128, "layout": "half", "bits": 16, "page": 64, "dtype": "bfloat16"},
        # an 8192-token prompt of the 7B layer into the 4-bit cache, and the cache read back
        {"name": "append_prompt_4bit", "kind": "append", "S": 1, "new": 8192, "context": 0, "ragged": False, "Hq": 32, "Hkv": 32,
         "d": 128, "rot": 128, "layout": "half", "bits": 4, "page": 64, "dtype": "bfloat16"},
        # a ragged batch of short chunks, fp32 states with shared heads of 64, 8 bits, pages of 16
        {"name": "append_ragged_8bit", "kind": "append", "S": 23, "new": 117, "context": 333, "ragged": True, "Hq": 32, "Hkv": 8,
         "d": 64, "rot": 32, "layout": "interleaved", "bits": 8, "page": 16, "dtype": "float32"},
        # one sequence's decode step at a short context, 16-bit states of the 7B layer
        {"name": "attend_decode_b1", "kind": "attention", "S": 1, "new": 1, "context": 1100, "ragged": False, "Hq": 32, "Hkv": 32,
         "d": 128, "bits": 16, "page": 64, "cap": 0.0, "window": 0, "slopes": False, "prefix": 0},
        # a full serving batch of ragged contexts on the 4-bit cache, four queries to a key head
        {"name": "attend_decode_b64_4bit", "kind": "attention", "S": 64, "new": 1, "context": 8000, "ragged": True, "Hq": 32,
         "Hkv": 8, "d": 128, "bits": 4, "page": 64, "cap": 0.0, "window": 0, "slopes": False, "prefix": 0},
        # a few very long contexts, 16 bits, three tokens a step (speculative decoding)
        {"name": "attend_long_b3", "kind": "attention", "S": 3, "new": 3, "context": 131000, "ragged": True, "Hq": 32, "Hkv": 8,
         "d": 128, "bits": 16, "page": 128, "cap": 0.0, "window": 0, "slopes": False, "prefix": 0},
        # an 8192-token prompt against its own keys, heads of the 7B layer
        {"name": "attend_prompt_7b", "kind": "attention", "S": 1, "new": 8192, "context": 0, "ragged": False, "Hq": 32, "Hkv": 32,
         "d": 128, "bits": 16, "page": 64, "cap": 0.0, "window": 0, "slopes": False, "prefix": 0},
        # chunks of long prompts over an 8-bit cache, scores capped
        {"name": "attend_chunk_8bit_cap", "kind": "attention", "S": 2, "new": 512, "context": 12345, "ragged": True, "Hq": 32,
         "Hkv": 8, "d": 128, "bits": 8, "page": 64, "cap": 30.0, "window": 0, "slopes": False, "prefix": 0},
        # a mixed batch of small heads on the 3-bit cache: a window, a bias by distance, a prefix that all tokens see
        {"name": "attend_mixed_3bit", "kind": "attention", "S": 19, "new": 157, "context": 1500, "ragged": True, "Hq": 16,
         "Hkv": 16, "d": 64, "bits": 3, "page": 16, "cap": 0.0, "window": 700, "slopes": True, "prefix": 64},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("rope", "append", "attention", "attention"))
    if kind == "rope":
        H, d = rng.choice((4, 8, 12, 16, 32)), rng.choice((64, 64, 80, 128, 128, 256))
        T = _log_int(rng, 1, min(16384, (1 << 25) // (H * d)))
        return {"kind": kind, "T": T, "H": H, "d": d, "rot": min(d, rng.choice((32, 64, d, d))), "layout": rng.choice(("half", "interleaved")),
                "backward": rng.random() < 0.4, "dtype": rng.choice(("bfloat16", "float32")), "stride": H * d * rng.choice((1, 1, 3)),
                "first": _log_int(rng, 1, 1000000) - 1, "stretch": rng.choice((1.0, 4.0, 32.0))}
    d, bits, page = rng.choice((64, 128, 128, 256)), rng.choice((16, 16, 8, 4, 3)), rng.choice((16, 32, 64, 128))
    Hkv, G = rng.choice((1, 2, 4, 8, 8, 16, 32)), rng.choice((1, 1, 2, 4, 7, 8))
    Hkv = min(Hkv, 4096 // d)
    G = min(G, 4096 // (d * Hkv))
    case = {"kind": kind, "Hq": Hkv * G, "Hkv": Hkv, "d": d, "bits": bits, "page": page, "ragged": rng.random() < 0.6}
    if kind == "append":
        S = _log_int(rng, 1, 128)
        new = 1 if rng.random() < 0.4 else _log_int(rng, 1, max(1, 8192 // S))
        context = _log_int(rng, 1, max(1, min(4096, (1 << 25) // (S * Hkv * d)))) - 1
        return {**case, "S": S, "new": new, "context": context, "rot": min(d, rng.choice((32, 64, d, d))),
                "layout": rng.choice(("half", "interleaved")), "dtype": rng.choice(("bfloat16", "bfloat16", "float32"))}
    decode = rng.random() < 0.5
    S = _log_int(rng, 1, 128 if decode else 16)
    new = rng.choice((1, 1, 1, 2, 4)) if decode else _log_int(rng, 2, max(2, 8192 // S))
    # rows of states, and scores in the plain form, no more than the largest listed cases have
    most = min(131072, 2 * 131000 * 1024 // (S * Hkv * d), (1 << 30) // (S * Hkv * G * new))
    context = _log_int(rng, 1, max(1, most - new)) - 1
    return {**case, "S": S, "new": new, "context": context, "cap": rng.choice((0.0, 0.0, 30.0)),
            "window": rng.choice((0, 0, 0, _log_int(rng, 16, 4096))), "slopes": rng.random() < 0.2,
            "prefix": rng.choice((0, 0, 0, _log_int(rng, 1, 256)))}


# --- inputs, from the seed alone -------------------------------------------------------------------------------

def _lengths(case):
    """(new tokens, keys) of every sequence; the first is the longest, the others of a ragged batch spread below it."""
    new, total = [], []
    for s in range(case["S"]):
        part = 1.0 if s == 0 or not case["ragged"] else 1.0 - 0.8 * ((s * 0.6180339887) % 1.0)
        n = max(1, int(case["new"] * part))
        new.append(n)
        total.append(n + int(case["context"] * part))
    return new, total


def _frequencies(rot, stretch):
    return (1.0 / (BASE * stretch) ** (torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()


def _quantise(x, bits):
    """Codes (one to a byte) and scales of rows: absmax at `bits` bits, unsigned."""
    half = 1 << (bits - 1)
    gamma = x.abs().amax(-1, keepdim=True)
    u = torch.round(x * ((half - 1) / (gamma + EPS))).clamp_(-half, half - 1) + half
    return u.to(torch.uint8), (gamma / (half - 1)).squeeze(-1)


def _pack(u, bits):
    if bits == 8:
        return u
    if bits == 4:
        return u[..., 0::2] | (u[..., 1::2] << 4)
    w = u.unflatten(-1, (-1, 8)).to(torch.int32)
    w = (w << torch.arange(0, 24, 3, device=u.device, dtype=torch.int32)).sum(-1, dtype=torch.int32)
    return (w[..., None] >> torch.arange(0, 24, 8, device=u.device, dtype=torch.int32)).bitwise_and_(255).flatten(-2).to(torch.uint8)


def _unpack(packed, bits):
    if bits == 8:
        return packed
    if bits == 4:
        return torch.stack((packed & 15, packed >> 4), -1).flatten(-2)
    w = packed.unflatten(-1, (-1, 3)).to(torch.int32)
    w = w[..., 0] | (w[..., 1] << 8) | (w[..., 2] << 16)
    return ((w[..., None] >> torch.arange(0, 24, 3, device=packed.device, dtype=torch.int32)) & 7).flatten(-2).to(torch.uint8)


def _pages(g, case, n_pages):
    """One side (keys or values) of a cache: pages and, for codes, scales."""
    shape = (n_pages, case["Hkv"], case["page"], case["d"])
    bits = case["bits"]
    if bits == 16:
        return torch.randn(shape, device="cuda", generator=g, dtype=torch.bfloat16), None
    pages = torch.empty((*shape[:-1], case["d"] * bits // 8), device="cuda", dtype=torch.uint8)
    scales = torch.empty(shape[:-1], device="cuda")
    some = max(1, (1 << 26) // (shape[1] * shape[2] * shape[3]))
    for at in range(0, n_pages, some):
        u, s = _quantise(torch.randn((min(some, n_pages - at), *shape[1:]), device="cuda", generator=g), bits)
        pages[at:at + some], scales[at:at + some] = _pack(u, bits), s
    return pages, scales


def _batch(g, case):
    new, total = _lengths(case)
    page = case["page"]
    each = [-(-t // page) for t in total]
    order = torch.randperm(sum(each), device="cuda", generator=g).to(torch.int32)
    table = torch.full((case["S"], max(each)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(each):
        table[s, :n] = order[at:at + n]
        at += n
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    state = {"q_starts": torch.tensor(starts, dtype=torch.int32, device="cuda"),
             "kv_lens": torch.tensor(total, dtype=torch.int32, device="cuda"), "block_table": table,
             "max_new": max(new), "max_len": max(total)}
    for name in ("k", "v"):
        state[name + "_pages"], state[name + "_scales"] = _pages(g, case, sum(each))
    return state, starts[-1]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["kind"] == "rope":
        dtype = getattr(torch, case["dtype"])
        rows = torch.randn((case["T"], case["stride"]), device="cuda", generator=g).to(dtype)
        x = rows[:, :case["H"] * case["d"]].unflatten(-1, (case["H"], case["d"]))
        far = torch.randint(0, 4 * case["T"] + 64, (case["T"],), device="cuda", generator=g, dtype=torch.int32)
        return {**case, "x": x, "positions": far + case["first"], "freqs": _frequencies(case["rot"], case["stretch"]),
                "magnitude": 1.0 + 0.1 * math.log(case["stretch"])}
    state, T = _batch(g, case)
    state.update(case)
    if case["kind"] == "append":
        dtype, Hq, Hkv, d = getattr(torch, case["dtype"]), case["Hq"], case["Hkv"], case["d"]
        qkv = torch.randn((T, (Hq + 2 * Hkv) * d), device="cuda", generator=g)
        qkv[:, d // 3::d] *= 8.0   # a feature of every head that sticks out, as one does in keys
        parts = qkv.to(dtype).split((Hq * d, Hkv * d, Hkv * d), -1)
        state["q"], state["k"], state["v"] = (p.unflatten(-1, (-1, d)) for p in parts)
        state["freqs"] = _frequencies(case["rot"], 1.0)
        return state
    state["q"] = (2.0 * torch.randn((T, case["Hq"], case["d"]), device="cuda", generator=g)).bfloat16()
    state["slope_of"] = (2.0 ** (-8.0 * torch.arange(1, case["Hq"] + 1) / case["Hq"])).float().cuda() if case["slopes"] else None
    state["prefix_lens"] = torch.full((case["S"],), case["prefix"], dtype=torch.int32, device="cuda") if case["prefix"] else None
    # scratch that a serving program keeps from step to step
    state["scratch"] = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    return state


# --- the plain form, in 32 bits --------------------------------------------------------------------------------

def _rotated(x, positions, freqs, layout, magnitude=1.0, backward=False):
    """x [T, H, d] with the first 2 * len(freqs) features of every head rotated, in 32 bits (angles in 64)."""
    angle = positions.double()[:, None] * freqs.double()
    cos, sin = (magnitude * angle.cos()).float()[:, None], (magnitude * angle.sin()).float()[:, None]
    if backward:
        sin = -sin
    x, rot = x.float(), 2 * freqs.numel()
    r, rest = x[..., :rot], x[..., rot:]
    if layout == "half":
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        r = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    return torch.cat((r, rest), -1)


def _sequence_of(q_starts, T):
    return torch.searchsorted(q_starts, torch.arange(T, device="cuda", dtype=torch.int32), right=True) - 1


def _positions(s, T):
    """(sequence, position) of every new token."""
    seq = _sequence_of(s["q_starts"], T)
    at = torch.arange(T, device="cuda") - s["q_starts"][seq]
    return seq, s["kv_lens"][seq] - (s["q_starts"][seq + 1] - s["q_starts"][seq]) + at


def _values(pages, scales, bits):
    """What pages stand for, in 32 bits."""
    if bits == 16:
        return pages.float()
    return (_unpack(pages, bits).float() - (1 << (bits - 1))) * scales[..., None]


def _plain_append(s):
    T, page, bits = s["k"].shape[0], s["page"], s["bits"]
    seq, p = _positions(s, T)
    where = s["block_table"][seq, p // page].long()
    slot = (p % page).long()
    k = _rotated(s["k"], p, s["freqs"], s["layout"])
    q = _rotated(s["q"], p, s["freqs"], s["layout"]).to(s["q"].dtype)
    if bits == 16:
        s["k_pages"][where, :, slot], s["v_pages"][where, :, slot] = k.bfloat16(), s["v"].bfloat16()
        return {"q": q, "k": s["k_pages"], "v": s["v_pages"]}
    (ku, ks), (vu, vs) = _quantise(k, bits), _quantise(s["v"].float(), bits)
    s["k_pages"][where, :, slot], s["k_scales"][where, :, slot] = _pack(ku, bits), ks
    s["v_pages"][where, :, slot], s["v_scales"][where, :, slot] = _pack(vu, bits), vs
    return {"q": q, "k": _values(s["k_pages"], s["k_scales"], bits).bfloat16(), "v": _values(s["v_pages"], s["v_scales"], bits).bfloat16()}


def _plain_attention(s):
    q, S, Hkv, d = s["q"], s["S"], s["Hkv"], s["d"]
    T, M, N = q.shape[0], s["max_new"], s["max_len"]
    seq, p = _positions(s, T)
    # sequences side by side, padded to the longest: [S, Hkv, keys, d] and [S, Hkv, group, tokens, d]
    table = s["block_table"].clamp(min=0).long()

    def gathered(pages, scales):
        v = _values(pages[table], None if scales is None else scales[table], s["bits"])   # [S, P, Hkv, page, d]
        return v.transpose(1, 2).flatten(2, 3)[:, :, :N]

    row = (torch.arange(T, device="cuda") - s["q_starts"][seq]).long()
    padded = torch.zeros((S, M, s["Hq"], d), device="cuda")
    padded[seq, row] = q.float()
    at = torch.full((S, M), -1, dtype=torch.int64, device="cuda")
    at[seq, row] = p.long()
    padded = padded.unflatten(2, (Hkv, -1)).permute(0, 2, 3, 1, 4).flatten(2, 3)
    k = gathered(s["k_pages"], s["k_scales"])
    scores = torch.matmul(padded, k.transpose(2, 3).contiguous()).unflatten(2, (-1, M)).mul_(1.0 / math.sqrt(d))
    del k
    if s["cap"]:
        scores = torch.tanh(scores.div_(s["cap"])).mul_(s["cap"])
    key, at = torch.arange(N, device="cuda"), at[:, :, None]
    if s["slope_of"] is not None:
        scores -= s["slope_of"].view(1, Hkv, -1, 1, 1) * (at - key).abs().float()[:, None, None]
    seen = key <= at
    if s["prefix_lens"] is not None:
        seen = seen | ((key < s["prefix_lens"][:, None, None]) & (at >= 0))
    if s["window"]:
        seen = seen & (key > at - s["window"])
    seen = seen & (key < s["kv_lens"][:, None, None])
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    most = scores.amax(-1, keepdim=True).clamp_(min=-1e30)
    scores = scores.sub_(most).exp_()
    total = scores.sum(-1, keepdim=True)
    o = torch.matmul(scores.flatten(2, 3), gathered(s["v_pages"], s["v_scales"])).unflatten(2, (-1, M))
    o = o / torch.where(total > 0, total, torch.ones_like(total))
    return o.permute(0, 3, 1, 2, 4).flatten(2, 3)[seq, row].bfloat16()


# --- one pass --------------------------------------------------------------------------------------------------

def _own_cache(s):
    """The library's handle on the pages: a program makes it once for a cache."""
    from paper_2504_18415_amd import hbl
    if "cache" not in s:
        s["cache"] = hbl.KvCache(s["k_pages"], s["v_pages"], s["bits"], s["k_scales"], s["v_scales"])
    return hbl, s["cache"]


def _own_rope(s):
    from paper_2504_18415_amd import hbl
    return hbl.rope(s["x"], s["positions"], s["freqs"], layout=s["layout"], magnitude=s["magnitude"], backward=s["backward"])


def _own_append(s):
    hbl, cache = _own_cache(s)
    q = hbl.kv_append(cache, s["k"], s["v"], s["q_starts"], s["kv_lens"], s["block_table"], freqs=s["freqs"], layout=s["layout"],
                      q=s["q"], eps=EPS)
    if s["bits"] == 16:
        return {"q": q, "k": s["k_pages"], "v": s["v_pages"]}
    shape = (*s["k_pages"].shape[:-1], s["d"])
    k, v = (hbl.kv_dequant(s[n + "_pages"], s[n + "_scales"].view(-1), s["d"], s["bits"]).view(shape) for n in ("k", "v"))
    return {"q": q, "k": k, "v": v}


def _own_attention(s):
    hbl, cache = _own_cache(s)
    return hbl.paged_attention(s["q"], cache, s["q_starts"], s["kv_lens"], s["block_table"], s["max_new"], softcap=s["cap"],
                               window=s["window"], slopes=s["slope_of"], prefix_lens=s["prefix_lens"], workspace=s["scratch"])


def run(s):
    if own:
        return {"rope": _own_rope, "append": _own_append, "attention": _own_attention}[s["kind"]](s)
    if s["kind"] == "rope":
        return _rotated(s["x"], s["positions"], s["freqs"], s["layout"], s["magnitude"], s["backward"]).to(s["x"].dtype)
    return _plain_append(s) if s["kind"] == "append" else _plain_attention(s)


# --- what a pass cannot do without ------------------------------------------------------------------------------

def _visible(case):
    """(pairs of a new token and a key it sees, keys that some new token sees), over the sequences."""
    pairs = keys = 0
    for n, total in zip(*_lengths(case)):
        first = total
        for p in range(total - n, total):
            lo = max(0, p - case["window"] + 1) if case["window"] else 0
            pairs += max(0, min(total, max(p + 1, case["prefix"])) - lo)
            first = min(first, lo)
        keys += total - first
    return pairs, keys


def work(case):
    d = case["d"]
    if case["kind"] == "rope":
        values = case["T"] * case["H"] * d
        return {"bytes": values * (4 if case["dtype"] == "bfloat16" else 8) + 4 * case["T"] + 2 * case["rot"],
                "flops": 3 * case["T"] * case["H"] * case["rot"]}
    new, total = _lengths(case)
    T, Hq, Hkv, bits = sum(new), case["Hq"], case["Hkv"], case["bits"]
    row = d * bits // 8 + (0 if bits == 16 else 4)
    if case["kind"] == "append":
        size = 2 if case["dtype"] == "bfloat16" else 4
        moved = T * d * size * (2 * Hq + 2 * Hkv) + 2 * T * Hkv * row
        if bits != 16:   # the cache read back: codes in, bf16 out
            rows = 2 * Hkv * case["page"] * sum(-(-t // case["page"]) for t in total)
            moved += rows * (row + 2 * d)
        return {"bytes": moved, "flops": 3 * T * (Hq + Hkv) * case["rot"] + (0 if bits == 16 else 4 * T * Hkv * d)}
    pairs, keys = _visible(case)
    return {"bytes": 4 * T * Hq * d + 2 * keys * Hkv * row, "flops": 4 * pairs * Hq * d}


# --- the definition, in 64 bits, row by row ---------------------------------------------------------------------

def _exact_rope(x, positions, freqs, layout, magnitude=1.0, sign=1.0):
    turn = torch.polar(torch.full((), magnitude, dtype=torch.float64, device="cuda"),
                       sign * positions.double()[:, None] * freqs.double())[:, None]
    y, n = x.double().clone(), freqs.numel()
    first, second = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    z = torch.complex(y[..., first], y[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_side(pages, scales, bits):
    if bits == 16:
        return pages.double()
    rows = pages.reshape(-1, pages.shape[-1]).to(torch.int64)
    d = pages.shape[-1] * 8 // bits
    out = torch.empty((rows.shape[0], d), dtype=torch.float64, device="cuda")
    for i in range(d):
        b, shift = bits * i // 8, bits * i % 8
        word = rows[:, b] + (rows[:, b + 1] * 256 if shift + bits > 8 else 0)
        out[:, i] = (word // (1 << shift)) % (1 << bits) - (1 << (bits - 1))
    return (out * scales.reshape(-1, 1).double()).view(*pages.shape[:-1], d)


def _exact_append(s):
    T, page, bits = s["k"].shape[0], s["page"], s["bits"]
    k_all, v_all = (_exact_side(s[n + "_pages"], s[n + "_scales"], bits) for n in ("k", "v"))
    starts, lens, table = s["q_starts"].tolist(), s["kv_lens"].tolist(), s["block_table"].tolist()
    position, pages, slots = [], [], []
    for i, total in enumerate(lens):
        for t in range(starts[i + 1] - starts[i]):
            p = total - (starts[i + 1] - starts[i]) + t
            position.append(p)
            pages.append(table[i][p // page])
            slots.append(p % page)
    position, pages, slots = (torch.tensor(v, device="cuda") for v in (position, pages, slots))
    k, v = _exact_rope(s["k"], position, s["freqs"], s["layout"]), s["v"].double()
    for rows, into in ((k, k_all), (v, v_all)):
        if bits != 16:
            top = (1 << (bits - 1)) - 1
            gamma = rows.abs().amax(-1, keepdim=True)
            rows = (rows * top / (gamma + EPS)).round().clamp(-top - 1, top) * gamma / top
        into[pages, :, slots] = rows
    return {"q": _exact_rope(s["q"], position, s["freqs"], s["layout"]), "k": k_all, "v": v_all}


def _exact_attention(s):
    starts, lens, page, G = s["q_starts"].tolist(), s["kv_lens"].tolist(), s["page"], s["Hq"] // s["Hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for i, total in enumerate(lens):
        mine = s["block_table"][i, :-(-total // page)].long()
        n = starts[i + 1] - starts[i]
        for h in range(s["Hkv"]):
            k, v = (_exact_side(s[x + "_pages"][mine, h], None if s[x + "_scales"] is None else s[x + "_scales"][mine, h], s["bits"])
                    .reshape(-1, s["d"])[:total] for x in ("k", "v"))
            for at in range(0, n, 1024):
                rows = torch.arange(at, min(n, at + 1024), device="cuda")
                p = (total - n + rows)[:, None]
                key = torch.arange(total, device="cuda")[None]
                hidden = key > torch.maximum(p, torch.full_like(p, s["prefix"] - 1))
                if s["window"]:
                    hidden = hidden | (key <= p - s["window"])
                for head in range(h * G, h * G + G):
                    x = s["q"][starts[i] + rows, head].double() @ k.T / math.sqrt(s["d"])
                    if s["cap"]:
                        x = s["cap"] * torch.tanh(x / s["cap"])
                    if s["slope_of"] is not None:
                        x = x - s["slope_of"][head].double() * (p - key).abs()
                    x = x.masked_fill(hidden, -math.inf)
                    out[starts[i] + rows, head] = torch.nan_to_num(torch.softmax(x, -1)) @ v
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return _exact_rope(s["x"], s["positions"], s["freqs"], s["layout"], s["magnitude"], -1.0 if s["backward"] else 1.0)
    if case["kind"] == "append":
        return _exact_append(s)
    return _exact_attention(s)
