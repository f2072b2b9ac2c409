"""The attention side's operators from their definitions, in 64 bits and element by element where that is practical: what the
tests of rope, kv_append and paged_attention compare with.  Uses torch for tensors and elementary arithmetic only."""
import math

import torch

EPS = 1e-5
U32 = 2.0 ** -24          # half a step, relative: fp32, bf16
U16 = 2.0 ** -8


def frequencies(rot, base=10000.0):
    return (base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float()


def rotate(x, positions, freqs, layout, magnitude=1.0, backward=False):
    """x [T, H, d] fp64."""
    y, n = x.double().clone(), freqs.numel()
    angle = (-1.0 if backward else 1.0) * positions.double()[:, None] * freqs.double()
    c, s = magnitude * angle.cos()[:, None], magnitude * angle.sin()[:, None]
    first, second = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    a, b = y[..., first].clone(), y[..., second].clone()
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    return y


def rotate_bound(x, freqs, layout, magnitude=1.0):
    """How far fp32 arithmetic may be off, per feature: the angle's last rounding (pi 2^-24 of a turn's half), the sine's and
    cosine's own error (4 half steps), the magnitude's, the products' and the sum's roundings (one each)."""
    n = freqs.numel()
    first, second = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    x = x.double().abs()
    b = torch.zeros_like(x)
    b[..., first] = b[..., second] = (x[..., first] + x[..., second]) * magnitude * (math.pi + 4 + 3) * U32
    return b


def unpack(pages, bits):
    """Codes of packed rows, less the offset: [..., d] fp64."""
    flat = pages.reshape(-1, pages.shape[-1]).to(torch.int64)
    d = pages.shape[-1] * 8 // bits
    out = torch.empty((flat.shape[0], d), dtype=torch.float64, device=pages.device)
    for i in range(d):
        byte, shift = bits * i // 8, bits * i % 8
        w = flat[:, byte] + (flat[:, byte + 1] << 8 if shift + bits > 8 else 0)
        out[:, i] = ((w >> shift) & ((1 << bits) - 1)) - (1 << (bits - 1))
    return out.view(*pages.shape[:-1], d)


def random_pages(g, n_pages, heads, page, d, bits, device, spread=1.0):
    """A pool with something in every slot: (pages, scales)."""
    if bits == 16:
        return (spread * torch.randn((n_pages, heads, page, d), generator=g)).bfloat16().to(device), None
    codes = torch.randint(0, 256, (n_pages, heads, page, d * bits // 8), generator=g, dtype=torch.uint8)
    scales = spread * (0.5 + torch.rand((n_pages, heads, page), generator=g)) * 2.0 ** (1 - bits)
    return codes.to(device), scales.to(device)


def page_table(g, kv_lens, page, spare=0, width=0):
    """Pages of the sequences in a shuffled order: (table int32 [S, width], number of pages)."""
    each = [-(-n // page) for n in kv_lens]
    order = torch.randperm(sum(each) + spare, generator=g).to(torch.int32)
    table = torch.full((len(kv_lens), max(max(each, default=0), width)), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(each):
        table[s, :n] = order[at:at + n]
        at += n
    return table, sum(each) + spare


def attention(q, k_pages, v_pages, k_scales, v_scales, bits, q_starts, kv_lens, table, scale, softcap=0.0, window=0, slopes=None,
              prefix_lens=None, out=None):
    """-> (out fp64 [T, Hq, d], bound): the outputs from the definition and how far the kernels may be off before the output's
    own rounding.  q_starts, kv_lens, prefix_lens are lists, table a list of lists."""
    T, Hq, d = q.shape
    Hkv, page = k_pages.shape[1], k_pages.shape[2]
    G, n_pages = Hq // Hkv, k_pages.shape[0]
    out = torch.zeros((T, Hq, d), dtype=torch.float64, device=q.device) if out is None else out.double().clone()
    bound = torch.zeros_like(out)
    offset = {16: 0.0, 8: 128.0, 4: 24.0, 3: 12.0}[bits]   # codes may travel with a constant added that sums take away again
    for s, total in enumerate(kv_lens):
        first, n = q_starts[s], q_starts[s + 1] - q_starts[s]
        keys = min(total, len(table[s]) * page)
        if n <= 0 or keys <= 0:
            continue
        j = torch.arange(keys, device=q.device)
        pages = torch.tensor(table[s][:-(-keys // page)], dtype=torch.int64, device=q.device)
        there = ((pages >= 0) & (pages < n_pages))
        safe = torch.where(there, pages, torch.zeros_like(pages))
        there = there.repeat_interleave(page)[:keys]
        p = (total - n + torch.arange(n, device=q.device))[:, None]
        seen = (j[None] <= p) & there[None] & (p >= 0)
        if prefix_lens is not None:
            seen = seen | ((j[None] < prefix_lens[s]) & there[None] & (p >= 0))
        if window:
            seen = seen & (j[None] > p - window)
        for h in range(Hkv):
            def side(pool, scales):
                rows = (pool[safe, h].double() if bits == 16 else unpack(pool[safe, h], bits)).reshape(-1, d)[:keys]
                return rows, (torch.ones(keys, dtype=torch.float64, device=q.device) if bits == 16
                              else scales[safe, h].double().reshape(-1)[:keys])
            k, ks = side(k_pages, k_scales)
            v, vs = side(v_pages, v_scales)
            v = v * vs[:, None]
            for head in range(h * G, (h + 1) * G):
                x = q[first:first + n, head].double()
                y = (x @ k.T) * ks * scale
                # fp32 sums of d products, in any order
                off = (x.abs() @ (k.abs() + offset).T) * ks * abs(scale) * (d + 4) * 2 * U32
                if softcap:
                    y = softcap * torch.tanh(y / softcap)
                    off = off + softcap * 8 * U32 + y.abs() * 4 * U32
                if slopes is not None:
                    y = y - slopes[head].double() * (p - j[None]).abs()
                y = y.masked_fill(~seen, -math.inf)
                top = y.amax(-1, keepdim=True)
                top = torch.where(top == -math.inf, torch.zeros_like(top), top)
                # the exponent is a rounded difference in units of ln 2
                off = torch.where(seen, off + ((y - top).abs() + y.abs() + top.abs()).nan_to_num(posinf=0.0) * 4 * U32, torch.zeros_like(off))
                w = (y - top).exp()
                total_w = w.sum(-1, keepdim=True)
                w = w / torch.where(total_w > 0, total_w, torch.ones_like(total_w))
                o = w @ v
                out[first:first + n, head] = o
                # each weight off by its bf16 rounding and by e^(2 off) - 1 (its own and the sum's); sums in fp32
                part = w * (U16 + torch.expm1(2 * off.amax(-1, keepdim=True)) + 2.0 ** -17)
                bound[first:first + n, head] = part @ (v.abs() + 2 * offset * vs[:, None] * (U32 * 64)) + 1e-30
    return out, bound
