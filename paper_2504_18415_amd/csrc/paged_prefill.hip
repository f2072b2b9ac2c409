// Attention of many rows (tokens times query heads of a key head) against the paged cache: prompts, chunks of them, mixed batches.
//
// Bound by the matrix cores and by the exponentials beside them.  A workgroup has kRows rows of one sequence and key head (tokens in
// order, the heads of the group side by side, so that the group shares what is read); each of its four waves keeps 32 of them in
// registers: queries, output, maximum and sum.  Tiles of keys and values pass through LDS as bf16, two of each, the next tile loaded
// while this one is used: 16-bit states straight to LDS, codes through registers, where they are widened once for all waves.
//
// Where there are few workgroups the keys are cut into equal parts, joined by a second launch in a fixed order.
#include "gemm_common.h"
#include "hbl_internal.h"
#include "paged_attention.h"

namespace hbl {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = 32 * kWaves;
template <int D>
constexpr int kTile = D == 256 ? 32 : 64;   // keys of a tile: two tiles of keys and values are 32 KiB (64), 64 KiB else

__device__ __align__(16) uint32_t no_state[128];   // a row of zeros, read in place of rows that are not there

// 16-byte chunks of a row lie in LDS at places that differ from row to row: those of keys so that 16 rows of the same chunk fall
// into different banks, those of values so that four rows of the same four chunks do.
template <int D>
__device__ __forceinline__ int k_place(int row, int chunk) {
    return row * (2 * D) + ((chunk ^ (D == 64 ? (row >> 1) & 7 : row & 15)) << 4);
}
template <int D>
__device__ __forceinline__ int v_place(int row, int chunk) {
    return row * (2 * D) + ((chunk ^ (D == 64 ? 4 * ((row >> 1) & 1) : 4 * (row & 3))) << 4);
}

struct Item {
    int s, tile;   // sequence, row tile in it
    SeqSpan span;
    int rows;      // of the sequence (tokens looked at times group)
};
__device__ __forceinline__ int row_tiles(const AttentionArgs& a, int s) {
    const SeqSpan span = span_of(a.batch, a.cache.page_shift, a.T, s);
    const int n = span.n < a.max_q ? span.n : a.max_q;
    return (int)(((int64_t)n * a.group + kRows - 1) / kRows);
}
// The row tiles of all sequences and where the rank-th is (the last tiles first: they see most keys).  false: there are not so many.
struct Search {
    int sums[kWaves], found[2], all;
};
__device__ __forceinline__ int count_row_tiles(const AttentionArgs& a, Search* lds, int from, int to, int& before) {
    int mine = 0;
    for (int s = from; s < to; ++s) mine += row_tiles(a, s);
    int v = mine;
    for (int m = 1; m < 64; m <<= 1) {
        const int u = __shfl_up(v, m, 64);
        if ((int)(threadIdx.x & 63) >= m) v += u;
    }
    if ((threadIdx.x & 63) == 63) lds->sums[threadIdx.x >> 6] = v;
    __syncthreads();
    int all = 0;
    before = v - mine;
    for (int w = 0; w < kWaves; ++w) {
        if (w < (int)(threadIdx.x >> 6)) before += lds->sums[w];
        all += lds->sums[w];
    }
    return all;
}
__device__ __forceinline__ void thread_share(const AttentionArgs& a, int& from, int& to) {
    const int per = (a.batch.n_seqs + kThreads - 1) / kThreads;
    from = min((int)threadIdx.x * per, a.batch.n_seqs);
    to = min(from + per, a.batch.n_seqs);
}
__device__ __forceinline__ Item find_item(const AttentionArgs& a, Search* lds, int from, int to, int before, int index) {
    for (int s = from, at = before; s < to; ++s) {
        const int n = row_tiles(a, s);
        if (index >= at && index < at + n) {
            lds->found[0] = s;
            lds->found[1] = index - at;
        }
        at += n;
    }
    __syncthreads();
    Item it;
    it.s = __builtin_amdgcn_readfirstlane(lds->found[0]);
    it.tile = __builtin_amdgcn_readfirstlane(lds->found[1]);
    it.span = span_of(a.batch, a.cache.page_shift, a.T, it.s);
    it.rows = (it.span.n < a.max_q ? it.span.n : a.max_q) * a.group;
    return it;
}

// Keys that some row of the tile sees, from a multiple of 16 on.
struct TileKeys {
    int base, end;
};
__device__ __forceinline__ TileKeys tile_keys(const AttentionArgs& a, const Item& it, int prefix) {
    const int before = it.span.total - it.span.n;
    int first = it.tile * kRows / a.group;
    const int last = min((it.tile + 1) * kRows, it.rows) - 1;
    if (first < -before) first = -before;
    if (first > last / a.group) return {0, 0};
    const KeyRange lo = visible_keys(before + first, it.span.keys, a.window, prefix);
    const KeyRange hi = visible_keys(before + last / a.group, it.span.keys, a.window, prefix);
    if (hi.hi <= lo.lo) return {0, 0};
    return {lo.lo & ~15, hi.hi};
}
struct Part {
    int from, to;   // tiles of keys
};
__device__ __forceinline__ Part part_of(int tiles, int part, int parts) {
    return {(int)((int64_t)tiles * part / parts), (int)((int64_t)tiles * (part + 1) / parts)};
}

template <int D, int BITS, bool SHAPED>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void paged_prefill_kernel(AttentionArgs a, int parts) {
    constexpr int TK = kTile<D>, KB = TK / 32;              // blocks of 32 keys
    constexpr int RW = TK / kWaves;                         // rows of a tile that a wave loads (16 bits)
    constexpr int RI = 512 / D, NI = RW / RI;               // rows a load, loads
    constexpr int CR = D / 32, CHUNKS = TK * CR;            // chunks of 32 codes: a row, a tile
    constexpr int CW = BITS;                                // dwords of one
    constexpr float kBias = Codes<BITS>::kBias;
    constexpr bool CODES = BITS != 16;
    constexpr int SIDE = TK * D * 2;                        // bytes of a tile's keys, or values, in LDS
    extern __shared__ __align__(16) char lds[];             // [2][keys, values], [2][key scales, value scales]
    __shared__ Search search;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 31, half = lane >> 5;
    const int heads = a.cache.heads, page_mask = (1 << a.cache.page_shift) - 1;

    int from, to, before_me;
    thread_share(a, from, to);
    const int items = count_row_tiles(a, &search, from, to, before_me);
    // workgroups go round the eight XCDs: where it divides, each works through whole heads, whose keys its cache then holds
    int head, rank;
    if (heads % 8 == 0) {
        const int in_xcd = blockIdx.x >> 3;
        if (items == 0) return;
        head = (int)(blockIdx.x & 7) + 8 * (in_xcd / (items * parts));
        rank = in_xcd % (items * parts);
    } else {
        head = blockIdx.x % heads;
        rank = blockIdx.x / heads;
    }
    if (head >= heads || rank >= items * parts) return;
    const int part = rank % parts, index = items - 1 - rank / parts;
    const Item it = find_item(a, &search, from, to, before_me, index);
    const int prefix = a.prefix_lens ? a.prefix_lens[it.s] : 0;
    const TileKeys keys = tile_keys(a, it, prefix);
    const Part mine = part_of((keys.end - keys.base + TK - 1) / TK, part, parts);
    const int32_t* table = a.batch.block_table + it.s * a.batch.table_stride;

    // my column's row: queries, range
    const int row = it.tile * kRows + wave * 32 + col, token = row / a.group, h = head * a.group + row - token * a.group;
    const bool live = row < it.rows;
    const int position = live ? it.span.total - it.span.n + token : -1;
    const KeyRange see = visible_keys(position, it.span.keys, a.window, prefix);
    const float slope = SHAPED && a.slopes && live ? a.slopes[h] : 0.0f;
    bf16x8 q[D / 16];
    float start = 0.0f;
    {
        // (a negative scale turns the queries round: what follows takes a scale of at least 0)
        const uint32_t sign = a.scale < 0.0f ? 0x80008000u : 0u;
        const uint16_t* from_q = a.q + (it.span.first + token) * a.q_stride + (int64_t)h * D;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            uint4 x = make_uint4(0, 0, 0, 0);
            if (live) x = *reinterpret_cast<const uint4*>(from_q + 16 * i + 8 * half);
            const uint32_t y[4] = {x.x ^ sign, x.y ^ sign, x.z ^ sign, x.w ^ sign};
            u32x4 z;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                z[j] = !Codes<BITS>::kPaired ? y[j] : __builtin_amdgcn_perm(y[2 + (j >> 1)], y[j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
                if constexpr (CODES) sum += as_f(y[j] << 16) + as_f(y[j] & 0xFFFF0000u);
            }
            q[i] = __builtin_bit_cast(bf16x8, z);
        }
        if constexpr (CODES) start = -kBias * join32(sum, SumOf());
    }
    // (at least the smallest normal number: minus infinity, in hidden places, has to stay what it is)
    const float scale = fabsf(a.scale), scale2 = fmaxf(scale * kLog2e, 1.17549435e-38f);
    // keys that all of the wave's rows see, and those that some does
    int all_lo = live ? see.lo : 0, all_hi = live ? see.hi : 0x7FFFFFFF, any_lo = see.hi > see.lo ? see.lo : 0x7FFFFFFF, any_hi = see.hi > see.lo ? see.hi : 0;
    for (int m = 1; m < 32; m <<= 1) {
        all_lo = max(all_lo, __shfl_xor(all_lo, m, 64));
        all_hi = min(all_hi, __shfl_xor(all_hi, m, 64));
        any_lo = min(any_lo, __shfl_xor(any_lo, m, 64));
        any_hi = max(any_hi, __shfl_xor(any_hi, m, 64));
    }
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    any_lo = __builtin_amdgcn_readfirstlane(any_lo);
    any_hi = __builtin_amdgcn_readfirstlane(any_hi);

    f32x16 o[D / 32], psum;
#pragma unroll
    for (int i = 0; i < 16; ++i) psum[i] = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = psum;
    float m = -INFINITY, l = 0.0f;

    auto page_of = [&](int key) {   // of a group of 16 keys; -1: none
        int p = -1;
        if (key < keys.end) p = table[key >> a.cache.page_shift];
        return (uint32_t)p < (uint32_t)a.cache.n_pages ? p : -1;
    };
    auto row_of = [&](int page, int key) {
        return (int64_t)page * a.cache.page_rows + ((int64_t)head << a.cache.page_shift) + (key & page_mask);
    };
    auto side = [&](int buffer, int which) { return lds + (2 * buffer + which) * SIDE; };
    float* const scales = reinterpret_cast<float*>(lds + 4 * SIDE);
    typedef __attribute__((address_space(3))) void lds_void;

    // 16 bits: rows of a tile to LDS, 1 KiB a wave and load.  A wave's rows lie in one page.
    uint32_t offset[2][NI];   // of my 16 bytes from the wave's first row; the place of a chunk in LDS and the chunk change roles here
#pragma unroll
    for (int i = 0; i < NI; ++i) {
        const int in_wave = i * RI + lane / (D / 8), r = wave * RW + in_wave, at = lane % (D / 8);
        offset[0][i] = k_place<D>(r, at) - wave * RW * (2 * D);
        offset[1][i] = v_place<D>(r, at) - wave * RW * (2 * D);
    }
    auto fetch16 = [&](int key0, int buffer) {
        const int first = key0 + wave * RW, page = __builtin_amdgcn_readfirstlane(page_of(first));
        const int64_t row0 = page < 0 ? 0 : row_of(page, first);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const uint8_t* from_row = (which ? a.cache.v : a.cache.k) + row0 * (2 * D);
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const uint32_t to = (uint32_t)(uintptr_t)(lds_void*)(side(buffer, which) + (wave * RW + i * RI) * (2 * D));
                if (page >= 0 && first + RW <= keys.end) {
                    gemm::lds_dma16(to, from_row, offset[which][i]);
                } else if (page >= 0 && first + i * RI + lane / (D / 8) < keys.end) {
                    gemm::lds_dma16(to, from_row, offset[which][i]);
                } else {   // (each lane's bytes land in the lane's place, whichever of the two copies takes them there)
                    gemm::lds_dma16(to, no_state, 16 * (lane % (D / 8)));
                }
            }
        }
    };
    // codes: a chunk of keys and one of values a thread (D = 64: the first half of the threads keys, the second values)
    constexpr bool BOTH = CHUNKS == kThreads;
    const int chunk = BOTH ? threadIdx.x : threadIdx.x % CHUNKS, chunk_row = chunk / CR, chunk_at = chunk % CR;
    uint32_t raw[2][CW];
    float raw_scale = 0.0f;
    auto fetch_codes = [&](int key0) {
        const int key = key0 + chunk_row, page = page_of(key);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (!BOTH && which == 1) continue;
            const uint8_t* pool = (BOTH ? which == 1 : (int)threadIdx.x >= CHUNKS) ? a.cache.v : a.cache.k;
#pragma unroll
            for (int i = 0; i < CW; ++i) raw[which][i] = 0;
            if (page >= 0) load_dwords<CW>(pool + row_of(page, key) * (D * BITS / 8) + chunk_at * (4 * BITS), raw[which]);
        }
        raw_scale = 0.0f;
        if ((int)threadIdx.x < 2 * TK) {
            const int k = key0 + (int)(threadIdx.x % TK), p = page_of(k);
            if (p >= 0) raw_scale = ((int)threadIdx.x < TK ? a.cache.k_scales : a.cache.v_scales)[row_of(p, k)];
        }
    };
    auto store_codes = [&](int buffer) {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (!BOTH && which == 1) continue;
            const bool values = BOTH ? which == 1 : (int)threadIdx.x >= CHUNKS;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int place = values ? v_place<D>(chunk_row, 4 * chunk_at + g) : k_place<D>(chunk_row, 4 * chunk_at + g);
                *reinterpret_cast<u32x4*>(side(buffer, values) + place) = widen_codes<BITS>(raw[which], g);
            }
        }
        if ((int)threadIdx.x < 2 * TK) scales[buffer * 2 * TK + threadIdx.x] = raw_scale;
    };

    if (mine.from < mine.to) {
        const int key0 = keys.base + mine.from * TK;
        if constexpr (CODES) {
            fetch_codes(key0);
            store_codes(0);
        } else {
            fetch16(key0, 0);
        }
    }
    gemm::wait_loads_then_barrier<0>();
    for (int t = mine.from; t < mine.to; ++t) {
        const int buffer = (t - mine.from) & 1, key0 = keys.base + t * TK;
        const bool more = t + 1 < mine.to;
        if (more) {
            if constexpr (CODES) fetch_codes(key0 + TK);
            else fetch16(key0 + TK, buffer ^ 1);
        }
        if (key0 < any_hi && key0 + TK > any_lo) {
            const char* const kt = side(buffer, 0);
            char* const vt = side(buffer, 1);
            f32x16 score[KB];
#pragma unroll
            for (int b = 0; b < KB; ++b) {
#pragma unroll
                for (int i = 0; i < 16; ++i) score[b][i] = start;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const bf16x8 kk = *reinterpret_cast<const bf16x8*>(kt + k_place<D>(32 * b + col, 2 * i + half));
                    score[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kk, q[i], score[b], 0, 0, 0);
                }
            }
            // element 4 j + i of block b is key 32 b + 8 j + 4 half + i
            if constexpr (CODES || SHAPED) {
#pragma unroll
                for (int b = 0; b < KB; ++b)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        f32x4 ks = {1, 1, 1, 1};
                        if constexpr (CODES) ks = *reinterpret_cast<const f32x4*>(scales + buffer * 2 * TK + 32 * b + 8 * j + 4 * half);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float x = score[b][4 * j + i];
                            if constexpr (CODES) x *= ks[i];
                            if constexpr (SHAPED) {
                                const int apart = position - (key0 + 32 * b + 8 * j + 4 * half + i);
                                x = shaped_score(x * scale, a.softcap, slope, apart < 0 ? -apart : apart);
                            }
                            score[b][4 * j + i] = x;
                        }
                    }
            }
            int absent = 0;   // groups of 16 keys without a page
#pragma unroll
            for (int g = 0; g < TK / 16; ++g)
                if (page_of(key0 + 16 * g) < 0) absent |= 1 << g;
            const bool plain = key0 >= all_lo && key0 + TK <= all_hi && absent == 0;
            if (!plain) {
#pragma unroll
                for (int b = 0; b < KB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int in_tile = 32 * b + 8 * (i >> 2) + 4 * half + (i & 3), j = key0 + in_tile;
                        if (j < see.lo || j >= see.hi || (absent >> (2 * b + (i >> 3)) & 1)) score[b][i] = -INFINITY;
                    }
            }
            float top = -INFINITY;
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, score[b][i]);
            const float unit = SHAPED ? 1.0f : scale2;
            top = join32(top, MaxOf());
            top = top == -INFINITY ? top : top * unit;
            // The reference stays until a maximum is far above it: weights up to 2^8 are as good as those up to 1.
            if (__any(top > m + 8.0f || (m == -INFINITY && top > m))) {
                const float to = fmaxf(m, top), keep = to > m ? __builtin_amdgcn_exp2f(m - to) : 1.0f;
                l *= keep;
                if constexpr (CODES) psum *= keep;
#pragma unroll
                for (int i = 0; i < D / 32; ++i) o[i] *= keep;
                m = to;
            }
            const float ref = m == -INFINITY ? 0.0f : -m;
            bf16x8 p[KB][2];
#pragma unroll
            for (int b = 0; b < KB; ++b) {
                uint32_t w[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float e[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = score[b][4 * j + i];
                        e[i] = __builtin_amdgcn_exp2f(SHAPED ? x + ref : __builtin_fmaf(x, unit, ref));
                        l += e[i];
                    }
                    if constexpr (CODES) {
                        const f32x4 vs = *reinterpret_cast<const f32x4*>(scales + buffer * 2 * TK + TK + 32 * b + 8 * j + 4 * half);
#pragma unroll
                        for (int i = 0; i < 4; ++i) e[i] = plain || e[i] > 0.0f ? e[i] * vs[i] : 0.0f;
                    }
                    w[2 * j] = pack_bf16(e[0], e[1]);
                    w[2 * j + 1] = pack_bf16(e[2], e[3]);
                }
                p[b][0] = __builtin_bit_cast(bf16x8, (u32x4){w[0], w[1], w[2], w[3]});
                p[b][1] = __builtin_bit_cast(bf16x8, (u32x4){w[4], w[5], w[6], w[7]});
            }
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if constexpr (CODES) {
                        const bf16x8 ones = __builtin_bit_cast(bf16x8, (u32x4){0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
                        psum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ones, p[b][c], psum, 0, 0, 0);
                    }
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {
                        uint32_t v[4];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            // each 16 lanes take 4 rows of 16 features: a lane gets a feature of them
                            const int r = 32 * b + 16 * c + 8 * e + 4 * half + ((lane & 15) >> 2);
                            const int byte = v_place<D>(r, 4 * i + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + 8 * (lane & 1);
                            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
                            const uint2 u = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vt + byte)));
                            v[2 * e] = u.x;
                            v[2 * e + 1] = u.y;
                        }
                        o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, (u32x4){v[0], v[1], v[2], v[3]}), p[b][c], o[i], 0, 0, 0);
                    }
                }
        }
        if constexpr (CODES)
            if (more) store_codes(buffer ^ 1);
        gemm::wait_loads_then_barrier<0>();
    }

    const float sum = join32(l, SumOf());
    const bool whole = parts == 1;
    const float inverse = whole ? (sum > 0.0f ? 1.0f / sum : 0.0f) : 1.0f;
    if (!live) return;
    const size_t slot_row = ((size_t)(index * heads + head) * parts + part) * kRows + wave * 32 + col;
    const size_t slots = (size_t)items * heads * parts;
    float* const part_o = a.partial;
    float2* const part_ml = reinterpret_cast<float2*>(a.partial + slots * kRows * D);
    if (!whole && half == 0) part_ml[slot_row] = make_float2(m, sum);
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // places 32 i + 8 j + 4 half on: where codes are paired, features 0 4 1 5 and 2 6 3 7 of the eight
            float y[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) y[x] = (o[i][4 * j + x] - kBias * psum[4 * j + x]) * inverse;
            if constexpr (Codes<BITS>::kPaired) {   // the halves exchange so that each has four in a row
                // half 0 has features 0 4 1 5, half 1 has 2 6 3 7; half 0 keeps 0 1 and gets 2 3, half 1 keeps 6 7 and gets 4 5
                const float give0 = half ? y[0] : y[1], give1 = half ? y[2] : y[3];
                const float got0 = __shfl_xor(give0, 32, 64), got1 = __shfl_xor(give1, 32, 64);
                const float a0 = half ? got0 : y[0], a1 = half ? got1 : y[2], a2 = half ? y[1] : got0, a3 = half ? y[3] : got1;
                y[0] = a0; y[1] = a1; y[2] = a2; y[3] = a3;
            }
            const int at = 32 * i + 8 * j + 4 * half;
            if (whole)
                *reinterpret_cast<uint2*>(a.out + (it.span.first + token) * a.out_stride + (int64_t)h * D + at) =
                    make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
            else
                *reinterpret_cast<f32x4*>(part_o + slot_row * D + at) = (f32x4){y[0], y[1], y[2], y[3]};
        }
}

// Joins the parts of one row tile and key head a workgroup.
__global__ __launch_bounds__(kThreads) void paged_prefill_join_kernel(AttentionArgs a, int parts, int tile) {
    __shared__ Search search;
    const int heads = a.cache.heads, index = blockIdx.x / heads, head = blockIdx.x - index * heads;
    int from, to, before_me;
    thread_share(a, from, to);
    const int items = count_row_tiles(a, &search, from, to, before_me);
    if (index >= items) return;
    const Item it = find_item(a, &search, from, to, before_me, index);
    const TileKeys keys = tile_keys(a, it, a.prefix_lens ? a.prefix_lens[it.s] : 0);
    const int tiles = (keys.end - keys.base + tile - 1) / tile;
    const size_t slots = (size_t)items * heads * parts, slot0 = ((size_t)index * heads + head) * parts;
    const float2* const part_ml = reinterpret_cast<const float2*>(a.partial + slots * kRows * a.d);
    const int rows = min(kRows, it.rows - it.tile * kRows);
    for (int i = threadIdx.x; i < rows * (a.d / 4); i += kThreads) {
        const int r = i / (a.d / 4), at = 4 * (i - r * (a.d / 4)), row = it.tile * kRows + r;
        const int token = row / a.group, h = head * a.group + row - token * a.group;
        float top = -INFINITY, total = 0.0f;
        f32x4 y = {0, 0, 0, 0};
        for (int x = 0; x < parts; ++x) top = fmaxf(top, part_ml[(slot0 + x) * kRows + r].x);
        for (int x = 0; x < parts && top > -INFINITY; ++x) {
            const Part p = part_of(tiles, x, parts);
            if (p.from == p.to) continue;
            const size_t at_row = (slot0 + x) * kRows + r;
            const float2 ml = part_ml[at_row];
            const float f = __builtin_amdgcn_exp2f(ml.x - top);
            total += f * ml.y;
            y += f * *reinterpret_cast<const f32x4*>(a.partial + at_row * a.d + at);
        }
        const float inverse = total > 0.0f ? 1.0f / total : 0.0f;
        *reinterpret_cast<uint2*>(a.out + (it.span.first + token) * a.out_stride + (int64_t)h * a.d + at) =
            make_uint2(pack_bf16(y[0] * inverse, y[1] * inverse), pack_bf16(y[2] * inverse, y[3] * inverse));
    }
}

// Row tiles that a call may have (the host knows no lengths): whole ones, and an incomplete one a sequence.
int64_t most_row_tiles(int64_t T, int n_seqs, int group) {
    const int64_t rows = T * group, seqs = n_seqs < T ? n_seqs : T;
    return rows / kRows + seqs;
}
// Parts of the keys: until there are two workgroups for each of the 256 CUs, and at most eight.
int key_parts(int64_t T, int n_seqs, int group, int heads) {
    const int64_t wgs = most_row_tiles(T, n_seqs, group) * heads;
    int parts = 1;
    while (parts < 8 && wgs * parts * 2 <= 640) parts *= 2;
    return parts;
}

template <int D, int BITS>
int launch_form(const AttentionArgs& a, hipStream_t stream) {
    constexpr size_t lds = (size_t)4 * kTile<D> * D * 2 + (BITS == 16 ? 0 : 4 * kTile<D> * sizeof(float));
    const int heads = a.cache.heads, parts = key_parts(a.T, a.batch.n_seqs, a.group, heads);
    const int64_t tiles = most_row_tiles(a.T, a.batch.n_seqs, a.group);
    const int64_t wgs = tiles * parts * heads;
    if (wgs > 0x7FFFFFFF) return HBL_E_SHAPE;
    if (a.softcap > 0.0f || a.slopes) {
        if (int rc = allow_dynamic_lds<&paged_prefill_kernel<D, BITS, true>, lds>(); rc != HBL_OK) return rc;
        launch_kernel("paged_prefill_kernel", paged_prefill_kernel<D, BITS, true>, dim3((unsigned)wgs), dim3(kThreads), lds, stream, a, parts);
    } else {
        if (int rc = allow_dynamic_lds<&paged_prefill_kernel<D, BITS, false>, lds>(); rc != HBL_OK) return rc;
        launch_kernel("paged_prefill_kernel", paged_prefill_kernel<D, BITS, false>, dim3((unsigned)wgs), dim3(kThreads), lds, stream, a, parts);
    }
    if (parts > 1)
        launch_kernel("paged_prefill_join_kernel", paged_prefill_join_kernel, dim3((unsigned)(tiles * heads)), dim3(kThreads), 0, stream, a, parts,
                      kTile<D>);
    return after_launch();
}
template <int D>
int launch_bits(const AttentionArgs& a, int bits, hipStream_t stream) {
    switch (bits) {
        case 16: return launch_form<D, 16>(a, stream);
        case 8: return launch_form<D, 8>(a, stream);
        case 4: return launch_form<D, 4>(a, stream);
        default: return launch_form<D, 3>(a, stream);
    }
}

}  // namespace

size_t paged_prefill_workspace(int64_t T, int n_seqs, int group, int heads, int d) {
    const int parts = key_parts(T, n_seqs, group, heads);
    return parts == 1 ? 0 : (size_t)(most_row_tiles(T, n_seqs, group) * heads * parts) * kRows * (d + 2) * sizeof(float);
}

int launch_paged_prefill(const AttentionArgs& a, int bits, hipStream_t stream) {
    return a.d == 64 ? launch_bits<64>(a, bits, stream) : a.d == 128 ? launch_bits<128>(a, bits, stream) : launch_bits<256>(a, bits, stream);
}

}  // namespace hbl
