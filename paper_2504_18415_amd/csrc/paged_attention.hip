// Attention of new tokens against the paged cache.  One workgroup a (token, query head): its four waves take 64 keys in turn, a key a
// lane for the scores, then a feature a lane for the sums; maxima, sums and outputs of the waves are joined in LDS.
#include "hbl_internal.h"
#include "kv_codes.h"
#include "paged.h"
#include "paged_attention.h"

namespace hbl {
namespace {

template <int BITS>
__device__ __forceinline__ float state(const uint8_t* pool, int64_t row, int d, int i) {
    if constexpr (BITS == 16) {
        return as_f((uint32_t) reinterpret_cast<const uint16_t*>(pool)[row * d + i] << 16);
    } else {
        const uint8_t* p = pool + row * (d * BITS / 8);
        const int bit = BITS * i, in = bit & 7;
        uint32_t w = p[bit >> 3];
        if (in + BITS > 8) w |= (uint32_t)p[(bit >> 3) + 1] << 8;
        return (float)(int)((w >> in) & ((1 << BITS) - 1)) - (float)(1 << (BITS - 1));
    }
}

template <int BITS>
__global__ __launch_bounds__(256) void paged_attention_kernel(AttentionArgs a) {
    __shared__ float part[4][256 + 2];
    const int t = blockIdx.x, head = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int s = -1;
    for (int i = 0; i < a.batch.n_seqs; ++i)
        if (a.batch.q_starts[i] <= t) s = i;
    if (s < 0) return;
    const SeqSpan span = span_of(a.batch, a.cache.page_shift, a.T, s);
    if (t - span.first >= span.n) return;
    const int position = span.total - span.n + t - span.first, h = head / a.group;
    const KeyRange see = visible_keys(position, span.keys, a.window, a.prefix_lens ? a.prefix_lens[s] : 0);
    const uint16_t* q = a.q + t * a.q_stride + head * a.d;
    const float slope = a.slopes ? a.slopes[head] : 0.0f;
    float m = -INFINITY, l = 0.0f, o[4] = {0, 0, 0, 0};
    for (int j0 = see.lo + 64 * wave; j0 < see.hi; j0 += 256) {
        const int j = j0 + lane;
        const int64_t row = j < see.hi ? key_row(a.cache, a.batch, s, j, h) : -1;
        float x = -INFINITY, vs = 0.0f;
        if (row >= 0) {
            float dot = 0.0f;
            for (int i = 0; i < a.d; ++i) dot += as_f((uint32_t)q[i] << 16) * state<BITS>(a.cache.k, row, a.d, i);
            if (BITS != 16) dot *= a.cache.k_scales[row];
            x = dot * a.scale;
            if (a.softcap > 0.0f) x = a.softcap * tanhf(x / a.softcap);
            x -= slope * fabsf((float)(position - j));
            vs = BITS != 16 ? a.cache.v_scales[row] : 1.0f;
        }
        float top = x;
        for (int k = 1; k < 64; k <<= 1) top = fmaxf(top, __shfl_xor(top, k, 64));
        if (top == -INFINITY) continue;
        const float m2 = fmaxf(m, top), keep = expf(m - m2), p = expf(x - m2);
        float sum = p;
        for (int k = 1; k < 64; k <<= 1) sum += __shfl_xor(sum, k, 64);
        l = l * keep + sum;
        m = m2;
        for (int c = 0; c < 4; ++c) o[c] *= keep;
        for (int k = 0; k < 64; ++k) {
            const int64_t r = __shfl(row, k, 64);
            if (r < 0) continue;
            const float w = __shfl(p * vs, k, 64);
            for (int c = 0; c < a.d / 64; ++c) o[c] += w * state<BITS>(a.cache.v, r, a.d, 64 * c + lane);
        }
    }
    for (int c = 0; c < a.d / 64; ++c) part[wave][64 * c + lane] = o[c];
    part[wave][256] = m;
    part[wave][257] = l;
    __syncthreads();
    if ((int)threadIdx.x >= a.d) return;
    float top = -INFINITY, sum = 0.0f, y = 0.0f;
    for (int w = 0; w < 4; ++w) top = fmaxf(top, part[w][256]);
    if (top > -INFINITY)
        for (int w = 0; w < 4; ++w) {
            const float keep = expf(part[w][256] - top);
            sum += keep * part[w][257];
            y += keep * part[w][threadIdx.x];
        }
    typedef __bf16 bf16;
    reinterpret_cast<bf16*>(a.out)[t * a.out_stride + head * a.d + threadIdx.x] = (bf16)(sum > 0.0f ? y / sum : 0.0f);
}

}  // namespace

size_t paged_attention_workspace(int64_t, int, int Hq, int Hkv, int d, int64_t max_q_len) {
    const int64_t rows = max_q_len * (Hq / Hkv);
    return rows <= kDecodeRows ? round_up(paged_decode_workspace((int)rows, d), 256) : 256;
}

int launch_paged_attention(const AttentionArgs& args, int bits, void* workspace, hipStream_t stream) {
    AttentionArgs a = args;
    a.partial = static_cast<float*>(workspace);
    if ((int64_t)a.max_q * a.group <= kDecodeRows) return launch_paged_decode(a, bits, stream);
    const dim3 grid((unsigned)a.T, (unsigned)(a.group * a.cache.heads)), block(256);
    auto kern = bits == 16 ? paged_attention_kernel<16> : bits == 8 ? paged_attention_kernel<8> : bits == 4 ? paged_attention_kernel<4> : paged_attention_kernel<3>;
    launch_kernel("paged_attention_kernel", kern, grid, block, 0, stream, a);
    return after_launch();
}

}  // namespace hbl
