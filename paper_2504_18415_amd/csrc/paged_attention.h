// What the kernels of paged_attention.hip and its companions take.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged.h"

namespace hbl {

struct AttentionArgs {
    const uint16_t* q;      // bf16, [T][Hq][d], q_stride values between two tokens
    uint16_t* out;          // bf16, likewise
    int64_t q_stride, out_stride;
    PagedCache cache;
    PagedBatch batch;
    const float* slopes;          // [Hq] or nullptr
    const int32_t* prefix_lens;   // [n_seqs] or nullptr
    float scale, softcap;
    int T, group, d, window;      // group: query heads of a key head
};

// Bytes of workspace of a call (T tokens, n_seqs sequences, Hq / Hkv heads of d).
size_t paged_attention_workspace(int64_t T, int n_seqs, int Hq, int Hkv, int d, int64_t max_q_len);
int launch_paged_attention(const AttentionArgs& a, int bits, int64_t max_q_len, void* workspace, hipStream_t stream);

}  // namespace hbl
