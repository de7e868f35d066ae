// Attention of packed sequences over bf16 keys and values: what api.hip and the kernels share.
#pragma once
#include "qvggt_common.h"

namespace qvggt {

struct Attention {
    const uint16_t *q, *k, *v;
    long long q_stride, k_stride, v_stride;     // elements from token to token
    int T, S, q_heads, kv_heads;
    float scale;
    int causal;
    const int32_t *q_starts, *kv_starts, *kv_lens;      // kv_lens == nullptr: kv_starts has an end for every sequence
    int seqs, max_q, max_kv;
    uint16_t *out;
    void *workspace;
};
hipError_t run_attention(const Attention &a, int d, hipStream_t stream);

}  // namespace qvggt
