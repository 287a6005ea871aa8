// What the calls on several new tokens per sequence share: where a sequence's tokens lie, and the launches of their kernels.
#pragma once

#include "rkv_common.cuh"

namespace rkv {

// The packed new tokens of a call (rkv_tokens_t) as the kernels see them.
struct TokenMap {
    const int32_t *offsets;     // [count + 1], or null: `longest` each
    int count, total, longest;
};

// Rows [first, first + n) of the token tensors are sequence b's; n = -1 for entries that are no such range.
__device__ __forceinline__ int token_span(const TokenMap &m, int b, int *first)
{
    if (!m.offsets) {
        *first = b * m.longest;
        return m.longest;
    }
    const int lo = m.offsets[b], hi = m.offsets[b + 1];
    *first = lo;
    return lo < 0 || hi < lo || hi > m.total || hi - lo > m.longest ? -1 : hi - lo;
}

struct RotaryParams {
    void *k_cache, *v_cache;
    const void *k_new, *v_new, *q_new;
    void *q_out;
    long long k_stride, v_stride, q_stride, out_stride;     // elements from token to token
    int32_t *seq_lens;
    int hkv, hq;                // hq = 0: no queries
    int d, cap;
    TokenMap tokens;
    const float *table;
    int rows, dim, interleaved;
    const int32_t *positions;
    const int32_t *block_table;
    long long pool_pages;
    int32_t *status;
    int warps_per_token;
};
cudaError_t launch_append_rotary(RotaryParams p, int dtype, cudaStream_t s);

}  // namespace rkv
