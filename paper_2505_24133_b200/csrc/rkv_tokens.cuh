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

// ---- attention of many query rows: "problems" (sequences, or prefixes), each a run of query tokens over one cache ----------------------
// The rows of a problem and KV head are its tokens' G query heads, token after token: row r is head r % G of token r / G.
struct RowsParams {
    const void *q;                  // [total][hq][d], q_stride elements from token to token
    long long q_stride, out_stride;
    const void *k, *v;              // [count][hkv][cap][d], or pools
    const int32_t *lens;            // [count]
    const int32_t *block_table;
    long long pool_pages;
    TokenMap tokens;                // count = problems
    int hkv, hq, group, d, cap;
    int causal, window, sinks;      // causal: token t of n stands in row len - n + t and sees rows up to its own; else every token sees all rows
    int compact_tiles;              // > 0: k and v are [count][hkv][compact_tiles][128][d], the tiles that the call sees (CallTiles), in turn
    int splits, slot, slots;        // blocks that share a row tile's keys; their partial results are slots slot .. of the rows' `slots`
    float *part;                    // [total * hq][slots][d + 4]: weighted sum, maximum (base 2), sum of weights; null: `out` is written
    void *out;
    int32_t *status;
    long long wait_cycles;
};
__host__ __device__ constexpr int slot_floats(int d) { return d + 4; }        // (whole 16-byte vectors)
// The key tiles of 128 rows that tokens t0 .. t1 of a problem look at: the first `sink_tiles`, then those from `first` on.
struct KeyTiles {
    int sink_tiles, first, count;
    int lo, hi, sinks;              // rows seen by some of the tokens: [0, sinks) and [lo, hi)
    __device__ __forceinline__ int tile(int i) const { return i < sink_tiles ? i : first + i - sink_tiles; }
    __device__ __forceinline__ bool wanted(int row) const { return row < sinks || (row >= lo && row < hi); }
};
__device__ __forceinline__ KeyTiles key_tiles(int causal, int window, int sinks, int len, int n, int t0, int t1)
{
    KeyTiles k;
    k.hi = causal ? len - n + t1 + 1 : len;
    k.lo = causal && window > 0 ? max(0, len - n + t0 + 1 - window) : 0;
    k.sinks = causal && window > 0 ? min(sinks, k.hi) : 0;
    k.first = k.lo / kTile;
    k.sink_tiles = min((k.sinks + kTile - 1) / kTile, k.first);
    k.count = k.sink_tiles + (k.hi + kTile - 1) / kTile - k.first;
    if (k.hi <= 0) k.count = 0;
    return k;
}
// The same for all tokens of a problem: rows [0, sinks) and [lo, len).
struct CallTiles {
    int sink_tiles, first, count, lo, sinks;
    __device__ __forceinline__ int tile(int i) const { return i < sink_tiles ? i : first + i - sink_tiles; }
    __device__ __forceinline__ int place(int t) const { return t < sink_tiles ? t : sink_tiles + t - first; }
    __device__ __forceinline__ bool wanted(int row, int len) const { return row < sinks || (row >= lo && row < len); }
};
__device__ __forceinline__ CallTiles call_tiles(int causal, int window, int sinks, int len, int n)
{
    const KeyTiles k = key_tiles(causal, window, sinks, len, n, 0, n - 1);
    return CallTiles{k.sink_tiles, k.first, k.count, k.lo, k.sinks};
}
// Rows of a cache: where 128-row tile t of a head starts, or -1 for a page that does not exist.
__device__ __forceinline__ long long rows_tile_start(const RowsParams &p, int head, int t)
{
    if (!p.block_table) return (long long)head * p.cap + (long long)t * kTile;
    const int page = p.block_table[(size_t)head * (p.cap / kTile) + t];
    return page < 0 || page >= p.pool_pages ? -1 : (long long)page * kTile;
}
// 8-bit caches: the tiles that a call sees, as bf16, rows that it does not see as zeros; `wide` holds K's, then V's.  `p` becomes the call on them.
cudaError_t launch_rows_widen(RowsParams *p, void *wide, int tiles, cudaStream_t s);
int rows_simt_rows(const RowsParams &p);
cudaError_t launch_rows_simt(const RowsParams &p, int dtype, cudaStream_t s);
bool rows_sm100_supported(int dtype, int d, int group);
int rows_sm100_tiles(const RowsParams &p);                  // row tiles of a block
cudaError_t launch_rows_sm100(const RowsParams &p, cudaStream_t s);
// One token per problem by the decode attention's kernel (rkv_attend_tc.cuh): K and V at the rate that memory gives.  p.slots > 0: slots of
// other kernels, and of the splits where they are blocks of their own (then the merge kernel follows); `late`: the kernel before this one
// leaves those slots and lets this one in only when everything before itself is done.
bool attend_more_supported(int dtype, int d, int group, long long tiles);
void attend_more_plan(RowsParams *p, int dtype, long long tiles, int sms, bool others, bool *separate);
// `prefix`: prefixes that the kernel reads itself, in front of every sequence's own rows; null: none.
cudaError_t launch_attend_more(const RowsParams &p, int dtype, long long tiles, bool separate, int others, bool late, const RowsParams *prefix,
                               cudaStream_t s);
int attend_f32_more_splits(int heads, long long rows, int sms);
cudaError_t launch_attend_f32_more(const RowsParams &p, bool separate, const RowsParams *prefix, cudaStream_t s);      // (fp32 caches)
cudaError_t launch_rows_merge(const RowsParams &p, int dtype, cudaStream_t s);

}  // namespace rkv
