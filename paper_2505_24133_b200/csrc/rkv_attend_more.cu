// Decode-step attention for single tokens that see part of their cache, or a shared prefix as well: on the tensor cores (rkv_attend_tc.cuh), and for
// fp32 caches rkv_attend.cu.
#include "rkv_attend_tc.cuh"

namespace rkv {

namespace {

int source_of(int dtype, int d) { return dtype == RKV_FP8_E4M3 ? 1 : d == 64 ? 2 : 0; }

}  // namespace

// `tiles`: key tiles that a token sees at most: 448, what blocks of two chunks in a cluster take (the rows' kernel takes longer ones).
bool attend_more_supported(int dtype, int d, int group, long long tiles)
{
    return attend_supported(group, dtype, d) && tiles <= (dtype == RKV_F32 ? 1ll << 23 : (long long)kTcMaxSplits * 2 * kTcChunkTiles);
}

// Splits as for rkv_decode_attention.  They are a cluster, but beside another kernel, where not all blocks are on the GPU at a time, blocks of their
// own: one that waited for the other kernel's results would keep the next block out (256 sequences of 1152 rows and four prefixes of 16000:
// 259 us, 238 with a merge kernel; 64 of 580 and one of 2048: 60, 45).  Nor are they where the keys of many heads go to more blocks than a cluster
// has (from 241 tiles on; 128 heads of 32768 rows, 18 shares each: 307 us, 7.0 TB/s, of 8-bit caches 166 us).
void attend_more_plan(RowsParams *p, int dtype, long long tiles, int sms, bool others, bool *separate)
{
    const int heads = p->tokens.count * p->hkv;
    if (dtype == RKV_F32) {
        p->splits = attend_f32_more_splits(heads, tiles * kTile, sms);
        *separate = others || p->splits > 1;
        return;
    }
    p->splits = attend_tc_splits(heads, (int)tiles * kTile, sms);
    *separate = p->splits > kTcMaxSplits || (others && (long long)heads * p->splits > 2ll * sms);
}

cudaError_t launch_attend_more(const RowsParams &r, int dtype, long long tiles, bool separate, int others, bool late, const RowsParams *prefix,
                               cudaStream_t s)
{
    if (dtype == RKV_F32) return launch_attend_f32_more(r, separate, prefix, s);
    AttendTcMore p = {};
    p.seq_lens = r.lens;
    p.out = static_cast<float *>(r.out);         // (of bf16)
    p.separate = separate ? 1 : 0;
    p.hkv = r.hkv;
    p.hq = r.hq;
    p.cap = r.cap;
    p.splits = r.splits;
    p.tiles_per_split = (int)((tiles + r.splits - 1) / r.splits);
    p.status = r.status;
    p.wait_cycles = r.wait_cycles;
    p.block_table = r.block_table;
    p.least = r.causal ? 1 : 0;
    p.window = r.window;
    p.sinks = r.sinks;
    p.pool_pages = r.pool_pages;
    p.slots = r.part;
    p.slots_per_row = r.slots;
    p.others = others;
    p.late = late ? 1 : 0;
    if (p.tiles_per_split > 2 * kTcChunkTiles) return cudaErrorInvalidValue;
    AttendTcMoreMaps maps;
    p.per_prefix = 1;
    if (prefix) {
        p.prefix_lens = prefix->lens;
        p.prefix_table = prefix->block_table;
        p.prefix_pages = prefix->pool_pages;
        p.prefix_cap = prefix->cap;
        p.per_prefix = prefix->tokens.longest;
    }
    // (without prefixes the maps of their tiles are never looked at)
    const RowsParams &x = prefix ? *prefix : r;
    const uint64_t rows = x.block_table ? (uint64_t)x.pool_pages * kTile : (uint64_t)x.tokens.count * x.hkv * x.cap;
    if (!make_cache_map(&maps.prefix_k, x.k, rows, source_of(dtype, r.d)) || !make_cache_map(&maps.prefix_v, x.v, rows, source_of(dtype, r.d)))
        return cudaErrorInvalidValue;
    return launch_tc_group(p, maps, r.k, r.v, r.q, r.tokens.count, r.pool_pages, source_of(dtype, r.d), s);
}

}  // namespace rkv
