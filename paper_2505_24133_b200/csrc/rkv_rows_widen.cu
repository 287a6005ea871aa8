// 8-bit caches for the rows' tensor-core kernel: the key tiles that a call sees, once, as bf16 (exactly: every E4M3 value is a bf16 value).
//
// Bound by HBM: one byte read and two written per element.  A prompt's products take far longer (8000 tokens of 8 KV heads: 16 MB written,
// 2 * 4 * 8000^2 * 4096 flops), and the widening of a tile is done once, not by every block that uses it.  Of a few tokens over long caches it is most of
// the call: five times the cache's bytes (2 new tokens of each of 64 sequences of 8000 rows, 8 heads: 949 us, 350 over bf16 caches).
#include "rkv_tokens.cuh"

namespace rkv {

namespace {

constexpr int kWidenThreads = 256;

template <int kDim>
__global__ void __launch_bounds__(kWidenThreads) widen_rows_kernel(RowsParams p, uint4 *wide, int tiles)
{
    pdl_wait();
    pdl_trigger();                                           // (in this order: see AttendTcMore::late)
    const int head = blockIdx.x / tiles, i = blockIdx.x % tiles, b = head / p.hkv;
    int first;
    const int n = token_span(p.tokens, b, &first), len = p.lens[b];
    if (n <= 0 || len <= 0 || len > p.cap || (p.causal && len < n)) return;
    const CallTiles call = call_tiles(p.causal, p.window, p.sinks, len, n);
    if (i >= call.count) return;
    const int t = call.tile(i);
    const long long start = rows_tile_start(p, head, t);
    if (start < 0 && threadIdx.x == 0) report(p.status, RKV_ERR_INVALID_ARG);
    constexpr int kVecs = kDim / 16, kPer = kTile * kVecs / kWidenThreads;        // vectors of a row; of a tile per thread
    const size_t all = (size_t)p.tokens.count * p.hkv * tiles * kTile * kVecs * 2;
    uint4 codes[2][kPer];
#pragma unroll
    for (int kv = 0; kv < 2; ++kv)
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int x = e * kWidenThreads + threadIdx.x, row = x / kVecs;
            codes[kv][e] = make_uint4(0u, 0u, 0u, 0u);
            if (start >= 0 && call.wanted(t * kTile + row, len))
                codes[kv][e] = reinterpret_cast<const uint4 *>(kv ? p.v : p.k)[(size_t)(start + row) * kVecs + x % kVecs];
        }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv)
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            uint4 *to = wide + kv * all + ((size_t)blockIdx.x * kTile * kVecs + e * kWidenThreads + threadIdx.x) * 2;
            widen16(codes[kv][e], to, to + 1);
        }
}

}  // namespace

cudaError_t launch_rows_widen(RowsParams *p, void *wide, int tiles, cudaStream_t s)
{
    const long long blocks = (long long)p->tokens.count * p->hkv * tiles;
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    const cudaError_t e = launch_early(p->d == 64 ? widen_rows_kernel<64> : widen_rows_kernel<128>, (unsigned)blocks, kWidenThreads, 0, s, 1, *p,
                                       static_cast<uint4 *>(wide), tiles);
    p->k = wide;
    p->v = static_cast<char *>(wide) + (size_t)blocks * kTile * p->d * sizeof(__nv_bfloat16);
    p->block_table = nullptr;
    p->compact_tiles = tiles;
    return e;
}

}  // namespace rkv
