// Decode-step attention over the compressed cache (Section 3.1, Eq. 1 with one query row per head), tensor-core form
// for bf16 and 8-bit caches with d = 128:
//
//   out[b][q] = sum_j softmax_j( q_new[b][q] . K[b][q / G][j] / sqrt(d) ) V[b][q / G][j],   j < seq_lens[b]
//
// The work is HBM-bound (every cached K and V row is read once), but with G query heads per KV head a CUDA-core
// kernel spends 4 G d fp32 operations per 512 bytes and runs out of issue slots from G = 5 on.  Here the two
// contractions go to the tensor cores, with the keys -- not the G <= 8 queries -- as the 128-row M dimension:
//
//   scores   S^T [128 keys x 16] = K_tile [128 x d] . Q^T [d x 16]     (K-major operands; the group's queries, padded to
//            N = 16, are the B operand; one accumulator of 16 TMEM columns PER key tile of the block)
//   values   O^T [d x 16] += V_tile^T [d x 128 keys] . P [128 keys x 16]   (the V tile as TMA leaves it, used transposed:
//            MN-major A operand; P = the softmax weights in bf16, written to shared memory by the softmax threads)
//
// A block owns one (KV head, split of the key tiles) with at most 15 tiles, or two chunks of up to 14 that go through the following
// one after the other.  First all its K tiles stream through the
// ring and leave their scores in TMEM (16 columns each, 240 at most, beside the 16 output columns); then the exact
// maximum per query over the whole split is taken, so the weights need no running rescale; then the V tiles stream
// through the same ring while the softmax threads turn score columns into P tiles (double-buffered).  Every weight
// is split into two bf16 parts (rows g and 8 + g of P: N = 16 has the room), so the products carry fp32-accurate
// weights; the sum of the weights is taken from the same parts.  The splits of a head are one thread-block cluster: each
// leaves its partial result in its shared memory, then every block merges a share of the outputs from all of them (a merge
// kernel of its own behind this one took 4 us of a decode step's 33 per layer).  Where the tiles pass through the softmax threads
// (8-bit caches, 64 dimensions) and the blocks queue up, the splits are blocks of their own all the same and leave their
// partial results in the workspace for that kernel: a cluster holds its SMs until its slowest block is done, and starts when all
// of its blocks fit (4096 heads of 4224 tokens, 3 splits: 8-bit 1267 us as clusters, 1116 as blocks; 64 dimensions 1065, 925; bf16 of
// 128 dimensions, whose blocks end together, 1204, 1243).
//
// Warps 0..3: softmax (thread = TMEM lane = key row of a tile, later = output dimension), warp 4: TMA producer,
// warp 5: MMA issuer and TMEM owner.
//
// 8-bit caches (E4M3 codes, kFp8): the tiles arrive as 128 rows of 128 bytes (a ring of two 16 KB stages) and are
// widened into one of two bf16 operand tiles by the softmax threads, one row each, on their way to the tensor cores
// (four raw stages and a single operand tile were measured slower: the chain widen -> product must not serialise); everything else is the same, at half the bytes per cached
// row.  Rows beyond the length are written as zeros there.
//
// 8-bit caches, as they are stored (kCodes, the calls of AttendTcMore): with bf16 operands the chain widen -> product of a block bounds the
// call at 4 TB/s, so here both products take the codes themselves (kind::f8f6f4; products of codes are exact, the accumulators fp32), and the other
// operands come in parts that add up to them.  A query row is scaled by a power of two to a largest element in [128, 256) and has two E4M3 parts, hi
// and 16 times what hi left, in the rows g and 8 + g that the bf16 weights' two parts take: four bits each hold a bf16 number exactly, elements below
// 2^-13 of the largest to 2^-21 of it, which moves a score by less than its fp32 sum may be off by.  A weight times 2^15 is rounded to fp16 (2^-11 of
// itself down to 2^-29, 2^-40 below) and that is held exactly in four E5M2 parts, each the upper byte of 8 times what the one before left, in the
// rows g, 8 + g, 16 + g and 24 + g (N = 32); the sum of the weights is taken from the fp16 numbers.  (Two E4M3 parts lose weights below 2^-22, and with them
// the whole output where a row whose values are small has nearly all of the weight.  64 sequences x 8 heads of 4224 rows, two parts and these: four queries
// to a head 102.0 us, 102.3; eight 116, 124.)
// The output's 32 columns lie over score columns that have been read: tile 0's, and of a second chunk tiles 0's and 1's.
//
// Of 64 dimensions, as they are stored (kHalf, the calls of AttendTcMore): the tiles go to the tensor cores as they land, too, keys as four steps of 16
// columns, values as the lower half of M.
//
// Every mbarrier wait is bounded; on expiry the block records RKV_ERR_TIMEOUT,
// writes zeros and leaves through the common exit that frees TMEM.  No TMA multicast.
#pragma once

#include <type_traits>

#include "rkv_sm100.cuh"
#include "rkv_tokens.cuh"

namespace rkv {

namespace {

using namespace sm100;

constexpr int kTcThreads = 192;
constexpr int kTcStages = 3;                         // ring of key / value tiles
constexpr int kTcMaxTiles = 15;                      // key tiles per block in one chunk
constexpr int kTcChunkTiles = 14;                    // ... and in each of two
constexpr int kTcMaxSplits = 16;                     // blocks of a cluster
constexpr int kTcHalf = kTile * 64 * 2;              // one TMA box: 128 rows x 64 bf16
constexpr int kTcTileBytes = 2 * kTcHalf;            // 32 KB
constexpr int kTcSmall = 16 * kHeadDim * 2;          // a [16 x 128] bf16 operand (Q^T or P): two [16 x 64] halves of 2 KB
constexpr uint32_t kTcTmemCols = 256;                // 16 (output) per chunk + 16 per key tile of a chunk

constexpr int kOffRing = 0;                          // bf16 caches: kTcStages tiles.  8-bit caches: kConvBufs widened tiles,
constexpr int kConvBufs = 2;
constexpr int kRawStages = 2;
constexpr int kCodeStages = 6;                       // ring of 16 KB tiles as they are stored, in the room of kTcStages of 32 KB
constexpr int kOffRaw = kConvBufs * kTcTileBytes;    // then kRawStages raw stages of 16 KB
constexpr int kRawBytes = kTile * kHeadDim;          // a tile of E4M3 codes
constexpr int kOffQ = kOffRing + kTcStages * kTcTileBytes;
static_assert(kOffRaw + kRawStages * kRawBytes <= kOffQ, "the 8-bit layout fits the room of the ring");
constexpr float kCodeWeight = 32768.f;               // kCodes: what the weights are multiplied by
// two buffers.  kCodes: [32 x 128] codes each; the queries' parts, [16 x 128] codes, take the queries' place
constexpr int kOffP = kOffQ + kTcSmall;
constexpr int kOffRed = kOffP + 2 * kTcSmall;        // [4 warps][8] floats: reductions over the softmax threads
constexpr int kOffBars = kOffRed + 4 * 8 * 4;
enum {
    kBarFull = 0,                        // [kTcStages] tile landed
    kBarEmpty = kBarFull + kTcStages,    // [kTcStages] tile read by the tensor cores
    kBarQ = kBarEmpty + kTcStages,       // queries landed
    kBarScores,                          // every score column of the split is in TMEM
    kBarPFull,                           // [2] P tile written (128 softmax threads)
    kBarPEmpty = kBarPFull + 2,          // [2] ... read by the tensor cores
    kBarOut = kBarPEmpty + 2,            // the output columns are final
    kBarRawFull,                                 // [kRawStages] 8-bit caches: codes landed
    kBarRawEmpty = kBarRawFull + kRawStages,     // [kRawStages] ... widened (128 softmax threads)
    kBarCodeFull = kBarRawEmpty + kRawStages,    // [kCodeStages] codes as they are stored: tile landed
    kBarCodeEmpty = kBarCodeFull + kCodeStages,  // [kCodeStages] ... read by the tensor cores
    kBarCodeQ = kBarCodeEmpty + kCodeStages,     // the queries' parts are written (128 softmax threads)
    kTcNumBars
};
constexpr int kOffMisc = kOffBars + kTcNumBars * 8;  // TMEM base, abort flag
constexpr int kTcSmem = kOffMisc + 16 + 1024;        // + slack for the 1024-byte alignment
static_assert(2 * (kTcSmem + 1024) <= 227 * 1024, "two blocks per SM");
static_assert(16 + 16 * kTcMaxTiles <= (int)kTcTmemCols && 32 + 16 * kTcChunkTiles <= (int)kTcTmemCols, "TMEM columns");

struct AttendTcParams {          // (64 bytes: the tensor maps behind it start at the next multiple of 64)
    const int32_t *seq_lens;
    float *out;                 // [batch][hq][d]; separate: [P][splits][G][d + 2], the splits' partial results
    int separate;               // the splits are blocks of their own, not a cluster
    int hkv, hq, cap, splits, tiles_per_split;
    int32_t *status;
    long long wait_cycles;
    const int32_t *block_table; // paged caches: [P][cap / 128] page ids, else null
};

// The same for rkv_window_attention's single tokens and for the sequences' own rows of rkv_prefix_attention: the output in bf16, only the key
// tiles that the token sees, and other partial results of the same softmax to be merged with.
struct AttendTcMore : AttendTcParams {
    int least;                  // a length below it is an error
    int window, sinks;          // the token sees rows L - window .. L - 1 (0: all) and 0 .. sinks - 1
    long long pool_pages;
    float *slots;               // [batch][hq][slots_per_row][d + 4]: what other kernels (and, with `separate`, the splits) leave
    int slots_per_row, others;  // others: slots 0 .. others - 1 are there when the kernel before this one is done
    // prefixes that stand in front of the sequences' own rows (as rkv_prefix_t; sequence b has prefix b / per_prefix); prefix_lens null: none
    const int32_t *prefix_lens, *prefix_table;
    long long prefix_pages;
    int prefix_cap, per_prefix;
    int late;                   // everything but those slots and the output was there when this kernel could start
};

// The tensor maps of a launch.
struct AttendTcMaps {
    CUtensorMap k, v, q;
};
struct AttendTcMoreMaps : AttendTcMaps {
    CUtensorMap prefix_k, prefix_v;
};
template <class Args>
using MapsFor = typename std::conditional<std::is_same<Args, AttendTcMore>::value, AttendTcMoreMaps, AttendTcMaps>::type;

__device__ __forceinline__ void tmem_wait16(uint32_t (&r)[16])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
                 :: "memory");
}
// a float of block `rank` of the cluster, at the shared-memory address `addr` of this block
__device__ __forceinline__ float ld_cluster(uint32_t addr, int rank)
{
    uint32_t remote;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// barrier among the 128 softmax threads only
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

// Byte offset of element (row g, column k) of a [16 x 128] bf16 operand kept as two K-major halves of 64 columns,
// 128-byte rows, 128-byte swizzle (the 16-byte chunk index of a row is XORed with the row's low three bits).
__device__ __forceinline__ uint32_t small_off(int g, int k)
{
    const int half = k >> 6, kk = k & 63;
    return (uint32_t)(half * (kTcSmall / 2) + g * 128 + ((((kk >> 3) ^ (g & 7)) << 4) | ((kk & 7) << 1)));
}

// The same for a [16 x 128] operand of codes: rows of 128 bytes.
__device__ __forceinline__ uint32_t code_off(int g, int k) { return (uint32_t)(g * 128 + (((k >> 4) ^ (g & 7)) << 4) + (k & 15)); }
// x as hi + lo / 16 in two codes
__device__ __forceinline__ void two_codes(float x, uint8_t *hi, uint8_t *lo)
{
    *hi = __nv_cvt_float_to_fp8(x, __NV_SATFINITE, __NV_E4M3);
    *lo = __nv_cvt_float_to_fp8((x - __half2float(__half(__nv_cvt_fp8_to_halfraw(*hi, __NV_E4M3)))) * 16.f, __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ void umma_codes(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accum)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accum)
        : "memory");
}

// With kFp8, kBarFull / kBarEmpty [0 .. kConvBufs) stand for the widened tiles (filled by the softmax threads, 128 arrivals).
// kForm: instances of their own, since a block's time is a chain of latencies that code for the others' sake lengthens.
//   kPlain  the length first, then what it says there is
//   kEarly  small grids, which nothing but latencies bound: the queries and the first key tile are under way together with the length (the
//           tile is part of the cache whatever that is), and the merge asks for all that the other blocks hold before it uses any of it
//           (8 heads of one tile 6.5 us, 5.6; 8 of 9 tiles 6.8, 6.5).  In larger ones the tiles of idle splits are bytes taken from the others
//           (1024 heads of 9 tiles, three quarters of the sequences empty: 25.4 us, and 32.2 with the early tiles).
//   kTwo    blocks of more tiles than one chunk takes
// kSrc: 0 = bf16 caches of 128 dimensions (tiles go to the tensor cores as they land), 1 = E4M3 codes of 128 dimensions,
// 3 = E4M3 codes of 128 dimensions, 4 = bf16 caches of 64 dimensions, both as they are stored (AttendTcMore), 2 = bf16 caches of 64 dimensions (1 and 2: rows of 128 bytes, widened / padded with zeros into bf16 operand tiles of
// 128 dimensions; the queries of the 64-dimension case fill the first half of their operand, the rest stays zero).
enum { kPlain, kEarly, kTwo };
template <int G, int kSrc, int kForm, class Args>
__global__ void __launch_bounds__(kTcThreads, 2)
attend_tc_kernel(Args p, const __grid_constant__ MapsFor<Args> maps)
{
    constexpr bool kFp8 = kSrc == 1 || kSrc == 2;            // the tiles pass through the softmax threads on their way to the tensor cores
    constexpr bool kCodes = kSrc == 3;          // E4M3 codes as they are stored
    constexpr bool kHalf = kSrc == 4;           // bf16 rows of 64 dimensions as they are stored
    constexpr bool kNarrow = kCodes || kHalf;   // tiles of 16 KB as they land
    constexpr int kStages = kCodes ? kCodeStages : kHalf ? kCodeStages - 1 : kTcStages, kTileRoom = kNarrow ? kRawBytes : kTcTileBytes;
    constexpr int kRingFull = kNarrow ? (int)kBarCodeFull : (int)kBarFull, kRingEmpty = kNarrow ? (int)kBarCodeEmpty : (int)kBarEmpty;
    constexpr int kDim = kSrc == 2 || kSrc == 4 ? 64 : kHeadDim;          // head dimension of the caches, the queries and the output
    constexpr bool kMore = std::is_same<Args, AttendTcMore>::value;
    constexpr bool kSeparate = kFp8 || kMore;   // the splits may be blocks of their own
    using Out = typename std::conditional<kMore, __nv_bfloat16, float>::type;
    extern __shared__ uint8_t att_tc_raw[];
    uint8_t *smem = align_smem(att_tc_raw);
    const uint32_t sbase = smem_u32(smem);
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(smem + kOffMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + kOffMisc + 4);
    float *red = reinterpret_cast<float *>(smem + kOffRed);
    auto bar = [&](int i) { return sbase + kOffBars + 8 * i; };
    const ErrSink sink{p.status, nullptr, p.wait_cycles};

    const int head = blockIdx.x / p.splits, split = blockIdx.x % p.splits;
    const int b = head / p.hkv, h = head % p.hkv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kTcStages; ++s) {
            mbar_init(bar(kBarFull + s), kFp8 ? 128 : 1);
            mbar_init(bar(kBarEmpty + s), 1);
        }
        for (int s = 0; s < kRawStages; ++s) {
            mbar_init(bar(kBarRawFull + s), 1);
            mbar_init(bar(kBarRawEmpty + s), 128);
        }
        if (kNarrow) {
            for (int s = 0; s < kStages; ++s) {
                mbar_init(bar(kBarCodeFull + s), 1);
                mbar_init(bar(kBarCodeEmpty + s), 1);
            }
            mbar_init(bar(kBarCodeQ), 128);
        }
        mbar_init(bar(kBarQ), 1);
        mbar_init(bar(kBarScores), 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(bar(kBarPFull + s), 128);
            mbar_init(bar(kBarPEmpty + s), 1);
        }
        mbar_init(bar(kBarOut), 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(tmem_holder)), "r"(kTcTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (kForm == kEarly && warp == 4 && lane == 0)
        for (const CUtensorMap *m : {&maps.q, &maps.k, &maps.v}) prefetch_map(m);
    // the P buffers start as zeros: rows of queries the group does not have are never written (and so does the query
    // operand: with 64 dimensions only its first half is loaded)
    for (int x = threadIdx.x; x < 3 * kTcSmall / 16; x += kTcThreads)
        reinterpret_cast<uint4 *>(smem + kOffQ)[x] = make_uint4(0u, 0u, 0u, 0u);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_holder;
    pdl_trigger();
    if constexpr (kMore) {
        if (!p.late) pdl_wait();
    } else {
        pdl_wait();                         // what is above uses nothing that an earlier kernel writes
    }

    const int t0 = split * p.tiles_per_split;                       // first key tile of this block
    // where key tile t of the head starts, in rows of the 2-D [rows][d] view of the caches
    KeyTiles keys = {};                     // (kMore: of the sequence's own rows, behind `prefix_tiles` of its prefix's `prefix_len` rows)
    int prefix_tiles = 0, prefix_len = 0;
    auto tile_y = [&](int t) -> int {
        if constexpr (kMore) {
            if (t < prefix_tiles) {
                const int prefix_head = b / p.per_prefix * p.hkv + h;
                if (!p.prefix_table) return prefix_head * p.prefix_cap + t * kTile;
                const int page = p.prefix_table[(size_t)prefix_head * (p.prefix_cap / kTile) + t];
                if (page >= 0 && page < p.prefix_pages) return page * kTile;
                report(p.status, RKV_ERR_INVALID_ARG);
                return -kTile;              // (in front of the tensor: zeros)
            }
            t -= prefix_tiles;
            if (!p.block_table) return head * p.cap + keys.tile(t) * kTile;
            const int page = p.block_table[(size_t)head * (p.cap / kTile) + keys.tile(t)];
            if (page >= 0 && page < p.pool_pages) return page * kTile;
            report(p.status, RKV_ERR_INVALID_ARG);
            return -kTile;                  // (in front of the tensor: zeros)
        }
        return p.block_table ? p.block_table[(size_t)head * (p.cap / kTile) + t] * kTile : head * p.cap + t * kTile;
    };
    // tile i of the block's source tiles (the K tiles, then the V tiles), from row y on, into its place in the ring
    auto fetch_tile = [&](const CUtensorMap *map, int i, int y) {
        if (kFp8) {
            const int s = i % kRawStages;
            mbar_expect_tx(bar(kBarRawFull + s), kRawBytes);
            tma_load_2d(sbase + kOffRaw + s * kRawBytes, map, 0, y, bar(kBarRawFull + s));
        } else if (kNarrow) {
            const int s = i % kStages;
            mbar_expect_tx(bar(kBarCodeFull + s), kRawBytes);
            tma_load_2d(sbase + kOffRing + s * kRawBytes, map, 0, y, bar(kBarCodeFull + s));
        } else {
            const int s = i % kTcStages;
            const uint32_t dst = sbase + kOffRing + s * kTcTileBytes;
            mbar_expect_tx(bar(kBarFull + s), kTcTileBytes);
            tma_load_2d(dst, map, 0, y, bar(kBarFull + s));
            tma_load_2d(dst + kTcHalf, map, 64, y, bar(kBarFull + s));
        }
    };
    auto fetch_queries = [&]() {
        mbar_expect_tx(bar(kBarQ), kDim == 64 ? kTcSmall / 2 : kTcSmall);
        const int qy = b * p.hq + h * G;                 // the group's G query rows (the rows after them are not used)
        tma_load_2d(sbase + kOffQ, &maps.q, 0, qy, bar(kBarQ));
        if (kDim != 64) tma_load_2d(sbase + kOffQ + kTcSmall / 2, &maps.q, 64, qy, bar(kBarQ));
    };
    // kMore: with a window or a prefix the first tile depends on the lengths, and so does whether a page has to exist
    bool early_tile = true;
    if constexpr (kMore) early_tile = p.window == 0 && !p.prefix_lens && !p.block_table;
    if (kForm == kEarly && warp == 4 && lane == 0) {
        fetch_queries();
        if (early_tile) fetch_tile(&maps.k, 0, tile_y(t0));
    }
    int L = p.seq_lens[b];
    bool short_of = false;
    if constexpr (kMore) short_of = L < p.least;
    if (L < 0 || L > p.cap || short_of) {   // reported, and treated as an empty cache
        report(p.status, RKV_ERR_INVALID_ARG);
        L = 0;
    }
    int tiles = (L + kTile - 1) / kTile;
    if constexpr (kMore) {
        keys = key_tiles(1, p.window, p.sinks, L, 1, 0, 0);
        tiles = keys.count;
        if (p.prefix_lens) {
            prefix_len = p.prefix_lens[b / p.per_prefix];
            if (prefix_len < 0 || prefix_len > p.prefix_cap) {
                report(p.status, RKV_ERR_INVALID_ARG);
                prefix_len = 0;
            }
            prefix_tiles = (prefix_len + kTile - 1) / kTile;
            tiles += prefix_tiles;
        }
    }
    const int T = min(p.tiles_per_split, tiles - t0);                // its tiles (<= 0: none)
    // row r of the block's tile t is cached and the query sees it
    auto seen = [&](int t, int r) -> bool {
        if constexpr (kMore) {
            if (t0 + t < prefix_tiles) return (t0 + t) * kTile + r < prefix_len;
            return keys.wanted(keys.tile(t0 + t - prefix_tiles) * kTile + r);
        }
        return (t0 + t) * kTile + r < L;
    };
    // more than a block's columns hold the scores of: two chunks, one after the other, each with its own maximum and output columns
    const int chunks = kForm == kTwo && T > kTcMaxTiles ? 2 : 1, T0 = chunks == 2 ? (T + 1) / 2 : T;        // T0: tiles of the first chunk
    // in the order of the ring -- the first chunk's K tiles, its V tiles, the second's -- tile i is this one of the block, of K or of V
    auto source = [&](int i, bool *value) -> int {
        const int c = kForm == kTwo && i >= 2 * T0, j = c ? i - 2 * T0 : i, n = c ? T - T0 : T0;
        *value = j >= n;
        return (c ? T0 : 0) + (j >= n ? j - n : j);
    };
    constexpr int kStride = kHeadDim + 2;
    // [G][d + 2]: unnormalised output, maximum (base-2 domain), sum of weights
    float *part = reinterpret_cast<float *>(smem + kOffP);
    int part_stride = kStride, part_max = kHeadDim;
    if (kSeparate && p.separate) {
        if constexpr (kMore) {
            part = p.slots + (((size_t)b * p.hq + (size_t)h * G) * p.slots_per_row + p.others + split) * slot_floats(kDim);
            part_stride = p.slots_per_row * slot_floats(kDim);
            part_max = kDim;
        } else {
            part = p.out + ((size_t)head * p.splits + split) * G * kStride;
        }
    }
    static_assert(G * kStride * 4 <= 2 * kTcSmall, "the partial result takes the room of P");
    Out *out = reinterpret_cast<Out *>(p.out) + ((size_t)b * p.hq + (size_t)h * G) * kDim;
    auto put = [](Out *to, float v) {
        if constexpr (kMore) *to = __float2bfloat16_rn(v);
        else *to = v;
    };
    // 0 where no row takes part; kMore: NaN for a query that is no number, as the rows' kernels give (rkv_decode_attention: 0)
    auto quotient = [](float num, float den) -> float { return (kMore ? den != 0.f : den > 0.f) ? num / den : 0.f; };
    bool merges = p.splits > 1;              // the result is merged with those of other blocks, or other kernels
    if constexpr (kMore) merges = merges || p.others > 0 || p.separate;

    if (T <= 0) {       // no cached row falls into this split (uniform for the block)
        if (kForm == kEarly) {                           // what is under way lands before the block's memory is given up
            if (warp == 4 && lane == 0) {
                mbar_wait(bar(kBarQ), 0, abort_flag, sink);
                if (early_tile) mbar_wait(bar(kFp8 ? (int)kBarRawFull : kRingFull), 0, abort_flag, sink);
            }
            __syncwarp();
        }
        if (!merges) {
            for (int x = threadIdx.x; x < G * kDim; x += kTcThreads) put(out + x, 0.f);
        } else {
            if (!kMore && kSeparate && p.separate) {          // (what the merge kernel multiplies by 0 must not be NaN)
                for (int x = threadIdx.x; x < G * kStride; x += kTcThreads) part[x] = 0.f;
                __syncthreads();
            }
            if (threadIdx.x < G) {
                part[threadIdx.x * part_stride + part_max] = -INFINITY;
                part[threadIdx.x * part_stride + part_max + 1] = 0.f;
            }
        }
    } else if (warp == 4) {
        // ------------------------------------------------------------------ TMA producer
        if (lane == 0) {
            constexpr int kRing = kFp8 ? kRawStages : kStages, kEmpty = kFp8 ? (int)kBarRawEmpty : kRingEmpty;
            if (kForm != kEarly) fetch_queries();
            for (int i = kForm == kEarly && early_tile ? 1 : 0; i < 2 * T; ++i) {
                bool value;
                const int t = t0 + source(i, &value), y = tile_y(t);
                if (!mbar_wait(bar(kEmpty + i % kRing), ((i / kRing) & 1) ^ 1, abort_flag, sink)) break;
                const CUtensorMap *map = value ? &maps.v : &maps.k;
                if constexpr (kMore) {
                    if (t < prefix_tiles) map = value ? &maps.prefix_v : &maps.prefix_k;
                }
                fetch_tile(map, i, y);
            }
        }
        __syncwarp();
    } else if (warp == 5) {
        // ------------------------------------------------------------------ MMA issuer
        if (lane == 0) {
            bool ok = mbar_wait(bar(kCodes ? kBarCodeQ : kBarQ), 0, abort_flag, sink);
            const uint32_t idesc_s = kCodes ? instr_desc_codes(kTile, 16) : instr_desc(kTile, 16);
            constexpr int kBufs = kFp8 ? kConvBufs : kStages;        // operand tiles the tensor cores read from
            // f32 accumulate, bf16 x bf16, A MN-major (bit 15), B K-major, M = 128, N = 16
            const uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | ((16u >> 3) << 17) | ((128u >> 4) << 24);
            int i = 0;                                       // tiles of the ring so far
            for (int c = 0; c < (kForm == kTwo ? chunks : 1) && ok; ++c) {
                const int n = c ? T - T0 : T0, done = c ? T0 : 0;
                // (the second chunk's scores take the columns of the first's: the last of its weights have been waited for)
                for (int t = 0; t < n && ok; ++t, ++i) {     // scores of key tile t into its own 16 columns
                    const int s = i % kBufs;
                    ok = mbar_wait(bar(kRingFull + s), (i / kBufs) & 1, abort_flag, sink);
                    if (!ok) break;
                    tc_fence_after();
                    if (kHalf)
                        umma_tile_k64(tmem + 16 * (chunks + t), sbase + kOffRing + s * kRawBytes, sbase + kOffQ, idesc_s);
                    else if (kCodes)
                        umma_tile_row128<true>(tmem + 16 * (chunks + t), sbase + kOffRing + s * kRawBytes, sbase + kOffQ, idesc_s);
                    else
                        umma_tile_k128_halves(tmem + 16 * (chunks + t), sbase + kOffRing + s * kTcTileBytes, kTcHalf, sbase + kOffQ,
                                          kTcSmall / 2, idesc_s);
                    umma_commit(bar(kRingEmpty + s));
                }
                if (ok) umma_commit(bar(kBarScores));
                for (int t = 0; t < n && ok; ++t, ++i) {     // O^T += V_t^T . P_t
                    const int s = i % kBufs, pt = done + t, pb = pt & 1;
                    ok = mbar_wait(bar(kRingFull + s), (i / kBufs) & 1, abort_flag, sink) &&
                         mbar_wait(bar(kBarPFull + pb), (pt >> 1) & 1, abort_flag, sink);
                    // (the second chunk's output lies over the scores of its first two tiles, the first's over those of its first at most)
                    if (kCodes && kForm == kTwo && c && t == 0 && ok) ok = mbar_wait(bar(kBarPFull + (pb ^ 1)), ((pt + 1) >> 1) & 1, abort_flag, sink);
                    if (!ok) break;
                    tc_fence_after();
                    if (kCodes) {
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks) {     // 32 keys per step
                            const uint32_t a_addr = sbase + kOffRing + s * kRawBytes + ks * 4096, b_addr = sbase + kOffP + pb * kTcSmall + ks * 32;
                            // A: E4M3, B: E5M2; the 128 dimensions are one atom along M, 8-row groups along K 1 KB apart
                            umma_codes(tmem + 32 * c, smem_desc(a_addr), smem_desc(b_addr), instr_desc_codes(kTile, 32) | (1u << 10) | (1u << 15),
                                       (t > 0 || ks > 0) ? 1u : 0u);
                        }
                        umma_commit(bar(kRingEmpty + s));
                        umma_commit(bar(kBarPEmpty + pb));
                        continue;
                    }
                    // (64 dimensions as they are stored: the upper half of M is the next stage of the ring, whatever it holds; its rows of the
                    // output are nobody's)
                    const uint32_t v_tile = sbase + kOffRing + s * kTileRoom, p_tile = sbase + kOffP + pb * kTcSmall;
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks) {         // 16 keys per step
                        const uint32_t a_addr = v_tile + ks * 2048;             // 16 rows of 128 bytes further
                        const uint32_t b_addr = p_tile + (ks >> 2) * (kTcSmall / 2) + (ks & 3) * 32;
                        // A: 64-element (128-byte) atoms along M 16 KB apart (the second TMA box), 8-row groups along K 1 KB apart
                        const uint64_t da = (uint64_t)((a_addr & 0x3FFFFu) >> 4) | ((uint64_t)(16384u >> 4) << 16) |
                                            ((uint64_t)(1024u >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
                        umma(tmem + 16 * c, da, smem_desc(b_addr), idesc_o, (t > 0 || ks > 0) ? 1u : 0u);
                    }
                    umma_commit(bar(kRingEmpty + s));
                    umma_commit(bar(kBarPEmpty + pb));
                }
            }
            if (ok) umma_commit(bar(kBarOut));
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ softmax threads (warps 0..3)
        const int r = threadIdx.x;                                   // TMEM lane: key row of a tile, later output dimension
        const uint32_t lane_base = tmem + ((uint32_t)(warp * 32) << 16);
        const float c2 = 1.4426950408889634f * rsqrtf((float)kDim);          // scores in the base-2 domain
        // 8-bit caches: source tile i (the K tiles, then the V tiles) from its raw stage into a bf16 operand buffer, this
        // thread's row; a row beyond the length becomes zeros
        auto widen_tile = [&](int i) -> bool {
            const int s = i % kRawStages, cb = i % kConvBufs;
            if (!mbar_wait(bar(kBarRawFull + s), (i / kRawStages) & 1, abort_flag, sink)) return false;
            if (!mbar_wait(bar(kBarEmpty + cb), ((i / kConvBufs) & 1) ^ 1, abort_flag, sink)) return false;
            bool value;
            const bool row_valid = seen(source(i, &value), r);
            const uint8_t *raw = smem + kOffRaw + s * kRawBytes + r * 128;
            uint8_t *dst = smem + kOffRing + cb * kTcTileBytes + r * 128;
            uint4 codes[8];                                  // the whole row first: the loads must not wait for the stores
#pragma unroll
            for (int c = 0; c < 8; ++c) codes[c] = *reinterpret_cast<const uint4 *>(raw + ((c ^ (r & 7)) << 4));
#pragma unroll
            for (int c = 0; c < 8; ++c) {                    // codes 16 c .. 16 c + 15 -> the row's bf16 chunks 2 c and 2 c + 1
                if (kSrc == 2) {                             // 64 dimensions: the row is the first half, the second half zeros
                    *reinterpret_cast<uint4 *>(dst + ((c ^ (r & 7)) << 4)) = row_valid ? codes[c] : make_uint4(0u, 0u, 0u, 0u);
                    *reinterpret_cast<uint4 *>(dst + kTcHalf + ((c ^ (r & 7)) << 4)) = make_uint4(0u, 0u, 0u, 0u);
                    continue;
                }
                uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo;
                if (row_valid) widen16(codes[c], &lo, &hi);
                const int half = c >> 2, pos = (2 * c) & 7;
                *reinterpret_cast<uint4 *>(dst + half * kTcHalf + ((pos ^ (r & 7)) << 4)) = lo;
                *reinterpret_cast<uint4 *>(dst + half * kTcHalf + (((pos + 1) ^ (r & 7)) << 4)) = hi;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // generic writes -> tensor-core reads
            mbar_arrive(bar(kBarFull + cb));
            mbar_arrive(bar(kBarRawEmpty + s));
            return true;
        };
        bool ok = true;
        float unscale[G];                            // kCodes: from the scaled query's scores back, in the base-2 domain
        if constexpr (kCodes) {
            // 16 threads to a query row, eight elements each: the row's scale, then its parts
            ok = mbar_wait(bar(kBarQ), 0, abort_flag, sink);
            float f[8], most = 0.f;
            const int g = r >> 4, k0 = (r & 15) * 8;
            Elem<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4 *>(smem + kOffQ + small_off(g, k0)), f);
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(f[e]));
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, off));
            // 2^(134 - exponent field) puts the largest into [128, 256); a row of zeros, or of numbers under 2^-100, by 2^100 at most
            const int up = min(max(134 - (int)(__float_as_uint(most) >> 23), -100), 100);
            const float scale = __uint_as_float((uint32_t)(127 + up) << 23);
            softmax_sync();                              // the codes take the queries' place
            if (g < G) {
                uint8_t hi[8], lo[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) two_codes(f[e] * scale + f[e] * 0.f, hi + e, lo + e);      // (an infinity has no code: NaN)
                *reinterpret_cast<uint2 *>(smem + kOffQ + code_off(g, k0)) = make_uint2(hi[0] | hi[1] << 8 | hi[2] << 16 | (uint32_t)hi[3] << 24, hi[4] | hi[5] << 8 | hi[6] << 16 | (uint32_t)hi[7] << 24);
                *reinterpret_cast<uint2 *>(smem + kOffQ + code_off(8 + g, k0)) = make_uint2(lo[0] | lo[1] << 8 | lo[2] << 16 | (uint32_t)lo[3] << 24, lo[4] | lo[5] << 8 | lo[6] << 16 | (uint32_t)lo[7] << 24);
                if ((r & 15) == 0) red[g] = __uint_as_float((uint32_t)(127 - up) << 23) * c2;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // generic writes -> tensor-core reads
            mbar_arrive(bar(kBarCodeQ));
            softmax_sync();
#pragma unroll
            for (int q = 0; q < G; ++q) unscale[q] = red[q];
            softmax_sync();                              // `red` is used again
        }
        // a query's score of this thread's row, in the base-2 domain
        auto score = [&](const uint32_t (&acc)[16], int g) -> float {
            if constexpr (kCodes) return fmaf(__uint_as_float(acc[8 + g]), 0.0625f, __uint_as_float(acc[g])) * unscale[g];
            return __uint_as_float(acc[g]) * c2;
        };
        float m[G], l[G], m0[G], l0[G];              // of the present chunk, and of the first
#pragma unroll
        for (int g = 0; g < G; ++g) m0[g] = -INFINITY, l0[g] = 0.f;
        for (int c = 0; c < (kForm == kTwo ? chunks : 1); ++c) {
            const int n = c ? T - T0 : T0, done = c ? T0 : 0;
            if (kFp8)
                for (int t = 0; t < n && ok; ++t) ok = widen_tile(2 * done + t);
            if (ok) ok = mbar_wait(bar(kBarScores), c, abort_flag, sink);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                if (c > 0) m0[g] = m[g], l0[g] = l[g];
                m[g] = -3.402823466e38f, l[g] = 0.f;      // (-inf stands for a split without rows in the merge)
            }
            if (ok) {
                tc_fence_after();
                for (int t = 0; t < n; ++t) {
                    uint32_t acc[16];
                    tmem_ld16(lane_base + 16 * (chunks + t), acc);
                    tmem_wait16(acc);
                    const bool valid = seen(done + t, r);
#pragma unroll
                    for (int g = 0; g < G; ++g)
                        if (valid) m[g] = fmaxf(m[g], score(acc, g));
                }
            }
#pragma unroll
            for (int g = 0; g < G; ++g) {
#pragma unroll
                for (int off = 16; off > 0; off >>= 1) m[g] = fmaxf(m[g], __shfl_xor_sync(0xffffffffu, m[g], off));
                if (lane == 0) red[warp * 8 + g] = m[g];
            }
            softmax_sync();
#pragma unroll
            for (int g = 0; g < G; ++g) m[g] = fmaxf(fmaxf(red[g], red[8 + g]), fmaxf(red[16 + g], red[24 + g]));
            softmax_sync();                              // `red` is used again

            for (int t = 0; t < n && ok; ++t) {
                const int pt = done + t, pb = pt & 1, i = 2 * done + n + t;
                if (kFp8) ok = widen_tile(i);
                if (ok) ok = mbar_wait(bar(kBarPEmpty + pb), ((pt >> 1) & 1) ^ 1, abort_flag, sink);
                if (!ok) break;
                uint32_t acc[16];
                tmem_ld16(lane_base + 16 * (chunks + t), acc);
                tmem_wait16(acc);
                if (kForm == kTwo || kCodes) tc_fence_before();    // (the second chunk's scores, or outputs, are written behind this thread's arrival below)
                const bool valid = seen(done + t, r);
                uint8_t *pt_smem = smem + kOffP + pb * kTcSmall;
                // (a NaN or infinite score of a row that is not cached never gets here: `valid` decides)
                auto weight = [&](int g) -> float { return valid ? exp2f(score(acc, g) - m[g]) : 0.f; };
                if constexpr (kCodes) {
#pragma unroll
                    for (int g = 0; g < G; g += 2) {         // two queries at a time
                        __half2 left = __floats2half2_rn(weight(g) * kCodeWeight, g + 1 < G ? weight(g + 1) * kCodeWeight : 0.f);
                        l[g] += __low2float(left);           // (of weights times 2^15, like the products)
                        if (g + 1 < G) l[g + 1] += __high2float(left);
#pragma unroll
                        for (int part = 0; part < 4; ++part) {
                            const uint32_t bits = *reinterpret_cast<const uint32_t *>(&left) & 0xFF00FF00u;
                            pt_smem[code_off(g + 8 * part, r)] = (uint8_t)(bits >> 8);
                            if (g + 1 < G) pt_smem[code_off(g + 1 + 8 * part, r)] = (uint8_t)(bits >> 24);
                            left = __hmul2(__hsub2(left, *reinterpret_cast<const __half2 *>(&bits)), __float2half2_rn(8.f));
                        }
                    }
                } else {
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const float w = weight(g);
                        const __nv_bfloat16 hi = __float2bfloat16_rn(w);
                        const __nv_bfloat16 lo = __float2bfloat16_rn(w - __bfloat162float(hi));
                        l[g] += __bfloat162float(hi) + __bfloat162float(lo);
                        *reinterpret_cast<__nv_bfloat16 *>(pt_smem + small_off(g, r)) = hi;
                        *reinterpret_cast<__nv_bfloat16 *>(pt_smem + small_off(8 + g, r)) = lo;
                    }
                }
                if (!kFp8 && !valid) {
                    // a row beyond the sequence's length may hold anything, and 0 x NaN would spoil the product: its V row
                    // is cleared in shared memory (only the split's last tile has such rows)
                    const int s = i % kStages;
                    ok = mbar_wait(bar(kRingFull + s), (i / kStages) & 1, abort_flag, sink);
                    if (ok) {
                        uint8_t *vt = smem + kOffRing + s * kTileRoom;
#pragma unroll
                        for (int x = 0; x < 8; ++x) {
                            *reinterpret_cast<uint4 *>(vt + r * 128 + x * 16) = make_uint4(0u, 0u, 0u, 0u);
                            if (!kNarrow) *reinterpret_cast<uint4 *>(vt + kTcHalf + r * 128 + x * 16) = make_uint4(0u, 0u, 0u, 0u);
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");       // generic writes -> tensor-core reads
                mbar_arrive(bar(kBarPFull + pb));
            }
        }
        // the chunks relative to the larger of their maxima (one chunk: w0 = 0, w1 = 1)
        float w0[G], w1[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const float top = fmaxf(m0[g], m[g]);
            w0[g] = chunks > 1 ? exp2f(m0[g] - top) : 0.f;
            w1[g] = chunks > 1 ? exp2f(m[g] - top) : 1.f;
            l[g] = chunks > 1 ? l0[g] * w0[g] + l[g] * w1[g] : l[g];
            m[g] = top;
        }

        // ---- the sums of the weights over the 128 key rows, then the output columns
#pragma unroll
        for (int g = 0; g < G; ++g) {
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) l[g] += __shfl_xor_sync(0xffffffffu, l[g], off);
            if (lane == 0) red[warp * 8 + g] = l[g];
        }
        softmax_sync();
        if (ok) ok = mbar_wait(bar(kBarOut), 0, abort_flag, sink);
        // the queries' outputs of this thread's dimension and chunk c, from the columns of the parts
        constexpr int kOutCols = kCodes ? 32 : 16;
        constexpr float kLow = kCodes ? 0.125f : 1.f, kScale = kCodes ? 1.f / kCodeWeight : 1.f;
        float num[G], num0[G];
        auto outputs = [&](int c, float (&to)[G]) {
            uint32_t o[16];
            tmem_ld16(lane_base + kOutCols * c, o);
            tmem_wait16(o);
#pragma unroll
            for (int g = 0; g < G; ++g) to[g] = fmaf(__uint_as_float(o[8 + g]), kLow, __uint_as_float(o[g]));
            if constexpr (kCodes) {
                tmem_ld16(lane_base + kOutCols * c + 16, o);
                tmem_wait16(o);
#pragma unroll
                for (int g = 0; g < G; ++g) to[g] = fmaf(fmaf(__uint_as_float(o[8 + g]), kLow, __uint_as_float(o[g])), kLow * kLow, to[g]);
            }
        };
#pragma unroll
        for (int g = 0; g < G; ++g) num[g] = num0[g] = 0.f;
        if (ok) {
            tc_fence_after();
            outputs(chunks - 1, num);
            if (chunks > 1) outputs(0, num0);
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float den = ok ? (red[g] + red[8 + g]) + (red[16 + g] + red[24 + g]) : 0.f;     // error path: zeros
            if (chunks > 1) num[g] = num0[g] * w0[g] + num[g] * w1[g];
            num[g] *= kScale, den *= kScale;
            if (r >= kDim) continue;                          // (64 dimensions: the padded half of the output)
            if (!merges) {
                put(out + (size_t)g * kDim + r, quotient(num[g], den));
            } else {
                part[g * part_stride + r] = num[g];
                if (r == 0) {
                    part[g * part_stride + part_max] = ok ? m[g] : -INFINITY;
                    part[g * part_stride + part_max + 1] = den;
                }
            }
        }
    }

    // ---- merge the splits: out = sum_s 2^(m_s - m) num_s / sum_s 2^(m_s - m) l_s, block r of the cluster taking its share
    if (merges && !(kSeparate && p.separate)) {
        __syncwarp();
        if constexpr (kMore) {
            if (p.late) pdl_wait();         // the other kernel's slots
        }
        cluster_sync();
        const uint32_t base = sbase + kOffP;
        for (int x = split * kTcThreads + threadIdx.x; x < G * kDim; x += p.splits * kTcThreads) {
            const int g = x / kDim, c = x % kDim;
            const uint32_t row = base + (uint32_t)(g * kStride) * 4u;
            float ms[kTcMaxSplits], ns[kTcMaxSplits], ls[kTcMaxSplits], m = -INFINITY, num = 0.f, den = 0.f;
#pragma unroll
            for (int s = 0; s < kTcMaxSplits; ++s) {
                ms[s] = -INFINITY;
                if (s < p.splits) {
                    ms[s] = ld_cluster(row + kHeadDim * 4u, s);
                    if (kForm == kEarly) {
                        ns[s] = ld_cluster(row + (uint32_t)c * 4u, s);
                        ls[s] = ld_cluster(row + (kHeadDim + 1) * 4u, s);
                    }
                }
            }
#pragma unroll
            for (int s = 0; s < kTcMaxSplits; ++s) m = fmaxf(m, ms[s]);
#pragma unroll
            for (int s = 0; s < kTcMaxSplits; ++s) {                   // fixed order; a split without rows has m = -inf
                if (ms[s] == -INFINITY) continue;
                const float w = exp2f(ms[s] - m);
                num = fmaf(w, kForm == kEarly ? ns[s] : ld_cluster(row + (uint32_t)c * 4u, s), num);
                den = fmaf(w, kForm == kEarly ? ls[s] : ld_cluster(row + (kHeadDim + 1) * 4u, s), den);
            }
            if constexpr (kMore) {
                // the other kernel's slots, the loads of eight under way at a time
                const float *other = p.slots + (((size_t)b * p.hq + (size_t)h * G + g) * p.slots_per_row) * slot_floats(kDim);
                constexpr int kAhead = 8;
                for (int s0 = 0; s0 < p.others; s0 += kAhead) {
                    float mo[kAhead], lo[kAhead], no[kAhead], top = m;
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        mo[i] = -INFINITY;
                        if (s0 + i < p.others) {
                            const float *slot = other + (s0 + i) * slot_floats(kDim);
                            mo[i] = slot[kDim], lo[i] = slot[kDim + 1], no[i] = slot[c];
                        }
                        top = fmaxf(top, mo[i]);
                    }
                    if (top == -INFINITY) continue;
                    const float old = exp2f(m - top);
                    num *= old, den *= old, m = top;
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) {
                        if (mo[i] == -INFINITY) continue;
                        const float w = exp2f(mo[i] - m);
                        num = fmaf(w, no[i], num);
                        den = fmaf(w, lo[i], den);
                    }
                }
            }
            put(out + x, quotient(num, den));
        }
        cluster_sync();                     // nobody leaves while its partial result is still being read
    } else if constexpr (kMore) {
        // The merge kernel waits for this kernel's end, which is to be behind the other kernel's: the last block waits.  (Not all: a block that
        // waits keeps the next one out.)
        if (p.late && blockIdx.x == gridDim.x - 1) pdl_wait();
    }

    // ---------------------------------------------------------------------- common exit
    tc_fence_before();
    __syncthreads();
    if (warp == 5) {
        if (*abort_flag) __nanosleep(200000);      // error path only: let copies and products in flight land
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTcTmemCols) : "memory");
    }
}

template <int G, int kSrc, int kForm, class Args>
cudaError_t launch_tc_one(const Args &p, int heads, const MapsFor<Args> &maps, int dev, cudaStream_t s)
{
    static PerDevice done;
    const cudaError_t e = allow_smem_once(done, dev, attend_tc_kernel<G, kSrc, kForm, Args>, kTcSmem, true);
    if (e != cudaSuccess) return e;
    return launch_early(attend_tc_kernel<G, kSrc, kForm, Args>, (unsigned)(heads * p.splits), kTcThreads, kTcSmem, s,
                        p.separate ? 1u : (unsigned)p.splits, p, maps);
}
template <int G, int kSrc, class Args>
cudaError_t launch_tc_form(const Args &p, int heads, const MapsFor<Args> &maps, cudaStream_t s)
{
    int dev = 0, sms = 0;
    const cudaError_t e = device_sms(&dev, &sms);
    if (e != cudaSuccess) return e;
    if (p.tiles_per_split > kTcMaxTiles) return launch_tc_one<G, kSrc, kTwo, Args>(p, heads, maps, dev, s);
    // A block per SM, or two of few tiles: beside a second block of many an idle one's tile costs more than an early start gives (32 heads of 9
    // tiles, 288 blocks of one: 13.0 us, 12.1 early; 256 blocks of nine, 256 heads of which half are empty: 12.6, 13.2; 128 heads of 17 tiles, 1000
    // tokens: 15.6, 16.0).
    const long long blocks = (long long)heads * p.splits;
    return blocks <= sms || (blocks <= 2ll * sms && p.tiles_per_split <= 4) ? launch_tc_one<G, kSrc, kEarly, Args>(p, heads, maps, dev, s)
                                                                            : launch_tc_one<G, kSrc, kPlain, Args>(p, heads, maps, dev, s);
}
template <int G, class Args>
cudaError_t launch_tc_for(const Args &p, int heads, int src, const MapsFor<Args> &maps, cudaStream_t s)
{
    constexpr bool kMore = std::is_same<Args, AttendTcMore>::value;
    return src == 1 ? launch_tc_form<G, kMore ? 3 : 1, Args>(p, heads, maps, s) : src == 2 ? launch_tc_form<G, kMore ? 4 : 2, Args>(p, heads, maps, s)
                                                                           : launch_tc_form<G, 0, Args>(p, heads, maps, s);
}


// src: 0 = bf16 caches of 128 dimensions, 1 = E4M3 codes of 128 dimensions, 2 = bf16 caches of 64 dimensions
inline bool make_cache_map(CUtensorMap *map, const void *base, uint64_t rows, int src)
{
    return src != 0 ? sm100::make_map_row128(map, base, rows, src == 1) : sm100::make_map(map, base, rows, kTile);
}
// The tensor maps of the caches and the queries, and the instance for the group.
template <class Args>
cudaError_t launch_tc_group(const Args &p, MapsFor<Args> maps, const void *k_cache, const void *v_cache, const void *q_new, int batch,
                            long long pool_pages, int src, cudaStream_t s)
{
    const uint64_t rows = p.block_table ? (uint64_t)pool_pages * kTile : (uint64_t)batch * p.hkv * p.cap;
    const bool maps_ok = make_cache_map(&maps.k, k_cache, rows, src) && make_cache_map(&maps.v, v_cache, rows, src);
    const bool q_ok = src == 2 ? sm100::make_map_rows(&maps.q, q_new, (uint64_t)batch * p.hq, 64, 16) : sm100::make_map(&maps.q, q_new, (uint64_t)batch * p.hq, 16);
    if (!maps_ok || !q_ok) return cudaErrorInvalidValue;
    switch (p.hq / p.hkv) {
        case 1: return launch_tc_for<1>(p, batch * p.hkv, src, maps, s);
        case 2: return launch_tc_for<2>(p, batch * p.hkv, src, maps, s);
        case 3: return launch_tc_for<3>(p, batch * p.hkv, src, maps, s);
        case 4: return launch_tc_for<4>(p, batch * p.hkv, src, maps, s);
        case 5: return launch_tc_for<5>(p, batch * p.hkv, src, maps, s);
        case 6: return launch_tc_for<6>(p, batch * p.hkv, src, maps, s);
        case 7: return launch_tc_for<7>(p, batch * p.hkv, src, maps, s);
        case 8: return launch_tc_for<8>(p, batch * p.hkv, src, maps, s);
        default: return cudaErrorInvalidValue;
    }
}

}  // namespace

}  // namespace rkv
