// Attention of many query rows over a cache on the tensor cores (see RowsParams): bf16 products, fp32 accumulation and softmax.
//
//   S = Q K^T   [128 rows x 128 keys], Q and K tiles in shared memory, accumulator in tensor memory
//   P = 2^(S c - m)   by eight warps, two threads per row, 64 keys each; rounded to bf16 and written back over S in tensor memory
//   O += P V    P from tensor memory, V as TMA leaves it (keys along K, so the transposed form of the operand), O in tensor memory
//
// A block takes kTiles (one or two) row tiles of one (problem, KV head); a row tile holds 128 / G whole tokens with their G heads.
//
// Two row tiles (one block to an SM): each K and V tile serves both.  The scores have one accumulator, which the row tiles take in turn, and the
// weights columns of their own: as soon as a tile's threads have its scores in registers the tensor cores form the other tile's, so scores are
// there before the threads that need them and nobody waits for a chain of product, weights, product, scores (with the weights over
// the scores, and two accumulators, that chain took 4700 cycles for 128 keys where the products take 2048).  Order of the products:
// S_0(j+1) after S_1(j) has been read, then O_1(j-1), S_1(j+1), O_0(j) .., tiles K_0 K_1 V_0 K_2 V_1 ..
// One row tile (two blocks to an SM): weights over the scores, S(j), O(j), S(j+1) .., tiles K_0 V_0 K_1 V_1 ..; the blocks fill each other's gaps.
//
// The maximum that the weights refer to moves only when a row's scores outgrow it by 2^8: until then weights up to 2^8 are as exact as
// others in bf16, and O and the sum need no correction.
//
// Rows that no token of the call sees may hold anything: their scores are masked, their V rows cleared in shared memory by the producer
// warp before the tile is handed on (0 x NaN).  Only tiles at the borders of what the call sees have such rows.
//
// Every wait is bounded; on expiry the block records RKV_ERR_TIMEOUT and leaves through the common exit.  No TMA multicast.
#include "rkv_sm100.cuh"
#include "rkv_tokens.cuh"

namespace rkv {

namespace {

using namespace sm100;

template <int kDim, int kTiles>
struct RowsShape {
    static constexpr int kHalves = kDim / 64;
    static constexpr int kBox = kTile * 64 * 2;                          // 128 rows x 64 columns
    static constexpr int kTileBytes = kHalves * kBox;
    static constexpr int kStages = kTiles == 2 ? (kDim == 128 ? 4 : 8) : (kDim == 128 ? 2 : 4);
    static constexpr int kOffRing = kTiles * kTileBytes;
    static constexpr int kOffBars = kOffRing + kStages * kTileBytes;
    // barriers: full[stages], empty[stages], queries, border tile landed, scores[tiles], weights[tiles], ..
    static constexpr int kFull = 0, kEmpty = kFull + kStages, kQ = kEmpty + kStages, kBorder = kQ + 1, kScores = kBorder + 1,
                         kWeights = kScores + kTiles, kOut = kWeights + kTiles,           // kOut[tiles]: a product with V is through
                         kRead = kOut + kTiles,              // kRead[tiles]: scores in registers
                         kFree = kRead + kTiles,             // kFree[tiles]: the output has left tensor memory
                         kQFree = kFree + kTiles,            // kQFree: the queries have been read
                         kNext = kQFree + 1,                 // kNext[2]: the answer to the question for a next item is there
                         kNextFree = kNext + 2, kBars = kNextFree + 2;                     // kNextFree[2]: every warp has read it
    static constexpr int kOffMisc = kOffBars + kBars * 8;
    static constexpr int kOffNext = (kOffMisc + 16 + 15) / 16 * 16;      // two answers of 16 bytes
    static constexpr int kOffMost = kOffNext + 32;      // [tiles][2 key tiles in turn][2 halves][128]: the rows' largest scores
    static constexpr int kOffSums = kOffMost + kTiles * 512 * 4;         // [tiles][2 halves][128]: the rows' sums of weights
    static constexpr int kSmem = kOffSums + kTiles * 256 * 4 + 1024;
    static constexpr int kThreads = kTiles * 256 + 64;
    static constexpr uint32_t kCols = kTiles == 2 ? 512 : 256;
    // tensor memory: scores, weights, outputs; one row tile: the weights of each half of the keys over its scores
    __host__ __device__ static constexpr int kWeightCol(int i, int half) { return kTiles == 2 ? 128 + i * 64 + half * 32 : half * 64; }
    __host__ __device__ static constexpr int kOutCol(int i) { return kTiles * 128 + i * kDim; }
    // the ring's i-th tile of 2 T: K or V, and of which keys; and the places of K_j and V_j
    __device__ static __forceinline__ bool value_at(int i, int T) { return kTiles == 1 || T == 1 ? i & 1 : i == 2 * T - 1 || (i >= 2 && !(i & 1)); }
    __device__ static __forceinline__ int index_at(int i, int T)
    {
        return kTiles == 1 || T == 1 ? i >> 1 : i == 2 * T - 1 ? T - 1 : i < 2 ? i : i & 1 ? (i + 1) >> 1 : (i - 2) >> 1;
    }
    __device__ static __forceinline__ int place_k(int j, int T) { return kTiles == 1 || T == 1 ? 2 * j : j == 0 ? 0 : 2 * j - 1; }
    __device__ static __forceinline__ int place_v(int j, int T) { return kTiles == 1 || T == 1 ? 2 * j + 1 : j == T - 1 ? 2 * T - 1 : 2 * j + 2; }
    static_assert(kTiles * (128 + kDim) <= (int)kCols, "tensor memory");
    static_assert(kSmem <= (kTiles == 2 ? 227 : 113) * 1024, "shared memory");
};

constexpr float kSlack = 8.f;              // the weights' reference may fall behind the maximum by 2^8

__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// D[128 x N] += A[128 x 16, tensor memory] . B[16 x N, shared memory]
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accum)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accum)
        : "memory");
}
// true for one lane of the warp
__device__ __forceinline__ bool elect_one()
{
    uint32_t is;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is != 0;
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}
// 2^x to about 2^-22; results below 2^-126 are 0
__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// two fp32 at a time
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "add.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b, d;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "mul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
// 2^x for two x <= 127 without the special-function unit: x = n + f, |f| <= 1/2, by adding and subtracting 3 2^22 + 127, whose sum's last bits
// are the exponent field of 2^n; times 2^f by the polynomial of degree 4 with the smallest relative error (2.7e-6 with fp32 rounding; a weight's
// own rounding is up to 3.9e-3).  From -126.5 down the field is 0 and so is the result: hidden keys, whose scores are -inf, count for nothing,
// whatever their values are.
__device__ __forceinline__ float2 exp2_poly(float2 x)
{
    x = make_float2(fmaxf(x.x, -127.f), fmaxf(x.y, -127.f));
    const float2 big = make_float2(12583039.f, 12583039.f), t = add2(x, big);
    const float2 f = add2(x, fma2(t, make_float2(-1.f, -1.f), big));
    float2 y = fma2(make_float2(0.009570101276040077f, 0.009570101276040077f), f, make_float2(0.05591785907745361f, 0.05591785907745361f));
    y = fma2(y, f, make_float2(0.240247443318367f, 0.240247443318367f));
    y = fma2(y, f, make_float2(0.6931217908859253f, 0.6931217908859253f));
    y = fma2(y, f, make_float2(0.9999992847442627f, 0.9999992847442627f));
    return mul2(y, make_float2(__uint_as_float(__float_as_uint(t.x) << 23), __uint_as_float(__float_as_uint(t.y) << 23)));
}
// v[e] of lane i and v[i] of lane e change places among four lanes
__device__ __forceinline__ void transpose4(uint4 (&v)[4])
{
    const int lane = threadIdx.x & 3;
#pragma unroll
    for (int bit = 1; bit <= 2; bit <<= 1) {
        const bool high = lane & bit;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (e & bit) continue;                                       // the pair v[e], v[e + bit]: one goes, the other stays
            uint4 &a = v[e], &b = v[e + bit];
            const uint4 give = high ? a : b;
            uint4 got;
            got.x = __shfl_xor_sync(0xffffffffu, give.x, bit);
            got.y = __shfl_xor_sync(0xffffffffu, give.y, bit);
            got.z = __shfl_xor_sync(0xffffffffu, give.z, bit);
            got.w = __shfl_xor_sync(0xffffffffu, give.w, bit);
            if (high) a = got;
            else b = got;
        }
    }
}
// bit e set: e <= last
__device__ __forceinline__ uint32_t bits_to(int last) { return last < 0 ? 0u : last >= 31 ? 0xFFFFFFFFu : (2u << last) - 1u; }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&b);
}

// What a block does at a time: its row tiles of a problem and KV head, against its share of the key tiles.
struct Item {
    int b, h, first, n, len;     // problem, KV head; the problem's tokens and cached rows
    int t0, t1;                  // its first and last token, from the problem's first
    int split, i0, T;            // its key tiles: [i0, i0 + T) of `keys`
    KeyTiles keys;
};
// The last tokens see the most keys: they come first, of all problems.  False: no rows.
__device__ __forceinline__ bool load_item(const RowsParams &p, int idx, int items, int tokens, int pieces, bool tell, Item *x)
{
    if (idx >= items) return false;
    x->split = idx % p.splits;
    idx /= p.splits;
    const int pairs = p.hkv * p.tokens.count, pair = idx % pairs;
    x->h = pair % p.hkv;
    x->b = pair / p.hkv;
    x->n = token_span(p.tokens, x->b, &x->first);
    x->len = p.lens[x->b];
    if (x->n < 0 || x->len < 0 || x->len > p.cap || (p.causal && x->len < x->n)) {
        if (tell) report(p.status, RKV_ERR_INVALID_ARG);
        x->len = 0;
    }
    x->t0 = (pieces - 1 - idx / pairs) * tokens;
    if (x->n <= 0 || x->t0 >= x->n) return false;
    x->t1 = min(x->n, x->t0 + tokens) - 1;
    x->keys = key_tiles(p.causal, p.window, p.sinks, x->len, x->n, x->t0, x->t1);
    if (x->len == 0) x->keys.count = 0;
    const int per = (x->keys.count + p.splits - 1) / p.splits;
    x->i0 = x->split * per;
    x->T = max(0, min(x->keys.count, x->i0 + per) - x->i0);
    return true;
}

// Items are blocks of the grid that have not started: a block that is done with one takes the next one over by cancelling its launch, in the
// grid's order, so that items of unlike length, or of none, leave no SM idle.  (By a fixed stride the busiest of 148 blocks had 1.1 to 1.3 times
// the mean on prompts of unlike lengths.)  `answer` gets 16 bytes, which complete the phase of `bar`.
__device__ __forceinline__ void ask_next(uint32_t answer, uint32_t bar)
{
    mbar_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(answer), "r"(bar) : "memory");
}
// The block that was taken over, or -1 when none was left.
__device__ __forceinline__ int read_next(uint32_t answer)
{
    int x;
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 lo, hi;\n\t.reg .b128 r;\n\t"
        "ld.shared.v2.u64 {lo, hi}, [%1];\n\tmov.b128 r, {lo, hi};\n\tmov.b32 %0, -1;\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, r;\n\t}"
        : "=r"(x) : "r"(answer) : "memory");
    return x;
}

template <int kDim, int kTiles>
__global__ void __launch_bounds__(RowsShape<kDim, kTiles>::kThreads, kTiles == 2 ? 1 : 2)
rows_tc_kernel(RowsParams p, int tokens_per_tile, int pieces, int items, const __grid_constant__ CUtensorMap map_k,
               const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_q)
{
    using S = RowsShape<kDim, kTiles>;
    extern __shared__ uint8_t rows_tc_raw[];
    uint8_t *smem = align_smem(rows_tc_raw);
    const uint32_t sbase = smem_u32(smem);
    uint32_t *tmem_holder = reinterpret_cast<uint32_t *>(smem + S::kOffMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + S::kOffMisc + 4);
    auto bar = [&](int i) { return sbase + S::kOffBars + 8 * i; };
    const ErrSink sink{p.status, nullptr, p.wait_cycles};
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kProducer = kTiles * 8, kIssuer = kProducer + 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(bar(S::kFull + s), 1);
            mbar_init(bar(S::kEmpty + s), 1);
        }
        mbar_init(bar(S::kQ), 1);
        mbar_init(bar(S::kBorder), 1);
        for (int i = 0; i < kTiles; ++i) {
            mbar_init(bar(S::kScores + i), 1);
            mbar_init(bar(S::kWeights + i), 256);
            mbar_init(bar(S::kOut + i), 1);
            mbar_init(bar(S::kRead + i), 256);
            mbar_init(bar(S::kFree + i), 256);
        }
        mbar_init(bar(S::kQFree), 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(S::kNext + i), 1);
            mbar_init(bar(S::kNextFree + i), kTiles * 8 + 2);            // warps
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kProducer && lane == 0)
        for (const CUtensorMap *m : {&map_q, &map_k, &map_v}) prefetch_map(m);
    pdl_wait();
    if (warp == kIssuer) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(tmem_holder)), "r"(S::kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_holder;
    // Only now may a later kernel's blocks come in: one that took tensor memory and waited for this kernel's end, while a block of this
    // kernel waited for tensor memory, would wait for good.  (And only behind the wait above: see AttendTcMore::late.)
    pdl_trigger();

    // The item behind the nth of this block, -1: none, or a wait of one of the warp's lanes ran out.
    auto next_item = [&](int nth, bool ok) -> int {
        const bool there = __all_sync(0xffffffffu, ok && mbar_wait(bar(S::kNext + (nth & 1)), (nth >> 1) & 1, abort_flag, sink));
        const int idx = there ? read_next(sbase + S::kOffNext + 16 * (nth & 1)) : -1;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(S::kNextFree + (nth & 1)));
        return idx;
    };
    if (warp == kProducer) {
        // ------------------------------------------------------------------ TMA producer
        int base = 0, turn = 0, borders = 0;                             // tiles through the ring, items with keys, border tiles so far
        bool ok = true;
        for (int nth = 0, idx = blockIdx.x; idx >= 0; idx = next_item(nth++, ok)) {
            // the question for the next item, when the answer before the last has been read
            ok = __all_sync(0xffffffffu, mbar_wait(bar(S::kNextFree + (nth & 1)), ((nth >> 1) & 1) ^ 1, abort_flag, sink));
            if (!ok) continue;
            if (lane == 0) ask_next(sbase + S::kOffNext + 16 * (nth & 1), bar(S::kNext + (nth & 1)));
            Item x;
            if (!load_item(p, idx, items, kTiles * tokens_per_tile, pieces, lane == 0, &x) || x.T == 0) continue;
            const int head = x.b * p.hkv + x.h;
            const CallTiles call = call_tiles(p.causal, p.window, p.sinks, x.len, x.n);
            ok = __all_sync(0xffffffffu, mbar_wait(bar(S::kQFree), (turn & 1) ^ 1, abort_flag, sink));
            if (lane == 0 && ok) {
                mbar_expect_tx(bar(S::kQ), kTiles * S::kHalves * 128 * tokens_per_tile * p.group);
                for (int i = 0; i < kTiles; ++i)
                    for (int half = 0; half < S::kHalves; ++half)
                        tma_load_3d(sbase + i * S::kTileBytes + half * S::kBox, &map_q, 64 * half, x.h * p.group,
                                    x.first + x.t0 + i * tokens_per_tile, bar(S::kQ));
            }
            for (int i = 0; i < 2 * x.T && ok; ++i) {
                const bool value = S::value_at(i, x.T);
                const int t = x.keys.tile(x.i0 + S::index_at(i, x.T)), s = (base + i) % S::kStages, j0 = t * kTile;
                const bool border = value && !p.compact_tiles && (j0 + kTile > x.len || (j0 < call.lo && j0 + kTile > call.sinks));
                const long long start = p.compact_tiles ? ((long long)head * p.compact_tiles + call.place(t)) * kTile : rows_tile_start(p, head, t);
                if (start < 0 && lane == 0) report(p.status, RKV_ERR_INVALID_ARG);
                const int y = start < 0 ? -kTile : (int)start;           // (beyond the tensor: zeros)
                ok = __all_sync(0xffffffffu, mbar_wait(bar(S::kEmpty + s), (((base + i) / S::kStages) & 1) ^ 1, abort_flag, sink));
                if (!ok) break;
                const uint32_t dst = sbase + S::kOffRing + s * S::kTileBytes, full = border ? bar(S::kBorder) : bar(S::kFull + s);
                if (lane == 0) {
                    mbar_expect_tx(full, S::kTileBytes);
                    for (int half = 0; half < S::kHalves; ++half)
                        tma_load_2d(dst + half * S::kBox, value ? &map_v : &map_k, 64 * half, y, full);
                }
                if (border) {
                    ok = __all_sync(0xffffffffu, mbar_wait(full, borders++ & 1, abort_flag, sink));
                    if (!ok) break;
                    uint8_t *tile = smem + S::kOffRing + s * S::kTileBytes;
                    for (int r = 0; r < kTile; r += 4) {                 // 8 lanes to a row of a box
                        const int row = r + (lane >> 3);
                        if (!call.wanted(j0 + row, x.len))
                            for (int half = 0; half < S::kHalves; ++half)
                                *reinterpret_cast<uint4 *>(tile + half * S::kBox + row * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(S::kFull + s));
                }
            }
            base += 2 * x.T;
            ++turn;
        }
        __syncwarp();
    } else if (warp == kIssuer) {
        // ------------------------------------------------------------------ MMA issuer
        // The whole warp goes through the loop and the waits, so that descriptors stay in uniform registers; one elected lane issues.  (With
        // the loop in one lane's branch a product of 16 took 65 to 85 cycles to issue, twice what it takes to run.)
        const bool leader = elect_one();
        const uint32_t idesc_s = instr_desc(kTile, kTile), idesc_o = instr_desc(kTile, kDim) | (1u << 16);          // V: keys along K
        const uint64_t q_desc = smem_desc(sbase), k_desc = smem_desc(sbase + S::kOffRing);
        // V: 64 columns to a box, boxes kBox apart; 8 keys every 1024 bytes
        const uint64_t v_desc = (uint64_t)(((sbase + S::kOffRing) & 0x3FFFFu) >> 4) | ((uint64_t)(S::kBox >> 4) << 16) |
                                ((uint64_t)(1024u >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
        constexpr uint32_t kStep = S::kTileBytes >> 4;                   // from stage to stage, in a descriptor's units
        int base = 0, steps = 0, turn = 0;                               // tiles through the ring, key tiles, items with keys so far
        bool ok = true;
        int T = 0;
        auto scores = [&](int r, int j) {
            const int i = base + S::place_k(j, T);
            const uint64_t dq = q_desc + (uint64_t)(r * kStep), dk = k_desc + (uint64_t)((i % S::kStages) * kStep);
            if (leader) {
#pragma unroll
                for (int ks = 0; ks < kDim / 16; ++ks) {
                    const uint64_t off = (ks >> 2) * (S::kBox >> 4) + (ks & 3) * 2;          // 16 columns further
                    umma(tmem, dq + off, dk + off, idesc_s, ks > 0 ? 1u : 0u);
                }
                umma_commit(bar(S::kScores + r));
                if (r == kTiles - 1) {
                    umma_commit(bar(S::kEmpty + i % S::kStages));
                    if (j == T - 1) umma_commit(bar(S::kQFree));
                }
            }
        };
        auto values = [&](int r, int j) {
            const int i = base + S::place_v(j, T);
            const uint64_t dv = v_desc + (uint64_t)((i % S::kStages) * kStep);
            const uint32_t o = tmem + S::kOutCol(0) + r * kDim, w = tmem + S::kWeightCol(0, 0) + r * 64;
            if (leader) {
#pragma unroll
                for (int ks = 0; ks < kTile / 16; ++ks)                  // 16 keys further
                    umma_ts(o, w + (ks >> 2) * (S::kWeightCol(0, 1) - S::kWeightCol(0, 0)) + (ks & 3) * 8, dv + (uint64_t)(ks * 128), idesc_o,
                            ks > 0 ? 1u : (uint32_t)(j > 0));
                umma_commit(bar(S::kOut + r));
                if (r == kTiles - 1) umma_commit(bar(S::kEmpty + i % S::kStages));
            }
        };
        for (int nth = 0, idx = blockIdx.x; idx >= 0; idx = next_item(nth++, ok)) {
            Item x;
            if (!load_item(p, idx, items, kTiles * tokens_per_tile, pieces, false, &x) || x.T == 0) continue;
            T = x.T;
            auto full = [&](int i) { return mbar_wait(bar(S::kFull + (base + i) % S::kStages), ((base + i) / S::kStages) & 1, abort_flag, sink); };
            auto weights = [&](int r, int j) { return mbar_wait(bar(S::kWeights + r), (steps + j) & 1, abort_flag, sink); };
            auto read = [&](int r, int j) { return mbar_wait(bar(S::kRead + r), (steps + j) & 1, abort_flag, sink); };
            auto out_free = [&](int r) { return mbar_wait(bar(S::kFree + r), (turn & 1) ^ 1, abort_flag, sink); };       // the item's before
            ok = mbar_wait(bar(S::kQ), turn & 1, abort_flag, sink) && full(0);
            // (the accumulator's last scores have been read: their weights have been waited for)
            tc_fence_after();
            if (ok) scores(0, 0);
            if constexpr (kTiles == 1) {
                for (int j = 0; j < T && ok; ++j) {
                    if (!(ok = full(2 * j + 1) && weights(0, j) && (j > 0 || out_free(0)))) break;
                    tc_fence_after();
                    values(0, j);
                    if (j + 1 == T) break;
                    if (!(ok = full(2 * j + 2))) break;
                    scores(0, j + 1);
                }
            } else {
                // A wait costs some 100 cycles even where nothing is left to wait for: one between any two products, which the product before
                // hides.  (That a tile's scores have been read says that its weights before them are there.)
                for (int j = 0; j <= T && ok; ++j) {
                    if (!(ok = j < T ? read(0, j) : weights(0, j - 1))) break;
                    tc_fence_after();
                    if (j < T) scores(1, j);
                    if (j + 1 < T && !(ok = full(S::place_k(j + 1, T)))) break;
                    if (j == 1) {
                        if (!(ok = out_free(0))) break;
                        tc_fence_after();
                    }
                    if (j > 0) values(0, j - 1);
                    if (!(ok = j < T ? read(1, j) : weights(1, j - 1))) break;
                    tc_fence_after();
                    if (j + 1 < T) scores(0, j + 1);
                    if (j < T && !(ok = full(S::place_v(j, T)))) break;
                    if (j == 1) {
                        if (!(ok = out_free(1))) break;
                        tc_fence_after();
                    }
                    if (j > 0) values(1, j - 1);
                }
            }
            base += 2 * T;
            steps += T;
            ++turn;
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ softmax, two threads per row
        const int r = warp >> 3, half = (warp >> 2) & 1, row = threadIdx.x & 127;        // row tile, keys 64 half .., row (= lane of tensor memory)
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t s_col = lanes + 64 * half, w_col = lanes + S::kWeightCol(r, half), o_col = lanes + S::kOutCol(r) + half * (kDim / 2);
        float *mosts = reinterpret_cast<float *>(smem + S::kOffMost) + r * 512, *sums = reinterpret_cast<float *>(smem + S::kOffSums) + r * 256;
        auto pair_sync = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + r * 4 + (warp & 3)) : "memory"); };       // the two warps of 32 rows
        const float c2 = 1.4426950408889634f * rsqrtf((float)kDim);
        int steps = 0;                                                   // key tiles so far
        bool ok = true;
        // (both warps of a pair go on, or neither: they wait for each other in every item)
        auto pair_next = [&](int nth) -> int {
            int idx = next_item(nth, true), both;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ge.s32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, %2, 64, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                         : "=r"(both) : "r"(idx), "r"(1 + r * 4 + (warp & 3)) : "memory");
            return both ? idx : -1;
        };
        for (int nth = 0, idx = blockIdx.x; idx >= 0; idx = pair_next(nth++)) {
            // what the loop needs; the rest is looked up once more behind it, in registers that the scores take until then
            int T, i0, sink_tiles, first_tile, last, from, last_all, from_all;
            {
                Item x;
                if (!load_item(p, idx, items, kTiles * tokens_per_tile, pieces, false, &x)) continue;
                T = x.T, i0 = x.i0, sink_tiles = x.keys.sink_tiles, first_tile = x.keys.first;
                // the cached rows that this row sees, and what all rows of the tile see
                const int tt0 = x.t0 + r * tokens_per_tile, at0 = x.len - x.n + tt0, at = at0 + row / p.group;
                const int at1 = x.len - x.n + min(x.t1, tt0 + tokens_per_tile - 1);
                last = p.causal ? at : x.len - 1, from = p.causal && p.window > 0 ? at + 1 - p.window : 0;
                last_all = p.causal ? at0 : x.len - 1, from_all = p.causal && p.window > 0 ? at1 + 1 - p.window : 0;
            }
            float m = -INFINITY, l = 0.f;                                    // reference of the weights (raw scores), sum of this thread's weights
            for (int j = 0; j < T; ++j) {
                if (ok) ok = __all_sync(0xffffffffu, mbar_wait(bar(S::kScores + r), (steps + j) & 1, abort_flag, sink));
                if (!ok) {                                                   // (every warp comes to every one of its pair's barriers)
                    pair_sync();
                    continue;
                }
                tc_fence_after();
                uint32_t s[2][32];
                tmem_ld32(s_col, s[0]);
                tmem_ld32(s_col + 32, s[1]);
                tmem_wait32(s[0]);
                tmem_wait32(s[1]);
                if (kTiles == 2) {                                           // the accumulator is the other tile's
                    tc_fence_before();
                    mbar_arrive(bar(S::kRead + r));
                }
                const int j0 = (i0 + j < sink_tiles ? i0 + j : first_tile + i0 + j - sink_tiles) * kTile + 64 * half;
                if (!(j0 + 63 <= last_all && (j0 >= from_all || j0 + 64 <= p.sinks))) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int k0 = j0 + 32 * c;
                        const uint32_t sees = bits_to(last - k0) & (~bits_to(from - 1 - k0) | bits_to(p.sinks - 1 - k0));
                        if (__all_sync(0xffffffffu, sees == 0xFFFFFFFFu)) continue;
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (!(sees & (1u << e))) s[c][e] = 0xFF800000u;  // -inf
                    }
                }
                float top[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t *x = &s[i >> 1][(i & 1) * 16];
                    top[i] = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
#pragma unroll
                    for (int e = 2; e < 16; e += 2) top[i] = max3(top[i], __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
                }
                float most = max3(fmaxf(top[0], top[1]), top[2], top[3]);
                // Two buffers in turn: a thread writes one again two key tiles later, behind the pair's next barrier, which the other thread comes to
                // when it has read this.  (With one, nothing but time would lie between that read and the next write: of two row tiles the next
                // scores are formed as soon as these are in registers.)
                float *now = mosts + ((steps + j) & 1) * 256;
                now[half * 128 + row] = most;
                pair_sync();
                most = fmaxf(most, now[(half ^ 1) * 128 + row]);
                const bool outgrown = (most - m) * c2 > kSlack || (m == -INFINITY && most > -INFINITY);
                if (__any_sync(0xffffffffu, outgrown)) {
                    const float next = outgrown ? most : m, shrink = outgrown ? exp2f((m - next) * c2) : 1.f;
                    m = next;
                    l *= shrink;
                    if (j > 0) {
                        // all products so far are through (one row tile: they were before these scores): O is the row's threads' to change, a half each
                        if (kTiles == 2) {
                            ok = __all_sync(0xffffffffu, mbar_wait(bar(S::kOut + r), (steps + j - 1) & 1, abort_flag, sink));
                            tc_fence_after();
                        }
#pragma unroll 1
                        for (int c = 0; c < kDim / 2; c += 8) {              // (few registers at a time: the scores stay in theirs)
                            uint32_t o[8];
                            tmem_ld8(o_col + c, o);
                            tmem_wait8(o);
#pragma unroll
                            for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * shrink);
                            tmem_st8(o_col + c, o);
                        }
                    }
                }
                const float base = m == -INFINITY ? 0.f : -m * c2;
                const float2 scale = make_float2(c2, c2), shift = make_float2(base, base);
                float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                uint32_t w[2][16];
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float2 y = fma2(make_float2(__uint_as_float(s[c][2 * e]), __uint_as_float(s[c][2 * e + 1])), scale, shift);
                        // 64 dimensions, where the exponentials bound a step and not the products: one of eight elsewhere than in the special-
                        // function unit (a causal prompt of 8192 tokens 369 us, 337; one of four 358; 128 dimensions 424, 430 with one of eight)
                        y = kDim == 64 && e % 8 == 1 ? exp2_poly(y) : make_float2(exp2_approx(y.x), exp2_approx(y.y));
                        sum[e & 1] = add2(sum[e & 1], y);
                        w[c][e] = pack_bf16(y.x, y.y);
                    }
                if (kTiles == 2 && j > 0 && ok) {                            // the weights before these have been read
                    ok = __all_sync(0xffffffffu, mbar_wait(bar(S::kOut + r), (steps + j - 1) & 1, abort_flag, sink));
                    tc_fence_after();
                }
                tmem_st16(w_col, w[0]);
                tmem_st16(w_col + 16, w[1]);
                sum[0] = add2(sum[0], sum[1]);
                l += sum[0].x + sum[0].y;
                tmem_st_wait();
                tc_fence_before();
                mbar_arrive(bar(S::kWeights + r));
            }
            steps += T;
            Item x;
            load_item(p, idx, items, kTiles * tokens_per_tile, pieces, false, &x);
            if (ok && T > 0) ok = __all_sync(0xffffffffu, mbar_wait(bar(S::kOut + r), (steps - 1) & 1, abort_flag, sink));
            tc_fence_after();
            if (T > 0) {                                                     // (the other thread comes to the next item's when it has read these)
                sums[half * 128 + row] = l;
                pair_sync();
                l += sums[(half ^ 1) * 128 + row];
            }
            const int t = x.t0 + r * tokens_per_tile + row / p.group, qh = x.h * p.group + row % p.group, c0 = half * (kDim / 2);
            const bool mine = row < tokens_per_tile * p.group && t <= x.t1;  // else: nobody's row, computed and dropped
            const float inv = l == 0.f ? 0.f : 1.f / l;
            float *part = p.part ? p.part + (((size_t)(x.first + t) * p.hq + qh) * p.slots + p.slot + x.split) * slot_floats(kDim) : nullptr;
            __nv_bfloat16 *out = p.part ? nullptr : static_cast<__nv_bfloat16 *>(p.out) + (x.first + t) * p.out_stride + (size_t)qh * kDim;
#pragma unroll 1
            for (int c = 0; c < kDim / 2; c += 32) {
                uint32_t o[32];
                if (T > 0 && ok) {
                    tmem_ld32(o_col + c, o);
                    tmem_wait32(o);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = 0u;
                }
                if (T > 0 && c + 32 == kDim / 2) {                           // the next item's products may begin
                    tc_fence_before();
                    mbar_arrive(bar(S::kFree + r));
                }
                if (part) {
                    if (mine)
#pragma unroll
                        for (int e = 0; e < 32; e += 4) *reinterpret_cast<uint4 *>(part + c0 + c + e) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                    continue;
                }
                // Four lanes exchange the vectors of their rows, so that a store writes 64 bytes of eight rows, not 16 of 32: the rows lie far apart,
                // and a store takes a cycle per row.  (Written row by row the output held the next item up by 4000 cycles.)
                uint4 v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t *y = o + 8 * e;
                    v[e].x = pack_bf16(__uint_as_float(y[0]) * inv, __uint_as_float(y[1]) * inv);
                    v[e].y = pack_bf16(__uint_as_float(y[2]) * inv, __uint_as_float(y[3]) * inv);
                    v[e].z = pack_bf16(__uint_as_float(y[4]) * inv, __uint_as_float(y[5]) * inv);
                    v[e].w = pack_bf16(__uint_as_float(y[6]) * inv, __uint_as_float(y[7]) * inv);
                }
                transpose4(v);
#pragma unroll
                for (int e = 0; e < 4; ++e) {                            // row e of the four lanes', vector lane % 4
                    const unsigned long long to = __shfl_sync(0xffffffffu, mine ? reinterpret_cast<unsigned long long>(out) : 0ull, (lane & ~3) + e);
                    if (to) *reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(to) + c0 + c + (lane & 3) * 8) = v[e];
                }
            }
            // (a query that is no number leaves no maximum: any finite one makes the merge take the share in)
            if (mine && part && half == 0)
                *reinterpret_cast<float2 *>(part + kDim) = make_float2(!ok || T == 0 ? -INFINITY : l != l ? 0.f : m * c2, ok ? l : 0.f);
        }
    }

    // ---------------------------------------------------------------------- common exit
    tc_fence_before();
    __syncthreads();
    if (warp == kIssuer) {
        if (*abort_flag) __nanosleep(200000);      // error path only: let copies and products in flight land
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kCols) : "memory");
    }
}

// The queries as [token][head][dim]: a box is a row tile's whole tokens with the group's heads, 64 dimensions at a time.
bool make_map_queries(CUtensorMap *map, const RowsParams &p, int tokens_per_tile)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)p.d, (cuuint64_t)p.hq, (cuuint64_t)p.tokens.total};
    const cuuint64_t strides[2] = {(cuuint64_t)p.d * 2, (cuuint64_t)p.q_stride * 2};
    const cuuint32_t box[3] = {64u, (cuuint32_t)p.group, (cuuint32_t)tokens_per_tile}, estr[3] = {1u, 1u, 1u};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(p.q), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kDim, int kTiles>
cudaError_t launch_tc_for(const RowsParams &p, cudaStream_t s)
{
    using S = RowsShape<kDim, kTiles>;
    static PerDevice done;
    int dev = 0, sms = 0;
    cudaError_t e = device_sms(&dev, &sms);
    if (e != cudaSuccess) return e;
    if ((e = allow_smem_once(done, dev, rows_tc_kernel<kDim, kTiles>, S::kSmem)) != cudaSuccess) return e;
    const int tokens = kTile / p.group;
    const long long per_problem = ((long long)p.tokens.longest + kTiles * tokens - 1) / (kTiles * tokens);
    const long long items = per_problem * p.hkv * p.tokens.count * p.splits;
    if (items > 0x3fffffffll) return cudaErrorInvalidValue;
    const uint64_t rows = p.block_table ? (uint64_t)p.pool_pages * kTile
                                        : (uint64_t)p.tokens.count * p.hkv * (p.compact_tiles ? p.compact_tiles * kTile : p.cap);
    CUtensorMap mk, mv, mq;
    if (!make_map_rows(&mk, p.k, rows, kDim, kTile) || !make_map_rows(&mv, p.v, rows, kDim, kTile) || !make_map_queries(&mq, p, tokens))
        return cudaErrorInvalidValue;
    return launch_early(rows_tc_kernel<kDim, kTiles>, (unsigned)items, S::kThreads, S::kSmem, s, 1, p, tokens, (int)per_problem,
                        (int)items, mk, mv, mq);
}

}  // namespace

bool rows_sm100_supported(int dtype, int d, int group) { return dtype != RKV_F32 && (d == 64 || d == 128) && group <= kTile; }

// Two row tiles to a block where a problem has more than one (128 dimensions, windows of 512 and 2048: 13.0 and 35.7 us an item of 64 tokens, 15.0 and
// 41.8 as two; 64 sequences of 16 tokens, half a row tile each: 139 us with two, 98 with one).
int rows_sm100_tiles(const RowsParams &p) { return p.tokens.longest > kTile / p.group ? 2 : 1; }

cudaError_t launch_rows_sm100(const RowsParams &p, cudaStream_t s)
{
    if (rows_sm100_tiles(p) == 2) return p.d == 128 ? launch_tc_for<128, 2>(p, s) : launch_tc_for<64, 2>(p, s);
    return p.d == 128 ? launch_tc_for<128, 1>(p, s) : launch_tc_for<64, 1>(p, s);
}

}  // namespace rkv
