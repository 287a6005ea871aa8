// Attention of many query rows over a cache, CUDA-core form (fp32 products), and the merge of partial results.
//
// A block takes 64 query rows (or 16: see rows_simt_rows) of one (problem, KV head) and goes once over its share of the key tiles, 64 keys
// at a time, with the running maximum and sum of the softmax; the weighted sum stays in registers.  256 threads as 16 x 16: a thread owns
// 4 x 4 scores (1 x 4), then 4 rows (1) x d / 16 columns of the output; the 16 threads that share rows are half a warp, so that the weights
// change hands within the warp.  Bound by fp32 FMAs and the shared-memory reads that feed them (8 vectors per 64 FMAs of the scores; 5 per 16).
#include <algorithm>

#include "rkv_tokens.cuh"

namespace rkv {

namespace {

constexpr int kKeys = 64, kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

template <typename T> __device__ __forceinline__ float4 load4(const T *p);
template <> __device__ __forceinline__ float4 load4<float>(const float *p) { return *reinterpret_cast<const float4 *>(p); }
template <> __device__ __forceinline__ float4 load4<__nv_bfloat16>(const __nv_bfloat16 *p)
{
    const uint2 v = *reinterpret_cast<const uint2 *>(p);
    const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&v.x)), b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&v.y));
    return make_float4(a.x, a.y, b.x, b.y);
}
template <> __device__ __forceinline__ float4 load4<uint8_t>(const uint8_t *p)           // E4M3 codes
{
    const uint32_t v = *reinterpret_cast<const uint32_t *>(p);
    const __half2_raw a = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v & 0xFFFFu), __NV_E4M3);
    const __half2_raw b = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v >> 16), __NV_E4M3);
    const float2 x = __half22float2(*reinterpret_cast<const __half2 *>(&a)), y = __half22float2(*reinterpret_cast<const __half2 *>(&b));
    return make_float4(x.x, x.y, y.x, y.y);
}
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }

__device__ __forceinline__ void store4(float *p, float4 v) { *reinterpret_cast<float4 *>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float4 v)
{
    const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}

template <int kDim, int kPer> constexpr int rows_simt_smem()
{
    return ((16 * kPer + kKeys) * (kDim + 4) + kKeys * kDim + 16 * kPer * (kKeys + 4)) * 4;
}

// kPer: rows of a thread
template <typename TQ, typename TC, int kDim, int kPer>
__global__ void __launch_bounds__(kThreads, kDim == 256 ? 1 : 2) rows_simt_kernel(RowsParams p, int row_tiles)
{
    constexpr int kRows = 16 * kPer, kStride = kDim + 4, kPStride = kKeys + 4, kVecs = kDim / 4, kCols = kDim / 64;
    extern __shared__ float rows_smem[];
    float *sq = rows_smem, *sk = sq + kRows * kStride, *sv = sk + kKeys * kStride, *sp = sv + kKeys * kDim;
    pdl_wait();
    pdl_trigger();                                               // (in this order: see AttendTcMore::late)
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    int x = blockIdx.x;
    const int split = x % p.splits;
    x /= p.splits;
    const int tile = row_tiles - 1 - x % row_tiles;              // a prompt's last rows see the most keys: first
    x /= row_tiles;
    const int h = x % p.hkv, b = x / p.hkv;

    int first;
    const int n = token_span(p.tokens, b, &first);
    int len = p.lens[b];
    if (n < 0 || len < 0 || len > p.cap || (p.causal && len < n)) {
        if (threadIdx.x == 0) report(p.status, RKV_ERR_INVALID_ARG);
        len = 0;
    }
    const int r0 = tile * kRows, rows = min(kRows, n * p.group - r0);
    if (n <= 0 || rows <= 0) return;
    const bool empty = len == 0;
    KeyTiles keys = key_tiles(p.causal, p.window, p.sinks, len, n, r0 / p.group, (r0 + rows - 1) / p.group);
    if (empty) keys.count = 0;
    const int per = (keys.count + p.splits - 1) / p.splits, i0 = split * per, i1 = min(keys.count, i0 + per);

    const TQ *q = static_cast<const TQ *>(p.q);
    for (int v = threadIdx.x; v < kRows * kVecs; v += kThreads) {
        const int r = v / kVecs, c = v % kVecs * 4;
        float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < rows) {
            const int t = (r0 + r) / p.group, g = (r0 + r) % p.group;
            f = load4<TQ>(q + (first + t) * p.q_stride + ((size_t)h * p.group + g) * kDim + c);
        }
        *reinterpret_cast<float4 *>(sq + r * kStride + c) = f;
    }

    // of this thread's rows: the last and the first cached row that each sees
    int last[kPer], from[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int at = len - n + (r0 + ty * kPer + i) / p.group;
        last[i] = p.causal ? at : len - 1;
        from[i] = p.causal && p.window > 0 ? at + 1 - p.window : 0;
    }
    const float scale = kLog2e * rsqrtf((float)kDim);
    float m[kPer], l[kPer], o[kPer][kDim / 16];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        m[i] = -INFINITY, l[i] = 0.f;
#pragma unroll
        for (int c = 0; c < kDim / 16; ++c) o[i][c] = 0.f;
    }
    const TC *kc = static_cast<const TC *>(p.k), *vc = static_cast<const TC *>(p.v);
    const int head = b * p.hkv + h;
    // half a tile of 128 keys at a time; with one row to a thread there are registers to have the next half under way meanwhile
    constexpr int kLoads = kKeys * kVecs / kThreads;
    constexpr bool kAhead = kPer == 1;
    float4 next_k[kLoads], next_v[kLoads];
    auto fetch = [&](int step) {
        const int t = keys.tile(step >> 1), j0 = t * kTile + (step & 1) * kKeys;
        const long long tile_start = rows_tile_start(p, head, t), start = tile_start + (step & 1) * kKeys;
        if (tile_start < 0 && threadIdx.x == 0) report(p.status, RKV_ERR_INVALID_ARG);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int v = i * kThreads + threadIdx.x, r = v / kVecs, c = v % kVecs * 4;
            next_k[i] = next_v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (tile_start >= 0 && keys.wanted(j0 + r)) {
                next_k[i] = load4<TC>(kc + (start + r) * kDim + c);
                next_v[i] = load4<TC>(vc + (start + r) * kDim + c);
            }
        }
    };
    if (kAhead && i0 < i1) fetch(2 * i0);
    for (int step = 2 * i0; step < 2 * i1; ++step) {
        const int j0 = keys.tile(step >> 1) * kTile + (step & 1) * kKeys;
        if (!kAhead) fetch(step);
        __syncthreads();                                         // the tiles of the step before have been read
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int v = i * kThreads + threadIdx.x, r = v / kVecs, c = v % kVecs * 4;
            *reinterpret_cast<float4 *>(sk + r * kStride + c) = next_k[i];
            *reinterpret_cast<float4 *>(sv + r * kDim + c) = next_v[i];
        }
        __syncthreads();
        if (kAhead && step + 1 < 2 * i1) fetch(step + 1);
        float s[kPer][4];
#pragma unroll
        for (int i = 0; i < kPer; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
        for (int c = 0; c < kDim; c += 4) {
            float4 a[kPer], e[4];
#pragma unroll
            for (int i = 0; i < kPer; ++i) a[i] = *reinterpret_cast<const float4 *>(sq + (ty * kPer + i) * kStride + c);
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = *reinterpret_cast<const float4 *>(sk + (tx + 16 * j) * kStride + c);
#pragma unroll
            for (int i = 0; i < kPer; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    s[i][j] = fmaf(a[i].x, e[j].x, fmaf(a[i].y, e[j].y, fmaf(a[i].z, e[j].z, fmaf(a[i].w, e[j].w, s[i][j]))));
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            float top = m[i];
            bool sees[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int key = j0 + tx + 16 * j;
                sees[j] = key <= last[i] && (key >= from[i] || key < p.sinks);
                s[i][j] *= scale;
                if (sees[j]) top = fmaxf(top, s[i][j]);
            }
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            const float base = top == -INFINITY ? 0.f : top;     // (no key seen yet: every weight is 0)
            const float shrink = exp2f(m[i] - base);
            m[i] = top;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float w = sees[j] ? exp2f(s[i][j] - base) : 0.f;
                sum += w;
                sp[(ty * kPer + i) * kPStride + tx + 16 * j] = w;
            }
            l[i] = l[i] * shrink + sum;                          // (of this thread's keys; added up at the end)
#pragma unroll
            for (int c = 0; c < kDim / 16; ++c) o[i][c] *= shrink;
        }
        __syncwarp();
#pragma unroll 4
        for (int k = 0; k < kKeys; k += 4) {
            float4 w[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) w[i] = *reinterpret_cast<const float4 *>(sp + (ty * kPer + i) * kPStride + k);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                    const float4 e = *reinterpret_cast<const float4 *>(sv + (k + kk) * kDim + c * 64 + tx * 4);
#pragma unroll
                    for (int i = 0; i < kPer; ++i) {
                        const float f = kk == 0 ? w[i].x : kk == 1 ? w[i].y : kk == 2 ? w[i].z : w[i].w;
                        o[i][4 * c] = fmaf(f, e.x, o[i][4 * c]), o[i][4 * c + 1] = fmaf(f, e.y, o[i][4 * c + 1]);
                        o[i][4 * c + 2] = fmaf(f, e.z, o[i][4 * c + 2]), o[i][4 * c + 3] = fmaf(f, e.w, o[i][4 * c + 3]);
                    }
                }
        }
        __syncwarp();
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], off);
        const int r = ty * kPer + i;
        if (r >= rows) continue;
        const int t = first + (r0 + r) / p.group, qh = h * p.group + (r0 + r) % p.group;
        if (p.part) {
            float *dst = p.part + (((size_t)t * p.hq + qh) * p.slots + p.slot + split) * slot_floats(kDim);
#pragma unroll
            for (int c = 0; c < kDim / 16; ++c) dst[(c >> 2) * 64 + tx * 4 + (c & 3)] = o[i][c];
            if (tx == 0) dst[kDim] = l[i] != l[i] ? 0.f : m[i], dst[kDim + 1] = l[i];      // (no number: the merge must take it in)
        } else {
            TQ *dst = static_cast<TQ *>(p.out) + t * p.out_stride + (size_t)qh * kDim;
#pragma unroll
            for (int c = 0; c < kDim / 16; ++c) put(dst + (c >> 2) * 64 + tx * 4 + (c & 3), l[i] == 0.f ? 0.f : o[i][c] / l[i]);
        }
    }
}

// out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s over a row's slots, in fixed order; a warp per row.  The loads of eight slots are under way
// at a time (one after the other they took a memory latency each).
constexpr int kMergeWarps = 4, kMergeAhead = 8;
template <typename TQ>
__global__ void __launch_bounds__(kMergeWarps * 32) rows_merge_kernel(RowsParams p)
{
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * kMergeWarps + (threadIdx.x >> 5);
    if (row >= (long long)p.tokens.total * p.hq) return;
    const int t = (int)(row / p.hq), qh = (int)(row % p.hq);
    if (p.tokens.offsets) {                                      // rows of no sequence stay as they are
        int first = 0, lo = 0, hi = p.tokens.count;              // the last sequence that starts at or before t
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            (p.tokens.offsets[mid] <= t ? lo : hi) = mid;
        }
        const int n = token_span(p.tokens, lo, &first);
        if (t < first || t >= first + n) return;
    }
    const int stride = slot_floats(p.d);
    const float *part = p.part + (size_t)row * p.slots * stride;
    for (int c = lane * 4; c < p.d; c += 128) {
        float m = -INFINITY, den = 0.f;
        float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s0 = 0; s0 < p.slots; s0 += kMergeAhead) {
            float4 o[kMergeAhead];
            float2 ml[kMergeAhead];
            float top = m;
#pragma unroll
            for (int i = 0; i < kMergeAhead; ++i) {
                ml[i] = make_float2(-INFINITY, 0.f);
                if (s0 + i < p.slots) {
                    o[i] = *reinterpret_cast<const float4 *>(part + (s0 + i) * stride + c);
                    ml[i] = *reinterpret_cast<const float2 *>(part + (s0 + i) * stride + p.d);
                }
                top = fmaxf(top, ml[i].x);
            }
            if (top == -INFINITY) continue;                      // no visible key so far
            const float old = exp2f(m - top);
            den *= old, num.x *= old, num.y *= old, num.z *= old, num.w *= old;
            m = top;
#pragma unroll
            for (int i = 0; i < kMergeAhead; ++i) {
                if (ml[i].x == -INFINITY) continue;              // a share without a visible key
                const float w = exp2f(ml[i].x - m);
                den = fmaf(w, ml[i].y, den);
                num.x = fmaf(w, o[i].x, num.x), num.y = fmaf(w, o[i].y, num.y), num.z = fmaf(w, o[i].z, num.z), num.w = fmaf(w, o[i].w, num.w);
            }
        }
        const float inv = den == 0.f ? 0.f : 1.f / den;
        store4(static_cast<TQ *>(p.out) + t * p.out_stride + (size_t)qh * p.d + c, make_float4(num.x * inv, num.y * inv, num.z * inv, num.w * inv));
    }
}

template <typename TQ, typename TC, int kDim, int kPer>
cudaError_t launch_simt_for(const RowsParams &p, cudaStream_t s)
{
    static PerDevice done;
    int dev = 0, sms = 0;
    cudaError_t e = device_sms(&dev, &sms);
    if (e != cudaSuccess) return e;
    if ((e = allow_smem_once(done, dev, rows_simt_kernel<TQ, TC, kDim, kPer>, rows_simt_smem<kDim, kPer>())) != cudaSuccess) return e;
    const long long row_tiles = ((long long)p.tokens.longest * p.group + 16 * kPer - 1) / (16 * kPer);
    const long long blocks = row_tiles * p.hkv * p.tokens.count * p.splits;
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    return launch_early(rows_simt_kernel<TQ, TC, kDim, kPer>, (unsigned)blocks, kThreads, rows_simt_smem<kDim, kPer>(), s, 1, p, (int)row_tiles);
}
template <typename TQ, typename TC, int kDim>
cudaError_t launch_simt_dim(const RowsParams &p, cudaStream_t s)
{
    return rows_simt_rows(p) == 16 ? launch_simt_for<TQ, TC, kDim, 1>(p, s) : launch_simt_for<TQ, TC, kDim, 4>(p, s);
}
template <typename TQ, typename TC>
cudaError_t launch_simt_type(const RowsParams &p, cudaStream_t s)
{
    return p.d == 64 ? launch_simt_dim<TQ, TC, 64>(p, s) : p.d == 128 ? launch_simt_dim<TQ, TC, 128>(p, s) : launch_simt_dim<TQ, TC, 256>(p, s);
}

}  // namespace

// Query rows of a block: 16 where the problems have no more, or where tiles of 64 and all splits of the keys would leave most of the SMs idle.
// (Four heads a token, us with 64, 16.  16 single tokens of window 1024: 195, 114.  64 dimensions, tiles of 64 rows x key tiles: 8 sequences behind 300
// rows, 24, 45.1, 31.1; 32 behind 330, 48, 72.3, 36.9; 64 behind 150, 64, 66.6, 51.1; 16 behind 2000, 128, 38.9, 41.3; 64 behind 1000, 256, 51.3, 75.0.
// A prompt of 64 tokens, 32, 23.9, 14.9; of 200, 208, 42.0, 58.1.)
int rows_simt_rows(const RowsParams &p)
{
    const long long rows = (long long)p.tokens.longest * p.group;
    if (rows <= 16) return 16;
    long long keys = p.cap;
    if (p.causal && p.window > 0) keys = std::min(keys, (long long)p.window + p.sinks + p.tokens.longest);
    const double pairs = (double)((rows + 63) / 64) * p.hkv * p.tokens.count * (double)((keys + kTile - 1) / kTile);
    return pairs <= 64 ? 16 : 64;
}

cudaError_t launch_rows_simt(const RowsParams &p, int dtype, cudaStream_t s)
{
    return dtype == RKV_F32 ? launch_simt_type<float, float>(p, s) : dtype == RKV_BF16 ? launch_simt_type<__nv_bfloat16, __nv_bfloat16>(p, s)
                                                                                       : launch_simt_type<__nv_bfloat16, uint8_t>(p, s);
}

cudaError_t launch_rows_merge(const RowsParams &p, int dtype, cudaStream_t s)
{
    const long long blocks = ((long long)p.tokens.total * p.hq + kMergeWarps - 1) / kMergeWarps;
    if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
    return launch_early(dtype == RKV_F32 ? rows_merge_kernel<float> : rows_merge_kernel<__nv_bfloat16>, (unsigned)blocks, kMergeWarps * 32, 0, s, 1, p);
}

}  // namespace rkv
