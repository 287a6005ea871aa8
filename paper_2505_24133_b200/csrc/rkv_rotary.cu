// New tokens enter their caches with the position rotation on the way: for every pair (x, y) of a head and the pair's angle a at the
// token's position, (x cos a - y sin a, x sin a + y cos a), in fp32 from a table of cosines and sines, rounded once to the cache's type.
//
// Byte movement with a few products on the way: every element is read once and written once.  A thread takes 16 elements of a head
// at a time, two vectors of eight that hold eight whole pairs, in either order of pairing; d / 16 threads take a head, and a warp stays
// with one token, so that the eight cosines and sines of a thread's pairs are loaded once for all heads that it comes to.
#include "rkv_tokens.cuh"

namespace rkv {

namespace {

constexpr int kRotThreads = 256, kRotStepThreads = 512;

// Eight consecutive elements of the token tensors as they lie, and as fp32.
template <typename T> struct Vec8;
template <> struct Vec8<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { *reinterpret_cast<uint4 *>(p) = v; }
    __device__ __forceinline__ void get(float *f) const { Elem<__nv_bfloat16>::unpack(v, f); }
    __device__ __forceinline__ void set(const float *f)
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <> struct Vec8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) { a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1]; }
    __device__ __forceinline__ void store(float *p) const { reinterpret_cast<float4 *>(p)[0] = a, reinterpret_cast<float4 *>(p)[1] = b; }
    __device__ __forceinline__ void get(float *f) const
    {
        f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w;
        f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    }
    __device__ __forceinline__ void set(const float *f) { a = make_float4(f[0], f[1], f[2], f[3]), b = make_float4(f[4], f[5], f[6], f[7]); }
};
// eight values to E4M3 codes: to nearest, beyond the largest code to that one, NaN to NaN
__device__ __forceinline__ uint2 to_codes(const float *f)
{
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * i], f[4 * i + 1]), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(f[4 * i + 2], f[4 * i + 3]), __NV_SATFINITE, __NV_E4M3);
        w[i] = lo | (hi << 16);
    }
    return make_uint2(w[0], w[1]);
}

// The sequence that token row t belongs to, or -1; the warp's lanes look at 32 entries at a time (a batch of up to 31 sequences in one
// load, of up to 1023 in two).  Entries that do not ascend give some sequence or none, and the caller checks that t lies in its range.
__device__ __forceinline__ int warp_find_sequence(const TokenMap &m, int t)
{
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = m.count + 1;                        // the last entry <= t lies in [lo, hi), if any does
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, i = lo + lane * step;
        const unsigned not_beyond = __ballot_sync(0xffffffffu, i < hi && m.offsets[i] <= t);
        if (!not_beyond) return -1;
        lo += (31 - __clz(not_beyond)) * step;
        hi = min(hi, lo + step);
    }
    return lo < m.count ? lo : -1;
}

// kOne, kFew: a block per sequence, for one token or a few; the length grows behind the block's own barrier.  Otherwise the warps of all blocks
// take tokens one by one (warps_per_token to each) and bump_tokens_kernel below follows, 3 us and a launch more.
enum { kMany, kOne, kFew };
template <typename T, bool kCodes, int kMode>
__global__ void __launch_bounds__(kMode != kMany ? kRotStepThreads : kRotThreads, kMode != kMany ? 1 : kCodes || sizeof(T) == 4 ? 2 : 3)
append_rotary_kernel(RotaryParams p)
{
    // Heads whose vectors a thread has under way.  16 prompts of 4096 tokens of 56 bf16 heads: 296 us with four and three blocks to an SM (0.98 of the
    // copy rate), 317 with two blocks; into 8-bit pages 161 with four, 187 with two.  Single tokens 3.6 us with one, 4.0 with four.
    constexpr int kAhead = kMode == kOne ? 1 : 4;
    constexpr bool kStep = kMode != kMany;
    constexpr int kWarps = (kStep ? kRotStepThreads : kRotThreads) / 32;
    pdl_trigger();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int lanes = p.d >> 4, u = lane & (lanes - 1);                  // threads of a head; this one's 16 elements
    const int per_warp = 32 / lanes, wpt = p.warps_per_token;
    int b, first, n, nth, sub;                                           // sequence, its tokens, the warp's (first) of them and its share of that
    if (kStep) {
        b = blockIdx.x;
        n = token_span(p.tokens, b, &first);
        if (n <= 0) {
            if (n < 0 && threadIdx.x == 0) report(p.status, RKV_ERR_INVALID_ARG);
            return;
        }
        nth = warp / wpt;
        sub = warp % wpt;
    } else {
        const long long slot = (long long)blockIdx.x * kWarps + warp;
        const int t = (int)(slot / wpt);
        sub = (int)(slot % wpt);
        if (t >= p.tokens.total) return;
        b = p.tokens.offsets ? warp_find_sequence(p.tokens, t) : t / p.tokens.longest;
        if (b < 0) return;                               // behind the last sequence
        n = token_span(p.tokens, b, &first);
        nth = t - first;
        if (n < 0 || nth < 0 || nth >= n) return;        // (bump_tokens_kernel reports the sequence)
    }

    const int half = p.dim >> 1;
    const bool turns = 16 * u < p.dim;
    const int at0 = turns && !p.interleaved ? 8 * u : 16 * u, at1 = turns && !p.interleaved ? half + 8 * u : 16 * u + 8;
    const int heads = 2 * p.hkv + p.hq, step = wpt * per_warp;
    const int item0 = sub * per_warp + lane / lanes;     // heads of K, then of V, then of the queries

    Vec8<T> x0[kAhead], x1[kAhead];
    long long t = (long long)first + nth;
    auto fetch = [&](int i, int it) {
        if (it >= heads || nth >= n) return;
        const T *src = it < p.hkv ? static_cast<const T *>(p.k_new) + t * p.k_stride + (size_t)it * p.d
                     : it < 2 * p.hkv ? static_cast<const T *>(p.v_new) + t * p.v_stride + (size_t)(it - p.hkv) * p.d
                                      : static_cast<const T *>(p.q_new) + t * p.q_stride + (size_t)(it - 2 * p.hkv) * p.d;
        const bool rotates = it < p.hkv || it >= 2 * p.hkv;
        x0[i].load(src + (rotates ? at0 : 16 * u));
        x1[i].load(src + (rotates ? at1 : 16 * u + 8));
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) fetch(i, item0 + i * step);         // under way together with what follows

    const int L = p.seq_lens[b];
    const long long pos0 = p.positions ? p.positions[b] : L;
    const bool fits = L >= 0 && n <= p.cap - L && (p.dim == 0 || (pos0 >= 0 && pos0 + n <= p.rows));
    if (!fits) {                                         // uniform for the warp (kStep: for the block)
        if (kStep && threadIdx.x == 0) report(p.status, RKV_ERR_INVALID_ARG);
        return;
    }
    for (; nth < n; nth += kWarps / wpt) {               // (kStep: its tokens; otherwise the one)
        float c[8], s[8];
        if (turns) {
            const float4 *row = reinterpret_cast<const float4 *>(p.table + (size_t)(pos0 + nth) * p.dim);
            const float4 c0 = row[2 * u], c1 = row[2 * u + 1], s0 = row[(half >> 2) + 2 * u], s1 = row[(half >> 2) + 2 * u + 1];
            c[0] = c0.x, c[1] = c0.y, c[2] = c0.z, c[3] = c0.w, c[4] = c1.x, c[5] = c1.y, c[6] = c1.z, c[7] = c1.w;
            s[0] = s0.x, s[1] = s0.y, s[2] = s0.z, s[3] = s0.w, s[4] = s1.x, s[5] = s1.y, s[6] = s1.z, s[7] = s1.w;
        }
        const int row = L + nth;
        for (int item = item0; item < heads; item += kAhead * step) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int it = item + i * step;
                if (it >= heads) break;
                const bool query = it >= 2 * p.hkv, turn = turns && (query || it < p.hkv);
                float f0[8], f1[8];
                if (turn || (kCodes && !query)) {
                    x0[i].get(f0);
                    x1[i].get(f1);
                }
                if (turn) {
                    if (p.interleaved) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float a = f0[2 * j], y = f0[2 * j + 1], e = f1[2 * j], z = f1[2 * j + 1];
                            f0[2 * j] = a * c[j] - y * s[j], f0[2 * j + 1] = a * s[j] + y * c[j];
                            f1[2 * j] = e * c[4 + j] - z * s[4 + j], f1[2 * j + 1] = e * s[4 + j] + z * c[4 + j];
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float a = f0[j], y = f1[j];
                            f0[j] = a * c[j] - y * s[j], f1[j] = a * s[j] + y * c[j];
                        }
                    }
                    if (!kCodes || query) {
                        x0[i].set(f0);
                        x1[i].set(f1);
                    }
                }
                const int o0 = query || it < p.hkv ? at0 : 16 * u, o1 = query || it < p.hkv ? at1 : 16 * u + 8;
                if (query) {
                    T *dst = static_cast<T *>(p.q_out) + t * p.out_stride + (size_t)(it - 2 * p.hkv) * p.d;
                    x0[i].store(dst + o0);
                    x1[i].store(dst + o1);
                    continue;
                }
                const int head = b * p.hkv + (it < p.hkv ? it : it - p.hkv);
                long long at = (long long)head * p.cap + row;
                if (p.block_table) {
                    const int page = p.block_table[(size_t)head * (p.cap / kTile) + row / kTile];
                    if (page < 0 || page >= p.pool_pages) {
                        report(p.status, RKV_ERR_INVALID_ARG);
                        continue;
                    }
                    at = (long long)page * kTile + row % kTile;
                }
                void *cache = it < p.hkv ? p.k_cache : p.v_cache;
                if (kCodes) {
                    uint8_t *dst = static_cast<uint8_t *>(cache) + at * p.d;
                    const uint2 c0 = to_codes(f0), c1 = to_codes(f1);
                    if (o1 == o0 + 8) {                      // side by side: values, keys whose pairs are
                        *reinterpret_cast<uint4 *>(dst + o0) = make_uint4(c0.x, c0.y, c1.x, c1.y);
                    } else {
                        *reinterpret_cast<uint2 *>(dst + o0) = c0;
                        *reinterpret_cast<uint2 *>(dst + o1) = c1;
                    }
                } else {
                    T *dst = static_cast<T *>(cache) + at * p.d;
                    x0[i].store(dst + o0);
                    x1[i].store(dst + o1);
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) fetch(i, item + (kAhead + i) * step);
        }
        if (!kStep) break;
        t += kWarps / wpt;
        nth += kWarps / wpt;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fetch(i, item0 + i * step);
        nth -= kWarps / wpt;
    }
    if (!kStep) return;
    __syncthreads();
    if (threadIdx.x == 0) p.seq_lens[b] = L + n;
}

// seq_lens[b] grows by the sequence's new tokens, by the same conditions, when the copies are through
__global__ void __launch_bounds__(kRotThreads) bump_tokens_kernel(RotaryParams p)
{
    pdl_trigger();
    pdl_wait();
    const int b = blockIdx.x * kRotThreads + threadIdx.x;
    if (b >= p.tokens.count) return;
    int first;
    const int n = token_span(p.tokens, b, &first), L = p.seq_lens[b];
    const long long pos0 = p.positions ? p.positions[b] : L;
    if (n == 0) return;
    if (n > 0 && L >= 0 && n <= p.cap - L && (p.dim == 0 || (pos0 >= 0 && pos0 + n <= p.rows))) p.seq_lens[b] = L + n;
    else report(p.status, RKV_ERR_INVALID_ARG);
}

template <typename T, bool kCodes>
cudaError_t launch_type(RotaryParams p, cudaStream_t s)
{
    const int groups = 32 / (p.d >> 4), most = (2 * p.hkv + p.hq + groups - 1) / groups;       // warps that a token's heads keep busy
    // A block per sequence where that gives its warps at most eight rounds of heads (8 tokens of 48 heads of 128 dimensions: 6), or one token.  In a
    // graph the two ways take about as long (8 tokens of 1 and of 64 sequences 6.7 and 7.2 us, 5.4 and 9.0 as two kernels; 3 tokens of 256: 10.3, 8.0);
    // eager calls save the second launch (8 tokens of 236 sequences 10.2 us, 15.6).
    constexpr int kStepWarps = kRotStepThreads / 32;
    if (p.tokens.longest == 1 || (long long)p.tokens.longest * most <= 8 * kStepWarps) {
        p.warps_per_token = 1;
        while (p.warps_per_token < kStepWarps && p.warps_per_token < most && p.warps_per_token * p.tokens.longest < kStepWarps) p.warps_per_token *= 2;
        return launch_early(p.tokens.longest == 1 ? append_rotary_kernel<T, kCodes, kOne> : append_rotary_kernel<T, kCodes, kFew>, (unsigned)p.tokens.count, kRotStepThreads, 0, s, 1, p);
    }
    // as many warps to a token as its heads keep busy, where the tokens alone do not fill the GPU (16 warps to each of 148 SMs)
    int wpt = 1;
    while (wpt < 8 && wpt < most && (long long)p.tokens.total * wpt < 148 * 16) wpt *= 2;
    p.warps_per_token = wpt;
    constexpr int kWarps = kRotThreads / 32;
    const long long blocks = ((long long)p.tokens.total * wpt + kWarps - 1) / kWarps;
    const cudaError_t e = launch_early(append_rotary_kernel<T, kCodes, kMany>, (unsigned)blocks, kRotThreads, 0, s, 1, p);
    if (e != cudaSuccess) return e;
    return launch_early(bump_tokens_kernel, (unsigned)((p.tokens.count + kRotThreads - 1) / kRotThreads), kRotThreads, 0, s, 1, p);
}

}  // namespace

cudaError_t launch_append_rotary(RotaryParams p, int dtype, cudaStream_t s)
{
    return dtype == RKV_F32 ? launch_type<float, false>(p, s) : dtype == RKV_BF16 ? launch_type<__nv_bfloat16, false>(p, s)
                                                                                  : launch_type<__nv_bfloat16, true>(p, s);
}

}  // namespace rkv
