// C ABI of the calls on several new tokens per sequence: argument checks and launches.  See include/rkv.h for their contracts.
#include "rkv_tokens.cuh"

namespace rkv {

namespace {

// The descriptor and the capacity.
int check_cache(const rkv_desc_t *d, int budget, int buffer)
{
    if (!d || d->batch < 1 || d->n_kv_heads < 1 || d->n_q_heads < 1 || d->n_q_heads % d->n_kv_heads != 0) return RKV_ERR_INVALID_ARG;
    if (budget < 1 || buffer < 0) return RKV_ERR_INVALID_ARG;
    if (d->head_dim != 64 && d->head_dim != 128 && d->head_dim != 256) return RKV_ERR_UNSUPPORTED;
    if (d->dtype != RKV_BF16 && d->dtype != RKV_F32 && d->dtype != RKV_FP8_E4M3) return RKV_ERR_UNSUPPORTED;
    const long long cap = (long long)budget + buffer;
    if (cap > RKV_MAX_ROWS || (long long)d->batch * d->n_kv_heads > (1ll << 24) || d->n_q_heads > (1 << 16)) return RKV_ERR_UNSUPPORTED;
    if (d->block_table) {
        if (cap % kTile != 0 || d->pool_pages < 1 || d->pool_pages > (1ll << 23)) return RKV_ERR_INVALID_ARG;
        if (reinterpret_cast<uintptr_t>(d->block_table) & 3u) return RKV_ERR_INVALID_ARG;
    }
    return RKV_OK;
}

// Elements from token to token: `stride` as the caller gives it, or rows back to back.  0: no valid one.
long long row_stride(int64_t stride, long long heads, int head_dim, size_t esz)
{
    const long long row = heads * head_dim;
    if (stride == 0) return row;
    return stride < row || stride > (1ll << 40) || (stride * (long long)esz) % 16 != 0 ? 0 : stride;
}

int check_tokens(const rkv_desc_t *d, const rkv_tokens_t *t, TokenMap *m)
{
    if (!t || t->total < 0 || t->longest < 1 || (reinterpret_cast<uintptr_t>(t->offsets) & 3u)) return RKV_ERR_INVALID_ARG;
    if (!t->offsets && (long long)d->batch * t->longest != t->total) return RKV_ERR_INVALID_ARG;
    if (t->total > (1 << 26)) return RKV_ERR_UNSUPPORTED;
    *m = TokenMap{t->offsets, d->batch, t->total, t->longest};
    return RKV_OK;
}

}  // namespace
}  // namespace rkv

using namespace rkv;

extern "C" {

int rkv_append_rotary(const rkv_desc_t *d, void *k_cache, void *v_cache, const void *k_new, const void *v_new, int32_t *seq_lens,
                      int32_t budget, int32_t buffer, const rkv_tokens_t *tokens, const rkv_rotary_t *rotary, const void *q_new,
                      void *q_out, void *stream)
{
    int rc = check_cache(d, budget, buffer);
    if (rc != RKV_OK) return rc;
    RotaryParams p = {};
    if ((rc = check_tokens(d, tokens, &p.tokens)) != RKV_OK) return rc;
    if (!k_cache || !v_cache || !k_new || !v_new || !seq_lens || !rotary || !q_new != !q_out) return RKV_ERR_INVALID_ARG;
    for (const void *x : {(const void *)k_cache, (const void *)v_cache, k_new, v_new, q_new, (const void *)q_out})
        if (!aligned16(x)) return RKV_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(seq_lens) | reinterpret_cast<uintptr_t>(rotary->positions)) & 3u) return RKV_ERR_INVALID_ARG;
    if (rotary->dim < 0 || rotary->dim % 16 != 0 || rotary->dim > d->head_dim) return RKV_ERR_INVALID_ARG;
    if (rotary->dim > 0 && (!rotary->table || !aligned16(rotary->table) || rotary->rows < 1)) return RKV_ERR_INVALID_ARG;
    const size_t esz = d->dtype == RKV_F32 ? 4 : 2;
    p.k_stride = row_stride(tokens->k_stride, d->n_kv_heads, d->head_dim, esz);
    p.v_stride = row_stride(tokens->v_stride, d->n_kv_heads, d->head_dim, esz);
    p.q_stride = row_stride(tokens->q_stride, d->n_q_heads, d->head_dim, esz);
    p.out_stride = row_stride(tokens->out_stride, d->n_q_heads, d->head_dim, esz);
    if (!p.k_stride || !p.v_stride || (q_new && (!p.q_stride || !p.out_stride))) return RKV_ERR_INVALID_ARG;
    if (q_new && q_new == q_out && p.q_stride != p.out_stride) return RKV_ERR_INVALID_ARG;
    if (tokens->total == 0) return RKV_OK;
    p.k_cache = k_cache, p.v_cache = v_cache;
    p.k_new = k_new, p.v_new = v_new, p.q_new = q_new, p.q_out = q_out;
    p.seq_lens = seq_lens;
    p.hkv = d->n_kv_heads;
    p.hq = q_new ? d->n_q_heads : 0;
    p.d = d->head_dim;
    p.cap = budget + buffer;
    p.table = rotary->table;
    p.rows = rotary->rows;
    p.dim = rotary->dim;
    p.interleaved = rotary->interleaved ? 1 : 0;
    p.positions = rotary->positions;
    p.block_table = d->block_table;
    p.pool_pages = d->pool_pages;
    p.status = d->device_status;
    const cudaError_t e = launch_append_rotary(p, d->dtype, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? RKV_OK : cuda_fail(e, "rotated append launch");
}

}  // extern "C"
