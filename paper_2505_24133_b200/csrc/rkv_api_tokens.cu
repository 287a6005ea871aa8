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
    // (rows of all heads are numbered in 32 bits; so many would not fit the GPU's memory)
    if (!d->block_table && (long long)d->batch * d->n_kv_heads * cap > 0x7fffffffll) return RKV_ERR_UNSUPPORTED;
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

int sm_count()
{
    int dev = 0, sms = 0;
    return device_sms(&dev, &sms) == cudaSuccess ? sms : 148;    // sizing only (no device here): the B200's count
}

constexpr int kSimtRows = 64, kMaxSplits = 64;
// key tiles that so many tokens in a row see at most
long long tiles_seen(const RowsParams &p, int tokens)
{
    const long long all = (p.cap + kTile - 1) / kTile;
    if (!p.causal || p.window == 0) return all;
    const long long tiles = ((long long)p.window + tokens) / kTile + 2 + ((long long)p.sinks + kTile - 1) / kTile;
    return tiles < all ? tiles : all;
}
// Splits of the key tiles: the shortest run, counted in key tiles of a block -- waves of blocks times the tiles of each and three more
// for its start and end, and for the merge two and what it takes to write and read the shares at 4 TB/s (a key tile takes `tile_us`).
// (Without that last term a chunk of 1000 tokens over 8000 rows was cut in four: 270 us, and 130 for the merge of 118 MB.)
int rows_splits(const RowsParams &p, int tokens_per_block, long long resident, double tile_us)
{
    const long long blocks = ((long long)p.tokens.longest + tokens_per_block - 1) / tokens_per_block * p.hkv * p.tokens.count;
    const long long tiles = tiles_seen(p, tokens_per_block);
    const double share = (double)p.tokens.total * p.hq * (p.d + 2) * 4 * 2 / 4e6 / tile_us;
    long long best = 1;
    double best_cost = 0;
    for (long long s = 1; s <= tiles && s <= kMaxSplits; ++s) {
        const long long per = (tiles + s - 1) / s;
        if (s > 1 && (tiles + per - 1) / per < s) continue;              // the last ones would have no tile
        const double cost = (double)((blocks * s + resident - 1) / resident) * (per + 3) + (s > 1 ? 2 + s * share : 0);
        if (s == 1 || cost < best_cost) best = s, best_cost = cost;
    }
    return (int)best;
}
bool on_tensor_cores(const rkv_desc_t *d) { return rows_sm100_supported(d->dtype, d->head_dim, d->n_q_heads / d->n_kv_heads); }
int splits_for(const rkv_desc_t *d, const RowsParams &p, long long sms)
{
    if (!on_tensor_cores(d)) {
        const int rows = rows_simt_rows(p);
        return rows_splits(p, p.group >= rows ? 1 : rows / p.group, 2 * sms, rows == 16 ? 4.0 : 12.0);
    }
    const int tiles = rows_sm100_tiles(p);
    return rows_splits(p, tiles * (kTile / p.group), tiles == 2 ? sms : 2 * sms, 1.6);
}
// Room for the bf16 copy of what a call of the tensor-core kernel sees of 8-bit caches.
size_t wide_bytes(const rkv_desc_t *d, const RowsParams &p)
{
    if (d->dtype != RKV_FP8_E4M3 || !on_tensor_cores(d)) return 0;
    return (size_t)p.tokens.count * p.hkv * tiles_seen(p, p.tokens.longest) * kTile * p.d * 2 * sizeof(__nv_bfloat16);
}
cudaError_t launch_rows(const rkv_desc_t *d, RowsParams p, void *wide, cudaStream_t s)
{
    if (!on_tensor_cores(d)) return launch_rows_simt(p, d->dtype, s);
    if (d->dtype == RKV_FP8_E4M3) {
        const cudaError_t e = launch_rows_widen(&p, wide, (int)tiles_seen(p, p.tokens.longest), s);
        if (e != cudaSuccess) return e;
    }
    return launch_rows_sm100(p, s);
}
size_t part_bytes(const RowsParams &p) { return align_up((size_t)p.tokens.total * p.hq * p.slots * slot_floats(p.d) * sizeof(float), 256); }

int check_room(const rkv_desc_t *d, size_t bytes)
{
    if (bytes == 0) return RKV_OK;
    if (!d->workspace || d->workspace_bytes < bytes || (reinterpret_cast<uintptr_t>(d->workspace) & 255u)) return RKV_ERR_WORKSPACE;
    return RKV_OK;
}

// What a descriptor says about the rows' kernels.
void fill_rows(const rkv_desc_t *d, int cap, RowsParams *p)
{
    p->hkv = d->n_kv_heads;
    p->hq = d->n_q_heads;
    p->group = d->n_q_heads / d->n_kv_heads;
    p->d = d->head_dim;
    p->cap = cap;
    p->block_table = d->block_table;
    p->pool_pages = d->pool_pages;
    p->status = d->device_status;
    p->wait_cycles = d->wait_limit_cycles > 0 ? (long long)d->wait_limit_cycles : sm100_default_wait_cycles();
    p->splits = p->slots = 1;
}

// A call's kernels: the rows' kernel, or for single tokens the decode attention's.
struct Plan {
    RowsParams rows;
    bool single, separate;       // separate: its splits are blocks of their own
    bool joined;                 // single: the kernel reads the prefixes itself, for every sequence again
    long long tiles;             // single: key tiles that a token sees at most
    size_t wide, bytes;          // workspace: the partial results, then from `wide` on the copies of 8-bit caches
};
bool back_to_back(const rkv_desc_t *d, int64_t stride) { return stride == 0 || stride == (int64_t)d->n_q_heads * d->head_dim; }

int plan_window(const rkv_desc_t *d, int budget, int buffer, const rkv_tokens_t *tokens, int window, int sinks, Plan *x)
{
    int rc = check_cache(d, budget, buffer);
    if (rc != RKV_OK) return rc;
    *x = Plan{};
    RowsParams *p = &x->rows;
    if ((rc = check_tokens(d, tokens, &p->tokens)) != RKV_OK) return rc;
    if (window < 0 || sinks < 0) return RKV_ERR_INVALID_ARG;
    const long long rows = (long long)tokens->longest * (d->n_q_heads / d->n_kv_heads);
    if (rows > (1ll << 30) || (rows + kSimtRows - 1) / kSimtRows * d->n_kv_heads * d->batch > (1ll << 28)) return RKV_ERR_UNSUPPORTED;
    fill_rows(d, budget + buffer, p);
    p->causal = 1;
    p->window = window;
    p->sinks = sinks;
    const long long tiles = x->tiles = tiles_seen(*p, 1);
    x->single = !tokens->offsets && tokens->longest == 1 && back_to_back(d, tokens->q_stride) && back_to_back(d, tokens->out_stride) &&
                attend_more_supported(d->dtype, d->head_dim, p->group, tiles);
    if (x->single) {
        attend_more_plan(p, d->dtype, tiles, sm_count(), false, &x->separate);
        p->slots = x->separate ? p->splits : 0;
        x->wide = x->bytes = x->separate ? part_bytes(*p) : 0;
    } else {
        p->splits = p->slots = splits_for(d, *p, sm_count());
        x->wide = p->slots > 1 ? part_bytes(*p) : 0;
        x->bytes = x->wide + wide_bytes(d, *p);
    }
    return RKV_OK;
}

int check_prefix(const rkv_desc_t *d, const rkv_prefix_t *x)
{
    if (!x || x->count < 1 || d->batch % x->count != 0 || x->rows < 1) return RKV_ERR_INVALID_ARG;
    if (x->rows > RKV_MAX_ROWS || (!x->table && (long long)x->count * d->n_kv_heads * x->rows > 0x7fffffffll)) return RKV_ERR_UNSUPPORTED;
    if (x->table && (x->rows % kTile != 0 || x->pages < 1 || x->pages > (1ll << 23) || (reinterpret_cast<uintptr_t>(x->table) & 3u)))
        return RKV_ERR_INVALID_ARG;
    return RKV_OK;
}

// (Eager figures, one kernel and two: 8 sequences x 4 heads, 333 rows, 5 MB 9.1 us, 15.8; 32 x 8, 330 rows, 41 MB 13.5, 18.8; 4 x 8, 3000 rows, 47 MB
// 17.4, 14.5; 64 x 8, 500 rows, 125 MB 27.7, 22.4; one sequence, 16000 rows 14.4, 25.3.  Fp32 caches, whose prefixes go to the CUDA cores otherwise:
// 32 x 8, 330 rows, 82 MB 45.8, 97.5; 4 x 8, 3000 rows, 94 MB 25.2, 35.6; 16 x 8, 2000 rows, 250 MB 57.5, 39.4; 64 x 8, 500 rows, 250 MB 88.8, 75.6;
// 64 x 8, 1000 rows, 500 MB 113.9, 73.0.)
constexpr long long kReadAgainBytes = 48ll << 20, kReadAgainBytesF32 = 160ll << 20;

// shared: the prefixes' rows, whose partial results are a row's first slots; own: the sequences'.
int plan_prefix(const rkv_desc_t *d, int budget, int buffer, const rkv_prefix_t *x, RowsParams *shared, Plan *own)
{
    int rc = check_cache(d, budget, buffer);
    if (rc != RKV_OK || (rc = check_prefix(d, x)) != RKV_OK) return rc;
    if ((long long)d->batch * d->n_q_heads > (1ll << 28)) return RKV_ERR_UNSUPPORTED;
    *shared = RowsParams{};
    *own = Plan{};
    RowsParams *p = &own->rows;
    fill_rows(d, x->rows, shared);
    shared->block_table = x->table;
    shared->pool_pages = x->pages;
    shared->tokens = TokenMap{nullptr, x->count, d->batch, d->batch / x->count};
    const int sms = sm_count();
    fill_rows(d, budget + buffer, p);
    p->tokens = TokenMap{nullptr, d->batch, d->batch, 1};
    // Prefixes of few rows or few sequences are read again for every sequence, mostly from L2: one kernel instead of two, the second of which
    // waits for the first.
    const long long elem = d->dtype == RKV_F32 ? 4 : d->dtype == RKV_BF16 ? 2 : 1;
    const long long again = (long long)d->batch * d->n_kv_heads * x->rows * 2 * d->head_dim * elem;
    const long long tiles = tiles_seen(*p, 1), with_prefix = tiles + tiles_seen(*shared, 1);
    own->joined = (again <= (d->dtype == RKV_F32 ? kReadAgainBytesF32 : kReadAgainBytes) || d->batch == x->count) &&
                  attend_more_supported(d->dtype, d->head_dim, p->group, with_prefix);
    own->tiles = own->joined ? with_prefix : tiles;
    own->single = own->joined || attend_more_supported(d->dtype, d->head_dim, p->group, tiles);
    if (own->single) attend_more_plan(p, d->dtype, own->tiles, sms, !own->joined, &own->separate);
    else p->splits = splits_for(d, *p, sms);
    if (own->joined) {
        p->slots = own->separate ? p->splits : 0;
        own->wide = own->bytes = own->separate ? part_bytes(*p) : 0;
        return RKV_OK;
    }
    shared->splits = splits_for(d, *shared, sms);
    p->slot = shared->splits;
    shared->slots = p->slots = shared->splits + (own->single && !own->separate ? 0 : p->splits);
    own->wide = part_bytes(*p);
    own->bytes = own->wide + wide_bytes(d, *shared) + (own->single ? 0 : wide_bytes(d, *p));
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

size_t rkv_window_workspace_bytes(const rkv_desc_t *d, int32_t budget, int32_t buffer, const rkv_tokens_t *tokens, int32_t window,
                                  int32_t sinks)
{
    Plan x;
    return plan_window(d, budget, buffer, tokens, window, sinks, &x) == RKV_OK ? x.bytes : 0;
}

int rkv_window_attention(const rkv_desc_t *d, const void *k_cache, const void *v_cache, const void *q, const int32_t *seq_lens, void *out,
                         int32_t budget, int32_t buffer, const rkv_tokens_t *tokens, int32_t window, int32_t sinks, void *stream)
{
    Plan x;
    int rc = plan_window(d, budget, buffer, tokens, window, sinks, &x);
    if (rc != RKV_OK) return rc;
    if (!k_cache || !v_cache || !q || !seq_lens || !out) return RKV_ERR_INVALID_ARG;
    if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(q) || !aligned16(out)) return RKV_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(seq_lens) & 3u) return RKV_ERR_INVALID_ARG;
    RowsParams &p = x.rows;
    const size_t esz = d->dtype == RKV_F32 ? 4 : 2;
    p.q_stride = row_stride(tokens->q_stride, d->n_q_heads, d->head_dim, esz);
    p.out_stride = row_stride(tokens->out_stride, d->n_q_heads, d->head_dim, esz);
    if (!p.q_stride || !p.out_stride) return RKV_ERR_INVALID_ARG;
    if ((rc = check_room(d, x.bytes)) != RKV_OK) return rc;
    if (tokens->total == 0) return RKV_OK;
    p.q = q;
    p.k = k_cache;
    p.v = v_cache;
    p.lens = seq_lens;
    p.out = out;
    p.part = x.wide ? static_cast<float *>(d->workspace) : nullptr;
    char *wide = static_cast<char *>(d->workspace) + x.wide;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = x.single ? launch_attend_more(p, d->dtype, x.tiles, x.separate, 0, false, nullptr, s) : launch_rows(d, p, wide, s);
    if (e == cudaSuccess && p.part) e = launch_rows_merge(p, d->dtype, s);
    return e == cudaSuccess ? RKV_OK : cuda_fail(e, "window attention launch");
}

size_t rkv_prefix_workspace_bytes(const rkv_desc_t *d, int32_t budget, int32_t buffer, const rkv_prefix_t *prefix)
{
    RowsParams shared;
    Plan own;
    return plan_prefix(d, budget, buffer, prefix, &shared, &own) == RKV_OK ? own.bytes : 0;
}

int rkv_prefix_attention(const rkv_desc_t *d, const void *k_cache, const void *v_cache, const void *q_new, const int32_t *seq_lens, void *out,
                         int32_t budget, int32_t buffer, const rkv_prefix_t *prefix, void *stream)
{
    RowsParams shared;
    Plan own;
    int rc = plan_prefix(d, budget, buffer, prefix, &shared, &own);
    if (rc != RKV_OK) return rc;
    if (!k_cache || !v_cache || !q_new || !seq_lens || !out || !prefix->k || !prefix->v || !prefix->lens) return RKV_ERR_INVALID_ARG;
    for (const void *x : {k_cache, v_cache, q_new, (const void *)out, prefix->k, prefix->v})
        if (!aligned16(x)) return RKV_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(seq_lens) | reinterpret_cast<uintptr_t>(prefix->lens)) & 3u) return RKV_ERR_INVALID_ARG;
    if ((rc = check_room(d, own.bytes)) != RKV_OK) return rc;
    shared.k = prefix->k, shared.v = prefix->v, shared.lens = prefix->lens;
    own.rows.k = k_cache, own.rows.v = v_cache, own.rows.lens = seq_lens;
    for (RowsParams *p : {&shared, &own.rows}) {
        p->q = q_new;
        p->out = out;
        p->q_stride = p->out_stride = (long long)d->n_q_heads * d->head_dim;
        p->part = static_cast<float *>(d->workspace);
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    char *wide = static_cast<char *>(d->workspace) + own.wide;
    cudaError_t e = cudaSuccess;
    if (own.joined) {
        e = launch_attend_more(own.rows, d->dtype, own.tiles, own.separate, 0, false, &shared, s);
    } else {
        e = launch_rows(d, shared, wide, s);
        if (e == cudaSuccess)
            e = own.single ? launch_attend_more(own.rows, d->dtype, own.tiles, own.separate, shared.splits, true, nullptr, s)
                           : launch_rows(d, own.rows, wide + wide_bytes(d, shared), s);
    }
    if (e == cudaSuccess && (!own.single || own.separate)) e = launch_rows_merge(own.rows, d->dtype, s);
    return e == cudaSuccess ? RKV_OK : cuda_fail(e, "prefix attention launch");
}

}  // extern "C"
