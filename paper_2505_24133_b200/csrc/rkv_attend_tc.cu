// Decode-step attention on the tensor cores (rkv_attend_tc.cuh): rkv_decode_attention's instances, and how many blocks share a head.
#include "rkv_attend_tc.cuh"

namespace rkv {
// Splits of a head's key tiles (blocks of a cluster) for the tensor-core kernel: at most 28 tiles per block, and among those the number
// with the shortest run: waves of resident blocks (2 per SM) times what a block spends, its tiles and about three tiles' worth of
// set-up and merge, and one and a half more for a second chunk.  (128 heads of 33 tiles: 4 splits, two waves of 9 tiles, 49 us; 5, the
// fewest that give two waves of blocks, 54.  With two tiles' worth 600 heads of 15 tiles were cut in three, 98 us and 114 for 8-bit
// caches, 93 and 97 uncut; 512 heads of 33 tiles in four, 167 and 192, 163 and 172 in three.  Two chunks, where one block of 16 to 28
// tiles takes the place of two: 200 heads of 16 tiles 49.7 us with two splits, 39.0; 512 of 16 99.7, 84.1; 296 of 20 70.4, 63.7; 148 of
// 33 60.7, 54.7; 8-bit 296 of 17 52.2, 42.9; where the rule keeps one chunk nothing moved.)  The fewest splits of one chunk where
// they give four waves: a part of the last one counts for little then (256 heads of 64 tiles: 159 us with 5 splits, 165 with 8).
int attend_tc_splits(int heads, int cap, int sms)
{
    const int tiles = (cap + kTile - 1) / kTile, least = (tiles + kTcMaxTiles - 1) / kTcMaxTiles;
    if ((long long)heads * least >= 8ll * sms) return least;
    int best = 0;
    long long best_cost = 0;
    for (int s = (tiles + 2 * kTcChunkTiles - 1) / (2 * kTcChunkTiles); s <= tiles && s <= kTcMaxSplits; ++s) {
        const int per = (tiles + s - 1) / s;
        if (s > 1 && (tiles + per - 1) / per < s) continue;          // the last blocks would have no tile
        const long long waves = ((long long)heads * s + 2 * sms - 1) / (2 * sms);
        const long long cost = waves * (2 * (per + 3) + (per > kTcMaxTiles ? 3 : 0));
        if (best == 0 || cost < best_cost) best = s, best_cost = cost;
    }
    return best;
}

// Splits that the size of the workspace is counted by: the fewest that give two waves of resident blocks.  The clusters need none
// of it; the size has always been this, and callers that needed no workspace still need none.
int attend_tc_workspace_splits(int heads, int cap, int sms)
{
    const int tiles = (cap + kTile - 1) / kTile;
    int splits = (4 * sms + heads - 1) / heads;
    const int least = (tiles + kTcMaxTiles - 1) / kTcMaxTiles;
    splits = splits < least ? least : splits;
    return splits > tiles ? tiles : splits;
}

// The splits are blocks of their own: more than two waves of them, of a kind that clusters slow down, and the workspace holds their
// partial results.  (Up to two waves clusters are the faster, by 10-30 % below one; from there on blocks are, by 1 to 17 %.)
bool attend_tc_separate(int heads, int cap, int splits, int sms, int src)
{
    return splits > 1 && src != 0 && (long long)heads * splits > 4ll * sms && splits <= attend_tc_workspace_splits(heads, cap, sms);
}

cudaError_t launch_attend_tc(const void *k_cache, const void *v_cache, const void *q_new, const int32_t *seq_lens, float *out,
                             float *partial, int batch, int hkv, int hq, int cap, int splits, int32_t *status, long long wait_cycles,
                             const int32_t *block_table, long long pool_pages, int src, cudaStream_t s)
{
    const int tiles = (cap + kTile - 1) / kTile;
    AttendTcParams p;
    p.seq_lens = seq_lens;
    p.out = partial ? partial : out;
    p.separate = partial ? 1 : 0;
    p.hkv = hkv;
    p.hq = hq;
    p.cap = cap;
    p.splits = splits;
    p.tiles_per_split = (tiles + splits - 1) / splits;
    p.status = status;
    p.wait_cycles = wait_cycles;
    p.block_table = block_table;
    if (p.tiles_per_split > 2 * kTcChunkTiles) return cudaErrorInvalidValue;
    return launch_tc_group(p, AttendTcMaps(), k_cache, v_cache, q_new, batch, pool_pages, src, s);
}

}  // namespace rkv
