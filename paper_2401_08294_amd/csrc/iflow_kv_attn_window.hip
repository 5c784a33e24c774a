// Attention over the quantized key/value cache with a sliding window and a few first positions that stay visible: the kernels of iflow_kv_attn.h over the tiles that a workgroup's tokens see, the first
// ones and those from the first token's window on, as one list; what of a tile a row does not see is hidden where its scores are made.
// 32 sequences' next tokens, window 1024, 32/8 heads x 128, 4 bits: 11.0 us, 3.5 TB/s of codes; three prompts of up to 4001 tokens, window 512, 64/8 heads: 228, 0.5 PFLOP/s (vector issue and matrix cores in turn).
#include "iflow_kv_attn.h"

namespace iflow {

// positions that a token sees, and with it the others of its sixteen rows, in whole tiles: at most (KvSeesWindow::line_tiles)
static int64_t kv_window_seen(const KvView &v, int n_heads, int window, int sinks)
{
    const int64_t group = n_heads / v.n_kv_heads, n = window + (15 + group - 1) / group, tiles = (sinks + KV_TILE - 1) / KV_TILE + (n + KV_TILE - 2) / KV_TILE + 1;
    return std::min<int64_t>(v.max_seq, tiles * KV_TILE);
}
// a window, or first positions, that no sequence is longer than: causal attention
static bool kv_window_is_all(const KvView &v, int window, int sinks) { return window >= v.max_seq || sinks >= v.max_seq; }

// Blocks of rows, or sixteens: a window's tiles are few, and what a block of rows takes to begin and end counts for more than in causal attention; sixteens leave no row of a single head's tokens empty.  By
// the rows that there are (padded, a batch of a long prompt and short ones would seem to be many).  Us, by sixteens / 64 rows / 128 rows, windows of 64, 512 and 2048:
//   32/8 heads x 128, 4 bits    128 blocks of 64 rows: 7 / 13 / 16, 13 / 18 / 27, 25 / 29 / 48    296: 14 / 31 / 22, 25 / 44 / 36, 42 / 46 / 57    504: 17 / 26 / 17, 37 / 37 / 30, 90 / 73 / 69
//                               1064: 37 / 58 / 36, 75 / 85 / 63, 176 / 147 / 111                 2000: 58 / 96 / 43, 129 / 136 / 82, 348 / 285 / 218
//   64/8 x 64, 4 bits           256: 10 / 11 / 13, 16 / 14 / 23, 27 / 20 / 41    576: 21 / 30 / 21, 32 / 42 / 36, 47 / 49 / 48    1000: 32 / 35 / 17, 51 / 49 / 32, 112 / 89 / 72    4000: 123 / 132 / 57, 192 / 181 / 109, 431 / 360 / 276
//   32/32 x 128, 8 bits         352: 15 / 22 / 37, 27 / 32 / 56, 45 / 46 / 89    512: 21 / 27 / 35, 39 / 41 / 52, 102 / 85 / 110    1088: 42 / 65 / 58, 78 / 92 / 93, 193 / 173 / 141    2208: 78 / 115 / 82, 147 / 171 / 139, 417 / 337 / 278
// A line of sixteen rows is a workgroup's of eight or four wavefronts, or cut: a window's lines are all as long as one another, and one for every compute unit leaves nothing to even out.  Us, cut / four / eight,
// windows of 256, 1024, 1536 and 4000:
//   128 components, 4 bits    8 lines: 9.0 / 6.9 / 6.1, 9.9 / 12.0 / 10.0, 9.9 / 15.6 / 12.7, 10.4 / 31.7 / 26.3     64: 9.5 / 7.3 / 6.6, 11.8 / 12.3 / 10.7, 12.5 / 16.1 / 13.6, 17.7 / 32.4 / 26.7
//                             128: 11.1 / 7.4 / 7.3, 14.7 / 12.7 / 11.2, 16.9 / 16.0 / 13.8, 25.7 / 33.2 / 27.9      256: 13.2 / 7.6 / 7.1, 18.3 / 13.4 / 12.0, 22.1 / 18.7 / 15.1, 38.9 / 39.8 / 31.5
//                             384: 16.3 / 9.5 / 11.3, 22.9 / 18.2 / 20.0, 28.4 / 24.8 / 25.9                         1024: 22.3 / 14.8 / 21.3, 40.3 / 34.6 / 40.7
//   ... 8 bits                128: 11.3 / 7.6 / 7.3, 15.7 / 13.0 / 12.0, 18.6 / 18.6 / 16.3, 37.0 / 38.3 / 31.1      256: 13.8 / 8.1 / 7.6, 20.7 / 14.8 / 15.4, 27.6 / 20.7 / 20.4, 59.3 / 46.7 / 48.4
//   64 components, 4 bits     64: 8.8 / 6.6 / 6.0, 10.5 / 10.4 / 8.8, 11.0 / 13.2 / 10.9, 15.3 / 25.4 / 19.8         512: 16.2 / 8.4 / 8.2, 21.9 / 14.7 / 13.7, 26.0 / 20.3 / 17.6    1024: 18.1 / 10.8 / 14.0, 28.2 / 22.6 / 24.3
static KvPlan kv_window_plan(const KvView &v, int head_dim, int n_heads, int window, int sinks)
{
    const int64_t seen = kv_window_seen(v, n_heads, window, sinks), rows = v.n_tokens * n_heads;          // (of all key/value heads)
    const bool bits8 = v.page_bytes > (int64_t)v.n_kv_heads * v.tiles_per_page * 50 * head_dim, wide = seen > 1280;
    const int64_t fills = !bits8 ? 240 : wide ? 500 : 900;
    KvPlan plan(v, head_dim, n_heads, seen, rows / 128 >= fills ? 128 : wide && rows / 64 >= (head_dim == 64 ? 256 : 450) ? 64 : 0);
    // (lines that there are, not padded to the most tokens; three sequences of 60, 27 and 27 tokens, 32/8 heads, window 6000: 252 of 360, 71 -> 50 us)
    const int64_t lines = std::min(plan.lines, v.n_kv_heads * (v.n_tokens * (n_heads / v.n_kv_heads) / KVA_ROWS + v.n_seqs));
    plan.direct = lines <= (head_dim == 64 ? 512 : 256) ? 8 : 4;
    // (beyond 2^30 there are more tiles than the cut counts in 32 bits)
    if (plan.lines * ((seen + KV_TILE - 1) / KV_TILE) <= (1LL << 30) && lines < 256 && seen > (lines > 64 ? 4000 : head_dim == 64 && lines > 32 ? 2000 : 1250)) plan.direct = 0;
    return plan;
}

size_t kv_attn_window_workspace_bytes(const KvView &v, int head_dim, int n_heads, int window, int sinks)
{
    if (kv_window_is_all(v, window, sinks)) return kv_attn_workspace_bytes(v, head_dim, n_heads);
    const KvPlan plan = kv_window_plan(kv_rows_bound(v), head_dim, n_heads, window, sinks);
    return plan.sixteens && !plan.direct ? KvPartial::bytes(v.n_seqs, head_dim) : 0;
}

hipError_t launch_kv_attn_window(int format, int head_dim, const KvView &batch, const uint16_t *q, int n_heads, int window, int sinks, float scale, uint16_t *out, void *workspace, hipStream_t s)
{
    if (kv_window_is_all(batch, window, sinks)) return launch_kv_attn(format, head_dim, batch, q, n_heads, scale, out, workspace, s);
    const KvView v = kv_rows_bound(batch);
    return kv_attn_launches(format, head_dim, v, q, n_heads, scale, out, workspace, s, kv_window_seen(v, n_heads, window, sinks), kv_window_plan(v, head_dim, n_heads, window, sinks), KvSeesWindow{window, sinks});
}

}  // namespace iflow
