// Attention over the quantized key/value cache with a sliding window and a few first positions that stay visible: the kernels of iflow_kv_attn.h over the tiles that a workgroup's tokens see, the first
// ones and those from the first token's window on, as one list; what of a tile a row does not see is hidden where its scores are made.
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

size_t kv_attn_window_workspace_bytes(const KvView &v, int head_dim, int n_heads, int window, int sinks)
{
    if (kv_window_is_all(v, window, sinks)) return kv_attn_workspace_bytes(v, head_dim, n_heads);
    const KvPlan plan(v, head_dim, n_heads, kv_window_seen(v, n_heads, window, sinks));
    return plan.sixteens && !plan.direct ? KvPartial::bytes(v.n_seqs, head_dim) : 0;
}

hipError_t launch_kv_attn_window(int format, int head_dim, const KvView &v, const uint16_t *q, int n_heads, int window, int sinks, float scale, uint16_t *out, void *workspace, hipStream_t s)
{
    if (kv_window_is_all(v, window, sinks)) return launch_kv_attn(format, head_dim, v, q, n_heads, scale, out, workspace, s);
    return kv_attn_launches(format, head_dim, v, q, n_heads, scale, out, workspace, s, kv_window_seen(v, n_heads, window, sinks), KvSeesWindow{window, sinks});
}

}  // namespace iflow
