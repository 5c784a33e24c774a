// Causal attention over the quantized key/value cache: a token sees every position up to its own (the kernels: iflow_kv_attn.h).
#include "iflow_kv_attn.h"

namespace iflow {

size_t kv_attn_workspace_bytes(const KvView &v, int head_dim, int n_heads)
{
    const KvPlan plan(v, head_dim, n_heads, v.max_seq);
    return plan.sixteens && !plan.direct ? KvPartial::bytes(v.n_seqs, head_dim) : 0;
}

hipError_t launch_kv_attn(int format, int head_dim, const KvView &v, const uint16_t *q, int n_heads, float scale, uint16_t *out, void *workspace, hipStream_t s)
{
    return kv_attn_launches(format, head_dim, v, q, n_heads, scale, out, workspace, s, v.max_seq, KvPlan(v, head_dim, n_heads, v.max_seq), KvSeesAll{});
}

hipError_t launch_kv_attn_blocks(int format, int head_dim, const KvView &v, const uint16_t *q, int n_heads, float scale, uint16_t *out, int rows, int few, hipStream_t s)
{
    const int group = n_heads / v.n_kv_heads;
    const int64_t all = v.n_tokens * group, blocks = all / rows + std::min<int64_t>(v.n_seqs, all / few);
    return kv_attn_by_blocks(format, head_dim, v, q, n_heads, scale * 1.4426950408889634f, out, s, rows, few, kv_numbered(blocks * v.n_kv_heads), KvSeesAll{});
}

}  // namespace iflow
