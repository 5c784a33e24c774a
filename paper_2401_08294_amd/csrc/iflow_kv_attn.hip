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
    return kv_attn_launches(format, head_dim, v, q, n_heads, scale, out, workspace, s, v.max_seq, KvSeesAll{});
}

}  // namespace iflow
