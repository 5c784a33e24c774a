// Attention over the quantized key/value cache for a batch whose sequences share a prefix: the prefix's positions once, for the rows of all tokens (by blocks of rows, a part of the
// positions each), what every sequence has behind them by itself, and the sum of both (the kernels: iflow_kv_attn.h).
#include "iflow_kv_attn.h"

namespace iflow {

// How a call is served.  Sequences of `few` rows and more fill blocks of their own, which decode a tile for as many rows as the prefix's would: they go as in causal attention.
struct KvSharedPlan {
    bool alone;                                               // not worth it: causal attention
    int big, rows, parts;                                     // rows of a block: of a sequence of `few` rows and more (0: there are none), of the prefix; parts of the prefix's positions
    int64_t blocks;                                           // of the prefix's rows
    KvPlan tail;                                              // of what lies behind the prefix
    KvSharedPlan(const KvView &v, int head_dim, int n_heads, int max_shared) : tail(v, head_dim, n_heads, v.max_seq)
    {
        const int64_t group = n_heads / v.n_kv_heads, most = v.max_tokens * group, all = v.n_tokens * group, seqs = v.n_seqs, kv = v.n_kv_heads, tiles = max_shared / KV_TILE;
        alone = seqs < 2 || all > (1 << 21) || max_shared < KV_TILE * v.tiles_per_page;
        big = most < KVA_FEW || kv * (all / 64) < 256 ? 0 : kv * (all / 128) >= 512 ? 128 : 64;
        rows = 64;
        blocks = (all + rows - 1) / rows;
        parts = (int)std::max<int64_t>(1, std::min<int64_t>(KVA_CUS / std::max<int64_t>(1, blocks * kv), (tiles + 15) / 16));
        // the rest by sixteens
        tail.rows = 0;
        tail.sixteens = true;
        tail.few = big ? KVA_FEW : 0;
        tail.packed = seqs > 1 && 2 * v.n_tokens < seqs * v.max_tokens;
        tail.lines = seqs * kv * (((big ? std::min<int64_t>(most, KVA_FEW - 1) : most) + KVA_ROWS - 1) / KVA_ROWS);
        if (tail.packed) tail.lines = std::min(tail.lines, kv * (all / KVA_ROWS + seqs));
        const int64_t seen = std::max<int64_t>(1, v.max_seq - max_shared);
        tail.direct = head_dim == 64 || tail.lines < 256 ? 8 : 4;
        if (tail.lines * ((v.max_seq + KV_TILE - 1) / KV_TILE) <= (1LL << 30) && seen > (tail.lines >= 256 ? 2560 : head_dim == 64 ? 1024 : 768)) tail.direct = 0;
    }
    size_t prefix_bytes(int64_t n_rows, int head_dim) const { return (size_t)parts * n_rows * (head_dim + 2) * 4 + 32; }      // (the values behind the others, 16-byte aligned)
};

size_t kv_attn_shared_workspace_bytes(const KvView &v, int head_dim, int n_heads, int max_shared)
{
    const KvSharedPlan plan(v, head_dim, n_heads, max_shared);
    if (plan.alone) return kv_attn_workspace_bytes(v, head_dim, n_heads);
    return (plan.prefix_bytes(v.n_tokens * n_heads, head_dim) + 15) / 16 * 16 + (plan.tail.direct ? 0 : KvPartial::bytes(v.n_seqs, head_dim));
}

hipError_t launch_kv_attn_shared(int format, int head_dim, const KvView &v, const int32_t *pages, const int32_t *len, int max_shared, const uint16_t *q, int n_heads, float scale, uint16_t *out,
                                 void *workspace, hipStream_t s)
{
    const KvSharedPlan plan(v, head_dim, n_heads, max_shared);
    if (plan.alone) return launch_kv_attn(format, head_dim, v, q, n_heads, scale, out, workspace, s);
    const int group = n_heads / v.n_kv_heads;
    const float scale_log2e = scale * 1.4426950408889634f;
    const KvDivide by_group(group);
    const int64_t n_rows = v.n_tokens * n_heads;
    float *const m = static_cast<float *>(workspace), *const l = m + plan.parts * n_rows, *const o = m + (2 * plan.parts * n_rows + 3) / 4 * 4;
    const KvShared shared = {pages, len, m, l, o, n_rows, max_shared, plan.parts};
    if (plan.big) {
        const hipError_t e = launch_kv_attn_blocks(format, head_dim, v, q, n_heads, scale, out, plan.big, KVA_FEW, s);
        if (e != hipSuccess) return e;
    }
    const hipError_t e = for_kv_tile(format, head_dim, [&](auto tag) {
        typedef decltype(tag) T;
        const KvSeesPrefix sees = {shared, plan.big ? KVA_FEW : 0x7fffffff};
        hipLaunchKernelGGL((kv_attn_rows_kernel<T, 2, 4, 1, KvSeesPrefix>), dim3((unsigned)v.n_kv_heads, (unsigned)plan.blocks, (unsigned)plan.parts), dim3(512), 0, s, v, q, n_heads, group, 0, by_group,
                           scale_log2e, out, sees);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    uint8_t *const rest = static_cast<uint8_t *>(workspace) + (plan.prefix_bytes(n_rows, head_dim) + 15) / 16 * 16;
    return kv_attn_by_sixteens(format, head_dim, v, q, n_heads, scale_log2e, out, rest, s, plan.tail, std::max<int64_t>(1, v.max_seq - max_shared), KvSeesTail{shared, head_dim, 0});
}

}  // namespace iflow
