// Attention over the quantized key/value cache for a batch whose sequences share a prefix: the prefix's positions once, for the rows of all tokens (by blocks of rows, a part of the
// positions each), what every sequence has behind them by itself, and the sum of both (the kernels: iflow_kv_attn.h):
//   out = sum_i O_i 2^(m_i - m) / sum_i l_i 2^(m_i - m)      over the prefix's parts and the rest, m the largest reference m_i.
// 64 sequences behind 4096 positions, up to 905 of their own, 32/8 heads x 128, 4 bits: 31 us, of which the prefix 16 (4.3 GFLOP; two steps of 64 positions to a wavefront, and what it takes to begin and to merge) and the
// rest 16 (37 MB of codes, unpacked for 4 rows of 16); each sequence by itself 62.
#include "iflow_kv_attn.h"

namespace iflow {

// How a call is served.  Sequences of `few` rows and more fill blocks of their own, which decode a tile for as many rows as the prefix's would: they go as in causal attention.
// The prefix's blocks have 64 rows, whose positions four groups of wavefronts share (us of the call, for it / 128 rows in two groups / 128 rows, pipelined / 64 rows in two groups; 32/8 heads x 128, 4 bits, 64
// sequences, 1024 positions 18.9 / 21.4 / 20.9 / 20.8, 4096 23.8 / 25.6 / 26.5 / 28.6, 16000 46.3 / 45.8 / 49.9 / 53.8; 16 sequences of 32/32 heads, 4096 21.2 / 26.1 / 25.7 / 24.1), and parts of its
// positions as many as fill the device, of eight tiles at least (a step of all four groups).
// `alone`: causal attention, where the second launch and the sum cost more than sharing saves.  A line of sixteen rows takes about 0.8 ns of the device for a tile, a block of 64 rows 1.9.  Us, shared / alone,
// by lines less 1.3 for each block, times tiles of the prefix (of 64 components two thirds of that):
//   32/8 heads x 128, 4 bits   seqs 4: 6700 20.8 / 18.8, 10800 22.7 / 23.2   8: 5000 16.7 / 15.7, 13400 19.6 / 22.8   16: 5400 16.9 / 15.9, 14500 18.5 / 22.6   32: 8900 17.9 / 14.8, 14600 18.6 / 20.3
//                              seqs 64: 8500 19.6 / 14.4, 14100 19.9 / 19.2, 23500 20.8 / 26.7
//   32/8 heads x 128, 8 bits   seqs 8: 8400 19.2 / 18.8, 13400 21.0 / 23.3   16: 9100 19.0 / 18.8, 14500 19.9 / 22.9   64: 14100 21.6 / 19.7, 23500 22.5 / 27.1
//   32/32 x 128, 4 bits        seqs 2: 8900 27.2 / 22.9   4: 6700 17.6 / 17.7, 10700 19.4 / 22.3   8: 8100 16.1 / 14.4, 13300 16.7 / 20.2   16: 14100 17.9 / 19.0   64, of 6 pages: 24000 32.0 / 33.4, of 3: 12000 32 / 26
//   64/8 x 64, 4 bits          seqs 8: 6600 15.9 / 17.1, 11100 18.5 / 20.9   16: 6600 15.0 / 16.5, 11100 16.5 / 20.4   32: 6600 14.1 / 11.3, 11100 16.0 / 20.6   64: 10900 17.3 / 15.2, 17700 18.5 / 20.6
//   64 sequences of 4000 positions behind 2048: 30000 60 / 68; eight of 8000 behind 8000: 13400 35 / 30 (where what is behind is cut, its merge comes on top)
struct KvSharedPlan {
    static constexpr int ROWS = 64, PART = 8, LEAST = 9000, LEAST_CUT = 18000;
    bool alone;
    int big;                                                  // rows of a block of a sequence of `few` rows and more (0: there are none)
    int parts, per;                                           // of the prefix's positions, tiles of one
    int64_t blocks;                                           // of the prefix's rows, at most
    int64_t sharing;                                          // tokens that share, at most: with big sequences beside them, those of fewer rows than `few`
    KvPlan tail;                                              // of what lies behind the prefix
    KvSharedPlan(const KvView &v, int head_dim, int n_heads, int max_shared) : tail(v, head_dim, n_heads, v.max_seq)
    {
        const int64_t group = n_heads / v.n_kv_heads, most = v.max_tokens * group, all = v.n_tokens * group, seqs = v.n_seqs, kv = v.n_kv_heads, tiles = max_shared / KV_TILE;
        auto pieces = [](int64_t n) { return (n + KVA_ROWS - 1) / KVA_ROWS; };
        big = most < KVA_FEW || kv * (all / 64) < 256 ? 0 : kv * (all / 128) >= 512 ? 128 : 64;
        sharing = big ? std::min(v.n_tokens, seqs * ((KVA_FEW - 1) / group)) : v.n_tokens;
        blocks = ((big ? std::min(all, seqs * (KVA_FEW - 1)) : all) + ROWS - 1) / ROWS;
        parts = (int)std::max<int64_t>(1, std::min<int64_t>(KVA_CUS / (blocks * kv), (tiles + PART - 1) / PART));
        per = (int)(((tiles + parts - 1) / parts + 1) / 2 * 2);
        // the rest by sixteens
        tail.rows = 0;
        tail.sixteens = true;
        tail.few = big ? KVA_FEW : 0;
        tail.packed = seqs > 1 && 2 * v.n_tokens < seqs * v.max_tokens;
        tail.lines = seqs * kv * pieces(big ? std::min<int64_t>(most, KVA_FEW - 1) : most);
        if (tail.packed) tail.lines = std::min(tail.lines, kv * (all / KVA_ROWS + seqs));
        const int64_t behind = std::max<int64_t>(1, v.max_seq - max_shared);
        tail.direct = head_dim == 64 || tail.lines <= 256 ? 8 : 4;
        if (tail.lines * ((v.max_seq + KV_TILE - 1) / KV_TILE) <= (1LL << 30) && behind > (tail.lines >= 256 ? 2560 : head_dim == 64 ? 1024 : 768)) tail.direct = 0;
        // (of the sequences beside big ones one token each is expected; where that is the most, and `few` rows, nobody is left to share)
        const int64_t lines = big ? seqs * kv * pieces(group) : tail.lines, together = big ? (seqs * group + ROWS - 1) / ROWS : blocks;
        const int64_t saved = (10 * lines - 13 * together * kv) * tiles * (head_dim + 64) / (10 * 192);
        alone = seqs < 2 || (big && most == group) || all > (1 << 21) || v.n_tokens * n_heads > (1 << 22) || tiles < 2 * PART || saved < (tail.direct ? LEAST : LEAST_CUT);
    }
    size_t prefix_bytes(int64_t n_rows, int head_dim) const { return ((size_t)parts * n_rows * (head_dim + 2) * 4 + 32 + 15) / 16 * 16; }      // (the values behind the others, 16-byte aligned)
    static size_t served_bytes(int64_t n_tokens) { return (n_tokens * sizeof(KvServed) + 15) / 16 * 16; }
};

// Rows of the call's tokens that no sequence has yet.  (Where sequences of `few` rows and more are served otherwise the prefix's blocks write only the others', and find those that there are rows for: first
// tokens that go back may claim more.)
__global__ __launch_bounds__(256) void kv_served_none_kernel(KvServed *__restrict__ served, int64_t n)
{
    for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) served[i] = {-1, -1};
}

// Positions of a prefix's whole pages.  The kernels ask for its pages before they know its length: what bounds them is how many entries the array has.
static int kv_whole_pages(const KvView &v, int positions)
{
    const int page = v.tiles_per_page * KV_TILE;
    return positions / page * page;
}

size_t kv_attn_shared_workspace_bytes(const KvView &v, int head_dim, int n_heads, int most)
{
    const int max_shared = kv_whole_pages(v, most);
    const KvSharedPlan plan(kv_rows_bound(v), head_dim, n_heads, max_shared);
    if (plan.alone) return kv_attn_workspace_bytes(v, head_dim, n_heads);
    return plan.prefix_bytes(plan.sharing * n_heads, head_dim) + plan.served_bytes(v.n_tokens) + (plan.tail.direct ? 0 : KvPartial::bytes(v.n_seqs, head_dim));
}

hipError_t launch_kv_attn_shared(int format, int head_dim, const KvView &batch, const int32_t *pages, const int32_t *len, int most, const uint16_t *q, int n_heads, float scale, uint16_t *out,
                                 void *workspace, hipStream_t s)
{
    const KvView v = kv_rows_bound(batch);
    const int max_shared = kv_whole_pages(v, most);
    const KvSharedPlan plan(v, head_dim, n_heads, max_shared);
    if (plan.alone) return launch_kv_attn(format, head_dim, batch, q, n_heads, scale, out, workspace, s);
    const int group = n_heads / v.n_kv_heads;
    const float scale_log2e = scale * 1.4426950408889634f;
    const KvDivide by_group(group);
    const int64_t n_rows = plan.sharing * n_heads;
    float *const m = static_cast<float *>(workspace), *const l = m + plan.parts * n_rows, *const o = m + (2 * plan.parts * n_rows + 3) / 4 * 4;
    uint8_t *const behind = static_cast<uint8_t *>(workspace) + plan.prefix_bytes(n_rows, head_dim);
    const KvShared shared = {pages, len, m, l, o, reinterpret_cast<KvServed *>(behind), n_rows, max_shared, plan.parts};
    if (plan.big) {
        hipLaunchKernelGGL(kv_served_none_kernel, dim3((unsigned)std::min<int64_t>(1024, (v.n_tokens + 255) / 256)), dim3(256), 0, s, shared.served, v.n_tokens);
        const hipError_t e = launch_kv_attn_blocks(format, head_dim, v, q, n_heads, scale, out, plan.big, KVA_FEW, s);
        if (e != hipSuccess) return e;
    }
    const hipError_t e = for_kv_tile(format, head_dim, [&](auto tag) {
        typedef decltype(tag) T;
        const KvSeesPrefix sees = {shared, plan.big ? KVA_FEW : KVA_ALL, plan.per};
        hipLaunchKernelGGL((kv_attn_rows_kernel<T, 2, 4, 1, KvSeesPrefix>), dim3((unsigned)v.n_kv_heads, (unsigned)plan.blocks, (unsigned)plan.parts), dim3(512), 0, s, v, q, n_heads, group, 0, by_group,
                           scale_log2e, out, sees);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    return kv_attn_by_sixteens(format, head_dim, v, q, n_heads, scale_log2e, out, behind + plan.served_bytes(v.n_tokens), s, plan.tail, std::max<int64_t>(1, v.max_seq - max_shared), KvSeesTail{shared, head_dim, 0});
}

}  // namespace iflow
