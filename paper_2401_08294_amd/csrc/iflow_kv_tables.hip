// Page tables and slot maps of the paged key/value cache from the sequences' lengths (include/iflow.h: iflow_kv_tables).
//
// Of sequence b the lengths say how many pages it needs, held[b] how many it has: it takes or gives back the difference.  Exclusive sums over the sequences number all pages taken, all given
// back and all tokens; number k taken is the ring's k-th page, number k given back goes k behind its end.  So every page and every token is found by its number alone, and
// nothing waits for anything but the sums: what is taken lies in front of the ring's end as it was, what is given back behind it, and a token's page is one that its sequence had (in the table as it
// was) or one that it takes (in the ring).
// The work is launches and latencies.  Up to 1024 sequences every workgroup adds up all of them for itself, in LDS, and the rest is shared among the wavefronts of all; more
// sequences, and a larger batch whose state is updated in place (its workgroups would read what one of them has written), take launches of their own for the sums.
// 64 sequences' next tokens 3.5 us, a mixed step of 256 sequences and 30 thousand tokens 4.3 (in place 6.3), a third of a million tokens of 1000 sequences 5.8 (7.9) (graph replay): lengths -> sums -> search -> page -> slot, one after another.
#include <algorithm>

#include "iflow_kv.h"

namespace iflow {

constexpr int KVT_ONE = 1024, KVT_THREADS = 1024, KVT_WAVES = KVT_THREADS / 64;
// Of a wavefront at a time: one of each lane's.  (Four tokens a lane, loads side by side, 4.9 / 6.4 / 6.5 us instead of 3.4 / 4.3 / 5.8 for 64 sequences' next tokens, a mixed step of 256, a third of a million
// tokens of 1000 prompts: longer code, which the first wavefront of every compute unit waits for.)
constexpr int KVT_TOKENS = 64, KVT_PAGES = 64;

// What is known of all sequences: sums of tokens (null: one each), of pages taken and given back, [n_seqs + 1]; pages that they held, their lengths.
struct KvSums {
    const int32_t *tokens, *take, *give, *held, *lens;
    int32_t start, count, n_tokens, n_take, n_give;
};
// work space: {start, count, tokens, taken, given back}, tokens, pages taken and given back of every 1024 sequences, then the sums
struct KvSumsSpace {
    static constexpr int CHUNKS = 64, HEAD = 8 + 3 * CHUNKS;
    int32_t *head, *chunk, *take, *give, *held;
    __device__ __forceinline__ KvSumsSpace(void *ws, int n) : head(static_cast<int32_t *>(ws)), chunk(head + 8), take(head + HEAD), give(take + n + 1), held(give + n + 1) {}
    static size_t bytes(int n) { return ((size_t)(HEAD + 3 * n + 2) * 4 + 15) / 16 * 16; }
};

struct KvWants { int tokens, held, need, len; };
__device__ __forceinline__ KvWants kvt_wants(const KvView &v, const KvTables &t, int b)
{
    KvWants w;
    w.tokens = !v.first ? 1 : max(0, min(t.new_tokens[b], v.max_tokens));
    w.held = max(0, min(t.held[b], v.max_pages - t.n_shared));
    w.len = v.lens[b];
    const int len = max(0, min(w.len, v.max_seq));
    w.need = max(0, v.page_of((len + KV_TILE - 1) / KV_TILE + v.tiles_per_page - 1) - t.n_shared);
    return w;
}
__device__ __forceinline__ int32_t kvt_ring(const KvView &v, int start, int k)      // where the k-th page from `start` on lies; k < n_pages
{
    const uint32_t at = (uint32_t)start + (uint32_t)k, n = (uint32_t)v.n_pages;
    return (int32_t)(at >= n ? at - n : at);
}

// The sums' state of one workgroup that takes 1024 sequences at a time.
struct KvScan {
    int tokens = 0, take = 0, give = 0;                       // before these sequences; in front of the next
    // sums before sequence `threadIdx.x` of these; `shared`: [3][KVT_WAVES], read until the next barrier
    __device__ __forceinline__ void step(const KvWants &w, int32_t (*shared)[KVT_WAVES], int &my_tokens, int &my_take, int &my_give)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int x[3] = {w.tokens, max(0, w.need - w.held), max(0, w.held - w.need)};
        int upto[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            upto[i] = wave_scan(x[i]);
            if (lane == 63) shared[i][wave] = upto[i];
        }
        __syncthreads();
        int *before[3] = {&tokens, &take, &give}, *mine[3] = {&my_tokens, &my_take, &my_give};
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int of_wave = lane < KVT_WAVES ? shared[i][lane] : 0, upto_wave = wave_scan(of_wave);
            *mine[i] = *before[i] + __shfl(upto_wave - of_wave, wave) + upto[i] - x[i];
            *before[i] += __builtin_amdgcn_readlane(upto_wave, 63);
        }
    }
};

__device__ __forceinline__ void kvt_range(const KvView &v, const KvTables &t, int &start, int &count)
{
    const uint32_t n = (uint32_t)v.n_pages, s = (uint32_t)t.free_state[0];
    start = (int)(s < n ? s : s % n);
    count = max(0, (int)min((int64_t)t.free_state[1], v.n_pages));
}
__device__ __forceinline__ void kvt_new_range(const KvView &v, const KvTables &t, const KvSums &s)
{
    const int taken = min(s.n_take, s.count);
    t.free_out[0] = (taken == (int)v.n_pages) ? s.start : kvt_ring(v, s.start, taken);
    t.free_out[1] = (int32_t)min((int64_t)(s.count - taken) + s.n_give, v.n_pages);
    t.free_out[2] = s.n_take - taken;
}

// Everything but the sums, by wavefront `wave` of `waves`: the tokens' slots, pages taken, pages given back, the shared pages.  (Every number is checked against its buffer again: in a launch of
// its own the lengths may be others than the sums were made of, where another stream changes them.)
__device__ __forceinline__ void kvt_fill(const KvView &v, const KvTables &t, const KvSums &s, int wave, int waves)
{
    const int lane = threadIdx.x & 63, n = v.n_seqs, P = v.tiles_per_page * KV_TILE;
    int32_t *table = const_cast<int32_t *>(v.table);
    const int rows = t.slots ? min(s.n_tokens, (int)v.n_tokens) : 0;
    const int token_chunks = (rows + KVT_TOKENS - 1) / KVT_TOKENS, take_chunks = (s.n_take + KVT_PAGES - 1) / KVT_PAGES, give_chunks = (s.n_give + KVT_PAGES - 1) / KVT_PAGES;
    const int per_row = (t.n_shared + KVT_PAGES - 1) / KVT_PAGES;
    const int64_t chunks = (int64_t)token_chunks + take_chunks + give_chunks + (int64_t)per_row * n;
    for (int64_t c = wave; c < chunks; c += waves) {
        if (c < token_chunks) {
            const int r0 = (int)c * KVT_TOKENS, r1 = min(rows, r0 + KVT_TOKENS) - 1, row = min(r0 + lane, r1), b = s.tokens ? kv_last_of(s.tokens, n, r0, r1, row) : row;
            const int p = (int)((uint32_t)s.lens[b] - (s.tokens ? (uint32_t)(s.tokens[b + 1] - row) : 1u));
            int64_t slot = -1;
            if ((uint32_t)p < (uint32_t)v.max_seq) {
                const int page_of = v.page_of(p / KV_TILE), j = page_of - t.n_shared, held = s.held[b];
                // (one load, wherever from: three in branches wait for one another)
                const int taken = s.take[b] + (j - held);
                const int32_t *from = j < 0 ? t.shared + page_of : j < held ? table + ((int64_t)b * v.max_pages + page_of) : taken < s.count ? t.ring + kvt_ring(v, s.start, taken) : nullptr;
                const int page = from ? *from : -1;
                if (page >= 0 && page < v.n_pages) slot = (int64_t)page * P + (p - page_of * P);
            }
            if (r0 + lane <= r1) t.slots[row] = slot;
            continue;
        }
        const int64_t d = c - token_chunks;
        if (d < take_chunks) {
            const int k0 = (int)d * KVT_PAGES, k1 = min(s.n_take, k0 + KVT_PAGES) - 1, k = k0 + lane;
            const int b = kv_last_of(s.take, n, k0, k1, min(k, k1));
            if (k <= k1) {
                const int entry = t.n_shared + s.held[b] + (k - s.take[b]);
                if (entry < v.max_pages) table[(int64_t)b * v.max_pages + entry] = k < s.count ? t.ring[kvt_ring(v, s.start, k)] : -1;
            }
        } else if (d < take_chunks + give_chunks) {
            const int k0 = (int)(d - take_chunks) * KVT_PAGES, k1 = min(s.n_give, k0 + KVT_PAGES) - 1, k = k0 + lane;
            const int b = kv_last_of(s.give, n, k0, k1, min(k, k1));
            if (k <= k1 && (int64_t)s.count + k < v.n_pages) {
                // (the last of the sequence's pages that go is its last)
                const int entry = t.n_shared + s.held[b] - (s.give[b + 1] - k);
                if (entry >= 0 && entry < v.max_pages) t.ring[kvt_ring(v, s.start, s.count + k)] = table[(int64_t)b * v.max_pages + entry];
            }
        } else {
            const int64_t e = d - take_chunks - give_chunks;
            const int b = (int)(e / per_row), j = (int)(e - (int64_t)b * per_row) * KVT_PAGES + lane;
            if (j < t.n_shared && s.lens[b] > 0) table[(int64_t)b * v.max_pages + j] = t.shared[j];
        }
    }
}

// Up to 1024 sequences: every workgroup's own sums; the first writes what is new of the sequences.
__global__ __launch_bounds__(KVT_THREADS) void kv_tables_kernel(KvView v, KvTables t)
{
    __shared__ int32_t s_tokens[KVT_ONE + 1], s_take[KVT_ONE + 1], s_give[KVT_ONE + 1], s_held[KVT_ONE], s_lens[KVT_ONE], s_waves[3][KVT_WAVES];
    const int b = threadIdx.x;
    KvSums s = {v.first ? s_tokens : nullptr, s_take, s_give, s_held, s_lens};
    kvt_range(v, t, s.start, s.count);
    KvWants w = {0, 0, 0, 0};
    if (b < v.n_seqs) w = kvt_wants(v, t, b);
    KvScan scan;
    int tokens, take, give;
    scan.step(w, s_waves, tokens, take, give);
    if (b < v.n_seqs) { s_tokens[b] = tokens; s_take[b] = take; s_give[b] = give; s_held[b] = w.held; s_lens[b] = w.len; }
    if (b == 0) { s_tokens[v.n_seqs] = scan.tokens; s_take[v.n_seqs] = scan.take; s_give[v.n_seqs] = scan.give; }
    s.n_tokens = scan.tokens; s.n_take = scan.take; s.n_give = scan.give;
    __syncthreads();                                          // (also: the lengths and states have been read before any is written)
    if (blockIdx.x == 0) {
        if (b < v.n_seqs) {
            t.held_out[b] = w.held - max(0, w.held - w.need) + max(0, min(s.count - take, w.need - w.held));
            if (v.first) const_cast<int32_t *>(v.first)[b] = tokens;
        }
        if (b == 0) {
            if (v.first) const_cast<int32_t *>(v.first)[v.n_seqs] = scan.tokens;
            kvt_new_range(v, t, s);
        }
    }
    kvt_fill(v, t, s, __builtin_amdgcn_readfirstlane(blockIdx.x * KVT_WAVES + (b >> 6)), gridDim.x * KVT_WAVES);
}

// Any number of sequences, 1024 to a workgroup: what they want together; the sums; then the rest.  (The ring's ends go by way of the work space, or one workgroup has read them: free_out may be free_state.
// Us, 1025, 8000 and 60000 sequences' next tokens 8.8, 12.1, 13.2; the sums by one workgroup, without the first launch, 7.8, 17.2, 72: what one compute unit loads and stores.)
__global__ __launch_bounds__(KVT_THREADS) void kv_tables_totals_kernel(KvView v, KvTables t, void *ws)
{
    __shared__ int32_t s_waves[3][KVT_WAVES];
    const KvSumsSpace to(ws, v.n_seqs);
    const int b = blockIdx.x * KVT_THREADS + threadIdx.x;
    KvWants w = {0, 0, 0, 0};
    if (b < v.n_seqs) w = kvt_wants(v, t, b);
    KvScan scan;
    int tokens, take, give;
    scan.step(w, s_waves, tokens, take, give);
    if (threadIdx.x == 0) { to.chunk[3 * blockIdx.x] = scan.tokens; to.chunk[3 * blockIdx.x + 1] = scan.take; to.chunk[3 * blockIdx.x + 2] = scan.give; }
    if (b == 0) kvt_range(v, t, to.head[0], to.head[1]);
}
__global__ __launch_bounds__(KVT_THREADS) void kv_tables_sums_kernel(KvView v, KvTables t, void *ws)
{
    __shared__ int32_t s_waves[3][KVT_WAVES];
    const KvSumsSpace to(ws, v.n_seqs);
    const int b = blockIdx.x * KVT_THREADS + threadIdx.x, lane = threadIdx.x & 63;
    KvWants w = {0, 0, 0, 0};
    if (b < v.n_seqs) w = kvt_wants(v, t, b);
    KvSums s = {};
    if (gridDim.x > 1) { s.start = to.head[0]; s.count = to.head[1]; }
    else kvt_range(v, t, s.start, s.count);
    KvScan scan;
    auto before = [&](int i) { return __builtin_amdgcn_readlane(wave_scan(lane < (int)blockIdx.x ? to.chunk[3 * lane + i] : 0), 63); };
    if (gridDim.x > 1) { scan.tokens = before(0); scan.take = before(1); scan.give = before(2); }
    int tokens, take, give;
    scan.step(w, s_waves, tokens, take, give);
    if (b < v.n_seqs) {
        if (v.first) const_cast<int32_t *>(v.first)[b] = tokens;
        to.take[b] = take; to.give[b] = give; to.held[b] = w.held;
        t.held_out[b] = w.held - max(0, w.held - w.need) + max(0, min(s.count - take, w.need - w.held));
    }
    if (b == v.n_seqs - 1) {
        s.n_tokens = scan.tokens; s.n_take = scan.take; s.n_give = scan.give;
        if (v.first) const_cast<int32_t *>(v.first)[v.n_seqs] = s.n_tokens;
        to.take[v.n_seqs] = s.n_take; to.give[v.n_seqs] = s.n_give;
        to.head[0] = s.start; to.head[1] = s.count; to.head[2] = s.n_tokens; to.head[3] = s.n_take; to.head[4] = s.n_give;
        kvt_new_range(v, t, s);
    }
}
__global__ __launch_bounds__(256) void kv_tables_fill_kernel(KvView v, KvTables t, void *ws)
{
    const KvSumsSpace from(ws, v.n_seqs);
    const KvSums s = {v.first, from.take, from.give, from.held, v.lens, from.head[0], from.head[1], from.head[2], from.head[3], from.head[4]};
    kvt_fill(v, t, s, __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), gridDim.x * 4);
}

// Chunks of work that the host knows of: tokens, and the pages that these and the shared ones lie in.
static int64_t kvt_chunks(const KvView &v, const KvTables &t)
{
    return (v.n_tokens + KVT_TOKENS - 1) / KVT_TOKENS + (int64_t)v.n_seqs * ((t.n_shared + KVT_PAGES - 1) / KVT_PAGES) + (v.n_tokens / (v.tiles_per_page * KV_TILE) + v.n_seqs) / KVT_PAGES;
}
// Chunks that one workgroup does by itself where more may not (us, in place: 1392 tokens of 64 sequences 4.0, 1901 of 256 5.2, 3753 of 64 5.7; two launches 5.8 to 6.6, 2277 to 6871 tokens).
constexpr int KVT_ALONE = 4 * KVT_WAVES;

size_t kv_tables_workspace_bytes(const KvView &v) { return KvSumsSpace::bytes(v.n_seqs); }

hipError_t launch_kv_tables(const KvView &v, const KvTables &t, void *workspace, hipStream_t s)
{
    const int64_t chunks = kvt_chunks(v, t);
    const bool in_place = t.held == t.held_out || t.free_state == t.free_out;
    if (v.n_seqs <= KVT_ONE && (!in_place || chunks <= KVT_ALONE)) {
        const int64_t groups = in_place ? 1 : std::max<int64_t>(1, std::min<int64_t>(256, (chunks + KVT_WAVES - 1) / KVT_WAVES));
        hipLaunchKernelGGL(kv_tables_kernel, dim3((unsigned)groups), dim3(KVT_THREADS), 0, s, v, t);
        return hipGetLastError();
    }
    const dim3 thousands((unsigned)((v.n_seqs + KVT_THREADS - 1) / KVT_THREADS));
    hipError_t e = hipSuccess;
    if (thousands.x > 1) {
        hipLaunchKernelGGL(kv_tables_totals_kernel, thousands, dim3(KVT_THREADS), 0, s, v, t, workspace);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kv_tables_sums_kernel, thousands, dim3(KVT_THREADS), 0, s, v, t, workspace);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kv_tables_fill_kernel, dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(2048, (chunks + 3) / 4))), dim3(256), 0, s, v, t, workspace);
    return hipGetLastError();
}

}  // namespace iflow
