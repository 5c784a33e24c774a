// Attention over the quantized key/value cache: every query token of a batch attends to the positions of its own sequence up to its own
// (layout: include/iflow.h).
//
// Queries of one key/value head are rows: row r of a sequence is token r / group, query head r % group of the group, so that a draft of four tokens with four
// heads fills the sixteen columns of a matrix instruction as a group of sixteen heads does.  Of a tile of 32 positions
//   S[position][row]  = sum_c K[position][c] Q[row][c]
//   O[row][component] = sum_position P[row][position] V[position][component]
// v_mfma_f32_16x16x32_f16 does the first in D / 16 instructions and the second in D / 8, with the probabilities as two fp16 numbers each.  Operand layouts, lane =
// i + 16 g: A: lane holds A[i][8g..8g+7]; B: lane holds B[8g..8g+7][i]; C/D: lane holds D[4g..4g+3][i].  The cache is laid out for exactly these:
//   - Keys are the A operand: lane (i, g) has a quarter of position i's components (and of i + 16's) as one run of its 16-byte loads; which components
//     share an instruction does not matter as long as the queries agree.
//   - The scores' D layout, positions 4g .. 4g+3 of both halves for row i, is P^T's A operand layout of the second product when its positions are taken in that order.
//   - Values are the B operand: lane (i, g) has components i, 16 + i, .. of just these eight positions, eight codes to a run's 32 (64) bits.
// So codes come in with 1 KB per load instruction and become operands in registers: nothing crosses lanes or LDS.
#include "iflow_kv.h"

namespace iflow {

constexpr int KVA_WAVES = 4;
constexpr int KVA_ROWS = 16;                                  // rows of a workgroup
constexpr int KVA_MAX_SPLITS = 128;                           // ranges a sequence is split into
constexpr int KVA_MAX_CHUNK = 64 * KVA_WAVES * KV_TILE;       // positions of a range: a wavefront's tiles have their pages in its 64 lanes
constexpr float KVA_BELOW = 7.f, KVA_LAG = 15.f, KVA_SPARE = 16.f;       // in units of log2: see attn_decode_mfma_kernel

// the maximum over the four lanes i, i + 16, i + 32, i + 48
__device__ __forceinline__ float kva_max_of_rows(float x)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    x = fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}

// where the partial results of the ranges lie: O [output row][range][D], then M [output row][range], then L
struct KvPartial {
    float *o, *m, *l;
    int splits;
    __device__ __host__ KvPartial(float *ws, int64_t rows, int splits_, int d) : o(ws), m(ws + rows * splits_ * d), l(m + rows * splits_), splits(splits_) {}
};

// A tile as it is loaded: a lane's runs, and the headers of its positions.
template <typename T>
struct KvTileRegs {
    kv_u32x4 k[T::PIECES], v[T::PIECES];
    uint32_t kh[2];                                           // (scale, offset) of position i, of 16 + i, in the block of the lane's quarter
    kv_u32x4 vh[T::NB][2];                                    // scales, offsets of its eight positions, by block
};

template <typename T>
__global__ __launch_bounds__(64 * KVA_WAVES) void kv_attn_kernel(KvView v, const uint16_t *__restrict__ q, int n_heads, int group, float scale_log2e, int chunk, int nsplit,
                                                                 int pieces, uint16_t *__restrict__ out, float *__restrict__ ws)
{
    constexpr int D = T::D, NU = D / 32, NC = D / 16;
    __shared__ float s_o[KVA_WAVES][KVA_ROWS][D];
    __shared__ float s_m[KVA_WAVES][KVA_ROWS], s_l[KVA_WAVES][KVA_ROWS];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int li = lane & 15, g = lane >> 4;
    // workgroup -> (sequence, key/value head, range, piece of rows)
    int at = blockIdx.x;
    const int piece = at % pieces; at /= pieces;
    const int sp = at % nsplit; at /= nsplit;
    const int head = at % v.n_kv_heads, b = at / v.n_kv_heads;
    const KvSequence seq(v, b);
    const int r0 = piece * KVA_ROWS, rows = min(KVA_ROWS, seq.count * group - r0);
    if (rows <= 0) return;
    const int longest = seq.sees((r0 + rows - 1) / group);    // the last row sees most
    const int t_begin = sp * chunk;
    if (t_begin >= longest && sp > 0) return;
    const int t_end = min(longest, t_begin + chunk);
    const int mine = longest > chunk ? (longest + chunk - 1) / chunk : 1;      // ranges that this piece's rows have

    const int my_row = r0 + min(li, rows - 1), token = my_row / group;
    const int64_t my_out = (seq.row + token) * n_heads + head * group + (my_row - token * group);
    const bool real = li < rows && seq.has_row(token);
    const int limit = seq.sees(token);
    // queries as B operands: lane (row li, g) holds components g D/4 + 8u .. +8
    kv_half8 qb[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        kv_u32x4 w = {0u, 0u, 0u, 0u};
        if (real) w = *reinterpret_cast<const kv_u32x4 *>(q + my_out * D + g * (D / 4) + 8 * u);
        qb[u] = __builtin_bit_cast(kv_half8, w);
    }

    // this wavefront's tiles: first + 4 n; lane n knows where tile n is
    const int first = t_begin / KV_TILE + wave, tiles = max(0, ((t_end + KV_TILE - 1) / KV_TILE - first + KVA_WAVES - 1) / KVA_WAVES);
    uint64_t my_tile = 0;
    if (lane < tiles) my_tile = reinterpret_cast<uint64_t>(kv_tile_at(v, b, head, first + KVA_WAVES * lane, T::BYTES));
    auto tile_address = [&](int n) {
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)my_tile, n), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(my_tile >> 32), n);
        return (uint64_t)hi << 32 | lo;
    };
    // A tile is a buffer that ends with it, and is empty past the range and where its page is none: then zeros arrive, without a branch and without a request.
    auto load = [&](KvTileRegs<T> &x, int n) {
        const uint64_t address = n < tiles ? tile_address(n) : 0;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(address), 0, address ? T::BYTES : 0, 0x00027000);
        auto b128 = [&](int byte) { return __builtin_bit_cast(kv_u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, byte, 0, 2)); };
#pragma unroll
        for (int i = 0; i < T::PIECES; ++i) x.k[i] = b128(lane * 16 + i * 1024);
        const auto h = __builtin_amdgcn_raw_buffer_load_b64(rsrc, T::KH_AT + ((g * (D / 4) / T::BLOCK) * 16 + li) * 8, 0, 2);
        x.kh[0] = h[0]; x.kh[1] = h[1];
#pragma unroll
        for (int i = 0; i < T::PIECES; ++i) x.v[i] = b128(T::V_AT + lane * 16 + i * 1024);
#pragma unroll
        for (int i = 0; i < T::NB; ++i) {
            x.vh[i][0] = b128(T::VH_AT + (i * 4 + g) * 32);
            x.vh[i][1] = b128(T::VH_AT + (i * 4 + g) * 32 + 16);
        }
    };

    float m = -INFINITY, l = 0.f;                             // of row li (m is the same in the row's four lanes)
    kv_float4 oacc[NC];                                       // oacc[c][e] = O[row 4g+e][16c + li]
#pragma unroll
    for (int c = 0; c < NC; ++c) oacc[c] = (kv_float4){0.f, 0.f, 0.f, 0.f};

    auto process = [&](KvTileRegs<T> &x, int n) {
        const int p0 = (first + KVA_WAVES * n) * KV_TILE;
        const bool there = tile_address(n) != 0;
        // scores
        kv_float4 sacc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const half2_t pair = as_h2(x.kh[h]), sc = {pair.x, pair.x}, of = {pair.y, pair.y};
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                constexpr int W = 8 / T::PER_WORD;            // words of eight components
                const int word = (h * NU + u) * W;
                uint32_t w[2] = {x.k[word / 4][word % 4], W == 2 ? x.k[word / 4][(word + W - 1) % 4] : 0u};
                KvPairs a = kv_levels<T::BITS>(w);
#pragma unroll
                for (int e = 0; e < 4; ++e) a.p[e] = kv_value(a.p[e], sc, of);
                sacc[h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(kv_half8, a), qb[u], sacc[h], 0, 0, 0);
            }
        }
        float sc[8], bm = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) {                         // position p0 + 16 (e / 4) + 4g + e % 4, row li
            sc[e] = there && p0 + 16 * (e >> 2) + 4 * g + (e & 3) < limit ? sacc[e >> 2][e & 3] * scale_log2e : -INFINITY;
            bm = fmaxf(bm, sc[e]);
        }
        bm = kva_max_of_rows(bm);
        const bool follow = bm > m + KVA_LAG;                 // (the first tile with a score above -inf: always)
        if (__builtin_amdgcn_ballot_w64(follow) != 0) {
            const float alpha = follow ? __builtin_amdgcn_exp2f(m - (bm - KVA_BELOW)) : 1.0f;
            l *= alpha;
            m = follow ? bm - KVA_BELOW : m;
            float al[4];                                      // the accumulators hold rows 4g .. 4g+3: their factors live in lanes 4g .. 4g+3
#pragma unroll
            for (int e = 0; e < 4; ++e) al[e] = __shfl(alpha, 4 * g + e);
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) oacc[c][e] *= al[e];
        }
        const float base = (m == -INFINITY) ? 0.f : m;        // (a row that has seen nothing: no -inf - -inf)
        kv_half8 pa, pr;                                      // the probabilities as two fp16 numbers
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float p = __builtin_amdgcn_exp2f(sc[e] - base);                     // exp2(-inf) = 0 for masked positions
            l += p;
            pa[e] = (_Float16)p;
            pr[e] = (_Float16)(p - (float)pa[e]);
        }
        // what lies behind the last position that a row sees may be anything, also no number: its values are zeros
        if (p0 + KV_TILE > t_end) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int p = p0 + 16 * (e >> 1) + 4 * g + 2 * (e & 1);
                const uint32_t keep = p + 1 < t_end ? 0xFFFFFFFFu : p < t_end ? 0x0000FFFFu : 0u;
#pragma unroll
                for (int i = 0; i < T::NB; ++i) { x.vh[i][0][e] &= keep; x.vh[i][1][e] &= keep; }
            }
        }
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            constexpr int W = 8 / T::PER_WORD;
            const int word = c * W, block = c * 16 / T::BLOCK;
            uint32_t w[2] = {x.v[word / 4][word % 4], W == 2 ? x.v[word / 4][(word + W - 1) % 4] : 0u};
            KvPairs a = kv_levels<T::BITS>(w);
#pragma unroll
            for (int e = 0; e < 4; ++e) a.p[e] = kv_value(a.p[e], as_h2(x.vh[block][0][e]), as_h2(x.vh[block][1][e]));
            oacc[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pa, __builtin_bit_cast(kv_half8, a), oacc[c], 0, 0, 0);
            oacc[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(pr, __builtin_bit_cast(kv_half8, a), oacc[c], 0, 0, 0);
        }
    };

    KvTileRegs<T> xa, xb;
    load(xa, 0);
    __builtin_amdgcn_sched_barrier(0);
    load(xb, 1);
    __builtin_amdgcn_sched_barrier(0);
    for (int n = 0; n < tiles; n += 2) {
        process(xa, n);
        __builtin_amdgcn_sched_barrier(0);
        load(xa, n + 2);
        __builtin_amdgcn_sched_barrier(0);
        if (n + 1 < tiles) process(xb, n + 1);
        __builtin_amdgcn_sched_barrier(0);
        load(xb, n + 3);
        __builtin_amdgcn_sched_barrier(0);
    }

    // ---- merge the four wavefronts' states --------------------------------------------------------------------------------
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) { s_m[wave][li] = m; s_l[wave][li] = l; }
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) s_o[wave][4 * g + e][16 * c + li] = oacc[c][e];
    __syncthreads();
    const KvPartial part(ws, v.n_tokens * n_heads, nsplit, D);
#pragma unroll
    for (int i = 0; i < KVA_ROWS * D / (64 * KVA_WAVES); ++i) {
        const int idx = tid + i * 64 * KVA_WAVES, r = idx / D, d = idx & (D - 1);
        const int tok = (r0 + r) / group;
        if (r >= rows || !seq.has_row(tok)) continue;
        float M = s_m[0][r];
#pragma unroll
        for (int w = 1; w < KVA_WAVES; ++w) M = fmaxf(M, s_m[w][r]);
        const float base = M == -INFINITY ? 0.f : M - KVA_SPARE;
        float L = 0.f, O = 0.f;
#pragma unroll
        for (int w = 0; w < KVA_WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(s_m[w][r] - base);                 // (nothing seen: zero)
            L = __builtin_fmaf(s_l[w][r], f, L);
            O = __builtin_fmaf(s_o[w][r][d], f, O);
        }
        const int64_t to = (seq.row + tok) * n_heads + head * group + (r0 + r - tok * group);
        if (mine == 1) {
            out[to * D + d] = as_u16((half_t)(L > 0.f ? O / L : 0.f));
        } else {
            part.o[(to * nsplit + sp) * D + d] = O;
            if (d == 0) { part.m[to * nsplit + sp] = M == -INFINITY ? M : base; part.l[to * nsplit + sp] = L; }
        }
    }
}

// Merge of the ranges: one workgroup of D threads per (sequence, token, query head).
__global__ void kv_attn_merge_kernel(KvView v, int n_heads, int group, int d_head, int chunk, int nsplit, const float *__restrict__ ws, uint16_t *__restrict__ out)
{
    const int h = blockIdx.x % n_heads, i = blockIdx.x / n_heads % v.max_tokens, b = blockIdx.x / n_heads / v.max_tokens, d = threadIdx.x;
    const KvSequence seq(v, b);
    if (!seq.has_row(i)) return;
    const int piece = (i * group + h % group) / KVA_ROWS, last = min(seq.count * group, (piece + 1) * KVA_ROWS) - 1;
    const int longest = seq.sees(last / group), mine = longest > chunk ? (longest + chunk - 1) / chunk : 1;
    if (mine == 1) return;                                    // (written by the first launch)
    const KvPartial part(const_cast<float *>(ws), v.n_tokens * n_heads, nsplit, d_head);
    const int64_t to = (seq.row + i) * n_heads + h;
    float M = -INFINITY;
    for (int s = 0; s < mine; ++s) M = fmaxf(M, part.m[to * nsplit + s]);
    const float base = M == -INFINITY ? 0.f : M - KVA_SPARE;
    float L = 0.f, O = 0.f;
    for (int s = 0; s < mine; ++s) {
        const float f = __builtin_amdgcn_exp2f(part.m[to * nsplit + s] - base);
        L = __builtin_fmaf(part.l[to * nsplit + s], f, L);
        O = __builtin_fmaf(part.o[(to * nsplit + s) * d_head + d], f, O);
    }
    out[to * d_head + d] = as_u16((half_t)(L > 0.f ? O / L : 0.f));
}

// Positions of a range and the number of ranges: about two workgroups per compute unit (of the 256 that a whole device has), none of fewer than 256 positions.
struct KvAttnGeometry { int chunk, nsplit, pieces; };
static KvAttnGeometry kv_attn_geometry(const KvView &v, int n_heads)
{
    const int group = n_heads / v.n_kv_heads;
    KvAttnGeometry r;
    r.pieces = (int)(((int64_t)v.max_tokens * group + KVA_ROWS - 1) / KVA_ROWS);
    const int64_t workgroups = (int64_t)v.n_seqs * v.n_kv_heads * r.pieces;
    int64_t want = (512 + workgroups - 1) / workgroups;
    int64_t chunk = (v.max_seq + want - 1) / want;
    const int64_t unit = KV_TILE * KVA_WAVES;
    chunk = (chunk + unit - 1) / unit * unit;
    if (chunk < 2 * unit) chunk = 2 * unit;
    if (chunk > KVA_MAX_CHUNK) chunk = KVA_MAX_CHUNK;
    r.chunk = (int)chunk;
    r.nsplit = (int)((v.max_seq + chunk - 1) / chunk);
    return r;
}

size_t kv_attn_workspace_bytes(const KvView &v, int head_dim, int n_heads)
{
    const KvAttnGeometry geo = kv_attn_geometry(v, n_heads);
    return geo.nsplit == 1 ? 0 : (size_t)v.n_tokens * n_heads * geo.nsplit * (head_dim + 2) * sizeof(float);
}

hipError_t launch_kv_attn(int format, int head_dim, const KvView &v, const uint16_t *q, int n_heads, float scale, uint16_t *out, void *workspace, hipStream_t s)
{
    const KvAttnGeometry geo = kv_attn_geometry(v, n_heads);
    const int group = n_heads / v.n_kv_heads;
    const int64_t grid = (int64_t)v.n_seqs * v.n_kv_heads * geo.nsplit * geo.pieces;
    const int64_t merge = (int64_t)v.n_seqs * v.max_tokens * n_heads;
    if (geo.nsplit > KVA_MAX_SPLITS || grid > 0x7fffffff || merge > 0x7fffffff) return hipErrorInvalidValue;
    hipError_t e = for_kv_tile(format, head_dim, [&](auto tag) {
        typedef decltype(tag) T;
        hipLaunchKernelGGL((kv_attn_kernel<T>), dim3((unsigned)grid), dim3(64 * KVA_WAVES), 0, s, v, q, n_heads, group, scale * 1.4426950408889634f, geo.chunk, geo.nsplit, geo.pieces,
                           out, static_cast<float *>(workspace));
        return hipGetLastError();
    });
    if (e != hipSuccess || geo.nsplit == 1) return e;
    hipLaunchKernelGGL(kv_attn_merge_kernel, dim3((unsigned)merge), dim3((unsigned)head_dim), 0, s, v, n_heads, group, head_dim, geo.chunk, geo.nsplit,
                       static_cast<const float *>(workspace), out);
    return hipGetLastError();
}

}  // namespace iflow
