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
#include <algorithm>

#include "iflow_kv.h"

namespace iflow {

constexpr int KVA_ROWS = 16;                                  // rows of a workgroup
// workgroups that a compute unit holds at once (by their registers), and the whole device
template <typename T> constexpr int KVA_PER_CU = T::D == 64 ? 4 : 3;
constexpr int KVA_CUS = 256;
constexpr float KVA_BELOW = 7.f, KVA_LAG = 15.f, KVA_SPARE = 16.f;       // in units of log2: see attn_decode_mfma_kernel
// A score's distance from the reference is one multiply-add, rounded once, while the reference is a rounded product: they differ by half a step of it, 2^-4 at 2^20.  Where a reference is as large, the scores
// are multiplied and rounded first, as it was (else the largest probability is two to that difference: no number from 2^32 on).
constexpr float KVA_FAR = 1048576.f;

// (The compiler quiets every operand of fmaxf first.  It does not see what these read: an accumulator of the matrix instructions is read by one of its own before, on whose result these depend, because it
// waits for them - up to twelve instructions long - only there.)
__device__ __forceinline__ float kv_max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// x - h.x, x - h.y in one instruction
__device__ __forceinline__ float kv_less_low(float x, half2_t h)
{
    float r;
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r) : "v"(as_u32(h)), "v"(x));
    return r;
}
__device__ __forceinline__ float kv_less_high(float x, half2_t h)
{
    float r;
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r) : "v"(as_u32(h)), "v"(x));
    return r;
}
// the maximum over the four lanes i, i + 16, i + 32, i + 48
__device__ __forceinline__ float kva_max_of_rows(float x)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    x = kv_max3(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]), -INFINITY);
    const auto b = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
    return kv_max3(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]), -INFINITY);
}

// Who does what.  The rows of a sequence's key/value head, sixteen at a time (a piece), go over all the sequence's tiles: that is a line of work.  How long the lines are only the device
// knows: every workgroup adds up all sequences' tiles and cuts the lines into parts of at most `share` tiles, and takes the part that its number says.  A part of several
// leaves partial results, which a second launch adds up.
// (Tried: ranges of a fixed number of positions: a die gets the same range of every sequence, 66 us for 32 sequences of 1000 to 8001 positions, 32/8 heads, turned by head and
// sequence 51; exactly equal shares of consecutive tiles that cross from line to line: a workgroup that crosses takes 5 us longer, and the rest wait for it, 45.)
// (Tiles are counted in 32 bits: where all lines might have more, every line is a workgroup's.  The device trusts no count that the host has not bounded: where the arrays make more lines than
// `max_lines`, which only sequences that claim rows twice or rows that there are not do, a line is one part, however long, and nothing but lines is counted: those are below 2^30 whatever the arrays hold.)
constexpr int KVA_WHOLE = 1 << 20;                            // a part of more tiles than a line has
struct KvLines { int tiles, lines; };                         // of each line; lines of the sequence
// (sequences of `few` rows and more are not served by sixteens)
__device__ __forceinline__ KvLines kv_lines_of(const KvView &v, const KvSequence &seq, int group, int few)
{
    KvLines x;
    x.lines = seq.count * group < few ? v.n_kv_heads * ((seq.count * group + KVA_ROWS - 1) / KVA_ROWS) : 0;
    x.tiles = max(1, (seq.sees(seq.count - 1) + KV_TILE - 1) / KV_TILE);       // (one that sees nothing has zeros to write)
    return x;
}
// work space: the partial results' slots before each sequence [n_seqs], the parts' tiles, then the partial results: M [slot][row], L [slot][row], O [slot][row][D].  (Lines of several parts have
// more tiles than a part has, and parts have at least 1 / capacity of all tiles: there are less than two for each workgroup that the device holds.)
struct KvPartial {
    static constexpr int SLOTS = 2 * 4 * KVA_CUS;
    int32_t *before;
    float *m, *l, *o;
    static __host__ __device__ __forceinline__ size_t head(int n_seqs) { return ((size_t)n_seqs + 4) / 4 * 4; }
    __device__ __forceinline__ KvPartial(void *ws, int n_seqs)
        : before(static_cast<int32_t *>(ws)), m(reinterpret_cast<float *>(before + head(n_seqs))), l(m + SLOTS * KVA_ROWS), o(l + SLOTS * KVA_ROWS) {}
    // (number n is one of them; also where another stream changes the lengths meanwhile)
    static __device__ __forceinline__ int slot(int n) { return (int)min((uint32_t)n, (uint32_t)(SLOTS - 1)); }
    static size_t bytes(int n_seqs, int d) { return head(n_seqs) * 4 + (size_t)SLOTS * KVA_ROWS * (2 + d) * 4; }
};
__device__ __forceinline__ int kv_parts(int tiles, int share) { return (int)((uint32_t)(tiles + share - 1) / (uint32_t)share); }
// n / d of numbers whose product is below 2^32, by a multiplication
struct KvDivide {
    uint32_t magic;
    KvDivide(int d) : magic(d == 1 ? 0u : (uint32_t)(((1ULL << 32) + d - 1) / (uint32_t)d)) {}
    __device__ __forceinline__ int operator()(int n) const { return magic ? (int)__umulhi((uint32_t)n, magic) : n; }
};

// A tile as it is loaded: a lane's runs, and the headers of its positions.
template <typename T>
struct KvTileRegs {
    kv_u32x4 k[T::PIECES], v[T::PIECES];
    uint32_t kh[2];                                           // (scale, offset) of position i, of 16 + i, in the block of the lane's quarter
    kv_u32x4 vh[T::NB][2];                                    // scales, offsets of its eight positions, by block
};

// DIRECT: a workgroup is a line: blockIdx.x of sequence blockIdx.y (max_lines 0), or, by its number in both, of all.
template <typename T, int WAVES, bool DIRECT>
__global__ __launch_bounds__(64 * WAVES, WAVES == 4 ? KVA_PER_CU<T> : 1) void kv_attn_kernel(KvView v, const uint16_t *__restrict__ q, int n_heads, int group, int few, int max_lines,
                                                                                           KvDivide by_group, KvDivide by_heads, float scale_log2e, uint16_t *__restrict__ out, void *ws)
{
    constexpr int D = T::D, NU = D / 32, NC = D / 16;
    constexpr int PAD = 4;                                    // floats: rows four apart in banks of their own
    __shared__ __align__(16) float s_o[WAVES][KVA_ROWS][D + PAD];
    __shared__ float s_m[WAVES][KVA_ROWS], s_l[WAVES][KVA_ROWS];
    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const KvPartial part(ws, v.n_seqs);

    const int lane = tid & 63, li = lane & 15, g = lane >> 4;
    // which sequence, which line and part of it, and where the sequence's partial results begin
    int b = 0, at = 0, slots = 0, share = 0;
    if constexpr (DIRECT) {
        at = max_lines ? blockIdx.y * gridDim.x + blockIdx.x : blockIdx.x;
        if (!max_lines) b = blockIdx.y;
        else if (!kv_find(v, at, b, [&](const KvSequence &seq) { return kv_lines_of(v, seq, group, few).lines; })) return;
    } else {
        auto lines_of = [&](int s) {
            if (s >= v.n_seqs) return KvLines{0, 0};
            const KvSequence seq(v, s);
            return kv_lines_of(v, seq, group, few);
        };
        auto last = [](int x) { return __builtin_amdgcn_readlane(x, 63); };
        KvLines mine = lines_of(lane);                        // (the first 64 sequences are all in most calls)
        // (unsigned: where lines turn out to be too many, this has wrapped and is not used)
        auto tiles_of = [&](const KvLines &x) { return (uint32_t)last(wave_scan((int)((uint32_t)x.tiles * (uint32_t)x.lines))); };
        uint32_t sum = tiles_of(mine);
        int lines = last(wave_scan(mine.lines));
        for (int s = 64; s < v.n_seqs; s += 64) {
            const KvLines x = lines_of(s + lane);
            sum += tiles_of(x); lines += last(wave_scan(x.lines));
        }
        const int total = (int)sum;
        // The parts' tiles: one for each wavefront where all are few, else at least two (a part costs about as much as four tiles besides).  The fewest that leave no more parts than the device
        // holds at once, for what does not fit waits for a whole part; where there are half as many lines already, 1 / capacity of all tiles: parts are then about as many again as lines.
        constexpr int UNIT = WAVES, CAPACITY = KVA_PER_CU<T> * KVA_CUS;
        if (lines > max_lines) {
            share = KVA_WHOLE;
        } else if (lines > CAPACITY / 2) {
            share = max(2 * UNIT, (total / CAPACITY + UNIT) / UNIT * UNIT);
        } else if (v.n_seqs > 64) {
            share = max(2 * UNIT, (total / (CAPACITY - lines) + UNIT) / UNIT * UNIT);      // (a line has less than one part more than its tiles over a part's)
        } else {
            share = total <= KVA_CUS * UNIT ? UNIT : max(2 * UNIT, (total / (CAPACITY - lines / 2) + UNIT - 1) / UNIT * UNIT);
            while (last(wave_scan(mine.lines * kv_parts(mine.tiles, share))) > CAPACITY) share += UNIT;
        }
        const bool clerk = blockIdx.x == gridDim.x - 1;       // the last workgroup writes down what the merge wants to know
        if (clerk && wave > 0) return;
        at = blockIdx.x;
        for (;;) {
            const int parts = kv_parts(mine.tiles, share), work = mine.lines * parts, upto = wave_scan(work), held = parts > 1 ? work : 0, held_upto = wave_scan(held);
            if (clerk) {
                if (b + lane < v.n_seqs) part.before[b + lane] = slots + held_upto - held;
                if (b == 0 && lane == 0) part.before[v.n_seqs] = share;
            } else {
                const uint64_t mask = __builtin_amdgcn_ballot_w64(upto > at);
                if (mask != 0) {
                    const int skip = __builtin_ctzll(mask);
                    b += skip;
                    at -= __builtin_amdgcn_readlane(upto - work, skip);
                    slots += __builtin_amdgcn_readlane(held_upto - held, skip);
                    break;
                }
                at -= last(upto);
            }
            slots += last(held_upto);
            b += 64;
            if (b >= v.n_seqs) return;                        // (there are more workgroups than parts)
            mine = lines_of(b + lane);
        }
    }
    const KvSequence seq(v, b);
    const KvLines x = kv_lines_of(v, seq, group, few);
    if (DIRECT && at >= x.lines) return;
    const int parts = DIRECT ? 1 : kv_parts(x.tiles, share);
    const int line = DIRECT ? at : __builtin_amdgcn_readfirstlane((int)((uint32_t)at / (uint32_t)parts)), my_part = at - line * parts;
    // (parts as long as one another, in whole tiles for each wavefront)
    const int per = DIRECT ? x.tiles : min(share, (kv_parts(x.tiles, parts) + WAVES - 1) / WAVES * WAVES), t0 = DIRECT ? 0 : my_part * per, n_tiles = min(per, x.tiles - t0);
    const int piece = by_heads(line), head = line - piece * v.n_kv_heads;
    const KvMagic magic;
    {
        const int r0 = piece * KVA_ROWS, rows = min(KVA_ROWS, seq.count * group - r0);
        const int longest = seq.sees(by_group(r0 + rows - 1)), shortest = seq.sees(by_group(r0));      // the last row sees most
        const int my_row = r0 + min(li, rows - 1), token = by_group(my_row);
        const int64_t my_out = (int64_t)(seq.row + token) * n_heads + head * group + (my_row - token * group);
        const int limit = seq.sees(token);
        // queries as B operands: lane (row li, g) holds components g D/4 + 8u .. +8
        kv_half8 qb[NU];
        const bool real = li < rows && seq.has_row(token);
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            kv_u32x4 w = {0u, 0u, 0u, 0u};
            if (real) w = *reinterpret_cast<const kv_u32x4 *>(q + my_out * D + g * (D / 4) + 8 * u);
            qb[u] = __builtin_bit_cast(kv_half8, w);
        }
        float m = -INFINITY, l = 0.f;                         // of row li (m is the same in the row's four lanes)
        bool far = false;                                     // a row's reference is, or was, as large as KVA_FAR
        kv_float4 oacc[NC];                                   // oacc[c][e] = O[row 4g+e][16c + li]
#pragma unroll
        for (int c = 0; c < NC; ++c) oacc[c] = (kv_float4){0.f, 0.f, 0.f, 0.f};

        // 256 tiles at a time; this wavefront's: first + 4 n, and lane n knows where tile n is
        for (int done = 0; done < n_tiles; done += 64 * WAVES) {
            const int first = t0 + done + wave, last = min(t0 + min(n_tiles, done + 64 * WAVES), (longest + KV_TILE - 1) / KV_TILE);
            const int tiles = __builtin_amdgcn_readfirstlane(max(0, (last - first + WAVES - 1) / WAVES));       // (the same for the wavefront, as the compiler is told)
            uint64_t my_tile = 0;
            if (lane < tiles) my_tile = reinterpret_cast<uint64_t>(kv_tile_at(v, b, head, first + WAVES * lane, T::BYTES));
            auto tile_address = [&](int n) {
                const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)my_tile, n), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(my_tile >> 32), n);
                return (uint64_t)hi << 32 | lo;
            };
            // A tile is a buffer that ends with it, and is empty past the range and where its page is none: then zeros arrive, without a branch and without a request.
            auto tile_buffer = [&](int n) {
                const uint64_t address = n < tiles ? tile_address(n) : 0;
                return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(address), 0, address ? T::BYTES : 0, 0x00027000);
            };
            auto load_keys = [&](KvTileRegs<T> &y, int n) {
                const auto rsrc = tile_buffer(n);
#pragma unroll
                for (int i = 0; i < T::PIECES; ++i) y.k[i] = __builtin_bit_cast(kv_u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane * 16 + i * 1024, 0, 2));
                const auto h = __builtin_amdgcn_raw_buffer_load_b64(rsrc, T::KH_AT + ((g * (D / 4) / T::BLOCK) * 16 + li) * 8, 0, 2);
                y.kh[0] = h[0]; y.kh[1] = h[1];
            };
            auto load_values = [&](KvTileRegs<T> &y, int n) {
                const auto rsrc = tile_buffer(n);
#pragma unroll
                for (int i = 0; i < T::PIECES; ++i) y.v[i] = __builtin_bit_cast(kv_u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, T::V_AT + lane * 16 + i * 1024, 0, 2));
#pragma unroll
                for (int i = 0; i < T::NB; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) y.vh[i][j] = __builtin_bit_cast(kv_u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, T::VH_AT + (i * 4 + g) * 32 + 16 * j, 0, 2));
            };

            KvTileRegs<T> y;
            // (Scheduling barriers: the waits count requests, so keys and values have to be requested in the same order in front of the loop and in it, or a wait becomes one for everything.)
            __builtin_amdgcn_sched_barrier(0);
            load_keys(y, 0);
            __builtin_amdgcn_sched_barrier(0);
            load_values(y, 0);
            __builtin_amdgcn_sched_barrier(0);
            for (int n = 0; n < tiles; ++n) {
                const int p0 = (first + WAVES * n) * KV_TILE;
                // scores
                kv_float4 sacc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const half2_t pair = as_h2(y.kh[h]), sc = {pair.x, pair.x}, of = {pair.y, pair.y};
#pragma unroll
                    for (int u = 0; u < NU; ++u) {
                        constexpr int W = 8 / T::PER_WORD;    // words of eight components
                        const int word = (h * NU + u) * W;
                        uint32_t w[2] = {y.k[word / 4][word % 4], W == 2 ? y.k[word / 4][(word + W - 1) % 4] : 0u};
                        KvPairs a = kv_levels<T::BITS>(w, magic);
#pragma unroll
                        for (int e = 0; e < 4; ++e) a.p[e] = kv_value(a.p[e], sc, of);
                        sacc[h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(kv_half8, a), qb[u], sacc[h], 0, 0, 0);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                load_keys(y, n + 1);                          // (into the registers that have just been read)
                __builtin_amdgcn_sched_barrier(0);
                // position p0 + 16 (e / 4) + 4g + e % 4, row li: not seen from the row's limit on, nor on a page that is not there
                const bool there = tile_address(n) != 0;
                if (!there || p0 + KV_TILE > shortest) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (!there || p0 + 16 * (e >> 2) + 4 * g + (e & 3) >= limit) sacc[e >> 2][e & 3] = -INFINITY;
                }
                float bm = fmaxf(sacc[0][3], sacc[1][3]);     // (the compiler's own: see kv_max3)
                bm = kv_max3(bm, sacc[0][0], sacc[0][1]);
                bm = kv_max3(bm, sacc[0][2], sacc[1][0]);
                bm = kv_max3(bm, sacc[1][1], sacc[1][2]);
                bm = kva_max_of_rows(bm) * scale_log2e;
                const bool follow = bm > m + KVA_LAG;         // (the first tile with a score above -inf: always)
                if (__builtin_amdgcn_ballot_w64(follow) != 0) {
                    const float alpha = follow ? __builtin_amdgcn_exp2f(m - (bm - KVA_BELOW)) : 1.0f;
                    const bool nothing = __builtin_amdgcn_ballot_w64(m != -INFINITY) == 0;
                    l *= alpha;
                    m = follow ? bm - KVA_BELOW : m;
                    far = far || __builtin_amdgcn_ballot_w64(fabsf(m) >= KVA_FAR && m != -INFINITY) != 0;
                    if (!nothing) {                           // the accumulators hold rows 4g .. 4g+3: their factors live in lanes 4g .. 4g+3
                        float al[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) al[e] = __shfl(alpha, 4 * g + e);
#pragma unroll
                        for (int c = 0; c < NC; ++c)
#pragma unroll
                            for (int e = 0; e < 4; ++e) oacc[c][e] *= al[e];
                    }
                }
                const float below = (m == -INFINITY) ? 0.f : -m;       // (a row that has seen nothing: no -inf - -inf)
                if (__builtin_expect(far, false)) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) sacc[e >> 2][e & 3] *= scale_log2e;
                }
                const float by = far ? 1.f : scale_log2e;
                // the probabilities as two fp16 numbers, the first cut off so that both are positive: together within 2^-21 of them
                KvPairs pa, pr;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p0e = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[e >> 1][2 * (e & 1)], by, below));          // exp2(-inf) = 0 for masked positions
                    const float p1e = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[e >> 1][2 * (e & 1) + 1], by, below));
                    l += p0e; l += p1e;
                    pa.p[e] = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_pkrtz(p0e, p1e));
                    pr.p[e] = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_pkrtz(kv_less_low(p0e, pa.p[e]), kv_less_high(p1e, pa.p[e])));
                }
                // what lies behind the last position that a row sees may be anything, also no number: its values are zeros
                if (p0 + KV_TILE > longest) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int p = p0 + 16 * (e >> 1) + 4 * g + 2 * (e & 1);
                        const uint32_t keep = p + 1 < longest ? 0xFFFFFFFFu : p < longest ? 0x0000FFFFu : 0u;
#pragma unroll
                        for (int i = 0; i < T::NB; ++i) { y.vh[i][0][e] &= keep; y.vh[i][1][e] &= keep; }
                    }
                }
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    constexpr int W = 8 / T::PER_WORD;
                    const int word = c * W, block = c * 16 / T::BLOCK;
                    uint32_t w[2] = {y.v[word / 4][word % 4], W == 2 ? y.v[word / 4][(word + W - 1) % 4] : 0u};
                    KvPairs a = kv_levels<T::BITS>(w, magic);
#pragma unroll
                    for (int e = 0; e < 4; ++e) a.p[e] = kv_value(a.p[e], as_h2(y.vh[block][0][e]), as_h2(y.vh[block][1][e]));
                    oacc[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(kv_half8, pa), __builtin_bit_cast(kv_half8, a), oacc[c], 0, 0, 0);
                    oacc[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(kv_half8, pr), __builtin_bit_cast(kv_half8, a), oacc[c], 0, 0, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
                load_values(y, n + 1);
                __builtin_amdgcn_sched_barrier(0);
            }
        }

        // ---- merge the four wavefronts' states ----------------------------------------------------------------------------
        int id = tid;
        asm volatile("" : "+v"(id));                          // (the addresses below are made here, not kept in registers through the tiles)
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if ((id & 48) == 0) { s_m[wave][id & 15] = m; s_l[wave][id & 15] = l; }
        float *my_o = &s_o[wave][4 * (id >> 4 & 3)][id & 15];
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) my_o[e * (D + PAD) + 16 * c] = oacc[c][e];
        __syncthreads();
        const int slot = KvPartial::slot(slots + at);
        constexpr int QUADS = D / 4;                          // a thread takes four components of a row
#pragma unroll
        for (int i = 0; i < (KVA_ROWS * QUADS + 64 * WAVES - 1) / (64 * WAVES); ++i) {
            const int r = id / QUADS + i * (64 * WAVES / QUADS), d = id % QUADS * 4, tok = by_group(r0 + r);
            if (KVA_ROWS * QUADS < 64 * WAVES && r >= KVA_ROWS) break;        // (64 components, eight wavefronts: half the threads)
            float M = s_m[0][r];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) M = fmaxf(M, s_m[w][r]);
            const float to_base = M == -INFINITY ? 0.f : M - KVA_SPARE;
            float L = 0.f;
            kv_float4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = __builtin_amdgcn_exp2f(s_m[w][r] - to_base);          // (nothing seen: zero)
                const kv_float4 o = *reinterpret_cast<const kv_float4 *>(&s_o[w][r][d]);
                L = __builtin_fmaf(s_l[w][r], f, L);
#pragma unroll
                for (int e = 0; e < 4; ++e) O[e] = __builtin_fmaf(o[e], f, O[e]);
            }
            if (parts == 1) {
                if (r < rows && seq.has_row(tok)) {
                    const float div = L > 0.f ? L : 1.f;      // (nothing seen: zeros)
                    const half2_t a = {(half_t)(O[0] / div), (half_t)(O[1] / div)}, c = {(half_t)(O[2] / div), (half_t)(O[3] / div)};
                    const int64_t to = (int64_t)(seq.row + tok) * n_heads + head * group + (r0 + r - tok * group);
                    *reinterpret_cast<kv_u32x2 *>(out + to * D + d) = (kv_u32x2){as_u32(a), as_u32(c)};
                }
            } else {
                *reinterpret_cast<kv_float4 *>(part.o + (slot * KVA_ROWS + r) * D + d) = O;
                if (d == 0) { part.m[slot * KVA_ROWS + r] = M == -INFINITY ? M : to_base; part.l[slot * KVA_ROWS + r] = L; }
            }
        }
    }
}

// Merge of a line's partial results: one workgroup per (sequence, token, query head), thread (d, u) for component d of results 8u .. 8u + 7, then 8 (u + groups) ..: a group's eight are requested
// at once, and the groups' states meet in LDS and are added in order.
constexpr int KVA_MERGE = 8;
__device__ __forceinline__ void kv_attn_merge(const KvView &v, int b, int i, int h, int n_heads, int group, int few, void *ws, uint16_t *__restrict__ out)
{
    __shared__ float s_o[8][128], s_m[8], s_l[8];
    const int D = blockDim.x, d = threadIdx.x, groups = blockDim.y, u = threadIdx.y;
    const KvPartial part(ws, v.n_seqs);
    const int before = part.before[b], share = part.before[v.n_seqs];
    const KvSequence seq(v, b);
    if (!seq.has_row(i)) return;
    const KvLines x = kv_lines_of(v, seq, group, few);
    if (x.lines == 0) return;
    const int row = i * group + h % group, piece = row / KVA_ROWS, r = row % KVA_ROWS, line = piece * v.n_kv_heads + h / group;
    const int mine = kv_parts(x.tiles, share);
    if (mine == 1) return;                                    // (written by the first launch)
    auto slot = [&](int s) { return KvPartial::slot(before + line * mine + s) * KVA_ROWS + r; };
    float M = -INFINITY, L = 0.f, O = 0.f;                    // relative to to_base(M)
    auto to_base = [](float m) { return m == -INFINITY ? 0.f : m - KVA_SPARE; };
    for (int s0 = u * KVA_MERGE; s0 < mine; s0 += groups * KVA_MERGE) {
        float m[KVA_MERGE], l[KVA_MERGE], o[KVA_MERGE], top = M;
#pragma unroll
        for (int e = 0; e < KVA_MERGE; ++e) {
            const int s = slot(min(s0 + e, mine - 1));    // past the end: the last one again, with no weight
            m[e] = part.m[s]; l[e] = part.l[s]; o[e] = part.o[s * D + d];
        }
#pragma unroll
        for (int e = 0; e < KVA_MERGE; ++e) top = fmaxf(top, m[e]);
        const float now = to_base(top), again = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(to_base(M) - now);
        L *= again; O *= again;
        M = top;
#pragma unroll
        for (int e = 0; e < KVA_MERGE; ++e) {
            const float f = s0 + e < mine ? __builtin_amdgcn_exp2f(m[e] - now) : 0.f;
            L = __builtin_fmaf(l[e], f, L);
            O = __builtin_fmaf(o[e], f, O);
        }
    }
    if (groups > 1) {
        s_o[u][d] = O;
        if (d == 0) { s_m[u] = M; s_l[u] = L; }
        __syncthreads();
        if (u > 0) return;
        for (int e = 1; e < groups; ++e) M = fmaxf(M, s_m[e]);
        L = 0.f; O = 0.f;
        for (int e = 0; e < groups; ++e) {
            const float f = s_m[e] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(to_base(s_m[e]) - to_base(M));
            L = __builtin_fmaf(s_l[e], f, L);
            O = __builtin_fmaf(s_o[e][d], f, O);
        }
    }
    out[((int64_t)(seq.row + i) * n_heads + h) * D + d] = as_u16((half_t)(L > 0.f ? O / L : 0.f));
}
// Token y of sequence z for head x; packed (one z): the x-th, the x + grid-th, .. token of the sequences that sixteens serve, for head y.
__global__ __launch_bounds__(1024) void kv_attn_merge_kernel(KvView v, int n_heads, int group, int few, void *ws, uint16_t *__restrict__ out)
{
    if ((int)gridDim.z == v.n_seqs) return kv_attn_merge(v, blockIdx.z, blockIdx.y, blockIdx.x, n_heads, group, few, ws, out);
    for (int x = blockIdx.x, b, i; i = x, kv_find(v, i, b, [&](const KvSequence &seq) { return seq.count * group < few ? seq.count : 0; }); x += gridDim.x) {
        kv_attn_merge(v, b, i, blockIdx.y, n_heads, group, few, ws, out);
        __syncthreads();
    }
}

// ---- many rows: prompts -----------------------------------------------------------------------------------------------------
// With dozens of rows a tile is decoded once for all of them: RG wavefronts of 32 rows each share 64 positions, which they decode into LDS together, in the order in which
// v_mfma_f32_32x32x16_f16 takes its operands (A: lane i + 32 h holds A[i][8h..8h+7], B alike, D: element e of lane j + 32 h is D[8 (e / 4) + 4h + e % 4][j]):
//   S[position][row] = K Q^T with the queries in registers; a lane has one row's scores, sixteen of every 32 positions, and its half of the row's maximum and sum;
//   O[component][row] = V^T P^T: element e of a tile's scores is position 4g + e % 4 or 16 + 4g + e % 4 of g = 2 (e / 8) + h where row i of S is position i with bits 3 and 4 changed
//   over, so a lane's probabilities are its own operand, and a value's eight positions are a word of the cache's.  The sums' factors are the lane's own too.
// Keys in LDS: [tile][component / 8][i: 32][8 components], values: [tile][g][component][8 positions]: 16-byte pieces that 32 lanes read side by side.
// PG groups of wavefronts take every PG-th 64 positions and add up in LDS: where there are too few rows to fill the device.  The probabilities are two fp16 numbers each, and two products of every value,
// as in kv_attn_kernel: a token's output does not depend on how many rows its batch has but for the order of fp32 sums.  (Rounded to fp16 once, with one product, they made the largest error 1.4e-3 of a
// row's rms where the output's own rounding is 4.9e-4, and prompts of 2500 tokens, 64/8 heads, took 284 us for the 352 now; 512 tokens behind 3888, 32/8 heads, 60 for 71.)
typedef float kv_float16 __attribute__((ext_vector_type(16)));

template <typename T, int RG, int PG, int STAGES>
__global__ __launch_bounds__(64 * RG * PG, RG * PG == 4 ? 2 : 1) void kv_attn_rows_kernel(KvView v, const uint16_t *__restrict__ q, int n_heads, int group, int few, KvDivide by_group, float scale_log2e,
                                                                                          uint16_t *__restrict__ out)
{
    constexpr int D = T::D, NU = D / 16, NC = D / 32, STEP = 2 * KV_TILE;      // NU: steps of 16 components; NC: groups of 32
    constexpr int UNITS = 2 * T::PIECES;                      // 1 KB of key codes (and of value codes) of a step
    constexpr bool SPLIT = UNITS < RG;                        // half the wavefronts decode keys, half values
    constexpr int MINE = SPLIT ? 1 : UNITS / RG;
    constexpr int KEYS = STEP * D * 2, GROUP = 2 * STAGES * KEYS;      // bytes of a step's keys (its values are as many), of what a group of wavefronts stages
    constexpr int ROWS = 32 * RG;
    static_assert(SPLIT ? 2 * UNITS == RG : UNITS % RG == 0, "the wavefronts share the decoding evenly");
    constexpr int MERGE = (PG > 1 ? PG * ROWS * (D + 4) * 4 : 0), LDS = GROUP * PG > MERGE ? GROUP * PG : MERGE;
    __shared__ __align__(16) uint8_t s_mem[LDS];
    __shared__ float s_m[PG][ROWS], s_l[PG][ROWS];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), rg = wave % RG, pg = wave / RG;
    const int li = lane & 31, hf = lane >> 5;
    int head = blockIdx.x, b = blockIdx.z, block = blockIdx.y;
    if (few > 0) {                                            // the blocks of the sequences that have as many rows, one after another
        const unsigned number = blockIdx.y * gridDim.x + blockIdx.x;
        block = number / (unsigned)v.n_kv_heads;
        head = number - block * v.n_kv_heads;
        if (!kv_find(v, block, b, [&](const KvSequence &seq) { return seq.count * group < few ? 0 : (seq.count * group + ROWS - 1) / ROWS; })) return;
    }
    // where tile 64 n + lane is: the first 64 are asked for before the sequence's length is known
    uint64_t my_tile = 0;
    auto find_tiles = [&](int t0) { my_tile = (t0 + lane) * KV_TILE < v.max_seq ? reinterpret_cast<uint64_t>(kv_tile_at(v, b, head, t0 + lane, T::BYTES)) : 0; };
    find_tiles(0);
    const KvSequence seq(v, b);
    const int n_rows = seq.count * group;
    const int r0 = ((few > 0 ? (n_rows + ROWS - 1) / ROWS : (int)gridDim.y) - 1 - block) * ROWS;      // (the last rows, which see most, first)
    if (r0 >= n_rows) return;
    // (the same for the wavefront, as the compiler is told: what it takes for different in the lanes costs a loop around every load)
    auto same = [](int n) { return __builtin_amdgcn_readfirstlane(n); };
    const int longest = same(seq.sees(by_group(min(n_rows, r0 + ROWS) - 1)));
    const int my_row = min(n_rows - 1, r0 + rg * 32 + li), token = by_group(my_row), limit = seq.sees(token);
    const bool real = r0 + rg * 32 + li < n_rows && seq.has_row(token);
    const int64_t my_out = ((int64_t)(seq.row + token) * n_heads + head * group + (my_row - token * group)) * D;
    // of the wavefront's rows: what the first sees, and the last
    const int shortest = same(seq.sees(by_group(min(n_rows - 1, r0 + rg * 32)))), limit_of_wave = same(seq.sees(by_group(min(n_rows - 1, r0 + rg * 32 + 31))));
    uint8_t *stage = s_mem + pg * GROUP;

    // queries as B operands: lane (row li, hf) holds components 16u + 8 hf .. +8
    kv_half8 qb[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        kv_u32x4 w = {0u, 0u, 0u, 0u};
        if (real) w = *reinterpret_cast<const kv_u32x4 *>(q + my_out + 16 * u + 8 * hf);
        qb[u] = __builtin_bit_cast(kv_half8, w);
    }
    float m = -INFINITY, l = 0.f;
    bool far = false;                                         // a row's reference is, or was, as large as KVA_FAR
    kv_float16 oacc[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e) oacc[c][e] = 0.f;

    const KvMagic magic;
    const int tiles = (longest + KV_TILE - 1) / KV_TILE, steps = (tiles + 1) / 2;
    const int trips = (steps + PG - 1) / PG;                  // the same for all groups: they meet at the barriers
    auto tile_address = [&](int t) {
        const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)my_tile, t & 63), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(my_tile >> 32), t & 63);
        return (uint64_t)hi << 32 | lo;
    };
    // What this wavefront decodes of a step: units of 1 KB, a piece of a tile's key codes or value codes.
    constexpr int W = 8 / T::PER_WORD, CH = 4 / W;            // words of eight elements; eights of a lane's 16 bytes
    constexpr int VB = CH * 16 > T::BLOCK ? CH * 16 / T::BLOCK : 1;    // blocks that a value piece's components lie in
    struct Keys { kv_u32x4 k[MINE]; uint32_t kh[MINE][2]; };
    struct Codes : Keys { kv_u32x4 v[MINE], vh[MINE][VB][2]; } x;
    const int g = lane >> 4, i = lane & 15;                   // the cache's (g, i)
    const bool keys = !SPLIT || rg < UNITS, values = !SPLIT || rg >= UNITS;
    auto unit_of = [&](int j) { return SPLIT ? rg % UNITS : rg + RG * j; };
    auto buffer_of = [&](int t) {                             // (empty where there is none: zeros arrive)
        const uint64_t address = t < tiles ? tile_address(t) : 0;
        return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(address), 0, address ? T::BYTES : 0, 0x00027000);
    };
    auto load_keys = [&](int t0) {                            // t0: the step's first tile
        if (!keys) return;
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
            const int unit = unit_of(j), n = unit % T::PIECES;
            const auto rsrc = buffer_of(t0 + unit / T::PIECES);
            x.k[j] = __builtin_bit_cast(kv_u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane * 16 + n * 1024, 0, 0));
            const auto h = __builtin_amdgcn_raw_buffer_load_b64(rsrc, T::KH_AT + ((g * (D / 4) / T::BLOCK) * 16 + i) * 8, 0, 0);
            x.kh[j][0] = h[0]; x.kh[j][1] = h[1];
        }
    };
    auto load_values = [&](int t0) {
        if (!values) return;
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
            const int unit = unit_of(j), n = unit % T::PIECES;
            const auto rsrc = buffer_of(t0 + unit / T::PIECES);
            x.v[j] = __builtin_bit_cast(kv_u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, T::V_AT + lane * 16 + n * 1024, 0, 0));
#pragma unroll
            for (int y = 0; y < VB; ++y)
#pragma unroll
                for (int z = 0; z < 2; ++z)
                    x.vh[j][y][z] = __builtin_bit_cast(kv_u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, T::VH_AT + (y * 4 + g) * 32 + 16 * z + n * CH * 16 / T::BLOCK * 128, 0, 0));
        }
    };
    auto decode_key = [&](uint8_t *to, int j, int y) {         // word 4 n + y W of the run: half h of the tile, components c ..
        const int unit = unit_of(j), tile = unit / T::PIECES, n = unit % T::PIECES;
        constexpr bool SHORT = T::RUN / 2 < 4;
        const int h = SHORT ? y * W / (T::RUN / 2) : n / (SHORT ? 1 : T::RUN / 8), c = g * (D / 4) + (SHORT ? y * W % (T::RUN / 2) : (4 * n + y * W) % (T::RUN / 2)) * T::PER_WORD;
        const half2_t pair = as_h2(h ? x.kh[j][1] : x.kh[j][0]), sc = {pair.x, pair.x}, of = {pair.y, pair.y};
        uint32_t w[2] = {x.k[j][y * W], W == 2 ? x.k[j][(y * W + W - 1) % 4] : 0u};
        KvPairs a = kv_levels<T::BITS>(w, magic);
#pragma unroll
        for (int e = 0; e < 4; ++e) a.p[e] = kv_value(a.p[e], sc, of);
        const int at = (i & 7) | h << 3 | (i >> 3) << 4;
        *reinterpret_cast<kv_u32x4 *>(to + ((tile * (D / 8) + c / 8) * 32 + at) * 16) = __builtin_bit_cast(kv_u32x4, a);
    };
    auto decode_value = [&](uint8_t *to, int j, int y) {
        const int unit = unit_of(j), tile = unit / T::PIECES, n = unit % T::PIECES;
        uint32_t w[2] = {x.v[j][y * W], W == 2 ? x.v[j][(y * W + W - 1) % 4] : 0u};
        KvPairs a = kv_levels<T::BITS>(w, magic);
#pragma unroll
        for (int e = 0; e < 4; ++e) a.p[e] = kv_value(a.p[e], as_h2(x.vh[j][y * VB / CH][0][e]), as_h2(x.vh[j][y * VB / CH][1][e]));
        *reinterpret_cast<kv_u32x4 *>(to + ((tile * 4 + g) * D + (n * CH + y) * 16 + i) * 16) = __builtin_bit_cast(kv_u32x4, a);
    };
    constexpr int CHUNKS = MINE * CH;                         // eights of a lane: of keys, and of values
    auto decode_keys = [&](uint8_t *to) {
        if (!keys) return;
#pragma unroll
        for (int n = 0; n < CHUNKS; ++n) decode_key(to, n / CH, n % CH);
    };
    auto decode_values = [&](uint8_t *to) {
        if (!values) return;
#pragma unroll
        for (int n = 0; n < CHUNKS; ++n) decode_value(to, n / CH, n % CH);
    };
    // what lies behind the last position that a row sees may be anything, also no number: its values are zeros
    auto cut_values = [&](int t0) {
        if (!values || t0 * KV_TILE + STEP <= longest) return;
#pragma unroll
        for (int j = 0; j < MINE; ++j) {
            const int p0 = (t0 + unit_of(j) / T::PIECES) * KV_TILE;
            {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int p = p0 + 16 * (e >> 1) + 4 * g + 2 * (e & 1);
                    const uint32_t keep = p + 1 < longest ? 0xFFFFFFFFu : p < longest ? 0x0000FFFFu : 0u;
#pragma unroll
                    for (int y = 0; y < VB; ++y) { x.vh[j][y][0][e] &= keep; x.vh[j][y][1][e] &= keep; }
                }
            }
        }
    };
    // scores of a step from its keys in LDS: product n of 2 NU is components 16 (n / 2) .. of tile n % 2
    kv_float16 sacc[2];
    auto key_operand = [&](const uint8_t *from, int n) { return *reinterpret_cast<const kv_half8 *>(from + ((n % 2 * (D / 8) + 2 * (n / 2) + hf) * 32 + li) * 16); };
    auto clear = [&](kv_float16 (&to)[2]) {
#pragma unroll
        for (int tl = 0; tl < 2; ++tl)
#pragma unroll
            for (int e = 0; e < 16; ++e) to[tl][e] = 0.f;
    };
    auto score = [&](const uint8_t *from, kv_float16 (&to)[2]) {
        clear(to);
#pragma unroll
        for (int n = 0; n < 2 * NU; ++n) to[n % 2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(key_operand(from, n), qb[n / 2], to[n % 2], 0, 0, 0);
    };
    // what a row does not see goes, and the reference and the sums follow where a score is far above
    float by = scale_log2e;                                   // what the scores that have been settled are still to be multiplied by
    auto settle = [&](int t0, bool there0, bool there1) {
        if (!there0 || !there1 || t0 * KV_TILE + STEP > shortest) {
            int seen = limit - t0 * KV_TILE - 4 * hf;         // of the step's positions, less the lane's own first
            asm volatile("" : "+v"(seen));                    // (else the compiler keeps the limit less each of 32 constants in registers through the steps)
#pragma unroll
            for (int tl = 0; tl < 2; ++tl) {
                const int seen_of_tile = (tl ? there1 : there0) ? seen : 0;
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (32 * tl + 16 * ((e >> 2) & 1) + 8 * (e >> 3) + (e & 3) >= seen_of_tile) sacc[tl][e] = -INFINITY;
            }
        }
        float bm = fmaxf(sacc[0][15], sacc[1][15]);           // (the compiler's own: see kv_max3)
#pragma unroll
        for (int e = 0; e < 15; ++e) bm = kv_max3(bm, sacc[0][e], sacc[1][e]);
        const auto other = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, bm), __builtin_bit_cast(uint32_t, bm), false, false);
        bm = kv_max3(__builtin_bit_cast(float, (uint32_t)other[0]), __builtin_bit_cast(float, (uint32_t)other[1]), -INFINITY) * scale_log2e;
        const bool follow = bm > m + KVA_LAG;                 // (the first step with a score above -inf: always)
        if (__builtin_amdgcn_ballot_w64(follow) != 0) {
            const float alpha = follow ? __builtin_amdgcn_exp2f(m - (bm - KVA_BELOW)) : 1.0f;
            l *= alpha;
            m = follow ? bm - KVA_BELOW : m;
            far = far || __builtin_amdgcn_ballot_w64(fabsf(m) >= KVA_FAR && m != -INFINITY) != 0;
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e) oacc[c][e] *= alpha;
        }
        if (__builtin_expect(far, false)) {
#pragma unroll
            for (int tl = 0; tl < 2; ++tl)
#pragma unroll
                for (int e = 0; e < 16; ++e) sacc[tl][e] *= scale_log2e;
        }
        by = far ? 1.f : scale_log2e;
    };
    // The probabilities of eight positions as operand n of four: two fp16 numbers each, the first cut off, together within 2^-21 of them (as in kv_attn_kernel).
    KvPairs pb[2], pr[2];                                     // of operands n % 2
    float below = 0.f;                                        // what is added to a score (a row that has seen nothing: no -inf - -inf)
    auto weigh_pair = [&](int n) {                            // scores 2 n, 2 n + 1 of 32 to probabilities, in place of operand n / 4
        const int tl = n / 8, z = n / 4 % 2, e = n % 4;
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[tl][8 * z + 2 * e], by, below));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[tl][8 * z + 2 * e + 1], by, below));
        l += p0; l += p1;
        asm volatile("" : "+v"(l));                           // (added here, not all of a step's at its end, kept in registers until then)
        const half2_t first = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_pkrtz(p0, p1));
        pb[z].p[e] = first;
        pr[z].p[e] = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_pkrtz(kv_less_low(p0, first), kv_less_high(p1, first)));
    };
    // products n of 4 NC: operand n / NC, components 32 (n % NC) ..
    auto value_operand = [&](const uint8_t *from, int n) { return *reinterpret_cast<const kv_half8 *>(from + ((n / (2 * NC) * 4 + 2 * (n / NC % 2) + hf) * D + 32 * (n % NC) + li) * 16); };
    auto add = [&](kv_half8 a, const KvPairs *p, int n) { oacc[n % NC] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, __builtin_bit_cast(kv_half8, p[n / NC % 2]), oacc[n % NC], 0, 0, 0); };
    // which tiles are there, of the 64 that lanes know and of the 64 before
    uint64_t known = 0, before = 0;
    int window = 0;
    auto there = [&](int t) { return t < tiles && ((t >> 6 == window ? known : before) >> (t & 63) & 1) != 0; };
    auto first_of = [&](int trip) { return 2 * (trip * PG + pg); };
    auto advance = [&](int t0) {
        if (t0 >> 6 != window) {
            window = t0 >> 6;
            find_tiles(t0 & ~63);
            before = known;
            known = __builtin_amdgcn_ballot_w64(my_tile != 0);
        }
    };
    known = __builtin_amdgcn_ballot_w64(my_tile != 0);

    if constexpr (STAGES == 1) {
        uint8_t *k_at = stage, *v_at = stage + KEYS;
        load_keys(first_of(0)); load_values(first_of(0));
        // Half the groups are a phase behind: the two wavefronts of a SIMD are of either half, and one decodes while the other uses the matrix cores.  (512 tokens behind 3888, 32/8 heads x 128, 4 bits:
        // 75.8 us in step, 72.3 so; neighbouring groups in turn 84.8.)
        if (pg >= PG / 2) __syncthreads();
        for (int trip = 0; trip < trips; ++trip) {
            const int t0 = first_of(trip);
            if (trip > 0) __syncthreads();                    // (the last step's operands have been read)
            cut_values(t0);
            decode_keys(k_at); decode_values(v_at);
            advance(first_of(trip + 1));
            load_keys(first_of(trip + 1)); load_values(first_of(trip + 1));
            __syncthreads();
            if (t0 * KV_TILE >= limit_of_wave) continue;
            score(k_at, sacc);
            settle(t0, there(t0), there(t0 + 1));
            below = (m == -INFINITY) ? 0.f : -m;
#pragma unroll
            for (int o = 0; o < 4; ++o) {
#pragma unroll
                for (int n = 4 * o; n < 4 * o + 4; ++n) weigh_pair(n);
#pragma unroll
                for (int n = o * NC; n < (o + 1) * NC; ++n) {
                    const kv_half8 a = value_operand(v_at, n);
                    add(a, pb, n); add(a, pr, n);
                }
            }
        }
        if (pg < PG / 2) __syncthreads();
    } else {
        // Step n's probabilities are made while step n + 1 is scored, and its values added while step n + 2's keys and n + 1's values are decoded: matrix and vector instructions of one
        // wavefront do not wait for one another.  Two places for keys and for values, one barrier a step: what a step overwrites was read before the barrier at the end of the step before.
        // (The first step overwrites the keys that were scored in front of it: a barrier of its own.)
        auto k_at = [&](int trip) { return stage + (trip & 1) * KEYS; };
        auto v_at = [&](int trip) { return stage + (2 + (trip & 1)) * KEYS; };
        load_keys(first_of(0));
        const Keys keys0 = x;
        load_keys(first_of(1));
        load_values(first_of(0));
        const Keys keys1 = x;
        static_cast<Keys &>(x) = keys0;
        decode_keys(k_at(0));
        static_cast<Keys &>(x) = keys1;
        decode_keys(k_at(1));
        load_keys(first_of(2));
        cut_values(first_of(0));
        decode_values(v_at(0));
        load_values(first_of(1));
        __syncthreads();
        score(k_at(0), sacc);
        __syncthreads();
        settle(first_of(0), there(first_of(0)), there(first_of(0) + 1));
        for (int trip = 0; trip < trips; ++trip) {
            kv_float16 next[2];
            clear(next);
            below = (m == -INFINITY) ? 0.f : -m;
            cut_values(first_of(trip + 1));
            // Of 2 NU = 4 NC scores' products NC are ahead of the values' by which the first operand is made; then a value's two products, a score's and the making of a part of the next operand go
            // together.  (Values and keys are read two products ahead; the barriers hold the order, which the scheduler takes apart into matrix and vector instructions.)
            static_assert(NU == 2 * NC, "as many products for the scores of a step as operands of its values");
            kv_half8 ka[2], va[2];
#pragma unroll
            for (int n = 0; n < 2; ++n) { ka[n] = key_operand(k_at(trip + 1), n); va[n] = value_operand(v_at(trip), n); }
            auto score_and_weigh = [&](int n) {
                next[n % 2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ka[n % 2], qb[n / 2], next[n % 2], 0, 0, 0);
                if (n + 2 < 2 * NU) ka[n % 2] = key_operand(k_at(trip + 1), n + 2);
#pragma unroll
                for (int y = 0; y < 4 / NC; ++y) weigh_pair(n * (4 / NC) + y);
            };
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                __builtin_amdgcn_sched_barrier(0);
                score_and_weigh(n);
            }
#pragma unroll
            for (int n = 0; n < 4 * NC; ++n) {
                __builtin_amdgcn_sched_barrier(0);
                add(va[n % 2], pb, n);
                add(va[n % 2], pr, n);
                if (n + 2 < 4 * NC) va[n % 2] = value_operand(v_at(trip), n + 2);
                if (n + NC < 4 * NC) score_and_weigh(n + NC);
                if (n % 2 == 0) {
                    constexpr int EACH = 2 * CHUNKS / (2 * NC) > 0 ? 2 * CHUNKS / (2 * NC) : 1;
#pragma unroll
                    for (int y = 0; y < EACH; ++y) {
                        const int c = n / 2 * EACH + y;
                        if (SPLIT) {
                            if (keys && c < CHUNKS) decode_key(k_at(trip), c / CH, c % CH);
                            if (values && c < CHUNKS) decode_value(v_at(trip + 1), c / CH, c % CH);
                        } else if (c < CHUNKS) {
                            decode_key(k_at(trip), c / CH, c % CH);
                        } else if (c < 2 * CHUNKS) {
                            decode_value(v_at(trip + 1), (c - CHUNKS) / CH, c % CH);
                        }
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            load_values(first_of(trip + 2));
            advance(first_of(trip + 3));
            load_keys(first_of(trip + 3));
            __syncthreads();
            sacc[0] = next[0]; sacc[1] = next[1];
            if (trip + 1 < trips) settle(first_of(trip + 1), there(first_of(trip + 1)), there(first_of(trip + 1) + 1));
        }
    }

    // element 4 y + e of oacc[c] is component 32 c + 8 y + 4 hf + e of row li
    l += __shfl_xor(l, 32);
    if constexpr (PG == 1) {
        if (!real) return;
        const float f = l > 0.f ? 1.f / l : 0.f;              // (nothing seen: zeros; 64 divisions would take as long as two steps)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const half2_t a = {(half_t)(oacc[c][4 * y] * f), (half_t)(oacc[c][4 * y + 1] * f)}, d = {(half_t)(oacc[c][4 * y + 2] * f), (half_t)(oacc[c][4 * y + 3] * f)};
                *reinterpret_cast<kv_u32x2 *>(out + my_out + 32 * c + 8 * y + 4 * hf) = (kv_u32x2){as_u32(a), as_u32(d)};
            }
    } else {
        constexpr int PITCH = D + 4;
        __syncthreads();
        float *mine = reinterpret_cast<float *>(s_mem) + (pg * ROWS + rg * 32 + li) * PITCH + 4 * hf;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int y = 0; y < 4; ++y) *reinterpret_cast<kv_float4 *>(mine + 32 * c + 8 * y) = (kv_float4){oacc[c][4 * y], oacc[c][4 * y + 1], oacc[c][4 * y + 2], oacc[c][4 * y + 3]};
        if (hf == 0) { s_m[pg][rg * 32 + li] = m; s_l[pg][rg * 32 + li] = l; }
        __syncthreads();
        constexpr int QUADS = D / 4;
        for (int n = tid; n < ROWS * QUADS; n += 64 * RG * PG) {
            const int r = n / QUADS, d = n % QUADS * 4, tok = by_group(min(n_rows - 1, r0 + r));
            float M = s_m[0][r];
#pragma unroll
            for (int w = 1; w < PG; ++w) M = fmaxf(M, s_m[w][r]);
            const float to_base = M == -INFINITY ? 0.f : M - KVA_SPARE;
            float L = 0.f;
            kv_float4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < PG; ++w) {
                const float f = __builtin_amdgcn_exp2f(s_m[w][r] - to_base);
                const kv_float4 o = *reinterpret_cast<const kv_float4 *>(reinterpret_cast<const float *>(s_mem) + (w * ROWS + r) * PITCH + d);
                L = __builtin_fmaf(s_l[w][r], f, L);
#pragma unroll
                for (int e = 0; e < 4; ++e) O[e] = __builtin_fmaf(o[e], f, O[e]);
            }
            if (r0 + r >= n_rows || !seq.has_row(tok)) continue;
            const float div = L > 0.f ? L : 1.f;
            const half2_t a = {(half_t)(O[0] / div), (half_t)(O[1] / div)}, c = {(half_t)(O[2] / div), (half_t)(O[3] / div)};
            const int64_t to = (int64_t)(seq.row + tok) * n_heads + head * group + (r0 + r - tok * group);
            *reinterpret_cast<kv_u32x2 *>(out + to * D + d) = (kv_u32x2){as_u32(a), as_u32(c)};
        }
    }
}

// How a call is served.  `rows`: of a workgroup that decodes for many (0: by sixteens).  Us, by sixteens / 64 rows / 128 rows, for so many blocks of 64 rows (graph replay):
//   32/8 heads x 128, 4 bits, one sequence of 4000                   64: 40 / 56 / 102   128: 66 / 59 / 103   256: 103 / 71 / 107  512: 177 / 122 / 122  1024: 291 / 204 / 172
//   ... eight of 250 to 2000 (blocks: if all had as many as most)    128: 24 / 33 / 56   256: 30 / 34 / 57    512: 49 / 50 / 60    1024: 81 / 69 / 70
//   64/8 heads x 128, 8 bits, one of 1000                            64: 13 / 23 / 41    128: 19 / 24 / 43    256: 30 / 26 / 48    512: 49 / 43 / 55
//   71/1 heads x 64, 4 bits, one of 2000                             71: 19 / 23 / 49    142: 27 / 23 / 50
// and of several sequences, by sixteens / 64 rows at 256 blocks and 384:
//   32/8 x 128, 4 bits, two of 4000  74 / 59, 98 / 68    four of 4000  68 / 59, 76 / 62    32/32 x 128, two of 2000  32 / 35, 48 / 44
//   64/8 x 128, 8 bits, four of 1000  20 / 24, 23 / 25   64/8 x 64, three of 2000  27 / 24, 24 / 29   64/64 x 64, two of 300  11 / 10, 13 / 13
// Blocks of 64 rows take as long for one as for 256; those of 128 take two for each compute unit to hide one another's waits.
// A batch with a few long sequences among many short ones (`packed`: fewer than half of n_seqs * max_tokens rows) is numbered by what there is of it, and its sequences of fewer rows
// than `few` go by sixteens beside the others.  (Us, numbered by max_tokens and all in blocks / so, 32/8 heads x 128, 4 bits: 2000 tokens of one sequence and one each of 63 others, all of 2000
// positions, 202 / 101; of 255 others 547 / 168; 8000 tokens and 63 others of 8000 positions 1553 / 850; two of 2000 and five single ones 164 / 137, three and five 206 / 195.  Where most have many tokens it
// is two launches for little or nothing, and left: one of 2000 and one single one 90, where the prompt alone takes 84; but also three of 500 and three single ones of 4000 positions, on the boundary, 107,
// where the prompts alone take 35 and the others 11.)
// `direct`: a line is a workgroup's, without a second launch, of so many wavefronts (0: lines are cut).  Us (graph replay; one page table, lengths an eighth to the whole), cut / direct with four
// wavefronts / with eight, for the longest sequence's positions:
//                                        512               768               1024              2048
//   32/8 heads x 128, 4 bits,  8 lines   8.0 / 6.5 / 6.0   8.3 / 8.5 / 7.6   8.4 / 10.2 / 9.1  8.7 / 16.9 / 14.4
//                             64 lines   8.6 / 7.0 / 6.5   8.6 / 8.7 / 7.9   9.6 / 10.5 / 9.4  12.2 / 17.2 / 14.7
//                            512 lines   18.6 / 10.1 / 12  20.9 / 13.1 / 15  22.8 / 15.6 / 18  31.0 / 26.6 / 27.8
//   32/32 heads x 128, 8 bits, 256       12.6 / 8.7 / 8.3  15.0 / 10.3 / 9.8 16.6 / 12.9 / 12  24.9 / 21.7 / 20.4
//   71/1 heads x 64, 4 bits,   5         7.3 / 5.5 / 5.2   7.3 / 6.6 / 6.0   7.3 / 7.7 / 6.9   7.8 / 12.2 / 11
//                            320         11.9 / 7.8 / 7.8  14.0 / 9.6 / 9.4  15.5 / 10.9 / 10.4 18.3 / 16.9 / 15.9
// The boundaries lie where the longest line alone takes as long as the parts and their merge, and later where there is a line for every compute unit.
constexpr int KVA_SPLIT_WAVES = 4, KVA_FEW = 128;
struct KvPlan {
    int rows, few, direct;
    bool packed, sixteens;
    int64_t blocks, lines;                                    // at most: blocks of `rows` rows of a key/value head if packed; lines of sixteen rows
    KvPlan(const KvView &v, int head_dim, int n_heads)
    {
        const int64_t group = n_heads / v.n_kv_heads, most = v.max_tokens * group, all = v.n_tokens * group, seqs = v.n_seqs, kv = v.n_kv_heads;
        packed = seqs > 1 && 2 * v.n_tokens < seqs * v.max_tokens;
        auto blocks_of = [&](int n) { return packed ? kv * (all / n) : seqs * kv * ((most + n - 1) / n); };
        rows = most < 64 || blocks_of(64) < (seqs == 1 ? 128 : 256) ? 0 : blocks_of(128) >= 512 ? 128 : 64;
        few = rows && packed ? KVA_FEW : 0;
        sixteens = !rows || few;
        blocks = rows ? all / rows + std::min(seqs, all / KVA_FEW) : 0;
        lines = seqs * kv * (((few ? std::min<int64_t>(most, few - 1) : most) + KVA_ROWS - 1) / KVA_ROWS);
        if (packed) lines = std::min(lines, kv * (all / KVA_ROWS + seqs));
        const int64_t tiles = (v.max_seq + KV_TILE - 1) / KV_TILE;
        direct = head_dim == 64 || lines < 256 ? 8 : 4;
        // (beyond 2^30 there are more tiles than the cut counts in 32 bits)
        if (lines * tiles <= (1LL << 30) && v.max_seq > (lines >= 256 ? 2560 : head_dim == 64 ? 1024 : 768)) direct = 0;
    }
};

// The launch of n numbered workgroups: in x and y, because a launch has less than 2^32 threads in either (65535 sequences of 64 key/value heads and 1.1 million rows make 8.4 million lines, 512 threads each).
static dim3 kv_numbered(int64_t n)
{
    const int64_t x = std::min<int64_t>(n, 1 << 22);
    return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}

size_t kv_attn_workspace_bytes(const KvView &v, int head_dim, int n_heads)
{
    const KvPlan plan(v, head_dim, n_heads);
    return plan.sixteens && !plan.direct ? KvPartial::bytes(v.n_seqs, head_dim) : 0;
}

hipError_t launch_kv_attn(int format, int head_dim, const KvView &v, const uint16_t *q, int n_heads, float scale, uint16_t *out, void *workspace, hipStream_t s)
{
    const int group = n_heads / v.n_kv_heads;
    const float scale_log2e = scale * 1.4426950408889634f;
    const KvPlan plan(v, head_dim, n_heads);
    const KvDivide by_group(group), by_heads(v.n_kv_heads);
    if (plan.rows) {
        const int64_t blocks = ((int64_t)v.max_tokens * group + plan.rows - 1) / plan.rows;      // (at most 2^22 rows: 32768)
        const dim3 grid = plan.packed ? kv_numbered(plan.blocks * v.n_kv_heads) : dim3((unsigned)v.n_kv_heads, (unsigned)blocks, (unsigned)v.n_seqs);
        const hipError_t e = for_kv_tile(format, head_dim, [&](auto tag) {
            typedef decltype(tag) T;
            if (plan.rows == 64) hipLaunchKernelGGL((kv_attn_rows_kernel<T, 2, 4, 1>), grid, dim3(512), 0, s, v, q, n_heads, group, plan.few, by_group, scale_log2e, out);
            else hipLaunchKernelGGL((kv_attn_rows_kernel<T, 4, 1, 2>), grid, dim3(256), 0, s, v, q, n_heads, group, plan.few, by_group, scale_log2e, out);
            return hipGetLastError();
        });
        if (e != hipSuccess || !plan.sixteens) return e;
    }
    const int few = plan.few ? plan.few : 0x7fffffff;
    hipError_t e = for_kv_tile(format, head_dim, [&](auto tag) {
        typedef decltype(tag) T;
        const dim3 direct = plan.packed ? kv_numbered(plan.lines) : dim3((unsigned)(plan.lines / v.n_seqs), (unsigned)v.n_seqs);
        const int max_lines = plan.packed || !plan.direct ? (int)plan.lines : 0;
#define IFLOW_KVA_GO(W, DIRECT, GRID) hipLaunchKernelGGL((kv_attn_kernel<T, W, DIRECT>), GRID, dim3(64 * W), 0, s, v, q, n_heads, group, few, max_lines, by_group, by_heads, scale_log2e, out, workspace)
        if (plan.direct == 8) IFLOW_KVA_GO(8, true, direct);
        else if (plan.direct) IFLOW_KVA_GO(4, true, direct);
        else IFLOW_KVA_GO(KVA_SPLIT_WAVES, false, dim3((unsigned)(KVA_PER_CU<T> * KVA_CUS + plan.lines + 1)));
#undef IFLOW_KVA_GO
        return hipGetLastError();
    });
    if (e != hipSuccess || plan.direct) return e;
    // Groups of threads for the results that a long line is likely to have: sequences as long as max_seq, or of several, half of it in the mean.
    const int tiles = (v.max_seq + KV_TILE - 1) / KV_TILE;
    const int64_t part = std::max<int64_t>(2 * KVA_SPLIT_WAVES, plan.lines * tiles / (v.n_seqs > 1 ? 2 : 1) / (4 * KVA_CUS));
    const int groups = (int)((tiles / part + 2 + KVA_MERGE - 1) / KVA_MERGE);
    const dim3 tokens = plan.packed ? dim3((unsigned)std::min<int64_t>(v.n_tokens, 2 * (int64_t)v.n_seqs), (unsigned)n_heads) : dim3((unsigned)n_heads, (unsigned)v.max_tokens, (unsigned)v.n_seqs);
    hipLaunchKernelGGL(kv_attn_merge_kernel, tokens, dim3((unsigned)head_dim, (unsigned)(groups > 8 ? 8 : groups)), 0, s, v, n_heads, group, few, workspace, out);
    return hipGetLastError();
}

}  // namespace iflow
