// The quantized key/value cache as it is written and read back (layout: include/iflow.h).
#include "iflow_kv.h"

namespace iflow {

// Whole rows of results are not kept in the caches.  (Us, kept / not, when both took longer than now: 16001 positions of 8 heads read back 20.0 / 18.7, prompts of 5400 tokens appended 42.9 / 38.4.)
template <typename V> __device__ __forceinline__ void kv_store(uint16_t *to, V x) { __builtin_nontemporal_store(x, reinterpret_cast<V *>(to)); }

// ---- append -------------------------------------------------------------------------------------------------------------------
// Eight lanes share a position of a head; lane s holds components s D/16 .. (s + 1) D/16 - 1 of both halves of the head, so that the pairs of either pairing, and a word of key codes (half
// of one at 64 components in 4 bits), are its own.
template <typename T> constexpr int KV_PART = T::D / 16;      // components of either half that a lane holds, and pairs

// Turns of the pairs of a lane: pair first() + e for e < KV_PART, or in two halves of consecutive ones (adjacent pairing).
struct KvTurns {
    double log2_base;
    double ratio[8];                                          // base^(-2e/d): frequencies of consecutive pairs
    int pair_mode;
};

// sin and cos of an angle of up to 2^21 in fp64: the multiple of pi/2 is taken off in two parts with one rounding each (the first exact but for the rounding of the small
// difference), then Taylor's series to r^15 and r^14, |r| <= pi/4: r^17 / 17! and r^16 / 16!, at most 2^-54.2 and 2^-49.8, are left out.  (The library's functions, which take any angle, were most of the append's time: 157 us of it for
// 5000 tokens of 32/8 heads, one per pair and head.)
__device__ __forceinline__ void kv_sincos(double angle, double *sn, double *cs)
{
    const double turns = rint(angle * 0.63661977236758134308);                       // 2 / pi
    const double r = __builtin_fma(-turns, 6.123233995736766036e-17, __builtin_fma(-turns, 1.57079632679489661923, angle));      // pi / 2 = 1.57.. + 6.1e-17
    const int quadrant = (int)turns;
    const double r2 = r * r;
    double a = -1.0 / 1307674368000.0, b = -1.0 / 87178291200.0;                     // 1/15!, 1/14!
    a = __builtin_fma(a, r2, 1.0 / 6227020800.0);  b = __builtin_fma(b, r2, 1.0 / 479001600.0);
    a = __builtin_fma(a, r2, -1.0 / 39916800.0);   b = __builtin_fma(b, r2, -1.0 / 3628800.0);
    a = __builtin_fma(a, r2, 1.0 / 362880.0);      b = __builtin_fma(b, r2, 1.0 / 40320.0);
    a = __builtin_fma(a, r2, -1.0 / 5040.0);       b = __builtin_fma(b, r2, -1.0 / 720.0);
    a = __builtin_fma(a, r2, 1.0 / 120.0);         b = __builtin_fma(b, r2, 1.0 / 24.0);
    a = __builtin_fma(a, r2, -1.0 / 6.0);          b = __builtin_fma(b, r2, -0.5);
    a = __builtin_fma(a * r2, r, r);               b = __builtin_fma(b, r2, 1.0);
    const double s = quadrant & 1 ? b : a, c = quadrant & 1 ? a : b;
    *sn = quadrant & 2 ? -s : s;
    *cs = (quadrant + 1) & 2 ? -c : c;
}

// fp64 to fp16 with one rounding: cut to 24 bits, the last of them set where something was cut off, so that the second rounding sees what the first one saw
__device__ __forceinline__ half_t kv_half_once(double x)
{
    const float f = (float)x;
    const double back = (double)f;
    uint32_t u = __builtin_bit_cast(uint32_t, f);
    u -= fabs(back) > fabs(x) ? 1u : 0u;
    u |= back != x ? 1u : 0u;
    return (half_t)__builtin_bit_cast(float, u);
}

template <typename T> struct KvLane {
    static constexpr int H = KV_PART<T>, D = T::D;
    float x[2 * H];                                           // components of both halves: fp16 values, a register each (of 16-bit ones, picked by the pairing, the compiler made an array in memory)

    static __device__ __forceinline__ int pair_of(int s, int e, int pair_mode)
    {
        return pair_mode == IFLOW_ROPE_HALVES ? s * H + e : e < H / 2 ? s * H / 2 + e : D / 4 + s * H / 2 + e - H / 2;
    }
    // what is loaded ahead of its use waits packed
    struct Words { uint32_t w[H]; };
    static __device__ __forceinline__ Words load(const uint16_t *row, int s)
    {
        Words n;
#pragma unroll
        for (int half = 0; half < 2; ++half)
            if constexpr (H == 8) *reinterpret_cast<kv_u32x4 *>(n.w + half * (H / 2)) = *reinterpret_cast<const kv_u32x4 *>(row + half * (D / 2) + s * H);
            else *reinterpret_cast<kv_u32x2 *>(n.w + half * (H / 2)) = *reinterpret_cast<const kv_u32x2 *>(row + half * (D / 2) + s * H);
        return n;
    }
    __device__ __forceinline__ explicit KvLane(const Words &n)
    {
#pragma unroll
        for (int e = 0; e < H; ++e) { const half2_t p = as_h2(n.w[e]); x[2 * e] = (float)p.x; x[2 * e + 1] = (float)p.y; }
    }
    __device__ __forceinline__ void store(uint16_t *row, int s) const
    {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t w[H / 2];
#pragma unroll
            for (int e = 0; e < H / 2; ++e) w[e] = as_u32((half2_t){(half_t)x[half * H + 2 * e], (half_t)x[half * H + 2 * e + 1]});
            if constexpr (H == 8) kv_store(row + half * (D / 2) + s * H, *reinterpret_cast<kv_u32x4 *>(w));
            else kv_store(row + half * (D / 2) + s * H, *reinterpret_cast<kv_u32x2 *>(w));
        }
    }
    template <typename Turn> __device__ __forceinline__ void rotate(int pair_mode, Turn turn)
    {
        // Four pairs at a time are rounded by way of 32 bits, which differs from one rounding only where the 32 bits end on a tie of fp16, with twelve zeros: then they are rounded again, with care.
        auto pairs = [&](int e0, auto first, auto second) {
            double sn[4], cs[4];
            float a[4], b[4];
            uint32_t low = 0xFFFFFFFFu;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                turn(e0 + e, &sn[e], &cs[e]);
                const double u = (double)x[first(e0 + e)], w = (double)x[second(e0 + e)];
                a[e] = (float)__builtin_fma(u, cs[e], -(w * sn[e]));
                b[e] = (float)__builtin_fma(u, sn[e], w * cs[e]);
                low = min(low, min(__builtin_bit_cast(uint32_t, a[e]) & 0xFFFu, __builtin_bit_cast(uint32_t, b[e]) & 0xFFFu));
            }
            if (low == 0) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const double u = (double)x[first(e0 + e)], w = (double)x[second(e0 + e)];
                    a[e] = (float)kv_half_once(__builtin_fma(u, cs[e], -(w * sn[e])));
                    b[e] = (float)kv_half_once(__builtin_fma(u, sn[e], w * cs[e]));
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) { x[first(e0 + e)] = (float)(half_t)a[e]; x[second(e0 + e)] = (float)(half_t)b[e]; }
        };
        if (pair_mode == IFLOW_ROPE_HALVES) {
#pragma unroll
            for (int e = 0; e < H; e += 4) pairs(e, [](int n) { return n; }, [](int n) { return H + n; });
        } else {
#pragma unroll
            for (int e = 0; e < H; e += 4) pairs(e, [](int n) { return 2 * n; }, [](int n) { return 2 * n + 1; });
        }
    }
    // The lane's levels, as iflow_quantize_'s kernel finds them (multiplied by the reciprocal, divided where that could decide differently), and the headers of its blocks, by half of the head.
    __device__ __forceinline__ void quantize(uint32_t (&level)[2 * H], uint32_t (&header)[2]) const
    {
        float mn[2], mx[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            mn[half] = mx[half] = x[half * H];
#pragma unroll
            for (int e = 1; e < H; ++e) { mn[half] = fminf(mn[half], x[half * H + e]); mx[half] = fmaxf(mx[half], x[half * H + e]); }
        }
        if (T::NB == 1) { mn[0] = mn[1] = fminf(mn[0], mn[1]); mx[0] = mx[1] = fmaxf(mx[0], mx[1]); }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            // over the eight lanes, or, where a half has two blocks, over four
            float low = mn[half], high = mx[half];
            low = fminf(low, dpp_f32<0xB1, 0xF>(low));  high = fmaxf(high, dpp_f32<0xB1, 0xF>(high));
            low = fminf(low, dpp_f32<0x4E, 0xF>(low));  high = fmaxf(high, dpp_f32<0x4E, 0xF>(high));
            if (T::NB <= 2) { low = fminf(low, dpp_f32<0x141, 0xF>(low)); high = fmaxf(high, dpp_f32<0x141, 0xF>(high)); }
            low += 0.0f; high += 0.0f;                        // a zero of either sign becomes +0
            // the quotient by L as iflow_quantize has it: with 1/L rounded to nearest and one correction by the exact remainder it is the IEEE one (ranges here are multiples of 2^-24 and finite)
            constexpr float y = 1.0f / (float)T::L;
            const float range = high - low, q0 = range * y;
            float step = __builtin_fmaf(__builtin_fmaf(-q0, (float)T::L, range), y, q0);
            step = fabsf(q0) < INFINITY ? step : q0;
            asm("" : "+v"(step));                              // (fused with the conversion it would be rounded once, not twice)
            const half_t sh = (half_t)step, oh = (half_t)low;
            header[half] = as_u16(sh) | (uint32_t)as_u16(oh) << 16;
            const float sc = (float)sh, of = (float)oh, rs = sc == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(sc);
            float edge = 0.f;
#pragma unroll
            for (int e = 0; e < H; ++e) {
                const float f = __builtin_fmaf(x[half * H + e] - of, rs, 0.5f);       // (not negative: the offset is the smallest)
                edge = fmaxf(edge, fabsf(__builtin_amdgcn_fractf(f) - 0.5f));
                level[half * H + e] = min((uint32_t)f, (uint32_t)T::L);
            }
            if (edge > 0.5f - 0.0001220703125f) {
#pragma unroll
                for (int e = 0; e < H; ++e) {
                    const float t = (x[half * H + e] - of) / sc;
                    float r = floorf(t);
                    r = t - r >= 0.5f ? r + 1.0f : r;
                    r = r >= 0.0f ? r : 0.0f;
                    level[half * H + e] = sc == 0.0f ? 0u : (uint32_t)fminf(r, (float)T::L);
                }
            }
        }
    }
    // which lanes hold a block's header, and whose
    static __device__ __forceinline__ bool has_header(int s, int half) { return T::NB == 4 ? (s & 3) == 0 : s == 0 && (T::NB == 2 || half == 0); }
    static __device__ __forceinline__ int block_of(int s, int half) { return T::NB == 1 ? 0 : T::NB == 2 ? half : half * 2 + (s >> 2); }
    // words of key codes of one half: put(first component, word)
    template <typename Put> static __device__ __forceinline__ void key_words(const uint32_t *level, int s, int half, Put put)
    {
        const int c = half * (D / 2) + s * H;
        if constexpr (T::BITS == 8) {
#pragma unroll
            for (int e = 0; e < H; e += 4) put(c + e, level[e] | level[e + 1] << 8 | level[e + 2] << 16 | level[e + 3] << 24);
        } else if constexpr (H == 8) {
            put(c, level[0] | level[2] << 4 | level[4] << 8 | level[6] << 12 | level[1] << 16 | level[3] << 20 | level[5] << 24 | level[7] << 28);
        } else {
            uint32_t part = level[0] | level[2] << 4 | level[1] << 16 | level[3] << 20;
            if (s & 1) part <<= 8;
            const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)part, 0xB1, 0xF, 0xF, true);
            if (!(s & 1)) put(c, part | other);
        }
    }
};

// Workgroup x of a head runs for tile x % tiles_per_seq of sequence x / tiles_per_seq, or, FIND, for the x-th, the x + grid-th, .. of the tiles that there are.
template <bool FIND, typename Do> __device__ __forceinline__ void kv_each_tile(const KvView &v, int tiles_per_seq, Do run)
{
    if constexpr (FIND) {
        for (int x = blockIdx.x, b, nth; nth = x, kv_find(v, nth, b, [](const KvSequence &seq) { return seq.tiles(); }); x += gridDim.x) {
            int tid = threadIdx.x;
            asm volatile("" : "+v"(tid));                     // (made anew for every tile: what follows from it is not kept in registers from one to the next)
            run(b, nth, tid);
            __syncthreads();                                  // (what run() has in LDS has been read)
        }
    } else {
        const int b = blockIdx.x / (unsigned)tiles_per_seq;
        run(b, (int)blockIdx.x - b * tiles_per_seq, (int)threadIdx.x);
    }
}

// One token per sequence: a workgroup takes 32 rows of one token, keys' heads first, then values', then queries'.  Bound by the latency of what follows on one another: the sequence's length, its page, the
// row, and for values the words that eight positions share (read, changed, written by one lane; requested as soon as the page is known).
template <typename T>
__global__ __launch_bounds__(256) void kv_append_token_kernel(KvView v, const uint16_t *q, const uint16_t *__restrict__ k_new, const uint16_t *__restrict__ v_new, int n_heads, KvTurns turns,
                                                              uint16_t *q_out)
{
    constexpr int D = T::D, H = KV_PART<T>;
    __shared__ double s_turn[2][D / 2];
    __shared__ uint8_t s_level[32][D];
    const int tid = threadIdx.x, r = tid >> 3, s = tid & 7, b = blockIdx.x;
    const KvSequence seq(v, b);
    if (!seq.has(0)) return;
    const int line = blockIdx.y * 32 + r, kind = line < v.n_kv_heads ? 0 : line < 2 * v.n_kv_heads ? 1 : line < 2 * v.n_kv_heads + n_heads ? 2 : 3;
    const int head = line - min(kind, 2) * v.n_kv_heads, heads = kind >= 2 ? n_heads : v.n_kv_heads;
    // (lines past the last: the last query head again, not stored)
    const typename KvLane<T>::Words words = KvLane<T>::load((kind == 0 ? k_new : kind == 1 ? v_new : q) + ((int64_t)seq.row * heads + (kind == 3 ? n_heads - 1 : head)) * D, s);
    uint8_t *tile = kind < 2 ? kv_tile_at(v, b, head, (int)(seq.position / KV_TILE), T::BYTES) : nullptr;
    const int at = (int)(seq.position % KV_TILE), g = (at & 15) >> 2, k = (at >> 4) * 4 + (at & 3);
    // the values' pieces: a lane takes those of components s and s + 8 of every sixteen
    kv_u32x4 old[T::PIECES][2];
    if (kind == 1 && tile) {
#pragma unroll
        for (int n = 0; n < T::PIECES; ++n)
#pragma unroll
            for (int u = 0; u < 2; ++u) old[n][u] = *reinterpret_cast<const kv_u32x4 *>(tile + T::V_AT + (n * 64 + g * 16 + s + 8 * u) * 16);
    }
    if (tid < D / 2) kv_sincos((double)seq.position * exp2(-(2.0 * tid / D) * turns.log2_base), &s_turn[0][tid], &s_turn[1][tid]);
    __syncthreads();
    KvLane<T> lane(words);
    if (kind != 1) {
        lane.rotate(turns.pair_mode, [&](int e, double *sn, double *cs) {
            const int pair = KvLane<T>::pair_of(s, e, turns.pair_mode);
            *sn = s_turn[0][pair]; *cs = s_turn[1][pair];
        });
    }
    if (kind == 2) lane.store(q_out + ((int64_t)seq.row * heads + head) * D, s);
    uint32_t level[2 * H], header[2];
    if (kind < 2) {
        lane.quantize(level, header);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (tile && KvLane<T>::has_header(s, half)) {
                const int block = KvLane<T>::block_of(s, half);
                if (kind == 0) {
                    *reinterpret_cast<uint32_t *>(tile + T::KH_AT + 2 * kv_key_header(at, block)) = header[half];
                } else {
                    uint16_t *to = reinterpret_cast<uint16_t *>(tile + T::VH_AT) + kv_value_header(at, block);
                    to[0] = (uint16_t)header[half]; to[8] = (uint16_t)(header[half] >> 16);
                }
            }
            if (kind == 0) {
                KvLane<T>::key_words(level + half * H, s, half, [&](int c, uint32_t w) { if (tile) reinterpret_cast<uint32_t *>(tile)[kv_key_word<T>(at, c)] = w; });
            } else {
#pragma unroll
                for (int e = 0; e < H; ++e) s_level[r][half * (D / 2) + s * H + e] = (uint8_t)level[half * H + e];
            }
        }
    }
    __syncthreads();
    if (kind == 1 && tile) {
        // word w of piece n holds, of component i, element k of the eight positions in 4 bits: components 64 n + 16 w + i; in 8 bits four positions to a word, two words to a component
#pragma unroll
        for (int n = 0; n < T::PIECES; ++n)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int i = s + 8 * u;
                kv_u32x4 x = old[n][u];
                if constexpr (T::BITS == 4) {
                    const int shift = (k >> 1) * 4 + (k & 1) * 16;
#pragma unroll
                    for (int w = 0; w < 4; ++w) x[w] = (x[w] & ~(15u << shift)) | (uint32_t)s_level[r][64 * n + 16 * w + i] << shift;
                } else {
                    const int shift = (k & 3) * 8;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t changed = (x[w] & ~(255u << shift)) | (uint32_t)s_level[r][32 * n + 16 * (w >> 1) + i] << shift;
                        x[w] = (w & 1) == (k >> 2) ? changed : x[w];
                    }
                }
                *reinterpret_cast<kv_u32x4 *>(tile + T::V_AT + (n * 64 + g * 16 + i) * 16) = x;
            }
    }
}

// Any number of tokens: a workgroup takes the new positions of one tile, of one key/value head or of several query heads.  A tile is put together in LDS, over what it held where
// positions of it are older, and leaves in 16-byte pieces; nobody else writes it in this call.
template <typename T>
__device__ __forceinline__ void kv_append_tile(const KvView &v, int b, int nth, int tid, const uint16_t *q, const uint16_t *__restrict__ k_new, const uint16_t *__restrict__ v_new, int n_heads,
                                               const KvTurns &turns, uint16_t *q_out, int heads_per_group)
{
    constexpr int D = T::D, H = KV_PART<T>;
    __shared__ __align__(16) uint32_t s_image[T::BYTES / 4];
    __shared__ __align__(16) uint8_t s_level[KV_TILE][D];
    const int r = tid >> 3, s = tid & 7;
    const KvSequence seq(v, b);
    const int t = seq.first_tile() + nth, first_token = (int)((uint32_t)t * KV_TILE - (uint32_t)seq.position), token = first_token + r;
    const int64_t row = (int64_t)seq.row + token;
    const uint32_t fresh = (uint32_t)__builtin_amdgcn_ballot_w64(seq.has(first_token + (tid & 31)));       // positions of the tile that are new
    if (fresh == 0) return;
    const bool mine = fresh >> r & 1;

    const double position = (double)(seq.position + token), f0 = exp2(-(2.0 * KvLane<T>::pair_of(s, 0, turns.pair_mode) / D) * turns.log2_base);
    const double f1 = turns.pair_mode == IFLOW_ROPE_HALVES ? f0 * turns.ratio[H / 2] : exp2(-(2.0 * KvLane<T>::pair_of(s, H / 2, turns.pair_mode) / D) * turns.log2_base);
    auto turn = [&](int e, double *sn, double *cs) { kv_sincos(position * ((e < H / 2 ? f0 : f1) * turns.ratio[e % (H / 2)]), sn, cs); };

    // Query heads' workgroups stand evenly among the keys' and values': those wait for memory, these for instructions.
    const int groups = gridDim.y - v.n_kv_heads, group = blockIdx.y * groups / gridDim.y, next_group = (blockIdx.y + 1) * groups / gridDim.y;
    if (next_group > group) {                                 // query heads
        const int h0 = group * heads_per_group, h1 = min(n_heads, h0 + heads_per_group);
        if (!mine) return;
        typename KvLane<T>::Words next = KvLane<T>::load(q + (row * n_heads + h0) * D, s);
        double sn[H], cs[H];
#pragma unroll
        for (int e = 0; e < H; ++e) turn(e, &sn[e], &cs[e]);
        for (int h = h0; h < h1; ++h) {
            KvLane<T> lane(next);
            if (h + 1 < h1) next = KvLane<T>::load(q + (row * n_heads + h + 1) * D, s);
            lane.rotate(turns.pair_mode, [&](int e, double *a, double *c) { *a = sn[e]; *c = cs[e]; });
            lane.store(q_out + (row * n_heads + h) * D, s);
        }
        return;
    }
    const int head = blockIdx.y - group;
    // (a position that is new is in 0 .. max_seq - 1: no other tile is looked up)
    uint8_t *tile = kv_tile_at(v, b, head, (int)t, T::BYTES);
    if (!tile) return;
    typename KvLane<T>::Words key_words = {}, value_words = {};
    if (mine) {
        key_words = KvLane<T>::load(k_new + (row * v.n_kv_heads + head) * D, s);
        value_words = KvLane<T>::load(v_new + (row * v.n_kv_heads + head) * D, s);
    }
    if (fresh != 0xFFFFFFFFu) {
        for (int n = tid; n < T::BYTES / 16; n += 256) reinterpret_cast<kv_u32x4 *>(s_image)[n] = reinterpret_cast<const kv_u32x4 *>(tile)[n];
        __syncthreads();
    }
    KvLane<T> key(key_words);
    key.rotate(turns.pair_mode, turn);
    uint32_t level[2 * H], header[2];
    key.quantize(level, header);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if (mine && KvLane<T>::has_header(s, half)) s_image[T::KH_AT / 4 + kv_key_header(r, KvLane<T>::block_of(s, half)) / 2] = header[half];
        KvLane<T>::key_words(level + half * H, s, half, [&](int c, uint32_t w) { if (mine) s_image[kv_key_word<T>(r, c)] = w; });
    }
    KvLane<T>(value_words).quantize(level, header);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if (mine && KvLane<T>::has_header(s, half)) {
            uint16_t *to = reinterpret_cast<uint16_t *>(s_image) + T::VH_AT / 2 + kv_value_header(r, KvLane<T>::block_of(s, half));
            to[0] = (uint16_t)header[half]; to[8] = (uint16_t)(header[half] >> 16);
        }
#pragma unroll
        for (int e = 0; e < H; e += 4) {
            const uint32_t *l = level + half * H + e;
            *reinterpret_cast<uint32_t *>(&s_level[r][half * (D / 2) + s * H + e]) = l[0] | l[1] << 8 | l[2] << 16 | l[3] << 24;
        }
    }
    __syncthreads();
    // values' words: four components at once, a byte each, of the eight (four) positions of a word; then bytes to words
    constexpr int WORDS = 8 / T::PER_WORD;                    // of the eight positions of g
    for (int n = tid; n < 4 * WORDS * (D / 4); n += 256) {
        const int c = n % (D / 4) * 4, x = n / (D / 4), g = x / WORDS, k0 = x % WORDS * T::PER_WORD;
        uint32_t l[T::PER_WORD], keep = 0;
#pragma unroll
        for (int e = 0; e < T::PER_WORD; ++e) {
            const int p = kv_value_position(g, k0 + e);
            l[e] = *reinterpret_cast<const uint32_t *>(&s_level[p][c]);
            if (!(fresh >> p & 1)) keep |= (uint32_t)T::L << (T::BITS == 8 ? 8 * e : (e >> 1) * 4 + (e & 1) * 16);
        }
        uint32_t byte[4];                                     // byte j of component c + i's word is byte i of byte[j]
        if constexpr (T::BITS == 4) {
            byte[0] = l[0] | l[2] << 4; byte[1] = l[4] | l[6] << 4; byte[2] = l[1] | l[3] << 4; byte[3] = l[5] | l[7] << 4;
        } else {
            byte[0] = l[0]; byte[1] = l[1]; byte[2] = l[2]; byte[3] = l[3];
        }
        const uint32_t a = __builtin_amdgcn_perm(byte[1], byte[0], 0x05010400u), d = __builtin_amdgcn_perm(byte[3], byte[2], 0x05010400u);       // bytes of components 0, 1
        const uint32_t e = __builtin_amdgcn_perm(byte[1], byte[0], 0x07030602u), f = __builtin_amdgcn_perm(byte[3], byte[2], 0x07030602u);       // 2, 3
        const uint32_t w[4] = {(a & 0xFFFFu) | d << 16, a >> 16 | (d & 0xFFFF0000u), (e & 0xFFFFu) | f << 16, e >> 16 | (f & 0xFFFF0000u)};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t *to = s_image + T::V_AT / 4 + kv_value_word<T>(g, k0, c + i);
            *to = keep ? (w[i] & ~keep) | (*to & keep) : w[i];
        }
    }
    __syncthreads();
    for (int n = tid; n < T::BYTES / 16; n += 256) reinterpret_cast<kv_u32x4 *>(tile)[n] = reinterpret_cast<const kv_u32x4 *>(s_image)[n];
}

template <typename T, bool FIND>
__global__ __launch_bounds__(256) void kv_append_tile_kernel(KvView v, const uint16_t *q, const uint16_t *__restrict__ k_new, const uint16_t *__restrict__ v_new, int n_heads, KvTurns turns,
                                                             uint16_t *q_out, int tiles_per_seq, int heads_per_group)
{
    kv_each_tile<FIND>(v, tiles_per_seq, [&](int b, int nth, int tid) { kv_append_tile<T>(v, b, nth, tid, q, k_new, v_new, n_heads, turns, q_out, heads_per_group); });
}

// ---- read back ----------------------------------------------------------------------------------------------------------------
// A workgroup takes a tile of a head; bound by memory where there are many (16001 positions of 8 heads, 84 MB: 15.4 us), else by length -> page -> codes.  (Us, values asked for behind the keys' results /
// all at first: prompts of 5400 tokens 8.0 / 7.6.  Whether any row is the batch's was a loop over 32 positions before, 16001 positions 18.6.)
template <typename T>
__device__ __forceinline__ void kv_read_tile(const KvView &v, int b, int nth, int tid, uint16_t *__restrict__ k_out, uint16_t *__restrict__ v_out)
{
    constexpr int D = T::D, ROW = D + 8;
    const KvMagic magic;
    __shared__ __align__(16) uint16_t s_value[KV_TILE][ROW];
    const int head = blockIdx.y;
    const KvSequence seq(v, b);
    const int t = seq.first_tile() + nth, first_token = (int)((uint32_t)t * KV_TILE - (uint32_t)seq.position);
    auto has = [&](int p) { return seq.has_row(first_token + p); };
    if (__builtin_amdgcn_ballot_w64(has(tid & (KV_TILE - 1))) == 0) return;
    const uint8_t *tile = t >= 0 && t <= (v.max_seq - 1) / KV_TILE ? kv_tile_at(v, b, head, (int)t, T::BYTES) : nullptr;
    auto there = [&](int p) { return tile && t * KV_TILE + p < v.max_seq; };
    auto out_at = [&](int p, int c) { return (((int64_t)seq.row + first_token + p) * v.n_kv_heads + head) * D + c; };
    // Eight components of a position's key, and one component of eight positions' values, N times for each thread; all of it is asked for before any of it is used.
    constexpr int N = KV_TILE * D / 8 / 256, W = 8 / T::PER_WORD;
    static_assert(N * 256 == 4 * D, "as many runs of eight positions as of eight components");
    uint32_t key[N][W], key_header[N], value[N][W];
    kv_u32x4 scales[N], offsets[N];
    if (tile) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int n = tid + 256 * i, p = n / (D / 8), c = n % (D / 8) * 8, vc = n % D, g = n / D;
            const uint32_t *k_at = reinterpret_cast<const uint32_t *>(tile) + kv_key_word<T>(p, c), *v_at = reinterpret_cast<const uint32_t *>(tile + T::V_AT) + kv_value_word<T>(g, 0, vc);
#pragma unroll
            for (int x = 0; x < W; ++x) { key[i][x] = k_at[x]; value[i][x] = v_at[x]; }
            key_header[i] = *reinterpret_cast<const uint32_t *>(tile + T::KH_AT + 2 * kv_key_header(p, c / T::BLOCK));
            const kv_u32x4 *header = reinterpret_cast<const kv_u32x4 *>(tile + T::VH_AT + 2 * kv_value_header(4 * g, vc / T::BLOCK));
            scales[i] = header[0]; offsets[i] = header[1];
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int n = tid + 256 * i, p = n / (D / 8), c = n % (D / 8) * 8;
        if (!has(p)) continue;
        kv_u32x4 w = {0u, 0u, 0u, 0u};
        if (there(p)) {
            const KvPairs level = kv_levels<T::BITS>(key[i], magic);
            const half2_t pair = as_h2(key_header[i]);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = as_u32(kv_value(level.p[e], (half2_t){pair.x, pair.x}, (half2_t){pair.y, pair.y}));
        }
        kv_store(k_out + out_at(p, c), w);
    }
    if (tile) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int n = tid + 256 * i, c = n % D, g = n / D;
            const KvPairs level = kv_levels<T::BITS>(value[i], magic);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const half2_t x = kv_value(level.p[e], as_h2(scales[i][e]), as_h2(offsets[i][e]));
                s_value[kv_value_position(g, 2 * e)][c] = as_u16(x.x);
                s_value[kv_value_position(g, 2 * e + 1)][c] = as_u16(x.y);
            }
        }
    }
    __syncthreads();
    for (int n = tid; n < KV_TILE * D / 8; n += 256) {
        const int p = n / (D / 8), c = n % (D / 8) * 8;
        if (!has(p)) continue;
        kv_u32x4 w = {0u, 0u, 0u, 0u};
        if (there(p)) w = *reinterpret_cast<const kv_u32x4 *>(&s_value[p][c]);
        kv_store(v_out + out_at(p, c), w);
    }
}

template <typename T, bool FIND>
__global__ __launch_bounds__(256) void kv_read_kernel(KvView v, uint16_t *__restrict__ k_out, uint16_t *__restrict__ v_out, int tiles_per_seq)
{
    kv_each_tile<FIND>(v, tiles_per_seq, [&](int b, int nth, int tid) { kv_read_tile<T>(v, b, nth, tid, k_out, v_out); });
}

// The tiles of a call: as many for each sequence as max_tokens can touch, wherever they begin, or, if the batch's rows touch fewer together, as many as those, to be found by the kernel.
// (Us, one way / the other: 2000 tokens of one sequence and one each of 63 others appended 193 / 27, of 255 others 693 / 58: 196 thousand workgroups, the few with work of the others all on one die; prompts of
// 5400 tokens, the longest 2000 of four, 37.5 / 34; 12 sequences of up to 777 positions read back 9.9 / 9.2.)
struct KvGrid { int64_t all; int per_seq; };
static KvGrid kv_grid(const KvView &v)
{
    const int64_t per_seq = (v.max_tokens + 2 * KV_TILE - 2) / KV_TILE, all = per_seq * v.n_seqs, rows = v.n_tokens / KV_TILE + 2 * v.n_seqs;
    return v.n_seqs > 1 && all > rows ? KvGrid{rows, 0} : KvGrid{all, (int)per_seq};
}

hipError_t launch_kv_append(int format, int head_dim, const KvView &v, const uint16_t *q, const uint16_t *k_new, const uint16_t *v_new, int n_heads, double base, int pair_mode,
                            uint16_t *q_out, hipStream_t s)
{
    const KvGrid grid = kv_grid(v);
    KvTurns turns;
    turns.log2_base = log2(base);
    turns.pair_mode = pair_mode;
    for (int e = 0; e < 8; ++e) turns.ratio[e] = exp2(-(2.0 * e / head_dim) * turns.log2_base);
    // query heads of a workgroup: as many as leave a thousand workgroups, up to eight
    const int64_t per = grid.all * n_heads / 1024;
    const int heads_per_group = per < 1 ? 1 : per > 8 ? 8 : (int)per;
    return for_kv_tile(format, head_dim, [&](auto tag) {
        typedef decltype(tag) T;
        if (v.max_tokens == 1) {
            hipLaunchKernelGGL((kv_append_token_kernel<T>), dim3((unsigned)v.n_seqs, (unsigned)((2 * v.n_kv_heads + n_heads + 31) / 32)), dim3(256), 0, s, v, q, k_new, v_new, n_heads, turns,
                               q_out);
        } else {
            const dim3 blocks((unsigned)grid.all, (unsigned)(v.n_kv_heads + (n_heads + heads_per_group - 1) / heads_per_group));
#define IFLOW_KV_GO(FIND) hipLaunchKernelGGL((kv_append_tile_kernel<T, FIND>), blocks, dim3(256), 0, s, v, q, k_new, v_new, n_heads, turns, q_out, grid.per_seq, heads_per_group)
            if (grid.per_seq) IFLOW_KV_GO(false);
            else IFLOW_KV_GO(true);
#undef IFLOW_KV_GO
        }
        return hipGetLastError();
    });
}

hipError_t launch_kv_read(int format, int head_dim, const KvView &v, uint16_t *k_out, uint16_t *v_out, hipStream_t s)
{
    const KvGrid grid = kv_grid(v);
    return for_kv_tile(format, head_dim, [&](auto tag) {
        typedef decltype(tag) T;
        const dim3 blocks((unsigned)grid.all, (unsigned)v.n_kv_heads);
        if (grid.per_seq) hipLaunchKernelGGL((kv_read_kernel<T, false>), blocks, dim3(256), 0, s, v, k_out, v_out, grid.per_seq);
        else hipLaunchKernelGGL((kv_read_kernel<T, true>), blocks, dim3(256), 0, s, v, k_out, v_out, 0);
        return hipGetLastError();
    });
}

int kv_tile_bytes(int format, int head_dim)
{
    int bytes = 0;
    for_kv_tile(format, head_dim, [&](auto tag) { bytes = decltype(tag)::BYTES; return hipSuccess; });
    return bytes;
}

}  // namespace iflow
