// The quantized key/value cache as it is written and read back (layout: include/iflow.h).
#include "iflow_kv.h"

namespace iflow {

// the block's extremes over the eight lanes of a position (or the four of a quad)
template <bool EIGHT> __device__ __forceinline__ float kv_min(float v)
{
    v = fminf(v, dpp_f32<0xB1, 0xF>(v));
    v = fminf(v, dpp_f32<0x4E, 0xF>(v));
    if (EIGHT) v = fminf(v, dpp_f32<0x141, 0xF>(v));
    return v;
}
template <bool EIGHT> __device__ __forceinline__ float kv_max(float v)
{
    v = fmaxf(v, dpp_f32<0xB1, 0xF>(v));
    v = fmaxf(v, dpp_f32<0x4E, 0xF>(v));
    if (EIGHT) v = fmaxf(v, dpp_f32<0x141, 0xF>(v));
    return v;
}

// ---- append -------------------------------------------------------------------------------------------------------------------
// One workgroup per sequence, tile of positions and key/value head or query heads.  Eight lanes share a position; a lane holds components
// s D/16 .. of both halves of the head, so that the pairs of either pairing are its own.
template <typename T>
__global__ __launch_bounds__(256) void kv_append_kernel(KvView v, const uint16_t *q, const uint16_t *__restrict__ k_new, const uint16_t *__restrict__ v_new, int n_heads,
                                                        double log2_base, int pair_mode, uint16_t *q_out, int tiles_per_seq)
{
    constexpr int D = T::D, H = D / 16;                       // H: components of either half that a lane holds
    __shared__ uint8_t s_level[2][KV_TILE][D];
    const int tid = threadIdx.x, r = tid >> 3, s = tid & 7;
    const int b = blockIdx.x / tiles_per_seq;
    const KvSequence seq(v, b);
    const int64_t t = seq.first_tile() + (blockIdx.x - b * tiles_per_seq);
    const int64_t token = t * KV_TILE + r - seq.position;
    const bool mine = seq.has(token);
    const int64_t row = seq.row + token;

    double sn[H], cs[H];
#pragma unroll
    for (int e = 0; e < H; ++e) {
        const int pair = pair_mode == IFLOW_ROPE_HALVES ? s * H + e : e < H / 2 ? s * H / 2 + e : D / 4 + s * H / 2 + e - H / 2;
        sincos((double)(seq.position + token) * exp2(-(2.0 * pair / D) * log2_base), &sn[e], &cs[e]);
    }
    auto load = [&](const uint16_t *from, half_t (&x)[2 * H]) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t w[H / 2];
            if constexpr (H == 8) *reinterpret_cast<kv_u32x4 *>(w) = *reinterpret_cast<const kv_u32x4 *>(from + half * (D / 2) + s * H);
            else *reinterpret_cast<kv_u32x2 *>(w) = *reinterpret_cast<const kv_u32x2 *>(from + half * (D / 2) + s * H);
#pragma unroll
            for (int e = 0; e < H / 2; ++e) { const half2_t p = as_h2(w[e]); x[half * H + 2 * e] = p.x; x[half * H + 2 * e + 1] = p.y; }
        }
    };
    auto rotate = [&](half_t (&x)[2 * H]) {
#pragma unroll
        for (int e = 0; e < H; ++e) {
            const int ia = pair_mode == IFLOW_ROPE_HALVES ? e : 2 * e, ib = pair_mode == IFLOW_ROPE_HALVES ? H + e : 2 * e + 1;
            const double a = (double)(float)x[ia], c = (double)(float)x[ib];
            x[ia] = (half_t)(a * cs[e] - c * sn[e]);
            x[ib] = (half_t)(a * sn[e] + c * cs[e]);
        }
    };

    if ((int)blockIdx.y >= v.n_kv_heads) {                    // a query head
        const int h = blockIdx.y - v.n_kv_heads;
        if (!mine) return;
        half_t x[2 * H];
        load(q + (row * n_heads + h) * D, x);
        rotate(x);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t w[H / 2];
#pragma unroll
            for (int e = 0; e < H / 2; ++e) w[e] = as_u32((half2_t){x[half * H + 2 * e], x[half * H + 2 * e + 1]});
            uint16_t *to = q_out + (row * n_heads + h) * D + half * (D / 2) + s * H;
            if constexpr (H == 8) *reinterpret_cast<kv_u32x4 *>(to) = *reinterpret_cast<kv_u32x4 *>(w);
            else *reinterpret_cast<kv_u32x2 *>(to) = *reinterpret_cast<kv_u32x2 *>(w);
        }
        return;
    }
    const int head = blockIdx.y;
    // (t of a tile with a token is in 0 .. max_seq / 32: no other is looked up)
    const int64_t first_token = t * KV_TILE - seq.position;
    bool any = false;
    for (int i = 0; i < KV_TILE; ++i) any |= seq.has(first_token + i);
    if (!any) return;
    uint8_t *tile = kv_tile_at(v, b, head, (int)t, T::BYTES);
    if (!tile) return;

    for (int which = 0; which < 2; ++which) {
        half_t x[2 * H];
        if (mine) {
            load((which ? v_new : k_new) + (row * v.n_kv_heads + head) * D, x);
            if (!which) rotate(x);
        } else {
#pragma unroll
            for (int e = 0; e < 2 * H; ++e) x[e] = (half_t)0.f;
        }
        float mn[2], mx[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            mn[half] = mx[half] = (float)x[half * H];
#pragma unroll
            for (int e = 1; e < H; ++e) { mn[half] = fminf(mn[half], (float)x[half * H + e]); mx[half] = fmaxf(mx[half], (float)x[half * H + e]); }
        }
        if (T::NB == 1) { mn[0] = mn[1] = fminf(mn[0], mn[1]); mx[0] = mx[1] = fmaxf(mx[0], mx[1]); }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            constexpr bool EIGHT = T::NB <= 2;                // a half of the head, or (128 components in blocks of 32) a quarter of it
            const float low = kv_min<EIGHT>(mn[half]) + 0.0f, high = kv_max<EIGHT>(mx[half]) + 0.0f;
            const half_t sh = (half_t)((high - low) / (float)T::L), oh = (half_t)low;
            const float sc = (float)sh, of = (float)oh;
#pragma unroll
            for (int e = 0; e < H; ++e) {
                const float quotient = ((float)x[half * H + e] - of) / sc;
                float f = floorf(quotient);
                f = quotient - f >= 0.5f ? f + 1.0f : f;
                f = f >= 0.0f ? f : 0.0f;
                f = fminf(f, (float)T::L);
                s_level[which][r][half * (D / 2) + s * H + e] = sc == 0.0f ? 0 : (uint8_t)f;
            }
            const int block = T::NB == 1 ? 0 : T::NB == 2 ? half : half * 2 + (s >> 2);
            const bool writes = mine && (T::NB == 4 ? (s & 3) == 0 : s == 0) && (T::NB > 1 || half == 0);
            if (writes) {
                uint16_t *headers = reinterpret_cast<uint16_t *>(tile + (which ? T::VH_AT : T::KH_AT));
                const int at = which ? kv_value_header(r, block) : kv_key_header(r, block);
                headers[at] = as_u16(sh);
                headers[at + (which ? 8 : 1)] = as_u16(oh);
            }
        }
    }
    __syncthreads();
    auto is_new = [&](int p) { return seq.has(first_token + p); };
    auto place = [](int e) { return T::BITS == 8 ? 8 * e : (e >> 1) * 4 + (e & 1) * 16; };
    for (int n = tid; n < KV_TILE * D / T::PER_WORD; n += 256) {
        // keys: a word is PER_WORD components of one position
        {
            const int p = n / (D / T::PER_WORD), c = n % (D / T::PER_WORD) * T::PER_WORD;
            if (is_new(p)) {
                uint32_t w = 0;
#pragma unroll
                for (int e = 0; e < T::PER_WORD; ++e) w |= (uint32_t)s_level[0][p][c + e] << place(e);
                reinterpret_cast<uint32_t *>(tile)[kv_key_word<T>(p, c)] = w;
            }
        }
        // values: PER_WORD positions of one component, of which some may be older
        {
            const int c = n % D, x = n / D, g = x / (8 / T::PER_WORD), k = x % (8 / T::PER_WORD) * T::PER_WORD;
            uint32_t w = 0, keep = 0;
#pragma unroll
            for (int e = 0; e < T::PER_WORD; ++e) {
                const int p = kv_value_position(g, k + e);
                if (is_new(p)) w |= (uint32_t)s_level[1][p][c] << place(e);
                else keep |= (uint32_t)T::L << place(e);
            }
            if (keep != 0xFFFFFFFFu) {
                uint32_t *at = reinterpret_cast<uint32_t *>(tile + T::V_AT) + kv_value_word<T>(g, k, c);
                *at = keep ? w | (*at & keep) : w;
            }
        }
    }
}

// ---- read back ----------------------------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void kv_read_kernel(KvView v, uint16_t *__restrict__ k_out, uint16_t *__restrict__ v_out, int tiles_per_seq)
{
    constexpr int D = T::D, ROW = D + 8;
    __shared__ __align__(16) uint16_t s_value[KV_TILE][ROW];
    const int tid = threadIdx.x, head = blockIdx.y;
    const int b = blockIdx.x / tiles_per_seq;
    const KvSequence seq(v, b);
    const int64_t t = seq.first_tile() + (blockIdx.x - b * tiles_per_seq);
    const int64_t first_token = t * KV_TILE - seq.position;
    auto has = [&](int p) { return seq.has_row(first_token + p); };
    bool any = false;
    for (int i = 0; i < KV_TILE; ++i) any |= has(i);
    if (!any) return;
    const uint8_t *tile = t >= 0 && t * KV_TILE < v.max_seq ? kv_tile_at(v, b, head, (int)t, T::BYTES) : nullptr;
    auto there = [&](int p) { return tile && t * KV_TILE + p < v.max_seq; };
    auto out_at = [&](int p, int c) { return ((seq.row + first_token + p) * v.n_kv_heads + head) * D + c; };
    const uint16_t *kh = reinterpret_cast<const uint16_t *>(tile + T::KH_AT), *vh = reinterpret_cast<const uint16_t *>(tile + T::VH_AT);
    for (int n = tid; n < KV_TILE * D / 8; n += 256) {
        const int p = n / (D / 8), c = n % (D / 8) * 8;
        if (!has(p)) continue;
        kv_u32x4 w = {0u, 0u, 0u, 0u};
        if (there(p)) {
            const KvPairs level = kv_levels<T::BITS>(reinterpret_cast<const uint32_t *>(tile) + kv_key_word<T>(p, c));
            const int at = kv_key_header(p, c / T::BLOCK);
            const half_t sc = as_h(kh[at]), of = as_h(kh[at + 1]);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = as_u32(kv_value(level.p[e], (half2_t){sc, sc}, (half2_t){of, of}));
        }
        *reinterpret_cast<kv_u32x4 *>(k_out + out_at(p, c)) = w;
    }
    if (tile) {
        for (int n = tid; n < 4 * D; n += 256) {
            const int c = n % D, g = n / D;
            const KvPairs level = kv_levels<T::BITS>(reinterpret_cast<const uint32_t *>(tile + T::V_AT) + kv_value_word<T>(g, 0, c));
            const int at = kv_value_header(4 * g, c / T::BLOCK);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const half2_t x = kv_value(level.p[e], (half2_t){as_h(vh[at + 2 * e]), as_h(vh[at + 2 * e + 1])}, (half2_t){as_h(vh[at + 8 + 2 * e]), as_h(vh[at + 9 + 2 * e])});
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
        *reinterpret_cast<kv_u32x4 *>(v_out + out_at(p, c)) = w;
    }
}

// tiles that a sequence's new tokens can touch, wherever they begin
static int64_t kv_tiles_touched(const KvView &v) { return (v.max_tokens + 2 * KV_TILE - 2) / KV_TILE; }

hipError_t launch_kv_append(int format, int head_dim, const KvView &v, const uint16_t *q, const uint16_t *k_new, const uint16_t *v_new, int n_heads, double base, int pair_mode,
                            uint16_t *q_out, hipStream_t s)
{
    const int64_t tiles = kv_tiles_touched(v), grid = tiles * v.n_seqs;
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    return for_kv_tile(format, head_dim, [&](auto tag) {
        typedef decltype(tag) T;
        hipLaunchKernelGGL((kv_append_kernel<T>), dim3((unsigned)grid, (unsigned)(v.n_kv_heads + n_heads)), dim3(256), 0, s, v, q, k_new, v_new, n_heads, log2(base), pair_mode, q_out,
                           (int)tiles);
        return hipGetLastError();
    });
}

hipError_t launch_kv_read(int format, int head_dim, const KvView &v, uint16_t *k_out, uint16_t *v_out, hipStream_t s)
{
    const int64_t tiles = kv_tiles_touched(v), grid = tiles * v.n_seqs;
    if (grid > 0x7fffffff) return hipErrorInvalidValue;
    return for_kv_tile(format, head_dim, [&](auto tag) {
        typedef decltype(tag) T;
        hipLaunchKernelGGL((kv_read_kernel<T>), dim3((unsigned)grid, (unsigned)v.n_kv_heads), dim3(256), 0, s, v, k_out, v_out, (int)tiles);
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
