// The quantized key/value cache: where its pages, tiles and codes lie, and how a code becomes an fp16 number.  Shared by the kernels that write the
// cache, read it back and attend over it; the layout itself is stated in include/iflow.h.
#pragma once

#include "iflow_common.h"

namespace iflow {

constexpr int KV_TILE = 32;                                   // positions of a tile (first_tile() shifts by it)

template <int BITS_, int BLOCK_, int D_>
struct KvTile {
    static constexpr int BITS = BITS_, BLOCK = BLOCK_, D = D_, L = (1 << BITS_) - 1;
    static constexpr int NB = D / BLOCK;                      // blocks of a position
    static constexpr int CODES = KV_TILE * D * BITS / 8;      // bytes of the keys' codes; the values have as many
    static constexpr int PIECES = CODES / 1024;               // 16 bytes for each of 64 lanes
    static constexpr int RUN = CODES / 256;                   // 32-bit words of a lane's run
    static constexpr int HEADERS = KV_TILE * NB * 4;
    static constexpr int V_AT = CODES, KH_AT = 2 * CODES, VH_AT = 2 * CODES + HEADERS, BYTES = 2 * (CODES + HEADERS);
    static constexpr int PER_WORD = 32 / BITS;
};

// Host side: run fn(KvTile<..>{}) for a format and head dimension; hipErrorInvalidValue for one that a cache does not take.
template <typename Fn>
inline hipError_t for_kv_tile(int format, int head_dim, Fn fn)
{
    switch (format * 1000 + head_dim) {
    case IFLOW_Q4_B32 * 1000 + 64: return fn(KvTile<4, 32, 64>{});
    case IFLOW_Q4_B32 * 1000 + 128: return fn(KvTile<4, 32, 128>{});
    case IFLOW_Q4_B64 * 1000 + 64: return fn(KvTile<4, 64, 64>{});
    case IFLOW_Q4_B64 * 1000 + 128: return fn(KvTile<4, 64, 128>{});
    case IFLOW_Q8_B32 * 1000 + 64: return fn(KvTile<8, 32, 64>{});
    case IFLOW_Q8_B32 * 1000 + 128: return fn(KvTile<8, 32, 128>{});
    case IFLOW_Q8_B64 * 1000 + 64: return fn(KvTile<8, 64, 64>{});
    case IFLOW_Q8_B64 * 1000 + 128: return fn(KvTile<8, 64, 128>{});
    default: return hipErrorInvalidValue;
    }
}

// What a kernel knows of the cache and the batch (by value; every array is the caller's).
struct KvView {
    uint8_t *pages;
    const int32_t *table, *lens, *first;                      // table, first: may be null
    int64_t n_pages, n_tokens, page_bytes;
    int32_t n_seqs, max_pages, max_tokens, max_seq, n_kv_heads, tiles_per_page;
    uint32_t page_magic;                                      // ceil(2^32 / tiles_per_page); 0 for 1
    __device__ __forceinline__ int page_of(int t) const { return page_magic ? (int)__umulhi((uint32_t)t, page_magic) : t; }      // t / tiles_per_page, exact for t, tiles_per_page < 2^16
};

// Who has which page, as iflow_kv_tables reads and writes it.
struct KvTables {
    const int32_t *new_tokens, *held, *free_state, *shared;   // new_tokens: not read where every sequence has one
    int32_t *held_out, *free_out, *ring;
    int64_t *slots;                                           // may be null
    int32_t n_shared;
};

// One sequence's new tokens as the kernels take them: rows row .. row + count - 1 of the batch's tokens at positions position .. .  Whatever the arrays
// hold, what comes out of here stays inside the call's buffers: count is at most max_tokens, and every token is asked for with has().  (In 32 bits: where numbers that no batch has
// leave them, what has() sees is other numbers, and it still sees them.)
struct KvSequence {
    int row, position, count, n_tokens, max_seq;
    __device__ __forceinline__ KvSequence(const KvView &v, int b)
    {
        row = v.first ? v.first[b] : b;
        const int n = v.first ? (int)((uint32_t)v.first[b + 1] - (uint32_t)row) : 1;
        n_tokens = (int)v.n_tokens; max_seq = v.max_seq;
        position = (int)((uint32_t)v.lens[b] - (uint32_t)n);
        count = max(0, min(n, v.max_tokens));
    }
    // token i has a row, and a position that the cache has
    __device__ __forceinline__ bool has_row(int i) const { return (uint32_t)i < (uint32_t)count && (uint32_t)row + (uint32_t)i < (uint32_t)n_tokens; }
    __device__ __forceinline__ bool has(int i) const { return has_row(i) && (uint32_t)position + (uint32_t)i < (uint32_t)max_seq; }
    __device__ __forceinline__ int first_tile() const { return position >> 5; }          // (rounded down, also below zero)
    __device__ __forceinline__ int tiles() const { return count > 0 ? ((position & (KV_TILE - 1)) + count + KV_TILE - 1) >> 5 : 0; }       // that its tokens lie in
    // positions that token i sees: its own and all before
    __device__ __forceinline__ int sees(int i) const { return max(0, min((int)((uint32_t)position + (uint32_t)i + 1u), max_seq)); }
};

// inclusive sum over the lanes up to this one
__device__ __forceinline__ int wave_scan(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);       // row_shr 1, 2, 4, 8: within rows of sixteen
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);       // row_bcast:15 into rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);       // row_bcast:31 into rows 2 and 3
    return x;
}
// the last of n with upto[i] <= x, for a lane's x of x0 .. x1 (upto in order, upto[0] not above x0; otherwise any of the n): by the whole wavefront for both ends, then by each lane between them
__device__ __forceinline__ int kv_last_of(const int32_t *upto, int n, int x0, int x1, int x)
{
    const int lane = threadIdx.x & 63;
    int lo0 = 0, lo1 = 0, size = n;                           // (they are below lo + size)
    while (size > 1) {
        const int step = (size + 63) >> 6, i0 = lo0 + lane * step, i1 = lo1 + lane * step;
        const int at0 = upto[min(i0, n - 1)], at1 = upto[min(i1, n - 1)];
        const bool in = lane * step < size;
        lo0 += max(0, __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && i0 < n && at0 <= x0)) - 1) * step;
        lo1 += max(0, __builtin_popcountll(__builtin_amdgcn_ballot_w64(in && i1 < n && at1 <= x1)) - 1) * step;
        size = step;
    }
    const int span = lo1 - lo0;
    for (int step = span > 0 ? 1 << (31 - __builtin_clz(span)) : 0; step > 0; step >>= 1) {
        const int i = lo0 + step;
        if (i <= lo1 && upto[i] <= x) lo0 = i;
    }
    return lo0;
}
// Number w of all sequences' units, units(b) of each, in order: whose it is (b), and which of that sequence's (w); false past the last.  By every wavefront alike, 64 sequences at a time.
// For batches whose longest sequence has many more tokens than most, where a grid of max_tokens for each would be workgroups with nothing to do.
template <typename Units> __device__ __forceinline__ bool kv_find(const KvView &v, int &w, int &b, Units units)
{
    const int lane = threadIdx.x & 63;
    for (b = 0; b < v.n_seqs; b += 64) {
        const int mine = b + lane < v.n_seqs ? units(KvSequence(v, b + lane)) : 0, upto = wave_scan(mine);
        const uint64_t mask = __builtin_amdgcn_ballot_w64(upto > w);
        if (mask != 0) {
            const int skip = __builtin_ctzll(mask);
            b += skip;
            w -= __builtin_amdgcn_readlane(upto - mine, skip);
            return true;
        }
        w -= __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// The tile that holds positions 32 t .. 32 t + 31 of sequence b; null where its page is none of the cache's.  (t < max_seq / 32, rounded up: inside the table's row.)
__device__ __forceinline__ int64_t kv_page(const KvView &v, int b, int p)
{
    const int64_t entry = (int64_t)b * v.max_pages + p;
    return v.table ? (int64_t)v.table[entry] : entry;
}
__device__ __forceinline__ uint8_t *kv_tile_in(const KvView &v, int64_t page, int kv_head, int tile_of_page, int tile_bytes)
{
    if (page < 0 || page >= v.n_pages) return nullptr;
    return v.pages + page * v.page_bytes + ((int64_t)kv_head * v.tiles_per_page + tile_of_page) * tile_bytes;
}
__device__ __forceinline__ uint8_t *kv_tile_at(const KvView &v, int b, int kv_head, int t, int tile_bytes)
{
    const int p = v.page_of(t);
    return kv_tile_in(v, kv_page(v, b, p), kv_head, t - p * v.tiles_per_page, tile_bytes);
}

// ---- where an element lies in its tile ------------------------------------------------------------------------------------
// key codes: 32-bit word that holds the first of PER_WORD consecutive components 'c' (a multiple of it) of position r
template <typename T> __host__ __device__ constexpr int kv_key_word(int r, int c)
{
    const int g = c / (T::D / 4), at = (r >> 4) * (T::RUN / 2) + (c - g * (T::D / 4)) / T::PER_WORD;
    return ((at >> 2) * 64 + g * 16 + (r & 15)) * 4 + (at & 3);
}
// value codes: the word that holds element k (a multiple of PER_WORD) of the eight positions of g, of component c
template <typename T> __host__ __device__ constexpr int kv_value_word(int g, int k, int c)
{
    const int at = (c >> 4) * (8 / T::PER_WORD) + k / T::PER_WORD;
    return ((at >> 2) * 64 + g * 16 + (c & 15)) * 4 + (at & 3);
}
__host__ __device__ constexpr int kv_value_position(int g, int k) { return (k >> 2) * 16 + 4 * g + (k & 3); }
// headers, in 16-bit units from the tile's headers of keys or of values: the scale; the offset 1 (keys) or 8 (values) behind it
__host__ __device__ constexpr int kv_key_header(int r, int block) { return ((block * 16 + (r & 15)) * 2 + (r >> 4)) * 2; }
__host__ __device__ constexpr int kv_value_header(int r, int block) { return (block * 4 + ((r & 15) >> 2)) * 16 + (r >> 4) * 4 + (r & 3); }

// ---- codes to fp16 ----------------------------------------------------------------------------------------------------------
typedef uint32_t kv_u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t kv_u32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 kv_half8 __attribute__((ext_vector_type(8)));
typedef float kv_float4 __attribute__((ext_vector_type(4)));
struct KvPairs { half2_t p[4]; };                             // eight consecutive elements

// the eight levels that begin at `word` (one word of nibbles, two of bytes) as fp16 numbers: or-ed into the mantissa of 1024 (64 for the nibbles four bits up), which is subtracted, exactly
struct KvMagic {
    uint32_t at0, at4;                                        // (in registers: v_and_or_b32 takes no literals)
    __device__ __forceinline__ KvMagic() : at0(0x64006400u), at4(0x54005400u) { asm volatile("" : "+v"(at0), "+v"(at4)); }
};
template <int BITS>
__device__ __forceinline__ KvPairs kv_levels(const uint32_t *word, const KvMagic &magic)
{
    KvPairs v;
    const half2_t b0 = {(half_t)1024.f, (half_t)1024.f};
    if constexpr (BITS == 4) {
        const uint32_t w = word[0], w8 = w >> 8;
        const half2_t b4 = {(half_t)64.f, (half_t)64.f};
        v.p[0] = as_h2(and_or(w, 0x000F000Fu, magic.at0)) - b0;
        v.p[1] = as_h2(and_or(w, 0x00F000F0u, magic.at4)) - b4;
        v.p[2] = as_h2(and_or(w8, 0x000F000Fu, magic.at0)) - b0;
        v.p[3] = as_h2(and_or(w8, 0x00F000F0u, magic.at4)) - b4;
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            v.p[2 * i] = as_h2(__builtin_amdgcn_perm(magic.at0, word[i], 0x05010500u)) - b0;
            v.p[2 * i + 1] = as_h2(__builtin_amdgcn_perm(magic.at0, word[i], 0x05030502u)) - b0;
        }
    }
    return v;
}
// level * scale + offset, rounded once: what iflow_dequant makes of the same three numbers
__device__ __forceinline__ half2_t kv_value(half2_t level, half2_t scale, half2_t offset) { return __builtin_elementwise_fma(level, scale, offset); }

}  // namespace iflow
