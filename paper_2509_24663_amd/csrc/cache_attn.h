// What the two kernels of infllmv2_cache_attn and infllmv2_cache_tree_attn share: cache_attn.hip (16 columns per workgroup, any data) and cache_attn_tile.hip
// (chunks of prompts and a few tokens over long contexts, bf16).
#pragma once
#include "cache.h"
#include "gen_unit.h"

namespace ifv2 {
namespace cache_attn {

constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.4028234e38f;

// Sums of weights times values are finite wherever the result is: a mean of values.  Relative to the largest logit, or one near it, they may pass the
// largest float although their quotient by the sum of the weights does not, so
//  - elements of a walk's sums that are not finite are taken from a second walk whose references lie kLift binary orders above the largest logit (2^34 keys
//    of weight 2^6 x 2^-kLift add up to 1; the other elements keep the first walk's, whose small weights reach 40 orders further down),
//  - sums are joined as means: each divided by its own weights, then added up with its share of all weights.
constexpr float kLift = 40.f;
// (a factor that is formed before it is multiplied with anything else)
__device__ inline float formed(float x) {
    asm("" : "+v"(x));
    return x;
}

// over lanes with equal lane % 16
__device__ inline float rows_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float rows_add(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}
// two codes (the lower or the upper half of w) as two bf16 values; of the scale, a power of two, the exponent counts
template <bool UPPER>
__device__ inline uint32_t widen(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, UPPER));
}
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ inline uint32_t pack(float a, float b) {          // nearest even
    const bf16x2 x = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, x);
}
// all ones in the elements of w (e4m3 codes, bf16) that are infinities or NaN
template <bool CODES>
__device__ inline uint32_t not_finite(uint32_t w) {
    if (CODES) return ((((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xffu;
    return ((((w & 0x7fff7fffu) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu;
}
// Two weights as two bf16 pieces each, the upper 16 bits and the rest rounded to nearest: off by at most 2^-16 of the weight, either way.  The first piece is
// that of the next smaller float: below the weight, also where 16 bits hold it, so that the second is above 0 and both products with an infinite value are
// that infinity (0 x infinity is not a number).
struct Pieces {
    uint32_t hi, lo;
};
__device__ inline Pieces pieces(float a, float b) {
    const uint32_t u = __builtin_elementwise_sub_sat(__float_as_uint(a), 1u), v = __builtin_elementwise_sub_sat(__float_as_uint(b), 1u);      // (0 stays 0)
    return Pieces{gen::upper_halves(u, v), pack(a - __uint_as_float(u & 0xffff0000u), b - __uint_as_float(v & 0xffff0000u))};
}

// Queries in a row: each is at the place of its key and attends to those up to it.
struct AttnArgs {
    static constexpr bool kTree = false;
    cache::Args c;
    const char *q;
    char *out;
    float *lse;                        // or nullptr
    const int32_t *cu, *ctx, *idx;     // idx: nullptr: all keys
    int batch, hq, topk, dense_below;
    int group_tokens;                  // of 16 columns over all keys (16 / G)
    int wide_from;                     // sequences over all keys with so many queries are the tile kernel's
    int tile_groups;                   // column groups of a tile of this launch (1: cache_attn.hip; rules::tile_size)
    int fine;                          // tile kernel: weights of two pieces (small tiles)
    int pps;                           // pages of a split
    int even;                          // > 0: one query token for each sequence, item = (sequence, head, split < even); slots alike
    int multi;                         // some tile of cache_attn.hip has more than one token
    float scale;
    float *part;                       // [slots][16 tile_groups][D] means over the split's keys
    float *ml;                         // [slots][16 tile_groups][2] reference, sum of weights
    // how the n queries of a sequence of len tokens are cut (always inlined: a call in a kernel that is long already takes registers from all of it)
    __host__ __device__ __attribute__((always_inline)) bool listed(int len) const { return idx != nullptr && len >= dense_below; }
    __host__ __device__ __attribute__((always_inline)) int tile_tokens(int len) const { return listed(len) ? 1 : group_tokens * tile_groups; }
    __host__ __device__ __attribute__((always_inline)) int tiles(int n, int len) const {
        if ((tile_groups > 1) != (!listed(len) && n >= wide_from)) return 0;
        const int t = tile_tokens(len);
        return (n + t - 1) / t;
    }
    // pages of the tile whose last token is at pos_last: at most so many are there (listed: a list may hold them anywhere)
    __host__ __device__ __attribute__((always_inline)) int pages(int len, int pos_last) const {
        const int all = pos_last / kBlock + 1;
        return listed(len) && topk < (len + kBlock - 1) / kBlock ? topk : all;
    }
    __host__ __device__ __attribute__((always_inline)) int splits(int len, int pos_last) const { return (pages(len, pos_last) + pps - 1) / pps; }
    __host__ __device__ __attribute__((always_inline)) int most_splits(int n, int len) const { return n == 0 ? 0 : splits(len, len - 1); }
    // pages of a tile that begins with token `first` of n, as far as the tile's first token sees them, and in all
    __host__ int first_pages(int n, int len, int first) const { return (len - n + first) / kBlock + 1; }
    __host__ int most_pages(int, int len) const { return pages(len, len - 1); }
};

// A tree of drafted tokens: queries and keys are the last n of a sequence's len rows.  Query i attends to the context (the rows in front of the n; of it, a
// list picks blocks for the whole sequence) and to those of the n that row i of the mask names.  The entries that a tile goes through are the list's, or all
// blocks in front of the first drafted row's, and then the blocks of drafted rows: an entry's number is what splits are counted in.
struct TreeArgs : AttnArgs {
    static constexpr bool kTree = true;
    const uint32_t *mask;              // [total][words]
    int words;
    int even_n, even_tiles;            // even > 0: as many drafted tokens for each sequence, so many tiles
    __host__ __device__ __attribute__((always_inline)) int tile_tokens(int) const { return group_tokens * tile_groups; }
    __host__ __device__ __attribute__((always_inline)) int tiles(int n, int) const {
        if ((tile_groups > 1) != (n >= wide_from)) return 0;
        const int t = group_tokens * tile_groups;
        return (n + t - 1) / t;
    }
    // entries in front of those of drafted rows: a list may be longer than the blocks that it can name, and holds them anywhere
    __host__ __device__ __attribute__((always_inline)) int listed_entries(int n, int len) const { return listed(len) ? topk : (len - n) / kBlock; }
    __host__ __device__ __attribute__((always_inline)) int most_pages(int n, int len) const {
        const int front = (len - n) / kBlock, last = (len - 1) / kBlock;
        return (listed(len) && topk < front ? topk : front) + last - front + 1;
    }
    __host__ __device__ __attribute__((always_inline)) int most_splits(int n, int len) const { return n == 0 ? 0 : (most_pages(n, len) + pps - 1) / pps; }
    __host__ int first_pages(int n, int len, int) const { return most_pages(n, len); }
    // which of the N <= 32 keys from `key` on a query sees by its row of the mask: drafted rows start at row `front`, open: the context's rows in front of it are seen
    template <int N>
    __device__ __attribute__((always_inline)) uint32_t seen(const uint32_t *row, int key, int front, int n, bool open) const {
        const int d = key - front;
        uint32_t x = 0;
        if (d < n && d > -N) {
            const int w = d >> 5;                                   // (-1: in front of the mask)
            const uint64_t lo = w >= 0 ? row[w] : 0u, hi = 32 * (w + 1) < n ? row[w + 1] : 0u;
            x = (uint32_t)((lo | hi << 32) >> (d & 31));
            if (n - d < 32) x &= (1u << (n - d)) - 1u;              // bits behind the tree say nothing
        }
        const uint32_t before = d >= 0 ? 0u : d <= -N ? ~0u : (1u << -d) - 1u;
        return ((x & ~before) | (open ? before : 0u)) & (N == 32 ? ~0u : (1u << (N & 31)) - 1u);
    }
    template <int N>                   // the same of N <= 64 keys
    __device__ __attribute__((always_inline)) uint64_t seen_step(const uint32_t *row, int key, int front, int n, bool open) const {
        if constexpr (N <= 32) return seen<N>(row, key, front, n, open);
        else return seen<32>(row, key, front, n, open) | (uint64_t)seen<N - 32>(row, key + 32, front, n, open) << 32;
    }
    // Trees of up to 64 tokens: a row of the mask is requested with the query and kept (at the edge it would be one more trip to memory, in tiles behind the
    // pages that are on their way)
    __device__ __attribute__((always_inline)) uint64_t kept_row(const uint32_t *row, int n) const {
        if (n > 64) return 0;
        const uint64_t x = row[0] | (n > 32 ? (uint64_t)row[1] << 32 : 0u);
        return n == 64 ? x : x & ((1ull << n) - 1);
    }
    template <int N>
    __device__ __attribute__((always_inline)) uint64_t seen_kept(uint64_t kept, const uint32_t *row, int key, int front, int n, bool open) const {
        if (n > 64) return seen_step<N>(row, key, front, n, open);
        const int d = key - front;
        const uint64_t x = d >= 64 || d <= -64 ? 0 : d >= 0 ? kept >> d : kept << -d;
        const uint64_t before = d >= 0 ? 0 : d <= -64 ? ~0ull : (1ull << -d) - 1;
        return (x | (open ? before : 0)) & (N == 64 ? ~0ull : (1ull << (N & 63)) - 1);          // (x has nothing in front of the drafted rows)
    }
};

// cache_attn_tile.hip
constexpr int kTileThreads = 512;
template <class A>
int launch_tile(const A &a, const infllmv2_params *p, bool codes, int64_t items, hipStream_t stream);

}  // namespace cache_attn
}  // namespace ifv2
