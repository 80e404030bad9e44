// What the two kernels of infllmv2_cache_attn share: cache_attn.hip (16 columns per workgroup, any data) and cache_attn_tile.hip (chunks of prompts and a few
// tokens over long contexts, bf16).
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

struct AttnArgs {
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
};

// cache_attn_tile.hip
constexpr int kTileThreads = 512;
int launch_tile(const AttnArgs &a, const infllmv2_params *p, bool codes, int64_t items, hipStream_t stream);

}  // namespace cache_attn
}  // namespace ifv2
