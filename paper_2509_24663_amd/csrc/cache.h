// The paged K/V cache on the device: where a page's rows are, e4m3 codes and their scales, which sequence a work item belongs to.
#pragma once
#include "common.h"

namespace ifv2 {
namespace cache {

struct Args {
    char *k, *v;
    int64_t page_stride, head_stride, tok_stride;      // bytes
    float *ks, *vs;                                    // [num_pages, hkv], e4m3 only
    const int32_t *table;
    int32_t table_stride, num_pages, hkv;
    // page of block j of sequence b, or -1
    __device__ inline int page(int b, int j) const {
        const int g = table[(int64_t)b * table_stride + j];
        return g >= 0 && g < num_pages ? g : -1;
    }
    __device__ inline int64_t at(int page, int h) const { return page * page_stride + h * head_stride; }
};

int check(const infllmv2_params *p, const infllmv2_cache *c, int max_ctx, bool values);
// a launch's threads are counted in 32 bits
inline bool fits_launch(int64_t workgroups, int threads) { return workgroups < (1ll << 32) / threads; }
Args args(const infllmv2_params *p, const infllmv2_cache *c);

constexpr float kTop = 448.f;                          // largest e4m3 magnitude
constexpr int kMinExp = -100, kMaxExp = 119;           // of a scale

// smallest power of two 2^e with top <= 448 * 2^e, e clamped
__device__ inline float scale_for(float top) {
    // top = 2^x * f, f in [1, 2): 448 = 1.75 * 2^8, so e = x - 8, one more if f > 1.75 (subnormal tops have x = -127 here: clamped anyway)
    const uint32_t u = __float_as_uint(top);
    int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = e < kMinExp ? kMinExp : e > kMaxExp ? kMaxExp : e;
    return __uint_as_float((uint32_t)(e + 127) << 23);
}
__device__ inline float reciprocal_of_power(float s) { return __uint_as_float((254u << 23) - __float_as_uint(s)); }

// a value in units of the scale as a code: nearest, ties to even; saturating; NaN and infinities as NaN
__device__ inline uint32_t code(float x) {
    return fabsf(x) <= 3.4028234e38f ? (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(fminf(fmaxf(x, -kTop), kTop), 0.f, 0, false) & 0xffu : 0x7fu;
}
// four values; FITS: none is infinite or above the largest code
template <bool FITS>
__device__ inline uint32_t codes4(float a, float b, float c, float d) {
    if (!FITS) return code(a) | code(b) << 8 | code(c) << 16 | code(d) << 24;
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

// Which sequence the item-th of a batch's work items belongs to, when sequence s has count(s) of them; rem: which of the sequence's; before: the sum
// of weight(s) over the sequences in front.  Both sums are below 2^31 (fits_launch).  As find_seq_count (common.h), for counts that do not come from one
// list of offsets.  Called by every thread of a workgroup; one barrier; returns >= batch past the last item.  facts(s, i), i = 0, 1, 2: what else is wanted of
// the sequence (the lane that found it has just read it).
struct Facts {
    int x[3];
};
// op over the lanes up to a lane's own (0: what op leaves as it is)
template <class Op>
__device__ inline int wave_scan(int x, Op op) {
    x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true));      // row_shr:1, 2, 4, 8 (zeros shifted in)
    x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true));
    x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true));
    x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true));
    x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));     // row_bcast:15 into rows 1 and 3
    x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));     // row_bcast:31 into rows 2 and 3
    return x;
}
__device__ inline int wave_sums(int x) {
    return wave_scan(x, [](int a, int b) { return a + b; });
}
template <class Count, class Weight, class Fact>
__device__ inline int find_item(int batch, int item, int &rem, int &before, Facts &facts, int (&s_out)[6], Count count, Weight weight, Fact fact) {
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        int items = 0, sum = 0, bef = 0, seq = batch, r = 0;
        for (int s0 = 0; s0 < batch; s0 += 64) {
            const int s = s0 + lane;
            const int n = s < batch ? count(s) : 0, wt = s < batch ? weight(s) : 0;
            const int incl = wave_sums(n), wincl = wave_sums(wt);
            const uint64_t hit = __ballot(items + incl > item);
            if (hit) {
                const int l = __ffsll((long long)hit) - 1;
                seq = s0 + l;
                r = item - items - __builtin_amdgcn_readlane(incl - n, l);
                bef = sum + __builtin_amdgcn_readlane(wincl - wt, l);
                if (lane == l) {
#pragma unroll
                    for (int i = 0; i < 3; ++i) s_out[3 + i] = fact(s, i);
                }
                break;
            }
            items += __builtin_amdgcn_readlane(incl, 63);
            sum += __builtin_amdgcn_readlane(wincl, 63);
        }
        if (lane == 0) { s_out[0] = seq; s_out[1] = r; s_out[2] = bef; }
    }
    __syncthreads();
    // (uniform values, for the compiler as well: what follows from them stays in scalar registers)
    rem = __builtin_amdgcn_readfirstlane(s_out[1]);
    before = __builtin_amdgcn_readfirstlane(s_out[2]);
#pragma unroll
    for (int i = 0; i < 3; ++i) facts.x[i] = __builtin_amdgcn_readfirstlane(s_out[3 + i]);
    return __builtin_amdgcn_readfirstlane(s_out[0]);
}

}  // namespace cache
}  // namespace ifv2
