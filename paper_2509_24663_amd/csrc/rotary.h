// Rotary positions on the device: angles, and the pairs of channels that a group of eight pair numbers stands for.
#pragma once
#include "common.h"

namespace ifv2 {
namespace rotary {

struct Args {
    const uint64_t *turns;        // [rot_dim / 2]
    int32_t pairs;                // rot_dim / 2; 0: nothing is turned
    int32_t interleaved;
    float magnitude;
};

int check(const infllmv2_params *p, const infllmv2_rotary *r);
inline Args args(const infllmv2_rotary *r) { return Args{r->turns_d, r->rot_dim / 2, r->layout == INFLLMV2_ROTARY_INTERLEAVED, r->magnitude}; }

// magnitude * (cos, sin) of pos * turns, an angle in units of 2^-64 of a full turn: the upper 32 bits of the product modulo 2^64 (an angle error below
// 2^-32 turns, 1.5e-9).
// bf16 data: by the hardware's sine and cosine, which take turns: off by at most 1.3e-7 over a turn (measured at 2^22 angles) and 1.9e-7 by the angle's
// rounding to 24 bits, 2^-12 of a bf16 rounding.  fp32 data: the angle is cut into the nearest quarter turn and a rest of at most an eighth, whose sine and
// cosine are their Taylor series: the first terms left out are x^11 / 11! and x^12 / 12!, below 2e-9 at x = pi / 4.
template <typename T>
__device__ inline float2 cos_sin(int32_t pos, uint64_t turns, float magnitude) {
    const uint32_t p = (uint32_t)pos, lo = (uint32_t)turns, hi = (uint32_t)(turns >> 32);
    const uint32_t u = p * hi + __umulhi(p, lo) - (pos < 0 ? lo : 0u);      // (a negative position is p - 2^32)
    if constexpr (sizeof(T) == 2) {
        const float x = (float)(int32_t)u * 2.3283064365386963e-10f;        // 2^-32
        return float2{__builtin_amdgcn_cosf(x) * magnitude, __builtin_amdgcn_sinf(x) * magnitude};
    }
    const uint32_t quarter = (u + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(u - (quarter << 30)) * 1.4629180792671596e-9f;      // 2 pi / 2^32
    const float y = x * x;
    float s = 2.7557319e-6f, c = -2.7557319e-7f;
    s = __builtin_fmaf(s, y, -1.9841270e-4f);
    s = __builtin_fmaf(s, y, 8.3333333e-3f);
    s = __builtin_fmaf(s, y, -1.6666667e-1f);
    s = __builtin_fmaf(s * y, x, x);
    c = __builtin_fmaf(c, y, 2.4801587e-5f);
    c = __builtin_fmaf(c, y, -1.3888889e-3f);
    c = __builtin_fmaf(c, y, 4.1666667e-2f);
    c = __builtin_fmaf(c, y, -0.5f);
    c = __builtin_fmaf(c, y, 1.0f);
    const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
    return float2{(quarter + 1) & 2 ? -a * magnitude : a * magnitude, quarter & 2 ? -b * magnitude : b * magnitude};
}

// a pair turned; the fused form is written out so that every kernel rounds alike
__device__ inline float2 turn(float x, float y, float co, float si) {
    return float2{__builtin_fmaf(x, co, -(y * si)), __builtin_fmaf(x, si, y * co)};
}

// Channels of pair number q < d / 2: the pairs that are turned, then neighbours among the channels that are not.
__device__ inline int first_channel(const Args &r, int q) {
    return q >= r.pairs ? 2 * q : r.interleaved ? 2 * q : q;
}
__device__ inline int second_channel(const Args &r, int q) {
    return q >= r.pairs || r.interleaved ? 2 * q + 1 : q + r.pairs;
}

}  // namespace rotary
}  // namespace ifv2
