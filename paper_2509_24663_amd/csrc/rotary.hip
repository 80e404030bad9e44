// Rotary positions of Q or K and their gradient: (x1, x2) -> m (x1 cos - x2 sin, x1 sin + x2 cos) for each pair of channels; the gradient
// turns the other way.  HBM-bound for long prompts, one trip to memory for a decode step's rows.
//
// 32768 tokens of 32 heads of 128, bf16: 100.4 us, 5.3 TB/s read and written (a large copy reaches 4.9 on this card); 1985 tokens of 8 heads of 64, fp32: 4.8
// us, 16 tokens: 3.5 us, what a launch takes.
//
// A thread owns N pairs (N = 8, 4 or 1: the largest that divides both the turned and the other pairs, so that its channels are one run, or one
// in each half) of a token and goes through `per` of its heads: the angles are worked out once for all of them.  Neighbouring threads
// take neighbouring channels, then neighbouring heads.
#include <math.h>

#include "gen_unit.h"
#include "rotary.h"

namespace ifv2 {

namespace {

struct RotaryLaunch {
    rotary::Args r;
    const char *x;
    char *y;
    int64_t x_tok, x_head, y_tok, y_head;       // elements
    const int32_t *pos;
    int64_t tokens;
    int heads, slices, per, d;                  // slices * per >= heads: head s, s + slices, ... by thread slice s
    float sign;                                 // -1: the gradient
};

template <typename T, int N>
__device__ inline void load_run(float (&v)[N], const T *src) {
    typedef typename gen::Unaligned<typename std::conditional<sizeof(T) == 2, uint16_t, float>::type, N>::type Vec;
    const Vec x = *reinterpret_cast<const Vec *>(src);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (sizeof(T) == 2) v[i] = bf16_to_float(x[i]);
        else v[i] = x[i];
    }
}
template <typename T, int N>
__device__ inline void store_run(T *dst, const float (&v)[N]) {
    typedef typename gen::Unaligned<typename std::conditional<sizeof(T) == 2, uint16_t, float>::type, N>::type Vec;
    Vec x;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if constexpr (sizeof(T) == 2) x[i] = float_to_bf16(v[i]);
        else x[i] = v[i];
    }
    *reinterpret_cast<Vec *>(dst) = x;
}

template <typename T, int N, bool HALF>
__global__ void __launch_bounds__(256) rotary_kernel(RotaryLaunch a) {
    const uint32_t groups = (uint32_t)a.d / (2 * N), id = blockIdx.x * 256u + threadIdx.x, row = id / groups;
    const int q = (int)(id - row * groups) * N;
    const int64_t token = row / (uint32_t)a.slices;
    if (token >= a.tokens) return;
    const int slice = (int)(row - (uint32_t)token * (uint32_t)a.slices);
    const bool turned = q < a.r.pairs;
    float co[N], si[N];
#pragma unroll
    for (int i = 0; i < N; ++i) co[i] = 1.f, si[i] = 0.f;
    if (turned) {
        const int32_t pos = a.pos[token];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float2 cs = rotary::cos_sin<T>(pos, a.r.turns[q + i], a.r.magnitude);
            co[i] = cs.x;
            si[i] = cs.y * a.sign;
        }
    }
    const bool apart = HALF && turned;                       // two runs of N channels, else one of 2 N
    const int c0 = apart ? q : 2 * q, c1 = apart ? q + a.r.pairs : 2 * q + N;
    const T *x = reinterpret_cast<const T *>(a.x) + token * a.x_tok;
    T *y = reinterpret_cast<T *>(a.y) + token * a.y_tok;
    for (int h = slice; h < a.heads; h += a.slices) {
        float u[N], v[N];
        load_run<T, N>(u, x + h * a.x_head + c0);
        load_run<T, N>(v, x + h * a.x_head + c1);
        float s[N], t[N];
        if (HALF || N == 1) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float2 w = rotary::turn(u[i], v[i], co[i], si[i]);
                s[i] = turned ? w.x : u[i];
                t[i] = turned ? w.y : v[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {                    // pair i: elements 2 i and 2 i + 1 of the run
                const float p = 2 * i < N ? u[(2 * i) % N] : v[(2 * i) % N], w = 2 * i < N ? u[(2 * i + 1) % N] : v[(2 * i + 1) % N];
                const float2 z = rotary::turn(p, w, co[i], si[i]);
                const float e = turned ? z.x : p, f = turned ? z.y : w;
                if (2 * i < N) s[(2 * i) % N] = e, s[(2 * i + 1) % N] = f;
                else t[(2 * i) % N] = e, t[(2 * i + 1) % N] = f;
            }
        }
        store_run<T, N>(y + h * a.y_head + c0, s);
        store_run<T, N>(y + h * a.y_head + c1, t);
    }
}

template <typename T, int N>
int launch_n(const RotaryLaunch &a, hipStream_t stream) {
    const uint64_t threads = (uint64_t)a.tokens * a.slices * (a.d / (2 * N));
    const dim3 grid((unsigned)((threads + 255) / 256));
    if (a.r.interleaved) hipLaunchKernelGGL((rotary_kernel<T, N, false>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((rotary_kernel<T, N, true>), grid, dim3(256), 0, stream, a);
    return hip_status(hipGetLastError());
}
template <typename T>
int launch_t(const RotaryLaunch &a, int n, hipStream_t stream) {
    return n == 8 ? launch_n<T, 8>(a, stream) : n == 4 ? launch_n<T, 4>(a, stream) : launch_n<T, 1>(a, stream);
}

int rotary_common(const infllmv2_params *p, const infllmv2_rotary *r, const void *x, int64_t x_tok, int64_t x_head, void *y,
                  int64_t y_tok, int64_t y_head, const int32_t *pos, int64_t tokens, int32_t heads, float sign, void *stream) {
    int st = check_params(p);
    if (st) return st;
    st = rotary::check(p, r);
    if (st) return st;
    if (tokens < 0 || heads < 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (tokens == 0 || heads == 0) return INFLLMV2_OK;
    if (x == nullptr || y == nullptr || pos == nullptr || r->turns_d == nullptr) return INFLLMV2_ERR_INVALID_ARGUMENT;
    const int64_t d = p->head_dim;
    int64_t span_t, span_h;
    if (__builtin_mul_overflow(tokens - 1, y_tok, &span_t) || __builtin_mul_overflow((int64_t)heads - 1, y_head, &span_h)) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (tokens > 0xffffff00ll || heads > (1 << 24)) return INFLLMV2_ERR_UNSUPPORTED;      // (thread numbers are 32 bits)
    if (x_tok < 0 || x_head < 0 || y_tok < 0 || y_head < 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    // rows of the output stand apart: one of the two strides steps over everything that the other reaches
    if (tokens > 1 && heads > 1 && !(y_head >= d && y_tok - d >= span_h) && !(y_tok >= d && y_head - d >= span_t))
        return INFLLMV2_ERR_INVALID_ARGUMENT;
    if ((tokens > 1 && y_tok < d) || (heads > 1 && y_head < d)) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (x == y && ((tokens > 1 && x_tok != y_tok) || (heads > 1 && x_head != y_head))) return INFLLMV2_ERR_INVALID_ARGUMENT;
    const int pairs = r->rot_dim / 2, rest = p->head_dim / 2 - pairs;
    const int n = pairs % 8 == 0 && rest % 8 == 0 ? 8 : pairs % 4 == 0 && rest % 4 == 0 ? 4 : 1;
    const int64_t groups = d / (2 * n);
    RotaryLaunch a{rotary::args(r), (const char *)x, (char *)y, x_tok, x_head, y_tok, y_head, pos, tokens, heads, 0, 1, p->head_dim, sign};
    // heads per thread: as many as leave every CU its 2048 threads
    while (a.per < 8 && tokens * ((heads + 2 * a.per - 1) / (2 * a.per)) * groups >= 256 * 2048) a.per *= 2;
    a.slices = (heads + a.per - 1) / a.per;
    if (tokens > (int64_t)0xffffff00u / (a.slices * groups)) return INFLLMV2_ERR_UNSUPPORTED;
    return p->dtype == INFLLMV2_BF16 ? launch_t<bf16_t>(a, n, (hipStream_t)stream) : launch_t<float>(a, n, (hipStream_t)stream);
}

}  // namespace

int rotary::check(const infllmv2_params *p, const infllmv2_rotary *r) {
    if (r == nullptr || r->rot_dim < 2 || r->rot_dim % 2 != 0 || r->rot_dim > p->head_dim) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (r->layout != INFLLMV2_ROTARY_HALF && r->layout != INFLLMV2_ROTARY_INTERLEAVED) return INFLLMV2_ERR_UNSUPPORTED;
    if (!(r->magnitude > 0.f) || !isfinite(r->magnitude) || r->reserved != 0 || ((uintptr_t)r->turns_d & 7) != 0)
        return INFLLMV2_ERR_INVALID_ARGUMENT;
    return INFLLMV2_OK;
}

}  // namespace ifv2

extern "C" {

int infllmv2_rotary_turns(int32_t rot_dim, double base, int32_t scaling, double factor, double original_len,
                          double beta_fast, double beta_slow, uint64_t *turns_h) {
    if (rot_dim < 2 || rot_dim % 2 != 0 || turns_h == nullptr || !(base > 1.0) || !isfinite(base) || !(factor >= 1.0) || !isfinite(factor))
        return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (scaling < INFLLMV2_SCALING_NONE || scaling > INFLLMV2_SCALING_PARTS) return INFLLMV2_ERR_UNSUPPORTED;
    if (scaling == INFLLMV2_SCALING_BASE && rot_dim <= 2) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (scaling == INFLLMV2_SCALING_PARTS &&
        (!(original_len > 0.0) || !isfinite(original_len) || !(beta_slow > 0.0) || !(beta_fast > beta_slow) || !isfinite(beta_fast)))
        return INFLLMV2_ERR_INVALID_ARGUMENT;
    const double two_pi = 6.283185307179586476925;
    if (scaling == INFLLMV2_SCALING_BASE) base *= pow(factor, rot_dim / (rot_dim - 2.0));
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = pow(base, -2.0 * i / rot_dim) / two_pi;        // turns per position, below 0.16
        if (scaling == INFLLMV2_SCALING_LINEAR) f /= factor;
        if (scaling == INFLLMV2_SCALING_PARTS) {
            const double turns = original_len * f, mix = (turns - beta_slow) / (beta_fast - beta_slow);
            const double keep = mix < 0.0 ? 0.0 : mix > 1.0 ? 1.0 : mix;
            f *= keep + (1.0 - keep) / factor;
        }
        turns_h[i] = (uint64_t)(f * 18446744073709551616.0 + 0.5);
    }
    return INFLLMV2_OK;
}

int infllmv2_rotary_fwd(const infllmv2_params *p, const infllmv2_rotary *r, const void *x_d, int64_t x_tok_stride,
                        int64_t x_head_stride, void *y_d, int64_t y_tok_stride, int64_t y_head_stride, const int32_t *pos_d,
                        int64_t tokens, int32_t heads, void *stream) {
    return ifv2::rotary_common(p, r, x_d, x_tok_stride, x_head_stride, y_d, y_tok_stride, y_head_stride, pos_d, tokens, heads, 1.f, stream);
}

int infllmv2_rotary_bwd(const infllmv2_params *p, const infllmv2_rotary *r, const void *dy_d, int64_t dy_tok_stride,
                        int64_t dy_head_stride, void *dx_d, int64_t dx_tok_stride, int64_t dx_head_stride, const int32_t *pos_d,
                        int64_t tokens, int32_t heads, void *stream) {
    return ifv2::rotary_common(p, r, dy_d, dy_tok_stride, dy_head_stride, dx_d, dx_tok_stride, dx_head_stride, pos_d, tokens, heads, -1.f,
                               stream);
}

}  // extern "C"
