// Stage 1 for a growing paged cache: K^{C1}_i = Mean(K[i*s : i*s + l]) (Sec. 3.3, Eq. 3) for the rows that became complete while sequence b grew
// from prev[b] to ctx[b] tokens, from the keys as the pages hold them.  As the append of compress_k.hip, with a page looked up for every 64
// tokens of a window; the additions are in the order of the window, in 32 bits.
//
// Bound: memory latency.  A window's rows are requested together, behind one lookup of the pages they are in.  128 sequences with a new row each: 4.6 us (fewer
// rows at a time: 7.3; every row asked whether it is there: 5.7); 65536 tokens of 2 heads of 128, e4m3, 21 MB: 7.3 us (9.5; 8.8), every row read for two
// windows.  (Adding each run of stride rows once would be half the requests, and another order of additions than that of compress_k.hip, whose rows these equal.)
#include <type_traits>

#include "cache.h"
#include "gen_unit.h"

namespace ifv2 {

namespace {

constexpr int VEC = 8;            // channels per thread

struct CompressArgs {
    cache::Args c;
    float *kc;
    int64_t kc_head_stride;
    const int32_t *prev, *ctx;
    int batch;
    int64_t pairs;
    int lc, sc, rows;
};

// LOOKUP: workgroups are those of the new rows, each finds its sequence; else as many for every sequence, those past its rows with nothing to do
template <typename T, int D, bool CODES, bool LOOKUP>
__global__ void __launch_bounds__(64) cache_compress_kernel(CompressArgs a) {
    constexpr int VPR = D / VEC;
    // rows requested at once, of two pages at most, both looked up first (fp32 rows: registers)
    constexpr int U = CODES || sizeof(T) == 2 ? 32 : 16;
    typedef typename std::conditional<CODES, uint2, typename std::conditional<sizeof(T) == 2, gen::u16x8_u, gen::f32x8_u>::type>::type Vec;
    const int slot = threadIdx.x / VPR;
    int b, h, i;
    int64_t pair;
    if constexpr (LOOKUP) {
        __shared__ int s_item[6];
        constexpr int PER = 64 / VPR;
        int rem, before;
        cache::Facts f;
        b = cache::find_item(a.batch, (int)blockIdx.x, rem, before, f, s_item,
                             [&](int s) { return (num_cmp(a.ctx[s], a.lc, a.sc) - num_cmp(a.prev[s], a.lc, a.sc) + PER - 1) / PER * a.c.hkv; },
                             [](int) { return 0; }, [&](int s, int) { return num_cmp(a.prev[s], a.lc, a.sc); });
        if (b >= a.batch) return;
        h = rem % a.c.hkv;
        pair = (int64_t)b * a.c.hkv + h;
        i = f.x[0] + rem / a.c.hkv * PER + slot;
    } else {
        pair = (blockIdx.y * (64u / VPR) + slot) / (unsigned)a.rows;
        if (pair >= a.pairs) return;
        b = (int)pair / a.c.hkv, h = (int)pair - b * a.c.hkv;
        i = num_cmp(a.prev[b], a.lc, a.sc) + (int)blockIdx.x * a.rows + (slot & (a.rows - 1));
    }
    if (i >= num_cmp(a.ctx[b], a.lc, a.sc)) return;
    const int c0 = (threadIdx.x % VPR) * VEC;
    float acc[VEC];
#pragma unroll
    for (int c = 0; c < VEC; ++c) acc[c] = 0.f;
    const int end = i * a.sc + a.lc;
    for (int t = i * a.sc; t < end; t += U) {
        const int last = min(t + U, end) - 1, block = t / kBlock, edge = (block + 1) * kBlock;     // rows from edge on are the next page's
        const int page0 = a.c.page(b, block), page1 = last >= edge ? a.c.page(b, block + 1) : -1;
        // (rows of a page that is not there: any row's address, taken as 0)
        const int safe0 = page0 >= 0 ? page0 : 0, safe1 = page1 >= 0 ? page1 : 0;
        const char *base0 = a.c.k + a.c.at(safe0, h) + (int64_t)(t - block * kBlock) * a.c.tok_stride + c0 * (CODES ? 1 : (int)sizeof(T));
        const char *base1 = a.c.k + a.c.at(safe1, h) + (int64_t)(t - edge) * a.c.tok_stride + c0 * (CODES ? 1 : (int)sizeof(T));
        float s0 = 1.f, s1 = 1.f;
        if constexpr (CODES) {
            s0 = a.c.ks[(int64_t)safe0 * a.c.hkv + h];
            s1 = a.c.ks[(int64_t)safe1 * a.c.hkv + h];
        }
        const int n0 = min(edge, last + 1) - t, n = last + 1 - t;   // rows of the first page, of both
        Vec x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int v = min(u, n - 1);
            x[u] = *reinterpret_cast<const Vec *>((v < n0 ? base0 : base1) + (int64_t)v * a.c.tok_stride);
        }
        __builtin_amdgcn_sched_barrier(0);       // (left alone, the scheduler trades the requests for registers)
        auto add = [&](auto some) {                                  // some: rows that are not the window's or of no page are among them
            constexpr bool SOME = decltype(some)::value;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool in = !SOME || (u < n && (u < n0 ? page0 : page1) >= 0);
                if constexpr (CODES) {
                    const float scale = u < n0 ? s0 : s1;            // (a power of two: the product is exact, fused or not)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int w = (int)(j ? x[u].y : x[u].x);
                        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
                        const float v[4] = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[4 * j + i] = in ? __builtin_fmaf(v[i], scale, acc[4 * j + i]) : acc[4 * j + i];
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < VEC; ++c) {
                        if constexpr (sizeof(T) == 2) acc[c] += in ? bf16_to_float(x[u][c]) : 0.f;
                        else acc[c] += in ? x[u][c] : 0.f;
                    }
                }
            }
        };
        if (__all(n == U && page0 >= 0 && (n0 == n || page1 >= 0))) add(std::false_type());
        else add(std::true_type());
    }
    const float inv = 1.0f / (float)a.lc;
#pragma unroll
    for (int c = 0; c < VEC; ++c) acc[c] *= inv;
    gen::store_row<float, VEC>(a.kc + pair * a.kc_head_stride + (int64_t)i * D + c0, acc);
}

template <typename T, int D>
int launch_t(CompressArgs a, bool codes, int max_new, int64_t n, hipStream_t stream) {
    // consecutive new rows of a pair share a workgroup; n: workgroups that have rows then
    constexpr int per = 64 / (D / VEC);
    a.rows = 1;
    while (a.rows < per && a.rows < max_new) a.rows *= 2;
    const int64_t x = ((int64_t)max_new + a.rows - 1) / a.rows, y = (a.pairs * a.rows + per - 1) / per;
    // As many workgroups for every sequence and head need no search, but those of short ones stand idle, some 1000 a microsecond.  Both ways, us a call: one
    // prompt of 65536 tokens beside 127 sequences with a new row 89.6, looked up 8.3; of 4096 beside 63 11.3 / 5.8; of 65536 beside one 9.0 / 7.6 (2046 idle);
    // 16 of 4000 to 64000 42.5 / 35.0; of 1024 beside 63 5.8 / 6.0 (1890 idle); 65536 alone 6.6 / 6.9.
    if (y > 65535 || x * y - n > 2000) {
        if (!cache::fits_launch(n, 64)) return INFLLMV2_ERR_UNSUPPORTED;
        if (codes) hipLaunchKernelGGL((cache_compress_kernel<T, D, true, true>), dim3((unsigned)n), dim3(64), 0, stream, a);
        else hipLaunchKernelGGL((cache_compress_kernel<T, D, false, true>), dim3((unsigned)n), dim3(64), 0, stream, a);
    } else {
        if (!cache::fits_launch(x, 64)) return INFLLMV2_ERR_UNSUPPORTED;
        const dim3 grid((unsigned)x, (unsigned)y);
        if (codes) hipLaunchKernelGGL((cache_compress_kernel<T, D, true, false>), grid, dim3(64), 0, stream, a);
        else hipLaunchKernelGGL((cache_compress_kernel<T, D, false, false>), grid, dim3(64), 0, stream, a);
    }
    return hip_status(hipGetLastError());
}

}  // namespace

}  // namespace ifv2

extern "C" int infllmv2_cache_compress_k(const infllmv2_params *p, const infllmv2_cache *c, float *kc_cache_d, int64_t kc_head_stride,
                                         const int32_t *prev_lens_h, const int32_t *prev_lens_d, const int32_t *ctx_lens_h,
                                         const int32_t *ctx_lens_d, int32_t batch, void *stream) {
    using namespace ifv2;
    int st = check_params(p);
    if (st) return st;
    if (batch < 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (batch == 0) return INFLLMV2_OK;
    if (prev_lens_h == nullptr || prev_lens_d == nullptr || ctx_lens_h == nullptr || ctx_lens_d == nullptr)
        return INFLLMV2_ERR_INVALID_ARGUMENT;
    int max_new = 0, max_nc = 0, max_ctx = 0;
    const int shift = p->head_dim == 128 ? 2 : 3;            // rows of a workgroup, as in the kernel
    int64_t items = 0;
    for (int b = 0; b < batch; ++b) {
        if (prev_lens_h[b] < 0 || ctx_lens_h[b] < prev_lens_h[b] || ctx_lens_h[b] > INT32_MAX - kBlock) return INFLLMV2_ERR_INVALID_ARGUMENT;
        const int n1 = num_cmp(ctx_lens_h[b], p->cmp_len, p->cmp_stride);
        const int grown = n1 - num_cmp(prev_lens_h[b], p->cmp_len, p->cmp_stride);
        if (grown > max_new) max_new = grown;
        items += ((int64_t)grown + (1 << shift) - 1) >> shift;
        if (n1 > max_nc) max_nc = n1;
        if (ctx_lens_h[b] > max_ctx) max_ctx = ctx_lens_h[b];
    }
    if (max_new == 0) return INFLLMV2_OK;
    if (kc_cache_d == nullptr || kc_head_stride < (int64_t)max_nc * p->head_dim) return INFLLMV2_ERR_INVALID_ARGUMENT;
    st = cache::check(p, c, max_ctx, false);
    if (st) return st;
    items *= p->num_kv_heads;
    CompressArgs a{cache::args(p, c), kc_cache_d, kc_head_stride, prev_lens_d, ctx_lens_d, batch, (int64_t)batch * p->num_kv_heads, p->cmp_len, p->cmp_stride, 1};
    const bool codes = c->kv_type == INFLLMV2_CACHE_E4M3;
    const hipStream_t s = (hipStream_t)stream;
    if (p->head_dim == 128)
        return p->dtype == INFLLMV2_BF16 ? launch_t<bf16_t, 128>(a, codes, max_new, items, s) : launch_t<float, 128>(a, codes, max_new, items, s);
    return p->dtype == INFLLMV2_BF16 ? launch_t<bf16_t, 64>(a, codes, max_new, items, s) : launch_t<float, 64>(a, codes, max_new, items, s);
}
