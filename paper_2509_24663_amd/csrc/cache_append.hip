// New keys and values into the pages of each sequence's cache, keys turned by their positions on the way; the pages hold the data's type or e4m3 codes
// with a power-of-two scale per page and head.
//
// A workgroup owns what a call writes to one (page, KV head) of K or of V: up to 64 rows.  So the page's scale is one workgroup's business: it
// turns its rows in registers, takes the largest magnitude over them (and, where a page is continued, the scale that the page has: a scale
// only grows), rounds once, and rounds the older codes again if the scale grew.  No atomics, no second pass over the new rows.
// A thread owns eight pair numbers of a row (16 channels; rotary.h says which) of every kRows-th row.
#include "cache.h"
#include "gen_unit.h"
#include "rotary.h"

namespace ifv2 {

namespace {

constexpr int kThreads = 256;

struct AppendArgs {
    cache::Args c;
    rotary::Args r;
    const char *k, *v;
    int64_t tok_stride, head_stride;       // of the new rows, elements
    const int32_t *cu, *prev, *pos;
    int batch;
    int single;                            // every sequence has new tokens, all in one page: item = sequence
};

template <typename T>
__device__ inline float element(const T *p) { return Elem<T>::load(p); }

// the 16 channels of the pair numbers q .. q + 7 as (x[i], y[i]), i = 0..7
template <typename T>
__device__ inline void load_pairs(const rotary::Args &r, int q, const T *row, float (&x)[8], float (&y)[8]) {
    typedef typename gen::Unaligned<typename std::conditional<sizeof(T) == 2, uint16_t, float>::type, 8>::type Vec;
    auto wide = [](auto e) -> float {
        if constexpr (sizeof(T) == 2) return bf16_to_float(e);
        else return e;
    };
    if (r.pairs % 8 != 0) {                                                  // the eight may straddle the two kinds of pairs
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = element(row + rotary::first_channel(r, q + i));
            y[i] = element(row + rotary::second_channel(r, q + i));
        }
    } else if (q < r.pairs && !r.interleaved) {
        const Vec a = *reinterpret_cast<const Vec *>(row + q), b = *reinterpret_cast<const Vec *>(row + q + r.pairs);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = wide(a[i]), y[i] = wide(b[i]);
    } else {
        const Vec a = *reinterpret_cast<const Vec *>(row + 2 * q), b = *reinterpret_cast<const Vec *>(row + 2 * q + 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = wide(i < 4 ? a[(2 * i) & 7] : b[(2 * i) & 7]), y[i] = wide(i < 4 ? a[(2 * i + 1) & 7] : b[(2 * i + 1) & 7]);
    }
}

// the same channels of a row of codes, from values in units of the scale
__device__ inline void store_codes(const rotary::Args &r, int q, char *row, const float (&x)[8], const float (&y)[8]) {
    if (r.pairs % 8 != 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            row[rotary::first_channel(r, q + i)] = (char)cache::code(x[i]);
            row[rotary::second_channel(r, q + i)] = (char)cache::code(y[i]);
        }
    } else if (q < r.pairs && !r.interleaved) {
        *reinterpret_cast<uint2 *>(row + q) = uint2{cache::codes4(x[0], x[1], x[2], x[3]), cache::codes4(x[4], x[5], x[6], x[7])};
        *reinterpret_cast<uint2 *>(row + q + r.pairs) = uint2{cache::codes4(y[0], y[1], y[2], y[3]), cache::codes4(y[4], y[5], y[6], y[7])};
    } else {
        *reinterpret_cast<uint4 *>(row + 2 * q) = uint4{cache::codes4(x[0], y[0], x[1], y[1]), cache::codes4(x[2], y[2], x[3], y[3]),
                                                        cache::codes4(x[4], y[4], x[5], y[5]), cache::codes4(x[6], y[6], x[7], y[7])};
    }
}

// the same channels of a row of the data's type
template <typename T>
__device__ inline void store_native(const rotary::Args &r, int q, T *row, const float (&x)[8], const float (&y)[8]) {
    if (r.pairs % 8 != 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            Elem<T>::store(row + rotary::first_channel(r, q + i), x[i]);
            Elem<T>::store(row + rotary::second_channel(r, q + i), y[i]);
        }
    } else if (q < r.pairs && !r.interleaved) {
        gen::store_row<T, 8>(row + q, x);
        gen::store_row<T, 8>(row + q + r.pairs, y);
    } else {
        float a[8], b[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[2 * i] = x[i], a[2 * i + 1] = y[i], b[2 * i] = x[4 + i], b[2 * i + 1] = y[4 + i];
        gen::store_row<T, 8>(row + 2 * q, a);
        gen::store_row<T, 8>(row + 2 * q + 8, b);
    }
}

// pages that n new tokens behind prev cached ones fall into
__host__ __device__ inline int pages_touched(int prev, int n) { return n == 0 ? 0 : (prev + n - 1) / kBlock - prev / kBlock + 1; }

template <typename T, int D, bool CODES>
__global__ void __launch_bounds__(kThreads) cache_append_kernel(AppendArgs a) {
    constexpr int PER = D / 16;                       // threads per row
    constexpr int ROWS = kThreads / PER, STEPS = kBlock / ROWS;
    __shared__ int64_t s_item[3];
    __shared__ float s_top[kThreads / 64];
    const int h = blockIdx.y, tid = threadIdx.x;
    const bool values = blockIdx.z != 0;
    int seq = blockIdx.x, nth = 0;
    if (!a.single) {
        int64_t before;
        seq = cache::find_item(a.batch, blockIdx.x, nth, before, s_item,
                               [&](int s) { return pages_touched(a.prev[s], a.cu[s + 1] - a.cu[s]); }, [](int) { return 0; });
        if (seq >= a.batch) return;
    }
    const int prev = a.prev[seq], row0 = a.cu[seq], n = a.cu[seq + 1] - row0;
    const int block = prev / kBlock + nth;
    const int page = a.c.page(seq, block);
    if (page < 0) return;
    const int first = max(prev, block * kBlock), end = min(prev + n, block * kBlock + kBlock);     // tokens of this page that are new
    rotary::Args r = a.r;
    if (values) r.pairs = 0;
    const int q = (tid % PER) * 8, t0 = block * kBlock + tid / PER;
    const T *src = reinterpret_cast<const T *>(values ? a.v : a.k) + (int64_t)(row0 - prev) * a.tok_stride + h * a.head_stride;
    char *dst = (values ? a.c.v : a.c.k) + a.c.at(page, h);
    float x[STEPS][8], y[STEPS][8], top = 0.f;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int t = t0 + i * ROWS;
        if (t >= first && t < end) {
            load_pairs(r, q, src + (int64_t)t * a.tok_stride, x[i], y[i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = y[i][e] = 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int t = t0 + i * ROWS;
        if (q < r.pairs && t >= first && t < end) {
            const int32_t pos = a.pos ? a.pos[row0 + t - prev] : t;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (q + e >= r.pairs) continue;
                const float2 cs = rotary::cos_sin(pos, r.turns[q + e], r.magnitude);
                const float2 z = rotary::turn(x[i][e], y[i][e], cs.x, cs.y);
                x[i][e] = z.x;
                y[i][e] = z.y;
            }
        }
        if constexpr (CODES) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float u = fabsf(x[i][e]), w = fabsf(y[i][e]);
                top = fmaxf(top, fmaxf(u <= 3.4028234e38f ? u : 0.f, w <= 3.4028234e38f ? w : 0.f));
            }
        }
    }
    if constexpr (!CODES) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int t = t0 + i * ROWS;
            if (t >= first && t < end) store_native(r, q, reinterpret_cast<T *>(dst + (t - block * kBlock) * a.c.tok_stride), x[i], y[i]);
        }
    } else {
        float *scale = (values ? a.c.vs : a.c.ks) + (int64_t)page * a.c.hkv + h;
        const bool continued = first > block * kBlock;
        const float was = continued ? *scale : 0.f;
        top = wave_max(top);
        if ((tid & 63) == 0) s_top[tid >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) top = fmaxf(top, s_top[w]);
        const float now = fmaxf(cache::scale_for(top), was), inv = cache::reciprocal_of_power(now);
        if (continued && now != was) {                // the older rows, sixteen codes at a time
            const float down = was * inv;
            for (int i = tid; i < (first - block * kBlock) * PER; i += kThreads) {
                uint4 *at = reinterpret_cast<uint4 *>(dst + (i / PER) * a.c.tok_stride + (i % PER) * 16);
                uint4 old = *at;
                uint32_t w[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
                    w[j] = cache::codes4(lo[0] * down, lo[1] * down, hi[0] * down, hi[1] * down);
                }
                *at = uint4{w[0], w[1], w[2], w[3]};
            }
        }
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int t = t0 + i * ROWS;
            if (t < first || t >= end) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] *= inv, y[i][e] *= inv;
            store_codes(r, q, dst + (t - block * kBlock) * a.c.tok_stride, x[i], y[i]);
        }
        if (tid == 0 && now != was) *scale = now;
    }
}

template <typename T, int D>
int launch_t(const AppendArgs &a, bool codes, unsigned items, hipStream_t stream) {
    const dim3 grid(items, a.c.hkv, 2);
    if (codes) hipLaunchKernelGGL((cache_append_kernel<T, D, true>), grid, dim3(kThreads), 0, stream, a);
    else hipLaunchKernelGGL((cache_append_kernel<T, D, false>), grid, dim3(kThreads), 0, stream, a);
    return hip_status(hipGetLastError());
}

}  // namespace

int cache::check(const infllmv2_params *p, const infllmv2_cache *c, int max_ctx, bool values) {
    if (c == nullptr) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (c->kv_type != INFLLMV2_CACHE_NATIVE && c->kv_type != INFLLMV2_CACHE_E4M3) return INFLLMV2_ERR_UNSUPPORTED;
    const int e = c->kv_type == INFLLMV2_CACHE_E4M3 ? 1 : p->dtype == INFLLMV2_BF16 ? 2 : 4;
    if (c->num_pages < 1 || c->reserved != 0 || c->page_table_d == nullptr || c->k_d == nullptr || (values && c->v_d == nullptr))
        return INFLLMV2_ERR_INVALID_ARGUMENT;
    if ((((uintptr_t)c->k_d | (values ? (uintptr_t)c->v_d : 0)) & 15) != 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (c->page_stride < p->head_dim || c->head_stride < p->head_dim || c->tok_stride < p->head_dim) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (c->page_stride * e % 16 != 0 || c->head_stride * e % 16 != 0 || c->tok_stride * e % 16 != 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (e == 1 && (c->k_scale_d == nullptr || (values && c->v_scale_d == nullptr))) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (c->table_stride < (max_ctx + (int64_t)kBlock - 1) / kBlock) return INFLLMV2_ERR_INVALID_ARGUMENT;
    return INFLLMV2_OK;
}

cache::Args cache::args(const infllmv2_params *p, const infllmv2_cache *c) {
    const int e = c->kv_type == INFLLMV2_CACHE_E4M3 ? 1 : p->dtype == INFLLMV2_BF16 ? 2 : 4;
    return Args{(char *)c->k_d, (char *)c->v_d, c->page_stride * e, c->head_stride * e, c->tok_stride * e, c->k_scale_d, c->v_scale_d,
                c->page_table_d, c->table_stride, c->num_pages, p->num_kv_heads};
}

}  // namespace ifv2

extern "C" int infllmv2_cache_append(const infllmv2_params *p, const infllmv2_cache *c, const infllmv2_rotary *r, const void *k_d,
                                     const void *v_d, int64_t kv_tok_stride, int64_t kv_head_stride, const int32_t *cu_new_h,
                                     const int32_t *cu_new_d, const int32_t *prev_lens_h, const int32_t *prev_lens_d,
                                     const int32_t *pos_d, int32_t batch, void *stream) {
    using namespace ifv2;
    int st = check_params(p);
    if (st) return st;
    if (r != nullptr) {
        st = rotary::check(p, r);
        if (st) return st;
    }
    int64_t total;
    int32_t max_len;
    st = check_cu(cu_new_h, cu_new_d, batch, &total, &max_len);
    if (st) return st;
    if (total == 0) return INFLLMV2_OK;
    if (k_d == nullptr || v_d == nullptr || prev_lens_h == nullptr || prev_lens_d == nullptr || (r != nullptr && r->turns_d == nullptr))
        return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (kv_tok_stride < p->head_dim || kv_head_stride < p->head_dim) return INFLLMV2_ERR_INVALID_ARGUMENT;
    int64_t items = 0;
    int max_ctx = 0;
    bool single = true;
    for (int b = 0; b < batch; ++b) {
        const int n = cu_new_h[b + 1] - cu_new_h[b];
        if (prev_lens_h[b] < 0 || prev_lens_h[b] > INT32_MAX - kBlock - n) return INFLLMV2_ERR_INVALID_ARGUMENT;
        const int pages = pages_touched(prev_lens_h[b], n);
        items += pages;
        single = single && pages == 1;
        if (n > 0 && prev_lens_h[b] + n > max_ctx) max_ctx = prev_lens_h[b] + n;
    }
    st = cache::check(p, c, max_ctx, true);
    if (st) return st;
    if (p->num_kv_heads > 65535) return INFLLMV2_ERR_UNSUPPORTED;
    AppendArgs a{cache::args(p, c), r ? rotary::args(r) : rotary::Args{nullptr, 0, 0, 1.f}, (const char *)k_d, (const char *)v_d,
                 kv_tok_stride, kv_head_stride, cu_new_d, prev_lens_d, pos_d, batch, single};
    const bool codes = c->kv_type == INFLLMV2_CACHE_E4M3;
    const hipStream_t s = (hipStream_t)stream;
    if (p->head_dim == 128)
        return p->dtype == INFLLMV2_BF16 ? launch_t<bf16_t, 128>(a, codes, (unsigned)items, s) : launch_t<float, 128>(a, codes, (unsigned)items, s);
    return p->dtype == INFLLMV2_BF16 ? launch_t<bf16_t, 64>(a, codes, (unsigned)items, s) : launch_t<float, 64>(a, codes, (unsigned)items, s);
}
