// New keys and values into the pages of each sequence's cache, keys turned by their positions on the way; the pages hold the data's type or e4m3 codes
// with a power-of-two scale per page and head.
//
// A workgroup owns what a call writes to one page of K or of V, for one KV head or (many pages) for several in turn: up to 64 rows.  So the page's
// scale is one workgroup's business: it turns its rows in registers, takes the largest magnitude over them (and, where a page is continued, the
// scale that the page has: a scale only grows), rounds once, and rounds the older codes again if the scale grew.  No atomics, no second pass over
// the new rows.  The angles are worked out once for all heads of a workgroup.
// A thread owns eight pair numbers of a row (16 channels; rotary.h says which); all 64 rows of a page have threads of their own, so that a page is requested at once, and
// in front of the page's number, which is one more trip to memory.
//
// Bound: HBM for prompts.  6 prompts of 24001 tokens, 2 heads of 128, bf16 to e4m3, 175 MB: 38.1 us, 4.6 TB/s read and written, of the 4.9 of a large copy.
// Before: rows behind the page's number, half the threads 53.8; maxima of floats, each made quiet first, frequencies one by one 49.2; the addresses of
// single channels kept beside (122 registers for 90) 45.5; sums over the batch in 64 bits through LDS 41.2.  One token of 16 sequences: 3.6 us; 3 x 511
// tokens, fp32, d 64: 4.6: launch, page lookup and rows, one after the other.
#include "cache.h"
#include "gen_unit.h"
#include "rotary.h"

namespace ifv2 {

namespace {

struct AppendArgs {
    cache::Args c;
    rotary::Args r;
    const char *k, *v;
    int64_t tok_stride, head_stride;       // of the new rows, elements
    const int32_t *cu, *prev, *pos;
    int batch;
    int single;                            // every sequence has new tokens, all in one page: item = sequence
    int heads;                             // of a workgroup
};

// The 16 channels of the pair numbers q .. q + 7: two runs of eight, as requested ..
template <typename T>
struct Pairs {
    typedef typename gen::Unaligned<typename std::conditional<sizeof(T) == 2, uint16_t, float>::type, 8>::type Vec;
    Vec a, b;
    // (r.pairs % 8 == 0)
    __device__ inline void load(const rotary::Args &r, int q, const T *row) {
        const bool half = q < r.pairs && !r.interleaved;
        a = *reinterpret_cast<const Vec *>(row + (half ? q : 2 * q));
        b = *reinterpret_cast<const Vec *>(row + (half ? q + r.pairs : 2 * q + 8));
    }
    static __device__ inline float wide(uint16_t e) { return bf16_to_float(e); }
    static __device__ inline float wide(float e) { return e; }
    // .. and as pairs (x[i], y[i])
    __device__ inline void spread(const rotary::Args &r, int q, float (&x)[8], float (&y)[8]) const {
        if (q < r.pairs && !r.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = wide(a[i]), y[i] = wide(b[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = wide(i < 4 ? a[(2 * i) & 7] : b[(2 * i) & 7]), y[i] = wide(i < 4 ? a[(2 * i + 1) & 7] : b[(2 * i + 1) & 7]);
        }
    }
};

// the same channels of a row of codes, from values in units of the scale
template <bool FITS, bool RUNS>
__device__ inline void store_codes(const rotary::Args &r, int q, char *row, const float (&x)[8], const float (&y)[8]) {
    if (!RUNS && r.pairs % 8 != 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            row[rotary::first_channel(r, q + i)] = (char)cache::code(x[i]);
            row[rotary::second_channel(r, q + i)] = (char)cache::code(y[i]);
        }
    } else if (q < r.pairs && !r.interleaved) {
        *reinterpret_cast<uint2 *>(row + q) = uint2{cache::codes4<FITS>(x[0], x[1], x[2], x[3]), cache::codes4<FITS>(x[4], x[5], x[6], x[7])};
        *reinterpret_cast<uint2 *>(row + q + r.pairs) = uint2{cache::codes4<FITS>(y[0], y[1], y[2], y[3]), cache::codes4<FITS>(y[4], y[5], y[6], y[7])};
    } else {
        *reinterpret_cast<uint4 *>(row + 2 * q) = uint4{cache::codes4<FITS>(x[0], y[0], x[1], y[1]), cache::codes4<FITS>(x[2], y[2], x[3], y[3]),
                                                        cache::codes4<FITS>(x[4], y[4], x[5], y[5]), cache::codes4<FITS>(x[6], y[6], x[7], y[7])};
    }
}

// the same channels of a row of the data's type
template <typename T, bool RUNS>
__device__ inline void store_native(const rotary::Args &r, int q, T *row, const float (&x)[8], const float (&y)[8]) {
    if (!RUNS && r.pairs % 8 != 0) {
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

// The bits of |x|: as whole numbers they are in the order of the magnitudes, infinities above every number and NaN above those, and a maximum of them is one instruction
// for three (of floats the compiler has every input made quiet first).
__device__ inline uint32_t magnitude_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }
// over the wavefront, for all of it
__device__ inline uint32_t wave_top(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_readlane(cache::wave_scan((int)x, [](int a, int b) { return (int)max((uint32_t)a, (uint32_t)b); }), 63);
}

// pages that n new tokens behind prev cached ones fall into
__host__ __device__ inline int pages_touched(int prev, int n) { return n == 0 ? 0 : (prev + n - 1) / kBlock - prev / kBlock + 1; }

// RUNS: the pairs that are turned are a multiple of eight (the single channels' addresses of the other form take registers and instructions)
template <typename T, int D, bool CODES, bool RUNS>
__global__ void __launch_bounds__(4 * D) cache_append_kernel(AppendArgs a) {
    constexpr int PER = D / 16, kThreads = 4 * D;     // threads per row; every row of a page has its own
    __shared__ int s_item[6];
    __shared__ uint32_t s_top[2][2][kThreads / 64];   // by turns
    const int tid = threadIdx.x, h0 = blockIdx.y * a.heads, h1 = min(h0 + a.heads, a.c.hkv);
    const bool values = blockIdx.z != 0;
    int seq = (int)blockIdx.x, nth = 0, prev, row0, n;
    if (a.single) {
        prev = a.prev[seq];
        row0 = a.cu[seq];
        n = a.cu[seq + 1] - row0;
    } else {
        int before;
        cache::Facts f;
        seq = cache::find_item(a.batch, (int)blockIdx.x, nth, before, f, s_item,
                               [&](int s) { return pages_touched(a.prev[s], a.cu[s + 1] - a.cu[s]); }, [](int) { return 0; },
                               [&](int s, int i) { return i == 0 ? a.prev[s] : a.cu[s + i - 1]; });
        if (seq >= a.batch) return;
        prev = f.x[0];
        row0 = f.x[1];
        n = f.x[2] - row0;
    }
    const int block = prev / kBlock + nth;
    const int first = max(prev, block * kBlock), end = min(prev + n, block * kBlock + kBlock);     // tokens of this page that are new
    rotary::Args r = a.r;
    if (values) r.pairs = 0;
    const int q = (tid % PER) * 8, t = block * kBlock + tid / PER;
    const bool mine = t >= first && t < end;
    const T *src = reinterpret_cast<const T *>(values ? a.v : a.k) + (int64_t)(row0 + t - prev) * a.tok_stride;
    const bool runs = RUNS || r.pairs % 8 == 0;             // the eight are pairs of one kind
    Pairs<T> raw;
    if (mine && runs) raw.load(r, q, src + h0 * a.head_stride);      // (beside the page's number, not behind it)
    const int page = a.c.page(seq, block);
    if (page < 0) return;
    float co[8], si[8];
    const bool turns = mine && q < r.pairs;
    if (turns) {
        const int32_t pos = a.pos ? a.pos[row0 + t - prev] : t;
        uint64_t f[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = r.turns[runs ? q + e : min(q + e, r.pairs - 1)];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 cs = rotary::cos_sin<T>(pos, f[e], r.magnitude);
            co[e] = cs.x;
            si[e] = cs.y;
        }
    }
    for (int h = h0, turn = 0; h < h1; ++h, turn ^= 1) {
        char *page_at = (values ? a.c.v : a.c.k) + a.c.at(page, h), *dst = page_at + (t - block * kBlock) * a.c.tok_stride;
        float x[8], y[8];                             // (of a row that is not written: nothing)
        if (mine && runs) {
            raw.spread(r, q, x, y);
            if (h + 1 < h1) raw.load(r, q, src + (h + 1) * a.head_stride);
        } else if (mine) {
            const T *row = src + h * a.head_stride;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = Elem<T>::load(row + rotary::first_channel(r, q + e));
                y[e] = Elem<T>::load(row + rotary::second_channel(r, q + e));
            }
        }
        if (turns && runs) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 z = rotary::turn(x[e], y[e], co[e], si[e]);
                x[e] = z.x;
                y[e] = z.y;
            }
        } else if (turns) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 z = rotary::turn(x[e], y[e], co[e], si[e]);
                x[e] = q + e < r.pairs ? z.x : x[e];
                y[e] = q + e < r.pairs ? z.y : y[e];
            }
        }
        if constexpr (!CODES) {
            if (mine) store_native<T, RUNS>(r, q, reinterpret_cast<T *>(dst), x, y);
        } else {
            uint32_t bits = 0;
            if (mine) {
#pragma unroll
                for (int e = 0; e < 8; ++e) bits = max(bits, max(magnitude_bits(x[e]), magnitude_bits(y[e])));
            }
            float *scale = (values ? a.c.vs : a.c.ks) + (int64_t)page * a.c.hkv + h;
            const bool continued = first > block * kBlock;
            const float was = continued ? *scale : 0.f;
            auto over_all = [&](uint32_t v, uint32_t (&s)[kThreads / 64]) {
                v = wave_top(v);
                if ((tid & 63) == 0) s[tid >> 6] = v;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < kThreads / 64; ++w) v = max(v, s[w]);
                return v;
            };
            bits = over_all(bits, s_top[turn][0]);
            const bool fits = bits <= __float_as_uint(448.f * 0x1p119f);
            if (!fits) {                              // infinities, NaN, or numbers that no scale is large enough for: the finite ones again
                bits = 0;
                if (mine) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t u = magnitude_bits(x[e]), w = magnitude_bits(y[e]);
                        bits = max(bits, max(u < 0x7f800000u ? u : 0u, w < 0x7f800000u ? w : 0u));
                    }
                }
                bits = over_all(bits, s_top[turn][1]);
            }
            const float now = fmaxf(cache::scale_for(__uint_as_float(bits)), was), inv = cache::reciprocal_of_power(now);
            if (continued && now != was) {            // the older rows, sixteen codes at a time
                const float down = was * inv;
                for (int i = tid; i < (first - block * kBlock) * PER; i += kThreads) {
                    uint4 *at = reinterpret_cast<uint4 *>(page_at + (i / PER) * a.c.tok_stride + (i % PER) * 16);
                    uint4 old = *at;
                    uint32_t w[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
                        w[j] = cache::codes4<true>(lo[0] * down, lo[1] * down, hi[0] * down, hi[1] * down);
                    }
                    *at = uint4{w[0], w[1], w[2], w[3]};
                }
            }
            if (mine) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= inv, y[e] *= inv;
                if (fits) store_codes<true, RUNS>(r, q, dst, x, y);
                else store_codes<false, RUNS>(r, q, dst, x, y);
            }
            if (tid == 0 && now != was) *scale = now;
        }
    }
}

template <typename T, int D>
int launch_t(const AppendArgs &a, bool codes, unsigned items, hipStream_t stream) {
    const dim3 grid(items, (a.c.hkv + a.heads - 1) / a.heads, 2);
    const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(4 * D), 0, stream, a); };
    const bool runs = a.r.pairs % 8 == 0;
    if (codes) launch(runs ? cache_append_kernel<T, D, true, true> : cache_append_kernel<T, D, true, false>);
    else launch(runs ? cache_append_kernel<T, D, false, true> : cache_append_kernel<T, D, false, false>);
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
    if (p->num_kv_heads > 65535 || !cache::fits_launch(items, 4 * p->head_dim)) return INFLLMV2_ERR_UNSUPPORTED;
    AppendArgs a{cache::args(p, c), r ? rotary::args(r) : rotary::Args{nullptr, 0, 0, 1.f}, (const char *)k_d, (const char *)v_d,
                 kv_tok_stride, kv_head_stride, cu_new_d, prev_lens_d, pos_d, batch, single, 1};
    // heads of a workgroup: all, while that leaves a few workgroups for each CU (the angles of a key page are worked out once for them)
    while (a.heads < p->num_kv_heads && items * 2 * ((p->num_kv_heads + 2 * a.heads - 1) / (2 * a.heads)) >= 1024) a.heads *= 2;
    const bool codes = c->kv_type == INFLLMV2_CACHE_E4M3;
    const hipStream_t s = (hipStream_t)stream;
    if (p->head_dim == 128)
        return p->dtype == INFLLMV2_BF16 ? launch_t<bf16_t, 128>(a, codes, (unsigned)items, s) : launch_t<float, 128>(a, codes, (unsigned)items, s);
    return p->dtype == INFLLMV2_BF16 ? launch_t<bf16_t, 64>(a, codes, (unsigned)items, s) : launch_t<float, 64>(a, codes, (unsigned)items, s);
}
