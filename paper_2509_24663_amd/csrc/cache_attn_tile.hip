// Attention of a chunk of a prompt over its paged cache, bf16 data: tiles of 8 x CG groups of 16 columns (a column is a token and a head of one KV head).
//
// The workgroup's eight wavefronts go through the pages together and each keeps CG column groups (CG = 3, head dim 64: 4) with their queries and sums in
// registers, so that an operand read from LDS feeds CG products; the other way round (one group per wavefront) LDS reads bound the kernel at half the
// matrix cores' rate.  S^T = K Q^T and O^T += V^T P^T on 16x16x32 products; a lane's logits of a half page are eight consecutive keys of one
// column, which is the operand that the second product wants.
// A page is requested while the one before it is worked on: half of the wavefronts hold its K, half its V, in registers, widen them (codes times
// the page's scale: exact in bf16) and write them to the other of two LDS buffers, V transposed: a thread holds 8 keys of 4 channels, so it
// writes whole 16-byte operand pieces.  One barrier per page.
// Rounding: weights go into the second product as bf16 (2^-9 of each, as the output's own rounding); their sum takes them as they are.  References move only
// where eight weights of a lane add up to more than kSlack, so a weight is below it.
#include "attn_unit.h"
#include "cache_attn.h"

namespace ifv2 {

namespace {

using namespace gen;
using attn_unit::lds_read16;
using cache_attn::AttnArgs;
using cache_attn::kLn2;
using cache_attn::kLowest;

constexpr int NW = 8;
constexpr int kThreads = NW * 64;
constexpr float kSlack = 64.f, kNoReference = -1e38f;
constexpr int groups_of(int d) { return d == 128 ? 3 : 4; }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <bool UPPER>
__device__ inline uint32_t widen(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, UPPER));
}
__device__ inline uint32_t pack(float a, float b) {          // nearest even
    const bf16x2 x = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, x);
}
// all ones in the elements of w that are infinities or NaN
template <bool CODES>
__device__ inline uint32_t not_finite(uint32_t w) {
    if (CODES) return ((((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xffu;
    return ((((w & 0x7fff7fffu) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu;
}
__device__ inline float rows_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float rows_add(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}
__device__ inline void lds_write16(uint32_t at, u32x4 x) {
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    *(lds_u32x4 *)(uintptr_t)at = x;
}

// A page in LDS: K [64 keys][D] and V^T [D][64 keys], bf16, 16-byte chunks of a row swizzled so that the sixteen lanes of an operand read (rows 8 (m / 4) + m % 4
// of K, 16 consecutive rows of V^T, one logical chunk) and the lanes of a write take different positions.
template <int D>
struct Page {
    static constexpr uint32_t kKBytes = 64 * D * 2, kBytes = 2 * kKBytes;
    static __device__ inline uint32_t k_swizzle(int row) {
        return D == 128 ? 4 * ((row >> 3) & 3) + (row & 3) : 2 * ((row >> 3) & 3) + ((row >> 1) & 1);
    }
    static __device__ inline uint32_t v_swizzle(int ch) { return ((ch >> 1) & 7) ^ ((ch >> 4) & 1); }
    static __device__ inline uint32_t k_at(int row, int chunk) { return (uint32_t)row * (2 * D) + ((chunk ^ k_swizzle(row)) << 4); }
    static __device__ inline uint32_t v_at(int ch, int octet) { return kKBytes + (uint32_t)ch * 128 + ((octet ^ v_swizzle(ch)) << 4); }
};

template <int D, int CG, bool CODES>
__global__ void __launch_bounds__(kThreads, 2) cache_attn_tile_kernel(AttnArgs a) {
    constexpr int KS = D / 32, DT = D / 16;
    constexpr int KB = CODES ? 1 : 2;                               // bytes of an element
    extern __shared__ __attribute__((aligned(1024))) char smem[];   // two pages
    __shared__ int64_t s_item[3];
    __shared__ int s_odd;                                           // a value of a page's edge (see write) is not finite
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m = lane & 15, g = lane >> 4, hkv = a.c.hkv, G = a.hq / hkv, GT = a.group_tokens;

    int rem;
    int64_t slot0;
    const int seq = cache::find_item(a.batch, blockIdx.x, rem, slot0, s_item,
        [&](int s) {
            const int n = a.cu[s + 1] - a.cu[s], len = a.ctx[s];
            return (int64_t)a.tiles(n, len) * hkv * a.most_splits(n, len);
        },
        [&](int s) {
            const int n = a.cu[s + 1] - a.cu[s], len = a.ctx[s], sp = a.most_splits(n, len);
            return sp > 1 ? (int64_t)a.tiles(n, len) * hkv * sp : 0;
        });
    if (seq >= a.batch) return;
    const int row0 = a.cu[seq], n = a.cu[seq + 1] - row0, len = a.ctx[seq];
    const int per = a.most_splits(n, len), ntiles = a.tiles(n, len);
    const int split = rem % per, th = rem / per, h = th % hkv, tile = ntiles - 1 - th / hkv;          // (longest first)
    const int64_t slot = slot0 + (int64_t)(tile * hkv + h) * per + split;
    const int T0 = GT * NW * CG, first = tile * T0, ntok = min(T0, n - first);
    const int pos0 = len - n + first, pos_last = pos0 + ntok - 1;
    const int nsplit = a.splits(len, pos_last);
    if (split >= nsplit) return;

    int ti[CG];
    bool used[CG];
    bf16x8 qf[CG][KS];
#pragma unroll
    for (int x = 0; x < CG; ++x) {
        ti[x] = (w * CG + x) * GT + m / G;
        used[x] = m / G < GT && ti[x] < ntok;
        const int64_t row = row0 + first + (used[x] ? ti[x] : 0);
        const int qh = h * G + (used[x] ? m % G : 0);
        const uint16_t *q = reinterpret_cast<const uint16_t *>(a.q) + (row * a.hq + qh) * D;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[x][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u16x8_u *>(q + 32 * s + 8 * g));
    }
    const int wave_first = w * CG * GT;                             // tokens of this wavefront: from here ..
    const int wave_last = min(wave_first + CG * GT, ntok) - 1;      // .. to here (none: last < first)
    const float c = a.scale * kLog2e;

    f32x4 acc[CG][DT];
    float ref[CG], sum[CG];
#pragma unroll
    for (int x = 0; x < CG; ++x) {
        ref[x] = kNoReference;
        sum[x] = 0.f;
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[x][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const uint32_t lds = __builtin_amdgcn_readfirstlane(attn_unit::lds_address(smem));
    const uint32_t k_lane = Page<D>::k_at(8 * (m >> 2) + (m & 3), g), v_lane = Page<D>::v_at(m, g);
    const uint32_t tok = (uint32_t)a.c.tok_stride;
    // what this thread brings of a page: threads 0..255 a quarter of a K row, the next 2 D eight keys of four channels of V
    const bool is_k = w < 4, is_v = tid >= 256 && tid < 256 + 2 * D;
    const int k_row = tid >> 2, quarter = tid & 3, vid = tid - 256, octet = vid / (D / 4), ch0 = vid % (D / 4) * 4;
    const uint32_t from = is_k ? k_row * tok + quarter * (D / 4 * KB) : 8 * octet * tok + ch0 * KB;
    constexpr int KW = D / 4 * KB / 16, VW = KB;
    uint32_t raw[4 * KW > 8 * VW ? 4 * KW : 8 * VW];
    auto bring = [&](int page) {
        const char *base = (is_k ? a.c.k : a.c.v) + a.c.at(page, h);
        if (is_k) {
#pragma unroll
            for (int i = 0; i < KW; ++i) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(base + from + 16 * i);
#pragma unroll
                for (int e = 0; e < 4; ++e) raw[4 * i + e] = x[e];
            }
        } else if (is_v) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (CODES) {
                    raw[i] = *reinterpret_cast<const uint32_t *>(base + from + i * tok);
                } else {
                    const uint2 x = *reinterpret_cast<const uint2 *>(base + from + i * tok);
                    raw[2 * i] = x.x, raw[2 * i + 1] = x.y;
                }
            }
        }
    };
    auto write = [&](int buf, int key0, float scale) {
        const uint32_t at = lds + buf * Page<D>::kBytes;
        if (is_k) {
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {                      // 8 channels at a time
                u32x4 x;
                if constexpr (CODES) x = u32x4{widen<false>(raw[2 * i], scale), widen<true>(raw[2 * i], scale), widen<false>(raw[2 * i + 1], scale), widen<true>(raw[2 * i + 1], scale)};
                else x = u32x4{raw[4 * i], raw[4 * i + 1], raw[4 * i + 2], raw[4 * i + 3]};
                lds_write16(at + Page<D>::k_at(k_row, quarter * (D / 32) + i), x);
            }
        } else if (is_v) {
            if (key0 + kBlock - 1 > pos0) {                         // a page of which not all is visible to all tokens of the tile
                uint32_t odd = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int e = 0; e < VW; ++e) {
                        uint32_t &x = raw[VW * i + e];
                        const uint32_t o = not_finite<CODES>(x);
                        const bool any_sees = key0 + 8 * octet + i <= pos_last;
                        odd |= any_sees ? o : 0u;
                        x = any_sees ? x & ~o : 0u;
                    }
                if (odd != 0) s_odd = 1;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u32x4 x;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if constexpr (CODES) {
                        const uint32_t two = __builtin_amdgcn_perm(raw[2 * k + 1], raw[2 * k], j < 2 ? 0x05010400u : 0x07030602u);
                        x[k] = j & 1 ? widen<true>(two, scale) : widen<false>(two, scale);
                    } else {
                        const uint32_t lo = raw[4 * k + j / 2], hi = raw[4 * k + 2 + j / 2];
                        x[k] = j & 1 ? upper_halves(lo, hi) : lower_halves(lo, hi);
                    }
                }
                lds_write16(at + Page<D>::v_at(ch0 + j, octet), x);
            }
        }
    };

    // the pages of the split: lane l holds the l-th of the next 64
    const int e_end = min(a.pages(len, pos_last), (split + 1) * a.pps);
    int e0 = split * a.pps, list_page, list_key0 = 0;
    float list_scale = 1.f;
    uint64_t there = 0;
    auto next = [&](int &page, int &key0, float &scale) -> bool {   // the next page that is there
        while (there == 0) {
            if (e0 >= e_end) return false;
            const int j = e0 + lane;
            list_page = j < e_end ? a.c.page(seq, j) : -1;
            list_key0 = j * kBlock;
            if (CODES && list_page >= 0) list_scale = (is_k ? a.c.ks : a.c.vs)[(int64_t)list_page * hkv + h];
            there = __ballot(list_page >= 0);
            e0 += 64;
        }
        const int l = __ffsll((long long)there) - 1;
        there &= there - 1;
        page = __builtin_amdgcn_readlane(list_page, l);
        key0 = __builtin_amdgcn_readlane(list_key0, l);
        scale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(list_scale), l));
        return true;
    };
    int page, key0 = 0, next_key0 = 0, low = INT32_MAX;
    float scale = 1.f;
    bool here = next(page, key0, scale), more = false;
    if (tid == 0) s_odd = 0;
    if (here) {
        bring(page);
        __syncthreads();                                            // (s_odd)
        write(0, key0, scale);
        more = next(page, next_key0, scale);
        if (more) bring(page);
        low = key0;
        __syncthreads();
    }
    for (int buf = 0; here; buf ^= 1) {
        const bool edge = key0 + kBlock - 1 > pos0;
        if (wave_first <= wave_last && key0 <= pos0 + wave_last) {
            const uint32_t kp = lds + buf * Page<D>::kBytes + k_lane, vp = lds + buf * Page<D>::kBytes + v_lane;
#pragma unroll
            for (int hb = 0; hb < 2; ++hb) {
                f32x4 s[CG][2];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        const bf16x8 f = lds_read16((kp ^ (uint32_t)(64 * ks)) + (uint32_t)((32 * hb + 4 * kt) * 2 * D));
#pragma unroll
                        for (int x = 0; x < CG; ++x)
                            s[x][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, qf[x][ks], ks ? s[x][kt] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                    }
                if (edge) {
#pragma unroll
                    for (int x = 0; x < CG; ++x) {
                        const int lim = used[x] ? pos0 + ti[x] - (key0 + 32 * hb + 8 * g) : -1;
#pragma unroll
                        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[x][kt][r] = 4 * kt + r <= lim ? s[x][kt][r] : -INFINITY;
                    }
                }
                bf16x8 pb[CG];
#pragma unroll
                for (int x = 0; x < CG; ++x) {
                    float p[8], part = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        p[i] = exp2_fast(__builtin_fmaf(s[x][i >> 2][i & 3], c, -ref[x]));
                        part += p[i];
                    }
                    if (__any(part > kSlack)) {
                        float mx = s[x][0][0];
#pragma unroll
                        for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[x][i >> 2][i & 3]);
                        const float to = fmaxf(ref[x], rows_max(mx) * c), f = exp2_fast(ref[x] - to);
                        ref[x] = to;
                        sum[x] *= f;
#pragma unroll
                        for (int i = 0; i < DT; ++i) acc[x][i] *= f;
                        part = 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            p[i] = exp2_fast(__builtin_fmaf(s[x][i >> 2][i & 3], c, -to));
                            part += p[i];
                        }
                    }
                    sum[x] += part;
                    pb[x] = __builtin_bit_cast(bf16x8, (u32x4){pack(p[0], p[1]), pack(p[2], p[3]), pack(p[4], p[5]), pack(p[6], p[7])});
                }
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    const bf16x8 f = lds_read16((vp ^ (uint32_t)(64 * hb) ^ (uint32_t)(16 * (i & 1))) + (uint32_t)(2048 * i));
#pragma unroll
                    for (int x = 0; x < CG; ++x) acc[x][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, pb[x], acc[x][i], 0, 0, 0);
                }
            }
        }
        here = more;
        if (more) {
            key0 = next_key0;
            low = min(low, key0);
            write(buf ^ 1, key0, scale);
            more = next(page, next_key0, scale);
            if (more) bring(page);
        }
        __syncthreads();
    }

#pragma unroll
    for (int x = 0; x < CG; ++x) {
        const float total = rows_add(sum[x]);
        const bool seen = used[x] && low <= pos0 + ti[x];
        if (nsplit == 1) {
            if (!used[x]) continue;
            const int64_t row = row0 + first + ti[x];
            const int qh = h * G + m % G;
            const float inv = seen ? 1.f / total : 0.f;
            bf16_t *dst = reinterpret_cast<bf16_t *>(a.out) + (row * a.hq + qh) * D + 4 * g;
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                const float o[4] = {acc[x][i][0] * inv, acc[x][i][1] * inv, acc[x][i][2] * inv, acc[x][i][3] * inv};
                store_row<bf16_t, 4>(dst + 16 * i, o);
            }
            if (g == 0 && a.lse != nullptr) a.lse[row * a.hq + qh] = seen ? ref[x] * kLn2 + logf(total) : -INFINITY;
        } else {
            const int64_t col = slot * (16 * NW * CG) + (w * CG + x) * 16 + m;
            float *dst = a.part + col * D + 4 * g;
#pragma unroll
            for (int i = 0; i < DT; ++i) *reinterpret_cast<f32x4 *>(dst + 16 * i) = acc[x][i];
            if (g == 0) {
                a.ml[col * 2] = seen ? ref[x] : -INFINITY;
                a.ml[col * 2 + 1] = total;
            }
        }
    }
    if (low == INT32_MAX || s_odd == 0) return;
    // Values that are not finite were taken as 0 in pages that some tokens see further than others (0 x infinity): the tokens that do see them get them now.
    __threadfence_block();
    for (int j = max(pos0 / kBlock, split * a.pps); j <= pos_last / kBlock && j < e_end; ++j) {
        const int odd_page = __builtin_amdgcn_readfirstlane(a.c.page(seq, j));
        if (odd_page < 0) continue;
        const char *vb = a.c.v + a.c.at(odd_page, h);
        for (int x = 0; x < CG; ++x) {
            const int t = (w * CG + x) * GT + m / G;
            if (m / G >= GT || t >= ntok) continue;
            const int rows = min(kBlock, pos0 + t + 1 - j * kBlock);
            for (int i = 0; i < DT; ++i) {
                float add[4] = {0.f, 0.f, 0.f, 0.f};
                bool any = false;
                for (int u = 0; u < rows; ++u) {
                    const char *at = vb + (int64_t)u * tok + (16 * i + 4 * g) * KB;
                    for (int r = 0; r < 4; ++r) {
                        float y;
                        if constexpr (CODES) y = ((uint8_t)at[r] & 0x7f) == 0x7f ? __uint_as_float(0x7fc00000u) : 0.f;
                        else y = bf16_to_float(reinterpret_cast<const uint16_t *>(at)[r]);
                        if (finite(y)) continue;
                        add[r] += y;
                        any = true;
                    }
                }
                if (!any) continue;
                if (nsplit == 1) {
                    bf16_t *dst = reinterpret_cast<bf16_t *>(a.out) + ((int64_t)(row0 + first + t) * a.hq + h * G + m % G) * D + 16 * i + 4 * g;
                    for (int r = 0; r < 4; ++r) Elem<bf16_t>::store(dst + r, Elem<bf16_t>::load(dst + r) + add[r]);
                } else {
                    float *dst = a.part + (slot * (16 * NW * CG) + (w * CG + x) * 16 + m) * D + 16 * i + 4 * g;
                    for (int r = 0; r < 4; ++r) dst[r] += add[r];
                }
            }
        }
    }
}

template <int D, bool CODES>
int launch_d(const AttnArgs &a, int64_t items, hipStream_t stream) {
    constexpr int CG = groups_of(D), LDS = 2 * Page<D>::kBytes;
    const auto kernel = cache_attn_tile_kernel<D, CG, CODES>;
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS) != hipSuccess)
        return INFLLMV2_ERR_HIP;
    hipLaunchKernelGGL(kernel, dim3((unsigned)items), dim3(kThreads), LDS, stream, a);
    return hip_status(hipGetLastError());
}

}  // namespace

namespace cache_attn {

int tile_groups(const infllmv2_params *p) { return NW * groups_of(p->head_dim); }

// From half a tile of column groups on.
int tile_wide_from(const infllmv2_params *p) {
    if (p->dtype != INFLLMV2_BF16) return INT32_MAX;
    return (kCols / (p->num_q_heads / p->num_kv_heads)) * tile_groups(p) / 2;
}

int launch_tile(const AttnArgs &a, const infllmv2_params *p, bool codes, int64_t items, hipStream_t stream) {
    if (p->head_dim == 128) return codes ? launch_d<128, true>(a, items, stream) : launch_d<128, false>(a, items, stream);
    return codes ? launch_d<64, true>(a, items, stream) : launch_d<64, false>(a, items, stream);
}

}  // namespace cache_attn
}  // namespace ifv2
