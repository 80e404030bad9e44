// Attention of the newest tokens of each sequence over its paged cache (infllmv2_cache_attn): a decode step, a few proposed tokens, or a chunk of a prompt;
// over all keys or over the listed blocks; the pages in the data's type or as e4m3 codes.
//
// Columns and products as in gen_unit.h: a wavefront works on 16 columns (16 / G consecutive tokens of a KV head with their G heads; with block lists
// one token) and goes through pages of 64 keys, STEP keys at a time, with a running reference and sum of the softmax.  K rows are operands as
// they are.  V rows are wanted with the keys along the registers: a lane loads D / 16 neighbouring channels of 8 keys of 32 and byte permutes pair
// the keys.  Codes are widened on the way: K codes to bf16 with their page's scale (exact, a 3-bit mantissa times a power of two), V codes
// after the permute, two keys of a channel per instruction.
// A step's K is requested when the previous step's logits are done and its V when the previous step's sums are, so that one step is always
// in flight.  The work of a (tile, KV head) is split along the keys over workgroups (launch_rules.h: unit_pps), and over the four wavefronts of each; partial
// results are joined in LDS, then by cache_merge_kernel.
//
// Bound: HBM where the pages are many (64 sequences of 16384 to 65536 keys, 16 heads on 1, e4m3: 258 + 8 us for 1.37 GB, 5.2 TB/s, the matrix cores busy for 10 % of
// it; one of 500000: 54 us for 256 MB), else a chain of trips to memory: length, page number, rows, partial results, joined results (16 sequences, 64 listed
// blocks each: 11.0 + 4.0 us traced, of which some 0.5 to the length, 1.4 to the page, 1.7 to its first logits, 2.8 for the rest of two pages, 0.5 in LDS; 5
// sequences of 300 to 2011 keys with 4 tokens each, fp32: 10.6 + 3.9).  fp32 data: the products, 2.6 us for a page of 64 channels and wavefront.  Measured and
// not taken: a word of each line of the page after the next requested ahead, for the L2 (16 sequences of 33000 keys: 56 -> 64 us).
#include <type_traits>

#include "cache_attn.h"
#include "launch_rules.h"

namespace ifv2 {

namespace {

using namespace gen;
using cache_attn::AttnArgs;
using cache_attn::formed;
using cache_attn::kLift;
using cache_attn::kLn2;
using cache_attn::kLowest;
using cache_attn::rows_add;
using cache_attn::rows_max;
using cache_attn::widen;

constexpr int NW = 4;                  // wavefronts of a workgroup

// ------------------------------------------------------------------------------------------ rows of a page, by element type and store
// Keys: sixteen rows of a product, as loaded; the channels that a lane group takes are those of the query operand (load_query).
template <typename T, int D, bool CODES> struct KeyTile;
template <typename T, int D> struct KeyTile<T, D, false> {
    RowFrag<T, D> f;
    static __device__ inline uint32_t lane_offset(int g) { return 16 * g; }
    __device__ inline void load(const char *base, uint32_t off) { f.load_at(base, off); }
    __device__ inline RowFrag<T, D> operand(float) const { return f; }
    static __device__ inline void load_query(RowFrag<T, D> &q, const T *row, int g) { q.load(row, g); }
};
template <int D> struct KeyTile<bf16_t, D, true> {
    u32x4 raw[D / 64];                 // channels 64 s + 16 g .. + 15
    static __device__ inline uint32_t lane_offset(int g) { return 16 * g; }
    __device__ inline void load(const char *base, uint32_t off) {
#pragma unroll
        for (int s = 0; s < D / 64; ++s) raw[s] = *reinterpret_cast<const u32x4 *>(base + off + 64 * s);
    }
    __device__ inline RowFrag<bf16_t, D> operand(float scale) const {
        RowFrag<bf16_t, D> f;
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
            const uint32_t a = raw[s / 2][2 * (s & 1)], b = raw[s / 2][2 * (s & 1) + 1];
            f.x[s] = __builtin_bit_cast(bf16x8, (u32x4){widen<false>(a, scale), widen<true>(a, scale), widen<false>(b, scale), widen<true>(b, scale)});
        }
        return f;
    }
    static __device__ inline void load_query(RowFrag<bf16_t, D> &q, const bf16_t *row, int g) {
#pragma unroll
        for (int s = 0; s < D / 32; ++s)
            q.x[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u16x8_u *>(row + 64 * (s / 2) + 16 * g + 8 * (s & 1)));
    }
};
template <int D> struct KeyTile<float, D, true> {
    u32x4 raw[D / 64];
    static __device__ inline uint32_t lane_offset(int g) { return 16 * g; }
    __device__ inline void load(const char *base, uint32_t off) {
#pragma unroll
        for (int s = 0; s < D / 64; ++s) raw[s] = *reinterpret_cast<const u32x4 *>(base + off + 64 * s);
    }
    __device__ inline RowFrag<float, D> operand(float scale) const {
        RowFrag<float, D> f;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            const int w = (int)raw[s / 4][s & 3];
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
            f.x[s] = f32x4{lo[0] * scale, lo[1] * scale, hi[0] * scale, hi[1] * scale};
        }
        return f;
    }
    static __device__ inline void load_query(RowFrag<float, D> &q, const float *row, int g) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) q.x[s] = __builtin_bit_cast(f32x4, *reinterpret_cast<const f32x4_u *>(row + 64 * (s / 4) + 16 * g + 4 * (s & 3)));
    }
};

// Values: D / 16 channels of one row per lane, in 32-bit words as stored
template <typename T, int D, bool CODES>
struct ValueRow {
    static constexpr int BYTES = D / 16 * (CODES ? 1 : (int)sizeof(T));
    static constexpr int W = BYTES / 4;
    typedef uint32_t Words __attribute__((ext_vector_type(W)));
    Words raw;
    __device__ inline void load(const char *base, uint32_t off) { raw = *reinterpret_cast<const Words *>(base + off); }
    __device__ inline uint32_t word(int i) const {
        if constexpr (W == 1) return raw[0];
        else return raw[i];
    }
    __device__ inline void clear_unless(bool keep) {
#pragma unroll
        for (int i = 0; i < W; ++i) raw[i] = keep ? raw[i] : 0u;
    }
    __device__ inline bool odd() const {                     // holds an infinity or a NaN
        bool any = false;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const uint32_t w = raw[i];
            if constexpr (CODES) any |= (((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) != 0;
            else if constexpr (sizeof(T) == 2) any |= (((w & 0x7fff7fffu) + 0x00800080u) & 0x80008000u) != 0;
            else any |= (w & 0x7fffffffu) >= 0x7f800000u;
        }
        return any;
    }
};

// Weights of a step as operands: bf16 data as two bf16 pieces, so that an output is off by little more than its own rounding; fp32 data as they are.
template <typename T, int TILES> struct Weights;
template <int TILES> struct Weights<bf16_t, TILES> {
    bf16x8 hi[TILES / 2], lo[TILES / 2];
    __device__ inline void set(const f32x4 (&p)[TILES], float) {
#pragma unroll
        for (int t = 0; t < TILES / 2; ++t) {
            u32x4 h, l;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 x = p[2 * t + i / 2];
                const cache_attn::Pieces w = cache_attn::pieces(x[2 * (i & 1)], x[2 * (i & 1) + 1]);
                h[i] = w.hi;
                l[i] = w.lo;
            }
            hi[t] = __builtin_bit_cast(bf16x8, h);
            lo[t] = __builtin_bit_cast(bf16x8, l);
        }
    }
};
template <int TILES> struct Weights<float, TILES> {
    f32x4 w[TILES];
    __device__ inline void set(const f32x4 (&p)[TILES], float scale) {
#pragma unroll
        for (int t = 0; t < TILES; ++t) w[t] = p[t] * scale;
    }
};

// acc[j] += (rows' channel N (4 g + r) + j) x (weights of column m); rows v[4 t + r]: key 16 t + 4 g + r of the step
// SOLO: only into the columns (lanes) that take
template <bool SOLO, int D, int TILES, bool CODES>
__device__ inline void add_values(f32x4 (&acc)[D / 16], const Weights<bf16_t, TILES> &w, const ValueRow<bf16_t, D, CODES> (&v)[4 * TILES], float scale, bool take) {
    auto add = [&](f32x4 &to, bf16x8 row, int t) {
        f32x4 x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(row, w.lo[t], to, 0, 0, 0);
        x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(row, w.hi[t], x, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) to[r] = !SOLO || take ? x[r] : to[r];
    };
#pragma unroll
    for (int t = 0; t < TILES / 2; ++t) {
        const ValueRow<bf16_t, D, CODES> *a = &v[8 * t];
        if constexpr (CODES) {
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                uint32_t lo[4], hi[4];                       // channels 4 i, 4 i + 1 and 4 i + 2, 4 i + 3 of two keys each
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    lo[k] = __builtin_amdgcn_perm(a[2 * k + 1].word(i), a[2 * k].word(i), 0x05010400u);
                    hi[k] = __builtin_amdgcn_perm(a[2 * k + 1].word(i), a[2 * k].word(i), 0x07030602u);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t *s = j < 2 ? lo : hi;
                    u32x4 x;
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[k] = j & 1 ? widen<true>(s[k], scale) : widen<false>(s[k], scale);
                    add(acc[4 * i + j], __builtin_bit_cast(bf16x8, x), t);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                const int i = j / 2;
                u32x4 x;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    x[k] = j & 1 ? upper_halves(a[2 * k].word(i), a[2 * k + 1].word(i)) : lower_halves(a[2 * k].word(i), a[2 * k + 1].word(i));
                add(acc[j], __builtin_bit_cast(bf16x8, x), t);
            }
        }
    }
}
template <bool SOLO, int D, int TILES, bool CODES>
__device__ inline void add_values(f32x4 (&acc)[D / 16], const Weights<float, TILES> &w, const ValueRow<float, D, CODES> (&v)[4 * TILES], float, bool take) {
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
        f32x4 sum = acc[j];
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float x;
                if constexpr (CODES) {
                    const auto two = (j & 2) ? __builtin_amdgcn_cvt_pk_f32_fp8((int)v[4 * t + r].word(j / 4), true)
                                             : __builtin_amdgcn_cvt_pk_f32_fp8((int)v[4 * t + r].word(j / 4), false);
                    x = two[j & 1];
                } else {
                    x = __uint_as_float(v[4 * t + r].word(j));
                }
                sum = __builtin_amdgcn_mfma_f32_16x16x4f32(x, w.w[t][r], sum, 0, 0, 0);
            }
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[j][r] = !SOLO || take ? sum[r] : acc[j][r];
    }
}

// ------------------------------------------------------------------------------------------ a split of a tile
// MULTI: tiles may have several tokens
template <typename T, int D, bool CODES, int TILES, bool MULTI>
__global__ void __launch_bounds__(NW * 64, 2) cache_attn_kernel(AttnArgs a) {
    constexpr int STEP = 16 * TILES, STEPS = kBlock / STEP, N = D / 16;
    __shared__ int s_item[6];
    __shared__ float s_m[NW][16], s_l[NW][16];
    __shared__ __attribute__((aligned(16))) float s_o[NW][16][D + 4];          // (rows four banks apart)
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m = lane & 15, g = lane >> 4, hkv = a.c.hkv, G = a.hq / hkv;

    // the item: sequence, tile, KV head, split; slot: where a partial result goes
    int seq, rem, row0, n, len, early = -1;
    int64_t slot = blockIdx.x;
    if (a.even) {
        seq = (int)(blockIdx.x / (unsigned)(hkv * a.even));
        rem = (int)(blockIdx.x - (unsigned)seq * (unsigned)(hkv * a.even));
        row0 = seq;
        n = 1;
        len = a.ctx[seq];
        // (the first list entries are requested beside the length that says whether there is a list)
        if (a.idx != nullptr)
            early = a.idx[((int64_t)seq * hkv + rem / a.even) * a.topk + min(rem % a.even * NW + w + lane * NW * a.even, a.topk - 1)];
    } else {
        int slot0;
        cache::Facts f;
        seq = cache::find_item(a.batch, (int)blockIdx.x, rem, slot0, f, s_item,
            [&](int s) {
                const int n = a.cu[s + 1] - a.cu[s], len = a.ctx[s];
                return a.tiles(n, len) * hkv * a.most_splits(n, len);
            },
            [&](int s) {
                const int n = a.cu[s + 1] - a.cu[s], len = a.ctx[s], sp = a.most_splits(n, len);
                return sp > 1 ? a.tiles(n, len) * hkv * sp : 0;
            },
            [&](int s, int i) { return i < 2 ? a.cu[s + i] : a.ctx[s]; });
        if (seq >= a.batch) return;
        slot = (int64_t)slot0 + rem;
        row0 = f.x[0];
        n = f.x[1] - row0;
        len = f.x[2];
    }
    const int per = a.even ? a.even : a.most_splits(n, len);
    const bool listed = a.listed(len);
    const int split = rem % per, th = rem / per, h = th % hkv, tile = th / hkv;
    const int T0 = a.tile_tokens(len), first = tile * T0, ntok = min(T0, n - first);       // tokens of this tile
    const int pos0 = len - n + first, pos_last = pos0 + ntok - 1;
    const int nsplit = a.splits(len, pos_last);
    if (split >= nsplit) return;
    // the entries of this wavefront: of all pages a run for each split; of a list (which may be longer than the pages there can be, and hold them
    // anywhere) every (NW x nsplit)-th
    const int e_first = listed ? split * NW + w : split * a.pps + w, e_step = listed ? NW * nsplit : NW;
    const int e_end = listed ? a.topk : min(a.pages(len, pos_last), (split + 1) * a.pps);
    const int ti = m / G;                                                                // this lane's column
    const bool used = ti < ntok;
    const int pos = used ? pos0 + ti : -1;
    const int64_t row = row0 + first + (used ? ti : 0);
    const int qh = h * G + (used ? m - ti * G : 0);

    RowFrag<T, D> qf;
    KeyTile<T, D, CODES>::load_query(qf, reinterpret_cast<const T *>(a.q) + (row * a.hq + qh) * D, g);
    const float c = a.scale * kLog2e;

    f32x4 acc[N];
    float ref, sum;                              // reference in units of log2; this lane's share of the sum, then the column's
    int low = INT32_MAX;                         // first key of any page that this wavefront went through

    const int32_t *list = a.idx + ((int64_t)(row0 + first) * hkv + h) * a.topk;
    const uint32_t tok = (uint32_t)a.c.tok_stride;
    const uint32_t k_off = m * tok + KeyTile<T, D, CODES>::lane_offset(g), v_off = 4 * g * tok + m * ValueRow<T, D, CODES>::BYTES;
    // (a walk as a loop's body instead of twice in the code keeps some 24 more registers)
    auto walk = [&](auto second) {
        constexpr float lift = decltype(second)::value ? kLift : 0.f;
        ref = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        // lane l holds the l-th of the next 64 pages: where it is, its first key, its scales
        for (int e0 = e_first; e0 < e_end; e0 += 64 * e_step) {
            const int e = e0 + lane * e_step;
            int my_page = -1, my_key0 = 0;
            float my_ks = 1.f, my_vs = 1.f;
            if (e < e_end) {
                const int j = !listed ? e : nsplit == a.even && e0 == e_first ? early : list[e];
                if (j >= 0 && j <= pos_last / kBlock) {
                    my_page = a.c.page(seq, j);
                    my_key0 = j * kBlock;
                }
            }
            uint64_t there = __ballot(my_page >= 0);
            if (there == 0) continue;
            if (CODES && my_page >= 0) {
                my_ks = a.c.ks[(int64_t)my_page * hkv + h];
                my_vs = a.c.vs[(int64_t)my_page * hkv + h];
            }
            KeyTile<T, D, CODES> k[TILES];
            ValueRow<T, D, CODES> v[4 * TILES];
            auto base_of = [&](const char *p, int l) { return p + a.c.at(__builtin_amdgcn_readlane(my_page, l), h); };
            auto load_k = [&](const char *base) {
#pragma unroll
                for (int t = 0; t < TILES; ++t) k[t].load(base + (int64_t)(16 * t) * tok, k_off);
            };
            auto load_v = [&](const char *base) {
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[4 * t + r].load(base + (int64_t)(16 * t + r) * tok, v_off);
            };
            int l = __ffsll((long long)there) - 1;
            const char *kb = base_of(a.c.k, l), *vb = base_of(a.c.v, l);
            load_k(kb);
            load_v(vb);
            while (there) {
                const int page_key0 = __builtin_amdgcn_readlane(my_key0, l);
                const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_ks), l));
                const float vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(my_vs), l));
                there &= there - 1;
                low = min(low, page_key0);
                if (there) l = __ffsll((long long)there) - 1;
#pragma unroll 1
                for (int part = 0; part < STEPS; ++part) {
                    const int key0 = page_key0 + part * STEP;
                    f32x4 s[TILES];
#pragma unroll
                    for (int t = 0; t < TILES; ++t) {
                        s[t] = row_product<D>(k[t].operand(ks), qf);
                        if (CODES && t % 2 == 1) __builtin_amdgcn_sched_barrier(0);      // (widened rows of two tiles at a time: registers)
                    }
                    const bool last_part = part == STEPS - 1, more = !last_part || there;
                    if (more) {
                        kb = last_part ? base_of(a.c.k, l) : kb + (int64_t)STEP * tok;
                        load_k(kb);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    const bool edge = key0 + STEP - 1 > pos0;                        // keys behind a token
                    if (edge) {
#pragma unroll
                        for (int t = 0; t < TILES; ++t)
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[t][r] = key0 + 16 * t + 4 * g + r <= pos ? s[t][r] : -INFINITY;
                    }
                    float mx = s[0][0];
#pragma unroll
                    for (int t = 0; t < TILES; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[t][r]);
                    mx = __builtin_fmaf(rows_max(mx), c, lift);
                    if (__any(mx > ref)) {
                        const float to = fmaxf(ref, mx), base = to == -INFINITY ? 0.f : to;
                        const float f = exp2_fast(ref - base);
                        ref = to;
                        sum *= f;
#pragma unroll
                        for (int j = 0; j < N; ++j) acc[j] *= f;
                    }
                    const float base = ref == -INFINITY ? 0.f : ref;
                    float part_sum = 0.f;
#pragma unroll
                    for (int t = 0; t < TILES; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            s[t][r] = exp2_fast(__builtin_fmaf(s[t][r], c, -base));
                            part_sum += s[t][r];
                        }
                    sum += part_sum;
                    Weights<T, TILES> wt;
                    wt.set(s, vs);
                    int rounds = 1;
                    if (edge) {                                                      // rows that no token of the tile sees, and those that only some see
                        bool odd = false;
#pragma unroll
                        for (int t = 0; t < TILES; ++t)
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                v[4 * t + r].clear_unless(key0 + 16 * t + 4 * g + r <= pos_last);
                                if (MULTI) odd |= v[4 * t + r].odd();
                            }
                        if (MULTI && __any(odd)) rounds = ntok;
                    }
                    if (!MULTI) {
                        add_values<false, D, TILES, CODES>(acc, wt, v, vs, true);
                    } else {
                        // 0 x infinity: where rows are not finite, the sums of each token from the rows that it sees, latest token first
#pragma unroll 1
                        for (int i = rounds - 1; i >= 0; --i) {
                            if (rounds > 1) {
#pragma unroll
                                for (int t = 0; t < TILES; ++t)
#pragma unroll
                                    for (int r = 0; r < 4; ++r) v[4 * t + r].clear_unless(key0 + 16 * t + 4 * g + r <= pos0 + i);
                            }
                            add_values<true, D, TILES, CODES>(acc, wt, v, vs, rounds == 1 || ti == i);
                        }
                    }
                    if (more) {
                        vb = last_part ? base_of(a.c.v, l) : vb + (int64_t)STEP * tok;
                        load_v(vb);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        sum = rows_add(sum);
    };
    walk(std::false_type());
    // sums that are not finite: a second walk (cache_attn.h)
    uint32_t again = 0;                          // elements 4 j + r that are the second walk's
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) again |= finite(acc[j][r]) ? 0u : 1u << (4 * j + r);
    again = used ? again : 0u;
    const bool twice = __any(again != 0u);
    float more = 1.f;                            // the second walk's share of the first's sums
    if (twice) {
        const float first_ref = ref, first_sum = sum;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < N; ++j) s_o[w][m][N * (4 * g + r) + j] = acc[j][r];
        walk(std::true_type());
        more = first_sum / sum;
        ref = first_ref;
        sum = first_sum;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < N; ++j) acc[j][r] = (again >> (4 * j + r)) & 1u ? acc[j][r] : s_o[w][m][N * (4 * g + r) + j];
    }

    // the four wavefronts' results together
    if (ref == -INFINITY && low <= pos) ref = kLowest;       // only logits of minus infinity (0 / 0 below), not no key at all
    if (lane < 16) s_m[w][m] = ref, s_l[w][m] = sum;
    __syncthreads();
    const bool direct = nsplit == 1;
    float top = s_m[0][m];
#pragma unroll
    for (int x = 1; x < NW; ++x) top = fmaxf(top, s_m[x][m]);
    const float base = top == -INFINITY ? 0.f : top;
    float total = 0.f;
#pragma unroll
    for (int x = 0; x < NW; ++x) total += s_l[x][m] * exp2_fast(s_m[x][m] - base);
    // (a split without weight is 0 with no weight: others of the column may have some)
    const float inv = top == -INFINITY || (!direct && total == 0.f) ? 0.f : 1.f / total;
    const float f = formed(exp2_fast(ref - base) * inv);
    // (element r of acc[j]: channel N (4 g + r) + j of column m)
    if (twice) {
        const float f2 = formed(f * more);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < N; ++j) acc[j][r] *= (again >> (4 * j + r)) & 1u ? f2 : f;
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) acc[j] *= f;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < N; j += 4)
            *reinterpret_cast<f32x4 *>(&s_o[w][m][N * (4 * g + r) + j]) = f32x4{acc[j][r], acc[j + 1][r], acc[j + 2][r], acc[j + 3][r]};
    __syncthreads();
    // a thread: PER channels of a column
    constexpr int PER = 16 * D / (NW * 64);
    const int col = tid / (D / PER), ch = tid % (D / PER) * PER, ci = col / G;
    float o[PER];
#pragma unroll
    for (int i = 0; i < PER; i += 4) {
        f32x4 v = *reinterpret_cast<const f32x4 *>(&s_o[0][col][ch + i]);
#pragma unroll
        for (int x = 1; x < NW; ++x) v += *reinterpret_cast<const f32x4 *>(&s_o[x][col][ch + i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i + e] = v[e];
    }
    if (!direct) {
        store_row<float, PER>(a.part + (slot * 16 + col) * D + ch, o);
    } else if (ci < ntok) {
        store_row<T, PER>(reinterpret_cast<T *>(a.out) + (((int64_t)row0 + first + ci) * a.hq + h * G + col - ci * G) * D + ch, o);
    }
    if (w == 0 && lane < 16) {
        if (direct) {
            if (used && a.lse != nullptr) a.lse[row * a.hq + qh] = top == -INFINITY ? -INFINITY : top * kLn2 + logf(total);
        } else {
            a.ml[(slot * 16 + m) * 2] = top;
            a.ml[(slot * 16 + m) * 2 + 1] = total;
        }
    }
}

// ------------------------------------------------------------------------------------------ joining the splits of a tile
// COLS columns per workgroup, D / 4 threads of four channels each for SG shares of the splits; up to kAhead splits are requested at once by each.
// Four columns and one share where that is all of the splits or there are columns enough for the chip, else one column and 16 shares (one token of one
// sequence, 33000 keys, 65 splits: 20.7 -> 16.0 us; 130 tokens, 4608 columns, 15 splits: 92.8 -> 112.8).
constexpr int kAhead = 8;

template <typename T, int D, int SG, int COLS>
__global__ void __launch_bounds__(D / 4 * COLS * SG) cache_merge_kernel(AttnArgs a) {
    constexpr int kThreads = D / 4 * COLS;               // of a share
    __shared__ int s_item[6];
    __shared__ f32x4 s_o[SG == 1 ? 1 : SG - 1][SG == 1 ? 1 : kThreads];
    __shared__ float2 s_ml[SG == 1 ? 1 : SG - 1][COLS];
    const int tid = threadIdx.x % kThreads, sg = threadIdx.x / kThreads, hkv = a.c.hkv, G = a.hq / hkv;
    int th, seq, row0, n, len;
    int64_t slot;
    if (a.even) {
        seq = (int)(blockIdx.x / (unsigned)hkv);
        th = (int)(blockIdx.x - (unsigned)seq * (unsigned)hkv);
        slot = (int64_t)blockIdx.x * a.even;
        row0 = seq;
        n = 1;
        len = a.ctx[seq];
    } else {
        cache::Facts f;
        int slot0;
        seq = cache::find_item(a.batch, (int)blockIdx.x, th, slot0, f, s_item,
            [&](int s) {
                const int n = a.cu[s + 1] - a.cu[s], len = a.ctx[s];
                return a.most_splits(n, len) > 1 ? a.tiles(n, len) * hkv : 0;
            },
            [&](int s) {
                const int n = a.cu[s + 1] - a.cu[s], len = a.ctx[s], sp = a.most_splits(n, len);
                return sp > 1 ? a.tiles(n, len) * hkv * sp : 0;
            },
            [&](int s, int i) { return i < 2 ? a.cu[s + i] : a.ctx[s]; });
        if (seq >= a.batch) return;
        slot = slot0;
        row0 = f.x[0];
        n = f.x[1] - row0;
        len = f.x[2];
    }
    const int cols = 16 * a.tile_groups;
    if (!a.even) slot += (int64_t)th * a.most_splits(n, len);
    const int h = th % hkv, tile = th / hkv, T0 = a.tile_tokens(len), first = tile * T0, ntok = min(T0, n - first);
    const int nsplit = a.splits(len, len - n + first + ntok - 1);
    if (nsplit == 1) return;                             // (written by the split itself)
    const int col = blockIdx.y * COLS + tid / (D / 4), c0 = (tid % (D / 4)) * 4, m = col & 15;
    const int in_group = m / G, ti = (col >> 4) * a.group_tokens + in_group;
    const bool used = in_group < min(T0, a.group_tokens) && ti < ntok;
    const float *src = a.part + (slot * cols + col) * D + c0;
    const float2 *ml = reinterpret_cast<const float2 *>(a.ml) + slot * cols + col;
    float top = -INFINITY, total = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};                      // the mean so far
    auto part_of = [](float sum) { return sum == 0.f ? 0.f : 1.f / sum; };
    for (int s0 = sg * kAhead; used && s0 < nsplit; s0 += SG * kAhead) {
        float2 x[kAhead];
        f32x4 y[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t s = min(s0 + i, nsplit - 1);
            x[i] = ml[s * cols];
            y[i] = *reinterpret_cast<const f32x4 *>(src + s * cols * D);
        }
        float to = top;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) to = fmaxf(to, x[i].x);
        const float base = to == -INFINITY ? 0.f : to, before = total * exp2_fast(top - base);
        total = before;
        float f[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            f[i] = s0 + i < nsplit ? x[i].y * exp2_fast(x[i].x - base) : 0.f;
            total += f[i];
        }
        const float inv = part_of(total);
        o *= formed(before * inv);
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (s0 + i < nsplit) o += y[i] * formed(f[i] * inv);
        top = to;
    }
    if constexpr (SG > 1) {                              // the shares' results, by the threads of the first
        if (sg > 0) {
            s_o[sg - 1][tid] = o;
            if (c0 == 0) s_ml[sg - 1][tid / (D / 4)] = float2{top, total};
        }
        __syncthreads();
        if (sg > 0) return;
        float to = top;
#pragma unroll
        for (int i = 0; i < SG - 1; ++i) to = fmaxf(to, s_ml[i][tid / (D / 4)].x);
        const float base = to == -INFINITY ? 0.f : to, before = total * exp2_fast(top - base);
        total = before;
        float f[SG - 1];
#pragma unroll
        for (int i = 0; i < SG - 1; ++i) {
            const float2 x = s_ml[i][tid / (D / 4)];
            f[i] = x.y * exp2_fast(x.x - base);
            total += f[i];
        }
        const float inv = part_of(total);
        o *= formed(before * inv);
#pragma unroll
        for (int i = 0; i < SG - 1; ++i) o += s_o[i][tid] * formed(f[i] * inv);
        top = to;
    }
    if (!used) return;
    const int64_t row = row0 + first + ti;
    const int qh = h * G + m - in_group * G;
    // (only logits of minus infinity: 0 / 0, not no key at all)
    const float none = top != -INFINITY && total == 0.f ? NAN : 0.f;
    const float r[4] = {o[0] + none, o[1] + none, o[2] + none, o[3] + none};
    gen::store_row<T, 4>(reinterpret_cast<T *>(a.out) + (row * a.hq + qh) * D + c0, r);
    if (c0 == 0 && a.lse != nullptr) a.lse[row * a.hq + qh] = top == -INFINITY ? -INFINITY : top * kLn2 + logf(total);
}

// what a launch covers: workgroups, tiles with several splits, their partial results
struct Launches {
    int64_t items = 0, merges = 0, slots = 0;
    int most = 0;
    void add(const AttnArgs &a, int n, int len) {
        const int64_t t = (int64_t)a.tiles(n, len) * a.c.hkv;
        if (t == 0) return;
        const int sp = a.most_splits(n, len);
        items += t * sp;
        if (sp > 1) merges += t, slots += t * sp;
        if (sp > most) most = sp;
    }
};

template <typename T, int D>
void merge(const AttnArgs &a, const Launches &l, hipStream_t stream) {
    if (l.merges == 0) return;
    const unsigned cols = 16 * a.tile_groups;
    if (l.most <= kAhead || l.merges * cols > 1024) hipLaunchKernelGGL((cache_merge_kernel<T, D, 1, 4>), dim3((unsigned)l.merges, cols / 4), dim3(D), 0, stream, a);
    else hipLaunchKernelGGL((cache_merge_kernel<T, D, 16, 1>), dim3((unsigned)l.merges, cols), dim3(4 * D), 0, stream, a);
}

template <typename T, int D, bool CODES, int TILES>
int launch_t(const AttnArgs &a, const Launches &l, hipStream_t stream) {
    if (a.multi) hipLaunchKernelGGL((cache_attn_kernel<T, D, CODES, TILES, true>), dim3((unsigned)l.items), dim3(NW * 64), 0, stream, a);
    else hipLaunchKernelGGL((cache_attn_kernel<T, D, CODES, TILES, false>), dim3((unsigned)l.items), dim3(NW * 64), 0, stream, a);
    merge<T, D>(a, l, stream);
    return hip_status(hipGetLastError());
}

constexpr int kMostGroups = 2048;          // a workgroup has at least all pages / kMostGroups (64 sequences of 16384 to 65536 keys: 480 313 us, 2048 272)
constexpr int kLeastPages = NW;            // .. and a page for each wavefront
constexpr int kMostPages = 1 << 25;        // of a context: with so many to a split there is one split
// Bytes of a partial result.  A sequence with more than one split has at most twice pages / pps of them; cache_attn.hip has pps >= all pages /
// kMostGroups, so at most 2 kMostGroups partial results.
size_t slot_bytes(int d, int groups) { return (size_t)16 * groups * (d + 2) * sizeof(float); }
// Least queries of a sequence for which the tile kernel is thought of (bf16 data)
int tile_from(const infllmv2_params *p) {
    return p->dtype == INFLLMV2_BF16 ? (rules::kTileFrom - 1) * (kCols / (p->num_q_heads / p->num_kv_heads)) + 1 : INT32_MAX;
}
size_t unit_bytes(const infllmv2_params *p, int64_t slots) { return align256((size_t)slots * slot_bytes(p->head_dim, 1)); }
size_t tile_bytes(const infllmv2_params *p, int64_t slots, int groups) { return align256((size_t)slots * slot_bytes(p->head_dim, groups)); }

}  // namespace

size_t cache_attn_ws_bound(const infllmv2_params *p, int32_t batch, int64_t tokens, int32_t max_ctx) {
    const int64_t most = (max_ctx + (int64_t)kBlock - 1) / kBlock, per = (most + kLeastPages - 1) / kLeastPages;
    const int64_t units = tokens * p->num_kv_heads;
    const int64_t slots = per <= 1 ? 0 : units < 2 * kMostGroups && units * per < 2 * kMostGroups ? units * per : 2 * kMostGroups;
    // the tile kernel: at most tokens / (tokens of a tile) tiles and one more for each sequence
    const int64_t from = tile_from(p);
    int64_t groups = 0;
    for (bool small : {false, true}) {
        if (tokens < from || most <= 1) break;
        const int64_t tile = rules::tile_size(p->head_dim, small).groups, per_tile = kCols / (p->num_q_heads / p->num_kv_heads) * tile;
        const int64_t seqs = tokens / from < batch ? tokens / from : batch;
        const int64_t n = (tokens / per_tile + seqs) * p->num_kv_heads * (most < rules::kMostTileSplits ? most : rules::kMostTileSplits) * tile;
        if (n > groups) groups = n;
    }
    if (groups > rules::kMostTileGroups) groups = rules::kMostTileGroups;
    return unit_bytes(p, slots) + tile_bytes(p, groups, 1);
}

}  // namespace ifv2

extern "C" int infllmv2_cache_attn(const infllmv2_params *p, const infllmv2_cache *c, const void *q_d, const int32_t *cu_q_h,
                                   const int32_t *cu_q_d, const int32_t *ctx_lens_h, const int32_t *ctx_lens_d, int32_t batch,
                                   const int32_t *block_idx_d, void *out_d, float *lse_d, void *workspace_d, size_t workspace_bytes,
                                   void *stream) {
    using namespace ifv2;
    int st = check_params(p);
    if (st) return st;
    int64_t total;
    int32_t max_new;
    st = check_cu(cu_q_h, cu_q_d, batch, &total, &max_new);
    if (st) return st;
    if (total == 0) return INFLLMV2_OK;
    if (q_d == nullptr || out_d == nullptr || ctx_lens_h == nullptr || ctx_lens_d == nullptr) return INFLLMV2_ERR_INVALID_ARGUMENT;
    const int hkv = p->num_kv_heads;
    AttnArgs a{};
    a.c.hkv = hkv;
    a.idx = block_idx_d;
    a.batch = batch;
    a.topk = p->topk_total;
    a.dense_below = p->dense_threshold;
    a.group_tokens = kCols / (p->num_q_heads / hkv);
    a.wide_from = tile_from(p);
    a.tile_groups = 1;
    AttnArgs wide = a;                         // the tile kernel's launch, with large tiles or small ones
    const rules::TileSize size[2] = {rules::tile_size(p->head_dim, false), rules::tile_size(p->head_dim, true)};
    int max_ctx = 0;
    rules::PageWork work;                      // of the kernel of 16 columns
    // The sequences that could be either kernel's: what they are as its work, in large and in small tiles, their pages in all.  few: those of kFewTokens and
    // fewer, whose weights keep 16 bits in any batch: tiles with weights of two pieces if the batch has no longer ones, else the kernel of 16 columns.
    struct Either {
        rules::PageWork work;
        int most = 0;
        int64_t tiles[2] = {0, 0}, tile_pages[2] = {0, 0}, unit_pages = 0;
    } chunks, few;
    for (int b = 0; b < batch; ++b) {
        const int n = cu_q_h[b + 1] - cu_q_h[b], len = ctx_lens_h[b];
        if (len < n || len > INT32_MAX - kBlock) return INFLLMV2_ERR_INVALID_ARGUMENT;
        if (n == 0) continue;
        if (len > max_ctx) max_ctx = len;
        const int pages = a.pages(len, len - 1);
        const int64_t groups = (int64_t)((n + a.tile_tokens(len) - 1) / a.tile_tokens(len)) * hkv;
        if (a.listed(len) || n < a.wide_from) {
            work.add(groups, pages, a.listed(len) ? groups * pages : (int64_t)hkv * pages);
            continue;
        }
        Either &e = n > rules::kFewTokens ? chunks : few;
        e.work.add(groups, pages, (int64_t)hkv * pages);
        if (pages > e.most) e.most = pages;
        const int first = (len - n) / kBlock + 1;                            // pages that the first token sees
        e.unit_pages += groups * (first + pages) / 2;
        for (int i = 0; i < 2; ++i) {
            const int t0 = a.group_tokens * size[i].groups, t = (n + t0 - 1) / t0, low = t > 1 ? (len - n + t0 - 1) / kBlock + 1 : pages;
            e.tiles[i] += (int64_t)t * hkv;
            e.tile_pages[i] += (int64_t)t * hkv * (low + pages) / 2;
        }
    }
    wide.fine = chunks.tiles[0] == 0;
    const Either &tiled = wide.fine ? few : chunks;
    const rules::TileSplits large = rules::tile_splits(size[0], tiled.tiles[0], tiled.most, tiled.tile_pages[0]);
    const rules::TileSplits small = rules::tile_splits(wide.fine ? rules::fine_tile_size(p->head_dim) : size[1], tiled.tiles[1], tiled.most, tiled.tile_pages[1]);
    const bool use_small = wide.fine || small.us < large.us;
    wide.tile_groups = size[use_small].groups;
    wide.pps = use_small ? small.pps : large.pps;
    const double unit_us = wide.fine ? rules::few_us(p->head_dim * (c != nullptr && c->kv_type == INFLLMV2_CACHE_E4M3 ? 1 : 2), tiled.most, tiled.unit_pages)
                                     : rules::unit_us(p->head_dim, tiled.most, tiled.unit_pages);
    if (tiled.tiles[0] == 0 || unit_us <= (use_small ? small.us : large.us)) {
        a.wide_from = wide.wide_from = INT32_MAX;
        work.add(chunks.work);
        work.add(few.work);
    } else if (!wide.fine) {
        a.wide_from = wide.wide_from = a.wide_from > rules::kFewTokens ? a.wide_from : rules::kFewTokens + 1;
        work.add(few.work);
    }
    for (int b = 0; b < batch && !a.multi; ++b) {
        const int n = cu_q_h[b + 1] - cu_q_h[b], len = ctx_lens_h[b];
        a.multi = n > 1 && a.tiles(n, len) > 0 && a.tile_tokens(len) > 1;
    }
    st = cache::check(p, c, max_ctx, true);
    if (st) return st;
    // (rows of a page are addressed with 32-bit offsets)
    if (c->tok_stride > (1ll << 24)) return INFLLMV2_ERR_UNSUPPORTED;
    const bool codes = c->kv_type == INFLLMV2_CACHE_E4M3, fp32 = p->dtype == INFLLMV2_FP32;
    const int64_t share = (work.sum + kMostGroups - 1) / kMostGroups;
    a.pps = share >= kMostPages ? kMostPages : rules::unit_pps(work, p->head_dim, fp32, codes ? 1 : fp32 ? 4 : 2, share);
    Launches mine, other;
    bool single = true;                        // one query token for each sequence
    for (int b = 0; b < batch; ++b) {
        const int n = cu_q_h[b + 1] - cu_q_h[b], len = ctx_lens_h[b];
        mine.add(a, n, len);
        other.add(wide, n, len);
        single = single && n == 1;
    }
    // as many workgroups for each (sequence, head): nothing has to be looked up.  Where those with nothing to do are few, or a CU each: others are placed
    // beside them, not evenly (16 sequences of 1000 to 33000 keys: 54.5 us, looked up 41.4)
    const int64_t alike = (int64_t)batch * hkv * mine.most;
    if (single && alike <= 2 * kMostGroups && (alike <= 256 || 10 * alike <= 11 * mine.items)) {
        a.even = mine.most;
        mine.items = alike;
        mine.merges = mine.most > 1 ? (int64_t)batch * hkv : 0;
        mine.slots = mine.most > 1 ? mine.items : 0;
    }
    const size_t need = unit_bytes(p, mine.slots), wide_need = tile_bytes(p, other.slots, wide.tile_groups);
    st = check_ws(workspace_d, workspace_bytes, need + wide_need);
    if (st) return st;
    if (!cache::fits_launch(mine.items, NW * 64) || !cache::fits_launch(other.items, cache_attn::kTileThreads)) return INFLLMV2_ERR_UNSUPPORTED;
    for (AttnArgs *x : {&a, &wide}) {
        x->c = cache::args(p, c);
        x->q = (const char *)q_d;
        x->out = (char *)out_d;
        x->lse = lse_d;
        x->cu = cu_q_d;
        x->ctx = ctx_lens_d;
        x->hq = p->num_q_heads;
        x->scale = p->softmax_scale;
    }
    a.part = (float *)workspace_d;
    a.ml = a.part + mine.slots * 16 * p->head_dim;
    wide.part = (float *)((char *)workspace_d + need);
    wide.ml = wide.part + other.slots * 16 * wide.tile_groups * p->head_dim;
    const hipStream_t s = (hipStream_t)stream;
    if (other.items > 0) {
        st = cache_attn::launch_tile(wide, p, codes, other.items, s);
        if (st) return st;
        if (p->head_dim == 128) merge<bf16_t, 128>(wide, other, s);
        else merge<bf16_t, 64>(wide, other, s);
        if (mine.items == 0) return hip_status(hipGetLastError());
    }
    // keys of a step: 64 codes, 32 bf16, 16 fp32 rows take the same registers
    if (p->head_dim == 128) {
        if (p->dtype == INFLLMV2_BF16) return codes ? launch_t<bf16_t, 128, true, 4>(a, mine, s) : launch_t<bf16_t, 128, false, 2>(a, mine, s);
        return codes ? launch_t<float, 128, true, 2>(a, mine, s) : launch_t<float, 128, false, 1>(a, mine, s);
    }
    if (p->dtype == INFLLMV2_BF16) return codes ? launch_t<bf16_t, 64, true, 4>(a, mine, s) : launch_t<bf16_t, 64, false, 4>(a, mine, s);
    return codes ? launch_t<float, 64, true, 2>(a, mine, s) : launch_t<float, 64, false, 2>(a, mine, s);
}
