// Attention of the newest tokens of each sequence over its paged cache (infllmv2_cache_attn): a decode step, a few proposed tokens, or a chunk of a prompt;
// over all keys or over the listed blocks; the pages in the data's type or as e4m3 codes.
//
// Columns and products as in gen_unit.h: a wavefront works on 16 columns (16 / G consecutive tokens of a KV head with their G heads; with block lists
// one token) and goes through pages of 64 keys, STEP keys at a time, with a running reference and sum of the softmax.  K rows are operands as
// they are.  V rows are wanted with the keys along the registers: a lane loads D / 16 neighbouring channels of 8 keys of 32 and byte permutes pair
// the keys.  Codes are widened on the way: K codes to bf16 with their page's scale (exact, a 3-bit mantissa times a power of two), V codes
// after the permute, two keys of a channel per instruction.
// A step's K is requested when the previous step's logits are done and its V when the previous step's sums are, so that one step is always
// in flight.  The work of a (tile, KV head) is split along the keys over workgroups, and over the four wavefronts of each; partial results are joined in
// LDS, then by cache_merge_kernel.
#include "cache.h"
#include "gen_unit.h"

namespace ifv2 {

namespace {

using namespace gen;

constexpr int NW = 4;                  // wavefronts of a workgroup
constexpr int kEntries = 256;          // pages that a workgroup lists at a time
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.4028234e38f;

struct AttnArgs {
    cache::Args c;
    const char *q;
    char *out;
    float *lse;                        // or nullptr
    const int32_t *cu, *ctx, *idx;     // idx: nullptr: all keys
    int batch, hq, topk, dense_below;
    int tokens;                        // of a tile over all keys (16 / G)
    int pps;                           // pages of a split
    int plain;                         // one query token for each sequence, no splits: item = (sequence, head)
    float scale;
    float *part;                       // [slots][16][D] sums, relative to the reference
    float *ml;                         // [slots][16][2] reference, sum of weights
    // how sequence s is cut
    __host__ __device__ bool listed(int len) const { return idx != nullptr && len >= dense_below; }
    __host__ __device__ int tiles(int n, int len) const { return listed(len) ? n : (n + tokens - 1) / tokens; }
    __host__ __device__ int pages(int len) const {
        const int all = (len + kBlock - 1) / kBlock;
        return listed(len) && topk < all ? topk : all;
    }
    __host__ __device__ int splits(int n, int len) const { return n == 0 ? 0 : (pages(len) + pps - 1) / pps; }
};

__device__ inline float rows_max(float x) {          // over lanes with equal lane % 16
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ inline float rows_add(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// two codes (the lower or the upper half of w) as two bf16 values
template <bool UPPER>
__device__ inline uint32_t widen(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, UPPER));
}

// ------------------------------------------------------------------------------------------ rows of a page, by element type and store
// Keys: sixteen rows of a product, as loaded; the channels that a lane group takes are those of the query operand (load_query).
template <typename T, int D, bool CODES> struct KeyTile;
template <typename T, int D> struct KeyTile<T, D, false> {
    RowFrag<T, D> f;
    __device__ inline void load(const char *row, int g) { f.load(reinterpret_cast<const T *>(row), g); }
    __device__ inline RowFrag<T, D> operand(float) const { return f; }
    static __device__ inline void load_query(RowFrag<T, D> &q, const T *row, int g) { q.load(row, g); }
};
template <int D> struct KeyTile<bf16_t, D, true> {
    u32x4 raw[D / 64];                 // channels 64 s + 16 g .. + 15
    __device__ inline void load(const char *row, int g) {
#pragma unroll
        for (int s = 0; s < D / 64; ++s) raw[s] = *reinterpret_cast<const u32x4 *>(row + 64 * s + 16 * g);
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
    __device__ inline void load(const char *row, int g) {
#pragma unroll
        for (int s = 0; s < D / 64; ++s) raw[s] = *reinterpret_cast<const u32x4 *>(row + 64 * s + 16 * g);
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
    __device__ inline void load(const char *row, int m) { raw = *reinterpret_cast<const Words *>(row + m * BYTES); }
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

// Weights of a step as operands: bf16 data as two bf16 pieces (the upper 16 bits and the rest, 2^-16 of the weight left), so that the sums round like
// sums of 32-bit weights and an output is off by its own rounding only; fp32 data as they are.
template <typename T, int TILES> struct Weights;
template <int TILES> struct Weights<bf16_t, TILES> {
    bf16x8 hi[TILES / 2], lo[TILES / 2];
    __device__ inline void set(const f32x4 (&p)[TILES], float) {
#pragma unroll
        for (int t = 0; t < TILES / 2; ++t) {
            f32x4 a = p[2 * t], b = p[2 * t + 1];
            hi[t] = take_piece32<true>(a, b);
            lo[t] = take_piece32<true>(a, b);
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
template <int D, int TILES, bool CODES>
__device__ inline void add_values(f32x4 (&acc)[D / 16], const Weights<bf16_t, TILES> &w, const ValueRow<bf16_t, D, CODES> (&v)[4 * TILES], float scale) {
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
                    const bf16x8 row = __builtin_bit_cast(bf16x8, x);
                    acc[4 * i + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(row, w.lo[t], acc[4 * i + j], 0, 0, 0);
                    acc[4 * i + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(row, w.hi[t], acc[4 * i + j], 0, 0, 0);
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
                const bf16x8 row = __builtin_bit_cast(bf16x8, x);
                acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(row, w.lo[t], acc[j], 0, 0, 0);
                acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(row, w.hi[t], acc[j], 0, 0, 0);
            }
        }
    }
}
template <int D, int TILES, bool CODES>
__device__ inline void add_values(f32x4 (&acc)[D / 16], const Weights<float, TILES> &w, const ValueRow<float, D, CODES> (&v)[4 * TILES], float) {
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                float x;
                if constexpr (CODES) {
                    const auto two = (j & 2) ? __builtin_amdgcn_cvt_pk_f32_fp8((int)v[4 * t + r].word(j / 4), true)
                                             : __builtin_amdgcn_cvt_pk_f32_fp8((int)v[4 * t + r].word(j / 4), false);
                    x = two[j & 1];
                } else {
                    x = __uint_as_float(v[4 * t + r].word(j));
                }
                acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(x, w.w[t][r], acc[j], 0, 0, 0);
            }
}

struct Entry {
    int page, key0;                    // key0: the page's first key
    float ks, vs;
};

// ------------------------------------------------------------------------------------------ a split of a tile
template <typename T, int D, bool CODES, int TILES>
__global__ void __launch_bounds__(NW * 64) cache_attn_kernel(AttnArgs a) {
    constexpr int STEP = 16 * TILES, STEPS = kBlock / STEP, N = D / 16;
    __shared__ int64_t s_item[3];
    __shared__ Entry s_entry[kEntries];
    __shared__ int s_count;
    __shared__ float s_m[NW][16], s_l[NW][16];
    __shared__ f32x4 s_o[NW][N][64];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m = lane & 15, g = lane >> 4, hkv = a.c.hkv, G = a.hq / hkv;

    // the item: sequence, tile, KV head, split; slot: where a partial result goes
    int seq, rem;
    int64_t slot0 = 0;
    if (a.plain) {
        seq = (int)(blockIdx.x / (unsigned)hkv);
        rem = (int)(blockIdx.x - (unsigned)seq * (unsigned)hkv);
    } else {
        seq = cache::find_item(a.batch, blockIdx.x, rem, slot0, s_item,
            [&](int s) {
                const int n = a.cu[s + 1] - a.cu[s], len = a.ctx[s];
                return (int64_t)a.tiles(n, len) * hkv * a.splits(n, len);
            },
            [&](int s) {
                const int n = a.cu[s + 1] - a.cu[s], len = a.ctx[s], sp = a.splits(n, len);
                return sp > 1 ? (int64_t)a.tiles(n, len) * hkv * sp : 0;
            });
        if (seq >= a.batch) return;
    }
    const int row0 = a.cu[seq], n = a.cu[seq + 1] - row0, len = a.ctx[seq], nsplit = a.splits(n, len);
    const bool listed = a.listed(len);
    const int split = rem % nsplit, th = rem / nsplit, h = th % hkv, tile = th / hkv;
    const int T0 = listed ? 1 : a.tokens, first = tile * T0, ntok = min(T0, n - first);    // tokens of this tile
    const int pos0 = len - n + first, pos_last = pos0 + ntok - 1;
    const int ti = m / G;                                                                // this lane's column
    const bool used = ti < ntok;
    const int pos = used ? pos0 + ti : -1;
    const int64_t row = row0 + first + (used ? ti : 0);
    const int qh = h * G + (used ? m - ti * G : 0);

    RowFrag<T, D> qf;
    KeyTile<T, D, CODES>::load_query(qf, reinterpret_cast<const T *>(a.q) + (row * a.hq + qh) * D, g);
    const float c = a.scale * kLog2e;

    f32x4 acc[N];
#pragma unroll
    for (int j = 0; j < N; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float ref = -INFINITY, sum = 0.f;            // reference in units of log2; this lane's share of the sum
    int low = INT32_MAX;                         // first key of any page that this wavefront went through

    const int all = listed ? min(a.topk, (len + kBlock - 1) / kBlock) : pos_last / kBlock + 1;
    const int e_end = min(all, (split + 1) * a.pps);
    const int32_t *list = listed ? a.idx + (row * hkv + h) * a.topk : nullptr;
    for (int e0 = split * a.pps; e0 < e_end; e0 += kEntries) {
        // the pages of this part, those that are there side by side
        __syncthreads();
        if (w == 0) {
            int count = 0;
            for (int x0 = 0; x0 < kEntries && e0 + x0 < e_end; x0 += 64) {
                const int e = e0 + x0 + lane;
                int page = -1, j = -1;
                if (e < e_end) {
                    j = listed ? list[e] : e;
                    if (j >= 0 && j <= pos_last / kBlock) page = a.c.page(seq, j);
                }
                const uint64_t there = __ballot(page >= 0);
                if (page >= 0) {
                    const int64_t at = (int64_t)page * hkv + h;
                    s_entry[count + __popcll(there & ((1ull << lane) - 1ull))] = Entry{page, j * kBlock, CODES ? a.c.ks[at] : 1.f, CODES ? a.c.vs[at] : 1.f};
                }
                count += __popcll(there);
            }
            if (lane == 0) s_count = count;
        }
        __syncthreads();
        const int count = __builtin_amdgcn_readfirstlane(s_count);
        KeyTile<T, D, CODES> k[TILES];
        ValueRow<T, D, CODES> v[4 * TILES];
        auto entry = [&](int e) {
            Entry x = s_entry[e];
            x.page = __builtin_amdgcn_readfirstlane(x.page);
            x.key0 = __builtin_amdgcn_readfirstlane(x.key0);
            x.ks = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x.ks)));
            x.vs = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x.vs)));
            return x;
        };
        auto load_k = [&](const Entry &x, int part) {
            const char *base = a.c.k + a.c.at(x.page, h);
#pragma unroll
            for (int t = 0; t < TILES; ++t) k[t].load(base + (part * STEP + 16 * t + m) * a.c.tok_stride, g);
        };
        auto load_v = [&](const Entry &x, int part) {
            const char *base = a.c.v + a.c.at(x.page, h);
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) v[4 * t + r].load(base + (part * STEP + 16 * t + 4 * g + r) * a.c.tok_stride, m);
        };
        Entry cur{};
        if (w < count) {
            cur = entry(w);
            load_k(cur, 0);
            load_v(cur, 0);
        }
        for (int e = w; e < count; e += NW) {
            Entry next = cur;
            low = min(low, cur.key0);
#pragma unroll 1
            for (int part = 0; part < STEPS; ++part) {
                const int key0 = cur.key0 + part * STEP;
                f32x4 s[TILES];
#pragma unroll
                for (int t = 0; t < TILES; ++t) s[t] = row_product<D>(k[t].operand(cur.ks), qf);
                const bool last_part = part == STEPS - 1, more = !last_part || e + NW < count;
                if (last_part && more) next = entry(e + NW);
                if (more) load_k(last_part ? next : cur, last_part ? 0 : part + 1);
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
                mx = rows_max(mx) * c;
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
                wt.set(s, cur.vs);
                bool solo = false;
                if (edge) {                                                      // rows that no token of the tile sees, and those that only some see
                    bool odd = false;
#pragma unroll
                    for (int t = 0; t < TILES; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            v[4 * t + r].clear_unless(key0 + 16 * t + 4 * g + r <= pos_last);
                            odd |= v[4 * t + r].odd();
                        }
                    solo = ntok > 1 && __any(odd);
                }
                if (!solo) {
                    add_values<D, TILES, CODES>(acc, wt, v, cur.vs);
                } else {
                    // 0 x infinity: the sums of each token from the rows that it sees, latest token first
                    for (int i = ntok - 1; i >= 0; --i) {
#pragma unroll
                        for (int t = 0; t < TILES; ++t)
#pragma unroll
                            for (int r = 0; r < 4; ++r) v[4 * t + r].clear_unless(key0 + 16 * t + 4 * g + r <= pos0 + i);
                        f32x4 own[N];
#pragma unroll
                        for (int j = 0; j < N; ++j) own[j] = acc[j];
                        add_values<D, TILES, CODES>(own, wt, v, cur.vs);
#pragma unroll
                        for (int j = 0; j < N; ++j)
#pragma unroll
                            for (int r = 0; r < 4; ++r) acc[j][r] = ti == i ? own[j][r] : acc[j][r];
                    }
                }
                if (more) load_v(last_part ? next : cur, last_part ? 0 : part + 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            cur = next;
        }
    }

    // the four wavefronts' results together
    sum = rows_add(sum);
    if (ref == -INFINITY && low <= pos) ref = kLowest;       // only logits of minus infinity (0 / 0 below), not no key at all
    if (lane < 16) s_m[w][m] = ref, s_l[w][m] = sum;
    __syncthreads();
    float top = s_m[0][m];
#pragma unroll
    for (int x = 1; x < NW; ++x) top = fmaxf(top, s_m[x][m]);
    const float base = top == -INFINITY ? 0.f : top;
    float total = 0.f;
#pragma unroll
    for (int x = 0; x < NW; ++x) total += s_l[x][m] * exp2_fast(s_m[x][m] - base);
    const float f = exp2_fast(ref - base);
#pragma unroll
    for (int j = 0; j < N; ++j) s_o[w][j][lane] = acc[j] * f;
    __syncthreads();
    // wavefront w: results j = w, w + NW, ..: element r is channel N (4 g + r) + j of column m
    const bool direct = nsplit == 1;
    const int64_t slot = slot0 + rem;
    const float inv = top == -INFINITY ? 0.f : 1.f / total;
#pragma unroll
    for (int jj = 0; jj < N / NW; ++jj) {
        const int j = jj * NW + w;
        f32x4 o = s_o[0][j][lane];
#pragma unroll
        for (int x = 1; x < NW; ++x) o += s_o[x][j][lane];
        if (direct) {
            if (used) {
                T *dst = reinterpret_cast<T *>(a.out) + (row * a.hq + qh) * D;
#pragma unroll
                for (int r = 0; r < 4; ++r) Elem<T>::store(dst + N * (4 * g + r) + j, o[r] * inv);
            }
        } else {
            float *dst = a.part + (slot * 16 + m) * D;
#pragma unroll
            for (int r = 0; r < 4; ++r) dst[N * (4 * g + r) + j] = o[r];
        }
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
template <typename T, int D>
__global__ void __launch_bounds__(256) cache_merge_kernel(AttnArgs a) {
    __shared__ int64_t s_item[3];
    const int tid = threadIdx.x, hkv = a.c.hkv, G = a.hq / hkv;
    int th;
    int64_t slot0;
    const int seq = cache::find_item(a.batch, blockIdx.x, th, slot0, s_item,
        [&](int s) {
            const int n = a.cu[s + 1] - a.cu[s], len = a.ctx[s];
            return a.splits(n, len) > 1 ? (int64_t)a.tiles(n, len) * hkv : 0;
        },
        [&](int s) {
            const int n = a.cu[s + 1] - a.cu[s], len = a.ctx[s], sp = a.splits(n, len);
            return sp > 1 ? (int64_t)a.tiles(n, len) * hkv * sp : 0;
        });
    if (seq >= a.batch) return;
    const int row0 = a.cu[seq], n = a.cu[seq + 1] - row0, len = a.ctx[seq], nsplit = a.splits(n, len);
    const int h = th % hkv, tile = th / hkv, T0 = a.listed(len) ? 1 : a.tokens, first = tile * T0, ntok = min(T0, n - first);
    const int64_t slot = slot0 + (int64_t)th * nsplit;
    constexpr int PER = D / 16;                          // channels per thread: 16 threads a column
    const int m = tid >> 4, c0 = (tid & 15) * PER, ti = m / G;
    if (ti >= ntok) return;
    float top = -INFINITY, total = 0.f, o[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) o[i] = 0.f;
    for (int s = 0; s < nsplit; ++s) {
        const float ref = a.ml[((slot + s) * 16 + m) * 2], l = a.ml[((slot + s) * 16 + m) * 2 + 1];
        const float to = fmaxf(top, ref), base = to == -INFINITY ? 0.f : to;
        const float f0 = exp2_fast(top - base), f1 = exp2_fast(ref - base);
        total = total * f0 + l * f1;
        const float *src = a.part + ((slot + s) * 16 + m) * D + c0;
#pragma unroll
        for (int i = 0; i < PER; ++i) o[i] = o[i] * f0 + src[i] * f1;
        top = to;
    }
    const int64_t row = row0 + first + ti;
    const int qh = h * G + m - ti * G;
    const float inv = top == -INFINITY ? 0.f : 1.f / total;
#pragma unroll
    for (int i = 0; i < PER; ++i) o[i] *= inv;
    gen::store_row<T, PER>(reinterpret_cast<T *>(a.out) + (row * a.hq + qh) * D + c0, o);
    if (c0 == 0 && a.lse != nullptr) a.lse[row * a.hq + qh] = top == -INFINITY ? -INFINITY : top * kLn2 + logf(total);
}

template <typename T, int D, bool CODES, int TILES>
int launch_t(const AttnArgs &a, int64_t items, int64_t merges, hipStream_t stream) {
    hipLaunchKernelGGL((cache_attn_kernel<T, D, CODES, TILES>), dim3((unsigned)items), dim3(NW * 64), 0, stream, a);
    if (merges > 0) hipLaunchKernelGGL((cache_merge_kernel<T, D>), dim3((unsigned)merges), dim3(256), 0, stream, a);
    return hip_status(hipGetLastError());
}

constexpr int kTargetGroups = 1024;        // workgroups that a call is cut into: two rounds of two for each CU
constexpr int kLeastPages = NW;            // a page for each wavefront

// Where splits are more than one, they are at most twice pages / pps, and pps >= all pages / kTargetGroups: at most 2 kTargetGroups partial results.
size_t slot_bytes(int d) { return (size_t)16 * (d + 2) * sizeof(float); }

}  // namespace

size_t cache_attn_ws_bound(const infllmv2_params *p, int64_t tokens, int32_t max_ctx) {
    const int64_t most = (max_ctx + (int64_t)kBlock - 1) / kBlock, per = (most + kLeastPages - 1) / kLeastPages;
    if (per <= 1) return 0;
    const int64_t units = tokens * p->num_kv_heads;
    const int64_t slots = units < 2 * kTargetGroups && units * per < 2 * kTargetGroups ? units * per : 2 * kTargetGroups;
    return align256((size_t)slots * slot_bytes(p->head_dim));
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
    const int hkv = p->num_kv_heads, G = p->num_q_heads / hkv;
    AttnArgs a{};
    a.idx = block_idx_d;
    a.topk = p->topk_total;
    a.dense_below = p->dense_threshold;
    a.tokens = kCols / G;
    int max_ctx = 0;
    int64_t work = 0;                          // pages over all tiles and heads
    for (int b = 0; b < batch; ++b) {
        const int n = cu_q_h[b + 1] - cu_q_h[b], len = ctx_lens_h[b];
        if (len < n || len > INT32_MAX - kBlock) return INFLLMV2_ERR_INVALID_ARGUMENT;
        if (n == 0) continue;
        if (len > max_ctx) max_ctx = len;
        work += (int64_t)a.tiles(n, len) * hkv * a.pages(len);
    }
    st = cache::check(p, c, max_ctx, true);
    if (st) return st;
    const int64_t even = (work + kTargetGroups - 1) / kTargetGroups;
    a.pps = even < kLeastPages ? kLeastPages : even > (1 << 24) ? 1 << 24 : (int)even;
    int64_t items = 0, merges = 0, slots = 0;
    bool plain = true;
    for (int b = 0; b < batch; ++b) {
        const int n = cu_q_h[b + 1] - cu_q_h[b], len = ctx_lens_h[b];
        const int sp = a.splits(n, len);
        const int64_t t = n == 0 ? 0 : (int64_t)a.tiles(n, len) * hkv;
        items += t * sp;
        if (sp > 1) merges += t, slots += t * sp;
        plain = plain && n == 1 && sp == 1;
    }
    const size_t need = slots > 0 ? align256((size_t)slots * slot_bytes(p->head_dim)) : 0;
    st = check_ws(workspace_d, workspace_bytes, need);
    if (st) return st;
    if (items >= (1ll << 31)) return INFLLMV2_ERR_UNSUPPORTED;
    a.c = cache::args(p, c);
    a.q = (const char *)q_d;
    a.out = (char *)out_d;
    a.lse = lse_d;
    a.cu = cu_q_d;
    a.ctx = ctx_lens_d;
    a.batch = batch;
    a.hq = p->num_q_heads;
    a.plain = plain;
    a.scale = p->softmax_scale;
    a.part = (float *)workspace_d;
    a.ml = a.part + slots * 16 * p->head_dim;
    const bool codes = c->kv_type == INFLLMV2_CACHE_E4M3;
    const hipStream_t s = (hipStream_t)stream;
    // keys of a step: 64 codes, 32 bf16, 16 fp32 rows take the same registers
    if (p->head_dim == 128) {
        if (p->dtype == INFLLMV2_BF16) return codes ? launch_t<bf16_t, 128, true, 4>(a, items, merges, s) : launch_t<bf16_t, 128, false, 2>(a, items, merges, s);
        return codes ? launch_t<float, 128, true, 2>(a, items, merges, s) : launch_t<float, 128, false, 1>(a, items, merges, s);
    }
    if (p->dtype == INFLLMV2_BF16) return codes ? launch_t<bf16_t, 64, true, 4>(a, items, merges, s) : launch_t<bf16_t, 64, false, 4>(a, items, merges, s);
    return codes ? launch_t<float, 64, true, 2>(a, items, merges, s) : launch_t<float, 64, false, 2>(a, items, merges, s);
}
