// Attention of a chunk of a prompt, or of a few tokens over a long context, bf16 data: tiles of 8 x CG groups of 16 columns (a column is a token and a head of
// one KV head); CG = 2 (head dim 64: 4), or 1 where large tiles are too few for the chip (launch_rules.h).
//
// The workgroup's eight wavefronts go through the pages together and each keeps CG column groups with their queries and sums in
// registers, so that an operand read from LDS feeds CG products.  S^T = K Q^T and O^T += V^T P^T on 16x16x32 products; a lane's logits of a
// half page are eight consecutive keys of one column, which is the operand that the second product wants.
// Half a page is a step: its logits, then the sums of the half before it with the weights of this one between the products (they do not depend on
// each other: the vector unit works while the matrix core does).  A page is requested two pages ahead: K rows into registers, V rows (asynchronously) into a
// buffer of the wavefront's own, from where transposing reads give a lane eight keys of a channel.  Beside the products of a first half they are widened
// (codes times the page's scale: exact in bf16) and written as bf16 K and V^T pages, two and three buffers: one barrier per page.
// Rounding: a chunk's weights go into the second product as bf16 (2^-8 of each at most, like the output's own rounding), those of up to eight tokens as two
// bf16 pieces (2^-16); their sum takes them as they are.  Two pieces for chunks: 2048 tokens over 34816 943 -> 1330 us, 512 over 8000 84 -> 106.  References
// move only where eight weights of a lane add up to more than kSlack, so a weight is below it; sums that pass the largest float for that: cache_attn.h.
//
// What bounds it: LDS and the matrix cores together, at the clocks that the products leave.  2048 tokens over 34816, 32 heads on 2, e4m3: 943 to 996 us on
// different cards, 1140 to 1200 TFLOP/s (a large library product reaches 1212 on this card); the matrix cores are busy 49 % of the clocks and LDS 40 %, conflicts 8 %
// (counters).  Parts left out, when the whole took 966: without LDS reads 786, without the rows' way through LDS 822, products and weights alone 656,
// products alone 591.  Steps on the way: rows through registers by role and phases in lockstep 1208; queries waited for in front of the loop (their wait
// stood in it and waited for the pages) 1102; the rows' work between the products 1043; the step of this form 1017; V through LDS with transposing reads
// 985; the second four wavefronts ahead in first halves 966.  Measured and not taken: CG = 3 (two thirds of the LDS reads: 1013; fewer, larger tiles leave
// CUs idle), the wavefronts of a SIMD taking turns behind barriers (1043), operands eight ahead (994).  A page takes a workgroup 1.75 us with CG = 2 and 1.13
// with CG = 1, 1.46 with two pieces (head dim 64: 1.9 with CG = 4, 0.75 with CG = 1): a small tile has half or a quarter of the columns, so it is taken
// where the call is short of workgroups.
#include <type_traits>

#include "attn_unit.h"
#include "cache_attn.h"
#include "launch_rules.h"

namespace ifv2 {

namespace {

using namespace gen;
using attn_unit::lds_read16;
using cache_attn::AttnArgs;
using cache_attn::kLift;
using cache_attn::kLn2;
using cache_attn::kLowest;
using cache_attn::pack;
using cache_attn::rows_add;
using cache_attn::rows_max;
using cache_attn::widen;

constexpr int NW = 8;
constexpr int kThreads = cache_attn::kTileThreads;
static_assert(kThreads == NW * 64, "eight wavefronts");
constexpr float kSlack = 64.f;
constexpr float kTopBf16 = 3.3895314e38f;  // largest bf16 number
constexpr int kAhead = 4;                  // operands requested in front of their product

// all ones in the elements of w that are infinities or NaN
template <bool CODES>
__device__ inline uint32_t not_finite(uint32_t w) {
    if (CODES) return ((((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 0xffu;
    return ((((w & 0x7fff7fffu) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu;
}
__device__ inline void lds_write16(uint32_t at, u32x4 x) {
    typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
    *(lds_u32x4 *)(uintptr_t)at = x;
}

// A page in LDS: K [64 keys][D] and V^T [D][64 keys], bf16, 16-byte chunks of a row swizzled so that the sixteen lanes of an operand read (rows 8 (m / 4) + m % 4
// of K, 16 consecutive rows of V^T, one logical chunk) and the lanes of a write take different positions.
template <int D>
struct Page {
    static constexpr uint32_t kBytes = 64 * D * 2;                // of K or of V
    static __device__ inline uint32_t k_swizzle(int row) {
        return D == 128 ? 4 * ((row >> 3) & 3) + (row & 3) : 2 * ((row >> 3) & 3) + ((row >> 1) & 1);
    }
    static __device__ inline uint32_t v_swizzle(int ch) { return ((ch >> 1) & 7) ^ ((ch >> 4) & 1); }
    static __device__ inline uint32_t k_at(int row, int chunk) { return (uint32_t)row * (2 * D) + ((chunk ^ k_swizzle(row)) << 4); }
    static __device__ inline uint32_t v_at(int ch, int octet) { return (uint32_t)ch * 128 + ((octet ^ v_swizzle(ch)) << 4); }
};

// PIECES: bf16 pieces of a weight in the second product
template <int D, int CG, int W, int PIECES, bool CODES>
__global__ void __launch_bounds__(kThreads, D == 64 && CG == 1 ? 4 : 2) cache_attn_tile_kernel(AttnArgs a) {
    constexpr int KS = D / 32, DT = D / 16;
    constexpr int KB = CODES ? 1 : 2;                               // bytes of an element
    extern __shared__ __attribute__((aligned(1024))) char smem[];   // two K pages, three V pages, rows of V as they come
    __shared__ int s_item[6];
    __shared__ int s_odd;                                           // a value of a page's edge (see write) is not finite
    __shared__ int s_again;                                         // sums are not finite ..
    __shared__ uint32_t s_bad[CG][kThreads];                        // .. a thread's: bit 4 i + r (registers: kept here through the second walk)
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m = lane & 15, g = lane >> 4, hkv = a.c.hkv, G = a.hq / hkv, GT = a.group_tokens;

    int rem;
    int slot0;
    cache::Facts facts;
    const int seq = cache::find_item(a.batch, (int)blockIdx.x, rem, slot0, facts, s_item,
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
    const int row0 = facts.x[0], n = facts.x[1] - row0, len = facts.x[2];
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
    // (the queries have landed here: left to the first product, the wait for them stands in the loop and waits for the pages requested ahead as well)
#pragma unroll
    for (int x = 0; x < CG; ++x)
#pragma unroll
        for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[x][s]));
    const int wave_first = w * CG * GT;                             // first token of this wavefront
    const float c = a.scale * kLog2e;

    f32x4 acc[CG][DT];
    float ref[CG], sum[CG];

    const uint32_t lds = __builtin_amdgcn_readfirstlane(attn_unit::lds_address(smem));
    const uint32_t k_lane = Page<D>::k_at(8 * (m >> 2) + (m & 3), g), v_lane = Page<D>::v_at(m, g);
    const uint32_t tok = (uint32_t)a.c.tok_stride;
    // What a wavefront brings of a page: eight rows of K (a lane an eighth of one, through registers) and of V (copied to an LDS buffer of its own, from where
    // transposing reads give a lane the eight keys of a channel).
    constexpr int CV = D / 64, KP = D / 64;                         // channels of V; 16-byte pieces of K in LDS
    constexpr int KL = D / 8 * KB > 16 ? 2 : 1, KW = D / 8 * KB / KL / 4;            // requests for K, words of one
    constexpr int VL = 8 * D * KB > 1024 ? 2 : 1, VW = 2 * KB;      // copies of V, words of eight keys
    constexpr uint32_t kRawBytes = 8 * D * KB;                      // of V
    const int k_row = tid >> 3, eighth = tid & 7;
    const uint32_t k_from = k_row * tok + eighth * (D / 8 * KB);
    const uint32_t k_to_lane = Page<D>::k_at(k_row, eighth * KP), v_to_lane = Page<D>::v_at(lane, w);
    constexpr int RL = D * KB / 16;                                 // lanes of a V row
    const uint32_t v_from = (8 * w + lane / RL) * tok + lane % RL * 16;
    const uint32_t raw_at = lds + 5 * Page<D>::kBytes + w * kRawBytes;
    // (codes: lane 2 r + c of a group of sixteen points at half c of row r's sixteen bytes; bf16: lane 4 r + c at quarter c of row r's 32 bytes)
    const uint32_t raw_lane = raw_at + (CODES ? (m >> 1) * (D * KB) + g * 16 + (m & 1) * 8 : (m >> 2) * (D * KB) + g * 32 + (m & 3) * 8);
    uint32_t raw_k[KL * KW], raw_v[CV][VW];
    struct Where {                                                  // a page: offset of its rows, first key, scales
        int64_t at;
        int key0;
        float ks, vs;
    };
    auto request = [&](int i, const Where &p) {                     // i < KL + VL
        if (i < KL) {
            typedef uint32_t Words __attribute__((ext_vector_type(KW)));
            const Words x = *reinterpret_cast<const Words *>(a.c.k + p.at + k_from + 16 * i);
#pragma unroll
            for (int e = 0; e < KW; ++e) raw_k[KW * i + e] = x[e];
        } else if (RL * 8 >= 64 || lane < RL * 8) {
            attn_unit::async_copy16(a.c.v + p.at + (int64_t)((i - KL) * (64 / RL)) * tok, v_from, raw_at + (i - KL) * 1024);
        }
    };
    // The rows that were requested are here: V from the wavefront's buffer.
    auto collect = [&]() {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
        for (int q = 0; q < CV; ++q) {
            if constexpr (CODES) {
                typedef int Two __attribute__((ext_vector_type(2)));
                typedef __attribute__((address_space(3))) Two lds_two;
                const Two x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_two *)(uintptr_t)(raw_lane + 64 * q));
                raw_v[q][0] = x[0], raw_v[q][1] = x[1];
            } else {
                typedef short Four __attribute__((ext_vector_type(4)));
                typedef __attribute__((address_space(3))) Four lds_four;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_four *)(uintptr_t)(raw_lane + 128 * q + 4 * k * D * KB)));
                    raw_v[q][2 * k] = x.x, raw_v[q][2 * k + 1] = x.y;
                }
            }
        }
    };
    auto clean = [&](int key0) {                                    // a page of which not all is visible to all tokens of the tile
        uint32_t odd = 0;
#pragma unroll
        for (int q = 0; q < CV; ++q)
#pragma unroll
            for (int k = 0; k < VW; ++k) {
                constexpr int PER = 4 / KB;                         // keys of a word
                const int seen = pos_last + 1 - (key0 + 8 * w + PER * k);            // .. that some token sees
                const uint32_t keep = seen >= PER ? ~0u : seen <= 0 ? 0u : (1u << (8 * KB * seen)) - 1u;
                const uint32_t o = not_finite<CODES>(raw_v[q][k]);
                odd |= o & keep;
                raw_v[q][k] &= ~o & keep;
            }
        if (odd != 0) s_odd = 1;
    };
    auto write = [&](int i, uint32_t k_to, uint32_t v_to, float ks, float vs) {      // i < KP + CV
        u32x4 x;
        if (i < KP) {                                               // 8 channels of a row
            if constexpr (CODES) x = u32x4{widen<false>(raw_k[2 * i], ks), widen<true>(raw_k[2 * i], ks), widen<false>(raw_k[2 * i + 1], ks), widen<true>(raw_k[2 * i + 1], ks)};
            else x = u32x4{raw_k[4 * i], raw_k[4 * i + 1], raw_k[4 * i + 2], raw_k[4 * i + 3]};
            lds_write16((k_to + k_to_lane) ^ (16u * i), x);         // (KP = 2: the lower bit of the piece's number)
        } else {                                                    // 8 keys of channel 64 q + lane
            const int q = i - KP;
            if constexpr (CODES) x = u32x4{widen<false>(raw_v[q][0], vs), widen<true>(raw_v[q][0], vs), widen<false>(raw_v[q][1], vs), widen<true>(raw_v[q][1], vs)};
            else x = u32x4{raw_v[q][0], raw_v[q][1], raw_v[q][2], raw_v[q][3]};
            lds_write16(v_to + v_to_lane + 8192u * q, x);           // (64 rows on: one swizzle)
        }
    };

    // the pages of the split: lane l holds the l-th of the next 64
    const int e_end = min(a.pages(len, pos_last), (split + 1) * a.pps);
    int e0 = 0, list_key0 = 0;
    int64_t list_at = 0;
    float list_ks = 1.f, list_vs = 1.f;
    uint64_t there = 0;
    auto refill = [&]() {
        while (there == 0 && e0 < e_end) {
            const int j = e0 + lane, page = j < e_end ? a.c.page(seq, j) : -1;
            list_at = a.c.at(page, h);
            list_key0 = j * kBlock;
            if (CODES && page >= 0) {
                list_ks = a.c.ks[(int64_t)page * hkv + h];
                list_vs = a.c.vs[(int64_t)page * hkv + h];
            }
            there = __ballot(page >= 0);
            e0 += 64;
        }
    };
    auto next = [&](Where &p) {                                     // the next page of the list, which is not empty
        const int l = __ffsll((long long)there) - 1;
        there &= there - 1;
        p.at = (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(list_at >> 32), l) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)list_at, l));
        p.key0 = __builtin_amdgcn_readlane(list_key0, l);
        p.ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(list_ks), l));
        p.vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(list_vs), l));
    };
    if (tid == 0) s_odd = s_again = 0;

    // The walk, in steps of half a page k (32 keys): logits of k; then sums of the weights of k - 1 and, between those products, the weights of k.
    constexpr int LOGITS = 8 * CG, KF = 2 * KS;                     // logits of a lane, K operands of a step
    f32x4 s[CG][2];
    uint32_t pb[2][CG][PIECES][4];                                  // by the parity of k
    bf16x8 f[W];                                                    // operands, requested W ahead: KF of K, then DT of V^T
    static_assert((KF + DT) % W == 0, "an operand's place does not depend on the step");
    const uint32_t k_at = lds + k_lane, v_at = lds + 2 * Page<D>::kBytes + v_lane;
    auto k_half = [&](int p2, int hb) { return k_at + p2 * Page<D>::kBytes + hb * (32 * 2 * D); };
    auto v_half = [&](int p3, int hb) { return (v_at + p3 * Page<D>::kBytes) ^ (uint32_t)(64 * hb); };
    auto fetch_k = [&](int j, uint32_t kb) { f[j % W] = lds_read16((kb ^ (uint32_t)(64 * (j % KS))) + (uint32_t)(4 * (j / KS) * 2 * D)); };
    auto fetch_v = [&](int j, uint32_t vb) { f[(KF + j) % W] = lds_read16((vb ^ (uint32_t)(16 * (j & 1))) + (uint32_t)(2048 * j)); };
    auto sums = [&](int j, const uint32_t (&w)[CG][PIECES][4]) {
#pragma unroll
        for (int x = 0; x < CG; ++x)
#pragma unroll
            for (int i = PIECES - 1; i >= 0; --i) {
                const bf16x8 wt = __builtin_bit_cast(bf16x8, (u32x4){w[x][i][0], w[x][i][1], w[x][i][2], w[x][i][3]});
                acc[x][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[(KF + j) % W], wt, acc[x][j], 0, 0, 0);
            }
    };
    auto set = [&](uint32_t (&w)[PIECES][4], int i, float a, float b) {
        if constexpr (PIECES == 2) {
            const cache_attn::Pieces two = cache_attn::pieces(a, b);
            w[0][i] = two.hi;
            w[1][i] = two.lo;
        } else {
            w[0][i] = pack(a, b);
        }
    };
    // kb: K of k; vb: V of k - 1; kb_on: K of k + 1 where it is there already (ON); beside(j): what else is issued at K operand j
    // slack, lift: see pass
    auto step = [&](auto parity, auto on, float slack, float lift, int first_key, uint32_t kb, uint32_t vb, uint32_t kb_on, auto beside) __attribute__((always_inline)) {
        constexpr int P = decltype(parity)::value;
        constexpr bool ON = decltype(on)::value;
#pragma unroll
        for (int j = 0; j < KF; ++j) {
            const int kt = j / KS, ks = j % KS;
#pragma unroll
            for (int x = 0; x < CG; ++x)
                s[x][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[j % W], qf[x][ks], ks ? s[x][kt] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
            if (j + W < KF) fetch_k(j + W, kb);
            else fetch_v(j + W - KF, vb);
            beside(j);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (first_key + 31 > pos0 + wave_first) {                   // keys behind a token
#pragma unroll
            for (int x = 0; x < CG; ++x) {
                const int lim = used[x] ? pos0 + ti[x] - (first_key + 8 * g) : -1;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[x][kt][r] = 4 * kt + r <= lim ? s[x][kt][r] : -INFINITY;
            }
        }
        float part[CG], last = 0.f;
#pragma unroll
        for (int j = 0; j < DT; ++j) {
            sums(j, pb[1 - P]);
            if (j + W < DT) fetch_v(j + W, vb);
            else if (ON) fetch_k(j + W - DT, kb_on);
#pragma unroll
            for (int n = j * LOGITS / DT; n < (j + 1) * LOGITS / DT; ++n) {
                const int x = n / 8, i = n % 8;
                const float p = exp2_fast(__builtin_fmaf(s[x][i >> 2][i & 3], c, -ref[x]));
                part[x] = i ? part[x] + p : p;
                asm volatile("" : "+v"(part[x]));                   // (added here: left alone, all weights are kept to the end of the step)
                if (i & 1) set(pb[P][x], i >> 1, last, p);
                last = p;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        // references move where weights are large: the sums so far are those of k - 1, the weights are formed again
        float largest = part[0];
#pragma unroll
        for (int x = 1; x < CG; ++x) largest = fmaxf(largest, part[x]);
        if (__any(largest > slack)) {
#pragma unroll
            for (int x = 0; x < CG; ++x) {
                float mx = s[x][0][0];
#pragma unroll
                for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[x][i >> 2][i & 3]);
                const float to = fmaxf(ref[x], __builtin_fmaf(rows_max(mx), c, lift)), down = exp2_fast(ref[x] - to);
                ref[x] = to;
                sum[x] *= down;
#pragma unroll
                for (int i = 0; i < DT; ++i) acc[x][i] *= down;
                part[x] = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float p = exp2_fast(__builtin_fmaf(s[x][i >> 2][i & 3], c, -to));
                    part[x] += p;
                    if (i & 1) set(pb[P][x], i >> 1, last, p);
                    last = p;
                }
            }
        }
#pragma unroll
        for (int x = 0; x < CG; ++x) sum[x] += part[x];
    };
    constexpr int MOVES = KP + CV + KL + VL, PER_STEP = (MOVES + KF - 1) / KF;

    // Between two barriers K and V of page p and V of p - 1 are read, K and V of p + 1 written to the other buffers (two of K, three of V) from the registers
    // that hold them, and p + 2 is requested.
    int low = INT32_MAX;
    // (the pass as a loop's body instead of twice in the code keeps 30 to 50 more registers)
    auto pass = [&](auto second) __attribute__((always_inline)) {
        constexpr float lift = decltype(second)::value ? kLift : 0.f, slack = decltype(second)::value ? kSlack * 0x1p-40f : kSlack;
#pragma unroll
        for (int x = 0; x < CG; ++x) {
            ref[x] = kLowest;                                       // (below every logit)
            sum[x] = 0.f;
#pragma unroll
            for (int i = 0; i < DT; ++i) acc[x][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        Where now{}, then{}, after{};                                   // pages p, p + 1, p + 2 (those that are not there repeat the last)
        e0 = split * a.pps;
        there = 0;
        refill();
        const bool here = there != 0;
        low = INT32_MAX;
        if (here) {
            next(now);
            low = now.key0;
            refill();
            then = now;
            bool more = there != 0;                                     // p + 1 is there
            if (more) next(then);
#pragma unroll
            for (int i = 0; i < KL + VL; ++i) request(i, now);
            // V of "page -1", for the sums of the weights 0 in front of the first: zeros
            for (uint32_t at = 16 * tid; at < Page<D>::kBytes; at += 16 * kThreads) lds_write16(lds + 4 * Page<D>::kBytes + at, u32x4{0, 0, 0, 0});
            __syncthreads();                                            // (s_odd)
            collect();
            if (now.key0 + kBlock - 1 > pos0) clean(now.key0);
#pragma unroll
            for (int i = 0; i < KP + CV; ++i) write(i, lds, lds + 2 * Page<D>::kBytes, now.ks, now.vs);
#pragma unroll
            for (int i = 0; i < KL + VL; ++i) request(i, then);
#pragma unroll
            for (int x = 0; x < CG; ++x)
#pragma unroll
                for (int i = 0; i < 4 * PIECES; ++i) pb[1][x][i / 4][i % 4] = 0u;
            int p2 = 0, p3 = 0, before = 2;                             // buffers of page p (K, V) and of V of p - 1
            for (;;) {
                collect();
                refill();
                after = then;
                const bool most = there != 0;
                if (most) next(after);
                const int ahead3 = p3 == 2 ? 0 : p3 + 1;
                if (then.key0 + kBlock - 1 > pos0) clean(then.key0);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // (what this wavefront wrote)
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
#pragma unroll
                for (int j = 0; j < W; ++j) fetch_k(j, k_half(p2, 0));
                if (w >= 4) __builtin_amdgcn_s_setprio(1);              // (of two wavefronts of a SIMD the older wins otherwise, and waits at the barrier)
                const uint32_t k_to = lds + (p2 ^ 1) * Page<D>::kBytes, v_to = lds + (2 + ahead3) * Page<D>::kBytes;
                step(std::integral_constant<int, 0>(), std::true_type(), slack, lift, now.key0, k_half(p2, 0), v_half(before, 1), k_half(p2, 1), [&](int j) {
#pragma unroll
                    for (int i = j * PER_STEP; i < (j + 1) * PER_STEP && i < MOVES; ++i) {
                        if (i < KP + CV) write(i, k_to, v_to, then.ks, then.vs);
                        else request(i - KP - CV, after);
                    }
                });
                __builtin_amdgcn_s_setprio(0);
                step(std::integral_constant<int, 1>(), std::false_type(), slack, lift, now.key0 + 32, k_half(p2, 1), v_half(p3, 0), 0, [](int) {});
                before = p3;
                p3 = ahead3;
                p2 ^= 1;
                if (!more) break;
                now = then;
                then = after;
                more = most;
            }
            // sums of the last half
#pragma unroll
            for (int j = 0; j < DT; ++j) {
                fetch_v(j, v_half(before, 1));
                sums(j, pb[1]);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");            // (no copy is under way into LDS that this workgroup gives back)
            if (lift == 0.f) {
#pragma unroll
                for (int x = 0; x < CG; ++x) {
                    uint32_t bad = 0u;
#pragma unroll
                    for (int i = 0; i < DT; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) bad |= finite(acc[x][i][r]) ? 0u : 1u << (4 * i + r);
                    bad = used[x] ? bad : 0u;
                    s_bad[x][tid] = bad;
                    if (bad != 0u) s_again = 1;
                }
            }
            __syncthreads();                                            // (s_odd, s_again)
        }

#pragma unroll
        for (int x = 0; x < CG; ++x) {
            int t = ti[x];
            asm volatile("" : "+v"(t));                             // (addresses are formed here: kept through the second walk they take registers)
            const float total = rows_add(sum[x]);
            const bool seen = used[x] && low <= pos0 + t;
            // (a split without weight is 0 with no weight: others of the column may have some)
            const float inv = seen && (nsplit == 1 || total != 0.f) ? 1.f / total : 0.f;
            // (weights rounded up may bring a mean of the largest numbers past them)
            auto mean = [&](float s) { return total > 0.f && finite(s) ? __builtin_amdgcn_fmed3f(s * inv, -kTopBf16, kTopBf16) : s * inv; };
            const uint32_t kept = lift != 0.f ? ~s_bad[x][tid] : 0u;                     // elements that are the first walk's
            if (nsplit == 1) {
                if (!used[x]) continue;
                const int64_t row = row0 + first + t;
                const int qh = h * G + m % G;
                bf16_t *dst = reinterpret_cast<bf16_t *>(a.out) + (row * a.hq + qh) * D + 4 * g;
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    float o[4] = {mean(acc[x][i][0]), mean(acc[x][i][1]), mean(acc[x][i][2]), mean(acc[x][i][3])};
                    if (lift != 0.f) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[r] = (kept >> (4 * i + r)) & 1u ? Elem<bf16_t>::load(dst + 16 * i + r) : o[r];
                    }
                    store_row<bf16_t, 4>(dst + 16 * i, o);
                }
                if (lift == 0.f && g == 0 && a.lse != nullptr) a.lse[row * a.hq + qh] = seen ? ref[x] * kLn2 + logf(total) : -INFINITY;
            } else {
                const int64_t col = slot * (16 * NW * CG) + (w * CG + x) * 16 + m + (t - ti[x]);
                float *dst = a.part + col * D + 4 * g;
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    f32x4 o = {mean(acc[x][i][0]), mean(acc[x][i][1]), mean(acc[x][i][2]), mean(acc[x][i][3])};
                    if (lift != 0.f) {
                        const f32x4 was = *reinterpret_cast<const f32x4 *>(dst + 16 * i);
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[r] = (kept >> (4 * i + r)) & 1u ? was[r] : o[r];
                    }
                    *reinterpret_cast<f32x4 *>(dst + 16 * i) = o;
                }
                if (lift == 0.f && g == 0) {
                    a.ml[col * 2] = seen ? ref[x] : -INFINITY;
                    a.ml[col * 2 + 1] = total;
                }
            }
        }
        return here;
    };
    if (pass(std::false_type()) && s_again != 0) pass(std::true_type());
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

template <int D, int CG, int PIECES, bool CODES>
int launch_d(const AttnArgs &a, int64_t items, hipStream_t stream) {
    constexpr int LDS = 5 * Page<D>::kBytes + 64 * D * (CODES ? 1 : 2);
    const auto kernel = cache_attn_tile_kernel<D, CG, kAhead, PIECES, CODES>;
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, LDS) != hipSuccess)
        return INFLLMV2_ERR_HIP;
    hipLaunchKernelGGL(kernel, dim3((unsigned)items), dim3(kThreads), LDS, stream, a);
    return hip_status(hipGetLastError());
}

}  // namespace

namespace cache_attn {

int launch_tile(const AttnArgs &a, const infllmv2_params *p, bool codes, int64_t items, hipStream_t stream) {
    static_assert(rules::tile_size(128, false).groups == 2 * NW && rules::tile_size(64, false).groups == 4 * NW, "the tiles that the rules count with");
    static_assert(rules::tile_size(128, true).groups == NW && rules::tile_size(64, true).groups == NW, "the tiles that the rules count with");
    const auto launch = [&](auto d, auto groups, auto pieces) {
        constexpr int D = decltype(d)::value, CG = decltype(groups)::value, PIECES = decltype(pieces)::value;
        return codes ? launch_d<D, CG, PIECES, true>(a, items, stream) : launch_d<D, CG, PIECES, false>(a, items, stream);
    };
    const std::integral_constant<int, 1> one;
    const std::integral_constant<int, 2> two;
    const std::integral_constant<int, 4> four;
    const std::integral_constant<int, 64> d64;
    const std::integral_constant<int, 128> d128;
    const bool small = a.tile_groups == NW;
    if (p->head_dim == 128) return !small ? launch(d128, two, one) : a.fine ? launch(d128, one, two) : launch(d128, one, one);
    return !small ? launch(d64, four, one) : a.fine ? launch(d64, one, two) : launch(d64, one, one);
}

}  // namespace cache_attn
}  // namespace ifv2
