// The accepted path of each sequence's tree of drafted tokens, brought together: row i of the path, which stands at drafted row j_i >= i, moves to
// drafted row i, keys and values, in every page and head that it touches.
//
// A workgroup owns the K or the V rows of one (sequence, KV head) and goes through the pages that rows move into, first page first: all rows for a page are
// requested, then (a barrier) written.  The order makes it safe in place: a row comes from its own place or from behind it, so what later pages need is in
// pages that are not written yet.  e4m3 pages: the scale grows to hold the rows that come in, as in an append; they are rounded to it, and so are the
// page's other rows if it grew.
//
// Bound: latency: lengths, path, page numbers, rows, one after the other.  16 trees of 26 tokens, up to 6 kept, e4m3: 4.2 us, 7.2 where
// scales grow and the other rows of their pages are rounded again; 5 of 301, up to 99 kept, fp32, d 64: 7.8, rows that another kernel has just written 9.0 (a
// page's rows requested while the page before is written).
#include "cache.h"

namespace ifv2 {

namespace {

typedef uint32_t Piece __attribute__((ext_vector_type(4)));      // 16 bytes of a row

constexpr int kThreads = 256;

struct AcceptArgs {
    cache::Args c;
    const int32_t *cu, *ctx, *path;
    int32_t *lens;                         // or nullptr
    int stride;                            // of path
    int vecs, vecs_log2;                   // 16-byte pieces of a row
};

// sixteen codes, values times `by`, a power of two
__device__ inline Piece rescaled(Piece x, float by) {
    uint32_t w[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
        w[j] = cache::codes4<false>(lo[0] * by, lo[1] * by, hi[0] * by, hi[1] * by);
    }
    return Piece{w[0], w[1], w[2], w[3]};
}
// the largest magnitude among sixteen codes, as a code (NaN, 0x7f, left out)
__device__ inline uint32_t top_code(Piece x) {
    const uint32_t w[4] = {x[0], x[1], x[2], x[3]};
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const uint32_t c = w[j / 4] >> (8 * (j % 4)) & 0x7fu;
        top = c != 0x7fu && c > top ? c : top;
    }
    return top;
}

// PER: pieces of a page for a thread
template <bool CODES, int PER>
__global__ void __launch_bounds__(kThreads) cache_accept_kernel(AcceptArgs a) {
    __shared__ int s_count, s_same;
    __shared__ uint32_t s_top[2][kThreads / 64];
    const int tid = threadIdx.x, b = blockIdx.x, h = blockIdx.y, row0 = a.cu[b], n = a.cu[b + 1] - row0, len = a.ctx[b], front = len - n;
    const bool values = blockIdx.z != 0;
    const int32_t *path = a.path + (int64_t)b * a.stride;
    // the path: as long as its entries rise and are in the tree; its first entries may be where they are already
    const int most = min(n, a.stride);
    if (tid == 0) s_count = most, s_same = most;
    __syncthreads();
    for (int i = tid; i < most; i += kThreads) {
        const int j = path[i];
        if (j >= n || j <= (i > 0 ? path[i - 1] : -1)) atomicMin(&s_count, i);
        if (j != i) atomicMin(&s_same, i);
    }
    __syncthreads();
    const int count = s_count, same = min(s_same, count);
    if (tid == 0 && h == 0 && !values && a.lens != nullptr) a.lens[b] = front + count;
    char *pool = values ? a.c.v : a.c.k;
    float *scales = values ? a.c.vs : a.c.ks;
    // what moves into a page, as requested
    struct Rows {
        Piece x[PER];
        float scale[PER];                  // of the row's page; 0: the row is not there
    };
    const int block1 = (front + count - 1) / kBlock;
    auto request = [&](int block) {
        Rows m;
        const int first = max(front + same, block * kBlock), end = min(front + count, block * kBlock + kBlock), to_page = a.c.page(b, block);
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int v = tid + e * kThreads, row = first + (v >> a.vecs_log2);
            m.x[e] = Piece{0, 0, 0, 0};
            m.scale[e] = 0.f;
            if (row < end && to_page >= 0) {
                const int from = front + path[row - front], page = a.c.page(b, from / kBlock);
                if (page >= 0) {
                    m.x[e] = *reinterpret_cast<const Piece *>(pool + a.c.at(page, h) + (from % kBlock) * a.c.tok_stride + (v & (a.vecs - 1)) * 16);
                    m.scale[e] = CODES ? scales[(int64_t)page * a.c.hkv + h] : 1.f;
                }
            }
        }
        return m;
    };
    if (same >= count) return;
    int block = (front + same) / kBlock, turn = 0;
    Rows m = request(block);
    for (;; ++block, turn ^= 1) {
        const int first = max(front + same, block * kBlock), end = min(front + count, block * kBlock + kBlock);          // rows that are written
        const int to_page = a.c.page(b, block);
        char *to = pool + a.c.at(to_page, h);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");             // (all rows are here before any is written)
        float now = 1.f;
        if constexpr (CODES) {
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < PER; ++e) top = max(top, __float_as_uint(__builtin_amdgcn_cvt_f32_fp8((int)top_code(m.x[e]), 0) * m.scale[e]));
            const float was = to_page >= 0 ? scales[(int64_t)to_page * a.c.hkv + h] : 1.f;
            top = (uint32_t)__builtin_amdgcn_readlane(cache::wave_scan((int)top, [](int p, int q) { return (int)max((uint32_t)p, (uint32_t)q); }), 63);
            if ((tid & 63) == 0) s_top[turn][tid >> 6] = top;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kThreads / 64; ++w) top = max(top, s_top[turn][w]);
            now = fmaxf(was, cache::scale_for(__uint_as_float(top)));
            if (to_page >= 0 && now != was) {                        // the page's other rows
                for (int v = tid; v < kBlock << a.vecs_log2; v += kThreads) {
                    const int row = v >> a.vecs_log2, t = block * kBlock + row;
                    bool stays = t < first || t >= end;
                    if (!stays) stays = a.c.page(b, (front + path[t - front]) / kBlock) < 0;
                    if (!stays) continue;
                    Piece *at = reinterpret_cast<Piece *>(to + row * a.c.tok_stride + (v & (a.vecs - 1)) * 16);
                    *at = rescaled(*at, was * cache::reciprocal_of_power(now));
                }
                if (tid == 0) scales[(int64_t)to_page * a.c.hkv + h] = now;
            }
        } else {
            __syncthreads();
        }
        // (the next page's rows are from pages behind this one, which it does not write)
        Rows next;
        if (block < block1) next = request(block + 1);
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int v = tid + e * kThreads, row = first + (v >> a.vecs_log2);
            if (m.scale[e] == 0.f) continue;
            Piece y = m.x[e];
            // (a code that is not 0 is at least 2^-9, and the largest 448, so the new scale is at least 2^-17 of its own: no such row needs more than 2^17.  A row of
            // zeros may come from any scale to the least one, 2^219 times as small: a factor of infinity would make NaN of it.)
            if (CODES && m.scale[e] != now) y = rescaled(y, fminf(m.scale[e] * cache::reciprocal_of_power(now), 0x1p17f));
            *reinterpret_cast<Piece *>(to + (row - block * kBlock) * a.c.tok_stride + (v & (a.vecs - 1)) * 16) = y;
        }
        if (block == block1) break;
        m = next;
    }
}

}  // namespace

}  // namespace ifv2

extern "C" int infllmv2_cache_accept(const infllmv2_params *p, const infllmv2_cache *c, const int32_t *cu_q_h, const int32_t *cu_q_d,
                                     const int32_t *ctx_lens_h, const int32_t *ctx_lens_d, int32_t batch, const int32_t *path_d,
                                     int32_t path_stride, int32_t *new_lens_d, void *stream) {
    using namespace ifv2;
    int st = check_params(p);
    if (st) return st;
    int64_t total;
    int32_t max_new;
    st = check_cu(cu_q_h, cu_q_d, batch, &total, &max_new);
    if (st) return st;
    if (batch == 0 || (total == 0 && new_lens_d == nullptr)) return INFLLMV2_OK;
    if (ctx_lens_h == nullptr || ctx_lens_d == nullptr || path_d == nullptr || path_stride < 1) return INFLLMV2_ERR_INVALID_ARGUMENT;
    int max_ctx = 0;
    for (int b = 0; b < batch; ++b) {
        if (ctx_lens_h[b] < cu_q_h[b + 1] - cu_q_h[b] || ctx_lens_h[b] > INT32_MAX - kBlock) return INFLLMV2_ERR_INVALID_ARGUMENT;
        if (cu_q_h[b + 1] > cu_q_h[b] && ctx_lens_h[b] > max_ctx) max_ctx = ctx_lens_h[b];
    }
    // (every workgroup of a sequence reads its lengths and path, one writes the new length)
    if (new_lens_d != nullptr && (cache::overlap(new_lens_d, batch, ctx_lens_d, batch) || cache::overlap(new_lens_d, batch, cu_q_d, batch + 1ll) ||
                                  cache::overlap(new_lens_d, batch, path_d, (int64_t)batch * path_stride)))
        return INFLLMV2_ERR_INVALID_ARGUMENT;
    st = cache::check(p, c, max_ctx, true);
    if (st) return st;
    if (p->num_kv_heads > 65535 || !cache::fits_launch((int64_t)batch * p->num_kv_heads * 2, kThreads)) return INFLLMV2_ERR_UNSUPPORTED;
    const bool codes = c->kv_type == INFLLMV2_CACHE_E4M3;
    const int vecs = p->head_dim * (codes ? 1 : p->dtype == INFLLMV2_BF16 ? 2 : 4) / 16;
    const AcceptArgs a{cache::args(p, c), cu_q_d, ctx_lens_d, path_d, new_lens_d, path_stride, vecs, __builtin_ctz(vecs)};
    const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(batch, p->num_kv_heads, 2), dim3(kThreads), 0, (hipStream_t)stream, a); };
    // 64 rows of 4 to 32 pieces
    if (codes) launch(vecs == 8 ? cache_accept_kernel<true, 2> : cache_accept_kernel<true, 1>);
    else launch(vecs == 32 ? cache_accept_kernel<false, 8> : vecs == 16 ? cache_accept_kernel<false, 4> : cache_accept_kernel<false, 2>);
    return hip_status(hipGetLastError());
}
