// Who is whose ancestor in each sequence's tree of drafted tokens, as bits, from the tokens' parents; and the position at which every token stands.
//
// A workgroup has one tree in LDS: a row of bits and a jump for each token.  A round gives every token the bits of the token its jump leads to and doubles the
// jump, so that after round r a row holds the 2^r nearest of {itself, its ancestors}, and log2 of the deepest chain rounds are all.  (Rows are read while others
// add to them: a row may come with more ancestors than its round has, never with others.)  Chains that close into a circle, which is no tree, end after log2(n)
// rounds with the tokens that can be reached.
//
// Bound: launch and the chain parents, rounds, rows (one tree of 26 tokens; 64 trees of 127 to 509).
#include "common.h"

namespace ifv2 {

namespace {

constexpr int kMost = INFLLMV2_TREE_MOST;

struct MaskArgs {
    const int32_t *parents, *cu, *ctx;
    uint32_t *mask;
    int32_t *pos;                          // or nullptr
    int words, words_log2;                 // of a row; threads of one
};

// Threads of a row stand side by side, 2^words_log2 of them (a power of two: a division for every word would be most of the kernel).
__global__ void tree_masks_kernel(MaskArgs a) {
    extern __shared__ int32_t s_tree[];                       // jumps [2][n], rows [n][W]
    const int row0 = a.cu[blockIdx.x], n = a.cu[blockIdx.x + 1] - row0, W = (n + 31) / 32;
    if (n == 0) return;
    int32_t *jump = s_tree, *next = s_tree + n;
    uint32_t *rows = (uint32_t *)(s_tree + 2 * n);
    const int w = threadIdx.x & ((1 << a.words_log2) - 1), r0 = threadIdx.x >> a.words_log2, by = blockDim.x >> a.words_log2;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const int p = a.parents[row0 + i];
        jump[i] = p >= 0 && p < n ? p : -1;
    }
    for (int r = r0; w < W && r < n; r += by) rows[r * W + w] = r / 32 == w ? 1u << (r % 32) : 0u;
    __syncthreads();
    for (int far = 1; far < n; far *= 2) {
        for (int r = r0; w < W && r < n; r += by) {
            const int j = jump[r];
            if (j >= 0) rows[r * W + w] |= rows[j * W + w];
        }
        int more = 0;
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const int j = jump[i], to = j >= 0 ? jump[j] : -1;
            next[i] = to;
            more |= to >= 0;
        }
        if (!__syncthreads_or(more)) break;
        int32_t *was = jump;
        jump = next;
        next = was;
    }
    const int front = a.pos != nullptr ? a.ctx[blockIdx.x] - n : 0;
    for (int r = r0; r < n; r += by) {
        const uint32_t bits = w < W ? rows[r * W + w] : 0u;
        for (int x = w; x < a.words; x += 1 << a.words_log2) a.mask[(int64_t)(row0 + r) * a.words + x] = x < W ? bits : 0u;
        int count = __popc(bits);
        for (int o = 1 << a.words_log2 >> 1; o > 0; o >>= 1) count += __shfl_xor(count, o);
        if (a.pos != nullptr && w == 0) a.pos[row0 + r] = front + count - 1;
    }
}

}  // namespace

}  // namespace ifv2

extern "C" int infllmv2_tree_masks(const int32_t *parents_d, const int32_t *cu_q_h, const int32_t *cu_q_d, const int32_t *ctx_lens_h,
                                   const int32_t *ctx_lens_d, int32_t batch, uint32_t *mask_d, int32_t mask_words, int32_t *pos_d,
                                   void *stream) {
    using namespace ifv2;
    int64_t total;
    int32_t most;
    const int st = check_cu(cu_q_h, cu_q_d, batch, &total, &most);
    if (st) return st;
    if (total == 0) return INFLLMV2_OK;
    if (parents_d == nullptr || mask_d == nullptr || (pos_d != nullptr && (ctx_lens_h == nullptr || ctx_lens_d == nullptr))) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if ((int64_t)mask_words * 32 < most) return INFLLMV2_ERR_INVALID_ARGUMENT;
    for (int b = 0; pos_d != nullptr && b < batch; ++b)
        if (ctx_lens_h[b] < cu_q_h[b + 1] - cu_q_h[b] || ctx_lens_h[b] > INT32_MAX - kBlock) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (most > kMost) return INFLLMV2_ERR_UNSUPPORTED;
    const int words = (most + 31) / 32, words_log2 = words > 16 ? 5 : words > 8 ? 4 : words > 4 ? 3 : words > 2 ? 2 : words - 1;
    const int lds = (2 + words) * most * (int)sizeof(int32_t), items = most << words_log2, threads = items > 1024 ? 1024 : (items + 63) / 64 * 64;
    if (lds > 64 * 1024 &&
        hipFuncSetAttribute(reinterpret_cast<const void *>(tree_masks_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (2 + kMost / 32) * kMost * (int)sizeof(int32_t)) != hipSuccess)
        return INFLLMV2_ERR_HIP;
    const MaskArgs a{parents_d, cu_q_d, ctx_lens_d, mask_d, pos_d, mask_words, words_log2};
    hipLaunchKernelGGL(tree_masks_kernel, dim3(batch), dim3(threads), lds, (hipStream_t)stream, a);
    return hip_status(hipGetLastError());
}
