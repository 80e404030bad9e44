// Who is whose ancestor in each sequence's tree of drafted tokens, as bits, from the tokens' parents; and the position at which every token stands.
//
// A workgroup has four words of every row of a tree, a thread one token: its bits and a jump.  A round gives every token the bits of the token its jump leads to and
// doubles the jump, so that after round r a row holds the 2^r nearest of {itself, its ancestors}, and log2 of the deepest chain rounds are all.  (Rows are
// read while others add to them: a row may come with more ancestors than its round has, never with others.)  The ancestors are counted on the way.  Chains that close into a
// circle, which is no tree, end after log2(n) rounds with the tokens that can be reached, which are then counted by going along the chain.
//
// Bound: launch and the chain parents, rounds (a barrier each), rows.  One tree of 26 tokens 2.7 us; 64 trees of 127 to 509 tokens, the deepest chain some 120: 7.0
// (13.4 with all words of a tree in one workgroup, and 18.6 with a division for every word).
#include "cache.h"

namespace ifv2 {

namespace {

constexpr int kMost = INFLLMV2_TREE_MOST;
constexpr int kWords = 4;                  // of a workgroup
typedef uint32_t Words __attribute__((ext_vector_type(kWords)));

struct MaskArgs {
    const int32_t *parents, *cu, *ctx;
    uint32_t *mask;
    int32_t *pos;                          // or nullptr
    int words;                             // of a row
};

// how many tokens a chain that does not end goes through, from token i on: those in front of the circle and the circle's (Brent's way of finding both)
__device__ int tokens_to_circle(const int32_t *parent, int i) {
    int power = 1, circle = 1, slow = i, fast = parent[i];
    while (slow != fast) {
        if (power == circle) {
            slow = fast;
            power *= 2;
            circle = 0;
        }
        fast = parent[fast];
        ++circle;
    }
    int front = 0;
    slow = fast = i;
    for (int k = 0; k < circle; ++k) fast = parent[fast];
    while (slow != fast) {
        slow = parent[slow];
        fast = parent[fast];
        ++front;
    }
    return front + circle;
}

__global__ void __launch_bounds__(kMost) tree_masks_kernel(MaskArgs a) {
    __shared__ Words s_rows[kMost];
    __shared__ int s_parent[kMost], s_jump[2][kMost], s_above[2][kMost];
    const int row0 = a.cu[blockIdx.x], n = a.cu[blockIdx.x + 1] - row0, r = threadIdx.x, w0 = blockIdx.y * kWords;
    if (n == 0) return;
    const bool counts = blockIdx.y == 0 && a.pos != nullptr;
    const int front = counts ? a.ctx[blockIdx.x] - n : 0;
    Words mine = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kWords; ++i) mine[i] = r / 32 == w0 + i ? 1u << (r % 32) : 0u;
    int jump = -1, above = 0;
    if (32 * w0 < n) {                     // (else words behind the tree's)
        if (r < n) {
            const int p = a.parents[row0 + r];
            jump = p >= 0 && p < n ? p : -1;
            above = jump >= 0 ? 1 : 0;
            s_parent[r] = s_jump[0][r] = jump;
            s_above[0][r] = above;
            s_rows[r] = mine;
        }
        int turn = 0, far = 1;
        while (__syncthreads_or(jump >= 0) && far < n) {
            if (jump >= 0) {
                mine |= s_rows[jump];
                above += s_above[turn][jump];
                jump = s_jump[turn][jump];
                s_rows[r] = mine;
            }
            far *= 2;
            turn ^= 1;
            if (r < n) {
                s_jump[turn][r] = jump;
                s_above[turn][r] = above;
            }
        }
    }
    if (r >= n) return;
    uint32_t *to = a.mask + (int64_t)(row0 + r) * a.words + w0;
#pragma unroll
    for (int i = 0; i < kWords; ++i)
        if (w0 + i < a.words) to[i] = mine[i];
    if (counts) a.pos[row0 + r] = front + (jump < 0 ? above : tokens_to_circle(s_parent, r) - 1);
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
    const MaskArgs a{parents_d, cu_q_d, ctx_lens_d, mask_d, pos_d, mask_words};
    // (words behind those of the largest tree are written by workgroups of their own)
    const int64_t chunks = (mask_words + (int64_t)kWords - 1) / kWords;
    if (chunks > 65535 || !cache::fits_launch(batch * chunks, kMost)) return INFLLMV2_ERR_UNSUPPORTED;
    // (every workgroup of a tree reads its parents, one writes the positions)
    if (pos_d != nullptr && (cache::overlap(pos_d, total, parents_d, total) || cache::overlap(pos_d, total, ctx_lens_d, batch) ||
                             cache::overlap(pos_d, total, cu_q_d, batch + 1ll)))
        return INFLLMV2_ERR_INVALID_ARGUMENT;
    hipLaunchKernelGGL(tree_masks_kernel, dim3(batch, (unsigned)chunks), dim3((most + 63) / 64 * 64), 0, (hipStream_t)stream, a);
    return hip_status(hipGetLastError());
}
