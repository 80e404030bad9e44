// Which pages a sequence's blocks are in: pages handed out and taken back (infllmv2_pages_resize), a sequence that continues another
// (infllmv2_pages_fork), the pages in use brought to the front (infllmv2_pages_compact), and the copies that follow from the two
// (infllmv2_cache_copy_pages).
//
// refs[g] counts the table entries that name page g; a page with none is free.  That is all the state there is: pages are taken lowest number first, for
// sequences and blocks in order, so that what a call does depends on table and refs alone, not on the order in which its threads arrive.
//
// Bound: latency.  Entries are given back and shared by as many workgroups as they are worth (counts added with atomics, whose order does not matter);
// handing out needs every free page's rank, which one workgroup works out, 8192 counts at a time, only as far as pages are wanted.  64 rows that give 3000 pages
// back and get 3200 of a pool of 12288: 2.6 and 5.6 us.  32 forks of up to 47 blocks 9.1 (rows that
// held other pages: 11.2).  240 forks of 512 blocks of one row, the kernel that shares: 3.5 where they had its pages before, so that no count and no entry changes (with
// an add and a subtract for each entry: 58); into rows that hold nothing 35 where the pages are anywhere in the pool and 7.5 where they are in order, so that a
// wavefront's adds meet in few lines; in the place of others 39.6.  Their last pages: 3.7 to 5.  8192 pages, 6126 of them in use: 5.4 to find the 1529 that move, 5.4 to renumber 12288 entries.  Copies: HBM, those 1529
// pages of 32 KB 17.5 us, 5.7 TB/s read and written.
#include <algorithm>

#include "cache.h"

namespace ifv2 {

namespace {

typedef uint32_t Piece __attribute__((ext_vector_type(4)));      // 16 bytes of a row

constexpr int kMostRows = INFLLMV2_PAGES_MOST_ROWS;
constexpr int kTakeThreads = 1024, kTakeWaves = kTakeThreads / 64, kDeep = 8;      // counts of a round: kTakeThreads * kDeep

struct Pool {
    int32_t *table, *refs;
    int stride, num_pages;
    __device__ inline int32_t *row(int r) const { return table + (int64_t)r * stride; }
    __device__ inline bool is_page(int g) const { return g >= 0 && g < num_pages; }
};
Pool pool_of(const infllmv2_pages *g) { return Pool{g->page_table_d, g->refs_d, g->table_stride, g->num_pages}; }

__host__ __device__ inline int blocks_of(int tokens) { return (int)(((int64_t)tokens + kBlock - 1) / kBlock); }

// ------------------------------------------------------------------------------------------ the lowest free pages
struct Ranks {
    int cell[kDeep * kTakeWaves];          // flags of (k, wavefront), then how many stand in front
    int total;
};
// a thread's counts of a round: those of pages base + k * kTakeThreads + its number
struct Counts {
    int x[kDeep];
    __device__ inline void load(const int32_t *refs, int64_t base, int num_pages) {
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            const int64_t g = base + k * kTakeThreads + threadIdx.x;
            x[k] = refs[g < num_pages ? g : num_pages - 1];
        }
    }
};

// Workgroup-wide: found(page, rank) for the pages of refs[0 .. num_pages) whose count is wanted, in order of their numbers, until there are `most` or none are
// left; returns how many there were.  c: the first round's counts (each round's are requested a round ahead).
template <class Wanted, class Found>
__device__ inline int ranked_pages(const int32_t *refs, int num_pages, int most, Counts c, Ranks &s, Wanted wanted, Found found) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int before = 0;
    for (int64_t base = 0; base < num_pages && before < most; base += kTakeThreads * kDeep) {
        bool is[kDeep];
        uint64_t hits[kDeep];
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            is[k] = base + k * kTakeThreads + tid < num_pages && wanted(c.x[k]);
            hits[k] = __ballot(is[k]);
            if (lane == 0) s.cell[k * kTakeWaves + w] = __popcll(hits[k]);
        }
        if (base + kTakeThreads * kDeep < num_pages) c.load(refs, base + kTakeThreads * kDeep, num_pages);
        __syncthreads();
        if (w == 0) {                      // two cells a lane
            const int x = s.cell[2 * lane], y = s.cell[2 * lane + 1], incl = cache::wave_sums(x + y);
            s.cell[2 * lane] = incl - x - y;
            s.cell[2 * lane + 1] = incl - y;
            if (lane == 63) s.total = incl;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kDeep; ++k)
            if (is[k]) found((int)(base + k * kTakeThreads + tid), before + s.cell[k * kTakeWaves + w] + __popcll(hits[k] & ((1ull << lane) - 1)));
        before += s.total;
        __syncthreads();
    }
    return before;
}
static_assert(kDeep * kTakeWaves == 128, "two cells a lane");

// Sums in front of each of `rows` counts, in LDS; returns the sum of all
template <class Count>
__device__ inline int sums_before(int rows, int *s_before, Ranks &s, Count count) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int before = 0;
    for (int r0 = 0; r0 < rows; r0 += kTakeThreads) {
        const int r = r0 + tid, x = r < rows ? count(r) : 0, incl = cache::wave_sums(x);
        if (lane == 63) s.cell[w] = incl;
        __syncthreads();
        int front = before;
#pragma unroll
        for (int i = 0; i < kTakeWaves; ++i) {
            const int y = s.cell[i];
            front += i < w ? y : 0;
            before += y;
        }
        if (r < rows) s_before[r] = front + incl - x;
        __syncthreads();
    }
    return before;
}
// the last of `rows` sums that is at most x
__device__ inline int row_of(int rows, const int *s_before, int x) {
    int lo = 0, hi = rows - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s_before[mid] <= x) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Hands out the `wanted` lowest free pages: set(x, page) for the x-th, -1 where there is none
template <class Set>
__device__ inline void hand_out(const Pool &g, int wanted, const Counts &c, Ranks &s, int32_t *shortage, Set set) {
    const int all = ranked_pages(g.refs, g.num_pages, wanted, c, s, [](int x) { return x <= 0; },
                                 [&](int page, int rank) {
                                     if (rank >= wanted) return;
                                     g.refs[page] = 1;
                                     set(rank, page);
                                 });
    const int found = min(all, wanted);
    for (int x = found + threadIdx.x; x < wanted; x += kTakeThreads) set(x, -1);
    if (threadIdx.x == 0 && shortage != nullptr) *shortage = wanted - found;
}

// ------------------------------------------------------------------------------------------ resize
struct ResizeArgs {
    Pool g;
    const int32_t *old_lens, *new_lens;
    int rows;
    int32_t *shortage;                     // or nullptr
};

__global__ void __launch_bounds__(256) pages_release_kernel(ResizeArgs a) {
    const int r = blockIdx.x, want = blocks_of(a.new_lens[r]), have = blocks_of(a.old_lens[r]);
    int32_t *row = a.g.row(r);
    if (r == 0 && blockIdx.y == 0 && threadIdx.x == 0 && a.shortage != nullptr) *a.shortage = 0;
    for (int64_t j = (int64_t)want + blockIdx.y * 256 + threadIdx.x; j < have; j += 256 * gridDim.y) {
        const int page = row[j];
        if (a.g.is_page(page)) atomicSub(&a.g.refs[page], 1);
        row[j] = -1;
    }
}

__global__ void __launch_bounds__(kTakeThreads) pages_take_kernel(ResizeArgs a) {
    __shared__ int s_before[kMostRows], s_have[kMostRows];
    __shared__ Ranks s_ranks;
    Counts c;
    c.load(a.g.refs, 0, a.g.num_pages);
    const int wanted = sums_before(a.rows, s_before, s_ranks, [&](int r) {
        const int have = blocks_of(a.old_lens[r]);
        s_have[r] = have;
        return max(blocks_of(a.new_lens[r]) - have, 0);
    });
    hand_out(a.g, wanted, c, s_ranks, a.shortage, [&](int x, int page) {
        const int r = row_of(a.rows, s_before, x);
        a.g.row(r)[s_have[r] + (x - s_before[r])] = page;
    });
}

// ------------------------------------------------------------------------------------------ fork
struct ForkArgs {
    Pool g;
    const infllmv2_fork *forks;
    int count;
    int pitch_log2;                        // >= 0: pages are shared by the workgroup that hands out, 2^pitch_log2 >= the blocks of any fork
    int per;                               // forks of a workgroup that only shares
    int32_t *copies, *shortage;            // (each or nullptr)
};

// A count that a thread changes for several forks in turn, added up as long as they name the same page: forks of one source share its pages, and the
// rows they take the place of mostly did
struct Change {
    int page = -1, by = 0;
    __device__ inline void add(const Pool &g, int to, int d) {
        if (to != page) {
            flush(g);
            page = to;
            by = 0;
        }
        by += d;
    }
    __device__ inline void flush(const Pool &g) {
        if (by != 0 && g.is_page(page)) atomicAdd(&g.refs[page], by);
    }
};
// block j of a fork: what the row holds, what it gets (a page that stays needs no change)
struct Shared {
    int was, page;
    __device__ inline void load(const Pool &g, const infllmv2_fork &f, int64_t j) {
        was = j < blocks_of(f.old_tokens) ? g.row(f.dst)[j] : -1;
        page = j < f.tokens / kBlock ? g.row(f.src)[j] : -1;
        if (!g.is_page(page)) page = -1;
    }
    __device__ inline void apply(const Pool &g, const infllmv2_fork &f, int64_t j, Change &gained, Change &lost) const {
        if (j >= max(blocks_of(f.tokens), blocks_of(f.old_tokens))) return;
        if (was != page) {
            gained.add(g, page, 1);
            lost.add(g, was, -1);
        }
        if (was != page || page < 0) g.row(f.dst)[j] = page;
    }
};

// whole pages shared, what the row held before given back: a workgroup goes through a.per forks
__global__ void __launch_bounds__(256) pages_share_kernel(ForkArgs a) {
    const int first = blockIdx.x * a.per, end = min(first + a.per, a.count);
    int most = 0;
    for (int i = first; i < end; ++i) most = max(most, max(blocks_of(a.forks[i].tokens), blocks_of(a.forks[i].old_tokens)));
    for (int64_t j = blockIdx.y * 256 + threadIdx.x; j < most; j += 256 * gridDim.y) {
        Change gained, lost;
        for (int i0 = first; i0 < end; i0 += 8) {
            Shared s[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (i0 + k < end) s[k].load(a.g, a.forks[i0 + k], j);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (i0 + k < end) s[k].apply(a.g, a.forks[i0 + k], j, gained, lost);
        }
        gained.flush(a.g);
        lost.flush(a.g);
    }
}

// a page for every last one that is not whole
__global__ void __launch_bounds__(kTakeThreads) pages_split_kernel(ForkArgs a) {
    __shared__ int s_before[kMostRows], s_from[kMostRows];
    __shared__ Ranks s_ranks;
    Counts c;
    if (a.pitch_log2 >= 0) {
        const int items = a.count << a.pitch_log2;
        for (int i0 = threadIdx.x; i0 < items; i0 += 4 * kTakeThreads) {
            Shared s[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = i0 + k * kTakeThreads;
                if (i < items) s[k].load(a.g, a.forks[i >> a.pitch_log2], i & ((1 << a.pitch_log2) - 1));
            }
            Change gained, lost;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = i0 + k * kTakeThreads;
                if (i < items) s[k].apply(a.g, a.forks[i >> a.pitch_log2], i & ((1 << a.pitch_log2) - 1), gained, lost);
            }
            gained.flush(a.g);
            lost.flush(a.g);
        }
        __threadfence();                   // (the counts below are read as the atomics left them; entries are written again behind these)
        __syncthreads();
    }
    c.load(a.g.refs, 0, a.g.num_pages);
    auto copy = [&](int i, int from, int to) {
        if (a.copies == nullptr) return;
        a.copies[2 * i] = from;
        a.copies[2 * i + 1] = to;
    };
    const int wanted = sums_before(a.count, s_before, s_ranks, [&](int i) {
        const infllmv2_fork f = a.forks[i];
        const int page = f.tokens % kBlock != 0 ? a.g.row(f.src)[f.tokens / kBlock] : -1;          // the page that is continued
        s_from[i] = page;
        if (a.g.is_page(page)) return 1;
        copy(i, -1, -1);
        return 0;
    });
    hand_out(a.g, wanted, c, s_ranks, a.shortage, [&](int x, int page) {
        const int i = row_of(a.count, s_before, x);
        const infllmv2_fork f = a.forks[i];
        a.g.row(f.dst)[f.tokens / kBlock] = page;
        copy(i, page >= 0 ? s_from[i] : -1, page);
    });
}

// ------------------------------------------------------------------------------------------ compact
struct CompactArgs {
    Pool g, out;
    const int32_t *lens;
    int rows, blocks, out_rows, out_blocks;        // rows: with lengths; those of `out` behind them get no pages
    int32_t *moves, *live;                 // [num_pages / 2][2], [2]: pages in use, moves
};

// The counts by the new numbers, and the entries of the table; move(i): the i-th move.  In may be out: an entry, and the two counts of a move, are one thread's.
template <class Move>
__device__ inline void renumber_counts(const CompactArgs &a, int used, int n, int64_t first, int64_t step, Move move) {
    for (int64_t g = first; g < a.g.num_pages; g += step) {
        // (counts of moved pages are the move's: of one of those, read while it changes, the same comes out either way)
        const int x = a.g.refs[g];
        if (g < used ? x > 0 : x <= 0) a.out.refs[g] = g < used ? x : 0;
        if (g < n) {
            const int2 m = move((int)g);
            const int y = a.g.refs[m.x];
            a.out.refs[m.y] = y;
            a.out.refs[m.x] = 0;
        }
    }
}
template <class Move>
__device__ inline void renumber_entries(const CompactArgs &a, int used, int n, int64_t first, int64_t step, Move move) {
    const int64_t entries = (int64_t)a.out_rows * a.out_blocks;
    for (int64_t i = first; i < entries; i += step) {
        const int r = (int)(i / a.out_blocks), j = (int)(i - (int64_t)r * a.out_blocks);
        if (r >= a.rows) {
            a.out.row(r)[j] = -1;
            continue;
        }
        int page = a.g.row(r)[min(j, a.blocks - 1)];                  // (beside the length, not behind it)
        if (j >= min(blocks_of(a.lens[r]), a.blocks) || !a.g.is_page(page)) page = -1;
        if (page >= used) {                // (pages to move are in order; seven looked at together take longer: 9.1 us of the kernel, not 5.2)
            int lo = 0, hi = n;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (move(mid).x < page) lo = mid + 1;
                else hi = mid;
            }
            const int2 m = lo < n ? move(lo) : int2{-1, -1};
            page = m.x == page ? m.y : -1;
        }
        a.out.row(r)[j] = page;
    }
}

// Pages (whose moves are kept in LDS) and entries up to which the workgroup that finds the moves renumbers as well, one launch for two: with the copies, 331 pages and
// 299 entries 14.0 -> 11.8 us, 1300 and 940 13.6 -> 11.5, 2600 and 1890 14.1 -> 13.0, 4000 and 2840 18.7 -> 19.2.
constexpr int kSmallPages = 4096, kSmallEntries = 2048;

// Of the pages in use those from number `used` on move, in order, to the free ones below it, in order: there are as many of either.
template <bool SMALL>
__global__ void __launch_bounds__(kTakeThreads) pages_moves_kernel(CompactArgs a) {
    __shared__ Ranks s_ranks;
    __shared__ int2 s_moves[SMALL ? kSmallPages / 2 : 1];
    const auto in_use = [](int x) { return x > 0; };
    Counts c;
    c.load(a.g.refs, 0, a.g.num_pages);
    const int used = ranked_pages(a.g.refs, a.g.num_pages, INT32_MAX, c, s_ranks, in_use, [](int, int) {});
    const int n = ranked_pages(a.g.refs, used, INT32_MAX, c, s_ranks, [](int x) { return x <= 0; }, [&](int g, int rank) {
        a.moves[2 * rank + 1] = g;
        if (SMALL) s_moves[rank].y = g;
    });
    if (n > 0) {
        c.load(a.g.refs + used, 0, a.g.num_pages - used);
        ranked_pages(a.g.refs + used, a.g.num_pages - used, INT32_MAX, c, s_ranks, in_use, [&](int g, int rank) {
            a.moves[2 * rank] = used + g;
            if (SMALL) s_moves[rank].x = used + g;
        });
    }
    for (int64_t i = 2 * (int64_t)n + threadIdx.x; i < a.g.num_pages / 2 * 2; i += kTakeThreads) a.moves[i] = -1;
    if (threadIdx.x == 0) a.live[0] = used, a.live[1] = n;
    if constexpr (SMALL) {                 // (every count has been read: ranked_pages ends with a barrier)
        const auto move = [&](int i) { return s_moves[i]; };
        renumber_entries(a, used, n, threadIdx.x, kTakeThreads, move);
        renumber_counts(a, used, n, threadIdx.x, kTakeThreads, move);
    }
}

__global__ void __launch_bounds__(256) pages_renumber_kernel(CompactArgs a) {
    const int used = a.live[0], n = a.live[1];
    const auto move = [&](int i) { return int2{a.moves[2 * (int64_t)i], a.moves[2 * (int64_t)i + 1]}; };
    const int64_t step = (int64_t)gridDim.x * 256;
    if (blockIdx.y == 0) renumber_counts(a, used, n, (int64_t)blockIdx.x * 256 + threadIdx.x, step, move);
    else renumber_entries(a, used, n, ((int64_t)(blockIdx.y - 1) * gridDim.x + blockIdx.x) * 256 + threadIdx.x, (gridDim.y - 1) * step, move);
}

// ------------------------------------------------------------------------------------------ copies
struct CopyArgs {
    cache::Args c;
    const int32_t *pairs;
    int vecs, vecs_log2;                   // 16-byte pieces of a row
};

// a workgroup: K or V of one head of a page; PER pieces a thread
template <int PER>
__global__ void __launch_bounds__(256) cache_copy_kernel(CopyArgs a) {
    const int from = a.pairs[2 * (int64_t)blockIdx.x], to = a.pairs[2 * (int64_t)blockIdx.x + 1], h = blockIdx.y;
    if (from < 0 || from >= a.c.num_pages || to < 0 || to >= a.c.num_pages || from == to) return;
    char *pool = blockIdx.z != 0 ? a.c.v : a.c.k;
    float *scales = blockIdx.z != 0 ? a.c.vs : a.c.ks;
    const char *src = pool + a.c.at(from, h);
    char *dst = pool + a.c.at(to, h);
    Piece x[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const int v = threadIdx.x + e * 256;
        x[e] = *reinterpret_cast<const Piece *>(src + (v >> a.vecs_log2) * a.c.tok_stride + (v & (a.vecs - 1)) * 16);
    }
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const int v = threadIdx.x + e * 256;
        *reinterpret_cast<Piece *>(dst + (v >> a.vecs_log2) * a.c.tok_stride + (v & (a.vecs - 1)) * 16) = x[e];
    }
    if (threadIdx.x == 0 && scales != nullptr) scales[(int64_t)to * a.c.hkv + h] = scales[(int64_t)from * a.c.hkv + h];
}

int check_pages(const infllmv2_pages *g) {
    if (g == nullptr || g->num_pages < 1 || g->rows < 1 || g->blocks < 1 || g->table_stride < g->blocks || g->reserved != 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (g->page_table_d == nullptr || g->refs_d == nullptr) return INFLLMV2_ERR_INVALID_ARGUMENT;
    return INFLLMV2_OK;
}
bool fits(const infllmv2_pages *g, int tokens) { return tokens >= 0 && blocks_of(tokens) <= g->blocks; }
int pitch_log2(int x) {                    // least power of two that is at least x
    int p = 0;
    while ((1ll << p) < x) ++p;
    return p;
}
// Blocks of forks, with those that a fork does not have, up to which one workgroup shares them and hands out pages after it, one launch for two: 4 forks of 500 tokens
// and their copies 14.0 -> 11.2 us, 32 of 3000 14.8 -> 12.2, 64 of 4000 14.9 -> 14.4.  (Entries that are given back by the workgroup that hands out: 64 rows with
// 3000 of them 8.7 -> 14.7 us of kernels, with 30 to 400 no gain.)
constexpr int64_t kTogether = 4096;
unsigned chunks(int64_t entries, int per) { return (unsigned)std::max<int64_t>(std::min<int64_t>((entries + per - 1) / per, 64), 1); }

}  // namespace

}  // namespace ifv2

extern "C" int infllmv2_pages_resize(const infllmv2_pages *g, const int32_t *old_lens_h, const int32_t *old_lens_d, const int32_t *new_lens_h,
                                     const int32_t *new_lens_d, int32_t batch, int32_t *short_d, void *stream) {
    using namespace ifv2;
    const int st = check_pages(g);
    if (st) return st;
    if (batch < 0 || batch > g->rows) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (batch == 0) return INFLLMV2_OK;
    if (old_lens_h == nullptr || old_lens_d == nullptr || new_lens_h == nullptr || new_lens_d == nullptr) return INFLLMV2_ERR_INVALID_ARGUMENT;
    int64_t more = 0;
    int less = 0;                                                    // the most blocks that a sequence gives back
    for (int b = 0; b < batch; ++b) {
        if (!fits(g, old_lens_h[b]) || !fits(g, new_lens_h[b])) return INFLLMV2_ERR_INVALID_ARGUMENT;
        const int change = blocks_of(new_lens_h[b]) - blocks_of(old_lens_h[b]);
        if (change > 0) more += change;
        less = std::max(less, -change);
    }
    if (batch > kMostRows || more > INT32_MAX) return INFLLMV2_ERR_UNSUPPORTED;
    if (less == 0 && more == 0 && short_d == nullptr) return INFLLMV2_OK;
    const ResizeArgs a{pool_of(g), old_lens_d, new_lens_d, batch, short_d};
    if (less > 0) hipLaunchKernelGGL(pages_release_kernel, dim3(batch, chunks(less, 256)), dim3(256), 0, (hipStream_t)stream, a);
    if (more > 0 || less == 0) hipLaunchKernelGGL(pages_take_kernel, dim3(1), dim3(kTakeThreads), 0, (hipStream_t)stream, a);
    return hip_status(hipGetLastError());
}

extern "C" int infllmv2_pages_fork(const infllmv2_pages *g, const infllmv2_fork *forks_h, const infllmv2_fork *forks_d, int32_t count,
                                   int32_t *copies_d, int32_t *short_d, void *stream) {
    using namespace ifv2;
    const int st = check_pages(g);
    if (st) return st;
    if (count < 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (count == 0) return INFLLMV2_OK;
    if (forks_h == nullptr || forks_d == nullptr || ((uintptr_t)forks_d & 15) != 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (g->rows > kMostRows || count > kMostRows) return INFLLMV2_ERR_UNSUPPORTED;
    uint64_t to[kMostRows / 64] = {};                                // rows that are written
    int most = 0;
    bool part = false;
    for (int i = 0; i < count; ++i) {
        const infllmv2_fork &f = forks_h[i];
        if (f.src < 0 || f.src >= g->rows || f.dst < 0 || f.dst >= g->rows || !fits(g, f.tokens) || !fits(g, f.old_tokens)) return INFLLMV2_ERR_INVALID_ARGUMENT;
        if (to[f.dst / 64] >> (f.dst % 64) & 1) return INFLLMV2_ERR_INVALID_ARGUMENT;
        to[f.dst / 64] |= 1ull << (f.dst % 64);
        most = std::max(most, blocks_of(std::max(f.tokens, f.old_tokens)));
        part = part || f.tokens % kBlock != 0;
    }
    for (int i = 0; i < count; ++i)
        if (to[forks_h[i].src / 64] >> (forks_h[i].src % 64) & 1) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (most == 0 && copies_d == nullptr && short_d == nullptr) return INFLLMV2_OK;
    const int pitch = pitch_log2(most);
    const bool together = most > 0 && (int64_t)count << pitch <= kTogether;
    // Forks of a workgroup: more add up more of their counts, as long as there is a workgroup for each CU.  A call, us, all pages others than before, in order in the pool, by 1 / 2 / 4 / 8 / 16 forks:
    // 240 of 512 blocks 10.9 / 9.2 / 9.7 / 11.6 / 18.3 (1 here), 1000 of 100 14.8 / 11.2 / 10.6 / 12.2 / 17.7 (3), 3000 of 64 65 / 37 / 25 / 21 / 23 (11).
    const int per = (int)std::max<int64_t>(std::min<int64_t>((int64_t)count * chunks(most, 256) / 256, 16), 1);
    const ForkArgs a{pool_of(g), forks_d, count, together ? pitch : -1, per, copies_d, short_d};
    if (most > 0 && !together) hipLaunchKernelGGL(pages_share_kernel, dim3((count + per - 1) / per, chunks(most, 256)), dim3(256), 0, (hipStream_t)stream, a);
    if (part || together || copies_d != nullptr || short_d != nullptr) hipLaunchKernelGGL(pages_split_kernel, dim3(1), dim3(kTakeThreads), 0, (hipStream_t)stream, a);
    return hip_status(hipGetLastError());
}

extern "C" int infllmv2_pages_compact(const infllmv2_pages *g, const int32_t *lens_h, const int32_t *lens_d, int32_t batch,
                                      const infllmv2_pages *out, int32_t *moves_d, int32_t *live_d, void *stream) {
    using namespace ifv2;
    int st = check_pages(g);
    if (!st) st = check_pages(out);
    if (st) return st;
    if (batch < 0 || batch > g->rows || batch > out->rows || out->num_pages != g->num_pages) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if ((batch > 0 && (lens_h == nullptr || lens_d == nullptr)) || (moves_d == nullptr && g->num_pages > 1) || live_d == nullptr) return INFLLMV2_ERR_INVALID_ARGUMENT;
    // in place, or apart
    if ((out->page_table_d == g->page_table_d && out->table_stride != g->table_stride)) return INFLLMV2_ERR_INVALID_ARGUMENT;
    for (int b = 0; b < batch; ++b)
        if (!fits(g, lens_h[b]) || !fits(out, lens_h[b])) return INFLLMV2_ERR_INVALID_ARGUMENT;
    const CompactArgs a{pool_of(g), pool_of(out), lens_d, batch, g->blocks, out->rows, out->blocks, moves_d, live_d};
    const int64_t entries = (int64_t)out->rows * out->blocks;
    if (g->num_pages <= kSmallPages && entries <= kSmallEntries) {
        hipLaunchKernelGGL(pages_moves_kernel<true>, dim3(1), dim3(kTakeThreads), 0, (hipStream_t)stream, a);
        return hip_status(hipGetLastError());
    }
    hipLaunchKernelGGL(pages_moves_kernel<false>, dim3(1), dim3(kTakeThreads), 0, (hipStream_t)stream, a);
    const unsigned x = chunks(g->num_pages, 256), y = 1 + chunks(entries, 256 * (int)x);
    hipLaunchKernelGGL(pages_renumber_kernel, dim3(x, y), dim3(256), 0, (hipStream_t)stream, a);
    return hip_status(hipGetLastError());
}

extern "C" int infllmv2_cache_copy_pages(const infllmv2_params *p, const infllmv2_cache *c, const int32_t *pairs_d, int32_t count, void *stream) {
    using namespace ifv2;
    int st = check_params(p);
    if (st) return st;
    if (count < 0) return INFLLMV2_ERR_INVALID_ARGUMENT;
    if (count == 0) return INFLLMV2_OK;
    if (pairs_d == nullptr) return INFLLMV2_ERR_INVALID_ARGUMENT;
    st = cache::check(p, c, 0, true);
    if (st) return st;
    if (p->num_kv_heads > 65535 || !cache::fits_launch((int64_t)count * p->num_kv_heads * 2, 256)) return INFLLMV2_ERR_UNSUPPORTED;
    const bool codes = c->kv_type == INFLLMV2_CACHE_E4M3;
    const int vecs = p->head_dim * (codes ? 1 : p->dtype == INFLLMV2_BF16 ? 2 : 4) / 16;
    CopyArgs a{cache::args(p, c), pairs_d, vecs, __builtin_ctz(vecs)};
    if (!codes) a.c.ks = a.c.vs = nullptr;
    const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(count, p->num_kv_heads, 2), dim3(256), 0, (hipStream_t)stream, a); };
    if (vecs == 32) launch(cache_copy_kernel<8>);
    else if (vecs == 16) launch(cache_copy_kernel<4>);
    else if (vecs == 8) launch(cache_copy_kernel<2>);
    else launch(cache_copy_kernel<1>);
    return hip_status(hipGetLastError());
}
