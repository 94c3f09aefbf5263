// What happens to cache pages after loma_paged_extend handed them out: back to the free list (loma_paged_release), shared or copied
// when sequences go on from another's cache (loma_paged_fork), moved to the pool's low numbers (loma_paged_compact), and the
// copying itself (loma_paged_copy).
//
// The bookkeeping is integer work on a few numbers per sequence and page; what takes time is the chain of steps that each need
// the whole result of the one before (count every owner, then see which pages have none left, then number them, then hand
// them out).  So a call is one launch of one cluster: eight CTAs of 1024 threads, whose hardware barrier is the step from one
// phase to the next (a fraction of a microsecond, where a launch or a round trip through memory would be one or more), with
// counts exchanged through each other's shared memory.  Pages and sequences are dealt to the CTAs in contiguous parts, so ranks
// follow from block-wide sums and the parts' totals, in ascending order of page or sequence: results repeat bit for bit, and the
// only atomics are additions and ORs of integers.
// Measured with the launch: release of 64 sequences 6 us, of 2000 with 500 000 pages 25; fork of 8 / 256 sequences 9 / 18; compaction of 16
// sequences 10, of 500 with 94 500 pages 27; copy of 21 000 pages of 8 KB in two pools (346 MB in, 346 out) 124 (0.85 of a plain copy).
#include <limits.h>

#include <algorithm>

#include <cooperative_groups.h>

#include "paged_pages.cuh"

namespace cg = cooperative_groups;

namespace loma {

__host__ __device__ static inline int clampi(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }
__host__ __device__ static inline int saturate(int64_t x) { return x > INT_MAX ? INT_MAX : (int)x; }
__host__ __device__ static inline int pages_of(int64_t entries, int log2_ps) { return (int)((entries + (1 << log2_ps) - 1) >> log2_ps); }
__host__ __device__ static inline bool in_pool(const PageList& pl, int page) { return page >= 0 && page < pl.n_pages; }
__host__ __device__ static inline int start_of(const PageList& pl, int taken) { return clampi(taken, 0, pl.n_free); }

// pages that row b keeps of the `held` it has
__host__ __device__ static inline int pages_kept(const ReleaseArgs& a, int keep, int held) {
    const int want = pages_of(keep < 0 ? 0 : keep, a.log2_ps);
    return keep < 0 || want > held ? held : want;
}

// What goes on from row a: pages held, pages that every child names, pages with entries
struct Parent {
    int held, share, used;
};
__host__ __device__ static inline Parent fork_parent(const ForkArgs& a, int row) {
    const int room = a.max_pages << a.log2_ps, len = clampi(a.cache_lens[row], 0, room);
    const int fixed = a.fixed_lens ? clampi(a.fixed_lens[row], 0, len) : len, used = pages_of(len, a.log2_ps);
    Parent p;
    p.held = a.held ? clampi(a.held[row], 0, a.max_pages) : used;
    p.share = (fixed >> a.log2_ps) < p.held ? fixed >> a.log2_ps : p.held;
    p.used = used < p.held ? used : p.held;
    return p;
}
// the parent of row b, or -1
__host__ __device__ static inline int fork_from(const ForkArgs& a, int b) {
    const int p = a.parents[b];
    return p >= 0 && p < a.B ? p : -1;
}

// ------------------------------------------------------------------ host forms
// pages whose count has fallen below 0, in ascending order, go in front of the free list; returns how many, *lost of which had no room
static int host_settle(const PageList& pl, int* lost) {
    int freed = 0;
    for (int p = 0; p < pl.n_pages; ++p) freed += pl.refs[p] < 0;
    const int taken = start_of(pl, *pl.taken), n = std::min(freed, taken);
    int i = 0;
    for (int p = 0; p < pl.n_pages; ++p)
        if (pl.refs[p] < 0) {
            pl.refs[p] = 0;
            if (i < n) pl.free_pages[taken - n + i] = p;
            ++i;
        }
    *pl.taken = taken - n;
    *lost = freed - n;
    return freed;
}

static void put_counts(int32_t* counts, int64_t a, int64_t b, int64_t c, int64_t d) {
    counts[0] = saturate(a);
    counts[1] = saturate(b);
    counts[2] = saturate(c);
    counts[3] = saturate(d);
}

void host_paged_release(const ReleaseArgs& a) {
    for (int b = 0; b < a.B; ++b) {
        const int held = clampi(a.held[b], 0, a.max_pages), kept = pages_kept(a, a.keep_lens[b], held);
        int32_t* row = a.block_table + (int64_t)b * a.max_pages;
        for (int j = kept; j < held; ++j) {
            if (in_pool(a.pl, row[j])) --a.pl.refs[row[j]];
            row[j] = -1;
        }
        a.held_out[b] = kept;
    }
    int lost;
    const int freed = host_settle(a.pl, &lost);
    put_counts(a.counts, 0, freed, lost, 0);
}

void host_paged_fork(const ForkArgs& a) {
    int32_t *kids = a.ws, *heir = a.ws + a.B;
    for (int b = 0; b < a.B; ++b) { kids[b] = 0; heir[b] = INT_MAX; }
    for (int b = 0; b < a.B; ++b) {
        const int p = fork_from(a, b);
        if (p < 0) continue;
        ++kids[p];
        if (b < heir[p]) heir[p] = b;
        if (b == p) heir[p] = -1;   // the sequence itself goes on
    }
    for (int r = 0; r < a.B; ++r) {
        const Parent p = fork_parent(a, r);
        const int32_t* row = a.block_table + (int64_t)r * a.max_pages;
        const int gain = kids[r] - 1, n = kids[r] > 0 ? p.share : p.held;
        for (int j = 0; j < n; ++j)
            if (in_pool(a.pl, row[j])) a.pl.refs[row[j]] += gain;
    }
    int lost;
    const int freed = host_settle(a.pl, &lost), taken = *a.pl.taken;
    const int64_t room = std::min<int64_t>(a.pl.n_free - taken, a.max_copies);
    int64_t drawn = 0;
    for (int b = 0; b < a.B; ++b) {
        const int r = fork_from(a, b);
        int32_t* out = a.table_out + (int64_t)b * a.max_pages;
        for (int j = 0; j < a.max_pages; ++j) out[j] = -1;
        a.lens_out[b] = -1;
        a.held_out[b] = 0;
        if (r < 0) continue;
        const Parent p = fork_parent(a, r);
        const int32_t* row = a.block_table + (int64_t)r * a.max_pages;
        const bool is_heir = heir[r] == (b == r ? -1 : b);
        a.lens_out[b] = a.cache_lens[r];
        for (int j = 0; j < (is_heir ? p.held : p.share); ++j) out[j] = row[j];
        a.held_out[b] = is_heir ? p.held : p.share;
        if (is_heir) continue;
        for (int j = p.share; j < p.used; ++j, ++drawn) {
            if (drawn >= room) continue;
            out[j] = a.pl.free_pages[taken + drawn];
            a.copy_src[drawn] = in_pool(a.pl, row[j]) ? row[j] : -1;
            a.copy_dst[drawn] = out[j];
            ++a.held_out[b];
        }
    }
    const int64_t got = std::min(drawn, room);
    for (int64_t i = got; i < a.max_copies; ++i) a.copy_src[i] = a.copy_dst[i] = -1;
    *a.pl.taken = (int)(taken + got);
    put_counts(a.counts, got, freed, lost, drawn - got);
}

void host_paged_compact(const CompactArgs& a) {
    const PageList& pl = a.pl;
    const int taken = start_of(pl, *pl.taken);
    int32_t* state = a.page_map;   // 1 free, 2 named
    for (int p = 0; p < pl.n_pages; ++p) state[p] = 0;
    for (int i = taken; i < pl.n_free; ++i)
        if (in_pool(pl, pl.free_pages[i])) state[pl.free_pages[i]] = 1;
    for (int b = 0; b < a.B; ++b)
        for (int j = 0; j < clampi(a.held[b], 0, a.max_pages); ++j) {
            const int p = a.block_table[(int64_t)b * a.max_pages + j];
            if (in_pool(pl, p)) state[p] = 2;
        }
    int named = 0, free = 0, rank = 0, from = 0, to = 0;
    for (int p = 0; p < pl.n_pages; ++p) { named += state[p] == 2; free += state[p] == 1; }
    for (int p = 0; p < pl.n_pages; ++p) {
        if (!state[p]) continue;
        const bool low = rank++ < named;
        if (state[p] == 2 && !low && from++ < a.max_copies) a.copy_src[from - 1] = p;
        if (state[p] == 1 && low && to++ < a.max_copies) a.copy_dst[to - 1] = p;
    }
    const int n = std::min(from, a.max_copies);
    for (int i = 0; i < n; ++i) {
        state[a.copy_src[i]] = 1;
        state[a.copy_dst[i]] = 2;
    }
    int at = pl.n_free - free;
    *pl.taken = at;
    for (int p = 0; p < pl.n_pages; ++p) {
        if (state[p] == 1) pl.free_pages[at++] = p;
        a.page_map[p] = p;
    }
    for (int i = 0; i < n; ++i) {
        a.page_map[a.copy_src[i]] = a.copy_dst[i];
        pl.refs[a.copy_dst[i]] = pl.refs[a.copy_src[i]];
        pl.refs[a.copy_src[i]] = 0;
    }
    for (int i = n; i < a.max_copies; ++i) a.copy_src[i] = a.copy_dst[i] = -1;
    for (int b = 0; b < a.B; ++b)
        for (int j = 0; j < clampi(a.held[b], 0, a.max_pages); ++j) {
            int32_t& p = a.block_table[(int64_t)b * a.max_pages + j];
            if (in_pool(pl, p)) p = a.page_map[p];
        }
    put_counts(a.counts, n, free, named, from - n);
}

// ------------------------------------------------------------------ device forms
constexpr int PG_CTAS = 8, PG_THREADS = 1024, PG_WARPS = PG_THREADS / 32, PG_ALL = PG_CTAS * PG_THREADS, PG_ALL_WARPS = PG_CTAS * PG_WARPS;

// A CTA's part [lo, hi) of n things, in units of `unit`
struct Part {
    int64_t lo, hi;
    __device__ __forceinline__ Part(int64_t n, int unit, int rank) {
        const int64_t per = ((n + unit - 1) / unit + PG_CTAS - 1) / PG_CTAS * unit;
        lo = min(per * rank, n);
        hi = min(lo + per, n);
    }
};

__device__ __forceinline__ int64_t warp_exclusive(int64_t x, int64_t* total) {
    const int lane = threadIdx.x & 31;
    int64_t incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
    }
    *total = __shfl_sync(0xffffffffu, incl, 31);
    return incl - x;
}

// Exclusive sums over the warps of a block of one number per warp (the same in all its lanes), and the total.
__device__ __forceinline__ int64_t block_sums(int64_t of_warp, int64_t* total) {
    __shared__ int64_t s_warp[PG_WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __syncthreads();
    if (lane == 0) s_warp[warp] = of_warp;
    __syncthreads();
    const int64_t before = warp_exclusive(s_warp[lane], total);   // one per lane: PG_WARPS is 32
    return __shfl_sync(0xffffffffu, before, warp);
}

// Two numbers of each CTA to every CTA, and a barrier of the cluster; then the sums of the lower ranks' and of everyone's.
// slot: in shared memory, one set per exchange.  put() writes to the other CTAs, so a barrier of the cluster comes before it in every kernel:
// without one a CTA may not have started yet.
struct Exchange {
    int64_t slot[2][PG_CTAS];
    __device__ __forceinline__ void put(cg::cluster_group& cl, int64_t x, int64_t y) {
        const int rank = cl.block_rank();
        if (threadIdx.x < 2 * PG_CTAS) {
            const int i = threadIdx.x / PG_CTAS, to = threadIdx.x % PG_CTAS;
            *cl.map_shared_rank(&slot[i][rank], to) = i ? y : x;
        }
        cl.sync();
    }
    __device__ __forceinline__ int64_t get(int i, int rank, int64_t* all) const {
        int64_t before = 0, sum = 0;
#pragma unroll
        for (int r = 0; r < PG_CTAS; ++r) {
            before += r < rank ? slot[i][r] : 0;
            sum += slot[i][r];
        }
        *all = sum;
        return before;
    }
};

// Pages of a CTA's part by words of 32, a word to a warp at a time: a lane loads one page's number, a ballot makes the word, and the words'
// counts are summed up over the block.  N kinds of pages are told apart at once.
template <int N>
struct Words {
    static constexpr int MAX = 2048;        // words at a time: pools of up to 8 x 65536 pages are looked at once
    unsigned mask[N][MAX];
    int before[N][MAX];                     // pages of the kind in the words before

    // words of pages [lo, hi); kind(value, k) says whether a page belongs to kind k.  Ends with a barrier.
    template <typename F>
    __device__ __forceinline__ void fill(const int32_t* values, int64_t lo, int64_t hi, F&& kind) {
        constexpr int AHEAD = 8;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, words = (int)((hi - lo + 31) / 32);
        for (int w0 = warp; w0 < words; w0 += PG_WARPS * AHEAD) {
            int v[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int64_t p = lo + (int64_t)(w0 + u * PG_WARPS) * 32 + lane;
                v[u] = p < hi ? __ldcg(values + p) : 0;          // 0: of no kind
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int w = w0 + u * PG_WARPS;
                if (w >= words) break;
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const unsigned m = __ballot_sync(0xffffffffu, kind(v[u], k));
                    if (lane == 0) mask[k][w] = m;
                }
            }
        }
        __syncthreads();
    }
    // the sums; total[k]: pages of kind k.  Ends with a barrier.
    __device__ __forceinline__ void sum(int words, int64_t (&total)[N]) {
        constexpr int PER = MAX / PG_THREADS;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            int n[PER];
            int64_t mine = 0, of_warp;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int w = threadIdx.x * PER + i;
                n[i] = w < words ? __popc(mask[k][w]) : 0;
                mine += n[i];
            }
            const int64_t in_warp = warp_exclusive(mine, &of_warp);
            int at = (int)(block_sums(of_warp, &total[k]) + in_warp);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int w = threadIdx.x * PER + i;
                if (w < words) before[k][w] = at;
                at += n[i];
            }
        }
        __syncthreads();
    }
};
// the part [lo, hi) in stretches that fit
template <typename F>
__device__ __forceinline__ void stretches(const Part& part, F&& body) {
    constexpr int64_t STEP = 32 * Words<1>::MAX;
    for (int64_t lo = part.lo; lo < part.hi; lo += STEP) body(lo, min(lo + STEP, part.hi), part.hi - part.lo > STEP);
}

// The pages without an owner, numbered by all CTAs.  count() needs the owners' counts complete (a barrier of the cluster before); between
// it and write() the CTAs' totals are exchanged.
struct Settle {
    Words<1>& words;
    const Part part;
    __device__ __forceinline__ Settle(Words<1>& w, const PageList& pl, int rank) : words(w), part(pl.n_pages, 32, rank) {}

    __device__ __forceinline__ int64_t look(const PageList& pl, int64_t lo, int64_t hi) const {
        int64_t total[1];
        words.fill(pl.refs, lo, hi, [](int v, int) { return v < 0; });
        words.sum((int)((hi - lo + 31) / 32), total);
        return total[0];
    }
    __device__ __forceinline__ int64_t count(const PageList& pl) const {
        int64_t n = 0;
        stretches(part, [&](int64_t lo, int64_t hi, bool) { n += look(pl, lo, hi); });
        return n;
    }
    // `at`: the number of this CTA's first page; the first n of all go to the places in front of `taken`
    __device__ __forceinline__ void write(const PageList& pl, int64_t at, int64_t n, int taken) const {
        const int lane = threadIdx.x & 31;
        stretches(part, [&](int64_t lo, int64_t hi, bool again) {
            const int64_t here = again ? look(pl, lo, hi) : 0;
            for (int w = threadIdx.x >> 5; w < (hi - lo + 31) / 32; w += PG_WARPS) {
                const unsigned m = words.mask[0][w];
                if (!(m >> lane & 1)) continue;
                const int64_t k = at + words.before[0][w] + __popc(m & ((1u << lane) - 1)), page = lo + w * 32 + lane;
                pl.refs[page] = 0;
                if (k < n) pl.free_pages[taken - n + k] = (int)page;
            }
            at += here;
            if (again) __syncthreads();
        });
    }
    // in place of write(): the number of a word's lowest page, less 2^31, in the place of its count; list_pages does the rest
    __device__ __forceinline__ void mark(const PageList& pl, int64_t at) const {
        stretches(part, [&](int64_t lo, int64_t hi, bool again) {
            const int64_t here = again ? look(pl, lo, hi) : 0;
            for (int w = threadIdx.x; w < (hi - lo + 31) / 32; w += PG_THREADS) {
                const unsigned m = words.mask[0][w];
                if (m) pl.refs[lo + w * 32 + __ffs(m) - 1] = (int)(INT_MIN + at + words.before[0][w]);
            }
            at += here;
            if (again) __syncthreads();
        });
    }
};
// the first n of the pages without an owner to the places from `taken` on, a word to a warp at a time
__device__ __forceinline__ void list_pages(const PageList& pl, int n, int taken, int64_t warp, int64_t warps) {
    const int lane = threadIdx.x & 31;
    for (int64_t w = warp; w < (pl.n_pages + 31) / 32; w += warps) {
        const int64_t page = w * 32 + lane;
        const int v = page < pl.n_pages ? __ldcg(pl.refs + page) : 0;
        const unsigned m = __ballot_sync(0xffffffffu, v < 0);
        const int first = __shfl_sync(0xffffffffu, v, __ffs(m | 1u << 31) - 1) & INT_MAX;
        if (v < 0) {
            const int k = first + __popc(m & ((1u << lane) - 1));
            pl.refs[page] = 0;
            if (k < n) pl.free_pages[taken + k] = (int)page;
        }
    }
}

// Rows of a release: a warp to a row at a time.  held_out may be held itself: a row's count is written behind a barrier of the warp, when all
// its lanes have read it (one row ahead), and the count of a row is read and written by one warp alone.
__device__ __forceinline__ void drop_rows(const ReleaseArgs& a, int first, int warps) {
    const int lane = threadIdx.x & 31;
    int keep = 0, held = 0;
    if (first < a.B) { keep = __ldg(a.keep_lens + first); held = __ldcg(a.held + first); }
    for (int b = first; b < a.B; b += warps) {
        const int h = clampi(held, 0, a.max_pages), kept = pages_kept(a, keep, h);
        if (b + warps < a.B) { keep = __ldg(a.keep_lens + b + warps); held = __ldcg(a.held + b + warps); }
        int32_t* row = a.block_table + (int64_t)b * a.max_pages;
#pragma unroll 4
        for (int j = kept + lane; j < h; j += 32) {
            const int page = row[j];
            if (in_pool(a.pl, page)) atomicSub(a.pl.refs + page, 1);
            row[j] = -1;
        }
        __syncwarp();
        if (lane == 0) a.held_out[b] = kept;
    }
}

// Batches of more rows than a cluster has warps let go of their pages in a launch of their own, over all SMs.
constexpr int DROP_THREADS = 256;
__global__ void __launch_bounds__(DROP_THREADS) paged_drop_kernel(const ReleaseArgs a) {
    let_next_start();
    drop_rows(a, (threadIdx.x >> 5) * gridDim.x + blockIdx.x, gridDim.x * (DROP_THREADS / 32));
}

// list: a launch over all SMs that lists the pages comes behind
template <bool DROPPED>
__global__ void __cluster_dims__(PG_CTAS, 1, 1) __launch_bounds__(PG_THREADS) paged_release_kernel(const ReleaseArgs a, const bool list) {
    cg::cluster_group cl = cg::this_cluster();
    __shared__ Exchange ex;
    __shared__ Words<1> words;
    const int rank = cl.block_rank();
    let_next_start();
    if constexpr (DROPPED) wait_for_previous();
    const int taken = start_of(a.pl, __ldcg(a.pl.taken));
    if constexpr (!DROPPED) drop_rows(a, (threadIdx.x >> 5) * PG_CTAS + rank, PG_ALL_WARPS);   // neighbours on different SMs
    cl.sync();
    const Settle s(words, a.pl, rank);
    int64_t freed;
    const int64_t mine = s.count(a.pl);
    ex.put(cl, mine, 0);
    const int64_t at = ex.get(0, rank, &freed), n = min(freed, (int64_t)taken);
    if (mine > 0 && list) s.mark(a.pl, at);
    else if (mine > 0) s.write(a.pl, at, n, taken);
    if (rank == 0 && threadIdx.x == 0) {
        *a.pl.taken = (int)(taken - n);
        a.counts[0] = 0;
        a.counts[1] = saturate(freed);
        a.counts[2] = saturate(freed - n);
        a.counts[3] = 0;
    }
}

__global__ void __launch_bounds__(DROP_THREADS) paged_list_kernel(const ReleaseArgs a) {
    wait_for_previous();
    const int freed = __ldcg(a.counts + 1);
    if (freed > 0)
        list_pages(a.pl, freed - __ldcg(a.counts + 2), __ldcg(a.pl.taken), (int64_t)(threadIdx.x >> 5) * gridDim.x + blockIdx.x, (int64_t)gridDim.x * (DROP_THREADS / 32));
}

// Pages that a release may free beyond which they are listed over all SMs: eight SMs store them at 20 bytes a cycle each.  Measured (us, in the
// cluster against a launch of its own): 125 000 pages 13.2 / 15.9, 250 000 22.3 / 22.7, 500 000 34.1 / 29.5, a million 70 / 56.  The host
// knows what may be freed, not what is: 64 pages that come back to a pool pay for the look through its counts and, past this bound, for that
// launch: pools of 512 / 230 000 / 300 000 / 500 000 / a million pages 6 / 11 / 15 / 18 / 40.
constexpr int PG_LIST = 1 << 18;

// Rows to a cluster's warp beyond which the rows' own work goes over all SMs in launches of its own, each behind the other.  Measured (us, one
// launch against several, up to 1900 entries in pages of 16, tables of 128 columns): 128 / 256 / 320 / 1000 sequences: fork 12.5 / 13.4 / 16.1 / 25.7
// against 14.3 / 15.5 / 15.7 / 18.9; release 8.7 / 9.3 / 9.7 / 18.3 against 8.9 / 9.3 / 9.5 / 12.7; compaction, which would change over
// at 128 by itself, 17.5 / 21.4 / 25.3 / 54.5 against 17.4 / 18.5 / 19.2 / 27.0.  Columns shift it little: 256 forks with tables of 32 / 512 columns 10.9 /
// 17.4 against 12.9 / 19.2, 256 releases with 512 columns 17.4 against 16.4.
constexpr int PG_ROWS = 1, PG_FEW = PG_ROWS * PG_ALL_WARPS;

// rows' owners gained and lost; kids_of: children of a row
template <typename F>
__device__ __forceinline__ void change_owners(const ForkArgs& a, int first, int warps, F&& kids_of) {
    const int lane = threadIdx.x & 31;
    for (int r = first; r < a.B; r += warps) {
        const Parent p = fork_parent(a, r);
        const int k = kids_of(r), n = k > 0 ? p.share : p.held;
        if (k == 1) continue;
        const int32_t* row = a.block_table + (int64_t)r * a.max_pages;
#pragma unroll 4
        for (int j = lane; j < n; j += 32) {
            const int page = __ldg(row + j);
            if (in_pool(a.pl, page)) atomicAdd(a.pl.refs + page, k - 1);
        }
    }
}

// One row of the new table by a warp.  r: its parent or -1; all: it takes over all the parent's pages; draw: the number of its first fresh
// page, of which `room` can be had, from free_pages[from] on.
__device__ __forceinline__ void write_row(const ForkArgs& a, int64_t b, int r, bool all, int64_t draw, int64_t room, int from) {
    const int lane = threadIdx.x & 31;
    int32_t* out = a.table_out + b * a.max_pages;
    if (r < 0) {
        for (int j = lane; j < a.max_pages; j += 32) out[j] = -1;
        if (lane == 0) { a.lens_out[b] = -1; a.held_out[b] = 0; }
        return;
    }
    const Parent p = fork_parent(a, r);
    const int32_t* row = a.block_table + (int64_t)r * a.max_pages;
    const int named = all ? p.held : p.share, used = all ? p.held : p.used;
#pragma unroll 8
    for (int j = lane; j < a.max_pages; j += 32) {
        int page = j < used ? __ldg(row + j) : -1;
        if (j >= named && j < used) {
            const int64_t i = draw + j - named;
            const int was = page;
            page = -1;
            if (i < room) {
                page = __ldcg(a.pl.free_pages + from + i);
                a.copy_src[i] = in_pool(a.pl, was) ? was : -1;
                a.copy_dst[i] = page;
            }
        }
        out[j] = page;
    }
    if (lane == 0) {
        a.lens_out[b] = a.cache_lens[r];
        a.held_out[b] = named + (int)min(max(room - draw, (int64_t)0), (int64_t)(used - named));
    }
}

// One launch (ALL: up to PG_FEW rows, whose children every CTA counts for itself in shared memory), or the two parts that need every row's result, with owners and rows in launches over all SMs between and behind them:
// COUNT (children and heirs into the workspace) and NUMBER (free pages, draws; the workspace's first half takes the draws' numbers).
enum ForkPart { FORK_ALL, FORK_COUNT, FORK_NUMBER };

template <int PART>
__global__ void __cluster_dims__(PG_CTAS, 1, 1) __launch_bounds__(PG_THREADS) paged_fork_kernel(const ForkArgs a) {
    cg::cluster_group cl = cg::this_cluster();
    __shared__ Exchange ex;
    __shared__ Words<1> words;
    __shared__ int32_t s_kids[PG_FEW], s_heir[PG_FEW], s_start[PG_FEW / PG_CTAS];
    const int rank = cl.block_rank();
    const int64_t me = (int64_t)rank * PG_THREADS + threadIdx.x;
    constexpr bool local = PART == FORK_ALL;
    int32_t *kids = local ? s_kids : a.ws, *heir = local ? s_heir : a.ws + a.B;
    let_next_start();
    if constexpr (PART == FORK_NUMBER) wait_for_previous();
    const int taken = start_of(a.pl, __ldcg(a.pl.taken));
    if constexpr (PART != FORK_NUMBER) {
        const int64_t b0 = local ? threadIdx.x : me, step = local ? PG_THREADS : PG_ALL;
        auto together = [&] { if (local) __syncthreads(); else cl.sync(); };
        for (int64_t b = b0; b < a.B; b += step) { kids[b] = 0; heir[b] = INT_MAX; }
        together();
        for (int64_t b = b0; b < a.B; b += step) {
            const int p = fork_from(a, (int)b);
            if (p < 0) continue;
            atomicAdd(kids + p, 1);
            atomicMin(heir + p, b == p ? -1 : (int)b);
        }
        if constexpr (PART == FORK_COUNT) return;
        together();
        change_owners(a, (threadIdx.x >> 5) * PG_CTAS + rank, PG_ALL_WARPS, [&](int r) { return local ? kids[r] : __ldcg(kids + r); });
    }
    cl.sync();   // owners' counts are complete (NUMBER: the launch before did that), and every CTA runs, so its shared memory may be written to
    auto is_heir = [&](int b, int r) { return (local ? heir[r] : __ldcg(heir + r)) == (b == r ? -1 : b); };
    // pages to draw, numbered through this CTA's rows; in the workspace the numbers take the place of kids
    const Part part(a.B, 1, rank);
    int32_t* const start = local ? s_start : kids;
    const int64_t start0 = local ? part.lo : 0;
    int64_t need_all = 0;
    for (int64_t base = part.lo; base < part.hi; base += PG_THREADS) {
        const int64_t b = base + threadIdx.x;
        int need = 0;
        if (b < part.hi) {
            const int r = fork_from(a, (int)b);
            if (r >= 0 && !is_heir((int)b, r)) {
                const Parent p = fork_parent(a, r);
                need = p.used - p.share;
            }
        }
        int64_t of_warp, total;
        const int64_t in_warp = warp_exclusive(need, &of_warp), before = block_sums(of_warp, &total);
        if (b < part.hi) start[b - start0] = saturate(need_all + before + in_warp);
        need_all += total;
    }
    const Settle s(words, a.pl, rank);
    int64_t freed, drawn;
    const int64_t mine = s.count(a.pl);
    ex.put(cl, mine, need_all);
    const int64_t at = ex.get(0, rank, &freed), back = min(freed, (int64_t)taken), draw0 = ex.get(1, rank, &drawn);
    if (mine > 0) s.write(a.pl, at, back, taken);
    if (PART == FORK_ALL && freed > 0) cl.sync();        // pages that came back are drawn from
    else __syncthreads();
    const int from = (int)(taken - back);
    const int64_t room = min((int64_t)a.pl.n_free - from, (int64_t)a.max_copies), got = min(drawn, room);
    if constexpr (PART == FORK_ALL) {
        for (int64_t b = part.lo + (threadIdx.x >> 5); b < part.hi; b += PG_WARPS) {
            const int r = fork_from(a, (int)b);
            write_row(a, b, r, r >= 0 && is_heir((int)b, r), draw0 + start[b - start0], room, from);
        }
    } else {
        for (int64_t b = part.lo + threadIdx.x; b < part.hi; b += PG_THREADS) kids[b] = saturate(draw0 + kids[b]);
    }
    for (int64_t i = got + me; i < a.max_copies; i += PG_ALL) a.copy_src[i] = a.copy_dst[i] = -1;
    if (rank == 0 && threadIdx.x == 0) {
        *a.pl.taken = (int)(from + got);
        a.counts[0] = saturate(got);
        a.counts[1] = saturate(freed);
        a.counts[2] = saturate(freed - back);
        a.counts[3] = saturate(drawn - got);
    }
}

constexpr int WIDE_THREADS = 256;
__global__ void __launch_bounds__(WIDE_THREADS) paged_owners_kernel(const ForkArgs a) {
    let_next_start();
    wait_for_previous();
    change_owners(a, (threadIdx.x >> 5) * gridDim.x + blockIdx.x, gridDim.x * (WIDE_THREADS / 32), [&](int r) { return __ldcg(a.ws + r); });
}
__global__ void __launch_bounds__(WIDE_THREADS) paged_rows_kernel(const ForkArgs a) {
    let_next_start();
    wait_for_previous();
    const int from = __ldcg(a.pl.taken) - __ldcg(a.counts);
    const int64_t room = min((int64_t)a.pl.n_free - from, (int64_t)a.max_copies);
    for (int64_t b = (threadIdx.x >> 5) * gridDim.x + blockIdx.x; b < a.B; b += gridDim.x * (WIDE_THREADS / 32)) {
        const int r = fork_from(a, (int)b);
        write_row(a, b, r, r >= 0 && __ldcg(a.ws + a.B + r) == (b == r ? -1 : (int)b), __ldcg(a.ws + b), room, from);
    }
}

// Every page's state (bit 0: free, bit 1: named), in page_map, from the free list and the tables; and the tables' new numbers: an entry of
// page_map is the page's new number, or -1 - i for the source of move i whose number has not been written yet.
__device__ __forceinline__ void mark_pages(const CompactArgs& a, int64_t thread, int64_t threads, int warp, int warps) {
    const int lane = threadIdx.x & 31;
    for (int64_t i = start_of(a.pl, __ldcg(a.pl.taken)) + thread; i < a.pl.n_free; i += threads) {
        const int p = a.pl.free_pages[i];
        if (in_pool(a.pl, p)) atomicOr(a.page_map + p, 1);
    }
    for (int b = warp; b < a.B; b += warps) {
        const int h = clampi(__ldg(a.held + b), 0, a.max_pages);
#pragma unroll 4
        for (int j = lane; j < h; j += 32) {
            const int p = a.block_table[(int64_t)b * a.max_pages + j];
            if (in_pool(a.pl, p)) atomicOr(a.page_map + p, 2);
        }
    }
}
__device__ __forceinline__ void rename_pages(const CompactArgs& a, int warp, int warps) {
    const int lane = threadIdx.x & 31;
    for (int b = warp; b < a.B; b += warps) {
        const int h = clampi(__ldg(a.held + b), 0, a.max_pages);
        int32_t* row = a.block_table + (int64_t)b * a.max_pages;
#pragma unroll 4
        for (int j = lane; j < h; j += 32) {
            const int p = row[j];
            if (!in_pool(a.pl, p)) continue;
            const int to = __ldcg(a.page_map + p);
            row[j] = to >= 0 ? to : __ldcg(a.copy_dst - 1 - to);
        }
    }
}
// owners of the pages that move, their new numbers, and the end of the list
__device__ __forceinline__ void move_owners(const CompactArgs& a, int64_t count, int64_t thread, int64_t threads) {
    for (int64_t i = thread; i < a.max_copies; i += threads) {
        if (i < count) {
            const int s = __ldcg(a.copy_src + i), d = __ldcg(a.copy_dst + i);
            a.page_map[s] = d;
            a.pl.refs[d] = __ldcg(a.pl.refs + s);
            a.pl.refs[s] = 0;
        } else {
            a.copy_src[i] = a.copy_dst[i] = -1;
        }
    }
}

// Long batches: clearing, marking and renaming in launches of their own, over all SMs.
__global__ void __launch_bounds__(WIDE_THREADS) paged_clear_kernel(const CompactArgs a) {
    let_next_start();
    for (int64_t p = (int64_t)blockIdx.x * WIDE_THREADS + threadIdx.x; p < a.pl.n_pages; p += (int64_t)gridDim.x * WIDE_THREADS) a.page_map[p] = 0;
}
__global__ void __launch_bounds__(WIDE_THREADS) paged_mark_kernel(const CompactArgs a) {
    let_next_start();
    wait_for_previous();
    mark_pages(a, (int64_t)blockIdx.x * WIDE_THREADS + threadIdx.x, (int64_t)gridDim.x * WIDE_THREADS, (threadIdx.x >> 5) * gridDim.x + blockIdx.x,
               gridDim.x * (WIDE_THREADS / 32));
}
__global__ void __launch_bounds__(WIDE_THREADS) paged_rename_kernel(const CompactArgs a) {
    let_next_start();
    wait_for_previous();
    const int count = __ldcg(a.counts);
    if (count > 0) rename_pages(a, (threadIdx.x >> 5) * gridDim.x + blockIdx.x, gridDim.x * (WIDE_THREADS / 32));
    move_owners(a, count, (int64_t)blockIdx.x * WIDE_THREADS + threadIdx.x, (int64_t)gridDim.x * WIDE_THREADS);
}

template <bool WIDE>
__global__ void __cluster_dims__(PG_CTAS, 1, 1) __launch_bounds__(PG_THREADS) paged_compact_kernel(const CompactArgs a) {
    cg::cluster_group cl = cg::this_cluster();
    __shared__ Exchange ex[2];
    __shared__ Words<2> words;
    const PageList& pl = a.pl;
    const int rank = cl.block_rank(), lane = threadIdx.x & 31, warp = threadIdx.x >> 5, first_row = warp * PG_CTAS + rank;
    const int64_t me = (int64_t)rank * PG_THREADS + threadIdx.x;
    int32_t* state = a.page_map;
    let_next_start();
    if constexpr (WIDE) {
        wait_for_previous();
    } else {
        for (int64_t p = me; p < pl.n_pages; p += PG_ALL) state[p] = 0;
        cl.sync();
        mark_pages(a, me, PG_ALL, first_row, PG_ALL_WARPS);
    }
    cl.sync();
    const Part part(pl.n_pages, 32, rank);
    // kind 0: named, kind 1: free and not named
    auto look = [&](int64_t lo, int64_t hi, int64_t (&total)[2]) {
        words.fill(state, lo, hi, [](int v, int k) { return k == 0 ? (v & 2) != 0 : v == 1; });
        words.sum((int)((hi - lo + 31) / 32), total);
    };
    int64_t mine_n = 0, mine_f = 0, all_n, all_f, here[2];
    stretches(part, [&](int64_t lo, int64_t hi, bool) {
        look(lo, hi, here);
        mine_n += here[0];
        mine_f += here[1];
    });
    ex[0].put(cl, mine_n, mine_f);
    const int64_t n0 = ex[0].get(0, rank, &all_n), f0 = ex[0].get(1, rank, &all_f);
    // Of the pages that are free or named the lowest all_n are to be the named ones.  Page p, with f free and n named ones before it, is
    // among them if f + n < all_n.  Named pages above move, in order, to the free ones below.
    int64_t above = 0, moves;
    {
        int64_t n = n0, f = f0, mine = 0;
        stretches(part, [&](int64_t lo, int64_t hi, bool again) {
            if (again) look(lo, hi, here);
            for (int w = threadIdx.x; w < (hi - lo + 31) / 32; w += PG_THREADS) {
                const unsigned named = words.mask[0][w], free = words.mask[1][w];
                const int64_t before = n + words.before[0][w] + f + words.before[1][w];
                if (before + __popc(named | free) <= all_n) continue;
                for (unsigned m = named; m; m &= m - 1) mine += before + __popc((named | free) & ((m & -m) - 1)) >= all_n;
            }
            if (again) { n += here[0]; f += here[1]; __syncthreads(); }
        });
        warp_exclusive(mine, &mine);
        block_sums(mine, &above);
    }
    ex[1].put(cl, above, 0);
    ex[1].get(0, rank, &moves);
    const int64_t count = min(moves, (int64_t)a.max_copies), stay = all_n - moves;   // named pages below: their ranks are 0 .. stay - 1
    {
        int64_t n = n0, f = f0;
        stretches(part, [&](int64_t lo, int64_t hi, bool again) {
            if (again) look(lo, hi, here);
            for (int w = warp; w < (hi - lo + 31) / 32; w += PG_WARPS) {
                const int64_t page = lo + w * 32 + lane;
                if (page >= hi) continue;
                const unsigned wn = words.mask[0][w], wf = words.mask[1][w], below = (1u << lane) - 1;
                const int64_t pn = n + words.before[0][w] + __popc(wn & below), pf = f + words.before[1][w] + __popc(wf & below);
                const bool is_named = wn >> lane & 1, is_free = wf >> lane & 1;
                // of the free pages the first `count` become named (there are that many below), of the named ones those of rank stay ..
                // stay + count - 1 become free
                const bool to = is_free && pf < count, from = is_named && pn >= stay && pn - stay < count;
                if (to) a.copy_dst[pf] = (int)page;
                if (from) a.copy_src[pn - stay] = (int)page;
                if ((is_free && !to) || from)
                    pl.free_pages[pl.n_free - all_f + pf - min(pf, count) + min(max(pn - stay, (int64_t)0), count)] = (int)page;
                state[page] = from ? (int)(-1 - (pn - stay)) : (int)page;
            }
            if (again) { n += here[0]; f += here[1]; __syncthreads(); }
        });
    }
    if (rank == 0 && threadIdx.x == 0) {
        *pl.taken = (int)(pl.n_free - all_f);
        a.counts[0] = saturate(count);
        a.counts[1] = saturate(all_f);
        a.counts[2] = saturate(all_n);
        a.counts[3] = saturate(moves - count);
    }
    if constexpr (WIDE) return;
    cl.sync();
    move_owners(a, count, me, PG_ALL);
    if (count > 0) rename_pages(a, first_row, PG_ALL_WARPS);
}

// Copying: a warp takes 4 KB of one page of one pool at a time, eight 16-byte loads per lane in flight, then as many stores.
constexpr int COPY_THREADS = 256, COPY_BYTES = 4096, COPY_CTAS = 148 * 6;

__global__ void __launch_bounds__(COPY_THREADS) paged_copy_kernel(const __grid_constant__ CopyArgs a) {
    const int lane = threadIdx.x & 31;
    int64_t per = 0;   // pieces of one page in all pools
    for (int k = 0; k < a.n_pools; ++k) per += (a.bytes[k] + COPY_BYTES - 1) / COPY_BYTES;
    wait_for_previous();   // the list is often the result of the launch before this one
    const int64_t n = min(max(__ldcg(a.n), 0), a.max_copies);
    const int64_t warps = (int64_t)gridDim.x * (COPY_THREADS / 32);
    for (int64_t u = (int64_t)(threadIdx.x >> 5) * gridDim.x + blockIdx.x; u < n * per; u += warps) {
        const int64_t i = u / per;
        int64_t piece = u - i * per;
        int k = 0;
        for (int64_t x; piece >= (x = (a.bytes[k] + COPY_BYTES - 1) / COPY_BYTES); ++k) piece -= x;
        const int s = __ldcg(a.src + i), d = __ldcg(a.dst + i);
        if (s < 0 || s >= a.n_pages || d < 0 || d >= a.n_pages || s == d) continue;
        const int64_t at = piece * COPY_BYTES + lane * 16, end = a.bytes[k];
        const uint8_t* from = a.pool[k] + s * end;
        uint8_t* to = a.pool[k] + d * end;
        uint4 x[COPY_BYTES / 512];
#pragma unroll
        for (int y = 0; y < COPY_BYTES / 512; ++y)
            if (at + y * 512 < end) x[y] = *reinterpret_cast<const uint4*>(from + at + y * 512);
#pragma unroll
        for (int y = 0; y < COPY_BYTES / 512; ++y)
            if (at + y * 512 < end) *reinterpret_cast<uint4*>(to + at + y * 512) = x[y];
    }
}

// ------------------------------------------------------------------ host side
cudaError_t launch_paged_release(const ReleaseArgs& a, cudaStream_t st) {
    const bool list = std::min<int64_t>(a.pl.n_pages, (int64_t)a.B * a.max_pages) > PG_LIST, dropped = a.B > PG_FEW;
    cudaError_t e = cudaSuccess;
    if (dropped) {
        const unsigned grid = (unsigned)std::min(148 * 8, (a.B + DROP_THREADS / 32 - 1) / (DROP_THREADS / 32));
        e = launch_behind(paged_drop_kernel, dim3(grid), DROP_THREADS, 0, st, false, a);
    }
    if (e == cudaSuccess) e = launch_behind(dropped ? paged_release_kernel<true> : paged_release_kernel<false>, dim3(PG_CTAS), PG_THREADS, 0, st, dropped, a, list);
    if (e == cudaSuccess && list) e = launch_behind(paged_list_kernel, dim3(148 * 8), DROP_THREADS, 0, st, true, a);
    return e;
}
cudaError_t launch_paged_fork(const ForkArgs& a, cudaStream_t st) {
    if (a.B <= PG_FEW) return launch_behind(paged_fork_kernel<FORK_ALL>, dim3(PG_CTAS), PG_THREADS, 0, st, false, a);
    const dim3 grid((unsigned)std::min(148 * 8, (a.B + WIDE_THREADS / 32 - 1) / (WIDE_THREADS / 32)));
    cudaError_t e = launch_behind(paged_fork_kernel<FORK_COUNT>, dim3(PG_CTAS), PG_THREADS, 0, st, false, a);
    if (e == cudaSuccess) e = launch_behind(paged_owners_kernel, grid, WIDE_THREADS, 0, st, true, a);
    if (e == cudaSuccess) e = launch_behind(paged_fork_kernel<FORK_NUMBER>, dim3(PG_CTAS), PG_THREADS, 0, st, true, a);
    if (e == cudaSuccess) e = launch_behind(paged_rows_kernel, grid, WIDE_THREADS, 0, st, true, a);
    return e;
}
cudaError_t launch_paged_compact(const CompactArgs& a, cudaStream_t st) {
    if (a.B <= PG_FEW) return launch_behind(paged_compact_kernel<false>, dim3(PG_CTAS), PG_THREADS, 0, st, false, a);
    const dim3 grid(148 * 4);
    cudaError_t e = launch_behind(paged_clear_kernel, grid, WIDE_THREADS, 0, st, false, a);
    if (e == cudaSuccess) e = launch_behind(paged_mark_kernel, grid, WIDE_THREADS, 0, st, true, a);
    if (e == cudaSuccess) e = launch_behind(paged_compact_kernel<true>, dim3(PG_CTAS), PG_THREADS, 0, st, true, a);
    if (e == cudaSuccess) e = launch_behind(paged_rename_kernel, grid, WIDE_THREADS, 0, st, true, a);
    return e;
}
cudaError_t launch_paged_copy(const CopyArgs& a, cudaStream_t st) {
    return launch_behind(paged_copy_kernel, dim3(COPY_CTAS), COPY_THREADS, 0, st, true, a);
}

}  // namespace loma
