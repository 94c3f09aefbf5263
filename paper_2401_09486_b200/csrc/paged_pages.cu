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
#include <limits.h>

#include <algorithm>
#include <vector>

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
constexpr int PG_CTAS = 8, PG_THREADS = 1024, PG_WARPS = PG_THREADS / 32, PG_ALL = PG_CTAS * PG_THREADS;

// A CTA's part [lo, hi) of n things
struct Part {
    int64_t lo, hi;
    __device__ __forceinline__ Part(int64_t n, int rank) {
        const int64_t per = (n + PG_CTAS - 1) / PG_CTAS;
        lo = min(per * rank, n);
        hi = min(lo + per, n);
    }
};

// Exclusive sums over the block of one number per thread, and the block's total.  Ends with a barrier before the next use.
__device__ __forceinline__ int64_t block_sums(int64_t x, int64_t* total) {
    __shared__ int64_t s_warp[PG_WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
    }
    __syncthreads();
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < PG_WARPS; ++w) {
        const int64_t s = s_warp[w];
        before += w < warp ? s : 0;
        all += s;
    }
    *total = all;
    return before + incl - x;
}

// Each CTA's number to every CTA; returns the sum of the lower ranks' and, in *all, of everyone's.  slot: PG_CTAS int64 in shared
// memory, one set per exchange.  A barrier of the cluster.
__device__ __forceinline__ int64_t exchange(cg::cluster_group& cl, int64_t* slot, int64_t mine, int64_t* all) {
    const int rank = cl.block_rank();
    if (threadIdx.x < PG_CTAS) *cl.map_shared_rank(slot + rank, threadIdx.x) = mine;
    cl.sync();
    int64_t before = 0, sum = 0;
#pragma unroll
    for (int r = 0; r < PG_CTAS; ++r) {
        const int64_t s = slot[r];
        before += r < rank ? s : 0;
        sum += s;
    }
    *all = sum;
    return before;
}

constexpr int PG_RUN = 8;   // consecutive pages to a thread

// bit i: page first + i (below end) has a count below 0
__device__ __forceinline__ unsigned unowned(const PageList& pl, int64_t first, int64_t end) {
    unsigned bits = 0;
#pragma unroll
    for (int i = 0; i < PG_RUN; ++i)
        if (first + i < end && __ldcg(pl.refs + first + i) < 0) bits |= 1u << i;
    return bits;
}

// As host_settle, by all CTAs, after the counts are complete (a barrier of the cluster before); *taken becomes the list's new start.
// Another barrier makes the list visible.
__device__ __forceinline__ int64_t settle(cg::cluster_group& cl, const PageList& pl, int64_t* slot, int* taken, int64_t* lost) {
    const Part part(pl.n_pages, cl.block_rank());
    int64_t mine = 0, total = 0, all;
    for (int64_t p = part.lo + threadIdx.x * PG_RUN; p < part.hi; p += PG_THREADS * PG_RUN) mine += __popc(unowned(pl, p, part.hi));
    block_sums(mine, &total);
    int64_t at = exchange(cl, slot, total, &all);
    const int64_t n = min(all, (int64_t)*taken);
    if (total > 0)
        for (int64_t base = part.lo; base < part.hi; base += PG_THREADS * PG_RUN) {
            const int64_t p = base + threadIdx.x * PG_RUN;
            unsigned bits = unowned(pl, p, part.hi);
            int64_t here;
            int64_t i = at + block_sums(__popc(bits), &here);
            at += here;
            for (; bits; bits &= bits - 1, ++i) {
                const int64_t page = p + __ffs(bits) - 1;
                pl.refs[page] = 0;
                if (i < n) pl.free_pages[*taken - n + i] = (int)page;
            }
        }
    *lost = all - n;
    *taken -= (int)n;
    return all;
}

__global__ void __cluster_dims__(PG_CTAS, 1, 1) __launch_bounds__(PG_THREADS) paged_release_kernel(const ReleaseArgs a) {
    cg::cluster_group cl = cg::this_cluster();
    __shared__ int64_t slot[PG_CTAS];
    const int lane = threadIdx.x & 31, warps = PG_CTAS * PG_WARPS;
    const int first = (threadIdx.x >> 5) * PG_CTAS + cl.block_rank();   // a warp to a row, neighbours on different SMs
    int taken = start_of(a.pl, __ldcg(a.pl.taken));
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
        if (lane == 0) a.held_out[b] = kept;
    }
    cl.sync();
    int64_t lost;
    const int64_t freed = settle(cl, a.pl, slot, &taken, &lost);
    if (cl.block_rank() == 0 && threadIdx.x == 0) {
        *a.pl.taken = taken;
        a.counts[0] = 0;
        a.counts[1] = saturate(freed);
        a.counts[2] = saturate(lost);
        a.counts[3] = 0;
    }
}

__global__ void __cluster_dims__(PG_CTAS, 1, 1) __launch_bounds__(PG_THREADS) paged_fork_kernel(const ForkArgs a) {
    cg::cluster_group cl = cg::this_cluster();
    __shared__ int64_t slot[2][PG_CTAS];
    const int rank = cl.block_rank(), lane = threadIdx.x & 31, warps = PG_CTAS * PG_WARPS;
    const int first = (threadIdx.x >> 5) * PG_CTAS + rank;
    const int64_t me = (int64_t)rank * PG_THREADS + threadIdx.x;
    int32_t *kids = a.ws, *heir = a.ws + a.B;
    int taken = start_of(a.pl, __ldcg(a.pl.taken));
    for (int64_t b = me; b < a.B; b += PG_ALL) { kids[b] = 0; heir[b] = INT_MAX; }
    cl.sync();
    for (int64_t b = me; b < a.B; b += PG_ALL) {
        const int p = fork_from(a, (int)b);
        if (p < 0) continue;
        atomicAdd(kids + p, 1);
        atomicMin(heir + p, b == p ? -1 : (int)b);
    }
    cl.sync();
    // owners gained and lost
    for (int r = first; r < a.B; r += warps) {
        const Parent p = fork_parent(a, r);
        const int k = __ldcg(kids + r), n = k > 0 ? p.share : p.held;
        if (k == 1) continue;
        const int32_t* row = a.block_table + (int64_t)r * a.max_pages;
#pragma unroll 4
        for (int j = lane; j < n; j += 32) {
            const int page = __ldg(row + j);
            if (in_pool(a.pl, page)) atomicAdd(a.pl.refs + page, k - 1);
        }
    }
    // pages to draw: this CTA's rows, numbered from the first row of all on.  kids is done with: it takes the first number of a row
    // (within this CTA's part)
    const Part part(a.B, rank);
    cl.sync();
    int64_t need_before = 0;
    for (int64_t base = part.lo; base < part.hi; base += PG_THREADS) {
        const int64_t b = base + threadIdx.x;
        int need = 0;
        if (b < part.hi) {
            const int r = fork_from(a, (int)b);
            if (r >= 0 && __ldcg(heir + r) != (b == r ? -1 : (int)b)) {
                const Parent p = fork_parent(a, r);
                need = p.used > p.share ? p.used - p.share : 0;
            }
        }
        int64_t total;
        const int64_t at = need_before + block_sums(need, &total);
        if (b < part.hi) kids[b] = saturate(at);
        need_before += total;
    }
    int64_t drawn, lost;
    const int64_t draw0 = exchange(cl, slot[0], need_before, &drawn);
    const int64_t freed = settle(cl, a.pl, slot[1], &taken, &lost);
    cl.sync();
    const int64_t room = min((int64_t)a.pl.n_free - taken, (int64_t)a.max_copies), got = min(drawn, room);
    for (int64_t b = part.lo + (threadIdx.x >> 5); b < part.hi; b += PG_WARPS) {
        const int r = fork_from(a, (int)b);
        int32_t* out = a.table_out + b * a.max_pages;
        if (r < 0) {
            for (int j = lane; j < a.max_pages; j += 32) out[j] = -1;
            if (lane == 0) { a.lens_out[b] = -1; a.held_out[b] = 0; }
            continue;
        }
        const Parent p = fork_parent(a, r);
        const bool is_heir = __ldcg(heir + r) == (b == r ? -1 : (int)b);
        const int32_t* row = a.block_table + (int64_t)r * a.max_pages;
        const int named = is_heir ? p.held : p.share, used = is_heir ? p.held : p.used;
        const int64_t start = draw0 + kids[b];   // written by this CTA
#pragma unroll 4
        for (int j = lane; j < a.max_pages; j += 32) {
            int page = j < used ? __ldg(row + j) : -1;
            if (j >= named && j < used) {
                const int64_t i = start + j - named;
                const int from = page;
                page = -1;
                if (i < room) {
                    page = __ldcg(a.pl.free_pages + taken + i);
                    a.copy_src[i] = in_pool(a.pl, from) ? from : -1;
                    a.copy_dst[i] = page;
                }
            }
            out[j] = page;
        }
        if (lane == 0) {
            a.lens_out[b] = a.cache_lens[r];
            a.held_out[b] = named + (int)min(max(room - start, (int64_t)0), (int64_t)(used - named));
        }
    }
    for (int64_t i = got + me; i < a.max_copies; i += PG_ALL) a.copy_src[i] = a.copy_dst[i] = -1;
    if (rank == 0 && threadIdx.x == 0) {
        *a.pl.taken = (int)(taken + got);
        a.counts[0] = saturate(got);
        a.counts[1] = saturate(freed);
        a.counts[2] = saturate(lost);
        a.counts[3] = saturate(drawn - got);
    }
}

__global__ void __cluster_dims__(PG_CTAS, 1, 1) __launch_bounds__(PG_THREADS) paged_compact_kernel(const CompactArgs a) {
    cg::cluster_group cl = cg::this_cluster();
    __shared__ int64_t slot[3][PG_CTAS];
    const PageList& pl = a.pl;
    const int rank = cl.block_rank(), lane = threadIdx.x & 31, warps = PG_CTAS * PG_WARPS;
    const int first = (threadIdx.x >> 5) * PG_CTAS + rank;
    const int64_t me = (int64_t)rank * PG_THREADS + threadIdx.x;
    int32_t* state = a.page_map;   // bit 0: free, bit 1: named
    const int taken = start_of(pl, __ldcg(pl.taken));
    for (int64_t p = me; p < pl.n_pages; p += PG_ALL) state[p] = 0;
    cl.sync();
    for (int64_t i = taken + me; i < pl.n_free; i += PG_ALL) {
        const int p = pl.free_pages[i];
        if (in_pool(pl, p)) atomicOr(state + p, 1);
    }
    for (int b = first; b < a.B; b += warps) {
        const int h = clampi(__ldg(a.held + b), 0, a.max_pages);
#pragma unroll 4
        for (int j = lane; j < h; j += 32) {
            const int p = a.block_table[(int64_t)b * a.max_pages + j];
            if (in_pool(pl, p)) atomicOr(state + p, 2);
        }
    }
    cl.sync();
    // bits of PG_RUN pages: free ones in the low half, named ones in the high half
    const Part part(pl.n_pages, rank);
    auto run_of = [&](int64_t p) {
        unsigned bits = 0;
#pragma unroll
        for (int i = 0; i < PG_RUN; ++i)
            if (p + i < part.hi) {
                const int s = __ldcg(state + p + i);
                bits |= s & 2 ? 0x10000u << i : (unsigned)(s & 1) << i;
            }
        return bits;
    };
    int64_t mine_f = 0, mine_n = 0, tot_f, tot_n, all_f, all_n;
    for (int64_t p = part.lo + threadIdx.x * PG_RUN; p < part.hi; p += PG_THREADS * PG_RUN) {
        const unsigned bits = run_of(p);
        mine_f += __popc(bits & 0xffff);
        mine_n += __popc(bits >> 16);
    }
    block_sums(mine_f, &tot_f);
    block_sums(mine_n, &tot_n);
    if (threadIdx.x < PG_CTAS) *cl.map_shared_rank(&slot[0][rank], threadIdx.x) = tot_f;
    int64_t n0 = exchange(cl, slot[1], tot_n, &all_n), f0 = 0;
    all_f = 0;
    for (int r = 0; r < PG_CTAS; ++r) {
        f0 += r < rank ? slot[0][r] : 0;
        all_f += slot[0][r];
    }
    // Of the pages that are free or named the lowest all_n are to be the named ones.  Page p, with f free and n named ones before it, is
    // among them if f + n < all_n.  Named pages above move, in order, to the free ones below.
    int64_t above = 0, tot_above, moves;
    for (int64_t base = part.lo, f = f0, n = n0; base < part.hi; base += PG_THREADS * PG_RUN) {
        const int64_t p = base + threadIdx.x * PG_RUN;
        const unsigned bits = p < part.hi ? run_of(p) : 0;
        int64_t hf, hn;
        int64_t pf = f + block_sums(__popc(bits & 0xffff), &hf), pn = n + block_sums(__popc(bits >> 16), &hn);
        for (int i = 0; i < PG_RUN; ++i) {
            if (bits >> (16 + i) & 1) { above += pf + pn >= all_n; ++pn; }
            pf += bits >> i & 1;
        }
        f += hf;
        n += hn;
    }
    block_sums(above, &tot_above);
    exchange(cl, slot[2], tot_above, &moves);
    const int64_t count = min(moves, (int64_t)a.max_copies), stay = all_n - moves;   // named pages below: their ranks are 0 .. stay - 1
    for (int64_t base = part.lo, f = f0, n = n0; base < part.hi; base += PG_THREADS * PG_RUN) {
        const int64_t p = base + threadIdx.x * PG_RUN;
        const unsigned bits = p < part.hi ? run_of(p) : 0;
        int64_t hf, hn;
        int64_t pf = f + block_sums(__popc(bits & 0xffff), &hf), pn = n + block_sums(__popc(bits >> 16), &hn);
        for (int i = 0; i < PG_RUN && p + i < part.hi; ++i) {
            const int page = (int)(p + i);
            const bool is_free = bits >> i & 1, is_named = bits >> (16 + i) & 1;
            // of the free pages the first `count` become named (there are that many below), of the named ones those of rank stay ..
            // stay + count - 1 become free
            const bool to = is_free && pf < count, from = is_named && pn >= stay && pn - stay < count;
            if (to) a.copy_dst[pf] = page;
            if (from) a.copy_src[pn - stay] = page;
            if ((is_free && !to) || from)
                pl.free_pages[pl.n_free - all_f + pf - min(pf, count) + min(max(pn - stay, (int64_t)0), count)] = page;
            state[page] = page;
            pf += is_free;
            pn += is_named;
        }
        f += hf;
        n += hn;
    }
    cl.sync();
    for (int64_t i = me; i < a.max_copies; i += PG_ALL) {
        if (i < count) {
            const int s = __ldcg(a.copy_src + i), d = __ldcg(a.copy_dst + i);
            a.page_map[s] = d;
            pl.refs[d] = __ldcg(pl.refs + s);
            pl.refs[s] = 0;
        } else {
            a.copy_src[i] = a.copy_dst[i] = -1;
        }
    }
    cl.sync();
    if (count > 0)
        for (int b = first; b < a.B; b += warps) {
            const int h = clampi(__ldg(a.held + b), 0, a.max_pages);
            int32_t* row = a.block_table + (int64_t)b * a.max_pages;
#pragma unroll 4
            for (int j = lane; j < h; j += 32) {
                const int p = row[j];
                if (in_pool(pl, p)) row[j] = __ldcg(a.page_map + p);
            }
        }
    if (rank == 0 && threadIdx.x == 0) {
        *pl.taken = (int)(pl.n_free - all_f);
        a.counts[0] = saturate(count);
        a.counts[1] = saturate(all_f);
        a.counts[2] = saturate(all_n);
        a.counts[3] = saturate(moves - count);
    }
}

// Copying: a warp takes 4 KB of one page of one pool at a time, eight 16-byte loads per lane in flight, then as many stores.
constexpr int COPY_THREADS = 256, COPY_BYTES = 4096, COPY_CTAS = 148 * 6;

__global__ void __launch_bounds__(COPY_THREADS) paged_copy_kernel(const __grid_constant__ CopyArgs a) {
    const int lane = threadIdx.x & 31;
    const int64_t n = min(max(__ldg(a.n), 0), a.max_copies);
    int64_t per = 0;   // pieces of one page in all pools
    for (int k = 0; k < a.n_pools; ++k) per += (a.bytes[k] + COPY_BYTES - 1) / COPY_BYTES;
    const int64_t warps = (int64_t)gridDim.x * (COPY_THREADS / 32);
    for (int64_t u = (int64_t)(threadIdx.x >> 5) * gridDim.x + blockIdx.x; u < n * per; u += warps) {
        const int64_t i = u / per;
        int64_t piece = u - i * per;
        int k = 0;
        for (int64_t x; piece >= (x = (a.bytes[k] + COPY_BYTES - 1) / COPY_BYTES); ++k) piece -= x;
        const int s = __ldg(a.src + i), d = __ldg(a.dst + i);
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
template <typename A>
static cudaError_t launch_cluster(void (*kernel)(A), const A& a, cudaStream_t st) {
    kernel<<<PG_CTAS, PG_THREADS, 0, st>>>(a);
    count_launches(1);
    return cudaGetLastError();
}
cudaError_t launch_paged_release(const ReleaseArgs& a, cudaStream_t st) { return launch_cluster(paged_release_kernel, a, st); }
cudaError_t launch_paged_fork(const ForkArgs& a, cudaStream_t st) { return launch_cluster(paged_fork_kernel, a, st); }
cudaError_t launch_paged_compact(const CompactArgs& a, cudaStream_t st) { return launch_cluster(paged_compact_kernel, a, st); }
cudaError_t launch_paged_copy(const CopyArgs& a, cudaStream_t st) {
    paged_copy_kernel<<<COPY_CTAS, COPY_THREADS, 0, st>>>(a);
    count_launches(1);
    return cudaGetLastError();
}

}  // namespace loma
