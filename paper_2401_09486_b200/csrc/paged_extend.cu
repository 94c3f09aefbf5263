// Block tables and slot maps of a paged cache, built from request lengths (loma_paged_extend).
//
// For every sequence b of the batch, with ps entries to a page and M columns in the block table:
//     len = clamp(cache_lens[b], 0, M ps)      n = new_lens[b] (0 for an idle sequence)
//     h   = pages the table row already holds  f = max(0, ceil(min(len + n, M ps) / ps) - h) fresh ones, if n > 0
//     row_start, page_start = exclusive sums of n and f
// and for every packed row r = row_start[b] + i: entry e = len + i of its sequence, slot = page of block e / ps times
// ps plus e mod ps.  All of it is integer arithmetic on a few numbers per sequence, so a call is bound by the latency of
// its dependent steps (lengths -> sums -> pages -> slots) when the batch is small and by the three row outputs when
// many prompts arrive at once.
//
// Up to FUSED_MAX_B sequences one launch does everything: every CTA scans all sequences for itself in shared memory (12
// bytes a sequence out of L2) and then writes its own slab of rows and its own share of the sequences, so nothing waits for
// another CTA.  What a single-token step needs after the sums -- the page of each sequence's next entry and the head of the
// free list -- is fetched before them.  Longer batches, and calls that update `held` or `taken` in place (where one CTA's
// write would be another CTA's input), scan in one CTA and write rows in a second launch.
// Measured: 64 sequences with one token each 4.4 us, 1000 prompts with a million rows (11 MB written) 10.0 us; with held and taken
// updated in place 8.5 and 15.4 us.
#include <limits.h>

#include <algorithm>

#include "loma_internal.cuh"

namespace loma {

__host__ __device__ inline int clampi(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// What one sequence asks for.
struct SeqNeed {
    int len, n, h, fresh;
};

__host__ __device__ inline SeqNeed seq_need(const ExtendArgs& a, int given, int fresh, int held) {
    SeqNeed s;
    const int room = a.max_pages << a.log2_ps;
    s.len = clampi(given, 0, room);
    s.n = given < 0 ? 0 : clampi(fresh, 0, INT_MAX);
    const int mask = (1 << a.log2_ps) - 1;
    s.h = a.held ? clampi(held, 0, a.max_pages) : (int)(((int64_t)s.len + mask) >> a.log2_ps);
    const int64_t end = (int64_t)s.len + s.n < room ? (int64_t)s.len + s.n : room;
    const int want = (int)((end + mask) >> a.log2_ps);
    s.fresh = s.n > 0 && want > s.h ? want - s.h : 0;
    return s;
}

__host__ __device__ inline SeqNeed seq_need(const ExtendArgs& a, int b) {
    return seq_need(a, a.cache_lens[b], a.new_lens ? a.new_lens[b] : 1, a.held ? a.held[b] : 0);
}

__host__ __device__ inline int saturate(int64_t x) { return x > INT_MAX ? INT_MAX : (int)x; }

// the idx-th page of the free list, or -1 past its end
__host__ __device__ inline int free_page(const ExtendArgs& a, int64_t idx) {
    return idx < a.n_free ? a.free_pages[idx] : -1;
}

// pages sequence b gets of the `fresh` it asks for from index `first` of the free list on
__host__ __device__ inline int pages_got(const ExtendArgs& a, int first, int fresh) {
    const int left = a.n_free > first ? a.n_free - first : 0;
    return left < fresh ? left : fresh;
}

// the free list's new start: pages handed out are behind it, pages asked for past the list's end are not (the sequences ask
// again, and a longer list begins where this one ended)
__host__ __device__ inline int taken_after(const ExtendArgs& a, int before, int64_t end) {
    const int64_t drawn = end < a.n_free ? end : a.n_free;
    return drawn > before ? (int)drawn : before;
}

// slot of entry e of a sequence from its page, or -1
__host__ __device__ inline int slot_of(const ExtendArgs& a, int page, int64_t e) {
    const int mask = (1 << a.log2_ps) - 1;
    return page >= 0 && page <= ((INT_MAX - mask) >> a.log2_ps) ? (page << a.log2_ps) + (int)(e & mask) : -1;
}

// slot of entry len + i of sequence b; h, first: its pages before the call, its first fresh page
__host__ __device__ inline int row_slot(const ExtendArgs& a, int b, int i, int len, int h, int first) {
    const int64_t e = (int64_t)len + i;
    if (e >= ((int64_t)a.max_pages << a.log2_ps)) return -1;
    const int block = (int)(e >> a.log2_ps);
    return slot_of(a, block < h ? a.block_table[(int64_t)b * a.max_pages + block] : free_page(a, (int64_t)first + block - h), e);
}
__host__ __device__ inline int first_pos(const ExtendArgs& a, int b, int len) { return a.pos0 ? a.pos0[b] : len; }

// ------------------------------------------------------------------ host form
void host_paged_extend(const ExtendArgs& a) {
    const int before = a.taken ? clampi(*a.taken, 0, INT_MAX) : 0;
    int64_t rows = 0, pages = before;
    for (int b = 0; b < a.B; ++b) {
        const SeqNeed s = seq_need(a, b);
        const int first = saturate(pages), got = pages_got(a, first, s.fresh);
        a.row_start[b] = saturate(rows);
        a.page_start[b] = first;
        for (int i = 0; i < s.n && rows + i < a.max_rows; ++i) {
            const int64_t r = rows + i;
            a.slots[r] = row_slot(a, b, i, s.len, s.h, first);
            a.row_seq[r] = b;
            a.row_pos[r] = saturate((int64_t)first_pos(a, b, s.len) + i);
        }
        for (int i = 0; i < s.fresh; ++i)
            a.block_table[(int64_t)b * a.max_pages + s.h + i] = free_page(a, (int64_t)first + i);
        a.held_out[b] = s.h + got;
        rows += s.n;
        pages += s.fresh;
    }
    a.row_start[a.B] = saturate(rows);
    a.page_start[a.B] = saturate(pages);
    if (a.taken) *a.taken = taken_after(a, before, pages);
    for (int64_t r = rows; r < a.max_rows; ++r) {
        a.slots[r] = a.row_seq[r] = -1;
        a.row_pos[r] = 0;
    }
}

// ------------------------------------------------------------------ device form
constexpr int EXT_THREADS = 512;
constexpr int FUSED_MAX_B = 1536;    // six numbers per sequence in shared memory: 36 KB
constexpr int ROWS_PER_THREAD = 4;   // consecutive rows: one search, 16-byte stores

// Exclusive sums over the block of one (rows, pages) pair per thread; every thread gets the block's totals too.
__device__ __forceinline__ void block_scan2(int64_t& x, int64_t& y, int64_t& tx, int64_t& ty) {
    __shared__ int64_t wx[32], wy[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
    int64_t ix = x, iy = y;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t ux = __shfl_up_sync(0xffffffffu, ix, o), uy = __shfl_up_sync(0xffffffffu, iy, o);
        if (lane >= o) { ix += ux; iy += uy; }
    }
    if (lane == 31) { wx[warp] = ix; wy[warp] = iy; }
    __syncthreads();
    if (warp == 0) {
        int64_t vx = lane < nw ? wx[lane] : 0, vy = lane < nw ? wy[lane] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t ux = __shfl_up_sync(0xffffffffu, vx, o), uy = __shfl_up_sync(0xffffffffu, vy, o);
            if (lane >= o) { vx += ux; vy += uy; }
        }
        wx[lane] = vx; wy[lane] = vy;
    }
    __syncthreads();
    tx = wx[nw - 1]; ty = wy[nw - 1];
    x = ix - x + (warp ? wx[warp - 1] : 0);
    y = iy - y + (warp ? wy[warp - 1] : 0);
}

// last b in [lo, hi) with start[b] <= r (start is non-decreasing, start[lo] <= r): sequences without rows are passed over
__device__ __forceinline__ int find_seq(const int* start, int lo, int hi, int r) {
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (start[mid] <= r) lo = mid; else hi = mid;
    }
    return lo;
}

// Rows r0 .. r0+3 of the packed batch; start: row_start (B + 1 values).  enter(b) makes b the current sequence, slot(i) and
// pos(i) are those of its i-th new entry.
template <typename Enter, typename Slot, typename Pos>
__device__ __forceinline__ void write_rows(const ExtendArgs& a, const int* start, int r0, bool vec, Enter&& enter, Slot&& slot_at, Pos&& pos_at) {
    int slot[ROWS_PER_THREAD], seq[ROWS_PER_THREAD], pos[ROWS_PER_THREAD];
    const int total = start[a.B];
    int b = r0 < total ? find_seq(start, 0, a.B, r0) : a.B, have = -1;
    bool done = false;
    if (r0 < total && start[b + 1] - r0 >= ROWS_PER_THREAD) {   // the usual case of a prompt: one sequence, and one page
        enter(b);
        have = b;
        const int i = r0 - start[b], s0 = slot_at(i), p0 = pos_at(i);
        const int mask = (1 << a.log2_ps) - 1;
        done = s0 >= 0 && (s0 & mask) + ROWS_PER_THREAD - 1 <= mask && p0 <= INT_MAX - ROWS_PER_THREAD;
        if (done) {
#pragma unroll
            for (int u = 0; u < ROWS_PER_THREAD; ++u) { slot[u] = s0 + u; seq[u] = b; pos[u] = p0 + u; }
        }
    }
    if (!done)
#pragma unroll
    for (int u = 0; u < ROWS_PER_THREAD; ++u) {
        const int r = r0 + u;
        slot[u] = -1; seq[u] = -1; pos[u] = 0;
        if (r >= total || r < 0) continue;
        while (start[b + 1] <= r) ++b;
        if (b != have) { enter(b); have = b; }
        slot[u] = slot_at(r - start[b]);
        pos[u] = pos_at(r - start[b]);
        seq[u] = b;
    }
    if (vec && r0 + ROWS_PER_THREAD <= a.max_rows) {
        *reinterpret_cast<int4*>(a.slots + r0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
        *reinterpret_cast<int4*>(a.row_seq + r0) = make_int4(seq[0], seq[1], seq[2], seq[3]);
        *reinterpret_cast<int4*>(a.row_pos + r0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
    } else {
#pragma unroll
        for (int u = 0; u < ROWS_PER_THREAD; ++u)
            if (r0 + u < a.max_rows) {
                a.slots[r0 + u] = slot[u];
                a.row_seq[r0 + u] = seq[u];
                a.row_pos[r0 + u] = pos[u];
            }
    }
}

__global__ void __launch_bounds__(EXT_THREADS)
paged_extend_fused_kernel(const ExtendArgs a, int vec) {
    __shared__ int s_row[FUSED_MAX_B + 1], s_page[FUSED_MAX_B + 1], s_len[FUSED_MAX_B], s_h[FUSED_MAX_B], s_pos[FUSED_MAX_B];
    __shared__ int s_next[FUSED_MAX_B], s_free[EXT_THREADS];   // page of a sequence's entry len; head of the free list
    const int tid = threadIdx.x, room = a.max_pages << a.log2_ps;
    // a thread's sequences are neighbours: up to PER of them, all their numbers in flight at once
    constexpr int PER = FUSED_MAX_B / EXT_THREADS;
    const int per = (a.B + EXT_THREADS - 1) / EXT_THREADS, b0 = tid * per;
    int lens[PER], news[PER], helds[PER], pos0s[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const bool in = u < per && b0 + u < a.B;
        lens[u] = in ? __ldg(a.cache_lens + b0 + u) : -1;
        news[u] = in && a.new_lens ? __ldg(a.new_lens + b0 + u) : 1;
        helds[u] = in && a.held ? __ldg(a.held + b0 + u) : 0;
        pos0s[u] = in && a.pos0 ? __ldg(a.pos0 + b0 + u) : 0;
    }
    const int head = tid < a.n_free ? __ldg(a.free_pages + tid) : -1;
    SeqNeed need[PER];
    int next[PER];
    int64_t rows = 0, pages = 0, tr, tp;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        need[u] = seq_need(a, lens[u], news[u], helds[u]);
        next[u] = -1;
        if (u < per && b0 + u < a.B) {
            const int len = need[u].len;
            if (len < room && (len >> a.log2_ps) < need[u].h) next[u] = a.block_table[(int64_t)(b0 + u) * a.max_pages + (len >> a.log2_ps)];
            rows += need[u].n;
            pages += need[u].fresh;
        }
    }
    block_scan2(rows, pages, tr, tp);
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int b = b0 + u;
        if (u < per && b < a.B) {
            s_row[b] = saturate(rows);
            s_page[b] = saturate(pages);
            s_len[b] = need[u].len;
            s_h[b] = need[u].h;
            s_pos[b] = a.pos0 ? pos0s[u] : need[u].len;
            s_next[b] = next[u];
            rows += need[u].n;
            pages += need[u].fresh;
        }
    }
    if (tid == 0) { s_row[a.B] = saturate(tr); s_page[a.B] = saturate(tp); }
    s_free[tid] = head;
    __syncthreads();
    auto free_at = [&](int64_t idx) { return idx < EXT_THREADS ? s_free[idx] : free_page(a, idx); };

    // this CTA's share of the sequences: sums and held pages, then the fresh table entries (a warp per sequence)
    for (int b = blockIdx.x * EXT_THREADS + tid; b <= a.B; b += gridDim.x * EXT_THREADS) {
        a.row_start[b] = s_row[b];
        a.page_start[b] = s_page[b];
        if (b < a.B) a.held_out[b] = s_h[b] + pages_got(a, s_page[b], s_page[b + 1] - s_page[b]);
    }
    const int64_t step = (int64_t)gridDim.x * EXT_THREADS * ROWS_PER_THREAD;
    for (int64_t r = ((int64_t)blockIdx.x * EXT_THREADS + tid) * ROWS_PER_THREAD; r < a.max_rows; r += step) {
        int cur = 0, len = 0, h = 0, first = 0, pos = 0, block = -1, page = -1;
        write_rows(a, s_row, (int)r, vec,
                   [&](int b) { cur = b; len = s_len[b]; h = s_h[b]; first = s_page[b]; pos = s_pos[b]; block = -1; },
                   [&](int i) {
                       const int64_t e = (int64_t)len + i;
                       if (e >= room) return -1;
                       const int blk = (int)(e >> a.log2_ps);
                       if (blk != block) {   // rows of one page look it up once
                           block = blk;
                           if (blk >= h) page = free_at((int64_t)first + blk - h);
                           else if (blk == len >> a.log2_ps) page = s_next[cur];
                           else page = a.block_table[(int64_t)cur * a.max_pages + blk];
                       }
                       return slot_of(a, page, e);
                   },
                   [&](int i) { return saturate((int64_t)pos + i); });
    }
    const int lane = tid & 31;
    for (int b = blockIdx.x * (EXT_THREADS / 32) + (tid >> 5); b < a.B; b += gridDim.x * (EXT_THREADS / 32)) {
        const int fresh = s_page[b + 1] - s_page[b];
        for (int i = lane; i < fresh; i += 32) a.block_table[(int64_t)b * a.max_pages + s_h[b] + i] = free_at((int64_t)s_page[b] + i);
    }
}

// One CTA: the sums, held pages and the free list's new start.  Every value a thread reads of `held` it reads before it
// writes held_out, and no other thread reads that entry, so the two may be one array.
constexpr int SCAN_THREADS = 1024, SCAN_AT_ONCE = 4;
__global__ void __launch_bounds__(SCAN_THREADS)
paged_extend_scan_kernel(const ExtendArgs a) {
    // SCAN_THREADS * SCAN_AT_ONCE neighbouring sequences at a time
    __shared__ int s_taken;
    let_next_start();
    if (threadIdx.x == 0) s_taken = a.taken ? clampi(*a.taken, 0, INT_MAX) : 0;
    __syncthreads();
    int64_t rows0 = 0, pages0 = s_taken;
    for (int64_t base = 0; base < a.B; base += SCAN_THREADS * SCAN_AT_ONCE) {
        const int64_t b0 = base + (int64_t)threadIdx.x * SCAN_AT_ONCE;
        int lens[SCAN_AT_ONCE], news[SCAN_AT_ONCE], helds[SCAN_AT_ONCE];
#pragma unroll
        for (int u = 0; u < SCAN_AT_ONCE; ++u) {
            const bool in = b0 + u < a.B;
            lens[u] = in ? a.cache_lens[b0 + u] : -1;
            news[u] = in && a.new_lens ? a.new_lens[b0 + u] : 1;
            helds[u] = in && a.held ? a.held[b0 + u] : 0;
        }
        SeqNeed need[SCAN_AT_ONCE];
        int64_t rows = 0, pages = 0, tr, tp;
#pragma unroll
        for (int u = 0; u < SCAN_AT_ONCE; ++u) {
            need[u] = seq_need(a, lens[u], news[u], helds[u]);
            rows += need[u].n;
            pages += need[u].fresh;
        }
        block_scan2(rows, pages, tr, tp);
        rows += rows0;
        pages += pages0;
#pragma unroll
        for (int u = 0; u < SCAN_AT_ONCE; ++u)
            if (b0 + u < a.B) {
                const int first = saturate(pages);
                a.row_start[b0 + u] = saturate(rows);
                a.page_start[b0 + u] = first;
                a.held_out[b0 + u] = need[u].h + pages_got(a, first, need[u].fresh);
                rows += need[u].n;
                pages += need[u].fresh;
            }
        rows0 += tr;
        pages0 += tp;
        __syncthreads();   // the scan's shared sums are used again
    }
    if (threadIdx.x == 0) {
        a.row_start[a.B] = saturate(rows0);
        a.page_start[a.B] = saturate(pages0);
        if (a.taken) *a.taken = taken_after(a, s_taken, pages0);
    }
}

__global__ void __launch_bounds__(EXT_THREADS)
paged_extend_rows_kernel(const ExtendArgs a, int vec) {
    wait_for_previous();   // launched while the scan runs
    const int lane = threadIdx.x & 31;
    for (int64_t b = (int64_t)blockIdx.x * (EXT_THREADS / 32) + (threadIdx.x >> 5); b < a.B;
         b += (int64_t)gridDim.x * (EXT_THREADS / 32)) {
        const int first = a.page_start[b], fresh = a.page_start[b + 1] - first;
        const int h = a.held_out[b] - pages_got(a, first, fresh);
        for (int i = lane; i < fresh; i += 32) a.block_table[b * a.max_pages + h + i] = free_page(a, (int64_t)first + i);
    }
    const int64_t step = (int64_t)gridDim.x * EXT_THREADS * ROWS_PER_THREAD;
    for (int64_t r = ((int64_t)blockIdx.x * EXT_THREADS + threadIdx.x) * ROWS_PER_THREAD; r < a.max_rows; r += step)
    {
        int cur = 0, len = 0, h = 0, first = 0;
        write_rows(a, a.row_start, (int)r, vec,
                   [&](int b) {   // `held` may have been updated in place: a sequence's pages before the call are what it holds now less what it got
                       cur = b;
                       len = clampi(a.cache_lens[b], 0, a.max_pages << a.log2_ps);
                       first = a.page_start[b];
                       h = a.held_out[b] - pages_got(a, first, a.page_start[b + 1] - first);
                   },
                   [&](int i) { return row_slot(a, cur, i, len, h, first); },
                   [&](int i) { return saturate((int64_t)first_pos(a, cur, len) + i); });
    }
}

cudaError_t launch_paged_extend(const ExtendArgs& a, cudaStream_t st) {
    const int vec = (((uintptr_t)a.slots | (uintptr_t)a.row_seq | (uintptr_t)a.row_pos) & 15u) == 0;
    const int64_t row_ctas = ((int64_t)a.max_rows + EXT_THREADS * ROWS_PER_THREAD - 1) / (EXT_THREADS * ROWS_PER_THREAD);
    const int64_t seq_ctas = ((int64_t)a.B + EXT_THREADS / 32 - 1) / (EXT_THREADS / 32);
    // every CTA repeats the scan: two per SM at most (1000 prompts, a million rows: 148 CTAs 11.3 us, 296 10.1, 592 11.1)
    const int grid = (int)std::max<int64_t>(1, std::min<int64_t>(296, std::max(row_ctas, seq_ctas)));
    if (a.B <= FUSED_MAX_B && a.held != a.held_out && !a.taken) {
        paged_extend_fused_kernel<<<grid, EXT_THREADS, 0, st>>>(a, vec);
        count_launches(1);
        return cudaGetLastError();
    }
    paged_extend_scan_kernel<<<1, SCAN_THREADS, 0, st>>>(a);
    count_launches(1);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_behind(paged_extend_rows_kernel, dim3(grid), EXT_THREADS, 0, st, true, a, vec);
}

}  // namespace loma
