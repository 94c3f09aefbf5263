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
// Up to FUSED_MAX_B sequences one launch does everything: every CTA scans all sequences for itself in shared memory
// (12 bytes a sequence out of L2, two or three microseconds at 4096) and then writes its own slab of rows and its own
// share of the sequences, so nothing waits for another CTA.  Longer batches, and calls that update `held` or `taken`
// in place (where one CTA's write would be another CTA's input), scan in one CTA and write rows in a second launch.
#include <limits.h>

#include <algorithm>

#include "loma_internal.cuh"

namespace loma {

__host__ __device__ inline int clampi(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }

// What one sequence asks for.
struct SeqNeed {
    int len, n, h, fresh;
};

__host__ __device__ inline SeqNeed seq_need(const ExtendArgs& a, int b) {
    SeqNeed s;
    const int room = a.max_pages << a.log2_ps;
    const int given = a.cache_lens[b];
    s.len = clampi(given, 0, room);
    s.n = given < 0 ? 0 : (a.new_lens ? clampi(a.new_lens[b], 0, INT_MAX) : 1);
    const int mask = (1 << a.log2_ps) - 1;
    s.h = a.held ? clampi(a.held[b], 0, a.max_pages) : (int)(((int64_t)s.len + mask) >> a.log2_ps);
    const int64_t end = (int64_t)s.len + s.n < room ? (int64_t)s.len + s.n : room;
    const int want = (int)((end + mask) >> a.log2_ps);
    s.fresh = s.n > 0 && want > s.h ? want - s.h : 0;
    return s;
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

// slot and position of entry len + i of sequence b; h, first: its pages before the call, its first fresh page
__host__ __device__ inline void row_values(const ExtendArgs& a, int b, int i, int len, int h, int first, int& slot, int& pos) {
    const int64_t e = (int64_t)len + i;
    const int64_t p = (a.pos0 ? (int64_t)a.pos0[b] : (int64_t)len) + i;
    pos = saturate(p);
    slot = -1;
    if (e < ((int64_t)a.max_pages << a.log2_ps)) {
        const int block = (int)(e >> a.log2_ps);
        const int page = block < h ? a.block_table[(int64_t)b * a.max_pages + block] : free_page(a, (int64_t)first + block - h);
        const int mask = (1 << a.log2_ps) - 1;
        if (page >= 0 && page <= ((INT_MAX - mask) >> a.log2_ps)) slot = (page << a.log2_ps) + (int)(e & mask);
    }
}

// ------------------------------------------------------------------ host form
void host_paged_extend(const ExtendArgs& a) {
    int64_t rows = 0, pages = a.taken ? clampi(*a.taken, 0, INT_MAX) : 0;
    for (int b = 0; b < a.B; ++b) {
        const SeqNeed s = seq_need(a, b);
        const int first = saturate(pages), got = pages_got(a, first, s.fresh);
        a.row_start[b] = saturate(rows);
        a.page_start[b] = first;
        for (int i = 0; i < s.n && rows + i < a.max_rows; ++i) {
            const int64_t r = rows + i;
            row_values(a, b, i, s.len, s.h, first, a.slots[r], a.row_pos[r]);
            a.row_seq[r] = b;
        }
        for (int i = 0; i < s.fresh; ++i)
            a.block_table[(int64_t)b * a.max_pages + s.h + i] = free_page(a, (int64_t)first + i);
        a.held_out[b] = s.h + got;
        rows += s.n;
        pages += s.fresh;
    }
    a.row_start[a.B] = saturate(rows);
    a.page_start[a.B] = saturate(pages);
    if (a.taken) *a.taken = saturate(pages);
    for (int64_t r = rows; r < a.max_rows; ++r) {
        a.slots[r] = a.row_seq[r] = -1;
        a.row_pos[r] = 0;
    }
}

// ------------------------------------------------------------------ device form
constexpr int EXT_THREADS = 512;
constexpr int FUSED_MAX_B = 4096;    // two int32 sums per sequence in shared memory: 32 KB
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

// Rows r0 .. r0+3 of the packed batch.  start / first: row_start and page_start (B + 1 values, shared or global memory).
// h_from_out: `held` is being updated in place, so a sequence's pages before the call are what it holds now less what it got.
__device__ __forceinline__ void write_rows(const ExtendArgs& a, const int* start, const int* first, int r0, bool vec, bool h_from_out) {
    int slot[ROWS_PER_THREAD], seq[ROWS_PER_THREAD], pos[ROWS_PER_THREAD];
    const int total = start[a.B];
    int b = r0 < total ? find_seq(start, 0, a.B, r0) : a.B;
    int len = 0, h = 0, have = -1;
#pragma unroll
    for (int u = 0; u < ROWS_PER_THREAD; ++u) {
        const int r = r0 + u;
        slot[u] = -1; seq[u] = -1; pos[u] = 0;
        if (r >= total || r < 0) continue;
        while (start[b + 1] <= r) ++b;
        if (b != have) {
            if (h_from_out) {
                const int room = a.max_pages << a.log2_ps;
                len = clampi(a.cache_lens[b], 0, room);
                h = a.held_out[b] - pages_got(a, first[b], first[b + 1] - first[b]);
            } else {
                const SeqNeed s = seq_need(a, b);
                len = s.len; h = s.h;
            }
            have = b;
        }
        row_values(a, b, r - start[b], len, h, first[b], slot[u], pos[u]);
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
    __shared__ int s_row[FUSED_MAX_B + 1], s_page[FUSED_MAX_B + 1];
    for (int b = threadIdx.x; b < a.B; b += EXT_THREADS) {
        const SeqNeed s = seq_need(a, b);
        s_row[b] = s.n;
        s_page[b] = s.fresh;
    }
    __syncthreads();
    const int per = (a.B + EXT_THREADS - 1) / EXT_THREADS;
    const int b0 = min(a.B, (int)threadIdx.x * per), b1 = min(a.B, b0 + per);
    int64_t rows = 0, pages = 0, tr, tp;
    for (int b = b0; b < b1; ++b) { rows += s_row[b]; pages += s_page[b]; }
    block_scan2(rows, pages, tr, tp);
    for (int b = b0; b < b1; ++b) {
        const int n = s_row[b], f = s_page[b];
        s_row[b] = saturate(rows);
        s_page[b] = saturate(pages);
        rows += n;
        pages += f;
    }
    if (threadIdx.x == 0) { s_row[a.B] = saturate(tr); s_page[a.B] = saturate(tp); }
    __syncthreads();

    // this CTA's share of the sequences: sums, held pages, fresh table entries (a warp per sequence)
    for (int b = blockIdx.x * EXT_THREADS + threadIdx.x; b <= a.B; b += gridDim.x * EXT_THREADS) {
        a.row_start[b] = s_row[b];
        a.page_start[b] = s_page[b];
        if (b < a.B) {
            const SeqNeed s = seq_need(a, b);
            a.held_out[b] = s.h + pages_got(a, s_page[b], s.fresh);
        }
    }
    const int lane = threadIdx.x & 31;
    for (int b = blockIdx.x * (EXT_THREADS / 32) + (threadIdx.x >> 5); b < a.B; b += gridDim.x * (EXT_THREADS / 32)) {
        const SeqNeed s = seq_need(a, b);
        for (int i = lane; i < s.fresh; i += 32)
            a.block_table[(int64_t)b * a.max_pages + s.h + i] = free_page(a, (int64_t)s_page[b] + i);
    }
    const int64_t step = (int64_t)gridDim.x * EXT_THREADS * ROWS_PER_THREAD;
    for (int64_t r = ((int64_t)blockIdx.x * EXT_THREADS + threadIdx.x) * ROWS_PER_THREAD; r < a.max_rows; r += step)
        write_rows(a, s_row, s_page, (int)r, vec, false);
}

// One CTA: the sums, held pages and the free list's new start.  Every value a thread reads of `held` it reads before it
// writes held_out, and no other thread reads that entry, so the two may be one array.
constexpr int SCAN_THREADS = 1024;
__global__ void __launch_bounds__(SCAN_THREADS)
paged_extend_scan_kernel(const ExtendArgs a) {
    const int per = (a.B + SCAN_THREADS - 1) / SCAN_THREADS;
    const int b0 = min((int64_t)a.B, (int64_t)threadIdx.x * per), b1 = min((int64_t)a.B, (int64_t)b0 + per);
    int64_t rows = 0, pages = 0, tr, tp;
    for (int b = b0; b < b1; ++b) {
        const SeqNeed s = seq_need(a, b);
        rows += s.n;
        pages += s.fresh;
    }
    const int64_t base = a.taken ? clampi(*a.taken, 0, INT_MAX) : 0;
    block_scan2(rows, pages, tr, tp);   // its barriers also order every read of *taken before the write below
    pages += base;
    for (int b = b0; b < b1; ++b) {
        const SeqNeed s = seq_need(a, b);
        const int first = saturate(pages);
        a.row_start[b] = saturate(rows);
        a.page_start[b] = first;
        a.held_out[b] = s.h + pages_got(a, first, s.fresh);
        rows += s.n;
        pages += s.fresh;
    }
    if (threadIdx.x == 0) {
        a.row_start[a.B] = saturate(tr);
        a.page_start[a.B] = saturate(base + tp);
        if (a.taken) *a.taken = saturate(base + tp);
    }
}

__global__ void __launch_bounds__(EXT_THREADS)
paged_extend_rows_kernel(const ExtendArgs a, int vec) {
    const int lane = threadIdx.x & 31;
    for (int64_t b = (int64_t)blockIdx.x * (EXT_THREADS / 32) + (threadIdx.x >> 5); b < a.B;
         b += (int64_t)gridDim.x * (EXT_THREADS / 32)) {
        const int first = a.page_start[b], fresh = a.page_start[b + 1] - first;
        const int h = a.held_out[b] - pages_got(a, first, fresh);
        for (int i = lane; i < fresh; i += 32) a.block_table[b * a.max_pages + h + i] = free_page(a, (int64_t)first + i);
    }
    const int64_t step = (int64_t)gridDim.x * EXT_THREADS * ROWS_PER_THREAD;
    for (int64_t r = ((int64_t)blockIdx.x * EXT_THREADS + threadIdx.x) * ROWS_PER_THREAD; r < a.max_rows; r += step)
        write_rows(a, a.row_start, a.page_start, (int)r, vec, true);
}

cudaError_t launch_paged_extend(const ExtendArgs& a, cudaStream_t st) {
    const int vec = (((uintptr_t)a.slots | (uintptr_t)a.row_seq | (uintptr_t)a.row_pos) & 15u) == 0;
    const int64_t row_ctas = ((int64_t)a.max_rows + EXT_THREADS * ROWS_PER_THREAD - 1) / (EXT_THREADS * ROWS_PER_THREAD);
    const int64_t seq_ctas = ((int64_t)a.B + EXT_THREADS / 32 - 1) / (EXT_THREADS / 32);
    // two CTAs of 512 threads per SM hide the page loads of the rows; more would repeat the scan for nothing
    const int grid = (int)std::max<int64_t>(1, std::min<int64_t>(148 * 2, std::max(row_ctas, seq_ctas)));
    if (a.B <= FUSED_MAX_B && a.held != a.held_out && !a.taken) {
        paged_extend_fused_kernel<<<grid, EXT_THREADS, 0, st>>>(a, vec);
        count_launches(1);
        return cudaGetLastError();
    }
    paged_extend_scan_kernel<<<1, SCAN_THREADS, 0, st>>>(a);
    count_launches(1);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    paged_extend_rows_kernel<<<grid, EXT_THREADS, 0, st>>>(a, vec);
    count_launches(1);
    return cudaGetLastError();
}

}  // namespace loma
