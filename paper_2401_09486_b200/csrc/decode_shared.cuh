// What the kernels of the shared-prefix decode step have in common: how the work is cut and where partial results lie.
#pragma once

#include <algorithm>

#include "loma_internal.cuh"

namespace loma {

constexpr int SHP_ROWS = 128;   // query rows of a prefix tile
constexpr int SHP_CTAS = 148;   // prefix CTAs a call is cut into where its keys allow it

// The cut of a call.  Depends on the sizes alone, so results repeat and the workspace can be sized before the call.
//
// Prefix: tiles of SHP_ROWS query rows times key ranges of equal length.
//
// Own caches: lengths are known on the device only and may be anything from nothing to max_len, so the work is cut there:
// a sequence of n keys is ceil(n / 16) blocks, the blocks of all (kv head, head tile, sequence) are numbered through, and
// worker w of W takes blocks [T w / W, T (w + 1) / W): equal shares whatever the lengths.  A worker's stay in one (kv head,
// head tile, sequence) is a segment with one partial result; segment w + index of that triple is a slot of its own, since
// along the numbering either the worker or the triple moves on.
struct SharedPlan {
    int m_tiles;      // prefix: tiles of SHP_ROWS query rows per kv head
    int p_splits;     // prefix: key ranges (0: no prefix)
    int p_len;        //         keys per range, a multiple of 128
    int g_rows;       // own: query heads of a kv head per head tile (8 or 16 rows of a warp-level product, or fewer heads)
    int g_tiles;      //      head tiles per kv head
    int workers;      //      W, before it is cut down to the number of blocks
    // partial results in the workspace, as offsets in floats.  Prefix tile (split, kv head, tile): outputs [D/4][128][4]
    // (so that a warp whose lanes are rows stores 512 contiguous bytes) and 128 log2-sum-exps.  Own segment: outputs
    // [g_rows][D] and g_rows log2-sum-exps.  cum: int64 [B + 1], blocks before sequence b within one (kv head, head tile).
    int64_t p_o, p_lse, own_o, own_lse, cum, total;
};

constexpr int OWN_KEYS = 16;                  // keys per block
constexpr int OWN_WARPS = 4;                  // a worker is a warp
constexpr int OWN_CTAS = 148, STREAM_CTAS = 4 * 148;

__host__ __device__ inline int64_t own_blocks(int len) { return len < 0 ? 0 : len / OWN_KEYS + 1; }   // keys 0 .. len: len is the new token

// the worker that block t of T belongs to, and the first block of worker w (W <= T)
__host__ __device__ inline int64_t own_worker(int64_t t, int64_t T, int64_t W) { return ((t + 1) * W - 1) / T; }
__host__ __device__ inline int64_t own_first(int64_t w, int64_t T, int64_t W) { return T / W * w + T % W * w / W; }

// cuda_cores: the own part runs on shared_own_stream_kernel (fp32, small pages, second opinion)
inline SharedPlan make_shared_plan(int B, int Hq, int Hkv, int D, int prefix_len, bool cuda_cores) {
    SharedPlan p;
    const int64_t g = Hq / Hkv, rows = (int64_t)B * g;
    p.m_tiles = (int)((rows + SHP_ROWS - 1) / SHP_ROWS);
    p.p_splits = 0;
    p.p_len = 128;
    if (prefix_len > 0) {
        // one CTA per SM (the other half of the SM works on the own caches); a range is never shorter than 128 keys
        const int64_t tiles = (int64_t)p.m_tiles * Hkv, key_tiles = (prefix_len + 127) / 128;
        int64_t splits = std::max<int64_t>(1, SHP_CTAS / tiles);
        splits = std::min<int64_t>(std::min<int64_t>(splits, key_tiles), 64);
        const int64_t per = (key_tiles + splits - 1) / splits;
        p.p_len = (int)per * 128;
        p.p_splits = (int)((key_tiles + per - 1) / per);
    }
    p.g_rows = cuda_cores ? (g < 3 ? (int)g : 4) : (g <= 8 ? (int)g : 16);
    p.g_tiles = (int)((g + p.g_rows - 1) / p.g_rows);
    p.workers = (cuda_cores ? STREAM_CTAS : OWN_CTAS) * OWN_WARPS;
    int64_t at = 0;
    auto take = [&](int64_t n) { const int64_t o = at; at += (n + 63) / 64 * 64; return o; };
    const int64_t p_tiles = (int64_t)p.p_splits * Hkv * p.m_tiles, segments = p.workers + (int64_t)B * Hkv * p.g_tiles;
    p.p_o = take(p_tiles * SHP_ROWS * D);
    p.p_lse = take(p_tiles * SHP_ROWS);
    p.own_o = take(segments * p.g_rows * D);
    p.own_lse = take(segments * p.g_rows);
    p.cum = take(2 * ((int64_t)B + 1));
    p.total = at;
    return p;
}

#ifdef __CUDACC__
// row of own entry j of (b, h), in rows of D elements from the start of the cache or pool
__device__ __forceinline__ int64_t own_row(const SharedArgs& a, int b, int h, int j) {
    if (!a.pg.table) return ((int64_t)b * a.Hkv + h) * a.cap + j;
    const int page = min(max(__ldg(a.pg.table + (int64_t)b * a.pg.max_pages + (j >> a.pg.log2_ps)), 0), a.pg.n_pages - 1);
    return ((((int64_t)page * a.Hkv + h) << a.pg.log2_ps) + (j & ((1 << a.pg.log2_ps) - 1)));
}

// The numbering of the own blocks, found again by every CTA from the lengths (B of them, out of L2 once per CTA).
struct SeqBlocks {
    static constexpr int MAX_GROUPS = 512;
    struct Cursor {
        int hh, b, blk, len;   // kv head * g_tiles + head tile, sequence, block, the sequence's length
    };
    const SharedArgs& a;

    __device__ __forceinline__ int len(int b) const { return min(__ldg(a.cache_lens + b), a.max_len); }

    // s[i]: blocks before sequence i * per of one (kv head, head tile), i = 0 .. groups; returns per.  out: all B + 1 sums,
    // stored for the merge kernel (or NULL).  Called by all threads of a block of WARPS warps; ends with a barrier.
    template <int WARPS>
    __device__ __forceinline__ int scan(int64_t* s, int64_t* wsum, int64_t* out) const {
        constexpr int THREADS = WARPS * 32, PER_THREAD = MAX_GROUPS / THREADS;
        const int per = (a.B + MAX_GROUPS - 1) / MAX_GROUPS, groups = (a.B + per - 1) / per;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        int64_t mine[PER_THREAD], sum = 0;
#pragma unroll
        for (int u = 0; u < PER_THREAD; ++u) {
            const int i = threadIdx.x * PER_THREAD + u;
            mine[u] = 0;
            for (int b = i * per; b < min(a.B, (i + 1) * per); ++b) mine[u] += own_blocks(len(b));
            sum += mine[u];
        }
        int64_t incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        if (lane == 31) wsum[warp] = incl;
        __syncthreads();
        int64_t at = incl - sum;
        for (int x = 0; x < warp; ++x) at += wsum[x];
#pragma unroll
        for (int u = 0; u < PER_THREAD; ++u) {
            const int i = threadIdx.x * PER_THREAD + u;
            if (i <= groups) s[i] = at;
            if (out) {
                int64_t c = at;
                for (int b = i * per; b < min(a.B, (i + 1) * per); ++b) {
                    out[b] = c;
                    c += own_blocks(len(b));
                }
                if (i == groups - 1) out[a.B] = c;
            }
            at += mine[u];
        }
        if (threadIdx.x == THREADS - 1 && groups == MAX_GROUPS) s[MAX_GROUPS] = at;
        __syncthreads();
        return per;
    }

    __device__ __forceinline__ Cursor find(int64_t t, const int64_t* s, int per) const {
        const int groups = (a.B + per - 1) / per;
        Cursor c;
        c.hh = (int)(t / s[groups]);
        int64_t rem = t - c.hh * s[groups];
        int lo = 0, hi = groups;   // s[lo] <= rem < s[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s[mid] <= rem) lo = mid; else hi = mid;
        }
        rem -= s[lo];
        c.b = lo * per;
        for (;; ++c.b) {
            c.len = len(c.b);
            const int64_t n = own_blocks(c.len);
            if (rem < n) break;
            rem -= n;
        }
        c.blk = (int)rem;
        return c;
    }

    // the next block; there has to be one.  Returns whether it belongs to another sequence or head
    __device__ __forceinline__ bool advance(Cursor& c) const {
        if ((c.blk + 1) * OWN_KEYS <= c.len) {
            ++c.blk;
            return false;
        }
        c.blk = 0;
        do {
            if (++c.b == a.B) { c.b = 0; ++c.hh; }
            c.len = len(c.b);
        } while (c.len < 0);
        return true;
    }
};

// Programmatic dependent launch: the next kernel of the stream may start once every CTA of this one has called the first;
// the second waits until the kernels this one was launched behind have finished.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
#endif

// Two kernels share an SM only while it is split between L1 and shared memory the same way: all three ask for the same split.
template <typename K>
cudaError_t prepare_kernel(K kernel, int smem) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e == cudaSuccess && smem > 0) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    return e;
}

// Launch a kernel that may start while the one before it in the stream still runs.
template <typename... P, typename... A>
cudaError_t launch_behind(void (*kernel)(P...), dim3 grid, int threads, int smem, cudaStream_t st, bool behind, A... args) {
    cudaError_t e = prepare_kernel(kernel, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = behind ? 1 : 0;
    e = cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
    if (e == cudaSuccess) count_launches(1);
    return e;
}

// The three kernels of a step: prefix, own (beside it: launched behind it, sharing no result) and merge (launched behind
// own, which ends after the prefix kernel).  The own kernel, bf16 (decode_shared_own.cu); cudaErrorNotSupported = use the
// CUDA-core kernel
cudaError_t launch_shared_own_tma(const SharedArgs& a, const SharedPlan& p, int D, bool behind, cudaStream_t st);
// the prefix on the tensor cores (decode_shared_tc.cu); cudaErrorNotSupported = use the CUDA-core kernel
cudaError_t launch_shared_prefix_tc(const SharedArgs& a, const SharedPlan& p, int D, cudaStream_t st);

}  // namespace loma
