// What the kernels of the shared-prefix decode step have in common: how the work is cut and where partial results lie.
#pragma once

#include <algorithm>

#include "loma_internal.cuh"

namespace loma {

constexpr int SHP_ROWS = 128;   // query rows of a prefix tile
constexpr int SHP_KEYS = 64;    // prefix keys per block on the tensor cores
constexpr int SIMT_K = 32;      // and on CUDA cores, where a block takes a few microseconds: finer shares
constexpr int OWN_KEYS = 16;    // own keys per block
constexpr int OWN_WARPS = 4;    // an own worker is a warp
constexpr int OWN_CTAS = 148, STREAM_CTAS = 4 * 148;
// sequences of so many blocks are not cut, while there are so few query rows that the workers join their parts quickly and
// so few prefix blocks that it does not matter which kernel starts first (B32 H32, own caches up to 64, prefix 8192: 36 us cut, 42
// whole; B32 Hq32 Hkv8, prefix 16384: 30 against 46)
constexpr int OWN_WHOLE = 8, OWN_WHOLE_ROWS = 2 * OWN_CTAS * OWN_WARPS;

// Prefix CTAs that a call is cut for: one or two per SM.  Alone, two fill each other's waits (B128 Hq32 Hkv8, prefix 16384: 33-35
// us against 45-48; B32 H32, the HBM-bound one: 40-43 against 48-51).  But beside a CTA of the own kernel an SM has room for
// one, so two per SM become two waves wherever the own kernel lasts as long as a CTA's share.  Hence two only where the
// prefix is the longer part by far (see make_shared_plan).
constexpr int SHP_CTAS = 148;

// The cut of a call.  Depends on the sizes alone, so results repeat and the workspace can be sized before the call.
//
// Both parts are cut into equal shares whatever their shape.  The blocks of all units of work are numbered through -- prefix:
// unit = kv head, p_keys keys a block; own: unit = (kv head, head tile, sequence), OWN_KEYS keys a block -- and worker w of
// W takes blocks [T w / W, T (w + 1) / W).  A worker's stay in one unit is a segment with a partial result in slot w + unit:
// along the numbering either the worker or the unit moves on, so no two segments share a slot, and the segments of one unit
// lie behind one another.  Own lengths are known on the device only, so T is found there.
// A prefix worker is m_tiles CTAs, one per tile of SHP_ROWS query rows: they walk the same keys at the same time, so K and V
// come out of HBM once and reach the other tiles through L2 while the own kernel streams through it.
struct SharedPlan {
    int m_tiles;        // prefix: tiles of SHP_ROWS query rows per kv head
    int p_keys;         //         keys per block
    int p_blocks;       //         blocks per kv head (0: no prefix)
    int p_workers;      //         W: m_tiles CTAs each
    int g_rows;         // own: query heads of a kv head per head tile (8 or 16 rows of a warp-level product, or fewer heads)
    int g_tiles;        //      head tiles per kv head
    int workers;        //      W, before it is cut down for few blocks
    bool whole;         //      units are not cut: worker w takes units w, w + W, ..., and slot = unit
    // partial results in the workspace, as offsets in floats.  Prefix segment: outputs [D/4][128][4] (so that a warp whose lanes
    // are rows stores 512 contiguous bytes) and 128 log2-sum-exps.  Own segment: outputs [g_rows][D] and g_rows
    // log2-sum-exps.  cum: int64 [B + 1], blocks before sequence b within one (kv head, head tile).
    int64_t p_o, p_lse, own_o, own_lse, cum, total;
};

__host__ __device__ inline int64_t own_blocks(int len) { return len < 0 ? 0 : len / OWN_KEYS + 1; }   // keys 0 .. len: len is the new token

// the worker that block t of T belongs to, and the first block of worker w (W <= T)
__host__ __device__ inline int64_t block_worker(int64_t t, int64_t T, int64_t W) { return ((t + 1) * W - 1) / T; }
__host__ __device__ inline int64_t first_block(int64_t w, int64_t T, int64_t W) { return T / W * w + T % W * w / W; }

__host__ __device__ inline int64_t own_workers(int64_t T, int workers) { return T < workers ? T : workers; }

// pages: entries to a page of the prefix (0: contiguous).  cuda_cores: both parts run on CUDA cores (fp32, pages of fewer than 8,
// own caches of fewer than 16 rows in all, second opinion)
inline SharedPlan make_shared_plan(int B, int Hq, int Hkv, int D, int prefix_len, int max_len, int pages, bool cuda_cores) {
    SharedPlan p;
    const int64_t g = Hq / Hkv, rows = (int64_t)B * g;
    p.m_tiles = (int)((rows + SHP_ROWS - 1) / SHP_ROWS);
    p.p_keys = cuda_cores ? SIMT_K : SHP_KEYS;
    p.p_blocks = (prefix_len + p.p_keys - 1) / p.p_keys;
    p.g_rows = cuda_cores ? (g < 3 ? (int)g : 4) : (g <= 8 ? (int)g : 16);
    p.g_tiles = (int)((g + p.g_rows - 1) / p.g_rows);
    // Blocks per SM of both parts (own: at most).  A prefix block takes an SM 0.8 us, an own block 0.2, starting the own kernel
    // five.  Measured, one CTA per SM against two: B128 Hq32 Hkv8 own 1500, prefix 16384 / 40000: 92 / 119 us against 94 / 134; own 64:
    // 54 / 103 against 54 / 88; B200 Hq64 Hkv8 own 300, prefix 30000: 244 against 211; B16 Hq32 Hkv8 own 100, prefix 4096 / 32768:
    // 15.5 / 36.5 against 20.3 / 39.8.  max_len is the caller's bound, the lengths being on the device: where it is a table's capacity
    // and own caches are short, a long prefix is cut for one CTA per SM as if they were long.  Tiles of several pages are work for the one thread that asks for them, and two CTAs have
    // two: the last case in pages of 16, 48 against 43.
    // Where the prefix kernel goes first (p.whole) it has the SMs to itself.
    const int64_t all = (int64_t)Hkv * p.p_blocks;
    p.whole = !cuda_cores && own_blocks(max_len) <= OWN_WHOLE && (int64_t)B * Hq <= OWN_WHOLE_ROWS && all * p.m_tiles <= 2 * SHP_CTAS;
    const int64_t p_sm = all * p.m_tiles / 148, own_sm = (int64_t)B * Hkv * p.g_tiles * own_blocks(max_len) / 148;
    const bool two = p.whole || (!cuda_cores && (pages > 0 && pages < SHP_KEYS ? p_sm > 6 + own_sm : p_sm > 30 + own_sm + own_sm / 8));
    // CUDA cores: B60 Hq16 Hkv2, prefix 4000 84 us cut for one per SM, 96 for two
    int64_t w = std::max(1, SHP_CTAS * (two ? 2 : 1) / p.m_tiles);
    // shares that end inside a kv head make most workers change heads once, which costs about as much as six blocks (draining
    // the products, storing a partial result, new query rows): whole workers per kv head where their longer shares cost less
    const int64_t whole = w / Hkv * Hkv;
    if (whole > 0 && (all + whole - 1) / whole <= (all + w - 1) / w + 6) w = whole;
    p.p_workers = (int)std::min<int64_t>(w, all);
    p.workers = (cuda_cores ? STREAM_CTAS : OWN_CTAS) * OWN_WARPS;
    int64_t at = 0;
    auto take = [&](int64_t n) { const int64_t o = at; at += (n + 63) / 64 * 64; return o; };
    const int64_t p_segments = p.p_blocks ? (int64_t)(p.p_workers + Hkv) * p.m_tiles : 0, segments = p.workers + (int64_t)B * Hkv * p.g_tiles;
    p.p_o = take(p_segments * SHP_ROWS * D);
    p.p_lse = take(p_segments * SHP_ROWS);
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

// the row that the new token of (b, h), entry j, is stored to, or -1: its sequence has no page for it (loma_paged_extend writes -1
// into the table when the free list runs out), and the page that reads are clamped to is somebody else's
__device__ __forceinline__ int64_t token_row(const SharedArgs& a, int b, int h, int j) {
    if (a.pg.table) {
        const int page = __ldg(a.pg.table + (int64_t)b * a.pg.max_pages + (j >> a.pg.log2_ps));
        if (page < 0 || page >= a.pg.n_pages) return -1;
    }
    return own_row(a, b, h, j);
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

#endif

#ifdef __CUDACC__
// One query row's four features joined from partial results under a running maximum.  The time of a merge is that of its chain
// of dependent loads, so AT_ONCE results are taken at a time, values and log2-sum-exps together.
struct RowMerge {
    float M = -INFINITY, total = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    // n results: log2-sum-exps at lse[s * lse_step], values at v[s * v_step]; of every WAYS batches the way-th
    template <int WAYS, int AT_ONCE>
    __device__ __forceinline__ void add(int n, const float* lse, int64_t lse_step, const float* v, int64_t v_step, int way) {
        for (int s0 = way * AT_ONCE; s0 < n; s0 += WAYS * AT_ONCE) {
            float e[AT_ONCE];
            float4 y[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                e[u] = -INFINITY;
                if (s0 + u < n) {
                    e[u] = __ldcg(lse + (s0 + u) * lse_step);
                    y[u] = __ldcg(reinterpret_cast<const float4*>(v + (s0 + u) * v_step));
                }
            }
            float m = M;
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) m = fmaxf(m, e[u]);
            const float keep = M == -INFINITY ? 0.f : exp2f(M - m);
            M = m;
            total *= keep;
            o.x *= keep; o.y *= keep; o.z *= keep; o.w *= keep;
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                if (e[u] == -INFINITY) continue;   // no weight: past the last, or scores of -inf (values 0/0)
                const float f = exp2f(e[u] - m);
                total += f;
                o.x = fmaf(f, y[u].x, o.x); o.y = fmaf(f, y[u].y, o.y); o.z = fmaf(f, y[u].z, o.z); o.w = fmaf(f, y[u].w, o.w);
            }
        }
    }
    template <typename T, int D>
    __device__ __forceinline__ void store(const SharedArgs& a, int64_t row, int c4) const {   // row = b * Hq + head
        const float inv = 1.f / total;
        if constexpr (sizeof(T) == 2)
            *reinterpret_cast<uint2*>(static_cast<T*>(a.o) + row * D + c4 * 4) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
        else
            *reinterpret_cast<float4*>(static_cast<T*>(a.o) + row * D + c4 * 4) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        if (a.lse && c4 == 0) a.lse[row] = (M + log2f(total)) * 0.6931471805599453f;
    }
};

// the prefix segments of query tile mt of kv head h: how many, and the first one's slot (the next is m_tiles further)
struct PrefixSegments {
    int n = 0;
    int64_t first = 0;
    __device__ __forceinline__ PrefixSegments(const SharedArgs& a, const SharedPlan& p, int h, int mt) {
        if (p.p_blocks == 0) return;
        const int64_t all = (int64_t)a.Hkv * p.p_blocks, w0 = block_worker((int64_t)h * p.p_blocks, all, p.p_workers);
        n = (int)(block_worker((int64_t)(h + 1) * p.p_blocks - 1, all, p.p_workers) - w0) + 1;
        first = (w0 + h) * p.m_tiles + mt;
    }
};
#endif

// The three kernels of a step: own, prefix (launched behind it, sharing no result, so that it starts beside it) and merge
// (launched behind the prefix kernel, which ends after the own kernel).  Where own caches hold a few blocks at most and the
// prefix is short (p.whole), the prefix kernel comes first, each sequence stays with one warp of the own kernel, and that joins
// the parts itself: two kernels.  On CUDA cores: prefix, own, merge.
// bf16 own caches (decode_shared_own.cu), and whether TMA can address them
bool shared_own_tma_fits(const SharedArgs& a);
cudaError_t launch_shared_own_tma(const SharedArgs& a, const SharedPlan& p, int D, bool behind, cudaStream_t st);
// the prefix on the tensor cores (decode_shared_tc.cu), and whether TMA can address it
bool shared_prefix_tc_fits(const SharedArgs& a);
cudaError_t launch_shared_prefix_tc(const SharedArgs& a, const SharedPlan& p, int D, bool behind, cudaStream_t st);

}  // namespace loma
