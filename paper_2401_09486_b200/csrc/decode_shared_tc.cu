// The prefix part of the shared-prefix decode step on the 5th-generation tensor cores (bf16).
//
// The B g query rows of a kv head all see the same prefix keys, so their scores and outputs are two matrix products with
// an online softmax between them: S = Q K^T, O = sum over keys of P V.  No mask but the end of the prefix.  A CTA takes 128
// query rows (one row per TMEM lane) and a range of keys at a time; ranges are joined by the merge kernel.  With few rows the kernel
// is bound by HBM (the prefix is read once per 128 rows), with many by the chain tensor pipe -> softmax -> tensor pipe, so
// two CTAs fit on an SM and fill each other's waits: each has 256 of the 512 TMEM columns and half of the shared memory.  How
// many a call is cut for: make_shared_plan.
//
//   warps 0-3  query rows, softmax: thread = query row.  64 keys (an "event") at a time: scores out of TMEM, row maximum, probabilities
//              2^(s scale - ref) as bf16 back over the scores.  The reference maximum only moves, and the accumulator in TMEM
//              is only rescaled, when a row's maximum has grown by more than 2^8, which bounds a probability by 2^8
//   warps 4-7  a warpgroup of their own, so that registers can be moved to the softmax; warps 6 and 7 do nothing
//   warp 4     TMA: K and V in tiles of 64 keys through one ring of NS slots, in the order in which they are used
//              K0 K1 V0 K2 V1 K3 V2 ...
//   warp 5     MMA: S(e+2) is issued right after P V(e) into the score buffer that event e has left, so the tensor pipe works
//              on one buffer while the warpgroup works on the other
// P is rounded to bf16 for the second product (off by 2^-8 of its value at most); row sums are taken in fp32 before the
// rounding, scores, maxima, sums and outputs are fp32 throughout.
// Measured alone: B128 Hq32 Hkv8 D128, prefix 16384: 33-35 us, 1.03 PFLOP/s (0.62 of a library GEMM; tensor pipe active 52 % of the
// cycles); B32 H32, prefix 16384, bound by HBM: 40-43 us, 6.2-6.7 TB/s.
#include "decode_shared.cuh"
#include "tcgen05_common.cuh"

namespace loma {

struct SharedMaps {
    CUtensorMap k, v;
};

// features 0..63 of a panel (or of all panels, by the map's box), rows from `row`, of head or page-head z
__device__ __forceinline__ void tma_prefix(uint32_t dst, const CUtensorMap* map, uint32_t bar, int row, int panel, int z) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(0), "r"(row), "r"(panel), "r"(z)
                 : "memory");
}

constexpr int SHT_THREADS = 256, SHT_TMEM = 256;

template <int D>
struct ShtSmem {
    static constexpr int PANELS = D / 64;
    static constexpr int Q_PANEL = SHP_ROWS * 128, KV_PANEL = SHP_KEYS * 128;      // 64 features of every row
    static constexpr int SLOT = PANELS * KV_PANEL;
    static constexpr int NS = D == 128 ? 5 : 10;                                   // ring slots: 80 KB either way
    static constexpr int RING = PANELS * Q_PANEL;
    // 1 KB more than the tiles: they start on a 1 KB boundary, and the gap before or behind them holds the barriers.  Twice
    // this and the 1 KB the system takes per CTA is exactly an SM's 228 KB.
    static constexpr int TILES = RING + NS * SLOT, TOTAL = TILES + 1024;
};

struct ShtShared {   // in the gap (512 bytes at least)
    uint64_t full[10], empty[10], sf[2], pf[2], of[2], qf;
    uint32_t tmem;
    int abort_flag;
};

struct ShtParams {
    const __nv_bfloat16* q;
    const int32_t* prefix_table;   // NULL: contiguous
    float *o, *lse;                // partial results (see SharedPlan)
    int* status;
    int B, Hq, Hkv, g, m_tiles, p_blocks, p_workers, prefix_len, log2_ps, n_pages, box_rows;
    float scale_log2;
};

template <int D>
__global__ void __launch_bounds__(SHT_THREADS, 2)
shared_prefix_tc_kernel(const __grid_constant__ SharedMaps maps, const ShtParams p) {
    using SM = ShtSmem<D>;
    constexpr int PANELS = SM::PANELS, NS = SM::NS;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u, before = base - raw;
    uint8_t* tiles = smem_raw + before;
    ShtShared* sh = reinterpret_cast<ShtShared*>(before >= 512 ? smem_raw + ((16u - (raw & 15u)) & 15u) : tiles + SM::TILES);
    static_assert(sizeof(ShtShared) <= 496, "the barriers fit in the gap");
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    auto bar = [&](uint64_t* b) { return smem_u32(b); };

    let_next_start();
    // this CTA's share of the blocks, unit by unit
    const int worker = blockIdx.x / p.m_tiles, mt = blockIdx.x - worker * p.m_tiles;
    const int64_t all = (int64_t)p.Hkv * p.p_blocks;
    const int64_t t_first = first_block(worker, all, p.p_workers), t_end = first_block(worker + 1, all, p.p_workers);
    struct Segment {
        int h, begin, E;   // kv head; first key; blocks ("events"), at least one
    };
    auto segment = [&](int64_t t) {
        Segment g;
        g.h = (int)(t / p.p_blocks);
        const int blk = (int)(t - (int64_t)g.h * p.p_blocks);
        g.E = (int)min((int64_t)(p.p_blocks - blk), t_end - t);
        g.begin = blk * SHP_KEYS;
        return g;
    };
    volatile int* abortp = &sh->abort_flag;

    if (threadIdx.x == 0) {
        sh->abort_flag = 0;
        for (int i = 0; i < NS; ++i) { mbar_init(bar(&sh->full[i]), 1); mbar_init(bar(&sh->empty[i]), 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(bar(&sh->sf[i]), 1); mbar_init(bar(&sh->pf[i]), 128); mbar_init(bar(&sh->of[i]), 1); }
        mbar_init(bar(&sh->qf), 128);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem)), "r"(SHT_TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh->tmem;   // score buffers at +0 and +64, output accumulator at +128

    // Items (tiles of 64 keys) and events are numbered through over all segments: item n lies in ring slot n mod NS, event e uses
    // score buffer e & 1.
    // registers: launched with 128 a thread (two CTAs fill an SM's, and each of its four schedulers has the same share), of which
    // warps 4-7 leave most to the softmax
    if (warp == 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;" ::: "memory");
        // ------------------------------------------------------------ TMA producer
        bool ok = true;
        // a box of a whole tile's 64 rows takes all panels; smaller ones (short pages, a short prefix) go panel by panel, since the
        // products want a panel's rows behind one another
        const int parts = p.prefix_table ? SHP_KEYS / p.box_rows : 1, boxes = p.box_rows == SHP_KEYS ? 1 : parts * PANELS;
        int n = 0;
        for (int64_t t = t_first; ok && t < t_end;) {
            const Segment g = segment(t);
            t += g.E;
            int e_k = 0, e_v = 0;
            for (int i = 0; i < 2 * g.E; ++i, ++n) {
                const bool is_k = e_k < g.E && e_k < e_v + 2;
                const int e = is_k ? e_k++ : e_v++;
                const int slot = n % NS;
                ok = __all_sync(0xffffffffu, mbar_wait(bar(&sh->empty[slot]), ((n / NS) & 1) ^ 1, abortp, p.status));
                if (!ok) break;
                const uint32_t full = bar(&sh->full[slot]), dst = base + SM::RING + slot * SM::SLOT;
                if (lane == 0) mbar_expect_tx(full, parts * p.box_rows * 128 * PANELS);
                __syncwarp();
                const CUtensorMap* map = is_k ? &maps.k : &maps.v;
                if (lane < boxes) {
                    const int pn = lane % PANELS, part = lane / PANELS;
                    int row = g.begin + e * SHP_KEYS + part * p.box_rows, z = g.h;
                    if (p.prefix_table) {
                        // past the last page of the prefix the last entry's page is loaded again (its rows are masked)
                        const int at = min(row, p.prefix_len - 1);
                        const int page = min(max(__ldg(p.prefix_table + (at >> p.log2_ps)), 0), p.n_pages - 1);
                        z = page * p.Hkv + g.h;
                        row &= (1 << p.log2_ps) - 1;
                    }
                    tma_prefix(dst + pn * SM::KV_PANEL + part * p.box_rows * 128, map, full, row, pn, z);
                }
            }
        }
        if (!ok) {
            // leaving early: give copies already in flight a bounded time to land in this CTA's shared memory
            const long long t0 = clock64();
            while (clock64() - t0 < 2000000ll) {}
        }
    } else if (warp == 5) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;" ::: "memory");
        // ------------------------------------------------------------ MMA issuer: uniform control flow, one elected lane issues
        // instruction descriptors: fp32 accumulate, bf16 x bf16, M = 128; N = 64 keys, or N = D with V as the MN-major operand
        constexpr uint32_t IDESC_S = (1u << 4) | (1u << 7) | (1u << 10) | ((64u >> 3) << 17) | ((128u >> 4) << 24);
        constexpr uint32_t IDESC_PV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | (((uint32_t)D >> 3) << 17) | ((128u >> 4) << 24);
        const uint64_t qd = smem_desc(base, 16, 1024);
        int n = 0, e0 = 0, seg = 0;   // items used; events and segments before this one
        bool ok = true;
        auto take = [&]() {
            ok = __all_sync(0xffffffffu, mbar_wait(bar(&sh->full[n % NS]), (n / NS) & 1, abortp, p.status));
            return n++ % NS;
        };
        auto scores = [&](int e) {
            const int slot = take();
            if (!ok) return;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t kd = smem_desc(base + SM::RING + slot * SM::SLOT, 16, 1024);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                    mma_ss(tmem + (e & 1) * 64, qd + (uint64_t)(((kk >> 2) * SM::Q_PANEL + (kk & 3) * 32) >> 4),
                           kd + (uint64_t)(((kk >> 2) * SM::KV_PANEL + (kk & 3) * 32) >> 4), IDESC_S, kk > 0);
                tc_commit(bar(&sh->empty[slot]));
                tc_commit(bar(&sh->sf[e & 1]));
            }
            __syncwarp();
        };
        for (int64_t t = t_first; ok && t < t_end; ++seg) {
            const int E = segment(t).E;
            t += E;
            ok = __all_sync(0xffffffffu, mbar_wait(bar(&sh->qf), seg & 1, abortp, p.status));   // the segment's query rows
            if (!ok) break;
            scores(e0);
            if (ok && E > 1) scores(e0 + 1);
            for (int i = 0; ok && i < E; ++i) {
                const int e = e0 + i, b = e & 1;
                ok = __all_sync(0xffffffffu, mbar_wait(bar(&sh->pf[b]), (e >> 1) & 1, abortp, p.status));
                if (!ok) break;
                const int slot = take();
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
                    const uint64_t vd = smem_desc(base + SM::RING + slot * SM::SLOT, SM::KV_PANEL, 1024);
#pragma unroll
                    for (int k4 = 0; k4 < 4; ++k4)
                        mma_ts(tmem + 128, tmem + b * 64 + k4 * 8, vd + (uint64_t)((k4 * 2048) >> 4), IDESC_PV, i > 0 || k4 > 0);
                    tc_commit(bar(&sh->empty[slot]));
                    tc_commit(bar(&sh->of[b]));   // last: whoever leaves on it leaves no arrival behind
                }
                __syncwarp();
                if (i + 2 < E) scores(e + 2);
            }
            e0 += E;
        }
    } else if (warp >= 6) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;" ::: "memory");
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;" ::: "memory");
        // ------------------------------------------------------------ query rows, softmax and partial results
        const int rr = threadIdx.x, rows = p.B * p.g;
        const uint32_t lane_addr = tmem + ((uint32_t)(warp * 32) << 16), o_addr = lane_addr + 128;
        bool ok = true;
        // query rows into the swizzled panels: row m of the kv head is head h g + m mod g of sequence m div g; rows past the
        // last are zero
        auto load_q = [&](const Segment& g) {
            constexpr int CH = D / 8, RPP = 128 / CH, PASSES = SHP_ROWS / RPP;   // chunks per row, rows per pass
            const int c = rr % CH, r0 = rr / CH;
            uint4 v[PASSES];                                                     // all loads in flight at once
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int m = mt * SHP_ROWS + r0 + i * RPP, b = m / p.g;
                v[i] = make_uint4(0, 0, 0, 0);
                if (m < rows) v[i] = __ldg(reinterpret_cast<const uint4*>(p.q + ((int64_t)b * p.Hq + g.h * p.g + (m - b * p.g)) * D) + c);
            }
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int r = r0 + i * RPP;
                *reinterpret_cast<uint4*>(tiles + (c >> 3) * SM::Q_PANEL + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v[i];
            }
            fence_async_smem();
            mbar_arrive(bar(&sh->qf));
        };
        int e0 = 0, n_last = -1;   // events before this segment; number of its last item
        Segment g = segment(t_first), next = g;
        if (t_first < t_end) load_q(g);
        for (int64_t t = t_first; ok && t < t_end; g = next) {
            float m_used = -INFINITY, l = 0.f;
            const int E = g.E;
            n_last += 2 * E;
            t += E;
            for (int i = 0; i < E; ++i) {
                const int e = e0 + i, b = e & 1;
                const uint32_t s_addr = lane_addr + b * 64;
                ok = __all_sync(0xffffffffu, mbar_wait(bar(&sh->sf[b]), (e >> 1) & 1, abortp, p.status));
                if (!ok) break;
                tc_fence_after();
                uint32_t s[64];
                tmem_ld32(s_addr, s);
                tmem_ld32(s_addr + 32, s + 32);
                tmem_wait_ld();
                const int valid = p.prefix_len - (g.begin + i * SHP_KEYS);
                if (valid < SHP_KEYS) {
                    // the last tile of the prefix: keys past its end are blocked, and V rows there become zero (a page or an
                    // unused row may hold anything, and 0 x NaN is not 0)
#pragma unroll
                    for (int k = 0; k < 64; ++k)
                        if (k >= valid) s[k] = 0xff800000u;
                    const int slot = n_last % NS;   // V of a unit's last event is the segment's last item
                    ok = __all_sync(0xffffffffu, mbar_wait(bar(&sh->full[slot]), (n_last / NS) & 1, abortp, p.status));
                    if (!ok) break;
                    uint8_t* v = tiles + SM::RING + slot * SM::SLOT;
                    for (int k = rr; k < (SHP_KEYS - valid) * 8 * PANELS; k += 128) {
                        const int pn = k / ((SHP_KEYS - valid) * 8), rest = k - pn * (SHP_KEYS - valid) * 8;
                        *reinterpret_cast<uint4*>(v + pn * SM::KV_PANEL + valid * 128 + rest * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_async_smem();
                }
                float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
                for (int k = 0; k < 64; k += 8) {
                    mx0 = max3(mx0, __uint_as_float(s[k]), __uint_as_float(s[k + 1]));
                    mx1 = max3(mx1, __uint_as_float(s[k + 2]), __uint_as_float(s[k + 3]));
                    mx2 = max3(mx2, __uint_as_float(s[k + 4]), __uint_as_float(s[k + 5]));
                    mx3 = max3(mx3, __uint_as_float(s[k + 6]), __uint_as_float(s[k + 7]));
                }
                const float mrow = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3)) * p.scale_log2;
                const bool need = mrow > m_used + 8.f;
                if (i > 0 && __any_sync(0xffffffffu, need)) {
                    ok = __all_sync(0xffffffffu, mbar_wait(bar(&sh->of[b ^ 1]), ((e - 1) >> 1) & 1, abortp, p.status));
                    if (!ok) break;
                    tc_fence_after();
                    const float alpha = need ? fast_ex2(m_used - mrow) : 1.f;
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t r[32];
                        tmem_ld32(o_addr + c * 32, r);
                        tmem_wait_ld();
#pragma unroll
                        for (int k = 0; k < 32; ++k) r[k] = __float_as_uint(__uint_as_float(r[k]) * alpha);
                        tmem_st32(o_addr + c * 32, r);
                    }
                    l *= alpha;
                }
                if (need) m_used = mrow;
                const float neg_ref = m_used == -INFINITY ? 0.f : -m_used;
                const uint64_t sc2 = pack2(p.scale_log2, p.scale_log2), nr2 = pack2(neg_ref, neg_ref);
                uint64_t lsa = pack2(0.f, 0.f), lsb = lsa;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t pk[16];
#pragma unroll
                    for (int k = 0; k < 32; k += 4) {
                        float x0, x1, x2, x3;
                        unpack2(fma2(pack2(__uint_as_float(s[c * 32 + k]), __uint_as_float(s[c * 32 + k + 1])), sc2, nr2), x0, x1);
                        unpack2(fma2(pack2(__uint_as_float(s[c * 32 + k + 2]), __uint_as_float(s[c * 32 + k + 3])), sc2, nr2), x2, x3);
                        const float p0 = fast_ex2(x0), p1 = fast_ex2(x1), p2 = fast_ex2(x2), p3 = fast_ex2(x3);
                        lsa = add2(lsa, pack2(p0, p1));
                        lsb = add2(lsb, pack2(p2, p3));
                        pk[k >> 1] = pack_bf16(p0, p1);
                        pk[(k >> 1) + 1] = pack_bf16(p2, p3);
                    }
                    tmem_st16(s_addr + c * 16, pk);
                }
                {
                    float a0, a1, b0, b1;
                    unpack2(lsa, a0, a1);
                    unpack2(lsb, b0, b1);
                    l += (a0 + a1) + (b0 + b1);
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(bar(&sh->pf[b]));
            }
            if (!ok) break;
            e0 += E;
            // every score product of the segment has completed (its last scores have been read): the next segment's query rows
            // may go in while the last P V runs
            if (t < t_end) {
                next = segment(t);
                load_q(next);
            }
            ok = __all_sync(0xffffffffu, mbar_wait(bar(&sh->of[(e0 - 1) & 1]), ((e0 - 1) >> 1) & 1, abortp, p.status));
            if (!ok) break;
            tc_fence_after();
            const float inv = 1.f / l;
            const int64_t slot = (int64_t)(worker + g.h) * p.m_tiles + mt;
            const bool live = mt * SHP_ROWS + rr < rows;
            float4* out = reinterpret_cast<float4*>(p.o + slot * SHP_ROWS * D) + rr;
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                uint32_t r[32];
                tmem_ld32(o_addr + c * 32, r);
                tmem_wait_ld();
                if (live) {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        __stcg(out + (c * 8 + k) * SHP_ROWS, make_float4(__uint_as_float(r[4 * k]) * inv, __uint_as_float(r[4 * k + 1]) * inv,
                                                                        __uint_as_float(r[4 * k + 2]) * inv, __uint_as_float(r[4 * k + 3]) * inv));
                }
            }
            if (live) p.lse[slot * SHP_ROWS + rr] = m_used + log2f(l);
            tc_fence_before();   // the accumulator has been read before the next segment's probabilities are announced
        }
    }
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(SHT_TMEM) : "memory");
    }
    // the merge needs the own kernel's results too: this kernel ends after it.  One CTA waits; the others leave their places
    if (blockIdx.x == 0) wait_for_previous();
}

// ------------------------------------------------------------------ host side
// (64 features, rows, panels, heads or page-heads) of the prefix; box: 64 features of box_rows rows, of all panels if a tile is
// one box.
static bool encode_prefix(CUtensorMap* map, const void* p, int D, int64_t rows, int64_t row_stride_outer, int64_t outer, int box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[4] = {64, (cuuint64_t)rows, (cuuint64_t)(D / 64), (cuuint64_t)outer};
    const cuuint64_t strides[3] = {(cuuint64_t)D * 2, 128, (cuuint64_t)row_stride_outer * D * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)box_rows, (cuuint32_t)(box_rows == SHP_KEYS ? D / 64 : 1), 1}, es[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(p), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static int64_t prefix_outer(const SharedArgs& a) { return a.prefix_table ? (int64_t)a.pg.n_pages * a.Hkv : a.Hkv; }

// a box of fewer than 8 rows of a page would start inside a swizzle group, and a coordinate is 32 bits
bool shared_prefix_tc_fits(const SharedArgs& a) {
    return encode_fn() && (!a.prefix_table || a.pg.log2_ps >= 3) && prefix_outer(a) <= INT_MAX;
}

template <int D>
static cudaError_t prefix_tc_t(const SharedArgs& a, const SharedPlan& p, bool behind, cudaStream_t st) {
    ShtParams t;
    SharedMaps maps;
    const int ps = 1 << a.pg.log2_ps;
    const int64_t rows = a.prefix_table ? ps : a.prefix_len, step = a.prefix_table ? ps : a.prefix_cap, outer = prefix_outer(a);
    t.box_rows = (int)std::min<int64_t>(rows, SHP_KEYS);
    if (p.p_keys != SHP_KEYS || !encode_prefix(&maps.k, a.k_prefix, D, rows, step, outer, t.box_rows) ||
        !encode_prefix(&maps.v, a.v_prefix, D, rows, step, outer, t.box_rows))
        return cudaErrorInvalidValue;
    float* ws = static_cast<float*>(a.ws);
    t.q = static_cast<const __nv_bfloat16*>(a.q);
    t.prefix_table = a.prefix_table;
    t.o = ws + p.p_o;
    t.lse = ws + p.p_lse;
    t.status = device_status_word();
    if (!t.status) return cudaErrorUnknown;
    t.B = a.B; t.Hq = a.Hq; t.Hkv = a.Hkv; t.g = a.g; t.m_tiles = p.m_tiles; t.p_blocks = p.p_blocks; t.p_workers = p.p_workers; t.prefix_len = a.prefix_len;
    t.log2_ps = a.pg.log2_ps; t.n_pages = a.pg.n_pages;
    t.scale_log2 = a.scale * 1.4426950408889634f;
    constexpr int smem = ShtSmem<D>::TOTAL;
    return launch_behind(shared_prefix_tc_kernel<D>, dim3(p.p_workers * p.m_tiles), SHT_THREADS, smem, st, behind, maps, t);
}

cudaError_t launch_shared_prefix_tc(const SharedArgs& a, const SharedPlan& p, int D, bool behind, cudaStream_t st) {
    return D == 64 ? prefix_tc_t<64>(a, p, behind, st) : prefix_tc_t<128>(a, p, behind, st);
}

}  // namespace loma
