// The sequences' own entries in the shared-prefix decode step (bf16): a stream bound by HBM.
//
// A worker (one warp) walks its share of the blocks (see SharedPlan) with a ring of its own in shared memory: one TMA
// instruction fetches the 16 K rows of a block and one the V rows, NS - 1 blocks ahead and across the borders between
// sequences, so short sequences stream as well as long ones and no warp waits for another.
//
// The g query heads of a kv head share every K and V row: with 16 keys as the rows and 8 heads as the columns of warp-level
// m16n8k16 products,
//     S^T [keys x heads] = K Q^T          O^T [features x heads] += V^T P^T
// K and (transposed on the way) V fragments come from the 128-byte-swizzled tiles with ldmatrix, without a bank conflict and
// without padding; P^T changes from the accumulator's layout to the operand's with two 8 x 8 transposes (movmatrix), and a
// lane's heads are the same two in scores, maxima, sums and outputs.  A block takes about 150 instructions; four warps per
// SM turn them over faster than HBM delivers (44 bytes per SM and nanosecond, 190 ns for the 8 KB of a block), and 96 KB
// of rings leave room beside a CTA of the prefix kernel: the two run at the same time.
// Measured alone: B128 Hq32 Hkv8 D128, lengths up to 1500, 397 MB: 67.7 us, 5.9 TB/s (0.91 of a copy).
#include "decode_shared.cuh"
#include "tcgen05_common.cuh"

namespace loma {

struct OwnMaps {
    CUtensorMap k, v;
};

template <int D>
struct OwnSmem {
    static constexpr int PANELS = D / 64, TILE = OWN_KEYS * D * 2, STAGE = 2 * TILE;      // K and V of 16 keys
    static constexpr int NS = D == 128 ? 3 : 6;                                           // 24 KB a warp either way
    static constexpr int RING = OWN_WARPS * NS * STAGE;
    static constexpr int TOTAL = RING + 1024;
};

// D += A B, m16n8k16
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

__device__ __forceinline__ void ldsm(uint32_t addr, uint32_t (&v)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t addr, uint32_t (&v)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}

// all features of OWN_KEYS (or box_rows) rows: features 0..63, rows, 64-feature panels
__device__ __forceinline__ void tma_rows(uint32_t dst, const CUtensorMap* map, uint32_t bar, int row) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %3}], [%2];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(0), "r"(row)
                 : "memory");
}

// R: column tiles of 8 query heads.  WHOLE: p.whole.
template <int D, int R, bool WHOLE>
__global__ void __launch_bounds__(OWN_WARPS * 32, R == 1 ? 3 : 2)
shared_own_tma_kernel(const __grid_constant__ OwnMaps maps, const SharedArgs a, const SharedPlan p, int* status) {
    using SM = OwnSmem<D>;
    constexpr int KS = D / 16, NS = SM::NS, PANELS = SM::PANELS;   // KS: k-steps of the scores, and output tiles of 16 features
    extern __shared__ uint8_t own_smem[];
    __shared__ __align__(8) uint64_t bars[OWN_WARPS][NS];
    __shared__ int64_t scan[SeqBlocks::MAX_GROUPS + 1];
    __shared__ int64_t wsum[OWN_WARPS];
    __shared__ int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, j = lane & 3;
    if (lane == 0)
        for (int i = 0; i < NS; ++i) mbar_init(smem_u32(&bars[warp][i]), 1);
    if (threadIdx.x == 0) abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");

    let_next_start();
    if (threadIdx.x == 0) {   // fetched while the lengths are
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&maps.k)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&maps.v)) : "memory");
    }
    const SeqBlocks sb{a};
    const int w = warp * gridDim.x + blockIdx.x;   // neighbours on different SMs
    const int units = a.Hkv * p.g_tiles * a.B;
    // Cursors over this worker's blocks: `c` is being worked on, `f` is being fetched.  `left`: blocks of the share still to come,
    // or (WHOLE) the unit the cursor is in.
    struct Cursor {
        SeqBlocks::Cursor at;
        int left;
    } c, f;
    enum { END, SAME, NEW };       // what the next block is: none, of the same sequence and head, of another
    auto to_unit = [&](Cursor& x, int u) {   // WHOLE: the first unit from u on, in steps of the workers, that holds a request
        for (; u < units; u += p.workers) {
            x.at.hh = u / a.B;
            x.at.b = u - x.at.hh * a.B;
            x.at.len = sb.len(x.at.b);
            if (x.at.len >= 0) break;
        }
        x.at.blk = 0;
        x.left = u;
        return u < units;
    };
    auto next = [&](Cursor& x) -> int {
        if constexpr (WHOLE) {
            if ((x.at.blk + 1) * OWN_KEYS <= x.at.len) { ++x.at.blk; return SAME; }
            return to_unit(x, x.left + p.workers) ? NEW : END;
        } else {
            if (--x.left == 0) return END;
            return sb.advance(x.at) ? NEW : SAME;
        }
    };
    bool busy;
    if constexpr (WHOLE) {
        busy = to_unit(c, w);
        __syncthreads();           // barriers and abort flag are set up
    } else {
        const int per = sb.scan<OWN_WARPS>(scan, wsum, blockIdx.x == 0 ? reinterpret_cast<int64_t*>(static_cast<float*>(a.ws) + p.cum) : nullptr);
        const int64_t T = scan[(a.B + per - 1) / per] * a.Hkv * p.g_tiles, W = own_workers(T, p.workers);
        busy = w < W;
        if (busy) {
            const int64_t t0 = first_block(w, T, W);
            c.left = (int)(first_block(w + 1, T, W) - t0);
            c.at = sb.find(t0, scan, per);
        }
    }
    if (busy) {
        f = c;
        const uint32_t ring = ((smem_u32(own_smem) + 1023u) & ~1023u) + warp * NS * SM::STAGE;
        uint8_t* ring_gen = own_smem + (ring - smem_u32(own_smem));
        volatile int* abortp = &abort_flag;
        // a box holds its rows panel by panel: where panel 1 and rows 8..15 of a tile lie
        const int boxes = a.pg.table ? max(1, OWN_KEYS >> a.pg.log2_ps) : 1, box_rows = OWN_KEYS / boxes;
        const uint32_t panel = box_rows * 128, upper = boxes == 1 ? 1024 : 1024 * PANELS;
        // row of the fetch cursor's block (this lane's box of it), from the top of the cache or pool; a table entry is read one
        // block before it is used
        int base_f = 0, h_f = 0;         // contiguous: first row of the fetch cursor's (sequence, kv head)
        const int32_t* table_f = nullptr;
        auto enter_f = [&]() {
            h_f = p.g_tiles == 1 ? f.at.hh : f.at.hh / p.g_tiles;
            base_f = (f.at.b * a.Hkv + h_f) * a.cap;   // the cache has less than 2^31 rows
            table_f = a.pg.table + (int64_t)f.at.b * a.pg.max_pages;
            // the segment's query heads and new token, wanted when its blocks have arrived
            const int gt_f = f.at.hh - h_f * p.g_tiles, lines = min(p.g_rows, a.g - gt_f * p.g_rows) * PANELS;   // of 128 bytes
            const __nv_bfloat16* line = nullptr;
            if (lane < lines) line = static_cast<const __nv_bfloat16*>(a.q) + ((int64_t)f.at.b * a.Hq + h_f * a.g + gt_f * p.g_rows) * D + lane * 64;
            else if (lane >= 32 - 2 * PANELS && a.k_new)
                line = static_cast<const __nv_bfloat16*>(lane >= 32 - PANELS ? a.k_new : a.v_new) + ((int64_t)f.at.b * a.Hkv + h_f) * D + (lane & (PANELS - 1)) * 64;
            if (line) asm volatile("prefetch.global.L2 [%0];" ::"l"(line));
        };
        auto row_f = [&]() -> int {
            if (!a.pg.table) return base_f + f.at.blk * OWN_KEYS;
            const int key = f.at.blk * OWN_KEYS + (lane < boxes ? lane : 0) * box_rows;
            const int page = min(max(__ldg(table_f + (min(key, f.at.len) >> a.pg.log2_ps)), 0), a.pg.n_pages - 1);
            return ((page * a.Hkv + h_f) << a.pg.log2_ps) + (key & ((1 << a.pg.log2_ps) - 1));
        };
        enter_f();
        int next_row = row_f(), slot_f = 0;
        bool fetching = true;
        auto fetch = [&]() {
            const uint32_t bar = smem_u32(&bars[warp][slot_f]), dst = ring + slot_f * SM::STAGE;
            if (lane == 0) mbar_expect_tx(bar, SM::STAGE);
            __syncwarp();
            if (lane < boxes) {
                tma_rows(dst + lane * 1024 * PANELS, &maps.k, bar, next_row);
                tma_rows(dst + SM::TILE + lane * 1024 * PANELS, &maps.v, bar, next_row);
            }
            slot_f = slot_f + 1 == NS ? 0 : slot_f + 1;
            const int what = next(f);
            fetching = what != END;
            if (what == NEW) enter_f();
            if (fetching) next_row = row_f();
        };
        for (int i = 0; i < NS && fetching; ++i) fetch();

        // ldmatrix addresses of the operands A.  K: rows = keys 0-7 | 8-15, k = features 16 i .. + 7 | + 8 .. + 15.  V: rows = features
        // 16 i .. + 7 | + 8 .. + 15, k = keys 0-7 | 8-15, each 8 x 8 part transposed.  The swizzle exchanges a row's 16-byte
        // chunks: chunk x of row k lies at x ^ (k mod 8).
        const int mi = lane >> 3, mr = lane & 7;
        const uint32_t k_lane = (mi & 1) * upper + mr * 128, k_x = (mi >> 1) ^ mr;
        const uint32_t v_lane = (mi >> 1) * upper + mr * 128 + SM::TILE, v_x = (mi & 1) ^ mr;

        const float scale_log2 = a.scale * 1.4426950408889634f;
        const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q);
        float* ws = static_cast<float*>(a.ws);
        uint32_t qf[R][KS][2];                           // operand B: column = head x * 8 + r, k = features 2j, 2j + 1 and + 8
        float m[R][2], l[R][2], acc[R][KS][4];           // heads x * 8 + 2j, + 1
        int slot = 0, h = 0, gt = 0, heads = 0;
        uint32_t phase = 0;
        bool fresh = true, ok = true;
        for (;;) {
            if (fresh) {   // a new segment: this triple's query heads
                h = p.g_tiles == 1 ? c.at.hh : c.at.hh / p.g_tiles;
                gt = c.at.hh - h * p.g_tiles;
                heads = min(p.g_rows, a.g - gt * p.g_rows);
#pragma unroll
                for (int x = 0; x < R; ++x) {
                    const int hd = x * 8 + r;
                    const uint32_t* qp = reinterpret_cast<const uint32_t*>(q + ((int64_t)c.at.b * a.Hq + h * a.g + gt * p.g_rows + min(hd, heads - 1)) * D);
#pragma unroll
                    for (int i = 0; i < KS; ++i) {
                        qf[x][i][0] = hd < heads ? __ldg(qp + 8 * i + j) : 0u;
                        qf[x][i][1] = hd < heads ? __ldg(qp + 8 * i + j + 4) : 0u;
                    }
                    m[x][0] = m[x][1] = -INFINITY;
                    l[x][0] = l[x][1] = 0.f;
#pragma unroll
                    for (int i = 0; i < KS; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[x][i][e] = 0.f;
                }
                fresh = false;
            }
            const int valid = c.at.len + 1 - c.at.blk * OWN_KEYS;   // keys from this block on, the new token the last of them
            const bool tail = valid <= OWN_KEYS;
            uint4 k_tok, v_tok;   // this lane's part of the new token's rows
            if (tail && a.k_new && lane < D / 8) {
                const int64_t src = (((int64_t)c.at.b * a.Hkv + h) * D) / 8 + lane;
                k_tok = __ldg(static_cast<const uint4*>(a.k_new) + src);
                v_tok = __ldg(static_cast<const uint4*>(a.v_new) + src);
            }
            ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars[warp][slot]), phase, abortp, status));
            if (!ok) break;
            const uint32_t st = ring + slot * SM::STAGE;
            if (tail) {
                // the sequence's last block: the new token's rows go into the tiles and, where it is this warp's to do, into the
                // cache; V rows behind it become zero (they may hold anything, and 0 x NaN is not 0)
                uint8_t* tile = ring_gen + slot * SM::STAGE;
                auto at = [&](int k, int chunk) { return (k >> 3) * upper + (chunk >> 3) * panel + (k & 7) * 128 + (((chunk & 7) ^ (k & 7)) << 4); };
                if (a.k_new && lane < D / 8) {
                    *reinterpret_cast<uint4*>(tile + at(valid - 1, lane)) = k_tok;
                    *reinterpret_cast<uint4*>(tile + SM::TILE + at(valid - 1, lane)) = v_tok;
                    const int64_t cell = gt == 0 ? token_row(a, c.at.b, h, c.at.len) : -1;
                    if (cell >= 0) {   // no fetch of this launch uses what lies there
                        const int64_t dst = cell * (D / 8) + lane;
                        static_cast<uint4*>(a.k_cache)[dst] = k_tok;
                        static_cast<uint4*>(a.v_cache)[dst] = v_tok;
                    }
                }
                for (int i = lane; i < (OWN_KEYS - valid) * (D / 8); i += 32)
                    *reinterpret_cast<uint4*>(tile + SM::TILE + at(valid + i / (D / 8), i % (D / 8))) = make_uint4(0, 0, 0, 0);
                fence_async_smem();   // before the next fetch into this stage
                __syncwarp();
            }
            float s[R][2][4];   // two sums over every other k-step: keys r (0, 1) and r + 8 (2, 3), heads 2j, 2j + 1
#pragma unroll
            for (int x = 0; x < R; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[x][0][e] = s[x][1][e] = 0.f;
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                uint32_t kf[4];
                ldsm(st + k_lane + (i >> 2) * panel + ((k_x ^ (2 * (i & 3))) << 4), kf);
#pragma unroll
                for (int x = 0; x < R; ++x) mma16816(s[x][i & 1], kf, qf[x][i][0], qf[x][i][1]);
            }
            uint32_t pf[R][2];   // P rounded to bf16: off by 2^-8 of its value at most; the sums stay in fp32
#pragma unroll
            for (int x = 0; x < R; ++x) {
                float z[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    z[e] = (s[x][0][e] + s[x][1][e]) * scale_log2;
                    if (tail && (e >> 1) * 8 + r >= valid) z[e] = -INFINITY;
                }
                float m0 = fmaxf(z[0], z[2]), m1 = fmaxf(z[1], z[3]);
                // the reference moves only when a head's maximum has grown by more than 2^8 (probabilities stay below 2^8)
                if (__any_sync(0xffffffffu, m0 > m[x][0] + 8.f || m1 > m[x][1] + 8.f)) {
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) {
                        m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, o));
                        m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, o));
                    }
                    m0 = fmaxf(m0, m[x][0]);
                    m1 = fmaxf(m1, m[x][1]);
                    const float f0 = m0 == -INFINITY ? 1.f : fast_ex2(m[x][0] - m0), f1 = m1 == -INFINITY ? 1.f : fast_ex2(m[x][1] - m1);
                    m[x][0] = m0;
                    m[x][1] = m1;
                    l[x][0] *= f0;
                    l[x][1] *= f1;
#pragma unroll
                    for (int i = 0; i < KS; ++i) {
                        acc[x][i][0] *= f0; acc[x][i][1] *= f1;
                        acc[x][i][2] *= f0; acc[x][i][3] *= f1;
                    }
                }
                const float r0 = m[x][0] == -INFINITY ? 0.f : m[x][0], r1 = m[x][1] == -INFINITY ? 0.f : m[x][1];
                const float p0 = fast_ex2(z[0] - r0), p1 = fast_ex2(z[1] - r1), p2 = fast_ex2(z[2] - r0), p3 = fast_ex2(z[3] - r1);
                l[x][0] += p0 + p2;
                l[x][1] += p1 + p3;
                pf[x][0] = transpose8x8(pack_bf16(p0, p1));   // keys 0..7
                pf[x][1] = transpose8x8(pack_bf16(p2, p3));   // keys 8..15
            }
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                uint32_t vf[4];
                ldsm_t(st + v_lane + (i >> 2) * panel + ((v_x ^ (2 * (i & 3))) << 4), vf);
#pragma unroll
                for (int x = 0; x < R; ++x) mma16816(acc[x][i], vf, pf[x][0], pf[x][1]);
            }
            // every lane has read the stage (its values are in registers): fetch the next block into it
            __syncwarp();
            if (fetching) fetch();
            if (++slot == NS) { slot = 0; phase ^= 1; }

            if (tail || (!WHOLE && c.left == 1)) {   // the segment ends
                const int64_t seg = (WHOLE ? 0 : (int64_t)w) + (int64_t)c.at.hh * a.B + c.at.b;
#pragma unroll
                for (int x = 0; x < R; ++x)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        float lt = l[x][y];
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) lt += __shfl_xor_sync(0xffffffffu, lt, o);
                        const int hd = x * 8 + 2 * j + y;
                        if (hd < heads) {
                            const float inv = 1.f / lt;
                            float* o = ws + p.own_o + (seg * p.g_rows + hd) * D + r;   // 8 lanes: 32 contiguous bytes
#pragma unroll
                            for (int i = 0; i < KS; ++i) {
                                o[16 * i] = acc[x][i][y] * inv;
                                o[16 * i + 8] = acc[x][i][2 + y] * inv;
                            }
                            if (r == 0) ws[p.own_lse + seg * p.g_rows + hd] = m[x][y] + log2f(lt);
                        }
                    }
                fresh = true;
            }
            if (next(c) == END) break;
        }
        if (!ok) {
            // leaving early: give copies already in flight a bounded time to land in this CTA's shared memory
            const long long t_off = clock64();
            while (clock64() - t_off < 2000000ll) {}
        }
    }
    if constexpr (WHOLE) {
        wait_for_previous();   // the prefix kernel's results

        // this warp's units: its own results (each lane reads what the warp has written) and the prefix segments.  A lane has
        // four features of a row, so D / 4 lanes share one
        __syncwarp();
        constexpr int LANES = D / 4, ROWS = 32 / LANES;
        const int c4 = lane % LANES;
        const float* part = static_cast<const float*>(a.ws);
        Cursor u;
        for (bool any = to_unit(u, w); any; any = to_unit(u, u.left + p.workers)) {
            const int h = u.at.hh / p.g_tiles, gt = u.at.hh - h * p.g_tiles, heads = min(p.g_rows, a.g - gt * p.g_rows);
            for (int x = lane / LANES; x < heads; x += ROWS) {
                const int row = u.at.b * a.g + gt * p.g_rows + x, mt = row / SHP_ROWS, rt = row - mt * SHP_ROWS;
                const PrefixSegments ps(a, p, h, mt);
                const int64_t own = (int64_t)u.left * p.g_rows + x;
                RowMerge m;
                m.add<1, 1>(1, part + p.own_lse + own, 0, part + p.own_o + own * D + c4 * 4, 0, 0);
                m.add<1, 8>(ps.n, part + p.p_lse + ps.first * SHP_ROWS + rt, (int64_t)p.m_tiles * SHP_ROWS,
                         part + p.p_o + ps.first * SHP_ROWS * D + ((int64_t)c4 * SHP_ROWS + rt) * 4, (int64_t)p.m_tiles * SHP_ROWS * D, 0);
                m.store<__nv_bfloat16, D>(a, (int64_t)u.at.b * a.Hq + h * a.g + gt * p.g_rows + x, c4);
            }
        }
    }
}

// ------------------------------------------------------------------ host side
static bool encode_rows(CUtensorMap* map, const void* p, int D, int64_t rows, int box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {64, (cuuint64_t)rows, (cuuint64_t)(D / 64)};
    const cuuint64_t strides[2] = {(cuuint64_t)D * 2, 128};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, (cuuint32_t)(D / 64)}, es[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(p), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// rows of the cache or pool as TMA sees it, and rows of a box
static int64_t own_rows(const SharedArgs& a) {
    return a.pg.table ? ((int64_t)a.pg.n_pages * a.Hkv << a.pg.log2_ps) : (int64_t)a.B * a.Hkv * a.cap;
}
static int own_box_rows(const SharedArgs& a) { return a.pg.table ? std::min(1 << a.pg.log2_ps, OWN_KEYS) : OWN_KEYS; }

// a box of fewer than 8 rows would start inside a swizzle group, a tile has 16 rows at least, and a row's number is 32 bits
bool shared_own_tma_fits(const SharedArgs& a) {
    const int64_t rows = own_rows(a);
    return encode_fn() && own_box_rows(a) >= 8 && rows >= OWN_KEYS && rows <= INT_MAX;
}

template <int D, int R, bool WHOLE>
static cudaError_t own_tma_t(const SharedArgs& a, const SharedPlan& p, bool behind, cudaStream_t st) {
    OwnMaps maps;
    const int64_t rows = own_rows(a);
    const int box_rows = own_box_rows(a);
    if (!encode_rows(&maps.k, a.k_cache, D, rows, box_rows) || !encode_rows(&maps.v, a.v_cache, D, rows, box_rows)) return cudaErrorInvalidValue;
    int* status = device_status_word();
    if (!status) return cudaErrorUnknown;
    constexpr int smem = OwnSmem<D>::TOTAL;
    return launch_behind(shared_own_tma_kernel<D, R, WHOLE>, dim3(OWN_CTAS), OWN_WARPS * 32, smem, st, behind, maps, a, p, status);
}

template <int D, int R>
static cudaError_t own_tma_r(const SharedArgs& a, const SharedPlan& p, bool behind, cudaStream_t st) {
    return p.whole ? own_tma_t<D, R, true>(a, p, behind, st) : own_tma_t<D, R, false>(a, p, behind, st);
}

cudaError_t launch_shared_own_tma(const SharedArgs& a, const SharedPlan& p, int D, bool behind, cudaStream_t st) {
    if (p.g_rows <= 8) return D == 64 ? own_tma_r<64, 1>(a, p, behind, st) : own_tma_r<128, 1>(a, p, behind, st);
    return D == 64 ? own_tma_r<64, 2>(a, p, behind, st) : own_tma_r<128, 2>(a, p, behind, st);
}

}  // namespace loma
