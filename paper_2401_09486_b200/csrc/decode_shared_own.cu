// The sequences' own entries in the shared-prefix decode step (bf16): a stream bound by HBM.
//
// A worker (one warp) walks its share of the blocks (see SharedPlan) with a ring of its own in shared memory: one TMA
// instruction fetches the 16 K rows of a block and one the V rows, NS - 1 blocks ahead and across the borders between
// sequences, so short sequences stream as well as long ones and no warp waits for another.  The g query heads of a kv head
// are the rows of a warp-level m16n8k16 product, so a K or V row is fetched once for all of them; K and V fragments come
// from the 128-byte-swizzled tiles with ldmatrix (V transposed on the way), without a bank conflict.  A block then takes
// about 200 instructions; four warps per SM turn them over faster than HBM delivers (44 bytes per SM and nanosecond, 190 ns
// for the 8 KB of a block), and 96 KB of rings leave room beside a CTA of the prefix kernel: the two run at the same time.
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

// D += A B, m16n8k16, rows 8..15 of A all zero (their results are not kept)
__device__ __forceinline__ void mma_lo(float (&d)[2], uint32_t a0, uint32_t a2, uint32_t b0, uint32_t b1) {
    [[maybe_unused]] float x, y;
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%10,%10};"
        : "+f"(d[0]), "+f"(d[1]), "=f"(x), "=f"(y)
        : "r"(a0), "r"(0u), "r"(a2), "r"(0u), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_full(float (&d)[2], float (&e)[2], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(e[0]), "+f"(e[1])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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

// R: rows of 8 query heads.
template <int D, int R>
__global__ void __launch_bounds__(OWN_WARPS * 32, R == 1 ? 3 : 2)
shared_own_tma_kernel(const __grid_constant__ OwnMaps maps, const SharedArgs a, const SharedPlan p, int* status) {
    using SM = OwnSmem<D>;
    constexpr int KS = D / 16, NT = D / 8, NS = SM::NS, PANELS = SM::PANELS;   // k-steps of the scores, output tiles of 8 features
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
    const SeqBlocks sb{a};
    const int per = sb.scan<OWN_WARPS>(scan, wsum, blockIdx.x == 0 ? reinterpret_cast<int64_t*>(static_cast<float*>(a.ws) + p.cum) : nullptr);
    const int64_t T = scan[(a.B + per - 1) / per] * a.Hkv * p.g_tiles;
    const int64_t W = min((int64_t)p.workers, T), w = (int64_t)warp * gridDim.x + blockIdx.x;   // neighbours on different SMs
    if (w < W) {
        const uint32_t ring = ((smem_u32(own_smem) + 1023u) & ~1023u) + warp * NS * SM::STAGE;
        uint8_t* ring_gen = own_smem + (ring - smem_u32(own_smem));
        volatile int* abortp = &abort_flag;
        const int64_t t0 = own_first(w, T, W);
        int left = (int)(own_first(w + 1, T, W) - t0);   // blocks still to be worked on
        int to_fetch = left;
        // two cursors over the same blocks: `c` is being worked on, `f` is being fetched
        SeqBlocks::Cursor c = sb.find(t0, scan, per), f = c;
        // a box holds its rows panel by panel: where panel 1 and rows 8..15 of a tile lie
        const int boxes = a.pg.table ? max(1, OWN_KEYS >> a.pg.log2_ps) : 1, box_rows = OWN_KEYS / boxes;
        const uint32_t panel = box_rows * 128, upper = boxes == 1 ? 1024 : 1024 * PANELS;
        // row of the fetch cursor's block (this lane's box of it), from the top of the cache or pool; the table entry is read
        // here, one block before it is used
        int64_t base_f = 0;              // contiguous: first row of the fetch cursor's (sequence, kv head)
        const int32_t* table_f = nullptr;
        int h_f = 0;
        auto enter_f = [&]() {
            h_f = f.hh / p.g_tiles;
            base_f = ((int64_t)f.b * a.Hkv + h_f) * a.cap;
            table_f = a.pg.table + (int64_t)f.b * a.pg.max_pages;
        };
        auto row_f = [&]() -> int {
            if (!a.pg.table) return (int)base_f + f.blk * OWN_KEYS;
            const int key = f.blk * OWN_KEYS + (lane < boxes ? lane : 0) * box_rows;
            const int page = min(max(__ldg(table_f + (min(key, f.len) >> a.pg.log2_ps)), 0), a.pg.n_pages - 1);
            return ((page * a.Hkv + h_f) << a.pg.log2_ps) + (key & ((1 << a.pg.log2_ps) - 1));   // the pool has at most 2^31 rows
        };
        enter_f();
        int next_row = row_f(), slot_f = 0;
        auto fetch = [&]() {
            const uint32_t bar = smem_u32(&bars[warp][slot_f]), dst = ring + slot_f * SM::STAGE;
            if (lane == 0) mbar_expect_tx(bar, SM::STAGE);
            __syncwarp();
            if (lane < boxes) {
                tma_rows(dst + lane * 1024 * PANELS, &maps.k, bar, next_row);
                tma_rows(dst + SM::TILE + lane * 1024 * PANELS, &maps.v, bar, next_row);
            }
            slot_f = slot_f + 1 == NS ? 0 : slot_f + 1;
            if (--to_fetch > 0) {
                if (sb.advance(f)) enter_f();
                next_row = row_f();
            }
        };
        for (int i = 0; i < NS && to_fetch > 0; ++i) fetch();

        // ldmatrix addresses.  K (score operand B: k = features, n = keys): matrices (keys 0-7 | 8-15) x (features 16 kk .. +7 |
        // +8 .. +15); V (operand B: k = keys, n = features, transposed): keys 0-7, 8-15 of tiles 2 nn and 2 nn + 1.  A row's
        // 16-byte chunks are exchanged by the swizzle: chunk x of row k lies at x ^ (k mod 8).
        const int mi = lane >> 3, mr = lane & 7;
        const uint32_t k_lane = (mi >> 1) * upper + mr * 128, k_x = (mi & 1) ^ mr;
        const uint32_t v_lane = (mi & 1) * upper + mr * 128 + SM::TILE, v_x = (mi >> 1) ^ mr;

        const float scale_log2 = a.scale * 1.4426950408889634f;
        const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q);
        float* ws = static_cast<float*>(a.ws);
        uint32_t qf[R][KS][2];
        float m[R], l[R], acc[R][NT][2];
        int slot = 0, h = 0, gt = 0, heads = 0;
        uint32_t phase = 0;
        bool fresh = true, ok = true;
        for (; left > 0; --left) {
            if (fresh) {   // a new segment: this triple's query heads (operand A: row = head, k = features 2j, 2j+1 and + 8)
                h = c.hh / p.g_tiles;
                gt = c.hh - h * p.g_tiles;
                heads = min(p.g_rows, a.g - gt * p.g_rows);
#pragma unroll
                for (int x = 0; x < R; ++x) {
                    const int hd = x * 8 + r;
                    const uint32_t* qp = reinterpret_cast<const uint32_t*>(q + ((int64_t)c.b * a.Hq + h * a.g + gt * p.g_rows + min(hd, heads - 1)) * D);
#pragma unroll
                    for (int i = 0; i < KS; ++i) {
                        qf[x][i][0] = hd < heads ? __ldg(qp + 8 * i + j) : 0u;
                        qf[x][i][1] = hd < heads ? __ldg(qp + 8 * i + j + 4) : 0u;
                    }
                    m[x] = -INFINITY;
                    l[x] = 0.f;
#pragma unroll
                    for (int n = 0; n < NT; ++n) acc[x][n][0] = acc[x][n][1] = 0.f;
                }
                fresh = false;
            }
            const int valid = c.len + 1 - c.blk * OWN_KEYS;   // keys from this block on, the new token the last of them
            const bool tail = valid <= OWN_KEYS;
            ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars[warp][slot]), phase, abortp, status));
            if (!ok) break;
            const uint32_t st = ring + slot * SM::STAGE;
            if (tail) {
                // the sequence's last block: the new token's rows go into the tiles and, where it is this warp's to do, into the
                // cache; V rows behind it become zero (they may hold anything, and 0 x NaN is not 0)
                uint8_t* tile = ring_gen + slot * SM::STAGE;
                const int row = valid - 1;
                auto at = [&](int k, int chunk) { return (k >> 3) * upper + (chunk >> 3) * panel + (k & 7) * 128 + (((chunk & 7) ^ (k & 7)) << 4); };
                if (a.k_new && lane < D / 8) {
                    const int64_t src = (((int64_t)c.b * a.Hkv + h) * D) / 8 + lane;
                    const uint4 kv = __ldg(static_cast<const uint4*>(a.k_new) + src), vv = __ldg(static_cast<const uint4*>(a.v_new) + src);
                    *reinterpret_cast<uint4*>(tile + at(row, lane)) = kv;
                    *reinterpret_cast<uint4*>(tile + SM::TILE + at(row, lane)) = vv;
                    if (gt == 0) {   // no fetch of this launch uses what lies there
                        const int64_t dst = own_row(a, c.b, h, c.len) * (D / 8) + lane;
                        static_cast<uint4*>(a.k_cache)[dst] = kv;
                        static_cast<uint4*>(a.v_cache)[dst] = vv;
                    }
                }
                for (int i = lane; i < (OWN_KEYS - valid) * (D / 8); i += 32)
                    *reinterpret_cast<uint4*>(tile + SM::TILE + at(valid + i / (D / 8), i % (D / 8))) = make_uint4(0, 0, 0, 0);
                fence_async_smem();   // before the next fetch into this stage
                __syncwarp();
            }
            float s[R][2][2];   // head x*8 + r, keys n*8 + 2j, +1
#pragma unroll
            for (int x = 0; x < R; ++x)
#pragma unroll
                for (int n = 0; n < 2; ++n) s[x][n][0] = s[x][n][1] = 0.f;
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                uint32_t kf[4];
                ldsm(st + k_lane + (i >> 2) * panel + ((k_x ^ (2 * (i & 3))) << 4), kf);
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    if constexpr (R == 1) mma_lo(s[0][n], qf[0][i][0], qf[0][i][1], kf[2 * n], kf[2 * n + 1]);
                    else mma_full(s[0][n], s[1][n], qf[0][i][0], qf[1][i][0], qf[0][i][1], qf[1][i][1], kf[2 * n], kf[2 * n + 1]);
                }
            }
            uint32_t pf[R][2];   // P rounded to bf16: off by 2^-8 of its value at most; the sums stay in fp32
#pragma unroll
            for (int x = 0; x < R; ++x) {
                if (tail) {
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if (n * 8 + 2 * j + e >= valid) s[x][n][e] = -INFINITY;
                }
                float mx = fmaxf(fmaxf(s[x][0][0], s[x][0][1]), fmaxf(s[x][1][0], s[x][1][1])) * scale_log2;
                // the reference moves only when a row's maximum has grown by more than 2^8 (probabilities stay below 2^8)
                if (__any_sync(0xffffffffu, mx > m[x] + 8.f)) {
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                    const float m_new = fmaxf(m[x], mx), alpha = m_new == -INFINITY ? 1.f : fast_ex2(m[x] - m_new);
                    m[x] = m_new;
                    l[x] *= alpha;
#pragma unroll
                    for (int n = 0; n < NT; ++n) { acc[x][n][0] *= alpha; acc[x][n][1] *= alpha; }
                }
                const float ref = m[x] == -INFINITY ? 0.f : -m[x];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const float p0 = fast_ex2(fmaf(s[x][n][0], scale_log2, ref)), p1 = fast_ex2(fmaf(s[x][n][1], scale_log2, ref));
                    l[x] += p0 + p1;
                    pf[x][n] = pack_bf16(p0, p1);
                }
            }
#pragma unroll
            for (int nn = 0; nn < NT / 2; ++nn) {
                uint32_t vf[4];
                ldsm_t(st + v_lane + (nn >> 2) * panel + ((v_x ^ (2 * (nn & 3))) << 4), vf);
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    if constexpr (R == 1) mma_lo(acc[0][2 * nn + n], pf[0][0], pf[0][1], vf[2 * n], vf[2 * n + 1]);
                    else mma_full(acc[0][2 * nn + n], acc[1][2 * nn + n], pf[0][0], pf[1][0], pf[0][1], pf[1][1], vf[2 * n], vf[2 * n + 1]);
                }
            }
            // every lane has read the stage (its values are in registers): fetch the next block into it
            __syncwarp();
            if (to_fetch > 0) fetch();
            if (++slot == NS) { slot = 0; phase ^= 1; }

            if (tail || left == 1) {   // the segment ends
                const int64_t seg = w + (int64_t)c.hh * a.B + c.b;
#pragma unroll
                for (int x = 0; x < R; ++x) {
                    float lt = l[x] + __shfl_xor_sync(0xffffffffu, l[x], 1);
                    lt += __shfl_xor_sync(0xffffffffu, lt, 2);
                    const int hd = x * 8 + r;
                    if (hd < heads) {
                        const float inv = 1.f / lt;
                        float2* o = reinterpret_cast<float2*>(ws + p.own_o + (seg * p.g_rows + hd) * D) + j;
#pragma unroll
                        for (int n = 0; n < NT; ++n) o[4 * n] = make_float2(acc[x][n][0] * inv, acc[x][n][1] * inv);
                        if (j == 0) ws[p.own_lse + seg * p.g_rows + hd] = m[x] + log2f(lt);
                    }
                }
                fresh = true;
            }
            if (left > 1) sb.advance(c);
        }
        if (!ok) {
            // leaving early: give copies already in flight a bounded time to land in this CTA's shared memory
            const long long t_off = clock64();
            while (clock64() - t_off < 2000000ll) {}
        }
    }
    wait_for_previous();   // the merge needs the prefix kernel's results too: this kernel ends after it
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

template <int D, int R>
static cudaError_t own_tma_t(const SharedArgs& a, const SharedPlan& p, bool behind, cudaStream_t st) {
    OwnMaps maps;
    const int ps = 1 << a.pg.log2_ps;
    const int64_t rows = a.pg.table ? ((int64_t)a.pg.n_pages * a.Hkv << a.pg.log2_ps) : (int64_t)a.B * a.Hkv * a.cap;
    const int box_rows = a.pg.table ? std::min(ps, OWN_KEYS) : OWN_KEYS;
    // a box of fewer than 8 rows would start inside a swizzle group; a tile has 16 rows at least
    if (box_rows < 8 || rows < OWN_KEYS || rows > INT_MAX || !encode_rows(&maps.k, a.k_cache, D, rows, box_rows) ||
        !encode_rows(&maps.v, a.v_cache, D, rows, box_rows))
        return cudaErrorNotSupported;
    int* status = device_status_word();
    if (!status) return cudaErrorUnknown;
    constexpr int smem = OwnSmem<D>::TOTAL;
    return launch_behind(shared_own_tma_kernel<D, R>, dim3(OWN_CTAS), OWN_WARPS * 32, smem, st, behind, maps, a, p, status);
}

cudaError_t launch_shared_own_tma(const SharedArgs& a, const SharedPlan& p, int D, bool behind, cudaStream_t st) {
    if (p.g_rows <= 8) return D == 64 ? own_tma_t<64, 1>(a, p, behind, st) : own_tma_t<128, 1>(a, p, behind, st);
    return D == 64 ? own_tma_t<64, 2>(a, p, behind, st) : own_tma_t<128, 2>(a, p, behind, st);
}

}  // namespace loma
