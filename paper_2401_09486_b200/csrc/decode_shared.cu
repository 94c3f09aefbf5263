// Decode attention for a batch whose sequences share a long prefix (loma_decode_attn_shared and its paged form).
//
// Query head hq of sequence b sees the prefix's keys of kv head hq div g (g = Hq / Hkv), then the sequence's own cache
// and its new token, under one softmax.  A softmax over a union of key sets is the mean of the softmaxes over the parts
// with weights 2^(lse_i - max), so the parts are computed where they are cheap and joined at the end:
//
//   prefix   all B g query rows of a kv head against the same K and V: a matrix product, 128 rows at a time, that reads
//            the prefix once for the batch instead of once per sequence (bf16: tcgen05, decode_shared_tc.cu; fp32, page
//            sizes below 8 and own caches of fewer than 16 rows in all: shared_prefix_simt_kernel)
//   own      one query row per head of a group against rows nobody else reads: a stream bound by HBM, cut into equal
//            shares of keys whatever the lengths (SharedPlan).  bf16: decode_shared_own.cu; else, and wherever the
//            prefix stays off the tensor cores: shared_own_stream_kernel
//   merge    one thread per query row and four features adds the parts in a fixed order (results repeat bit for bit)
//
// The own and the prefix kernel share no result, so the second starts beside the first (programmatic dependent launch) and
// an HBM-bound stream runs under a tensor-bound product; the merge waits for both.
#include <math.h>

#include "decode_shared.cuh"

namespace loma {

__device__ __forceinline__ uint4 ld_stream16(const void* p) {
    uint4 r;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

__device__ __forceinline__ int64_t prefix_row(const SharedArgs& a, int h, int j) {
    if (!a.prefix_table) return (int64_t)h * a.prefix_cap + j;
    const int page = min(max(__ldg(a.prefix_table + (j >> a.pg.log2_ps)), 0), a.pg.n_pages - 1);
    return ((((int64_t)page * a.Hkv + h) << a.pg.log2_ps) + (j & ((1 << a.pg.log2_ps) - 1)));
}

// Sums over the lanes that differ in bit O, each keeping one half of the M values
template <int M, int O>
__device__ __forceinline__ void halve(float* s, int lane) {
    const bool up = lane & O;
#pragma unroll
    for (int i = 0; i < M / 2; ++i) {
        const float lo = s[i], hi = s[i + M / 2];
        s[i] = (up ? hi : lo) + __shfl_xor_sync(0xffffffffu, up ? lo : hi, O);
    }
}

// ... over the lanes that differ in any bit of 2 O - 1: value li * M / (2 O) + v of the M, or each value in 2 O / M lanes
template <int M, int O>
__device__ __forceinline__ void spread_sum(float* s, int lane) {
    if constexpr (M > 1) halve<M, O>(s, lane);
    else s[0] += __shfl_xor_sync(0xffffffffu, s[0], O);
    if constexpr (O > 1) spread_sum<(M > 1 ? M / 2 : 1), O / 2>(s, lane);
}

// ------------------------------------------------------------------ own cache on CUDA cores (fp32, second opinion)
// A worker is a warp, as in shared_own_tma_kernel.  The lanes that share a row hold 16 bytes of it each; G heads of the
// group at a time, so a row is loaded once for them.  The G x NL partial scores of a lane are added up over those lanes with
// the results spread over them (16 shuffles for 16 scores instead of 80), so a lane keeps the maximum and the sum of one head
// and takes one exponential where it would take 16; probabilities go back to all lanes through the warp's shared memory.
// Loads in flight come from 16 warps per SM.  With the merge, fp32 B60 Hq16 Hkv2, lengths up to 300: 20.8 us (32.2 with every score
// in every lane).
template <typename T, int D, int G>
__global__ void __launch_bounds__(OWN_WARPS * 32, 4)
shared_own_stream_kernel(const SharedArgs a, const SharedPlan p) {
    using V = Vec16<T>;
    constexpr int N = V::N, LPK = D / N, KPL = 32 / LPK, NL_MOST = G == 4 ? 4 : 8, NL = OWN_KEYS / KPL < NL_MOST ? OWN_KEYS / KPL : NL_MOST;
    // scores of a lane's keys and heads; how many a lane keeps, in how many lanes each is; lanes of a head
    constexpr int M = G * NL, KEEP = M > LPK ? M / LPK : 1, DUP = LPK > M ? LPK / M : 1, LH = LPK / G;
    __shared__ __align__(16) float s_prob[OWN_WARPS][KPL][M];
    __shared__ int64_t scan[SeqBlocks::MAX_GROUPS + 1];
    __shared__ int64_t wsum[OWN_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / LPK, li = lane % LPK;
    float* ws = static_cast<float*>(a.ws);
    let_next_start();
    const SeqBlocks sb{a};
    const int per = sb.scan<OWN_WARPS>(scan, wsum, blockIdx.x == 0 ? reinterpret_cast<int64_t*>(ws + p.cum) : nullptr);
    const int64_t total = scan[(a.B + per - 1) / per] * a.Hkv * p.g_tiles;
    const int64_t W = own_workers(total, p.workers), w = (int64_t)warp * gridDim.x + blockIdx.x;
    if (w < W) {
        int64_t t = first_block(w, total, W);
        const int64_t t_end = first_block(w + 1, total, W);
        SeqBlocks::Cursor c = sb.find(t, scan, per);
        const float scale_log2 = a.scale * 1.4426950408889634f;
        float q[G][N], acc[G][N], m = -INFINITY, l = 0.f;   // m, l: of head li / LH, this lane's share of its keys
        bool fresh = true;
        for (; t < t_end; ++t) {
            const int h = c.hh / p.g_tiles, gt = c.hh - h * p.g_tiles, heads = min(G, a.g - gt * G), len = c.len;
            const T* kn = a.k_new ? static_cast<const T*>(a.k_new) + ((int64_t)c.b * a.Hkv + h) * D : nullptr;
            const T* vn = a.v_new ? static_cast<const T*>(a.v_new) + ((int64_t)c.b * a.Hkv + h) * D : nullptr;
            if (fresh) {
#pragma unroll
                for (int x = 0; x < G; ++x) {
                    const T* qp = static_cast<const T*>(a.q) + ((int64_t)c.b * a.Hq + h * a.g + gt * G + min(x, heads - 1)) * D;
                    V::unpack(__ldg(reinterpret_cast<const uint4*>(qp) + li), q[x]);
#pragma unroll
                    for (int e = 0; e < N; ++e) { q[x][e] *= scale_log2; acc[x][e] = 0.f; }
                }
                m = -INFINITY;
                l = 0.f;
                fresh = false;
            }
#pragma unroll 1
            for (int j0 = c.blk * OWN_KEYS; j0 < min(len + 1, (c.blk + 1) * OWN_KEYS); j0 += NL * KPL) {
                uint4 kr[NL], vr[NL];
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    const int key = min(j0 + i * KPL + sub, len);   // no row of another sequence is ever read
                    const int64_t row = key == len && kn ? 0 : own_row(a, c.b, h, key) * D;
                    kr[i] = ld_stream16((key == len && kn ? kn : static_cast<const T*>(a.k_cache) + row) + li * N);
                    vr[i] = ld_stream16((key == len && vn ? vn : static_cast<const T*>(a.v_cache) + row) + li * N);
                }
                float s[M];
#pragma unroll
                for (int i = 0; i < NL; ++i) {
                    float kf[N];
                    V::unpack(kr[i], kf);
#pragma unroll
                    for (int x = 0; x < G; ++x) {
                        s[x * NL + i] = 0.f;
#pragma unroll
                        for (int e = 0; e < N; ++e) s[x * NL + i] = fmaf(q[x][e], kf[e], s[x * NL + i]);
                    }
                }
                spread_sum<M, LPK / 2>(s, lane);
                float top = -INFINITY;
#pragma unroll
                for (int v = 0; v < KEEP; ++v) {
                    if (j0 + (li % LH / DUP * KEEP + v) * KPL + sub > len) s[v] = -INFINITY;
                    top = fmaxf(top, s[v]);
                }
#pragma unroll
                for (int o = DUP; o < LH; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
#pragma unroll
                for (int o = LPK; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                // the reference moves only when a head's maximum has grown by more than 2^8 (probabilities stay below 2^8)
                if (__any_sync(0xffffffffu, top > m + 8.f)) {
                    const float m_new = fmaxf(m, top), alpha = m_new == -INFINITY ? 1.f : exp2f(m - m_new);
                    m = m_new;
                    l *= alpha;
#pragma unroll
                    for (int x = 0; x < G; ++x) {
                        const float f = __shfl_sync(0xffffffffu, alpha, x * LH);
#pragma unroll
                        for (int e = 0; e < N; ++e) acc[x][e] *= f;
                    }
                }
                const float ref = m == -INFINITY ? 0.f : m;
                __syncwarp();   // the last round's probabilities have been read
#pragma unroll
                for (int v = 0; v < KEEP; ++v) {
                    const float pr = exp2f(s[v] - ref);
                    l += pr;
                    if (li % DUP == 0) s_prob[warp][sub][li / DUP * KEEP + v] = pr;
                }
                __syncwarp();
                if (j0 + NL * KPL > len + 1) {   // repeated keys have no weight, but 0 x inf is not 0
#pragma unroll
                    for (int i = 0; i < NL; ++i)
                        if (j0 + i * KPL + sub > len) vr[i] = make_uint4(0, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < NL; i += 4) {
                    float4 pr[G];
#pragma unroll
                    for (int x = 0; x < G; ++x) pr[x] = *reinterpret_cast<const float4*>(&s_prob[warp][sub][x * NL + i]);
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        float vf[N];
                        V::unpack(vr[i + y], vf);
#pragma unroll
                        for (int x = 0; x < G; ++x) {
                            const float f = y == 0 ? pr[x].x : y == 1 ? pr[x].y : y == 2 ? pr[x].z : pr[x].w;
#pragma unroll
                            for (int e = 0; e < N; ++e) acc[x][e] = fmaf(f, vf[e], acc[x][e]);
                        }
                    }
                }
            }
            const bool tail = c.blk == len / OWN_KEYS;
            if (tail || t + 1 == t_end) {
                const int64_t seg = w + (int64_t)c.hh * a.B + c.b;
#pragma unroll
                for (int o = DUP; o < LH; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
#pragma unroll
                for (int o = LPK; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
                const int mine = li / LH;
                if (lane < LPK && li % LH == 0 && mine < heads) ws[p.own_lse + seg * p.g_rows + mine] = m + log2f(l);
#pragma unroll
                for (int x = 0; x < G; ++x) {
                    const float inv = 1.f / __shfl_sync(0xffffffffu, l, x * LH);
#pragma unroll
                    for (int e = 0; e < N; ++e)
#pragma unroll
                        for (int o = 16; o >= LPK; o >>= 1) acc[x][e] += __shfl_xor_sync(0xffffffffu, acc[x][e], o);
                    if (x < heads && lane < LPK) {
                        float4* o = reinterpret_cast<float4*>(ws + p.own_o + (seg * p.g_rows + x) * D + li * N);
#pragma unroll
                        for (int e = 0; e < N; e += 4) o[e / 4] = make_float4(acc[x][e] * inv, acc[x][e + 1] * inv, acc[x][e + 2] * inv, acc[x][e + 3] * inv);
                    }
                }
                // the new token's K and V go to entry len (read by nobody in this launch)
                const int64_t cell = tail && kn && gt == 0 && lane < LPK ? token_row(a, c.b, h, len) : -1;
                if (cell >= 0) {
                    const int64_t row = cell * D;
                    reinterpret_cast<uint4*>(static_cast<T*>(a.k_cache) + row)[lane] = __ldg(reinterpret_cast<const uint4*>(kn) + lane);
                    reinterpret_cast<uint4*>(static_cast<T*>(a.v_cache) + row)[lane] = __ldg(reinterpret_cast<const uint4*>(vn) + lane);
                }
                fresh = true;
            }
            if (t + 1 < t_end) sb.advance(c);
        }
    }
    if (blockIdx.x == 0) wait_for_previous();   // this kernel ends after the prefix kernel where it is launched behind it
}

// ------------------------------------------------------------------ prefix on CUDA cores (fp32, small pages, second opinion)
// RT query rows against 32 keys at a time, all in fp32, RT / 8 rows to a warp from the scores to the outputs: between two
// barriers (one per block, K and V are double buffered) a warp waits for nobody.
//   scores   a lane has 4 keys x up to 4 rows and every 2nd or 4th group of 4 features; the lanes that share a tile then halve
//            it between them while they add their sums.  That takes 12 shared-memory wavefronts for 32 two-wide FMAs a lane,
//            fewer than the FMAs take; a tile of 2 keys x 4 rows needed twice as many.
//   outputs  a lane has D / 32 features of all of the warp's rows; probabilities come through the warp's own shared memory.
// Bound by fp32 FMA for many rows, by the latency of a block's steps for few.  Measured: 480 query rows, 2 kv heads, D128, prefix 4000:
// 67.8 us, FMA pipe active 53 % of the cycles, shared memory 57 %.  Query row m of kv head h is head h g + m mod g of sequence m / g.
constexpr int SIMT_THREADS = 256;

template <int D, int RT>
struct SimtSmem {   // in floats
    static constexpr int K_TILE = SIMT_K * (D + 4), TILE = K_TILE + SIMT_K * D;   // K rows padded: lanes read 8 rows at a time
    static constexpr int Q = 0, KV = Q + RT * (D + 4), P = KV + 2 * TILE, A = P + RT * SIMT_K, FLOATS = A + RT;
};

template <typename T, int D, int RT>
__global__ void __launch_bounds__(SIMT_THREADS, 2)
shared_prefix_simt_kernel(const SharedArgs a, const SharedPlan p) {
    using V = Vec16<T>;
    using SM = SimtSmem<D, RT>;
    static_assert(SIMT_K == 32, "8 lanes x 4 keys");
    constexpr int N = V::N, LPK = D / N, DC = D / 32, PASSES = SIMT_K * LPK / SIMT_THREADS;
    constexpr int WR = RT / 8, TR = WR < 4 ? WR : 4, RL = WR / TR, DL = 4 / RL;   // rows of a warp and a lane; lanes over rows, features
    constexpr int M = TR * 4 / DL, KR = M < 4 ? 1 : M / 4, KK = M < 4 ? M : 4;    // scores a lane keeps: KR rows x KK keys
    constexpr bool ASYNC = sizeof(T) == 4;                                        // bf16 is widened on its way, through registers
    extern __shared__ __align__(16) float sm[];
    let_next_start();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rows = a.B * a.g;
    const float scale_log2 = a.scale * 1.4426950408889634f;
    const int worker = blockIdx.x / p.m_tiles, mt = blockIdx.x - worker * p.m_tiles;
    const int64_t blocks = (int64_t)a.Hkv * p.p_blocks;
    int64_t t = first_block(worker, blocks, p.p_workers);
    const int64_t t_end = first_block(worker + 1, blocks, p.p_workers);
    const int r_in = blockIdx.y * RT, row0 = mt * SHP_ROWS + r_in;   // RT rows of the tile per blockIdx.y
    if (row0 >= rows) t = t_end;
    const int kl = lane & 7, rl = (lane >> 3) % RL, dl = (lane >> 3) / RL;        // scores: keys kl + 8 w, rows rl * TR + u
    const int base = DL == 2 ? dl * M : (dl >> 1) * 2 * M + (dl & 1) * M;         // the first (row, key) that the lane keeps
    const int row_k = warp * WR + rl * TR + base / 4, col_k = base % 4;
    const float* q_at = sm + SM::Q + (warp * WR + rl * TR) * (D + 4) + 4 * dl;
    float* p_warp = sm + SM::P + warp * WR * SIMT_K;

    // the fetch is a block ahead, and the rows' places (a table entry away) are known another block earlier
    int h_f = 0, blk_f = 0;
    int64_t row_f[PASSES];
    uint4 kv[ASYNC ? 1 : 2][ASYNC ? 1 : PASSES];
    auto find_rows = [&]() {
#pragma unroll
        for (int i = 0; i < PASSES; ++i)   // keys past the end repeat the last one
            row_f[i] = prefix_row(a, h_f, min(blk_f * SIMT_K + (tid + i * SIMT_THREADS) / LPK, a.prefix_len - 1)) * D;
    };
    auto fetch = [&](int buf, bool more) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int r = (tid + i * SIMT_THREADS) / LPK, c = (tid + i * SIMT_THREADS) % LPK;
            const T* kp = static_cast<const T*>(a.k_prefix) + row_f[i] + c * N;
            const T* vp = static_cast<const T*>(a.v_prefix) + row_f[i] + c * N;
            const bool in = blk_f * SIMT_K + r < a.prefix_len;   // a repeated key's values are zero: its weight is, and 0 x inf is not 0
            if constexpr (ASYNC) {
                float* tile = sm + SM::KV + buf * SM::TILE;
                cp_async16((uint32_t)__cvta_generic_to_shared(tile + r * (D + 4) + c * N), kp);
                cp_async16_or_zero((uint32_t)__cvta_generic_to_shared(tile + SM::K_TILE + r * D + c * N), vp, in);
            } else {
                kv[0][i] = __ldg(reinterpret_cast<const uint4*>(kp));
                kv[1][i] = in ? __ldg(reinterpret_cast<const uint4*>(vp)) : make_uint4(0, 0, 0, 0);
            }
        }
        if (++blk_f == p.p_blocks) { blk_f = 0; ++h_f; }
        if (more) find_rows();
    };
    int buf = 0, h = 0, blk = 0;
    if (t < t_end) {
        h = h_f = (int)(t / p.p_blocks);
        blk = blk_f = (int)(t - (int64_t)h * p.p_blocks);
        find_rows();
        fetch(0, t + 1 < t_end);
    }
    while (t < t_end) {                                   // segments of the CTA's share
        const int64_t seg = (int64_t)(worker + h) * p.m_tiles + mt;
        __syncthreads();
#pragma unroll 4
        for (int idx = tid; idx < RT * LPK; idx += SIMT_THREADS) {
            const int r = idx / LPK, c = idx - r * LPK, m = min(row0 + r, rows - 1);
            const T* qp = static_cast<const T*>(a.q) + ((int64_t)(m / a.g) * a.Hq + h * a.g + m % a.g) * D;
            float f[N];
            V::unpack(__ldg(reinterpret_cast<const uint4*>(qp) + c), f);
#pragma unroll
            for (int e = 0; e < N; ++e) sm[SM::Q + r * (D + 4) + c * N + e] = f[e] * scale_log2;
        }
        uint64_t acc[WR][DC / 2];
        float mx[KR], l[KR];
#pragma unroll
        for (int u = 0; u < WR; ++u)
#pragma unroll
            for (int c = 0; c < DC / 2; ++c) acc[u][c] = 0;
#pragma unroll
        for (int u = 0; u < KR; ++u) { mx[u] = -INFINITY; l[u] = 0.f; }
        for (; blk < p.p_blocks && t < t_end; ++blk, buf ^= 1) {
            float* k_tile = sm + SM::KV + buf * SM::TILE;
            float* v_tile = k_tile + SM::K_TILE;
            if constexpr (ASYNC) {
                asm volatile("cp.async.wait_all;" ::: "memory");
            } else {
#pragma unroll
                for (int i = 0; i < PASSES; ++i) {
                    const int r = (tid + i * SIMT_THREADS) / LPK, c = (tid + i * SIMT_THREADS) % LPK;
                    float f[N];
                    V::unpack(kv[0][i], f);
#pragma unroll
                    for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(k_tile + r * (D + 4) + c * N + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
                    V::unpack(kv[1][i], f);
#pragma unroll
                    for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(v_tile + r * D + c * N + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
                }
            }
            __syncthreads();                              // the tile is there, and the other one has been read
            if (++t < t_end) fetch(buf ^ 1, t + 1 < t_end);
            uint64_t s2[TR][4];                           // two-wide FMA: sums over even and odd features side by side
#pragma unroll
            for (int u = 0; u < TR; ++u)
#pragma unroll
                for (int w = 0; w < 4; ++w) s2[u][w] = 0;
            const float* k_at = k_tile + kl * (D + 4) + 4 * dl;
#pragma unroll 2
            for (int d = 0; d < D; d += 4 * DL) {
                ulonglong2 qv[TR];
#pragma unroll
                for (int u = 0; u < TR; ++u) qv[u] = *reinterpret_cast<const ulonglong2*>(q_at + u * (D + 4) + d);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const ulonglong2 kf = *reinterpret_cast<const ulonglong2*>(k_at + 8 * w * (D + 4) + d);
#pragma unroll
                    for (int u = 0; u < TR; ++u) s2[u][w] = fma2(qv[u].y, kf.y, fma2(qv[u].x, kf.x, s2[u][w]));
                }
            }
            float s[TR * 4];
#pragma unroll
            for (int u = 0; u < TR; ++u)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    float lo, hi;
                    unpack2(s2[u][w], lo, hi);
                    s[4 * u + w] = lo + hi;
                }
            halve<TR * 4, 16>(s, lane);
            if constexpr (DL == 4) halve<TR * 2, 8>(s, lane);
            // the reference moves only when a row's maximum has grown by more than 2^8 (probabilities stay below 2^8)
            float top[KR];
            bool grown = false;
#pragma unroll
            for (int u = 0; u < KR; ++u) {
                top[u] = -INFINITY;
#pragma unroll
                for (int w = 0; w < KK; ++w) {
                    float& x = s[u * KK + w];
                    if (blk * SIMT_K + kl + 8 * (col_k + w) >= a.prefix_len) x = -INFINITY;
                    top[u] = fmaxf(top[u], x);
                }
#pragma unroll
                for (int o = 1; o < (KK < 4 ? 16 : 8); o <<= 1) top[u] = fmaxf(top[u], __shfl_xor_sync(0xffffffffu, top[u], o));
                grown |= top[u] > mx[u] + 8.f;
            }
            if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
                for (int u = 0; u < KR; ++u) {
                    const float m_new = fmaxf(mx[u], top[u]), alpha = m_new == -INFINITY ? 1.f : exp2f(mx[u] - m_new);
                    mx[u] = m_new;
                    l[u] *= alpha;
                    if (kl == 0 && col_k == 0) sm[SM::A + row_k + u] = alpha;
                }
                __syncwarp();
#pragma unroll
                for (int u = 0; u < WR; ++u) {
                    const float alpha = sm[SM::A + warp * WR + u];
#pragma unroll
                    for (int c = 0; c < DC / 2; ++c) acc[u][c] = fma2(acc[u][c], pack2(alpha, alpha), 0);
                }
            }
#pragma unroll
            for (int u = 0; u < KR; ++u) {
                const float ref = mx[u] == -INFINITY ? 0.f : mx[u];
#pragma unroll
                for (int w = 0; w < KK; ++w) {
                    s[u * KK + w] = exp2f(s[u * KK + w] - ref);
                    l[u] += s[u * KK + w];
                }
                float* dst = sm + SM::P + (row_k + u) * SIMT_K + kl * 4 + col_k;      // column 4 kl + w: key kl + 8 w
                if constexpr (KK == 4) *reinterpret_cast<float4*>(dst) = make_float4(s[u * 4], s[u * 4 + 1], s[u * 4 + 2], s[u * 4 + 3]);
                else *reinterpret_cast<float2*>(dst) = make_float2(s[u * KK], s[u * KK + 1]);
            }
            __syncwarp();
#pragma unroll 2
            for (int k = 0; k < 8; ++k) {
                float4 pv[WR];
#pragma unroll
                for (int u = 0; u < WR; ++u) pv[u] = *reinterpret_cast<const float4*>(p_warp + u * SIMT_K + 4 * k);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float* vp = v_tile + (k + 8 * w) * D + lane * DC;
                    uint64_t vv[DC / 2];
                    if constexpr (DC == 4) {
                        const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(vp);
                        vv[0] = x.x;
                        vv[DC / 2 - 1] = x.y;
                    } else {
                        vv[0] = *reinterpret_cast<const uint64_t*>(vp);
                    }
#pragma unroll
                    for (int u = 0; u < WR; ++u) {
                        const float pr = w == 0 ? pv[u].x : w == 1 ? pv[u].y : w == 2 ? pv[u].z : pv[u].w;
                        const uint64_t pr2 = pack2(pr, pr);
#pragma unroll
                        for (int c = 0; c < DC / 2; ++c) acc[u][c] = fma2(pr2, vv[c], acc[u][c]);
                    }
                }
            }
        }
        // the segment ends: sums over the lanes of a row, outputs divided by them
        float* ws = static_cast<float*>(a.ws);
        __syncwarp();
#pragma unroll
        for (int u = 0; u < KR; ++u) {
#pragma unroll
            for (int o = 1; o < (KK < 4 ? 16 : 8); o <<= 1) l[u] += __shfl_xor_sync(0xffffffffu, l[u], o);
            if (kl == 0 && col_k == 0) {
                sm[SM::A + row_k + u] = 1.f / l[u];
                if (row0 + row_k + u < rows) ws[p.p_lse + seg * SHP_ROWS + r_in + row_k + u] = mx[u] + log2f(l[u]);
            }
        }
        __syncwarp();
#pragma unroll
        for (int u = 0; u < WR; ++u) {
            const float inv = sm[SM::A + warp * WR + u];
            if (row0 + warp * WR + u < rows) {
#pragma unroll
                for (int c = 0; c < DC / 2; ++c) {
                    const int d = lane * DC + 2 * c;
                    float lo, hi;
                    unpack2(acc[u][c], lo, hi);
                    *reinterpret_cast<float2*>(ws + p.p_o + seg * SHP_ROWS * D + ((int64_t)(d >> 2) * SHP_ROWS + r_in + warp * WR + u) * 4 + (d & 3)) =
                        make_float2(lo * inv, hi * inv);
                }
            }
        }
        if (blk == p.p_blocks) { blk = 0; ++h; }
    }
}

// ------------------------------------------------------------------ merge
// CTA: 32 query rows of one kv head (lanes) x 8 / WAYS groups of 4 features (warps) x WAYS shares of the partial results: a
// long list of them is read by WAYS warps.
// Many rows have one warp each and take four results at a time: registers for four CTAs per SM, so that 592 of them are one wave
// (4096 rows, 5 prefix segments: 6.5 us after the last result with eight at a time and two CTAs per SM).
constexpr int MERGE_THREADS = 256;

template <typename T, int D, int WAYS>
__global__ void __launch_bounds__(MERGE_THREADS, WAYS == 1 ? 4 : 2)
shared_merge_kernel(const SharedArgs a, const SharedPlan p) {
    constexpr int AT_ONCE = WAYS == 1 ? 4 : 8;
    constexpr int GROUPS = 8 / WAYS;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, way = warp / GROUPS, c4 = blockIdx.y * GROUPS + warp % GROUPS;
    const int h = blockIdx.z, row = min((int)(blockIdx.x * 32 + lane), a.B * a.g - 1);   // rows past the last repeat it
    const int b = row / a.g, j = row - b * a.g;
    const int len = __ldg(a.cache_lens + b);
    const float* ws = static_cast<const float*>(a.ws);
    const int mt = row / SHP_ROWS, r = row - mt * SHP_ROWS;
    const PrefixSegments ps(a, p, h, mt);
    const int gt = j / p.g_rows, x = j - gt * p.g_rows;
    const int64_t hh = (int64_t)h * p.g_tiles + gt;
    // before any thread may leave: the kernel after this one counts on all three having finished
    wait_for_previous();
    const int64_t* cum = reinterpret_cast<const int64_t*>(ws + p.cum);
    const int64_t per_head = __ldcg(cum + a.B), cum0 = __ldcg(cum + b), cum1 = __ldcg(cum + b + 1);
    RowMerge m;
    m.add<WAYS, AT_ONCE>(ps.n, ws + p.p_lse + ps.first * SHP_ROWS + r, (int64_t)p.m_tiles * SHP_ROWS,
                ws + p.p_o + ps.first * SHP_ROWS * D + ((int64_t)c4 * SHP_ROWS + r) * 4, (int64_t)p.m_tiles * SHP_ROWS * D, way);
    const bool live = len >= 0 && blockIdx.x * 32 + lane < a.B * a.g;   // a request, and no repeated row
    if (live) {
        const int64_t all = per_head * a.Hkv * p.g_tiles, W = own_workers(all, p.workers);
        const int64_t w0 = block_worker(hh * per_head + cum0, all, W), first = w0 + hh * a.B + b;
        const int n_own = (int)(block_worker(hh * per_head + cum1 - 1, all, W) - w0) + 1;
        m.add<WAYS, AT_ONCE>(n_own, ws + p.own_lse + first * p.g_rows + x, p.g_rows, ws + p.own_o + (first * p.g_rows + x) * D + c4 * 4,
                    (int64_t)p.g_rows * D, WAYS - 1 - way);   // the last way begins here, beside the first one's prefix results
    }
    if constexpr (WAYS > 1) {
        __shared__ RowMerge s_part[WAYS][GROUPS][32];
        const int grp = warp % GROUPS;
        s_part[way][grp][lane] = m;
        __syncthreads();
        if (way > 0) return;
        // a share that took no result, or only ones without weight, has a total of 0.  One whose log-sum-exps were all NaN has a maximum
        // of -inf too, but its total is NaN and goes on into the row
        RowMerge all;
#pragma unroll
        for (int y = 0; y < WAYS; ++y) all.M = fmaxf(all.M, s_part[y][grp][lane].M);
#pragma unroll
        for (int y = 0; y < WAYS; ++y) {
            const RowMerge& q = s_part[y][grp][lane];
            if (q.total == 0.f) continue;
            const float f = exp2f(q.M - all.M);
            all.total += f * q.total;
            all.o.x = fmaf(f, q.o.x, all.o.x); all.o.y = fmaf(f, q.o.y, all.o.y); all.o.z = fmaf(f, q.o.z, all.o.z); all.o.w = fmaf(f, q.o.w, all.o.w);
        }
        m = all;
    }
    if (live) m.store<T, D>(a, (int64_t)b * a.Hq + h * a.g + j, c4);
}

// ------------------------------------------------------------------ host side
// What the largest cut of a call takes, whatever kernels it runs, and of every smaller one: a buffer made for an engine's largest
// batch, prefix and cache bound has to do for its other steps too.  A plan's own size does not grow with them (short own caches
// are cut for twice the prefix CTAs: B32 Hq32 Hkv8, prefix 2048, 19 MB up to 127 own entries, 15 MB from 128 on), so each of its
// arrays is bounded apart.
size_t decode_shared_workspace_bytes(int B, int Hq, int Hkv, int D, int prefix_len, int max_len) {
    int64_t own_rows = 0, m_tiles = 0;
    for (bool cuda_cores : {false, true}) {
        const SharedPlan p = make_shared_plan(B, Hq, Hkv, D, prefix_len, max_len, 0, cuda_cores);
        m_tiles = p.m_tiles;
        own_rows = std::max(own_rows, (p.workers + (int64_t)B * Hkv * p.g_tiles) * p.g_rows);
    }
    // a worker per block at most, and as many CTAs as two per SM, or one per query tile; a partial result more per kv head
    const int64_t blocks = ((int64_t)prefix_len + SIMT_K - 1) / SIMT_K;
    const int64_t p_segments = blocks ? std::min(std::max<int64_t>(2 * SHP_CTAS, m_tiles), Hkv * blocks * m_tiles) + Hkv * m_tiles : 0;
    const int64_t floats[] = {p_segments * SHP_ROWS * D, p_segments * SHP_ROWS, own_rows * D, own_rows, 2 * ((int64_t)B + 1)};
    int64_t n = 0;
    for (int64_t x : floats) n += (x + 63) / 64 * 64;
    return (size_t)n * sizeof(float);
}

template <typename T, int D>
static cudaError_t own_stream(const SharedArgs& a, const SharedPlan& p, bool behind, cudaStream_t st) {
    auto* kernel = p.g_rows == 1 ? shared_own_stream_kernel<T, D, 1> : p.g_rows == 2 ? shared_own_stream_kernel<T, D, 2> : shared_own_stream_kernel<T, D, 4>;
    return launch_behind(kernel, dim3(STREAM_CTAS), OWN_WARPS * 32, 0, st, behind, a, p);
}

template <typename T, int D, int RT>
static cudaError_t prefix_simt_rt(const SharedArgs& a, const SharedPlan& p, bool behind, cudaStream_t st) {
    constexpr int smem = SimtSmem<D, RT>::FLOATS * (int)sizeof(float);
    const int rows = std::min(a.B * a.g, SHP_ROWS);
    return launch_behind(shared_prefix_simt_kernel<T, D, RT>, dim3(p.p_workers * p.m_tiles, (rows + RT - 1) / RT), SIMT_THREADS, smem, st, behind, a, p);
}
// Row tiles of 64 where that leaves two CTAs for an SM, which fill each other's waits, or else of 32 (B12 Hq16 Hkv4, prefix
// 2500: 30.4 us with 64, 28.5 with 32); 16 for up to 16 rows only (28 rows: 41.7 us in one tile of 32, 53.7 in two of 16).
template <typename T, int D>
static cudaError_t prefix_simt(const SharedArgs& a, const SharedPlan& p, bool behind, cudaStream_t st) {
    if (p.p_keys != SIMT_K) return cudaErrorInvalidValue;
    const int rows = std::min(a.B * a.g, SHP_ROWS), share = p.p_workers * p.m_tiles;
    if (rows > 32 && share * ((rows + 63) / 64) > 148) return prefix_simt_rt<T, D, 64>(a, p, behind, st);
    return rows > 16 ? prefix_simt_rt<T, D, 32>(a, p, behind, st) : prefix_simt_rt<T, D, 16>(a, p, behind, st);
}

template <typename T, int D>
static cudaError_t shared_t(const SharedArgs& a, bool generic, cudaStream_t st) {
    // both parts on the tensor cores or both on CUDA cores: a cut and the kernels that follow it belong together
    const bool tc = sizeof(T) == 2 && !generic && shared_own_tma_fits(a) && (a.prefix_len == 0 || shared_prefix_tc_fits(a));
    const SharedPlan p = make_shared_plan(a.B, a.Hq, a.Hkv, D, a.prefix_len, a.max_len, a.prefix_table ? 1 << a.pg.log2_ps : 0, !tc);
    auto prefix = [&](bool behind) {
        return p.p_blocks == 0 ? cudaSuccess : tc ? launch_shared_prefix_tc(a, p, D, behind, st) : prefix_simt<T, D>(a, p, behind, st);
    };
    cudaError_t e;
    if (p.whole) {
        e = prefix(false);
        return e == cudaSuccess ? launch_shared_own_tma(a, p, D, p.p_blocks > 0, st) : e;
    }
    if (tc) {
        e = launch_shared_own_tma(a, p, D, false, st);
        if (e == cudaSuccess) e = prefix(true);
    } else {   // the longer one goes first; the other's CTAs take the room it leaves
        e = prefix(false);
        if (e == cudaSuccess) e = own_stream<T, D>(a, p, p.p_blocks > 0, st);
    }
    if (e != cudaSuccess) return e;
    // as many warps to a row's partial results as there is room for in one wave
    const dim3 grid((a.B * a.g + 31) / 32, D / 32, a.Hkv);
    const int64_t ctas = (int64_t)grid.x * grid.y * grid.z;
    auto merge = [&](auto* kernel, int ways) { return launch_behind(kernel, dim3(grid.x, grid.y * ways, grid.z), MERGE_THREADS, 0, st, true, a, p); };
    if (ctas * 4 <= 296) return merge(shared_merge_kernel<T, D, 4>, 4);
    if (ctas * 2 <= 296) return merge(shared_merge_kernel<T, D, 2>, 2);
    return merge(shared_merge_kernel<T, D, 1>, 1);
}

cudaError_t launch_decode_shared(const SharedArgs& a, int D, loma_dtype dt, bool generic, cudaStream_t st) {
    if (dt == LOMA_F32) return D == 64 ? shared_t<float, 64>(a, generic, st) : shared_t<float, 128>(a, generic, st);
    return D == 64 ? shared_t<__nv_bfloat16, 64>(a, generic, st) : shared_t<__nv_bfloat16, 128>(a, generic, st);
}

}  // namespace loma
