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

// ------------------------------------------------------------------ own cache on CUDA cores (fp32, second opinion)
// A worker is a warp, as in shared_own_tma_kernel.  The lanes that share a row hold 16 bytes of it each; G heads of the
// group at a time, so a row is loaded once for them.
template <typename T, int D, int G>
__global__ void __launch_bounds__(OWN_WARPS * 32)
shared_own_stream_kernel(const SharedArgs a, const SharedPlan p) {
    using V = Vec16<T>;
    constexpr int N = V::N, LPK = D / N, KPL = 32 / LPK, NL = OWN_KEYS / KPL < 8 ? OWN_KEYS / KPL : 8;
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
        float q[G][N], acc[G][N], m[G], l[G];
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
                    m[x] = -INFINITY;
                    l[x] = 0.f;
                }
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
#pragma unroll
                for (int x = 0; x < G; ++x) {
                    float s[NL], mb = -INFINITY;
#pragma unroll
                    for (int i = 0; i < NL; ++i) {
                        float kf[N];
                        V::unpack(kr[i], kf);
                        s[i] = 0.f;
#pragma unroll
                        for (int e = 0; e < N; ++e) s[i] = fmaf(q[x][e], kf[e], s[i]);
                    }
#pragma unroll
                    for (int o = LPK / 2; o > 0; o >>= 1)
#pragma unroll
                        for (int i = 0; i < NL; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
#pragma unroll
                    for (int i = 0; i < NL; ++i) {
                        s[i] = j0 + i * KPL + sub <= len ? s[i] : -INFINITY;
                        mb = fmaxf(mb, s[i]);
                    }
#pragma unroll
                    for (int o = 16; o >= LPK; o >>= 1) mb = fmaxf(mb, __shfl_xor_sync(0xffffffffu, mb, o));
                    const float m_new = fmaxf(m[x], mb), ref = m_new == -INFINITY ? 0.f : m_new, alpha = exp2f(m[x] - ref);
                    m[x] = m_new;
                    l[x] *= alpha;
#pragma unroll
                    for (int e = 0; e < N; ++e) acc[x][e] *= alpha;
#pragma unroll
                    for (int i = 0; i < NL; ++i) {
                        const float pr = exp2f(s[i] - ref);
                        float vf[N];
                        V::unpack(vr[i], vf);
                        l[x] += pr;
#pragma unroll
                        for (int e = 0; e < N; ++e) acc[x][e] = fmaf(pr, vf[e], acc[x][e]);
                    }
                }
            }
            const bool tail = c.blk == len / OWN_KEYS;
            if (tail || t + 1 == t_end) {
                const int64_t seg = w + (int64_t)c.hh * a.B + c.b;
#pragma unroll
                for (int x = 0; x < G; ++x) {
                    float lt = l[x], ot[N];
#pragma unroll
                    for (int e = 0; e < N; ++e) ot[e] = acc[x][e];
#pragma unroll
                    for (int o = 16; o >= LPK; o >>= 1) {
                        lt += __shfl_xor_sync(0xffffffffu, lt, o);
#pragma unroll
                        for (int e = 0; e < N; ++e) ot[e] += __shfl_xor_sync(0xffffffffu, ot[e], o);
                    }
                    if (x < heads && lane < LPK) {
                        const float inv = 1.f / lt;
                        float4* o = reinterpret_cast<float4*>(ws + p.own_o + (seg * p.g_rows + x) * D + li * N);
#pragma unroll
                        for (int e = 0; e < N; e += 4) o[e / 4] = make_float4(ot[e] * inv, ot[e + 1] * inv, ot[e + 2] * inv, ot[e + 3] * inv);
                        if (lane == 0) ws[p.own_lse + seg * p.g_rows + x] = m[x] + log2f(lt);
                    }
                }
                // the new token's K and V go to entry len (read by nobody in this launch)
                if (tail && kn && gt == 0 && lane < LPK) {
                    const int64_t row = own_row(a, c.b, h, len) * D;
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
// RT query rows against 32 keys at a time, all in fp32 in shared memory, with RT / 16 x 2 scores and RT / 8 x (D / 32) outputs
// per thread in registers; the next keys are on their way from memory while these are worked on.  Bound by fp32 FMA for many
// rows, by the latency of a block's steps for few.  Query row m of kv head h is head h g + m mod g of sequence m / g.
constexpr int SIMT_THREADS = 256;

template <int D, int RT>
struct SimtSmem {
    static constexpr int Q = 0, K = Q + RT * (D + 4), V = K + SIMT_K * (D + 4), S = V + SIMT_K * D, ML = S + RT * (SIMT_K + 4),
                         FLOATS = ML + 3 * RT;
};

template <typename T, int D, int RT>
__global__ void __launch_bounds__(SIMT_THREADS, RT == 64 ? 1 : 2)
shared_prefix_simt_kernel(const SharedArgs a, const SharedPlan p) {
    using V = Vec16<T>;
    using SM = SimtSmem<D, RT>;
    constexpr int N = V::N, LPK = D / N, DC = D / 32, PASSES = SIMT_K * LPK / SIMT_THREADS, SR = RT / 16, KU = SIMT_K / 16, OR = RT / 8;
    extern __shared__ __align__(16) float sm[];
    let_next_start();
    const int tid = threadIdx.x, rows = a.B * a.g;
    const float scale_log2 = a.scale * 1.4426950408889634f;
    const int worker = blockIdx.x / p.m_tiles, mt = blockIdx.x - worker * p.m_tiles;
    const int64_t blocks = (int64_t)a.Hkv * p.p_blocks;
    int64_t t = first_block(worker, blocks, p.p_workers);
    const int64_t t_end = first_block(worker + 1, blocks, p.p_workers);
    const int r_in = blockIdx.y * RT, row0 = mt * SHP_ROWS + r_in;   // RT rows of the tile per blockIdx.y
    if (row0 >= rows) t = t_end;
    const int sr = (tid >> 4) * SR, sk = tid & 15;        // scores: rows sr ..; keys sk + 16 u
    const int orow = (tid >> 5) * OR, oc = tid & 31;      // outputs: rows orow .. (a warp's own); features oc * DC ..
    uint4 kv[2][PASSES];
    auto load = [&](int h, int k0) {                      // all of the thread's loads at once
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int r = (tid + i * SIMT_THREADS) / LPK, c = (tid + i * SIMT_THREADS) % LPK;
            const int64_t row = prefix_row(a, h, min(k0 + r, a.prefix_len - 1)) * D;   // keys past the end repeat the last one
            kv[0][i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(a.k_prefix) + row) + c);
            kv[1][i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(a.v_prefix) + row) + c);
        }
    };
    if (t < t_end) load((int)(t / p.p_blocks), (int)(t % p.p_blocks) * SIMT_K);
    while (t < t_end) {                                   // segments of the CTA's share
        const int h = (int)(t / p.p_blocks), blk0 = (int)(t - (int64_t)h * p.p_blocks);
        const int blk1 = (int)min((int64_t)p.p_blocks, blk0 + (t_end - t));
        const int begin = blk0 * SIMT_K, end = min(a.prefix_len, blk1 * SIMT_K);
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
        if (tid < RT) { sm[SM::ML + tid] = -INFINITY; sm[SM::ML + RT + tid] = 0.f; }
        uint64_t acc[OR][DC / 2];
#pragma unroll
        for (int u = 0; u < OR; ++u)
#pragma unroll
            for (int c = 0; c < DC / 2; ++c) acc[u][c] = 0;
        for (int k0 = begin; k0 < end; k0 += SIMT_K) {
            if (k0 > begin) __syncthreads();              // the tiles have been read
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int r = (tid + i * SIMT_THREADS) / LPK, c = (tid + i * SIMT_THREADS) % LPK;
                float f[N];
                V::unpack(kv[0][i], f);
#pragma unroll
                for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(&sm[SM::K + r * (D + 4) + c * N + e]) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
                V::unpack(kv[1][i], f);
#pragma unroll
                for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(&sm[SM::V + r * D + c * N + e]) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
            }
            if (++t < t_end) load((int)(t / p.p_blocks), (int)(t % p.p_blocks) * SIMT_K);
            __syncthreads();
            // two-wide FMA: sums over even and odd features side by side
            uint64_t s2[SR][KU];
#pragma unroll
            for (int u = 0; u < SR; ++u)
#pragma unroll
                for (int w = 0; w < KU; ++w) s2[u][w] = 0;
#pragma unroll 4
            for (int d = 0; d < D; d += 4) {
                ulonglong2 qv[SR], kf[KU];
#pragma unroll
                for (int u = 0; u < SR; ++u) qv[u] = *reinterpret_cast<const ulonglong2*>(&sm[SM::Q + (sr + u) * (D + 4) + d]);
#pragma unroll
                for (int u = 0; u < KU; ++u) kf[u] = *reinterpret_cast<const ulonglong2*>(&sm[SM::K + (sk + 16 * u) * (D + 4) + d]);
#pragma unroll
                for (int u = 0; u < SR; ++u)
#pragma unroll
                    for (int w = 0; w < KU; ++w) s2[u][w] = fma2(qv[u].y, kf[w].y, fma2(qv[u].x, kf[w].x, s2[u][w]));
            }
            float s[SR][KU];
#pragma unroll
            for (int u = 0; u < SR; ++u)
#pragma unroll
                for (int w = 0; w < KU; ++w) {
                    float lo, hi;
                    unpack2(s2[u][w], lo, hi);
                    s[u][w] = lo + hi;
                }
#pragma unroll
            for (int u = 0; u < SR; ++u) {   // 16 lanes share a row
                float mx = -INFINITY;
#pragma unroll
                for (int w = 0; w < KU; ++w) {
                    if (k0 + sk + 16 * w >= end) s[u][w] = -INFINITY;
                    mx = fmaxf(mx, s[u][w]);
                }
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                const float m_old = sm[SM::ML + sr + u], m_new = fmaxf(m_old, mx), ref = m_new == -INFINITY ? 0.f : m_new;
                float sum = 0.f;
#pragma unroll
                for (int w = 0; w < KU; ++w) {
                    const float e = exp2f(s[u][w] - ref);
                    sum += e;
                    sm[SM::S + (sr + u) * (SIMT_K + 4) + sk + 16 * w] = e;
                }
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                __syncwarp();
                if ((tid & 15) == 0) {
                    const float alpha = exp2f(m_old - ref);
                    sm[SM::ML + sr + u] = m_new;
                    sm[SM::ML + RT + sr + u] = sm[SM::ML + RT + sr + u] * alpha + sum;
                    sm[SM::ML + 2 * RT + sr + u] = alpha;
                }
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < OR; ++u) {
                const float alpha = sm[SM::ML + 2 * RT + orow + u];
#pragma unroll
                for (int c = 0; c < DC / 2; ++c) acc[u][c] = fma2(acc[u][c], pack2(alpha, alpha), 0);
            }
#pragma unroll 2
            for (int k = 0; k < SIMT_K; k += 4) {
                float4 pv[OR];
#pragma unroll
                for (int u = 0; u < OR; ++u) pv[u] = *reinterpret_cast<const float4*>(&sm[SM::S + (orow + u) * (SIMT_K + 4) + k]);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) {
                    uint64_t vv[DC / 2];
#pragma unroll
                    for (int c = 0; c < DC / 2; ++c) vv[c] = *reinterpret_cast<const uint64_t*>(&sm[SM::V + (k + kk) * D + oc * DC + 2 * c]);
#pragma unroll
                    for (int u = 0; u < OR; ++u) {
                        const float pr = kk == 0 ? pv[u].x : kk == 1 ? pv[u].y : kk == 2 ? pv[u].z : pv[u].w;
                        const uint64_t pr2 = pack2(pr, pr);
#pragma unroll
                        for (int c = 0; c < DC / 2; ++c) acc[u][c] = fma2(pr2, vv[c], acc[u][c]);
                    }
                }
            }
        }
        __syncthreads();
        float* ws = static_cast<float*>(a.ws);
#pragma unroll
        for (int u = 0; u < OR; ++u) {
            const float inv = 1.f / sm[SM::ML + RT + orow + u];
            if (row0 + orow + u < rows) {
#pragma unroll
                for (int c = 0; c < DC / 2; ++c) {
                    const int d = oc * DC + 2 * c;
                    float lo, hi;
                    unpack2(acc[u][c], lo, hi);
                    *reinterpret_cast<float2*>(ws + p.p_o + seg * SHP_ROWS * D + ((int64_t)(d >> 2) * SHP_ROWS + r_in + orow + u) * 4 + (d & 3)) =
                        make_float2(lo * inv, hi * inv);
                }
            }
        }
        if (tid < RT && row0 + tid < rows) ws[p.p_lse + seg * SHP_ROWS + r_in + tid] = sm[SM::ML + tid] + log2f(sm[SM::ML + RT + tid]);
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
        RowMerge all;
#pragma unroll
        for (int y = 0; y < WAYS; ++y) all.M = fmaxf(all.M, s_part[y][grp][lane].M);
#pragma unroll
        for (int y = 0; y < WAYS; ++y) {
            const RowMerge& q = s_part[y][grp][lane];
            if (q.M == -INFINITY) continue;
            const float f = exp2f(q.M - all.M);
            all.total += f * q.total;
            all.o.x = fmaf(f, q.o.x, all.o.x); all.o.y = fmaf(f, q.o.y, all.o.y); all.o.z = fmaf(f, q.o.z, all.o.z); all.o.w = fmaf(f, q.o.w, all.o.w);
        }
        m = all;
    }
    if (live) m.store<T, D>(a, (int64_t)b * a.Hq + h * a.g + j, c4);
}

// ------------------------------------------------------------------ host side
size_t decode_shared_workspace_bytes(int B, int Hq, int Hkv, int D, int prefix_len, int max_len) {
    const int64_t n = std::max(make_shared_plan(B, Hq, Hkv, D, prefix_len, max_len, false).total, make_shared_plan(B, Hq, Hkv, D, prefix_len, max_len, true).total);
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
// the tallest row tile that the rows fill
template <typename T, int D>
static cudaError_t prefix_simt(const SharedArgs& a, const SharedPlan& p, bool behind, cudaStream_t st) {
    if (p.p_keys != SIMT_K) return cudaErrorInvalidValue;
    const int rows = a.B * a.g;
    return rows <= 16 ? prefix_simt_rt<T, D, 16>(a, p, behind, st) : rows <= 32 ? prefix_simt_rt<T, D, 32>(a, p, behind, st)
                                                                                 : prefix_simt_rt<T, D, 64>(a, p, behind, st);
}

template <typename T, int D>
static cudaError_t shared_t(const SharedArgs& a, bool generic, cudaStream_t st) {
    // both parts on the tensor cores or both on CUDA cores: a cut and the kernels that follow it belong together
    const bool tc = sizeof(T) == 2 && !generic && shared_own_tma_fits(a) && (a.prefix_len == 0 || shared_prefix_tc_fits(a));
    const SharedPlan p = make_shared_plan(a.B, a.Hq, a.Hkv, D, a.prefix_len, a.max_len, !tc);
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
    } else {   // neither kernel leaves room for the other, and the longer one goes first
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
