// RMS norm of every head of q and k and the rotary embedding in one pass: training layout forward and backward, and the
// serving form that writes keys and values straight into cache pages.
//
//     r = (mean_d x_d^2 + eps)^(-1/2)        y = R(p) (w * x r)         R(p): the rotation of rope.cu at the row's id p
// and, with g the gradient of y and u = R(-p) g,
//     dw = sum over rows of u * x r          dx = r (w u - x r^2 mean_d(w u x))
//
// Everything is held in fp32 between the one read and the one rounding at the end, so normalising and rotating in one
// pass is also more exact than two passes with a bf16 tensor between them.  The kernels are bound by HBM: q and k are
// read once and written once (backward: read twice as much, written once); nothing is saved for the backward but q and k,
// since r costs three shuffles and reading it back would cost a load.
//
// A lane owns N = 16 / sizeof(T) adjacent features of a row's first half and their partners in the second half (two
// 16-byte accesses a row), so the rotation pairs and the products with w stay in its registers; (D/2) / N lanes share a
// row and add their sums with shuffles.  A lane keeps the cos / sin of its row's id for every (batch, head) it walks, and
// fetches its next pairs into a ring of its own in shared memory (cp.async, nobody else reads it, so there is no barrier):
// bytes in flight cost no registers, which w, cos / sin and the sums of dw need.  The rows that a warp takes together lie
// behind one another in memory: consecutive rows of a head, or, in a projection's [B, S, H, D] output, heads of a row.
// Measured, bf16, 4608 rows of B4, D128: forward of 32 + 32 heads 98.4 us (6.1 TB/s, 0.95 of a copy), backward of 32 + 8 heads 98.7 us
// (5.7 TB/s, 0.89; issue slots 62 % taken).  The gains' sums are one partial result per CTA added up by D / 16 CTAs: 2 us there, 10 of 34
// us for 34816 rows of 2 + 2 heads.  A few hundred rows in fp32: 3.4 us forward, 5.5 us backward (two launches).
#include <math.h>

#include <algorithm>

#include "loma_internal.cuh"

namespace loma {

constexpr int QKN_WARPS = 8;

template <typename T>
__device__ __forceinline__ void load_gain(const T* w, int d0, float (&lo)[Vec16<T>::N], float (&hi)[Vec16<T>::N], int half) {
    if (w) {
        Vec16<T>::unpack(__ldg(reinterpret_cast<const uint4*>(w + d0)), lo);
        Vec16<T>::unpack(__ldg(reinterpret_cast<const uint4*>(w + d0 + half)), hi);
    } else {
#pragma unroll
        for (int u = 0; u < Vec16<T>::N; ++u) lo[u] = hi[u] = 1.f;
    }
}

// cos and sin of pos * theta, the angle formed and reduced in double (see rope_cos_sin).  The reduced angle is rounded to fp32 for
// sincosf: off by 2^-23 at most, and the results by about as much
__device__ __forceinline__ void angle_cos_sin(int pos, double theta, float& c, float& s) {
    double a = (double)pos * theta;
    a -= 6.283185307179586476925 * rint(a * 0.15915494309189533577);
    sincosf((float)a, &s, &c);
}

template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// Pairs (batch, head) of one tensor that this lane walks: first, first + step, ... below p1.  `stages` fetches are in flight.
// BWD: v.grad is read too, acc[0..N) / acc[N..2N) collect the lane's share of dw.
template <typename T, int D, bool BWD, int STAGES>
__device__ __forceinline__ void walk_pairs(const HeadsView& v, int p0, int p1, int first, int step, int i, bool live, int d0, uint32_t ring,
                                           const float (&cs)[Vec16<T>::N], const float (&sn)[Vec16<T>::N], float eps,
                                           float (&acc)[2 * Vec16<T>::N]) {
    using V = Vec16<T>;
    constexpr int N = V::N, HALF = D / 2, LPR = HALF / N, CHUNKS = BWD ? 4 : 2;
    constexpr uint32_t CHUNK = QKN_WARPS * 32 * 16, STAGE = CHUNKS * CHUNK;   // bytes of one chunk of all lanes
    float wl[N], wh[N];
    load_gain(static_cast<const T*>(v.w), d0, wl, wh, HALF);
    const T* in = static_cast<const T*>(v.in) + (int64_t)i * v.ss + d0;
    const T* grad = BWD ? static_cast<const T*>(v.grad) + (int64_t)i * v.ss + d0 : nullptr;
    T* out = static_cast<T*>(v.out) + (int64_t)i * v.ss + d0;
    // the fetch runs ahead of the work: both know their pair as (b, h); past the end the last pair is taken again
    int bf = min(first, p1 - 1) / v.H, hf = min(first, p1 - 1) - bf * v.H, pf = first;
    int b = bf, h = hf;
    auto advance = [&](int& p, int& bb, int& hh) {
        p += step;
        if (p < p1) {
            hh += step;
            while (hh >= v.H) { hh -= v.H; ++bb; }
        }
    };
    uint32_t slot_f = ring;
    auto fetch = [&](bool any) {
        if (any) {
            const int64_t off = (int64_t)bf * v.sb + (int64_t)hf * v.sh;
            cp_async16(slot_f, in + off);
            cp_async16(slot_f + CHUNK, in + off + HALF);
            if (BWD) {
                cp_async16(slot_f + 2 * CHUNK, grad + off);
                cp_async16(slot_f + 3 * CHUNK, grad + off + HALF);
            }
            advance(pf, bf, hf);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        slot_f = slot_f == ring + (STAGES - 1) * STAGE ? ring : slot_f + STAGE;
    };
    const int rounds = (p1 - p0 + step - 1) / step;   // the same for all lanes of the warp: shuffles below
#pragma unroll
    for (int u = 0; u < STAGES - 1; ++u) fetch(u < rounds);
    uint32_t slot = ring;
    int p = first;
#pragma unroll 1
    for (int n = 0; n < rounds; ++n) {
        fetch(n + STAGES - 1 < rounds);
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
        auto chunk = [&](int c) {
            uint4 x;
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(slot + c * CHUNK) : "memory");
            return x;
        };
        float a[N], c[N], ra[N], rc[N];
        V::unpack(chunk(0), a);
        V::unpack(chunk(1), c);
        float ssq = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) ssq = fmaf(a[e], a[e], fmaf(c[e], c[e], ssq));
        const bool counts = live && p < p1;   // rows and pairs that are taken again write nothing and count once
        if (!BWD) {
            const float r = rsqrtf(row_sum<LPR>(ssq) * (1.f / D) + eps);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float ya = a[e] * r * wl[e], yc = c[e] * r * wh[e];
                ra[e] = ya * cs[e] - yc * sn[e];
                rc[e] = yc * cs[e] + ya * sn[e];
            }
        } else {
            float ga[N], gc[N];
            V::unpack(chunk(2), ga);
            V::unpack(chunk(3), gc);
            float dot = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) {      // u = R(-p) g, over ga / gc
                const float ua = ga[e] * cs[e] + gc[e] * sn[e], uc = gc[e] * cs[e] - ga[e] * sn[e];
                ga[e] = ua;
                gc[e] = uc;
                dot = fmaf(wl[e] * ua, a[e], fmaf(wh[e] * uc, c[e], dot));
            }
            const float r = rsqrtf(row_sum<LPR>(ssq) * (1.f / D) + eps);
            const float mean = row_sum<LPR>(dot) * (1.f / D) * r * r;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (counts) {
                    acc[e] = fmaf(ga[e] * a[e], r, acc[e]);
                    acc[N + e] = fmaf(gc[e] * c[e], r, acc[N + e]);
                }
                ra[e] = r * (wl[e] * ga[e] - a[e] * mean);
                rc[e] = r * (wh[e] * gc[e] - c[e] * mean);
            }
        }
        if (counts) {
            const int64_t off = (int64_t)b * v.sb + (int64_t)h * v.sh;
            __stcs(reinterpret_cast<uint4*>(out + off), V::pack(ra));
            __stcs(reinterpret_cast<uint4*>(out + off + HALF), V::pack(rc));
        }
        advance(p, b, h);
        slot = slot == ring + (STAGES - 1) * STAGE ? ring : slot + STAGE;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <bool BWD>
struct QknRing {
    static constexpr int STAGES = BWD ? 4 : 6, BYTES = STAGES * (BWD ? 4 : 2) * QKN_WARPS * 32 * 16;   // 64 KB / 48 KB a CTA
};

// A CTA takes rows of the laid-out sequence and a slice of the (batch, head) pairs, q's and k's as one list.  Lanes of a warp
// that do not share a row take RPW consecutive rows, or (by_heads) RPW consecutive pairs of one row.
// part (backward): [2][CTAs][D] fp32, this CTA's sums of dw.
template <typename T, int D, bool BWD>
__global__ void __launch_bounds__(QKN_WARPS * 32, BWD ? 2 : 3)
qk_norm_rope_kernel(const HeadsView q, const HeadsView k, int B, Layout L, float eps, double log2_base, int position_type, int by_heads,
                    float* __restrict__ part) {
    using V = Vec16<T>;
    constexpr int N = V::N, HALF = D / 2, LPR = HALF / N, RPW = 32 / LPR;
    extern __shared__ __align__(16) uint8_t qkn_ring[];
    __shared__ double theta[HALF];
    __shared__ float red[BWD ? QKN_WARPS : 1][BWD ? D : 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = lane / LPR;
    for (int d = threadIdx.x; d < HALF; d += QKN_WARPS * 32) theta[d] = exp2(-log2_base * (2.0 * d / D));
    __syncthreads();
    const int row = by_heads ? blockIdx.x * QKN_WARPS + warp : (blockIdx.x * QKN_WARPS + warp) * RPW + group;
    const bool live = row < L.S;
    const int i = min(row, L.S - 1);   // a row past the end reads the last row and writes nothing
    const RowInfo ri = layout_row(i, L.n_chunks, L.c, L.t, L.s);
    const int pos = (position_type & 1) && ri.zone == LOMA_ZONE_MEM ? ri.chunk * L.t + ri.offset : ri.pos;
    const int d0 = (lane % LPR) * N;
    float cs[N], sn[N];
#pragma unroll
    for (int u = 0; u < N; ++u) angle_cos_sin(pos, theta[d0 + u], cs[u], sn[u]);
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(qkn_ring) + threadIdx.x * 16;
    const int nq = B * q.H, total = nq + B * k.H;
    const int per = (total + gridDim.y - 1) / gridDim.y;
    const int p0 = min(total, (int)blockIdx.y * per), p1 = min(total, p0 + per);
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        const HeadsView& v = which == 0 ? q : k;
        const int a0 = which == 0 ? min(p0, nq) : max(p0, nq) - nq, a1 = which == 0 ? min(p1, nq) : max(p1, nq) - nq;
        float acc[2 * N];
#pragma unroll
        for (int e = 0; e < 2 * N; ++e) acc[e] = 0.f;
        if (a0 < a1)
            walk_pairs<T, D, BWD, QknRing<BWD>::STAGES>(v, a0, a1, a0 + (by_heads ? group : 0), by_heads ? RPW : 1, i, live, d0, ring, cs, sn, eps, acc);
        if (BWD && v.dw) {
            // the warp's rows, then the CTA's warps, in a fixed order
#pragma unroll
            for (int e = 0; e < 2 * N; ++e)
#pragma unroll
                for (int o = LPR; o < 32; o <<= 1) acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], o);
            if (lane < LPR) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    red[warp][d0 + e] = acc[e];
                    red[warp][HALF + d0 + e] = acc[N + e];
                }
            }
            __syncthreads();
            if (which == 1 || !k.dw) let_next_start();   // the sums of dw: here, so that their CTAs take no room from these
            if (threadIdx.x < D) {
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < QKN_WARPS; ++w) s += red[w][threadIdx.x];
                const int cta = blockIdx.y * gridDim.x + blockIdx.x, n_cta = gridDim.x * gridDim.y;
                part[((int64_t)which * n_cta + cta) * D + threadIdx.x] = s;
            }
            __syncthreads();
        }
    }
}

// dw of q (block y = 0) and k (1): the CTAs' sums added up in double, 32 features per block.
template <typename T>
__global__ void __launch_bounds__(1024)
qk_norm_dw_kernel(const float* __restrict__ part, int n_cta, int D, T* __restrict__ dwq, T* __restrict__ dwk) {
    __shared__ double s[32][33];
    T* dw = blockIdx.y == 0 ? dwq : dwk;
    wait_for_previous();   // launched while the last CTAs finish
    if (!dw) return;
    const int d = blockIdx.x * 32 + threadIdx.x;
    const float* p = part + (int64_t)blockIdx.y * n_cta * D + d;
    double x = 0.0;
#pragma unroll 4
    for (int c = threadIdx.y; c < n_cta; c += 32) x += (double)p[(int64_t)c * D];
    s[threadIdx.y][threadIdx.x] = x;
    __syncthreads();
    if (threadIdx.y == 0) {
        double t = 0.0;
        for (int y = 0; y < 32; ++y) t += s[y][threadIdx.x];
        if constexpr (sizeof(T) == 2) dw[d] = __float2bfloat16_rn((float)t);
        else dw[d] = (float)t;
    }
}

// Rows per CTA, and slices of the pairs.  Every slice computes its rows' angles again, so there are as many as it takes to give
// every SM two CTAs, and up to six per SM (waves that even out) only while a slice keeps 16 pairs a lane.
constexpr int NORM_CTAS = 148 * 6;
struct NormGrid {
    int rows, slices;
    int64_t most;   // CTAs of this call at most, and of every smaller one: rows * slices does not grow with the rows
};
static NormGrid norm_grid(int B, int Hq, int Hk, int D, const Layout& L, int elt_bytes, bool by_heads) {
    const int rpw = 32 / ((D / 2) / (16 / elt_bytes));
    NormGrid g;
    g.rows = (L.S + QKN_WARPS * (by_heads ? 1 : rpw) - 1) / (QKN_WARPS * (by_heads ? 1 : rpw));
    const int pairs = B * (Hq + Hk), lane_pairs = by_heads ? (pairs + rpw - 1) / rpw : pairs;
    int slices = 1;
    while (slices < lane_pairs &&
           ((int64_t)g.rows * slices < 148 * 2 || ((int64_t)g.rows * slices < NORM_CTAS && lane_pairs / slices >= 32)))
        slices *= 2;
    g.slices = std::min(slices, lane_pairs);
    g.most = std::min<int64_t>(std::max(g.rows, 2 * NORM_CTAS), (int64_t)g.rows * lane_pairs);   // the last doubling began below NORM_CTAS
    return g;
}

size_t qk_norm_rope_bwd_workspace_bytes(int B, int Hq, int Hk, int D, const Layout& L) {
    int64_t most = 0;
    for (int es = 2; es <= 4; es += 2)
        for (bool by_heads : {false, true}) most = std::max(most, norm_grid(B, Hq, Hk, D, L, es, by_heads).most);
    return (size_t)2 * most * D * sizeof(float);
}

template <typename T, int D>
static cudaError_t norm_t(const HeadsView& q, const HeadsView& k, int B, const Layout& L, float eps, double theta_base, int position_type,
                          bool backward, void* ws, cudaStream_t st) {
    const HeadsView& lead = q.H > 0 ? q : k;
    const bool by_heads = lead.H > 1 && lead.sh < lead.ss;   // heads of a row behind one another: [B, S, H, D]
    const NormGrid ng = norm_grid(B, q.H, k.H, D, L, sizeof(T), by_heads);
    const dim3 grid(ng.rows, ng.slices);
    if (!backward) {
        cudaError_t e = prepare_kernel(reinterpret_cast<const void*>(qk_norm_rope_kernel<T, D, false>), QknRing<false>::BYTES);
        if (e != cudaSuccess) return e;
        qk_norm_rope_kernel<T, D, false><<<grid, QKN_WARPS * 32, QknRing<false>::BYTES, st>>>(q, k, B, L, eps, log2(theta_base), position_type, by_heads,
                                                                                          nullptr);
        count_launches(1);
        return cudaGetLastError();
    }
    cudaError_t e0 = prepare_kernel(reinterpret_cast<const void*>(qk_norm_rope_kernel<T, D, true>), QknRing<true>::BYTES);
    if (e0 != cudaSuccess) return e0;
    qk_norm_rope_kernel<T, D, true><<<grid, QKN_WARPS * 32, QknRing<true>::BYTES, st>>>(q, k, B, L, eps, log2(theta_base), position_type, by_heads,
                                                                                    static_cast<float*>(ws));
    count_launches(1);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess || (!q.dw && !k.dw)) return e;
    return launch_behind(qk_norm_dw_kernel<T>, dim3(D / 32, 2), dim3(32, 32), 0, st, true, static_cast<const float*>(ws), (int)(grid.x * grid.y), D,
                         static_cast<T*>(q.dw), static_cast<T*>(k.dw));
}

cudaError_t launch_qk_norm_rope(const HeadsView& q, const HeadsView& k, int B, int D, const Layout& L, loma_dtype dt, float eps,
                                double theta_base, int position_type, bool backward, void* ws, cudaStream_t st) {
    if (dt == LOMA_F32)
        return D == 64 ? norm_t<float, 64>(q, k, B, L, eps, theta_base, position_type, backward, ws, st)
                       : norm_t<float, 128>(q, k, B, L, eps, theta_base, position_type, backward, ws, st);
    return D == 64 ? norm_t<__nv_bfloat16, 64>(q, k, B, L, eps, theta_base, position_type, backward, ws, st)
                   : norm_t<__nv_bfloat16, 128>(q, k, B, L, eps, theta_base, position_type, backward, ws, st);
}

// ------------------------------------------------------------------ serving form
// A warp takes a packed row (token), or one of `parts` shares of its heads where there are few tokens: RPW heads at a time out
// of the row's list [q heads | k heads | v heads], fetched ahead across the borders between rows.  The D / 2 angles of a row are
// computed once, two per lane, and reach the other lanes through shared memory of the warp's own; no barrier.  Bound by
// instruction issue as much as by HBM, so what does not change from row to row (theta, gains) is kept.  Measured, bf16, 32 + 8 heads,
// D128: 6000 rows 28.4 us (5.2 TB/s, 0.80 of a copy), 32 rows 3.8 us.
constexpr int APP_STAGES = 6, APP_RING = APP_STAGES * 2 * QKN_WARPS * 32 * 16;   // 48 KB a CTA

template <typename T, int D>
__global__ void __launch_bounds__(QKN_WARPS * 32, 3)
qk_norm_rope_append_kernel(const AppendArgs a, int parts) {
    using V = Vec16<T>;
    constexpr int N = V::N, HALF = D / 2, LPR = HALF / N, RPW = 32 / LPR, AP = HALF / 32;   // AP: angles a lane computes
    constexpr uint32_t CHUNK = QKN_WARPS * 32 * 16, STAGE = 2 * CHUNK;
    extern __shared__ __align__(16) uint8_t qkn_ring[];
    __shared__ __align__(16) float s_gain[2][D];                    // wq, wk
    __shared__ __align__(16) float s_ang[QKN_WARPS][2][HALF];       // cos, sin of the warp's row
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = lane / LPR, d0 = (lane % LPR) * N;
    const int total = a.Hq + 2 * a.Hk, steps = (total + RPW - 1) / RPW;       // heads of a row; steps of RPW heads
    const int64_t items = (int64_t)a.T * parts, stride = (int64_t)gridDim.x * QKN_WARPS;
    int64_t item = (int64_t)warp * gridDim.x + blockIdx.x;                     // neighbours on different SMs
    // the fetch runs ahead: its own row and step
    int64_t item_f = item;
    int row_f = 0, step_f = 0, last_f = 0;
    auto enter = [&](int64_t it, int& row, int& first, int& last) {
        row = parts == 1 ? (int)it : (int)(it / parts);
        const int part = parts == 1 ? 0 : (int)(it - (int64_t)row * parts);
        first = steps * part / parts;
        last = steps * (part + 1) / parts;
    };
    if (item < items) enter(item_f, row_f, step_f, last_f);
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(qkn_ring) + threadIdx.x * 16;
    uint32_t slot_f = ring;
    auto fetch = [&]() {
        if (item_f < items) {
            const int it = min(step_f * RPW + group, total - 1);               // past the last head: it again
            const T* src;
            if (it < a.Hq) src = static_cast<const T*>(a.q) + row_f * a.q_row + it * a.q_head;
            else if (it < a.Hq + a.Hk) src = static_cast<const T*>(a.k) + row_f * a.k_row + (it - a.Hq) * a.k_head;
            else src = static_cast<const T*>(a.v) + row_f * a.v_row + (it - a.Hq - a.Hk) * a.v_head;
            cp_async16(slot_f, src + d0);
            cp_async16(slot_f + CHUNK, src + d0 + HALF);
            if (++step_f == last_f) {
                item_f += stride;
                if (item_f < items) enter(item_f, row_f, step_f, last_f);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        slot_f = slot_f == ring + (APP_STAGES - 1) * STAGE ? ring : slot_f + STAGE;
    };
#pragma unroll
    for (int u = 0; u < APP_STAGES - 1; ++u) fetch();
    uint32_t slot_at = ring;
    int row = 0, step = 0, last = 0, pos = 0, cell = 0;
    if (item < items) {
        enter(item, row, step, last);
        pos = __ldg(a.positions + row);
        cell = __ldg(a.slots + row);
    }
    // under the first loads: what all rows share
    for (int d = threadIdx.x; d < 2 * D; d += QKN_WARPS * 32) {
        const T* w = static_cast<const T*>(d < D ? a.wq : a.wk);
        s_gain[d / D][d % D] = w ? (float)w[d % D] : 1.f;
    }
    double theta[AP];
#pragma unroll
    for (int u = 0; u < AP; ++u) theta[u] = exp2(-a.log2_base * (2.0 * (lane + 32 * u) / D));
    __syncthreads();

    if (item >= items) return;
    for (;;) {
        // this row's angles; the next row's position and slot are on their way
        const int64_t next = item + stride;
        int row_n = row, step_n = 0, last_n = 0, pos_n = 0, cell_n = 0;
        if (next < items) {
            enter(next, row_n, step_n, last_n);
            pos_n = __ldg(a.positions + row_n);
            cell_n = __ldg(a.slots + row_n);
        }
        __syncwarp();
#pragma unroll
        for (int u = 0; u < AP; ++u) angle_cos_sin(pos, theta[u], s_ang[warp][0][lane + 32 * u], s_ang[warp][1][lane + 32 * u]);
        __syncwarp();
        float cs[N], sn[N];
#pragma unroll
        for (int u = 0; u < N; u += 4) {
            const float4 c4 = *reinterpret_cast<const float4*>(&s_ang[warp][0][d0 + u]), s4 = *reinterpret_cast<const float4*>(&s_ang[warp][1][d0 + u]);
            cs[u] = c4.x; cs[u + 1] = c4.y; cs[u + 2] = c4.z; cs[u + 3] = c4.w;
            sn[u] = s4.x; sn[u + 1] = s4.y; sn[u + 2] = s4.z; sn[u + 3] = s4.w;
        }
        const bool stored = cell >= 0 && cell < (int64_t)a.n_pages * a.page_size;
        const int page = stored ? cell / a.page_size : 0, in_page = stored ? cell - page * a.page_size : 0;
        T* q_row = static_cast<T*>(a.q_out) + (int64_t)row * a.Hq * D + d0;
        const int64_t kv_row = ((int64_t)page * a.Hk * a.page_size + in_page) * D + d0, kv_head = (int64_t)a.page_size * D;
#pragma unroll 1
        for (; step < last; ++step) {
            fetch();
            asm volatile("cp.async.wait_group %0;" ::"n"(APP_STAGES - 1) : "memory");
            uint4 xl, xh;
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(xl.x), "=r"(xl.y), "=r"(xl.z), "=r"(xl.w) : "r"(slot_at) : "memory");
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(xh.x), "=r"(xh.y), "=r"(xh.z), "=r"(xh.w) : "r"(slot_at + CHUNK) : "memory");
            slot_at = slot_at == ring + (APP_STAGES - 1) * STAGE ? ring : slot_at + STAGE;
            const int it = step * RPW + group;
            const bool is_q = it < a.Hq, is_v = it >= a.Hq + a.Hk;
            if (step * RPW < a.Hq + a.Hk) {   // some head of the step is not a value
                float x[N], y[N];
                V::unpack(xl, x);
                V::unpack(xh, y);
                float ssq = 0.f;
#pragma unroll
                for (int e = 0; e < N; ++e) ssq = fmaf(x[e], x[e], fmaf(y[e], y[e], ssq));
                const float r = rsqrtf(row_sum<LPR>(ssq) * (1.f / D) + a.eps);
                const float* gain = s_gain[is_q ? 0 : 1] + d0;
                float ra[N], rc[N];
#pragma unroll
                for (int u = 0; u < N; u += 4) {
                    const float4 wl = *reinterpret_cast<const float4*>(gain + u), wh = *reinterpret_cast<const float4*>(gain + HALF + u);
                    const float l[4] = {wl.x, wl.y, wl.z, wl.w}, g[4] = {wh.x, wh.y, wh.z, wh.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float ya = x[u + e] * r * l[e], yc = y[u + e] * r * g[e];
                        ra[u + e] = ya * cs[u + e] - yc * sn[u + e];
                        rc[u + e] = yc * cs[u + e] + ya * sn[u + e];
                    }
                }
                if (!is_v) {
                    xl = V::pack(ra);
                    xh = V::pack(rc);
                }
            }
            if (it < total && (is_q || stored)) {
                T* dst = is_q ? q_row + it * D : static_cast<T*>(is_v ? a.v_pool : a.k_pool) + kv_row + (is_v ? it - a.Hq - a.Hk : it - a.Hq) * kv_head;
                *reinterpret_cast<uint4*>(dst) = xl;
                *reinterpret_cast<uint4*>(dst + HALF) = xh;
            }
        }
        if (next >= items) break;
        item = next;
        row = row_n; step = step_n; last = last_n; pos = pos_n; cell = cell_n;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <typename T, int D>
static cudaError_t append_t(const AppendArgs& a, cudaStream_t st) {
    constexpr int RPW = 32 / ((D / 2) / Vec16<T>::N);
    const cudaError_t e = prepare_kernel(reinterpret_cast<const void*>(qk_norm_rope_append_kernel<T, D>), APP_RING);
    if (e != cudaSuccess) return e;
    // few tokens: their heads over several warps, until every SM has eight of them or a warp has one step
    const int steps = (a.Hq + 2 * a.Hk + RPW - 1) / RPW;
    const int parts = (int)std::max<int64_t>(1, std::min<int64_t>(steps, 148 * QKN_WARPS / a.T));
    const int64_t ctas = ((int64_t)a.T * parts + QKN_WARPS - 1) / QKN_WARPS;
    qk_norm_rope_append_kernel<T, D><<<(unsigned)std::min<int64_t>(ctas, 148 * 3), QKN_WARPS * 32, APP_RING, st>>>(a, parts);
    count_launches(1);
    return cudaGetLastError();
}

cudaError_t launch_qk_norm_rope_append(const AppendArgs& a, int D, loma_dtype dt, cudaStream_t st) {
    if (dt == LOMA_F32) return D == 64 ? append_t<float, 64>(a, st) : append_t<float, 128>(a, st);
    return D == 64 ? append_t<__nv_bfloat16, 64>(a, st) : append_t<__nv_bfloat16, 128>(a, st);
}

}  // namespace loma
