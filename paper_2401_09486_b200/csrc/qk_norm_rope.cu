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

// cos and sin of pos * theta, the angle formed and reduced in double (see rope_cos_sin)
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

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
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
static void norm_grid(int B, int Hq, int Hk, int D, const Layout& L, int elt_bytes, bool by_heads, dim3* grid) {
    const int rpw = 32 / ((D / 2) / (16 / elt_bytes));
    const int rows = (L.S + QKN_WARPS * (by_heads ? 1 : rpw) - 1) / (QKN_WARPS * (by_heads ? 1 : rpw));
    const int pairs = B * (Hq + Hk), lane_pairs = by_heads ? (pairs + rpw - 1) / rpw : pairs;
    int slices = 1;
    while (slices < lane_pairs &&
           ((int64_t)rows * slices < 148 * 2 || ((int64_t)rows * slices < 148 * 6 && lane_pairs / slices >= 32)))
        slices *= 2;
    *grid = dim3(rows, std::min(slices, lane_pairs));
}

size_t qk_norm_rope_bwd_workspace_bytes(int B, int Hq, int Hk, int D, const Layout& L) {
    size_t most = 0;
    for (int es = 2; es <= 4; es += 2)
        for (int by = 0; by < 2; ++by) {
            dim3 g;
            norm_grid(B, Hq, Hk, D, L, es, by != 0, &g);
            most = std::max(most, (size_t)2 * g.x * g.y * D * sizeof(float));
        }
    return most;
}

template <typename T, int D>
static cudaError_t norm_t(const HeadsView& q, const HeadsView& k, int B, const Layout& L, float eps, double theta_base, int position_type,
                          bool backward, void* ws, cudaStream_t st) {
    const HeadsView& lead = q.H > 0 ? q : k;
    const bool by_heads = lead.H > 1 && lead.sh < lead.ss;   // heads of a row behind one another: [B, S, H, D]
    dim3 grid;
    norm_grid(B, q.H, k.H, D, L, sizeof(T), by_heads, &grid);
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
    qk_norm_dw_kernel<T><<<dim3(D / 32, 2), dim3(32, 32), 0, st>>>(static_cast<const float*>(ws), grid.x * grid.y, D,
                                                                   static_cast<T*>(q.dw), static_cast<T*>(k.dw));
    count_launches(1);
    return cudaGetLastError();
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
// One packed row (token) per blockIdx.x; its Hq + 2 Hk heads are dealt to the warps of gridDim.y CTAs.  A lane's first
// AT_ONCE heads are all in flight while the angles are computed.
constexpr int APP_WARPS = 4, AT_ONCE = 4;

template <typename T, int D>
__global__ void __launch_bounds__(APP_WARPS * 32)
qk_norm_rope_append_kernel(const AppendArgs a) {
    using V = Vec16<T>;
    constexpr int N = V::N, HALF = D / 2, LPR = HALF / N, HPW = 32 / LPR;   // heads per warp access
    __shared__ float s_cs[HALF], s_sn[HALF];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, d0 = (lane % LPR) * N;
    const int64_t row = blockIdx.x;
    const int total = a.Hq + 2 * a.Hk, step = gridDim.y * APP_WARPS * HPW;
    const int slot = __ldg(a.slots + row);
    const bool stored = slot >= 0 && slot < (int64_t)a.n_pages * a.page_size;
    auto source = [&](int it) -> const T* {
        if (it < a.Hq) return static_cast<const T*>(a.q) + row * a.q_row + it * a.q_head + d0;
        if (it < a.Hq + a.Hk) return static_cast<const T*>(a.k) + row * a.k_row + (it - a.Hq) * a.k_head + d0;
        return static_cast<const T*>(a.v) + row * a.v_row + (it - a.Hq - a.Hk) * a.v_head + d0;
    };
    // the heads this lane works on, AT_ONCE of them in flight at a time
    const int first = (blockIdx.y * APP_WARPS + warp) * HPW;
    uint4 xl[AT_ONCE], xh[AT_ONCE];
    auto load = [&](int base) {
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const T* src = source(min(base + u * step + lane / LPR, total - 1));
            if (base + u * step < total) {
                xl[u] = __ldcs(reinterpret_cast<const uint4*>(src));
                xh[u] = __ldcs(reinterpret_cast<const uint4*>(src + HALF));
            }
        }
    };
    load(first);
    const int pos = __ldg(a.positions + row);
    for (int d = threadIdx.x; d < HALF; d += APP_WARPS * 32) angle_cos_sin(pos, exp2(-a.log2_base * (2.0 * d / D)), s_cs[d], s_sn[d]);
    __syncthreads();
    float cs[N], sn[N];
#pragma unroll
    for (int u = 0; u < N; ++u) { cs[u] = s_cs[d0 + u]; sn[u] = s_sn[d0 + u]; }
    const int page = stored ? slot / a.page_size : 0, in_page = stored ? slot - page * a.page_size : 0;
    for (int base = first; base < total; base += AT_ONCE * step) {
        if (base > first) load(base);
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            if (base + u * step >= total) break;
            const int it = base + u * step + lane / LPR;
            const bool is_q = it < a.Hq, is_v = it >= a.Hq + a.Hk;
            float x[N], y[N], wl[N], wh[N];
            V::unpack(xl[u], x);
            V::unpack(xh[u], y);
            load_gain(static_cast<const T*>(is_q ? a.wq : a.wk), d0, wl, wh, HALF);
            float ssq = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) ssq = fmaf(x[e], x[e], fmaf(y[e], y[e], ssq));
            const float r = rsqrtf(row_sum<LPR>(ssq) * (1.f / D) + a.eps);
            if (!is_v) {
                float ra[N], rc[N];
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float ya = x[e] * r * wl[e], yc = y[e] * r * wh[e];
                    ra[e] = ya * cs[e] - yc * sn[e];
                    rc[e] = yc * cs[e] + ya * sn[e];
                }
                xl[u] = V::pack(ra);
                xh[u] = V::pack(rc);
            }
            if (it < total && (is_q || stored)) {
                T* dst;
                if (is_q) {
                    dst = static_cast<T*>(a.q_out) + (row * a.Hq + it) * D;
                } else {
                    const int h = is_v ? it - a.Hq - a.Hk : it - a.Hq;
                    dst = static_cast<T*>(is_v ? a.v_pool : a.k_pool) + (((int64_t)page * a.Hk + h) * a.page_size + in_page) * D;
                }
                *reinterpret_cast<uint4*>(dst + d0) = xl[u];
                *reinterpret_cast<uint4*>(dst + d0 + HALF) = xh[u];
            }
        }
    }
}

template <typename T, int D>
static cudaError_t append_t(const AppendArgs& a, cudaStream_t st) {
    constexpr int HPW = 32 / ((D / 2) / Vec16<T>::N);
    const int most = (a.Hq + 2 * a.Hk + APP_WARPS * HPW - 1) / (APP_WARPS * HPW);
    int split = 1;   // few tokens: their heads over several CTAs
    while (split < most && (int64_t)a.T * split < 148 * 4) ++split;
    qk_norm_rope_append_kernel<T, D><<<dim3(a.T, split), APP_WARPS * 32, 0, st>>>(a);
    count_launches(1);
    return cudaGetLastError();
}

cudaError_t launch_qk_norm_rope_append(const AppendArgs& a, int D, loma_dtype dt, cudaStream_t st) {
    if (dt == LOMA_F32) return D == 64 ? append_t<float, 64>(a, st) : append_t<float, 128>(a, st);
    return D == 64 ? append_t<__nv_bfloat16, 64>(a, st) : append_t<__nv_bfloat16, 128>(a, st);
}

}  // namespace loma
