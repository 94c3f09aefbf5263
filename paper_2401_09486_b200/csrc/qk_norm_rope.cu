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
// row and add their sums with shuffles.  A lane keeps the cos / sin of its row's id for every (batch, head) it walks.
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

// (batch, head) pairs [p0, p1) of one tensor for the warp's rows.  U rows' loads are issued before the first is used.
// BWD: v.grad is read too, acc[0..N) / acc[N..2N) collect the lane's share of dw.
template <typename T, int D, bool BWD, int U>
__device__ __forceinline__ void walk_pairs(const HeadsView& v, int p0, int p1, int i, bool live, int d0, const float (&cs)[Vec16<T>::N],
                                           const float (&sn)[Vec16<T>::N], float eps, float (&acc)[2 * Vec16<T>::N]) {
    using V = Vec16<T>;
    constexpr int N = V::N, HALF = D / 2, LPR = HALF / N;
    float wl[N], wh[N];
    load_gain(static_cast<const T*>(v.w), d0, wl, wh, HALF);
    const T* in = static_cast<const T*>(v.in) + (int64_t)i * v.ss + d0;
    const T* grad = BWD ? static_cast<const T*>(v.grad) + (int64_t)i * v.ss + d0 : nullptr;
    T* out = static_cast<T*>(v.out) + (int64_t)i * v.ss + d0;
    int b = p0 / v.H, h = p0 - b * v.H;
    for (int p = p0; p < p1; p += U) {
        int64_t off[U];
        uint4 xl[U], xh[U], gl[U], gh[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            off[u] = (int64_t)b * v.sb + (int64_t)h * v.sh;
            if (p + u + 1 < p1 && ++h == v.H) { h = 0; ++b; }   // past the end the last pair is read again
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            xl[u] = __ldcs(reinterpret_cast<const uint4*>(in + off[u]));
            xh[u] = __ldcs(reinterpret_cast<const uint4*>(in + off[u] + HALF));
            if (BWD) {
                gl[u] = __ldcs(reinterpret_cast<const uint4*>(grad + off[u]));
                gh[u] = __ldcs(reinterpret_cast<const uint4*>(grad + off[u] + HALF));
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float a[N], c[N], ra[N], rc[N];
            V::unpack(xl[u], a);
            V::unpack(xh[u], c);
            float ssq = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) ssq = fmaf(a[e], a[e], fmaf(c[e], c[e], ssq));
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
                V::unpack(gl[u], ga);
                V::unpack(gh[u], gc);
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
                const bool counts = live && p + u < p1;   // rows and pairs that were read twice count once
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
            if (live && p + u < p1) {
                __stcs(reinterpret_cast<uint4*>(out + off[u]), V::pack(ra));
                __stcs(reinterpret_cast<uint4*>(out + off[u] + HALF), V::pack(rc));
            }
        }
    }
}

// A CTA takes QKN_WARPS * RPW rows of the laid-out sequence and a slice of the (batch, head) pairs, q's and k's as one list.
// part (backward): [2][CTAs][D] fp32, this CTA's sums of dw.
template <typename T, int D, bool BWD>
__global__ void __launch_bounds__(QKN_WARPS * 32)
qk_norm_rope_kernel(const HeadsView q, const HeadsView k, int B, Layout L, float eps, double log2_base, int position_type,
                    float* __restrict__ part) {
    using V = Vec16<T>;
    constexpr int N = V::N, HALF = D / 2, LPR = HALF / N, RPW = 32 / LPR, U = BWD ? 2 : 4;
    __shared__ double theta[HALF];
    __shared__ float red[BWD ? QKN_WARPS : 1][BWD ? D : 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int d = threadIdx.x; d < HALF; d += QKN_WARPS * 32) theta[d] = exp2(-log2_base * (2.0 * d / D));
    __syncthreads();
    const int row = (blockIdx.x * QKN_WARPS + warp) * RPW + lane / LPR;
    const bool live = row < L.S;
    const int i = min(row, L.S - 1);   // a row past the end reads the last row and writes nothing
    const RowInfo ri = layout_row(i, L.n_chunks, L.c, L.t, L.s);
    const int pos = (position_type & 1) && ri.zone == LOMA_ZONE_MEM ? ri.chunk * L.t + ri.offset : ri.pos;
    const int d0 = (lane % LPR) * N;
    float cs[N], sn[N];
#pragma unroll
    for (int u = 0; u < N; ++u) angle_cos_sin(pos, theta[d0 + u], cs[u], sn[u]);
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
        if (a0 < a1) walk_pairs<T, D, BWD, U>(v, a0, a1, i, live, d0, cs, sn, eps, acc);
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

// rows per CTA and CTAs per row block: enough CTAs to fill the GPU several times over, since every slice computes its rows' angles again
static void norm_grid(int B, int Hq, int Hk, int D, const Layout& L, int elt_bytes, dim3* grid) {
    const int rpw = 32 / ((D / 2) / (16 / elt_bytes));
    const int rows = (L.S + QKN_WARPS * rpw - 1) / (QKN_WARPS * rpw);
    const int pairs = B * (Hq + Hk);
    int slices = 1;
    while (slices < pairs && (int64_t)rows * slices < 148 * 6) slices *= 2;
    *grid = dim3(rows, std::min(slices, pairs));
}

size_t qk_norm_rope_bwd_workspace_bytes(int B, int Hq, int Hk, int D, const Layout& L) {
    size_t most = 0;
    for (int es = 2; es <= 4; es += 2) {
        dim3 g;
        norm_grid(B, Hq, Hk, D, L, es, &g);
        most = std::max(most, (size_t)2 * g.x * g.y * D * sizeof(float));
    }
    return most;
}

template <typename T, int D>
static cudaError_t norm_t(const HeadsView& q, const HeadsView& k, int B, const Layout& L, float eps, double theta_base, int position_type,
                          bool backward, void* ws, cudaStream_t st) {
    dim3 grid;
    norm_grid(B, q.H, k.H, D, L, sizeof(T), &grid);
    if (!backward) {
        qk_norm_rope_kernel<T, D, false><<<grid, QKN_WARPS * 32, 0, st>>>(q, k, B, L, eps, log2(theta_base), position_type, nullptr);
        count_launches(1);
        return cudaGetLastError();
    }
    qk_norm_rope_kernel<T, D, true><<<grid, QKN_WARPS * 32, 0, st>>>(q, k, B, L, eps, log2(theta_base), position_type,
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
// One packed row (token) per blockIdx.x; its Hq + 2 Hk heads are dealt to the warps of gridDim.y CTAs.  The loads of the
// first heads are in flight while the angles are computed.
constexpr int APP_WARPS = 4;

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
    const int first = (blockIdx.y * APP_WARPS + warp) * HPW + lane / LPR;
    uint4 xl, xh;
    {
        const T* src = source(min(first, total - 1));
        xl = __ldg(reinterpret_cast<const uint4*>(src));
        xh = __ldg(reinterpret_cast<const uint4*>(src + HALF));
    }
    const int pos = __ldg(a.positions + row);
    for (int d = threadIdx.x; d < HALF; d += APP_WARPS * 32) angle_cos_sin(pos, exp2(-a.log2_base * (2.0 * d / D)), s_cs[d], s_sn[d]);
    __syncthreads();
    float cs[N], sn[N];
#pragma unroll
    for (int u = 0; u < N; ++u) { cs[u] = s_cs[d0 + u]; sn[u] = s_sn[d0 + u]; }
    const int page = stored ? slot / a.page_size : 0, in_page = stored ? slot - page * a.page_size : 0;
    for (int base = first - lane / LPR; base < total; base += step) {
        const int it = base + lane / LPR;
        uint4 nl = xl, nh = xh;
        if (base + step < total) {   // the next heads while these are worked on
            const T* src = source(min(it + step, total - 1));
            nl = __ldg(reinterpret_cast<const uint4*>(src));
            nh = __ldg(reinterpret_cast<const uint4*>(src + HALF));
        }
        const bool is_q = it < a.Hq, is_v = it >= a.Hq + a.Hk;
        float x[N], y[N], wl[N], wh[N];
        V::unpack(xl, x);
        V::unpack(xh, y);
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
            xl = V::pack(ra);
            xh = V::pack(rc);
        }
        if (it < total && (is_q || stored)) {
            T* dst;
            if (is_q) {
                dst = static_cast<T*>(a.q_out) + (row * a.Hq + it) * D;
            } else {
                const int h = is_v ? it - a.Hq - a.Hk : it - a.Hq;
                dst = static_cast<T*>(is_v ? a.v_pool : a.k_pool) + (((int64_t)page * a.Hk + h) * a.page_size + in_page) * D;
            }
            *reinterpret_cast<uint4*>(dst + d0) = xl;
            *reinterpret_cast<uint4*>(dst + d0 + HALF) = xh;
        }
        xl = nl;
        xh = nh;
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
