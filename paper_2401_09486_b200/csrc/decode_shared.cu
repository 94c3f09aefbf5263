// Decode attention for a batch whose sequences share a long prefix (loma_decode_attn_shared and its paged form).
//
// Query head hq of sequence b sees the prefix's keys of kv head hq div g (g = Hq / Hkv), then the sequence's own cache
// and its new token, under one softmax.  A softmax over a union of key sets is the mean of the softmaxes over the parts
// with weights 2^(lse_i - max), so the parts are computed where they are cheap and joined at the end:
//
//   prefix   all B g query rows of a kv head against the same K and V: a matrix product, 128 rows at a time, that reads
//            the prefix once for the batch instead of once per sequence (bf16: tcgen05, decode_shared_tc.cu; fp32 and
//            page sizes below 8: shared_prefix_simt_kernel)
//   own      one query row per head of a group against rows nobody else reads: a stream bound by HBM.  bf16:
//            shared_own_mma_kernel, where the g heads of a kv head are rows of a warp-level m16n8k16 product, so a K or
//            V row is loaded once for all of them; fp32: shared_own_stream_kernel on CUDA cores
//   merge    one thread per query row and four features adds the parts in a fixed order (results repeat bit for bit)
#include <math.h>

#include "decode_shared.cuh"

namespace loma {

__device__ __forceinline__ uint4 ld_stream16(const void* p) {
    uint4 r;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
    return r;
}

// length of sequence b's own cache, negative for a slot of the batch without a request
__device__ __forceinline__ int own_length(const SharedArgs& a, int b) { return min(__ldg(a.cache_lens + b), a.max_len); }

// row of own entry j of (b, h), in elements of D, from the start of the cache or pool
__device__ __forceinline__ int64_t own_row(const SharedArgs& a, int b, int h, int j) {
    if (!a.pg.table) return ((int64_t)b * a.Hkv + h) * a.cap + j;
    const int page = min(max(__ldg(a.pg.table + (int64_t)b * a.pg.max_pages + (j >> a.pg.log2_ps)), 0), a.pg.n_pages - 1);
    return ((((int64_t)page * a.Hkv + h) << a.pg.log2_ps) + (j & ((1 << a.pg.log2_ps) - 1)));
}

__device__ __forceinline__ int64_t prefix_row(const SharedArgs& a, int h, int j) {
    if (!a.prefix_table) return (int64_t)h * a.prefix_cap + j;
    const int page = min(max(__ldg(a.prefix_table + (j >> a.pg.log2_ps)), 0), a.pg.n_pages - 1);
    return ((((int64_t)page * a.Hkv + h) << a.pg.log2_ps) + (j & ((1 << a.pg.log2_ps) - 1)));
}

// ------------------------------------------------------------------ own cache, bf16
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

constexpr int OWN_WARPS = 4;

// One CTA: one (sequence, kv head, key range) and up to 8 R heads of the group (R = 1, 2).  A warp takes 16 keys at a time.
// The contraction over d and the columns of the output may be permuted freely as long as both operands agree, so K and V
// go from global memory straight into the fragments with 16-byte loads, without shared memory:
//   scores   lane (r = lane / 4, j = lane % 4) loads bytes 16 (4 i + j) .. of key row r (and r + 8); its 8 features are
//            the lane's contraction slots of two k-steps, and the q fragments are loaded the same way
//   P V      the lane loads features 64 f + 8 r .. + 7 of key rows 2j, 2j+1, 2j+8, 2j+9; feature e of the 8 belongs to
//            output tile (f, e), whose column n = r is feature 64 f + 8 r + e; pairs of rows are packed by byte permutes
template <int D, int R>
__global__ void __launch_bounds__(OWN_WARPS * 32)
shared_own_mma_kernel(const SharedArgs a, const SharedPlan p) {
    constexpr int KC = D / 32, VF = D / 64;   // 16-byte chunks of a K row per lane; 64-feature parts of a V row
    __shared__ float s_m[OWN_WARPS][8 * R], s_l[OWN_WARPS][8 * R];
    __shared__ __align__(16) float s_o[OWN_WARPS][8 * R][D + 4];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, j = lane & 3;
    const int g_tiles = (a.g + 8 * R - 1) / (8 * R);
    int x = blockIdx.x;
    const int split = x % p.own_splits; x /= p.own_splits;
    const int gt = x % g_tiles; x /= g_tiles;
    const int h = x % a.Hkv, b = x / a.Hkv;
    const int len = own_length(a, b);
    if (len < 0) return;
    const int heads = min(8 * R, a.g - gt * 8 * R), head0 = h * a.g + gt * 8 * R;
    const int begin = split * p.own_len, end = min(len + 1, begin + p.own_len);   // key len is the new token
    const float scale_log2 = a.scale * 1.4426950408889634f;
    const __nv_bfloat16* kc = static_cast<const __nv_bfloat16*>(a.k_cache);
    const __nv_bfloat16* vc = static_cast<const __nv_bfloat16*>(a.v_cache);
    const __nv_bfloat16* kn = a.k_new ? static_cast<const __nv_bfloat16*>(a.k_new) + ((int64_t)b * a.Hkv + h) * D : nullptr;
    const __nv_bfloat16* vn = a.v_new ? static_cast<const __nv_bfloat16*>(a.v_new) + ((int64_t)b * a.Hkv + h) * D : nullptr;
    // every key index is clamped to the sequence's last visible entry: no row of another sequence is ever read
    auto k_ptr = [&](int key) { key = min(key, len); return key == len && kn ? kn : kc + own_row(a, b, h, key) * D; };
    auto v_ptr = [&](int key) { key = min(key, len); return key == len && vn ? vn : vc + own_row(a, b, h, key) * D; };

    uint32_t qf[R][KC][4];
#pragma unroll
    for (int t = 0; t < R; ++t) {
        const int hd = t * 8 + r;
        const __nv_bfloat16* qp = static_cast<const __nv_bfloat16*>(a.q) + ((int64_t)b * a.Hq + head0 + min(hd, heads - 1)) * D;
#pragma unroll
        for (int i = 0; i < KC; ++i) {
            uint4 v = __ldg(reinterpret_cast<const uint4*>(qp + (4 * i + j) * 8));
            if (hd >= heads) v = make_uint4(0, 0, 0, 0);
            qf[t][i][0] = v.x; qf[t][i][1] = v.y; qf[t][i][2] = v.z; qf[t][i][3] = v.w;
        }
    }
    float m[R], l[R], acc[R][VF * 8][2];
#pragma unroll
    for (int t = 0; t < R; ++t) {
        m[t] = -INFINITY;
        l[t] = 0.f;
#pragma unroll
        for (int n = 0; n < VF * 8; ++n) acc[t][n][0] = acc[t][n][1] = 0.f;
    }
    uint4 kr[2][KC], vr[4][VF];
    auto load_k = [&](int key0) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const __nv_bfloat16* kp = k_ptr(key0 + n * 8 + r) + j * 8;
#pragma unroll
            for (int i = 0; i < KC; ++i) kr[n][i] = ld_stream16(kp + 32 * i);
        }
    };
    int key0 = begin + warp * 16;
    if (key0 < end) load_k(key0);
    for (; key0 < end; key0 += OWN_WARPS * 16) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const __nv_bfloat16* vp = v_ptr(key0 + 2 * j + (u & 1) + (u >> 1) * 8) + r * 8;
#pragma unroll
            for (int f = 0; f < VF; ++f) vr[u][f] = ld_stream16(vp + 64 * f);
        }
        float s[R][2][2];   // head t*8 + r, keys n*8 + 2j, +1
#pragma unroll
        for (int n = 0; n < 2; ++n) {
#pragma unroll
            for (int t = 0; t < R; ++t) s[t][n][0] = s[t][n][1] = 0.f;
#pragma unroll
            for (int i = 0; i < KC; ++i) {
                if constexpr (R == 1) {
                    mma_lo(s[0][n], qf[0][i][0], qf[0][i][1], kr[n][i].x, kr[n][i].y);
                    mma_lo(s[0][n], qf[0][i][2], qf[0][i][3], kr[n][i].z, kr[n][i].w);
                } else {
                    mma_full(s[0][n], s[1][n], qf[0][i][0], qf[1][i][0], qf[0][i][1], qf[1][i][1], kr[n][i].x, kr[n][i].y);
                    mma_full(s[0][n], s[1][n], qf[0][i][2], qf[1][i][2], qf[0][i][3], qf[1][i][3], kr[n][i].z, kr[n][i].w);
                }
            }
        }
        const int next = key0 + OWN_WARPS * 16;
        if (next < end) load_k(next);   // in flight during the softmax and P V of this block
        uint32_t pf[R][2];              // P rounded to bf16: off by 2^-8 of its value at most; the sums stay in fp32
#pragma unroll
        for (int t = 0; t < R; ++t) {
            float mx = -INFINITY;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    s[t][n][e] = key0 + n * 8 + 2 * j + e < end ? s[t][n][e] * scale_log2 : -INFINITY;
                    mx = fmaxf(mx, s[t][n][e]);
                }
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
            const float m_new = fmaxf(m[t], mx), ref = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = exp2f(m[t] - ref);
            m[t] = m_new;
            l[t] *= alpha;
#pragma unroll
            for (int n = 0; n < VF * 8; ++n) { acc[t][n][0] *= alpha; acc[t][n][1] *= alpha; }
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const float p0 = exp2f(s[t][n][0] - ref), p1 = exp2f(s[t][n][1] - ref);
                l[t] += p0 + p1;
                pf[t][n] = pack_bf16(p0, p1);
            }
        }
#pragma unroll
        for (int f = 0; f < VF; ++f) {
            const uint32_t* w0 = reinterpret_cast<const uint32_t*>(&vr[0][f]);
            const uint32_t* w1 = reinterpret_cast<const uint32_t*>(&vr[1][f]);
            const uint32_t* w2 = reinterpret_cast<const uint32_t*>(&vr[2][f]);
            const uint32_t* w3 = reinterpret_cast<const uint32_t*>(&vr[3][f]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t sel = (e & 1) ? 0x7632u : 0x5410u;
                const uint32_t b0 = __byte_perm(w0[e >> 1], w1[e >> 1], sel), b1 = __byte_perm(w2[e >> 1], w3[e >> 1], sel);
                if constexpr (R == 1) mma_lo(acc[0][f * 8 + e], pf[0][0], pf[0][1], b0, b1);
                else mma_full(acc[0][f * 8 + e], acc[1][f * 8 + e], pf[0][0], pf[1][0], pf[0][1], pf[1][1], b0, b1);
            }
        }
    }
    // the quad's shares of the row sums, then the CTA's warps in shared memory
#pragma unroll
    for (int t = 0; t < R; ++t) {
        l[t] += __shfl_xor_sync(0xffffffffu, l[t], 1);
        l[t] += __shfl_xor_sync(0xffffffffu, l[t], 2);
        if (j == 0) { s_m[warp][t * 8 + r] = m[t]; s_l[warp][t * 8 + r] = l[t]; }
#pragma unroll
        for (int f = 0; f < VF; ++f)
#pragma unroll
            for (int c = 0; c < 2; ++c)   // accumulator column 2j + c of tile (f, e) is feature 64 f + 8 (2j + c) + e
#pragma unroll
                for (int e = 0; e < 8; e += 4)
                    *reinterpret_cast<float4*>(&s_o[warp][t * 8 + r][64 * f + 8 * (2 * j + c) + e]) =
                        make_float4(acc[t][f * 8 + e][c], acc[t][f * 8 + e + 1][c], acc[t][f * 8 + e + 2][c], acc[t][f * 8 + e + 3][c]);
    }
    __syncthreads();
    float* ws = static_cast<float*>(a.ws);
    const int64_t out = (((int64_t)b * a.Hkv + h) * p.own_splits + split) * a.g + gt * 8 * R;
    for (int idx = threadIdx.x; idx < heads * D; idx += OWN_WARPS * 32) {
        const int hd = idx / D, d = idx - hd * D;
        float M = s_m[0][hd];
#pragma unroll
        for (int w = 1; w < OWN_WARPS; ++w) M = fmaxf(M, s_m[w][hd]);
        if (M == -INFINITY) {
            if (d == 0) ws[p.own_lse + out + hd] = -INFINITY;
            continue;
        }
        float lt = 0.f, ot = 0.f;
#pragma unroll
        for (int w = 0; w < OWN_WARPS; ++w) {
            const float f = exp2f(s_m[w][hd] - M);
            lt = fmaf(s_l[w][hd], f, lt);
            ot = fmaf(s_o[w][hd][d], f, ot);
        }
        ws[p.own_o + (out + hd) * D + d] = ot / lt;
        if (d == 0) ws[p.own_lse + out + hd] = M + log2f(lt);
    }
    // the new token's K and V go to slot len (read by nobody in this launch)
    if (kn && split == 0 && gt == 0 && threadIdx.x < D / 8) {
        const int64_t row = own_row(a, b, h, len) * D;
        reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.k_cache) + row)[threadIdx.x] = __ldg(reinterpret_cast<const uint4*>(kn) + threadIdx.x);
        reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.v_cache) + row)[threadIdx.x] = __ldg(reinterpret_cast<const uint4*>(vn) + threadIdx.x);
    }
}

// ------------------------------------------------------------------ own cache on CUDA cores (fp32, second opinion)
// The lanes that share a row hold 16 bytes of it each; G heads of the group per CTA, so a row is loaded once for them.
template <typename T, int D, int G>
__global__ void __launch_bounds__(OWN_WARPS * 32)
shared_own_stream_kernel(const SharedArgs a, const SharedPlan p) {
    using V = Vec16<T>;
    constexpr int N = V::N, LPK = D / N, KPL = 32 / LPK, NL = 4, BK = NL * KPL;
    __shared__ float s_m[OWN_WARPS][G], s_l[OWN_WARPS][G];
    __shared__ __align__(16) float s_o[OWN_WARPS][G][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / LPK, li = lane % LPK;
    const int g_tiles = (a.g + G - 1) / G;
    int x = blockIdx.x;
    const int split = x % p.own_splits; x /= p.own_splits;
    const int gt = x % g_tiles; x /= g_tiles;
    const int h = x % a.Hkv, b = x / a.Hkv;
    const int len = own_length(a, b);
    if (len < 0) return;
    const int heads = min(G, a.g - gt * G), head0 = h * a.g + gt * G;
    const int begin = split * p.own_len, end = min(len + 1, begin + p.own_len);
    const float scale_log2 = a.scale * 1.4426950408889634f;
    const T* kn = a.k_new ? static_cast<const T*>(a.k_new) + ((int64_t)b * a.Hkv + h) * D : nullptr;
    const T* vn = a.v_new ? static_cast<const T*>(a.v_new) + ((int64_t)b * a.Hkv + h) * D : nullptr;
    float q[G][N], acc[G][N], m[G], l[G];
#pragma unroll
    for (int t = 0; t < G; ++t) {
        const T* qp = static_cast<const T*>(a.q) + ((int64_t)b * a.Hq + head0 + min(t, heads - 1)) * D;
        V::unpack(__ldg(reinterpret_cast<const uint4*>(qp) + li), q[t]);
#pragma unroll
        for (int e = 0; e < N; ++e) { q[t][e] *= scale_log2; acc[t][e] = 0.f; }
        m[t] = -INFINITY;
        l[t] = 0.f;
    }
    for (int j0 = begin + warp * BK; j0 < end; j0 += OWN_WARPS * BK) {
        uint4 kr[NL], vr[NL];
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int key = min(j0 + i * KPL + sub, len);
            const int64_t row = key == len && kn ? 0 : own_row(a, b, h, key) * D;
            kr[i] = ld_stream16((key == len && kn ? kn : static_cast<const T*>(a.k_cache) + row) + li * N);
            vr[i] = ld_stream16((key == len && vn ? vn : static_cast<const T*>(a.v_cache) + row) + li * N);
        }
#pragma unroll
        for (int t = 0; t < G; ++t) {
            float s[NL], mb = -INFINITY;
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                float kf[N];
                V::unpack(kr[i], kf);
                s[i] = 0.f;
#pragma unroll
                for (int e = 0; e < N; ++e) s[i] = fmaf(q[t][e], kf[e], s[i]);
            }
#pragma unroll
            for (int o = LPK / 2; o > 0; o >>= 1)
#pragma unroll
                for (int i = 0; i < NL; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                s[i] = j0 + i * KPL + sub < end ? s[i] : -INFINITY;
                mb = fmaxf(mb, s[i]);
            }
#pragma unroll
            for (int o = 16; o >= LPK; o >>= 1) mb = fmaxf(mb, __shfl_xor_sync(0xffffffffu, mb, o));
            const float m_new = fmaxf(m[t], mb), ref = m_new == -INFINITY ? 0.f : m_new, alpha = exp2f(m[t] - ref);
            m[t] = m_new;
            l[t] *= alpha;
#pragma unroll
            for (int e = 0; e < N; ++e) acc[t][e] *= alpha;
#pragma unroll
            for (int i = 0; i < NL; ++i) {
                const float pr = exp2f(s[i] - ref);
                float vf[N];
                V::unpack(vr[i], vf);
                l[t] += pr;
#pragma unroll
                for (int e = 0; e < N; ++e) acc[t][e] = fmaf(pr, vf[e], acc[t][e]);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < G; ++t) {
#pragma unroll
        for (int o = 16; o >= LPK; o >>= 1) {
            l[t] += __shfl_xor_sync(0xffffffffu, l[t], o);
#pragma unroll
            for (int e = 0; e < N; ++e) acc[t][e] += __shfl_xor_sync(0xffffffffu, acc[t][e], o);
        }
        if (lane < LPK)
#pragma unroll
            for (int e = 0; e < N; ++e) s_o[warp][t][li * N + e] = acc[t][e];
        if (lane == 0) { s_m[warp][t] = m[t]; s_l[warp][t] = l[t]; }
    }
    __syncthreads();
    float* ws = static_cast<float*>(a.ws);
    const int64_t out = (((int64_t)b * a.Hkv + h) * p.own_splits + split) * a.g + gt * G;
    for (int idx = threadIdx.x; idx < heads * D; idx += OWN_WARPS * 32) {
        const int hd = idx / D, d = idx - hd * D;
        float M = -INFINITY, lt = 0.f, ot = 0.f;
#pragma unroll
        for (int w = 0; w < OWN_WARPS; ++w) M = fmaxf(M, s_m[w][hd]);
        if (M == -INFINITY) {
            if (d == 0) ws[p.own_lse + out + hd] = -INFINITY;
            continue;
        }
#pragma unroll
        for (int w = 0; w < OWN_WARPS; ++w) {
            const float f = exp2f(s_m[w][hd] - M);
            lt = fmaf(s_l[w][hd], f, lt);
            ot = fmaf(s_o[w][hd][d], f, ot);
        }
        ws[p.own_o + (out + hd) * D + d] = ot / lt;
        if (d == 0) ws[p.own_lse + out + hd] = M + log2f(lt);
    }
    if (kn && split == 0 && gt == 0 && threadIdx.x < LPK) {
        const int64_t row = own_row(a, b, h, len) * D;
        reinterpret_cast<uint4*>(static_cast<T*>(a.k_cache) + row)[threadIdx.x] = __ldg(reinterpret_cast<const uint4*>(kn) + threadIdx.x);
        reinterpret_cast<uint4*>(static_cast<T*>(a.v_cache) + row)[threadIdx.x] = __ldg(reinterpret_cast<const uint4*>(vn) + threadIdx.x);
    }
}

// ------------------------------------------------------------------ prefix on CUDA cores (fp32, small pages, second opinion)
// 32 query rows against 64 keys at a time, all in fp32 in shared memory: scores with 2 x 4 and outputs with 4 x (D / 32)
// values per thread in registers.  Query row m of kv head h is head h g + m mod g of sequence m / g.
constexpr int SIMT_R = 32, SIMT_K = 64, SIMT_THREADS = 256;

template <typename T, int D>
struct SimtSmem {
    static constexpr int Q = 0, K = Q + SIMT_R * (D + 4), V = K + SIMT_K * (D + 4), S = V + SIMT_K * D, ML = S + SIMT_R * (SIMT_K + 4),
                         FLOATS = ML + 3 * SIMT_R;
};

template <typename T, int D>
__global__ void __launch_bounds__(SIMT_THREADS)
shared_prefix_simt_kernel(const SharedArgs a, const SharedPlan p) {
    using V = Vec16<T>;
    using SM = SimtSmem<T, D>;
    constexpr int N = V::N, LPK = D / N, DC = D / 32;   // output features per thread: 4 rows x DC
    extern __shared__ __align__(16) float sm[];
    const int tid = threadIdx.x, rows = a.B * a.g;
    const int h = blockIdx.y, split = blockIdx.z, row0 = blockIdx.x * SIMT_R;
    const int begin = split * p.p_len, end = min(a.prefix_len, begin + p.p_len);
    const float scale_log2 = a.scale * 1.4426950408889634f;
    for (int idx = tid; idx < SIMT_R * LPK; idx += SIMT_THREADS) {
        const int r = idx / LPK, c = idx - r * LPK, m = min(row0 + r, rows - 1);
        const T* qp = static_cast<const T*>(a.q) + ((int64_t)(m / a.g) * a.Hq + h * a.g + m % a.g) * D;
        float f[N];
        V::unpack(__ldg(reinterpret_cast<const uint4*>(qp) + c), f);
#pragma unroll
        for (int e = 0; e < N; ++e) sm[SM::Q + r * (D + 4) + c * N + e] = f[e] * scale_log2;
    }
    if (tid < SIMT_R) { sm[SM::ML + tid] = -INFINITY; sm[SM::ML + SIMT_R + tid] = 0.f; }
    float acc[4][DC];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int c = 0; c < DC; ++c) acc[u][c] = 0.f;
    const int sr = (tid >> 4) * 2, sk = tid & 15;         // scores: rows sr, sr+1; keys sk + 16 u
    const int orow = (tid >> 5) * 4, oc = tid & 31;       // outputs: rows orow .. +3 (a warp's own); features oc*DC ..
    for (int k0 = begin; k0 < end; k0 += SIMT_K) {
        __syncthreads();
        for (int idx = tid; idx < SIMT_K * LPK; idx += SIMT_THREADS) {
            const int r = idx / LPK, c = idx - r * LPK;
            const int64_t row = prefix_row(a, h, min(k0 + r, a.prefix_len - 1)) * D;   // keys past the end repeat the last one
            float f[N];
            V::unpack(__ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(a.k_prefix) + row) + c), f);
#pragma unroll
            for (int e = 0; e < N; ++e) sm[SM::K + r * (D + 4) + c * N + e] = f[e];
            V::unpack(__ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(a.v_prefix) + row) + c), f);
#pragma unroll
            for (int e = 0; e < N; ++e) sm[SM::V + r * D + c * N + e] = f[e];
        }
        __syncthreads();
        float s[2][4] = {};
#pragma unroll 4
        for (int d = 0; d < D; d += 4) {
            float4 qv[2], kv[4];
#pragma unroll
            for (int u = 0; u < 2; ++u) qv[u] = *reinterpret_cast<const float4*>(&sm[SM::Q + (sr + u) * (D + 4) + d]);
#pragma unroll
            for (int u = 0; u < 4; ++u) kv[u] = *reinterpret_cast<const float4*>(&sm[SM::K + (sk + 16 * u) * (D + 4) + d]);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    s[u][w] = fmaf(qv[u].x, kv[w].x, fmaf(qv[u].y, kv[w].y, fmaf(qv[u].z, kv[w].z, fmaf(qv[u].w, kv[w].w, s[u][w]))));
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {   // 16 lanes share a row
            float mx = -INFINITY;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if (k0 + sk + 16 * w >= end) s[u][w] = -INFINITY;
                mx = fmaxf(mx, s[u][w]);
            }
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float m_old = sm[SM::ML + sr + u], m_new = fmaxf(m_old, mx), ref = m_new == -INFINITY ? 0.f : m_new;
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
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
                sm[SM::ML + SIMT_R + sr + u] = sm[SM::ML + SIMT_R + sr + u] * alpha + sum;
                sm[SM::ML + 2 * SIMT_R + sr + u] = alpha;
            }
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float alpha = sm[SM::ML + 2 * SIMT_R + orow + u];
#pragma unroll
            for (int c = 0; c < DC; ++c) acc[u][c] *= alpha;
        }
#pragma unroll 4
        for (int k = 0; k < SIMT_K; k += 4) {
            float4 pv[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) pv[u] = *reinterpret_cast<const float4*>(&sm[SM::S + (orow + u) * (SIMT_K + 4) + k]);
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                float vv[DC];
#pragma unroll
                for (int c = 0; c < DC; ++c) vv[c] = sm[SM::V + (k + kk) * D + oc * DC + c];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float pr = kk == 0 ? pv[u].x : kk == 1 ? pv[u].y : kk == 2 ? pv[u].z : pv[u].w;
#pragma unroll
                    for (int c = 0; c < DC; ++c) acc[u][c] = fmaf(pr, vv[c], acc[u][c]);
                }
            }
        }
    }
    __syncthreads();
    float* ws = static_cast<float*>(a.ws);
    const int mt = row0 / SHP_ROWS, r_in = row0 % SHP_ROWS;
    const int64_t tile = ((int64_t)split * a.Hkv + h) * p.m_tiles + mt;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const float inv = 1.f / sm[SM::ML + SIMT_R + orow + u];
#pragma unroll
        for (int c = 0; c < DC; ++c) {
            const int d = oc * DC + c;
            ws[p.p_o + tile * SHP_ROWS * D + ((int64_t)(d >> 2) * SHP_ROWS + r_in + orow + u) * 4 + (d & 3)] = acc[u][c] * inv;
        }
    }
    if (tid < SIMT_R) ws[p.p_lse + tile * SHP_ROWS + r_in + tid] = sm[SM::ML + tid] + log2f(sm[SM::ML + SIMT_R + tid]);
}

// ------------------------------------------------------------------ merge
// CTA: 32 query rows of one kv head (lanes) x 8 groups of 4 features (warps).
constexpr int MERGE_THREADS = 256;

template <typename T, int D>
__global__ void __launch_bounds__(MERGE_THREADS)
shared_merge_kernel(const SharedArgs a, const SharedPlan p) {
    const int lane = threadIdx.x & 31, c4 = blockIdx.y * 8 + (threadIdx.x >> 5);
    const int h = blockIdx.z, row = blockIdx.x * 32 + lane;
    if (row >= a.B * a.g) return;
    const int b = row / a.g, j = row - b * a.g;
    if (__ldg(a.cache_lens + b) < 0) return;
    const float* ws = static_cast<const float*>(a.ws);
    const int mt = row / SHP_ROWS, r = row - mt * SHP_ROWS;
    const int64_t tile0 = (int64_t)h * p.m_tiles + mt, tile_step = (int64_t)a.Hkv * p.m_tiles;
    const int64_t own0 = ((int64_t)b * a.Hkv + h) * p.own_splits * a.g + j;
    float M = -INFINITY;
    for (int s = 0; s < p.p_splits; ++s) M = fmaxf(M, ws[p.p_lse + (tile0 + s * tile_step) * SHP_ROWS + r]);
    for (int s = 0; s < p.own_splits; ++s) M = fmaxf(M, ws[p.own_lse + own0 + (int64_t)s * a.g]);
    float total = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float lse, const float* part) {
        if (lse == -INFINITY) return;   // an empty range: its outputs were never written
        const float w = exp2f(lse - M);
        const float4 x = *reinterpret_cast<const float4*>(part);
        total += w;
        o.x = fmaf(w, x.x, o.x); o.y = fmaf(w, x.y, o.y); o.z = fmaf(w, x.z, o.z); o.w = fmaf(w, x.w, o.w);
    };
#pragma unroll 4
    for (int s = 0; s < p.p_splits; ++s) {
        const int64_t tile = tile0 + s * tile_step;
        add(ws[p.p_lse + tile * SHP_ROWS + r], ws + p.p_o + tile * SHP_ROWS * D + ((int64_t)c4 * SHP_ROWS + r) * 4);
    }
#pragma unroll 2
    for (int s = 0; s < p.own_splits; ++s) {
        const int64_t own = own0 + (int64_t)s * a.g;
        add(ws[p.own_lse + own], ws + p.own_o + own * D + c4 * 4);
    }
    const float inv = 1.f / total;
    const int64_t out = (int64_t)b * a.Hq + h * a.g + j;
    if constexpr (sizeof(T) == 2)
        *reinterpret_cast<uint2*>(static_cast<T*>(a.o) + out * D + c4 * 4) =
            make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    else
        *reinterpret_cast<float4*>(static_cast<T*>(a.o) + out * D + c4 * 4) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    if (a.lse && c4 == 0) a.lse[out] = (M + log2f(total)) * 0.6931471805599453f;
}

// ------------------------------------------------------------------ host side
size_t decode_shared_workspace_bytes(int B, int Hq, int Hkv, int D, int prefix_len, int max_len) {
    return (size_t)make_shared_plan(B, Hq, Hkv, D, prefix_len, max_len).total * sizeof(float);
}

template <typename T, int D, int G>
static void own_stream(const SharedArgs& a, const SharedPlan& p, cudaStream_t st) {
    shared_own_stream_kernel<T, D, G><<<a.B * a.Hkv * ((a.g + G - 1) / G) * p.own_splits, OWN_WARPS * 32, 0, st>>>(a, p);
}

template <typename T, int D>
static cudaError_t prefix_simt(const SharedArgs& a, const SharedPlan& p, cudaStream_t st) {
    constexpr int smem = SimtSmem<T, D>::FLOATS * (int)sizeof(float);
    cudaError_t e = cudaFuncSetAttribute(shared_prefix_simt_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    const int rows = a.B * a.g;
    shared_prefix_simt_kernel<T, D><<<dim3((rows + SIMT_R - 1) / SIMT_R, a.Hkv, p.p_splits), SIMT_THREADS, smem, st>>>(a, p);
    count_launches(1);
    return cudaGetLastError();
}

template <typename T, int D>
static cudaError_t shared_t(const SharedArgs& a, bool generic, cudaStream_t st) {
    const SharedPlan p = make_shared_plan(a.B, a.Hq, a.Hkv, D, a.prefix_len, a.max_len);
    cudaError_t e = cudaSuccess;
    if (p.p_splits > 0) {
        e = cudaErrorNotSupported;
        if (sizeof(T) == 2 && !generic) e = launch_shared_prefix_tc(a, p, D, st);
        if (e == cudaErrorNotSupported) e = prefix_simt<T, D>(a, p, st);
        if (e != cudaSuccess) return e;
    }
    bool done = false;
    if constexpr (sizeof(T) == 2) {
        if (!generic) {
            const int R = a.g <= 8 ? 1 : 2;
            const unsigned ctas = (unsigned)a.B * a.Hkv * ((a.g + 8 * R - 1) / (8 * R)) * p.own_splits;
            if (R == 1) shared_own_mma_kernel<D, 1><<<ctas, OWN_WARPS * 32, 0, st>>>(a, p);
            else shared_own_mma_kernel<D, 2><<<ctas, OWN_WARPS * 32, 0, st>>>(a, p);
            done = true;
        }
    }
    if (!done) {
        if (a.g == 1) own_stream<T, D, 1>(a, p, st);
        else if (a.g == 2) own_stream<T, D, 2>(a, p, st);
        else own_stream<T, D, 4>(a, p, st);
    }
    count_launches(1);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    shared_merge_kernel<T, D><<<dim3((a.B * a.g + 31) / 32, D / 32, a.Hkv), MERGE_THREADS, 0, st>>>(a, p);
    count_launches(1);
    return cudaGetLastError();
}

cudaError_t launch_decode_shared(const SharedArgs& a, int D, loma_dtype dt, bool generic, cudaStream_t st) {
    if (dt == LOMA_F32) return D == 64 ? shared_t<float, 64>(a, generic, st) : shared_t<float, 128>(a, generic, st);
    return D == 64 ? shared_t<__nv_bfloat16, 64>(a, generic, st) : shared_t<__nv_bfloat16, 128>(a, generic, st);
}

}  // namespace loma
