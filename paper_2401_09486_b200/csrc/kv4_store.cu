// Memory entries into a 4-bit pool and back (loma_kv4_append, loma_kv4_load); format in kv4.cuh.
//
// Eight lanes share a row: lane x has features 32 g + 4 x .. + 3 of every group g, which are the four of a half-word, so a group's
// maximum takes three shuffles and a lane writes one chunk of 8 (or 4) bytes.  Keys and values of an entry go together: eight
// loads in flight per lane.  Both directions are bound by HBM: 256 bytes of bf16 against 72 for a row of 128 features.  The three
// comparisons per value that make m (instead of a division) are exact and leave the arithmetic well below the time of the bytes.
#include "kv4.cuh"

namespace loma {

constexpr int STORE_THREADS = 256, STORE_ROWS = STORE_THREADS / 8;   // rows a block takes at a time

template <typename T>
__device__ __forceinline__ float4 load4(const T* p);
template <>
__device__ __forceinline__ float4 load4(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }
template <>
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
    const uint2 u = __ldg(reinterpret_cast<const uint2*>(p));
    return make_float4(bf16lo(u.x), bf16hi(u.x), bf16lo(u.y), bf16hi(u.y));
}
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float a, float b, float c, float d) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(a, b), pack_bf16(c, d));
}

__device__ __forceinline__ float max_nan(float a, float b) {   // a NaN stays
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// the step of a group whose largest magnitude is `top`, as bf16 bits
__device__ __forceinline__ uint32_t kv4_step(float top) {
    const __nv_bfloat16 h = __float2bfloat16_rn(__fdiv_rn(top, 15.f));
    const uint32_t bits = __bfloat16_as_ushort(h);
    return bits >= 0x7f80u ? 0x7fffu : bits < 0x0080u ? 0u : bits;
}

// sign and m of a value whose group has step h: |x| >= 8h, then 4h, then 2h; the differences are exact (the larger is at most
// twice the smaller where they are taken, since |x| <= 15 h (1 + 2^-8) < 16 h)
__device__ __forceinline__ uint32_t kv4_code(float x, float h) {
    float a = fabsf(x);
    uint32_t m = 0;
    if (a >= 8.f * h) { m = 4; a -= 8.f * h; }
    if (a >= 4.f * h) { m |= 2; a -= 4.f * h; }
    if (a >= 2.f * h) m |= 1;
    return h > 0.f ? m | (x < 0.f ? 8u : 0u) : 0u;
}
// a half-word of four codes
__device__ __forceinline__ uint32_t kv4_half(const float4& x, float h) {
    const uint32_t c0 = kv4_code(x.x, h), c1 = kv4_code(x.y, h), c2 = kv4_code(x.z, h), c3 = kv4_code(x.w, h);
    return (c0 & 7) | (c1 & 7) << 3 | (c2 >> 3) << 6 | (c3 >> 3) << 7 | (c2 & 7) << 8 | (c3 & 7) << 11 | (c0 >> 3) << 14 | (c1 >> 3) << 15;
}
__device__ __forceinline__ float kv4_value(uint32_t m, uint32_t sign, float h) {
    const float v = (float)(2 * m + 1) * h;
    return sign ? -v : v;
}

// G half-words: a chunk's bytes, or a row's steps
template <int G>
__device__ __forceinline__ void put_halves(uint8_t* p, const uint32_t (&w)[G]) {
    if constexpr (G == 4) *reinterpret_cast<uint2*>(p) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
    else *reinterpret_cast<uint32_t*>(p) = w[0] | w[1] << 16;
}
template <int G>
__device__ __forceinline__ void get_halves(const uint8_t* p, uint32_t (&w)[G]) {
    if constexpr (G == 4) {
        const uint2 u = __ldg(reinterpret_cast<const uint2*>(p));
        w[0] = u.x & 0xffff; w[1] = u.x >> 16; w[2] = u.y & 0xffff; w[3] = u.y >> 16;
    } else {
        const uint32_t u = __ldg(reinterpret_cast<const uint32_t*>(p));
        w[0] = u & 0xffff; w[1] = u >> 16;
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(STORE_THREADS) kv4_append_kernel(const Kv4AppendArgs a) {
    using TL = Kv4Tile<D>;
    constexpr int G = TL::GROUPS;
    const int x = threadIdx.x & 7, sub = threadIdx.x >> 3;
    const unsigned mine = 0xffu << (threadIdx.x & 24);   // the lanes of this row
    const int per = (a.l + STORE_ROWS - 1) / STORE_ROWS;
    const int64_t units = (int64_t)a.B * a.Hkv * per, room = (int64_t)a.m.max_pages << a.m.log2_ps;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t bh = u / per;
        const int i = (int)(u - bh * per) * STORE_ROWS + sub, b = (int)(bh / a.Hkv), h = (int)(bh - (int64_t)b * a.Hkv);
        const int len = __ldg(a.mem_lens + b), n = a.new_lens ? min(__ldg(a.new_lens + b), a.l) : a.l;
        const int64_t j = (int64_t)len + i;
        if (len < 0 || i >= n || j >= room) continue;
        const int page = kv4_page(a.m, b, (int)(j >> a.m.log2_ps));
        if (page < 0) continue;
        const T* k = static_cast<const T*>(a.k) + b * a.k_stride[0] + h * a.k_stride[1] + i * a.k_stride[2] + 4 * x;
        const T* v = static_cast<const T*>(a.v) + b * a.v_stride[0] + h * a.v_stride[1] + i * a.v_stride[2] + 4 * x;
        float4 f[2][G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            f[0][g] = load4(k + 32 * g);
            f[1][g] = load4(v + 32 * g);
        }
        uint8_t* tile = a.m.pool + kv4_tile<D>(a.m, a.Hkv, page, h, (int)j);
        const int row = (int)j & 15;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            uint32_t half[G], step[G];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const float4& y = f[w][g];
                float top = max_nan(max_nan(fabsf(y.x), fabsf(y.y)), max_nan(fabsf(y.z), fabsf(y.w)));
#pragma unroll
                for (int o = 1; o < 8; o <<= 1) top = max_nan(top, __shfl_xor_sync(mine, top, o));
                step[g] = kv4_step(top);
                half[g] = kv4_half(y, __uint_as_float(step[g] << 16));
            }
            put_halves<G>(tile + w * TL::V + kv4_chunk<D>(row, x), half);
            if (x == 0) put_halves<G>(tile + TL::K_STEPS + w * (TL::V_STEPS - TL::K_STEPS) + row * TL::STEPS, step);
        }
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(STORE_THREADS) kv4_load_kernel(const Kv4LoadArgs a) {
    using TL = Kv4Tile<D>;
    constexpr int G = TL::GROUPS;
    const int x = threadIdx.x & 7, sub = threadIdx.x >> 3;
    const int per = (a.cap + STORE_ROWS - 1) / STORE_ROWS;
    const int64_t units = (int64_t)a.B * a.Hkv * per, room = (int64_t)a.m.max_pages << a.m.log2_ps;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t bh = u / per;
        const int j = (int)(u - bh * per) * STORE_ROWS + sub, b = (int)(bh / a.Hkv), h = (int)(bh - (int64_t)b * a.Hkv);
        if (j >= a.cap || j >= __ldg(a.mem_lens + b) || j >= room) continue;
        const int page = min(max(__ldg(a.m.table + (int64_t)b * a.m.max_pages + (j >> a.m.log2_ps)), 0), a.m.n_pages - 1);
        const uint8_t* tile = a.m.pool + kv4_tile<D>(a.m, a.Hkv, page, h, j);
        const int row = j & 15;
        uint32_t half[2][G], step[2][G];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            get_halves<G>(tile + w * TL::V + kv4_chunk<D>(row, x), half[w]);
            get_halves<G>(tile + TL::K_STEPS + w * (TL::V_STEPS - TL::K_STEPS) + row * TL::STEPS, step[w]);
        }
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            T* out = static_cast<T*>(w ? a.v : a.k) + (bh * a.cap + j) * D + 4 * x;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const uint32_t y = half[w][g];
                const float s = __uint_as_float(step[w][g] << 16);
                store4(out + 32 * g, kv4_value(y & 7, y >> 14 & 1, s), kv4_value(y >> 3 & 7, y >> 15 & 1, s), kv4_value(y >> 8 & 7, y >> 6 & 1, s),
                       kv4_value(y >> 11 & 7, y >> 7 & 1, s));
            }
        }
    }
}

// eight blocks of 256 threads fit an SM; more blocks than that take turns anyway
static unsigned store_grid(int64_t bh, int rows) {
    return (unsigned)std::min<int64_t>(bh * ((rows + STORE_ROWS - 1) / STORE_ROWS), 148 * 8 * 4);
}

template <typename A>
static cudaError_t launch_store(void (*kernel)(A), const A& a, unsigned grid, cudaStream_t st) {
    kernel<<<grid, STORE_THREADS, 0, st>>>(a);
    count_launches(1);
    return cudaGetLastError();
}

cudaError_t launch_kv4_append(const Kv4AppendArgs& a, int D, loma_dtype dt, cudaStream_t st) {
    const unsigned grid = store_grid((int64_t)a.B * a.Hkv, a.l);
    if (dt == LOMA_F32) return launch_store(D == 64 ? kv4_append_kernel<float, 64> : kv4_append_kernel<float, 128>, a, grid, st);
    return launch_store(D == 64 ? kv4_append_kernel<__nv_bfloat16, 64> : kv4_append_kernel<__nv_bfloat16, 128>, a, grid, st);
}

cudaError_t launch_kv4_load(const Kv4LoadArgs& a, int D, loma_dtype dt, cudaStream_t st) {
    const unsigned grid = store_grid((int64_t)a.B * a.Hkv, a.cap);
    if (dt == LOMA_F32) return launch_store(D == 64 ? kv4_load_kernel<float, 64> : kv4_load_kernel<float, 128>, a, grid, st);
    return launch_store(D == 64 ? kv4_load_kernel<__nv_bfloat16, 64> : kv4_load_kernel<__nv_bfloat16, 128>, a, grid, st);
}

}  // namespace loma
