// Memory entries into a 4-bit pool and back (loma_kv4_append, loma_kv4_load); format in kv4.cuh.
//
// Eight lanes share a row: lane x has features 32 g + 4 x .. + 3 of every group g, which are the four of half-word (x, g).
// Keys and values of an entry go together: eight loads in flight per lane, and the largest magnitudes of the eight groups are found with
// results spread over the lanes (seven shuffles), so each lane works out one step.  Both directions are bound by HBM (256 bytes of bf16
// against 72 for a row of 128 features) as long as a value costs few instructions: m is the integer part of |x| / (2 h), a product and an
// addition that rounds towards zero; see kv4_half for why that is exact.
// Measured (D = 128): bf16, 1.36 million rows of keys and as many of values stored in 203 us (4.4 TB/s, issue-bound), 1.41 million read back in 161
// us (5.8 TB/s); fp32, half as many of each: 135 us (5.9 TB/s) and 138 us (6.0 TB/s).  D = 64, bf16: 141 us (3.2 TB/s) and 90 us (5.2 TB/s).
#include "kv4.cuh"

namespace loma {

constexpr int STORE_THREADS = 256, STORE_ROWS = STORE_THREADS / 8;   // rows a block takes at a time

__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float a, float b, float c, float d) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(a, b), pack_bf16(c, d));
}

__device__ __forceinline__ float max_nan(float a, float b) {   // a NaN stays
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint32_t permute(uint32_t a, uint32_t b, uint32_t sel) {   // selectors from 8 on: the byte's sign, eight times
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(sel));
    return r;
}

// Four features as they were loaded; -0 becomes 0, which is held with a positive sign.
template <typename T>
struct Four;
template <>
struct Four<float> {
    float x[4];
    __device__ __forceinline__ void clear() { x[0] = x[1] = x[2] = x[3] = 0.f; }
    __device__ __forceinline__ void load(const float* p) {
        const float4 u = __ldg(reinterpret_cast<const float4*>(p));
        x[0] = u.x + 0.f; x[1] = u.y + 0.f; x[2] = u.z + 0.f; x[3] = u.w + 0.f;
    }
    __device__ __forceinline__ float top() const { return max_nan(max_nan(fabsf(x[0]), fabsf(x[1])), max_nan(fabsf(x[2]), fabsf(x[3]))); }
    __device__ __forceinline__ float at(int i) const { return x[i]; }
    // upper halves of features 2 i and 2 i + 1
    __device__ __forceinline__ uint32_t signs(int i) const { return __byte_perm(__float_as_uint(x[2 * i]), __float_as_uint(x[2 * i + 1]), 0x7632); }
};
template <>
struct Four<__nv_bfloat16> {
    __nv_bfloat162 w[2];
    __device__ __forceinline__ void clear() { w[0] = w[1] = __floats2bfloat162_rn(0.f, 0.f); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        const uint2 u = __ldg(reinterpret_cast<const uint2*>(p));
        const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
        w[0] = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&u.x), zero);
        w[1] = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&u.y), zero);
    }
    __device__ __forceinline__ uint32_t signs(int i) const { return *reinterpret_cast<const uint32_t*>(&w[i]); }
    __device__ __forceinline__ float top() const {
        const __nv_bfloat162 m = __hmax2_nan(__habs2(w[0]), __habs2(w[1]));
        const uint32_t u = *reinterpret_cast<const uint32_t*>(&m);
        return max_nan(bf16lo(u), bf16hi(u));
    }
    __device__ __forceinline__ float at(int i) const { return i & 1 ? bf16hi(signs(i / 2)) : bf16lo(signs(i / 2)); }
};

// The step of a group whose largest magnitude is `top`, as bf16 bits.  For bf16 input the product with 1 / 15 will do: top has 8 bits, a
// number half way between two bf16 has 9, so top / 15 misses it by 2^-13 of itself at least, and the product is off by 2^-23.
template <typename T>
__device__ __forceinline__ uint32_t kv4_step(float top) {
    const __nv_bfloat16 h = __float2bfloat16_rn(sizeof(T) == 2 ? top * (1.f / 15.f) : __fdiv_rn(top, 15.f));
    const uint32_t bits = __bfloat16_as_ushort(h);
    return bits >= 0x7f80u ? 0x7fffu : bits < 0x0080u ? 0u : bits;
}

// A half-word of four codes.  r is 1 / (2 h) and a little more (2^-20 of itself, the reciprocal and the product are off by 2^-22), so
// t = |x| r is at least m, and its integer part is m, or m + 1 where |x| lies less than 2^-19 below 2 h (m + 1).  bf16 input does not
// (8 bits against 11: the two differ by 2^-11 of themselves or not at all); for fp32 the sign of |x| - 2 h k, exact in one FMA, tells.
// |x| <= 15 h (1 + 2^-8), so m <= 7.
template <typename T>
__device__ __forceinline__ uint32_t kv4_half(const Four<T>& f, float h) {
    constexpr float BIG = 8388608.f;   // 2^23: sums with it have the integer part in their low bits
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(2.f * h));
    r *= 1.f + 0x1p-20f;
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = fabsf(f.at(i)), t = __fadd_rz(__fmul_rn(a, r), BIG);
        u[i] = __float_as_uint(t);
        if constexpr (sizeof(T) == 4) u[i] -= __float_as_uint(fmaf(-2.f * h, t - BIG, a)) >> 31;
    }
    const uint32_t m = u[0] + 8 * u[1] + 256 * u[2] + 2048 * u[3];   // what is above the low 16 bits does not matter
    // byte 0: signs of features 2 (bit 6) and 3 (bit 7), byte 1: of 0 and 1
    const uint32_t lo = permute(f.signs(0), f.signs(1), 0x009d), hi = permute(f.signs(0), f.signs(1), 0x00bf);
    return h > 0.f ? (m & 0x3f3fu) | (lo & 0x4040u) | (hi & 0x8080u) : 0u;
}

// maxima over eight lanes of M values each; lane x keeps value x * M / 8
template <int M, int O>
__device__ __forceinline__ void spread_max8(float* s, int x) {
    if constexpr (M > 1) {
        const bool up = x & O;
#pragma unroll
        for (int i = 0; i < M / 2; ++i) {
            const float lo = s[i], hi = s[i + M / 2];
            s[i] = max_nan(up ? hi : lo, __shfl_xor_sync(0xffffffffu, up ? lo : hi, O));
        }
    } else {
        s[0] = max_nan(s[0], __shfl_xor_sync(0xffffffffu, s[0], O));
    }
    if constexpr (O > 1) spread_max8<(M > 1 ? M / 2 : 1), O / 2>(s, x);
}

template <int N>
__device__ __forceinline__ void put_words(uint8_t* p, const uint32_t (&w)[N]) {
    if constexpr (N == 2) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(p) = w[0];
}

// A block's walk over (sequence, head, turn of STORE_ROWS rows), in steps of the grid, whose parts are found once (two divisions of 64 bits
// every turn took 8 % of the append's time).
struct StoreWalk {
    int per, H, turn, h, step_turn, step_h;
    int64_t b, step_b;
    __device__ __forceinline__ StoreWalk(int turns, int heads) : per(turns), H(heads) {
        split(blockIdx.x, &b, &h, &turn);
        split(gridDim.x, &step_b, &step_h, &step_turn);
    }
    __device__ __forceinline__ void split(unsigned u, int64_t* x, int* y, int* z) const {
        const unsigned bh = u / (unsigned)per;
        *z = (int)(u - bh * (unsigned)per);
        *x = bh / (unsigned)H;
        *y = (int)(bh - (unsigned)*x * (unsigned)H);
    }
    __device__ __forceinline__ void next() {
        turn += step_turn;
        h += step_h;
        b += step_b;
        if (turn >= per) { turn -= per; ++h; }
        if (h >= H) { h -= H; ++b; }
    }
};

template <typename T, int D>
__global__ void __launch_bounds__(STORE_THREADS) kv4_append_kernel(const Kv4AppendArgs a) {
    using TL = Kv4Tile<D>;
    constexpr int G = TL::GROUPS;
    const int x = threadIdx.x & 7, sub = threadIdx.x >> 3;
    const int per = a.l / STORE_ROWS + 1;                // rows -1 .. l - 1, so that odd entries are odd rows' whatever mem_lens is
    const int64_t room = (int64_t)a.m.max_pages << a.m.log2_ps;
    constexpr unsigned ALL = 0xffffffffu;
    for (StoreWalk at(per, a.Hkv); at.b < a.B; at.next()) {
        const int b = (int)at.b, h = at.h;
        const int len = __ldg(a.mem_lens + b), n = a.new_lens ? min(__ldg(a.new_lens + b), a.l) : a.l;
        const int i = at.turn * STORE_ROWS + sub - (len & 1);
        const int64_t j = (int64_t)len + i;
        bool live = len >= 0 && i >= 0 && i < n && j < room;
        const int page = live ? kv4_page(a.m, b, (int)(j >> a.m.log2_ps)) : -1;
        live = page >= 0;
        const unsigned lanes = __ballot_sync(ALL, live);
        if (lanes == 0) continue;
        Four<T> f[2][G];
        if (live) {
            const T* k = static_cast<const T*>(a.k) + b * a.k_stride[0] + h * a.k_stride[1] + i * a.k_stride[2] + 4 * x;
            const T* v = static_cast<const T*>(a.v) + b * a.v_stride[0] + h * a.v_stride[1] + i * a.v_stride[2] + 4 * x;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                f[0][g].load(k + 32 * g);
                f[1][g].load(v + 32 * g);
            }
        } else {
#pragma unroll
            for (int g = 0; g < G; ++g) f[0][g].clear(), f[1][g].clear();
        }
        uint8_t* tile = a.m.pool + kv4_tile<D>(a.m, a.Hkv, max(page, 0), h, (int)j);
        const int row = (int)j & 15;
        float top[2 * G];
#pragma unroll
        for (int i = 0; i < 2 * G; ++i) top[i] = f[i / G][i % G].top();
        spread_max8<2 * G, 4>(top, x);   // lane x: of group x G / 4 (keys' groups, then values')
        const uint32_t bits = kv4_step<T>(top[0]), other = __shfl_xor_sync(ALL, bits, 4 / G);
        const uint32_t two = x & (4 / G) ? other | bits << 16 : bits | other << 16;
        uint32_t step[2][G / 2];
#pragma unroll
        for (int i = 0; i < G; ++i) step[i / (G / 2)][i % (G / 2)] = __shfl_sync(ALL, two, i * (8 / G), 8);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            uint32_t half[G / 2];
#pragma unroll
            for (int i = 0; i < G / 2; ++i)
                half[i] = kv4_half(f[w][2 * i], bf16lo(step[w][i])) | kv4_half(f[w][2 * i + 1], bf16hi(step[w][i])) << 16;
            // A unit's words are made of two lanes' half-words, of x and x ^ 1 (keys) or of two rows (values): the even one makes those of the
            // lower groups, the odd one those of the upper.  Where the other row is not there, its half of the words stays as it is.
            const int partner = w ? 8 : 1;
            const bool odd = w ? row & 1 : x & 1;
            uint32_t word[G / 2];
            if constexpr (G == 4) {
                const uint32_t other = __shfl_xor_sync(ALL, odd ? half[0] : half[1], partner), own = odd ? half[1] : half[0];
                word[0] = odd ? __byte_perm(other, own, 0x5410) : __byte_perm(own, other, 0x5410);
                word[1] = odd ? __byte_perm(other, own, 0x7632) : __byte_perm(own, other, 0x7632);
            } else {
                const uint32_t other = __shfl_xor_sync(ALL, half[0], partner);
                word[0] = odd ? __byte_perm(other, half[0], 0x7632) : __byte_perm(half[0], other, 0x5410);
            }
            if (!live) continue;
            uint8_t* unit = tile + (w ? kv4_v_unit<D>(row, x) : kv4_k_unit<D>(row, x));
            if (w == 0 || lanes >> (threadIdx.x & 31 ^ 8) & 1) {
                put_words(unit + odd * (TL::UNIT / 2), word);
            } else {
#pragma unroll
                for (int g = 0; g < G; ++g) *reinterpret_cast<uint16_t*>(unit + 4 * g + odd * 2) = (uint16_t)(half[g / 2] >> g % 2 * 16);
            }
            if (x == w) put_words(tile + TL::K_STEPS + w * (TL::V_STEPS - TL::K_STEPS) + row * TL::STEPS, step[w]);
        }
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(STORE_THREADS) kv4_load_kernel(const Kv4LoadArgs a) {
    using TL = Kv4Tile<D>;
    constexpr int G = TL::GROUPS;
    const int x = threadIdx.x & 7, sub = threadIdx.x >> 3;
    const int per = (a.cap + STORE_ROWS - 1) / STORE_ROWS;
    const int64_t room = (int64_t)a.m.max_pages << a.m.log2_ps;
    for (StoreWalk at(per, a.Hkv); at.b < a.B; at.next()) {
        const int b = (int)at.b, h = at.h, j = at.turn * STORE_ROWS + sub;
        if (j >= a.cap || j >= __ldg(a.mem_lens + b) || j >= room) continue;
        const int page = min(max(__ldg(a.m.table + (int64_t)b * a.m.max_pages + (j >> a.m.log2_ps)), 0), a.m.n_pages - 1);
        const uint8_t* tile = a.m.pool + kv4_tile<D>(a.m, a.Hkv, page, h, j);
        const int row = j & 15;
        uint32_t half[2][G / 2], step[2][G / 2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            kv4_halves<G>(tile + (w ? kv4_v_unit<D>(row, x) : kv4_k_unit<D>(row, x)), w ? row & 1 : x & 1, half[w]);
            kv4_steps<G>(tile + TL::K_STEPS + w * (TL::V_STEPS - TL::K_STEPS) + row * TL::STEPS, step[w]);
        }
        // n 2^-133 times 2^127, the step and 2^6 (2^4 for odd e): exact in this order, whatever the step
        constexpr float UP = 1.7014118346046923e38f;   // 2^127
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            T* out = static_cast<T*>(w ? a.v : a.k) + (((int64_t)b * a.Hkv + h) * a.cap + j) * D + 4 * x;
#pragma unroll
            for (int g = 0; g < G; g += 2) {
                uint32_t n[4];
                kv4_word(half[w][g / 2], a.ones, n);
                const float h0 = bf16lo(step[w][g / 2]), h1 = bf16hi(step[w][g / 2]);
                store4(out + 32 * g, bf16lo(n[0]) * UP * h0 * 64.f, bf16lo(n[1]) * UP * h0 * 16.f, bf16lo(n[2]) * UP * h0 * 64.f, bf16lo(n[3]) * UP * h0 * 16.f);
                store4(out + 32 * g + 32, bf16hi(n[0]) * UP * h1 * 64.f, bf16hi(n[1]) * UP * h1 * 16.f, bf16hi(n[2]) * UP * h1 * 64.f, bf16hi(n[3]) * UP * h1 * 16.f);
            }
        }
    }
}

// eight blocks of 256 threads fit an SM; more blocks than that take turns anyway
static unsigned store_grid(int64_t bh, int turns) { return (unsigned)std::min<int64_t>(bh * turns, 148 * 8 * 4); }

template <typename A>
static cudaError_t launch_store(void (*kernel)(A), const A& a, unsigned grid, cudaStream_t st) {
    kernel<<<grid, STORE_THREADS, 0, st>>>(a);
    count_launches(1);
    return cudaGetLastError();
}

cudaError_t launch_kv4_append(const Kv4AppendArgs& a, int D, loma_dtype dt, cudaStream_t st) {
    const unsigned grid = store_grid((int64_t)a.B * a.Hkv, a.l / STORE_ROWS + 1);
    if (dt == LOMA_F32) return launch_store(D == 64 ? kv4_append_kernel<float, 64> : kv4_append_kernel<float, 128>, a, grid, st);
    return launch_store(D == 64 ? kv4_append_kernel<__nv_bfloat16, 64> : kv4_append_kernel<__nv_bfloat16, 128>, a, grid, st);
}

cudaError_t launch_kv4_load(const Kv4LoadArgs& a, int D, loma_dtype dt, cudaStream_t st) {
    const unsigned grid = store_grid((int64_t)a.B * a.Hkv, (a.cap + STORE_ROWS - 1) / STORE_ROWS);
    if (dt == LOMA_F32) return launch_store(D == 64 ? kv4_load_kernel<float, 64> : kv4_load_kernel<float, 128>, a, grid, st);
    return launch_store(D == 64 ? kv4_load_kernel<__nv_bfloat16, 64> : kv4_load_kernel<__nv_bfloat16, 128>, a, grid, st);
}

}  // namespace loma
