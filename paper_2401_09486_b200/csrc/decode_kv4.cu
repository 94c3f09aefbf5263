// Decode attention over memory entries held in 4 bits and an uncompressed tail (loma_decode_attn_kv4).
//
// Query head hq of sequence b sees the memory entries [0, mem_lens[b]) of kv head hq div g (g = Hq / Hkv), the tail's entries
// [0, tail_lens[b]) and the new token, under one softmax.  One query row per head against rows that no other sequence reads: a
// stream bound by HBM, 144 bytes of 4-bit tiles per memory entry (D = 128) where bf16 has 512.  So few bytes leave little time for
// arithmetic: 23 bytes per SM and clock from HBM are a tile of 16 entries every 100 clocks, in which the four schedulers of an SM issue
// 400 instructions; a tile takes a warp 290, 112 of them to turn its 4096 numbers into operands.
//
// Cut: units are (kv head, head tile, sequence); a unit's blocks -- 32 entries of memory each first, then 16 of the tail with the new
// token last -- are numbered through, and worker w of W (a warp) takes blocks [T w / W, T (w + 1) / W).  A worker's stay in
// one unit is a segment with a partial result in slot w + unit; kv4_merge_kernel joins a unit's segments in a fixed order.  The
// lengths are known on the device only, so every CTA finds the cut from them.  Few or short units are not cut (KV4_WHOLE).
//
// bf16: kv4_decode_kernel, warp-level products.  fp32, and the second opinion: kv4_stream_kernel on CUDA cores.
// Measured: B64 Hq32 Hkv8 D128, up to 16384 entries and tails of up to 127 (829 MB): 164 us, 5.0 TB/s (0.77 of a copy; the copies alone take 134 us)
// in a short run; 169 to 180 us in long ones, which the power limit holds at 1.8 GHz.  B32 H32, 2048 entries 56 us; B4 H8 D64, 200 entries 5.4 us.
// In between 0.2 to 0.4 of a copy's rate (Hkv 8: B16, 1000 entries 11.5 us; B8, 8000 24; B64, 1000 26).  16 heads to a kv head: B64 Hq128, 8000
// entries 137 us (0.48).  fp32: B11 Hq15 Hkv3, 2501 entries 23 us; B32 Hq32 Hkv8, 4000 entries 87 us.
#include <cooperative_groups.h>

#include "kv4.cuh"
#include "tcgen05_common.cuh"

namespace cg = cooperative_groups;

namespace loma {

constexpr int KV4_WARPS = 4;
constexpr int KV4_STEP = 32;   // memory entries to a block: two tiles

struct Kv4Plan {
    int g_rows, g_tiles;   // query heads of a kv head per head tile, head tiles per kv head
    int ctas, workers;     // W, before it is cut down for few blocks
    int whole;             // CTAs of a cluster per unit, whose warps share its blocks and join their parts in shared memory: one launch (0: no)
    // in the workspace, in floats.  Segment: outputs [g_rows][D], g_rows log2-sum-exps.  ends: int32 [2][units], the workers of a unit's
    // first and of its last segment
    int64_t o, lse, ends, total;
    uint32_t ones;         // 0x00010001 (see kv4_word)
};

// Units stay whole, with the warps of one CTA or of a cluster of two to eight, while all of them run at once and no warp gets more than
// KV4_WHOLE blocks: that saves finding the cut, a launch and the merge through memory, 3 to 5 us together, and costs that sequences of different
// lengths do not even out.  Somewhat more CTAs than run at once will do for short units (up to KV4_WHOLE_SHORT blocks).  Measured, whole
// against cut (D = 128, us): 32 units of up to 4 / 35 / 66 / 129 blocks 5.8 / 8.7 / 9.6 / 12.0 against 9.9 / 11.1 / 12.4 / 15.3; 128 units of 35 / 66
// 11.8 / 16.8 against 14.7 / 18.5; 256 units of 35 / 51 16.0 / 22.1 against 20.2 / 24.2; 512 units of 14 14.7 against 17.2; but 64 units of 254, 16 blocks
// to a warp, 26.4 against 24.9, and 1024 units of 14 27.3 against 24.3.
// The rule goes by the host's bounds, not by the lengths, which only the device knows: a step captured for a capacity of 150000 entries is cut
// however short its sequences are (D = 128 but for the first; own bound / capacity, us: 32 units of up to 200 entries, D = 64, 5.6 / 9.2; 32 of 100 5.9 / 10.0;
// 32 of 1000 8.6 / 11.1; 128 of 1000 11.6 / 14.4; 256 of 1000 15.6 / 19.6).
constexpr int KV4_WHOLE = 12, KV4_WHOLE_SHORT = 16;

static Kv4Plan make_kv4_plan(int B, int Hq, int Hkv, int D, int max_mem, int max_tail, bool cuda_cores) {
    Kv4Plan p;
    const int g = Hq / Hkv;
    p.g_rows = cuda_cores ? (g < 3 ? g : 4) : (g <= 8 ? g : 16);
    p.g_tiles = (g + p.g_rows - 1) / p.g_rows;
    p.ctas = 148 * (cuda_cores ? (p.g_rows == 4 ? 2 : 4) : p.g_rows <= 8 ? 3 : 2);
    p.workers = p.ctas * KV4_WARPS;
    const int64_t units = (int64_t)B * Hkv * p.g_tiles, blocks = ((int64_t)max_mem + KV4_STEP - 1) / KV4_STEP + max_tail / KV4_ROWS + 1;
    p.whole = 0;
    if (!cuda_cores) {
        int c = 8;   // as many CTAs as run at once and have more than a block to a warp; a cluster is not worth it for KV4_WHOLE_SHORT blocks
        while (c > 1 && (units * c > p.ctas || blocks <= std::max(KV4_WHOLE_SHORT, KV4_WARPS * c))) c /= 2;
        if (units * c <= p.ctas ? blocks <= (int64_t)KV4_WHOLE * KV4_WARPS * c : units <= 4 * 148 && blocks <= KV4_WHOLE_SHORT) p.whole = c;
    }
    int64_t at = 0;
    auto take = [&](int64_t n) { const int64_t o = at; at += (n + 63) / 64 * 64; return o; };
    const int64_t segments = p.workers + units;
    p.o = take(segments * p.g_rows * D);
    p.lse = take(segments * p.g_rows);
    p.ends = take(2 * units);
    p.total = at;
    p.ones = 0x00010001u;
    return p;
}

// the first block of worker w of W <= T (W^2 fits 32 bits; a division of 64 bits takes a hundred instructions)
__device__ __forceinline__ int64_t kv4_first(int64_t w, int64_t T, int64_t W) {
    if (T > UINT32_MAX) return T / W * w + T % W * w / W;
    const uint32_t q = (uint32_t)T / (uint32_t)W, r = (uint32_t)T - q * (uint32_t)W;
    return (int64_t)q * w + r * (uint32_t)w / (uint32_t)W;
}

// One sequence's part of a unit.
struct Kv4Seq {
    int mem, tail;   // memory entries; tail entries before the new token (negative: no request)
    int nm, n;       // blocks of memory, and in all
};
__device__ __forceinline__ Kv4Seq kv4_seq(const Kv4DecodeArgs& a, int b) {
    Kv4Seq s;
    s.mem = min(max(__ldg(a.mem_lens + b), 0), a.max_mem);
    s.tail = min(__ldg(a.tail_lens + b), a.max_tail);
    s.nm = (s.mem + KV4_STEP - 1) / KV4_STEP;
    s.n = s.tail < 0 ? 0 : s.nm + s.tail / KV4_ROWS + 1;
    return s;
}

// A worker that does blocks [from, to) of a unit of n notes where the unit's segments begin and end; a unit that it does all of has none left
// to be joined.
__device__ __forceinline__ void kv4_note(const Kv4DecodeArgs& a, const Kv4Plan& p, int64_t unit, int64_t w, int from, int to, int n) {
    int32_t* ends = reinterpret_cast<int32_t*>(static_cast<float*>(a.ws) + p.ends);
    const bool all = from == 0 && to == n;
    if (from == 0) ends[unit] = all ? 1 : (int)w;
    if (to == n) ends[(int64_t)a.B * a.Hkv * p.g_tiles + unit] = all ? 0 : (int)w;
}

// The numbering of the blocks, found again by every CTA.
struct Kv4Blocks {
    static constexpr int MAX_GROUPS = 512, THREADS = KV4_WARPS * 32, PER_THREAD = MAX_GROUPS / THREADS;
    struct Cursor {
        int hh, b, blk;   // kv head * g_tiles + head tile, sequence, block
        Kv4Seq s;
    };
    const Kv4DecodeArgs& a;

    // s[i]: blocks before sequence i * per of one (kv head, head tile), i = 0 .. groups; returns per.  Ends with a barrier.
    __device__ __forceinline__ int scan(int64_t* s, int64_t* wsum) const {
        const int per = (a.B + MAX_GROUPS - 1) / MAX_GROUPS, groups = (a.B + per - 1) / per;
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        int64_t mine[PER_THREAD], sum = 0;
#pragma unroll
        for (int u = 0; u < PER_THREAD; ++u) {
            const int i = threadIdx.x * PER_THREAD + u;
            mine[u] = 0;
            for (int b = i * per; b < min(a.B, (i + 1) * per); ++b) mine[u] += kv4_seq(a, b).n;
            sum += mine[u];
        }
        int64_t incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        if (lane == 31) wsum[warp] = incl;
        __syncthreads();
        int64_t at = incl - sum;
        for (int x = 0; x < warp; ++x) at += wsum[x];
#pragma unroll
        for (int u = 0; u < PER_THREAD; ++u) {
            const int i = threadIdx.x * PER_THREAD + u;
            if (i <= groups) s[i] = at;
            at += mine[u];
        }
        if (threadIdx.x == THREADS - 1 && groups == MAX_GROUPS) s[MAX_GROUPS] = at;
        __syncthreads();
        return per;
    }

    __device__ __forceinline__ Cursor find(int64_t t, const int64_t* s, int per) const {
        const int groups = (a.B + per - 1) / per;
        Cursor c;
        const int64_t n = s[groups];
        c.hh = t <= UINT32_MAX && n <= UINT32_MAX ? (int)((uint32_t)t / (uint32_t)n) : (int)(t / n);
        int64_t rem = t - c.hh * n;
        // the last group with s[lo] <= rem, by a warp: 16 groups to a lane, then one
        const int lane = threadIdx.x & 31;
        int lo = 16 * (__popc(__ballot_sync(0xffffffffu, lane * 16 < groups && s[min(lane * 16, groups)] <= rem)) - 1);
        lo += __popc(__ballot_sync(0xffffffffu, lane < 16 && lo + lane < groups && s[min(lo + lane, groups)] <= rem)) - 1;
        rem -= s[lo];
        for (c.b = lo * per;; ++c.b) {
            c.s = kv4_seq(a, c.b);
            if (rem < c.s.n) break;
            rem -= c.s.n;
        }
        c.blk = (int)rem;
        return c;
    }

    // The next unit that holds a request; there has to be one.  Slots without one are passed over 32 at a time, up to the batch's end (one by one, 40
    // requests in 4096 slots took 64 us for 47, 8 of 16384 entries in 256 slots 52 for 46).
    __device__ __forceinline__ void next_unit(Cursor& c) const {
        c.blk = 0;
        if (++c.b == a.B) { c.b = 0; ++c.hh; }
        c.s = kv4_seq(a, c.b);
#pragma unroll 1
        while (__builtin_expect(c.s.n == 0, 0)) {
            unsigned idle;
            do {
                const int b = c.b + (threadIdx.x & 31);
                idle = __ballot_sync(0xffffffffu, b < a.B && __ldg(a.tail_lens + b) < 0);
                c.b += idle == 0xffffffffu ? 32 : __ffs(~idle) - 1;
            } while (idle == 0xffffffffu);
            if (c.b == a.B) { c.b = 0; ++c.hh; }
            c.s = kv4_seq(a, c.b);
        }
    }
};

__device__ __forceinline__ int kv4_page_read(const Kv4Pool& m, int b, int j) {   // numbers outside the pool are clamped to it
    return min(max(__ldg(m.table + (int64_t)b * m.max_pages + (j >> m.log2_ps)), 0), m.n_pages - 1);
}

// ------------------------------------------------------------------ CUDA cores
// Eight lanes share an entry (half-words x of every group, 16 or 8 of its features), so a warp takes a tile in four rounds of four entries, G heads
// of the group together.  The 4 G partial scores of a lane are added up over those lanes with the results spread over them, so a lane
// keeps the maximum and the sum of one head; weights go back to all lanes through the warp's shared memory.  All arithmetic in
// fp32; the one rounding is that of the output.

// sums over the lanes that differ in bit O and below, M values; lane x keeps value x * M / 8 + v (or each value lies in 8 / M lanes)
template <int M, int O>
__device__ __forceinline__ void spread_sum8(float* s, int lane) {
    if constexpr (M > 1) {
        const bool up = lane & O;
#pragma unroll
        for (int i = 0; i < M / 2; ++i) {
            const float lo = s[i], hi = s[i + M / 2];
            s[i] = (up ? hi : lo) + __shfl_xor_sync(0xffffffffu, up ? lo : hi, O);
        }
    } else {
        s[0] += __shfl_xor_sync(0xffffffffu, s[0], O);
    }
    if constexpr (O > 1) spread_sum8<(M > 1 ? M / 2 : 1), O / 2>(s, lane);
}

// four features
__device__ __forceinline__ void load4(const float* p, float (&x)[4]) {
    const float4 u = *reinterpret_cast<const float4*>(p);
    x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
}
__device__ __forceinline__ void load4(const __nv_bfloat16* p, float (&x)[4]) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    x[0] = bf16lo(u.x); x[1] = bf16hi(u.x); x[2] = bf16lo(u.y); x[3] = bf16hi(u.y);
}

__device__ __forceinline__ uint64_t times2(uint64_t v, float lo, float hi) { return fma2(v, pack2(lo, hi), 0); }
__device__ __forceinline__ float both(uint64_t v) {
    float lo, hi;
    unpack2(v, lo, hi);
    return lo + hi;
}
__device__ __forceinline__ void kv4_put(float* p, const float4& o) { *reinterpret_cast<float4*>(p) = o; }
__device__ __forceinline__ void kv4_put(__nv_bfloat16* p, const float4& o) { *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(o.x, o.y), pack_bf16(o.z, o.w)); }

template <typename T, int D, int G>
__global__ void __launch_bounds__(KV4_WARPS * 32, G == 4 ? 2 : 4)
kv4_stream_kernel(const Kv4DecodeArgs a, const Kv4Plan p) {
    using TL = Kv4Tile<D>;
    constexpr int NG = TL::GROUPS, M = 4 * G, KEEP = M > 8 ? M / 8 : 1, DUP = M < 8 ? 8 / M : 1, LH = 8 / G;
    __shared__ int64_t scan[Kv4Blocks::MAX_GROUPS + 1];
    __shared__ int64_t wsum[KV4_WARPS];
    __shared__ __align__(16) float s_weight[KV4_WARPS][4][M];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, x = lane & 7, sub = lane >> 3;
    float* ws = static_cast<float*>(a.ws);
    let_next_start();
    const Kv4Blocks kb{a};
    const int per = kb.scan(scan, wsum);
    const int64_t total = scan[(a.B + per - 1) / per] * a.Hkv * p.g_tiles, W = min(total, (int64_t)p.workers);
    const int64_t w = (int64_t)warp * gridDim.x + blockIdx.x;
    if (w >= W) return;
    int left = (int)(kv4_first(w + 1, total, W) - kv4_first(w, total, W));
    Kv4Blocks::Cursor c = kb.find(kv4_first(w, total, W), scan, per);
    const uint32_t ones = p.ones;
    const float scale_log2 = a.scale * 1.4426950408889634f;
    // two-wide arithmetic: groups 2 i and 2 i + 1 go together
    uint64_t q[G][NG / 2][4], acc[G][NG / 2][4];
    float m = -INFINITY, ref = 0.f, l = 0.f;       // m (a score in powers of two), ref (what exponents are taken off), l: of head x / LH
    // s: scores of the lane's four entries (rows i * 4 + sub of a tile) for all heads; the weights of all heads come back in it
    auto weights = [&](float (&s)[M], int valid, float factor) {
        spread_sum8<M, 4>(s, lane);
        float top = -INFINITY;
#pragma unroll
        for (int v = 0; v < KEEP; ++v) {
            s[v] = (x * KEEP / DUP + v) % 4 * 4 + sub < valid ? s[v] * factor : -INFINITY;
            top = fmaxf(top, s[v]);
        }
#pragma unroll
        for (int o = DUP; o < LH; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
        // the reference moves only when a head's maximum has grown by more than 2^8 (weights stay below 2^8)
        if (__any_sync(0xffffffffu, top > m + 8.f)) {
            const float m_new = fmaxf(m, top), keep = m_new == -INFINITY ? 1.f : exp2f(m - m_new);
            m = m_new;
            ref = m == -INFINITY ? 0.f : m;
            l *= keep;
#pragma unroll
            for (int y = 0; y < G; ++y) {
                const float f = __shfl_sync(0xffffffffu, keep, y * LH);
#pragma unroll
                for (int g = 0; g < NG / 2; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[y][g][e] = times2(acc[y][g][e], f, f);
            }
        }
        __syncwarp();   // the last tile's weights have been read
#pragma unroll
        for (int v = 0; v < KEEP; ++v) {
            const float pr = exp2f(s[v] - ref);
            l += pr;
            if (x % DUP == 0) s_weight[warp][sub][x * KEEP / DUP + v] = pr;
        }
        __syncwarp();
#pragma unroll
        for (int y = 0; y < M; y += 4) load4(&s_weight[warp][sub][y], *reinterpret_cast<float(*)[4]>(s + y));
    };
    for (;;) {   // a segment: blocks of memory, then of the tail
        const int h = c.hh / p.g_tiles, gt = c.hh - h * p.g_tiles, heads = min(G, a.g - gt * G);
        const int blocks = min(max(c.s.nm - c.blk, 0), left), tails = min(c.s.n - c.blk - blocks, left - blocks);
#pragma unroll
        for (int y = 0; y < G; ++y) {
            const T* qp = static_cast<const T*>(a.q) + ((int64_t)c.b * a.Hq + h * a.g + gt * G + min(y, heads - 1)) * D + 4 * x;
#pragma unroll
            for (int g = 0; g < NG; g += 2) {
                float lo[4], hi[4];
                load4(qp + 32 * g, lo);
                load4(qp + 32 * g + 32, hi);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float f = !blocks ? 1.f : e & 1 ? KV4_Q / 4 : KV4_Q;
                    q[y][g / 2][e] = pack2(lo[e] * f, hi[e] * f);
                    acc[y][g / 2][e] = 0;
                }
            }
        }
        m = -INFINITY;
        ref = l = 0.f;
        const int end = min(c.s.mem, (c.blk + blocks) * KV4_STEP);
        const uint8_t* next = blocks ? a.m.pool + kv4_tile<D>(a.m, a.Hkv, kv4_page_read(a.m, c.b, c.blk * KV4_STEP), h, c.blk * KV4_STEP) : nullptr;
#pragma unroll 1
        for (int j0 = c.blk * KV4_STEP; j0 < end; j0 += KV4_ROWS) {
            const uint8_t* tile = next;
            const int valid = end - j0;
            if (valid > KV4_ROWS) {   // the next tile's way from memory begins a tile ahead
                next = a.m.pool + kv4_tile<D>(a.m, a.Hkv, kv4_page_read(a.m, c.b, j0 + KV4_ROWS), h, j0 + KV4_ROWS);
                if (lane < (TL::BYTES + 127) / 128) asm volatile("prefetch.global.L1 [%0];" ::"l"(next + min(lane * 128, TL::BYTES - 1)));
            }
            uint32_t kw[4][NG / 2], vw[4][NG / 2], kh[4][NG / 2], vh[4][NG / 2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = i * 4 + sub;
                kv4_halves<NG>(tile + kv4_k_unit<D>(row, x), x & 1, kw[i]);
                kv4_steps<NG>(tile + TL::K_STEPS + row * TL::STEPS, kh[i]);
                kv4_halves<NG>(tile + kv4_v_unit<D>(row, x), row & 1, vw[i]);
                kv4_steps<NG>(tile + TL::V_STEPS + row * TL::STEPS, vh[i]);
            }
            float s[M];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint64_t sum[G] = {};
#pragma unroll
                for (int g = 0; g < NG / 2; ++g) {
                    uint32_t n[4];
                    kv4_word(kw[i][g], ones, n);
                    uint64_t n2[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) n2[e] = pack2(bf16lo(n[e]), bf16hi(n[e]));
                    const uint64_t step = pack2(bf16lo(kh[i][g]), bf16hi(kh[i][g]));
#pragma unroll
                    for (int y = 0; y < G; ++y) {
                        uint64_t t = fma2(q[y][g][0], n2[0], 0);
#pragma unroll
                        for (int e = 1; e < 4; ++e) t = fma2(q[y][g][e], n2[e], t);
                        sum[y] = fma2(t, step, sum[y]);
                    }
                }
#pragma unroll
                for (int y = 0; y < G; ++y) s[y * 4 + i] = both(sum[y]);
            }
            weights(s, valid, scale_log2 * KV4_S);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool there = i * 4 + sub < valid;   // rows past the last entry may hold anything, and 0 x NaN is not 0
#pragma unroll
                for (int g = 0; g < NG / 2; ++g) {
                    uint32_t n[4];
                    kv4_word(vw[i][g], ones, n);
                    uint64_t n2[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) n2[e] = pack2(bf16lo(n[e]), bf16hi(n[e]));
                    const float h0 = there ? bf16lo(vh[i][g]) * KV4_P : 0.f, h1 = there ? bf16hi(vh[i][g]) * KV4_P : 0.f;
#pragma unroll
                    for (int y = 0; y < G; ++y) {
                        const uint64_t weight = pack2(s[y * 4 + i] * h0, s[y * 4 + i] * h1);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[y][g][e] = fma2(weight, n2[e], acc[y][g][e]);
                    }
                }
            }
        }
        if (blocks) {   // the powers of two are taken off
#pragma unroll
            for (int y = 0; y < G; ++y)
#pragma unroll
                for (int g = 0; g < NG / 2; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float f = e & 1 ? KV4_O / 4 : KV4_O, back = e & 1 ? 4 / KV4_Q : 1 / KV4_Q;
                        acc[y][g][e] = times2(acc[y][g][e], f, f);
                        q[y][g][e] = times2(q[y][g][e], back, back);
                    }
        }
#pragma unroll 1
        for (int t = 0; t < tails; ++t) {   // 16 entries of the tail; the last one is the new token
            const int base = (c.blk + blocks + t - c.s.nm) * KV4_ROWS, valid = c.s.tail + 1 - base;
            const T* row[2][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = min(base + i * 4 + sub, c.s.tail);   // no row of another sequence is ever read
                const bool token = j == c.s.tail && a.k_new;
                const int64_t at = (token ? (int64_t)c.b * a.Hkv + h : ((int64_t)c.b * a.Hkv + h) * a.cap + j) * D + 4 * x;
                row[0][i] = static_cast<const T*>(token ? a.k_new : a.k_tail) + at;
                row[1][i] = static_cast<const T*>(token ? a.v_new : a.v_tail) + at;
            }
            float s[M];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint64_t sum[G] = {};
#pragma unroll
                for (int g = 0; g < NG / 2; ++g) {
                    float lo[4], hi[4];
                    load4(row[0][i] + 64 * g, lo);
                    load4(row[0][i] + 64 * g + 32, hi);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint64_t k2 = pack2(lo[e], hi[e]);
#pragma unroll
                        for (int y = 0; y < G; ++y) sum[y] = fma2(q[y][g][e], k2, sum[y]);
                    }
                }
#pragma unroll
                for (int y = 0; y < G; ++y) s[y * 4 + i] = both(sum[y]);
            }
            weights(s, valid, scale_log2);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int g = 0; g < NG / 2; ++g) {
                    float lo[4], hi[4];
                    load4(row[1][i] + 64 * g, lo);
                    load4(row[1][i] + 64 * g + 32, hi);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint64_t v2 = i * 4 + sub < valid ? pack2(lo[e], hi[e]) : 0;   // a repeated row has no weight, but 0 x inf is not 0
#pragma unroll
                        for (int y = 0; y < G; ++y) acc[y][g][e] = fma2(pack2(s[y * 4 + i], s[y * 4 + i]), v2, acc[y][g][e]);
                    }
                }
            if (valid <= KV4_ROWS && a.k_new && gt == 0) {   // entry `tail` of the cache is read by nobody in this launch
                constexpr int N = 16 / sizeof(T);
                if (lane < D / N) {
                    const int64_t from = ((int64_t)c.b * a.Hkv + h) * D / N + lane, to = (((int64_t)c.b * a.Hkv + h) * a.cap + c.s.tail) * D / N + lane;
                    static_cast<uint4*>(a.k_tail)[to] = __ldg(static_cast<const uint4*>(a.k_new) + from);
                    static_cast<uint4*>(a.v_tail)[to] = __ldg(static_cast<const uint4*>(a.v_new) + from);
                }
            }
        }
        const int64_t unit = (int64_t)c.hh * a.B + c.b, seg = w + unit;
        if (lane == 0) kv4_note(a, p, unit, w, c.blk, c.blk + blocks + tails, c.s.n);
#pragma unroll
        for (int o = DUP; o < LH; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
        l += __shfl_xor_sync(0xffffffffu, l, 8);
        l += __shfl_xor_sync(0xffffffffu, l, 16);
        const bool all = c.blk == 0 && blocks + tails == c.s.n;       // the rows' results, not parts of them
        const int64_t row0 = (int64_t)c.b * a.Hq + h * a.g + gt * G;
        if (sub == 0 && x % LH == 0 && x / LH < heads) {
            const float e = ref + log2f(l);
            if (!all) ws[p.lse + seg * p.g_rows + x / LH] = e;
            else if (a.lse) a.lse[row0 + x / LH] = e * 0.6931471805599453f;
        }
#pragma unroll
        for (int y = 0; y < G; ++y) {
            const float inv = 1.f / __shfl_sync(0xffffffffu, l, y * LH);
#pragma unroll
            for (int g = 0; g < NG; g += 2) {
                float lo[4], hi[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    unpack2(acc[y][g / 2][e], lo[e], hi[e]);
#pragma unroll
                    for (int o = 8; o < 32; o <<= 1) {
                        lo[e] += __shfl_xor_sync(0xffffffffu, lo[e], o);
                        hi[e] += __shfl_xor_sync(0xffffffffu, hi[e], o);
                    }
                }
                if (y >= heads || sub != 0) continue;
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const float(&f)[4] = z ? hi : lo;
                    const float4 o = make_float4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
                    if (all) kv4_put(static_cast<T*>(a.o) + (row0 + y) * D + 32 * (g + z) + 4 * x, o);
                    else *reinterpret_cast<float4*>(ws + p.o + (seg * p.g_rows + y) * D + 32 * (g + z) + 4 * x) = o;
                }
            }
        }
        left -= blocks + tails;
        if (left == 0) break;
        kb.next_unit(c);
    }
}

// ------------------------------------------------------------------ tensor cores
// A worker streams its blocks through a ring of its own in shared memory: one bulk copy per block of two tiles (two where pages hold one
// tile), NS - 1 blocks ahead and across the borders between sequences.  The g query heads of a kv head share every row: with 16 entries as the rows and 8 heads as the
// columns of m16n8k16 products,
//     S^T [entries x heads] = K Q^T          O^T [features x heads] += V^T P^T
// A group's step is the same for all entries of a column of K Q^T only within a row, so each group's product (two k-steps) goes
// to an accumulator of its own and into the scores times the row's step; for V the step goes into the weights, so P^T is
// rounded once per group.  P^T changes from the accumulator's layout to the operand's with 8 x 8 transposes (movmatrix).
//
// A tile's numbers are n 2^-133 (n odd, up to 15; times 4 for odd e, see kv4.cuh); the powers of two that queries and weights carry are
// exact and are taken off where memory ends and the tail begins (to_plain), or with the partial result.
template <int D>
struct Kv4Ring {
    static_assert(KV4_ROWS * D * 2 <= 2 * Kv4Tile<D>::BYTES);
    static constexpr int NS = D == 128 ? 3 : 6, STAGE = 2 * Kv4Tile<D>::BYTES,   // two tiles, or 16 rows of the tail
                          WARP = NS * STAGE, TOTAL = KV4_WARPS * WARP;
};

__device__ __forceinline__ void mma_acc(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_new(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// G half-words of eight or four bytes as floats (bf16 bits)
template <int G>
__device__ __forceinline__ void steps_of(const uint8_t* p, float (&h)[G]) {
    if constexpr (G == 4) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        h[0] = bf16lo(u.x); h[1] = bf16hi(u.x); h[2] = bf16lo(u.y); h[3] = bf16hi(u.y);
    } else {
        const uint32_t u = *reinterpret_cast<const uint32_t*>(p);
        h[0] = bf16lo(u); h[1] = bf16hi(u);
    }
}
// Partial results joined: a maximum, a sum and four features, result by result in a fixed order.
struct Kv4Join {
    float M = -INFINITY, total = 0.f;
    float4 o_ = make_float4(0.f, 0.f, 0.f, 0.f);
    // N results at a time, e: log2-sum-exps (-inf: no weight: past the last, or scores of -inf, whose values are 0/0)
    template <int N>
    __device__ __forceinline__ void add(const float (&e)[N], const float4 (&y)[N]) {
        float top = M;
#pragma unroll
        for (int u = 0; u < N; ++u) top = fmaxf(top, e[u]);
        const float keep = M == -INFINITY ? 1.f : exp2f(M - top);   // no weight yet, or NaN, which stays
        M = top;
        total *= keep;
        o_.x *= keep; o_.y *= keep; o_.z *= keep; o_.w *= keep;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if (e[u] == -INFINITY) continue;
            const float f = exp2f(e[u] - top);
            total += f;
            o_.x = fmaf(f, y[u].x, o_.x); o_.y = fmaf(f, y[u].y, o_.y); o_.z = fmaf(f, y[u].z, o_.z); o_.w = fmaf(f, y[u].w, o_.w);
        }
    }
    // the other lane's results, too (lanes that differ in bit o)
    __device__ __forceinline__ void exchange(int o) {
        const float m = __shfl_xor_sync(0xffffffffu, M, o), t = __shfl_xor_sync(0xffffffffu, total, o), top = fmaxf(M, m);
        // a side that took no result, or only ones without weight, has a total of 0; one of NaN alone a total of NaN
        const float f = total == 0.f ? 0.f : exp2f(M - top), g = t == 0.f ? 0.f : exp2f(m - top);
        const float4 y = make_float4(__shfl_xor_sync(0xffffffffu, o_.x, o), __shfl_xor_sync(0xffffffffu, o_.y, o), __shfl_xor_sync(0xffffffffu, o_.z, o),
                                     __shfl_xor_sync(0xffffffffu, o_.w, o));
        M = top;
        total = f * total + g * t;
        o_.x = f * o_.x + g * y.x; o_.y = f * o_.y + g * y.y; o_.z = f * o_.z + g * y.z; o_.w = f * o_.w + g * y.w;
    }
    template <typename T, int D>
    __device__ __forceinline__ void store(const Kv4DecodeArgs& a, int64_t row, int c4) const {   // row = b * Hq + head
        const float inv = 1.f / total;
        kv4_put(static_cast<T*>(a.o) + row * D + c4 * 4, make_float4(o_.x * inv, o_.y * inv, o_.z * inv, o_.w * inv));
        if (a.lse && c4 == 0) a.lse[row] = (M + log2f(total)) * 0.6931471805599453f;
    }
};

// R: column tiles of 8 query heads.  How units are dealt: CUT to workers, or WHOLE to a CTA, or to a cluster of p.whole CTAs.
enum Kv4Dealt { KV4_CUT, KV4_CTA, KV4_CLUSTER };
template <int D, int R, int DEALT>
__global__ void __launch_bounds__(KV4_WARPS * 32, R == 1 ? 3 : 2)
kv4_decode_kernel(const Kv4DecodeArgs a, const Kv4Plan p, int* status) {
    using TL = Kv4Tile<D>;
    constexpr int G = TL::GROUPS, NS = Kv4Ring<D>::NS;
    constexpr bool WHOLE = DEALT != KV4_CUT;
    const int ctas = DEALT == KV4_CLUSTER ? p.whole : 1;
    extern __shared__ __align__(128) uint8_t kv4_smem[];
    __shared__ __align__(8) uint64_t bars[KV4_WARPS][NS];
    __shared__ int64_t scan[WHOLE ? 1 : Kv4Blocks::MAX_GROUPS + 1];
    __shared__ int64_t wsum[KV4_WARPS];
    __shared__ float s_lse[KV4_WARPS][8 * R];
    __shared__ int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, j = lane & 3;
    float* ws = static_cast<float*>(a.ws);
    if (lane == 0)
        for (int i = 0; i < NS; ++i) mbar_init(smem_u32(&bars[warp][i]), 1);
    if (threadIdx.x == 0) abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    let_next_start();
    const Kv4Blocks kb{a};
    int left;                 // blocks of the share still to come
    int64_t w = 0;
    Kv4Blocks::Cursor c;
    if constexpr (WHOLE) {
        const int unit = blockIdx.x / ctas, at = blockIdx.x % ctas * KV4_WARPS + warp;
        c.hh = unit / a.B;
        c.b = unit - c.hh * a.B;
        c.s = kv4_seq(a, c.b);
        if (c.s.n == 0) return;
        c.blk = (int)((int64_t)c.s.n * at / (KV4_WARPS * ctas));
        left = (int)((int64_t)c.s.n * (at + 1) / (KV4_WARPS * ctas)) - c.blk;
        if (left == 0 && lane < 8 * R) s_lse[warp][lane] = -INFINITY;
        __syncthreads();      // barriers and abort flag are set up
    } else {
        const int per = kb.scan(scan, wsum);
        const int64_t T = scan[(a.B + per - 1) / per] * a.Hkv * p.g_tiles, W = min(T, (int64_t)p.workers);
        w = (int64_t)warp * gridDim.x + blockIdx.x;   // neighbours on different SMs
        if (w >= W) return;
        left = (int)(kv4_first(w + 1, T, W) - kv4_first(w, T, W));
        c = kb.find(kv4_first(w, T, W), scan, per);
    }
    int left_f = left;        // blocks still to be fetched
    Kv4Blocks::Cursor f = c;

    // Fetching goes by runs: of memory blocks that lie behind one another in a page (where a page is one tile, lanes 0 and 1 fetch one
    // each), or of a unit's tail blocks, which take two places of the ring, one for the keys' rows and one for the values'; the new token's
    // row is lane 1's.
    const bool small_pages = a.m.log2_ps == 4;
    const int page_blocks = small_pages ? 1 : 1 << (a.m.log2_ps - 5);
    const uint8_t* src = nullptr;
    // rest: entries of the sequence's memory (or tail and new token) from the next block on; values: the next fetch is of a tail block's values
    int run = 0, rest = 0, h_f = p.g_tiles == 1 ? f.hh : f.hh / p.g_tiles;
    bool tail_run = false, values = false;
    auto next_run = [&]() {
        if (left_f <= 0) return;
        if (f.blk == f.s.n) {
            kb.next_unit(f);
            h_f = p.g_tiles == 1 ? f.hh : f.hh / p.g_tiles;
        }
        int blocks;
        tail_run = f.blk >= f.s.nm;
        if (tail_run) {
            blocks = min(f.s.n - f.blk, left_f);
            run = 2 * blocks;
            const int base = (f.blk - f.s.nm) * KV4_ROWS;
            rest = f.s.tail + 1 - base;
            src = reinterpret_cast<const uint8_t*>((((int64_t)f.b * a.Hkv + h_f) * a.cap + base) * D * 2);   // from the start of either cache
        } else {
            rest = f.s.mem - f.blk * KV4_STEP;
            const int entry = f.blk * KV4_STEP + (small_pages && lane == 1 && rest > KV4_ROWS ? KV4_ROWS : 0);
            src = a.m.pool + kv4_tile<D>(a.m, a.Hkv, kv4_page_read(a.m, f.b, entry), h_f, entry);
            blocks = run = min(min(page_blocks - (f.blk & (page_blocks - 1)), f.s.nm - f.blk), left_f);
        }
        f.blk += blocks;
        left_f -= blocks;
    };
    uint8_t* const ring = kv4_smem + warp * Kv4Ring<D>::WARP;
    const uint32_t ring_s = smem_u32(ring), bars_s = smem_u32(&bars[warp][0]);
    int slot_f = 0;
    auto bulk = [&](uint32_t dst, const void* from, int bytes, uint32_t bar) {
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(from), "r"(bytes), "r"(bar) : "memory");
    };
    auto fetch = [&]() {
        const uint32_t bar = bars_s + slot_f * 8, dst = ring_s + slot_f * Kv4Ring<D>::STAGE;
        if (tail_run) {
            const int rows = min(rest, KV4_ROWS), old = rows - (rest <= KV4_ROWS && a.k_new ? 1 : 0);   // without the new token
            if (lane == 0) mbar_expect_tx(bar, rows * D * 2);
            __syncwarp();
            if (lane == 0 && old > 0) bulk(dst, static_cast<const uint8_t*>(values ? a.v_tail : a.k_tail) + reinterpret_cast<uintptr_t>(src), old * D * 2, bar);
            if (lane == 1 && old < rows)
                bulk(dst + old * D * 2, static_cast<const uint8_t*>(values ? a.v_new : a.k_new) + ((int64_t)f.b * a.Hkv + h_f) * D * 2, D * 2, bar);
            if (values) {
                src += KV4_ROWS * D * 2;
                rest -= KV4_ROWS;
            }
            values = !values;
        } else {
            const int bytes = rest > KV4_ROWS ? 2 * TL::BYTES : TL::BYTES;
            if (lane == 0) mbar_expect_tx(bar, bytes);
            __syncwarp();
            if (lane == 0 || (small_pages && lane == 1 && rest > KV4_ROWS)) bulk(dst + lane * TL::BYTES, src, small_pages ? TL::BYTES : bytes, bar);
            src += 2 * TL::BYTES;
            rest -= KV4_STEP;
        }
        slot_f = slot_f + 1 == NS ? 0 : slot_f + 1;
        if (--run == 0) next_run();
    };
    next_run();
    for (int i = 0; i < NS && run > 0; ++i) fetch();

    const uint32_t ones = p.ones;
    const float sc_tail = a.scale * 1.4426950408889634f, sc_mem = sc_tail * KV4_S;
    const int k_at = kv4_k_unit<D>(r, 2 * j), v_at = kv4_v_unit<D>(2 * j, r);   // this lane's keys' row r, and its values' rows 2j, 2j + 1
    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q);
    uint32_t qf[R][2 * G][2];                    // operand B: column = head x * 8 + r
    float m[R][2] = {}, ref[R][2] = {}, l[R][2] = {};   // heads x * 8 + 2j, + 1.  m: the reference as a raw product; ref: what exponents are taken off
    float acc[R][2 * G][4];
    int slot = 0, h = 0, gt = 0, heads = 0;
    uint32_t phase = 0;
    bool ok = true;

    auto load_q = [&](float even, float odd) {
#pragma unroll
        for (int x = 0; x < R; ++x) {
            const int hd = x * 8 + r;
            const __nv_bfloat16* row = q + ((int64_t)c.b * a.Hq + h * a.g + gt * p.g_rows + min(hd, heads - 1)) * D + 8 * j;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                uint4 u = __ldg(reinterpret_cast<const uint4*>(row + 32 * g));
                if (hd >= heads) u = make_uint4(0, 0, 0, 0);
                const uint32_t e0 = __byte_perm(u.x, u.z, 0x5410), e1 = __byte_perm(u.x, u.z, 0x7632), e2 = __byte_perm(u.y, u.w, 0x5410),
                               e3 = __byte_perm(u.y, u.w, 0x7632);
                qf[x][2 * g][0] = pack_bf16(bf16lo(e0) * even, bf16hi(e0) * even);
                qf[x][2 * g][1] = pack_bf16(bf16lo(e1) * odd, bf16hi(e1) * odd);
                qf[x][2 * g + 1][0] = pack_bf16(bf16lo(e2) * even, bf16hi(e2) * even);
                qf[x][2 * g + 1][1] = pack_bf16(bf16lo(e3) * odd, bf16hi(e3) * odd);
            }
        }
    };
    auto to_plain = [&]() {
#pragma unroll
        for (int x = 0; x < R; ++x) {
#pragma unroll
            for (int i = 0; i < 2 * G; ++i) {
                acc[x][i][0] *= KV4_O; acc[x][i][1] *= KV4_O;
                acc[x][i][2] *= KV4_O / 4; acc[x][i][3] *= KV4_O / 4;
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) m[x][y] *= KV4_S;
#pragma unroll
            for (int i = 0; i < 2 * G; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float f = e ? 4 / KV4_Q : 1 / KV4_Q;
                    qf[x][i][e] = pack_bf16(bf16lo(qf[x][i][e]) * f, bf16hi(qf[x][i][e]) * f);
                }
        }
    };
    // the next place of the ring, once its copies are there; and its use for the next fetch, once every lane is done with it
    auto arrived = [&]() {
        ok = __all_sync(0xffffffffu, mbar_wait(bars_s + slot * 8, phase, &abort_flag, status));
        return ring + slot * Kv4Ring<D>::STAGE;
    };
    auto done_with = [&]() {
        __syncwarp();
        if (run > 0) fetch();
        if (++slot == NS) { slot = 0; phase ^= 1; }
    };
    // z: raw products of rows r (0, 1) and r + 8 (2, 3) of one or two tiles, heads 2j, 2j + 1 (-inf: no weight) -> weights
    // 2^(z sc - ref)
    const float grow_mem = 8.f / sc_mem, grow_tail = 8.f / sc_tail;
    auto weights = [&](int x, auto& z, float sc, float grow) {
        constexpr int N = sizeof(z) / sizeof(float);
        float m0 = fmaxf(z[0], z[2]), m1 = fmaxf(z[1], z[3]);
        if constexpr (N > 4) {
            m0 = fmaxf(m0, fmaxf(z[4], z[6]));
            m1 = fmaxf(m1, fmaxf(z[5], z[7]));
        }
        // the reference moves only when a head's maximum has grown by more than 2^8 (weights stay below 2^8)
        if (__any_sync(0xffffffffu, m0 > m[x][0] + grow || m1 > m[x][1] + grow)) {
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, o));
                m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, o));
            }
            m0 = fmaxf(m0, m[x][0]);
            m1 = fmaxf(m1, m[x][1]);
            const float f0 = m0 == -INFINITY ? 1.f : fast_ex2((m[x][0] - m0) * sc), f1 = m1 == -INFINITY ? 1.f : fast_ex2((m[x][1] - m1) * sc);
            m[x][0] = m0;
            m[x][1] = m1;
            ref[x][0] = m0 == -INFINITY ? 0.f : m0 * sc;
            ref[x][1] = m1 == -INFINITY ? 0.f : m1 * sc;
            l[x][0] *= f0;
            l[x][1] *= f1;
#pragma unroll
            for (int i = 0; i < 2 * G; ++i) {
                acc[x][i][0] *= f0; acc[x][i][1] *= f1;
                acc[x][i][2] *= f0; acc[x][i][3] *= f1;
            }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = fast_ex2(fmaf(z[e], sc, -ref[x][e & 1]));
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            l[x][0] += z[e] + z[e + 2];
            l[x][1] += z[e + 1] + z[e + 3];
        }
    };

    while (left > 0) {   // a segment: blocks of memory, then of the tail
        h = p.g_tiles == 1 ? c.hh : c.hh / p.g_tiles;
        gt = c.hh - h * p.g_tiles;
        heads = min(p.g_rows, a.g - gt * p.g_rows);
        const int tiles = min(max(c.s.nm - c.blk, 0), left), tails = min(c.s.n - c.blk - tiles, left - tiles);
        load_q(tiles ? KV4_Q : 1.f, tiles ? KV4_Q / 4 : 1.f);
#pragma unroll
        for (int x = 0; x < R; ++x) {
            m[x][0] = m[x][1] = -INFINITY;
            ref[x][0] = ref[x][1] = 0.f;
            l[x][0] = l[x][1] = 0.f;
#pragma unroll
            for (int i = 0; i < 2 * G; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[x][i][e] = 0.f;
        }
        int valid = c.s.mem - c.blk * KV4_STEP;   // entries from the block on
#pragma unroll 1
        for (int i = 0; i < tiles; ++i, valid -= KV4_STEP) {
            const uint8_t* st = arrived();
            if (!ok) break;
            float s[R][8];   // of the two tiles
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint8_t* tile = st + u * TL::BYTES;
                uint32_t k0[G], k1[G];
                float h0[G], h1[G];
                kv4_unit<G>(tile + k_at, k0);
                kv4_unit<G>(tile + k_at + 8 * TL::ROW, k1);
                steps_of<G>(tile + TL::K_STEPS + r * TL::STEPS, h0);
                steps_of<G>(tile + TL::K_STEPS + (r + 8) * TL::STEPS, h1);
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    uint32_t e0[4], e1[4];
                    kv4_word(k0[g], ones, e0);
                    kv4_word(k1[g], ones, e1);
#pragma unroll
                    for (int x = 0; x < R; ++x) {
                        float t[4];
                        mma_new(t, e0[0], e1[0], e0[1], e1[1], qf[x][2 * g][0], qf[x][2 * g][1]);
                        mma_acc(t, e0[2], e1[2], e0[3], e1[3], qf[x][2 * g + 1][0], qf[x][2 * g + 1][1]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float hs = e < 2 ? h0[g] : h1[g];
                            s[x][4 * u + e] = g == 0 ? t[e] * hs : fmaf(t[e], hs, s[x][4 * u + e]);
                        }
                    }
                }
            }
            if (valid < KV4_STEP) {   // rows past the last entry may hold anything: no weight
#pragma unroll
                for (int x = 0; x < R; ++x)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (r + (e >> 1) * 8 >= valid) s[x][e] = -INFINITY;
            }
#pragma unroll
            for (int x = 0; x < R; ++x) {
                weights(x, s[x], sc_mem, grow_mem);
#pragma unroll
                for (int e = 0; e < 8; ++e) s[x][e] *= KV4_P;
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint8_t* tile = st + u * TL::BYTES;
                uint32_t v0[G], v1[G];
                float h0[G], h1[G];
                kv4_unit<G>(tile + v_at, v0);
                kv4_unit<G>(tile + v_at + 8 * TL::ROW, v1);
                steps_of<G>(tile + TL::V_STEPS + r * TL::STEPS, h0);
                steps_of<G>(tile + TL::V_STEPS + (r + 8) * TL::STEPS, h1);
                if (valid < KV4_STEP) {   // ... and 0 x NaN is not 0
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        if (r + 16 * u >= valid) h0[g] = 0.f;
                        if (r + 16 * u + 8 >= valid) h1[g] = 0.f;
                    }
                }
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    uint32_t e0[4], e1[4];
                    kv4_word(v0[g], ones, e0);
                    kv4_word(v1[g], ones, e1);
#pragma unroll
                    for (int x = 0; x < R; ++x) {
                        // weight times step, rounded to bf16: off by 2^-8 of its value at most; the sums stay in fp32
                        const float* z = s[x] + 4 * u;
                        const uint32_t b0 = transposed(pack_bf16(z[0] * h0[g], z[1] * h0[g])), b1 = transposed(pack_bf16(z[2] * h1[g], z[3] * h1[g]));
                        mma_acc(acc[x][2 * g], e0[0], e0[1], e1[0], e1[1], b0, b1);
                        mma_acc(acc[x][2 * g + 1], e0[2], e0[3], e1[2], e1[3], b0, b1);
                    }
                }
            }
            done_with();
        }
        if (!ok) break;
        if (tiles) to_plain();
#pragma unroll 1
        for (int i = 0; i < tails; ++i) {   // 16 entries of the tail; the last one is the new token
            const int valid = c.s.tail + 1 - (c.blk + tiles + i - c.s.nm) * KV4_ROWS;
            const int64_t cell = ((((int64_t)c.b * a.Hkv + h) * a.cap + c.s.tail) * D) / 8 + lane;
            const bool token = valid <= KV4_ROWS && a.k_new && gt == 0 && lane < D / 8;   // its rows go to the cache, where nobody reads them in this launch
            const uint8_t* st = arrived();
            if (!ok) break;
            float s[R][4];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const uint4 u0 = *reinterpret_cast<const uint4*>(st + (r * D + 32 * g + 8 * j) * 2), u1 = *reinterpret_cast<const uint4*>(st + ((r + 8) * D + 32 * g + 8 * j) * 2);
#pragma unroll
                for (int x = 0; x < R; ++x) {
                    const uint32_t e0[4] = {__byte_perm(u0.x, u0.z, 0x5410), __byte_perm(u0.x, u0.z, 0x7632), __byte_perm(u0.y, u0.w, 0x5410), __byte_perm(u0.y, u0.w, 0x7632)};
                    const uint32_t e1[4] = {__byte_perm(u1.x, u1.z, 0x5410), __byte_perm(u1.x, u1.z, 0x7632), __byte_perm(u1.y, u1.w, 0x5410), __byte_perm(u1.y, u1.w, 0x7632)};
                    if (g == 0) mma_new(s[x], e0[0], e1[0], e0[1], e1[1], qf[x][0][0], qf[x][0][1]);
                    else mma_acc(s[x], e0[0], e1[0], e0[1], e1[1], qf[x][2 * g][0], qf[x][2 * g][1]);
                    mma_acc(s[x], e0[2], e1[2], e0[3], e1[3], qf[x][2 * g + 1][0], qf[x][2 * g + 1][1]);
                }
            }
            if (token) static_cast<uint4*>(a.k_tail)[cell] = *reinterpret_cast<const uint4*>(st + (valid - 1) * D * 2 + lane * 16);
            done_with();
            uint32_t b0[R], b1[R];
#pragma unroll
            for (int x = 0; x < R; ++x) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (r + (e >> 1) * 8 >= valid) s[x][e] = -INFINITY;
                weights(x, s[x], sc_tail, grow_tail);
                b0[x] = transposed(pack_bf16(s[x][0], s[x][1]));
                b1[x] = transposed(pack_bf16(s[x][2], s[x][3]));
            }
            st = arrived();
            if (!ok) break;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                uint2 v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int e = 2 * j + (k & 1) + (k & 2) * 4;
                    v[k] = *reinterpret_cast<const uint2*>(st + (e * D + 32 * g + 4 * r) * 2);
                    if (e >= valid) v[k] = make_uint2(0, 0);   // rows past the last one may hold anything, and 0 x NaN is not 0
                }
#pragma unroll
                for (int x = 0; x < R; ++x) {
                    mma_acc(acc[x][2 * g], __byte_perm(v[0].x, v[1].x, 0x5410), __byte_perm(v[0].x, v[1].x, 0x7632), __byte_perm(v[2].x, v[3].x, 0x5410),
                            __byte_perm(v[2].x, v[3].x, 0x7632), b0[x], b1[x]);
                    mma_acc(acc[x][2 * g + 1], __byte_perm(v[0].y, v[1].y, 0x5410), __byte_perm(v[0].y, v[1].y, 0x7632), __byte_perm(v[2].y, v[3].y, 0x5410),
                            __byte_perm(v[2].y, v[3].y, 0x7632), b0[x], b1[x]);
                }
            }
            if (token) static_cast<uint4*>(a.v_tail)[cell] = *reinterpret_cast<const uint4*>(st + (valid - 1) * D * 2 + lane * 16);
            done_with();
        }
        if (!ok) break;
        // the partial result: in the workspace, or (WHOLE) in place of the ring, which has been used up.  A worker that has done all of a unit
        // has the rows' results
        const bool all = !WHOLE && c.blk == 0 && tiles + tails == c.s.n;
        const int64_t unit = (int64_t)c.hh * a.B + c.b, seg = w + unit;
        if (!WHOLE && lane == 0) kv4_note(a, p, unit, w, c.blk, c.blk + tiles + tails, c.s.n);
        float *const o_part = WHOLE ? reinterpret_cast<float*>(ring) : ws + p.o + seg * p.g_rows * D, *const lse_part = WHOLE ? s_lse[warp] : ws + p.lse + seg * p.g_rows;
#pragma unroll
        for (int x = 0; x < R; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                float lt = l[x][y];
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) lt += __shfl_xor_sync(0xffffffffu, lt, o);
                const int hd = x * 8 + 2 * j + y;
                if (hd < heads) {
                    const float inv = 1.f / lt, e = ref[x][y] + log2f(lt);
                    const int64_t row = (int64_t)c.b * a.Hq + h * a.g + gt * p.g_rows + hd;
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const float4 o = make_float4(acc[x][2 * g][y] * inv, acc[x][2 * g][2 + y] * inv, acc[x][2 * g + 1][y] * inv, acc[x][2 * g + 1][2 + y] * inv);
                        if (all) kv4_put(static_cast<__nv_bfloat16*>(a.o) + row * D + 32 * g + 4 * r, o);
                        else *reinterpret_cast<float4*>(o_part + hd * D + 32 * g + 4 * r) = o;   // 8 lanes: 128 contiguous bytes
                    }
                    if (r == 0 && !all) lse_part[hd] = e;
                    if (r == 0 && all && a.lse) a.lse[row] = e * 0.6931471805599453f;
                }
            }
        left -= tiles + tails;
        if (left > 0) kb.next_unit(c);
    }
    if constexpr (WHOLE) {
        // the unit's rows are dealt to the threads: `ctas` neighbouring lanes to four features of a row, each taking the parts of one CTA
        cg::cluster_group cl = cg::this_cluster();
        if constexpr (DEALT == KV4_CLUSTER) cl.sync();
        else __syncthreads();
        h = c.hh / p.g_tiles;
        gt = c.hh - h * p.g_tiles;
        heads = min(p.g_rows, a.g - gt * p.g_rows);
        const int items = heads * (D / 4), cta = lane % ctas, per = KV4_WARPS * 32 / ctas;
        const float* lse = &s_lse[0][0];
        const uint8_t* part = kv4_smem;
        if constexpr (DEALT == KV4_CLUSTER) {
            lse = cl.map_shared_rank(lse, cta);
            part = cl.map_shared_rank(part, cta);
        }
        for (int i0 = blockIdx.x % ctas * per; i0 < items; i0 += KV4_WARPS * 32) {
            const int i = min(i0 + (int)threadIdx.x / ctas, items - 1), hd = i / (D / 4), c4 = i % (D / 4);
            float e[KV4_WARPS];
            float4 y[KV4_WARPS];
#pragma unroll
            for (int u = 0; u < KV4_WARPS; ++u) {
                e[u] = lse[u * 8 * R + hd];
                y[u] = *reinterpret_cast<const float4*>(part + u * Kv4Ring<D>::WARP + (hd * D + c4 * 4) * 4);
            }
            Kv4Join join;
            join.add(e, y);
            for (int o = 1; o < ctas; o <<= 1) join.exchange(o);
            if (cta == 0 && i0 + (int)threadIdx.x / ctas < items) join.store<__nv_bfloat16, D>(a, (int64_t)c.b * a.Hq + h * a.g + gt * p.g_rows + hd, c4);
        }
        if constexpr (DEALT == KV4_CLUSTER) cl.sync();   // nobody leaves while its results are being read
    }
    if (!ok) {
        // leaving early: give copies already in flight a bounded time to land in this CTA's shared memory
        const long long t_off = clock64();
        while (clock64() - t_off < 2000000ll) {}
    }
}

// ------------------------------------------------------------------ merge
// A row's D features are D / 4 lanes; WAYS sets of lanes share a row's partial results.  Results are fetched several at a time: the chain of
// loads is what takes time.
constexpr int KV4_MERGE_THREADS = 128;

template <typename T, int D, int WAYS>
__global__ void __launch_bounds__(KV4_MERGE_THREADS)
kv4_merge_kernel(const Kv4DecodeArgs a, const Kv4Plan p) {
    constexpr int LANES = D / 4, ROWS = KV4_MERGE_THREADS / LANES / WAYS, AT_ONCE = WAYS > 1 ? 8 : 4;
    const int c4 = threadIdx.x % LANES, set = threadIdx.x / LANES, way = set % WAYS;
    const int row = blockIdx.x * ROWS + set / WAYS;       // B * Hq fits 32 bits
    const bool there = row < a.B * a.Hq;
    const int b = there ? row / a.Hq : 0, hq = there ? row - b * a.Hq : 0;
    const int h = hq / a.g, j = hq - h * a.g, gt = j / p.g_rows, x = j - gt * p.g_rows;
    const bool live = there && __ldg(a.tail_lens + b) >= 0;
    const float* ws = static_cast<const float*>(a.ws);
    wait_for_previous();
    Kv4Join join;
    int n = 0;               // partial results; 0: a worker has done all of the unit
    if (live) {
        const int64_t unit = (int64_t)(h * p.g_tiles + gt) * a.B + b;
        const int32_t* ends = reinterpret_cast<const int32_t*>(ws + p.ends) + unit;
        int w0;
        n = kv4_parts(__ldcg(ends), __ldcg(ends + (int64_t)a.B * a.Hkv * p.g_tiles), p.workers, &w0);
        const int64_t first = (w0 + unit) * p.g_rows + x;
        const float *lse = ws + p.lse + first, *v = ws + p.o + first * D + c4 * 4;
        for (int s0 = way * AT_ONCE; s0 < n; s0 += WAYS * AT_ONCE) {
            float e[AT_ONCE];
            float4 y[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                e[u] = -INFINITY;
                if (s0 + u < n) {
                    e[u] = __ldcg(lse + (int64_t)(s0 + u) * p.g_rows);
                    y[u] = __ldcg(reinterpret_cast<const float4*>(v + (int64_t)(s0 + u) * p.g_rows * D));
                }
            }
            join.add(e, y);
        }
    }
    if constexpr (WAYS > 1) {
        __shared__ Kv4Join s_part[KV4_MERGE_THREADS];
        s_part[threadIdx.x] = join;
        __syncthreads();
        if (way > 0) return;
        Kv4Join all;
        for (int y = 0; y < WAYS; ++y) all.M = fmaxf(all.M, s_part[threadIdx.x + y * LANES].M);
        for (int y = 0; y < WAYS; ++y) {
            const Kv4Join& q = s_part[threadIdx.x + y * LANES];
            if (q.total == 0.f) continue;   // took no result, or only ones without weight (one of NaN alone has a total of NaN)
            const float f = exp2f(q.M - all.M);
            all.total += f * q.total;
            all.o_.x = fmaf(f, q.o_.x, all.o_.x); all.o_.y = fmaf(f, q.o_.y, all.o_.y); all.o_.z = fmaf(f, q.o_.z, all.o_.z); all.o_.w = fmaf(f, q.o_.w, all.o_.w);
        }
        join = all;
    }
    if (n > 0) join.store<T, D>(a, row, c4);
}

// ------------------------------------------------------------------ host side
// both kernels' cuts, array by array, so that a buffer made for the largest call serves the smaller ones
size_t decode_kv4_workspace_bytes(int B, int Hq, int Hkv, int D, int max_mem, int max_tail) {
    int64_t rows = 0, units = 0;
    for (bool cuda_cores : {false, true}) {
        const Kv4Plan p = make_kv4_plan(B, Hq, Hkv, D, max_mem, max_tail, cuda_cores);
        units = std::max(units, (int64_t)B * Hkv * p.g_tiles);
        rows = std::max(rows, (p.workers + (int64_t)B * Hkv * p.g_tiles) * p.g_rows);
    }
    int64_t n = 0;
    for (int64_t x : {rows * D, rows, 2 * units}) n += (x + 63) / 64 * 64;
    return (size_t)n * sizeof(float);
}

// Rows of long lists of partial results are shared by all of a CTA's sets of lanes.
template <typename T, int D>
static cudaError_t merge(const Kv4DecodeArgs& a, const Kv4Plan& p, cudaStream_t st) {
    constexpr int SETS = KV4_MERGE_THREADS / (D / 4);
    const int rows = a.B * a.Hq;
    if (p.workers > 8 * (int64_t)a.B * a.Hkv * p.g_tiles)
        return launch_behind(kv4_merge_kernel<T, D, SETS>, dim3(rows), KV4_MERGE_THREADS, 0, st, true, a, p);
    return launch_behind(kv4_merge_kernel<T, D, 1>, dim3((rows + SETS - 1) / SETS), KV4_MERGE_THREADS, 0, st, true, a, p);
}

template <typename T, int D>
static cudaError_t stream(const Kv4DecodeArgs& a, cudaStream_t st) {
    const Kv4Plan p = make_kv4_plan(a.B, a.Hq, a.Hkv, D, a.max_mem, a.max_tail, true);
    auto* kernel = p.g_rows == 1 ? kv4_stream_kernel<T, D, 1> : p.g_rows == 2 ? kv4_stream_kernel<T, D, 2> : kv4_stream_kernel<T, D, 4>;
    const cudaError_t e = launch_behind(kernel, dim3(p.ctas), KV4_WARPS * 32, 0, st, false, a, p);
    return e == cudaSuccess ? merge<T, D>(a, p, st) : e;
}

template <int D>
static cudaError_t tensor_cores(const Kv4DecodeArgs& a, cudaStream_t st) {
    const Kv4Plan p = make_kv4_plan(a.B, a.Hq, a.Hkv, D, a.max_mem, a.max_tail, false);
    int* status = device_status_word();
    if (!status) return cudaErrorUnknown;
    const bool narrow = p.g_rows <= 8;
    const dim3 units(a.B * a.Hkv * p.g_tiles), threads(KV4_WARPS * 32);
    constexpr int smem = Kv4Ring<D>::TOTAL;
    if (p.whole == 1) return launch_behind(narrow ? kv4_decode_kernel<D, 1, KV4_CTA> : kv4_decode_kernel<D, 2, KV4_CTA>, units, threads, smem, st, false, a, p, status);
    if (p.whole) {
        auto* kernel = narrow ? kv4_decode_kernel<D, 1, KV4_CLUSTER> : kv4_decode_kernel<D, 2, KV4_CLUSTER>;
        cudaError_t e = prepare_kernel(reinterpret_cast<const void*>(kernel), smem);
        if (e != cudaSuccess) return e;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(units.x * p.whole);
        cfg.blockDim = threads;
        cfg.dynamicSmemBytes = smem;
        cfg.stream = st;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = p.whole;
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        e = cudaLaunchKernelEx(&cfg, kernel, a, p, status);
        if (e == cudaSuccess) count_launches(1);
        return e;
    }
    const cudaError_t e = launch_behind(narrow ? kv4_decode_kernel<D, 1, KV4_CUT> : kv4_decode_kernel<D, 2, KV4_CUT>, dim3(p.ctas), threads, smem, st, false, a, p, status);
    return e == cudaSuccess ? merge<__nv_bfloat16, D>(a, p, st) : e;
}

cudaError_t launch_decode_kv4(const Kv4DecodeArgs& a, int D, loma_dtype dt, bool generic, cudaStream_t st) {
    if (dt == LOMA_F32) return D == 64 ? stream<float, 64>(a, st) : stream<float, 128>(a, st);
    if (generic) return D == 64 ? stream<__nv_bfloat16, 64>(a, st) : stream<__nv_bfloat16, 128>(a, st);
    return D == 64 ? tensor_cores<64>(a, st) : tensor_cores<128>(a, st);
}

}  // namespace loma
