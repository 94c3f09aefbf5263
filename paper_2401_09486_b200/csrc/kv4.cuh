// Memory entries held in 4 bits: the format, and what its kernels have in common.
//
// 32 consecutive features of a row share a step h = bf16(fp32(max |x| / 15)); a value is held as its sign and m = 0 .. 7, the number of
// k in 1 .. 7 with |x| >= 2 h k, and stands for +-(2 m + 1) h: sixteen evenly spaced values around zero, the outermost of which
// is the group's largest.  Thresholds 2 h k are exact in fp32, so is 2 m + 1 times h, and nothing is rounded but h.  A step below 2^-126
// is stored as 0 (all values 0), one that is no number as NaN (all values NaN).
//
// A pool is [n_pages][Hkv][page_size / 16] tiles of 16 entries.  A tile holds, for its 16 rows, the keys' bits, the values' bits, the
// keys' steps, the values' steps, one behind the other, so one copy fetches it: 2304 bytes for D = 128 (in bf16: 8192).
//
// The bits are laid out for warp-level m16n8k16 products.  Feature 32 g + 4 x + e (group g, x = 0 .. 7, e = 0 .. 3) lies in half-word (x, g)
// of its row, whose 16 bits are
//     m0 m1 s2 s3 | m2 m3 s0 s1        (3 3 1 1 | 3 3 1 1 bits, lowest first; s: sign)
// In a word of two half-words that want to be neighbours in an operand, the word itself (e = 1), doubled (e = 0), and the same with the
// bytes of each half exchanged (e = 3, 2) have sign and m where one AND and one OR make them the bf16 pattern of +-(2 m + 1) 2^-133
// (times 4 for odd e): a number below the normal range, which the products take as it is.  So 4 bits turn into operands in under two
// instructions a pair, with no offset to be taken off again; powers of two bring the sums back (see KV4_Q and the like).
// Neighbours are, for keys, half-words x and x + 1 (x even) of a row: word g of unit x / 2, four units to a row, row after row.  For
// values, rows k and k + 1 (k even): word g of unit x, eight units to a pair of rows, unit x of pair p at x ^ 2 (p & 3) (D = 64: p & 2), which
// spreads the reads of a tile in shared memory over its banks.
#pragma once

#include <algorithm>

#include "loma_internal.cuh"

namespace loma {

constexpr int KV4_ROWS = 16;    // entries to a tile
constexpr int KV4_GROUP = 32;   // features that share a step

template <int D>
struct Kv4Tile {
    static constexpr int GROUPS = D / KV4_GROUP;
    static constexpr int UNIT = 4 * GROUPS;                      // bytes: a word per group
    static constexpr int ROW = D / 2, STEPS = GROUPS * 2;        // bytes of a row's bits and of its steps
    static constexpr int V = KV4_ROWS * ROW, K_STEPS = 2 * V, V_STEPS = K_STEPS + KV4_ROWS * STEPS;   // where they begin
    static constexpr int BYTES = V_STEPS + KV4_ROWS * STEPS;
};

inline int64_t kv4_tile_bytes(int D) { return D == 64 ? Kv4Tile<64>::BYTES : Kv4Tile<128>::BYTES; }

// the 4-bit memory of a batch
struct Kv4Pool {
    uint8_t* pool = nullptr;
    const int32_t* table = nullptr;   // [B, max_pages]
    int max_pages = 0, log2_ps = 0, n_pages = 0;
};

struct Kv4AppendArgs {
    Kv4Pool m;
    const void *k = nullptr, *v = nullptr;
    int64_t k_stride[3] = {0, 0, 0}, v_stride[3] = {0, 0, 0};   // batch, head, row, in elements
    const int32_t *mem_lens = nullptr, *new_lens = nullptr;
    int B = 0, Hkv = 0, l = 0;
};
struct Kv4LoadArgs {
    Kv4Pool m;
    void *k = nullptr, *v = nullptr;   // [B, Hkv, cap, D]
    const int32_t* mem_lens = nullptr;
    int B = 0, Hkv = 0, cap = 0;
    uint32_t ones = 0x00010001u;       // see kv4_word
};
cudaError_t launch_kv4_append(const Kv4AppendArgs& a, int D, loma_dtype dt, cudaStream_t st);   // kv4_store.cu
cudaError_t launch_kv4_load(const Kv4LoadArgs& a, int D, loma_dtype dt, cudaStream_t st);

struct Kv4DecodeArgs {
    Kv4Pool m;
    const void *q = nullptr, *k_new = nullptr, *v_new = nullptr;   // [B, Hq, D], [B, Hkv, D]; k_new, v_new may be NULL
    void *k_tail = nullptr, *v_tail = nullptr;                     // [B, Hkv, cap, D]
    void* o = nullptr;                                             // [B, Hq, D]
    float* lse = nullptr;                                          // [B, Hq] or NULL
    const int32_t *mem_lens = nullptr, *tail_lens = nullptr;       // [B]; tail_lens negative: no request, nothing is written
    int B = 0, Hq = 0, Hkv = 0, g = 0;
    int max_mem = 0, max_tail = 0, cap = 0;
    float scale = 0.f;
    void* ws = nullptr;
};
// The partial results of a cut unit, from the notes of its first and its last worker: how many, and the first one's worker.  first 1, last 0: none,
// one worker has done all of it.  A worker whose bounded wait has run out leaves its notes as they were in the workspace, so any number may
// stand there: what is read stays among the workers' slots.
__host__ __device__ inline int kv4_parts(int first, int last, int workers, int* begin) {
    *begin = first < 0 ? 0 : first >= workers ? workers - 1 : first;
    return last < *begin ? 0 : (last >= workers ? workers - 1 : last) - *begin + 1;
}
size_t decode_kv4_workspace_bytes(int B, int Hq, int Hkv, int D, int max_mem, int max_tail);   // decode_kv4.cu
cudaError_t launch_decode_kv4(const Kv4DecodeArgs& a, int D, loma_dtype dt, bool generic, cudaStream_t st);

#ifdef __CUDACC__
// page of block `block` of sequence b, or -1 where the table names none in the pool
__device__ __forceinline__ int kv4_page(const Kv4Pool& m, int b, int block) {
    const int page = __ldg(m.table + (int64_t)b * m.max_pages + block);
    return page >= 0 && page < m.n_pages ? page : -1;
}
// where the tile of entry j of (page, h) begins
template <int D>
__device__ __forceinline__ int64_t kv4_tile(const Kv4Pool& m, int Hkv, int page, int h, int j) {
    const int tiles = 1 << (m.log2_ps - 4), t = (j & ((1 << m.log2_ps) - 1)) >> 4;
    return (((int64_t)page * Hkv + h) * tiles + t) * Kv4Tile<D>::BYTES;
}
// byte offsets of the units that hold half-words x of row k, among a tile's keys and from its beginning (values)
template <int D>
__device__ __forceinline__ int kv4_k_unit(int k, int x) { return k * Kv4Tile<D>::ROW + (x >> 1) * Kv4Tile<D>::UNIT; }
template <int D>
__device__ __forceinline__ int kv4_v_unit(int k, int x) {
    return Kv4Tile<D>::V + (k >> 1) * 2 * Kv4Tile<D>::ROW + (x ^ (k & (D == 128 ? 6 : 4))) * Kv4Tile<D>::UNIT;
}

// The four elements e of a word's two half-words as bf16 pairs, +-(2 m + 1) 2^-133, times 4 for odd e.  ones: 0x00010001, from a kernel
// parameter: an AND-OR takes one constant in the instruction, and the other one, where the compiler knows it, is moved to a register
// before every use.
__device__ __forceinline__ void kv4_word(uint32_t u, uint32_t ones, uint32_t (&p)[4]) {
    const uint32_t w = __byte_perm(u, 0, 0x2301);
    p[0] = ((u << 1) & 0x800E800Eu) | ones;
    p[1] = (u & 0x80388038u) | ones << 2;
    p[2] = ((w << 1) & 0x800E800Eu) | ones;
    p[3] = (w & 0x80388038u) | ones << 2;
}
// Powers of two that keep sums over these patterns in the normal range: queries carry 2^64 (2^62 against odd e), weights 2^80 (after
// their sum has been taken), so scores come out times 2^-69 and outputs times 2^-53 (2^-51).
constexpr float KV4_Q = 18446744073709551616.f;                    // 2^64
constexpr float KV4_S = 590295810358705651712.f;                   // 2^69
constexpr float KV4_P = 1208925819614629174706176.f;               // 2^80
constexpr float KV4_O = 9007199254740992.f;                        // 2^53

// the G words of a unit
template <int G>
__device__ __forceinline__ void kv4_unit(const uint8_t* p, uint32_t (&w)[G]) {
    if constexpr (G == 4) {
        const uint4 u = *reinterpret_cast<const uint4*>(p);
        w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
    } else {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        w[0] = u.x; w[1] = u.y;
    }
}
// one row's half-words of a unit, groups 2 i and 2 i + 1 in word i
template <int G>
__device__ __forceinline__ void kv4_halves(const uint8_t* p, bool upper, uint32_t (&w)[G / 2]) {
    uint32_t u[G];
    kv4_unit<G>(p, u);
#pragma unroll
    for (int i = 0; i < G / 2; ++i) w[i] = __byte_perm(u[2 * i], u[2 * i + 1], upper ? 0x7632 : 0x5410);
}
// a row's steps, groups 2 i and 2 i + 1 in word i
template <int G>
__device__ __forceinline__ void kv4_steps(const uint8_t* p, uint32_t (&w)[G / 2]) {
    if constexpr (G == 4) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        w[0] = u.x; w[1] = u.y;
    } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
}
#endif

}  // namespace loma
