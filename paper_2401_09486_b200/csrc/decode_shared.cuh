// What the kernels of the shared-prefix decode step have in common: how the work is cut and where partial results lie.
#pragma once

#include <algorithm>

#include "loma_internal.cuh"

namespace loma {

constexpr int SHP_ROWS = 128;   // query rows of a prefix tile

// The cut of a call.  Depends on the sizes alone, so results repeat and the workspace can be sized before the call.
struct SharedPlan {
    int m_tiles;      // prefix: tiles of SHP_ROWS query rows per kv head
    int p_splits;     // prefix: key ranges (0: no prefix)
    int p_len;        //         keys per range, a multiple of 128
    int own_splits;   // own cache: key ranges per (sequence, kv head)
    int own_len;      //            keys per range, a multiple of 64
    // partial results in the workspace, as offsets in floats.  Prefix tile (split, kv head, tile): outputs [D/4][128][4]
    // (so that a warp whose lanes are rows stores 512 contiguous bytes) and 128 log2-sum-exps.  Own range
    // (sequence, kv head, split): outputs [g][D] and g log2-sum-exps.  -inf marks an empty range, whose outputs are not written.
    int64_t p_o, p_lse, own_o, own_lse, total;
};

inline SharedPlan make_shared_plan(int B, int Hq, int Hkv, int D, int prefix_len, int max_len) {
    SharedPlan p;
    const int64_t g = Hq / Hkv, rows = (int64_t)B * g;
    p.m_tiles = (int)((rows + SHP_ROWS - 1) / SHP_ROWS);
    p.p_splits = 0;
    p.p_len = 128;
    if (prefix_len > 0) {
        // two CTAs per SM; a range is never shorter than 128 keys (one key tile)
        const int64_t tiles = (int64_t)p.m_tiles * Hkv, key_tiles = (prefix_len + 127) / 128;
        int64_t splits = std::max<int64_t>(1, 296 / tiles);
        splits = std::min<int64_t>(std::min<int64_t>(splits, key_tiles), 64);
        const int64_t per = (key_tiles + splits - 1) / splits;
        p.p_len = (int)per * 128;
        p.p_splits = (int)((key_tiles + per - 1) / per);
    }
    const int64_t pairs = (int64_t)B * Hkv * ((g + 15) / 16), keys = (int64_t)max_len + 1;
    int64_t splits = std::max<int64_t>((keys + 1023) / 1024, (4 * 148 + pairs - 1) / pairs);
    splits = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(splits, keys / 128), 64));
    p.own_len = (int)(((keys + splits - 1) / splits + 63) / 64 * 64);
    p.own_splits = (int)((keys + p.own_len - 1) / p.own_len);
    int64_t at = 0;
    auto take = [&](int64_t n) { const int64_t o = at; at += (n + 63) / 64 * 64; return o; };
    const int64_t p_tiles = (int64_t)p.p_splits * Hkv * p.m_tiles, own = (int64_t)B * Hkv * p.own_splits;
    p.p_o = take(p_tiles * SHP_ROWS * D);
    p.p_lse = take(p_tiles * SHP_ROWS);
    p.own_o = take(own * g * D);
    p.own_lse = take(own * g);
    p.total = at;
    return p;
}

// the prefix on the tensor cores (decode_shared_tc.cu); cudaErrorNotSupported = use the CUDA-core kernel
cudaError_t launch_shared_prefix_tc(const SharedArgs& a, const SharedPlan& p, int D, cudaStream_t st);

}  // namespace loma
