// Checks of arguments that the extern "C" entry points of several files share.
#pragma once

#include <algorithm>

#include "loma_internal.cuh"

namespace loma {

inline bool misaligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }
inline size_t elt_bytes(loma_dtype dt) { return dt == LOMA_F32 ? 4 : 2; }
inline int from_cuda(cudaError_t e) { return e == cudaSuccess ? LOMA_OK : LOMA_ERR_CUDA; }

// do [a, a + na) and [b, b + nb) bytes meet?
inline bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
    if (!a || !b || na <= 0 || nb <= 0) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

// n strided axes over rows of D elements: false if two rows may share an element (a stride of 0 included)
inline bool rows_apart(int n, const int64_t* extent, const int64_t* stride, int D) {
    int order[3] = {0, 1, 2};
    std::sort(order, order + n, [&](int x, int y) { return stride[x] < stride[y]; });
    int64_t span = D;
    for (int i = 0; i < n; ++i) {
        const int a = order[i];
        if (extent[a] <= 1) continue;
        if (stride[a] < span) return false;
        if (stride[a] > INT64_MAX / 4 / extent[a]) return false;
        span = stride[a] * (extent[a] - 1) + span;
    }
    return true;
}

}  // namespace loma
