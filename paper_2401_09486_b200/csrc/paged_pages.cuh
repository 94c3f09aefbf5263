// The life of cache pages after loma_paged_extend handed them out: arguments shared by paged_pages.cu and its callers.
#pragma once

#include "loma_internal.cuh"

namespace loma {

// Pages of the pool: free_pages[taken .. n_free) are free, refs[p] counts the table rows beyond the first that name page p.
struct PageList {
    int n_pages = 0, n_free = 0;
    int32_t *refs = nullptr, *free_pages = nullptr, *taken = nullptr;
};
struct ReleaseArgs {
    PageList pl;
    int B = 0, log2_ps = 0, max_pages = 0;
    const int32_t *keep_lens = nullptr, *held = nullptr;
    int32_t *block_table = nullptr, *held_out = nullptr, *counts = nullptr;
};
struct ForkArgs {
    PageList pl;
    int B = 0, log2_ps = 0, max_pages = 0, max_copies = 0;
    const int32_t *parents = nullptr, *cache_lens = nullptr, *fixed_lens = nullptr, *held = nullptr, *block_table = nullptr;
    int32_t *table_out = nullptr, *lens_out = nullptr, *held_out = nullptr, *copy_src = nullptr, *copy_dst = nullptr, *counts = nullptr;
    int32_t* ws = nullptr;   // [2 * B]
};
struct CompactArgs {
    PageList pl;
    int B = 0, max_pages = 0, max_copies = 0;
    const int32_t* held = nullptr;
    int32_t *block_table = nullptr, *page_map = nullptr, *copy_src = nullptr, *copy_dst = nullptr, *counts = nullptr;
};
constexpr int COPY_POOLS = 64;   // of one launch
struct CopyArgs {
    int n_pools = 0, n_pages = 0, max_copies = 0;
    const int32_t *src = nullptr, *dst = nullptr, *n = nullptr;
    uint8_t* pool[COPY_POOLS] = {};
    int64_t bytes[COPY_POOLS] = {};   // of a page
};

void host_paged_release(const ReleaseArgs& a);
void host_paged_fork(const ForkArgs& a);
void host_paged_compact(const CompactArgs& a);
cudaError_t launch_paged_release(const ReleaseArgs& a, cudaStream_t st);
cudaError_t launch_paged_fork(const ForkArgs& a, cudaStream_t st);
cudaError_t launch_paged_compact(const CompactArgs& a, cudaStream_t st);
cudaError_t launch_paged_copy(const CopyArgs& a, cudaStream_t st);

}  // namespace loma
