// extern "C" boundary of the operators around a paged cache: memory entries in 4 bits, and the pages' life after loma_paged_extend.
// Every check happens on the host before anything is enqueued.
#include <limits.h>
#include <math.h>

#include <initializer_list>

#include "api_checks.cuh"
#include "kv4.cuh"
#include "paged_pages.cuh"

using namespace loma;

namespace {

struct Range {
    const void* p;
    int64_t n;   // bytes
};

// no output may meet an input or another output
bool apart(std::initializer_list<Range> ins, std::initializer_list<Range> outs) {
    for (const Range* x = outs.begin(); x != outs.end(); ++x) {
        for (const Range& y : ins)
            if (overlap(x->p, x->n, y.p, y.n)) return false;
        for (const Range* y = outs.begin(); y != x; ++y)
            if (overlap(x->p, x->n, y->p, y->n)) return false;
    }
    return true;
}

// Can an array of that many bytes be?  Offsets and ends of arrays are 64-bit sums.
bool fits(std::initializer_list<int64_t> factors) {
    int64_t n = 1;
    for (int64_t x : factors)
        if (x == 0) return true;
    for (int64_t x : factors) {
        if (n > (INT64_MAX >> 3) / x) return false;
        n *= x;
    }
    return true;
}

// ------------------------------------------------------------------ 4-bit memory
int kv4_sizes(int B, int Hkv, int D, int page_size, int max_pages, int n_pages, loma_dtype dtype, int* l2) {
    if (B < 0 || Hkv < 0 || max_pages < 0 || n_pages < 0) return LOMA_ERR_INVALID_ARG;
    if (dtype != LOMA_F32 && dtype != LOMA_BF16) return LOMA_ERR_UNSUPPORTED;
    if (D != 64 && D != 128) return LOMA_ERR_UNSUPPORTED;
    *l2 = log2_exact(page_size);
    if (*l2 < 4 || page_size > 65536) return LOMA_ERR_INVALID_ARG;
    if ((int64_t)max_pages * page_size > INT_MAX) return LOMA_ERR_INVALID_ARG;
    if (!fits({n_pages, Hkv, page_size, 2 * D}) || !fits({4, B, max_pages})) return LOMA_ERR_INVALID_ARG;
    return LOMA_OK;
}

Kv4Pool kv4_pool(void* pool, const int32_t* table, int max_pages, int l2, int n_pages) {
    Kv4Pool m;
    m.pool = static_cast<uint8_t*>(pool);
    m.table = table; m.max_pages = max_pages; m.log2_ps = l2; m.n_pages = n_pages;
    return m;
}

int64_t kv4_pool_bytes(int Hkv, int D, int l2, int n_pages) { return ((int64_t)n_pages * Hkv << (l2 - 4)) * kv4_tile_bytes(D); }

}  // namespace

extern "C" {

size_t loma_kv4_page_bytes(int Hkv, int D, int page_size) {
    const int l2 = log2_exact(page_size);
    if (Hkv <= 0 || (D != 64 && D != 128) || l2 < 4 || page_size > 65536) return 0;
    return (size_t)kv4_pool_bytes(Hkv, D, l2, 1);
}

int loma_kv4_append(const void* k, const void* v, void* kv_pool, const int32_t* block_table, const int32_t* mem_lens, const int32_t* new_lens,
                    int B, int Hkv, int D, int l, int page_size, int max_pages, int n_pages, const int64_t* k_strides, const int64_t* v_strides,
                    loma_dtype dtype, void* stream) {
    int l2;
    const int rc = kv4_sizes(B, Hkv, D, page_size, max_pages, n_pages, dtype, &l2);
    if (rc != LOMA_OK) return rc;
    if (l < 0 || l > INT_MAX - 4096 || !fits({B, Hkv, l, D, 4})) return LOMA_ERR_INVALID_ARG;
    if (B == 0 || Hkv == 0 || l == 0) return LOMA_OK;
    if (!k || !v || !kv_pool || !block_table || !mem_lens || !k_strides || !v_strides || n_pages < 1) return LOMA_ERR_INVALID_ARG;
    Kv4AppendArgs a;
    const int64_t extent[3] = {B, Hkv, l};
    const int64_t* st[2] = {k_strides, v_strides};
    for (int i = 0; i < 2; ++i) {
        for (int x = 0; x < 3; ++x) if (st[i][x] < 0) return LOMA_ERR_INVALID_ARG;
        if (!rows_apart(3, extent, st[i], D)) return LOMA_ERR_INVALID_ARG;
        for (int x = 0; x < 3; ++x)
            if (extent[x] > 1 && (st[i][x] * (int64_t)elt_bytes(dtype)) % 16) return LOMA_ERR_ALIGNMENT;
        for (int x = 0; x < 3; ++x) (i ? a.v_stride : a.k_stride)[x] = st[i][x];
    }
    for (const void* p : {k, v, (const void*)kv_pool}) if (misaligned(p, 16)) return LOMA_ERR_ALIGNMENT;
    for (const int32_t* p : {block_table, mem_lens, new_lens}) if (misaligned(p, 4)) return LOMA_ERR_ALIGNMENT;
    const Range pool{kv_pool, kv4_pool_bytes(Hkv, D, l2, n_pages)};
    int64_t span[2];
    for (int i = 0; i < 2; ++i) {
        span[i] = D;
        for (int x = 0; x < 3; ++x) span[i] += (extent[x] - 1) * st[i][x];
        if (!fits({span[i], 4})) return LOMA_ERR_INVALID_ARG;
    }
    if (!apart({{k, span[0] * (int64_t)elt_bytes(dtype)}, {v, span[1] * (int64_t)elt_bytes(dtype)}, {block_table, 4ll * B * max_pages},
                {mem_lens, 4ll * B}, {new_lens, 4ll * B}}, {pool})) return LOMA_ERR_INVALID_ARG;
    const int dc = check_device();
    if (dc != LOMA_OK) return dc;
    a.m = kv4_pool(kv_pool, block_table, max_pages, l2, n_pages);
    a.k = k; a.v = v; a.mem_lens = mem_lens; a.new_lens = new_lens; a.B = B; a.Hkv = Hkv; a.l = l;
    return from_cuda(launch_kv4_append(a, D, dtype, static_cast<cudaStream_t>(stream)));
}

int loma_kv4_load(const void* kv_pool, const int32_t* block_table, const int32_t* mem_lens, void* k_cache, void* v_cache, int B, int Hkv, int D,
                  int cap, int page_size, int max_pages, int n_pages, loma_dtype dtype, void* stream) {
    int l2;
    const int rc = kv4_sizes(B, Hkv, D, page_size, max_pages, n_pages, dtype, &l2);
    if (rc != LOMA_OK) return rc;
    if (cap < 0 || cap > INT_MAX - 4096 || !fits({B, Hkv, cap, D, 4})) return LOMA_ERR_INVALID_ARG;
    if (B == 0 || Hkv == 0 || cap == 0) return LOMA_OK;
    if (!kv_pool || !block_table || !mem_lens || !k_cache || !v_cache || n_pages < 1) return LOMA_ERR_INVALID_ARG;
    for (const void* p : {kv_pool, (const void*)k_cache, (const void*)v_cache}) if (misaligned(p, 16)) return LOMA_ERR_ALIGNMENT;
    for (const int32_t* p : {block_table, mem_lens}) if (misaligned(p, 4)) return LOMA_ERR_ALIGNMENT;
    const int64_t bytes = (int64_t)B * Hkv * cap * D * (int64_t)elt_bytes(dtype);
    if (!apart({{kv_pool, kv4_pool_bytes(Hkv, D, l2, n_pages)}, {block_table, 4ll * B * max_pages}, {mem_lens, 4ll * B}},
               {{k_cache, bytes}, {v_cache, bytes}})) return LOMA_ERR_INVALID_ARG;
    const int dc = check_device();
    if (dc != LOMA_OK) return dc;
    Kv4LoadArgs a;
    a.m = kv4_pool(const_cast<void*>(kv_pool), block_table, max_pages, l2, n_pages);
    a.k = k_cache; a.v = v_cache; a.mem_lens = mem_lens; a.B = B; a.Hkv = Hkv; a.cap = cap;
    return from_cuda(launch_kv4_load(a, D, dtype, static_cast<cudaStream_t>(stream)));
}

static int kv4_decode_sizes(int B, int Hq, int Hkv, int D, int max_mem, int max_tail) {
    if (B < 0 || Hq < 0 || Hkv < 0 || max_mem < 0 || max_tail < 0) return LOMA_ERR_INVALID_ARG;
    if (D != 64 && D != 128) return LOMA_ERR_UNSUPPORTED;
    if (B == 0 || Hq == 0) return LOMA_OK;
    if (Hkv == 0 || Hq % Hkv) return LOMA_ERR_INVALID_ARG;
    if ((int64_t)B * Hq * 128 > INT_MAX) return LOMA_ERR_INVALID_ARG;
    if (max_mem > INT_MAX - 256 || max_tail > INT_MAX - 256) return LOMA_ERR_INVALID_ARG;
    return LOMA_OK;
}

size_t loma_decode_kv4_workspace_bytes(int B, int Hq, int Hkv, int D, int max_mem_len, int max_tail_len) {
    if (B <= 0 || Hq <= 0 || kv4_decode_sizes(B, Hq, Hkv, D, max_mem_len, max_tail_len) != LOMA_OK) return 0;
    return decode_kv4_workspace_bytes(B, Hq, Hkv, D, max_mem_len, max_tail_len);
}

int loma_decode_attn_kv4(const void* q, const void* k_new, const void* v_new, void* k_tail, void* v_tail, const void* kv_pool,
                         const int32_t* block_table, void* o, float* lse, int B, int Hq, int Hkv, int D, int cap, const int32_t* tail_lens,
                         int max_tail_len, int page_size, int max_pages, int n_pages, const int32_t* mem_lens, int max_mem_len,
                         loma_dtype dtype, float softmax_scale, unsigned flags, void* workspace, size_t workspace_bytes, void* stream) {
    const int sc = kv4_decode_sizes(B, Hq, Hkv, D, max_mem_len, max_tail_len);
    if (sc != LOMA_OK) return sc;
    int l2;
    const int rc = kv4_sizes(B, Hkv, D, page_size, max_pages, n_pages, dtype, &l2);
    if (rc != LOMA_OK) return rc;
    if (cap < 0 || !fits({B, Hkv, cap, D, 4}) || (k_new == nullptr) != (v_new == nullptr)) return LOMA_ERR_INVALID_ARG;
    if (softmax_scale > 0x1p50f || (softmax_scale > 0.f && softmax_scale < 0x1p-50f)) return LOMA_ERR_INVALID_ARG;   // sums carry powers of two
    if (max_tail_len >= cap || max_mem_len > (int64_t)max_pages * page_size) return LOMA_ERR_CAPACITY;
    if (B == 0 || Hq == 0) return LOMA_OK;
    if (!q || !k_tail || !v_tail || !o || !tail_lens || !mem_lens) return LOMA_ERR_INVALID_ARG;
    if (max_mem_len > 0 && (!kv_pool || !block_table || n_pages < 1)) return LOMA_ERR_INVALID_ARG;
    for (const void* p : {q, k_new, v_new, (const void*)k_tail, (const void*)v_tail, kv_pool, (const void*)o, (const void*)workspace})
        if (misaligned(p, 16)) return LOMA_ERR_ALIGNMENT;
    for (const void* p : {(const void*)block_table, (const void*)lse, (const void*)tail_lens, (const void*)mem_lens})
        if (misaligned(p, 4)) return LOMA_ERR_ALIGNMENT;
    const int64_t es = (int64_t)elt_bytes(dtype), rows = (int64_t)B * Hq * D * es, news = (int64_t)B * Hkv * D * es, tails = news * cap;
    const size_t need = loma_decode_kv4_workspace_bytes(B, Hq, Hkv, D, max_mem_len, max_tail_len);
    if (!apart({{q, rows}, {k_new, news}, {v_new, news}, {kv_pool, max_mem_len > 0 ? kv4_pool_bytes(Hkv, D, l2, n_pages) : 0},
                {block_table, max_mem_len > 0 ? 4ll * B * max_pages : 0}, {tail_lens, 4ll * B}, {mem_lens, 4ll * B}},
               {{k_tail, tails}, {v_tail, tails}, {o, rows}, {lse, 4ll * B * Hq}, {workspace, (int64_t)std::min(need, workspace_bytes)}}))
        return LOMA_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < need) return LOMA_ERR_WORKSPACE;
    const int dc = check_device();
    if (dc != LOMA_OK) return dc;
    Kv4DecodeArgs a;
    a.m = kv4_pool(const_cast<void*>(kv_pool), block_table, max_pages, l2, n_pages);
    a.q = q; a.k_new = k_new; a.v_new = v_new; a.k_tail = k_tail; a.v_tail = v_tail; a.o = o; a.lse = lse;
    a.mem_lens = mem_lens; a.tail_lens = tail_lens; a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.g = Hq / Hkv;
    a.max_mem = max_mem_len; a.max_tail = max_tail_len; a.cap = cap;
    a.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)D);
    a.ws = workspace;
    return from_cuda(launch_decode_kv4(a, D, dtype, (flags & LOMA_FLAG_FORCE_GENERIC) != 0, static_cast<cudaStream_t>(stream)));
}

// ------------------------------------------------------------------ pages
static int page_sizes(int B, int page_size, int max_pages, int n_pages, int n_free, int* l2) {
    if (B < 0 || max_pages < 0 || n_pages < 0 || n_free < 0) return LOMA_ERR_INVALID_ARG;
    // kernels go over rows, columns and pages in 32-bit steps of up to 9472 (rows: the warps of a full launch)
    constexpr int TOP = INT_MAX - 65536;
    if (B > TOP || max_pages > TOP || n_pages > TOP || n_free == INT_MAX || !fits({4, B, max_pages})) return LOMA_ERR_INVALID_ARG;
    *l2 = log2_exact(page_size);
    if (*l2 < 0 || page_size > 65536) return LOMA_ERR_INVALID_ARG;
    if ((int64_t)max_pages * page_size > INT_MAX) return LOMA_ERR_INVALID_ARG;
    return LOMA_OK;
}

static bool words_misaligned(std::initializer_list<const void*> all) {
    for (const void* p : all) if (misaligned(p, 4)) return true;
    return false;
}

int loma_paged_release(int B, int page_size, int max_pages, int n_pages, int n_free, const int32_t* keep_lens, const int32_t* held,
                       int32_t* block_table, int32_t* held_out, int32_t* refs, int32_t* free_pages, int32_t* taken, int32_t* counts,
                       int on_device, void* stream) {
    ReleaseArgs a;
    const int rc = page_sizes(B, page_size, max_pages, n_pages, n_free, &a.log2_ps);
    if (rc != LOMA_OK) return rc;
    if (!taken || !counts || (n_pages > 0 && !refs) || (n_free > 0 && !free_pages)) return LOMA_ERR_INVALID_ARG;
    if (B > 0 && (!keep_lens || !held || !held_out || (max_pages > 0 && !block_table))) return LOMA_ERR_INVALID_ARG;
    if (words_misaligned({keep_lens, held, block_table, held_out, refs, free_pages, taken, counts})) return LOMA_ERR_ALIGNMENT;
    const int64_t nb = 4ll * B;
    // held_out may be held, and then neither of them keep_lens
    if (!apart({{keep_lens, nb}, {held_out == held ? nullptr : held, nb}}, {{block_table, nb * max_pages}, {held_out, nb}, {refs, 4ll * n_pages},
                {free_pages, 4ll * n_free}, {taken, 4}, {counts, 16}})) return LOMA_ERR_INVALID_ARG;
    a.pl.n_pages = n_pages; a.pl.n_free = n_free; a.pl.refs = refs; a.pl.free_pages = free_pages; a.pl.taken = taken;
    a.B = B; a.max_pages = max_pages; a.keep_lens = keep_lens; a.held = held; a.block_table = block_table; a.held_out = held_out; a.counts = counts;
    if (!on_device) {
        host_paged_release(a);
        return LOMA_OK;
    }
    const int dc = check_device();
    if (dc != LOMA_OK) return dc;
    return from_cuda(launch_paged_release(a, static_cast<cudaStream_t>(stream)));
}

size_t loma_paged_fork_workspace_bytes(int B) { return B <= 0 ? 0 : 8 * (size_t)B; }

int loma_paged_fork(int B, int page_size, int max_pages, int n_pages, int n_free, int max_copies, const int32_t* parents, const int32_t* cache_lens,
                    const int32_t* fixed_lens, const int32_t* held, const int32_t* block_table, int32_t* table_out, int32_t* lens_out,
                    int32_t* held_out, int32_t* refs, int32_t* free_pages, int32_t* taken, int32_t* copy_src, int32_t* copy_dst, int32_t* counts,
                    void* workspace, size_t workspace_bytes, int on_device, void* stream) {
    ForkArgs a;
    const int rc = page_sizes(B, page_size, max_pages, n_pages, n_free, &a.log2_ps);
    if (rc != LOMA_OK) return rc;
    if (max_copies < 0 || !taken || !counts || (n_pages > 0 && !refs) || (n_free > 0 && !free_pages)) return LOMA_ERR_INVALID_ARG;
    if (max_copies > 0 && (!copy_src || !copy_dst)) return LOMA_ERR_INVALID_ARG;
    if (B > 0 && (!parents || !cache_lens || !lens_out || !held_out || (max_pages > 0 && (!block_table || !table_out)))) return LOMA_ERR_INVALID_ARG;
    if (words_misaligned({parents, cache_lens, fixed_lens, held, block_table, table_out, lens_out, held_out, refs, free_pages, taken, copy_src,
                          copy_dst, counts, workspace})) return LOMA_ERR_ALIGNMENT;
    const int64_t nb = 4ll * B, nc = 4ll * max_copies;
    if (!apart({{parents, nb}, {cache_lens, nb}, {fixed_lens, nb}, {held, nb}, {block_table, nb * max_pages}},
               {{table_out, nb * max_pages}, {lens_out, nb}, {held_out, nb}, {refs, 4ll * n_pages}, {free_pages, 4ll * n_free}, {taken, 4},
                {copy_src, nc}, {copy_dst, nc}, {counts, 16}, {workspace, 2 * nb}})) return LOMA_ERR_INVALID_ARG;
    if (B > 0 && (!workspace || workspace_bytes < loma_paged_fork_workspace_bytes(B))) return LOMA_ERR_WORKSPACE;
    a.pl.n_pages = n_pages; a.pl.n_free = n_free; a.pl.refs = refs; a.pl.free_pages = free_pages; a.pl.taken = taken;
    a.B = B; a.max_pages = max_pages; a.max_copies = max_copies; a.parents = parents; a.cache_lens = cache_lens; a.fixed_lens = fixed_lens;
    a.held = held; a.block_table = block_table; a.table_out = table_out; a.lens_out = lens_out; a.held_out = held_out;
    a.copy_src = copy_src; a.copy_dst = copy_dst; a.counts = counts; a.ws = static_cast<int32_t*>(workspace);
    if (!on_device) {
        host_paged_fork(a);
        return LOMA_OK;
    }
    const int dc = check_device();
    if (dc != LOMA_OK) return dc;
    return from_cuda(launch_paged_fork(a, static_cast<cudaStream_t>(stream)));
}

int loma_paged_compact(int B, int max_pages, int n_pages, int n_free, int max_copies, const int32_t* held, int32_t* block_table, int32_t* refs,
                       int32_t* free_pages, int32_t* taken, int32_t* page_map, int32_t* copy_src, int32_t* copy_dst, int32_t* counts,
                       int on_device, void* stream) {
    int l2;
    const int rc = page_sizes(B, 1, max_pages, n_pages, n_free, &l2);
    if (rc != LOMA_OK) return rc;
    if (max_copies < 0 || !taken || !counts || (n_pages > 0 && (!refs || !page_map)) || (n_free > 0 && !free_pages)) return LOMA_ERR_INVALID_ARG;
    if (max_copies > 0 && (!copy_src || !copy_dst)) return LOMA_ERR_INVALID_ARG;
    if (B > 0 && (!held || (max_pages > 0 && !block_table))) return LOMA_ERR_INVALID_ARG;
    if (words_misaligned({held, block_table, refs, free_pages, taken, page_map, copy_src, copy_dst, counts})) return LOMA_ERR_ALIGNMENT;
    const int64_t nb = 4ll * B, nc = 4ll * max_copies, np = 4ll * n_pages;
    if (!apart({{held, nb}}, {{block_table, nb * max_pages}, {refs, np}, {free_pages, 4ll * n_free}, {taken, 4}, {page_map, np}, {copy_src, nc},
                {copy_dst, nc}, {counts, 16}})) return LOMA_ERR_INVALID_ARG;
    CompactArgs a;
    a.pl.n_pages = n_pages; a.pl.n_free = n_free; a.pl.refs = refs; a.pl.free_pages = free_pages; a.pl.taken = taken;
    a.B = B; a.max_pages = max_pages; a.max_copies = max_copies; a.held = held; a.block_table = block_table; a.page_map = page_map;
    a.copy_src = copy_src; a.copy_dst = copy_dst; a.counts = counts;
    if (!on_device) {
        host_paged_compact(a);
        return LOMA_OK;
    }
    const int dc = check_device();
    if (dc != LOMA_OK) return dc;
    return from_cuda(launch_paged_compact(a, static_cast<cudaStream_t>(stream)));
}

int loma_paged_copy(int n_pools, void* const* pools, const int64_t* page_bytes, int n_pages, const int32_t* copy_src, const int32_t* copy_dst,
                    const int32_t* n_copies, int max_copies, void* stream) {
    if (n_pools < 0 || n_pages < 0 || max_copies < 0) return LOMA_ERR_INVALID_ARG;
    if (n_pools == 0 || n_pages == 0 || max_copies == 0) return LOMA_OK;
    if (!pools || !page_bytes || !copy_src || !copy_dst || !n_copies) return LOMA_ERR_INVALID_ARG;
    if (words_misaligned({copy_src, copy_dst, n_copies})) return LOMA_ERR_ALIGNMENT;
    for (int k = 0; k < n_pools; ++k) {
        if (!pools[k] || page_bytes[k] < 0 || page_bytes[k] > INT64_MAX / 4 / n_pages) return LOMA_ERR_INVALID_ARG;
        if (misaligned(pools[k], 16) || page_bytes[k] % 16) return LOMA_ERR_ALIGNMENT;
        for (const int32_t* p : {copy_src, copy_dst}) if (overlap(p, 4ll * max_copies, pools[k], page_bytes[k] * n_pages)) return LOMA_ERR_INVALID_ARG;
        if (overlap(n_copies, 4, pools[k], page_bytes[k] * n_pages)) return LOMA_ERR_INVALID_ARG;
    }
    const int dc = check_device();
    if (dc != LOMA_OK) return dc;
    for (int k0 = 0; k0 < n_pools; k0 += COPY_POOLS) {
        CopyArgs a;
        a.n_pools = std::min(COPY_POOLS, n_pools - k0);
        a.n_pages = n_pages; a.max_copies = max_copies; a.src = copy_src; a.dst = copy_dst; a.n = n_copies;
        for (int k = 0; k < a.n_pools; ++k) {
            a.pool[k] = static_cast<uint8_t*>(pools[k0 + k]);
            a.bytes[k] = page_bytes[k0 + k];
        }
        const cudaError_t e = launch_paged_copy(a, static_cast<cudaStream_t>(stream));
        if (e != cudaSuccess) return from_cuda(e);
    }
    return LOMA_OK;
}

}  // extern "C"
