// extern "C" boundary of the serving-step operators (page tables, per-head norm with rotation, shared-prefix decode):
// argument validation and kernel selection.  Every check happens on the host before anything is enqueued.
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <mutex>

#include "decode_shared.cuh"

namespace loma {

cudaError_t prepare_kernel(const void* kernel, int smem) {
    static std::mutex mu;
    static struct { const void* kernel; uint64_t devices; } done[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    std::lock_guard<std::mutex> lock(mu);
    int i = 0;
    while (i < 64 && done[i].kernel && done[i].kernel != kernel) ++i;
    if (i < 64 && dev < 64 && done[i].kernel == kernel && (done[i].devices >> dev & 1)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
    if (e == cudaSuccess && smem > 0) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess && i < 64 && dev < 64) {
        done[i].kernel = kernel;
        done[i].devices |= 1ull << dev;
    }
    return e;
}

}  // namespace loma

using namespace loma;

static inline bool misaligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; }
static inline size_t elt_bytes(loma_dtype dt) { return dt == LOMA_F32 ? 4 : 2; }
static inline int from_cuda(cudaError_t e) { return e == cudaSuccess ? LOMA_OK : LOMA_ERR_CUDA; }

// do [a, a + na) and [b, b + nb) bytes meet?
static inline bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
    if (!a || !b || na <= 0 || nb <= 0) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

// n strided axes over rows of D elements: false if two rows may share an element (a stride of 0 included)
static bool rows_apart(int n, const int64_t* extent, const int64_t* stride, int D) {
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

extern "C" {

// ------------------------------------------------------------------ page tables
int loma_paged_extend(int B, int page_size, int max_pages, int max_rows, int n_free, const int32_t* cache_lens, const int32_t* new_lens,
                      const int32_t* held, const int32_t* pos0, const int32_t* free_pages, int32_t* taken, int32_t* block_table,
                      int32_t* row_start, int32_t* page_start, int32_t* held_out, int32_t* slots, int32_t* row_seq, int32_t* row_pos,
                      int on_device, void* stream) {
    if (B < 0 || max_pages < 0 || max_rows < 0 || n_free < 0) return LOMA_ERR_INVALID_ARG;
    const int l2 = log2_exact(page_size);
    if (l2 < 0 || page_size > 65536) return LOMA_ERR_INVALID_ARG;
    if ((int64_t)max_pages * page_size > INT_MAX) return LOMA_ERR_INVALID_ARG;
    if (B == INT_MAX || max_rows > INT_MAX - 4096) return LOMA_ERR_INVALID_ARG;
    if (!row_start || !page_start) return LOMA_ERR_INVALID_ARG;
    if (B > 0 && (!cache_lens || !held_out || (max_pages > 0 && !block_table))) return LOMA_ERR_INVALID_ARG;
    if (max_rows > 0 && (!slots || !row_seq || !row_pos)) return LOMA_ERR_INVALID_ARG;
    if (n_free > 0 && !free_pages) return LOMA_ERR_INVALID_ARG;
    const void* all[] = {cache_lens, new_lens, held, pos0, free_pages, taken, block_table, row_start, page_start, held_out, slots, row_seq, row_pos};
    for (const void* p : all) if (misaligned(p, 4)) return LOMA_ERR_ALIGNMENT;
    // no output may meet an input or another output; held and held_out may be one array
    const int64_t nb = 4ll * B, nr = 4ll * max_rows;
    const struct { const void* p; int64_t n; } ins[] = {{cache_lens, nb}, {new_lens, nb}, {held, nb}, {pos0, nb}, {free_pages, 4ll * n_free}};
    const struct { const void* p; int64_t n; } outs[] = {{taken, 4}, {block_table, nb * max_pages}, {row_start, nb + 4}, {page_start, nb + 4},
                                                         {held_out, nb}, {slots, nr}, {row_seq, nr}, {row_pos, nr}};
    for (int i = 0; i < 8; ++i) {
        for (const auto& x : ins)
            if (overlap(outs[i].p, outs[i].n, x.p, x.n) && !(outs[i].p == held_out && x.p == held && held == held_out)) return LOMA_ERR_INVALID_ARG;
        for (int k = 0; k < i; ++k)
            if (overlap(outs[i].p, outs[i].n, outs[k].p, outs[k].n)) return LOMA_ERR_INVALID_ARG;
    }
    const ExtendArgs a{B, l2, max_pages, max_rows, n_free, cache_lens, new_lens, held, pos0, free_pages, taken, block_table,
                       row_start, page_start, held_out, slots, row_seq, row_pos};
    if (!on_device) {
        host_paged_extend(a);
        return LOMA_OK;
    }
    const int dc = check_device();
    if (dc != LOMA_OK) return dc;
    return from_cuda(launch_paged_extend(a, static_cast<cudaStream_t>(stream)));
}

// ------------------------------------------------------------------ norm + rotation
static int norm_args(int B, int Hq, int Hk, int D, int n_chunks, int c, int t, int tc, int tail_read, const int64_t* q_strides,
                     const int64_t* k_strides, loma_dtype dtype, int position_type, unsigned flags, Layout* L, HeadsView* q, HeadsView* k) {
    if (B < 0 || Hq < 0 || Hk < 0) return LOMA_ERR_INVALID_ARG;
    if (dtype != LOMA_F32 && dtype != LOMA_BF16) return LOMA_ERR_UNSUPPORTED;
    if (D != 64 && D != 128) return LOMA_ERR_UNSUPPORTED;
    if (position_type < 0 || position_type > 1) return LOMA_ERR_INVALID_ARG;
    const int rc = make_layout(n_chunks, c, t, tail_read, flags, L);
    if (rc != LOMA_OK) return rc;
    if (tc != L->tc) return LOMA_ERR_INVALID_ARG;
    if ((int64_t)B * Hq > 65535 || (int64_t)B * Hk > 65535) return LOMA_ERR_INVALID_ARG;
    HeadsView* v[2] = {q, k};
    const int64_t* st[2] = {q_strides, k_strides};
    for (int i = 0; i < 2; ++i) {
        v[i]->H = i == 0 ? Hq : Hk;
        if (v[i]->H == 0 || B == 0 || L->S == 0) continue;
        if (!st[i]) return LOMA_ERR_INVALID_ARG;
        const int64_t extent[3] = {B, v[i]->H, L->S};
        for (int x = 0; x < 3; ++x) if (st[i][x] < 0) return LOMA_ERR_INVALID_ARG;
        if (!rows_apart(3, extent, st[i], D)) return LOMA_ERR_INVALID_ARG;
        for (int x = 0; x < 3; ++x)
            if (extent[x] > 1 && (st[i][x] * (int64_t)elt_bytes(dtype)) % 16) return LOMA_ERR_ALIGNMENT;
        v[i]->sb = st[i][0]; v[i]->sh = st[i][1]; v[i]->ss = st[i][2];
    }
    return LOMA_OK;
}

int loma_qk_norm_rope_fwd(const void* q, const void* k, const void* wq, const void* wk, void* q_out, void* k_out, int B, int Hq, int Hk,
                          int D, int n_chunks, int c, int t, int tc, int tail_read, const int64_t* q_strides, const int64_t* k_strides,
                          loma_dtype dtype, float eps, float theta_base, int position_type, unsigned flags, void* stream) {
    Layout L;
    HeadsView vq, vk;
    const int rc = norm_args(B, Hq, Hk, D, n_chunks, c, t, tc, tail_read, q_strides, k_strides, dtype, position_type, flags, &L, &vq, &vk);
    if (rc != LOMA_OK) return rc;
    if (L.S == 0 || B == 0 || Hq + Hk == 0) return LOMA_OK;
    if ((Hq > 0 && (!q || !q_out)) || (Hk > 0 && (!k || !k_out))) return LOMA_ERR_INVALID_ARG;
    if (Hq > 0 && Hk > 0 && (q_out == k_out || q_out == k || k_out == q)) return LOMA_ERR_INVALID_ARG;
    const void* all[] = {q, k, wq, wk, q_out, k_out};
    for (const void* p : all) if (misaligned(p, 16)) return LOMA_ERR_ALIGNMENT;
    const int dc = check_device();
    if (dc != LOMA_OK) return dc;
    vq.in = q; vq.out = q_out; vq.w = wq;
    vk.in = k; vk.out = k_out; vk.w = wk;
    return from_cuda(launch_qk_norm_rope(vq, vk, B, D, L, dtype, eps > 0.f ? eps : 1e-6f, theta_base > 0.f ? (double)theta_base : 10000.0,
                                         position_type, false, nullptr, static_cast<cudaStream_t>(stream)));
}

size_t loma_qk_norm_rope_bwd_workspace_bytes(int B, int Hq, int Hk, int D, int n_chunks, int c, int t, int tail_read, unsigned flags) {
    Layout L;
    if (B < 0 || Hq < 0 || Hk < 0 || (D != 64 && D != 128) || (int64_t)B * Hq > 65535 || (int64_t)B * Hk > 65535) return 0;
    if (make_layout(n_chunks, c, t, tail_read, flags, &L) != LOMA_OK || L.S == 0 || B == 0 || Hq + Hk == 0) return 0;
    return (qk_norm_rope_bwd_workspace_bytes(B, Hq, Hk, D, L) + 255) & ~(size_t)255;
}

int loma_qk_norm_rope_bwd(const void* q, const void* k, const void* wq, const void* wk, const void* d_q_out, const void* d_k_out, void* dq,
                          void* dk, void* dwq, void* dwk, int B, int Hq, int Hk, int D, int n_chunks, int c, int t, int tc, int tail_read,
                          const int64_t* q_strides, const int64_t* k_strides, loma_dtype dtype, float eps, float theta_base,
                          int position_type, unsigned flags, void* workspace, size_t workspace_bytes, void* stream) {
    Layout L;
    HeadsView vq, vk;
    const int rc = norm_args(B, Hq, Hk, D, n_chunks, c, t, tc, tail_read, q_strides, k_strides, dtype, position_type, flags, &L, &vq, &vk);
    if (rc != LOMA_OK) return rc;
    const bool empty = L.S == 0 || B == 0 || Hq + Hk == 0;
    const void* ins[] = {q, k, wq, wk, d_q_out, d_k_out};
    void* outs[] = {dq, dk, dwq, dwk};
    for (const void* p : ins) if (misaligned(p, 16)) return LOMA_ERR_ALIGNMENT;
    for (void* p : outs) if (misaligned(p, 16)) return LOMA_ERR_ALIGNMENT;
    if (dwq && dwq == dwk) return LOMA_ERR_INVALID_ARG;
    if (!empty) {
        if ((Hq > 0 && (!q || !d_q_out || !dq)) || (Hk > 0 && (!k || !d_k_out || !dk))) return LOMA_ERR_INVALID_ARG;
        for (int x = 0; x < 4; ++x) {
            if (!outs[x]) continue;
            for (const void* p : ins) if (outs[x] == p) return LOMA_ERR_INVALID_ARG;
            for (int y = 0; y < x; ++y) if (outs[x] == outs[y]) return LOMA_ERR_INVALID_ARG;
        }
        const size_t need = loma_qk_norm_rope_bwd_workspace_bytes(B, Hq, Hk, D, n_chunks, c, t, tail_read, flags);
        if (!workspace || workspace_bytes < need) return LOMA_ERR_WORKSPACE;
        if (misaligned(workspace, 256)) return LOMA_ERR_ALIGNMENT;
    }
    if (empty && !dwq && !dwk) return LOMA_OK;
    const int dc = check_device();
    if (dc != LOMA_OK) return dc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (empty) {   // no rows: the gains' gradients are zero
        for (void* p : {dwq, dwk})
            if (p && cudaMemsetAsync(p, 0, D * elt_bytes(dtype), st) != cudaSuccess) return LOMA_ERR_CUDA;
        return LOMA_OK;
    }
    vq.in = q; vq.grad = d_q_out; vq.out = dq; vq.w = wq; vq.dw = dwq;
    vk.in = k; vk.grad = d_k_out; vk.out = dk; vk.w = wk; vk.dw = dwk;
    return from_cuda(launch_qk_norm_rope(vq, vk, B, D, L, dtype, eps > 0.f ? eps : 1e-6f, theta_base > 0.f ? (double)theta_base : 10000.0,
                                         position_type, true, workspace, st));
}

int loma_qk_norm_rope_append(const void* q, const void* k_new, const void* v_new, const void* wq, const void* wk, void* q_out, void* k_pool,
                             void* v_pool, const int32_t* slots, const int32_t* positions, int T, int Hq, int Hk, int D, int page_size,
                             int n_pages, const int64_t* q_strides, const int64_t* k_strides, const int64_t* v_strides, loma_dtype dtype,
                             float eps, float theta_base, void* stream) {
    if (T < 0 || Hq < 0 || Hk < 0 || page_size < 1 || n_pages < 0) return LOMA_ERR_INVALID_ARG;
    if (dtype != LOMA_F32 && dtype != LOMA_BF16) return LOMA_ERR_UNSUPPORTED;
    if (D != 64 && D != 128) return LOMA_ERR_UNSUPPORTED;
    if (Hq > 65535 || Hk > 65535) return LOMA_ERR_INVALID_ARG;
    if (T == 0 || Hq + Hk == 0) return LOMA_OK;
    if (!slots || !positions) return LOMA_ERR_INVALID_ARG;
    if (Hq > 0 && (!q || !q_out)) return LOMA_ERR_INVALID_ARG;
    if (Hk > 0 && (!k_new || !v_new || !k_pool || !v_pool || k_pool == v_pool || n_pages < 1)) return LOMA_ERR_INVALID_ARG;
    if (Hq > 0 && (q_out == k_new || q_out == v_new || q_out == k_pool || q_out == v_pool)) return LOMA_ERR_INVALID_ARG;
    const int64_t* st[3] = {q_strides, k_strides, v_strides};
    const void* in[3] = {q, k_new, v_new};
    for (int i = 0; i < 3; ++i) {
        const int H = i == 0 ? Hq : Hk;
        if (H == 0) continue;
        if (!st[i]) return LOMA_ERR_INVALID_ARG;
        const int64_t extent[2] = {T, H};
        if (st[i][0] < 0 || st[i][1] < 0 || !rows_apart(2, extent, st[i], D)) return LOMA_ERR_INVALID_ARG;
        for (int x = 0; x < 2; ++x)
            if (extent[x] > 1 && (st[i][x] * (int64_t)elt_bytes(dtype)) % 16) return LOMA_ERR_ALIGNMENT;
        // q_out is contiguous: in place only where q is contiguous too
        if (i == 0 && q_out == q && ((T > 1 && st[0][0] != (int64_t)Hq * D) || (Hq > 1 && st[0][1] != D))) return LOMA_ERR_INVALID_ARG;
        if (misaligned(in[i], 16)) return LOMA_ERR_ALIGNMENT;
    }
    const void* rest[] = {wq, wk, q_out, k_pool, v_pool};
    for (const void* p : rest) if (misaligned(p, 16)) return LOMA_ERR_ALIGNMENT;
    if (misaligned(slots, 4) || misaligned(positions, 4)) return LOMA_ERR_ALIGNMENT;
    const int dc = check_device();
    if (dc != LOMA_OK) return dc;
    AppendArgs a;
    a.q = q; a.k = k_new; a.v = v_new; a.wq = wq; a.wk = wk; a.q_out = q_out; a.k_pool = k_pool; a.v_pool = v_pool;
    a.slots = slots; a.positions = positions; a.T = T; a.Hq = Hq; a.Hk = Hk; a.page_size = page_size; a.n_pages = n_pages;
    if (Hq > 0) { a.q_row = q_strides[0]; a.q_head = q_strides[1]; }
    if (Hk > 0) { a.k_row = k_strides[0]; a.k_head = k_strides[1]; a.v_row = v_strides[0]; a.v_head = v_strides[1]; }
    a.eps = eps > 0.f ? eps : 1e-6f;
    a.log2_base = log2(theta_base > 0.f ? (double)theta_base : 10000.0);
    return from_cuda(launch_qk_norm_rope_append(a, D, dtype, static_cast<cudaStream_t>(stream)));
}

// ------------------------------------------------------------------ shared-prefix decode
static int shared_sizes(int B, int Hq, int Hkv, int D, int prefix_len, int max_len) {
    if (B < 0 || Hq < 0 || Hkv < 0 || prefix_len < 0 || max_len < 0) return LOMA_ERR_INVALID_ARG;
    if (D != 64 && D != 128) return LOMA_ERR_UNSUPPORTED;
    if (B == 0 || Hq == 0) return LOMA_OK;
    if (Hkv == 0 || Hq % Hkv) return LOMA_ERR_INVALID_ARG;
    if ((int64_t)B * Hq * 128 > INT_MAX || Hkv > 65535) return LOMA_ERR_INVALID_ARG;
    if (prefix_len > INT_MAX - 256 || max_len > INT_MAX - 256) return LOMA_ERR_INVALID_ARG;
    return LOMA_OK;
}

size_t loma_decode_shared_workspace_bytes(int B, int Hq, int Hkv, int D, int prefix_len, int max_cache_len) {
    if (B <= 0 || Hq <= 0 || shared_sizes(B, Hq, Hkv, D, prefix_len, max_cache_len) != LOMA_OK) return 0;
    return decode_shared_workspace_bytes(B, Hq, Hkv, D, prefix_len, max_cache_len);
}

static int shared_impl(SharedArgs& a, int D, loma_dtype dtype, float softmax_scale, unsigned flags, void* workspace, size_t workspace_bytes,
                       void* stream) {
    const void* vec[] = {a.q, a.k_new, a.v_new, a.k_prefix, a.v_prefix, a.k_cache, a.v_cache, a.o, workspace};
    for (const void* p : vec) if (misaligned(p, 16)) return LOMA_ERR_ALIGNMENT;
    const void* words[] = {a.lse, a.cache_lens, a.prefix_table, a.pg.table};
    for (const void* p : words) if (misaligned(p, 4)) return LOMA_ERR_ALIGNMENT;
    const size_t need = loma_decode_shared_workspace_bytes(a.B, a.Hq, a.Hkv, D, a.prefix_len, a.max_len);
    if (!workspace || workspace_bytes < need) return LOMA_ERR_WORKSPACE;
    const int dc = check_device();
    if (dc != LOMA_OK) return dc;
    a.g = a.Hq / a.Hkv;
    a.scale = softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)D);
    a.ws = workspace;
    return from_cuda(launch_decode_shared(a, D, dtype, (flags & LOMA_FLAG_FORCE_GENERIC) != 0, static_cast<cudaStream_t>(stream)));
}

int loma_decode_attn_shared(const void* q, const void* k_new, const void* v_new, const void* k_prefix, const void* v_prefix, void* k_cache,
                            void* v_cache, void* o, float* lse, int B, int Hq, int Hkv, int D, int prefix_cap, int prefix_len, int cap,
                            const int32_t* cache_lens, int max_cache_len, loma_dtype dtype, float softmax_scale, unsigned flags,
                            void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = shared_sizes(B, Hq, Hkv, D, prefix_len, max_cache_len);
    if (rc != LOMA_OK) return rc;
    if (prefix_cap < 0 || cap < 0) return LOMA_ERR_INVALID_ARG;
    if (dtype != LOMA_F32 && dtype != LOMA_BF16) return LOMA_ERR_UNSUPPORTED;
    if ((k_new == nullptr) != (v_new == nullptr)) return LOMA_ERR_INVALID_ARG;
    if (prefix_len > prefix_cap || max_cache_len >= cap) return LOMA_ERR_CAPACITY;
    if (B == 0 || Hq == 0) return LOMA_OK;
    if (!q || !k_cache || !v_cache || !o || !cache_lens || (prefix_len > 0 && (!k_prefix || !v_prefix))) return LOMA_ERR_INVALID_ARG;
    SharedArgs a;
    a.q = q; a.k_new = k_new; a.v_new = v_new; a.k_prefix = k_prefix; a.v_prefix = v_prefix; a.k_cache = k_cache; a.v_cache = v_cache;
    a.o = o; a.lse = lse; a.cache_lens = cache_lens;
    a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.prefix_len = prefix_len; a.prefix_cap = prefix_cap; a.cap = cap; a.max_len = max_cache_len;
    return shared_impl(a, D, dtype, softmax_scale, flags, workspace, workspace_bytes, stream);
}

int loma_decode_attn_shared_paged(const void* q, const void* k_new, const void* v_new, void* k_pool, void* v_pool, const int32_t* prefix_table,
                                  const int32_t* block_table, void* o, float* lse, int B, int Hq, int Hkv, int D, int page_size,
                                  int prefix_pages, int prefix_len, int max_pages, int n_pages, const int32_t* cache_lens, int max_cache_len,
                                  loma_dtype dtype, float softmax_scale, unsigned flags, void* workspace, size_t workspace_bytes,
                                  void* stream) {
    const int rc = shared_sizes(B, Hq, Hkv, D, prefix_len, max_cache_len);
    if (rc != LOMA_OK) return rc;
    if (prefix_pages < 0 || max_pages < 0 || n_pages < 0) return LOMA_ERR_INVALID_ARG;
    if (dtype != LOMA_F32 && dtype != LOMA_BF16) return LOMA_ERR_UNSUPPORTED;
    const int l2 = log2_exact(page_size);
    if (l2 < 0 || page_size > 65536) return LOMA_ERR_INVALID_ARG;
    if ((k_new == nullptr) != (v_new == nullptr)) return LOMA_ERR_INVALID_ARG;
    if (prefix_len > (int64_t)prefix_pages * page_size || max_cache_len >= (int64_t)max_pages * page_size) return LOMA_ERR_CAPACITY;
    if ((int64_t)max_pages * page_size > INT_MAX) return LOMA_ERR_INVALID_ARG;
    if (B == 0 || Hq == 0) return LOMA_OK;
    if (!q || !k_pool || !v_pool || !o || !cache_lens || !block_table || n_pages < 1 || (prefix_len > 0 && !prefix_table))
        return LOMA_ERR_INVALID_ARG;
    SharedArgs a;
    a.q = q; a.k_new = k_new; a.v_new = v_new; a.k_prefix = k_pool; a.v_prefix = v_pool; a.k_cache = k_pool; a.v_cache = v_pool;
    a.o = o; a.lse = lse; a.cache_lens = cache_lens; a.prefix_table = prefix_table;
    a.pg.table = block_table; a.pg.max_pages = max_pages; a.pg.log2_ps = l2; a.pg.n_pages = n_pages;
    a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.prefix_len = prefix_len; a.max_len = max_cache_len;
    return shared_impl(a, D, dtype, softmax_scale, flags, workspace, workspace_bytes, stream);
}

}  // extern "C"
