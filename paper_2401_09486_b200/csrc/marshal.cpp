// Argument marshalling for the entry points of libloma whose calls take less time than checking a dozen tensors in Python
// does (a call of loma_paged_extend for 64 sequences: 13.5 us of host time from Python, 5 us on the GPU).  A CPython
// extension module: each function takes the tensors and numbers of the function of the same name in binding.py by position,
// checks shapes, types and devices, and calls the C entry point; it returns the entry point's status.  No arithmetic of the
// method happens here.  The entry points' addresses come from the loaded library (bind), so nothing is linked twice.
#include <Python.h>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <stdexcept>
#include <string>

#include "loma.h"

namespace {

decltype(&loma_paged_extend) p_extend;
decltype(&loma_qk_norm_rope_fwd) p_norm_fwd;
decltype(&loma_qk_norm_rope_bwd) p_norm_bwd;
decltype(&loma_qk_norm_rope_append) p_append;
decltype(&loma_decode_attn_shared) p_shared;
decltype(&loma_decode_attn_shared_paged) p_shared_paged;

struct Refused : std::runtime_error {   // becomes a ValueError
    using std::runtime_error::runtime_error;
};
struct PyFailed {};                     // a Python error is set

// The arguments of one call, taken one after the other.
struct Args {
    const char* where;
    PyObject* const* v;
    Py_ssize_t n, at = 0;
    int dev = -1;

    Args(const char* w, PyObject* const* args, Py_ssize_t count, Py_ssize_t want) : where(w), v(args), n(count) {
        if (count != want) no("wrong number of arguments");
    }
    [[noreturn]] void no(const std::string& what) const { throw Refused(std::string(where) + ": " + what); }

    const at::Tensor* tensor(const char* name, bool optional = false) {
        PyObject* o = v[at++];
        if (o == Py_None) {
            if (!optional) no(std::string(name) + " is missing");
            return nullptr;
        }
        if (!THPVariable_Check(o)) no(std::string(name) + " must be a tensor");
        return &THPVariable_Unpack(o);
    }
    long integer() {
        const long x = PyLong_AsLong(v[at++]);
        if (x == -1 && PyErr_Occurred()) throw PyFailed();
        return x;
    }
    int i32() {
        const long x = integer();
        if (x < INT32_MIN || x > INT32_MAX) no("a number does not fit 32 bits");
        return (int)x;
    }
    float number() {
        const double x = PyFloat_AsDouble(v[at++]);
        if (x == -1.0 && PyErr_Occurred()) throw PyFailed();
        return (float)x;
    }
    // None: the current stream of the call's device; a torch stream or a raw handle otherwise
    void* stream() {
        PyObject* o = v[at++];
        if (dev < 0) return nullptr;
        if (o == Py_None) return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
        PyObject* h = nullptr;
        if (!PyLong_Check(o) && !(h = PyObject_GetAttrString(o, "cuda_stream"))) throw PyFailed();
        void* p = PyLong_AsVoidPtr(h ? h : o);
        Py_XDECREF(h);
        if (!p && PyErr_Occurred()) throw PyFailed();
        return p;
    }
    // a pointer of another device than the current one would reach the wrong GPU's kernel
    void device_of(const at::Tensor& t, bool host_too = false) {
        dev = t.is_cuda() ? (int)t.get_device() : -1;
        if (dev < 0) {
            if (host_too && t.is_cpu()) return;
            no("tensors must be on a CUDA device");
        }
        const int cur = (int)c10::cuda::current_device();
        if (cur != dev) no("tensors on cuda:" + std::to_string(dev) + ", but the current device is cuda:" + std::to_string(cur));
    }
    void here(const char* name, const at::Tensor& t) const {
        if ((t.is_cuda() ? (int)t.get_device() : -1) != dev || (dev < 0 && !t.is_cpu())) no(std::string(name) + " is on another device than the call's other tensors");
    }
    // contiguous int32 with `numel` entries (any number if negative)
    int32_t* words(const char* name, const at::Tensor* t, int64_t numel) const {
        if (!t) return nullptr;
        here(name, *t);
        if (t->scalar_type() != at::kInt || !t->is_contiguous() || (numel >= 0 && t->numel() != numel))
            no(std::string(name) + " must be a contiguous int32 tensor" + (numel >= 0 ? " with " + std::to_string(numel) + " entries" : ""));
        return static_cast<int32_t*>(t->data_ptr());
    }
    void* dense(const char* name, const at::Tensor* t, at::IntArrayRef shape, at::ScalarType type) const {
        if (!t) return nullptr;
        here(name, *t);
        if (t->scalar_type() != type || t->sizes() != shape || !t->is_contiguous()) {
            std::string s = std::string(name) + " must be a contiguous " + c10::toString(type) + " tensor of shape (";
            for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
            no(s + ")");
        }
        return t->data_ptr();
    }
    void* scratch(const at::Tensor* t, size_t* bytes) const {
        *bytes = 0;
        if (!t) return nullptr;
        here("workspace", *t);
        if (!t->is_contiguous()) no("workspace must be contiguous");
        *bytes = t->nbytes();
        return t->data_ptr();
    }
    loma_dtype dtype(const at::Tensor& t) const {
        if (t.scalar_type() == at::kFloat) return LOMA_F32;
        if (t.scalar_type() == at::kBFloat16) return LOMA_BF16;
        no(std::string("unsupported dtype ") + c10::toString(t.scalar_type()));
    }
};

// an axis of one element has no stride of its own (torch reports any number there)
void strides_of(const at::Tensor& t, int axes, int64_t* out) {
    for (int i = 0; i < axes; ++i) out[i] = t.size(i) > 1 ? t.stride(i) : 0;
}

// The entry point runs without the interpreter lock; C++ exceptions end here.
template <typename F>
PyObject* guarded(F&& body) {
    try {
        return PyLong_FromLong(body());
    } catch (const Refused& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const PyFailed&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}
template <typename F>
int unlocked(F&& call) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return rc;
}

PyObject* paged_extend(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return guarded([&] {
        Args a("loma_paged_extend", args, n, 15);
        const at::Tensor &lens = *a.tensor("cache_lens"), *fresh = a.tensor("new_lens", true), *held = a.tensor("held", true),
                         *pos0 = a.tensor("pos0", true), *free_pages = a.tensor("free_pages", true), *taken = a.tensor("taken", true),
                         &table = *a.tensor("block_table");
        const int page_size = a.i32();
        const at::Tensor &row_start = *a.tensor("row_start"), &page_start = *a.tensor("page_start"), &held_out = *a.tensor("held_out"),
                         &slots = *a.tensor("slots"), &row_seq = *a.tensor("row_seq"), &row_pos = *a.tensor("row_pos");
        a.device_of(lens, true);
        void* stream = a.stream();
        const int64_t B = lens.numel(), rows = slots.numel(), n_free = free_pages ? free_pages->numel() : 0;
        if (table.dim() != 2 || table.size(0) != B) a.no("block_table must be [B, max_pages]");
        if (B >= INT32_MAX || rows > INT32_MAX || n_free > INT32_MAX || table.size(1) > INT32_MAX) a.no("too many entries");
        int32_t *p0 = a.words("cache_lens", &lens, B), *p1 = a.words("new_lens", fresh, B), *p2 = a.words("held", held, B),
                *p3 = a.words("pos0", pos0, B), *p4 = a.words("free_pages", free_pages, -1), *p5 = a.words("taken", taken, 1),
                *p6 = a.words("block_table", &table, -1), *p7 = a.words("row_start", &row_start, B + 1),
                *p8 = a.words("page_start", &page_start, B + 1), *p9 = a.words("held_out", &held_out, B),
                *p10 = a.words("slots", &slots, rows), *p11 = a.words("row_seq", &row_seq, rows), *p12 = a.words("row_pos", &row_pos, rows);
        return unlocked([&] {
            return p_extend((int)B, page_size, (int)table.size(1), (int)rows, (int)n_free, p0, p1, p2, p3, p4, p5, p6, p7, p8, p9, p10, p11, p12,
                            a.dev >= 0, stream);
        });
    });
}

// What forward and backward of the training-layout norm share.
struct NormCall {
    int B, Hq, Hk, S, D;
    loma_dtype dt;
    int64_t qs[3], ks[3];

    NormCall(Args& a, const at::Tensor& q, const at::Tensor& k) {
        if (q.dim() != 4 || k.dim() != 4 || q.size(0) != k.size(0) || q.size(2) != k.size(2) || q.size(3) != k.size(3) || q.scalar_type() != k.scalar_type())
            a.no("q [B, Hq, S, D] and k [B, Hk, S, D] must share B, S, D and dtype");
        for (int i = 0; i < 4; ++i)
            if (q.size(i) > INT32_MAX || k.size(i) > INT32_MAX) a.no("tensors too large");
        B = (int)q.size(0); Hq = (int)q.size(1); Hk = (int)k.size(1); S = (int)q.size(2); D = (int)q.size(3);
        dt = a.dtype(q);
        if (q.stride(3) != 1 || k.stride(3) != 1) a.no("head dimension must be contiguous");
        strides_of(q, 3, qs);
        strides_of(k, 3, ks);
    }
    // x goes with ref: same shape, strides, dtype and device
    void* with(const Args& a, const char* name, const at::Tensor& ref, const at::Tensor& x) const {
        a.here(name, x);
        bool same = x.scalar_type() == ref.scalar_type() && x.sizes() == ref.sizes();
        for (int i = 0; same && i < 4; ++i) same = x.size(i) <= 1 || x.stride(i) == ref.stride(i);
        if (!same) a.no(std::string(name) + " must have the shape, strides and dtype of the tensor it belongs to");
        return x.data_ptr();
    }
    void rows(const Args& a, int n, int c, int t, int tail, unsigned flags) const {
        if ((int64_t)c * t > INT32_MAX || c > (1 << 30) || c < 0 || t < 0) a.no("c and t out of range");
        const int64_t chunk = (int64_t)t * ((flags & LOMA_FLAG_NO_REP_ZONE) ? c + 1 : 2 * (int64_t)c + 1), want = chunk * n + tail;
        if (want != S) a.no("the layout has " + std::to_string(want) + " rows, the tensors " + std::to_string(S));
    }
};

PyObject* qk_norm_rope_fwd(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    return guarded([&] {
        Args a("loma_qk_norm_rope_fwd", args, n_args, 15);
        const at::Tensor &q = *a.tensor("q"), &k = *a.tensor("k"), *wq = a.tensor("wq", true), *wk = a.tensor("wk", true), &qo = *a.tensor("q_out"),
                         &ko = *a.tensor("k_out");
        const int n = a.i32(), c = a.i32(), t = a.i32(), tail = a.i32();
        const unsigned flags = (unsigned)a.integer();
        const float eps = a.number(), theta = a.number();
        const int ptype = a.i32();
        const NormCall f(a, q, k);
        void *pqo, *pko;
        a.dev = q.is_cuda() ? (int)q.get_device() : -1;
        pqo = f.with(a, "q_out", q, qo);
        pko = f.with(a, "k_out", k, ko);
        a.here("k", k);
        void *pwq = a.dense("wq", wq, {f.D}, q.scalar_type()), *pwk = a.dense("wk", wk, {f.D}, q.scalar_type());
        f.rows(a, n, c, t, tail, flags);
        a.device_of(q);
        void* stream = a.stream();
        return unlocked([&] {
            return p_norm_fwd(q.data_ptr(), k.data_ptr(), pwq, pwk, pqo, pko, f.B, f.Hq, f.Hk, f.D, n, c, t, c * t, tail, f.qs, f.ks, f.dt, eps, theta,
                              ptype, flags, stream);
        });
    });
}

PyObject* qk_norm_rope_bwd(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    return guarded([&] {
        Args a("loma_qk_norm_rope_bwd", args, n_args, 20);
        const at::Tensor &q = *a.tensor("q"), &k = *a.tensor("k"), *wq = a.tensor("wq", true), *wk = a.tensor("wk", true), &gq = *a.tensor("d_q_out"),
                         &gk = *a.tensor("d_k_out"), &dq = *a.tensor("dq"), &dk = *a.tensor("dk"), *dwq = a.tensor("dwq", true),
                         *dwk = a.tensor("dwk", true);
        const int n = a.i32(), c = a.i32(), t = a.i32(), tail = a.i32();
        const unsigned flags = (unsigned)a.integer();
        const at::Tensor* ws = a.tensor("workspace", true);
        const float eps = a.number(), theta = a.number();
        const int ptype = a.i32();
        const NormCall f(a, q, k);
        a.dev = q.is_cuda() ? (int)q.get_device() : -1;
        void *pgq = f.with(a, "d_q_out", q, gq), *pgk = f.with(a, "d_k_out", k, gk), *pdq = f.with(a, "dq", q, dq), *pdk = f.with(a, "dk", k, dk);
        a.here("k", k);
        const auto ty = q.scalar_type();
        void *pwq = a.dense("wq", wq, {f.D}, ty), *pwk = a.dense("wk", wk, {f.D}, ty), *pdwq = a.dense("dwq", dwq, {f.D}, ty),
             *pdwk = a.dense("dwk", dwk, {f.D}, ty);
        f.rows(a, n, c, t, tail, flags);
        a.device_of(q);
        size_t bytes;
        void* pws = a.scratch(ws, &bytes);
        void* stream = a.stream();
        return unlocked([&] {
            return p_norm_bwd(q.data_ptr(), k.data_ptr(), pwq, pwk, pgq, pgk, pdq, pdk, pdwq, pdwk, f.B, f.Hq, f.Hk, f.D, n, c, t, c * t, tail, f.qs,
                              f.ks, f.dt, eps, theta, ptype, flags, pws, bytes, stream);
        });
    });
}

PyObject* qk_norm_rope_append(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    return guarded([&] {
        Args a("loma_qk_norm_rope_append", args, n_args, 13);
        const at::Tensor &q = *a.tensor("q"), &k = *a.tensor("k_new"), &v = *a.tensor("v_new"), *wq = a.tensor("wq", true), *wk = a.tensor("wk", true),
                         &qo = *a.tensor("q_out"), &kp = *a.tensor("k_pool"), &vp = *a.tensor("v_pool"), &slots = *a.tensor("slots"),
                         &pos = *a.tensor("positions");
        const float eps = a.number(), theta = a.number();
        if (q.dim() != 3 || k.dim() != 3 || kp.dim() != 4) a.no("q [T, Hq, D], k_new, v_new [T, Hk, D], pools [n_pages, Hk, page_size, D]");
        const int64_t T = q.size(0), Hq = q.size(1), D = q.size(2), pages = kp.size(0), Hk = kp.size(1), ps = kp.size(2);
        if (T > INT32_MAX || pages > INT32_MAX || ps > INT32_MAX || D > INT32_MAX || Hq > INT32_MAX || Hk > INT32_MAX) a.no("tensors too large");
        const auto ty = q.scalar_type();
        const loma_dtype dt = a.dtype(q);
        a.dev = q.is_cuda() ? (int)q.get_device() : -1;
        for (const at::Tensor* x : {&k, &v})
            if (x->dim() != 3 || x->size(0) != T || x->size(1) != Hk || x->size(2) != D || x->scalar_type() != ty) a.no("k_new and v_new must be [T, Hk, D] in q's dtype");
        for (const at::Tensor* x : {&q, &k, &v})
            if (x->numel() && x->stride(2) != 1) a.no("head dimension must be contiguous");
        a.here("k_new", k);
        a.here("v_new", v);
        void *pqo = a.dense("q_out", &qo, {T, Hq, D}, ty), *pkp = a.dense("k_pool", &kp, {pages, Hk, ps, D}, ty),
             *pvp = a.dense("v_pool", &vp, {pages, Hk, ps, D}, ty), *pwq = a.dense("wq", wq, {D}, ty), *pwk = a.dense("wk", wk, {D}, ty);
        int32_t *psl = a.words("slots", &slots, T), *ppo = a.words("positions", &pos, T);
        a.device_of(q);
        void* stream = a.stream();
        int64_t qs[2], ks[2], vs[2];
        strides_of(q, 2, qs);
        strides_of(k, 2, ks);
        strides_of(v, 2, vs);
        return unlocked([&] {
            return p_append(q.data_ptr(), k.data_ptr(), v.data_ptr(), pwq, pwk, pqo, pkp, pvp, psl, ppo, (int)T, (int)Hq, (int)Hk, (int)D, (int)ps,
                            (int)pages, qs, ks, vs, dt, eps, theta, stream);
        });
    });
}

// What both forms of the shared-prefix decode step check alike.
struct SharedCall {
    int B, Hq, Hkv, D;
    loma_dtype dt;
    void *pkn, *pvn, *po, *ws;
    float* plse;
    int32_t* plens;
    size_t ws_bytes;

    SharedCall(Args& a, const at::Tensor& q, const at::Tensor* kn, const at::Tensor* vn, const at::Tensor& o, const at::Tensor* lse, const at::Tensor& lens,
               int64_t heads, const at::Tensor* workspace) {
        if (q.dim() != 4 || q.size(2) != 1 || !q.is_contiguous()) a.no("q must be a contiguous [B, Hq, 1, D] tensor");
        if (q.size(0) > INT32_MAX || q.size(1) > INT32_MAX || q.size(3) > INT32_MAX || heads > INT32_MAX) a.no("tensors too large");
        B = (int)q.size(0); Hq = (int)q.size(1); D = (int)q.size(3); Hkv = (int)heads;
        dt = a.dtype(q);
        a.dev = q.is_cuda() ? (int)q.get_device() : -1;
        const auto ty = q.scalar_type();
        po = a.dense("o", &o, q.sizes(), ty);
        pkn = a.dense("k_new", kn, {B, Hkv, 1, D}, ty);
        pvn = a.dense("v_new", vn, {B, Hkv, 1, D}, ty);
        plse = static_cast<float*>(a.dense("lse", lse, {B, Hq}, at::kFloat));
        plens = a.words("cache_lens", &lens, B);
        ws = a.scratch(workspace, &ws_bytes);
    }
};

PyObject* decode_attn_shared(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    return guarded([&] {
        Args a("loma_decode_attn_shared", args, n_args, 16);
        const at::Tensor &q = *a.tensor("q"), *kn = a.tensor("k_new", true), *vn = a.tensor("v_new", true), *kp = a.tensor("k_prefix", true),
                         *vp = a.tensor("v_prefix", true);
        const int prefix_len = a.i32();
        const at::Tensor &kc = *a.tensor("k_cache"), &vc = *a.tensor("v_cache"), &o = *a.tensor("o"), *lse = a.tensor("lse", true),
                         &lens = *a.tensor("cache_lens");
        const int max_len = a.i32();
        const at::Tensor* ws = a.tensor("workspace", true);
        const unsigned flags = (unsigned)a.integer();
        const float scale = a.number();
        if (kc.dim() != 4) a.no("k_cache must be [B, Hkv, cap, D]");
        const SharedCall f(a, q, kn, vn, o, lse, lens, kc.size(1), ws);
        const auto ty = q.scalar_type();
        if (kc.size(2) > INT32_MAX) a.no("tensors too large");
        void *pkc = a.dense("k_cache", &kc, {f.B, f.Hkv, kc.size(2), f.D}, ty), *pvc = a.dense("v_cache", &vc, {f.B, f.Hkv, kc.size(2), f.D}, ty);
        if (kp && (kp->dim() != 3 || kp->size(1) > INT32_MAX)) a.no("k_prefix must be [Hkv, prefix_cap, D]");
        const int64_t cap = kp ? kp->size(1) : 0;
        void *pkp = a.dense("k_prefix", kp, {f.Hkv, cap, f.D}, ty), *pvp = a.dense("v_prefix", vp, {f.Hkv, cap, f.D}, ty);
        a.device_of(q);
        void* stream = a.stream();
        return unlocked([&] {
            return p_shared(q.data_ptr(), f.pkn, f.pvn, pkp, pvp, pkc, pvc, f.po, f.plse, f.B, f.Hq, f.Hkv, f.D, (int)cap, prefix_len, (int)kc.size(2),
                            f.plens, max_len, f.dt, scale, flags, f.ws, f.ws_bytes, stream);
        });
    });
}

PyObject* decode_attn_shared_paged(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    return guarded([&] {
        Args a("loma_decode_attn_shared_paged", args, n_args, 16);
        const at::Tensor &q = *a.tensor("q"), *kn = a.tensor("k_new", true), *vn = a.tensor("v_new", true), &kp = *a.tensor("k_pool"),
                         &vp = *a.tensor("v_pool"), *ptable = a.tensor("prefix_table", true);
        const int prefix_len = a.i32();
        const at::Tensor &table = *a.tensor("block_table"), &o = *a.tensor("o"), *lse = a.tensor("lse", true), &lens = *a.tensor("cache_lens");
        const int max_len = a.i32();
        const at::Tensor* ws = a.tensor("workspace", true);
        const unsigned flags = (unsigned)a.integer();
        const float scale = a.number();
        if (kp.dim() != 4) a.no("k_pool must be [n_pages, Hkv, page_size, D]");
        const SharedCall f(a, q, kn, vn, o, lse, lens, kp.size(1), ws);
        const auto ty = q.scalar_type();
        const int64_t pages = kp.size(0), ps = kp.size(2), n_prefix = ptable ? ptable->numel() : 0;
        if (table.dim() != 2 || table.size(0) != f.B) a.no("block_table must be [B, max_pages]");
        if (pages > INT32_MAX || ps > INT32_MAX || n_prefix > INT32_MAX || table.size(1) > INT32_MAX) a.no("tensors too large");
        void *pkp = a.dense("k_pool", &kp, {pages, f.Hkv, ps, f.D}, ty), *pvp = a.dense("v_pool", &vp, {pages, f.Hkv, ps, f.D}, ty);
        int32_t *ppt = a.words("prefix_table", ptable, -1), *pbt = a.words("block_table", &table, -1);
        a.device_of(q);
        void* stream = a.stream();
        return unlocked([&] {
            return p_shared_paged(q.data_ptr(), f.pkn, f.pvn, pkp, pvp, ppt, pbt, f.po, f.plse, f.B, f.Hq, f.Hkv, f.D, (int)ps, (int)n_prefix, prefix_len,
                                  (int)table.size(1), (int)pages, f.plens, max_len, f.dt, scale, flags, f.ws, f.ws_bytes, stream);
        });
    });
}

// Addresses of the six entry points, in the order of their declarations above.
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    void* p[6];
    if (n != 6) {
        PyErr_SetString(PyExc_ValueError, "bind takes six addresses");
        return nullptr;
    }
    for (int i = 0; i < 6; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: an address is zero");
            return nullptr;
        }
    }
    p_extend = reinterpret_cast<decltype(p_extend)>(p[0]);
    p_norm_fwd = reinterpret_cast<decltype(p_norm_fwd)>(p[1]);
    p_norm_bwd = reinterpret_cast<decltype(p_norm_bwd)>(p[2]);
    p_append = reinterpret_cast<decltype(p_append)>(p[3]);
    p_shared = reinterpret_cast<decltype(p_shared)>(p[4]);
    p_shared_paged = reinterpret_cast<decltype(p_shared_paged)>(p[5]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)())bind, METH_FASTCALL, "addresses of the entry points"},
    {"paged_extend", (PyCFunction)(void (*)())paged_extend, METH_FASTCALL, "loma_paged_extend"},
    {"qk_norm_rope_fwd", (PyCFunction)(void (*)())qk_norm_rope_fwd, METH_FASTCALL, "loma_qk_norm_rope_fwd"},
    {"qk_norm_rope_bwd", (PyCFunction)(void (*)())qk_norm_rope_bwd, METH_FASTCALL, "loma_qk_norm_rope_bwd"},
    {"qk_norm_rope_append", (PyCFunction)(void (*)())qk_norm_rope_append, METH_FASTCALL, "loma_qk_norm_rope_append"},
    {"decode_attn_shared", (PyCFunction)(void (*)())decode_attn_shared, METH_FASTCALL, "loma_decode_attn_shared"},
    {"decode_attn_shared_paged", (PyCFunction)(void (*)())decode_attn_shared_paged, METH_FASTCALL, "loma_decode_attn_shared_paged"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling for libloma", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the Python and torch this module was compiled against; binding.py refuses it under any other
PyMODINIT_FUNC PyInit__marshal(void) {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", LOMA_BUILT_FOR) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
