// The calls of a rollout's inner loop without Python between the tensors and the library: checks every tensor (device,
// contiguity, type), takes addresses and sizes and calls the C entry point.  A step of a small block is bound by the host:
// the call cost it 17.3 us, of which the library's own 3 launches 10.  8 steps of one block of 32 rows at D = 256, V = 4096:
// 155 us with ctypes, 104 us with this.
//
// Each function returns the entry point's status, or None when an argument is not what it should be: the caller then
// goes through the checks of binding.py, which say what is wrong.  A tensor without memory of its own (a FakeTensor of a
// trace, the batched tensor of vmap) throws where it is asked for its address: that is caught, and None as well.
#include <Python.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/dare.h"

namespace {

decltype(&dare_denoise_block) f_denoise = nullptr;
decltype(&dare_denoise_block_sampled) f_denoise_sampled = nullptr;
decltype(&dare_attn_varlen) f_varlen = nullptr;
decltype(&dare_attn_paged) f_attn_paged = nullptr;
decltype(&dare_paged_kv_append) f_paged_append = nullptr;
decltype(&dare_qk_norm_rope) f_qk_norm = nullptr;
decltype(&dare_qk_norm_rope_backward) f_qk_norm_back = nullptr;

// Walks the argument list; `ok` turns false at the first argument that does not fit.
struct Args {
    PyObject* const* v;
    Py_ssize_t n, at = 0;
    bool ok = true;
    long device = -1;

    PyObject* next() {
        if (at >= n) { ok = false; return Py_None; }
        return v[at++];
    }
    const at::Tensor* tensor(at::ScalarType type) {      // NULL for None
        PyObject* o = next();
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) { ok = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.is_cuda() || t.get_device() != device || !t.is_contiguous() || t.scalar_type() != type) ok = false;
        return &t;
    }
    void* ptr(at::ScalarType type) {
        const at::Tensor* t = tensor(type);
        return t && ok ? t->data_ptr() : nullptr;
    }
    void* bf16() { return ptr(at::kBFloat16); }
    int32_t* i32() { return static_cast<int32_t*>(ptr(at::kInt)); }
    float* f32() { return static_cast<float*>(ptr(at::kFloat)); }
    int32_t* counts() {                                   // a device tensor or a page-locked host tensor
        PyObject* o = v[at < n ? at : n - 1];
        if (o != Py_None && THPVariable_Check(o)) {
            const at::Tensor& t = THPVariable_Unpack(o);
            if (!t.is_cuda()) {
                ++at;
                if (!t.is_pinned() || !t.is_contiguous() || t.scalar_type() != at::kInt) { ok = false; return nullptr; }
                return static_cast<int32_t*>(t.data_ptr());
            }
        }
        return i32();
    }
    long long integer() {
        const long long x = PyLong_AsLongLong(next());
        if (x == -1 && PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return x;
    }
    unsigned long long bits() {                           // an integer modulo 2^64
        const unsigned long long x = PyLong_AsUnsignedLongLongMask(next());
        if (PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return x;
    }
    int flag() {
        const int x = PyObject_IsTrue(next());
        if (x < 0) { PyErr_Clear(); ok = false; }
        return x > 0;
    }
    double real() {
        const double x = PyFloat_AsDouble(next());
        if (x == -1.0 && PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return x;
    }
    void* address() { return reinterpret_cast<void*>(static_cast<uintptr_t>(integer())); }
};

// (handle, device, stream, scale, q, k_pre, v_pre, prefix_len, k_blk, v_blk, k_suf, v_suf, suffix_len, attn_out, lse, hidden, w,
//  mask_id, exclude, [temperature, seed, step,] tokens, block_start, mode, threshold, k, pred, conf, n_committed, n_remaining)
template <bool SAMPLED>
PyObject* denoise_checked(PyObject* const* argv, Py_ssize_t n) {
    Args a{argv, n};
    dare_ctx* ctx = static_cast<dare_ctx*>(a.address());
    a.device = static_cast<long>(a.integer());
    void* stream = a.address();
    const float scale = static_cast<float>(a.real());
    const at::Tensor* q = a.tensor(at::kBFloat16);
    const at::Tensor* k_pre = a.tensor(at::kBFloat16);
    if (!a.ok || !q || !k_pre || q->dim() != 4 || k_pre->dim() != 4) Py_RETURN_NONE;
    void* v_pre = a.bf16();
    const int32_t* prefix_len = a.i32();
    void *k_blk = a.bf16(), *v_blk = a.bf16();
    const at::Tensor* k_suf = a.tensor(at::kBFloat16);
    void* v_suf = a.bf16();
    const int32_t* suffix_len = a.i32();
    void* out = a.bf16();
    float* lse = a.f32();
    const at::Tensor* hidden = a.tensor(at::kBFloat16);
    const at::Tensor* w = a.tensor(at::kBFloat16);
    const int32_t mask_id = static_cast<int32_t>(a.integer());
    const int exclude = a.flag();
    const float temperature = SAMPLED ? static_cast<float>(a.real()) : 0.f;
    const uint64_t seed = SAMPLED ? a.bits() : 0;
    const uint32_t step = SAMPLED ? static_cast<uint32_t>(a.bits()) : 0;
    const at::Tensor* tokens = a.tensor(at::kInt);
    const int block_start = static_cast<int>(a.integer()), mode = static_cast<int>(a.integer());
    const float threshold = static_cast<float>(a.real());
    const int k = static_cast<int>(a.integer());
    int32_t* pred = a.i32();
    float* conf = a.f32();
    int32_t *n_committed = a.counts(), *n_remaining = a.counts();
    if (!a.ok || a.at != n || !hidden || !w || !tokens || hidden->dim() != 2 || w->dim() < 1 || tokens->dim() < 2 ||
        (k_suf && k_suf->dim() != 4))
        Py_RETURN_NONE;
    const int B = static_cast<int>(q->size(0)), L = static_cast<int>(q->size(1)), Hq = static_cast<int>(q->size(2));
    const int d = static_cast<int>(q->size(3)), Hkv = static_cast<int>(k_pre->size(1));
    const int prefix_cap = static_cast<int>(k_pre->size(2)), suffix_cap = k_suf ? static_cast<int>(k_suf->size(2)) : 0;
    // (everything that may throw stands in front of the part without the interpreter's lock)
    const void *q_ptr = q->data_ptr(), *k_ptr = k_pre->data_ptr(), *suf = k_suf ? k_suf->data_ptr() : nullptr;
    const void *x_ptr = hidden->data_ptr(), *w_ptr = w->data_ptr();
    const int D = static_cast<int>(hidden->size(1)), V = static_cast<int>(w->size(0));
    int32_t* tok = static_cast<int32_t*>(tokens->data_ptr());
    const int64_t row_stride = tokens->size(1);
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    if (SAMPLED)
        rc = f_denoise_sampled(ctx, B, L, Hq, Hkv, d, prefix_cap, suffix_cap, scale, q_ptr, k_ptr, v_pre, prefix_len, k_blk, v_blk,
                               suf, v_suf, suffix_len, out, lse, x_ptr, D, w_ptr, V, mask_id, exclude, temperature, seed, step, tok,
                               row_stride, block_start, mode, threshold, k, pred, conf, n_committed, n_remaining, stream);
    else
        rc = f_denoise(ctx, B, L, Hq, Hkv, d, prefix_cap, suffix_cap, scale, q_ptr, k_ptr, v_pre, prefix_len, k_blk, v_blk, suf,
                       v_suf, suffix_len, out, lse, x_ptr, D, w_ptr, V, mask_id, exclude, tok, row_stride, block_start, mode,
                       threshold, k, pred, conf, n_committed, n_remaining, stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(rc);
}

// (handle, device, stream, scale, q, k, v, cu_seqlens, max_seqlen, out, lse)
PyObject* varlen_checked(PyObject* const* argv, Py_ssize_t n) {
    Args a{argv, n};
    dare_ctx* ctx = static_cast<dare_ctx*>(a.address());
    a.device = static_cast<long>(a.integer());
    void* stream = a.address();
    const float scale = static_cast<float>(a.real());
    const at::Tensor *q = a.tensor(at::kBFloat16), *k = a.tensor(at::kBFloat16);
    void* v = a.bf16();
    const at::Tensor* cu = a.tensor(at::kInt);
    const int max_seqlen = static_cast<int>(a.integer());
    void* out = a.bf16();
    float* lse = a.f32();
    if (!a.ok || a.at != n || !q || !k || !cu || q->dim() != 3 || k->dim() < 2) Py_RETURN_NONE;
    const int total = static_cast<int>(q->size(0)), Hq = static_cast<int>(q->size(1)), d = static_cast<int>(q->size(2));
    const int Hkv = static_cast<int>(k->size(1)), n_seqs = static_cast<int>(cu->numel()) - 1;
    const void *q_ptr = q->data_ptr(), *k_ptr = k->data_ptr();
    const int32_t* cu_ptr = static_cast<const int32_t*>(cu->data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = f_varlen(ctx, total, n_seqs, max_seqlen, Hq, Hkv, d, scale, q_ptr, k_ptr, v, cu_ptr, out, lse, stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(rc);
}

// Whether a tensor has this shape (NULL: an argument that was left out).
bool has_shape(const at::Tensor* t, std::initializer_list<int64_t> shape) { return !t || t->sizes() == at::IntArrayRef(shape); }
const void* data_of(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
int as_int(int64_t x) { return x >= 0 && x <= 0x7fffffff ? static_cast<int>(x) : -1; }      // (the library refuses -1)

// (handle, device, stream, scale, q, k_pages, v_pages, block_table, kv_lens, window, sinks, out, lse)
PyObject* attn_paged_checked(PyObject* const* argv, Py_ssize_t n) {
    Args a{argv, n};
    dare_ctx* ctx = static_cast<dare_ctx*>(a.address());
    a.device = static_cast<long>(a.integer());
    void* stream = a.address();
    const float scale = static_cast<float>(a.real());
    const at::Tensor *q = a.tensor(at::kBFloat16), *k = a.tensor(at::kBFloat16), *v = a.tensor(at::kBFloat16);
    const at::Tensor *table = a.tensor(at::kInt), *lens = a.tensor(at::kInt);
    const long long window = a.integer(), sinks = a.integer();
    const at::Tensor *out = a.tensor(at::kBFloat16), *lse = a.tensor(at::kFloat);
    if (!a.ok || a.at != n || !q || !k || !v || !table || !lens || !out || q->dim() != 4 || k->dim() != 4 || table->dim() != 2) Py_RETURN_NONE;
    const int64_t B = q->size(0), L = q->size(1), Hq = q->size(2), d = q->size(3);
    if (k->size(3) != d || v->sizes() != k->sizes() || out->sizes() != q->sizes() || table->size(0) != B || !has_shape(lens, {B}) ||
        !has_shape(lse, {B, Hq, L}))
        Py_RETURN_NONE;
    const void *q_ptr = q->data_ptr(), *k_ptr = k->data_ptr(), *v_ptr = v->data_ptr();
    const int32_t *t_ptr = static_cast<const int32_t*>(table->data_ptr()), *n_ptr = static_cast<const int32_t*>(lens->data_ptr());
    void* o_ptr = out->data_ptr();
    float* l_ptr = static_cast<float*>(const_cast<void*>(data_of(lse)));
    const int n_pages = as_int(k->size(0)), Hkv = as_int(k->size(1)), page = as_int(k->size(2)), max_pages = as_int(table->size(1));
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = f_attn_paged(ctx, as_int(B), as_int(L), as_int(Hq), Hkv, as_int(d), scale, q_ptr, k_ptr, v_ptr, n_pages, page, t_ptr, max_pages, n_ptr,
                      as_int(window), as_int(sinks), o_ptr, l_ptr, stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(rc);
}

// (handle, device, stream, qkv, seq_ids, positions, block_table, k_pages, v_pages, rope_table, q_weight, k_weight, eps, q_out)
PyObject* paged_append_checked(PyObject* const* argv, Py_ssize_t n) {
    Args a{argv, n};
    dare_ctx* ctx = static_cast<dare_ctx*>(a.address());
    a.device = static_cast<long>(a.integer());
    void* stream = a.address();
    const at::Tensor *x = a.tensor(at::kBFloat16), *seq = a.tensor(at::kInt), *pos = a.tensor(at::kInt), *table = a.tensor(at::kInt);
    const at::Tensor *k = a.tensor(at::kBFloat16), *v = a.tensor(at::kBFloat16), *rope = a.tensor(at::kFloat);
    const at::Tensor *wq = a.tensor(at::kBFloat16), *wk = a.tensor(at::kBFloat16);
    const float eps = static_cast<float>(a.real());
    const at::Tensor* q = a.tensor(at::kBFloat16);
    if (!a.ok || a.at != n || !x || !seq || !pos || !table || !k || !v || !rope || !q || x->dim() != 2 || k->dim() != 4 ||
        table->dim() != 2 || rope->dim() != 3 || q->dim() != 3)
        Py_RETURN_NONE;
    const int64_t rows = x->size(0), Hkv = k->size(1), d = k->size(3), Hq = q->size(1);
    if (!has_shape(x, {rows, (Hq + 2 * Hkv) * d}) || !has_shape(seq, {rows}) || !has_shape(pos, {rows}) || v->sizes() != k->sizes() ||
        !has_shape(rope, {rope->size(0), d / 2, 2}) || !has_shape(wq, {d}) || !has_shape(wk, {d}) || !has_shape(q, {rows, Hq, d}))
        Py_RETURN_NONE;
    const void *x_ptr = x->data_ptr(), *wq_ptr = data_of(wq), *wk_ptr = data_of(wk);
    const float* r_ptr = static_cast<const float*>(rope->data_ptr());
    const int32_t *s_ptr = static_cast<const int32_t*>(seq->data_ptr()), *p_ptr = static_cast<const int32_t*>(pos->data_ptr());
    const int32_t* t_ptr = static_cast<const int32_t*>(table->data_ptr());
    void *k_ptr = k->data_ptr(), *v_ptr = v->data_ptr(), *q_ptr = q->data_ptr();
    const int n_pos = as_int(rope->size(0)), n_seqs = as_int(table->size(0)), max_pages = as_int(table->size(1));
    const int n_pages = as_int(k->size(0)), page = as_int(k->size(2));
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = f_paged_append(ctx, x_ptr, as_int(rows), as_int(Hq), as_int(Hkv), as_int(d), wq_ptr, wk_ptr, eps, r_ptr, n_pos, s_ptr, p_ptr, t_ptr,
                        n_seqs, max_pages, n_pages, page, k_ptr, v_ptr, q_ptr, stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(rc);
}

// (handle, device, stream, qkv, positions, rope_table, q_weight, k_weight, eps, q_out, k_out, v_out)
PyObject* qk_norm_checked(PyObject* const* argv, Py_ssize_t n) {
    Args a{argv, n};
    dare_ctx* ctx = static_cast<dare_ctx*>(a.address());
    a.device = static_cast<long>(a.integer());
    void* stream = a.address();
    const at::Tensor *x = a.tensor(at::kBFloat16), *pos = a.tensor(at::kInt), *rope = a.tensor(at::kFloat);
    const at::Tensor *wq = a.tensor(at::kBFloat16), *wk = a.tensor(at::kBFloat16);
    const float eps = static_cast<float>(a.real());
    const at::Tensor *q = a.tensor(at::kBFloat16), *k = a.tensor(at::kBFloat16), *v = a.tensor(at::kBFloat16);
    if (!a.ok || a.at != n || !x || !pos || !rope || !q || !k || !v || x->dim() != 2 || rope->dim() != 3 || q->dim() != 3 || k->dim() != 3)
        Py_RETURN_NONE;
    const int64_t rows = x->size(0), Hq = q->size(1), Hkv = k->size(1), d = q->size(2);
    if (!has_shape(x, {rows, (Hq + 2 * Hkv) * d}) || !has_shape(pos, {rows}) || !has_shape(rope, {rope->size(0), d / 2, 2}) ||
        !has_shape(wq, {d}) || !has_shape(wk, {d}) || !has_shape(q, {rows, Hq, d}) || !has_shape(k, {rows, Hkv, d}) || !has_shape(v, {rows, Hkv, d}))
        Py_RETURN_NONE;
    const void *x_ptr = x->data_ptr(), *wq_ptr = data_of(wq), *wk_ptr = data_of(wk);
    const float* r_ptr = static_cast<const float*>(rope->data_ptr());
    const int32_t* p_ptr = static_cast<const int32_t*>(pos->data_ptr());
    void *q_ptr = q->data_ptr(), *k_ptr = k->data_ptr(), *v_ptr = v->data_ptr();
    const int n_pos = as_int(rope->size(0));
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = f_qk_norm(ctx, x_ptr, as_int(rows), as_int(Hq), as_int(Hkv), as_int(d), wq_ptr, wk_ptr, eps, p_ptr, r_ptr, n_pos, q_ptr, k_ptr, v_ptr,
                   stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(rc);
}

// (handle, device, stream, qkv, positions, rope_table, d_q, d_k, d_v, q_weight, k_weight, eps, d_qkv, d_q_weight, d_k_weight)
PyObject* qk_norm_back_checked(PyObject* const* argv, Py_ssize_t n) {
    Args a{argv, n};
    dare_ctx* ctx = static_cast<dare_ctx*>(a.address());
    a.device = static_cast<long>(a.integer());
    void* stream = a.address();
    const at::Tensor *x = a.tensor(at::kBFloat16), *pos = a.tensor(at::kInt), *rope = a.tensor(at::kFloat);
    const at::Tensor *gq = a.tensor(at::kBFloat16), *gk = a.tensor(at::kBFloat16), *gv = a.tensor(at::kBFloat16);
    const at::Tensor *wq = a.tensor(at::kBFloat16), *wk = a.tensor(at::kBFloat16);
    const float eps = static_cast<float>(a.real());
    const at::Tensor *dx = a.tensor(at::kBFloat16), *dwq = a.tensor(at::kFloat), *dwk = a.tensor(at::kFloat);
    if (!a.ok || a.at != n || !x || !pos || !rope || !gq || !gk || !gv || !dx || x->dim() != 2 || rope->dim() != 3 || gq->dim() != 3 ||
        gk->dim() != 3)
        Py_RETURN_NONE;
    const int64_t rows = x->size(0), Hq = gq->size(1), Hkv = gk->size(1), d = gq->size(2);
    if (!has_shape(x, {rows, (Hq + 2 * Hkv) * d}) || !has_shape(pos, {rows}) || !has_shape(rope, {rope->size(0), d / 2, 2}) ||
        !has_shape(wq, {d}) || !has_shape(wk, {d}) || !has_shape(dwq, {d}) || !has_shape(dwk, {d}) || !has_shape(gq, {rows, Hq, d}) ||
        !has_shape(gk, {rows, Hkv, d}) || !has_shape(gv, {rows, Hkv, d}) || dx->sizes() != x->sizes())
        Py_RETURN_NONE;
    const void *x_ptr = x->data_ptr(), *wq_ptr = data_of(wq), *wk_ptr = data_of(wk);
    const void *gq_ptr = gq->data_ptr(), *gk_ptr = gk->data_ptr(), *gv_ptr = gv->data_ptr();
    const float* r_ptr = static_cast<const float*>(rope->data_ptr());
    const int32_t* p_ptr = static_cast<const int32_t*>(pos->data_ptr());
    void* dx_ptr = dx->data_ptr();
    float *dwq_ptr = static_cast<float*>(const_cast<void*>(data_of(dwq))), *dwk_ptr = static_cast<float*>(const_cast<void*>(data_of(dwk)));
    const int n_pos = as_int(rope->size(0));
    int rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = f_qk_norm_back(ctx, x_ptr, as_int(rows), as_int(Hq), as_int(Hkv), as_int(d), wq_ptr, wk_ptr, eps, p_ptr, r_ptr, n_pos, gq_ptr, gk_ptr,
                        gv_ptr, dx_ptr, dwq_ptr, dwk_ptr, stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(rc);
}

template <PyObject* (*CALL)(PyObject* const*, Py_ssize_t)>
PyObject* entry(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    try {
        return CALL(argv, n);
    } catch (...) {      // (none comes from the library: its entry points do not throw)
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// bind(path of libdare.so): resolves the entry points in the library that binding.py has loaded
PyObject* bind(PyObject*, PyObject* arg) {
    const char* path = PyUnicode_AsUTF8(arg);
    if (!path) return nullptr;
    void* lib = dlopen(path, RTLD_NOW | RTLD_LOCAL);
    if (lib) {
        f_denoise = reinterpret_cast<decltype(f_denoise)>(dlsym(lib, "dare_denoise_block"));
        f_denoise_sampled = reinterpret_cast<decltype(f_denoise_sampled)>(dlsym(lib, "dare_denoise_block_sampled"));
        f_varlen = reinterpret_cast<decltype(f_varlen)>(dlsym(lib, "dare_attn_varlen"));
        f_attn_paged = reinterpret_cast<decltype(f_attn_paged)>(dlsym(lib, "dare_attn_paged"));
        f_paged_append = reinterpret_cast<decltype(f_paged_append)>(dlsym(lib, "dare_paged_kv_append"));
        f_qk_norm = reinterpret_cast<decltype(f_qk_norm)>(dlsym(lib, "dare_qk_norm_rope"));
        f_qk_norm_back = reinterpret_cast<decltype(f_qk_norm_back)>(dlsym(lib, "dare_qk_norm_rope_backward"));
    }
    if (!f_denoise || !f_denoise_sampled || !f_varlen || !f_attn_paged || !f_paged_append || !f_qk_norm || !f_qk_norm_back) {
        PyErr_Format(PyExc_RuntimeError, "%s does not export the library's entry points", path);
        return nullptr;
    }
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", bind, METH_O, nullptr},
    {"denoise_block", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&entry<denoise_checked<false>>)), METH_FASTCALL, nullptr},
    {"denoise_block_sampled", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&entry<denoise_checked<true>>)), METH_FASTCALL, nullptr},
    {"attn_varlen", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&entry<varlen_checked>)), METH_FASTCALL, nullptr},
    {"attn_paged", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&entry<attn_paged_checked>)), METH_FASTCALL, nullptr},
    {"paged_kv_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&entry<paged_append_checked>)), METH_FASTCALL, nullptr},
    {"qk_norm_rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&entry<qk_norm_checked>)), METH_FASTCALL, nullptr},
    {"qk_norm_rope_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&entry<qk_norm_back_checked>)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
