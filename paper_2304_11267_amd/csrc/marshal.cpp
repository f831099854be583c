// marshal.cpp -- the binding's per-call work in native code: tensors' shapes,
// types and placement checked, their pointers taken, and the C entry point
// called.  A call of the attention's smaller kernels lasts 4 to 6 us
// on the GPU; marshalling it through Python and ctypes takes 10, here 3.
//
// Each function takes the entry point's address and the Python function's
// arguments, and returns its status, or None for a call that it does not take:
// anything but plain strided GPU tensors of the expected shapes and types.  The
// Python function then goes its own way, which raises the error (or takes what
// is left, tensor subclasses for one).  No tensor, pointer or result is kept
// between calls.
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <initializer_list>

namespace {

// torch's functions for the current device, and for a device's current stream
PyObject* current_device = nullptr;
PyObject* current_stream = nullptr;

struct Args {
    PyObject* const* v;
    Py_ssize_t n;
    bool ok = true;
    void* fn() { return PyLong_AsVoidPtr(v[0]); }
    // tensor i, or null and ok = false
    const at::Tensor* tensor(Py_ssize_t i) {
        if (!ok || i >= n || !THPVariable_CheckExact(v[i])) return fail();
        const at::Tensor& t = THPVariable_Unpack(v[i]);
        if (!t.defined() || !t.has_storage() || t.layout() != c10::kStrided || !t.is_cuda() || !t.is_contiguous())
            return fail();
        return &t;
    }
    const at::Tensor* tensor(Py_ssize_t i, at::IntArrayRef shape, c10::ScalarType type) {
        const at::Tensor* t = tensor(i);
        if (t && (t->sizes() != shape || t->scalar_type() != type)) return fail();
        return t;
    }
    // tensor i of any strides, or null and ok = false
    const at::Tensor* strided(Py_ssize_t i) {
        if (!ok || i >= n || !THPVariable_CheckExact(v[i])) return fail();
        const at::Tensor& t = THPVariable_Unpack(v[i]);
        if (!t.defined() || !t.has_storage() || t.layout() != c10::kStrided || !t.is_cuda()) return fail();
        return &t;
    }
    bool none(Py_ssize_t i) { return i < n && v[i] == Py_None; }
    // a tensor or None (then null, with ok as it was)
    const at::Tensor* maybe(Py_ssize_t i, at::IntArrayRef shape, c10::ScalarType type) {
        return ok && i < n && v[i] == Py_None ? nullptr : tensor(i, shape, type);
    }
    long long integer(Py_ssize_t i) {
        if (!ok || i >= n || !PyLong_CheckExact(v[i])) return fail(), 0;
        int over = 0;
        const long long r = PyLong_AsLongLongAndOverflow(v[i], &over);
        if (over || r < INT_MIN || r > INT_MAX) fail();
        return r;
    }
    float real(Py_ssize_t i) {
        if (!ok || i >= n || !PyFloat_CheckExact(v[i])) return fail(), 0.0f;
        return (float)PyFloat_AS_DOUBLE(v[i]);
    }
    // stream, where every tensor so far has to live on the current device
    void* stream_here(Py_ssize_t i) {
        PyObject* dev = ok && current_device ? PyObject_CallNoArgs(current_device) : nullptr;
        const long now = dev && PyLong_Check(dev) ? PyLong_AsLong(dev) : -1;
        Py_XDECREF(dev);
        for (Py_ssize_t j = 1; ok && j < i; ++j)
            if (THPVariable_CheckExact(v[j]) && THPVariable_Unpack(v[j]).device().index() != now) fail();
        return stream(i);
    }
    // the stream argument: None for the current stream of the current device
    void* stream(Py_ssize_t i) {
        if (!ok || i >= n) return fail();
        PyObject* h = nullptr;
        if (v[i] != Py_None) {
            h = PyObject_GetAttrString(v[i], "cuda_stream");
        } else if (PyObject* dev = current_device ? PyObject_CallNoArgs(current_device) : nullptr) {
            h = PyObject_CallOneArg(current_stream, dev);
            Py_DECREF(dev);
        }
        void* s = h && PyLong_Check(h) ? PyLong_AsVoidPtr(h) : fail();
        Py_XDECREF(h);
        if (PyErr_Occurred()) fail();
        return s;
    }
    std::nullptr_t fail() {
        ok = false;
        return nullptr;
    }
};

// the C ABI's element types; -1 for another
int type_code(const at::Tensor& t) {
    switch (t.scalar_type()) {
        case c10::kHalf: return 0;
        case c10::kBFloat16: return 1;
        case c10::kFloat: return 2;
        default: return -1;
    }
}
void* ptr(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
bool fits(std::initializer_list<int64_t> sizes) {
    for (int64_t s : sizes)
        if (s > INT_MAX) return false;
    return true;
}

// Call the entry point without the interpreter lock, as ctypes does.
template <typename... A>
PyObject* call(void* fn, A... a) {
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = reinterpret_cast<int (*)(A...)>(fn)(a...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// A C++ exception (a tensor without storage, a device without a runtime) leaves
// the call to the Python function.
template <PyObject* (*F)(Args&)>
PyObject* entry(PyObject*, PyObject* const* v, Py_ssize_t n) {
    try {
        Args a{v, n};
        PyObject* r = n > 0 ? F(a) : nullptr;
        if (r) return r;
    } catch (...) {
    }
    if (PyErr_Occurred()) PyErr_Clear();
    Py_RETURN_NONE;
}

// fn, q, k, v, out, scale, stream
PyObject* forward(Args& a) {
    const at::Tensor* q = a.tensor(1);
    const at::Tensor* k = a.tensor(2);
    if (!q || !k || q->dim() != 4 || k->dim() != 4 || q->scalar_type() != c10::kHalf) return nullptr;
    const int64_t B = q->size(0), H = q->size(1), Lq = q->size(2), D = q->size(3), Lk = k->size(2);
    const int64_t kv[] = {B, H, Lk, D};
    a.tensor(2, kv, c10::kHalf);
    const at::Tensor *v = a.tensor(3, kv, c10::kHalf), *out = a.tensor(4, q->sizes(), c10::kHalf);
    const float scale = a.real(5);
    void* s = a.stream(6);
    if (!a.ok || !fits({B, H, Lq, Lk, D})) return nullptr;
    return call(a.fn(), ptr(q), ptr(k), ptr(v), ptr(out), (int)B, (int)H, (int)Lq, (int)Lk, (int)D, scale, s);
}

// fn, q, k, v, out, ls, scale, stream
PyObject* forward_ex(Args& a) {
    const at::Tensor* q = a.tensor(1);
    if (!q || q->dim() != 4) return nullptr;
    const auto type = q->scalar_type();
    const int64_t B = q->size(0), H = q->size(1), Lq = q->size(2), D = q->size(3);
    const at::Tensor* k = a.tensor(2);
    if (!k || k->dim() != 4) return nullptr;
    const int64_t Lk = k->size(2);
    const int64_t kv[] = {B, H, Lk, D}, st[] = {B, H, Lq, 2};
    a.tensor(2, kv, type);
    const at::Tensor* v = a.tensor(3, kv, type);
    const at::Tensor* out = a.tensor(4, q->sizes(), type);
    const at::Tensor* ls = a.maybe(5, st, c10::kFloat);
    const float scale = a.real(6);
    void* s = a.stream(7);
    const int code = type_code(*q);
    if (!a.ok || code < 0 || !fits({B, H, Lq, Lk, D})) return nullptr;
    return call(a.fn(), ptr(q), ptr(k), ptr(v), ptr(out), ptr(ls), (int)B, (int)H, (int)Lq, (int)Lk, (int)D, scale, code, s);
}

// fn, a, ls, p, scale, stream
PyObject* softmax_rows(Args& a) {
    const at::Tensor* x = a.tensor(1);
    if (!x || x->dim() != 2) return nullptr;
    const at::Tensor* ls = a.tensor(2);
    const at::Tensor* p = a.maybe(3, x->sizes(), x->scalar_type());
    const float scale = a.real(4);
    void* s = a.stream(5);
    const int code = type_code(*x);
    if (!a.ok || code < 0 || ls->scalar_type() != c10::kFloat || ls->numel() != 2 * x->size(0)) return nullptr;
    return call(a.fn(), ptr(x), ptr(ls), ptr(p), (long long)x->size(0), (long long)x->size(1), scale, code, s);
}

// fn, q, k, a, scale, stream
PyObject* logits(Args& a) {
    const at::Tensor* q = a.tensor(1);
    const at::Tensor* k = a.tensor(2);
    if (!q || !k || q->dim() != 4 || k->dim() != 4) return nullptr;
    const int64_t B = q->size(0), H = q->size(1), Lq = q->size(2), D = q->size(3), Lk = k->size(2);
    const int64_t ks[] = {B, H, Lk, D}, as[] = {B, H, Lq, Lk};
    a.tensor(2, ks, q->scalar_type());
    const at::Tensor* x = a.tensor(3);
    const float scale = a.real(4);
    void* s = a.stream(5);
    if (!a.ok || x->sizes() != at::IntArrayRef(as) || !fits({B, H, Lq, Lk, D})) return nullptr;
    const int code = type_code(*q), acode = type_code(*x);
    if (code < 0 || acode < 0) return nullptr;
    return call(a.fn(), ptr(q), ptr(k), ptr(x), (int)B, (int)H, (int)Lq, (int)Lk, (int)D, scale, code, acode, s);
}

// fn, a, ls, v, out, stream
PyObject* softmax_pv(Args& a) {
    const at::Tensor* x = a.tensor(1);
    const at::Tensor* ls = a.tensor(2);
    const at::Tensor* v = a.tensor(3);
    if (!x || !ls || !v || x->dim() != 4 || v->dim() != 4) return nullptr;
    const int64_t B = x->size(0), H = x->size(1), Lq = x->size(2), Lk = x->size(3), D = v->size(3);
    const int64_t vs[] = {B, H, Lk, D}, os[] = {B, H, Lq, D};
    a.tensor(3, vs, v->scalar_type());
    const at::Tensor* out = a.tensor(4, os, v->scalar_type());
    void* s = a.stream(5);
    const int code = type_code(*v), acode = type_code(*x);
    if (!a.ok || code < 0 || acode < 0 || ls->scalar_type() != c10::kFloat || ls->numel() != 2 * B * H * Lq ||
        !fits({B, H, Lq, Lk, D}))
        return nullptr;
    return call(a.fn(), ptr(x), ptr(ls), ptr(v), ptr(out), (int)B, (int)H, (int)Lq, (int)Lk, (int)D, acode, code, s);
}

// fn, x, ctx, wq, wk, wv, wo, bo, out, workspace, heads, scale, stream
PyObject* attention_block(Args& a) {
    const at::Tensor* x = a.tensor(1);
    const at::Tensor* ctx = a.tensor(2);
    if (!x || !ctx || x->dim() != 3 || ctx->dim() != 3) return nullptr;
    const auto type = x->scalar_type();
    const int64_t B = x->size(0), Lq = x->size(1), C = x->size(2), Lk = ctx->size(1), Cc = ctx->size(2);
    const int64_t cs[] = {B, Lk, Cc}, cc[] = {C, C}, ccc[] = {C, Cc}, c1[] = {C};
    a.tensor(2, cs, type);
    const at::Tensor *wq = a.tensor(3, cc, type), *wk = a.tensor(4, ccc, type), *wv = a.tensor(5, ccc, type),
                     *wo = a.tensor(6, cc, type), *bo = a.maybe(7, c1, type), *out = a.tensor(8, x->sizes(), type),
                     *ws = a.tensor(9);
    const int heads = (int)a.integer(10);
    const float scale = a.real(11);
    void* s = a.stream(12);
    const int code = type_code(*x);
    if (!a.ok || code < 0 || !fits({B, Lq, Lk, C, Cc})) return nullptr;
    return call(a.fn(), ptr(x), ptr(ctx), ptr(wq), ptr(wk), ptr(wv), ptr(wo), ptr(bo), ptr(out), ptr(ws),
                (long long)(ws->numel() * ws->element_size()), (int)B, (int)Lq, (int)Lk, (int)C, (int)Cc, heads, scale,
                code, s);
}

// fn, x, wq, k, v, wo, bo, out, workspace, scale, stream
PyObject* attention_block_kv(Args& a) {
    const at::Tensor* x = a.tensor(1);
    const at::Tensor* k = a.tensor(3);
    if (!x || !k || x->dim() != 3 || k->dim() != 4) return nullptr;
    const auto type = x->scalar_type();
    const int64_t B = x->size(0), Lq = x->size(1), C = x->size(2), H = k->size(1), Lk = k->size(2);
    if (H < 1) return nullptr;
    const int64_t ks[] = {B, H, Lk, C / H}, cc[] = {C, C}, c1[] = {C};
    a.tensor(3, ks, type);
    const at::Tensor *wq = a.tensor(2, cc, type), *v = a.tensor(4, ks, type), *wo = a.tensor(5, cc, type),
                     *bo = a.maybe(6, c1, type), *out = a.tensor(7, x->sizes(), type), *ws = a.tensor(8);
    const float scale = a.real(9);
    void* s = a.stream(10);
    const int code = type_code(*x);
    if (!a.ok || code < 0 || !fits({B, Lq, Lk, C, H})) return nullptr;
    return call(a.fn(), ptr(x), ptr(wq), ptr(k), ptr(v), ptr(wo), ptr(bo), ptr(out), ptr(ws),
                (long long)(ws->numel() * ws->element_size()), (int)B, (int)Lq, (int)Lk, (int)C, (int)H, scale, code, s);
}

// fn, x, groups, y, gamma, beta, eps, stream
PyObject* group_norm(Args& a) {
    const at::Tensor* x = a.tensor(1);
    if (!x || x->dim() < 2) return nullptr;
    const auto type = x->scalar_type();
    const int64_t B = x->size(0), C = x->size(1), c1[] = {C};
    int64_t HW = 1;
    for (int64_t i = 2; i < x->dim(); ++i) HW *= x->size(i);
    const int groups = (int)a.integer(2);
    const at::Tensor *y = a.tensor(3, x->sizes(), type), *gamma = a.maybe(4, c1, type), *beta = a.maybe(5, c1, type);
    const float eps = a.real(6);
    void* s = a.stream(7);
    const int code = type_code(*x);
    if (!a.ok || code < 0 || !fits({B, C})) return nullptr;
    return call(a.fn(), ptr(x), ptr(gamma), ptr(beta), ptr(y), (int)B, (int)C, (long long)HW, groups, eps, code, s);
}

// fn, h, out, stream
PyObject* geglu(Args& a) {
    const at::Tensor* h = a.tensor(1);
    if (!h || h->dim() < 1 || h->numel() == 0) return nullptr;
    const int64_t F2 = h->size(-1);
    if (F2 % 2) return nullptr;
    const at::Tensor* out = a.tensor(2);
    void* s = a.stream(3);
    const int code = type_code(*h);
    if (!a.ok || code < 0 || out->scalar_type() != h->scalar_type() || out->dim() != h->dim() ||
        out->sizes().slice(0, out->dim() - 1) != h->sizes().slice(0, h->dim() - 1) || out->size(-1) != F2 / 2 ||
        !fits({F2 / 2}))
        return nullptr;
    return call(a.fn(), ptr(h), ptr(out), (long long)(h->numel() / F2), (int)(F2 / 2), code, s);
}

// fn, x, u, y, workspace, bias, stream
PyObject* conv3x3(Args& a) {
    const at::Tensor* x = a.tensor(1);
    const at::Tensor* u = a.tensor(2);
    if (!x || !u || x->dim() != 4 || u->dim() != 3) return nullptr;
    const auto type = x->scalar_type();
    const int64_t B = x->size(0), Ci = x->size(1), H = x->size(2), W = x->size(3), Co = u->size(1);
    const int64_t us[] = {36, Co, Ci}, ys[] = {B, Co, H, W}, c1[] = {Co};
    a.tensor(2, us, type);
    const at::Tensor *y = a.tensor(3, ys, type), *ws = a.tensor(4), *bias = a.maybe(5, c1, type);
    void* s = a.stream(6);
    const int code = type_code(*x);
    if (!a.ok || code < 0 || !fits({B, Ci, Co, H, W})) return nullptr;
    return call(a.fn(), ptr(x), ptr(u), ptr(bias), ptr(y), ptr(ws), (long long)(ws->numel() * ws->element_size()),
                (int)B, (int)Ci, (int)Co, (int)H, (int)W, code, s);
}

// a layout's sizes: rows [B, L, C] or heads [B, H, L, C / H]
bool row_sizes(const at::Tensor& t, long long layout, int64_t heads, int64_t* B, int64_t* L, int64_t* C) {
    if (layout == 1) {
        if (t.dim() != 4 || t.size(1) != heads) return false;
        *B = t.size(0), *L = t.size(2), *C = heads * t.size(3);
    } else {
        if (layout != 0 || t.dim() != 3) return false;
        *B = t.size(0), *L = t.size(1), *C = t.size(2);
    }
    return true;
}
bool is_rows(const at::Tensor* t, long long layout, int64_t heads, int64_t B, int64_t L, int64_t C, c10::ScalarType type) {
    int64_t b, l, c;
    return t && t->scalar_type() == type && row_sizes(*t, layout, heads, &b, &l, &c) && b == B && l == L && c == C;
}

// fn, x, w, y, down, up, ids, workspace, scales, bias, heads, x_layout, y_layout, stream
PyObject* linear_adapters(Args& a) {
    const at::Tensor *x = a.tensor(1), *w = a.tensor(2), *y = a.tensor(3), *down = a.tensor(4), *ws = a.tensor(7);
    const long long heads = a.integer(10), xl = a.integer(11), yl = a.integer(12);
    int64_t B, L, K;
    if (!a.ok || w->dim() != 2 || down->dim() != 3 || heads < 1 || !row_sizes(*x, xl, heads, &B, &L, &K)) return nullptr;
    const auto type = x->scalar_type();
    const int64_t N = w->size(0), A = down->size(0), R = down->size(1);
    const int64_t wsz[] = {N, K}, ds[] = {A, R, K}, us[] = {A, N, R}, b1[] = {B}, a1[] = {A}, n1[] = {N};
    a.tensor(2, wsz, type);
    a.tensor(4, ds, type);
    const at::Tensor *up = a.tensor(5, us, type), *ids = a.tensor(6, b1, c10::kInt), *scales = a.maybe(8, a1, c10::kFloat),
                     *bias = a.maybe(9, n1, type);
    void* s = a.stream_here(13);
    const int code = type_code(*x);
    if (!a.ok || code < 0 || !is_rows(y, yl, heads, B, L, N, type) || !fits({B, L, K, N, R, A})) return nullptr;
    return call(a.fn(), ptr(x), ptr(w), ptr(bias), ptr(down), ptr(up), ptr(ids), ptr(scales), ptr(y), ptr(ws),
                (long long)(ws->numel() * ws->element_size()), (int)B, (int)L, (int)K, (int)N, (int)R, (int)A, (int)heads,
                (int)xl, (int)yl, code, s);
}

// fn, q, qo, heads, k, ko, gamma_q, gamma_k, pos, freqs, pairs, norm, eps, pairing, x_layout, y_layout, stream
PyObject* norm_rotate(Args& a) {
    const at::Tensor *q = a.tensor(1), *qo = a.tensor(2);
    const long long H = a.integer(3), norm = a.integer(11), pairing = a.integer(13), xl = a.integer(14), yl = a.integer(15);
    const float eps = a.real(12);
    int64_t B, L, C;
    if (!a.ok || H < 1 || !row_sizes(*q, xl, H, &B, &L, &C) || C % H) return nullptr;
    const auto type = q->scalar_type();
    const int64_t D = C / H, d1[] = {D};
    const at::Tensor *k = a.maybe(4, q->sizes(), type), *ko = a.maybe(5, qo->sizes(), type),
                     *gq = a.maybe(6, d1, type), *gk = a.maybe(7, d1, type);
    if (!a.ok || !k != !ko || !PyTuple_CheckExact(a.v[10])) return nullptr;
    const Py_ssize_t axes = PyTuple_GET_SIZE(a.v[10]);
    int pairs[4] = {0, 0, 0, 0};
    int64_t P = 0, batches = 1;
    if (axes > 4) return nullptr;
    for (Py_ssize_t i = 0; i < axes; ++i) {
        PyObject* o = PyTuple_GET_ITEM(a.v[10], i);
        const long n = PyLong_CheckExact(o) ? PyLong_AsLong(o) : -1;
        if (n < 1 || n > 65536) return nullptr;
        pairs[i] = (int)n;
        P += n;
    }
    const at::Tensor *pos = nullptr, *freqs = nullptr;
    if (axes) {
        pos = a.tensor(8);
        if (!pos || pos->dim() != 3 || pos->scalar_type() != c10::kInt) return nullptr;
        batches = pos->size(0);
        if ((batches != 1 && batches != B) || pos->size(1) != L || pos->size(2) != axes) return nullptr;
        const int64_t p1[] = {P};
        freqs = a.tensor(9, p1, c10::kFloat);
    }
    void* s = a.stream_here(16);
    const int code = type_code(*q);
    if (!a.ok || code < 0 || !is_rows(qo, yl, H, B, L, C, type) || !fits({B, H, L, D})) return nullptr;
    return call(a.fn(), ptr(q), ptr(k), ptr(gq), ptr(gk), ptr(pos), ptr(freqs), ptr(qo), ptr(ko), (int)B, (int)H, (int)L,
                (int)D, (int)axes, (const int*)pairs, (int)batches, (int)norm, eps, (int)pairing, (int)xl, (int)yl, code, s);
}

int64_t blocks(int64_t n, int64_t block) { return (n + block - 1) / block; }

// fn, x, means, stream
PyObject* block_means(Args& a) {
    const at::Tensor* x = a.tensor(1);
    if (!x || x->dim() != 4) return nullptr;
    const int64_t B = x->size(0), H = x->size(1), L = x->size(2), D = x->size(3), ms[] = {B, H, blocks(L, 64), D};
    const at::Tensor* means = a.tensor(2, ms, c10::kFloat);
    void* s = a.stream_here(3);
    const int code = type_code(*x);
    if (!a.ok || code < 0 || !fits({B, H, L, D})) return nullptr;
    return call(a.fn(), ptr(x), ptr(means), (int)B, (int)H, (int)L, (int)D, code, s);
}

// fn, q, means, mask, keep, qblock, stream
PyObject* select_blocks(Args& a) {
    const at::Tensor *q = a.tensor(1), *means = a.tensor(2);
    const long long keep = a.integer(4), qblock = a.integer(5);
    if (!a.ok || q->dim() != 4 || means->dim() != 4 || qblock < 1) return nullptr;
    const int64_t B = q->size(0), H = q->size(1), Lq = q->size(2), D = q->size(3), NB = means->size(2);
    const int64_t ms[] = {B, H, NB, D}, ws[] = {B, H, blocks(Lq, qblock), blocks(NB, 64)};
    a.tensor(2, ms, c10::kFloat);
    const at::Tensor* mask = a.tensor(3, ws, c10::kLong);
    void* s = a.stream_here(6);
    const int code = type_code(*q);
    if (!a.ok || code < 0 || !fits({B, H, Lq, D, NB})) return nullptr;
    return call(a.fn(), ptr(q), ptr(means), ptr(mask), (int)B, (int)H, (int)Lq, (int)NB, (int)D, (int)qblock, (int)keep,
                code, s);
}

// fn, q, k, v, mask, out, scale, qblock, stream
PyObject* sparse_forward(Args& a) {
    const at::Tensor *q = a.tensor(1), *k = a.tensor(2);
    const long long qblock = a.integer(7);
    if (!a.ok || q->dim() != 4 || k->dim() != 4 || qblock < 1) return nullptr;
    const auto type = q->scalar_type();
    const int64_t B = q->size(0), H = q->size(1), Lq = q->size(2), D = q->size(3), Lk = k->size(2);
    const int64_t kv[] = {B, H, Lk, D}, ws[] = {B, H, blocks(Lq, qblock), blocks(blocks(Lk, 64), 64)};
    a.tensor(2, kv, type);
    const at::Tensor *v = a.tensor(3, kv, type), *mask = a.tensor(4, ws, c10::kLong), *out = a.tensor(5, q->sizes(), type);
    const float scale = a.real(6);
    void* s = a.stream_here(8);
    const int code = type_code(*q);
    if (!a.ok || code < 0 || !fits({B, H, Lq, Lk, D})) return nullptr;
    return call(a.fn(), ptr(q), ptr(k), ptr(v), ptr(mask), ptr(out), (int)B, (int)H, (int)Lq, (int)Lk, (int)D, (int)qblock,
                scale, code, s);
}

// fn, x, y, r, h, gate, scale, shift, gamma_r, gamma, beta, skip, norm_r, norm, eps, stream
PyObject* gated_norm(Args& a) {
    const at::Tensor* x = a.tensor(1);
    if (!x || x->dim() != 3 || a.n < 16 || (a.none(2) && a.none(4))) return nullptr;
    const int64_t B = x->size(0), L = x->size(1), C = x->size(2), c1[] = {C};
    // the 16-bit type is that of any tensor that has to have it
    auto type = x->scalar_type();
    for (Py_ssize_t i : {2, 3, 5, 6, 7, 8, 9, 10}) {
        if (a.none(i)) continue;
        const at::Tensor* t = a.strided(i);
        if (!t) return nullptr;
        type = t->scalar_type();
        break;
    }
    if (type == c10::kFloat || (x->scalar_type() != type && x->scalar_type() != c10::kFloat)) return nullptr;
    const at::Tensor *y = a.maybe(2, x->sizes(), type), *r = a.maybe(3, x->sizes(), type),
                     *h = a.maybe(4, x->sizes(), x->scalar_type());
    int64_t batches = 1, groups = 1, strides[3] = {0, 0, 0};
    const at::Tensor* mods[3] = {nullptr, nullptr, nullptr};
    bool first = true;
    for (int i = 0; i < 3; ++i) {
        if (a.none(5 + i)) continue;
        const at::Tensor* t = mods[i] = a.strided(5 + i);
        if (!t || t->dim() != 3 || t->scalar_type() != type || t->size(2) != C) return nullptr;
        if (first) batches = t->size(0), groups = t->size(1);
        first = false;
        if (t->size(0) != batches || t->size(1) != groups || (batches != 1 && batches != B)) return nullptr;
        if (C > 1 && t->stride(2) != 1) return nullptr;
        if (batches * groups > 1) strides[i] = groups > 1 ? t->stride(1) : t->stride(0);
        if (batches > 1 && groups > 1 && t->stride(0) != groups * strides[i]) return nullptr;
    }
    const at::Tensor *gr = a.maybe(8, c1, type), *g = a.maybe(9, c1, type), *beta = a.maybe(10, c1, type);
    const float skip = a.real(11), eps = a.real(14);
    const long long norm_r = a.integer(12), norm = a.integer(13);
    void* s = a.stream_here(15);
    const int xcode = type_code(*x);
    const int code = type == c10::kHalf ? 0 : type == c10::kBFloat16 ? 1 : -1;
    if (!a.ok || code < 0 || xcode < 0 || !fits({B, L, C, groups})) return nullptr;
    return call(a.fn(), ptr(x), ptr(r), ptr(mods[0]), ptr(mods[1]), ptr(mods[2]), ptr(gr), ptr(g), ptr(beta), ptr(h), ptr(y),
                (int)B, (int)L, (int)C, (int)batches, (int)groups, (long long)strides[0], (long long)strides[1],
                (long long)strides[2], skip, (int)norm_r, (int)norm, eps, xcode, code, s);
}

// The cache's tensors from argument i on: k_pages, v_pages, k_scales, v_scales, table, starts
struct Cache {
    const at::Tensor *kp, *vp, *ks, *vs, *table, *starts;
    int64_t pages, Hk, slots;
};
bool cache_of(Args& a, Py_ssize_t i, int64_t B, int64_t D, Cache* c) {
    c->kp = a.tensor(i);
    if (!c->kp || c->kp->dim() != 4) return false;
    c->pages = c->kp->size(0), c->Hk = c->kp->size(1);
    const int64_t ps[] = {c->pages, c->Hk, 64, D}, ss[] = {c->pages, c->Hk}, b1[] = {B};
    for (Py_ssize_t j = 0; j < 2; ++j) {
        const at::Tensor* t = a.tensor(i + j);
        if (!t || t->sizes() != at::IntArrayRef(ps) || (t->scalar_type() != c10::kByte && t->scalar_type() != c10::kFloat8_e4m3fn))
            return false;
        (j ? c->vp : c->kp) = t;
    }
    c->ks = a.tensor(i + 2, ss, c10::kFloat);
    c->vs = a.tensor(i + 3, ss, c10::kFloat);
    c->table = a.tensor(i + 4);
    if (!a.ok || c->table->dim() != 2 || c->table->size(0) != B || c->table->scalar_type() != c10::kInt) return false;
    c->slots = c->table->size(1);
    c->starts = a.tensor(i + 5, b1, c10::kInt);
    return a.ok && fits({c->pages, c->Hk, c->slots});
}

// fn, k, v, k_pages, v_pages, k_scales, v_scales, table, starts, counts, layout, stream
template <bool WRITE>
PyObject* cache_call(Args& a) {
    const at::Tensor *k = a.tensor(1), *kp = a.tensor(3);
    const long long layout = a.integer(10);
    int64_t B, L, C;
    if (!a.ok || kp->dim() != 4 || kp->size(1) < 1 || !row_sizes(*k, layout, kp->size(1), &B, &L, &C) || C % kp->size(1))
        return nullptr;
    const int64_t D = C / kp->size(1), b1[] = {B};
    Cache c;
    if (!cache_of(a, 3, B, D, &c)) return nullptr;
    const at::Tensor *v = a.tensor(2, k->sizes(), k->scalar_type()), *counts = a.maybe(9, b1, c10::kInt);
    void* s = a.stream_here(11);
    const int code = type_code(*k);
    if (!a.ok || code < 0 || !fits({B, L, D})) return nullptr;
    if (WRITE)
        return call(a.fn(), ptr(k), ptr(v), ptr(c.kp), ptr(c.vp), ptr(c.ks), ptr(c.vs), ptr(c.table), ptr(c.starts),
                    ptr(counts), (int)B, (int)c.Hk, (int)L, (int)D, (int)c.pages, (int)c.slots, (int)layout, code, s);
    return call(a.fn(), ptr(c.kp), ptr(c.vp), ptr(c.ks), ptr(c.vs), ptr(c.table), ptr(c.starts), ptr(counts), ptr(k), ptr(v),
                (int)B, (int)c.Hk, (int)L, (int)D, (int)c.pages, (int)c.slots, (int)layout, code, s);
}
PyObject* cache_write(Args& a) { return cache_call<true>(a); }
PyObject* cache_read(Args& a) { return cache_call<false>(a); }

// the workspace: a tensor, or None (then no bytes)
bool workspace_of(Args& a, Py_ssize_t i, void** p, long long* bytes) {
    *p = nullptr, *bytes = 0;
    if (a.none(i)) return true;
    const at::Tensor* t = a.tensor(i);
    if (!t) return false;
    if (t->numel() > 0) *p = t->data_ptr(), *bytes = (long long)(t->numel() * t->element_size());
    return true;
}

// fn, q, k_pages, v_pages, k_scales, v_scales, table, starts, out, scale, heads, workspace, counts, frame, window,
// sinks, x_layout, y_layout, stream
PyObject* cache_forward(Args& a) {
    const at::Tensor *q = a.tensor(1), *out = a.tensor(8);
    const float scale = a.real(9);
    const long long H = a.integer(10), frame = a.integer(13), window = a.integer(14), sinks = a.integer(15),
                    xl = a.integer(16), yl = a.integer(17);
    int64_t B, L, C;
    if (!a.ok || H < 1 || !row_sizes(*q, xl, H, &B, &L, &C) || C % H) return nullptr;
    const int64_t D = C / H, b1[] = {B};
    Cache c;
    void* ws;
    long long nws;
    if (!cache_of(a, 2, B, D, &c) || !workspace_of(a, 11, &ws, &nws)) return nullptr;
    const at::Tensor* counts = a.maybe(12, b1, c10::kInt);
    void* s = a.stream_here(18);
    const int code = type_code(*q);
    if (!a.ok || code < 0 || !is_rows(out, yl, H, B, L, C, q->scalar_type()) || !fits({B, L, D})) return nullptr;
    return call(a.fn(), ptr(q), ptr(c.kp), ptr(c.vp), ptr(c.ks), ptr(c.vs), ptr(c.table), ptr(c.starts), ptr(counts), ptr(out),
                ws, nws, (int)B, (int)H, (int)c.Hk, (int)L, (int)D, (int)c.pages, (int)c.slots, (int)frame, (int)window,
                (int)sinks, scale, (int)xl, (int)yl, code, s);
}

// fn, q, k, v, out, scale, heads, kv_heads, workspace, starts, counts, frame, window, sinks, x_layout, y_layout, stream
PyObject* window_forward(Args& a) {
    const at::Tensor *q = a.tensor(1), *k = a.tensor(2), *out = a.tensor(4);
    const float scale = a.real(5);
    const long long H = a.integer(6), Hk = a.integer(7), frame = a.integer(11), window = a.integer(12), sinks = a.integer(13),
                    xl = a.integer(14), yl = a.integer(15);
    int64_t B, L, C, Bk, Lk, Ck;
    if (!a.ok || H < 1 || Hk < 1 || !row_sizes(*q, xl, H, &B, &L, &C) || C % H || !row_sizes(*k, xl, Hk, &Bk, &Lk, &Ck))
        return nullptr;
    const int64_t D = C / H, b1[] = {B};
    const auto type = q->scalar_type();
    if (Bk != B || Ck != Hk * D || k->scalar_type() != type) return nullptr;
    void* ws;
    long long nws;
    if (!workspace_of(a, 8, &ws, &nws)) return nullptr;
    const at::Tensor *v = a.tensor(3, k->sizes(), type), *starts = a.maybe(9, b1, c10::kInt),
                     *counts = a.maybe(10, b1, c10::kInt);
    void* s = a.stream_here(16);
    const int code = type_code(*q);
    if (!a.ok || code < 0 || !is_rows(out, yl, H, B, L, C, type) || !fits({B, L, Lk, D})) return nullptr;
    return call(a.fn(), ptr(q), ptr(k), ptr(v), ptr(starts), ptr(counts), ptr(out), ws, nws, (int)B, (int)H, (int)Hk, (int)L,
                (int)Lk, (int)D, (int)frame, (int)window, (int)sinks, scale, (int)xl, (int)yl, code, s);
}

PyObject* use_streams(PyObject*, PyObject* const* v, Py_ssize_t n) {
    if (n == 2) {
        Py_INCREF(v[0]);
        Py_INCREF(v[1]);
        current_device = v[0];
        current_stream = v[1];
    }
    Py_RETURN_NONE;
}

#define FAST(f) {#f, (PyCFunction)(void (*)(void))entry<f>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"use_streams", (PyCFunction)(void (*)(void))use_streams, METH_FASTCALL, nullptr},
                         FAST(forward), FAST(forward_ex), FAST(softmax_rows), FAST(logits), FAST(softmax_pv), FAST(attention_block),
                         FAST(attention_block_kv), FAST(group_norm), FAST(geglu), FAST(conv3x3),
                         FAST(linear_adapters), FAST(norm_rotate), FAST(block_means), FAST(select_blocks), FAST(sparse_forward),
                         FAST(gated_norm), FAST(cache_write), FAST(cache_read), FAST(cache_forward), FAST(window_forward),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__marshal(void) { return PyModule_Create(&module); }
