// Argument marshalling of the calls a serving loop makes eagerly, once per draft position and once per round
// (binding.py has the same in Python, which is the reference for what is accepted).  In Python the some forty
// attribute look-ups and the ctypes call of a draft step take about 10 us of host time, twice what its kernels run
// at small batches; here about 1 us.
//
// Every function returns the call's svip_status, or DECLINED without having done anything where an argument is not plainly
// right: the Python path then takes the call, or says what is wrong with it.  Nothing is kept between calls.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/svip.h"

namespace {

constexpr long DECLINED = -1;
decltype(&svip_draft_step) g_draft_step;
decltype(&svip_draft_step_greedy) g_draft_step_greedy;
decltype(&svip_verify) g_verify;
decltype(&svip_verify_greedy) g_verify_greedy;
decltype(&svip_quantize_blocks) g_quantize_blocks;
decltype(&svip_head_logits) g_head_logits;
decltype(&svip_quantize_mx) g_quantize_mx;
decltype(&svip_mx_rows) g_mx_rows;
decltype(&svip_head_logits_mx) g_head_logits_mx;
decltype(&svip_sample) g_sample;

// A plain dense device tensor, or nullptr: no subclass, nothing wrapped by a transform (those have no pointer to give).
const at::Tensor *device_tensor(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    const c10::TensorImpl *impl = t.unsafeGetTensorImpl();
    const c10::DispatchKeySet keys = impl->key_set();
    constexpr c10::DispatchKeySet wrapped = c10::DispatchKeySet(
        {c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize,
         c10::DispatchKey::Python, c10::DispatchKey::PythonTLSSnapshot, c10::DispatchKey::Conjugate, c10::DispatchKey::Negative,
         c10::DispatchKey::ZeroTensor});
    if (!keys.has_all(c10::DispatchKeySet(c10::DispatchKey::CUDA)) || keys.has_any(wrapped) || !impl->has_storage() ||
        impl->has_symbolic_sizes_strides())
        return nullptr;
    return &t;
}

int dtype_of(const at::Tensor &t)
{
    switch (t.scalar_type()) {
        case at::kFloat: return SVIP_F32;
        case at::kBFloat16: return SVIP_BF16;
        case at::kHalf: return SVIP_F16;
        default: return -1;
    }
}

// Reads arguments one after the other; `ok` turns false at the first that is not plainly right.
struct Args {
    PyObject *const *v;
    bool ok = true;
    int i = 0;

    const at::Tensor *logits(int dims, int *dtype)
    {
        const at::Tensor *t = device_tensor(v[i++]);
        if (!t || t->dim() != dims || t->stride(dims - 1) != 1 || (*dtype = dtype_of(*t)) < 0) {
            ok = false;
            return nullptr;
        }
        return t;
    }
    // [B], [B, k]: contiguous, of the given type; None (if optional) gives nullptr
    template <typename T>
    T *array(at::ScalarType type, bool optional, long long B, long long k = -1)
    {
        PyObject *o = v[i++];
        if (!ok) return nullptr;
        if (o == Py_None && optional) return nullptr;
        const at::Tensor *t = device_tensor(o);
        if (!t || t->scalar_type() != type || t->dim() != (k < 0 ? 1 : 2) || t->size(0) != B || (k >= 0 && t->size(1) != k) ||
            !t->is_contiguous()) {
            ok = false;
            return nullptr;
        }
        return static_cast<T *>(t->data_ptr());
    }
    // [B], possibly a column of a larger array; all of a call's share one stride (-1: none seen yet)
    template <typename T>
    T *column(at::ScalarType type, bool optional, long long B, long long *stride)
    {
        PyObject *o = v[i++];
        if (!ok) return nullptr;
        if (o == Py_None && optional) return nullptr;
        const at::Tensor *t = device_tensor(o);
        if (!t || t->scalar_type() != type || t->dim() != 1 || t->size(0) != B || (B > 1 && (t->stride(0) == 0 || (*stride >= 0 && t->stride(0) != *stride)))) {
            ok = false;
            return nullptr;
        }
        if (*stride < 0) *stride = B > 1 ? t->stride(0) : 1;
        return static_cast<T *>(t->data_ptr());
    }
    // A matrix with unit stride along its rows on the current device; *stride: between its rows.
    const at::Tensor *matrix(at::ScalarType type, long long rows, long long cols, long long *stride)
    {
        const at::Tensor *t = device_tensor(v[i++]);
        if (!t || t->dim() != 2 || (type != at::ScalarType::Undefined && t->scalar_type() != type) || (rows >= 0 && t->size(0) != rows) ||
            (cols >= 0 && t->size(1) != cols) || t->stride(1) != 1 || t->device().index() != c10::hip::current_device()) {
            ok = false;
            return nullptr;
        }
        *stride = t->size(0) > 1 ? t->stride(0) : (t->size(1) + 15) / 16 * 16;       // (of one row there is none: any that is aligned)
        return t;
    }
    // A 4-bit matrix [rows, cols / 2], rows and cols of any size where negative, and its scales, which come next
    const at::Tensor *mx(long long rows, long long cols, long long *stride, const at::Tensor **scale, long long *scale_stride)
    {
        const at::Tensor *q = matrix(at::ScalarType::Float4_e2m1fn_x2, rows, cols < 0 ? cols : cols / 2, stride);
        *scale = ok ? matrix(at::kFloat8_e8m0fnu, q->size(0), q->size(1) / 16, scale_stride) : nullptr;
        return q;
    }
    const at::Tensor *workspace()
    {
        const at::Tensor *t = device_tensor(v[i++]);
        if (!t || t->scalar_type() != at::kByte) ok = false;
        return t;
    }
    float real()
    {
        PyObject *o = v[i++];
        if (PyFloat_CheckExact(o)) return (float)PyFloat_AS_DOUBLE(o);
        return (float)whole();
    }
    int whole(bool again = true)
    {
        PyObject *o = v[again ? i - 1 : i++];
        int over = 0;
        const long n = PyLong_CheckExact(o) ? PyLong_AsLongAndOverflow(o, &over) : 0;
        if (!PyLong_CheckExact(o) || over || n < INT32_MIN || n > INT32_MAX) ok = false;
        return (int)n;
    }
    void *stream()          // None: the current one; otherwise its handle
    {
        PyObject *o = v[i++];
        if (o == Py_None) return c10::hip::getCurrentHIPStream().stream();
        if (!PyLong_CheckExact(o)) {
            ok = false;
            return nullptr;
        }
        void *p = PyLong_AsVoidPtr(o);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            ok = false;
        }
        return p;
    }
};

bool fits(long long n) { return n >= 0 && n <= INT32_MAX; }

template <typename F>
PyObject *answer(F f)
{
    long status = DECLINED;
    try {
        status = f();
    } catch (const std::exception &) {       // (a tensor without a pointer to give)
        status = DECLINED;
    }
    return PyLong_FromLong(status);
}

// draft_step(draft_logits, temperature, h, step_j, k_max, u_sample or None for greedy, token_out, entropy_out, q_tok_out, lse_out,
//            stop_in, stop_out, draft_len_out, workspace, stream)
PyObject *draft_step(PyObject *, PyObject *const *argv, Py_ssize_t n)
{
    return answer([&]() -> long {
        if (n != 15) return DECLINED;
        Args a{argv};
        int dtype = -1;
        const at::Tensor *z = a.logits(2, &dtype);
        if (!a.ok) return DECLINED;
        const long long B = z->size(0), V = z->size(1), s0 = z->stride(0), row_stride = B > 1 ? s0 : (V > s0 ? V : s0);
        const float temperature = a.real(), h = a.real();
        const int step_j = a.whole(false), k_max = a.whole(false);
        const bool greedy = argv[5] == Py_None;
        long long stride = -1;
        const float *u = a.column<float>(at::kFloat, true, B, &stride);
        int *token = a.column<int>(at::kInt, false, B, &stride);
        float *entropy = a.column<float>(at::kFloat, true, B, &stride), *q_tok = a.column<float>(at::kFloat, true, B, &stride);
        double *lse = a.column<double>(at::kDouble, false, B, &stride);
        const unsigned char *stop_in = a.array<unsigned char>(at::kByte, true, B);
        unsigned char *stop_out = a.array<unsigned char>(at::kByte, false, B);
        int *draft_len = a.array<int>(at::kInt, true, B);
        const at::Tensor *ws = a.workspace();
        void *stream = a.stream();
        if (!a.ok || !fits(B) || !fits(V)) return DECLINED;
        const void *logits = z->data_ptr();
        void *wp = ws->data_ptr();
        const size_t wn = (size_t)ws->numel();
        long status;
        Py_BEGIN_ALLOW_THREADS
        status = greedy ? g_draft_step_greedy(logits, dtype, (int)B, (int)V, row_stride, temperature, h, step_j, k_max, stop_in, token, entropy,
                                              q_tok, lse, stop_out, draft_len, stride, wp, wn, stream)
                        : g_draft_step(logits, dtype, (int)B, (int)V, row_stride, temperature, h, step_j, k_max, u, stop_in, token, entropy,
                                       q_tok, lse, stop_out, draft_len, stride, wp, wn, stream);
        Py_END_ALLOW_THREADS
        return status;
    });
}

// verify(target_logits, draft_logits, temperature, draft_tokens, draft_len, draft_lse, u_accept, u_resample, n_accepted_out,
//        next_token_out, accept_prob_out, workspace, stream)
PyObject *verify(PyObject *, PyObject *const *argv, Py_ssize_t n)
{
    return answer([&]() -> long {
        if (n != 13) return DECLINED;
        Args a{argv};
        int dtype = -1, dtype_q = -1;
        const at::Tensor *p = a.logits(3, &dtype), *q = a.logits(3, &dtype_q);
        if (!a.ok || dtype != dtype_q) return DECLINED;
        const long long B = p->size(0), k = p->size(1) - 1, V = p->size(2), row_stride = p->stride(1);
        if (q->size(0) != B || q->size(1) != k || q->size(2) != V || (k > 1 && q->stride(1) != row_stride)) return DECLINED;
        const long long seq_t = B > 1 ? p->stride(0) : (k + 1) * row_stride, seq_d = B > 1 ? q->stride(0) : k * row_stride;
        const float temperature = a.real();
        const int *tokens = a.array<int>(at::kInt, false, B, k), *len = a.array<int>(at::kInt, false, B);
        const double *lse = a.array<double>(at::kDouble, true, B, k);
        const float *ua = a.array<float>(at::kFloat, false, B, k), *ur = a.array<float>(at::kFloat, false, B);
        int *nacc = a.array<int>(at::kInt, false, B), *next = a.array<int>(at::kInt, false, B);
        float *prob = a.array<float>(at::kFloat, true, B, k);
        const at::Tensor *ws = a.workspace();
        void *stream = a.stream();
        if (!a.ok || !fits(B) || !fits(k) || !fits(V)) return DECLINED;
        const void *pp = p->data_ptr(), *qp = q->data_ptr();
        void *wp = ws->data_ptr();
        const size_t wn = (size_t)ws->numel();
        long status;
        Py_BEGIN_ALLOW_THREADS
        status = g_verify(pp, qp, dtype, (int)B, (int)k, (int)V, seq_t, seq_d, row_stride, temperature, tokens, len, lse, ua, ur, nacc, next,
                          prob, wp, wn, stream);
        Py_END_ALLOW_THREADS
        return status;
    });
}

// verify_greedy(target_logits, draft_tokens, draft_len, n_accepted_out, next_token_out, workspace, stream)
PyObject *verify_greedy(PyObject *, PyObject *const *argv, Py_ssize_t n)
{
    return answer([&]() -> long {
        if (n != 7) return DECLINED;
        Args a{argv};
        int dtype = -1;
        const at::Tensor *p = a.logits(3, &dtype);
        if (!a.ok) return DECLINED;
        const long long B = p->size(0), k = p->size(1) - 1, V = p->size(2), row_stride = p->stride(1);
        const long long seq_t = B > 1 ? p->stride(0) : (k + 1) * row_stride;
        if (!fits(k)) return DECLINED;
        const int *tokens = a.array<int>(at::kInt, false, B, k), *len = a.array<int>(at::kInt, false, B);
        int *nacc = a.array<int>(at::kInt, false, B), *next = a.array<int>(at::kInt, false, B);
        const at::Tensor *ws = a.workspace();
        void *stream = a.stream();
        if (!a.ok || !fits(B) || !fits(V)) return DECLINED;
        const void *pp = p->data_ptr();
        void *wp = ws->data_ptr();
        const size_t wn = (size_t)ws->numel();
        long status;
        Py_BEGIN_ALLOW_THREADS
        status = g_verify_greedy(pp, dtype, (int)B, (int)k, (int)V, seq_t, row_stride, tokens, len, nacc, next, wp, wn, stream);
        Py_END_ALLOW_THREADS
        return status;
    });
}

// quantize_blocks(x, block_rows, q_out, scale_out, stream)
PyObject *quantize_blocks(PyObject *, PyObject *const *argv, Py_ssize_t n)
{
    return answer([&]() -> long {
        if (n != 5) return DECLINED;
        Args a{argv};
        long long sx = 0, sq = 0, ss = 0;
        const at::Tensor *x = a.matrix(at::ScalarType::Undefined, -1, -1, &sx);
        if (!a.ok) return DECLINED;
        const int dtype = dtype_of(*x), block_rows = a.whole(false);
        const long long rows = x->size(0), cols = x->size(1), kb = (cols + 127) / 128;
        if (dtype < 0 || (block_rows != 1 && block_rows != 128)) return DECLINED;
        const at::Tensor *q = a.matrix(at::kFloat8_e4m3fn, rows, kb * 128, &sq);
        const at::Tensor *s = a.matrix(at::kFloat8_e8m0fnu, (rows + block_rows - 1) / block_rows, kb, &ss);
        void *stream = a.stream();
        if (!a.ok || !fits(rows) || !fits(cols)) return DECLINED;
        const void *xp = x->data_ptr();
        void *qp = q->data_ptr(), *sp = s->data_ptr();
        long status;
        Py_BEGIN_ALLOW_THREADS
        status = g_quantize_blocks(xp, dtype, (int)rows, (int)cols, sx, block_rows, qp, sq, sp, ss, stream);
        Py_END_ALLOW_THREADS
        return status;
    });
}

// head_logits(hidden_q, hidden_scale, weight_q, weight_scale, logits_out, workspace, stream)
PyObject *head_logits(PyObject *, PyObject *const *argv, Py_ssize_t n)
{
    return answer([&]() -> long {
        if (n != 7) return DECLINED;
        Args a{argv};
        long long sh = 0, shs = 0, sw = 0, sws = 0, so = 0;
        const at::Tensor *h = a.matrix(at::kFloat8_e4m3fn, -1, -1, &sh);
        if (!a.ok) return DECLINED;
        const long long N = h->size(0), K = h->size(1);
        const at::Tensor *hs = a.matrix(at::kFloat8_e8m0fnu, N, K / 128, &shs), *w = a.matrix(at::kFloat8_e4m3fn, -1, K, &sw);
        if (!a.ok) return DECLINED;
        const long long V = w->size(0);
        const at::Tensor *ws = a.matrix(at::kFloat8_e8m0fnu, (V + 127) / 128, K / 128, &sws), *out = a.matrix(at::ScalarType::Undefined, N, V, &so);
        const at::Tensor *space = a.workspace();
        void *stream = a.stream();
        if (!a.ok || !fits(N) || !fits(V) || !fits(K) || space->device() != h->device()) return DECLINED;
        const int dtype = dtype_of(*out);
        if (dtype < 0) return DECLINED;
        const void *hp = h->data_ptr(), *hsp = hs->data_ptr(), *wp = w->data_ptr(), *wsp = ws->data_ptr();
        void *op = out->data_ptr(), *sp = space->data_ptr();
        const size_t sn = (size_t)space->numel();
        long status;
        Py_BEGIN_ALLOW_THREADS
        status = g_head_logits(hp, hsp, wp, wsp, (int)N, (int)V, (int)K, sh, shs, sw, sws, op, dtype, so, sp, sn, stream);
        Py_END_ALLOW_THREADS
        return status;
    });
}

// quantize_mx(x, q_out, scale_out, stream)
PyObject *quantize_mx(PyObject *, PyObject *const *argv, Py_ssize_t n)
{
    return answer([&]() -> long {
        if (n != 4) return DECLINED;
        Args a{argv};
        long long sx = 0, sq = 0, ss = 0;
        const at::Tensor *x = a.matrix(at::ScalarType::Undefined, -1, -1, &sx);
        if (!a.ok) return DECLINED;
        const int dtype = dtype_of(*x);
        const long long rows = x->size(0), cols = x->size(1);
        const at::Tensor *s = nullptr, *q = a.mx(rows, (cols + 127) / 128 * 128, &sq, &s, &ss);
        if (!a.ok) return DECLINED;
        void *stream = a.stream();
        if (!a.ok || dtype < 0 || !fits(rows) || !fits(cols)) return DECLINED;
        const void *xp = x->data_ptr();
        void *qp = q->data_ptr(), *sp = s->data_ptr();
        long status;
        Py_BEGIN_ALLOW_THREADS
        status = g_quantize_mx(xp, dtype, (int)rows, (int)cols, sx, qp, sq, sp, ss, stream);
        Py_END_ALLOW_THREADS
        return status;
    });
}

// mx_rows(q, scale, ids or None, out, stream)
PyObject *mx_rows(PyObject *, PyObject *const *argv, Py_ssize_t n)
{
    return answer([&]() -> long {
        if (n != 5) return DECLINED;
        Args a{argv};
        long long sq = 0, ss = 0, so = 0;
        const at::Tensor *s = nullptr, *q = a.mx(-1, -1, &sq, &s, &ss);
        if (!a.ok) return DECLINED;
        const at::Tensor *ids = argv[a.i] == Py_None ? nullptr : device_tensor(argv[a.i]);
        if (argv[a.i++] != Py_None && (!ids || ids->scalar_type() != at::kInt || ids->dim() != 1 || !ids->is_contiguous())) return DECLINED;
        const at::Tensor *out = a.matrix(at::ScalarType::Undefined, ids ? ids->size(0) : -1, -1, &so);
        if (!a.ok) return DECLINED;
        const int dtype = dtype_of(*out);
        const long long rows = q->size(0), count = out->size(0), cols = out->size(1);
        void *stream = a.stream();
        if (!a.ok || dtype < 0 || !fits(rows) || !fits(count) || !fits(cols) || (cols + 127) / 128 * 128 != 2 * q->size(1) ||
            (ids && ids->device() != q->device()))
            return DECLINED;
        const void *qp = q->data_ptr(), *sp = s->data_ptr();
        const int *ip = ids ? static_cast<const int *>(ids->data_ptr()) : nullptr;
        void *op = out->data_ptr();
        long status;
        Py_BEGIN_ALLOW_THREADS
        status = g_mx_rows(qp, sp, (int)rows, (int)cols, sq, ss, ip, (int)count, op, dtype, so, stream);
        Py_END_ALLOW_THREADS
        return status;
    });
}

// head_logits_mx(hidden_q, hidden_scale, weight_q, weight_scale, logits_out, workspace, stream)
PyObject *head_logits_mx(PyObject *, PyObject *const *argv, Py_ssize_t n)
{
    return answer([&]() -> long {
        if (n != 7) return DECLINED;
        Args a{argv};
        long long sh = 0, shs = 0, sw = 0, sws = 0, so = 0;
        const at::Tensor *first = device_tensor(argv[0]);
        if (!first) return DECLINED;
        const int bits = first->scalar_type() == at::ScalarType::Float4_e2m1fn_x2 ? 4 : first->scalar_type() == at::kFloat8_e4m3fn ? 8 : 0;
        if (!bits) return DECLINED;
        const at::Tensor *h = a.matrix(first->scalar_type(), -1, -1, &sh);
        if (!a.ok) return DECLINED;
        const long long N = h->size(0), K = h->size(1) * 8 / bits;
        const at::Tensor *hs = a.matrix(at::kFloat8_e8m0fnu, N, bits == 4 ? K / 32 : K / 128, &shs), *ws = nullptr;
        if (!a.ok) return DECLINED;
        const at::Tensor *w = a.mx(-1, K, &sw, &ws, &sws);
        if (!a.ok) return DECLINED;
        const long long V = w->size(0);
        const at::Tensor *out = a.matrix(at::ScalarType::Undefined, N, V, &so);
        const at::Tensor *space = a.workspace();
        void *stream = a.stream();
        if (!a.ok || !fits(N) || !fits(V) || !fits(K) || space->device() != h->device()) return DECLINED;
        const int dtype = dtype_of(*out);
        if (dtype < 0 || (bits == 8 && dtype == SVIP_F32)) return DECLINED;
        const void *hp = h->data_ptr(), *hsp = hs->data_ptr(), *wp = w->data_ptr(), *wsp = ws->data_ptr();
        void *op = out->data_ptr(), *sp = space->data_ptr();
        const size_t sn = (size_t)space->numel();
        long status;
        Py_BEGIN_ALLOW_THREADS
        status = g_head_logits_mx(hp, hsp, bits, wp, wsp, (int)N, (int)V, (int)K, sh, shs, sw, sws, op, dtype, so, sp, sn, stream);
        Py_END_ALLOW_THREADS
        return status;
    });
}

// sample(logits, u, temperature, top_k, top_p, min_p, token_out, prob_out, kept_out, workspace, stream), settings, prob_out and kept_out each or None
PyObject *sample(PyObject *, PyObject *const *argv, Py_ssize_t n)
{
    return answer([&]() -> long {
        if (n != 11) return DECLINED;
        Args a{argv};
        long long sz = 0;
        const at::Tensor *z = a.matrix(at::ScalarType::Undefined, -1, -1, &sz);
        if (!a.ok) return DECLINED;
        const int dtype = dtype_of(*z);
        const long long N = z->size(0), V = z->size(1);
        const float *u = a.array<float>(at::kFloat, false, N), *T = a.array<float>(at::kFloat, true, N);
        const int *k = a.array<int>(at::kInt, true, N);
        const float *p = a.array<float>(at::kFloat, true, N), *m = a.array<float>(at::kFloat, true, N);
        int *token = a.array<int>(at::kInt, false, N);
        float *prob = a.array<float>(at::kFloat, true, N);
        int *kept = a.array<int>(at::kInt, true, N);
        const at::Tensor *space = a.workspace();
        void *stream = a.stream();
        if (!a.ok || dtype < 0 || !fits(N) || !fits(V)) return DECLINED;
        for (int i = 1; i < 10; ++i)
            if (argv[i] != Py_None && device_tensor(argv[i])->device() != z->device()) return DECLINED;
        const void *zp = z->data_ptr();
        void *sp = space->data_ptr();
        const size_t sn = (size_t)space->numel();
        long status;
        Py_BEGIN_ALLOW_THREADS
        status = g_sample(zp, dtype, (int)N, (int)V, sz, T, k, p, m, u, token, prob, kept, sp, sn, stream);
        Py_END_ALLOW_THREADS
        return status;
    });
}

// bind(addresses of svip_draft_step, svip_draft_step_greedy, svip_verify, svip_verify_greedy, svip_quantize_blocks, svip_head_logits,
//      svip_quantize_mx, svip_mx_rows, svip_head_logits_mx, svip_sample)
PyObject *bind(PyObject *, PyObject *const *argv, Py_ssize_t n)
{
    void *f[10];
    if (n != 10) {
        PyErr_SetString(PyExc_TypeError, "bind takes ten addresses");
        return nullptr;
    }
    for (int i = 0; i < 10; ++i) {
        f[i] = PyLong_AsVoidPtr(argv[i]);
        if (!f[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: a null address");
            return nullptr;
        }
    }
    g_draft_step = reinterpret_cast<decltype(g_draft_step)>(f[0]);
    g_draft_step_greedy = reinterpret_cast<decltype(g_draft_step_greedy)>(f[1]);
    g_verify = reinterpret_cast<decltype(g_verify)>(f[2]);
    g_verify_greedy = reinterpret_cast<decltype(g_verify_greedy)>(f[3]);
    g_quantize_blocks = reinterpret_cast<decltype(g_quantize_blocks)>(f[4]);
    g_head_logits = reinterpret_cast<decltype(g_head_logits)>(f[5]);
    g_quantize_mx = reinterpret_cast<decltype(g_quantize_mx)>(f[6]);
    g_mx_rows = reinterpret_cast<decltype(g_mx_rows)>(f[7]);
    g_head_logits_mx = reinterpret_cast<decltype(g_head_logits_mx)>(f[8]);
    g_sample = reinterpret_cast<decltype(g_sample)>(f[9]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind)), METH_FASTCALL, nullptr},
    {"draft_step", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(draft_step)), METH_FASTCALL, nullptr},
    {"verify", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(verify)), METH_FASTCALL, nullptr},
    {"verify_greedy", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(verify_greedy)), METH_FASTCALL, nullptr},
    {"quantize_blocks", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(quantize_blocks)), METH_FASTCALL, nullptr},
    {"head_logits", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(head_logits)), METH_FASTCALL, nullptr},
    {"quantize_mx", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(quantize_mx)), METH_FASTCALL, nullptr},
    {"mx_rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(mx_rows)), METH_FASTCALL, nullptr},
    {"head_logits_mx", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(head_logits_mx)), METH_FASTCALL, nullptr},
    {"sample", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(sample)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "native argument marshalling of binding.py", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
