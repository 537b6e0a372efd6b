// The linear calls of binding.py, and those of a token's way between linears, in one native step: checks on the tensors, the output, the current stream and the library
// call.  One token through a 512 -> 512 linear, called eagerly, is bound by the host: in Python the same steps took 3.4 us beside
// the 3.3 of the call itself (the output alone 1.7, the checks of rows and strides 0.5, the stream's handle 0.4).
#include <Python.h>
#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "paro.h"

namespace {

// The ctypes classes of the structures (binding.py hands them over once).
PyObject *g_rotation, *g_weight, *g_rope, *g_cache;

// A ctypes structure of class `type` through the buffer protocol; NULL with an exception set if it is anything else.
template <class T>
const T *structure(PyObject *o, PyObject *type)
{
    if (!type || !PyObject_TypeCheck(o, (PyTypeObject *)type)) {
        PyErr_SetString(PyExc_TypeError, "not the structure that this call takes");
        return nullptr;
    }
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) return nullptr;
    const void *p = view.buf;
    PyBuffer_Release(&view);                          // the caller's reference keeps the structure
    return (const T *)p;
}

PyObject *keep_types(PyObject *const *a, Py_ssize_t n, PyObject *&first, PyObject *&second)
{
    if (n != 2 || !PyType_Check(a[0]) || !PyType_Check(a[1])) { PyErr_SetString(PyExc_TypeError, "types takes two classes"); return nullptr; }
    Py_INCREF(a[0]); Py_INCREF(a[1]);
    Py_XDECREF(first); Py_XDECREF(second);
    first = a[0]; second = a[1];
    Py_RETURN_NONE;
}
PyObject *types(PyObject *, PyObject *const *a, Py_ssize_t n) { return keep_types(a, n, g_rotation, g_weight); }
PyObject *token_types(PyObject *, PyObject *const *a, Py_ssize_t n) { return keep_types(a, n, g_rope, g_cache); }

const at::Tensor *tensor(PyObject *o)
{
    if (THPVariable_Check(o)) return &THPVariable_Unpack(o);
    PyErr_SetString(PyExc_TypeError, "expected a tensor");
    return nullptr;
}

// fp16 rows; false with an exception set for anything else
bool rows(const at::Tensor &t)
{
    if (t.scalar_type() == at::kHalf && t.dim() == 2 && t.stride(1) == 1) return true;
    PyErr_SetString(PyExc_AssertionError, "expected a 2-D float16 tensor with contiguous rows");
    return false;
}

// X, Y or None -> the output; undefined with an exception set on failure
at::Tensor output(const at::Tensor &x, PyObject *y, int64_t width)
{
    if (y == Py_None) return at::empty({x.size(0), width}, x.options().requires_grad(false));
    const at::Tensor *t = tensor(y);
    return t && rows(*t) ? *t : at::Tensor();
}

// The result: the output, or the status of a call that was refused.
PyObject *result(paro_status st, PyObject *y, at::Tensor &&out)
{
    if (st != PARO_OK) return PyLong_FromLong(st);
    if (y != Py_None) { Py_INCREF(y); return y; }
    return THPVariable_Wrap(std::move(out));
}

// linear(rotation or None, weight, c_out, X, Y or None, workspace or None, bytes)
PyObject *linear(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 7) { PyErr_SetString(PyExc_TypeError, "linear takes 7 arguments"); return nullptr; }
    const paro_rotation *rot = a[0] == Py_None ? nullptr : structure<paro_rotation>(a[0], g_rotation);
    if (!rot && a[0] != Py_None) return nullptr;
    const paro_w4_weight *w = structure<paro_w4_weight>(a[1], g_weight);
    if (!w) return nullptr;
    const int64_t c_out = PyLong_AsLongLong(a[2]);
    const at::Tensor *x = tensor(a[3]);
    if (!x || !rows(*x)) return nullptr;
    const at::Tensor *ws = a[5] == Py_None ? nullptr : tensor(a[5]);
    if (!ws && a[5] != Py_None) return nullptr;
    const size_t bytes = PyLong_AsSize_t(a[6]);
    if (PyErr_Occurred()) return nullptr;
    at::Tensor out = output(*x, a[4], c_out);
    if (!out.defined()) return nullptr;
    const paro_half_t *xp = (const paro_half_t *)x->data_ptr();
    paro_half_t *yp = (paro_half_t *)out.data_ptr();
    void *wp = ws ? ws->data_ptr() : nullptr, *stream = (void *)c10::hip::getCurrentHIPStream().stream();
    const int64_t ldx = x->stride(0), ldy = out.stride(0);
    const int32_t T = (int32_t)x->size(0);
    paro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = rot ? paro_rotated_linear(rot, w, xp, ldx, yp, ldy, T, wp, bytes, stream) : paro_w4a16_linear(w, xp, ldx, yp, ldy, T, wp, bytes, stream);
    Py_END_ALLOW_THREADS
    return result(st, a[4], std::move(out));
    END_HANDLE_TH_ERRORS
}

// rotate(rotation, c_in, X, Xr or None)
PyObject *rotate(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 4) { PyErr_SetString(PyExc_TypeError, "rotate takes 4 arguments"); return nullptr; }
    const paro_rotation *rot = structure<paro_rotation>(a[0], g_rotation);
    if (!rot) return nullptr;
    const int64_t c_in = PyLong_AsLongLong(a[1]);
    const at::Tensor *x = tensor(a[2]);
    if (!x || !rows(*x) || PyErr_Occurred()) return nullptr;
    at::Tensor out = output(*x, a[3], c_in);
    if (!out.defined()) return nullptr;
    const paro_half_t *xp = (const paro_half_t *)x->data_ptr();
    paro_half_t *yp = (paro_half_t *)out.data_ptr();
    void *stream = (void *)c10::hip::getCurrentHIPStream().stream();
    const int64_t ldx = x->stride(0), ldy = out.stride(0);
    const int32_t T = (int32_t)x->size(0);
    paro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = paro_rotate_scale(rot, xp, ldx, yp, ldy, T, stream);
    Py_END_ALLOW_THREADS
    return result(st, a[3], std::move(out));
    END_HANDLE_TH_ERRORS
}

// ---- Between the linears ---------------------------------------------------------------------------------------------

bool refuse(const char *why)
{
    PyErr_SetString(PyExc_AssertionError, why);
    return false;
}

// A call's tensors, its cache and its frequencies are on the GPU of its first tensor, and that GPU is the current one: the
// kernels go to the current stream and follow the pointers of all.
struct RopeOn { paro_rope_t c; int32_t device; };               // _CRope, _CKVCache: -1 in host memory
struct CacheOn { paro_kv_cache c; int32_t device; };
bool same_gpu(int device, const at::Tensor &first) { return device == first.device().index() || refuse("expected tensors, cache and frequencies on one GPU"); }
bool on_gpu(const at::Tensor &x, const at::Tensor &first)
{
    if (!x.is_cuda()) return refuse("expected a tensor on the GPU");
    return same_gpu(x.device().index(), first);
}
bool current(const at::Tensor &first) { return first.device().index() == c10::hip::current_device() || refuse("the tensors' GPU is not the current one"); }

// fp16 rows of `width` channels on the GPU of `first`; `t` tokens (-1: any)
bool gpu_rows(const at::Tensor &x, int64_t t, int64_t width, const at::Tensor &first)
{
    if (!rows(x) || !on_gpu(x, first)) return false;
    if (x.size(0) > INT32_MAX) return refuse("more rows than 32 bits count");
    if ((t >= 0 && x.size(0) != t) || x.size(1) != width) return refuse("tensors of different shapes");
    return true;
}
bool gpu_vector(const at::Tensor &x, at::ScalarType type, int64_t n, const at::Tensor &first)
{
    if (x.scalar_type() != type || x.dim() != 1 || !x.is_contiguous() || x.size(0) != n) return refuse("expected a contiguous vector of another type or length");
    return on_gpu(x, first);
}
// A number of 32 bits; false with an exception set if it is none.
bool number(PyObject *o, int32_t &to)
{
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) return false;
    to = (int32_t)x;
    return to == x || refuse("a number beyond 32 bits");
}
// An optional tensor argument; false with an exception set if it is anything else.
bool maybe(PyObject *o, const at::Tensor *&t)
{
    t = nullptr;
    return o == Py_None || (t = tensor(o));
}
// A new dense tensor where `like` is (the current GPU), from the allocator that `like` came from: 0.3 us of host time, 0.85 by way of the dispatcher.
at::Tensor fresh(const at::Tensor &like, at::IntArrayRef sizes, at::ScalarType type)
{
    c10::Allocator *allocator = like.storage().allocator();
    if (!allocator) return at::empty(sizes, like.options().dtype(type).requires_grad(false));
    return at::Tensor(at::detail::empty_generic(sizes, allocator, c10::DispatchKeySet(c10::DispatchKey::CUDA), type, std::nullopt));
}
// `o` if given, else new rows; undefined with an exception set on failure
at::Tensor rows_or_new(PyObject *o, int64_t t, int64_t width, const at::Tensor &like)
{
    if (o == Py_None) return fresh(like, {t, width}, at::kHalf);
    const at::Tensor *x = tensor(o);
    return x && gpu_rows(*x, t, width, like) ? *x : at::Tensor();
}
const paro_half_t *half_ptr(const at::Tensor *t) { return t ? (const paro_half_t *)t->data_ptr() : nullptr; }
paro_half_t *half_out(const at::Tensor &t) { return (paro_half_t *)t.data_ptr(); }
void *current_stream() { return (void *)c10::hip::getCurrentHIPStream().stream(); }
PyObject *wrap(PyObject *given, at::Tensor &&t)
{
    if (given != Py_None) { Py_INCREF(given); return given; }
    return THPVariable_Wrap(std::move(t));
}
PyObject *together(std::initializer_list<PyObject *> parts)
{
    PyObject *out = PyTuple_New((Py_ssize_t)parts.size());
    Py_ssize_t i = 0;
    for (PyObject *p : parts) {
        if (!p || !out) { Py_XDECREF(p); continue; }
        PyTuple_SET_ITEM(out, i++, p);
    }
    if (out && i == (Py_ssize_t)parts.size()) return out;
    Py_XDECREF(out);
    return nullptr;
}

// rms_norm(X, weight, eps, residual or None, Y or None, H or None) -> Y, or (Y, H) with a residual
PyObject *rms_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 6) { PyErr_SetString(PyExc_TypeError, "rms_norm takes 6 arguments"); return nullptr; }
    const at::Tensor *x = tensor(a[0]), *w = x ? tensor(a[1]) : nullptr, *r;
    if (!w || !rows(*x) || !gpu_rows(*x, -1, x->size(1), *x) || !gpu_vector(*w, at::kHalf, x->size(1), *x)) return nullptr;
    const float eps = (float)PyFloat_AsDouble(a[2]);
    const int64_t T = x->size(0), C = x->size(1);
    if (PyErr_Occurred() || !maybe(a[3], r) || (r && !gpu_rows(*r, T, C, *x)) || !current(*x)) return nullptr;
    if (!r && a[5] != Py_None) { refuse("H takes the sum with a residual"); return nullptr; }
    at::Tensor y = rows_or_new(a[4], T, C, *x), h;
    if (!y.defined()) return nullptr;
    if (r && !(h = rows_or_new(a[5], T, C, *x)).defined()) return nullptr;
    void *stream = current_stream();
    paro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = paro_rms_norm(half_ptr(x), x->stride(0), half_ptr(r), r ? r->stride(0) : 0, half_ptr(w), eps, (int32_t)T, (int32_t)C,
                       r ? half_out(h) : nullptr, r ? h.stride(0) : 0, half_out(y), y.stride(0), stream);
    Py_END_ALLOW_THREADS
    if (st != PARO_OK) return PyLong_FromLong(st);
    PyObject *first = wrap(a[4], std::move(y));
    return r ? together({first, wrap(a[5], std::move(h))}) : first;
    END_HANDLE_TH_ERRORS
}

// rms_norm_quantize_e4m3(X, weight, eps, group, residual or None, H or None) -> (codes, scales), or (codes, scales, H) with a residual
PyObject *rms_norm_quantize_e4m3(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 6) { PyErr_SetString(PyExc_TypeError, "rms_norm_quantize_e4m3 takes 6 arguments"); return nullptr; }
    const at::Tensor *x = tensor(a[0]), *w = x ? tensor(a[1]) : nullptr, *r;
    if (!w || !rows(*x) || !gpu_rows(*x, -1, x->size(1), *x) || !gpu_vector(*w, at::kHalf, x->size(1), *x)) return nullptr;
    const float eps = (float)PyFloat_AsDouble(a[2]);
    int32_t group;
    const int64_t T = x->size(0), C = x->size(1);
    if (PyErr_Occurred() || !number(a[3], group) || !maybe(a[4], r) || (r && !gpu_rows(*r, T, C, *x)) || !current(*x)) return nullptr;
    if (!r && a[5] != Py_None) { refuse("H takes the sum with a residual"); return nullptr; }
    at::Tensor h;
    if (r && !(h = rows_or_new(a[5], T, C, *x)).defined()) return nullptr;
    at::Tensor codes = fresh(*x, {T, C}, at::kByte);
    at::Tensor scales = fresh(*x, {T, group > 0 ? C / group : 1}, at::kFloat);
    void *stream = current_stream();
    paro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = paro_rms_norm_quantize_e4m3(half_ptr(x), x->stride(0), half_ptr(r), r ? r->stride(0) : 0, half_ptr(w), eps, group, (int32_t)T,
                                     (int32_t)C, r ? half_out(h) : nullptr, r ? h.stride(0) : 0, (uint8_t *)codes.data_ptr(),
                                     (float *)scales.data_ptr(), stream);
    Py_END_ALLOW_THREADS
    if (st != PARO_OK) return PyLong_FromLong(st);
    PyObject *first = THPVariable_Wrap(std::move(codes)), *second = THPVariable_Wrap(std::move(scales));
    return r ? together({first, second, wrap(a[5], std::move(h))}) : together({first, second});
    END_HANDLE_TH_ERRORS
}

// rope(rope, X, positions, Y or None)
PyObject *rope(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 4) { PyErr_SetString(PyExc_TypeError, "rope takes 4 arguments"); return nullptr; }
    const RopeOn *on = structure<RopeOn>(a[0], g_rope);
    const paro_rope_t *rp = on ? &on->c : nullptr;
    const at::Tensor *x = rp ? tensor(a[1]) : nullptr, *at_ = x ? tensor(a[2]) : nullptr;
    if (!at_ || !rows(*x) || !gpu_rows(*x, -1, x->size(1), *x) || !gpu_vector(*at_, at::kInt, x->size(0), *x) || !same_gpu(on->device, *x) || !current(*x)) return nullptr;
    const int64_t T = x->size(0), C = x->size(1);
    if (rp->head_dim <= 0 || C % rp->head_dim) { refuse("rows are not whole heads"); return nullptr; }
    at::Tensor y = rows_or_new(a[3], T, C, *x);
    if (!y.defined()) return nullptr;
    void *stream = current_stream();
    paro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = paro_rope(rp, half_ptr(x), x->stride(0), (const int32_t *)at_->data_ptr(), (int32_t)(C / rp->head_dim), (int32_t)T,
                   half_out(y), y.stride(0), stream);
    Py_END_ALLOW_THREADS
    return st != PARO_OK ? PyLong_FromLong(st) : wrap(a[3], std::move(y));
    END_HANDLE_TH_ERRORS
}

// kv_append(cache, rope or None, K, V, slots, positions or None, Q or None, Qr or None) -> Qr, or None without Q
PyObject *kv_append(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 8) { PyErr_SetString(PyExc_TypeError, "kv_append takes 8 arguments"); return nullptr; }
    const CacheOn *held = structure<CacheOn>(a[0], g_cache);
    const RopeOn *on = !held || a[1] == Py_None ? nullptr : structure<RopeOn>(a[1], g_rope);
    if (!held || (!on && a[1] != Py_None)) return nullptr;
    const paro_kv_cache *c = &held->c;
    const paro_rope_t *rp = on ? &on->c : nullptr;
    const at::Tensor *k = tensor(a[2]), *v = k ? tensor(a[3]) : nullptr, *slots = v ? tensor(a[4]) : nullptr, *at_, *q;
    if (!slots || !maybe(a[5], at_) || !maybe(a[6], q)) return nullptr;
    const int64_t width = (int64_t)c->kv_heads * c->head_dim;
    if (!rows(*k) || !gpu_rows(*k, -1, width, *k) || !gpu_rows(*v, k->size(0), width, *k)) return nullptr;
    const int64_t T = k->size(0);
    if (!gpu_vector(*slots, at::kLong, T, *k) || (at_ && !gpu_vector(*at_, at::kInt, T, *k))) return nullptr;
    if (!same_gpu(held->device, *k) || (on && !same_gpu(on->device, *k)) || (q && (!rows(*q) || !gpu_rows(*q, T, q->size(1), *k))) || !current(*k)) return nullptr;
    if (!q && a[7] != Py_None) { refuse("Qr takes rotated queries, and there are none"); return nullptr; }
    at::Tensor out;
    int64_t heads = 0;
    if (q) {
        if (c->head_dim <= 0 || q->size(1) % c->head_dim) { refuse("rows are not whole heads"); return nullptr; }
        heads = q->size(1) / c->head_dim;
        if (!(out = rows_or_new(a[7], T, q->size(1), *q)).defined()) return nullptr;
    }
    void *stream = current_stream();
    paro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = paro_kv_append(c, rp, half_ptr(k), k->stride(0), half_ptr(v), v->stride(0), (const int64_t *)slots->data_ptr(),
                        at_ ? (const int32_t *)at_->data_ptr() : nullptr, (int32_t)T, half_ptr(q), q ? q->stride(0) : 0,
                        (int32_t)heads, q ? half_out(out) : nullptr, q ? out.stride(0) : 0, stream);
    Py_END_ALLOW_THREADS
    if (st != PARO_OK) return PyLong_FromLong(st);
    if (!q) Py_RETURN_NONE;
    return wrap(a[7], std::move(out));
    END_HANDLE_TH_ERRORS
}

// paged_attention(cache, Q, block_table, lengths, workspace, bytes, scale, window, O or None, with_lse) -> O, or (O, lse)
PyObject *paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 10) { PyErr_SetString(PyExc_TypeError, "paged_attention takes 10 arguments"); return nullptr; }
    const CacheOn *held = structure<CacheOn>(a[0], g_cache);
    const paro_kv_cache *c = held ? &held->c : nullptr;
    const at::Tensor *q = c ? tensor(a[1]) : nullptr, *table = q ? tensor(a[2]) : nullptr, *lengths = table ? tensor(a[3]) : nullptr;
    const at::Tensor *ws = lengths ? tensor(a[4]) : nullptr;
    if (!ws || !rows(*q) || !gpu_rows(*q, -1, q->size(1), *q)) return nullptr;
    const int64_t B = q->size(0);
    if (c->head_dim <= 0 || q->size(1) % c->head_dim) { refuse("rows are not whole heads"); return nullptr; }
    if (table->scalar_type() != at::kInt || table->dim() != 2 || (table->stride(1) != 1 && table->size(1) != 1) || table->size(0) != B) {
        refuse("expected a block table of int32 rows, one per sequence");
        return nullptr;
    }
    if (!on_gpu(*table, *q) || !gpu_vector(*lengths, at::kInt, B, *q) || !on_gpu(*ws, *q) || !same_gpu(held->device, *q) || !current(*q)) return nullptr;
    const size_t bytes = PyLong_AsSize_t(a[5]);
    const float scale = (float)PyFloat_AsDouble(a[6]);
    int32_t window;
    const int want = PyObject_IsTrue(a[9]);
    if (PyErr_Occurred() || want < 0 || !number(a[7], window)) return nullptr;
    if (table->size(1) > INT32_MAX) { refuse("more pages than 32 bits count"); return nullptr; }
    const int64_t heads = q->size(1) / c->head_dim, ld = B == 1 ? table->size(1) : table->stride(0);
    at::Tensor o = rows_or_new(a[8], B, q->size(1), *q), lse;
    if (!o.defined()) return nullptr;
    if (want) lse = fresh(*q, {B, heads}, at::kFloat);
    void *stream = current_stream();
    paro_status st;
    Py_BEGIN_ALLOW_THREADS
    st = paro_paged_attention(c, half_ptr(q), q->stride(0), (int32_t)heads, (const int32_t *)table->data_ptr(), ld,
                              (int32_t)table->size(1), (const int32_t *)lengths->data_ptr(), (int32_t)B, scale, window, half_out(o),
                              o.stride(0), want ? (float *)lse.data_ptr() : nullptr, ws->data_ptr(), bytes, stream);
    Py_END_ALLOW_THREADS
    if (st != PARO_OK) return PyLong_FromLong(st);
    PyObject *first = wrap(a[8], std::move(o));
    return want ? together({first, THPVariable_Wrap(std::move(lse))}) : first;
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {
    {"types", (PyCFunction)(void (*)(void))types, METH_FASTCALL, nullptr},
    {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, nullptr},
    {"rotate", (PyCFunction)(void (*)(void))rotate, METH_FASTCALL, nullptr},
    {"token_types", (PyCFunction)(void (*)(void))token_types, METH_FASTCALL, nullptr},
    {"rms_norm", (PyCFunction)(void (*)(void))rms_norm, METH_FASTCALL, nullptr},
    {"rms_norm_quantize_e4m3", (PyCFunction)(void (*)(void))rms_norm_quantize_e4m3, METH_FASTCALL, nullptr},
    {"rope", (PyCFunction)(void (*)(void))rope, METH_FASTCALL, nullptr},
    {"kv_append", (PyCFunction)(void (*)(void))kv_append, METH_FASTCALL, nullptr},
    {"paged_attention", (PyCFunction)(void (*)(void))paged_attention, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "paro_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_paro_host(void) { return PyModule_Create(&module); }
