// The library's per-layer calls for Python: the checks of types, shapes, strides and devices, and the marshalling of
// tensors into plain pointers, in C++.  A decode step makes these calls several times per layer; with the checks in
// Python and ctypes a call took 5.8 us of host time, of which the launch itself is 2.5 us.  Every function returns the
// library's status; a tensor that does not fit gives kBadTensor, which the binding reports as an invalid argument.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/lckv.h"

namespace {

constexpr int kBadTensor = -1;

// The arguments of one call, taken in order; `ok` turns false at the first that is not what is asked for.
struct Args {
    PyObject* const* a;
    Py_ssize_t n, at = 0;
    bool ok = true;
    PyObject* take()
    {
        if (at >= n) { ok = false; return Py_None; }
        return a[at++];
    }
    const at::Tensor* tensor()                       // null where None
    {
        PyObject* o = take();
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) { ok = false; return nullptr; }
        return &THPVariable_Unpack(o);
    }
    int64_t integer()
    {
        const long long v = PyLong_AsLongLong(take());
        if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return v;
    }
    int32_t integer32()
    {
        const int64_t v = integer();
        if (v != (int32_t)v) ok = false;
        return (int32_t)v;
    }
    void* address() { return reinterpret_cast<void*>(integer()); }
    double real()
    {
        const double v = PyFloat_AsDouble(take());
        if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return v;
    }
};

bool on(const at::Tensor* t, int64_t dev) { return t->is_cuda() && t->get_device() == dev; }
bool dense(const at::Tensor* t, at::ScalarType type, int64_t dev) { return t->scalar_type() == type && t->is_contiguous() && on(t, dev); }
// 0 bf16, 1 fp32, else -1
int float_kind(const at::Tensor* t)
{
    return t->scalar_type() == at::kBFloat16 ? 0 : t->scalar_type() == at::kFloat ? 1 : -1;
}
const void* ptr(const at::Tensor* t) { return t ? t->const_data_ptr() : nullptr; }
void* mut(const at::Tensor* t) { return t ? t->mutable_data_ptr() : nullptr; }

PyObject* code(int rc) { return PyLong_FromLong(rc); }

// `call(stream)` with `dev` current, on the stream given (an address, or None for the current stream of `dev`).
template <typename F>
PyObject* run(Args& args, int64_t dev, F call)
{
    PyObject* given = args.take();
    if (!args.ok) return code(kBadTensor);
    void* stream = nullptr;
    if (given == Py_None) {
        stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
    } else {
        stream = PyLong_AsVoidPtr(given);
        if (!stream && PyErr_Occurred()) return nullptr;
    }
    if (c10::cuda::current_device() == dev) return code(call(stream));
    const c10::cuda::CUDAGuard guard((c10::DeviceIndex)dev);
    return code(call(stream));
}

// No C++ exception leaves a call: torch's checks throw.
template <PyObject* (*F)(Args&)>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    try {
        Args args{a, n};
        return F(args);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// cos, sin, scaling, stream
PyObject* rope_tables(Args& a)
{
    const at::Tensor *c = a.tensor(), *s = a.tensor();
    const auto* scaling = static_cast<const lckv_rope_scaling_t*>(a.address());
    if (!a.ok || !c || !s || c->dim() != 2 || c->sizes() != s->sizes() || !c->is_cuda()) return code(kBadTensor);
    const int64_t dev = c->get_device();
    if (!dense(c, at::kFloat, dev) || !dense(s, at::kFloat, dev) || c->size(0) > INT32_MAX || c->size(1) > INT32_MAX / 2) return code(kBadTensor);
    return run(a, dev, [&](void* st) {
        return lckv_rope_tables(static_cast<float*>(mut(c)), static_cast<float*>(mut(s)), (int32_t)c->size(0), (int32_t)(2 * c->size(1)), scaling, st);
    });
}

// rope, its device, positions, x, out, transpose, stream
PyObject* rope_apply(Args& a)
{
    const auto* rope = static_cast<const lckv_rope_t*>(a.address());
    const int64_t dev = a.integer();
    const at::Tensor *pos = a.tensor(), *x = a.tensor(), *y = a.tensor();
    const int64_t transpose = a.integer();
    if (!a.ok || !pos || !x || !y || x->dim() != 3 || x->sizes() != y->sizes()) return code(kBadTensor);
    const int kind = float_kind(x);
    if (kind < 0 || y->scalar_type() != x->scalar_type() || x->stride(2) != 1 || y->stride(2) != 1 || !on(x, dev) || !on(y, dev) ||
        !dense(pos, at::kInt, dev) || pos->dim() != 1 || pos->size(0) != x->size(0))
        return code(kBadTensor);
    if (x->size(0) > INT32_MAX || x->size(1) > INT32_MAX) return code(kBadTensor);
    if (x->size(0) == 0) return code(LCKV_OK);
    return run(a, dev, [&](void* st) {
        return lckv_rope_apply(rope, static_cast<const int32_t*>(ptr(pos)), ptr(x), x->stride(0), x->stride(1), mut(y), y->stride(0), y->stride(1),
                               (int32_t)x->size(0), (int32_t)x->size(1), (int32_t)x->size(2), kind, transpose ? 1 : 0, st);
    });
}

// x, weight, out, residual, residual_out, out_scale, scale_group, eps, stream
PyObject* rms_norm(Args& a)
{
    const at::Tensor *x = a.tensor(), *w = a.tensor(), *y = a.tensor(), *r = a.tensor(), *h = a.tensor(), *s = a.tensor();
    const int32_t group = a.integer32();
    const double eps = a.real();
    if (!a.ok || !x || !w || !y || x->dim() != 2 || !x->is_cuda()) return code(kBadTensor);
    const int64_t dev = x->get_device(), rows = x->size(0), width = x->size(1);
    const int xk = float_kind(x), wk = float_kind(w), yk = y->scalar_type() == at::kFloat8_e4m3fn ? 2 : float_kind(y);
    if (xk < 0 || wk < 0 || yk < 0 || y->sizes() != x->sizes() || w->dim() != 1 || w->size(0) != width || !y->is_contiguous() || !on(y, dev) ||
        !w->is_contiguous() || !on(w, dev) || (x->stride(1) != 1 && width > 1) || (rows > 1 && x->stride(0) < width) || rows > INT32_MAX || width > INT32_MAX)
        return code(kBadTensor);
    int rk = 0;
    if (r) {
        rk = float_kind(r);
        if (rk < 0 || r->sizes() != x->sizes() || !r->is_contiguous() || !on(r, dev)) return code(kBadTensor);
    }
    if (h && (!r || h->sizes() != x->sizes() || !dense(h, r->scalar_type(), dev))) return code(kBadTensor);
    if (s && (!dense(s, at::kFloat, dev) || s->numel() != rows * (group ? (width + 127) / 128 : 1))) return code(kBadTensor);
    if (rows == 0) return code(LCKV_OK);
    return run(a, dev, [&](void* st) {
        return lckv_rms_norm(ptr(x), rows > 1 ? x->stride(0) : 0, xk, ptr(r), mut(h), rk, ptr(w), wk, mut(y), yk, static_cast<float*>(mut(s)), group,
                             (int32_t)rows, (int32_t)width, (float)eps, st);
    });
}

// packed, its device, n, k, group, has_zeros, x, out, x_scale, dev_status, stream
PyObject* quant_linear(Args& a)
{
    const void* packed = a.address();
    const int64_t dev = a.integer(), n = a.integer(), k = a.integer(), group = a.integer(), zeros = a.integer();
    const at::Tensor *x = a.tensor(), *y = a.tensor(), *s = a.tensor(), *status = a.tensor();
    if (!a.ok || !x || !y || x->dim() != 2 || y->dim() != 2) return code(kBadTensor);
    const int64_t rows = x->size(0);
    const int xk = x->scalar_type() == at::kBFloat16 ? 0 : x->scalar_type() == at::kFloat8_e4m3fn ? 1 : -1, yk = float_kind(y);
    if (xk < 0 || yk < 0 || x->size(1) != k || x->stride(1) != 1 || y->size(0) != rows || y->size(1) != n || (y->stride(1) != 1 && n > 1) ||
        (rows > 1 && (x->stride(0) < k || y->stride(0) < n)) || !on(x, dev) || !on(y, dev) || rows > INT32_MAX)
        return code(kBadTensor);
    int32_t x_group = 0;
    if (s) {
        x_group = s->numel() == rows ? 0 : 128;
        if (xk != 1 || !dense(s, at::kFloat, dev) || s->numel() != (x_group ? rows * ((k + 127) / 128) : rows)) return code(kBadTensor);
    }
    if (status && !(status->scalar_type() == at::kInt && status->numel() > 0 && on(status, dev))) return code(kBadTensor);
    if (rows == 0) return code(LCKV_OK);
    return run(a, dev, [&](void* st) {
        return lckv_quant_linear(packed, (int32_t)n, (int32_t)k, (int32_t)group, (int32_t)zeros, ptr(x), rows > 1 ? x->stride(0) : 0, xk,
                                 static_cast<const float*>(ptr(s)), x_group, mut(y), rows > 1 ? y->stride(0) : 0, yk, (int32_t)rows,
                                 static_cast<int32_t*>(mut(status)), st);
    });
}

// Elements between consecutive tokens of a bf16 tensor [batch, n, heads, d] (or [batch, heads, d]: n = 1) whose heads
// are dense; 0 for a single token, -1 where there is no such number.
int64_t token_stride(const at::Tensor* t, int64_t dev, int64_t batch, int64_t n, bool one, int64_t heads, int64_t d)
{
    if (t->scalar_type() != at::kBFloat16 || !on(t, dev) || t->dim() != (one ? 3 : 4)) return -1;
    const auto z = t->sizes();
    const auto st = t->strides();
    const int h = one ? 1 : 2;
    if (z[0] != batch || (!one && z[1] != n) || z[h] != heads || z[h + 1] != d) return -1;
    if (st[h + 1] != 1 || (st[h] != d && heads > 1)) return -1;
    int64_t step = st[0];
    if (n > 1) {
        step = st[1];
        if (batch > 1 && st[0] != n * step) return -1;
    }
    return batch * n == 1 ? 0 : step >= heads * d ? step : -1;
}

// cache, its device, slot, rope, the rope's device, H_q, H_kv, d, q, k, v, q_out, advance (-1: a prompt), stream
PyObject* rope_cache(Args& a)
{
    auto* cache = static_cast<lckv_cache_t*>(a.address());
    const int64_t dev = a.integer();
    const int32_t slot = a.integer32();
    const auto* rope = static_cast<const lckv_rope_t*>(a.address());
    const int64_t rope_dev = a.integer(), hq = a.integer(), hkv = a.integer(), d = a.integer();
    const at::Tensor *q = a.tensor(), *k = a.tensor(), *v = a.tensor(), *o = a.tensor();
    const int64_t advance = a.integer();
    const at::Tensor* ref = q ? q : k;
    if (!a.ok || !cache || !ref || rope_dev != dev || (!k) != (!v) || (!q) != (!o)) return code(kBadTensor);
    const bool one = ref->dim() == 3;
    if (!one && ref->dim() != 4) return code(kBadTensor);
    const int64_t batch = ref->size(0), n = one ? 1 : ref->size(1);
    if (batch < 1 || n < 1 || batch > INT32_MAX || n > INT32_MAX) return code(kBadTensor);
    int64_t q_step = 0, kv_step = 0;
    if (q) {
        q_step = token_stride(q, dev, batch, n, one, hq, d);
        if (q_step < 0 || o->sizes() != q->sizes() || !dense(o, at::kBFloat16, dev)) return code(kBadTensor);
    }
    if (k) {
        kv_step = token_stride(k, dev, batch, n, one, hkv, d);
        if (kv_step < 0 || token_stride(v, dev, batch, n, one, hkv, d) != kv_step) return code(kBadTensor);
    }
    return run(a, dev, [&](void* st) {
        if (advance < 0)
            return lckv_rope_prefill_write_kv(cache, slot, rope, ptr(q), q_step, mut(o), ptr(k), ptr(v), kv_step, (int32_t)n, (int32_t)batch, st);
        return lckv_rope_append_kv(cache, slot, rope, ptr(q), q_step, mut(o), ptr(k), ptr(v), kv_step, (int32_t)n, (int32_t)batch, (int32_t)advance, st);
    });
}

// Is t dense, on the device, with at least n elements of the type: fp32, or bf16 (as such or as raw 16-bit patterns)?  Not more is
// asked of its shape.
bool holds(const at::Tensor* t, int64_t dev, int64_t n, bool f32 = false)
{
    if (!t) return false;
    const auto type = t->scalar_type();
    const bool fits = f32 ? type == at::kFloat : type == at::kBFloat16 || type == at::kShort || type == at::kUInt16;
    return fits && t->is_contiguous() && on(t, dev) && n >= 0 && t->numel() >= n;
}

// cache, its device, slot, mode, H_q, d, fp32 outputs?, q, out, lse, batch, stream
PyObject* decode_attention(Args& a)
{
    auto* cache = static_cast<lckv_cache_t*>(a.address());
    const int64_t dev = a.integer();
    const int32_t slot = a.integer32(), mode = a.integer32();
    const int64_t hq = a.integer(), d = a.integer(), f32 = a.integer();
    const at::Tensor *q = a.tensor(), *out = a.tensor(), *lse = a.tensor();
    const int32_t batch = a.integer32();
    if (!a.ok || !cache || !holds(q, dev, batch * hq * d) || !holds(out, dev, batch * hq * d, f32 != 0) || (lse && !holds(lse, dev, batch * hq, true)))
        return code(kBadTensor);
    return run(a, dev, [&](void* st) { return lckv_decode_attention(cache, slot, mode, ptr(q), mut(out), static_cast<float*>(mut(lse)), batch, st); });
}

// cache, its device, slot, H_kv, d, k, v, batch, advance, stream
PyObject* append_kv(Args& a)
{
    auto* cache = static_cast<lckv_cache_t*>(a.address());
    const int64_t dev = a.integer();
    const int32_t slot = a.integer32();
    const int64_t hkv = a.integer(), d = a.integer();
    const at::Tensor *k = a.tensor(), *v = a.tensor();
    const int32_t batch = a.integer32(), advance = a.integer32();
    if (!a.ok || !cache || !holds(k, dev, batch * hkv * d) || !holds(v, dev, batch * hkv * d)) return code(kBadTensor);
    return run(a, dev, [&](void* st) { return lckv_append_kv(cache, slot, ptr(k), ptr(v), batch, advance, st); });
}

// cache, its device, slot, H_kv, d, k, v, n_max, batch, stream
PyObject* prefill_write_kv(Args& a)
{
    auto* cache = static_cast<lckv_cache_t*>(a.address());
    const int64_t dev = a.integer();
    const int32_t slot = a.integer32();
    const int64_t hkv = a.integer(), d = a.integer();
    const at::Tensor *k = a.tensor(), *v = a.tensor();
    const int32_t n = a.integer32(), batch = a.integer32();
    if (!a.ok || !cache || n < 0 || batch < 0 || hkv < 1 || d < 1 || (int64_t)n * batch > INT64_MAX / (hkv * d)) return code(kBadTensor);
    const int64_t elements = (int64_t)n * batch * hkv * d;
    if (!holds(k, dev, elements) || !holds(v, dev, elements)) return code(kBadTensor);
    return run(a, dev, [&](void* st) { return lckv_prefill_write_kv(cache, slot, ptr(k), ptr(v), n, batch, st); });
}

// cache, its device, slot, H_kv, d, k, v, stream
PyObject* read_kv(Args& a)
{
    auto* cache = static_cast<lckv_cache_t*>(a.address());
    const int64_t dev = a.integer();
    const int32_t slot = a.integer32();
    const int64_t hkv = a.integer(), d = a.integer();
    const at::Tensor *k = a.tensor(), *v = a.tensor();
    if (!a.ok || !cache || !k || !v || k->dim() != 4 || k->sizes() != v->sizes() || k->size(2) != hkv || k->size(3) != d) return code(kBadTensor);
    const int kind = float_kind(k);
    if (kind < 0 || !dense(k, k->scalar_type(), dev) || !dense(v, k->scalar_type(), dev) || k->size(0) > INT32_MAX || k->size(1) > INT32_MAX) return code(kBadTensor);
    return run(a, dev, [&](void* st) { return lckv_cache_read_kv(cache, slot, mut(k), mut(v), kind, (int32_t)k->size(1), (int32_t)k->size(0), st); });
}

// fp32 [batch, heads, n] with n >= rows
bool weights_like(const at::Tensor* t, int64_t dev, int64_t batch, int64_t heads, int64_t rows)
{
    return dense(t, at::kFloat, dev) && t->dim() == 3 && t->size(0) == batch && t->size(1) == heads && t->size(2) >= rows;
}

// cache, its device, slot, mode, H_q, H_kv, d, max_seq, q, lse, previous, weights, stream
PyObject* attention_weights(Args& a)
{
    auto* cache = static_cast<lckv_cache_t*>(a.address());
    const int64_t dev = a.integer();
    const int32_t slot = a.integer32(), mode = a.integer32();
    const int64_t hq = a.integer(), hkv = a.integer(), d = a.integer(), rows = a.integer();
    const at::Tensor *q = a.tensor(), *lse = a.tensor(), *prev = a.tensor(), *w = a.tensor();
    if (!a.ok || !cache || !q || !lse || !w || !dense(q, at::kBFloat16, dev) || q->dim() != 3 || q->size(1) != hq || q->size(2) != d) return code(kBadTensor);
    const int64_t batch = q->size(0);
    if (!dense(lse, at::kFloat, dev) || lse->dim() != 2 || lse->size(0) != batch || lse->size(1) != hq || batch > INT32_MAX) return code(kBadTensor);
    if (!weights_like(w, dev, batch, hkv, rows) || (prev && (!weights_like(prev, dev, batch, hkv, rows) || prev->size(2) != w->size(2)))) return code(kBadTensor);
    return run(a, dev, [&](void* st) {
        return lckv_attention_weights(cache, slot, mode, ptr(q), static_cast<const float*>(ptr(lse)), static_cast<const float*>(ptr(prev)),
                                      static_cast<float*>(mut(w)), w->size(2), (int32_t)batch, st);
    });
}

// cache, its device, slot, source cache, its device, its slot, H_kv, the source's max_seq, the cache's, kept, weights, weights_out, n_sink,
// n_recent, set_len, stream
PyObject* evict_kv(Args& a)
{
    auto* cache = static_cast<lckv_cache_t*>(a.address());
    const int64_t dev = a.integer();
    const int32_t slot = a.integer32();
    const auto* src = static_cast<const lckv_cache_t*>(a.address());
    const int64_t src_dev = a.integer();
    const int32_t src_slot = a.integer32();
    const int64_t hkv = a.integer(), src_rows = a.integer(), rows = a.integer();
    const at::Tensor *kept = a.tensor(), *w = a.tensor(), *out = a.tensor();
    const int32_t sink = a.integer32(), recent = a.integer32(), set_len = a.integer32();
    if (!a.ok || !cache || !src || src_dev != dev || !kept || !dense(kept, at::kInt, dev) || kept->dim() != 3 || kept->size(1) != hkv) return code(kBadTensor);
    const int64_t batch = kept->size(0), keep = kept->size(2);
    if (batch > INT32_MAX || keep > INT32_MAX) return code(kBadTensor);
    if ((w && !weights_like(w, dev, batch, hkv, src_rows)) || (out && !weights_like(out, dev, batch, hkv, rows))) return code(kBadTensor);
    return run(a, dev, [&](void* st) {
        return lckv_evict_kv(cache, slot, src, src_slot, static_cast<const float*>(ptr(w)), w ? w->size(2) : 0, static_cast<float*>(mut(out)),
                             out ? out->size(2) : 0, static_cast<int32_t*>(mut(kept)), sink, recent, (int32_t)keep, (int32_t)batch, set_len, st);
    });
}

#define LCKV_CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(entry<name>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {LCKV_CALL(rope_tables), LCKV_CALL(rope_apply), LCKV_CALL(rms_norm), LCKV_CALL(quant_linear), LCKV_CALL(rope_cache),
                         LCKV_CALL(decode_attention), LCKV_CALL(append_kv), LCKV_CALL(prefill_write_kv), LCKV_CALL(read_kv), LCKV_CALL(attention_weights), LCKV_CALL(evict_kv),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lckv_calls", "Per-layer calls of liblckv.so on torch tensors.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lckv_calls(void) { return PyModule_Create(&module); }
