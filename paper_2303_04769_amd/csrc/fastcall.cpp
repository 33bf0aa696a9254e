// The single-layer calls of binding.py, and the calls of attn.py and cache.py, from Python, without ctypes: a call of a few microseconds on the GPU is bound by its
// host time, and of that the launch itself takes 3.0 us; attribute reads, argument conversion and the foreign-function
// interface took another 1.6 (ReLU) to 3 (convolution), here some 0.4.
//
// Every function takes the arguments of the binding's function of that name, positionally, with the stream last, and
// returns the library's status. It returns None, having done nothing, for whatever is not the plain case (a stream given,
// tensors of a subclass, integers or paddings or quantization records of other types): the binding then makes the same call
// through ctypes, which accepts or refuses it.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <c10/hip/HIPStream.h>

#include <dlfcn.h>
#include <limits.h>
#include <stddef.h>
#include <string.h>

#include <initializer_list>

#include "../../include/small.h"
#include "../include/small_cache.h"

namespace {

PyTypeObject *quant_type = nullptr;        // binding.small_quant
PyTypeObject *attn_type = nullptr;         // attn.small_attn
PyTypeObject *rotation_type = nullptr, *cache_type = nullptr;      // cache.small_rotation, cache.small_cache

#define SMALL_FUNCTIONS(X)                                                                                                        \
    X(small_pack) X(small_unpack) X(small_conv2d) X(small_dwconv2d) X(small_pool2d) X(small_relu) X(small_add) X(small_dense)     \
    X(small_pack_u8) X(small_unpack_u8) X(small_conv2d_u8) X(small_dwconv2d_u8) X(small_dense_u8) X(small_pool2d_u8) X(small_relu_u8) \
    X(small_groupnorm) X(small_groupnorm_grad) X(small_attention) X(small_attention_grad)                                         \
    X(small_rotary) X(small_rotary_grad) X(small_cache_write) X(small_cache_read) X(small_cache_attention)
struct Library {
#define X(f) decltype(&::f) f = nullptr;
    SMALL_FUNCTIONS(X)
#undef X
} lib;

// Reads one call's arguments; `plain` turns false at the first that is not the plain case.
struct Reader {
    PyObject *const *a;
    bool plain, error = false;
    Py_buffer quant = {};

    Reader(PyObject *const *args, Py_ssize_t n, Py_ssize_t expected) : a(args), plain(n == expected && lib.small_relu && args[n - 1] == Py_None) {}
    ~Reader()
    {
        if (quant.obj) PyBuffer_Release(&quant);
    }
    unsigned long number(int k)
    {
        if (!plain) return 0;
        if (!PyLong_CheckExact(a[k])) {
            plain = false;
            return 0;
        }
        return PyLong_AsUnsignedLongMask(a[k]);          // (as ctypes converts: modulo the type's range)
    }
    int i(int k) { return (int)number(k); }
    small_pad pad(int k)
    {
        int side[4] = {0, 0, 0, 0};
        if (!plain) return {0, 0, 0, 0};
        PyObject *p = a[k];
        if (!PyTuple_CheckExact(p) || PyTuple_GET_SIZE(p) > 4) {
            plain = false;
            return {0, 0, 0, 0};
        }
        for (Py_ssize_t j = 0; j < PyTuple_GET_SIZE(p); ++j) {
            PyObject *v = PyTuple_GET_ITEM(p, j);
            if (!PyLong_CheckExact(v)) plain = false;
            else side[j] = (int)PyLong_AsUnsignedLongMask(v);
        }
        return {side[0], side[1], side[2], side[3]};
    }
    const small_quant *q(int k)
    {
        if (!plain) return nullptr;
        if (Py_TYPE(a[k]) != quant_type || PyObject_GetBuffer(a[k], &quant, PyBUF_SIMPLE) != 0 || quant.len != (Py_ssize_t)sizeof(small_quant)) {
            PyErr_Clear();
            plain = false;
            return nullptr;
        }
        return static_cast<const small_quant *>(quant.buf);
    }
    template <typename T>
    T *tensor(int k, at::ScalarType type, const char *refusal)
    {
        if (!plain || error || a[k] == Py_None) return nullptr;
        if (!THPVariable_CheckExact(a[k])) {
            plain = false;
            return nullptr;
        }
        const at::Tensor &t = THPVariable_Unpack(a[k]);
        if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous()) {
            PyErr_SetString(PyExc_TypeError, refusal);
            error = true;
            return nullptr;
        }
        return static_cast<T *>(t.data_ptr());
    }
    float number32(int k)
    {
        if (!plain) return 0.f;
        if (!PyFloat_CheckExact(a[k])) {
            plain = false;
            return 0.f;
        }
        return (float)PyFloat_AS_DOUBLE(a[k]);
    }
    // The record of an attention plan, without its pointers and strides.
    small_attn record(int k)
    {
        small_attn r = {};
        if (!plain) return r;
        if (!attn_type || Py_TYPE(a[k]) != attn_type || PyObject_GetBuffer(a[k], &quant, PyBUF_SIMPLE) != 0 || quant.len != (Py_ssize_t)sizeof(small_attn)) {
            PyErr_Clear();
            plain = false;
            return r;
        }
        memcpy(&r, quant.buf, sizeof r);
        return r;
    }
    // A record of a plan of cache.py, copied.
    template <typename T>
    T record(int k, PyTypeObject *type)
    {
        T r = {};
        Py_buffer b = {};
        if (!plain) return r;
        if (!type || Py_TYPE(a[k]) != type || PyObject_GetBuffer(a[k], &b, PyBUF_SIMPLE) != 0) {
            PyErr_Clear();
            plain = false;
            return r;
        }
        if (b.len == (Py_ssize_t)sizeof r) memcpy(&r, b.buf, sizeof r);
        else plain = false;
        PyBuffer_Release(&b);
        return r;
    }
    // An activation [N][blocks][S][Cb] that may be a view, of at least `channels` channels.
    float *view(int k, const small_attn &r, int S, long channels, small_tokens *strides) { return view(k, r.N, S, r.Cb, channels, strides); }
    float *view(int k, long N, long S, long Cb, long channels, small_tokens *strides, bool optional = false)
    {
        if (!plain || error || (optional && a[k] == Py_None)) return nullptr;
        if (!THPVariable_CheckExact(a[k])) {
            plain = false;
            return nullptr;
        }
        const at::Tensor &t = THPVariable_Unpack(a[k]);
        if (!t.is_cuda() || t.scalar_type() != at::kFloat || t.dim() != 4 || t.size(0) != N || t.size(2) != S || t.size(3) != Cb ||
            (Cb > 1 && t.stride(3) != 1) || t.size(1) * Cb < channels) {
            plain = false;                               // (the binding says what is wrong with it)
            return nullptr;
        }
        *strides = small_tokens{(size_t)t.stride(0), (size_t)t.stride(1), (size_t)t.stride(2)};
        return static_cast<float *>(t.data_ptr());
    }
    // Sizes [N][..][S][Cb] of an activation.
    bool sizes(int k, int *N, int *S, int *Cb)
    {
        if (plain && !THPVariable_CheckExact(a[k])) plain = false;
        if (!plain || error) return false;
        const at::Tensor &t = THPVariable_Unpack(a[k]);
        if (t.dim() != 4 || t.size(0) > INT_MAX || t.size(2) > INT_MAX || t.size(3) > INT_MAX) return plain = false;
        *N = (int)t.size(0);
        *S = (int)t.size(2);
        *Cb = (int)t.size(3);
        return true;
    }
    // A table of pages [N][..], with its place in the cache's record.
    void pages(int k, int N, small_cache &c)
    {
        if (plain && !THPVariable_CheckExact(a[k])) plain = false;
        if (!plain || error) return;
        const at::Tensor &t = THPVariable_Unpack(a[k]);
        if (!t.is_cuda() || t.scalar_type() != at::kInt || !t.is_contiguous() || t.dim() != 2 || t.size(0) != N || t.size(1) > INT_MAX) {
            plain = false;
            return;
        }
        c.N = N;
        c.per_stream = (int)t.size(1);
        c.table = static_cast<const int *>(t.data_ptr());
    }
    // A rotation's frequencies and places, from arguments k and k + 1.
    void places(int k, small_rotation &r)
    {
        r.freq = of<float>(k, at::kFloat, {r.freq_heads, r.axes, r.pairs});
        r.positions = of<int>(k + 1, at::kInt, {r.N, r.S, r.axes});
        if (a[k] == Py_None) plain = false;
        if (!r.positions)
            for (int x = 1; x < r.axes && x < 4; ++x)
                if (r.extent[x] < 1) plain = false;
    }
    // A contiguous tensor of these sizes, or null for None.
    template <typename T>
    T *of(int k, at::ScalarType type, std::initializer_list<long> sizes)
    {
        if (!plain || error || a[k] == Py_None) return nullptr;
        if (!THPVariable_CheckExact(a[k])) {
            plain = false;
            return nullptr;
        }
        const at::Tensor &t = THPVariable_Unpack(a[k]);
        bool fits = t.is_cuda() && t.scalar_type() == type && t.is_contiguous() && t.dim() == (long)sizes.size();
        long d = 0;
        if (fits)
            for (long n : sizes) fits = fits && t.size(d++) == n;
        if (!fits) {
            plain = false;
            return nullptr;
        }
        return static_cast<T *>(t.data_ptr());
    }
    // Argument k, if there is one, has so many values (the binding says so where not; sizes that the library refuses are its to refuse).
    void holds(int k, long long values)
    {
        if (!plain || error || a[k] == Py_None || values <= 0) return;
        if (THPVariable_Unpack(a[k]).numel() != values) plain = false;
    }
    void *bytes(int k, size_t *size)
    {
        *size = 0;
        if (!plain || error || a[k] == Py_None) return nullptr;
        if (!THPVariable_CheckExact(a[k])) {
            plain = false;
            return nullptr;
        }
        const at::Tensor &t = THPVariable_Unpack(a[k]);
        *size = t.nbytes();
        return t.data_ptr();
    }
    // lengths, first, prefix, docs, slopes, table, bucket from argument k on.
    void masks(int k, small_attn &r)
    {
        r.lengths = of<int>(k, at::kInt, {r.N});
        r.first = of<int>(k + 1, at::kInt, {r.N});
        r.prefix = of<int>(k + 2, at::kInt, {r.N});
        r.docs = of<int>(k + 3, at::kInt, {r.N, r.Sk});
        r.slopes = of<float>(k + 4, at::kFloat, {r.heads});
        r.table = of<float>(k + 5, at::kFloat, {r.heads, r.buckets});
        r.bucket = of<int>(k + 6, at::kInt, {2L * r.reach + 1});
    }
    float *f32(int k) { return tensor<float>(k, at::kFloat, "expected a contiguous float32 CUDA tensor"); }
    unsigned char *u8(int k) { return tensor<unsigned char>(k, at::kByte, "expected a contiguous uint8 CUDA tensor"); }
    int *i32(int k) { return tensor<int>(k, at::kInt, "expected a contiguous int32 CUDA tensor"); }

    // The call, if everything was plain, on the current stream of the current device; without the interpreter lock, which ctypes
    // does not hold either.
    template <typename F>
    PyObject *call(F f)
    {
        if (error) return nullptr;
        if (!plain) Py_RETURN_NONE;
        void *stream = c10::hip::getCurrentHIPStream().stream();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = f(stream);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    }
};

// The other arguments are read before the tensors, so that a call that is not plain raises nothing here.
#define ENTRY(name, n_args, ...)                                              \
    PyObject *name(PyObject *, PyObject *const *args, Py_ssize_t n)           \
    {                                                                         \
        HANDLE_TH_ERRORS                                                      \
        Reader r(args, n, n_args);                                            \
        __VA_ARGS__                                                           \
        END_HANDLE_TH_ERRORS                                                  \
    }

#define LAYOUT(name, fn, tensor)                                                                                    \
    ENTRY(name, 8, const int N = r.i(2), C = r.i(3), H = r.i(4), W = r.i(5), Cb = r.i(6);                           \
          auto *src = r.tensor(0); auto *dst = r.tensor(1);                                                         \
          return r.call([&](void *s) { return lib.fn(src, dst, N, C, H, W, Cb, s); });)
LAYOUT(pack, small_pack, f32)
LAYOUT(unpack, small_unpack, f32)
LAYOUT(pack_u8, small_pack_u8, u8)
LAYOUT(unpack_u8, small_unpack_u8, u8)

ENTRY(conv2d, 15, const int N = r.i(3), Ci = r.i(4), Co = r.i(5), H = r.i(6), W = r.i(7), kh = r.i(8), kw = r.i(9), st = r.i(10);
      const small_pad pad = r.pad(11); const int Cib = r.i(12), Cob = r.i(13);
      auto *x = r.f32(0); auto *w = r.f32(1); auto *y = r.f32(2);
      return r.call([&](void *s) { return lib.small_conv2d(x, w, y, N, Ci, Co, H, W, kh, kw, st, pad, Cib, Cob, s); });)
ENTRY(conv2d_u8, 17, const int N = r.i(3), Ci = r.i(4), Co = r.i(5), H = r.i(6), W = r.i(7), kh = r.i(8), kw = r.i(9), st = r.i(10);
      const small_pad pad = r.pad(11); const int Cib = r.i(12), Cob = r.i(13); const small_quant *q = r.q(14);
      auto *x = r.u8(0); auto *w = r.u8(1); auto *y = r.u8(2); auto *sums = r.i32(15);
      return r.call([&](void *s) { return lib.small_conv2d_u8(x, w, y, N, Ci, Co, H, W, kh, kw, st, pad, Cib, Cob, q, sums, s); });)
ENTRY(dwconv2d, 13, const int N = r.i(3), C = r.i(4), H = r.i(5), W = r.i(6), kh = r.i(7), kw = r.i(8), st = r.i(9);
      const small_pad pad = r.pad(10); const int Cb = r.i(11);
      auto *x = r.f32(0); auto *w = r.f32(1); auto *y = r.f32(2);
      return r.call([&](void *s) { return lib.small_dwconv2d(x, w, y, N, C, H, W, kh, kw, st, pad, Cb, s); });)
ENTRY(dwconv2d_u8, 14, const int N = r.i(3), C = r.i(4), H = r.i(5), W = r.i(6), kh = r.i(7), kw = r.i(8), st = r.i(9);
      const small_pad pad = r.pad(10); const int Cb = r.i(11); const small_quant *q = r.q(12);
      auto *x = r.u8(0); auto *w = r.u8(1); auto *y = r.u8(2);
      return r.call([&](void *s) { return lib.small_dwconv2d_u8(x, w, y, N, C, H, W, kh, kw, st, pad, Cb, q, s); });)

#define POOL(name, fn, tensor)                                                                                                  \
    ENTRY(name, 13, const int N = r.i(2), C = r.i(3), H = r.i(4), W = r.i(5), kh = r.i(6), kw = r.i(7), st = r.i(8);            \
          const small_pad pad = r.pad(9); const int Cb = r.i(10), mode = r.i(11);                                               \
          auto *x = r.tensor(0); auto *y = r.tensor(1);                                                                         \
          return r.call([&](void *s) { return lib.fn(x, y, N, C, H, W, kh, kw, st, pad, Cb, mode, s); });)
POOL(pool2d, small_pool2d, f32)
POOL(pool2d_u8, small_pool2d_u8, u8)

ENTRY(relu, 4, const size_t n_el = r.number(2); auto *x = r.f32(0); auto *y = r.f32(1);
      return r.call([&](void *s) { return lib.small_relu(x, y, n_el, s); });)
ENTRY(relu_u8, 5, const size_t n_el = r.number(2); const int z = r.i(3); auto *x = r.u8(0); auto *y = r.u8(1);
      return r.call([&](void *s) { return lib.small_relu_u8(x, y, n_el, z, s); });)
ENTRY(add, 5, const size_t n_el = r.number(3); auto *x = r.f32(0); auto *b = r.f32(1); auto *y = r.f32(2);
      return r.call([&](void *s) { return lib.small_add(x, b, y, n_el, s); });)
ENTRY(dense, 9, const int N = r.i(3), Ci = r.i(4), Co = r.i(5), Cib = r.i(6), Cob = r.i(7);
      auto *x = r.f32(0); auto *w = r.f32(1); auto *y = r.f32(2);
      return r.call([&](void *s) { return lib.small_dense(x, w, y, N, Ci, Co, Cib, Cob, s); });)
ENTRY(dense_u8, 11, const int N = r.i(3), Ci = r.i(4), Co = r.i(5), Cib = r.i(6), Cob = r.i(7); const small_quant *q = r.q(8);
      auto *x = r.u8(0); auto *w = r.u8(1); auto *y = r.u8(2); auto *sums = r.i32(9);
      return r.call([&](void *s) { return lib.small_dense_u8(x, w, y, N, Ci, Co, Cib, Cob, q, sums, s); });)

ENTRY(groupnorm, 15, const int N = r.i(5), C = r.i(6), H = r.i(7), W = r.i(8), G = r.i(9); const float eps = r.number32(10); const int act = r.i(11), Cb = r.i(12);
      size_t size; void *ws = r.bytes(13, &size);
      auto *x = r.f32(0); auto *ga = r.f32(1); auto *be = r.f32(2); auto *y = r.f32(3); auto *st = r.f32(4);
      const long long all = (long long)N * C * H * W; r.holds(0, all); r.holds(1, C); r.holds(2, C); r.holds(3, all); r.holds(4, 2LL * N * G);
      return r.call([&](void *s) { return lib.small_groupnorm(x, ga, be, y, st, N, C, H, W, G, eps, act, Cb, ws, size, s); });)
ENTRY(groupnorm_grad, 17, const int N = r.i(8), C = r.i(9), H = r.i(10), W = r.i(11), G = r.i(12), act = r.i(13), Cb = r.i(14);
      size_t size; void *ws = r.bytes(15, &size);
      auto *x = r.f32(0); auto *ga = r.f32(1); auto *be = r.f32(2); auto *st = r.f32(3); auto *dy = r.f32(4); auto *dx = r.f32(5); auto *dg = r.f32(6); auto *db = r.f32(7);
      const long long all = (long long)N * C * H * W; r.holds(0, all); r.holds(1, C); r.holds(2, C); r.holds(3, 2LL * N * G); r.holds(4, all); r.holds(5, all); r.holds(6, C); r.holds(7, C);
      return r.call([&](void *s) { return lib.small_groupnorm_grad(x, ga, be, st, dy, dx, dg, db, N, C, H, W, G, act, Cb, ws, size, s); });)

// (record, q, k, v, out, lse, workspace, lengths, first, prefix, docs, slopes, table, bucket, stream): of a plan
ENTRY(attention, 15, small_attn rec = r.record(0); const long cq = (long)rec.heads * rec.D, ck = (long)rec.kv_heads * rec.D;
      size_t size; void *ws = r.bytes(6, &size);
      r.masks(7, rec);
      auto *q = r.view(1, rec, rec.Sq, cq, &rec.q); auto *k = r.view(2, rec, rec.Sk, ck, &rec.k); auto *v = r.view(3, rec, rec.Sk, ck, &rec.v);
      auto *o = r.view(4, rec, rec.Sq, cq, &rec.out); auto *l = r.of<float>(5, at::kFloat, {rec.N, rec.heads, rec.Sq});
      return r.call([&](void *s) { return lib.small_attention(&rec, q, k, v, o, l, ws, size, s); });)
// (record, q, k, v, out, lse, dout, dq, dk, dv, dtable, workspace, the same masks, stream)
ENTRY(attention_grad, 20, small_attn rec = r.record(0); const long cq = (long)rec.heads * rec.D, ck = (long)rec.kv_heads * rec.D;
      size_t size; void *ws = r.bytes(11, &size);
      r.masks(12, rec);
      auto *q = r.view(1, rec, rec.Sq, cq, &rec.q); auto *k = r.view(2, rec, rec.Sk, ck, &rec.k); auto *v = r.view(3, rec, rec.Sk, ck, &rec.v);
      auto *o = r.view(4, rec, rec.Sq, cq, &rec.out); auto *l = r.of<float>(5, at::kFloat, {rec.N, rec.heads, rec.Sq});
      auto *d = r.view(6, rec, rec.Sq, cq, &rec.dout); auto *dq = r.view(7, rec, rec.Sq, cq, &rec.dq);
      auto *dk = r.view(8, rec, rec.Sk, ck, &rec.dk); auto *dv = r.view(9, rec, rec.Sk, ck, &rec.dv);
      auto *dt = r.of<float>(10, at::kFloat, {rec.heads, rec.buckets});
      return r.call([&](void *s) { return lib.small_attention_grad(&rec, q, k, v, o, l, d, dq, dk, dv, dt, ws, size, s); });)

// (record, q, k, freq, positions, first, q_out, k_out, stream): q_out, k_out None: in place
ENTRY(rotary, 9, small_rotation rec = r.record<small_rotation>(0, rotation_type); const long cq = (long)rec.heads * rec.D, ck = (long)rec.kv_heads * rec.D;
      r.places(3, rec); rec.first = r.of<int>(5, at::kInt, {rec.N});
      auto *q = r.view(1, rec.N, rec.S, rec.Cb, cq, &rec.q, true); auto *k = r.view(2, rec.N, rec.S, rec.Cb, ck, &rec.k, true);
      auto *qo = r.view(args[6] == Py_None ? 1 : 6, rec.N, rec.S, rec.Cb, cq, &rec.q_out, true);
      auto *ko = r.view(args[7] == Py_None ? 2 : 7, rec.N, rec.S, rec.Cb, ck, &rec.k_out, true);
      return r.call([&](void *s) { return lib.small_rotary(&rec, q, k, qo, ko, s); });)
// (record, dq_out, dk_out, freq, positions, first, dq, dk, q, k, dfreq, workspace, from_inputs, stream)
ENTRY(rotary_grad, 14, small_rotation rec = r.record<small_rotation>(0, rotation_type); rec.from_inputs = r.i(12); const long cq = (long)rec.heads * rec.D, ck = (long)rec.kv_heads * rec.D;
      size_t size; void *ws = r.bytes(11, &size);
      r.places(3, rec); rec.first = r.of<int>(5, at::kInt, {rec.N});
      auto *dqo = r.view(1, rec.N, rec.S, rec.Cb, cq, &rec.q_out, true); auto *dko = r.view(2, rec.N, rec.S, rec.Cb, ck, &rec.k_out, true);
      auto *dq = r.view(args[6] == Py_None ? 1 : 6, rec.N, rec.S, rec.Cb, cq, &rec.dq, true);
      auto *dk = r.view(args[7] == Py_None ? 2 : 7, rec.N, rec.S, rec.Cb, ck, &rec.dk, true);
      auto *q = r.view(8, rec.N, rec.S, rec.Cb, cq, &rec.q, true); auto *k = r.view(9, rec.N, rec.S, rec.Cb, ck, &rec.k, true);
      auto *df = r.of<float>(10, at::kFloat, {rec.freq_heads, rec.axes, rec.pairs});
      return r.call([&](void *s) { return lib.small_rotary_grad(&rec, dqo, dko, q, k, dq, dk, df, ws, size, s); });)
// (cache, k, v, pages, first, counts, rotation or None, freq, positions, q, q_out, stream)
ENTRY(cache_write, 12, small_cache c = r.record<small_cache>(0, cache_type); small_span sp = {}; int N = 0;
      r.sizes(1, &N, &sp.S, &sp.Cb); r.pages(3, N, c);
      sp.first = r.of<int>(4, at::kInt, {N}); sp.counts = r.of<int>(5, at::kInt, {N});
      const long ck = (long)c.kv_heads * c.D; const bool turn = r.plain && args[6] != Py_None;
      auto *k = r.view(1, N, sp.S, sp.Cb, ck, &sp.k); auto *v = r.view(2, N, sp.S, sp.Cb, ck, &sp.v);
      small_rotation rec = {}; float *q = nullptr, *qo = nullptr;
      if (turn) {
          rec = r.record<small_rotation>(6, rotation_type);
          r.places(7, rec);
          rec.first = nullptr;
          rec.k = rec.k_out = small_tokens{};
          q = r.view(9, rec.N, rec.S, rec.Cb, (long)rec.heads * rec.D, &rec.q, true);
          qo = r.view(args[10] == Py_None ? 9 : 10, rec.N, rec.S, rec.Cb, (long)rec.heads * rec.D, &rec.q_out, true);
      } else if (r.plain && args[9] != Py_None) {
          r.plain = false;
      }
      return r.call([&](void *s) { return lib.small_cache_write(&c, &sp, k, v, turn ? &rec : nullptr, q, qo, s); });)
// (cache, k, v, pages, first, counts, stream)
ENTRY(cache_read, 7, small_cache c = r.record<small_cache>(0, cache_type); small_span sp = {}; int N = 0;
      r.sizes(1, &N, &sp.S, &sp.Cb); r.pages(3, N, c);
      sp.first = r.of<int>(4, at::kInt, {N}); sp.counts = r.of<int>(5, at::kInt, {N});
      const long ck = (long)c.kv_heads * c.D;
      auto *k = r.view(1, N, sp.S, sp.Cb, ck, &sp.k); auto *v = r.view(2, N, sp.S, sp.Cb, ck, &sp.v);
      return r.call([&](void *s) { return lib.small_cache_read(&c, &sp, k, v, s); });)
// (cache, record, q, out, lse, workspace, pages, lengths, first, slopes, table, bucket, stream)
ENTRY(cache_attention, 13, small_cache c = r.record<small_cache>(0, cache_type); small_attn rec = r.record<small_attn>(1, attn_type); const long cq = (long)rec.heads * rec.D;
      size_t size; void *ws = r.bytes(5, &size);
      r.pages(6, rec.N, c);
      if (r.plain && (long)c.per_stream * c.page != rec.Sk) r.plain = false;
      rec.lengths = r.of<int>(7, at::kInt, {rec.N}); rec.first = r.of<int>(8, at::kInt, {rec.N}); rec.slopes = r.of<float>(9, at::kFloat, {rec.heads});
      rec.table = r.of<float>(10, at::kFloat, {rec.heads, rec.buckets}); rec.bucket = r.of<int>(11, at::kInt, {2L * rec.reach + 1});
      rec.prefix = rec.docs = nullptr;
      auto *q = r.view(2, rec, rec.Sq, cq, &rec.q); auto *o = r.view(3, rec, rec.Sq, cq, &rec.out);
      auto *l = r.of<float>(4, at::kFloat, {rec.N, rec.heads, rec.Sq});
      return r.call([&](void *s) { return lib.small_cache_attention(&c, &rec, q, o, l, ws, size, s); });)

// bind_cache(cache's small_rotation and small_cache)
PyObject *bind_cache(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 2 || !PyType_Check(args[0]) || !PyType_Check(args[1])) {
        PyErr_SetString(PyExc_TypeError, "bind_cache(small_rotation, small_cache)");
        return nullptr;
    }
    Py_INCREF(args[0]);                    // (kept for the module's life)
    Py_INCREF(args[1]);
    rotation_type = reinterpret_cast<PyTypeObject *>(args[0]);
    cache_type = reinterpret_cast<PyTypeObject *>(args[1]);
    Py_RETURN_NONE;
}

// bind_attention(attn's small_attn)
PyObject *bind_attention(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 1 || !PyType_Check(args[0])) {
        PyErr_SetString(PyExc_TypeError, "bind_attention(small_attn)");
        return nullptr;
    }
    Py_INCREF(args[0]);                    // (kept for the module's life)
    attn_type = reinterpret_cast<PyTypeObject *>(args[0]);
    Py_RETURN_NONE;
}

// bind(handle of the loaded library, the binding's small_quant)
PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 2 || !PyLong_Check(args[0]) || !PyType_Check(args[1])) {
        PyErr_SetString(PyExc_TypeError, "bind(handle, small_quant)");
        return nullptr;
    }
    void *handle = PyLong_AsVoidPtr(args[0]);
    if (!handle) return nullptr;
#define X(f)                                                        \
    lib.f = reinterpret_cast<decltype(&::f)>(dlsym(handle, #f));    \
    if (!lib.f) {                                                   \
        lib.small_relu = nullptr;                                   \
        PyErr_SetString(PyExc_AttributeError, #f);                  \
        return nullptr;                                             \
    }
    SMALL_FUNCTIONS(X)
#undef X
    Py_INCREF(args[1]);                    // (kept for the module's life)
    quant_type = reinterpret_cast<PyTypeObject *>(args[1]);
    Py_RETURN_NONE;
}

#define METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(bind), METHOD(pack), METHOD(unpack), METHOD(pack_u8), METHOD(unpack_u8), METHOD(conv2d), METHOD(conv2d_u8),
                         METHOD(dwconv2d), METHOD(dwconv2d_u8), METHOD(pool2d), METHOD(pool2d_u8), METHOD(relu), METHOD(relu_u8), METHOD(add),
                         METHOD(dense), METHOD(dense_u8), METHOD(groupnorm), METHOD(groupnorm_grad), METHOD(attention), METHOD(attention_grad),
                         METHOD(bind_attention), METHOD(rotary), METHOD(rotary_grad), METHOD(cache_write), METHOD(cache_read), METHOD(cache_attention),
                         METHOD(bind_cache), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() { return PyModule_Create(&module); }
