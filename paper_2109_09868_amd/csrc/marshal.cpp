// Argument marshalling of the binding's calls in their ordinary form: exact torch tensors in device memory of the right type,
// shape and contiguity, float64 node arrays, Python ints, outputs given, torch's current stream.  Anything else returns None and
// the binding's own checks take over (they raise, convert or allocate), so what is accepted and refused is decided there.
// Bound by host time: a decode of 64 groups took 6.8 us to enqueue, 3.4 of it in Python around the 3.4 of call and launch.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>

#include "approxifer.h"

namespace {

struct Library {
    decltype(&approxifer_encode) encode;
    decltype(&approxifer_decode) decode;
    decltype(&approxifer_decode_top1) decode_top1;
    decltype(&approxifer_decode_byzantine) byzantine;
    decltype(&approxifer_decode_byzantine_homogeneous) homogeneous;
    decltype(&approxifer_pad_last_group) pad_last_group;
    decltype(&approxifer_top1) top1;
    decltype(&approxifer_wait_mask) wait_mask;
    decltype(&approxifer_append) append;
    decltype(&approxifer_attend) attend;
    decltype(&approxifer_cache_reserve) cache_reserve;
    decltype(&approxifer_cache_fork) cache_fork;
    decltype(&approxifer_cache_compact) cache_compact;
    decltype(&approxifer_cache_evict) cache_evict;
    decltype(&approxifer_attend_mass) attend_mass;
    decltype(&approxifer_attend_shared) attend_shared;
};

// The handle of a loaded library: its entry points, by address, in the order above.
constexpr const char *kCapsule = "approxifer.library";
const Library *library(PyObject *o) { return static_cast<const Library *>(PyCapsule_GetPointer(o, kCapsule)); }

PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n) {
    constexpr int kEntries = sizeof(Library) / sizeof(void *);
    if (n != kEntries) {
        PyErr_SetString(PyExc_TypeError, "expected an address for every entry point");
        return nullptr;
    }
    void *p[kEntries];
    for (int i = 0; i < kEntries; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    Library *lib = new Library{
        reinterpret_cast<decltype(Library::encode)>(p[0]),         reinterpret_cast<decltype(Library::decode)>(p[1]),
        reinterpret_cast<decltype(Library::decode_top1)>(p[2]),    reinterpret_cast<decltype(Library::byzantine)>(p[3]),
        reinterpret_cast<decltype(Library::homogeneous)>(p[4]),    reinterpret_cast<decltype(Library::pad_last_group)>(p[5]),
        reinterpret_cast<decltype(Library::top1)>(p[6]),           reinterpret_cast<decltype(Library::wait_mask)>(p[7]),
        reinterpret_cast<decltype(Library::append)>(p[8]),         reinterpret_cast<decltype(Library::attend)>(p[9]),
        reinterpret_cast<decltype(Library::cache_reserve)>(p[10]), reinterpret_cast<decltype(Library::cache_fork)>(p[11]),
        reinterpret_cast<decltype(Library::cache_compact)>(p[12]), reinterpret_cast<decltype(Library::cache_evict)>(p[13]),
        reinterpret_cast<decltype(Library::attend_mass)>(p[14]),   reinterpret_cast<decltype(Library::attend_shared)>(p[15])};
    PyObject *c = PyCapsule_New(lib, kCapsule, [](PyObject *o) { delete static_cast<Library *>(PyCapsule_GetPointer(o, kCapsule)); });
    if (c == nullptr) delete lib;
    return c;
}

// A plain device tensor: no subclass, no wrapper of a transform or mode, strided.
const at::Tensor *device_tensor(PyObject *o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided) return nullptr;
    const c10::TensorImpl *impl = t.unsafeGetTensorImpl();
    const c10::DispatchKeySet keys = impl->key_set();
    if (!impl->has_storage() || impl->is_python_dispatch() || keys.has(c10::DispatchKey::FuncTorchBatched) ||
        keys.has(c10::DispatchKey::FuncTorchGradWrapper) || keys.has(c10::DispatchKey::Functionalize) ||
        keys.has(c10::DispatchKey::ZeroTensor) || impl->has_symbolic_sizes_strides())
        return nullptr;
    return &t;
}
// One of this type that is contiguous too.
const at::Tensor *plain(PyObject *o, at::ScalarType type) {
    const at::Tensor *t = device_tensor(o);
    return t != nullptr && t->scalar_type() == type && t->is_contiguous() ? t : nullptr;
}
template <class... Size>
void *shaped(PyObject *o, at::ScalarType type, Size... sizes) {
    const at::Tensor *t = plain(o, type);
    const int64_t want[] = {static_cast<int64_t>(sizes)...};
    if (t == nullptr || t->dim() != static_cast<int64_t>(sizeof...(sizes))) return nullptr;
    for (size_t d = 0; d < sizeof...(sizes); ++d)
        if (t->size(d) != want[d]) return nullptr;
    return t->data_ptr();
}

bool integer(PyObject *o, int &v) {
    if (!PyLong_Check(o)) return false;
    int over = 0;
    const long x = PyLong_AsLongAndOverflow(o, &over);
    if (over != 0 || x != static_cast<int>(x)) return false;
    v = static_cast<int>(x);
    return true;
}

// A float64 array in host memory, held for the call.
struct Nodes {
    Py_buffer b{};
    bool held = false;
    explicit Nodes(PyObject *o) {
        if (PyObject_GetBuffer(o, &b, PyBUF_FORMAT | PyBUF_C_CONTIGUOUS) != 0) {
            PyErr_Clear();
            return;
        }
        held = true;
    }
    ~Nodes() {
        if (held) PyBuffer_Release(&b);
    }
    bool ok() const { return held && b.itemsize == 8 && b.format != nullptr && b.format[0] == 'd' && b.format[1] == '\0'; }
    int64_t size() const { return b.len / 8; }
    const double *data() const { return static_cast<const double *>(b.buf); }
};

void *current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// The call itself without the interpreter lock, as ctypes makes it; its status as a Python int.
template <class F>
PyObject *status_of(F call) {
    int rc;
    void *stream = current_stream();                          // may throw: not without the lock
    Py_BEGIN_ALLOW_THREADS
    rc = call(stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

constexpr at::ScalarType kF32 = at::kFloat, kI32 = at::kInt, kU8 = at::kByte;

// (library, queries, alpha, beta, coded)
PyObject *encode(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 5 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    const Nodes al(a[2]), be(a[3]);
    const at::Tensor *q = plain(a[1], kF32);
    if (q == nullptr || !al.ok() || !be.ok() || q->dim() != 3 || q->size(1) != al.size()) Py_RETURN_NONE;
    const int64_t G = q->size(0), K = q->size(1), D = q->size(2), N = be.size();
    void *coded = shaped(a[4], kF32, G, N, D);
    void *queries = q->data_ptr();
    if (coded == nullptr || queries == nullptr) Py_RETURN_NONE;
    return status_of([&](void *s) {
        return lib->encode(static_cast<const float *>(queries), static_cast<float *>(coded), G, static_cast<int>(K),
                           static_cast<int>(N), D, al.data(), be.data(), s);
    });
}

struct Decode {
    int64_t G, N, C, K;
    void *preds, *mask, *status;
    int S, sign;
    bool ok;
    Decode(PyObject *p, PyObject *m, const Nodes &al, const Nodes &be, PyObject *s, PyObject *g, PyObject *st) : ok(false) {
        const at::Tensor *t = plain(p, kF32);
        if (t == nullptr || !al.ok() || !be.ok() || t->dim() != 3 || t->size(1) != be.size()) return;
        G = t->size(0);
        N = t->size(1);
        C = t->size(2);
        K = al.size();
        preds = t->data_ptr();
        mask = shaped(m, kU8, G, N);
        status = shaped(st, kI32, G);
        ok = preds != nullptr && mask != nullptr && status != nullptr && integer(s, S) && integer(g, sign);
    }
};

// (library, preds, mask, alpha, beta, S, sign_mode, out, status)
PyObject *decode(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 9 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    const Nodes al(a[3]), be(a[4]);
    const Decode d(a[1], a[2], al, be, a[5], a[6], a[8]);
    void *out = d.ok ? shaped(a[7], kF32, d.G, d.K, d.C) : nullptr;
    if (out == nullptr) Py_RETURN_NONE;
    return status_of([&](void *s) {
        return lib->decode(static_cast<const float *>(d.preds), static_cast<const uint8_t *>(d.mask), static_cast<float *>(out),
                           static_cast<int32_t *>(d.status), d.G, static_cast<int>(d.K), static_cast<int>(d.N), d.S, d.C,
                           al.data(), be.data(), d.sign, s);
    });
}

// (library, preds, mask, alpha, beta, S, sign_mode, top1, score or None, status)
PyObject *decode_top1(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 10 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    const Nodes al(a[3]), be(a[4]);
    const Decode d(a[1], a[2], al, be, a[5], a[6], a[9]);
    void *top1 = d.ok ? shaped(a[7], kI32, d.G, d.K) : nullptr;
    if (top1 == nullptr) Py_RETURN_NONE;
    void *score = nullptr;
    if (a[8] != Py_None && (score = shaped(a[8], kF32, d.G, d.K)) == nullptr) Py_RETURN_NONE;
    return status_of([&](void *s) {
        return lib->decode_top1(static_cast<const float *>(d.preds), static_cast<const uint8_t *>(d.mask),
                                static_cast<int32_t *>(top1), static_cast<float *>(score), static_cast<int32_t *>(d.status), d.G,
                                static_cast<int>(d.K), static_cast<int>(d.N), d.S, d.C, al.data(), be.data(), d.sign, s);
    });
}

// (library, homogeneous, preds, mask, alpha, beta, S, A, sign_mode, out, adv, status, workspace or None)
PyObject *byzantine(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 13 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    const Nodes al(a[4]), be(a[5]);
    const Decode d(a[2], a[3], al, be, a[6], a[8], a[11]);
    int A = 0;
    if (!d.ok || !integer(a[7], A) || A < 1) Py_RETURN_NONE;
    void *out = shaped(a[9], kF32, d.G, d.K, d.C);
    void *adv = shaped(a[10], kI32, d.G, A);
    if (out == nullptr || adv == nullptr) Py_RETURN_NONE;
    void *ws = nullptr;
    size_t ws_bytes = 0;
    if (a[12] != Py_None) {
        const at::Tensor *w = plain(a[12], kU8);
        if (w == nullptr) Py_RETURN_NONE;
        ws = w->data_ptr();
        ws_bytes = static_cast<size_t>(w->numel());
    }
    const auto entry = a[1] == Py_True ? lib->homogeneous : lib->byzantine;
    return status_of([&](void *s) {
        return entry(static_cast<const float *>(d.preds), static_cast<const uint8_t *>(d.mask), static_cast<float *>(out),
                     static_cast<int32_t *>(adv), static_cast<int32_t *>(d.status), d.G, static_cast<int>(d.K),
                     static_cast<int>(d.N), d.S, A, d.C, al.data(), be.data(), d.sign, ws, ws_bytes, s);
    });
}

// (library, buffer, Q, K): buffer [rows, D] with rows >= ceil(Q / K) K
PyObject *pad_last_group(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 4 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    const at::Tensor *b = plain(a[1], kF32);
    int Q = 0, K = 0;
    if (b == nullptr || b->dim() != 2 || !integer(a[2], Q) || !integer(a[3], K) || Q < 1 || K < 1) Py_RETURN_NONE;
    const int64_t G = (static_cast<int64_t>(Q) + K - 1) / K;
    void *p = b->data_ptr();
    if (b->size(0) < G * K || p == nullptr) Py_RETURN_NONE;
    const int64_t D = b->size(1);
    return status_of([&](void *s) { return lib->pad_last_group(static_cast<float *>(p), Q, K, D, s); });
}

// (library, values [rows.., C], top1 [rows..], score or None)
PyObject *top1(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 4 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    const at::Tensor *v = plain(a[1], kF32), *t = plain(a[2], kI32);
    if (v == nullptr || t == nullptr || v->dim() < 1 || v->sizes().slice(0, v->dim() - 1) != t->sizes()) Py_RETURN_NONE;
    const at::Tensor *sc = a[3] == Py_None ? nullptr : plain(a[3], kF32);
    if (a[3] != Py_None && (sc == nullptr || sc->sizes() != t->sizes())) Py_RETURN_NONE;
    const int64_t C = v->size(v->dim() - 1), rows = t->numel();
    void *vp = v->data_ptr(), *tp = t->data_ptr(), *sp = sc != nullptr ? sc->data_ptr() : nullptr;
    if (vp == nullptr || tp == nullptr || (sc != nullptr && sp == nullptr)) Py_RETURN_NONE;
    return status_of([&](void *s) {
        return lib->top1(static_cast<const float *>(vp), static_cast<int32_t *>(tp), static_cast<float *>(sp), rows, C, s);
    });
}

// (library, arrival, wait_for, mask, count)
PyObject *wait_mask(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 5 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    const at::Tensor *t = plain(a[1], kF32);
    int wait_for = 0;
    if (t == nullptr || t->dim() != 2 || !integer(a[2], wait_for)) Py_RETURN_NONE;
    const int64_t G = t->size(0), N = t->size(1);
    void *arrival = t->data_ptr(), *mask = shaped(a[3], kU8, G, N), *count = shaped(a[4], kI32, G);
    if (arrival == nullptr || mask == nullptr || count == nullptr) Py_RETURN_NONE;
    return status_of([&](void *s) {
        return lib->wait_mask(static_cast<const float *>(arrival), static_cast<uint8_t *>(mask), static_cast<int32_t *>(count), G,
                              static_cast<int>(N), wait_for, s);
    });
}

// ---- sequences in pages ----
bool integer64(PyObject *o, int64_t &v) {
    if (!PyLong_Check(o)) return false;
    int over = 0;
    const long long x = PyLong_AsLongLongAndOverflow(o, &over);
    v = x;
    return over == 0;
}
bool real(PyObject *o, double &v) {
    if (!PyFloat_Check(o)) return false;
    v = PyFloat_AS_DOUBLE(o);
    return true;
}

int dtype_of(const at::Tensor *t) {
    switch (t->scalar_type()) {
        case at::kFloat: return APPROXIFER_F32;
        case at::kHalf: return APPROXIFER_F16;
        case at::kBFloat16: return APPROXIFER_BF16;
        default: return -1;
    }
}

// [T, heads, Dh] whose tokens are contiguous, at any distance.
struct TokenRows {
    void *data = nullptr;
    int64_t T = 0, heads = 0, Dh = 0, stride = 0;
    TokenRows(PyObject *o, at::ScalarType type) {
        const at::Tensor *t = device_tensor(o);
        if (t == nullptr || t->scalar_type() != type || t->dim() != 3) return;
        T = t->size(0);
        heads = t->size(1);
        Dh = t->size(2);
        if ((Dh > 1 && t->stride(2) != 1) || (heads > 1 && t->stride(1) != Dh)) return;
        stride = T > 1 ? t->stride(0) : heads * Dh;
        data = t->data_ptr();
    }
};

// Pools and descriptor of a call.
struct Cache {
    approxifer_sequences seq{};
    void *k = nullptr, *v = nullptr;
    int Hkv = 0, Dh = 0, dtype = -1;
    at::ScalarType type = at::kFloat;
    bool ok = false;
    Cache(PyObject *kp, PyObject *vp, PyObject *table, PyObject *lens, PyObject *starts) {
        const at::Tensor *p = device_tensor(kp);
        if (p == nullptr || p->dim() != 4 || !p->is_contiguous() || (dtype = dtype_of(p)) < 0) return;
        type = p->scalar_type();
        const at::Tensor *t = plain(table, kI32);
        if (t == nullptr || t->dim() != 2) return;
        if (p->size(1) > APPROXIFER_MAX_HEADS || p->size(2) > APPROXIFER_MAX_PAGE || p->size(3) > APPROXIFER_MAX_HEAD_DIM) return;
        seq.B = t->size(0);
        seq.M = t->size(1);
        seq.P = p->size(0);
        seq.page = static_cast<int32_t>(p->size(2));
        Hkv = static_cast<int>(p->size(1));
        Dh = static_cast<int>(p->size(3));
        k = p->data_ptr();
        v = shaped(vp, type, p->size(0), p->size(1), p->size(2), p->size(3));
        seq.d_table = static_cast<const int32_t *>(t->data_ptr());
        seq.d_lens = static_cast<const int32_t *>(shaped(lens, kI32, seq.B));
        seq.d_starts = static_cast<const int32_t *>(shaped(starts, kI32, seq.B + 1));
        ok = k != nullptr && v != nullptr && seq.d_table != nullptr && seq.d_lens != nullptr && seq.d_starts != nullptr;
    }
};

// (library, q, k, v, k_pool, v_pool, table, lens, starts, freq, q_weight or None, k_weight or None, eps, positions or None, axis or None,
//  interleaved, q_out, status)
PyObject *append(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 18 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    Cache c(a[4], a[5], a[6], a[7], a[8]);
    if (!c.ok) Py_RETURN_NONE;
    const TokenRows q(a[1], c.type), k(a[2], c.type), v(a[3], c.type);
    const int64_t T = q.T, Hq = q.heads;
    if (q.data == nullptr || k.data == nullptr || v.data == nullptr || q.Dh != c.Dh || k.Dh != c.Dh || v.Dh != c.Dh || k.T != T ||
        v.T != T || k.heads != c.Hkv || v.heads != c.Hkv || Hq > APPROXIFER_MAX_HEADS)
        Py_RETURN_NONE;
    const Nodes freq(a[9]);
    if (!freq.ok() || freq.size() > APPROXIFER_MAX_HEAD_DIM) Py_RETURN_NONE;
    void *qw = nullptr, *kw = nullptr, *positions = nullptr;
    if (a[10] != Py_None && (qw = shaped(a[10], c.type, c.Dh)) == nullptr) Py_RETURN_NONE;
    if (a[11] != Py_None && (kw = shaped(a[11], c.type, c.Dh)) == nullptr) Py_RETURN_NONE;
    double eps = 0.0;
    if (!real(a[12], eps) || !PyBool_Check(a[15])) Py_RETURN_NONE;    // other truth values are the binding's to read
    int axes = 1;
    if (a[13] != Py_None) {
        const at::Tensor *p = plain(a[13], kI32);
        if (p == nullptr || p->dim() != 2 || p->size(0) != T || p->size(1) > APPROXIFER_MAX_AXES) Py_RETURN_NONE;
        axes = static_cast<int>(p->size(1));
        positions = p->data_ptr();
    }
    Py_buffer axis{};
    if (a[14] != Py_None) {
        if (PyObject_GetBuffer(a[14], &axis, PyBUF_FORMAT | PyBUF_C_CONTIGUOUS) != 0) {
            PyErr_Clear();
            Py_RETURN_NONE;
        }
        if (axis.itemsize != 4 || axis.format == nullptr || axis.format[0] != 'i' || axis.len / 4 != freq.size()) {
            PyBuffer_Release(&axis);
            Py_RETURN_NONE;
        }
    }
    PyObject *done = nullptr;
    void *out = shaped(a[16], c.type, T, Hq, c.Dh), *status = shaped(a[17], kI32, c.seq.B);
    if (out != nullptr && status != nullptr) {
        c.seq.T = T;
        const int turned = a[15] == Py_True;
        done = status_of([&](void *s) {
            return lib->append(&c.seq, static_cast<int>(Hq), c.Hkv, c.Dh, c.dtype, q.data, q.stride, k.data, k.stride, v.data, v.stride, out,
                               c.k, c.v, qw, kw, eps, static_cast<const int32_t *>(positions), axes, freq.data(),
                               static_cast<const int32_t *>(axis.buf), static_cast<int>(freq.size()), turned,
                               static_cast<int32_t *>(status), s);
        });
    }
    if (axis.obj != nullptr) PyBuffer_Release(&axis);
    if (done == nullptr && !PyErr_Occurred()) Py_RETURN_NONE;
    return done;
}

// (library, q, k_pool, v_pool, table, lens, starts, max_rows, max_len, window, sinks, scale or None, out, status, workspace or None)
PyObject *attend(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 15 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    Cache c(a[2], a[3], a[4], a[5], a[6]);
    if (!c.ok) Py_RETURN_NONE;
    const TokenRows q(a[1], c.type);
    int64_t rows, length, window, sinks;
    if (q.data == nullptr || q.Dh != c.Dh || q.heads > APPROXIFER_MAX_HEADS || !integer64(a[7], rows) || !integer64(a[8], length) ||
        !integer64(a[9], window) || !integer64(a[10], sinks))
        Py_RETURN_NONE;
    double scale = 1.0 / std::sqrt(static_cast<double>(c.Dh));
    if (a[11] != Py_None && !real(a[11], scale)) Py_RETURN_NONE;
    void *out = shaped(a[12], c.type, q.T, q.heads, q.Dh), *status = shaped(a[13], kI32, c.seq.B);
    if (out == nullptr || status == nullptr) Py_RETURN_NONE;
    const at::Tensor *w = a[14] == Py_None ? nullptr : plain(a[14], kU8);
    if (a[14] != Py_None && w == nullptr) Py_RETURN_NONE;
    void *ws = w != nullptr ? w->data_ptr() : nullptr;
    const size_t ws_bytes = w != nullptr ? static_cast<size_t>(w->numel()) : 0;
    c.seq.T = q.T;
    return status_of([&](void *s) {
        return lib->attend(&c.seq, static_cast<int>(q.heads), c.Hkv, c.Dh, c.dtype, q.data, q.stride, c.k, c.v, out, rows, length, window,
                           sinks, scale, static_cast<int32_t *>(status), ws, ws_bytes, s);
    });
}

// (library, q, k_pool, v_pool, table, lens, starts, mass, max_rows, max_len, window, sinks, scale or None, out, status, workspace or None)
PyObject *attend_mass(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 16 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    Cache c(a[2], a[3], a[4], a[5], a[6]);
    if (!c.ok) Py_RETURN_NONE;
    const TokenRows q(a[1], c.type);
    const at::Tensor *m = plain(a[7], kF32), *w = a[15] == Py_None ? nullptr : plain(a[15], kU8);
    int64_t rows, length, window, sinks;
    if (q.data == nullptr || q.Dh != c.Dh || q.heads > APPROXIFER_MAX_HEADS || !integer64(a[8], rows) || !integer64(a[9], length) ||
        !integer64(a[10], window) || !integer64(a[11], sinks) || m == nullptr || m->dim() != 2 || m->size(0) != c.seq.B ||
        (a[15] != Py_None && w == nullptr))
        Py_RETURN_NONE;
    double scale = 1.0 / std::sqrt(static_cast<double>(c.Dh));
    if (a[12] != Py_None && !real(a[12], scale)) Py_RETURN_NONE;
    void *out = shaped(a[13], c.type, q.T, q.heads, q.Dh), *status = shaped(a[14], kI32, c.seq.B), *mass = m->data_ptr();
    if (out == nullptr || status == nullptr || mass == nullptr) Py_RETURN_NONE;
    const int64_t stride = m->size(1);
    void *ws = w != nullptr ? w->data_ptr() : nullptr;
    const size_t ws_bytes = w != nullptr ? static_cast<size_t>(w->numel()) : 0;
    c.seq.T = q.T;
    return status_of([&](void *s) {
        return lib->attend_mass(&c.seq, static_cast<int>(q.heads), c.Hkv, c.Dh, c.dtype, q.data, q.stride, c.k, c.v, out,
                                static_cast<float *>(mass), stride, rows, length, window, sinks, scale, static_cast<int32_t *>(status), ws,
                                ws_bytes, s);
    });
}

// (library, q, k_pool, v_pool, table, lens, starts, groups, shared, max_rows, max_len, max_shared, window, sinks, scale or None, out, status,
//  workspace or None)
PyObject *attend_shared(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 18 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    Cache c(a[2], a[3], a[4], a[5], a[6]);
    if (!c.ok) Py_RETURN_NONE;
    const TokenRows q(a[1], c.type);
    const at::Tensor *length = plain(a[8], kI32), *w = a[17] == Py_None ? nullptr : plain(a[17], kU8);
    int64_t rows, most, common, window, sinks;
    if (q.data == nullptr || q.Dh != c.Dh || q.heads > APPROXIFER_MAX_HEADS || !integer64(a[9], rows) || !integer64(a[10], most) ||
        !integer64(a[11], common) || !integer64(a[12], window) || !integer64(a[13], sinks) || length == nullptr || length->dim() != 1 ||
        (a[17] != Py_None && w == nullptr))
        Py_RETURN_NONE;
    double scale = 1.0 / std::sqrt(static_cast<double>(c.Dh));
    if (a[14] != Py_None && !real(a[14], scale)) Py_RETURN_NONE;
    const int64_t C = length->numel();
    void *groups = shaped(a[7], kI32, C + 1), *shared = length->data_ptr(), *out = shaped(a[15], c.type, q.T, q.heads, q.Dh),
         *status = shaped(a[16], kI32, c.seq.B);
    if (groups == nullptr || shared == nullptr || out == nullptr || status == nullptr) Py_RETURN_NONE;
    void *ws = w != nullptr ? w->data_ptr() : nullptr;
    const size_t ws_bytes = w != nullptr ? static_cast<size_t>(w->numel()) : 0;
    c.seq.T = q.T;
    return status_of([&](void *s) {
        return lib->attend_shared(&c.seq, static_cast<int>(q.heads), c.Hkv, c.Dh, c.dtype, q.data, q.stride, c.k, c.v, out,
                                  static_cast<const int32_t *>(groups), static_cast<const int32_t *>(shared), C, rows, most, common, window,
                                  sinks, scale, static_cast<int32_t *>(status), ws, ws_bytes, s);
    });
}

int32_t *ints(void *p) { return static_cast<int32_t *>(p); }

// (library, table, lens, refs, add, page, status)
PyObject *cache_reserve(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 7 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    const at::Tensor *t = plain(a[1], kI32), *r = plain(a[3], kI32);
    int page = 0;
    if (t == nullptr || r == nullptr || t->dim() != 2 || !integer(a[5], page)) Py_RETURN_NONE;
    const int64_t B = t->size(0), M = t->size(1), P = r->numel();
    void *lens = shaped(a[2], kI32, B), *add = shaped(a[4], kI32, B), *status = shaped(a[6], kI32, B);
    void *table = t->data_ptr(), *refs = r->data_ptr();
    if (lens == nullptr || add == nullptr || status == nullptr || table == nullptr || refs == nullptr) Py_RETURN_NONE;
    return status_of([&](void *s) { return lib->cache_reserve(ints(table), ints(lens), ints(refs), ints(add), ints(status), B, M, P, page, s); });
}

// Pools [.., P, Hkv, page, Dh] of any type, table, lens, refs and workspace.
struct Pages {
    int64_t B = 0, M = 0, P = 0, planes = 0, page_bytes = 0, heads = 0;
    int page = 0;
    void *pools = nullptr, *table = nullptr, *lens = nullptr, *refs = nullptr, *ws = nullptr;
    size_t ws_bytes = 0;
    bool ok = false;
    Pages(PyObject *p, PyObject *t, PyObject *l, PyObject *r, PyObject *w) {
        const at::Tensor *pool = device_tensor(p), *tab = plain(t, kI32), *ref = plain(r, kI32), *work = plain(w, kU8);
        if (pool == nullptr || tab == nullptr || ref == nullptr || work == nullptr || pool->dim() < 4 || !pool->is_contiguous() ||
            tab->dim() != 2 || pool->numel() == 0 || pool->size(-2) > APPROXIFER_MAX_PAGE)
            return;
        B = tab->size(0);
        M = tab->size(1);
        P = ref->numel();
        if (pool->size(-4) != P) return;
        page = static_cast<int>(pool->size(-2));
        heads = pool->size(-3);
        page_bytes = pool->size(-1) * pool->size(-2) * pool->size(-3) * static_cast<int64_t>(pool->element_size());
        planes = pool->numel() / (pool->size(-1) * pool->size(-2) * pool->size(-3) * P);
        pools = pool->data_ptr();
        table = tab->data_ptr();
        refs = ref->data_ptr();
        lens = shaped(l, kI32, B);
        ws = work->data_ptr();
        ws_bytes = static_cast<size_t>(work->numel());
        ok = table != nullptr && refs != nullptr && lens != nullptr && ws != nullptr;
    }
};

// (library, pools, table, lens, refs, parents, keep or None, table_out, lens_out, refs_out, status, workspace)
PyObject *cache_fork(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 12 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    const Pages c(a[1], a[2], a[3], a[4], a[11]);
    const at::Tensor *p = plain(a[5], kI32);
    if (!c.ok || p == nullptr) Py_RETURN_NONE;
    const int64_t B_out = p->numel();
    void *keep = nullptr;
    if (a[6] != Py_None && (keep = shaped(a[6], kI32, B_out)) == nullptr) Py_RETURN_NONE;
    void *parents = p->data_ptr(), *table = shaped(a[7], kI32, B_out, c.M), *lens = shaped(a[8], kI32, B_out),
         *refs = shaped(a[9], kI32, c.P), *status = shaped(a[10], kI32, B_out);
    if (parents == nullptr || table == nullptr || lens == nullptr || refs == nullptr || status == nullptr) Py_RETURN_NONE;
    return status_of([&](void *s) {
        return lib->cache_fork(ints(c.table), ints(c.lens), ints(c.refs), ints(parents), ints(keep), ints(table), ints(lens), ints(refs),
                               ints(status), c.pools, c.planes, c.page_bytes, c.B, B_out, c.M, c.P, c.page, c.ws, c.ws_bytes, s);
    });
}

// (library, pools, table, lens, refs, moved, live, workspace)
PyObject *cache_compact(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 8 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    const Pages c(a[1], a[2], a[3], a[4], a[7]);
    if (!c.ok) Py_RETURN_NONE;
    void *moved = shaped(a[5], kI32, c.P), *live = shaped(a[6], kI32, 1);
    if (moved == nullptr || live == nullptr) Py_RETURN_NONE;
    return status_of([&](void *s) {
        return lib->cache_compact(ints(c.table), ints(c.lens), ints(c.refs), ints(moved), ints(live), c.pools, c.planes, c.page_bytes, c.B,
                                  c.M, c.P, c.page, c.ws, c.ws_bytes, s);
    });
}

// (library, pools, table, lens, refs, mass, budget, first, recent, kept, status, workspace)
PyObject *cache_evict(PyObject *const *a, Py_ssize_t n) {
    const Library *lib = n == 12 ? library(a[0]) : nullptr;
    if (lib == nullptr) return nullptr;
    const Pages c(a[1], a[2], a[3], a[4], a[11]);
    const at::Tensor *m = plain(a[5], kF32);
    int64_t budget, first, recent;
    if (!c.ok || m == nullptr || m->dim() != 2 || m->size(0) != c.B || !integer64(a[6], budget) || !integer64(a[7], first) ||
        !integer64(a[8], recent))
        Py_RETURN_NONE;
    const int64_t stride = m->size(1);
    void *mass = m->data_ptr(), *kept = shaped(a[9], kI32, c.B, budget), *status = shaped(a[10], kI32, c.B);
    if (mass == nullptr || kept == nullptr || status == nullptr) Py_RETURN_NONE;
    return status_of([&](void *s) {
        return lib->cache_evict(ints(c.table), ints(c.lens), ints(c.refs), static_cast<float *>(mass), stride, ints(kept), ints(status),
                                c.pools, c.planes, c.heads, c.page_bytes / (c.heads * c.page), c.B, c.M, c.P, c.page, budget, first, recent,
                                c.ws, c.ws_bytes, s);
    });
}

// No C++ exception leaves the module: what torch throws makes the call one for the binding's own checks.
template <PyObject *(*F)(PyObject *const *, Py_ssize_t)>
PyObject *guarded(PyObject *, PyObject *const *args, Py_ssize_t n) {
    try {
        PyObject *r = F(args, n);
        if (r == nullptr && !PyErr_Occurred()) PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return r;
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

#define APPROXIFER_METHOD(name) \
    {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<name>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&bind)), METH_FASTCALL, nullptr},
    APPROXIFER_METHOD(encode),    APPROXIFER_METHOD(decode),         APPROXIFER_METHOD(decode_top1),
    APPROXIFER_METHOD(byzantine), APPROXIFER_METHOD(pad_last_group), APPROXIFER_METHOD(top1),
    APPROXIFER_METHOD(wait_mask), APPROXIFER_METHOD(append),         APPROXIFER_METHOD(attend),
    APPROXIFER_METHOD(cache_reserve), APPROXIFER_METHOD(cache_fork), APPROXIFER_METHOD(cache_compact),
    APPROXIFER_METHOD(cache_evict),   APPROXIFER_METHOD(attend_mass),
    APPROXIFER_METHOD(attend_shared),
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the interpreter and the torch whose layouts are compiled in; the binding uses the module with no other.
PyMODINIT_FUNC PyInit__marshal(void) {
    PyObject *m = PyModule_Create(&module);
    if (m != nullptr && PyModule_AddStringConstant(m, "built_for", APPROXIFER_BUILT_FOR) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
