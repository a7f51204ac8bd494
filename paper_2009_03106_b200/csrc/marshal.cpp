// Argument marshalling of the transformer-block entry points, as a Python module: checks tensors and hands their addresses, sizes and
// strides to the C ABI.  No arithmetic.  The calls are short (a decoded token's kernel runs for 3 us), and checking a dozen tensors in
// Python took 8 to 16 us of a call; here it takes one.
//
// Every function returns the library's status; arguments that are no valid call at all raise ValueError or TypeError.  The library is the
// one the package has loaded: bind(path) looks its functions up in it.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>

#include <stdexcept>
#include <string>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "dpclip.h"

namespace {

struct BadValue : std::runtime_error { using std::runtime_error::runtime_error; };
struct BadType : std::runtime_error { using std::runtime_error::runtime_error; };

// ------------------------------------------------------------------------------------------------ the library's functions
#define FUNCTIONS(X) X(dpclip_stored_clipped_grad) X(dpclip_relbias_forward) X(dpclip_relbias_sqnorms) X(dpclip_qknorm_forward) \
    X(dpclip_qknorm_backward) X(dpclip_gated_forward) X(dpclip_gated_backward)
struct Library {
#define DECLARE(name) decltype(&::name) name = nullptr;
    FUNCTIONS(DECLARE)
#undef DECLARE
} lib;

PyObject* bind(PyObject*, PyObject* path) {
    const char* p = PyUnicode_AsUTF8(path);
    if (!p) return nullptr;
    void* h = dlopen(p, RTLD_NOW | RTLD_LOCAL);
    if (!h) { PyErr_Format(PyExc_ImportError, "%s", dlerror()); return nullptr; }
#define LOOKUP(name) \
    lib.name = reinterpret_cast<decltype(lib.name)>(dlsym(h, #name)); \
    if (!lib.name) { PyErr_SetString(PyExc_ImportError, "the library lacks " #name); return nullptr; }
    FUNCTIONS(LOOKUP)
#undef LOOKUP
    Py_RETURN_NONE;
}

// ------------------------------------------------------------------------------------------------ arguments
struct Args {
    PyObject* const* v;
    Py_ssize_t n;
    Args(PyObject* const* v_, Py_ssize_t n_, Py_ssize_t want) : v(v_), n(n_) {
        if (n != want) throw BadType("wrong number of arguments");
    }
    const at::Tensor* maybe(int i) const {
        if (v[i] == Py_None) return nullptr;
        if (!THPVariable_Check(v[i])) throw BadType("expected a tensor");
        return &THPVariable_Unpack(v[i]);
    }
    const at::Tensor& tensor(int i) const {
        const at::Tensor* t = maybe(i);
        if (!t) throw BadType("expected a tensor, got None");
        return *t;
    }
    long integer(int i) const {
        const long x = PyLong_AsLong(v[i]);
        if (x == -1 && PyErr_Occurred()) { PyErr_Clear(); throw BadType("expected an integer"); }
        return x;
    }
    int int32(int i) const {
        const long x = integer(i);
        if (x < INT_MIN || x > INT_MAX) throw BadValue("an integer is out of range");
        return (int)x;
    }
    unsigned long long u64(int i) const {
        const unsigned long long x = PyLong_AsUnsignedLongLongMask(v[i]);
        if (PyErr_Occurred()) { PyErr_Clear(); throw BadType("expected an integer"); }
        return x;
    }
    double number(int i) const {
        const double x = PyFloat_AsDouble(v[i]);
        if (x == -1.0 && PyErr_Occurred()) { PyErr_Clear(); throw BadType("expected a number"); }
        return x;
    }
    bool truth(int i) const {
        const int x = PyObject_IsTrue(v[i]);
        if (x < 0) { PyErr_Clear(); throw BadType("expected a truth value"); }
        return x == 1;
    }
};

// Tensors lie on the current device, where the calls run.
struct Device {
    int current = -1;
    void check(const at::Tensor* t) {
        if (!t) return;
        if (!t->is_cuda()) throw BadValue("expected a CUDA tensor, got one of the host");
        if (current < 0) current = c10::cuda::current_device();
        if (t->get_device() != current)
            throw BadValue("expected a tensor on the current device " + std::to_string(current) + ", got one on " + std::to_string(t->get_device()));
    }
};
// None: the current stream; a torch stream (its address has been taken by the caller) or an address
void* stream_of(PyObject* o) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    void* p = PyLong_AsVoidPtr(o);
    if (PyErr_Occurred()) { PyErr_Clear(); throw BadType("expected a stream"); }
    return p;
}
dpclip_dtype dtype_of(const at::Tensor& t) {
    if (t.scalar_type() == at::kFloat) return DPCLIP_F32;
    if (t.scalar_type() == at::kBFloat16) return DPCLIP_BF16;
    throw BadType("unsupported dtype: fp32 or bf16 is wanted");
}
template <typename T> T* dense(const at::Tensor* t, at::ScalarType type, at::IntArrayRef sizes, const char* what) {
    if (!t) return nullptr;
    if (t->scalar_type() != type || t->sizes() != sizes || !t->is_contiguous()) throw BadValue(std::string(what) + ": expected a contiguous tensor of another shape or type");
    return static_cast<T*>(t->data_ptr());
}
float* dense_f32(const at::Tensor* t, at::IntArrayRef sizes, const char* what) { return dense<float>(t, at::kFloat, sizes, what); }
// an output's elements have places of their own
void writable(const at::Tensor& t, const char* what) {
    for (int64_t i = 0; i < t.dim(); ++i)
        if (t.stride(i) == 0 && t.size(i) > 1) throw BadValue(std::string(what) + ": an output may not be a broadcast tensor");
}
// a workspace owns every byte that it counts: an expanded tensor would not
const at::Tensor& workspace_of(const at::Tensor& t) {
    if (!t.is_contiguous()) throw BadValue("workspace: expected a contiguous tensor");
    return t;
}
int size32(int64_t n) {
    if (n > INT_MAX) throw BadValue("a dimension is out of range");
    return (int)n;
}
bool inner_one(const at::Tensor& t) { return t.size(-1) <= 1 || t.stride(-1) == 1; }

template <typename F> PyObject* guarded(F f) {
    try {
        return PyLong_FromLong(f());
    } catch (const BadValue& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const BadType& e) {
        PyErr_SetString(PyExc_TypeError, e.what());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown failure");
    }
    return nullptr;
}

// The library's call, without the interpreter's lock: a launch may have to wait for room in the device's queue, and work in front of it may need
// another thread of Python (a host function) to go on.  The arguments are worked out before.
struct Unlocked {
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename F, typename... A> int call(F function, A... arguments) {
    const Unlocked unlocked;
    return function(arguments...);
}

// ------------------------------------------------------------------------------------------------ the calls
// grads, clip, g, sigma, C, seed, stream_id, stream
PyObject* stored_clipped_grad(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded([&] {
        const Args a(v, n, 8);
        const at::Tensor& grads = a.tensor(0), &g = a.tensor(2);
        const at::Tensor* clip = a.maybe(1);
        Device d;
        d.check(&grads); d.check(clip); d.check(&g);
        if (grads.dim() < 1) throw BadValue("grads must have a dimension of examples");
        const int64_t B = grads.size(0), width = g.numel();
        if (grads.numel() != B * width) throw BadValue("g must have the size of one example's gradients");
        return call(lib.dpclip_stored_clipped_grad, dense_f32(&grads, grads.sizes(), "grads"), width, size32(B), size32(width), dense_f32(clip, {B}, "clip"),
                                              dense_f32(&g, g.sizes(), "g"), (float)a.number(3), (float)a.number(4), a.u64(5), a.u64(6), stream_of(v[7]));
    });
}

// table, bias, max_distance, bidirectional, causal, q_offset, stream
PyObject* relbias_forward(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded([&] {
        const Args a(v, n, 7);
        const at::Tensor& table = a.tensor(0), &bias = a.tensor(1);
        Device d;
        d.check(&table); d.check(&bias);
        if (table.dim() != 2 || table.scalar_type() != at::kFloat || !inner_one(table)) throw BadValue("table must be (n_buckets, H) fp32 with contiguous rows");
        const int64_t buckets = table.size(0), H = table.size(1);
        if (bias.dim() != 3 || bias.size(0) != H || !inner_one(bias)) throw BadValue("bias must be (H, Tq, Tk) with contiguous keys");
        writable(bias, "bias");
        const int64_t Tq = bias.size(1), Tk = bias.size(2);
        const dpclip_relbias c = {size32(buckets), a.int32(2), a.truth(3), a.truth(4)};
        return call(lib.dpclip_relbias_forward, static_cast<const float*>(table.data_ptr()), buckets > 1 ? table.stride(0) : H, &c, size32(H), size32(Tq), size32(Tk),
                                          a.integer(5), dtype_of(bias), bias.data_ptr(), Tq > 1 ? bias.stride(1) : Tk, bias.stride(0), stream_of(v[6]));
    });
}

// dS, grads, sq_layer, workspace, max_distance, bidirectional, causal, q_offset, q_lens, k_lens, accumulate, stream
PyObject* relbias_sqnorms(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded([&] {
        const Args a(v, n, 12);
        const at::Tensor& dS = a.tensor(0), &grads = a.tensor(1), &sq = a.tensor(2), &ws = workspace_of(a.tensor(3));
        const at::Tensor* ql = a.maybe(8), *kl = a.maybe(9);
        Device d;
        d.check(&dS); d.check(&grads); d.check(&sq); d.check(&ws); d.check(ql); d.check(kl);
        if (dS.dim() != 4 || !inner_one(dS)) throw BadValue("dS must be (B, H, Tq, Tk) with contiguous keys");
        if (grads.dim() != 3) throw BadValue("grads must be (B, n_buckets, H)");
        const int64_t B = dS.size(0), H = dS.size(1), Tq = dS.size(2), Tk = dS.size(3), buckets = grads.size(1);
        const dpclip_relbias c = {size32(buckets), a.int32(4), a.truth(5), a.truth(6)};
        return call(lib.dpclip_relbias_sqnorms, dS.data_ptr(), Tq > 1 ? dS.stride(2) : Tk, dS.stride(1), dS.stride(0), size32(B), size32(H), size32(Tq), size32(Tk),
                                          a.integer(7), dense<int>(ql, at::kInt, {B}, "q_lens"), dense<int>(kl, at::kInt, {B}, "k_lens"), &c, dtype_of(dS),
                                          a.truth(10), dense_f32(&grads, {B, buckets, H}, "grads"), dense_f32(&sq, {B}, "sq_layer"), ws.data_ptr(),
                                          ws.nbytes(), stream_of(v[11]));
    });
}

dpclip_heads heads_of(Device& d, const at::Tensor& x, const at::Tensor* gain, const at::Tensor& out, const at::Tensor* dy, const at::Tensor& first) {
    d.check(&x); d.check(gain); d.check(&out); d.check(dy);
    const int64_t D = first.size(3);
    auto fine = [&](const at::Tensor& t) {
        return t.dim() == 4 && t.scalar_type() == first.scalar_type() && t.size(0) == first.size(0) && t.size(1) == first.size(1) && t.size(2) == x.size(2) &&
               t.size(3) == D && inner_one(t);
    };
    if (!fine(x) || !fine(out) || (dy && !fine(*dy))) throw BadValue("expected tensors (B, T, H, D) of one type with contiguous heads");
    writable(out, "out");
    dpclip_heads h;
    h.x = x.data_ptr(); h.x_example = x.stride(0); h.x_token = x.stride(1); h.x_head = x.stride(2);
    h.dy = nullptr; h.dy_example = h.dy_token = h.dy_head = 0;
    if (dy) { h.dy = dy->data_ptr(); h.dy_example = dy->stride(0); h.dy_token = dy->stride(1); h.dy_head = dy->stride(2); }
    h.out = out.data_ptr(); h.out_example = out.stride(0); h.out_token = out.stride(1); h.out_head = out.stride(2);
    h.H = size32(x.size(2));
    h.gain = dense_f32(gain, {D}, "gain");
    return h;
}
struct Angles { const float* table; int rot; long n_pos; const int* pos; };
// rotation, rot_dim (None or a number), positions
Angles angles_of(Device& d, const at::Tensor* rotation, PyObject* rot_dim, const at::Tensor* positions, const at::Tensor& q) {
    d.check(rotation); d.check(positions);
    Angles r = {nullptr, 0, 1L << 62, dense<int>(positions, at::kInt, {q.size(0), q.size(1)}, "positions")};
    if (rotation) {
        if (rotation->dim() != 3 || rotation->size(1) != 2) throw BadValue("rotation must be (n_pos, 2, rot_dim / 2)");
        r.table = dense_f32(rotation, rotation->sizes(), "rotation");
        r.rot = size32(2 * rotation->size(2));
        r.n_pos = rotation->size(0);
    }
    if (rot_dim != Py_None) {
        const long want = PyLong_AsLong(rot_dim);
        if (PyErr_Occurred()) { PyErr_Clear(); throw BadType("rot_dim: expected an integer"); }
        if (want != r.rot) throw BadValue("rot_dim is not that of the table of angles");
    }
    return r;
}

// q, k, gain_q, gain_k, rotation, q_out, k_out, rot_dim, interleaved, positions, pos0, eps, stream
PyObject* qknorm_forward(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded([&] {
        const Args a(v, n, 13);
        const at::Tensor& q = a.tensor(0);
        const at::Tensor* k = a.maybe(1);
        Device d;
        if (q.dim() != 4) throw BadValue("q must be (B, T, H, D)");
        dpclip_heads parts[2];
        parts[0] = heads_of(d, q, a.maybe(2), a.tensor(5), nullptr, q);
        if (k) parts[1] = heads_of(d, *k, a.maybe(3), a.tensor(6), nullptr, q);
        const Angles r = angles_of(d, a.maybe(4), v[7], a.maybe(9), q);
        return call(lib.dpclip_qknorm_forward, parts, k ? 2 : 1, size32(q.size(0)), size32(q.size(1)), size32(q.size(3)), r.rot, a.truth(8), r.table, r.n_pos, r.pos,
                                         a.integer(10), (float)a.number(11), dtype_of(q), stream_of(v[12]));
    });
}

// dq_out, dk_out, q, k, gain_q, gain_k, rotation, dq, dk, grads_q, grads_k, sq_q, sq_k, workspace, rot_dim, interleaved, positions, pos0, eps, stream
PyObject* qknorm_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded([&] {
        const Args a(v, n, 20);
        const at::Tensor& q = a.tensor(2), &ws = workspace_of(a.tensor(13));
        const at::Tensor* k = a.maybe(3);
        Device d;
        if (q.dim() != 4) throw BadValue("q must be (B, T, H, D)");
        const int64_t B = q.size(0), D = q.size(3);
        dpclip_heads parts[2];
        parts[0] = heads_of(d, q, a.maybe(4), a.tensor(7), &a.tensor(0), q);
        if (k) parts[1] = heads_of(d, *k, a.maybe(5), a.tensor(8), &a.tensor(1), q);
        const Angles r = angles_of(d, a.maybe(6), v[14], a.maybe(16), q);
        float* grads[2], *sq[2];
        for (int i = 0; i < 2; ++i) {
            const at::Tensor* g = a.maybe(9 + i), *s = a.maybe(11 + i);
            d.check(g); d.check(s);
            grads[i] = dense_f32(g, {B, D}, "grads");
            sq[i] = dense_f32(s, {B}, "sq");
        }
        d.check(&ws);
        return call(lib.dpclip_qknorm_backward, parts, k ? 2 : 1, size32(B), size32(q.size(1)), size32(D), r.rot, a.truth(15), r.table, r.n_pos, r.pos, a.integer(17),
                                          (float)a.number(18), dtype_of(q), grads, sq, ws.data_ptr(), ws.nbytes(), stream_of(v[19]));
    });
}

// A (..., columns) tensor as a matrix of equally spaced rows.
struct Matrix { void* p; long ld; int64_t rows, cols; };
Matrix matrix_of(Device& d, const at::Tensor& t, at::ScalarType type, int64_t rows, int64_t cols, const char* what) {
    d.check(&t);
    Matrix m = {t.data_ptr(), 0, 1, t.dim() ? t.size(-1) : 0};
    bool fine = t.dim() >= 1 && t.scalar_type() == type && inner_one(t);
    // leading dimensions that count fall into one stride
    m.ld = m.cols;
    bool first = true;
    long next = 0;
    for (int64_t i = t.dim() - 2; i >= 0 && fine; --i) {
        if (t.size(i) != 1) {
            if (first) { m.ld = t.stride(i); first = false; }
            else fine = t.stride(i) == next;
            next = t.stride(i) * t.size(i);
        }
        m.rows *= t.size(i);
    }
    fine = fine && (rows < 0 || m.rows == rows) && (cols < 0 || m.cols == cols);
    if (!fine) throw BadValue(std::string(what) + ": expected rows with contiguous columns, equally spaced, of the other tensors' type and sizes");
    return m;
}

// X, W, bias, H, Z, act, workspace, stream
PyObject* gated_forward(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded([&] {
        const Args a(v, n, 8);
        const at::Tensor& X = a.tensor(0), &Wt = a.tensor(1), &Ht = a.tensor(3), &ws = workspace_of(a.tensor(6));
        const at::Tensor* bias = a.maybe(2), *Zt = a.maybe(4);
        Device d;
        const auto type = X.scalar_type();
        const Matrix x = matrix_of(d, X, type, -1, -1, "X"), w = matrix_of(d, Wt, type, -1, x.cols, "W");
        if (w.rows % 2) throw BadValue("W must have an even number of rows: gate rows, then up rows");
        const int64_t F = w.rows / 2;
        const Matrix h = matrix_of(d, Ht, type, x.rows, F, "H");
        writable(Ht, "H");
        Matrix z = {nullptr, 0, 0, 0};
        if (Zt) { z = matrix_of(d, *Zt, type, x.rows, 2 * F, "Z"); writable(*Zt, "Z"); }
        d.check(bias); d.check(&ws);
        return call(lib.dpclip_gated_forward, x.p, x.ld, w.p, w.ld, dense_f32(bias, {2 * F}, "bias"), size32(x.rows), size32(x.cols), size32(F), dtype_of(X),
                                        (dpclip_activation)a.int32(5), h.p, h.ld, z.p, z.ld, ws.data_ptr(), ws.nbytes(), stream_of(v[7]));
    });
}

// dH, Z, W, dZ, dX, act, workspace, stream
PyObject* gated_backward(PyObject*, PyObject* const* v, Py_ssize_t n) {
    return guarded([&] {
        const Args a(v, n, 8);
        const at::Tensor& dHt = a.tensor(0), &Zt = a.tensor(1), &dZt = a.tensor(3);
        const at::Tensor* Wt = a.maybe(2), *dXt = a.maybe(4), *ws = a.maybe(6);
        Device d;
        const auto type = Zt.scalar_type();
        const Matrix z = matrix_of(d, Zt, type, -1, -1, "Z");
        if (z.cols % 2) throw BadValue("Z must have an even number of columns: gate, then up");
        const int64_t F = z.cols / 2;
        const Matrix dh = matrix_of(d, dHt, type, z.rows, F, "dH"), dz = matrix_of(d, dZt, type, z.rows, z.cols, "dZ");
        writable(dZt, "dZ");
        Matrix w = {nullptr, 0, 0, 1}, dx = {nullptr, 0, 0, 0};
        if (dXt) {
            if (!Wt || !ws) throw BadValue("dX needs W and a workspace");
            w = matrix_of(d, *Wt, type, z.cols, -1, "W");
            dx = matrix_of(d, *dXt, type, z.rows, w.cols, "dX");
            writable(*dXt, "dX");
        }
        d.check(ws);
        if (ws) workspace_of(*ws);
        return call(lib.dpclip_gated_backward, dh.p, dh.ld, z.p, z.ld, w.p, w.ld, size32(z.rows), size32(w.cols), size32(F), dtype_of(Zt), (dpclip_activation)a.int32(5),
                                         dz.p, dz.ld, dx.p, dx.ld, ws ? ws->data_ptr() : nullptr, ws ? ws->nbytes() : 0, stream_of(v[7]));
    });
}

PyMethodDef methods[] = {
    {"bind", bind, METH_O, "bind(path of the shared library)"},
#define METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, "positional arguments only; the library's status"}
    METHOD(stored_clipped_grad), METHOD(relbias_forward), METHOD(relbias_sqnorms), METHOD(qknorm_forward), METHOD(qknorm_backward),
    METHOD(gated_forward), METHOD(gated_backward),
#undef METHOD
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of libdpclip's transformer-block entry points", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
