/*
 * The client operators' marshalling for torch tensors as a CPython module
 * (_client), against torch's C++ interface: client.py's calls with the checks,
 * the new tensors and the argument structs made here.
 *
 * Why: a small call is bound by the host.  On a GB300's Arm cores each call from
 * Python into torch costs 1.4 us by itself and up to 3.7 us next to a kernel
 * launch, and a join with its gradients makes eleven new tensors: 50 us from
 * Python, about a third of it here (client.py says what it measured).
 *
 * client.py holds the same code in Python, which serves where torch's headers were
 * not installed when the library was built; tests compare the two.  Built for
 * one torch version, which `torch_version` names.
 */
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <optional>
#include <stdexcept>

#include "fasgd.h"

namespace {

using at::Tensor;

/* Errors: a ValueError, or one of the library's statuses (client.py raises it). */
struct Status {
    int64_t code;
};
[[noreturn]] void wrong(const char* what) { throw std::invalid_argument(what); }

const Tensor* tensor(PyObject* o) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) wrong("a tensor is expected");
    return &THPVariable_Unpack(o);
}
int dtype_of(const Tensor& t) {
    switch (t.scalar_type()) {
        case at::kFloat: return FASGD_F32;
        case at::kBFloat16: return FASGD_BF16;
        case at::kHalf: return FASGD_F16;
        default: wrong("activations are fp32, bf16 or fp16");
    }
}
/* A tensor without elements may have no address; one that is never followed. */
void* address(const Tensor& t) {
    void* p = t.data_ptr();
    return p != nullptr ? p : reinterpret_cast<void*>(16);
}
void on_gpu(const Tensor& t) {
    if (!t.is_cuda()) wrong("CUDA tensors are expected");
}

/* A matrix [..., cols] whose rows are evenly spaced. */
struct Matrix {
    int64_t rows, cols, ld;
    void* p;
    explicit Matrix(const Tensor& t) {
        on_gpu(t);
        const auto size = t.sizes(), step = t.strides();
        const int64_t n = t.dim();
        if (n < 1) wrong("a matrix [..., cols] is expected");
        cols = ld = size[n - 1];
        if (step[n - 1] != 1 && cols > 1) wrong("the values of a row must be contiguous");
        rows = 1;
        int64_t next = 0;
        for (int64_t i = n - 2; i >= 0; --i) {
            if (size[i] == 1) continue;
            if (rows == 1)
                ld = step[i];
            else if (rows != 0 && size[i] != 0 && step[i] != next)
                wrong("the rows must be evenly spaced");
            next = step[i] * size[i];
            rows *= size[i];
        }
        p = address(t);
    }
};
Matrix like(const Tensor& t, const Tensor& first) {
    if (t.sizes() != first.sizes() || t.scalar_type() != first.scalar_type())
        wrong("matrices of one shape and type are expected");
    return Matrix(t);
}
/* New tensors on like's device, without gaps. */
Tensor fresh(at::IntArrayRef size, at::ScalarType type, const Tensor& like) {
    return at::detail::empty_cuda(size, type, like.device(), std::nullopt);
}
Tensor fresh(const Tensor& like) { return fresh(like.sizes(), like.scalar_type(), like); }
Tensor fresh(int64_t n, at::ScalarType type, const Tensor& like) { return fresh(at::IntArrayRef(&n, 1), type, like); }
/* `size` values of `flat` from `offset` on, as a tensor that shares its memory. */
Tensor part(const Tensor& flat, int64_t offset, at::IntArrayRef size) {
    Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(flat.storage()), flat.key_set(), flat.dtype());
    t.unsafeGetTensorImpl()->set_storage_offset(offset);
    t.unsafeGetTensorImpl()->set_sizes_contiguous(size);
    return t;
}

float* vector(const Tensor* t, int64_t cols) {
    if (t == nullptr) return nullptr;
    on_gpu(*t);
    if (t->scalar_type() != at::kFloat || t->numel() != cols || !t->is_contiguous())
        wrong("parameters are contiguous fp32 vectors of cols values");
    return static_cast<float*>(address(*t));
}

/* torch's current stream, which is to be on t's device. */
void* stream(const Tensor& t) {
    const auto device = c10::cuda::current_device();
    if (t.get_device() != device) wrong("CUDA tensors on the current device are expected");
    return c10::cuda::getCurrentCUDAStream(device).stream();
}

template <class F>
int64_t unlocked(F call) {
    int64_t rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    if (rc < 0) throw Status{rc};
    return rc;
}

/* Draws(rate, seed, client, n), or None. */
template <class Args>
void draws(PyObject* o, Args& a) {
    if (o == Py_None) return;
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) wrong("draws are (rate, seed, client, n)");
    a.rate = PyFloat_AsDouble(PyTuple_GET_ITEM(o, 0));
    a.seed = PyLong_AsUnsignedLongLongMask(PyTuple_GET_ITEM(o, 1));
    a.client = (int32_t)PyLong_AsUnsignedLongLongMask(PyTuple_GET_ITEM(o, 2));
    a.n = PyLong_AsUnsignedLongLongMask(PyTuple_GET_ITEM(o, 3));
    if (PyErr_Occurred()) throw Status{0};
}
float real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Status{0};
    return (float)v;
}
int64_t whole(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Status{0};
    return v;
}

PyObject* object(const Tensor& t) { return THPVariable_Wrap(t); }
/* The tensor of a call: the caller's own object where there was one. */
PyObject* object(PyObject* given, const std::optional<Tensor>& made) {
    if (made) return object(*made);
    Py_INCREF(given);
    return given;
}
PyObject* tuple(std::initializer_list<PyObject*> items) {
    PyObject* out = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    bool ok = out != nullptr;
    for (PyObject* item : items) {
        ok = ok && item != nullptr;
        if (out != nullptr)
            PyTuple_SET_ITEM(out, i++, item);
        else
            Py_XDECREF(item);
    }
    if (!ok) Py_CLEAR(out);
    return out;
}

/* Runs an entry: no C++ exception leaves it.  A status is returned as an int. */
template <class F>
PyObject* entry(Py_ssize_t got, Py_ssize_t wanted, F body) {
    try {
        if (got != wanted) {
            PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
            return nullptr;
        }
        return body();
    } catch (const Status& s) {
        return s.code != 0 ? PyLong_FromLongLong(s.code) : nullptr;
    } catch (const std::invalid_argument& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

/* dropout(x, draws, residual, out) -> out */
PyObject* py_dropout(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return entry(nargs, 4, [&]() -> PyObject* {
        const Tensor *x = tensor(args[0]), *residual = tensor(args[2]), *out = tensor(args[3]);
        if (x == nullptr) wrong("a tensor is expected");
        fasgd_dropout_args a;
        std::memset(&a, 0, sizeof a);
        const Matrix m(*x);
        a.rows = m.rows;
        a.cols = m.cols;
        a.x = m.p;
        a.ld_x = m.ld;
        a.dtype = dtype_of(*x);
        draws(args[1], a);
        if (residual != nullptr) {
            const Matrix r = like(*residual, *x);
            a.residual = r.p;
            a.ld_residual = r.ld;
        }
        std::optional<Tensor> made;
        if (out == nullptr) made = fresh(*x);
        const Matrix o = like(made ? *made : *out, *x);
        a.out = o.p;
        a.ld_out = o.ld;
        void* s = stream(*x);
        unlocked([&] { return (int64_t)fasgd_dropout(&a, s); });
        return object(args[3], made);
    });
}

/* join(x, y, post, post_bias, gate, pre, pre_bias, norm, eps, carry, branch, draws, h, z)
 * -> (h, z, stats, the argument struct as bytes) */
PyObject* py_join(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return entry(nargs, 14, [&]() -> PyObject* {
        const Tensor *x = tensor(args[0]), *y = tensor(args[1]), *gate = tensor(args[4]), *pre = tensor(args[5]);
        const Tensor *h = tensor(args[12]), *z = tensor(args[13]);
        if (x == nullptr) wrong("a tensor is expected");
        if ((h != nullptr && y == nullptr) || (z != nullptr && pre == nullptr)) wrong("h goes with y, z with pre");
        fasgd_join_args a;
        std::memset(&a, 0, sizeof a);
        const Matrix m(*x);
        a.rows = m.rows;
        a.cols = m.cols;
        a.x = m.p;
        a.ld_x = m.ld;
        a.dtype = dtype_of(*x);
        a.groups = 1;
        std::optional<Tensor> made_h, made_z;
        if (y != nullptr) {
            const Matrix k = like(*y, *x);
            a.y = k.p;
            a.ld_y = k.ld;
            if (h == nullptr) made_h = fresh(*x);
            const Matrix o = like(made_h ? *made_h : *h, *x);
            a.h = o.p;
            a.ld_h = o.ld;
        }
        if (pre != nullptr) {
            if (z == nullptr) made_z = fresh(*x);
            const Matrix o = like(made_z ? *made_z : *z, *x);
            a.z = o.p;
            a.ld_z = o.ld;
        }
        a.post = vector(tensor(args[2]), m.cols);
        a.post_bias = vector(tensor(args[3]), m.cols);
        a.pre = vector(pre, m.cols);
        a.pre_bias = vector(tensor(args[6]), m.cols);
        if (gate != nullptr) {
            on_gpu(*gate);
            if (gate->dim() < 1 || gate->dim() > 2 || gate->size(-1) != m.cols || !gate->is_contiguous())
                wrong("a gate is contiguous, [cols] or [groups, cols]");
            if (gate->dim() == 2) a.groups = gate->size(0);
            a.gate = address(*gate);
            a.gate_dtype = dtype_of(*gate);
        }
        a.norm = (int32_t)whole(args[7]);
        a.eps = real(args[8]);
        a.carry = real(args[9]);
        a.branch = real(args[10]);
        draws(args[11], a);
        const Tensor stats = fresh(4 * m.rows, at::kFloat, *x);
        a.stats = static_cast<float*>(address(stats));
        void* s = stream(*x);
        unlocked([&] { return (int64_t)fasgd_join(&a, s); });
        return tuple({object(args[12], made_h), object(args[13], made_z), object(stats),
                      PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&a), sizeof a)});
    });
}

/* join_grad(join's struct, x, y, dh, dz, (post, post_bias, gate, pre, pre_bias),
 * (x, y, post, post_bias, gate, pre, pre_bias)): the parameters, and where their
 * gradients go (None: a new tensor) -> those seven */
PyObject* py_join_grad(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return entry(nargs, 7, [&]() -> PyObject* {
        fasgd_join_args a;
        if (!PyBytes_Check(args[0]) || PyBytes_GET_SIZE(args[0]) != (Py_ssize_t)sizeof a ||
            !PyTuple_Check(args[5]) || PyTuple_GET_SIZE(args[5]) != 5 || !PyTuple_Check(args[6]) ||
            PyTuple_GET_SIZE(args[6]) != 7)
            wrong("join_grad: not a join's record");
        std::memcpy(&a, PyBytes_AS_STRING(args[0]), sizeof a);
        const Tensor *x = tensor(args[1]), *y = tensor(args[2]), *dh = tensor(args[3]), *dz = tensor(args[4]);
        if (x == nullptr) wrong("a tensor is expected");
        if (dh != nullptr) {
            const Matrix m = like(*dh, *x);
            a.dh = m.p;
            a.ld_dh = m.ld;
        }
        if (dz != nullptr) {
            const Matrix m = like(*dz, *x);
            a.dz = m.p;
            a.ld_dz = m.ld;
        }
        PyObject* const* into = &PyTuple_GET_ITEM(args[6], 0);
        std::optional<Tensor> made[7];
        PyObject* out[7];
        for (int i = 0; i < 7; ++i) out[i] = into[i];
        const auto matrix = [&](int i, void*& p, int64_t& ld) {
            const Tensor* t = tensor(into[i]);
            if (t == nullptr) made[i] = fresh(*x);
            const Matrix m = like(made[i] ? *made[i] : *t, *x);
            p = m.p;
            ld = m.ld;
        };
        matrix(0, a.dx, a.ld_dx);
        if (y != nullptr)
            matrix(1, a.dy, a.ld_dy);
        else
            out[1] = Py_None;
        // The parameters' new fp32 gradients share one allocation (one costs 1.4 us).
        int64_t values = 0;
        for (int i = 0; i < 5; ++i) {
            const Tensor* of = tensor(PyTuple_GET_ITEM(args[5], i));
            if (of != nullptr && into[2 + i] == Py_None && of->scalar_type() == at::kFloat) values += (of->numel() + 3) / 4 * 4;
        }
        Tensor flat;
        if (values > 0) flat = fresh(values, at::kFloat, *x);
        values = 0;
        void* at[5];
        for (int i = 0; i < 5; ++i) {
            const Tensor *of = tensor(PyTuple_GET_ITEM(args[5], i)), *t = tensor(into[2 + i]);
            at[i] = nullptr;
            if (of == nullptr) {
                out[2 + i] = Py_None;
            } else if (t == nullptr && of->scalar_type() == at::kFloat) {
                made[2 + i] = part(flat, values, of->sizes());
                values += (of->numel() + 3) / 4 * 4;
                at[i] = address(*made[2 + i]);
            } else if (t == nullptr) {
                made[2 + i] = fresh(*of);
                at[i] = address(*made[2 + i]);
            } else if (i == 2) {
                if (t->sizes() != of->sizes() || t->scalar_type() != of->scalar_type() || !t->is_contiguous() || !t->is_cuda())
                    wrong("the gate's gradient must be as the gate");
                at[i] = address(*t);
            } else {
                at[i] = vector(t, a.cols);
            }
        }
        a.dpost = static_cast<float*>(at[0]);
        a.dpost_bias = static_cast<float*>(at[1]);
        a.dgate = at[2];
        a.dpre = static_cast<float*>(at[3]);
        a.dpre_bias = static_cast<float*>(at[4]);
        void* s = stream(*x);
        const int64_t size = fasgd_join_workspace(&a);
        if (size < 0) throw Status{size};
        const Tensor space = fresh(size, at::kByte, *x);
        a.workspace = space.data_ptr();
        a.workspace_bytes = size;
        unlocked([&] { return (int64_t)fasgd_join_grad(&a, s); });
        return tuple({object(out[0], made[0]), object(out[1], made[1]), object(out[2], made[2]), object(out[3], made[3]),
                      object(out[4], made[4]), object(out[5], made[5]), object(out[6], made[6])});
    });
}

/* balance(logits, chosen, balance, z, groups, valid, upstream, grad)
 * -> (loss, counts, dlogits or None) */
PyObject* py_balance(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return entry(nargs, 8, [&]() -> PyObject* {
        const Tensor *logits = tensor(args[0]), *chosen = tensor(args[1]), *valid = tensor(args[5]), *up = tensor(args[6]);
        if (logits == nullptr || chosen == nullptr) wrong("a tensor is expected");
        fasgd_balance_args a;
        std::memset(&a, 0, sizeof a);
        const Matrix m(*logits);
        a.rows = m.rows;
        a.cols = m.cols;
        a.logits = m.p;
        a.ld_logits = m.ld;
        a.dtype = dtype_of(*logits);
        a.balance_scale = real(args[2]);
        a.z_scale = real(args[3]);
        a.groups = whole(args[4]);
        on_gpu(*chosen);
        a.top = chosen->dim() > 0 ? chosen->size(-1) : 0;
        if (chosen->scalar_type() != at::kInt || !chosen->is_contiguous() || chosen->numel() != m.rows * a.top)
            wrong("chosen must be contiguous int32 [..., top] on the GPU, a row for each of logits");
        a.chosen = static_cast<int32_t*>(address(*chosen));
        if (valid != nullptr) {
            on_gpu(*valid);
            if ((valid->scalar_type() != at::kByte && valid->scalar_type() != at::kBool) || !valid->is_contiguous() ||
                valid->numel() != m.rows)
                wrong("valid must be contiguous bool or uint8 on the GPU, one for each row");
            a.valid = static_cast<uint8_t*>(address(*valid));
        }
        if (up != nullptr) {
            on_gpu(*up);
            if (up->scalar_type() != at::kFloat || up->numel() != 1) wrong("upstream must be one fp32 value on the GPU");
            a.upstream = static_cast<float*>(address(*up));
        }
        const int64_t size = fasgd_balance_workspace(&a);
        if (size < 0) throw Status{size};
        std::optional<Tensor> dlogits;
        if (args[7] == Py_True) {
            dlogits = fresh(*logits);
            a.dlogits = address(*dlogits);
            a.ld_dlogits = m.cols;
        }
        const int64_t shape[2] = {a.groups, m.cols};
        const Tensor counts = fresh(shape, at::kInt, *logits);
        const Tensor loss = fresh(3, at::kFloat, *logits), space = fresh(size, at::kByte, *logits);
        a.counts = static_cast<int32_t*>(address(counts));
        a.loss = static_cast<float*>(address(loss));
        a.workspace = space.data_ptr();
        a.workspace_bytes = size;
        void* s = stream(*logits);
        unlocked([&] { return (int64_t)fasgd_balance(&a, s); });
        return tuple({object(loss), object(counts), object(Py_None, dlogits)});
    });
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(dropout), METHOD(join), METHOD(join_grad), METHOD(balance), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_client", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__client(void) {
    PyObject* m = PyModule_Create(&module);
    if (m != nullptr && PyModule_AddStringConstant(m, "torch_version", BUILT_FOR_TORCH) < 0) Py_CLEAR(m);
    return m;
}
