/*
 * The client operators' marshalling for torch tensors as a CPython module
 * (_client), against torch's C++ interface: client.py's calls with the checks,
 * the new tensors and the argument structs made here.
 *
 * Why: a small call is bound by the host.  On a GB300's Arm cores each call from
 * Python into torch costs 1.4 us by itself and up to 3.7 us next to a kernel
 * launch, and a join with its gradients makes eleven new tensors: 51 us from
 * Python for 128 rows of 200.
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
#include <initializer_list>
#include <stdexcept>
#include <type_traits>

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
/* A call's tensors (null: absent), the first of which says where they are to be; no
 * address is taken before. */
void one_device(std::initializer_list<const Tensor*> tensors) {
    const Tensor* first = nullptr;
    for (const Tensor* t : tensors) {
        if (t == nullptr) continue;
        if (first == nullptr) first = t;
        if (!t->is_cuda() || t->device() != first->device()) wrong("CUDA tensors on one device are expected");
    }
}

/* A matrix [..., cols] whose rows are evenly spaced. */
struct Matrix {
    int64_t rows, cols, ld;
    void* p;
    explicit Matrix(const Tensor& t) {
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
/* The new tensors of a call, on one device and without gaps.  Each would cost
 * 1.4 us of the host, so where all of them are small (1 MiB together) they share
 * one allocation, and one that outlives the others keeps no more than that. */
class New {
  public:
    explicit New(const Tensor& like) : device_(like.device()) {}
    /* Announces a tensor, whose address will be in *p after make(). */
    template <class P>
    int add(at::IntArrayRef size, at::ScalarType type, P** p) {
        Item& i = items_[count_];
        i.size.assign(size.begin(), size.end());
        i.type = type;
        i.p = reinterpret_cast<void**>(p);
        i.bytes = (int64_t)c10::elementSize(type);
        for (const int64_t s : size) i.bytes *= s;
        total_ += (i.bytes + 255) / 256 * 256;
        return count_++;
    }
    template <class P>
    int add(int64_t n, at::ScalarType type, P** p) { return add(at::IntArrayRef(&n, 1), type, p); }
    template <class P>
    int add(const Tensor& like, P** p) { return add(like.sizes(), like.scalar_type(), p); }
    void make() {
        const bool shared = count_ > 1 && total_ <= kShared;
        Tensor base;
        if (shared && total_ > 0) base = at::detail::empty_cuda({total_}, at::kByte, device_, std::nullopt);
        int64_t at = 0;
        for (int k = 0; k < count_; ++k) {
            Item& i = items_[k];
            if (base.defined() && i.bytes > 0) {
                i.tensor = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(base.storage()), base.key_set(),
                                                                    c10::scalarTypeToTypeMeta(i.type));
                i.tensor.unsafeGetTensorImpl()->set_storage_offset(at / (int64_t)c10::elementSize(i.type));
                i.tensor.unsafeGetTensorImpl()->set_sizes_contiguous(i.size);
                at += (i.bytes + 255) / 256 * 256;
            } else {
                i.tensor = at::detail::empty_cuda(i.size, i.type, device_, std::nullopt);
            }
            *i.p = address(i.tensor);
        }
    }
    PyObject* object(int k) const { return THPVariable_Wrap(items_[k].tensor); }

  private:
    static constexpr int64_t kShared = 1 << 20;
    struct Item {
        c10::SmallVector<int64_t, 5> size;
        at::ScalarType type;
        int64_t bytes;
        void** p;
        Tensor tensor;
    };
    c10::Device device_;
    Item items_[10];
    int count_ = 0;
    int64_t total_ = 0;
};

float* vector(const Tensor* t, int64_t cols) {
    if (t == nullptr) return nullptr;
    if (t->scalar_type() != at::kFloat || t->numel() != cols || !t->is_contiguous())
        wrong("parameters are contiguous fp32 vectors of cols values");
    return static_cast<float*>(address(*t));
}

/* A join's inputs into its struct: the matrices, and the shape and types they fix;
 * of: (post, post_bias, gate, pre, pre_bias), null where absent. */
void join_inputs(fasgd_join_args& a, const Tensor& x, const Tensor* y, const Tensor* const (&of)[5]) {
    const Matrix m(x);
    a.rows = m.rows;
    a.cols = m.cols;
    a.x = m.p;
    a.ld_x = m.ld;
    a.dtype = dtype_of(x);
    a.groups = 1;
    if (y != nullptr) {
        const Matrix k = like(*y, x);
        a.y = k.p;
        a.ld_y = k.ld;
    }
    a.post = vector(of[0], m.cols);
    a.post_bias = vector(of[1], m.cols);
    a.pre = vector(of[3], m.cols);
    a.pre_bias = vector(of[4], m.cols);
    if (const Tensor* gate = of[2]) {
        if (gate->dim() < 1 || gate->dim() > 2 || gate->size(-1) != m.cols || !gate->is_contiguous())
            wrong("a gate is contiguous, [cols] or [groups, cols]");
        if (gate->dim() == 2) a.groups = gate->size(0);
        a.gate = address(*gate);
        a.gate_dtype = dtype_of(*gate);
    }
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

/* Draws(rate, seed, client, n), or None.  A client or n beyond its field becomes one
 * that the library refuses, not another's draws. */
template <class Args>
void draws(PyObject* o, Args& a) {
    if (o == Py_None) return;
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) wrong("draws are (rate, seed, client, n)");
    a.rate = PyFloat_AsDouble(PyTuple_GET_ITEM(o, 0));
    a.seed = PyLong_AsUnsignedLongLongMask(PyTuple_GET_ITEM(o, 1));
    if (PyErr_Occurred()) throw Status{0};
    const auto within = [](PyObject* v, int64_t most) {
        int beyond = 0;
        const long long k = PyLong_AsLongLongAndOverflow(v, &beyond);
        if (PyErr_Occurred()) throw Status{0};
        return beyond != 0 || k < 0 || k > most ? (int64_t)-1 : (int64_t)k;
    };
    a.client = (int32_t)within(PyTuple_GET_ITEM(o, 2), INT32_MAX);
    a.n = (uint64_t)within(PyTuple_GET_ITEM(o, 3), INT64_MAX);
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

/* A result: the caller's own object (or None), or (k >= 0) a new tensor.  What was
 * written into a tensor of the caller's shows in its version, which automatic
 * differentiation looks at before it reads a tensor that it has saved. */
PyObject* object(const New& made, int k, PyObject* given) {
    if (k >= 0) return made.object(k);
    if (given != Py_None && !THPVariable_Unpack(given).is_inference())
        THPVariable_Unpack(given).unsafeGetTensorImpl()->bump_version();
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
        one_device({x, residual, out});
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
        New made(*x);
        int k = -1;
        if (out == nullptr) {
            k = made.add(*x, &a.out);
            a.ld_out = m.cols;
        } else {
            const Matrix o = like(*out, *x);
            a.out = o.p;
            a.ld_out = o.ld;
        }
        void* s = stream(*x);
        made.make();
        unlocked([&] { return (int64_t)fasgd_dropout(&a, s); });
        return object(made, k, args[3]);
    });
}

/* join(x, y, post, post_bias, gate, pre, pre_bias, norm, eps, carry, branch, draws, h, z)
 * -> (h, z, stats, the argument struct as bytes) */
PyObject* py_join(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return entry(nargs, 14, [&]() -> PyObject* {
        const Tensor *x = tensor(args[0]), *y = tensor(args[1]), *h = tensor(args[12]), *z = tensor(args[13]);
        const Tensor* const of[5] = {tensor(args[2]), tensor(args[3]), tensor(args[4]), tensor(args[5]), tensor(args[6])};
        if (x == nullptr) wrong("a tensor is expected");
        one_device({x, y, of[0], of[1], of[2], of[3], of[4], h, z});
        if ((h != nullptr && y == nullptr) || (z != nullptr && of[3] == nullptr)) wrong("h goes with y, z with pre");
        fasgd_join_args a;
        std::memset(&a, 0, sizeof a);
        join_inputs(a, *x, y, of);
        New made(*x);
        int at_h = -1, at_z = -1;
        const auto output = [&](const Tensor* t, void*& p, int64_t& ld) {
            if (t == nullptr) {
                ld = a.cols;
                return made.add(*x, &p);
            }
            const Matrix o = like(*t, *x);
            p = o.p;
            ld = o.ld;
            return -1;
        };
        if (y != nullptr) at_h = output(h, a.h, a.ld_h);
        if (of[3] != nullptr) at_z = output(z, a.z, a.ld_z);
        a.norm = (int32_t)whole(args[7]);
        a.eps = real(args[8]);
        a.carry = real(args[9]);
        a.branch = real(args[10]);
        draws(args[11], a);
        const int at_stats = made.add(4 * a.rows, at::kFloat, &a.stats);
        void* s = stream(*x);
        made.make();
        unlocked([&] { return (int64_t)fasgd_join(&a, s); });
        return tuple({object(made, at_h, args[12]), object(made, at_z, args[13]), made.object(at_stats),
                      PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&a), sizeof a)});
    });
}

/* join_grad(join's struct, x, y, dh, dz, (post, post_bias, gate, pre, pre_bias),
 * (x, y, post, post_bias, gate, pre, pre_bias), stats): the parameters, and where their
 * gradients go (None: a new tensor) -> those seven.  Of the struct only the settings
 * are taken: the tensors may have moved since (saved elsewhere, or computed again). */
PyObject* py_join_grad(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return entry(nargs, 8, [&]() -> PyObject* {
        fasgd_join_args a, was;
        if (!PyBytes_Check(args[0]) || PyBytes_GET_SIZE(args[0]) != (Py_ssize_t)sizeof a ||
            !PyTuple_Check(args[5]) || PyTuple_GET_SIZE(args[5]) != 5 || !PyTuple_Check(args[6]) ||
            PyTuple_GET_SIZE(args[6]) != 7)
            wrong("join_grad: not a join's record");
        const Tensor *x = tensor(args[1]), *y = tensor(args[2]), *dh = tensor(args[3]), *dz = tensor(args[4]);
        const Tensor* stats = tensor(args[7]);
        const Tensor* of[5];
        for (int i = 0; i < 5; ++i) of[i] = tensor(PyTuple_GET_ITEM(args[5], i));
        if (x == nullptr || stats == nullptr) wrong("a tensor is expected");
        PyObject* const* into = &PyTuple_GET_ITEM(args[6], 0);
        one_device({x, y, dh, dz, of[0], of[1], of[2], of[3], of[4], stats, tensor(into[0]), tensor(into[1]),
                    tensor(into[2]), tensor(into[3]), tensor(into[4]), tensor(into[5]), tensor(into[6])});
        std::memcpy(&was, PyBytes_AS_STRING(args[0]), sizeof was);
        std::memset(&a, 0, sizeof a);
        a.rate = was.rate;
        a.seed = was.seed;
        a.n = was.n;
        a.client = was.client;
        a.norm = was.norm;
        a.eps = was.eps;
        a.carry = was.carry;
        a.branch = was.branch;
        join_inputs(a, *x, y, of);
        if (a.rows != was.rows || a.cols != was.cols || a.dtype != was.dtype || a.groups != was.groups ||
            (y != nullptr) != (was.y != nullptr) || (of[0] != nullptr) != (was.post != nullptr) ||
            (of[3] != nullptr) != (was.pre != nullptr))
            wrong("join_grad: not the join's tensors");
        a.stats = vector(stats, 4 * a.rows);
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
        New made(*x);
        int at[7];
        PyObject* out[7];
        for (int i = 0; i < 7; ++i) {
            out[i] = into[i];
            at[i] = -1;
        }
        const auto matrix = [&](int i, void*& p, int64_t& ld) {
            const Tensor* t = tensor(into[i]);
            if (t == nullptr) {
                at[i] = made.add(*x, &p);
                ld = a.cols;
            } else {
                const Matrix m = like(*t, *x);
                p = m.p;
                ld = m.ld;
            }
        };
        matrix(0, a.dx, a.ld_dx);
        if (y != nullptr)
            matrix(1, a.dy, a.ld_dy);
        else if (tensor(into[1]) != nullptr)
            wrong("the gradient of a tensor that is not there");
        const auto parameter = [&](int i, auto*& p) {
            const Tensor *p_of = of[i - 2], *t = tensor(into[i]);
            if (p_of == nullptr) {
                if (t != nullptr) wrong("the gradient of a parameter that is not there");
            } else if (t == nullptr) {
                at[i] = made.add(*p_of, &p);
                // What the workspace depends on: that it is there, and aligned.
                p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(256);
            } else if (i == 4) {
                if (t->sizes() != p_of->sizes() || t->scalar_type() != p_of->scalar_type() || !t->is_contiguous())
                    wrong("the gate's gradient must be as the gate");
                p = static_cast<std::remove_reference_t<decltype(p)>>(address(*t));
            } else {
                p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(vector(t, a.cols));
            }
        };
        parameter(2, a.dpost);
        parameter(3, a.dpost_bias);
        parameter(4, a.dgate);
        parameter(5, a.dpre);
        parameter(6, a.dpre_bias);
        void* s = stream(*x);
        // New matrices are aligned as the fast kernels want them, wherever they will lie.
        if (at[0] >= 0) a.dx = reinterpret_cast<void*>(256);
        if (at[1] >= 0) a.dy = reinterpret_cast<void*>(256);
        const int64_t size = fasgd_join_workspace(&a);
        if (size < 0) throw Status{size};
        made.add(size, at::kByte, &a.workspace);
        a.workspace_bytes = size;
        made.make();
        unlocked([&] { return (int64_t)fasgd_join_grad(&a, s); });
        return tuple({object(made, at[0], out[0]), object(made, at[1], out[1]), object(made, at[2], out[2]),
                      object(made, at[3], out[3]), object(made, at[4], out[4]), object(made, at[5], out[5]),
                      object(made, at[6], out[6])});
    });
}

/* balance(logits, chosen, balance, z, groups, valid, upstream, grad)
 * -> (loss, counts, dlogits or None) */
PyObject* py_balance(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return entry(nargs, 8, [&]() -> PyObject* {
        const Tensor *logits = tensor(args[0]), *chosen = tensor(args[1]), *valid = tensor(args[5]), *up = tensor(args[6]);
        if (logits == nullptr || chosen == nullptr) wrong("a tensor is expected");
        one_device({logits, chosen, valid, up});
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
        a.top = chosen->dim() > 0 ? chosen->size(-1) : 0;
        if (chosen->scalar_type() != at::kInt || !chosen->is_contiguous() || chosen->numel() != m.rows * a.top)
            wrong("chosen must be contiguous int32 [..., top] on the GPU, a row for each of logits");
        a.chosen = static_cast<int32_t*>(address(*chosen));
        if (valid != nullptr) {
            if ((valid->scalar_type() != at::kByte && valid->scalar_type() != at::kBool) || !valid->is_contiguous() ||
                valid->numel() != m.rows)
                wrong("valid must be contiguous bool or uint8 on the GPU, one for each row");
            a.valid = static_cast<uint8_t*>(address(*valid));
        }
        if (up != nullptr) {
            if (up->scalar_type() != at::kFloat || up->numel() != 1) wrong("upstream must be one fp32 value on the GPU");
            a.upstream = static_cast<float*>(address(*up));
        }
        const int64_t size = fasgd_balance_workspace(&a);
        if (size < 0) throw Status{size};
        New made(*logits);
        int at_dlogits = -1;
        if (args[7] == Py_True) {
            at_dlogits = made.add(*logits, &a.dlogits);
            a.ld_dlogits = m.cols;
        }
        const int64_t shape[2] = {a.groups, m.cols};
        const int at_counts = made.add(shape, at::kInt, &a.counts), at_loss = made.add(3, at::kFloat, &a.loss);
        made.add(size, at::kByte, &a.workspace);
        a.workspace_bytes = size;
        void* s = stream(*logits);
        made.make();
        unlocked([&] { return (int64_t)fasgd_balance(&a, s); });
        return tuple({made.object(at_loss), made.object(at_counts), object(made, at_dlogits, Py_None)});
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
