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
#include <ATen/ops/empty_like.h>
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

// ---- routed experts and the score over classes ------------------------------------------
int32_t* ints(const Tensor& t, const char* what) {
    if (t.scalar_type() != at::kInt || !t.is_contiguous()) wrong(what);
    return static_cast<int32_t*>(address(t));
}
void same_type(const Tensor& t, const Tensor& of) {
    if (t.scalar_type() != of.scalar_type()) wrong("matrices of one type are expected");
}

/* A matrix, or several one step apart, whose rows or (flip) columns are consecutive values. */
struct Matrices {
    int64_t first, rows, cols, ld, step;
    int32_t flip;
    void* p;
    Matrices(const Tensor& t, int64_t dims) {
        if (t.dim() != dims) wrong(dims == 2 ? "a matrix is expected" : "[experts, inputs, outputs] is expected");
        first = t.size(0);
        rows = t.size(-2);
        cols = t.size(-1);
        const int64_t down = t.stride(-2), along = t.stride(-1);
        if (along == 1 || cols == 1) {
            flip = 0;
            ld = down;
        } else if (down == 1 || rows == 1) {
            flip = 1;
            ld = along;
        } else {
            wrong("the values of a matrix' rows or columns must be contiguous");
        }
        step = dims == 3 ? t.stride(0) : 0;
        p = address(t);
    }
};
/* A new tensor like t, in its layout (torch's empty_like): dense ones keep their strides. */
at::Tensor alike(const Tensor& t) { return at::empty_like(t); }

/* route(chosen, experts) -> (offsets, order, place) */
PyObject* py_route(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return entry(nargs, 2, [&]() -> PyObject* {
        const Tensor* chosen = tensor(args[0]);
        if (chosen == nullptr) wrong("a tensor is expected");
        one_device({chosen});
        fasgd_route_args a;
        std::memset(&a, 0, sizeof a);
        if (chosen->dim() == 0) wrong("chosen must be contiguous int32 on the GPU, [..., top]");
        a.chosen = ints(*chosen, "chosen must be contiguous int32 on the GPU");
        a.top = chosen->size(-1);
        a.rows = a.top != 0 ? chosen->numel() / a.top : 0;
        a.experts = whole(args[1]);
        const int64_t size = fasgd_route_workspace(&a);
        if (size < 0) throw Status{size};
        New made(*chosen);
        const int offsets = made.add(a.experts + 1, at::kInt, &a.offsets), order = made.add(chosen->numel(), at::kInt, &a.order),
                  place = made.add(*chosen, &a.place);
        made.add(size, at::kByte, &a.workspace);
        a.workspace_bytes = size;
        void* s = stream(*chosen);
        made.make();
        unlocked([&] { return (int64_t)fasgd_route(&a, s); });
        return tuple({made.object(offsets), made.object(order), made.object(place)});
    });
}

/* A route (offsets, order, place) into a struct of the calls between rows and places. */
struct Way {
    const Tensor *order, *place;
    explicit Way(PyObject* o) {
        if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 3) wrong("a route is (offsets, order, place)");
        order = tensor(PyTuple_GET_ITEM(o, 1));
        place = tensor(PyTuple_GET_ITEM(o, 2));
        if (order == nullptr || place == nullptr) wrong("a tensor is expected");
    }
    void fill(fasgd_exchange_args& a, const Tensor& of, const Tensor* weight) const {
        std::memset(&a, 0, sizeof a);
        if (place->dim() == 0) wrong("a route's place is [..., top]");
        a.top = place->size(-1);
        a.rows = a.top != 0 ? place->numel() / a.top : 0;
        a.place = ints(*place, "a route's place must be contiguous int32 on the GPU");
        a.order = ints(*order, "a route's order must be contiguous int32 on the GPU");
        if (order->numel() != place->numel()) wrong("a route's order and place have as many entries as each other");
        a.dtype = dtype_of(of);
        if (weight != nullptr) {
            if (weight->scalar_type() != at::kFloat || weight->numel() != place->numel() || !weight->is_contiguous())
                wrong("weight must be contiguous fp32, one for each entry");
            a.weight = static_cast<float*>(address(*weight));
        }
    }
};
void at_rows(fasgd_exchange_args& a, const Tensor& t) {
    const Matrix m(t);
    if (m.rows != a.rows || (a.cols != 0 && m.cols != a.cols))
        wrong("a matrix with a row for each of the route's is expected, as wide as its places");
    a.cols = m.cols;
    a.row_values = m.p;
    a.ld_rows = m.ld;
}
Matrix at_places(fasgd_exchange_args& a, const Tensor& t) {
    const Matrix m(t);
    if (m.rows != a.rows * a.top || (a.cols != 0 && m.cols != a.cols))
        wrong("a matrix with a row for each of the route's places is expected, as wide as its rows");
    a.cols = m.cols;
    return m;
}

/* gather(x, route, out) -> out */
PyObject* py_gather(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return entry(nargs, 3, [&]() -> PyObject* {
        const Tensor *x = tensor(args[0]), *out = tensor(args[2]);
        const Way way(args[1]);
        if (x == nullptr) wrong("a tensor is expected");
        one_device({x, way.order, way.place, out});
        fasgd_exchange_args a;
        way.fill(a, *x, nullptr);
        at_rows(a, *x);
        New made(*x);
        int k = -1;
        if (out == nullptr) {
            const int64_t shape[2] = {a.rows * a.top, a.cols};
            k = made.add(shape, x->scalar_type(), &a.places);
            a.ld_places = a.cols;
        } else {
            same_type(*out, *x);
            const Matrix m = at_places(a, *out);
            a.places = m.p;
            a.ld_places = m.ld;
        }
        void* s = stream(*x);
        made.make();
        unlocked([&] { return (int64_t)fasgd_gather(&a, s); });
        return object(made, k, args[2]);
    });
}

/* combine(y, route, weight, out) -> out */
PyObject* py_combine(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return entry(nargs, 4, [&]() -> PyObject* {
        const Tensor *y = tensor(args[0]), *weight = tensor(args[2]), *out = tensor(args[3]);
        const Way way(args[1]);
        if (y == nullptr) wrong("a tensor is expected");
        one_device({y, way.order, way.place, weight, out});
        fasgd_exchange_args a;
        way.fill(a, *y, weight);
        const Matrix m = at_places(a, *y);
        a.places = m.p;
        a.ld_places = m.ld;
        New made(*y);
        int k = -1;
        if (out == nullptr) {
            c10::SmallVector<int64_t, 5> shape(way.place->sizes().begin(), way.place->sizes().end());
            shape.back() = a.cols;
            k = made.add(shape, y->scalar_type(), &a.row_values);
            a.ld_rows = a.cols;
        } else {
            same_type(*out, *y);
            at_rows(a, *out);
        }
        void* s = stream(*y);
        made.make();
        unlocked([&] { return (int64_t)fasgd_combine(&a, s); });
        return object(made, k, args[3]);
    });
}

/* combine_grad(y, route, weight, dout, dy, dweight) -> (dy, dweight) */
PyObject* py_combine_grad(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return entry(nargs, 6, [&]() -> PyObject* {
        const Tensor *y = tensor(args[0]), *weight = tensor(args[2]), *dout = tensor(args[3]), *dy = tensor(args[4]),
                     *dweight = tensor(args[5]);
        const Way way(args[1]);
        if (y == nullptr || dout == nullptr) wrong("a tensor is expected");
        one_device({y, way.order, way.place, weight, dout, dy, dweight});
        if (weight == nullptr) wrong("the gradient of a combination without weights is gather's");
        fasgd_exchange_args a;
        way.fill(a, *y, weight);
        const Matrix m = at_places(a, *y);
        a.places = m.p;
        a.ld_places = m.ld;
        same_type(*dout, *y);
        at_rows(a, *dout);
        New made(*y);
        int at_dy = -1, at_dweight = -1;
        if (dy == nullptr) {
            const int64_t shape[2] = {a.rows * a.top, a.cols};
            at_dy = made.add(shape, y->scalar_type(), &a.dplaces);
            a.ld_dplaces = a.cols;
        } else {
            same_type(*dy, *y);
            const Matrix d = at_places(a, *dy);
            a.dplaces = d.p;
            a.ld_dplaces = d.ld;
        }
        if (dweight == nullptr) {
            at_dweight = made.add(*weight, &a.dweight);
        } else {
            if (dweight->scalar_type() != at::kFloat || dweight->numel() != weight->numel() || !dweight->is_contiguous())
                wrong("the weights' gradient must be as the weights");
            a.dweight = static_cast<float*>(address(*dweight));
        }
        void* s = stream(*y);
        made.make();
        unlocked([&] { return (int64_t)fasgd_combine_grad(&a, s); });
        return tuple({object(made, at_dy, args[4]), object(made, at_dweight, args[5])});
    });
}

/* The struct of the experts' products without results. */
void products(fasgd_multiply_args& a, const Tensor& x, const Tensor& w, const Tensor& offsets) {
    std::memset(&a, 0, sizeof a);
    const Matrix m(x);
    a.x = m.p;
    a.rows = m.rows;
    a.inputs = m.cols;
    a.ld_x = m.ld;
    a.dtype = dtype_of(x);
    const Matrices e(w, 3);
    a.w = e.p;
    a.experts = e.first;
    a.outputs = e.cols;
    a.ld_w = e.ld;
    a.step_w = e.step;
    a.w_flip = e.flip;
    if (e.rows != a.inputs) wrong("w is [experts, x's columns, outputs]");
    if (w.scalar_type() != at::kFloat && w.scalar_type() != x.scalar_type()) wrong("w is of fp32 or of x's type");
    a.w_dtype = dtype_of(w);
    a.offsets = ints(offsets, "offsets must be contiguous int32 on the GPU");
    if (offsets.numel() != a.experts + 1) wrong("offsets has one entry more than there are experts");
}

/* multiply(x, w, offsets, out) -> out */
PyObject* py_multiply(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return entry(nargs, 4, [&]() -> PyObject* {
        const Tensor *x = tensor(args[0]), *w = tensor(args[1]), *offsets = tensor(args[2]), *out = tensor(args[3]);
        if (x == nullptr || w == nullptr || offsets == nullptr) wrong("a tensor is expected");
        one_device({x, w, offsets, out});
        fasgd_multiply_args a;
        products(a, *x, *w, *offsets);
        New made(*x);
        int k = -1;
        if (out == nullptr) {
            c10::SmallVector<int64_t, 5> shape(x->sizes().begin(), x->sizes().end());
            shape.back() = a.outputs;
            k = made.add(shape, x->scalar_type(), &a.y);
            a.ld_y = a.outputs;
            a.y = reinterpret_cast<void*>(256);
        } else {
            same_type(*out, *x);
            const Matrix m(*out);
            if (m.rows != a.rows || m.cols != a.outputs) wrong("out is [x's rows, w's outputs]");
            a.y = m.p;
            a.ld_y = m.ld;
        }
        void* s = stream(*x);
        const int64_t size = fasgd_multiply_workspace(&a);
        if (size < 0) throw Status{size};
        if (size > 0) made.add(size, at::kByte, &a.workspace);
        a.workspace_bytes = size;
        made.make();
        unlocked([&] { return (int64_t)fasgd_multiply(&a, s); });
        return object(made, k, args[3]);
    });
}

/* A result that is laid out like `of`: the caller's (given), or a new tensor. */
struct Alike {
    Tensor own;
    PyObject* given;
    const Tensor& take(PyObject* o, const Tensor* t, const Tensor& of, const char* what) {
        given = o;
        if (t == nullptr) {
            own = alike(of);
            return own;
        }
        same_type(*t, of);
        if (t->sizes() != of.sizes()) wrong(what);
        return *t;
    }
    PyObject* object(const New& made) const { return own.defined() ? THPVariable_Wrap(own) : ::object(made, -1, given); }
};

/* multiply_grad(x, w, offsets, dy, whether dx, whether dw, dx, dw) -> (dx, dw) */
PyObject* py_multiply_grad(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return entry(nargs, 8, [&]() -> PyObject* {
        const Tensor *x = tensor(args[0]), *w = tensor(args[1]), *offsets = tensor(args[2]), *dy = tensor(args[3]),
                     *dx = tensor(args[6]), *dw = tensor(args[7]);
        if (x == nullptr || w == nullptr || offsets == nullptr || dy == nullptr) wrong("a tensor is expected");
        one_device({x, w, offsets, dy, dx, dw});
        fasgd_multiply_args a;
        products(a, *x, *w, *offsets);
        const Matrix d(*dy);
        same_type(*dy, *x);
        if (d.rows != a.rows || d.cols != a.outputs) wrong("dy is [x's rows, w's outputs]");
        a.dy = d.p;
        a.ld_dy = d.ld;
        const bool by_x = args[4] == Py_True, by_w = args[5] == Py_True;
        if ((dx != nullptr && !by_x) || (dw != nullptr && !by_w)) wrong("a place for a gradient that is not wanted");
        New made(*x);
        int at_dx = -1;
        Alike of_w;
        of_w.given = Py_None;
        if (by_x && dx == nullptr) {
            at_dx = made.add(*x, &a.dx);
            a.ld_dx = a.inputs;
            a.dx = reinterpret_cast<void*>(256);
        } else if (by_x) {
            same_type(*dx, *x);
            const Matrix m(*dx);
            if (m.rows != a.rows || m.cols != a.inputs) wrong("x's gradient is as x");
            a.dx = m.p;
            a.ld_dx = m.ld;
        }
        if (by_w) {
            const Matrices m(of_w.take(args[7], dw, *w, "w's gradient is as w"), 3);
            a.dw = m.p;
            a.ld_dw = m.ld;
            a.step_dw = m.step;
            a.dw_flip = m.flip;
        }
        void* s = stream(*x);
        const int64_t size = by_x || by_w ? fasgd_multiply_workspace(&a) : 0;
        if (size < 0) throw Status{size};
        if (size > 0) made.add(size, at::kByte, &a.workspace);
        a.workspace_bytes = size;
        made.make();
        unlocked([&] { return (int64_t)fasgd_multiply_grad(&a, s); });
        return tuple({object(made, at_dx, args[6]), of_w.object(made)});
    });
}

/* score(z, w, labels, upstream, whether dz, whether dw, known loss, rows and lse (or Nones), dz, dw)
 * -> (loss, rows, dz, dw, lse) */
PyObject* py_score(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    return entry(nargs, 11, [&]() -> PyObject* {
        const Tensor *z = tensor(args[0]), *w = tensor(args[1]), *labels = tensor(args[2]), *up = tensor(args[3]),
                     *loss = tensor(args[6]), *rows = tensor(args[7]), *lse = tensor(args[8]), *dz = tensor(args[9]),
                     *dw = tensor(args[10]);
        if (z == nullptr || w == nullptr || labels == nullptr) wrong("a tensor is expected");
        one_device({z, w, labels, up, loss, rows, lse, dz, dw});
        fasgd_score_args a;
        std::memset(&a, 0, sizeof a);
        const Matrix m(*z);
        a.z = m.p;
        a.rows = m.rows;
        a.cols = m.cols;
        a.ld_z = m.ld;
        a.dtype = dtype_of(*z);
        const Matrices e(*w, 2);
        a.w = e.p;
        a.classes = e.cols;
        a.ld_w = e.ld;
        a.w_flip = e.flip;
        same_type(*w, *z);
        if (e.rows != a.cols) wrong("w is [z's columns, classes]");
        if (labels->scalar_type() != at::kLong || !labels->is_contiguous() || labels->numel() != a.rows)
            wrong("labels must be contiguous int64 on the GPU, one for each row");
        a.labels = static_cast<int64_t*>(address(*labels));
        if (up != nullptr) {
            if (up->scalar_type() != at::kFloat || up->numel() != 1) wrong("upstream must be one fp32 value on the GPU");
            a.upstream = static_cast<float*>(address(*up));
        }
        const bool by_z = args[4] == Py_True, by_w = args[5] == Py_True;
        if ((dz != nullptr && !by_z) || (dw != nullptr && !by_w)) wrong("a place for a gradient that is not wanted");
        New made(*z);
        int at_dz = -1, at_loss = -1, at_rows = -1, at_lse = -1;
        Alike of_w;
        of_w.given = Py_None;
        if (by_z && dz == nullptr) {
            at_dz = made.add(*z, &a.dz);
            a.ld_dz = a.cols;
            a.dz = reinterpret_cast<void*>(256);
        } else if (by_z) {
            same_type(*dz, *z);
            const Matrix d(*dz);
            if (d.rows != a.rows || d.cols != a.cols) wrong("z's gradient is as z");
            a.dz = d.p;
            a.ld_dz = d.ld;
        }
        if (by_w) {
            const Matrices d(of_w.take(args[10], dw, *w, "w's gradient is as w"), 2);
            a.dw = d.p;
            a.ld_dw = d.ld;
            a.dw_flip = d.flip;
        }
        if (rows == nullptr || lse == nullptr) {
            at_loss = made.add(1, at::kFloat, &a.loss);
            at_rows = made.add(labels->sizes(), at::kFloat, &a.row_loss);
            at_lse = made.add(labels->sizes(), at::kFloat, &a.lse);
            a.loss = a.row_loss = a.lse = reinterpret_cast<float*>(256);
        } else {
            for (const Tensor* t : {rows, lse})
                if (t->scalar_type() != at::kFloat || t->numel() != a.rows || !t->is_contiguous())
                    wrong("known rows and lse must be contiguous fp32, one for each row");
            a.row_loss = static_cast<float*>(address(*rows));
            a.lse = static_cast<float*>(address(*lse));
            a.known = 1;
        }
        void* s = stream(*z);
        const int64_t size = fasgd_score_workspace(&a);
        if (size < 0) throw Status{size};
        made.add(size, at::kByte, &a.workspace);
        a.workspace_bytes = size;
        made.make();
        unlocked([&] { return (int64_t)fasgd_score(&a, s); });
        const auto kept = [&](int k, PyObject* given) {      // what was known is not written into
            if (k >= 0) return made.object(k);
            Py_INCREF(given);
            return given;
        };
        return tuple({kept(at_loss, args[6]), kept(at_rows, args[7]), object(made, at_dz, args[9]), of_w.object(made),
                      kept(at_lse, args[8])});
    });
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(dropout), METHOD(join), METHOD(join_grad), METHOD(balance), METHOD(route), METHOD(gather),
                         METHOD(combine), METHOD(combine_grad), METHOD(multiply), METHOD(multiply_grad), METHOD(score), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_client", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__client(void) {
    PyObject* m = PyModule_Create(&module);
    if (m != nullptr && PyModule_AddStringConstant(m, "torch_version", BUILT_FOR_TORCH) < 0) Py_CLEAR(m);
    return m;
}
