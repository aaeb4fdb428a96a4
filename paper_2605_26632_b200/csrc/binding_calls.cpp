// The calls of the Python binding that are made once per layer, as plain CPython functions: tensors are read through
// torch's own objects, the result is allocated, and the C ABI is called, without a Python frame or a ctypes object in
// between.  On the smallest layers (7 us of GPU work) the host side is what a caller waits for.
//
// A function takes a call only if every argument has its plain form: tensors of torch's own classes, strided, on CUDA, with
// no wrapper around them (vmap, functionalisation, subclasses), integers as Python ints, no torch-function or
// dispatch mode.  Anything
// else -- wrong types among it -- is answered with None, and the caller (binding.py) takes its general path, which is where
// arguments are refused.  Otherwise the result is what the general path returns, or the library's status as an int.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/Context.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/TensorBody.h>
#include <ATen/cuda/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>

#include "../../include/lynx.h"

namespace {

// dense CUDA tensors, with the bookkeeping every one of them carries (autograd, autocast, views)
bool plain_keys(const at::Tensor& t) {
    constexpr c10::DispatchKeySet allowed({c10::DispatchKey::CUDA, c10::DispatchKey::ADInplaceOrView, c10::DispatchKey::AutogradCUDA,
                                           c10::DispatchKey::AutocastCUDA});
    return (t.key_set().raw_repr() & ~allowed.raw_repr()) == 0 && t.has_storage();
}

struct Args {
    bool ok = true;

    const at::Tensor* tensor(PyObject* o) {
        if (!THPVariable_CheckExact(o)) return fail();
        const at::Tensor& t = THPVariable_Unpack(o);
        return t.defined() && plain_keys(t) ? &t : fail();
    }
    const at::Tensor* tensor_or_none(PyObject* o) { return o == Py_None ? nullptr : tensor(o); }
    // 2-D bf16 with unit inner stride
    const at::Tensor* matrix(PyObject* o) {
        const at::Tensor* t = tensor(o);
        return t && t->dim() == 2 && t->scalar_type() == at::kBFloat16 && t->stride(1) == 1 ? t : fail();
    }
    const at::Tensor* two_d(const at::Tensor* t) { return t && t->dim() == 2 ? t : fail(); }
    int64_t integer(PyObject* o) {
        if (!PyLong_CheckExact(o)) return fail(), 0;
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) return PyErr_Clear(), fail(), 0;
        return v;
    }
    lynx_ctx* context(PyObject* o) { return reinterpret_cast<lynx_ctx*>(integer(o)); }

private:
    const at::Tensor* fail() {
        ok = false;
        return nullptr;
    }
};

void* ptr(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
template <class T>
T* ptr_as(const at::Tensor* t) { return static_cast<T*>(ptr(t)); }
int64_t ld(const at::Tensor* t) { return t ? t->stride(0) : 0; }
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }
// (What at::empty comes to on a CUDA device, without the dispatcher's way there: a call that makes two tensors 5.1 -> 4.6 us.  In
// torch's deterministic mode at::empty also fills the new memory, which rows of no group show.)
at::Tensor empty(at::IntArrayRef shape, const at::Tensor& like, at::ScalarType type = at::kBFloat16) {
    if (C10_UNLIKELY(at::globalContext().deterministicAlgorithms() && at::globalContext().deterministicFillUninitializedMemory()))
        return at::empty(shape, at::TensorOptions().dtype(type).device(like.device()));
    return at::Tensor(at::detail::empty_cuda(shape, type, like.device(), std::nullopt));
}

// What a call returns: `out` as it came in if there was one, else the new tensor.
PyObject* give(PyObject* given, const at::Tensor& made) { return given != Py_None ? Py_NewRef(given) : THPVariable_Wrap(made); }

bool takes(Py_ssize_t nargs, Py_ssize_t want) {
    return nargs == want && !at::impl::torch_function_mode_enabled() && !c10::impl::TorchDispatchModeTLS::any_modes_set();
}

// layer(ctx, X, W, bias, mode, residual, out, fuse)
PyObject* layer(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!takes(n, 8)) Py_RETURN_NONE;
    Args g;
    lynx_ctx* ctx = g.context(a[0]);
    const at::Tensor *X = g.matrix(a[1]), *W = g.matrix(a[2]), *bias = g.tensor_or_none(a[3]), *res = g.tensor_or_none(a[5]);
    const int64_t mode = g.integer(a[4]), fuse = g.integer(a[7]);
    const at::Tensor* out = a[6] == Py_None ? nullptr : g.two_d(g.tensor(a[6]));
    if (res) g.two_d(res);
    if (!g.ok) Py_RETURN_NONE;
    at::Tensor made;
    int s;
    {
        pybind11::gil_scoped_release no_gil;
        const int64_t M = X->size(0), K = X->size(1), N = W->size(0);
        if (!out) out = &(made = empty({M, N}, *X));
        s = lynx_act_sparse_linear(ctx, ptr(X), M, K, ld(X), ptr(W), N, ld(W), ptr(bias), static_cast<lynx_comp_mode>(mode), ptr(res), ld(res),
                                   ptr(out), ld(out), static_cast<lynx_fuse_mode>(fuse), stream());
    }
    return s ? PyLong_FromLong(s) : give(a[6], made);
    END_HANDLE_TH_ERRORS
}

// layer_lora(ctx, X, W, LA, LB, bias, mode, residual, out)
PyObject* layer_lora(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!takes(n, 9)) Py_RETURN_NONE;
    Args g;
    lynx_ctx* ctx = g.context(a[0]);
    const at::Tensor *X = g.matrix(a[1]), *W = g.matrix(a[2]), *LA = g.matrix(a[3]), *LB = g.matrix(a[4]), *bias = g.tensor_or_none(a[5]),
                     *res = g.tensor_or_none(a[7]);
    const int64_t mode = g.integer(a[6]);
    const at::Tensor* out = a[8] == Py_None ? nullptr : g.two_d(g.tensor(a[8]));
    if (res) g.two_d(res);
    if (!g.ok) Py_RETURN_NONE;
    at::Tensor made;
    int s;
    {
        pybind11::gil_scoped_release no_gil;
        const int64_t M = X->size(0), K = X->size(1), N = W->size(0), R = LB->size(0);
        if (!out) out = &(made = empty({M, N}, *X));
        s = lynx_act_sparse_linear_lora(ctx, ptr(X), M, K, ld(X), ptr(W), N, ld(W), ptr(bias), ptr(LA), ld(LA), ptr(LB), ld(LB), R,
                                        static_cast<lynx_comp_mode>(mode), ptr(res), ld(res), ptr(out), ld(out), stream());
    }
    return s ? PyLong_FromLong(s) : give(a[8], made);
    END_HANDLE_TH_ERRORS
}

// layer_fp8(ctx, X, Wq, wscale, bias, mode, residual, out, row_amax)
PyObject* layer_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!takes(n, 9)) Py_RETURN_NONE;
    Args g;
    lynx_ctx* ctx = g.context(a[0]);
    const at::Tensor *X = g.matrix(a[1]), *Wq = g.two_d(g.tensor(a[2])), *ws = g.tensor_or_none(a[3]), *bias = g.tensor_or_none(a[4]),
                     *res = g.tensor_or_none(a[6]), *amax = g.tensor_or_none(a[8]);
    const int64_t mode = g.integer(a[5]);
    const at::Tensor* out = a[7] == Py_None ? nullptr : g.two_d(g.tensor(a[7]));
    if (res) g.two_d(res);
    if (!g.ok) Py_RETURN_NONE;
    at::Tensor made;
    int s;
    {
        pybind11::gil_scoped_release no_gil;
        const int64_t M = X->size(0), K = X->size(1), N = Wq->size(0);
        if (!out) out = &(made = empty({M, N}, *X));
        s = lynx_act_sparse_linear_fp8(ctx, ptr(X), M, K, ld(X), ptr_as<float>(amax), ptr(Wq), N, ld(Wq), ptr_as<float>(ws), ptr(bias),
                                       static_cast<lynx_comp_mode>(mode), ptr(res), ld(res), ptr(out), ld(out), stream());
    }
    return s ? PyLong_FromLong(s) : give(a[7], made);
    END_HANDLE_TH_ERRORS
}

// prune(ctx, X, mode, values, meta, row_scale) -> (values, meta, row_scale or None)
PyObject* prune(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!takes(n, 6)) Py_RETURN_NONE;
    Args g;
    lynx_ctx* ctx = g.context(a[0]);
    const at::Tensor *X = g.matrix(a[1]), *values = g.tensor_or_none(a[3]), *meta = g.tensor_or_none(a[4]), *scale = g.tensor_or_none(a[5]);
    const int64_t mode = g.integer(a[2]);
    if (!g.ok) Py_RETURN_NONE;
    const bool scaled = mode == LYNX_COMP_ROW || mode == LYNX_COMP_TENSOR;
    at::Tensor v, m, sc;
    int s;
    {
        pybind11::gil_scoped_release no_gil;
        const int64_t M = X->size(0), K = X->size(1);
        if (!values) values = &(v = empty({M, K / 2}, *X));
        if (!meta) meta = &(m = empty({static_cast<int64_t>(lynx_meta_bytes(M, K))}, *X, at::kByte));
        if (!scale && scaled) scale = &(sc = empty({M}, *X, at::kFloat));
        s = lynx_prune_compress(ctx, ptr(X), M, K, ld(X), ptr(values), ptr(meta), ptr_as<float>(scale), static_cast<lynx_comp_mode>(mode),
                                stream());
    }
    if (s) return PyLong_FromLong(s);
    PyObject* t = PyTuple_New(3);
    if (!t) return nullptr;
    PyTuple_SET_ITEM(t, 0, give(a[3], v));
    PyTuple_SET_ITEM(t, 1, give(a[4], m));
    PyTuple_SET_ITEM(t, 2, sc.defined() ? THPVariable_Wrap(sc) : Py_NewRef(a[5]));
    return t;
    END_HANDLE_TH_ERRORS
}

// gemm(ctx, values, meta, W, bias, row_scale, residual, out)
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!takes(n, 8)) Py_RETURN_NONE;
    Args g;
    lynx_ctx* ctx = g.context(a[0]);
    const at::Tensor *values = g.matrix(a[1]), *meta = g.tensor(a[2]), *W = g.matrix(a[3]), *bias = g.tensor_or_none(a[4]),
                     *scale = g.tensor_or_none(a[5]), *res = g.tensor_or_none(a[6]);
    const at::Tensor* out = a[7] == Py_None ? nullptr : g.two_d(g.tensor(a[7]));
    if (res) g.two_d(res);
    if (!g.ok) Py_RETURN_NONE;
    at::Tensor made;
    int s;
    {
        pybind11::gil_scoped_release no_gil;
        const int64_t M = values->size(0), K = values->size(1) * 2, N = W->size(0);
        if (!out) out = &(made = empty({M, N}, *values));
        const lynx_comp comp{ptr_as<float>(scale), ptr(res), ld(res)};
        s = lynx_sparse_linear(ctx, ptr(values), ptr(meta), M, K, ptr(W), N, ld(W), ptr(bias), &comp, ptr(out), ld(out), stream());
    }
    return s ? PyLong_FromLong(s) : give(a[7], made);
    END_HANDLE_TH_ERRORS
}

// ---- MXFP4 operands and products grouped by expert ----
// These take a call only if every tensor is on the context's device, which is the current one, and has the shape and type that
// the general path asks for.
struct MxArgs : Args {
    int device;
    explicit MxArgs(PyObject* dev) : device(static_cast<int>(integer(dev))) {
        if (ok && c10::cuda::current_device() != device) ok = false;
    }
    bool need(bool condition) { return ok = ok && condition; }
    const at::Tensor* on_device(PyObject* o) {
        const at::Tensor* t = tensor(o);
        return t && need(t->device().index() == device) ? t : nullptr;
    }
    const at::Tensor* dense(PyObject* o, at::ScalarType type, int64_t dim) {
        const at::Tensor* t = on_device(o);
        return t && need(t->scalar_type() == type && t->dim() == dim && t->is_contiguous()) ? t : nullptr;
    }
    const at::Tensor* rows(PyObject* o) {
        const at::Tensor* t = on_device(o);
        return t && need(t->scalar_type() == at::kBFloat16 && t->dim() == 2 && (t->stride(1) == 1 || t->size(1) == 1)) ? t : nullptr;
    }
    const at::Tensor* shaped(PyObject* o, int64_t M, int64_t N) {
        if (o == Py_None) return nullptr;
        const at::Tensor* t = rows(o);
        return t && need(t->size(0) == M && t->size(1) == N) ? t : nullptr;
    }
    const at::Tensor* scales(PyObject* o, int64_t M, int64_t K, int64_t groups, bool ragged) {
        const at::Tensor* t = on_device(o);
        return t && need(t->scalar_type() == at::kByte && t->is_contiguous() && t->numel() >= bytes(M, K, groups, ragged)) ? t : nullptr;
    }
    static int64_t bytes(int64_t M, int64_t K, int64_t groups, bool ragged) {
        return static_cast<int64_t>(lynx_mxfp4_scale_bytes(M, K, groups, ragged));
    }
    // int32 [groups + 1], or null for None; `groups` is left as it is then
    const at::Tensor* offsets(PyObject* o, int64_t& groups) {
        if (o == Py_None) return nullptr;
        const at::Tensor* t = dense(o, at::kInt, 1);
        if (!t || !need(t->numel() >= 2)) return nullptr;
        groups = t->numel() - 1;
        return t;
    }
};
int64_t row_pitch(const at::Tensor* t) { return !t ? 0 : t->size(0) > 1 ? t->stride(0) : t->size(1); }

// One product: X (bf16 rows, quantised in the call if the weights are MXFP4) or its codes and scales, plain or grouped.
struct MxProduct {
    const at::Tensor *X = nullptr, *codes = nullptr, *scales = nullptr, *offsets = nullptr, *W = nullptr, *ws = nullptr, *bias = nullptr,
                     *row_scale = nullptr, *residual = nullptr, *out = nullptr;
    int64_t M = 0, K = 0, N = 0, groups = 1;

    // the arguments from `a` on: [offsets,] W, [wscales,] bias, row_scale, residual, out
    void read(MxArgs& g, PyObject* const* a, bool grouped, bool mx) {
        if (grouped) {
            offsets = g.offsets(*a++, groups);
            g.need(offsets != nullptr);
        }
        const int64_t dim = grouped ? 3 : 2;
        if (mx) {
            W = g.dense(*a++, at::kByte, dim);
        } else {
            W = g.on_device(*a++);
            if (W) g.need(W->scalar_type() == at::kBFloat16 && W->dim() == 3 && W->stride(2) == 1 && W->stride(0) == W->size(1) * W->stride(1));
        }
        if (!g.ok || !W) return;
        N = W->size(dim - 2);
        g.need(W->size(dim - 1) == (mx ? K / 2 : K) && (!grouped || W->size(0) == groups));
        if (!g.ok) return;
        if (mx) ws = g.scales(*a++, groups * N, K, groups, false);
        if (*a != Py_None) {
            bias = g.dense(*a, at::kBFloat16, grouped ? 2 : 1);
            if (bias) g.need(bias->size(0) == (grouped ? groups : N) && (!grouped || bias->size(1) == N));
        }
        if (*++a != Py_None) {
            row_scale = g.dense(*a, at::kFloat, 1);
            if (row_scale) g.need(row_scale->size(0) == M);
        }
        residual = g.shaped(*++a, M, N);
        out = g.shaped(*++a, M, N);
    }

    PyObject* call(lynx_ctx* ctx, PyObject* given, bool grouped, bool mx) {
        at::Tensor made, own;
        int s;
        {
            pybind11::gil_scoped_release no_gil;
            const at::Tensor& like = X ? *X : *codes;
            if (!out) out = &(made = empty({M, N}, like));
            const lynx_comp comp{ptr_as<float>(row_scale), ptr(residual), row_pitch(residual)};
            const int32_t* off = ptr_as<int32_t>(offsets);
            void *y = ptr(out), *st = stream();
            if (!mx) {
                s = lynx_grouped_linear(ctx, ptr(X), M, K, row_pitch(X), off, groups, ptr(W), N, W->stride(1), ptr(bias), &comp, y, row_pitch(out), st);
            } else if (X) {
                // where the activations are quantised: memory of the call's own (M K / 2 is a multiple of 16)
                char *c = nullptr, *sc = nullptr;
                if (grouped || lynx_mxfp4_layer_needs_codes(M, K)) {
                    own = empty({M * (K / 2) + MxArgs::bytes(M, K, groups, grouped)}, like, at::kByte);
                    c = ptr_as<char>(&own);
                    sc = c + M * (K / 2);
                }
                s = grouped ? lynx_act_grouped_linear_mxfp4(ctx, ptr(X), M, K, row_pitch(X), off, groups, c, sc, ptr(W), ptr(ws), N, ptr(bias), &comp,
                                                            y, row_pitch(out), st)
                            : lynx_act_linear_mxfp4(ctx, ptr(X), M, K, row_pitch(X), c, sc, ptr(W), ptr(ws), N, ptr(bias), &comp, y, row_pitch(out),
                                                    st);
            } else {
                s = grouped ? lynx_grouped_linear_mxfp4(ctx, ptr(codes), ptr(scales), M, K, off, groups, ptr(W), ptr(ws), N, ptr(bias), &comp, y,
                                                        row_pitch(out), st)
                            : lynx_linear_mxfp4(ctx, ptr(codes), ptr(scales), M, K, ptr(W), ptr(ws), N, ptr(bias), &comp, y, row_pitch(out), st);
            }
        }
        return s ? PyLong_FromLong(s) : give(given, made);
    }
};

// X times W: (ctx, device, X, [offsets,] W, [wscales,] bias, row_scale, residual, out)
PyObject* product_of_rows(PyObject* const* a, Py_ssize_t n, bool grouped, bool mx) {
    const Py_ssize_t want = 8 + grouped + mx;
    if (!takes(n, want)) Py_RETURN_NONE;
    MxArgs g(a[1]);
    lynx_ctx* ctx = g.context(a[0]);
    MxProduct p;
    p.X = g.rows(a[2]);
    if (!g.ok || !p.X) Py_RETURN_NONE;
    p.M = p.X->size(0), p.K = p.X->size(1);
    p.read(g, a + 3, grouped, mx);
    if (!g.ok) Py_RETURN_NONE;
    return p.call(ctx, a[want - 1], grouped, mx);
}
// codes and scales times W: (ctx, device, codes, scales, [offsets,] W, wscales, bias, row_scale, residual, out)
PyObject* product_of_codes(PyObject* const* a, Py_ssize_t n, bool grouped) {
    const Py_ssize_t want = 10 + grouped;
    if (!takes(n, want)) Py_RETURN_NONE;
    MxArgs g(a[1]);
    lynx_ctx* ctx = g.context(a[0]);
    MxProduct p;
    p.codes = g.dense(a[2], at::kByte, 2);
    if (!g.ok || !p.codes) Py_RETURN_NONE;
    p.M = p.codes->size(0), p.K = p.codes->size(1) * 2;
    p.read(g, a + 4, grouped, true);
    if (!g.ok) Py_RETURN_NONE;
    p.scales = g.scales(a[3], p.M, p.K, p.groups, grouped);
    if (!g.ok) Py_RETURN_NONE;
    return p.call(ctx, a[want - 1], grouped, true);
}
PyObject* mx_layer(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    return product_of_rows(a, n, false, true);
    END_HANDLE_TH_ERRORS
}
PyObject* mx_grouped_layer(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    return product_of_rows(a, n, true, true);
    END_HANDLE_TH_ERRORS
}
PyObject* grouped(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    return product_of_rows(a, n, true, false);
    END_HANDLE_TH_ERRORS
}
PyObject* mx_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    return product_of_codes(a, n, false);
    END_HANDLE_TH_ERRORS
}
PyObject* mx_grouped(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    return product_of_codes(a, n, true);
    END_HANDLE_TH_ERRORS
}

// mx_quantize(ctx, device, X, offsets, groups, codes, scales) -> (codes, scales)
PyObject* mx_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!takes(n, 7)) Py_RETURN_NONE;
    MxArgs g(a[1]);
    lynx_ctx* ctx = g.context(a[0]);
    const at::Tensor* X = g.rows(a[2]);
    int64_t groups = g.integer(a[4]);
    const at::Tensor* off = g.offsets(a[3], groups);
    if (!g.ok || !X || !g.need(groups >= 1)) Py_RETURN_NONE;
    const int64_t M = X->size(0), K = X->size(1);
    const at::Tensor* codes = a[5] == Py_None ? nullptr : g.dense(a[5], at::kByte, 2);
    if (codes) g.need(codes->size(0) == M && codes->size(1) == K / 2);
    const at::Tensor* scales = a[6] == Py_None ? nullptr : g.scales(a[6], M, K, groups, off != nullptr);
    if (!g.ok) Py_RETURN_NONE;
    at::Tensor c, sc;
    int s;
    {
        pybind11::gil_scoped_release no_gil;
        if (!codes) codes = &(c = empty({M, K / 2}, *X, at::kByte));
        if (!scales) scales = &(sc = empty({MxArgs::bytes(M, K, groups, off != nullptr)}, *X, at::kByte));
        s = lynx_quantize_mxfp4(ctx, ptr(X), M, K, row_pitch(X), ptr_as<int32_t>(off), groups, ptr(codes), ptr(scales), stream());
    }
    if (s) return PyLong_FromLong(s);
    PyObject* t = PyTuple_New(2);
    if (!t) return nullptr;
    PyTuple_SET_ITEM(t, 0, give(a[5], c));
    PyTuple_SET_ITEM(t, 1, give(a[6], sc));
    return t;
    END_HANDLE_TH_ERRORS
}
// mx_dequantize(ctx, device, codes, scales, offsets, groups, out)
PyObject* mx_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!takes(n, 7)) Py_RETURN_NONE;
    MxArgs g(a[1]);
    lynx_ctx* ctx = g.context(a[0]);
    const at::Tensor* codes = g.dense(a[2], at::kByte, 2);
    int64_t groups = g.integer(a[5]);
    const at::Tensor* off = g.offsets(a[4], groups);
    if (!g.ok || !codes || !g.need(groups >= 1)) Py_RETURN_NONE;
    const int64_t M = codes->size(0), K = codes->size(1) * 2;
    const at::Tensor *scales = g.scales(a[3], M, K, groups, off != nullptr), *out = g.shaped(a[6], M, K);
    if (!g.ok) Py_RETURN_NONE;
    at::Tensor made;
    int s;
    {
        pybind11::gil_scoped_release no_gil;
        if (!out) out = &(made = empty({M, K}, *codes));
        s = lynx_dequantize_mxfp4(ctx, ptr(codes), ptr(scales), M, K, ptr_as<int32_t>(off), groups, ptr(out), row_pitch(out), stream());
    }
    return s ? PyLong_FromLong(s) : give(a[6], made);
    END_HANDLE_TH_ERRORS
}

#define LYNX_FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {LYNX_FAST(layer), LYNX_FAST(layer_lora), LYNX_FAST(layer_fp8), LYNX_FAST(prune), LYNX_FAST(gemm), LYNX_FAST(mx_layer),
                         LYNX_FAST(mx_grouped_layer), LYNX_FAST(grouped), LYNX_FAST(mx_linear), LYNX_FAST(mx_grouped), LYNX_FAST(mx_quantize),
                         LYNX_FAST(mx_dequantize), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_lynx_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__lynx_calls() { return PyModule_Create(&module); }
