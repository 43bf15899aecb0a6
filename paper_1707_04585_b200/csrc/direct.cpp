// Calls from Python to the operators on rows of tokens without ctypes.  Small ones are bound by the host: the forward norm of 1 x 4096 takes 6.6 us of
// it when binding.py checks its seven tensors and marshals the call, 2.8 here, launch included (loading 1 x 4096 from 8 bits: 4.3 and 2.5).  The checks
// are the same.  A call answers the entry point's status, or None where anything is not as it has to be: binding.py then checks again, attribute
// by attribute, and says what is wrong.
#include <Python.h>
#include <cstring>
#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include "../../include/revnet.h"

namespace {

struct Refused {};

// A call's arguments: handle, device, descriptor, tensors
struct Call {
    PyObject *const *args;
    Py_ssize_t n;
    Py_ssize_t next = 3;
    int device;
    revnet_ctx *ctx;
    Py_buffer buffer{};

    Call(PyObject *const *a, Py_ssize_t count, Py_ssize_t tensors, const char *desc_type, size_t desc_bytes) : args(a), n(count) {
        if (n != 3 + tensors || strcmp(Py_TYPE(args[2])->tp_name, desc_type) || !PyLong_CheckExact(args[0]) || !PyLong_CheckExact(args[1])) throw Refused();
        ctx = (revnet_ctx *)PyLong_AsVoidPtr(args[0]);
        device = (int)PyLong_AsLong(args[1]);
        if (PyErr_Occurred() || !ctx || device < 0) throw Refused();
        if (PyObject_GetBuffer(args[2], &buffer, PyBUF_SIMPLE)) throw Refused();
        if ((size_t)buffer.len != desc_bytes) { PyBuffer_Release(&buffer); throw Refused(); }
    }
    Call(const Call &) = delete;
    ~Call() { PyBuffer_Release(&buffer); }

    template <class D> const D &desc() const { return *static_cast<const D *>(buffer.buf); }
    void *stream() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }

    const at::Tensor *tensor() {
        PyObject *o = args[next++];
        if (o == Py_None) return nullptr;
        if (!THPVariable_CheckExact(o)) throw Refused();
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda() || t.get_device() != device || t.layout() != at::kStrided || !t.has_storage()) throw Refused();
        return &t;
    }
    static at::ScalarType type(int dtype) { return dtype == REVNET_F32 ? at::kFloat : at::kBFloat16; }
    // [rows][channels], rows ld (0: channels) elements apart
    void *rows(int64_t rows, int64_t channels, int64_t ld, int dtype) {
        const at::Tensor *t = tensor();
        if (!t) return nullptr;
        if (t->scalar_type() != type(dtype) || t->dim() != 2 || t->size(0) != rows || t->size(1) != channels) throw Refused();
        if (ld == 0) ld = channels;
        const bool strided = (t->stride(1) == 1 || channels <= 1) && (t->stride(0) == ld || rows <= 1);
        if (!strided && !(ld == channels && t->is_contiguous())) throw Refused();
        return t->data_ptr();
    }
    void *flat(int64_t count, at::ScalarType dtype = at::kFloat) {
        const at::Tensor *t = tensor();
        if (!t) return nullptr;
        if (t->scalar_type() != dtype || !t->is_contiguous() || t->numel() != count) throw Refused();
        return t->data_ptr();
    }
    void *checkpoint(int64_t rows, int64_t channels) {
        const at::Tensor *t = tensor();
        if (!t) return nullptr;
        const int64_t bytes = ((rows * ((channels + 31) & ~int64_t(31)) + 255) & ~int64_t(255)) + ((channels + 127) >> 7) * ((rows + 63) & ~int64_t(63)) * 4;
        if (t->scalar_type() != at::kByte || !t->is_contiguous() || t->numel() < bytes) throw Refused();
        return t->data_ptr();
    }
    void *workspace(size_t &bytes) {
        const at::Tensor *t = tensor();
        bytes = 0;
        if (!t) return nullptr;
        if (!t->is_contiguous()) throw Refused();
        bytes = (size_t)t->nbytes();
        return t->data_ptr();
    }
};

// Python's lock is given back for the entry point itself, as ctypes does: a launch waits while its stream's queue is full, perhaps for a host function
// that a Python thread has to run.  Made behind the last look at a Python object.
struct Unlocked {
    PyThreadState *state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked &) = delete;
    ~Unlocked() { PyEval_RestoreThread(state); }
};

// (the operands in the binding's order)
template <class F> PyObject *guarded(F &&f) {
    int status;
    try {
        status = f();
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(status);
}
int64_t a_channels(const revnet_act_desc &d) { return d.act == REVNET_ACT_SWIGLU ? d.channels / 2 : d.channels; }

PyObject *act_store(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded([&] {
        Call c(args, n, 3, "ActDesc", sizeof(revnet_act_desc));
        const auto &d = c.desc<revnet_act_desc>();
        void *x = c.rows(d.rows, d.channels, d.ld_x, d.dtype), *ck = c.checkpoint(d.rows, d.channels), *a = c.rows(d.rows, a_channels(d), d.ld_a, d.dtype);
        void *const stream = c.stream();
        Unlocked u;
        return revnet_act_store(c.ctx, &d, x, ck, a, stream);
    });
}
PyObject *act_load(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded([&] {
        Call c(args, n, 2, "ActDesc", sizeof(revnet_act_desc));
        const auto &d = c.desc<revnet_act_desc>();
        void *ck = c.checkpoint(d.rows, d.channels), *a = c.rows(d.rows, a_channels(d), d.ld_a, d.dtype);
        void *const stream = c.stream();
        Unlocked u;
        return revnet_act_load(c.ctx, &d, ck, a, stream);
    });
}
PyObject *act_bwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded([&] {
        Call c(args, n, 4, "ActDesc", sizeof(revnet_act_desc));
        const auto &d = c.desc<revnet_act_desc>();
        void *ck = c.checkpoint(d.rows, d.channels), *da = c.rows(d.rows, a_channels(d), d.ld_a, d.dtype), *dx = c.rows(d.rows, d.channels, d.ld_x, d.dtype);
        void *a_ck = c.checkpoint(d.rows, a_channels(d));
        void *const stream = c.stream();
        Unlocked u;
        return revnet_act_bwd(c.ctx, &d, ck, da, dx, a_ck, stream);
    });
}
PyObject *rmsnorm_fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded([&] {
        Call c(args, n, 7, "NormDesc", sizeof(revnet_norm_desc));
        const auto &d = c.desc<revnet_norm_desc>();
        auto stream_row = [&] { return c.rows(d.rows, d.channels, d.ld_stream, d.stream_dtype); };
        auto branch_row = [&] { return c.rows(d.rows, d.channels, d.ld_branch, d.branch_dtype); };
        void *x = stream_row(), *r = branch_row(), *gamma = c.flat(d.channels), *h = stream_row(), *out = branch_row(), *ck = c.checkpoint(d.rows, d.channels);
        void *rstd = c.flat(d.rows);
        void *const stream = c.stream();
        Unlocked u;
        return revnet_rmsnorm_fwd(c.ctx, &d, x, r, (const float *)gamma, h, out, ck, (float *)rstd, stream);
    });
}
PyObject *rmsnorm_bwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded([&] {
        Call c(args, n, 10, "NormDesc", sizeof(revnet_norm_desc));
        const auto &d = c.desc<revnet_norm_desc>();
        auto stream_row = [&] { return c.rows(d.rows, d.channels, d.ld_stream, d.stream_dtype); };
        auto branch_row = [&] { return c.rows(d.rows, d.channels, d.ld_branch, d.branch_dtype); };
        void *dn = branch_row(), *dh = stream_row(), *h = stream_row(), *ck = c.checkpoint(d.rows, d.channels), *rstd = c.flat(d.rows), *gamma = c.flat(d.channels);
        void *dx = stream_row(), *dr = branch_row(), *dgamma = c.flat(d.channels);
        size_t bytes;
        void *ws = c.workspace(bytes);
        void *const stream = c.stream();
        Unlocked u;
        return revnet_rmsnorm_bwd(c.ctx, &d, dn, dh, h, ck, (const float *)rstd, (const float *)gamma, dx, dr, (float *)dgamma, ws, bytes, stream);
    });
}
PyObject *linear_wgrad(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded([&] {
        Call c(args, n, 5, "WgradDesc", sizeof(revnet_wgrad_desc));
        const auto &d = c.desc<revnet_wgrad_desc>();
        void *dy = c.rows(d.rows, d.cout, d.ld_dy, d.dy_dtype), *ck = c.checkpoint(d.rows, d.cin), *gamma = c.flat(d.cin), *dW = c.flat((int64_t)d.cin * d.cout);
        size_t bytes;
        void *ws = c.workspace(bytes);
        void *const stream = c.stream();
        Unlocked u;
        return revnet_linear_wgrad(c.ctx, &d, dy, ck, (const float *)gamma, (float *)dW, ws, bytes, stream);
    });
}
PyObject *logprobs_fwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded([&] {
        Call c(args, n, 7, "LogprobDesc", sizeof(revnet_logprob_desc));
        const auto &d = c.desc<revnet_logprob_desc>();
        void *logits = c.rows(d.rows, d.vocab, d.ld, d.dtype), *targets = c.flat(d.rows, at::kInt), *logp = c.flat(d.rows), *entropy = c.flat(d.rows);
        void *lse = c.flat(d.rows), *top = c.flat(d.rows * d.k), *index = c.flat(d.rows * d.k, at::kInt);
        void *const stream = c.stream();
        Unlocked u;
        return revnet_logprobs_fwd(c.ctx, &d, logits, (const int32_t *)targets, (float *)logp, (float *)entropy, (float *)lse, (float *)top, (int32_t *)index, stream);
    });
}
PyObject *logprobs_bwd(PyObject *, PyObject *const *args, Py_ssize_t n) {
    return guarded([&] {
        Call c(args, n, 7, "LogprobDesc", sizeof(revnet_logprob_desc));
        const auto &d = c.desc<revnet_logprob_desc>();
        void *logits = c.rows(d.rows, d.vocab, d.ld, d.dtype), *targets = c.flat(d.rows, at::kInt), *lse = c.flat(d.rows), *entropy = c.flat(d.rows);
        void *dlogp = c.flat(d.rows), *dentropy = c.flat(d.rows), *dlogits = c.rows(d.rows, d.vocab, d.ld, d.dtype);
        void *const stream = c.stream();
        Unlocked u;
        return revnet_logprobs_bwd(c.ctx, &d, logits, (const int32_t *)targets, (const float *)lse, (const float *)entropy, (const float *)dlogp, (const float *)dentropy,
                                   dlogits, stream);
    });
}

#define CALL(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL(act_store), CALL(act_load), CALL(act_bwd), CALL(rmsnorm_fwd), CALL(rmsnorm_bwd), CALL(linear_wgrad), CALL(logprobs_fwd), CALL(logprobs_bwd),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_direct", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the versions whose headers are in here (build.py); binding.py takes the module for no others
PyMODINIT_FUNC PyInit__direct() {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", BUILT_FOR)) { Py_DECREF(m); return nullptr; }
    return m;
}
