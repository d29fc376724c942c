// What the extension modules of the calls on logits share: how a tensor is looked at, memory from torch's allocator, calls that nothing is thrown across.
//   As in _native, a call that is not the ordinary case -- other types, shapes that do not fit, tensors that cannot be looked at -- is not
// taken (None is returned), and the Python module does, or refuses, what it defines.
#pragma once
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/TracerMode.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <optional>
#include <string>
#include <vector>
#include "../../include/zapformat.h"

namespace {

using at::Tensor;

PyObject *check_py = nullptr;          // binding._check: raises for a return code

struct Failed { int rc; };             // a code of the library

int logit_type(const Tensor &t) { return t.scalar_type() == at::kFloat ? 0 : t.scalar_type() == at::kBFloat16 ? 1 : -1; }
bool has_tangent(const Tensor &t) { return t._fw_grad(0).defined(); }
bool plain(const Tensor &t) { return t.layout() == at::kStrided && t.is_cuda() && !t.is_nested() && !t.unsafeGetTensorImpl()->has_symbolic_sizes_strides() && !t.is_neg() && !t.is_conj() && !has_tangent(t); }
bool matrix(const Tensor &t) { return plain(t) && t.dim() == 2; }
bool rows_without_gaps(const Tensor &t) { return t.size(1) <= 1 || t.stride(1) == 1; }
int64_t row_stride(const Tensor &t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }
void *stream_of(const Tensor &t) { return (void *)c10::hip::getCurrentHIPStream(t.get_device()).stream(); }
// From torch's allocator, without the way through its dispatcher (a call of token_logprobs with four of them 8.0 us of the host, so 6.6).
Tensor fresh(c10::IntArrayRef size, at::ScalarType type, const Tensor &like) { return at::detail::empty_cuda(size, type, like.device(), std::nullopt); }
void must(int rc) { if (rc != ZF_OK) throw Failed{rc}; }

// None for an object that is None, a tensor; false: neither, or not a plain one
bool tensor_or_none(PyObject *o, std::optional<Tensor> *out) {
    if (o == Py_None) { out->reset(); return true; }
    if (!THPVariable_CheckExact(o)) return false;
    *out = THPVariable_Unpack(o);
    return true;
}
bool mask_fits(const std::optional<Tensor> &m, int64_t rows, int64_t V, const Tensor &with) {
    return !m || (matrix(*m) && m->scalar_type() == at::kInt && m->is_contiguous() && m->size(0) == rows && m->size(1) == (V + 31) / 32 && m->device() == with.device());
}

// A saved tensor, or an incoming gradient, for a kernel to read: what hooks on saved tensors give back may lie anywhere, in any order.
Tensor kept(const char *of, const Tensor &t, const char *what, const Tensor &with, at::ScalarType type, c10::IntArrayRef size, bool rows_apart = false) {
    TORCH_CHECK(t.layout() == at::kStrided && t.is_cuda() && !t.is_nested() && t.device() == with.device() && t.scalar_type() == type && t.sizes() == size, of, ": saved ", what,
                " came back with another device, type or shape: ", t.toString(), " ", t.sizes(), " on ", t.device(), " instead of ", size, " on ", with.device());
    TORCH_CHECK(!has_tangent(t), of, ": its gradient has no forward-mode derivative");
    const bool as_it_is = rows_apart ? t.dim() == 2 && t.stride(1) == 1 && row_stride(t) >= t.size(1) : t.is_contiguous();
    return as_it_is && plain(t) ? t : t.detach().resolve_neg().contiguous();
}

// Somebody watches what torch is asked for on this thread: a tracer, which the Python modules refuse, or a dispatch mode that wants to see the allocations.
bool watched() {
    return at::tracer::impl::is_dispatch_enabled() || c10::impl::tls_is_dispatch_key_included(at::DispatchKey::PreDispatch) || c10::impl::TorchDispatchModeTLS::any_modes_set();
}

// Python calls C: no C++ exception goes that way.
typedef PyObject *(*Call)(PyObject *const *, Py_ssize_t);
template <Call F>
PyObject *guarded(PyObject *, PyObject *const *args, Py_ssize_t n) {
    try {
        if (watched()) Py_RETURN_NONE;
        PyObject *r = F(args, n);
        if (r || PyErr_Occurred()) return r;
    } catch (const Failed &e) {
        PyObject *code = PyLong_FromLong(e.rc);
        if (!code) return nullptr;
        PyObject *r = PyObject_CallOneArg(check_py, code);      // raises
        Py_DECREF(code);
        Py_XDECREF(r);
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "an error code that raises nothing");
        return nullptr;
    } catch (...) {}                   // a tensor that torch does not let be looked at, no memory: the Python module meets the same and raises what torch raises
    Py_RETURN_NONE;
}

}  // namespace
