// What the extension modules of the Python package share: errors, workspaces, the interpreter lock.
#pragma once
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdio.h>
#include <string.h>

#include "mcf_internal.h"

namespace {

PyObject *g_error = nullptr; // binding.McfError(status, text)

inline PyObject *fail(int status, const char *text) {
    PyObject *e = PyObject_CallFunction(g_error, "is", status, text);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    return nullptr;
}

inline PyObject *fail_status(int status) {
    const char *more = mcf_last_error();
    char text[512];
    if (*more) snprintf(text, sizeof(text), "%s (%s)", mcf_status_string(status), more);
    else snprintf(text, sizeof(text), "%s", mcf_status_string(status));
    return fail(status, text);
}

// One element broadcast over a whole tensor: every stride is zero, which the C ABI reads as "packed".
inline bool one_element(const at::Tensor &t) {
    if (t.layout() != at::kStrided || t.numel() <= 1) return false;
    for (int64_t d = 0; d < t.dim(); ++d)
        if (t.size(d) > 1 && t.stride(d) != 0) return false;
    return true;
}

// The workspace of a call from torch's allocator, for the device of its operands (which need not be the current one) and the
// stream that the call runs on: given back right after the launches, it is only handed out again to later work of that
// stream.  While the stream is captured it has to stay with the graph instead.  torch's own capture allocates from the graph's
// pool, which does that; where someone else captures, memory given back would be used by others between the replays:
// nullptr then (and in any capture nothing here may end it, so that an allocation may go past the allocator's cache).
inline void *workspace(size_t bytes, hipStream_t stream, c10::Device device) {
    namespace alloc = c10::hip::HIPCachingAllocator;
    c10::DeviceGuard on(device);
    if (!mcf::stream_capturing(stream)) return alloc::raw_alloc_with_stream(bytes, stream);
    c10::hip::HIPStreamCaptureModeGuard allowed(hipStreamCaptureModeRelaxed);
    void *ws = alloc::raw_alloc_with_stream(bytes, stream);
    for (const auto &seg : alloc::snapshot().segments)
        if ((size_t)ws - seg.address < seg.total_size && seg.owner_private_pool_id != c10::MempoolId_t(0, 0)) return ws;
    alloc::raw_delete(ws);
    return nullptr;
}

// The interpreter lock is let go while a call allocates and launches, both of which may wait for the device
// (and work that is queued may wait for a Python thread); costs 0.1 us a call.
struct NoGil {
    PyThreadState *state = PyEval_SaveThread();
    NoGil() = default;
    NoGil(const NoGil &) = delete;
    ~NoGil() { PyEval_RestoreThread(state); }
};

bool is_tensor(PyObject *o) { return THPVariable_Check(o); }

inline PyObject *set_error(PyObject *, PyObject *type) {
    Py_INCREF(type);
    Py_XDECREF(g_error);
    g_error = type;
    Py_RETURN_NONE;
}

} // namespace
