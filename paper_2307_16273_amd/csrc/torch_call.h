// What the parts of Python's side share (layers8_torch.cpp, train_torch.cpp): a call's context, device and stream, tensors looked at and
// made, results as a dict.
//
// Every function takes (context handle, device, stream of the context, in order, ..).  It returns the outputs; a negative zkdl_err as an
// int; or None where the current stream is not the context's and `in order` is false: the caller then orders the two and calls again.
// Arguments that do not fit raise ValueError.
#pragma once
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPStream.h>

#include "../../include/zkdl.h"

namespace {

struct Refused {};      // a Python error is set

inline int code_of(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return ZKDL_F32;
        case at::kHalf: return ZKDL_F16;
        case at::kBFloat16: return ZKDL_BF16;
        case at::kChar: return ZKDL_I8;
        case at::kInt: return ZKDL_I32;
        default: return -1;
    }
}

struct Call {
    zkdl_ctx* ctx;
    int device;
    bool ordered;

    Call(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) {
        if (n != want) {
            PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
            throw Refused();
        }
        ctx = (zkdl_ctx*)PyLong_AsVoidPtr(args[0]);
        device = (int)PyLong_AsLong(args[1]);
        void* stream = PyLong_AsVoidPtr(args[2]);
        if (PyErr_Occurred()) throw Refused();
        ordered = args[3] == Py_True || c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream() == (hipStream_t)stream;
    }
    const at::Tensor& tensor(PyObject* o, const char* what) const {
        if (!THPVariable_Check(o)) {
            PyErr_Format(PyExc_ValueError, "%s: a tensor is needed", what);
            throw Refused();
        }
        return THPVariable_Unpack(o);
    }
    // A stack of matrices (dims 3: or one matrix) whose rows or, with `turned`, columns are adjacent in memory.
    const at::Tensor& mat(PyObject* o, const char* what, zkdl_mat* m, int dims, bool* turned = nullptr) const {
        const at::Tensor& t = tensor(o, what);
        const int code = code_of(t.scalar_type()), d = (int)t.dim();
        if (code < 0 || d < 2 || d > dims || !t.is_cuda() || t.get_device() != device) {
            PyErr_Format(PyExc_ValueError, "%s: %s on device %d of a type the operator knows is needed, not %d dimensions of %s on %s", what,
                         dims == 2 ? "a matrix" : "a matrix or a stack of matrices", device, d, c10::toString(t.scalar_type()), t.device().str().c_str());
            throw Refused();
        }
        const auto sh = t.sizes(), st = t.strides();
        const int64_t rows = sh[d - 2], cols = sh[d - 1];
        *m = {t.data_ptr(), d == 3 ? (uint64_t)sh[0] : 1, (uint64_t)rows, (uint64_t)cols, (uint64_t)st[d - 2], d == 3 ? (uint64_t)st[0] : 0, code, 0};
        if (turned) *turned = false;
        if (st[d - 1] == 1 || cols <= 1) return t;
        if (turned && (st[d - 2] == 1 || rows <= 1)) {
            *turned = true;
            m->rows = (uint64_t)cols;
            m->cols = (uint64_t)rows;
            m->row_stride = (uint64_t)st[d - 1];
            return t;
        }
        PyErr_Format(PyExc_ValueError, "%s: the entries of a row have to be adjacent in memory (strides %lld, %lld)", what, (long long)st[d - 2], (long long)st[d - 1]);
        throw Refused();
    }
    // A contiguous tensor of 32-bit floats (or of `also`) with the sizes `lead` and then n; null for None.
    const void* vec(PyObject* o, const char* what, at::IntArrayRef lead, int64_t n, at::ScalarType also = at::kFloat, int* code = nullptr) const {
        if (o == Py_None) return nullptr;
        const at::Tensor& t = tensor(o, what);
        const auto type = t.scalar_type();
        bool ok = t.dim() == (int64_t)lead.size() + 1 && (type == at::kFloat || type == also) && t.is_cuda() && t.get_device() == device && t.is_contiguous();
        if (ok) ok = t.size(-1) == n && t.sizes().slice(0, lead.size()) == lead;
        if (!ok) {
            PyErr_Format(PyExc_ValueError, "%s: a contiguous float32 tensor of %lld entries%s on device %d is needed", what, (long long)n,
                         lead.empty() ? "" : " for each matrix", device);
            throw Refused();
        }
        if (code) *code = code_of(type);
        return t.data_ptr();
    }
    at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type) const {
        return at::Tensor(at::detail::empty_cuda(sizes, type, c10::Device(c10::DeviceType::CUDA, (c10::DeviceIndex)device), std::nullopt));
    }
    // A new matrix or stack; `pitch`: entries from row to row.
    at::Tensor make(at::IntArrayRef sizes, at::ScalarType type, zkdl_mat* m, int64_t pitch = -1) const {
        const size_t d = sizes.size();
        const int64_t rows = sizes[d - 2], cols = sizes[d - 1];
        if (pitch < 0) pitch = cols;
        at::Tensor t;
        if (pitch == cols) {
            t = empty(sizes, type);
        } else {
            const int64_t strides[3] = {rows * pitch, pitch, 1};
            t = at::Tensor(at::detail::empty_strided_cuda(sizes, at::IntArrayRef(strides + 3 - d, d), type,
                                                          c10::Device(c10::DeviceType::CUDA, (c10::DeviceIndex)device)));
        }
        *m = {t.data_ptr(), d == 3 ? (uint64_t)sizes[0] : 1, (uint64_t)rows, (uint64_t)cols, (uint64_t)pitch, (uint64_t)(rows * pitch), code_of(type), 0};
        return t;
    }
    // New 8-bit matrices: rows start at multiples of 16 bytes, as the products like them.
    at::Tensor make_codes(at::IntArrayRef sizes, zkdl_mat* m) const { return make(sizes, at::kChar, m, (sizes.back() + 15) & -16); }
};

struct Dict {
    PyObject* d = PyDict_New();
    void put(PyObject* key, at::Tensor t) {
        PyObject* o = t.defined() ? THPVariable_Wrap(std::move(t)) : Py_NewRef(Py_None);
        PyDict_SetItem(d, key, o);
        Py_DECREF(o);
    }
};

inline float* floats(const at::Tensor& t) { return (float*)t.data_ptr(); }
inline const zkdl_mat* if_there(const at::Tensor& t, const zkdl_mat* m) { return t.defined() ? m : nullptr; }

template <PyObject* (*F)(const Call&, PyObject* const*), int N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    try {
        return F(Call(args, n, N), args);
    } catch (const Refused&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

}  // namespace
