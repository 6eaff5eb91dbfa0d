// Python's side of the 8-bit layer operators (zkdl_quantize_i8, zkdl_rmsnorm_i8, .., zkdl_matmul_i8_backward): looks at the tensors, makes
// the outputs, fills in the descriptors and makes the call.  The operators of a single token are over in a few microseconds, as long as
// Python takes to look at two tensors, so this part is compiled; everything else is binding.py's.
//
// Every function takes (context handle, device, stream of the context, in order, ..).  It returns the outputs; a negative zkdl_err as an
// int; or None where the current stream is not the context's and `in order` is false: the caller then orders the two and calls again.
// Arguments that do not fit raise ValueError.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPStream.h>

#include "../../include/zkdl.h"

namespace {

decltype(&zkdl_quantize_i8) f_quantize;
decltype(&zkdl_rmsnorm_i8) f_rmsnorm;
decltype(&zkdl_rmsnorm_i8_backward) f_rmsnorm_backward;
decltype(&zkdl_matmul_i8) f_matmul;
decltype(&zkdl_matmul_i8_backward) f_matmul_backward;

struct Refused {};      // a Python error is set

int code_of(at::ScalarType t) {
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

PyObject *k_q, *k_scale, *k_rstd, *k_total, *k_values, *k_dx, *k_dweight, *k_da, *k_dw;

struct Dict {
    PyObject* d = PyDict_New();
    void put(PyObject* key, at::Tensor t) {
        PyObject* o = t.defined() ? THPVariable_Wrap(std::move(t)) : Py_NewRef(Py_None);
        PyDict_SetItem(d, key, o);
        Py_DECREF(o);
    }
};

float* floats(const at::Tensor& t) { return (float*)t.data_ptr(); }
const zkdl_mat* if_there(const at::Tensor& t, const zkdl_mat* m) { return t.defined() ? m : nullptr; }

// (.., x, axis, mult, values)
PyObject* quantize_i8(const Call& c, PyObject* const* a) {
    zkdl_mat mx, mq, mv;
    const at::Tensor& x = c.mat(a[4], "x", &mx, 3);
    const long axis = PyLong_AsLong(a[5]);
    if (axis != -1 && axis != -2) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "axis: -1 (a scale for each row) or -2 (a scale for each column)");
        throw Refused();
    }
    const auto sh = x.sizes();
    const auto lead = sh.slice(0, sh.size() - 2);
    const void* mult = c.vec(a[6], "mult", lead, x.size(axis));
    if (!c.ordered) Py_RETURN_NONE;
    c10::SmallVector<int64_t, 2> ss(lead.begin(), lead.end());
    ss.push_back(x.size(axis == -1 ? -2 : -1));
    at::Tensor q = c.make_codes(sh, &mq), scale = c.empty(ss, at::kFloat), v;
    if (a[7] == Py_True) v = c.make(sh, x.scalar_type(), &mv);
    const int rc = f_quantize(c.ctx, &mx, axis == -1 ? 1 : 0, (const float*)mult, &mq, floats(scale), if_there(v, &mv));
    if (rc) return PyLong_FromLong(rc);
    Dict d;
    d.put(k_q, std::move(q));
    d.put(k_scale, std::move(scale));
    d.put(k_values, std::move(v));
    return d.d;
}

// (.., x, weight, residual, eps, values)
PyObject* rmsnorm_i8(const Call& c, PyObject* const* a) {
    zkdl_mat mx, mr, mq, mt, mv;
    const at::Tensor& x = c.mat(a[4], "x", &mx, 2);
    const auto sh = x.sizes();
    int wt = ZKDL_F32;
    const void* w = c.vec(a[5], "weight", {}, sh[1], x.scalar_type(), &wt);
    const bool residual = a[6] != Py_None;
    if (residual) c.mat(a[6], "residual", &mr, 2);
    const float eps = (float)PyFloat_AsDouble(a[7]);
    if (PyErr_Occurred()) throw Refused();
    if (!c.ordered) Py_RETURN_NONE;
    at::Tensor q = c.make_codes(sh, &mq), scale = c.empty(sh[0], at::kFloat), rstd = c.empty(sh[0], at::kFloat), total, v;
    if (residual) total = c.make(sh, x.scalar_type(), &mt);
    if (a[8] == Py_True) v = c.make(sh, x.scalar_type(), &mv);
    const int rc = f_rmsnorm(c.ctx, &mx, residual ? &mr : nullptr, w, wt, eps, &mq, floats(scale), floats(rstd), if_there(total, &mt), if_there(v, &mv));
    if (rc) return PyLong_FromLong(rc);
    Dict d;
    d.put(k_q, std::move(q));
    d.put(k_scale, std::move(scale));
    d.put(k_rstd, std::move(rstd));
    d.put(k_total, std::move(total));
    d.put(k_values, std::move(v));
    return d.d;
}

// (.., dy, h, weight, rstd, dtotal)
PyObject* rmsnorm_i8_backward(const Call& c, PyObject* const* a) {
    zkdl_mat my, mh, mt, mx;
    const at::Tensor& dy = c.mat(a[4], "dy", &my, 2);
    c.mat(a[5], "h", &mh, 2);
    const auto sh = dy.sizes();
    int wt = ZKDL_F32;
    const void* w = c.vec(a[6], "weight", {}, sh[1], dy.scalar_type(), &wt);
    const void* rstd = c.vec(a[7], "rstd", {}, sh[0]);
    const bool more = a[8] != Py_None;
    if (more) c.mat(a[8], "dtotal", &mt, 2);
    if (!c.ordered) Py_RETURN_NONE;
    at::Tensor dx = c.make(sh, dy.scalar_type(), &mx), dw = c.empty(sh[1], at::kFloat);
    const int rc = f_rmsnorm_backward(c.ctx, &my, &mh, w, wt, (const float*)rstd, more ? &mt : nullptr, &mx, floats(dw));
    if (rc) return PyLong_FromLong(rc);
    Dict d;
    d.put(k_dx, std::move(dx));
    d.put(k_dweight, std::move(dw));
    return d.d;
}

// (.., a, b, a_scale, b_scale, trans_a, trans_b, dtype or None)
PyObject* matmul_i8(const Call& c, PyObject* const* a) {
    zkdl_mat ma, mb, mo;
    bool ta, tb;
    const at::Tensor& x = c.mat(a[4], "a", &ma, 3, &ta);
    const at::Tensor& y = c.mat(a[5], "b", &mb, 3, &tb);
    if (x.dim() != y.dim()) {
        PyErr_SetString(PyExc_ValueError, "a and b: two matrices or two stacks");
        throw Refused();
    }
    const bool trans_a = a[8] == Py_True, trans_b = a[9] == Py_True;
    const auto lead = x.sizes().slice(0, x.dim() - 2);
    const int64_t m = x.size(trans_a ? -1 : -2), n = y.size(trans_b ? -2 : -1);
    at::ScalarType type = a[6] == Py_None && a[7] == Py_None ? at::kInt : at::kBFloat16;
    if (a[10] != Py_None) {
        if (!THPDtype_Check(a[10])) {
            PyErr_SetString(PyExc_ValueError, "dtype: int32, float32, float16 or bfloat16");
            throw Refused();
        }
        type = ((THPDtype*)a[10])->scalar_type;
        if (code_of(type) < 0) {
            PyErr_SetString(PyExc_ValueError, "dtype: int32, float32, float16 or bfloat16");
            throw Refused();
        }
    }
    const void *sa = c.vec(a[6], "a_scale", lead, m), *sb = c.vec(a[7], "b_scale", lead, n);
    if (!c.ordered) Py_RETURN_NONE;
    c10::SmallVector<int64_t, 3> sh(lead.begin(), lead.end());
    sh.push_back(m);
    sh.push_back(n);
    at::Tensor out = c.make(sh, type, &mo);
    const int rc = f_matmul(c.ctx, &ma, &mb, trans_a != ta, trans_b != tb, (const float*)sa, (const float*)sb, &mo);
    if (rc) return PyLong_FromLong(rc);
    return THPVariable_Wrap(std::move(out));
}

// (.., dy, a, a_scale, w, w_scale, trans_w, need_da, need_dw)
PyObject* matmul_i8_backward(const Call& c, PyObject* const* a) {
    zkdl_mat my, ma, mw, mda, mdw;
    const at::Tensor& dy = c.mat(a[4], "dy", &my, 3);
    const at::Tensor& x = c.mat(a[5], "a", &ma, 3);
    const at::Tensor& w = c.mat(a[7], "w", &mw, 3);
    if (dy.dim() != x.dim() || dy.dim() != w.dim()) {
        PyErr_SetString(PyExc_ValueError, "dy, a and w: three matrices or three stacks");
        throw Refused();
    }
    const auto lead = dy.sizes().slice(0, dy.dim() - 2);
    const void *sa = c.vec(a[6], "a_scale", lead, dy.size(-2)), *sw = c.vec(a[8], "w_scale", lead, dy.size(-1));
    if (!sa || !sw) {
        if (a[6] == Py_None || a[8] == Py_None) {
            PyErr_SetString(PyExc_ValueError, "a_scale and w_scale are needed");
            throw Refused();
        }
    }
    if (!c.ordered) Py_RETURN_NONE;
    at::Tensor da, dw;
    if (a[10] == Py_True) da = c.make(x.sizes(), dy.scalar_type(), &mda);
    if (a[11] == Py_True) dw = c.make(w.sizes(), at::kFloat, &mdw);
    const int rc = f_matmul_backward(c.ctx, &my, &ma, &mw, a[9] == Py_True, (const float*)sa, (const float*)sw, if_there(da, &mda), if_there(dw, &mdw));
    if (rc) return PyLong_FromLong(rc);
    Dict d;
    d.put(k_da, std::move(da));
    d.put(k_dw, std::move(dw));
    return d.d;
}

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

// the addresses of the five entry points, in the order of the declarations above
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "five addresses");
        return nullptr;
    }
    f_quantize = (decltype(f_quantize))PyLong_AsVoidPtr(args[0]);
    f_rmsnorm = (decltype(f_rmsnorm))PyLong_AsVoidPtr(args[1]);
    f_rmsnorm_backward = (decltype(f_rmsnorm_backward))PyLong_AsVoidPtr(args[2]);
    f_matmul = (decltype(f_matmul))PyLong_AsVoidPtr(args[3]);
    f_matmul_backward = (decltype(f_matmul_backward))PyLong_AsVoidPtr(args[4]);
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

#define L8_METHOD(name, n) {#name, (PyCFunction)(void (*)(void))entry<name, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
                         L8_METHOD(quantize_i8, 8),
                         L8_METHOD(rmsnorm_i8, 9),
                         L8_METHOD(rmsnorm_i8_backward, 9),
                         L8_METHOD(matmul_i8, 11),
                         L8_METHOD(matmul_i8_backward, 12),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_layers8", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__layers8(void) {
    k_q = PyUnicode_InternFromString("q");
    k_scale = PyUnicode_InternFromString("scale");
    k_rstd = PyUnicode_InternFromString("rstd");
    k_total = PyUnicode_InternFromString("total");
    k_values = PyUnicode_InternFromString("values");
    k_dx = PyUnicode_InternFromString("dx");
    k_dweight = PyUnicode_InternFromString("dweight");
    k_da = PyUnicode_InternFromString("da");
    k_dw = PyUnicode_InternFromString("dw");
    return PyModule_Create(&module);
}
