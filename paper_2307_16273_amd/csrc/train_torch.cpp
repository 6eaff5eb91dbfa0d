// Python's side of the losses and the update (zkdl_token_logprobs, .., zkdl_adamw_step): looks at the tensors, makes the outputs, fills in the
// descriptors and makes the call.  (torch_call.h: what a call takes and returns.)
#include "torch_call.h"

#include <vector>

PyMethodDef* train_methods();

namespace {

decltype(&zkdl_token_logprobs) f_logprobs;
decltype(&zkdl_token_logprobs_backward) f_logprobs_backward;
decltype(&zkdl_policy_loss) f_policy;
decltype(&zkdl_preference_loss) f_preference;
decltype(&zkdl_gradient_norm) f_norm;
decltype(&zkdl_adamw_step) f_adamw;

PyObject* name(const char* s) { return PyUnicode_InternFromString(s); }
#define NAME(s) ([] { static PyObject* const o = name(s); return o; }())

[[noreturn]] void refuse(const char* what, const char* need) {
    PyErr_Format(PyExc_ValueError, "%s: %s", what, need);
    throw Refused();
}

// A contiguous vector of integers of 32 or 64 bits; n < 0: of any length.
const at::Tensor& ints(const Call& c, PyObject* o, const char* what, int64_t n, int* code) {
    const at::Tensor& t = c.tensor(o, what);
    const auto type = t.scalar_type();
    if ((type != at::kInt && type != at::kLong) || t.dim() != 1 || (n >= 0 && t.size(0) != n) || !t.is_cuda() || t.get_device() != c.device || !t.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s: a contiguous int32 or int64 vector%s on device %d is needed", what, n >= 0 ? " with an entry for each row" : "", c.device);
        throw Refused();
    }
    *code = type == at::kInt ? ZKDL_I32 : ZKDL_I64;
    return t;
}
const float* rows_of(const Call& c, PyObject* o, const char* what, int64_t n, bool needed) {
    if (needed && o == Py_None) refuse(what, "needed");
    return (const float*)c.vec(o, what, {}, n);
}
// One number in device memory, or null for None.
const void* number(const Call& c, PyObject* o, const char* what, at::ScalarType type) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = c.tensor(o, what);
    if (t.scalar_type() != type || t.numel() != 1 || !t.is_cuda() || t.get_device() != c.device) {
        PyErr_Format(PyExc_ValueError, "%s: one %s on device %d is needed", what, c10::toString(type), c.device);
        throw Refused();
    }
    return t.data_ptr();
}
double real(PyObject* o) {
    const double x = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) throw Refused();
    return x;
}
// Entry i of a vector as a number, on the same memory.
at::Tensor entry_of(const at::Tensor& t, int64_t i) {
    auto impl = c10::make_intrusive<c10::TensorImpl>(c10::Storage(t.storage()), t.key_set(), t.dtype());
    impl->set_storage_offset(t.storage_offset() + i);
    impl->set_sizes_and_strides(at::IntArrayRef(), at::IntArrayRef());
    return at::Tensor(std::move(impl));
}

// (.., logits, tokens, temperature)
PyObject* token_logprobs(const Call& c, PyObject* const* a) {
    zkdl_mat mx;
    int code;
    const at::Tensor& x = c.mat(a[4], "logits", &mx, 2);
    const int64_t rows = x.size(0);
    const at::Tensor& y = ints(c, a[5], "tokens", rows, &code);
    const float tau = (float)real(a[6]);
    if (!c.ordered) Py_RETURN_NONE;
    at::Tensor logp = c.empty(rows, at::kFloat), top = c.empty(rows, at::kFloat), log_sum = c.empty(rows, at::kFloat);
    const int rc = f_logprobs(c.ctx, &mx, y.data_ptr(), code, tau, floats(logp), floats(top), floats(log_sum));
    if (rc) return PyLong_FromLong(rc);
    Dict d;
    d.put(NAME("logp"), std::move(logp));
    d.put(NAME("top"), std::move(top));
    d.put(NAME("log_sum"), std::move(log_sum));
    return d.d;
}

// (.., dlogp, logits, tokens, top, log_sum, temperature)
PyObject* token_logprobs_backward(const Call& c, PyObject* const* a) {
    zkdl_mat mx, md;
    int code;
    const at::Tensor& x = c.mat(a[5], "logits", &mx, 2);
    const int64_t rows = x.size(0);
    const float* dlogp = rows_of(c, a[4], "dlogp", rows, true);
    const at::Tensor& y = ints(c, a[6], "tokens", rows, &code);
    const float *top = rows_of(c, a[7], "top", rows, true), *log_sum = rows_of(c, a[8], "log_sum", rows, true);
    const float tau = (float)real(a[9]);
    if (!c.ordered) Py_RETURN_NONE;
    at::Tensor out = c.make(x.sizes(), x.scalar_type(), &md);
    const int rc = f_logprobs_backward(c.ctx, dlogp, &mx, y.data_ptr(), code, top, log_sum, tau, &md);
    if (rc) return PyLong_FromLong(rc);
    return THPVariable_Wrap(std::move(out));
}

// (.., logits, tokens, old_logp, advantage, ref_logp, weight, clip_low, clip_high, kl, temperature, gradient)
PyObject* policy_loss(const Call& c, PyObject* const* a) {
    zkdl_mat mx, md;
    int code;
    const at::Tensor& x = c.mat(a[4], "logits", &mx, 2);
    const int64_t rows = x.size(0);
    const at::Tensor& y = ints(c, a[5], "tokens", rows, &code);
    zkdl_policy p = {rows_of(c, a[6], "old_logp", rows, true), rows_of(c, a[7], "advantage", rows, true), rows_of(c, a[8], "ref_logp", rows, false),
                     rows_of(c, a[9], "weight", rows, false), (float)real(a[10]), (float)real(a[11]), (float)real(a[12]), (float)real(a[13])};
    if (!c.ordered) Py_RETURN_NONE;
    at::Tensor sums = c.empty(3, at::kFloat), logp = c.empty(rows, at::kFloat), out;
    if (a[14] == Py_True) out = c.make(x.sizes(), x.scalar_type(), &md);
    const int rc = f_policy(c.ctx, &mx, y.data_ptr(), code, &p, floats(sums), floats(logp), if_there(out, &md));
    if (rc) return PyLong_FromLong(rc);
    Dict d;
    d.put(NAME("loss"), entry_of(sums, 0));
    d.put(NAME("divergence"), entry_of(sums, 1));
    d.put(NAME("clipped"), entry_of(sums, 2));
    d.put(NAME("logp"), std::move(logp));
    d.put(NAME("dlogits"), std::move(out));
    return d.d;
}

// (.., logits, tokens, offsets, ref_logp, weight, beta, target, smoothing, form, average, temperature, gradient)
PyObject* preference_loss(const Call& c, PyObject* const* a) {
    zkdl_mat mx, md;
    int code, off_code;
    const at::Tensor& x = c.mat(a[4], "logits", &mx, 2);
    const int64_t rows = x.size(0);
    const at::Tensor& y = ints(c, a[5], "tokens", rows, &code);
    const at::Tensor& off = ints(c, a[6], "offsets", -1, &off_code);
    if (off.size(0) % 2 == 0) refuse("offsets", "two sequences a pair and the end of the last one are needed, an odd number");
    const int64_t pairs = off.size(0) / 2;
    zkdl_preference p = {};
    p.offsets = off.data_ptr();
    p.offsets_dtype = off_code;
    p.ref_logp = rows_of(c, a[7], "ref_logp", rows, false);
    p.weight = rows_of(c, a[8], "weight", pairs, false);
    p.pairs = (uint64_t)pairs;
    p.beta = (float)real(a[9]);
    p.target = (float)real(a[10]);
    p.smoothing = (float)real(a[11]);
    p.form = (int)PyLong_AsLong(a[12]);
    p.average = a[13] == Py_True;
    p.temperature = (float)real(a[14]);
    if (!c.ordered) Py_RETURN_NONE;
    at::Tensor loss = c.empty({}, at::kFloat), margin = c.empty(pairs, at::kFloat), logp = c.empty(rows, at::kFloat), out;
    if (a[15] == Py_True) out = c.make(x.sizes(), x.scalar_type(), &md);
    const int rc = f_preference(c.ctx, &mx, y.data_ptr(), code, &p, floats(loss), floats(margin), floats(logp), if_there(out, &md));
    if (rc) return PyLong_FromLong(rc);
    Dict d;
    d.put(NAME("loss"), std::move(loss));
    d.put(NAME("margin"), std::move(margin));
    d.put(NAME("logp"), std::move(logp));
    d.put(NAME("dlogits"), std::move(out));
    return d.d;
}

// A list or tuple of contiguous tensors.
struct List {
    PyObject* seq;
    const char* what;
    List(PyObject* o, const char* w) : seq(PySequence_Fast(o, "")), what(w) {
        if (!seq) {
            PyErr_Clear();
            refuse(w, "a list of tensors is needed");
        }
    }
    ~List() { Py_DECREF(seq); }
    List(const List&) = delete;
    Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(seq); }
    const at::Tensor& at(const Call& c, Py_ssize_t i) const {
        const at::Tensor& t = c.tensor(PySequence_Fast_GET_ITEM(seq, i), what);
        if (!t.is_cuda() || t.get_device() != c.device || !t.is_contiguous()) {
            PyErr_Format(PyExc_ValueError, "%s[%zd]: a contiguous tensor on device %d is needed", what, i, c.device);
            throw Refused();
        }
        return t;
    }
    // of floats in 16 or 32 bits
    const at::Tensor& floating(const Call& c, Py_ssize_t i) const {
        const at::Tensor& t = at(c, i);
        const auto type = t.scalar_type();
        if (type != at::kFloat && type != at::kHalf && type != at::kBFloat16) {
            PyErr_Format(PyExc_ValueError, "%s[%zd]: float32, float16 or bfloat16 is needed, not %s", what, i, c10::toString(type));
            throw Refused();
        }
        return t;
    }
    // of a given type and shape
    const at::Tensor& like(const Call& c, Py_ssize_t i, at::ScalarType type, at::IntArrayRef sizes) const {
        const at::Tensor& t = at(c, i);
        if (t.scalar_type() != type || t.sizes() != sizes) {
            PyErr_Format(PyExc_ValueError, "%s[%zd]: %s in the parameter's shape is needed", what, i, c10::toString(type));
            throw Refused();
        }
        return t;
    }
};

// (.., gradients, limit)
PyObject* gradient_norm(const Call& c, PyObject* const* a) {
    const List list(a[4], "gradients");
    const double limit = real(a[5]);
    std::vector<zkdl_vec> v((size_t)list.size());
    for (size_t i = 0; i < v.size(); ++i) {
        const at::Tensor& t = list.floating(c, (Py_ssize_t)i);
        v[i] = {t.data_ptr(), (uint64_t)t.numel(), code_of(t.scalar_type()), 0};
    }
    if (!c.ordered) Py_RETURN_NONE;
    at::Tensor norm = c.empty({}, at::kFloat), factor = c.empty({}, at::kFloat);
    const int rc = f_norm(c.ctx, v.data(), v.size(), (float)limit, floats(norm), floats(factor));
    if (rc) return PyLong_FromLong(rc);
    Dict d;
    d.put(NAME("norm"), std::move(norm));
    d.put(NAME("factor"), std::move(factor));
    return d.d;
}

// (.., params, gradients, m, v, m_scale, v_scale, step, lr, beta1, beta2, eps, decay, factor, seed, bits, values)
PyObject* adamw_step(const Call& c, PyObject* const* a) {
    const List params(a[4], "params"), grads(a[5], "gradients"), ms(a[6], "state m"), vs(a[7], "state v"), m_scales(a[8], "state m_scale"), v_scales(a[9], "state v_scale");
    const Py_ssize_t n = params.size();
    zkdl_adamw how = {};
    how.bits = (int)PyLong_AsLong(a[18]);
    if (PyErr_Occurred()) throw Refused();
    const bool eight = how.bits == 8, values = a[19] == Py_True;
    if (grads.size() != n || ms.size() != n || vs.size() != n || (eight && (m_scales.size() != n || v_scales.size() != n)))
        refuse("params, gradients and state", "as many tensors of each are needed");
    if (values && !eight) refuse("values", "of 8-bit states alone");
    if (THPVariable_Check(a[10])) {
        how.step_ptr = (const int64_t*)number(c, a[10], "step", at::kLong);
    } else {
        how.step = PyLong_AsLongLong(a[10]);
        if (PyErr_Occurred()) throw Refused();
    }
    if (THPVariable_Check(a[11])) how.lr_ptr = (const float*)number(c, a[11], "lr", at::kFloat);
    else how.lr = real(a[11]);
    how.beta1 = real(a[12]);
    how.beta2 = real(a[13]);
    how.eps = real(a[14]);
    how.decay = real(a[15]);
    how.factor = (const float*)number(c, a[16], "factor", at::kFloat);
    how.seed = PyLong_AsUnsignedLongLongMask(a[17]);
    if (PyErr_Occurred()) throw Refused();
    const at::ScalarType type = eight ? at::kByte : at::kFloat;
    std::vector<zkdl_adamw_tensor> t((size_t)n);
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor &p = params.floating(c, i), &g = grads.floating(c, i), &m = ms.like(c, i, type, p.sizes()), &v = vs.like(c, i, type, p.sizes());
        if (g.sizes() != p.sizes()) {
            PyErr_Format(PyExc_ValueError, "gradients[%zd]: the parameter's shape is needed", i);
            throw Refused();
        }
        t[i] = {p.data_ptr(), g.data_ptr(), m.data_ptr(), v.data_ptr(), nullptr, nullptr, nullptr, nullptr, (uint64_t)p.numel(), code_of(p.scalar_type()),
                code_of(g.scalar_type())};
        if (eight) {
            const int64_t blocks[1] = {(p.numel() + 255) / 256};
            t[i].m_scale = (uint8_t*)m_scales.like(c, i, at::kByte, blocks).data_ptr();
            t[i].v_scale = (uint8_t*)v_scales.like(c, i, at::kByte, blocks).data_ptr();
        }
    }
    if (!c.ordered) Py_RETURN_NONE;
    std::vector<at::Tensor> outs;
    if (values) {
        outs.reserve((size_t)(2 * n));
        for (Py_ssize_t i = 0; i < n; ++i)
            for (int k = 0; k < 2; ++k) {
                outs.push_back(c.empty(params.at(c, i).sizes(), at::kFloat));
                (k ? t[i].v_value : t[i].m_value) = floats(outs.back());
            }
    }
    const auto written = [&](auto of) {
        for (Py_ssize_t i = 0; i < n; ++i)
            for (const List* l : {&params, &ms, &vs, &m_scales, &v_scales})
                if (eight || (l != &m_scales && l != &v_scales)) of(l->at(c, i));
    };
    written([](const at::Tensor& x) {
        TORCH_CHECK(!x.is_inference() || c10::InferenceMode::is_enabled(), "adamw_step: tensors of inference mode cannot be updated outside of it");
    });
    const int rc = f_adamw(c.ctx, t.data(), t.size(), &how);
    // what autograd keeps of these tensors is not theirs any more, unless the call was refused
    if (rc != ZKDL_EINVAL && rc != ZKDL_ETOOBIG) written([](const at::Tensor& x) { x.unsafeGetTensorImpl()->bump_version(); });
    if (rc) return PyLong_FromLong(rc);
    PyObject* d = PyDict_New();
    for (int k = 0; k < 2; ++k) {
        PyObject* o = values ? PyList_New(n) : Py_NewRef(Py_None);
        for (Py_ssize_t i = 0; values && i < n; ++i) PyList_SET_ITEM(o, i, THPVariable_Wrap(std::move(outs[2 * i + k])));
        PyDict_SetItem(d, k ? NAME("v") : NAME("m"), o);
        Py_DECREF(o);
    }
    return d;
}

// the addresses of the six entry points, in the order of the declarations above
PyObject* bind_train(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "six addresses");
        return nullptr;
    }
    f_logprobs = (decltype(f_logprobs))PyLong_AsVoidPtr(args[0]);
    f_logprobs_backward = (decltype(f_logprobs_backward))PyLong_AsVoidPtr(args[1]);
    f_policy = (decltype(f_policy))PyLong_AsVoidPtr(args[2]);
    f_preference = (decltype(f_preference))PyLong_AsVoidPtr(args[3]);
    f_norm = (decltype(f_norm))PyLong_AsVoidPtr(args[4]);
    f_adamw = (decltype(f_adamw))PyLong_AsVoidPtr(args[5]);
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

#define TRAIN_METHOD(name, n) {#name, (PyCFunction)(void (*)(void))entry<name, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind_train", (PyCFunction)(void (*)(void))bind_train, METH_FASTCALL, nullptr},
                         TRAIN_METHOD(token_logprobs, 7),
                         TRAIN_METHOD(token_logprobs_backward, 10),
                         TRAIN_METHOD(policy_loss, 15),
                         TRAIN_METHOD(preference_loss, 16),
                         TRAIN_METHOD(gradient_norm, 6),
                         TRAIN_METHOD(adamw_step, 20),
                         {nullptr, nullptr, 0, nullptr}};

}  // namespace

PyMethodDef* train_methods() { return methods; }
