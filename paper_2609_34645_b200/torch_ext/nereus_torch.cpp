// Argument marshalling of paper_2609_34645_b200/logits.py: from torch tensors to the C ABI's calls on logits, with the
// checks of types, devices and shapes.  A decode step's calls are a few microseconds of GPU time each; through ctypes their
// arguments alone took two to three times that.  Host code only; every kernel is in libnereus.so.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <string>

#include "nereus.h"

namespace {

PyObject* g_error = nullptr;        // NereusError(code, what)

// A wrong argument, as ValueError.
struct Wrong {
    std::string what;
};

const at::Tensor& tensor_of(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) throw Wrong{std::string(what) + ": expected a tensor"};
    return THPVariable_Unpack(o);
}

struct View {
    nereus_logits_t v;
    c10::Device     device{c10::DeviceType::CPU};
};

// A tensor or a sequence of column shards; vocab < 0: all columns.
View view_of(PyObject* x, int64_t vocab, const View* like) {
    View r;
    const bool one = THPVariable_Check(x);
    PyObject*  items = nullptr;
    if (!one) {
        items = PySequence_Fast(x, "logits: expected a tensor or a sequence of shards");
        if (!items) throw python_error();
    }
    THPObjectPtr hold(items);
    const int64_t tp = one ? 1 : PySequence_Fast_GET_SIZE(items);
    if (tp < 1 || tp > NEREUS_VOCAB_MAX_TP) throw Wrong{"logits: 1 to " + std::to_string(NEREUS_VOCAB_MAX_TP) + " shards"};
    r.v.tp = (int32_t)tp;
    for (int64_t s = 0; s < tp; ++s) {
        const at::Tensor& t = tensor_of(one ? x : PySequence_Fast_GET_ITEM(items, s), "logits");
        if (t.dim() != 2) throw Wrong{"logits are [rows, columns] tensors"};
        const auto    type = t.scalar_type();
        const int32_t dtype = type == at::kBFloat16 ? NEREUS_BF16 : type == at::kFloat ? NEREUS_FP32 : 0;
        if (!dtype || !t.is_cuda()) throw Wrong{"logits are bf16 or fp32 tensors on a CUDA device"};
        const int64_t rows = t.size(0), cols = t.size(1);
        if (s == 0) {
            r.device = t.device();
            r.v.dtype = dtype;
            r.v.rows = rows;
            r.v.shard_cols = cols;
            r.v.row_stride = rows > 1 ? t.stride(0) : cols;
            r.v.vocab = vocab < 0 ? tp * cols : vocab;
            if (like && r.device != like->device) throw Wrong{"read and written logits are on different devices"};
        } else {
            if (dtype != r.v.dtype || t.device() != r.device || rows != r.v.rows) throw Wrong{"shards differ in type, device or rows"};
            // the last shard of a trimmed vocabulary may be narrower
            if (cols != r.v.shard_cols && (s + 1 < tp || vocab < 0 || cols < std::min(r.v.shard_cols, vocab - s * r.v.shard_cols)))
                throw Wrong{"shards differ in columns"};
            if (rows > 1 && t.stride(0) != r.v.row_stride) throw Wrong{"shards differ in the stride between rows"};
        }
        if (cols > 1 && t.stride(1) != 1) throw Wrong{"logits are contiguous along the vocabulary"};
        r.v.shard[s] = t.data_ptr();
    }
    for (int64_t s = tp; s < NEREUS_VOCAB_MAX_TP; ++s) r.v.shard[s] = nullptr;
    return r;
}

int64_t vocab_of(PyObject* o) {
    if (o == Py_None) return -1;
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v < 0 ? 0 : v;                          // refused by the library
}

// Address of an optional argument of a given type and shape, contiguous; d1 < 0: one dimension.
void* arg_of(PyObject* o, at::ScalarType type, int64_t d0, int64_t d1, const View& like, const char* what) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor_of(o, what);
    const bool fits = d1 < 0 ? t.dim() == 1 && t.size(0) == d0 : t.dim() == 2 && t.size(0) == d0 && t.size(1) == d1;
    if (t.scalar_type() != type || t.device() != like.device || !fits || !t.is_contiguous())
        throw Wrong{std::string(what) + ": expected a contiguous " + (type == at::kInt ? "int32" : "fp32") + " tensor of shape [" +
                    std::to_string(d0) + (d1 < 0 ? "" : ", " + std::to_string(d1)) + "] on the logits' device"};
    return t.data_ptr();
}

// New logits of x's shape, in x's type or another.  Shards are tensors of their own, unless the last is narrower than the
// others: then, as all shards have one stride between rows, they are column slices of one tensor.
PyObject* empty_like(PyObject* x, PyObject* dtype) {
    if (dtype != Py_None && !THPDtype_Check(dtype)) throw Wrong{"out_dtype: expected a torch.dtype"};
    auto make = [&](const at::Tensor& t, c10::IntArrayRef shape) {
        return at::empty(shape, t.options().dtype(dtype == Py_None ? t.scalar_type() : reinterpret_cast<THPDtype*>(dtype)->scalar_type));
    };
    if (THPVariable_Check(x)) return THPVariable_Wrap(make(THPVariable_Unpack(x), THPVariable_Unpack(x).sizes()));
    THPObjectPtr items(PySequence_Fast(x, "logits"));
    if (!items) throw python_error();
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(items.get());
    if (n < 1) throw Wrong{"logits: expected a tensor or a sequence of shards"};          // an iterator, gone through already
    auto shard = [&](Py_ssize_t i) -> const at::Tensor& { return tensor_of(PySequence_Fast_GET_ITEM(items.get(), i), "logits"); };
    THPObjectPtr list(PyList_New(n));
    if (!list) throw python_error();
    const int64_t rows = shard(0).size(0), cols = shard(0).size(1), last = shard(n - 1).size(1);
    const at::Tensor whole = cols == last ? at::Tensor() : make(shard(0), {rows, (n - 1) * cols + last});
    for (Py_ssize_t i = 0; i < n; ++i) {
        PyObject* o = THPVariable_Wrap(whole.defined() ? whole.narrow(1, i * cols, i + 1 < n ? cols : last) : make(shard(i), shard(i).sizes()));
        if (!o) throw python_error();
        PyList_SET_ITEM(list.get(), i, o);
    }
    return list.release();
}

// The caller's tensors that a call has written: autograd has to notice where it had saved one of them.
void written(PyObject* x) {
    auto bump = [](PyObject* o) {
        const at::Tensor& t = tensor_of(o, "logits");
        if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    };
    if (THPVariable_Check(x)) return bump(x);
    THPObjectPtr items(PySequence_Fast(x, "logits"));
    if (!items) throw python_error();
    for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(items.get()); ++i) bump(PySequence_Fast_GET_ITEM(items.get(), i));
}

at::Tensor empty(c10::IntArrayRef shape, at::ScalarType type, const View& like) {
    return at::empty(shape, at::TensorOptions().dtype(type).device(like.device));
}
void* stream_of(const View& v) { return (void*)c10::cuda::getCurrentCUDAStream(v.device.index()).stream(); }

// Raises for an error code of the library.
bool failed(int rc, const char* what) {
    if (rc == NEREUS_OK) return false;
    THPObjectPtr e(PyObject_CallFunction(g_error, "is", rc, what));
    if (e) PyErr_SetObject(g_error, e.get());
    return true;
}

double double_of(PyObject* o) {
    const double d = PyFloat_AsDouble(o);
    if (d == -1.0 && PyErr_Occurred()) throw python_error();
    return d;
}

bool counted(Py_ssize_t got, Py_ssize_t want) {
    if (got == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
    return false;
}

#define NEREUS_BEGIN HANDLE_TH_ERRORS try {
#define NEREUS_END                                       \
    } catch (const Wrong& w) {                           \
        PyErr_SetString(PyExc_ValueError, w.what.c_str()); \
        return nullptr;                                  \
    }                                                    \
    END_HANDLE_TH_ERRORS

// (x, vocab, out, out_dtype, history, prompt_len, total_len, repetition, presence, frequency, bias_ids, bias_values, mask,
// mask_row) -> (out, token, lse)
PyObject* process(PyObject*, PyObject* const* a, Py_ssize_t n) {
    NEREUS_BEGIN
    if (!counted(n, 14)) return nullptr;
    const View x = view_of(a[0], vocab_of(a[1]), nullptr);
    const c10::cuda::OptionalCUDAGuard guard(x.device);
    const int64_t rows = x.v.rows;
    THPObjectPtr out;
    if (a[2] == Py_None) out = empty_like(a[0], a[3]);
    else { Py_INCREF(a[2]); out = a[2]; }
    const View y = view_of(out.get(), x.v.vocab, &x);
    nereus_penalties_t how = {};
    if (a[4] != Py_None) {
        const at::Tensor& h = tensor_of(a[4], "history");
        if (h.scalar_type() != at::kInt || h.dim() != 2 || h.size(0) != rows || h.device() != x.device || (h.size(1) > 1 && h.stride(1) != 1))
            throw Wrong{"history: expected int32 [rows, n], contiguous along n, on the logits' device"};
        if (h.size(1)) {
            how.history = h.const_data_ptr<int32_t>();
            how.history_len = h.size(1);
            how.history_stride = rows > 1 ? h.stride(0) : h.size(1);
            how.prompt_len = (const int32_t*)arg_of(a[5], at::kInt, rows, -1, x, "prompt_len");
            how.total_len = (const int32_t*)arg_of(a[6], at::kInt, rows, -1, x, "total_len");
        }
    } else if (a[5] != Py_None || a[6] != Py_None) {
        throw Wrong{"prompt_len and total_len belong to a history"};
    }
    how.repetition = (const float*)arg_of(a[7], at::kFloat, rows, -1, x, "repetition");
    how.presence = (const float*)arg_of(a[8], at::kFloat, rows, -1, x, "presence");
    how.frequency = (const float*)arg_of(a[9], at::kFloat, rows, -1, x, "frequency");
    if (a[10] != Py_None && tensor_of(a[10], "bias_ids").numel()) {
        how.bias_count = tensor_of(a[10], "bias_ids").size(-1);
        how.bias_ids = (const int32_t*)arg_of(a[10], at::kInt, rows, how.bias_count, x, "bias_ids");
        how.bias_values = (const float*)arg_of(a[11], at::kFloat, rows, how.bias_count, x, "bias_values");
    } else if (a[11] != Py_None && tensor_of(a[11], "bias_values").numel()) {
        throw Wrong{"bias_values belong to bias_ids"};
    }
    if (a[12] != Py_None) {
        const at::Tensor& m = tensor_of(a[12], "mask");
        if (m.scalar_type() != at::kInt || m.dim() != 2 || m.device() != x.device || (m.size(1) > 1 && m.stride(1) != 1) || m.size(1) * 32 < x.v.vocab)
            throw Wrong{"mask: expected int32 [grammars, >= vocab / 32], contiguous along the words"};
        how.mask = m.const_data_ptr<int32_t>();
        how.mask_rows = m.size(0);
        how.mask_stride = m.size(0) > 1 ? m.stride(0) : m.size(1);
        how.mask_row = (const int32_t*)arg_of(a[13], at::kInt, rows, -1, x, "mask_row");
    } else if (a[13] != Py_None) {
        throw Wrong{"mask_row belongs to a mask"};
    }
    at::Tensor token = empty({rows}, at::kInt, x), lse = empty({rows}, at::kFloat, x);
    if (failed(nereus_logits_process(&x.v, &y.v, &how, (int32_t*)token.data_ptr(), (float*)lse.data_ptr(), stream_of(x)), "nereus_logits_process"))
        return nullptr;
    if (a[2] != Py_None) written(a[2]);
    THPObjectPtr t(THPVariable_Wrap(std::move(token))), l(THPVariable_Wrap(std::move(lse)));
    return PyTuple_Pack(3, out.get(), t.get(), l.get());
    NEREUS_END
}

// (x, k, vocab, temperature) -> (values, ids, lse)
PyObject* teacher_top(PyObject*, PyObject* const* a, Py_ssize_t n) {
    NEREUS_BEGIN
    if (!counted(n, 4)) return nullptr;
    const View x = view_of(a[0], vocab_of(a[2]), nullptr);
    const c10::cuda::OptionalCUDAGuard guard(x.device);
    const int64_t k = PyLong_AsLongLong(a[1]);
    if (k == -1 && PyErr_Occurred()) throw python_error();
    const int64_t room = k < 1 || k > NEREUS_TOP_MAX_K ? 1 : k;             // out of range: refused by the library
    at::Tensor values = empty({x.v.rows, room}, at::kFloat, x), ids = empty({x.v.rows, room}, at::kInt, x), lse = empty({x.v.rows}, at::kFloat, x);
    if (failed(nereus_teacher_top(&x.v, room == k ? (int)k : 0, double_of(a[3]), (float*)values.data_ptr(), (int32_t*)ids.data_ptr(),
                                  (float*)lse.data_ptr(), stream_of(x)), "nereus_teacher_top"))
        return nullptr;
    THPObjectPtr v(THPVariable_Wrap(std::move(values))), i(THPVariable_Wrap(std::move(ids))), l(THPVariable_Wrap(std::move(lse)));
    return PyTuple_Pack(3, v.get(), i.get(), l.get());
    NEREUS_END
}

// The arguments that the three distillation calls share: ids, values, lse, weight, divergence, temperature, beta.
nereus_distill_t distill_of(PyObject* const* a, const View& x) {
    const at::Tensor& ids = tensor_of(a[0], "ids");
    if (ids.dim() != 2) throw Wrong{"ids: expected int32 [rows, k]"};
    const int64_t k = ids.size(1), rows = x.v.rows;
    nereus_distill_t how = {};
    how.k = (int32_t)std::min<int64_t>(k, 1 << 20);
    how.ids = (const int32_t*)arg_of(a[0], at::kInt, rows, k, x, "ids");
    how.values = (const float*)arg_of(a[1], at::kFloat, rows, k, x, "values");
    how.lse = (const float*)arg_of(a[2], at::kFloat, rows, -1, x, "lse");
    how.weight = (const float*)arg_of(a[3], at::kFloat, rows, -1, x, "weight");
    how.divergence = (int32_t)PyLong_AsLong(a[4]);
    if (how.divergence == -1 && PyErr_Occurred()) throw python_error();
    how.temperature = double_of(a[5]);
    how.beta = double_of(a[6]);
    return how;
}

// (x, vocab, ids, values, lse, weight, divergence, temperature, beta) -> (loss, saved)
PyObject* distill_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    NEREUS_BEGIN
    if (!counted(n, 9)) return nullptr;
    const View x = view_of(a[0], vocab_of(a[1]), nullptr);
    const c10::cuda::OptionalCUDAGuard guard(x.device);
    const nereus_distill_t how = distill_of(a + 2, x);
    at::Tensor loss = empty({x.v.rows}, at::kFloat, x), saved = empty({x.v.rows, 4}, at::kFloat, x);
    if (failed(nereus_distill_forward(&x.v, &how, (float*)loss.data_ptr(), (float*)saved.data_ptr(), stream_of(x)), "nereus_distill_forward"))
        return nullptr;
    THPObjectPtr l(THPVariable_Wrap(std::move(loss))), s(THPVariable_Wrap(std::move(saved)));
    return PyTuple_Pack(2, l.get(), s.get());
    NEREUS_END
}

// (x, vocab, ids, values, lse, weight, divergence, temperature, beta, saved, grad_loss, grad) -> grad
PyObject* distill_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    NEREUS_BEGIN
    if (!counted(n, 12)) return nullptr;
    const View x = view_of(a[0], vocab_of(a[1]), nullptr);
    const c10::cuda::OptionalCUDAGuard guard(x.device);
    const nereus_distill_t how = distill_of(a + 2, x);
    THPObjectPtr grad;
    if (a[11] == Py_None) grad = empty_like(a[0], Py_None);
    else { Py_INCREF(a[11]); grad = a[11]; }
    const View y = view_of(grad.get(), x.v.vocab, &x);
    const float* saved = (const float*)arg_of(a[9], at::kFloat, x.v.rows, 4, x, "saved");
    const float* up = (const float*)arg_of(a[10], at::kFloat, x.v.rows, -1, x, "grad_loss");
    if (failed(nereus_distill_backward(&x.v, &how, saved, up, &y.v, stream_of(x)), "nereus_distill_backward")) return nullptr;
    if (a[11] != Py_None) written(a[11]);
    return grad.release();
    NEREUS_END
}

// (x, vocab, ids, values, lse, weight, divergence, temperature, beta, grad) -> (loss, grad)
PyObject* distill_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
    NEREUS_BEGIN
    if (!counted(n, 10)) return nullptr;
    const View x = view_of(a[0], vocab_of(a[1]), nullptr);
    const c10::cuda::OptionalCUDAGuard guard(x.device);
    const nereus_distill_t how = distill_of(a + 2, x);
    THPObjectPtr grad;
    if (a[9] == Py_None) grad = empty_like(a[0], Py_None);
    else { Py_INCREF(a[9]); grad = a[9]; }
    const View y = view_of(grad.get(), x.v.vocab, &x);
    at::Tensor loss = empty({x.v.rows}, at::kFloat, x);
    if (failed(nereus_distill_step(&x.v, &how, (float*)loss.data_ptr(), &y.v, stream_of(x)), "nereus_distill_step")) return nullptr;
    if (a[9] != Py_None) written(a[9]);
    THPObjectPtr l(THPVariable_Wrap(std::move(loss)));
    return PyTuple_Pack(2, l.get(), grad.get());
    NEREUS_END
}

// x -> uninitialised logits like x
PyObject* empty_like_of(PyObject*, PyObject* x) {
    NEREUS_BEGIN
    view_of(x, 1, nullptr);
    return empty_like(x, Py_None);
    NEREUS_END
}

PyObject* set_error(PyObject*, PyObject* cls) {
    Py_INCREF(cls);
    Py_XSETREF(g_error, cls);
    Py_RETURN_NONE;
}

#define NEREUS_FAST(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {NEREUS_FAST(process),         NEREUS_FAST(teacher_top),  NEREUS_FAST(distill_forward),
                           NEREUS_FAST(distill_backward), NEREUS_FAST(distill_step), {"empty_like", empty_like_of, METH_O, nullptr},
                           {"set_error", set_error, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_nereus_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__nereus_torch(void) { return PyModule_Create(&g_module); }
