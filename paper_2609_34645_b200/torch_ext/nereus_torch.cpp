// Argument marshalling of paper_2609_34645_b200/logits.py and cache.py: from torch tensors to the C ABI's calls, with the
// checks of types, devices and shapes.  A decode step's calls are a few microseconds of GPU time each; through ctypes their
// arguments alone took two to three times that.  Host code only; every kernel is in libnereus.so.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>
#include <c10/core/StorageImpl.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <algorithm>
#include <string>
#include <vector>

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
// The same in half the time: a decode step's calls have several results of a few hundred bytes each.  On the current device, as
// the caching allocator has it for the current stream.
template <class T> at::Tensor fresh(c10::IntArrayRef shape) {
    int64_t n = sizeof(T);
    for (int64_t d : shape) n *= d;
    auto*         allocator = c10::cuda::CUDACachingAllocator::get();
    c10::Storage  storage(c10::make_intrusive<c10::StorageImpl>(c10::StorageImpl::use_byte_size_t(), (size_t)n, allocator->allocate((size_t)n), allocator, true));
    auto          impl = c10::make_intrusive<c10::TensorImpl>(std::move(storage), c10::DispatchKeySet(c10::DispatchKey::CUDA), caffe2::TypeMeta::Make<T>());
    impl->set_sizes_contiguous(shape);
    return at::Tensor(std::move(impl));
}
void* stream_of(const View& v) { return (void*)c10::cuda::getCurrentCUDAStream(v.device.index()).stream(); }

// Raises for an error code of the library.
bool failed(int rc, const char* what) {
    if (rc == NEREUS_OK) return false;
    THPObjectPtr e(PyObject_CallFunction(g_error, "is", rc, what));
    if (e) PyErr_SetObject(g_error, e.get());
    return true;
}

int64_t int_of(PyObject* o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
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

// (x, vocab, score, k, beams, ended, norm, settle) -> (score, parent, token)
PyObject* beam_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
    NEREUS_BEGIN
    if (!counted(n, 8)) return nullptr;
    const View x = view_of(a[0], vocab_of(a[1]), nullptr);
    const c10::cuda::OptionalCUDAGuard guard(x.device);
    const int64_t rows = x.v.rows, k = int_of(a[3]), beams = int_of(a[4]);
    nereus_beams_t how = {};
    // out of range: refused by the library
    how.beams = beams < 1 || beams > NEREUS_BEAM_MAX ? 0 : (int32_t)beams;
    how.k = k < 1 || k > NEREUS_BEAM_MAX_K ? 0 : (int32_t)k;
    how.settle = PyObject_IsTrue(a[7]);
    if (how.settle < 0) throw python_error();
    if (a[2] == Py_None) throw Wrong{"score: expected a tensor"};
    how.score = (const float*)arg_of(a[2], at::kFloat, rows, -1, x, "score");
    how.ended = (const int32_t*)arg_of(a[5], at::kInt, rows, -1, x, "ended");
    how.norm = (const float*)arg_of(a[6], at::kFloat, rows, -1, x, "norm");
    const int64_t requests = how.beams ? rows / how.beams : 0, room = std::max<int64_t>(how.k, 1);
    at::Tensor score = fresh<float>({requests, room}), parent = fresh<int32_t>({requests, room}), token = fresh<int32_t>({requests, room});
    size_t bytes = 0;
    if (failed(nereus_beam_workspace(&x.v, &how, &bytes), "nereus_beam_select")) return nullptr;
    const c10::DataPtr workspace = c10::cuda::CUDACachingAllocator::get()->allocate(bytes);
    if (failed(nereus_beam_select(&x.v, &how, workspace.get(), bytes, (float*)score.data_ptr(), (int32_t*)parent.data_ptr(), (int32_t*)token.data_ptr(),
                                  stream_of(x)), "nereus_beam_select"))
        return nullptr;
    THPObjectPtr s(THPVariable_Wrap(std::move(score))), p(THPVariable_Wrap(std::move(parent))), t(THPVariable_Wrap(std::move(token)));
    return PyTuple_Pack(3, s.get(), p.get(), t.get());
    NEREUS_END
}

// ---- states and cache ------------------------------------------------------------------------------------------

// The tensors of an argument that is one or a sequence of them, with one device, element size, shape and strides.
struct Buffers {
    const at::Tensor* t[NEREUS_MAX_BUFFERS];
    size_t       n = 0;
    THPObjectPtr hold;
    c10::Device  device{c10::DeviceType::CPU};
};
void buffers_of(PyObject* x, const char* what, Buffers* b) {
    if (THPVariable_Check(x)) b->t[b->n++] = &THPVariable_Unpack(x);
    else {
        b->hold = PySequence_Fast(x, "expected a tensor or a sequence of tensors");
        if (!b->hold) throw python_error();
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(b->hold.get());
        if (n > NEREUS_MAX_BUFFERS) throw Wrong{std::string(what) + ": at most " + std::to_string(NEREUS_MAX_BUFFERS) + " buffers"};
        for (Py_ssize_t i = 0; i < n; ++i) b->t[b->n++] = &tensor_of(PySequence_Fast_GET_ITEM(b->hold.get(), i), what);
    }
    if (!b->n) return;
    const at::Tensor& u = *b->t[0];
    if (!u.is_cuda() || u.dim() < 1) throw Wrong{std::string(what) + ": expected tensors [rows, ...] on a CUDA device"};
    b->device = u.device();
    const c10::IntArrayRef sizes = u.sizes(), strides = u.strides();
    const size_t size = u.itemsize();
    const bool   empty = u.numel() == 0;
    for (size_t i = 1; i < b->n; ++i) {
        const at::Tensor& t = *b->t[i];
        if (t.device() != b->device || t.itemsize() != size || t.sizes() != sizes || (!empty && t.strides() != strides))
            throw Wrong{std::string(what) + ": the buffers differ in device, element size, shape or strides"};
    }
}
// Tensors that a call writes.
void writable(const Buffers& b, const char* what) {
    if (!at::GradMode::is_enabled()) return;
    for (size_t i = 0; i < b.n; ++i)
        if (b.t[i]->requires_grad()) throw Wrong{std::string(what) + ": written without a gradient; detach it"};
}
void written(const Buffers& b) {
    for (size_t i = 0; i < b.n; ++i)
        if (!b.t[i]->is_inference()) b.t[i]->unsafeGetTensorImpl()->bump_version();
}
// Whether dimensions from `first` on lie one after the other; *elements: their product.
bool packed(const at::Tensor& t, int64_t first, int64_t* elements) {
    int64_t step = 1;
    for (int64_t d = t.dim() - 1; d >= first; --d) {
        if (t.size(d) != 1 && t.stride(d) != step) return false;
        step *= t.size(d);
    }
    *elements = step;
    return true;
}

// States [rows, ..., tokens, ...], tokens at `dim`.
nereus_states_t states_of(const Buffers& b, int64_t dim, const char* what) {
    if (!b.n) throw Wrong{std::string(what) + ": expected a tensor at least"};
    const at::Tensor& t = *b.t[0];
    if (dim < 0) dim += t.dim();
    if (dim < 1 || (dim >= t.dim() && !(dim == 1 && t.dim() == 1))) throw Wrong{std::string(what) + ": dim is the tokens' axis, behind that of the rows"};
    nereus_states_t s;
    s.outer_stride = 0;
    const int64_t size = t.element_size();
    s.buffers = (int32_t)b.n;
    if (t.size(0) > INT32_MAX) throw Wrong{std::string(what) + ": too many rows"};
    s.rows = (int32_t)t.size(0);
    s.row_stride = t.stride(0) * size;
    s.outer = 1;
    s.tokens = 1;
    s.token_bytes = size;
    for (size_t i = 0; i < b.n; ++i) s.buffer[i] = b.t[i]->data_ptr();
    if (t.numel() == 0) {
        s.tokens = 0;
        return s;
    }
    if (t.dim() == 1) return s;
    int64_t token = 1;
    if (!packed(t, dim + 1, &token) || (t.size(dim) != 1 && t.stride(dim) != token)) throw Wrong{std::string(what) + ": not contiguous from the tokens' axis on"};
    s.tokens = t.size(dim);
    s.token_bytes = token * size;
    // the axes between the rows and the tokens are one, or steps of one stride
    for (int64_t d = dim - 1; d >= 1; --d) {
        if (t.size(d) == 1) continue;
        if (s.outer > 1 && t.stride(d) * size != s.outer * s.outer_stride) throw Wrong{std::string(what) + ": the axes before the tokens' have no common stride"};
        if (s.outer == 1) s.outer_stride = t.stride(d) * size;
        s.outer *= t.size(d);
    }
    return s;
}

// Pools [pages, ...]; none: `pages` pages that hold nothing.
nereus_pages_t pools_of(const Buffers& b, int64_t pages, const char* what) {
    nereus_pages_t p;
    p.pools = (int32_t)b.n;
    p.page_bytes = p.page_stride = 0;
    if (!b.n) {
        p.pages = (int32_t)std::min<int64_t>(pages, INT32_MAX);
        return p;
    }
    const at::Tensor& t = *b.t[0];
    int64_t page = 1;
    if (!packed(t, 1, &page)) throw Wrong{std::string(what) + ": a page is not contiguous"};
    p.pages = (int32_t)std::min<int64_t>(t.size(0), INT32_MAX);
    p.page_bytes = page * t.element_size();
    p.page_stride = t.stride(0) * t.element_size();
    for (size_t i = 0; i < b.n; ++i) p.pool[i] = b.t[i]->data_ptr();
    return p;
}

// An int32 vector on `device`; size < 0: any.
int32_t* ints_of(PyObject* o, int64_t size, c10::Device device, const char* what) {
    const at::Tensor& t = tensor_of(o, what);
    if (t.scalar_type() != at::kInt || t.device() != device || t.dim() != 1 || (size >= 0 && t.size(0) != size) || !t.is_contiguous())
        throw Wrong{std::string(what) + ": expected a contiguous int32 tensor of shape [" + (size < 0 ? "n" : std::to_string(size)) + "] on the same device"};
    return (int32_t*)t.data_ptr();
}
const at::Tensor& table_of(PyObject* o, nereus_page_table_t* b, const char* what) {
    const at::Tensor& t = tensor_of(o, what);
    if (t.scalar_type() != at::kInt || !t.is_cuda() || t.dim() != 2 || (t.numel() && t.size(1) > 1 && t.stride(1) != 1) || t.size(0) > INT32_MAX || t.size(1) > INT32_MAX)
        throw Wrong{std::string(what) + ": expected int32 [rows, columns], contiguous along the columns, on a CUDA device"};
    b->rows = (int32_t)t.size(0);
    b->columns = (int32_t)t.size(1);
    b->stride = t.size(0) > 1 ? t.stride(0) : t.size(1);
    b->table = (int32_t*)t.data_ptr();
    return t;
}
void* stream_on(c10::Device d) { return (void*)c10::cuda::getCurrentCUDAStream(d.index()).stream(); }
// The pools' and the page table's device are one.
void same_device(const Buffers& b, c10::Device d) {
    if (b.n && b.device != d) throw Wrong{"pools and page table are on different devices"};
}
// Item i of the tuple `out`.
PyObject* item_of(PyObject* out, Py_ssize_t i, Py_ssize_t n) {
    if (!PyTuple_Check(out) || PyTuple_GET_SIZE(out) != n) throw Wrong{"out: expected a tuple of " + std::to_string(n) + " tensors"};
    return PyTuple_GET_ITEM(out, i);
}

// (states, parent, beams, length, dim, out) -> None
PyObject* reorder(PyObject*, PyObject* const* a, Py_ssize_t n) {
    NEREUS_BEGIN
    if (!counted(n, 6)) return nullptr;
    Buffers from, to;
    buffers_of(a[0], "states", &from);
    const bool in_place = a[5] == Py_None;
    if (!in_place) buffers_of(a[5], "out", &to);
    const Buffers& dst = in_place ? from : to;
    const int64_t  dim = int_of(a[4]), beams = a[2] == Py_None ? 0 : int_of(a[2]);
    const nereus_states_t s = states_of(from, dim, "states"), d = states_of(dst, dim, in_place ? "states" : "out");
    if (dst.device != from.device) throw Wrong{"out: on another device than the states"};
    if (dst.t[0]->itemsize() != from.t[0]->itemsize() || dst.n != from.n || dst.t[0]->sizes().slice(1) != from.t[0]->sizes().slice(1))
        throw Wrong{"out: other buffers than the states but for their rows"};
    writable(dst, in_place ? "states" : "out");
    const c10::cuda::OptionalCUDAGuard guard(from.device);
    const int32_t* parent = ints_of(a[1], d.rows, from.device, "parent");
    const int32_t* length = a[3] == Py_None ? nullptr : ints_of(a[3], s.rows, from.device, "length");
    if (failed(nereus_states_reorder(&s, &d, beams < 0 || beams > INT32_MAX ? -1 : (int)beams, parent, length, stream_on(from.device)), "nereus_states_reorder"))
        return nullptr;
    written(dst);
    Py_RETURN_NONE;
    NEREUS_END
}

// (pools, src, dst, to) -> None
PyObject* copy(PyObject*, PyObject* const* a, Py_ssize_t n) {
    NEREUS_BEGIN
    if (!counted(n, 4)) return nullptr;
    Buffers from, to;
    buffers_of(a[0], "pools", &from);
    const bool within = a[3] == Py_None;
    if (!within) buffers_of(a[3], "to", &to);
    const Buffers& dst = within ? from : to;
    if (!from.n || !dst.n) throw Wrong{"pools: expected a pool at least"};
    if (dst.device != from.device) throw Wrong{"to: on another device than the pools"};
    writable(dst, within ? "pools" : "to");
    const c10::cuda::OptionalCUDAGuard guard(from.device);
    const nereus_pages_t p = pools_of(from, 0, "pools"), q = pools_of(dst, 0, "to");
    const int64_t pairs = tensor_of(a[1], "src").numel();
    const int32_t* src = ints_of(a[1], pairs, from.device, "src");
    const int32_t* at = ints_of(a[2], pairs, from.device, "dst");
    if (failed(nereus_cache_copy(&p, &q, pairs, src, at, stream_on(from.device)), "nereus_cache_copy")) return nullptr;
    written(dst);
    Py_RETURN_NONE;
    NEREUS_END
}

// (pools, table, length, refs, parent, page_size, room, out) -> (table, length, refs, copies, status)
PyObject* fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
    NEREUS_BEGIN
    if (!counted(n, 8)) return nullptr;
    Buffers pools;
    buffers_of(a[0], "pools", &pools);
    nereus_page_table_t from = {}, to = {};
    const c10::Device device = table_of(a[1], &from, "table").device();
    same_device(pools, device);
    const c10::cuda::OptionalCUDAGuard guard(device);
    writable(pools, "pools");
    from.length = ints_of(a[2], from.rows, device, "length");
    const nereus_pages_t p = pools_of(pools, tensor_of(a[3], "refs").numel(), "pools");
    from.refs = ints_of(a[3], p.pages, device, "refs");
    const int64_t  rows = tensor_of(a[4], "parent").numel(), page_size = int_of(a[5]);
    const int32_t* parent = ints_of(a[4], rows, device, "parent");
    const int32_t* room_of = nullptr;
    int64_t room = 0;
    if (THPVariable_Check(a[6])) room_of = ints_of(a[6], rows, device, "room");
    else room = int_of(a[6]);
    THPObjectPtr table, length, refs;
    if (a[7] == Py_None) {
        table = THPVariable_Wrap(fresh<int32_t>({rows, from.columns}));
        length = THPVariable_Wrap(fresh<int32_t>({rows}));
        refs = THPVariable_Wrap(fresh<int32_t>({p.pages}));
    } else {
        PyObject* o[3] = {item_of(a[7], 0, 3), item_of(a[7], 1, 3), item_of(a[7], 2, 3)};
        for (PyObject* x : o) Py_INCREF(x);
        table = o[0]; length = o[1]; refs = o[2];
    }
    if (table_of(table.get(), &to, "out").device() != device || to.rows != rows) throw Wrong{"out: the table has a row for each parent, on the same device"};
    to.length = ints_of(length.get(), rows, device, "out");
    to.refs = ints_of(refs.get(), p.pages, device, "out");
    at::Tensor copies = fresh<int32_t>({rows, 2}), status = fresh<int32_t>({4});
    auto narrow = [](int64_t v) { return v < 0 || v > INT32_MAX ? -1 : (int)v; };            // out of range: refused by the library
    if (failed(nereus_cache_fork(&p, &from, &to, parent, narrow(page_size), narrow(room), room_of, (int32_t*)copies.data_ptr(), (int32_t*)status.data_ptr(),
                                 stream_on(device)), "nereus_cache_fork"))
        return nullptr;
    written(pools);
    if (a[7] != Py_None)
        for (PyObject* x : {table.get(), length.get(), refs.get()}) written(x);
    THPObjectPtr c(THPVariable_Wrap(std::move(copies))), s(THPVariable_Wrap(std::move(status)));
    return PyTuple_Pack(5, table.get(), length.get(), refs.get(), c.get(), s.get());
    NEREUS_END
}

// (pools, table, refs, keep, out) -> (table, refs, map, moves, status)
PyObject* compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
    NEREUS_BEGIN
    if (!counted(n, 5)) return nullptr;
    Buffers pools;
    buffers_of(a[0], "pools", &pools);
    nereus_page_table_t from = {}, to = {};
    const c10::Device device = table_of(a[1], &from, "table").device();
    same_device(pools, device);
    const c10::cuda::OptionalCUDAGuard guard(device);
    writable(pools, "pools");
    const nereus_pages_t p = pools_of(pools, tensor_of(a[2], "refs").numel(), "pools");
    from.refs = ints_of(a[2], p.pages, device, "refs");
    int64_t keep = -1;
    if (a[3] != Py_None && (keep = int_of(a[3])) < 0) throw Wrong{"keep: a number of pages, or None"};
    THPObjectPtr table, refs;
    if (a[4] == Py_None) {
        table = THPVariable_Wrap(fresh<int32_t>({from.rows, from.columns}));
        refs = THPVariable_Wrap(fresh<int32_t>({p.pages}));
    } else {
        PyObject* o[2] = {item_of(a[4], 0, 2), item_of(a[4], 1, 2)};
        for (PyObject* x : o) Py_INCREF(x);
        table = o[0]; refs = o[1];
    }
    if (table_of(table.get(), &to, "out").device() != device) throw Wrong{"out: on another device"};
    to.refs = ints_of(refs.get(), p.pages, device, "out");
    at::Tensor map = fresh<int32_t>({p.pages}), moves = fresh<int32_t>({p.pages / 2, 2}), status = fresh<int32_t>({4});
    if (failed(nereus_cache_compact(&p, &from, &to, keep, (int32_t*)map.data_ptr(), (int32_t*)moves.data_ptr(), (int32_t*)status.data_ptr(), stream_on(device)),
               "nereus_cache_compact"))
        return nullptr;
    written(pools);
    if (a[4] != Py_None)
        for (PyObject* x : {table.get(), refs.get()}) written(x);
    THPObjectPtr m(THPVariable_Wrap(std::move(map))), v(THPVariable_Wrap(std::move(moves))), s(THPVariable_Wrap(std::move(status)));
    return PyTuple_Pack(5, table.get(), refs.get(), m.get(), v.get(), s.get());
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
                           NEREUS_FAST(distill_backward), NEREUS_FAST(distill_step),
                           NEREUS_FAST(beam_select),     NEREUS_FAST(reorder),     NEREUS_FAST(fork),
                           NEREUS_FAST(compact),         NEREUS_FAST(copy),        {"empty_like", empty_like_of, METH_O, nullptr},
                           {"set_error", set_error, METH_O, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_nereus_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__nereus_torch(void) { return PyModule_Create(&g_module); }
