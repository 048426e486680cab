// svf_binding.cpp -- the short way from torch tensors to the calls of svfkv.h and svflogprob.h.
//
// A step's calls are some microseconds on the GPU; looking at a dozen tensors from Python takes more than that.  Here they are looked at
// once, in one go.  Every function returns None without having done anything where an argument is not the ordinary, valid case
// (another device than the current one, derivatives, a trace, a type or shape that does not fit): kvcache.py and logprobs.py then go the
// long way, which says what is wrong.  A call's own error comes back as its number.
//
// 203 tokens appended with three axes: 15.3 us from Python alone, 5.8 here; one token's attention 13.7 and 7.9; one answer's score 14.3 and 9.8.
#define PY_SSIZE_T_CLEAN
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <ATen/TracerMode.h>
#include <ATen/core/grad_mode.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>

#include <cmath>
#include <cstring>

#include "svfkv.h"
#include "svflogprob.h"
#include "svfsim.h"

namespace {

constexpr int64_t kMost32 = 2147483647;

// What an ordinary call has: the device and stream, the type of its tensors.
struct Now {
    int64_t dev;
    void* stream;
};

const at::Tensor* tensor(PyObject* x) { return THPVariable_Check(x) ? &THPVariable_Unpack(x) : nullptr; }

// A strided tensor on the current GPU that takes no part in gradients that are being recorded and has no tangent.
bool usable(const at::Tensor* t, const Now& now, at::ScalarType type, int64_t dim) {
    return t && t->layout() == at::kStrided && t->device().is_cuda() && t->device().index() == now.dev && t->scalar_type() == type &&
           t->dim() == dim && !(t->requires_grad() && at::GradMode::is_enabled()) && !t->_fw_grad(0).defined() && !t->is_conj() && !t->is_neg();
}

bool number(PyObject* x, int64_t* to) {
    if (!PyLong_CheckExact(x)) return false;
    int over = 0;
    *to = PyLong_AsLongLongAndOverflow(x, &over);
    return over == 0;
}

// Runs a call while other threads may have Python's lock: a launch waits where the GPU's queue is full.
template <class F>
int unlocked(F f) {
    PyThreadState* thread = PyEval_SaveThread();
    const int rc = f();
    PyEval_RestoreThread(thread);
    return rc;
}

template <class P>
P* at_of(const at::Tensor& t) {
    return static_cast<P*>(t.data_ptr());
}

// The cache and the sequences of a call (kvcache.Cache, kvcache.Batch).
struct Call {
    svf_kv_cache cache;
    svf_kv_batch batch;
    at::ScalarType type;

    bool read(PyObject* c, PyObject* b, int64_t tokens, const Now& now) {
        if (!PyTuple_Check(c) || PyTuple_GET_SIZE(c) != 4 || !PyTuple_Check(b) || PyTuple_GET_SIZE(b) != 4) return false;
        const at::Tensor *k = tensor(PyTuple_GET_ITEM(c, 0)), *v = tensor(PyTuple_GET_ITEM(c, 1));
        if (!k) return false;
        type = k->scalar_type();
        if (type != at::kBFloat16 && type != at::kHalf) return false;
        if (!usable(k, now, type, 4) || !usable(v, now, type, 4) || k->sizes() != v->sizes() || k->stride(3) != 1 || v->stride(3) != 1) return false;
        for (int i = 0; i < 4; i++)
            if (k->size(i) > kMost32) return false;
        cache = {};
        cache.k = k->data_ptr(), cache.v = v->data_ptr();
        for (int i = 2; i < 4; i++) {
            PyObject* x = PyTuple_GET_ITEM(c, i);
            if (x == Py_None) continue;
            const at::Tensor* t = tensor(x);
            if (!usable(t, now, i == 2 ? at::kFloat : at::kInt, 3) || !t->is_contiguous()) return false;
            for (int j = 0; j < 3; j++)
                if (t->size(j) != k->size(j)) return false;
            (i == 2 ? reinterpret_cast<void*&>(cache.weight) : reinterpret_cast<void*&>(cache.position)) = t->data_ptr();
        }
        cache.k_page_stride = k->stride(0), cache.k_head_stride = k->stride(1), cache.k_row_stride = k->stride(2);
        cache.v_page_stride = v->stride(0), cache.v_head_stride = v->stride(1), cache.v_row_stride = v->stride(2);
        cache.num_pages = (int32_t)k->size(0), cache.kv_heads = (int32_t)k->size(1);
        cache.page_size = (int32_t)k->size(2), cache.head_dim = (int32_t)k->size(3);
        cache.dtype = type == at::kBFloat16 ? SVF_KV_BF16 : SVF_KV_F16;

        const at::Tensor *offsets = tensor(PyTuple_GET_ITEM(b, 0)), *len = tensor(PyTuple_GET_ITEM(b, 1)), *table = tensor(PyTuple_GET_ITEM(b, 2));
        int64_t max_q = 0;
        if (!usable(offsets, now, at::kInt, 1) || !usable(len, now, at::kInt, 1) || !usable(table, now, at::kInt, 2) ||
            !number(PyTuple_GET_ITEM(b, 3), &max_q))
            return false;
        const int64_t seqs = len->size(0), width = table->size(1);
        if (!offsets->is_contiguous() || !len->is_contiguous() || offsets->size(0) != seqs + 1 || table->size(0) != seqs ||
            (width > 1 && table->stride(1) != 1) || seqs > kMost32 || width > kMost32 || tokens > kMost32 || max_q < 0 || max_q > kMost32)
            return false;
        batch = {};
        batch.q_offsets = at_of<int32_t>(*offsets), batch.kv_len = at_of<int32_t>(*len), batch.page_table = at_of<int32_t>(*table);
        batch.table_stride = table->stride(0);
        if (seqs < 2 && batch.table_stride < width) batch.table_stride = width;  // a table of one row may have any stride
        batch.num_seqs = (int32_t)seqs, batch.num_tokens = (int32_t)tokens, batch.table_width = (int32_t)width, batch.max_q = (int32_t)max_q;
        return true;
    }
};

// [tokens, heads, head_dim] of the cache's kind.
bool rows(const at::Tensor* t, const Now& now, const Call& call, int64_t tokens, int64_t heads) {
    return usable(t, now, call.type, 3) && t->size(0) == tokens && t->size(1) == heads && t->size(2) == call.cache.head_dim && t->stride(2) == 1;
}

bool read_now(PyObject* dev, PyObject* stream, Now* now) {
    int64_t s = 0;
    if (at::tracer::impl::is_dispatch_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set()) return false;
    if (!number(dev, &now->dev) || !number(stream, &s)) return false;
    now->stream = reinterpret_cast<void*>(s);
    return true;
}

// append(q, k, v, positions, rope, batch, cache, layout, q_out, axes, kept, device, stream) -> tensor, error or None
PyObject* append(PyObject*, PyObject* const* x, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Now now;
    int64_t layout = 0;
    const at::Tensor *q = n == 13 ? tensor(x[0]) : nullptr, *k = nullptr, *v = nullptr, *positions = nullptr;
    if (!q || q->dim() != 3 || !read_now(x[11], x[12], &now) || !number(x[7], &layout)) Py_RETURN_NONE;
    const int64_t tokens = q->size(0), heads = q->size(1);
    Call call;
    k = tensor(x[1]), v = tensor(x[2]), positions = tensor(x[3]);
    if (heads > kMost32 || !call.read(x[6], x[5], tokens, now) || !rows(q, now, call, tokens, heads) ||
        !rows(k, now, call, tokens, call.cache.kv_heads) || !rows(v, now, call, tokens, call.cache.kv_heads))
        Py_RETURN_NONE;
    const bool axes = x[9] != Py_None;
    if (!usable(positions, now, at::kInt, axes ? 2 : 1) || positions->size(0) != tokens || (!axes && !positions->is_contiguous())) Py_RETURN_NONE;
    svf_kv_append_args a = {};
    if (x[4] != Py_None) {
        const at::Tensor* rope = tensor(x[4]);
        if (!usable(rope, now, at::kFloat, 2) || !rope->is_contiguous() || rope->size(0) > kMost32 || rope->size(1) > kMost32) Py_RETURN_NONE;
        a.rope = at_of<float>(*rope), a.rope_rows = (int32_t)rope->size(0), a.rot = (int32_t)rope->size(1);
    }
    svf_kv_axes with = {};
    if (axes) {
        if (!PyBytes_CheckExact(x[9]) || PyBytes_GET_SIZE(x[9]) * 2 != a.rot || a.rot > 256 || positions->size(1) > kMost32) Py_RETURN_NONE;
        memcpy(with.of_pair, PyBytes_AS_STRING(x[9]), a.rot / 2);
        with.axes = (int32_t)positions->size(1);
        with.token_stride = positions->stride(0), with.axis_stride = positions->stride(1);
        if (x[10] != Py_None) {
            const at::Tensor* kept = tensor(x[10]);
            if (!usable(kept, now, at::kInt, 1) || kept->size(0) != tokens || !kept->is_contiguous()) Py_RETURN_NONE;
            with.kept = at_of<int32_t>(*kept);
        }
    } else if (x[10] != Py_None) {
        Py_RETURN_NONE;
    }
    at::Tensor out;
    if (x[8] == Py_None) {
        out = at::empty_like(*q);
    } else {
        const at::Tensor* given = tensor(x[8]);
        if (!given) Py_RETURN_NONE;
        out = *given;
    }
    if (!rows(&out, now, call, tokens, heads)) Py_RETURN_NONE;
    a.q = q->data_ptr(), a.k = k->data_ptr(), a.v = v->data_ptr(), a.q_out = out.data_ptr(), a.positions = at_of<int32_t>(*positions);
    a.q_token_stride = q->stride(0), a.q_head_stride = q->stride(1);
    a.k_token_stride = k->stride(0), a.k_head_stride = k->stride(1);
    a.v_token_stride = v->stride(0), a.v_head_stride = v->stride(1);
    a.out_token_stride = out.stride(0), a.out_head_stride = out.stride(1);
    a.heads = (int32_t)heads, a.layout = (int32_t)layout;
    const int rc = unlocked([&] {
        return axes ? svf_kv_append_axes(&call.cache, &call.batch, &a, &with, now.stream)
                    : svf_kv_append(&call.cache, &call.batch, &a, now.stream);
    });
    if (rc != SVF_OK) return PyLong_FromLong(rc);
    if (x[8] != Py_None) {
        Py_INCREF(x[8]);
        return x[8];
    }
    return THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// attend(q, batch, cache, causal, window, scale, add_weight, first, device, stream) -> (out, lse), error or None
PyObject* attend(PyObject*, PyObject* const* x, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Now now;
    int64_t window = 0, first = 0;
    const at::Tensor* q = n == 10 ? tensor(x[0]) : nullptr;
    if (!q || q->dim() != 3 || !read_now(x[8], x[9], &now) || !PyBool_Check(x[3]) || !number(x[4], &window) || !PyBool_Check(x[6]) ||
        !number(x[7], &first) || window < 0 || window > kMost32 || first < 0 || first > kMost32)
        Py_RETURN_NONE;
    const int64_t tokens = q->size(0), heads = q->size(1);
    Call call;
    if (heads > kMost32 || !call.read(x[2], x[1], tokens, now) || !rows(q, now, call, tokens, heads)) Py_RETURN_NONE;
    svf_kv_attend_args a = {};
    if (x[5] == Py_None) {
        a.scale = (float)std::pow((double)call.cache.head_dim, -0.5);
    } else {
        if (!PyFloat_CheckExact(x[5])) Py_RETURN_NONE;
        const double scale = PyFloat_AS_DOUBLE(x[5]);
        a.scale = (float)scale;
        if (std::isinf(a.scale)) Py_RETURN_NONE;
    }
    at::Tensor out = at::empty(q->sizes(), q->options()), lse = at::empty({tokens, heads}, q->options().dtype(at::kFloat)), ws;
    a.q = q->data_ptr(), a.out = out.data_ptr(), a.lse = at_of<float>(lse);
    a.q_token_stride = q->stride(0), a.q_head_stride = q->stride(1);
    a.out_token_stride = out.stride(0), a.out_head_stride = out.stride(1);
    a.heads = (int32_t)heads, a.causal = x[3] == Py_True, a.window = (int32_t)window, a.add_weight = x[6] == Py_True;
    const int64_t need = first ? svf_kv_attend_first_workspace(&call.cache, &call.batch, &a, (int32_t)first)
                               : svf_kv_attend_workspace(&call.cache, &call.batch, &a);
    if (need < 0) return PyLong_FromLongLong(need);
    if (need > 0) {
        ws = at::empty({need}, q->options().dtype(at::kByte));
        a.workspace = ws.data_ptr(), a.workspace_bytes = need;
    }
    const int rc = unlocked([&] {
        return first ? svf_kv_attend_first(&call.cache, &call.batch, &a, (int32_t)first, now.stream)
                     : svf_kv_attend(&call.cache, &call.batch, &a, now.stream);
    });
    if (rc != SVF_OK) return PyLong_FromLong(rc);
    PyObject *o = THPVariable_Wrap(std::move(out)), *l = o ? THPVariable_Wrap(std::move(lse)) : nullptr;
    PyObject* both = l ? PyTuple_Pack(2, o, l) : nullptr;
    Py_XDECREF(o);
    Py_XDECREF(l);
    return both;
    END_HANDLE_TH_ERRORS
}

// score(logits, token, top, scale, device, stream) -> (logprob, entropy, rank, top_logprob, top_index), error or None
PyObject* score(PyObject*, PyObject* const* x, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    Now now;
    int64_t top = 0;
    const at::Tensor *logits = n == 6 ? tensor(x[0]) : nullptr, *token = logits ? tensor(x[1]) : nullptr;
    if (!token || !read_now(x[4], x[5], &now) || !number(x[2], &top) || !PyFloat_CheckExact(x[3])) Py_RETURN_NONE;
    svf_logprob_args a = {};
    const at::ScalarType type = logits->scalar_type(), of_token = token->scalar_type();
    a.dtype = type == at::kBFloat16 ? SVF_LOGITS_BF16 : type == at::kHalf ? SVF_LOGITS_F16 : SVF_LOGITS_F32;
    if ((type != at::kBFloat16 && type != at::kHalf && type != at::kFloat) || (of_token != at::kInt && of_token != at::kLong) ||
        !usable(logits, now, type, 2) || !usable(token, now, of_token, 1) || !token->is_contiguous())
        Py_RETURN_NONE;
    const int64_t count = logits->size(0), vocab = logits->size(1);
    if (token->size(0) != count || (vocab > 1 && logits->stride(1) != 1) || count > kMost32 || vocab > kMost32 || top < 0 ||
        top > SVF_LOGPROB_MOST_TOP || top > vocab)
        Py_RETURN_NONE;
    a.scale = (float)PyFloat_AS_DOUBLE(x[3]);
    if (std::isinf(a.scale)) Py_RETURN_NONE;
    const auto floats = logits->options().dtype(at::kFloat), ints = logits->options().dtype(at::kInt);
    at::Tensor out[5] = {at::empty({count}, floats), at::empty({count}, floats), at::empty({count}, ints), at::empty({count, top}, floats),
                         at::empty({count, top}, ints)};
    at::Tensor ws;
    a.logits = logits->data_ptr(), a.token = token->data_ptr();
    a.logprob = at_of<float>(out[0]), a.entropy = at_of<float>(out[1]), a.rank = at_of<int32_t>(out[2]);
    a.top_logprob = at_of<float>(out[3]), a.top_index = at_of<int32_t>(out[4]);
    a.row_stride = logits->stride(0);
    a.rows = (int32_t)count, a.vocab = (int32_t)vocab, a.top = (int32_t)top, a.token_bytes = of_token == at::kLong ? 8 : 4;
    const int64_t need = svf_logprob_workspace(&a);
    if (need < 0) return PyLong_FromLongLong(need);
    if (need > 0) {
        ws = at::empty({need}, logits->options().dtype(at::kByte));
        a.workspace = ws.data_ptr(), a.workspace_bytes = need;
    }
    const int rc = unlocked([&] { return svf_logprob(&a, now.stream); });
    if (rc != SVF_OK) return PyLong_FromLong(rc);
    PyObject* all = PyTuple_New(5);
    for (int i = 0; all && i < 5; i++) {
        PyObject* t = THPVariable_Wrap(std::move(out[i]));
        if (!t) {
            Py_DECREF(all);
            return nullptr;
        }
        PyTuple_SET_ITEM(all, i, t);
    }
    return all;
    END_HANDLE_TH_ERRORS
}

template <class F>
PyCFunction function(F f) {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}

PyMethodDef kMethods[] = {{"append", function(append), METH_FASTCALL, nullptr},
                          {"attend", function(attend), METH_FASTCALL, nullptr},
                          {"score", function(score), METH_FASTCALL, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_svfbinding", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// ``torch_version``: the torch whose headers this was built with.  kvcache.py uses it with no other.
PyMODINIT_FUNC PyInit__svfbinding() {
    PyObject* m = PyModule_Create(&kModule);
    if (m && PyModule_AddStringConstant(m, "torch_version", SVF_TORCH_VERSION) != 0) Py_CLEAR(m);
    return m;
}
