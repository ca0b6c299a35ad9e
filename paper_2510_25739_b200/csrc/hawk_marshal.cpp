// Python marshalling of the calls around the paged cache (hawk_qk_norm_rope, hawk_rope_append, hawk_paged_attn, hawk_pages_*) and of
// hawk_sample.
//
// These calls run once or twice a layer, or several a step, on tensors of a few kilobytes, where the kernel takes 3 us and looking at a dozen tensors
// from Python takes 7.  So the tensors are checked and turned into the C ABI's argument structs here, in under 1 us; nothing
// is computed.  Entry points are reached by the address that the caller passes (of the library build it has loaded).
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <optional>
#include <string>

#include "../../include/hawk.h"

namespace {

struct Refused {};  // a Python error is set

[[noreturn]] void refuse(PyObject *type, const std::string &text)
{
    PyErr_SetString(type, text.c_str());
    throw Refused{};
}

std::string name_of(at::ScalarType t)
{
    switch (t) {
        case at::kBFloat16: return "torch.bfloat16";
        case at::kHalf: return "torch.float16";
        case at::kFloat: return "torch.float32";
        case at::kDouble: return "torch.float64";
        case at::kInt: return "torch.int32";
        case at::kLong: return "torch.int64";
        default: return std::string("torch ") + c10::toString(t);
    }
}

std::string text_of(at::IntArrayRef s)
{
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + (s.size() == 1 ? ",)" : ")");
}

// A tensor argument; NULL for None where that is allowed.
const at::Tensor *tensor(PyObject *o, const char *name, bool needed = true)
{
    if (o == Py_None) {
        if (needed) refuse(PyExc_TypeError, std::string(name) + ": a tensor is needed");
        return nullptr;
    }
    if (!THPVariable_Check(o)) refuse(PyExc_TypeError, std::string(name) + ": expected a torch.Tensor");
    return &THPVariable_Unpack(o);
}

struct Where {
    at::ScalarType dtype;
    int index;  // GPU
};

// The tensor that decides type and GPU of a call.
Where where(const at::Tensor &t, const char *name)
{
    if (!t.is_cuda()) refuse(PyExc_ValueError, std::string(name) + ": must be a CUDA tensor");
    const at::ScalarType d = t.scalar_type();
    if (d != at::kBFloat16 && d != at::kHalf)
        refuse(PyExc_TypeError, std::string(name) + ": expected torch.bfloat16 or torch.float16, got " + name_of(d));
    return {d, t.get_device()};
}

void check(const at::Tensor &t, const char *name, at::ScalarType dtype, at::IntArrayRef shape, int index)
{
    if (t.scalar_type() != dtype)
        refuse(PyExc_TypeError, std::string(name) + ": expected " + name_of(dtype) + ", got " + name_of(t.scalar_type()));
    if (t.sizes() != shape)
        refuse(PyExc_ValueError, std::string(name) + ": expected shape " + text_of(shape) + ", got " + text_of(t.sizes()));
    if (!t.is_cuda() || t.get_device() != index)
        refuse(PyExc_ValueError, std::string(name) + ": must be on cuda:" + std::to_string(index) + ", is on " + t.device().str());
}

// Contiguous tensor, NULL for none.
const void *dense(const at::Tensor *t, const char *name, at::ScalarType dtype, at::IntArrayRef shape, int index)
{
    if (!t) return nullptr;
    check(*t, name, dtype, shape, index);
    if (!t->is_contiguous()) refuse(PyExc_ValueError, std::string(name) + ": must be contiguous");
    return t->data_ptr();
}

// [.., D] with a contiguous last dimension (a dimension of one element may have any stride).
void *strided(const at::Tensor &t, const char *name, at::ScalarType dtype, at::IntArrayRef shape, int index)
{
    check(t, name, dtype, shape, index);
    if (t.stride(-1) != 1) refuse(PyExc_ValueError, std::string(name) + ": the head dimension must be contiguous");
    return t.data_ptr();
}

void dims(const at::Tensor &t, const char *name, int64_t n)
{
    if (t.dim() != n)
        refuse(PyExc_ValueError, std::string(name) + ": expected " + std::to_string(n) + " dimensions, got " + text_of(t.sizes()));
}

int as_int(int64_t v, const char *name)
{
    if (v < INT32_MIN || v > INT32_MAX) refuse(PyExc_ValueError, std::string(name) + ": out of range");
    return static_cast<int>(v);
}

int integer(PyObject *o, const char *name)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{};
    return as_int(v, name);
}

float number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused{};
    return static_cast<float>(v);
}

bool truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Refused{};
    return v != 0;
}

void *address(PyObject *o)
{
    void *p = PyLong_AsVoidPtr(o);
    if (!p) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "entry point: NULL");
        throw Refused{};
    }
    return p;
}

int norm_kind(PyObject *o)
{
    if (PyUnicode_Check(o)) {
        if (PyUnicode_CompareWithASCIIString(o, "none") == 0) return HAWK_NORM_NONE;
        if (PyUnicode_CompareWithASCIIString(o, "rms") == 0) return HAWK_NORM_RMS;
        if (PyUnicode_CompareWithASCIIString(o, "layer") == 0) return HAWK_NORM_LAYER;
    }
    refuse(PyExc_ValueError, "norm: expected one of 'none', 'rms', 'layer'");
}

int32_t *status_word(PyObject *o, int index)
{
    return static_cast<int32_t *>(const_cast<void *>(dense(tensor(o, "dev_status", false), "dev_status", at::kInt, {1}, index)));
}

// Runs `call(stream)` with GPU `index` current, on its current stream.
template <class F>
long run_on(int index, F &&call)
{
    std::optional<c10::cuda::CUDAGuard> guard;
    if (c10::cuda::current_device() != index) guard.emplace(static_cast<c10::DeviceIndex>(index));
    return static_cast<long>(call(reinterpret_cast<hawk_stream_t>(c10::cuda::getCurrentCUDAStream(index).stream())));
}

PyObject *owned(PyObject *given, const at::Tensor *made)
{
    if (made) return THPVariable_Wrap(*made);
    Py_INCREF(given);
    return given;
}

// Arguments that hawk_qk_norm_rope and hawk_rope_append share, in this order from args[0] on: q, k, position, cos_sin; norm,
// eps, q_weight, k_weight, q_bias, k_bias, interleaved from opts[0] on.
struct Rope {
    hawk_qk_rope_args a = {};
    Where w;
    const at::Tensor *q, *k;
    std::optional<at::Tensor> q_made, k_made;

    Rope(PyObject *const *args, PyObject *const *opts, PyObject *q_out, PyObject *k_out)
    {
        q = tensor(args[0], "q", false);
        k = tensor(args[1], "k", false);
        if (!q && !k) refuse(PyExc_ValueError, "q, k: one of them is needed");
        const at::Tensor &x = q ? *q : *k;
        w = where(x, q ? "q" : "k");
        dims(x, q ? "q" : "k", 3);
        const int64_t T = x.size(0), D = x.size(2);
        a.dtype = w.dtype == at::kBFloat16 ? HAWK_BF16 : HAWK_F16;
        a.T = as_int(T, "rows");
        a.D = as_int(D, "head dimension");
        a.norm = norm_kind(opts[0]);
        a.eps = number(opts[1]);
        a.interleaved = truth(opts[6]);
        if (q) {
            a.H = as_int(q->size(1), "heads");
            a.q = strided(*q, "q", w.dtype, q->sizes(), w.index);
            a.q_row_stride = q->stride(0);
            a.q_head_stride = q->stride(1);
            const at::Tensor *o = tensor(q_out, "q_out", false);
            if (!o) o = &q_made.emplace(at::empty(q->sizes(), q->options()));
            a.q_out = strided(*o, "q_out", w.dtype, q->sizes(), w.index);
            a.q_out_row_stride = o->stride(0);
            a.q_out_head_stride = o->stride(1);
        }
        if (k) {
            dims(*k, "k", 3);
            const int64_t shape[3] = {T, k->size(1), D};
            a.H_kv = as_int(k->size(1), "heads");
            a.k = strided(*k, "k", w.dtype, shape, w.index);
            a.k_row_stride = k->stride(0);
            a.k_head_stride = k->stride(1);
            if (k_out) {
                const at::Tensor *o = tensor(k_out, "k_out", false);
                if (!o) o = &k_made.emplace(at::empty(shape, k->options()));
                a.k_out = strided(*o, "k_out", w.dtype, shape, w.index);
                a.k_out_row_stride = o->stride(0);
                a.k_out_head_stride = o->stride(1);
            }
        }
        if (a.norm != HAWK_NORM_NONE) {
            const at::Tensor *wq = tensor(opts[2], "q_weight", false), *wk = tensor(opts[3], "k_weight", false);
            const at::Tensor *first = wq ? wq : wk;
            a.per_head = first && first->dim() == 2;
            const int64_t qs[2] = {a.H, D}, ks[2] = {a.H_kv, D};
            const at::IntArrayRef q_shape = a.per_head ? at::IntArrayRef(qs, 2) : at::IntArrayRef(qs + 1, 1);
            const at::IntArrayRef k_shape = a.per_head ? at::IntArrayRef(ks, 2) : at::IntArrayRef(ks + 1, 1);
            a.q_weight = dense(wq, "q_weight", w.dtype, q_shape, w.index);
            a.k_weight = dense(wk, "k_weight", w.dtype, k_shape, w.index);
            a.q_bias = dense(tensor(opts[4], "q_bias", false), "q_bias", w.dtype, q_shape, w.index);
            a.k_bias = dense(tensor(opts[5], "k_bias", false), "k_bias", w.dtype, k_shape, w.index);
            if (a.norm == HAWK_NORM_RMS && (a.q_bias || a.k_bias))
                refuse(PyExc_ValueError, std::string(a.q_bias ? "q_bias" : "k_bias") + ": goes with norm 'layer', not with 'rms'");
        }
        if (const at::Tensor *cs = tensor(args[3], "cos_sin", false)) {
            dims(*cs, "cos_sin", 2);
            a.n_positions = as_int(cs->size(0), "positions");
            a.rot_dim = as_int(cs->size(1), "rotated dimension");
            a.cos_sin = static_cast<const float *>(dense(cs, "cos_sin", at::kFloat, cs->sizes(), w.index));
            a.position = static_cast<const int32_t *>(dense(tensor(args[2], "position"), "position", at::kInt, {T}, w.index));
        }
    }
};

// Pointers, strides and sizes of the page tensors and of the batch's index tensors.
template <class Args>
void pages_and_batch(Args &a, const Where &w, PyObject *k_pages, PyObject *v_pages, PyObject *block_table, PyObject *row_begin,
                     PyObject *kv_len, int64_t H_kv, int64_t D)
{
    const at::Tensor &kp = *tensor(k_pages, "k_pages"), &vp = *tensor(v_pages, "v_pages");
    dims(kp, "k_pages", 4);
    const int64_t shape[4] = {kp.size(0), H_kv, kp.size(2), D};
    a.n_pages = as_int(shape[0], "pages");
    a.page_size = as_int(shape[2], "page size");
    a.k_pages = strided(kp, "k_pages", w.dtype, shape, w.index);
    a.v_pages = strided(vp, "v_pages", w.dtype, shape, w.index);
    a.k_page_stride = kp.stride(0);
    a.k_page_head_stride = kp.stride(1);
    a.k_page_row_stride = kp.stride(2);
    a.v_page_stride = vp.stride(0);
    a.v_page_head_stride = vp.stride(1);
    a.v_page_row_stride = vp.stride(2);
    const at::Tensor &bt = *tensor(block_table, "block_table");
    dims(bt, "block_table", 2);
    a.S = as_int(bt.size(0), "streams");
    a.table_width = as_int(bt.size(1), "table width");
    a.block_table = static_cast<const int32_t *>(dense(&bt, "block_table", at::kInt, bt.sizes(), w.index));
    const int64_t S = a.S;
    a.row_begin = static_cast<const int32_t *>(dense(tensor(row_begin, "row_begin"), "row_begin", at::kInt, {S + 1}, w.index));
    a.kv_len = static_cast<const int32_t *>(dense(tensor(kv_len, "kv_len"), "kv_len", at::kInt, {S}, w.index));
}

// A C++ or Python error inside becomes the Python error that torch has for it (torch.OutOfMemoryError of an allocation among
// them); nothing leaves through the C boundary.
template <class F>
PyObject *guarded(F &&f)
{
    try {
        return f();
    } catch (const Refused &) {
    } catch (...) {
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

void expect(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want) refuse(PyExc_TypeError, "expected " + std::to_string(want) + " arguments, got " + std::to_string(n));
}

// (entry point, q, k, position, cos_sin, norm, eps, q_weight, k_weight, q_bias, k_bias, interleaved, q_out, k_out, dev_status)
// -> (status, q_out, k_out)
PyObject *qk_norm_rope(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        expect(n, 15);
        const auto fn = reinterpret_cast<decltype(&hawk_qk_norm_rope)>(address(args[0]));
        const Rope r(args + 1, args + 5, args[12], args[13]);
        int32_t *status = status_word(args[14], r.w.index);
        const long rc = run_on(r.w.index, [&](hawk_stream_t st) { return fn(&r.a, status, st); });
        return Py_BuildValue("lNN", rc, owned(r.q ? args[12] : Py_None, r.q_made ? &*r.q_made : nullptr),
                             owned(r.k ? args[13] : Py_None, r.k_made ? &*r.k_made : nullptr));
    });
}

// (entry point, q, k, position, cos_sin, v, k_pages, v_pages, block_table, row_begin, kv_len, norm, eps, q_weight, k_weight,
// q_bias, k_bias, interleaved, q_out, dev_status) -> (status, q_out)
PyObject *rope_append(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        expect(n, 20);
        const auto fn = reinterpret_cast<decltype(&hawk_rope_append)>(address(args[0]));
        tensor(args[2], "k");
        const Rope r(args + 1, args + 11, args[18], nullptr);
        hawk_rope_append_args a = {};
        a.qk = r.a;
        const at::Tensor &v = *tensor(args[5], "v");
        a.v = strided(v, "v", r.w.dtype, r.k->sizes(), r.w.index);
        a.v_row_stride = v.stride(0);
        a.v_head_stride = v.stride(1);
        pages_and_batch(a, r.w, args[6], args[7], args[8], args[9], args[10], r.a.H_kv, r.a.D);
        int32_t *status = status_word(args[19], r.w.index);
        const long rc = run_on(r.w.index, [&](hawk_stream_t st) { return fn(&a, status, st); });
        return Py_BuildValue("lN", rc, owned(r.q ? args[18] : Py_None, r.q_made ? &*r.q_made : nullptr));
    });
}

// (entry point, workspace query, q, k_pages, v_pages, block_table, row_begin, kv_len, max_new, max_kv, sm_scale, anc_mask, out,
// workspace, dev_status) -> (status, out)
PyObject *paged_attn(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        expect(n, 15);
        const auto fn = reinterpret_cast<decltype(&hawk_paged_attn)>(address(args[0]));
        const auto need_of = reinterpret_cast<decltype(&hawk_paged_attn_workspace_bytes)>(address(args[1]));
        const at::Tensor &q = *tensor(args[2], "q");
        const Where w = where(q, "q");
        dims(q, "q", 3);
        const at::Tensor &kp = *tensor(args[3], "k_pages");
        dims(kp, "k_pages", 4);
        const int64_t T = q.size(0), H = q.size(1), D = q.size(2), H_kv = kp.size(1);
        hawk_paged_attn_args a = {};
        a.dtype = w.dtype == at::kBFloat16 ? HAWK_BF16 : HAWK_F16;
        a.T = as_int(T, "rows");
        a.H = as_int(H, "heads");
        a.H_kv = as_int(H_kv, "heads");
        a.D = as_int(D, "head dimension");
        a.q = strided(q, "q", w.dtype, q.sizes(), w.index);
        a.q_row_stride = q.stride(0);
        a.q_head_stride = q.stride(1);
        pages_and_batch(a, w, args[3], args[4], args[5], args[6], args[7], H_kv, D);
        a.max_new = integer(args[8], "max_new");
        a.max_kv = integer(args[9], "max_kv");
        a.sm_scale = number(args[10]);
        a.anc_mask = static_cast<const uint64_t *>(
            dense(tensor(args[11], "anc_mask", false), "anc_mask", at::kLong, {a.max_new}, w.index));
        std::optional<at::Tensor> out_made, ws_made;
        const at::Tensor *out = tensor(args[12], "out", false);
        if (!out) out = &out_made.emplace(at::empty({T, H * D}, q.options()));
        a.out = const_cast<void *>(dense(out, "out", w.dtype, {T, H * D}, w.index));
        if (const at::Tensor *ws = tensor(args[13], "workspace", false)) {
            a.workspace = const_cast<void *>(dense(ws, "workspace", ws->scalar_type(), ws->sizes(), w.index));
            a.workspace_bytes = static_cast<size_t>(ws->numel()) * ws->element_size();
        } else if (const size_t need = need_of(a.S, a.T, a.max_new, a.H, a.H_kv, a.D, a.max_kv)) {
            a.workspace = ws_made.emplace(at::empty({static_cast<int64_t>(need)}, q.options().dtype(at::kByte))).data_ptr();
            a.workspace_bytes = need;
        }
        int32_t *status = status_word(args[14], w.index);
        const long rc = run_on(w.index, [&](hawk_stream_t st) { return fn(&a, status, st); });
        return Py_BuildValue("lN", rc, owned(args[12], out_made ? &*out_made : nullptr));
    });
}

// ---------------------------------------------------------------------------------------------- sampling
// A setting of the rows: a number for all, or a tensor with one for each.
template <typename N, class Read>
const N *setting(PyObject *o, const char *name, at::ScalarType dtype, int64_t rows, int index, N &all, Read &&read)
{
    if (THPVariable_Check(o)) return static_cast<const N *>(dense(&THPVariable_Unpack(o), name, dtype, {rows}, index));
    all = read(o);
    return nullptr;
}

// Rows of a matrix: last dimension contiguous, any row stride.
void *rows_of(const at::Tensor &t, const char *name, at::ScalarType dtype, at::IntArrayRef shape, int index, long long &stride)
{
    check(t, name, dtype, shape, index);
    if (t.size(1) > 1 && t.stride(1) != 1) refuse(PyExc_ValueError, std::string(name) + ": the last dimension must be contiguous");
    stride = t.size(0) > 1 ? t.stride(0) : t.size(1);
    return t.data_ptr();
}

// (entry point, logits, u, temperature, top_k, top_p, min_p, cfg_scale, v_begin, v_end, token, token_prob, probs, dev_status) ->
// (status, token)
PyObject *sample(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        expect(n, 14);
        const auto fn = reinterpret_cast<decltype(&hawk_sample)>(address(args[0]));
        const at::Tensor &x = *tensor(args[1], "logits");
        if (!x.is_cuda()) refuse(PyExc_ValueError, "logits: must be a CUDA tensor");
        dims(x, "logits", 2);
        const int index = x.get_device();
        const at::ScalarType dtype = x.scalar_type();
        if (dtype != at::kFloat && dtype != at::kBFloat16 && dtype != at::kHalf)
            refuse(PyExc_TypeError, "logits: expected torch.float32, torch.bfloat16 or torch.float16, got " + name_of(dtype));
        const bool guided = args[7] != Py_None;
        if (guided && x.size(0) % 2) refuse(PyExc_ValueError, "logits: with cfg_scale, the conditional rows come first, then as many unconditional");
        const int64_t R = guided ? x.size(0) / 2 : x.size(0), V = x.size(1);
        hawk_sample_args a = {};
        a.dtype = dtype == at::kFloat ? HAWK_F32 : dtype == at::kBFloat16 ? HAWK_BF16 : HAWK_F16;
        a.R = as_int(R, "rows");
        a.V = as_int(V, "ids");
        a.logits = rows_of(x, "logits", dtype, x.sizes(), index, a.row_stride);
        if (guided) {
            a.uncond = static_cast<const char *>(a.logits) + R * a.row_stride * static_cast<int64_t>(x.element_size());
            a.uncond_row_stride = a.row_stride;
        }
        a.row_temperature = setting(args[3], "temperature", at::kFloat, R, index, a.temperature, number);
        a.row_top_k = setting(args[4], "top_k", at::kInt, R, index, a.top_k, [](PyObject *o) { return integer(o, "top_k"); });
        a.row_top_p = setting(args[5], "top_p", at::kFloat, R, index, a.top_p, number);
        a.row_min_p = setting(args[6], "min_p", at::kFloat, R, index, a.min_p, number);
        if (guided) a.row_cfg_scale = setting(args[7], "cfg_scale", at::kFloat, R, index, a.cfg_scale, number);
        a.u = static_cast<const float *>(dense(tensor(args[2], "u"), "u", at::kFloat, {R}, index));
        a.v_begin = integer(args[8], "v_begin");
        a.v_end = args[9] == Py_None ? a.V : integer(args[9], "v_end");
        std::optional<at::Tensor> made;
        const at::Tensor *out = tensor(args[10], "token", false);
        if (!out) out = &made.emplace(at::empty({R}, x.options().dtype(at::kInt)));
        a.token = static_cast<int32_t *>(const_cast<void *>(dense(out, "token", at::kInt, {R}, index)));
        a.token_prob = static_cast<float *>(const_cast<void *>(dense(tensor(args[11], "token_prob", false), "token_prob", at::kFloat, {R}, index)));
        if (const at::Tensor *probs = tensor(args[12], "probs", false)) {
            const int64_t shape[2] = {R, V};
            a.probs = static_cast<float *>(rows_of(*probs, "probs", at::kFloat, shape, index, a.probs_row_stride));
        }
        int32_t *status = status_word(args[13], index);
        const long rc = run_on(index, [&](hawk_stream_t st) { return fn(&a, status, st); });
        return Py_BuildValue("lN", rc, owned(args[10], made ? &*made : nullptr));
    });
}

// ---------------------------------------------------------------------------------------------- pages
const int32_t *ints(PyObject *o, const char *name, at::IntArrayRef shape, int index, bool needed = true)
{
    return static_cast<const int32_t *>(dense(tensor(o, name, needed), name, at::kInt, shape, index));
}

// An int32 result: the given tensor, or `made`, new.
int32_t *result(PyObject *o, const char *name, at::IntArrayRef shape, int index, const at::Tensor &like, std::optional<at::Tensor> &made)
{
    if (o == Py_None) return static_cast<int32_t *>(made.emplace(at::empty(shape, like.options())).data_ptr());
    return const_cast<int32_t *>(ints(o, name, shape, index));
}

// An int32 result in place of `input` where none is given.
int32_t *in_place(PyObject *o, const char *name, at::IntArrayRef shape, int index, const int32_t *input)
{
    return o == Py_None ? const_cast<int32_t *>(input) : const_cast<int32_t *>(ints(o, name, shape, index));
}

// The cache's state: block_table, kv_len, page_refs, page_size from args[0], args[1], args[at], args[at + 1] on.
struct Pages {
    const at::Tensor &table;
    int index, S, W, n_pages, page_size;
    const int32_t *block_table, *kv_len, *refs;

    Pages(PyObject *t, PyObject *kv, PyObject *r, PyObject *page) : table(*tensor(t, "block_table"))
    {
        if (!table.is_cuda()) refuse(PyExc_ValueError, "block_table: must be a CUDA tensor");
        dims(table, "block_table", 2);
        index = table.get_device();
        S = as_int(table.size(0), "streams");
        W = as_int(table.size(1), "table width");
        block_table = ints(t, "block_table", table.sizes(), index);
        kv_len = ints(kv, "kv_len", {table.size(0)}, index);
        const at::Tensor &counts = *tensor(r, "page_refs");
        dims(counts, "page_refs", 1);
        n_pages = as_int(counts.size(0), "pages");
        refs = ints(r, "page_refs", counts.sizes(), index);
        page_size = integer(page, "page_size");
    }
};

// (entry point, block_table, kv_len, new_len, page_refs, page_size, out_table, out_len, out_refs, copies, dev_status) -> (status, copies)
PyObject *pages_resize(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        expect(n, 11);
        const auto fn = reinterpret_cast<decltype(&hawk_pages_resize)>(address(args[0]));
        const Pages p(args[1], args[2], args[4], args[5]);
        const int64_t S = p.S, W = p.W, N = p.n_pages, all[2] = {S, W}, three[2] = {S, 3};
        hawk_pages_resize_args a = {};
        a.S = p.S;
        a.table_width = p.W;
        a.n_pages = p.n_pages;
        a.page_size = p.page_size;
        a.block_table = p.block_table;
        a.kv_len = p.kv_len;
        a.page_refs = p.refs;
        a.new_len = ints(args[3], "new_len", {S}, p.index);
        a.out_table = in_place(args[6], "out_table", all, p.index, p.block_table);
        a.out_len = in_place(args[7], "out_len", {S}, p.index, p.kv_len);
        a.out_refs = in_place(args[8], "out_refs", {N}, p.index, p.refs);
        std::optional<at::Tensor> made;
        a.copies = result(args[9], "copies", three, p.index, p.table, made);
        int32_t *status = status_word(args[10], p.index);
        const long rc = run_on(p.index, [&](hawk_stream_t st) { return fn(&a, status, st); });
        return Py_BuildValue("lN", rc, owned(args[9], made ? &*made : nullptr));
    });
}

// (entry point, block_table, kv_len, parent, page_refs, page_size, length, out_table, out_len, out_refs, dev_status) -> (status, out_table,
// out_len)
PyObject *pages_fork(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        expect(n, 11);
        const auto fn = reinterpret_cast<decltype(&hawk_pages_fork)>(address(args[0]));
        const Pages p(args[1], args[2], args[4], args[5]);
        const at::Tensor &parent = *tensor(args[3], "parent");
        dims(parent, "parent", 1);
        const int64_t S = parent.size(0), W = p.W, N = p.n_pages, all[2] = {S, W};
        hawk_pages_fork_args a = {};
        a.S = p.S;
        a.S_out = as_int(S, "streams");
        a.table_width = p.W;
        a.n_pages = p.n_pages;
        a.page_size = p.page_size;
        a.block_table = p.block_table;
        a.kv_len = p.kv_len;
        a.page_refs = p.refs;
        a.parent = ints(args[3], "parent", {S}, p.index);
        a.length = ints(args[6], "length", {S}, p.index, false);
        std::optional<at::Tensor> table_made, len_made;
        a.out_table = result(args[7], "out_table", all, p.index, p.table, table_made);
        a.out_len = result(args[8], "out_len", {S}, p.index, p.table, len_made);
        a.out_refs = in_place(args[9], "out_refs", {N}, p.index, p.refs);
        int32_t *status = status_word(args[10], p.index);
        const long rc = run_on(p.index, [&](hawk_stream_t st) { return fn(&a, status, st); });
        return Py_BuildValue("lNN", rc, owned(args[7], table_made ? &*table_made : nullptr), owned(args[8], len_made ? &*len_made : nullptr));
    });
}

// (entry point, workspace query, block_table, kv_len, page_refs, page_size, max_moves, first_page, out_table, out_refs, copies, top, workspace,
// dev_status) -> (status, copies)
PyObject *pages_compact(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        expect(n, 14);
        const auto fn = reinterpret_cast<decltype(&hawk_pages_compact)>(address(args[0]));
        const auto need_of = reinterpret_cast<decltype(&hawk_pages_compact_workspace_bytes)>(address(args[1]));
        const Pages p(args[2], args[3], args[4], args[5]);
        hawk_pages_compact_args a = {};
        a.S = p.S;
        a.table_width = p.W;
        a.n_pages = p.n_pages;
        a.page_size = p.page_size;
        a.block_table = p.block_table;
        a.kv_len = p.kv_len;
        a.page_refs = p.refs;
        a.max_moves = integer(args[6], "max_moves");
        if (a.max_moves < 0) refuse(PyExc_ValueError, "max_moves: must not be negative");
        a.first_page = integer(args[7], "first_page");
        const int64_t S = p.S, W = p.W, N = p.n_pages, all[2] = {S, W}, three[2] = {a.max_moves, 3};
        a.out_table = in_place(args[8], "out_table", all, p.index, p.block_table);
        a.out_refs = in_place(args[9], "out_refs", {N}, p.index, p.refs);
        std::optional<at::Tensor> made, ws_made;
        a.copies = result(args[10], "copies", three, p.index, p.table, made);
        a.top = const_cast<int32_t *>(ints(args[11], "top", {1}, p.index, false));
        if (const at::Tensor *ws = tensor(args[12], "workspace", false)) {
            a.workspace = const_cast<void *>(dense(ws, "workspace", ws->scalar_type(), ws->sizes(), p.index));
            a.workspace_bytes = static_cast<size_t>(ws->numel()) * ws->element_size();
        } else if (const size_t need = need_of(a.n_pages, a.max_moves)) {
            a.workspace = ws_made.emplace(at::empty({static_cast<int64_t>(need)}, p.table.options().dtype(at::kByte))).data_ptr();
            a.workspace_bytes = need;
        }
        int32_t *status = status_word(args[13], p.index);
        const long rc = run_on(p.index, [&](hawk_stream_t st) { return fn(&a, status, st); });
        return Py_BuildValue("lN", rc, owned(args[10], made ? &*made : nullptr));
    });
}

// Page tensors [n_pages, H_kv, page_size, D], or [layers, n_pages, H_kv, page_size, D].
hawk_page_tensors page_tensors(PyObject *k, PyObject *v, int &index)
{
    const at::Tensor &kp = *tensor(k, "k_pages"), &vp = *tensor(v, "v_pages");
    const Where w = where(kp, "k_pages");
    index = w.index;
    if (kp.dim() != 4 && kp.dim() != 5) refuse(PyExc_ValueError, "k_pages: expected 4 or 5 dimensions, got " + text_of(kp.sizes()));
    hawk_page_tensors p = {};
    const int64_t at = kp.dim() - 4;
    p.k_pages = strided(kp, "k_pages", w.dtype, kp.sizes(), w.index);
    p.v_pages = strided(vp, "v_pages", w.dtype, kp.sizes(), w.index);
    p.layers = at ? as_int(kp.size(0), "layers") : 1;
    p.n_pages = as_int(kp.size(at), "pages");
    p.H_kv = as_int(kp.size(at + 1), "heads");
    p.page_size = as_int(kp.size(at + 2), "page size");
    p.D = as_int(kp.size(at + 3), "head dimension");
    auto stride = [](const at::Tensor &t, int64_t d) -> long long { return t.size(d) > 1 ? t.stride(d) : 0; };
    p.k_layer_stride = at ? stride(kp, 0) : 0;
    p.v_layer_stride = at ? stride(vp, 0) : 0;
    p.k_page_stride = stride(kp, at);
    p.v_page_stride = stride(vp, at);
    p.k_head_stride = stride(kp, at + 1);
    p.v_head_stride = stride(vp, at + 1);
    p.k_row_stride = stride(kp, at + 2);
    p.v_row_stride = stride(vp, at + 2);
    return p;
}

// (entry point, k_pages, v_pages, copies, dev_status) -> status
PyObject *pages_copy(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        expect(n, 5);
        const auto fn = reinterpret_cast<decltype(&hawk_pages_copy)>(address(args[0]));
        int index;
        const hawk_page_tensors p = page_tensors(args[1], args[2], index);
        const at::Tensor &copies = *tensor(args[3], "copies");
        dims(copies, "copies", 2);
        const int64_t three[2] = {copies.size(0), 3};
        const int32_t *list = ints(args[3], "copies", three, index);
        const int count = as_int(copies.size(0), "copies");
        int32_t *status = status_word(args[4], index);
        const long rc = run_on(index, [&](hawk_stream_t st) { return fn(&p, list, count, status, st); });
        return Py_BuildValue("l", rc);
    });
}

// (entry point, k_pages, v_pages, block_table, row_begin, kv_len, path, accept_len, first, out_len, dev_status) -> (status, out_len)
PyObject *pages_keep(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        expect(n, 11);
        const auto fn = reinterpret_cast<decltype(&hawk_pages_keep)>(address(args[0]));
        const at::Tensor &kv = *tensor(args[5], "kv_len");
        if (!kv.is_cuda()) refuse(PyExc_ValueError, "kv_len: must be a CUDA tensor");
        dims(kv, "kv_len", 1);
        int index = kv.get_device();
        const int64_t S = kv.size(0);
        hawk_pages_keep_args a = {};
        a.S = as_int(S, "streams");
        a.kv_len = ints(args[5], "kv_len", {S}, index);
        a.row_begin = ints(args[4], "row_begin", {S + 1}, index);
        const at::Tensor &accepted = *tensor(args[7], "accept_len");
        dims(accepted, "accept_len", 1);
        const int64_t B = accepted.size(0);
        a.B = as_int(B, "sequences");
        a.accept_len = ints(args[7], "accept_len", {B}, index);
        a.first = integer(args[8], "first");
        if (const at::Tensor *path = tensor(args[6], "path", false)) {
            dims(*path, "path", 2);
            const int64_t shape[2] = {B, path->size(1)};
            a.path = ints(args[6], "path", shape, index);
            if (!a.path) a.path = a.accept_len;  // (a path without columns has no address, and none of it is read; NULL would be a chain)
            a.path_width = as_int(path->size(1), "path");
            int pages_index;
            a.pages = page_tensors(args[1], args[2], pages_index);
            if (pages_index != index) refuse(PyExc_ValueError, "k_pages: must be on cuda:" + std::to_string(index));
            const at::Tensor &table = *tensor(args[3], "block_table");
            dims(table, "block_table", 2);
            const int64_t all[2] = {S, table.size(1)};
            a.block_table = ints(args[3], "block_table", all, index);
            a.table_width = as_int(table.size(1), "table width");
        }
        std::optional<at::Tensor> made;
        a.out_len = result(args[9], "out_len", {S}, index, kv, made);
        int32_t *status = status_word(args[10], index);
        const long rc = run_on(index, [&](hawk_stream_t st) { return fn(&a, status, st); });
        return Py_BuildValue("lN", rc, owned(args[9], made ? &*made : nullptr));
    });
}

PyMethodDef methods[] = {
    {"qk_norm_rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(qk_norm_rope)), METH_FASTCALL, nullptr},
    {"rope_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(rope_append)), METH_FASTCALL, nullptr},
    {"paged_attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(paged_attn)), METH_FASTCALL, nullptr},
    {"sample", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(sample)), METH_FASTCALL, nullptr},
    {"pages_resize", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(pages_resize)), METH_FASTCALL, nullptr},
    {"pages_fork", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(pages_fork)), METH_FASTCALL, nullptr},
    {"pages_compact", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(pages_compact)), METH_FASTCALL, nullptr},
    {"pages_copy", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(pages_copy)), METH_FASTCALL, nullptr},
    {"pages_keep", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(pages_keep)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_hawk_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__hawk_marshal()
{
    PyObject *m = PyModule_Create(&module_def);
    if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0) {  // whose tensors it can look into
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
