// Python entry of the serving attention: argument checks and marshalling in C++.
//
// A decode step calls these operators once per layer on small tensors, where the kernels take a few microseconds;
// checking and boxing some thirty arguments in Python takes 12 to 15.  This module does the same checks on the
// tensors' metadata directly and calls the C ABI (about 2 us on top of the launches).  It computes nothing.
#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <string>

#include "../../include/wht_attention.h"

namespace {

PyObject* g_raise = nullptr;  // binding._check(status, where): raises WhtError

struct Refused {
    std::string what;
};
[[noreturn]] void refuse(std::string what) { throw Refused{std::move(what)}; }

std::string shape_of(const at::Tensor& t) {
    std::string s = "[";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + "]";
}

const at::Tensor* tensor(PyObject* o, const char* name) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) refuse(std::string(name) + " must be a tensor");
    return &THPVariable_Unpack(o);
}
const at::Tensor& required(PyObject* o, const char* name) {
    const at::Tensor* t = tensor(o, name);
    if (!t) refuse(std::string(name) + " is missing");
    return *t;
}
int64_t integer(PyObject* o, const char* name) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        refuse(std::string(name) + " must be an integer");
    }
    return v;
}

// These operators have no backward: rather than cut a graph without a word they refuse to be part of one.
void no_gradient(const at::Tensor& t, const char* name) {
    if (t.requires_grad() && at::GradMode::is_enabled())
        refuse(std::string(name) + " requires a gradient and the serving attention has no backward: call it under torch.no_grad() or detach it");
}

struct Caches {
    const at::Tensor &k, &v;
    at::Device device;
    at::ScalarType type;
    int code;
    int64_t pages, hkv, page, dim;
};

Caches caches(PyObject* ko, PyObject* vo) {
    const at::Tensor &k = required(ko, "k_cache"), &v = required(vo, "v_cache");
    if (k.dim() != 4 || v.sizes() != k.sizes()) refuse("k_cache and v_cache must be [num_pages, kv_heads, page, head_dim] and of one shape");
    const auto type = k.scalar_type();
    if (v.scalar_type() != type || (type != at::kBFloat16 && type != at::kFloat))
        refuse("unsupported storage types: the caches must both be bf16 or both fp32");
    if (!k.is_cuda() || v.device() != k.device() || !k.is_contiguous() || !v.is_contiguous())
        refuse("caches must be contiguous tensors on one CUDA device");
    no_gradient(k, "k_cache");
    no_gradient(v, "v_cache");
    if (k.device().index() != c10::cuda::current_device()) refuse("all tensors must live on the current CUDA device");
    const int64_t page = k.size(2), dim = k.size(3);
    if ((page != 16 && page != 32 && page != 64 && page != 128) || (dim != 64 && dim != 96 && dim != 128))
        refuse("page must be 16, 32, 64 or 128 and head_dim 64, 96 or 128, got " + std::to_string(page) + " and " + std::to_string(dim));
    return {k, v, k.device(), type, type == at::kFloat ? WHT_F32 : WHT_BF16, k.size(0), k.size(1), page, dim};
}

// A [tokens, heads, head_dim] tensor with any token and head strides; heads or tokens < 0: any.
void rows(const at::Tensor& t, const char* name, int64_t tokens, int64_t heads, const Caches& c) {
    if (t.dim() != 3 || t.size(2) != c.dim || (heads >= 0 && t.size(1) != heads) || (tokens >= 0 && t.size(0) != tokens))
        refuse(std::string(name) + " must be [tokens, heads, head_dim] and match the other tensors, got " + shape_of(t));
    if (t.scalar_type() != c.type || t.device() != c.device) refuse(std::string(name) + " must have the caches' type and device");
    if (t.stride(2) != 1) refuse(std::string(name) + " must have contiguous channels");
    no_gradient(t, name);
}

void* vec(const at::Tensor& t, const char* name, at::ScalarType type, const Caches& c, at::IntArrayRef sizes) {
    if (t.scalar_type() != type || t.device() != c.device || t.sizes() != sizes || !t.is_contiguous())
        refuse(std::string(name) + " must be a contiguous " + c10::toString(type) + " tensor of the right shape on the caches' device, got " + shape_of(t));
    return t.data_ptr();
}

at::Tensor output(const at::Tensor* given, const at::Tensor& like, const char* name, const Caches& c) {
    if (!given) return at::detail::empty_cuda(like.sizes(), c.type, c.device, std::nullopt);
    if (given->sizes() != like.sizes() || given->scalar_type() != c.type || given->device() != c.device || !given->is_contiguous())
        refuse(std::string(name) + " must be contiguous and match q");
    return *given;
}

// Scratch of one call, taken from the caching allocator on the current stream.  When the call runs on another
// stream, the allocator is told of all its tensors, so that no block is handed out before that stream is done with it.
struct Scratch {
    c10::DataPtr mem;
    void* take(size_t bytes) {
        if (bytes) mem = c10::cuda::CUDACachingAllocator::get()->allocate(bytes);
        return mem.get();
    }
};

struct Stream {
    cudaStream_t raw;
    bool other;
    c10::DeviceIndex device;
    Stream(PyObject* o, const Caches& c) : device(c.device.index()) {
        const cudaStream_t current = c10::cuda::getCurrentCUDAStream(device).stream();
        raw = o == Py_None ? current : reinterpret_cast<cudaStream_t>(PyLong_AsVoidPtr(o));
        other = raw != current;
    }
    void uses(const c10::DataPtr& p) const {
        if (other && p) c10::cuda::CUDACachingAllocator::recordStream(p, c10::cuda::getStreamFromExternal(raw, device));
    }
    void uses(const at::Tensor& t) const { uses(t.storage().data_ptr()); }
    // every tensor among the arguments of a call
    void uses(PyObject* const* a, Py_ssize_t n) const {
        if (!other) return;
        for (Py_ssize_t i = 0; i < n; ++i)
            if (THPVariable_Check(a[i])) uses(THPVariable_Unpack(a[i]));
    }
};

struct Batch {
    int64_t size, width;
    void *table, *lens, *start;
};
Batch batch(PyObject* table_o, PyObject* lens_o, PyObject* start_o, int64_t tokens, int64_t max_q_len, const Caches& c) {
    const at::Tensor &table = required(table_o, "page_table"), &lens = required(lens_o, "kv_lens");
    if (table.dim() != 2) refuse("page_table must be [batch, pages]");
    Batch b{table.size(0), table.size(1), nullptr, nullptr, nullptr};
    b.table = vec(table, "page_table", at::kInt, c, {b.size, b.width});
    b.lens = vec(lens, "kv_lens", at::kInt, c, {b.size});
    if (const at::Tensor* start = tensor(start_o, "q_start")) {
        b.start = vec(*start, "q_start", at::kInt, c, {b.size + 1});
    } else if (tokens != b.size || max_q_len != 1) {
        refuse("without q_start every sequence has one token: got " + std::to_string(tokens) + " tokens for " + std::to_string(b.size) +
               " sequences, max_q_len " + std::to_string(max_q_len));
    }
    return b;
}

bool ok(int status, const char* where) {
    if (status == WHT_OK) return true;
    PyObject* r = PyObject_CallFunction(g_raise, "is", status, where);
    Py_XDECREF(r);
    return false;
}

PyObject* keep(PyObject* o) {
    Py_INCREF(o);
    return o;
}

template <typename F>
PyObject* guarded(F f) {
    try {
        return f();
    } catch (const Refused& r) {
        PyErr_SetString(PyExc_ValueError, r.what.c_str());
    } catch (const c10::OutOfMemoryError& e) {
        PyErr_SetString(PyExc_MemoryError, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

bool count(Py_ssize_t got, Py_ssize_t want) {
    if (got == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments, expected %zd", got, want);
    return false;
}

// kv_append(k, v, k_cache, v_cache, slots, positions, cos, sin, q, q_out, summary, summary_scale, interleaved, stream)
PyObject* kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!count(n, 14)) return nullptr;
    return guarded([&]() -> PyObject* {
        const at::Tensor &k = required(a[0], "k"), &v = required(a[1], "v");
        const Caches c = caches(a[2], a[3]);
        rows(k, "k", -1, c.hkv, c);
        const int64_t tokens = k.size(0);
        rows(v, "v", tokens, c.hkv, c);
        void* slots = vec(required(a[4], "slots"), "slots", at::kLong, c, {tokens});
        const at::Tensor *pos = tensor(a[5], "positions"), *cos = tensor(a[6], "cos"), *sin = tensor(a[7], "sin");
        int64_t rot = 0, max_pos = 0;
        void *pos_p = nullptr, *cos_p = nullptr, *sin_p = nullptr;
        if (pos || cos || sin) {
            if (!pos || !cos || !sin || cos->dim() != 2) refuse("positions, cos and sin [max_pos, rot/2] come together");
            max_pos = cos->size(0);
            rot = 2 * cos->size(1);
            if (rot % 16 || rot > c.dim || max_pos < 1)
                refuse("rot = " + std::to_string(rot) + " must be a multiple of 16 up to head_dim, with at least one position");
            cos_p = vec(*cos, "cos", at::kFloat, c, {max_pos, rot / 2});
            sin_p = vec(*sin, "sin", at::kFloat, c, {max_pos, rot / 2});
            pos_p = vec(*pos, "positions", at::kInt, c, {tokens});
        }
        const at::Tensor *q = tensor(a[8], "q"), *q_given = tensor(a[9], "q_out");
        const Stream s(a[13], c);
        at::Tensor q_out;
        int64_t hq = c.hkv, q_st = 0, q_sh = 0;
        void *q_p = nullptr, *out_p = nullptr;
        if (q) {
            rows(*q, "q", tokens, -1, c);
            hq = q->size(1);
            q_st = q->stride(0);
            q_sh = q->stride(1);
            q_out = output(q_given, *q, "q_out", c);
            q_p = q->data_ptr();
            out_p = q_out.data_ptr();
        } else if (q_given) {
            refuse("q_out without q");
        }
        void *sum_p = nullptr, *scale_p = nullptr;
        if (const at::Tensor* summary = tensor(a[10], "summary")) {
            sum_p = vec(*summary, "summary", at::kChar, c, {c.pages, c.hkv, 2, c.dim});
            scale_p = vec(required(a[11], "summary_scale"), "summary_scale", at::kFloat, c, {c.hkv});
        }
        const int interleaved = PyObject_IsTrue(a[12]);
        if (interleaved < 0) return nullptr;  // (no truth value: the error is set)
        const int rc = wht_kv_append(k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1), q_p, q_st, q_sh, out_p,
                                     static_cast<const int64_t*>(slots), static_cast<const int32_t*>(pos_p), static_cast<const float*>(cos_p),
                                     static_cast<const float*>(sin_p), c.k.data_ptr(), c.v.data_ptr(), static_cast<int8_t*>(sum_p),
                                     static_cast<const float*>(scale_p), tokens, static_cast<int32_t>(hq), static_cast<int32_t>(c.hkv),
                                     static_cast<int32_t>(c.dim), static_cast<int32_t>(rot), interleaved, max_pos, c.pages,
                                     static_cast<int32_t>(c.page), c.code, s.raw);
        s.uses(a, n);
        if (!ok(rc, "wht_kv_append")) return nullptr;
        if (!q) return keep(Py_None);
        if (q_given) return keep(a[9]);
        s.uses(q_out);
        return THPVariable_Wrap(std::move(q_out));
    });
}

float scale_of(PyObject* o, const Caches& c) {
    if (o == Py_None) return static_cast<float>(1.0 / std::sqrt(static_cast<double>(c.dim)));
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        refuse("scale must be a number");
    }
    return static_cast<float>(v);
}

// shared_prefix_attention(q, k_cache, v_cache, prefix_pages, prefix_len, page_table, kv_lens, q_start, max_q_len, scale, out, stream)
PyObject* shared_prefix_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!count(n, 12)) return nullptr;
    return guarded([&]() -> PyObject* {
        const at::Tensor& q = required(a[0], "q");
        const Caches c = caches(a[1], a[2]);
        rows(q, "q", -1, -1, c);
        const int64_t tokens = q.size(0), hq = q.size(1), prefix_len = integer(a[4], "prefix_len"), max_q = integer(a[8], "max_q_len");
        const Batch b = batch(a[5], a[6], a[7], tokens, max_q, c);
        if (prefix_len < 0) refuse("prefix_len must be >= 0");
        void* prefix_p = nullptr;
        if (prefix_len > 0) {
            const at::Tensor& pages = required(a[3], "prefix_pages");
            prefix_p = vec(pages, "prefix_pages", at::kInt, c, {pages.numel()});
            if (pages.numel() * c.page < prefix_len)
                refuse(std::to_string(pages.numel()) + " prefix pages do not hold " + std::to_string(prefix_len) + " keys");
        }
        const float scale = scale_of(a[9], c);
        const Stream s(a[11], c);
        const at::Tensor* given = tensor(a[10], "out");
        at::Tensor out = output(given, q, "out", c);
        const auto i32 = [](int64_t v) { return static_cast<int32_t>(v > 0x7fffffff ? 0x7fffffff : v); };
        const size_t need = wht_attn_prefix_workspace_bytes(prefix_len, i32(b.width), tokens, i32(b.size), i32(max_q), i32(hq), i32(c.hkv),
                                                            i32(c.dim), i32(c.page), c.code);
        Scratch work;
        void* ws = work.take(need);
        const int rc = wht_attn_prefix(q.data_ptr(), q.stride(0), q.stride(1), c.k.data_ptr(), c.v.data_ptr(), static_cast<const int32_t*>(prefix_p),
                                       prefix_len, static_cast<const int32_t*>(b.table), i32(b.width), static_cast<const int32_t*>(b.lens),
                                       static_cast<const int32_t*>(b.start), out.data_ptr(), tokens, i32(b.size), i32(max_q), i32(hq), i32(c.hkv),
                                       i32(c.dim), c.pages, i32(c.page), scale, c.code, ws, need, s.raw);
        s.uses(work.mem);
        s.uses(a, n);
        if (!ok(rc, "wht_attn_prefix")) return nullptr;
        if (given) return keep(a[10]);
        s.uses(out);
        return THPVariable_Wrap(std::move(out));
    });
}

// selected_page_attention(q, k_cache, v_cache, summary, page_table, kv_lens, select, q_start, max_q_len, scale, out, pages_out, stream)
PyObject* selected_page_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!count(n, 13)) return nullptr;
    return guarded([&]() -> PyObject* {
        const at::Tensor& q = required(a[0], "q");
        const Caches c = caches(a[1], a[2]);
        rows(q, "q", -1, -1, c);
        const int64_t tokens = q.size(0), hq = q.size(1), select = integer(a[6], "select"), max_q = integer(a[8], "max_q_len");
        const Batch b = batch(a[4], a[5], a[7], tokens, max_q, c);
        void* sum_p = vec(required(a[3], "summary"), "summary", at::kChar, c, {c.pages, c.hkv, 2, c.dim});
        if (select < 1 || select > 1024) refuse("select must be between 1 and 1024");
        const float scale = scale_of(a[9], c);
        const Stream s(a[12], c);
        const at::Tensor *given = tensor(a[10], "out"), *given_pages = tensor(a[11], "pages_out");
        at::Tensor out = output(given, q, "out", c);
        at::Tensor pages;
        if (given_pages) pages = *given_pages;
        else pages = at::detail::empty_cuda({tokens, c.hkv, select}, at::kInt, c.device, std::nullopt);
        void* pages_p = vec(pages, "pages_out", at::kInt, c, {tokens, c.hkv, select});
        const auto i32 = [](int64_t v) { return static_cast<int32_t>(v > 0x7fffffff ? 0x7fffffff : v); };
        const size_t need = wht_attn_select_workspace_bytes(i32(b.width), i32(select), tokens, i32(b.size), i32(max_q), i32(hq), i32(c.hkv),
                                                            i32(c.dim), i32(c.page), c.code);
        Scratch work;
        void* ws = work.take(need);
        const int rc = wht_attn_select(q.data_ptr(), q.stride(0), q.stride(1), c.k.data_ptr(), c.v.data_ptr(), static_cast<const int8_t*>(sum_p),
                                       static_cast<const int32_t*>(b.table), i32(b.width), static_cast<const int32_t*>(b.lens),
                                       static_cast<const int32_t*>(b.start), i32(select), out.data_ptr(), static_cast<int32_t*>(pages_p), tokens,
                                       i32(b.size), i32(max_q), i32(hq), i32(c.hkv), i32(c.dim), c.pages, i32(c.page), scale, c.code, ws, need, s.raw);
        s.uses(work.mem);
        s.uses(a, n);
        if (!ok(rc, "wht_attn_select")) return nullptr;
        if (!given) s.uses(out);
        if (!given_pages) s.uses(pages);
        PyObject* r = PyTuple_New(2);
        if (!r) return nullptr;
        PyTuple_SET_ITEM(r, 0, given ? keep(a[10]) : THPVariable_Wrap(std::move(out)));
        PyTuple_SET_ITEM(r, 1, given_pages ? keep(a[11]) : THPVariable_Wrap(std::move(pages)));
        return r;
    });
}

PyObject* raise_with(PyObject*, PyObject* f) {
    Py_INCREF(f);
    Py_XDECREF(g_raise);
    g_raise = f;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"kv_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv_append)), METH_FASTCALL, nullptr},
    {"shared_prefix_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(shared_prefix_attention)), METH_FASTCALL, nullptr},
    {"selected_page_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(selected_page_attention)), METH_FASTCALL, nullptr},
    {"raise_with", raise_with, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_attention", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__attention(void) { return PyModule_Create(&module); }
