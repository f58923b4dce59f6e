// CPython side of the calls a decode loop makes once or twice per layer: argument checks, output allocation, stream
// lookup and the C-ABI call, in C++.  Through ctypes and torch's Python API the same steps took 11 us of host time per
// call (17 us with outputs to allocate), more than the kernels of a one-token layer; here they take 1 to 2 us besides
// the launches themselves.  No arithmetic, no CUDA calls of its own: the entry points of libexmoe.so come in as
// addresses (set_entry_points), everything else is marshalling with the rules of binding.py.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>

#include <algorithm>

#include "../../include/exmoe.h"

// read from the file before it is loaded (build.native_is_current)
extern "C" __attribute__((used)) const char exmoe_native_torch_tag[] = EXMOE_TORCH_TAG;

namespace {

decltype(&exmoe_route) g_route = nullptr;
decltype(&exmoe_moe_forward) g_forward = nullptr;
decltype(&exmoe_moe_forward_host) g_forward_host = nullptr;
decltype(&exmoe_route_gated) g_route_gated = nullptr;
decltype(&exmoe_gate_logits) g_gate_logits = nullptr;
decltype(&exmoe_lora_plan_bytes) g_lora_plan_bytes = nullptr;
decltype(&exmoe_lora_plan) g_lora_plan = nullptr;
decltype(&exmoe_lora) g_lora = nullptr;

PyObject *s_d_model, *s_d_ff, *s_experts, *s_top_k, *s_group, *s_cuda_stream;
PyObject *s_score, *s_num_groups, *s_top_groups, *s_group_score, *s_renormalise, *s_scale;

PyObject* bad_tensor(const char* what, bool cuda, const char* dtype) {
    PyErr_Format(PyExc_ValueError, "%s: need a contiguous %s tensor of %s", what, cuda ? "CUDA" : "CPU", dtype);
    return nullptr;
}
const at::Tensor* tensor(PyObject* o, at::ScalarType dt, bool cuda, const char* what, const char* name) {
    if (THPVariable_Check(o)) {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.is_cuda() == cuda && t.scalar_type() == dt && t.is_contiguous()) return &t;
    }
    bad_tensor(what, cuda, name);
    return nullptr;
}
constexpr const char *kBf16 = "torch.bfloat16", *kF32 = "torch.float32", *kI32 = "torch.int32";

// int(o): whatever Python's int() takes, a float or a zero-dimensional array among them
bool to_int(PyObject* o, int* v) {
    PyObject* i = PyLong_CheckExact(o) ? Py_NewRef(o) : PyNumber_Long(o);
    if (!i) return false;
    const long x = PyLong_AsLong(i);
    Py_DECREF(i);
    if (x == -1 && PyErr_Occurred()) return false;
    *v = (int)x;
    return true;
}
bool int_attr(PyObject* o, PyObject* name, int* v) {
    PyObject* a = PyObject_GetAttr(o, name);
    if (!a) return false;
    const bool ok = to_int(a, v);
    Py_DECREF(a);
    return ok;
}
bool gate_shape_of(PyObject* o, exmoe_shape* s, bool d_model) {            // what a gate needs of a layer's shape
    *s = exmoe_shape{};
    return (!d_model || int_attr(o, s_d_model, &s->d_model)) && int_attr(o, s_experts, &s->num_experts) && int_attr(o, s_top_k, &s->top_k);
}
bool shape_of(PyObject* o, exmoe_shape* s) {
    if (!int_attr(o, s_d_model, &s->d_model) || !int_attr(o, s_d_ff, &s->d_ff) || !int_attr(o, s_experts, &s->num_experts) ||
        !int_attr(o, s_top_k, &s->top_k))
        return false;
    if (!int_attr(o, s_group, &s->group_size)) {
        if (!PyErr_ExceptionMatches(PyExc_AttributeError)) return false;
        PyErr_Clear();
        s->group_size = 128;
    }
    return true;
}
bool stream_of(PyObject* o, void** st) {
    if (o == Py_None) {
        *st = c10::cuda::getCurrentCUDAStream().stream();
        return true;
    }
    PyObject* a = PyObject_GetAttr(o, s_cuda_stream);
    if (!a) return false;
    *st = PyLong_AsVoidPtr(a);
    Py_DECREF(a);
    return !(PyErr_Occurred());
}
at::Tensor empty_on(const at::Tensor& like, at::IntArrayRef sizes, at::ScalarType dt) {
    return at::detail::empty_cuda(sizes, dt, like.device(), std::nullopt);
}
// Every entry returns the result object, or the (non-zero) status as an int, or nullptr with an exception set (torch's
// own, an exhausted allocator among them, translated as torch does).
template <typename F>
PyObject* guarded(F f) {
    HANDLE_TH_ERRORS
    return f();
    END_HANDLE_TH_ERRORS
}

// route(shape, hidden, w_router, bias, topk_ids, topk_weights, stream) -> (ids, weights)
PyObject* route(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 7) return PyErr_Format(PyExc_TypeError, "route: 7 arguments");
    return guarded([&]() -> PyObject* {
        exmoe_shape s;
        if (!shape_of(a[0], &s)) return nullptr;
        const at::Tensor *h, *w, *b = nullptr, *i = nullptr, *p = nullptr;
        if (!(h = tensor(a[1], at::kBFloat16, true, "hidden", kBf16))) return nullptr;
        if (!(w = tensor(a[2], at::kBFloat16, true, "w_router", kBf16))) return nullptr;
        if (a[3] != Py_None && !(b = tensor(a[3], at::kFloat, true, "bias", kF32))) return nullptr;
        if (a[4] != Py_None && !(i = tensor(a[4], at::kInt, true, "topk_ids", kI32))) return nullptr;
        if (a[5] != Py_None && !(p = tensor(a[5], at::kFloat, true, "topk_weights", kF32))) return nullptr;
        void* st;
        if (!stream_of(a[6], &st)) return nullptr;
        const int T = (int)h->size(0);
        at::Tensor ids = i ? *i : empty_on(*h, {T, s.top_k}, at::kInt);
        at::Tensor wts = p ? *p : empty_on(*h, {T, s.top_k}, at::kFloat);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_route(&s, h->data_ptr(), w->data_ptr(), b ? static_cast<const float*>(b->data_ptr()) : nullptr, T,
                     static_cast<int32_t*>(ids.data_ptr()), static_cast<float*>(wts.data_ptr()), st);
        Py_END_ALLOW_THREADS
        if (rc) return PyLong_FromLong(rc);
        PyObject* oi = i ? Py_NewRef(a[4]) : THPVariable_Wrap(std::move(ids));
        PyObject* op = p ? Py_NewRef(a[5]) : THPVariable_Wrap(std::move(wts));
        PyObject* r = oi && op ? PyTuple_Pack(2, oi, op) : nullptr;
        Py_XDECREF(oi);
        Py_XDECREF(op);
        return r;
    });
}

// forward(handle, layer, hidden, topk_ids, topk_weights, out, stream) -> out
PyObject* forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 7) return PyErr_Format(PyExc_TypeError, "forward: 7 arguments");
    return guarded([&]() -> PyObject* {
        exmoe_cache* c = static_cast<exmoe_cache*>(PyLong_AsVoidPtr(a[0]));
        int layer;
        if (PyErr_Occurred() || !to_int(a[1], &layer)) return nullptr;
        const at::Tensor *h, *i, *p, *o = nullptr;
        if (!(h = tensor(a[2], at::kBFloat16, true, "hidden", kBf16))) return nullptr;
        if (!(i = tensor(a[3], at::kInt, true, "topk_ids", kI32))) return nullptr;
        if (!(p = tensor(a[4], at::kFloat, true, "topk_weights", kF32))) return nullptr;
        if (a[5] != Py_None && !(o = tensor(a[5], at::kBFloat16, true, "out", kBf16))) return nullptr;
        void* st;
        if (!stream_of(a[6], &st)) return nullptr;
        at::Tensor out = o ? *o : empty_on(*h, h->sizes(), at::kBFloat16);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_forward(c, layer, h->data_ptr(), static_cast<const int32_t*>(i->data_ptr()), static_cast<const float*>(p->data_ptr()),
                       (int)h->size(0), out.data_ptr(), st);
        Py_END_ALLOW_THREADS
        if (rc) return PyLong_FromLong(rc);
        return o ? Py_NewRef(a[5]) : THPVariable_Wrap(std::move(out));
    });
}

// forward_host(handle, layer, hidden, topk_ids, topk_weights, out, stream) -> None (host tensors, `out` given)
PyObject* forward_host(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 7) return PyErr_Format(PyExc_TypeError, "forward_host: 7 arguments");
    return guarded([&]() -> PyObject* {
        exmoe_cache* c = static_cast<exmoe_cache*>(PyLong_AsVoidPtr(a[0]));
        int layer;
        if (PyErr_Occurred() || !to_int(a[1], &layer)) return nullptr;
        const at::Tensor *h, *i, *p, *o;
        if (!(h = tensor(a[2], at::kBFloat16, false, "hidden", kBf16))) return nullptr;
        if (!(i = tensor(a[3], at::kInt, false, "topk_ids", kI32))) return nullptr;
        if (!(p = tensor(a[4], at::kFloat, false, "topk_weights", kF32))) return nullptr;
        if (!(o = tensor(a[5], at::kBFloat16, false, "out", kBf16))) return nullptr;
        void* st;
        if (!stream_of(a[6], &st)) return nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_forward_host(c, layer, h->data_ptr(), static_cast<const int32_t*>(i->data_ptr()),
                            static_cast<const float*>(p->data_ptr()), (int)h->size(0), o->data_ptr(), st);
        Py_END_ALLOW_THREADS
        if (rc) return PyLong_FromLong(rc);
        Py_RETURN_NONE;
    });
}

// ---- the gate and the adapters --------------------------------------------------------------------------------------
// Their tensors' sizes are checked, and that they are on one device, the current one (the library launches there).
bool wrong(const char* what, const char* need) {
    PyErr_Format(PyExc_ValueError, "%s: need %s", what, need);
    return false;
}
bool sized(const at::Tensor& t, at::IntArrayRef sizes, const char* what, const char* need) {
    return t.sizes() == sizes || wrong(what, need);
}
bool here(const at::Tensor& t, const char* what) {
    return t.device().index() == c10::cuda::current_device() || wrong(what, "a tensor on the current CUDA device");
}
// a CUDA tensor with rows of consecutive elements, at any distance
const at::Tensor* rows(PyObject* o, at::ScalarType dt, const char* what, const char* need) {
    if (THPVariable_Check(o)) {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.is_cuda() && t.scalar_type() == dt && t.dim() == 2 && (t.stride(1) == 1 || t.size(1) <= 1) && t.stride(0) >= 0) return &t;
    }
    wrong(what, need);
    return nullptr;
}
int64_t pitch(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : std::max<int64_t>(t.stride(0), t.size(1)); }
// rows of a single-row tensor have no distance: any multiple of eight will do
int64_t pitch8(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : (t.size(1) + 7) / 8 * 8; }
bool int32_of(int64_t v, int* out, const char* what) {
    if (v > INT32_MAX) return wrong(what, "fewer than 2^31 rows and columns");
    *out = (int)v;
    return true;
}
// "softmax" / "sigmoid" and "max" / "top2", or the numbers of exmoe.h
bool choice_attr(PyObject* o, PyObject* name, const char* zero, const char* one, int* v) {
    PyObject* a = PyObject_GetAttr(o, name);
    if (!a) return false;
    bool ok = true;
    if (PyUnicode_Check(a)) {
        *v = PyUnicode_CompareWithASCIIString(a, zero) == 0 ? 0 : PyUnicode_CompareWithASCIIString(a, one) == 0 ? 1 : -1;
        if (*v < 0) ok = PyErr_Format(PyExc_ValueError, "gate.%U: '%s' or '%s'", name, zero, one) != nullptr;
    } else {
        ok = to_int(a, v);
    }
    Py_DECREF(a);
    return ok;
}
bool gate_of(PyObject* o, exmoe_gate* g) {
    if (!choice_attr(o, s_score, "softmax", "sigmoid", &g->score) || !int_attr(o, s_num_groups, &g->num_groups) ||
        !int_attr(o, s_top_groups, &g->top_groups) || !choice_attr(o, s_group_score, "max", "top2", &g->group_score) ||
        !int_attr(o, s_renormalise, &g->renormalise))
        return false;
    PyObject* a = PyObject_GetAttr(o, s_scale);
    if (!a) return false;
    g->weight_scale = (float)PyFloat_AsDouble(a);
    Py_DECREF(a);
    return !PyErr_Occurred();
}
// Outputs are allocated on the stream that writes them: memory that the allocator hands out again is ordered by it.
class OnStream {
  public:
    OnStream(PyObject* o, void* st) {
        if (o != Py_None) guard_.reset_stream(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(st), c10::cuda::current_device()));
    }

  private:
    c10::cuda::OptionalCUDAStreamGuard guard_;
};
const at::Tensor* optional_f32(PyObject* o, at::IntArrayRef sizes, const char* what, const char* need, bool* ok) {
    if (o == Py_None) return nullptr;
    const at::Tensor* t = tensor(o, at::kFloat, true, what, kF32);
    *ok = t && sized(*t, sizes, what, need) && here(*t, what);
    return t;
}
const float* data_of(const at::Tensor* t) { return t ? static_cast<const float*>(t->data_ptr()) : nullptr; }

// The ids and weights of a gate: those given, checked, or new ones.
struct Choice {
    at::Tensor ids, weights;
    PyObject *oi, *op;
    bool init(PyObject* i, PyObject* p, const at::Tensor& like, int T, int k) {
        oi = i;
        op = p;
        const at::Tensor* t;
        if (i != Py_None) {
            if (!(t = tensor(i, at::kInt, true, "topk_ids", kI32)) || !sized(*t, {T, k}, "topk_ids", "[T, top_k]") || !here(*t, "topk_ids")) return false;
            ids = *t;
        } else {
            ids = empty_on(like, {T, k}, at::kInt);
        }
        if (p != Py_None) {
            if (!(t = tensor(p, at::kFloat, true, "topk_weights", kF32)) || !sized(*t, {T, k}, "topk_weights", "[T, top_k]") || !here(*t, "topk_weights")) return false;
            weights = *t;
        } else {
            weights = empty_on(like, {T, k}, at::kFloat);
        }
        return true;
    }
    PyObject* result() {
        PyObject* i = oi != Py_None ? Py_NewRef(oi) : THPVariable_Wrap(std::move(ids));
        PyObject* p = op != Py_None ? Py_NewRef(op) : THPVariable_Wrap(std::move(weights));
        PyObject* r = i && p ? PyTuple_Pack(2, i, p) : nullptr;
        Py_XDECREF(i);
        Py_XDECREF(p);
        return r;
    }
};

// route_gated(shape, gate, hidden, w_router, bias, addend, balance, topk_ids, topk_weights, stream) -> (ids, weights)
PyObject* route_gated(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 10) return PyErr_Format(PyExc_TypeError, "route_gated: 10 arguments");
    return guarded([&]() -> PyObject* {
        exmoe_shape s;
        exmoe_gate g;
        if (!gate_shape_of(a[0], &s, true) || !gate_of(a[1], &g)) return nullptr;
        const at::Tensor *h, *w;
        if (!(h = tensor(a[2], at::kBFloat16, true, "hidden", kBf16))) return nullptr;
        if (!(w = tensor(a[3], at::kBFloat16, true, "w_router", kBf16))) return nullptr;
        int T;
        if (h->dim() != 2 || h->size(1) != s.d_model) return wrong("hidden", "[T, d_model]"), nullptr;
        if (!int32_of(h->size(0), &T, "hidden") || !sized(*w, {s.num_experts, s.d_model}, "w_router", "[num_experts, d_model]")) return nullptr;
        if (!here(*h, "hidden") || !here(*w, "w_router")) return nullptr;
        bool ok = true;
        const at::Tensor* b = optional_f32(a[4], {s.num_experts}, "bias", "[num_experts]", &ok);
        if (!ok) return nullptr;
        const at::Tensor* add = optional_f32(a[5], {T, s.num_experts}, "addend", "[T, num_experts]", &ok);
        if (!ok) return nullptr;
        const at::Tensor* bal = optional_f32(a[6], {s.num_experts}, "balance", "[num_experts]", &ok);
        if (!ok) return nullptr;
        void* st;
        if (!stream_of(a[9], &st)) return nullptr;
        const OnStream on(a[9], st);
        Choice c;
        if (!c.init(a[7], a[8], *h, T, s.top_k)) return nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_route_gated(&s, &g, h->data_ptr(), w->data_ptr(), data_of(b), data_of(add), data_of(bal), T, static_cast<int32_t*>(c.ids.data_ptr()),
                           static_cast<float*>(c.weights.data_ptr()), st);
        Py_END_ALLOW_THREADS
        return rc ? PyLong_FromLong(rc) : c.result();
    });
}

// gate_logits(shape, gate, logits, balance, topk_ids, topk_weights, stream) -> (ids, weights)
PyObject* gate_logits(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 7) return PyErr_Format(PyExc_TypeError, "gate_logits: 7 arguments");
    return guarded([&]() -> PyObject* {
        exmoe_shape s;
        exmoe_gate g;
        if (!gate_shape_of(a[0], &s, false) || !gate_of(a[1], &g)) return nullptr;
        const bool bf16 = THPVariable_Check(a[2]) && THPVariable_Unpack(a[2]).scalar_type() == at::kBFloat16;
        const at::Tensor* z = rows(a[2], bf16 ? at::kBFloat16 : at::kFloat, "logits", "a CUDA matrix of torch.float32 or torch.bfloat16 with rows of consecutive elements");
        if (!z) return nullptr;
        if (z->size(1) != s.num_experts) return wrong("logits", "[T, num_experts]"), nullptr;
        int T;
        if (!int32_of(z->size(0), &T, "logits") || !here(*z, "logits")) return nullptr;
        bool ok = true;
        const at::Tensor* bal = optional_f32(a[3], {s.num_experts}, "balance", "[num_experts]", &ok);
        if (!ok) return nullptr;
        void* st;
        if (!stream_of(a[6], &st)) return nullptr;
        const OnStream on(a[6], st);
        Choice c;
        if (!c.init(a[4], a[5], *z, T, s.top_k)) return nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = g_gate_logits(&s, &g, z->data_ptr(), bf16 ? EXMOE_BF16 : EXMOE_F32, pitch(*z), data_of(bal), T, static_cast<int32_t*>(c.ids.data_ptr()),
                           static_cast<float*>(c.weights.data_ptr()), st);
        Py_END_ALLOW_THREADS
        return rc ? PyLong_FromLong(rc) : c.result();
    });
}

// lora_plan(adapter_ids, num_adapters, plan, stream) -> plan
PyObject* lora_plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 4) return PyErr_Format(PyExc_TypeError, "lora_plan: 4 arguments");
    return guarded([&]() -> PyObject* {
        const at::Tensor *ids, *p = nullptr;
        int T, na;
        if (!(ids = tensor(a[0], at::kInt, true, "adapter_ids", kI32)) || !to_int(a[1], &na)) return nullptr;
        if (ids->dim() != 1) return wrong("adapter_ids", "[T]"), nullptr;
        if (!int32_of(ids->size(0), &T, "adapter_ids") || !here(*ids, "adapter_ids")) return nullptr;
        size_t bytes = 0;
        int rc = g_lora_plan_bytes(T, na, &bytes);
        if (rc) return PyLong_FromLong(rc);
        void* st;
        if (!stream_of(a[3], &st)) return nullptr;
        if (a[2] != Py_None) {
            if (!(p = tensor(a[2], at::kInt, true, "plan", kI32)) || !here(*p, "plan")) return nullptr;
            if (p->dim() != 1 || p->size(0) != (int64_t)bytes / 4) return wrong("plan", "one of as many tokens and adapters"), nullptr;
        }
        const OnStream on(a[3], st);
        at::Tensor plan = p ? *p : empty_on(*ids, {(int64_t)bytes / 4}, at::kInt);
        Py_BEGIN_ALLOW_THREADS
        rc = g_lora_plan(static_cast<const int32_t*>(ids->data_ptr()), T, na, plan.data_ptr(), st);
        Py_END_ALLOW_THREADS
        if (rc) return PyLong_FromLong(rc);
        return p ? Py_NewRef(a[2]) : THPVariable_Wrap(std::move(plan));
    });
}

// lora(plan, x, a, b, scale, base, out, out_dtype, stream) -> out
PyObject* lora(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 9) return PyErr_Format(PyExc_TypeError, "lora: 9 arguments");
    return guarded([&]() -> PyObject* {
        const at::Tensor *p, *x, *wa, *wb, *sc, *base = nullptr, *o = nullptr;
        if (!(p = tensor(a[0], at::kInt, true, "plan", kI32))) return nullptr;
        if (!(x = rows(a[1], at::kBFloat16, "x", "a CUDA matrix of torch.bfloat16 with rows of consecutive elements"))) return nullptr;
        if (!(wa = tensor(a[2], at::kBFloat16, true, "a", kBf16)) || !(wb = tensor(a[3], at::kBFloat16, true, "b", kBf16))) return nullptr;
        if (!(sc = tensor(a[4], at::kFloat, true, "scale", kF32))) return nullptr;
        if (wa->dim() != 3 || wb->dim() != 3) return wrong(wa->dim() != 3 ? "a" : "b", "[num_adapters, rank, d_in] and [num_adapters, d_out, rank]"), nullptr;
        int T, na, r, K, N;
        if (!int32_of(x->size(0), &T, "x") || !int32_of(wa->size(0), &na, "a") || !int32_of(wa->size(1), &r, "a") || !int32_of(wa->size(2), &K, "a") ||
            !int32_of(wb->size(1), &N, "b"))
            return nullptr;
        if (x->size(1) != K) return wrong("x", "[T, d_in]"), nullptr;
        if (!sized(*wb, {na, N, r}, "b", "[num_adapters, d_out, rank]") || !sized(*sc, {na}, "scale", "[num_adapters]")) return nullptr;
        size_t bytes = 0;
        int rc = g_lora_plan_bytes(T, na, &bytes);
        if (rc) return PyLong_FromLong(rc);
        if (p->dim() != 1 || p->size(0) != (int64_t)bytes / 4) return wrong("plan", "one of as many tokens and adapters"), nullptr;
        at::ScalarType dt = at::kBFloat16;
        PyObject* like = a[5] != Py_None ? a[5] : a[6];
        if (like != Py_None) {
            if (THPVariable_Check(like)) dt = THPVariable_Unpack(like).scalar_type();
            if (a[7] != Py_None && (!THPDtype_Check(a[7]) || reinterpret_cast<THPDtype*>(a[7])->scalar_type != dt)) return wrong("out_dtype", "the type of base and out"), nullptr;
        } else if (a[7] != Py_None) {
            if (!THPDtype_Check(a[7])) return wrong("out_dtype", "a torch.dtype"), nullptr;
            dt = reinterpret_cast<THPDtype*>(a[7])->scalar_type;
        }
        if (dt != at::kFloat && dt != at::kBFloat16) return wrong("out_dtype", "torch.float32 or torch.bfloat16"), nullptr;
        constexpr const char* kRows = "a CUDA matrix [T, d_out] of torch.float32 or torch.bfloat16 with rows of consecutive elements";
        if (a[5] != Py_None && (!(base = rows(a[5], dt, "base", kRows)) || !sized(*base, {T, N}, "base", kRows))) return nullptr;
        if (a[6] != Py_None && (!(o = rows(a[6], dt, "out", kRows)) || !sized(*o, {T, N}, "out", kRows))) return nullptr;
        if (!here(*p, "plan") || !here(*x, "x") || !here(*wa, "a") || !here(*wb, "b") || !here(*sc, "scale") || (base && !here(*base, "base")) || (o && !here(*o, "out")))
            return nullptr;
        void* st;
        if (!stream_of(a[8], &st)) return nullptr;
        const OnStream on(a[8], st);
        at::Tensor out = o ? *o : empty_on(*x, {T, N}, dt);
        const exmoe_lora_shape s{na, K, N, r};
        Py_BEGIN_ALLOW_THREADS
        rc = g_lora(&s, p->data_ptr(), x->data_ptr(), pitch8(*x), wa->data_ptr(), wb->data_ptr(), static_cast<const float*>(sc->data_ptr()), T,
                    base ? base->data_ptr() : nullptr, base ? pitch(*base) : 0, out.data_ptr(), pitch(out), dt == at::kFloat ? EXMOE_F32 : EXMOE_BF16, st);
        Py_END_ALLOW_THREADS
        if (rc) return PyLong_FromLong(rc);
        return o ? Py_NewRef(a[6]) : THPVariable_Wrap(std::move(out));
    });
}

// set_entry_points(addresses in the loaded libexmoe.so, in the order of binding.py's list)
PyObject* set_entry_points(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 8) return PyErr_Format(PyExc_TypeError, "set_entry_points: 8 addresses");
    g_route = reinterpret_cast<decltype(g_route)>(PyLong_AsVoidPtr(a[0]));
    g_forward = reinterpret_cast<decltype(g_forward)>(PyLong_AsVoidPtr(a[1]));
    g_forward_host = reinterpret_cast<decltype(g_forward_host)>(PyLong_AsVoidPtr(a[2]));
    g_route_gated = reinterpret_cast<decltype(g_route_gated)>(PyLong_AsVoidPtr(a[3]));
    g_gate_logits = reinterpret_cast<decltype(g_gate_logits)>(PyLong_AsVoidPtr(a[4]));
    g_lora_plan_bytes = reinterpret_cast<decltype(g_lora_plan_bytes)>(PyLong_AsVoidPtr(a[5]));
    g_lora_plan = reinterpret_cast<decltype(g_lora_plan)>(PyLong_AsVoidPtr(a[6]));
    g_lora = reinterpret_cast<decltype(g_lora)>(PyLong_AsVoidPtr(a[7]));
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"route", reinterpret_cast<PyCFunction>(route), METH_FASTCALL, nullptr},
    {"forward", reinterpret_cast<PyCFunction>(forward), METH_FASTCALL, nullptr},
    {"forward_host", reinterpret_cast<PyCFunction>(forward_host), METH_FASTCALL, nullptr},
    {"route_gated", reinterpret_cast<PyCFunction>(route_gated), METH_FASTCALL, nullptr},
    {"gate_logits", reinterpret_cast<PyCFunction>(gate_logits), METH_FASTCALL, nullptr},
    {"lora_plan", reinterpret_cast<PyCFunction>(lora_plan), METH_FASTCALL, nullptr},
    {"lora", reinterpret_cast<PyCFunction>(lora), METH_FASTCALL, nullptr},
    {"set_entry_points", reinterpret_cast<PyCFunction>(set_entry_points), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_exmoe_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__exmoe_native(void) {
    s_d_model = PyUnicode_InternFromString("d_model");
    s_d_ff = PyUnicode_InternFromString("d_ff");
    s_experts = PyUnicode_InternFromString("num_experts");
    s_top_k = PyUnicode_InternFromString("top_k");
    s_group = PyUnicode_InternFromString("group_size");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_score = PyUnicode_InternFromString("score");
    s_num_groups = PyUnicode_InternFromString("num_groups");
    s_top_groups = PyUnicode_InternFromString("top_groups");
    s_group_score = PyUnicode_InternFromString("group_score");
    s_renormalise = PyUnicode_InternFromString("renormalise");
    s_scale = PyUnicode_InternFromString("scale");
    return PyModule_Create(&module);
}
