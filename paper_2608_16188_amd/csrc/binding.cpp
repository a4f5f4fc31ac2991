// Python calls of vmoe_train.h (module _train). A launch takes a few
// microseconds on the host, which small calls wait for: argument checks and
// marshalling in Python cost 5 to 8 us a call, here less than one.
//
// Every function takes its C call's arguments in order (tensors or None; a shape
// as the ctypes structure; the stream as None, a handle or an object with
// .cuda_stream) and returns the status. A tensor of the wrong type, layout,
// device (a launch's are on the current GPU, a plan's on one) or size raises ValueError before anything is called.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <exception>
#include <vector>

#include "../../include/vmoe_train.h"

namespace {

struct Refused {};  // a Python error is set

constexpr at::ScalarType kF32 = at::kFloat, kBf16 = at::kBFloat16, kI32 = at::kInt, kU8 = at::kByte;

// An unknown vmoe_dtype stays the library's to refuse.
at::ScalarType scalar(int32_t dtype) { return dtype == VMOE_BF16 ? kBf16 : kF32; }

const at::Tensor& tensor_of(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: a tensor or None is wanted, got %s", name,
                     Py_TYPE(o)->tp_name);
        throw Refused();
    }
    return THPVariable_Unpack(o);
}

// The GPU that a call's tensors are on: that of the first of them.
constexpr int kNone = -1;
thread_local int gpu_of_call = kNone;

void check_gpu(const at::Tensor& t, const char* name) {
    const int gpu = t.device().index();
    if (gpu_of_call == kNone) gpu_of_call = gpu;
    if (gpu == gpu_of_call) return;
    PyErr_Format(PyExc_ValueError, "%s: a tensor on cuda:%d is wanted, as those before it, got one "
                 "on cuda:%d", name, gpu_of_call, gpu);
    throw Refused();
}

// Pointer of a contiguous tensor of `type` on the GPU with at least `numel`
// elements; NULL for None.
void* pointer(PyObject* o, const char* name, at::ScalarType type, int64_t numel) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor_of(o, name);
    if (t.scalar_type() != type || !t.is_cuda() || !t.is_contiguous() || t.numel() < numel) {
        PyErr_Format(PyExc_ValueError,
                     "%s: a contiguous %s tensor of at least %lld elements on the GPU is wanted, "
                     "got %s, %lld elements%s%s",
                     name, c10::toString(type), static_cast<long long>(numel),
                     c10::toString(t.scalar_type()), static_cast<long long>(t.numel()),
                     t.is_contiguous() ? "" : ", not contiguous", t.is_cuda() ? "" : ", not on the GPU");
        throw Refused();
    }
    check_gpu(t, name);
    return t.data_ptr();
}

float* f32(void* p) { return static_cast<float*>(p); }

struct Workspace {
    void* p = nullptr;
    size_t bytes = 0;
    explicit Workspace(PyObject* o) {
        if (o == Py_None) return;
        const at::Tensor& t = tensor_of(o, "workspace");
        if (!t.is_cuda() || !t.is_contiguous()) {
            PyErr_SetString(PyExc_ValueError, "workspace: a contiguous tensor on the GPU is wanted");
            throw Refused();
        }
        check_gpu(t, "workspace");
        p = t.data_ptr();
        bytes = t.nbytes();
    }
};

// The call's stream, which comes after its tensors: they have to be on the current
// GPU, as the launch will be.
void* stream_of(PyObject* o) {
    const bool current = o == Py_None;
    if (gpu_of_call != kNone || current) {
        const c10::hip::HIPStream s = c10::hip::getCurrentHIPStream();
        if (gpu_of_call != kNone && gpu_of_call != s.device_index()) {
            PyErr_Format(PyExc_ValueError, "tensors on cuda:%d, while the current GPU is cuda:%d",
                         gpu_of_call, static_cast<int>(s.device_index()));
            throw Refused();
        }
        if (current) return s.stream();
    }
    PyObject* handle = PyObject_GetAttrString(o, "cuda_stream");
    if (handle == nullptr) {
        PyErr_Clear();
        handle = o;
        Py_INCREF(o);
    }
    void* s = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    if (s == nullptr && PyErr_Occurred()) throw Refused();
    return s;
}

// Memory of a ctypes structure, told from others (of the same size) by its
// class's name.
template <typename T>
struct Shape {
    Py_buffer view;
    Shape(PyObject* o, const char* name) {
        if (strcmp(Py_TYPE(o)->tp_name, name) != 0) {
            PyErr_Format(PyExc_TypeError, "shape: a %s is wanted, got %s", name,
                         Py_TYPE(o)->tp_name);
            throw Refused();
        }
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Refused();
        if (view.len != static_cast<Py_ssize_t>(sizeof(T))) {
            PyBuffer_Release(&view);
            PyErr_SetString(PyExc_TypeError, "shape: not the structure of this call");
            throw Refused();
        }
    }
    ~Shape() { PyBuffer_Release(&view); }
    Shape(const Shape&) = delete;
    Shape& operator=(const Shape&) = delete;
    const T* operator->() const { return static_cast<const T*>(view.buf); }
    const T* get() const { return static_cast<const T*>(view.buf); }
};

double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused();
    return v;
}
long long whole(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused();
    return v;
}
void* plan_of(PyObject* o) { return pointer(o, "plan", kU8, 0); }

// Argument count, C++ exceptions to Python ones, status to int.
template <typename F>
PyObject* guarded(Py_ssize_t got, Py_ssize_t wanted, F f) {
    if (got != wanted) {
        PyErr_Format(PyExc_TypeError, "%zd arguments are wanted, got %zd", wanted, got);
        return nullptr;
    }
    gpu_of_call = kNone;
    try {
        return PyLong_FromLong(f());
    } catch (const Refused&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

PyObject* block_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 14, [&] {
        const Shape<vmoe_norm_shape> s(a[0], "NormShape");
        const at::ScalarType act = scalar(s->dtype), res = scalar(s->stream_dtype);
        const int64_t d = s->d_model, rows = s->n_tokens, all = rows * d;
        void* const p[] = {
            pointer(a[1], "x", res, all), pointer(a[2], "y", act, all),
            pointer(a[3], "post_weight", act, d), pointer(a[4], "post_bias", act, d),
            pointer(a[5], "gate", act, s->n_groups * d), pointer(a[6], "row_scale", kF32, rows),
            pointer(a[7], "pre_weight", act, d), pointer(a[8], "pre_bias", act, d),
            pointer(a[9], "x_out", res, all), pointer(a[10], "h", act, all),
            pointer(a[11], "post_stats", kF32, 2 * rows),
            pointer(a[12], "pre_stats", kF32, 2 * rows)};
        return vmoe_block_norm_fwd(s.get(), p[0], p[1], p[2], p[3], p[4], f32(p[5]), p[6], p[7],
                                   p[8], p[9], f32(p[10]), f32(p[11]), stream_of(a[13]));
    });
}

PyObject* block_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 21, [&] {
        const Shape<vmoe_norm_shape> s(a[0], "NormShape");
        const at::ScalarType act = scalar(s->dtype), res = scalar(s->stream_dtype);
        const int64_t d = s->d_model, rows = s->n_tokens, all = rows * d;
        void* const p[] = {
            pointer(a[1], "dx_out", res, all), pointer(a[2], "dh", scalar(s->dh_dtype), all),
            pointer(a[3], "x_out", res, all), pointer(a[4], "y", act, all),
            pointer(a[5], "post_weight", act, d), pointer(a[6], "post_bias", act, d),
            pointer(a[7], "gate", act, s->n_groups * d), pointer(a[8], "row_scale", kF32, rows),
            pointer(a[9], "pre_weight", act, d), pointer(a[10], "post_stats", kF32, 2 * rows),
            pointer(a[11], "pre_stats", kF32, 2 * rows), pointer(a[12], "dx", res, all),
            pointer(a[13], "dy", act, all), pointer(a[14], "dpost_weight", kF32, d),
            pointer(a[15], "dpost_bias", kF32, d), pointer(a[16], "dgate", kF32, s->n_groups * d),
            pointer(a[17], "dpre_weight", kF32, d), pointer(a[18], "dpre_bias", kF32, d)};
        const Workspace ws(a[19]);
        return vmoe_block_norm_bwd(s.get(), p[0], p[1], p[2], p[3], p[4], p[5], p[6], f32(p[7]),
                                   p[8], f32(p[9]), f32(p[10]), p[11], p[12], f32(p[13]),
                                   f32(p[14]), f32(p[15]), f32(p[16]), f32(p[17]), ws.p, ws.bytes,
                                   stream_of(a[20]));
    });
}

PyObject* load_balance_loss(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 15, [&] {
        const Shape<vmoe_shape> s(a[0], "Shape");
        const int64_t rows = s->n_tokens, E = s->n_experts, G = s->n_groups;
        void* const p[] = {
            pointer(a[1], "logits", kF32, rows * E), pointer(a[2], "logit_bias", kF32, E),
            pointer(a[3], "noise", kF32, rows * E), pointer(a[4], "probs", kF32, rows * E),
            pointer(a[5], "expert_idx", kI32, rows * s->k), pointer(a[6], "token_mask", kU8, rows),
            pointer(a[9], "losses", kF32, 2 * G), pointer(a[10], "demand", kI32, G * E),
            pointer(a[11], "mean_probs", kF32, G * E), pointer(a[12], "dlogits", kF32, rows * E)};
        const Workspace ws(a[13]);
        const float w_balance = static_cast<float>(real(a[7])), w_z = static_cast<float>(real(a[8]));
        return vmoe_load_balance_loss(s.get(), f32(p[0]), f32(p[1]), f32(p[2]), f32(p[3]),
                                      static_cast<int32_t*>(p[4]), static_cast<uint8_t*>(p[5]),
                                      w_balance, w_z, f32(p[6]), static_cast<int32_t*>(p[7]),
                                      f32(p[8]), f32(p[9]), ws.p, ws.bytes, stream_of(a[14]));
    });
}

// (plan or None, chunks, grad_scale, max_norm, clip, workspace, stream)
PyObject* grad_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 7, [&] {
        const Workspace ws(a[5]);
        void *const plan = plan_of(a[0]), *const clip = pointer(a[4], "clip", kF32, 2);
        return vmoe_grad_norm(plan, whole(a[1]), real(a[2]), real(a[3]), f32(clip), ws.p,
                              ws.bytes, stream_of(a[6]));
    });
}

// (plan or None, chunks, lr, beta1, beta2, eps, grad_scale, step, seed, clip, stream)
PyObject* adamw(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 11, [&] {
        vmoe_adamw_hyper h = {};
        h.lr = real(a[2]);
        h.beta1 = real(a[3]);
        h.beta2 = real(a[4]);
        h.eps = real(a[5]);
        h.grad_scale = real(a[6]);
        h.step = whole(a[7]);
        const long long seed = whole(a[8]);
        if (seed < 0 || seed > 0xFFFFFFFFLL) {
            PyErr_Format(PyExc_ValueError, "seed: a number of 32 bits is wanted, got %lld", seed);
            throw Refused();
        }
        h.seed = static_cast<uint32_t>(seed);
        void *const plan = plan_of(a[0]), *const clip = pointer(a[9], "clip", kF32, 2);
        return vmoe_adamw(plan, whole(a[1]), &h, f32(clip), stream_of(a[10]));
    });
}

// A new reference, released at the end of its scope.
struct Held {
    PyObject* o;
    explicit Held(PyObject* p) : o(p) {
        if (o == nullptr) throw Refused();
    }
    ~Held() { Py_DECREF(o); }
    Held(const Held&) = delete;
    Held& operator=(const Held&) = delete;
};

int32_t float_type(const at::Tensor& t, const char* name) {
    if (t.scalar_type() != kF32 && t.scalar_type() != kBf16) {
        PyErr_Format(PyExc_ValueError, "%s: a float32 or bfloat16 tensor is wanted, got %s", name,
                     c10::toString(t.scalar_type()));
        throw Refused();
    }
    return t.scalar_type() == kF32 ? VMOE_F32 : VMOE_BF16;
}

// Pointer of o.name, a tensor of exactly `numel` elements (or None).
void* sized(PyObject* o, const char* name, at::ScalarType type, int64_t numel) {
    const Held h(PyObject_GetAttrString(o, name));
    void* p = pointer(h.o, name, type, numel);
    if (h.o != Py_None && tensor_of(h.o, name).numel() != numel) {
        PyErr_Format(PyExc_ValueError, "%s: %lld elements are wanted, got %lld", name,
                     static_cast<long long>(numel),
                     static_cast<long long>(tensor_of(h.o, name).numel()));
        throw Refused();
    }
    return p;
}

double real_of(PyObject* o, const char* name) {
    const Held h(PyObject_GetAttrString(o, name));
    return real(h.o);
}

// One AdamWTensor; the element after it, rounded up to a state block, to `next`.
vmoe_adamw_tensor tensor_entry(PyObject* o, uint64_t& next) {
    vmoe_adamw_tensor t = {};
    const Held param(PyObject_GetAttrString(o, "param")), grad(PyObject_GetAttrString(o, "grad"));
    const Held m(PyObject_GetAttrString(o, "m")), index0(PyObject_GetAttrString(o, "index0"));
    const at::Tensor& p = tensor_of(param.o, "param");
    const at::Tensor& g = tensor_of(grad.o, "grad");
    const bool bits8 = tensor_of(m.o, "m").scalar_type() == kU8;
    const at::ScalarType state = bits8 ? kU8 : kF32;
    t.n = p.numel();
    const int64_t blocks = (t.n + 127) / 128;
    t.param_dtype = float_type(p, "param");
    t.grad_dtype = float_type(g, "grad");
    t.state = bits8 ? VMOE_STATE_8BIT : VMOE_STATE_F32;
    t.param = sized(o, "param", p.scalar_type(), t.n);
    t.grad = sized(o, "grad", g.scalar_type(), t.n);
    t.m = sized(o, "m", state, t.n);
    t.v = sized(o, "v", state, t.n);
    t.master = static_cast<float*>(sized(o, "master", kF32, t.n));
    t.m_scale = static_cast<uint8_t*>(sized(o, "m_scale", kU8, blocks));
    t.v_scale = static_cast<uint8_t*>(sized(o, "v_scale", kU8, blocks));
    t.lr_mult = real_of(o, "lr_mult");
    t.weight_decay = real_of(o, "weight_decay");
    if (index0.o != Py_None) {
        next = PyLong_AsUnsignedLongLong(index0.o);
        if (PyErr_Occurred()) throw Refused();
    }
    t.index0 = next;
    next += static_cast<uint64_t>(blocks) * 128;
    return t;
}

// (list of AdamWTensor) -> (status, chunks, plan as bytes)
PyObject* adamw_plan(PyObject*, PyObject* list) {
    gpu_of_call = kNone;
    try {
        const Held items(PySequence_Fast(list, "tensors: a sequence is wanted"));
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(items.o);
        std::vector<vmoe_adamw_tensor> t(static_cast<size_t>(n));
        uint64_t next = 0;
        for (Py_ssize_t i = 0; i < n; ++i)
            t[i] = tensor_entry(PySequence_Fast_GET_ITEM(items.o, i), next);
        const int32_t count = static_cast<int32_t>(n);
        const int64_t chunks = vmoe_adamw_plan_chunks(t.data(), count);
        const size_t bytes = chunks > 0 ? static_cast<size_t>(chunks) * VMOE_ADAMW_PLAN_ENTRY_BYTES : 0;
        std::vector<uint64_t> plan(bytes / 8);
        const vmoe_status st = vmoe_adamw_plan(t.data(), count, plan.data(), bytes);
        return Py_BuildValue("iLy#", static_cast<int>(st), static_cast<long long>(chunks),
                             reinterpret_cast<const char*>(plan.data()),
                             static_cast<Py_ssize_t>(bytes));
    } catch (const Refused&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// (codes, scale, is_signed, out, stream)
PyObject* adamw_state_values(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 5, [&] {
        const int is_signed = PyObject_IsTrue(a[2]);
        if (is_signed < 0) throw Refused();
        const int64_t count = tensor_of(a[0], "codes").numel();
        const at::Tensor& out = tensor_of(a[3], "out");
        const int32_t dtype = float_type(out, "out");
        void* const p[] = {pointer(a[0], "codes", kU8, count),
                           pointer(a[1], "scale", kU8, (count + 127) / 128),
                           pointer(a[3], "out", out.scalar_type(), count)};
        return vmoe_adamw_state_values(static_cast<uint8_t*>(p[0]), static_cast<uint8_t*>(p[1]),
                                       is_signed, count, p[2], dtype, stream_of(a[4]));
    });
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL,
            nullptr};
}

PyMethodDef methods[] = {method<block_norm_fwd>("block_norm_fwd"),
                         method<block_norm_bwd>("block_norm_bwd"),
                         method<load_balance_loss>("load_balance_loss"),
                         method<grad_norm>("grad_norm"),
                         method<adamw>("adamw"),
                         {"adamw_plan", adamw_plan, METH_O, nullptr},
                         method<adamw_state_values>("adamw_state_values"),
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_train", "Calls of vmoe_train.h", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__train() { return PyModule_Create(&module); }
