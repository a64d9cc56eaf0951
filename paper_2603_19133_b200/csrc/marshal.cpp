// Argument marshalling of the hot calls: torch tensors to the plain pointers and sizes of the C-ABI
// (include/picospec.h), with the checks a caller relies on (CUDA tensor, dtype, shape, contiguity).
// A call has 10 to 20 tensors; done in Python the checks, the ctypes objects and the foreign call
// cost 8 to 14 us of host time, as much as the kernel launches behind them.  The library itself stays
// free of torch and Python: it is opened here by path.
#include <Python.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/core/AutogradState.h>
#include <c10/cuda/CUDAStream.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <climits>
#include <initializer_list>
#include <memory>
#include <string>
#include <vector>

#include "../../include/picospec.h"

namespace {

struct Refused {
    std::string why;
};

struct Api {
    decltype(&picospec_compress) compress;
    decltype(&picospec_verify) verify;
    decltype(&picospec_verify_range) verify_range;
    decltype(&picospec_residual_sample) residual_sample;
    decltype(&picospec_target_topk) target_topk;
    decltype(&picospec_edge_resample) edge_resample;
    decltype(&picospec_wire_pack) wire_pack;
    decltype(&picospec_wire_unpack) wire_unpack;
    decltype(&picospec_distill) distill;
    decltype(&picospec_sample) sample;
    decltype(&picospec_penalize) penalize;
    decltype(&picospec_penalize_grad) penalize_grad;
    decltype(&picospec_rules_workspace) rules_workspace;
    decltype(&picospec_append) append;
    decltype(&picospec_grad_norm) grad_norm;
    decltype(&picospec_clip_grad) clip_grad;
    decltype(&picospec_grad_workspace) grad_workspace;
    void* handle;
} api;

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) throw Refused{"expected a tensor"};
    return THPVariable_Unpack(o);
}

// data pointer of a contiguous CUDA tensor of the given type (and shape, if given); None is null
void* ptr(PyObject* o, at::ScalarType type, const std::initializer_list<int64_t>* shape) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o);
    if (!t.is_cuda()) throw Refused{"picospec takes CUDA tensors only (there is no CPU path)"};
    if (t.scalar_type() != type)
        throw Refused{std::string("expected dtype ") + c10::toString(type) + ", got " + c10::toString(t.scalar_type())};
    if (shape && !t.sizes().equals(at::IntArrayRef(shape->begin(), shape->size()))) {
        std::string want;
        for (int64_t d : *shape) want += (want.empty() ? "" : ", ") + std::to_string(d);
        std::string got;
        for (int64_t d : t.sizes()) got += (got.empty() ? "" : ", ") + std::to_string(d);
        throw Refused{"expected shape (" + want + "), got (" + got + ")"};
    }
    if (!t.is_contiguous()) throw Refused{"expected a contiguous tensor"};
    return t.data_ptr();
}
int* i32(PyObject* o, std::initializer_list<int64_t> shape) { return (int*)ptr(o, at::kInt, &shape); }
float* f32(PyObject* o, std::initializer_list<int64_t> shape) { return (float*)ptr(o, at::kFloat, &shape); }

// [B, R, V] logits with a contiguous vocabulary and uniformly pitched rows
struct Logits {
    const void* p;
    picospec_dtype dtype;
    int64_t B, R, V, pitch;
    explicit Logits(PyObject* o) : Logits(tensor(o)) {}
    explicit Logits(const at::Tensor& t) {
        if (!t.is_cuda() || t.dim() != 3 || t.stride(2) != 1)
            throw Refused{"logits must be a CUDA tensor [B, R, V] with contiguous vocabulary"};
        B = t.size(0); R = t.size(1); V = t.size(2);
        pitch = R > 1 ? t.stride(1) : (B > 1 ? t.stride(0) : V);
        if ((R > 1 && B > 1 && t.stride(0) != R * pitch) || pitch < V) throw Refused{"rows must be uniformly pitched"};
        if (t.scalar_type() == at::kFloat) dtype = PICOSPEC_F32;
        else if (t.scalar_type() == at::kBFloat16) dtype = PICOSPEC_BF16;
        else throw Refused{"logits must be float32 or bfloat16"};
        p = t.data_ptr();
    }
};

long long integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{""};
    return v;
}
double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused{""};
    return v;
}
picospec_ctx* context(PyObject* o) { return (picospec_ctx*)(uintptr_t)PyLong_AsVoidPtr(o); }
void* stream() { return (void*)c10::cuda::getCurrentCUDAStream().stream(); }
int64_t last_size(PyObject* o) {
    const at::Tensor& t = tensor(o);
    if (t.dim() < 1) throw Refused{"expected a tensor with at least one dimension"};
    return t.size(-1);
}

// Runs `body(args)` (which returns the library's code) without the interpreter lock around the call
// itself; a refused argument becomes a ValueError.
template <typename F> PyObject* guarded(Py_ssize_t n, Py_ssize_t want, F&& body) {
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
        return nullptr;
    }
    try {
        return PyLong_FromLong(body());
    } catch (const Refused& r) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, r.why.c_str());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
// The same for a body that returns (the library's code, a result to return where the code is PICOSPEC_OK): a caller that passes None for it has the
// result made here, which costs half of what it does in Python.
template <typename F> PyObject* guarded_result(Py_ssize_t n, Py_ssize_t want, F&& body) {
    at::Tensor result;
    PyObject* code = guarded(n, want, [&] { return body(result); });
    if (!code || PyLong_AsLong(code) != PICOSPEC_OK) return code;
    Py_DECREF(code);
    return THPVariable_Wrap(std::move(result));
}
// `outputs`: what the call writes.  Autograd is told, so that a backward pass which saved one of them for what it held before raises.
template <typename F> int unlocked(std::initializer_list<PyObject*> outputs, F&& call) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    if (rc == PICOSPEC_OK)
        for (PyObject* o : outputs)
            if (o != Py_None && !tensor(o).is_inference()) tensor(o).unsafeGetTensorImpl()->bump_version();
    return rc;
}

// context, logits, temperature, top_k, top_p, k_max, u_draft, q_idx, q_prob, q_count, draft_tok
PyObject* py_compress(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 11, [&] {
        picospec_ctx* ctx = context(a[0]);
        const Logits l(a[1]);
        const int64_t B = l.B, G = l.R, K = integer(a[5]);
        const float* T = f32(a[2], {B});
        const int top_k = (int)integer(a[3]);
        const float top_p = (float)real(a[4]);
        int* idx = i32(a[7], {B, G, K});
        float* prob = f32(a[8], {B, G, K});
        int* count = i32(a[9], {B, G});
        const float* u = f32(a[6], {B, G});
        int* tok = i32(a[10], {B, G});
        void* s = stream();
        return unlocked({a[7], a[8], a[9], a[10]}, [&] {
            return api.compress(ctx, l.p, l.dtype, (int)B, (int)G, (int)l.V, l.pitch, T, top_k, top_p, (int)K, idx, prob, count,
                                u, tok, s);
        });
    });
}

// context, logits, temperature, draft_tok, q_idx, q_prob, q_count, u_accept, u_resample, accept_len, p_draft,
// resid_mass, borderline_count, token
PyObject* py_verify(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 14, [&] {
        picospec_ctx* ctx = context(a[0]);
        const Logits l(a[1]);
        const int64_t B = l.B, G = l.R - 1, K = last_size(a[4]);
        const float* T = f32(a[2], {B});
        const int* dt = i32(a[3], {B, G});
        const int* idx = i32(a[4], {B, G, K});
        const float* prob = f32(a[5], {B, G, K});
        const int* count = i32(a[6], {B, G});
        const float* ua = f32(a[7], {B, G});
        int* alen = i32(a[9], {B});
        float* pd = f32(a[10], {B, G});
        float* rm = f32(a[11], {B, G});
        int* bc = i32(a[12], {1});
        const float* ur = f32(a[8], {B, 2});
        int* tok = i32(a[13], {B});
        void* s = stream();
        return unlocked({a[9], a[10], a[11], a[12], a[13]}, [&] {
            return api.verify(ctx, l.p, l.dtype, (int)B, (int)G, (int)l.V, l.pitch, T, dt, idx, prob, count, (int)K, ua, alen, pd,
                              rm, bc, ur, tok, s);
        });
    });
}

// context, logits, temperature, gamma, r0, r1, state_in, draft_tok, q_idx, q_prob, q_count, u_accept, u_resample,
// accept_len, p_draft, resid_mass, borderline_count, token, state
PyObject* py_verify_range(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 19, [&] {
        picospec_ctx* ctx = context(a[0]);
        const Logits l(a[1]);
        const int64_t B = l.B, G = l.R - 1, K = last_size(a[8]);
        const float* T = f32(a[2], {B});
        const int* gamma = i32(a[3], {B});
        const int r0 = (int)integer(a[4]), r1 = (int)integer(a[5]);
        const int* state_in = i32(a[6], {B});
        const int* dt = i32(a[7], {B, G});
        const int* idx = i32(a[8], {B, G, K});
        const float* prob = f32(a[9], {B, G, K});
        const int* count = i32(a[10], {B, G});
        const float* ua = f32(a[11], {B, G});
        int* alen = i32(a[13], {B});
        float* pd = f32(a[14], {B, G});
        float* rm = f32(a[15], {B, G});
        int* bc = i32(a[16], {1});
        const float* ur = f32(a[12], {B, 2});
        int* tok = i32(a[17], {B});
        int* state = i32(a[18], {B});
        void* s = stream();
        return unlocked({a[13], a[14], a[15], a[16], a[17], a[18]}, [&] {
            return api.verify_range(ctx, l.p, l.dtype, (int)B, (int)G, (int)l.V, l.pitch, T, gamma, r0, r1, state_in, dt, idx,
                                    prob, count, (int)K, ua, alen, pd, rm, bc, ur, tok, state, s);
        });
    });
}

// context, logits, temperature, pos, q_idx, q_prob, q_count, u_resample, token, mass
PyObject* py_residual_sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 10, [&] {
        picospec_ctx* ctx = context(a[0]);
        const Logits l(a[1]);
        const int64_t B = l.B, G = l.R - 1, K = G > 0 ? last_size(a[4]) : 1;
        const float* T = f32(a[2], {B});
        const int* pos = i32(a[3], {B});
        const int* idx = (const int*)ptr(a[4], at::kInt, nullptr);
        const float* prob = (const float*)ptr(a[5], at::kFloat, nullptr);
        const int* count = (const int*)ptr(a[6], at::kInt, nullptr);
        const float* ur = f32(a[7], {B, 2});
        int* tok = i32(a[8], {B});
        float* mass = f32(a[9], {B});
        void* s = stream();
        return unlocked({a[8], a[9]}, [&] {
            return api.residual_sample(ctx, l.p, l.dtype, (int)B, (int)G, (int)l.V, l.pitch, T, pos, idx, prob, count, (int)K, ur,
                                       tok, mass, s);
        });
    });
}

// context, logits, temperature, pos, k, p_idx, p_prob, p_count
PyObject* py_target_topk(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 8, [&] {
        picospec_ctx* ctx = context(a[0]);
        const Logits l(a[1]);
        const int64_t B = l.B, K = integer(a[4]);
        int* idx = i32(a[5], {B, K});
        float* prob = f32(a[6], {B, K});
        int* count = i32(a[7], {B});
        const float* T = f32(a[2], {B});
        const int* pos = i32(a[3], {B});
        void* s = stream();
        return unlocked({a[5], a[6], a[7]}, [&] {
            return api.target_topk(ctx, l.p, l.dtype, (int)B, (int)l.R, (int)l.V, l.pitch, T, pos, (int)K, idx, prob, count, s);
        });
    });
}

// context, logits, temperature, pos, p_idx, p_prob, p_count, u, token, mass
PyObject* py_edge_resample(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 10, [&] {
        picospec_ctx* ctx = context(a[0]);
        const Logits l(a[1]);
        const int64_t B = l.B, K = last_size(a[4]);
        int* tok = i32(a[8], {B});
        float* mass = f32(a[9], {B});
        const float* T = f32(a[2], {B});
        const int* pos = i32(a[3], {B});
        const int* idx = i32(a[4], {B, K});
        const float* prob = f32(a[5], {B, K});
        const int* count = i32(a[6], {B});
        const float* u = f32(a[7], {B});
        void* s = stream();
        return unlocked({a[8], a[9]}, [&] {
            return api.edge_resample(ctx, l.p, l.dtype, (int)B, (int)l.R, (int)l.V, l.pitch, T, pos, idx, prob, count, (int)K, u,
                                     tok, mass, s);
        });
    });
}

// context, q_idx, q_prob, q_count, rows, K, prob_type, buf, bytes_out
PyObject* py_wire_pack(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 9, [&] {
        picospec_ctx* ctx = context(a[0]);
        const int* idx = (const int*)ptr(a[1], at::kInt, nullptr);
        const float* prob = (const float*)ptr(a[2], at::kFloat, nullptr);
        const int* count = (const int*)ptr(a[3], at::kInt, nullptr);
        const int R = (int)integer(a[4]), K = (int)integer(a[5]), type = (int)integer(a[6]);
        void* buf = ptr(a[7], at::kByte, nullptr);
        const long long capacity = tensor(a[7]).numel();
        const std::initializer_list<int64_t> one = {1};
        long long* bytes = (long long*)ptr(a[8], at::kLong, &one);
        void* s = stream();
        return unlocked({a[7], a[8]}, [&] { return api.wire_pack(ctx, idx, prob, count, R, K, type, buf, capacity, bytes, s); });
    });
}

// context, buf, nbytes, rows, K, q_idx, q_prob, q_count
PyObject* py_wire_unpack(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 8, [&] {
        picospec_ctx* ctx = context(a[0]);
        const void* buf = ptr(a[1], at::kByte, nullptr);
        const long long nbytes = integer(a[2]);
        const int64_t R = integer(a[3]), K = integer(a[4]);
        int* idx = i32(a[5], {R, K});
        float* prob = f32(a[6], {R, K});
        int* count = i32(a[7], {R});
        void* s = stream();
        return unlocked({a[5], a[6], a[7]}, [&] { return api.wire_unpack(ctx, buf, nbytes, (int)R, (int)K, idx, prob, count, s); });
    });
}

// For calls that take the context's device: every tensor has to be there, and the stream is that device's current one.
struct Device {
    int64_t index;
    explicit Device(PyObject* o) : index(integer(o)) {}
    void check(std::initializer_list<PyObject*> tensors) const {
        for (PyObject* o : tensors)
            if (o != Py_None && tensor(o).is_cuda() && tensor(o).get_device() != index)
                throw Refused{"expected tensors on the context's device, cuda:" + std::to_string(index)};
    }
    void* stream() const { return (void*)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)index).stream(); }
    // device memory for one call: torch hands it out again in the order of the current stream
    at::Tensor scratch(long long bytes) const {
        if (bytes <= 0) return at::Tensor();
        return at::empty({bytes}, at::TensorOptions().dtype(at::kByte).device(at::Device(at::kCUDA, (c10::DeviceIndex)index)));
    }
};
void* address(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
void written(const at::Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// `o` itself or, for None, new memory
at::Tensor given_or_empty(PyObject* o, at::IntArrayRef sizes, at::ScalarType type, const Device& dev) {
    if (o != Py_None) return tensor(o);
    return at::empty(sizes, at::TensorOptions().dtype(type).device(at::Device(at::kCUDA, (c10::DeviceIndex)dev.index)));
}
// `o` itself or, for None, new rows that lie to 16-byte boundaries as those of `like` do, with less than 16 bytes between them (`like` may be every
// hundredth row of something larger)
at::Tensor given_or_rows(PyObject* o, const Logits& like, const Device& dev) {
    const at::ScalarType type = like.dtype == PICOSPEC_F32 ? at::kFloat : at::kBFloat16;
    const int64_t between = (like.pitch - like.V) % (like.dtype == PICOSPEC_F32 ? 4 : 8);
    if (o != Py_None || between == 0) return given_or_empty(o, {like.B, like.R, like.V}, type, dev);
    return given_or_empty(o, {like.B, like.R, like.V + between}, type, dev).narrow(2, 0, like.V);
}

// context, device, logits, temperature, t_idx, t_prob, t_count, weight, tail, loss, grad
PyObject* py_distill(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 11, [&] {
        picospec_ctx* ctx = context(a[0]);
        const Device dev(a[1]);
        const Logits l(a[2]);
        const int64_t B = l.B, R = l.R, K = last_size(a[4]);
        const float* T = f32(a[3], {B});
        const int* idx = i32(a[4], {B, R, K});
        const float* prob = f32(a[5], {B, R, K});
        const int* count = i32(a[6], {B, R});
        const float* weight = f32(a[7], {B, R});
        const int tail = PyObject_IsTrue(a[8]);
        if (tail < 0) throw Refused{""};
        float* loss = f32(a[9], {B, R});
        void* grad = nullptr;
        int64_t pitch = l.V;
        if (a[10] != Py_None) {
            const Logits g(a[10]);
            if (g.dtype != l.dtype || g.B != B || g.R != R || g.V != l.V)
                throw Refused{"the gradient must have the type and the shape of the logits"};
            grad = const_cast<void*>(g.p);
            pitch = g.pitch;
        }
        dev.check({a[2], a[3], a[4], a[5], a[6], a[7], a[9], a[10]});
        void* s = dev.stream();
        return unlocked({a[9], a[10]}, [&] {
            return api.distill(ctx, l.p, l.dtype, (int)B, (int)R, (int)l.V, l.pitch, T, idx, prob, count, (int)K, tail, weight, loss,
                               grad, pitch, s);
        });
    });
}

// context, device, logits, temperature, u, top_k, top_p, min_p, token, prob, logprob, count
PyObject* py_sample(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 12, [&] {
        picospec_ctx* ctx = context(a[0]);
        const Device dev(a[1]);
        const Logits l(a[2]);
        const int64_t B = l.B, R = l.R;
        const float* T = f32(a[3], {B});
        const float* u = f32(a[4], {B, R, 2});
        const int* k = i32(a[5], {B});
        const float* p = f32(a[6], {B});
        const float* m = f32(a[7], {B});
        int* token = i32(a[8], {B, R});
        float* prob = f32(a[9], {B, R});
        float* logprob = f32(a[10], {B, R});
        int* count = i32(a[11], {B, R});
        dev.check({a[2], a[3], a[4], a[5], a[6], a[7], a[8], a[9], a[10], a[11]});
        void* s = dev.stream();
        return unlocked({a[8], a[9], a[10], a[11]}, [&] {
            return api.sample(ctx, l.p, l.dtype, (int)B, (int)R, (int)l.V, l.pitch, T, k, p, m, u, token, prob, logprob, count, s);
        });
    });
}

// Whether autograd follows a tensor, backward or forward: what is computed from it here would be a constant to it.
bool watched(const at::Tensor& t) {
    return (t.requires_grad() && at::GradMode::is_enabled()) || (c10::AutogradState::get_tls_state().get_fw_grad_mode() && t._fw_grad(0).defined());
}
void unwatched(std::initializer_list<PyObject*> tensors, const char* what, const char* instead) {
    for (PyObject* o : tensors)
        if (o != Py_None && watched(tensor(o))) throw Refused{std::string(what) + " goes past autograd: " + instead};
}

// int32 [rows, n] with contiguous rows at any pitch, 0 among them; rows < 0: any number of them
struct Rows {
    int* p = nullptr;
    int64_t rows = 0, n = 0, stride = 0;
    Rows(PyObject* o, const char* what, int64_t want_rows, bool written) {
        if (o == Py_None) return;
        const at::Tensor& t = tensor(o);
        if (!t.is_cuda()) throw Refused{"picospec takes CUDA tensors only (there is no CPU path)"};
        if (t.scalar_type() != at::kInt) throw Refused{std::string("expected dtype Int, got ") + c10::toString(t.scalar_type())};
        if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) throw Refused{std::string(what) + " must be two-dimensional with contiguous rows"};
        rows = t.size(0); n = t.size(1); stride = rows > 1 ? t.stride(0) : n;
        if (want_rows >= 0 && rows != want_rows)
            throw Refused{std::string(what) + " must have " + std::to_string(want_rows) + " rows, has " + std::to_string(rows)};
        if (stride < n && (written || stride != 0)) throw Refused{std::string(what) + " has rows that overlap"};
        if (n > INT_MAX || rows > INT_MAX) throw Refused{std::string(what) + " is too large"};
        p = (int*)t.data_ptr();
    }
};

// history, length, prompt_length, draft_tok, repetition, presence, frequency, bias_idx, bias, bias_count, mask, mask_row
constexpr int RULES = 12;
struct Rules : picospec_rules {
    Rules(PyObject* const* a, int64_t B, int64_t R, int64_t V) : picospec_rules{} {
        const Rows h(a[0], "history", B, false);
        history = h.p; history_stride = h.stride; capacity = (int)h.n;
        length = i32(a[1], {B});
        if ((a[0] == Py_None) != (a[1] == Py_None)) throw Refused{"history and length come together"};
        prompt_length = i32(a[2], {B});
        if (a[2] != Py_None && a[0] == Py_None) throw Refused{"prompt_length comes with history"};
        if (h.n == 0) {                 // (a history without a place: nothing to read, the lengths are still checked)
            static int none;
            history = a[0] == Py_None ? nullptr : &none;
        }
        draft_tok = R > 0 ? i32(a[3], {B, R - 1}) : nullptr;
        repetition = f32(a[4], {B}); presence = f32(a[5], {B}); frequency = f32(a[6], {B});
        if (a[7] != Py_None) {
            bias_k = (int)last_size(a[7]);
            bias_idx = i32(a[7], {B, bias_k});
            bias = f32(a[8], {B, bias_k});
            bias_count = i32(a[9], {B});
            if (a[8] == Py_None || a[9] == Py_None) throw Refused{"a bias has indices, values and counts"};
            if (bias_k == 0) bias_idx = nullptr;
        }
        if (a[11] != Py_None && a[10] == Py_None) throw Refused{"mask_row comes with mask"};
        if (a[10] != Py_None) {
            const at::Tensor& t = tensor(a[10]);
            if (a[11] == Py_None) {
                const int64_t words = last_size(a[10]);
                mask = i32(a[10], {B, R, words});
                mask_stride = words; mask_rows = (int)(B * R);
            } else {
                const Rows m(a[10], "mask", -1, false);
                mask = m.p; mask_stride = m.stride; mask_rows = (int)m.rows;
                mask_row = i32(a[11], {B, R});
                if (m.rows == 0 && B * R > 0) throw Refused{"mask has no rows"};
            }
            if (t.size(-1) < (V + 31) / 32) throw Refused{"mask has a word for every 32 entries"};
        }
    }
};

// context, device, logits, the rules, out (or None) -> out, or the code of an error
PyObject* py_penalize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded_result(n, RULES + 4, [&](at::Tensor& out) {
        picospec_ctx* ctx = context(a[0]);
        const Device dev(a[1]);
        unwatched({a[2], a[RULES + 3]}, "penalize", "use penalized, or detach");
        unwatched({a[7], a[8], a[9], a[11]}, "penalize", "its rules have no gradient, detach them");
        const Logits l(a[2]);
        const Rules rules(a + 3, l.B, l.R, l.V);
        for (int i = 2; i < n; ++i) dev.check({a[i]});
        out = given_or_rows(a[RULES + 3], l, dev);
        const Logits o(out);
        if (o.dtype != l.dtype || o.B != l.B || o.R != l.R || o.V != l.V) throw Refused{"the result must have the type and the shape of the logits"};
        const at::Tensor work = dev.scratch(api.rules_workspace(&rules, 0, (int)l.B, (int)l.R, (int)l.V));
        void* s = dev.stream();
        const int rc = unlocked({}, [&] {
            return api.penalize(ctx, l.p, l.dtype, (int)l.B, (int)l.R, (int)l.V, l.pitch, &rules, const_cast<void*>(o.p), o.pitch, address(work), s);
        });
        if (rc == PICOSPEC_OK) written(out);
        return rc;
    });
}

// context, device, grad, logits (or None), the rules, out (or None) -> out, or the code of an error
PyObject* py_penalize_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded_result(n, RULES + 5, [&](at::Tensor& out) {
        picospec_ctx* ctx = context(a[0]);
        const Device dev(a[1]);
        // (the logits' signs alone count: nothing of their derivative is lost)
        unwatched({a[2], a[RULES + 4], a[8], a[9], a[10], a[12]}, "penalize_grad", "it has no gradient of its own, detach");
        const Logits g(a[2]);
        const void* logits = nullptr;
        int64_t pitch = 0;
        if (a[3] != Py_None) {
            const Logits l(a[3]);
            if (l.dtype != g.dtype || l.B != g.B || l.R != g.R || l.V != g.V) throw Refused{"the gradient must have the type and the shape of the logits"};
            logits = l.p; pitch = l.pitch;
        }
        const Rules rules(a + 4, g.B, g.R, g.V);
        if (rules.repetition && !logits) throw Refused{"the gradient of a repetition penalty needs the logits"};
        for (int i = 2; i < n; ++i) dev.check({a[i]});
        out = given_or_rows(a[RULES + 4], g, dev);
        const Logits o(out);
        if (o.dtype != g.dtype || o.B != g.B || o.R != g.R || o.V != g.V) throw Refused{"the result must have the type and the shape of the gradient"};
        const at::Tensor work = dev.scratch(api.rules_workspace(&rules, 1, (int)g.B, (int)g.R, (int)g.V));
        void* s = dev.stream();
        const int rc = unlocked({}, [&] {
            return api.penalize_grad(ctx, g.p, g.dtype, (int)g.B, (int)g.R, (int)g.V, g.pitch, logits, pitch, &rules, const_cast<void*>(o.p), o.pitch, address(work), s);
        });
        if (rc == PICOSPEC_OK) written(out);
        return rc;
    });
}

// context, device, history, length, token, draft_tok, accept_len, length_out (or None) -> length_out, or the code of an error
PyObject* py_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded_result(n, 8, [&](at::Tensor& out_length) {
        picospec_ctx* ctx = context(a[0]);
        const Device dev(a[1]);
        if (a[2] == Py_None || a[3] == Py_None) throw Refused{"expected a tensor"};
        const Rows h(a[2], "history", -1, true);
        const int64_t B = h.rows;
        const int* length = i32(a[3], {B});
        const int* token = i32(a[4], {B});
        if ((a[5] == Py_None) != (a[6] == Py_None)) throw Refused{"draft_tok and accept_len come together"};
        if (a[4] == Py_None && a[5] == Py_None) throw Refused{"expected token, or draft_tok and accept_len"};
        const int64_t G = a[5] == Py_None ? 0 : last_size(a[5]);
        const int* draft = i32(a[5], {B, G});
        const int* accepted = i32(a[6], {B});
        int* out = i32(a[7], {B});
        dev.check({a[2], a[3], a[4], a[5], a[6], a[7]});
        out_length = given_or_empty(a[7], {B}, at::kInt, dev);
        if (!out) out = (int*)out_length.data_ptr();
        void* s = dev.stream();
        const int rc = unlocked({a[2]}, [&] {
            return api.append(ctx, h.p, h.stride, (int)h.n, (int)B, length, G ? draft : nullptr, (int)G, accepted, token, out, s);
        });
        if (rc == PICOSPEC_OK) written(out_length);
        return rc;
    });
}

// A list of gradients; None in it is passed over.  `written`: the call writes them, so none may be a parameter that autograd watches.  Nor may one
// be a function of others to it, as those of a backward pass with create_graph are (the norm of parameters, say, is one as it is now).
struct Grads {
    std::vector<picospec_tensor> t;
    std::vector<PyObject*> held;        // (with a reference: the list is the caller's own, who may change it while the interpreter
                                        // lock is released.  Of 30 tensors' storage instead: 9.5 us a call for 9.0)
    Grads(PyObject* sequence, const Device& dev, bool written) {
        struct List {
            PyObject* o;
            ~List() { Py_XDECREF(o); }
        } list{PySequence_Fast(sequence, "expected a list of tensors")};
        if (!list.o) throw Refused{""};
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(list.o);
        if (n > (1 << 24)) throw Refused{"too many tensors"};
        t.reserve((size_t)n);
        held.reserve((size_t)n);
        struct Undo {                   // (the destructor does not run where the constructor throws)
            std::vector<PyObject*>* held;
            ~Undo() {
                if (held) release(*held);
            }
        } undo{&held};
        for (Py_ssize_t i = 0; i < n; ++i) {
            PyObject* x = PySequence_Fast_GET_ITEM(list.o, i);
            if (x == Py_None) continue;
            const at::Tensor& g = tensor(x);
            if (written && g.requires_grad() && at::GradMode::is_enabled()) throw Refused{"a tensor that requires a gradient is not one: pass the parameters' .grad"};
            if (watched(g) && !(g.requires_grad() && g.is_leaf())) throw Refused{"a norm of gradients goes past autograd: detach them"};
            if (!g.is_cuda() || g.layout() != at::kStrided) throw Refused{"gradients must be dense CUDA tensors"};
            if (g.get_device() != dev.index) throw Refused{"expected tensors on the context's device, cuda:" + std::to_string(dev.index)};
            if (!g.is_non_overlapping_and_dense()) throw Refused{"gradients must lie in memory without gaps"};
            picospec_tensor y{g.data_ptr(), (long long)g.numel(), PICOSPEC_F32};
            if (g.scalar_type() == at::kBFloat16) y.dtype = PICOSPEC_BF16;
            else if (g.scalar_type() != at::kFloat) throw Refused{"gradients must be float32 or bfloat16"};
            t.push_back(y);
            held.push_back(x);
            Py_INCREF(x);
        }
        undo.held = nullptr;
    }
    Grads(const Grads&) = delete;
    ~Grads() { release(held); }
    static void release(const std::vector<PyObject*>& held) {
        for (PyObject* x : held) Py_DECREF(x);
    }
};

// context, device, grads, norm (or None) -> norm, or the code of an error
PyObject* py_grad_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded_result(n, 4, [&](at::Tensor& got) {
        picospec_ctx* ctx = context(a[0]);
        const Device dev(a[1]);
        const Grads g(a[2], dev, false);
        unwatched({a[3]}, "grad_norm", "it has no gradient, detach");
        float* norm = f32(a[3], {1});
        dev.check({a[3]});
        got = given_or_empty(a[3], {1}, at::kFloat, dev);
        if (!norm) norm = (float*)got.data_ptr();
        const at::Tensor work = dev.scratch(api.grad_workspace((int)g.t.size()));
        void* s = dev.stream();
        const int rc = unlocked({}, [&] { return api.grad_norm(ctx, g.t.data(), (int)g.t.size(), address(work), norm, s); });
        if (rc == PICOSPEC_OK) written(got);
        return rc;
    });
}

// context, device, grads, outs (or None), max_norm, norm_in (or None) -> norm_in or the norm, or the code of an error
PyObject* py_clip_grad(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded_result(n, 6, [&](at::Tensor& got) {
        picospec_ctx* ctx = context(a[0]);
        const Device dev(a[1]);
        const Grads g(a[2], dev, a[3] == Py_None);
        const Grads* o = &g;
        std::unique_ptr<Grads> own;
        if (a[3] != Py_None) {
            own.reset(new Grads(a[3], dev, true));
            o = own.get();
            if (o->t.size() != g.t.size()) throw Refused{"as many results as gradients are needed"};
            for (size_t i = 0; i < g.t.size(); ++i) {
                const at::Tensor &x = tensor(g.held[i]), &y = tensor(o->held[i]);
                if (!x.sizes().equals(y.sizes()) || !x.strides().equals(y.strides()) || x.scalar_type() != y.scalar_type())
                    throw Refused{"results must have the gradients' types, shapes and strides"};
            }
        }
        const float max_norm = (float)real(a[4]);
        unwatched({a[5]}, "clip_grad", "the norm has no gradient, detach it");
        const float* norm_in = f32(a[5], {1});
        dev.check({a[5]});
        // (every CTA reads it, while others write)
        for (size_t i = 0; norm_in && i < o->t.size(); ++i) {
            const char* p = (const char*)o->t[i].data;
            if ((const char*)norm_in < p + o->t[i].count * (o->t[i].dtype == PICOSPEC_BF16 ? 2 : 4) && p < (const char*)(norm_in + 1))
                throw Refused{"norm lies in a tensor that is written"};
        }
        got = given_or_empty(a[5], {1}, at::kFloat, dev);
        float* norm = norm_in ? nullptr : (float*)got.data_ptr();
        const at::Tensor work = dev.scratch(norm_in ? 0 : api.grad_workspace((int)g.t.size()));
        void* s = dev.stream();
        const int rc = unlocked({}, [&] {
            return api.clip_grad(ctx, g.t.data(), own ? o->t.data() : nullptr, (int)g.t.size(), max_norm, norm_in, address(work), norm, s);
        });
        if (rc == PICOSPEC_OK) {
            if (norm) written(got);
            for (PyObject* x : o->held) written(tensor(x));
        }
        return rc;
    });
}

// logits -> (B, R, V), checked: for calls that allocate their outputs from the shape
PyObject* py_logits(PyObject*, PyObject* const* a, Py_ssize_t n) {
    int64_t size[3] = {0, 0, 0};
    PyObject* ok = guarded(n, 1, [&] {
        const Logits l(a[0]);
        size[0] = l.B; size[1] = l.R; size[2] = l.V;
        return 0;
    });
    if (!ok) return nullptr;
    Py_DECREF(ok);
    return Py_BuildValue("(LLL)", (long long)size[0], (long long)size[1], (long long)size[2]);
}

// path of libpicospec.so
PyObject* py_open(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 1, [&] {
        const char* path = PyUnicode_AsUTF8(a[0]);
        if (!path) throw Refused{""};
        api.handle = dlopen(path, RTLD_NOW | RTLD_LOCAL);
        if (!api.handle) throw Refused{dlerror()};
        auto find = [&](const char* name) {
            void* f = dlsym(api.handle, name);
            if (!f) throw Refused{std::string("libpicospec.so lacks ") + name};
            return f;
        };
#define PICOSPEC_FIND(f) api.f = (decltype(api.f))find("picospec_" #f)
        PICOSPEC_FIND(compress);
        PICOSPEC_FIND(verify);
        PICOSPEC_FIND(verify_range);
        PICOSPEC_FIND(residual_sample);
        PICOSPEC_FIND(target_topk);
        PICOSPEC_FIND(edge_resample);
        PICOSPEC_FIND(wire_pack);
        PICOSPEC_FIND(wire_unpack);
        PICOSPEC_FIND(distill);
        PICOSPEC_FIND(sample);
        PICOSPEC_FIND(penalize);
        PICOSPEC_FIND(penalize_grad);
        PICOSPEC_FIND(rules_workspace);
        PICOSPEC_FIND(append);
        PICOSPEC_FIND(grad_norm);
        PICOSPEC_FIND(clip_grad);
        PICOSPEC_FIND(grad_workspace);
#undef PICOSPEC_FIND
        return 0;
    });
}

#define PICOSPEC_METHOD(f) {#f, (PyCFunction)(void (*)())py_##f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {PICOSPEC_METHOD(open),
                         PICOSPEC_METHOD(logits),
                         PICOSPEC_METHOD(compress),
                         PICOSPEC_METHOD(verify),
                         PICOSPEC_METHOD(verify_range),
                         PICOSPEC_METHOD(residual_sample),
                         PICOSPEC_METHOD(target_topk),
                         PICOSPEC_METHOD(edge_resample),
                         PICOSPEC_METHOD(wire_pack),
                         PICOSPEC_METHOD(wire_unpack),
                         PICOSPEC_METHOD(distill),
                         PICOSPEC_METHOD(sample),
                         PICOSPEC_METHOD(penalize),
                         PICOSPEC_METHOD(penalize_grad),
                         PICOSPEC_METHOD(append),
                         PICOSPEC_METHOD(grad_norm),
                         PICOSPEC_METHOD(clip_grad),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__marshal() { return PyModule_Create(&module); }
