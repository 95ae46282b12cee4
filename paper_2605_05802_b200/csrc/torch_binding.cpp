// Native half of binding.py: takes the tensors of a call apart and calls the C ABI.
//
// A gate call on a handful of groups lasts a few microseconds on the device; marshalled in
// Python (attribute look-ups, dtype comparisons and numel() per tensor, ctypes conversions)
// it cost 7-10 us of host time and the GPU waited for it.  Here a call is a few dozen plain
// loads.  The checks are those the C side cannot make: a tensor must live where the call
// dereferences it, have the declared element type, be contiguous and hold at least the
// elements the call reads or writes.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <string>
#include <vector>

#include "sr_gate.h"
#include "sr_probe.h"
#include "sr_tokens.h"
#include "sr_train.h"

namespace {

struct Raised {};                        // a Python exception has been set

[[noreturn]] void raise(PyObject* type, const std::string& text) {
    PyErr_SetString(type, text.c_str());
    throw Raised();
}

const char* dtype_name(c10::ScalarType t) {
    switch (t) {
        case c10::ScalarType::Int: return "torch.int32";
        case c10::ScalarType::Long: return "torch.int64";
        case c10::ScalarType::Byte: return "torch.uint8";
        case c10::ScalarType::Float: return "torch.float32";
        case c10::ScalarType::Double: return "torch.float64";
        case c10::ScalarType::Half: return "torch.float16";
        case c10::ScalarType::BFloat16: return "torch.bfloat16";
        default: return c10::toString(t);
    }
}

constexpr int64_t kAnySize = -1;
constexpr c10::ScalarType kAnyType = c10::ScalarType::Undefined;
PyObject* g_cuda_stream = nullptr;       // interned "cuda_stream"

// The positional arguments of one call, read one after the other.
struct Args {
    PyObject* const* at;

    const at::Tensor* tensor(const char* name) {
        PyObject* o = *at++;
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) raise(PyExc_TypeError, std::string(name) + " must be a tensor or None");
        return &THPVariable_Unpack(o);
    }
    static void* address(const at::Tensor* t, c10::ScalarType type, int64_t need, bool host, const char* name) {
        if (t == nullptr) return nullptr;
        if (type != kAnyType && t->scalar_type() != type)
            raise(PyExc_TypeError, std::string(name) + ": expected " + dtype_name(type) + ", got " + dtype_name(t->scalar_type()));
        if (!t->is_contiguous()) raise(PyExc_ValueError, std::string(name) + " must be contiguous");
        if (t->is_cuda() == host)
            raise(PyExc_ValueError, std::string(name) + " must be a " + (host ? "host" : "CUDA") + " tensor");
        if (need != kAnySize && t->numel() < need)
            raise(PyExc_ValueError, std::string(name) + " holds " + std::to_string(t->numel()) +
                                        " elements, the call writes or reads " + std::to_string(need));
        return t->data_ptr();
    }
    template <typename T>
    T* buffer(c10::ScalarType type, int64_t need, const char* name, bool host = false) {
        return static_cast<T*>(address(tensor(name), type, need, host, name));
    }
    // workspace / state / arena: any element type, its size in bytes
    void* scratch(const char* name, size_t& bytes) {
        const at::Tensor* t = tensor(name);
        bytes = t ? (size_t)t->numel() * t->element_size() : 0;
        return address(t, kAnyType, kAnySize, false, name);
    }
    int32_t integer() {                  // modulo 2^32, as a C caller's conversion
        PyObject* o = PyNumber_Index(*at++);
        if (o == nullptr) throw Raised();
        const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
        Py_DECREF(o);
        if (v == (unsigned long long)-1 && PyErr_Occurred()) throw Raised();
        return (int32_t)v;
    }
    double real() {                      // whatever float() takes
        PyObject* o = *at++;
        if (PyFloat_Check(o)) return PyFloat_AS_DOUBLE(o);
        PyObject* f = PyNumber_Float(o);
        if (f == nullptr) throw Raised();
        const double v = PyFloat_AS_DOUBLE(f);
        Py_DECREF(f);
        return v;
    }
    static void* handle(PyObject* stream) {
        PyObject* v = PyObject_GetAttr(stream, g_cuda_stream);
        if (v == nullptr) throw Raised();
        void* h = PyLong_AsVoidPtr(v);
        Py_DECREF(v);
        if (h == nullptr && PyErr_Occurred()) throw Raised();
        return h;
    }
    void* stream() {                     // None: the current stream of the current device
        PyObject* o = *at++;
        return o == Py_None ? c10::cuda::getCurrentCUDAStream().stream() : handle(o);
    }
    void* copy_stream() {
        PyObject* o = *at++;
        return o == Py_None ? nullptr : handle(o);
    }
};

struct Shape3 { int32_t G, N, stride; int64_t P; };
Shape3 group_shape(const at::Tensor* t, const char* name) {
    if (t == nullptr || t->dim() != 3) raise(PyExc_ValueError, std::string(name) + " must be [groups, N, stride]");
    Shape3 s{(int32_t)t->size(0), (int32_t)t->size(1), (int32_t)t->size(2), 0};
    s.P = (int64_t)s.N * (s.N - 1) / 2;
    return s;
}
void two_dims(const at::Tensor* t, const char* name, int32_t& G, int32_t& N) {
    if (t == nullptr || t->dim() != 2) raise(PyExc_ValueError, std::string(name) + " must be [groups, N]");
    G = (int32_t)t->size(0);
    N = (int32_t)t->size(1);
}

// Runs `body(args)` -> return code, without the GIL around the library call itself.
template <typename Body>
PyObject* guarded(PyObject* const* argv, Py_ssize_t argc, Py_ssize_t want, Body body) {
    if (argc != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, argc);
        return nullptr;
    }
    try {
        Args a{argv};
        const int rc = body(a);
        if (rc == SR_OK) Py_RETURN_NONE;
        return PyLong_FromLong(rc);
    } catch (const Raised&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}
template <typename Call>
int unlocked(Call call) {
    PyThreadState* st = PyEval_SaveThread();
    const int rc = call();
    PyEval_RestoreThread(st);
    return rc;
}

constexpr auto kI32 = c10::ScalarType::Int;
constexpr auto kI64 = c10::ScalarType::Long;
constexpr auto kU8 = c10::ScalarType::Byte;
constexpr auto kF32 = c10::ScalarType::Float;
constexpr auto kF64 = c10::ScalarType::Double;

// What every gate call has in common: inputs, threshold and the outputs of a batch.
struct GateCall {
    Shape3 d;
    int32_t *seqs, *lens, K, norm, *pair_dist, *pair_sum, *status;
    double threshold, *mean;
    uint8_t* stop;

    void inputs(Args& a, bool host) {
        const at::Tensor* s = a.tensor("seqs");
        d = group_shape(s, "seqs");
        seqs = static_cast<int32_t*>(Args::address(s, kI32, kAnySize, host, "seqs"));
        lens = a.buffer<int32_t>(kI32, (int64_t)d.G * d.N, "lens", host);
    }
    void setting(Args& a) {
        K = a.integer();
        threshold = a.real();
        norm = a.integer();
    }
    void outputs(Args& a, bool host) {
        pair_dist = a.buffer<int32_t>(kI32, d.G * d.P, "pair_dist", host);
        pair_sum = a.buffer<int32_t>(kI32, d.G, "pair_sum", host);
        mean = a.buffer<double>(kF64, d.G, "mean", host);
        stop = a.buffer<uint8_t>(kU8, d.G, "stop", host);
    }
};

PyObject* py_gate(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 12, [](Args& a) {
        GateCall c;
        c.inputs(a, false); c.setting(a); c.outputs(a, false);
        c.status = a.buffer<int32_t>(kI32, 1, "status");
        size_t bytes;
        void* ws = a.scratch("workspace", bytes);
        void* s = a.stream();
        return unlocked([&] { return sr_gate(c.seqs, c.lens, c.d.G, c.d.N, c.d.stride, c.K, c.threshold, c.norm, c.pair_dist, c.pair_sum, c.mean, c.stop, c.status, ws, bytes, s); });
    });
}

PyObject* py_gate_noalloc(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 11, [](Args& a) {
        GateCall c;
        c.inputs(a, false); c.setting(a); c.outputs(a, false);
        c.status = a.buffer<int32_t>(kI32, 1, "status");
        void* s = a.stream();
        return unlocked([&] { return sr_gate_noalloc(c.seqs, c.lens, c.d.G, c.d.N, c.d.stride, c.K, c.threshold, c.norm, c.pair_dist, c.pair_sum, c.mean, c.stop, c.status, s); });
    });
}

PyObject* py_gate_decide(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 13, [](Args& a) {
        GateCall c;
        c.inputs(a, false); c.setting(a); c.outputs(a, false);
        uint8_t* exact = a.buffer<uint8_t>(kU8, c.d.G, "exact");
        c.status = a.buffer<int32_t>(kI32, 1, "status");
        size_t bytes;
        void* ws = a.scratch("workspace", bytes);
        void* s = a.stream();
        return unlocked([&] { return sr_gate_decide(c.seqs, c.lens, c.d.G, c.d.N, c.d.stride, c.K, c.threshold, c.norm, c.pair_dist, c.pair_sum, c.mean, c.stop, exact, c.status, ws, bytes, s); });
    });
}

PyObject* py_gate_host(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 13, [](Args& a) {
        GateCall c;
        c.inputs(a, true); c.setting(a); c.outputs(a, true);
        c.status = a.buffer<int32_t>(kI32, 1, "status", true);
        size_t bytes;
        void* arena = a.scratch("arena", bytes);
        void* s = a.stream();
        void* cs = a.copy_stream();
        return unlocked([&] { return sr_gate_host(c.seqs, c.lens, c.d.G, c.d.N, c.d.stride, c.K, c.threshold, c.norm, c.pair_dist, c.pair_sum, c.mean, c.stop, c.status, arena, bytes, s, cs); });
    });
}

PyObject* py_gate_host_packed(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 15, [](Args& a) {
        GateCall c;
        int32_t* symbols = a.buffer<int32_t>(kI32, kAnySize, "symbols", true);
        const at::Tensor* rs = a.tensor("row_start");
        c.d.N = a.integer();
        c.d.stride = a.integer();
        const int64_t rows = rs ? rs->numel() - 1 : -1;
        if (rows < 0 || c.d.N == 0 || rows % c.d.N) raise(PyExc_ValueError, "row_start needs n_groups * N + 1 entries");
        c.d.G = (int32_t)(rows / c.d.N);
        c.d.P = (int64_t)c.d.N * (c.d.N - 1) / 2;
        int64_t* start = static_cast<int64_t*>(Args::address(rs, kI64, kAnySize, true, "row_start"));
        c.setting(a); c.outputs(a, true);
        c.status = a.buffer<int32_t>(kI32, 1, "status", true);
        size_t bytes;
        void* arena = a.scratch("arena", bytes);
        void* s = a.stream();
        void* cs = a.copy_stream();
        return unlocked([&] { return sr_gate_host_packed(symbols, start, c.d.G, c.d.N, c.d.stride, c.K, c.threshold, c.norm, c.pair_dist, c.pair_sum, c.mean, c.stop, c.status, arena, bytes, s, cs); });
    });
}

PyObject* py_incr_init(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 5, [](Args& a) {
        size_t bytes;
        void* state = a.scratch("state", bytes);
        const int32_t G = a.integer(), N = a.integer(), steps = a.integer();
        void* s = a.stream();
        return unlocked([&] { return sr_incr_init(state, bytes, G, N, steps, s); });
    });
}

PyObject* py_gate_step_incremental(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 10, [](Args& a) {
        GateCall c;
        size_t bytes;
        void* state = a.scratch("state", bytes);
        const at::Tensor* na = a.tensor("new_actions");
        two_dims(na, "new_actions", c.d.G, c.d.N);
        c.d.P = (int64_t)c.d.N * (c.d.N - 1) / 2;
        int32_t* actions = static_cast<int32_t*>(Args::address(na, kI32, kAnySize, false, "new_actions"));
        c.threshold = a.real();
        c.norm = a.integer();
        c.outputs(a, false);
        c.status = a.buffer<int32_t>(kI32, 1, "status");
        void* s = a.stream();
        return unlocked([&] { return sr_gate_step_incremental(state, bytes, actions, c.d.G, c.d.N, c.threshold, c.norm, c.pair_dist, c.pair_sum, c.mean, c.stop, c.status, s); });
    });
}

PyObject* py_gate_or_rule(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 10, [](Args& a) {
        const at::Tensor *mt = a.tensor("mean"), *lt = a.tensor("lens"), *dt = a.tensor("done");
        const int32_t N = a.integer(), K = a.integer();
        const double threshold = a.real(), tau_high = a.real();
        if (mt == nullptr || mt->dim() < 1) raise(PyExc_ValueError, "mean must be [groups]");
        const int32_t G = (int32_t)mt->size(0);
        const double* mean = static_cast<double*>(Args::address(mt, kF64, kAnySize, false, "mean"));
        const int32_t* lens = static_cast<int32_t*>(Args::address(lt, kI32, (int64_t)G * N, false, "lens"));
        const uint8_t* done = static_cast<uint8_t*>(Args::address(dt, kU8, (int64_t)G * N, false, "done"));
        double* tau = a.buffer<double>(kF64, G, "tau");
        uint8_t* stop = a.buffer<uint8_t>(kU8, G, "stop");
        void* s = a.stream();
        return unlocked([&] { return sr_gate_or_rule(mean, lens, done, G, N, K, threshold, tau_high, tau, stop, s); });
    });
}

PyObject* py_group_signals(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 8, [](Args& a) {
        GateCall c;
        c.inputs(a, false);
        const int32_t K = a.integer();
        double* upr = a.buffer<double>(kF64, c.d.G, "unique_prefix_ratio");
        double* uar = a.buffer<double>(kF64, c.d.G, "unique_action_ratio");
        double* ent = a.buffer<double>(kF64, c.d.G, "action_entropy");
        double* jac = a.buffer<double>(kF64, c.d.G, "bigram_jaccard_mean");
        void* s = a.stream();
        return unlocked([&] { return sr_group_signals(c.seqs, c.lens, c.d.G, c.d.N, c.d.stride, K, upr, uar, ent, jac, s); });
    });
}

PyObject* py_batch_stats(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 5, [](Args& a) {
        const at::Tensor* t = a.tensor("adv");
        int32_t G, N;
        two_dims(t, "adv", G, N);
        const float* adv = static_cast<float*>(Args::address(t, kF32, kAnySize, false, "adv"));
        const uint8_t* stop = a.buffer<uint8_t>(kU8, G, "stop");
        int64_t* counts = a.buffer<int64_t>(kI64, 3, "counts");
        double* sumsq = a.buffer<double>(kF64, 2, "sumsq");
        void* s = a.stream();
        return unlocked([&] { return sr_batch_stats(adv, stop, G, N, counts, sumsq, s); });
    });
}

PyObject* py_kept_groups(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 7, [](Args& a) {
        const at::Tensor *st = a.tensor("stop"), *zt = a.tensor("zero_var"), *it = a.tensor("index"), *ct = a.tensor("count");
        size_t bytes;
        void* ws = a.scratch("workspace", bytes);
        PyObject* g = *a.at++;
        int32_t G;
        if (g == Py_None) {
            const at::Tensor* from = st ? st : (zt ? zt : it);
            if (from == nullptr || from->dim() < 1) raise(PyExc_ValueError, "n_groups is not given and no tensor tells it");
            G = (int32_t)from->size(0);
        } else {
            Args one{&g};
            G = one.integer();
        }
        const uint8_t* stop = static_cast<uint8_t*>(Args::address(st, kU8, G, false, "stop"));
        const uint8_t* zero_var = static_cast<uint8_t*>(Args::address(zt, kU8, G, false, "zero_var"));
        int32_t* index = static_cast<int32_t*>(Args::address(it, kI32, G, false, "index"));
        int32_t* count = static_cast<int32_t*>(Args::address(ct, kI32, 1, false, "count"));
        void* s = a.stream();
        return unlocked([&] { return sr_kept_groups(stop, zero_var, G, index, count, ws, bytes, s); });
    });
}

PyObject* py_grpo_advantage(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 6, [](Args& a) {
        const at::Tensor* t = a.tensor("rewards");
        int32_t G, N;
        two_dims(t, "rewards", G, N);
        const float* rewards = static_cast<float*>(Args::address(t, kF32, kAnySize, false, "rewards"));
        const uint8_t* drop = a.buffer<uint8_t>(kU8, G, "drop_mask");
        const float eps = (float)a.real();
        float* adv = a.buffer<float>(kF32, (int64_t)G * N, "adv");
        uint8_t* zero_var = a.buffer<uint8_t>(kU8, G, "zero_var");
        void* s = a.stream();
        return unlocked([&] { return sr_grpo_advantage(rewards, drop, G, N, eps, adv, zero_var, s); });
    });
}

// ------------------------------------------------------------------ the trainer's operators (sr_train.h)
// These run on the device their tensors are on, whichever is current; all tensors of a call share it.
struct OneDevice {
    c10::cuda::OptionalCUDAGuard guard;
    int index = -1;
    const at::Tensor* add(const at::Tensor* t, const char* name) {
        if (t == nullptr) return t;
        if (!t->is_cuda()) raise(PyExc_ValueError, std::string(name) + " must be a CUDA tensor");
        const int at = t->device().index();
        if (index < 0) {
            index = at;
            guard.set_index((c10::DeviceIndex)at);
        } else if (at != index) {
            raise(PyExc_ValueError, std::string(name) + " is on another device than the tensors before it");
        }
        return t;
    }
};
template <typename T>
T* on(OneDevice& dev, const at::Tensor* t, c10::ScalarType type, int64_t need, const char* name) {
    return static_cast<T*>(Args::address(dev.add(t, name), type, need, false, name));
}
void* scratch_on(OneDevice& dev, Args& a, size_t& bytes) {
    const at::Tensor* t = dev.add(a.tensor("workspace"), "workspace");
    bytes = t ? (size_t)t->numel() * t->element_size() : 0;
    return Args::address(t, kAnyType, kAnySize, false, "workspace");
}
int32_t dtype_code(const at::Tensor& t, const char* name) {
    switch (t.scalar_type()) {
        case c10::ScalarType::Float: return SR_DTYPE_F32;
        case c10::ScalarType::BFloat16: return SR_DTYPE_BF16;
        case c10::ScalarType::Half: return SR_DTYPE_F16;
        default: raise(PyExc_TypeError, std::string(name) + ": expected torch.float32, torch.bfloat16 or torch.float16, got " + dtype_name(t.scalar_type()));
    }
}
int32_t count32(int64_t n, const char* name) {
    if (n > INT32_MAX) raise(PyExc_ValueError, std::string(name) + " has more than 2^31 - 1 rows or elements a row");
    return (int32_t)n;
}

// [tokens, vocabulary], rows apart by any pitch that does not make them overlap
struct Logits {
    void* data;
    int32_t dtype, n, vocab;
    int64_t pitch;
    Logits(OneDevice& dev, const at::Tensor* t, const char* name) {
        if (t == nullptr || t->dim() != 2) raise(PyExc_ValueError, std::string(name) + " must be [tokens, vocabulary]");
        dtype = dtype_code(*dev.add(t, name), name);
        n = count32(t->size(0), name);
        vocab = count32(t->size(1), name);
        if (vocab > 1 && t->stride(1) != 1) raise(PyExc_ValueError, std::string(name) + ": the logits of a row must be consecutive");
        pitch = n > 1 ? t->stride(0) : vocab;
        data = t->data_ptr();
    }
};
Logits same_logits(OneDevice& dev, const at::Tensor* t, const Logits& as, const char* name) {
    Logits l(dev, t, name);
    if (l.dtype != as.dtype) raise(PyExc_TypeError, std::string(name) + " must have the logits' type");
    if (l.n != as.n || l.vocab != as.vocab) raise(PyExc_ValueError, std::string(name) + " must have the logits' shape");
    return l;
}

PyObject* py_token_logprob(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 8, [](Args& a) {
        OneDevice dev;
        const Logits x(dev, a.tensor("logits"), "logits");
        const int32_t* targets = on<int32_t>(dev, a.tensor("targets"), kI32, x.n, "targets");
        const double temperature = a.real();
        float* logp = on<float>(dev, a.tensor("logp"), kF32, x.n, "logp");
        float* stats = on<float>(dev, a.tensor("row_stats"), kF32, 2 * (int64_t)x.n, "row_stats");
        float* entropy = on<float>(dev, a.tensor("entropy"), kF32, x.n, "entropy");
        int32_t* status = on<int32_t>(dev, a.tensor("status"), kI32, 1, "status");
        void* s = a.stream();
        return unlocked([&] { return sr_token_logprob(x.data, x.dtype, x.n, x.vocab, x.pitch, targets, temperature, logp, stats, entropy, status, s); });
    });
}

PyObject* py_token_logprob_backward(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 9, [](Args& a) {
        OneDevice dev;
        const Logits x(dev, a.tensor("logits"), "logits");
        const int32_t* targets = on<int32_t>(dev, a.tensor("targets"), kI32, x.n, "targets");
        const float* stats = on<float>(dev, a.tensor("row_stats"), kF32, 2 * (int64_t)x.n, "row_stats");
        const float* entropy = on<float>(dev, a.tensor("entropy"), kF32, x.n, "entropy");
        const float* d_logp = on<float>(dev, a.tensor("d_logp"), kF32, x.n, "d_logp");
        const float* d_entropy = on<float>(dev, a.tensor("d_entropy"), kF32, x.n, "d_entropy");
        const double temperature = a.real();
        const Logits dx = same_logits(dev, a.tensor("d_logits"), x, "d_logits");
        void* s = a.stream();
        return unlocked([&] { return sr_token_logprob_backward(x.data, x.dtype, x.n, x.vocab, x.pitch, targets, stats, entropy, d_logp, d_entropy, temperature, dx.data, dx.pitch, s); });
    });
}

int32_t rollouts_of(const at::Tensor* row_start) {
    if (row_start == nullptr || row_start->numel() < 1) raise(PyExc_ValueError, "row_start needs an entry for every rollout and one more");
    return count32(row_start->numel() - 1, "row_start");
}

PyObject* py_loss_weights(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 10, [](Args& a) {
        OneDevice dev;
        const at::Tensor *rt = a.tensor("row_start"), *mt = a.tensor("mask"), *dt = a.tensor("drop_mask");
        const int32_t rows = rollouts_of(rt), N = a.integer(), mode = a.integer();
        if (N < 1 || rows % N) raise(PyExc_ValueError, "row_start needs n_groups * N + 1 entries");
        const double scale = a.real();
        const int64_t* start = on<int64_t>(dev, rt, kI64, kAnySize, "row_start");
        const uint8_t* mask = on<uint8_t>(dev, mt, kU8, kAnySize, "mask");
        const int32_t n = mt ? count32(mt->numel(), "mask") : 0;
        const uint8_t* drop = on<uint8_t>(dev, dt, kU8, rows / N, "drop_mask");
        float* weight = on<float>(dev, a.tensor("weight"), kF32, rows, "weight");
        int64_t* counts = on<int64_t>(dev, a.tensor("counts"), kI64, 2, "counts");
        size_t bytes;
        void* ws = scratch_on(dev, a, bytes);
        void* s = a.stream();
        return unlocked([&] { return sr_loss_weights(start, mask, n, drop, rows / N, N, mode, scale, weight, counts, ws, bytes, s); });
    });
}

// What the loss is computed over, as the calls take it: old and reference log-probabilities, advantages, weights, row starts, mask, clip range, beta.
struct Batch {
    const float *old_logp, *ref_logp, *adv, *weight;
    const int64_t* row_start;
    const uint8_t* mask;
    int32_t rows;
    double clip_low, clip_high, beta;
    Batch(OneDevice& dev, Args& a, int32_t n) {
        old_logp = on<float>(dev, a.tensor("logp_old"), kF32, n, "logp_old");
        ref_logp = on<float>(dev, a.tensor("logp_ref"), kF32, n, "logp_ref");
        const at::Tensor *at = a.tensor("adv"), *wt = a.tensor("weight"), *rt = a.tensor("row_start");
        rows = rollouts_of(rt);
        adv = on<float>(dev, at, kF32, rows, "adv");
        weight = on<float>(dev, wt, kF32, rows, "weight");
        row_start = on<int64_t>(dev, rt, kI64, kAnySize, "row_start");
        mask = on<uint8_t>(dev, a.tensor("mask"), kU8, n, "mask");
        clip_low = a.real();
        clip_high = a.real();
        beta = a.real();
    }
};

PyObject* py_policy_loss(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 15, [](Args& a) {
        OneDevice dev;
        const at::Tensor* t = a.tensor("logp");
        if (t == nullptr) raise(PyExc_ValueError, "logp must be a tensor");
        const float* logp = on<float>(dev, t, kF32, kAnySize, "logp");
        const int32_t n = count32(t->numel(), "logp");
        const Batch b(dev, a, n);
        float* loss = on<float>(dev, a.tensor("loss"), kF32, 1, "loss");
        float* d_logp = on<float>(dev, a.tensor("d_logp"), kF32, n, "d_logp");
        float* stats = on<float>(dev, a.tensor("stats"), kF32, 4, "stats");
        size_t bytes;
        void* ws = scratch_on(dev, a, bytes);
        void* s = a.stream();
        return unlocked([&] { return sr_policy_loss(logp, b.old_logp, b.ref_logp, b.adv, b.weight, b.row_start, b.rows, b.mask, n, b.clip_low, b.clip_high, b.beta, loss, d_logp, stats, ws, bytes, s); });
    });
}

PyObject* py_policy_loss_logits(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 19, [](Args& a) {
        OneDevice dev;
        const Logits x(dev, a.tensor("logits"), "logits");
        const int32_t* targets = on<int32_t>(dev, a.tensor("targets"), kI32, x.n, "targets");
        const Batch b(dev, a, x.n);
        const double temperature = a.real();
        float* loss = on<float>(dev, a.tensor("loss"), kF32, 1, "loss");
        float* logp = on<float>(dev, a.tensor("logp"), kF32, x.n, "logp");
        const Logits dx = same_logits(dev, a.tensor("d_logits"), x, "d_logits");
        float* stats = on<float>(dev, a.tensor("stats"), kF32, 4, "stats");
        int32_t* status = on<int32_t>(dev, a.tensor("status"), kI32, 1, "status");
        size_t bytes;
        void* ws = scratch_on(dev, a, bytes);
        void* s = a.stream();
        return unlocked([&] { return sr_policy_loss_logits(x.data, x.dtype, x.n, x.vocab, x.pitch, targets, b.old_logp, b.ref_logp, b.adv, b.weight, b.row_start, b.rows, b.mask, b.clip_low, b.clip_high, b.beta, temperature, loss, logp, dx.data, dx.pitch, stats, status, ws, bytes, s); });
    });
}

// A list or tuple of tensors, each dense (whatever the order of its dimensions).
struct Grads {
    std::vector<const void*> data;
    std::vector<int64_t> counts;
    std::vector<int32_t> dtypes;
    std::vector<const at::Tensor*> tensors;
    Grads(OneDevice& dev, PyObject* list, const char* name) {
        if (!PyList_Check(list) && !PyTuple_Check(list)) raise(PyExc_TypeError, std::string(name) + " must be a list or tuple of tensors");
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(list);
        count32(n, name);
        PyObject** items = PySequence_Fast_ITEMS(list);
        data.reserve(n); counts.reserve(n); dtypes.reserve(n); tensors.reserve(n);
        for (Py_ssize_t i = 0; i < n; ++i) {
            if (!THPVariable_Check(items[i])) raise(PyExc_TypeError, std::string(name) + " must be a list or tuple of tensors");
            const at::Tensor& t = THPVariable_Unpack(items[i]);
            dev.add(&t, name);
            dtypes.push_back(dtype_code(t, name));
            if (!t.is_non_overlapping_and_dense()) raise(PyExc_ValueError, std::string(name) + ": every tensor must be dense");
            counts.push_back(t.numel());
            data.push_back(t.numel() ? t.data_ptr() : nullptr);
            tensors.push_back(&t);
        }
    }
};

PyObject* py_grad_norm(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 4, [](Args& a) {
        OneDevice dev;
        const Grads g(dev, *a.at++, "grads");
        float* norm = on<float>(dev, a.tensor("norm"), kF32, 1, "norm");
        size_t bytes;
        void* ws = scratch_on(dev, a, bytes);
        void* s = a.stream();
        return unlocked([&] { return sr_grad_norm(g.data.data(), g.counts.data(), g.dtypes.data(), (int32_t)g.data.size(), norm, ws, bytes, s); });
    });
}

PyObject* py_clip_grads(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 6, [](Args& a) {
        OneDevice dev;
        const Grads g(dev, *a.at++, "grads");
        const float* norm = on<float>(dev, a.tensor("norm"), kF32, 1, "norm");
        const double max_norm = a.real();
        PyObject* given = *a.at++;
        std::vector<void*> out;
        if (given != Py_None) {
            const Grads o(dev, given, "out");
            if (o.data.size() != g.data.size()) raise(PyExc_ValueError, "out must have a tensor for every gradient");
            for (size_t i = 0; i < o.data.size(); ++i) {
                if (o.dtypes[i] != g.dtypes[i]) raise(PyExc_TypeError, "out: a tensor has another type than its gradient");
                if (o.tensors[i]->sizes() != g.tensors[i]->sizes() || o.tensors[i]->strides() != g.tensors[i]->strides())
                    raise(PyExc_ValueError, "out: a tensor has another shape or layout than its gradient");
                out.push_back(const_cast<void*>(o.data[i]));
            }
        }
        int32_t* status = on<int32_t>(dev, a.tensor("status"), kI32, 1, "status");
        void* s = a.stream();
        return unlocked([&] { return sr_clip_grads(g.data.data(), g.counts.data(), g.dtypes.data(), (int32_t)g.data.size(), norm, max_norm, given != Py_None ? out.data() : nullptr, status, s); });
    });
}

// ------------------------------------------------------------------ operators on token ids (sr_tokens.h)
// Histories and masks, as both directions take them.
struct Rules {
    const int32_t *history, *history_len;
    const int64_t* history_start;
    int64_t n_history = 0, mask_pitch = 0;
    const uint32_t* allowed;
    const int32_t* mask_row;
    int32_t n_masks = 0;
    void histories(OneDevice& dev, Args& a, int32_t n) {
        const at::Tensor* t = a.tensor("history");
        history = on<int32_t>(dev, t, kI32, kAnySize, "history");
        n_history = t ? t->numel() : 0;
        if (n_history == 0) history = nullptr;
        history_start = on<int64_t>(dev, a.tensor("history_start"), kI64, n, "history_start");
        history_len = on<int32_t>(dev, a.tensor("history_len"), kI32, n, "history_len");
    }
    void masks(OneDevice& dev, Args& a, int32_t n, int32_t vocab) {
        const at::Tensor* t = dev.add(a.tensor("allowed"), "allowed");
        allowed = nullptr;
        if (t) {
            if (t->dim() != 2) raise(PyExc_ValueError, "allowed must be [masks, words]");
            if (t->scalar_type() != kI32) raise(PyExc_TypeError, std::string("allowed: expected torch.int32, got ") + dtype_name(t->scalar_type()));
            if (t->size(1) < ((int64_t)vocab + 31) / 32) raise(PyExc_ValueError, "allowed needs a bit for every token of the vocabulary");
            if (t->size(1) > 1 && t->stride(1) != 1) raise(PyExc_ValueError, "allowed: the words of a mask must be consecutive");
            n_masks = count32(t->size(0), "allowed");
            mask_pitch = n_masks > 1 ? t->stride(0) : t->size(1);
            allowed = static_cast<const uint32_t*>(t->data_ptr());
        }
        mask_row = on<int32_t>(dev, a.tensor("mask_row"), kI32, n, "mask_row");
        if (t && !mask_row && n_masks < n) raise(PyExc_ValueError, "allowed needs a row for every row of logits, or mask_row");
        if (n_masks == 0 && t && n > 0) raise(PyExc_ValueError, "allowed has no rows");
    }
};
// [rows, width], rows apart by any pitch that does not make them overlap
struct Rows {
    void* data;
    int32_t dtype, n, width;
    int64_t pitch;
    Rows(OneDevice& dev, const at::Tensor* t, const char* name, const char* shape) {
        if (t == nullptr || t->dim() != 2) raise(PyExc_ValueError, std::string(name) + " must be " + shape);
        dtype = dtype_code(*dev.add(t, name), name);
        n = count32(t->size(0), name);
        width = count32(t->size(1), name);
        if (width > 1 && t->stride(1) != 1) raise(PyExc_ValueError, std::string(name) + ": the elements of a row must be consecutive");
        pitch = n > 1 ? t->stride(0) : width;
        data = t->data_ptr();
    }
};

PyObject* py_adjust_logits(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 17, [](Args& a) {
        OneDevice dev;
        const Logits x(dev, a.tensor("logits"), "logits");
        Rules r;
        r.histories(dev, a, x.n);
        const int32_t* prompt = on<int32_t>(dev, a.tensor("prompt_len"), kI32, x.n, "prompt_len");
        const float* repetition = on<float>(dev, a.tensor("repetition"), kF32, x.n, "repetition");
        const float* presence = on<float>(dev, a.tensor("presence"), kF32, x.n, "presence");
        const float* frequency = on<float>(dev, a.tensor("frequency"), kF32, x.n, "frequency");
        const at::Tensor *bt = a.tensor("bias_token"), *bv = a.tensor("bias_value");
        const int64_t n_bias = bv ? bv->numel() : 0;
        const int32_t* bias_token = on<int32_t>(dev, bt, kI32, n_bias, "bias_token");
        const float* bias_value = on<float>(dev, bv, kF32, kAnySize, "bias_value");
        const int64_t* bias_start = on<int64_t>(dev, a.tensor("bias_start"), kI64, x.n, "bias_start");
        const int32_t* bias_len = on<int32_t>(dev, a.tensor("bias_len"), kI32, x.n, "bias_len");
        if (n_bias == 0) bias_value = nullptr;
        r.masks(dev, a, x.n, x.vocab);
        const Logits y = same_logits(dev, a.tensor("out"), x, "out");
        int32_t* status = on<int32_t>(dev, a.tensor("status"), kI32, 1, "status");
        void* s = a.stream();
        return unlocked([&] { return sr_adjust_logits(x.data, x.dtype, x.n, x.vocab, x.pitch, r.history, r.n_history, r.history_start, r.history_len, prompt, repetition, presence, frequency, bias_token, bias_value, n_bias, bias_start, bias_len, r.allowed, r.n_masks, r.mask_pitch, r.mask_row, y.data, y.pitch, status, s); });
    });
}

PyObject* py_adjust_logits_backward(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 11, [](Args& a) {
        OneDevice dev;
        const Logits d(dev, a.tensor("d_out"), "d_out");
        const at::Tensor* xt = a.tensor("logits");
        void* x = nullptr;
        int64_t pitch = d.vocab;
        if (xt) {
            const Logits l = same_logits(dev, xt, d, "logits");
            x = l.data;
            pitch = l.pitch;
        }
        Rules r;
        r.histories(dev, a, d.n);
        const float* repetition = on<float>(dev, a.tensor("repetition"), kF32, d.n, "repetition");
        r.masks(dev, a, d.n, d.vocab);
        const Logits dx = same_logits(dev, a.tensor("d_logits"), d, "d_logits");
        int32_t* status = on<int32_t>(dev, a.tensor("status"), kI32, 1, "status");
        void* s = a.stream();
        return unlocked([&] { return sr_adjust_logits_backward(d.data, d.dtype, d.n, d.vocab, d.pitch, x, pitch, r.history, r.n_history, r.history_start, r.history_len, repetition, r.allowed, r.n_masks, r.mask_pitch, r.mask_row, dx.data, dx.pitch, status, s); });
    });
}

PyObject* py_embed_tokens(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 6, [](Args& a) {
        OneDevice dev;
        const Rows table(dev, a.tensor("table"), "table", "[vocabulary, width]");
        const at::Tensor* tt = a.tensor("tokens");
        const double scale = a.real();
        const Rows out(dev, a.tensor("out"), "out", "[tokens, width]");
        if (out.width != table.width) raise(PyExc_ValueError, "out must have the table's width");
        const int32_t* tokens = on<int32_t>(dev, tt, kI32, out.n, "tokens");
        if (tt && tt->numel() != out.n) raise(PyExc_ValueError, "out must have a row for every token");
        int32_t* status = on<int32_t>(dev, a.tensor("status"), kI32, 1, "status");
        void* s = a.stream();
        return unlocked([&] { return sr_embed_tokens(table.data, table.dtype, table.n, table.width, table.pitch, tokens, out.n, scale, out.data, out.dtype, out.pitch, status, s); });
    });
}

PyObject* py_embed_tokens_backward(PyObject*, PyObject* const* argv, Py_ssize_t argc) {
    return guarded(argv, argc, 8, [](Args& a) {
        OneDevice dev;
        const Rows d(dev, a.tensor("d_out"), "d_out", "[tokens, width]");
        const at::Tensor* tt = a.tensor("tokens");
        const int32_t* tokens = on<int32_t>(dev, tt, kI32, d.n, "tokens");
        if (tt && tt->numel() != d.n) raise(PyExc_ValueError, "d_out must have a row for every token");
        const double scale = a.real();
        const Rows table(dev, a.tensor("d_table"), "d_table", "[vocabulary, width]");
        if (d.width != table.width) raise(PyExc_ValueError, "d_table must have d_out's width");
        const int32_t accumulate = a.integer();
        int32_t* status = on<int32_t>(dev, a.tensor("status"), kI32, 1, "status");
        size_t bytes;
        void* ws = scratch_on(dev, a, bytes);
        void* s = a.stream();
        return unlocked([&] { return sr_embed_tokens_backward(d.data, d.dtype, d.n, d.width, d.pitch, tokens, table.n, scale, table.data, table.dtype, table.pitch, accumulate, status, ws, bytes, s); });
    });
}

#define SR_METHOD(name) {"sr_" #name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    SR_METHOD(gate), SR_METHOD(gate_noalloc), SR_METHOD(gate_decide), SR_METHOD(gate_host),
    SR_METHOD(gate_host_packed), SR_METHOD(incr_init), SR_METHOD(gate_step_incremental),
    SR_METHOD(gate_or_rule), SR_METHOD(group_signals), SR_METHOD(batch_stats),
    SR_METHOD(kept_groups), SR_METHOD(grpo_advantage), SR_METHOD(token_logprob), SR_METHOD(token_logprob_backward),
    SR_METHOD(loss_weights), SR_METHOD(policy_loss), SR_METHOD(policy_loss_logits), SR_METHOD(grad_norm),
    SR_METHOD(clip_grads), SR_METHOD(adjust_logits), SR_METHOD(adjust_logits_backward), SR_METHOD(embed_tokens),
    SR_METHOD(embed_tokens_backward), {nullptr, nullptr, 0, nullptr}};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) {
    g_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    if (g_cuda_stream == nullptr) return nullptr;
    return PyModule_Create(&g_module);
}
