// Argument marshalling of the Python binding (binding.py): tensors, optional streams and sequences become the plain
// pointers and numbers of include/tq.h.  Nothing else happens here; the functions called are libtq.so's, whose addresses
// binding.py hands over once.  Through ctypes and tensor attributes a call spent 2 to 3.7 us of host time beyond the 2.2 to
// 2.6 us of the launch, which bounds rounds of short gradients.
#include <Python.h>

#include <ATen/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <exception>
#include <initializer_list>
#include <string>
#include <vector>

#include "tq.h"

namespace {

struct Functions {
    decltype(&tq_stats) stats;
    decltype(&tq_stats_hinted) stats_hinted;
    decltype(&tq_stats_static) stats_static;
    decltype(&tq_params_batch) params_batch;
    decltype(&tq_params_device) params_device;
    decltype(&tq_compress) compress;
    decltype(&tq_compress_device_params) compress_device_params;
    decltype(&tq_decompress_aggregate) decompress_aggregate;
    decltype(&tq_decompress_aggregate_rows) decompress_aggregate_rows;
    decltype(&tq_decompress_aggregate_apply) decompress_aggregate_apply;
    decltype(&tq_decompress_aggregate_device_params) decompress_aggregate_device_params;
    decltype(&tq_stats_segments) stats_segments;
    decltype(&tq_stats_hinted_segments) stats_hinted_segments;
    decltype(&tq_compress_segments) compress_segments;
    decltype(&tq_decompress_aggregate_segments) decompress_aggregate_segments;
    decltype(&tq_mx_quantize) mx_quantize;
    decltype(&tq_mx_quantize_both) mx_quantize_both;
    decltype(&tq_mx_dequantize) mx_dequantize;
    decltype(&tq_mx_decompress_aggregate) mx_decompress_aggregate;
    decltype(&tq_mx_product) mx_product;
    decltype(&tq_mx_gated) mx_gated;
    decltype(&tq_mx_gated_backward) mx_gated_backward;
} F;

struct Failed {};                              // a Python exception is set

[[noreturn]] void fail(PyObject* type, const char* what) {
    PyErr_SetString(type, what);
    throw Failed();
}

// Calls the library with the interpreter lock released, as ctypes does: a launch may wait for room in a full queue, behind a host
// callback that needs the lock.  Arguments are ready before; what they point to is held by the caller's arguments or by Args.
template <class... P, class... A>
tq_status call(tq_status (*f)(P...), const A&... args) {
    struct Unlocked {
        PyThreadState* state = PyEval_SaveThread();
        ~Unlocked() { PyEval_RestoreThread(state); }
    } unlocked;
    return f(args...);
}

// Device address of a tensor, or of anything else with a data_ptr() (a storage, say).
void* address_of(PyObject* o) {
    if (THPVariable_Check(o)) return THPVariable_Unpack(o).data_ptr();
    PyObject* v = PyObject_CallMethod(o, "data_ptr", nullptr);
    if (!v) {
        if (PyErr_ExceptionMatches(PyExc_AttributeError)) fail(PyExc_TypeError, "a tensor is needed");
        throw Failed();
    }
    void* p = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) throw Failed();
    return p;
}

// One call's positional arguments, taken in order.
class Args {
public:
    Args(PyObject* const* args, Py_ssize_t n) : args_(args), n_(n) {}
    ~Args() { for (Py_buffer& b : held_) PyBuffer_Release(&b); }
    Args(const Args&) = delete;
    Args& operator=(const Args&) = delete;

    PyObject* next() {
        if (at_ >= n_) fail(PyExc_TypeError, "too few arguments");
        return args_[at_++];
    }
    const at::Tensor& tensor() {
        PyObject* o = next();
        if (!THPVariable_Check(o)) fail(PyExc_TypeError, "a tensor is needed");
        return THPVariable_Unpack(o);
    }
    void* address() {                          // nullptr for None
        PyObject* o = next();
        return o == Py_None ? nullptr : address_of(o);
    }
    // a ctypes array (or anything else with a buffer): its address and size
    void* buffer(Py_ssize_t* bytes = nullptr) {
        held_.emplace_back();
        if (PyObject_GetBuffer(next(), &held_.back(), PyBUF_SIMPLE) != 0) { held_.pop_back(); throw Failed(); }
        if (bytes) *bytes = held_.back().len;
        return held_.back().buf;
    }
    uint64_t u64() {                           // wraps, as a C conversion does; the library checks ranges
        const uint64_t v = PyLong_AsUnsignedLongLongMask(next());
        if (v == ~0ull && PyErr_Occurred()) throw Failed();
        return v;
    }
    uint32_t u32() { return static_cast<uint32_t>(u64()); }
    double f64() {
        const double v = PyFloat_AsDouble(next());
        if (v == -1.0 && PyErr_Occurred()) throw Failed();
        return v;
    }
    float f32() { return static_cast<float>(f64()); }
    // None: torch's current stream; else a stream object, or a raw handle: anything that int() takes (other libraries' handles do)
    void* stream() { return stream_of(next()); }
    // The stream argument of a call whose last it is: for what is made before its turn.
    PyObject* last() {
        if (n_ < 1) fail(PyExc_TypeError, "too few arguments");
        return args_[n_ - 1];
    }
    static void* stream_of(PyObject* o) {
        if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
        PyObject* handle = PyObject_HasAttrString(o, "cuda_stream") ? PyObject_GetAttrString(o, "cuda_stream") : PyNumber_Long(o);
        if (!handle) throw Failed();
        void* s = PyLong_AsVoidPtr(handle);
        Py_DECREF(handle);
        if (PyErr_Occurred()) throw Failed();
        return s;
    }
    // None, or up to n values that float() takes, the rest zeros.  Only the first TQ_MAX_WORKERS are kept: the library refuses more rows before
    // it reads a weight.
    const float* weights(uint32_t n) {
        PyObject* o = next();
        if (o == Py_None) return nullptr;
        PyObject* seq = PySequence_Fast(o, "weights must be a sequence of numbers");
        if (!seq) throw Failed();
        const Py_ssize_t have = PySequence_Fast_GET_SIZE(seq);
        for (Py_ssize_t i = 0; i < have; ++i) {
            PyObject* w = PyNumber_Float(PySequence_Fast_GET_ITEM(seq, i));
            if (!w) break;
            if (i < TQ_MAX_WORKERS) weights_[i] = static_cast<float>(PyFloat_AS_DOUBLE(w));
            Py_DECREF(w);
        }
        Py_DECREF(seq);
        if (PyErr_Occurred()) throw Failed();
        if (have > n) fail(PyExc_IndexError, "invalid index");
        for (Py_ssize_t i = have; i < TQ_MAX_WORKERS; ++i) weights_[i] = 0.0f;
        return weights_;
    }

private:
    PyObject* const* args_;
    Py_ssize_t n_, at_ = 0;
    std::vector<Py_buffer> held_;
    float weights_[TQ_MAX_WORKERS];
};

// A [N, stride] or [d] gradient block.
struct Grad {
    void* data;
    tq_dtype dtype;
    uint64_t width, stride;
    uint32_t n;
};
Grad gradient(Args& a) {
    const at::Tensor& t = a.tensor();
    if (!t.is_cuda()) fail(PyExc_ValueError, "gradient must be a CUDA tensor");
    const int64_t dims = t.dim();
    if ((dims != 1 && dims != 2) || t.stride(dims - 1) != 1) fail(PyExc_ValueError, "gradient must be [N, stride] with unit inner stride");
    Grad g;
    if (t.scalar_type() == at::kFloat) g.dtype = TQ_F32;
    else if (t.scalar_type() == at::kBFloat16) g.dtype = TQ_BF16;
    else fail(PyExc_TypeError, "gradient must be float32 or bfloat16");
    g.data = t.data_ptr();
    g.n = dims == 2 ? static_cast<uint32_t>(t.size(0)) : 1u;
    g.width = static_cast<uint64_t>(t.size(dims - 1));
    g.stride = g.n > 1 ? static_cast<uint64_t>(t.stride(0)) : g.width;
    return g;
}
uint64_t elements(Args& a, const Grad& g) {     // None: the whole width
    PyObject* o = a.next();
    if (o == Py_None) return g.width;
    const uint64_t v = PyLong_AsUnsignedLongLongMask(o);
    if (v == ~0ull && PyErr_Occurred()) throw Failed();
    return v;
}
// A [N, words] block of packed rows.
struct Packed {
    uint32_t* data;
    size_t stride;
    uint32_t n;
};
Packed packed_rows(const at::Tensor& t) {       // in any memory the GPU reads (pinned host memory too); a row may have several dimensions
    if (t.dim() < 1) fail(PyExc_ValueError, "packed must have a row per worker");
    return Packed{static_cast<uint32_t*>(t.data_ptr()), static_cast<size_t>(t.size(0) > 1 ? t.stride(0) : t.size(1)), static_cast<uint32_t>(t.size(0))};
}
Packed packed_out(Args& a, uint32_t n) {        // as many rows as the gradient has; one row may be given as a vector
    const at::Tensor& t = a.tensor();
    const bool rows = t.dim() == 2 && n > 1;
    return Packed{static_cast<uint32_t*>(t.data_ptr()), static_cast<size_t>(rows ? t.stride(0) : t.size(t.dim() - 1)), n};
}
const tq_params_t* host_params(Args& a, uint32_t n, bool or_more = false) {
    Py_ssize_t bytes = 0;
    void* p = a.buffer(&bytes);
    const Py_ssize_t need = static_cast<Py_ssize_t>(n * sizeof(tq_params_t));
    if (or_more ? bytes < need : bytes != need) fail(PyExc_ValueError, "one Params per worker");
    return static_cast<const tq_params_t*>(p);
}
const tq_segment_t* segments(Args& a, uint32_t* n) {
    Py_ssize_t bytes = 0;
    void* p = a.buffer(&bytes);
    *n = static_cast<uint32_t>(bytes / sizeof(tq_segment_t));
    return static_cast<const tq_segment_t*>(p);
}
struct Scratch { void* data; size_t bytes; };
Scratch scratch(Args& a) {
    const at::Tensor& t = a.tensor();
    return Scratch{t.data_ptr(), static_cast<size_t>(t.numel())};
}

tq_status stats(Args& a) {                      // grad, d, g_min, kappa, stats, workspace, stream
    const Grad g = gradient(a);
    const uint64_t d = elements(a, g);
    const float g_min = a.f32(), kappa = a.f32();
    void* st = a.address();
    const Scratch ws = scratch(a);
    return call(F.stats, g.data, g.dtype, d, g.stride, g.n, g_min, kappa, static_cast<tq_stats_t*>(st), ws.data, ws.bytes, a.stream());
}
tq_status stats_hinted(Args& a) {               // grad, d, kappa, hint, stats, workspace, stream
    const Grad g = gradient(a);
    const uint64_t d = elements(a, g);
    const float kappa = a.f32();
    void* hint = a.address();
    void* st = a.address();
    const Scratch ws = scratch(a);
    return call(F.stats_hinted, g.data, g.dtype, d, g.stride, g.n, kappa, static_cast<tq_gmin_hint_t*>(hint), static_cast<tq_stats_t*>(st), ws.data,
                          ws.bytes, a.stream());
}
tq_status stats_static(Args& a) {               // grad, d, g_min, kappa, stats, stream
    const Grad g = gradient(a);
    const uint64_t d = elements(a, g);
    const float g_min = a.f32(), kappa = a.f32();
    void* st = a.address();
    return call(F.stats_static, g.data, g.dtype, d, g.stride, g.n, g_min, kappa, static_cast<tq_stats_t*>(st), a.stream());
}
tq_status params_batch(Args& a) {               // address of the records, n, num_levels, mode, gamma, rule, alpha_user, out
    PyObject* src = a.next();
    const void* records = THPVariable_Check(src) ? THPVariable_Unpack(src).data_ptr() : PyLong_AsVoidPtr(src);
    if (PyErr_Occurred()) throw Failed();
    const uint32_t n = a.u32(), levels = a.u32(), mode = a.u32();
    const double gamma = a.f64();
    const uint32_t rule = a.u32();
    const double alpha = a.f64();
    return call(F.params_batch, static_cast<const tq_stats_t*>(records), n, levels, static_cast<tq_mode>(mode), gamma, static_cast<tq_alpha_rule>(rule),
                          alpha, static_cast<tq_params_t*>(a.buffer()));
}
tq_status params_device(Args& a) {              // stats, n, num_levels, mode, gamma, rule, alpha_user, params, stream
    void* st = a.address();
    const uint32_t n = a.u32(), levels = a.u32(), mode = a.u32();
    const double gamma = a.f64();
    const uint32_t rule = a.u32();
    const double alpha = a.f64();
    void* out = a.address();
    return call(F.params_device, static_cast<tq_stats_t*>(st), n, levels, static_cast<tq_mode>(mode), gamma, static_cast<tq_alpha_rule>(rule), alpha,
                           static_cast<tq_params_t*>(out), a.stream());
}
tq_status compress(Args& a) {                   // grad, d, params, seed, first_worker, packed, stream
    const Grad g = gradient(a);
    const uint64_t d = elements(a, g);
    const tq_params_t* params = host_params(a, g.n);
    const uint64_t seed = a.u64();
    const uint32_t first = a.u32();
    const Packed p = packed_out(a, g.n);
    return call(F.compress, g.data, g.dtype, d, g.stride, g.n, params, seed, first, p.data, p.stride, a.stream());
}
tq_status compress_device_params(Args& a) {     // grad, d, params, num_levels, mode, seed, first_worker, packed, stream
    const Grad g = gradient(a);
    const uint64_t d = elements(a, g);
    void* params = a.address();
    const uint32_t levels = a.u32(), mode = a.u32();
    const uint64_t seed = a.u64();
    const uint32_t first = a.u32();
    const Packed p = packed_out(a, g.n);
    return call(F.compress_device_params, g.data, g.dtype, d, g.stride, g.n, static_cast<tq_params_t*>(params), levels, static_cast<tq_mode>(mode), seed,
                                    first, p.data, p.stride, a.stream());
}
tq_status decompress_aggregate(Args& a) {       // packed, d, params, weights, out, stream
    const at::Tensor& t = a.tensor();
    if (!t.is_cuda() || t.dim() != 2) fail(PyExc_ValueError, "packed must be a [N, words] CUDA tensor");
    const Packed p = packed_rows(t);
    const uint64_t d = a.u64();
    const tq_params_t* params = host_params(a, p.n);
    const float* w = a.weights(p.n);
    void* out = a.address();
    return call(F.decompress_aggregate, p.data, p.stride, p.n, d, params, w, static_cast<float*>(out), a.stream());
}
tq_status decompress_aggregate_rows(Args& a) {  // rows (tensors or addresses), d, params, weights, out, stream
    PyObject* seq = PySequence_Fast(a.next(), "rows must be a sequence");
    if (!seq) throw Failed();
    const uint32_t* rows[TQ_MAX_WORKERS];
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
    try {
        for (Py_ssize_t i = 0; i < n && i < TQ_MAX_WORKERS; ++i) {
            PyObject* r = PySequence_Fast_GET_ITEM(seq, i);
            rows[i] = static_cast<const uint32_t*>(PyLong_Check(r) ? PyLong_AsVoidPtr(r) : address_of(r));
            if (PyErr_Occurred()) throw Failed();
        }
    } catch (...) {
        Py_DECREF(seq);
        throw;
    }
    Py_DECREF(seq);
    const uint64_t d = a.u64();
    const tq_params_t* params = host_params(a, static_cast<uint32_t>(n));
    if (n > TQ_MAX_WORKERS) return TQ_ERR_INVALID_ARG;
    const float* w = a.weights(static_cast<uint32_t>(n));
    void* out = a.address();
    return call(F.decompress_aggregate_rows, rows, static_cast<uint32_t>(n), d, params, w, static_cast<float*>(out), a.stream());
}
tq_status decompress_aggregate_apply(Args& a) { // packed, d, params, weights, theta, momentum, lr, mu, weight_decay, stream
    const Packed p = packed_rows(a.tensor());
    const uint64_t d = a.u64();
    const tq_params_t* params = host_params(a, p.n, true);
    const float* w = a.weights(p.n);
    void* theta = a.address();
    void* momentum = a.address();
    const float lr = a.f32(), mu = a.f32(), wd = a.f32();
    return call(F.decompress_aggregate_apply, p.data, p.stride, p.n, d, params, w, static_cast<float*>(theta), static_cast<float*>(momentum), lr, mu, wd,
                                        a.stream());
}
tq_status decompress_aggregate_device_params(Args& a) {      // packed, d, params, num_levels, weights, out, stream
    const Packed p = packed_rows(a.tensor());
    const uint64_t d = a.u64();
    void* params = a.address();
    const uint32_t levels = a.u32();
    const float* w = a.weights(p.n);
    void* out = a.address();
    return call(F.decompress_aggregate_device_params, p.data, p.stride, p.n, d, static_cast<tq_params_t*>(params), levels, w, static_cast<float*>(out),
                                                a.stream());
}
tq_status stats_segments(Args& a) {             // grad, segments, g_min, kappa, stats, workspace, stream
    const Grad g = gradient(a);
    uint32_t n_seg;
    const tq_segment_t* seg = segments(a, &n_seg);
    const float g_min = a.f32(), kappa = a.f32();
    void* st = a.address();
    const Scratch ws = scratch(a);
    return call(F.stats_segments, g.data, g.dtype, g.stride, g.n, seg, n_seg, g_min, kappa, static_cast<tq_stats_t*>(st), ws.data, ws.bytes, a.stream());
}
tq_status stats_hinted_segments(Args& a) {      // grad, segments, kappa, hint, stats, workspace, stream
    const Grad g = gradient(a);
    uint32_t n_seg;
    const tq_segment_t* seg = segments(a, &n_seg);
    const float kappa = a.f32();
    void* hint = a.address();
    void* st = a.address();
    const Scratch ws = scratch(a);
    return call(F.stats_hinted_segments, g.data, g.dtype, g.stride, g.n, seg, n_seg, kappa, static_cast<tq_gmin_hint_t*>(hint), static_cast<tq_stats_t*>(st),
                                   ws.data, ws.bytes, a.stream());
}
tq_status compress_segments(Args& a) {          // grad, segments, params, num_levels, mode, seed, first_worker, packed, stream
    const Grad g = gradient(a);
    uint32_t n_seg;
    const tq_segment_t* seg = segments(a, &n_seg);
    void* params = a.address();
    const uint32_t levels = a.u32(), mode = a.u32();
    const uint64_t seed = a.u64();
    const uint32_t first = a.u32();
    const Packed p = packed_out(a, g.n);
    return call(F.compress_segments, g.data, g.dtype, g.stride, g.n, seg, n_seg, static_cast<tq_params_t*>(params), levels, static_cast<tq_mode>(mode), seed,
                               first, p.data, p.stride, a.stream());
}
tq_status decompress_aggregate_segments(Args& a) {           // packed, segments, params, num_levels, weights, out, stream
    const Packed p = packed_rows(a.tensor());
    uint32_t n_seg;
    const tq_segment_t* seg = segments(a, &n_seg);
    void* params = a.address();
    const uint32_t levels = a.u32();
    const float* w = a.weights(p.n);
    void* out = a.address();
    return call(F.decompress_aggregate_segments, p.data, p.stride, p.n, seg, n_seg, static_cast<tq_params_t*>(params), levels, w, static_cast<float*>(out),
                                           a.stream());
}

// ---- microscaled 4-bit floating point: an MxMatrix (binding.py) is six attributes ---------------------------------
struct MxNames {
    PyObject *rows, *cols, *layout, *memory, *own_codes, *own_scales;
} N;
// A matrix in one piece of memory: codes, and on the next 128-byte boundary scales.  Rows of codes that are longer than 128 bytes start on such a
// boundary: the products load 128 bytes of a row at a time.
struct MxPlace {
    uint64_t width, stride, scales, scale_rows, scale_stride, bytes;
};
MxPlace mx_place(uint64_t rows, uint64_t cols, bool tiles) {
    MxPlace p;
    const uint64_t blocks = (cols + 31) / 32;
    p.width = blocks * 16;
    p.stride = p.width > 128 ? (p.width + 127) / 128 * 128 : p.width;
    p.scales = (rows * p.stride + 127) / 128 * 128;
    p.scale_rows = tiles ? (rows + 127) / 128 : rows;
    p.scale_stride = tiles ? (blocks + 3) / 4 * 512 : (blocks + 15) / 16 * 16;
    p.bytes = p.scales + p.scale_rows * p.scale_stride;
    return p;
}

// Kernels run on the current device and take addresses of no other.
void on_current_device(const at::Tensor& t, const char* what) {
    if (!t.is_cuda()) fail(PyExc_ValueError, (std::string(what) + " must be a CUDA tensor").c_str());
    if (t.device().index() != c10::cuda::current_device()) fail(PyExc_ValueError, (std::string(what) + " is not on the current device").c_str());
}
uint64_t attribute(PyObject* o, PyObject* name) {
    PyObject* v = PyObject_GetAttr(o, name);
    if (!v) throw Failed();
    const uint64_t x = PyLong_AsUnsignedLongLong(v);               // refuses what is negative or no whole number
    Py_DECREF(v);
    if (x == ~0ull && PyErr_Occurred()) throw Failed();
    return x;
}
// The bytes of one attribute: `rows` rows of at least `width` bytes, wherever they start.
uint8_t* bytes_of(PyObject* o, PyObject* name, const char* what, uint64_t rows, uint64_t width, uint64_t* stride) {
    PyObject* v = PyObject_GetAttr(o, name);
    if (!v) throw Failed();
    Py_DECREF(v);                                                  // held by the matrix, which the caller's arguments hold
    if (!THPVariable_Check(v)) fail(PyExc_TypeError, "codes and scales must be tensors");
    const at::Tensor& t = THPVariable_Unpack(v);
    on_current_device(t, what);
    if (t.scalar_type() != at::kByte || t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) fail(PyExc_TypeError, "codes and scales must be [rows, bytes] uint8 with unit inner stride");
    if (static_cast<uint64_t>(t.size(0)) < rows || (rows && static_cast<uint64_t>(t.size(1)) < width)) fail(PyExc_ValueError, "codes or scales are smaller than the matrix");
    *stride = t.size(0) > 1 ? static_cast<uint64_t>(t.stride(0)) : static_cast<uint64_t>(t.size(1)) / 16 * 16;
    return static_cast<uint8_t*>(t.data_ptr());
}
tq_mx_t mx(PyObject* o) {
    tq_mx_t m{};
    m.rows = attribute(o, N.rows); m.cols = attribute(o, N.cols);
    m.layout = static_cast<uint32_t>(attribute(o, N.layout));
    PyObject* memory = PyObject_GetAttr(o, N.memory);
    if (!memory) throw Failed();
    Py_DECREF(memory);                                             // held by the matrix
    if (memory != Py_None) {
        if (!THPVariable_Check(memory)) fail(PyExc_TypeError, "a matrix's memory must be a tensor");
        const at::Tensor& t = THPVariable_Unpack(memory);
        on_current_device(t, "matrix");
        if (m.rows >= (1ull << 31) || m.cols > (1ull << 40)) return m;                       // the library refuses it
        const MxPlace p = mx_place(m.rows, m.cols, m.layout == TQ_MX_TILES);
        if (t.scalar_type() != at::kByte || !t.is_contiguous() || static_cast<uint64_t>(t.numel()) < p.bytes) fail(PyExc_ValueError, "the memory is smaller than the matrix");
        m.codes = static_cast<uint8_t*>(t.data_ptr()); m.scales = m.codes + p.scales;
        m.code_stride = p.stride; m.scale_stride = p.scale_stride;
        return m;
    }
    const uint64_t blocks = m.cols / 32 + (m.cols % 32 != 0);
    const bool tiles = m.layout == TQ_MX_TILES;
    m.codes = bytes_of(o, N.own_codes, "codes", m.rows, blocks * 16, &m.code_stride);
    m.scales = bytes_of(o, N.own_scales, "scales", tiles ? m.rows / 128 + (m.rows % 128 != 0) : m.rows, tiles ? (blocks + 3) / 4 * 512 : (blocks + 15) / 16 * 16, &m.scale_stride);
    return m;
}
// A plain [rows, cols] tensor, fp32 or bf16; a vector is one row.
struct Plain {
    void* data;
    tq_dtype dtype;
    uint64_t stride;
};
// Its size is that of the call: of a larger tensor the part that is meant has to be passed, or projections of more features would give u from
// g's columns.  `longer`: rows may have more elements than the call takes.
Plain plain(const at::Tensor& t, const char* what, uint64_t rows, uint64_t cols, bool longer = false) {
    on_current_device(t, what);
    const int64_t dims = t.dim();
    if ((dims != 1 && dims != 2) || (t.size(dims - 1) > 1 && t.stride(dims - 1) != 1)) fail(PyExc_ValueError, (std::string(what) + " must be [rows, cols] with unit inner stride").c_str());
    Plain p;
    if (t.scalar_type() == at::kFloat) p.dtype = TQ_F32;
    else if (t.scalar_type() == at::kBFloat16) p.dtype = TQ_BF16;
    else fail(PyExc_TypeError, (std::string(what) + " must be float32 or bfloat16").c_str());
    const uint64_t have = dims == 2 ? static_cast<uint64_t>(t.size(0)) : 1u, wide = static_cast<uint64_t>(t.size(dims - 1));
    if (have < rows || wide < cols) fail(PyExc_ValueError, (std::string(what) + " is smaller than the call needs").c_str());
    if (have > rows || (wide > cols && !longer)) fail(PyExc_ValueError, (std::string(what) + " is larger than the call needs").c_str());
    if (have > 1 && rows > 1 && t.stride(0) < static_cast<int64_t>(cols)) fail(PyExc_ValueError, (std::string(what) + " has rows that overlap").c_str());
    p.data = t.data_ptr();
    p.stride = have > 1 ? static_cast<uint64_t>(t.stride(0)) : wide;
    return p;
}
// Memory from torch's allocator, as torch.empty takes it but straight: through the dispatcher a matrix costs 1.9 us of host time.  On the current device, where
// the kernels run; a tensor for another one comes from at::empty.
// It is the memory of `stream`, on which the call writes it: earlier work on the current stream may still use what that one's memory last held.  The
// current stream, whose program drops the result, is noted for the allocator, which hands the memory out again when both have passed that.
at::Tensor empty_like_device(const at::Tensor& like, at::IntArrayRef sizes, at::ScalarType type, PyObject* stream) {
    if (!like.is_cuda() || like.device().index() != c10::cuda::current_device()) return at::empty(sizes, at::TensorOptions().dtype(type).device(like.device()));
    const auto make = [&] { return at::detail::empty_generic(sizes, c10::GetAllocator(c10::kCUDA), c10::DispatchKeySet(c10::DispatchKey::CUDA), type, std::nullopt); };
    if (stream == Py_None) return make();
    const c10::cuda::CUDAStream current = c10::cuda::getCurrentCUDAStream();
    cudaStream_t given = static_cast<cudaStream_t>(Args::stream_of(stream));
    if (given == cudaStreamLegacy) given = nullptr;                // two names of one stream; torch knows the other
    if (current.stream() == given) return make();
    const c10::cuda::CUDAStreamGuard on(c10::cuda::getStreamFromExternal(given, like.device().index()));
    at::Tensor t = make();
    c10::cuda::CUDACachingAllocator::recordStream(t.storage().data_ptr(), current);
    return t;
}
// A Python object that this call owns until it hands it over.
class Owned {
public:
    explicit Owned(PyObject* o = nullptr) : o_(o) {}
    Owned(Owned&& other) : o_(other.o_) { other.o_ = nullptr; }
    ~Owned() { Py_XDECREF(o_); }
    Owned(const Owned&) = delete;
    PyObject* get() const { return o_; }
    PyObject* release() { PyObject* o = o_; o_ = nullptr; return o; }

private:
    PyObject* o_;
};
PyObject* mx_class = nullptr;                   // binding.MxMatrix

// A matrix in memory of its own, on the device of a tensor.
Owned new_matrix(const at::Tensor& like, uint64_t rows, uint64_t cols, uint64_t layout, PyObject* stream) {
    if (rows >= (1ull << 31) || cols > (1ull << 40)) fail(PyExc_ValueError, "a matrix of this size is not possible");
    const int64_t bytes = static_cast<int64_t>(mx_place(rows, cols, layout == TQ_MX_TILES).bytes);
    static PyObject* const nothing = PyTuple_New(0);
    PyTypeObject* const type = reinterpret_cast<PyTypeObject*>(mx_class);
    Owned m(type->tp_new(type, nothing, nullptr));
    if (!m.get()) throw Failed();
    const auto set = [&](PyObject* name, PyObject* value) {
        const Owned v(value);
        if (!value || PyObject_SetAttr(m.get(), name, value) != 0) throw Failed();
    };
    set(N.memory, THPVariable_Wrap(empty_like_device(like, at::IntArrayRef(&bytes, 1), at::kByte, stream)));
    set(N.rows, PyLong_FromUnsignedLongLong(rows));
    set(N.cols, PyLong_FromUnsignedLongLong(cols));
    set(N.layout, PyLong_FromUnsignedLongLong(layout));
    Py_INCREF(Py_None);
    set(N.own_codes, Py_None);
    Py_INCREF(Py_None);
    set(N.own_scales, Py_None);
    return m;
}
// The next argument, or for None a new matrix.
Owned matrix_or_new(Args& a, const at::Tensor& like, uint64_t rows, uint64_t cols, uint64_t layout) {
    PyObject* o = a.next();
    if (o == Py_None) return new_matrix(like, rows, cols, layout, a.last());
    Py_INCREF(o);
    return Owned(o);
}
// The next argument, or for None a new [rows, cols] tensor; with rows -1 a vector.
Owned tensor_or_new(Args& a, const at::Tensor& like, int64_t rows, int64_t cols, bool bf16) {
    PyObject* o = a.next();
    if (o != Py_None) {
        if (!THPVariable_Check(o)) fail(PyExc_TypeError, "a tensor is needed");
        Py_INCREF(o);
        return Owned(o);
    }
    const int64_t sizes[2] = {rows, cols};
    Owned t(THPVariable_Wrap(empty_like_device(like, rows < 0 ? at::IntArrayRef(&cols, 1) : at::IntArrayRef(sizes, 2), bf16 ? at::kBFloat16 : at::kFloat, a.last())));
    if (!t.get()) throw Failed();
    return t;
}
// Some tensor of a matrix, for its device.
const at::Tensor& tensor_of(PyObject* matrix) {
    PyObject* v = PyObject_GetAttr(matrix, N.memory);
    if (!v) throw Failed();
    Py_DECREF(v);                                                  // held by the matrix
    if (v == Py_None) {
        v = PyObject_GetAttr(matrix, N.own_codes);
        if (!v) throw Failed();
        Py_DECREF(v);
    }
    if (!THPVariable_Check(v)) fail(PyExc_TypeError, "codes and scales must be tensors");
    return THPVariable_Unpack(v);
}
uint64_t high(const at::Tensor& t) { return t.dim() == 2 ? static_cast<uint64_t>(t.size(0)) : 1u; }
uint64_t wide(const at::Tensor& t) {
    if (t.dim() < 1) fail(PyExc_ValueError, "a matrix or a vector is needed");
    return static_cast<uint64_t>(t.size(t.dim() - 1));
}

// These calls return what they made, or the library's status.
PyObject* made(tq_status s, Owned& o) { return s == TQ_OK ? o.release() : PyLong_FromLong(s); }
PyObject* made(tq_status s, std::initializer_list<Owned*> all) {
    if (s != TQ_OK) return PyLong_FromLong(s);
    PyObject* t = PyTuple_New(static_cast<Py_ssize_t>(all.size()));
    if (!t) throw Failed();
    Py_ssize_t i = 0;
    for (Owned* o : all) PyTuple_SET_ITEM(t, i++, o->release());
    return t;
}
PyObject* new_mx(Args& a) {                     // like, rows, cols, layout
    const at::Tensor& like = a.tensor();
    const uint64_t rows = a.u64(), cols = a.u64(), layout = a.u64();
    return new_matrix(like, rows, cols, layout, Py_None).release();
}
// Where a matrix in one piece is: (bytes of a row, row stride, first byte of the scales, their rows, their stride).
PyObject* mx_layout(Args& a) {                  // rows, cols, layout
    const uint64_t rows = a.u64(), cols = a.u64(), layout = a.u64();
    const MxPlace p = mx_place(rows, cols, layout == TQ_MX_TILES);
    return Py_BuildValue("KKKKK", p.width, p.stride, p.scales, p.scale_rows, p.scale_stride);
}
PyObject* mx_quantize(Args& a) {                // x, rounding, seed, first_row, cols, layout, out, stream
    const at::Tensor& x = a.tensor();
    const uint32_t rounding = a.u32();
    const uint64_t seed = a.u64();
    const uint32_t first = a.u32();
    PyObject* c = a.next();
    const uint64_t cols = c == Py_None ? wide(x) : PyLong_AsUnsignedLongLong(c), layout = a.u64();
    if (PyErr_Occurred()) throw Failed();
    Owned out = matrix_or_new(a, x, high(x), cols, layout);
    const tq_mx_t m = mx(out.get());
    if (m.cols != cols) fail(PyExc_ValueError, m.cols < cols ? "out has fewer columns than are quantised" : "out has more columns than are quantised");
    const Plain p = plain(x, "x", m.rows, m.cols, c != Py_None);
    return made(call(F.mx_quantize, p.data, p.dtype, p.stride, static_cast<tq_mx_rounding>(rounding), seed, first, &m, a.stream()), out);
}
PyObject* mx_quantize_both(Args& a) {           // x, rounding, seed, first_row, out, out_t, stream
    const at::Tensor& x = a.tensor();
    const uint32_t rounding = a.u32();
    const uint64_t seed = a.u64();
    const uint32_t first = a.u32();
    Owned out = matrix_or_new(a, x, high(x), wide(x), TQ_MX_TILES);
    const tq_mx_t m = mx(out.get());
    Owned out_t = matrix_or_new(a, x, m.cols, m.rows, TQ_MX_TILES);
    const tq_mx_t m_t = mx(out_t.get());
    const Plain p = plain(x, "x", m.rows, m.cols);
    return made(call(F.mx_quantize_both, p.data, p.dtype, p.stride, static_cast<tq_mx_rounding>(rounding), seed, first, &m, &m_t, a.stream()), {&out, &out_t});
}
PyObject* mx_dequantize(Args& a) {              // matrix, bf16, out, stream
    PyObject* o = a.next();
    const tq_mx_t m = mx(o);
    const bool bf16 = a.u32() != 0;
    Owned out = tensor_or_new(a, tensor_of(o), static_cast<int64_t>(m.rows), static_cast<int64_t>(m.cols), bf16);
    const Plain p = plain(THPVariable_Unpack(out.get()), "out", m.rows, m.cols);
    return made(call(F.mx_dequantize, &m, p.data, p.dtype, p.stride, a.stream()), out);
}
PyObject* mx_decompress_aggregate(Args& a) {    // matrix, weights, out, stream
    PyObject* o = a.next();
    const tq_mx_t m = mx(o);
    const float* w = a.weights(static_cast<uint32_t>(m.rows < TQ_MAX_WORKERS ? m.rows : TQ_MAX_WORKERS));
    Owned out = tensor_or_new(a, tensor_of(o), -1, static_cast<int64_t>(m.cols), false);
    const Plain p = plain(THPVariable_Unpack(out.get()), "out", 1, m.cols, true);
    if (p.dtype != TQ_F32) fail(PyExc_TypeError, "out must be float32");
    return made(call(F.mx_decompress_aggregate, &m, w, static_cast<float*>(p.data), a.stream()), out);
}
PyObject* mx_product(Args& a) {                 // a, b, bf16, out, stream
    PyObject* o = a.next();
    const tq_mx_t x = mx(o), y = mx(a.next());
    const bool bf16 = a.u32() != 0;
    Owned out = tensor_or_new(a, tensor_of(o), static_cast<int64_t>(x.rows), static_cast<int64_t>(y.rows), bf16);
    const Plain p = plain(THPVariable_Unpack(out.get()), "out", x.rows, y.rows);
    return made(call(F.mx_product, &x, &y, p.data, p.dtype, p.stride, a.stream()), out);
}
PyObject* mx_gated(Args& a) {                   // x, w_gate, w_up, activation, projections, out, stream
    PyObject* o = a.next();
    const tq_mx_t x = mx(o), wg = mx(a.next()), wu = mx(a.next());
    const uint32_t act = a.u32();
    PyObject* kept = a.next();
    Plain p{nullptr, TQ_F32, 0};
    if (kept != Py_None) {
        if (!THPVariable_Check(kept)) fail(PyExc_TypeError, "a tensor is needed");
        p = plain(THPVariable_Unpack(kept), "projections", x.rows, 2 * wg.rows);
    }
    Owned out = matrix_or_new(a, tensor_of(o), x.rows, wg.rows, TQ_MX_TILES);
    const tq_mx_t h = mx(out.get());
    return made(call(F.mx_gated, &x, &wg, &wu, static_cast<tq_mx_activation>(act), &h, p.data, p.dtype, p.stride, a.stream()), out);
}
PyObject* mx_gated_backward(Args& a) {          // dh, projections, activation, rounding, seed, dgu, dgu_t, h_t, stream
    const at::Tensor& dh = a.tensor();
    const at::Tensor& gu = a.tensor();
    const uint32_t act = a.u32(), rounding = a.u32();
    const uint64_t seed = a.u64(), tokens = high(dh), features = wide(dh);
    Owned dgu = matrix_or_new(a, dh, tokens, 2 * features, TQ_MX_TILES), dgu_t = matrix_or_new(a, dh, 2 * features, tokens, TQ_MX_TILES);
    Owned h_t = matrix_or_new(a, dh, features, tokens, TQ_MX_TILES);
    const tq_mx_t m = mx(dgu.get()), m_t = mx(dgu_t.get()), h = mx(h_t.get());
    const Plain p = plain(dh, "dh", m.rows, h.rows), q = plain(gu, "projections", m.rows, m.cols);
    if (p.dtype != q.dtype) fail(PyExc_TypeError, "dh and projections must be of one type");
    return made(call(F.mx_gated_backward, p.data, p.stride, q.data, q.stride, p.dtype, static_cast<tq_mx_activation>(act), static_cast<tq_mx_rounding>(rounding), seed, &m, &m_t,
                     &h, a.stream()), {&dgu, &dgu_t, &h_t});
}

template <tq_status (*CALL)(Args&)>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        Args a(args, n);
        return PyLong_FromLong(CALL(a));
    } catch (const Failed&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

template <PyObject* (*CALL)(Args&)>
PyObject* maker(PyObject*, PyObject* const* args, Py_ssize_t n) {
    try {
        Args a(args, n);
        return CALL(a);
    } catch (const Failed&) {
        return nullptr;
    } catch (const c10::OutOfMemoryError&) {           // as from torch.empty
        torch::translate_exception_to_python(std::current_exception());
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// bind([addresses in the order of Functions], MxMatrix)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    constexpr Py_ssize_t count = sizeof(Functions) / sizeof(void*);
    if (n < 1 || n > 2 || !PyList_Check(args[0]) || PyList_GET_SIZE(args[0]) != count || (n == 2 && !PyType_Check(args[1]))) {
        PyErr_SetString(PyExc_TypeError, "a list of function addresses is needed");
        return nullptr;
    }
    void* p[count];
    for (Py_ssize_t i = 0; i < count; ++i) p[i] = PyLong_AsVoidPtr(PyList_GET_ITEM(args[0], i));
    if (PyErr_Occurred()) return nullptr;
    memcpy(&F, p, sizeof(F));
    if (n == 2) {
        Py_INCREF(args[1]);
        Py_XDECREF(mx_class);
        mx_class = args[1];
    }
    Py_RETURN_NONE;
}

#define TQ_ENTRY(name) {#name, reinterpret_cast<PyCFunction>(entry<name>), METH_FASTCALL, nullptr}
#define TQ_MAKER(name) {#name, reinterpret_cast<PyCFunction>(maker<name>), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(bind), METH_FASTCALL, nullptr},
    TQ_ENTRY(stats), TQ_ENTRY(stats_hinted), TQ_ENTRY(stats_static), TQ_ENTRY(params_batch), TQ_ENTRY(params_device), TQ_ENTRY(compress),
    TQ_ENTRY(compress_device_params), TQ_ENTRY(decompress_aggregate), TQ_ENTRY(decompress_aggregate_rows), TQ_ENTRY(decompress_aggregate_apply),
    TQ_ENTRY(decompress_aggregate_device_params), TQ_ENTRY(stats_segments), TQ_ENTRY(stats_hinted_segments), TQ_ENTRY(compress_segments),
    TQ_ENTRY(decompress_aggregate_segments), TQ_MAKER(new_mx), TQ_MAKER(mx_layout), TQ_MAKER(mx_quantize), TQ_MAKER(mx_quantize_both), TQ_MAKER(mx_dequantize),
    TQ_MAKER(mx_decompress_aggregate), TQ_MAKER(mx_product), TQ_MAKER(mx_gated), TQ_MAKER(mx_gated_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module{PyModuleDef_HEAD_INIT, "_tq_python", "Argument marshalling for libtq.so.", -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__tq_python() {
    N = MxNames{PyUnicode_InternFromString("rows"), PyUnicode_InternFromString("cols"),
                PyUnicode_InternFromString("layout"), PyUnicode_InternFromString("memory"),
                PyUnicode_InternFromString("_codes"), PyUnicode_InternFromString("_scales")};
    if (!N.rows || !N.cols || !N.layout || !N.memory || !N.own_codes || !N.own_scales) return nullptr;
    return PyModule_Create(&module);
}
