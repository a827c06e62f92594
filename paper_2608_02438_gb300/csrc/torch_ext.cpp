// torch_ext.cpp -- the torch side of the drafter head's entry points: the
// checks of the tensors and the argument blocks of xpress_rmsnorm,
// xpress_quantize_weight, xpress_matmul_fp8, xpress_linear, xpress_process_logits
// and xpress_sample.
//
// The calls take a few microseconds on the GPU at a decode step's sizes, and as
// many Python operations as a dozen tensors need (shape, strides, type, device,
// address of each) take longer than that: 13.5 us per xpress_rmsnorm call on
// the GPU host's cores against 3.4 us for the launch.  binding.py keeps the
// signatures, defaults and documentation and calls these with positional
// arguments; they return the library's status.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/zeros.h>
#include <c10/cuda/CUDAException.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <c10/util/Exception.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <map>
#include <string>
#include <utility>

#include "xpress.h"

namespace {

constexpr auto BF16 = at::kBFloat16, F32 = at::kFloat, I32 = at::kInt, I64 = at::kLong;
constexpr auto E4M3 = at::kFloat8_e4m3fn;

// ValueError / TypeError in Python.
template <typename... A> [[noreturn]] void bad_value(const A &...a) { C10_THROW_ERROR(ValueError, c10::str(a...)); }
template <typename... A> [[noreturn]] void bad_type(const A &...a) { C10_THROW_ERROR(TypeError, c10::str(a...)); }

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

const at::Tensor &tensor(const char *name, PyObject *o)
{
    if (!THPVariable_Check(o)) bad_type(name, ": expected a tensor");
    return THPVariable_Unpack(o);
}

int dtype_code(const at::Tensor &t)
{
    if (t.scalar_type() == BF16) return XPRESS_BF16;
    if (t.scalar_type() == F32) return XPRESS_F32;
    bad_value("bfloat16 or float32 tensors are supported, not ", c10::toString(t.scalar_type()));
}

std::string shape_of(const at::Tensor &t) { return c10::str(c10::toString(t.scalar_type()), " ", t.sizes(), " on ", t.device()); }

// Address and row pitch of the [rows, cols] matrix `o` on device `dev` (rows
// may be padded, columns are contiguous).
void *matrix(const char *name, PyObject *o, int64_t rows, int64_t cols, at::ScalarType dt, int dev, int64_t &pitch)
{
    const at::Tensor &t = tensor(name, o);
    if (t.dim() != 2 || t.size(0) != rows || t.size(1) != cols || t.scalar_type() != dt || t.get_device() != dev)
        bad_value(name, ": expected a ", c10::toString(dt), " [", rows, ", ", cols, "] tensor on device ", dev, ", got ",
                  shape_of(t));
    if (cols > 1 && t.stride(1) != 1) bad_value(name, ": columns must be contiguous");
    // the pitch of a single row is never used
    pitch = rows > 1 ? t.stride(0) : ceil_div(cols, 16) * 16;
    return t.data_ptr();
}

// Address of the contiguous vector `o` of n elements (any number if n < 0).
void *vector(const char *name, PyObject *o, int64_t n, at::ScalarType dt, int dev)
{
    const at::Tensor &t = tensor(name, o);
    if (t.dim() != 1 || (n >= 0 && t.size(0) != n) || t.scalar_type() != dt || t.get_device() != dev ||
        (t.size(0) > 1 && t.stride(0) != 1))
        bad_value(name, ": expected a contiguous ", c10::toString(dt), " vector of ",
                  n < 0 ? "any length" : std::to_string(n), " on device ", dev, ", got ", shape_of(t));
    return t.data_ptr();
}

const at::Tensor &rank2(const char *name, PyObject *o)
{
    const at::Tensor &t = tensor(name, o);
    if (t.dim() != 2) bad_value(name, ": expected a matrix, got ", shape_of(t));
    return t;
}

int narrow(const char *name, int64_t n)
{
    if (n > INT32_MAX || n < INT32_MIN) bad_value(name, ": ", n, " is outside the supported range");
    return (int)n;
}

// Memory that a call reads or writes: n rows of `bytes`, `pitch` bytes apart.
struct Place {
    const char *name;
    uintptr_t at;
    int64_t n, pitch, bytes;

    Place(const char *name, const void *p, int64_t n, int64_t pitch, int64_t cols, int64_t es)
        : name(name), at(reinterpret_cast<uintptr_t>(p)), n(cols > 0 && p ? n : 0), pitch(pitch * es), bytes(cols * es) {}
    Place(const char *name, const void *p, int64_t n) : Place(name, p, 1, n, n, 4) {}      // a vector of 4-byte elements
    int64_t end() const { return (n - 1) * pitch + bytes; }
};

// Whether two places share a byte.  (Rows longer than their pitch are the entry points' to refuse.)
bool share(const Place &a, const Place &b)
{
    if (!a.n || !b.n || (a.n > 1 && a.pitch < a.bytes) || (b.n > 1 && b.pitch < b.bytes)) return false;
    const int64_t d = (int64_t)(b.at - a.at);                        // where b begins, from a
    if (d >= a.end() || -d >= b.end()) return false;
    if (a.n > 1 && b.n > 1 && a.pitch == b.pitch) {
        // rows that keep between one another
        const int64_t r = (d % a.pitch + a.pitch) % a.pitch;
        if (r >= a.bytes && r + b.bytes <= a.pitch) return false;
    }
    const Place &few = a.n < b.n ? a : b, &other = a.n < b.n ? b : a;
    const int64_t off = a.n < b.n ? -d : d;                          // where `few` begins, from the other
    for (int64_t i = 0; i < few.n; ++i) {
        // the last of the other's rows that begins before this one ends
        const int64_t from = off + i * few.pitch, last = from + few.bytes - 1;
        if (last < 0) continue;
        const int64_t row = other.n == 1 ? 0 : std::min(last / other.pitch, other.n - 1);
        if (row * other.pitch + other.bytes > from) return true;
    }
    return false;
}
void apart(const Place &out, const Place &in)
{
    if (share(out, in)) bad_value(out.name, " overlaps ", in.name);
}

// Torch's current stream on the tensors' device, which has to be the current one.
void *current_stream(int dev)
{
    if (dev < 0) bad_value("the tensors have to be on a CUDA device");
    const int cur = c10::cuda::current_device();
    if (cur != dev) bad_value("the tensors are on cuda:", dev, ", the current device is cuda:", cur);
    return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
}

void count(const char *name, Py_ssize_t n, Py_ssize_t want)
{
    if (n != want) bad_type(name, ": ", want, " arguments expected, got ", n);
}

bool given(PyObject *o) { return o != Py_None; }

// (x, weight, eps, residual, sum_out, y_out, q_out, scale_out)
PyObject *rmsnorm(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("rmsnorm", n, 8);
    const at::Tensor &x = rank2("x", v[0]);
    const int64_t rows = x.size(0), H = x.size(1);
    const auto dt = x.scalar_type();
    const int dev = x.get_device();
    xpress_norm_args a{};
    a.rows = narrow("rows", rows);
    a.H = narrow("H", H);
    a.dtype = dtype_code(x);
    a.eps = (float)PyFloat_AsDouble(v[2]);
    if (PyErr_Occurred()) return nullptr;
    a.x = matrix("x", v[0], rows, H, dt, dev, a.ldx);
    a.weight = vector("weight", v[1], H, dt, dev);
    if (given(v[3])) a.residual = matrix("residual", v[3], rows, H, dt, dev, a.ldr);
    if (given(v[4])) a.sum = matrix("sum_out", v[4], rows, H, dt, dev, a.lds);
    if (given(v[5])) a.y = matrix("y_out", v[5], rows, H, dt, dev, a.ldy);
    if (given(v[6])) {
        if (!given(v[7])) bad_value("q_out needs scale_out");
        a.q = matrix("q_out", v[6], rows, H, E4M3, dev, a.ldq);
        a.scale = static_cast<float *>(matrix("scale_out", v[7], rows, ceil_div(H, 128), F32, dev, a.ldscale));
    }
    void *st = current_stream(dev);
    return PyLong_FromLong(rows == 0 ? XPRESS_OK : xpress_rmsnorm(&a, st));   // empty tensors have no address
    END_HANDLE_TH_ERRORS
}

// (W, q_out, scale_out)
PyObject *quantize_weight(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("quantize_weight", n, 3);
    const at::Tensor &W = rank2("W", v[0]);
    const int64_t rows = W.size(0), cols = W.size(1), nrb = ceil_div(rows, 128), ncb = ceil_div(cols, 128);
    const int dev = W.get_device(), code = dtype_code(W);
    int64_t ldw, ldq, lds;
    void *w = matrix("W", v[0], rows, cols, W.scalar_type(), dev, ldw);
    void *q = matrix("q_out", v[1], rows, cols, E4M3, dev, ldq);
    void *sc = matrix("scale_out", v[2], nrb, ncb, F32, dev, lds);
    if (nrb > 1 && lds != ncb) bad_value("scale_out must be contiguous");
    void *st = current_stream(dev);
    return PyLong_FromLong(rows == 0 ? XPRESS_OK
                                     : xpress_quantize_weight(w, code, narrow("rows", rows), narrow("cols", cols), ldw, q,
                                                              ldq, static_cast<float *>(sc), st));
    END_HANDLE_TH_ERRORS
}

// The zeroed workspace of matmul_fp8 and linear on a device (its status word), made once.
void *matmul_workspace(int dev)
{
    constexpr int MAX_DEVICES = 64;
    static void *at_dev[MAX_DEVICES];
    if (dev < 0 || dev >= MAX_DEVICES) bad_value("device ", dev, " is not supported");
    if (!at_dev[dev]) {
        const int64_t size = (int64_t)xpress_matmul_fp8_workspace_size();
        auto *t = new at::Tensor(at::zeros({size}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, dev)));   // for good
        c10::cuda::device_synchronize();                 // zero before a call on any stream uses it
        at_dev[dev] = t->data_ptr();                     // torch's blocks start on 512 bytes
    }
    return at_dev[dev];
}

// (a, a_scale, w, w_scale, out)
PyObject *matmul_fp8(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("matmul_fp8", n, 5);
    const at::Tensor &a = rank2("a", v[0]), &w = rank2("w", v[2]), &out = rank2("out", v[4]);
    const int64_t M = a.size(0), K = a.size(1), N = w.size(0), kb = ceil_div(K, 128);
    const int dev = a.get_device();
    xpress_matmul_args g{};
    g.M = narrow("M", M);
    g.N = narrow("N", N);
    g.K = narrow("K", K);
    g.out_dtype = dtype_code(out);
    g.a = matrix("a", v[0], M, K, E4M3, dev, g.lda);
    g.a_scale = static_cast<float *>(matrix("a_scale", v[1], M, kb, F32, dev, g.ld_a_scale));
    g.w = matrix("w", v[2], N, K, E4M3, dev, g.ldw);
    g.w_scale = static_cast<float *>(matrix("w_scale", v[3], ceil_div(N, 128), kb, F32, dev, g.ld_w_scale));
    g.out = matrix("out", v[4], M, N, out.scalar_type(), dev, g.ldo);
    void *st = current_stream(dev);
    if (M == 0) return PyLong_FromLong(XPRESS_OK);
    return PyLong_FromLong(xpress_matmul_fp8(&g, matmul_workspace(dev), xpress_matmul_fp8_workspace_size(), st));
    END_HANDLE_TH_ERRORS
}

// (x, w, out, bias, act, residual)
PyObject *linear(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("linear", n, 6);
    const at::Tensor &x = rank2("x", v[0]), &w = rank2("w", v[1]), &out = rank2("out", v[2]);
    const int64_t M = x.size(0), K = x.size(1), N = w.size(0);
    const int dev = x.get_device();
    xpress_linear_args g{};
    g.M = narrow("M", M);
    g.N = narrow("N", N);
    g.K = narrow("K", K);
    g.out_dtype = dtype_code(out);
    const long act = PyLong_AsLong(v[4]);
    if (PyErr_Occurred()) return nullptr;
    g.act = narrow("act", act);
    g.x = matrix("x", v[0], M, K, BF16, dev, g.ldx);
    g.w = matrix("w", v[1], N, K, BF16, dev, g.ldw);
    g.out = matrix("out", v[2], M, N, out.scalar_type(), dev, g.ldo);
    if (given(v[3])) g.bias = vector("bias", v[3], N, BF16, dev);
    if (given(v[5])) g.residual = matrix("residual", v[5], M, N, out.scalar_type(), dev, g.ldr);
    const int64_t es = out.element_size();
    const Place to("out", g.out, M, g.ldo, N, es);
    apart(to, {"x", g.x, M, g.ldx, K, 2});
    apart(to, {"w", g.w, N, g.ldw, K, 2});
    apart(to, {"bias", g.bias, 1, N, N, 2});
    if (g.residual != g.out) apart(to, {"residual", g.residual, M, g.ldr, N, es});      // (one place: the entry point sees to the pitch)
    void *st = current_stream(dev);
    if (M == 0) return PyLong_FromLong(XPRESS_OK);                    // empty tensors have no address
    return PyLong_FromLong(xpress_linear(&g, matmul_workspace(dev), xpress_linear_workspace_size(), st));
    END_HANDLE_TH_ERRORS
}

// () -> address of the current device's matmul_fp8 workspace
PyObject *matmul_fp8_workspace(PyObject *, PyObject *const *, Py_ssize_t)
{
    HANDLE_TH_ERRORS
    return PyLong_FromVoidPtr(matmul_workspace(c10::cuda::current_device()));
    END_HANDLE_TH_ERRORS
}

// A workspace of process_logits on torch's current stream st, small ones kept for the
// stream's next calls, which its order keeps apart (one row of 151936: 18 us for a
// call and a wait for it, 20 to 22 with a new allocation).  A stream is known by its
// id: its handle may be a later stream's.  At most KEPT are kept, 8 MB in all.  A call
// that is captured gets one of its graph's own (graphs of one capturing stream may
// replay side by side).
at::Tensor logits_workspace(int dev, void *stream, size_t size)
{
    constexpr size_t KEEP = 256 << 10, KEPT = 32;
    // guarded by the interpreter's lock; for good: torch may end before this library
    static auto &kept = *new std::map<std::pair<int, unsigned long long>, at::Tensor>;
    const auto opt = at::TensorOptions().dtype(at::kByte).device(at::kCUDA, dev);
    const auto st = static_cast<cudaStream_t>(stream);
    cudaStreamCaptureStatus capture;
    C10_CUDA_CHECK(cudaStreamIsCapturing(st, &capture));
    if (capture != cudaStreamCaptureStatusNone || size > KEEP) return at::empty({(int64_t)size}, opt);
    unsigned long long id;
    C10_CUDA_CHECK(cudaStreamGetId(st, &id));
    const auto at = kept.find({dev, id});
    if (at != kept.end() && (size_t)at->second.numel() >= size) return at->second;
    if (kept.size() >= KEPT) kept.clear();             // each goes back to its own stream's pool
    return kept[{dev, id}] = at::empty({(int64_t)size}, opt);
}

// (logits, out, argmax_out, rows, repetition, frequency, presence, history,
//  history_offsets, prompt_len, draft, bias_ids, bias_values, bias_offsets,
//  mask, mask_row, mask_value)
PyObject *process_logits(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("process_logits", n, 17);
    const at::Tensor &x = rank2("logits", v[0]);
    const int64_t rows = PyLong_AsLongLong(v[3]);
    if (PyErr_Occurred()) return nullptr;
    const int64_t total = x.size(0), V = x.size(1);
    if (rows < 1 || total % rows) bad_value("logits: expected [n_seq * rows, V] with rows = ", rows);
    const int64_t n_seq = total / rows;
    const auto dt = x.scalar_type();
    const int dev = x.get_device();
    xpress_logits_args g{};
    g.n_seq = narrow("n_seq", n_seq);
    g.rows = narrow("rows", rows);
    g.V = narrow("V", V);
    g.dtype = dtype_code(x);
    g.logits = matrix("logits", v[0], total, V, dt, dev, g.ld);
    if (given(v[1])) g.out = matrix("out", v[1], total, V, dt, dev, g.ldo);
    if (given(v[2])) g.argmax = static_cast<int32_t *>(vector("argmax_out", v[2], total, I32, dev));
    if (given(v[4])) g.repetition = static_cast<float *>(vector("repetition", v[4], n_seq, F32, dev));
    if (given(v[5])) g.frequency = static_cast<float *>(vector("frequency", v[5], n_seq, F32, dev));
    if (given(v[6])) g.presence = static_cast<float *>(vector("presence", v[6], n_seq, F32, dev));
    if (given(v[7])) {
        if (!given(v[8])) bad_value("history needs history_offsets");
        g.history = static_cast<int32_t *>(vector("history", v[7], -1, I32, dev));
        g.n_history = tensor("history", v[7]).size(0);
        if (g.n_history == 0) g.history = nullptr;
        g.history_offsets = static_cast<int64_t *>(vector("history_offsets", v[8], n_seq + 1, I64, dev));
        if (given(v[9])) g.prompt_len = static_cast<int32_t *>(vector("prompt_len", v[9], n_seq, I32, dev));
    }
    if (given(v[10]) && rows > 1) {
        const at::Tensor &d = rank2("draft", v[10]);
        if (d.size(1) < rows - 1) bad_value("draft: expected at least ", rows - 1, " tokens per sequence");
        g.draft = static_cast<int32_t *>(matrix("draft", v[10], n_seq, d.size(1), I32, dev, g.ld_draft));
    }
    if (given(v[11])) {
        if (!given(v[12]) || !given(v[13])) bad_value("bias_ids needs bias_values and bias_offsets");
        g.bias_ids = static_cast<int32_t *>(vector("bias_ids", v[11], -1, I32, dev));
        g.n_bias = tensor("bias_ids", v[11]).size(0);
        g.bias_values = static_cast<float *>(vector("bias_values", v[12], g.n_bias, F32, dev));
        g.bias_offsets = static_cast<int64_t *>(vector("bias_offsets", v[13], n_seq + 1, I64, dev));
        if (g.n_bias == 0) g.bias_ids = nullptr;
    }
    if (given(v[14])) {
        const at::Tensor &m = rank2("mask", v[14]);
        g.mask_rows = narrow("mask rows", m.size(0));
        g.mask = static_cast<int32_t *>(matrix("mask", v[14], m.size(0), ceil_div(V, 32), I32, dev, g.ld_mask));
        if (g.mask_rows == 0) g.mask = nullptr;
        if (given(v[15])) g.mask_row = static_cast<int32_t *>(vector("mask_row", v[15], total, I32, dev));
    }
    g.mask_value = (float)PyFloat_AsDouble(v[16]);
    if (PyErr_Occurred()) return nullptr;
    void *st = current_stream(dev);
    if (total == 0) return PyLong_FromLong(XPRESS_OK);
    if (!g.argmax) return PyLong_FromLong(xpress_process_logits(&g, nullptr, 0, st));
    const size_t size = xpress_process_logits_workspace_size(g.n_seq, g.rows, g.V);
    const at::Tensor ws = logits_workspace(dev, st, size);
    return PyLong_FromLong(xpress_process_logits(&g, ws.data_ptr(), size, st));
    END_HANDLE_TH_ERRORS
}

// (logits, temperature, u, tokens_out, out, rows, top_k, top_p, min_p, mask_value)
PyObject *sample(PyObject *, PyObject *const *v, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("sample", n, 10);
    const at::Tensor &x = rank2("logits", v[0]);
    const int64_t rows = PyLong_AsLongLong(v[5]);
    if (PyErr_Occurred()) return nullptr;
    const int64_t total = x.size(0), V = x.size(1);
    if (rows < 1 || total % rows) bad_value("logits: expected [n_seq * rows, V] with rows = ", rows);
    const int64_t n_seq = total / rows;
    const auto dt = x.scalar_type();
    const int dev = x.get_device();
    xpress_sample_args g{};
    g.n_seq = narrow("n_seq", n_seq);
    g.rows = narrow("rows", rows);
    g.V = narrow("V", V);
    g.dtype = dtype_code(x);
    g.logits = matrix("logits", v[0], total, V, dt, dev, g.ld);
    g.temperature = static_cast<float *>(vector("temperature", v[1], n_seq, F32, dev));
    if (given(v[3])) {
        if (!given(v[2])) bad_value("tokens_out needs u");
        g.u = static_cast<float *>(vector("u", v[2], total, F32, dev));
        g.tokens = static_cast<int32_t *>(vector("tokens_out", v[3], total, I32, dev));
    }
    if (given(v[4])) g.out = matrix("out", v[4], total, V, dt, dev, g.ldo);
    if (given(v[6])) g.top_k = static_cast<int32_t *>(vector("top_k", v[6], n_seq, I32, dev));
    if (given(v[7])) g.top_p = static_cast<float *>(vector("top_p", v[7], n_seq, F32, dev));
    if (given(v[8])) g.min_p = static_cast<float *>(vector("min_p", v[8], n_seq, F32, dev));
    g.mask_value = (float)PyFloat_AsDouble(v[9]);
    if (PyErr_Occurred()) return nullptr;
    const int64_t es = x.element_size();
    const Place in("logits", g.logits, total, g.ld, V, es), to("out", g.out, total, g.ldo, V, es), tok("tokens_out", g.tokens, total);
    if (g.out != g.logits) apart(to, in);                            // (one place: the entry point sees to the pitch)
    apart(tok, in);
    apart(tok, to);
    for (const Place &p : {Place("temperature", g.temperature, n_seq), Place("top_k", g.top_k, n_seq), Place("top_p", g.top_p, n_seq),
                           Place("min_p", g.min_p, n_seq)}) {
        apart(to, p);
        if (rows > 1 || p.at != tok.at) apart(tok, p);               // (a row's own are read before its token is written)
    }
    const Place u("u", g.u, total);
    apart(to, u);
    if (u.at != tok.at) apart(tok, u);
    void *st = current_stream(dev);
    return PyLong_FromLong(total == 0 ? XPRESS_OK : xpress_sample(&g, st));   // empty tensors have no address
    END_HANDLE_TH_ERRORS
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(rmsnorm), FAST(quantize_weight), FAST(matmul_fp8), FAST(matmul_fp8_workspace),
                         FAST(linear), FAST(process_logits), FAST(sample), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "xpress_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_xpress_torch(void) { return PyModule_Create(&module); }
