// Python side of the calls around a block's linears: tensors -> the C entry points of trdq.h.  These calls are short (a token's
// norm runs 3 us), and reading a dozen tensors' shapes, strides and addresses through the interpreter takes longer than the launch
// (a small product: 8.3 us a call, of which 3 the launch).  Shapes and types are checked here, everything else by the entry points.
// Each function returns None, or a status and what is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <string>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "trdq.h"

namespace {

struct Bad {
    trdq_status status;
    std::string why;
};

const at::Tensor *tensor_of(PyObject *o, const char *name)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) throw Bad{TRDQ_ERR_NULL, std::string(name) + ": expected a tensor"};
    return &THPVariable_Unpack(o);
}

const at::Tensor &needed(PyObject *o, const char *name)
{
    const at::Tensor *const t = tensor_of(o, name);
    if (!t) throw Bad{TRDQ_ERR_NULL, std::string(name) + " is missing"};
    return *t;
}

// the library's number for a tensor's type; -1, which every call refuses, for another.  uint8 holds e8m0 scales
int type_of(const at::Tensor &t)
{
    switch (t.scalar_type()) {
        case at::kBFloat16: return TRDQ_BF16;
        case at::kFloat: return TRDQ_F32;
        case at::kFloat8_e4m3fn: return TRDQ_E4M3;
        case at::kFloat8_e5m2: return TRDQ_E5M2;
        case at::kFloat8_e8m0fnu: case at::kByte: return TRDQ_E8M0;
        default: return -1;
    }
}

// The device that the call will launch on; -1 where there is none (every launch fails there, and arguments are still checked).
thread_local int the_device = -1;

// A kernel that is given host memory, or another device's, faults: refused here, for every tensor of a call.
void *address(const at::Tensor &t, const char *name)
{
    if (the_device >= 0 && (!t.is_cuda() || t.get_device() != the_device))
        throw Bad{TRDQ_ERR_MISMATCH, std::string(name) + " is not on the current device"};
    return t.data_ptr();
}

int64_t up128(int64_t n) { return (n + 127) / 128 * 128; }

std::string sizes(const at::Tensor &t)
{
    std::string s = "[";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + "]";
}

struct Matrix {
    void *p = nullptr;
    int64_t ld = 0;
};

// [rows, cols] whose rows are contiguous
Matrix matrix(const at::Tensor *t, int64_t rows, int64_t cols, const char *name)
{
    if (!t) return {};
    if (t->dim() != 2 || t->size(0) != rows || t->size(1) != cols)
        throw Bad{TRDQ_ERR_SHAPE, std::string(name) + ": expected [" + std::to_string(rows) + ", " + std::to_string(cols) + "], got " + sizes(*t)};
    if (t->stride(1) != 1 && cols > 1 && rows > 0) throw Bad{TRDQ_ERR_SHAPE, std::string(name) + ": values of a row have to lie together"};
    return {address(*t, name), rows > 1 ? t->stride(0) : std::max(t->stride(0), cols)};
}

void *vector(const at::Tensor *t, int64_t n, const char *name)
{
    if (!t) return nullptr;
    if (t->dim() != 1 || t->size(0) != n || (n > 1 && t->stride(0) != 1))
        throw Bad{TRDQ_ERR_SHAPE, std::string(name) + ": expected a vector of " + std::to_string(n)};
    return address(*t, name);
}

float *gradient(PyObject *o, int64_t rows, int64_t c, const char *name)       // rows < 0: a vector
{
    const at::Tensor *const t = tensor_of(o, name);
    if (!t) return nullptr;
    const bool shape = rows < 0 ? t->dim() == 1 && t->size(0) == c : t->dim() == 2 && t->size(0) == rows && t->size(1) == c;
    if (!shape || type_of(*t) != TRDQ_F32 || !t->is_contiguous())
        throw Bad{TRDQ_ERR_SHAPE, std::string(name) + ": expected a contiguous float32 tensor of " + (rows < 0 ? "" : std::to_string(rows) + " x ") + std::to_string(c)};
    return static_cast<float *>(address(*t, name));
}

struct Workspace {
    void *p = nullptr;
    size_t bytes = 0;
};

// of any type and shape, but in one piece: its elements have to be the bytes behind its address
Workspace workspace(PyObject *o)
{
    const at::Tensor *const t = tensor_of(o, "ws");
    if (!t) return {};
    if (!t->is_contiguous()) throw Bad{TRDQ_ERR_SHAPE, "ws: expected a contiguous tensor"};
    return {address(*t, "ws"), (size_t)t->numel() * t->element_size()};
}

int64_t integer(PyObject *o)
{
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw std::exception();
    return v;
}

// a stream: None (the current one of the current device), a hipStream_t as a number, or an object that has one
void *stream_of(PyObject *o)
{
    if (o == Py_None) return static_cast<void *>(c10::hip::getCurrentHIPStream().stream());
    if (PyLong_Check(o)) return reinterpret_cast<void *>(integer(o));
    PyObject *const v = PyObject_GetAttrString(o, "cuda_stream");
    if (!v) throw std::exception();
    void *const s = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    if (!s && PyErr_Occurred()) throw std::exception();
    return s;
}

PyObject *answer(trdq_status st)
{
    if (st == TRDQ_OK) Py_RETURN_NONE;
    return Py_BuildValue("(is)", (int)st, "");
}

template <class F>
PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F &&f)
{
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
        return nullptr;
    }
    static const bool any = c10::hip::device_count() > 0;
    the_device = any ? (int)c10::hip::current_device() : -1;
    try {
        return answer(f());
    } catch (const Bad &b) {
        return Py_BuildValue("(is)", (int)b.status, b.why.c_str());
    } catch (const std::exception &e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// X, Q, S, blocks, stream
PyObject *fp8_quant(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 5, [&] {
        const at::Tensor &X = needed(a[0], "X"), &Q = needed(a[1], "Q"), &S = needed(a[2], "S");
        if (X.dim() != 2) throw Bad{TRDQ_ERR_SHAPE, "X: expected a matrix"};
        const int64_t rows = X.size(0), c = X.size(1), blocks = integer(a[3]);
        if (c > (1 << 24)) throw Bad{TRDQ_ERR_UNSUPPORTED, "X: too many channels"};
        const bool turned = blocks == TRDQ_BLOCKS_COLS || blocks == TRDQ_BLOCKS_TILES_T, tiles = blocks >= TRDQ_BLOCKS_TILES;
        const int64_t r = turned ? c : rows, k = up128(turned ? rows : c);
        const Matrix x = matrix(&X, rows, c, "X"), q = matrix(&Q, r, k, "Q"), s = matrix(&S, k / 128, tiles ? (r + 127) / 128 : r, "S");
        return trdq_fp8_quant(x.p, type_of(X), rows, (int)c, x.ld, (int)blocks, type_of(Q), q.p, q.ld, type_of(S), s.p, s.ld, stream_of(a[4]));
    });
}

// A, sa, B, sb, Y, bias, ws, stream
PyObject *fp8_gemm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 8, [&] {
        const at::Tensor &A = needed(a[0], "A"), &sa = needed(a[1], "sa"), &B = needed(a[2], "B"), &sb = needed(a[3], "sb"), &Y = needed(a[4], "Y");
        const at::Tensor *const bias = tensor_of(a[5], "bias");
        const Workspace ws = workspace(a[6]);
        if (A.dim() != 2 || B.dim() != 2 || sb.dim() != 2) throw Bad{TRDQ_ERR_SHAPE, "A, B, sb: expected matrices"};
        const int64_t M = A.size(0), K = A.size(1), N = B.size(0), nkb = (K + 127) / 128, n_sb = (N + 127) / 128;
        if (K > INT32_MAX || N > INT32_MAX) throw Bad{TRDQ_ERR_UNSUPPORTED, "A, B: too large"};
        const bool tiles = sb.size(1) == n_sb;
        if (type_of(sa) != type_of(sb)) throw Bad{TRDQ_ERR_UNSUPPORTED, "sa and sb are of different types"};
        if (bias && type_of(*bias) != TRDQ_F32) throw Bad{TRDQ_ERR_SHAPE, "bias: expected a float32 vector"};
        const Matrix ma = matrix(&A, M, K, "A"), msa = matrix(&sa, nkb, M, "sa"), mb = matrix(&B, N, K, "B"), msb = matrix(&sb, nkb, tiles ? n_sb : N, "sb"),
                     y = matrix(&Y, M, N, "Y");
        return trdq_fp8_gemm(M, (int)N, (int)K, ma.p, type_of(A), ma.ld, msa.p, msa.ld, mb.p, type_of(B), mb.ld, msb.p, msb.ld, tiles, type_of(sa),
                             static_cast<const float *>(vector(bias, N, "bias")), y.p, type_of(Y), y.ld, ws.p, ws.bytes, stream_of(a[7]));
    });
}

// pre, pre_weight, pre_bias, scale, shift, post, post_weight, post_bias, gate, eps, seg_len, seg_off from a[0] on
constexpr int kNormArgs = 12;
trdq_norm norm_of(const at::Tensor &X, PyObject *const *a, int64_t *segments_out)
{
    trdq_norm d{};
    if (X.dim() != 2) throw Bad{TRDQ_ERR_SHAPE, "X: expected a matrix"};
    if (X.size(1) > INT32_MAX) throw Bad{TRDQ_ERR_UNSUPPORTED, "X: too many channels"};
    const int64_t c = X.size(1);
    d.rows = X.size(0);
    d.c = (int)c;
    d.x_dtype = type_of(X);
    d.param_dtype = TRDQ_F32;
    d.pre = (int)integer(a[0]);
    d.post = (int)integer(a[5]);
    const double eps = PyFloat_AsDouble(a[9]);
    if (eps == -1.0 && PyErr_Occurred()) throw std::exception();
    d.eps = (float)eps;
    d.seg_len = integer(a[10]);
    int64_t segments = 1;
    if (d.seg_len > 0) {
        segments = d.rows / d.seg_len + (d.rows % d.seg_len != 0);          // (their sum may not fit 64 bits)
    } else if (const at::Tensor *const off = tensor_of(a[11], "seg_off")) {
        if (off->dim() != 1 || off->scalar_type() != at::kInt || off->size(0) > INT32_MAX) throw Bad{TRDQ_ERR_SHAPE, "seg_off: expected an int32 vector"};
        if (off->size(0) < 2) throw Bad{TRDQ_ERR_RANGE, "seg_off: expected two borders at least"};       // (none has no address: no borders)
        segments = off->size(0) - 1;
        d.n_seg = (int)segments;
        d.seg_off = static_cast<const int32_t *>(vector(off, segments + 1, "seg_off"));
    }
    const at::Tensor *const w = tensor_of(a[1], "pre_weight"), *const b = tensor_of(a[2], "pre_bias"), *const scale = tensor_of(a[3], "scale"),
                     *const shift = tensor_of(a[4], "shift"), *const w2 = tensor_of(a[6], "post_weight"), *const b2 = tensor_of(a[7], "post_bias"),
                     *const gate = tensor_of(a[8], "gate");
    int kind = -2;
    for (const at::Tensor *t : {w, b, scale, shift, w2, b2, gate})
        if (t) {
            if (kind != -2 && type_of(*t) != kind) throw Bad{TRDQ_ERR_UNSUPPORTED, "parameters of different types"};
            d.param_dtype = kind = type_of(*t);
        }
    d.pre_weight = vector(w, c, "pre_weight");
    d.pre_bias = vector(b, c, "pre_bias");
    d.post_weight = vector(w2, c, "post_weight");
    d.post_bias = vector(b2, c, "post_bias");
    if (d.rows > 0) {
        const Matrix sc = matrix(scale, segments, c, "scale"), sh = matrix(shift, segments, c, "shift");
        d.scale = sc.p; d.ld_scale = sc.ld; d.shift = sh.p; d.ld_shift = sh.ld;
        if (gate && gate->dim() == 1) {
            d.gate = vector(gate, c, "gate");
        } else {
            const Matrix g = matrix(gate, segments, c, "gate");
            d.gate = g.p; d.ld_gate = g.ld;
        }
    } else {
        // no row reads them (their segments may be those of no rows); their gradients are zeros
        d.scale = scale ? address(*scale, "scale") : nullptr; d.ld_scale = c;
        d.shift = shift ? address(*shift, "shift") : nullptr; d.ld_shift = c;
        d.gate = gate ? address(*gate, "gate") : nullptr; d.ld_gate = gate && gate->dim() == 2 ? c : 0;
    }
    *segments_out = segments;
    return d;
}

void same_type(const at::Tensor *t, const at::Tensor &like, const char *name)
{
    if (t && t->scalar_type() != like.scalar_type()) throw Bad{TRDQ_ERR_UNSUPPORTED, std::string(name) + " has to be of the stream's type"};
}
void is_bf16(const at::Tensor *t, const char *name)
{
    if (t && t->scalar_type() != at::kBFloat16) throw Bad{TRDQ_ERR_UNSUPPORTED, std::string(name) + " has to be bf16"};
}

// X, Xout, H, Y, codes, code_scales, <norm>, stream
PyObject *block_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 7 + kNormArgs, [&] {
        const at::Tensor &X = needed(a[0], "X");
        const at::Tensor *const Xo = tensor_of(a[1], "Xout"), *const H = tensor_of(a[2], "H"), *const Y = tensor_of(a[3], "Y"),
                         *const codes = tensor_of(a[4], "codes"), *const cs = tensor_of(a[5], "code_scales");
        int64_t segments = 0;
        const trdq_norm d = norm_of(X, a + 6, &segments);
        is_bf16(Y, "Y");
        same_type(Xo, X, "Xout");
        if (codes && H) throw Bad{TRDQ_ERR_SHAPE, "H and codes: one of them"};
        const Matrix x = matrix(&X, d.rows, d.c, "X"), y = matrix(Y, d.rows, d.c, "Y"), xo = matrix(Xo, d.rows, d.c, "Xout");
        const Matrix h = codes ? matrix(codes, d.rows, up128(d.c), "codes") : matrix(H, d.rows, d.c, "H"),
                     s = codes ? matrix(cs, up128(d.c) / 128, d.rows, "code_scales") : Matrix{};
        int ht = TRDQ_BF16;
        if (codes) ht = type_of(*codes) == TRDQ_E4M3 ? TRDQ_E4M3 : -1;
        else if (H) ht = type_of(*H) == TRDQ_BF16 || type_of(*H) == TRDQ_F32 ? type_of(*H) : -1;
        return trdq_block_norm(&d, x.p, x.ld, y.p, y.ld, xo.p, xo.ld, ht, h.p, h.ld, cs ? type_of(*cs) : -1, s.p, s.ld, stream_of(a[6 + kNormArgs]));
    });
}

// dX, dY, Xout, dH, Y, dXout, dscale, dshift, dgate, dpre_weight, dpre_bias, dpost_weight, dpost_bias, ws, <norm>, stream
PyObject *block_norm_bwd(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded(n, 15 + kNormArgs, [&] {
        const at::Tensor &X = needed(a[2], "Xout");
        const at::Tensor *const dX = tensor_of(a[0], "dX"), *const dY = tensor_of(a[1], "dY"), *const dH = tensor_of(a[3], "dH"),
                         *const Y = tensor_of(a[4], "Y"), *const dXo = tensor_of(a[5], "dXout");
        const Workspace ws = workspace(a[13]);
        int64_t segments = 0;
        const trdq_norm d = norm_of(X, a + 14, &segments);
        same_type(dX, X, "dX");
        same_type(dXo, X, "dXout");
        is_bf16(dH, "dH");
        is_bf16(Y, "Y");
        is_bf16(dY, "dY");
        trdq_norm_grads g{};
        auto put = [&](const void *&p, int64_t &ld, const at::Tensor *t, const char *name) {
            const Matrix m = matrix(t, d.rows, d.c, name);
            p = m.p;
            ld = m.ld;
        };
        const void *dx = nullptr, *dy = nullptr;
        put(g.Xout_dev, g.ldxo, &X, "Xout");
        put(g.Y_dev, g.ldy, Y, "Y");
        put(g.dXout_dev, g.lddxo, dXo, "dXout");
        put(g.dH_dev, g.lddh, dH, "dH");
        put(dx, g.lddx, dX, "dX");
        put(dy, g.lddy, dY, "dY");
        g.dX_dev = const_cast<void *>(dx);
        g.dY_dev = const_cast<void *>(dy);
        const at::Tensor *const gate = tensor_of(a[14 + 8], "gate");
        g.dscale_dev = gradient(a[6], segments, d.c, "dscale");
        g.dshift_dev = gradient(a[7], segments, d.c, "dshift");
        g.dgate_dev = gradient(a[8], gate && gate->dim() == 2 ? segments : -1, d.c, "dgate");
        // (an expanded vector: the library would take its gradient for a vector's too, and leave the other segments' unwritten)
        if (g.dgate_dev && gate && gate->dim() == 2 && segments > 1 && d.ld_gate == 0)
            throw Bad{TRDQ_ERR_SHAPE, "dgate: the gate is one vector for every segment; give it and its gradient as vectors"};
        g.dpre_weight_dev = gradient(a[9], -1, d.c, "dpre_weight");
        g.dpre_bias_dev = gradient(a[10], -1, d.c, "dpre_bias");
        g.dpost_weight_dev = gradient(a[11], -1, d.c, "dpost_weight");
        g.dpost_bias_dev = gradient(a[12], -1, d.c, "dpost_bias");
        return trdq_block_norm_bwd(&d, &g, ws.p, ws.bytes, stream_of(a[14 + kNormArgs]));
    });
}

template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
PyCFunction fast() { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)); }

PyMethodDef methods[] = {{"fp8_quant", fast<fp8_quant>(), METH_FASTCALL, nullptr},
                         {"fp8_gemm", fast<fp8_gemm>(), METH_FASTCALL, nullptr},
                         {"block_norm", fast<block_norm>(), METH_FASTCALL, nullptr},
                         {"block_norm_bwd", fast<block_norm_bwd>(), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_trdq_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__trdq_calls() { return PyModule_Create(&module); }
