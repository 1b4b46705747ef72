// The feed-forward and the training step's operators as Python functions on torch tensors: argument checks, outputs and workspaces
// from torch's allocator, and the call of the C entry point, in one C function each.  (Through ctypes and
// torch's Python functions the same steps took 9 to 16 us a call, several times the kernels' own time for a
// single token.)  Every step of the computation is in libspingtp.so, whose entry points bind() is given.
//
// Functions take the raw stream last and return tensors; a Block8's two tensors come as a pair.  A refused
// argument raises ValueError; a status other than 0 raises the error class that bind() was given.
#include <ATen/ATen.h>
#include <Python.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <exception>
#include <initializer_list>
#include <stdexcept>
#include <string>
#include <tuple>
#include <utility>
#include <vector>

#include "overlap.h"
#include "spingtp.h"

namespace {

struct Refused : std::runtime_error {
    using std::runtime_error::runtime_error;
};
struct Failed {
    spingtp_status status;
    const char* where;
};
struct PythonError {};  // already set

PyObject* error_class = nullptr;  // SpinGTPError(status, where)

struct Entries {
    decltype(&spingtp_pack8) pack8;
    decltype(&spingtp_unpack8) unpack8;
    decltype(&spingtp_rms_norm) rms_norm;
    decltype(&spingtp_rms_norm_backward) rms_norm_backward;
    decltype(&spingtp_rms_norm_backward_workspace_size) rms_norm_backward_workspace_size;
    decltype(&spingtp_matmul8) matmul8;
    decltype(&spingtp_gated_forward) gated_forward;
    decltype(&spingtp_gated_forward_workspace_size) gated_forward_workspace_size;
    decltype(&spingtp_gated_forward8) gated_forward8;
    decltype(&spingtp_gated_forward8_workspace_size) gated_forward8_workspace_size;
    decltype(&spingtp_gated_backward) gated_backward;
    decltype(&spingtp_gated_backward_workspace_size) gated_backward_workspace_size;
    decltype(&spingtp_linear_forward) linear_forward;
    decltype(&spingtp_linear_forward_workspace_size) linear_forward_workspace_size;
    decltype(&spingtp_linear_forward8) linear_forward8;
    decltype(&spingtp_linear_forward8_workspace_size) linear_forward8_workspace_size;
    decltype(&spingtp_linear_backward) linear_backward;
    decltype(&spingtp_linear_backward_workspace_size) linear_backward_workspace_size;
    decltype(&spingtp_embedding) embedding;
    decltype(&spingtp_sort_index) sort_index;
    decltype(&spingtp_sort_index_workspace_size) sort_index_workspace_size;
    decltype(&spingtp_embedding_backward) embedding_backward;
    decltype(&spingtp_embedding_backward_workspace_size) embedding_backward_workspace_size;
    decltype(&spingtp_adamw) adamw;
} lib;

int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }

std::string shape_text(int64_t rows, int64_t columns) {
    return "[" + std::to_string(rows) + ", " + std::to_string(columns) + "]";
}

typedef PyObject* const* Args;

// ---------------------------------------------------------------- arguments

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) throw Refused(std::string(name) + " must be a tensor");
    return THPVariable_Unpack(o);
}

int64_t integer(PyObject* o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PythonError{};
    return v;
}

bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw PythonError{};
    return v != 0;
}

struct Matrix {
    void* p = nullptr;
    int64_t rows = 0, columns = 0, ld = 0;
    at::ScalarType type = at::kFloat;
    const at::Tensor* t = nullptr;
};

// A [rows, columns] tensor of fp32 or bf16 with contiguous rows; `like`: of its device and type.
Matrix matrix(PyObject* o, const char* name, const Matrix* like = nullptr, int64_t rows = -1, int64_t columns = -1) {
    const at::Tensor& t = tensor(o, name);
    const std::string n = name;
    if (t.dim() != 2) throw Refused(n + " must be a 2-D tensor");
    Matrix m;
    m.t = &t;
    m.type = t.scalar_type();
    m.rows = t.size(0);
    m.columns = t.size(1);
    if (m.type != at::kFloat && m.type != at::kBFloat16) throw Refused(n + " must be fp32 or bf16");
    if (!t.is_cuda()) throw Refused(n + " must be on a GPU");
    if (like != nullptr) {
        if (m.type != like->type) throw Refused(n + " must have the type of the other operands");
        if (t.device() != like->t->device()) throw Refused(n + " must be on the device of the other operands");
    }
    if ((rows >= 0 && m.rows != rows) || (columns >= 0 && m.columns != columns))
        throw Refused(n + " must be " + shape_text(rows >= 0 ? rows : m.rows, columns >= 0 ? columns : m.columns) +
                      ", not " + shape_text(m.rows, m.columns));
    if (m.columns > 1 && t.stride(1) != 1) throw Refused(n + " must have contiguous rows");
    m.ld = m.rows > 1 ? t.stride(0) : m.columns;  // the stride of a single row says nothing
    if (m.ld < m.columns) throw Refused(n + " has overlapping rows");
    if (m.ld < 1) m.ld = 1;
    m.p = t.data_ptr();
    return m;
}

void need_bf16(const Matrix& m, const char* name) {
    if (m.type != at::kBFloat16) throw Refused(std::string(name) + " must be bf16");
}

float* vector(PyObject* o, const char* name, int64_t n, const at::Device& device) {
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() != at::kFloat || t.dim() != 1 || t.size(0) != n || t.device() != device ||
        (n > 1 && t.stride(0) != 1))
        throw Refused(std::string(name) + " must be a contiguous fp32 [" + std::to_string(n) +
                      "] tensor beside the other operands");
    return t.data_ptr<float>();
}

// The tensors of a Block8, whose constructor has checked them.
struct Block {
    void* values = nullptr;
    void* scales = nullptr;
    const at::Tensor* t = nullptr;
};
Block block(PyObject* values, PyObject* scales) {
    Block b;
    b.t = &tensor(values, "values");
    b.values = b.t->data_ptr();
    b.scales = tensor(scales, "scales").data_ptr();
    return b;
}

// values, scales, R, D: refuses what is no Block8 of that shape
void check_block(PyObject* values, PyObject* scales, int64_t R, int64_t D) {
    const at::Tensor& v = tensor(values, "values");
    const at::Tensor& s = tensor(scales, "scales");
    if (R < 0 || D < 0) throw Refused("no matrix has the shape " + shape_text(R, D));
    const int64_t pitch = up(D, 128), spitch = up(D, 512) / 128;
    if (v.scalar_type() != at::kFloat8_e4m3fn || v.dim() != 2 || v.size(0) != R || v.size(1) != pitch ||
        !v.is_contiguous() || !v.is_cuda())
        throw Refused("values must be a contiguous float8_e4m3fn " + shape_text(R, pitch) + " device tensor");
    if (s.scalar_type() != at::kFloat8_e8m0fnu || s.dim() != 2 || s.size(0) != R || s.size(1) != spitch ||
        !s.is_contiguous() || s.device() != v.device())
        throw Refused("scales must be a contiguous float8_e8m0fnu " + shape_text(R, spitch) + " tensor beside the values");
}
PyObject* check_block(Args a) {
    check_block(a[0], a[1], integer(a[2]), integer(a[3]));
    Py_RETURN_NONE;
}

// ---------------------------------------------------------------- results

at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, const at::Tensor& beside) {
    return at::empty(shape, beside.options().dtype(type));
}
struct NewBlock {
    at::Tensor values, scales;
    NewBlock() = default;
    NewBlock(int64_t R, int64_t D, const at::Tensor& beside)
        : values(empty({R, up(D, 128)}, at::kFloat8_e4m3fn, beside)),
          scales(empty({R, up(D, 512) / 128}, at::kFloat8_e8m0fnu, beside)) {}
    void* v() const { return values.defined() ? values.data_ptr() : nullptr; }
    void* s() const { return scales.defined() ? scales.data_ptr() : nullptr; }
};
at::Tensor workspace(size_t bytes, const at::Tensor& beside) {
    return bytes == 0 ? at::Tensor() : empty({static_cast<int64_t>(bytes)}, at::kByte, beside);
}
void* address(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

PyObject* wrap(const at::Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
PyObject* tuple(std::initializer_list<PyObject*> parts) {
    PyObject* r = PyTuple_New(static_cast<Py_ssize_t>(parts.size()));
    Py_ssize_t i = 0;
    bool whole = r != nullptr;
    for (PyObject* p : parts) {
        whole = whole && p != nullptr;
        if (r != nullptr)
            PyTuple_SET_ITEM(r, i++, p);
        else
            Py_XDECREF(p);
    }
    if (!whole) {
        Py_XDECREF(r);
        throw PythonError{};
    }
    return r;
}
PyObject* wrap(const NewBlock& b) { return tuple({wrap(b.values), wrap(b.scales)}); }

// Autograd sees that a given output is written (before the launch: it refuses what may not be).
void writes(const Matrix& out) { out.t->unsafeGetTensorImpl()->bump_version(); }

void done(spingtp_status s, const char* where) {
    if (s != SPINGTP_OK) throw Failed{s, where};
}
void* stream_of(PyObject* o) { return reinterpret_cast<void*>(static_cast<intptr_t>(integer(o))); }
spingtp_dtype dtype_of(at::ScalarType t) { return t == at::kFloat ? SPINGTP_FP32 : SPINGTP_BF16; }

// ---------------------------------------------------------------- operators

// x, transpose (0 rows, 1 columns, 2 both), stream -> (rows | None, columns | None)
PyObject* pack8(Args a) {
    const Matrix x = matrix(a[0], "x");
    const int64_t how = integer(a[1]);
    if (x.columns < 1) throw Refused("no blocks in a matrix of shape " + shape_text(x.rows, x.columns));
    NewBlock rows, columns;
    if (how != 1) rows = NewBlock(x.rows, x.columns, *x.t);
    if (how != 0) columns = NewBlock(x.columns, x.rows, *x.t);
    done(lib.pack8(dtype_of(x.type), x.p, x.ld, rows.v(), rows.s(), columns.v(), columns.s(), x.rows, x.columns,
                   stream_of(a[2])),
         "spingtp_pack8");
    if (how == 0) return wrap(rows);
    if (how == 1) return wrap(columns);
    return tuple({wrap(rows), wrap(columns)});
}

// values, scales, R, D, bf16, out | None, stream -> out
PyObject* unpack8(Args a) {
    const Block b = block(a[0], a[1]);
    const int64_t R = integer(a[2]), D = integer(a[3]);
    const at::ScalarType type = truth(a[4]) ? at::kBFloat16 : at::kFloat;
    at::Tensor made;
    Matrix out, like;
    like.t = b.t;
    like.type = type;
    if (a[5] != Py_None) {
        out = matrix(a[5], "out", &like, R, D);
        writes(out);
    } else {
        made = empty({R, D}, type, *b.t);
        out.p = made.data_ptr();
        out.ld = D;
    }
    if (D > 0)  // else a transposed matrix of no rows
        done(lib.unpack8(b.values, b.scales, dtype_of(type), out.p, out.ld, R, D, stream_of(a[6])), "spingtp_unpack8");
    return made.defined() ? wrap(made) : Py_NewRef(a[5]);
}

// x, gain, residual | None, eps, out8, stream -> (y, h | None, rstd)
PyObject* rms_norm(Args a) {
    const Matrix x = matrix(a[0], "x");
    const int64_t R = x.rows, D = x.columns;
    if (D < 1) throw Refused("x has no columns");
    const float* gain = vector(a[1], "gain", D, x.t->device());
    const double eps = PyFloat_AsDouble(a[3]);
    if (eps == -1.0 && PyErr_Occurred()) throw PythonError{};
    if (!(eps >= 0)) throw Refused("eps must not be negative");
    Matrix r;
    at::Tensor h, y;
    NewBlock y8;
    if (a[2] != Py_None) {
        r = matrix(a[2], "residual", &x, R, D);
        h = empty({R, D}, x.type, *x.t);
    }
    if (truth(a[4]))
        y8 = NewBlock(R, D, *x.t);
    else
        y = empty({R, D}, x.type, *x.t);
    const at::Tensor rstd = empty({R}, at::kFloat, *x.t);
    done(lib.rms_norm(dtype_of(x.type), x.p, x.ld, r.p, r.ld, gain, static_cast<float>(eps), address(h), D, address(y), D,
                      y8.v(), y8.s(), rstd.data_ptr<float>(), R, D, stream_of(a[5])),
         "spingtp_rms_norm");
    return tuple({y.defined() ? wrap(y) : wrap(y8), wrap(h), wrap(rstd)});
}

// grad_y, h, rstd, gain, grad_h | None, need_gain, stream -> (grad_x, grad_gain | None)
PyObject* rms_norm_backward(Args a) {
    const Matrix dy = matrix(a[0], "grad_y");
    const int64_t R = dy.rows, D = dy.columns;
    if (D < 1) throw Refused("grad_y has no columns");
    const Matrix h = matrix(a[1], "h", &dy, R, D);
    const float* rstd = vector(a[2], "rstd", R, dy.t->device());
    const float* gain = vector(a[3], "gain", D, dy.t->device());
    Matrix gh;
    if (a[4] != Py_None) gh = matrix(a[4], "grad_h", &dy, R, D);
    const at::Tensor dx = empty({R, D}, dy.type, *dy.t);
    at::Tensor dgain, ws;
    size_t bytes = 0;
    if (truth(a[5])) {
        dgain = empty({D}, at::kFloat, *dy.t);
        done(lib.rms_norm_backward_workspace_size(R, D, &bytes), "spingtp_rms_norm_backward_workspace_size");
        ws = workspace(bytes, *dy.t);
    }
    done(lib.rms_norm_backward(dtype_of(dy.type), dy.p, dy.ld, h.p, h.ld, rstd, gain, gh.p, gh.ld, dx.data_ptr(), D,
                               static_cast<float*>(address(dgain)), address(ws), bytes, R, D, stream_of(a[6])),
         "spingtp_rms_norm_backward");
    return tuple({wrap(dx), wrap(dgain)});
}

// a's values, scales, b's, M, N, K, bf16, out | None, stream -> out
PyObject* matmul8(Args a) {
    const Block x = block(a[0], a[1]), w = block(a[2], a[3]);
    const int64_t M = integer(a[4]), N = integer(a[5]), K = integer(a[6]);
    const at::ScalarType type = truth(a[7]) ? at::kBFloat16 : at::kFloat;
    if (x.t->device() != w.t->device()) throw Refused("a and b must be on one device");
    at::Tensor made;
    Matrix out, like;
    like.t = x.t;
    like.type = type;
    if (a[8] != Py_None) {
        out = matrix(a[8], "out", &like, M, N);
        writes(out);
    } else {
        made = empty({M, N}, type, *x.t);
        out.p = made.data_ptr();
        out.ld = N > 0 ? N : 1;
    }
    if (K == 0)  // sums of no terms: a gradient over an empty batch
        (made.defined() ? made : *out.t).zero_();
    else
        done(lib.matmul8(x.values, x.scales, w.values, w.scales, dtype_of(type), out.p, out.ld, M, N, K,
                         stream_of(a[9])),
             "spingtp_matmul8");
    return made.defined() ? wrap(made) : Py_NewRef(a[8]);
}

// The weights [F, K] of a gated block, at one row stride.
std::pair<Matrix, Matrix> weights(PyObject* gate, PyObject* up_, const Matrix& like, int64_t F, int64_t K) {
    const Matrix g = matrix(gate, "w_gate", &like, F, K);
    const Matrix u = matrix(up_, "w_up", &like, g.rows, g.columns);
    if (g.columns < 1 || g.rows < 1) throw Refused("the weights are empty");
    if (g.ld != u.ld) throw Refused("w_gate and w_up must have the same row stride");
    return {g, u};
}

// x, w_gate, w_up, act, save, stream -> (h, x as a pair | None, g | pair | None, u | pair | None)
PyObject* gated(Args a) {
    const Matrix x = matrix(a[0], "x");
    need_bf16(x, "x");
    const int64_t M = x.rows, K = x.columns;
    const auto w = weights(a[1], a[2], x, -1, K);
    const int64_t F = w.first.rows;
    const auto act = integer(a[3]);
    const auto save = integer(a[4]);
    void* stream = stream_of(a[5]);
    const at::Tensor h = empty({M, F}, at::kBFloat16, *x.t);
    at::Tensor g, u;
    NewBlock x8, g8, u8;
    if (save == SPINGTP_SAVE_BF16) {
        g = empty({M, F}, at::kBFloat16, *x.t);
        u = empty({M, F}, at::kBFloat16, *x.t);
    } else if (save == SPINGTP_SAVE_BLOCK8) {
        x8 = NewBlock(M, K, *x.t);
        g8 = NewBlock(M, F, *x.t);
        u8 = NewBlock(M, F, *x.t);
        done(lib.pack8(SPINGTP_BF16, x.p, x.ld, x8.v(), x8.s(), nullptr, nullptr, M, K, stream), "spingtp_pack8");
    }
    size_t bytes = 0;
    done(lib.gated_forward_workspace_size(M, K, F, x.ld, w.first.ld, save, &bytes),
         "spingtp_gated_forward_workspace_size");
    const at::Tensor ws = workspace(bytes, *x.t);
    const bool in8 = save == SPINGTP_SAVE_BLOCK8;
    done(lib.gated_forward(act, x.p, x.ld, w.first.p, w.second.p, w.first.ld, h.data_ptr(), F, save,
                           in8 ? g8.v() : address(g), g8.s(), in8 ? u8.v() : address(u), u8.s(), address(ws), bytes, M, K,
                           F, stream),
         "spingtp_gated_forward");
    if (in8) return tuple({wrap(h), wrap(x8), wrap(g8), wrap(u8)});
    return tuple({wrap(h), Py_NewRef(Py_None), wrap(g), wrap(u)});
}

// x's, w_gate's and w_up's values and scales, M, K, F, act, out8, stream -> h | pair
PyObject* gated8(Args a) {
    const Block x = block(a[0], a[1]), g = block(a[2], a[3]), u = block(a[4], a[5]);
    if (x.t->device() != g.t->device() || x.t->device() != u.t->device())
        throw Refused("x and the weights must be on one device");
    const int64_t M = integer(a[6]), K = integer(a[7]), F = integer(a[8]);
    const auto act = integer(a[9]);
    const bool out8 = truth(a[10]);
    at::Tensor h, ws;
    NewBlock h8;
    size_t bytes = 0;
    if (out8) {
        h8 = NewBlock(M, F, *x.t);
        done(lib.gated_forward8_workspace_size(M, K, F, 1, &bytes), "spingtp_gated_forward8_workspace_size");
        ws = workspace(bytes, *x.t);
    } else {
        h = empty({M, F}, at::kBFloat16, *x.t);
    }
    done(lib.gated_forward8(act, x.values, x.scales, g.values, g.scales, u.values, u.scales, out8 ? h8.v() : address(h), F,
                            h8.s(), address(ws), bytes, M, K, F, stream_of(a[11])),
         "spingtp_gated_forward8");
    return out8 ? wrap(h8) : wrap(h);
}

// grad_h, save, x | (values, scales, columns), g, u likewise, w_gate, w_up, act, need_x, need_w, stream
// -> (grad_x | None, grad_w [2F, K] | None)
PyObject* gated_backward(Args a) {
    const Matrix dh = matrix(a[0], "grad_h");
    need_bf16(dh, "grad_h");
    const int64_t M = dh.rows, F = dh.columns;
    const auto save = integer(a[1]);
    const auto w = weights(a[5], a[6], dh, F, -1);
    const int64_t K = w.first.columns;
    Matrix kept[3];
    Block kept8[3];
    const char* const names[3] = {"saved.x", "saved.g", "saved.u"};
    for (int i = 0; i < 3; ++i) {
        const int64_t columns = i == 0 ? K : F;
        if (save == SPINGTP_SAVE_BLOCK8) {
            if (!PyTuple_Check(a[2 + i]) || PyTuple_GET_SIZE(a[2 + i]) != 3) throw Refused(std::string(names[i]) + " must be a Block8");
            kept8[i] = block(PyTuple_GET_ITEM(a[2 + i], 0), PyTuple_GET_ITEM(a[2 + i], 1));
            if (kept8[i].t->size(0) != M || integer(PyTuple_GET_ITEM(a[2 + i], 2)) != columns ||
                kept8[i].t->device() != dh.t->device())
                throw Refused(std::string(names[i]) + " must be " + shape_text(M, columns) + " beside grad_h");
            kept[i].p = kept8[i].values;
            kept[i].ld = columns;
        } else {
            kept[i] = matrix(a[2 + i], names[i], &dh, M, columns);
            if (i > 0 && kept[i].ld != F) throw Refused(std::string(names[i]) + " must be dense");
        }
    }
    at::Tensor dx, dw;
    if (truth(a[8])) dx = empty({M, K}, at::kBFloat16, *dh.t);
    if (truth(a[9])) dw = empty({2 * F, K}, at::kBFloat16, *dh.t);
    size_t bytes = 0;
    done(lib.gated_backward_workspace_size(M, K, F, kept[0].ld, w.first.ld, save == SPINGTP_SAVE_BLOCK8, &bytes),
         "spingtp_gated_backward_workspace_size");
    const at::Tensor ws = workspace(bytes, *dh.t);
    done(lib.gated_backward(integer(a[7]), dh.p, dh.ld, save, kept[1].p, kept8[1].scales,
                            kept[2].p, kept8[2].scales, kept[0].p, kept[0].ld, kept8[0].scales, w.first.p, w.second.p,
                            w.first.ld, address(dx), K, address(dw), address(ws), bytes, M, K, F, stream_of(a[10])),
         "spingtp_gated_backward");
    return tuple({wrap(dx), wrap(dw)});
}

Rows rows_of(const Matrix& m) { return Rows(m.p, m.rows, m.columns, m.ld, m.t->element_size()); }
Rows rows_of(const at::Tensor& dense) { return Rows(dense.data_ptr(), 1, dense.numel(), dense.numel(), dense.element_size()); }
template <typename T>
void apart(const Matrix& out, const T& other, const char* name) {
    if (overlap(rows_of(out), rows_of(other))) throw Refused(std::string("out overlaps ") + name);
}

// What follows a linear layer's product: bias [N] | None, residual [M, N] | None and y [M, N], new or given.
struct LinearTail {
    const float* bias = nullptr;
    Matrix r, y;
    at::Tensor made;
    LinearTail(PyObject* bias_, PyObject* residual, PyObject* out, at::ScalarType type, const at::Tensor& beside, int64_t M,
               int64_t N) {
        Matrix like;
        like.t = &beside;
        like.type = type;
        if (bias_ != Py_None) bias = vector(bias_, "bias", N, beside.device());
        if (residual != Py_None) r = matrix(residual, "residual", &like, M, N);
        if (out != Py_None) {
            y = matrix(out, "out", &like, M, N);
            if (bias != nullptr) apart(y, tensor(bias_, "bias"), "bias");
            // the residual itself may be written: each of its elements is read where its output is made, before it
            if (residual != Py_None && (r.p != y.p || r.ld != y.ld)) apart(y, r, "residual");
        } else {
            made = empty({M, N}, type, beside);
            y.p = made.data_ptr();
            y.ld = N;
        }
    }
    PyObject* result(PyObject* out) const { return made.defined() ? wrap(made) : Py_NewRef(out); }
};

// x, w, bias | None, act, residual | None, save, bf16, out | None, stream -> (y, z | None)
PyObject* linear(Args a) {
    const Matrix x = matrix(a[0], "x");
    need_bf16(x, "x");
    const int64_t M = x.rows, K = x.columns;
    const Matrix w = matrix(a[1], "w", &x, -1, K);
    const int64_t N = w.rows;
    if (N < 1 || K < 1) throw Refused("the weights are empty");
    const auto act = integer(a[3]);
    const at::ScalarType type = truth(a[6]) ? at::kBFloat16 : at::kFloat;
    const LinearTail t(a[2], a[4], a[7], type, *x.t, M, N);
    if (a[7] != Py_None) {
        apart(t.y, x, "x");
        apart(t.y, w, "w");
        writes(t.y);
    }
    at::Tensor z;
    if (truth(a[5]) && act != SPINGTP_IDENTITY) z = empty({M, N}, at::kBFloat16, *x.t);
    size_t bytes = 0;
    done(lib.linear_forward_workspace_size(x.p, x.ld, w.p, w.ld, M, K, N, &bytes),
         "spingtp_linear_forward_workspace_size");
    const at::Tensor ws = workspace(bytes, *x.t);
    done(lib.linear_forward(act, x.p, x.ld, w.p, w.ld, t.bias, dtype_of(type), t.r.p, t.r.ld, t.y.p, t.y.ld, address(z),
                            address(ws), bytes, M, K, N, stream_of(a[8])),
         "spingtp_linear_forward");
    return tuple({t.result(a[7]), wrap(z)});
}

// x's and w's values and scales, M, K, N, bias | None, act, residual | None, bf16, out | None, stream -> y
PyObject* linear8(Args a) {
    const Block x = block(a[0], a[1]), w = block(a[2], a[3]);
    if (x.t->device() != w.t->device()) throw Refused("x and w must be on one device");
    const int64_t M = integer(a[4]), K = integer(a[5]), N = integer(a[6]);
    if (N < 1 || K < 1) throw Refused("the weights are empty");
    const at::ScalarType type = truth(a[10]) ? at::kBFloat16 : at::kFloat;
    const LinearTail t(a[7], a[9], a[11], type, *x.t, M, N);
    if (a[11] != Py_None) {
        for (int i = 0; i < 4; ++i) apart(t.y, tensor(a[i], "a block"), i < 2 ? "x" : "w");
        writes(t.y);
    }
    size_t bytes = 0;
    done(lib.linear_forward8_workspace_size(M, K, N, &bytes), "spingtp_linear_forward8_workspace_size");
    const at::Tensor ws = workspace(bytes, *x.t);
    done(lib.linear_forward8(integer(a[8]), x.values, x.scales, w.values, w.scales, t.bias, dtype_of(type), t.r.p, t.r.ld,
                             t.y.p, t.y.ld, address(ws), bytes, M, K, N, stream_of(a[12])),
         "spingtp_linear_forward8");
    return t.result(a[11]);
}

// grad_y, x, z | None, act, w, need_x, need_w, need_bias, bf16, stream -> (grad_x | None, grad_w | None, grad_bias | None)
PyObject* linear_backward(Args a) {
    const Matrix dy = matrix(a[0], "grad_y");
    const int64_t M = dy.rows, N = dy.columns;
    Matrix like = dy;
    like.type = at::kBFloat16;
    const Matrix x = matrix(a[1], "saved.x", &like, M, -1);
    const int64_t K = x.columns;
    const Matrix w = matrix(a[4], "w", &like, N, K);
    if (N < 1 || K < 1) throw Refused("the weights are empty");
    const auto act = integer(a[3]);
    Matrix z;
    if (act != SPINGTP_IDENTITY) {
        z = matrix(a[2], "saved.z", &like, M, N);
        if (M > 1 && z.ld != N) throw Refused("saved.z must be dense");
    }
    const at::ScalarType type = truth(a[8]) ? at::kBFloat16 : at::kFloat;
    at::Tensor dx, dw, db;
    if (truth(a[5])) dx = empty({M, K}, at::kBFloat16, *dy.t);
    if (truth(a[6])) dw = empty({N, K}, type, *dy.t);
    if (truth(a[7])) db = empty({N}, at::kFloat, *dy.t);
    float* const bias = static_cast<float*>(address(db));
    size_t bytes = 0;
    done(lib.linear_backward_workspace_size(act, dtype_of(dy.type), dy.p, dy.ld, x.p, x.ld, w.p, w.ld, address(dx),
                                            address(dw), bias, M, K, N, &bytes),
         "spingtp_linear_backward_workspace_size");
    const at::Tensor ws = workspace(bytes, *dy.t);
    done(lib.linear_backward(act, dtype_of(dy.type), dy.p, dy.ld, z.p, x.p, x.ld, w.p, w.ld, address(dx), K,
                             dtype_of(type), address(dw), bias, address(ws), bytes, M, K, N, stream_of(a[9])),
         "spingtp_linear_backward");
    return tuple({wrap(dx), wrap(dw), wrap(db)});
}

double number(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PythonError{};
    return v;
}

// A contiguous [n] tensor of int64 or int32 on a device (`beside`: on its device).
struct Index {
    const at::Tensor* t;
    const void* p;
    int64_t n;
    int bytes;
    Index(PyObject* o, const char* name, const at::Tensor* beside) : t(&tensor(o, name)) {
        const std::string text = name;
        const at::ScalarType type = t->scalar_type();
        if (type != at::kLong && type != at::kInt) throw Refused(text + " must be int64 or int32");
        if (t->dim() != 1) throw Refused(text + " must be a 1-D tensor");
        if (!t->is_cuda()) throw Refused(text + " must be on a GPU");
        if (beside != nullptr && t->device() != beside->device())
            throw Refused(text + " must be on the device of the other operands");
        n = t->size(0);
        if (n > 1 && t->stride(0) != 1) throw Refused(text + " must be contiguous");
        bytes = type == at::kLong ? 8 : 4;
        p = t->data_ptr();
    }
};

// table, index, scale, stream -> out
PyObject* embedding(Args a) {
    const Matrix table = matrix(a[0], "table");
    const Index index(a[1], "index", table.t);
    const double scale = number(a[2]);
    if (table.rows < 1 || table.columns < 1) throw Refused("the table is empty");
    const at::Tensor out = empty({index.n, table.columns}, table.type, *table.t);
    done(lib.embedding(dtype_of(table.type), table.p, table.ld, index.p, index.bytes, static_cast<float>(scale),
                       out.data_ptr(), table.columns, index.n, table.rows, table.columns, stream_of(a[3])),
         "spingtp_embedding");
    return wrap(out);
}

// index sorted for a table of V rows: (order, rows)
std::pair<at::Tensor, at::Tensor> sorted(const Index& index, int64_t V, void* stream) {
    if (V < 1) throw Refused("V must be positive");
    size_t bytes = 0;
    done(lib.sort_index_workspace_size(index.n, V, &bytes), "spingtp_sort_index_workspace_size");
    const at::Tensor order = empty({index.n}, at::kInt, *index.t), rows = empty({index.n}, at::kInt, *index.t);
    const at::Tensor ws = workspace(bytes, *index.t);
    done(lib.sort_index(index.p, index.bytes, order.data_ptr<int32_t>(), rows.data_ptr<int32_t>(), address(ws), bytes,
                        index.n, V, stream),
         "spingtp_sort_index");
    return {order, rows};
}

// index, V, stream -> (order, rows)
PyObject* sort_index(Args a) {
    const Index index(a[0], "index", nullptr);
    const auto pair = sorted(index, integer(a[1]), stream_of(a[2]));
    return tuple({wrap(pair.first), wrap(pair.second)});
}

// grad, index | order, None | rows, V, scale, bf16 | None, stream -> [V, D]
PyObject* embedding_backward(Args a) {
    const Matrix grad = matrix(a[0], "grad");
    const int64_t D = grad.columns, V = integer(a[3]);
    if (D < 1) throw Refused("grad has no columns");
    if (V < 1) throw Refused("V must be positive");
    const Index index(a[1], "index", grad.t);
    if (index.n != grad.rows)
        throw Refused("index must have " + std::to_string(grad.rows) + " entries, not " + std::to_string(index.n));
    const double scale = number(a[4]);
    const at::ScalarType type = a[5] == Py_None ? grad.type : (truth(a[5]) ? at::kBFloat16 : at::kFloat);
    void* stream = stream_of(a[6]);
    at::Tensor order, rows;
    if (a[2] == Py_None) {
        std::tie(order, rows) = sorted(index, V, stream);
    } else {
        order = *index.t;
        const Index second(a[2], "index.rows", grad.t);
        rows = *second.t;
        if (second.n != index.n || index.bytes != 4 || second.bytes != 4)
            throw Refused("index.order and index.rows must be int32 [" + std::to_string(grad.rows) + "]");
    }
    size_t bytes = 0;
    done(lib.embedding_backward_workspace_size(index.n, D, &bytes), "spingtp_embedding_backward_workspace_size");
    const at::Tensor ws = workspace(bytes, *grad.t), out = empty({V, D}, type, *grad.t);
    done(lib.embedding_backward(dtype_of(grad.type), grad.p, grad.ld, order.data_ptr<int32_t>(), rows.data_ptr<int32_t>(),
                                static_cast<float>(scale), dtype_of(type), out.data_ptr(), D, address(ws), bytes, index.n,
                                V, D, stream),
         "spingtp_embedding_backward");
    return wrap(out);
}

// The tensors of an AdamW step: of one device, contiguous, of `n` elements; and what memory they take, a list of each
// kind (mostly in the order of its addresses already).
struct Places {
    struct Range {
        uintptr_t first, last;
    };
    enum Kind { kParam, kGrad, kM, kV, kScaleM, kScaleV, kCopy, kKinds };
    std::vector<Range> all[kKinds];
    const at::Tensor* beside = nullptr;

    const at::Tensor& take(PyObject* o, const char* name, int64_t n, Kind kind) {
        const at::Tensor& t = tensor(o, name);
        if (!t.is_cuda()) throw Refused(std::string(name) + " must be on a GPU");
        if (beside == nullptr) beside = &t;
        if (t.device() != beside->device()) throw Refused("all tensors must be on one device");
        if (!t.is_contiguous()) throw Refused(std::string(name) + " must be contiguous");
        const int64_t have = t.numel();
        if (n >= 0 && have != n)
            throw Refused(std::string(name) + " must have the param's " + std::to_string(n) + " elements, not " +
                          std::to_string(have));
        const auto p = reinterpret_cast<uintptr_t>(t.data_ptr());
        if (have > 0) all[kind].push_back({p, p + static_cast<uintptr_t>(have) * t.element_size()});
        return t;
    }
    // Refuses memory that is written and held by another as well.
    void apart() {
        const auto less = [](const Range& x, const Range& y) { return x.first < y.first; };
        const Range* at[kKinds];
        const Range* end[kKinds];
        for (int k = 0; k < kKinds; ++k) {
            if (!std::is_sorted(all[k].begin(), all[k].end(), less)) std::sort(all[k].begin(), all[k].end(), less);
            at[k] = all[k].data();
            end[k] = at[k] + all[k].size();
        }
        uintptr_t any = 0, written = 0;  // the ends so far
        for (;;) {
            int next = -1;
            for (int k = 0; k < kKinds; ++k)
                if (at[k] != end[k] && (next < 0 || at[k]->first < at[next]->first)) next = k;
            if (next < 0) return;
            const Range& r = *at[next]++;
            if (r.first < (next != kGrad ? any : written)) throw Refused("tensors that are written overlap others");
            any = std::max(any, r.last);
            if (next != kGrad) written = std::max(written, r.last);
        }
    }
};
bool floating(at::ScalarType t) { return t == at::kFloat || t == at::kBFloat16; }

// a list's items
struct Items {
    PyObject* const* at;
    Py_ssize_t n;
    Items(PyObject* o, const char* name, Py_ssize_t want) {
        if (!PyList_Check(o)) throw Refused(std::string(name) + " must be a list");
        n = PyList_GET_SIZE(o);
        if (want >= 0 && n != want)
            throw Refused(std::string(name) + " must have " + std::to_string(want) + " items, not " + std::to_string(n));
        at = PySequence_Fast_ITEMS(o);
    }
};

// A number of device memory, [1] or a scalar; null for None.
template <typename T>
const T* device_number(PyObject* o, const char* name, at::ScalarType type, const at::Tensor& beside) {
    const at::Tensor& t = tensor(o, name);
    if (t.scalar_type() != type || t.numel() != 1 || t.device() != beside.device())
        throw Refused(std::string(name) + " must be one " + (type == at::kLong ? "int64" : "fp32") +
                      " number beside the params");
    return t.data_ptr<T>();
}

// A new reference that goes with its place.
struct Held {
    PyObject* o;
    explicit Held(PyObject* o_) : o(o_) {}
    Held(const Held&) = delete;
    ~Held() { Py_XDECREF(o); }
};

// params, grads, m, v (tensors or Block8), copies | None, step, lr, beta1, beta2, eps, weight_decay,
// grad_scale | None, seed, stream
PyObject* adamw(Args a) {
    const Items params(a[0], "params", -1), grads(a[1], "grads", params.n), m(a[2], "m", params.n), v(a[3], "v", params.n);
    const bool some = a[4] != Py_None;
    const Items copies(some ? a[4] : a[0], "copies", params.n);
    std::vector<spingtp_adamw_tensor> list(static_cast<size_t>(params.n));
    Places places;
    for (auto& ranges : places.all) ranges.reserve(list.size());
    for (Py_ssize_t i = 0; i < params.n; ++i) {
        spingtp_adamw_tensor& to = list[static_cast<size_t>(i)];
        const at::Tensor& p = places.take(params.at[i], "params", -1, Places::kParam);
        const int64_t n = p.numel();
        const at::Tensor& g = places.take(grads.at[i], "grads", n, Places::kGrad);
        if (!floating(p.scalar_type()) || !floating(g.scalar_type())) throw Refused("params and grads must be fp32 or bf16");
        if (g.sizes() != p.sizes()) throw Refused("a gradient must have its param's shape");
        to = {p.data_ptr(), g.data_ptr(), nullptr, nullptr, nullptr, nullptr, nullptr, n, dtype_of(p.scalar_type()),
              dtype_of(g.scalar_type())};
        PyObject* const states[2] = {m.at[i], v.at[i]};
        const char* const names[2] = {"m", "v"};
        const bool eight = !THPVariable_Check(states[0]);
        if (eight == static_cast<bool>(THPVariable_Check(states[1])))
            throw Refused("m and v of a tensor must be of one kind");
        for (int k = 0; k < 2; ++k) {
            if (eight) {
                const Held values(PyObject_GetAttrString(states[k], "values")),
                    scales(PyObject_GetAttrString(states[k], "scales"));
                if (values.o == nullptr || scales.o == nullptr) {
                    PyErr_Clear();
                    throw Refused(std::string(names[k]) + " must be tensors or Block8");
                }
                check_block(values.o, scales.o, 1, n);
                (k == 0 ? to.m : to.v) =
                    places.take(values.o, names[k], -1, k == 0 ? Places::kM : Places::kV).data_ptr();
                (k == 0 ? to.m_scales : to.v_scales) =
                    places.take(scales.o, names[k], -1, k == 0 ? Places::kScaleM : Places::kScaleV).data_ptr();
            } else {
                const at::Tensor& s = places.take(states[k], names[k], n, k == 0 ? Places::kM : Places::kV);
                if (s.scalar_type() != at::kFloat) throw Refused(std::string(names[k]) + " must be fp32 or a Block8");
                (k == 0 ? to.m : to.v) = s.data_ptr();
            }
        }
        if (some && copies.at[i] != Py_None) {
            const at::Tensor& c = places.take(copies.at[i], "copies", n, Places::kCopy);
            if (c.scalar_type() != at::kBFloat16 || p.scalar_type() != at::kFloat)
                throw Refused("copies must be bf16, of fp32 params");
            to.copy = c.data_ptr();
        }
    }
    places.apart();
    spingtp_adamw_options o{};
    if (THPVariable_Check(a[5]))
        o.device_step = device_number<int64_t>(a[5], "step", at::kLong, *places.beside);
    else if ((o.step = integer(a[5])) < 1)
        throw Refused("step must be 1 or more");
    if (THPVariable_Check(a[6]))
        o.device_lr = device_number<float>(a[6], "lr", at::kFloat, *places.beside);
    else
        o.lr = number(a[6]);
    o.beta1 = number(a[7]);
    o.beta2 = number(a[8]);
    o.eps = number(a[9]);
    o.weight_decay = number(a[10]);
    if (!(o.beta1 >= 0 && o.beta1 < 1 && o.beta2 >= 0 && o.beta2 < 1)) throw Refused("betas must be in [0, 1)");
    if (!(o.eps >= 0)) throw Refused("eps must not be negative");
    if (a[11] != Py_None) o.grad_scale = device_number<float>(a[11], "grad_scale", at::kFloat, *places.beside);
    o.seed = PyLong_AsUnsignedLongLongMask(a[12]);
    if (PyErr_Occurred()) throw PythonError{};
    for (Py_ssize_t i = 0; i < params.n; ++i) {  // before the launch: it refuses what may not be written
        tensor(params.at[i], "params").unsafeGetTensorImpl()->bump_version();
        if (some && copies.at[i] != Py_None) tensor(copies.at[i], "copies").unsafeGetTensorImpl()->bump_version();
    }
    done(lib.adamw(list.data(), params.n, &o, stream_of(a[13])), "spingtp_adamw");
    Py_RETURN_NONE;
}

// ---------------------------------------------------------------- module

template <PyObject* (*OP)(Args), Py_ssize_t N>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != N) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, %zd wanted", n, N);
        return nullptr;
    }
    try {
        return OP(args);
    } catch (const Refused& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const Failed& e) {
        PyObject* value = PyObject_CallFunction(error_class, "is", static_cast<int>(e.status), e.where);
        if (value != nullptr) {
            PyErr_SetObject(error_class, value);
            Py_DECREF(value);
        }
    } catch (const PythonError&) {
    } catch (...) {  // torch's, as torch raises them
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

// bind(addresses of the C entry points in the order of Entries, error class)
PyObject* bind(Args a) {
    void** to = reinterpret_cast<void**>(&lib);
    constexpr Py_ssize_t n = sizeof(lib) / sizeof(void*);
    if (!PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) != n) throw Refused("the addresses of all entry points are wanted");
    for (Py_ssize_t i = 0; i < n; ++i) to[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(a[0], i));
    if (PyErr_Occurred()) throw PythonError{};
    Py_XSETREF(error_class, Py_NewRef(a[1]));
    Py_RETURN_NONE;
}

#define OP(NAME, N) \
    { #NAME, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<static_cast<PyObject* (*)(Args)>(&NAME), N>)), METH_FASTCALL, nullptr }
PyMethodDef methods[] = {OP(bind, 2),
                         OP(check_block, 4),
                         OP(pack8, 3),
                         OP(unpack8, 7),
                         OP(rms_norm, 6),
                         OP(rms_norm_backward, 7),
                         OP(matmul8, 10),
                         OP(gated, 6),
                         OP(gated8, 12),
                         OP(gated_backward, 11),
                         OP(linear, 9),
                         OP(linear8, 13),
                         OP(linear_backward, 10),
                         OP(embedding, 4),
                         OP(sort_index, 3),
                         OP(embedding_backward, 7),
                         OP(adamw, 14),
                         {nullptr, nullptr, 0, nullptr}};
#undef OP
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
