// The training calls and those on 4-bit weights as PyTorch sees them: tensors in, tensors out.  These calls are
// made once per layer and step, often on few rows, where marshalling in Python and a Python-level allocation per
// output took longer than the kernels; here a call looks at each tensor once, allocates, and enters
// the C ABI.  Nothing is computed here.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/pwlq.h"
#include "pwlq_overlap.h"

namespace {

// Entry points of the library that the Python module has loaded (init), and its error class.
struct Library {
    decltype(&pwlq_act8_encode) encode;
    decltype(&pwlq_act8_decode) decode;
    decltype(&pwlq_block_norm) block_norm;
    decltype(&pwlq_block_norm_backward_workspace_bytes) backward_bytes;
    decltype(&pwlq_block_norm_backward) backward;
    decltype(&pwlq_act8_weight_grad_workspace_bytes) grad_bytes;
    decltype(&pwlq_act8_weight_grad) grad;
    decltype(&pwlq_w4_bytes) w4_bytes;
    decltype(&pwlq_w4_encode) w4_encode;
    decltype(&pwlq_w4_decode) w4_decode;
    decltype(&pwlq_w4_linear_workspace_bytes) w4_linear_bytes;
    decltype(&pwlq_w4_linear) w4_linear;
    decltype(&pwlq_w4_moe_workspace_bytes) moe_bytes;
    decltype(&pwlq_w4_moe) moe;
} lib;
PyObject* error_class = nullptr;

// What a call found wrong: raised as PwlqError(status, name of the entry point).
struct Failed {
    int status;
    const char* what;
};
void check(int status, const char* what) {
    if (status != PWLQ_OK) throw Failed{status, what};
}

// A group length as the C ABI takes it: memory is sized with it before the library sees it.
int group_of(int64_t v) {
    if (v < 1 || v > 256) throw Failed{PWLQ_ERR_INVALID_ARG, "checkpoint group"};
    return (int)v;
}

struct Args {
    PyObject* const* a;
    int i = 0;
    PyObject* next() { return a[i++]; }
    bool none() const { return a[i] == Py_None; }
    at::Tensor tensor(const char* what) {
        PyObject* o = next();
        TORCH_CHECK_VALUE(THPVariable_Check(o), what, " must be a tensor");
        return THPVariable_Unpack(o);
    }
    // an undefined tensor for None
    at::Tensor maybe(const char* what) {
        if (none()) { ++i; return at::Tensor(); }
        return tensor(what);
    }
    int64_t integer() {
        const long long v = PyLong_AsLongLong(next());
        if (v == -1 && PyErr_Occurred()) throw python_error();
        return v;
    }
    double real() {
        const double v = PyFloat_AsDouble(next());
        if (v == -1.0 && PyErr_Occurred()) throw python_error();
        return v;
    }
    void* pointer() { return reinterpret_cast<void*>((uintptr_t)integer()); }
};

int dtype_code(at::ScalarType t) {
    switch (t) {
        case at::kFloat: return PWLQ_F32;
        case at::kBFloat16: return PWLQ_BF16;
        case at::kHalf: return PWLQ_F16;
        default: TORCH_CHECK_VALUE(false, "values must be float32, bfloat16 or float16, not ", t);
    }
}
at::ScalarType dtype_of(int64_t code) {
    TORCH_CHECK_VALUE(code >= 0 && code <= 2, "values must be float32, bfloat16 or float16");
    return code == PWLQ_F32 ? at::kFloat : code == PWLQ_BF16 ? at::kBFloat16 : at::kHalf;
}

// Device of a call's first tensor, which has to be the current one: the library launches there.
int home(const at::Tensor& t, const char* what) {
    TORCH_CHECK_VALUE(t.is_cuda() && t.get_device() == c10::cuda::current_device(), what,
                      " must be on the current CUDA device, it is on ", t.device());
    return (int)t.get_device();
}
void* stream_of(int device) { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }

struct Matrix {
    void* p = nullptr;
    int64_t ld = 0;
};
// A tensor of this shape, type and device with adjacent values in its rows.
Matrix matrix(const at::Tensor& t, const char* what, int64_t rows, int64_t cols, at::ScalarType type, int device) {
    TORCH_CHECK_VALUE(t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && t.scalar_type() == type &&
                          t.is_cuda() && t.get_device() == device,
                      what, " must be [", rows, ", ", cols, "] of ", type, " on cuda:", device, ", got ", t.sizes(),
                      " of ", t.scalar_type(), " on ", t.device());
    TORCH_CHECK_VALUE(cols < 2 || t.stride(1) == 1, what, ": the values of a row must be adjacent");
    Matrix m{t.data_ptr(), rows < 2 ? cols : t.stride(0)};
    TORCH_CHECK_VALUE(m.ld >= cols, what, ": rows overlap (a broadcast tensor must be made whole first)");
    return m;
}
void* vector(const at::Tensor& t, const char* what, int64_t cols, at::ScalarType type, int device) {
    TORCH_CHECK_VALUE(t.dim() == 1 && t.size(0) == cols && t.scalar_type() == type && t.is_cuda() &&
                          t.get_device() == device && t.is_contiguous(),
                      what, " must be contiguous [", cols, "] of ", type, " on cuda:", device, ", got ", t.sizes(),
                      " of ", t.scalar_type(), " on ", t.device());
    return t.data_ptr();
}
void two_dimensions(const at::Tensor& t, const char* what) {
    TORCH_CHECK_VALUE(t.dim() == 2, what, " must be [rows, cols]");
    dtype_code(t.scalar_type());
}
at::Tensor like(const at::Tensor& t) {
    return t.is_contiguous() ? at::empty_like(t) : at::empty(t.sizes(), t.options());
}
at::Tensor bytes(int64_t n, const at::Tensor& beside) { return at::empty({n}, beside.options().dtype(at::kByte)); }
PyObject* wrap(const at::Tensor& t) {
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(t);
}
PyObject* tuple(std::initializer_list<PyObject*> items) {
    PyObject* t = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    for (PyObject* o : items) PyTuple_SET_ITEM(t, i++, o);
    return t;
}

// Weights and gate of a block norm, which both directions take from the tensors they are given.
void weights_of(pwlq_block_norm_args& b, const at::Tensor& pre, const at::Tensor& post, const at::Tensor& gate,
                at::ScalarType wtype, int device) {
    b.pre_weight = pre.defined() ? vector(pre, "pre_weight", b.cols, wtype, device) : nullptr;
    b.post_weight = post.defined() ? vector(post, "post_weight", b.cols, wtype, device) : nullptr;
    b.gate = nullptr;
    if (!gate.defined()) return;
    const Matrix m = matrix(gate, "gate", b.gate_rows, b.cols, wtype, device);
    b.gate = m.p;
    b.ldgate = m.ld;
}

// A checkpoint in one piece: the codes, then the ranges, to the next multiple of 32.
int64_t pitch_of(int64_t cols) { return (cols + 15) / 16 * 16; }
int64_t act8_bytes(int64_t rows, int64_t cols, int64_t group) {
    if (group < 1 || cols < 1) throw Failed{PWLQ_ERR_INVALID_ARG, "checkpoint"};
    return (rows * (pitch_of(cols) + 4 * ((cols + group - 1) / group)) + 31) / 32 * 32;
}
struct Codes {
    uint8_t* codes;
    int64_t ld;
    float* ranges;
};
Codes codes_at(void* memory, int64_t rows, int64_t cols) {
    uint8_t* p = static_cast<uint8_t*>(memory);
    return {p, pitch_of(cols), reinterpret_cast<float*>(p + rows * pitch_of(cols))};
}

// What a block norm keeps for its backward pass, in one piece: r's checkpoint (with pre_weight), f's (with
// post_weight or gate), the factors of both norms.
struct Kept {
    int64_t f_at = 0, rstd_at = 0, bytes = 0;
    bool keeps_f = false;
    Kept() = default;
    Kept(const pwlq_block_norm_args& b, bool pre, bool post, bool gate) : keeps_f(post || gate) {
        const int64_t size = act8_bytes(b.rows, b.cols, b.group);
        f_at = pre ? size : 0;
        rstd_at = f_at + (keeps_f ? size : 0);
        bytes = rstd_at + 8 * b.rows;
    }
    void place(pwlq_block_norm_args& b, void* memory, bool pre, bool post) const {
        uint8_t* const base = static_cast<uint8_t*>(memory);
        float* const factors = reinterpret_cast<float*>(base + rstd_at);
        const Codes r = codes_at(base, b.rows, b.cols), f = codes_at(base + f_at, b.rows, b.cols);
        b.r_codes = pre ? r.codes : nullptr;
        b.r_ranges = pre ? r.ranges : nullptr;
        b.r_rstd = pre ? factors : nullptr;
        b.f_codes = keeps_f ? f.codes : nullptr;
        b.f_ranges = keeps_f ? f.ranges : nullptr;
        b.f_rstd = post ? factors + b.rows : nullptr;
    }
};

// (x, group, ratio, codes pointer or 0, pitch, ranges pointer) -> new memory, or None where given
PyObject* encode(Args a) {
    const at::Tensor x = a.tensor("x");
    const int group = group_of(a.integer());
    const double ratio = a.real();
    Codes c;
    c.codes = static_cast<uint8_t*>(a.pointer());
    c.ld = a.integer();
    c.ranges = static_cast<float*>(a.pointer());
    const bool given = a.integer() != 0;
    const int device = home(x, "x");
    two_dimensions(x, "x");
    const int64_t rows = x.size(0), cols = x.size(1);
    const Matrix m = matrix(x, "x", rows, cols, x.scalar_type(), device);
    at::Tensor memory;
    if (!given) {
        memory = bytes(act8_bytes(rows, cols, group), x);
        c = codes_at(memory.data_ptr(), rows, cols);
    }
    check(lib.encode(m.p, dtype_code(x.scalar_type()), rows, cols, m.ld, group, (float)ratio, c.codes, c.ld,
                     c.ranges, stream_of(device)),
          "pwlq_act8_encode");
    return wrap(memory);
}

// (a tensor of the checkpoint's, codes pointer, pitch, ranges pointer, rows, cols, group, ratio, type, out or None)
PyObject* decode(Args a) {
    const at::Tensor beside = a.tensor("checkpoint");
    uint8_t* codes = static_cast<uint8_t*>(a.pointer());
    const int64_t ldc = a.integer();
    float* ranges = static_cast<float*>(a.pointer());
    const int64_t rows = a.integer(), cols = a.integer();
    const int group = group_of(a.integer());
    const double ratio = a.real();
    const int64_t code = a.integer();
    at::Tensor out = a.maybe("out");
    const int device = home(beside, "the checkpoint");
    if (!out.defined()) out = at::empty({rows, cols}, beside.options().dtype(dtype_of(code)));
    const Matrix m = matrix(out, "out", rows, cols, out.scalar_type(), device);
    check(lib.decode(codes, ldc, ranges, rows, cols, group, (float)ratio, m.p, dtype_code(out.scalar_type()),
                     m.ld, stream_of(device)),
          "pwlq_act8_decode");
    return wrap(out);
}

// (x, f, pre, post, gate, gate_tokens or None, scale, eps, offset, group or 0, ratio, r or None, h or None)
//   -> (r, h, memory, argument block, offset of f's checkpoint, offset of the factors)
PyObject* block_norm(Args a) {
    const at::Tensor x = a.tensor("x"), f = a.maybe("f"), pre = a.maybe("pre_weight"), post = a.maybe("post_weight"),
                     gate = a.maybe("gate");
    const bool given = !a.none();          // without a gate its length does not matter
    const int64_t every = given ? a.integer() : (a.next(), 0);
    pwlq_block_norm_args b = {};
    b.residual_scale = a.real();
    b.eps = a.real();
    b.weight_offset = a.real();
    const int64_t group = a.integer();
    b.ratio = a.real();
    at::Tensor r = a.maybe("r"), h = a.maybe("h");

    const int device = home(x, "x");
    two_dimensions(x, "x");
    const int64_t rows = b.rows = x.size(0), cols = b.cols = x.size(1);
    const at::ScalarType type = x.scalar_type();
    b.dtype = dtype_code(type);
    Matrix m = matrix(x, "x", rows, cols, type, device);
    b.x = m.p;
    b.ldx = m.ld;
    if (f.defined()) {
        m = matrix(f, "f", rows, cols, type, device);
        b.f = m.p;
        b.ldf = m.ld;
    }
    const at::Tensor& some = pre.defined() ? pre : post.defined() ? post : gate;
    const at::ScalarType wtype = some.defined() ? some.scalar_type() : type;
    TORCH_CHECK_VALUE(wtype == type || wtype == at::kFloat, "weights and gate must be of x's type or float32");
    b.wtype = dtype_code(wtype);
    if (gate.defined()) {
        TORCH_CHECK_VALUE(gate.dim() == 2, "gate must be [gate_rows, cols]");
        b.gate_rows = gate.size(0);
        const int64_t n = std::max<int64_t>(b.gate_rows, 1);
        b.gate_tokens = given ? every : std::max<int64_t>((rows + n - 1) / n, 1);
    }
    weights_of(b, pre, post, gate, wtype, device);
    if (!r.defined()) r = like(x);
    m = matrix(r, "r", rows, cols, type, device);
    b.r = m.p;
    b.ldr = m.ld;
    if (pre.defined()) {
        if (!h.defined()) h = like(x);
        m = matrix(h, "h", rows, cols, type, device);
        b.h = m.p;
        b.ldh = m.ld;
    } else {
        h = at::Tensor();
    }
    at::Tensor memory;
    Kept kept;
    if (group) {
        b.group = group;
        b.ldc = pitch_of(cols);
        kept = Kept(b, pre.defined(), post.defined(), gate.defined());
        memory = bytes(kept.bytes, x);
        kept.place(b, memory.data_ptr(), pre.defined(), post.defined());
    }
    check(lib.block_norm(&b, stream_of(device)), "pwlq_block_norm");
    return tuple({wrap(r), wrap(h), wrap(memory),
                  PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&b), sizeof(b)),
                  PyLong_FromLongLong(kept.f_at), PyLong_FromLongLong(kept.rstd_at)});
}

// (argument block, memory, has_f, dh, dr, pre, post, gate, workspace or None)
//   -> (dx, df, dpre, dpost, dgate)
// Of the forward call's argument block only sizes, types and numbers are used: what the tensors' memory
// holds now is what counts, wherever it lies (a parameter's storage may have been replaced in between).
PyObject* block_norm_backward(Args a) {
    PyObject* block = a.next();
    pwlq_block_norm_args b;
    TORCH_CHECK_VALUE(PyBytes_Check(block) && PyBytes_GET_SIZE(block) == sizeof(b), "not an argument block");
    memcpy(&b, PyBytes_AS_STRING(block), sizeof(b));
    const at::Tensor memory = a.tensor("memory");
    const bool has_f = a.integer() != 0;
    const at::Tensor dh = a.maybe("dh"), dr = a.maybe("dr"), pre = a.maybe("pre_weight"),
                     post = a.maybe("post_weight"), gate = a.maybe("gate");
    at::Tensor workspace = a.maybe("workspace");
    const at::Tensor& some = dh.defined() ? dh : dr;
    TORCH_CHECK_VALUE(some.defined() && dh.defined() == pre.defined(),
                      "dh is needed exactly where the forward call had a pre_weight, dr where it had none");
    const int device = home(some, "the gradient");
    TORCH_CHECK_VALUE(memory.get_device() == device, "the forward call ran on ", memory.device(),
                      ", the gradient is on ", some.device());
    const at::ScalarType type = dtype_of(b.dtype);
    const Kept kept(b, pre.defined(), post.defined(), gate.defined());
    TORCH_CHECK_VALUE(memory.scalar_type() == at::kByte && memory.is_contiguous() && memory.numel() == kept.bytes,
                      "the kept memory is not that of a forward call with these weights");
    kept.place(b, memory.data_ptr(), pre.defined(), post.defined());
    weights_of(b, pre, post, gate, dtype_of(b.wtype), device);
    pwlq_block_norm_grads g = {};
    if (dh.defined()) {
        const Matrix m = matrix(dh, "dh", b.rows, b.cols, type, device);
        g.dh = m.p;
        g.lddh = m.ld;
    }
    if (dr.defined()) {
        const Matrix m = matrix(dr, "dr", b.rows, b.cols, type, device);
        g.dr = m.p;
        g.lddr = m.ld;
    }
    at::Tensor dx = like(some), df, dpre, dpost, dgate;
    g.dx = dx.data_ptr();
    g.lddx = g.lddf = b.cols;
    if (has_f) {
        df = like(some);
        g.df = df.data_ptr();
    }
    if (pre.defined()) {
        dpre = like(pre);
        g.dpre = dpre.data_ptr();
    }
    if (post.defined()) {
        dpost = like(post);
        g.dpost = dpost.data_ptr();
    }
    if (gate.defined()) {
        dgate = like(gate);
        g.dgate = dgate.data_ptr();
    }
    if (g.dpre || g.dpost || g.dgate) {
        if (!workspace.defined())
            workspace = bytes((int64_t)lib.backward_bytes(b.rows, b.cols, gate.defined() ? b.gate_rows : 0), memory);
        TORCH_CHECK_VALUE(workspace.scalar_type() == at::kByte && workspace.is_contiguous() && workspace.is_cuda() &&
                              workspace.get_device() == device,
                          "workspace must be contiguous uint8 on cuda:", device);
        g.workspace = workspace.data_ptr();
        g.workspace_bytes = workspace.numel();
    }
    check(lib.backward(&b, &g, stream_of(device)), "pwlq_block_norm_backward");
    return tuple({wrap(dx), wrap(df), wrap(dpre), wrap(dpost), wrap(dgate)});
}

// (dy, a tensor of the checkpoint's, codes pointer, pitch, ranges pointer, rows, cols, group, ratio, type or -1,
//  out or None, accumulate, workspace or None) -> dw
PyObject* weight_grad(Args a) {
    const at::Tensor dy = a.tensor("dy"), beside = a.tensor("checkpoint");
    uint8_t* codes = static_cast<uint8_t*>(a.pointer());
    const int64_t ldc = a.integer();
    float* ranges = static_cast<float*>(a.pointer());
    const int64_t kept = a.integer(), cols = a.integer();
    const int group = group_of(a.integer());
    const double ratio = a.real();
    const int64_t code = a.integer();
    at::Tensor out = a.maybe("out");
    const bool accumulate = a.integer() != 0;
    at::Tensor workspace = a.maybe("workspace");
    const int device = home(dy, "dy");
    two_dimensions(dy, "dy");
    const int64_t rows = dy.size(0), outputs = dy.size(1);
    TORCH_CHECK_VALUE(kept == rows, "the checkpoint is of ", kept, " rows, not ", rows);
    TORCH_CHECK_VALUE(beside.get_device() == device, "the checkpoint is on ", beside.device(), ", dy on ", dy.device());
    const Matrix y = matrix(dy, "dy", rows, outputs, dy.scalar_type(), device);
    if (!out.defined()) {
        TORCH_CHECK_VALUE(!accumulate, "accumulate needs out");
        out = at::empty({outputs, cols}, dy.options().dtype(code < 0 ? dy.scalar_type() : dtype_of(code)));
    }
    const Matrix w = matrix(out, "out", outputs, cols, out.scalar_type(), device);
    if (!workspace.defined())
        workspace = bytes((int64_t)lib.grad_bytes(rows, outputs, cols,
                                                  (((uintptr_t)y.p | (uintptr_t)(y.ld * 2)) & 15) == 0), dy);
    TORCH_CHECK_VALUE(workspace.scalar_type() == at::kByte && workspace.is_contiguous() && workspace.is_cuda() &&
                          workspace.get_device() == device,
                      "workspace must be contiguous uint8 on cuda:", device);
    check(lib.grad(y.p, dtype_code(dy.scalar_type()), rows, outputs, y.ld, codes, ldc, ranges, cols, group,
                   (float)ratio, w.p, dtype_code(out.scalar_type()), w.ld, accumulate, workspace.data_ptr(),
                   (size_t)workspace.numel(), stream_of(device)),
          "pwlq_act8_weight_grad");
    return wrap(out);
}

// A packed matrix from its fields (matrices, rows, cols, group, breakpoint, paired) and, where it has some, its
// memory.
struct Packed {
    pwlq_w4 w = {};
    int64_t bytes = 0;
    at::Tensor memory;
    explicit Packed(PyObject* fields) {
        TORCH_CHECK_VALUE(PyTuple_Check(fields) && PyTuple_GET_SIZE(fields) == 6, "not a packed matrix");
        int64_t* const to[6] = {&w.matrices, &w.rows, &w.cols, &w.group, &w.breakpoint, &w.paired};
        for (int i = 0; i < 6; ++i) {
            *to[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(fields, i));
            if (*to[i] == -1 && PyErr_Occurred()) throw python_error();
        }
        bytes = (int64_t)lib.w4_bytes(w.matrices, w.rows, w.cols, w.group, w.paired);
        const bool none = w.matrices < 1 || w.rows < 1 || w.cols < 1;
        if (!bytes) throw Failed{none ? PWLQ_ERR_INVALID_ARG : PWLQ_ERR_UNSUPPORTED, "packed matrix"};
    }
    void place(const at::Tensor& m, int device) {
        TORCH_CHECK_VALUE(m.scalar_type() == at::kByte && m.is_contiguous() && m.is_cuda() && m.get_device() == device &&
                              m.numel() == bytes,
                          "the memory of this packed matrix is ", bytes, " contiguous bytes on cuda:", device, ", got ",
                          m.numel(), " of ", m.scalar_type(), " on ", m.device());
        memory = m;
        w.data = m.data_ptr();
    }
};
Packed packed(Args& a, int device) {
    Packed p(a.next());
    p.place(a.tensor("the packed matrix's memory"), device);
    return p;
}

// The values of a packed matrix: [rows, cols], or [matrices, rows, cols].
struct Values {
    void* p = nullptr;
    int64_t ld = 0, ldm = 0;
};
Values values(const at::Tensor& t, const char* what, const pwlq_w4& w, int device) {
    const int64_t d = t.dim();
    dtype_code(t.scalar_type());
    TORCH_CHECK_VALUE((d == 3 ? t.size(0) == w.matrices : d == 2 && w.matrices == 1) && t.size(d - 2) == w.rows &&
                          t.size(d - 1) == w.cols && t.is_cuda() && t.get_device() == device,
                      what, " must be ", w.matrices, " of [", w.rows, ", ", w.cols, "] on cuda:", device, ", got ", t.sizes(),
                      " on ", t.device());
    TORCH_CHECK_VALUE(w.cols < 2 || t.stride(d - 1) == 1, what, ": the values of a row must be adjacent");
    Values v{t.data_ptr(), w.rows < 2 ? w.cols : t.stride(d - 2), w.matrices < 2 ? 0 : t.stride(0)};
    TORCH_CHECK_VALUE(v.ld >= w.cols, what, ": rows overlap (a broadcast tensor must be made whole first)");
    return v;
}

// (x, fields, memory or None) -> new memory, or None where given
PyObject* w4_encode(Args a) {
    const at::Tensor x = a.tensor("w");
    Packed p(a.next());
    const at::Tensor given = a.maybe("out");
    const int device = home(x, "w");
    const Values v = values(x, "w", p.w, device);
    const at::Tensor memory = given.defined() ? given : bytes(p.bytes, x);
    p.place(memory, device);
    check(lib.w4_encode(&p.w, v.p, dtype_code(x.scalar_type()), v.ld, v.ldm, stream_of(device)), "pwlq_w4_encode");
    return wrap(given.defined() ? at::Tensor() : memory);
}

// (fields, memory, type, three dimensions, out or None)
PyObject* w4_decode(Args a) {
    Packed p(a.next());
    const at::Tensor memory = a.tensor("the packed matrix's memory");
    const int64_t code = a.integer();
    const bool three = a.integer() != 0;
    at::Tensor out = a.maybe("out");
    const int device = home(memory, "the packed matrix");
    p.place(memory, device);
    if (!out.defined()) {
        const auto options = memory.options().dtype(dtype_of(code));
        out = three ? at::empty({p.w.matrices, p.w.rows, p.w.cols}, options) : at::empty({p.w.rows, p.w.cols}, options);
    }
    const Values v = values(out, "out", p.w, device);
    TORCH_CHECK_VALUE(!pwlq::matrices_meet(p.w.matrices, p.w.rows, p.w.cols, v.ld, v.ldm), "out: matrices overlap");
    check(lib.w4_decode(&p.w, v.p, dtype_code(out.scalar_type()), v.ld, v.ldm, stream_of(device)), "pwlq_w4_decode");
    return wrap(out);
}

void no_gradient(const at::Tensor& t, const char* what) {
    TORCH_CHECK_VALUE(!(t.requires_grad() && c10::GradMode::is_enabled()), what,
                      " requires a gradient, and this call has no backward pass: call it under torch.no_grad()");
}

// (x, fields, memory, out or None, workspace or None) -> y
PyObject* w4_linear(Args a) {
    const at::Tensor x = a.tensor("x");
    const int device = home(x, "x");
    two_dimensions(x, "x");
    no_gradient(x, "x");
    const Packed p = packed(a, device);
    at::Tensor y = a.maybe("out"), workspace = a.maybe("workspace");
    const int64_t tokens = x.size(0), outputs = p.w.paired ? p.w.rows / 2 : p.w.rows;
    const Matrix mx = matrix(x, "x", tokens, p.w.cols, x.scalar_type(), device);
    if (!y.defined()) y = at::empty({tokens, outputs}, x.options());
    const Matrix my = matrix(y, "out", tokens, outputs, x.scalar_type(), device);
    const int type = dtype_code(x.scalar_type());
    const int64_t size = type == PWLQ_F32 ? 4 : 2;
    const int64_t need = (int64_t)lib.w4_linear_bytes(tokens, p.w.rows, p.w.cols, type,
                                                      (((uintptr_t)mx.p | (uintptr_t)(mx.ld * size)) & 15) == 0);
    if (need && !workspace.defined()) workspace = bytes(need, x);
    TORCH_CHECK_VALUE(!workspace.defined() || (workspace.scalar_type() == at::kByte && workspace.is_contiguous() &&
                                               workspace.is_cuda() && workspace.get_device() == device),
                      "workspace must be contiguous uint8 on cuda:", device);
    check(lib.w4_linear(&p.w, mx.p, type, tokens, mx.ld, my.p, my.ld, workspace.defined() ? workspace.data_ptr() : nullptr,
                        workspace.defined() ? (size_t)workspace.numel() : 0, stream_of(device)),
          "pwlq_w4_linear");
    return wrap(y);
}

// (x, router, fields and memory of up, of down, top, normalize, want the routing, out or None, workspace or None)
//   -> (y, chosen, weights)
PyObject* w4_moe(Args a) {
    const at::Tensor x = a.tensor("x"), router = a.tensor("router");
    const int device = home(x, "x");
    two_dimensions(x, "x");
    no_gradient(x, "x");
    no_gradient(router, "router");
    const Packed up = packed(a, device), down = packed(a, device);
    pwlq_w4_moe_args m = {};
    m.top = a.integer();
    m.normalize = a.integer() != 0;
    const bool want = a.integer() != 0;
    at::Tensor y = a.maybe("out"), workspace = a.maybe("workspace");
    const at::ScalarType type = x.scalar_type(), rtype = router.scalar_type();
    TORCH_CHECK_VALUE(rtype == type || rtype == at::kFloat, "router must be of x's type or float32");
    m.tokens = x.size(0);
    m.dtype = dtype_code(type);
    m.router_dtype = dtype_code(rtype);
    Matrix t = matrix(x, "x", m.tokens, up.w.cols, type, device);
    m.x = t.p;
    m.ldx = t.ld;
    t = matrix(router, "router", up.w.matrices, up.w.cols, rtype, device);
    m.router = t.p;
    m.ldrouter = t.ld;
    m.up = &up.w;
    m.down = &down.w;
    if (!y.defined()) y = at::empty(x.sizes(), x.options());
    t = matrix(y, "out", m.tokens, up.w.cols, type, device);
    m.y = t.p;
    m.ldy = t.ld;
    // sizes that memory is made from, before the library sees them; with the library's statuses, in its order
    if (m.top < 1 || m.top > up.w.matrices) throw Failed{PWLQ_ERR_INVALID_ARG, "pwlq_w4_moe"};
    const int64_t need = (int64_t)lib.moe_bytes(m.tokens, m.top, down.w.rows, down.w.cols);
    if (!need) throw Failed{m.tokens > PWLQ_W4_MOE_MAX_TOKENS || m.top > PWLQ_W4_MOE_MAX_TOP ? PWLQ_ERR_UNSUPPORTED
                                                                                       : PWLQ_ERR_INVALID_ARG, "pwlq_w4_moe"};
    at::Tensor chosen, weights;
    if (want) {
        chosen = at::empty({m.tokens, m.top}, x.options().dtype(at::kInt));
        weights = at::empty({m.tokens, m.top}, x.options().dtype(at::kFloat));
        m.chosen = static_cast<int32_t*>(chosen.data_ptr());
        m.weights = static_cast<float*>(weights.data_ptr());
    }
    if (!workspace.defined()) workspace = bytes(need, x);
    TORCH_CHECK_VALUE(workspace.scalar_type() == at::kByte && workspace.is_contiguous() && workspace.is_cuda() &&
                          workspace.get_device() == device,
                      "workspace must be contiguous uint8 on cuda:", device);
    m.workspace = workspace.data_ptr();
    m.workspace_bytes = workspace.numel();
    check(lib.moe(&m, stream_of(device)), "pwlq_w4_moe");
    return tuple({wrap(y), wrap(chosen), wrap(weights)});
}

template <PyObject* (*FN)(Args), int N>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != N || !error_class) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments, or the module has not been initialised");
        return nullptr;
    }
    try {
        return FN(Args{args});
    } catch (const Failed& f) {
        PyObject* e = PyObject_CallFunction(error_class, "is", f.status, f.what);
        if (e) {
            PyErr_SetObject(error_class, e);
            Py_DECREF(e);
        }
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// init(addresses of the entry points in the order of Library, error class)
PyObject* init(PyObject*, PyObject* args) {
    PyObject *addresses, *cls;
    if (!PyArg_ParseTuple(args, "O!O", &PyTuple_Type, &addresses, &cls)) return nullptr;
    void** to = reinterpret_cast<void**>(&lib);
    constexpr Py_ssize_t kCount = sizeof(lib) / sizeof(void*);
    if (PyTuple_GET_SIZE(addresses) != kCount) {
        PyErr_SetString(PyExc_ValueError, "wrong number of entry points");
        return nullptr;
    }
    for (Py_ssize_t i = 0; i < kCount; ++i) {
        to[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(addresses, i));
        if (!to[i]) return nullptr;
    }
    Py_INCREF(cls);
    Py_XDECREF(error_class);
    error_class = cls;
    Py_RETURN_NONE;
}

#define PWLQ_CALL(name, n) {#name, (PyCFunction)(void (*)(void))call<name, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"init", init, METH_VARARGS, nullptr},
                         PWLQ_CALL(encode, 7),
                         PWLQ_CALL(decode, 10),
                         PWLQ_CALL(block_norm, 13),
                         PWLQ_CALL(block_norm_backward, 9),
                         PWLQ_CALL(weight_grad, 13),
                         PWLQ_CALL(w4_encode, 3),
                         PWLQ_CALL(w4_decode, 5),
                         PWLQ_CALL(w4_linear, 5),
                         PWLQ_CALL(w4_moe, 11),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pwlq_calls", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__pwlq_calls() { return PyModule_Create(&module); }
