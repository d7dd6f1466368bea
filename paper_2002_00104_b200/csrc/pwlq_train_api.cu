// C ABI of the training operators: argument checks and kernel launches, nothing else.
#include "../../include/pwlq.h"
#include "pwlq_train.h"

namespace {

constexpr int64_t kMaxRows = ((int64_t)1 << 31) - 1;
constexpr int64_t kMaxCols = (int64_t)1 << 24;
constexpr int64_t kMaxPitch = (int64_t)1 << 40;
constexpr float kMinRatio = 9.5367431640625e-07f;        // 2^-20
constexpr float kMaxRatio = 0.999755859375f;             // 1 - 2^-12: above it 63 / d may overflow

inline bool misaligned(const void* p, size_t a) {
    return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0;
}
inline cudaStream_t as_stream(void* s) { return static_cast<cudaStream_t>(s); }
inline int from_cuda(cudaError_t e) { return e == cudaSuccess ? PWLQ_OK : PWLQ_ERR_CUDA; }
inline bool is_dtype(int64_t d) { return d == PWLQ_F32 || d == PWLQ_BF16 || d == PWLQ_F16; }

int check_size(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1) return PWLQ_ERR_INVALID_ARG;
    if (rows > kMaxRows || cols > kMaxCols) return PWLQ_ERR_UNSUPPORTED;
    return PWLQ_OK;
}

// A value tensor: present (when there are rows), aligned to its elements, a pitch that holds a row.
bool bad_tensor(const void* p, int64_t dtype, int64_t ld, int64_t rows, int64_t cols) {
    return (!p && rows > 0) || misaligned(p, pwlq::type_size((int)dtype)) || ld < cols || ld > kMaxPitch;
}

bool bad_format(int64_t group, float ratio) {
    return (group != 32 && group != 64 && group != 128 && group != 256) ||
           !((ratio >= kMinRatio && ratio <= kMaxRatio) || ratio == 1.0f);
}
bool bad_codes(const uint8_t* codes, int64_t ldc, const float* ranges, int64_t rows, int64_t cols) {
    return ((!codes || !ranges) && rows > 0) || misaligned(codes, 16) || misaligned(ranges, 4) ||
           ldc < cols || ldc % 16 != 0 || ldc > kMaxPitch;
}

int check_act8(int64_t rows, int64_t cols, int dtype, const void* v, int64_t ld, const uint8_t* codes,
               int64_t ldc, const float* ranges, int group, float ratio) {
    if (int rc = check_size(rows, cols)) return rc;
    if (!is_dtype(dtype) || bad_tensor(v, dtype, ld, rows, cols) || bad_format(group, ratio) ||
        bad_codes(codes, ldc, ranges, rows, cols))
        return PWLQ_ERR_INVALID_ARG;
    // blocks of 2048 or 4096 columns of a row
    if (rows * ((cols + 2047) / 2048) > kMaxRows) return PWLQ_ERR_UNSUPPORTED;
    return PWLQ_OK;
}

pwlq::Act8Tensor act8(const uint8_t* codes, int64_t ldc, const float* ranges, int64_t rows,
                      int64_t cols, int group, float ratio) {
    return {const_cast<uint8_t*>(codes), ldc, const_cast<float*>(ranges), rows, cols, group, ratio};
}

// What both directions of the block norm require of the forward call's sizes, weights and gate.
int check_block(const pwlq_block_norm_args& a) {
    if (int rc = check_size(a.rows, a.cols)) return rc;
    if (a.cols > PWLQ_BLOCK_NORM_MAX_COLS) return PWLQ_ERR_UNSUPPORTED;
    if (!is_dtype(a.dtype) || (a.wtype != PWLQ_F32 && a.wtype != a.dtype)) return PWLQ_ERR_INVALID_ARG;
    const size_t ws = pwlq::type_size((int)a.wtype);
    if (misaligned(a.post_weight, ws) || misaligned(a.pre_weight, ws)) return PWLQ_ERR_INVALID_ARG;
    if (a.gate && (misaligned(a.gate, ws) || a.ldgate < a.cols || a.ldgate > kMaxPitch ||
                   a.gate_tokens < 1 || a.gate_rows < 0 || a.gate_rows > kMaxRows ||
                   (a.rows > 0 && a.gate_rows < (a.rows - 1) / a.gate_tokens + 1)))
        return PWLQ_ERR_INVALID_ARG;
    return PWLQ_OK;
}

// A gate for more rows than there are is one for all of them; the kernels add the length to row numbers.
pwlq_block_norm_args with_gate_length(const pwlq_block_norm_args& given) {
    pwlq_block_norm_args a = given;
    const int64_t most = a.rows > 0 ? a.rows : 1;
    if (a.gate && a.gate_tokens > most) a.gate_tokens = most;
    return a;
}

// A checkpoint of the block norm: all of its parts or none.
bool bad_saved(const pwlq_block_norm_args& a, const uint8_t* codes, const float* ranges,
               const float* rstd) {
    if (!codes && !ranges) return misaligned(rstd, 4);
    return bad_format(a.group, (float)a.ratio) || misaligned(rstd, 4) ||
           bad_codes(codes, a.ldc, ranges, a.rows > 0 ? a.rows : 1, a.cols);
}

}  // namespace

extern "C" {

int pwlq_act8_encode(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, int group,
                     float ratio, uint8_t* codes, int64_t ldc, float* ranges, void* stream) {
    if (int rc = check_act8(rows, cols, dtype, x, ldx, codes, ldc, ranges, group, ratio)) return rc;
    if (rows == 0) return PWLQ_OK;
    return from_cuda(pwlq::launch_act8_encode(
        x, dtype, ldx, act8(codes, ldc, ranges, rows, cols, group, ratio), as_stream(stream)));
}

int pwlq_act8_decode(const uint8_t* codes, int64_t ldc, const float* ranges, int64_t rows,
                     int64_t cols, int group, float ratio, void* y, int dtype, int64_t ldy,
                     void* stream) {
    if (int rc = check_act8(rows, cols, dtype, y, ldy, codes, ldc, ranges, group, ratio)) return rc;
    if (rows == 0) return PWLQ_OK;
    return from_cuda(pwlq::launch_act8_decode(
        act8(codes, ldc, ranges, rows, cols, group, ratio), y, dtype, ldy, as_stream(stream)));
}

int pwlq_block_norm(const pwlq_block_norm_args* args, void* stream) {
    if (!args) return PWLQ_ERR_INVALID_ARG;
    const pwlq_block_norm_args& a = *args;
    if (int rc = check_block(a)) return rc;
    const int64_t dt = a.dtype;
    if (bad_tensor(a.x, dt, a.ldx, a.rows, a.cols) ||
        (a.f ? bad_tensor(a.f, dt, a.ldf, a.rows, a.cols)
             : a.rows > 0 && (a.gate || a.post_weight || a.f_codes)) ||
        (a.r && bad_tensor(a.r, dt, a.ldr, a.rows, a.cols)) ||
        (a.pre_weight ? bad_tensor(a.h, dt, a.ldh, a.rows, a.cols) : a.h != nullptr) ||
        (a.rows > 0 && !a.r && !a.pre_weight))
        return PWLQ_ERR_INVALID_ARG;
    if (bad_saved(a, a.r_codes, a.r_ranges, a.r_rstd) || bad_saved(a, a.f_codes, a.f_ranges, a.f_rstd))
        return PWLQ_ERR_INVALID_ARG;
    if (a.rows == 0) return PWLQ_OK;
    return from_cuda(pwlq::launch_block_norm(with_gate_length(a), as_stream(stream)));
}

size_t pwlq_block_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int64_t gate_rows) {
    if (check_size(rows, cols) || cols > PWLQ_BLOCK_NORM_MAX_COLS || gate_rows < 0 ||
        gate_rows > kMaxRows)
        return 0;
    const size_t bytes = pwlq::block_norm_backward_workspace(rows, cols, gate_rows);
    return bytes ? bytes : 256;
}

int pwlq_block_norm_backward(const pwlq_block_norm_args* fwd, const pwlq_block_norm_grads* grads,
                             void* stream) {
    if (!fwd || !grads) return PWLQ_ERR_INVALID_ARG;
    pwlq_block_norm_args a = *fwd;
    pwlq_block_norm_grads g = *grads;
    if (int rc = check_block(a)) return rc;
    const int64_t dt = a.dtype;
    const bool some = a.rows > 0;
    if ((g.dh ? bad_tensor(g.dh, dt, g.lddh, a.rows, a.cols) : (a.pre_weight && some)) ||
        (g.dr && bad_tensor(g.dr, dt, g.lddr, a.rows, a.cols)) ||
        (g.dx && bad_tensor(g.dx, dt, g.lddx, a.rows, a.cols)) ||
        (g.df && bad_tensor(g.df, dt, g.lddf, a.rows, a.cols)))
        return PWLQ_ERR_INVALID_ARG;
    if (some && g.df && !a.f) return PWLQ_ERR_INVALID_ARG;        // the gradient of what was not there
    const size_t ws = pwlq::type_size((int)a.wtype);
    if (misaligned(g.dpre, ws) || misaligned(g.dpost, ws) || misaligned(g.dgate, ws) ||
        (g.dpre && !a.pre_weight) || (g.dpost && !a.post_weight) || (g.dgate && !a.gate))
        return PWLQ_ERR_INVALID_ARG;
    if (some && a.pre_weight &&
        (!a.r_codes || !a.r_rstd || bad_saved(a, a.r_codes, a.r_ranges, a.r_rstd)))
        return PWLQ_ERR_INVALID_ARG;
    if (some && (a.gate || a.post_weight) &&
        (!a.f_codes || bad_saved(a, a.f_codes, a.f_ranges, a.f_rstd) || (a.post_weight && !a.f_rstd)))
        return PWLQ_ERR_INVALID_ARG;
    if (g.dpre || g.dpost || g.dgate) {
        const size_t need = pwlq_block_norm_backward_workspace_bytes(a.rows, a.cols,
                                                                     a.gate ? a.gate_rows : 0);
        if (!g.workspace || g.workspace_bytes < 0 || (size_t)g.workspace_bytes < need)
            return PWLQ_ERR_WORKSPACE;
        if (misaligned(g.workspace, 256)) return PWLQ_ERR_INVALID_ARG;
    }
    if (a.gate_rows == 0) {                              // rows is 0, too: neither has a row to touch
        a.gate = nullptr;
        g.dgate = nullptr;
    }
    return from_cuda(pwlq::launch_block_norm_backward(with_gate_length(a), g, as_stream(stream)));
}

size_t pwlq_act8_weight_grad_workspace_bytes(int64_t rows, int64_t outputs, int64_t cols,
                                             int dy_aligned) {
    if (check_size(rows, cols) || check_size(rows, outputs)) return 0;
    return pwlq::weight_grad_workspace(rows, outputs, cols, dy_aligned != 0);
}

int pwlq_act8_weight_grad(const void* dy, int dtype, int64_t rows, int64_t outputs, int64_t lddy,
                          const uint8_t* codes, int64_t ldc, const float* ranges, int64_t cols,
                          int group, float ratio, void* dw, int dw_dtype, int64_t lddw,
                          int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = check_size(rows, outputs)) return rc;
    if (int rc = check_size(rows, cols)) return rc;
    if (!is_dtype(dtype) || !is_dtype(dw_dtype) || (dw_dtype != PWLQ_F32 && dw_dtype != dtype))
        return PWLQ_ERR_INVALID_ARG;
    if (dtype == PWLQ_F32 || rows * ((cols + 2047) / 2048 + 1) > kMaxRows) return PWLQ_ERR_UNSUPPORTED;
    if (bad_tensor(dy, dtype, lddy, rows, outputs) || bad_format(group, ratio) ||
        bad_codes(codes, ldc, ranges, rows, cols) || bad_tensor(dw, dw_dtype, lddw, outputs, cols))
        return PWLQ_ERR_INVALID_ARG;
    const size_t need = pwlq_act8_weight_grad_workspace_bytes(rows, outputs, cols,
                                                              pwlq::rows_aligned(dy, lddy, 2));
    if (need && (!workspace || workspace_bytes < need)) return PWLQ_ERR_WORKSPACE;
    if (misaligned(workspace, 256)) return PWLQ_ERR_INVALID_ARG;
    pwlq::WeightGrad w = {dy, dtype, rows, outputs, lddy,
                          act8(codes, ldc, ranges, rows, cols, group, ratio),
                          dw, dw_dtype, lddw, accumulate != 0};
    return from_cuda(pwlq::launch_weight_grad(w, workspace, as_stream(stream)));
}

}  // extern "C"
