// C ABI of the operators on 4-bit weights: argument checks and kernel launches, nothing else.
#include "../../include/pwlq.h"
#include "pwlq_overlap.h"
#include "pwlq_w4.h"

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 24;
constexpr int64_t kMaxCols = (int64_t)1 << 20;
constexpr int64_t kMaxMatrices = 65535;
constexpr int64_t kMaxBlocks = (int64_t)1 << 30;           // of 1 KB
constexpr int64_t kMaxTokens = (int64_t)1 << 19;           // blocks of sixteen along a grid's second axis (65535)
constexpr int64_t kMaxPitch = (int64_t)1 << 40;

inline bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
inline cudaStream_t as_stream(void* s) { return static_cast<cudaStream_t>(s); }
inline int from_cuda(cudaError_t e) { return e == cudaSuccess ? PWLQ_OK : PWLQ_ERR_CUDA; }
inline bool is_dtype(int64_t d) { return d == PWLQ_F32 || d == PWLQ_BF16 || d == PWLQ_F16; }

int check_size(int64_t matrices, int64_t rows, int64_t cols, int64_t paired) {
    if (matrices < 1 || rows < 1 || cols < 1 || (paired != 0 && paired != 1) || (paired && rows % 2)) return PWLQ_ERR_INVALID_ARG;
    if (matrices > kMaxMatrices || rows > kMaxRows || cols > kMaxCols ||
        matrices * pwlq::w4_tiles(rows, paired != 0) * pwlq::w4_blocks(cols) > kMaxBlocks)
        return PWLQ_ERR_UNSUPPORTED;
    return PWLQ_OK;
}
bool bad_group(int64_t group) { return group != 32 && group != 64 && group != 128 && group != 256; }

int check_w4(const pwlq_w4* w) {
    if (!w) return PWLQ_ERR_INVALID_ARG;
    if (int rc = check_size(w->matrices, w->rows, w->cols, w->paired)) return rc;
    if (bad_group(w->group) || w->breakpoint < 1 || w->breakpoint > 64 || !w->data || misaligned(w->data, 16))
        return PWLQ_ERR_INVALID_ARG;
    return PWLQ_OK;
}
bool bad_rows(const void* p, int64_t dtype, int64_t ld, int64_t cols) {
    return !p || misaligned(p, pwlq::type_size((int)dtype)) || ld < cols || ld > kMaxPitch;
}
// Values [matrices, rows, cols].
bool bad_matrices(const pwlq_w4& w, const void* p, int dtype, int64_t ld, int64_t ldm) {
    return !is_dtype(dtype) || bad_rows(p, dtype, ld, w.cols) || (w.matrices > 1 && (ldm < 0 || ldm > kMaxPitch));
}

}  // namespace

extern "C" {

size_t pwlq_w4_bytes(int64_t matrices, int64_t rows, int64_t cols, int64_t group, int64_t paired) {
    if (check_size(matrices, rows, cols, paired) || bad_group(group)) return 0;
    return (size_t)(matrices * pwlq::w4_tiles(rows, paired != 0) * pwlq::w4_blocks(cols)) *
           (size_t)pwlq::w4_block_bytes(pwlq::w4_ends(group));
}

int pwlq_w4_encode(const pwlq_w4* w, const void* x, int dtype, int64_t ldx, int64_t ldm, void* stream) {
    if (int rc = check_w4(w)) return rc;
    if (bad_matrices(*w, x, dtype, ldx, ldm)) return PWLQ_ERR_INVALID_ARG;
    return from_cuda(pwlq::launch_w4_encode(*w, x, dtype, ldx, ldm, as_stream(stream)));
}

int pwlq_w4_decode(const pwlq_w4* w, void* y, int dtype, int64_t ldy, int64_t ldm, void* stream) {
    if (int rc = check_w4(w)) return rc;
    if (bad_matrices(*w, y, dtype, ldy, ldm) ||
        pwlq::matrices_meet(w->matrices, w->rows, w->cols, ldy, ldm))
        return PWLQ_ERR_INVALID_ARG;
    return from_cuda(pwlq::launch_w4_decode(*w, y, dtype, ldy, ldm, as_stream(stream)));
}

size_t pwlq_w4_linear_workspace_bytes(int64_t tokens, int64_t rows, int64_t cols, int dtype, int x_aligned) {
    if (tokens < 1 || check_size(1, rows, cols, 0) || !is_dtype(dtype) ||
        !pwlq::w4_copies(rows, cols, dtype, x_aligned != 0) || tokens > kMaxTokens)
        return 0;
    return pwlq::w4_copy_bytes(tokens, cols, dtype);
}

int pwlq_w4_linear(const pwlq_w4* w, const void* x, int dtype, int64_t tokens, int64_t ldx, void* y,
                   int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = check_w4(w)) return rc;
    if (w->matrices != 1 || !is_dtype(dtype) || tokens < 0) return PWLQ_ERR_INVALID_ARG;
    if (tokens > kMaxTokens) return PWLQ_ERR_UNSUPPORTED;
    if (tokens == 0) return PWLQ_OK;
    const int64_t outputs = w->paired ? w->rows / 2 : w->rows;
    if (bad_rows(x, dtype, ldx, w->cols) || bad_rows(y, dtype, ldy, outputs) ||
        pwlq::rows_meet(x, ldx, w->cols, y, ldy, outputs, tokens, (int64_t)pwlq::type_size(dtype)))
        return PWLQ_ERR_INVALID_ARG;
    const size_t need = pwlq_w4_linear_workspace_bytes(tokens, w->rows, w->cols, dtype,
                                                       pwlq::rows_aligned(x, ldx, pwlq::type_size(dtype)));
    if (need && (!workspace || workspace_bytes < need)) return PWLQ_ERR_WORKSPACE;
    if (need && misaligned(workspace, 256)) return PWLQ_ERR_INVALID_ARG;
    return from_cuda(pwlq::launch_w4_linear(*w, x, dtype, tokens, ldx, y, ldy, workspace, as_stream(stream)));
}

size_t pwlq_w4_moe_workspace_bytes(int64_t tokens, int64_t top, int64_t features, int64_t hidden) {
    if (tokens < 0 || tokens > PWLQ_W4_MOE_MAX_TOKENS || top < 1 || top > PWLQ_W4_MOE_MAX_TOP || features < 1 ||
        features > kMaxCols || hidden < 1 || hidden > kMaxCols)
        return 0;
    const size_t bytes = pwlq::w4_moe_workspace(tokens, top, features, hidden);
    return bytes ? bytes : 256;
}

int pwlq_w4_moe(const pwlq_w4_moe_args* args, void* stream) {
    if (!args) return PWLQ_ERR_INVALID_ARG;
    const pwlq_w4_moe_args& a = *args;
    if (int rc = check_w4(a.up)) return rc;
    if (int rc = check_w4(a.down)) return rc;
    const pwlq_w4 &up = *a.up, &down = *a.down;
    if (!up.paired || down.paired || up.matrices != down.matrices || up.cols != down.rows || up.rows != 2 * down.cols ||
        a.tokens < 0 || a.top < 1 || a.top > up.matrices || (a.normalize != 0 && a.normalize != 1) ||
        !is_dtype(a.dtype) || (a.router_dtype != a.dtype && a.router_dtype != PWLQ_F32))
        return PWLQ_ERR_INVALID_ARG;
    if (a.tokens > PWLQ_W4_MOE_MAX_TOKENS || up.matrices > PWLQ_W4_MOE_MAX_EXPERTS || a.top > PWLQ_W4_MOE_MAX_TOP)
        return PWLQ_ERR_UNSUPPORTED;
    if (a.tokens == 0) return PWLQ_OK;
    if (bad_rows(a.x, a.dtype, a.ldx, up.cols) || bad_rows(a.y, a.dtype, a.ldy, up.cols) ||
        bad_rows(a.router, a.router_dtype, a.ldrouter, up.cols) || misaligned(a.chosen, 4) || misaligned(a.weights, 4))
        return PWLQ_ERR_INVALID_ARG;
    if (!a.workspace || a.workspace_bytes < 0 ||
        (size_t)a.workspace_bytes < pwlq_w4_moe_workspace_bytes(a.tokens, a.top, down.rows, down.cols))
        return PWLQ_ERR_WORKSPACE;
    if (misaligned(a.workspace, 256)) return PWLQ_ERR_INVALID_ARG;
    return from_cuda(pwlq::launch_w4_moe(a, as_stream(stream)));
}

}  // extern "C"
