// C ABI of the operators of a layer trained in 8-bit floating point: arguments are checked here, nothing is launched before all of them are.
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>

#include "../../include/teraio.h"
#include "fp8_blocks.h"
#include "kernels.h"
#include "ops_common.h"

using namespace tio;

namespace {

bool known_form(int32_t form) { return form == TIO_FP8_E4M3 || form == TIO_FP8_E5M2; }

// is one buffer handed in as two matrices whose rows are at different places?
bool crossed(const void *x, int64_t ldx, const void *y, int64_t ldy, int64_t rows) { return x == y && ldx != ldy && rows > 1; }
const char *const CROSSED = "a buffer that is read and written must have one stride";

// what is wrong with a stored matrix's sizes, or nullptr
const char *fp8_args(int64_t rows, int64_t cols) {
    if (rows < 1 || cols < 1) return "non-positive dimension";
    if (!k::fp8_fits(rows, cols)) return "rows and columns must be at most 2^22, their product (rounded up to 16 and 128) at most 2^36";
    return nullptr;
}

// the mask's parameters from a probability; false: not a probability
bool make_dropout(double p, uint64_t seed, uint64_t offset, k::Dropout &d) {
    if (!(p >= 0.0 && p < 1.0)) return false;
    const double limit = std::nearbyint(p * 65536.0);          // ties to even
    if (limit > 65535.0) return false;
    d = k::Dropout{(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)offset, (uint32_t)(offset >> 32), (uint32_t)limit, (float)(65536.0 / (65536.0 - limit))};
    return true;
}
const char *const BAD_PROBABILITY = "the probability must be at least 0 and, as a number of 1/65536, below 1";

// what is wrong with the arguments that both passes of the residual norm have, or nullptr
const char *residual_args(int32_t dtype, const tio_residual_cfg *cfg, int64_t rows, int64_t d, int64_t ld, const void *gate, int64_t ldg, const void *post_gain,
                          const void *post_bias, const void *gain) {
    if (!cfg || !gain) return "null argument";
    if (!known_type(dtype)) return "unknown element type";
    if (rows < 1 || d < 1) return "non-positive dimension";
    if (d > k::RESIDUAL_WIDEST) return "a row must be at most 8192 wide";
    if (rows > (int64_t)1 << 31) return "at most 2^31 rows";
    if (!stride_ok(ld, d) || (gate && ldg != 0 && !stride_ok(ldg, d))) return BAD_STRIDE;
    if (!(cfg->eps >= 0.f) || !std::isfinite(cfg->eps) || !std::isfinite(cfg->resid_scale) || !std::isfinite(cfg->branch_scale))
        return "eps must not be negative, and the scales finite";
    if (post_bias && !post_gain) return "a bias without the norm's gain";
    if (!aligned(gate) || !aligned(post_gain) || !aligned(post_bias) || !aligned(gain)) return BAD_POINTER;
    return nullptr;
}
bool residual_of(const tio_residual_cfg &c, k::ResidualArgs &a) {
    a.rms = c.rms != 0;
    a.eps = c.eps;
    a.resid_scale = c.resid_scale;
    a.branch_scale = c.branch_scale;
    return make_dropout(c.p, c.seed, c.offset, a.drop);
}

// the backward pass, from y or (from_x) from the forward pass's x in its place
int residual_backward(void *stream, int32_t dtype, const tio_residual_cfg *cfg, int64_t rows, int64_t d, int64_t ld, const void *branch, bool from_x, const void *y,
                      const void *gate, int64_t ldg, const void *post_gain, const void *post_bias, const void *gain, const float *stats,
                      const void *dy, const void *dh, void *dx, void *dbranch, void *dgate, void *dpost_gain, void *dpost_bias, void *dgain, void *dbias,
                      void *work) {
    TIO_OP_BEGIN
    if (!branch || !y || !stats || !dy || !dh || !dx || !dbranch || !dgain || !work) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (const char *wrong = residual_args(dtype, cfg, rows, d, ld, gate, ldg, post_gain, post_bias, gain)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (cfg->rms && (post_bias || dpost_bias || dbias)) return fail(TIO_ERR_INVALID_ARG, "the root-mean-square norm has no bias");
    if (!gate != !dgate || !post_gain != !dpost_gain || (dpost_bias && !post_gain))
        return fail(TIO_ERR_INVALID_ARG, "a gradient is given exactly where its operand is");
    if (!aligned(branch) || !aligned(y) || !aligned(stats) || !aligned(dy) || !aligned(dh) || !aligned(dx) || !aligned(dbranch) || !aligned(dgate) ||
        !aligned(dpost_gain) || !aligned(dpost_bias) || !aligned(dgain) || !aligned(dbias) || !aligned(work))
        return fail(TIO_ERR_INVALID_ARG, BAD_POINTER);
    k::ResidualArgs a = {};
    if (!residual_of(*cfg, a)) return fail(TIO_ERR_INVALID_ARG, BAD_PROBABILITY);
    a.rows = rows; a.d = d; a.ld = ld; a.ldg = ldg;
    a.branch = branch; a.gate = gate; a.post_gain = post_gain; a.post_bias = post_bias; a.gain = gain;
    a.from_x = from_x; a.y = const_cast<void *>(y); a.stats = const_cast<float *>(stats);
    a.dy = dy; a.dh = dh; a.dx = dx; a.dbranch = dbranch; a.dgate = dgate; a.dpost_gain = dpost_gain; a.dpost_bias = dpost_bias;
    a.dgain = dgain; a.dbias = dbias; a.work = work;
    const OnDeviceOf device((hipStream_t)stream);
    k::residual_norm_bwd((hipStream_t)stream, dtype, a);
    return launched();
    TIO_OP_END
}

}  // namespace

extern "C" {

int tio_fp8_bytes(int64_t rows, int64_t cols, uint64_t *out_bytes) {
    if (!out_bytes) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (const char *wrong = fp8_args(rows, cols)) return fail(TIO_ERR_INVALID_ARG, wrong);
    *out_bytes = (uint64_t)k::fp8_bytes(rows, cols);
    return TIO_OK;
}

int tio_op_fp8_store(void *stream, int32_t dtype, int32_t form, int32_t tiles, int64_t rows, int64_t cols, const void *x, int64_t ldx, void *out,
                     void *out_t) {
    TIO_OP_BEGIN
    if (!x || (!out && !out_t)) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (!known_type(dtype) || !known_form(form)) return fail(TIO_ERR_INVALID_ARG, "unknown element type");
    if (const char *wrong = fp8_args(rows, cols)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (out_t)
        if (const char *wrong = fp8_args(cols, rows)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (!stride_ok(ldx, cols)) return fail(TIO_ERR_INVALID_ARG, BAD_STRIDE);
    if (!aligned(x) || !aligned(out) || !aligned(out_t)) return fail(TIO_ERR_INVALID_ARG, BAD_POINTER);
    const OnDeviceOf device((hipStream_t)stream);
    k::fp8_store((hipStream_t)stream, dtype, form, tiles != 0, rows, cols, x, ldx, out, out_t);
    return launched();
    TIO_OP_END
}

int tio_op_fp8_load(void *stream, int32_t dtype, int32_t form, int64_t rows, int64_t cols, const void *in, void *x, int64_t ldx) {
    TIO_OP_BEGIN
    if (!in || !x) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (!known_type(dtype) || !known_form(form)) return fail(TIO_ERR_INVALID_ARG, "unknown element type");
    if (const char *wrong = fp8_args(rows, cols)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (!stride_ok(ldx, cols)) return fail(TIO_ERR_INVALID_ARG, BAD_STRIDE);
    if (!aligned(in) || !aligned(x)) return fail(TIO_ERR_INVALID_ARG, BAD_POINTER);
    const OnDeviceOf device((hipStream_t)stream);
    k::fp8_load((hipStream_t)stream, dtype, form, rows, cols, in, x, ldx);
    return launched();
    TIO_OP_END
}

int tio_op_gemm_fp8_work(int64_t M, int64_t N, int64_t K, uint64_t *out_bytes) {
    if (!out_bytes) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (const char *wrong = fp8_args(M, K)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (const char *wrong = fp8_args(N, K)) return fail(TIO_ERR_INVALID_ARG, wrong);
    *out_bytes = (uint64_t)k::gemm_fp8_work(M, N, K);
    return TIO_OK;
}

int tio_op_gemm_fp8(void *stream, int32_t dtype, int64_t M, int64_t N, int64_t K, int32_t form_a, const void *A, int32_t form_b, const void *B, const void *bias,
                    const void *resid, int64_t ldr, void *C, int64_t ldc, void *work) {
    TIO_OP_BEGIN
    if (!A || !B || !C) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (!known_type(dtype) || !known_form(form_a) || !known_form(form_b)) return fail(TIO_ERR_INVALID_ARG, "unknown element type");
    if (const char *wrong = fp8_args(M, K)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (const char *wrong = fp8_args(N, K)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (!stride_ok(ldc, N) || (resid && !stride_ok(ldr, N))) return fail(TIO_ERR_INVALID_ARG, BAD_STRIDE);
    if (!aligned(A) || !aligned(B) || !aligned(bias) || !aligned(resid) || !aligned(C) || !aligned(work)) return fail(TIO_ERR_INVALID_ARG, BAD_POINTER);
    if (crossed(resid, ldr, C, ldc, M)) return fail(TIO_ERR_INVALID_ARG, CROSSED);
    if (!work && k::gemm_fp8_work(M, N, K)) return fail(TIO_ERR_INVALID_ARG, "this product needs work memory");
    const OnDeviceOf device((hipStream_t)stream);
    k::gemm_fp8((hipStream_t)stream, dtype, k::Fp8Product{M, N, K, form_a, A, form_b, B, bias, resid, ldr, C, ldc, work});
    return launched();
    TIO_OP_END
}

int tio_op_gemm_fp8_route(int32_t dtype, int64_t M, int64_t N, int64_t K, int32_t *out_rows, int32_t *out_cols, int32_t *out_deep,
                          int32_t *out_ranges) {
    if (!out_rows || !out_cols || !out_deep || !out_ranges) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (!known_type(dtype)) return fail(TIO_ERR_INVALID_ARG, "unknown element type");
    if (const char *wrong = fp8_args(M, K)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (const char *wrong = fp8_args(N, K)) return fail(TIO_ERR_INVALID_ARG, wrong);
    k::gemm_fp8_route(dtype, M, N, K, out_rows, out_cols, out_deep, out_ranges);
    return TIO_OK;
}

int tio_op_residual_norm(void *stream, int32_t dtype, const tio_residual_cfg *cfg, int64_t rows, int64_t d, int64_t ld, const void *branch, const void *x,
                         const void *gate, int64_t ldg, const void *post_gain, const void *post_bias, const void *gain, const void *bias, void *y, void *h,
                         float *stats) {
    TIO_OP_BEGIN
    if (!branch || !x || !y || !h || !stats) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (const char *wrong = residual_args(dtype, cfg, rows, d, ld, gate, ldg, post_gain, post_bias, gain)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (cfg->rms && (post_bias || bias)) return fail(TIO_ERR_INVALID_ARG, "the root-mean-square norm has no bias");
    if (!aligned(branch) || !aligned(x) || !aligned(bias) || !aligned(y) || !aligned(h) || !aligned(stats)) return fail(TIO_ERR_INVALID_ARG, BAD_POINTER);
    k::ResidualArgs a = {};
    if (!residual_of(*cfg, a)) return fail(TIO_ERR_INVALID_ARG, BAD_PROBABILITY);
    a.rows = rows; a.d = d; a.ld = ld; a.ldg = ldg;
    a.branch = branch; a.x = x; a.gate = gate; a.post_gain = post_gain; a.post_bias = post_bias; a.gain = gain; a.bias = bias;
    a.y = y; a.h = h; a.stats = stats;
    const OnDeviceOf device((hipStream_t)stream);
    k::residual_norm((hipStream_t)stream, dtype, a);
    return launched();
    TIO_OP_END
}

int tio_op_residual_norm_bwd_work(int64_t rows, int64_t d, uint64_t *out_bytes) {
    if (!out_bytes) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (rows < 1 || d < 1 || d > k::RESIDUAL_WIDEST || rows > (int64_t)1 << 31) return fail(TIO_ERR_INVALID_ARG, "rows must be 1 to 2^31, their width 1 to 8192");
    *out_bytes = (uint64_t)k::residual_norm_bwd_work(rows, d);
    return TIO_OK;
}

int tio_op_residual_norm_bwd(void *stream, int32_t dtype, const tio_residual_cfg *cfg, int64_t rows, int64_t d, int64_t ld, const void *branch, const void *y,
                             const void *gate, int64_t ldg, const void *post_gain, const void *post_bias, const void *gain, const float *stats,
                             const void *dy, const void *dh, void *dx, void *dbranch, void *dgate, void *dpost_gain, void *dpost_bias, void *dgain, void *dbias,
                             void *work) {
    return residual_backward(stream, dtype, cfg, rows, d, ld, branch, false, y, gate, ldg, post_gain, post_bias, gain, stats, dy, dh, dx, dbranch, dgate, dpost_gain, dpost_bias,
                             dgain, dbias, work);
}

int tio_op_residual_norm_bwd_from_x(void *stream, int32_t dtype, const tio_residual_cfg *cfg, int64_t rows, int64_t d, int64_t ld, const void *branch, const void *x,
                                    const void *gate, int64_t ldg, const void *post_gain, const void *post_bias, const void *gain, const float *stats,
                                    const void *dy, const void *dh, void *dx, void *dbranch, void *dgate, void *dpost_gain, void *dpost_bias, void *dgain, void *dbias,
                                    void *work) {
    return residual_backward(stream, dtype, cfg, rows, d, ld, branch, true, x, gate, ldg, post_gain, post_bias, gain, stats, dy, dh, dx, dbranch, dgate, dpost_gain, dpost_bias,
                             dgain, dbias, work);
}

int tio_op_dropout(void *stream, int32_t dtype, int64_t rows, int64_t cols, const void *x, int64_t ldx, const void *resid, int64_t ldr, void *y, int64_t ldy,
                   double p, uint64_t seed, uint64_t offset) {
    TIO_OP_BEGIN
    if (!x || !y) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (!known_type(dtype)) return fail(TIO_ERR_INVALID_ARG, "unknown element type");
    if (rows < 1 || cols < 1) return fail(TIO_ERR_INVALID_ARG, "non-positive dimension");
    if (!k::dropout_fits(rows, cols)) return fail(TIO_ERR_INVALID_ARG, "rows times columns (in eights) must be below 2^31");
    if (!stride_ok(ldx, cols) || !stride_ok(ldy, cols) || (resid && !stride_ok(ldr, cols))) return fail(TIO_ERR_INVALID_ARG, BAD_STRIDE);
    if (!aligned(x) || !aligned(resid) || !aligned(y)) return fail(TIO_ERR_INVALID_ARG, BAD_POINTER);
    if (crossed(x, ldx, y, ldy, rows) || crossed(resid, ldr, y, ldy, rows)) return fail(TIO_ERR_INVALID_ARG, CROSSED);
    k::Dropout d;
    if (!make_dropout(p, seed, offset, d)) return fail(TIO_ERR_INVALID_ARG, BAD_PROBABILITY);
    const OnDeviceOf device((hipStream_t)stream);
    k::dropout((hipStream_t)stream, dtype, rows, cols, x, ldx, resid, ldr, y, ldy, d);
    return launched();
    TIO_OP_END
}

int tio_op_rope_axes(void *stream, int32_t dtype, int64_t rows, int64_t heads, int64_t dh, const void *x, int64_t ldx, void *y, int64_t ldy,
                     const int32_t *positions, int32_t n_axes, const int32_t *sections, float theta, int32_t own_ladder, int32_t inverse) {
    TIO_OP_BEGIN
    if (!x || !y || !positions || !sections) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (!known_type(dtype)) return fail(TIO_ERR_INVALID_ARG, "unknown element type");
    if (rows < 1 || heads < 1 || rows >= (int64_t)1 << 31 || heads > 65536) return fail(TIO_ERR_INVALID_ARG, "rows must be 1 to 2^31 - 1, heads 1 to 65536");
    if (dh < 8 || dh % 8 || dh > 2 * k::ROPE_PAIRS) return fail(TIO_ERR_INVALID_ARG, "the head size must be a multiple of 8, at most 256");
    if (n_axes < 1 || n_axes > 8) return fail(TIO_ERR_INVALID_ARG, "1 to 8 axes");
    int64_t pairs = 0;
    for (int i = 0; i < n_axes; ++i) {
        if (sections[i] < 1 || sections[i] > k::ROPE_PAIRS) return fail(TIO_ERR_INVALID_ARG, "every axis has 1 to 128 pairs");
        pairs += sections[i];
    }
    if (pairs > dh / 2) return fail(TIO_ERR_INVALID_ARG, "the axes have more pairs than a head");
    if (!(theta > 0.f) || !std::isfinite(theta)) return fail(TIO_ERR_INVALID_ARG, "theta must be positive");
    if (!stride_ok(ldx, heads * dh) || !stride_ok(ldy, heads * dh)) return fail(TIO_ERR_INVALID_ARG, BAD_STRIDE);
    if (!aligned(x) || !aligned(y) || !aligned(positions, 4)) return fail(TIO_ERR_INVALID_ARG, BAD_POINTER);
    if (crossed(x, ldx, y, ldy, rows)) return fail(TIO_ERR_INVALID_ARG, CROSSED);
    const OnDeviceOf device((hipStream_t)stream);
    k::rope_axes((hipStream_t)stream, dtype, rows, (int)heads, (int)dh, x, ldx, y, ldy, positions, n_axes, sections, theta, own_ladder != 0, inverse != 0);
    return launched();
    TIO_OP_END
}

}  // extern "C"
