// C ABI of the operators on packed batches and of activations kept in eight bits: arguments are checked here, nothing is launched before all of
// them are.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <stdexcept>
#include <string>

#include "../../include/teraio.h"
#include "handles.h"
#include "kernels.h"
#include "ops_common.h"

using namespace tio;

namespace {

// what is wrong with the arguments that both attention calls have, or nullptr
const char *attention_args(const tio_packing *packing, const void *device, const void *qkv, int64_t ld, const void *o, int64_t ldo, const float *lse) {
    if (!packing) return "null argument";
    const Packing &p = packing->p;
    if (!p.H) return "the packing was built without heads";
    if (!device || !qkv || !o || !lse) return "null argument";
    if (!aligned(device) || !aligned(qkv) || !aligned(o) || !aligned(lse, 4)) return "pointers must be 16-byte aligned";
    if (ld % 8 || ldo % 8 || ld < (int64_t)(p.H + 2 * p.Hkv) * p.dh || ldo < (int64_t)p.H * p.dh)
        return "row strides must be multiples of 8 elements and at least the width of a row";
    if (!k::attn_packed_fits(p, ld, ldo)) return "the longest sequence's rows reach past 32-bit offsets (2 GiB)";
    return nullptr;
}

// what is wrong with a matrix of rows of cols elements, or nullptr
const char *matrix_args(int32_t dtype, int64_t rows, int64_t cols) {
    if (!known_type(dtype)) return "unknown element type";
    if (rows < 1 || cols < 1) return "non-positive dimension";
    if (!k::ckpt8_fits(rows, cols)) return "rows and columns must be at most 2^31 - 2^10, their product (rounded up to 32 columns) at most 2^34 - 2^13";
    return nullptr;
}

}  // namespace

extern "C" {

int tio_packing_build(const int32_t *offsets, int32_t n_seqs, int32_t dtype, int64_t H, int64_t Hkv, int64_t dh, tio_packing **out) {
    if (!offsets || !out) return fail(TIO_ERR_INVALID_ARG, "null argument");
    TIO_OP_BEGIN
    *out = new tio_packing{build_packing(offsets, n_seqs, dtype, H, Hkv, dh)};
    return TIO_OK;
    TIO_OP_END
}

int tio_packing_export(const tio_packing *packing, tio_packing_view *out) {
    if (!packing || !out) return fail(TIO_ERR_INVALID_ARG, "null argument");
    const Packing &p = packing->p;
    out->n_seqs = p.n_seqs;
    out->rows = p.rows;
    out->max_len = p.max_len;
    out->reserved = 0;
    out->data = p.data.data();
    out->bytes = (uint64_t)p.data.size() * 4;
    return TIO_OK;
}

void tio_packing_free(tio_packing *packing) { delete packing; }

int tio_op_attention_packed(void *stream, const tio_packing *packing, const void *packing_dev, const void *qkv, int64_t ld_qkv, void *o, int64_t ld_o,
                            float *lse) {
    TIO_OP_BEGIN
    if (const char *wrong = attention_args(packing, packing_dev, qkv, ld_qkv, o, ld_o, lse)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (!packing->p.rows) return TIO_OK;
    const OnDeviceOf device((hipStream_t)stream);
    k::attn_packed_fwd((hipStream_t)stream, packing->p, packing_dev, qkv, ld_qkv, o, ld_o, lse);
    return launched();
    TIO_OP_END
}

int tio_op_attention_packed_work(const tio_packing *packing, uint64_t *out_bytes) {
    if (!packing || !out_bytes) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (!packing->p.H) return fail(TIO_ERR_INVALID_ARG, "the packing was built without heads");
    *out_bytes = (uint64_t)k::attn_packed_work(packing->p);
    return TIO_OK;
}

int tio_op_attention_packed_bwd(void *stream, const tio_packing *packing, const void *packing_dev, const void *qkv, int64_t ld_qkv, const void *o,
                                const void *dO, int64_t ld_o, const float *lse, void *work, void *dqkv) {
    TIO_OP_BEGIN
    if (const char *wrong = attention_args(packing, packing_dev, qkv, ld_qkv, o, ld_o, lse)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (!dO || !work || !dqkv) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (!aligned(dO) || !aligned(work) || !aligned(dqkv)) return fail(TIO_ERR_INVALID_ARG, BAD_POINTER);
    if (!k::attn_packed_bwd_fits(packing->p)) return fail(TIO_ERR_INVALID_ARG, "too many rows times heads for the backward pass: cut the batch");
    if (!packing->p.rows) return TIO_OK;
    const OnDeviceOf device((hipStream_t)stream);
    k::attn_packed_bwd((hipStream_t)stream, packing->p, packing_dev, qkv, ld_qkv, o, dO, ld_o, lse, work, dqkv);
    return launched();
    TIO_OP_END
}

int tio_op_preference_loss_work(const tio_packing *packing, uint64_t *out_bytes) {
    if (!packing || !out_bytes) return fail(TIO_ERR_INVALID_ARG, "null argument");
    *out_bytes = (uint64_t)k::preference_work(packing->p.rows, (packing->p.n_seqs + 1) / 2);
    return TIO_OK;
}

int tio_op_preference_loss(void *stream, int32_t dtype, const tio_packing *packing, const void *packing_dev, int64_t V, const void *logits, int64_t ld,
                           const int32_t *labels, const float *ref_logp, float beta, float smoothing, int64_t total_pairs, float *seq_logp,
                           float *losses, float *loss, void *work, void *dlogits) {
    TIO_OP_BEGIN
    if (!packing || !packing_dev || !ref_logp || !seq_logp || !losses || !loss || !work) return fail(TIO_ERR_INVALID_ARG, "null argument");
    const Packing &p = packing->p;
    if (p.rows && (!logits || !labels)) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (!known_type(dtype)) return fail(TIO_ERR_INVALID_ARG, "unknown element type");
    if (p.n_seqs % 2) return fail(TIO_ERR_INVALID_ARG, "an odd number of sequences: each preferred one is followed by its rejected one");
    if (V < 1 || V > ((int64_t)1 << 28)) return fail(TIO_ERR_INVALID_ARG, "the vocabulary must be 1 to 2^28");
    const int64_t c = chunk_of(dtype);
    if (ld % c || ld < (V + c - 1) / c * c) return fail(TIO_ERR_INVALID_ARG, "the row stride must be a multiple of 16 bytes and hold the vocabulary rounded up to 16 bytes");
    if (!(beta > 0.f) || !std::isfinite(beta)) return fail(TIO_ERR_INVALID_ARG, "beta must be positive");
    if (!(smoothing >= 0.f && smoothing <= 1.f)) return fail(TIO_ERR_INVALID_ARG, "label smoothing must be 0 to 1");
    const int64_t pairs = p.n_seqs / 2;
    if (p.rows >= 1 << 22 || pairs >= 1 << 22) return fail(TIO_ERR_INVALID_ARG, "at most 2^22 - 1 rows, and pairs");
    if (total_pairs && total_pairs < pairs) return fail(TIO_ERR_INVALID_ARG, "fewer pairs in total than in this batch");
    if (!aligned(packing_dev) || !aligned(logits) || !aligned(dlogits) || !aligned(work)) return fail(TIO_ERR_INVALID_ARG, BAD_POINTER);
    if (!aligned(labels, 4) || !aligned(ref_logp, 4) || !aligned(seq_logp, 4) || !aligned(losses, 4) || !aligned(loss, 4))
        return fail(TIO_ERR_INVALID_ARG, "labels, sums and losses must be 4-byte aligned");
    int64_t longest = 0;
    for (int64_t i = 0; i < pairs; ++i) longest = std::max<int64_t>(longest, p.data[2 * i + 2] - p.data[2 * i]);
    const OnDeviceOf device((hipStream_t)stream);
    k::preference_loss((hipStream_t)stream, dtype,
                       k::PreferenceArgs{p.rows, pairs, total_pairs ? total_pairs : pairs, longest, V, ld, (const int32_t *)packing_dev, labels, logits, ref_logp, beta,
                                         smoothing, seq_logp, losses, loss, work, dlogits});
    return launched();
    TIO_OP_END
}

int tio_ckpt8_bytes(int64_t rows, int64_t cols, uint64_t *out_bytes) {
    if (!out_bytes) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (const char *wrong = matrix_args(TIO_PREC_BF16, rows, cols)) return fail(TIO_ERR_INVALID_ARG, wrong);
    *out_bytes = (uint64_t)k::ckpt8_bytes(rows, cols);
    return TIO_OK;
}

int tio_op_ckpt8_store(void *stream, int32_t dtype, int64_t rows, int64_t cols, const void *x, int64_t ldx, void *ckpt) {
    TIO_OP_BEGIN
    if (!x || !ckpt) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (const char *wrong = matrix_args(dtype, rows, cols)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (!stride_ok(ldx, cols)) return fail(TIO_ERR_INVALID_ARG, BAD_STRIDE);
    if (!aligned(x) || !aligned(ckpt)) return fail(TIO_ERR_INVALID_ARG, BAD_POINTER);
    const OnDeviceOf device((hipStream_t)stream);
    k::ckpt8_store((hipStream_t)stream, dtype, rows, cols, x, ldx, ckpt);
    return launched();
    TIO_OP_END
}

int tio_op_ckpt8_load(void *stream, int32_t dtype, int64_t rows, int64_t cols, const void *ckpt, void *x, int64_t ldx) {
    TIO_OP_BEGIN
    if (!x || !ckpt) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (const char *wrong = matrix_args(dtype, rows, cols)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (!stride_ok(ldx, cols)) return fail(TIO_ERR_INVALID_ARG, BAD_STRIDE);
    if (!aligned(x) || !aligned(ckpt)) return fail(TIO_ERR_INVALID_ARG, BAD_POINTER);
    const OnDeviceOf device((hipStream_t)stream);
    k::ckpt8_load((hipStream_t)stream, dtype, rows, cols, ckpt, x, ldx);
    return launched();
    TIO_OP_END
}

int tio_op_act_ckpt8(void *stream, int32_t dtype, int32_t act, int64_t rows, int64_t f, const void *gate, const void *up, int64_t ldu, void *y,
                     int64_t ldy, void *ckpt) {
    TIO_OP_BEGIN
    if (act != TIO_ACT_GELU && act != TIO_ACT_SWIGLU) return fail(TIO_ERR_INVALID_ARG, "unknown activation");
    const bool swiglu = act == TIO_ACT_SWIGLU;
    if (!gate || !y || !ckpt || (swiglu && !up)) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (!swiglu && up) return fail(TIO_ERR_INVALID_ARG, "GELU has one input");
    if (const char *wrong = matrix_args(dtype, rows, f)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (!stride_ok(ldu, f) || !stride_ok(ldy, f)) return fail(TIO_ERR_INVALID_ARG, BAD_STRIDE);
    if (!aligned(gate) || !aligned(up) || !aligned(y) || !aligned(ckpt)) return fail(TIO_ERR_INVALID_ARG, BAD_POINTER);
    const OnDeviceOf device((hipStream_t)stream);
    k::act_ckpt8((hipStream_t)stream, dtype, swiglu, rows, f, gate, up, ldu, y, ldy, ckpt);
    return launched();
    TIO_OP_END
}

int tio_op_act_ckpt8_bwd(void *stream, int32_t dtype, int32_t act, int64_t rows, int64_t f, const void *ckpt, const void *dy, int64_t lddy, void *dgate,
                         void *dup, int64_t ldu, void *y, int64_t ldy) {
    TIO_OP_BEGIN
    if (act != TIO_ACT_GELU && act != TIO_ACT_SWIGLU) return fail(TIO_ERR_INVALID_ARG, "unknown activation");
    const bool swiglu = act == TIO_ACT_SWIGLU;
    if (!ckpt || !dy || !dgate || (swiglu && !dup)) return fail(TIO_ERR_INVALID_ARG, "null argument");
    if (!swiglu && dup) return fail(TIO_ERR_INVALID_ARG, "GELU has one input");
    if (const char *wrong = matrix_args(dtype, rows, f)) return fail(TIO_ERR_INVALID_ARG, wrong);
    if (!stride_ok(ldu, f) || !stride_ok(lddy, f) || (y && !stride_ok(ldy, f))) return fail(TIO_ERR_INVALID_ARG, BAD_STRIDE);
    if (!aligned(ckpt) || !aligned(dy) || !aligned(dgate) || !aligned(dup) || !aligned(y)) return fail(TIO_ERR_INVALID_ARG, BAD_POINTER);
    const OnDeviceOf device((hipStream_t)stream);
    k::act_ckpt8_bwd((hipStream_t)stream, dtype, swiglu, rows, f, ckpt, dy, lddy, dgate, dup, ldu, y, ldy);
    return launched();
    TIO_OP_END
}

}  // extern "C"
