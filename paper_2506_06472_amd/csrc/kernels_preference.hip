// Paired preference loss on the logits of a packed batch, and its gradient.
//
// Sequences 2 i and 2 i + 1 are a preferred and a rejected answer.  With x a row of logits and y its label, a counted row adds
// log p = x[y] - log sum exp x to its sequence; z = beta ((sum of the preferred - its reference) - (sum of the rejected - its reference)),
// a pair's loss is -(1 - s) log sigmoid(z) - s log sigmoid(-z) and the loss their mean.  The gradient of a counted row is
// w (onehot(y) - softmax(x)) with w the derivative of the loss by its sequence's sum, the other rows' is zero.
//
// The weight of a row depends on every row of its pair, so that the logits are needed twice: a launch over the rows takes maximum, sum
// and log p of each, one over the pairs their sums, losses and the rows' weights, one over the logits writes the gradient.  Bound: HBM.
// log p is summed over a sequence in 64 bits, in a fixed order: of sums of some thousand the difference of two counts.
#include "../../include/teraio.h"
#include "device_common.h"
#include "kernels.h"

namespace tio {
namespace k {

namespace {

constexpr int TPB = 256;
constexpr float L2E = 1.4426950408889634f;

// maximum and the base-2 logarithm of the sum of exp(x - maximum) of a row
struct RowStat {
    float top, log2_sum;
};

// the counted row's label, or -1
__device__ __forceinline__ int32_t label_of(const int32_t *labels, int64_t row, int64_t Vn) {
    const int32_t y = labels[row];
    return y >= 0 && y < Vn ? y : -1;
}

// A workgroup to a row, in pieces of NCH 16-byte chunks to a thread, all of a piece's loads on their way together; every thread has a maximum
// and a sum of its own, which meet at the end.
template <typename T, int NCH, int NT>
__global__ void __launch_bounds__(NT) pref_rows_k(const T *__restrict__ logits, int64_t ld, const int32_t *__restrict__ labels, int64_t Vn,
                                                  double *__restrict__ logp, RowStat *__restrict__ stats) {
    constexpr int V = Vec16<T>::N;
    __shared__ float red[NT / 64];
    const int64_t row = blockIdx.x;
    const int32_t y = label_of(labels, row, Vn);
    if (y < 0) {
        if (threadIdx.x == 0) logp[row] = 0.0;
        return;
    }
    const T *xr = logits + row * ld;
    const int nv = (int)Vn, nchunk = (nv + V - 1) / V;
    const __amdgpu_buffer_rsrc_t r = buffer_over(xr, (uint32_t)nchunk * 16u);
    float m = -INFINITY, s = 0.f;
    for (int base = 0; base < nchunk; base += NT * NCH) {
        Vec16<T> a[NCH];
#pragma unroll
        for (int i = 0; i < NCH; ++i) buffer_load16(a[i], r, (uint32_t)(base + threadIdx.x + NT * i) * 16u);
        float top = m;
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int c = base + threadIdx.x + NT * i;
            if (c >= nchunk) continue;
            float f[V]; a[i].get(f);
            if ((c + 1) * V <= nv) {
#pragma unroll
                for (int j = 0; j < V; ++j) top = fmaxf(top, f[j]);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) if (c * V + j < nv) top = fmaxf(top, f[j]);
            }
        }
        const float ref = top == -INFINITY ? 0.f : top;                  // nothing but -inf so far: probabilities 0, not NaN
        s *= __builtin_amdgcn_exp2f((m - ref) * L2E);
        m = top;
#pragma unroll
        for (int i = 0; i < NCH; ++i) {
            const int c = base + threadIdx.x + NT * i;
            if (c >= nchunk) continue;
            float f[V]; a[i].get(f);
            if ((c + 1) * V <= nv) {
#pragma unroll
                for (int j = 0; j < V; ++j) s += __builtin_amdgcn_exp2f((f[j] - ref) * L2E);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) if (c * V + j < nv) s += __builtin_amdgcn_exp2f((f[j] - ref) * L2E);
            }
        }
    }
    const float M = block_max<NT / 64>(m, red);
    const float tot = block_sum<NT / 64>(m == -INFINITY ? s : s * __builtin_amdgcn_exp2f((m - M) * L2E), red);
    if (threadIdx.x == 0) {
        logp[row] = ((double)to_f32(xr[y]) - (double)M) - (double)logf(tot);
        stats[row] = RowStat{M, log2f(tot)};
    }
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ double block_sum_f64(double v, double *red) {
    v = wave_sum_f64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int i = 0; i < TPB / 64; ++i) t += red[i];
    return t;
}

// A workgroup to a pair.  weight: the derivative of the loss by each row's log p.
__global__ void __launch_bounds__(TPB) pref_pairs_k(const int32_t *__restrict__ offsets, const double *__restrict__ logp,
                                                    const int32_t *__restrict__ labels, int64_t Vn, const float *__restrict__ ref, float beta,
                                                    float smoothing, float inv_pairs, float *__restrict__ seq, float *__restrict__ losses,
                                                    float *__restrict__ weight) {
    __shared__ double red[TPB / 64];
    const int64_t pair = blockIdx.x;
    const int32_t at[3] = {offsets[2 * pair], offsets[2 * pair + 1], offsets[2 * pair + 2]};
    double sum[2];
    for (int i = 0; i < 2; ++i) {
        double v = 0.0;
        for (int64_t r = at[i] + threadIdx.x; r < at[i + 1]; r += TPB) v += logp[r];
        sum[i] = block_sum_f64(v, red);
    }
    const double z = (double)beta * ((sum[0] - (double)ref[2 * pair]) - (sum[1] - (double)ref[2 * pair + 1]));
    const double t = exp(-fabs(z)), log_sigmoid = (z < 0.0 ? z : 0.0) - log1p(t);
    const double down = z >= 0.0 ? t / (1.0 + t) : 1.0 / (1.0 + t);      // sigmoid(-z)
    const double s = smoothing;
    if (threadIdx.x == 0) {
        seq[2 * pair] = (float)sum[0];
        seq[2 * pair + 1] = (float)sum[1];
        losses[pair] = (float)(-(1.0 - s) * log_sigmoid - s * (log_sigmoid - z));
    }
    if (weight) {
        // 1 - sigmoid(-z) is sigmoid(z)
        const float w = (float)(-(double)beta * (double)inv_pairs * ((1.0 - s) * down - s * (z >= 0.0 ? 1.0 / (1.0 + t) : t / (1.0 + t))));
        for (int64_t r = at[0] + threadIdx.x; r < at[2]; r += TPB) weight[r] = label_of(labels, r, Vn) < 0 ? 0.f : r < at[1] ? w : -w;
    }
}

// Piece blockIdx.x of row blockIdx.y: NCH chunks to a thread.  d may be the logits.
template <typename T, int NCH>
__global__ void __launch_bounds__(TPB) pref_grad_k(const T *logits, T *d, int64_t ld, const int32_t *__restrict__ labels, int64_t Vn,
                                                   const RowStat *__restrict__ stats, const float *__restrict__ weight) {
    constexpr int V = Vec16<T>::N;
    const int64_t row = blockIdx.y;
    const int nv = (int)Vn, nchunk = (nv + V - 1) / V, first = blockIdx.x * (TPB * NCH) + threadIdx.x;
    const int32_t y = label_of(labels, row, Vn);
    const __amdgpu_buffer_rsrc_t out = buffer_over(d + row * ld, (uint32_t)nchunk * 16u);
    if (y < 0) {
        Vec16<T> zero;
        const float f[V] = {};
        zero.set(f);
#pragma unroll
        for (int i = 0; i < NCH; ++i) buffer_store16(zero, out, (uint32_t)(first + TPB * i) * 16u);
        return;
    }
    const __amdgpu_buffer_rsrc_t in = buffer_over(logits + row * ld, (uint32_t)nchunk * 16u);
    Vec16<T> a[NCH];
#pragma unroll
    for (int i = 0; i < NCH; ++i) buffer_load16(a[i], in, (uint32_t)(first + TPB * i) * 16u);
    const RowStat st = stats[row];
    const float w = weight[row];
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
        const int c = first + TPB * i;
        if (c >= nchunk) continue;
        float f[V]; a[i].get(f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = -w * __builtin_amdgcn_exp2f(fmaf(f[j] - st.top, L2E, -st.log2_sum));
        if (y >= c * V && y < (c + 1) * V) {
#pragma unroll
            for (int j = 0; j < V; ++j) if (c * V + j == y) f[j] += w;
        }
        if ((c + 1) * V > nv) {
#pragma unroll
            for (int j = 0; j < V; ++j) if (c * V + j >= nv) f[j] = 0.f;
        }
        a[i].set(f);
        buffer_store16(a[i], out, (uint32_t)c * 16u);
    }
}

template <typename T, int NCH> void launch_grad(hipStream_t s, const PreferenceArgs &a, const RowStat *stats, const float *weight) {
    const int64_t nchunk = (a.V + Vec16<T>::N - 1) / Vec16<T>::N;
    // a grid has at most 2^16 - 1 rows of workgroups
    for (int64_t r = 0; r < a.rows; r += 65535) {
        const dim3 grid((unsigned)((nchunk + TPB * NCH - 1) / (TPB * NCH)), (unsigned)(a.rows - r < 65535 ? a.rows - r : 65535));
        pref_grad_k<T, NCH><<<grid, TPB, 0, s>>>((const T *)a.logits + r * a.ld, (T *)a.dlogits + r * a.ld, a.ld, a.labels + r, a.V, stats + r, weight + r);
    }
}
template <typename T> void launch(hipStream_t s, const PreferenceArgs &a) {
    double *const logp = (double *)a.work;
    RowStat *const stats = (RowStat *)(logp + a.rows);
    float *const weight = (float *)(stats + a.rows);
    const int64_t nchunk = (a.V + Vec16<T>::N - 1) / Vec16<T>::N;
    if (a.rows) {
        const unsigned rows = (unsigned)a.rows;
        if (nchunk <= TPB) pref_rows_k<T, 1, TPB><<<rows, TPB, 0, s>>>((const T *)a.logits, a.ld, a.labels, a.V, logp, stats);
        else if (nchunk <= 4 * TPB) pref_rows_k<T, 4, TPB><<<rows, TPB, 0, s>>>((const T *)a.logits, a.ld, a.labels, a.V, logp, stats);
        else pref_rows_k<T, 8, TPB><<<rows, TPB, 0, s>>>((const T *)a.logits, a.ld, a.labels, a.V, logp, stats);
    }
    pref_pairs_k<<<(unsigned)a.pairs, TPB, 0, s>>>(a.offsets, logp, a.labels, a.V, a.ref, a.beta, a.smoothing, 1.0f / (float)a.total_pairs, a.seq,
                                                  a.losses, a.dlogits ? weight : nullptr);
    loss_reduce(s, a.losses, a.loss, a.pairs, a.total_pairs, false);
    if (a.dlogits && a.rows) {
        if (nchunk <= TPB) launch_grad<T, 1>(s, a, stats, weight);
        else launch_grad<T, 4>(s, a, stats, weight);
    }
}

}  // namespace

int64_t preference_work(int64_t rows) { return (rows * (int64_t)(sizeof(double) + sizeof(RowStat) + sizeof(float)) + 15) / 16 * 16 + 16; }

void preference_loss(hipStream_t s, int dtype, const PreferenceArgs &a) {
    if (dtype == TIO_PREC_BF16) launch<bf16_t>(s, a);
    else launch<float>(s, a);
}

}  // namespace k
}  // namespace tio
