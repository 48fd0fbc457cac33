// Paired preference loss on the logits of a packed batch, and its gradient.
//
// Sequences 2 i and 2 i + 1 are a preferred and a rejected answer.  With x a row of logits and y its label, a counted row adds
// log p = x[y] - log sum exp x to its sequence; z = beta ((sum of the preferred - its reference) - (sum of the rejected - its reference)),
// a pair's loss is -(1 - s) log sigmoid(z) - s log sigmoid(-z) and the loss their mean.  The gradient of a counted row is
// w (onehot(y) - softmax(x)) with w the derivative of the loss by its sequence's sum, the other rows' is zero.
//
// The weight of a row depends on every row of its pair, so the logits are needed twice: a launch over the rows takes maximum, sum and log p of
// each (counted rows only), one over the pairs their sums, losses and weights, one over the logits writes the gradient.  Bound: HBM (8192 x 32000,
// bf16, 6368 rows counted: 68 us for 408 MB, 6.0 TB/s; 135 us for as much again, part of it from the memory-side cache, and 524 MB written).
// log p is summed over a sequence in 64 bits, in a fixed order: of sums of some thousand the difference of two counts.
#include "../../include/teraio.h"
#include "device_common.h"
#include "kernels.h"

namespace tio {
namespace k {

namespace {

constexpr int TPB = 256;
constexpr float L2E = 1.4426950408889634f;

// of a row, in the base-2 domain: the reference of its exponentials and the logarithm of their sum
struct RowStat {
    float top, log2_sum;
};

// the counted row's label, or -1
__device__ __forceinline__ int32_t label_of(const int32_t *labels, int64_t row, int64_t Vn) {
    const int32_t y = labels[row];
    return y >= 0 && y < Vn ? y : -1;
}

// A workgroup to a row, in pieces of NCH 16-byte chunks to a thread, all of a piece's loads on their way together; every thread has a maximum
// and a sum of its own, which meet at the end.  Exponentials are exp2(x log2(e) - t), one fused multiply-add, with t the thread's maximum times
// log2(e), rounded: any number near would do, so logits of 1e4 lose nothing by its rounding.
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
    float top = -INFINITY, t = -INFINITY, s = 0.f;
    for (int base = 0; base < nchunk; base += NT * NCH) {
        Vec16<T> a[NCH];
#pragma unroll
        for (int i = 0; i < NCH; ++i) buffer_load16(a[i], r, (uint32_t)(base + threadIdx.x + NT * i) * 16u);
        auto each = [&](auto take) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < NCH; ++i) {
                const int c = base + threadIdx.x + NT * i;
                if (c >= nchunk) continue;
                float f[V]; a[i].get(f);
                if ((c + 1) * V <= nv) {
#pragma unroll
                    for (int j = 0; j < V; ++j) take(f[j]);
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j) if (c * V + j < nv) take(f[j]);
                }
            }
        };
        each([&](float x) __attribute__((always_inline)) { top = fmaxf(top, x); });
        const float ref = top == -INFINITY ? 0.f : top * L2E;            // nothing but -inf so far: exponentials 0, not NaN
        s *= __builtin_amdgcn_exp2f(t - ref);
        t = top == -INFINITY ? top : ref;
        each([&](float x) __attribute__((always_inline)) { s += __builtin_amdgcn_exp2f(fmaf(x, L2E, -ref)); });
    }
    const float M = block_max<NT / 64>(t, red);
    const float tot = block_sum<NT / 64>(t == -INFINITY ? s : s * __builtin_amdgcn_exp2f(t - M), red);
    if (threadIdx.x == 0) {
        const float log2_sum = log2f(tot);
        // (x log2(e) - M) - log2(sum), over log2(e)
        logp[row] = (((double)to_f32(xr[y]) * (double)L2E - (double)M) - (double)log2_sum) / (double)L2E;
        stats[row] = RowStat{M, log2_sum};
    }
}

template <int NW> __device__ __forceinline__ double block_sum_f64(double v, double *red) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int i = 0; i < NW; ++i) t += red[i];
    return t;
}

// A workgroup to a pair.  weight: the derivative of the loss by the sum of a pair's preferred sequence.  The pairs' mean is left to the next launch: a
// counter that tells the last workgroup cost 6 us, for the caches it has to write back first.
constexpr int PAIR_THREADS = 1024;
__global__ void __launch_bounds__(PAIR_THREADS) pref_pairs_k(const int32_t *__restrict__ offsets, int rows, const double *__restrict__ logp,
                                                             const float *__restrict__ ref, float beta, float smoothing, float total_pairs,
                                                             float *__restrict__ seq, float *__restrict__ losses, float *__restrict__ weight) {
    __shared__ double red[2][PAIR_THREADS / 64];
    const int64_t pair = blockIdx.x;
    int32_t at[3];
    for (int i = 0; i < 3; ++i) at[i] = min(max(offsets[2 * pair + i], 0), rows);        // nothing outside the batch is read, whatever they are
    double sum[2] = {0.0, 0.0};
    for (int i = 0; i < 2; ++i) {
        int64_t r = at[i] + threadIdx.x;
        for (; r + 3 * PAIR_THREADS < at[i + 1]; r += 4 * PAIR_THREADS) {          // four loads on their way
            double v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = logp[r + u * PAIR_THREADS];
            sum[i] += (v[0] + v[1]) + (v[2] + v[3]);
        }
        for (; r < at[i + 1]; r += PAIR_THREADS) sum[i] += logp[r];
    }
    sum[0] = block_sum_f64<PAIR_THREADS / 64>(sum[0], red[0]);
    sum[1] = block_sum_f64<PAIR_THREADS / 64>(sum[1], red[1]);
    if (threadIdx.x == 0) {
        const double z = (double)beta * ((sum[0] - (double)ref[2 * pair]) - (sum[1] - (double)ref[2 * pair + 1]));
        // 32 bits are enough from here on: the functions of 64 take a single thread a microsecond each
        const float zf = (float)z, e = expf(-fabsf(zf)), big = 1.0f / (1.0f + e), small = e * big, log_big = -log1pf(e);
        const float up = zf >= 0.f ? big : small, down = zf >= 0.f ? small : big;                          // sigmoid(z), sigmoid(-z)
        const float log_up = zf >= 0.f ? log_big : log_big + zf, log_down = zf >= 0.f ? log_big - zf : log_big, s = smoothing;
        seq[2 * pair] = (float)sum[0];
        seq[2 * pair + 1] = (float)sum[1];
        losses[pair] = -(s < 1.f ? (1.0f - s) * log_up : 0.f) - (s > 0.f ? s * log_down : 0.f);      // no 0 times infinity
        weight[pair] = -beta * ((1.0f - s) * down - s * up) / total_pairs;
    }
}

// the mean of the pairs' losses, by a workgroup of TPB threads
__device__ __forceinline__ void mean_loss(const float *losses, int pairs, float total_pairs, float *loss) {
    __shared__ double red[TPB / 64];
    double v = 0.0;
    for (int i = threadIdx.x; i < pairs; i += TPB) v += (double)losses[i];
    v = block_sum_f64<TPB / 64>(v, red);
    if (threadIdx.x == 0) *loss = (float)(v / (double)total_pairs);
}
__global__ void __launch_bounds__(TPB) pref_mean_k(const float *__restrict__ losses, int pairs, float total_pairs, float *__restrict__ loss) {
    mean_loss(losses, pairs, total_pairs, loss);
}

// 16-byte chunk blockIdx.x TPB + the thread of row rows - 1 - blockIdx.y.  d may be the logits.  Bound: HBM.  The rows are taken from the last one, and the
// gradient goes past the caches: what the first launch has read last is then still in the memory-side cache, and neither launch waits for
// dirty lines.  8192 x 32000 and 4093 x 50257, whole pass: rows in order 253 / 165 us, gradient through the caches 269 / 199, as it is 219 / 156 (also
// at 1024 x 32000, whose gradient would fit the caches: 43 against 49); two chunks to a thread 226 / 160, four 236 / 165.  Not kept: pairs in groups of
// 64 MiB, each group's gradient in one launch with the sums of the next but one (269 / 196).  Two readings and the writing, at the rates that each
// reaches alone, would take 210.
template <typename T>
__global__ void __launch_bounds__(TPB) pref_grad_k(const T *logits, T *d, int64_t ld, const int32_t *__restrict__ labels, int64_t Vn, int64_t rows,
                                                   const int32_t *__restrict__ offsets, int pairs, const RowStat *__restrict__ stats,
                                                   const float *__restrict__ weight, const float *__restrict__ losses, float total_pairs,
                                                   float *__restrict__ loss) {
    constexpr int V = Vec16<T>::N;
    if (blockIdx.x == 0 && blockIdx.y == 0 && loss) mean_loss(losses, pairs, total_pairs, loss);
    const int64_t row = rows - 1 - blockIdx.y;
    const int nv = (int)Vn, c = blockIdx.x * TPB + threadIdx.x;
    if (c * (int64_t)V >= nv) return;
    const int32_t y = label_of(labels, row, Vn);
    T *const out = d + row * ld + (int64_t)c * V;
    Vec16<T> a;
    float f[V];
    if (y < 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = 0.f;
    } else {
        a.load(logits + row * ld + (int64_t)c * V);
        const RowStat st = stats[row];
        int s = 0, past = 2 * pairs;                                     // the row's sequence: offsets[s] <= row < offsets[past]
        while (past - s > 1) {
            const int mid = (s + past) >> 1;
            if (offsets[mid] <= row) s = mid;
            else past = mid;
        }
        const float w = s & 1 ? -weight[s >> 1] : weight[s >> 1];
        a.get(f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = -w * __builtin_amdgcn_exp2f(fmaf(f[j], L2E, -st.top) - st.log2_sum);
        const int in = y - c * V;
        if (in >= 0 && in < V) {
#pragma unroll
            for (int j = 0; j < V; ++j) if (j == in) f[j] += w;
        }
        if (c * V + V > nv) {
#pragma unroll
            for (int j = 0; j < V; ++j) if (c * V + j >= nv) f[j] = 0.f;
        }
    }
    a.set(f);
    __builtin_nontemporal_store(__builtin_bit_cast(tio_u32x4, a.raw), reinterpret_cast<tio_u32x4 *>(out));
}

template <typename T> void launch(hipStream_t s, const PreferenceArgs &a) {
    double *const logp = (double *)a.work;
    RowStat *const stats = (RowStat *)(logp + a.rows);
    float *const weight = (float *)(stats + a.rows);
    const int64_t nchunk = (a.V + Vec16<T>::N - 1) / Vec16<T>::N;
    if (a.rows) {
#define TIO_ROWS(NCH, NT) pref_rows_k<T, NCH, NT><<<(unsigned)a.rows, NT, 0, s>>>((const T *)a.logits, a.ld, a.labels, a.V, logp, stats)
        if (nchunk <= TPB) TIO_ROWS(1, TPB);
        else if (nchunk <= 4 * TPB) TIO_ROWS(4, TPB);
        else TIO_ROWS(4, 512);
#undef TIO_ROWS
    }
    const float total = (float)a.total_pairs;
    pref_pairs_k<<<(unsigned)a.pairs, PAIR_THREADS, 0, s>>>(a.offsets, (int)a.rows, logp, a.ref, a.beta, a.smoothing, total, a.seq, a.losses, weight);
    if (!a.dlogits || !a.rows) {
        pref_mean_k<<<1, TPB, 0, s>>>(a.losses, (int)a.pairs, total, a.loss);
        return;
    }
    // a grid has at most 2^16 - 1 rows of workgroups, and fewer than 2^32 threads
    const int64_t segments = (nchunk + TPB - 1) / TPB, most = ((int64_t)1 << 23) / segments, at_once = most < 65535 ? most : 65535;
    for (int64_t rows = a.rows; rows > 0; rows -= at_once) {
        const dim3 grid((unsigned)segments, (unsigned)(rows < at_once ? rows : at_once));
        pref_grad_k<T><<<grid, TPB, 0, s>>>((const T *)a.logits, (T *)a.dlogits, a.ld, a.labels, a.V, rows, a.offsets, (int)a.pairs, stats, weight, a.losses,
                                            total, rows == a.rows ? a.loss : nullptr);
    }
}

}  // namespace

int64_t preference_work(int64_t rows, int64_t pairs) { return (rows * (int64_t)(sizeof(double) + sizeof(RowStat)) + pairs * 4 + 15) / 16 * 16; }

void preference_loss(hipStream_t s, int dtype, const PreferenceArgs &a) {
    if (dtype == TIO_PREC_BF16) launch<bf16_t>(s, a);
    else launch<float>(s, a);
}

}  // namespace k
}  // namespace tio
