// Paired preference loss on the logits of a packed batch, and its gradient.
//
// Sequences 2 i and 2 i + 1 are a preferred and a rejected answer.  With x a row of logits and y its label, a counted row adds
// log p = x[y] - log sum exp x to its sequence; z = beta ((sum of the preferred - its reference) - (sum of the rejected - its reference)),
// a pair's loss is -(1 - s) log sigmoid(z) - s log sigmoid(-z) and the loss their mean.  The gradient of a counted row is
// w (onehot(y) - softmax(x)) with w the derivative of the loss by its sequence's sum, the other rows' is zero.
//
// The weight of a row depends on every row of its pair, so the logits are needed twice: a launch over the rows takes maximum, sum and log p of
// each (counted rows only), one over the pairs their sums, losses and weights, one over the logits writes the gradient; in small batches the last does the
// pairs too.  Bound: HBM (8192 x 32000,
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

// of a row: its largest logit, the reference of its exponentials, and the base-2 logarithm of their sum
struct RowStat {
    float top, log2_sum;
};

// the counted row's label, or -1
__device__ __forceinline__ int32_t label_of(const int32_t *labels, int64_t row, int64_t Vn) {
    const int32_t y = labels[row];
    return y >= 0 && y < Vn ? y : -1;
}

// A workgroup to a row, in pieces of NCH 16-byte chunks to a thread, all of a piece's loads on their way together; every thread has a maximum
// and a sum of its own, which meet at the end.  Exponentials are exp2((x - top) log2(e)): the difference first, because the type's lowest value, with which
// tokens are taken out, and its largest are beyond 32 bits times log2(e); the operation more than a fused one costs no time (within 0.6 %).
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
    float top = -INFINITY, s = 0.f;
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
        const float before = top;
        each([&](float x) __attribute__((always_inline)) { top = fmaxf(top, x); });
        const float ref = top == -INFINITY ? 0.f : top;                  // nothing but -inf so far: exponentials 0, not NaN
        s *= __builtin_amdgcn_exp2f((before - ref) * L2E);
        each([&](float x) __attribute__((always_inline)) { s += __builtin_amdgcn_exp2f((x - ref) * L2E); });
    }
    const float M = block_max<NT / 64>(top, red);
    const float tot = block_sum<NT / 64>(top == -INFINITY ? s : s * __builtin_amdgcn_exp2f((top - M) * L2E), red);
    if (threadIdx.x == 0) {
        const float log2_sum = log2f(tot);
        // over the log2(e) that the exponentials were taken with, rounded to 32 bits: by ln 2 a pair's loss is two to four times as far off
        logp[row] = ((double)to_f32(xr[y]) - (double)M) - (double)log2_sum / (double)L2E;
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

// Loss and weight of a pair; weight: the derivative of the mean loss by the sum of the preferred sequence.  32 bits are enough from z on: the functions
// of 64 take a single thread a microsecond each.
struct Pair {
    float loss, weight;
};
__device__ __forceinline__ Pair pair_of(double z, float beta, float s, float total_pairs) {
    const float zf = (float)z, e = expf(-fabsf(zf)), big = 1.0f / (1.0f + e), small = e * big, log_big = -log1pf(e);
    const float up = zf >= 0.f ? big : small, down = zf >= 0.f ? small : big;                          // sigmoid(z), sigmoid(-z)
    const float log_up = zf >= 0.f ? log_big : log_big + zf, log_down = zf >= 0.f ? log_big - zf : log_big;
    return Pair{-(s < 1.f ? (1.0f - s) * log_up : 0.f) - (s > 0.f ? s * log_down : 0.f),              // no 0 times infinity
                -beta * ((1.0f - s) * down - s * up) / total_pairs};
}

// what the launches behind the rows' share
struct Batch {
    const int32_t *offsets;
    int rows, pairs;
    const double *logp;
    const float *ref;
    float beta, smoothing, total_pairs;
    float *seq, *losses, *loss;
    // nothing outside the batch is read, whatever the offsets are
    __device__ __forceinline__ int32_t offset(int i) const { return min(max(offsets[i], 0), rows); }
};
// this thread's share of the sum of log p over rows [a, b), of `step` threads; eight loads on their way
__device__ __forceinline__ double share(const double *logp, int64_t a, int64_t b, int thread, int step) {
    double sum = 0.0;
    for (int64_t r = a + thread; r < b; r += 8 * step) {
        double v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = r + u * step < b ? logp[r + u * step] : 0.0;
#pragma unroll
        for (int u = 0; u < 8; ++u) sum += v[u];
    }
    return sum;
}

// A workgroup to a pair.  The pairs' mean is left to the next launch: a counter that tells the last workgroup cost 6 us, for the caches it has to write
// back first.
constexpr int PAIR_THREADS = 1024;
__global__ void __launch_bounds__(PAIR_THREADS) pref_pairs_k(const Batch b, float *__restrict__ weight) {
    __shared__ double red[2][PAIR_THREADS / 64];
    const int p = (int)blockIdx.x, at[3] = {b.offset(2 * p), b.offset(2 * p + 1), b.offset(2 * p + 2)};
    const double mine[2] = {share(b.logp, at[0], at[1], threadIdx.x, PAIR_THREADS), share(b.logp, at[1], at[2], threadIdx.x, PAIR_THREADS)};
    const double first = block_sum_f64<PAIR_THREADS / 64>(mine[0], red[0]), second = block_sum_f64<PAIR_THREADS / 64>(mine[1], red[1]);
    if (threadIdx.x == 0) {
        const Pair of = pair_of((double)b.beta * ((first - (double)b.ref[2 * p]) - (second - (double)b.ref[2 * p + 1])), b.beta, b.smoothing, b.total_pairs);
        b.seq[2 * p] = (float)first;
        b.seq[2 * p + 1] = (float)second;
        b.losses[p] = of.loss;
        weight[p] = of.weight;
    }
}

// the mean of the pairs' losses, by a workgroup of TPB threads
__device__ __forceinline__ void mean_loss(const Batch &b) {
    __shared__ double red[TPB / 64];
    double v = 0.0;
    for (int i = threadIdx.x; i < b.pairs; i += TPB) v += (double)b.losses[i];
    v = block_sum_f64<TPB / 64>(v, red);
    if (threadIdx.x == 0) *b.loss = (float)(v / (double)b.total_pairs);
}
__global__ void __launch_bounds__(TPB) pref_mean_k(const Batch b) { mean_loss(b); }

// Small batches: all pairs, a wavefront to each, and the mean, by one workgroup of TPB threads; at most FEW pairs.
constexpr int FEW = 8;
__device__ __forceinline__ void all_pairs(const Batch &b) {
    __shared__ float of_pair[FEW];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int p = wave; p < b.pairs; p += TPB / 64) {
        const int at[3] = {b.offset(2 * p), b.offset(2 * p + 1), b.offset(2 * p + 2)};
        double sum[2] = {share(b.logp, at[0], at[1], lane, 64), share(b.logp, at[1], at[2], lane, 64)};
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            sum[0] += __shfl_xor(sum[0], o, 64);
            sum[1] += __shfl_xor(sum[1], o, 64);
        }
        if (lane == 0) {
            const Pair of = pair_of((double)b.beta * ((sum[0] - (double)b.ref[2 * p]) - (sum[1] - (double)b.ref[2 * p + 1])), b.beta, b.smoothing, b.total_pairs);
            b.seq[2 * p] = (float)sum[0];
            b.seq[2 * p + 1] = (float)sum[1];
            b.losses[p] = of_pair[p] = of.loss;
        }
    }
    __syncthreads();
    if (wave == 0) {
        double v = lane < b.pairs ? (double)of_pair[lane] : 0.0;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
        if (lane == 0) *b.loss = (float)(v / (double)b.total_pairs);
    }
}
__global__ void __launch_bounds__(TPB) pref_all_pairs_k(const Batch b) { all_pairs(b); }

// 16-byte chunk blockIdx.x TPB + the thread of row rows - 1 - blockIdx.y.  d may be the logits.  Bound: HBM.  The rows are taken from the last one, and the
// gradient goes past the caches: what the first launch has read last is then still in the memory-side cache, and neither launch waits for
// dirty lines.  8192 x 32000 and 4093 x 50257, whole pass: rows in order 253 / 165 us, gradient through the caches 269 / 199, as it is 219 / 156 (also
// at 1024 x 32000, whose gradient would fit the caches: 43 against 49); two chunks to a thread 226 / 160, four 236 / 165.  Not kept: pairs in groups of
// 64 MiB, each group's gradient in one launch with the sums of the next but one (269 / 196).  Two readings and the writing, at the rates that each
// reaches alone, would take 210.
// The offsets are an argument of their own, for the scalar loads that a pointer within a struct does not get: without them the search for the row's
// sequence costs 20 us.  Weights written out for each row instead gain nothing (210 / 152).
// PAIRS: small batches, without a launch over the pairs: every workgroup sums its own pair, and one behind the rows' (blockIdx.y = rows) does all_pairs.
template <typename T, bool PAIRS>
__global__ void __launch_bounds__(TPB) pref_grad_k(const T *logits, T *d, int64_t ld, const int32_t *__restrict__ labels, int64_t Vn, int64_t rows,
                                                   const int32_t *__restrict__ offsets, const RowStat *__restrict__ stats, const float *__restrict__ weight,
                                                   bool mean, const Batch b) {
    constexpr int V = Vec16<T>::N;
    if (PAIRS && blockIdx.y == rows) {
        if (blockIdx.x == 0) all_pairs(b);
        return;
    }
    if (!PAIRS && mean && blockIdx.x == 0 && blockIdx.y == 0) mean_loss(b);
    const int64_t row = rows - 1 - blockIdx.y;
    const int nv = (int)Vn, c = blockIdx.x * TPB + threadIdx.x;
    const bool inside = c * (int64_t)V < nv;
    if (!PAIRS && !inside) return;
    const int32_t y = label_of(labels, row, Vn);
    T *const out = d + row * ld + (int64_t)c * V;
    Vec16<T> a;
    float f[V];
    if (y < 0) {
        if (PAIRS && !inside) return;
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = 0.f;
    } else {
        if (inside) a.load(logits + row * ld + (int64_t)c * V);
        const RowStat st = stats[row];
        int s = 0, past = 2 * b.pairs;                                   // the row's sequence: offsets[s] <= row < offsets[past]
        while (past - s > 1) {
            const int mid = (s + past) >> 1;
            if (offsets[mid] <= row) s = mid;
            else past = mid;
        }
        float w;
        if constexpr (PAIRS) {
            __shared__ double red[TPB / 64];
            const int p = s >> 1, at[3] = {b.offset(2 * p), b.offset(2 * p + 1), b.offset(2 * p + 2)};
            const double mine = share(b.logp, at[0], at[1], threadIdx.x, TPB) - share(b.logp, at[1], at[2], threadIdx.x, TPB);
            const double z = (double)b.beta * (block_sum_f64<TPB / 64>(mine, red) - ((double)b.ref[2 * p] - (double)b.ref[2 * p + 1]));
            w = pair_of(z, b.beta, b.smoothing, b.total_pairs).weight;
            if (!inside) return;
        } else {
            w = weight[s >> 1];
        }
        if (s & 1) w = -w;
        a.get(f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = -w * __builtin_amdgcn_exp2f(fmaf(f[j] - st.top, L2E, -st.log2_sum));
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
    const Batch b{a.offsets, (int)a.rows, (int)a.pairs, logp, a.ref, a.beta, a.smoothing, (float)a.total_pairs, a.seq, a.losses, a.loss};
    const bool grad = a.dlogits && a.rows;
    const int64_t segments = (nchunk + TPB - 1) / TPB;
    // Without the launch over the pairs where its few microseconds count: few pairs and rows for the one workgroup, for the gradient few readings of log p
    // by the others.  With it and without: 4 sequences of 60 rows, V = 32000, 17.7 -> 15.7 us; 2 of 1000, V = 1000, 15.4 -> 12.8; forward alone, 2 of 2000,
    // 13.7 -> 12.6.  Past the limits: 780 rows x 16 segments 34.6 -> 36.4; 2 sequences of 2000, V = 8000, 37.5 -> 53.1, V = 800, 16.6 -> 20.0; 12
    // pairs of 280 rows 17.3 -> 17.6.
    if (a.pairs <= FEW && a.rows <= 4096) {
        if (!grad) {
            pref_all_pairs_k<<<1, TPB, 0, s>>>(b);
            return;
        }
        if (a.longest_pair <= 2048 && a.rows * segments <= 4096) {
            pref_grad_k<T, true><<<dim3((unsigned)segments, (unsigned)a.rows + 1), TPB, 0, s>>>((const T *)a.logits, (T *)a.dlogits, a.ld, a.labels, a.V, a.rows,
                                                                                               a.offsets, stats, nullptr, false, b);
            return;
        }
    }
    pref_pairs_k<<<(unsigned)a.pairs, PAIR_THREADS, 0, s>>>(b, weight);
    if (!grad) {
        pref_mean_k<<<1, TPB, 0, s>>>(b);
        return;
    }
    // a grid has at most 2^16 - 1 rows of workgroups, and fewer than 2^32 threads
    const int64_t most = ((int64_t)1 << 23) / segments, at_once = most < 65535 ? most : 65535;
    for (int64_t rows = a.rows; rows > 0; rows -= at_once) {
        const dim3 grid((unsigned)segments, (unsigned)(rows < at_once ? rows : at_once));
        pref_grad_k<T, false><<<grid, TPB, 0, s>>>((const T *)a.logits, (T *)a.dlogits, a.ld, a.labels, a.V, rows, a.offsets, stats, weight, rows == a.rows, b);
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
