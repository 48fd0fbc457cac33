// What stands between two blocks of a decoder layer, in one pass over its rows:
//   n = N_post(branch), or branch;   u = dropout(n);   y = rs x + bs gate u;   h = N(y)
// with N the root-mean-square norm, v / sqrt(mean(v^2) + eps) gain, or the layer norm, (v - mean) / sqrt(mean((v - mean)^2) + eps) gain + bias, and
// its backward pass, from D = dy + N^T(dh):
//   dx = rs D,  dgate = bs u D,  dn = bs gate mask D,  dbranch = N_post^T(dn),
//   N^T(g) = rstd (g gain - vh mean(g gain vh) [- mean(g gain)]),  vh = (v - mean) rstd,  dgain = sum of g vh and dbias = sum of g over the rows.
//
// Bound: HBM.  A row is W wavefronts', who hold it in registers from its loads to its stores; statistics and sums are in 32 bits, the layer norm's
// variance from centred values.  A workgroup takes rows one after the other and keeps its share of the column sums in registers; a second launch
// adds the workgroups' shares in their order, so that results do not depend on timing.
#include "../../include/teraio.h"
#include "device_common.h"
#include "kernels.h"
#include "philox.h"
#include "rows8.h"

namespace tio {
namespace k {

namespace {

// Sums of V numbers over a row's wavefronts, in all of their threads.  `red`: LDS of 2 W V floats, halves used in turn (one barrier a sum).
template <int W, int V> struct RowSum {
    float *red;
    int turn = 0;
    __device__ __forceinline__ explicit RowSum(float *r) : red(r) {}
    __device__ __forceinline__ void operator()(float (&v)[V], int n = V) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) v[i] = wave_sum(v[i]);
        if (W == 1) return;
        float *const at = red + turn * W * V;
        turn ^= 1;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < n) at[wave * V + i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) {
                v[i] = at[i];
#pragma unroll
                for (int w = 1; w < W; ++w) v[i] += at[w * V + i];
            }
    }
};

template <typename T> __device__ __forceinline__ void load8(float (&f)[8], const T *p) {
    Row8<T> v;
    v.load(p);
    v.get(f);
}
template <typename T> __device__ __forceinline__ void put8(T *p, float (&f)[8], int n) {
    cut8(f, n);
    Row8<T> v;
    v.set(f);
    v.put(p);
}

// mean and 1 / sqrt(variance + eps) of a row, whose columns past the end are zero
template <bool RMS, int W, int NCH> __device__ __forceinline__ void stats_of(const float (&v)[NCH][8], const int (&n)[NCH], float inv_d, float eps, RowSum<W, 2> &sum,
                                                                             float &mean, float &rstd) {
    float t[2] = {0.f, 0.f};
    mean = 0.f;
    if (!RMS) {
#pragma unroll
        for (int c = 0; c < NCH; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) t[0] += v[c][j];
        sum(t, 1);
        mean = t[0] * inv_d;
        t[0] = 0.f;
    }
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float e = RMS ? v[c][j] : j < n[c] ? v[c][j] - mean : 0.f;
            t[0] += e * e;
        }
    sum(t, 1);
    rstd = 1.0f / sqrtf(t[0] * inv_d + eps);
}

template <typename T, int W, int NCH, bool RMS, bool POST>
__global__ void __launch_bounds__(W == 1 ? 256 : W * 64) residual_norm_k(ResidualArgs a) {
    constexpr int TEAMS = W == 1 ? 4 : 1;
    __shared__ float red[2 * W * 2];
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x, team = W == 1 ? threadIdx.x >> 6 : 0;
    RowSum<W, 2> sum(red);
    const T *const branch = (const T *)a.branch, *const x = (const T *)a.x, *const gate = (const T *)a.gate;
    const T *const post_gain = (const T *)a.post_gain, *const post_bias = (const T *)a.post_bias, *const gain = (const T *)a.gain, *const bias = (const T *)a.bias;
    const uint32_t groups = (uint32_t)((a.d + 7) / 8);
    const float inv_d = 1.0f / (float)a.d;
    int n[NCH];                                                // columns of this thread's chunks that are there
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int64_t left = a.d - (int64_t)(c * W * 64 + lane) * 8;
        n[c] = left < 0 ? 0 : left < 8 ? (int)left : 8;
    }
    for (int64_t row = (int64_t)blockIdx.x * TEAMS + team; row < a.rows; row += (int64_t)gridDim.x * TEAMS) {
        float v[NCH][8], r[NCH][8];
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int64_t at = row * a.ld + (c * W * 64 + lane) * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] = r[c][j] = 0.f;
            if (n[c]) {
                load8(v[c], branch + at);
                load8(r[c], x + at);
                cut8(v[c], n[c]);
                cut8(r[c], n[c]);
            }
        }
        float mean, rstd;
        if (POST) {
            stats_of<RMS, W, NCH>(v, n, inv_d, a.eps, sum, mean, rstd);
            if (lane == 0) *reinterpret_cast<float2 *>(a.stats + row * 4) = make_float2(mean, rstd);
        }
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            if (!n[c]) continue;
            const int at = (c * W * 64 + lane) * 8;
            if (POST) {
                float g[8], b[8];
                load8(g, post_gain + at);
                if (!RMS && post_bias) load8(b, post_bias + at);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] = (v[c][j] - mean) * rstd * g[j] + (!RMS && post_bias ? b[j] : 0.f);
            }
            if (a.drop.limit) {
                Mask8 m;
                m.draw(row, groups, c * W * 64 + lane, a.drop);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] = m.kept(j, a.drop) ? v[c][j] * a.drop.scale : 0.f;
            }
            if (gate) {
                float g[8];
                load8(g, gate + row * a.ldg + at);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[c][j] *= g[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] = a.resid_scale * r[c][j] + a.branch_scale * v[c][j];
            cut8(v[c], n[c]);
            put8((T *)a.y + row * a.ld + at, v[c], n[c]);
        }
        stats_of<RMS, W, NCH>(v, n, inv_d, a.eps, sum, mean, rstd);
        if (lane == 0) *reinterpret_cast<float2 *>(a.stats + row * 4 + 2) = make_float2(mean, rstd);
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            if (!n[c]) continue;
            const int at = (c * W * 64 + lane) * 8;
            float g[8], b[8];
            load8(g, gain + at);
            if (!RMS && bias) load8(b, bias + at);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] = (v[c][j] - mean) * rstd * g[j] + (!RMS && bias ? b[j] : 0.f);
            put8((T *)a.h + row * a.ld + at, v[c], n[c]);
        }
    }
}

// The column sums of a workgroup's rows: [kind][workgroup][columns rounded up to 8], kinds dgain, dbias, dgate, dpost_gain, dpost_bias.
template <typename T, int W, int NCH, bool RMS, bool POST>
__global__ void __launch_bounds__(W == 1 ? 256 : W * 64) residual_norm_bwd_k(ResidualArgs a) {
    constexpr int TEAMS = W == 1 ? 4 : 1;
    __shared__ float red[2 * W * 2];
    const int lane = W == 1 ? threadIdx.x & 63 : threadIdx.x, team = W == 1 ? threadIdx.x >> 6 : 0;
    RowSum<W, 2> sum(red);
    const T *const branch = (const T *)a.branch, *const y = (const T *)a.y, *const gate = (const T *)a.gate, *const dy = (const T *)a.dy, *const dh = (const T *)a.dh;
    const T *const post_gain = (const T *)a.post_gain, *const post_bias = (const T *)a.post_bias, *const gain = (const T *)a.gain;
    const uint32_t groups = (uint32_t)((a.d + 7) / 8);
    const float inv_d = 1.0f / (float)a.d;
    const bool sum_gate = gate && a.ldg == 0;
    int n[NCH];
    float s_gain[NCH][8], s_bias[NCH][8], s_gate[NCH][8], s_pgain[NCH][8], s_pbias[NCH][8];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        const int64_t left = a.d - (int64_t)(c * W * 64 + lane) * 8;
        n[c] = left < 0 ? 0 : left < 8 ? (int)left : 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) s_gain[c][j] = s_bias[c][j] = s_gate[c][j] = s_pgain[c][j] = s_pbias[c][j] = 0.f;
    }
    for (int64_t row = (int64_t)blockIdx.x * TEAMS + team; row < a.rows; row += (int64_t)gridDim.x * TEAMS) {
        const float4 st = *reinterpret_cast<const float4 *>(a.stats + row * 4);      // post mean, post rstd, mean, rstd
        float v[NCH][8], r[NCH][8], g[NCH][8], D[NCH][8];
        float t[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            const int64_t at = row * a.ld + (c * W * 64 + lane) * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[c][j] = r[c][j] = g[c][j] = D[c][j] = 0.f;
            if (n[c]) {
                float w[8];
                load8(v[c], branch + at);
                load8(r[c], y + at);
                load8(g[c], dh + at);
                load8(D[c], dy + at);
                load8(w, gain + (c * W * 64 + lane) * 8);
                cut8(v[c], n[c]);
                cut8(g[c], n[c]);
                cut8(D[c], n[c]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    r[c][j] = j < n[c] ? (r[c][j] - st.z) * st.w : 0.f;
                    s_gain[c][j] += g[c][j] * r[c][j];
                    if (!RMS) s_bias[c][j] += g[c][j];
                    g[c][j] *= j < n[c] ? w[j] : 0.f;
                    t[0] += g[c][j] * r[c][j];
                    t[1] += g[c][j];
                }
            }
        }
        sum(t, RMS ? 1 : 2);
        const float c1 = t[0] * inv_d, c2 = RMS ? 0.f : t[1] * inv_d;
        t[0] = t[1] = 0.f;
#pragma unroll
        for (int c = 0; c < NCH; ++c) {
            if (!n[c]) continue;
            const int at = (c * W * 64 + lane) * 8;
            float w[8], b[8], e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                D[c][j] += (g[c][j] - r[c][j] * c1 - c2) * st.w;
                e[j] = a.resid_scale * D[c][j];
            }
            put8((T *)a.dx + row * a.ld + at, e, n[c]);
            if (POST) {
                load8(w, post_gain + at);
                if (!RMS && post_bias) load8(b, post_bias + at);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[c][j] = j < n[c] ? (v[c][j] - st.x) * st.y : 0.f;
                    e[j] = v[c][j] * w[j] + (!RMS && post_bias ? b[j] : 0.f);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) e[j] = v[c][j];
            }
            float scale[8];                                    // what dropout multiplies by
            Mask8 m;
            if (a.drop.limit) m.draw(row, groups, c * W * 64 + lane, a.drop);
#pragma unroll
            for (int j = 0; j < 8; ++j) scale[j] = !a.drop.limit ? 1.f : m.kept(j, a.drop) ? a.drop.scale : 0.f;
            float q[8];
            if (gate) load8(q, gate + row * a.ldg + at);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float bD = a.branch_scale * D[c][j], u = scale[j] == 0.f ? 0.f : e[j] * scale[j];
                e[j] = bD * u;                                 // the gate's gradient
                g[c][j] = j < n[c] ? bD * scale[j] * (gate ? q[j] : 1.f) : 0.f;        // dn
            }
            if (sum_gate) {
#pragma unroll
                for (int j = 0; j < 8; ++j) s_gate[c][j] += e[j];
            } else if (gate) put8((T *)a.dgate + row * a.ldg + at, e, n[c]);
            if (POST) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    s_pgain[c][j] += g[c][j] * v[c][j];
                    if (!RMS) s_pbias[c][j] += g[c][j];
                    g[c][j] *= j < n[c] ? w[j] : 0.f;
                    t[0] += g[c][j] * v[c][j];
                    t[1] += g[c][j];
                }
            } else put8((T *)a.dbranch + row * a.ld + at, g[c], n[c]);
        }
        if (POST) {
            sum(t, RMS ? 1 : 2);
            const float p1 = t[0] * inv_d, p2 = RMS ? 0.f : t[1] * inv_d;
#pragma unroll
            for (int c = 0; c < NCH; ++c) {
                if (!n[c]) continue;
#pragma unroll
                for (int j = 0; j < 8; ++j) g[c][j] = (g[c][j] - v[c][j] * p1 - p2) * st.y;
                put8((T *)a.dbranch + row * a.ld + (c * W * 64 + lane) * 8, g[c], n[c]);
            }
        }
    }
    const int64_t d8 = (int64_t)groups * 8, teams = (int64_t)gridDim.x * TEAMS, mine = (int64_t)blockIdx.x * TEAMS + team;
    float *const work = (float *)a.work;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
        if (!n[c]) continue;
        const int64_t at = mine * d8 + (c * W * 64 + lane) * 8;
        auto out = [&](int kind, const float (&f)[8]) __attribute__((always_inline)) {
            float *const to = work + kind * teams * d8 + at;
            *reinterpret_cast<float4 *>(to) = make_float4(f[0], f[1], f[2], f[3]);
            *reinterpret_cast<float4 *>(to + 4) = make_float4(f[4], f[5], f[6], f[7]);
        };
        out(0, s_gain[c]);
        if (!RMS) out(1, s_bias[c]);
        if (sum_gate) out(2, s_gate[c]);
        if (POST) out(3, s_pgain[c]);
        if (POST && !RMS) out(4, s_pbias[c]);
    }
}

struct Sums {
    void *out[5];                // nullptr: none of that kind
};
// A workgroup adds 64 columns of one kind: four lanes' width of rows of parts, sixteen of which go on at a time.
template <typename T> __global__ void __launch_bounds__(256) residual_sums_k(const float *__restrict__ work, int64_t parts, int64_t d, Sums s) {
    __shared__ float4 part[16][16];
    const int kind = blockIdx.y, q = threadIdx.x & 15, slice = threadIdx.x >> 4;
    T *const out = (T *)s.out[kind];
    if (!out) return;
    const int64_t d8 = (d + 7) / 8 * 8, col = (int64_t)blockIdx.x * 64 + q * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (col < d8)
        for (int64_t p = slice; p < parts; p += 16) {
            const float4 t = *reinterpret_cast<const float4 *>(work + (kind * parts + p) * d8 + col);
            v.x += t.x; v.y += t.y; v.z += t.z; v.w += t.w;
        }
    part[slice][q] = v;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    const int64_t at = (int64_t)blockIdx.x * 64 + threadIdx.x;
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) t += reinterpret_cast<const float *>(part[i])[threadIdx.x];
    if (at < d8) out[at] = from_f32<T>(at < d ? t : 0.f);
}

constexpr int64_t MAX_GROUPS = 1024;                           // workgroups of the backward pass
// wavefronts of a row, and the workgroups that take them
int row_waves(int64_t d) { return d <= 1024 ? 1 : d <= 4096 ? 4 : d <= 8192 ? 8 : 16; }
int64_t groups_of(int64_t rows, int64_t d) {
    const int64_t teams = row_waves(d) == 1 ? 4 : 1, g = (rows + teams - 1) / teams;
    return g < MAX_GROUPS ? g : MAX_GROUPS;
}
int64_t parts_of(int64_t rows, int64_t d) { return groups_of(rows, d) * (row_waves(d) == 1 ? 4 : 1); }

}  // namespace

int64_t residual_norm_bwd_work(int64_t rows, int64_t d) { return 5 * parts_of(rows, d) * ((d + 7) / 8 * 8) * 4; }

#define TIO_BY_NORM(KERNEL, W, NCH)                                                                                                     \
    do {                                                                                                                                \
        const unsigned grid = (unsigned)groups_of(a.rows, a.d), block = W == 1 ? 256 : W * 64;                                          \
        if (dtype == TIO_PREC_BF16) {                                                                                                   \
            if (a.rms && a.post_gain) KERNEL<bf16_t, W, NCH, true, true><<<grid, block, 0, s>>>(a);                                     \
            else if (a.rms) KERNEL<bf16_t, W, NCH, true, false><<<grid, block, 0, s>>>(a);                                              \
            else if (a.post_gain) KERNEL<bf16_t, W, NCH, false, true><<<grid, block, 0, s>>>(a);                                        \
            else KERNEL<bf16_t, W, NCH, false, false><<<grid, block, 0, s>>>(a);                                                        \
        } else {                                                                                                                        \
            if (a.rms && a.post_gain) KERNEL<float, W, NCH, true, true><<<grid, block, 0, s>>>(a);                                      \
            else if (a.rms) KERNEL<float, W, NCH, true, false><<<grid, block, 0, s>>>(a);                                               \
            else if (a.post_gain) KERNEL<float, W, NCH, false, true><<<grid, block, 0, s>>>(a);                                         \
            else KERNEL<float, W, NCH, false, false><<<grid, block, 0, s>>>(a);                                                         \
        }                                                                                                                               \
    } while (0)
#define TIO_BY_WIDTH(KERNEL)                          \
    do {                                              \
        if (a.d <= 512) TIO_BY_NORM(KERNEL, 1, 1);    \
        else if (a.d <= 1024) TIO_BY_NORM(KERNEL, 1, 2); \
        else if (a.d <= 2048) TIO_BY_NORM(KERNEL, 4, 1); \
        else if (a.d <= 4096) TIO_BY_NORM(KERNEL, 4, 2); \
        else if (a.d <= 8192) TIO_BY_NORM(KERNEL, 8, 2); \
        else TIO_BY_NORM(KERNEL, 16, 2);              \
    } while (0)

void residual_norm(hipStream_t s, int dtype, const ResidualArgs &a) { TIO_BY_WIDTH(residual_norm_k); }

void residual_norm_bwd(hipStream_t s, int dtype, const ResidualArgs &a) {
    TIO_BY_WIDTH(residual_norm_bwd_k);
    const Sums sums{{a.dgain, a.rms ? nullptr : a.dbias, a.gate && a.ldg == 0 ? a.dgate : nullptr, a.post_gain ? a.dpost_gain : nullptr,
                     a.post_gain && !a.rms ? a.dpost_bias : nullptr}};
    const dim3 grid((unsigned)((a.d + 63) / 64), 5);
    const int64_t parts = parts_of(a.rows, a.d);
    if (dtype == TIO_PREC_BF16) residual_sums_k<bf16_t><<<grid, 256, 0, s>>>((const float *)a.work, parts, a.d, sums);
    else residual_sums_k<float><<<grid, 256, 0, s>>>((const float *)a.work, parts, a.d, sums);
}

}  // namespace k
}  // namespace tio
