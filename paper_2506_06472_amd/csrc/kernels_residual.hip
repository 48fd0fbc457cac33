// What stands between two blocks of a decoder layer, in one pass over its rows:
//   n = N_post(branch), or branch;   u = dropout(n);   y = rs x + bs gate u;   h = N(y)
// with N the root-mean-square norm, v / sqrt(mean(v^2) + eps) gain, or the layer norm, (v - mean) / sqrt(mean((v - mean)^2) + eps) gain + bias, and
// its backward pass, from D = dy + N^T(dh):
//   dx = rs D,  dgate = bs u D,  dn = bs gate mask D,  dbranch = N_post^T(dn),
//   N^T(g) = rstd (g gain - vh mean(g gain vh) [- mean(g gain)]),  vh = (v - mean) rstd,  dgain = sum of g vh and dbias = sum of g over the rows.
//
// Both passes have, of every element, only what varies from row to row: with s the mask's factor and bh the branch (normalised, with a norm behind it),
// the branch's part of y is kept ? bh w + c : 0, where w = bs s gate post_gain and c = bs s gate post_bias are a column's (a gate for every row is one
// factor more); and with m = kept ? D : 0 the gradients of gate, post_gain and post_bias are a column's factors of the same two sums over the rows,
//   S1 = sum of m bh,  S2 = sum of m:   dpost_gain = bs s gate S1,  dpost_bias = bs s gate S2,  dgate = bs s (post_gain S1 + post_bias S2).
//
// The backward pass needs y.  From x (from_x) it makes it again in 32 bits, as the forward pass had it when it took its norm: x has as many bytes as y, and the branch and the
// mask are there anyway.  From y as it was rounded, which is all that is left where y took x's place, vh is off by the rounding, and in bf16 dgain by 2.4e-3 of its norm
// where its own rounding is 1.7e-3.
//
// Bound: HBM; the vector ALU, with about 14 (forward) and 24 operations on an element beside the generator's, is not far behind (8192 x 4096 in bf16: forward
// 52 us, 5.2 TB/s; backward 65, 6.2, partly from the memory-side cache, and the sums 6).  A row is W
// wavefronts', who hold it in registers from its loads to its stores; statistics and sums are in 32 bits, the layer norm's variance from centred values.  A
// workgroup takes rows one after the other and keeps its share of the column sums in registers; a second launch adds the workgroups' shares in their
// order, so that results do not depend on timing.
#include <algorithm>

#include "../../include/teraio.h"
#include "device_common.h"
#include "kernels.h"
#include "philox.h"
#include "rows8.h"

namespace tio {
namespace k {

namespace {

template <int CTRL> __device__ __forceinline__ float dpp_add(float v) {
    return v + __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// the sum over a wavefront, in all lanes, without a trip through LDS
__device__ __forceinline__ float wave_total(float v) {
    v = dpp_add<0xB1>(v);                                      // lanes 1 0 3 2
    v = dpp_add<0x4E>(v);                                      // lanes 2 3 0 1
    v = dpp_add<0x141>(v);                                     // eight lanes mirrored
    v = dpp_add<0x140>(v);                                     // sixteen lanes mirrored
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Sums over a row's W wavefronts, in all of their threads.  `red`: LDS of 4 W floats, halves used in turn (one barrier a sum).  AT_ONCE: wavefronts' sums that a thread
// reads at a time, a register each.
template <int W, int AT_ONCE = W> struct RowSum {
    float *red;
    int turn = 0;
    __device__ __forceinline__ explicit RowSum(float *r) : red(r) {}
    __device__ __forceinline__ void operator()(float &u) {
        u = wave_total(u);
        if (W == 1) return;
        float *const at = half();
        if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = u;
        __syncthreads();
        u = at[0];
#pragma unroll AT_ONCE
        for (int w = 1; w < W; ++w) u += at[w];
    }
    __device__ __forceinline__ void operator()(float &u, float &v) {
        u = wave_total(u);
        v = wave_total(v);
        if (W == 1) return;
        float2 *const at = reinterpret_cast<float2 *>(half());
        if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = make_float2(u, v);
        __syncthreads();
        u = at[0].x;
        v = at[0].y;
#pragma unroll 1                                               // sixteen at once would be 32 registers
        for (int w = 1; w < W; ++w) {
            u += at[w].x;
            v += at[w].y;
        }
    }
private:
    __device__ __forceinline__ float *half() {
        float *const at = red + turn * 2 * W;
        turn ^= 1;
        return at;
    }
};

// A thread's eight columns of a row that W wavefronts share, and what stays the same for all rows.  Rows are read and written through descriptors of
// their columns rounded up to 8, so that threads without columns need no branches.
template <typename T, int W, bool RMS, bool POST> struct Columns {
    uint32_t lane, col, bytes;                                 // thread of the row, its first column, bytes of a row
    int n;                                                     // columns that are there
    bool ragged;                                               // the last eight are not whole
    float w[8], c[8], gain[8];                                 // c: of the layer norm behind the block
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t row(const void *base, int64_t at) const { return buffer_over((const T *)base + at, bytes); }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t row_or_none(const void *base, int64_t at) const { return buffer_over((const T *)base + at, base ? bytes : 0); }
    __device__ __forceinline__ void get(float (&f)[8], const Row8<T> &v) const {
        v.get(f);
        if (ragged) cut8(f, n);
    }
    // of a vector, which ends with the last column
    __device__ __forceinline__ void load(float (&f)[8], const void *base) const {
        const T *const from = (const T *)base + col;
        if (n == 8) {
            Row8<T> v;
            v.load(from);
            v.get(f);
            return;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = 0.f;
#pragma unroll
        for (int j = 0; j < 7; ++j)
            if (j < n) f[j] = to_f32(from[j]);
    }
    __device__ __forceinline__ void put(void *base, int64_t at, float (&f)[8]) const {
        if (ragged) cut8(f, n);
        Row8<T> v;
        v.set(f);
        row_put(v, row(base, at), col);
    }
    __device__ __forceinline__ Columns(const ResidualArgs &a)
        : lane(W == 1 ? threadIdx.x & 63 : threadIdx.x), col(lane * 8), bytes((uint32_t)((a.d + 7) / 8 * 8 * sizeof(T))), ragged(a.d % 8 != 0) {
        const int left = (int)a.d - (int)col;
        n = left < 0 ? 0 : left < 8 ? left : 8;
    }
    __device__ __forceinline__ void load_vectors(const ResidualArgs &a) {
        load(gain, a.gain);
        const float factor = a.branch_scale * (a.drop.limit ? a.drop.scale : 1.f);
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            w[j] = j < n ? factor : 0.f;
            c[j] = 0.f;
        }
        if (a.gate && !a.ldg) {
            load(f, a.gate);
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] *= f[j];
        }
        if (POST && !RMS && a.post_bias) {
            load(f, a.post_bias);
#pragma unroll
            for (int j = 0; j < 8; ++j) c[j] = w[j] * f[j];
        }
        if (POST) {
            load(f, a.post_gain);
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] *= f[j];
        }
    }
};

// 1 / sqrt(t) from the hardware's, which is off by one unit in the last place and has no subnormal arguments
__device__ __forceinline__ float inverse_root(float t) {
    const bool tiny = t < 0x1p-100f;
    return __builtin_amdgcn_rsqf(tiny ? t * 0x1p100f : t) * (tiny ? 0x1p50f : 1.f);
}
// mean and 1 / sqrt(variance + eps) of a row
template <bool RMS, int W> __device__ __forceinline__ void stats_of(const float (&v)[8], int n, float inv_d, float eps, RowSum<W> &sum, float &mean, float &rstd) {
    float t = 0.f;
    mean = 0.f;
    if (!RMS) {
#pragma unroll
        for (int j = 0; j < 8; ++j) t += v[j];
        sum(t);
        mean = t * inv_d;
        t = 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float e = RMS ? v[j] : j < n ? v[j] - mean : 0.f;
        t += e * e;
    }
    sum(t);
    rstd = inverse_root(t * inv_d + eps);
}

constexpr int teams_of(int W) { return W == 1 ? 4 : 1; }       // rows that a workgroup has at a time

template <typename T, int W, bool RMS, bool POST>
__global__ void __launch_bounds__(W == 1 ? 256 : W * 64) residual_norm_k(ResidualArgs a) {
    __shared__ float red[4 * W];
    RowSum<W> sum(red);
    Columns<T, W, RMS, POST> col(a);
    const void *const gate = a.ldg ? a.gate : nullptr;
    const uint32_t groups = (uint32_t)((a.d + 7) / 8);
    const float inv_d = 1.0f / (float)a.d;
    col.load_vectors(a);
    float bias[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (!RMS && a.bias) col.load(bias, a.bias);
    const int team = W == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const int64_t stride = (int64_t)gridDim.x * teams_of(W);
    int64_t row = (int64_t)blockIdx.x * teams_of(W) + team;
    Row8<T> next[3];
    auto fetch = [&](int64_t at) __attribute__((always_inline)) {
        if (at >= a.rows) at = a.rows - 1;
        row_load(next[0], col.row(a.branch, at * a.ld), col.col);
        row_load(next[1], col.row(a.x, at * a.ld), col.col);
        row_load(next[2], col.row_or_none(gate, at * a.ldg), col.col);
    };
    fetch(row);
    for (; row < a.rows; row += stride) {
        const Row8<T> raw[3] = {next[0], next[1], next[2]};
        fetch(row + stride);
        Mask8 m;
        if (a.drop.limit) m.draw(row, groups, col.lane, a.drop);
        float v[8], r[8], g[8], mean = 0.f, rstd = 1.f;
        col.get(v, raw[0]);
        if (POST) {
            stats_of<RMS, W>(v, col.n, inv_d, a.eps, sum, mean, rstd);
            if (col.lane == 0) *reinterpret_cast<float2 *>(a.stats + row * 4) = make_float2(mean, rstd);
        }
        col.get(r, raw[1]);
        if (gate) col.get(g, raw[2]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float t = POST ? (v[j] - mean) * rstd * col.w[j] : v[j] * col.w[j];
            if (POST && !RMS) t += col.c[j];
            if (gate) t *= g[j];
            if (a.drop.limit) t = m.kept(j, a.drop) ? t : 0.f;
            v[j] = a.resid_scale * r[j] + t;
        }
        cut8(v, col.n);                                        // where no columns are, a mean or 1 / sqrt that is large or no number left more than zeros
        col.put(a.y, row * a.ld, v);
        stats_of<RMS, W>(v, col.n, inv_d, a.eps, sum, mean, rstd);
        if (col.lane == 0) *reinterpret_cast<float2 *>(a.stats + row * 4 + 2) = make_float2(mean, rstd);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (v[j] - mean) * rstd * col.gain[j] + bias[j];
        col.put(a.h, row * a.ld, v);
    }
}

// The column sums of a workgroup's rows: [kind][workgroup][columns rounded up to 8], kinds dgain, S1, dbias, S2.
constexpr int KINDS = 4;
// FROM_X: a.y is the forward pass's x.  About eight operations more on an element (with the sums, bf16: 8192 x 4096 with both norms 71 us, from y 72; 2000 x 5120, whose sixteen
// wavefronts meet for every row, 37, from y 32): its sums are read five at a time there, as all sixteen would be more registers than there are.
template <typename T, int W, bool RMS, bool POST, bool FROM_X> __device__ __forceinline__ void residual_backward(const ResidualArgs &a) {
    __shared__ float red[4 * W];
    RowSum<W, FROM_X && W == 16 ? 5 : W> sum(red);
    Columns<T, W, RMS, POST> col(a);
    const void *const gate = a.ldg ? a.gate : nullptr;
    const uint32_t groups = (uint32_t)((a.d + 7) / 8);
    const float inv_d = 1.0f / (float)a.d;
    const bool sum1 = POST || (a.gate && !a.ldg);
    float s_gain[8], s_bias[8], s1[8], s2[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) s_gain[j] = s_bias[j] = s1[j] = s2[j] = 0.f;
    const int team = W == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const int64_t stride = (int64_t)gridDim.x * teams_of(W);
    int64_t row = (int64_t)blockIdx.x * teams_of(W) + team;
    // The next row's loads are under way while a row is computed, so that they do not wait behind its stores (8192 x 4096: 75 -> 70 us, with half the
    // workgroups, and so half the sums; forward 62 -> 51), where a thread has registers for them: four wavefronts to a SIMD count for more (layer norm, bf16,
    // 1000 x 4096, both passes: 50 us ahead, 45 so).
    constexpr bool AHEAD = sizeof(T) == 2 && (RMS || !POST);
    Row8<T> next[5];
    float4 next_st;                                            // branch's mean and 1 / sqrt, y's
    auto fetch_first = [&](int64_t at) __attribute__((always_inline)) {
        row_load(next[0], col.row(a.y, at * a.ld), col.col);
        row_load(next[1], col.row(a.dh, at * a.ld), col.col);
        next_st = *reinterpret_cast<const float4 *>(a.stats + at * 4);
    };
    auto fetch_others = [&](int64_t at) __attribute__((always_inline)) {
        row_load(next[2], col.row(a.dy, at * a.ld), col.col);
        row_load(next[3], col.row(a.branch, at * a.ld), col.col);
        row_load(next[4], col.row_or_none(gate, at * a.ldg), col.col);
    };
    auto fetch = [&](int64_t at) __attribute__((always_inline)) {
        if (at >= a.rows) at = a.rows - 1;
        fetch_first(at);
        fetch_others(at);
    };
    if (AHEAD) fetch(row);
    __builtin_amdgcn_sched_barrier(0);
    col.load_vectors(a);                                       // with the first row's loads under way (1021 x 6656 25.1 -> 23.3 us)
    // with a gate for every row, what the layer norm's bias adds to its gradient: a thread's own, in LDS for want of registers
    constexpr bool MOVED = POST && !RMS;
    constexpr int THREADS = W == 1 ? 256 : W * 64;
    __shared__ float4 moved[MOVED ? 2 : 1][MOVED ? THREADS : 1];
    if (MOVED) {
        moved[0][threadIdx.x] = make_float4(col.c[0], col.c[1], col.c[2], col.c[3]);
        moved[MOVED][threadIdx.x] = make_float4(col.c[4], col.c[5], col.c[6], col.c[7]);
    }
    for (; row < a.rows; row += stride) {
        if (!AHEAD) fetch_first(row);
        Row8<T> raw[5] = {next[0], next[1], next[2], next[3], next[4]};
        const float4 st = next_st;
        const int64_t at = row * a.ld;
        if (AHEAD) fetch(row + stride);
        Mask8 m;
        if (a.drop.limit) m.draw(row, groups, col.lane, a.drop);
        float r[8], g[8], D[8], v[8], t = 0.f, u = 0.f;
        if constexpr (!FROM_X) col.get(r, raw[0]);
        else {                                                 // y as the forward pass had it: from x, before its rounding
            if (!AHEAD) {                                      // once more below, from the caches
                row_load(raw[3], col.row(a.branch, at), col.col);
                row_load(raw[4], col.row_or_none(gate, row * a.ldg), col.col);
            }
            raw[0].get(r);
            raw[3].get(v);
            raw[4].get(g);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float n = POST ? (v[j] - (RMS ? 0.f : st.x)) * st.y * col.w[j] : v[j] * col.w[j];
                if (MOVED) n += reinterpret_cast<const float *>(&moved[j >> 2 & MOVED][threadIdx.x])[j & 3];
                if (gate) n *= g[j];
                if (a.drop.limit) n = m.kept(j, a.drop) ? n : 0.f;
                r[j] = a.resid_scale * r[j] + n;
                asm volatile("" : "+v"(r[j]));                 // one element after the other: there are no registers for all at once,
                __builtin_amdgcn_sched_barrier(0);
            }
            raw[3].forget();                                   // and none to keep what is found again below
            m.forget();
            cut8(r, col.n);
        }
        col.get(g, raw[1]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            r[j] = RMS ? r[j] * st.w : j < col.n ? (r[j] - st.z) * st.w : 0.f;
            s_gain[j] += g[j] * r[j];
            if (!RMS) s_bias[j] += g[j];
            g[j] *= col.gain[j];
            t += g[j] * r[j];
            if (!RMS) u += g[j];
        }
        if (RMS) sum(t);
        else sum(t, u);
        const float c1 = t * inv_d, c2 = RMS ? 0.f : u * inv_d;
        t = u = 0.f;
        if (!AHEAD) {
            fetch_others(row);
            raw[2] = next[2];
            raw[3] = next[3];
            raw[4] = next[4];
        }
        col.get(D, raw[2]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            D[j] += (g[j] - r[j] * c1 - c2) * st.w;
            r[j] = a.resid_scale * D[j];
        }
        col.put(a.dx, at, r);
        col.get(v, raw[3]);
        const bool finite = POST && st.y > 0.f && st.y < __builtin_inff();          // else what is dropped is not a number, perhaps
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (POST) v[j] = RMS ? v[j] * st.y : j < col.n ? (v[j] - st.x) * st.y : 0.f;
            if (a.drop.limit) {
                const bool kept = m.kept(j, a.drop);
                D[j] = kept ? D[j] : 0.f;
                v[j] = kept || finite ? v[j] : 0.f;
            }
        }
        if (gate) {
            col.get(g, raw[4]);
            float4 c[2];
            if (MOVED) {
                c[0] = moved[0][threadIdx.x];
                c[1] = moved[MOVED][threadIdx.x];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                r[j] = D[j] * (v[j] * col.w[j] + (MOVED ? reinterpret_cast<const float *>(&c[j >> 2])[j & 3] : 0.f));
                D[j] *= g[j];
            }
            col.put(a.dgate, row * a.ldg, r);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (sum1) {
                const float q = D[j] * v[j];
                s1[j] += q;
                if (POST) t += q * col.w[j];
            }
            if (POST && !RMS) s2[j] += D[j];
            g[j] = D[j] * col.w[j];
            if (POST && !RMS) u += g[j];
        }
        if (POST) {
            if (RMS) sum(t);
            else sum(t, u);
            const float p1 = t * inv_d, p2 = RMS ? 0.f : u * inv_d;
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = (g[j] - v[j] * p1 - p2) * st.y;
        }
        col.put(a.dbranch, at, g);
    }
    const int64_t d8 = (int64_t)groups * 8;
    __shared__ float rows_of[W == 1 ? 4 : 1][W == 1 ? 512 : 1];
    auto out = [&](int kind, const float (&f)[8]) __attribute__((always_inline)) {
        float *const to = (float *)a.work + ((int64_t)kind * gridDim.x + blockIdx.x) * d8;
        if constexpr (W == 1) {                                // the four rows' sums in their order
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) rows_of[team][col.col + j] = f[j];
            __syncthreads();
            for (int i = threadIdx.x; i < d8; i += 256) to[i] = rows_of[0][i] + rows_of[1][i] + rows_of[2][i] + rows_of[3][i];
        } else if (col.n) {
            *reinterpret_cast<float4 *>(to + col.col) = make_float4(f[0], f[1], f[2], f[3]);
            *reinterpret_cast<float4 *>(to + col.col + 4) = make_float4(f[4], f[5], f[6], f[7]);
        }
    };
    out(0, s_gain);
    if (sum1) out(1, s1);
    if (!RMS) out(2, s_bias);
    if (POST && !RMS) out(3, s2);
}
template <typename T, int W, bool RMS, bool POST> __global__ void __launch_bounds__(W == 1 ? 256 : W * 64, 4) residual_norm_bwd_k(ResidualArgs a) {
    residual_backward<T, W, RMS, POST, false>(a);
}
template <typename T, int W, bool RMS, bool POST> __global__ void __launch_bounds__(W == 1 ? 256 : W * 64, 4) residual_norm_bwd_x_k(ResidualArgs a) {
    residual_backward<T, W, RMS, POST, true>(a);
}

// A workgroup adds 16 columns, four wavefronts a kind: the workgroups' shares in their order within each of 64 slices, the slices in theirs.  Neighbouring
// workgroups, whose columns are in the same 128-byte lines, are on one XCD (8192 x 4096: 8.3 -> 5.8 us).
template <typename T> __global__ void __launch_bounds__(256 * KINDS) residual_sums_k(ResidualArgs a, int64_t parts) {
    __shared__ float4 part[KINDS][64][4];
    __shared__ float sums[KINDS][16];
    const int kind = threadIdx.x >> 8, q = threadIdx.x & 3, slice = threadIdx.x >> 2 & 63;
    const int64_t d8 = (a.d + 7) / 8 * 8, first = ((int64_t)(blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8) * 16, col = first + q * 4;
    const bool post = a.post_gain, shared = a.gate && !a.ldg;
    const bool there_is = kind == 0 || (kind == 1 ? post || shared : !a.rms && (kind == 2 || post));
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (there_is && col < d8) {
        const float *from = (const float *)a.work + kind * parts * d8 + col;
#pragma unroll 8
        for (int64_t p = slice; p < parts; p += 64) {
            const float4 t = *reinterpret_cast<const float4 *>(from + p * d8);
            v.x += t.x; v.y += t.y; v.z += t.z; v.w += t.w;
        }
    }
    part[kind][slice][q] = v;
    __syncthreads();
    if ((threadIdx.x & 255) < 16) {
        float t = 0.f;
#pragma unroll 16
        for (int i = 0; i < 64; ++i) t += reinterpret_cast<const float *>(part[kind][i])[threadIdx.x & 15];
        sums[kind][threadIdx.x & 15] = t;
    }
    __syncthreads();
    const int64_t at = first + threadIdx.x;
    if (threadIdx.x >= 16 || at >= a.d) return;
    const float factor = a.branch_scale * (a.drop.limit ? a.drop.scale : 1.f);
    auto value = [&](const void *p) __attribute__((always_inline)) { return p ? to_f32(((const T *)p)[at]) : 0.f; };
    auto out = [&](void *p, float f) __attribute__((always_inline)) {
        if (p) ((T *)p)[at] = from_f32<T>(f);
    };
    out(a.dgain, sums[0][threadIdx.x]);
    if (!a.rms) out(a.dbias, sums[2][threadIdx.x]);
    const float g = factor * (shared ? value(a.gate) : 1.f), one = sums[1][threadIdx.x], two = a.rms || !post ? 0.f : sums[3][threadIdx.x];
    if (post) out(a.dpost_gain, g * one);
    if (post && !a.rms) out(a.dpost_bias, g * two);
    if (shared) out(a.dgate, factor * (post ? value(a.post_gain) * one + (a.post_bias ? value(a.post_bias) * two : 0.f) : one));
}

// wavefronts of a row, and the workgroups that take the rows: what the compute units hold at a time
int row_waves(int64_t d) { return d <= 512 ? 1 : d <= 1024 ? 2 : d <= 2048 ? 4 : d <= 4096 ? 8 : 16; }
int64_t groups_of(int64_t rows, int64_t d, int waves, int64_t most) {
    const int W = row_waves(d), teams = teams_of(W);
    return std::min(std::min((rows + teams - 1) / teams, most), (int64_t)256 * std::max(1, waves / (W * teams)));
}
int64_t forward_groups(int64_t rows, int64_t d) { return groups_of(rows, d, 24, 4096); }
int64_t backward_groups(int64_t rows, int64_t d) { return groups_of(rows, d, 16, 1024); }

}  // namespace

int64_t residual_norm_bwd_work(int64_t rows, int64_t d) { return KINDS * backward_groups(rows, d) * ((d + 7) / 8 * 8) * 4; }

#define TIO_BY_NORM(KERNEL, W)                                                                                                      \
    do {                                                                                                                            \
        const unsigned block = W == 1 ? 256 : W * 64;                                      \
        if (dtype == TIO_PREC_BF16) {                                                                                               \
            if (a.rms && a.post_gain) KERNEL<bf16_t, W, true, true><<<grid, block, 0, s>>>(a);                                      \
            else if (a.rms) KERNEL<bf16_t, W, true, false><<<grid, block, 0, s>>>(a);                                               \
            else if (a.post_gain) KERNEL<bf16_t, W, false, true><<<grid, block, 0, s>>>(a);                                         \
            else KERNEL<bf16_t, W, false, false><<<grid, block, 0, s>>>(a);                                                         \
        } else {                                                                                                                    \
            if (a.rms && a.post_gain) KERNEL<float, W, true, true><<<grid, block, 0, s>>>(a);                                       \
            else if (a.rms) KERNEL<float, W, true, false><<<grid, block, 0, s>>>(a);                                                \
            else if (a.post_gain) KERNEL<float, W, false, true><<<grid, block, 0, s>>>(a);                                          \
            else KERNEL<float, W, false, false><<<grid, block, 0, s>>>(a);                                                          \
        }                                                                                                                           \
    } while (0)
#define TIO_BY_WIDTH(KERNEL)                  \
    do {                                      \
        switch (row_waves(a.d)) {             \
        case 1: TIO_BY_NORM(KERNEL, 1); break;  \
        case 2: TIO_BY_NORM(KERNEL, 2); break;  \
        case 4: TIO_BY_NORM(KERNEL, 4); break;  \
        case 8: TIO_BY_NORM(KERNEL, 8); break;  \
        default: TIO_BY_NORM(KERNEL, 16); break; \
        }                                     \
    } while (0)

void residual_norm(hipStream_t s, int dtype, const ResidualArgs &a) {
    const unsigned grid = (unsigned)forward_groups(a.rows, a.d);
    TIO_BY_WIDTH(residual_norm_k);
}

void residual_norm_bwd(hipStream_t s, int dtype, const ResidualArgs &a) {
    const unsigned grid = (unsigned)backward_groups(a.rows, a.d), columns = (unsigned)((a.d + 127) / 128 * 8);
    if (a.from_x) TIO_BY_WIDTH(residual_norm_bwd_x_k);
    else TIO_BY_WIDTH(residual_norm_bwd_k);
    if (dtype == TIO_PREC_BF16) residual_sums_k<bf16_t><<<columns, 256 * KINDS, 0, s>>>(a, grid);
    else residual_sums_k<float><<<columns, 256 * KINDS, 0, s>>>(a, grid);
}

}  // namespace k
}  // namespace tio
