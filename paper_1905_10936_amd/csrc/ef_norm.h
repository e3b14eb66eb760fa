// RMS norm with the residual's addition and an 8-bit output, and its backward pass.
//
// Both are bound by memory.  A row is held in registers by a team of LANES threads, CHUNKS times eight elements each, and read
// once: the sum of squares (forward) or of g * xhat (backward) needs the whole row before the first output can be
// formed.  CHUNKS is as many as the row takes, so that only the last may end inside the row: the others are read without a look at where it
// ends (16384 x 1031 in bf16, forward: 35 us, 44 with a look in every chunk).  Teams of up to 64 lanes meet without a barrier.
// 16384 x 1024 in bf16: forward 30 us, 5.0 TB/s; backward 28, 4.1 TB/s, of which the second launch (k_sum_parts) takes 5.  A copy of 1 GiB
// reaches 5.1.
#pragma once
#include "ef_rows.h"

namespace ef {

struct NormForward {
    int64_t rows, n;
    const void *x, *residual;
    int64_t x_stride, residual_stride;
    const float *weight;
    float eps;
    void *h, *y;
    int64_t h_stride, y_stride;
    ActRef act;                 // codes == nullptr: none is written
    float *rstd;
    int64_t first;              // the launch's first row
};

constexpr float NORM_SMALL = 0x1p-80f;      // a sum of squares below has lost some of them to underflow

constexpr int norm_threads(int lanes) { return lanes < 256 ? 256 : lanes; }

template <class T, int LANES, int CHUNKS>
__global__ __launch_bounds__(norm_threads(LANES)) void k_norm_forward(NormForward a)
{
    constexpr int TEAMS = norm_threads(LANES) / LANES;
    __shared__ float sums[2][LANES > 64 ? LANES / 64 : 1];
    const int lane = threadIdx.x % LANES;
    const int64_t row = a.first + (int64_t)blockIdx.x * TEAMS + threadIdx.x / LANES;
    if (row >= a.rows) return;          // whole teams; LANES > 64: never
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    float v[CHUNKS][8];
    {
        Eight<T> e[CHUNKS];
        times<CHUNKS>([&](auto c) {
            const int64_t i = (c.value * LANES + lane) * 8;
            load_piece<c.value == CHUNKS - 1>(e[c.value], x + i, a.n - i);
        });
        if (a.residual) {
            const T *r = static_cast<const T *>(a.residual) + row * a.residual_stride;
            Eight<T> f[CHUNKS];
            times<CHUNKS>([&](auto c) {
                const int64_t i = (c.value * LANES + lane) * 8;
                load_piece<c.value == CHUNKS - 1>(f[c.value], r + i, a.n - i);
            });
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[c][k] = e[c][k] + f[c][k];
        } else {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[c][k] = e[c][k];
        }
    }
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int k = 0; k < 8; ++k) s = __builtin_fmaf(v[c][k], v[c][k], s);
    s = over_row<Add, LANES>(s, sums[0]);
    const float mean = s / (float)a.n + a.eps;
    // xhat = v * before * rstd; `before` is 1 but for a row whose squares fp32 does not hold (from about 10^19 on, or below 10^-12 where eps does not
    // cover it): they are then taken of v times a power of two, and rstd, which may be out of fp32's range, is kept as two factors that are not.
    float rstd = 1.0f / sqrtf(mean), before = 1.0f;
    if (!(mean < INFINITY) || (s < NORM_SMALL && a.eps < NORM_SMALL)) {
        const bool small = s < NORM_SMALL;
        const float by = small ? 0x1p100f : 0x1p-72f;
        s = 0.0f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float t = v[c][k] * by;
                s = __builtin_fmaf(t, t, s);
            }
        s = over_row<Add, LANES>(s, sums[1]);
        before = small ? 0x1p24f : 0x1p-24f;
        rstd = 1.0f / sqrtf(s / (float)a.n + a.eps * by * by) * (small ? 0x1p76f : 0x1p-48f);
    }
    if (a.rstd && lane == 0) a.rstd[row] = before * rstd;
    if (a.h) {
        T *h = static_cast<T *>(a.h) + row * a.h_stride;
        times<CHUNKS>([&](auto c) {
            const int64_t i = (c.value * LANES + lane) * 8;
            Eight<T> e;
            e.round(v[c.value]);
            store_piece<c.value == CHUNKS - 1>(e, h + i, a.n - i);
        });
    }
    if (before != 1.0f) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int k = 0; k < 8; ++k) v[c][k] *= before;
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[c][k] *= rstd;
    if (a.act.codes) times<CHUNKS>([&](auto c) { a.act.template put<c.value == CHUNKS - 1>(row, (c.value * LANES + lane) * 8, a.n, v[c.value]); });
    if (a.y) {
        T *y = static_cast<T *>(a.y) + row * a.y_stride;
        times<CHUNKS>([&](auto c) {
            const int64_t i = (c.value * LANES + lane) * 8;
            if (a.weight) {
                Eight<float> w;
                load_piece<c.value == CHUNKS - 1>(w, a.weight + i, a.n - i);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[c.value][k] *= w[k];
            }
            Eight<T> e;
            e.round(v[c.value]);
            store_piece<c.value == CHUNKS - 1>(e, y + i, a.n - i);
        });
    }
}

struct NormBackward {
    int64_t rows, n;
    const void *dy, *dh;
    int64_t dy_stride, dh_stride;
    ActRef act;
    const float *rstd, *weight;
    void *dx;
    int64_t dx_stride;
    float *parts;               // [workgroups][n] sums of dy * xhat over each workgroup's rows, or NULL
};

// A team takes rows team, team + teams, ... and keeps its sums of dy * xhat in registers; a workgroup adds its teams' up through shared memory, in their
// order.
template <class T, int LANES, int CHUNKS>
__global__ __launch_bounds__(norm_threads(LANES)) void k_norm_backward(NormBackward a)
{
    constexpr int TEAMS = norm_threads(LANES) / LANES;
    __shared__ float sums[2][LANES > 64 ? LANES / 64 : 1];
    __shared__ float joined[TEAMS > 1 ? TEAMS : 1][TEAMS > 1 ? LANES * CHUNKS * 8 : 1];
    const int lane = threadIdx.x % LANES, team = threadIdx.x / LANES;
    float dw[CHUNKS][8], w[CHUNKS][8];
    times<CHUNKS>([&](auto c) {
        const int64_t i = (c.value * LANES + lane) * 8;
        Eight<float> e;
        if (a.weight)
            load_piece<c.value == CHUNKS - 1>(e, a.weight + i, a.n - i);
        else
            e.fill(0x3f800000u);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            w[c.value][k] = e[k];
            dw[c.value][k] = 0.0f;
        }
    });
    const float per = 1.0f / (float)a.n;
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * TEAMS + team; row < a.rows; row += (int64_t)gridDim.x * TEAMS) {
        const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
        Eight<T> e[CHUNKS], f[CHUNKS];
        float x[CHUNKS][8];
        times<CHUNKS>([&](auto c) {
            const int64_t i = (c.value * LANES + lane) * 8;
            load_piece<c.value == CHUNKS - 1>(e[c.value], dy + i, a.n - i);
            if (a.dh) load_piece<c.value == CHUNKS - 1>(f[c.value], static_cast<const T *>(a.dh) + row * a.dh_stride + i, a.n - i);
            a.act.template get<c.value == CHUNKS - 1>(row, i, x[c.value]);
        });
        const float rstd = a.rstd[row];
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float d = e[c][k];
                dw[c][k] = __builtin_fmaf(d, x[c][k], dw[c][k]);
                s = __builtin_fmaf(d * w[c][k], x[c][k], s);
            }
        s = over_row<Add, LANES>(s, sums[turn & 1]) * per;
        ++turn;
        T *dx = static_cast<T *>(a.dx) + row * a.dx_stride;
        times<CHUNKS>([&](auto c) {
            const int64_t i = (c.value * LANES + lane) * 8;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v[k] = rstd * __builtin_fmaf(-s, x[c.value][k], e[c.value][k] * w[c.value][k]);
                if (a.dh) v[k] += f[c.value][k];
            }
            Eight<T> o;
            o.round(v);
            store_piece<c.value == CHUNKS - 1>(o, dx + i, a.n - i);
        });
    }
    if (!a.parts) return;
    float *part = a.parts + (int64_t)blockIdx.x * a.n;
    if constexpr (TEAMS > 1) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int k = 0; k < 8; ++k) joined[team][(c * 8 + k) * LANES + lane] = dw[c][k];
        __syncthreads();
        for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
            const int at = (i / 8 / LANES * 8 + i % 8) * LANES + i / 8 % LANES;
            float s = joined[0][at];
#pragma unroll
            for (int t = 1; t < TEAMS; ++t) s += joined[t][at];
            part[i] = s;
        }
    } else {
        times<CHUNKS>([&](auto c) {
            const int64_t i = (c.value * LANES + lane) * 8;
            Eight<float> e;
            e.round(dw[c.value]);
            store_piece<c.value == CHUNKS - 1>(e, part + i, a.n - i);
        });
    }
}

// dweight <- [dweight +] the sum of `count` partial rows: 32 columns to a workgroup, whose 32 half wavefronts take every 32nd row, up to sixteen of
// them on their way at once, and add their sums up in order.
__global__ __launch_bounds__(1024) void k_sum_parts(const float *parts, int count, int64_t n, float *dweight, int accumulate)
{
    __shared__ float sums[32][33];
    const int col = threadIdx.x % 32, first = threadIdx.x / 32;
    const int64_t i = (int64_t)blockIdx.x * 32 + col;
    float s = 0.0f;
    if (i < n) {
        for (int p = first; p < count; p += 16 * 32) {
            float v[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = p + k * 32 < count ? parts[(int64_t)(p + k * 32) * n + i] : 0.0f;
#pragma unroll
            for (int k = 0; k < 16; ++k) s += v[k];
        }
    }
    sums[first][col] = s;
    __syncthreads();
    if (first == 0 && i < n) {
        s = 0.0f;
#pragma unroll
        for (int k = 0; k < 32; ++k) s += sums[k][col];
        dweight[i] = accumulate ? dweight[i] + s : s;
    }
}

}  // namespace ef
