// Log-probabilities of tokens, and the clipped policy loss with its gradient, on rows of logits.
//
// The gradient needs the whole row's sum of exponentials before its first element, and loss and gradient of a row depend on that row
// alone, so a team of LANES threads reads the row once, holds it in registers as it lies in memory (CHUNKS times eight elements a
// thread) and writes the gradient from there: 2 bytes an element read and 2 written in bf16, the least there is.  Rows too long for
// that are read twice.
//
// exp(l - m) is 2^(l * L - c) with L = log2(e) rounded and c = m * L rounded, one fused operation and one exponential an element; what
// c was rounded by is put right once a row.
#pragma once
#include "ef_rows.h"

namespace ef {

struct PolicyArgs {
    int64_t rows, vocab;
    const void *logits;
    int64_t stride;
    const int64_t *tokens;
    const float *logp_old, *logp_ref, *advantage, *token_weight;
    float low, high, kl;        // 1 - clip_low, 1 + clip_high
    float *logp, *losses;
    void *dlogits;
    int64_t dlogits_stride;
    int loss;                   // 0: log-probabilities alone
};

constexpr float LOG2E = 1.44269502162933349609375f;     // log2(e) rounded to fp32
constexpr float LN2 = 0.693147182464599609375f;

// Loss of a row and its derivative with respect to logp, times the row's weight.
__device__ __forceinline__ float2 row_loss(const PolicyArgs &a, int64_t row, float q, float logp)
{
    const float adv = a.advantage[row];
    const float r = a.logp_old ? expf(logp - a.logp_old[row]) : 1.0f;
    const float free = r * adv, held = fminf(fmaxf(r, a.low), a.high) * adv;
    float f = -(free <= held ? free : held), c = free <= held ? -free : 0.0f;
    if (!(free == free) || !(held == held)) f = c = free + held;      // NaN
    if (a.logp_ref) {
        const float d = a.logp_ref[row] - logp, m = expm1f(d);
        f += a.kl * (m - d);
        c -= a.kl * m;
    }
    return make_float2(q * f, q * c);
}

struct Exponent {
    float factor, c;
    // Where the largest logit is itself beyond 10^30 in size (a mask of the type's lowest value in every place), m * L would overflow, and any other
    // logit is at least 2^76 away: 2^-20 for L, which multiplies exactly, gives 1 and 0 as e would.
    __device__ __forceinline__ explicit Exponent(float top)
    {
        factor = fabsf(top) > 1e30f ? 0x1p-20f : LOG2E;
        c = top * factor;
    }
    __device__ __forceinline__ float of(float l) const { return __builtin_amdgcn_exp2f(__builtin_fmaf(l, factor, -c)); }
    // log of the row's sum of exponentials less `top`, from the sum of of(l)
    __device__ __forceinline__ float log_sum(float sum, float top) const { return logf(sum) - LN2 * __builtin_fmaf(top, factor, -c); }
};

// What a row's token says about it: its weight, 0 for a masked row.
__device__ __forceinline__ float row_weight(const PolicyArgs &a, int64_t row, int64_t token)
{
    if ((uint64_t)token >= (uint64_t)a.vocab) return 0.0f;
    return a.token_weight ? a.token_weight[row] : 1.0f;
}

constexpr int policy_threads(int lanes) { return lanes < 256 ? 256 : lanes; }

template <class T, int LANES, int CHUNKS>
__global__ __launch_bounds__(policy_threads(LANES)) void k_policy(PolicyArgs a)
{
    constexpr int TEAMS = policy_threads(LANES) / LANES;
    constexpr unsigned NONE = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;       // -inf
    __shared__ float tops[LANES > 64 ? LANES / 64 : 1], sums[LANES > 64 ? LANES / 64 : 1];
    const int lane = threadIdx.x % LANES;
    const int64_t row = (int64_t)blockIdx.x * TEAMS + threadIdx.x / LANES;
    if (row >= a.rows) return;
    const T *l = static_cast<const T *>(a.logits) + row * a.stride;
    T *g = a.dlogits ? static_cast<T *>(a.dlogits) + row * a.dlogits_stride : nullptr;
    const int64_t token = a.tokens[row];
    const float q = row_weight(a, row, token);
    if (q == 0.0f) {
        if (lane == 0) {
            if (a.logp) a.logp[row] = 0.0f;
            if (a.losses) a.losses[row] = 0.0f;
        }
        if (g) {
            Eight<T> zero;
            zero.fill(0u);
            for (int64_t i = (int64_t)lane * 8; i < a.vocab; i += LANES * 8) store_some(zero, g + i, a.vocab - i);
        }
        return;
    }
    Eight<T> e[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int64_t i = (c * LANES + lane) * 8;
        load_some(e[c], l + i, a.vocab - i, NONE);
    }
    // The token's logit goes into the maximum: it is there before the row's first barrier, and the gradient may be written over the row
    // behind it.
    const float chosen = to_float<T>(l[token]);
    float top = chosen;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int k = 0; k < 8; ++k) top = fmaxf(top, e[c][k]);
    top = over_row<Max, LANES>(top, tops);
    const Exponent x(top);
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += x.of(e[c][k]);
    sum = over_row<Add, LANES>(sum, sums);
    const float logp = (chosen - top) - x.log_sum(sum, top);
    float2 f = make_float2(0.0f, 0.0f);
    if (a.loss) f = row_loss(a, row, q, logp);
    if (lane == 0) {
        if (a.logp) a.logp[row] = logp;
        if (a.losses) a.losses[row] = f.x;
    }
    if (!g) return;
    const float p = -f.y / sum;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int64_t i = (c * LANES + lane) * 8;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = x.of(e[c][k]) * p;
        if ((uint64_t)(token - i) < 8u) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (token - i == k) v[k] += f.y;
        }
        Eight<T> o;
        o.round(v);
        store_some(o, g + i, a.vocab - i);
    }
}

// Rows longer than a workgroup's registers: maximum and sum kept up to date chunk by chunk, the row read again for the gradient.
constexpr int LONG_THREADS = 1024;
template <class T>
__global__ __launch_bounds__(LONG_THREADS) void k_policy_long(PolicyArgs a)
{
    constexpr unsigned NONE = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
    __shared__ float tops[LONG_THREADS / 64], sums[LONG_THREADS / 64];
    const int64_t row = blockIdx.x;
    const T *l = static_cast<const T *>(a.logits) + row * a.stride;
    T *g = a.dlogits ? static_cast<T *>(a.dlogits) + row * a.dlogits_stride : nullptr;
    const int64_t token = a.tokens[row];
    const float q = row_weight(a, row, token);
    if (q == 0.0f) {
        if (threadIdx.x == 0) {
            if (a.logp) a.logp[row] = 0.0f;
            if (a.losses) a.losses[row] = 0.0f;
        }
        if (g) {
            Eight<T> zero;
            zero.fill(0u);
            for (int64_t i = (int64_t)threadIdx.x * 8; i < a.vocab; i += LONG_THREADS * 8) store_some(zero, g + i, a.vocab - i);
        }
        return;
    }
    const float chosen = to_float<T>(l[token]);
    // sum of 2^((l - top) * L) so far; a thread that has seen nothing but -inf has top = -inf and sum 0
    float top = -INFINITY, sum = 0.0f;
    for (int64_t i = (int64_t)threadIdx.x * 8; i < a.vocab; i += LONG_THREADS * 8) {
        Eight<T> e;
        load_some(e, l + i, a.vocab - i, NONE);
        float t = top;
#pragma unroll
        for (int k = 0; k < 8; ++k) t = fmaxf(t, e[k]);
        if (t > top) {
            sum *= __builtin_amdgcn_exp2f((top - t) * LOG2E);
            top = t;
        }
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) s += __builtin_amdgcn_exp2f((e[k] - top) * LOG2E);
        if (top != -INFINITY) sum += s;
        else if (s != s) {
            // eight times -inf, or NaN among them: the latter has to show
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (e[k] != e[k]) sum = e[k];
        }
    }
    const float all = over_row<Max, LONG_THREADS>(fmaxf(top, chosen), tops);
    sum = over_row<Add, LONG_THREADS>(sum == 0.0f ? 0.0f : sum * __builtin_amdgcn_exp2f((top - all) * LOG2E), sums);
    if (all == -INFINITY) sum = NAN;        // nothing but -inf
    const float logp = (chosen - all) - logf(sum);
    float2 f = make_float2(0.0f, 0.0f);
    if (a.loss) f = row_loss(a, row, q, logp);
    if (threadIdx.x == 0) {
        if (a.logp) a.logp[row] = logp;
        if (a.losses) a.losses[row] = f.x;
    }
    if (!g) return;
    const float p = -f.y / sum;
    for (int64_t i = (int64_t)threadIdx.x * 8; i < a.vocab; i += LONG_THREADS * 8) {
        Eight<T> e;
        load_some(e, l + i, a.vocab - i, NONE);
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            v[k] = __builtin_amdgcn_exp2f((e[k] - all) * LOG2E) * p;
            if (token - i == k) v[k] += f.y;
        }
        Eight<T> o;
        o.round(v);
        store_some(o, g + i, a.vocab - i);
    }
}

// loss <- the sum of the rows' losses: thread t adds rows t, t + 1024, ..., then a fixed tree.
__global__ __launch_bounds__(1024) void k_sum_losses(const float *losses, int64_t rows, float *loss)
{
    __shared__ double sums[1024];
    double s = 0.0;
    for (int64_t i = threadIdx.x; i < rows; i += 1024) s += (double)losses[i];
    sums[threadIdx.x] = s;
    __syncthreads();
    for (int h = 512; h > 0; h /= 2) {
        if ((int)threadIdx.x < h) sums[threadIdx.x] += sums[threadIdx.x + h];
        __syncthreads();
    }
    if (threadIdx.x == 0) *loss = (float)sums[0];
}

}  // namespace ef
