// The norm of a worker's gradient over its tensors, and the clipped gradient in the worker's flat row (or in place).
//
// Two passes over memory: squares, added up in 64 bits in a fixed order, a workgroup to a chunk; then every workgroup adds up its worker's chunks (CLIP_CHUNKS
// numbers or a few more, from the caches) and scales its own.  A chunk is a range of places of the flat row, whatever tensors lie there: a kernel's arguments hold
// the tensors' addresses and first places, as many as fit them.
#pragma once
#include "ef_rows.h"

namespace ef {

constexpr int CLIP_THREADS = 256, CLIP_CHUNKS = 1024, CLIP_TENSORS = 224, CLIP_LEAST = 8 * CLIP_THREADS;

struct ClipArgs {
    int64_t base, length, chunk;        // the places of the flat rows that this launch covers, and how many of them a chunk has
    int tensors;                        // a worker's, of this launch
    int slot, slots;                    // where its sums begin among a worker's, and how many those are in all
    int worker;                         // the first of this launch; one to a row of the grid
    double *sums;                       // [workers][slots]
    float *flat;                        // null: in place
    int64_t flat_stride;
    float *norm;                        // null: not by this launch
    float max_norm;
    int64_t first[CLIP_TENSORS];        // a tensor's first place, from base on
    uint64_t at[CLIP_TENSORS];          // [workers][tensors] addresses; bit 0: fp32
};
static_assert(sizeof(ClipArgs) <= 4096, "a kernel's arguments");

// f(address, fp32?, first element, elements, place of the first) for each tensor's part of the workgroup's chunk.
template <class F>
__device__ __forceinline__ void each_part(const ClipArgs &a, F f)
{
    const int64_t begin = (int64_t)blockIdx.x * a.chunk, end = min(a.length, begin + a.chunk);
    int lo = 0, hi = a.tensors;         // the last tensor that begins at or before `begin`
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.first[mid] <= begin)
            lo = mid;
        else
            hi = mid;
    }
    for (int64_t at = begin; at < end; ++lo) {
        const int64_t next = min(end, lo + 1 < a.tensors ? a.first[lo + 1] : a.length);
        const uint64_t p = a.at[(int)blockIdx.y * a.tensors + lo];
        f(reinterpret_cast<void *>(p & ~1ull), (p & 1) != 0, at - a.first[lo], next - at, a.base + at);
        at = next;
    }
}

// Sum over the workgroup in a fixed order; every thread gets it.
__device__ __forceinline__ double clip_sum(double v, double *at)
{
#pragma unroll
    for (int d = 32; d >= 1; d /= 2) v += __shfl_xor(v, d);
    if (threadIdx.x % 64 == 0) at[threadIdx.x / 64] = v;
    __syncthreads();
    return (at[0] + at[1]) + (at[2] + at[3]);
}

template <class T>
__device__ __forceinline__ double squares(const T *p, int64_t n)
{
    double s = 0.0;
    for (int64_t i = (int64_t)threadIdx.x * 8; i < n; i += 8 * CLIP_THREADS) {
        Eight<T> e;
        load_some(e, p + i, n - i, 0u);
#pragma unroll
        for (int k = 0; k < 8; ++k) s = __builtin_fma((double)e[k], (double)e[k], s);
    }
    return s;
}

__global__ __launch_bounds__(CLIP_THREADS) void k_clip_norm(ClipArgs a)
{
    __shared__ double at[CLIP_THREADS / 64];
    double s = 0.0;
    each_part(a, [&](void *p, bool wide, int64_t i, int64_t n, int64_t) {
        s += wide ? squares(static_cast<const float *>(p) + i, n) : squares(static_cast<const bf16_t *>(p) + i, n);
    });
    s = clip_sum(s, at);
    if (threadIdx.x == 0) a.sums[(int64_t)(a.worker + (int)blockIdx.y) * a.slots + a.slot + blockIdx.x] = s;
}

// The product in 64 bits: next to a huge norm the factor is beyond fp32 though the products are not.
template <class T, class To>
__device__ __forceinline__ void scaled(const T *p, To *to, int64_t n, double factor)
{
    for (int64_t i = (int64_t)threadIdx.x * 8; i < n; i += 8 * CLIP_THREADS) {
        Eight<T> e;
        load_some(e, p + i, n - i, 0u);
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = (float)((double)e[k] * factor);
        Eight<To> o;
        o.round(v);
        store_some(o, to + i, n - i);
    }
}

__global__ __launch_bounds__(CLIP_THREADS) void k_clip_scale(ClipArgs a)
{
    __shared__ double at[CLIP_THREADS / 64];
    const int worker = a.worker + (int)blockIdx.y;
    const double *sums = a.sums + (int64_t)worker * a.slots;
    double s = 0.0;
    for (int i = threadIdx.x; i < a.slots; i += CLIP_THREADS) s += sums[i];
    const double norm = sqrt(clip_sum(s, at));
    if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) a.norm[worker] = (float)norm;
    // An infinite norm or a NaN clips nothing: the caller sees it in `norm`.
    const double factor = norm > (double)a.max_norm && norm < INFINITY ? (double)a.max_norm / norm : 1.0;
    if (!a.flat && factor == 1.0) return;
    each_part(a, [&](void *p, bool wide, int64_t i, int64_t n, int64_t place) {
        if (a.flat) {
            float *const to = a.flat + (int64_t)worker * a.flat_stride + place;
            if (wide)
                scaled(static_cast<const float *>(p) + i, to, n, factor);
            else
                scaled(static_cast<const bf16_t *>(p) + i, to, n, factor);
        } else if (wide) {
            scaled(static_cast<const float *>(p) + i, static_cast<float *>(p) + i, n, factor);
        } else {
            scaled(static_cast<const bf16_t *>(p) + i, static_cast<bf16_t *>(p) + i, n, factor);
        }
    });
}

}  // namespace ef
