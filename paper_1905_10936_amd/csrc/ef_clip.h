// The norm of a worker's gradient over its tensors, and the clipped gradient in the worker's flat row (or in place).
//
// Two passes over memory: squares, added up in 64 bits in a fixed order, a sum to a workgroup; then every workgroup adds up its worker's sums (CLIP_GROUPS at most, from the
// caches) and scales.  Workgroups take chunks of the flat row's places in turn, whatever tensors lie there, so that those that run together
// are at neighbouring addresses (a run of its own to each: 353.8 M elements in bf16 802 us, 618 this way; the two
// passes and the fp32 row written are 2.83 GB, 552 us at a copy's rate).  The tensors' addresses are in
// the kernels' arguments, or, where they are too many, in the workspace, put there by small launches before (seven workers of 161 tensors in launches of their own:
// 518 us, 380 this way).
#pragma once
#include <stddef.h>

#include "ef_rows.h"

namespace ef {

constexpr int CLIP_THREADS = 256, CLIP_GROUPS = 2048, CLIP_WORDS = 480, CLIP_LEAST = 8 * CLIP_THREADS, CLIP_MOST = 8 * CLIP_LEAST;

struct ClipArgs {
    int64_t length, chunk;              // places of a flat row, and how many of them a chunk has (a multiple of CLIP_LEAST)
    int tensors;                        // a worker's
    double *sums;                       // [workers][groups]
    float *flat;                        // null: in place
    int64_t flat_stride;
    float *norm;
    float max_norm;
};
// The tensors as words: their first places, then [workers][tensors] addresses whose bit 0 says fp32; in the kernel's arguments, or in the workspace.
struct ClipDirect {
    ClipArgs a;
    uint64_t words[CLIP_WORDS];
};
struct ClipListed {
    ClipArgs a;
    const uint64_t *words;
};
static_assert(sizeof(ClipDirect) <= 4096, "a kernel's arguments");
struct ClipWords {
    uint64_t *to;
    int n;
    uint64_t words[CLIP_WORDS];
};
__global__ __launch_bounds__(CLIP_WORDS) void k_clip_words(ClipWords a)
{
    if ((int)threadIdx.x < a.n) a.to[threadIdx.x] = a.words[threadIdx.x];
}

// Memory that no kernel writes while this one runs: read by scalar loads.
#define EF_CONSTANT __attribute__((address_space(4)))

// Who goes through a part: the workgroup, or a wavefront.
struct ClipTeam {
    int me, all;
};

// f(address, fp32?, first element, elements, place of the first, who) for each tensor's part of the workgroup's chunks.
template <bool BACKWARDS, class F>
__device__ __forceinline__ void each_part(const ClipArgs &a, const EF_CONSTANT uint64_t *words, F f)
{
    const int64_t chunks = (a.length + a.chunk - 1) / a.chunk;
    for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const int64_t begin = (BACKWARDS ? chunks - 1 - c : c) * a.chunk, end = min(a.length, begin + a.chunk);
        int lo = 0, hi = a.tensors;         // the last tensor that begins at or before `begin`
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if ((int64_t)words[mid] <= begin)
                lo = mid;
            else
                hi = mid;
        }
        lo = __builtin_amdgcn_readfirstlane(lo);
        for (int64_t at = begin, part = 0; at < end; ++lo, ++part) {
            const int64_t first = (int64_t)words[lo], next = min(end, lo + 1 < a.tensors ? (int64_t)words[lo + 1] : a.length);
            const uint64_t p = words[(1 + (int)blockIdx.y) * a.tensors + lo];
            // short parts one behind the other wait for memory each time: every fourth is a wavefront's (two workers of 65 tensors, 272 k
            // elements: 15.2 us, 13.1 this way)
            const int n = (int)(next - at), wave = (int)__builtin_amdgcn_readfirstlane(threadIdx.x / 64);
            if (n > 512)
                f(reinterpret_cast<void *>(p & ~1ull), (p & 1) != 0, at - first, n, at, ClipTeam{(int)threadIdx.x, CLIP_THREADS});
            else if ((int)(part & 3) == wave)
                f(reinterpret_cast<void *>(p & ~1ull), (p & 1) != 0, at - first, n, at, ClipTeam{(int)threadIdx.x % 64, 64});
            at = next;
        }
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

// Memory that is known to be global: the addresses come from the kernel's arguments as numbers, and an access that might be LDS's waits for LDS's too
// (the first pass over 302 M bf16 elements: 185 us that way).
template <class T>
__device__ __forceinline__ float element(const T *p, unsigned i)
{
    if constexpr (sizeof(T) == 2)
        return __uint_as_float((unsigned)((const EF_GLOBAL uint16_t *)p)[i] << 16);
    else
        return ((const EF_GLOBAL float *)p)[i];
}

// A part of n elements (of one chunk) in whole eights from the first 16-byte boundary of `p` on, AHEAD of them under way at a time, and what is left at its ends:
// load(place) and use(place, what it gave) for the eights, one(place) for an element.
template <class E, class P, class Load, class Use, class One>
__device__ __forceinline__ void eights_of_part(const P *p, int n, ClipTeam who, Load load, Use use, One one)
{
    constexpr int AHEAD = 4;
    const int ROUND = 8 * who.all;
    const int head = min(n, (int)((16 - reinterpret_cast<uintptr_t>(p) % 16) % 16 / sizeof(P)));
    const int end = head + (n - head) / 8 * 8;
    for (int r = head + who.me * 8; r < end; r += AHEAD * ROUND) {
        E e[AHEAD];
        // without a branch, beyond the end the last eight again: loads behind branches are waited for one by one
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) e[k] = load((unsigned)min(r + k * ROUND, end - 8));
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (r + k * ROUND < end) use((unsigned)(r + k * ROUND), e[k]);
    }
    if (who.me < head) one((unsigned)who.me);
    if (who.me < n - end) one((unsigned)(end + who.me));
}

template <class T>
__device__ __forceinline__ double squares(const T *p, int n, ClipTeam who)
{
    double s[2] = {0.0, 0.0};
    eights_of_part<Eight<T>>(
        p, n, who,
        [&](unsigned i) {
            Eight<T> e;
            e.load_at(p, i * (unsigned)sizeof(T));
            return e;
        },
        [&](unsigned, const Eight<T> &e) {
#pragma unroll
            for (int k = 0; k < 8; ++k) s[k & 1] = __builtin_fma((double)e[k], (double)e[k], s[k & 1]);
        },
        [&](unsigned i) {
            const double v = element(p, i);
            s[0] = __builtin_fma(v, v, s[0]);
        });
    return s[0] + s[1];
}

// Where the words are: behind the other arguments in the kernel's, or where those say.
template <class Args>
__device__ __forceinline__ const EF_CONSTANT uint64_t *words_of(const Args &args)
{
    if constexpr (std::is_same<Args, ClipDirect>::value)
        return (const EF_CONSTANT uint64_t *)((const EF_CONSTANT char *)__builtin_amdgcn_kernarg_segment_ptr() + offsetof(ClipDirect, words));
    else
        return (const EF_CONSTANT uint64_t *)args.words;
}

template <class Args>
__global__ __launch_bounds__(CLIP_THREADS) void k_clip_norm(Args args)
{
    const ClipArgs a = args.a;
    __shared__ double at[CLIP_THREADS / 64];
    double s = 0.0;
    each_part<false>(a, words_of(args), [&](void *p, bool wide, int64_t i, int n, int64_t, ClipTeam who) {
        s += wide ? squares(static_cast<const float *>(p) + i, n, who) : squares(static_cast<const bf16_t *>(p) + i, n, who);
    });
    s = clip_sum(s, at);
    if (threadIdx.x == 0) a.sums[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = s;
}

// The product in 64 bits: next to a huge norm the factor is beyond fp32 though the products are not.
template <class T, class To>
__device__ __forceinline__ void scaled(const T *p, To *to, int n, ClipTeam who, double factor)
{
    eights_of_part<Eight<T>>(
        to, n, who,
        [&](unsigned i) {
            Eight<T> e;
            e.load_at(p, i * (unsigned)sizeof(T));
            return e;
        },
        [&](unsigned i, const Eight<T> &e) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = (float)((double)e[k] * factor);
            Eight<To> o;
            o.round(v);
            o.store_at(to, i * (unsigned)sizeof(To));
        },
        [&](unsigned i) {
            const float v = (float)((double)element(p, i) * factor);
            if constexpr (sizeof(To) == 2)
                ((EF_GLOBAL uint16_t *)to)[i] = from_float<bf16_t>(v).bits;
            else
                ((EF_GLOBAL float *)to)[i] = v;
        });
}

template <class Args>
__global__ __launch_bounds__(CLIP_THREADS) void k_clip_scale(Args args)
{
    const ClipArgs a = args.a;
    __shared__ double at[CLIP_THREADS / 64];
    const int worker = (int)blockIdx.y;
    const double *sums = a.sums + (int64_t)worker * gridDim.x;
    double s = 0.0;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += CLIP_THREADS) s += sums[i];
    const double norm = sqrt(clip_sum(s, at));
    if (blockIdx.x == 0 && threadIdx.x == 0) a.norm[worker] = (float)norm;
    // An infinite norm or a NaN clips nothing: the caller sees it in `norm`.
    const double factor = norm > (double)a.max_norm && norm < INFINITY ? (double)a.max_norm / norm : 1.0;
    if (!a.flat && factor == 1.0) return;
    // backwards: it begins where the first pass ended, with what the caches still hold
    each_part<true>(a, words_of(args), [&](void *p, bool wide, int64_t i, int n, int64_t place, ClipTeam who) {
        if (a.flat) {
            float *const to = a.flat + (int64_t)worker * a.flat_stride + place;
            if (wide)
                scaled(static_cast<const float *>(p) + i, to, n, who, factor);
            else
                scaled(static_cast<const bf16_t *>(p) + i, to, n, who, factor);
        } else if (wide) {
            scaled(static_cast<const float *>(p) + i, static_cast<float *>(p) + i, n, who, factor);
        } else {
            scaled(static_cast<const bf16_t *>(p) + i, static_cast<bf16_t *>(p) + i, n, who, factor);
        }
    });
}

}  // namespace ef
