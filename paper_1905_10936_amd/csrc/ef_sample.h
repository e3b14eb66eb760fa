// Drawing tokens from rows of logits: temperature, top-k, top-p, min-p, and a given random number a row.
//
// The order of a row's entries is by value, downwards, then by place.  Every filter keeps a beginning of that order, so what is kept is told by a
// key (the value as an ordered whole number) and how many of the entries at that key stay, the first ones by place.  Both are found a byte of the
// key at a time from a histogram: of numbers of entries for top-k, of probability for top-p.
//
// Probabilities are 2^((v - top) log2(e) / T) in 64 bits, rounded to multiples of a power of two so large that sums of a whole row are exact (SampleRow::grid): they
// come out the same in whatever order they are added, and by LDS atomics too.  In fp32 a draw next to a border would go by the order of the sums.
#pragma once
#include "ef_rows.h"

namespace ef {

struct SampleArgs {
    int64_t rows, vocab;
    const void *logits;
    int64_t stride;
    const float *uniform, *temperature;
    const int *top_k;
    const float *top_p, *min_p;
    int64_t *tokens;
    float *logp;
};

constexpr int SAMPLE_THREADS = 1024, SAMPLE_WAVES = SAMPLE_THREADS / 64;

// 2^x for x <= 0 in 64 bits, to 1e-11 of it; 0 below 2^-60.
__device__ __forceinline__ double power_of_two(double x)
{
    const double r = __builtin_rint(x), f = (x - r) * 0.69314718055994530942;
    double p = 1.0 / 3628800.0;
    p = __builtin_fma(p, f, 1.0 / 362880.0);
    p = __builtin_fma(p, f, 1.0 / 40320.0);
    p = __builtin_fma(p, f, 1.0 / 5040.0);
    p = __builtin_fma(p, f, 1.0 / 720.0);
    p = __builtin_fma(p, f, 1.0 / 120.0);
    p = __builtin_fma(p, f, 1.0 / 24.0);
    p = __builtin_fma(p, f, 1.0 / 6.0);
    p = __builtin_fma(p, f, 0.5);
    p = __builtin_fma(p, f, 1.0);
    p = __builtin_fma(p, f, 1.0);
    return x >= -60.0 ? __builtin_amdgcn_ldexp(p, (int)r) : 0.0;
}

// A value as a whole number of the same order; -0 is 0.
__device__ __forceinline__ unsigned key_of(float v)
{
    const unsigned b = __float_as_uint(v + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

template <class V>
__device__ __forceinline__ V from_lane(V v, int lane);
template <>
__device__ __forceinline__ unsigned from_lane(unsigned v, int lane) { return (unsigned)__builtin_amdgcn_ds_bpermute(lane * 4, (int)v); }
template <>
__device__ __forceinline__ double from_lane(double v, int lane)
{
    const uint64_t b = (uint64_t)__double_as_longlong(v);
    return __longlong_as_double((long long)((uint64_t)from_lane((unsigned)b, lane) | (uint64_t)from_lane((unsigned)(b >> 32), lane) << 32));
}
// Sum over the lanes up to this one.
template <class V>
__device__ __forceinline__ V upto_lane(V v, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const V other = from_lane(v, lane - d < 0 ? lane : lane - d);
        if (lane >= d) v += other;
    }
    return v;
}

struct SampleShared {
    double mass[256], wave_mass[SAMPLE_WAVES];
    unsigned count[256], wave_count[SAMPLE_WAVES];
    float wave_top[SAMPLE_WAVES];
    unsigned key, bad;
    unsigned rank, ties;        // of what top-k or top-p look for: entries of it to keep, entries there are
    double above;
    int64_t place;
};

// Sums over the workgroup; every thread gets the result.
__device__ __forceinline__ double over_workgroup(double v, double *at)
{
    const int lane = threadIdx.x % 64;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += from_lane(v, lane ^ d);
    __syncthreads();
    if (lane == 0) at[threadIdx.x / 64] = v;
    __syncthreads();
    double s = 0.0;
    for (int i = 0; i < SAMPLE_WAVES; ++i) s += at[i];
    return s;
}

// One row.  Wavefront w has the elements from w * span on, in eights, 512 at a time, so that places ascend with the wavefront, the round and the lane.
template <class T>
struct SampleRow {
    const T *l;
    int64_t vocab, span;
    float top;
    double factor, grid;        // log2(e) / T; what makes (w + grid) - grid a multiple of a power of two

    __device__ __forceinline__ double weight(float v) const { return power_of_two(((double)v - (double)top) * factor); }
    __device__ __forceinline__ double mass(float v) const { return (weight(v) + grid) - grid; }
    // f(values, place of the first, how many there are) for every eight of the calling wavefront
    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
        const int64_t begin = (int64_t)(threadIdx.x / 64) * span, end = min(vocab, begin + span);
        for (int64_t i = begin; i < end; i += 512) {
            const int64_t at = i + threadIdx.x % 64 * 8;
            Eight<T> e;
            load_some(e, l + at, end - at, sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u);
            f(e, at, (int)max((int64_t)0, min((int64_t)8, end - at)));
        }
    }
};

template <class T>
__global__ __launch_bounds__(SAMPLE_THREADS) void k_sample(SampleArgs a)
{
    __shared__ SampleShared s;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t row = blockIdx.x;
    const float u = a.uniform[row], heat = a.temperature ? a.temperature[row] : 1.0f;
    const float top_p = a.top_p ? a.top_p[row] : 1.0f, min_p = a.min_p ? a.min_p[row] : 0.0f;
    const int64_t top_k = a.top_k ? a.top_k[row] : 0;
    SampleRow<T> r;
    r.l = static_cast<const T *>(a.logits) + row * a.stride;
    r.vocab = a.vocab;
    r.span = ((a.vocab + SAMPLE_WAVES - 1) / SAMPLE_WAVES + 511) / 512 * 512;

    // ---- the largest value; what is no distribution
    if (threadIdx.x == 0) s.bad = 0;
    float top = -INFINITY;
    bool bad = false;
    r.each([&](const Eight<T> &e, int64_t, int n) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            top = fmaxf(top, e[k]);
            bad = bad || e[k] != e[k];
        }
    });
    top = over_lanes<Max, 64>(top);
    __syncthreads();
    if (lane == 0) s.wave_top[wave] = top;
    if (bad) s.bad = 1;
    __syncthreads();
    for (int i = 0; i < SAMPLE_WAVES; ++i) top = fmaxf(top, s.wave_top[i]);
    // one comparison to each, false for a NaN
    const bool good = !s.bad && top > -INFINITY && top < INFINITY && u >= 0.0f && u < 1.0f && heat >= 0.0f && heat < INFINITY && top_p == top_p &&
                      min_p == min_p;
    if (!good) {
        if (threadIdx.x == 0) {
            a.tokens[row] = -1;
            if (a.logp) a.logp[row] = NAN;
        }
        return;
    }
    r.top = top;
    const unsigned top_key = key_of(top);
    // The sum of the row's masses stays below 2^52 times their grid.
    r.grid = __builtin_amdgcn_ldexp(1.5, 64 - __builtin_clzll((unsigned long long)a.vocab));
    const bool greedy = heat == 0.0f || top_p <= 0.0f;
    r.factor = 1.4426950408889634074;
    double whole = 0.0;         // at temperature 1
    if (a.logp) {
        r.each([&](const Eight<T> &e, int64_t, int) {
#pragma unroll
            for (int k = 0; k < 8; ++k) whole += r.weight(e[k]);
        });
        whole = over_workgroup(whole, s.wave_mass);
    }
    r.factor = greedy ? 0.0 : 1.4426950408889634074 / (double)heat;

    // ---- what is kept: keys above `key`, and the first `rank` entries at it
    unsigned key = 0, rank = 0xffffffffu, ties = 0xffffffffu;
    constexpr int BYTES = sizeof(T);        // a bf16 value's key ends in two bytes that its first two tell
    if (greedy) {
        key = top_key;
        rank = 1;
    } else if (top_k > 0 && top_k < a.vocab) {
        unsigned left = (unsigned)top_k, prefix = 0;
        for (int b = 3; b >= 4 - BYTES; --b) {
            const unsigned mask = b == 3 ? 0u : 0xffffffffu << 8 * (b + 1);
            __syncthreads();
            if (threadIdx.x < 256) s.count[threadIdx.x] = 0;
            __syncthreads();
            r.each([&](const Eight<T> &e, int64_t, int n) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const unsigned q = key_of(e[k]);
                    if (k < n && (q & mask) == prefix) atomicAdd(&s.count[q >> 8 * b & 255], 1u);
                }
            });
            __syncthreads();
            if (threadIdx.x == 0) {
                int i = 255;
                unsigned more = left;
                for (; s.count[i] < more; --i) more -= s.count[i];
                s.key = prefix | (unsigned)i << 8 * b;
                s.rank = more;
                s.ties = s.count[i];
            }
            __syncthreads();
            prefix = s.key;
            left = s.rank;
        }
        key = sizeof(T) == 2 && !(prefix & 0x80000000u) ? prefix | 0xffffu : prefix;
        rank = left;
        ties = s.ties;
    }
    if (!greedy && top_p < 1.0f) {
        double total = 0.0;
        r.each([&](const Eight<T> &e, int64_t, int) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (key_of(e[k]) > key) total += r.mass(e[k]);
        });
        total = over_workgroup(total, s.wave_mass);
        if (rank != 0xffffffffu) total += r.mass(value_of(key)) * (double)rank;
        const double target = (double)top_p * total;
        double above = 0.0;
        unsigned prefix = 0;
        for (int b = 3; b >= 4 - BYTES; --b) {
            const unsigned mask = b == 3 ? 0u : 0xffffffffu << 8 * (b + 1);
            __syncthreads();
            if (threadIdx.x < 256) {
                s.mass[threadIdx.x] = 0.0;
                s.count[threadIdx.x] = 0;
            }
            __syncthreads();
            r.each([&](const Eight<T> &e, int64_t, int n) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const unsigned q = key_of(e[k]);
                    if (k < n && q >= key && (q & mask) == prefix) {
                        unsafeAtomicAdd(&s.mass[q >> 8 * b & 255], r.mass(e[k]));
                        atomicAdd(&s.count[q >> 8 * b & 255], 1u);
                    }
                }
            });
            __syncthreads();
            if (threadIdx.x == 0) {
                // the first group that brings the mass to the target; it has mass of its own
                int i = 255, found = -1;
                double sum = above;
                for (; i >= 0; --i) {
                    if (s.mass[i] > 0.0) {
                        found = i;
                        s.above = sum;
                        if (sum + s.mass[i] >= target) break;
                        sum += s.mass[i];
                    }
                }
                s.key = prefix | (unsigned)found << 8 * b;
                s.ties = s.count[found];
            }
            __syncthreads();
            prefix = s.key;
            above = s.above;
        }
        const unsigned found = sizeof(T) == 2 && !(prefix & 0x80000000u) ? prefix | 0xffffu : prefix;
        const unsigned most = found == key && rank != 0xffffffffu ? rank : s.ties;
        // entries at the key while the mass before them is below the target
        const double w = r.mass(value_of(found));
        double j = __builtin_floor((target - above) / w);
        j = fmin(fmax(j, 0.0), (double)most);
        while (j < (double)most && above + j * w < target) j += 1.0;
        while (j > 1.0 && above + (j - 1.0) * w >= target) j -= 1.0;
        key = found;
        rank = (unsigned)fmax(j, 1.0);
        ties = s.ties;
    }

    // ---- where the last of the entries at the key stands
    int64_t last = a.vocab;
    if (rank < ties) {
        unsigned mine = 0;
        r.each([&](const Eight<T> &e, int64_t, int n) {
#pragma unroll
            for (int k = 0; k < 8; ++k) mine += k < n && key_of(e[k]) == key;
        });
        const unsigned sum = upto_lane(mine, lane);
        __syncthreads();
        if (lane == 63) s.wave_count[wave] = sum;
        __syncthreads();
        unsigned before = 0;
        int in = 0;
        while (in < SAMPLE_WAVES - 1 && before + s.wave_count[in] < rank) before += s.wave_count[in++];
        if (wave == in) {
            r.each([&](const Eight<T> &e, int64_t at, int n) {
                unsigned here = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) here += k < n && key_of(e[k]) == key;
                const unsigned upto = upto_lane(here, lane);
                unsigned c = before + upto - here;
                if (c < rank && before + upto >= rank) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (k < n && key_of(e[k]) == key && ++c == rank) s.place = at + k;
                    }
                }
                before += from_lane(upto, 63);
            });
        }
        __syncthreads();
        last = s.place;
    }

    // ---- the draw: the first entry with more than u of the kept mass up to it
    const double least = fmin((double)min_p, 1.0);
    const auto kept = [&](float v, int64_t at) {
        const unsigned q = key_of(v);
        if (q < key || (q == key && at > last)) return 0.0;
        const double w = r.weight(v);
        return w >= least ? (w + r.grid) - r.grid : 0.0;
    };
    double mine = 0.0;
    r.each([&](const Eight<T> &e, int64_t at, int n) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) mine += kept(e[k], at + k);
    });
    const double upto = upto_lane(mine, lane);
    __syncthreads();
    if (lane == 63) s.wave_mass[wave] = upto;
    __syncthreads();
    double total = 0.0;
    for (int i = 0; i < SAMPLE_WAVES; ++i) total += s.wave_mass[i];
    const double target = (double)u * total;
    double before = 0.0;
    int in = 0;
    while (in < SAMPLE_WAVES - 1 && before + s.wave_mass[in] <= target) before += s.wave_mass[in++];
    if (wave != in) return;
    r.each([&](const Eight<T> &e, int64_t at, int n) {
        double here = 0.0;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < n) here += kept(e[k], at + k);
        const double sum = upto_lane(here, lane);
        double c = before + (sum - here);
        if (c <= target && before + sum > target) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (k >= n) break;
                const double m = kept(e[k], at + k);
                if (c <= target && c + m > target) {
                    a.tokens[row] = at + k;
                    if (a.logp) a.logp[row] = (float)(((double)e[k] - (double)top) - log(whole));
                }
                c += m;
            }
        }
        before += from_lane(sum, 63);
    });
}

}  // namespace ef
