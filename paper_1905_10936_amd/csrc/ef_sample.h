// Drawing tokens from rows of logits: temperature, top-k, top-p, min-p, and a given random number a row.
//
// The order of a row's entries is by value, downwards, then by place.  Every filter keeps a beginning of that order, so what is kept is told by its last
// entry, a value and a place.  Top-k's is found from a histogram of the values, linear in the value and not in its bits (logits are spread over few powers of two: bins of
// bits would have a wavefront's atomics meet in one), and the order within the one bin where the count runs out; top-p's the same way by probability.  A bin with
// too many entries is binned again between its least and largest value; one of a single value is settled by counting places.
//
// Probabilities are 2^((v - top) log2(e) / T) in 64 bits, rounded to multiples of a power of two so large that sums of a whole row are exact (SampleRow::grid): they
// come out the same in whatever order they are added, by LDS atomics too.  In fp32 one draw in 300 over 50000 entries would go by the order of the sums.
// Sums and draws look only at what is kept; a team reads its row once and keeps it in LDS.
#pragma once
#include "ef_rows.h"

namespace ef {

struct SampleArgs {
    int64_t first, rows, vocab;         // of this launch: rows from `first` on
    const void *logits;
    int64_t stride;
    const float *uniform, *temperature;
    const int *top_k;
    const float *top_p, *min_p;
    int64_t *tokens;
    float *logp;
};

// 2^(j / POWERS) for the table that exponentials start from, by its series.
constexpr int POWERS = 512;
__device__ __forceinline__ double power(int j)
{
    const double f = (double)j / POWERS * 0.69314718055994530942;
    double p = 1.0;
#pragma unroll
    for (int k = 16; k >= 1; --k) p = __builtin_fma(p * f, 1.0 / k, 1.0);
    return p;
}

// A value as a whole number of the same order; 0 and -0 are one.
__device__ __forceinline__ unsigned key_of(float v)
{
    const unsigned b = __float_as_uint(v + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// What a lane gets of another one by a row's shift or broadcast; 0 where there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned moved(unsigned v)
{
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved(double v)
{
    const uint64_t b = (uint64_t)__double_as_longlong(v);
    return __longlong_as_double((long long)((uint64_t)moved<CTRL, ROWS>((unsigned)b) | (uint64_t)moved<CTRL, ROWS>((unsigned)(b >> 32)) << 32));
}
// Sum over the lanes up to this one: within rows of 16, then a row's last lane to the rows behind it.
template <class V>
__device__ __forceinline__ V upto_lane(V v)
{
    v += moved<0x111, 0xf>(v);
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);
    v += moved<0x143, 0xc>(v);
    return v;
}
__device__ __forceinline__ unsigned of_last_lane(unsigned v) { return (unsigned)__builtin_amdgcn_readlane((int)v, 63); }
__device__ __forceinline__ double of_last_lane(double v)
{
    const uint64_t b = (uint64_t)__double_as_longlong(v);
    return __longlong_as_double((long long)((uint64_t)of_last_lane((unsigned)b) | (uint64_t)of_last_lane((unsigned)(b >> 32)) << 32));
}

// LANES threads that have a row: a wavefront, or the whole workgroup.
template <int LANES>
struct Team {
    static constexpr int WAVES = LANES / 64, THREADS = LANES < 256 ? 256 : LANES, TEAMS = THREADS / LANES;
    static constexpr int BINS = LANES == 64 ? 512 : 2048, LISTED = LANES == 64 ? 64 : 256;
    struct Shared {
        double bins[BINS], wave_sum[WAVES], sorted_weight[LISTED], above;
        uint64_t list[LISTED], sorted[LISTED];
        int64_t place;
        unsigned long long first;
        unsigned wave_count[WAVES], listed, least, most, bin, key, bad;
        float wave_top[WAVES];
    };
    static __device__ __forceinline__ void sync()
    {
        if constexpr (LANES == 64) {
            // a wavefront's LDS operations are carried out in their order
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        } else {
            __syncthreads();
        }
    }
    // Sum over the team's threads up to this one, and over all of them.
    static __device__ __forceinline__ double upto(double v, double *at, double &all)
    {
        const int lane = threadIdx.x % 64;
        v = upto_lane(v);
        if constexpr (LANES == 64) {
            all = of_last_lane(v);
        } else {
            sync();
            if (lane == 63) at[threadIdx.x / 64] = v;
            sync();
            all = 0.0;
            double before = 0.0;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) {
                if (i == (int)threadIdx.x / 64) before = all;
                all += at[i];
            }
            v += before;
        }
        return v;
    }
};

template <class T>
__device__ __forceinline__ float largest(const Eight<T> &e)
{
    return fmaxf(fmaxf(fmaxf(e[0], e[1]), fmaxf(e[2], e[3])), fmaxf(fmaxf(e[4], e[5]), fmaxf(e[6], e[7])));
}

// A row that a team looks through again and again: in LDS as it lies in memory where HELD elements hold it, else from the caches.  Wavefront w has the elements from
// w * span on, 512 to a round: places ascend with the wavefront, the round and the lane.
template <class T, int LANES, int HELD>
struct SampleRow {
    const T *l;
    T *held;
    int64_t vocab, begin, end;
    static constexpr unsigned NONE = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;        // -inf

    // f(eight, place of its first element) for every eight of the thread: rounds of 64 of them, what lies behind the row's end is -inf
    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
        if constexpr (HELD) {
            for (int i = (int)begin; i < (int)end; i += 512) {
                const int at = i + threadIdx.x % 64 * 8;
                Eight<T> e;
                const u32x4 *p = reinterpret_cast<const u32x4 *>(held + at);
                if constexpr (sizeof(T) == 2) {
                    e.w = p[0];
                } else {
                    e.lo = p[0];
                    e.hi = p[1];
                }
                f(e, (int64_t)at);
            }
        } else {
            from_memory(f);
        }
    }
    template <class F>
    __device__ __forceinline__ void from_memory(F f) const
    {
        constexpr int AHEAD = 4;
        for (int64_t i = begin; i < end; i += AHEAD * 512) {
            Eight<T> e[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int64_t at = i + k * 512 + threadIdx.x % 64 * 8;
                load_some(e[k], l + at, end - at, NONE);
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (i + k * 512 < end) f(e[k], i + k * 512 + threadIdx.x % 64 * 8);
        }
    }
    __device__ __forceinline__ SampleRow(const T *row, T *buffer, int64_t n)
    {
        const int64_t span = ((n + LANES / 64 - 1) / (LANES / 64) + 511) / 512 * 512;
        l = row;
        held = buffer;
        vocab = n;
        begin = (int64_t)(threadIdx.x % LANES / 64) * span;
        end = min(n, begin + span);
    }
    // The first time through: to LDS besides.
    template <class F>
    __device__ __forceinline__ void load(F f)
    {
        from_memory([&](const Eight<T> &e, int64_t at) {
            if constexpr (HELD) {
                u32x4 *p = reinterpret_cast<u32x4 *>(held + at);
                if constexpr (sizeof(T) == 2) {
                    p[0] = e.w;
                } else {
                    p[0] = e.lo;
                    p[1] = e.hi;
                }
            }
            f(e, at);
        });
    }
};

template <class T, int LANES, int HELD>
struct Sampler {
    using Of = Team<LANES>;
    typename Of::Shared &s;
    SampleRow<T, LANES, HELD> row;
    float top;
    double factor, grid;        // log2(e) / T; what makes (w + grid) - grid a multiple of a power of two
    // kept: larger than `least`, or equal to it and at most at `last`
    float least;
    int64_t last;

    const double *powers;

    // 2^x, x = (v - top) log2(e) / T: a table's power for x in steps of 1 / POWERS, what is left of x, at most 1 / 1024, by three terms in fp32 (1e-10 of the
    // whole), the exponent added on.  Below 2^-60 all are that.
    __device__ __forceinline__ double weight(float v) const
    {
        constexpr double STEPS = 1.5 * (double)(1ll << 52) / POWERS;
        const double x = fmax(((double)v - (double)top) * factor, -60.0), steps = x + STEPS;
        const int k = (int)(unsigned)(uint64_t)__double_as_longlong(steps);
        const float f = (float)(x - (steps - STEPS));
        const float e = f * __builtin_fmaf(f, __builtin_fmaf(f, 0.0555041087f, 0.240226507f), 0.693147181f);
        const double from = powers[k & (POWERS - 1)], p = __builtin_fma(from, (double)e, from);
        return __longlong_as_double((long long)((uint64_t)__double_as_longlong(p) + ((uint64_t)(int64_t)(k >> 9) << 52)));
    }
    __device__ __forceinline__ double mass(float v) const { return (weight(v) + grid) - grid; }
    // f(value, place, weight_of(value)) of everything kept; the weights of eight first, without a branch
    template <class W, class F>
    __device__ __forceinline__ void each_kept(W weight_of, F f) const
    {
        row.each([&](const Eight<T> &e, int64_t at) {
            if (largest(e) >= least) {
                double w[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) w[k] = weight_of(e[k]);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (e[k] > least || (e[k] == least && at + k <= last)) f(e[k], at + k, w[k]);
            }
        });
    }
    // f(value, place) of everything kept
    template <class F>
    __device__ __forceinline__ void each_kept(F f) const
    {
        row.each([&](const Eight<T> &e, int64_t at) {
            if (largest(e) >= least) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (e[k] > least || (e[k] == least && at + k <= last)) f(e[k], at + k);
            }
        });
    }
    static __device__ __forceinline__ int bin_of(float v, double origin, double scale)
    {
        return (int)fmin((origin - (double)v) * scale, (double)(Of::BINS - 1));
    }
    __device__ __forceinline__ void clear_bins()
    {
        Of::sync();
#pragma unroll
        for (int k = 0; k < Of::BINS / LANES; ++k) s.bins[threadIdx.x % LANES + k * LANES] = 0.0;
        if (threadIdx.x % LANES == 0) {
            s.listed = s.most = 0;
            s.least = 0xffffffffu;
        }
        Of::sync();
    }
    // The bin in which the sums from the first one on reach the target, which `target_of` makes of the sum of all of them: s.bin, and in s.above `above` with
    // all bins before it.  Returns false where the target is not below that sum, unless it is known to be reached.
    template <class F>
    __device__ __forceinline__ bool find_bin(double above, F target_of, double &target, bool reached = false)
    {
        constexpr int PER = Of::BINS / LANES;
        Of::sync();
        const int first = threadIdx.x % LANES * PER;
        double own[PER], sum = 0.0, all;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            own[k] = s.bins[first + k];
            sum += own[k];
        }
        double before = Of::upto(sum, s.wave_sum, all) - sum + above;
        target = target_of(all);
        if (!reached && target >= all) return false;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (before < target && before + own[k] >= target) {
                s.bin = first + k;
                s.above = before;
            }
            before += own[k];
        }
        Of::sync();
        return true;
    }

    // Keeps, of what is kept, the beginning whose weights reach a target: all entries before which there is less.
    template <class W, class F>
    __device__ __forceinline__ void cut(double range, W weight_of, F target_of)
    {
        double origin = top, scale = Of::BINS / range, above = 0.0, target = 0.0;
        float low = least, high = top;
        for (int level = 0;; ++level) {
            clear_bins();
            each_kept(weight_of, [&](float v, int64_t, double w) {
                if (v >= low && v <= high) unsafeAtomicAdd(&s.bins[bin_of(v, origin, scale)], w);
            });
            // from the second level on it is a bin that reaches the target which is taken apart
            if (!find_bin(above, [&](double all) { return level == 0 ? target_of(all) : target; }, target, level > 0)) return;
            above = s.above;
            const int bin = (int)s.bin;
            each_kept([&](float v, int64_t at) {
                if (v >= low && v <= high && bin_of(v, origin, scale) == bin) {
                    const unsigned key = key_of(v);
                    const unsigned long long here = __ballot(1);
                    const int lane = threadIdx.x % 64, leader = __builtin_ctzll(here);
                    unsigned n = 0;
                    if (lane == leader) n = atomicAdd(&s.listed, (unsigned)__builtin_popcountll(here));
                    n = (unsigned)__builtin_amdgcn_readlane((int)n, leader) + (unsigned)__builtin_popcountll(here & ((1ull << lane) - 1));
                    if (n < Of::LISTED) s.list[n] = (uint64_t)~key << 32 | (uint64_t)(unsigned)at;
                    atomicMin(&s.least, key);
                    atomicMax(&s.most, key);
                }
            });
            Of::sync();
            const unsigned listed = s.listed, lo = s.least, hi = s.most;
            if (listed <= Of::LISTED) {
                in_list((int)listed, above, target, weight_of);
                return;
            }
            low = value_of(lo);
            high = value_of(hi);
            if (lo == hi) {
                in_places(low, listed, above, target, weight_of(low));
                return;
            }
            origin = high;
            scale = Of::BINS / ((double)high - (double)low);
        }
    }

    // The cut within the listed entries: each finds its rank among them, and the sum of weights up to it.
    template <class W>
    __device__ __forceinline__ void in_list(int n, double above, double target, W weight_of)
    {
        const int i = threadIdx.x % LANES;
        if (i < n) {
            const uint64_t mine = s.list[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += s.list[j] < mine;
            s.sorted[rank] = mine;
            s.sorted_weight[rank] = weight_of(value_of(~(unsigned)(mine >> 32)));
        }
        Of::sync();
        const double w = i < n ? s.sorted_weight[i] : 0.0;
        double all;
        const double sum = above + Of::upto(w, s.wave_sum, all), before = sum - w;
        // the last one before which there is less than the target; the first of the bin is one
        if (i < n && before < target && (i == n - 1 || sum >= target)) {
            s.key = ~(unsigned)(s.sorted[i] >> 32);
            s.place = (int64_t)(unsigned)s.sorted[i];
        }
        Of::sync();
        least = value_of(s.key);
        last = s.place;
    }

    // The first entry of the order alone.
    __device__ __forceinline__ void first_alone()
    {
        least = top;
        int64_t place = INT64_MAX;
        each_kept([&](float, int64_t at) { place = place < at ? place : at; });
        if (threadIdx.x % LANES == 0) s.first = ~0ull;
        Of::sync();
        if (place != INT64_MAX) atomicMin(&s.first, (unsigned long long)place);
        Of::sync();
        last = (int64_t)s.first;
    }

    // The cut among `n` entries of one value, each of weight w.
    __device__ __forceinline__ void in_places(float value, unsigned n, double above, double target, double w)
    {
        double j = __builtin_floor((target - above) / w);
        j = fmin(fmax(j, 0.0), (double)n);
        while (j < (double)n && above + j * w < target) j += 1.0;
        while (j > 1.0 && above + (j - 1.0) * w >= target) j -= 1.0;
        const unsigned rank = (unsigned)fmax(j, 1.0);
        const int lane = threadIdx.x % 64, wave = threadIdx.x % LANES / 64;
        const float was_least = least;
        const int64_t was_last = last;
        // those already cut off stand behind all that are kept
        const auto there = [&](const Eight<T> &e, int64_t at, int k) { return e[k] == value && (value > was_least || at + k <= was_last); };
        unsigned mine = 0;
        row.each([&](const Eight<T> &e, int64_t at) {
#pragma unroll
            for (int k = 0; k < 8; ++k) mine += there(e, at, k);
        });
        const unsigned sum = upto_lane(mine);
        Of::sync();
        if (lane == 63) s.wave_count[wave] = sum;
        Of::sync();
        unsigned before = 0;
        int in = 0;
        while (in < Of::WAVES - 1 && before + s.wave_count[in] < rank) before += s.wave_count[in++];
        if (wave == in) {
            row.each([&](const Eight<T> &e, int64_t at) {
                unsigned here = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) here += there(e, at, k);
                const unsigned upto = upto_lane(here);
                unsigned c = before + upto - here;
                if (c < rank && before + upto >= rank) {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (there(e, at, k) && ++c == rank) s.place = at + k;
                }
                before += of_last_lane(upto);
            });
        }
        Of::sync();
        least = value;
        last = s.place;
    }

    // Of few entries all but about those are left out at once: k threads' largest values are k entries, so that what is below the least of them cannot be among
    // the first k.
    __device__ __forceinline__ void leave_out(int64_t k, float mine)
    {
        if (k > LANES / 2) return;
        const double origin = top, scale = Of::BINS / 24.0;
        clear_bins();
        const bool some = mine >= least;
        const int bin = some ? bin_of(mine, origin, scale) : Of::BINS;
        if (some) unsafeAtomicAdd(&s.bins[bin], 1.0);
        double target;
        if (!find_bin(0.0, [&](double) { return (double)k; }, target)) return;
        if (bin <= (int)s.bin) atomicMin(&s.least, key_of(mine));
        Of::sync();
        least = value_of(s.least);
    }
};

template <class T, int LANES, int HELD>
__global__ __launch_bounds__(Team<LANES>::THREADS) void k_sample(SampleArgs a)
{
    using Of = Team<LANES>;
    __shared__ typename Of::Shared shared[Of::TEAMS];
    __shared__ double powers[POWERS];
    for (int i = threadIdx.x; i < POWERS; i += Of::THREADS) powers[i] = power(i);
    __syncthreads();
    const int lane = threadIdx.x % 64, wave = threadIdx.x % LANES / 64;
    const int64_t row = a.first + (int64_t)blockIdx.x * Of::TEAMS + (Of::TEAMS > 1 ? threadIdx.x / LANES : 0);
    if (row >= a.rows) return;          // whole wavefronts, which meet no other
    typename Of::Shared &s = shared[Of::TEAMS > 1 ? threadIdx.x / LANES : 0];
    __shared__ __align__(16) T held[Of::TEAMS][HELD ? HELD : 8];
    Sampler<T, LANES, HELD> r{s, {static_cast<const T *>(a.logits) + row * a.stride, held[Of::TEAMS > 1 ? threadIdx.x / LANES : 0], a.vocab}};
    const float u = a.uniform[row], heat = a.temperature ? a.temperature[row] : 1.0f;
    const float top_p = a.top_p ? a.top_p[row] : 1.0f, min_p = a.min_p ? a.min_p[row] : 0.0f;
    const int64_t top_k = a.top_k ? a.top_k[row] : 0;

    // ---- the largest value; what is no distribution
    float mine = -INFINITY;
    bool bad = false;
    r.row.load([&](const Eight<T> &e, int64_t) {
        mine = fmaxf(mine, largest(e));
#pragma unroll
        for (int k = 0; k < 8; ++k) bad = bad || e[k] != e[k];
    });
    float top = over_lanes<Max, 64>(mine);
    bad = __any(bad);
    if constexpr (LANES > 64) {
        if (lane == 0) s.wave_top[wave] = bad ? NAN : top;
        Of::sync();
#pragma unroll
        for (int i = 0; i < Of::WAVES; ++i) {
            const float t = s.wave_top[i];
            bad = bad || t != t;
            top = fmaxf(top, t);
        }
    }
    // one comparison to each, false for a NaN
    const bool good = !bad && top > -INFINITY && top < INFINITY && u >= 0.0f && u < 1.0f && heat >= 0.0f && heat < INFINITY && top_p == top_p && min_p == min_p;
    if (!good) {
        if (threadIdx.x % LANES == 0) {
            a.tokens[row] = -1;
            if (a.logp) a.logp[row] = NAN;
        }
        return;
    }
    r.top = top;
    r.powers = powers;
    r.least = -3.402823466e38f;
    r.last = INT64_MAX;
    // The sum of the row's masses stays below 2^52 times their grid.
    r.grid = __builtin_amdgcn_ldexp(1.5, 64 - __builtin_clzll((unsigned long long)a.vocab));
    // The policy's own sum, in fp32's exponentials: a term's error is its own, and the sums are in 64 bits.
    double whole = 0.0;
    if (a.logp) {
        r.row.each([&](const Eight<T> &e, int64_t) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = __builtin_amdgcn_exp2f((e[k] - top) * 1.44269504f);
            whole += (double)(((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])));
        });
        double all;
        Of::upto(whole, s.wave_sum, all);
        whole = all;
    }

    // ---- what is kept
    const bool greedy = heat == 0.0f || top_p <= 0.0f;
    r.factor = heat == 0.0f ? 1.0 : 1.4426950408889634074 / (double)heat;
    if (greedy || top_k == 1) {
        r.first_alone();
    } else if (top_k > 0 && top_k < a.vocab) {
        r.leave_out(top_k, mine);
        r.cut(24.0, [](float) { return 1.0; }, [&](double) { return (double)top_k; });
    }
    if (!greedy && top_k != 1 && top_p < 1.0f)
        r.cut(fmin(24.0 * (double)heat, 1e30), [&](float v) { return r.mass(v); }, [&](double all) { return (double)top_p * all; });
    const double floor_p = fmin((double)min_p, 1.0);
    const auto kept_mass = [&](float v) {
        const double w = r.weight(v);
        return w >= floor_p ? (w + r.grid) - r.grid : 0.0;
    };

    // ---- the draw: the first entry with more than u of the kept mass up to it
    double own = 0.0;
    r.each_kept(kept_mass, [&](float, int64_t, double m) { own += m; });
    const double upto = upto_lane(own);
    double total = 0.0, before = 0.0;
    if constexpr (LANES > 64) {
        Of::sync();
        if (lane == 63) s.wave_sum[wave] = upto;
        Of::sync();
#pragma unroll
        for (int i = 0; i < Of::WAVES; ++i) total += s.wave_sum[i];
    } else {
        total = of_last_lane(upto);
    }
    const double target = (double)u * total;
    if constexpr (LANES > 64) {
        int in = 0;
        while (in < Of::WAVES - 1 && before + s.wave_sum[in] <= target) before += s.wave_sum[in++];
        if (wave != in) return;
    }
    r.row.each([&](const Eight<T> &e, int64_t at) {
        if (!__any(largest(e) >= r.least)) return;
        double m[8], here = 0.0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            m[k] = e[k] > r.least || (e[k] == r.least && at + k <= r.last) ? kept_mass(e[k]) : 0.0;
            here += m[k];
        }
        const double sum = upto_lane(here);
        double c = before + (sum - here);
        if (c <= target && before + sum > target) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (c <= target && c + m[k] > target) {
                    a.tokens[row] = at + k;
                    if (a.logp) a.logp[row] = (float)(((double)e[k] - (double)top) - log(whole));
                }
                c += m[k];
            }
        }
        before += of_last_lane(sum);
    });
}

}  // namespace ef
