// Drawing tokens from rows of logits: temperature, top-k, top-p, min-p, and a given random number a row.
//
// The order of a row's entries is by value, downwards, then by place.  Every filter keeps a beginning of that order, so what is kept is told by its last
// entry, a value and a place.  Top-k's is found from a histogram of the values, linear in the value and not in its bits (logits are spread over few powers of two: bins of
// bits would have a wavefront's atomics meet in one), and the order within the one bin where the count runs out; top-p's the same way by probability.  A bin with
// too many entries is binned again between its least and largest value; one of a single value is settled by counting places.
//
// Probabilities are 2^((v - top) log2(e) / T) in 64 bits, rounded to multiples of a power of two so large that sums of a whole row are exact (Sampler::grid): they
// come out the same in whatever order they are added, by LDS atomics too.  In fp32 one draw in 300 over 50000 entries would go by the order of the sums.  That power goes by the row's
// own sum: by the number of its entries, 131071 of e^-24.5 beside one of 1 (3e-6 in all) would each be rounded to none.
// Sums and draws look only at what is kept; a team reads its row once and keeps it in LDS.
//
// A row of any length is bound by its CU's instructions, a pass over 50257 entries by 110 cycles for each of its inner loop: in bf16 on all CUs (256 rows) without logp 9 us greedy, 17
// with top-k 50, 25 with no filter, 44 with top-k 2000, 51 with top-p alone, where the bytes take 5 (logp: 3 more for the first two, else nothing); one row takes 2 to 5 us less.  64 rows of 128256 in
// fp32, top-p: 106.
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
        double bins[BINS], wave_sum[WAVES], sorted_weight[LISTED], above;      // bins of numbers of entries: words in the same place
        uint64_t list[LISTED], sorted[LISTED];
        unsigned wave_count[WAVES], listed, least, most, bin, key, place;
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

    __device__ __forceinline__ float value(unsigned place) const { return to_float<T>(HELD ? held[place] : l[place]); }
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
                f(e, (unsigned)at);
            }
        } else {
            from_memory(f);
        }
    }
    template <class F>
    __device__ __forceinline__ void from_memory(F f) const
    {
        constexpr int AHEAD = HELD || sizeof(T) == 2 ? 4 : 2;       // as many as registers hold
        for (int64_t i = begin; i < end; i += AHEAD * 512) {
            Eight<T> e[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int64_t at = i + k * 512 + threadIdx.x % 64 * 8;
                load_some(e[k], l + at, end - at, NONE);
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
                if (i + k * 512 < end) f(e[k], (unsigned)(i + k * 512) + threadIdx.x % 64 * 8);
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
        from_memory([&](const Eight<T> &e, unsigned at) {
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
    const double *powers;
    float top;
    double factor, grid;        // log2(e) / T; what makes (w + grid) - grid a multiple of a power of two
    // kept: larger than `least`, or equal to it and at most at `last`
    float least;
    unsigned last;

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

    // f(eight values, place of the first) for the eights that hold something kept, -inf in the place of what is not.
    template <class F>
    __device__ __forceinline__ void each_kept(F f) const
    {
        const float above = value_of(key_of(least) + 1);
        row.each([&](const Eight<T> &e, unsigned at) {
            // one comparison to an entry: all of them at most at `last`, or (but for the one eight that has it) behind
            const float from = at + 7 <= last ? least : above;
            float v[8], most = -INFINITY;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v[k] = e[k] >= from ? e[k] : -INFINITY;
                most = fmaxf(most, v[k]);
            }
            if (last - at < 7) {
#pragma unroll
                for (int k = 0; k < 7; ++k)
                    if (at + k <= last && e[k] == least) v[k] = most = e[k];
            }
            if (most > -INFINITY) f(v, at);
        });
    }

    // f(value, place) for the entries whose bits those_of(values, place of the first) sets, of eights with something kept: a lane has few, so it goes through its own, read
    // again, and not through all eight with branches (top-k 2000 of 50257: 5 us more that way).
    template <class M, class F>
    __device__ __forceinline__ void each_of(M those_of, F f) const
    {
        each_kept([&](const float *v, unsigned at) {
            for (unsigned those = those_of(v, at); those; those &= those - 1) {
                const unsigned place = at + (unsigned)__builtin_ctz(those);
                f(row.value(place), place);
            }
        });
    }

    // A bin's number for a value: linear, from 0 for `origin` on, the last for all that is far.  `unit`: a power of two that keeps differences in fp32's range, and with it
    // `origin` finite: next to an origin of 2^20 or more values are a sixteenth or more apart, which at a unit of 1 is beyond any range that asks for 2^100.  So no value up to `origin` has a place
    // below 0; a bin's number is an index in any case.
    struct Scale {
        float unit, origin, factor;
        __device__ __forceinline__ float at(float v) const { return __builtin_fmaf(v, -unit, origin) * factor; }
        __device__ __forceinline__ int bin(float v) const { return (int)__builtin_amdgcn_fmed3f(at(v), 0.0f, (float)(Of::BINS - 1)); }
    };
    static __device__ __forceinline__ Scale scale_of(float origin, double range)
    {
        Scale x;
        x.unit = range > 1e30 || fabsf(origin) > 1e37f ? 0x1p-20f : range < 1e-30 && fabsf(origin) < 0x1p20f ? 0x1p100f : 1.0f;
        x.origin = origin * x.unit;
        x.factor = (float)fmin(Of::BINS / (range * (double)x.unit), 1e30);
        return x;
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
    template <bool COUNT>
    __device__ __forceinline__ void add(int bin, double w)
    {
        if constexpr (COUNT)
            atomicAdd(reinterpret_cast<unsigned *>(s.bins) + bin, 1u);
        else
            unsafeAtomicAdd(&s.bins[bin], w);
    }
    // One entry more in the list, if it has room, and in any case in `listed`.
    __device__ __forceinline__ void list(float v, unsigned place)
    {
        const unsigned long long here = __ballot(1);
        const int lane = threadIdx.x % 64, leader = __builtin_ctzll(here);
        unsigned n = 0;
        if (lane == leader) n = atomicAdd(&s.listed, (unsigned)__builtin_popcountll(here));
        n = (unsigned)__builtin_amdgcn_readlane((int)n, leader) + (unsigned)__builtin_popcountll(here & ((1ull << lane) - 1));
        if (n < Of::LISTED) s.list[n] = (uint64_t)~key_of(v) << 32 | (uint64_t)place;
    }
    // Where entry i of the list stands among its n.
    __device__ __forceinline__ int rank(int i, int n) const
    {
        const uint64_t mine = s.list[i];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) rank += s.list[j] < mine;
        return rank;
    }
    // The bin in which the sums from the first one on reach the target, which `target_of` makes of the sum of all of them: s.bin, and in s.above `above` with
    // all bins before it.  Returns false where the target is not below that sum, unless it is known to be reached.
    template <bool COUNT, class F>
    __device__ __forceinline__ bool find_bin(double above, F target_of, double &target, bool reached = false)
    {
        constexpr int PER = Of::BINS / LANES;
        Of::sync();
        const int first = threadIdx.x % LANES * PER;
        double own[PER], sum = 0.0, all;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            own[k] = COUNT ? (double)reinterpret_cast<const unsigned *>(s.bins)[first + k] : s.bins[first + k];
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

    // Keeps, of what is kept, the beginning whose weights (COUNT: of one each) reach a target: all entries before which there is less.
    template <bool COUNT, class F>
    __device__ __forceinline__ void cut(double range, F target_of)
    {
        double above = 0.0, target = 0.0;
        float low = -3.402823466e38f, high = top;
        Scale x = scale_of(top, range);
        for (int level = 0;; ++level) {
            clear_bins();
            if constexpr (COUNT) {
                each_of(
                    [&](const float *v, unsigned) {
                        unsigned those = 0;
#pragma unroll
                        for (int k = 0; k < 8; ++k) those |= v[k] >= low && v[k] <= high ? 1u << k : 0u;
                        return those;
                    },
                    [&](float v, unsigned) { add<true>(x.bin(v), 1.0); });
            } else {
                each_kept([&](const float *v, unsigned) {
                    double w[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) w[k] = mass(v[k]);
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (v[k] >= low && v[k] <= high) add<false>(x.bin(v[k]), w[k]);
                });
            }
            // from the second level on it is a bin that reaches the target which is taken apart
            if (!find_bin<COUNT>(above, [&](double all) { return level == 0 ? target_of(all) : target; }, target, level > 0)) return;
            above = s.above;
            // A place on the scale from `first` on and not from `behind` on is in the bin (the last one: wherever it lies, infinity included).  Of a part that is taken
            // apart, what is above it lies before 0 and what is below it is under `low`.
            const int bin = (int)s.bin;
            const float first = (float)bin, behind = bin == Of::BINS - 1 ? NAN : (float)(bin + 1);
            each_of(
                [&](const float *v, unsigned) {
                    unsigned those = 0;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float t = x.at(v[k]);
                        those |= t >= first && !(t >= behind) && v[k] >= low ? 1u << k : 0u;
                    }
                    return those;
                },
                [&](float v, unsigned at) {
                    list(v, at);
                    atomicMin(&s.least, key_of(v));
                    atomicMax(&s.most, key_of(v));
                });
            Of::sync();
            const unsigned listed = s.listed, lo = s.least, hi = s.most;
            if (listed <= Of::LISTED) {
                in_list<COUNT>((int)listed, above, target);
                return;
            }
            low = value_of(lo);
            high = value_of(hi);
            if (lo == hi) {
                in_places(low, listed, above, target, COUNT ? 1.0 : mass(low));
                return;
            }
            x = scale_of(high, (double)high - (double)low);
        }
    }

    // The cut within the listed entries: each finds its rank among them, and the sum of weights up to it.
    template <bool COUNT>
    __device__ __forceinline__ void in_list(int n, double above, double target)
    {
        const int i = threadIdx.x % LANES;
        if (i < n) {
            const uint64_t mine = s.list[i];
            const int at = rank(i, n);
            s.sorted[at] = mine;
            s.sorted_weight[at] = COUNT ? 1.0 : mass(value_of(~(unsigned)(mine >> 32)));
        }
        Of::sync();
        const double w = i < n ? s.sorted_weight[i] : 0.0;
        double all;
        const double sum = above + Of::upto(w, s.wave_sum, all), before = sum - w;
        // the last one before which there is less than the target; the first of the bin is one
        if (i < n && before < target && (i == n - 1 || sum >= target)) {
            s.key = ~(unsigned)(s.sorted[i] >> 32);
            s.place = (unsigned)s.sorted[i];
        }
        Of::sync();
        least = value_of(s.key);
        last = s.place;
    }

    // The first entry of the order alone.
    __device__ __forceinline__ void first_alone()
    {
        least = top;
        unsigned place = 0xffffffffu;
        each_kept([&](const float *v, unsigned at) {
#pragma unroll
            for (int k = 7; k >= 0; --k)
                if (v[k] > -INFINITY) place = min(place, at + k);
        });
        Of::sync();
        if (threadIdx.x % LANES == 0) s.place = 0xffffffffu;
        Of::sync();
        if (place != 0xffffffffu) atomicMin(&s.place, place);
        Of::sync();
        last = s.place;
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
        // those already cut off stand behind all that are kept
        const unsigned until = value > least ? 0xffffffffu : last;
        const auto there = [&](const Eight<T> &e, unsigned at, int k) { return e[k] == value && at + k <= until; };
        unsigned mine = 0;
        row.each([&](const Eight<T> &e, unsigned at) {
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
            row.each([&](const Eight<T> &e, unsigned at) {
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

    // Of few entries all but about those are left out at once: k values from different places (`mine`: a thread's largest; else the eights' largest) are k
    // entries, so that what is below the least of them is not among the first k.
    __device__ __forceinline__ void leave_out(int64_t k, float mine)
    {
        const bool few = k <= LANES / 2;
        if (!few && k * 16 > row.vocab) return;
        const Scale x = scale_of(top, 24.0);
        const auto each = [&](auto f) {
            if (few) {
                if (mine > -INFINITY) f(mine);
            } else {
                row.each([&](const Eight<T> &e, unsigned) {
                    const float most = largest(e);
                    if (most > -INFINITY) f(most);
                });
            }
        };
        clear_bins();
        each([&](float v) { add<true>(x.bin(v), 1.0); });
        double target;
        if (!find_bin<true>(0.0, [&](double) { return (double)k; }, target)) return;
        const int bin = (int)s.bin;
        float lowest = INFINITY;
        each([&](float v) {
            if (x.bin(v) <= bin) lowest = fminf(lowest, v);
        });
        lowest = -over_lanes<Max, 64>(-lowest);
        if (threadIdx.x % 64 == 0 && lowest < INFINITY) atomicMin(&s.least, key_of(lowest));
        Of::sync();
        least = value_of(s.least);
    }

    // Draws among at most k entries, all of which the list holds: every filter and the draw within it.  False: it does not hold them.
    __device__ __forceinline__ bool draw_listed(int k, double top_p, double floor_p, double u, unsigned &token, float &value)
    {
        each_kept([&](const float *v, unsigned at) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (v[i] > -INFINITY) list(v[i], at + i);
        });
        Of::sync();
        const int n = (int)s.listed, i = threadIdx.x % LANES;
        if (n > Of::LISTED) return false;
        const uint64_t mine = i < n ? s.list[i] : 0;
        const int order = i < n ? rank(i, n) : 0;
        const float v = value_of(~(unsigned)(mine >> 32));
        const double w = i < n && order < k ? weight(v) : 0.0;
        if (i < n) s.sorted_weight[order] = (w + grid) - grid;
        Of::sync();
        // the mass of the first k, and before each
        const double m = i < n ? s.sorted_weight[i] : 0.0;
        double all;
        const double upto = Of::upto(m, s.wave_sum, all);
        if (i < n) s.bins[i] = upto - m;
        Of::sync();
        const bool kept = i < n && order < k && (order == 0 || (s.bins[order] < top_p * all && w >= floor_p));
        const double mass = kept ? (w + grid) - grid : 0.0;
        if (i < n) {
            s.sorted[i] = mine & 0xffffffffu;
            s.sorted_weight[i] = mass;
        }
        Of::sync();
        double before = 0.0, total = 0.0;
        if (kept) {
#pragma unroll 4
            for (int j = 0; j < n; ++j) {
                const double other = s.sorted_weight[j];
                total += other;
                before += s.sorted[j] < (mine & 0xffffffffu) ? other : 0.0;
            }
        }
        token = kept && before <= u * total && before + mass > u * total ? (unsigned)mine : 0xffffffffu;       // one thread's
        value = v;
        return true;
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
    r.row.load([&](const Eight<T> &e, unsigned) {
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
    r.last = 0xffffffffu;
    // The grid of the masses: their sum has to stay below 2^52 times it.  No more than as many as entries can stay, none above 1: of n, what is rounded away is below n^2 2^-52.  From
    // COUNTED on that would show, and the row's own sum is the bound: what stays then has, of the row's n entries, at least its share, and is off by less than n 2^-51 of itself.
    // At temperature 1 logp's sum is that one; else it is 8 exponentials more to a pass, without logp a pass (256 x 50257 in bf16 22.2 -> 25.0 us; by eight times the largest of every
    // eight 24.4, and 26.2 with logp, which takes 25.0).
    constexpr double COUNTED = 1024.0;
    const bool greedy = heat == 0.0f || top_p <= 0.0f || top_k == 1;
    double most = top_k > 0 ? fmin((double)top_k, (double)a.vocab) : (double)a.vocab;
    const bool by_sum = !greedy && most > COUNTED;
    r.factor = 1.4426950408889634074 / (double)heat;
    // The policy's own sum and, at another temperature, the masses', in fp32's exponentials: a term's error is its own, and the sums are in 64 bits.
    double whole = 0.0, heated = 0.0;
    if (a.logp || by_sum) {
        const float factor = (float)fmin(r.factor, 1e30), first = a.logp || heat == 1.0f ? 1.44269504f : factor;
        // by halves, which keeps differences within fp32: at the highest temperatures an entry at the type's other end has weight
        const float half = 0.5f * top;
        const bool both = a.logp && by_sum && heat != 1.0f;
        const auto sum_of = [&](const Eight<T> &e, float factor) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = __builtin_amdgcn_exp2f(__builtin_fmaf(e[k], 0.5f, -half) * (2.0f * factor));
            return (double)(((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])));
        };
        r.row.each([&](const Eight<T> &e, unsigned) {
            whole += sum_of(e, first);
            if (both) heated += sum_of(e, factor);
        });
        double all;
        Of::upto(whole, s.wave_sum, all);
        whole = all;
        if (both) Of::upto(heated, s.wave_sum, all);
        if (by_sum) most = fmin(most, 1.01 * all);
    }

    // ---- what is kept
    if (greedy) {
        r.first_alone();
        if (threadIdx.x % LANES == 0) {
            a.tokens[row] = (int64_t)r.last;
            if (a.logp) a.logp[row] = (float)-log(whole);
        }
        return;
    }
    r.grid = __builtin_amdgcn_ldexp(1.5, __builtin_amdgcn_frexp_exp(most));
    if (top_k > 0 && top_k < a.vocab) {
        r.leave_out(top_k, mine);
        if (top_k <= Of::LISTED / 2) {
            unsigned token;
            float value;
            if (r.draw_listed((int)top_k, (double)top_p, fmin((double)min_p, 1.0), (double)u, token, value)) {
                if (token != 0xffffffffu) {
                    a.tokens[row] = (int64_t)token;
                    if (a.logp) a.logp[row] = (float)(((double)value - (double)top) - log(whole));
                }
                return;
            }
        }
        r.template cut<true>(24.0, [&](double) { return (double)top_k; });
    }
    if (top_p < 1.0f)
        r.template cut<false>(24.0 * (double)heat, [&](double all) { return (double)top_p * all; });
    const double floor_p = fmin((double)min_p, 1.0);
    const auto kept_mass = [&](float v) {
        const double w = r.weight(v);
        return w >= floor_p ? (w + r.grid) - r.grid : 0.0;
    };

    // ---- the draw: the first entry with more than u of the kept mass up to it
    double own = 0.0;
    const auto sum_of = [&](const double *m) { return ((m[0] + m[1]) + (m[2] + m[3])) + ((m[4] + m[5]) + (m[6] + m[7])); };
    const bool uncut = r.last == 0xffffffffu && r.least == -3.402823466e38f;
    if (uncut && floor_p <= 0.0) {
        // nothing is left out: -inf has no mass by itself
        r.row.each([&](const Eight<T> &e, unsigned) {
            double m[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) m[k] = r.mass(e[k]);
            own += sum_of(m);
        });
    } else {
        // where no lane of the wavefront has more than a few of eight, each its own one by one, read again (without a cut none is looked for: 1 us of 25)
        r.each_kept([&](const float *v, unsigned at) {
            unsigned those = 0;
            if (!uncut) {
#pragma unroll
                for (int k = 0; k < 8; ++k) those |= v[k] > -INFINITY ? 1u << k : 0u;
            }
            if (uncut || __any(__builtin_popcount(those) > 3)) {
                double m[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) m[k] = kept_mass(v[k]);
                own += sum_of(m);
            } else {
                for (; those; those &= those - 1) own += kept_mass(r.row.value(at + (unsigned)__builtin_ctz(those)));
            }
        });
    }
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
    // every eight of the wavefront, those with nothing kept too: the sums are the whole wavefront's
    const float above = value_of(key_of(r.least) + 1);
    r.row.each([&](const Eight<T> &e, unsigned at) {
        if (!__any(largest(e) >= r.least)) return;
        double m[8], here = 0.0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            m[k] = kept_mass(e[k] >= (at + k <= r.last ? r.least : above) ? e[k] : -INFINITY);
            here += m[k];
        }
        const double sum = upto_lane(here);
        double c = before + (sum - here);
        if (c <= target && before + sum > target) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (c <= target && c + m[k] > target) {
                    a.tokens[row] = (int64_t)(at + k);
                    if (a.logp) a.logp[row] = (float)(((double)e[k] - (double)top) - log(whole));
                }
                c += m[k];
            }
        }
        before += of_last_lane(sum);
    });
}

}  // namespace ef
