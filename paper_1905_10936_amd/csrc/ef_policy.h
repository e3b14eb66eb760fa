// Log-probabilities of tokens, and the clipped policy loss with its gradient, on rows of logits.
//
// The gradient needs the whole row's sum of exponentials before its first element, and loss and gradient of a row depend on that row
// alone, so a team of LANES threads reads the row once, holds it in registers as it lies in memory (CHUNKS times eight elements a
// thread) and writes the gradient from there: 2 bytes an element read and 2 written in bf16, the least there is.  Rows too long for
// that are read twice.  4096 rows of 50257 in bf16: 168 us, 4.9 TB/s, of which the sum of the losses (k_sum_losses) takes 4; a copy of 1 GiB
// reaches 5.1.
//
// exp(l - m) is 2^(l * L - c) with L = log2(e) rounded and c = m * L rounded, one fused operation and one exponential an element; what
// c was rounded by is put right once a row.  That holds as long as it is little beside the exponents that count: rows whose maximum m is a large number
// (LARGE) have it taken off first, without a rounding of its product.
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

// What a row's loss needs besides its logits, asked for a row ahead.
struct RowArgs {
    int64_t token;
    float q, old, ref, adv;     // q: the row's weight, 0 if it is masked
    __device__ __forceinline__ void load(const PolicyArgs &a, int64_t row)
    {
        token = a.tokens[row];
        q = a.token_weight ? a.token_weight[row] : 1.0f;
        old = a.logp_old ? a.logp_old[row] : 0.0f;
        ref = a.logp_ref ? a.logp_ref[row] : 0.0f;
        adv = a.loss ? a.advantage[row] : 0.0f;
    }
    // the same in scalar registers, where the wavefront has one row
    __device__ __forceinline__ RowArgs scalar() const
    {
        const auto one = [](float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); };
        RowArgs s;
        s.token = (int64_t)((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((unsigned)token) |
                            (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((unsigned)((uint64_t)token >> 32)) << 32);
        s.q = one(q);
        s.old = one(old);
        s.ref = one(ref);
        s.adv = one(adv);
        return s;
    }
    __device__ __forceinline__ bool masked(const PolicyArgs &a) const { return q == 0.0f || (uint64_t)token >= (uint64_t)a.vocab; }
};

// Loss of a row and its derivative with respect to logp, times the row's weight.
__device__ __forceinline__ float2 row_loss(const PolicyArgs &a, const RowArgs &w, float logp)
{
    const float r = a.logp_old ? expf(logp - w.old) : 1.0f;
    const float free = r * w.adv, held = fminf(fmaxf(r, a.low), a.high) * w.adv;
    float f = -(free <= held ? free : held), c = free <= held ? -free : 0.0f;
    if (!(free == free) || !(held == held)) f = c = free + held;      // NaN
    if (a.logp_ref) {
        const float d = w.ref - logp, m = expm1f(d);
        f += a.kl * (m - d);
        c -= a.kl * m;
    }
    return make_float2(w.q * f, w.q * c);
}

// A row's maximum that is larger in size: c would be rounded by more than 2^-4, and from 2^31 on by more than an exponential's range.
constexpr float LARGE = 0x1p20f;

struct Exponent {
    float factor, c;
    // From LARGE on bf16 numbers are 2^12 apart and more, so that any other logit's exponential is 0 whatever the factor: 1 multiplies exactly.
    // A row of fp32 comes here with its maximum taken off (shift_large).
    __device__ __forceinline__ explicit Exponent(float top)
    {
        factor = fabsf(top) > LARGE ? 1.0f : LOG2E;
        c = top * factor;
    }
    __device__ __forceinline__ float of(float l) const { return __builtin_amdgcn_exp2f(__builtin_fmaf(l, factor, -c)); }
    // log of the row's sum of exponentials less `top`, from the sum of of(l)
    __device__ __forceinline__ float log_sum(float sum, float top) const { return logf(sum) - LN2 * __builtin_fmaf(top, factor, -c); }
};

// A row of fp32 whose maximum is large in size less that maximum, in place: 0 and the differences, each rounded once.
template <int CHUNKS>
__device__ __forceinline__ void shift_large(Eight<float> (&e)[CHUNKS], float &tail, float &chosen, float &top)
{
    if (!(fabsf(top) > LARGE)) return;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int k = 0; k < 8; ++k) e[c].set(k, __float_as_uint(e[c][k] - top));
    tail -= top;
    chosen -= top;
    top = 0.0f;
}

constexpr int policy_threads(int lanes) { return lanes < 256 ? 256 : lanes; }

// A masked row's outputs.
template <class T, int LANES>
__device__ __forceinline__ void masked_row(const PolicyArgs &a, int64_t row, int lane)
{
    if (lane == 0) {
        if (a.logp) a.logp[row] = 0.0f;
        if (a.losses) a.losses[row] = 0.0f;
    }
    if (!a.dlogits) return;
    T *g = static_cast<T *>(a.dlogits) + row * a.dlogits_stride;
    Eight<T> zero;
    zero.fill(0u);
    for (int64_t i = (int64_t)lane * 8; i < a.vocab; i += LANES * 8) store_some(zero, g + i, a.vocab - i);
}

// A row as accesses see it: `head` elements up to the first 16-byte boundary, `whole` (a multiple of 8) from there, and the rest.  Accesses at
// any place are allowed but slower: 4096 rows of 50257 in bf16, which start at odd places, take 210 us that way, 173 on boundaries.
struct RowParts {
    int head, whole;
    template <class T>
    __device__ __forceinline__ RowParts(const T *l, int vocab)
    {
        head = min(vocab, (int)(-(unsigned)(uintptr_t)l % 16u / sizeof(T)));
        whole = (vocab - head) & ~7;
    }
    // of head and rest the one element that lane 0..15 takes: below 8 the head's, above the rest's; vocab or more: none
    __device__ __forceinline__ int edge(int lane, int vocab) const
    {
        if (lane < 8) return lane < head ? lane : vocab;
        return lane < 16 && lane - 8 < vocab - head - whole ? head + whole + lane - 8 : vocab;
    }
};

// A team takes rows team, team + teams, ...; of a row, thread `lane` holds elements (c LANES + lane) 8 .. + 7 of its whole part for c < CHUNKS, and one
// of its edges.
template <class T, int LANES, int CHUNKS>
__global__ __launch_bounds__(policy_threads(LANES), LANES == 1024 && sizeof(T) * CHUNKS <= 16 ? 8 : 4) void k_policy(PolicyArgs a)
{
    constexpr int TEAMS = policy_threads(LANES) / LANES;
    constexpr unsigned NONE = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;       // -inf
    __shared__ float tops[LANES > 64 ? LANES / 64 : 1], sums[LANES > 64 ? LANES / 64 : 1], slope;
    const int lane = threadIdx.x % LANES, vocab = (int)a.vocab;
    const unsigned off = lane * 8 * (unsigned)sizeof(T);
    const int64_t teams = (int64_t)gridDim.x * TEAMS;
    int64_t row = (int64_t)blockIdx.x * TEAMS + (LANES < 64 ? (int)threadIdx.x / LANES : LANES < 256 ? (int)__builtin_amdgcn_readfirstlane(threadIdx.x / LANES) : 0);
    RowArgs next;
    if (row < a.rows) next.load(a, row);
    for (; row < a.rows; row += teams) {
        const RowArgs w = LANES >= 64 ? next.scalar() : next;
        if (row + teams < a.rows) next.load(a, row + teams);
        if (w.masked(a)) {
            masked_row<T, LANES>(a, row, lane);
            continue;
        }
        const T *l = static_cast<const T *>(a.logits) + row * a.stride;
        const RowParts part(l, vocab);
        const int whole = part.whole, last = part.edge(lane, vocab), chunks = (whole + LANES * 8 - 1) / (LANES * 8);
        // Of chunk c a thread has the eight from byte `from(c)` of the whole part on: formed where it is used (a number kept for each chunk costs registers:
        // 2048 rows of 65000 in bf16 140 us, 119 this way).
        const auto from = [&](int c) { return here(off) + c * LANES * 8 * (unsigned)sizeof(T); };
        const unsigned whole_bytes = whole * (unsigned)sizeof(T);
        Eight<T> e[CHUNKS];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const unsigned at = from(c);
            e[c].fill(NONE);
            if (at < whole_bytes) e[c].load_at(l + part.head, at);
        }
        float tail = last < vocab ? to_float<T>(l[last]) : -INFINITY;
        // The token's logit goes into the maximum: it is there before the row's first barrier, and the gradient may be written over the row
        // behind it.
        float chosen = to_float<T>(l[w.token]);
        float top = fmaxf(chosen, tail);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            if (c < chunks) {
#pragma unroll
                for (int k = 0; k < 8; ++k) top = fmaxf(top, e[c][k]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        top = over_row<Max, LANES>(top, tops);
        if constexpr (sizeof(T) == 4) shift_large(e, tail, chosen, top);
        const Exponent x(top);
        float sum = x.of(tail);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            if (c < chunks) {
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = x.of(e[c][k]);
                sum += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        sum = over_row<Add, LANES>(sum, sums);
        // The row's own arithmetic is one wavefront's: a hundred instructions that sixteen need not repeat.
        float2 f = make_float2(0.0f, 0.0f);
        if (LANES <= 64 || threadIdx.x < 64) {
            const float logp = (chosen - top) - x.log_sum(sum, top);
            if (a.loss) f = row_loss(a, w, logp);
            if (lane == 0) {
                if (a.logp) a.logp[row] = logp;
                if (a.losses) a.losses[row] = f.x;
                if (LANES > 64) slope = f.y;
            }
        }
        if (!a.dlogits) continue;
        if (LANES > 64) {
            __syncthreads();
            f.y = slope;
        }
        T *g = static_cast<T *>(a.dlogits) + row * a.dlogits_stride;
        const float p = -f.y / sum;
        const unsigned token_at = ((int)w.token - part.head) * (unsigned)sizeof(T);         // wraps where it lies before the whole part
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            if (c < chunks) {
                const unsigned to = from(c), at = token_at - to;
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = x.of(e[c][k]) * p;
                if (at < 8 * sizeof(T)) {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (at == k * sizeof(T)) v[k] += f.y;
                }
                Eight<T> o;
                o.round(v);
                if (to < whole_bytes) o.store_at(g + part.head, to);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (last < vocab) g[last] = from_float<T>(x.of(tail) * p + (w.token == last ? f.y : 0.0f));
    }
}

// Eight more elements to a maximum and the sum of 2^((l - maximum) L) up to here; -inf and 0 while there has been nothing but -inf.
template <class T>
__device__ __forceinline__ void more_of_row(const Eight<T> &e, float &top, float &sum)
{
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
    if (top != -INFINITY) {
        sum += s;
    } else {
        // nothing but -inf gives NaN here; a NaN among the eight has to show
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (e[k] != e[k]) sum = e[k];
    }
}

// Rows longer than a workgroup's registers (196608 entries in bf16, 98304 in fp32: 96 registers a thread of the 128 there are; 2048 rows of 128256 in bf16
// take 225 us that way, 266 here; of 196000 350 and 450; of 80000 in fp32 268 and 340): maximum and sum kept up to date chunk by chunk, the row read again
// for the gradient.
constexpr int LONG_THREADS = 1024;
template <class T>
__global__ __launch_bounds__(LONG_THREADS) void k_policy_long(PolicyArgs a)
{
    constexpr unsigned NONE = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
    __shared__ float tops[LONG_THREADS / 64], sums[LONG_THREADS / 64];
    const int64_t row = blockIdx.x;
    const T *l = static_cast<const T *>(a.logits) + row * a.stride;
    T *g = a.dlogits ? static_cast<T *>(a.dlogits) + row * a.dlogits_stride : nullptr;
    RowArgs w;
    w.load(a, row);
    if (w.masked(a)) {
        masked_row<T, LONG_THREADS>(a, row, threadIdx.x);
        return;
    }
    const int64_t token = w.token;
    const float chosen = to_float<T>(l[token]);
    // sum of 2^((l - top) * L) so far; a thread that has seen nothing but -inf has top = -inf and sum 0
    float top = -INFINITY, sum = 0.0f;
    for (int64_t i = (int64_t)threadIdx.x * 8; i < a.vocab; i += LONG_THREADS * 8) {
        Eight<T> e;
        load_some(e, l + i, a.vocab - i, NONE);
        more_of_row(e, top, sum);
    }
    const float all = over_row<Max, LONG_THREADS>(fmaxf(top, chosen), tops);
    sum = over_row<Add, LONG_THREADS>(sum == 0.0f ? 0.0f : sum * __builtin_amdgcn_exp2f((top - all) * LOG2E), sums);
    if (all == -INFINITY) sum = NAN;        // nothing but -inf
    const float logp = (chosen - all) - logf(sum);
    float2 f = make_float2(0.0f, 0.0f);
    if (a.loss) f = row_loss(a, w, logp);
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

// Few rows of many entries: a row cut into slices, a workgroup each, in two kernels.  The first leaves every slice's maximum and sum of exponentials, and the
// token's logit; in the second each workgroup joins its row's and writes its slice's gradient.  5 rows of 50304 in fp32: 11.8 us with a
// workgroup to a row, 8.3 with 25; 16 rows of 200000 in bf16: 34.6 and 11.2; 16 of 9000, where a workgroup has its row in registers: 8.0 and 8.3.
// About SLICES_ALL workgroups at most: 64 rows of 128256 in bf16 14.5 us with 16 slices a row, 17.5 with 63.
constexpr int SLICE_THREADS = 256, SLICE = 2048, SLICES_MAX = 64, SLICES_ALL = 1024, SLICED_ROWS = 64, SLICED_VOCAB = 32768;
struct SliceRef {
    float2 *joint;              // [rows][SLICES_MAX] maximum, sum of 2^((l - maximum) L)
    float *chosen;              // [rows]
    int count, length;          // slices of a row, elements of one (a multiple of 8)
};

template <class T>
__global__ __launch_bounds__(SLICE_THREADS) void k_policy_slices(PolicyArgs a, SliceRef s)
{
    __shared__ float tops[SLICE_THREADS / 64], sums[SLICE_THREADS / 64];
    const int64_t row = blockIdx.x / s.count;
    const int slice = blockIdx.x % s.count, vocab = (int)a.vocab;
    RowArgs w;
    w.load(a, row);
    if (w.masked(a)) return;
    const T *l = static_cast<const T *>(a.logits) + row * a.stride;
    const RowParts part(l, vocab);
    const int64_t end = min((int64_t)part.whole, (int64_t)(slice + 1) * s.length);
    const int last = slice == 0 ? part.edge(threadIdx.x, vocab) : vocab;
    float top = last < vocab ? to_float<T>(l[last]) : -INFINITY, sum = top == -INFINITY ? 0.0f : 1.0f;
    if (top != top) sum = top;
    for (int64_t i = (int64_t)slice * s.length + threadIdx.x * 8; i < end; i += SLICE_THREADS * 8) {
        Eight<T> e;
        e.load(l + part.head + i);
        more_of_row(e, top, sum);
    }
    const float all = over_row<Max, SLICE_THREADS>(top, tops);
    sum = over_row<Add, SLICE_THREADS>(sum == 0.0f ? 0.0f : sum * __builtin_amdgcn_exp2f((top - all) * LOG2E), sums);
    if (threadIdx.x == 0) {
        s.joint[row * SLICES_MAX + slice] = make_float2(all, sum);
        if (slice == 0) s.chosen[row] = to_float<T>(l[w.token]);
    }
}

// Maximum and sum of a row from its slices', one to a lane; all 64 lanes get them.
__device__ __forceinline__ float2 join_slices(float2 v)
{
    const float top = over_lanes<Max, 64>(v.x);
    const float sum = over_lanes<Add, 64>(v.y == 0.0f ? 0.0f : v.y * __builtin_amdgcn_exp2f((v.x - top) * LOG2E));
    return make_float2(top, top == -INFINITY ? NAN : sum);      // NaN: nothing but -inf
}
__device__ __forceinline__ float2 slice_of(const SliceRef &s, int64_t row, int lane)
{
    return lane < s.count ? s.joint[row * SLICES_MAX + lane] : make_float2(-INFINITY, 0.0f);
}

// The sum of all rows' losses, formed once more from the slices by a workgroup of its own beside those that write the gradient: wavefront w joins
// rows w, w + 4, ..., whose losses its lanes 0, 1, ... then form at once.
__device__ __forceinline__ void sum_of_slices(const PolicyArgs &a, const SliceRef &s, float *loss)
{
    static_assert(SLICED_ROWS <= 64, "sixteen rows to a wavefront");
    __shared__ double part[4];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t mine = wave + 4 * lane;
    const bool there = lane < 16 && mine < a.rows;
    RowArgs w;
    float chosen = 0.0f;
    if (there) {
        w.load(a, mine);
        chosen = s.chosen[mine];
    }
    float2 j = make_float2(0.0f, 1.0f);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float2 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t row = wave + 4 * (half * 8 + k);
            v[k] = row < a.rows ? slice_of(s, row, lane) : make_float2(0.0f, 1.0f);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float2 r = join_slices(v[k]);
            if (lane == half * 8 + k) j = r;
        }
    }
    double total = 0.0;
    if (there && !w.masked(a)) total = (double)row_loss(a, w, (chosen - j.x) - logf(j.y)).x;
#pragma unroll
    for (int h = 8; h > 0; h /= 2) total += __shfl_down(total, h, 16);
    if (lane == 0) part[wave] = total;
    __syncthreads();
    if (threadIdx.x == 0) *loss = (float)((part[0] + part[1]) + (part[2] + part[3]));
}

template <class T>
__global__ __launch_bounds__(SLICE_THREADS) void k_policy_join(PolicyArgs a, SliceRef s, float *loss)
{
    __shared__ float joined[3];
    const int64_t row = blockIdx.x / s.count;
    const int slice = blockIdx.x % s.count, vocab = (int)a.vocab, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    if (row == a.rows) {
        sum_of_slices(a, s, loss);
        return;
    }
    RowArgs w;
    w.load(a, row);
    float2 v = make_float2(0.0f, 1.0f);
    float chosen = 0.0f;
    if (wave == 0) {
        v = slice_of(s, row, lane);
        chosen = s.chosen[row];
    }
    const bool masked = w.masked(a);
    if (wave == 0 && !masked) {
        const float2 r = join_slices(v);
        const float logp = (chosen - r.x) - logf(r.y);
        const float2 f = row_loss(a, w, logp);
        if (lane == 0) {
            joined[0] = r.x;
            joined[1] = r.y;
            joined[2] = f.y;
            if (slice == 0) {
                if (a.logp) a.logp[row] = logp;
                if (a.losses) a.losses[row] = f.x;
            }
        }
    }
    if (masked && slice == 0 && threadIdx.x == 0) {
        if (a.logp) a.logp[row] = 0.0f;
        if (a.losses) a.losses[row] = 0.0f;
    }
    if (!a.dlogits) return;
    __syncthreads();
    const T *l = static_cast<const T *>(a.logits) + row * a.stride;
    T *g = static_cast<T *>(a.dlogits) + row * a.dlogits_stride;
    const RowParts part(l, vocab);
    const int64_t end = min((int64_t)part.whole, (int64_t)(slice + 1) * s.length);
    const int last = slice == 0 ? part.edge(threadIdx.x, vocab) : vocab;
    const float top = masked ? 0.0f : joined[0], c = masked ? 0.0f : joined[2], p = masked ? 0.0f : -c / joined[1];
    const int token = masked ? -1 : (int)w.token;
    for (int64_t i = (int64_t)slice * s.length + threadIdx.x * 8; i < end; i += SLICE_THREADS * 8) {
        float v[8] = {};
        if (!masked) {
            Eight<T> e;
            e.load(l + part.head + i);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v[k] = __builtin_amdgcn_exp2f((e[k] - top) * LOG2E) * p;
                if (token - part.head - i == k) v[k] += c;
            }
        }
        Eight<T> o;
        o.round(v);
        o.store(g + part.head + i);
    }
    if (last < vocab)
        g[last] = from_float<T>(masked ? 0.0f : __builtin_amdgcn_exp2f((to_float<T>(l[last]) - top) * LOG2E) * p + (token == last ? c : 0.0f));
}

// loss <- the sum of the rows' losses: a thread adds four neighbouring ones and those 4096 further on, eight times four on their way at once, then a fixed
// tree.
__global__ __launch_bounds__(1024) void k_sum_losses(const float *losses, int64_t rows, float *loss)
{
    __shared__ double sums[16];
    double s = 0.0;
    for (int64_t i = (int64_t)threadIdx.x * 4; i < rows; i += 8 * 4096) {
        Eight<float> v[4];
        float e[4] = {};
        if (i + 7 * 4096 + 4 <= rows) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[k].lo = *reinterpret_cast<const u32x4_word *>(losses + i + 2 * k * 4096);
                v[k].hi = *reinterpret_cast<const u32x4_word *>(losses + i + (2 * k + 1) * 4096);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) s += (double)v[k][j];
        } else {
            for (int64_t k = i; k < rows; k += 4096) {
#pragma unroll
                for (int j = 0; j < 4; ++j) e[j] = k + j < rows ? losses[k + j] : 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) s += (double)e[j];
            }
        }
    }
#pragma unroll
    for (int h = 32; h > 0; h /= 2) s += __shfl_down(s, h);
    if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = s;
    __syncthreads();
    if (threadIdx.x < 16) {
        s = sums[threadIdx.x];
#pragma unroll
        for (int h = 8; h > 0; h /= 2) s += __shfl_down(s, h, 16);
        if (threadIdx.x == 0) *loss = (float)s;
    }
}

}  // namespace ef
