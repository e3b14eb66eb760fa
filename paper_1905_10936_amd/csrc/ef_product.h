// Tiles of a matrix product on matrix instructions, for kernels that end it in their own ways:
//     sum over k of a[c][k] * b[t][k],   c: output channels, t: tokens, k: what is summed over.
//
// Four wavefronts make a tile of 64 WC channels x 64 WT tokens, a quarter each (two along the channels, two along the tokens): WC x WT results of
// 32 x 32 a wavefront.  Operands go through LDS in steps of 128 bytes of k: 64 in bf16, 32 in fp32.  The tokens' rows, and a weight's rows where it is
// used as it lies in memory (RowsOperand), have k contiguous: they lie in LDS row by row, 144 bytes apart so that the rows that are read together fall
// on different banks, and a lane reads 16 bytes of its row.  A weight whose rows are what is summed over (ColumnsOperand) lies there with its channels
// contiguous and is read transposed.
//
// bf16 products are exact in the instruction and added up in fp32.  fp32 ones run on the fp32 instruction: nothing is lost but the sums' rounding.
// The order in which a region's k fall on the instruction's is the same for both operands, which is all that a sum needs.
#pragma once
#include "ef_grad.h"

namespace ef {

constexpr int PRODUCT_THREADS = 256, STEP_BYTES = 128, ROW_PITCH = STEP_BYTES + 16, REGIONS = 4;
template <class T>
constexpr int STEP = STEP_BYTES / (int)sizeof(T);           // k of a step
template <class T>
constexpr int WORD = 16 / (int)sizeof(T);                   // elements of a 16-byte word

template <class T>
__device__ __forceinline__ u32x4 load_word(const EF_GLOBAL char *p)
{
    if constexpr (sizeof(T) == 2)
        return *(const EF_GLOBAL u32x4_any *)p;
    else
        return *(const EF_GLOBAL u32x4_word *)p;
}
// The first `left` (any number, also none or less) elements of a word, zeros for the rest; nothing behind them is read.
template <class T>
__device__ __forceinline__ u32x4 load_part(const EF_GLOBAL char *p, int64_t left)
{
    if (left >= WORD<T>) return load_word<T>(p);
    u32x4 w = {0, 0, 0, 0};
    if (left > 0) {
        const int n = (int)left;
        unsigned e[WORD<T> - 1];
#pragma unroll
        for (int i = 0; i < WORD<T> - 1; ++i) {
            if constexpr (sizeof(T) == 2)
                e[i] = *((const EF_GLOBAL uint16_t *)p + min(i, n - 1));
            else
                e[i] = *((const EF_GLOBAL unsigned *)p + min(i, n - 1));
        }
#pragma unroll
        for (int i = 0; i < WORD<T> - 1; ++i) {
            if (i >= n) e[i] = 0;
            if constexpr (sizeof(T) == 2)
                w[i / 2] |= i & 1 ? e[i] << 16 : e[i];
            else
                w[i] = e[i];
        }
    }
    return w;
}

// An operand of 32 BLOCKS rows with k contiguous; a thread carries one word of each block.  `place` gives the row of the matrix (one that is there) that
// is row `row()` of block b.
template <class T, int BLOCKS>
struct RowsOperand {
    static constexpr int N = BLOCKS, BYTES = 32 * BLOCKS * ROW_PITCH;
    u32x4 w[N];
    const EF_GLOBAL char *base;
    unsigned off[N];
    static __device__ __forceinline__ int word() { return threadIdx.x % 8; }
    static __device__ __forceinline__ int row() { return threadIdx.x / 8; }
    // Whole steps of k, if its rows are within 32 bits of one another.
    static __device__ __forceinline__ int64_t safe(int64_t k, int64_t stride, int64_t span)
    {
        return stride > ((int64_t)1 << 32) / (int64_t)sizeof(T) / (span + 1) ? 0 : k / STEP<T>;
    }
    template <class Place>
    __device__ __forceinline__ void begin(const void *m, int64_t stride, int64_t k0, int64_t base_row, Place place)
    {
        base = (const EF_GLOBAL char *)m + (base_row * stride + k0) * (int64_t)sizeof(T);
#pragma unroll
        for (int b = 0; b < N; ++b) off[b] = (unsigned)((place(b) - base_row) * stride * (int64_t)sizeof(T)) + word() * 16;
    }
    __device__ __forceinline__ void load(int b)
    {
        stay(off[b]);
        w[b] = load_word<T>(base + off[b]);
    }
    __device__ __forceinline__ void next() { base += STEP_BYTES; }
    // the step from k0 on with zeros behind the rows' end
    template <class Place>
    __device__ __forceinline__ void load_guarded(const void *m, int64_t stride, int64_t k0, int64_t k, Place place)
    {
        const int64_t at = k0 + word() * WORD<T>;
#pragma unroll
        for (int b = 0; b < N; ++b) w[b] = load_part<T>((const EF_GLOBAL char *)m + (place(b) * stride + at) * (int64_t)sizeof(T), k - at);
    }
    __device__ __forceinline__ void put(int b, char *buffer) const { *reinterpret_cast<u32x4 *>(buffer + (32 * b + row()) * ROW_PITCH + word() * 16) = w[b]; }
    // 16 bytes of k of lane % 32's row of block b: the instruction's operand, in as many parts as HALVES
    static constexpr int HALVES = 1;
    static __device__ __forceinline__ int lane_at(int lane) { return lane % 32 * ROW_PITCH + lane / 32 * 16; }
    static __device__ __forceinline__ void fragment(u32x4 &f, const char *buffer, int lane_at, int b, int region, int)
    {
        f = *reinterpret_cast<const u32x4 *>(buffer + lane_at + 32 * b * ROW_PITCH + region * 32);
    }
};

// An operand whose rows are what is summed over: STEP rows of 32 BLOCKS channels, contiguous.
template <class T, int BLOCKS>
struct ColumnsOperand {
    // Four rows that a read takes together fall on different banks: 64 bytes more than the channels take in bf16, 32 in fp32 (two rows four apart).
    static constexpr int WIDTH = 32 * BLOCKS, PITCH = WIDTH * (int)sizeof(T) + (sizeof(T) == 2 ? 64 : 32), BYTES = STEP<T> * PITCH;
    static constexpr int WORDS = WIDTH / WORD<T>, ROWS = PRODUCT_THREADS / WORDS, N = STEP<T> / ROWS;
    u32x4 w[N];
    const EF_GLOBAL char *base;
    unsigned off[N];
    static __device__ __forceinline__ int word() { return threadIdx.x % WORDS; }
    static __device__ __forceinline__ int row() { return threadIdx.x / WORDS; }
    // The first step that load() may not take: a row's last word may reach WORD - 1 elements past its row, and the offsets have to fit 32 bits.
    static __device__ __forceinline__ int64_t safe(int64_t k, int64_t stride, int64_t c0, int64_t channels)
    {
        if (stride > (int64_t)1 << 24) return 0;
        const int64_t spare = c0 + WIDTH <= channels ? 0 : (WORD<T> - 1 + stride - 1) / stride;
        return max((int64_t)0, k - spare) / STEP<T>;
    }
    // channels past the end are read from the first ones; what they give is not stored
    __device__ __forceinline__ void begin(const void *m, int64_t stride, int64_t k0, int64_t c0, int64_t channels)
    {
        const int64_t c = c0 + word() * WORD<T>;
        base = (const EF_GLOBAL char *)m + k0 * stride * (int64_t)sizeof(T);
#pragma unroll
        for (int b = 0; b < N; ++b) off[b] = (unsigned)(((row() + b * ROWS) * stride + (c < channels ? c : 0)) * (int64_t)sizeof(T));
    }
    __device__ __forceinline__ void load(int b)
    {
        stay(off[b]);
        w[b] = load_word<T>(base + off[b]);
    }
    __device__ __forceinline__ void next(int64_t stride) { base += STEP<T> * stride * (int64_t)sizeof(T); }
    __device__ __forceinline__ void load_guarded(const void *m, int64_t stride, int64_t k0, int64_t k, int64_t c0, int64_t channels)
    {
        const int64_t c = c0 + word() * WORD<T>;
#pragma unroll
        for (int b = 0; b < N; ++b) {
            const int64_t at = k0 + row() + b * ROWS;
            w[b] = load_part<T>((const EF_GLOBAL char *)m + (min(at, k - 1) * stride + c) * (int64_t)sizeof(T), at < k ? channels - c : 0);
        }
    }
    __device__ __forceinline__ void put(int b, char *buffer) const { *reinterpret_cast<u32x4 *>(buffer + (row() + b * ROWS) * PITCH + word() * 16) = w[b]; }
    static constexpr int HALVES = 2;
    static __device__ __forceinline__ int lane_at(int lane) { return sizeof(T) == 2 ? grad_lane_offset(lane, PITCH) : lane / 32 * 4 * PITCH + lane % 32 * 4; }
    static __device__ __forceinline__ void fragment(u32x4 &f, const char *buffer, int lane_at, int b, int region, int half)
    {
        if constexpr (sizeof(T) == 2) {
            typedef __attribute__((address_space(3))) s16x4 shared_s16x4;
            const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared_s16x4 *)(buffer + lane_at + b * 64 + (region * 16 + half * 4) * PITCH));
            const u32x2 t = __builtin_bit_cast(u32x2, v);
            f[2 * half] = t.x;
            f[2 * half + 1] = t.y;
        } else {
#pragma unroll
            for (int q = 2 * half; q < 2 * half + 2; ++q) f[q] = *reinterpret_cast<const unsigned *>(buffer + lane_at + b * 128 + (region * 8 + q) * PITCH);
        }
    }
};

template <class T>
__device__ __forceinline__ void multiply(const u32x4 &a, const u32x4 &b, f32x16 &acc)
{
    if constexpr (sizeof(T) == 2) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[q]), __uint_as_float(b[q]), acc, 0, 0, 0);
    }
}

// The products of steps first .. last - 1 into acc.  The operands stand at step `first`; advance(): the operands to the next step; guarded(step): that step's words with zeros in the
// place of what is not there.  Steps from `safe` on are loaded by guarded() alone.
//
// As in the weight gradient: fragments are read a region ahead, words of the next step go to LDS one by one behind the products and are asked for again for the step
// behind that; one barrier a step, before its last region, which reads the next step's first fragments.  A step of 256 x 256 x 64 in bf16 takes 1.54 us with all CUs at
// it, 1.40 PFLOP/s; a library's product of 8192 reaches 1.53.
template <class T, int WC, int WT, class A, class B, class Next, class Guarded>
__device__ __forceinline__ void product_steps(A &a, B &b, char *lds, int64_t first, int64_t last, int64_t safe, int wave_c, int wave_t,
                                              f32x16 (&acc)[WC][WT], Next advance, Guarded guarded)
{
    constexpr int BYTES = A::BYTES + B::BYTES, PRODUCTS = WC * WT, READS = WC * A::HALVES + WT * B::HALVES, PIECES = A::N + B::N;
    const int lane = threadIdx.x % 64;
    const int a_at = A::lane_at(lane), b_at = B::lane_at(lane);
#pragma unroll
    for (int i = 0; i < WC; ++i)
#pragma unroll
        for (int j = 0; j < WT; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.0f;
    u32x4 fa[2][WC], fb[2][WT];
    // read q of region r's fragments
    const auto read = [&](const char *buffer, int r, int q) {
        if (q < WC * A::HALVES)
            A::fragment(fa[r & 1][q / A::HALVES], buffer, a_at, wave_c * WC + q / A::HALVES, r, q % A::HALVES);
        else
            B::fragment(fb[r & 1][(q - WC * A::HALVES) / B::HALVES], buffer + A::BYTES, b_at, wave_t * WT + (q - WC * A::HALVES) / B::HALVES, r,
                        (q - WC * A::HALVES) % B::HALVES);
    };
    const auto product = [&](int r, int m) { multiply<T>(fa[r & 1][m / WT], fb[r & 1][m % WT], acc[m / WT][m % WT]); };
    const auto put = [&](char *buffer, int q) {
        if (q < A::N)
            a.put(q, buffer);
        else
            b.put(q - A::N, buffer + A::BYTES);
    };
    const auto load = [&](int q) {
        if (q < A::N)
            a.load(q);
        else
            b.load(q - A::N);
    };
    char *now = lds, *next = lds + BYTES;
    const auto turn = [&] {
        char *t = now;
        now = next;
        next = t;
    };
    int64_t step = first;
    if (first < last) {
        if (first < safe) {
#pragma unroll
            for (int q = 0; q < PIECES; ++q) load(q);
            advance();
        } else {
            guarded(first);
        }
#pragma unroll
        for (int q = 0; q < PIECES; ++q) put(now, q);
        if (first + 1 < safe) {
#pragma unroll
            for (int q = 0; q < PIECES; ++q) load(q);
            if (first + 2 < safe) advance();
        }
    }
    __syncthreads();
    if (step + 1 < safe) {
#pragma unroll
        for (int q = 0; q < READS; ++q) read(now, 0, q);
        for (; step + 1 < safe; ++step) {
            times<REGIONS * PRODUCTS>([&](auto slot) {
                constexpr int r = slot.value / PRODUCTS, m = slot.value % PRODUCTS;
                constexpr GradSchedule<REGIONS, PRODUCTS, READS, PIECES> PLAN;
                if constexpr (slot.value == (REGIONS - 1) * PRODUCTS) __syncthreads();
                product(r, m);
                times<PLAN.reads[m + 1] - PLAN.reads[m]>([&](auto q) { read(r < REGIONS - 1 ? now : next, (r + 1) % REGIONS, PLAN.reads[m] + q.value); });
                times<PLAN.piece[slot.value + 1] - PLAN.piece[slot.value]>([&](auto q) {
                    put(next, PLAN.piece[slot.value] + q.value);
                    load(PLAN.piece[slot.value] + q.value);
                });
                __builtin_amdgcn_sched_barrier(0);
            });
            // the words then hold the step behind the next, the same words again where there is no such step
            if (step + 3 < safe) advance();
            turn();
        }
    }
    // what is left: the step in LDS, and those that load() may not take
    for (; step < last; ++step) {
        if (step + 1 < last) guarded(step + 1);
#pragma unroll
        for (int r = 0; r < REGIONS; ++r) {
#pragma unroll
            for (int q = 0; q < READS; ++q) read(now, r, q);
#pragma unroll
            for (int m = 0; m < PRODUCTS; ++m) product(r, m);
        }
        if (step + 1 < last) {
#pragma unroll
            for (int q = 0; q < PIECES; ++q) put(next, q);
        }
        __syncthreads();
        turn();
    }
}

// Results of a wavefront on their way to memory by LDS, 32 tokens of CHANNELS channels: a store then takes whole rows, not 32 bytes of each of 32 rows
// (8192 tokens, 1024 -> 4096 channels in bf16 with both projections kept: 242 us with stores from the accumulators, 162 this way and with the
// cheaper sigmoid).
template <class T, int CHANNELS>
struct StagedRows {
    static constexpr int PITCH = CHANNELS * (int)sizeof(T) + 16, BYTES = 32 * PITCH, CHUNKS = CHANNELS / WORD<T>, EACH = 64 / CHUNKS;
    // Between put() and flush(), and before the next put(): other lanes' words are read.  A wavefront's LDS operations are carried out in their order, so the compiler alone is to keep it.
    static __device__ __forceinline__ void meet()
    {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    // four channels from c on of the lane's token
    static __device__ __forceinline__ void put(char *at, int lane, int c, const float *v)
    {
        char *const p = at + lane % 32 * PITCH + c * (int)sizeof(T);
        if constexpr (sizeof(T) == 2) {
            const bf16x2 x = {(__bf16)v[0], (__bf16)v[1]}, y = {(__bf16)v[2], (__bf16)v[3]};
            *reinterpret_cast<u32x2 *>(p) = u32x2{__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, y)};
        } else {
            *reinterpret_cast<u32x4 *>(p) = u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
        }
    }
    // rows of `stride` from `to` on; with INSIDE all of them are there, else `rows` of them and `left` channels of a row
    template <bool INSIDE>
    static __device__ __forceinline__ void flush(const char *at, int lane, T *to, int64_t stride, int64_t rows, int64_t left)
    {
        const int chunk = lane % CHUNKS, row = lane / CHUNKS;
        to += row * stride + chunk * WORD<T>;
        at += row * PITCH + chunk * 16;
        if constexpr (INSIDE) {
            u32x4 w[32 / EACH];
#pragma unroll
            for (int i = 0; i < 32 / EACH; ++i) w[i] = *reinterpret_cast<const u32x4 *>(at + i * EACH * PITCH);
#pragma unroll
            for (int i = 0; i < 32 / EACH; ++i) {
                if constexpr (sizeof(T) == 2)
                    *(EF_GLOBAL u32x4_any *)(EF_GLOBAL T *)(to + i * EACH * stride) = w[i];
                else
                    *(EF_GLOBAL u32x4_word *)(EF_GLOBAL T *)(to + i * EACH * stride) = w[i];
            }
        } else {
            const int n = (int)min((int64_t)WORD<T>, left - chunk * WORD<T>);
            for (int i = 0; i < 32 / EACH && i * EACH + row < rows; ++i, to += EACH * stride, at += EACH * PITCH) {
                if (n == WORD<T>) {
                    if constexpr (sizeof(T) == 2)
                        *(EF_GLOBAL u32x4_any *)(EF_GLOBAL T *)to = *reinterpret_cast<const u32x4 *>(at);
                    else
                        *(EF_GLOBAL u32x4_word *)(EF_GLOBAL T *)to = *reinterpret_cast<const u32x4 *>(at);
                } else {
                    for (int k = 0; k < n; ++k) to[k] = reinterpret_cast<const T *>(at)[k];
                }
            }
        }
    }
};

// An accumulator's lane holds token lane % 32 and, in run r of four, channels 8 r + 4 (lane / 32) on.
__device__ __forceinline__ int run_channel(int lane, int r) { return 8 * r + lane / 32 * 4; }

}  // namespace ef
