// Weight gradient of a linear layer from its input's checkpoint, dw[o][i] = s[i] * sum_t dz[t][o] * x[t][i], on matrix instructions.
//
// What a checkpoint stands for is a bf16 number exactly (the scales are powers of two), so the product runs on bf16 matrix
// instructions with nothing lost but fp32's own rounding of the sums; an fp32 gradient enters as three bf16 numbers, which are its 24 bits.
//
// A workgroup of four wavefronts makes a square tile of dw of 64 SIDE channels, a quarter each: with SIDE = 4 256 x 256, 256 accumulators a lane.
// Both operands lie in memory with the tokens as the slow index, and the instruction wants eight tokens of one channel in a lane: the tiles
// are kept in LDS as they lie in memory, codes already decoded, and read transposed (four tokens by 16 channels to a read).  From a token's channels to
// the next token's are 64 bytes more than they take, so that the four tokens of a read fall on different banks.
#pragma once
#include "ef_rows.h"

namespace ef {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int GRAD_THREADS = 256;
constexpr int GRAD_ROWS = 128;          // tokens' rows in an LDS buffer: dz's (three to a token in fp32), then x's

// Tokens in a step, bf16 parts of an element of dz.
template <class T>
struct GradStep;
template <>
struct GradStep<bf16_t> { static constexpr int TOKENS = 64, PARTS = 1; };
template <>
struct GradStep<float> { static constexpr int TOKENS = 32, PARTS = 3; };

struct GradArgs {
    int64_t rows, out, n;
    const void *dz;
    int64_t dz_stride;
    ActRef act;
    const float *scale;
    float *dw;
    int accumulate;
    int tiles, tiles_n;                 // in all, and in a row of them
    // The last tiles, from `whole` on, are cut into `splits` parts along the tokens, a workgroup each; their sums go to `parts`, tile by tile, and
    // k_join_splits adds them up.
    int whole, splits;
    float *parts;
    int64_t steps;                      // of the tokens
};

// An fp32 number is the sum of three bf16 ones: its upper half, that of what is left, and the rest, each cut off, not rounded.  Of an infinity or NaN
// nothing is left (fmaxf takes a number over NaN; a NaN is one in its upper half, as arithmetic makes them).
__device__ __forceinline__ float upper(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }
__device__ __forceinline__ float cut_off(float v) { return copysignf(fmaxf(fabsf(v - upper(v)), 0.0f), v); }
__device__ __forceinline__ unsigned uppers(unsigned lo, unsigned hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }

// What a thread carries from memory to LDS for one step.  load() masks nothing: channels past the operands' ends hold whatever lies there, and what they
// give is not stored; steps whose reads could pass the end of dz are loaded by load_guarded().
template <class T, int SIDE>
struct GradStage {
    // Steps on their way at a time: a step of a small tile takes less than its loads.
    static constexpr int DEPTH = SIDE == 4 ? 1 : (SIDE == 2 ? 2 : 3);
    static constexpr int TOKENS = GradStep<T>::TOKENS, PARTS = GradStep<T>::PARTS, TILE = 64 * SIDE, PITCH = TILE * 2 + 64;
    static constexpr int Z_ELEMS = 16 / (int)sizeof(T), Z_WORDS = TILE / Z_ELEMS, Z_ROWS = GRAD_THREADS / Z_WORDS, Z = TOKENS / Z_ROWS;
    static constexpr int X_WORDS = TILE / 16, X_ROWS = GRAD_THREADS / X_WORDS < TOKENS ? GRAD_THREADS / X_WORDS : TOKENS, X = TOKENS / X_ROWS;
    u32x4 z[DEPTH][Z], x[DEPTH][X];
    unsigned s[DEPTH][X];
    // Where the step to load next begins, the same for the whole workgroup, and the bytes from there of each of this thread's words: a load adds the two
    // itself, and nothing but the three bases changes from step to step.  In global memory: a load that might be LDS's would have every LDS
    // read waited for.
    const EF_GLOBAL char *z_base;
    const EF_GLOBAL uint8_t *x_base, *s_base;
    unsigned z_off[Z], x_off[X], s_off[X];

    // the thread's place in a step's words of dz and of codes (threads beyond X_ROWS rows of codes do what others do)
    static __device__ __forceinline__ int z_row() { return threadIdx.x / Z_WORDS; }
    static __device__ __forceinline__ int x_row() { return threadIdx.x / X_WORDS % X_ROWS; }
    static __device__ __forceinline__ int z_word() { return threadIdx.x % Z_WORDS; }
    static __device__ __forceinline__ int x_word() { return threadIdx.x % X_WORDS; }

    __device__ __forceinline__ void begin(const GradArgs &a, int64_t token0, int64_t o0, int64_t n0)
    {
        const int64_t o = o0 + z_word() * Z_ELEMS, i = n0 + x_word() * 16;
        z_base = (const EF_GLOBAL char *)a.dz + token0 * a.dz_stride * (int64_t)sizeof(T);
        x_base = (const EF_GLOBAL uint8_t *)a.act.code_at(token0, 0);
        s_base = (const EF_GLOBAL uint8_t *)a.act.scale_at(token0, 0);
        // channels past the ends are read from the first ones
#pragma unroll
        for (int k = 0; k < Z; ++k) z_off[k] = (unsigned)(((z_row() + k * Z_ROWS) * a.dz_stride + (o < a.out ? o : 0)) * (int64_t)sizeof(T));
#pragma unroll
        for (int k = 0; k < X; ++k) {
            x_off[k] = (unsigned)((x_row() + k * X_ROWS) * a.act.groups * GROUP + (i < a.act.groups * GROUP ? i : 0));
            s_off[k] = (unsigned)((x_row() + k * X_ROWS) * a.act.groups + (i < a.act.groups * GROUP ? i / GROUP : 0));
        }
    }
    // The first step that load() may not take: a token's last word may reach Z_ELEMS - 1 elements past its row, and the offsets have to fit 32 bits.
    static __device__ __forceinline__ int64_t unsafe(const GradArgs &a, int64_t o0)
    {
        if (a.dz_stride > (int64_t)1 << 24) return 0;
        const int64_t spare = o0 + TILE <= a.out ? 0 : (Z_ELEMS - 1 + a.dz_stride - 1) / a.dz_stride;
        return max((int64_t)0, a.rows - spare) / TOKENS;
    }
    __device__ __forceinline__ void load_z(const GradArgs &a, int d, int k)
    {
        stay(z_off[k]);
        const EF_GLOBAL char *p = z_base + z_off[k];
        if constexpr (sizeof(T) == 2)
            z[d][k] = *(const EF_GLOBAL u32x4_any *)p;
        else
            z[d][k] = *(const EF_GLOBAL u32x4_word *)p;
    }
    __device__ __forceinline__ void load_x(const GradArgs &a, int d, int k)
    {
        stay(x_off[k]);
        stay(s_off[k]);
        x[d][k] = *(const EF_GLOBAL u32x4 *)(x_base + x_off[k]);
        s[d][k] = *(s_base + s_off[k]);
    }
    __device__ __forceinline__ void load(const GradArgs &a, int d)
    {
#pragma unroll
        for (int k = 0; k < Z; ++k) load_z(a, d, k);
#pragma unroll
        for (int k = 0; k < X; ++k) load_x(a, d, k);
    }
    __device__ __forceinline__ void next(const GradArgs &a)
    {
        z_base += TOKENS * a.dz_stride * (int64_t)sizeof(T);
        x_base += TOKENS * a.act.groups * GROUP;
        s_base += TOKENS * a.act.groups;
    }

    // The step at token0 with zeros in the place of what is not there: whole words where a row has them, else element by element.  All loads are
    // on their way before the first is used.
    __device__ __forceinline__ void load_guarded(const GradArgs &a, int d, int64_t token0, int64_t o0, int64_t n0)
    {
        const int64_t o = o0 + z_word() * Z_ELEMS, i = n0 + x_word() * 16, end = a.rows - 1;
        const EF_GLOBAL T *dz = (const EF_GLOBAL T *)a.dz;
        if (o + Z_ELEMS <= a.out) {
#pragma unroll
            for (int k = 0; k < Z; ++k) {
                const EF_GLOBAL T *p = dz + min(token0 + z_row() + k * Z_ROWS, end) * a.dz_stride + o;
                if constexpr (sizeof(T) == 2)
                    z[d][k] = *(const EF_GLOBAL u32x4_any *)p;
                else
                    z[d][k] = *(const EF_GLOBAL u32x4_word *)p;
            }
        } else if (o < a.out) {
#pragma unroll
            for (int k = 0; k < Z; ++k) {
                const EF_GLOBAL T *p = dz + min(token0 + z_row() + k * Z_ROWS, end) * a.dz_stride;
                unsigned e[Z_ELEMS];
#pragma unroll
                for (int j = 0; j < Z_ELEMS; ++j) {
                    if constexpr (sizeof(T) == 2)
                        e[j] = *(const EF_GLOBAL uint16_t *)(p + min(o + j, a.out - 1));
                    else
                        e[j] = *(const EF_GLOBAL unsigned *)(p + min(o + j, a.out - 1));
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (sizeof(T) == 2)
                        z[d][k][j] = e[2 * j] | e[2 * j + 1] << 16;
                    else
                        z[d][k][j] = e[j];
                }
            }
        }
        const bool there = i < a.act.groups * GROUP;
        const EF_GLOBAL uint8_t *codes = (const EF_GLOBAL uint8_t *)a.act.codes, *scales = (const EF_GLOBAL uint8_t *)a.act.scales;
#pragma unroll
        for (int k = 0; k < X; ++k) {
            const int64_t t = min(token0 + x_row() + k * X_ROWS, end);
            x[d][k] = *(const EF_GLOBAL u32x4 *)(codes + t * a.act.groups * GROUP + (there ? i : 0));
            s[d][k] = scales[t * a.act.groups + (there ? i / GROUP : 0)];
        }
#pragma unroll
        for (int k = 0; k < Z; ++k)
            if (o >= a.out || token0 + z_row() + k * Z_ROWS > end) z[d][k] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < X; ++k)
            if (!there || token0 + x_row() + k * X_ROWS > end) {
                x[d][k] = u32x4{0, 0, 0, 0};
                s[d][k] = SCALE_MIN;
            }
    }

    // What is carried goes to LDS in pieces of about four instructions, as many as hide behind one product; where RELOAD is set, each word's last piece
    // asks for the next step's.  A word of bf16: one piece.  A word of codes: four.  A word of fp32: its elements' second parts, the third ones two at
    // a time, then a part of all four to LDS at a time.
    static constexpr int Z_PIECES = sizeof(T) == 2 ? 1 : 9, X_PIECES = 4;
    static constexpr int PIECES = Z * Z_PIECES + X * X_PIECES;
    float rest[sizeof(T) == 2 ? 1 : 4];
    unsigned third[sizeof(T) == 2 ? 1 : 4];
    u32x2 held;
    template <int Q, bool RELOAD>
    __device__ __forceinline__ void piece(const GradArgs &a, int d, char *buffer)
    {
        if constexpr (Q < Z * Z_PIECES) {
            constexpr int k = Q / Z_PIECES, part = Q % Z_PIECES;
            char *at = buffer + (z_row() + k * Z_ROWS) * PITCH + z_word() * (2 * Z_ELEMS);
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<u32x4 *>(at) = z[d][k];
                if (RELOAD) load_z(a, d, k);
            } else if constexpr (part < 4) {
                rest[part] = cut_off(__uint_as_float(z[d][k][part]));
            } else if constexpr (part < 6) {
#pragma unroll
                for (int e = 2 * (part - 4); e < 2 * (part - 4) + 2; ++e) third[e] = __float_as_uint(rest[e] - upper(rest[e]));
            } else if constexpr (part == 6) {
                *reinterpret_cast<u32x2 *>(at) = u32x2{uppers(z[d][k][0], z[d][k][1]), uppers(z[d][k][2], z[d][k][3])};
                if (RELOAD) load_z(a, d, k);
            } else if constexpr (part == 7) {
                *reinterpret_cast<u32x2 *>(at + TOKENS * PITCH) =
                    u32x2{uppers(__float_as_uint(rest[0]), __float_as_uint(rest[1])), uppers(__float_as_uint(rest[2]), __float_as_uint(rest[3]))};
            } else {
                *reinterpret_cast<u32x2 *>(at + 2 * TOKENS * PITCH) = u32x2{uppers(third[0], third[1]), uppers(third[2], third[3])};
            }
        } else {
            constexpr int k = (Q - Z * Z_PIECES) / X_PIECES, part = (Q - Z * Z_PIECES) % X_PIECES, h = part / 2;
            const float scale = scale_value(s[d][k]);
            if constexpr (part % 2 == 0) {
                held = decode_four(x[d][k][2 * h], scale);
            } else {
                const u32x2 more = decode_four(x[d][k][2 * h + 1], scale);
                char *at = buffer + (PARTS * TOKENS + x_row() + k * X_ROWS) * PITCH + x_word() * 32;
                *reinterpret_cast<u32x4 *>(at + 16 * h) = u32x4{held.x, held.y, more.x, more.y};
                if constexpr (h == 1 && RELOAD) load_x(a, d, k);
            }
        }
    }
};

// Eight tokens of a channel to a lane, in two reads of four: lane l gets channel l % 32 and tokens l / 32 * 8 + 0..7 of the 32 channels x 16
// tokens at p (p: the lane's own place, see grad_lane_offset).
struct Fragment {
    s16x4 half[2];
    template <int PITCH>
    __device__ __forceinline__ void read(const char *p, int h)
    {
        typedef __attribute__((address_space(3))) s16x4 shared_s16x4;
        half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared_s16x4 *)(p + h * 4 * PITCH));
    }
    __device__ __forceinline__ bf16x8 whole() const
    {
        return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
};
// 16 lanes read four tokens x 16 channels, lane i of them four channels of token i / 4 (and get four tokens of channel i).
__device__ __forceinline__ int grad_lane_offset(int lane, int pitch)
{
    const int block = lane / 16, i = lane % 16;
    return ((block >> 1) * 8 + i / 4) * pitch + ((block & 1) * 16 + i % 4 * 4) * 2;
}

// What follows product m of region r of a step (a region: the products on one set of fragments): the pieces from piece[PRODUCTS r + m] on up to the next
// entry, and the halves reads[m] .. reads[m + 1] of the next region's fragments, all on their way when three quarters of the products are.
template <int REGIONS, int PRODUCTS, int HALVES, int PIECES>
struct GradSchedule {
    int piece[REGIONS * PRODUCTS + 1] = {}, reads[PRODUCTS + 1] = {};
    constexpr GradSchedule()
    {
        constexpr int SLOTS = (REGIONS - 1) * PRODUCTS, EARLY = PRODUCTS > 1 ? PRODUCTS * 3 / 4 : 1;
        for (int k = 0; k <= REGIONS * PRODUCTS; ++k) piece[k] = k < SLOTS ? k * PIECES / SLOTS : PIECES;
        for (int m = 0; m <= PRODUCTS; ++m) reads[m] = m < EARLY ? (m * HALVES + EARLY - 1) / EARLY : HALVES;
    }
};

// A step is REGIONS sets of SIDE x SIDE products a wavefront.  With SIDE = 4 there is one wavefront to a SIMD: what it does besides products has to
// hide behind them, about four instructions of 4 to 6 cycles to a product's 32 (measured: one more costs its own time).  So with SIDE = 4 and 2
// everything is given its place (GradSchedule): fragments are read a region ahead, words of the next step go to LDS piece by piece, and words of a later
// step are asked for as the registers get free; one barrier a step.  SIDE = 4 runs at 1.37 PFLOP/s over 16384 tokens of 4096 x 4096, what a
// library's bf16 product of 16384 reaches here, the clock being the power's; SIDE = 2 has 110 instructions beside 16 products and is bound by issuing
// them.  Tiles of 64 have several workgroups on a CU that hide one another's waits.
template <class T, int SIDE>
__global__ __launch_bounds__(GRAD_THREADS, SIDE == 4 ? 1 : 2) void k_weight_grad(GradArgs a)
{
    using Stage = GradStage<T, SIDE>;
    constexpr int TOKENS = Stage::TOKENS, PARTS = Stage::PARTS, TILE = Stage::TILE, PITCH = Stage::PITCH, REGIONS = TOKENS / 16 * PARTS;
    constexpr int PRODUCTS = SIDE * SIDE, HALVES = 4 * SIDE;
    constexpr bool PLANNED = SIDE >= 2;
    __shared__ __align__(16) char buffers[2][GRAD_ROWS * PITCH];
    // Workgroups go to the eight XCDs in turn: each XCD takes a run of neighbouring tiles, which share rows of dz in its L2.
    const auto in_runs = [](int id, int all) { return id % 8 * (all / 8) + min(id % 8, all % 8) + id / 8; };
    int tile, split = 0, splits = 1;
    if ((int)blockIdx.x < a.whole) {
        tile = in_runs(blockIdx.x, a.whole);
    } else {
        const int cut = a.tiles - a.whole, id = in_runs(blockIdx.x - a.whole, cut * a.splits);
        splits = a.splits;
        split = id / cut;
        tile = a.whole + id % cut;
    }
    const int64_t o0 = (int64_t)(tile / a.tiles_n) * TILE, n0 = (int64_t)(tile % a.tiles_n) * TILE;
    const int64_t first = a.steps * split / splits, last = a.steps * (split + 1) / splits, safe = min(last, Stage::unsafe(a, o0));

    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int z_at = grad_lane_offset(lane, PITCH) + wave / 2 * TILE;
    const int x_at = grad_lane_offset(lane, PITCH) + wave % 2 * TILE + PARTS * TOKENS * PITCH;
    f32x16 acc[SIDE][SIDE];
#pragma unroll
    for (int i = 0; i < SIDE; ++i)
#pragma unroll
        for (int j = 0; j < SIDE; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.0f;

    Fragment z[2][SIDE], x[2][SIDE];
    // Half h of region r's fragments, x's first; those only where a region begins with another sixteen tokens.
    auto fragment = [&](const char *buffer, int r, int h) {
        const int k = r / PARTS, p = r % PARTS, f = h / 2;
        if (f < SIDE) {
            if (p == 0) x[k & 1][f].template read<PITCH>(buffer + x_at + k * 16 * PITCH + f * 64, h % 2);
        } else {
            z[r & 1][f - SIDE].template read<PITCH>(buffer + z_at + (p * TOKENS + k * 16) * PITCH + (f - SIDE) * 64, h % 2);
        }
    };
    auto product = [&](int r, int i, int j) {
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(z[r & 1][i].whole(), x[r / PARTS & 1][j].whole(), acc[i][j], 0, 0, 0);
    };
    char *now = buffers[0], *next = buffers[1];
    auto turn = [&] {
        char *t = now;
        now = next;
        next = t;
    };
    Stage stage;
    int64_t step = first;
    stage.begin(a, first * TOKENS, o0, n0);
    auto fetch = [&](int64_t q, int d) {
        if (q < safe) {
            stage.load(a, d);
            stage.next(a);
        } else if (q < last) {
            stage.load_guarded(a, d, q * TOKENS, o0, n0);
        }
    };
    auto put = [&](int d, char *buffer) { times<Stage::PIECES>([&](auto q) { stage.template piece<q.value, false>(a, d, buffer); }); };
    if (first < last) {
        fetch(first, 0);
        put(0, now);
        // the sets of words then hold the steps behind it, the same words again where there is no such step
        if constexpr (PLANNED) {
            if (first + 1 < safe) {
#pragma unroll
                for (int d = 1; d <= Stage::DEPTH; ++d) {
                    stage.load(a, d % Stage::DEPTH);
                    if (first + d + 1 < safe) stage.next(a);
                }
            }
        } else {
#pragma unroll
            for (int d = 1; d < Stage::DEPTH; ++d) fetch(first + d, d);
        }
    }
    __syncthreads();
    if constexpr (PLANNED) {
        if (step + 1 < safe) {
#pragma unroll
            for (int h = 0; h < HALVES; ++h) fragment(now, 0, h);
            // Behind the products of all regions but a step's last, pieces of the next step go to LDS and the next region's fragments are read.  The last
            // region begins with the barrier and reads the next step's first fragments.
            auto planned = [&](auto d) {
                times<REGIONS * PRODUCTS>([&](auto slot) {
                    constexpr int r = slot.value / PRODUCTS, m = slot.value % PRODUCTS, set = (d.value + 1) % Stage::DEPTH;
                    constexpr GradSchedule<REGIONS, PRODUCTS, HALVES, Stage::PIECES> PLAN;
                    if constexpr (slot.value == (REGIONS - 1) * PRODUCTS) __syncthreads();
                    product(r, m / SIDE, m % SIDE);
                    times<PLAN.reads[m + 1] - PLAN.reads[m]>(
                        [&](auto h) { fragment(r < REGIONS - 1 ? now : next, (r + 1) % REGIONS, PLAN.reads[m] + h.value); });
                    times<PLAN.piece[slot.value + 1] - PLAN.piece[slot.value]>(
                        [&](auto q) { stage.template piece<PLAN.piece[slot.value] + q.value, true>(a, set, next); });
                    __builtin_amdgcn_sched_barrier(0);
                });
                if (step + Stage::DEPTH + 2 < safe) stage.next(a);
                turn();
                ++step;
            };
            // whole turns of the sets without a look at the end, then the rest
            while (step + Stage::DEPTH < safe) times<Stage::DEPTH>(planned);
            times<Stage::DEPTH - 1>([&](auto d) {
                if (step + 1 < safe) planned(d);
            });
        }
    }
    auto products = [&] {
#pragma unroll
        for (int r = 0; r < REGIONS; ++r) {
#pragma unroll
            for (int h = 0; h < HALVES; ++h) fragment(now, r, h);
#pragma unroll
            for (int m = 0; m < PRODUCTS; ++m) product(r, m / SIDE, m % SIDE);
        }
    };
    if constexpr (PLANNED) {
        // what is left: the step in LDS, and those that load() may not take
        for (; step < last; ++step) {
            if (step + 1 < last) stage.load_guarded(a, 0, (step + 1) * TOKENS, o0, n0);
            products();
            if (step + 1 < last) put(0, next);
            __syncthreads();
            turn();
        }
    } else {
        // without a branch: behind one, a wait for a load would be a wait for all behind it too
        for (; step + 2 * Stage::DEPTH <= safe; step += Stage::DEPTH) {
            times<Stage::DEPTH>([&](auto d) {
                stage.load(a, d.value);
                stage.next(a);
                products();
                put((d.value + 1) % Stage::DEPTH, next);
                __syncthreads();
                turn();
            });
        }
        for (; step < last; step += Stage::DEPTH) {
            times<Stage::DEPTH>([&](auto d) {
                if (step + d.value >= last) return;
                fetch(step + d.value + Stage::DEPTH, d.value);
                products();
                if (step + d.value + 1 < last) put((d.value + 1) % Stage::DEPTH, next);
                __syncthreads();
                turn();
            });
        }
    }

    // An accumulator's lane holds channel lane % 32 of x's side and four runs of four of dz's.
    const int r0 = wave / 2 * (TILE / 2) + 4 * (lane / 32), c0 = wave % 2 * (TILE / 2) + lane % 32;
    if ((int)blockIdx.x >= a.whole) {
        float *const at = a.parts + ((int64_t)(tile - a.whole) * splits + split) * (TILE * TILE) + r0 * TILE + c0;
#pragma unroll
        for (int i = 0; i < SIDE; ++i)
#pragma unroll
            for (int j = 0; j < SIDE; ++j)
#pragma unroll
                for (int k = 0; k < 16; ++k) at[(i * 32 + 8 * (k / 4) + k % 4) * TILE + j * 32] = acc[i][j][k];
        return;
    }
    float *const dw = a.dw + (o0 + r0) * a.n;
    const int64_t left = a.out - (o0 + r0);
#pragma unroll
    for (int j = 0; j < SIDE; ++j) {
        const int64_t c = n0 + c0 + j * 32;
        if (c >= a.n) continue;
        const float s = a.scale ? a.scale[c] : 1.0f;
#pragma unroll
        for (int i = 0; i < SIDE; ++i) {
            float v[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = acc[i][j][k] * s;
            float *const at = dw + i * 32 * a.n + c;
            if (a.accumulate) {
                float old[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) old[k] = i * 32 + 8 * (k / 4) + k % 4 < left ? at[(8 * (k / 4) + k % 4) * a.n] : 0.0f;
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] += old[k];
            }
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (i * 32 + 8 * (k / 4) + k % 4 < left) at[(8 * (k / 4) + k % 4) * a.n] = v[k];
        }
    }
}

// dw <- [dw +] scale * the sum of the splits' results, in their order: four neighbouring channels to a thread.
template <int TILE>
__global__ __launch_bounds__(256) void k_join_splits(GradArgs a)
{
    constexpr int EACH = TILE * TILE / 4 / 256;         // workgroups to a tile
    const int cut = blockIdx.x / EACH, tile = a.whole + cut, at = (blockIdx.x % EACH * 256 + threadIdx.x) * 4;
    const int64_t o = (int64_t)(tile / a.tiles_n) * TILE + at / TILE, i = (int64_t)(tile % a.tiles_n) * TILE + at % TILE;
    if (o >= a.out || i >= a.n) return;
    const float *from = a.parts + (int64_t)cut * a.splits * (TILE * TILE) + at;
    float v[4] = {};
    for (int p = 0; p < a.splits; p += 8) {
        u32x4 w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (p + k < a.splits) w[k] = *reinterpret_cast<const u32x4 *>(from + (int64_t)(p + k) * (TILE * TILE));
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (p + k < a.splits) {
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] += __uint_as_float(w[k][c]);
            }
    }
    float *dw = a.dw + o * a.n + i;
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (i + c < a.n) {
            const float s = a.scale ? v[c] * a.scale[i + c] : v[c];
            dw[c] = a.accumulate ? dw[c] + s : s;
        }
}

}  // namespace ef
