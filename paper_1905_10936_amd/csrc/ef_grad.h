// Weight gradient of a linear layer from its input's checkpoint, dw[o][i] = s[i] * sum_t dz[t][o] * x[t][i], on matrix instructions.
//
// What a checkpoint stands for is a bf16 number exactly (the scales are powers of two), so the product runs on bf16 matrix
// instructions with nothing lost but fp32's own rounding of the sums; an fp32 gradient enters as three bf16 numbers, which are its 24 bits.
//
// A workgroup of four wavefronts makes a tile of 256 x 256 of dw, 128 x 128 to a wavefront in 256 accumulators a lane: per product
// step of 16 tokens a wavefront reads 8 KiB from LDS for 16 instructions of 32 cycles, 64 of the 128 bytes a cycle that LDS gives.
// Both operands lie in memory with the tokens as the slow index, and the instruction wants eight tokens of one channel in a lane: the
// tiles are kept in LDS as they lie in memory and read transposed (four tokens by 16 channels to a read).  Rows of a tile are
// 576 bytes apart, so that the four tokens of two neighbouring reads fall on different banks.
#pragma once
#include "ef_rows.h"

namespace ef {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int GRAD_THREADS = 256;
constexpr int GRAD_TILE = 256;          // channels of either side
constexpr int GRAD_PITCH = 576;         // bytes from a token's channels to the next one's in LDS
constexpr int GRAD_ROWS = 128;          // such rows in a buffer: dz's, then x's

struct GradArgs {
    int64_t rows, out, n;
    const void *dz;
    int64_t dz_stride;
    ActRef act;
    const float *scale;
    float *dw;                          // or the partial results, [splits][out][n]
    int accumulate;
    int tiles_out, tiles_n;
    int splits;
    int64_t steps;                      // product steps in all; a split takes an equal share of them
};

// Tokens in a step: dz takes one row of LDS a token in bf16 and three in fp32.
template <class T>
struct GradStep;
template <>
struct GradStep<bf16_t> { static constexpr int TOKENS = 64, PARTS = 1; };
template <>
struct GradStep<float> { static constexpr int TOKENS = 32, PARTS = 3; };

// The three bf16 numbers whose sum a finite fp32 number is, each cut off, not rounded; an infinity is its own first part.
struct ThreeParts { unsigned a, b, c; };        // in the upper halves
__device__ __forceinline__ ThreeParts three_parts(float v)
{
    ThreeParts p;
    p.a = __float_as_uint(v) & 0xffff0000u;
    float rest = v - __uint_as_float(p.a);
    if (__float_as_uint(v) << 1 == 0xff000000u) rest = 0.0f;
    p.b = __float_as_uint(rest) & 0xffff0000u;
    rest -= __uint_as_float(p.b);
    p.c = __float_as_uint(rest) & 0xffff0000u;
    return p;
}

// What a thread carries from memory to LDS for one step.
template <class T>
struct GradStage {
    static constexpr int TOKENS = GradStep<T>::TOKENS, PARTS = GradStep<T>::PARTS;
    static constexpr int Z = TOKENS * GRAD_TILE * (int)sizeof(T) / 16 / GRAD_THREADS;   // 128-bit words of dz: 8
    static constexpr int X = TOKENS * GRAD_TILE / 16 / GRAD_THREADS;                    // of codes: 4 or 2
    u32x4 z[Z], x[X];
    unsigned s[X];

    static constexpr int Z_WORDS = GRAD_TILE * (int)sizeof(T) / 16;     // words a token
    static constexpr int Z_ELEMS = 16 / (int)sizeof(T);

    __device__ __forceinline__ void load(const GradArgs &a, int64_t token0, int64_t o0, int64_t n0)
    {
        const int tid = threadIdx.x;
        const int64_t o = o0 + tid % Z_WORDS * Z_ELEMS;
#pragma unroll
        for (int k = 0; k < Z; ++k) {
            const int64_t t = token0 + tid / Z_WORDS + k * (GRAD_THREADS / Z_WORDS);
            const T *p = static_cast<const T *>(a.dz) + t * a.dz_stride + o;
            z[k] = u32x4{0, 0, 0, 0};
            if (t < a.rows) {
                if (o + Z_ELEMS <= a.out) {
                    if constexpr (sizeof(T) == 2)
                        z[k] = *reinterpret_cast<const u32x4_any *>(p);
                    else
                        z[k] = *reinterpret_cast<const u32x4_word *>(p);
                } else {
#pragma unroll
                    for (int i = 0; i < Z_ELEMS - 1; ++i)
                        if (o + i < a.out) {
                            const unsigned b = element_bits(p + i);
                            if constexpr (sizeof(T) == 2)
                                z[k][i / 2] |= i & 1 ? b << 16 : b;
                            else
                                z[k][i] = b;
                        }
                }
            }
        }
        const int64_t i = n0 + tid % 16 * 16;
#pragma unroll
        for (int k = 0; k < X; ++k) {
            const int64_t t = token0 + tid / 16 + k * (GRAD_THREADS / 16);
            x[k] = u32x4{0, 0, 0, 0};
            s[k] = SCALE_MIN;
            if (t < a.rows && i < a.act.groups * GROUP) {
                x[k] = *reinterpret_cast<const u32x4 *>(a.act.code_at(t, i));
                s[k] = *a.act.scale_at(t, i);
            }
        }
    }

    __device__ __forceinline__ void store(char *buffer) const
    {
        const int tid = threadIdx.x;
#pragma unroll
        for (int k = 0; k < Z; ++k) {
            const int t = tid / Z_WORDS + k * (GRAD_THREADS / Z_WORDS);
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<u32x4 *>(buffer + t * GRAD_PITCH + tid % Z_WORDS * 16) = z[k];
            } else {
                ThreeParts p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = three_parts(__uint_as_float(z[k][i]));
                char *at = buffer + t * GRAD_PITCH + tid % Z_WORDS * 8;
                *reinterpret_cast<u32x2 *>(at) = u32x2{p[0].a >> 16 | p[1].a, p[2].a >> 16 | p[3].a};
                *reinterpret_cast<u32x2 *>(at + TOKENS * GRAD_PITCH) = u32x2{p[0].b >> 16 | p[1].b, p[2].b >> 16 | p[3].b};
                *reinterpret_cast<u32x2 *>(at + 2 * TOKENS * GRAD_PITCH) = u32x2{p[0].c >> 16 | p[1].c, p[2].c >> 16 | p[3].c};
            }
        }
        char *const xs = buffer + PARTS * TOKENS * GRAD_PITCH;
#pragma unroll
        for (int k = 0; k < X; ++k) {
            const int t = tid / 16 + k * (GRAD_THREADS / 16);
            const float scale = scale_value(s[k]);
            u32x4 w[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x2 lo = decode_four(x[k][2 * h], scale), hi = decode_four(x[k][2 * h + 1], scale);
                w[h] = u32x4{lo.x, lo.y, hi.x, hi.y};
            }
            char *at = xs + t * GRAD_PITCH + tid % 16 * 32;
            *reinterpret_cast<u32x4 *>(at) = w[0];
            *reinterpret_cast<u32x4 *>(at + 16) = w[1];
        }
    }
};

// Eight tokens of a channel to a lane: lane l gets channel l % 32 and tokens l / 32 * 8 + 0..7 of the 32 channels x 16 tokens at p (p: the
// lane's own place, see grad_lane_offset).
__device__ __forceinline__ bf16x8 read_transposed(const char *p)
{
    typedef __attribute__((address_space(3))) s16x4 shared_s16x4;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared_s16x4 *)(p));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared_s16x4 *)(p + 4 * GRAD_PITCH));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
// 16 lanes read four tokens x 16 channels, lane i of them four channels of token i / 4 (and get four tokens of channel i).
__device__ __forceinline__ int grad_lane_offset(int lane)
{
    const int block = lane / 16, i = lane % 16;
    return ((block >> 1) * 8 + i / 4) * GRAD_PITCH + ((block & 1) * 16 + i % 4 * 4) * 2;
}

template <class T>
__global__ __launch_bounds__(GRAD_THREADS, 1) void k_weight_grad(GradArgs a)
{
    constexpr int TOKENS = GradStep<T>::TOKENS, PARTS = GradStep<T>::PARTS;
    __shared__ __align__(16) char buffers[2][GRAD_ROWS * GRAD_PITCH];
    // Workgroups go to the eight XCDs in turn: each XCD takes a run of neighbouring tiles, which share rows of dz in its L2.
    const int n_tiles = a.tiles_out * a.tiles_n, all = n_tiles * a.splits;
    int id = blockIdx.x;
    {
        const int per = all / 8, more = all % 8, xcd = id % 8, k = id / 8;
        id = xcd * per + min(xcd, more) + k;
    }
    const int split = id / n_tiles, tile = id % n_tiles;
    const int64_t o0 = (int64_t)(tile / a.tiles_n) * GRAD_TILE, n0 = (int64_t)(tile % a.tiles_n) * GRAD_TILE;
    const int64_t first = a.steps * split / a.splits, last = a.steps * (split + 1) / a.splits;

    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int z_at = grad_lane_offset(lane) + wave / 2 * 256;
    const int x_at = grad_lane_offset(lane) + wave % 2 * 256 + PARTS * TOKENS * GRAD_PITCH;
    f32x16 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.0f;

    if (first < last) {
        GradStage<T> stage;
        stage.load(a, first * TOKENS, o0, n0);
        stage.store(buffers[0]);
        stage.load(a, (first + 1) * TOKENS, o0, n0);        // past the last token: zeros, nothing is read
        __syncthreads();
        for (int64_t step = first; step < last; ++step) {
            const char *now = buffers[(step - first) & 1];
            if (step + 1 < last) {
                stage.store(buffers[(step - first + 1) & 1]);
                stage.load(a, (step + 2) * TOKENS, o0, n0);
            }
#pragma unroll
            for (int k = 0; k < TOKENS / 16; ++k) {
                bf16x8 x[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = read_transposed(now + x_at + k * 16 * GRAD_PITCH + j * 64);
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    bf16x8 z[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[i] = read_transposed(now + z_at + (p * TOKENS + k * 16) * GRAD_PITCH + i * 64);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(z[i], x[j], acc[i][j], 0, 0, 0);
                }
            }
            __syncthreads();
        }
    }

    float *dw = a.dw + (a.splits > 1 ? (int64_t)split * a.out * a.n : 0);
    const bool whole = a.splits == 1;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t i = n0 + wave % 2 * 128 + j * 32 + lane % 32;
        if (i >= a.n) continue;
        const float s = whole && a.scale ? a.scale[i] : 1.0f;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int64_t o = o0 + wave / 2 * 128 + m * 32 + 8 * (k / 4) + 4 * (lane / 32) + k % 4;
                if (o < a.out) {
                    float *at = dw + o * a.n + i;
                    float v = acc[m][j][k] * s;
                    if (whole && a.accumulate) v += *at;
                    *at = v;
                }
            }
        }
    }
}

// dw <- [dw +] scale * the sum of the splits' results, in their order.
__global__ __launch_bounds__(256) void k_join_splits(const float *parts, int splits, int64_t out, int64_t n, const float *scale, float *dw,
                                                     int accumulate)
{
    const int64_t total = out * n;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < total; at += (int64_t)gridDim.x * 256) {
        float s = parts[at];
        for (int p = 1; p < splits; ++p) s += parts[(int64_t)p * total + at];
        if (scale) s *= scale[at % n];
        dw[at] = accumulate ? dw[at] + s : s;
    }
}

}  // namespace ef
