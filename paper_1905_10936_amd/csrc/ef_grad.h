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

// What a thread carries from memory to LDS for one step.  Nothing is masked: channels past the operands' ends hold whatever lies there, and
// what they give is not stored.  Steps whose reads could pass the end of dz are filled in by fill() instead.
template <class T>
struct GradStage {
    static constexpr int TOKENS = GradStep<T>::TOKENS, PARTS = GradStep<T>::PARTS;
    static constexpr int Z = TOKENS * GRAD_TILE * (int)sizeof(T) / 16 / GRAD_THREADS;   // 128-bit words of dz: 8
    static constexpr int X = TOKENS * GRAD_TILE / 16 / GRAD_THREADS;                    // of codes: 4 or 2
    static constexpr int Z_WORDS = GRAD_TILE * (int)sizeof(T) / 16;     // words a token
    static constexpr int Z_ELEMS = 16 / (int)sizeof(T);
    u32x4 z[Z], x[X];
    unsigned s[X];
    // This thread's first words of the step to load next, in global memory: a load that might be LDS's would have every LDS read waited for.
    const EF_GLOBAL T *z_from;
    const EF_GLOBAL uint8_t *x_from, *s_from;

    __device__ __forceinline__ void begin(const GradArgs &a, int64_t token0, int64_t o0, int64_t n0)
    {
        const int tid = threadIdx.x;
        int64_t o = o0 + tid % Z_WORDS * Z_ELEMS, i = n0 + tid % 16 * 16;
        if (o >= a.out) o = 0;
        if (i >= a.act.groups * GROUP) i = 0;
        z_from = (const EF_GLOBAL T *)(static_cast<const T *>(a.dz) + (token0 + tid / Z_WORDS) * a.dz_stride + o);
        x_from = (const EF_GLOBAL uint8_t *)a.act.code_at(token0 + tid / 16, i);
        s_from = (const EF_GLOBAL uint8_t *)a.act.scale_at(token0 + tid / 16, i);
    }
    // Word k of dz (k < Z) or of the codes (k - Z); next() goes on to the following step.
    __device__ __forceinline__ void load(const GradArgs &a, int k)
    {
        if (k < Z) {
            const EF_GLOBAL T *p = z_from + (int64_t)k * (GRAD_THREADS / Z_WORDS) * a.dz_stride;
            if constexpr (sizeof(T) == 2)
                z[k] = *(const EF_GLOBAL u32x4_any *)p;
            else
                z[k] = *(const EF_GLOBAL u32x4_word *)p;
        } else {
            k -= Z;
            x[k] = *(const EF_GLOBAL u32x4 *)(x_from + k * (GRAD_THREADS / 16) * a.act.groups * GROUP);
            s[k] = s_from[k * (GRAD_THREADS / 16) * a.act.groups];
        }
    }
    __device__ __forceinline__ void next(const GradArgs &a)
    {
        z_from += TOKENS * a.dz_stride;
        x_from += TOKENS * a.act.groups * GROUP;
        s_from += TOKENS * a.act.groups;
    }
    __device__ __forceinline__ void store(char *buffer, int k) const
    {
        const int tid = threadIdx.x;
        if (k < Z) {
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
        } else {
            k -= Z;
            const int t = tid / 16 + k * (GRAD_THREADS / 16);
            const float scale = scale_value(s[k]);
            char *at = buffer + (PARTS * TOKENS + t) * GRAD_PITCH + tid % 16 * 32;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const u32x2 lo = decode_four(x[k][2 * h], scale), hi = decode_four(x[k][2 * h + 1], scale);
                *reinterpret_cast<u32x4 *>(at + 16 * h) = u32x4{lo.x, lo.y, hi.x, hi.y};
            }
        }
    }

    // The same for the step at token0, element by element and nothing read that is not there; zeros in its place.
    static __device__ void fill(const GradArgs &a, int64_t token0, int64_t o0, int64_t n0, char *buffer)
    {
        for (int k = threadIdx.x; k < TOKENS * GRAD_TILE; k += GRAD_THREADS) {
            const int t = k / GRAD_TILE, c = k % GRAD_TILE;
            const bool there = token0 + t < a.rows;
            char *at = buffer + t * GRAD_PITCH + c * 2;
            unsigned v = 0;
            if (there && o0 + c < a.out) v = element_bits(static_cast<const T *>(a.dz) + (token0 + t) * a.dz_stride + o0 + c);
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<uint16_t *>(at) = (uint16_t)v;
            } else {
                const ThreeParts p = three_parts(__uint_as_float(v));
                *reinterpret_cast<uint16_t *>(at) = (uint16_t)(p.a >> 16);
                *reinterpret_cast<uint16_t *>(at + TOKENS * GRAD_PITCH) = (uint16_t)(p.b >> 16);
                *reinterpret_cast<uint16_t *>(at + 2 * TOKENS * GRAD_PITCH) = (uint16_t)(p.c >> 16);
            }
            uint16_t x = 0;
            if (there && n0 + c < a.n) {
                const unsigned code = *a.act.code_at(token0 + t, n0 + c), scale = *a.act.scale_at(token0 + t, n0 + c);
                x = (uint16_t)decode_four(code, scale_value(scale)).x;
            }
            *reinterpret_cast<uint16_t *>(buffer + (PARTS * TOKENS + t) * GRAD_PITCH + c * 2) = x;
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

    // Steps before `safe` read nothing past dz's end: a token's last word may reach seven elements past its row.
    const int64_t spare = o0 + GRAD_TILE <= a.out ? 0 : (7 + a.dz_stride - 1) / a.dz_stride;
    const int64_t safe = min(last, (a.rows - spare) / TOKENS);
    constexpr int REGIONS = TOKENS / 16 * PARTS, WORDS = GradStage<T>::Z + GradStage<T>::X;
    bf16x8 z[2][4], x[2][4];
    // fragment f of region r: x's where a region begins with another sixteen tokens, then dz's
    auto fragment = [&](const char *buffer, int r, int f) {
        const int k = r / PARTS, p = r % PARTS;
        if (f < 4) {
            if (p == 0) x[k & 1][f] = read_transposed(buffer + x_at + k * 16 * GRAD_PITCH + f * 64);
        } else {
            z[r & 1][f - 4] = read_transposed(buffer + z_at + (p * TOKENS + k * 16) * GRAD_PITCH + (f - 4) * 64);
        }
    };
    auto product = [&](int r, int i, int j) {
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(z[r & 1][i], x[r / PARTS & 1][j], acc[i][j], 0, 0, 0);
    };
    int64_t step = first;
    char *now = buffers[0], *next = buffers[1];
    GradStage<T> stage;
    stage.begin(a, first * TOKENS, o0, n0);
    if (first < safe) {
#pragma unroll
        for (int k = 0; k < WORDS; ++k) stage.load(a, k);
        if (first + 1 < safe) stage.next(a);
#pragma unroll
        for (int k = 0; k < WORDS; ++k) {
            stage.store(now, k);
            stage.load(a, k);
        }
        if (first + 2 < safe) stage.next(a);
    } else if (first < last) {
        GradStage<T>::fill(a, first * TOKENS, o0, n0, now);
    }
    __syncthreads();
    if (step + 1 < safe) {
#pragma unroll
        for (int f = 0; f < 8; ++f) fragment(now, 0, f);
        for (; step + 1 < safe; ++step) {
#pragma unroll
            for (int r = 0; r < REGIONS; ++r) {
                if (r == REGIONS - 1) __syncthreads();
#pragma unroll
                for (int m = 0; m < 16; ++m) {
                    product(r, m / 4, m % 4);
                    if (m < 8) {
                        if (r < REGIONS - 1)
                            fragment(now, r + 1, m);
                        else
                            fragment(next, 0, m);
                    } else if (r < REGIONS - 1) {
                        // words of the next step to LDS, those of the one behind it on their way into the same registers
                        constexpr int EACH = (WORDS + REGIONS - 2) / (REGIONS - 1);
                        const int w = r * EACH + (m - 8) / 2;
                        if (m % 2 == 0 && (m - 8) / 2 < EACH && w < WORDS) {
                            stage.store(next, w);
                            stage.load(a, w);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (step + 3 < safe) stage.next(a);
            char *t = now;
            now = next;
            next = t;
        }
    }
    for (; step < last; ++step) {
        if (step + 1 < last) GradStage<T>::fill(a, (step + 1) * TOKENS, o0, n0, next);
#pragma unroll
        for (int r = 0; r < REGIONS; ++r) {
#pragma unroll
            for (int f = 0; f < 8; ++f) fragment(now, r, f);
#pragma unroll
            for (int m = 0; m < 16; ++m) product(r, m / 4, m % 4);
        }
        __syncthreads();
        char *t = now;
        now = next;
        next = t;
    }

    // An accumulator's lane holds channel lane % 32 of x's side and four runs of four of dz's.
    float *const dw = a.dw + (a.splits > 1 ? (int64_t)split * a.out * a.n : 0) + (o0 + wave / 2 * 128 + 4 * (lane / 32)) * a.n;
    const bool whole = a.splits == 1;
    const int64_t left = a.out - (o0 + wave / 2 * 128 + 4 * (lane / 32));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t i = n0 + wave % 2 * 128 + j * 32 + lane % 32;
        if (i >= a.n) continue;
        const float s = whole && a.scale ? a.scale[i] : 1.0f;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            float v[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = acc[m][j][k] * s;
            float *const at = dw + m * 32 * a.n + i;
            if (whole && a.accumulate) {
                float old[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) old[k] = m * 32 + 8 * (k / 4) + k % 4 < left ? at[(8 * (k / 4) + k % 4) * a.n] : 0.0f;
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] += old[k];
            }
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (m * 32 + 8 * (k / 4) + k % 4 < left) at[(8 * (k / 4) + k % 4) * a.n] = v[k];
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
