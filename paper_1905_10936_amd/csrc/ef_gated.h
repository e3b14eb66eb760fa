// The gated feed-forward block: z = act(a) * u with a = x Wg^T and u = x Wu^T, and its backward pass.
//
// Both projections are one product with the rows of w = [Wg; Wu]; a tile takes the same channels of both, so that a lane ends up with a and u of the
// same place and makes z there: neither goes to memory unless it is kept.  The activations are a * sigmoid(F(a)).
//
// Bound by products: 8192 tokens, 1024 -> 4096 in bf16 with both projections kept 152 to 165 us (0.83 to 0.90 PFLOP/s, the ending included), 2048 -> 8192 451 to 485 (1.13 to 1.22).
//
// Backward: da = dz u act'(a) and du = dz act(a) side by side (dpre), a pass over memory; then dx = dpre w, a product whose sum runs over all 2 f rows
// of w.
#pragma once
#include "ef_product.h"

namespace ef {

constexpr int GATE_SILU = 0, GATE_GELU = 1;

struct GatedArgs {
    int64_t rows, n, f;         // tokens, the input's channels, the product's
    const void *x;
    int64_t x_stride;
    const void *w;
    int64_t w_stride;
    int gate;
    void *pre;                  // [rows][2 f], or null
    int64_t pre_stride;
    void *z;                    // or null
    int64_t z_stride;
    ActRef act;                 // codes null: none
    int tiles_t, tiles_c;
};

constexpr float GELU_SLOPE = 1.5957691216057308f, GELU_CUBIC = 0.044715f;      // 2 sqrt(2 / pi)

// sigmoid(F(a)) and 1 - sigmoid(F(a)), from exp(-|F(a)|) so that neither loses what the other one rounds away.  The bf16 block takes the instructions'
// exponential and reciprocal: their errors and the exponent's rounding, |F| 2^-24, are far below half a step of what is stored wherever the sigmoid is
// not.  (With a division and expf a tile of 256 tokens by 128 channels spends 13 us behind its products, 4 this way.)
template <class T>
__device__ __forceinline__ float2 sigmoid(float a, int gate)
{
    const float s = gate == GATE_GELU ? GELU_SLOPE * __builtin_fmaf(GELU_CUBIC * a * a, a, a) : a;
    float e, big;
    if constexpr (sizeof(T) == 2) {
        e = __builtin_amdgcn_exp2f(-1.44269504f * fabsf(s));
        big = __builtin_amdgcn_rcpf(1.0f + e);
    } else {
        e = expf(-fabsf(s));
        big = 1.0f / (1.0f + e);
    }
    const float small = e * big;
    return s < 0.0f ? make_float2(small, big) : make_float2(big, small);        // a NaN goes on: both are NaN
}
// act(a) * u.  In bf16 as a / (1 + exp(-F)): three instructions fewer than by sigmoid(); a sigmoid below 2^-126 (SILU: a below -87.3, GELU: below -10) is 0, as it is there: the
// instructions take no smaller numbers.
template <class T>
__device__ __forceinline__ float gated(float a, float u, int gate)
{
    if constexpr (sizeof(T) == 2) {
        const float s = gate == GATE_GELU ? __builtin_fmaf(GELU_SLOPE * GELU_CUBIC * a * a, a, GELU_SLOPE * a) : a;
        return a * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * s)) * u;
    } else {
        return a * sigmoid<T>(a, gate).x * u;
    }
}

// Tiles go to the eight XCDs in turn: each takes a run of them, eight token tiles by as many channel tiles as fit, which share their rows in its L2.
__device__ __forceinline__ int2 tile_place(int id, int all, int tiles_t, int tiles_c)
{
    id = id % 8 * (all / 8) + min(id % 8, all % 8) + id / 8;
    const int group = id / (8 * tiles_c), in = id % (8 * tiles_c), high = min(8, tiles_t - group * 8);
    return make_int2(group * 8 + in % high, in / high);
}

template <class T, int WC, int WT>
__global__ __launch_bounds__(PRODUCT_THREADS, WC * WT > 4 ? 1 : 2) void k_gated(GatedArgs g)
{
    using A = RowsOperand<T, 2 * WC>;
    using B = RowsOperand<T, 2 * WT>;
    constexpr int PAIRS = WC / 2, TILE_C = 64 * PAIRS, TILE_T = 64 * WT;
    __shared__ __align__(16) char lds[2 * (A::BYTES + B::BYTES)];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, wave_c = wave / 2, wave_t = wave % 2;
    const int2 place = tile_place(blockIdx.x, g.tiles_t * g.tiles_c, g.tiles_t, g.tiles_c);
    const int64_t t0 = (int64_t)place.x * TILE_T, c0 = (int64_t)place.y * TILE_C;
    const int64_t steps = (g.n + STEP<T> - 1) / STEP<T>, safe = min(A::safe(g.n, g.w_stride, g.f + TILE_C), B::safe(g.n, g.x_stride, TILE_T));
    // Block b of the weight's rows: wavefronts' blocks one after the other, in each the gate's, then the other projection's of the same channels.
    const auto w_row = [&](int b) {
        const int64_t c = min(c0 + (b / WC * PAIRS + b % WC % PAIRS) * 32 + A::row(), g.f - 1);
        return b % WC >= PAIRS ? c + g.f : c;
    };
    const auto x_row = [&](int b) { return min(t0 + 32 * b + B::row(), g.rows - 1); };
    A a;
    B b;
    f32x16 acc[WC][WT];
    a.begin(g.w, g.w_stride, 0, c0, w_row);
    b.begin(g.x, g.x_stride, 0, t0, x_row);
    product_steps<T, WC, WT>(
        a, b, lds, 0, steps, safe, wave_c, wave_t, acc,
        [&] {
            a.next();
            b.next();
        },
        [&](int64_t step) {
            a.load_guarded(g.w, g.w_stride, step * STEP<T>, g.n, w_row);
            b.load_guarded(g.x, g.x_stride, step * STEP<T>, g.n, x_row);
        });

    using Rows = StagedRows<T, 32 * PAIRS>;
    static_assert(3 * 4 * Rows::BYTES <= (int)sizeof lds, "three results of four wavefronts");
    char *const mine = lds + wave * 3 * Rows::BYTES;
    const auto ending = [&](auto inside) {
        constexpr bool INSIDE = decltype(inside)::value;
        const int64_t c1 = c0 + wave_c * PAIRS * 32, left = g.f - c1;
        if (!INSIDE && left <= 0) return;
#pragma unroll
        for (int j = 0; j < WT; ++j) {
            const int64_t t1 = t0 + (wave_t * WT + j) * 32, rows = g.rows - t1;
            if (!INSIDE && rows <= 0) return;
            const bool there = INSIDE || lane % 32 < rows;
#pragma unroll
            for (int i = 0; i < PAIRS; ++i) {
                float z[16];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float va[4], vu[4];
                    const int c = 32 * i + run_channel(lane, r);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        va[k] = acc[i][j][4 * r + k];
                        vu[k] = acc[i + PAIRS][j][4 * r + k];
                        z[4 * r + k] = gated<T>(va[k], vu[k], g.gate);
                    }
                    if (g.z) Rows::put(mine, lane, c, z + 4 * r);
                    if (g.pre) {
                        Rows::put(mine + Rows::BYTES, lane, c, va);
                        Rows::put(mine + 2 * Rows::BYTES, lane, c, vu);
                    }
                }
                if (g.act.codes && (INSIDE || 32 * i < left)) {
                    // a group of 32 channels: lanes l and l + 32, sixteen values each
                    unsigned top = 0;
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        if (!INSIDE && 32 * i + run_channel(lane, k / 4) + k % 4 >= left) z[k] = 0.0f;
                        top = larger(top, __float_as_uint(z[k]) & 0x7fffffffu);
                    }
                    const u32x2 s = __builtin_amdgcn_permlane32_swap(top, top, false, false);
                    const unsigned byte = scale_byte(__uint_as_float(larger(s.x, s.y)));
                    if (there) {
                        const int64_t t = t1 + lane % 32;
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            const int64_t c = c1 + 32 * i + run_channel(lane, 2 * p);
                            g.act.template put_two_fours<!INSIDE>(t, c, c + 8, g.f, z + 8 * p, byte);
                        }
                        if (lane < 32) *g.act.scale_at(t, c1 + 32 * i) = (uint8_t)byte;
                    }
                }
            }
            Rows::meet();
            if (g.z) Rows::template flush<INSIDE>(mine, lane, static_cast<T *>(g.z) + t1 * g.z_stride + c1, g.z_stride, rows, left);
            if (g.pre) {
                T *const to = static_cast<T *>(g.pre) + t1 * g.pre_stride + c1;
                Rows::template flush<INSIDE>(mine + Rows::BYTES, lane, to, g.pre_stride, rows, left);
                Rows::template flush<INSIDE>(mine + 2 * Rows::BYTES, lane, to + g.f, g.pre_stride, rows, left);
            }
            Rows::meet();
        }
    };
    if (t0 + TILE_T <= g.rows && c0 + TILE_C <= g.f)
        ending(std::true_type());
    else
        ending(std::false_type());
}

// Few tokens: bound by the weights' bytes (one token, 1024 -> 4096 in bf16: 6.1 us for 16.8 MB, half of it launch and the join).
// A workgroup takes CHANNELS = 16 or 32 channels of the product (both projections) and up to 32 tokens, its wavefronts the steps in turn;
// their sums meet in LDS.  Fragments come straight from memory, 128 bytes of a row to a step; the instruction's 32 rows are 16 of the gate and 16 of the other projection.
constexpr int FEW_WAVES = 8;
template <class T, int CHANNELS>
__global__ __launch_bounds__(64 * FEW_WAVES) void k_gated_few(GatedArgs g)
{
    constexpr int TILES = CHANNELS / 16;
    __shared__ float sums[FEW_WAVES][TILES][64][17];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t c0 = (int64_t)(blockIdx.x / g.tiles_t) * CHANNELS, t0 = (int64_t)(blockIdx.x % g.tiles_t) * 32;
    const EF_GLOBAL char *wp[TILES], *xp;
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
        const int64_t c = min(c0 + 16 * i + lane % 16, g.f - 1) + (lane % 32 >= 16 ? g.f : 0);
        wp[i] = (const EF_GLOBAL char *)g.w + c * g.w_stride * (int64_t)sizeof(T);
    }
    xp = (const EF_GLOBAL char *)g.x + min(t0 + lane % 32, g.rows - 1) * g.x_stride * (int64_t)sizeof(T);
    f32x16 acc[TILES];
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[i][k] = 0.0f;
    const int64_t steps = (g.n + STEP<T> - 1) / STEP<T>, whole = g.n / STEP<T>;
    for (int64_t step = wave; step < steps; step += FEW_WAVES) {
        u32x4 fa[TILES][4], fb[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            // lanes l and l + 32 have a row's two halves of a step
            const int64_t k = step * STEP<T> + lane / 32 * (STEP<T> / 2) + q * WORD<T>;
            if (step < whole) {
#pragma unroll
                for (int i = 0; i < TILES; ++i) fa[i][q] = load_word<T>(wp[i] + k * (int64_t)sizeof(T));
                fb[q] = load_word<T>(xp + k * (int64_t)sizeof(T));
            } else {
#pragma unroll
                for (int i = 0; i < TILES; ++i) fa[i][q] = load_part<T>(wp[i] + k * (int64_t)sizeof(T), g.n - k);
                fb[q] = load_part<T>(xp + k * (int64_t)sizeof(T), g.n - k);
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < TILES; ++i) multiply<T>(fa[i][q], fb[q], acc[i]);
    }
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
        for (int k = 0; k < 16; ++k) sums[wave][i][lane][k] = acc[i][k];
    __syncthreads();
    // Eight channels of a token to a thread; a group's four are neighbours.  Channel c of 16 lies in run c / 8 (the gate's: 0, 1; the other's: 2, 3), lanes l + 32 (c / 4 % 2).
    constexpr int EIGHTS = CHANNELS / 8;
    if (threadIdx.x >= 32 * EIGHTS) return;
    const int token = threadIdx.x / EIGHTS, eight = threadIdx.x % EIGHTS;
    const int64_t t = t0 + token, c = c0 + eight * 8;
    float va[8], vu[8], z[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int l = token + 32 * (k / 4), run = eight % 2 * 4 + k % 4;
        va[k] = vu[k] = 0.0f;
        for (int s = 0; s < FEW_WAVES; ++s) {
            va[k] += sums[s][eight / 2][l][run];
            vu[k] += sums[s][eight / 2][l][8 + run];
        }
        z[k] = c + k < g.f ? gated<T>(va[k], vu[k], g.gate) : 0.0f;
    }
    if (t >= g.rows) return;            // whole groups
    Eight<T> e;
    if (g.pre) {
        T *const row = static_cast<T *>(g.pre) + t * g.pre_stride + c;
        e.round(va);
        store_some(e, row, g.f - c);
        e.round(vu);
        store_some(e, row + g.f, g.f - c);
    }
    if (g.z) {
        e.round(z);
        store_some(e, static_cast<T *>(g.z) + t * g.z_stride + c, g.f - c);
    }
    if constexpr (CHANNELS == GROUP)
        if (g.act.codes) g.act.put(t, c, g.f, z);
}

// ------------------------------------------------------------------------------------------- backward ---

struct SlopeArgs {
    int64_t rows, f;
    const void *dz;
    int64_t dz_stride;
    const void *pre;
    int64_t pre_stride;
    void *dpre;
    int64_t dpre_stride;
    int gate;
    int64_t first;
};

// dpre, eight channels of both halves to a thread: five numbers moved to a place of z, nothing else counts (8192 x 4096 in bf16: 50 us, 6.5 TB/s).
template <class T>
__global__ __launch_bounds__(256) void k_gated_slopes(SlopeArgs g)
{
    const int64_t per_row = (g.f + 7) / 8, at = g.first + (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = at / per_row, c = (at - row * per_row) * 8;
    if (row >= g.rows) return;
    Eight<T> z, a, u;
    const T *const pre = static_cast<const T *>(g.pre) + row * g.pre_stride + c;
    load_some(z, static_cast<const T *>(g.dz) + row * g.dz_stride + c, g.f - c, 0u);
    load_some(a, pre, g.f - c, 0u);
    load_some(u, pre + g.f, g.f - c, 0u);
    float da[8], du[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float v = a[k];
        const float2 s = sigmoid<T>(v, g.gate);
        // where the sigmoid has ended, its slope is 0 however large F'(a) is
        const float both = s.x * s.y, slope = g.gate == GATE_GELU ? GELU_SLOPE * (1.0f + 3.0f * GELU_CUBIC * v * v) : 1.0f;
        const float change = both == 0.0f ? 0.0f : v * both * slope;
        da[k] = z[k] * u[k] * (s.x + change);
        du[k] = z[k] * (v * s.x);
    }
    T *const to = static_cast<T *>(g.dpre) + row * g.dpre_stride + c;
    a.round(da);
    u.round(du);
    store_some(a, to, g.f - c);
    store_some(u, to + g.f, g.f - c);
}

struct InputGradArgs {
    int64_t rows, n, k;         // tokens, the input's channels, 2 f
    const void *dpre;
    int64_t dpre_stride;
    const void *w;
    int64_t w_stride;
    void *dx;
    int64_t dx_stride;
    int tiles_t, tiles_c, splits;
    float *parts;               // [splits][rows][n] with more than one
};

// dx = dpre w, bound by products (8192 tokens, 2 x 4096 -> 1024 in bf16: 137 us, 1.0 PFLOP/s); with splits > 1 a workgroup sums over a part of k and leaves it in `parts`.
template <class T, int WC, int WT>
__global__ __launch_bounds__(PRODUCT_THREADS, WC * WT > 4 ? 1 : 2) void k_input_grad(InputGradArgs g)
{
    using A = ColumnsOperand<T, 2 * WC>;
    using B = RowsOperand<T, 2 * WT>;
    constexpr int TILE_C = 64 * WC, TILE_T = 64 * WT;
    __shared__ __align__(16) char lds[2 * (A::BYTES + B::BYTES)];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, wave_c = wave / 2, wave_t = wave % 2;
    const int tiles = g.tiles_t * g.tiles_c, split = blockIdx.x / tiles;
    const int2 place = tile_place(blockIdx.x % tiles, tiles, g.tiles_t, g.tiles_c);
    const int64_t t0 = (int64_t)place.x * TILE_T, c0 = (int64_t)place.y * TILE_C;
    const int64_t steps = (g.k + STEP<T> - 1) / STEP<T>, first = steps * split / g.splits, last = steps * (split + 1) / g.splits;
    const int64_t safe = min(last, min(A::safe(g.k, g.w_stride, c0, g.n), B::safe(g.k, g.dpre_stride, TILE_T)));
    const auto row = [&](int b) { return min(t0 + 32 * b + B::row(), g.rows - 1); };
    A a;
    B b;
    f32x16 acc[WC][WT];
    a.begin(g.w, g.w_stride, first * STEP<T>, c0, g.n);
    b.begin(g.dpre, g.dpre_stride, first * STEP<T>, t0, row);
    product_steps<T, WC, WT>(
        a, b, lds, first, last, safe, wave_c, wave_t, acc,
        [&] {
            a.next(g.w_stride);
            b.next();
        },
        [&](int64_t step) {
            a.load_guarded(g.w, g.w_stride, step * STEP<T>, g.k, c0, g.n);
            b.load_guarded(g.dpre, g.dpre_stride, step * STEP<T>, g.k, row);
        });
    const auto ending = [&](auto inside, auto of, auto *to, int64_t stride) {
        constexpr bool INSIDE = decltype(inside)::value;
        using Rows = StagedRows<decltype(of), 32 * WC>;
        static_assert(4 * Rows::BYTES <= (int)sizeof lds, "of four wavefronts");
        char *const mine = lds + wave * Rows::BYTES;
        const int64_t c1 = c0 + wave_c * WC * 32, left = g.n - c1;
        if (!INSIDE && left <= 0) return;
#pragma unroll
        for (int j = 0; j < WT; ++j) {
            const int64_t t1 = t0 + (wave_t * WT + j) * 32, rows = g.rows - t1;
            if (!INSIDE && rows <= 0) return;
#pragma unroll
            for (int i = 0; i < WC; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float v[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] = acc[i][j][4 * r + k];
                    Rows::put(mine, lane, 32 * i + run_channel(lane, r), v);
                }
            Rows::meet();
            Rows::template flush<INSIDE>(mine, lane, to + t1 * stride + c1, stride, rows, left);
            Rows::meet();
        }
    };
    const bool inside = t0 + TILE_T <= g.rows && c0 + TILE_C <= g.n;
    if (g.splits > 1) {
        float *const to = g.parts + (int64_t)split * g.rows * g.n;
        if (inside)
            ending(std::true_type(), float(), to, g.n);
        else
            ending(std::false_type(), float(), to, g.n);
    } else {
        T *const to = static_cast<T *>(g.dx);
        if (inside)
            ending(std::true_type(), T(), to, g.dx_stride);
        else
            ending(std::false_type(), T(), to, g.dx_stride);
    }
}

// dx from the parts, added up in their order.
template <class T>
__global__ __launch_bounds__(256) void k_join_input_grad(InputGradArgs g)
{
    const int64_t per_row = (g.n + 7) / 8, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t t = at / per_row, c = (at - t * per_row) * 8;
    if (t >= g.rows) return;
    float v[8] = {};
    for (int s = 0; s < g.splits; ++s) {
        Eight<float> e;
        load_some(e, (const float *)g.parts + ((int64_t)s * g.rows + t) * g.n + c, g.n - c, 0u);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += e[k];
    }
    Eight<T> e;
    e.round(v);
    store_some(e, static_cast<T *>(g.dx) + t * g.dx_stride + c, g.n - c);
}

}  // namespace ef
