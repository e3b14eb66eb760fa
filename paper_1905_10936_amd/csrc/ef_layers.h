// Host side of the operators of a worker's forward and backward pass: argument checks, choice of kernel, launches.
// Part of ef_api.hip, whose helpers it uses.
#pragma once
#include "ef_act.h"
#include "ef_grad.h"
#include "ef_norm.h"
#include "ef_policy.h"

struct ef_workspace {
    int device;
    int64_t max_rows;
    float *row_sums;            // [max_rows]
    float *parts;               // [PART_FLOATS]
    void *base;
};

namespace {

constexpr int64_t PART_FLOATS = 1 << 24;        // 64 MiB of partial results
constexpr int64_t WIDTH_MAX = 1 << 24;
constexpr int64_t ROWS_MAX = 0x7fffffff;
constexpr int64_t GRID_MAX = 1 << 22;           // workgroups of a launch that grows with the rows: a grid holds less than 2^32 threads

bool good_type(int type) { return type == EF_TYPE_FP32 || type == EF_TYPE_BF16; }
size_t type_size(int type) { return type == EF_TYPE_BF16 ? 2 : 4; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t act_groups(int64_t width) { return ceil_div(width, ef::GROUP); }

// Is one of the pointers missing that a call on rows needs?  Without rows they point to nothing, and an empty tensor's address is null.
template <class... P>
bool missing(int64_t rows, const P *...p) { return rows != 0 && (!p || ...); }

// A matrix argument as the checks see it; p == nullptr: not given.
struct Matrix {
    const void *p;
    int64_t stride;
    int64_t rows, width;
    size_t size;
    int64_t pitch() const { return (rows > 1 ? stride : width) * (int64_t)size; }
    size_t bytes() const { return rows > 0 ? (size_t)(rows - 1) * (size_t)pitch() + (size_t)width * size : 0; }
    bool good_stride() const { return rows < 2 || (stride >= width && stride <= INT64_MAX / 8 / rows); }
};

// Do the two share an element?  Rows side by side in one buffer do not.
bool share(const Matrix &a, const Matrix &b)
{
    if (!a.p || !b.p || !overlap(a.p, a.bytes(), b.p, b.bytes())) return false;
    if (!a.bytes() || !b.bytes()) return false;
    if (a.pitch() != b.pitch() || a.rows < 2 || b.rows < 2) return true;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    const uintptr_t pitch = (uintptr_t)a.pitch(), off = y >= x ? (y - x) % pitch : (pitch - (x - y) % pitch) % pitch;
    // modulo the pitch, a takes [0, its width) and b takes [off, off + its width)
    return !(off >= a.width * a.size && off + b.width * b.size <= pitch);
}
bool same(const Matrix &a, const Matrix &b) { return a.p == b.p && a.size == b.size && (a.rows < 2 || a.stride == b.stride); }
Matrix vector_of(const void *p, int64_t n, size_t size) { return Matrix{p, n, n > 0 ? 1 : 0, n, size}; }

// Outputs against each other and against inputs; out[i] may be `in[j]` itself where bit j of in_place[i] is set.
bool apart(const Matrix *out, int n_out, const Matrix *in, int n_in, const unsigned *in_place)
{
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < i; ++j)
            if (share(out[i], out[j])) return false;
        for (int j = 0; j < n_in; ++j)
            if (share(out[i], in[j]) && !((in_place[i] >> j & 1) && same(out[i], in[j]))) return false;
    }
    return true;
}

ef::ActRef act_ref(const void *act, int64_t rows, int64_t width)
{
    ef::ActRef r;
    r.codes = static_cast<uint8_t *>(const_cast<void *>(act));
    r.groups = act_groups(width);
    r.scales = r.codes ? r.codes + rows * r.groups * ef::GROUP : nullptr;
    return r;
}

int on_workspace_device(const ef_workspace *w)
{
    int device = -1;
    EF_HIP(hipGetDevice(&device));
    return device == w->device ? EF_OK : EF_ERR_ARG;
}

int act_args(int64_t rows, int64_t width, int type, const void *m, int64_t stride, const void *act)
{
    if (missing(rows, m, act)) return EF_ERR_NULL;
    if (rows < 0 || rows > ROWS_MAX || width < 1 || !good_type(type)) return EF_ERR_ARG;
    if (width > WIDTH_MAX) return EF_ERR_SIZE;
    const Matrix a{m, stride, rows, width, type_size(type)};
    if (!a.good_stride()) return EF_ERR_ARG;
    if (!aligned(m, type_size(type)) || !aligned(act, 16)) return EF_ERR_ALIGN;
    if (ceil_div(rows * act_groups(width) * (ef::GROUP / 8), ef::ACT_THREADS) > 0x7fffffff) return EF_ERR_SIZE;      // more than any memory holds
    return share(a, vector_of(act, (int64_t)ef_act_bytes(rows, width), 1)) ? EF_ERR_ARG : EF_OK;
}

#define EF_BY_TYPE(type, T, ...)                          \
    do {                                                  \
        if ((type) == EF_TYPE_BF16) {                     \
            using T = ef::bf16_t;                         \
            __VA_ARGS__;                                  \
        } else {                                          \
            using T = float;                              \
            __VA_ARGS__;                                  \
        }                                                 \
    } while (0)

// `groups` workgroups in launches of GRID_MAX at most; f gets each launch's grid and the number of its first workgroup.
template <class F>
void in_launches(int64_t groups, F f)
{
    for (int64_t first = 0; first < groups; first += GRID_MAX) f(dim3((unsigned)std::min(groups - first, GRID_MAX)), first);
}

template <class T, int LANES, int CHUNKS>
void launch_norm_forward(ef::NormForward a, hipStream_t s)
{
    constexpr int threads = ef::norm_threads(LANES);
    in_launches(ceil_div(a.rows, threads / LANES), [&](dim3 grid, int64_t first) {
        a.first = first * (threads / LANES);
        hipLaunchKernelGGL((ef::k_norm_forward<T, LANES, CHUNKS>), grid, dim3(threads), 0, s, a);
    });
}
template <class T, int LANES, int CHUNKS>
int launch_norm_backward(ef::NormBackward &a, hipStream_t s)
{
    constexpr int threads = ef::norm_threads(LANES);
    // As many workgroups as have rows, up to two to a CU, or one where they are of 512 threads or two would leave a team no more than two rows: the workgroups'
    // sums are written and read (bf16, one and two to a CU: 512 x 8192 15.1 and 17.4 us, 2048 x 16384 54.5 and 60.1, 4096 x 4096 32.1 and 28.6).
    // They have to fit the workspace.
    const int64_t turns = ceil_div(a.rows, threads / LANES), most = threads >= 512 || turns <= 1024 ? 256 : 512;
    const int64_t groups = std::min(std::min(turns, most), PART_FLOATS / a.n);
    hipLaunchKernelGGL((ef::k_norm_backward<T, LANES, CHUNKS>), dim3((unsigned)groups), dim3(threads), 0, s, a);
    return (int)groups;
}

// The team that holds a row of n, with just as many chunks as it takes: 16 lanes up to 128 channels, a wavefront up to 2048 (no barrier), a workgroup
// beyond.
#define EF_NORM_TEAM(n, CALL)            \
    ((n) <= 128     ? CALL(16, 1)        \
     : (n) <= 512   ? CALL(64, 1)        \
     : (n) <= 1024  ? CALL(64, 2)        \
     : (n) <= 1536  ? CALL(64, 3)        \
     : (n) <= 2048  ? CALL(64, 4)        \
     : (n) <= 4096  ? CALL(256, 2)       \
     : (n) <= 6144  ? CALL(256, 3)       \
     : (n) <= 8192  ? CALL(256, 4)       \
     : (n) <= 12288 ? CALL(512, 3)       \
                    : CALL(512, 4))

template <class T, int LANES, int CHUNKS>
void launch_policy(const ef::PolicyArgs &a, hipStream_t s)
{
    // as many workgroups as the CUs hold at most (2048 threads a CU); they go on to further rows
    constexpr int threads = ef::policy_threads(LANES);
    const int64_t groups = std::min(ceil_div(a.rows, threads / LANES), (int64_t)256 * 2048 / threads);
    hipLaunchKernelGGL((ef::k_policy<T, LANES, CHUNKS>), dim3((unsigned)groups), dim3(threads), 0, s, a);
}

// The first of the listed teams that holds a row; false: none does.
template <class T, int LANES, int... CHUNKS>
bool policy_teams(const ef::PolicyArgs &a, hipStream_t s)
{
    return ((a.vocab <= LANES * 8 * CHUNKS && (launch_policy<T, LANES, CHUNKS>(a, s), true)) || ...);
}

// A row's own arithmetic, a hundred instructions, is a wavefront's whatever the row's length, so short rows are four to a wavefront (32768 rows of 259 in bf16
// 22 us, 32 with a wavefront to a row; of 600 20 and 31); it costs a workgroup three barriers besides, so a wavefront has rows of up to 4096 or 5120 (16384
// of 2500 in bf16 41 us, 66 with 256 threads) and a thread of a workgroup many eights where its type lets it (bf16, in us: 8192 x 9000 65 with
// 256 threads, 99 with 1024; 4096 x 18000 63 and 73; 2048 x 65000 115 with 512, 120 with 1024).  Between, rows of 24577 to 40960 have 1024 threads: 4 or 5 eights
// and 64 registers a thread put two workgroups on a CU (8192 x 32768 204, with 512 threads 213, with 256 222; 1024 x 32000 30, 34 and 31; the
// shortest of them lose, 8192 x 25000 173 and 168; the longest are alike, 4096 x 40000 133 and 134).  fp32 gains nothing from many eights.
template <class T>
void policy_rows(const ef::PolicyArgs &a, hipStream_t s)
{
    bool done = false;
    if constexpr (sizeof(T) == 2)
        done = policy_teams<T, 16, 1, 4, 8>(a, s) || policy_teams<T, 64, 4, 8, 10>(a, s) || policy_teams<T, 256, 4, 8, 12>(a, s) || policy_teams<T, 1024, 4, 5>(a, s) ||
               policy_teams<T, 512, 12, 14, 16>(a, s) || policy_teams<T, 1024, 10, 12, 14, 16, 18, 20, 22, 24>(a, s);
    else
        done = policy_teams<T, 16, 1, 4, 6>(a, s) || policy_teams<T, 64, 4, 8>(a, s) || policy_teams<T, 256, 4>(a, s) || policy_teams<T, 1024, 2, 3, 4, 5, 6, 7, 8, 10, 12>(a, s);
    if (!done) hipLaunchKernelGGL(ef::k_policy_long<T>, dim3((unsigned)a.rows), dim3(ef::LONG_THREADS), 0, s, a);
}

template <class T>
void policy_slices(const ef::PolicyArgs &a, float *parts, float *loss, hipStream_t s)
{
    ef::SliceRef r;
    r.joint = reinterpret_cast<float2 *>(parts);
    r.chosen = parts + 2 * ef::SLICED_ROWS * ef::SLICES_MAX;
    r.count = (int)std::min<int64_t>(ceil_div(a.vocab, ef::SLICE), std::min<int64_t>(ef::SLICES_MAX, ceil_div(ef::SLICES_ALL, a.rows)));
    r.length = (int)(ceil_div(a.vocab, r.count * 8) * 8);
    const dim3 grid((unsigned)(a.rows * r.count));
    hipLaunchKernelGGL(ef::k_policy_slices<T>, grid, dim3(ef::SLICE_THREADS), 0, s, a, r);
    hipLaunchKernelGGL(ef::k_policy_join<T>, dim3(grid.x + (loss ? 1u : 0u)), dim3(ef::SLICE_THREADS), 0, s, a, r, loss);
}

int policy_args(int64_t rows, int64_t vocab, int type, const void *logits, int64_t stride, const int64_t *tokens)
{
    if (missing(rows, logits, tokens)) return EF_ERR_NULL;
    if (rows < 0 || rows > ROWS_MAX || vocab < 1 || vocab > 0x7fffffff || !good_type(type)) return EF_ERR_ARG;
    const Matrix l{logits, stride, rows, vocab, type_size(type)};
    if (!l.good_stride()) return EF_ERR_ARG;
    if (!aligned(logits, type_size(type)) || !aligned(tokens, 8)) return EF_ERR_ALIGN;
    return EF_OK;
}

// How a weight gradient is cut: the tile's side, and for the tiles that do not fill a round of the CUs the number of parts along the tokens.
struct GradCut {
    int side;
    int64_t tiles_n, tiles, whole;
    int splits;
};

// The choice is the least of a sum of what was measured: a step of a tile of 256, 128 or 64 channels takes `alone` us with few workgroups on the GPU and
// `loaded` us with as many as it holds (`most` on a CU; more slow the others down with the square of their share), a launch and a workgroup's
// beginning and end `base`, and joining parts 4 us and their bytes at 4.5 TB/s.  Large tiles win where there are many (4096 x 4096, 4096
// tokens, bf16: 116, 140 and 276 us), small ones where there are few tokens (1024 x 1024, 1024 tokens: 34, 14 and 9 us), parts where there are
// many (200 x 200, 8000 tokens, tiles of 64: 42 us in one part, 12 in 8 to 16).
GradCut grad_cut(int type, int64_t steps, int64_t out, int64_t n)
{
    struct Side { int side, most; double alone, loaded, base; };
    static constexpr Side SIDES[2][3] = {{{4, 1, 1.7, 2.3, 15.0}, {2, 2, 0.7, 1.43, 6.0}, {1, 3, 0.44, 0.82, 5.5}},         // EF_TYPE_FP32
                                         {{4, 1, 1.14, 1.5, 15.0}, {2, 2, 0.52, 1.08, 6.0}, {1, 2, 0.3, 0.55, 5.5}}};
    GradCut best{};
    double least = 0.0;
    for (const Side &c : SIDES[type == EF_TYPE_BF16]) {
        const int64_t tile = 64 * c.side, tiles_n = ceil_div(n, tile), tiles = ceil_div(out, tile) * tiles_n, round = 256 * c.most;
        const int64_t whole = tiles / round * round, cut = tiles - whole;
        const auto took = [&](int64_t groups, int64_t of) {
            const double share = (double)std::min(groups, round) / (double)round;
            return (double)(ceil_div(groups, round) * of) * (c.alone + (c.loaded - c.alone) * share * share);
        };
        for (int64_t splits = 1; splits <= 64 && splits <= std::max<int64_t>(1, steps); ++splits) {
            const int64_t part = cut * splits * tile * tile;
            if (splits > 1 && (cut == 0 || part > PART_FLOATS)) break;
            const double cost = c.base + took(whole, steps) + took(cut * splits, ceil_div(steps, splits)) +
                                (splits > 1 ? 4.0 + (double)(part + part / splits) * 4.0 / 4.5e6 : 0.0);
            if (best.side == 0 || cost < least) {
                best = GradCut{c.side, tiles_n, tiles, splits > 1 ? whole : tiles, (int)splits};
                least = cost;
            }
        }
    }
    return best;
}

template <class T, int SIDE>
void launch_weight_grad(const ef::GradArgs &a, hipStream_t s)
{
    const int64_t cut = a.tiles - a.whole;
    hipLaunchKernelGGL((ef::k_weight_grad<T, SIDE>), dim3((unsigned)(a.whole + cut * a.splits)), dim3(ef::GRAD_THREADS), 0, s, a);
    if (cut) {
        constexpr int TILE = 64 * SIDE;
        hipLaunchKernelGGL(ef::k_join_splits<TILE>, dim3((unsigned)(cut * (TILE * TILE / 1024))), dim3(256), 0, s, a);
    }
}

}  // namespace

extern "C" {

size_t ef_act_scales_offset(int64_t rows, int64_t width)
{
    if (rows < 0 || width < 1 || width > INT64_MAX - ef::GROUP) return 0;
    const int64_t groups = act_groups(width);
    if (rows > 0 && groups > ((int64_t)1 << 56) / rows) return 0;
    return (size_t)(rows * groups * ef::GROUP);
}

size_t ef_act_bytes(int64_t rows, int64_t width)
{
    const size_t codes = ef_act_scales_offset(rows, width);
    return (codes + codes / ef::GROUP + 15) / 16 * 16;
}

int ef_act_encode(int64_t rows, int64_t width, int type, const void *x, int64_t x_stride, void *act, void *stream)
{
    const int rc = act_args(rows, width, type, x, x_stride, act);
    if (rc || !rows) return rc;
    const ef::ActRef r = act_ref(act, rows, width);
    in_launches(ceil_div(rows * r.groups * (ef::GROUP / 8), ef::ACT_THREADS), [&](dim3 grid, int64_t first) {
        EF_BY_TYPE(type, T, hipLaunchKernelGGL(ef::k_act_encode<T>, grid, dim3(ef::ACT_THREADS), 0, static_cast<hipStream_t>(stream),
                                               static_cast<const T *>(x), x_stride, rows, width, r, first * ef::ACT_THREADS));
    });
    EF_HIP(hipGetLastError());
    return EF_OK;
}

int ef_act_decode(int64_t rows, int64_t width, const void *act, int type, void *y, int64_t y_stride, void *stream)
{
    const int rc = act_args(rows, width, type, y, y_stride, act);
    if (rc || !rows) return rc;
    const ef::ActRef r = act_ref(act, rows, width);
    in_launches(ceil_div(rows * r.groups * (ef::GROUP / 8), ef::ACT_THREADS), [&](dim3 grid, int64_t first) {
        EF_BY_TYPE(type, T, hipLaunchKernelGGL(ef::k_act_decode<T>, grid, dim3(ef::ACT_THREADS), 0, static_cast<hipStream_t>(stream), r, rows,
                                               width, static_cast<T *>(y), y_stride, first * ef::ACT_THREADS));
    });
    EF_HIP(hipGetLastError());
    return EF_OK;
}

int ef_norm_forward(int64_t rows, int64_t width, int type, const void *x, int64_t x_stride, const void *residual,
                    int64_t residual_stride, const float *weight, float eps, void *h, int64_t h_stride, void *y, int64_t y_stride,
                    void *act, float *rstd, void *stream)
{
    if (missing(rows, x) || (rows && !h && !y && !act && !rstd)) return EF_ERR_NULL;
    if (rows < 0 || rows > ROWS_MAX || width < 1 || !good_type(type) || !(std::isfinite(eps) && eps >= 0.0f)) return EF_ERR_ARG;
    if (width > EF_NORM_MAX_WIDTH) return EF_ERR_SIZE;
    const size_t size = type_size(type);
    const Matrix in[3] = {{x, x_stride, rows, width, size}, {residual, residual_stride, rows, width, size}, vector_of(weight, width, 4)};
    const Matrix out[4] = {{h, h_stride, rows, width, size}, {y, y_stride, rows, width, size},
                           vector_of(act, (int64_t)ef_act_bytes(rows, width), 1), vector_of(rstd, rows, 4)};
    for (const Matrix *m : {&in[0], &in[1], &out[0], &out[1]}) {
        if (m->p && !m->good_stride()) return EF_ERR_ARG;
        if (!aligned(m->p, size)) return EF_ERR_ALIGN;
    }
    if (!aligned(weight, 4) || !aligned(act, 16) || !aligned(rstd, 4)) return EF_ERR_ALIGN;
    const unsigned in_place[4] = {3u, 3u, 0u, 0u};
    if (!apart(out, 4, in, 3, in_place)) return EF_ERR_ARG;
    if (!rows) return EF_OK;
    const ef::NormForward a{rows, width, x, residual, x_stride, residual_stride, weight, eps, h, y, h_stride, y_stride,
                            act_ref(act, rows, width), rstd, 0};
    const hipStream_t s = static_cast<hipStream_t>(stream);
#define EF_CALL(LANES, CHUNKS) launch_norm_forward<T, LANES, CHUNKS>(a, s)
    EF_BY_TYPE(type, T, EF_NORM_TEAM(width, EF_CALL));
#undef EF_CALL
    EF_HIP(hipGetLastError());
    return EF_OK;
}

int ef_workspace_create(ef_workspace **out, int64_t max_rows, void *stream)
{
    (void)stream;
    if (!out) return EF_ERR_NULL;
    *out = nullptr;
    if (max_rows < 0 || max_rows > ROWS_MAX) return EF_ERR_ARG;
    ef_workspace *w = new (std::nothrow) ef_workspace();
    if (!w) return EF_ERR_ARG;
    w->max_rows = max_rows;
    const size_t rows_bytes = ((size_t)max_rows * sizeof(float) + 255) / 256 * 256;
    hipError_t e = hipGetDevice(&w->device);
    if (e == hipSuccess) e = hipMalloc(&w->base, rows_bytes + sizeof(float) * (size_t)PART_FLOATS);
    if (e != hipSuccess) {
        delete w;
        return hip_fail(e);
    }
    w->row_sums = static_cast<float *>(w->base);
    w->parts = reinterpret_cast<float *>(static_cast<char *>(w->base) + rows_bytes);
    *out = w;
    return EF_OK;
}

int ef_workspace_destroy(ef_workspace *workspace)
{
    if (!workspace) return EF_ERR_NULL;
    // on its own device, which need not be the current one
    int current = workspace->device;
    (void)hipGetDevice(&current);
    if (current != workspace->device) (void)hipSetDevice(workspace->device);
    (void)hipDeviceSynchronize();
    (void)hipFree(workspace->base);
    if (current != workspace->device) (void)hipSetDevice(current);
    delete workspace;
    return EF_OK;
}

int ef_norm_backward(ef_workspace *workspace, int64_t rows, int64_t width, int type, const void *dy, int64_t dy_stride,
                     const void *act, const float *rstd, const float *weight, const void *dh, int64_t dh_stride, void *dx,
                     int64_t dx_stride, float *dweight, int accumulate, void *stream)
{
    if (!workspace || missing(rows, dy, act, rstd, dx)) return EF_ERR_NULL;
    if (rows < 0 || rows > ROWS_MAX || width < 1 || !good_type(type)) return EF_ERR_ARG;
    if (width > EF_NORM_MAX_WIDTH || rows > workspace->max_rows) return EF_ERR_SIZE;
    const size_t size = type_size(type);
    const Matrix in[5] = {{dy, dy_stride, rows, width, size}, {dh, dh_stride, rows, width, size},
                          vector_of(act, (int64_t)ef_act_bytes(rows, width), 1), vector_of(rstd, rows, 4), vector_of(weight, width, 4)};
    const Matrix out[2] = {{dx, dx_stride, rows, width, size}, vector_of(dweight, width, 4)};
    for (const Matrix *m : {&in[0], &in[1], &out[0]}) {
        if (m->p && !m->good_stride()) return EF_ERR_ARG;
        if (!aligned(m->p, size)) return EF_ERR_ALIGN;
    }
    if (!aligned(act, 16) || !aligned(rstd, 4) || !aligned(weight, 4) || !aligned(dweight, 4)) return EF_ERR_ALIGN;
    const unsigned in_place[2] = {3u, 0u};
    if (!apart(out, 2, in, 5, in_place)) return EF_ERR_ARG;
    { const int rc = on_workspace_device(workspace); if (rc) return rc; }
    const hipStream_t s = static_cast<hipStream_t>(stream);
    int groups = 0;
    if (rows) {
        ef::NormBackward a{rows, width, dy, dh, dy_stride, dh_stride, act_ref(act, rows, width), rstd, weight, dx, dx_stride,
                           dweight ? workspace->parts : nullptr};
#define EF_CALL(LANES, CHUNKS) launch_norm_backward<T, LANES, CHUNKS>(a, s)
        EF_BY_TYPE(type, T, groups = EF_NORM_TEAM(width, EF_CALL));
#undef EF_CALL
        EF_HIP(hipGetLastError());
    }
    if (dweight) {
        hipLaunchKernelGGL(ef::k_sum_parts, dim3((unsigned)ceil_div(width, 32)), dim3(1024), 0, s, workspace->parts, groups, width, dweight,
                           accumulate ? 1 : 0);
        EF_HIP(hipGetLastError());
    }
    return EF_OK;
}

int ef_weight_grad(ef_workspace *workspace, int64_t rows, int64_t out_width, int64_t width, int type, const void *dz,
                   int64_t dz_stride, const void *act, const float *column_scale, float *dw, int accumulate, void *stream)
{
    if (!workspace || !dw || missing(rows, dz, act)) return EF_ERR_NULL;
    if (rows < 0 || rows > ROWS_MAX || width < 1 || out_width < 1 || !good_type(type)) return EF_ERR_ARG;
    if (width > WIDTH_MAX || out_width > WIDTH_MAX || rows > workspace->max_rows) return EF_ERR_SIZE;
    const size_t size = type_size(type);
    const Matrix in[3] = {{dz, dz_stride, rows, out_width, size}, vector_of(act, (int64_t)ef_act_bytes(rows, width), 1),
                          vector_of(column_scale, width, 4)};
    const Matrix out[1] = {vector_of(dw, out_width * width, 4)};
    if (!in[0].good_stride()) return EF_ERR_ARG;
    if (!aligned(dz, size) || !aligned(act, 16) || !aligned(column_scale, 4) || !aligned(dw, 4)) return EF_ERR_ALIGN;
    const unsigned in_place[1] = {0u};
    if (!apart(out, 1, in, 3, in_place)) return EF_ERR_ARG;
    { const int rc = on_workspace_device(workspace); if (rc) return rc; }
    const hipStream_t s = static_cast<hipStream_t>(stream);
    ef::GradArgs a;
    a.rows = rows;
    a.out = out_width;
    a.n = width;
    a.dz = dz;
    a.dz_stride = rows > 1 ? dz_stride : out_width;      // the kernel divides by it
    a.act = act_ref(act, rows, width);
    a.scale = column_scale;
    a.accumulate = accumulate ? 1 : 0;
    a.steps = ceil_div(rows, type == EF_TYPE_BF16 ? ef::GradStep<ef::bf16_t>::TOKENS : ef::GradStep<float>::TOKENS);
    const GradCut c = grad_cut(type, a.steps, out_width, width);
    if (c.tiles > 0x1ffffff) return EF_ERR_SIZE;
    a.dw = dw;
    a.parts = workspace->parts;
    a.tiles = (int)c.tiles;
    a.tiles_n = (int)c.tiles_n;
    a.whole = (int)c.whole;
    a.splits = c.splits;
    if (c.side == 4)
        EF_BY_TYPE(type, T, launch_weight_grad<T, 4>(a, s));
    else if (c.side == 2)
        EF_BY_TYPE(type, T, launch_weight_grad<T, 2>(a, s));
    else
        EF_BY_TYPE(type, T, launch_weight_grad<T, 1>(a, s));
    EF_HIP(hipGetLastError());
    return EF_OK;
}

int ef_token_logp(int64_t rows, int64_t vocab, int type, const void *logits, int64_t stride, const int64_t *tokens, float *logp,
                  void *stream)
{
    if (missing(rows, logp)) return EF_ERR_NULL;
    const int rc = policy_args(rows, vocab, type, logits, stride, tokens);
    if (rc) return rc;
    if (!aligned(logp, 4)) return EF_ERR_ALIGN;
    const Matrix in[2] = {{logits, stride, rows, vocab, type_size(type)}, vector_of(tokens, rows, 8)};
    const Matrix out[1] = {vector_of(logp, rows, 4)};
    const unsigned in_place[1] = {0u};
    if (!apart(out, 1, in, 2, in_place)) return EF_ERR_ARG;
    if (!rows) return EF_OK;
    ef::PolicyArgs a{};
    a.rows = rows;
    a.vocab = vocab;
    a.logits = logits;
    a.stride = stride;
    a.tokens = tokens;
    a.logp = logp;
    EF_BY_TYPE(type, T, policy_rows<T>(a, static_cast<hipStream_t>(stream)));
    EF_HIP(hipGetLastError());
    return EF_OK;
}

int ef_policy_loss(ef_workspace *workspace, int64_t rows, int64_t vocab, int type, const void *logits, int64_t stride,
                   const int64_t *tokens, const float *logp_old, const float *logp_ref, const float *advantage,
                   const float *token_weight, float clip_low, float clip_high, float kl, float *logp, float *losses, float *loss,
                   void *dlogits, int64_t dlogits_stride, void *stream)
{
    if (!workspace || missing(rows, advantage) || (rows && !logp && !losses && !loss && !dlogits)) return EF_ERR_NULL;
    int rc = policy_args(rows, vocab, type, logits, stride, tokens);
    if (rc) return rc;
    if (!(clip_low >= 0.0f && clip_low <= 1.0f) || !(std::isfinite(clip_high) && clip_high >= 0.0f) || !(std::isfinite(kl) && kl >= 0.0f))
        return EF_ERR_ARG;
    if (rows > workspace->max_rows) return EF_ERR_SIZE;
    const size_t size = type_size(type);
    const Matrix in[6] = {{logits, stride, rows, vocab, size}, vector_of(tokens, rows, 8),   vector_of(logp_old, rows, 4),
                          vector_of(logp_ref, rows, 4),        vector_of(advantage, rows, 4), vector_of(token_weight, rows, 4)};
    const Matrix out[4] = {{dlogits, dlogits_stride, rows, vocab, size}, vector_of(logp, rows, 4), vector_of(losses, rows, 4),
                           vector_of(loss, 1, 4)};
    if (dlogits && !out[0].good_stride()) return EF_ERR_ARG;
    if (!aligned(dlogits, size) || !aligned(logp_old, 4) || !aligned(logp_ref, 4) || !aligned(advantage, 4) || !aligned(token_weight, 4) ||
        !aligned(logp, 4) || !aligned(losses, 4) || !aligned(loss, 4))
        return EF_ERR_ALIGN;
    const unsigned in_place[4] = {1u, 0u, 0u, 0u};
    if (!apart(out, 4, in, 6, in_place)) return EF_ERR_ARG;
    rc = on_workspace_device(workspace);
    if (rc) return rc;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    float *row_losses = losses ? losses : workspace->row_sums;
    if (rows) {
        const ef::PolicyArgs a{rows, vocab, logits, stride, tokens, logp_old, logp_ref, advantage, token_weight, 1.0f - clip_low,
                               1.0f + clip_high, kl, logp, row_losses, dlogits, dlogits_stride, 1};
        if (rows <= ef::SLICED_ROWS && vocab > ef::SLICED_VOCAB) {
            EF_BY_TYPE(type, T, policy_slices<T>(a, workspace->parts, loss, s));
            EF_HIP(hipGetLastError());
            return EF_OK;
        }
        EF_BY_TYPE(type, T, policy_rows<T>(a, s));
        EF_HIP(hipGetLastError());
    }
    if (loss) {
        hipLaunchKernelGGL(ef::k_sum_losses, dim3(1), dim3(1024), 0, s, row_losses, rows, loss);
        EF_HIP(hipGetLastError());
    }
    return EF_OK;
}

}  // extern "C"
