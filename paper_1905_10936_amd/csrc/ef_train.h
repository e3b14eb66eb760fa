// Host side of the gated block, of drawing tokens and of clipping: argument checks, choice of kernel, launches.  Part of ef_api.hip, behind
// ef_layers.h, whose helpers it uses.
#pragma once
#include <new>
#include <vector>

#include "ef_clip.h"
#include "ef_gated.h"
#include "ef_layers.h"
#include "ef_sample.h"

namespace {

constexpr int64_t TILES_MAX = 0x1ffffff;

template <class T, int WC, int WT>
void launch_gated(ef::GatedArgs a, hipStream_t s)
{
    a.tiles_t = (int)ceil_div(a.rows, 64 * WT);
    a.tiles_c = (int)ceil_div(a.f, 32 * WC);
    hipLaunchKernelGGL((ef::k_gated<T, WC, WT>), dim3((unsigned)(a.tiles_t * a.tiles_c)), dim3(ef::PRODUCT_THREADS), 0, s, a);
}

template <class T, int CHANNELS>
void launch_gated_few(ef::GatedArgs a, hipStream_t s)
{
    a.tiles_t = (int)ceil_div(a.rows, 32);
    a.tiles_c = (int)ceil_div(a.f, CHANNELS);
    hipLaunchKernelGGL((ef::k_gated_few<T, CHANNELS>), dim3((unsigned)(a.tiles_t * a.tiles_c)), dim3(64 * ef::FEW_WAVES), 0, s, a);
}

constexpr int64_t FEW_ROWS = 64;

template <class T>
void launch_gated(const ef::GatedArgs &a, hipStream_t s)
{
    if (a.rows <= FEW_ROWS) {
        if (a.act.codes)
            launch_gated_few<T, 32>(a, s);
        else
            launch_gated_few<T, 16>(a, s);
    } else if (ceil_div(a.rows, 256) * ceil_div(a.f, 128) >= 192) {
        launch_gated<T, 4, 4>(a, s);
    } else {
        launch_gated<T, 2, 2>(a, s);
    }
}

// How the product of the backward pass is cut: the tile (64 wc channels by 64 wt tokens) and the parts along what is summed over.
struct InputCut {
    int wc, wt, splits;
};

// The least of a sum of what was measured (bf16, us): a step of a tile with all CUs at it, a workgroup's beginning and end, and for parts a launch more and their bytes at
// 4.5 TB/s.  fp32 steps take five times as long.
InputCut input_cut(int type, int64_t rows, int64_t n, int64_t steps)
{
    struct Shape { int wc, wt, on_cu; double step, base; };
    static constexpr Shape SHAPES[3] = {{4, 4, 1, 1.5, 10.0}, {4, 2, 1, 0.85, 7.0}, {2, 2, 2, 1.1, 6.0}};
    InputCut best{};
    double least = 0.0;
    for (const Shape &c : SHAPES) {
        const int64_t tiles = ceil_div(rows, 64 * c.wt) * ceil_div(n, 64 * c.wc), slots = 256 * c.on_cu;
        for (int64_t splits = 1; splits <= 64 && splits <= steps; ++splits) {
            if (splits > 1 && splits * rows * n > PART_FLOATS) break;
            const double rounds = (double)ceil_div(tiles * splits, slots);
            const double cost = rounds * ((double)ceil_div(steps, splits) * c.step * (type == EF_TYPE_BF16 ? 1.0 : 5.0) + c.base) +
                                (splits > 1 ? 4.0 + (double)(splits + 1) * (double)(rows * n) * 4.0 / 4.5e6 : 0.0);
            if (!best.splits || cost < least) {
                best = InputCut{c.wc, c.wt, (int)splits};
                least = cost;
            }
        }
    }
    return best;
}

template <class T, int WC, int WT>
void launch_input_grad(ef::InputGradArgs a, hipStream_t s)
{
    a.tiles_t = (int)ceil_div(a.rows, 64 * WT);
    a.tiles_c = (int)ceil_div(a.n, 64 * WC);
    hipLaunchKernelGGL((ef::k_input_grad<T, WC, WT>), dim3((unsigned)(a.tiles_t * a.tiles_c * a.splits)), dim3(ef::PRODUCT_THREADS), 0, s, a);
    if (a.splits > 1)
        hipLaunchKernelGGL(ef::k_join_input_grad<T>, dim3((unsigned)ceil_div(a.rows * ceil_div(a.n, 8), 256)), dim3(256), 0, s, a);
}

template <class T>
void launch_input_grad(ef::InputGradArgs a, hipStream_t s)
{
    const InputCut c = input_cut(sizeof(T) == 2 ? EF_TYPE_BF16 : EF_TYPE_FP32, a.rows, a.n, ceil_div(a.k, ef::STEP<T>));
    a.splits = c.splits;
    if (c.wc == 4 && c.wt == 4)
        launch_input_grad<T, 4, 4>(a, s);
    else if (c.wc == 4)
        launch_input_grad<T, 4, 2>(a, s);
    else
        launch_input_grad<T, 2, 2>(a, s);
}

template <class T, int LANES, int HELD>
void launch_sample(ef::SampleArgs a, hipStream_t s)
{
    using Of = ef::Team<LANES>;
    in_launches(ceil_div(a.rows, Of::TEAMS), [&](dim3 grid, int64_t first) {
        a.first = first * Of::TEAMS;
        hipLaunchKernelGGL((ef::k_sample<T, LANES, HELD>), grid, dim3(Of::THREADS), 0, s, a);
    });
}
// A wavefront takes rows of up to 2048, a workgroup longer ones: in 48 KB of LDS, which leaves room for a second one on the CU, in 128 KB, or from the caches.
template <class T>
void launch_sample(const ef::SampleArgs &a, hipStream_t s)
{
    constexpr int KB = 1024 / (int)sizeof(T);
    if (a.vocab <= 512)
        launch_sample<T, 64, 512>(a, s);
    else if (a.vocab <= 2048)
        launch_sample<T, 64, 2048>(a, s);
    else if (a.vocab <= 48 * KB)
        launch_sample<T, 1024, 48 * KB>(a, s);
    else if (a.vocab <= 128 * KB)
        launch_sample<T, 1024, 128 * KB>(a, s);
    else
        launch_sample<T, 1024, 0>(a, s);
}

int gated_sizes(int64_t rows, int64_t width, int64_t inner, int type, int gate)
{
    if (rows < 0 || rows > ROWS_MAX || width < 1 || inner < 1 || !good_type(type) || (gate != EF_GATE_SILU && gate != EF_GATE_GELU)) return EF_ERR_ARG;
    if (width > WIDTH_MAX || inner > WIDTH_MAX || ceil_div(rows, 64) * ceil_div(std::max(width, inner), 16) > TILES_MAX) return EF_ERR_SIZE;
    return EF_OK;
}

int good_matrices(std::initializer_list<const Matrix *> ms)
{
    for (const Matrix *m : ms)
        if (m->p && !m->good_stride()) return EF_ERR_ARG;
    for (const Matrix *m : ms)
        if (!aligned(m->p, m->size)) return EF_ERR_ALIGN;
    return EF_OK;
}

}  // namespace

extern "C" {

int ef_gated_forward(int64_t rows, int64_t width, int64_t inner, int type, const void *x, int64_t x_stride, const void *w, int64_t w_stride,
                     int gate, void *pre, int64_t pre_stride, void *z, int64_t z_stride, void *act, void *stream)
{
    if (missing(rows, x, w) || (rows && !pre && !z && !act)) return EF_ERR_NULL;
    int rc = gated_sizes(rows, width, inner, type, gate);
    if (rc) return rc;
    const size_t size = type_size(type);
    const Matrix in[2] = {{x, x_stride, rows, width, size}, {w, w_stride, 2 * inner, width, size}};
    const Matrix out[3] = {{pre, pre_stride, rows, 2 * inner, size}, {z, z_stride, rows, inner, size},
                           vector_of(act, (int64_t)ef_act_bytes(rows, inner), 1)};
    rc = good_matrices({&in[0], &in[1], &out[0], &out[1]});
    if (rc) return rc;
    if (!aligned(act, 16)) return EF_ERR_ALIGN;
    const unsigned in_place[3] = {0u, 0u, 0u};
    if (!apart(out, 3, in, 2, in_place)) return EF_ERR_ARG;
    if (!rows) return EF_OK;
    const ef::GatedArgs a{rows, width, inner, x, x_stride, w, w_stride, gate, pre, pre_stride, z, z_stride, act_ref(act, rows, inner), 0, 0};
    EF_BY_TYPE(type, T, launch_gated<T>(a, static_cast<hipStream_t>(stream)));
    EF_HIP(hipGetLastError());
    return EF_OK;
}

int ef_gated_backward(ef_workspace *workspace, int64_t rows, int64_t width, int64_t inner, int type, const void *dz, int64_t dz_stride,
                      const void *pre, int64_t pre_stride, const void *w, int64_t w_stride, int gate, void *dpre, int64_t dpre_stride, void *dx,
                      int64_t dx_stride, void *stream)
{
    if (!workspace || missing(rows, dz, pre, dpre) || (rows && dx && !w)) return EF_ERR_NULL;
    int rc = gated_sizes(rows, width, inner, type, gate);
    if (rc) return rc;
    if (rows > workspace->max_rows) return EF_ERR_SIZE;
    const size_t size = type_size(type);
    const Matrix in[3] = {{dz, dz_stride, rows, inner, size}, {pre, pre_stride, rows, 2 * inner, size}, {w, w_stride, 2 * inner, width, size}};
    const Matrix out[2] = {{dpre, dpre_stride, rows, 2 * inner, size}, {dx, dx_stride, rows, width, size}};
    rc = good_matrices({&in[0], &in[1], &in[2], &out[0], &out[1]});
    if (rc) return rc;
    const unsigned in_place[2] = {2u, 0u};
    if (!apart(out, 2, in, 3, in_place)) return EF_ERR_ARG;
    rc = on_workspace_device(workspace);
    if (rc || !rows) return rc;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    in_launches(ceil_div(rows * ceil_div(inner, 8), 256), [&](dim3 grid, int64_t first) {
        const ef::SlopeArgs a{rows, inner, dz, dz_stride, pre, pre_stride, dpre, dpre_stride, gate, first * 256};
        EF_BY_TYPE(type, T, hipLaunchKernelGGL(ef::k_gated_slopes<T>, grid, dim3(256), 0, s, a));
    });
    EF_HIP(hipGetLastError());
    if (!dx) return EF_OK;
    const ef::InputGradArgs a{rows, width, 2 * inner, dpre, dpre_stride, w, w_stride, dx, dx_stride, 0, 0, 1, workspace->parts};
    EF_BY_TYPE(type, T, launch_input_grad<T>(a, s));
    EF_HIP(hipGetLastError());
    return EF_OK;
}

int ef_sample_tokens(ef_workspace *workspace, int64_t rows, int64_t vocab, int type, const void *logits, int64_t stride, const float *uniform,
                     const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p, int64_t *tokens, float *logp,
                     void *stream)
{
    if (!workspace || missing(rows, uniform)) return EF_ERR_NULL;
    int rc = policy_args(rows, vocab, type, logits, stride, tokens);
    if (rc) return rc;
    if (rows > workspace->max_rows) return EF_ERR_SIZE;
    for (const void *p : {(const void *)uniform, (const void *)temperature, (const void *)top_k, (const void *)top_p, (const void *)min_p, (const void *)logp})
        if (!aligned(p, 4)) return EF_ERR_ALIGN;
    const Matrix in[6] = {{logits, stride, rows, vocab, type_size(type)}, vector_of(uniform, rows, 4), vector_of(temperature, rows, 4),
                          vector_of(top_k, rows, 4), vector_of(top_p, rows, 4), vector_of(min_p, rows, 4)};
    const Matrix out[2] = {vector_of(tokens, rows, 8), vector_of(logp, rows, 4)};
    const unsigned in_place[2] = {0u, 0u};
    if (!apart(out, 2, in, 6, in_place)) return EF_ERR_ARG;
    rc = on_workspace_device(workspace);
    if (rc || !rows) return rc;
    const ef::SampleArgs a{0, rows, vocab, logits, stride, uniform, temperature, top_k, top_p, min_p, tokens, logp};
    EF_BY_TYPE(type, T, launch_sample<T>(a, static_cast<hipStream_t>(stream)));
    EF_HIP(hipGetLastError());
    return EF_OK;
}

int ef_grad_clip(ef_workspace *workspace, int n_workers, int64_t n_tensors, void *const *grads, const int64_t *sizes, const int *types, float max_norm,
                 float *flat, int64_t flat_stride, float *norm, void *stream)
try {
    if (!workspace || !norm) return EF_ERR_NULL;
    if (n_workers < 1 || n_tensors < 0 || n_tensors > (1 << 20) || !(max_norm >= 0.0f)) return EF_ERR_ARG;
    if (n_tensors && (!grads || !sizes || !types)) return EF_ERR_NULL;
    int64_t total = 0;
    for (int64_t i = 0; i < n_tensors; ++i) {
        if (sizes[i] < 0 || !good_type(types[i])) return EF_ERR_ARG;
        if (sizes[i] > (int64_t)1 << 50) return EF_ERR_SIZE;
        total += sizes[i];
        if (total > (int64_t)1 << 50) return EF_ERR_SIZE;
        for (int w = 0; w < n_workers; ++w) {
            const void *p = grads[(int64_t)w * n_tensors + i];
            if (!p && sizes[i]) return EF_ERR_NULL;
            if (!aligned(p, type_size(types[i]))) return EF_ERR_ALIGN;
        }
    }
    if (flat && n_workers > 1 && (flat_stride < total || flat_stride > INT64_MAX / 8 / n_workers)) return EF_ERR_ARG;
    if (!aligned(flat, 4) || !aligned(norm, 4)) return EF_ERR_ALIGN;
    // What is written shares nothing with what else is read or written: a list of spans by address, each marked as written or read.
    struct Span { uintptr_t begin, end; bool written; };
    std::vector<Span> spans;
    spans.reserve((size_t)n_workers * ((size_t)n_tensors + 1) + 1);
    const auto span = [&](const void *p, size_t bytes, bool written) {
        if (p && bytes) spans.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, written});
    };
    for (int w = 0; w < n_workers; ++w) {
        for (int64_t i = 0; i < n_tensors; ++i) span(grads[(int64_t)w * n_tensors + i], (size_t)sizes[i] * type_size(types[i]), !flat);
        if (flat) span(flat + (int64_t)w * (n_workers > 1 ? flat_stride : 0), (size_t)total * 4, true);
    }
    span(norm, (size_t)n_workers * 4, true);
    std::sort(spans.begin(), spans.end(), [](const Span &a, const Span &b) { return a.begin < b.begin; });
    uintptr_t read_end = 0, written_end = 0;
    for (const Span &s : spans) {
        if (s.begin < written_end || (s.written && s.begin < read_end)) return EF_ERR_ARG;
        (s.written ? written_end : read_end) = std::max(s.written ? written_end : read_end, s.end);
    }
    const int rc = on_workspace_device(workspace);
    if (rc) return rc;

    // Tensors that follow one another in memory for every worker are one.
    struct Entry { int64_t place; int64_t tensor; };
    std::vector<Entry> entries;
    entries.reserve((size_t)n_tensors);
    for (int64_t i = 0, place = 0, before = -1; i < n_tensors; place += sizes[i], ++i) {
        if (!sizes[i]) continue;
        bool next = before >= 0 && types[before] == types[i];
        for (int w = 0; w < n_workers && next; ++w)
            next = static_cast<char *>(grads[(int64_t)w * n_tensors + before]) + sizes[before] * (int64_t)type_size(types[i]) == grads[(int64_t)w * n_tensors + i];
        if (!next) entries.push_back({place, i});
        before = i;
    }
    const int64_t n = (int64_t)entries.size(), words = n * (n_workers + 1), count = std::max<int64_t>(1, total);
    ef::ClipArgs a;
    a.length = total;
    // Chunks of 2048 to 16384 places; workgroups for 4096 in all, or 2048 for a worker.
    a.chunk = std::min<int64_t>(ef::CLIP_MOST, ceil_div(count, (int64_t)ef::CLIP_GROUPS * ef::CLIP_LEAST) * ef::CLIP_LEAST);
    const int64_t groups = std::min<int64_t>(ceil_div(count, a.chunk), std::max<int64_t>(256, std::min<int64_t>(ef::CLIP_GROUPS, 2 * ef::CLIP_GROUPS / n_workers)));
    if (words + groups * n_workers > PART_FLOATS / 2 || words > 0x7fffffff || n_workers > 0xffff) return EF_ERR_SIZE;
    a.tensors = (int)n;
    a.sums = reinterpret_cast<double *>(workspace->parts);
    a.flat = flat;
    a.flat_stride = n_workers > 1 ? flat_stride : 0;
    a.norm = norm;
    a.max_norm = max_norm;
    const auto word = [&](int64_t i) {
        if (i < n) return (uint64_t)entries[(size_t)i].place;
        const int64_t tensor = entries[(size_t)(i % n)].tensor;
        return reinterpret_cast<uint64_t>(grads[(i / n - 1) * n_tensors + tensor]) | (types[tensor] == EF_TYPE_FP32 ? 1 : 0);
    };
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)groups, (unsigned)n_workers), threads(ef::CLIP_THREADS);
    if (words <= ef::CLIP_WORDS) {
        ef::ClipDirect d;
        d.a = a;
        for (int64_t i = 0; i < words; ++i) d.words[i] = word(i);
        hipLaunchKernelGGL(ef::k_clip_norm<ef::ClipDirect>, grid, threads, 0, s, d);
        hipLaunchKernelGGL(ef::k_clip_scale<ef::ClipDirect>, grid, threads, 0, s, d);
    } else {
        ef::ClipListed l;
        l.a = a;
        uint64_t *const to = reinterpret_cast<uint64_t *>(workspace->parts) + groups * n_workers;
        l.words = to;
        for (int64_t i = 0; i < words; i += ef::CLIP_WORDS) {
            ef::ClipWords w;
            w.to = to + i;
            w.n = (int)std::min<int64_t>(ef::CLIP_WORDS, words - i);
            for (int k = 0; k < w.n; ++k) w.words[k] = word(i + k);
            hipLaunchKernelGGL(ef::k_clip_words, dim3(1), dim3(ef::CLIP_WORDS), 0, s, w);
        }
        hipLaunchKernelGGL(ef::k_clip_norm<ef::ClipListed>, grid, threads, 0, s, l);
        hipLaunchKernelGGL(ef::k_clip_scale<ef::ClipListed>, grid, threads, 0, s, l);
    }
    EF_HIP(hipGetLastError());
    return EF_OK;
} catch (const std::bad_alloc &) {
    return EF_ERR_SIZE;
}

}  // extern "C"
