// Host side of the gated block, of drawing tokens and of clipping: argument checks, choice of kernel, launches.  Part of ef_api.hip, behind
// ef_layers.h, whose helpers it uses.
#pragma once
#include <new>
#include <utility>
#include <vector>

#include "ef_clip.h"
#include "ef_gated.h"
#include "ef_layers.h"
#include "ef_sample.h"

namespace {

constexpr int64_t TILES_MAX = 1 << 22;          // tiles to a launch of a product: a grid holds less than 2^32 threads
// Tokens to a launch: no more than 2^22, and no more than the largest tiles (256 tokens by 128 channels) take.
int64_t rows_at_once(int64_t channels) { return std::min(TILES_MAX / ceil_div(channels, 128) * 256, (int64_t)1 << 22); }

// A tile of a product, 64 wc channels by 64 wt tokens, and what it was measured to take: a step (128 bytes of what is summed over) `alone` us with few workgroups
// on the GPU and `loaded` us with as many as it holds (`most` on a CU; more slow the others down with the square of their share), a workgroup's beginning
// and end `over`.
struct TileShape {
    int wc, wt, most;
    double alone, loaded, over;
    // `groups` workgroups of `steps` each
    double cost(int64_t groups, int64_t steps) const
    {
        const int64_t round = 256 * most, full = groups / round, rest = groups % round;
        const double share = (double)rest / (double)round;
        return 3.0 + (double)full * ((double)steps * loaded + over) + (rest ? (double)steps * (alone + (loaded - alone) * share * share) + over : 0.0);
    }
};

// What ef_gated_kernels has set.
struct GatedChoice {
    int forward = -1, backward = -1, splits = 0;
};
thread_local GatedChoice gated_choice;

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

// The least of the costs, the same whatever outputs are asked for: each then has the same bits.  1024 -> 4096 channels in bf16, us for 32, 128, 512, 1024 and 2048 tokens: few tokens 7.5, 24, 80; tiles of 64 tokens 9.0, 9.1, 14.4, 25.5, 47;
// of 128 10.7, 11.2, 13.2, 21.1, 38; of 256 23, 28, 27, 29.5, 36.  In fp32 15, 46, 158; 38, 39, 74, 147, 274; 66, 67, 73, 139, 258; 235 to 253.
template <class T>
void launch_gated(const ef::GatedArgs &a, hipStream_t s)
{
    static constexpr TileShape SHAPES[2][3] = {{{4, 4, 1, 7.1, 7.5, 7.0}, {2, 2, 2, 1.9, 4.2, 1.5}, {2, 1, 2, 1.05, 2.15, 1.0}},
                                               {{4, 4, 1, 0.9, 1.5, 7.0}, {2, 2, 2, 0.38, 1.1, 1.5}, {2, 1, 2, 0.3, 0.63, 1.0}}};
    const int64_t steps = ceil_div(a.n, ef::STEP<T>);
    const double round = sizeof(T) == 2 ? 1.6 + 3.9 * (double)a.n / 1024.0 : 1.5 + 9.5 * (double)a.n / 1024.0;
    const int64_t few = ceil_div(a.rows, 32) * ceil_div(a.f, 16);
    double least = few <= TILES_MAX ? 1.5 + round * (double)ceil_div(few, 256) : 1e30;
    int best = -1, asked = gated_choice.forward == 0 && few > TILES_MAX ? -1 : gated_choice.forward;
    for (int i = 0; i < 3; ++i) {
        const TileShape &c = SHAPES[sizeof(T) == 2][i];
        const int64_t tiles = ceil_div(a.rows, 64 * c.wt) * ceil_div(a.f, 32 * c.wc);
        const double cost = c.cost(tiles, steps);
        if (cost < least && tiles <= TILES_MAX) {
            least = cost;
            best = i;
        }
        if (asked == i + 1 && tiles > TILES_MAX) asked = -1;
    }
    if (asked >= 0) best = asked - 1;
    if (best == 0)
        launch_gated<T, 4, 4>(a, s);
    else if (best == 1)
        launch_gated<T, 2, 2>(a, s);
    else if (best == 2)
        launch_gated<T, 2, 1>(a, s);
    else if (a.act.codes)
        launch_gated_few<T, 32>(a, s);
    else
        launch_gated_few<T, 16>(a, s);
}

// How the product of the backward pass is cut: the tile and the parts along what is summed over; parts cost a launch more and their bytes at 4.5 TB/s.  us, each
// tile with its best number of parts, 256 x 256, 256 x 128, 128 x 128 and 64 x 64: bf16, 8192 summed over, 4096 x 1024 86, 76, 77, 102; 300 x 2048 33, 28, 27, 25; 64 x 1024 26,
// 20, 16, 13; fp32, 2062 summed over, 777 x 515 77, 54, 46, 32.
struct InputCut {
    int wc, wt, splits;
};
InputCut input_cut(int type, int64_t rows, int64_t n, int64_t steps)
{
    static constexpr TileShape SHAPES[2][4] = {{{4, 4, 1, 7.1, 7.3, 7.0}, {4, 2, 1, 3.7, 3.8, 5.0}, {2, 2, 2, 2.0, 3.8, 2.0}, {1, 1, 4, 0.57, 1.9, 1.0}},
                                               {{4, 4, 1, 1.1, 1.5, 7.0}, {4, 2, 1, 0.65, 0.95, 5.0}, {2, 2, 2, 0.43, 1.1, 2.0}, {1, 1, 4, 0.28, 0.84, 1.0}}};
    const auto tiles_of = [&](const TileShape &c) { return ceil_div(rows, 64 * c.wt) * ceil_div(n, 64 * c.wc); };
    const TileShape *const shapes = SHAPES[type == EF_TYPE_BF16], *const asked = gated_choice.backward >= 0 ? shapes + gated_choice.backward : nullptr;
    InputCut best{};
    double least = 0.0;
    for (const TileShape &c : SHAPES[type == EF_TYPE_BF16]) {
        if (asked && &c != asked && tiles_of(*asked) <= TILES_MAX) continue;
        const int64_t tiles = tiles_of(c);
        if (tiles > TILES_MAX) continue;
        for (int64_t splits = 1; splits <= 64 && splits <= steps; ++splits) {
            if (splits > 1 && splits * rows * n > PART_FLOATS) break;
            const double cost = c.cost(tiles * splits, ceil_div(steps, splits)) +
                                (splits > 1 ? 4.0 + (double)(splits + 1) * (double)(rows * n) * 4.0 / 4.5e6 : 0.0);
            if (!best.splits || cost < least || splits <= gated_choice.splits) {
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
    if (c.wt == 4)
        launch_input_grad<T, 4, 4>(a, s);
    else if (c.wc == 4)
        launch_input_grad<T, 4, 2>(a, s);
    else if (c.wc == 2)
        launch_input_grad<T, 2, 2>(a, s);
    else
        launch_input_grad<T, 1, 1>(a, s);
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
// Rows of up to 512 are a wavefront's, and so are rows of up to 2048 where there are more of them than CUs; longer ones are a workgroup's, in 128 KB of LDS or from the
// caches.  us with logp, each way (wavefront, workgroup): 4096 x 2048 in bf16 without a filter 23, 80, with top-k 50 36, 160; 256 x 2048 9.0, 6.1 and 17, 12; 1 x 1024 with top-k 50 and
// top-p 14, 11.  (LDS, caches): 256 x 50257 in bf16 with top-p 52, 65; 1024 x 32000 in fp32 125, 141.  Many rows of just over 2048 pay for it: 4096 x 2049 takes 87 without a filter and 164 with top-k 50.  With 48 KB of LDS rows of 20000 in bf16 took as long as with 128.
template <class T>
void launch_sample(const ef::SampleArgs &a, hipStream_t s)
{
    constexpr int KB = 1024 / (int)sizeof(T), CUS = 256;
    if (a.vocab <= 512)
        launch_sample<T, 64, 512>(a, s);
    else if (a.vocab <= 2048 && a.rows > CUS)
        launch_sample<T, 64, 2048>(a, s);
    else if (a.vocab <= 128 * KB)
        launch_sample<T, 1024, 128 * KB>(a, s);
    else
        launch_sample<T, 1024, 0>(a, s);
}

int gated_sizes(int64_t rows, int64_t width, int64_t inner, int type, int gate)
{
    if (rows < 0 || rows > ROWS_MAX || width < 1 || inner < 1 || !good_type(type) || (gate != EF_GATE_SILU && gate != EF_GATE_GELU)) return EF_ERR_ARG;
    return width > WIDTH_MAX || inner > WIDTH_MAX ? EF_ERR_SIZE : EF_OK;
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
    const ef::ActRef whole = act_ref(act, rows, inner);
    const int64_t most = rows_at_once(inner);
    for (int64_t first = 0; first < rows; first += most) {
        const auto from = [&](auto *p, int64_t stride) { return p ? reinterpret_cast<decltype(p)>(reinterpret_cast<uintptr_t>(p) + (size_t)(first * stride) * size) : p; };
        ef::ActRef part = whole;
        if (act) {
            part.codes = whole.code_at(first, 0);
            part.scales = whole.scale_at(first, 0);
        }
        const ef::GatedArgs a{std::min(rows - first, most), width, inner, from(x, x_stride), x_stride, w, w_stride, gate, from(pre, pre_stride), pre_stride,
                              from(z, z_stride), z_stride, part, 0, 0};
        EF_BY_TYPE(type, T, launch_gated<T>(a, static_cast<hipStream_t>(stream)));
    }
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
    const int64_t most = rows_at_once(width);
    for (int64_t first = 0; first < rows; first += most) {
        const auto from = [&](void *p, int64_t stride) { return static_cast<void *>(static_cast<char *>(p) + (size_t)(first * stride) * size); };
        const ef::InputGradArgs a{std::min(rows - first, most), width, 2 * inner, from(dpre, dpre_stride), dpre_stride, w, w_stride, from(dx, dx_stride), dx_stride, 0, 0, 1,
                                  workspace->parts};
        EF_BY_TYPE(type, T, launch_input_grad<T>(a, s));
    }
    EF_HIP(hipGetLastError());
    return EF_OK;
}

int ef_gated_kernels(int forward, int backward, int splits)
{
    if (forward < -1 || forward > 3 || backward < -1 || backward > 3 || splits < 0 || splits > 64) return EF_ERR_ARG;
    gated_choice = GatedChoice{forward, backward, splits};
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
    if (n_workers > 0xffff) return EF_ERR_SIZE;
    if (flat && n_workers > 1 && (flat_stride < total || flat_stride > INT64_MAX / 8 / n_workers)) return EF_ERR_ARG;
    if (!aligned(flat, 4) || !aligned(norm, 4)) return EF_ERR_ALIGN;
    // What is written shares nothing with what else is read or written.
    const size_t norm_bytes = (size_t)n_workers * 4, row_bytes = (size_t)total * 4;
    const int64_t stride = n_workers > 1 ? flat_stride : 0;
    const size_t flat_bytes = (size_t)(n_workers - 1) * (size_t)stride * 4 + row_bytes;
    const auto bytes_of = [&](int64_t i) { return (size_t)sizes[i] * type_size(types[i]); };
    for (int64_t i = 0; i < n_tensors * n_workers; ++i) {
        const void *p = grads[i];
        const size_t bytes = bytes_of(i % n_tensors);
        if (!bytes) continue;
        if (overlap(p, bytes, norm, norm_bytes)) return EF_ERR_ARG;
        if (flat && overlap(p, bytes, flat, flat_bytes))
            for (int w = 0; w < n_workers; ++w)
                if (row_bytes && overlap(p, bytes, flat + w * stride, row_bytes)) return EF_ERR_ARG;
    }
    for (int w = 0; flat && w < n_workers; ++w)
        if (row_bytes && overlap(norm, norm_bytes, flat + w * stride, row_bytes)) return EF_ERR_ARG;
    if (!flat) {
        // in place: no two tensors share anything
        std::vector<std::pair<uintptr_t, uintptr_t>> spans;
        spans.reserve((size_t)(n_tensors * n_workers));
        for (int64_t i = 0; i < n_tensors * n_workers; ++i)
            if (sizes[i % n_tensors]) spans.emplace_back(reinterpret_cast<uintptr_t>(grads[i]), reinterpret_cast<uintptr_t>(grads[i]) + bytes_of(i % n_tensors));
        std::sort(spans.begin(), spans.end());
        for (size_t i = 1; i < spans.size(); ++i)
            if (spans[i].first < spans[i - 1].second) return EF_ERR_ARG;
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
    if (words + groups * n_workers > PART_FLOATS / 2 || words > 0x7fffffff) return EF_ERR_SIZE;
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
