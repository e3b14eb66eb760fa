// Checkpoints of activations in 8 bits: writing and reading one.
//
// Bound by memory: an element's two or four bytes one way and 33/32 bytes the other.  A thread takes eight elements, so that
// a row of any length and start is read and written in 128-bit (bf16) accesses; the four threads of a group find its
// scale among themselves.  16384 x 4096 in bf16: 38 us either way, 5.3 TB/s, where a copy of 1 GiB reaches 5.1.
#pragma once
#include "ef_rows.h"

namespace ef {

constexpr int ACT_THREADS = 256;

// One thread to eight elements of the padded rows, rows one after the other, from the `first` eight on.
template <class T>
__global__ __launch_bounds__(ACT_THREADS) void k_act_encode(const T *x, int64_t stride, int64_t rows, int64_t n, ActRef act,
                                                             int64_t first)
{
    const int64_t per_row = act.groups * (GROUP / 8), at = first + (int64_t)blockIdx.x * ACT_THREADS + threadIdx.x;
    const int64_t row = at / per_row, i = (at - row * per_row) * 8;
    if (row >= rows) return;            // whole groups: four lanes at a time
    Eight<T> e;
    load_some(e, x + row * stride + i, n - i, 0u);
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = e[k];
    act.put(row, i, n, v);
}

template <class T>
__global__ __launch_bounds__(ACT_THREADS) void k_act_decode(ActRef act, int64_t rows, int64_t n, T *y, int64_t stride,
                                                             int64_t first)
{
    const int64_t per_row = act.groups * (GROUP / 8), at = first + (int64_t)blockIdx.x * ACT_THREADS + threadIdx.x;
    const int64_t row = at / per_row, i = (at - row * per_row) * 8;
    if (row >= rows) return;
    float v[8];
    act.get(row, i, v);
    Eight<T> e;
    e.round(v);
    store_some(e, y + row * stride + i, n - i);
}

}  // namespace ef
