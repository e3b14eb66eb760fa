// What the kernels over rows of activations and logits share: loads and stores of eight elements at any alignment, sums over
// the lanes that hold a row, and the 8-bit format of checkpoints.
//
// A lane holds eight consecutive elements of a row at a time (16 bytes of bf16, 32 of fp32), so four lanes hold a checkpoint's
// group of 32.  Rows start wherever their stride puts them: accesses are 128 bits wide at the element's alignment, which global
// memory allows; what the row's end cuts is read one by one.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>
#include <utility>

namespace ef {

#define EF_GLOBAL __attribute__((address_space(1)))

constexpr int GROUP = 32;       // elements to a scale

struct bf16_t { uint16_t bits; };

typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned u32x4_word __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Keeps an offset 32 bits wide up to where it is used: an access then adds it to a scalar base itself.
__device__ __forceinline__ void stay(unsigned &off) { asm volatile("" : "+v"(off)); }
__device__ __forceinline__ unsigned here(unsigned off)
{
    stay(off);
    return off;
}

// Eight elements as they lie in memory.  load_at, store_at: at a base that is the same for the wavefront and a lane's bytes from there.
template <class T>
struct Eight;
template <>
struct Eight<bf16_t> {
    u32x4 w;
    __device__ __forceinline__ void load(const bf16_t *p) { w = *reinterpret_cast<const u32x4_any *>(p); }
    __device__ __forceinline__ void store(bf16_t *p) const { *reinterpret_cast<u32x4_any *>(p) = w; }
    __device__ __forceinline__ void load_at(const void *base, unsigned off) { w = *(const EF_GLOBAL u32x4_any *)((const EF_GLOBAL char *)base + here(off)); }
    __device__ __forceinline__ void store_at(void *base, unsigned off) const { *(EF_GLOBAL u32x4_any *)((EF_GLOBAL char *)base + here(off)) = w; }
    __device__ __forceinline__ void fill(unsigned two) { w = u32x4{two, two, two, two}; }
    __device__ __forceinline__ float operator[](int i) const
    {
        return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    __device__ __forceinline__ void set(int i, unsigned bits)
    {
        w[i / 2] = i & 1 ? (w[i / 2] & 0xffffu) | bits << 16 : (w[i / 2] & 0xffff0000u) | bits;
    }
    // rounded to nearest even
    __device__ __forceinline__ void round(const float *v)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bf16x2 t = {(__bf16)v[2 * i], (__bf16)v[2 * i + 1]};
            w[i] = __builtin_bit_cast(unsigned, t);
        }
    }
};
template <>
struct Eight<float> {
    u32x4 lo, hi;
    __device__ __forceinline__ void load(const float *p)
    {
        lo = *reinterpret_cast<const u32x4_word *>(p);
        hi = *reinterpret_cast<const u32x4_word *>(p + 4);
    }
    __device__ __forceinline__ void store(float *p) const
    {
        *reinterpret_cast<u32x4_word *>(p) = lo;
        *reinterpret_cast<u32x4_word *>(p + 4) = hi;
    }
    __device__ __forceinline__ void load_at(const void *base, unsigned off)
    {
        const EF_GLOBAL char *p = (const EF_GLOBAL char *)base + here(off);
        lo = *(const EF_GLOBAL u32x4_word *)p;
        hi = *(const EF_GLOBAL u32x4_word *)(p + 16);
    }
    __device__ __forceinline__ void store_at(void *base, unsigned off) const
    {
        EF_GLOBAL char *p = (EF_GLOBAL char *)base + here(off);
        *(EF_GLOBAL u32x4_word *)p = lo;
        *(EF_GLOBAL u32x4_word *)(p + 16) = hi;
    }
    __device__ __forceinline__ void fill(unsigned one) { lo = hi = u32x4{one, one, one, one}; }
    __device__ __forceinline__ float operator[](int i) const { return __uint_as_float(i < 4 ? lo[i & 3] : hi[i & 3]); }
    __device__ __forceinline__ void set(int i, unsigned bits)
    {
        if (i < 4)
            lo[i & 3] = bits;
        else
            hi[i & 3] = bits;
    }
    __device__ __forceinline__ void round(const float *v)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo[i] = __float_as_uint(v[i]);
            hi[i] = __float_as_uint(v[4 + i]);
        }
    }
};

template <class T>
__device__ __forceinline__ unsigned element_bits(const T *p);
template <>
__device__ __forceinline__ unsigned element_bits<bf16_t>(const bf16_t *p) { return p->bits; }
template <>
__device__ __forceinline__ unsigned element_bits<float>(const float *p) { return __float_as_uint(*p); }

template <class T>
__device__ __forceinline__ void put_element(T *p, const Eight<T> &e, int i);
template <>
__device__ __forceinline__ void put_element<bf16_t>(bf16_t *p, const Eight<bf16_t> &e, int i)
{
    p->bits = (uint16_t)(i & 1 ? e.w[i / 2] >> 16 : e.w[i / 2] & 0xffffu);
}
template <>
__device__ __forceinline__ void put_element<float>(float *p, const Eight<float> &e, int i) { *p = e[i]; }

template <class T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_float<bf16_t>(bf16_t v) { return __uint_as_float((unsigned)v.bits << 16); }

template <class T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16_t from_float<bf16_t>(float v) { return bf16_t{__builtin_bit_cast(uint16_t, (__bf16)v)}; }

// The first `left` (any number, also none or less) of eight elements at p; `other` (a bit pattern; bf16: twice) for the rest.  A row's last elements are
// asked for one by one, all at once.
template <class T>
__device__ __forceinline__ void load_some(Eight<T> &e, const T *p, int64_t left, unsigned other)
{
    if (left >= 8) {
        e.load(p);
    } else {
        e.fill(other);
        if (left > 0) {
            const int n = (int)left;
            unsigned b[7];
#pragma unroll
            for (int i = 0; i < 7; ++i) b[i] = element_bits(p + min(i, n - 1));
#pragma unroll
            for (int i = 0; i < 7; ++i)
                e.set(i, i < n ? b[i] : sizeof(T) == 2 ? other & 0xffffu : other);
        }
    }
}
template <class T>
__device__ __forceinline__ void store_some(const Eight<T> &e, T *p, int64_t left)
{
    if (left >= 8) {
        e.store(p);
    } else if (left > 0) {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < left) put_element(p + i, e, i);
    }
}

// The same where LAST is set; else all eight are there.
template <bool LAST, class T>
__device__ __forceinline__ void load_piece(Eight<T> &e, const T *p, int64_t left)
{
    if constexpr (LAST)
        load_some(e, p, left, 0u);
    else
        e.load(p);
}
template <bool LAST, class T>
__device__ __forceinline__ void store_piece(const Eight<T> &e, T *p, int64_t left)
{
    if constexpr (LAST)
        store_some(e, p, left);
    else
        e.store(p);
}

template <class F, int... I>
__device__ __forceinline__ void times(F f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>()), ...); }
// f(0), f(1), ... f(N - 1), the index known to the compiler
template <int N, class F>
__device__ __forceinline__ void times(F f) { times(f, std::make_integer_sequence<int, N>()); }

// ------------------------------------------------------------------------------- sums over a row's lanes ---

template <int CTRL>
__device__ __forceinline__ float lane_move(float v)
{
    return __uint_as_float((unsigned)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;

struct Add { static __device__ __forceinline__ float of(float a, float b) { return a + b; } };
struct Max { static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); } };

// Over WIDTH = 4, 16 or 64 neighbouring lanes, in a fixed order; every one of them ends with the result.
template <class Op, int WIDTH>
__device__ __forceinline__ float over_lanes(float v)
{
    v = Op::of(v, lane_move<DPP_XOR1>(v));
    v = Op::of(v, lane_move<DPP_XOR2>(v));
    if constexpr (WIDTH >= 16) {
        v = Op::of(v, lane_move<DPP_HALF_MIRROR>(v));
        v = Op::of(v, lane_move<DPP_MIRROR>(v));
    }
    if constexpr (WIDTH == 64) {
        u32x2 t = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = Op::of(__uint_as_float(t.x), __uint_as_float(t.y));
        t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = Op::of(__uint_as_float(t.x), __uint_as_float(t.y));
    }
    return v;
}

// Over the LANES threads that hold a row; with more than 64 they are the whole workgroup and meet at a barrier.  `at`: LANES / 64 floats
// of shared memory that nobody else touches before the next barrier but one.
template <class Op, int LANES>
__device__ __forceinline__ float over_row(float v, float *at)
{
    if constexpr (LANES <= 64) {
        return over_lanes<Op, LANES>(v);
    } else {
        v = over_lanes<Op, 64>(v);
        if (threadIdx.x % 64 == 0) at[threadIdx.x / 64] = v;
        __syncthreads();
        // 4, 8 or 16 wavefronts: each lane takes one of their results, the lanes of a row of 16 then have all of them
        v = at[threadIdx.x % (LANES / 64)];
        v = Op::of(v, lane_move<DPP_XOR1>(v));
        v = Op::of(v, lane_move<DPP_XOR2>(v));
        if constexpr (LANES >= 512) v = Op::of(v, lane_move<DPP_HALF_MIRROR>(v));
        if constexpr (LANES >= 1024) v = Op::of(v, lane_move<DPP_MIRROR>(v));
        return v;
    }
}

// ---------------------------------------------------------------------------------- the 8-bit format ---

// Scale byte of a group whose largest magnitude is `top`: 2^e >= top / 448 = top / (1.75 * 2^8), the least such power.  Adding
// 2^21 - 1 to the fraction carries into the exponent just if it is above .75.  NaN if the group holds an infinity or NaN: `top` has to show it.
constexpr unsigned SCALE_MIN = 127 - 117, SCALE_MAX = 127 + 119, SCALE_NAN = 255, CODE_NAN = 0x7f;
__device__ __forceinline__ unsigned scale_byte(float top)
{
    const unsigned b = __float_as_uint(top);
    if (b >= 0x7f800000u) return SCALE_NAN;
    const int e = (int)((b + 0x1fffffu) >> 23) - 8;
    return (unsigned)min(max(e, (int)SCALE_MIN), (int)SCALE_MAX);
}
// The larger of two magnitudes as bit patterns (no sign): infinities and NaN are larger than any number.
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }
template <int CTRL>
__device__ __forceinline__ unsigned lane_bits(unsigned v)
{
    return (unsigned)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}
// Scale byte of the group that four neighbouring lanes hold, eight values each.
__device__ __forceinline__ unsigned group_scale(const float *v)
{
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = larger(top, __float_as_uint(v[i]) & 0x7fffffffu);
    top = larger(top, lane_bits<DPP_XOR1>(top));
    top = larger(top, lane_bits<DPP_XOR2>(top));
    return scale_byte(__uint_as_float(top));
}
// Eight codes, first in the lowest byte.  2^-e is a normal number for every scale byte; only at SCALE_MAX can a quotient pass 448.
__device__ __forceinline__ u32x2 codes_of(const float *v, unsigned byte)
{
    if (byte == SCALE_NAN) return u32x2{0x7f7f7f7fu, 0x7f7f7f7fu};
    const float inv = __uint_as_float((254u - byte) << 23);
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = __builtin_amdgcn_fmed3f(v[i] * inv, -448.0f, 448.0f);
    u32x2 c;
    int t = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
    c.x = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], t, true);
    t = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], 0, false);
    c.y = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], t, true);
    return c;
}
// What four codes stand for, as bf16, two to a word.  A scale byte of 255 makes NaN of NaN codes.
__device__ __forceinline__ u32x2 decode_four(unsigned codes, float scale)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true);
    return u32x2{__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b)};
}
__device__ __forceinline__ float scale_value(unsigned byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ void decode_eight(u32x2 codes, unsigned byte, float *v)
{
    Eight<bf16_t> e;
    const float s = scale_value(byte);
    const u32x2 a = decode_four(codes.x, s), b = decode_four(codes.y, s);
    e.w = u32x4{a.x, a.y, b.x, b.y};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = e[i];
}

// A checkpoint's buffer, seen from its rows.
struct ActRef {
    uint8_t *codes, *scales;
    int64_t groups;             // scales a row; a row of codes takes 32 times as many bytes
    __device__ __forceinline__ uint8_t *code_at(int64_t row, int64_t i) const { return codes + row * groups * GROUP + i; }
    __device__ __forceinline__ uint8_t *scale_at(int64_t row, int64_t i) const { return scales + row * groups + i / GROUP; }
    // Eight values of a group, from element i (a multiple of 8) of a row of n on; the four lanes of a group call it together.  Without LAST they
    // all lie in the row.
    template <bool LAST = true>
    __device__ __forceinline__ void put(int64_t row, int64_t i, int64_t n, const float *v) const
    {
        const unsigned byte = group_scale(v);
        if (LAST && i >= groups * GROUP) return;
        u32x2 c = codes_of(v, byte);
        if (LAST && byte == SCALE_NAN && i + 8 > n) {       // the padding stays 0
            const int left = (int)max((int64_t)0, n - i);
            const unsigned long long keep = left == 0 ? 0 : ~0ull >> (64 - 8 * left);
            c.x &= (unsigned)keep;
            c.y &= (unsigned)(keep >> 32);
        }
        *reinterpret_cast<u32x2 *>(code_at(row, i)) = c;
        if (i % GROUP == 0) *scale_at(row, i) = (uint8_t)byte;
    }
    template <bool LAST = true>
    __device__ __forceinline__ void get(int64_t row, int64_t i, float *v) const
    {
        if (LAST && i >= groups * GROUP) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 0.0f;
            return;
        }
        decode_eight(*reinterpret_cast<const u32x2 *>(code_at(row, i)), *scale_at(row, i), v);
    }
};

}  // namespace ef
