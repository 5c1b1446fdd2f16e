// Shared by the operators on vectors (qadc_vec.h): element types, loads and stores of eight elements at any
// alignment, sums over groups of lanes, scales of 8-bit blocks; and the host's checks of arguments.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qadc_internal.h"
#include "qadc_vec.h"

typedef float vec_f4 __attribute__((ext_vector_type(4)));
typedef float vec_f8 __attribute__((ext_vector_type(8)));
typedef int vec_i4 __attribute__((ext_vector_type(4)));

// E elements (eight, unless said otherwise) as they lie in memory.  Global loads and stores work at any byte address here; the
// types only promise the alignment of one element.
template <class T, int E = 8>
struct VecPack {
    typedef T type __attribute__((ext_vector_type(E), aligned(sizeof(T))));
    typedef float wide __attribute__((ext_vector_type(E)));
};
template <class T, int E = 8>
using vec_pack = typename VecPack<T, E>::type;
template <int E>
using vec_f = typename VecPack<float, E>::wide;

// The vector's elements from the N-th on, zeros behind.
template <int N, int E, class V>
__device__ __forceinline__ V vec_down(V v) {
    V r = v;
#pragma unroll
    for (int i = 0; i < E; ++i) r[i] = i + N < E ? v[i + N] : 0;
    return r;
}

// left: elements of the row from p on (those beyond it read as zero and are not touched); before: elements of the row before p.  At the
// end of a row the last E elements are read and moved into place: one load, where one for each element of odd widths cost half the time of
// a row of 257.
template <class T, int E = 8>
__device__ __forceinline__ vec_pack<T, E> vec_load(const T *p, int64_t left, int64_t before) {
    typedef vec_pack<T, E> pack;
    if (left >= E) return *(const pack *)p;
    pack v = (pack)(T)0.0f;
    if (left <= 0) return v;
    if (before + left >= E) {
        const int k = E - (int)left;
        v = *(const pack *)(p - k);
        if constexpr (E > 4)
            if (k & 4) v = vec_down<4, E>(v);
        if constexpr (E > 2)
            if (k & 2) v = vec_down<2, E>(v);
        if (k & 1) v = vec_down<1, E>(v);
        return v;
    }
#pragma unroll
    for (int i = 0; i < E - 1; ++i)
        if (i < left) v[i] = p[i];
    return v;
}
template <class T, int E = 8>
__device__ __forceinline__ vec_f<E> vec_wide(vec_pack<T, E> v) {
    return __builtin_convertvector(v, vec_f<E>);
}
// (the end of a row: four, two and one of its elements)
template <class T, int E = 8>
__device__ __forceinline__ void vec_store(T *p, int64_t left, vec_f<E> f) {
    typedef vec_pack<T, E> pack;
    pack v = __builtin_convertvector(f, pack);
    if (left >= E) {
        *(pack *)p = v;
        return;
    }
    if (left <= 0) return;
    if constexpr (E > 4)
        if (left & 4) {
            vec_pack<T, 4> w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = v[i];
            *(vec_pack<T, 4> *)p = w;
            p += 4;
            v = vec_down<4, E>(v);
        }
    if constexpr (E > 2)
        if (left & 2) {
            vec_pack<T, 2> w;
            w[0] = v[0], w[1] = v[1];
            *(vec_pack<T, 2> *)p = w;
            p += 2;
            v = vec_down<2, E>(v);
        }
    if (left & 1) *p = v[0];
}
// eight bytes, sixteen bytes
__device__ __forceinline__ void vec_store_bytes(uint8_t *p, int64_t left, uint64_t v) {
    typedef uint64_t any64 __attribute__((aligned(1)));
    typedef uint32_t any32 __attribute__((aligned(1)));
    typedef uint16_t any16 __attribute__((aligned(1)));
    if (left >= 8) {
        *(any64 *)p = v;
        return;
    }
    if (left <= 0) return;
    if (left & 4) *(any32 *)p = (uint32_t)v, p += 4, v >>= 32;
    if (left & 2) *(any16 *)p = (uint16_t)v, p += 2, v >>= 16;
    if (left & 1) *p = (uint8_t)v;
}
__device__ __forceinline__ void vec_store_bytes(uint8_t *p, int64_t left, vec_i4 v) {
    typedef int any128 __attribute__((ext_vector_type(4), aligned(1)));
    if (left >= 16) {
        *(any128 *)p = v;
        return;
    }
    vec_store_bytes(p, left, (uint64_t)(uint32_t)v[1] << 32 | (uint32_t)v[0]);
    vec_store_bytes(p + 8, left - 8, (uint64_t)(uint32_t)v[3] << 32 | (uint32_t)v[2]);
}

// Sum, or largest, over the LANES (16, 32 or 64) neighbouring lanes of a row; every one of them has the result.  Sixteen lanes by
// rotations in the vector unit (both partners of a step add the same two values, so all agree); their sums meet in scalar registers.
template <int N>
__device__ __forceinline__ float vec_rotate(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + N, 0xf, 0xf, true));
}
template <int LANES>
__device__ __forceinline__ float vec_sum(float v) {
    v += vec_rotate<8>(v);
    v += vec_rotate<4>(v);
    v += vec_rotate<2>(v);
    v += vec_rotate<1>(v);
    if constexpr (LANES > 16) {
        const int u = __float_as_int(v);
        const float a = __int_as_float(__builtin_amdgcn_readlane(u, 0)) + __int_as_float(__builtin_amdgcn_readlane(u, 16));
        const float b = __int_as_float(__builtin_amdgcn_readlane(u, 32)) + __int_as_float(__builtin_amdgcn_readlane(u, 48));
        v = LANES == 64 ? a + b : ((threadIdx.x & 63) < 32 ? a : b);
    }
    return v;
}
__device__ __forceinline__ float vec_max16(float v) {
    v = fmaxf(v, vec_rotate<8>(v));
    v = fmaxf(v, vec_rotate<4>(v));
    v = fmaxf(v, vec_rotate<2>(v));
    return fmaxf(v, vec_rotate<1>(v));
}

// The largest finite magnitude of eight values.
__device__ __forceinline__ float vec_top(vec_f8 f) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = fabsf(f[i]);
        m = fmaxf(m, a < INFINITY ? a : 0.0f);
    }
    return m;
}

// A block's scale from its largest finite magnitude.  448 = 1.75 * 2^8 and 57344 = 1.75 * 2^15, so that the smallest power of
// two that brings a = f * 2^e within range is 2^(e - 8) or 2^(e - 15), one more where f exceeds 1.75.
struct VecScale {
    float scale;     // F32
    uint32_t e8m0;   // E8M0: the byte
    float inverse;   // one over the scale
    bool divide;     // F32: quotients of such scales take a division
};
__device__ __forceinline__ VecScale vec_scale(float top, bool e5m2, bool pow2) {
    VecScale s;
    const uint32_t u = __float_as_uint(top);
    int e = (int)(u >> 23) - (e5m2 ? 15 : 8) + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = top == 0.0f ? 127 : (e < 0 ? 0 : e);
    s.e8m0 = (uint32_t)e;
    s.inverse = __uint_as_float((uint32_t)(254 - e) << 23);
    s.scale = 1.0f;
    s.divide = false;
    if (!pow2) {
        s.scale = top == 0.0f ? 1.0f : fmaxf(top / (e5m2 ? 57344.0f : 448.0f), 1.17549435e-38f);
        s.inverse = 1.0f / s.scale;
        s.divide = s.scale < 2.58493941e-26f || (__float_as_uint(s.scale) & 0x7fffffu) == 0x7fffffu;
    }
    return s;
}
// f over the scale as a division rounds it, in three operations: with r = 1 / scale rounded to nearest, q = f r is within one step of the
// quotient, f - q scale is exact, and q + r (f - q scale) rounds to the quotient's nearest (Markstein, 1990) unless scale's bits are
// all ones or the remainder falls below the smallest numbers; those take the division.  The remainder is a multiple of q's last bit times scale's.
// Quotients matter from 2^-18 on (E5M2's smallest border between two values is 2^-17), where q's last bit is 2^-41 or more: with scales from 2^-85
// on the product is 2^-149, the smallest number, or more.  (Searched next to such borders, scales of 2^-88 and less gave other bytes.)
__device__ __forceinline__ float vec_quotient(float f, const VecScale &s) {
    const float q = f * s.inverse;
    return __fmaf_rn(__fmaf_rn(-q, s.scale, f), s.inverse, q);
}
// Eight values over the scale, to 8 bits each (an infinity is made NaN where the type has none).
__device__ __forceinline__ uint64_t vec_to8(vec_f8 f, const VecScale &s, bool e5m2, bool pow2) {
    float v[8];
    if (pow2) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = f[i] * s.inverse;
    } else if (__builtin_expect(s.divide, 0)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = f[i] / s.scale;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fabsf(f[i]) < INFINITY ? vec_quotient(f[i], s) : f[i];
    }
    int lo = 0, hi = 0;
    if (e5m2) {
        lo = __builtin_amdgcn_cvt_pk_bf8_f32(v[0], v[1], lo, false);
        lo = __builtin_amdgcn_cvt_pk_bf8_f32(v[2], v[3], lo, true);
        hi = __builtin_amdgcn_cvt_pk_bf8_f32(v[4], v[5], hi, false);
        hi = __builtin_amdgcn_cvt_pk_bf8_f32(v[6], v[7], hi, true);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fabsf(v[i]) < INFINITY ? v[i] : NAN;
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], lo, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], hi, false);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], hi, true);
    }
    return (uint64_t)(uint32_t)hi << 32 | (uint32_t)lo;
}
__device__ __forceinline__ void vec_put_scale(void *scales, int64_t at, const VecScale &s, bool pow2) {
    if (pow2) ((uint8_t *)scales)[at] = (uint8_t)s.e8m0;
    else ((float *)scales)[at] = s.scale;
}

// The block's number in a launch of vec_grid's; the last ones may be beyond what was asked for.
__device__ __forceinline__ int64_t vec_block() { return blockIdx.y == 0 ? (int64_t)blockIdx.x : (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// ---------------------------------------------------------------------- host
#define VEC_MAX_BLOCKS 0x7fffffffLL
// A grid of at least `blocks` blocks (1 to VEC_MAX_BLOCKS).  One dimension's blocks times threads stay below 2^32, so that more take a second.
static inline dim3 vec_grid(int64_t blocks, int threads) {
    const int64_t most = 0xffffffffLL / threads, y = (blocks + most - 1) / most;
    return dim3((unsigned)((blocks + y - 1) / y), (unsigned)y);
}
static inline bool vec_is_wide(int t) { return t == VEC_F32 || t == VEC_BF16 || t == VEC_F16; }
static inline bool vec_is_8bit(int t) { return t == VEC_E4M3 || t == VEC_E5M2; }
static inline bool vec_is_scale(int t) { return t == VEC_E8M0 || t == VEC_F32; }
static inline size_t vec_bytes(int t) { return t == VEC_F32 ? 4 : (t == VEC_BF16 || t == VEC_F16 ? 2 : 1); }
static inline size_t vec_up256(size_t x) { return (x + 255) & ~(size_t)255; }
static inline bool vec_aligned(const void *p, int t) { return ((uintptr_t)p & (vec_bytes(t) - 1)) == 0; }

#define VEC_REQUIRE(cond, ...)           \
    do {                                 \
        if (!(cond)) {                   \
            qadc_set_error(__VA_ARGS__); \
            return PQ_EINVAL;            \
        }                                \
    } while (0)

// Calls BODY with T the C++ type of the element type t.
#define VEC_TYPED(t, T, ...)             \
    do {                                 \
        if ((t) == VEC_F32) {            \
            using T = float;             \
            __VA_ARGS__;                 \
        } else if ((t) == VEC_BF16) {    \
            using T = __bf16;            \
            __VA_ARGS__;                 \
        } else {                         \
            using T = _Float16;          \
            __VA_ARGS__;                 \
        }                                \
    } while (0)
