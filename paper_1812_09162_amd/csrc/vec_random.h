// Random numbers by position: the generator Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// 2011), whose ten rounds turn a 128-bit counter into four 32-bit words under a 64-bit key.  Counter (j / 8, i, step, layer) gives the
// sixteen-bit numbers of columns 8 (j / 8) .. + 7 of row i, low halves first: whoever holds eight neighbouring elements, as all kernels on
// vectors do, makes its part of the mask by one call, in the forward and again in the backward pass.  A call is 20 products of 32 bits, which run at a quarter of
// the rate, and about 60 other instructions: for 16,384 x 4096 elements 17 us of a kernel that the vector units bound, less where memory does.
#pragma once
#include "vec_device.h"

// Which elements are kept: those whose number is at least `threshold`; 0 (no dropout): all, and nothing is read.
struct VecMask {
    const uint64_t *state;  // seed, step
    uint32_t layer, threshold;
};
struct VecKey {
    uint32_t k0, k1, step;
};
__device__ __forceinline__ VecKey vec_key(const VecMask &m) {
    const uint64_t seed = m.state[0];
    return {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)m.state[1]};
}
// The eight numbers of columns 8 col8 .. + 7 of a row.
__device__ __forceinline__ vec_i4 vec_random(VecKey k, uint32_t layer, uint32_t row, uint32_t col8) {
    uint32_t c0 = col8, c1 = row, c2 = k.step, c3 = layer;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k.k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k.k1;
        c3 = (uint32_t)a;
        k.k0 += 0x9E3779B9u;
        k.k1 += 0xBB67AE85u;
    }
    return (vec_i4){(int)c0, (int)c1, (int)c2, (int)c3};
}
// Of a kept element's sixteen bits all are set, of a dropped one's none.
__device__ __forceinline__ vec_i4 vec_kept(vec_i4 numbers, uint32_t threshold) {
    vec_i4 m;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t u = (uint32_t)numbers[w];
        m[w] = (int)(((u & 0xffffu) >= threshold ? 0xffffu : 0u) | ((u >> 16) >= threshold ? 0xffff0000u : 0u));
    }
    return m;
}
// Zeros in place of the dropped elements, whatever these are.
template <class T>
__device__ __forceinline__ vec_pack<T> vec_drop(vec_pack<T> v, vec_i4 kept) {
    if constexpr (sizeof(T) == 2) {
        const vec_i4 u = __builtin_bit_cast(vec_i4, v) & kept;
        return __builtin_bit_cast(vec_pack<T>, u);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(kept[i >> 1] >> (16 * (i & 1)) & 1)) v[i] = 0;
        return v;
    }
}

// ---------------------------------------------------------------------- host
// The rate as sixteen bits and one over the share that is kept; false: not a rate.
static inline bool vec_rate(double p, uint32_t *threshold, float *factor) {
    if (!(p >= 0.0 && p * 65536.0 < 65535.5)) return false;
    *threshold = (uint32_t)__builtin_rint(p * 65536.0);
    *factor = (float)(65536.0 / (65536.0 - *threshold));
    return *threshold < 65536;
}
