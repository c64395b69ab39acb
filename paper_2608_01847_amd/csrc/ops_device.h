// Small device helpers of the operators around the linears (norms, attention, token log probabilities): element and
// vector access in either type, sums and maxima over a wave.
#pragma once

#include "gemm_common.h"

namespace focus {

// bf16 tensors are uint16_t here, fp32 tensors float
__device__ __forceinline__ float load_one(const uint16_t *p) { return bf16_bits_to_f32(*p); }
__device__ __forceinline__ float load_one(const float *p) { return *p; }
__device__ __forceinline__ void store_one(uint16_t *p, float v) { *p = (uint16_t)f32_to_bf16_bits(v); }
__device__ __forceinline__ void store_one(float *p, float v) { *p = v; }

// Two fp32 values rounded to bf16 (to nearest, ties to even), the first in the low half: one v_cvt_pk_bf16_f32, left to
// the compiler, which knows what may not directly precede it (the instruction after an exponential may not read it)
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    bf16x2_t v;
    v[0] = (__bf16)lo;
    v[1] = (__bf16)hi;
    return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ void zero8(float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = 0.0f;
}

__device__ __forceinline__ void unpack_bf16(uint32_t w, float &lo, float &hi) {
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xFFFF0000u);
}

// 8 elements at any element-aligned address, of which the first n exist (the others are read as zeros and not written).
// Rows of a tensor whose length is no multiple of 8 start at odd addresses: the hardware takes 16-byte accesses there
// too, so that only the last piece of such a row goes element by element.
typedef unsigned int u32x4_any_t __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any_t __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ void load8_n(const uint16_t *p, int n, float (&v)[8]) {
    if (n >= 8) {
        const u32x4_any_t w = *reinterpret_cast<const u32x4_any_t *>(p);
#pragma unroll
        for (int e = 0; e < 4; e++) unpack_bf16(w[e], v[2 * e], v[2 * e + 1]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = e < n ? load_one(p + e) : 0.0f;
    }
}

__device__ __forceinline__ void load8_n(const float *p, int n, float (&v)[8]) {
    if (n >= 8) {
        const f32x4_any_t a = reinterpret_cast<const f32x4_any_t *>(p)[0], b = reinterpret_cast<const f32x4_any_t *>(p)[1];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            v[e] = a[e];
            v[4 + e] = b[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = e < n ? p[e] : 0.0f;
    }
}

template <bool TAIL = true>
__device__ __forceinline__ void store8_n(uint16_t *p, int n, const float (&v)[8]) {
    if (!TAIL || n >= 8) {
        u32x4_any_t w;
#pragma unroll
        for (int e = 0; e < 4; e++) w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
        *reinterpret_cast<u32x4_any_t *>(p) = w;
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (e < n) store_one(p + e, v[e]);
    }
}

template <bool TAIL = true>
__device__ __forceinline__ void store8_n(float *p, int n, const float (&v)[8]) {
    if (!TAIL || n >= 8) {
        reinterpret_cast<f32x4_any_t *>(p)[0] = f32x4_any_t{v[0], v[1], v[2], v[3]};
        reinterpret_cast<f32x4_any_t *>(p)[1] = f32x4_any_t{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (e < n) p[e] = v[e];
    }
}

// Eight consecutive elements as they lie in memory (bf16: four registers), the missing ones zeros
template <typename T>
struct Raw8;
template <>
struct Raw8<uint16_t> {
    u32x4_any_t w;
    __device__ __forceinline__ void load(const uint16_t *p, int n) {
        if (n >= 8) {
            w = *reinterpret_cast<const u32x4_any_t *>(p);
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++) w[e] = (2 * e < n ? p[2 * e] : 0u) | (uint32_t)(2 * e + 1 < n ? p[2 * e + 1] : 0u) << 16;
        }
    }
    __device__ __forceinline__ float operator[](int e) const {
        return __uint_as_float((e & 1) ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
    }
    // the eight from element c on of a row of n (a multiple of 8) behind rs, zeros past its end: no branch
    __device__ __forceinline__ void load_row(__amdgpu_buffer_rsrc_t rs, int c) {
        w = __builtin_amdgcn_raw_buffer_load_b128(rs, c * 2, 0, 0);
    }
    // keeps the compiler from holding the unpacked values over this point in place of the packed ones
    __device__ __forceinline__ void keep_packed() { asm volatile("" : "+v"(w)); }
};
template <>
struct Raw8<float> {
    f32x4_any_t w[2];
    __device__ __forceinline__ void load(const float *p, int n) {
        if (n >= 8) {
            w[0] = reinterpret_cast<const f32x4_any_t *>(p)[0];
            w[1] = reinterpret_cast<const f32x4_any_t *>(p)[1];
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++) w[e >> 2][e & 3] = e < n ? p[e] : 0.0f;
        }
    }
    __device__ __forceinline__ void load_row(__amdgpu_buffer_rsrc_t rs, int c) {
        w[0] = __builtin_bit_cast(f32x4_any_t, __builtin_amdgcn_raw_buffer_load_b128(rs, c * 4, 0, 0));
        w[1] = __builtin_bit_cast(f32x4_any_t, __builtin_amdgcn_raw_buffer_load_b128(rs, c * 4 + 16, 0, 0));
    }
    __device__ __forceinline__ float operator[](int e) const { return w[e >> 2][e & 3]; }
    __device__ __forceinline__ void keep_packed() {}
};

// 8 consecutive parameters from element c on, of either type
__device__ __forceinline__ void load8_param(const void *base, int dtype, int c, int n, float (&v)[8]) {
    if (dtype == kBF16) load8_n(static_cast<const uint16_t *>(base) + c, n, v);
    else load8_n(static_cast<const float *>(base) + c, n, v);
}
__device__ __forceinline__ float load_param(const void *base, int dtype, int c) {
    return dtype == kBF16 ? load_one(static_cast<const uint16_t *>(base) + c) : static_cast<const float *>(base)[c];
}

// a <- a + b, rounded to the type T and back
template <typename T>
__device__ __forceinline__ void add_rounded(float (&a)[8], const float (&b)[8]) {
#pragma unroll
    for (int e = 0; e < 8; e++) {
        a[e] += b[e];
        if constexpr (sizeof(T) == 2) a[e] = bf16_bits_to_f32(f32_to_bf16_bits(a[e]));
    }
}

// 2^x by the hardware instruction: results below 2^-126 are zeros
__device__ __forceinline__ float exp2_raw(float x) { return __builtin_amdgcn_exp2f(x); }

// Sum and maximum over the 64 lanes, in every lane. The order is the same in each lane's result.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v = fmaxf(v, __shfl_xor(v, m, 64));
    return v;
}

}  // namespace focus
