// Shared device/host helpers for the gfx950 Temp-Lora kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

typedef uint16_t bf16_t;  // raw bf16 bit pattern in memory

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

#define TL_WAVE 64

__device__ __forceinline__ float bf16_to_f32(bf16_t x) { return __uint_as_float(((uint32_t)x) << 16); }

// round-to-nearest-even, NaN stays NaN: the hardware conversion of gfx950 (v_cvt_pk_bf16_f32), one instruction for two
// values instead of the six integer operations per value of a hand-written rounding
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ bf16_t f32_to_bf16(float f) { return __builtin_bit_cast(bf16_t, (__bf16)f); }

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    bf16x2_t v;
    v[0] = (__bf16)lo;
    v[1] = (__bf16)hi;
    return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
    return x;
}

// block-wide sum for blockDim.x a multiple of 64, up to 1024; `red` is >= 16 floats of LDS
__device__ __forceinline__ float block_sum(float x, float* red) {
    x = wave_sum(x);
    const int w = threadIdx.x >> 6, nw = blockDim.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[w] = x;
    __syncthreads();
    float t = 0.f;
    for (int i = 0; i < nw; ++i) t += red[i];
    return t;
}
__device__ __forceinline__ float block_max(float x, float* red) {
    x = wave_max(x);
    const int w = threadIdx.x >> 6, nw = blockDim.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[w] = x;
    __syncthreads();
    float t = red[0];
    for (int i = 1; i < nw; ++i) t = fmaxf(t, red[i]);
    return t;
}

// 16 bytes from an address that is a multiple of 2
struct __attribute__((packed, aligned(2))) any16_t { uint32_t w[4]; };
__device__ __forceinline__ bf16x8_t load_any16(const bf16_t* p) {
    const any16_t a = *(const any16_t*)p;
    return __builtin_bit_cast(bf16x8_t, make_uint4(a.w[0], a.w[1], a.w[2], a.w[3]));
}

// eight bf16 in a 16-byte word <-> eight floats
__device__ __forceinline__ void unpack8(uint4 r, float* f) {
    f[0] = bf16_to_f32(r.x & 0xffff); f[1] = bf16_to_f32(r.x >> 16);
    f[2] = bf16_to_f32(r.y & 0xffff); f[3] = bf16_to_f32(r.y >> 16);
    f[4] = bf16_to_f32(r.z & 0xffff); f[5] = bf16_to_f32(r.z >> 16);
    f[6] = bf16_to_f32(r.w & 0xffff); f[7] = bf16_to_f32(r.w >> 16);
}
__device__ __forceinline__ uint4 pack8(const float* f) {
    uint4 r;
    r.x = pack_bf16x2(f[0], f[1]); r.y = pack_bf16x2(f[2], f[3]);
    r.z = pack_bf16x2(f[4], f[5]); r.w = pack_bf16x2(f[6], f[7]);
    return r;
}

static inline int cdiv(long a, long b) { return (int)((a + b - 1) / b); }
