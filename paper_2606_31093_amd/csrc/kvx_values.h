// kvx_values.h -- the value types of cached rows on the device: 16-bit values
// and OCP e4m3, in vectors of 8, and the matrix instruction on them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kvx {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;

template <typename To, typename From>
__device__ __forceinline__ To bits(const From &x) {
    return __builtin_bit_cast(To, x);
}

template <bool F16>
struct Half;

template <>
struct Half<false> {
    // round to nearest even
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const bf16x2 v = {(__bf16)a, (__bf16)b};
        return bits<uint32_t>(v);
    }
    static __device__ __forceinline__ float lo(uint32_t w) { return bits<float>(w << 16); }
    static __device__ __forceinline__ float hi(uint32_t w) { return bits<float>(w & 0xffff0000u); }
    // two of the four e4m3 values in w, exact
    template <bool UPPER>
    static __device__ __forceinline__ uint32_t from_e4m3(uint32_t w) {
        return bits<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, UPPER));
    }
    // D(16 x 16) = A(16 x 32) B(32 x 16) + C: lane (c = lane % 16, q = lane / 16)
    // holds A(c, 8q..) , B(8q.., c) and D(4q.., c)
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(bits<bf16x8>(a), bits<bf16x8>(b), c, 0, 0, 0);
    }
};

template <>
struct Half<true> {
    static __device__ __forceinline__ uint32_t pack(float a, float b) {
        const f16x2 v = {(_Float16)a, (_Float16)b};
        return bits<uint32_t>(v);
    }
    static __device__ __forceinline__ float lo(uint32_t w) { return (float)bits<f16x2>(w)[0]; }
    static __device__ __forceinline__ float hi(uint32_t w) { return (float)bits<f16x2>(w)[1]; }
    template <bool UPPER>
    static __device__ __forceinline__ uint32_t from_e4m3(uint32_t w) {
        return bits<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, UPPER));
    }
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(bits<f16x8>(a), bits<f16x8>(b), c, 0, 0, 0);
    }
};

// x to e4m3's range; NaN stays NaN.
__device__ __forceinline__ float clamp_e4m3(float x) { return x > 448.0f ? 448.0f : x < -448.0f ? -448.0f : x; }

// Four values in e4m3, rounded to nearest even.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(a), clamp_e4m3(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(c), clamp_e4m3(d), w, true);
}

}  // namespace kvx
