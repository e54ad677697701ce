// Element types of the learner's operators (k_scan.hip, k_tokens.hip): storage, conversion to
// and from 32-bit arithmetic, and vectors of V elements moved as one word.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace av {

struct bf16_t { uint16_t bits; };

__device__ inline float to_f32(float v) { return v; }
__device__ inline float to_f32(_Float16 v) { return float(v); }
__device__ inline float to_f32(bf16_t v) { return __uint_as_float(uint32_t(v.bits) << 16); }

// Round to nearest, ties to even; bf16 through the hardware's conversion, which keeps NaN a NaN.
template <typename T> __device__ inline T from_f32(float v);
template <> __device__ inline float from_f32<float>(float v) { return v; }
template <> __device__ inline _Float16 from_f32<_Float16>(float v) { return _Float16(v); }
template <> __device__ inline bf16_t from_f32<bf16_t>(float v) {
    const __bf16 b = static_cast<__bf16>(v);
    bf16_t r;
    __builtin_memcpy(&r, &b, 2);
    return r;
}

template <typename T, int V> struct alignas(sizeof(T) * V) Vec { T v[V]; };

}  // namespace av
