// Element types of the learner's operators (k_scan.hip, k_tokens.hip): storage, conversion to
// and from 32-bit arithmetic, and groups of V elements moved as one word.
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

// V neighbouring elements.  Global memory takes an access of up to 16 bytes at any address, so one
// of V elements needs no more alignment than its element's.  The words stand for elements of any type, and
// for smaller words at the same place (a row's last, an output over its input): may_alias says so.
template <typename T, int V> struct Word { T v[V]; };
typedef uint64_t Any2 __attribute__((ext_vector_type(2)));
typedef uint64_t Any4 __attribute__((ext_vector_type(4)));
template <int kBytes> struct Bits;
template <> struct Bits<1> { typedef uint8_t type; };
template <> struct Bits<2> { typedef uint16_t type __attribute__((aligned(1), may_alias)); };
template <> struct Bits<4> { typedef uint32_t type __attribute__((aligned(1), may_alias)); };
template <> struct Bits<8> { typedef uint64_t type __attribute__((aligned(1), may_alias)); };
template <> struct Bits<16> { typedef Any2 type __attribute__((aligned(1), may_alias)); };
template <> struct Bits<32> { typedef Any4 type __attribute__((aligned(1), may_alias)); };    // two accesses

template <typename E> __device__ inline E load_any(const void *p) {
    const typename Bits<sizeof(E)>::type u =
        *static_cast<const typename Bits<sizeof(E)>::type *>(p);
    E e;
    __builtin_memcpy(&e, &u, sizeof e);
    return e;
}
// Written past the caches.
template <typename E> __device__ inline void store_past(void *p, const E &e) {
    typedef typename Bits<sizeof(E)>::type U;
    U u;
    __builtin_memcpy(&u, &e, sizeof u);
    __builtin_nontemporal_store(u, static_cast<U *>(p));
}

}  // namespace av
