// Sixteen-byte vectors of the storage types, at any element's address.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ebag {

typedef uint32_t vec16 __attribute__((ext_vector_type(4)));

// Global memory takes 16-byte accesses at any address, so rows need no alignment
// beyond their elements' (a vector across two cache lines costs a second one).
typedef vec16 vec16_any __attribute__((aligned(2)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ vec16 load16(const char* p) { return *reinterpret_cast<const vec16_any*>(p); }
__device__ __forceinline__ void store16(char* p, const vec16& v) { *reinterpret_cast<vec16_any*>(p) = v; }

// A storage type (EBAG_F32, EBAG_F16, EBAG_BF16): elements to and from fp32,
// rounded to nearest even.
template <int DT> struct Type;

// Its elements' bits.
template <int DT> struct Bits { typedef uint16_t type; };
template <> struct Bits<0> { typedef uint32_t type; };

template <> struct Type<0> {
  typedef float elt;
  static constexpr int N = 4;  // elements of a vector
  static __device__ __forceinline__ float widen(elt v) { return v; }
  static __device__ __forceinline__ elt narrow(float f) { return f; }
  static __device__ __forceinline__ void widen(const vec16& r, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(r[i]);
  }
  static __device__ __forceinline__ vec16 narrow(const float* f) {
    vec16 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(f[i]);
    return r;
  }
};

template <> struct Type<1> {
  typedef _Float16 elt;
  static constexpr int N = 8;
  static __device__ __forceinline__ float widen(elt v) { return (float)v; }
  static __device__ __forceinline__ elt narrow(float f) { return (_Float16)f; }
  static __device__ __forceinline__ void widen(const vec16& r, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r[i] & 0xffffu));
      f[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(r[i] >> 16));
    }
  }
  static __device__ __forceinline__ vec16 narrow(const float* f) {
    vec16 r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      r[i] = (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)f[2 * i]) |
             (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)f[2 * i + 1]) << 16;
    return r;
  }
};

template <> struct Type<2> {
  typedef __bf16 elt;
  static constexpr int N = 8;
  static __device__ __forceinline__ float widen(elt v) {
    return __uint_as_float((uint32_t)__builtin_bit_cast(uint16_t, v) << 16);
  }
  static __device__ __forceinline__ elt narrow(float f) { return (__bf16)f; }
  static __device__ __forceinline__ void widen(const vec16& r, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(r[i] << 16);
      f[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ vec16 narrow(const float* f) {
    vec16 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float2v v = {f[2 * i], f[2 * i + 1]};
      r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
    }
    return r;
  }
};

}  // namespace ebag
