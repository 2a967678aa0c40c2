// Pieces of 16 bytes of a row of floating-point numbers, at any alignment of their type, and single numbers.
#pragma once

#include "slim_device.h"

namespace slimnorm {
namespace {

using namespace slimdev;

template <typename T>
struct Elem;
template <>
struct Elem<__half> {
  static __device__ __forceinline__ float widen(unsigned short v) { return (float)__builtin_bit_cast(_Float16, v); }
  static __device__ __forceinline__ unsigned short narrow(float v) { return __builtin_bit_cast(unsigned short, (_Float16)v); }
};
template <>
struct Elem<__hip_bfloat16> {
  static __device__ __forceinline__ float widen(unsigned short v) { return __uint_as_float((unsigned)v << 16); }
  static __device__ __forceinline__ unsigned short narrow(float v) { return __builtin_bit_cast(unsigned short, (__bf16)v); }
};

// A piece: 16 bytes of a row (4 or 8 elements)
template <typename T>
struct Piece {
  static constexpr int E = 16 / sizeof(T);
  unsigned v[4];
  // from p on, of which `left` elements exist (the others are zero); p is aligned to its type only
  __device__ __forceinline__ void load(const T* p, int left) {
    if (left >= E) {
      __builtin_memcpy(v, p, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = 0u;
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i < left) v[i] = reinterpret_cast<const unsigned*>(p)[i];
      } else {
        const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < left) v[i / 2] |= (unsigned)q[i] << (16 * (i & 1));
      }
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[i]);
    else return Elem<T>::widen((unsigned short)(v[i / 2] >> (16 * (i & 1))));
  }
  __device__ __forceinline__ void set(const float (&f)[E]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) v[i] = __float_as_uint(f[i]);
      else v[i] = (unsigned)Elem<T>::narrow(f[2 * i]) | (unsigned)Elem<T>::narrow(f[2 * i + 1]) << 16;
    }
  }
  __device__ __forceinline__ void store(T* p, int left) const {
    if (left >= E) {
      store16_once(p, v);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < left) reinterpret_cast<unsigned*>(p)[i] = v[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) reinterpret_cast<unsigned short*>(p)[i] = (unsigned short)(v[i / 2] >> (16 * (i & 1)));
    }
  }
};

template <typename T>
__device__ __forceinline__ float value(const void* p, int64_t i) {
  if constexpr (sizeof(T) == 4) return static_cast<const float*>(p)[i];
  else return Elem<T>::widen(static_cast<const unsigned short*>(p)[i]);
}
template <typename T>
__device__ __forceinline__ void put(void* p, int64_t i, float v) {
  if constexpr (sizeof(T) == 4) static_cast<float*>(p)[i] = v;
  else static_cast<unsigned short*>(p)[i] = Elem<T>::narrow(v);
}

// E values one after another, of which `left` are wanted (as single stores, a lane's E apart, 16384 columns took 15 us)
template <typename T, int E>
__device__ __forceinline__ void put_run(void* p, int c, int left, const float (&f)[E]) {
  if (left >= E) {
    if constexpr (sizeof(T) == 4) {
      __builtin_memcpy(static_cast<float*>(p) + c, f, sizeof(f));
    } else {
      unsigned short h[E];
#pragma unroll
      for (int e = 0; e < E; ++e) h[e] = Elem<T>::narrow(f[e]);
      __builtin_memcpy(static_cast<unsigned short*>(p) + c, h, sizeof(h));
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e < left) put<T>(p, c + e, f[e]);
  }
}

}  // namespace
}  // namespace slimnorm
