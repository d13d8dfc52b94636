// bf_elem.cuh -- element types of the logits and embedding kernels: every
// value is computed with in 32 bits and rounded once, to nearest, when stored.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace bfk {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

template <typename E>
__device__ __forceinline__ E from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// Sixteen bytes of elements, as 32-bit values and back.
template <typename E>
struct Vec {
  static constexpr uint32_t kWidth = 16 / sizeof(E);
};

__device__ __forceinline__ uint32_t minus_inf_bits(float) { return 0xFF800000u; }
__device__ __forceinline__ uint32_t minus_inf_bits(__nv_bfloat16) { return 0xFF80FF80u; }
__device__ __forceinline__ uint32_t minus_inf_bits(__half) { return 0xFC00FC00u; }

__device__ __forceinline__ void unpack(uint32_t u, float, float* f) { f[0] = __uint_as_float(u); }
__device__ __forceinline__ void unpack(uint32_t u, __nv_bfloat16, float* f) {
  f[0] = __uint_as_float(u << 16);
  f[1] = __uint_as_float(u & 0xFFFF0000u);
}
__device__ __forceinline__ void unpack(uint32_t u, __half, float* f) {
  const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&u));
  f[0] = v.x;
  f[1] = v.y;
}

__device__ __forceinline__ uint32_t pack(const float* f, float) { return __float_as_uint(f[0]); }
__device__ __forceinline__ uint32_t pack(const float* f, __nv_bfloat16) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(f[0], f[1]);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack(const float* f, __half) {
  const __half2 v = __floats2half2_rn(f[0], f[1]);
  return *reinterpret_cast<const uint32_t*>(&v);
}

template <typename E>
__device__ __forceinline__ void unpack(const uint4& u, float* f) {
  constexpr int n = 4 / sizeof(E);
  unpack(u.x, E(), f);
  unpack(u.y, E(), f + n);
  unpack(u.z, E(), f + 2 * n);
  unpack(u.w, E(), f + 3 * n);
}
template <typename E>
__device__ __forceinline__ uint4 pack(const float* f) {
  constexpr int n = 4 / sizeof(E);
  return make_uint4(pack(f, E()), pack(f + n, E()), pack(f + 2 * n, E()), pack(f + 3 * n, E()));
}

// A row of elements as 16-byte vectors: vector v holds elements v * kWidth -
// shift and on, where shift is how far the row starts behind a 16-byte
// boundary.  The first and the last vector may reach outside the row: those are
// read and written element by element.
template <typename E>
struct Window {
  E* row;
  uint32_t shift, width, vectors;
  static constexpr uint32_t kWidth = Vec<E>::kWidth;

  __device__ __forceinline__ Window(E* p, uint32_t n)
      : row(p), shift((uint32_t)((uintptr_t)p % 16) / sizeof(E)), width(n), vectors((shift + n + kWidth - 1) / kWidth) {}

  __device__ __forceinline__ bool whole(uint32_t v) const {
    return v * kWidth >= shift && (v + 1) * kWidth <= shift + width;
  }
  __device__ __forceinline__ uint4* at(uint32_t v) const {
    return reinterpret_cast<uint4*>(row + ((int64_t)v * kWidth - shift));
  }
  // Vector v, with -inf outside the row.
  __device__ __forceinline__ uint4 load(uint32_t v) const {
    if (whole(v)) return __ldcs(at(v));
    const uint32_t none = minus_inf_bits(E());
    uint4 u = make_uint4(none, none, none, none);
    if (v < vectors) {
      float f[kWidth];
#pragma unroll
      for (uint32_t i = 0; i < kWidth; ++i) {
        const uint32_t j = v * kWidth + i;
        f[i] = j >= shift && j < shift + width ? to_f32(row[j - shift]) : -__builtin_huge_valf();
      }
      u = pack<E>(f);
    }
    return u;
  }
  __device__ __forceinline__ void store(uint32_t v, const float* f) const {
    if (whole(v)) {
      __stcs(at(v), pack<E>(f));
    } else if (v < vectors) {
#pragma unroll
      for (uint32_t i = 0; i < kWidth; ++i) {
        const uint32_t j = v * kWidth + i;
        if (j >= shift && j < shift + width) row[j - shift] = from_f32<E>(f[i]);
      }
    }
  }
  // As store, for values cut into vectors at another row's boundaries (`from` behind one).
  __device__ __forceinline__ void store_cut(uint32_t v, uint32_t from, const float* f) const {
#pragma unroll
    for (uint32_t i = 0; i < kWidth; ++i) {
      const uint32_t j = v * kWidth + i;
      if (j >= from && j < from + width) row[j - from] = from_f32<E>(f[i]);
    }
  }
};

}  // namespace bfk
