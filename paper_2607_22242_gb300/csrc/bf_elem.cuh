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

__device__ __forceinline__ float2 unpack2(uint32_t u, __nv_bfloat16) {
  return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
}
__device__ __forceinline__ float2 unpack2(uint32_t u, __half) {
  return __half22float2(*reinterpret_cast<const __half2*>(&u));
}
__device__ __forceinline__ uint32_t pack2(float2 f, __nv_bfloat16) {
  const __nv_bfloat162 v = __float22bfloat162_rn(f);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack2(float2 f, __half) {
  const __half2 v = __float22half2_rn(f);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// A vector's elements in pairs.
template <typename E>
__device__ __forceinline__ void unpack(const uint4& u, float2* f) {
  if constexpr (sizeof(E) == 4) {
    f[0] = make_float2(__uint_as_float(u.x), __uint_as_float(u.y));
    f[1] = make_float2(__uint_as_float(u.z), __uint_as_float(u.w));
  } else {
    f[0] = unpack2(u.x, E());
    f[1] = unpack2(u.y, E());
    f[2] = unpack2(u.z, E());
    f[3] = unpack2(u.w, E());
  }
}
template <typename E>
__device__ __forceinline__ uint4 pack(const float2* f) {
  if constexpr (sizeof(E) == 4)
    return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
  else
    return make_uint4(pack2(f[0], E()), pack2(f[1], E()), pack2(f[2], E()), pack2(f[3], E()));
}

// The largest element of N vectors that is a number (-inf if none is).
__device__ __forceinline__ float max_words(const uint32_t* u, int n, float) {
  float m = -__builtin_huge_valf();
#pragma unroll
  for (int i = 0; i < n; ++i) m = fmaxf(m, __uint_as_float(u[i]));
  return m;
}
template <typename E2>
__device__ __forceinline__ E2 max_pairs(const uint32_t* u, int n, uint32_t least) {
  E2 m = *reinterpret_cast<const E2*>(&least);
#pragma unroll
  for (int i = 0; i < n; ++i) m = __hmax2(m, *reinterpret_cast<const E2*>(&u[i]));
  return m;
}
__device__ __forceinline__ float max_words(const uint32_t* u, int n, __nv_bfloat16) {
  const float2 m = __bfloat1622float2(max_pairs<__nv_bfloat162>(u, n, 0xFF80FF80u));
  return fmaxf(m.x, m.y);
}
__device__ __forceinline__ float max_words(const uint32_t* u, int n, __half) {
  const float2 m = __half22float2(max_pairs<__half2>(u, n, 0xFC00FC00u));
  return fmaxf(m.x, m.y);
}
template <typename E, int N>
__device__ __forceinline__ float max_of(const uint4* u) {
  return max_words(reinterpret_cast<const uint32_t*>(u), 4 * N, E());
}

// The elements of one vector that lie inside [lo, hi), `none` elsewhere: for the
// ends of a row, which are read and written element by element.  Kept out of
// line: a row has two such vectors, and their code would be in every unrolled
// load and store (the kernels stalled for instructions a fifth of the time).
template <typename E>
__device__ __noinline__ uint4 load_ends(const E* p, int32_t lo, int32_t hi, uint32_t none) {
  constexpr int n = Vec<E>::kWidth;
  uint32_t b[n];
#pragma unroll
  for (int i = 0; i < n; ++i) {
    b[i] = none;
    if (i >= lo && i < hi) {
      if constexpr (sizeof(E) == 4) b[i] = reinterpret_cast<const uint32_t*>(p)[i];
      else b[i] = reinterpret_cast<const uint16_t*>(p)[i];
    }
  }
  if constexpr (sizeof(E) == 4) return make_uint4(b[0], b[1], b[2], b[3]);
  else
    return make_uint4(__byte_perm(b[0], b[1], 0x5410), __byte_perm(b[2], b[3], 0x5410), __byte_perm(b[4], b[5], 0x5410),
                      __byte_perm(b[6], b[7], 0x5410));
}
template <typename E>
__device__ __noinline__ void store_ends(E* p, uint4 u, int32_t lo, int32_t hi) {
  constexpr int n = Vec<E>::kWidth;
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < n; ++i)
    if (i >= lo && i < hi) {
      if constexpr (sizeof(E) == 4) reinterpret_cast<uint32_t*>(p)[i] = w[i];
      else reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)(w[i / 2] >> (i % 2 * 16));
    }
}

// A matrix's bytes.
struct Extent {
  uintptr_t begin, end;
  template <typename E>
  __device__ __forceinline__ Extent(const E* p, uint64_t rows, uint64_t ld, uint32_t width)
      : begin((uintptr_t)p), end((uintptr_t)(p + (rows - 1) * ld + width)) {}
};

// Sixteen bytes of a row from any element j on: the one or two aligned vectors
// that hold them, to be shifted by take().  Outside the row they are the
// neighbouring rows' and not used; at the matrix's own ends the row's elements are
// read one by one.
template <typename E>
struct Unaligned {
  uint4 lo, hi;
  uint32_t off;  // bytes of lo ahead of them

  __device__ __forceinline__ void load(const E* row, uint32_t width, int64_t j, const Extent& m) {
    const uintptr_t at = (uintptr_t)row + (uintptr_t)(j * (int64_t)sizeof(E)), base = at & ~(uintptr_t)15;
    off = (uint32_t)(at & 15);
    if (base >= m.begin && base + (off ? 32 : 16) <= m.end) {
      lo = *reinterpret_cast<const uint4*>(base);
      if (off) hi = *reinterpret_cast<const uint4*>(base + 16);
    } else {
      off = 0;
      lo = load_ends<E>(reinterpret_cast<const E*>(at), j < 0 ? (int32_t)-j : 0,
                        (int32_t)min((int64_t)Vec<E>::kWidth, (int64_t)width - j), 0);
    }
  }
  __device__ __forceinline__ uint4 take() const {
    if (off == 0) return lo;
    const bool two = off & 8, one = off & 4;
    const uint32_t a0 = two ? lo.z : lo.x, a1 = two ? lo.w : lo.y, a2 = two ? hi.x : lo.z, a3 = two ? hi.y : lo.w,
                   a4 = two ? hi.z : hi.x, a5 = two ? hi.w : hi.y;
    const uint32_t b0 = one ? a1 : a0, b1 = one ? a2 : a1, b2 = one ? a3 : a2, b3 = one ? a4 : a3, b4 = one ? a5 : a4;
    const uint32_t r = off % 4 * 8;
    return make_uint4(__funnelshift_r(b0, b1, r), __funnelshift_r(b1, b2, r), __funnelshift_r(b2, b3, r),
                      __funnelshift_r(b3, b4, r));
  }
};

// A row of elements as 16-byte vectors: vector v holds elements v * kWidth -
// shift and on, where shift is how far the row starts behind a 16-byte
// boundary; vectors [lo, hi) lie in the row as a whole.
template <typename E>
struct Window {
  static constexpr uint32_t kWidth = Vec<E>::kWidth;
  E* row;
  uint32_t shift, end, lo, whole, vectors;

  __device__ __forceinline__ Window(E* p, uint32_t n)
      : row(p), shift((uint32_t)((uintptr_t)p % 16) / sizeof(E)), end(shift + n), lo(shift ? 1 : 0),
        whole(end / kWidth > lo ? end / kWidth - lo : 0), vectors((end + kWidth - 1) / kWidth) {}

  // Where vector v starts; for a first vector that reaches before the row, before it.
  __device__ __forceinline__ E* at(uint32_t v) const { return row + ((int64_t)v * kWidth - shift); }
  // Vector v, with -inf outside the row; `last`: it will not be read again.
  __device__ __forceinline__ uint4 load(uint32_t v, bool last) const {
    const uint4* p = reinterpret_cast<const uint4*>(at(v));
    if (v - lo < whole) return last ? __ldcs(p) : __ldcg(p);
    const uint32_t none = minus_inf_bits(E());
    uint4 u = make_uint4(none, none, none, none);
    if (v < vectors) u = load_ends<E>(at(v), v ? 0 : (int32_t)shift, (int32_t)(end - v * kWidth), none);
    return u;
  }
  // Whether vectors v, v + step, ... (N of them) all lie in the row as a whole.
  template <int N>
  __device__ __forceinline__ bool all_whole(uint32_t v, uint32_t step) const {
    return v - lo < whole && v - lo + (N - 1) * step < whole;
  }
  // Those vectors: read by one address and a step where they lie in the row (the
  // tests and addresses of single ones took more instructions than the
  // arithmetic of their elements).
  template <int N>
  __device__ __forceinline__ void load_many(uint4 (&u)[N], uint32_t v, uint32_t step, bool last) const {
    if (all_whole<N>(v, step)) {
      const uint4* p = reinterpret_cast<const uint4*>(at(v));
#pragma unroll
      for (int k = 0; k < N; ++k, p += step) u[k] = last ? __ldcs(p) : __ldcg(p);
    } else {
#pragma unroll
      for (int k = 0; k < N; ++k) u[k] = load(v + k * step, last);
    }
  }
  __device__ __forceinline__ void store(uint32_t v, const uint4& u) const {
    if (v - lo < whole) __stcs(reinterpret_cast<uint4*>(at(v)), u);
    else if (v < vectors) store_ends<E>(at(v), u, v ? 0 : (int32_t)shift, (int32_t)(end - v * kWidth));
  }
  // As store, for what is read again soon.
  __device__ __forceinline__ void put(uint32_t v, const uint4& u) const {
    if (v - lo < whole) *reinterpret_cast<uint4*>(at(v)) = u;
    else if (v < vectors) store_ends<E>(at(v), u, v ? 0 : (int32_t)shift, (int32_t)(end - v * kWidth));
  }
  // As store, for values cut into vectors at another row's boundaries (`from` behind one).
  __device__ __forceinline__ void store_cut(uint32_t v, uint32_t from, const uint4& u) const {
    const int64_t first = (int64_t)v * kWidth - from;
    if (first < (int64_t)(end - shift))
      store_ends<E>(row + first, u, v ? 0 : (int32_t)from, (int32_t)min((int64_t)kWidth, (int64_t)(end - shift) - first));
  }
};

}  // namespace bfk
