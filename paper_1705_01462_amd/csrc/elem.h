// elem.h -- element types of the attention block's tensors (fp32, fp16, bf16)
// as the kernels load and store them.
#pragma once

#include "fgq_internal.h"

namespace fgq {

typedef float ev4f __attribute__((ext_vector_type(4)));
typedef uint32_t ev4u __attribute__((ext_vector_type(4)));

// A pack of eight elements; rows may start anywhere (odd row lengths), and
// the hardware reads 16 unaligned bytes in one load.
template <int kBytes>
struct Pack;
template <>
struct Pack<2> {
  typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2)));
  static constexpr int kWords = 1;
};
template <>
struct Pack<4> {
  typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4)));
  static constexpr int kWords = 2;
};

__device__ inline float bf16_f32(uint32_t h) { return __uint_as_float(h << 16); }

template <int kType>
struct Elem;

template <>
struct Elem<FGQ_F32> {
  typedef float type;
  static constexpr int kBytes = 4;
  static __device__ float get(const void* p, int64_t i) { return static_cast<const float*>(p)[i]; }
  static __device__ void put(void* p, int64_t i, float v) { static_cast<float*>(p)[i] = v; }
};
template <>
struct Elem<FGQ_F16> {
  typedef _Float16 type;
  static constexpr int kBytes = 2;
  static __device__ float get(const void* p, int64_t i) { return static_cast<float>(static_cast<const _Float16*>(p)[i]); }
  static __device__ void put(void* p, int64_t i, float v) { static_cast<_Float16*>(p)[i] = static_cast<_Float16>(v); }
};
template <>
struct Elem<FGQ_BF16> {
  typedef __bf16 type;
  static constexpr int kBytes = 2;
  static __device__ float get(const void* p, int64_t i) { return bf16_f32(static_cast<const uint16_t*>(p)[i]); }
  static __device__ void put(void* p, int64_t i, float v) { static_cast<__bf16*>(p)[i] = static_cast<__bf16>(v); }
};

// Raw 16-byte packs of eight consecutive elements (one pack of 16-bit ones,
// two of fp32), and their values.
template <int kType>
struct Raw8 {
  static constexpr int kN = Elem<kType>::kBytes / 2;
  ev4u w[kN];
};

template <int kType>
__device__ inline Raw8<kType> load8(const void* p, int64_t i) {
  typedef typename Pack<Elem<kType>::kBytes>::type pk;
  Raw8<kType> r;
  const pk* s = reinterpret_cast<const pk*>(static_cast<const char*>(p) + i * Elem<kType>::kBytes);
#pragma unroll
  for (int j = 0; j < Raw8<kType>::kN; ++j) {
    const pk v = s[j];
    r.w[j] = ev4u{v.x, v.y, v.z, v.w};
  }
  return r;
}

template <int kType>
__device__ inline void values8(const Raw8<kType>& r, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if constexpr (kType == FGQ_F32) {
      v[j] = __uint_as_float(r.w[j / 4][j % 4]);
    } else {
      const uint32_t h = j % 2 ? r.w[0][j / 2] >> 16 : r.w[0][j / 2] & 0xFFFFu;
      if constexpr (kType == FGQ_BF16)
        v[j] = bf16_f32(h);
      else
        v[j] = static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(h)));
    }
  }
}

__device__ inline uint32_t pack_f16(float a, float b) {
  typedef _Float16 v2h __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, v2h{static_cast<_Float16>(a), static_cast<_Float16>(b)});
}
__device__ inline uint32_t pack_bf16(float a, float b) {
  typedef __bf16 v2b __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, v2b{static_cast<__bf16>(a), static_cast<__bf16>(b)});
}

// The packs that hold eight values (rounded to the type).
template <int kType>
__device__ inline Raw8<kType> raw8(const float (&v)[8]) {
  Raw8<kType> r;
#pragma unroll
  for (int e = 0; e < 4 * Raw8<kType>::kN; ++e) {
    if constexpr (kType == FGQ_F32)
      r.w[e / 4][e % 4] = __float_as_uint(v[e]);
    else
      r.w[0][e] = kType == FGQ_F16 ? pack_f16(v[2 * e], v[2 * e + 1]) : pack_bf16(v[2 * e], v[2 * e + 1]);
  }
  return r;
}

template <int kType>
__device__ inline void store8(void* p, int64_t i, const float (&v)[8]) {
  typedef typename Pack<Elem<kType>::kBytes>::type pk;
  pk* d = reinterpret_cast<pk*>(static_cast<char*>(p) + i * Elem<kType>::kBytes);
  const Raw8<kType> r = raw8<kType>(v);
#pragma unroll
  for (int j = 0; j < Raw8<kType>::kN; ++j) d[j] = pk{r.w[j].x, r.w[j].y, r.w[j].z, r.w[j].w};
}

// Lanes of a wave exchange data through LDS: the compiler keeps the accesses
// in this order, and the hardware does for the accesses of one wave.
__device__ inline void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// fn(integral_constant<type>) for a type that was validated.
template <typename F>
inline auto with_type(int32_t type, F&& fn) {
  if (type == FGQ_F32) return fn(std::integral_constant<int, FGQ_F32>{});
  if (type == FGQ_F16) return fn(std::integral_constant<int, FGQ_F16>{});
  return fn(std::integral_constant<int, FGQ_BF16>{});
}

inline bool type_ok(int32_t t) { return t == FGQ_F32 || t == FGQ_F16 || t == FGQ_BF16; }
inline int64_t type_bytes(int32_t t) { return t == FGQ_F32 ? 4 : 2; }

}  // namespace fgq
