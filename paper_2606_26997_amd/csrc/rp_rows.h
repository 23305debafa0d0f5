// Device helpers for kernels that read rows of logits: loads of 16 bytes a
// lane from rows of any alignment, conversions, reductions over a workgroup.
#pragma once

#include "rp_device.h"
#include "rp_internal.h"

namespace rp {

// Sixteen bytes at an address that is a multiple of the element's size only
// (rows of an odd length): global memory takes such accesses.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

template <int DT>
struct Elem;
template <>
struct Elem<RP_LOGITS_BF16> {
  static constexpr int kBytes = 2, kPerVec = 8;
  static __device__ inline float get(const void* p, long long i) {
    return __uint_as_float((uint32_t) static_cast<const uint16_t*>(p)[i] << 16);
  }
  static __device__ inline uint32_t bits(float x) { return pack_bf16x2(x, 0.f) & 0xFFFFu; }
};
template <>
struct Elem<RP_LOGITS_F16> {
  static constexpr int kBytes = 2, kPerVec = 8;
  static __device__ inline float get(const void* p, long long i) {
    return (float)static_cast<const _Float16*>(p)[i];
  }
  static __device__ inline uint32_t bits(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
};
template <>
struct Elem<RP_LOGITS_F32> {
  static constexpr int kBytes = 4, kPerVec = 4;
  static __device__ inline float get(const void* p, long long i) { return static_cast<const float*>(p)[i]; }
  static __device__ inline uint32_t bits(float x) { return __float_as_uint(x); }
};

template <int DT>
__device__ inline void put_elem(void* p, long long i, float x) {
  if constexpr (Elem<DT>::kBytes == 2) static_cast<uint16_t*>(p)[i] = (uint16_t)Elem<DT>::bits(x);
  else static_cast<uint32_t*>(p)[i] = Elem<DT>::bits(x);
}

template <int DT>
__device__ inline void unpack(const u32x4_any& v, float (&x)[Elem<DT>::kPerVec]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (DT == RP_LOGITS_F32) {
      x[k] = __uint_as_float(v[k]);
    } else if constexpr (DT == RP_LOGITS_BF16) {
      x[2 * k] = bf16_lo(v[k]);
      x[2 * k + 1] = bf16_hi(v[k]);
    } else {
      x[2 * k] = (float)__builtin_bit_cast(_Float16, (uint16_t)v[k]);
      x[2 * k + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(v[k] >> 16));
    }
  }
}
template <int DT>
__device__ inline u32x4_any pack(const float (&x)[Elem<DT>::kPerVec]) {
  u32x4_any v;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (DT == RP_LOGITS_F32) v[k] = __float_as_uint(x[k]);
    else if constexpr (DT == RP_LOGITS_BF16) v[k] = pack_bf16x2(x[2 * k], x[2 * k + 1]);
    else v[k] = Elem<DT>::bits(x[2 * k]) | Elem<DT>::bits(x[2 * k + 1]) << 16;
  }
  return v;
}

// Vector `vec` of a row, all of whose elements are in the row.
__device__ inline u32x4_any load_whole(const void* row, int vec) {
  return *reinterpret_cast<const u32x4_any*>(static_cast<const char*>(row) + (size_t)vec * 16);
}
// The same where the row may end inside: elements from `vocab` on are -inf.
template <int DT>
__device__ inline u32x4_any load_vec(const void* row, int vec, int vocab) {
  constexpr int E = Elem<DT>::kPerVec;
  const int first = vec * E;
  if (first + E <= vocab) return load_whole(row, vec);
  float x[E];
#pragma unroll
  for (int k = 0; k < E; ++k) x[k] = first + k < vocab ? Elem<DT>::get(row, first + k) : -INFINITY;
  return pack<DT>(x);
}

// Sums and maxima over a wave and over a workgroup of NT threads, in every
// thread; `lds` has a slot per wave. The workgroup forms begin with a barrier,
// so one may follow another on the same slots at once; they end with reads of
// them, so whatever else writes there needs a barrier first. The order of
// additions is fixed.
template <class T>
__device__ inline T wave_sum(T x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
template <int NT, class T>
__device__ inline T block_sum(T x, T* lds) {
  x = wave_sum(x);
  __syncthreads();
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = x;
  __syncthreads();
  T s = lds[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) s += lds[w];
  return s;
}
template <int NT>
__device__ inline float block_max(float x, float* lds) {
  x = wave_max(x);
  __syncthreads();
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = x;
  __syncthreads();
  float m = lds[0];
#pragma unroll
  for (int w = 1; w < NT / 64; ++w) m = fmaxf(m, lds[w]);
  return m;
}

}  // namespace rp
