// Device helpers of the kernels on rows (gfx950): pieces of rows and a row's position.
#pragma once

#include "common.hpp"

namespace fck {

// A piece of a row: 16 bytes of it, 8 bf16 or 4 fp32 values, as fp32.
template <bool F32>
struct Piece {
  static constexpr int V = F32 ? 4 : 8;
  typedef uint32_t word __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ void load(float (&x)[V], const void* p, int64_t e) {
    const word w = *reinterpret_cast<const word*>(static_cast<const char*>(p) + e * (16 / V));
#pragma unroll
    for (int j = 0; j < V; ++j)
      x[j] = __uint_as_float(F32 ? w[j] : j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
  }
};
// V values stored, 16 bytes of fp32 or V of bf16, not to be kept in the L2: another
// kernel is the next to read them. Against plain stores: own rows of 32/8 heads of
// 128 over 64K tokens and 8 ranks 43.5 -> 39.2 us, their gather 87.9 -> 82.2.
template <bool F32, int V>
__device__ __forceinline__ void store(void* p, int64_t e, const float (&x)[V]) {
  constexpr int N = F32 ? V : V / 2;
  typedef uint32_t word __attribute__((ext_vector_type(N)));
  word w;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if constexpr (F32)
      w[j] = __float_as_uint(x[j]);
    else
      w[j] = uint32_t(f2bf(x[2 * j])) | uint32_t(f2bf(x[2 * j + 1])) << 16;
  }
  word* q = reinterpret_cast<word*>(static_cast<char*>(p) + e * (F32 ? 4 : 2));
  __builtin_nontemporal_store(w, q);
}

// The unaligned layout (halves that are no multiple of 8 values apart): single values.
template <bool F32>
__device__ __forceinline__ float load1(const void* p, int64_t e) {
  return F32 ? static_cast<const float*>(p)[e] : bf2f(static_cast<const u16*>(p)[e]);
}
template <bool F32>
__device__ __forceinline__ void store1(void* p, int64_t e, float x) {
  if constexpr (F32)
    static_cast<float*>(p)[e] = x;
  else
    static_cast<u16*>(p)[e] = f2bf(x);
}

// Position of row r of a tensor of own or received tokens (S: gpos, first, end): in its
// document, or in the packed sequence.
template <class S>
__device__ __forceinline__ int row_pos(const S& s, const int32_t* seg, bool packed, int r) {
  int x = s.gpos[r];
  if (!packed) {
    int i = s.first[r / 64];
    while (r >= seg[4 * i + s.end]) ++i;
    x -= seg[4 * i + 2];
  }
  return x;
}

}  // namespace fck
