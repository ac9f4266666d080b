// Pieces of eight elements of rows of fp16 or fp32, as floats: what the kernels over whole rows (embed.hip, logprob.hip, clip.hip) load and store.
#pragma once

#include "common.h"

namespace hgnn {

// The hardware takes 16-byte accesses to global memory at any element's address, so rows of any pitch go in whole pieces; only the last piece of a row goes by
// element, and nothing behind a row is touched.
typedef half8_t half8_any_t __attribute__((aligned(2)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef float4_t float4_any_t __attribute__((aligned(4)));

struct Piece {
  float v[8];
};

__device__ __forceinline__ Piece load_piece(const half_t* p) {
  const half8_t h = *reinterpret_cast<const half8_any_t*>(p);
  Piece r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.v[i] = float(h[i]);
  return r;
}
__device__ __forceinline__ Piece load_piece(const float* p) {
  const float4_t a = *reinterpret_cast<const float4_any_t*>(p), b = *reinterpret_cast<const float4_any_t*>(p + 4);
  return Piece{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}
// as it is in memory, the elements behind the first `left` as zeros
__device__ __forceinline__ half8_t load_halves(const half_t* p, int left) {
  if (left >= 8) return *reinterpret_cast<const half8_any_t*>(p);
  half8_t h = {};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < left) h[i] = p[i];
  return h;
}
// the first `left` elements, the others as `none`
template <class T>
__device__ __forceinline__ Piece load_piece(const T* p, int left, float none) {
  if (left >= 8) return load_piece(p);
  Piece r;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    r.v[i] = none;
    if (i < left) r.v[i] = float(p[i]);
  }
  return r;
}

__device__ __forceinline__ void store_piece(half_t* p, const Piece& x) {
  half8_t h;
#pragma unroll
  for (int i = 0; i < 8; ++i) h[i] = half_t(x.v[i]);
  *reinterpret_cast<half8_any_t*>(p) = h;
}
__device__ __forceinline__ void store_piece(float* p, const Piece& x) {
  *reinterpret_cast<float4_any_t*>(p) = float4_t{x.v[0], x.v[1], x.v[2], x.v[3]};
  *reinterpret_cast<float4_any_t*>(p + 4) = float4_t{x.v[4], x.v[5], x.v[6], x.v[7]};
}
template <class T>
__device__ __forceinline__ void store_piece(T* p, int left, const Piece& x) {
  if (left >= 8) return store_piece(p, x);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < left) p[i] = T(x.v[i]);
}

inline bool known_type(hgnn_type t) { return t == HGNN_F16 || t == HGNN_F32; }
inline bool aligned_to_type(const void* p, hgnn_type t) { return (reinterpret_cast<uintptr_t>(p) & (t == HGNN_F32 ? 3u : 1u)) == 0; }

}  // namespace hgnn
