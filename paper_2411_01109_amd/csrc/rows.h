// Pieces of eight elements of rows of fp16 or fp32, as floats: what the kernels over whole rows (embed.hip, logprob.hip, clip.hip) load and store.
#pragma once

#include "common.h"

namespace hgnn {

// The hardware takes 16-byte accesses to global memory at any element's address, so rows of any pitch go in whole pieces.  The last piece of a row is read
// whole, too, where that stays inside the tensor (what it brings from beyond the row never reaches a result), else, and when it is written, in parts of four,
// two and one elements.
typedef half8_t half8_any_t __attribute__((aligned(2)));
typedef half4_t half4_any_t __attribute__((aligned(2)));
typedef half2_t half2_any_t __attribute__((aligned(2)));
typedef float float2_t __attribute__((ext_vector_type(2)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef float4_t float4_any_t __attribute__((aligned(4)));
typedef float2_t float2_any_t __attribute__((aligned(4)));

typedef float float8_t __attribute__((ext_vector_type(8)));

template <class T>
struct Vec;
template <>
struct Vec<half_t> {
  typedef half8_t eight;
  typedef half4_any_t four;
  typedef half2_any_t two;
};
template <>
struct Vec<float> {
  typedef float8_t eight;
  typedef float4_any_t four;
  typedef float2_any_t two;
};

// a piece as it is in memory: 16 bytes of fp16 or 32 of fp32 (vectors: of arrays whose places are chosen at run time the compiler makes memory)
template <class T>
struct RawPiece {
  typename Vec<T>::eight v;
};
struct Piece {
  float8_t v;
};

template <class T>
__device__ __forceinline__ RawPiece<T> load_raw(const T* p) {
  RawPiece<T> r;
  if constexpr (sizeof(T) == 2) {
    r.v = *reinterpret_cast<const half8_any_t*>(p);
  } else {
    const float4_t a = *reinterpret_cast<const float4_any_t*>(p), b = *reinterpret_cast<const float4_any_t*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = a[i], r.v[4 + i] = b[i];
  }
  return r;
}
// the first `left` of fewer than eight elements, the others zero
template <class T>
__device__ __forceinline__ RawPiece<T> load_raw_part(const T* p, int left) {
  RawPiece<T> r;
  r.v = 0;
  if (left & 4) {
    const auto x = *reinterpret_cast<const typename Vec<T>::four*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = x[i];
  }
  T t0{}, t1{}, o{};
  if (left & 2) {
    const auto x = *reinterpret_cast<const typename Vec<T>::two*>(p + (left & 4));
    t0 = x[0], t1 = x[1];
  }
  if (left & 1) o = p[left - 1];
  const bool f = left & 4, t = left & 2;
  r.v[0] = f ? r.v[0] : (t ? t0 : o);
  r.v[1] = f ? r.v[1] : t1;
  r.v[2] = f ? r.v[2] : (t ? o : T{});
  r.v[4] = f ? (t ? t0 : o) : T{};
  r.v[5] = f ? t1 : T{};
  r.v[6] = f && t ? o : T{};
  return r;
}
// a piece of a row, the row's last `left` elements, of a tensor that goes on for `inside` elements from p
template <class T>
__device__ __forceinline__ RawPiece<T> load_raw(const T* p, int left, int64_t inside) {
  return inside >= 8 ? load_raw(p) : load_raw_part(p, left);
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
  const bool f = left & 4, t = left & 2;
  const float x0 = x.v[0], x1 = x.v[1], x2 = x.v[2], x4 = x.v[4], x5 = x.v[5], x6 = x.v[6];
  const float t0 = f ? x4 : x0, t1 = f ? x5 : x1, o = f ? (t ? x6 : x4) : (t ? x2 : x0);
  if (f) {
    typename Vec<T>::four v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = T(x.v[i]);
    *reinterpret_cast<typename Vec<T>::four*>(p) = v;
    p += 4;
  }
  if (t) {
    typename Vec<T>::two v;
    v[0] = T(t0), v[1] = T(t1);
    *reinterpret_cast<typename Vec<T>::two*>(p) = v;
    p += 2;
  }
  if (left & 1) *p = T(o);
}

// ---- four elements: what a lane takes of a row that is written in fp32, so that the lanes' 16 bytes lie beside each other
template <class T>
__device__ __forceinline__ typename Vec<T>::four load_quad(const T* p, int left, int64_t inside) {
  typename Vec<T>::four r;
  if (inside >= 4) return *reinterpret_cast<const typename Vec<T>::four*>(p);
  r = 0;
  T t0{}, t1{}, o{};
  if (left & 2) {
    const auto x = *reinterpret_cast<const typename Vec<T>::two*>(p);
    t0 = x[0], t1 = x[1];
  }
  if (left & 1) o = p[left - 1];
  r[0] = left & 2 ? t0 : o, r[1] = t1, r[2] = left & 2 ? o : T{};
  return r;
}
template <class T, bool PAST = false>  // PAST: past the caches, for what is not read again soon (whole lines that other lanes fill, or it costs three times as much)
__device__ __forceinline__ void store_quad(T* p, int left, float4_t x) {
  if (left >= 4) {
    typename Vec<T>::four v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = T(x[i]);
    if (PAST) __builtin_nontemporal_store(v, reinterpret_cast<typename Vec<T>::four*>(p));
    else *reinterpret_cast<typename Vec<T>::four*>(p) = v;
    return;
  }
  if (left & 2) {
    typename Vec<T>::two v;
    v[0] = T(x[0]), v[1] = T(x[1]);
    *reinterpret_cast<typename Vec<T>::two*>(p) = v;
  }
  const float x0 = x[0], x2 = x[2];
  if (left & 1) p[left - 1] = T(left & 2 ? x2 : x0);
}

// ---- V elements of a tensor as they are in memory, eight or four
template <class T, int V>
struct Part;
template <class T>
struct Part<T, 8> {
  typename Vec<T>::eight v;
  static __device__ __forceinline__ Part load(const T* p) { return Part{load_raw(p).v}; }
  static __device__ __forceinline__ Part load(const T* p, int left, int64_t inside) { return Part{load_raw(p, left, inside).v}; }
  template <bool PAST>
  static __device__ __forceinline__ void store(T* p, int left, const float (&x)[8]) {
    const Piece y{{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]}};
    if constexpr (PAST && sizeof(T) == 2) {
      if (left >= 8) {
        half8_any_t h;
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = half_t(x[i]);
        __builtin_nontemporal_store(h, reinterpret_cast<half8_any_t*>(p));
        return;
      }
    }
    store_piece(p, left, y);
  }
};
template <class T>
struct Part<T, 4> {
  typename Vec<T>::four v;
  static __device__ __forceinline__ Part load(const T* p) { return Part{*reinterpret_cast<const typename Vec<T>::four*>(p)}; }
  static __device__ __forceinline__ Part load(const T* p, int left, int64_t inside) { return Part{load_quad(p, left, inside)}; }
  template <bool PAST>
  static __device__ __forceinline__ void store(T* p, int left, const float (&x)[4]) { store_quad<T, PAST>(p, left, float4_t{x[0], x[1], x[2], x[3]}); }
};

// Outputs of so many bytes are written past the caches: the last-level cache (256 MiB) would have lost most of them before they are read.  us, rows of 128 by
// id and then a reader of them, through / past: 61 MB 35 / 38, 122 MB 62 / 66, 244 MB 126 / 121 (the rows alone: 20 / 16, 41 / 31, 81 / 58).
constexpr double kPastBytes = 192. * (1 << 20);

// what a launch holds: fewer than 2^32 lanes
constexpr int64_t kMostBlocks = 0xffffffffll / kBlock;

inline bool known_type(hgnn_type t) { return t == HGNN_F16 || t == HGNN_F32; }
inline bool aligned_to_type(const void* p, hgnn_type t) { return (reinterpret_cast<uintptr_t>(p) & (t == HGNN_F32 ? 3u : 1u)) == 0; }
// elements from a tensor's first to its last: what a row's last piece may be read from
inline int64_t extent_of(int64_t rows, int64_t cols, int64_t ld) { return rows > 0 ? (rows - 1) * ld + cols : 0; }

}  // namespace hgnn
