// Matrices made orthogonal by Newton-Schulz products:  X = G / |G|, then `steps` times  A = X X^T,  B = b A + c A A,  X <- a X + B X,  out = scale X
// (of the transpose where the matrix is higher than wide, so that A is the smaller product).
//
// The polynomial multiplies small singular values by a at each step, so an error of the first products comes out a^steps times as large: half precision products
// leave a result that is off by percents.  Every value is therefore kept as two fp16 numbers, v = hi + lo with hi = fp16(v) and lo = fp16(v - hi), some 22 bits, and
// a product is hi hi + hi lo + lo hi in fp32 sums (lo lo is below the last bit; narrow matrices, whose few sums do not hide it, add it): three products on the matrix cores, a fifth of what fp32's own rate would take.
// Powers of two bring the values into fp16's range: X at 2^11 (values up to 8 x 2^11 fit, what is lost at the small end is 2^-36), A and B at 2^9 (up to 64).
// A and B are symmetric: tiles on and below the diagonal alone, each written to its mirror place, too (a tile on the diagonal only once: its two triangles are
// summed in different orders, and two writers would make the result a race).
// All matrices are padded to multiples of 32 with zeros, which stay zeros through every product.
#include <algorithm>
#include <cmath>

#include "product.h"
#include "rows.h"

namespace hgnn {

constexpr float kX = 2048.f, kA = 512.f;  // what X, and A and B, are stored times
constexpr int kNormParts = 1024;

__device__ __forceinline__ void split_value(float v, half_t& hi, half_t& lo) {
  hi = half_t(v);
  lo = half_t(v - float(hi));
}
// a matrix of values in two parts, 32 high ones and their 32 low ones in turn; ld: halves of a line
struct Pairs {
  half_t* at;
  int64_t ld;
  __device__ half_t* place(int64_t q, int64_t p) const { return at + q * ld + 2 * p - (p & 31); }
  struct Four {
    half4_t h, l;
    __device__ float4_t value() const {
      float4_t r;
#pragma unroll
      for (int e = 0; e < 4; ++e) r[e] = float(h[e]) + float(l[e]);
      return r;
    }
  };
  __device__ Four get(int64_t q, int64_t p) const {
    const half_t* const v = place(q, p);
    return {*reinterpret_cast<const half4_t*>(v), *reinterpret_cast<const half4_t*>(v + 32)};
  }
  __device__ void put(int64_t q, int64_t p, const float4_t& v, bool mirror) const {
    half4_t h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      half_t a, b;
      split_value(v[e], a, b);
      h[e] = a, l[e] = b;
    }
    half_t* const to = place(q, p);
    *reinterpret_cast<half4_t*>(to) = h;
    *reinterpret_cast<half4_t*>(to + 32) = l;
    if (!mirror) return;
    half_t* const over = place(p, q);
#pragma unroll
    for (int e = 0; e < 4; ++e) over[e * ld] = h[e], over[e * ld + 32] = l[e];
  }
};

// ---- what becomes of the sums
struct GramOut {  // A, or b A where that is all of B
  Pairs to;
  float factor;
  int tile;
  typedef ProductNothing Read;
  __device__ Read read(int64_t, int64_t) const { return {}; }
  template <bool WHOLE>
  __device__ void put(int64_t, int64_t q, int64_t p, const Read&, const float4_t& v) const { to.put(q, p, v * factor, q / tile != p / tile); }
  __device__ float4_t join(int64_t q, int64_t p, const float4_t& v) const {  // the value that stands at (q, p) then
    to.put(q, p, v * factor, false);
    return v * factor;
  }
};
struct SquareOut {  // B = b A + c A A
  Pairs to, A;
  float b, c;
  int tile;
  typedef Pairs::Four Read;
  __device__ Read read(int64_t q, int64_t p) const { return A.get(q, p); }
  template <bool WHOLE>
  __device__ void put(int64_t, int64_t q, int64_t p, const Read& x, const float4_t& v) const { to.put(q, p, x.value() * b + v * c, q / tile != p / tile); }
  __device__ float4_t join(int64_t q, int64_t p, const float4_t& v) const {
    const float4_t y = read(q, p).value() * b + v * c;
    to.put(q, p, y, false);
    return y;
  }
};
struct StepOut {  // X = a X + B X
  Pairs to, X;
  float a;
  typedef Pairs::Four Read;
  __device__ Read read(int64_t q, int64_t p) const { return X.get(q, p); }
  template <bool WHOLE>
  __device__ void put(int64_t, int64_t q, int64_t p, const Read& x, const float4_t& v) const { to.put(q, p, x.value() * a + v * (1.f / kA), false); }
  __device__ float4_t join(int64_t q, int64_t p, const float4_t& v) const {
    put<false>(0, q, p, read(q, p), v);
    return v;
  }
};
struct LastOut {  // the same into the caller's matrix
  Pairs X, to;  // to: not used
  float a, scale;
  void* out;
  int64_t ld, rows, cols;  // of X without its padding
  int type, flip;
  typedef Pairs::Four Read;
  __device__ Read read(int64_t q, int64_t p) const { return X.get(q, p); }
  template <bool WHOLE>
  __device__ void put(int64_t, int64_t q, int64_t p, const Read& old, const float4_t& v) const {
    if (q >= rows) return;
    const float4_t x = (old.value() * a + v * (1.f / kA)) * scale;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (p + e >= cols) return;
      const int64_t at = flip ? (p + e) * ld + q : q * ld + p + e;
      if (type == HGNN_F16) static_cast<half_t*>(out)[at] = half_t(x[e]);
      else static_cast<float*>(out)[at] = x[e];
    }
  }
  __device__ float4_t join(int64_t q, int64_t p, const float4_t& v) const {
    put<false>(0, q, p, read(q, p), v);
    return v;
  }
};
struct SumsPart {  // [parts][nq - q0][np]
  float* part;
  int64_t q0, nq, np;
  typedef ProductNothing Read;
  __device__ Read read(int64_t, int64_t) const { return {}; }
  template <bool WHOLE>
  __device__ void put(int64_t k, int64_t q, int64_t p, const Read&, const float4_t& v) const { *reinterpret_cast<float4_t*>(part + (k * (nq - q0) + q - q0) * np + p) = v; }
};
// The parts of 32 x 32 sums in order (blockIdx.x and y, from line `from` on, of the tiles on and below the diagonal with `lower`, and of those the ones in tiles of
// 128 x 128 from number `first` on), four sums a lane, and what becomes of them; the mirror
// places get theirs through LDS, in whole pieces (by twos the join of 1024 x 1024 took 11 us; tiles of 64 x 64, sixteen sums a lane, took 10.4 us for 7 parts of
// 1024 x 1024, bound by their chains of loads, these 5.4).
constexpr int kJoinTile = 32;
template <class Out>
__global__ __launch_bounds__(kBlock) void sums_join_kernel(const float* part, int parts, int64_t from, int64_t nq, int64_t np, int lower, int first, Out out) {
  __shared__ __align__(16) float tile[kJoinTile][kJoinTile + 4];
  static_assert(kJoinTile * kJoinTile == 4 * kBlock, "four sums a lane");
  const int64_t tq = from / kJoinTile + blockIdx.x, tp = blockIdx.y, line = tq * kJoinTile / 128;
  if (lower && (tp > tq || line * (line + 1) / 2 + tp * kJoinTile / 128 < first)) return;  // uniform
  const int64_t q0 = tq * kJoinTile, p0 = tp * kJoinTile;
  const bool mirror = lower && tp < tq;
  const int r = threadIdx.x / (kJoinTile / 4), c = 4 * (threadIdx.x % (kJoinTile / 4));
  const int64_t q = q0 + r, p = p0 + c;
  if (q < nq && p < np) {
    float4_t v = {0.f, 0.f, 0.f, 0.f};
    const float* at = part + (q - from) * np + p;
#pragma unroll 8
    for (int k = 0; k < parts; ++k, at += (nq - from) * np) v += *reinterpret_cast<const float4_t*>(at);
    const float4_t y = out.join(q, p, v);
    if (mirror) {
#pragma unroll
      for (int e = 0; e < 4; ++e) tile[c + e][r] = y[e];
    }
  }
  if (!mirror) return;
  __syncthreads();
  if (p0 + r < np && q0 + c < nq) out.to.put(p0 + r, q0 + c, *reinterpret_cast<const float4_t*>(&tile[r][c]), false);
}

// ---- the way in: the norm, X = G / |G|
struct OrthMatrix {
  const void* grad;
  void* out;
  int64_t rows, cols, ld, ldo;
  int type, out_type;
};
// sum over a workgroup of N threads, on all threads
template <int N = kBlock>
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double lds[N];
  lds[threadIdx.x] = v;
  __syncthreads();
  for (int w = N / 2; w > 0; w >>= 1) {
    if (int(threadIdx.x) < w) lds[threadIdx.x] += lds[threadIdx.x + w];
    __syncthreads();
  }
  return lds[0];
}
// The sum of the squares of a share of a matrix, number `share` of `shares`, in 64 bits: no element's square is lost or overflows.  Pieces of eight elements, four
// of them on their way at a time.
template <class T>
__device__ __forceinline__ double squares_of(const OrthMatrix& m, int share, int shares) {
  const T* const g = static_cast<const T*>(m.grad);
  const bool flat = m.ld == m.cols;  // one row of all elements
  const int64_t rows = flat ? 1 : m.rows, cols = flat ? m.rows * m.cols : m.cols, each = (cols + 7) / 8, all = rows * each, extent = (rows - 1) * m.ld + cols;
  const int64_t step = int64_t(shares) * blockDim.x;
  double s = 0.;
  for (int64_t e = int64_t(share) * blockDim.x + threadIdx.x; e < all; e += 4 * step) {
    RawPiece<T> x[4];
    int left[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t at = e + u * step, r = flat ? 0 : at / each, c = 8 * (at - r * each);
      left[u] = at < all ? int(min(cols - c, int64_t(8))) : 0;
      x[u].v = 0;
      if (left[u] > 0) x[u] = load_raw(g + r * m.ld + c, left[u], extent - (r * m.ld + c));
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double v = i < left[u] ? double(x[u].v[i]) : 0.;
        s = fma(v, v, s);
      }
  }
  return s;
}
__device__ __forceinline__ double squares_of(const OrthMatrix& m, int share, int shares) {
  return m.type == HGNN_F16 ? squares_of<half_t>(m, share, shares) : squares_of<float>(m, share, shares);
}
__global__ __launch_bounds__(kBlock) void orth_squares_kernel(OrthMatrix m, double* part) {
  const double s = block_sum(squares_of(m, blockIdx.x, gridDim.x));
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}
// 1 / |G|, or 0 where that is none
__device__ __forceinline__ double inverse_root(double s) { return s > 0. && s < double(INFINITY) ? 1. / sqrt(s) : 0.; }
__device__ __forceinline__ double inverse_norm(const double* part, int parts) {
  double s = 0.;
  for (int k = threadIdx.x; k < parts; k += kBlock) s += part[k];
  s = block_sum(s);
  return inverse_root(s);
}
// 64 x 64 elements of X = G / |G| (of its transpose with `flip`) at kX times their values, zeros in the padding (hq x hp in all), by N threads; with `last` the scaled
// elements of the result in their place.  Through LDS, so that lines are read and written along themselves in pieces of eight either way.
constexpr int kTurn = 64;
template <class T>
__device__ __forceinline__ void load_turn(const OrthMatrix& m, int64_t r, int64_t c, double f, float (&v)[8]) {
  const T* const g = static_cast<const T*>(m.grad) + r * m.ld + c;
  const int left = r < m.rows && c < m.cols ? int(min(m.cols - c, int64_t(8))) : 0;
  RawPiece<T> x;
  x.v = 0;
  if (left > 0) x = load_raw(g, left, (m.rows - 1 - r) * m.ld + m.cols - c);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < left && f > 0. ? float(double(x.v[e]) * f) : 0.f;
}
template <int N>
__device__ __forceinline__ void orth_turn(const OrthMatrix& m, int flip, double inv, int64_t q0, int64_t p0, const Pairs& X, int64_t hq, int64_t hp, int last, float scale) {
  __shared__ float tile[kTurn][kTurn + 1];
  const int64_t r0 = flip ? p0 : q0, c0 = flip ? q0 : p0;
#pragma unroll
  for (int e = threadIdx.x; e < kTurn * 8; e += N) {
    const int r = e / 8, c = 8 * (e % 8);
    float v[8];
    if (m.type == HGNN_F16) load_turn<half_t>(m, r0 + r, c0 + c, inv * double(kX), v);
    else load_turn<float>(m, r0 + r, c0 + c, inv * double(kX), v);
    if (last && r0 + r < m.rows) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float y = v[k] * (scale / kX);
        if (c0 + c + k >= m.cols) break;
        const int64_t at = (r0 + r) * m.ldo + c0 + c + k;
        if (m.out_type == HGNN_F16) static_cast<half_t*>(m.out)[at] = half_t(y);
        else static_cast<float*>(m.out)[at] = y;
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) tile[r][c + k] = v[k];
  }
  if (last) return;
  __syncthreads();
#pragma unroll
  for (int e = threadIdx.x; e < kTurn * 8; e += N) {
    const int q = e / 8, p = 8 * (e % 8);
    if (q0 + q >= hq || p0 + p >= hp) continue;
    half8_t h, l;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      half_t a, b;
      split_value(flip ? tile[p + k][q] : tile[q][p + k], a, b);
      h[k] = a, l[k] = b;
    }
    half_t* const to = X.place(q0 + q, p0 + p);
    *reinterpret_cast<half8_t*>(to) = h;
    *reinterpret_cast<half8_t*>(to + 32) = l;
  }
}
__global__ __launch_bounds__(kBlock) void orth_begin_kernel(OrthMatrix m, int flip, const double* part, int parts, Pairs X, int64_t hq, int64_t hp, int last, float scale) {
  const double inv = inverse_norm(part, parts);
  orth_turn<kBlock>(m, flip, inv, int64_t(blockIdx.y) * kTurn, int64_t(blockIdx.x) * kTurn, X, hq, hp, last, scale);
}

static int64_t up32(int64_t n) { return (n + 31) / 32 * 32; }

// ---- shapes: tiles of 64 where a side is short, else of 128
template <bool PCOL>
using SplitSmall = ProductShape<2, 2, 2, 2, kSplit, false, PCOL, 3>;
template <bool PCOL>
using SplitMid = ProductShape<2, 2, 4, 4, kSplit, false, PCOL, 2>;
// ... and where there is at most one workgroup for a compute unit, all of its LDS for stages on their way
template <bool PCOL>
using SplitDeep = ProductShape<4, 2, 2, 4, kSplit, false, PCOL, 4>;
constexpr int kOrthFull = 256;
struct OrthSplit {
  int tile, parts;
  int64_t part;
  int first, rest, rest_parts;  // the tiles from `first` on by themselves, their contraction cut; rest = 0: none
  int64_t rest_part, from;      // lines from `from` on
};
// 128 x 128 tiles that run at a time, two a compute unit.  A few more than a multiple of that would take as long as half of all: they are a launch of their own, their
// contraction cut for as many workgroups.  Five steps, ten such products, ms in one launch each and so: 4096 x 4096 (528 tiles) 3.94 and 3.67, 4224 (561) 4.47 and 4.27, 4352 (595)
// 4.66 and 4.52, 4480 (630) 4.91 and 4.84, 5760 (1035) 10.43 and 9.95, 6016 (1128) 11.71 and 11.51, 7040 (1540) 18.96 and 18.45, 7296 (1653) 20.93 and 20.58; 4096 x 5120 4.67 and
// 4.31, 4480 x 5504 5.81 and 5.59.
constexpr int kOrthAtOnce = 512;
static OrthSplit orth_split(int64_t nq, int64_t np, int64_t K, bool lower) {
  const auto tiles = [&](int64_t b) {
    const int64_t l = ceil_div(nq, b);
    return lower ? l * (l + 1) / 2 : l * ceil_div(np, b);
  };
  OrthSplit s{};
  // Tiles of 64 read LDS twice as often for their products: where a side is short, or where a compute unit has at most one of them and a short contraction (1024 x
  // 1024, K = 1024, us: 136 of them 15, 36 of 128 in four parts 14 and a join of 5; K = 4096: 136 in four parts 22.5, 36 of 128 in seven 20.5, and the join).  Parts until
  // every compute unit has a workgroup, of 256 steps at least (a join costs about as much as those).
  s.tile = std::min(nq, np) < 192 || (tiles(64) <= kOrthFull && K <= 1024) ? 64 : 128;
  const int64_t t = tiles(s.tile), parts = t > kOrthFull / 2 || K <= 1024 ? 1 : std::min(kOrthFull / t, std::max<int64_t>(1, K / 256));
  s.part = std::max<int64_t>(32, up32(ceil_div(K, std::max<int64_t>(parts, 1))));
  s.parts = int(std::max<int64_t>(1, ceil_div(K, s.part)));
  const int64_t rest = t % kOrthAtOnce;
  if (lower && s.tile == 128 && t > kOrthAtOnce && t <= 4 * kOrthAtOnce && rest > 0 && rest <= kOrthAtOnce / 4 && K >= 1024) {
    s.first = int(t - rest), s.rest = int(rest);
    s.rest_part = up32(ceil_div(K, std::min(kOrthAtOnce / rest, K / 256)));
    s.rest_parts = int(ceil_div(K, s.rest_part));
    int64_t line = 0;
    while ((line + 1) * (line + 2) / 2 <= s.first) ++line;
    s.from = line * 128;
  }
  return s;
}
struct OrthSizes {
  int64_t m, k;  // padded, m <= k
  int flip;
  OrthSplit gram, square, step;
  size_t x, a, part, bytes;
};
static OrthSizes orth_sizes(int64_t rows, int64_t cols) {
  OrthSizes z{};
  z.flip = rows > cols;
  z.m = up32(std::min(rows, cols)), z.k = up32(std::max(rows, cols));
  z.gram = orth_split(z.m, z.m, z.k, true), z.square = orth_split(z.m, z.m, z.m, true), z.step = orth_split(z.m, z.k, z.m, false);
  const auto part = [](const OrthSplit& s, int64_t q, int64_t p) {
    return s.parts > 1 ? size_t(s.parts) * size_t(q) * size_t(p) * 4 : s.rest ? size_t(s.rest_parts) * size_t(q - s.from) * size_t(p) * 4 : 0;
  };
  z.x = size_t(z.m) * size_t(z.k) * 2, z.a = size_t(z.m) * size_t(z.m) * 2;
  z.part = std::max({part(z.gram, z.m, z.m), part(z.square, z.m, z.m), part(z.step, z.m, z.k)});
  z.bytes = kNormParts * sizeof(double) + 4 * z.x + 4 * z.a + z.part;
  return z;
}

// ---- matrices of at most 64 x 4096: a launch for a step of all of them.  A workgroup owns 64 columns of X, forms A and B by itself (each of a matrix's workgroups
// the same: their sums over the columns out of the L2 cost less than two launches more) and multiplies its columns.  X is padded to 64 rows and whole 64 columns.
// Two teams of four waves take 32 of 64 steps of A each, 32 x 32 of the 64 x 64 a wave; behind that a wave has 32 x 16.  A and B stand in LDS as the products read
// them.  (Five matrices of up to 608 x 64: 10.2 to 10.6 us a step, with one team 10.7; twenty of up to 64 x 4096 574 us in all, by a launch for a product of each 1230.)
// The low parts' product is formed here, too: it costs nothing beside the rest.
constexpr int kNarrowM = 64, kNarrowK = 4096, kNarrowMany = 24, kNarrowRing = 5, kNarrowTile = 64 * 128, kNarrowWaves = 8;
struct NarrowMatrix {
  OrthMatrix m;
  half_t *X, *next;
  int32_t first;  // workgroup
  int32_t k;      // padded columns
  float scale;
  int32_t flip;
};
struct NarrowArgs {
  NarrowMatrix m[kNarrowMany];
  int count;
  float a, b, c;
  int last;
};
__device__ __forceinline__ const NarrowMatrix& narrow_matrix(const NarrowArgs& a, int block) {
  int i = 0;
  while (i + 1 < a.count && a.m[i + 1].first <= block) ++i;  // uniform
  return a.m[i];
}
// the norm (each of a matrix's workgroups the same, from all of the gradient, which this launch therefore only reads) and X = G / |G|
__global__ __launch_bounds__(1024) void narrow_begin_kernel(NarrowArgs a) {
  const NarrowMatrix& n = narrow_matrix(a, blockIdx.x);
  const double inv = inverse_root(block_sum<1024>(squares_of(n.m, 0, 1)));
  orth_turn<1024>(n.m, n.flip, inv, 0, 64 * int64_t(int(blockIdx.x) - n.first), Pairs{n.X, 2 * int64_t(n.k)}, kNarrowM, n.k, 0, n.scale);
}
// Without steps the result is the scaled gradient, in place over the gradient itself: the norms, a workgroup a matrix, are a launch before it, since no workgroup may
// write its columns while another still sums the squares of all of them.
__global__ __launch_bounds__(1024) void narrow_norms_kernel(NarrowArgs a) {
  const NarrowMatrix& n = a.m[blockIdx.x];
  const double inv = inverse_root(block_sum<1024>(squares_of(n.m, 0, 1)));
  if (threadIdx.x == 0) *reinterpret_cast<double*>(n.X) = inv;
}
__global__ __launch_bounds__(1024) void narrow_scale_kernel(NarrowArgs a) {
  const NarrowMatrix& n = narrow_matrix(a, blockIdx.x);
  const double inv = *reinterpret_cast<const double*>(n.X);
  orth_turn<1024>(n.m, n.flip, inv, 0, 64 * int64_t(int(blockIdx.x) - n.first), Pairs{n.X, 2 * int64_t(n.k)}, kNarrowM, n.k, 1, n.scale);
}
// four values (q, p .. p + 3) of a 64 x 64 matrix to where ProductReads<false, true> finds them
__device__ __forceinline__ void narrow_put(unsigned char* at, int q, int p, const float4_t& v) {
  half4_t h, l;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    half_t a, b;
    split_value(v[e], a, b);
    h[e] = a, l[e] = b;
  }
  unsigned char* const line = at + (p >> 5) * kNarrowTile + q * 128 + (p & 4) * 2;
  const int piece = (p & 31) >> 3, turn = (q & 15) >> 1;
  *reinterpret_cast<half4_t*>(line + (piece ^ turn) * 16) = h;
  *reinterpret_cast<half4_t*>(line + ((piece + 4) ^ turn) * 16) = l;
}
__device__ __forceinline__ float4_t narrow_get(const unsigned char* at, int q, int p) {
  const unsigned char* const line = at + (p >> 5) * kNarrowTile + q * 128 + (p & 4) * 2;
  const int piece = (p & 31) >> 3, turn = (q & 15) >> 1;
  return Pairs::Four{*reinterpret_cast<const half4_t*>(line + (piece ^ turn) * 16), *reinterpret_cast<const half4_t*>(line + ((piece + 4) ^ turn) * 16)}.value();
}
// Sums of products of two parts each.  The matrix cores cut what they add off where a lane's addition rounds it, so the high parts of 32 steps are summed by
// themselves and added to the rest by the lane, and what the low parts add has a sum of its own: 9 x 809, eight steps, is off by 1.1e-6 of its norm (median of eight), in
// one sum for all by 1.7e-6, and products in fp32 by 1.1e-6.
template <int U>
struct NarrowSums {
  float4_t high[2][U], low[2][U];  // [16 lines][16 items]
  __device__ __forceinline__ NarrowSums() {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int u = 0; u < U; ++u) high[t][u] = low[t][u] = float4_t{0.f, 0.f, 0.f, 0.f};
  }
  __device__ __forceinline__ void add(const half8_t (&a)[2][2], const half8_t (&b)[2][U]) {  // [part][16 items]
    const float4_t none = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int u = 0; u < U; ++u) high[t][u] += __builtin_amdgcn_mfma_f32_16x16x32_f16(b[0][u], a[0][t], none, 0, 0, 0);
#pragma unroll
    for (int k = 3; k >= 1; --k)  // low low, then low high, high low
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int u = 0; u < U; ++u) low[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[k >> 1][u], a[k & 1][t], low[t][u], 0, 0, 0);
  }
  __device__ __forceinline__ float4_t sum(int t, int u) const { return high[t][u] + low[t][u]; }
};
__global__ __launch_bounds__(kNarrowWaves* kWave) void narrow_step_kernel(NarrowArgs a) {
  extern __shared__ __align__(1024) unsigned char lds[];
  constexpr int kStage = 2 * kNarrowTile;  // 64 steps
  unsigned char *const columns = lds + kNarrowRing * kStage, *const gram = columns + 2 * kNarrowTile, *const poly = gram + 2 * kNarrowTile;
  const NarrowMatrix& n = narrow_matrix(a, blockIdx.x);
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), i = lane & 15, qq = lane >> 4;
  const int k = n.k, steps = k / 64, p0 = 64 * (int(blockIdx.x) - n.first);
  const int64_t ld = 2 * int64_t(k);
  const uint32_t lds0 = uint32_t(uintptr_t((__attribute__((address_space(3))) unsigned char*)lds)) + wave * 1024;
  const half_t* const x = n.X;
  {  // the workgroup's own columns, 64 steps
    ProductLoads<1, true> own;
    product_loads<1, true, true, kNarrowWaves>(own, x, x, ld, p0, k, 0, wave, lane, 8);
#pragma unroll
    for (int s = 0; s < 2; ++s) load_to_lds(own.base[0] + s * own.inc, own.off[0], lds0 + kNarrowRing * kStage + s * kNarrowTile);
  }
  ProductLoads<1, false> lines;
  product_loads<1, false, true, kNarrowWaves>(lines, x, x, ld, 0, kNarrowM, 0, wave, lane, 8);
  uint32_t to = lds0;
  const auto ask = [&]() __attribute__((always_inline)) {
    load_to_lds(lines.base[0], lines.off[0], to);
    load_to_lds(lines.base[0] + lines.inc, lines.off[0], to + kNarrowTile);
    lines.base[0] += 2 * lines.inc;
    to += kStage;
    if (to >= lds0 + kNarrowRing * kStage) to -= kNarrowRing * kStage;
  };
  int asked = 0;
  for (; asked < kNarrowRing - 1 && asked < steps; ++asked) ask();
  {
    const int team = wave >> 2, wq = (wave >> 1) & 1, wp = wave & 1;
    const ProductReads<false, true, 2> read_q(2 * wq, lane), read_p(2 * wp, lane);
    NarrowSums<2> A;
    const unsigned char* stage = lds + team * kNarrowTile;
    for (int s = 0; s < steps; ++s) {
      const int behind = asked - 1 - s;
      if (behind >= 3) product_wait<6>();
      else if (behind == 2) product_wait<4>();
      else if (behind == 1) product_wait<2>();
      else product_wait<0>();
      if (asked < steps) ask(), ++asked;  // into the place of the stage before, which all waves have left
      half8_t u[2][2], v[2][2];
#pragma unroll
      for (int o = 0; o < 2; ++o)
#pragma unroll
        for (int t = 0; t < 2; ++t) u[o][t] = read_q.get(stage, t, o), v[o][t] = read_p.get(stage, t, o);
      A.add(u, v);
      stage += kStage;
      if (stage >= columns) stage -= kNarrowRing * kStage;
    }
    // the second team's sums to the first through what is B's place later
    float4_t* const over = reinterpret_cast<float4_t*>(poly) + (wave & 3) * 4 * kWave + lane;
    if (team == 1) {
#pragma unroll
      for (int t = 0; t < 4; ++t) over[t * kWave] = A.sum(t >> 1, t & 1);
    }
    __syncthreads();
    if (team == 0) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
        narrow_put(gram, 16 * (2 * wq + (t >> 1)) + i, 16 * (2 * wp + (t & 1)) + 4 * qq, (A.sum(t >> 1, t & 1) + over[t * kWave]) * (kA / (kX * kX)));
    }
    __syncthreads();
  }
  const int wq = wave >> 2, wp = wave & 3, p = 16 * wp + 4 * qq;
  const ProductReads<false, true, 2> read_q(2 * wq, lane);
  const ProductReads<false, true, 1> read_p(wp, lane);
  const auto q_of = [&](int t) { return 16 * (2 * wq + t) + i; };
  NarrowSums<1> B, Y;
  const auto lines_of = [&](const unsigned char* at, half8_t (&u)[2][2]) __attribute__((always_inline)) {
#pragma unroll
    for (int o = 0; o < 2; ++o)
#pragma unroll
      for (int t = 0; t < 2; ++t) u[o][t] = read_q.get(at, t, o);
  };
  if (a.c != 0.f) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      half8_t u[2][2], v[2][1];
      lines_of(gram + s * kNarrowTile, u);
#pragma unroll
      for (int o = 0; o < 2; ++o) v[o][0] = read_p.get(gram + s * kNarrowTile, 0, o);
      B.add(u, v);
    }
  }
#pragma unroll
  for (int t = 0; t < 2; ++t) narrow_put(poly, q_of(t), p, narrow_get(gram, q_of(t), p) * a.b + B.sum(t, 0) * (a.c / kA));
  __syncthreads();
  const ProductReads<true, true, 2> read_columns(wp & ~1, lane);
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    half8_t u[2][2], v[2][1];
    lines_of(poly + s * kNarrowTile, u);
#pragma unroll
    for (int o = 0; o < 2; ++o) {
      if (wp & 1) v[o][0] = read_columns.get(columns + s * kNarrowTile, 1, o);  // uniform
      else v[o][0] = read_columns.get(columns + s * kNarrowTile, 0, o);
    }
    Y.add(u, v);
  }
  const Pairs X{n.X, ld};
  if (a.last) {
    const LastOut out{X, X, a.a, n.scale / kX, n.m.out, n.m.ldo, n.flip ? n.m.cols : n.m.rows, n.flip ? n.m.rows : n.m.cols, n.m.out_type, n.flip};
#pragma unroll
    for (int t = 0; t < 2; ++t) out.put<false>(0, q_of(t), p0 + p, out.read(q_of(t), p0 + p), Y.sum(t, 0));
  } else {
    const StepOut out{Pairs{n.next, ld}, X, a.a};
#pragma unroll
    for (int t = 0; t < 2; ++t) out.put<false>(0, q_of(t), p0 + p, out.read(q_of(t), p0 + p), Y.sum(t, 0));
  }
}
static bool is_narrow(int64_t rows, int64_t cols) { return std::min(rows, cols) <= kNarrowM && std::max(rows, cols) <= kNarrowK; }
static int64_t up64(int64_t n) { return (n + 63) / 64 * 64; }
static size_t narrow_bytes(int64_t rows, int64_t cols) { return 2 * size_t(kNarrowM) * size_t(up64(std::max(rows, cols))) * 4; }

// all narrow ones of a list; their X lie one behind the other at ws
static hgnn_status orth_narrow(const char* who, int32_t count, const hgnn_grad* grads, int32_t steps, const float* coef, const float* scales, char* ws, hipStream_t s) {
  static uint64_t told = 0;
  constexpr int kBytes = (2 * kNarrowRing + 6) * kNarrowTile;
  for (int i = 0; i < count;) {
    NarrowArgs a{};
    int64_t blocks = 0;
    for (; i < count && a.count < kNarrowMany; ++i) {
      const hgnn_grad& g = grads[i];
      if (g.rows == 0 || g.cols == 0 || !is_narrow(g.rows, g.cols)) continue;
      NarrowMatrix& n = a.m[a.count++];
      n.m = OrthMatrix{g.grad, g.out ? g.out : const_cast<void*>(g.grad), g.rows, g.cols, g.ld, g.out ? g.ld_out : g.ld, int(g.type), int(g.out ? g.out_type : g.type)};
      n.flip = g.rows > g.cols, n.k = int32_t(up64(std::max(g.rows, g.cols))), n.scale = scales ? scales[i] : 1.f, n.first = int32_t(blocks);
      blocks += n.k / 64;
      n.X = reinterpret_cast<half_t*>(ws), n.next = n.X + 2 * kNarrowM * int64_t(n.k);
      ws += narrow_bytes(g.rows, g.cols);
    }
    if (a.count == 0) break;
    if (steps == 0) {
      narrow_norms_kernel<<<unsigned(a.count), 1024, 0, s>>>(a);
      HGNN_LAUNCH_CHECK("narrow_norms_kernel");
      narrow_scale_kernel<<<unsigned(blocks), 1024, 0, s>>>(a);
      HGNN_LAUNCH_CHECK("narrow_scale_kernel");
      continue;
    }
    const hgnn_status st = product_lds(reinterpret_cast<const void*>(&narrow_step_kernel), kBytes, &told);
    if (st != HGNN_OK) return st;
    narrow_begin_kernel<<<unsigned(blocks), 1024, 0, s>>>(a);
    HGNN_LAUNCH_CHECK("narrow_begin_kernel");
    for (int k = 0; k < steps; ++k) {
      a.a = coef[3 * k], a.b = coef[3 * k + 1], a.c = coef[3 * k + 2], a.last = k + 1 == steps;
      narrow_step_kernel<<<unsigned(blocks), kNarrowWaves * kWave, kBytes, s>>>(a);
      HGNN_LAUNCH_CHECK("narrow_step_kernel");
      for (int j = 0; j < a.count; ++j) std::swap(a.m[j].X, a.m[j].next);
    }
  }
  return HGNN_OK;
}

template <bool PCOL, class Out>
static hgnn_status orth_product(const char* who, const Pairs& Q, const Pairs& P, int64_t nq, int64_t np, int64_t K, bool lower, const OrthSplit& split, float* part, const Out& out,
                                hipStream_t s) {
  ProductArgs a{};
  a.Q0 = a.Q1 = Q.at, a.ldq = Q.ld, a.P0 = a.P1 = P.at, a.ldp = P.ld, a.nq = nq, a.np = np, a.K = K, a.part = split.part, a.parts = split.parts, a.lower = lower;
  const auto go = [&](const auto& to) {
    if (split.tile == 64) return product<SplitSmall<PCOL>>(who, a, to, s);
    product_tiles<SplitMid<PCOL>>(a);
    return int64_t(a.tiles) * a.parts <= kOrthFull ? product<SplitDeep<PCOL>>(who, a, to, s) : product<SplitMid<PCOL>>(who, a, to, s);
  };
  const auto join = [&](int parts, int64_t from, int first) -> hgnn_status {
    sums_join_kernel<<<dim3(unsigned(ceil_div(nq - from, kJoinTile)), unsigned(ceil_div(np, kJoinTile))), kBlock, 0, s>>>(part, parts, from, nq, np, lower, first, out);
    HGNN_LAUNCH_CHECK("sums_join_kernel");
    return HGNN_OK;
  };
  if (split.parts == 1) {
    a.some = split.first;
    hgnn_status st = go(out);
    if (st != HGNN_OK || !split.rest) return st;
    a.first = split.first, a.some = split.rest, a.part = split.rest_part, a.parts = split.rest_parts;
    st = go(SumsPart{part, split.from, nq, np});
    return st == HGNN_OK ? join(split.rest_parts, split.from, split.first) : st;
  }
  const hgnn_status st = go(SumsPart{part, 0, nq, np});
  return st == HGNN_OK ? join(split.parts, 0, 0) : st;
}

static hgnn_status orth_matrix(const char* who, const hgnn_grad& g, int32_t steps, const float* coef, float scale, char* ws, hipStream_t s) {
  const OrthSizes z = orth_sizes(g.rows, g.cols);
  double* const squares = reinterpret_cast<double*>(ws);
  half_t* at = reinterpret_cast<half_t*>(ws + kNormParts * sizeof(double));
  const auto pairs = [&](int64_t q, int64_t p) {
    const Pairs r{at, 2 * p};
    at += 2 * q * p;
    return r;
  };
  Pairs X = pairs(z.m, z.k), next = pairs(z.m, z.k);
  const Pairs A = pairs(z.m, z.m), B = pairs(z.m, z.m);
  float* const part = reinterpret_cast<float*>(at);
  const OrthMatrix m{g.grad, g.out ? g.out : const_cast<void*>(g.grad), g.rows, g.cols, g.ld, g.out ? g.ld_out : g.ld, int(g.type), int(g.out ? g.out_type : g.type)};
  const unsigned parts = unsigned(std::min<int64_t>(kNormParts, ceil_div(g.rows * g.cols, 32 * kBlock)));
  orth_squares_kernel<<<parts, kBlock, 0, s>>>(m, squares);
  HGNN_LAUNCH_CHECK("orth_squares_kernel");
  orth_begin_kernel<<<dim3(unsigned(ceil_div(z.k, kTurn)), unsigned(ceil_div(z.m, kTurn))), kBlock, 0, s>>>(m, z.flip, squares, int(parts), X, z.m, z.k, steps == 0, scale);
  HGNN_LAUNCH_CHECK("orth_begin_kernel");
  for (int i = 0; i < steps; ++i) {
    const float a = coef[3 * i], b = coef[3 * i + 1], c = coef[3 * i + 2];
    hgnn_status st = orth_product<false>(who, X, X, z.m, z.m, z.k, true, z.gram, part, GramOut{c == 0.f ? B : A, (c == 0.f ? b : 1.f) * (kA / (kX * kX)), z.gram.tile}, s);
    if (st == HGNN_OK && c != 0.f) st = orth_product<false>(who, A, A, z.m, z.m, z.m, true, z.square, part, SquareOut{B, A, b, c / kA, z.square.tile}, s);
    if (st != HGNN_OK) return st;
    if (i + 1 < steps) st = orth_product<true>(who, B, X, z.m, z.k, z.m, false, z.step, part, StepOut{next, X, a}, s);
    else
      st = orth_product<true>(who, B, X, z.m, z.k, z.m, false, z.step, part,
                              LastOut{X, X, a, scale / kX, m.out, m.ldo, std::min(g.rows, g.cols), std::max(g.rows, g.cols), m.out_type, z.flip}, s);
    if (st != HGNN_OK) return st;
    std::swap(X, next);
  }
  return HGNN_OK;
}

// The largest of |f| on [0, t] for f = t (b + c t)
static double largest_square(double b, double c, double t) {
  double most = std::fabs(t * (b + c * t));
  if (c != 0.) {
    const double v = -b / (2 * c);
    if (v > 0. && v < t) most = std::max(most, std::fabs(v * (b + c * v)));
  }
  return most;
}
// ... and of |s (a + b s^2 + c s^4)| on [0, s]
static double largest_value(double a, double b, double c, double s) {
  const auto f = [&](double v) { return std::fabs(v * (a + b * v * v + c * v * v * v * v)); };
  double most = f(s);
  const auto look = [&](double t) {  // a place where the slope a + 3 b t + 5 c t^2 is 0, t = s^2
    if (t > 0. && t < s * s) most = std::max(most, f(std::sqrt(t)));
  };
  if (c != 0.) {
    const double d = 9 * b * b - 20 * a * c;
    if (d >= 0.) look((-3 * b + std::sqrt(d)) / (10 * c)), look((-3 * b - std::sqrt(d)) / (10 * c));
  } else if (b != 0.) {
    look(-a / (3 * b));
  }
  return most;
}

static hgnn_status check_matrices(const char* who, int32_t count, const hgnn_grad* g) {
  HGNN_REQUIRE(count >= 0 && (g || count == 0), HGNN_EINVAL, "%s: count = %d, grads %s", who, count, g ? "given" : "NULL");
  for (int i = 0; i < count; ++i) {
    const hgnn_grad& t = g[i];
    HGNN_REQUIRE(t.rows >= 0 && t.cols >= 0, HGNN_EINVAL, "%s: matrix %d: %lld x %lld", who, i, static_cast<long long>(t.rows), static_cast<long long>(t.cols));
    HGNN_REQUIRE(known_type(t.type) && (!t.out || known_type(t.out_type)), HGNN_EINVAL, "%s: matrix %d: unknown type %d or %d", who, i, int(t.type), int(t.out_type));
    HGNN_REQUIRE(t.ld >= t.cols && (!t.out || t.ld_out >= t.cols), HGNN_EINVAL, "%s: matrix %d: leading dimension smaller than the row", who, i);
    HGNN_REQUIRE(t.rows <= 65536 && t.cols <= 65536, HGNN_EUNSUPPORTED, "%s: matrix %d: a side above 65536", who, i);
    if (t.rows == 0 || t.cols == 0) continue;
    HGNN_REQUIRE(t.grad && aligned_to_type(t.grad, t.type), HGNN_EINVAL, "%s: matrix %d: NULL, or not aligned to its type", who, i);
    if (!t.out) continue;
    HGNN_REQUIRE(aligned_to_type(t.out, t.out_type), HGNN_EINVAL, "%s: matrix %d: an output that is not aligned to its type", who, i);
    HGNN_REQUIRE(t.out != t.grad || (t.type == t.out_type && t.ld == t.ld_out), HGNN_EINVAL, "%s: matrix %d: in place as another type or with another leading dimension", who, i);
  }
  return check_outputs(who, count, g);
}

}  // namespace hgnn

using namespace hgnn;

extern "C" {

size_t hgnn_orthogonalize_workspace(int32_t count, const hgnn_grad* grads) {
  size_t most = 0, narrow = 0;
  for (int i = 0; grads && i < count; ++i) {
    const hgnn_grad& g = grads[i];
    if (g.rows < 0 || g.cols < 0 || g.rows > 65536 || g.cols > 65536) return 0;
    if (g.rows == 0 || g.cols == 0) continue;
    if (is_narrow(g.rows, g.cols)) narrow += narrow_bytes(g.rows, g.cols);
    else most = std::max(most, orth_sizes(g.rows, g.cols).bytes);
  }
  return std::max(narrow, most);  // the narrow ones are done before the others begin
}

hgnn_status hgnn_orthogonalize(int32_t count, const hgnn_grad* grads, int32_t steps, const float* coef, const float* scales, void* workspace, size_t workspace_bytes,
                               void* stream) {
  clear_error();
  const char* who = "hgnn_orthogonalize";
  hgnn_status st = check_matrices(who, count, grads);
  if (st != HGNN_OK) return st;
  HGNN_REQUIRE(steps >= 0 && steps <= 64 && (steps == 0 || coef), HGNN_EINVAL, "%s: steps = %d, coef %s", who, steps, coef ? "given" : "NULL");
  double s = 1.;
  for (int i = 0; i < steps; ++i) {
    const double a = coef[3 * i], b = coef[3 * i + 1], c = coef[3 * i + 2];
    HGNN_REQUIRE(std::isfinite(a) && std::isfinite(b) && std::isfinite(c), HGNN_EINVAL, "%s: coefficients of step %d that are not finite", who, i);
    HGNN_REQUIRE(largest_square(b, c, s * s) <= 64., HGNN_EINVAL, "%s: step %d: b A + c A A may pass 64", who, i);
    s = largest_value(a, b, c, s);
    HGNN_REQUIRE(s <= 8., HGNN_EINVAL, "%s: step %d: singular values may pass 8", who, i);
    s *= 1. + 1e-5;  // what roundings may add
  }
  for (int i = 0; scales && i < count; ++i) HGNN_REQUIRE(std::isfinite(scales[i]), HGNN_EINVAL, "%s: scales[%d] = %g", who, i, double(scales[i]));
  const size_t need = hgnn_orthogonalize_workspace(count, grads);
  HGNN_REQUIRE(need == 0 || (workspace && workspace_bytes >= need && aligned16(workspace)), HGNN_EINVAL,
               "%s: workspace of %zu bytes, needs %zu aligned to 16 (hgnn_orthogonalize_workspace)", who, workspace_bytes, need);
  st = orth_narrow(who, count, grads, steps, coef, scales, static_cast<char*>(workspace), static_cast<hipStream_t>(stream));
  for (int i = 0; i < count && st == HGNN_OK; ++i)
    if (grads[i].rows > 0 && grads[i].cols > 0 && !is_narrow(grads[i].rows, grads[i].cols))
      st = orth_matrix(who, grads[i], steps, coef, scales ? scales[i] : 1.f, static_cast<char*>(workspace), static_cast<hipStream_t>(stream));
  return st;
}

}  // extern "C"
