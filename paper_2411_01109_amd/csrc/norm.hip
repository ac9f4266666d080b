// The norms around a block of a network, with the gate of its branch and the residual, in one pass, and the gradients of all of that in another:
//   b = N1(Y),  H = alpha R + g b,  Z = N2(H),   N(x) = (x - mean(x)) r w + c,  r = 1 / sqrt(mean((x - mean(x))^2) + eps)   (mean(x) = 0 without centring)
// and with u = d w, xh = (x - mean) r, the gradient through a norm
//   N^T(d) = r (u - xh mean(u xh) - [centred] mean(u)),   dw = sum_rows d xh,   dc = sum_rows d.
// A row stays in registers from its load to its stores, so every tensor crosses the memory once, which is what bounds both kernels; sums over a row and all
// that is formed from them are fp32, the variance is formed from the differences to the mean.  The gradients recompute the statistics from the rows that they
// read in any case: two more reductions over lanes, no array of statistics that a caller could hand over stale.
// 2.4 M x 128 in fp16 with both norms and a gate, one MI355X, calls in a row: forward 2.46 GB in 468 us (5.2 TB/s, a large copy's rate), gradients 3.69 GB in 737 (5.0);
// of an fp32 stream 718 (3.69 GB, 5.1) and 1219 (5.53 GB, 4.5); 99 991 x 333 of an fp32 stream with a gate of every element, gradients, 742 MB in 183 (4.1).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "rows.h"

namespace hgnn {

struct BlockArgs {
  int64_t n;
  int F;
  int post, pre;  // hgnn_norm_kind
  float alpha, eps;
  const float *post_w, *post_b, *gate, *pre_w, *pre_b;
  const half_t* gate_rows;
  int64_t ld_gate;
  const void* R;
  int64_t ldr;
  const half_t* Y;
  int64_t ldy;
  void* H;  // the forward's output, the gradients' input
  int64_t ldh;
  half_t* Z;
  int64_t ldz;
};
enum { kPreW = 0, kPreB, kGate, kPostW, kPostB, kVectors };
struct BlockGradArgs : BlockArgs {
  const void* dH;
  int64_t lddh;
  const half_t* dZ;
  int64_t lddz;
  void* dR;
  int64_t lddr;
  half_t* dY;
  int64_t lddy;
  half_t* dgate_rows;
  int64_t ldd_gate;
  int past;     // 1: dR, 2: dY go past the caches
  int vectors;  // kPreW | ...: which sums over rows are wanted
  float* part;  // [gridDim.x][kVectors][pitch]
  int pitch;
  float* out[kVectors];  // where the sums of a single workgroup go
};

// ---- sums over the lanes of a row: L lanes of a wave, or W waves
__device__ __forceinline__ float lanes_sum(float v, int L) {
  if (L >= 2) v = dpp_add<0xB1>(v);
  if (L >= 4) v = dpp_add<0x4E>(v);
  if (L >= 8) v = dpp_add<0x141>(v);
  if (L >= 16) v = dpp_add<0x140>(v);
  typedef unsigned uint2_t __attribute__((ext_vector_type(2)));
  if (L >= 32) {
    const uint2_t r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if (L >= 64) {
    const uint2_t r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}

// Rows of L lanes (W = 1), or of W waves, eight elements a lane.
template <int L_, int W_>
struct RowShape {
  static constexpr int L = L_, W = W_;
  static constexpr int kRows = W > 1 ? 1 : kBlock / L;       // rows of a workgroup at a time
  static constexpr int kThreads = W > 1 ? W * kWave : kBlock;
  static constexpr int kLanes = W > 1 ? W * kWave : L;       // of a row
  static constexpr bool kKeep = W <= 4;                      // weights stay in registers over the rows of a workgroup
  __device__ static int lane() { return threadIdx.x % kLanes; }
  __device__ static int row() { return W > 1 ? 0 : threadIdx.x / L; }
  // of both at once: where the row is several waves', one turn through LDS
  __device__ static void sum(float& a, float& b, float* lds) {
    a = lanes_sum(a, W > 1 ? kWave : L), b = lanes_sum(b, W > 1 ? kWave : L);
    if constexpr (W > 1) {
      __syncthreads();  // what the turn before left has been read
      if (threadIdx.x % kWave == 0) lds[2 * (threadIdx.x / kWave)] = a, lds[2 * (threadIdx.x / kWave) + 1] = b;
      __syncthreads();
      a = 0.f, b = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) a += lds[2 * w], b += lds[2 * w + 1];
    }
  }
  __device__ static float sum(float a, float* lds) {
    float none = 0.f;
    if constexpr (W > 1) sum(a, none, lds);
    else a = lanes_sum(a, L);
    return a;
  }
};

struct Eight {
  float v[8];
};

// columns of the lane: [col, col + 8), `left` of them in the row
template <class S>
__device__ __forceinline__ int col_of() { return 8 * S::lane(); }

// Eight elements of a row as they are in memory, `left` of them the row's; zeros behind the row and for rows that do not exist, which then stay zeros through all that
// follows and add nothing anywhere.  after(): the elements from here to the tensor's end, behind which nothing is read.
template <class T, class After>
__device__ __forceinline__ RawPiece<T> fetch_eight(const T* at, int left, After&& after) {
  RawPiece<T> x;
  x.v = 0;
  if (left >= 8) x = load_raw(at);
  else if (left > 0) x = load_raw(at, left, after());  // with what is behind the row: eight_of takes that off, once the piece is there
  return x;
}
// a lane's place in a tensor, which moves with the rows that its workgroup takes
template <class T>
struct Place {
  T* at;
  int64_t ld, step;
  __device__ __forceinline__ Place(const void* base, int64_t ld_, int64_t row, int64_t rows, int col)
      : at(static_cast<T*>(const_cast<void*>(base)) + (base ? row * ld_ + col : 0)), ld(ld_), step(base ? rows * ld_ : 0) {}
  __device__ __forceinline__ void move() { at += step; }
  __device__ __forceinline__ RawPiece<T> fetch(int64_t row, int64_t n, int left) const {
    return fetch_eight(at, row < n ? left : 0, [&] { return (n - 1 - row) * ld + left; });
  }
};
template <class T>
__device__ __forceinline__ Eight eight_of(const RawPiece<T>& x, int left) {
  Eight r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.v[i] = float(x.v[i]);
  if (left > 0 && left < 8) {
#pragma unroll
    for (int i = 1; i < 8; ++i) r.v[i] = i < left ? r.v[i] : 0.f;
  }
  return r;
}
// x - v inside the row; what is behind it stays zero
__device__ __forceinline__ void less(Eight& x, float v, int left) {
  v = left > 0 ? v : 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) x.v[i] -= v;
  if (left > 0 && left < 8) {
#pragma unroll
    for (int i = 1; i < 8; ++i) x.v[i] = i < left ? x.v[i] : 0.f;
  }
}
// past: whole lines past the caches (kPastBytes)
template <class T>
__device__ __forceinline__ void store_eight(T* at, int left, const Eight& x, bool past = false) {
  if (left <= 0) return;
  if (past) {  // uniform; F is a multiple of eight
    if constexpr (sizeof(T) == 2) {
      half8_t h;
#pragma unroll
      for (int i = 0; i < 8; ++i) h[i] = half_t(x.v[i]);
      __builtin_nontemporal_store(h, reinterpret_cast<half8_t*>(at));
    } else {
      __builtin_nontemporal_store(float4_t{x.v[0], x.v[1], x.v[2], x.v[3]}, reinterpret_cast<float4_t*>(at));
      __builtin_nontemporal_store(float4_t{x.v[4], x.v[5], x.v[6], x.v[7]}, reinterpret_cast<float4_t*>(at + 4));
    }
    return;
  }
  store_piece(at, left, Piece{{x.v[0], x.v[1], x.v[2], x.v[3], x.v[4], x.v[5], x.v[6], x.v[7]}});
}
__device__ __forceinline__ Eight weights_at(const float* w, int col, int F, float otherwise) {
  if (w) return eight_of(fetch_eight(w + col, F - col, [&] { return int64_t(F - col); }), F - col);
  Eight r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.v[i] = otherwise;
  return r;
}

// (x - mean) r in the place of x, zeros behind the row; returns r
template <class S>
__device__ __forceinline__ float normed(Eight& x, int kind, int F, float eps, float* lds) {
  const float inv = 1.f / float(F);
  if (kind == HGNN_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += x.v[i];
    less(x, S::sum(s, lds) * inv, F - col_of<S>());
  }
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) q = fmaf(x.v[i], x.v[i], q);
  const float r = __builtin_amdgcn_rsqf(S::sum(q, lds) * inv + eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) x.v[i] *= r;
  return r;
}

// to + N^T(d) in the place of `to`: what comes back through a norm whose output was xh w + c
template <class S>
__device__ __forceinline__ void through(Eight& to, Eight& d, const Eight& xh, const Eight& w, float r, int kind, int F, float* lds) {
  float su = 0.f, sx = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    d.v[i] *= w.v[i];
    su += d.v[i];
    sx = fmaf(d.v[i], xh.v[i], sx);
  }
  if (kind == HGNN_NORM_LAYER) S::sum(su, sx, lds);
  else sx = S::sum(sx, lds);
  sx *= r / float(F), su *= r / float(F);
  if (kind == HGNN_NORM_LAYER) less(to, su, F - col_of<S>());
#pragma unroll
  for (int i = 0; i < 8; ++i) to.v[i] = fmaf(d.v[i], r, fmaf(-xh.v[i], sx, to.v[i]));
}

template <class T, int L, int W>
__global__ __launch_bounds__(W > 1 ? W * kWave : kBlock) void block_norm_kernel(BlockArgs a) {
  typedef RowShape<L, W> S;
  __shared__ float lds[2 * W];
  Eight post_w, post_b, gate, pre_w, pre_b;
  const int col = col_of<S>(), left = a.F - col;
  const auto weights = [&]() __attribute__((always_inline)) {
    post_w = weights_at(a.post_w, col, a.F, 1.f), post_b = weights_at(a.post_b, col, a.F, 0.f), gate = weights_at(a.gate, col, a.F, 1.f);
    pre_w = weights_at(a.pre_w, col, a.F, 1.f), pre_b = weights_at(a.pre_b, col, a.F, 0.f);
  };
  if (S::kKeep) weights();
  // (asking for the next rows ahead, as the gradients do, costs registers and with them waves: 2.4 M x 128 512 -> 567 us)
  const int64_t first = int64_t(blockIdx.x) * S::kRows + S::row(), stride = int64_t(gridDim.x) * S::kRows;
  Place<half_t> Y(a.Y, a.ldy, first, stride, col), G(a.gate_rows, a.ld_gate, first, stride, col), Z(a.Z, a.ldz, first, stride, col);
  Place<T> R(a.R, a.ldr, first, stride, col), H(a.H, a.ldh, first, stride, col);
  for (int64_t row = first; row - S::row() < a.n; row += stride) {  // all waves alike: the sums meet
    if (!S::kKeep) weights();
    const int mine = row < a.n ? left : 0;
    Eight b = {}, h = {};
    if (a.Y) b = eight_of(Y.fetch(row, a.n, left), left);
    if (a.R) h = eight_of(R.fetch(row, a.n, left), left);
    if (a.gate_rows) gate = eight_of(G.fetch(row, a.n, left), left);
    if (a.post != HGNN_NORM_NONE) {
      normed<S>(b, a.post, a.F, a.eps, lds);
#pragma unroll
      for (int i = 0; i < 8; ++i) b.v[i] = fmaf(b.v[i], post_w.v[i], post_b.v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) h.v[i] = float(T(fmaf(gate.v[i], b.v[i], a.alpha * h.v[i])));  // as it is stored
    if (a.H) store_eight(H.at, mine, h);
    if (a.pre != HGNN_NORM_NONE) {
      normed<S>(h, a.pre, a.F, a.eps, lds);
#pragma unroll
      for (int i = 0; i < 8; ++i) h.v[i] = fmaf(h.v[i], pre_w.v[i], pre_b.v[i]);
      store_eight(Z.at, mine, h);
    }
    Y.move(), R.move(), G.move(), H.move(), Z.move();
  }
}

// Sums over rows: a lane keeps those of its columns over all rows of its workgroup, the row groups of the workgroup are added in LDS in order, and the
// workgroup leaves one partial result, which block_sums_kernel adds in order: no atomics, the same bits on every run.
template <class T, int L, int W>
__global__ __launch_bounds__(W > 1 ? W * kWave : kBlock) void block_norm_grad_kernel(BlockGradArgs a) {
  typedef RowShape<L, W> S;
  __shared__ float lds[2 * W];
  __shared__ float sums[S::kRows > 1 ? S::kThreads * 9 : 1];
  Eight gate, total[kVectors] = {};
  const int col = col_of<S>(), left = a.F - col;
  // Weights stand in LDS: as registers of every lane they would cost a wave of three (153 registers, 2.4 M x 128 911 us).
  enum { kAtPreW, kAtPostW, kAtPostB, kAtGate, kWeights };
  __shared__ __align__(16) float s_weights[kWeights][S::kLanes * 8];
  if (S::row() == 0) {
    *reinterpret_cast<Eight*>(&s_weights[kAtPreW][col]) = weights_at(a.pre_w, col, a.F, 1.f);
    *reinterpret_cast<Eight*>(&s_weights[kAtPostW][col]) = weights_at(a.post_w, col, a.F, 1.f);
    *reinterpret_cast<Eight*>(&s_weights[kAtPostB][col]) = weights_at(a.post_b, col, a.F, 0.f);
    *reinterpret_cast<Eight*>(&s_weights[kAtGate][col]) = weights_at(a.gate, col, a.F, 1.f);
  }
  __syncthreads();
  const auto weight = [&](int k) __attribute__((always_inline)) {
    const float4_t* const at = reinterpret_cast<const float4_t*>(&s_weights[k][col]);
    const float4_t lo = at[0], hi = at[1];
    return Eight{{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}};
  };
  const int64_t first = int64_t(blockIdx.x) * S::kRows + S::row(), stride = int64_t(gridDim.x) * S::kRows;
  const bool pre = a.pre != HGNN_NORM_NONE, post = a.post != HGNN_NORM_NONE;
  struct {
    RawPiece<half_t> dZ, Y, gate;
    RawPiece<T> dH, H;
  } next = {};
  Place<T> in_dH(a.dH, a.lddh, first, stride, col), in_H(a.H, a.ldh, first, stride, col), out_R(a.dR, a.lddr, first, stride, col);
  Place<half_t> in_dZ(a.dZ, a.lddz, first, stride, col), in_Y(a.Y, a.ldy, first, stride, col), in_gate(a.gate_rows, a.ld_gate, first, stride, col),
      out_Y(a.dY, a.lddy, first, stride, col), out_gate(a.dgate_rows, a.ldd_gate, first, stride, col);
  const auto fetch = [&](int64_t row) __attribute__((always_inline)) {
    if (a.dH) next.dH = in_dH.fetch(row, a.n, left);
    if (pre) next.H = in_H.fetch(row, a.n, left), next.dZ = in_dZ.fetch(row, a.n, left);
    if (a.Y) next.Y = in_Y.fetch(row, a.n, left);
    if (a.gate_rows) next.gate = in_gate.fetch(row, a.n, left);
    in_dH.move(), in_H.move(), in_dZ.move(), in_Y.move(), in_gate.move();
  };
  constexpr bool kAhead = W <= 8;  // the next rows are on their way while these are worked on (where there are registers for it)
  if (kAhead) fetch(first);
  for (int64_t row = first; row - S::row() < a.n; row += stride) {
    asm volatile("" ::: "memory");  // weights are read again, not kept
    if (!kAhead) fetch(row);
    const int mine = row < a.n ? left : 0;
    Eight e = eight_of(next.dH, left), h = eight_of(next.H, left), d = eight_of(next.dZ, left), b = eight_of(next.Y, left);
    if (a.gate_rows) gate = eight_of(next.gate, left);
    if (kAhead && row - S::row() + stride < a.n) fetch(row + stride);
    if (pre) {
      const float r = normed<S>(h, a.pre, a.F, a.eps, lds);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        total[kPreW].v[i] = fmaf(d.v[i], h.v[i], total[kPreW].v[i]);
        total[kPreB].v[i] += d.v[i];
      }
      through<S>(e, d, h, weight(kAtPreW), r, a.pre, a.F, lds);
    }
    if (a.dR) {
      if (a.alpha == 1.f) {
        store_eight(out_R.at, mine, e, a.past & 1);
      } else {
        Eight out;
#pragma unroll
        for (int i = 0; i < 8; ++i) out.v[i] = a.alpha * e.v[i];
        store_eight(out_R.at, mine, out, a.past & 1);
      }
      out_R.move();
    }
    if (!a.dY && !a.dgate_rows && !(a.vectors & (1 << kGate | 1 << kPostW | 1 << kPostB))) continue;
    float r = 1.f;
    if (post) r = normed<S>(b, a.post, a.F, a.eps, lds);  // b: xh
    if (a.gate || a.gate_rows) {
      const Eight w = weight(kAtPostW), c = weight(kAtPostB);
      if (!a.gate_rows) gate = weight(kAtGate);
      Eight g;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        g.v[i] = e.v[i] * (post ? fmaf(b.v[i], w.v[i], c.v[i]) : b.v[i]);
        total[kGate].v[i] += g.v[i];
        e.v[i] *= gate.v[i];
      }
      if (a.dgate_rows) store_eight(out_gate.at, mine, g), out_gate.move();
    }
    if (post) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        total[kPostW].v[i] = fmaf(e.v[i], b.v[i], total[kPostW].v[i]);
        total[kPostB].v[i] += e.v[i];
      }
      Eight y = {};
      through<S>(y, e, b, weight(kAtPostW), r, a.post, a.F, lds);
      e = y;
    }
    if (a.dY) store_eight(out_Y.at, mine, e, a.past & 2), out_Y.move();
  }
  const auto part = [&](int k) { return gridDim.x == 1 ? a.out[k] : a.part + (int64_t(blockIdx.x) * kVectors + k) * a.pitch; };
#pragma unroll
  for (int k = 0; k < kVectors; ++k) {
    if (!(a.vectors & (1 << k))) continue;  // uniform
    if constexpr (S::kRows > 1) {  // lanes of a row, groups of rows
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) sums[threadIdx.x * 9 + i] = total[k].v[i];
      __syncthreads();
      for (int c = threadIdx.x; c < 8 * L; c += S::kThreads) {
        float s = 0.f;
        for (int g = 0; g < S::kRows; ++g) s += sums[(g * L + c / 8) * 9 + c % 8];
        if (c < a.F) part(k)[c] = s;
      }
    } else {
      store_eight(part(k) + col, left, total[k]);
    }
  }
}

struct BlockSumsArgs {
  const float* part;
  int parts, pitch, F;
  float* out[kVectors];
};
constexpr int kSumCols = 64, kSumRows = 16;
__global__ __launch_bounds__(kSumCols* kSumRows) void block_sums_kernel(BlockSumsArgs a) {
  __shared__ float lds[kSumRows][kSumCols];
  const int k = blockIdx.y, x = threadIdx.x % kSumCols, y = threadIdx.x / kSumCols, col = blockIdx.x * kSumCols + x;
  float* out = nullptr;
#pragma unroll
  for (int j = 0; j < kVectors; ++j) out = j == k ? a.out[j] : out;
  if (!out) return;  // uniform
  float s = 0.f;
  if (col < a.F) {
    const float* const in = a.part + int64_t(k) * a.pitch + col;
    const int64_t stride = int64_t(kVectors) * a.pitch;
    int j = y;
    constexpr int U = 16;  // on their way at a time
    for (; j < a.parts; j += U * kSumRows) {
      float v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = j + u * kSumRows < a.parts ? in[(j + u * kSumRows) * stride] : 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) s += v[u];
    }
  }
  lds[y][x] = s;
  __syncthreads();
  if (y != 0 || col >= a.F) return;
  s = 0.f;
#pragma unroll
  for (int j = 0; j < kSumRows; ++j) s += lds[j][x];
  out[col] = s;
}

constexpr int kMostNormed = 8192;

// The shape of a row of F elements: a piece of eight elements a lane, up to 512 elements of a wave's lanes, then of as many waves as it takes.
template <class Call>
static hgnn_status with_shape(int F, Call&& call) {
  const int lanes = pow2_at_least((F + 7) / 8);
  switch (lanes) {
    case 1: return call(RowShape<1, 1>());
    case 2: return call(RowShape<2, 1>());
    case 4: return call(RowShape<4, 1>());
    case 8: return call(RowShape<8, 1>());
    case 16: return call(RowShape<16, 1>());
    case 32: return call(RowShape<32, 1>());
    case 64: return call(RowShape<64, 1>());
    case 128: return call(RowShape<64, 2>());
    case 256: return call(RowShape<64, 4>());
    case 512: return call(RowShape<64, 8>());
    default: return call(RowShape<64, 16>());
  }
}

// Workgroups that are resident at once where a SIMD holds so many waves of a kernel: with more, the last ones run by themselves (the gradients of 2.4 M x 128 by
// 1024 workgroups, 768 of them at once, 910 us).
constexpr int kUnits = 256;
template <class S>
static int64_t resident(int waves) {
  return kUnits * int64_t(std::max(1, waves * 4 * kWave / S::kThreads));
}
// ... of the gradients: each with rows enough that its partial sums (as many bytes as three rows or so) cost little, up to eight in a row where a row is a wave's or more;
// few rows are dealt out one by one, since their time is that of a chain of rows (72 rows of 4096 in fp32, eight in a row 37 us).
template <class S>
static int64_t grad_blocks(int64_t n, hgnn_type type) {
  const int64_t per = std::max<int64_t>(S::kRows, S::kLanes >= 64 ? std::min<int64_t>(8, ceil_div(n, kUnits)) : 1);
  return std::max<int64_t>(1, std::min(resident<S>(type == HGNN_F16 ? 3 : 2), ceil_div(n, per)));
}

// the partial sums of a call, by the type with more workgroups
static size_t grad_bytes(int64_t n, int32_t F) {
  if (n == 0) return 0;
  int64_t blocks = 0;
  with_shape(F, [&](auto shape) -> hgnn_status {
    blocks = grad_blocks<decltype(shape)>(n, HGNN_F16);
    return HGNN_OK;
  });
  return size_t(blocks) * kVectors * size_t((F + 7) / 8 * 8) * sizeof(float);
}

static hgnn_status check_block(const char* who, int64_t n, int32_t F, const hgnn_block* b, hgnn_type type, bool branch) {
  HGNN_REQUIRE(n >= 0 && F > 0, HGNN_EINVAL, "%s: n = %lld, F = %d", who, static_cast<long long>(n), F);
  HGNN_REQUIRE(b != nullptr, HGNN_EINVAL, "%s: block is NULL", who);
  HGNN_REQUIRE(known_type(type), HGNN_EINVAL, "%s: unknown type %d", who, int(type));
  const auto known = [](hgnn_norm_kind k) { return k == HGNN_NORM_NONE || k == HGNN_NORM_RMS || k == HGNN_NORM_LAYER; };
  HGNN_REQUIRE(known(b->post) && known(b->pre), HGNN_EINVAL, "%s: unknown norm %d or %d", who, int(b->post), int(b->pre));
  HGNN_REQUIRE(F <= kMostNormed && n <= (int64_t(1) << 40), HGNN_EUNSUPPORTED, "%s: F = %d above %d, or n = %lld above 2^40", who, F, kMostNormed, static_cast<long long>(n));
  HGNN_REQUIRE(std::isfinite(b->alpha) && b->eps >= 1.17549435e-38f && std::isfinite(b->eps), HGNN_EINVAL, "%s: alpha = %g, eps = %g", who, double(b->alpha), double(b->eps));
  HGNN_REQUIRE(b->post != HGNN_NORM_NONE || (!b->post_w && !b->post_b), HGNN_EINVAL, "%s: weights of a norm behind the branch that is none", who);
  HGNN_REQUIRE(b->pre != HGNN_NORM_NONE || (!b->pre_w && !b->pre_b), HGNN_EINVAL, "%s: weights of a norm of the sum that is none", who);
  HGNN_REQUIRE(!b->gate || !b->gate_rows, HGNN_EINVAL, "%s: gate and gate_rows exclude each other", who);
  HGNN_REQUIRE(!b->gate_rows || b->ld_gate >= F, HGNN_EINVAL, "%s: leading dimension of the gate smaller than F", who);
  HGNN_REQUIRE(branch || (b->post == HGNN_NORM_NONE && !b->gate && !b->gate_rows), HGNN_EINVAL, "%s: a norm or a gate of a branch that is not there", who);
  HGNN_REQUIRE(aligned_to_type(b->post_w, HGNN_F32) && aligned_to_type(b->post_b, HGNN_F32) && aligned_to_type(b->gate, HGNN_F32) && aligned_to_type(b->pre_w, HGNN_F32) &&
                   aligned_to_type(b->pre_b, HGNN_F32) && aligned_to_type(b->gate_rows, HGNN_F16),
               HGNN_EINVAL, "%s: an array that is not aligned to its type", who);
  return HGNN_OK;
}
// whether an output goes past the caches: large, and in whole lines
static bool block_past(double bytes, const void* p, int64_t F, int64_t ld, hgnn_type type) {
  const int64_t size = type == HGNN_F16 ? 2 : 4;
  return p && bytes >= kPastBytes && F * size % 128 == 0 && ld * size % 128 == 0 && (reinterpret_cast<uintptr_t>(p) & 127u) == 0;
}
static void block_args(BlockArgs& a, int64_t n, int32_t F, const hgnn_block* b) {
  a.n = n, a.F = F, a.post = b->post, a.pre = b->pre, a.alpha = b->alpha, a.eps = b->eps;
  a.post_w = b->post_w, a.post_b = b->post_b, a.gate = b->gate, a.pre_w = b->pre_w, a.pre_b = b->pre_b;
  a.gate_rows = reinterpret_cast<const half_t*>(b->gate_rows), a.ld_gate = b->ld_gate;
}

}  // namespace hgnn

using namespace hgnn;

extern "C" {

hgnn_status hgnn_residual_norm(int64_t n, int32_t F, const hgnn_block* block, hgnn_type type, const void* R, int64_t ldr, const hgnn_half* Y, int64_t ldy, void* H,
                               int64_t ldh, hgnn_half* Z, int64_t ldz, void* stream) {
  clear_error();
  const char* who = "hgnn_residual_norm";
  hgnn_status st = check_block(who, n, F, block, type, Y != nullptr || n == 0);
  if (st != HGNN_OK) return st;
  HGNN_REQUIRE((!R || ldr >= F) && (!Y || ldy >= F) && (!H || ldh >= F) && (!Z || ldz >= F), HGNN_EINVAL, "%s: leading dimension smaller than F", who);
  if (n == 0) return HGNN_OK;
  HGNN_REQUIRE(R || Y, HGNN_EINVAL, "%s: neither R nor Y is given", who);
  HGNN_REQUIRE((block->pre == HGNN_NORM_NONE) == (Z == nullptr) && (H || Z), HGNN_EINVAL, "%s: Z goes with a norm of the sum, and one of H and Z has to be there", who);
  HGNN_REQUIRE(aligned_to_type(R, type) && aligned_to_type(H, type) && aligned_to_type(Y, HGNN_F16) && aligned_to_type(Z, HGNN_F16), HGNN_EINVAL,
               "%s: an array that is not aligned to its type", who);
  HGNN_REQUIRE(!H || H != R || ldh == ldr, HGNN_EINVAL, "%s: in place with another leading dimension", who);
  BlockArgs a{};
  block_args(a, n, F, block);
  a.R = R, a.ldr = ldr, a.Y = reinterpret_cast<const half_t*>(Y), a.ldy = ldy, a.H = H, a.ldh = ldh, a.Z = reinterpret_cast<half_t*>(Z), a.ldz = ldz;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return with_shape(F, [&](auto shape) -> hgnn_status {
    typedef decltype(shape) S;
    const unsigned blocks = unsigned(std::min<int64_t>(ceil_div(n, S::kRows), resident<S>(S::kThreads > 512 ? 4 : 5)));
    if (type == HGNN_F16) block_norm_kernel<half_t, S::L, S::W><<<blocks, S::kThreads, 0, s>>>(a);
    else block_norm_kernel<float, S::L, S::W><<<blocks, S::kThreads, 0, s>>>(a);
    HGNN_LAUNCH_CHECK("block_norm_kernel");
    return HGNN_OK;
  });
}

size_t hgnn_residual_norm_grad_workspace(int64_t n, int32_t F) {
  if (n <= 0 || F <= 0 || F > kMostNormed) return 0;
  size_t most = grad_bytes(n, F);
  for (int64_t rows = kUnits; rows < n && rows <= 8 * kUnits; rows += kUnits) most = std::max(most, grad_bytes(rows, F));  // fewer rows may be dealt out to more workgroups
  return most;
}

hgnn_status hgnn_residual_norm_grad(int64_t n, int32_t F, const hgnn_block* block, hgnn_type type, const void* H, int64_t ldh, const hgnn_half* Y, int64_t ldy,
                                    const void* dH, int64_t lddh, const hgnn_half* dZ, int64_t lddz, const hgnn_block_grad* grads, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  clear_error();
  const char* who = "hgnn_residual_norm_grad";
  HGNN_REQUIRE(grads != nullptr, HGNN_EINVAL, "%s: grads is NULL", who);
  const hgnn_block_grad& g = *grads;
  hgnn_status st = check_block(who, n, F, block, type, true);
  if (st != HGNN_OK) return st;
  HGNN_REQUIRE((!H || ldh >= F) && (!Y || ldy >= F) && (!dH || lddh >= F) && (!dZ || lddz >= F) && (!g.dR || g.lddr >= F) && (!g.dY || g.lddy >= F) &&
                   (!g.dgate_rows || g.ldd_gate >= F),
               HGNN_EINVAL, "%s: leading dimension smaller than F", who);
  HGNN_REQUIRE((block->pre != HGNN_NORM_NONE) || (!dZ && !g.dpre_w && !g.dpre_b), HGNN_EINVAL, "%s: gradients of a norm of the sum that is none", who);
  HGNN_REQUIRE(block->post != HGNN_NORM_NONE || (!g.dpost_w && !g.dpost_b), HGNN_EINVAL, "%s: gradients of a norm behind the branch that is none", who);
  HGNN_REQUIRE((!g.dgate || block->gate) && (!g.dgate_rows || block->gate_rows), HGNN_EINVAL, "%s: the gradient of a gate that is none", who);
  HGNN_REQUIRE(aligned_to_type(H, type) && aligned_to_type(dH, type) && aligned_to_type(g.dR, type) && aligned_to_type(Y, HGNN_F16) && aligned_to_type(dZ, HGNN_F16) &&
                   aligned_to_type(g.dY, HGNN_F16) && aligned_to_type(g.dgate_rows, HGNN_F16) && aligned_to_type(g.dgate, HGNN_F32) && aligned_to_type(g.dpost_w, HGNN_F32) &&
                   aligned_to_type(g.dpost_b, HGNN_F32) && aligned_to_type(g.dpre_w, HGNN_F32) && aligned_to_type(g.dpre_b, HGNN_F32),
               HGNN_EINVAL, "%s: an array that is not aligned to its type", who);
  HGNN_REQUIRE(!g.dR || g.dR != dH || g.lddr == lddh, HGNN_EINVAL, "%s: in place with another leading dimension", who);
  const bool branch = g.dY || g.dgate || g.dgate_rows || g.dpost_w || g.dpost_b;
  // what the branch's gradients need of it
  const bool needs_Y = branch && (block->post != HGNN_NORM_NONE || block->gate || block->gate_rows);
  if (n > 0) {
    HGNN_REQUIRE(block->pre == HGNN_NORM_NONE ? dH != nullptr : (H && dZ), HGNN_EINVAL, "%s: NULL argument", who);
    HGNN_REQUIRE(!needs_Y || Y, HGNN_EINVAL, "%s: Y is NULL", who);
  }
  BlockGradArgs a{};
  block_args(a, n, F, block);
  float* const out[kVectors] = {g.dpre_w, g.dpre_b, g.dgate, g.dpost_w, g.dpost_b};
  for (int k = 0; k < kVectors; ++k) a.vectors |= out[k] ? 1 << k : 0, a.out[k] = out[k];
  const size_t need = grad_bytes(n, F);
  HGNN_REQUIRE(a.vectors == 0 || need == 0 || (workspace && workspace_bytes >= need && aligned16(workspace)), HGNN_EINVAL,
               "%s: workspace of %zu bytes, needs %zu aligned to 16 (hgnn_residual_norm_grad_workspace)", who, workspace_bytes, need);
  if (n == 0 && a.vectors == 0) return HGNN_OK;
  a.H = const_cast<void*>(H), a.ldh = ldh, a.Y = needs_Y ? reinterpret_cast<const half_t*>(Y) : nullptr, a.ldy = ldy;
  a.dH = dH, a.lddh = lddh, a.dZ = reinterpret_cast<const half_t*>(dZ), a.lddz = lddz;
  a.dR = g.dR, a.lddr = g.lddr, a.dY = reinterpret_cast<half_t*>(g.dY), a.lddy = g.lddy;
  a.dgate_rows = reinterpret_cast<half_t*>(g.dgate_rows), a.ldd_gate = g.ldd_gate;
  const double bytes = double(n) * F * ((g.dR ? (type == HGNN_F16 ? 2 : 4) : 0) + (g.dY ? 2 : 0));
  a.past = (block_past(bytes, g.dR, F, g.lddr, type) ? 1 : 0) | (block_past(bytes, g.dY, F, g.lddy, HGNN_F16) ? 2 : 0);
  a.part = static_cast<float*>(workspace), a.pitch = (F + 7) / 8 * 8;
  hipStream_t s = static_cast<hipStream_t>(stream);
  int64_t blocks = 0;  // no rows: sums of nothing
  if (n > 0) {
    st = with_shape(F, [&](auto shape) -> hgnn_status {
      typedef decltype(shape) S;
      blocks = grad_blocks<S>(n, type);
      if (type == HGNN_F16) block_norm_grad_kernel<half_t, S::L, S::W><<<unsigned(blocks), S::kThreads, 0, s>>>(a);
      else block_norm_grad_kernel<float, S::L, S::W><<<unsigned(blocks), S::kThreads, 0, s>>>(a);
      HGNN_LAUNCH_CHECK("block_norm_grad_kernel");
      return HGNN_OK;
    });
    if (st != HGNN_OK) return st;
  }
  if (a.vectors && blocks != 1) {
    BlockSumsArgs q{a.part, int(blocks), a.pitch, F, {out[0], out[1], out[2], out[3], out[4]}};
    block_sums_kernel<<<dim3(unsigned(ceil_div(F, kSumCols)), kVectors), kSumCols * kSumRows, 0, s>>>(q);
    HGNN_LAUNCH_CHECK("block_sums_kernel");
  }
  return HGNN_OK;
}

}  // extern "C"
