// The gated projection  Y = act(G) * U,  G = X Wg,  U = X Wu,  and its gradients
//   dG = dY U act'(G),  dU = dY act(G),  dX = dG Wg^T + dU Wu^T,  dWg = X^T dG,  dWu = X^T dU
// on the product kernel of product.h.  The forward forms both sums of an element in the same lane, so the activation and the product cost no pass of their own.
// The gradients form G and U once more (two of their six products) and leave dG and dU beside each other in the workspace, [n][2 Fp] in fp16: a rounding of
// 2^-11 of each value (2^-25 below fp16's normal numbers; beyond 65 504 infinite, and then no output is finite that it is a part of), as every vertex-level gradient of this
// library takes it; then dX is one product over both halves and (dWg, dWu) is one, too.  What is stored is off by 2.9e-4 of its norm, where dG and dU in more bits
// would leave the 2.1e-4 of its own rounding: two parts of each would be four products of the six twice.
// Where C has too few tiles for the chip the contraction is cut; the parts' fp32 sums go through the workspace and are added in their order.
#include <algorithm>
#include <cmath>

#include "product.h"

namespace hgnn {

// ---- activations
__device__ __forceinline__ float gate_sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * -1.44269504f)); }
// Phi of the normal distribution, with e = exp(-x^2 / 2), which its density needs as well: Phi(-|x|) = e R(t), t = 1 / (1 + 0.375 |x| / sqrt 2), R the
// polynomial of degree 9 without a constant whose relative distance from exp(x^2 / 2) Phi(-|x|) is smallest up to |x| = 13.4 (1.2e-8; a weighted least squares fit),
// beyond which e is 0.  Relative to Phi itself some 10 (1 + |x|) 2^-24, mostly of the exponent.  (erff and exp apart: 99 991 x 100 -> 200 59 us.)
__device__ __forceinline__ float gate_normal(float x, float& e) {
  const float a = __builtin_fabsf(x), t = __builtin_amdgcn_rcpf(fmaf(a, 0.26516504f, 1.f));
  e = __builtin_amdgcn_exp2f(x * x * -0.72134752f);
  float r = 3.084830754e-02f;
  r = fmaf(r, t, -1.440376937e-01f), r = fmaf(r, t, 2.169468850e-01f), r = fmaf(r, t, -1.155382022e-01f), r = fmaf(r, t, 1.374220550e-01f);
  r = fmaf(r, t, 6.051947922e-02f), r = fmaf(r, t, 1.027152091e-01f), r = fmaf(r, t, 1.053167507e-01f), r = fmaf(r, t, 1.058072075e-01f);
  r *= t * e;
  return x < 0.f ? r : 1.f - r;
}
// Four at a time behind one question about the kind, which is uniform: a question for each value keeps the four from running beside each other.
__device__ __forceinline__ float4_t gate_value(int act, const float4_t& x) {
  float4_t y;
#define HGNN_EACH(...) { _Pragma("unroll") for (int e = 0; e < 4; ++e) { __VA_ARGS__; } break; }
  switch (act) {
    case HGNN_SILU: HGNN_EACH(y[e] = x[e] * gate_sigmoid(x[e]))
    case HGNN_GELU: HGNN_EACH(float d; y[e] = x[e] * gate_normal(x[e], d))
    case HGNN_SIGMOID: HGNN_EACH(y[e] = gate_sigmoid(x[e]))
    default: HGNN_EACH(y[e] = x[e] > 0.f ? x[e] : x[e] == x[e] ? 0.f : x[e])
  }
  return y;
}
__device__ __forceinline__ void gate_both(int act, const float4_t& x, float4_t& value, float4_t& slope) {
  switch (act) {
    case HGNN_SILU: HGNN_EACH(const float p = gate_sigmoid(x[e]); value[e] = x[e] * p; slope[e] = p * (1.f + x[e] * (1.f - p)))
    case HGNN_GELU:
      HGNN_EACH(float d; const float phi = gate_normal(x[e], d); value[e] = x[e] * phi; slope[e] = fmaf(x[e] * 0.39894228f, d, phi))
    case HGNN_SIGMOID:  // exp(-|x|) / (1 + exp(-|x|))^2: p (1 - p) would lose its digits where p is near 1 (all of them from x = 17 on)
      HGNN_EACH(const float d = __builtin_amdgcn_exp2f(__builtin_fabsf(x[e]) * -1.44269504f), r = __builtin_amdgcn_rcpf(1.f + d); value[e] = x[e] < 0.f ? d * r : r;
                slope[e] = d * r * r)
    default: HGNN_EACH(value[e] = x[e] > 0.f ? x[e] : x[e] == x[e] ? 0.f : x[e]; slope[e] = x[e] > 0.f ? 1.f : 0.f)
  }
#undef HGNN_EACH
}

// the first `left` of four values (all of them where it is four or more), at 8-byte aligned places
__device__ __forceinline__ void store_four(half_t* p, int64_t left, const float4_t& v) {
  const half4_t h = {half_t(v[0]), half_t(v[1]), half_t(v[2]), half_t(v[3])};
  if (left >= 4) {
    *reinterpret_cast<half4_t*>(p) = h;
  } else {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < left) p[e] = h[e];
  }
}

// ---- what becomes of the two sums of an element
struct GatedOut {
  int act, F;
  half_t* Y;
  int64_t ldy;
  typedef ProductNothing Read;
  __device__ Read read(int64_t, int64_t) const { return {}; }
  template <bool WHOLE>
  __device__ void put(int64_t, int64_t q, int64_t p, const Read&, const float4_t& g, const float4_t& u) const {
    const float4_t y = gate_value(act, g) * u;
    store_four(Y + q * ldy + p, WHOLE ? 4 : F - p, y);
  }
};
struct GatedGradOut {
  int act;
  const half_t* dY;
  int64_t lddy;
  half_t* D;  // [n][2 Fp]
  int64_t Fp;
  typedef half4_t Read;
  __device__ Read read(int64_t q, int64_t p) const { return *reinterpret_cast<const half4_t*>(dY + q * lddy + p); }  // what is behind F reaches what is behind F
  template <bool WHOLE>
  __device__ void put(int64_t, int64_t q, int64_t p, const Read& dy, const float4_t& g, const float4_t& u) const {
    float4_t value, slope;
    gate_both(act, g, value, slope);
    const float4_t d = {float(dy[0]), float(dy[1]), float(dy[2]), float(dy[3])}, dg = d * u * slope, du = d * value;
    store_four(D + q * 2 * Fp + p, 4, dg);
    store_four(D + q * 2 * Fp + Fp + p, 4, du);
  }
};
struct GatedPart {  // [parts][n][2][Fp]
  float* part;
  int64_t n, Fp;
  typedef ProductNothing Read;
  __device__ Read read(int64_t, int64_t) const { return {}; }
  template <bool WHOLE>
  __device__ void put(int64_t k, int64_t q, int64_t p, const Read&, const float4_t& g, const float4_t& u) const {
    float* const at = part + ((k * n + q) * 2) * Fp + p;
    *reinterpret_cast<float4_t*>(at) = g;
    *reinterpret_cast<float4_t*>(at + Fp) = u;
  }
};
// The parts of four sums in order: a workgroup takes 64 fours and cuts the parts in four, so that enough loads are on their way.  (121 parts of 100 x 512 by a
// thread a four 13 us.)  N values, `apart` floats from each other; those of thread < 64 are the sums.
constexpr int kJoinWays = 4, kJoinFours = kBlock / kJoinWays;
template <int N>
__device__ __forceinline__ void join_parts(float4_t (&v)[N], const float* at, int64_t apart, int64_t stride, int parts, bool in) {
  __shared__ __align__(16) float4_t lds[kJoinWays][N][kJoinFours];
  const int x = threadIdx.x % kJoinFours, way = threadIdx.x / kJoinFours, per = (parts + kJoinWays - 1) / kJoinWays, from = way * per, to = min(parts, from + per);
#pragma unroll
  for (int k = 0; k < N; ++k) v[k] = float4_t{0.f, 0.f, 0.f, 0.f};
  if (in) {
#pragma unroll 8
    for (int p = from; p < to; ++p)
#pragma unroll
      for (int k = 0; k < N; ++k) v[k] += *reinterpret_cast<const float4_t*>(at + p * stride + k * apart);
  }
#pragma unroll
  for (int k = 0; k < N; ++k) lds[way][k][x] = v[k];
  __syncthreads();
  if (way) return;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int w = 1; w < kJoinWays; ++w) v[k] += lds[w][k][x];
}
template <class Out>
__global__ __launch_bounds__(kBlock) void gated_join_kernel(const float* part, int parts, int64_t n, int F, int64_t Fp, Out out) {
  const int64_t t = int64_t(blockIdx.x) * kJoinFours + threadIdx.x % kJoinFours, each = (F + 3) / 4, q = t / each, p = 4 * (t - q * each);
  float4_t v[2];
  join_parts(v, part + q * 2 * Fp + p, Fp, n * 2 * Fp, parts, q < n);
  if (q < n && threadIdx.x < kJoinFours) out.template put<false>(0, q, p, out.read(q, p), v[0], v[1]);
}

// ---- products into one fp16 matrix, or into two that are the halves of C's lines or of its items along a line
struct HalfOut {
  half_t *a, *b;
  int64_t ld;
  int64_t split_q, split_p;  // from there on b's; beyond C: none
  int64_t lines, cols;       // of either
  typedef ProductNothing Read;
  __device__ Read read(int64_t, int64_t) const { return {}; }
  template <bool WHOLE>
  __device__ void put(int64_t, int64_t q, int64_t p, const Read&, const float4_t& v) const {
    half_t* to = a;
    if (q >= split_q) to = b, q -= split_q;
    if (p >= split_p) to = b, p -= split_p;
    if (q < lines && p < cols) store_four(to + q * ld + p, cols - p, v);
  }
};
struct HalfPart {  // [parts][nq][pitch]
  float* part;
  int64_t nq, pitch;
  typedef ProductNothing Read;
  __device__ Read read(int64_t, int64_t) const { return {}; }
  template <bool WHOLE>
  __device__ void put(int64_t k, int64_t q, int64_t p, const Read&, const float4_t& v) const { *reinterpret_cast<float4_t*>(part + (k * nq + q) * pitch + p) = v; }
};
__global__ __launch_bounds__(kBlock) void half_join_kernel(const float* part, int parts, int64_t nq, int64_t pitch, HalfOut out) {
  const int64_t t = int64_t(blockIdx.x) * kJoinFours + threadIdx.x % kJoinFours, each = pitch / 4, q = t / each, p = 4 * (t - q * each);
  float4_t v[1];
  join_parts(v, part + q * pitch + p, 0, nq * pitch, parts, q < nq);
  if (q < nq && threadIdx.x < kJoinFours) out.put<false>(0, q, p, out.read(q, p), v[0]);
}
__global__ __launch_bounds__(kBlock) void half_zero_kernel(half_t* out, int64_t lines, int64_t cols, int64_t ld) {
  const int64_t t = int64_t(blockIdx.x) * kBlock + threadIdx.x, each = (cols + 3) / 4, q = t / each, p = 4 * (t - q * each);
  if (q < lines) store_four(out + q * ld + p, cols - p, float4_t{0.f, 0.f, 0.f, 0.f});
}

static int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// ---- shapes.  A product of few rows takes tiles of 64, one whose tiles of 256 x 256 fill the chip those, any other 128 x 128.
enum Size { kFew, kMid, kWide };
constexpr int kFull = 256;  // compute units
constexpr int kLong = 512;
template <ProductKind KIND, bool QCOL, bool PCOL, class Call>
static hgnn_status with_product(Size size, Call&& call) {
  constexpr int two = KIND == kTwo ? 2 : 1;  // two results: half as many items of P
  if (size == kFew) return call(ProductShape<2, 2, 2, 2, KIND, QCOL, PCOL, 3>());
  if (size == kMid) return call(ProductShape<2, 2, 4, 4 / two, KIND, QCOL, PCOL, 2>());
  return call(ProductShape<2, 4, 8, 4 / two, KIND, QCOL, PCOL, 2>());
}
struct Split {
  Size size;
  int parts;
  int64_t part;  // contraction steps of a part
  int most;      // parts that were asked for: no fewer, and no fewer for a longer contraction
};
// nq x np sums (`two`: a pair of each) over segments of K steps, which are cut alike.
static Split split_of(int64_t nq, int64_t np, int64_t K, bool two, int segments) {
  const auto tiles = [&](int64_t b) { return ceil_div(nq, b) * ceil_div(np, two ? b / 2 : b); };
  Split s;
  s.size = nq <= 64 || np <= (two ? 32 : 64) ? kFew : K >= kLong && tiles(256) >= kFull ? kWide : kMid;
  const int64_t t = s.size == kFew ? ceil_div(nq, 64) * ceil_div(np, 64) : tiles(s.size == kWide ? 256 : 128);
  // A launch of these takes 6 us and 0.6 for 64 steps, a join 4 to 6: parts of 512 steps at least, and none where half of the units have a tile (370 x 565 -> 1173, us:
  // the pairs by 57 tiles in five parts 14.6 and 6.1 for the join, X^T D in three 13.0 and 6.0; 9611 x 1402 -> 91, 152 tiles in two 18.5 and 5.4).
  const int64_t parts = 2 * t > kFull ? 1 : std::min(ceil_div(kFull, t), std::max<int64_t>(1, segments * K / 512));
  s.most = int(parts);
  s.part = std::max<int64_t>(64, up(ceil_div(K, std::max<int64_t>(parts, 1)), 64));
  s.parts = int(std::max<int64_t>(1, ceil_div(K, s.part)));
  return s;
}

// ---- many rows through a narrow weight (K up to 256): bound by the rows of X and Y, which the product kernel's workgroups, a tile and two steps each, do not stream
// (233 000 x 128 -> 256 96 us, here 45 with X and Y in the last-level cache and 60 from memory, 35 by the bytes at a copy's rate).  Eight waves keep their features of both weights in registers for all rows of the
// workgroup, 32 features for K <= 128, 16 beyond; a ninth brings X into a ring in LDS, 64 rows at a time, and is the only one that waits for loads to LDS, so that
// the other waves' stores are never waited for.  A barrier a tile hands it over and takes back the one before.  (Two
// workgroups of four waves and one do not fit a compute unit's registers: 65 -> 100 us.)  Features are dealt out such that a lane's 2 x 4 sums are eight consecutive ones.
constexpr int kRowsWaves = 8, kRowsTile = 64;
// From 16 384 rows on, and from 2048 on where the features are one workgroup's or C is large (the product kernel behind, us: 16 384 x 128 -> 512 11.5 and 12.4, -> 2048 29.0 and
// 39.5; 6000 x 128 -> 40 4.3 and 5.8, -> 512 7.5 and 7.3, -> 2048 14.7 and 17.7, -> 5461 30 and 43; 2000 x 256 -> 5461 25.3 and 24.6).
static bool is_rows(int64_t n, int64_t K, int64_t F) { return K <= 256 && (n >= 16384 || (n >= 2048 && (F <= 64 || n * F >= int64_t(1) << 23))); }
struct GatedRowsArgs {
  const half_t *X, *Wg, *Wu;
  int64_t ldx, ldw, n;
  int32_t K, F, chunks;  // of features: a workgroup takes number blockIdx.x % chunks
};
template <int KS_, int TP_, int WF_, bool PCOL_, int RING_>
struct GatedRowsShape {  // KS: 64 steps of the contraction, TP: 16 features of a wave, WF: waves beside each other along the features, the others take other rows of the tile
  static constexpr int KS = KS_, TP = TP_, WF = WF_, kRing = RING_, kFeatures = 16 * TP * WF, kStage = KS * kRowsTile * 128;
  static constexpr int kGroups = kRowsWaves / WF, kBlocks = kRowsTile / 16 / kGroups;  // of waves along the rows, of 16 rows of a wave
  static constexpr bool PCOL = PCOL_;
  static constexpr int kWeights = KS * 2 * kFeatures * 128;
  static constexpr int kLds = kWeights > RING_ * kStage ? kWeights : RING_ * kStage;
  static constexpr int kChunks = KS * kRowsTile / 8;  // kilobytes of a tile of X
  static constexpr int kThreads = (kRowsWaves + 1) * kWave;
  static_assert(kLds <= 160 * 1024 && (RING_ - 2) * kChunks < 64, "LDS, vmcnt");
};
// fragment u of a wave's 16 TP features, whose items are dealt out, from where product_loads put them
template <bool COL, int TP>
__device__ __forceinline__ half8_t gated_weight(const unsigned char* tile, int wave, int lane, int u, int h) {
  const int i = lane & 15, qq = lane >> 4;
  if (!COL) {
    const int item = 16 * TP * wave + (TP == 2 ? 8 * (i >> 2) + 4 * u + (i & 3) : i);
    return *reinterpret_cast<const half8_t*>(tile + item * 128 + ((4 * h + qq) ^ ((item & 15) >> 1)) * 16);
  }
  const int r = 8 * qq + (i >> 2), item = 16 * TP * wave + (TP == 2 ? 8 * (i & 3) + 4 * u : 4 * (i & 3));  // the first of four
  const unsigned char* const p = tile + (item >> 6) * 8192 + h * 4096 + r * 128 + (((item & 63) >> 3) ^ product_turn(r)) * 16 + (item & 4) * 2;
  const short4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t*)p);
  const short4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t*)(p + 512));
  return __builtin_bit_cast(half8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
template <class S, class Out>
__global__ __launch_bounds__(S::kThreads) void gated_rows_kernel(GatedRowsArgs a, Out out) {
  extern __shared__ __align__(1024) unsigned char lds[];
  constexpr int KS = S::KS, TP = S::TP;
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), i = lane & 15, qq = lane >> 4;
  const int chunk = blockIdx.x % a.chunks, first = blockIdx.x / a.chunks, stride = gridDim.x / a.chunks;
  const int64_t f0 = int64_t(chunk) * S::kFeatures;
  const int tiles = int((a.n + kRowsTile - 1) / kRowsTile);
  const uint32_t lds0 = uint32_t(uintptr_t((__attribute__((address_space(3))) unsigned char*)lds));
  const char* const zero = reinterpret_cast<const char*>(&g_product_zero);
  const auto meet = [] {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  half8_t weight[2][TP][2 * KS];
  const int wf = wave % S::WF, group = wave / S::WF;
  {  // both weights' features of the workgroup into LDS, and a wave's into its registers
    constexpr int kOperand = S::kFeatures * 128;  // 64 steps of one weight
    constexpr int N = (2 * S::kFeatures / 8 + kRowsWaves - 1) / kRowsWaves;
    static_assert(2 * S::kFeatures / 8 % kRowsWaves == 0, "kilobytes of a wave");
    if (wave < kRowsWaves) {
      ProductLoads<N, S::PCOL> l;
      product_loads<N, S::PCOL, false, kRowsWaves>(l, a.Wg, a.Wu, a.ldw, f0, a.F, 0, wave, lane, S::kFeatures / 8);
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int j = 0; j < N; ++j)
          load_to_lds(l.k[j] + 64 * s < a.K ? l.base[j] + s * l.inc + l.off[j] : zero, lds0 + s * 2 * kOperand + (wave + j * kRowsWaves) * 1024);
    }
    product_wait<0>();
    if (wave < kRowsWaves) {
#pragma unroll
      for (int o = 0; o < 2; ++o)
#pragma unroll
        for (int u = 0; u < TP; ++u)
#pragma unroll
          for (int h = 0; h < 2 * KS; ++h) {
            half8_t v = gated_weight<S::PCOL, TP>(lds + (h / 2) * 2 * kOperand + o * kOperand, wf, lane, u, h % 2);
            // what stands behind the contraction's end inside a piece is the caller's padding
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (!S::PCOL && 32 * h + 8 * qq + e >= a.K) v[e] = half_t(0);
            weight[o][u][h] = v;
          }
    }
    meet();
  }
  const int mine = first < tiles ? (tiles - 1 - first) / stride + 1 : 0;  // tiles of the workgroup
  if (wave == kRowsWaves) {
    const auto ask = [&](int t) __attribute__((always_inline)) {
      const int64_t row0 = (int64_t(first) + int64_t(t) * stride) * kRowsTile;
      const uint32_t to = lds0 + (t % S::kRing) * S::kStage;
#pragma unroll
      for (int c = 0; c < S::kChunks; ++c) {  // eight rows, 64 steps
        const int s = c / 8, r = 8 * (c % 8) + (lane >> 3), u = (lane & 7) ^ ((r & 15) >> 1), k = 64 * s + 8 * u;
        const char* const src = reinterpret_cast<const char*>(a.X + min(row0 + r, a.n - 1) * a.ldx + k);
        load_to_lds(k < a.K ? src : zero, to + c * 1024);
      }
    };
    int asked = 0;
    for (; asked < S::kRing - 1 && asked < mine; ++asked) ask(asked);
    for (int t = 0; t < mine; ++t) {
      const int behind = asked - 1 - t;
      if (S::kRing > 3 && behind >= 2) product_wait<(S::kRing > 3 ? 2 : 0) * S::kChunks>();
      else if (S::kRing > 2 && behind >= 1) product_wait<(S::kRing > 2 ? 1 : 0) * S::kChunks>();
      else product_wait<0>();
      if (asked < mine) ask(asked), ++asked;  // in the place of the tile before, which all waves have left
    }
    return;
  }
  const ProductReads<false, false, kRowsTile / 16> read(S::kGroups > 1 ? group : 0, lane);
  // behind the contraction's end inside a piece: nothing of the rows, either
  const int h_end = a.K / 32, e_end = a.K - 32 * h_end - 8 * qq;
  const bool ragged = a.K & 7;
  const int64_t p0 = f0 + 16 * TP * wf + 4 * TP * qq;
  const bool whole_p = f0 + 16 * TP * (wf + 1) <= a.F;  // uniform
  for (int t = 0; t < mine; ++t) {
    const int64_t row0 = (int64_t(first) + int64_t(t) * stride) * kRowsTile;
    meet();
    const unsigned char* const stage = lds + (t % S::kRing) * S::kStage;
    const auto tile = [&](auto whole, auto cut) __attribute__((always_inline)) {
      constexpr bool kWhole = decltype(whole)::value, kCut = decltype(cut)::value;
      typename Out::Read early[S::kBlocks][TP];
      const auto each = [&](int x, auto&& f) __attribute__((always_inline)) {
        const int64_t q = row0 + 16 * (x * S::kGroups + group) + i;
#pragma unroll
        for (int u = 0; u < TP; ++u)
          if (kWhole || (q < a.n && p0 + 4 * u < a.F)) f(q, p0 + 4 * u, u);
      };
#pragma unroll
      for (int x = 0; x < S::kBlocks; ++x) each(x, [&](int64_t q, int64_t p, int u) __attribute__((always_inline)) { early[x][u] = out.read(q, p); });
#pragma unroll
      for (int x = 0; x < S::kBlocks; ++x) {
        float4_t acc[2][TP];
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
          for (int u = 0; u < TP; ++u) acc[o][u] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < 2 * KS; ++h) {
          half8_t v = read.get(stage + (h / 2) * (kRowsTile * 128), x * S::kGroups, h % 2);
          if (kCut && h == h_end) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e >= e_end) v[e] = half_t(0);
          }
#pragma unroll
          for (int o = 0; o < 2; ++o)
#pragma unroll
            for (int u = 0; u < TP; ++u) acc[o][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(weight[o][u][h], v, acc[o][u], 0, 0, 0);
        }
        each(x, [&](int64_t q, int64_t p, int u) __attribute__((always_inline)) { out.template put<kWhole>(0, q, p, early[x][u], acc[0][u], acc[1][u]); });
      }
    };
    if (whole_p && row0 + kRowsTile <= a.n) {
      if (ragged) tile(std::true_type(), std::true_type());
      else tile(std::true_type(), std::false_type());
    } else {
      tile(std::false_type(), std::true_type());
    }
  }
}
template <class S, class Out>
static hgnn_status gated_rows(const char* who, GatedRowsArgs& a, const Out& out, hipStream_t s) {
  a.chunks = int32_t(ceil_div(a.F, S::kFeatures));
  const int64_t blocks = std::max<int64_t>(1, kFull / a.chunks) * a.chunks;
  static uint64_t told = 0;
  const hgnn_status st = product_lds(reinterpret_cast<const void*>(&gated_rows_kernel<S, Out>), S::kLds, &told);
  if (st != HGNN_OK) return st;
  gated_rows_kernel<S, Out><<<unsigned(blocks), S::kThreads, S::kLds, s>>>(a, out);
  HGNN_LAUNCH_CHECK("gated_rows_kernel");
  return HGNN_OK;
}

// ---- few rows (up to 16) through a weight of up to 1024 inputs, a served model's: bound by reading the two weights once, and by latency.  A workgroup owns 32 features
// of both, its sixteen waves have 64 steps of the contraction each and take the weights straight into the registers that the products read, all of them at once; their
// sums meet in LDS.  One launch: by the product kernel the contraction is cut over workgroups, and joining the parts is a launch of 3 us (1 row of 1024 -> 4096, calls in
// a row, 8.8 us, by the product kernel 9.3; of 512 -> 512 4.5 and 6.4).  That is less than what a longer contraction or more workgroups than half of the units have
// cost here (1 row of 2048 -> 2048 11.7 and 9.1, of 4096 -> 32 11.7 and 9.5, of 1024 -> 11 008 18.8 and 10.9), or more rows (30 rows of 1024 -> 2048 9.9 and 9.3).
// Fragment e, item i is feature 2 i + e of the 32: of [K][F] a lane takes two neighbouring features of eight steps, 64 bytes of a line a load, and a lane's sums are
// eight consecutive features.
constexpr int kFewWaves = 16, kFewRows = 16, kFewFeatures = 32, kFewInputs = 64 * kFewWaves, kFewMost = 4096;
struct GatedFewArgs {
  const half_t *X, *Wg, *Wu;
  int64_t ldx, ldw;
  int32_t n, K, F;
};
struct FewStage {  // what a wave has in hand of 32 steps
  typedef unsigned uint4_t __attribute__((ext_vector_type(4)));
  uint4_t w[2][2];  // of both weights: [K][F] 2 x 4 lines of two features, [F][K] fragments
  half8_t x;
};
template <bool COL>
__device__ __forceinline__ void few_fetch(const GatedFewArgs& a, FewStage& st, int s, int f0, int lane) {
  const int i = lane & 15, qq = lane >> 4, k = 32 * s + 8 * qq;
#pragma unroll
  for (int o = 0; o < 2; ++o) {
    const half_t* const W = o ? a.Wu : a.Wg;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (COL) {
        const int f = f0 + 2 * i < a.F ? f0 + 2 * i : 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) st.w[o][e][j] = *reinterpret_cast<const uint32_t*>(W + int64_t(min(k + 4 * e + j, a.K - 1)) * a.ldw + f);
      } else {
        st.w[o][e] = *reinterpret_cast<const FewStage::uint4_t*>(W + int64_t(min(f0 + 2 * i + e, a.F - 1)) * a.ldw + (k < a.K ? k : 0));
      }
    }
  }
  st.x = *reinterpret_cast<const half8_t*>(a.X + int64_t(min(i, a.n - 1)) * a.ldx + (k < a.K ? k : 0));
}
template <bool COL>
__device__ __forceinline__ void few_multiply(const GatedFewArgs& a, const FewStage& st, int s, int lane, float4_t (&acc)[2][2]) {
  const int left = a.K - 32 * s - 8 * (lane >> 4);  // steps of the lane that exist: the others hold padding, or lines once more
  const bool cut = 32 * (s + 1) > a.K;              // uniform
  const auto ended = [&](half8_t v) __attribute__((always_inline)) {
    if (cut) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e >= left) v[e] = half_t(0);
    }
    return v;
  };
  const half8_t x = ended(st.x);
#pragma unroll
  for (int o = 0; o < 2; ++o)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      FewStage::uint4_t v = st.w[o][e];
      if (COL) {  // steps 2 j and 2 j + 1 of feature e of the pairs
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __builtin_amdgcn_perm(st.w[o][j / 2][2 * (j % 2) + 1], st.w[o][j / 2][2 * (j % 2)], e ? 0x07060302u : 0x05040100u);
      }
      acc[o][e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ended(__builtin_bit_cast(half8_t, v)), x, acc[o][e], 0, 0, 0);
    }
}
template <bool COL, class Out>
__global__ __launch_bounds__(kFewWaves* kWave) void gated_few_kernel(GatedFewArgs a, Out out) {
  typedef float float2_t __attribute__((ext_vector_type(2)));
  __shared__ __align__(16) float4_t sums[kFewWaves][2][2][kWave];
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int f0 = blockIdx.x * kFewFeatures, s = 2 * wave, steps = (a.K + 31) / 32;
  const float4_t none = {0.f, 0.f, 0.f, 0.f};
  float4_t acc[2][2] = {{none, none}, {none, none}};
  // Two neighbouring stages a wave: of [F][K] they are the two halves of a line.
  FewStage one, two;
  if (s < steps) few_fetch<COL>(a, one, s, f0, lane);
  if (s + 1 < steps) few_fetch<COL>(a, two, s + 1, f0, lane);
  if (s < steps) few_multiply<COL>(a, one, s, lane, acc);
  if (s + 1 < steps) few_multiply<COL>(a, two, s + 1, lane, acc);
  // thread (part of the waves, row, four features): waves 2 part and 2 part + 1, and then one of them the eight parts
  const int part = threadIdx.x >> 7, i = threadIdx.x & 15, m = (threadIdx.x >> 4) & 7, from = 16 * (m >> 1) + i, at = 2 * (m & 1);
#pragma unroll
  for (int o = 0; o < 2; ++o)
#pragma unroll
    for (int e = 0; e < 2; ++e) sums[wave][o][e][lane] = acc[o][e];
  __syncthreads();
  const auto value = [&](int w, int o, int e) { return reinterpret_cast<float2_t*>(reinterpret_cast<float*>(&sums[w][o][e][from]) + at); };
#pragma unroll
  for (int o = 0; o < 2; ++o)
#pragma unroll
    for (int e = 0; e < 2; ++e) *value(2 * part, o, e) += *value(2 * part + 1, o, e);
  __syncthreads();
  if (part) return;
  float2_t v[2][2];
#pragma unroll
  for (int o = 0; o < 2; ++o)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      v[o][e] = *value(0, o, e);
#pragma unroll
      for (int w = 2; w < kFewWaves; w += 2) v[o][e] += *value(w, o, e);
    }
  const int64_t p = f0 + 4 * m;
  if (i < a.n && p < a.F)
    out.template put<false>(0, i, p, out.read(i, p), float4_t{v[0][0][0], v[0][1][0], v[0][0][1], v[0][1][1]}, float4_t{v[1][0][0], v[1][1][0], v[1][0][1], v[1][1][1]});
}
template <bool COL, class Out>
static hgnn_status gated_few(const GatedFewArgs& a, const Out& out, hipStream_t s) {
  gated_few_kernel<COL><<<unsigned(ceil_div(a.F, kFewFeatures)), kFewWaves * kWave, 0, s>>>(a, out);
  HGNN_LAUNCH_CHECK("gated_few_kernel");
  return HGNN_OK;
}

struct GatedSizes {
  int64_t n, Fp;
  int K, F;
  Split gate, dx, dw;
  bool few, rows;  // gated_few_kernel, gated_rows_kernel
  size_t gate_part, dx_part, dw_part, d;
};
static GatedSizes gated_sizes(int64_t n, int32_t K, int32_t F) {
  GatedSizes z{};
  z.n = n, z.K = K, z.F = F, z.Fp = up(F, 32);  // rows of whole 128 bytes
  z.gate = split_of(n, F, K, true, 1);
  z.dx = split_of(n, K, F, false, 2);
  z.dw = split_of(K, 2 * z.Fp, n, false, 1);
  z.few = n <= kFewRows && K <= kFewInputs && F <= kFewMost;
  z.rows = is_rows(n, K, F);
  z.gate_part = z.gate.parts > 1 && !z.rows && !z.few ? size_t(z.gate.parts) * size_t(n) * 2 * size_t(z.Fp) * 4 : 0;
  z.dx_part = z.dx.parts > 1 ? size_t(z.dx.parts) * size_t(n) * size_t(up(K, 4)) * 4 : 0;
  z.dw_part = z.dw.parts > 1 ? size_t(z.dw.parts) * size_t(up(K, 4)) * 2 * size_t(z.Fp) * 4 : 0;
  z.d = size_t(up(n * 2 * z.Fp * 2, 256));
  return z;
}
// What the queries answer: enough for every number of rows up to n, since a program keeps one workspace for batches of all sizes, and fewer rows have fewer tiles
// and then more parts.  For the same number of tiles the most rows need most; from 128 rows on parts only become fewer, until there is one.  (The gradients' contraction
// over the rows has the parts of n, asked for.)
static size_t gated_most(int64_t n, int32_t K, int32_t F, bool grad) {
  size_t most = 0;
  const auto look = [&](int64_t rows) {
    const GatedSizes z = gated_sizes(rows, K, F);
    most = std::max(most, grad ? std::max(z.gate_part, z.dx_part) : z.gate_part);
    return rows < 128 || z.gate.parts > 1 || (grad && z.dx.parts > 1);
  };
  look(n);
  for (int64_t rows = 64; rows < n && look(rows); rows += 64) {}
  if (!grad) return most;
  const GatedSizes z = gated_sizes(n, K, F);
  return z.d + std::max(most, z.dw.most > 1 ? size_t(z.dw.most) * size_t(up(K, 4)) * 2 * size_t(z.Fp) * 4 : 0);
}

static hgnn_status join_grid(const char* who, int64_t fours, unsigned* blocks, int per = kJoinFours) {
  HGNN_REQUIRE(ceil_div(fours, per) <= 0xffffff, HGNN_EUNSUPPORTED, "%s: grid too large", who);
  *blocks = unsigned(ceil_div(fours, per));
  return HGNN_OK;
}

// both projections and `out` of their pairs of sums
template <class Out>
static hgnn_status gated_pairs(const char* who, const GatedSizes& z, const half_t* X, int64_t ldx, const half_t* Wg, const half_t* Wu, int64_t ldw, bool trans, float* part,
                               const Out& out, hipStream_t s) {
  if (z.few) {
    const GatedFewArgs f{X, Wg, Wu, ldx, ldw, int32_t(z.n), z.K, z.F};
    return trans ? gated_few<false>(f, out, s) : gated_few<true>(f, out, s);
  }
  if (z.rows) {
    GatedRowsArgs r{X, Wg, Wu, ldx, ldw, z.n, z.K, z.F, 1};
    const auto go = [&](auto pcol) -> hgnn_status {
      constexpr bool P = decltype(pcol)::value;
      if (z.K <= 64) return z.F <= 64 ? gated_rows<GatedRowsShape<1, 2, 2, P, 4>>(who, r, out, s) : z.F <= 128 ? gated_rows<GatedRowsShape<1, 2, 4, P, 4>>(who, r, out, s) : gated_rows<GatedRowsShape<1, 2, 8, P, 4>>(who, r, out, s);
      if (z.K <= 128) return z.F <= 64 ? gated_rows<GatedRowsShape<2, 2, 2, P, 4>>(who, r, out, s) : z.F <= 128 ? gated_rows<GatedRowsShape<2, 2, 4, P, 4>>(who, r, out, s) : gated_rows<GatedRowsShape<2, 2, 8, P, 4>>(who, r, out, s);
      if (z.F <= 64) return gated_rows<GatedRowsShape<4, 1, 4, P, 3>>(who, r, out, s);
      return z.K <= 192 ? gated_rows<GatedRowsShape<3, 1, 8, P, 3>>(who, r, out, s) : gated_rows<GatedRowsShape<4, 1, 8, P, 3>>(who, r, out, s);
    };
    return trans ? go(std::false_type()) : go(std::true_type());
  }
  ProductArgs a{};
  a.Q0 = X, a.Q1 = X, a.P0 = Wg, a.P1 = Wu, a.ldq = ldx, a.ldp = ldw, a.nq = z.n, a.np = z.F, a.K = z.K, a.part = z.gate.part, a.parts = z.gate.parts;
  const auto go = [&](auto shape) -> hgnn_status {
    typedef decltype(shape) S;
    if (z.gate.parts == 1) return product<S>(who, a, out, s);
    hgnn_status st = product<S>(who, a, GatedPart{part, z.n, z.Fp}, s);
    unsigned blocks;
    if (st == HGNN_OK) st = join_grid(who, z.n * ((z.F + 3) / 4), &blocks);
    if (st != HGNN_OK) return st;
    gated_join_kernel<<<blocks, kBlock, 0, s>>>(part, z.gate.parts, z.n, z.F, z.Fp, out);
    HGNN_LAUNCH_CHECK("gated_join_kernel");
    return HGNN_OK;
  };
  return trans ? with_product<kTwo, false, false>(z.gate.size, go) : with_product<kTwo, false, true>(z.gate.size, go);
}

template <ProductKind KIND, bool QCOL, bool PCOL>
static hgnn_status half_product(const char* who, ProductArgs& a, const Split& split, float* part, const HalfOut& out, hipStream_t s) {
  a.part = split.part, a.parts = split.parts;
  return with_product<KIND, QCOL, PCOL>(split.size, [&](auto shape) -> hgnn_status {
    typedef decltype(shape) S;
    if (split.parts == 1) return product<S>(who, a, out, s);
    const int64_t pitch = up(a.np, 4);
    hgnn_status st = product<S>(who, a, HalfPart{part, a.nq, pitch}, s);
    unsigned blocks;
    if (st == HGNN_OK) st = join_grid(who, a.nq * (pitch / 4), &blocks);
    if (st != HGNN_OK) return st;
    half_join_kernel<<<blocks, kBlock, 0, s>>>(part, split.parts, a.nq, pitch, out);
    HGNN_LAUNCH_CHECK("half_join_kernel");
    return HGNN_OK;
  });
}

static hgnn_status check_gated(const char* who, int64_t n, int32_t K, int32_t F, hgnn_activation act, int64_t ldx, int64_t ldw, int32_t trans_w, int64_t ldy) {
  HGNN_REQUIRE(n >= 0 && K > 0 && F > 0, HGNN_EINVAL, "%s: n = %lld, K = %d, F = %d", who, static_cast<long long>(n), K, F);
  HGNN_REQUIRE(act >= HGNN_SILU && act <= HGNN_RELU, HGNN_EINVAL, "%s: unknown activation %d", who, int(act));
  HGNN_REQUIRE(ldx >= K && ldy >= F && ldw >= (trans_w ? K : F), HGNN_EINVAL, "%s: leading dimension smaller than the row", who);
  HGNN_REQUIRE(K <= 65536 && F <= 65536 && n < (int64_t(1) << 31), HGNN_EUNSUPPORTED, "%s: K = %d / F = %d above 65536, or n = %lld from 2^31 on", who, K, F, static_cast<long long>(n));
  return HGNN_OK;
}
// (a tile's places are kept as 32-bit offsets from its first)
constexpr int64_t kMostPitch = int64_t(1) << 22;
static bool fits(const void* p, int64_t ld) { return aligned16(p) && ld % 8 == 0 && ld <= kMostPitch; }

}  // namespace hgnn

using namespace hgnn;

extern "C" {

size_t hgnn_gated_workspace(int64_t n, int32_t K, int32_t F) {
  if (n <= 0 || n > 0x7fffffff || K <= 0 || F <= 0 || K > 65536 || F > 65536) return 0;
  return gated_most(n, K, F, false);
}

hgnn_status hgnn_gated(int64_t n, int32_t K, int32_t F, hgnn_activation act, const hgnn_half* X, int64_t ldx, const hgnn_half* Wg, const hgnn_half* Wu, int64_t ldw,
                       int32_t trans_w, hgnn_half* Y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  const char* who = "hgnn_gated";
  hgnn_status st = check_gated(who, n, K, F, act, ldx, ldw, trans_w, ldy);
  if (st != HGNN_OK) return st;
  if (n == 0) return HGNN_OK;
  HGNN_REQUIRE(X && Wg && Wu && Y, HGNN_EINVAL, "%s: NULL argument", who);
  HGNN_REQUIRE(fits(X, ldx) && fits(Wg, ldw) && fits(Wu, ldw) && fits(Y, ldy), HGNN_EUNSUPPORTED, "%s: needs 16-byte aligned tensors and pitches that are multiples of 8, up to 2^22", who);
  const GatedSizes z = gated_sizes(n, K, F);
  HGNN_REQUIRE(z.gate_part == 0 || (workspace && workspace_bytes >= z.gate_part && aligned16(workspace)), HGNN_EINVAL,
               "%s: workspace of %zu bytes, needs %zu aligned to 16 (hgnn_gated_workspace)", who, workspace_bytes, z.gate_part);
  const auto half = [](const hgnn_half* p) { return reinterpret_cast<const half_t*>(p); };
  return gated_pairs(who, z, half(X), ldx, half(Wg), half(Wu), ldw, trans_w != 0, static_cast<float*>(workspace),
                     GatedOut{int(act), F, reinterpret_cast<half_t*>(Y), ldy}, static_cast<hipStream_t>(stream));
}

size_t hgnn_gated_grad_workspace(int64_t n, int32_t K, int32_t F) {
  if (n <= 0 || n > 0x7fffffff || K <= 0 || F <= 0 || K > 65536 || F > 65536) return 0;
  return gated_most(n, K, F, true);
}

hgnn_status hgnn_gated_grad(int64_t n, int32_t K, int32_t F, hgnn_activation act, const hgnn_half* X, int64_t ldx, const hgnn_half* Wg, const hgnn_half* Wu, int64_t ldw,
                            int32_t trans_w, const hgnn_half* dY, int64_t lddy, hgnn_half* dX, int64_t lddx, hgnn_half* dWg, hgnn_half* dWu, int64_t lddw, void* workspace,
                            size_t workspace_bytes, void* stream) {
  clear_error();
  const char* who = "hgnn_gated_grad";
  hgnn_status st = check_gated(who, n, K, F, act, ldx, ldw, trans_w, lddy);
  if (st != HGNN_OK) return st;
  HGNN_REQUIRE((dWg == nullptr) == (dWu == nullptr), HGNN_EINVAL, "%s: dWg and dWu go together", who);
  HGNN_REQUIRE((!dX || lddx >= K) && (!dWg || lddw >= (trans_w ? K : F)), HGNN_EINVAL, "%s: leading dimension smaller than the row", who);
  HGNN_REQUIRE((!dX || fits(dX, lddx)) && (!dWg || (fits(dWg, lddw) && fits(dWu, lddw))), HGNN_EUNSUPPORTED,
               "%s: needs 16-byte aligned tensors and pitches that are multiples of 8, up to 2^22", who);
  HGNN_REQUIRE(!dWg || dWg != dWu, HGNN_EINVAL, "%s: the same output twice", who);
  const bool trans = trans_w != 0;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const auto half = [](const hgnn_half* p) { return reinterpret_cast<const half_t*>(p); };
  const auto out = [](hgnn_half* p) { return reinterpret_cast<half_t*>(p); };
  const int64_t lines = trans ? F : K, cols = trans ? K : F;
  if (n == 0) {  // sums of nothing
    if (!dWg) return HGNN_OK;
    for (half_t* w : {out(dWg), out(dWu)}) {
      unsigned blocks;
      st = join_grid(who, lines * ceil_div(cols, 4), &blocks, kBlock);
      if (st != HGNN_OK) return st;
      half_zero_kernel<<<blocks, kBlock, 0, s>>>(w, lines, cols, lddw);
      HGNN_LAUNCH_CHECK("half_zero_kernel");
    }
    return HGNN_OK;
  }
  HGNN_REQUIRE(X && Wg && Wu && dY, HGNN_EINVAL, "%s: NULL argument", who);
  HGNN_REQUIRE(fits(X, ldx) && fits(Wg, ldw) && fits(Wu, ldw) && fits(dY, lddy), HGNN_EUNSUPPORTED,
               "%s: needs 16-byte aligned tensors and pitches that are multiples of 8, up to 2^22", who);
  const GatedSizes z = gated_sizes(n, K, F);
  const size_t need = z.d + std::max({z.gate_part, z.dx_part, z.dw_part});
  HGNN_REQUIRE(workspace && workspace_bytes >= need && aligned16(workspace), HGNN_EINVAL, "%s: workspace of %zu bytes, needs %zu aligned to 16 (hgnn_gated_grad_workspace)", who,
               workspace_bytes, need);
  if (!dX && !dWg) return HGNN_OK;
  half_t* const D = static_cast<half_t*>(workspace);
  float* const part = reinterpret_cast<float*>(static_cast<char*>(workspace) + z.d);
  st = gated_pairs(who, z, half(X), ldx, half(Wg), half(Wu), ldw, trans, part, GatedGradOut{int(act), half(dY), lddy, D, z.Fp}, s);
  if (st != HGNN_OK) return st;
  constexpr int64_t kNone = int64_t(1) << 62;
  if (dX) {
    ProductArgs a{};
    a.Q0 = D, a.Q1 = D + z.Fp, a.ldq = 2 * z.Fp, a.P0 = half(Wg), a.P1 = half(Wu), a.ldp = ldw, a.nq = n, a.np = K, a.K = F;
    const HalfOut to{out(dX), nullptr, lddx, kNone, kNone, n, K};
    st = trans ? half_product<kSegments, false, true>(who, a, z.dx, part, to, s) : half_product<kSegments, false, false>(who, a, z.dx, part, to, s);
    if (st != HGNN_OK) return st;
  }
  if (dWg) {
    ProductArgs a{};
    a.K = n;
    HalfOut to{out(dWg), out(dWu), lddw, kNone, kNone, lines, cols};
    if (trans) {
      a.Q0 = a.Q1 = D, a.ldq = 2 * z.Fp, a.nq = 2 * z.Fp, a.P0 = a.P1 = half(X), a.ldp = ldx, a.np = K;
      to.split_q = z.Fp;
    } else {
      a.Q0 = a.Q1 = half(X), a.ldq = ldx, a.nq = K, a.P0 = a.P1 = D, a.ldp = 2 * z.Fp, a.np = 2 * z.Fp;
      to.split_p = z.Fp;
    }
    st = half_product<kOne, true, true>(who, a, z.dw, part, to, s);
  }
  return st;
}

}  // extern "C"
