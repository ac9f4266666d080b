// Log probabilities of labels under a softmax over classes, with the entropy and the best alternatives, and their gradient: what stands behind the last
// layer.  m = max x, S = sum exp(x - m), L = log S; log p_c = (x_c - m) - L, entropy = L - sum exp(x - m) (x - m) / S.  The maximum and L are kept apart: their sum would
// lose the small differences of large scores to its rounding.
#include <math.h>

#include "common.h"
#include "rows.h"

namespace hgnn {

constexpr float kLow = -INFINITY;
constexpr int kMostTop = 32;   // alternatives at most: a lane of a wave each
constexpr int kMostSplits = 64;  // workgroups of a row at most: a lane of a wave each

// What a set of classes holds: the maximum, sum of exp(x - max), sum of exp(x - max) (x - max).  An empty one, or one of -inf alone, is (kNone, 0, 0): a maximum that is
// finite takes no part in inf - inf.
constexpr float kNone = -3.4028235e38f;
struct Mass {
  float m = kNone, s = 0.f, t = 0.f;
};

__device__ __forceinline__ Mass joined(const Mass& a, const Mass& b) {
  Mass r;
  r.m = fmaxf(a.m, b.m);
  const float da = a.m - r.m, db = b.m - r.m, fa = __expf(da), fb = __expf(db);
  r.s = fa * a.s + fb * b.s;
  // (a difference beyond the range comes with a factor of zero, whose product would be no number)
  r.t = fa * (a.t + fmaxf(da, -1e4f) * a.s) + fb * (b.t + fmaxf(db, -1e4f) * b.s);
  return r;
}

__device__ __forceinline__ float piece_max(const Piece& x) {
  return fmaxf(fmaxf(fmaxf(x.v[0], x.v[1]), fmaxf(x.v[2], x.v[3])), fmaxf(fmaxf(x.v[4], x.v[5]), fmaxf(x.v[6], x.v[7])));
}

// adds pieces to a lane's mass; a class that is masked by -inf adds nothing
template <int N>
__device__ __forceinline__ void add_pieces(Mass& a, const Piece (&x)[N], const float (&top)[N]) {
  float m = a.m;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, top[i]);
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = x[i].v[j] - m, e = __expf(d);
      s += e;
      t = fmaf(e, fmaxf(d, -1e4f), t);
    }
  const float d = a.m - m, f = __expf(d);
  a.t = fmaf(f, a.t + fmaxf(d, -1e4f) * a.s, t);
  a.s = fmaf(f, a.s, s);
  a.m = m;
}

template <int L>
__device__ __forceinline__ Mass lanes_mass(Mass a) {
#pragma unroll
  for (int d = 1; d < L; d <<= 1) a = joined(a, Mass{__shfl_xor(a.m, d), __shfl_xor(a.s, d), __shfl_xor(a.t, d)});
  return a;
}

// What is kept of a row: its maximum and the logarithm of the sum.  A row of -inf alone is (-inf, 0); one with +inf or NaN is no number.
struct RowStats {
  float m, l;
  __device__ __forceinline__ float log_p(float x) const { return m == kLow ? kLow : (x - m) - l; }
};
__device__ __forceinline__ RowStats stats_of(const Mass& a) {
  if (a.s == 0.f) return RowStats{kLow, 0.f};
  if (!(a.s > 0.f)) return RowStats{NAN, NAN};
  return RowStats{a.m, logf(a.s)};
}
__device__ __forceinline__ float entropy_of(const Mass& a) { return a.s == 0.f ? 0.f : logf(a.s) - a.t / a.s; }

// ---- the best k of a wave: lane j holds the j-th best (x > -inf), falling, classes rising among equals
struct Best {
  float v = kLow;
  int c = -1;
};

// Takes those of a wave's classes c0 + 8 lane + j (j < 8, scores x, -inf where there is none) that are among the best k.  They are taken in falling order, so no more than
// k are, and a wave comes by its classes in rising order, so among equals the first one stays ahead.
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ void take_best(Best& best, float& least, int k, Piece& x, float top, int c0) {
  const int lane = threadIdx.x & (kWave - 1);
  while (__ballot(top > least)) {
    const float v = wave_max(top);
    const int from = __builtin_ctzll(__ballot(top == v));
    int j = 0;
#pragma unroll
    for (int i = 7; i >= 0; --i) j = x.v[i] == v ? i : j;
    const int c = __shfl(c0 + 8 * lane + j, from);
    if (lane == from) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i == j) x.v[i] = kLow;
      top = piece_max(x);
    }
    const int rank = __popcll(__ballot(best.v >= v));
    const float pv = __shfl_up(best.v, 1);
    const int pc = __shfl_up(best.c, 1);
    if (lane > rank) best.v = pv, best.c = pc;
    if (lane == rank) best.v = v, best.c = c;
    least = __shfl(best.v, k - 1);
  }
}

struct ScoreArgs {
  int64_t n;
  int C, k;
  const void* logits;
  int64_t ld;
  const int* labels;
  float *logprob, *stats, *entropy, *top;
  int* top_class;
  // several workgroups to a row: what each of them has found
  int splits;
  int64_t span;      // classes of a wave
  float* part;       // [n][splits][3]
  float* part_top;   // [n][splits][k]
  int* part_class;
};

// The outputs of a row but for the alternatives, by one lane.
template <class T>
__device__ __forceinline__ void store_row(const ScoreArgs& a, int64_t row, const Mass& mass) {
  const RowStats st = stats_of(mass);
  if (a.stats) a.stats[2 * row] = st.m, a.stats[2 * row + 1] = st.l;
  if (a.entropy) a.entropy[row] = entropy_of(mass);
  if (a.logprob) {
    const int y = a.labels[row];
    float v = 0.f;
    if (uint32_t(y) < uint32_t(a.C)) v = st.log_p(float(static_cast<const T*>(a.logits)[row * a.ld + y]));
    a.logprob[row] = v;
  }
}

// The alternatives of a row, by a wave.  Where fewer than k scores are above -inf, the first of the other classes fill up.
template <class T>
__device__ __forceinline__ void store_best(const ScoreArgs& a, int64_t row, const Mass& mass, Best best) {
  const int lane = threadIdx.x & (kWave - 1);
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  int held = __popcll(__ballot(lane < a.k && best.c >= 0));
  for (int c0 = 0; held < a.k && c0 < a.C; c0 += kWave) {
    const bool low = c0 + lane < a.C && !(float(x[c0 + lane]) > kLow);
    const uint64_t lows = __ballot(low);
    const int at = held + __popcll(lows & ((uint64_t(1) << lane) - 1));
    if (low && at < a.k) {
      a.top[row * a.k + at] = mass.s == mass.s ? kLow : NAN;
      a.top_class[row * a.k + at] = c0 + lane;
    }
    held += __popcll(lows);
  }
  if (lane < a.k && best.c >= 0) {
    a.top[row * a.k + lane] = stats_of(mass).log_p(best.v);
    a.top_class[row * a.k + lane] = best.c;
  }
}

// lists of falling scores, one for each lane (p: its next entry, n entries in all, class -1: an empty one), become one; among equals a lower lane's come first
template <class Entry>
__device__ __forceinline__ Best merge_lists(int k, int n, Entry&& entry) {
  const int lane = threadIdx.x & (kWave - 1);
  Best out, mine;
  int p = 0;
  if (n > 0) mine = entry(0);
  for (int r = 0; r < k; ++r) {
    const float v = wave_max(mine.c >= 0 ? mine.v : kLow);
    const uint64_t have = __ballot(mine.c >= 0 && mine.v == v);
    if (!have) break;
    const int from = __builtin_ctzll(have), c = __shfl(mine.c, from);
    if (lane == r) out.v = v, out.c = c;
    if (lane == from) {
      ++p;
      mine = Best{};
      if (p < n) mine = entry(p);
    }
  }
  return out;
}

// Rows of up to 512 classes: L lanes hold a row, a piece each.
template <class T, int L>
__global__ __launch_bounds__(kBlock) void logprob_group_kernel(ScoreArgs a) {
  const int64_t row = (int64_t(blockIdx.x) * kBlock + threadIdx.x) / L;
  const int l = threadIdx.x % L;
  const bool real = row < a.n;
  const T* const x = static_cast<const T*>(a.logits) + (real ? row : a.n - 1) * a.ld;
  Piece p[1];
#pragma unroll
  for (int j = 0; j < 8; ++j) p[0].v[j] = kLow;
  if (8 * l < a.C) p[0] = load_piece(x + 8 * l, a.C - 8 * l, kLow);
  float top[1] = {piece_max(p[0])};
  Mass mass;
  add_pieces(mass, p, top);
  mass = lanes_mass<L>(mass);
  if (real && l == 0) store_row<T>(a, row, mass);
  const RowStats st = stats_of(mass);
  float t = top[0];
  // of equal scores the lowest class; those that are not above -inf, in their order, once the others are out
  uint32_t left = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) left |= uint32_t(8 * l + j < a.C) << j;
  for (int r = 0; r < a.k; ++r) {
    float v = t;
#pragma unroll
    for (int d = 1; d < L; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
    const bool fill = !(v > kLow);
    int c = 0x7fffffff;
#pragma unroll
    for (int j = 7; j >= 0; --j)
      if ((left >> j & 1) && (fill ? !(p[0].v[j] > kLow) : p[0].v[j] == v)) c = 8 * l + j;
#pragma unroll
    for (int d = 1; d < L; d <<= 1) c = min(c, __shfl_xor(c, d));
    if (c / 8 == l) {
      left &= ~(1u << (c % 8));
      t = kLow;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (left >> j & 1) t = fmaxf(t, p[0].v[j]);
    }
    if (real && l == 0) {
      a.top[row * a.k + r] = mass.s == mass.s ? st.log_p(v) : NAN;
      a.top_class[row * a.k + r] = c;
    }
  }
}

// A workgroup to a row, or to one of `splits` parts of it; every wave takes a stretch of classes, so that what it finds has a place among the others'.
constexpr int kPieces = 4;  // of a lane in flight
template <class T>
__global__ __launch_bounds__(kBlock) void logprob_row_kernel(ScoreArgs a) {
  __shared__ float s_mass[kWavesPerBlock][3], s_top[kWavesPerBlock][kMostTop];
  __shared__ int s_class[kWavesPerBlock][kMostTop];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int64_t row = blockIdx.x / a.splits;
  const int split = blockIdx.x % a.splits;
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  const int64_t first = (int64_t(split) * kWavesPerBlock + wave) * a.span;
  const int c0 = int(first < a.C ? first : a.C), c1 = int(first + a.span < a.C ? first + a.span : a.C);
  Mass mass;
  Best best;
  float least = kLow;
  for (int c = c0; c < c1; c += 8 * kWave * kPieces) {
    Piece p[kPieces];
    float top[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int at = c + 8 * (i * kWave + lane);
#pragma unroll
      for (int j = 0; j < 8; ++j) p[i].v[j] = kLow;
      if (at < c1) p[i] = load_piece(x + at, c1 - at, kLow);
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) top[i] = piece_max(p[i]);
    add_pieces(mass, p, top);
    if (a.k > 0)
#pragma unroll
      for (int i = 0; i < kPieces; ++i) take_best(best, least, a.k, p[i], top[i], c + 8 * i * kWave);
  }
  mass = lanes_mass<kWave>(mass);
  if (lane == 0) s_mass[wave][0] = mass.m, s_mass[wave][1] = mass.s, s_mass[wave][2] = mass.t;
  if (lane < a.k) s_top[wave][lane] = best.v, s_class[wave][lane] = best.c;
  __syncthreads();
  if (wave > 0) return;
  mass = Mass{s_mass[0][0], s_mass[0][1], s_mass[0][2]};
  for (int w = 1; w < kWavesPerBlock; ++w) mass = joined(mass, Mass{s_mass[w][0], s_mass[w][1], s_mass[w][2]});
  if (a.k > 0) best = merge_lists(a.k, lane < kWavesPerBlock ? a.k : 0, [&](int p) { return Best{s_top[lane][p], s_class[lane][p]}; });
  if (a.splits == 1) {
    if (lane == 0) store_row<T>(a, row, mass);
    if (a.k > 0) store_best<T>(a, row, mass, best);
    return;
  }
  if (lane == 0) {
    float* const q = a.part + 3 * (row * a.splits + split);
    q[0] = mass.m, q[1] = mass.s, q[2] = mass.t;
  }
  if (lane < a.k) {
    a.part_top[(row * a.splits + split) * a.k + lane] = best.v;
    a.part_class[(row * a.splits + split) * a.k + lane] = best.c;
  }
}

// the parts of a row, by a wave
template <class T>
__global__ __launch_bounds__(kWave) void logprob_join_kernel(ScoreArgs a) {
  const int lane = threadIdx.x;
  const int64_t row = blockIdx.x;
  Mass mass;
  if (lane < a.splits) {
    const float* const q = a.part + 3 * (row * a.splits + lane);
    mass = Mass{q[0], q[1], q[2]};
  }
  mass = lanes_mass<kWave>(mass);
  if (lane == 0) store_row<T>(a, row, mass);
  if (a.k == 0) return;
  const int64_t at = (row * a.splits + lane) * a.k;
  const Best best = merge_lists(a.k, lane < a.splits ? a.k : 0, [&](int p) { return Best{a.part_top[at + p], a.part_class[at + p]}; });
  store_best<T>(a, row, mass, best);
}

// ---- the gradient: dx_c = g (1[c = y] - p_c) - h p_c (log p_c + entropy), p_c = exp((x_c - m) - L)
struct ScoreGradArgs {
  int64_t n;
  int C, chunks;
  const void* logits;
  int64_t ld;
  const int* labels;
  const float *stats, *dlogprob, *entropy, *dentropy;
  void* dlogits;
  int64_t ldd;
};

// L lanes take a row, or 64 of them one of its chunks, a piece or kPieces each.  A lane reads what it overwrites: the logits may be the output.
template <class T, int L, int N>
__global__ __launch_bounds__(kBlock) void logprob_grad_kernel(ScoreGradArgs a) {
  const int64_t unit = (int64_t(blockIdx.x) * kBlock + threadIdx.x) / L;
  const int64_t row = N == 1 ? unit : unit / a.chunks;
  if (row >= a.n) return;
  const int l = threadIdx.x % L, c0 = N == 1 ? 0 : int(unit % a.chunks) * (8 * L * N);
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  T* const dx = static_cast<T*>(a.dlogits) + row * a.ldd;
  Piece p[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int at = c0 + 8 * (i * L + l);
    if (at < a.C) p[i] = load_piece(x + at, a.C - at, kLow);
  }
  const int y = a.labels ? a.labels[row] : -1;
  const bool real = uint32_t(y) < uint32_t(a.C);
  const float m = a.stats[2 * row], s = a.stats[2 * row + 1], g = real ? a.dlogprob[row] : 0.f;
  const float h = a.dentropy ? a.dentropy[row] : 0.f, e = a.dentropy ? a.entropy[row] : 0.f;
  const bool none = m == kLow;  // a row of -inf alone
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int at = c0 + 8 * (i * L + l);
    if (at >= a.C) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float lp = none ? kLow : (p[i].v[j] - m) - s, q = __expf(lp);
      float v = g * ((at + j == y && !none ? 1.f : 0.f) - q);
      v -= h * (q * (fmaxf(lp, -1e4f) + e));
      p[i].v[j] = v;
    }
    store_piece(dx + at, a.C - at, p[i]);
  }
}

constexpr int kGroupClasses = 8 * kWave;  // most classes that the lanes of a wave hold at once
// Workgroups of a row: as many as fill the chip, of no less than a piece chunk for every wave
static int splits_of(int64_t n, int C) {
  const int64_t most = ceil_div(C, int64_t(8) * kWave * kPieces * kWavesPerBlock);
  const int64_t want = ceil_div(1024, n);
  int64_t s = most < want ? most : want;
  return int(s < 1 ? 1 : (s > kMostSplits ? kMostSplits : s));
}
static size_t up256(size_t n) { return (n + 255) / 256 * 256; }

template <class T>
static hgnn_status logprob(ScoreArgs& a, hipStream_t s) {
  if (a.C <= kGroupClasses) {
    const int L = pow2_at_least((a.C + 7) / 8);
    const int64_t blocks = ceil_div(a.n * L, kBlock);
    HGNN_REQUIRE(blocks <= 0x7fffffff, HGNN_EUNSUPPORTED, "hgnn_logprob: grid too large");
    const dim3 grid{unsigned(blocks)};
    switch (L) {
      case 1: logprob_group_kernel<T, 1><<<grid, kBlock, 0, s>>>(a); break;
      case 2: logprob_group_kernel<T, 2><<<grid, kBlock, 0, s>>>(a); break;
      case 4: logprob_group_kernel<T, 4><<<grid, kBlock, 0, s>>>(a); break;
      case 8: logprob_group_kernel<T, 8><<<grid, kBlock, 0, s>>>(a); break;
      case 16: logprob_group_kernel<T, 16><<<grid, kBlock, 0, s>>>(a); break;
      case 32: logprob_group_kernel<T, 32><<<grid, kBlock, 0, s>>>(a); break;
      default: logprob_group_kernel<T, 64><<<grid, kBlock, 0, s>>>(a); break;
    }
    HGNN_LAUNCH_CHECK("logprob_group_kernel");
    return HGNN_OK;
  }
  HGNN_REQUIRE(a.n * a.splits <= 0x7fffffff, HGNN_EUNSUPPORTED, "hgnn_logprob: grid too large");
  a.span = ceil_div(ceil_div(a.C, int64_t(a.splits) * kWavesPerBlock), 8) * 8;
  logprob_row_kernel<T><<<dim3(unsigned(a.n * a.splits)), kBlock, 0, s>>>(a);
  HGNN_LAUNCH_CHECK("logprob_row_kernel");
  if (a.splits > 1) {
    logprob_join_kernel<T><<<dim3(unsigned(a.n)), kWave, 0, s>>>(a);
    HGNN_LAUNCH_CHECK("logprob_join_kernel");
  }
  return HGNN_OK;
}

template <class T>
static hgnn_status logprob_grad(ScoreGradArgs& a, hipStream_t s) {
  const bool group = a.C <= kGroupClasses;
  const int L = group ? pow2_at_least((a.C + 7) / 8) : kWave;
  a.chunks = group ? 1 : int(ceil_div(a.C, int64_t(8) * kWave * kPieces));
  const int64_t blocks = ceil_div(a.n * a.chunks * L, kBlock);
  HGNN_REQUIRE(blocks <= 0x7fffffff, HGNN_EUNSUPPORTED, "hgnn_logprob_grad: grid too large");
  const dim3 grid{unsigned(blocks)};
  if (!group) {
    logprob_grad_kernel<T, kWave, kPieces><<<grid, kBlock, 0, s>>>(a);
  } else {
    switch (L) {
      case 1: logprob_grad_kernel<T, 1, 1><<<grid, kBlock, 0, s>>>(a); break;
      case 2: logprob_grad_kernel<T, 2, 1><<<grid, kBlock, 0, s>>>(a); break;
      case 4: logprob_grad_kernel<T, 4, 1><<<grid, kBlock, 0, s>>>(a); break;
      case 8: logprob_grad_kernel<T, 8, 1><<<grid, kBlock, 0, s>>>(a); break;
      case 16: logprob_grad_kernel<T, 16, 1><<<grid, kBlock, 0, s>>>(a); break;
      case 32: logprob_grad_kernel<T, 32, 1><<<grid, kBlock, 0, s>>>(a); break;
      default: logprob_grad_kernel<T, 64, 1><<<grid, kBlock, 0, s>>>(a); break;
    }
  }
  HGNN_LAUNCH_CHECK("logprob_grad_kernel");
  return HGNN_OK;
}

struct ScoreSpace {
  float *part, *part_top;
  int* part_class;
  size_t bytes;
};
static ScoreSpace score_space(void* base, int64_t n, int C, int k) {
  ScoreSpace p{};
  if (n <= 0 || C <= kGroupClasses) return p;
  const int splits = splits_of(n, C);
  if (splits == 1) return p;
  const size_t each = size_t(n) * size_t(splits);
  char* const at = static_cast<char*>(base);
  p.part = reinterpret_cast<float*>(at);
  p.bytes = up256(each * 3 * sizeof(float));
  p.part_top = reinterpret_cast<float*>(at + p.bytes);
  p.bytes += up256(each * size_t(k) * sizeof(float));
  p.part_class = reinterpret_cast<int*>(at + p.bytes);
  p.bytes += up256(each * size_t(k) * sizeof(int));
  return p;
}

}  // namespace hgnn

using namespace hgnn;

extern "C" {

size_t hgnn_logprob_workspace(int64_t n, int32_t C, int32_t k) {
  if (n <= 0 || C <= 0 || k < 0 || k > kMostTop) return 0;
  return score_space(nullptr, n, C, k).bytes;
}

hgnn_status hgnn_logprob(int64_t n, int32_t C, hgnn_type type, const void* logits, int64_t ld, const int32_t* labels, float* logprob_out, float* stats,
                         float* entropy, int32_t k, float* top_logprob, int32_t* top_class, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  const char* who = "hgnn_logprob";
  HGNN_REQUIRE(n >= 0 && C > 0, HGNN_EINVAL, "%s: n = %lld, C = %d", who, static_cast<long long>(n), C);
  HGNN_REQUIRE(known_type(type), HGNN_EINVAL, "%s: unknown type %d", who, int(type));
  HGNN_REQUIRE(ld >= C, HGNN_EINVAL, "%s: leading dimension smaller than C", who);
  HGNN_REQUIRE(k >= 0 && k <= C, HGNN_EINVAL, "%s: %d alternatives of %d classes", who, k, C);
  HGNN_REQUIRE(k <= kMostTop, HGNN_EUNSUPPORTED, "%s: more than %d alternatives", who, kMostTop);
  HGNN_REQUIRE(C <= (1 << 30), HGNN_EUNSUPPORTED, "%s: C = %d above 2^30", who, C);
  if (n == 0) return HGNN_OK;
  HGNN_REQUIRE(logits && (k == 0 || (top_logprob && top_class)), HGNN_EINVAL, "%s: NULL argument", who);
  HGNN_REQUIRE((labels == nullptr) == (logprob_out == nullptr), HGNN_EINVAL, "%s: labels and logprob go together", who);
  const ScoreSpace w = score_space(workspace, n, C, k);
  HGNN_REQUIRE(w.bytes == 0 || (workspace != nullptr && workspace_bytes >= w.bytes), HGNN_EINVAL,
               "%s: workspace of %zu bytes, needs %zu (hgnn_logprob_workspace)", who, workspace_bytes, w.bytes);
  HGNN_REQUIRE(aligned_to_type(logits, type) && aligned_to_type(labels, HGNN_F32) && aligned_to_type(logprob_out, HGNN_F32) && aligned_to_type(stats, HGNN_F32) &&
                   aligned_to_type(entropy, HGNN_F32) && aligned_to_type(top_logprob, HGNN_F32) && aligned_to_type(top_class, HGNN_F32) &&
                   (w.bytes == 0 || aligned_to_type(workspace, HGNN_F32)),
               HGNN_EINVAL, "%s: an array that is not aligned to its type", who);
  ScoreArgs a{n, C, k, logits, ld, labels, logprob_out, stats, entropy, top_logprob, top_class, splits_of(n, C), 0, w.part, w.part_top, w.part_class};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return type == HGNN_F16 ? logprob<half_t>(a, s) : logprob<float>(a, s);
}

hgnn_status hgnn_logprob_grad(int64_t n, int32_t C, hgnn_type type, const void* logits, int64_t ld, const int32_t* labels, const float* stats,
                              const float* dlogprob, const float* entropy, const float* dentropy, void* dlogits, int64_t ldd, void* stream) {
  clear_error();
  const char* who = "hgnn_logprob_grad";
  HGNN_REQUIRE(n >= 0 && C > 0, HGNN_EINVAL, "%s: n = %lld, C = %d", who, static_cast<long long>(n), C);
  HGNN_REQUIRE(known_type(type), HGNN_EINVAL, "%s: unknown type %d", who, int(type));
  HGNN_REQUIRE(ld >= C && ldd >= C, HGNN_EINVAL, "%s: leading dimension smaller than C", who);
  HGNN_REQUIRE(C <= (1 << 30), HGNN_EUNSUPPORTED, "%s: C = %d above 2^30", who, C);
  HGNN_REQUIRE((labels == nullptr) == (dlogprob == nullptr), HGNN_EINVAL, "%s: labels and dlogprob go together", who);
  HGNN_REQUIRE((dentropy == nullptr) || entropy, HGNN_EINVAL, "%s: dentropy without the entropy", who);
  if (n == 0) return HGNN_OK;
  HGNN_REQUIRE(logits && stats && dlogits, HGNN_EINVAL, "%s: NULL argument", who);
  HGNN_REQUIRE(logits != dlogits || ld == ldd, HGNN_EINVAL, "%s: in place with another leading dimension", who);
  HGNN_REQUIRE(aligned_to_type(logits, type) && aligned_to_type(dlogits, type) && aligned_to_type(labels, HGNN_F32) && aligned_to_type(stats, HGNN_F32) &&
                   aligned_to_type(dlogprob, HGNN_F32) && aligned_to_type(entropy, HGNN_F32) && aligned_to_type(dentropy, HGNN_F32),
               HGNN_EINVAL, "%s: an array that is not aligned to its type", who);
  ScoreGradArgs a{n, C, 1, logits, ld, labels, stats, dlogprob, entropy, dentropy, dlogits, ldd};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return type == HGNN_F16 ? logprob_grad<half_t>(a, s) : logprob_grad<float>(a, s);
}

}  // extern "C"
