// Log probabilities of labels under a softmax over classes, with the entropy and the best alternatives, and their gradient: what stands behind the last layer.
// m = max x, S = sum exp(x - m), L = log S; log p_c = (x_c - m) - L, entropy = L - sum exp(x - m) (x - m) / S.  The maximum and L are kept apart: their sum
// would lose the small differences of large scores to its rounding.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "rows.h"

namespace hgnn {

constexpr float kLow = -INFINITY;
constexpr int kMostTop = 32;     // alternatives at most: a lane of a wave each
constexpr int kMostSplits = 64;  // workgroups of a row at most: a lane of a wave each
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// What a set of classes holds: the maximum m, s = sum 2^y and t = sum 2^y y, y = (x - m) log2(e).  An empty one, or one of -inf alone, has s = 0 and a maximum
// below all others, which is finite, so that it takes no part in inf - inf. fp16: y = fma(x, log2(e), -c) in one instruction, with the conversion; c, the
// rounded m log2(e), is the same for all classes, so its error goes in and out with it (shift_of). fp32, whose products with log2(e) may overflow: a difference
// and a product.
template <class T>
struct Mass {
  static constexpr bool kHalf = sizeof(T) == 2;
  static constexpr float kNone = kHalf ? -1e5f : -3.4028235e38f;
  float m, s, t;
  static __device__ __forceinline__ Mass none() { return Mass{kNone, 0.f, 0.f}; }
  static __device__ __forceinline__ float offset(float m) {
#pragma clang fp contract(off)  // rounded here, whatever it is added to: it has to be the same everywhere
    return kHalf ? m * kLog2e : m;
  }
  static __device__ __forceinline__ float y(float x, float offset) { return kHalf ? fmaf(x, kLog2e, -offset) : (x - offset) * kLog2e; }
  // from the maximum m to the maximum to, in y
  static __device__ __forceinline__ float step(float m, float to) { return kHalf ? offset(m) - offset(to) : (m - to) * kLog2e; }
  // what y lacks of (x - m) log2(e)
  static __device__ __forceinline__ float shift(float m) { return kHalf ? -fmaf(m, kLog2e, -offset(m)) : 0.f; }
};
__device__ __forceinline__ float exp2_of(float y) { return __builtin_amdgcn_exp2f(y); }
// (-inf comes with a factor of zero, whose product would be no number)
__device__ __forceinline__ float bounded(float y) { return fmaxf(y, -1e4f); }

// ---- over L lanes, L a power of two: pairs of lanes by data-parallel primitives (common.h), beyond a row of 16 by swaps
enum class Over { kSum, kMax, kMin };
template <Over OP>
__device__ __forceinline__ float both(float a, float b) {
  return OP == Over::kSum ? a + b : fmaxf(a, b);
}
template <Over OP>
__device__ __forceinline__ int both(int a, int b) {
  return OP == Over::kSum ? a + b : (OP == Over::kMax ? max(a, b) : min(a, b));
}
template <int CTRL, class V>
__device__ __forceinline__ V paired(V v) {
  int w;
  __builtin_memcpy(&w, &v, 4);
  w = __builtin_amdgcn_update_dpp(0, w, CTRL, 0xf, 0xf, false);
  __builtin_memcpy(&v, &w, 4);
  return v;
}
template <int L, Over OP, class V>
__device__ __forceinline__ V lanes_all(V v) {
  if (L >= 2) v = both<OP>(v, paired<0xB1>(v));
  if (L >= 4) v = both<OP>(v, paired<0x4E>(v));
  if (L >= 8) v = both<OP>(v, paired<0x141>(v));
  if (L >= 16) v = both<OP>(v, paired<0x140>(v));
  typedef unsigned uint2_t __attribute__((ext_vector_type(2)));
  auto halves = [](uint2_t r) {
    V a, b;
    const unsigned p = r[0], q = r[1];
    __builtin_memcpy(&a, &p, 4);
    __builtin_memcpy(&b, &q, 4);
    return both<OP>(a, b);
  };
  unsigned w;
  if (L >= 32) {
    __builtin_memcpy(&w, &v, 4);
    v = halves(__builtin_amdgcn_permlane16_swap(w, w, false, false));
  }
  if (L >= 64) {
    __builtin_memcpy(&w, &v, 4);
    v = halves(__builtin_amdgcn_permlane32_swap(w, w, false, false));
  }
  return v;
}
template <int L, class T>
__device__ __forceinline__ Mass<T> lanes_mass(const Mass<T>& a) {
  Mass<T> r;
  r.m = lanes_all<L, Over::kMax>(a.m);
  const float d = Mass<T>::step(a.m, r.m), f = exp2_of(d);
  r.s = lanes_all<L, Over::kSum>(f * a.s);
  r.t = lanes_all<L, Over::kSum>(f * (a.t + bounded(d) * a.s));
  return r;
}

template <class T>
__device__ __forceinline__ float piece_max(const RawPiece<T>& x) {
  if constexpr (sizeof(T) == 2) {
    const half4_t a = __builtin_elementwise_max(half4_t{x.v[0], x.v[1], x.v[2], x.v[3]}, half4_t{x.v[4], x.v[5], x.v[6], x.v[7]});
    const half2_t b = __builtin_elementwise_max(half2_t{a[0], a[1]}, half2_t{a[2], a[3]});
    return fmaxf(float(b[0]), float(b[1]));
  } else {
    return fmaxf(fmaxf(fmaxf(x.v[0], x.v[1]), fmaxf(x.v[2], x.v[3])), fmaxf(fmaxf(x.v[4], x.v[5]), fmaxf(x.v[6], x.v[7])));
  }
}
// a row's piece at class c; -inf behind the row's end
template <class T>
__device__ __forceinline__ RawPiece<T> load_classes(const T* row, int c, int C, int64_t inside) {
  RawPiece<T> r;
  r.v = T(kLow);
  if (c >= C) return r;
  const RawPiece<T> x = load_raw(row + c, C - c, inside - c);
  if (c + 8 <= C) return x;
#pragma unroll
  for (int j = 0; j < 8; ++j) r.v[j] = c + j < C ? x.v[j] : T(kLow);
  return r;
}

// adds pieces to a lane's mass; a class that is masked by -inf adds nothing
template <bool ENTROPY, class T, int N>
__device__ __forceinline__ void add_pieces(Mass<T>& a, const RawPiece<T> (&x)[N], const float (&top)[N]) {
  float m = a.m;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, top[i]);
  const float offset = Mass<T>::offset(m);
  float s = 0.f, t = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float y = Mass<T>::y(float(x[i].v[j]), offset), e = exp2_of(y);
      s += e;
      if (ENTROPY) t = fmaf(e, bounded(y), t);
    }
  const float d = Mass<T>::step(a.m, m), f = exp2_of(d);
  if (ENTROPY) a.t = fmaf(f, a.t + bounded(d) * a.s, t);
  a.s = fmaf(f, a.s, s);
  a.m = m;
}

// What is kept of a row: its maximum and the logarithm of the sum.  A row of -inf alone is (-inf, 0); one with +inf or NaN is no number.
struct RowStats {
  float m, l;
  __device__ __forceinline__ float log_p(float x) const { return m == kLow ? kLow : (x - m) - l; }
};
template <class T>
__device__ __forceinline__ RowStats stats_of(const Mass<T>& a) {
  if (a.s == 0.f) return RowStats{kLow, 0.f};
  if (!(a.s > 0.f)) return RowStats{NAN, NAN};
  return RowStats{a.m, fmaf(Mass<T>::shift(a.m), kLn2, logf(a.s))};
}
template <class T>
__device__ __forceinline__ float entropy_of(const Mass<T>& a) {
  return a.s == 0.f ? 0.f : logf(a.s) - kLn2 * (a.t / a.s);
}

// ---- the best k of a wave: lane j holds the j-th best (x > -inf), falling, classes rising among equals
struct Best {
  float v = kLow;
  int c = -1;
};
__device__ __forceinline__ float lane_value(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
// a piece whose scores are taken apart here and not ahead of the loop, where all pieces' would fill the registers
template <class T>
__device__ __forceinline__ RawPiece<T> held_back(const RawPiece<T>& x) {
  constexpr int kWords = int(sizeof(x) / 4);
  int w[kWords];
  __builtin_memcpy(w, &x, sizeof(x));
#pragma unroll
  for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(w[i]));
  RawPiece<T> r;
  __builtin_memcpy(&r, w, sizeof(r));
  return r;
}

// Lists are made of what lanes hold without rounds that wait for one another: who is ahead of whom is counted for all at once.
struct Candidates {  // of a wave, in shared memory, in any order
  float v[kWave];
  int c[kWave];
};
// adds those of the lanes that have one; n: how many there are, of which those behind the 64th are lost
__device__ __forceinline__ void add_candidates(Candidates& s, int& n, bool one, float v, int c) {
  const uint64_t ones = __ballot(one);
  if (!ones) return;
  const int at = n + int(__builtin_amdgcn_mbcnt_hi(uint32_t(ones >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(ones), 0)));
  if (one && at < kWave) s.v[at] = v, s.c[at] = c;
  n += __popcll(ones);
}
// no more than the k-th largest of the lanes' values: the k-th of the best of every four lanes, or of all lanes' (-inf where fewer than k are above it)
__device__ __forceinline__ float kth_of_lanes(float v, int k) {
  int ahead = 0;
  if (k <= 6) {
    v = fmaxf(v, paired<0xB1>(v));
    v = fmaxf(v, paired<0x4E>(v));
#pragma unroll
    for (int i = 0; i < kWave; i += 4) ahead += lane_value(v, i) > v ? 1 : 0;
  } else {
#pragma unroll
    for (int i = 0; i < kWave; ++i) ahead += lane_value(v, i) > v ? 1 : 0;
  }
  return -lanes_all<kWave, Over::kMax>(ahead < k ? -v : kLow);
}
// the next lower number of a type (of one that is above -inf)
__device__ __forceinline__ float lower(float x) {
  const int b = __float_as_int(x + 0.f);  // no -0
  return __int_as_float(b > 0 ? b - 1 : (b == 0 ? int(0x80000001u) : b + 1));
}
__device__ __forceinline__ half_t lower(half_t x) {
  uint16_t b;
  x = x + half_t(0);
  __builtin_memcpy(&b, &x, 2);
  b = uint16_t(b == 0 ? 0x8001 : (b & 0x8000 ? b + 1 : b - 1));
  __builtin_memcpy(&x, &b, 2);
  return x;
}
// a number that rises with the score and falls with the class (no two are the same)
__device__ __forceinline__ uint64_t place_of(float v, int c) {
  const uint32_t b = uint32_t(__float_as_int(v + 0.f));
  return uint64_t(b ^ (b >> 31 ? 0xffffffffu : 0x80000000u)) << 32 | uint32_t(~c);
}
// the candidates of the first `count` lanes, falling, classes rising among equals (no two have the same class)
__device__ __forceinline__ Best sorted(float v, int c, int count, Candidates& s) {
  const int lane = threadIdx.x & (kWave - 1);
  const uint64_t mine = place_of(v, c);
  int ahead = 0;
  for (int i = 0; i < count; ++i) {
    const uint32_t hi = uint32_t(__builtin_amdgcn_readlane(int(mine >> 32), i)), lo = uint32_t(__builtin_amdgcn_readlane(int(mine), i));
    ahead += (uint64_t(hi) << 32 | lo) > mine ? 1 : 0;
  }
  if (lane < count) s.v[ahead] = v, s.c[ahead] = c;
  wave_sync();
  Best r;
  if (lane < count) r.v = s.v[lane], r.c = s.c[lane];
  wave_sync();
  return r;
}
__device__ __forceinline__ Best sorted(Candidates& s, int count) {  // at most 64
  const int lane = threadIdx.x & (kWave - 1);
  wave_sync();
  const float v = lane < count ? s.v[lane] : kLow;
  const int c = lane < count ? s.c[lane] : -1;
  wave_sync();
  return sorted(v, c, count, s);
}

// Takes those of a wave's classes c0 + 512 i + 8 lane + j (i < N, j < 8, scores x, -inf where there is none) that are among the best k; `least`, the k-th so
// far.  A wave comes by its classes in rising order, so a score that equals the k-th is behind it.  What is better becomes candidates, of many no more than
// what is as good as the k-th of the lanes' best.  Where there are too many all the same (equal scores), pieces are gone through in their order.
template <class T, int N>
__device__ __forceinline__ void take_best(Best& best, float& least, int k, const RawPiece<T> (&x)[N], const float (&top)[N], int c0, Candidates& s) {
  const int lane = threadIdx.x & (kWave - 1);
  float t = top[0];
#pragma unroll
  for (int i = 1; i < N; ++i) t = fmaxf(t, top[i]);
  const uint64_t better = __ballot(t > least);
  if (!better) return;
  float bound = kLow;
  if (__popcll(better) > k) bound = kth_of_lanes(t > least ? t : kLow, k);
  int n = 0;
  add_candidates(s, n, lane < k && best.c >= 0, best.v, best.c);
  const T above = bound > least ? lower(T(bound)) : T(least);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (!__ballot(top[i] > float(above))) continue;
    const RawPiece<T> p = held_back(x[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) add_candidates(s, n, p.v[j] > above, float(p.v[j]), c0 + 8 * kWave * i + 8 * lane + j);
  }
  if (n <= kWave) {
    best = sorted(s, n);
    least = lane_value(best.v, k - 1);
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint64_t left = __ballot(top[i] > least);
    while (left) {
      const int from = __builtin_ctzll(left);
      const RawPiece<T> p = held_back(x[i]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = lane_value(float(p.v[j]), from);
        if (!(v > least)) continue;  // (the same on all lanes)
        const int at = __popcll(__ballot(best.v >= v)), c = c0 + 8 * kWave * i + 8 * from + j;
        const float pv = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(best.v), 0x138, 0xf, 0xf, false));  // of the lane before: wave_shr:1
        const int pc = __builtin_amdgcn_update_dpp(0, best.c, 0x138, 0xf, 0xf, false);
        if (lane > at) best.v = pv, best.c = pc;
        if (lane == at) best.v = v, best.c = c;
        least = lane_value(best.v, k - 1);
      }
      left &= left - 1;
      left &= __ballot(top[i] > least);
    }
  }
}

struct ScoreArgs {
  int64_t n;
  int C, k;
  const void* logits;
  int64_t ld, inside;  // inside: elements from the first of the logits to the last
  const int* labels;
  float *logprob, *stats, *entropy, *top;
  int* top_class;
  // several workgroups to a row: what each of them has found
  int splits;
  int span;          // classes of a part
  float* part;       // [n][splits][3]
  float* part_top;   // [n][splits][k]
  int* part_class;
};

// The outputs of a row but for the alternatives, by one lane; at: the score of its label.
template <class T>
__device__ __forceinline__ void store_row(const ScoreArgs& a, int64_t row, const Mass<T>& mass, int y, float at) {
  const RowStats st = stats_of(mass);
  if (a.stats) a.stats[2 * row] = st.m, a.stats[2 * row + 1] = st.l;
  if (a.entropy) a.entropy[row] = entropy_of(mass);
  if (a.logprob) a.logprob[row] = uint32_t(y) < uint32_t(a.C) ? st.log_p(at) : 0.f;
}
template <class T>
__device__ __forceinline__ float score_at(const ScoreArgs& a, int64_t row, int y) {
  return uint32_t(y) < uint32_t(a.C) ? float(static_cast<const T*>(a.logits)[row * a.ld + y]) : 0.f;
}

// The alternatives of a row, by a wave.  Where fewer than k scores are above -inf, the first of the other classes fill up.
template <class T>
__device__ __forceinline__ void store_best(const ScoreArgs& a, int64_t row, const Mass<T>& mass, const Best& best) {
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

// W lists of k, in shared memory, become one, by a wave: an entry's place is the number of those before it, in its own list and, found by halving, in the others
template <int W>
__device__ __forceinline__ Best joined_lists(const float (&v)[W][kMostTop], const int (&c)[W][kMostTop], int k, Candidates& s) {
  const int lane = threadIdx.x & (kWave - 1);
  s.v[lane] = kLow, s.c[lane] = -1;
  wave_sync();
  for (int q = lane; q < W * k; q += kWave) {
    const int w = q / k, p = q - w * k;
    if (c[w][p] < 0) continue;
    const uint64_t mine = place_of(v[w][p], c[w][p]);
    int lo[W - 1] = {}, at = p;
    for (int step = kMostTop / 2; step > 0; step >>= 1)
#pragma unroll
      for (int o = 0; o < W - 1; ++o) {
        const int u = o < w ? o : o + 1, x = lo[o] + step - 1;
        if (x < k && place_of(v[u][x], c[u][x]) > mine) lo[o] += step;
      }
#pragma unroll
    for (int o = 0; o < W - 1; ++o) {
      const int u = o < w ? o : o + 1;
      at += lo[o] + (lo[o] < k && place_of(v[u][lo[o]], c[u][lo[o]]) > mine ? 1 : 0);
    }
    if (at < k) s.v[at] = v[w][p], s.c[at] = c[w][p];
  }
  wave_sync();
  return Best{s.v[lane], s.c[lane]};
}

// lists of falling scores, one for each lane (n entries, class -1: an empty one), become one; among equals the lowest class comes first
template <class Entry>
__device__ __forceinline__ Best merge_lists(int k, int n, Entry&& entry) {
  const int lane = threadIdx.x & (kWave - 1);
  Best out, mine;
  int p = 0;
  if (n > 0) mine = entry(0);
  for (int r = 0; r < k; ++r) {
    const float v = lanes_all<kWave, Over::kMax>(mine.v);
    const uint64_t have = __ballot(mine.c >= 0 && mine.v == v);
    if (!have) break;
    int c;
    if (have & (have - 1)) c = lanes_all<kWave, Over::kMin>(mine.c >= 0 && mine.v == v ? mine.c : 0x7fffffff);
    else c = __builtin_amdgcn_readlane(mine.c, __builtin_ctzll(have));
    if (lane == r) out.v = v, out.c = c;
    if (mine.c == c) {
      ++p;
      mine = Best{};
      if (p < n) mine = entry(p);
    }
  }
  return out;
}

// ---- the best k of a row that a group of lanes holds, a piece each
// Every lane puts its eight in order once, then the row's best is the best of the lanes' first, k times.  us, with rounds that looked for score and class
// among all that is left / this: 212 828 rows of 247 (fp16) best five 137 / 82, twenty 461 / 135; 19 rows of 16, all sixteen 14 / 4.3.
// A score and its class.  NaN counts as -inf, and what is behind the row's end comes after both.
template <class T>
struct Place;
template <>
struct Place<half_t> {  // in one number, that rises with the score and falls with the class (less than 2^16)
  int key;
  Place() = default;
  __device__ __forceinline__ Place(half_t x, int c, bool there) {
    x = (x > half_t(kLow) ? x : half_t(kLow)) + half_t(0);  // no -0
    int16_t b;
    __builtin_memcpy(&b, &x, 2);
    key = there ? int(uint32_t(b >= 0 ? b : b ^ 0x7fff) << 16) | (0xffff - c) : int(0x80000000u);
  }
  static __device__ __forceinline__ void order(Place (&e)[8]) {
    constexpr int kPairs[19][2] = {{0, 1}, {2, 3}, {4, 5}, {6, 7}, {0, 2}, {1, 3}, {4, 6}, {5, 7}, {1, 2}, {5, 6},
                                   {0, 4}, {1, 5}, {2, 6}, {3, 7}, {2, 4}, {3, 5}, {1, 2}, {3, 4}, {5, 6}};
#pragma unroll
    for (int q = 0; q < 19; ++q) {
      const int x = e[kPairs[q][0]].key, y = e[kPairs[q][1]].key;
      e[kPairs[q][0]].key = max(x, y);
      e[kPairs[q][1]].key = min(x, y);
    }
  }
  template <int L>
  __device__ __forceinline__ bool best_of_lanes() const { return lanes_all<L, Over::kMax>(key) == key; }
  __device__ __forceinline__ float score() const {
    const int16_t s = int16_t(key >> 16), b = s >= 0 ? s : s ^ 0x7fff;
    half_t x;
    __builtin_memcpy(&x, &b, 2);
    return float(x);
  }
  __device__ __forceinline__ int cls() const { return 0xffff - (key & 0xffff); }
};
template <>
struct Place<float> {
  float v;
  int c;  // -1: none
  Place() = default;
  __device__ __forceinline__ Place(float x, int cls, bool there) : v(there && x > kLow ? x : kLow), c(there ? cls : -1) {}
  static __device__ __forceinline__ void order(Place (&e)[8]) {  // neighbours only, so that equal ones stay in the order of their classes
#pragma unroll
    for (int q = 0; q < 8; ++q)
#pragma unroll
      for (int j = q & 1; j + 1 < 8; j += 2) {
        const Place x = e[j], y = e[j + 1];
        const bool swap = y.v > x.v;
        e[j] = swap ? y : x;
        e[j + 1] = swap ? x : y;
      }
  }
  template <int L>
  __device__ __forceinline__ bool best_of_lanes() const {  // of equal ones the first lane's, whose classes are lower
    const int lane = threadIdx.x & (kWave - 1);
    const float m = lanes_all<L, Over::kMax>(v);
    const uint64_t those = __ballot(c >= 0 && v == m) >> (lane & ~(L - 1));
    return __builtin_ctzll(those) == (lane & (L - 1));
  }
  __device__ __forceinline__ float score() const { return v; }
  __device__ __forceinline__ int cls() const { return c; }
};

// Rows of up to 512 classes: L lanes hold a row, N pieces each.  What a row costs beside its classes (reductions, logarithm, stores) is a wave's for all of its
// 64 / L rows at once: 262 144 rows of 512, 64 lanes with a piece / 16 with four, 78 / 51 us.
template <class T, int L, int N, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(kBlock) void logprob_group_kernel(ScoreArgs a) {
  const int64_t i = (int64_t(blockIdx.x) * kBlock + threadIdx.x) / L, row = i < a.n ? i : a.n - 1;
  const int l = threadIdx.x % L;
  const bool writes = i < a.n && l == 0;
  const int y = a.labels ? a.labels[row] : -1;
  RawPiece<T> p[N];
  float top[N], m = Mass<T>::kNone, at = kLow;
#pragma unroll
  for (int q = 0; q < N; ++q) p[q] = load_classes(static_cast<const T*>(a.logits) + row * a.ld, 8 * (q * L + l), a.C, a.inside - row * a.ld);
#pragma unroll
  for (int q = 0; q < N; ++q) {
    top[q] = piece_max(p[q]);
    m = fmaxf(m, top[q]);
#pragma unroll
    for (int j = 0; j < 8; ++j) at = y == 8 * (q * L + l) + j ? float(p[q].v[j]) : at;
  }
  Mass<T> mass{lanes_all<L, Over::kMax>(m), 0.f, 0.f};
  at = lanes_all<L, Over::kMax>(at);
  add_pieces<ENTROPY>(mass, p, top);
  mass.s = lanes_all<L, Over::kSum>(mass.s);
  if (ENTROPY) mass.t = lanes_all<L, Over::kSum>(mass.t);
  if (writes) store_row(a, row, mass, y, at);
  if (!TOP) return;
  static_assert(!TOP || N == 1, "a piece each");
  constexpr int kRows = kWave / L, kMost = 8 * L < kMostTop ? 8 * L : kMostTop;
  __shared__ Place<T> s_best[TOP ? kWavesPerBlock : 1][TOP ? kRows * kMost : 1];
  __shared__ RowStats s_stats[TOP ? kWavesPerBlock : 1][TOP ? kRows : 1];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, r = lane / L;
  Place<T> e[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) e[j] = Place<T>(p[0].v[j], 8 * l + j, 8 * l + j < a.C);
  Place<T>::order(e);
  const Place<T> none(T(0), 0, false);
  for (int k = 0; k < a.k; ++k) {
    if (!e[0].template best_of_lanes<L>()) continue;
    s_best[wave][r * a.k + k] = e[0];
#pragma unroll
    for (int j = 0; j + 1 < 8; ++j) e[j] = e[j + 1];
    e[7] = none;
  }
  if (l == 0) s_stats[wave][r] = stats_of(mass);
  wave_sync();
  // the wave's rows lie one behind the other
  const int64_t row0 = i - r;
  const int count = int(a.n - row0 < kRows ? a.n - row0 : kRows) * a.k;
  for (int q = lane; q < count; q += kWave) {
    const Place<T> best = s_best[wave][q];
    a.top[row0 * a.k + q] = s_stats[wave][uint32_t(q) / uint32_t(a.k)].log_p(best.score());
    a.top_class[row0 * a.k + q] = best.cls();
  }
}

// Few alternatives of few classes, many rows: a lane takes a row by itself, with no reduction across lanes.  The 64 rows of a wave come in whole pieces through
// LDS (rows of P pieces and a pad word, so that lanes that read their own rows meet on no bank).  us, lanes in groups / a lane a row, 233 000 rows of 41
// (fp16): the best one 18.5 / 11.2, five 22 / 18.3, eight 26.2 / 25.5, twenty 34 / 76; of 16 five 9.5 / 8.8, eight 11 / 15; without alternatives 8.8 / 8.3 and
// the gradient, which would go back that way, 9.9 / 12.5: not kept.
template <class T, int P>
struct LaneRows {
  static constexpr int kPitch = 8 * P + 4 / int(sizeof(T));  // elements
  T x[kWave][kPitch];
  // pieces f, f + 64, ... of the wave's rows, neighbours to neighbouring lanes: f(row, piece)
  template <class F>
  static __device__ __forceinline__ void each(F&& f) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int at = i * kWave + int(threadIdx.x & (kWave - 1));
      f(i, at / P, at % P);
    }
  }
  __device__ __forceinline__ void fetch(const T* logits, int64_t ld, int64_t row0, int64_t n, int C, int64_t inside) {
    RawPiece<T> p[P];
    each([&](int i, int r, int q) __attribute__((always_inline)) {
      const int64_t row = row0 + r < n ? row0 + r : n - 1;
      p[i] = load_classes(logits + row * ld, 8 * q, C, inside - row * ld);
    });
    each([&](int i, int r, int q) __attribute__((always_inline)) { put(r, q, p[i]); });
    wave_sync();
  }
  __device__ __forceinline__ void put(int r, int q, const RawPiece<T>& p) {
    constexpr int kWords = int(sizeof(RawPiece<T>) / 4);
    int w[kWords];
    __builtin_memcpy(w, &p, sizeof(w));
#pragma unroll
    for (int j = 0; j < kWords; ++j) reinterpret_cast<int*>(&x[r][8 * q])[j] = w[j];
  }
  __device__ __forceinline__ RawPiece<T> piece(int r, int q) const {
    constexpr int kWords = int(sizeof(RawPiece<T>) / 4);
    int w[kWords];
#pragma unroll
    for (int j = 0; j < kWords; ++j) w[j] = reinterpret_cast<const int*>(&x[r][8 * q])[j];
    RawPiece<T> p;
    __builtin_memcpy(&p, w, sizeof(w));
    return p;
  }
};
template <class T, int P, bool ENTROPY>
__global__ __launch_bounds__(kBlock) void logprob_lane_kernel(ScoreArgs a) {
  __shared__ __align__(16) LaneRows<T, P> s_rows[kWavesPerBlock];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int64_t row0 = (int64_t(blockIdx.x) * kWavesPerBlock + wave) * kWave, row = row0 + lane;
  if (row0 >= a.n) return;
  const int y = a.labels && row < a.n ? a.labels[row] : -1;
  LaneRows<T, P>& s = s_rows[wave];
  s.fetch(static_cast<const T*>(a.logits), a.ld, row0, a.n, a.C, a.inside);
  RawPiece<T> p[P];
  float top[P];
  Mass<T> mass = Mass<T>::none();
#pragma unroll
  for (int q = 0; q < P; ++q) {
    p[q] = s.piece(lane, q);
    top[q] = piece_max(p[q]);
    mass.m = fmaxf(mass.m, top[q]);
  }
  add_pieces<ENTROPY>(mass, p, top);
  if (row >= a.n) return;
  store_row(a, row, mass, y, float(s.x[lane][uint32_t(y) < uint32_t(a.C) ? y : 0]));
  // the best one that is left, k times; those that are not above -inf, in their order, once the others are out
  const RowStats st = stats_of(mass);
  uint64_t left = a.C == 64 ? ~uint64_t(0) : (uint64_t(1) << a.C) - 1;
  for (int k = 0; k < a.k; ++k) {
    float v = kLow;
    int c = -1;
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float e = float(p[q].v[j]);
        const bool better = e > v && (left >> (8 * q + j) & 1);
        v = better ? e : v;
        c = better ? 8 * q + j : c;
      }
    if (c < 0) c = __builtin_ctzll(left);
    left &= ~(uint64_t(1) << c);
    a.top[row * a.k + k] = mass.s == mass.s ? st.log_p(v) : NAN;
    a.top_class[row * a.k + k] = c;
  }
}

// Longer rows: W waves take one, or one of its `splits` parts, W = 4 a workgroup, W = 1 a wave by itself.  The waves take 4 KB in turn, the next ones on their way.
template <class T>
constexpr int kPieces = sizeof(T) == 2 ? 4 : 2;  // 64 bytes
template <class T>
constexpr int kStep = 8 * kWave * kPieces<T>;  // classes that a wave takes at a time
template <class T, int W, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(kBlock) void logprob_row_kernel(ScoreArgs a) {
  constexpr int N = kPieces<T>;
  __shared__ float s_mass[kWavesPerBlock][3], s_top[TOP ? kWavesPerBlock : 1][kMostTop];
  __shared__ int s_class[TOP ? kWavesPerBlock : 1][kMostTop];
  __shared__ Candidates s_found[TOP ? kWavesPerBlock : 1];
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int64_t unit = W == 1 ? int64_t(blockIdx.x) * kWavesPerBlock + wave : int64_t(blockIdx.x);
  if (W == 1 && unit >= a.n) return;
  const int64_t row = W == 1 ? unit : int64_t(blockIdx.x / unsigned(a.splits));
  const int split = W == 1 ? 0 : int(blockIdx.x % unsigned(a.splits));
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  const int64_t inside = a.inside - row * a.ld, first = W == 1 ? 0 : int64_t(split) * a.span;
  const int c1 = int(first + a.span < a.C ? first + a.span : a.C), c0 = int(first < a.C ? first : a.C) + (W == 1 ? 0 : wave * kStep<T>);
  const int y = a.labels ? a.labels[row] : -1;
  Mass<T> mass = Mass<T>::none();
  Best best;
  float least = kLow;
  RawPiece<T> next[N];
  auto fetch = [&](int c) __attribute__((always_inline)) {
    if (c + kStep<T> <= c1) {
#pragma unroll
      for (int i = 0; i < N; ++i) next[i] = load_raw(x + c + 8 * (i * kWave + lane));
    } else if (c < c1) {
#pragma unroll
      for (int i = 0; i < N; ++i) next[i] = load_classes(x, c + 8 * (i * kWave + lane), c1, inside);
    }
  };
  fetch(c0);
  for (int c = c0; c < c1; c += W * kStep<T>) {
    RawPiece<T> p[N];
    float top[N];
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = next[i];
    fetch(c + W * kStep<T>);
#pragma unroll
    for (int i = 0; i < N; ++i) top[i] = piece_max(p[i]);
    add_pieces<ENTROPY>(mass, p, top);
    if (TOP) take_best(best, least, a.k, p, top, c, s_found[wave]);
  }
  mass = lanes_mass<kWave>(mass);
  if (W > 1) {
    if (lane == 0) s_mass[wave][0] = mass.m, s_mass[wave][1] = mass.s, s_mass[wave][2] = mass.t;
    if (TOP && lane < a.k) s_top[wave][lane] = best.v, s_class[wave][lane] = best.c;
    __syncthreads();
    if (wave > 0) return;
    mass = Mass<T>::none();
    if (lane < W) mass = Mass<T>{s_mass[lane][0], s_mass[lane][1], s_mass[lane][2]};
    mass = lanes_mass<kWave>(mass);
    if constexpr (TOP && W > 1) best = joined_lists<W>(s_top, s_class, a.k, s_found[0]);
    if (a.splits > 1) {
      if (lane == 0) {
        float* const q = a.part + 3 * (row * a.splits + split);
        q[0] = mass.m, q[1] = mass.s, q[2] = mass.t;
      }
      if (TOP && lane < a.k) {
        a.part_top[(row * a.splits + split) * a.k + lane] = best.v;
        a.part_class[(row * a.splits + split) * a.k + lane] = best.c;
      }
      return;
    }
  }
  if (lane == 0) store_row(a, row, mass, y, score_at<T>(a, row, y));
  if (TOP) store_best(a, row, mass, best);
}

// the parts of a row, by a wave
template <class T>
__global__ __launch_bounds__(kWave) void logprob_join_kernel(ScoreArgs a) {
  const int lane = threadIdx.x;
  const int64_t row = blockIdx.x;
  const int y = a.labels ? a.labels[row] : -1;
  const float score = score_at<T>(a, row, y);
  Mass<T> mass = Mass<T>::none();
  if (lane < a.splits) {
    const float* const q = a.part + 3 * (row * a.splits + lane);
    mass = Mass<T>{q[0], q[1], q[2]};
  }
  mass = lanes_mass<kWave>(mass);
  if (lane == 0) store_row(a, row, mass, y, score);
  if (a.k == 0) return;
  const int64_t at = (row * a.splits + lane) * a.k;
  const auto entry = [&](int p) { return Best{a.part_top[at + p], a.part_class[at + p]}; };
  // what is as good as the k-th of the parts' best, or, of many equal scores, one by one
  __shared__ Candidates s_found;
  int n = 0;
  if (a.splits * a.k <= kWave) {
    Best mine;
    if (lane < a.splits * a.k) mine = Best{a.part_top[row * a.splits * a.k + lane], a.part_class[row * a.splits * a.k + lane]};
    add_candidates(s_found, n, mine.c >= 0, mine.v, mine.c);
  } else {
    Best next;
    if (lane < a.splits) next = entry(0);
    const float bound = kth_of_lanes(next.v, a.k);
    for (int p = 0; p < a.k; ++p) {
      const Best mine = next;
      next = Best{};
      if (lane < a.splits && p + 1 < a.k) next = entry(p + 1);
      const bool here = mine.c >= 0 && mine.v >= bound;
      if (!__ballot(here)) break;
      add_candidates(s_found, n, here, mine.v, mine.c);
    }
  }
  const Best best = n <= kWave ? sorted(s_found, n) : merge_lists(a.k, lane < a.splits ? a.k : 0, entry);
  store_best(a, row, mass, best);
}

// ---- the gradient: dx_c = g (1[c = y] - p_c) - h p_c (log p_c + entropy), p_c = exp((x_c - m) - L)
struct ScoreGradArgs {
  int64_t n;
  int C, chunks;
  const void* logits;
  int64_t ld, inside;
  const int* labels;
  const float *stats, *dlogprob, *entropy, *dentropy;
  void* dlogits;
  int64_t ldd;
};

// With e = 2^y (Mass) p is e times a factor of the row, and a class's gradient e times a line in y.
template <class T>
struct RowGrad {
  int y;
  float g, offset, slope, at0;
  template <bool ENTROPY>
  __device__ __forceinline__ float grad(float x, int c) const {
    const float z = Mass<T>::y(x, offset), e = exp2_of(z), v = e * (ENTROPY ? fmaf(bounded(z), slope, at0) : at0);
    return c == y ? v + g : v;
  }
};
template <class T, bool ENTROPY>
__device__ __forceinline__ RowGrad<T> row_grad(const ScoreGradArgs& a, int64_t row) {
  RowGrad<T> r{-1, 0.f, 0.f, 0.f, 0.f};
  if (a.labels) r.y = a.labels[row], r.g = a.dlogprob[row];
  const float m = a.stats[2 * row], ls = a.stats[2 * row + 1];
  const bool none = m == kLow;  // a row of -inf alone
  r.g = uint32_t(r.y) < uint32_t(a.C) && !none ? r.g : 0.f;
  r.offset = none ? 0.f : Mass<T>::offset(m);
  const float shift = none ? 0.f : kLn2 * Mass<T>::shift(m), p = none ? 0.f : expf(shift - ls);  // p is this times e, log p = ln2 y + shift - ls
  r.at0 = -r.g * p;
  if (ENTROPY) {
    const float above = a.dentropy[row], h = none ? 0.f : above * p;  // (loaded with the stats, not behind them: 4096 rows of 50 021 165 / 145 us)
    r.slope = -h * kLn2;
    r.at0 -= h * (a.entropy[row] + shift - ls);
  }
  return r;
}

// L lanes take a row (ONE), or 64 of them one of its chunks, N parts of V each.  A lane reads what it overwrites: the logits may be the output.
template <class T, int L, int N, int V, bool ENTROPY, bool ONE, bool PAST>
__global__ __launch_bounds__(kBlock) void logprob_grad_kernel(ScoreGradArgs a) {
  const int64_t unit = (int64_t(blockIdx.x) * kBlock + threadIdx.x) / L;
  const int64_t row = ONE ? unit : int64_t(uint32_t(unit) / uint32_t(a.chunks));
  if (row >= a.n) return;
  const int l = threadIdx.x % L, c0 = ONE ? 0 : int(uint32_t(unit) - uint32_t(row) * uint32_t(a.chunks)) * (V * L * N);
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  T* const dx = static_cast<T*>(a.dlogits) + row * a.ldd;
  const int64_t inside = a.inside - row * a.ld;
  typedef Part<T, V> P;
  P p[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int at = c0 + V * (i * L + l);
    if (at < a.C) p[i] = P::load(x + at, a.C - at, inside - at);
  }
  const RowGrad<T> of = row_grad<T, ENTROPY>(a, row);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int at = c0 + V * (i * L + l);
    if (at >= a.C) continue;
    float out[V];
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = of.template grad<ENTROPY>(float(p[i].v[j]), at + j);
    P::template store<PAST>(dx + at, a.C - at, out);
  }
}

constexpr int kGroupClasses = 8 * kWave;  // most classes that the lanes of a wave hold at once
static int group_lanes(int C, int pieces) { return std::min(kWave, pow2_at_least(int(ceil_div(C, 8 * pieces)))); }
// Pieces of a lane, more than one where rows fill the chip all the same.  us, 1 / 2 / 4: 233 000 rows of 41 (fp16) 10.2 / 8.4 / 8.8, their gradient 11.5 / 11.2
// / 13.3; 262 144 of 512 78 / 57 / 51, gradient 97 / 94 / 94; 100 000 of 200 18 / 12.8 / 13.6; fp32, 100 000 of 512 - / 34.8 / 36.8, gradient - / 77.7 / 81.9.
static int row_pieces(int64_t n, int C, bool wide) {
  if (C > kGroupClasses) return C <= 2 * kGroupClasses ? 2 : 4;
  if (C <= 8 || n * group_lanes(C, 1) < int64_t(1) << 20) return 1;
  return wide && C > 256 ? 4 : 2;
}
template <class Call>
static void with_pieces(int pieces, Call&& call) {
  if (pieces == 1) call(std::integral_constant<int, 1>());
  else if (pieces == 2) call(std::integral_constant<int, 2>());
  else call(std::integral_constant<int, 4>());
}
constexpr int kWaveClasses = 4096;        // up to so many, a row is a wave's where there are rows enough
static bool by_waves(int64_t n, int C) { return C <= kWaveClasses && n >= 4096; }
// What a group of lanes holds: up to 512 classes, 2048 without alternatives (rows and their gradient, by waves / groups, us, fp16: 200 000 of 520 172 / 155, of 600
// 176 / 158, of 1000 233 / 216, 100 000 of 1500 170 / 174, of 2000 204 / 203, 5000 of 1000 10.3 / 9.4; fp32, 100 000 of 520 112 / 112, of 2000 407 / 408). Many alternatives of rows that take all lanes of a wave are found sooner among candidates (us, by groups / by waves, 100 000 rows of 500, fp32:
// best twenty 171 / 109, five 85 / 77; of 512, fp16, 127 / 122, 77 / 83; 400, best one 60 / 75; 212 828 of 247, two to a wave, best twenty 132 / 274).
constexpr int kGroupTop = 8;
static bool by_groups(int64_t n, int C, int k) {
  if (k > kGroupTop && C > kGroupClasses / 2 && by_waves(n, C)) return false;
  return C <= (k > 0 ? 1 : 4) * kGroupClasses;
}
// Workgroups of a row: as many as make 1024 in all, 64 at most, for no less than 2048 classes each.  Their waves take a part's classes by kStep in turn, so of a part
// of 2048 one wave of the four has classes in fp16 and two in fp32: one row of 100 003 is 49 workgroups (best eight 10.3 us in fp16, 10.4 in fp32; none 6.5, 6.3),
// rows of 513 to 2048 with alternatives one each where they are fewer than 4096 (best five of 1000: 100 rows 6.2 us, 1000 7.1, 4000 14.6).
static int splits_of(int64_t n, int C, int k) {
  if (by_groups(n, C, k) || by_waves(n, C)) return 1;
  const int64_t most = ceil_div(C, int64_t(8) * kWave * kWavesPerBlock), want = ceil_div(1024, n), s = most < want ? most : want;
  return int(s < 1 ? 1 : (s > kMostSplits ? kMostSplits : s));
}
static size_t up256(size_t n) { return (n + 255) / 256 * 256; }

template <class Call>
static void with_flags(bool x, bool y, Call&& call) {
  const std::true_type yes;
  const std::false_type no;
  if (x) y ? call(yes, yes) : call(yes, no);
  else y ? call(no, yes) : call(no, no);
}
// a lane to a row, for its alternatives, where a row has more than one piece and the rows fill the chip
constexpr int kLaneClasses = 64, kLaneTop = 5;
constexpr int64_t kLaneRows = 65536;
static bool by_lanes(int64_t n, int C, int k) { return k > 0 && k <= kLaneTop && C > 8 && C <= kLaneClasses && n >= kLaneRows; }
template <class Call>
static void with_lane_pieces(int C, Call&& call) {
  switch ((C + 7) / 8) {
    case 2: return call(std::integral_constant<int, 2>());
    case 3: return call(std::integral_constant<int, 3>());
    case 4: return call(std::integral_constant<int, 4>());
    case 5: return call(std::integral_constant<int, 5>());
    case 6: return call(std::integral_constant<int, 6>());
    case 7: return call(std::integral_constant<int, 7>());
    default: return call(std::integral_constant<int, 8>());
  }
}
template <class Call>
static void with_group(int lanes, Call&& call) {
  switch (lanes) {
    case 1: return call(std::integral_constant<int, 1>());
    case 2: return call(std::integral_constant<int, 2>());
    case 4: return call(std::integral_constant<int, 4>());
    case 8: return call(std::integral_constant<int, 8>());
    case 16: return call(std::integral_constant<int, 16>());
    case 32: return call(std::integral_constant<int, 32>());
    default: return call(std::integral_constant<int, 64>());
  }
}

template <class T>
static hgnn_status logprob(ScoreArgs& a, hipStream_t s) {
  const char* who = "hgnn_logprob";
  const bool group = by_groups(a.n, a.C, a.k), waves = by_waves(a.n, a.C);
  const int N = a.k > 0 ? 1 : row_pieces(a.n, a.C, sizeof(T) == 2), L = group_lanes(a.C, N);
  const bool lanes = by_lanes(a.n, a.C, a.k);
  const int64_t blocks = lanes ? ceil_div(a.n, kBlock) : group ? ceil_div(a.n * L, kBlock) : (waves ? ceil_div(a.n, kWavesPerBlock) : a.n * a.splits);
  HGNN_REQUIRE(blocks <= kMostBlocks, HGNN_EUNSUPPORTED, "%s: grid too large", who);
  const dim3 grid{unsigned(blocks)};
  a.span = waves ? a.C : int(ceil_div(ceil_div(a.C, a.splits), 8) * 8);
  with_flags(a.entropy != nullptr, a.k > 0, [&](auto entropy, auto top) {
    constexpr bool E = decltype(entropy)::value, K = decltype(top)::value;
    if (lanes) {
      with_lane_pieces(a.C, [&](auto pieces) { logprob_lane_kernel<T, decltype(pieces)::value, E><<<grid, kBlock, 0, s>>>(a); });
    } else if (group) {
      with_group(L, [&](auto width) {
        constexpr int W = decltype(width)::value;
        with_pieces(N, [&](auto pieces) { logprob_group_kernel<T, W, K ? 1 : decltype(pieces)::value, E, K><<<grid, kBlock, 0, s>>>(a); });
      });
    } else if (waves) {
      logprob_row_kernel<T, 1, E, K><<<grid, kBlock, 0, s>>>(a);
    } else {
      logprob_row_kernel<T, kWavesPerBlock, E, K><<<grid, kBlock, 0, s>>>(a);
    }
  });
  HGNN_LAUNCH_CHECK("logprob_lane_kernel, logprob_group_kernel or logprob_row_kernel");
  if (a.splits > 1) {
    logprob_join_kernel<T><<<dim3(unsigned(a.n)), kWave, 0, s>>>(a);
    HGNN_LAUNCH_CHECK("logprob_join_kernel");
  }
  return HGNN_OK;
}

template <class T>
static hgnn_status logprob_grad(ScoreGradArgs& a, hipStream_t s) {
  const bool group = a.C <= kGroupClasses;
  const int N = group ? row_pieces(a.n, a.C, false) : 1, L = group ? group_lanes(a.C, N) : kWave;
  constexpr int V = 16 / int(sizeof(T)), W = 4;  // of long rows: 16 bytes, four of them
  a.chunks = group ? 1 : int(ceil_div(a.C, V * kWave * W));
  // Long rows of large outputs are written past the caches, whether they are whole lines or not.  us, the log probabilities and this, through / past, 208 MB: fp16,
  // rows of 513 165 / 160, 520 152 / 151, 600 138 / 138, 777 126 / 121 (of a pitch of 784 128 / 122), 1000 116 / 108, 1500 119 / 114, 2000 126 / 101, 4000 126 / 99,
  // 16 001 133 / 110, 50 021 136 / 112; fp32, 520 120 / 112, 1001 126 / 101, 4000 124 / 98, 16 001 126 / 102.  Rows that a group of lanes holds go through: past
  // the caches those of 41 and 100 classes, whose ends share lines, took 28 for 19 and 214 for 159.
  const bool past = a.n * double(a.C) * sizeof(T) >= kPastBytes;
  HGNN_REQUIRE(double(a.n) * a.chunks * L <= double(kMostBlocks) * kBlock, HGNN_EUNSUPPORTED, "hgnn_logprob_grad: grid too large");
  const dim3 grid{unsigned(ceil_div(a.n * a.chunks * L, kBlock))};
  with_flags(a.dentropy != nullptr, group ? N == 2 : past, [&](auto entropy, auto flag) {
    constexpr bool E = decltype(entropy)::value, F = decltype(flag)::value;
    if (!group) logprob_grad_kernel<T, kWave, W, V, E, false, F><<<grid, kBlock, 0, s>>>(a);
    else with_group(L, [&](auto lanes) { logprob_grad_kernel<T, decltype(lanes)::value, F ? 2 : 1, 8, E, true, false><<<grid, kBlock, 0, s>>>(a); });
  });
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
  if (n <= 0) return p;
  const int splits = splits_of(n, C, k);
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
  HGNN_REQUIRE(C <= (1 << 30) && n <= (int64_t(1) << 40), HGNN_EUNSUPPORTED, "%s: C = %d above 2^30, or n = %lld above 2^40", who, C, static_cast<long long>(n));
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
  ScoreArgs a{n, C, k, logits, ld, extent_of(n, C, ld), labels, logprob_out, stats, entropy, top_logprob, top_class, splits_of(n, C, k), 0, w.part, w.part_top, w.part_class};
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
  HGNN_REQUIRE(C <= (1 << 30) && n <= (int64_t(1) << 40), HGNN_EUNSUPPORTED, "%s: C = %d above 2^30, or n = %lld above 2^40", who, C, static_cast<long long>(n));
  HGNN_REQUIRE((labels == nullptr) == (dlogprob == nullptr), HGNN_EINVAL, "%s: labels and dlogprob go together", who);
  HGNN_REQUIRE((dentropy == nullptr) || entropy, HGNN_EINVAL, "%s: dentropy without the entropy", who);
  if (n == 0) return HGNN_OK;
  HGNN_REQUIRE(logits && stats && dlogits, HGNN_EINVAL, "%s: NULL argument", who);
  HGNN_REQUIRE(logits != dlogits || ld == ldd, HGNN_EINVAL, "%s: in place with another leading dimension", who);
  HGNN_REQUIRE(aligned_to_type(logits, type) && aligned_to_type(dlogits, type) && aligned_to_type(labels, HGNN_F32) && aligned_to_type(stats, HGNN_F32) &&
                   aligned_to_type(dlogprob, HGNN_F32) && aligned_to_type(entropy, HGNN_F32) && aligned_to_type(dentropy, HGNN_F32),
               HGNN_EINVAL, "%s: an array that is not aligned to its type", who);
  ScoreGradArgs a{n, C, 1, logits, ld, extent_of(n, C, ld), labels, stats, dlogprob, entropy, dentropy, dlogits, ldd};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return type == HGNN_F16 ? logprob_grad<half_t>(a, s) : logprob_grad<float>(a, s);
}

}  // extern "C"
