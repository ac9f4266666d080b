// Dense products on the matrix cores for matrices of any size:  C[q][p] = sum_k Q(q, k) P(p, k), fp16 operands, fp32 sums, and an epilogue that takes the
// sums out of the registers.  Used by the gated projection (gated.hip) and the orthogonal updates (orthogonalize.hip).
//
// An operand lies with the contraction along its rows ([items][k], "rows") or across them ([k][items], "columns").  Both come into LDS by loads that write LDS
// directly, a kilobyte an instruction, 16 bytes a lane, 128 consecutive bytes of eight rows, a ring of stages ahead of the products, so that no register and no
// instruction of a lane carries them; lanes choose WHICH 16 bytes they ask for, such that the reads behind meet on no bank:
//  - rows: 64 steps of 8 items; piece u of item i (of 16) stands at place u ^ (i / 2), and ds_read_b128 gives a lane eight steps of an item (it serves lanes 0-3 and
//    12-15 of 16 together with 4-11 of the next 16);
//  - columns: 64 items of 8 steps; piece u of step r stands at place u ^ turn(r), and ds_read_b64_tr_b16 gives a lane four steps of an item.
// Values that are two fp16 numbers each lie as 32 high parts and 32 low parts in turn, so that the same 128 bytes are 32 steps (items) of both.
// (With 64 bytes of 16 rows an instruction, at pitches that are multiples of 4 KB, requests met on the L2's channels: 8192 x 16384 x 2048 592 us.)
// What is behind the contraction's end is asked for at a place that holds zeros; where the end lies inside a piece, the rest of the piece is cleared in LDS
// (the bytes there are the caller's padding and may be NaN).  Items that do not exist are asked for at one that does, in rows at the last, in columns at the tile's first
// eight: they meet only results that are not stored.
//
// v_mfma_f32_16x16x32_f16 with P as its first operand: a lane has four consecutive p of one q.  A wave's block of sums decides how often an operand is read
// from LDS, and that is what bounds the large shape (256 x 256: 8 waves of 128 x 64, (128 + 64) 64 bytes a step for 32 products of 16 cycles).
// Of 8192 rows, 2048 and 2 x 8192 features, 550 Gflop each, us at their fastest and in the middle: pairs with dY read and D written 554 / 599 (990 / 920 Tflop/s; the
// forward, which writes a fourth of that, 462), the sum of two segments 441 / 483 (1250 / 1140), X^T D 474 / 516 (1160 / 1070); two parts, 4096 x 4096 x 4096 at three
// products each, 343 / 358 (1200 / 1150).  A library's product reaches 1170 to 1510
// at such sizes.  The matrix units are busy for 46 to 61 % of the cycles, and the clock falls to 1.83 GHz under them.
#pragma once

#include <algorithm>
#include <type_traits>

#include "common.h"

namespace hgnn {

typedef float float4_t __attribute__((ext_vector_type(4)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef short short8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) short4_t lds_short4_t;

// Two operands each where the kernel takes two: of P for two results at once (kTwo), the second segment of the contraction (kSegments).  kSplit: values of two
// parts, Q P = Qhi Phi + Qhi Plo + Qlo Phi; its contraction is a multiple of 32 and its items are, too.
enum ProductKind { kOne, kTwo, kSegments, kSplit };

struct ProductArgs {
  const half_t *Q0, *Q1, *P0, *P1;
  int64_t ldq, ldp;
  int64_t nq, np;   // items
  int64_t K;        // of a segment
  int64_t part;     // contraction steps of a workgroup (blocks beyond the first take the next ones); a multiple of 64 (kSplit: 32), or K where there is one part
  int32_t tiles;    // of C, lines of tiles_p of them
  int32_t lines, tiles_p;
  int32_t parts;
  int32_t lower;    // square C of square tiles: those on and below the diagonal alone
  int32_t first, some;  // the first tile of this launch, and how many (0: all)
};

static __device__ const uint4 g_product_zero = {0, 0, 0, 0};

template <int WQ_, int WP_, int TQ_, int TP_, ProductKind KIND_, bool QCOL_, bool PCOL_, int STAGES_>
struct ProductShape {
  static constexpr int WQ = WQ_, WP = WP_, TQ = TQ_, TP = TP_, kStages = STAGES_;
  static constexpr ProductKind KIND = KIND_;
  static constexpr bool QCOL = QCOL_, PCOL = PCOL_;
  static constexpr int kWaves = WQ * WP, kThreads = kWaves * kWave;
  static constexpr int BQ = 16 * TQ * WQ, BP = 16 * TP * WP;
  static constexpr bool SPLIT = KIND == kSplit;
  static constexpr int NP = KIND == kTwo ? 2 : 1, NR = NP;        // operands of P in LDS, results
  static constexpr int kStep = SPLIT ? 32 : 64, kSubs = kStep / 32;  // contraction of a stage, instructions along it
  static constexpr int CQ = BQ / 8, CP = NP * BP / 8;              // kilobytes of a stage
  static constexpr int JQ = CQ / kWaves, JP = CP / kWaves, J = JQ + JP;
  static constexpr int kStageBytes = (CQ + CP) * 1024;
  static constexpr int kLds = kStageBytes * kStages;
  static_assert(CQ % kWaves == 0 && CP % kWaves == 0, "whole kilobytes of each operand to every wave");
  static_assert((!QCOL || BQ % 64 == 0) && (!PCOL || BP % 64 == 0), "panels of 64 items");
  static_assert(kLds <= 160 * 1024, "LDS");
};

// place of 16 bytes of step r (0..31) among the eight of 64 items
__device__ __forceinline__ int product_turn(int r) { return 2 * ((r >> 1) & 1) | 4 * ((r >> 3) & 1); }

// 16 bytes a lane from base (uniform) + off to LDS at `to` (uniform) + 16 * lane.  Written out, because behind the builtin the compiler waits for all of them before
// every read of LDS; what it does not know of is waited for by product_wait.  (Nothing else in these kernels uses m0.)
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t off, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %1" ::"s"(to), "s"(base), "v"(off) : "memory");
}
__device__ __forceinline__ void load_to_lds(const char* src, uint32_t to) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(src) : "memory");
}
// at most N of this wave's loads to LDS are left in flight, its reads of LDS have ended, and so have those of all waves
template <int N>
__device__ __forceinline__ void product_wait() {
  static_assert(N < 64, "vmcnt");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// One operand's kilobytes that a wave brings in: where they begin is uniform and moves with the steps, a lane's place behind it stays.
template <int N, bool COL>
struct ProductLoads {
  const char* base[N];
  uint32_t off[N];
  int k[N];  // step of the lane's piece inside 32
  int64_t inc;
};
template <int N, bool COL, bool SPLIT, int WAVES>
__device__ __forceinline__ void product_loads(ProductLoads<N, COL>& s, const half_t* first, const half_t* second, int64_t ld, int64_t item0, int64_t items, int64_t k0, int wave,
                                              int lane, int half) {
  constexpr int kStep = SPLIT ? 32 : 64, kParts = SPLIT ? 2 : 1;
  s.inc = (COL ? kStep * ld : 64) * int64_t(sizeof(half_t));
#pragma unroll
  for (int j = 0; j < N; ++j) {
    int c = wave + j * WAVES;
    const half_t* from = first;
    if (c >= half) c -= half, from = second;
    if (COL) {
      const int r = 8 * (c % (kStep / 8)) + (lane >> 3), u = (lane & 7) ^ product_turn(r), item = 64 * (c / (kStep / 8)) + 8 * u;
      s.k[j] = r;
      s.base[j] = reinterpret_cast<const char*>(from + k0 * ld + item0 * kParts);
      s.off[j] = uint32_t(r * uint32_t(ld) + (item0 * kParts + item < items * kParts ? item : 0)) * 2u;
    } else {
      const int n = 8 * (c & 1) + (lane >> 3), u = (lane & 7) ^ (n >> 1), item = int(min(int64_t(8 * c + (lane >> 3)), items - 1 - item0));
      s.k[j] = SPLIT ? 0 : 8 * u;
      s.base[j] = reinterpret_cast<const char*>(from + item0 * ld + k0 * kParts);
      s.off[j] = (uint32_t(item) * uint32_t(ld) + 8 * u) * 2u;
    }
  }
}

// where tile number t of C lies: groups of kGroup lines of tiles, walked along the lines' items, so that workgroups that run together share operands
__device__ __forceinline__ void product_tile(const ProductArgs& a, uint32_t t, uint32_t& tq, uint32_t& tp) {
  if (a.lower) {  // t = tq (tq + 1) / 2 + tp
    uint32_t r = uint32_t((sqrtf(8.f * float(t) + 1.f) - 1.f) * 0.5f);
    while (r * (r + 1) / 2 > t) --r;
    while ((r + 1) * (r + 2) / 2 <= t) ++r;
    tq = r, tp = t - r * (r + 1) / 2;
    return;
  }
  constexpr uint32_t kGroup = 8;
  const uint32_t per = kGroup * uint32_t(a.tiles_p), g = t / per, in = t - g * per, rows = min(kGroup, uint32_t(a.lines) - g * kGroup);
  tp = in / rows;
  tq = g * kGroup + (in - tp * rows);
}

// Where a lane reads its share of the T fragments (16 items of 32 steps) of a wave that begin with number f0; h: the stage's first or second 32 steps, or the high or
// low parts.
template <bool COL, bool SPLIT, int T>
struct ProductReads {
  static constexpr int A = !COL ? 2 : SPLIT || T >= 4 ? 4 : T;
  int at[A];
  __device__ __forceinline__ ProductReads(int f0, int lane) {
    const int i = lane & 15, qq = lane >> 4, r = 8 * qq + (i >> 2);
#pragma unroll
    for (int t = 0; t < A; ++t) {
      if (!COL) {
        at[t] = f0 * 2048 + i * 128 + ((4 * t + qq) ^ (i >> 1)) * 16;
      } else {
        const int f = f0 + t, place = SPLIT ? t : f & 3;  // of 16 items among the 64 (32 and their low parts)
        at[t] = (SPLIT ? (f0 >> 1) * 4096 : (f >> 2) * 8192) + r * 128 + (((2 * place + ((i & 3) >> 1)) ^ product_turn(r)) * 16) + (i & 1) * 8;
      }
    }
  }
  __device__ __forceinline__ half8_t get(const unsigned char* tile, int t, int h) const {
    if constexpr (!COL) {
      return *reinterpret_cast<const half8_t*>(tile + at[h] + t * 2048);
    } else {
      const unsigned char* p = tile + (SPLIT ? at[2 * h + t % 2] + (t / 2) * 4096 : at[t % A] + (t / 4) * 8192 + h * 4096);
      const short4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t*)p);
      const short4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t*)(p + 512));
      return __builtin_bit_cast(half8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
  }
};

template <class S, class Epilogue>
__global__ __launch_bounds__(S::kThreads, 2) void product_kernel(ProductArgs a, Epilogue epilogue) {
  extern __shared__ __align__(1024) unsigned char lds[];
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int i = lane & 15, qq = lane >> 4;
  // consecutive workgroups go to the XCDs in turn: each takes a run of tiles of its own
  const uint32_t all = gridDim.x, id = blockIdx.x, x = id & 7, more = all & 7;
  const uint32_t work = x * (all >> 3) + min(x, more) + (id >> 3);
  const int64_t part = __builtin_amdgcn_readfirstlane(int(a.parts == 1 ? 0 : work / uint32_t(a.tiles)));
  uint32_t tq, tp;
  product_tile(a, uint32_t(a.first) + work - uint32_t(part) * uint32_t(a.tiles), tq, tp);
  // (the divisions go through vector registers: back to scalar ones, which the loads to LDS take their places from)
  const int64_t q0 = int64_t(__builtin_amdgcn_readfirstlane(int(tq))) * S::BQ, p0 = int64_t(__builtin_amdgcn_readfirstlane(int(tp))) * S::BP;
  const int64_t k_begin = part * a.part, k_end = min(a.K, k_begin + a.part), count = k_end - k_begin;  // of a segment
  const int per = int((count + S::kStep - 1) / S::kStep), steps = S::KIND == kSegments ? 2 * per : per;

  ProductLoads<S::JQ, S::QCOL> lq;
  ProductLoads<S::JP, S::PCOL> lp;
  // steps of S::kStep
  const auto start = [&](bool second) __attribute__((always_inline)) {
    product_loads<S::JQ, S::QCOL, S::SPLIT, S::kWaves>(lq, second ? a.Q1 : a.Q0, a.Q1, a.ldq, q0, a.nq, k_begin, wave, lane, S::BQ / 8);
    product_loads<S::JP, S::PCOL, S::SPLIT, S::kWaves>(lp, second ? a.P1 : a.P0, a.P1, a.ldp, p0, a.np, k_begin, wave, lane, S::BP / 8);
  };
  start(false);
  const char* const zero = reinterpret_cast<const char*>(&g_product_zero);
  const uint32_t lds0 = uint32_t(uintptr_t((__attribute__((address_space(3))) unsigned char*)lds));
  int asked = 0, in_segment = 0;
  uint32_t to = lds0 + wave * 1024;
  const auto ask = [&]() __attribute__((always_inline)) {
    if (S::KIND == kSegments && in_segment == per) in_segment = 0, start(true);
    const int left = int(min(count - int64_t(in_segment) * S::kStep, int64_t(S::kStep)));
    if (S::SPLIT || left == S::kStep) {  // uniform
#pragma unroll
      for (int j = 0; j < S::JQ; ++j) load_to_lds(lq.base[j], lq.off[j], to + j * S::kWaves * 1024);
#pragma unroll
      for (int j = 0; j < S::JP; ++j) load_to_lds(lp.base[j], lp.off[j], to + (S::JQ + j) * S::kWaves * 1024);
    } else {
#pragma unroll
      for (int j = 0; j < S::JQ; ++j) load_to_lds(lq.k[j] < left ? lq.base[j] + lq.off[j] : zero, to + j * S::kWaves * 1024);
#pragma unroll
      for (int j = 0; j < S::JP; ++j) load_to_lds(lp.k[j] < left ? lp.base[j] + lp.off[j] : zero, to + (S::JQ + j) * S::kWaves * 1024);
    }
#pragma unroll
    for (int j = 0; j < S::JQ; ++j) lq.base[j] += lq.inc;
#pragma unroll
    for (int j = 0; j < S::JP; ++j) lp.base[j] += lp.inc;
    ++asked, ++in_segment;
    to += S::kStageBytes;
    if (to >= lds0 + S::kLds) to -= S::kLds;
  };

  const int wq = wave / S::WP, wp = wave % S::WP;
  const ProductReads<S::QCOL, S::SPLIT, S::TQ> read_q(wq * S::TQ, lane);
  const ProductReads<S::PCOL, S::SPLIT, S::TP> read_p(wp * S::TP, lane);

  float4_t acc[S::NR][S::TQ][S::TP];
#pragma unroll
  for (int r = 0; r < S::NR; ++r)
#pragma unroll
    for (int t = 0; t < S::TQ; ++t)
#pragma unroll
      for (int u = 0; u < S::TP; ++u) acc[r][t][u] = float4_t{0.f, 0.f, 0.f, 0.f};

#pragma unroll
  for (int s = 0; s < S::kStages; ++s)
    if (s < steps) ask();
  int at = 0;
  // step s is in LDS, as all waves see it; the stages behind it that have been asked for stay in flight
  const auto arrive = [&](int s, unsigned char* stage) __attribute__((always_inline)) {
    const int behind = asked - 1 - s;
    if (S::kStages > 3 && behind >= 2) product_wait<(S::kStages > 3 ? 2 : 0) * S::J>();
    else if (S::kStages > 2 && behind >= 1) product_wait<(S::kStages > 2 ? 1 : 0) * S::J>();
    else product_wait<0>();
    if (++at < per) return;  // else a segment's last step
    at = 0;
    const int left = int(count - int64_t(per - 1) * S::kStep);
    if (S::SPLIT || !(left & 7) || (S::QCOL && S::PCOL)) return;
    const auto clear = [&](unsigned char* tiles, int items) __attribute__((always_inline)) {
      for (int t = threadIdx.x; t < items; t += S::kThreads) {
        half8_t* const p = reinterpret_cast<half8_t*>(tiles + t * 128 + ((left >> 3) ^ ((t & 15) >> 1)) * 16);
        half8_t v = *p;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e >= (left & 7)) v[e] = half_t(0);
        *p = v;
      }
    };
    if (!S::QCOL) clear(stage, S::BQ);
    if (!S::PCOL) clear(stage + S::CQ * 1024, S::NP * S::BP);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // A wave's block in two halves of its lines: while the products of one half run, the operands of the next are on their way out of LDS.
  constexpr int HQ = S::TQ / 2;
  static_assert(S::TQ % 2 == 0, "halves");
  constexpr int NV = S::SPLIT ? 2 : 1;  // parts of a value
  half8_t p0s[NV * S::NP][S::TP], p1s[NV * S::NP][S::TP], fa[NV][HQ], fb[NV][HQ];
  typedef half8_t PValues[NV * S::NP][S::TP];
  typedef half8_t QValues[NV][HQ];
  const auto get_p = [&](PValues& f, const unsigned char* stage, int h, int u) __attribute__((always_inline)) {
#pragma unroll
    for (int o = 0; o < NV * S::NP; ++o) f[o][u] = read_p.get(stage + (S::CQ + (S::SPLIT ? 0 : o) * (S::BP / 8)) * 1024, u, S::SPLIT ? o : h);
  };
  const auto get_q = [&](QValues& f, const unsigned char* stage, int h, int half, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int o = 0; o < NV; ++o) f[o][t] = read_q.get(stage, half * HQ + t, S::SPLIT ? o : h);
  };
  const auto multiply = [&](const PValues& p, const QValues& q, int half, int t) __attribute__((always_inline)) {
    const int line = half * HQ + t;
#pragma unroll
    for (int u = 0; u < S::TP; ++u) {
      if (S::SPLIT) {
        acc[0][line][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[NV - 1][u], q[0][t], acc[0][line][u], 0, 0, 0);
        acc[0][line][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[0][u], q[NV - 1][t], acc[0][line][u], 0, 0, 0);
        acc[0][line][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[0][u], q[0][t], acc[0][line][u], 0, 0, 0);
      } else {
#pragma unroll
        for (int r = 0; r < S::NR; ++r) acc[r][line][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[r][u], q[0][t], acc[r][line][u], 0, 0, 0);
      }
    }
  };
  unsigned char* stage = lds;
  arrive(0, stage);
#pragma unroll
  for (int u = 0; u < S::TP; ++u) get_p(p0s, stage, 0, u);
#pragma unroll
  for (int t = 0; t < HQ; ++t) get_q(fa, stage, 0, 0, t);
  // 32 steps of stage s, with P's values in `p`; those of the next 32 go into `next`.  (Reads in a row would fill the queue to LDS, and products wait behind them: a few
  // at a time.)
  const auto sub = [&](int s, int h, const PValues& p, PValues& next) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < HQ; ++t) {
      get_q(fb, stage, h, 1, t);
      multiply(p, fa, 0, t);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (h == S::kSubs - 1 && s + 1 < steps) {
      stage += S::kStageBytes;
      if (stage >= lds + S::kLds) stage -= S::kLds;
      arrive(s + 1, stage);
      if (asked < steps) ask();  // into the place of stage s, which all waves have left
    }
    const int then = (h + 1) % S::kSubs;
#pragma unroll
    for (int t = 0; t < HQ; ++t) {  // (behind the last stage: what is there once more)
      get_q(fa, stage, then, 0, t);
#pragma unroll
      for (int u = t * S::TP / HQ; u < (t + 1) * S::TP / HQ; ++u) get_p(next, stage, then, u);
      multiply(p, fb, 1, t);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  for (int s = 0; s < steps; ++s) {
    sub(s, 0, p0s, p1s);
    if (S::kSubs == 1 && ++s >= steps) break;
    sub(s, S::kSubs - 1, p1s, p0s);
  }
  // What the epilogue reads is asked for first, half of the block at a time: behind its stores every load would wait for them.
  const auto finish = [&](auto whole) __attribute__((always_inline)) {  // whole: all of the tile exists, and nothing is asked about it
    constexpr bool kWhole = decltype(whole)::value;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      typename Epilogue::Read read[HQ][S::TP];
      const auto each = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < HQ; ++t) {
          const int64_t q = q0 + 16 * (wq * S::TQ + half * HQ + t) + i;
#pragma unroll
          for (int u = 0; u < S::TP; ++u) {
            const int64_t p = p0 + 16 * (wp * S::TP + u) + 4 * qq;
            if (kWhole || (q < a.nq && p < a.np)) f(q, p, t, u);
          }
        }
      };
      each([&](int64_t q, int64_t p, int t, int u) __attribute__((always_inline)) { read[t][u] = epilogue.read(q, p); });
      each([&](int64_t q, int64_t p, int t, int u) __attribute__((always_inline)) {
        const int line = half * HQ + t;
        if constexpr (S::NR == 2) epilogue.template put<kWhole>(part, q, p, read[t][u], acc[0][line][u], acc[1][line][u]);
        else epilogue.template put<kWhole>(part, q, p, read[t][u], acc[0][line][u]);
      });
    }
  };
  if (q0 + S::BQ <= a.nq && p0 + S::BP <= a.np) finish(std::true_type());
  else finish(std::false_type());
}

struct ProductNothing {};

// tiles of a product: all there are, and in a.tiles those of a launch
template <class S>
inline int64_t product_tiles(ProductArgs& a) {
  const int64_t lines = ceil_div(a.nq, S::BQ), tiles_p = ceil_div(a.np, S::BP);
  const int64_t tiles = a.lower ? lines * (lines + 1) / 2 : lines * tiles_p;
  a.lines = int32_t(lines), a.tiles_p = int32_t(tiles_p);
  a.tiles = a.some ? a.some : int32_t(std::min<int64_t>(tiles, 0x7fffffff));
  return a.some ? a.some : tiles;
}
// beyond 64 KB of dynamic LDS the runtime wants to be told, once for a kernel and a device (told: a bit a device; two threads write the same at worst)
inline hgnn_status product_lds(const void* kernel, int bytes, uint64_t* told) {
  if (bytes <= 65536) return HGNN_OK;
  int dev = 0;
  HGNN_HIP(hipGetDevice(&dev));
  if (dev < 64 && (__atomic_load_n(told, __ATOMIC_ACQUIRE) >> dev & 1)) return HGNN_OK;
  HGNN_HIP(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
  if (dev < 64) __atomic_fetch_or(told, uint64_t(1) << dev, __ATOMIC_RELEASE);
  return HGNN_OK;
}
template <class S, class Epilogue>
inline hgnn_status product(const char* who, ProductArgs& a, const Epilogue& e, hipStream_t s) {
  constexpr int64_t kMost = 0x7ffffe;  // workgroups of a launch: a grid's lanes fit 32 bits
  const int64_t tiles = product_tiles<S>(a);
  HGNN_REQUIRE(tiles <= 0x7fffffff && (a.parts == 1 || tiles * a.parts <= kMost), HGNN_EUNSUPPORTED, "%s: grid too large", who);
  static uint64_t told = 0;
  const hgnn_status st = product_lds(reinterpret_cast<const void*>(&product_kernel<S, Epilogue>), S::kLds, &told);
  if (st != HGNN_OK) return st;
  ProductArgs b = a;
  for (int64_t done = 0; done < tiles; done += b.tiles) {
    b.first = a.first + int32_t(done), b.tiles = int32_t(a.parts == 1 ? std::min(tiles - done, kMost) : tiles);
    product_kernel<S, Epilogue><<<dim3(unsigned(b.tiles) * unsigned(b.parts)), S::kThreads, S::kLds, s>>>(b, e);
    HGNN_LAUNCH_CHECK("product_kernel");
  }
  return HGNN_OK;
}

}  // namespace hgnn
