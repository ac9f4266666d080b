// Dense products on the matrix cores for matrices of any size:  C[q][p] = sum_k Q(q, k) P(p, k), fp16 operands, fp32 sums, and an epilogue that takes the
// sums out of the registers.  Used by the gated projection (gated.hip) and the orthogonal updates (orthogonalize.hip).
//
// An operand lies with the contraction along its rows ([items][k], "rows") or across them ([k][items], "columns").  Both come into LDS as 32 contraction steps
// of 64 or more items by loads that write LDS directly, a kilobyte an instruction, 16 bytes a lane, a ring of kStages ahead of the products, so that no register
// and no instruction of a lane carries them; lanes choose WHICH 16 bytes they ask for, such that the reads behind meet on no bank:
//  - rows: an instruction is 16 items of 32 steps; lane l asks for item l / 4, piece (l % 4) ^ (l / 16), and ds_read_b128 gives a lane eight steps of an item;
//  - columns: an instruction is 8 steps of 64 items; piece u of step r stands at place u ^ turn(r), and ds_read_b64_tr_b16 gives a lane four steps of an item.
// What is behind the contraction's end is asked for at a place that holds zeros; where the end lies inside a piece, the rest of the piece is cleared in LDS
// (the bytes there are the caller's padding and may be NaN).  Items that do not exist are asked for at the last one that does: they meet only results that
// are not stored.
//
// v_mfma_f32_16x16x32_f16 with P as its first operand: a lane has four consecutive p of one q.  A wave's block of sums decides how often an operand is read
// from LDS, and that is what bounds the large shape (256 x 256: 8 waves of 128 x 64, (128 + 64) 64 bytes a step for 32 products of 16 cycles).
#pragma once

#include "common.h"

namespace hgnn {

typedef float float4_t __attribute__((ext_vector_type(4)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef short short8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) short4_t lds_short4_t;

// Two operands each where the kernel takes two: of P for two results at once (kTwo), the second segment of the contraction (kSegments), or the low parts of
// values that are two fp16 numbers each (kSplit: Q0 P0 + Q0 P1 + Q1 P0).
enum ProductKind { kOne, kTwo, kSegments, kSplit };

struct ProductArgs {
  const half_t *Q0, *Q1, *P0, *P1;
  int64_t ldq, ldp;
  int64_t nq, np;   // items
  int64_t K;        // of a segment
  int64_t part;     // contraction steps of a workgroup (blocks beyond the first take the next ones); a multiple of 32, or K where there is one part
  int64_t tiles;    // of C, tiles_p of them on a line
  int32_t tiles_p;
  int32_t parts;
  int32_t lower;    // square C of square tiles: those on and below the diagonal alone
};

static __device__ const uint4 g_product_zero = {0, 0, 0, 0};

template <int WQ_, int WP_, int TQ_, int TP_, ProductKind KIND_, bool QCOL_, bool PCOL_, int STAGES_>
struct ProductShape {
  static constexpr int WQ = WQ_, WP = WP_, TQ = TQ_, TP = TP_, kStages = STAGES_;
  static constexpr ProductKind KIND = KIND_;
  static constexpr bool QCOL = QCOL_, PCOL = PCOL_;
  static constexpr int kWaves = WQ * WP, kThreads = kWaves * kWave;
  static constexpr int BQ = 16 * TQ * WQ, BP = 16 * TP * WP;
  static constexpr int NQ = KIND == kSplit ? 2 : 1, NP = KIND == kSplit || KIND == kTwo ? 2 : 1;  // operands in LDS
  static constexpr int NR = KIND == kTwo ? 2 : 1;                                                 // results
  static constexpr int CQ = NQ * BQ / 16, CP = NP * BP / 16;  // kilobytes of a stage
  static constexpr int JQ = CQ / kWaves, JP = CP / kWaves, J = JQ + JP;
  static constexpr int kStageBytes = (CQ + CP) * 1024;
  static constexpr int kLds = kStageBytes * kStages;
  static_assert(CQ % kWaves == 0 && CP % kWaves == 0, "whole kilobytes of each operand to every wave");
  static_assert((!QCOL || BQ % 64 == 0) && (!PCOL || BP % 64 == 0), "panels of 64 items");
  static_assert(kLds <= 160 * 1024, "LDS");
};

// place of 16 bytes of step r (0..31) among the eight of 64 items
__device__ __forceinline__ int product_turn(int r) { return 2 * ((r >> 1) & 1) | 4 * ((r >> 3) & 1); }

// 16 bytes a lane from src to LDS at `to` (uniform) + 16 * lane.  Written out, because behind the builtin the compiler waits for all of them before every
// read of LDS; what it does not know of is waited for by product_wait.  (Nothing else in these kernels uses m0.)
__device__ __forceinline__ void load_to_lds(const void* src, uint32_t to) {
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

// one operand's kilobytes that a wave brings in
template <int N, bool COL>
struct ProductLoads {
  const char* at[N];
  int k[N];  // step of the lane's piece inside 32
  int64_t inc;
};
template <int N, bool COL, int CHUNKS, int WAVES>
__device__ __forceinline__ void product_loads(ProductLoads<N, COL>& s, const half_t* first, const half_t* second, int64_t ld, int64_t item0, int64_t items, int64_t k0, int wave,
                                              int lane, int half) {
  s.inc = (COL ? 32 * ld : 32) * int64_t(sizeof(half_t));
#pragma unroll
  for (int j = 0; j < N; ++j) {
    int c = wave + j * WAVES;
    const half_t* base = first;
    if (c >= half) c -= half, base = second;  // uniform
    if (COL) {
      const int r = 8 * (c % 4) + (lane >> 3), u = (lane & 7) ^ product_turn(r);
      int64_t item = item0 + 64 * (c / 4) + 8 * u;
      if (item >= items) item = 0;
      s.k[j] = r;
      s.at[j] = reinterpret_cast<const char*>(base + (k0 + r) * ld + item);
    } else {
      const int64_t item = min(item0 + 16 * c + (lane >> 2), items - 1);
      s.k[j] = 8 * ((lane & 3) ^ (lane >> 4));
      s.at[j] = reinterpret_cast<const char*>(base + item * ld + k0 + s.k[j]);
    }
  }
}

// where tile number t of C lies: groups of kGroup lines of tiles, walked along the lines' items, so that workgroups that run together share operands
__device__ __forceinline__ void product_tile(const ProductArgs& a, int64_t t, int64_t& tq, int64_t& tp) {
  if (a.lower) {  // t = tq (tq + 1) / 2 + tp
    int64_t r = int64_t((sqrtf(8.f * float(t) + 1.f) - 1.f) * 0.5f);
    while (r * (r + 1) / 2 > t) --r;
    while ((r + 1) * (r + 2) / 2 <= t) ++r;
    tq = r, tp = t - r * (r + 1) / 2;
    return;
  }
  constexpr int64_t kGroup = 8;
  const int64_t lines = a.tiles / a.tiles_p, per = kGroup * a.tiles_p, g = t / per, in = t - g * per, rows = min(kGroup, lines - g * kGroup);
  tp = in / rows;
  tq = g * kGroup + (in - tp * rows);
}

template <class S>
__device__ __forceinline__ half8_t product_fragment(const unsigned char* tile, int f, bool col, const int (&off)[4]) {
  if (!col) return *reinterpret_cast<const half8_t*>(tile + f * 1024 + off[0]);
  const unsigned char* p = tile + (f / 4) * 4096 + off[f % 4];
  const short4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t*)p);
  const short4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t*)(p + 512));
  return __builtin_bit_cast(half8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <class S, class Epilogue>
__global__ __launch_bounds__(S::kThreads, 2) void product_kernel(ProductArgs a, Epilogue epilogue) {
  extern __shared__ __align__(1024) unsigned char lds[];
  const int lane = threadIdx.x & (kWave - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int i = lane & 15, qq = lane >> 4;
  // consecutive workgroups go to the XCDs in turn: each takes a run of tiles of its own
  const int64_t all = a.tiles * a.parts, id = blockIdx.x, x = id & 7, base = all >> 3, more = all & 7;
  const int64_t work = x * base + min(x, more) + (id >> 3);
  const int64_t part = work / a.tiles;
  int64_t tq, tp;
  product_tile(a, work - part * a.tiles, tq, tp);
  const int64_t q0 = tq * S::BQ, p0 = tp * S::BP;
  const int64_t k_begin = part * a.part, k_end = min(a.K, k_begin + a.part), count = k_end - k_begin;  // of a segment
  const int per = int((count + 31) / 32), steps = S::KIND == kSegments ? 2 * per : per;

  ProductLoads<S::JQ, S::QCOL> lq;
  ProductLoads<S::JP, S::PCOL> lp;
  const auto start = [&](bool second) __attribute__((always_inline)) {
    product_loads<S::JQ, S::QCOL, S::CQ, S::kWaves>(lq, second ? a.Q1 : a.Q0, a.Q1, a.ldq, q0, a.nq, k_begin, wave, lane, S::BQ / 16);
    product_loads<S::JP, S::PCOL, S::CP, S::kWaves>(lp, second ? a.P1 : a.P0, a.P1, a.ldp, p0, a.np, k_begin, wave, lane, S::BP / 16);
  };
  start(false);
  const char* const zero = reinterpret_cast<const char*>(&g_product_zero);
  const uint32_t lds0 = uint32_t(uintptr_t((__attribute__((address_space(3))) unsigned char*)lds));
  int asked = 0, in_segment = 0;
  uint32_t to = lds0 + wave * 1024;
  const auto ask = [&]() __attribute__((always_inline)) {
    if (S::KIND == kSegments && in_segment == per) in_segment = 0, start(true);
    const int left = int(min(count - int64_t(in_segment) * 32, int64_t(32)));
#pragma unroll
    for (int j = 0; j < S::JQ; ++j) {
      load_to_lds(lq.k[j] < left ? lq.at[j] : zero, to + j * S::kWaves * 1024);
      lq.at[j] += lq.inc;
    }
#pragma unroll
    for (int j = 0; j < S::JP; ++j) {
      load_to_lds(lp.k[j] < left ? lp.at[j] : zero, to + (S::JQ + j) * S::kWaves * 1024);
      lp.at[j] += lp.inc;
    }
    ++asked, ++in_segment;
    to += S::kStageBytes;
    if (to >= lds0 + S::kLds) to -= S::kLds;
  };

  const int wq = wave / S::WP, wp = wave % S::WP;
  int off_row[4], off_col[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int r = 8 * qq + (i >> 2);
    off_row[t] = 16 * (4 * i + (qq ^ (i >> 2)));
    off_col[t] = r * 128 + (((2 * t + ((i & 3) >> 1)) ^ product_turn(r)) * 16) + (i & 1) * 8;
  }

  float4_t acc[S::NR][S::TQ][S::TP];
#pragma unroll
  for (int r = 0; r < S::NR; ++r)
#pragma unroll
    for (int t = 0; t < S::TQ; ++t)
#pragma unroll
      for (int u = 0; u < S::TP; ++u) acc[r][t][u] = float4_t{0.f, 0.f, 0.f, 0.f};

#pragma unroll
  for (int s = 0; s < S::kStages - 1; ++s)
    if (s < steps) ask();
  const unsigned char* stage = lds;
  for (int s = 0, at = 0; s < steps; ++s) {
    // the stages behind this one that have been asked for stay in flight
    const int behind = asked - 1 - s;
    if (S::kStages > 3 && behind >= 2) product_wait<(S::kStages > 3 ? 2 : 0) * S::J>();
    else if (S::kStages > 2 && behind >= 1) product_wait<(S::kStages > 2 ? 1 : 0) * S::J>();
    else product_wait<0>();
    if (asked < steps) ask();
    if (++at == per) {  // a segment's last step
      at = 0;
      const int left = int(count - int64_t(per - 1) * 32);
      if ((left & 7) && (!S::QCOL || !S::PCOL)) {
        const auto clear = [&](unsigned char* tiles, int items) __attribute__((always_inline)) {
          for (int t = threadIdx.x; t < items; t += S::kThreads) {
            const int n = t & 15;
            half8_t* const p = reinterpret_cast<half8_t*>(tiles + (t >> 4) * 1024 + 16 * (4 * n + ((left >> 3) ^ (n >> 2))));
            half8_t v = *p;
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e >= (left & 7)) v[e] = half_t(0);
            *p = v;
          }
        };
        unsigned char* const here = const_cast<unsigned char*>(stage);
        if (!S::QCOL) clear(here, S::NQ * S::BQ);
        if (!S::PCOL) clear(here + S::CQ * 1024, S::NP * S::BP);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
    }
    half8_t fp[S::NP][S::TP];
#pragma unroll
    for (int o = 0; o < S::NP; ++o)
#pragma unroll
      for (int u = 0; u < S::TP; ++u) fp[o][u] = product_fragment<S>(stage + (S::CQ + o * (S::BP / 16)) * 1024, wp * S::TP + u, S::PCOL, S::PCOL ? off_col : off_row);
#pragma unroll
    for (int t = 0; t < S::TQ; ++t) {
      half8_t fq[S::NQ];
#pragma unroll
      for (int o = 0; o < S::NQ; ++o) fq[o] = product_fragment<S>(stage + o * (S::BQ / 16) * 1024, wq * S::TQ + t, S::QCOL, S::QCOL ? off_col : off_row);
#pragma unroll
      for (int u = 0; u < S::TP; ++u) {
        if (S::KIND == kSplit) {
          acc[0][t][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fp[S::NP - 1][u], fq[0], acc[0][t][u], 0, 0, 0);
          acc[0][t][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fp[0][u], fq[S::NQ - 1], acc[0][t][u], 0, 0, 0);
          acc[0][t][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fp[0][u], fq[0], acc[0][t][u], 0, 0, 0);
        } else {
#pragma unroll
          for (int r = 0; r < S::NR; ++r) acc[r][t][u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fp[r][u], fq[0], acc[r][t][u], 0, 0, 0);
        }
      }
    }
    stage += S::kStageBytes;
    if (stage >= lds + S::kLds) stage -= S::kLds;
  }
#pragma unroll
  for (int t = 0; t < S::TQ; ++t) {
    const int64_t q = q0 + 16 * (wq * S::TQ + t) + i;
    if (q >= a.nq) continue;
#pragma unroll
    for (int u = 0; u < S::TP; ++u) {
      const int64_t p = p0 + 16 * (wp * S::TP + u) + 4 * qq;
      if (p >= a.np) continue;
      if constexpr (S::NR == 2) epilogue(part, q, p, acc[0][t][u], acc[1][t][u]);
      else epilogue(part, q, p, acc[0][t][u]);
    }
  }
}

// tiles and workgroups of a product, and its launch
template <class S>
inline void product_tiles(ProductArgs& a) {
  const int64_t lines = ceil_div(a.nq, S::BQ);
  a.tiles_p = int32_t(ceil_div(a.np, S::BP));
  a.tiles = a.lower ? lines * (lines + 1) / 2 : lines * a.tiles_p;
}
template <class S, class Epilogue>
inline hgnn_status product(const char* who, ProductArgs& a, const Epilogue& e, hipStream_t s) {
  product_tiles<S>(a);
  HGNN_REQUIRE(a.tiles * a.parts <= 0x7ffffe, HGNN_EUNSUPPORTED, "%s: grid too large", who);
  if (S::kLds > 65536) {
    int dev = 0;
    HGNN_HIP(hipGetDevice(&dev));
    static uint64_t told = 0;  // devices, a bit each: the same value is written again at worst
    if (dev >= 64 || !(__atomic_load_n(&told, __ATOMIC_ACQUIRE) >> dev & 1)) {
      HGNN_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(&product_kernel<S, Epilogue>), hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds));
      if (dev < 64) __atomic_fetch_or(&told, uint64_t(1) << dev, __ATOMIC_RELEASE);
    }
  }
  product_kernel<S, Epilogue><<<dim3(unsigned(a.tiles * a.parts)), S::kThreads, S::kLds, s>>>(a, e);
  HGNN_LAUNCH_CHECK("product_kernel");
  return HGNN_OK;
}

}  // namespace hgnn
