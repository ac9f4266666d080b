// Rows of a learned vertex table by id, and the gradient of the table: what stands before the first layer of a graph without vertex features.
#include <algorithm>

#include "common.h"
#include "rows.h"
#include "sort.h"

namespace hgnn {

constexpr int kLookups = 4;                     // rows that L lanes take together, of many
constexpr int64_t kFewLookups = int64_t(1) << 20;  // lanes of all rows up to which they take one

struct LookupArgs {
  int64_t n;
  int F, V;
  const int* ids;
  const void* table;
  int64_t ldt, inside;  // elements from the table's first to its last
  float scale;
  half_t* out;
  int64_t ldo;
};

// out[i] = scale * T[ids[i]]: L lanes take N rows in pieces of eight, whose reads go out together.  Bound by memory.
template <class T, int L, int N, bool PAST>
__global__ __launch_bounds__(kBlock) void embedding_kernel(LookupArgs a) {
  constexpr int G = kBlock / L;
  const int64_t i0 = int64_t(blockIdx.x) * (G * N) + threadIdx.x / L;
  int id[N];
#pragma unroll
  for (int u = 0; u < N; ++u) id[u] = i0 + u * G < a.n ? a.ids[i0 + u * G] : -1;
  for (int f = 8 * (threadIdx.x % L); f < a.F; f += 8 * L) {
    RawPiece<T> x[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      x[u].v = 0;
      const int64_t at = int64_t(id[u]) * a.ldt + f;
      if (uint32_t(id[u]) < uint32_t(a.V)) x[u] = load_raw(static_cast<const T*>(a.table) + at, a.F - f, a.inside - at);
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      if (i0 + u * G >= a.n) break;
      const float scale = uint32_t(id[u]) < uint32_t(a.V) ? a.scale : 0.f;  // zeros for padding, whatever the scale
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = float(x[u].v[j]) * scale;
      Part<half_t, 8>::template store<PAST>(a.out + (i0 + u * G) * a.ldo + f, a.F - f, y);
    }
  }
}

// ---- the gradient -------------------------------------------------------------------------------------------
// dT[v] = scale * sum of dY[i] over the i with ids[i] = v.  The positions are sorted by id (stable, so the rows of an id keep their order).  L lanes walk a
// share of the sorted list, 8 or 16 positions, a workgroup so many consecutive ones as it has groups of L.  A run of equal ids inside a share is stored at
// once.  What shares hold of a run in common goes to LDS, `head` of a run that began before the share, `tail` of one that goes on behind it, and is added in
// order by the share where the run begins; what workgroups hold in common goes to memory in the same two forms, and a second pass adds it.  No atomics: the
// same bits on every run.  Rows without a position are zeros, which workgroups behind those of the shares write.

// words: (id, position), an id that is none counts as V
struct IdWords {
  const int* ids;
  int V, pos_bits;
  template <int PER>
  __device__ __forceinline__ void prepare(int64_t, int, int*) const {}
  __device__ __forceinline__ uint64_t word(int id, int64_t k) const {
    return (uint64_t(min(uint32_t(id), uint32_t(V))) << pos_bits) | uint64_t(k);
  }
  template <int PER>
  __device__ __forceinline__ void load(int64_t first, int n, int mine, const int*, uint64_t (&w)[PER]) const {
    int id[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) id[j] = ids[first + min(mine + j * kWave, n - 1)];
#pragma unroll
    for (int j = 0; j < PER; ++j) w[j] = word(id[j], first + min(mine + j * kWave, n - 1));
  }
  __device__ __forceinline__ uint64_t count(const SortPass&, int64_t k) const { return word(ids[k], k); }
};

enum { kPastZeros = 1, kPastAll = 2 };
struct TableGradArgs {
  const uint64_t* words;  // sorted
  int64_t n;
  int pos_bits, F, V;
  int zero_bits;   // 2^zero_bits lanes write the zeros of a row
  int zero_waves;  // waves that share 64 rows
  int zero_span;   // features of a workgroup's zeros
  const half_t* dY;
  int64_t ldy, inside;  // elements from the first of dY to its last
  float scale;
  void* dT;
  int64_t lddt;
  float* part;  // [blocks][2][pitch]: head and tail of a workgroup
  int pitch;
  int64_t blocks;  // workgroups of shares
  int share;
  int past;  // the caches: zeros, or all rows
  __device__ __forceinline__ int id(int64_t k) const { return int(words[k] >> pos_bits); }
  __device__ __forceinline__ int id_of(uint64_t w) const { return int(w >> pos_bits); }
  __device__ __forceinline__ int64_t pos(uint64_t w) const { return int64_t(w & ((uint64_t(1) << pos_bits) - 1)); }
  __device__ __forceinline__ float* partial(int64_t block, int tail) const { return part + (2 * block + tail) * pitch; }
};

// A lane's eight features of a row: four at f and four at f + 4 L, so that the 16 bytes that lanes store lie beside each other
struct Quads {
  float4_t lo, hi;
  __device__ __forceinline__ void add(const Quads& y) { lo += y.lo, hi += y.hi; }
};
template <int L>
__device__ __forceinline__ Quads load_quads(const float* p, int f, int F) {  // of a row that is padded to whole quads
  Quads r{};
  if (f < F) r.lo = *reinterpret_cast<const float4_t*>(p + f);
  if (f + 4 * L < F) r.hi = *reinterpret_cast<const float4_t*>(p + f + 4 * L);
  return r;
}
template <int L>
__device__ __forceinline__ void store_quads(float* p, int f, int F, const Quads& x) {
  if (f < F) *reinterpret_cast<float4_t*>(p + f) = x.lo;
  if (f + 4 * L < F) *reinterpret_cast<float4_t*>(p + f + 4 * L) = x.hi;
}
template <class T, bool ADD>
__device__ __forceinline__ void add_quad(const TableGradArgs& a, T* p, int left, float4_t v) {
  if (left <= 0) return;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] *= a.scale;
  if (ADD) {
    const auto y = load_quad(p, left, left);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] += float(y[j]);
  }
  if (a.past == kPastAll) store_quad<T, true>(p, left, v);
  else store_quad(p, left, v);
}
template <class T, bool ADD, int L>
__device__ __forceinline__ void add_row(const TableGradArgs& a, int id, int f, const Quads& x) {
  T* const p = static_cast<T*>(a.dT) + int64_t(id) * a.lddt + f;
  add_quad<T, ADD>(a, p, a.F - f, x.lo);
  add_quad<T, ADD>(a, p + 4 * L, a.F - f - 4 * L, x.hi);
}

// by a whole wave, 64 places looked at in each step: how many of the n sorted words have an id below id[0], and below id[1]
__device__ __forceinline__ void wave_words_below(const TableGradArgs& a, const int64_t (&id)[2], int64_t (&below)[2]) {
  const int lane = threadIdx.x & (kWave - 1);
  int64_t lo[2] = {0, 0}, hi[2] = {a.n, a.n};  // the answers are in [lo, hi]
  while (lo[0] < hi[0] || lo[1] < hi[1]) {
    int64_t step[2];
    bool holds[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      step[i] = (hi[i] - lo[i] + kWave - 1) / kWave;
      const int64_t at = lo[i] + lane * step[i];
      holds[i] = at < hi[i] && a.id(at < hi[i] ? at : 0) < id[i];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (lo[i] >= hi[i]) continue;
      const int held = __popcll(__ballot(holds[i]));  // the first lanes
      if (held == 0) {
        hi[i] = lo[i];
      } else {
        const int64_t last = lo[i] + (held - 1) * step[i];
        hi[i] = last + step[i] < hi[i] ? last + step[i] : hi[i];
        lo[i] = last + 1;
      }
    }
  }
  below[0] = lo[0], below[1] = lo[1];
}

constexpr int kZeroRows = kWave;  // table rows of a wave that writes zeros
constexpr int kMarked = 4;        // times 64 positions in those rows up to which each marks its row

// whether the 128-byte line of `at` lies in the row from..to
__device__ __forceinline__ bool in_whole_line(const char* at, const char* from, const char* to) {
  const char* const line = at - (reinterpret_cast<uintptr_t>(at) & 127u);
  return line >= from && line + 128 <= to;
}

// zeros in features f0 to f1 of those of 64 rows that no position has; s_there: 64 words of the wave's own
template <class T>
__device__ __forceinline__ void write_zeros(const TableGradArgs& a, int64_t r0, int part, int f0, int f1, int* s_there) {
  if (r0 >= a.V || f0 >= f1) return;
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t r = r0 + lane, ids[2] = {r0, r0 + kZeroRows};
  int64_t range[2] = {0, 0};
  if (a.n > 0) wave_words_below(a, ids, range);
  bool mine = r >= a.V;
  if (range[1] - range[0] <= kMarked * kWave) {
    int id[kMarked];
#pragma unroll
    for (int i = 0; i < kMarked; ++i) {
      const int64_t at = range[0] + i * kWave + lane;
      id[i] = at < range[1] ? a.id(at) - int(r0) : -1;
    }
    s_there[lane] = 0;
    wave_sync();
#pragma unroll
    for (int i = 0; i < kMarked; ++i)
      if (id[i] >= 0) s_there[id[i]] = 1;
    wave_sync();
    mine = mine || s_there[lane] != 0;
  } else {
    int64_t lo = range[0], hi = range[1];
    while (lo < hi) {
      const int64_t mid = (lo + hi) >> 1;
      if (a.id(mid) < r) lo = mid + 1;
      else hi = mid;
    }
    mine = mine || (lo < range[1] && a.id(lo) == r);
  }
  const uint64_t there = __ballot(mine);
  const int rows = kWave >> a.zero_bits;
  for (int k = (lane >> a.zero_bits) + part * rows; k < kZeroRows; k += rows * a.zero_waves) {
    if (there >> k & 1) continue;
    T* const p = static_cast<T*>(a.dT) + (r0 + k) * a.lddt;
    const char* const from = reinterpret_cast<const char*>(p);
    const char* const to = reinterpret_cast<const char*>(p + a.F);
    for (int f = f0 + 4 * (lane & ((1 << a.zero_bits) - 1)); f < f1; f += 4 << a.zero_bits)
      if (const char* const at = reinterpret_cast<const char*>(p + f); a.past != 0 && in_whole_line(at, from, to)) store_quad<T, true>(p + f, a.F - f, float4_t{});
      else store_quad(p + f, a.F - f, float4_t{});
  }
}

// Positions of a share: many positions leave more shares than the chip holds at once, and shares of some hundred workgroups' runs to be joined.  us, 8 / 16:
// 1024 of 64 into 4096 rows 15.2 / 18.5, 30 000 of 64 into 233 000 36 / 39, 200 000 of 128 into 233 000 59 / 57, 1 000 003 of 128 (power law) into 2.4 M 339 /
// 336, into 10 000 113 / 103, into 100 97 / 86.
static int share_of(int64_t n) { return n < int64_t(1) << 19 ? 8 : 16; }
constexpr int kAhead = 4;  // rows of a share that are fetched together

template <class T, bool ADD, int L>
__global__ __launch_bounds__(kBlock, 6) void table_grad_kernel(TableGradArgs a) {
  constexpr int G = kBlock / L;  // shares of a workgroup
  __shared__ Quads s_part[2][kBlock];  // head and tail of the shares
  if (int64_t(blockIdx.x) >= a.blocks) {
    const int wave = threadIdx.x / kWave;
    const int64_t r0 = ((int64_t(blockIdx.x) - a.blocks) * (kWavesPerBlock / a.zero_waves) + wave / a.zero_waves) * kZeroRows;
    const int f0 = min(a.F, a.zero_span * int(blockIdx.y));
    write_zeros<T>(a, r0, wave % a.zero_waves, f0, min(a.F, f0 + a.zero_span), reinterpret_cast<int*>(s_part) + wave * kZeroRows);
    return;
  }
  const int64_t block = blockIdx.x;
  __shared__ int s_through[G];         // whether a run that began before the share goes on behind it
  const int g = threadIdx.x / L, l = threadIdx.x % L, f = 8 * L * int(blockIdx.y) + 4 * l;
  const int64_t begin = block * (G * a.share), stop = begin + G * a.share < a.n ? begin + G * a.share : a.n;
  const int64_t first = begin + g * a.share < stop ? begin + g * a.share : stop, end = first + a.share < stop ? first + a.share : stop;
  const int before = first > 0 && first < end ? a.id(first - 1) : -1, after = end < a.n && first < end ? a.id(end) : -1;
  int cur = -1, tail_id = -1;
  bool head = false;
  Quads sum{};
  auto done = [&](bool goes_on) __attribute__((always_inline)) {  // with the run of cur
    if (cur < 0 || cur >= a.V) return;
    if (head || goes_on) {
      s_part[head ? 0 : 1][threadIdx.x] = sum;
      if (!head) tail_id = cur;
    } else {
      add_row<T, ADD, L>(a, cur, f, sum);
    }
  };
  for (int64_t k = first; k < end; k += kAhead) {
    uint64_t w[kAhead];
    half4_t x[kAhead][2];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) w[i] = a.words[k + i < end ? k + i : end - 1];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int64_t at = a.pos(w[i]) * a.ldy + f + 4 * L * q;
        x[i][q] = 0;
        if (f + 4 * L * q < a.F) x[i][q] = load_quad(a.dY + at, a.F - f - 4 * L * q, a.inside - at);
      }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (k + i >= end) break;
      const int id = a.id_of(w[i]);
      if (id != cur) {
        done(false);
        cur = id;
        head = k + i == first && id == before;
        sum = Quads{};
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) sum.lo[j] += float(x[i][0][j]), sum.hi[j] += float(x[i][1][j]);
    }
  }
  const bool goes_on = cur >= 0 && cur == after;
  done(goes_on);
  if (l == 0) s_through[g] = head && goes_on;
  __syncthreads();
  // the chain of a run: from the share where it begins, or the workgroup's first, through shares that hold nothing else, to the share where it ends
  auto chain = [&](Quads x, bool open, bool* beyond) __attribute__((always_inline)) {  // and the heads of the shares behind g
    for (int i = g + 1; open && i < G && begin + i * a.share < stop; ++i) {
      x.add(s_part[0][i * L + l]);
      open = s_through[i];
    }
    *beyond = open;  // the workgroup
    return x;
  };
  bool open;
  if (tail_id >= 0) {
    const Quads x = chain(s_part[1][threadIdx.x], true, &open);
    if (open) store_quads<L>(a.partial(block, 1), f, a.F, x);
    else add_row<T, ADD, L>(a, tail_id, f, x);
  }
  if (g == 0 && before >= 0 && before < a.V && a.id(first) == before)
    store_quads<L>(a.partial(block, 0), f, a.F, chain(s_part[0][threadIdx.x], s_through[0], &open));
}

// The runs that several workgroups hold, by a workgroup for each one where a run may begin: its tail and the heads of those behind it, every group of L lanes
// a part of them.  A very long run of wide rows is a compute unit's for every 512 features, of few groups: one id of 1 M positions, us of the sums and of this, rows
// of 128 features 53 + 39, of 512 211 + 685, of 1000 470 + 741 (the calls 131, 921 and 1227; with 10 007 ids alike 106, 292 and 571).
template <class T, bool ADD, int L>
__global__ __launch_bounds__(kBlock) void table_grad_join_kernel(TableGradArgs a) {
  constexpr int G = kBlock / L;
  __shared__ Quads s_part[kBlock];
  const int64_t per = int64_t(G) * a.share, b = blockIdx.x, begin = b * per, end = begin + per;
  const int id = a.id(end);
  if (id >= a.V || a.id(end - 1) != id || (begin > 0 && a.id(begin - 1) == id)) return;
  // workgroups behind this one that begin inside the run: all waves look for the last of them
  int64_t lo = 1, hi = a.blocks - b;  // first one (counted from here) that does not, in [lo, hi]
  while (lo < hi) {
    const int lane = threadIdx.x & (kWave - 1);
    const int64_t step = (hi - lo + kWave - 1) / kWave, at = lo + lane * step;
    const int held = __popcll(__ballot(at < hi && a.id((b + at) * per) == id));
    if (held == 0) {
      hi = lo;
    } else {
      const int64_t last = lo + (held - 1) * step;
      hi = last + step < hi ? last + step : hi;
      lo = last + 1;
    }
  }
  const int g = threadIdx.x / L, l = threadIdx.x % L, f = 8 * L * int(blockIdx.y) + 4 * l;
  Quads sum{};
  if (g == 0) sum = load_quads<L>(a.partial(b, 1), f, a.F);
#pragma unroll 4
  for (int64_t i = 1 + g; i < lo; i += G) sum.add(load_quads<L>(a.partial(b + i, 0), f, a.F));
  s_part[threadIdx.x] = sum;
  __syncthreads();
  if (g > 0) return;
  sum = Quads{};
  for (int i = 0; i < G && i < lo; ++i) sum.add(s_part[i * L + l]);
  add_row<T, ADD, L>(a, id, f, sum);
}

static int bits_of(int64_t values) {  // that tell so many values apart
  int b = 1;
  while ((int64_t(1) << b) < values) ++b;
  return b;
}

// Lanes of a share at least: what a workgroup's shares have in common is added share by share.  us, one lane to a row / two / four / eight: 97 985 positions of
// one row of 1 feature 47 / 36 / 27 / 24; 385 356 of 116 976 rows of 1 feature 43.6 / 42.6 / 43.6 / 47.6; 1 000 000 of as many rows of 8 97 / 93 / 95 / 97.
constexpr int kShareLanes = 4;
struct TableGradSpace {
  uint64_t *buf0, *buf1;
  void* scratch;
  float* part;
  int64_t blocks;
  int pitch;
  size_t bytes;
};
static TableGradSpace table_grad_space(void* base, int64_t n, int32_t F) {
  TableGradSpace p{};
  char* at = static_cast<char*>(base);
  auto take = [&](size_t bytes) {
    char* const q = at;
    at += (bytes + 255) / 256 * 256;
    return q;
  };
  const int groups = kBlock / std::max(kShareLanes, std::min(kWave, pow2_at_least((F + 7) / 8)));
  p.blocks = ceil_div(n, int64_t(groups) * share_of(n));
  p.pitch = (F + 7) / 8 * 8;
  p.buf0 = reinterpret_cast<uint64_t*>(take(8 * size_t(n)));
  p.buf1 = reinterpret_cast<uint64_t*>(take(8 * size_t(n)));
  p.scratch = take(n > 0 ? sort_scratch_bytes(n) : 0);
  p.part = reinterpret_cast<float*>(take(p.blocks > 1 ? 2 * size_t(p.blocks) * size_t(p.pitch) * sizeof(float) : 0));
  p.bytes = size_t(at - static_cast<char*>(base));
  return p;
}

template <int LEAST, class Call>
static void with_lanes(int F, Call&& call) {  // lanes that take a row of F, LEAST (1 or 4) or more
  const int lanes = pow2_at_least((F + 7) / 8);
  if constexpr (LEAST == 1) {
    if (lanes == 1) return call(std::integral_constant<int, 1>());
    if (lanes == 2) return call(std::integral_constant<int, 2>());
  }
  if (lanes <= 4) return call(std::integral_constant<int, 4>());
  if (lanes == 8) return call(std::integral_constant<int, 8>());
  if (lanes == 16) return call(std::integral_constant<int, 16>());
  if (lanes == 32) return call(std::integral_constant<int, 32>());
  call(std::integral_constant<int, 64>());
}

template <class T, bool ADD>
static hgnn_status table_grad(const TableGradArgs& a, hipStream_t s) {
  hgnn_status st = HGNN_OK;
  with_lanes<kShareLanes>(a.F, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    const int64_t zeros = ADD ? 0 : ceil_div(a.V, int64_t(kZeroRows) * (kWavesPerBlock / a.zero_waves));
    const unsigned fy = unsigned(ceil_div(a.F, 8 * L));  // 1 up to 512 features
    auto go = [&]() -> hgnn_status {
      HGNN_REQUIRE(a.blocks + zeros <= kMostBlocks, HGNN_EUNSUPPORTED, "hgnn_embedding_grad: grid too large");
      table_grad_kernel<T, ADD, L><<<dim3(unsigned(a.blocks + zeros), fy), kBlock, 0, s>>>(a);
      HGNN_LAUNCH_CHECK("table_grad_kernel");
      if (a.blocks > 1) {
        table_grad_join_kernel<T, ADD, L><<<dim3(unsigned(a.blocks - 1), fy), kBlock, 0, s>>>(a);
        HGNN_LAUNCH_CHECK("table_grad_join_kernel");
      }
      return HGNN_OK;
    };
    st = go();
  });
  return st;
}

}  // namespace hgnn

using namespace hgnn;

extern "C" {

hgnn_status hgnn_embedding(int64_t n, int32_t F, const int32_t* ids, int32_t V, hgnn_type table_type, const void* table, int64_t ldt, float scale,
                           hgnn_half* out, int64_t ldo, void* stream) {
  clear_error();
  const char* who = "hgnn_embedding";
  HGNN_REQUIRE(n >= 0 && F > 0 && V >= 0, HGNN_EINVAL, "%s: n = %lld, F = %d, V = %d", who, static_cast<long long>(n), F, V);
  HGNN_REQUIRE(known_type(table_type), HGNN_EINVAL, "%s: unknown type %d", who, int(table_type));
  HGNN_REQUIRE(ldt >= F && ldo >= F, HGNN_EINVAL, "%s: leading dimension smaller than F", who);
  HGNN_REQUIRE(F <= 65536 && n <= (int64_t(1) << 40), HGNN_EUNSUPPORTED, "%s: F = %d above 65536, or n = %lld above 2^40", who, F, static_cast<long long>(n));
  if (n == 0) return HGNN_OK;
  HGNN_REQUIRE(ids && out && (table || V == 0), HGNN_EINVAL, "%s: NULL argument", who);
  HGNN_REQUIRE(aligned_to_type(ids, HGNN_F32) && aligned_to_type(table, table_type) && aligned_to_type(out, HGNN_F16), HGNN_EINVAL,
               "%s: an array that is not aligned to its type", who);
  const LookupArgs a{n, F, V, ids, table, ldt, extent_of(V, F, ldt), scale, reinterpret_cast<half_t*>(out), ldo};
  hgnn_status st = HGNN_OK;
  with_lanes<1>(F, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    auto go = [&]() -> hgnn_status {
      const bool many = n * L >= kFewLookups, past = double(n) * F * sizeof(half_t) >= kPastBytes;
      const int64_t blocks = ceil_div(n, int64_t(kBlock / L) * (many ? kLookups : 1));
      HGNN_REQUIRE(blocks <= kMostBlocks, HGNN_EUNSUPPORTED, "%s: grid too large", who);
      const dim3 grid{unsigned(blocks)};
      hipStream_t s = static_cast<hipStream_t>(stream);
      auto launch = [&](auto type) {
        typedef decltype(type) T;
        if (many && past) embedding_kernel<T, L, kLookups, true><<<grid, kBlock, 0, s>>>(a);
        else if (many) embedding_kernel<T, L, kLookups, false><<<grid, kBlock, 0, s>>>(a);
        else embedding_kernel<T, L, 1, false><<<grid, kBlock, 0, s>>>(a);
      };
      if (table_type == HGNN_F16) launch(half_t());
      else launch(float());
      HGNN_LAUNCH_CHECK("embedding_kernel");
      return HGNN_OK;
    };
    st = go();
  });
  return st;
}

size_t hgnn_embedding_grad_workspace(int64_t n, int32_t F, int32_t V) {
  if (n <= 0 || n > 0x7fffffff || F <= 0 || V <= 0) return 0;
  return table_grad_space(nullptr, n, F).bytes;
}

hgnn_status hgnn_embedding_grad(int64_t n, int32_t F, const int32_t* ids, int32_t V, const hgnn_half* dY, int64_t ldy, float scale, int32_t accumulate,
                                hgnn_type grad_type, void* dT, int64_t lddt, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  const char* who = "hgnn_embedding_grad";
  HGNN_REQUIRE(n >= 0 && F > 0 && V >= 0, HGNN_EINVAL, "%s: n = %lld, F = %d, V = %d", who, static_cast<long long>(n), F, V);
  HGNN_REQUIRE(n <= 0x7fffffff, HGNN_EINVAL, "%s: n = %lld exceeds int32", who, static_cast<long long>(n));
  HGNN_REQUIRE(known_type(grad_type), HGNN_EINVAL, "%s: unknown type %d", who, int(grad_type));
  HGNN_REQUIRE(ldy >= F && lddt >= F, HGNN_EINVAL, "%s: leading dimension smaller than F", who);
  HGNN_REQUIRE(F <= 65536, HGNN_EUNSUPPORTED, "%s: F = %d above 65536", who, F);
  if (V == 0 || (n == 0 && accumulate)) return HGNN_OK;
  HGNN_REQUIRE(dT != nullptr && (n == 0 || (ids && dY)), HGNN_EINVAL, "%s: NULL argument", who);
  const size_t need = hgnn_embedding_grad_workspace(n, F, V);
  HGNN_REQUIRE(need == 0 || (workspace != nullptr && workspace_bytes >= need), HGNN_EINVAL,
               "%s: workspace of %zu bytes, needs %zu (hgnn_embedding_grad_workspace)", who, workspace_bytes, need);
  HGNN_REQUIRE(aligned_to_type(ids, HGNN_F32) && aligned_to_type(dY, HGNN_F16) && aligned_to_type(dT, grad_type) && (need == 0 || aligned16(workspace)),
               HGNN_EINVAL, "%s: an array that is not aligned to its type, or a workspace not to 16 bytes", who);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const TableGradSpace w = table_grad_space(workspace, n, F);
  TableGradArgs a{};
  a.n = n, a.blocks = w.blocks, a.share = share_of(n), a.F = F, a.V = V;
  a.pos_bits = bits_of(n), a.zero_bits = F <= 8 ? 0 : std::min(6, bits_of((F + 7) / 8));
  // Waves of a workgroup share 64 wide rows, a wave alone takes narrow ones.  us, alone / shared, 16 positions: 100 rows of 1000 (fp32) 22 / 12, 60 000 of 333 30 / 21,
  // 300 000 of 333 92 / 90, 1 M of 100 at a pitch of 104 118 / 109, of 128 102 / 103; 40 000 of 64 12.1 / 12.4; 100 000 positions of 233 000 rows of 128 54 / 56.
  a.zero_waves = F > 64 ? kWavesPerBlock : 1;
  // Of wide rows a workgroup for every 512 features writes zeros where rows are few; many are written from end to end (us, 512 / whole: 64 rows of 65 536, fp32, 12 /
  // 350, 10 000 of 1000 16 / 20, 20 000 21 / 21, 200 000 239 / 166).
  constexpr int kFewRows = 16384;
  a.zero_span = V < kFewRows ? 8 * kWave : F;

  // Large tables (kPastBytes) whose rows are whole 128-byte lines are written past the caches.  us, through the caches / zeros past them / all rows past them,
  // 64 M elements of gradients into 200 M (rows of 8 features 1 M into 3 M): rows of 128 bytes (32 x fp32) 191 / 182 / 183, 256 (64 x fp32) 265 / 236 / 229,
  // 512 233 / 227 / 215, 512 (256 x fp16) 162 / 153 / 143; but parts of lines cost more, rows of 32 bytes 127 / 136 / 198, of 168 bytes 312 / 343 / 371. Of
  // rows with gaps, whose parts of lines cost more either way, zeros in the whole lines alone: 16 positions into 400 MB of fp32, rows of 64 of a pitch of 72
  // 159 / 169, 80 of 88 154 / 119, 100 of 104 149 / 110, 200 of 208 134 / 87, 333 of 336 127 / 91, 1000 of 1008 107 / 93 (all of the row past them: 100 of 104
  // 174, 200 of 208 136); without gaps, where the caches join the parts, 100 91 / 122, 333 92 / 129.
  const size_t row_bytes = size_t(F) * (grad_type == HGNN_F16 ? 2 : 4), pitch_bytes = size_t(lddt) * (grad_type == HGNN_F16 ? 2 : 4);
  const bool lines = row_bytes % 128 == 0 && pitch_bytes % 128 == 0 && (reinterpret_cast<uintptr_t>(dT) & 127u) == 0;
  const bool gaps = pitch_bytes > row_bytes && row_bytes >= 288;
  a.past = double(V) * pitch_bytes < kPastBytes ? 0 : lines && row_bytes >= 256 ? kPastAll : lines || gaps ? kPastZeros : 0;
  a.dY = reinterpret_cast<const half_t*>(dY), a.ldy = ldy, a.inside = extent_of(n, F, ldy), a.scale = scale;
  a.dT = dT, a.lddt = lddt, a.part = w.part, a.pitch = w.pitch;
  if (n > 0) {
    a.words = sort_words(IdWords{ids, V, a.pos_bits}, n, a.pos_bits, a.pos_bits + bits_of(int64_t(V) + 1), w.buf0, w.buf1, w.scratch, s);
    HGNN_LAUNCH_CHECK("the sort of the ids");
  }
  if (grad_type == HGNN_F16) return accumulate ? table_grad<half_t, true>(a, s) : table_grad<half_t, false>(a, s);
  return accumulate ? table_grad<float, true>(a, s) : table_grad<float, false>(a, s);
}

}  // extern "C"
