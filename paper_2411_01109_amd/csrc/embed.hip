// Rows of a learned vertex table by id, and the gradient of the table: what stands before the first layer of a graph without vertex features.
#include "common.h"
#include "rows.h"
#include "sort.h"

namespace hgnn {

struct LookupArgs {
  int64_t n;
  int F, V;
  const int* ids;
  const void* table;
  int64_t ldt;
  float scale;
  half_t* out;
  int64_t ldo;
};

// out[i] = scale * T[ids[i]]: L lanes take a row in pieces of eight.  Bound by memory.
template <class T, int L>
__global__ __launch_bounds__(kBlock) void embedding_kernel(LookupArgs a) {
  const int64_t i = (int64_t(blockIdx.x) * kBlock + threadIdx.x) / L;
  if (i >= a.n) return;
  const int id = a.ids[i];
  const bool real = uint32_t(id) < uint32_t(a.V);
  const T* const row = static_cast<const T*>(a.table) + int64_t(real ? id : 0) * a.ldt;
  half_t* const out = a.out + i * a.ldo;
  for (int f = 8 * (threadIdx.x % L); f < a.F; f += 8 * L) {
    Piece x{};
    if (real) x = load_piece(row + f, a.F - f, 0.f);
#pragma unroll
    for (int j = 0; j < 8; ++j) x.v[j] *= a.scale;
    store_piece(out + f, a.F - f, x);
  }
}

// ---- the gradient -------------------------------------------------------------------------------------------
// dT[v] = scale * sum of dY[i] over the i with ids[i] = v.  The positions are sorted by id (stable, so the rows of an id keep their order), the sorted list is cut
// into shares of T positions, and L lanes walk a share: a run of equal ids that begins and ends inside it is stored at once; what a share holds of a run that
// it shares with its neighbours is left as a partial sum in fp32, `head` of a run that began earlier, `tail` of one that goes on, and a second pass adds the
// partial sums of a run in order.  No atomics: the same bits on every run.  Rows without a position are zeros, which the workgroups behind those of the shares write.

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

struct TableGradArgs {
  const uint64_t* words;  // sorted
  int64_t n, shares;
  int pos_bits, T, F, V;
  const half_t* dY;
  int64_t ldy;
  float scale;
  void* dT;
  int64_t lddt;
  float* part;  // [shares][2][pitch]: head and tail
  int pitch;
  int64_t share_blocks;
  __device__ __forceinline__ int id(int64_t k) const { return int(words[k] >> pos_bits); }
  __device__ __forceinline__ int64_t pos(uint64_t w) const { return int64_t(w & ((uint64_t(1) << pos_bits) - 1)); }
  __device__ __forceinline__ float* partial(int64_t share, int tail) const { return part + (2 * share + tail) * pitch; }
};

template <class T, bool ADD>
__device__ __forceinline__ void add_row(const TableGradArgs& a, int id, int f, Piece x) {
  T* const p = static_cast<T*>(a.dT) + int64_t(id) * a.lddt + f;
#pragma unroll
  for (int j = 0; j < 8; ++j) x.v[j] *= a.scale;
  if (ADD) {
    const Piece y = load_piece(p, a.F - f, 0.f);
#pragma unroll
    for (int j = 0; j < 8; ++j) x.v[j] += y.v[j];
  }
  store_piece(p, a.F - f, x);
}

constexpr int kZeroRows = kWave;  // table rows of a wave that writes zeros

template <class T, bool ADD, int L>
__global__ __launch_bounds__(kBlock) void table_grad_kernel(TableGradArgs a) {
  if (int64_t(blockIdx.x) >= a.share_blocks) {  // zeros
    const int lane = threadIdx.x & (kWave - 1);
    const int64_t r0 = ((int64_t(blockIdx.x) - a.share_blocks) * kWavesPerBlock + threadIdx.x / kWave) * kZeroRows, r = r0 + lane;
    if (r0 >= a.V) return;
    int64_t lo = 0, hi = a.n;
    while (lo < hi) {
      const int64_t mid = (lo + hi) >> 1;
      if (a.id(mid) < r) lo = mid + 1;
      else hi = mid;
    }
    const uint64_t there = __ballot(r >= a.V || (lo < a.n && a.id(lo) == r));
    const int pieces = (a.F + 7) / 8;
    for (int k = 0; k < kZeroRows; ++k) {
      if (there >> k & 1) continue;
      T* const p = static_cast<T*>(a.dT) + (r0 + k) * a.lddt;
      for (int f = lane; f < pieces; f += kWave) store_piece(p + 8 * f, a.F - 8 * f, Piece{});
    }
    return;
  }
  const int64_t share = (int64_t(blockIdx.x) * kBlock + threadIdx.x) / L;
  if (share >= a.shares) return;
  const int64_t first = share * a.T, end = first + a.T < a.n ? first + a.T : a.n;
  const int before = first > 0 ? a.id(first - 1) : -1, after = end < a.n ? a.id(end) : -1;
  for (int f = 8 * (threadIdx.x % L); f < a.F; f += 8 * L) {
    int cur = -1;
    bool head = false;
    Piece sum{};
    auto done = [&](bool tail) {
      if (cur < 0 || cur >= a.V) return;
      if (head || tail) store_piece(a.partial(share, head ? 0 : 1) + f, sum);
      else add_row<T, ADD>(a, cur, f, sum);
    };
    for (int64_t k = first; k < end; ++k) {
      const uint64_t w = a.words[k];
      const int id = int(w >> a.pos_bits);
      if (id != cur) {
        done(false);
        cur = id;
        head = k == first && id == before;
        sum = Piece{};
      }
      if (id >= a.V) break;  // the rest are ids that are none
      const Piece x = load_piece(a.dY + a.pos(w) * a.ldy + f, a.F - f, 0.f);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum.v[j] += x.v[j];
    }
    done(cur == after);
  }
}

// The runs that several shares hold, by the share where a run begins.
template <class T, bool ADD, int L>
__global__ __launch_bounds__(kBlock) void table_grad_join_kernel(TableGradArgs a) {
  const int64_t share = (int64_t(blockIdx.x) * kBlock + threadIdx.x) / L;
  if (share >= a.shares - 1) return;
  const int64_t first = share * a.T, end = first + a.T;
  const int id = a.id(end);
  if (id >= a.V || a.id(end - 1) != id || (first > 0 && a.id(first - 1) == id && a.id(first) == id)) return;
  for (int f = 8 * (threadIdx.x % L); f < a.F; f += 8 * L) {
    Piece sum = load_piece(a.partial(share, 1) + f);
    for (int64_t s = share + 1; s < a.shares && a.id(s * a.T) == id; ++s) {
      const Piece x = load_piece(a.partial(s, 0) + f);
#pragma unroll
      for (int j = 0; j < 8; ++j) sum.v[j] += x.v[j];
    }
    add_row<T, ADD>(a, id, f, sum);
  }
}

static int bits_of(int64_t values) {  // that tell so many values apart
  int b = 1;
  while ((int64_t(1) << b) < values) ++b;
  return b;
}

constexpr int kShare = 16;

struct TableGradSpace {
  uint64_t *buf0, *buf1;
  void* scratch;
  float* part;
  int64_t shares;
  int T, pitch;
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
  p.T = kShare;
  p.shares = ceil_div(n, p.T);
  p.pitch = (F + 7) / 8 * 8;
  p.buf0 = reinterpret_cast<uint64_t*>(take(8 * size_t(n)));
  p.buf1 = reinterpret_cast<uint64_t*>(take(8 * size_t(n)));
  p.scratch = take(n > 0 ? sort_scratch_bytes(n) : 0);
  p.part = reinterpret_cast<float*>(take(2 * size_t(p.shares) * size_t(p.pitch) * sizeof(float)));
  p.bytes = size_t(at - static_cast<char*>(base));
  return p;
}

template <class Call>
static void with_lanes(int F, Call&& call) {  // lanes that take a row of F
  switch (pow2_at_least((F + 7) / 8)) {
    case 1: return call(std::integral_constant<int, 1>());
    case 2: return call(std::integral_constant<int, 2>());
    case 4: return call(std::integral_constant<int, 4>());
    case 8: return call(std::integral_constant<int, 8>());
    case 16: return call(std::integral_constant<int, 16>());
    case 32: return call(std::integral_constant<int, 32>());
    default: return call(std::integral_constant<int, 64>());
  }
}

template <class T, bool ADD>
static hgnn_status table_grad(const TableGradArgs& a, hipStream_t s) {
  hgnn_status st = HGNN_OK;
  with_lanes(a.F, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    TableGradArgs b = a;
    b.share_blocks = ceil_div(a.shares * L, kBlock);
    const int64_t zeros = ADD ? 0 : ceil_div(a.V, int64_t(kZeroRows) * kWavesPerBlock);
    auto go = [&]() -> hgnn_status {
      HGNN_REQUIRE(b.share_blocks + zeros <= 0x7fffffff, HGNN_EUNSUPPORTED, "hgnn_embedding_grad: grid too large");
      if (b.share_blocks + zeros > 0) {
        table_grad_kernel<T, ADD, L><<<dim3(unsigned(b.share_blocks + zeros)), kBlock, 0, s>>>(b);
        HGNN_LAUNCH_CHECK("table_grad_kernel");
      }
      if (a.shares > 1) {
        table_grad_join_kernel<T, ADD, L><<<dim3(unsigned(b.share_blocks)), kBlock, 0, s>>>(b);
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
  HGNN_REQUIRE(F <= 65536, HGNN_EUNSUPPORTED, "%s: F = %d above 65536", who, F);
  if (n == 0) return HGNN_OK;
  HGNN_REQUIRE(ids && out && (table || V == 0), HGNN_EINVAL, "%s: NULL argument", who);
  HGNN_REQUIRE(aligned_to_type(ids, HGNN_F32) && aligned_to_type(table, table_type) && aligned_to_type(out, HGNN_F16), HGNN_EINVAL,
               "%s: an array that is not aligned to its type", who);
  const LookupArgs a{n, F, V, ids, table, ldt, scale, reinterpret_cast<half_t*>(out), ldo};
  hgnn_status st = HGNN_OK;
  with_lanes(F, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    auto go = [&]() -> hgnn_status {
      HGNN_REQUIRE(n <= int64_t(0x7fffffff) * kBlock / L, HGNN_EUNSUPPORTED, "%s: grid too large", who);
      const dim3 grid{unsigned(ceil_div(n * L, kBlock))};
      hipStream_t s = static_cast<hipStream_t>(stream);
      if (table_type == HGNN_F16) embedding_kernel<half_t, L><<<grid, kBlock, 0, s>>>(a);
      else embedding_kernel<float, L><<<grid, kBlock, 0, s>>>(a);
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
  a.n = n, a.shares = w.shares, a.T = w.T, a.F = F, a.V = V;
  a.pos_bits = bits_of(n);
  a.dY = reinterpret_cast<const half_t*>(dY), a.ldy = ldy, a.scale = scale;
  a.dT = dT, a.lddt = lddt, a.part = w.part, a.pitch = w.pitch;
  if (n > 0) {
    a.words = sort_words(IdWords{ids, V, a.pos_bits}, n, a.pos_bits, a.pos_bits + bits_of(int64_t(V) + 1), w.buf0, w.buf1, w.scratch, s);
    HGNN_LAUNCH_CHECK("the sort of the ids");
  }
  if (grad_type == HGNN_F16) return accumulate ? table_grad<half_t, true>(a, s) : table_grad<half_t, false>(a, s);
  return accumulate ? table_grad<float, true>(a, s) : table_grad<float, false>(a, s);
}

}  // extern "C"
