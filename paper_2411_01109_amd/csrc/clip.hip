// The norm over all gradients of a step, and the gradients unscaled and clipped by it: what guards a step in half precision, whose gradients are scaled up to stay
// above the underflow of fp16 and may overflow for it.
#include <math.h>

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

#include "common.h"
#include "rows.h"

namespace hgnn {

// Tensors of a launch, by value: the arguments of a kernel hold 4 KB, and a launch costs the host 3 us and more (200 tensors: eight launches of 56 39 us, four
// of 96 27).
constexpr int kClipTensors = 96;
constexpr int kClipParts = 1024;   // partial sums of squares at most, one for every workgroup
// Elements of a workgroup's turn, a multiple of kClipChunk: as many as give every workgroup one, at most kClipMost.
constexpr int kClipChunk = 8 * kBlock, kClipMost = 16 * kClipChunk;
constexpr int kClipAhead = 4;  // pieces of a lane that are fetched together

struct ClipTensor {
  const void* g;
  void* o;
  int64_t cols;               // of rows; a tensor without gaps is one row
  int32_t rows;
  int32_t first;              // its first chunk in the launch
  uint32_t g_pad, o_pad;      // elements between rows, and in the highest bit the type
  __device__ __forceinline__ int64_t ld() const { return cols + (g_pad & 0x7fffffffu); }
  __device__ __forceinline__ int64_t ldo() const { return cols + (o_pad & 0x7fffffffu); }
  __device__ __forceinline__ hgnn_type g_type() const { return hgnn_type(g_pad >> 31); }
  __device__ __forceinline__ hgnn_type o_type() const { return hgnn_type(o_pad >> 31); }
};
// rows of a chunk of a tensor with gaps
__host__ __device__ inline int band_of(int64_t cols, int chunk) {
  const int64_t padded = (cols + 7) / 8 * 8;
  return padded >= chunk ? 1 : chunk / int(padded);
}
struct ClipArgs {
  ClipTensor t[kClipTensors];
  int count, chunks, chunk;
  double* part;
  int parts;
  int add;             // to what an earlier launch left
  float inv_scale, max_norm;
  float* norm;
};

__device__ __forceinline__ const ClipTensor& tensor_of(const ClipArgs& a, int c) {  // the last one that begins at or before chunk c
  int i = 0;
  for (int step = 64; step > 0; step >>= 1)
    if (i + step < a.count && a.t[i + step].first <= c) i += step;
  return a.t[i];
}

// The elements of chunk c of a tensor, row by row in pieces of V, several of a lane's fetched together: use(row, column, columns left, piece).  V: 16 bytes of
// the wider of what is read and written, so that the lanes' 16 bytes lie beside each other.
template <class I, int V, class Use>
__device__ __forceinline__ void walk_chunk(const ClipArgs& a, const ClipTensor& t, int c, Use&& use) {
  constexpr int kAhead = kClipAhead * 8 / V, kTurn = V * kBlock;
  typedef Part<I, V> P;
  const int k = c - t.first;
  const I* const g = static_cast<const I*>(t.g);
  if (t.rows == 1) {
    const int64_t c0 = int64_t(k) * a.chunk, c1 = c0 + a.chunk < t.cols ? c0 + a.chunk : t.cols;
    int64_t p = c0 + V * threadIdx.x;
    for (; p + kTurn * (kAhead - 1) + V <= c1; p += kTurn * kAhead) {
      P x[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) x[i] = P::load(g + p + i * kTurn);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) use(0, p + i * kTurn, V, x[i]);
    }
    for (; p < c1; p += kTurn) use(0, p, int(c1 - p), P::load(g + p, int(c1 - p), c1 - p));
    return;
  }
  // A band of rows; rows that are longer than a chunk alone.  A lane has one piece on its way: us, fp32 in place, 2.4 M x 100 of a pitch of 104 / without gaps 607 / 541,
  // 100 000 x 42 of 48 24.5 / 19.0.
  const int band = band_of(t.cols, a.chunk), r0 = k * band, nr = min(band, t.rows - r0);
  const uint32_t per = uint32_t((t.cols + V - 1) / V);
  for (uint32_t q = threadIdx.x; q < per * uint32_t(nr); q += kBlock) {
    const uint32_t r = nr == 1 ? 0 : q / per;
    const int64_t row = r0 + int(r), col = int64_t(V) * (q - r * per);
    const int left = int(t.cols - col < V ? t.cols - col : V);
    use(row, col, left, P::load(g + row * t.ld() + col, left, left));
  }
}

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double s[kWavesPerBlock];
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & (kWave - 1)) == 0) s[threadIdx.x / kWave] = v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int w = 0; w < kWavesPerBlock; ++w) v += s[w];
  return v;
}

// Sums of squares, in 64 bits: squares of fp32 leave its range at 1.8e19, and a long sum its precision.  A workgroup's sum is its own slot's, so launches of
// one call add in order and the bits are the same on every run.
__global__ __launch_bounds__(kBlock) void grad_squares_kernel(ClipArgs a) {
  double sum = 0;
  for (int c = blockIdx.x; c < a.chunks; c += gridDim.x) {
    const ClipTensor& t = tensor_of(a, c);
    if (t.g_type() == HGNN_F16) {
      walk_chunk<half_t, 8>(a, t, c, [&](int64_t, int64_t, int, const Part<half_t, 8>& x) __attribute__((always_inline)) {
        float s = 0.f;  // at most 3.5e10
#pragma unroll
        for (int j = 0; j < 8; ++j) s = fmaf(float(x.v[j]), float(x.v[j]), s);
        sum += s;
      });
    } else {
      walk_chunk<float, 4>(a, t, c, [&](int64_t, int64_t, int, const Part<float, 4>& x) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sum = fma(double(x.v[j]), double(x.v[j]), sum);
      });
    }
  }
  sum = block_sum(sum);
  if (threadIdx.x == 0) a.part[blockIdx.x] = a.add ? a.part[blockIdx.x] + sum : sum;
}

// the norm from the partial sums, by a workgroup
__device__ __forceinline__ double norm_of(const ClipArgs& a) {
  double sum = 0;
  for (int i = threadIdx.x; i < a.parts; i += kBlock) sum += a.part[i];
  return sqrt(block_sum(sum)) * double(a.inv_scale);
}
__global__ __launch_bounds__(kBlock) void grad_norm_kernel(ClipArgs a) {
  const double norm = norm_of(a);
  if (threadIdx.x == 0) *a.norm = float(norm);
}

// What gradients are multiplied by: factor 2^exponent.  The exponent is not zero only below 2^-100, where the factor alone may leave fp32's normal numbers though
// the products do not (gradients near the largest fp32 values): there it is a number of [0.5, 1), whose product with a gradient is exact to its rounding.
struct ClipFactor {
  float factor;
  int exponent;
  __device__ __forceinline__ explicit ClipFactor(double f) : factor(float(f)), exponent(0) {
    if (f < 0x1p-100) factor = float(frexp(f, &exponent));
  }
  __device__ __forceinline__ float of(float g) const { return factor == 0.f ? 0.f : __builtin_ldexpf(g * factor, exponent); }
};

template <class I, class O, bool PAST>
__device__ __forceinline__ void clip_chunk(const ClipArgs& a, const ClipTensor& t, int c, const ClipFactor& factor) {
  constexpr int V = sizeof(I) == 2 && sizeof(O) == 2 ? 8 : 4;
  walk_chunk<I, V>(a, t, c, [&](int64_t row, int64_t col, int left, const Part<I, V>& x) __attribute__((always_inline)) {
    O* const o = static_cast<O*>(t.o) + row * t.ldo() + col;
    float y[V];
#pragma unroll
    for (int j = 0; j < V; ++j) y[j] = factor.of(float(x.v[j]));
    Part<O, V>::template store<PAST>(o, left, y);
  });
}

template <bool PAST>
__global__ __launch_bounds__(kBlock) void grad_clip_kernel(ClipArgs a) {
  const double norm = norm_of(a);
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = float(norm);
  // a norm that is none: zeros, so that a step that nobody looks at adds nothing
  double f = isfinite(float(norm)) ? double(a.inv_scale) : 0.;
  if (norm > double(a.max_norm)) f *= double(a.max_norm) / norm;
  const ClipFactor factor(f);
  // from the end: what the sums of squares read last is still in the last-level cache
  for (int c = a.chunks - 1 - int(blockIdx.x); c >= 0; c -= gridDim.x) {
    const ClipTensor& t = tensor_of(a, c);
    if (t.g_type() == HGNN_F16) {
      if (t.o_type() == HGNN_F16) clip_chunk<half_t, half_t, PAST>(a, t, c, factor);
      else clip_chunk<half_t, float, PAST>(a, t, c, factor);
    } else {
      if (t.o_type() == HGNN_F16) clip_chunk<float, half_t, PAST>(a, t, c, factor);
      else clip_chunk<float, float, PAST>(a, t, c, factor);
    }
  }
}

static hgnn_status check_grads(const char* who, int32_t count, const hgnn_grad* g, bool clip) {
  HGNN_REQUIRE(count >= 0 && (g || count == 0), HGNN_EINVAL, "%s: count = %d, grads %s", who, count, g ? "given" : "NULL");
  for (int i = 0; i < count; ++i) {
    const hgnn_grad& t = g[i];
    HGNN_REQUIRE(t.rows >= 0 && t.cols >= 0 && t.rows <= 0x7fffffff && t.cols < (int64_t(1) << 40), HGNN_EINVAL, "%s: tensor %d: %lld rows of %lld", who, i,
                 static_cast<long long>(t.rows), static_cast<long long>(t.cols));
    HGNN_REQUIRE(known_type(t.type), HGNN_EINVAL, "%s: tensor %d: unknown type %d", who, i, int(t.type));
    HGNN_REQUIRE(t.ld >= t.cols, HGNN_EINVAL, "%s: tensor %d: leading dimension smaller than the row", who, i);
    if (t.rows == 0 || t.cols == 0) continue;
    HGNN_REQUIRE(t.grad && aligned_to_type(t.grad, t.type), HGNN_EINVAL, "%s: tensor %d: NULL, or not aligned to its type", who, i);
    HGNN_REQUIRE(t.rows == 1 || (t.cols < (int64_t(1) << 31) && t.ld - t.cols < (int64_t(1) << 31)), HGNN_EUNSUPPORTED, "%s: tensor %d: rows of more than int32", who, i);
    if (!clip || !t.out) continue;
    HGNN_REQUIRE(known_type(t.out_type), HGNN_EINVAL, "%s: tensor %d: unknown type %d", who, i, int(t.out_type));
    HGNN_REQUIRE(t.ld_out >= t.cols, HGNN_EINVAL, "%s: tensor %d: leading dimension of the output smaller than the row", who, i);
    HGNN_REQUIRE(t.rows == 1 || t.ld_out - t.cols < (int64_t(1) << 31), HGNN_EUNSUPPORTED, "%s: tensor %d: rows of more than int32", who, i);
    HGNN_REQUIRE(aligned_to_type(t.out, t.out_type), HGNN_EINVAL, "%s: tensor %d: an output that is not aligned to its type", who, i);
    HGNN_REQUIRE(t.out != t.grad || (t.type == t.out_type && t.ld == t.ld_out), HGNN_EINVAL, "%s: tensor %d: in place as another type or with another leading dimension", who, i);
  }
  return HGNN_OK;
}

static hgnn_status check_outputs(const char* who, int32_t count, const hgnn_grad* g) {
  if (count < 2) return HGNN_OK;
  const std::unique_ptr<const void*[]> outs(new (std::nothrow) const void*[size_t(count)]);
  HGNN_REQUIRE(outs != nullptr, HGNN_ENOMEM, "%s: host allocation failed", who);
  const void** end = outs.get();
  for (int i = 0; i < count; ++i)
    if (g[i].rows > 0 && g[i].cols > 0) *end++ = g[i].out ? g[i].out : g[i].grad;
  std::sort(outs.get(), end);
  HGNN_REQUIRE(std::adjacent_find(outs.get(), end) == end, HGNN_EINVAL, "%s: the same output twice", who);
  return HGNN_OK;
}

// launches f(arguments, workgroups) over the tensors, as many at a time as the arguments hold
template <class Launch>
static hgnn_status over_tensors(const char* who, int32_t count, const hgnn_grad* g, bool clip, ClipArgs& a, Launch&& f) {
  double total = 0;
  for (int i = 0; i < count; ++i) total += double(g[i].rows) * double(g[i].cols);
  a.chunk = kClipChunk * int(std::min<double>(kClipMost / kClipChunk, std::ceil(std::max(total, 1.) / (double(kClipParts) * kClipChunk))));
  int i = 0;
  while (i < count) {
    a.count = 0;
    int64_t chunks = 0;
    for (; i < count && a.count < kClipTensors; ++i) {
      const hgnn_grad& q = g[i];
      if (q.rows == 0 || q.cols == 0) continue;
      const bool out = clip && q.out;
      const hgnn_type o_type = out ? q.out_type : q.type;
      int64_t rows = q.rows, cols = q.cols, g_pad = q.ld - q.cols, o_pad = (out ? q.ld_out : q.ld) - q.cols;
      if (rows == 1 || (g_pad == 0 && (!clip || o_pad == 0))) cols *= rows, rows = 1, g_pad = o_pad = 0;
      const int64_t n = rows == 1 ? ceil_div(cols, a.chunk) : ceil_div(rows, band_of(cols, a.chunk));
      ClipTensor t{q.grad, out ? q.out : const_cast<void*>(q.grad), cols, int32_t(rows), 0, uint32_t(g_pad) | uint32_t(q.type) << 31,
                   uint32_t(clip ? o_pad : 0) | uint32_t(o_type) << 31};
      HGNN_REQUIRE(chunks + n <= 0x7fffffff, HGNN_EUNSUPPORTED, "%s: tensor %d is too large", who, i);
      t.first = int32_t(chunks);
      chunks += n;
      a.t[a.count++] = t;
    }
    if (a.count == 0) break;
    a.chunks = int(chunks);
    const hgnn_status st = f(unsigned(std::min<int64_t>(chunks, kClipParts)));
    if (st != HGNN_OK) return st;
  }
  return HGNN_OK;
}

// the partial sums of squares, a.parts of them
static hgnn_status grad_squares(const char* who, int32_t count, const hgnn_grad* g, ClipArgs& a, hipStream_t s) {
  a.parts = 0;
  return over_tensors(who, count, g, false, a, [&](unsigned blocks) -> hgnn_status {
    // a later launch adds to what an earlier one left, so the first of several writes all slots
    a.add = a.parts > 0;
    if (!a.add) a.parts = count > kClipTensors ? kClipParts : int(blocks);
    grad_squares_kernel<<<dim3(a.add ? blocks : unsigned(a.parts)), kBlock, 0, s>>>(a);
    HGNN_LAUNCH_CHECK("grad_squares_kernel");
    return HGNN_OK;
  });
}

static hgnn_status check_norm(const char* who, float inv_scale, const float* norm, const void* workspace, size_t workspace_bytes) {
  HGNN_REQUIRE(inv_scale > 0.f && inv_scale < INFINITY, HGNN_EINVAL, "%s: inv_scale = %g", who, double(inv_scale));
  HGNN_REQUIRE(norm != nullptr && aligned_to_type(norm, HGNN_F32), HGNN_EINVAL, "%s: norm is NULL or not aligned", who);
  HGNN_REQUIRE(workspace != nullptr && workspace_bytes >= hgnn_grad_norm_workspace() && (reinterpret_cast<uintptr_t>(workspace) & 7u) == 0, HGNN_EINVAL,
               "%s: workspace of %zu bytes, needs %zu aligned to 8 (hgnn_grad_norm_workspace)", who, workspace_bytes, hgnn_grad_norm_workspace());
  return HGNN_OK;
}

}  // namespace hgnn

using namespace hgnn;

extern "C" {

size_t hgnn_grad_norm_workspace(void) { return kClipParts * sizeof(double); }

hgnn_status hgnn_grad_norm(int32_t count, const hgnn_grad* grads, float inv_scale, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  const char* who = "hgnn_grad_norm";
  hgnn_status st = check_grads(who, count, grads, false);
  if (st == HGNN_OK) st = check_norm(who, inv_scale, norm, workspace, workspace_bytes);
  if (st != HGNN_OK) return st;
  ClipArgs a;
  a.part = static_cast<double*>(workspace), a.inv_scale = inv_scale, a.max_norm = INFINITY, a.norm = norm;
  hipStream_t s = static_cast<hipStream_t>(stream);
  st = grad_squares(who, count, grads, a, s);
  if (st != HGNN_OK) return st;
  grad_norm_kernel<<<1, kBlock, 0, s>>>(a);
  HGNN_LAUNCH_CHECK("grad_norm_kernel");
  return HGNN_OK;
}

hgnn_status hgnn_grad_clip(int32_t count, const hgnn_grad* grads, float inv_scale, float max_norm, float* norm, void* workspace, size_t workspace_bytes,
                           void* stream) {
  clear_error();
  const char* who = "hgnn_grad_clip";
  hgnn_status st = check_grads(who, count, grads, true);
  if (st == HGNN_OK) st = check_outputs(who, count, grads);
  if (st == HGNN_OK) st = check_norm(who, inv_scale, norm, workspace, workspace_bytes);
  if (st != HGNN_OK) return st;
  HGNN_REQUIRE(max_norm >= 0.f, HGNN_EINVAL, "%s: max_norm = %g", who, double(max_norm));
  ClipArgs a;
  a.part = static_cast<double*>(workspace), a.inv_scale = inv_scale, a.max_norm = max_norm, a.norm = norm;
  hipStream_t s = static_cast<hipStream_t>(stream);
  st = grad_squares(who, count, grads, a, s);
  if (st != HGNN_OK) return st;
  if (a.parts == 0) {  // no elements
    grad_norm_kernel<<<1, kBlock, 0, s>>>(a);
    HGNN_LAUNCH_CHECK("grad_norm_kernel");
    return HGNN_OK;
  }
  // Large outputs are written past the caches.  us, fp32 to fp32, through / past: 307 M elements 677 / 647, 60 M 146 / 116; fp16 to fp32, 307 M 471 / 424.
  double bytes = 0;
  for (int i = 0; i < count; ++i) bytes += double(grads[i].rows) * double(grads[i].cols) * ((grads[i].out ? grads[i].out_type : grads[i].type) == HGNN_F32 ? 4 : 2);
  const bool past = bytes >= kPastBytes;
  return over_tensors(who, count, grads, true, a, [&](unsigned blocks) -> hgnn_status {
    if (past) grad_clip_kernel<true><<<dim3(blocks), kBlock, 0, s>>>(a);
    else grad_clip_kernel<false><<<dim3(blocks), kBlock, 0, s>>>(a);
    HGNN_LAUNCH_CHECK("grad_clip_kernel");
    return HGNN_OK;
  });
}

}  // extern "C"
