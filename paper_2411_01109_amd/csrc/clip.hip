// The norm over all gradients of a step, and the gradients unscaled and clipped by it: what guards a step in half precision, whose gradients are scaled up to stay
// above the underflow of fp16 and may overflow for it.
#include <math.h>

#include <algorithm>
#include <vector>

#include "common.h"
#include "rows.h"

namespace hgnn {

// Tensors of a launch, by value: the arguments of a kernel hold some 4 KB.
constexpr int kClipTensors = 56;
constexpr int kClipChunk = 32768;  // elements of a workgroup's turn
constexpr int kClipParts = 1024;   // partial sums of squares, one for every workgroup

struct ClipTensor {
  const void* g;
  void* o;
  int64_t cols, ld, ldo;  // of rows; a tensor without gaps is one row
  int32_t rows, band;     // rows, rows of a chunk
  int32_t first;          // its first chunk in the launch
  int16_t g_type, o_type;
};
struct ClipArgs {
  ClipTensor t[kClipTensors];
  int count, chunks;
  double* part;
  int parts;
  int add;             // to what an earlier launch left
  float inv_scale, max_norm;
  float* norm;
};

// the elements of chunk c, row by row in pieces of eight: f(tensor, row, column, columns left)
template <class Piecewise>
__device__ __forceinline__ void walk_chunk(const ClipArgs& a, int c, Piecewise&& f) {
  int i = 0;
  for (int step = 32; step > 0; step >>= 1)  // the last tensor that begins at or before c
    if (i + step < a.count && a.t[i + step].first <= c) i += step;
  const ClipTensor& t = a.t[i];
  const int k = c - t.first;
  if (t.rows == 1) {
    const int64_t c0 = int64_t(k) * kClipChunk, c1 = c0 + kClipChunk < t.cols ? c0 + kClipChunk : t.cols;
    for (int64_t p = c0 + 8 * threadIdx.x; p < c1; p += 8 * kBlock) f(t, 0, p, int(c1 - p));
    return;
  }
  // a band of rows; rows that are longer than a chunk alone
  const int r0 = k * t.band, nr = min(t.band, t.rows - r0);
  const uint32_t per = uint32_t((t.cols + 7) / 8);
  if (nr == 1) {
    for (uint32_t p = threadIdx.x; p < per; p += kBlock) f(t, r0, int64_t(8) * p, int(min(t.cols - int64_t(8) * p, int64_t(8))));
    return;
  }
  for (uint32_t q = threadIdx.x; q < per * uint32_t(nr); q += kBlock) {
    const uint32_t r = q / per, p = q - r * per;
    f(t, r0 + int(r), int64_t(8) * p, int(t.cols - int64_t(8) * p));
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

// Sums of squares, in 64 bits: squares of fp32 leave its range at 1.8e19, and a long sum its precision.  A workgroup's sum is its own slot's, so launches of one call
// add in order and the bits are the same on every run.
__global__ __launch_bounds__(kBlock) void grad_squares_kernel(ClipArgs a) {
  double sum = 0;
  for (int c = blockIdx.x; c < a.chunks; c += gridDim.x)
    walk_chunk(a, c, [&](const ClipTensor& t, int64_t row, int64_t col, int left) {
      if (t.g_type == HGNN_F16) {
        const Piece x = load_piece(static_cast<const half_t*>(t.g) + row * t.ld + col, left, 0.f);
        float s = 0.f;  // at most 3.5e10
#pragma unroll
        for (int j = 0; j < 8; ++j) s = fmaf(x.v[j], x.v[j], s);
        sum += s;
      } else {
        const Piece x = load_piece(static_cast<const float*>(t.g) + row * t.ld + col, left, 0.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fma(double(x.v[j]), double(x.v[j]), sum);
      }
    });
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

template <class I, class O>
__device__ __forceinline__ void clip_piece(const ClipTensor& t, int64_t row, int64_t col, int left, float factor) {
  Piece x{};
  if (factor != 0.f) x = load_piece(static_cast<const I*>(t.g) + row * t.ld + col, left, 0.f);
#pragma unroll
  for (int j = 0; j < 8; ++j) x.v[j] *= factor;
  store_piece(static_cast<O*>(t.o) + row * t.ldo + col, left, x);
}

__global__ __launch_bounds__(kBlock) void grad_clip_kernel(ClipArgs a) {
  const double norm = norm_of(a);
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = float(norm);
  // a norm that is none: zeros, so that a step that nobody looks at adds nothing
  double f = isfinite(float(norm)) ? double(a.inv_scale) : 0.;
  if (norm > double(a.max_norm)) f *= double(a.max_norm) / norm;
  const float factor = float(f);
  for (int c = blockIdx.x; c < a.chunks; c += gridDim.x)
    walk_chunk(a, c, [&](const ClipTensor& t, int64_t row, int64_t col, int left) {
      if (t.g_type == HGNN_F16) {
        if (t.o_type == HGNN_F16) clip_piece<half_t, half_t>(t, row, col, left, factor);
        else clip_piece<half_t, float>(t, row, col, left, factor);
      } else {
        if (t.o_type == HGNN_F16) clip_piece<float, half_t>(t, row, col, left, factor);
        else clip_piece<float, float>(t, row, col, left, factor);
      }
    });
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
    HGNN_REQUIRE(t.rows == 1 || t.cols < (int64_t(1) << 31), HGNN_EUNSUPPORTED, "%s: tensor %d: rows of more than int32", who, i);
    if (!clip || !t.out) continue;
    HGNN_REQUIRE(known_type(t.out_type), HGNN_EINVAL, "%s: tensor %d: unknown type %d", who, i, int(t.out_type));
    HGNN_REQUIRE(t.ld_out >= t.cols, HGNN_EINVAL, "%s: tensor %d: leading dimension of the output smaller than the row", who, i);
    HGNN_REQUIRE(aligned_to_type(t.out, t.out_type), HGNN_EINVAL, "%s: tensor %d: an output that is not aligned to its type", who, i);
    HGNN_REQUIRE(t.out != t.grad || (t.type == t.out_type && t.ld == t.ld_out), HGNN_EINVAL, "%s: tensor %d: in place as another type or with another leading dimension", who, i);
  }
  return HGNN_OK;
}

static hgnn_status check_outputs(const char* who, int32_t count, const hgnn_grad* g) {
  std::vector<const void*> outs;
  outs.reserve(size_t(count));
  for (int i = 0; i < count; ++i)
    if (g[i].rows > 0 && g[i].cols > 0) outs.push_back(g[i].out ? g[i].out : g[i].grad);
  std::sort(outs.begin(), outs.end());
  HGNN_REQUIRE(std::adjacent_find(outs.begin(), outs.end()) == outs.end(), HGNN_EINVAL, "%s: the same output twice", who);
  return HGNN_OK;
}

// launches f(arguments, workgroups) over the tensors, as many at a time as the arguments hold
template <class Launch>
static hgnn_status over_tensors(const char* who, int32_t count, const hgnn_grad* g, bool clip, ClipArgs& a, Launch&& f) {
  int i = 0;
  while (i < count) {
    a.count = 0;
    int64_t chunks = 0;
    for (; i < count && a.count < kClipTensors; ++i) {
      const hgnn_grad& q = g[i];
      if (q.rows == 0 || q.cols == 0) continue;
      ClipTensor t{q.grad, clip && q.out ? q.out : const_cast<void*>(q.grad), q.cols, q.ld, clip && q.out ? q.ld_out : q.ld, int32_t(q.rows), 1, 0, int16_t(q.type),
                   int16_t(clip && q.out ? q.out_type : q.type)};
      if (t.rows > 1 && t.ld == t.cols && (!clip || t.ldo == t.cols)) t.cols *= t.rows, t.rows = 1;
      int64_t n;
      if (t.rows == 1) {
        n = ceil_div(t.cols, kClipChunk);
      } else {
        t.band = int32_t(std::max<int64_t>(1, kClipChunk / ((t.cols + 7) / 8 * 8)));
        n = ceil_div(t.rows, t.band);
      }
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
  return over_tensors(who, count, grads, true, a, [&](unsigned blocks) -> hgnn_status {
    grad_clip_kernel<<<dim3(blocks), kBlock, 0, s>>>(a);
    HGNN_LAUNCH_CHECK("grad_clip_kernel");
    return HGNN_OK;
  });
}

}  // extern "C"
