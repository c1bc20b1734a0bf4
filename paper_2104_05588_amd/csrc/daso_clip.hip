// The norm of an averaged gradient over many tensors, and its clipping (daso_block.h).  Bound by memory:
// one pass reads the g replicas, sums the squares of their mean in 64 bits (where no square of a
// binary32 value overflows or vanishes) and writes the mean; a second one, whose workgroups all add the chunks'
// partial sums in the same fixed order for themselves, scales it.  Nothing waits for another workgroup.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "daso_block_host.h"
#include "daso_planes.h"

namespace daso {
namespace {

using host::ClipTable;

constexpr int kThreads = 256;

struct Norm {
  ClipTable table;
  int64_t chunk;
  double* partial;  // of the launch's first chunk
  float* mean;      // or null
  int32_t g;
};

struct Scale {
  ClipTable table;
  int64_t chunk, chunks;  // of all launches
  const double* partial;
  int64_t first;     // of the launch's partials
  const float* mean;
  float *out, *norm, *norms;
  float max_norm, eps;
  int32_t ready;     // out holds the mean
};

// Places of grads beyond the argument struct's: they are handed over apart, as their number varies.
struct Grads {
  const float* of[DASO_MAX_G];
};

// The run that a chunk of the launch is of: the last one whose first chunk is not beyond it (gaps have none).
__device__ inline int run_of(const ClipTable& t, int chunk) {
  int lo = 0, hi = t.runs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= chunk) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

struct Range {
  int64_t from, to;  // elements
};
__device__ inline Range range_of(const ClipTable& t, int64_t chunk, int at) {
  const int run = run_of(t, at);
  Range r;
  r.from = t.bound[run] + (at - t.first[run]) * chunk;
  r.to = min(r.from + chunk, t.bound[run + 1]);
  return r;
}

__device__ inline double square(float v) {
  const double d = v;
  return d * d;
}

// The mean of the replicas, in their order, as the fused step has it.  G: their number, or 0 for any.
template <int G>
__device__ inline f4v mean4(const Grads& g, int32_t count, int64_t j) {
  f4v v[G > 0 ? G : 1];
  f4v sum;
  if constexpr (G > 0) {
#pragma unroll
    for (int r = 0; r < G; ++r) v[r] = load4(g.of[r] + j);
    sum = v[0];
#pragma unroll
    for (int r = 1; r < G; ++r) sum += v[r];
    if constexpr (G == 1) return sum;
    if constexpr ((G & (G - 1)) == 0) return sum * (1.0f / G);  // exact, as the division is
    return sum / static_cast<float>(G);
  } else {
    sum = load4(g.of[0] + j);
    for (int r = 1; r < count; ++r) sum += load4(g.of[r] + j);
    return sum / static_cast<float>(count);
  }
}
__device__ inline float mean1(const Grads& g, int32_t count, int64_t j) {
  float sum = g.of[0][j];
  for (int r = 1; r < count; ++r) sum += g.of[r][j];
  return count > 1 ? sum / static_cast<float>(count) : sum;
}

template <int G>
__global__ __launch_bounds__(kThreads) void norm_kernel(Norm a, Grads g) {
  __shared__ double shared[kThreads / 64];
  const Range r = range_of(a.table, a.chunk, blockIdx.x);
  const int64_t from4 = (r.from + 3) / 4, to4 = max(r.to / 4, from4);  // whole vectors
  constexpr int kAhead = G == 0 ? 1 : G >= 4 ? 2 : 4;
  double sum = 0.0;
  for (int64_t i = from4 + threadIdx.x; i < to4; i += kThreads * kAhead) {
    f4v v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v[k] = mean4<G>(g, a.g, min(i + k * kThreads, to4 - 1) * 4);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i + k * kThreads >= to4) break;
      if (a.mean != nullptr) *(f4v*)(a.mean + (i + k * kThreads) * 4) = v[k];
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += square(v[k][j]);
    }
  }
  // up to three elements before the first vector, and three behind the last
  int64_t j = -1;
  if (threadIdx.x < 3) j = r.from + threadIdx.x < min(from4 * 4, r.to) ? r.from + threadIdx.x : -1;
  else if (threadIdx.x < 6) j = max(to4 * 4, r.from) + (threadIdx.x - 3) < r.to ? max(to4 * 4, r.from) + (threadIdx.x - 3) : -1;
  if (threadIdx.x >= 3 && from4 * 4 > r.to) j = -1;
  if (j >= 0) {
    const float v = mean1(g, a.g, j);
    if (a.mean != nullptr) a.mean[j] = v;
    sum += square(v);
  }
  sum = group_sum(sum, shared);
  if (threadIdx.x == 0) a.partial[blockIdx.x] = sum;
}

// The sum of partials, the same in every thread of every workgroup that asks.
__device__ inline double sum_of(const double* p, int64_t count, double* shared) {
  double sum = 0.0;
  for (int64_t i = threadIdx.x; i < count; i += kThreads) sum += p[i];
  return group_sum(sum, shared);
}

__global__ __launch_bounds__(kThreads) void scale_kernel(Scale a) {
  __shared__ double shared[kThreads / 64];
  const double norm = sqrt(sum_of(a.partial, a.chunks, shared));
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.norm != nullptr) *a.norm = static_cast<float>(norm);
  const int run = blockIdx.x;
  if (a.norms != nullptr && run < a.table.runs && a.table.number[run] >= 0) {
    __syncthreads();
    const int from = a.table.first[run];
    const double of = sqrt(sum_of(a.partial + a.first + from, a.table.first[run + 1] - from, shared));
    if (threadIdx.x == 0) a.norms[a.table.tensor + a.table.number[run]] = static_cast<float>(of);
  }
  if (a.out == nullptr || static_cast<int>(blockIdx.x) >= a.table.first[a.table.runs]) return;
  const double f = static_cast<double>(a.max_norm) / (norm + static_cast<double>(a.eps));
  const float factor = f >= 1.0 ? 1.0f : static_cast<float>(f);
  if (a.ready && factor == 1.0f) return;
  const Range r = range_of(a.table, a.chunk, blockIdx.x);
  const int64_t from4 = (r.from + 3) / 4, to4 = max(r.to / 4, from4);
  constexpr int kAhead = 4;
  for (int64_t i = from4 + threadIdx.x; i < to4; i += kThreads * kAhead) {
    f4v v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v[k] = load4(a.mean + min(i + k * kThreads, to4 - 1) * 4);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i + k * kThreads < to4) *(f4v*)(a.out + (i + k * kThreads) * 4) = v[k] * factor;
  }
  for (int64_t j = r.from + threadIdx.x; j < min(from4 * 4, r.to); j += kThreads) a.out[j] = a.mean[j] * factor;
  if (from4 * 4 <= r.to)
    for (int64_t j = max(to4 * 4, r.from) + threadIdx.x; j < r.to; j += kThreads) a.out[j] = a.mean[j] * factor;
}

size_t workspace_of(const daso_clip_args& s) { return static_cast<size_t>(host::plan_clip(s).chunks) * sizeof(double); }

}  // namespace
}  // namespace daso

extern "C" {

int daso_clip_gradients_workspace(const daso_clip_args* args, size_t* bytes) {
  if (args == nullptr || bytes == nullptr) return DASO_EINVAL;
  const int rc = daso::host::check_clip_sizes(*args);
  if (rc != DASO_OK) return rc;
  *bytes = daso::workspace_of(*args);
  return DASO_OK;
}

int daso_clip_gradients(const daso_clip_args* args, hipStream_t stream) {
  if (args == nullptr) return DASO_EINVAL;
  const daso_clip_args& s = *args;
  int rc = daso::host::check_clip(s);
  if (rc != DASO_OK) return rc;
  if ((rc = daso::host::check_workspace(s.workspace, s.workspace_bytes, daso::workspace_of(s))) != DASO_OK) return rc;
  if ((rc = daso::current_device(stream)) != DASO_OK) return rc;
  const daso::host::ClipPlan plan = daso::host::plan_clip(s);
  const int32_t count = s.ntensors > 0 ? s.ntensors : 1;
  double* const partial = static_cast<double*>(s.workspace);
  daso::Grads g = {};
  for (int32_t r = 0; r < s.g && s.n > 0; ++r) g.of[r] = s.grads[r];
  hipError_t err = hipSuccess;
  daso::Norm a;
  a.chunk = plan.chunk, a.g = s.g, a.mean = s.g > 1 ? s.out : nullptr;
  int64_t first = 0;
  for (int32_t t = 0; t < count && plan.chunks > 0 && err == hipSuccess;) {
    t += daso::host::fill_table(s, plan.chunk, t, &a.table);
    const int32_t chunks = a.table.first[a.table.runs];
    a.partial = partial + first;
    first += chunks;
    if (chunks == 0) continue;
    const dim3 grid(static_cast<uint32_t>(chunks)), block(daso::kThreads);
    switch (s.g) {
      case 1: err = daso::launch(&daso::norm_kernel<1>, grid, block, stream, a, g); break;
      case 2: err = daso::launch(&daso::norm_kernel<2>, grid, block, stream, a, g); break;
      case 3: err = daso::launch(&daso::norm_kernel<3>, grid, block, stream, a, g); break;
      case 4: err = daso::launch(&daso::norm_kernel<4>, grid, block, stream, a, g); break;
      case 8: err = daso::launch(&daso::norm_kernel<8>, grid, block, stream, a, g); break;
      default: err = daso::launch(&daso::norm_kernel<0>, grid, block, stream, a, g);
    }
  }
  daso::Scale b;
  b.chunk = plan.chunk, b.chunks = plan.chunks, b.partial = partial, b.first = 0;
  b.mean = s.g > 1 ? s.out : g.of[0];
  b.out = s.out, b.norm = s.norm, b.norms = s.norms, b.max_norm = s.max_norm, b.eps = s.eps;
  b.ready = s.g > 1 || s.out == g.of[0];
  for (int32_t t = 0; t < count && err == hipSuccess;) {
    t += daso::host::fill_table(s, plan.chunk, t, &b.table);
    const int32_t chunks = b.table.first[b.table.runs];
    // without elements to scale the launch has the norms alone to write
    const int32_t groups = std::max(s.out != nullptr ? chunks : 0, s.norms != nullptr ? b.table.runs : 1);
    err = daso::launch(&daso::scale_kernel, dim3(static_cast<uint32_t>(groups)), dim3(daso::kThreads), stream, b);
    b.first += chunks;
    b.norm = nullptr;
    if (s.out == nullptr && s.norms == nullptr) break;
  }
  return err == hipSuccess ? DASO_OK : DASO_EHIP;
}

}  // extern "C"
