// The norm of an averaged gradient over many tensors, and its clipping (daso_block.h).  Bound by memory:
// one pass reads the g replicas, sums the squares of their mean in 64 bits (where no square of a
// binary32 value overflows or vanishes) and writes the mean, a second one scales it.  Nothing waits for another
// workgroup: the partial sums, one a piece, are added in a fixed order by the scaling workgroups each for itself,
// or, where they are many, by two small kernels between the passes.
//
// A workgroup takes one piece of 4 KB a replica and ends, so that the chip sweeps the buffers front to back: the first pass over
// 25.6M elements of 4 replicas in 83 us (6.1 TB/s), 92 with two pieces a workgroup, 97 with eight, also with
// loads ahead of the piece in hand or fewer workgroups a CU.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "daso_block_host.h"
#include "daso_planes.h"

namespace daso {
namespace {

using host::ClipTable;
using host::kPiece;

constexpr int kThreads = 256, kJoinThreads = 1024;
static_assert(kPiece == kThreads * 4, "four elements a thread");

struct Norm {
  ClipTable table;
  double* partial;  // of the launch's first piece
  float* mean;      // or null
  int32_t g;
};
struct Grads {
  const float* of[DASO_MAX_G];
};

struct Scale {
  ClipTable table;
  const double* partial;     // of all launches
  int64_t pieces, first;     // of all launches; the launch's first
  const float* factor;       // or null: the sums are added here
  const float* mean;
  float *out, *norm, *norms;
  float max_norm, eps;
  int32_t ready;             // out holds the mean
};

struct Join {
  ClipTable table;
  const double* partial;  // of the launch's first piece
  double* sums;           // one a tensor
  float* norms;           // or null
};

// Where a thread's four elements of the launch's piece `at` begin, in a tensor of elements from..to: what is left of the piece's
// run, the last one whose first piece is not beyond it (gaps have none).
struct Four {
  int64_t j, from, to;
  bool whole;
};
__device__ inline Four four_of(const ClipTable& t, int at) {
  // (all runs at once: one read after another, in halves, took 12 us of 95 for a network's 161 tensors)
  int run = -1;
  if (t.runs == 1) {
    run = 0;
  } else {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < host::kClipRuns; k += 64) run += __popcll(__ballot(k + lane < t.runs && t.first[min(k + lane, host::kClipRuns)] <= at));
  }
  Four f;
  f.from = t.bound[run], f.to = t.bound[run + 1];
  f.j = (f.from / kPiece + at - t.first[run]) * kPiece + threadIdx.x * 4;
  f.whole = f.j >= f.from && f.j + 4 <= f.to;
  return f;
}

__device__ inline double square(float v) {
  const double d = v;
  return d * d;
}

// The mean of the replicas from their sum, as the fused step has it.
template <class V>
__device__ inline V mean_of(V sum, int32_t g) {
  if (g == 1) return sum;
  if ((g & (g - 1)) == 0) return sum * (1.0f / static_cast<float>(g));  // exact, as the division is
  return sum / static_cast<float>(g);
}

// G: replicas, or 0 for any number.
template <int G>
__global__ __launch_bounds__(kThreads) void norm_kernel(Norm a, Grads g) {
  __shared__ double shared[kThreads / 64];
  const Four f = four_of(a.table, blockIdx.x);
  const int32_t count = G > 0 ? G : a.g;
  double sum = 0.0;
  if (f.whole) {
    f4v v[G > 0 ? G : 1];
#pragma unroll
    for (int r = 0; r < (G > 0 ? G : 1); ++r) v[r] = load4(g.of[r] + f.j);
    f4v s = v[0];
#pragma unroll
    for (int r = 1; r < G; ++r) s += v[r];
    if constexpr (G == 0)
      for (int r = 1; r < count; ++r) s += load4(g.of[r] + f.j);
    s = mean_of(s, count);
    if (a.mean != nullptr) *(f4v*)(a.mean + f.j) = s;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum += square(s[e]);
  } else {  // at an end of the tensor
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (f.j + e < f.from || f.j + e >= f.to) continue;
      float s = g.of[0][f.j + e];
      for (int r = 1; r < count; ++r) s += g.of[r][f.j + e];
      s = mean_of(s, count);
      if (a.mean != nullptr) a.mean[f.j + e] = s;
      sum += square(s);
    }
  }
  sum = group_sum(sum, shared);
  if (threadIdx.x == 0) a.partial[blockIdx.x] = sum;
}

// The sum of partials, the same in every thread of every workgroup that asks, in an order that follows from their number and the
// workgroup's.
template <int THREADS>
__device__ inline double sum_of(const double* p, int64_t count, double* shared) {
  constexpr int kAhead = 8;
  double sum = 0.0;
  for (int64_t i = threadIdx.x; i < count; i += THREADS * kAhead) {
    double v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v[k] = p[min(i + k * THREADS, count - 1)];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) sum += i + k * THREADS < count ? v[k] : 0.0;
  }
  return group_sum(sum, shared);
}
__device__ inline float factor_of(double norm, float max_norm, float eps) {
  const double f = static_cast<double>(max_norm) / (norm + static_cast<double>(eps));
  return f >= 1.0 ? 1.0f : static_cast<float>(f);
}

// Each tensor's sum.
__global__ __launch_bounds__(kJoinThreads) void join_kernel(Join a) {
  __shared__ double shared[kJoinThreads / 64];
  const int run = blockIdx.x, number = a.table.number[run];
  if (number < 0) return;
  const int from = a.table.first[run];
  const double sum = sum_of<kJoinThreads>(a.partial + from, a.table.first[run + 1] - from, shared);
  if (threadIdx.x != 0) return;
  a.sums[a.table.tensor + number] = sum;
  if (a.norms != nullptr) a.norms[a.table.tensor + number] = static_cast<float>(sqrt(sum));
}
// All tensors' norm, and what it makes the factor.
__global__ __launch_bounds__(kThreads) void total_kernel(const double* sums, int32_t count, float max_norm, float eps, float* norm, float* factor) {
  __shared__ double shared[kThreads / 64];
  const double n = sqrt(sum_of<kThreads>(sums, count, shared));
  if (threadIdx.x != 0) return;
  *norm = static_cast<float>(n);
  *factor = factor_of(n, max_norm, eps);
}

__global__ __launch_bounds__(kThreads) void scale_kernel(Scale a) {
  __shared__ double shared[kThreads / 64];
  float factor;
  if (a.factor != nullptr) {
    factor = *a.factor;
  } else {
    const double norm = sqrt(sum_of<kThreads>(a.partial, a.pieces, shared));
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.norm != nullptr) *a.norm = static_cast<float>(norm);
    const int run = blockIdx.x;
    if (a.norms != nullptr && run < a.table.runs && a.table.number[run] >= 0) {
      __syncthreads();
      const int from = a.table.first[run];
      const double of = sqrt(sum_of<kThreads>(a.partial + a.first + from, a.table.first[run + 1] - from, shared));
      if (threadIdx.x == 0) a.norms[a.table.tensor + a.table.number[run]] = static_cast<float>(of);
    }
    factor = factor_of(norm, a.max_norm, a.eps);
  }
  if (a.out == nullptr || static_cast<int>(blockIdx.x) >= a.table.first[a.table.runs] || (a.ready && factor == 1.0f)) return;
  const Four f = four_of(a.table, blockIdx.x);
  if (f.whole) {
    *(f4v*)(a.out + f.j) = load4(a.mean + f.j) * factor;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (f.j + e >= f.from && f.j + e < f.to) a.out[f.j + e] = a.mean[f.j + e] * factor;
}

// Of the workspace: the partial sums and, where kernels of their own add them, the tensors' and the factor.
int32_t tensors_of(const daso_clip_args& s) { return s.ntensors > 0 ? s.ntensors : 1; }
size_t workspace_of(const daso_clip_args& s, int64_t pieces) {
  return (size_t(pieces) + (pieces > host::kJoined ? size_t(tensors_of(s)) + 1 : 0)) * sizeof(double);
}

template <class F>
hipError_t over_tables(const daso_clip_args& s, bool merged, ClipTable* table, F queue) {
  int64_t first = 0;
  hipError_t err = hipSuccess;
  for (int32_t t = 0; t < tensors_of(s) && err == hipSuccess;) {
    t += host::fill_table(s, t, merged, table);
    err = queue(first, table->first[table->runs]);
    first += table->first[table->runs];
  }
  return err;
}

hipError_t run(const daso_clip_args& s, int64_t pieces, hipStream_t stream) {
  const bool joined = pieces > host::kJoined;
  double* const partial = static_cast<double*>(s.workspace);
  double* const sums = joined ? partial + pieces : nullptr;
  float* const factor = joined ? reinterpret_cast<float*>(sums + tensors_of(s)) : nullptr;
  const dim3 block(kThreads);
  const auto grid = [](int64_t n) { return dim3(static_cast<uint32_t>(n)); };
  Grads g = {};
  for (int32_t r = 0; r < s.g && s.n > 0; ++r) g.of[r] = s.grads[r];
  Norm a;
  a.g = s.g, a.mean = s.g > 1 ? s.out : nullptr;
  hipError_t err = over_tables(s, false, &a.table, [&](int64_t first, int32_t count) {
    a.partial = partial + first;
    if (count == 0) return hipSuccess;
    switch (s.g) {
      case 1: return launch(&norm_kernel<1>, grid(count), block, stream, a, g);
      case 2: return launch(&norm_kernel<2>, grid(count), block, stream, a, g);
      case 3: return launch(&norm_kernel<3>, grid(count), block, stream, a, g);
      case 4: return launch(&norm_kernel<4>, grid(count), block, stream, a, g);
      case 8: return launch(&norm_kernel<8>, grid(count), block, stream, a, g);
      default: return launch(&norm_kernel<0>, grid(count), block, stream, a, g);
    }
  });
  if (err == hipSuccess && joined) {
    Join j;
    j.sums = sums, j.norms = s.norms;
    err = over_tables(s, false, &j.table, [&](int64_t first, int32_t) {
      j.partial = partial + first;
      return launch(&join_kernel, grid(j.table.runs), dim3(kJoinThreads), stream, j);
    });
    if (err == hipSuccess)
      err = launch(&total_kernel, grid(1), block, stream, (const double*)sums, tensors_of(s), s.max_norm, s.eps, s.norm, factor);
    if (s.out == nullptr) return err;
  }
  if (err != hipSuccess) return err;
  Scale b;
  b.partial = partial, b.pieces = pieces, b.factor = factor, b.mean = s.g > 1 ? s.out : g.of[0];
  b.out = s.out, b.norm = s.norm, b.norms = s.norms, b.max_norm = s.max_norm, b.eps = s.eps;
  b.ready = s.g > 1 || s.out == g.of[0];
  return over_tables(s, joined, &b.table, [&](int64_t first, int32_t count) {
    // a workgroup a piece to scale, and a tensor whose norm is to be written
    const int64_t groups = std::max(s.out != nullptr ? count : 0, factor == nullptr && s.norms != nullptr ? b.table.runs : 0);
    b.first = first;
    if (groups == 0 && (first > 0 || factor != nullptr)) return hipSuccess;
    const hipError_t e = launch(&scale_kernel, grid(std::max<int64_t>(groups, 1)), block, stream, b);
    b.norm = nullptr;
    return e;
  });
}

}  // namespace
}  // namespace daso

extern "C" {

int daso_clip_gradients_workspace(const daso_clip_args* args, size_t* bytes) {
  if (args == nullptr || bytes == nullptr) return DASO_EINVAL;
  const int rc = daso::host::check_clip_sizes(*args);
  if (rc != DASO_OK) return rc;
  *bytes = daso::workspace_of(*args, daso::host::pieces_of(*args));
  return DASO_OK;
}

int daso_clip_gradients(const daso_clip_args* args, hipStream_t stream) {
  if (args == nullptr) return DASO_EINVAL;
  const daso_clip_args& s = *args;
  int rc = daso::host::check_clip(s);
  if (rc != DASO_OK) return rc;
  const int64_t pieces = daso::host::pieces_of(s);
  if ((rc = daso::host::check_workspace(s.workspace, s.workspace_bytes, daso::workspace_of(s, pieces))) != DASO_OK) return rc;
  if ((rc = daso::current_device(stream)) != DASO_OK) return rc;
  return daso::run(s, pieces, stream) == hipSuccess ? DASO_OK : DASO_EHIP;
}

}  // extern "C"
