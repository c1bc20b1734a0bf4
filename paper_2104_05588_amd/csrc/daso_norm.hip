// Layer norm, forward and backward (daso_train.h).  Bound by memory: each row is read once
// into registers, its statistics are summed there (the variance from the differences to
// the mean, not from squares), and it is written once.
//
// A row of up to 2048 elements (1024 in the backward pass, whose registers hold five rows' worth) is a
// wavefront's, of up to 8192 a workgroup's of 256 threads; a team of threads keeps the weights in
// registers and walks over rows.  In the backward pass it also keeps its columns' sums for dweight and
// dbias, which end up as one partial row a workgroup; a second kernel adds those in order.  Longer rows are read
// again for each of their passes, from L2, an element a thread at a time: 2048 rows of 20000 in bf16 forward in 87 us,
// backward in 120, where rows of 8192 take 16 and 57.
//
// Measured: 8192 rows of 1024 in bf16 forward in 9 us (3.7 TB/s: a wavefront also loads 8 KB of weight and bias, for
// two rows of 2 KB); 32768 such rows backward in 34 us (6.0 TB/s) and 4 for the sums; 5003 rows of 1601 in fp32 backward in 25
// and 4 us, where the next row alone is on its way behind the one in hand.  More workgroups there are no help: the
// partial rows grow with them (768: 29.6 us in all, 1024: 32.0, 512: 28.8).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "daso_partials.h"
#include "daso_planes.h"
#include "daso_train_host.h"

namespace daso {
namespace {

constexpr int kThreads = 256;
constexpr int kForwardGroups = 1024;  // most workgroups of a forward pass
constexpr int kPartialGroups = 512;  // most workgroups of a backward pass: two a CU

struct Forward {
  int64_t rows, x_stride, y_stride;
  const void* x;
  const float *weight, *bias;
  void* y;
  float *mean, *rstd;
  int32_t d;
  float eps;
};

struct Backward {
  int64_t rows, dy_stride, x_stride, dx_stride;
  const void *dy, *x;
  const float *weight, *mean, *rstd;
  void* dx;
  float* partial;  // [workgroup][dweight, dbias][d]
  int32_t d;
};

// N elements of a row in a team of TEAM threads, eight neighbouring ones at a time, at any
// address.  Without WHOLE (d a multiple of 8) one thread of the team has the row's last, shorter run.
template <int TEAM, int N, bool WHOLE>
struct Slice {
  static constexpr int kRun = 8, kRuns = N / kRun;
  // the column of run i, element 0
  __device__ static int column(int i, int t) { return (i * TEAM + t) * kRun; }
  __device__ static bool full(int c, int d) { return WHOLE ? c < d : c + kRun <= d; }

  template <class T>
  __device__ static void load(const T* row, int d, int t, float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const int c = column(i, t);
      float a[8] = {};
      if (full(c, d)) load8(row + c, a);
      if (!WHOLE && c < d && c + kRun > d)
#pragma unroll
        for (int j = 0; j < kRun - 1; ++j)
          if (c + j < d) a[j] = load1(row + c + j);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i * 8 + j] = a[j];
    }
  }
  // a vector, or `none` where there is no such vector
  __device__ static void load_vector(const float* p, int d, int t, float none, float (&v)[N]) {
    if (p != nullptr) {
      load(p, d, t, v);
      return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = none;
  }
  template <class T>
  __device__ static void store(T* row, int d, int t, const float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < kRuns; ++i) {
      const int c = column(i, t);
      if (full(c, d)) {
        float a[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j] = v[i * 8 + j];
        store8(row + c, a);
      } else if (!WHOLE && c < d) {
#pragma unroll
        for (int j = 0; j < kRun - 1; ++j)
          if (c + j < d) store1(row + c + j, v[i * 8 + j]);
      }
    }
  }
  // elements as they lie in memory: a row that is on its way takes no more registers than that
  template <class T>
  struct Raw {
    static constexpr int kEach = kRun * sizeof(T) / 16;  // 16 bytes each, of a run
    typedef uint32_t word __attribute__((ext_vector_type(4)));
    word words[kRuns * kEach];
    T last[WHOLE ? 1 : kRun - 1];  // of the shorter run
    __device__ void load(const T* row, int d, int t) {
#pragma unroll
      for (int i = 0; i < kRuns; ++i) {
        const int c = column(i, t);
#pragma unroll
        for (int k = 0; k < kEach; ++k) words[i * kEach + k] = full(c, d) ? __builtin_bit_cast(word, load16(row + c + k * (16 / sizeof(T)))) : word{0, 0, 0, 0};
      }
      if constexpr (!WHOLE) {
        const int c = d / kRun * kRun;
        if (d / kRun % TEAM == t)
#pragma unroll
          for (int j = 0; j < kRun - 1; ++j)
            if (c + j < d) last[j] = row[c + j];
      }
    }
    __device__ void get(float (&v)[N], int d, int t) const {
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint32_t w = words[i / 4][i % 4];
          v[i] = __builtin_bit_cast(float, w);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint32_t w = words[i / 8][i / 2 % 4];
          v[i] = __builtin_bit_cast(float, i % 2 ? w & 0xffff0000u : w << 16);
        }
      }
      if constexpr (!WHOLE) {
#pragma unroll
        for (int i = 0; i < kRuns; ++i)
          if (d / (kRun * TEAM) == i && d / kRun % TEAM == t)
#pragma unroll
            for (int j = 0; j < kRun - 1; ++j) v[i * kRun + j] = j < d % kRun ? load1(&last[j]) : 0.0f;
      }
    }
  };
  __device__ static bool inside(int e, int d, int t) { return column(e / kRun, t) + e % kRun < d; }
};

template <int TEAM>
__device__ inline float team_sum(float v, float* shared) {
  if constexpr (TEAM == 64) return wave_sum(v);
  else return group_sum(v, shared);
}

template <class T, int TEAM, int N, bool WHOLE>
__global__ __launch_bounds__(kThreads) void forward_kernel(Forward a) {
  using S = Slice<TEAM, N, WHOLE>;
  __shared__ float shared[kThreads / 64];
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  constexpr int kTeams = kThreads / TEAM;
  const int64_t step = int64_t(gridDim.x) * kTeams;
  int64_t r = blockIdx.x * int64_t(kTeams) + team;
  float w[N], b[N];
  typename S::template Raw<T> next;
  if (r < a.rows) next.load((const T*)a.x + r * a.x_stride, a.d, t);
  S::load_vector(a.weight, a.d, t, 1.0f, w);
  S::load_vector(a.bias, a.d, t, 0.0f, b);
  const float df = static_cast<float>(a.d);
  for (; r < a.rows; r += step) {
    float v[N], sum = 0.0f, square = 0.0f;
    next.get(v, a.d, t);
    if (r + step < a.rows) next.load((const T*)a.x + (r + step) * a.x_stride, a.d, t);
#pragma unroll
    for (int i = 0; i < N; ++i) sum += v[i];
    const float mean = team_sum<TEAM>(sum, shared) / df;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = S::inside(i, a.d, t) ? v[i] - mean : 0.0f;
      square = fmaf(v[i], v[i], square);
    }
    const float rstd = 1.0f / sqrtf(team_sum<TEAM>(square, shared) / df + a.eps);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = fmaf(v[i] * rstd, w[i], b[i]);
    S::store((T*)a.y + r * a.y_stride, a.d, t, v);
    if (t == 0) {
      if (a.mean != nullptr) a.mean[r] = mean;
      if (a.rstd != nullptr) a.rstd[r] = rstd;
    }
  }
}

// A row longer than a workgroup holds.
template <class T>
__global__ __launch_bounds__(kThreads) void forward_long_kernel(Forward a) {
  __shared__ float shared[kThreads / 64];
  const float df = static_cast<float>(a.d);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = (const T*)a.x + r * a.x_stride;
    T* y = (T*)a.y + r * a.y_stride;
    float sum = 0.0f, square = 0.0f;
    for (int c = threadIdx.x; c < a.d; c += kThreads) sum += load1(x + c);
    const float mean = group_sum(sum, shared) / df;
    for (int c = threadIdx.x; c < a.d; c += kThreads) {
      const float v = load1(x + c) - mean;
      square = fmaf(v, v, square);
    }
    const float rstd = 1.0f / sqrtf(group_sum(square, shared) / df + a.eps);
    for (int c = threadIdx.x; c < a.d; c += kThreads)
      store1(y + c, fmaf((load1(x + c) - mean) * rstd, a.weight ? a.weight[c] : 1.0f, a.bias ? a.bias[c] : 0.0f));
    if (threadIdx.x == 0) {
      if (a.mean != nullptr) a.mean[r] = mean;
      if (a.rstd != nullptr) a.rstd[r] = rstd;
    }
  }
}

template <class T, int TEAM, int N, bool WHOLE>
__global__ __launch_bounds__(kThreads) void backward_kernel(Backward a) {
  using S = Slice<TEAM, N, WHOLE>;
  constexpr int kTeams = kThreads / TEAM;
  __shared__ float shared[kThreads / 64];
  __shared__ float meet[kTeams > 1 ? kTeams : 1][TEAM * S::kRun];
  const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  float w[N], dw[N], db[N];
  S::load_vector(a.weight, a.d, t, 1.0f, w);
#pragma unroll
  for (int i = 0; i < N; ++i) dw[i] = db[i] = 0.0f;
  const float inv = 1.0f / static_cast<float>(a.d);
  const int64_t step = int64_t(gridDim.x) * kTeams;
  int64_t r = blockIdx.x * int64_t(kTeams) + team;
  typename S::template Raw<T> next_x, next_g;
  float next_mean = 0.0f, next_rstd = 0.0f;
  const auto fetch = [&](int64_t row) {
    next_x.load((const T*)a.x + row * a.x_stride, a.d, t);
    next_g.load((const T*)a.dy + row * a.dy_stride, a.d, t);
    next_mean = a.mean[row], next_rstd = a.rstd[row];
  };
  if (r < a.rows) fetch(r);
  for (; r < a.rows; r += step) {
    float x[N], g[N], s1 = 0.0f, s2 = 0.0f;
    next_x.get(x, a.d, t), next_g.get(g, a.d, t);
    const float mean = next_mean, rstd = next_rstd;
    if (r + step < a.rows) fetch(r + step);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = S::inside(i, a.d, t) ? (x[i] - mean) * rstd : 0.0f;
      dw[i] = fmaf(g[i], x[i], dw[i]);
      db[i] += g[i];
      g[i] *= w[i];
      s1 += g[i];
      s2 = fmaf(g[i], x[i], s2);
    }
    s1 = team_sum<TEAM>(s1, shared) * inv;
    s2 = team_sum<TEAM>(s2, shared) * inv;
    if (a.dx == nullptr) continue;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = rstd * (g[i] - s1 - x[i] * s2);
    S::store((T*)a.dx + r * a.dx_stride, a.d, t, x);
  }
  if (a.partial == nullptr) return;
  float* out = a.partial + int64_t(blockIdx.x) * 2 * a.d;
#pragma unroll
  for (int half = 0; half < 2; ++half)
#pragma unroll
    for (int i = 0; i < S::kRuns; ++i) {
      if constexpr (kTeams > 1) __syncthreads();
#pragma unroll
      for (int j = 0; j < S::kRun; ++j) {
        const float v = half == 0 ? dw[i * S::kRun + j] : db[i * S::kRun + j];
        if constexpr (kTeams > 1) meet[team][t * S::kRun + j] = v;
        else if (S::column(i, t) + j < a.d) out[half * a.d + S::column(i, t) + j] = v;
      }
      if constexpr (kTeams > 1) {
        __syncthreads();
        for (int k = threadIdx.x; k < TEAM * S::kRun; k += kThreads) {
          float v = meet[0][k];
#pragma unroll
          for (int m = 1; m < kTeams; ++m) v += meet[m][k];
          const int c = i * TEAM * S::kRun + k;
          if (c < a.d) out[half * a.d + c] = v;
        }
      }
    }
}

// dx of long rows.
template <class T>
__global__ __launch_bounds__(kThreads) void backward_long_kernel(Backward a) {
  __shared__ float shared[kThreads / 64];
  const float inv = 1.0f / static_cast<float>(a.d);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *x = (const T*)a.x + r * a.x_stride, *dy = (const T*)a.dy + r * a.dy_stride;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s1 = 0.0f, s2 = 0.0f;
    for (int c = threadIdx.x; c < a.d; c += kThreads) {
      const float g = load1(dy + c) * (a.weight ? a.weight[c] : 1.0f);
      s1 += g;
      s2 = fmaf(g, (load1(x + c) - mean) * rstd, s2);
    }
    s1 = group_sum(s1, shared) * inv;
    s2 = group_sum(s2, shared) * inv;
    for (int c = threadIdx.x; c < a.d; c += kThreads) {
      const float g = load1(dy + c) * (a.weight ? a.weight[c] : 1.0f);
      store1((T*)a.dx + r * a.dx_stride + c, rstd * (g - s1 - (load1(x + c) - mean) * rstd * s2));
    }
  }
}

// The column sums of long rows: 256 columns and a share of the rows a workgroup.
template <class T>
__global__ __launch_bounds__(kThreads) void columns_long_kernel(Backward a, int32_t shares) {
  const int c = blockIdx.x * kThreads + threadIdx.x, share = blockIdx.y;
  if (c >= a.d) return;
  float dw = 0.0f, db = 0.0f;
  for (int64_t r = share; r < a.rows; r += shares) {
    const float g = load1((const T*)a.dy + r * a.dy_stride + c);
    dw = fmaf(g, (load1((const T*)a.x + r * a.x_stride + c) - a.mean[r]) * a.rstd[r], dw);
    db += g;
  }
  a.partial[int64_t(share) * 2 * a.d + c] = dw;
  a.partial[int64_t(share) * 2 * a.d + a.d + c] = db;
}

// ------------------------------------------------------------------------- host
constexpr int64_t kWaveForward = 2048, kWaveBackward = 1024;  // longest rows of a wavefront
bool is_long(int64_t d) { return d > 8192; }

// Workgroups of a pass whose teams walk over rows.
int64_t groups_of(int64_t rows, int64_t d, int64_t wave_d, int64_t most) {
  const int64_t teams = d <= wave_d ? kThreads / 64 : 1;
  return std::min((rows + teams - 1) / teams, most);
}

template <class T, bool WHOLE>
hipError_t forward(const Forward& a, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(groups_of(a.rows, a.d, kWaveForward, kForwardGroups))), block(kThreads);
  if (a.d <= 512) return launch(&forward_kernel<T, 64, 8, WHOLE>, grid, block, stream, a);
  if (a.d <= 1024) return launch(&forward_kernel<T, 64, 16, WHOLE>, grid, block, stream, a);
  if (a.d <= 2048) return launch(&forward_kernel<T, 64, 32, WHOLE>, grid, block, stream, a);
  if (a.d <= 4096) return launch(&forward_kernel<T, 256, 16, WHOLE>, grid, block, stream, a);
  if (a.d <= 8192) return launch(&forward_kernel<T, 256, 32, WHOLE>, grid, block, stream, a);
  return launch(&forward_long_kernel<T>, dim3(static_cast<uint32_t>(std::min<int64_t>(a.rows, 4096))), block, stream, a);
}

template <class T, bool WHOLE>
hipError_t backward(const Backward& a, int32_t groups, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(groups)), block(kThreads);
  if (a.d <= 512) return launch(&backward_kernel<T, 64, 8, WHOLE>, grid, block, stream, a);
  if (a.d <= 1024) return launch(&backward_kernel<T, 64, 16, WHOLE>, grid, block, stream, a);
  if (a.d <= 2048) return launch(&backward_kernel<T, 256, 8, WHOLE>, grid, block, stream, a);
  if (a.d <= 4096) return launch(&backward_kernel<T, 256, 16, WHOLE>, grid, block, stream, a);
  if (a.d <= 8192) return launch(&backward_kernel<T, 256, 32, WHOLE>, grid, block, stream, a);
  // the columns' sums first: dx may take dy's place
  hipError_t e = hipSuccess;
  if (a.partial != nullptr)
    e = launch(&columns_long_kernel<T>, dim3(static_cast<uint32_t>((a.d + kThreads - 1) / kThreads), static_cast<uint32_t>(groups)),
               block, stream, a, groups);
  if (e == hipSuccess && a.dx != nullptr)
    e = launch(&backward_long_kernel<T>, dim3(static_cast<uint32_t>(std::min<int64_t>(a.rows, 4096))), block, stream, a);
  return e;
}

// Partial rows of a backward pass.
int32_t partial_rows(int64_t rows, int64_t d) {
  return static_cast<int32_t>(is_long(d) ? std::min<int64_t>(rows, 64) : groups_of(rows, d, kWaveBackward, kPartialGroups));
}

size_t backward_bytes(const daso_layer_norm_backward_args& s) {
  if (s.rows == 0 || s.d == 0) return 0;
  return static_cast<size_t>(partial_rows(s.rows, s.d)) * 2 * static_cast<size_t>(s.d) * sizeof(float);
}

}  // namespace
}  // namespace daso

extern "C" {

int daso_layer_norm(const daso_layer_norm_args* args, hipStream_t stream) {
  if (args == nullptr) return DASO_EINVAL;
  const daso_layer_norm_args& s = *args;
  int rc = daso::host::check_layer_norm(s);
  if (rc != DASO_OK || s.rows == 0 || s.d == 0) return rc;
  if ((rc = daso::current_device(stream)) != DASO_OK) return rc;
  const daso::Forward a = {s.rows, s.x_stride, s.y_stride, s.x, s.weight, s.bias, s.y, s.mean, s.rstd, static_cast<int32_t>(s.d), s.eps};
  const bool whole = s.d % 8 == 0;
  hipError_t err;
  if (s.type == DASO_TYPE_BF16) err = whole ? daso::forward<uint16_t, true>(a, stream) : daso::forward<uint16_t, false>(a, stream);
  else err = whole ? daso::forward<float, true>(a, stream) : daso::forward<float, false>(a, stream);
  return err == hipSuccess ? DASO_OK : DASO_EHIP;
}

int daso_layer_norm_backward_workspace(const daso_layer_norm_backward_args* args, size_t* bytes) {
  if (args == nullptr || bytes == nullptr) return DASO_EINVAL;
  const int rc = daso::host::check_layer_norm_backward_sizes(*args);
  if (rc != DASO_OK) return rc;
  *bytes = daso::backward_bytes(*args);
  return DASO_OK;
}

int daso_layer_norm_backward(const daso_layer_norm_backward_args* args, hipStream_t stream) {
  if (args == nullptr) return DASO_EINVAL;
  const daso_layer_norm_backward_args& s = *args;
  int rc = daso::host::check_layer_norm_backward(s);
  if (rc != DASO_OK || s.d == 0) return rc;
  const bool sums = s.dweight != nullptr || s.dbias != nullptr;
  if (!sums && (s.rows == 0 || s.dx == nullptr)) return DASO_OK;
  if (sums && (rc = daso::host::check_workspace(s.workspace, s.workspace_bytes, daso::backward_bytes(s))) != DASO_OK) return rc;
  if ((rc = daso::current_device(stream)) != DASO_OK) return rc;
  const int32_t d = static_cast<int32_t>(s.d), groups = s.rows > 0 ? daso::partial_rows(s.rows, s.d) : 0;
  float* partial = sums ? static_cast<float*>(s.workspace) : nullptr;
  hipError_t err = hipSuccess;
  if (s.rows > 0) {
    const daso::Backward a = {s.rows, s.dy_stride, s.x_stride, s.dx_stride, s.dy, s.x, s.weight, s.mean, s.rstd, s.dx, partial, d};
    const bool whole = s.d % 8 == 0;
    if (s.type == DASO_TYPE_BF16)
      err = whole ? daso::backward<uint16_t, true>(a, groups, stream) : daso::backward<uint16_t, false>(a, groups, stream);
    else
      err = whole ? daso::backward<float, true>(a, groups, stream) : daso::backward<float, false>(a, groups, stream);
  }
  if (err == hipSuccess && sums)
    err = daso::launch(&daso::partials_kernel, dim3(static_cast<uint32_t>((2 * s.d + 15) / 16)), dim3(1024), stream, (const float*)partial,
                       groups, d, s.dweight, s.dbias);
  return err == hipSuccess ? DASO_OK : DASO_EHIP;
}

}  // extern "C"
