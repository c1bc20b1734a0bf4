// Newton-Schulz orthogonalisation and the optimizer step that uses it (daso_train.h).
//
// A step on X (m x n, m <= n) is three products: the gram matrix A = X X^T and its square,
// both symmetric, of which only the tiles on and below the diagonal are computed and
// stored twice, and X' = a X + B X with B = b A + c A^2: m^2 n + m^3 + 2 m^2 n operations in
// place of 4 m^2 n + 2 m^3.  Bound by the matrix cores, and so by the power they draw, where m is
// large; the epilogue's planes are the other part: for 96 matrices of 1024 x 1024 in 22 bits the last of the
// three products takes 834 us, of which 622 are the product (1240 TFLOP/s) and the rest its 800 MB read
// and written again.  Starting the workgroups apart, so that some compute while others write, gave nothing.
//
// Numbers.  With |X|_F <= 1 at the start and the polynomial's range, entries of X, A and B stay
// below 4 for the coefficients in use; they are stored times 2^11 as binary16.  A step
// raises weak directions by up to a (3.4 and more, some 480 times in five steps), so X,
// which the sum a X + B X carries forward, keeps 22 bits (hi + lo) always.  In the
// products an error of B or of X's operand form only reaches the result through a strong
// direction, which the steps do not raise: there 11 bits are enough for a bf16 result (against 64 bits it is off by 0.0017
// of its norm for 4096 x 4096, 0.0019 for 64 x 576, 0.0023 for 24 x 24, where rounding to bf16 alone makes 0.0017),
// while fp32 results take hi hi + hi lo + lo hi.  One error of 11 bits does not average out:
// where the rows of X are near orthogonal, A and B are near diagonal, and a X + B X takes the
// difference of two near numbers.  So what the rounding of the diagonals left over is kept
// in 32 bits (`rest`) and put into the products' epilogues, at the cost of one multiply-add.
#include <hip/hip_runtime.h>

#include <atomic>
#include <cmath>
#include <new>

#include "daso_planes.h"
#include "daso_product.h"
#include "daso_train_host.h"

namespace daso {
namespace {

using host::SchulzGroup;
using host::SchulzRound;
using product::f4;
using product::half8;

constexpr float kScale = 2048.0f, kUnscale = 1.0f / 2048.0f;

// What the final product needs of a matrix of a flat buffer.
struct Entry {
  int64_t start;
  float step;  // lr * scale
  float pad;
};
static_assert(sizeof(Entry) == 16, "the table of a round counts 16 bytes an entry");

// ------------------------------------------------------------------------- epilogues
// v = alpha * C + beta * (in_hi + in_lo) as planes, and transposed where `t_always` or the
// tile lies off the diagonal of a symmetric result.  With in one plane, `rest` is what its
// diagonal lacks (square) or what that of the left operand does.
struct PlanesOut {
  struct Params {
    const _Float16 *in_hi, *in_lo;
    _Float16 *hi, *lo, *t_hi, *t_lo;
    int64_t ld, batch, t_ld, t_batch;  // of in, hi and lo; of t_hi and t_lo
    float alpha, beta;
    int32_t t_always;
    const float* rest;   // rest_ld a matrix; null: nothing is lacking
    float* rest_out;     // of the result's diagonal
    int32_t rest_ld;
    int32_t square;      // C = in in^T; else C = left in
  };
  static constexpr auto kKind = product::kStaged;
  struct Inputs {
    half8 hi[product::kPasses], lo[product::kPasses];
    float left[product::kPasses], right[8];  // what the operands' diagonals lack, by rows and by columns
  };
  __device__ static void fetch(const Params& p, const product::Place& at, int row, int col, int lane, Inputs& in) {
    const int64_t from = at.batch * p.batch + int64_t(row + product::pass_row(0, lane)) * p.ld + col + product::pass_col(lane);
    const half8 none = (half8)(_Float16)0.0f;
    if (p.in_hi != nullptr) {
#pragma unroll
      for (int pass = 0; pass < product::kPasses; ++pass) in.hi[pass] = *(const half8*)(p.in_hi + from + pass * product::kPassRows * p.ld);
    } else {
#pragma unroll
      for (int pass = 0; pass < product::kPasses; ++pass) in.hi[pass] = none;
    }
    if (p.in_lo != nullptr) {
#pragma unroll
      for (int pass = 0; pass < product::kPasses; ++pass) in.lo[pass] = *(const half8*)(p.in_lo + from + pass * product::kPassRows * p.ld);
    } else {
#pragma unroll
      for (int pass = 0; pass < product::kPasses; ++pass) in.lo[pass] = none;
    }
    const float* rest = p.rest + int64_t(at.batch) * p.rest_ld;
#pragma unroll
    for (int pass = 0; pass < product::kPasses; ++pass)
      in.left[pass] = p.rest != nullptr ? rest[row + product::pass_row(pass, lane)] : 0.0f;
    const bool square = p.rest != nullptr && p.square;
#pragma unroll
    for (int i = 0; i < 8; ++i) in.right[i] = square ? rest[col + product::pass_col(lane) + i] : 0.0f;
  }
  template <class F>
  __device__ static void block(const Params& p, const product::Place& at, int row, int col, char* stage, int lane, const Inputs& in,
                               F next) {
    const bool turn = p.t_hi != nullptr && (p.t_always || at.tm != at.tn), t_lo = p.t_lo != nullptr;
    const int k = product::pass_col(lane);
    float v[product::kPasses][8];  // (all of them, before the planes take their place in LDS)
#pragma unroll
    for (int pass = 0; pass < product::kPasses; ++pass) product::pass_values(stage, pass, lane, v[pass]);
    product::wait_lds();
    __builtin_amdgcn_wave_barrier();
    half8 hi[product::kPasses], lo[product::kPasses];
    float missing[product::kPasses];
#pragma unroll
    for (int pass = 0; pass < product::kPasses; ++pass) {
      const int at_diagonal = row + product::pass_row(pass, lane) - col - k;  // which of the eight lies on it
      missing[pass] = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float x = static_cast<float>(in.hi[pass][i]) + static_cast<float>(in.lo[pass][i]);
        if (p.square) x += i == at_diagonal ? in.left[pass] : 0.0f;
        x = fmaf(p.beta, x, p.alpha * fmaf(in.left[pass] + in.right[i], x, v[pass][i]));
        _Float16 a, b;
        product::split(x, &a, &b);
        hi[pass][i] = a, lo[pass][i] = b;
        missing[pass] = i == at_diagonal ? x - static_cast<float>(a) : missing[pass];
      }
    }
    next();
    const int64_t to = at.batch * p.batch + int64_t(row + product::pass_row(0, lane)) * p.ld + col + k;
#pragma unroll
    for (int pass = 0; pass < product::kPasses; ++pass) {
      const int r = product::pass_row(pass, lane), at_diagonal = row + r - col - k;
      if (p.rest_out != nullptr && at_diagonal >= 0 && at_diagonal < 8)
        p.rest_out[int64_t(at.batch) * p.rest_ld + row + r] = missing[pass];
      *(half8*)(p.hi + to + pass * product::kPassRows * p.ld) = hi[pass];
      if (p.lo != nullptr) *(half8*)(p.lo + to + pass * product::kPassRows * p.ld) = lo[pass];
      if (turn) {
        *(half8*)(stage + product::plane_at(r, k)) = hi[pass];
        if (t_lo) *(half8*)(stage + product::kStagePlane + product::plane_at(r, k)) = lo[pass];
      }
    }
    if (!turn) return;
    product::wait_lds();
    __builtin_amdgcn_wave_barrier();
    const int64_t t_base = at.batch * p.t_batch + int64_t(col) * p.t_ld + row;
    product::by_columns(stage, lane, [&](int c, int r, half8 x) { *(half8*)(p.t_hi + t_base + c * p.t_ld + r) = x; });
    if (t_lo)
      product::by_columns(stage + product::kStagePlane, lane,
                          [&](int c, int r, half8 x) { *(half8*)(p.t_lo + t_base + c * p.t_ld + r) = x; });
  }
};

// The last step's X' = a X + C in the source's orientation: written as it is, or taken as
// the update of a matrix of the flat parameter buffer.
struct LastOut {
  enum Kind { kF32, kBf16, kStep };
  struct Params {
    const _Float16 *in_hi, *in_lo;
    int64_t ld, batch;
    float alpha, beta;
    int32_t kind;
    int32_t rows, cols;
    void* out;  // kF32, kBf16
    int64_t out_ld, out_batch;
    const Entry* table;  // kStep: of the group's matrices
    float* params;
    uint16_t* wire;
    float keep;  // 1 - lr * weight_decay
    const float* rest;  // as above, of the square operand, which is the right one where `right`
    int32_t rest_ld, right;
  };
  static constexpr auto kKind = product::kStaged;
  struct Inputs {
    half8 hi[product::kPasses], lo[product::kPasses];
    float x[product::kPasses][8];  // kStep: the parameters
    float left[product::kPasses], right[8];
    Entry entry;
  };
  // Where a matrix's result lies.
  __device__ static void place(const Params& p, int batch, const Entry& e, int64_t* out, int64_t* ld) {
    *out = p.kind == kStep ? e.start : p.out_batch * batch;
    *ld = p.kind == kStep ? p.cols : p.out_ld;
  }
  __device__ static void fetch(const Params& p, const product::Place& at, int row, int col, int lane, Inputs& in) {
    const int k = product::pass_col(lane), r0 = row + product::pass_row(0, lane), cc = col + k;
    const int64_t from = at.batch * p.batch + int64_t(r0) * p.ld + cc;
#pragma unroll
    for (int pass = 0; pass < product::kPasses; ++pass) {
      in.hi[pass] = *(const half8*)(p.in_hi + from + pass * product::kPassRows * p.ld);
      in.lo[pass] = *(const half8*)(p.in_lo + from + pass * product::kPassRows * p.ld);
    }
    const float* rest = p.rest + int64_t(at.batch) * p.rest_ld;
#pragma unroll
    for (int pass = 0; pass < product::kPasses; ++pass) in.left[pass] = p.rest != nullptr && !p.right ? rest[r0 + pass * product::kPassRows] : 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) in.right[i] = p.rest != nullptr && p.right ? rest[cc + i] : 0.0f;
    if (p.kind != kStep) return;
    in.entry = p.table[at.batch];
    int64_t out, ld;
    place(p, at.batch, in.entry, &out, &ld);
    const bool wide = cc + 8 <= p.cols;
#pragma unroll
    for (int pass = 0; pass < product::kPasses; ++pass) {
      if (r0 + pass * product::kPassRows >= p.rows) continue;
      const float* q = p.params + out + (r0 + pass * product::kPassRows) * ld + cc;
      if (wide) load8(q, in.x[pass]);
      else
#pragma unroll
        for (int i = 0; i < 8; ++i) in.x[pass][i] = cc + i < p.cols ? q[i] : 0.0f;
    }
  }
  template <class F>
  __device__ static void block(const Params& p, const product::Place& at, int row, int col, char* stage, int lane, const Inputs& in,
                               F next) {
    const int r0 = row + product::pass_row(0, lane), cc = col + product::pass_col(lane);
    int64_t out, ld;
    place(p, at.batch, in.entry, &out, &ld);
    const bool wide = cc + 8 <= p.cols;
    const float step = p.kind == kStep ? in.entry.step : 0.0f;
    float* const o32 = p.kind == kStep ? p.params : (float*)p.out;
    uint16_t* const o16 = p.kind == kStep ? p.wire : (uint16_t*)p.out;
    const bool has32 = p.kind != kBf16, has16 = p.kind == kBf16 || (p.kind == kStep && p.wire != nullptr);
    float v[product::kPasses][8];
#pragma unroll
    for (int pass = 0; pass < product::kPasses; ++pass) {
      product::pass_values(stage, pass, lane, v[pass]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = static_cast<float>(in.hi[pass][i]) + static_cast<float>(in.lo[pass][i]);
        float& o = v[pass][i];
        o = fmaf(p.beta, x, p.alpha * fmaf(in.left[pass] + in.right[i], x, o)) * kUnscale;
        if (p.kind == kStep) o = in.x[pass][i] * p.keep - step * o;
      }
    }
    next();
#pragma unroll
    for (int pass = 0; pass < product::kPasses; ++pass) {
      if (r0 + pass * product::kPassRows >= p.rows) continue;
      const int64_t to = out + (r0 + pass * product::kPassRows) * ld + cc;
      if (wide) {
        if (has32) store8(o32 + to, v[pass]);
        if (has16) store8(o16 + to, v[pass]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (cc + i >= p.cols) continue;
          if (has32) o32[to + i] = v[pass][i];
          if (has16) o16[to + i] = to_bf16(v[pass][i]);
        }
      }
    }
  }
};

// ------------------------------------------------------------------------- before the products
// The matrices of a round as kernel arguments.
struct RoundTable {
  int64_t start[host::kRoundMatrices];
  float step[host::kRoundMatrices];
  int32_t count;
  int32_t groups;
  int32_t first[host::kRoundGroups + 1];  // the first matrix of each group
  int64_t elems[host::kRoundGroups];
  float* source[host::kRoundGroups];
};

__device__ inline int group_of(const int32_t* first, int32_t groups, int matrix) {
  int k = 0;
  while (k + 1 < groups && matrix >= first[k + 1]) ++k;
  return k;
}

struct MomentumArgs {
  const float* grads[DASO_MAX_G];
  float* momentum;
  Entry* table;
  double* sums;  // kSumParts a matrix
  int32_t g, nesterov;
  float mu;
};

// gbar, m' and u of a part of a matrix, and the part's sum of u^2, in binary64.  Bound by memory:
// 302M elements with 4 replicas in 1.72 ms, 4.9 TB/s over its seven streams.
__global__ __launch_bounds__(256) void momentum_kernel(MomentumArgs a, RoundTable t) {
  __shared__ double shared[4];
  const int matrix = blockIdx.y, k = group_of(t.first, t.groups, matrix);
  const int64_t elems = t.elems[k], start = t.start[matrix];
  float* u = t.source[k] + (matrix - t.first[k]) * elems;
  const int64_t each = ((elems + gridDim.x - 1) / gridDim.x + 3) / 4 * 4;
  const int64_t lo = each * blockIdx.x, hi = lo + each < elems ? lo + each : elems;
  const float gf = static_cast<float>(a.g);
  double sum = 0;
  auto one = [&](float s, float m, float* m_out) {
    const float gbar = a.g > 1 ? s / gf : s;
    const float mm = a.mu * m + gbar;
    *m_out = mm;
    const float v = a.nesterov ? gbar + a.mu * mm : mm;
    sum += static_cast<double>(v) * v;
    return v;
  };
  if (((start | elems) & 3) == 0) {
    for (int64_t i = lo + 4 * threadIdx.x; i < hi; i += 1024) {
      // four replicas' loads at a time are on their way together, with the momentum's
      f4v m = *(const f4v*)(a.momentum + start + i), v, s = (f4v)0.0f;
      for (int r = 0; r < a.g; r += 4) {
        f4v x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (r + j < a.g) x[j] = *(const f4v*)(a.grads[r + j] + start + i);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (r + j < a.g) s = r + j == 0 ? x[j] : s + x[j];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float mm;
        v[j] = one(s[j], m[j], &mm);
        m[j] = mm;
      }
      *(f4v*)(a.momentum + start + i) = m;
      *(f4v*)(u + i) = v;
    }
  } else {
    for (int64_t i = lo + threadIdx.x; i < hi; i += 256) {
      float s = a.grads[0][start + i];
      for (int r = 1; r < a.g; ++r) s += a.grads[r][start + i];
      float mm;
      u[i] = one(s, a.momentum[start + i], &mm);
      a.momentum[start + i] = mm;
    }
  }
  sum = group_sum(sum, shared);
  if (threadIdx.x == 0) {
    a.sums[matrix * host::kSumParts + blockIdx.x] = sum;
    if (blockIdx.x == 0) a.table[matrix] = {start, t.step[matrix], 0.0f};
  }
}

// The sum of squares of a part of a matrix that is only read (4096 x 4096 in bf16: 20 us).
template <class T>
__global__ __launch_bounds__(256) void squares_kernel(const T* src, int64_t batch_stride, int64_t stride, int32_t rows,
                                                      int32_t cols, double* sums) {
  __shared__ double shared[4];
  const T* p = src + blockIdx.y * batch_stride;
  const int32_t each = (rows + gridDim.x - 1) / gridDim.x;
  const int32_t lo = each * blockIdx.x, hi = lo + each < rows ? lo + each : rows;
  double sum = 0;
  const int32_t whole = cols / 8 * 8;
  for (int32_t r = lo + (threadIdx.x >> 6); r < hi; r += 4) {
    const T* q = p + r * stride;
    for (int32_t c = (threadIdx.x & 63) * 8; c < whole; c += 512) {
      float v[8];
      load8(q + c, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += static_cast<double>(v[i]) * v[i];
    }
    for (int32_t c = whole + (threadIdx.x & 63); c < cols; c += 64) {
      const double v = load1(q + c);
      sum += v * v;
    }
  }
  sum = group_sum(sum, shared);
  if (threadIdx.x == 0) sums[blockIdx.y * host::kSumParts + blockIdx.x] = sum;
}

// What brings a matrix to kScale / (|u| + eps) of itself: the factor `then`, and before it `first`, which is 1 but where the
// norm is so small, or so large, that the factor would be no normal fp32 number.
struct Normal {
  float first, then;
  __device__ Normal(double squares, float eps) {
    const double scale = kScale / (sqrt(squares) + eps);
    first = scale > 0x1p100 && scale < 0x1p1000 ? 0x1p100f : scale < 0x1p-100 ? 0x1p-100f : 1.0f;
    then = static_cast<float>(scale / first);
  }
};

struct LayOut {
  int32_t groups;
  int32_t parts;  // sums of a matrix
  int64_t first_tile[host::kRoundGroups + 1];
  int32_t first_matrix[host::kRoundGroups];
  PlanesArgs p[host::kRoundGroups];
  const double* sums;
  float eps;
};

// X = u / (|u| + eps) as planes.  Bound by memory: 100M fp32 elements in 205 us, 3.9 TB/s.
template <class T>
__global__ __launch_bounds__(256) void normalise_kernel(LayOut a) {
  __shared__ uint16_t lds[2][64][66];
  const int64_t id = blockIdx.x + int64_t(blockIdx.y) * gridDim.x;
  if (id >= a.first_tile[a.groups]) return;
  int k = 0;
  while (k + 1 < a.groups && id >= a.first_tile[k + 1]) ++k;
  const PlanesArgs& p = a.p[k];
  const int64_t t = id - a.first_tile[k], across = p.cols_p / 64, per = across * (p.rows_p / 64);
  const int64_t batch = t / per;
  __shared__ double shared[4];
  const double* s = a.sums + (a.first_matrix[k] + batch) * host::kSumParts;
  const double sum = group_sum(static_cast<int>(threadIdx.x) < a.parts ? s[threadIdx.x] : 0.0, shared);
  const Normal scaled(sum, a.eps);
  planes_tile<T, false>(p, batch, static_cast<int>((t % per) / across), static_cast<int>(t % across),
                        [scaled](float v) { return v * scaled.first * scaled.then; }, lds);
}

// ------------------------------------------------------------------------- small matrices
// All steps of a matrix whose shorter side is at most 64, in one workgroup of 8 wavefronts, from its
// norm to its result: sixteen launches of a few microseconds each become one, 34 us in place of 169 for
// 64 x 576 in bf16.  Bound by the latency of its chain of products, five times three, and by one CU's
// matrix cores; batches take a CU each.
//
// X (m x n, m padded to 64) stays in registers in 32 bits, in the layout in which the matrix
// instructions leave X' = a X + B X: a wavefront has every eighth group of 16 columns.  Its planes,
// for the products, are in LDS: one layout serves both X X^T, whose operands run along n, and B X,
// whose operand runs along m and is read with the transposing LDS loads.  Rows are padded by 16 bytes,
// which makes their distance an odd number of 16-byte pieces: 16 lanes that read one piece of 16
// rows meet no bank twice.  The gram matrix and B take turns in one place of LDS, 2 of their 16
// tiles a wavefront, and stay in 32 bits in the registers of the wavefront that computed them.
// With one plane (bf16 results), what the planes' diagonals lack is kept as above.
using host::kGramStride;
using host::kSmallGroups;
using host::kSmallM;
using host::small_stride;
constexpr int kSmallThreads = 512;

struct SmallArgs {
  int32_t groups;
  int32_t first[host::kRoundGroups + 1];  // workgroups of each group of matrices
  struct {
    const void* src;
    int64_t stride, batch_stride;
    int32_t rows, cols;
    LastOut::Params out;
  } of[host::kRoundGroups];
  int32_t steps;
  float eps;
  float coefficients[3 * DASO_MAX_SCHULZ_STEPS];
};

template <class T, bool FULL>
__global__ __launch_bounds__(kSmallThreads, 2) void small_kernel(SmallArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  int g = 0;
  while (g + 1 < a.groups && static_cast<int>(blockIdx.x) >= a.first[g + 1]) ++g;
  const auto& of = a.of[g];
  const int batch = static_cast<int>(blockIdx.x) - a.first[g];
  const bool tall = of.rows > of.cols;
  const int m = tall ? of.cols : of.rows, n = tall ? of.rows : of.cols;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, kq = lane >> 4;
  const int stride = small_stride(n), plane = kSmallM * stride, n_steps = (n + 63) / 64;
  char* x_lds = lds;
  char* gram = lds + (FULL ? 2 : 1) * plane;  // planes of kSmallM * kGramStride
  float* rest = (float*)(gram + (FULL ? 2 : 1) * kSmallM * kGramStride);  // 64; and 8 doubles behind it
  double* sums = (double*)(rest + kSmallM);

  // X: x[i][j] has row j * 16 + r16 of columns (wave + 8 i) * 16 + kq * 4 ..
  f4 x[kSmallGroups][4];
  const T* src = (const T*)of.src + batch * of.batch_stride;
  // four neighbouring columns at a time, where they lie so: one by one, each load would touch 64 lines
  const bool wide = !tall && ((reinterpret_cast<uintptr_t>(src) | (of.stride * sizeof(T))) & (4 * sizeof(T) - 1)) == 0;
#pragma unroll
  for (int i = 0; i < kSmallGroups; ++i) {
    const int col = (wave + 8 * i) * 16 + kq * 4;
    if ((wave + 8 * i) * 16 >= n) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = j * 16 + r16;
      if (wide && col + 4 <= n) {
        x[i][j] = (f4)0.0f;
        if (row < m) x[i][j] = load4(src + row * of.stride + col);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          x[i][j][e] = row < m && col + e < n ? load1(src + (tall ? (col + e) * of.stride + row : row * of.stride + col + e)) : 0.0f;
      }
    }
  }
  double square = 0;
#pragma unroll
  for (int i = 0; i < kSmallGroups; ++i) {
    if ((wave + 8 * i) * 16 >= n) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) square += static_cast<double>(x[i][j][e]) * x[i][j][e];
  }
  const Normal scaled(group_sum(square, sums), a.eps);
  if (scaled.first != 1.0f)
#pragma unroll
    for (int i = 0; i < kSmallGroups; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) x[i][j] *= scaled.first;
#pragma unroll
  for (int i = 0; i < kSmallGroups; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) x[i][j] *= scaled.then;
  // columns between n and the last step's end are read as zeros
  for (int k = threadIdx.x; k < kSmallM * 8; k += kSmallThreads) {
    const int row = k >> 3, at = (n_steps * 64 - 64 + (k & 7) * 8) * 2;
#pragma unroll
    for (int p = 0; p < (FULL ? 2 : 1); ++p) *(half8*)(x_lds + p * plane + row * stride + at) = (half8)(_Float16)0.0f;
  }
  __syncthreads();

  const auto put = [&](char* to, int next_plane, const f4& v) {
    product::half4 h, l;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      _Float16 hi, lo;
      product::split(v[e], &hi, &lo);
      h[e] = hi, l[e] = lo;
    }
    *(product::half4*)to = h;
    if constexpr (FULL) *(product::half4*)(to + next_plane) = l;
    return h;
  };
  const auto multiply = [&](const half8 (&b)[FULL ? 2 : 1], const half8 (&c)[FULL ? 2 : 1], f4 acc) {
    if constexpr (FULL) {
      acc = product::mfma<false>(b[1], c[0], acc);
      acc = product::mfma<false>(b[0], c[1], acc);
    }
    return product::mfma<false>(b[0], c[0], acc);
  };
  // tiles (wave / 2, wave % 2 * 2) and the one to its right of a square product of rows in LDS
  const int ti = wave >> 1, tj = (wave & 1) * 2;
  const auto square_product = [&](const char* rows, int row_stride, int next_plane, int k_steps, f4 (&c)[2]) {
    c[0] = c[1] = (f4)0.0f;
    // 64 of the contraction at a time: what is read of LDS is on its way together
    for (int k = 0; k < k_steps; ++k) {
      half8 left[2][FULL ? 2 : 1], right[2][2][FULL ? 2 : 1];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int p = 0; p < (FULL ? 2 : 1); ++p) {
          const char* at = rows + p * next_plane + k * 128 + h * 64 + kq * 16;
          left[h][p] = *(const half8*)(at + (ti * 16 + r16) * row_stride);
#pragma unroll
          for (int t = 0; t < 2; ++t) right[h][t][p] = *(const half8*)(at + ((tj + t) * 16 + r16) * row_stride);
        }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < 2; ++t) c[t] = multiply(right[h][t], left[h], c[t]);
    }
  };
  // a square's tiles into their place, and what the diagonal's one plane lacks
  const auto put_square = [&](const f4 (&c)[2]) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int row = ti * 16 + r16, col = (tj + t) * 16 + kq * 4;
      const product::half4 h = put(gram + row * kGramStride + col * 2, kSmallM * kGramStride, c[t]);
      if constexpr (!FULL) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (col + e == row) rest[row] = c[t][e] - static_cast<float>(h[e]);
      }
    }
  };

  for (int step = 0; step < a.steps; ++step) {
    const float ca = a.coefficients[3 * step], cb = a.coefficients[3 * step + 1], cc = a.coefficients[3 * step + 2];
#pragma unroll
    for (int i = 0; i < kSmallGroups; ++i) {
      if ((wave + 8 * i) * 16 >= n) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j) put(x_lds + (j * 16 + r16) * stride + ((wave + 8 * i) * 16 + kq * 4) * 2, plane, x[i][j]);
    }
    __syncthreads();
    f4 gram_c[2], c[2];
    square_product(x_lds, stride, plane, n_steps, gram_c);
    gram_c[0] *= kUnscale, gram_c[1] *= kUnscale;
    put_square(gram_c);
    __syncthreads();
    square_product(gram, kGramStride, kSmallM * kGramStride, 1, c);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int row = ti * 16 + r16, col = (tj + t) * 16 + kq * 4;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float more = FULL ? 0.0f : rest[row] + rest[col + e];
        c[t][e] = fmaf(cb, gram_c[t][e], cc * kUnscale * fmaf(more, gram_c[t][e], c[t][e]));
      }
    }
    __syncthreads();  // the gram matrix and its rest have been read
    put_square(c);
    __syncthreads();
    half8 left[2][4][FULL ? 2 : 1];
    float more[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      more[j] = FULL ? 0.0f : rest[j * 16 + r16];
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int p = 0; p < (FULL ? 2 : 1); ++p)
          left[k][j][p] = *(const half8*)(gram + p * kSmallM * kGramStride + (j * 16 + r16) * kGramStride + k * 64 + kq * 16);
    }
#pragma unroll
    for (int i = 0; i < kSmallGroups; ++i) {
      const int col = (wave + 8 * i) * 16;
      if (col >= n) continue;
      f4 y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = (f4)0.0f;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        half8 right[FULL ? 2 : 1];  // column r16 of X, rows k * 32 + kq * 8 ..
#pragma unroll
        for (int p = 0; p < (FULL ? 2 : 1); ++p) {
          const char* at = x_lds + p * plane + (k * 32 + kq * 8 + (r16 >> 2)) * stride + (col + (r16 & 3) * 4) * 2;
          right[p] = __builtin_shufflevector(product::read_turned(at), product::read_turned(at + 4 * stride), 0, 1, 2, 3, 4, 5, 6, 7);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = multiply(right, left[k][j], y[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i][j][e] = fmaf(ca, x[i][j][e], kUnscale * fmaf(more[j], x[i][j][e], y[j][e]));
    }
    __syncthreads();  // X's planes and B have been read
  }

  const LastOut::Params& out = of.out;
  int64_t to = out.out_batch * batch, ld = out.out_ld;
  float lr = 0.0f;
  if (out.kind == LastOut::kStep) {
    const Entry e = out.table[batch];
    to = e.start, ld = of.cols, lr = e.step;
  }
  const int64_t esz = out.kind == LastOut::kBf16 ? 2 : 4;
  const uintptr_t base = reinterpret_cast<uintptr_t>(out.kind == LastOut::kStep ? (void*)out.params : out.out);
  const bool wide_out = !tall && ((base + to * esz) & (4 * esz - 1)) == 0 && ((to | ld) & 3) == 0;
#pragma unroll
  for (int i = 0; i < kSmallGroups; ++i) {
    const int col = (wave + 8 * i) * 16 + kq * 4;
    if ((wave + 8 * i) * 16 >= n) continue;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = j * 16 + r16;
      if (row >= m) continue;
      f4 v = x[i][j] * kUnscale;
      if (wide_out && col + 4 <= n) {
        const int64_t at = to + row * ld + col;
        if (out.kind == LastOut::kStep) {
          v = load4(out.params + at) * out.keep - lr * v;
          store4(out.params + at, v);
          if (out.wire != nullptr) store4(out.wire + at, v);
        } else if (out.kind == LastOut::kF32) {
          store4((float*)out.out + at, v);
        } else {
          store4((uint16_t*)out.out + at, v);
        }
        continue;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (col + e >= n) continue;
        const int64_t at = to + (tall ? (col + e) * ld + row : row * ld + col + e);
        if (out.kind == LastOut::kStep) {
          const float p = out.params[at] * out.keep - lr * v[e];
          out.params[at] = p;
          if (out.wire != nullptr) out.wire[at] = to_bf16(p);
        } else if (out.kind == LastOut::kF32) {
          ((float*)out.out)[at] = v[e];
        } else {
          ((uint16_t*)out.out)[at] = to_bf16(v[e]);
        }
      }
    }
  }
}

// ------------------------------------------------------------------------- host
_Float16* plane(char* ws, size_t at) { return reinterpret_cast<_Float16*>(ws + at); }

int32_t parts_of(int64_t elems) {
  const int64_t p = (elems + 8191) / 8192;
  return static_cast<int32_t>(p < 1 ? 1 : p > host::kSumParts ? host::kSumParts : p);
}

// Planes of X from the sources' matrices.  src: null for the round's own copies.
template <class T>
hipError_t normalise(const SchulzRound& r, char* ws, const T* src, int64_t src_batch, int64_t src_stride, int32_t parts,
                     float eps, bool only_step, hipStream_t stream) {
  LayOut a = {};
  a.groups = static_cast<int32_t>(r.groups.size());
  a.parts = parts;
  a.eps = eps;
  a.sums = reinterpret_cast<const double*>(ws + host::kRoundMatrices * sizeof(Entry));
  for (int32_t k = 0; k < a.groups; ++k) {
    const SchulzGroup& g = r.groups[k];
    PlanesArgs& p = a.p[k];
    p.src = src != nullptr ? (const void*)src : (const void*)(ws + g.source);
    p.stride = src != nullptr ? src_stride : g.cols;
    p.batch_stride = src != nullptr ? src_batch : g.rows * g.cols;
    p.rows = static_cast<int32_t>(g.rows), p.cols = static_cast<int32_t>(g.cols);
    p.rows_p = static_cast<int32_t>(g.tall ? g.n : g.m), p.cols_p = static_cast<int32_t>(g.tall ? g.m : g.n);
    // X, and for a tall matrix's last step, where that is the first, X^T, which the source then is
    for (int i = 0; i < 2; ++i) {
      uint16_t* x = reinterpret_cast<uint16_t*>(ws + g.x[0][i]);
      if (g.tall) p.t[i] = x;
      else p.d[i] = x;
      if (g.tall && only_step) p.d[i] = reinterpret_cast<uint16_t*>(ws + g.xt[i]);
    }
    a.first_matrix[k] = g.first;
    a.first_tile[k + 1] = a.first_tile[k] + int64_t(p.rows_p / 64) * (p.cols_p / 64) * g.count;
  }
  const int64_t tiles = a.first_tile[a.groups], row = int64_t(1) << 20;
  return launch(&normalise_kernel<T>, dim3(static_cast<uint32_t>(tiles < row ? tiles : row), static_cast<uint32_t>((tiles + row - 1) / row)),
                dim3(256), stream, a);
}

// Operands of a product: X's or the square's planes, in one segment or three.
void operands(product::Args& p, const _Float16* a_hi, const _Float16* a_lo, const _Float16* b_hi, const _Float16* b_lo,
              bool full) {
  p.segments = full ? 3 : 1;
  p.a[0] = a_hi, p.b[0] = b_hi;
  p.a[1] = a_hi, p.b[1] = b_lo;
  p.a[2] = a_lo, p.b[2] = b_hi;
}

// The steps of one round, from planes in buffer 0 to `last`, whose Params lack only what
// the steps know.
hipError_t schulz_steps(const SchulzRound& r, char* ws, int32_t steps, const float* coefficients, bool full,
                        const std::vector<LastOut::Params>& last, hipStream_t stream) {
  const int32_t groups = static_cast<int32_t>(r.groups.size());
  const product::Sums sums = {reinterpret_cast<float*>(ws + r.sums), r.sums_bytes};
  for (int32_t s = 0; s < steps; ++s) {
    const float a = coefficients[3 * s], b = coefficients[3 * s + 1], c = coefficients[3 * s + 2];
    const int from = s & 1, to = from ^ 1;
    const bool end = s + 1 == steps;
    product::Launch<PlanesOut> gram = {}, poly = {}, next = {};
    product::Launch<LastOut> wide = {}, tall = {};
    gram.count = poly.count = groups;
    for (int32_t k = 0; k < groups; ++k) {
      const SchulzGroup& g = r.groups[k];
      const int32_t m = static_cast<int32_t>(g.m), n = static_cast<int32_t>(g.n);
      _Float16 *x[2], *xt[2], *y[2], *q[2], *w[2];
      for (int i = 0; i < 2; ++i) {
        x[i] = plane(ws, g.x[from][i]), y[i] = plane(ws, g.x[to][i]), xt[i] = g.tall ? plane(ws, g.xt[i]) : nullptr;
        q[i] = plane(ws, g.gram[i]), w[i] = plane(ws, g.poly[i]);
      }
      float *rest_q = full ? nullptr : reinterpret_cast<float*>(ws + g.rest[0]), *rest_w = full ? nullptr : reinterpret_cast<float*>(ws + g.rest[1]);
      // A = X X^T
      product::Args& pa = gram.args[k];
      operands(pa, x[0], x[1], x[0], x[1], full);
      pa.lda = pa.ldb = n, pa.batch_a = pa.batch_b = int64_t(m) * n;
      pa.steps = n / 64, pa.M = pa.N = m, pa.tri = 1, pa.batch = g.count;
      PlanesOut::Params& ga = gram.out[k];
      ga.hi = ga.t_hi = q[0], ga.lo = ga.t_lo = full ? q[1] : nullptr;
      ga.ld = ga.t_ld = m, ga.batch = ga.t_batch = int64_t(m) * m;
      ga.alpha = kUnscale;
      ga.rest_out = rest_q, ga.rest_ld = m;
      // B = b A + c A A^T
      product::Args& pb = poly.args[k];
      operands(pb, q[0], q[1], q[0], q[1], full);
      pb.lda = pb.ldb = m, pb.batch_a = pb.batch_b = int64_t(m) * m;
      pb.steps = m / 64, pb.M = pb.N = m, pb.tri = 1, pb.batch = g.count;
      PlanesOut::Params& gb = poly.out[k];
      gb = ga;
      gb.in_hi = q[0], gb.in_lo = full ? q[1] : nullptr;
      gb.hi = gb.t_hi = w[0], gb.lo = gb.t_lo = full ? w[1] : nullptr;
      gb.alpha = c * kUnscale, gb.beta = b;
      gb.rest = rest_q, gb.rest_out = rest_w, gb.square = 1;
      // X' = a X + B X, X being read turned; the last step of a tall matrix as X^T B
      product::Args pc = {};
      pc.lda = m, pc.steps = m / 64, pc.batch = g.count;
      if (end && g.tall) {
        operands(pc, xt[0], xt[1], w[0], w[1], full);
        pc.ldb = m, pc.batch_a = int64_t(m) * n, pc.batch_b = int64_t(m) * m, pc.M = n, pc.N = m;
      } else {
        operands(pc, w[0], w[1], x[0], x[1], full);
        pc.ldb = n, pc.batch_a = int64_t(m) * m, pc.batch_b = int64_t(m) * n, pc.M = m, pc.N = n;
      }
      if (!end) {
        PlanesOut::Params& gc = next.out[next.count];
        gc.in_hi = x[0], gc.in_lo = x[1];
        gc.hi = y[0], gc.lo = y[1];
        gc.ld = n, gc.batch = gc.t_batch = int64_t(m) * n, gc.t_ld = m;
        if (g.tall && s + 2 == steps) gc.t_hi = xt[0], gc.t_lo = xt[1], gc.t_always = 1;
        gc.alpha = kUnscale, gc.beta = a;
        gc.rest = rest_w, gc.rest_ld = m;
        next.args[next.count++] = pc;
      } else {
        product::Launch<LastOut>& to_last = g.tall ? tall : wide;
        LastOut::Params& gc = to_last.out[to_last.count];
        gc = last[k];
        gc.in_hi = g.tall ? xt[0] : x[0], gc.in_lo = g.tall ? xt[1] : x[1];
        gc.ld = g.tall ? m : n, gc.batch = int64_t(m) * n;
        gc.alpha = kUnscale, gc.beta = a;
        gc.rest = rest_w, gc.rest_ld = m, gc.right = g.tall ? 1 : 0;
        gc.rows = static_cast<int32_t>(g.rows), gc.cols = static_cast<int32_t>(g.cols);
        to_last.args[to_last.count++] = pc;
      }
    }
    hipError_t e = product::launch_products<false, false>(gram, sums, stream);
    if (e == hipSuccess) e = product::launch_products<false, false>(poly, sums, stream);
    if (e == hipSuccess && next.count > 0) e = product::launch_products<false, true>(next, sums, stream);
    if (e == hipSuccess && wide.count > 0) e = product::launch_products<false, true>(wide, sums, stream);
    if (e == hipSuccess && tall.count > 0) e = product::launch_products<false, false>(tall, sums, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// The small matrices of a round, their groups' Params as for the products.
template <class T>
hipError_t small_steps(const SchulzRound& r, char* ws, const T* src, int64_t src_batch, int64_t src_stride, int32_t steps,
                       const float* coefficients, float eps, bool full, const std::vector<LastOut::Params>& last,
                       hipStream_t stream) {
  SmallArgs a = {};
  a.steps = steps, a.eps = eps;
  for (int32_t i = 0; i < 3 * steps; ++i) a.coefficients[i] = coefficients[i];
  int lds_bytes = 0;
  for (size_t k = 0; k < r.groups.size(); ++k) {
    const SchulzGroup& g = r.groups[k];
    if (!g.small) continue;
    auto& of = a.of[a.groups];
    of.src = src != nullptr ? (const void*)src : (const void*)(ws + g.source);
    of.stride = src != nullptr ? src_stride : g.cols;
    of.batch_stride = src != nullptr ? src_batch : g.rows * g.cols;
    of.rows = static_cast<int32_t>(g.rows), of.cols = static_cast<int32_t>(g.cols);
    of.out = last[k];
    a.first[a.groups + 1] = a.first[a.groups] + g.count;
    ++a.groups;
    lds_bytes = std::max(lds_bytes, host::small_lds(static_cast<int>(std::max(g.rows, g.cols)), full));
  }
  if (a.groups == 0) return hipSuccess;
  const void* kernel = full ? reinterpret_cast<const void*>(&small_kernel<T, true>) : reinterpret_cast<const void*>(&small_kernel<T, false>);
  static std::atomic<uint64_t> allowed[2];
  const hipError_t e = product::allow_lds(kernel, 160 * 1024, allowed[full ? 1 : 0]);
  if (e != hipSuccess) return e;
  void* list[] = {&a};
  return hipLaunchKernel(kernel, dim3(static_cast<uint32_t>(a.first[a.groups])), dim3(kSmallThreads), list,
                         static_cast<size_t>(lds_bytes), stream);
}

// A round from its sources to its results.  parts: the sums of squares of a matrix.
template <class T>
hipError_t run_round(const SchulzRound& r, char* ws, const T* src, int64_t src_batch, int64_t src_stride, int32_t parts,
                     int32_t steps, const float* coefficients, float eps, bool full, const std::vector<LastOut::Params>& last,
                     hipStream_t stream) {
  hipError_t e = small_steps<T>(r, ws, src, src_batch, src_stride, steps, coefficients, eps, full, last, stream);
  SchulzRound large = r;
  large.groups.clear();
  std::vector<LastOut::Params> large_last;
  for (size_t k = 0; k < r.groups.size(); ++k) {
    if (r.groups[k].small) continue;
    large.groups.push_back(r.groups[k]);
    large_last.push_back(last[k]);
  }
  if (e != hipSuccess || large.groups.empty()) return e;
  e = normalise<T>(large, ws, src, src_batch, src_stride, parts, eps, steps == 1, stream);
  return e == hipSuccess ? schulz_steps(large, ws, steps, coefficients, full, large_last, stream) : e;
}

size_t most_bytes(const std::vector<SchulzRound>& rounds) {
  size_t most = 0;
  for (const SchulzRound& r : rounds) most = r.bytes > most ? r.bytes : most;
  return most;
}

std::vector<host::Shape> shapes_of(const daso_muon_args& s) {
  std::vector<host::Shape> v;
  for (int32_t i = 0; i < s.nmatrices; ++i) v.push_back({s.matrices[i].rows, s.matrices[i].cols});
  return v;
}

// The matrices from `at` on.
template <class T>
hipError_t orthogonalize_round(const daso_orthogonalize_args& s, const SchulzRound& r, int64_t at, hipStream_t stream) {
  char* ws = static_cast<char*>(s.workspace);
  const SchulzGroup& g = r.groups[0];  // one shape
  const T* src = static_cast<const T*>(s.src) + at * s.src_batch_stride;
  const int64_t rows = s.rows;
  const int32_t parts = static_cast<int32_t>(std::min<int64_t>(parts_of(rows * s.cols), rows));
  double* sums = reinterpret_cast<double*>(ws + host::kRoundMatrices * sizeof(Entry));
  if (!g.small) {
    const hipError_t e = launch(&squares_kernel<T>, dim3(parts, g.count), dim3(256), stream, src, s.src_batch_stride, s.src_stride,
                                static_cast<int32_t>(rows), static_cast<int32_t>(s.cols), sums);
    if (e != hipSuccess) return e;
  }
  const bool full = s.out_type == DASO_TYPE_F32;
  LastOut::Params last = {};
  last.kind = full ? LastOut::kF32 : LastOut::kBf16;
  last.out = static_cast<char*>(s.out) + at * s.out_batch_stride * static_cast<int64_t>(host::bytes_of(s.out_type));
  last.out_ld = s.out_stride, last.out_batch = s.out_batch_stride;
  return run_round<T>(r, ws, src, s.src_batch_stride, s.src_stride, parts, s.steps, s.coefficients, s.eps, full, {last}, stream);
}

hipError_t muon_round(const daso_muon_args& s, const SchulzRound& r, hipStream_t stream) {
  char* ws = static_cast<char*>(s.workspace);
  Entry* table = reinterpret_cast<Entry*>(ws);
  MomentumArgs a = {};
  for (int32_t k = 0; k < s.g; ++k) a.grads[k] = s.grads[k];
  a.momentum = s.momentum;
  a.table = table;
  a.sums = reinterpret_cast<double*>(ws + host::kRoundMatrices * sizeof(Entry));
  a.g = s.g, a.nesterov = (s.flags & DASO_MUON_NESTEROV) ? 1 : 0, a.mu = s.mu;
  RoundTable t = {};
  t.count = static_cast<int32_t>(r.matrices.size());
  t.groups = static_cast<int32_t>(r.groups.size());
  int64_t most = 0;
  for (int32_t k = 0; k < t.groups; ++k) {
    const SchulzGroup& g = r.groups[k];
    t.first[k] = g.first;
    t.elems[k] = g.rows * g.cols;
    t.source[k] = reinterpret_cast<float*>(ws + g.source);
    most = std::max(most, t.elems[k]);
  }
  t.first[t.groups] = t.count;
  for (int32_t i = 0; i < t.count; ++i) {
    const daso_matrix& m = s.matrices[r.matrices[i]];
    t.start[i] = m.start;
    t.step[i] = s.lr * m.scale;
  }
  const int32_t parts = parts_of(most);
  hipError_t e = launch(&momentum_kernel, dim3(parts, t.count), dim3(256), stream, a, t);
  if (e != hipSuccess) return e;
  std::vector<LastOut::Params> last(r.groups.size());
  for (int32_t k = 0; k < t.groups; ++k) {
    LastOut::Params& p = last[k];
    p = {};
    p.kind = LastOut::kStep;
    p.table = table + r.groups[k].first;
    p.params = s.params, p.wire = s.wire;
    p.keep = 1.0f - s.lr * s.weight_decay;
  }
  return run_round<float>(r, ws, nullptr, 0, 0, parts, s.steps, s.coefficients, s.eps, true, last, stream);
}

}  // namespace
}  // namespace daso

using daso::host::SchulzRound;

extern "C" {

int daso_orthogonalize_workspace(const daso_orthogonalize_args* args, size_t* bytes) {
  if (args == nullptr || bytes == nullptr) return DASO_EINVAL;
  const int rc = daso::host::check_orthogonalize_sizes(*args);
  if (rc != DASO_OK) return rc;
  *bytes = 0;
  if (args->batch == 0 || args->rows == 0 || args->cols == 0) return DASO_OK;
  try {
    *bytes = daso::host::plan_batch(args->batch, {args->rows, args->cols}, args->out_type == DASO_TYPE_F32).full.bytes;
  } catch (const std::bad_alloc&) {
    return DASO_EHIP;
  }
  return DASO_OK;
}

int daso_orthogonalize(const daso_orthogonalize_args* args, hipStream_t stream) {
  if (args == nullptr) return DASO_EINVAL;
  const daso_orthogonalize_args& s = *args;
  int rc = daso::host::check_orthogonalize(s);
  if (rc != DASO_OK || s.batch == 0 || s.rows == 0 || s.cols == 0) return rc;
  try {
    const daso::host::SchulzBatch b = daso::host::plan_batch(s.batch, {s.rows, s.cols}, s.out_type == DASO_TYPE_F32);
    if ((rc = daso::host::check_workspace(s.workspace, s.workspace_bytes, b.full.bytes)) != DASO_OK) return rc;
    if ((rc = daso::current_device(stream)) != DASO_OK) return rc;
    for (int64_t k = 0; k < b.rounds; ++k) {
      const SchulzRound& r = k + 1 < b.rounds ? b.full : b.last;
      const hipError_t e = s.type == DASO_TYPE_F32 ? daso::orthogonalize_round<float>(s, r, k * b.each, stream)
                                                   : daso::orthogonalize_round<uint16_t>(s, r, k * b.each, stream);
      if (e != hipSuccess) return DASO_EHIP;
    }
  } catch (const std::bad_alloc&) {
    return DASO_EHIP;
  }
  return DASO_OK;
}

int daso_muon_workspace(const daso_muon_args* args, size_t* bytes) {
  if (args == nullptr || bytes == nullptr) return DASO_EINVAL;
  try {
    const int rc = daso::host::check_muon_sizes(*args);
    if (rc != DASO_OK) return rc;
    *bytes = daso::most_bytes(daso::host::plan_rounds(daso::shapes_of(*args), true, true));
  } catch (const std::bad_alloc&) {
    return DASO_EHIP;
  }
  return DASO_OK;
}

int daso_muon_step(const daso_muon_args* args, hipStream_t stream) {
  if (args == nullptr) return DASO_EINVAL;
  const daso_muon_args& s = *args;
  try {
    int rc = daso::host::check_muon(s);
    if (rc != DASO_OK || s.n == 0 || s.nmatrices == 0) return rc;
    const std::vector<SchulzRound> rounds = daso::host::plan_rounds(daso::shapes_of(s), true, true);
    if ((rc = daso::host::check_workspace(s.workspace, s.workspace_bytes, daso::most_bytes(rounds))) != DASO_OK) return rc;
    if ((rc = daso::current_device(stream)) != DASO_OK) return rc;
    for (const SchulzRound& r : rounds)
      if (daso::muon_round(s, r, stream) != hipSuccess) return DASO_EHIP;
  } catch (const std::bad_alloc&) {
    return DASO_EHIP;
  }
  return DASO_OK;
}

}  // extern "C"
