// The cross entropy of an output projection and its gradients (daso_train.h), over pieces of
// the vocabulary, without keeping the logits.
//
// Forward: one product hidden weight^T, whose epilogue reduces each 256 (or 128) columns of a
// row to their maximum and their sum of exponentials; a second kernel joins them.
// Backward, per piece of the vocabulary: the piece's logits again, whose epilogue turns them
// into s (p - onehot), stored as 16-bit planes; then dhidden += dz weight
// and dweight = dz^T hidden, in one launch.  6 N V d multiply-adds at least, 8 with the logits taken
// twice: keeping them would cost N V 4 bytes written and read, which takes as long as the
// product at d = 1024 and grows the memory by N V.
//
// Bound by the matrix cores: 4096 tokens over 50257 classes of 1024 features forward in 364 to 395 us by machine
// (1070 to 1160 TFLOP/s; 16 steps a tile leave less of the pipeline's rate than 128 do), 8192 with gradients
// and an fp32 dweight in 4.0 ms, 4.2 PFLOP counting the logits twice and dweight in two planes.  A few
// tokens or classes are bound by the chain of eight launches, 3 to 18 us each.  Where a launch has few tiles, they are cut, and
// the parts' sums of logits lie in the workspace until the second kernel has added them.
//
// Numbers.  bf16 operands are multiplied as they are in the forward product; fp32 ones as two
// binary16 planes each (22 bits), hidden scaled by a power of two from each row's largest value, weight by one from the
// tensor's.  In the backward products dz is binary16, a token's values in [-1, 1] times 2^14 and the power of
// two of its dloss, which keeps 3 bits more than bf16 would whatever the other tokens' dloss are.  For dhidden
// that power comes back by rows in the epilogue; for dweight it is put into hidden's rows, where those of tokens without a
// gradient are zeros.  They and weight are turned to binary16 by a scale each (exact for a bf16 value within 2^-31 of the
// largest), so that a bf16 result is off by 2e-4 before it is rounded; fp32 results take dz as two planes.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <new>

#include "daso_planes.h"
#include "daso_product.h"
#include "daso_train_host.h"

namespace daso {
namespace {

using product::f4;
using product::half4;
using product::half8;

constexpr float kLog2E = 1.44269504f;
// exp(z - m) is 2^(z log2 e - m log2 e) in one multiply-add, whose second product is rounded: of m = 2^10 it is off by up to
// 2^-14, of 2^32 by 2^8, and the power by its exponential.  From here on m is subtracted first.
constexpr float kLargeLogit = 1 << 10;
constexpr int kProbExponent = 14;  // dz is in [-1, 1] times its token's power of two; as binary16, times 2^14

// Exponents of scales: weight times 2^to is below 2^15, and hidden, each token's with its dloss's power of two, likewise.
enum Tensor { kHidden, kWeight };
constexpr int kTopParts = 512;     // workgroups that look for the largest values of one
constexpr int kNone = -(1 << 20);  // the exponent of zero
struct Scales {
  int32_t top[2][kTopParts];  // exponents of the largest finite magnitudes
  int32_t to[2];
};

// What the backward epilogues need of a token.
struct Row {
  float lse;
  float g;         // dloss times 2^(kProbExponent - by)
  int32_t target;  // -1: the whole row is zero
  int16_t to;      // fp32 operands: the exponent of its scale in the logits
  int16_t by;      // dloss times 2^-by is in [-1, 1]
};

// floor(log2) of a magnitude (of a subnormal one the least normal's).
__device__ inline int exponent_of(float magnitude) {
  const uint32_t bits = __builtin_bit_cast(uint32_t, magnitude);
  return bits == 0 ? kNone : static_cast<int>(max(bits >> 23, 1u)) - 127;
}
// The exponent that brings what has `top` for its largest value's into binary16, below 2^15.
__device__ inline int to_half(int top) { return top == kNone ? 0 : 14 - top; }

// What a token's part in the gradients goes by.
struct Token {
  float dloss;
  int64_t target;
  // The power of two that its dloss is taken by; kNone: nothing of the token reaches the gradients, whatever it holds.
  __device__ int by(int64_t ignore) const {
    if (target == ignore || dloss == 0.0f) return kNone;
    const float m = __builtin_fabsf(dloss);
    return m < __builtin_inff() ? exponent_of(m) + 1 : 0;
  }
};

struct TopArgs {
  const void *hidden, *weight;
  int64_t hidden_stride, weight_stride, tokens, vocab, d;
  const float* dloss;  // null: only the rows' own are wanted of hidden
  const int64_t* targets;
  int64_t ignore;
  int32_t* row_top;    // of each token's hidden
  Scales* out;
};

__device__ inline void take_finite(float v, float& m) {
  v = __builtin_fabsf(v);
  m = fmaxf(m, v < __builtin_inff() ? v : 0.0f);
}

// The largest magnitude of a run of elements, of which a thread takes eight in four places at a time.
template <class T>
__device__ inline float top_of_run(const T* src, int64_t n) {
  float m = 0.0f;
  const int64_t whole = n / 8 * 8, id = blockIdx.x * 256 + threadIdx.x, step = gridDim.x * int64_t(2048);
  for (int64_t i = id * 8; i < whole; i += 4 * step) {
    float v[4][8] = {};
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * step < whole) load8(src + i + k * step, v[k]);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) take_finite(v[k][j], m);
  }
  if (whole + id < n) take_finite(load1(src + whole + id), m);
  return wave_max(m);
}

// Calls f(row, largest magnitude, get(row)), in every lane, for a wavefront's rows, get before they are read: four rows at a
// time for loads in flight, or, where there are no more rows than wavefronts, four places of one (a classifier's 256 rows of
// 2048: 1.5 us less).
template <class T, class G, class F>
__device__ inline void tops_of_rows(const T* src, int64_t stride, int64_t rows, int64_t cols, G get, F f) {
  const int64_t wave = (blockIdx.x * 256 + threadIdx.x) >> 6, waves = gridDim.x * 4;
  const int lane = threadIdx.x & 63;
  const int64_t whole = cols / 8 * 8;
  const bool few = rows <= waves;
  const int64_t next = few ? 0 : waves, along = few ? 512 : 0, step = few ? 2048 : 512;
  for (int64_t r = wave; r < rows; r += 4 * waves) {
    float m[4] = {};
    decltype(get(r)) with[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) with[k] = get(min(r + k * next, rows - 1));
    for (int64_t c = lane * 8; c < whole; c += step) {
      float v[4][8] = {};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (r + k * next < rows && c + k * along < whole) load8(src + (r + k * next) * stride + c + k * along, v[k]);
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) take_finite(v[k][i], m[k]);
    }
    if (whole + lane < cols) {
      float v[4] = {};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (r + k * next < rows) v[k] = load1(src + (r + k * next) * stride + whole + lane);
#pragma unroll
      for (int k = 0; k < 4; ++k) take_finite(v[k], m[k]);
    }
    if (few) {
      f(r, wave_max(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]))), with[0]);
      continue;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (r + k * waves < rows) f(r + k * waves, wave_max(m[k]), with[k]);
  }
}

// Workgroup (x, y): part x of tensor y.
template <class T>
__global__ __launch_bounds__(256) void tops_kernel(TopArgs a) {
  __shared__ int32_t shared[4];
  int top = kNone;
  if (blockIdx.y == kHidden) {
    const auto token = [&](int64_t row) { return a.dloss != nullptr ? Token{a.dloss[row], a.targets[row]} : Token{0.0f, 0}; };
    tops_of_rows((const T*)a.hidden, a.hidden_stride, a.tokens, a.d, token, [&](int64_t row, float m, const Token& t) {
      const int e = exponent_of(m), by = t.by(a.ignore);
      if ((threadIdx.x & 63) == 0) a.row_top[row] = e;
      if (e != kNone && by != kNone) top = max(top, e + by);
    });
  } else if (a.weight_stride == a.d) {
    top = exponent_of(top_of_run((const T*)a.weight, a.vocab * a.d));
  } else {
    tops_of_rows((const T*)a.weight, a.weight_stride, a.vocab, a.d, [](int64_t) { return 0; },
                 [&](int64_t, float m, int) { top = max(top, exponent_of(m)); });
  }
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = top;
  __syncthreads();
  if (threadIdx.x == 0) a.out->top[blockIdx.y][blockIdx.x] = max(max(shared[0], shared[1]), max(shared[2], shared[3]));
}

// The exponent of a tensor's scale, by a workgroup of 256.
__device__ inline int scale_exponent(const Scales* s, int tensor, int32_t* shared) {
  int m = max(s->top[tensor][threadIdx.x], s->top[tensor][threadIdx.x + 256]);
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) m = max(m, __shfl_xor(m, k));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = m;
  __syncthreads();
  m = max(max(shared[0], shared[1]), max(shared[2], shared[3]));
  return to_half(m);
}
static_assert(kTopParts == 512, "two parts a thread");

// What comes before the products of a pass, in one launch: planes of hidden and weight, and the
// backward pass's rows.
constexpr int kMaxPlanes = 4;
// Not at all; rows of hidden for the logits; weight; rows of hidden for dweight, each with its dloss's power of two.
enum ScaleBy { kRaw, kByRow, kByWeight, kByGrad };
struct PrepareArgs {
  int32_t count;
  int64_t first[kMaxPlanes + 2];  // workgroups of each job: the planes, then the rows
  PlanesArgs planes[kMaxPlanes];
  int32_t by[kMaxPlanes];         // how a job's values are scaled
  Scales* scales;                 // null: none are needed
  const int32_t* row_top;
  Row* rows;
  int64_t padded, tokens, vocab;
  const float *lse, *dloss;
  const int64_t* targets;
  int64_t ignore;
};

template <class T>
__global__ __launch_bounds__(256) void prepare_kernel(PrepareArgs a) {
  __shared__ uint16_t lds[2][64][66];
  __shared__ int32_t shared[4];
  const int64_t id = blockIdx.x + int64_t(blockIdx.y) * gridDim.x;
  if (id >= a.first[a.count + 1]) return;
  if (id == 0 && a.scales != nullptr) {
    for (int t = 0; t < 2; ++t) {
      const int e = scale_exponent(a.scales, t, shared);
      if (threadIdx.x == 0) a.scales->to[t] = e;
    }
  }
  if (id < a.first[a.count]) {
    int k = 0;
    while (id >= a.first[k + 1]) ++k;
    const PlanesArgs& p = a.planes[k];
    const int64_t t = id - a.first[k], across = p.cols_p / 64;
    const int tr = static_cast<int>(t / across), tc = static_cast<int>(t % across);
    if (a.by[k] == kRaw) {
      planes_tile<T, true>(p, 0, tr, tc, [](float v) { return v; }, lds);
      return;
    }
    const int row = min(tr * 64 + static_cast<int>(threadIdx.x >> 2), p.rows - 1);  // this thread's
    const bool grad = a.by[k] == kByGrad;
    const Token token = grad ? Token{a.dloss[row], a.targets[row]} : Token{0.0f, 0};
    const int to_all = a.by[k] == kByRow ? to_half(a.row_top[row]) : scale_exponent(a.scales, grad ? kHidden : kWeight, shared);
    const int by = grad ? token.by(a.ignore) : 0, to = to_all + by;
    planes_tile<T, false>(p, 0, tr, tc, [to, by](float v) { return by == kNone ? 0.0f : __builtin_ldexpf(v, to); }, lds);
    return;
  }
  const int64_t i = (id - a.first[a.count]) * 256 + threadIdx.x;
  if (i >= a.padded) return;
  Row r = {0.0f, 0.0f, -1, 0, 0};
  if (i < a.tokens) {
    const int64_t t = a.targets[i];
    const Token token = {a.dloss[i], t};
    const int by = token.by(a.ignore);
    if (t >= 0 && t < a.vocab) {
      if (by != kNone) {
        r.lse = a.lse[i];
        r.g = __builtin_ldexpf(token.dloss, kProbExponent - by);
        r.target = static_cast<int32_t>(t);
        r.to = static_cast<int16_t>(to_half(a.row_top[i]));
        r.by = static_cast<int16_t>(by);
      }
    } else if (t != a.ignore) {
      r.g = __builtin_nanf("");
      r.target = 0;
    }
  }
  a.rows[i] = r;
}

// ------------------------------------------------------------------------- forward epilogue
// For each row the maximum and the sum of exponentials of the tile's columns, and the logit of
// the target where the tile has it.  With SCALED the operands' scaling is taken back first, by its exponent: as a factor
// it may be zero or infinite where the logits are neither.
template <bool SCALED>
struct LseOut {
  static constexpr auto kKind = product::kWhole;
  struct Params {
    float2* parts;  // [tile column][token]
    float* at_target;
    const int64_t* targets;
    const int32_t *row_top, *to_b;  // SCALED: of the left operand's rows, and the exponent of the right one's scale
  };
  // Strip i of a band: 16 rows of it a wavefront, 64 columns of which are in c (two blocks' two
  // columns of 16).
  template <class Tile>
  __device__ static void strip(const Params& out, const product::Args& p, const product::Place& at, const f4& c0, const f4& c1,
                               const f4& c2, const f4& c3, int band, int i, int32_t target, int shift, int wave, int lane,
                               float2* to) {
    const int kq = lane >> 4;
    int row0, col0, col1;
    Tile::block_at(wave, band * 2, &row0, &col0);
    Tile::block_at(wave, band * 2 + 1, &row0, &col1);
    const int row = at.tm * Tile::kRows + row0 + i * 16 + (lane & 15);
    const f4 c[4] = {c0, c1, c2, c3};
    const auto column = [&](int k, int e) { return at.tn * Tile::kCols + (k < 2 ? col0 : col1) + (k & 1) * 16 + kq * 4 + e; };
    float z[16], m = -__builtin_inff();
#pragma unroll
    for (int k = 0; k < 16; ++k) z[k] = SCALED ? __builtin_ldexpf(c[k / 4][k % 4], shift) : c[k / 4][k % 4];
    // few tiles hold a row's target, and fewer reach past the classes
    if (target >= at.tn * Tile::kCols && target - at.tn * Tile::kCols < Tile::kCols)
#pragma unroll
      for (int k = 0; k < 16; ++k)
        if (target == column(k / 4, k % 4)) out.at_target[row] = z[k];
    if ((at.tn + 1) * Tile::kCols > p.N)
#pragma unroll
      for (int k = 0; k < 16; ++k) z[k] = column(k / 4, k % 4) < p.N ? z[k] : -__builtin_inff();
#pragma unroll
    for (int k = 0; k < 16; ++k) m = fmaxf(m, z[k]);
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    // columns that are all -inf, or none, add nothing; +inf or NaN make the sum NaN
    float base = m == -__builtin_inff() ? 0.0f : m * kLog2E, s = 0.0f;
    if (__builtin_fabsf(base) >= kLargeLogit) {
#pragma unroll
      for (int k = 0; k < 16; ++k) z[k] -= m;
      base = 0.0f;
    }
#pragma unroll
    for (int k = 0; k < 16; ++k) s += __builtin_amdgcn_exp2f(fmaf(z[k], kLog2E, -base));
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if (kq == 0) *to = make_float2(m, s);
  }
  // A row's parts of the wavefronts side by side.
  template <int kAcross>
  __device__ static void row_of(const Params& out, const product::Args& p, const product::Place& at, int row, const float2* from) {
    if (row >= p.M) return;
    float m = -__builtin_inff(), s = 0.0f;
#pragma unroll
    for (int w = 0; w < kAcross; ++w) m = fmaxf(m, from[w].x);
    const float base = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
    for (int w = 0; w < kAcross; ++w) s += from[w].y * __expf(from[w].x - base);
    out.parts[int64_t(at.tn) * p.M + row] = make_float2(m, s);
  }
  // What takes the scales of a row's logits back.
  __device__ static int shift_of(const Params& out, const product::Args& p, int row) {
    return SCALED ? -(to_half(out.row_top[min(row, p.M - 1)]) + *out.to_b) : 0;
  }
  // A row's target as a column of the product, or none.
  __device__ static int32_t target_of(const Params& out, const product::Args& p, int row) {
    const int64_t t = out.targets[min(row, p.M - 1)];
    return row < p.M && t >= 0 && t < p.N ? static_cast<int32_t>(t) : -1;
  }

  template <class Tile>
  __device__ static void tile(const Params& out, const product::Args& p, const product::Place& at, f4 (&acc)[Tile::kBlocks][8],
                              char* lds) {
    constexpr int kAcross = Tile::kThreads / 128;  // wavefronts side by side, of two rows of them
    constexpr int kBands = Tile::kBlocks / 2;      // runs of 64 rows a wavefront holds
    const int lane = product::thread_here() & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    float2* shared = (float2*)lds;  // [row][kAcross]
    int32_t target[kBands][4], shift[kBands][4];
    int row0, col0;
#pragma unroll
    for (int k = 0; k < kBands * 4; ++k) {
      Tile::block_at(wave, k / 4 * 2, &row0, &col0);
      const int row = at.tm * Tile::kRows + row0 + k % 4 * 16 + (lane & 15);
      target[k / 4][k % 4] = target_of(out, p, row), shift[k / 4][k % 4] = shift_of(out, p, row);
    }
#pragma unroll
    for (int band = 0; band < kBands; ++band)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        Tile::block_at(wave, band * 2, &row0, &col0);
        strip<Tile>(out, p, at, acc[band * 2][i * 2], acc[band * 2][i * 2 + 1], acc[band * 2 + 1][i * 2], acc[band * 2 + 1][i * 2 + 1],
                    band, i, target[band][i], shift[band][i], wave, lane, shared + (row0 + i * 16 + (lane & 15)) * kAcross + wave % kAcross);
      }
    __syncthreads();
    for (int in = threadIdx.x; in < Tile::kRows; in += Tile::kThreads)
      row_of<kAcross>(out, p, at, at.tm * Tile::kRows + in, shared + in * kAcross);
  }
  // Strip `i` of `band` alone, of a tile whose values c are the sums of its parts.
  template <class Tile>
  __device__ static void part(const Params& out, const product::Args& p, const product::Place& at, const f4 (&c)[4], int band, int i) {
    constexpr int kAcross = Tile::kThreads / 128;
    __shared__ float2 shared[2 * 16 * kAcross];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int row0, col0;
    Tile::block_at(wave, band * 2, &row0, &col0);
    const int row = at.tm * Tile::kRows + row0 + i * 16 + (lane & 15);
    strip<Tile>(out, p, at, c[0], c[1], c[2], c[3], band, i, target_of(out, p, row), shift_of(out, p, row), wave, lane,
                shared + (wave / kAcross * 16 + (lane & 15)) * kAcross + wave % kAcross);
    __syncthreads();
    if (threadIdx.x >= 32) return;
    Tile::block_at((threadIdx.x >> 4) * kAcross, band * 2, &row0, &col0);
    row_of<kAcross>(out, p, at, at.tm * Tile::kRows + row0 + i * 16 + (threadIdx.x & 15), shared + threadIdx.x * kAcross);
  }
};

// Joins a token's parts: 16 tokens a workgroup, 16 shares of the parts each, four of which are on
// their way at a time.
__global__ __launch_bounds__(256) void join_kernel(const float2* parts, int32_t count, int64_t tokens, int64_t vocab,
                                                   const int64_t* targets, int64_t ignore, const float* at_target, float* loss,
                                                   float* lse) {
  __shared__ float2 shared[16][16];
  const int in = threadIdx.x & 15, share = threadIdx.x >> 4;
  const int64_t i = blockIdx.x * int64_t(16) + in;
  float m = -__builtin_inff(), s = 0.0f;
  bool bad = false;
  if (i < tokens)
    for (int32_t k = share; k < count; k += 64) {
      float2 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = parts[min(k + 16 * j, count - 1) * tokens + i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (k + 16 * j >= count) continue;
        bad = bad || v[j].y != v[j].y;
        if (v[j].x > m) s = s * __expf(m - v[j].x), m = v[j].x;
        if (v[j].x > -__builtin_inff()) s += v[j].y * __expf(v[j].x - m);
      }
    }
  shared[share][in] = make_float2(m, bad ? __builtin_nanf("") : s);
  __syncthreads();
  if (share != 0 || i >= tokens) return;
  m = shared[0][in].x;
  for (int k = 1; k < 16; ++k) m = fmaxf(m, shared[k][in].x);
  s = 0.0f;
  for (int k = 0; k < 16; ++k) {
    const float2 v = shared[k][in];
    s += v.x > -__builtin_inff() ? v.y * __expf(v.x - m) : v.y;
  }
  const float l = m + logf(s);
  lse[i] = l;
  const int64_t t = targets[i];
  loss[i] = t == ignore ? 0.0f : t >= 0 && t < vocab ? l - at_target[i] : __builtin_nanf("");
}

// ------------------------------------------------------------------------- backward epilogues
// dz of a piece's columns as planes; columns beyond the vocabulary are zero.
template <bool SCALED>
struct ProbOut {
  static constexpr auto kKind = product::kBlocks;
  struct Params {
    const Row* rows;
    _Float16 *hi, *lo;  // lo may be null
    int64_t ld;
    int32_t first, columns, padded;  // the piece: its first class, its classes, its columns with padding
    int32_t padded_rows;             // tokens with padding: the planes are contracted over both
    const int32_t* to_b;             // SCALED: the exponent of the right operand's scale
  };
  struct Inputs {
    Row rows[4];
  };
  __device__ static void fetch(const Params& out, const product::Place&, int row0, int, int lane, Inputs& in) {
    if (row0 >= out.padded_rows) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) in.rows[i] = out.rows[row0 + i * 16 + (lane & 15)];
  }
  template <class F>
  __device__ static void block(const Params& out, const product::Place&, const f4 (&acc)[8], int row0, int col0, char* hi, int lane,
                               const Inputs& in, F next) {
    if (row0 >= out.padded_rows || col0 >= out.padded) {
      next();
      return;
    }
    const int r16 = lane & 15, kq = lane >> 4;
    char* lo = hi + product::kStagePlane;
    const int to_b = SCALED ? *out.to_b : 0;
    const bool two = out.lo != nullptr, edge = col0 + product::kBlockCols > out.columns;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const Row r = in.rows[i];
      float base = r.lse * kLog2E;
      const int target = r.target - out.first - col0;
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = SCALED ? __builtin_ldexpf(acc[i * 2 + k / 4][k % 4], -(r.to + to_b)) : acc[i * 2 + k / 4][k % 4];
      if (__builtin_fabsf(base) >= kLargeLogit) {
        // (a logit that is summed in another order than the forward pass's may come out above the log-sum-exp)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = v[k] > r.lse ? 0.0f : v[k] - r.lse;
        base = 0.0f;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = __builtin_amdgcn_exp2f(fmaf(v[k], kLog2E, -base));
      // few blocks hold a row's target, and fewer reach past the classes
      if (target >= 0 && target < product::kBlockCols)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] -= k / 4 * 16 + kq * 4 + k % 4 == target ? 1.0f : 0.0f;
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = r.target >= 0 ? v[k] * r.g : 0.0f;
      if (edge)
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = col0 + k / 4 * 16 + kq * 4 + k % 4 < out.columns ? v[k] : 0.0f;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        half4 h, l;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          _Float16 a, c;
          product::split(v[j * 4 + e], &a, &c);
          h[e] = a, l[e] = c;
        }
        *(half4*)(hi + product::plane_at(i * 16 + r16, j * 16 + kq * 4)) = h;
        if (two) *(half4*)(lo + product::plane_at(i * 16 + r16, j * 16 + kq * 4)) = l;
      }
    }
    next();
    product::wait_lds();
    __builtin_amdgcn_wave_barrier();
    const auto straight = [&](const char* plane, _Float16* to) {
#pragma unroll
      for (int pass = 0; pass < product::kPasses; ++pass) {
        const int r = product::pass_row(pass, lane), c = product::pass_col(lane);
        *(half8*)(to + int64_t(row0 + r) * out.ld + col0 + c) = *(const half8*)(plane + product::plane_at(r, c));
      }
    };
    straight(hi, out.hi);
    if (two) straight(lo, out.lo);
  }
};

// A gradient: C with the scales of dz and its partner taken back [+ sum], as the sum so far or as the result; or, where
// `turned`, C^T of that.
struct GradOut {
  static constexpr auto kKind = product::kStaged;
  struct Params {
    const Row* tokens;   // of dhidden's rows: the powers of two of their dloss; null: they are in the partner
    const int32_t* to;   // the exponent of the partner's scale
    const float* before;  // the sum of the pieces so far, or null
    int64_t before_ld;
    void* out;
    int64_t ld;
    int32_t bf16;
    int32_t rows, cols;  // of what is written
    int32_t turned;
  };
  struct Inputs {
    float before[product::kPasses][8];
    int shift[product::kPasses];  // what takes the scales back, by rows
  };
  __device__ static void fetch(const Params& p, const product::Place&, int row, int col, int lane, Inputs& in) {
    const int r0 = row + product::pass_row(0, lane), cc = col + product::pass_col(lane);
    const int to = *p.to + kProbExponent;
#pragma unroll
    for (int pass = 0; pass < product::kPasses; ++pass)
      in.shift[pass] = (p.tokens != nullptr ? p.tokens[r0 + pass * product::kPassRows].by : 0) - to;
    if (p.before == nullptr) return;
#pragma unroll
    for (int pass = 0; pass < product::kPasses; ++pass)  // padded to whole vectors
      if (r0 + pass * product::kPassRows < p.rows && cc < p.cols) load8(p.before + int64_t(r0 + pass * product::kPassRows) * p.before_ld + cc, in.before[pass]);
  }
  template <class F>
  __device__ static void block(const Params& p, const product::Place&, int row, int col, char* stage, int lane, const Inputs& in,
                               F next) {
    if (p.turned) {
      // 8 columns of C in a pass, 8 lanes a column, 8 rows of it each
      const int cc = row + (lane & 7) * 8, left = p.cols - cc;
      float v[4][8];
#pragma unroll
      for (int pass = 0; pass < 4; ++pass)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int r = (lane & 7) * 8 + i, c = pass * 8 + (lane >> 3);
          v[pass][i] = *(const float*)(stage + r * 128 + (((c >> 2) ^ ((r >> 1) & 7)) * 16) + (c & 3) * 4);
          v[pass][i] = __builtin_ldexpf(v[pass][i], in.shift[0]);
        }
      next();
#pragma unroll
      for (int pass = 0; pass < 4; ++pass) {
        const int rr = col + pass * 8 + (lane >> 3);
        if (rr < p.rows && left > 0) store_run(p, rr * p.ld + cc, left, v[pass]);
      }
      return;
    }
    const int r0 = row + product::pass_row(0, lane), cc = col + product::pass_col(lane), left = p.cols - cc;
    float v[product::kPasses][8];
#pragma unroll
    for (int pass = 0; pass < product::kPasses; ++pass) {
      product::pass_values(stage, pass, lane, v[pass]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[pass][i] = __builtin_ldexpf(v[pass][i], in.shift[pass]);
        if (p.before != nullptr) v[pass][i] += in.before[pass][i];
      }
    }
    next();
#pragma unroll
    for (int pass = 0; pass < product::kPasses; ++pass) {
      if (r0 + pass * product::kPassRows >= p.rows || left <= 0) continue;
      store_run(p, (r0 + pass * product::kPassRows) * p.ld + cc, left, v[pass]);
    }
  }
  // Eight neighbouring values, or the `left` of them that there are.
  __device__ static void store_run(const Params& p, int64_t to, int left, const float (&v)[8]) {
    float* const o32 = (float*)p.out + to;
    uint16_t* const o16 = (uint16_t*)p.out + to;
    if (left >= 8) {
      if (p.bf16) store8(o16, v);
      else store8(o32, v);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (i >= left) continue;
        if (p.bf16) o16[i] = to_bf16(v[i]);
        else o32[i] = v[i];
      }
    }
  }
};

template <class T>
__global__ __launch_bounds__(256) void zero_rows_kernel(T* out, int64_t stride, int64_t rows, int64_t cols) {
  const int64_t n = rows * cols;
  for (int64_t i = blockIdx.x * int64_t(256) + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256)
    out[i / cols * stride + i % cols] = T(0);
}

// ------------------------------------------------------------------------- host
int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// The backward pass takes the vocabulary in pieces of so many classes that a plane of dz
// holds 2^27 values, which bounds the workspace (256 MB a plane).  Each piece is two launches whose last
// tiles leave CUs idle, and reads dhidden's sum so far: 8192 tokens x 50257 classes x 1024 with an fp32
// dweight take 4.27 ms with 2^26, 4.09 with 2^27, 3.98 with 2^28, and twice the memory each time.
constexpr int64_t kPieceElems = int64_t(1) << 27;

struct Plan {
  int64_t n_p, d_p, v_p;          // padded tokens, features, classes
  int64_t piece, pieces;          // classes of a piece (but the last), pieces
  bool f32, copy_h, copy_w;       // operands of the logits that are copied
  size_t scales, row_top, sums, sums_bytes, parts, at_target, rows, h[2], w[2], ht[2], wp[2], p[2], sum;
  size_t bytes;
};

bool direct(const void* p, int64_t stride, int64_t d) {
  return d % 64 == 0 && d >= 128 && stride % 8 == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
}

Plan plan_of(const daso_loss_args& s, bool backward) {
  Plan q = {};
  q.f32 = s.type == DASO_TYPE_F32;
  q.n_p = std::max<int64_t>(128, up(s.tokens, 64));
  q.d_p = std::max<int64_t>(128, up(s.d, 64));
  const int64_t most = std::max<int64_t>(256, kPieceElems / q.n_p / 256 * 256);
  q.pieces = (s.vocab + most - 1) / most;
  q.piece = up((s.vocab + q.pieces - 1) / q.pieces, 256);
  q.pieces = (s.vocab + q.piece - 1) / q.piece;
  const int64_t last = s.vocab - (q.pieces - 1) * q.piece;
  q.v_p = (q.pieces - 1) * q.piece + std::max<int64_t>(128, up(last, 64));
  q.copy_h = q.f32 || !direct(s.hidden, s.hidden_stride, s.d);
  q.copy_w = q.f32 || !direct(s.weight, s.weight_stride, s.d);
  size_t to = 0;
  const auto take = [&to](int64_t bytes) {
    const size_t from = to;
    to += (static_cast<size_t>(bytes) + 255) / 256 * 256;
    return from;
  };
  const int planes = q.f32 ? 2 : 1;
  q.scales = take(sizeof(Scales));
  q.row_top = take(q.f32 || backward ? 4 * s.tokens : 0);
  for (int i = 0; i < planes; ++i) {
    // with a copy or without: what a call needs is then known from its sizes alone
    q.h[i] = take(2 * q.n_p * q.d_p);
    q.w[i] = take(2 * q.v_p * q.d_p);
  }
  if (!backward) {
    q.parts = take(8 * s.tokens * ((s.vocab + 127) / 128));
    q.at_target = take(4 * s.tokens);
  } else {
    q.rows = take(sizeof(Row) * q.n_p);
    for (int i = 0; i < planes; ++i) {
      q.ht[i] = take(2 * q.n_p * q.d_p);
      q.wp[i] = q.f32 ? q.w[i] : take(2 * q.v_p * q.d_p);
    }
    const int64_t width = q.pieces > 1 ? q.piece : q.v_p;
    const int dz_planes = q.f32 || (s.dweight != nullptr && s.dweight_type == DASO_TYPE_F32) ? 2 : 1;
    for (int i = 0; i < dz_planes; ++i) q.p[i] = take(2 * q.n_p * width);
    q.sum = take(q.pieces > 1 ? 4 * q.n_p * q.d_p : 0);
  }
  // the largest product's steps, in tiles of 128 and three segments
  const int64_t nt = (q.n_p + 127) / 128, dt = (q.d_p + 127) / 128, width = std::min(q.v_p, q.piece), vt = (width + 127) / 128;
  q.sums_bytes = host::sums_bytes(3 * std::max(nt * (backward ? vt : (q.v_p + 127) / 128) * (q.d_p / 64),
                                               backward ? dt * (nt * (width / 64) + vt * (q.n_p / 64)) : 0));
  q.sums = take(static_cast<int64_t>(q.sums_bytes));
  q.bytes = to;
  return q;
}

// The operands of the logits, for the classes from `first`.
struct Operands {
  const char *h[2], *w[2];
  int64_t h_ld, w_ld;
};

void logits(product::Args& a, const Plan& q, const Operands& o, int64_t tokens, int64_t first, int64_t classes) {
  a.segments = q.f32 ? 3 : 1;
  const int64_t skip = first * o.w_ld * 2;
  a.a[0] = o.h[0], a.b[0] = o.w[0] + skip;
  a.a[1] = o.h[0], a.b[1] = q.f32 ? o.w[1] + skip : nullptr;
  a.a[2] = o.h[1], a.b[2] = o.w[0] + skip;
  a.lda = o.h_ld, a.ldb = o.w_ld;
  a.steps = static_cast<int32_t>(q.d_p / 64);
  a.M = static_cast<int32_t>(tokens), a.N = static_cast<int32_t>(classes), a.batch = 1;
}

void add_planes(PrepareArgs& a, int32_t by, const void* src, int64_t stride, int64_t rows, int64_t cols,
                int64_t rows_p, int64_t cols_p, char* d0, char* d1, char* t0, char* t1) {
  PlanesArgs& p = a.planes[a.count];
  p.src = src, p.stride = stride;
  p.rows = static_cast<int32_t>(rows), p.cols = static_cast<int32_t>(cols);
  p.rows_p = static_cast<int32_t>(rows_p), p.cols_p = static_cast<int32_t>(cols_p);
  p.d[0] = (uint16_t*)d0, p.d[1] = (uint16_t*)d1, p.t[0] = (uint16_t*)t0, p.t[1] = (uint16_t*)t1;
  a.by[a.count] = by;
  a.first[a.count + 1] = a.first[a.count] + (rows_p / 64) * (cols_p / 64);
  ++a.count;
}

// Scales, the planes of hidden and weight that the pass needs, and the backward pass's rows.
hipError_t prepare(const daso_loss_args& s, const Plan& q, bool backward, Operands* o, hipStream_t stream) {
  char* ws = static_cast<char*>(s.workspace);
  Scales* sc = reinterpret_cast<Scales*>(ws + q.scales);
  hipError_t e = hipSuccess;
  const bool scaled = q.f32 || backward;
  int32_t* row_top = reinterpret_cast<int32_t*>(ws + q.row_top);
  if (scaled) {
    const TopArgs t = {s.hidden, s.weight, s.hidden_stride, s.weight_stride, s.tokens, s.vocab, s.d, backward ? s.dloss : nullptr, s.targets, s.ignore_index, row_top, sc};
    e = s.type == DASO_TYPE_BF16 ? launch(&tops_kernel<uint16_t>, dim3(kTopParts, 2), dim3(256), stream, t)
                                 : launch(&tops_kernel<float>, dim3(kTopParts, 2), dim3(256), stream, t);
  }
  PrepareArgs a = {};
  const bool ht = backward && s.dweight != nullptr, wp = backward && s.dhidden != nullptr;
  const auto hidden = [&](int32_t by, char* d0, char* d1, char* t0, char* t1) {
    add_planes(a, by, s.hidden, s.hidden_stride, s.tokens, s.d, q.n_p, q.d_p, d0, d1, t0, t1);
  };
  const auto weight = [&](int32_t by, char* d0, char* d1) {
    add_planes(a, by, s.weight, s.weight_stride, s.vocab, s.d, q.v_p, q.d_p, d0, d1, nullptr, nullptr);
  };
  if (q.f32) {
    weight(kByWeight, ws + q.w[0], ws + q.w[1]);
    hidden(kByRow, ws + q.h[0], ws + q.h[1], nullptr, nullptr);
    if (ht) hidden(kByGrad, nullptr, nullptr, ws + q.ht[0], ws + q.ht[1]);
  } else {
    if (q.copy_w) weight(kRaw, ws + q.w[0], nullptr);
    if (q.copy_h) hidden(kRaw, ws + q.h[0], nullptr, nullptr, nullptr);
    if (wp) weight(kByWeight, ws + q.wp[0], nullptr);
    if (ht) hidden(kByGrad, nullptr, nullptr, ws + q.ht[0], nullptr);
  }
  a.first[a.count + 1] = a.first[a.count];
  if (backward) {
    a.first[a.count + 1] += (q.n_p + 255) / 256;
    a.rows = reinterpret_cast<Row*>(ws + q.rows);
    a.padded = q.n_p, a.tokens = s.tokens, a.vocab = s.vocab;
    a.lse = s.lse, a.dloss = s.dloss, a.targets = s.targets, a.ignore = s.ignore_index;
  }
  a.scales = scaled ? sc : nullptr;
  a.row_top = row_top;
  const int64_t groups = a.first[a.count + 1], row = int64_t(1) << 20;
  if (e == hipSuccess && groups > 0) {
    const dim3 grid(static_cast<uint32_t>(std::min(groups, row)), static_cast<uint32_t>((groups + row - 1) / row));
    e = s.type == DASO_TYPE_BF16 ? launch(&prepare_kernel<uint16_t>, grid, dim3(256), stream, a)
                                 : launch(&prepare_kernel<float>, grid, dim3(256), stream, a);
  }
  o->h[0] = q.copy_h ? ws + q.h[0] : (const char*)s.hidden;
  o->w[0] = q.copy_w ? ws + q.w[0] : (const char*)s.weight;
  o->h[1] = ws + q.h[1], o->w[1] = ws + q.w[1];
  o->h_ld = q.copy_h ? q.d_p : s.hidden_stride;
  o->w_ld = q.copy_w ? q.d_p : s.weight_stride;
  return e;
}

// F32: the operands are fp32, in two planes each, and scaled.
template <bool F32>
hipError_t forward(const daso_loss_args& s, const Plan& q, hipStream_t stream) {
  char* ws = static_cast<char*>(s.workspace);
  const product::Sums sums = {reinterpret_cast<float*>(ws + q.sums), q.sums_bytes};
  const Scales* sc = reinterpret_cast<const Scales*>(ws + q.scales);
  Operands o;
  hipError_t e = prepare(s, q, false, &o, stream);
  if (e != hipSuccess) return e;
  product::Launch<LseOut<F32>> all = {};
  all.count = 1;
  logits(all.args[0], q, o, s.tokens, 0, s.vocab);
  auto& out = all.out[0];
  out.parts = reinterpret_cast<float2*>(ws + q.parts);
  out.at_target = reinterpret_cast<float*>(ws + q.at_target);
  out.targets = s.targets;
  out.row_top = reinterpret_cast<const int32_t*>(ws + q.row_top), out.to_b = &sc->to[kWeight];
  const int64_t across = product::large_tiles(all) ? 256 : 128;
  e = product::launch_products<!F32, false>(all, sums, stream);
  if (e != hipSuccess) return e;
  return launch(&join_kernel, dim3(static_cast<uint32_t>((s.tokens + 15) / 16)), dim3(256), stream, (const float2*)out.parts,
                static_cast<int32_t>((s.vocab + across - 1) / across), s.tokens, s.vocab, s.targets, s.ignore_index,
                (const float*)out.at_target, s.loss, s.lse);
}

template <bool F32>
hipError_t backward(const daso_loss_args& s, const Plan& q, hipStream_t stream) {
  char* ws = static_cast<char*>(s.workspace);
  const product::Sums sums = {reinterpret_cast<float*>(ws + q.sums), q.sums_bytes};
  const Scales* sc = reinterpret_cast<const Scales*>(ws + q.scales);
  Operands o;
  hipError_t e = prepare(s, q, true, &o, stream);
  if (e != hipSuccess) return e;
  Row* rows = reinterpret_cast<Row*>(ws + q.rows);
  const bool dh = s.dhidden != nullptr, dw = s.dweight != nullptr, dw32 = s.dweight_type == DASO_TYPE_F32;
  const auto at = [ws](size_t off) { return reinterpret_cast<_Float16*>(ws + off); };
  for (int64_t k = 0; k < q.pieces && e == hipSuccess; ++k) {
    const int64_t first = k * q.piece, classes = std::min(q.piece, s.vocab - first);
    const int64_t width = std::max<int64_t>(128, up(classes, 64));
    product::Launch<ProbOut<F32>> prob = {};
    prob.count = 1;
    logits(prob.args[0], q, o, s.tokens, first, classes);
    auto& out = prob.out[0];
    out.rows = rows;
    // dz in two planes where a product in 22 bits reads it
    out.hi = at(q.p[0]), out.lo = q.p[1] != 0 ? at(q.p[1]) : nullptr;
    out.ld = width;
    out.first = static_cast<int32_t>(first), out.columns = static_cast<int32_t>(classes), out.padded = static_cast<int32_t>(width);
    out.padded_rows = static_cast<int32_t>(q.n_p);
    out.to_b = &sc->to[kWeight];
    e = product::launch_products<!F32, false>(prob, sums, stream);
    if (e != hipSuccess) break;
    // dhidden = dz weight and dweight^T = hidden^T dz, both with the right operand read turned
    product::Launch<GradOut> grads = {};
    if (dh) {
      product::Args& a = grads.args[grads.count];
      const _Float16 *w0 = at(q.wp[0]) + first * q.d_p, *w1 = at(q.wp[1]) + first * q.d_p;
      a.segments = F32 ? 3 : 1;
      a.a[0] = at(q.p[0]), a.b[0] = w0;
      a.a[1] = at(q.p[0]), a.b[1] = w1;
      a.a[2] = at(q.p[1]), a.b[2] = w0;
      a.lda = width, a.ldb = q.d_p, a.steps = static_cast<int32_t>(width / 64);
      a.M = static_cast<int32_t>(s.tokens), a.N = static_cast<int32_t>(q.d_p), a.batch = 1;
      GradOut::Params& g = grads.out[grads.count++];
      g.tokens = rows, g.to = &sc->to[kWeight];
      float* sum = reinterpret_cast<float*>(ws + q.sum);
      if (k > 0) g.before = sum, g.before_ld = q.d_p;
      g.rows = a.M;
      if (k + 1 < q.pieces) g.out = sum, g.ld = q.d_p, g.bf16 = 0, g.cols = static_cast<int32_t>(q.d_p);
      else g.out = s.dhidden, g.ld = s.dhidden_stride, g.bf16 = s.type == DASO_TYPE_BF16, g.cols = static_cast<int32_t>(s.d);
    }
    if (dw) {
      product::Args& a = grads.args[grads.count];
      // dz in one plane or two; hidden in one (exact) where it is bf16
      a.segments = F32 ? 3 : dw32 ? 2 : 1;
      a.a[0] = at(q.ht[0]), a.b[0] = at(q.p[0]);
      a.a[1] = at(q.ht[0]), a.b[1] = at(q.p[1]);
      a.a[2] = at(q.ht[1]), a.b[2] = at(q.p[0]);
      a.lda = q.n_p, a.ldb = width, a.steps = static_cast<int32_t>(q.n_p / 64);
      a.M = static_cast<int32_t>(s.d), a.N = static_cast<int32_t>(width), a.batch = 1;
      GradOut::Params& g = grads.out[grads.count++];
      g.to = &sc->to[kHidden];
      g.out = static_cast<char*>(s.dweight) + first * s.dweight_stride * static_cast<int64_t>(host::bytes_of(s.dweight_type));
      g.ld = s.dweight_stride, g.bf16 = !dw32;
      g.rows = static_cast<int32_t>(classes), g.cols = a.M, g.turned = 1;
    }
    e = product::launch_products<false, true>(grads, sums, stream);
  }
  return e;
}

}  // namespace
}  // namespace daso

extern "C" {

int daso_linear_cross_entropy_workspace(const daso_loss_args* args, int backward, size_t* bytes) {
  if (args == nullptr || bytes == nullptr) return DASO_EINVAL;
  const int rc = daso::host::check_loss_sizes(*args);
  if (rc != DASO_OK) return rc;
  *bytes = args->tokens == 0 ? 0 : daso::plan_of(*args, backward != 0).bytes;
  return DASO_OK;
}

int daso_linear_cross_entropy(const daso_loss_args* args, hipStream_t stream) {
  if (args == nullptr) return DASO_EINVAL;
  int rc = daso::host::check_loss(*args, false);
  if (rc != DASO_OK || args->tokens == 0) return rc;
  const daso::Plan q = daso::plan_of(*args, false);
  if ((rc = daso::host::check_workspace(args->workspace, args->workspace_bytes, q.bytes)) != DASO_OK) return rc;
  if ((rc = daso::current_device(stream)) != DASO_OK) return rc;
  const hipError_t e = q.f32 ? daso::forward<true>(*args, q, stream) : daso::forward<false>(*args, q, stream);
  return e == hipSuccess ? DASO_OK : DASO_EHIP;
}

int daso_linear_cross_entropy_backward(const daso_loss_args* args, hipStream_t stream) {
  if (args == nullptr) return DASO_EINVAL;
  const daso_loss_args& s = *args;
  int rc = daso::host::check_loss(s, true);
  if (rc != DASO_OK) return rc;
  if (s.dweight == nullptr && (s.dhidden == nullptr || s.tokens == 0)) return DASO_OK;
  const daso::Plan q = daso::plan_of(s, true);
  if (s.tokens > 0 && (rc = daso::host::check_workspace(s.workspace, s.workspace_bytes, q.bytes)) != DASO_OK) return rc;
  if ((rc = daso::current_device(stream)) != DASO_OK) return rc;
  hipError_t e;
  if (s.tokens == 0) {
    const dim3 grid(1024), block(256);
    e = s.dweight_type == DASO_TYPE_F32
            ? daso::launch(&daso::zero_rows_kernel<float>, grid, block, stream, (float*)s.dweight, s.dweight_stride, s.vocab, s.d)
            : daso::launch(&daso::zero_rows_kernel<uint16_t>, grid, block, stream, (uint16_t*)s.dweight, s.dweight_stride, s.vocab, s.d);
  } else {
    e = q.f32 ? daso::backward<true>(s, q, stream) : daso::backward<false>(s, q, stream);
  }
  return e == hipSuccess ? DASO_OK : DASO_EHIP;
}

}  // extern "C"
