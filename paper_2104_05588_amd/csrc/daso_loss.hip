// The cross entropy of an output projection and its gradients (daso_train.h), over pieces of
// the vocabulary, without keeping the logits.
//
// Forward: one product hidden weight^T, whose epilogue reduces each 256 (or 128) columns of a
// row to their maximum and their sum of exponentials; a second kernel joins them.
// Backward, per piece of the vocabulary: the piece's logits again, whose epilogue turns them
// into s (p - onehot), stored straight and transposed as 16-bit planes; then dhidden += dz weight
// and dweight = dz^T hidden, in one launch.  6 N V d multiply-adds at least, 8 with the logits taken
// twice: keeping them would cost N V 4 bytes written and read, which takes as long as the
// product at d = 1024 and grows the memory by N V.
//
// Numbers.  bf16 operands are multiplied as they are in the forward product; fp32 ones as two
// binary16 planes each, scaled by a power of two from the tensor's largest value (22
// bits).  In the backward products dz is binary16, of values in [-1, 1] times 2^14, which keeps 3 bits
// more than bf16 would, and hidden and weight are turned to binary16 by the same scaling
// (exact for a bf16 value within 2^-32 of the largest), so that a bf16 result is off by 2e-4 before it is
// rounded; fp32 results take dz as two planes.
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

constexpr float kProbScale = 16384.0f;  // dz / dloss in [-1, 1] as binary16

// Powers of two and their reciprocals, worked out on the device.
struct Scales {
  uint32_t top[3];  // bits of the largest finite magnitude: hidden, weight, dloss
  uint32_t pad;
  float hidden, hidden_inv;  // hidden * scale <= 2^15
  float weight, weight_inv;
  float grad, grad_inv;  // |dloss| * grad_inv <= 1
};

// What the backward epilogue needs of a token.
struct Row {
  float lse;
  float g;         // dloss * grad_inv * kProbScale
  int32_t target;  // -1: the whole row is zero
  int32_t pad;
};

__device__ inline float power_of_two(int e) { return __builtin_bit_cast(float, uint32_t(min(max(e, -126), 127) + 127) << 23); }

__global__ void clear_kernel(Scales* s) {
  if (threadIdx.x < 3) s->top[threadIdx.x] = 0;
}

// The largest finite magnitude of a matrix.
template <class T>
__global__ __launch_bounds__(256) void top_kernel(const T* src, int64_t stride, int64_t rows, int64_t cols, uint32_t* top) {
  const int64_t wave = (blockIdx.x * 256 + threadIdx.x) >> 6, waves = gridDim.x * 4;
  const int lane = threadIdx.x & 63;
  const bool wide = ((reinterpret_cast<uintptr_t>(src) | (stride * sizeof(T))) & 15) == 0;
  const int64_t whole = wide ? cols / 8 * 8 : 0;
  float m = 0.0f;
  auto take = [&](float v) {
    v = __builtin_fabsf(v);
    if (v < __builtin_inff()) m = fmaxf(m, v);
  };
  for (int64_t r = wave; r < rows; r += waves) {
    const T* p = src + r * stride;
    for (int64_t c = lane * 8; c < whole; c += 512) {
      float v[8];
      load8(p + c, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) take(v[i]);
    }
    for (int64_t c = whole + lane; c < cols; c += 64) take(load1(p + c));
  }
  m = wave_max(m);
  if (lane == 0 && m > 0.0f) atomicMax(top, __builtin_bit_cast(uint32_t, m));
}

__global__ void scales_kernel(Scales* s) {
  if (threadIdx.x != 0) return;
  const auto exponent = [](uint32_t bits) { return bits == 0 ? 0 : static_cast<int>(max(bits >> 23, 1u)) - 127; };
  const int h = min(max(14 - exponent(s->top[0]), -126), 126), w = min(max(14 - exponent(s->top[1]), -126), 126);
  s->hidden = power_of_two(h), s->hidden_inv = power_of_two(-h);
  s->weight = power_of_two(w), s->weight_inv = power_of_two(-w);
  const int g = min(max(exponent(s->top[2]) + 1, -126), 126);
  s->grad = power_of_two(g), s->grad_inv = power_of_two(-g);
}

__global__ __launch_bounds__(256) void rows_kernel(Row* out, int64_t padded, int64_t tokens, int64_t vocab, const float* lse,
                                                   const float* dloss, const int64_t* targets, int64_t ignore,
                                                   const Scales* s) {
  const int64_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= padded) return;
  Row r = {0.0f, 0.0f, -1, 0};
  if (i < tokens) {
    const int64_t t = targets[i];
    if (t >= 0 && t < vocab && t != ignore) {
      r.lse = lse[i];
      r.g = dloss[i] * s->grad_inv * kProbScale;
      r.target = static_cast<int32_t>(t);
    } else if (t != ignore) {
      r.g = __builtin_nanf("");
      r.target = 0;
    }
  }
  out[i] = r;
}

template <class T, bool RAW>
__global__ __launch_bounds__(256) void planes_kernel(PlanesArgs p, const float* scale) {
  __shared__ uint16_t lds[2][64][66];
  const int64_t id = blockIdx.x + int64_t(blockIdx.y) * gridDim.x, across = p.cols_p / 64;
  if (id >= across * (p.rows_p / 64)) return;
  planes_tile<T, RAW>(p, 0, static_cast<int>(id / across), static_cast<int>(id % across), RAW ? 1.0f : *scale, lds);
}

// ------------------------------------------------------------------------- forward epilogue
// For each row the maximum and the sum of exponentials of the tile's columns, and the logit of
// the target where the tile has it.
struct LseOut {
  struct Params {
    float2* parts;  // [tile column][token]
    float* at_target;
    const int64_t* targets;
    const float *inv_a, *inv_b;  // null, or what takes the operands' scaling back
  };
  template <class Tile>
  __device__ static void tile(const Params& out, const product::Args& p, const product::Place& at, f4 (&acc)[Tile::kBlocks][8],
                              char* lds) {
    constexpr int kAcross = Tile::kThreads / 128;  // wavefronts side by side, of two rows of them
    constexpr int kBands = Tile::kBlocks / 2;      // runs of 64 rows a wavefront holds
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, kq = lane >> 4, wn = wave % kAcross;
    float2* shared = (float2*)lds;  // [row][kAcross]
    const float inv = out.inv_a != nullptr ? *out.inv_a * *out.inv_b : 1.0f;
#pragma unroll
    for (int band = 0; band < kBands; ++band)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        int row0, col0, col1;
        Tile::block_at(wave, band * 2, &row0, &col0);
        Tile::block_at(wave, band * 2 + 1, &row0, &col1);
        const int in = row0 + i * 16 + r16, row = at.tm * Tile::kRows + in;
        const int64_t t = row < p.M ? out.targets[row] : -1;
        float z[16], m = -__builtin_inff();
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int col = at.tn * Tile::kCols + (b ? col1 : col0) + j * 16 + kq * 4 + e;
              float v = acc[band * 2 + b][i * 2 + j][e] * inv;
              if (row < p.M && t == col && col < p.N) out.at_target[row] = v;
              v = col < p.N ? v : -__builtin_inff();
              z[(b * 2 + j) * 4 + e] = v;
              m = fmaxf(m, v);
            }
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        // columns that are all -inf, or none, add nothing; +inf or NaN make the sum NaN
        const float base = m == -__builtin_inff() ? 0.0f : m;
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) s += __expf(z[e] - base);
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if (kq == 0) shared[in * kAcross + wn] = make_float2(m, s);
      }
    __syncthreads();
    for (int in = threadIdx.x; in < Tile::kRows; in += Tile::kThreads) {
      const int row = at.tm * Tile::kRows + in;
      if (row >= p.M) continue;
      float m = -__builtin_inff(), s = 0.0f;
#pragma unroll
      for (int w = 0; w < kAcross; ++w) m = fmaxf(m, shared[in * kAcross + w].x);
      const float base = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
      for (int w = 0; w < kAcross; ++w) s += shared[in * kAcross + w].y * __expf(shared[in * kAcross + w].x - base);
      out.parts[int64_t(at.tn) * p.M + row] = make_float2(m, s);
    }
  }
};

// Joins a token's parts: 32 tokens a workgroup, eight shares of the parts each.
__global__ __launch_bounds__(256) void join_kernel(const float2* parts, int32_t count, int64_t tokens, int64_t vocab,
                                                   const int64_t* targets, int64_t ignore, const float* at_target, float* loss,
                                                   float* lse) {
  __shared__ float2 shared[8][32];
  const int in = threadIdx.x & 31, share = threadIdx.x >> 5;
  const int64_t i = blockIdx.x * 32 + in;
  float m = -__builtin_inff(), s = 0.0f;
  bool bad = false;
  if (i < tokens)
    for (int32_t k = share; k < count; k += 8) {
      const float2 v = parts[k * tokens + i];
      bad = bad || v.y != v.y;
      if (v.x > m) s = s * __expf(m - v.x), m = v.x;
      if (v.x > -__builtin_inff()) s += v.y * __expf(v.x - m);
    }
  shared[share][in] = make_float2(m, bad ? __builtin_nanf("") : s);
  __syncthreads();
  if (share != 0 || i >= tokens) return;
  m = shared[0][in].x;
  for (int k = 1; k < 8; ++k) m = fmaxf(m, shared[k][in].x);
  s = 0.0f;
  for (int k = 0; k < 8; ++k) {
    const float2 v = shared[k][in];
    s += v.x > -__builtin_inff() ? v.y * __expf(v.x - m) : v.y;
  }
  const float l = m + logf(s);
  lse[i] = l;
  const int64_t t = targets[i];
  loss[i] = t == ignore ? 0.0f : t >= 0 && t < vocab ? l - at_target[i] : __builtin_nanf("");
}

// ------------------------------------------------------------------------- backward epilogues
// dz of a piece's columns as planes, straight and transposed; columns beyond the vocabulary are zero.
struct ProbOut {
  struct Params {
    const Row* rows;
    _Float16 *hi, *lo, *t_hi, *t_lo;  // any may be null but hi's or t_hi's
    int64_t ld, t_ld;
    int32_t first, columns, padded;  // the piece: its first class, its classes, its columns with padding
    int32_t padded_rows;             // tokens with padding: the planes are contracted over both
    const float *inv_a, *inv_b;
  };
  template <class Tile>
  __device__ static void tile(const Params& out, const product::Args&, const product::Place& at, f4 (&acc)[Tile::kBlocks][8],
                              char* lds) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, kq = lane >> 4;
    char* hi = lds + wave * product::kWaveStage;
    char* lo = hi + product::kStagePlane;
    const float inv = out.inv_a != nullptr ? *out.inv_a * *out.inv_b : 1.0f;
    const bool two = out.lo != nullptr || out.t_lo != nullptr;
#pragma unroll
    for (int b = 0; b < Tile::kBlocks; ++b) {
      int row0, col0;
      Tile::block_at(wave, b, &row0, &col0);
      row0 += at.tm * Tile::kRows, col0 += at.tn * Tile::kCols;
      if (row0 >= out.padded_rows || col0 >= out.padded) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const Row r = out.rows[row0 + i * 16 + r16];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int col = col0 + j * 16 + kq * 4;
          half4 h, l;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float v = __expf(acc[b][i * 2 + j][e] * inv - r.lse) - (out.first + col + e == r.target ? 1.0f : 0.0f);
            v = r.target >= 0 && col + e < out.columns ? v * r.g : 0.0f;
            _Float16 a, c;
            product::split(v, &a, &c);
            h[e] = a, l[e] = c;
          }
          *(half4*)(hi + product::plane_at(i * 16 + r16, j * 16 + kq * 4)) = h;
          if (two) *(half4*)(lo + product::plane_at(i * 16 + r16, j * 16 + kq * 4)) = l;
        }
      }
      product::wait_lds();
      __builtin_amdgcn_wave_barrier();
      const auto straight = [&](const char* plane, _Float16* to) {
#pragma unroll
        for (int pass = 0; pass < 4; ++pass) {
          const int r = pass * 16 + (lane >> 2), c = (lane & 3) * 8;
          *(half8*)(to + int64_t(row0 + r) * out.ld + col0 + c) = *(const half8*)(plane + product::plane_at(r, c));
        }
      };
      const auto turned = [&](const char* plane, _Float16* to) {
        product::by_columns(plane, lane, [&](int c, int r, half8 v) {
          *(half8*)(to + int64_t(col0 + c) * out.t_ld + row0 + r) = v;
        });
      };
      if (out.hi != nullptr) straight(hi, out.hi);
      if (out.lo != nullptr) straight(lo, out.lo);
      if (out.t_hi != nullptr) turned(hi, out.t_hi);
      if (out.t_lo != nullptr) turned(lo, out.t_lo);
    }
  }
};

// A gradient: (C * grad * inv / kProbScale) [+ sum], as the sum so far or as the result.
struct GradOut {
  struct Params {
    const float *grad, *inv;
    const float* before;  // the sum of the pieces so far, or null
    int64_t before_ld;
    void* out;
    int64_t ld;
    int32_t bf16;
    int32_t rows, cols;
  };
  template <class Tile>
  __device__ static void tile(const Params& p, const product::Args& args, const product::Place& at, f4 (&acc)[Tile::kBlocks][8],
                              char* lds) {
    product::by_blocks<Tile, GradOut>(p, args, at, acc, lds);
  }
  __device__ static void block(const Params& p, const product::Place&, const f4 (&c)[8], int row, int col, char* stage, int lane) {
    const float factor = *p.grad * (1.0f / kProbScale), inv = *p.inv;
    const bool wide = ((reinterpret_cast<uintptr_t>(p.out) | (p.ld * (p.bf16 ? 2 : 4))) & 15) == 0;
    product::by_rows(c, stage, lane, [&](int r, int k, float(&v)[8]) {
      const int32_t rr = row + r, cc = col + k, left = p.cols - cc;
      if (rr >= p.rows || left <= 0) return;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = v[i] * inv * factor;
      if (p.before != nullptr) {
        float b[8];
        load8(p.before + int64_t(rr) * p.before_ld + cc, b);  // padded to whole vectors
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += b[i];
      }
      const int64_t to = int64_t(rr) * p.ld + cc;
      if (p.bf16) {
        uint16_t* o = (uint16_t*)p.out + to;
        if (wide && left >= 8) store8(o, v);
        else
          for (int i = 0; i < 8 && i < left; ++i) o[i] = to_bf16(v[i]);
      } else {
        float* o = (float*)p.out + to;
        if (wide && left >= 8) store8(o, v);
        else
          for (int i = 0; i < 8 && i < left; ++i) o[i] = v[i];
      }
    });
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
// holds 2^26 values (128 MB): enough tiles for every CU, and small enough that the
// planes are read back from the 256 MB cache in front of HBM.
constexpr int64_t kPieceElems = int64_t(1) << 26;

struct Plan {
  int64_t n_p, d_p, v_p;          // padded tokens, features, classes
  int64_t piece, pieces;          // classes of a piece (but the last), pieces
  bool f32, copy_h, copy_w;       // operands of the logits that are copied
  size_t scales, parts, at_target, rows, h[2], w[2], ht[2], wt[2], p[2], pt[2], sum;
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
      q.wt[i] = take(2 * q.v_p * q.d_p);
    }
    const int64_t width = q.pieces > 1 ? q.piece : q.v_p;
    for (int i = 0; i < 2; ++i) q.p[i] = take(2 * q.n_p * width), q.pt[i] = take(2 * q.n_p * width);
    q.sum = take(q.pieces > 1 ? 4 * q.n_p * q.d_p : 0);
  }
  q.bytes = to;
  return q;
}

hipError_t lay_out(const void* src, int32_t type, int64_t stride, int64_t rows, int64_t cols, int64_t rows_p, int64_t cols_p,
                   bool raw, const float* scale, char* d0, char* d1, char* t0, char* t1, hipStream_t stream) {
  PlanesArgs p = {};
  p.src = src, p.stride = stride;
  p.rows = static_cast<int32_t>(rows), p.cols = static_cast<int32_t>(cols);
  p.rows_p = static_cast<int32_t>(rows_p), p.cols_p = static_cast<int32_t>(cols_p);
  p.d[0] = (uint16_t*)d0, p.d[1] = (uint16_t*)d1, p.t[0] = (uint16_t*)t0, p.t[1] = (uint16_t*)t1;
  const int64_t tiles = (rows_p / 64) * (cols_p / 64), row = int64_t(1) << 20;
  const dim3 grid(static_cast<uint32_t>(std::min(tiles, row)), static_cast<uint32_t>((tiles + row - 1) / row));
  if (raw) return launch(&planes_kernel<uint16_t, true>, grid, dim3(256), stream, p, scale);
  if (type == DASO_TYPE_BF16) return launch(&planes_kernel<uint16_t, false>, grid, dim3(256), stream, p, scale);
  return launch(&planes_kernel<float, false>, grid, dim3(256), stream, p, scale);
}

hipError_t top_of(const void* src, int32_t type, int64_t stride, int64_t rows, int64_t cols, uint32_t* top, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(std::min<int64_t>((rows + 3) / 4, 2048)));
  if (type == DASO_TYPE_BF16)
    return launch(&top_kernel<uint16_t>, grid, dim3(256), stream, (const uint16_t*)src, stride, rows, cols, top);
  return launch(&top_kernel<float>, grid, dim3(256), stream, (const float*)src, stride, rows, cols, top);
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

// Scales, and the planes of hidden and weight that the pass needs.
hipError_t operands_of(const daso_loss_args& s, const Plan& q, bool backward, Operands* o, hipStream_t stream) {
  char* ws = static_cast<char*>(s.workspace);
  Scales* sc = reinterpret_cast<Scales*>(ws + q.scales);
  hipError_t e = hipSuccess;
  if (q.f32 || backward) {
    e = launch(&clear_kernel, dim3(1), dim3(64), stream, sc);
    if (e == hipSuccess) e = top_of(s.hidden, s.type, s.hidden_stride, s.tokens, s.d, &sc->top[0], stream);
    if (e == hipSuccess) e = top_of(s.weight, s.type, s.weight_stride, s.vocab, s.d, &sc->top[1], stream);
    // in rows of 512, so that long ones are taken by many wavefronts
    const int64_t rows = s.tokens / 512, rest = s.tokens - rows * 512;
    if (e == hipSuccess && backward && rows > 0) e = top_of(s.dloss, DASO_TYPE_F32, 512, rows, 512, &sc->top[2], stream);
    if (e == hipSuccess && backward && rest > 0) e = top_of(s.dloss + rows * 512, DASO_TYPE_F32, rest, 1, rest, &sc->top[2], stream);
    if (e == hipSuccess) e = launch(&scales_kernel, dim3(1), dim3(64), stream, sc);
  }
  const bool need_ht = backward && s.dweight != nullptr, need_wt = backward && s.dhidden != nullptr;
  char *h[2] = {ws + q.h[0], ws + q.h[1]}, *w[2] = {ws + q.w[0], ws + q.w[1]};
  if (q.f32) {
    char *ht0 = need_ht ? ws + q.ht[0] : nullptr, *ht1 = need_ht ? ws + q.ht[1] : nullptr;
    char *wt0 = need_wt ? ws + q.wt[0] : nullptr, *wt1 = need_wt ? ws + q.wt[1] : nullptr;
    if (e == hipSuccess)
      e = lay_out(s.hidden, s.type, s.hidden_stride, s.tokens, s.d, q.n_p, q.d_p, false, &sc->hidden, h[0], h[1], ht0, ht1, stream);
    if (e == hipSuccess)
      e = lay_out(s.weight, s.type, s.weight_stride, s.vocab, s.d, q.v_p, q.d_p, false, &sc->weight, w[0], w[1], wt0, wt1, stream);
  } else {
    if (e == hipSuccess && q.copy_h)
      e = lay_out(s.hidden, s.type, s.hidden_stride, s.tokens, s.d, q.n_p, q.d_p, true, nullptr, h[0], nullptr, nullptr, nullptr, stream);
    if (e == hipSuccess && q.copy_w)
      e = lay_out(s.weight, s.type, s.weight_stride, s.vocab, s.d, q.v_p, q.d_p, true, nullptr, w[0], nullptr, nullptr, nullptr, stream);
    if (e == hipSuccess && need_ht)
      e = lay_out(s.hidden, s.type, s.hidden_stride, s.tokens, s.d, q.n_p, q.d_p, false, &sc->hidden, nullptr, nullptr, ws + q.ht[0], nullptr, stream);
    if (e == hipSuccess && need_wt)
      e = lay_out(s.weight, s.type, s.weight_stride, s.vocab, s.d, q.v_p, q.d_p, false, &sc->weight, nullptr, nullptr, ws + q.wt[0], nullptr, stream);
  }
  o->h[0] = q.copy_h ? h[0] : (const char*)s.hidden;
  o->w[0] = q.copy_w ? w[0] : (const char*)s.weight;
  o->h[1] = h[1], o->w[1] = w[1];
  o->h_ld = q.copy_h ? q.d_p : s.hidden_stride;
  o->w_ld = q.copy_w ? q.d_p : s.weight_stride;
  return e;
}

hipError_t forward(const daso_loss_args& s, const Plan& q, hipStream_t stream) {
  char* ws = static_cast<char*>(s.workspace);
  const Scales* sc = reinterpret_cast<const Scales*>(ws + q.scales);
  Operands o;
  hipError_t e = operands_of(s, q, false, &o, stream);
  if (e != hipSuccess) return e;
  product::Launch<LseOut> all = {};
  all.count = 1;
  logits(all.args[0], q, o, s.tokens, 0, s.vocab);
  LseOut::Params& out = all.out[0];
  out.parts = reinterpret_cast<float2*>(ws + q.parts);
  out.at_target = reinterpret_cast<float*>(ws + q.at_target);
  out.targets = s.targets;
  out.inv_a = q.f32 ? &sc->hidden_inv : nullptr, out.inv_b = q.f32 ? &sc->weight_inv : nullptr;
  const bool large = product::large_tiles(all);
  const int64_t across = large ? product::Tile256::kCols : product::Tile128::kCols;
  if (q.f32) e = product::launch_products<false>(all, stream);
  else e = product::launch_products<true>(all, stream);
  if (e != hipSuccess) return e;
  return launch(&join_kernel, dim3(static_cast<uint32_t>((s.tokens + 31) / 32)), dim3(256), stream, (const float2*)out.parts,
                static_cast<int32_t>((s.vocab + across - 1) / across), s.tokens, s.vocab, s.targets, s.ignore_index,
                (const float*)out.at_target, s.loss, s.lse);
}

hipError_t backward(const daso_loss_args& s, const Plan& q, hipStream_t stream) {
  char* ws = static_cast<char*>(s.workspace);
  const Scales* sc = reinterpret_cast<const Scales*>(ws + q.scales);
  Operands o;
  hipError_t e = operands_of(s, q, true, &o, stream);
  if (e != hipSuccess) return e;
  Row* rows = reinterpret_cast<Row*>(ws + q.rows);
  e = launch(&rows_kernel, dim3(static_cast<uint32_t>((q.n_p + 255) / 256)), dim3(256), stream, rows, q.n_p, s.tokens, s.vocab,
             (const float*)s.lse, s.dloss, s.targets, s.ignore_index, sc);
  const bool dh = s.dhidden != nullptr, dw = s.dweight != nullptr, dw32 = s.dweight_type == DASO_TYPE_F32;
  const auto at = [ws](size_t off) { return reinterpret_cast<_Float16*>(ws + off); };
  for (int64_t k = 0; k < q.pieces && e == hipSuccess; ++k) {
    const int64_t first = k * q.piece, classes = std::min(q.piece, s.vocab - first);
    const int64_t width = std::max<int64_t>(128, up(classes, 64));
    product::Launch<ProbOut> prob = {};
    prob.count = 1;
    logits(prob.args[0], q, o, s.tokens, first, classes);
    ProbOut::Params& out = prob.out[0];
    out.rows = rows;
    out.hi = dh ? at(q.p[0]) : nullptr, out.lo = dh && q.f32 ? at(q.p[1]) : nullptr;
    out.t_hi = dw ? at(q.pt[0]) : nullptr, out.t_lo = dw && (q.f32 || dw32) ? at(q.pt[1]) : nullptr;
    out.ld = width, out.t_ld = q.n_p;
    out.first = static_cast<int32_t>(first), out.columns = static_cast<int32_t>(classes), out.padded = static_cast<int32_t>(width);
    out.padded_rows = static_cast<int32_t>(q.n_p);
    out.inv_a = q.f32 ? &sc->hidden_inv : nullptr, out.inv_b = q.f32 ? &sc->weight_inv : nullptr;
    e = q.f32 ? product::launch_products<false>(prob, stream) : product::launch_products<true>(prob, stream);
    if (e != hipSuccess) break;
    product::Launch<GradOut> grads = {};
    if (dh) {
      product::Args& a = grads.args[grads.count];
      const _Float16* w0 = at(q.wt[0]) + first;
      const _Float16* w1 = at(q.wt[1]) + first;
      a.segments = q.f32 ? 3 : 1;
      a.a[0] = at(q.p[0]), a.b[0] = w0;
      a.a[1] = at(q.p[0]), a.b[1] = w1;
      a.a[2] = at(q.p[1]), a.b[2] = w0;
      a.lda = width, a.ldb = q.v_p, a.steps = static_cast<int32_t>(width / 64);
      a.M = static_cast<int32_t>(s.tokens), a.N = static_cast<int32_t>(s.d), a.batch = 1;
      GradOut::Params& g = grads.out[grads.count++];
      g.grad = &sc->grad, g.inv = &sc->weight_inv;
      float* sum = reinterpret_cast<float*>(ws + q.sum);
      if (k > 0) g.before = sum, g.before_ld = q.d_p;
      g.rows = a.M, g.cols = a.N;
      if (k + 1 < q.pieces) g.out = sum, g.ld = q.d_p, g.bf16 = 0, g.cols = static_cast<int32_t>(q.d_p);
      else g.out = s.dhidden, g.ld = s.dhidden_stride, g.bf16 = s.type == DASO_TYPE_BF16;
    }
    if (dw) {
      product::Args& a = grads.args[grads.count];
      // dz in one plane or two; hidden in one (exact) where it is bf16
      a.segments = q.f32 ? 3 : dw32 ? 2 : 1;
      a.a[0] = at(q.pt[0]), a.b[0] = at(q.ht[0]);
      a.a[1] = at(q.pt[1]), a.b[1] = at(q.ht[0]);
      a.a[2] = at(q.pt[0]), a.b[2] = at(q.ht[1]);
      a.lda = a.ldb = q.n_p, a.steps = static_cast<int32_t>(q.n_p / 64);
      a.M = static_cast<int32_t>(classes), a.N = static_cast<int32_t>(s.d), a.batch = 1;
      GradOut::Params& g = grads.out[grads.count++];
      g.grad = &sc->grad, g.inv = &sc->hidden_inv;
      g.out = static_cast<char*>(s.dweight) + first * s.dweight_stride * static_cast<int64_t>(host::bytes_of(s.dweight_type));
      g.ld = s.dweight_stride, g.bf16 = !dw32;
      g.rows = a.M, g.cols = a.N;
    }
    e = product::launch_products<false>(grads, stream);
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
  return daso::forward(*args, q, stream) == hipSuccess ? DASO_OK : DASO_EHIP;
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
    e = daso::backward(s, q, stream);
  }
  return e == hipSuccess ? DASO_OK : DASO_EHIP;
}

}  // extern "C"
