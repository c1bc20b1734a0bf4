// The norm of each head's row of queries and keys and its rotation, forward and backward (daso_block.h).  Bound
// by memory: a row is read once, into the registers of neighbouring lanes, and written once.
//
// A lane holds eight pairs of a head, as many lanes as that takes (2, 4 or 8) a head, and the other lanes of
// the wavefront further heads of the same token.  The angles are the token's: one lane takes a pair's, in 64 bits,
// for all heads of a wavefront, and hands it over through LDS.  What the rotation turns lies in one lane, whichever
// elements make a pair.  The sums of squares cross the head's lanes.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "daso_block_host.h"
#include "daso_partials.h"
#include "daso_planes.h"

namespace daso {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kForwardGroups = 2048;  // most workgroups of a forward pass
constexpr int kPartialGroups = 1024;  // of a backward one: four a CU
constexpr int kShareTokens = 4096;    // with fewer tokens several wavefronts take a token's heads

struct Rows {
  void* p;
  int64_t token, head;  // strides in elements
};

struct Rotary {
  int64_t tokens;
  int32_t heads, all;  // query heads; with key heads
  int32_t dim, half, turned;  // elements; pairs; pairs that are turned
  int32_t shares;  // wavefronts that take a token's heads together
  float eps, inv;  // 1 / dim
  const int64_t* positions;
  const double* frequencies;
  const float* weight[2];
  Rows x[2], to[2], dy[2];
  float* partial;  // backward: [workgroup][q, k][dim], or null
};

enum Order { kHalves, kFours, kNeighbours };  // where a lane's pairs lie: runs of eight, of four, or side by side

// Where a lane's pairs lie in a row, and whether they are there: eight pairs from `pair` on as two runs of eight elements
// (kHalves, kNeighbours) or four runs of four (kFours).
template <Order ORDER>
struct Place {
  int at[4];
  bool is[4];
  __device__ Place(const Rotary& a, int pair) {
    if constexpr (ORDER == kNeighbours) {
#pragma unroll
      for (int r = 0; r < 4; ++r) at[r] = 2 * pair + (r & 1) * 8, is[r] = at[r] < a.dim;
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int p = ORDER == kHalves ? pair : pair + (r & 1) * 4;
        is[r] = p < a.half;
        // beyond the turned pairs any two elements will do
        if (r < (ORDER == kHalves ? 1 : 2)) at[r] = p < a.turned ? p : p + a.turned;
        else at[r] = p < a.turned ? p + a.turned : p + a.half;
      }
      if constexpr (ORDER == kHalves) at[1] = at[2], is[1] = is[2];
    }
  }
};

// A lane's part of a row as it lies in memory.
template <class T, Order ORDER>
struct Raw {
  typedef uint32_t word __attribute__((ext_vector_type(4)));
  typedef uint32_t pair_word __attribute__((ext_vector_type(2)));
  typedef word word_any __attribute__((aligned(2)));
  typedef pair_word pair_word_any __attribute__((aligned(2)));
  static constexpr int kWords = 16 * sizeof(T) / 4;
  uint32_t w[kWords];

  __device__ void load(const T* row, const Place<ORDER>& at, bool there) {
    if constexpr (ORDER == kFours) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (sizeof(T) == 2) {
          const pair_word v = there && at.is[r] ? *(const pair_word_any*)(row + at.at[r]) : pair_word{0, 0};
          w[r * 2] = v[0], w[r * 2 + 1] = v[1];
        } else {
          const word v = there && at.is[r] ? *(const word_any*)(row + at.at[r]) : word{0, 0, 0, 0};
#pragma unroll
          for (int k = 0; k < 4; ++k) w[r * 4 + k] = v[k];
        }
      }
    } else {
      constexpr int kEach = sizeof(T) / 2;  // 16 bytes of a run
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
          const word v = there && at.is[r] ? *(const word_any*)(row + at.at[r] + q * (16 / sizeof(T))) : word{0, 0, 0, 0};
#pragma unroll
          for (int k = 0; k < 4; ++k) w[(r * kEach + q) * 4 + k] = v[k];
        }
    }
  }
  __device__ float value(int i) const {  // element i of the two runs (or four)
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[i]);
    else return __builtin_bit_cast(float, i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  // two elements, rounded to nearest even by the hardware's conversion (written out it is five instructions an element)
  __device__ static uint32_t two(float a, float b) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, b2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
  }
  // the pairs' elements
  __device__ void get(float (&a)[8], float (&b)[8]) const {
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      if constexpr (ORDER == kNeighbours) a[p] = value(2 * p), b[p] = value(2 * p + 1);
      else a[p] = value(p), b[p] = value(8 + p);
    }
  }
  __device__ static void store(T* row, const Place<ORDER>& at, const float (&a)[8], const float (&b)[8]) {
    float v[16];
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      if constexpr (ORDER == kNeighbours) v[2 * p] = a[p], v[2 * p + 1] = b[p];
      else v[p] = a[p], v[8 + p] = b[p];
    }
    if constexpr (ORDER == kFours) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (!at.is[r]) continue;
        if constexpr (sizeof(T) == 2) {
          *(pair_word_any*)(row + at.at[r]) = pair_word{two(v[4 * r], v[4 * r + 1]), two(v[4 * r + 2], v[4 * r + 3])};
        } else {
          *(f4v_any*)(row + at.at[r]) = f4v{v[4 * r], v[4 * r + 1], v[4 * r + 2], v[4 * r + 3]};
        }
      }
    } else {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        if (!at.is[r]) continue;
        if constexpr (sizeof(T) == 2) {
          *(word_any*)(row + at.at[r]) = word{two(v[8 * r], v[8 * r + 1]), two(v[8 * r + 2], v[8 * r + 3]), two(v[8 * r + 4], v[8 * r + 5]),
                                              two(v[8 * r + 6], v[8 * r + 7])};
        } else {
          float e[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) e[i] = v[8 * r + i];
          store8(row + at.at[r], e);
        }
      }
    }
  }
};

// What a lane in a head needs of a vector, 16 floats, lies together in LDS; 80 bytes from lane to lane, so that the reads of a
// head's lanes take all banks evenly.
constexpr int kLaneFloats = 20;
__device__ inline void read_pairs(const float* p, float (&a)[8], float (&b)[8]) {
  const f4v v[4] = {*(const f4v*)p, *(const f4v*)(p + 4), *(const f4v*)(p + 8), *(const f4v*)(p + 12)};
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = v[i / 4][i % 4], b[i] = v[2 + i / 4][i % 4];
}
// The weights of queries and keys (ones where there are none), by the first lanes of the workgroup.
template <int LANES, Order ORDER>
__device__ inline void keep_weights(const Rotary& a, float (*lds)[LANES * kLaneFloats]) {
  if (threadIdx.x < 2 * LANES) {
    const int of = threadIdx.x / LANES, in = threadIdx.x % LANES;
    const Place<ORDER> at(a, in * 8);
    float x[8], y[8];
#pragma unroll
    for (int p = 0; p < 8; ++p) x[p] = y[p] = 1.0f;
    if (a.weight[of] != nullptr) {
      Raw<float, ORDER> raw;
      raw.load(a.weight[of], at, true);
      raw.get(x, y);
    }
#pragma unroll
    for (int p = 0; p < 8; ++p) lds[of][in * kLaneFloats + p] = x[p], lds[of][in * kLaneFloats + 8 + p] = y[p];
  }
  __syncthreads();
}

// cos and sin of the token's angle, pair by pair, in the wavefront's part of LDS; pairs that are not turned have 1 and 0.
__device__ inline void angles(const Rotary& a, int64_t token, double turns, float* table, int lane) {
  float cosine = 1.0f, sine = 0.0f;
  if (lane < a.turned) {
    // whole turns are taken off in 64 bits; twice what is left is in [-1, 1]
    const double at = static_cast<double>(a.positions[token]) * turns;
    sincospif(2.0f * static_cast<float>(at - rint(at)), &sine, &cosine);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  float* const to = table + lane / 8 * kLaneFloats + lane % 8;
  to[0] = cosine, to[8] = sine;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}
__device__ inline double turns_of(const Rotary& a, int lane) {
  return lane < a.turned ? a.frequencies[lane] * 0.15915494309189533577 : 0.0;  // 1 / (2 pi)
}

template <int LANES>
__device__ inline float head_sum(float v) {
#pragma unroll
  for (int s = 1; s < LANES; s <<= 1) v += __shfl_xor(v, s);
  return v;
}

// 1 / sqrt(mean square + eps) of a head's elements x and y, whose mean square is `mean`.  Squares of elements beyond 2^64 or
// below 2^-75 do not fit 32 bits: where any head's mean is far out, the elements are multiplied by a power of two, `scale`, first, and what is
// returned is of those.  (2^-70 brings the largest to 2^58, and the sum of 128 squares below 2^123; eps goes along.)
struct Size {
  float rstd, scale;
  bool scaled;  // of any head of the wavefront
};
template <int LANES>
__device__ inline Size size_of(const Rotary& a, float mean, float (&x)[8], float (&y)[8]) {
  Size s = {0.0f, 1.0f, __any(!(mean >= 0x1p-100f && mean <= 0x1p100f)) != 0};
  if (__builtin_expect(s.scaled, 0)) {
    s.scale = mean > 0x1p100f ? 0x1p-70f : mean < 0x1p-100f ? 0x1p96f : 1.0f;
    float sum = 0.0f;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      x[p] *= s.scale, y[p] *= s.scale;
      sum = fmaf(x[p], x[p], fmaf(y[p], y[p], sum));
    }
    mean = fmaf(head_sum<LANES>(sum), a.inv, a.eps * s.scale * s.scale);
  }
  s.rstd = 1.0f / sqrtf(mean);
  return s;
}

// A wavefront's walk: tokens (or shares of them), and within one the heads, 64 / LANES at a time.
template <int LANES>
struct Walk {
  static constexpr int kHeads = 64 / LANES;
  int64_t item, items, step;
  int32_t pass, passes;
  __device__ Walk(const Rotary& a) {
    passes = (a.all + kHeads - 1) / kHeads;
    items = a.tokens * a.shares;
    step = int64_t(gridDim.x) * kWaves;
    item = blockIdx.x * int64_t(kWaves) + (threadIdx.x >> 6);
    pass = share(a);
  }
  __device__ int32_t share(const Rotary& a) const { return a.shares == 1 ? 0 : static_cast<int32_t>(item % a.shares); }
  __device__ bool there() const { return item < items; }
  __device__ int64_t token(const Rotary& a) const { return a.shares == 1 ? item : item / a.shares; }
  __device__ void next(const Rotary& a) {
    pass += a.shares;
    if (pass >= passes) item += step, pass = share(a);
  }
};

template <class T, int LANES, Order ORDER>
__global__ __launch_bounds__(kThreads) void forward_kernel(Rotary a) {
  __shared__ __attribute__((aligned(16))) float tables[kWaves][8 * kLaneFloats];
  __shared__ __attribute__((aligned(16))) float weights[2][LANES * kLaneFloats];
  const int lane = threadIdx.x & 63, in = lane % LANES, slot = lane / LANES;
  float* const table = tables[threadIdx.x >> 6];
  const Place<ORDER> at(a, in * 8);
  Walk<LANES> w(a);
  Raw<T, ORDER> raw;
  const auto load = [&] {
    const int h = w.pass * Walk<LANES>::kHeads + slot, of = h >= a.heads;
    const T* row = (const T*)a.x[of].p + w.token(a) * a.x[of].token + (h - (of ? a.heads : 0)) * a.x[of].head;
    raw.load(row, at, h < a.all);
  };
  if (w.there()) load();
  const double turns = turns_of(a, lane);
  keep_weights<LANES, ORDER>(a, weights);
  int64_t known = -1;
  while (w.there()) {
    const int64_t token = w.token(a);
    const int h = w.pass * Walk<LANES>::kHeads + slot, of = h >= a.heads;
    float x[8], y[8], cosine[8], sine[8], wa[8], wb[8], sum = 0.0f;
    raw.get(x, y);
    w.next(a);
    if (w.there()) load();
    if (token != known) angles(a, token, turns, table, lane);
    known = token;
#pragma unroll
    for (int p = 0; p < 8; ++p) sum = fmaf(x[p], x[p], fmaf(y[p], y[p], sum));
    const float rstd = size_of<LANES>(a, fmaf(head_sum<LANES>(sum), a.inv, a.eps), x, y).rstd;
    read_pairs(table + in * kLaneFloats, cosine, sine);
    read_pairs(weights[of] + in * kLaneFloats, wa, wb);
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const float u = x[p] * rstd * wa[p], v = y[p] * rstd * wb[p];
      x[p] = fmaf(u, cosine[p], -(v * sine[p]));
      y[p] = fmaf(v, cosine[p], u * sine[p]);
    }
    if (h < a.all)
      Raw<T, ORDER>::store((T*)a.to[of].p + token * a.to[of].token + (h - (of ? a.heads : 0)) * a.to[of].head, at, x, y);
  }
}

// Registers for four wavefronts a SIMD, three where rows are wider or in runs of four: 16384 tokens of 40 heads of 128 in 114 us
// (108 where the clocks have settled), with the weights in registers and two wavefronts 120, with three 130.
template <class T, Order ORDER>
constexpr int kPerSimd = sizeof(T) == 2 && ORDER != kFours ? 4 : 3;
template <class T, int LANES, Order ORDER>
__global__ __launch_bounds__(kThreads, (kPerSimd<T, ORDER>)) void backward_kernel(Rotary a) {
  __shared__ __attribute__((aligned(16))) float tables[kWaves][8 * kLaneFloats];
  __shared__ __attribute__((aligned(16))) float weights[2][LANES * kLaneFloats];
  __shared__ float sums[kWaves][2][LANES * 16];
  constexpr int kHeads = Walk<LANES>::kHeads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in = lane % LANES, slot = lane / LANES;
  float* const table = tables[wave];
  const Place<ORDER> at(a, in * 8);
  Walk<LANES> w(a);
  Raw<T, ORDER> raw, grad;
  const auto load = [&] {
    const int h = w.pass * kHeads + slot, of = h >= a.heads, in_of = h - (of ? a.heads : 0);
    const int64_t token = w.token(a);
    raw.load((const T*)a.x[of].p + token * a.x[of].token + in_of * a.x[of].head, at, h < a.all);
    grad.load((const T*)a.dy[of].p + token * a.dy[of].token + in_of * a.dy[of].head, at, h < a.all);
  };
  if (w.there()) load();
  const double turns = turns_of(a, lane);
  keep_weights<LANES, ORDER>(a, weights);
  float da[2][8], db[2][8];
#pragma unroll
  for (int p = 0; p < 8; ++p) da[0][p] = da[1][p] = db[0][p] = db[1][p] = 0.0f;
  int64_t known = -1;
  while (w.there()) {
    const int64_t token = w.token(a);
    const int first = w.pass * kHeads, h = first + slot, of = h >= a.heads;
    float x[8], y[8], u[8], v[8], s[8], t[8], wa[8], wb[8], sum = 0.0f, dot = 0.0f;
    raw.get(x, y), grad.get(u, v);
    w.next(a);
    if (w.there()) load();
    if (token != known) angles(a, token, turns, table, lane);
    known = token;
#pragma unroll
    for (int p = 0; p < 8; ++p) sum = fmaf(x[p], x[p], fmaf(y[p], y[p], sum));
    // (lanes beyond the last head hold zeros, which without eps are no numbers once divided by their norm: their part of the
    // weights' sums is to be 0)
    const Size size = size_of<LANES>(a, fmaf(head_sum<LANES>(sum), a.inv, a.eps), x, y);
    const float rstd = h < a.all ? size.rstd : 0.0f;
    read_pairs(table + in * kLaneFloats, wa, wb);
#pragma unroll
    for (int p = 0; p < 8; ++p) {  // turned back
      s[p] = fmaf(u[p], wa[p], v[p] * wb[p]), t[p] = fmaf(v[p], wa[p], -(u[p] * wb[p]));
      x[p] *= rstd, y[p] *= rstd;
    }
    if (first + kHeads <= a.heads) {  // queries alone
#pragma unroll
      for (int p = 0; p < 8; ++p) da[0][p] = fmaf(s[p], x[p], da[0][p]), db[0][p] = fmaf(t[p], y[p], db[0][p]);
    } else if (first >= a.heads) {  // keys alone
#pragma unroll
      for (int p = 0; p < 8; ++p) da[1][p] = fmaf(s[p], x[p], da[1][p]), db[1][p] = fmaf(t[p], y[p], db[1][p]);
    } else {
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        const float m = s[p] * x[p], n = t[p] * y[p];
        da[0][p] += of ? 0.0f : m, da[1][p] += of ? m : 0.0f;
        db[0][p] += of ? 0.0f : n, db[1][p] += of ? n : 0.0f;
      }
    }
    read_pairs(weights[of] + in * kLaneFloats, wa, wb);
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      u[p] = s[p] * wa[p], v[p] = t[p] * wb[p];
      dot = fmaf(u[p], x[p], fmaf(v[p], y[p], dot));
    }
    dot = head_sum<LANES>(dot) * a.inv;
#pragma unroll
    for (int p = 0; p < 8; ++p) x[p] = rstd * fmaf(-x[p], dot, u[p]), y[p] = rstd * fmaf(-y[p], dot, v[p]);
    if (__builtin_expect(size.scaled, 0))
#pragma unroll
      for (int p = 0; p < 8; ++p) x[p] *= size.scale, y[p] *= size.scale;
    if (h < a.all)
      Raw<T, ORDER>::store((T*)a.to[of].p + token * a.to[of].token + (h - (of ? a.heads : 0)) * a.to[of].head, at, x, y);
  }
  if (a.partial == nullptr) return;
  // the wavefront's heads, then the wavefronts in order
#pragma unroll
  for (int of = 0; of < 2; ++of)
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      float s = da[of][p], t = db[of][p];
#pragma unroll
      for (int k = LANES; k < 64; k <<= 1) s += __shfl_xor(s, k), t += __shfl_xor(t, k);
      if (slot == 0) sums[wave][of][in * 16 + p] = s, sums[wave][of][in * 16 + 8 + p] = t;
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * LANES * 16; i += kThreads) {
    const int of = i / (LANES * 16), e = i % (LANES * 16);
    float s = sums[0][of][e];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) s += sums[k][of][e];
    const Place<ORDER> from(a, e / 16 * 8);
    // element e % 16 of the lane that holds eight pairs from e / 16 * 8 on
    int run, place;
    if constexpr (ORDER == kNeighbours) run = (e % 8) / 4, place = (e % 8) % 4 * 2 + (e % 16) / 8;
    else if constexpr (ORDER == kFours) run = (e % 16) / 4, place = e % 4;
    else run = (e % 16) / 8, place = e % 8;
    int c = -1;
#pragma unroll
    for (int r = 0; r < 4; ++r) c = r == run && from.is[r] ? from.at[r] + place : c;
    if (c >= 0) a.partial[(int64_t(blockIdx.x) * 2 + of) * a.dim + c] = s;
  }
}

// ------------------------------------------------------------------------- host
int lanes_of(int32_t dim) { return dim <= 32 ? 2 : dim <= 64 ? 4 : 8; }
int32_t shares_of(const daso_rotary_args& s) {
  const int32_t each = 64 / lanes_of(s.dim);
  return s.tokens >= kShareTokens ? 1 : (s.heads + s.kv_heads + each - 1) / each;
}
int32_t groups_of(const daso_rotary_args& s, int32_t most) {
  return static_cast<int32_t>(std::min<int64_t>((s.tokens * shares_of(s) + kWaves - 1) / kWaves, most));
}
size_t backward_bytes(const daso_rotary_args& s) {
  return s.tokens == 0 ? 0 : size_t(groups_of(s, kPartialGroups)) * 2 * size_t(s.dim) * sizeof(float);
}

template <class T, int LANES, Order ORDER>
hipError_t queue(const Rotary& a, bool backward, int32_t groups, hipStream_t stream) {
  const dim3 grid(static_cast<uint32_t>(groups)), block(kThreads);
  return backward ? launch(&backward_kernel<T, LANES, ORDER>, grid, block, stream, a)
                  : launch(&forward_kernel<T, LANES, ORDER>, grid, block, stream, a);
}
template <class T, Order ORDER>
hipError_t queue(const Rotary& a, bool backward, int32_t groups, hipStream_t stream) {
  switch (lanes_of(a.dim)) {
    case 2: return queue<T, 2, ORDER>(a, backward, groups, stream);
    case 4: return queue<T, 4, ORDER>(a, backward, groups, stream);
    default: return queue<T, 8, ORDER>(a, backward, groups, stream);
  }
}
template <class T>
hipError_t queue(const Rotary& a, bool neighbours, bool backward, int32_t groups, hipStream_t stream) {
  if (neighbours) return queue<T, kNeighbours>(a, backward, groups, stream);
  if (a.half % 8 == 0 && a.turned % 8 == 0) return queue<T, kHalves>(a, backward, groups, stream);
  return queue<T, kFours>(a, backward, groups, stream);
}

int run(const daso_rotary_args& s, bool backward, hipStream_t stream) {
  const auto rows = [](const daso_heads& h) { return Rows{h.data, h.token_stride, h.head_stride}; };
  Rotary a;
  a.tokens = s.tokens, a.heads = s.heads, a.all = s.heads + s.kv_heads;
  a.dim = s.dim, a.half = s.dim / 2, a.turned = s.rotated / 2, a.shares = shares_of(s);
  a.eps = s.eps, a.inv = 1.0f / static_cast<float>(s.dim);
  a.positions = s.positions, a.frequencies = s.frequencies, a.weight[0] = s.q_weight, a.weight[1] = s.k_weight;
  a.x[0] = rows(s.q), a.x[1] = rows(s.k);
  a.to[0] = rows(backward ? s.dq : s.q_out), a.to[1] = rows(backward ? s.dk : s.k_out);
  a.dy[0] = rows(s.dq_out), a.dy[1] = rows(s.dk_out);
  const bool sums = backward && (s.dq_weight != nullptr || s.dk_weight != nullptr);
  a.partial = sums ? static_cast<float*>(s.workspace) : nullptr;
  const bool neighbours = (s.flags & DASO_ROTARY_INTERLEAVED) != 0;
  const int32_t groups = s.tokens > 0 ? groups_of(s, backward ? kPartialGroups : kForwardGroups) : 0;
  hipError_t err = hipSuccess;
  if (s.tokens > 0)
    err = s.type == DASO_TYPE_BF16 ? queue<uint16_t>(a, neighbours, backward, groups, stream)
                                   : queue<float>(a, neighbours, backward, groups, stream);
  if (err == hipSuccess && sums)
    err = launch(&partials_kernel, dim3(static_cast<uint32_t>((2 * s.dim + 15) / 16)), dim3(1024), stream, (const float*)a.partial, groups,
                 s.dim, s.dq_weight, s.dk_weight);
  return err == hipSuccess ? DASO_OK : DASO_EHIP;
}

}  // namespace
}  // namespace daso

extern "C" {

int daso_head_norm_rotary(const daso_rotary_args* args, hipStream_t stream) {
  if (args == nullptr) return DASO_EINVAL;
  int rc = daso::host::check_rotary(*args, false);
  if (rc != DASO_OK || args->tokens == 0) return rc;
  if ((rc = daso::current_device(stream)) != DASO_OK) return rc;
  return daso::run(*args, false, stream);
}

int daso_head_norm_rotary_backward_workspace(const daso_rotary_args* args, size_t* bytes) {
  if (args == nullptr || bytes == nullptr) return DASO_EINVAL;
  const int rc = daso::host::check_rotary_sizes(*args);
  if (rc != DASO_OK) return rc;
  *bytes = daso::backward_bytes(*args);
  return DASO_OK;
}

int daso_head_norm_rotary_backward(const daso_rotary_args* args, hipStream_t stream) {
  if (args == nullptr) return DASO_EINVAL;
  const daso_rotary_args& s = *args;
  int rc = daso::host::check_rotary(s, true);
  if (rc != DASO_OK) return rc;
  const bool sums = s.dq_weight != nullptr || s.dk_weight != nullptr;
  if (s.tokens == 0 && !sums) return DASO_OK;
  if (sums && (rc = daso::host::check_workspace(s.workspace, s.workspace_bytes, daso::backward_bytes(s))) != DASO_OK) return rc;
  if ((rc = daso::current_device(stream)) != DASO_OK) return rc;
  return daso::run(s, true, stream);
}

}  // extern "C"
