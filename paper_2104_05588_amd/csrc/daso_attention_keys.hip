// Attention over packed sequences, the backward pass by keys (daso_block.h): a wavefront has 32 keys and walks over the queries
// that see them, of all query heads of the key head.
//
// Four products of 32 x 32 scores, 512 cycles of a SIMD's matrix cores for 64 elements and 1024 for 128, beside the forward pass's 16 powers a
// lane, 128 cycles of 476 and 744 in vector instructions, and 457 and 781 in LDS; counted are 1221 and 3247 in all, so that none of them
// alone bounds it: they wait for each other.  dk and dv of a wavefront take 32 registers for each 32 elements, its keys and values 32 more,
// which leaves one wavefront a SIMD with 128 elements, 1387 us for 8192 x 16 x 128, not causal (0.79 PFLOP/s), and two with
// fewer: 569 and 590 us on two machines for 8192 x 16 x 64 (0.97 and 0.93).
#include <hip/hip_runtime.h>

#include "daso_attention_tile.h"

namespace daso {
namespace attention {
namespace {

// Wavefronts a SIMD that the registers are dealt for.
template <class T, int D>
constexpr int kKeyPerSimd = sizeof(T) == 2 ? (D <= 96 ? 2 : 1) : D <= 32 ? 2 : 1;
// Rows of a tile of its queries.  (96 elements in tiles of 32 leave registers for two wavefronts a SIMD: 8192 x 16 x 96 in 1110 us.)
template <class T, int D>
constexpr int kQueryTile = D == 96 ? 32 : kTile<T>;
template <class T, int D>
__device__ inline void key_tile(const Attention& a, const Place& at,
                                char (&lds)[2][2][Stage<T, D, kQueryTile<T, D>, kThreads>::kBytes],
                                float (&stats)[2][2][kQueryTile<T, D>]) {
  using K = Kind<T, D>;
  constexpr int kQueries = kQueryTile<T, D>, kSubs = kQueries / 32;
  constexpr bool kAlone = sizeof(T) == 2 && kKeyPerSimd<T, D> == 1;
  using S = Stage<T, D, kQueries, kThreads>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = at.row + wave * 32, mine = first + (lane & 31);
  const int kv = at.head / a.parts, part = at.head % a.parts, each = a.share / a.parts;
  char* const room = lds[0][0];
  static_assert(sizeof lds >= Stage<T, D, kOwn, kThreads>::kBytes, "room for the workgroup's own rows");
  u4 k[K::kParts], v[K::kParts];
  {
    const Own<T, D> keys(head_of<T>(a.k, at.start, kv), a.k.token, at.row, at.len, a.dim);
    const Own<T, D> values(head_of<T>(a.v, at.start, kv), a.v.token, at.row, at.len, a.dim);
    keys.read(room, k);
    values.read(room, v);
  }
  f16v dk[D / 32], dv[D / 32];
#pragma unroll
  for (int b = 0; b < D / 32; ++b) dk[b] = dv[b] = (f16v)0.0f;
  // the queries that see a key of the workgroup, head by head
  const int from = a.causal ? at.row / kQueries * kQueries : 0, heads = kv * a.share + (part + 1) * each;
  S qs((const T*)nullptr, a.q.token, a.dim), gs((const T*)nullptr, a.dout.token, a.dim);
  float stat = 0.0f;
  // The next tile comes in two halves: its queries with their numbers during the first half of this one, then dout.
  const auto fetch = [&](int head, int row) {
    qs.p = head_of<T>(a.q, at.start, head), qs.load(row, at.len);
    if (threadIdx.x < 2 * kQueries) {
      const int r = row + threadIdx.x % kQueries;
      const int64_t i = head * a.tokens + at.start + r;
      if (threadIdx.x < kQueries) stat = r < at.len ? -a.lse[i] * kLog2e : -INFINITY;  // exp of rows that are not there is 0
      else stat = r < at.len ? -a.delta[i] : 0.0f;
    }
  };
  const auto turn = [&](int head, int row, int buffer) {
    qs.store(lds[buffer][0]);
    if (threadIdx.x < 2 * kQueries) stats[buffer][threadIdx.x / kQueries][threadIdx.x % kQueries] = stat;
    gs.p = head_of<T>(a.dout, at.start, head), gs.load(row, at.len);
  };
  int head = heads - each, row = from, buffer = 0;
  fetch(head, row);
  turn(head, row, 0);
  gs.store(lds[0][1]);
  __syncthreads();
  while (head < heads) {
    int next_head = head, next_row = row + kQueries;
    if (next_row >= at.len) ++next_head, next_row = from;
    const bool more = next_head < heads;
    if (more) fetch(next_head, next_row);
#pragma unroll
    for (int s = 0; s < kSubs; ++s) {
      const int i = row + s * 32;
      if (s == (kSubs + 1) / 2 && more) turn(next_head, next_row, buffer ^ 1);
      if (i >= at.len || (a.causal && i + 31 < first)) continue;
      f16v lse, dp;  // -lse log2 e and -delta of the queries, and what comes of the latter
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int r = s * 32 + 8 * g + 4 * (lane >> 5);
        const f4v x = *(const f4v*)&stats[buffer][0][r], y = *(const f4v*)&stats[buffer][1][r];
#pragma unroll
        for (int j = 0; j < 4; ++j) lse[4 * g + j] = x[j], dp[4 * g + j] = y[j];
      }
      f16v z = scores<T, D>(lds[buffer][0], s * 32, k, (f16v)0.0f);
      if constexpr (kAlone) {
        // one wavefront a SIMD: the powers are taken while the matrix cores work on dp
        Parts<T, D> g;
        g.read(lds[buffer][1], s * 32);
        pin();
#pragma unroll
        for (int j = 0; j < K::kParts; ++j) {
          dp = K::multiply(g.of[j], v[j], dp);
#pragma unroll
          for (int r = j * 16 / K::kParts; r < (j + 1) * 16 / K::kParts; ++r) z[r] = exp2_fast(fmaf(z[r], a.scale2, lse[r]));
          pin();
        }
      } else {
        dp = scores<T, D>(lds[buffer][1], s * 32, v, dp);
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r] = exp2_fast(fmaf(z[r], a.scale2, lse[r]));
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) dp[r] *= z[r];
      // where a query sees some of the keys, or is not there
      const bool part = (a.causal && i < first + 31) || i + 31 >= at.len;
      if (part)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const bool sees = i + row_in(r) < at.len && (!a.causal || i + row_in(r) >= mine);
          z[r] = sees ? z[r] : 0.0f, dp[r] = sees ? dp[r] : 0.0f;
        }
      const typename K::Right p(z), ds(dp);
      if (part) {
        const int limit = a.causal ? row - mine : INT32_MAX - 1;  // (rows that are not there are zeros: seen or not)
#pragma unroll
        for (int b = 0; b < D / 32; ++b) {
          K::template gather_part<-1>(lds[buffer][1], s * 32, b, p, limit, dv[b]);
          K::template gather_part<-1>(lds[buffer][0], s * 32, b, ds, limit, dk[b]);
        }
      } else {
#pragma unroll
        for (int b = 0; b < D / 32; ++b) {
          K::gather(lds[buffer][1], s * 32, b, p, dv[b]);
          K::gather(lds[buffer][0], s * 32, b, ds, dk[b]);
        }
      }
    }
    if (kSubs == 1 && more) turn(next_head, next_row, buffer ^ 1);
    if (more) gs.store(lds[buffer ^ 1][1]);
    head = next_head, row = next_row, buffer ^= 1;
    __syncthreads();
  }
  if (a.parts > 1) {
    const int64_t plane = a.tokens * a.kv_heads * a.dim, apart = int64_t(a.kv_heads) * a.dim;
    float* to = a.partial + 2 * part * plane + at.start * apart + kv * a.dim;
    if (mine >= at.len) return;
    put_own<D>(to + mine * apart, dk, a.scale, a.dim);
    put_own<D>(to + plane + mine * apart, dv, 1.0f, a.dim);
    return;
  }
  put_rows<T, D>(room, (T*)head_of<T>(a.dk, at.start, kv), a.dk.token, first, at.len, a.dim, dk, a.scale);
  put_rows<T, D>(room, (T*)head_of<T>(a.dv, at.start, kv), a.dv.token, first, at.len, a.dim, dv, 1.0f);
}

template <class T, int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(kKeyPerSimd<T, D>, kKeyPerSimd<T, D>))) void key_kernel(Attention a) {
  __shared__ __attribute__((aligned(16))) char lds[2][2][Stage<T, D, kQueryTile<T, D>, kThreads>::kBytes];
  __shared__ __attribute__((aligned(16))) float stats[2][2][kQueryTile<T, D>];
  Place at;
  const Found found = place_of<kOwn, false>(a, a.kv_heads * a.parts, &at);
  if (found == kSequence) return key_tile<T, D>(a, at, lds, stats);
  if (found == kNone || at.head % a.parts != 0) return;
  at.head /= a.parts;
  if (!a.zero_k && !a.zero_v) return;
  over_rest<kOwn>(a, at, [&](int from, int to) {
    if (a.zero_k) zero_rows((T*)head_of<T>(a.dk, at.start, at.head), a.dk.token, from, to, a.dim);
    if (a.zero_v) zero_rows((T*)head_of<T>(a.dv, at.start, at.head), a.dv.token, from, to, a.dim);
  });
}

// dk and dv of 32 rows from the parts, in order.
template <class T>
__global__ __launch_bounds__(kThreads) void join_kernel(Attention a) {
  constexpr int kRows = 32;
  Place at;
  if (place_of<kRows, false>(a, a.kv_heads, &at) != kSequence) return;
  const int64_t plane = a.tokens * a.kv_heads * a.dim;
  const int fours = a.dim / 4, rows = min(kRows, at.len - at.row);
  for (int i = threadIdx.x; i < 2 * rows * fours; i += kThreads) {
    const int which = i >= rows * fours, in = i - which * rows * fours, row = at.row + in / fours, c = in % fours * 4;
    const float* from = a.partial + which * plane + ((at.start + row) * a.kv_heads + at.head) * a.dim + c;
    f4v sum = load4(from);
    for (int p = 1; p < a.parts; ++p) sum += load4(from + 2 * p * plane);
    const Rows& to = which ? a.dv : a.dk;
    put4((T*)head_of<T>(to, at.start, at.head) + row * to.token + c, sum[0], sum[1], sum[2], sum[3]);
  }
}

// ------------------------------------------------------------------------- host
template <class T, int D>
hipError_t queue(const Attention& a, hipStream_t stream) {
  return launch(&key_kernel<T, D>, dim3(static_cast<uint32_t>(a.tiles * a.kv_heads * a.parts)), dim3(kThreads), stream, a);
}
template <class T>
hipError_t queue(const Attention& a, hipStream_t stream) {
  hipError_t err;
  if (a.dim <= 32) err = queue<T, 32>(a, stream);
  else if (a.dim <= 64) err = queue<T, 64>(a, stream);
  else if (a.dim <= 96) err = queue<T, 96>(a, stream);
  else err = queue<T, 128>(a, stream);
  if (err != hipSuccess || a.parts == 1) return err;
  Attention b = a;
  b.tiles = tiles_of<32>(a), b.sorted = 0;
  return launch(&join_kernel<T>, dim3(static_cast<uint32_t>(b.tiles * b.kv_heads)), dim3(kThreads), stream, b);
}

}  // namespace

hipError_t queue_keys(const Attention& from, int32_t type, hipStream_t stream) {
  Attention a = from;
  a.sorted = a.tiles * a.kv_heads * a.parts <= kFewTiles;
  return type == DASO_TYPE_BF16 ? queue<uint16_t>(a, stream) : queue<float>(a, stream);
}

}  // namespace attention
}  // namespace daso
