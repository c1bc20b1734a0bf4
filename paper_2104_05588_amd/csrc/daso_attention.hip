// Attention over packed sequences, forward and backward (daso_block.h).
//
// Forward: a wavefront has 32 queries and walks over the keys it sees, with the running maximum and sum of the softmax.
// Backward: two passes that each compute the scores again, so that no sum is added up across workgroups: one
// by queries (dq, and sum dout out, which the other reads), one by keys (dk and dv, over all query heads of the key
// head).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "daso_attention_tile.h"

namespace daso {
namespace attention {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

constexpr int kThreads = 256, kWaves = 4, kOwn = kWaves * 32;  // rows of a workgroup
constexpr float kGrowth = 10.0f;
constexpr int kPairs = 512;  // units that make pairs worth while: two workgroups a CU
// Wavefronts a SIMD that the registers are dealt for.
template <class T, int D>
constexpr int kForwardPerSimd = sizeof(T) == 2 && D <= 64 ? 3 : sizeof(T) == 2 || D < 128 ? 2 : 1;
template <class T, int D>
constexpr int kQueryPerSimd = sizeof(T) == 2 ? (D <= 32 ? 3 : D <= 96 ? 2 : 1) : D <= 64 ? 2 : 1;
template <class T, int D>
constexpr int kKeyPerSimd = sizeof(T) == 2 ? (D <= 64 ? 2 : 1) : D <= 32 ? 2 : 1;
template <class T>
constexpr int kTile = sizeof(T) == 2 ? 64 : 32;  // rows of a tile in LDS

template <class T>
__device__ inline const T* head_of(const Rows& r, int64_t start, int head) {
  return (const T*)r.p + start * r.token + head * r.head;
}

template <class T, int D>
__device__ inline void forward_tile(const Attention& a, const Place& at, char (&lds)[2][2][Stage<T, D, kTile<T>, kThreads>::kBytes]) {
  using K = Kind<T, D>;
  constexpr int kKeys = kTile<T>, kSubs = kKeys / 32;
  using S = Stage<T, D, kKeys, kThreads>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = at.row + wave * 32, mine = first + (lane & 31);
  const T *k = head_of<T>(a.k, at.start, at.head / a.share), *v = head_of<T>(a.v, at.start, at.head / a.share);
  u4 q[K::kParts];
  own_row<kOwn, T, D>(head_of<T>(a.q, at.start, at.head), a.q.token, at.row, wave * 32 + (lane & 31), at.len, a.dim, q);
  const int last = a.causal ? min(mine, at.len - 1) : at.len - 1;  // key that the lane's query sees
  const int keys = a.causal ? min(at.len, at.row + kOwn) : at.len;
  const int whole = (a.causal ? min(at.len, at.row + 1) : at.len) / kKeys * kKeys;  // keys below are seen by all queries
  f16v acc[D / 32];
#pragma unroll
  for (int b = 0; b < D / 32; ++b) acc[b] = (f16v)0.0f;
  // The exponents' base, of z log2 e, and the lane's keys' share of the sum.  The base follows the maximum only where that
  // has grown by more than 2^kGrowth, which the sums have room for.
  float top = -INFINITY, base = 0.0f, sum = 0.0f;
  S ks(k, a.k.token, a.dim), vs(v, a.v.token, a.dim);
  const auto fetch = [&](int key) { ks.load(key, at.len), vs.load(key, at.len); };
  const auto keep = [&](int buffer) { ks.store(lds[buffer][0]), vs.store(lds[buffer][1]); };
  // The base for the scores of 32 keys, and their powers in place of them.
  const auto raise = [&](const f16v& z) {
    float most = z[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) most = fmaxf(most, z[r]);
    most = halves_max(most) * a.scale2;
    const bool grown = most > top + kGrowth;  // (a row of its own: nothing that other rows hold changes its bits)
    if (__any(grown)) {
      const float alpha = grown ? exp2_fast(top - most) : 1.0f;
      top = grown ? most : top, base = grown ? most : base;
      sum *= alpha;
#pragma unroll
      for (int b = 0; b < D / 32; ++b) acc[b] *= alpha;
    }
  };
  const auto soften = [&](f16v& z) {
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = exp2_fast(fmaf(z[r], a.scale2, -base));
    sum += sum_of(z);
  };
  const auto step = [&](int buffer) {
    f16v z = scores<T, D>(lds[buffer][0], 0, q, (f16v)0.0f);
#pragma unroll
    for (int s = 0; s < kSubs; ++s) {
      raise(z);
      f16v next;
      if (s + 1 < kSubs) next = scores<T, D>(lds[buffer][0], (s + 1) * 32, q, (f16v)0.0f);
      soften(z);
      const typename K::Right p(z);
#pragma unroll
      for (int b = 0; b < D / 32; ++b) K::gather(lds[buffer][1], s * 32, b, p, acc[b]);
      z = next;
    }
  };
  // The same for keys of which each query sees its own.
  const auto step_part = [&](int key, int buffer) {
#pragma unroll 1
    for (int s = 0; s < kSubs; ++s) {
      if (a.causal && key + s * 32 >= first + 32) break;
      f16v z = scores<T, D>(lds[buffer][0], s * 32, q, (f16v)0.0f);
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = key + s * 32 + row_in(r) <= last ? z[r] : -INFINITY;
      raise(z);
      soften(z);
      const typename K::Right p(z);
#pragma unroll
      for (int b = 0; b < D / 32; ++b)
        K::template gather_part<1>(lds[buffer][1], s * 32, b, p, last - key, acc[b]);
    }
  };
  fetch(0);
  __syncthreads();
  keep(0);
  __syncthreads();
  int key = 0, buffer = 0;
  for (; key < whole; key += kKeys, buffer ^= 1) {
    const bool more = key + kKeys < keys;
    if (more) fetch(key + kKeys);
    step(buffer);
    if (more) keep(buffer ^ 1);
    __syncthreads();
  }
  for (; key < keys; key += kKeys, buffer ^= 1) {
    const bool more = key + kKeys < keys;
    if (more) fetch(key + kKeys);
    step_part(key, buffer);
    if (more) keep(buffer ^ 1);
    __syncthreads();
  }
  sum = halves_sum(sum);
  if (mine >= at.len) return;
  put_row<T, D>((T*)head_of<T>(a.out, at.start, at.head) + mine * a.out.token, acc, 1.0f / sum, a.dim);
  if (lane < 32) a.lse[at.head * a.tokens + at.start + mine] = (base + log2f(sum)) * kLn2;
}

template <class T, int D>
__global__ __launch_bounds__(kThreads, (kForwardPerSimd<T, D>)) void forward_kernel(Attention a) {
  __shared__ __attribute__((aligned(16))) char lds[2][2][Stage<T, D, kTile<T>, kThreads>::kBytes];
  Place at;
  const Found found = place_of<kOwn>(a, a.heads, &at);
  if (found == kNone) return;
  for (int t = 0; t < 2 && at.turn<kOwn>(a, t, true); ++t) {
    if (found == kSequence) {
      forward_tile<T, D>(a, at, lds);
      __syncthreads();
      continue;
    }
    if (!a.zero_q) return;
    zero_rows<kOwn>((T*)head_of<T>(a.out, at.start, at.head), a.out.token, at, a.dim);
    zero_rows<kOwn>(a.lse + at.head * a.tokens + at.start, 1, at, 1);
  }
}

template <class T, int D>
__device__ inline void query_tile(const Attention& a, const Place& at, char (&lds)[2][2][Stage<T, D, kTile<T>, kThreads>::kBytes]) {
  using K = Kind<T, D>;
  constexpr int kKeys = kTile<T>, kSubs = kKeys / 32;
  using S = Stage<T, D, kKeys, kThreads>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = at.row + wave * 32, mine = first + (lane & 31);
  const bool there = mine < at.len;
  const T *k = head_of<T>(a.k, at.start, at.head / a.share), *v = head_of<T>(a.v, at.start, at.head / a.share);
  u4 q[K::kParts], g[K::kParts];
  own_row<kOwn, T, D>(head_of<T>(a.q, at.start, at.head), a.q.token, at.row, wave * 32 + (lane & 31), at.len, a.dim, q);
  own_row<kOwn, T, D>(head_of<T>(a.dout, at.start, at.head), a.dout.token, at.row, wave * 32 + (lane & 31), at.len, a.dim, g);
  float delta = 0.0f;
  {
    u4 o[K::kParts];
    own_row<kOwn, T, D>(head_of<T>(a.out, at.start, at.head), a.out.token, at.row, wave * 32 + (lane & 31), at.len, a.dim, o);
#pragma unroll
    for (int c = 0; c < K::kParts; ++c) delta += K::dot(g[c], o[c]);
    delta = halves_sum(delta);
  }
  const int64_t stat = at.head * a.tokens + at.start + mine;
  const float lse2 = there ? a.lse[stat] * kLog2e : INFINITY;
  if (there && lane < 32) a.delta[stat] = delta;
  const int last = a.causal ? min(mine, at.len - 1) : at.len - 1;
  const int keys = a.causal ? min(at.len, at.row + kOwn) : at.len;
  const int wave_keys = a.causal ? min(at.len, first + 32) : at.len;
  const int all_see = a.causal ? min(at.len, first + 1) : at.len;
  f16v acc[D / 32];
#pragma unroll
  for (int b = 0; b < D / 32; ++b) acc[b] = (f16v)0.0f;
  S ks(k, a.k.token, a.dim), vs(v, a.v.token, a.dim);
  const auto fetch = [&](int key) { ks.load(key, at.len), vs.load(key, at.len); };
  const auto keep = [&](int buffer) { ks.store(lds[buffer][0]), vs.store(lds[buffer][1]); };
  fetch(0);
  __syncthreads();
  keep(0);
  __syncthreads();
  for (int key = 0, buffer = 0; key < keys; key += kKeys, buffer ^= 1) {
    const bool more = key + kKeys < keys;
    if (more) fetch(key + kKeys);
    if (key < wave_keys) {
#pragma unroll
      for (int s = 0; s < kSubs; ++s) {
        f16v z = scores<T, D>(lds[buffer][0], s * 32, q, (f16v)0.0f);
        const f16v dp = scores<T, D>(lds[buffer][1], s * 32, g, (f16v)(-delta));
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r] = exp2_fast(fmaf(z[r], a.scale2, -lse2)) * dp[r];
        const bool part = key + kKeys > all_see;
        if (part)
#pragma unroll
          for (int r = 0; r < 16; ++r) z[r] = key + s * 32 + row_in(r) <= last ? z[r] : 0.0f;
        const typename K::Right ds(z);
        if (part) {
#pragma unroll
          for (int b = 0; b < D / 32; ++b)
            K::template gather_part<1>(lds[buffer][0], s * 32, b, ds, last - key, acc[b]);
        } else {
#pragma unroll
          for (int b = 0; b < D / 32; ++b) K::gather(lds[buffer][0], s * 32, b, ds, acc[b]);
        }
      }
    }
    if (more) keep(buffer ^ 1);
    __syncthreads();
  }
  if (there) put_row<T, D>((T*)head_of<T>(a.dq, at.start, at.head) + mine * a.dq.token, acc, a.scale, a.dim);
}

template <class T, int D>
__global__ __launch_bounds__(kThreads, (kQueryPerSimd<T, D>)) void query_kernel(Attention a) {
  __shared__ __attribute__((aligned(16))) char lds[2][2][Stage<T, D, kTile<T>, kThreads>::kBytes];
  Place at;
  const Found found = place_of<kOwn>(a, a.heads, &at);
  if (found == kNone) return;
  for (int t = 0; t < 2 && at.turn<kOwn>(a, t, true); ++t) {
    if (found == kSequence) {
      query_tile<T, D>(a, at, lds);
      __syncthreads();
      continue;
    }
    if (a.zero_q) zero_rows<kOwn>((T*)head_of<T>(a.dq, at.start, at.head), a.dq.token, at, a.dim);
  }
}

template <class T, int D>
__device__ inline void key_tile(const Attention& a, const Place& at, char (&lds)[2][2][Stage<T, D, kTile<T>, kThreads>::kBytes],
                                float (&stats)[2][2][kTile<T>]) {
  using K = Kind<T, D>;
  constexpr int kQueries = kTile<T>, kSubs = kQueries / 32;
  using S = Stage<T, D, kQueries, kThreads>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = at.row + wave * 32, mine = first + (lane & 31);
  const bool there = mine < at.len;
  u4 k[K::kParts], v[K::kParts];
  own_row<kOwn, T, D>(head_of<T>(a.k, at.start, at.head), a.k.token, at.row, wave * 32 + (lane & 31), at.len, a.dim, k);
  own_row<kOwn, T, D>(head_of<T>(a.v, at.start, at.head), a.v.token, at.row, wave * 32 + (lane & 31), at.len, a.dim, v);
  f16v dk[D / 32], dv[D / 32];
#pragma unroll
  for (int b = 0; b < D / 32; ++b) dk[b] = dv[b] = (f16v)0.0f;
  // the queries that see a key of the workgroup, head by head
  const int from = a.causal ? at.row / kQueries * kQueries : 0;
  const int tiles = (at.len - from + kQueries - 1) / kQueries, steps = tiles * a.share;
  const int whole = a.causal ? first + 31 : 0;  // queries from here on see all keys of the wavefront
  S qs((const T*)nullptr, a.q.token, a.dim), gs((const T*)nullptr, a.dout.token, a.dim);
  float stat = 0.0f;
  const auto fetch = [&](int step) {
    const int head = at.head * a.share + step / tiles, row = from + step % tiles * kQueries;
    qs.p = head_of<T>(a.q, at.start, head), gs.p = head_of<T>(a.dout, at.start, head);
    qs.load(row, at.len), gs.load(row, at.len);
    if (threadIdx.x < 2 * kQueries) {
      const int r = row + threadIdx.x % kQueries;
      const int64_t i = head * a.tokens + at.start + r;
      if (threadIdx.x < kQueries) stat = r < at.len ? -a.lse[i] * kLog2e : -INFINITY;  // exp of rows that are not there is 0
      else stat = r < at.len ? -a.delta[i] : 0.0f;
    }
  };
  const auto keep = [&](int buffer) {
    qs.store(lds[buffer][0]), gs.store(lds[buffer][1]);
    if (threadIdx.x < 2 * kQueries) stats[buffer][threadIdx.x / kQueries][threadIdx.x % kQueries] = stat;
  };
  fetch(0);
  __syncthreads();
  keep(0);
  __syncthreads();
  for (int step = 0, buffer = 0; step < steps; ++step, buffer ^= 1) {
    const bool more = step + 1 < steps;
    if (more) fetch(step + 1);
    const int row = from + step % tiles * kQueries;
    if (!a.causal || row + kQueries > first) {
#pragma unroll
      for (int s = 0; s < kSubs; ++s) {
        f16v lse, z, dp;
        const int h = lane >> 5;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f4v x = *(const f4v*)&stats[buffer][0][s * 32 + 8 * g + 4 * h], y = *(const f4v*)&stats[buffer][1][s * 32 + 8 * g + 4 * h];
#pragma unroll
          for (int i = 0; i < 4; ++i) lse[4 * g + i] = x[i], dp[4 * g + i] = y[i];
        }
        z = scores<T, D>(lds[buffer][0], s * 32, k, (f16v)0.0f);
        dp = scores<T, D>(lds[buffer][1], s * 32, v, dp);
        const bool part = row < whole || row + kQueries > at.len;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          z[r] = exp2_fast(fmaf(z[r], a.scale2, lse[r]));
          dp[r] *= z[r];
        }
        if (part)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int i = row + s * 32 + row_in(r);
            const bool sees = i < at.len && (!a.causal || i >= mine);
            z[r] = sees ? z[r] : 0.0f, dp[r] = sees ? dp[r] : 0.0f;
          }
        const typename K::Right p(z), ds(dp);
        if (part) {
          const int limit = row - mine;  // (rows that are not there are zeros)
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
    }
    if (more) keep(buffer ^ 1);
    __syncthreads();
  }
  if (!there) return;
  put_row<T, D>((T*)head_of<T>(a.dk, at.start, at.head) + mine * a.dk.token, dk, a.scale, a.dim);
  put_row<T, D>((T*)head_of<T>(a.dv, at.start, at.head) + mine * a.dv.token, dv, 1.0f, a.dim);
}

template <class T, int D>
__global__ __launch_bounds__(kThreads, (kKeyPerSimd<T, D>)) void key_kernel(Attention a) {
  __shared__ __attribute__((aligned(16))) char lds[2][2][Stage<T, D, kTile<T>, kThreads>::kBytes];
  __shared__ __attribute__((aligned(16))) float stats[2][2][kTile<T>];
  Place at;
  const Found found = place_of<kOwn>(a, a.kv_heads, &at);
  if (found == kNone) return;
  for (int t = 0; t < 2 && at.turn<kOwn>(a, t, false); ++t) {
    if (found == kSequence) {
      key_tile<T, D>(a, at, lds, stats);
      __syncthreads();
      continue;
    }
    if (a.zero_k) zero_rows<kOwn>((T*)head_of<T>(a.dk, at.start, at.head), a.dk.token, at, a.dim);
    if (a.zero_v) zero_rows<kOwn>((T*)head_of<T>(a.dv, at.start, at.head), a.dv.token, at, a.dim);
  }
}

// ------------------------------------------------------------------------- host
// The units of a head, at most, and whether they are pairs of tiles.
Attention dealt(Attention a, int heads) {
  const int64_t tiles = (a.tokens + kOwn - 1) / kOwn;
  a.pairs = a.causal && tiles * heads / 2 >= kPairs;
  const int rows = a.pairs ? 2 * kOwn : kOwn;
  a.units = static_cast<int32_t>(a.offsets != nullptr ? a.tokens / rows + a.sequences + 1 : (a.tokens + rows - 1) / rows);
  return a;
}
template <class T, int D>
hipError_t queue(const Attention& a, bool backward, hipStream_t stream) {
  const Attention q = dealt(a, a.heads), k = dealt(a, a.kv_heads);
  const dim3 block(kThreads), queries(static_cast<uint32_t>(q.units * q.heads)), keys(static_cast<uint32_t>(k.units * k.kv_heads));
  if (!backward) return launch(&forward_kernel<T, D>, queries, block, stream, q);
  const hipError_t err = launch(&query_kernel<T, D>, queries, block, stream, q);
  return err == hipSuccess ? launch(&key_kernel<T, D>, keys, block, stream, k) : err;
}
template <class T>
hipError_t queue(const Attention& a, bool backward, hipStream_t stream) {
  if (a.dim <= 32) return queue<T, 32>(a, backward, stream);
  if (a.dim <= 64) return queue<T, 64>(a, backward, stream);
  if (a.dim <= 96) return queue<T, 96>(a, backward, stream);
  return queue<T, 128>(a, backward, stream);
}

size_t backward_bytes(const daso_attention_args& s) { return static_cast<size_t>(s.tokens) * size_t(s.heads) * sizeof(float); }

int run(const daso_attention_args& s, bool backward, hipStream_t stream) {
  // (of a single token the distance to the next may be anything)
  const auto rows = [&s](const daso_heads& h) { return Rows{h.data, s.tokens > 1 ? h.token_stride : s.dim, h.head_stride}; };
  Attention a;
  a.tokens = s.tokens, a.offsets = s.offsets, a.sequences = s.sequences, a.heads = s.heads, a.kv_heads = s.kv_heads;
  a.share = s.heads / s.kv_heads, a.dim = s.dim, a.causal = (s.flags & DASO_ATTENTION_CAUSAL) != 0;
  a.zero_q = (s.flags & DASO_ATTENTION_ZERO_Q) != 0, a.zero_k = (s.flags & DASO_ATTENTION_ZERO_K) != 0;
  a.zero_v = (s.flags & DASO_ATTENTION_ZERO_V) != 0;
  a.scale = s.scale, a.scale2 = s.scale * kLog2e;
  a.q = rows(s.q), a.k = rows(s.k), a.v = rows(s.v), a.out = rows(s.out), a.dout = rows(s.dout);
  a.dq = rows(s.dq), a.dk = rows(s.dk), a.dv = rows(s.dv), a.lse = s.lse, a.delta = static_cast<float*>(s.workspace);
  const hipError_t err = s.type == DASO_TYPE_BF16 ? queue<uint16_t>(a, backward, stream) : queue<float>(a, backward, stream);
  return err == hipSuccess ? DASO_OK : DASO_EHIP;
}

}  // namespace
}  // namespace attention
}  // namespace daso

extern "C" {

int daso_attention(const daso_attention_args* args, hipStream_t stream) {
  if (args == nullptr) return DASO_EINVAL;
  int rc = daso::host::check_attention(*args, false);
  if (rc != DASO_OK || args->tokens == 0 || (args->sequences == 0 && args->offsets == nullptr)) return rc;
  if ((rc = daso::current_device(stream)) != DASO_OK) return rc;
  return daso::attention::run(*args, false, stream);
}

int daso_attention_backward_workspace(const daso_attention_args* args, size_t* bytes) {
  if (args == nullptr || bytes == nullptr) return DASO_EINVAL;
  const int rc = daso::host::check_attention_sizes(*args);
  if (rc != DASO_OK) return rc;
  *bytes = daso::attention::backward_bytes(*args);
  return DASO_OK;
}

int daso_attention_backward(const daso_attention_args* args, hipStream_t stream) {
  if (args == nullptr) return DASO_EINVAL;
  int rc = daso::host::check_attention(*args, true);
  if (rc != DASO_OK || args->tokens == 0 || (args->sequences == 0 && args->offsets == nullptr)) return rc;
  rc = daso::host::check_workspace(args->workspace, args->workspace_bytes, daso::attention::backward_bytes(*args));
  if (rc != DASO_OK) return rc;
  if ((rc = daso::current_device(stream)) != DASO_OK) return rc;
  return daso::attention::run(*args, true, stream);
}

}  // extern "C"
