// Attention over packed sequences, forward and the backward pass by queries (daso_block.h).
//
// Forward: a wavefront has 32 queries and walks over the keys it sees, with the running maximum and sum of the softmax.
// Backward: two passes that each compute the scores again, so that no sum is added up across workgroups: one
// by queries (dq, and sum dout out, which the other reads), one by keys (dk and dv, over all query heads of the key
// head).
//
// Bound by vector instructions and the matrix cores together, which overlap little, from different wavefronts.  Forward, the two
// products of 32 x 32 scores of 64 elements take a SIMD 256 cycles (1024 operations each) and the vector instructions 458,
// 128 of them for the 16 powers, 8 each; counted are 684 in all.  With 128 elements 512 and 537, of 1134.  By queries, with the
// mean's product, 512 and 486 of 918, and with 128 elements and one wavefront a SIMD 1024 and 771 of 2394.  LDS is read for less than half of
// the time in all of them.  A workgroup of four wavefronts shares the tiles of 64 keys (32 in fp32): its own 128 rows are
// in registers, so what is read from LDS is the tile's alone, and the next tile is on its way meanwhile.
// 8192 x 16 x 64, not causal, on two machines: 340 and 353 us forward (0.81 and 0.78 PFLOP/s), 489 and 510 by queries (1.12 and 1.08 with the
// mean's product); 8192 x 16 x 128: 566 and 585 (0.97 and 0.94), 1047 and 1072 (1.05 and 1.03).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "daso_attention_tile.h"

namespace daso {
namespace attention {
namespace {

constexpr float kGrowth = 10.0f;
// Wavefronts a SIMD that the registers are dealt for: as many as leave no spills in the loop over whole tiles, which cost more than a
// wavefront (by queries with 96 elements and tiles of 64 keys: 970 us for 8192 x 16 with one, 1375 with two).
template <class T, int D>
constexpr int kForwardPerSimd = sizeof(T) == 2 && D <= 64 ? 3 : sizeof(T) == 2 || D < 128 ? 2 : 1;
template <class T, int D>
constexpr int kQueryPerSimd = D <= 64 || (sizeof(T) == 2 && D == 96) ? 2 : 1;
// Rows of a tile of its keys: with 96 elements 32, which leaves registers for two wavefronts a SIMD, 710 to 743 us.
template <class T, int D>
constexpr int kQueryKeys = D == 96 ? 32 : kTile<T>;

template <class T, int D>
__device__ inline void forward_tile(const Attention& a, const Place& at, char (&lds)[2][2][Stage<T, D, kTile<T>, kThreads>::kBytes]) {
  using K = Kind<T, D>;
  constexpr int kKeys = kTile<T>, kSubs = kKeys / 32;
  using S = Stage<T, D, kKeys, kThreads>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = at.row + wave * 32, mine = first + (lane & 31);
  const T *k = head_of<T>(a.k, at.start, at.head / a.share), *v = head_of<T>(a.v, at.start, at.head / a.share);
  char* const room = lds[0][0];
  static_assert(sizeof lds >= Stage<T, D, kOwn, kThreads>::kBytes, "room for the workgroup's own rows");
  S ks(k, a.k.token, a.dim), vs(v, a.v.token, a.dim);
  u4 q[K::kParts];
  {
    const Own<T, D> mine(head_of<T>(a.q, at.start, at.head), a.q.token, at.row, at.len, a.dim);
    ks.load(0, at.len), vs.load(0, at.len);
    mine.read(room, q);
  }
  const int last = a.causal ? min(mine, at.len - 1) : at.len - 1;  // key that the lane's query sees
  const int keys = a.causal ? min(at.len, at.row + kOwn) : at.len;
  const int whole = (a.causal ? min(at.len, at.row + 1) : at.len) / kKeys * kKeys;  // keys below are seen by all queries
  f16v acc[D / 32];
#pragma unroll
  for (int b = 0; b < D / 32; ++b) acc[b] = (f16v)0.0f;
  // The exponents' base, of z log2 e, and the lane's keys' share of the sum.  The base follows the maximum only where that
  // has grown by more than 2^kGrowth, which the sums have room for.
  float top = -INFINITY, base = 0.0f, sum = 0.0f;
  // The next tile comes in two halves, its keys during the first half of this one and its values during the second.
  const auto turn = [&](int key, int buffer) { ks.store(lds[buffer ^ 1][0]), vs.load(key + kKeys, at.len); };
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
  const auto step = [&](int key, int buffer) {
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
      if (s == (kSubs - 1) / 2) turn(key, buffer);
      z = next;
    }
  };
  // The same for keys of which each query sees its own.
  const auto step_part = [&](int key, int buffer) {
#pragma unroll 1
    for (int s = 0; s < kSubs; ++s) {
      const int from = key + s * 32;
      if (from >= keys || (a.causal && from >= first + 32)) break;
      f16v z = scores<T, D>(lds[buffer][0], s * 32, q, (f16v)0.0f);
      const bool part = from + 31 > (a.causal ? min(first, at.len - 1) : at.len - 1);
      if (part)
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r] = from + row_in(r) <= last ? z[r] : -INFINITY;
      raise(z);
      soften(z);
      const typename K::Right p(z);
#pragma unroll
      for (int b = 0; b < D / 32; ++b) {
        if (part) K::template gather_part<1>(lds[buffer][1], s * 32, b, p, last - key, acc[b]);
        else K::gather(lds[buffer][1], s * 32, b, p, acc[b]);
      }
    }
  };
  ks.store(lds[0][0]), vs.store(lds[0][1]);
  __syncthreads();
  int key = 0, buffer = 0;
  for (; key < whole; key += kKeys, buffer ^= 1) {
    ks.load(key + kKeys, at.len);
    step(key, buffer);
    vs.store(lds[buffer ^ 1][1]);
    __syncthreads();
  }
  for (; key < keys; key += kKeys, buffer ^= 1) {
    ks.load(key + kKeys, at.len);
    step_part(key, buffer);
    turn(key, buffer);
    vs.store(lds[buffer ^ 1][1]);
    __syncthreads();
  }
  sum = halves_sum(sum);
  put_rows<T, D>(room, (T*)head_of<T>(a.out, at.start, at.head), a.out.token, first, at.len, a.dim, acc, 1.0f / sum);
  if (lane < 32 && mine < at.len) a.lse[at.head * a.tokens + at.start + mine] = (base + log2f(sum)) * kLn2;
}

template <class T, int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(kForwardPerSimd<T, D>, kForwardPerSimd<T, D>))) void forward_kernel(Attention a) {
  __shared__ __attribute__((aligned(16))) char lds[2][2][Stage<T, D, kTile<T>, kThreads>::kBytes];
  Place at;
  const Found found = place_of<kOwn, true>(a, a.heads, &at);
  if (found == kSequence) return forward_tile<T, D>(a, at, lds);
  if (found == kNone || !a.zero_q) return;
  over_rest<kOwn>(a, at, [&](int from, int to) {
    zero_rows((T*)head_of<T>(a.out, at.start, at.head), a.out.token, from, to, a.dim);
    zero_rows(a.lse + at.head * a.tokens + at.start, 1, from, to, 1);
  });
}

template <class T, int D>
__device__ inline void query_tile(const Attention& a, const Place& at, char (&lds)[2][2][Stage<T, D, kQueryKeys<T, D>, kThreads>::kBytes]) {
  using K = Kind<T, D>;
  constexpr int kKeys = kQueryKeys<T, D>, kSubs = kKeys / 32;
  using S = Stage<T, D, kKeys, kThreads>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = at.row + wave * 32, mine = first + (lane & 31);
  const bool there = mine < at.len;
  const T *k = head_of<T>(a.k, at.start, at.head / a.share), *v = head_of<T>(a.v, at.start, at.head / a.share);
  char* const room = lds[0][0];
  static_assert(sizeof lds >= Stage<T, D, kOwn, kThreads>::kBytes, "room for the workgroup's own rows");
  S ks(k, a.k.token, a.dim), vs(v, a.v.token, a.dim);
  u4 q[K::kParts], g[K::kParts];
  float delta = 0.0f;
  {
    const auto own = [&](const Rows& rows) { return Own<T, D>(head_of<T>(rows, at.start, at.head), rows.token, at.row, at.len, a.dim); };
    const auto sum = [&] {
#pragma unroll
      for (int c = 0; c < K::kParts; ++c) delta += K::dot(g[c], q[c]);
      delta = halves_sum(delta);
    };
    if constexpr (D > 96) {  // (where registers are short one after the other)
      own(a.out).read(room, q), own(a.dout).read(room, g);
      sum();
      own(a.q).read(room, q);
      ks.load(0, at.len), vs.load(0, at.len);
    } else {
      const Own<T, D> o = own(a.out), dout = own(a.dout), mine = own(a.q);
      o.read(room, q), dout.read(room, g);
      sum();
      ks.load(0, at.len), vs.load(0, at.len);
      mine.read(room, q);
    }
  }
  const int64_t stat = at.head * a.tokens + at.start + mine;
  const float lse2 = there ? a.lse[stat] * kLog2e : INFINITY;
  const int last = a.causal ? min(mine, at.len - 1) : at.len - 1;
  const int keys = a.causal ? min(at.len, at.row + kOwn) : at.len;
  const int whole = sizeof(T) == 2 ? (a.causal ? min(at.len, at.row + 1) : at.len) / kKeys * kKeys : 0;  // as in the forward pass
  // delta is dout . out of the rounded out, so it is off by up to 2^-8 of its terms, and ds_j by p_j times as much, which is more
  // than the roundings of ds and dq make.  But the sum of ds is zero: what it comes to instead tells how far delta is off.  The
  // pass by keys gets delta set right, and dq gives back that much of the keys' mean by p, a fourth product.
  // With it dq and dk of 8 x 1024 x 16 x 64, causal, are off by 0.0024 of their norm and by 0.0031 without, where the two
  // roundings alone make 0.0023; it is a third of this pass's work (8 x 1024 x 16 x 64 causal 48 to 59 us and 8192 x 16 x 128 740 to 1129 when it came, with clocks not yet
  // settled; 54 to 57 and 1047 to 1072 now).
  constexpr bool kRounded = sizeof(T) == 2, kAlone = kRounded && kQueryPerSimd<T, D> == 1;
  float off = 0.0f;
  f16v acc[D / 32], mean[kRounded ? D / 32 : 1];
#pragma unroll
  for (int b = 0; b < D / 32; ++b) acc[b] = (f16v)0.0f;
#pragma unroll
  for (int b = 0; b < (kRounded ? D / 32 : 1); ++b) mean[b] = (f16v)0.0f;
  const auto fetch = [&](int key) { ks.load(key, at.len), vs.load(key, at.len); };
  const auto keep = [&](int buffer) { ks.store(lds[buffer][0]), vs.store(lds[buffer][1]); };
  const auto step = [&](int buffer) {
#pragma unroll
    for (int s = 0; s < kSubs; ++s) {
      f16v z = scores<T, D>(lds[buffer][0], s * 32, q, (f16v)0.0f);
      f16v dp = (f16v)(-delta);
      if constexpr (kAlone) {
        // one wavefront a SIMD: the powers are taken while the matrix cores work on dp, and ds while they work on the mean
        // (8192 x 16 x 128 in 1129 us, 1277 in the order below, one run against the other)
        Parts<T, D> rows;
        rows.read(lds[buffer][1], s * 32);
        pin();
#pragma unroll
        for (int j = 0; j < K::kParts; ++j) {
          dp = K::multiply(rows.of[j], g[j], dp);
#pragma unroll
          for (int r = j * 16 / K::kParts; r < (j + 1) * 16 / K::kParts; ++r) z[r] = exp2_fast(fmaf(z[r], a.scale2, -lse2));
          pin();
        }
        const typename K::Right p(z);
        const typename K::Left columns(lds[buffer][0], s * 32);
        columns.gather(p, mean);
        z *= dp;
        off += sum_of(z);
        const typename K::Right ds(z);
        columns.gather(ds, acc);
        continue;
      }
      dp = scores<T, D>(lds[buffer][1], s * 32, g, dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = exp2_fast(fmaf(z[r], a.scale2, -lse2));
      if constexpr (kRounded) {
        const typename K::Right p(z);
        z *= dp;
        off += sum_of(z);
        const typename K::Right ds(z);
#pragma unroll
        for (int b = 0; b < D / 32; ++b) K::gather(lds[buffer][0], s * 32, b, ds, p, acc[b], mean[b]);
      } else {
        z *= dp;
        const typename K::Right ds(z);
#pragma unroll
        for (int b = 0; b < D / 32; ++b) K::gather(lds[buffer][0], s * 32, b, ds, acc[b]);
      }
    }
  };
  const auto step_part = [&](int key, int buffer) {
#pragma unroll 1
    for (int s = 0; s < kSubs; ++s) {
      const int from = key + s * 32;
      if (from >= keys || (a.causal && from >= first + 32)) break;
      f16v z = scores<T, D>(lds[buffer][0], s * 32, q, (f16v)0.0f);
      const f16v dp = scores<T, D>(lds[buffer][1], s * 32, g, (f16v)(-delta));
      const bool part = from + 31 > (a.causal ? min(first, at.len - 1) : at.len - 1);
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = exp2_fast(fmaf(z[r], a.scale2, -lse2));
      if constexpr (kRounded) {
        f16v p = z;
        if (part)
#pragma unroll
          for (int r = 0; r < 16; ++r) p[r] = from + row_in(r) <= last ? p[r] : 0.0f;
        const typename K::Right weights(p);
#pragma unroll
        for (int b = 0; b < D / 32; ++b) {
          if (part) K::template gather_part<1>(lds[buffer][0], s * 32, b, weights, last - key, mean[b]);
          else K::gather(lds[buffer][0], s * 32, b, weights, mean[b]);
        }
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = !part || from + row_in(r) <= last ? z[r] * dp[r] : 0.0f;
      if constexpr (kRounded) off += sum_of(z);
      const typename K::Right ds(z);
#pragma unroll
      for (int b = 0; b < D / 32; ++b) {
        if (part) K::template gather_part<1>(lds[buffer][0], s * 32, b, ds, last - key, acc[b]);
        else K::gather(lds[buffer][0], s * 32, b, ds, acc[b]);
      }
    }
  };
  ks.store(lds[0][0]), vs.store(lds[0][1]);
  __syncthreads();
  int key = 0, buffer = 0;
  for (; key < whole; key += kKeys, buffer ^= 1) {
    fetch(key + kKeys);
    step(buffer);
    keep(buffer ^ 1);
    __syncthreads();
  }
  for (; key < keys; key += kKeys, buffer ^= 1) {
    fetch(key + kKeys);
    step_part(key, buffer);
    keep(buffer ^ 1);
    __syncthreads();
  }
  off = halves_sum(off);
  if constexpr (kRounded)
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[b][r] = fmaf(-off, mean[b][r], acc[b][r]);
  if (there && lane < 32) a.delta[stat] = delta + off;
  put_rows<T, D>(room, (T*)head_of<T>(a.dq, at.start, at.head), a.dq.token, first, at.len, a.dim, acc, a.scale);
}

template <class T, int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(kQueryPerSimd<T, D>, kQueryPerSimd<T, D>))) void query_kernel(Attention a) {
  __shared__ __attribute__((aligned(16))) char lds[2][2][Stage<T, D, kQueryKeys<T, D>, kThreads>::kBytes];
  Place at;
  const Found found = place_of<kOwn, true>(a, a.heads, &at);
  if (found == kSequence) return query_tile<T, D>(a, at, lds);
  if (found == kNone || !a.zero_q) return;
  over_rest<kOwn>(a, at, [&](int from, int to) { zero_rows((T*)head_of<T>(a.dq, at.start, at.head), a.dq.token, from, to, a.dim); });
}

// ------------------------------------------------------------------------- host
template <class T, int D>
hipError_t queue(const Attention& a, bool backward, hipStream_t stream) {
  const dim3 block(kThreads), grid(static_cast<uint32_t>(a.tiles * a.heads));
  return backward ? launch(&query_kernel<T, D>, grid, block, stream, a) : launch(&forward_kernel<T, D>, grid, block, stream, a);
}
template <class T>
hipError_t queue(const Attention& a, bool backward, hipStream_t stream) {
  if (a.dim <= 32) return queue<T, 32>(a, backward, stream);
  if (a.dim <= 64) return queue<T, 64>(a, backward, stream);
  if (a.dim <= 96) return queue<T, 96>(a, backward, stream);
  return queue<T, 128>(a, backward, stream);
}

// Of the workspace: delta, and the parts' sums of dk and dv.  (As many tiles as there may be: whether offsets are given does not
// count.)
size_t delta_bytes(const daso_attention_args& s) { return (size_t(s.tokens) * size_t(s.heads) * sizeof(float) + 255) / 256 * 256; }
int32_t key_parts(const daso_attention_args& s) { return parts_of(s.tokens / kOwn + s.sequences + 1, s.kv_heads, s.heads / s.kv_heads); }
size_t backward_bytes(const daso_attention_args& s) {
  const size_t parts = size_t(key_parts(s));
  return delta_bytes(s) + (parts > 1 ? parts * 2 * size_t(s.tokens) * size_t(s.kv_heads) * size_t(s.dim) * sizeof(float) : 0);
}

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
  a.parts = key_parts(s), a.partial = reinterpret_cast<float*>(static_cast<char*>(s.workspace) + (backward ? delta_bytes(s) : 0));
  a.tiles = tiles_of<kOwn>(a), a.sorted = a.tiles * a.heads <= kFewTiles;
  hipError_t err = s.type == DASO_TYPE_BF16 ? queue<uint16_t>(a, backward, stream) : queue<float>(a, backward, stream);
  if (backward && err == hipSuccess) err = queue_keys(a, s.type, stream);
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
