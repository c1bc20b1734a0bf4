// What the attention kernels are made of: where a workgroup's rows lie, tiles of rows in LDS, and
// the two kinds of products with them.
//
// All products are made with the tile's rows as the left operand and 32 rows of the wavefront's own as the right one,
// which are its columns: C[i][j], j = lane % 32, of which a lane holds i = 8 (r / 4) + 4 (lane / 32) + r % 4 for
// r = 0..15.  So what a softmax reduces over lies in one lane and the one 32 above it, and values of C are at once in place as
// the right operand of a product that contracts over i: the order of the contraction is free, so the left operand
// is read in the order in which the lanes hold them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "daso_block_host.h"
#include "daso_planes.h"
#include "daso_product.h"

namespace daso {
namespace attention {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef u4 u4_any __attribute__((aligned(2)));
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

constexpr int kThreads = 256, kWaves = 4, kOwn = kWaves * 32;  // rows of a workgroup
template <class T>
constexpr int kTile = sizeof(T) == 2 ? 64 : 32;  // rows of a tile in LDS
using product::bhalf8;
using product::half4;

struct Rows {
  void* p;
  int64_t token, head;  // strides in elements
};

struct Attention {
  int64_t tokens;
  const int64_t* offsets;  // or null: one sequence of all tokens
  int32_t sequences, heads, kv_heads, share;  // share: query heads of a key head
  int32_t dim, causal, zero_q, zero_k, zero_v;  // zeros in rows of no sequence
  int32_t tiles, sorted;  // tiles: of a head, at most
  float scale, scale2;  // scale2 = scale * log2 e
  Rows q, k, v, out, dout, dq, dk, dv;
  float *lse, *delta;  // heads x tokens
  // Parts that the query heads of a key head are taken in by the pass by keys, where its tiles are few: their sums of dk and
  // dv, [part][dk, dv][token][key head][dim], are added by a kernel of their own.
  int32_t parts;
  float* partial;
};

// What a workgroup works on: rows `row`.. of the sequence of `len` tokens from `start` on.  Of rows in no sequence (kRest) those from
// `row` on, or, with `apart`, of all tokens' rows those in no sequence of every tile `apart` rows from the one before.
struct Place {
  int64_t start;
  int32_t len, row, head, apart;
};

__device__ inline int64_t read_lane(int64_t v, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(v), lane);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(v >> 32), lane);
  return static_cast<int64_t>(uint64_t(hi) << 32 | lo);
}

constexpr int kSorted = 32;  // sequences, at most, whose tiles are taken in the order of their work

// Workgroups of neighbouring numbers go to the eight XCDs in turn, and in an XCD to its parts.  Where the heads can be dealt to
// them evenly an XCD takes heads of its own, so that their keys stay in its L2.
//
// In causal sequences a tile's work is its place from the light end, which is the first tile of queries and the last one of
// keys.  With Attention::sorted, for launches of few tiles a CU, all tiles of the heads and of up to kSorted sequences come in the
// order of their work, the most first.  Else, whose keys would not fit the L2s together, head by head and sequence
// by sequence, from another tile on in each, so that no part of an XCD is dealt the heavy ones alone: 32 x 1024 tokens of 16 heads of
// 64 forward in 154 us, 182 where each sequence begins with its heaviest tile.
// kRest: rows in no sequence.  They are those behind the last one, a tile each for the workgroups that are left, or, where
// offsets begin later than at 0 or some pair is no sequence, all that these workgroups find between the sequences.  (One is left
// at least: n sequences apart from each other have no more than tokens / ROWS + n tiles.)
enum Found { kNone, kSequence, kRest };

// The 64 pairs of offsets from `base` on, a lane's as from..to: empty where a pair falls or leaves the tokens and, once some
// pair has (`odd`), where it begins before the end of one before it (the last is `end`), so that no two sequences share a row.
// Pairs that all ascend need no look at each other, which in every workgroup took 32 x 1024 tokens of 16 heads of 64 forward from
// 124 to 128 us.
struct Pairs {
  int64_t from, to;
  __device__ Pairs(const Attention& a, int base, bool& odd, int& end) {
    const int lane = threadIdx.x & 63;
    from = to = 0;
    if (base + lane < a.sequences) from = a.offsets[base + lane], to = a.offsets[base + lane + 1];
    const bool fits = from >= 0 && to >= from && to <= a.tokens;
    if (!fits) to = from = 0;
    if (__builtin_expect(!odd && !__any(!fits), 1)) return;
    // (up to the first pair that does not fit the offsets ascend)
    if (!odd) end = a.offsets[base] > a.offsets[0] ? static_cast<int>(a.offsets[base]) : 0;
    odd = true;
    int upto = to > from ? static_cast<int>(to) : 0;
    for (int s = 1; s < 64; s <<= 1) {
      const int v = __shfl_up(upto, s);
      if (lane >= s) upto = max(upto, v);
    }
    int before = __shfl_up(upto, 1);
    before = max(lane == 0 ? 0 : before, end);
    if (from < before) to = from = 0;
    end = max(end, __builtin_amdgcn_readlane(upto, 63));
  }
};

template <int ROWS, bool QUERIES>
__device__ inline Found place_of(const Attention& a, int heads, Place* at) {
  const int id = blockIdx.x;
  int index;
  if (heads % 8 == 0) {
    const int in = id >> 3, each = heads >> 3;
    const int by = a.sorted ? each : a.tiles, rest = in % by;
    at->head = (id & 7) * each + (a.sorted ? rest : in / by);
    index = a.sorted ? in / by : rest;
  } else {
    at->head = id % heads;
    index = id / heads;
  }
  const bool last_first = QUERIES && a.causal;
  if (a.offsets == nullptr) {
    at->start = 0, at->len = static_cast<int32_t>(a.tokens);
    const int tiles = (at->len + ROWS - 1) / ROWS;
    at->row = (last_first ? tiles - 1 - index : index) * ROWS;
    return index < tiles ? kSequence : kNone;
  }
  const int lane = threadIdx.x & 63;
  int before = 0, end = 0;
  bool odd = false;
  for (int base = 0; base < a.sequences; base += 64) {
    const Pairs pairs(a, base, odd, end);
    const int64_t from = pairs.from, to = pairs.to;
    const int mine = (static_cast<int>(to - from) + ROWS - 1) / ROWS;
    if (a.causal && a.sorted && a.sequences <= kSorted) {
      // A tile's work is its place from the light end of its sequence, 1, 2, ..  more[j]: the tiles of more work than lane +
      // 64 j.  The index-th tile is of the least work w that no more than index tiles exceed.
      int more[4] = {0, 0, 0, 0}, all = 0;
      bool small = true;
      for (int s = 0; s < a.sequences; ++s) {
        const int n = __builtin_amdgcn_readlane(mine, s);
        small &= n < 256, all += n;
#pragma unroll
        for (int j = 0; j < 4; ++j) more[j] += max(n - lane - 64 * j, 0);
      }
      if (small && index < all) {
        int w = 0, above = 0;
        bool found = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint64_t few = __ballot(more[j] <= index);
          if (!found && few != 0) {
            const int l = __builtin_ctzll(few);
            w = 64 * j + l, above = __builtin_amdgcn_readlane(more[j], l), found = true;
          }
        }
        // the (index - above)-th of the sequences that have such a tile
        const uint64_t have = __ballot(mine >= w);
        const int rank = __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(have >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(have), 0));
        const int l = __builtin_ctzll(__ballot(mine >= w && rank == index - above));
        at->start = read_lane(from, l), at->len = static_cast<int32_t>(read_lane(to, l) - at->start);
        at->row = (QUERIES ? w - 1 : __builtin_amdgcn_readlane(mine, l) - w) * ROWS;
        return kSequence;
      }
    }
    int upto = mine;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int v = __shfl_up(upto, s);
      if (lane >= s) upto += v;
    }
    const uint64_t found = __ballot(before + upto > index);
    if (found != 0) {
      const int l = __builtin_ctzll(found), tiles = __builtin_amdgcn_readlane(mine, l);
      at->start = read_lane(from, l), at->len = static_cast<int32_t>(read_lane(to, l) - at->start);
      const int tile = (index - before - (__builtin_amdgcn_readlane(upto, l) - tiles) + base + l) % tiles;
      at->row = (last_first ? tiles - 1 - tile : tile) * ROWS;
      return kSequence;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  odd |= a.offsets[0] != 0;
  at->start = odd ? 0 : a.offsets[a.sequences];
  at->len = static_cast<int32_t>(a.tokens - at->start);
  at->row = (index - before) * ROWS;
  at->apart = odd ? (a.tiles - before) * ROWS : 0;
  return at->row < at->len ? kRest : kNone;
}

// Calls zero(from, to) for runs of at most ROWS of the workgroup's rows in no sequence, counted from at.start.
template <int ROWS, class F>
__device__ inline void over_rest(const Attention& a, const Place& at, F zero) {
  if (at.apart == 0) return zero(at.row, min(at.row + ROWS, at.len));
  const auto gap = [&](int from, int to) {
    int row = at.row;
    if (from > row) row += (from - row) / at.apart * at.apart;
    for (; row < to; row += at.apart) zero(max(row, from), min(row + ROWS, to));
  };
  int done = 0, end = 0;
  bool odd = false;
  for (int base = 0; base < a.sequences; base += 64) {
    const Pairs pairs(a, base, odd, end);
    for (uint64_t left = __ballot(pairs.to > pairs.from); left != 0; left &= left - 1) {
      const int l = __builtin_ctzll(left);
      gap(done, __builtin_amdgcn_readlane(static_cast<int>(pairs.from), l));
      done = __builtin_amdgcn_readlane(static_cast<int>(pairs.to), l);
    }
  }
  gap(done, at.len);
}

__device__ inline float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }
// The value in this lane and in the one 32 away, in the same order in both.
struct Halves {
  float lower, upper;
  __device__ explicit Halves(float v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto both = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    lower = __builtin_bit_cast(float, static_cast<uint32_t>(both[0])), upper = __builtin_bit_cast(float, static_cast<uint32_t>(both[1]));
  }
};
__device__ inline float halves_sum(float v) {
  const Halves h(v);
  return h.lower + h.upper;
}
__device__ inline float halves_max(float v) {
  const Halves h(v);
  return fmaxf(h.lower, h.upper);
}

__device__ inline bool special(uint16_t, uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }
__device__ inline bool special(float, uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u; }

// A tree, so that no add waits for more than three others.
__device__ inline float sum_of(const f16v& v) {
  float s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = (v[i] + v[4 + i]) + (v[8 + i] + v[12 + i]);
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// The row (of 32) that value r of C belongs to in this lane.
__device__ inline int row_in(int r) { return 8 * (r / 4) + 4 * ((threadIdx.x & 63) >> 5) + r % 4; }

// NaN in values of C whose column sees what is no number in the contraction: `least` is, in lane i % 32, the signed place
// of row i's first such value (of the half of the contraction that the lane holds), `limit` the last one that the lane's column sees.
__device__ inline void spoil(int least, int limit, f16v& acc) {
  least = min(least, __shfl_xor(least, 32));
  const bool upper = (threadIdx.x & 32) != 0;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int lo = __builtin_amdgcn_readlane(least, 8 * (r / 4) + r % 4), hi = __builtin_amdgcn_readlane(least, 8 * (r / 4) + 4 + r % 4);
    acc[r] = (upper ? hi : lo) <= limit ? __builtin_nanf("") : acc[r];
  }
}

// What differs by type.  A part is 16 bytes of a row, a lane's share of a contraction over elements: half h of
// the lanes has elements 16 c + 8 h.. of a bf16 row in part c, which is one instruction, and elements h * D / 2 + 4 c.. of an
// fp32 row, which is four.
template <class T, int D>
struct Kind;

template <int D>
struct Kind<uint16_t, D> {
  static constexpr int kParts = D / 16;
  static constexpr int kPitch = D <= 64 ? 128 : 256;  // bytes from row to row in LDS
  // 16-byte piece c of row r lies in place c ^ mixed(r): 16 lanes that read one piece of 16 rows then touch all 64 banks
  // once, and so do 16 that read four neighbouring pieces of four rows.
  __device__ static int mixed(int r) { return kPitch == 128 ? ((r >> 1) & 1) << 2 | ((r >> 2) & 3) : (r & 3) << 2 | ((r >> 2) & 3); }
  __device__ static int piece_at(int row, int piece) { return row * kPitch + ((piece ^ mixed(row)) << 4); }
  __device__ static int part_at(int row, int c, int h) { return piece_at(row, 2 * c + h); }
  __device__ static int part_element(int c, int h) { return 16 * c + 8 * h; }
  __device__ static f16v multiply(u4 a, u4 b, f16v c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bhalf8, a), __builtin_bit_cast(bhalf8, b), c, 0, 0, 0);
  }
  __device__ static float dot(u4 a, u4 b) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sum = fmaf(__builtin_bit_cast(float, a[i] << 16), __builtin_bit_cast(float, b[i] << 16), sum);
      sum = fmaf(__builtin_bit_cast(float, a[i] & 0xffff0000u), __builtin_bit_cast(float, b[i] & 0xffff0000u), sum);
    }
    return sum;
  }
  // Values of C as a right operand: of each half of the 32 rows, rounded to nearest even.
  struct Right {
    bhalf8 of[2];
    __device__ explicit Right(const f16v& v) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) of[j][i] = static_cast<__bf16>(v[8 * j + i]);
    }
  };
  // Columns 32 b.. of rows 16 j.. as a left operand: two transposed reads of four rows each.
  __device__ static bhalf8 turned(const char* tile, int row, int b, int j) {
    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int r = row + 16 * j + 4 * h + ((lane & 15) >> 2), piece = 4 * b + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
    const int in = (lane & 1) * 8;
    const half4 x = product::read_turned(tile + piece_at(r, piece) + in), y = product::read_turned(tile + piece_at(r + 8, piece) + in);
    return __builtin_bit_cast(bhalf8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  // acc += (columns 32 b.. of 32 rows)^T right
  __device__ static void gather(const char* tile, int row, int b, const Right& right, f16v& acc) {
#pragma unroll
    for (int j = 0; j < 2; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(turned(tile, row, b, j), right.of[j], acc, 0, 0, 0);
  }
  // All columns of 32 rows, for several right operands one after the other.
  struct Left {
    bhalf8 of[D / 32][2];
    __device__ Left(const char* tile, int row) {
#pragma unroll
      for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int j = 0; j < 2; ++j) of[b][j] = turned(tile, row, b, j);
    }
    __device__ void gather(const Right& right, f16v (&acc)[D / 32]) const {
#pragma unroll
      for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(of[b][j], right.of[j], acc[b], 0, 0, 0);
    }
  };
  // The same for two right operands at a time.
  __device__ static void gather(const char* tile, int row, int b, const Right& right, const Right& other, f16v& acc, f16v& more) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const bhalf8 left = turned(tile, row, b, j);
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(left, right.of[j], acc, 0, 0, 0);
      more = __builtin_amdgcn_mfma_f32_32x32x16_bf16(left, other.of[j], more, 0, 0, 0);
    }
  }
  // The same where a column sees row i only if SIGN * i <= limit: what is no number in a row counts only in columns that see it.
  template <int SIGN>
  __device__ static void gather_part(const char* tile, int row, int b, const Right& right, int limit, f16v& acc) {
    bhalf8 left[2];
    bool any = false;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      left[j] = turned(tile, row, b, j);
      const u4 words = __builtin_bit_cast(u4, left[j]);
#pragma unroll
      for (int i = 0; i < 4; ++i) any |= special(uint16_t(0), words[i]);
    }
    int least = INT32_MAX;  // SIGN * row of the element's first such value
    const bool odd = __any(any);
    if (__builtin_expect(odd, 0)) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        u4 words = __builtin_bit_cast(u4, left[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = row + 16 * j + row_in(4 * (i / 2) + i % 2 * 2);
          const uint32_t w = words[i];
          if ((w & 0x7f80u) == 0x7f80u) words[i] &= 0xffff0000u, least = min(least, SIGN * r);
          if ((w & 0x7f800000u) == 0x7f800000u) words[i] &= 0xffffu, least = min(least, SIGN * (r + 1));
        }
        left[j] = __builtin_bit_cast(bhalf8, words);
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(left[j], right.of[j], acc, 0, 0, 0);
    if (__builtin_expect(odd, 0)) spoil(least, limit, acc);
  }
};

template <int D>
struct Kind<float, D> {
  static constexpr int kParts = D / 8;
  static constexpr int kPitch = D * 4 + 16;
  __device__ static int piece_at(int row, int piece) { return row * kPitch + piece * 16; }
  __device__ static int part_at(int row, int c, int h) { return row * kPitch + h * (D * 2) + c * 16; }
  __device__ static int part_element(int c, int h) { return h * (D / 2) + 4 * c; }
  __device__ static f16v multiply(u4 a, u4 b, f16v c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = a[i], y = b[i];
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__builtin_bit_cast(float, x), __builtin_bit_cast(float, y), c, 0, 0, 0);
    }
    return c;
  }
  __device__ static float dot(u4 a, u4 b) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t x = a[i], y = b[i];
      sum = fmaf(__builtin_bit_cast(float, x), __builtin_bit_cast(float, y), sum);
    }
    return sum;
  }
  struct Right {
    f16v of;
    __device__ explicit Right(const f16v& v) : of(v) {}
  };
  __device__ static float turned(const char* tile, int row, int b, int r) {
    const int lane = threadIdx.x & 63;
    return *(const float*)(tile + (row + 8 * (r / 4) + 4 * (lane >> 5) + r % 4) * kPitch + (32 * b + (lane & 31)) * 4);
  }
  __device__ static void gather(const char* tile, int row, int b, const Right& right, f16v& acc) {
#pragma unroll
    for (int r = 0; r < 16; ++r) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(turned(tile, row, b, r), right.of[r], acc, 0, 0, 0);
  }
  template <int SIGN>
  __device__ static void gather_part(const char* tile, int row, int b, const Right& right, int limit, f16v& acc) {
    int least = INT32_MAX;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float v = turned(tile, row, b, r);
      const bool odd = special(0.0f, __builtin_bit_cast(uint32_t, v));
      least = min(least, odd ? SIGN * (row + row_in(r)) : INT32_MAX);
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(odd ? 0.0f : v, right.of[r], acc, 0, 0, 0);
    }
    if (__builtin_expect(__any(least != INT32_MAX), 0)) spoil(least, limit, acc);
  }
};

// Rows `row`.. of a sequence of `len`, at most ROWS: p is its row 0.  Reads beyond them, and at kNowhere, give zeros.
constexpr uint32_t kNowhere = 0x80000000u;
template <int ROWS, class T>
__device__ inline __amdgpu_buffer_rsrc_t window(const T* p, int64_t stride, int row, int len, int dim) {
  const int rows = max(min(len - row, ROWS), 0);
  const int bytes = rows == 0 ? 0 : ((rows - 1) * static_cast<int>(stride) + dim) * static_cast<int>(sizeof(T));
  return __builtin_amdgcn_make_buffer_rsrc((void*)(p + row * stride), 0, bytes, 0x00027000);
}
__device__ inline u4 read16(__amdgpu_buffer_rsrc_t from, uint32_t at) { return __builtin_amdgcn_raw_buffer_load_b128(from, at, 0, 0); }

// ROWS rows of a head on their way to LDS: loaded while the tile before is worked on, written after it.  Rows from `len`
// on and elements from `dim` on are zeros.
template <class T, int D, int ROWS, int THREADS>
struct Stage {
  using K = Kind<T, D>;
  // Pieces of 16 bytes a row, and threads across it.  A thread's pieces are whole rows apart: it has one place, and a window of its
  // own (in scalar registers) for each piece.
  static constexpr int kPieces = D * sizeof(T) / 16, kAcross = kPieces == 12 ? 16 : kPieces == 24 ? 32 : kPieces;
  static constexpr int kRows = THREADS / kAcross, kEach = ROWS / kRows;
  static constexpr int kBytes = ROWS * K::kPitch;
  static_assert(THREADS % kAcross == 0 && ROWS % kRows == 0, "every thread has as many pieces");
  const T* p;  // row 0 of the sequence
  int64_t stride;
  int dim;
  uint32_t from;
  u4 v[kEach];
  __device__ Stage(const T* p, int64_t stride, int dim) : p(p), stride(stride), dim(dim) {
    const int r = threadIdx.x / kAcross, c = threadIdx.x % kAcross * int(16 / sizeof(T));
    from = c < dim ? (r * static_cast<uint32_t>(stride) + c) * uint32_t(sizeof(T)) : kNowhere;
  }
  __device__ void load(int row, int len) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) v[i] = read16(window<kRows>(p, stride, row + i * kRows, len, dim), from);
  }
  __device__ void store(char* lds) const {
    const int r = threadIdx.x / kAcross, c = threadIdx.x % kAcross;
    if (kPieces != kAcross && c >= kPieces) return;
#pragma unroll
    for (int i = 0; i < kEach; ++i) *(u4*)(lds + K::piece_at(r + i * kRows, c)) = v[i];
  }
};

// A workgroup's kOwn rows come and go through LDS, by whole lines: a lane's own 16 bytes of 32 rows at a time would ask
// for each line four times or more.  `lds` has room for kOwn rows.
template <class T, int D>
struct Own {
  using K = Kind<T, D>;
  Stage<T, D, kOwn, kThreads> rows;
  __device__ Own(const T* p, int64_t stride, int row, int len, int dim) : rows(p, stride, dim) { rows.load(row, len); }
  // The lane's parts of its row.  All wavefronts take part; nobody uses `lds` before or after without a meeting.
  __device__ void read(char* lds, u4 (&parts)[K::kParts]) const {
    rows.store(lds);
    __syncthreads();
    const int own = (threadIdx.x >> 6) * 32 + (threadIdx.x & 31), h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int c = 0; c < K::kParts; ++c) parts[c] = *(const u4*)(lds + K::part_at(own, c, h));
    __syncthreads();
  }
};

// Four neighbouring elements of a row in LDS.
__device__ inline void keep4(uint16_t* p, float a, float b, float c, float d) { *(us4*)p = us4{to_bf16(a), to_bf16(b), to_bf16(c), to_bf16(d)}; }
__device__ inline void keep4(float* p, float a, float b, float c, float d) { *(f4v*)p = f4v{a, b, c, d}; }

// A wavefront's 32 rows of sums, times `factor`, rounded once: p is row 0 of the sequence, `first` the wavefront's first row.
template <class T, int D>
__device__ inline void put_rows(char* lds, T* p, int64_t stride, int first, int len, int dim, const f16v (&acc)[D / 32], float factor) {
  using K = Kind<T, D>;
  constexpr int kPieces = D * sizeof(T) / 16, kEach = 16 / sizeof(T);
  const int lane = threadIdx.x & 63, h = lane >> 5, wave = threadIdx.x >> 6;
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int e = 32 * b + 8 * g + 4 * h;
      keep4((T*)(lds + K::piece_at(wave * 32 + (lane & 31), e / kEach)) + e % kEach, acc[b][4 * g] * factor, acc[b][4 * g + 1] * factor,
            acc[b][4 * g + 2] * factor, acc[b][4 * g + 3] * factor);
    }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int i = 0; i < 32 * kPieces / 64; ++i) {
    const int id = lane + i * 64, r = id / kPieces, c = id % kPieces;
    const u4 v = *(const u4*)(lds + K::piece_at(wave * 32 + r, c));
    if (first + r < len && c * kEach < dim) *(u4_any*)(p + (first + r) * stride + c * kEach) = v;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// Nothing is moved across by the compiler.
__device__ inline void pin() { __builtin_amdgcn_sched_barrier(0); }

// A lane's parts of 32 rows of a tile.
template <class T, int D>
struct Parts {
  u4 of[Kind<T, D>::kParts];
  __device__ void read(const char* tile, int row) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < Kind<T, D>::kParts; ++i) of[i] = *(const u4*)(tile + Kind<T, D>::part_at(row + (lane & 31), i, lane >> 5));
  }
};

// C of 32 rows of a tile and the wavefront's columns.
template <class T, int D>
__device__ inline f16v scores(const char* tile, int row, const u4 (&own)[Kind<T, D>::kParts], f16v c) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < Kind<T, D>::kParts; ++i)
    c = Kind<T, D>::multiply(*(const u4*)(tile + Kind<T, D>::part_at(row + (lane & 31), i, lane >> 5)), own[i], c);
  return c;
}

// Four neighbouring elements of a row.
__device__ inline void put4(uint16_t* p, float a, float b, float c, float d) {
  typedef us4 us4_any __attribute__((aligned(2)));
  *(us4_any*)p = us4{to_bf16(a), to_bf16(b), to_bf16(c), to_bf16(d)};
}
__device__ inline void put4(float* p, float a, float b, float c, float d) { *(f4v_any*)p = f4v{a, b, c, d}; }

// A lane's sums of its own row, in 32 bits and by itself.
template <int D>
__device__ inline void put_own(float* row, const f16v (&acc)[D / 32], float factor, int dim) {
  const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      if (32 * b + 8 * g < dim)
        put4(row + 32 * b + 8 * g + 4 * h, acc[b][4 * g] * factor, acc[b][4 * g + 1] * factor, acc[b][4 * g + 2] * factor,
             acc[b][4 * g + 3] * factor);
}

// Zeros in rows from..to.
template <class T>
__device__ inline void zero_rows(T* p, int64_t stride, int from, int to, int dim) {
  for (int i = threadIdx.x; i < (to - from) * dim; i += kThreads) p[(from + i / dim) * stride + i % dim] = T(0);
}

template <class T>
__device__ inline const T* head_of(const Rows& r, int64_t start, int head) {
  return (const T*)r.p + start * r.token + head * r.head;
}

// Tiles of a head, at most.
template <int ROWS>
inline int32_t tiles_of(const Attention& a) {
  return static_cast<int32_t>(a.offsets != nullptr ? a.tokens / ROWS + a.sequences + 1 : (a.tokens + ROWS - 1) / ROWS);
}
constexpr int32_t kFewTiles = 2048;  // Attention::sorted: up to eight a CU

// The backward pass by keys (daso_attention_keys.hip), after the one by queries; and into how many parts it goes.
constexpr int kKeyTiles = 512;  // workgroups that make parts needless: two a CU
inline int32_t parts_of(int64_t tiles, int32_t kv_heads, int32_t share) {
  int32_t parts = 1;
  while (parts < share && (share % parts != 0 || tiles * kv_heads * parts < kKeyTiles)) ++parts;
  return parts;
}
hipError_t queue_keys(const Attention& a, int32_t type, hipStream_t stream);

}  // namespace attention
}  // namespace daso
