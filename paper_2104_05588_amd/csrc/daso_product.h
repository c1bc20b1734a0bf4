// Matrix products of 16-bit planes on the matrix cores: C = sum over segments of
// A_s B_s^T, A with its contraction contiguous and B either so or turned (as the rows of
// B_s^T), 32-bit sums, and an epilogue that takes C in blocks of 64 x 32 while it is still
// in registers.
//
// A value that needs more than 11 bits of significand is held as two binary16 planes,
// hi + lo (22 bits), and a product of such values as the segments hi hi, hi lo, lo hi;
// what is left out is below 2^-22 of the product of the magnitudes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "daso_train_host.h"

namespace daso {
namespace product {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef __bf16 bhalf8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int kMaxSegments = 3;
constexpr int kStepElems = 64;     // contraction elements a step: 128 bytes of a row, one cache line
constexpr int kLeastSteps = 2;     // the pipeline's depth: a product takes at least this many steps
constexpr int kBlockRows = 64, kBlockCols = 32;  // what an epilogue is handed at a time
// LDS of a wavefront's own for its epilogue: a block in 32 bits, or two planes of it in 16.
constexpr int kStagePlane = kBlockRows * kBlockCols * 2 + (kBlockRows / 8) * 16;
constexpr int kWaveStage = 2 * kStagePlane;
static_assert(kWaveStage >= kBlockRows * kBlockCols * 4, "a staged block fits");
constexpr int kMaxProblems = 8;               // products of one launch

// Operands: rows of `ld` elements, 16-byte aligned, ld a multiple of 8 and at most host::kMaxLd, of which the first
// steps * 64 are contracted (zeros beyond the true length).  Rows from M (N) on are not
// read: a tile that reaches past them reads the last row again, and its epilogue leaves
// what comes of it.  A turned B has steps * 64 rows, which are contracted, of N values; N is a multiple of 8.
struct Args {
  const void* a[kMaxSegments];
  const void* b[kMaxSegments];
  int64_t lda, ldb, batch_a, batch_b;  // in elements
  int32_t segments, steps;             // steps of 64 a segment
  int32_t M, N;
  int32_t tiles_m, tiles_n;            // tiles_m x tiles_n, or with tri the tiles on and below the diagonal
  int32_t tri;
  int32_t batch;
};

inline int64_t tile_count(const Args& p) {
  const int64_t per = p.tri ? int64_t(p.tiles_m) * (p.tiles_m + 1) / 2 : int64_t(p.tiles_m) * p.tiles_n;
  return per * p.batch;
}

#if defined(__HIP_DEVICE_COMPILE__) || defined(__HIPCC__)

#define DASO_LDS(p) ((__attribute__((address_space(3))) void*)(p))
#define DASO_GLOBAL(p) ((const __attribute__((address_space(1))) void*)(p))

template <bool BF16>
__device__ inline f4 mfma(half8 a, half8 b, f4 c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bhalf8, a), __builtin_bit_cast(bhalf8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// The thread's number, opaque to the compiler: what follows from it is worked out where it is
// used, and not kept in registers over the products (where it would not fit).
__device__ inline int thread_here() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

template <int N>
__device__ inline void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ inline void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// The workgroup meets; nothing is moved across by the compiler.
__device__ inline void meet() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
}

struct Place {
  int tm, tn, batch;
};

// The tile `id` of a product.  Tiles are counted in bands of four tile rows, so that the
// rows and columns that neighbouring tiles read stay in an L2.
__device__ inline Place place_of(const Args& p, int id) {
  Place at;
  const uint32_t per = static_cast<uint32_t>(p.tri ? p.tiles_m * (p.tiles_m + 1) / 2 : p.tiles_m * p.tiles_n);
  at.batch = static_cast<int>(static_cast<uint32_t>(id) / per);
  const int t = id - at.batch * static_cast<int>(per);
  if (p.tri) {
    int i = static_cast<int>((sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
    while (i * (i + 1) / 2 > t) --i;
    while ((i + 1) * (i + 2) / 2 <= t) ++i;
    at.tm = __builtin_amdgcn_readfirstlane(i);
    at.tn = t - at.tm * (at.tm + 1) / 2;
  } else {
    constexpr int kBand = 4;
    const int band = static_cast<int>(static_cast<uint32_t>(t) / static_cast<uint32_t>(kBand * p.tiles_n)), first = band * kBand;
    const uint32_t rows = static_cast<uint32_t>(min(p.tiles_m - first, kBand)), in = static_cast<uint32_t>(t - first * p.tiles_n);
    at.tm = first + static_cast<int>(in % rows);
    at.tn = static_cast<int>(in / rows);
  }
  return at;
}

// The operand's bytes at step t of all segments, whose steps are `step` bytes apart.
__device__ inline const char* step_of(const char* s0, const char* s1, const char* s2, int t, int steps, int64_t step) {
  const char* base = s0;
  if (t >= steps) {
    base = s1;
    t -= steps;
    if (t >= steps) {
      base = s2;
      t -= steps;
    }
  }
  return base + t * step;
}

// LDS holds operand rows of 128 bytes; the 16-byte piece c of row r lies in place
// c ^ (r / 2 % 8) of the row, so that 16 lanes that read one piece of 16 rows touch all
// 64 banks once.  Loads go straight to LDS, in lane order, so it is the source address
// that is permuted: a wavefront's load still takes whole lines.
//
// A turned B lies in LDS as it does in memory, 64 rows of 128 values a half, and is read with the
// transposing LDS loads: 16 lanes read 16 neighbouring values of 4 rows, and lane l gets column l
// of them.  Its 16-byte piece c of row r lies in place c ^ turned_place(r), so that the 32 pieces
// which the four groups of 16 lanes read at once take all banks evenly.  (Writing such an operand
// turned as a plane of its own instead cost 2 to 5 % of the whole: 4384 us against 4253 for the loss and gradients
// of 8192 x 50257 x 1024, 21.2 ms against 20.7 for a model's update of 302M elements.)
__device__ inline int turned_place(int row) { return (row & 3) << 1 | ((row >> 3) & 1) << 3; }

typedef short short4v __attribute__((ext_vector_type(4)));
__device__ inline half4 read_turned(const char* p) {
  return __builtin_bit_cast(half4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)DASO_LDS(p)));
}
// Four operands, each of eight rows' values of a column: 4 rows from a place on and the 4 below them.
// In one block with its wait: before the builtin the compiler would also wait for all loads that go
// to LDS, which here are for later steps.
__device__ inline void read_operands(const char* p0, const char* p1, const char* p2, const char* p3, half8 (&to)[4]) {
  const auto at = [](const char* p) { return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(DASO_LDS(p))); };
  half4 v[8];
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\t"
      "ds_read_b64_tr_b16 %1, %8 offset:1024\n\t"
      "ds_read_b64_tr_b16 %2, %9\n\t"
      "ds_read_b64_tr_b16 %3, %9 offset:1024\n\t"
      "ds_read_b64_tr_b16 %4, %10\n\t"
      "ds_read_b64_tr_b16 %5, %10 offset:1024\n\t"
      "ds_read_b64_tr_b16 %6, %11\n\t"
      "ds_read_b64_tr_b16 %7, %11 offset:1024\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
      : "v"(at(p0)), "v"(at(p1)), "v"(at(p2)), "v"(at(p3))
      : "memory");
#pragma unroll
  for (int i = 0; i < 4; ++i) to[i] = __builtin_shufflevector(v[2 * i], v[2 * i + 1], 0, 1, 2, 3, 4, 5, 6, 7);
}

// 256 x 256 a workgroup of 8 wavefronts.  A step's operands are four pieces of 128 rows
// (A0 A1 B0 B1, 16 KB each, two steps in LDS), and a step is four phases, one quarter
// (128 x 128) of the tile each, in an order in which a phase changes one piece only.  A piece
// is loaded again, for the step after the next, two phases after its last read: six
// phases before it is wanted.  Each phase is a part that reads LDS and issues loads and a
// part of 16 matrix instructions, and the two wavefronts of a SIMD take them in
// opposite turns, one barrier apart, so that one of them is always computing.
// Measured on 8192^3: 2285 cycles a step where the matrix instructions alone take 2048.  In
// time the clock decides: under this load it falls to 1.4 to 1.6 GHz, for the power that
// the matrix cores draw.  16x16x32 instructions draw less than 32x32x16 ones (registers
// only: 1950 and 1670 TFLOP/s), and the whole runs at 1235 TFLOP/s, with 32x32x16 at 1040.
struct Tile256 {
  static constexpr int kRows = 256, kCols = 256, kThreads = 512, kLds = 131072;
  static_assert(kLds >= 8 * kWaveStage, "the epilogue's LDS");
  static constexpr int kBlocks = 4;  // blocks of 64 x 32 a wavefront
  static constexpr int kOccupancy = 2;

  __device__ static void block_at(int wave, int b, int* row, int* col) {
    *row = (b >> 1) * 128 + (wave >> 2) * 64;
    *col = (b & 1) * 128 + (wave & 3) * 32;
  }

  template <bool BF16, bool TURNED>
  __device__ static void run(const Args& p, const Place& at, int from, int to, char* lds, f4 (&acc)[kBlocks][8]) {
    const int lane = thread_here() & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t skip_a = (at.batch * p.batch_a + int64_t(at.tm) * kRows * p.lda) * 2;
    const int64_t skip_b = (at.batch * p.batch_b + int64_t(at.tn) * kCols * (TURNED ? 1 : p.ldb)) * 2;
    const int64_t step_b = TURNED ? p.ldb * 128 : 128;
    const char *a0 = (const char*)p.a[0] + skip_a, *a1 = (const char*)p.a[1] + skip_a, *a2 = (const char*)p.a[2] + skip_a;
    const char *b0 = (const char*)p.b[0] + skip_b, *b1 = (const char*)p.b[1] + skip_b, *b2 = (const char*)p.b[2] + skip_b;
    const int last_a = min(kRows, p.M - at.tm * kRows) - 1, last_b = min(kCols, p.N - at.tn * kCols) - 1;
    const int steps = p.steps;
    uint32_t from_a[2][2], from_b[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = (wave * 2 + j) * 8 + (lane >> 3), c = ((lane & 7) ^ ((r >> 1) & 7)) * 16;
        from_a[h][j] = static_cast<uint32_t>(min(h * 128 + r, last_a)) * (static_cast<uint32_t>(p.lda) * 2) + c;
        if constexpr (TURNED) {
          const int k = (wave * 2 + j) * 4 + (lane >> 4), col = h * 128 + ((lane & 15) ^ turned_place(k)) * 8;
          from_b[h][j] = static_cast<uint32_t>(k) * (static_cast<uint32_t>(p.ldb) * 2) + min(col, last_b - 7) * 2;
        } else {
          from_b[h][j] = static_cast<uint32_t>(min(h * 128 + r, last_b)) * (static_cast<uint32_t>(p.ldb) * 2) + c;
        }
      }
    auto load_a = [&](int t, int h) {
      char* dst = lds + (t & 1) * 65536 + h * 16384 + wave * 2048;
      const char* g = step_of(a0, a1, a2, t, steps, 128);
#pragma unroll
      for (int j = 0; j < 2; ++j)
        __builtin_amdgcn_global_load_lds(DASO_GLOBAL(g + from_a[h][j]), DASO_LDS(dst + j * 1024), 16, 0, 0);
    };
    auto load_b = [&](int t, int h) {
      char* dst = lds + (t & 1) * 65536 + 32768 + h * 16384 + wave * 2048;
      const char* g = step_of(b0, b1, b2, t, steps, step_b);
#pragma unroll
      for (int j = 0; j < 2; ++j)
        __builtin_amdgcn_global_load_lds(DASO_GLOBAL(g + from_b[h][j]), DASO_LDS(dst + j * 1024), 16, 0, 0);
    };
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[i][j] = (f4)0.0f;
    const int wm = wave >> 2, wn = wave & 3, r16 = lane & 15, kq = lane >> 4;
    half8 a[8], bl[4], br[4], bnext[4];
    int at_a[2], at_b[2];  // by kk; of a turned B by the 16 columns
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const int c = ((kk * 4 + kq) ^ ((r16 >> 1) & 7)) * 16;
      at_a[kk] = (wm * 64 + r16) * 128 + c;
      const int row = kq * 8 + (r16 >> 2), piece = wn * 4 + kk * 2 + ((r16 & 3) >> 1);
      if constexpr (TURNED) at_b[kk] = 32768 + row * 256 + (piece ^ turned_place(row)) * 16 + (r16 & 1) * 8;
      else at_b[kk] = 32768 + (wn * 32 + r16) * 128 + c;
    }
    auto read_a = [&](int t, int h) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          a[kk * 4 + i] = *(const half8*)(lds + (t & 1) * 65536 + at_a[kk] + h * 16384 + i * 2048);
    };
    auto read_b = [&](int t, int h, half8 (&b)[4]) {
      const char* from = lds + (t & 1) * 65536 + h * 16384;
      if constexpr (TURNED) {
        read_operands(from + at_b[0], from + at_b[1], from + at_b[0] + 8192, from + at_b[1] + 8192, b);
      } else {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int j = 0; j < 2; ++j) b[kk * 2 + j] = *(const half8*)(from + at_b[kk] + j * 2048);
      }
    };
    // the operands are handed over as (b, a), so that a lane holds four neighbouring
    // columns of one row of C
    auto compute = [&](f4* c, const half8* b) {
      wait_lds();
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) c[i * 2 + j] = mfma<BF16>(b[kk * 2 + j], a[kk * 4 + i], c[i * 2 + j]);
      __builtin_amdgcn_s_setprio(0);
      meet();
    };
    load_b(from, 0), load_a(from, 0), load_b(from, 1), load_a(from, 1);
    load_b(from + 1, 0), load_a(from + 1, 0), load_b(from + 1, 1);
    wait_loads<10>();
    meet();
    if (wm == 1) meet();
    read_b(from, 0, bnext);
    // kLeft: steps after this one, 2 for two or more.  Each wait leaves in flight what was
    // issued after the piece that the next phase reads.
    auto step = [&](int k, auto left) {
      constexpr int kLeft = decltype(left)::value;
      read_a(k, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) bl[i] = bnext[i];
      if constexpr (kLeft > 0) load_a(k + 1, 1), wait_loads<10>();
      else wait_loads<2>();
      meet();
      compute(acc[0], bl);
      if constexpr (kLeft > 1) load_b(k + 2, 0);
      read_b(k, 1, br);
      if constexpr (kLeft > 1) wait_loads<10>();
      else wait_loads<kLeft == 1 ? 8 : 0>();
      meet();
      compute(acc[1], br);
      read_a(k, 1);
      if constexpr (kLeft > 1) load_a(k + 2, 0), wait_loads<10>();
      else if constexpr (kLeft == 1) wait_loads<6>();
      meet();
      compute(acc[3], br);
      if constexpr (kLeft > 1) load_b(k + 2, 1);
      if constexpr (kLeft > 0) read_b(k + 1, 0, bnext);
      if constexpr (kLeft > 1) wait_loads<10>();
      else if constexpr (kLeft == 1) wait_loads<4>();
      meet();
      compute(acc[2], bl);
    };
    int k = from;
    for (; k + 2 < to; ++k) step(k, Left<2>());
    step(k, Left<1>());
    step(k + 1, Left<0>());
    if (wm == 0) meet();
  }

 private:
  template <int N>
  struct Left {
    static constexpr int value = N;
  };
};

// 128 x 128 a workgroup of 4 wavefronts, for results too small to give every CU a larger tile.  Two
// steps in LDS, two workgroups a CU, which hide each other's waits; a step's second half runs
// while the next step's first operands are read.  (A ring of four steps, with one workgroup a CU, was
// no faster where there are few: 33 us against 27 for 16 tiles of 32 steps, which wait for what one
// CU gets of memory.)
struct Tile128 {
  static constexpr int kRows = 128, kCols = 128, kThreads = 256, kLds = 65536;
  static constexpr int kBlocks = 2;
  static constexpr int kOccupancy = 2;
  static_assert(kLds >= 4 * kWaveStage, "the epilogue's LDS");

  __device__ static void block_at(int wave, int b, int* row, int* col) {
    *row = (wave >> 1) * 64;
    *col = (wave & 1) * 64 + b * 32;
  }

  template <bool BF16, bool TURNED>
  __device__ static void run(const Args& p, const Place& at, int from, int to, char* lds, f4 (&acc)[kBlocks][8]) {
    const int lane = thread_here() & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t skip_a = (at.batch * p.batch_a + int64_t(at.tm) * kRows * p.lda) * 2;
    const int64_t skip_b = (at.batch * p.batch_b + int64_t(at.tn) * kCols * (TURNED ? 1 : p.ldb)) * 2;
    const int64_t step_b = TURNED ? p.ldb * 128 : 128;
    const char *a0 = (const char*)p.a[0] + skip_a, *a1 = (const char*)p.a[1] + skip_a, *a2 = (const char*)p.a[2] + skip_a;
    const char *b0 = (const char*)p.b[0] + skip_b, *b1 = (const char*)p.b[1] + skip_b, *b2 = (const char*)p.b[2] + skip_b;
    const int last_a = min(kRows, p.M - at.tm * kRows) - 1, last_b = min(kCols, p.N - at.tn * kCols) - 1;
    const int steps = p.steps;
    uint32_t from_a[4], from_b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = (wave * 4 + j) * 8 + (lane >> 3), c = ((lane & 7) ^ ((r >> 1) & 7)) * 16;
      from_a[j] = static_cast<uint32_t>(min(r, last_a)) * (static_cast<uint32_t>(p.lda) * 2) + c;
      if constexpr (TURNED) {
        const int k = (wave * 4 + j) * 4 + (lane >> 4), col = ((lane & 15) ^ turned_place(k)) * 8;
        from_b[j] = static_cast<uint32_t>(k) * (static_cast<uint32_t>(p.ldb) * 2) + min(col, last_b - 7) * 2;
      } else {
        from_b[j] = static_cast<uint32_t>(min(r, last_b)) * (static_cast<uint32_t>(p.ldb) * 2) + c;
      }
    }
    auto load = [&](int t) {
      char* dst = lds + (t & 1) * 32768 + wave * 4096;
      const char *ga = step_of(a0, a1, a2, t, steps, 128), *gb = step_of(b0, b1, b2, t, steps, step_b);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        __builtin_amdgcn_global_load_lds(DASO_GLOBAL(ga + from_a[j]), DASO_LDS(dst + j * 1024), 16, 0, 0);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        __builtin_amdgcn_global_load_lds(DASO_GLOBAL(gb + from_b[j]), DASO_LDS(dst + 16384 + j * 1024), 16, 0, 0);
    };
#pragma unroll
    for (int i = 0; i < kBlocks; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[i][j] = (f4)0.0f;
    const int wm = wave >> 1, wn = wave & 1, r16 = lane & 15, kq = lane >> 4;
    half8 a[2][4], b[2][4];
    auto read = [&](int t, int kk) {
      const int c = ((kk * 4 + kq) ^ ((r16 >> 1) & 7)) * 16;
      const char* s = lds + (t & 1) * 32768;
#pragma unroll
      for (int i = 0; i < 4; ++i) a[kk][i] = *(const half8*)(s + (wm * 64 + r16) * 128 + c + i * 2048);
      if constexpr (TURNED) {
        const int row = kq * 8 + (r16 >> 2), piece = (wn * 8 + ((r16 & 3) >> 1)) ^ turned_place(row);
        const char* from = s + 16384 + kk * 8192 + row * 256 + (r16 & 1) * 8;
        read_operands(from + piece * 16, from + (piece ^ 2) * 16, from + (piece ^ 4) * 16, from + (piece ^ 6) * 16, b[kk]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) b[kk][j] = *(const half8*)(s + 16384 + (wn * 64 + r16) * 128 + c + j * 2048);
      }
    };
    auto compute = [&](int kk) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[j >> 1][i * 2 + (j & 1)] = mfma<BF16>(b[kk][j], a[kk][i], acc[j >> 1][i * 2 + (j & 1)]);
    };
    load(from), load(from + 1);
    wait_loads<8>();
    meet();
    read(from, 0);
    for (int k = from; k < to; ++k) {
      read(k, 1);
      __builtin_amdgcn_sched_barrier(0);
      compute(0);
      __builtin_amdgcn_sched_barrier(0);
      wait_loads<0>();
      wait_lds();
      meet();
      if (k + 2 < to) load(k + 2);
      if (k + 1 < to) read(k + 1, 0);
      __builtin_amdgcn_sched_barrier(0);
      compute(1);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// ------------------------------------------------------------------------- epilogues
// A block in `stage` (the wavefront's own 8 KB of LDS): rows of 32 floats, 16-byte pieces
// permuted as above.
__device__ inline void stage_block(const f4 (&c)[8], char* stage, int lane) {
  const int r16 = lane & 15, kq = lane >> 4;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int row = i * 16 + r16;
      *(f4*)(stage + row * 128 + (((j * 4 + kq) ^ ((row >> 1) & 7)) * 16)) = c[i * 2 + j];
    }
}

// A staged block by rows, in four passes of 16 rows and four lanes a row: the row and the first of
// the eight neighbouring columns that a lane has in a pass, and their values.
constexpr int kPasses = 4, kPassRows = 16;
__device__ inline int pass_row(int pass, int lane) { return pass * kPassRows + (lane >> 2); }
__device__ inline int pass_col(int lane) { return (lane & 3) * 8; }
__device__ inline void pass_values(const char* stage, int pass, int lane, float (&v)[8]) {
  const int row = pass_row(pass, lane), piece = (lane & 3) * 2, s = (row >> 1) & 7;
  const f4 lo = *(const f4*)(stage + row * 128 + ((piece ^ s) * 16));
  const f4 hi = *(const f4*)(stage + row * 128 + (((piece + 1) ^ s) * 16));
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = lo[i], v[4 + i] = hi[i];
}

// Where a staged plane of 16-bit values (64 x 32) keeps (row, col): rows of 64 bytes, with 16
// more after every eighth, so that eight lanes that read rows eight apart meet no bank twice.
__device__ inline int plane_at(int row, int col) { return row * 64 + (row >> 3) * 16 + col * 2; }

// A staged plane by columns: calls f(col, row, v) with eight neighbouring rows of a column,
// eight lanes a column, columns 8 at a time.
template <class F>
__device__ inline void by_columns(const char* plane, int lane, F f) {
#pragma unroll
  for (int pass = 0; pass < 4; ++pass) {
    const int col = pass * 8 + (lane >> 3), row = (lane & 7) * 8;
    half8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = *(const _Float16*)(plane + plane_at(row + i, col));
    f(col, row, v);
  }
}

// v as hi + lo.  A value that binary16 has no finite form of keeps its infinity or NaN in
// hi, with nothing in lo.
__device__ inline void split(float v, _Float16* hi, _Float16* lo) {
  const _Float16 h = static_cast<_Float16>(v);
  const float rest = v - static_cast<float>(h);
  *hi = h;
  *lo = static_cast<_Float16>(__builtin_fabsf(rest) < __builtin_inff() ? rest : 0.0f);
}

// The products of one launch.  An epilogue E has a plain struct E::Params and one of
//   kStaged: fetch(params, place, row, col, lane) what is needed of memory, as Inputs, and
//            block(params, place, row, col, stage, lane, inputs, next), by a wavefront: the staged
//            block at (row, col) of C, of those that begin inside the result; next is called
//            once, after the last use of the inputs and before the first store
//   kBlocks: fetch as above, and block(params, place, c, row, col, stage, lane, inputs, next): the same with
//            the block in registers, of all blocks of a tile
//   kWhole:  tile<Tile>(params, args, place, acc, lds), by the whole workgroup, in the product's LDS;
//            and part<Tile>(params, args, place, c, band, i) of a cut tile: rows i * 16 .. of each wavefront's band
//
// A launch has up to as many workgroups as fit the chip (kPlaces); an XCD's, to which they go in
// turn, get a run of whole tiles, with about an eighth of all steps.  Of each product an XCD's
// workgroups take tiles side by side, in rounds, so that what they read at a time is shared
// in their L2.  What no whole round is left for is the XCD's pool.  Its tiles are dealt out, or,
// where that would leave much of the XCD idle, each is cut along the contraction into parts of
// about one length, and the parts are dealt out, first parts first, so that here too workgroups
// side by side read the same steps.  The sums of parts are left in memory, and a second kernel adds
// them, in order, and has the epilogue.  The cut, and so the order of sums, is fixed by
// the sizes.
enum EpilogueKind { kStaged, kBlocks, kWhole };

struct Run {
  int32_t tile;    // the first of the XCD's tiles of a product
  int32_t rounds;  // whole rounds of them
  int32_t rest;    // tiles after those, in the pool
  int32_t parts;   // that each of the pool's is cut into
};

template <class E>
struct Launch {
  int32_t count;
  int32_t across;                   // workgroups an XCD
  Run runs[8][kMaxProblems];
  Args args[kMaxProblems];
  typename E::Params out[kMaxProblems];
  int32_t slot[8];                  // the first of an XCD's places for sums
  int32_t cut[8];                   // the XCDs' cut tiles before an XCD's
  float* sums;                      // a tile for each part of a pool that has cut tiles
};

// The call's memory for sums: a launch that would need more of it cuts nothing.
struct Sums {
  float* to;
  size_t bytes;
};

// What cutting costs, in steps of a tile: the parts' sums are written and read again, 256 KB each
// for a 256 tile, and the second kernel takes 8 us and more.  A launch of few workgroups has the
// shortest second kernel, and its steps are the longest, since few CUs ask for memory.
// (4096 x 4096 orthogonalised in bf16, 136 tiles of 64 steps on 256 CUs: 1.94 ms at a cost of 16,
// which cuts them, 1.63 at 28, which does not; the gradients of a loss, 256 steps: 2.2 ms cut, 2.8 not.)
constexpr int kPartCost256 = 28, kPartCost128 = 24, kPartCostFew = 10;
using host::kLeastPart;
using host::kPoolParts;
// Steps that are worth a workgroup of their own, since a launch ends with its longest: the loss and gradients of
// 5 tokens, 31104 classes and 128 features take 114 us with 8, 90 with 4, 81 with 2; of 3905 x 276 x 64 in fp32 91, 75, 75.
constexpr int kLeastShare = 2;

constexpr int kPlaces256 = host::kPlaces256, kPlaces128 = 2 * kPlaces256;

inline __host__ __device__ int32_t steps_of(const Args& p) { return p.steps * p.segments; }

template <class Tile, class E>
__device__ inline void finish(const typename E::Params& params, const Args& p, const Place& at, f4 (&acc)[Tile::kBlocks][8], char* lds) {
  const typename E::Params out = params;  // read once
  if constexpr (E::kKind == kWhole) {
    E::template tile<Tile>(out, p, at, acc, lds);
  } else {
    const int lane = thread_here() & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    char* stage = lds + wave * kWaveStage;
    if constexpr (E::kKind == kStaged) {
      const auto block_at = [&](int b, int* row, int* col) {
        Tile::block_at(wave, b, row, col);
        *row += at.tm * Tile::kRows, *col += at.tn * Tile::kCols;
        return b < Tile::kBlocks && *row < p.M && *col < p.N;
      };
      typename E::Inputs in;
      if constexpr (Tile::kBlocks > 2) {
        // The blocks' code is there once: unrolled, with the next block's inputs on their way, it took more
        // registers than there are, and 6% more time over a GPT-medium's matrices.
#pragma unroll 1
        for (int b = 0; b < Tile::kBlocks; ++b) {
          int row, col;
          if (!block_at(b, &row, &col)) continue;
          E::fetch(out, at, row, col, lane, in);
#pragma unroll
          for (int k = 0; k < Tile::kBlocks; ++k)
            if (b == k) stage_block(acc[k], stage, lane);
          wait_lds();
          __builtin_amdgcn_wave_barrier();
          E::block(out, at, row, col, stage, lane, in, [] {});
        }
        return;
      }
      // A block's inputs are fetched before the stores of the block before it: fetched later, they
      // would be waited for with the stores, which take as long again.
      int row, col;
      bool has = block_at(0, &row, &col);
      if (has) E::fetch(out, at, row, col, lane, in);
#pragma unroll
      for (int b = 0; b < Tile::kBlocks; ++b) {
        int next_row, next_col;
        const bool next = block_at(b + 1, &next_row, &next_col);
        const auto fetch_next = [&] {
          if (next) E::fetch(out, at, next_row, next_col, lane, in);
        };
        if (has) {
          stage_block(acc[b], stage, lane);
          wait_lds();
          __builtin_amdgcn_wave_barrier();
          E::block(out, at, row, col, stage, lane, in, fetch_next);
        } else {
          fetch_next();
        }
        has = next, row = next_row, col = next_col;
      }
    } else {
      // (inputs before the stores of the block before, as above)
      int row, col;
      typename E::Inputs in;
      const auto fetch = [&](int b) {
        if (b >= Tile::kBlocks) return;
        Tile::block_at(wave, b, &row, &col);
        row += at.tm * Tile::kRows, col += at.tn * Tile::kCols;
        E::fetch(out, at, row, col, lane, in);
      };
      fetch(0);
#pragma unroll
      for (int b = 0; b < Tile::kBlocks; ++b) {
        const int of_row = row, of_col = col;
        E::block(out, at, acc[b], of_row, of_col, stage, lane, in, [&] { fetch(b + 1); });
      }
    }
  }
}

// Asks at once for the lines of a launch's arguments that its first tile takes: read where they are
// needed, each waits for the one before (0.9 of the 10.3 us of a launch of 16 tiles in 64 parts).
template <class E>
__device__ inline void fetch_arguments(const Launch<E>& all, int xcd) {
  const auto word = [](const void* p, int line) { return *((const int*)p + line * 16); };
  const Args* p = &all.args[0];
  const typename E::Params* out = &all.out[0];
  constexpr int kArgs = (sizeof(Args) - 4) / 64, kOut = (sizeof(*out) - 4) / 64;
  asm volatile("" ::"s"(all.count), "s"(all.runs[xcd][0].tile), "s"(word(p, 0)), "s"(word(p, kArgs)), "s"(word(out, 0)),
               "s"(word(out, kOut / 2)), "s"(word(out, kOut)), "s"(all.slot[xcd]), "s"(all.cut[xcd]), "s"(all.sums));
}

template <class Tile, bool BF16, bool TURNED, class E>
__global__ __launch_bounds__(Tile::kThreads, Tile::kOccupancy) void product_kernel(Launch<E> all) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int xcd = blockIdx.x & 7, across = all.across;
  fetch_arguments(all, xcd);
  f4 acc[Tile::kBlocks][8];
  // first the pool's parts, of which `part` is this workgroup's next (of all of them, and counted
  // from `problem`'s first), then whole rounds
  int problem = 0, place = blockIdx.x >> 3, part = place, round = -1;
  for (;;) {
    int tile, piece = 0, pieces = 1, slot = 0;
    if (round < 0) {
      for (; problem < all.count; ++problem) {
        const Run& run = all.runs[xcd][problem];
        if (part < run.rest * run.parts) break;
        part -= run.rest * run.parts;
      }
      if (problem < all.count) {
        const Run& run = all.runs[xcd][problem];
        piece = static_cast<int>(static_cast<uint32_t>(part) / static_cast<uint32_t>(run.rest));
        pieces = run.parts;
        tile = run.tile + run.rounds * across + part - piece * run.rest;
        slot = place;
        part += across, place += across;
      } else {
        problem = round = 0;
      }
    }
    if (round >= 0) {
      for (; problem < all.count && round >= all.runs[xcd][problem].rounds; ++problem) round = 0;
      if (problem >= all.count) break;
      tile = all.runs[xcd][problem].tile + round * across + static_cast<int>(blockIdx.x >> 3);
      ++round;
    }
    const Args p = all.args[problem];
    const int steps = steps_of(p), from = steps * piece / pieces, to = steps * (piece + 1) / pieces;
    const Place at = place_of(p, tile);
    Tile::template run<BF16, TURNED>(p, at, from, to, lds, acc);
    if (pieces > 1) {
      f4* left = (f4*)(all.sums + int64_t(all.slot[xcd] + slot) * (Tile::kRows * Tile::kCols)) + thread_here();
#pragma unroll
      for (int b = 0; b < Tile::kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 8; ++i) left[(b * 8 + i) * Tile::kThreads] = acc[b][i];
    } else {
      finish<Tile, E>(all.out[problem], p, at, acc, lds);
    }
    __syncthreads();  // LDS is free again
  }
}

// The cut tile t, counted over the XCDs' pools.
struct CutTile {
  int problem, tile, parts, rest;  // the parts' sums are `rest` places apart
  int slot;                        // the place of the first part's, -1: there is no such tile
};

template <class E>
__device__ inline CutTile cut_tile(const Launch<E>& all, int t) {
  int xcd = 0;
#pragma unroll
  for (int x = 1; x < 8; ++x) xcd += all.cut[x] <= t ? 1 : 0;
  t -= all.cut[xcd];
  int slot = all.slot[xcd];
  for (int k = 0; k < all.count; ++k) {
    const Run& run = all.runs[xcd][k];
    if (run.parts > 1) {
      if (t < run.rest) return {k, run.tile + run.rounds * all.across + t, run.parts, run.rest, slot + t};
      t -= run.rest;
    }
    slot += run.rest * run.parts;
  }
  return {0, 0, 0, 0, -1};
}

template <class Tile>
__device__ inline void add_parts(const float* sums, const CutTile& cut, int b, int thread, f4 (&c)[8]) {
  constexpr int64_t kTile = int64_t(Tile::kRows) * Tile::kCols / 4;  // in vectors
  const f4* from = (const f4*)sums + cut.slot * kTile + b * 8 * Tile::kThreads + thread;
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = from[i * Tile::kThreads];
  for (int k = 1; k < cut.parts; ++k) {
    from += cut.rest * kTile;
    f4 v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = from[i * Tile::kThreads];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] += v[i];
  }
}

// What is left of tiles that were cut: workgroups (x, y) take blocks of tile x.
constexpr int kJoinWaves = 4;

template <class Tile, class E>
__global__ __launch_bounds__(64 * kJoinWaves) void product_join_kernel(Launch<E> all) {
  __shared__ __attribute__((aligned(1024))) char lds[kJoinWaves * kWaveStage];
  fetch_arguments(all, 0);
  const CutTile cut = cut_tile(all, blockIdx.x);
  if (cut.slot < 0) return;
  const Args& p = all.args[cut.problem];
  const Place at = place_of(p, cut.tile);
  const int lane = threadIdx.x & 63, block = blockIdx.y * kJoinWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = block / Tile::kBlocks, b = block % Tile::kBlocks;
  int row, col;
  Tile::block_at(wave, b, &row, &col);
  row += at.tm * Tile::kRows, col += at.tn * Tile::kCols;
  if (E::kKind == kStaged && (row >= p.M || col >= p.N)) return;
  const typename E::Params out = all.out[cut.problem];
  f4 c[8];
  add_parts<Tile>(all.sums, cut, b, wave * 64 + lane, c);
  char* stage = lds + (threadIdx.x >> 6) * kWaveStage;
  if constexpr (E::kKind == kStaged) {
    typename E::Inputs in;
    E::fetch(out, at, row, col, lane, in);
    stage_block(c, stage, lane);
    wait_lds();
    __builtin_amdgcn_wave_barrier();
    E::block(out, at, row, col, stage, lane, in, [] {});
  } else {
    typename E::Inputs in;
    E::fetch(out, at, row, col, lane, in);
    E::block(out, at, c, row, col, stage, lane, in, [] {});
  }
}

// The same for an epilogue of whole tiles: workgroups (x, y) take strips of 16 rows of a
// wavefront's 64, as little code as can be: it is fetched for this alone.  (A workgroup a tile, with all
// of a thread's values: 10.8 us for 16 tiles of 128 in four parts each.)
template <class Tile, class E>
__global__ __launch_bounds__(Tile::kThreads) void product_join_whole_kernel(Launch<E> all) {
  fetch_arguments(all, 0);
  const CutTile cut = cut_tile(all, blockIdx.x);
  if (cut.slot < 0) return;
  const Args& p = all.args[cut.problem];
  const int band = blockIdx.y >> 2, i = blockIdx.y & 3;
  constexpr int64_t kTile = int64_t(Tile::kRows) * Tile::kCols / 4;  // in vectors
  const f4* from = (const f4*)all.sums + cut.slot * kTile + (band * 16 + i * 2) * Tile::kThreads + threadIdx.x;
  f4 c[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) c[k] = from[((k >> 1) * 8 + (k & 1)) * Tile::kThreads];
  for (int s = 1; s < cut.parts; ++s) {
    from += cut.rest * kTile;
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] += from[((k >> 1) * 8 + (k & 1)) * Tile::kThreads];
  }
  E::template part<Tile>(all.out[cut.problem], p, place_of(p, cut.tile), c, band, i);
}

// The steps that the busiest of `across` workgroups has of an XCD's pool, cut so that the longest
// tile has `pieces` parts and the others parts of about its parts' length; 0: there is no room for the
// parts.
inline int64_t pool_steps(Run* runs, const Args* args, int32_t count, int32_t across, int32_t pieces) {
  // the parts go around the workgroups, one product's after another's; of each, every workgroup has `all` and
  // those of `some` places from `from` on have one more
  struct {
    int64_t length, all;
    int32_t from, some;
  } dealt[kMaxProblems];
  int64_t longest = 0, parts = 0, most = 0;
  for (int32_t k = 0; k < count; ++k)
    if (runs[k].rest > 0 && steps_of(args[k]) > longest) longest = steps_of(args[k]);
  int32_t kinds = 0;
  for (int32_t k = 0; k < count; ++k) {
    if (runs[k].rest == 0) continue;
    const int64_t steps = steps_of(args[k]);
    int64_t s = pieces > 1 ? (steps * pieces + longest / 2) / longest : 1;
    if (s > steps / kLeastPart) s = steps / kLeastPart;
    runs[k].parts = static_cast<int32_t>(s < 1 ? 1 : s);
    const int64_t n = runs[k].rest * int64_t(runs[k].parts);
    dealt[kinds++] = {(steps + runs[k].parts - 1) / runs[k].parts, n / across, static_cast<int32_t>(parts % across),
                      static_cast<int32_t>(n % across)};
    parts += n;
  }
  if (pieces > 1 && parts > int64_t(kPoolParts) * across) return 0;
  // the busiest workgroup is where some product's last parts begin
  for (int32_t i = 0; i < kinds; ++i) {
    int64_t load = 0;
    for (int32_t k = 0; k < kinds; ++k) {
      const int32_t after = dealt[i].from - dealt[k].from;
      load += dealt[k].length * (dealt[k].all + ((after < 0 ? after + across : after) < dealt[k].some ? 1 : 0));
    }
    most = load > most ? load : most;
  }
  return most;
}

// Deals the launch's tiles to XCDs and plans their pools.  Returns the workgroups; *cut counts the
// tiles that are cut.
template <int kSide, class E>
int deal(Launch<E>& all, const Sums& sums, int* cut) {
  constexpr int kPlaces = kSide == 256 ? kPlaces256 : kPlaces128;
  int64_t first[kMaxProblems + 1] = {}, units = 0;
  for (int32_t k = 0; k < all.count; ++k) {
    Args& p = all.args[k];
    p.tiles_m = (p.M + kSide - 1) / kSide;
    p.tiles_n = (p.N + kSide - 1) / kSide;
    first[k + 1] = first[k] + tile_count(p);
    if (tile_count(p) > INT32_MAX / 2 || p.lda > host::kMaxLd || p.ldb > host::kMaxLd) return -1;
    units += tile_count(p) * steps_of(p);
  }
  *cut = 0;
  if (first[all.count] == 0) return 0;
  int64_t worth = (units / kLeastShare + 7) / 8;
  all.across = static_cast<int32_t>(worth < 1 ? 1 : worth < kPlaces / 8 ? worth : kPlaces / 8);
  const int cost = kSide == 256 ? kPartCost256 : all.across * 8 > kPlaces256 ? kPartCost128 : kPartCostFew;
  int64_t tile = 0;  // of all products, the first that is not dealt yet
  int64_t dealt = 0;
  int32_t problem = 0, slots = 0;
  for (int x = 0; x < 8; ++x) {
    // tiles until the XCD's part of the steps is reached
    const int64_t until = units * (x + 1) / 8;
    for (int32_t k = 0; k < all.count; ++k) all.runs[x][k] = Run{0, 0, 0, 1};
    while (tile < first[all.count] && (dealt < until || x == 7)) {
      while (tile >= first[problem + 1]) ++problem;
      const int64_t steps = steps_of(all.args[problem]), left = first[problem + 1] - tile;
      int64_t take = x == 7 ? left : (until - dealt + steps / 2) / steps;
      if (take > left) take = left;
      if (take == 0) break;
      Run& r = all.runs[x][problem];
      r.tile = static_cast<int32_t>(tile - first[problem]);
      r.rounds = static_cast<int32_t>(take / all.across);
      r.rest = static_cast<int32_t>(take % all.across);
      tile += take;
      dealt += take * steps;
    }
    int32_t best = 1;
    int64_t least = pool_steps(all.runs[x], all.args, all.count, all.across, 1);
    for (int32_t s = 2; s <= 16; ++s) {
      const int64_t n = pool_steps(all.runs[x], all.args, all.count, all.across, s);
      if (n > 0 && n + cost < least) best = s, least = n + cost;
    }
    pool_steps(all.runs[x], all.args, all.count, all.across, best);
    all.slot[x] = slots;
    if (best == 1) continue;
    for (int32_t k = 0; k < all.count; ++k) slots += all.runs[x][k].rest * all.runs[x][k].parts;
  }
  if (size_t(slots) * kSide * kSide * sizeof(float) > sums.bytes)
    for (int x = 0; x < 8; ++x) pool_steps(all.runs[x], all.args, all.count, all.across, 1);
  all.sums = sums.to;
  for (int x = 0; x < 8; ++x) {
    all.cut[x] = *cut;
    for (int32_t k = 0; k < all.count; ++k) *cut += all.runs[x][k].parts > 1 ? all.runs[x][k].rest : 0;
  }
  return all.across * 8;
}

// Lets a kernel have more than 64 KB of LDS: once a device, before its first launch there.
inline hipError_t allow_lds(const void* kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = uint64_t(1) << (dev & 63);
  if (dev < 64 && (done.load(std::memory_order_relaxed) & bit) != 0) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

template <class Tile, bool BF16, bool TURNED, class E>
hipError_t launch_tiles(Launch<E>& all, int groups, int cut, hipStream_t stream) {
  auto* kernel = product_kernel<Tile, BF16, TURNED, E>;
  static std::atomic<uint64_t> allowed{0};
  hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), Tile::kLds, allowed);
  if (e != hipSuccess) return e;
  void* list[] = {&all};
  e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3(static_cast<uint32_t>(groups)), dim3(Tile::kThreads), list,
                      Tile::kLds, stream);
  if (e != hipSuccess || cut == 0) return e;
  if constexpr (E::kKind == kWhole) {
    return hipLaunchKernel(reinterpret_cast<const void*>(&product_join_whole_kernel<Tile, E>),
                           dim3(static_cast<uint32_t>(cut), Tile::kBlocks / 2 * 4), dim3(Tile::kThreads), list, 0, stream);
  } else {
    constexpr uint32_t kBlocksOfTile = Tile::kRows * Tile::kCols / (kBlockRows * kBlockCols);
    return hipLaunchKernel(reinterpret_cast<const void*>(&product_join_kernel<Tile, E>),
                           dim3(static_cast<uint32_t>(cut), kBlocksOfTile / kJoinWaves), dim3(64 * kJoinWaves), list, 0, stream);
  }
}

// Whether the launch is better off in tiles of 256 x 256: by the steps that a CU takes.  A CU
// takes a step of a 256 tile in about the time in which two workgroups on it take 1.4 steps of a
// 128 tile each, and has at least 8 of them.
template <class E>
bool large_tiles(const Launch<E>& all) {
  int64_t u256 = 0, u128 = 0;
  for (int32_t k = 0; k < all.count; ++k) {
    Args p = all.args[k];
    p.tiles_m = (p.M + 255) / 256, p.tiles_n = (p.N + 255) / 256;
    u256 += tile_count(p) * steps_of(p);
    p.tiles_m = (p.M + 127) / 128, p.tiles_n = (p.N + 127) / 128;
    u128 += tile_count(p) * steps_of(p);
  }
  return u256 > kPlaces256 * 8 && u256 * 14 <= u128 * 5;
}

template <bool BF16, bool TURNED, class E>
hipError_t launch_products(Launch<E>& all, const Sums& sums, hipStream_t stream) {
  int cut = 0;
  const bool large = large_tiles(all);
  const int groups = large ? deal<256>(all, sums, &cut) : deal<128>(all, sums, &cut);
  if (groups == 0) return hipSuccess;
  if (groups < 0) return hipErrorInvalidValue;
  return large ? launch_tiles<Tile256, BF16, TURNED, E>(all, groups, cut, stream)
               : launch_tiles<Tile128, BF16, TURNED, E>(all, groups, cut, stream);
}

#endif

}  // namespace product
}  // namespace daso
