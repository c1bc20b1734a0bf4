// Device helpers shared by the training operators: element types, sums over a workgroup,
// and the laying out of a matrix as 16-bit planes, straight and transposed.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "daso_product.h"
#include "daso_train.h"

namespace daso {

typedef float f4v __attribute__((ext_vector_type(4)));
typedef uint16_t us8 __attribute__((ext_vector_type(8)));
typedef uint16_t us4 __attribute__((ext_vector_type(4)));
// The same at any element's place: one load or store all the same, which gfx950 takes at any address.
typedef f4v f4v_any __attribute__((aligned(4)));
typedef us8 us8_any __attribute__((aligned(2)));

#if defined(__HIP_DEVICE_COMPILE__) || defined(__HIPCC__)

__device__ inline float widen_bf16(uint16_t b) { return __builtin_bit_cast(float, uint32_t(b) << 16); }

// Round to nearest, ties to even; NaN becomes the quiet NaN of daso.h's wire.
__device__ inline uint16_t to_bf16(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0x7fc0;
  return static_cast<uint16_t>((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

template <class T>
__device__ inline float load1(const T* p);
template <>
__device__ inline float load1<float>(const float* p) { return *p; }
template <>
__device__ inline float load1<uint16_t>(const uint16_t* p) { return widen_bf16(*p); }
__device__ inline void store1(float* p, float v) { *p = v; }
__device__ inline void store1(uint16_t* p, float v) { *p = to_bf16(v); }

// 16 bytes as they are.
__device__ inline f4v load16(const float* p) { return *(const f4v_any*)p; }
__device__ inline us8 load16(const uint16_t* p) { return *(const us8_any*)p; }
// Eight elements.
__device__ inline void load8(const float* p, float (&v)[8]) {
  const f4v a = *(const f4v_any*)p, b = *(const f4v_any*)(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
}
__device__ inline void load8(const uint16_t* p, float (&v)[8]) {
  const us8 a = *(const us8_any*)p;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = widen_bf16(a[i]);
}
__device__ inline void store8(float* p, const float (&v)[8]) {
  *(f4v_any*)p = f4v{v[0], v[1], v[2], v[3]};
  *(f4v_any*)(p + 4) = f4v{v[4], v[5], v[6], v[7]};
}
__device__ inline void store8(uint16_t* p, const float (&v)[8]) {
  us8 a;
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = to_bf16(v[i]);
  *(us8_any*)p = a;
}

// Four, from a place aligned to four elements.
__device__ inline f4v load4(const float* p) { return *(const f4v*)p; }
__device__ inline f4v load4(const uint16_t* p) {
  const us4 a = *(const us4*)p;
  return f4v{widen_bf16(a[0]), widen_bf16(a[1]), widen_bf16(a[2]), widen_bf16(a[3])};
}
__device__ inline void store4(float* p, const f4v& v) { *(f4v*)p = v; }
__device__ inline void store4(uint16_t* p, const f4v& v) { *(us4*)p = us4{to_bf16(v[0]), to_bf16(v[1]), to_bf16(v[2]), to_bf16(v[3])}; }

// Sums over a wavefront, the same in every lane.
template <class T>
__device__ inline T wave_sum(T v) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) v += __shfl_xor(v, s);
  return v;
}
__device__ inline float wave_max(float v) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) v = fmaxf(v, __shfl_xor(v, s));
  return v;
}

// Over a workgroup of up to 16 wavefronts; `shared` holds one T a wavefront.  The same in
// every thread, summed in the wavefronts' order.
template <class T>
__device__ inline T group_sum(T v, T* shared) {
  v = wave_sum(v);
  const int waves = blockDim.x >> 6;
  if (waves == 1) return v;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
  __syncthreads();
  v = shared[0];
  for (int i = 1; i < waves; ++i) v += shared[i];
  return v;
}

// A matrix as planes.  Source: rows x cols, rows `stride` elements apart.  Straight planes:
// rows_p rows of cols_p, transposed ones: cols_p rows of rows_p; both padded with zeros
// (rows_p and cols_p are multiples of 64).  Null planes are left out.
struct PlanesArgs {
  const void* src;
  int64_t stride, batch_stride;
  int32_t rows, cols, rows_p, cols_p;
  uint16_t *d[2], *t[2];  // hi, lo
};

// One 64 x 64 tile by 256 threads, four neighbouring ones a row of the source.  RAW: the source's 16-bit patterns
// themselves (bf16), else scaled(value) as binary16 hi and lo.
template <class T, bool RAW, class F>
__device__ inline void planes_tile(const PlanesArgs& p, int64_t batch, int tr, int tc, F scaled, uint16_t (*lds)[64][66]) {
  const int row = threadIdx.x >> 2, col = (threadIdx.x & 3) * 16;
  const int r = tr * 64 + row, c = tc * 64 + col;
  const T* src = (const T*)p.src + batch * p.batch_stride + int64_t(r) * p.stride + c;
  uint16_t hi[16], lo[16];
  float v[16];
  const bool whole = r < p.rows && c + 16 <= p.cols;
  if (whole) {
    float a[8], b[8];
    load8(src, a), load8(src + 8, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = a[i], v[8 + i] = b[i];
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = r < p.rows && c + i < p.cols ? load1(src + i) : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if constexpr (RAW) {
      hi[i] = static_cast<uint16_t>(__builtin_bit_cast(uint32_t, v[i]) >> 16);
      lo[i] = 0;
    } else {
      _Float16 h, l;
      product::split(scaled(v[i]), &h, &l);
      hi[i] = __builtin_bit_cast(uint16_t, h), lo[i] = __builtin_bit_cast(uint16_t, l);
    }
  }
  const int64_t base = batch * p.rows_p * p.cols_p;
#pragma unroll
  for (int plane = 0; plane < 2; ++plane) {
    const uint16_t* from = plane == 0 ? hi : lo;
    if (p.d[plane] != nullptr) {
      us8 a, b;
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = from[i], b[i] = from[8 + i];
      us8* to = (us8*)(p.d[plane] + base + int64_t(r) * p.cols_p + c);
      to[0] = a, to[1] = b;
    }
    if (p.t[plane] != nullptr)
#pragma unroll
      for (int i = 0; i < 16; ++i) lds[plane][row][col + i] = from[i];
  }
  if (p.t[0] == nullptr && p.t[1] == nullptr) return;
  __syncthreads();
#pragma unroll
  for (int plane = 0; plane < 2; ++plane) {
    if (p.t[plane] == nullptr) continue;
    us8 a, b;  // the tile's column `row`, rows col..
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = lds[plane][col + i][row], b[i] = lds[plane][col + 8 + i][row];
    us8* to = (us8*)(p.t[plane] + base + int64_t(tc * 64 + row) * p.rows_p + tr * 64 + col);
    to[0] = a, to[1] = b;
  }
}

// A launch reports its own status, so that an error of the caller's that is pending stays so.
template <class K, class... A>
hipError_t launch(K* kernel, dim3 grid, dim3 block, hipStream_t stream, A... args) {
  void* list[] = {&args...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, block, list, 0, stream);
}

// The stream must be of the current device, as for every call of daso.h.
inline int current_device(hipStream_t stream) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return DASO_EHIP;
  if (stream == nullptr) return DASO_OK;
  hipDevice_t of = 0;
  if (hipStreamGetDevice(stream, &of) != hipSuccess) return DASO_EHIP;
  return of == dev ? DASO_OK : DASO_EINVAL;
}

#endif

}  // namespace daso
