// Quantising to 8-bit floating point (e4m3) with a power-of-two scale per block
// of 1 x 128 (activations) or 128 x 128 (weights).
//
// With a the largest finite magnitude of a block, its scale is the smallest
// power of two s with a <= 448 s, so x / s is exact (but for values that fall
// below fp32's range) and the conversion to e4m3, to nearest even, is the only
// rounding.  Memory bounds both kernels: x is read once, codes and scales written once
// (16717 x 6144 bf16 58.8 us and 16384 x 4096 bf16 in 128 x 128 39.0 us, 5.2 TB/s; fp32 87.9
// and 57.7, 5.8; a large copy reaches 4.8 - 5.4 by card).  In bits: a = 1.f 2^(E - 127) and 448 = 1.75 * 2^8, so the scale's
// byte (exponent + 127) is E - 8, one more where 1.f > 1.75.
#include "device_common.h"

namespace dit {

namespace {

// biased exponent of the scale of a block whose largest finite magnitude has bits a
__device__ __forceinline__ uint32_t scale_byte(uint32_t a) {
  if (a == 0) return 127;
  const int e = (int)(a >> 23) - 8 + ((a & 0x7fffff) > 0x600000);
  return (uint32_t)max(e, 0);
}
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254 - byte) << 23); }

// magnitude bits, 0 for infinities and NaN
__device__ __forceinline__ uint32_t finite_mag(float v) {
  const uint32_t m = __float_as_uint(v) & 0x7fffffff;
  return m < 0x7f800000 ? m : 0;
}

// 16 bytes at any element's address
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Bytes16 {
  uint32_t w[4];
};

// 8 consecutive elements x[0 .. 7], of which the first n exist (others 0).  Whole
// ones are loaded 16 bytes at a time wherever they lie: a row of odd length starts
// anywhere (5152 x 3186 bf16 12.3 us, element by element 24.5).
template <typename T>
__device__ __forceinline__ void load8(const T* x, int n, float* v) {
  if (n == 8) {
    const Bytes16<T>* const p = (const Bytes16<T>*)x;
    if constexpr (sizeof(T) == 2) {
      const Bytes16<T> u = p[0];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(u.w[i] << 16);
        v[2 * i + 1] = __uint_as_float(u.w[i] & 0xffff0000);
      }
    } else {
      const Bytes16<T> a = p[0], b = p[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = __uint_as_float(a.w[i]);
        v[4 + i] = __uint_as_float(b.w[i]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? to_f32<T>(x[i]) : 0.f;
  }
}

__device__ __forceinline__ uint2 codes8(const float* v, float inv) {
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inv, v[5] * inv, hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inv, v[7] * inv, hi, true);
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}

// 1 x 128: a wave takes 512 elements of a row, 8 per lane; 16 lanes share a
// scale and the wave's four scales leave as one word.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ x, long rows, int K, int Kp,
                                                            int chunks, uint8_t* __restrict__ q,
                                                            uint32_t* __restrict__ s) {
  const int lane = threadIdx.x & 63;
  const long unit = (long)block_id() * 4 + (threadIdx.x >> 6);
  if (unit >= rows * chunks) return;
  const long row = unit / chunks;
  const int c = (int)(unit - row * chunks), k = c * 512 + lane * 8;
  float v[8];
  load8<T>(x + row * K + k, min(max(K - k, 0), 8), v);
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = max(a, finite_mag(v[i]));
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) a = max(a, (uint32_t)__shfl_xor((int)a, o, 64));
  const uint32_t byte = scale_byte(a);
  if (k < Kp) *(uint2*)(q + row * Kp + k) = codes8(v, inverse_scale(byte));
  uint32_t w = 0;
#pragma unroll
  for (int g = 0; g < 4; ++g) w |= (uint32_t)__builtin_amdgcn_readlane((int)byte, g * 16) << (8 * g);
  if (lane == 0) s[row * chunks + c] = w;
}

// 128 x 128: a block of threads takes one tile, 16 lanes a row, 8 rows each
template <typename T>
__global__ __launch_bounds__(256) void quantize_tiles_kernel(const T* __restrict__ x, long rows, int K, int Kp, int kb,
                                                             int pitch, uint8_t* __restrict__ q,
                                                             uint8_t* __restrict__ s) {
  __shared__ uint32_t wave_max[4];
  const int tid = threadIdx.x;
  // kb is rounded up to whole words of scales: the tiles past Kp write theirs only
  const long id = block_id(), rb = id / pitch;
  if (rb * 128 >= rows) return;
  const int c = (int)(id - rb * pitch), k = c * 128 + (tid & 15) * 8;
  if (c >= kb) {
    if (tid == 0) s[id] = 127;
    return;
  }
  const long r0 = rb * 128 + (tid >> 4);
  float v[8][8];
  uint32_t a = 0;
  if (rows - rb * 128 >= 128 && K - c * 128 >= 128) {  // all loads ahead of the first wait
#pragma unroll
    for (int i = 0; i < 8; ++i) load8<T>(x + (r0 + i * 16) * K + k, 8, v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const long r = r0 + i * 16;
      load8<T>(x + r * K + k, r < rows ? min(max(K - k, 0), 8) : 0, v[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) a = max(a, finite_mag(v[i][j]));
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) a = max(a, (uint32_t)__shfl_xor((int)a, o, 64));
  if ((tid & 63) == 0) wave_max[tid >> 6] = a;
  __syncthreads();
  a = max(max(wave_max[0], wave_max[1]), max(wave_max[2], wave_max[3]));
  const uint32_t byte = scale_byte(a);
  const float inv = inverse_scale(byte);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const long r = r0 + i * 16;
    if (r < rows) *(uint2*)(q + r * Kp + k) = codes8(v[i], inv);
  }
  if (tid == 0) s[id] = (uint8_t)byte;
}

template <typename T>
hipError_t launch(const T* x, long rows, int K, int block_rows, uint8_t* q, uint8_t* s, hipStream_t st) {
  const int kb = fp8_k_blocks(K), Kp = kb * kFp8Block, pitch = fp8_scale_pitch(K);
  if (block_rows == 1) {
    const int chunks = pitch / 4;
    const dim3 grid = grid_of((rows * chunks + 3) / 4);
    hipLaunchKernelGGL((quantize_rows_kernel<T>), grid, dim3(256), 0, st, x, rows, K, Kp, chunks, q, (uint32_t*)s);
  } else {
    const dim3 grid = grid_of((rows + 127) / 128 * pitch);
    hipLaunchKernelGGL((quantize_tiles_kernel<T>), grid, dim3(256), 0, st, x, rows, K, Kp, kb, pitch, q, s);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_fp8(int dtype, const void* x, long rows, int K, int block_rows, void* q, void* scales,
                               hipStream_t s) {
  if (rows == 0) return hipSuccess;
  if (dtype == DIT_BF16) return launch((const bf16_t*)x, rows, K, block_rows, (uint8_t*)q, (uint8_t*)scales, s);
  return launch((const float*)x, rows, K, block_rows, (uint8_t*)q, (uint8_t*)scales, s);
}

}  // namespace dit
