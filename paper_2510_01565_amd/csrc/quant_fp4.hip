// Quantising to 4-bit floating point (e2m1) with a power-of-two scale per 1 x 32
// block, and back.
//
// With a the largest magnitude of a block, its scale is the smallest power of two s
// with a <= 6 s, so x / s is exact (but for values that fall below fp32's range) and
// the conversion to e2m1, to nearest even, is the only rounding.  In bits: a = 1.f
// 2^(E - 127) and 6 = 1.5 * 2^2, so the scale's byte (exponent + 127) is E - 2, one
// more where 1.f > 1.5.  A block with an infinity or a NaN gets the NaN scale, 255,
// and codes of 0.  Memory bounds both kernels: every value is read once and written once.
#include "device_common.h"

namespace dit {

namespace {

// biased exponent of the scale of a block whose largest magnitude has bits a
__device__ __forceinline__ uint32_t scale_byte(uint32_t a) {
  if (a == 0) return 127;
  if (a >= 0x7f800000) return 255;
  return (uint32_t)max((int)(a >> 23) - 2 + ((a & 0x7fffff) > 0x400000), 0);
}

// 16 bytes at any element's address
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Bytes16 {
  uint32_t w[4];
};

// 8 consecutive elements x[0 .. 7], of which the first n exist (others 0)
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

// A wave takes 512 elements of a row, 8 per lane: 4 lanes share a scale, and the
// wave's sixteen leave as one piece of 16 bytes.
template <typename T>
__global__ __launch_bounds__(256) void quantize_fp4_kernel(const T* __restrict__ x, long rows, int K, int pitch, int chunks,
                                                           uint8_t* __restrict__ q, uint4* __restrict__ s) {
  const int lane = threadIdx.x & 63;
  const long unit = (long)block_id() * 4 + (threadIdx.x >> 6);
  if (unit >= rows * chunks) return;
  const long row = unit / chunks;
  const int c = (int)(unit - row * chunks), k = c * 512 + lane * 8;
  float v[8];
  load8<T>(x + row * K + k, min(max(K - k, 0), 8), v);
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(v[i]) & 0x7fffffff);
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) a = max(a, (uint32_t)__shfl_xor((int)a, o, 64));
  const uint32_t byte = scale_byte(a);
  const float inv = __uint_as_float((254 - byte) << 23);
  uint32_t w = 0;
  static_for<4>([&](auto ic) {
    constexpr int i = decltype(ic)::value;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2 * i] * inv, v[2 * i + 1] * inv, 1.0f, i);
  });
  if (byte == 255) w = 0;
  if (k < pitch * 2) *(uint32_t*)(q + row * pitch + c * 256 + lane * 4) = w;
  // block 4 i + j, whose first lane is 16 i + 4 j, is byte i of word j
  uint32_t word[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    word[j] = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) word[j] |= (uint32_t)__builtin_amdgcn_readlane((int)byte, i * 16 + j * 4) << (8 * i);
  }
  if (lane == 0) s[unit] = make_uint4(word[0], word[1], word[2], word[3]);
}

// Back: a lane takes 8 neighbouring elements of a row
template <typename T>
__global__ __launch_bounds__(256) void dequantize_fp4_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ s,
                                                             long rows, int K, int pitch, int chunks, T* __restrict__ y) {
  const int lane = threadIdx.x & 63;
  const long unit = (long)block_id() * 4 + (threadIdx.x >> 6);
  if (unit >= rows * chunks) return;
  const long row = unit / chunks;
  const int c = (int)(unit - row * chunks), k = c * 512 + lane * 8, b = lane >> 2;
  if (k >= K) return;
  const uint32_t w = *(const uint32_t*)(q + row * pitch + c * 256 + lane * 4);
  const uint32_t byte = s[unit * 16 + (b & 3) * 4 + (b >> 2)];
  const float scale = __uint_as_float(byte == 0 ? 0x00400000 : byte == 255 ? 0x7fc00000 : byte << 23);
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // e2m1: 0 and 0.5, then (1 + m / 2) 2^(e - 1)
    const uint32_t n = w >> (4 * i), e = n >> 1 & 3, m = n & 1;
    const uint32_t bits = e ? (126 + e) << 23 | m << 22 : m * 0x3f000000;
    v[i] = __uint_as_float(bits | (n & 8) << 28) * scale;
  }
  T* const to = y + row * K + k;
  if (K - k >= 8) {
    Bytes16<T>* const p = (Bytes16<T>*)to;
    if constexpr (sizeof(T) == 2) {
      Bytes16<T> u;
#pragma unroll
      for (int i = 0; i < 4; ++i) u.w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
      p[0] = u;
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        Bytes16<T> u;
#pragma unroll
        for (int i = 0; i < 4; ++i) u.w[i] = __float_as_uint(v[4 * h + i]);
        p[h] = u;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < K - k) to[i] = from_f32<T>(v[i]);
  }
}

}  // namespace

hipError_t launch_quantize_fp4(int dtype, const void* x, long rows, int K, void* q, void* scales, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const int chunks = fp4_scale_pitch(K) / 16;
  const dim3 grid = grid_of((rows * chunks + 3) / 4);
  if (dtype == DIT_BF16)
    hipLaunchKernelGGL((quantize_fp4_kernel<bf16_t>), grid, dim3(256), 0, s, (const bf16_t*)x, rows, K, fp4_pitch(K), chunks,
                       (uint8_t*)q, (uint4*)scales);
  else
    hipLaunchKernelGGL((quantize_fp4_kernel<float>), grid, dim3(256), 0, s, (const float*)x, rows, K, fp4_pitch(K), chunks,
                       (uint8_t*)q, (uint4*)scales);
  return hipGetLastError();
}

hipError_t launch_dequantize_fp4(int dtype, const void* q, const void* scales, long rows, int K, void* y, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const int chunks = fp4_scale_pitch(K) / 16;
  const dim3 grid = grid_of((rows * chunks + 3) / 4);
  if (dtype == DIT_BF16)
    hipLaunchKernelGGL((dequantize_fp4_kernel<bf16_t>), grid, dim3(256), 0, s, (const uint8_t*)q, (const uint8_t*)scales, rows,
                       K, fp4_pitch(K), chunks, (bf16_t*)y);
  else
    hipLaunchKernelGGL((dequantize_fp4_kernel<float>), grid, dim3(256), 0, s, (const uint8_t*)q, (const uint8_t*)scales, rows,
                       K, fp4_pitch(K), chunks, (float*)y);
  return hipGetLastError();
}

}  // namespace dit
