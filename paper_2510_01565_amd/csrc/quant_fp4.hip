// Quantising to 4-bit floating point (e2m1) with a power-of-two scale per 1 x 32
// block, and back.
//
// With a the largest magnitude of a block, its scale is the smallest power of two s
// with a <= 6 s, so x / s is exact (but for values that fall below fp32's range) and
// the conversion to e2m1, to nearest even, is the only rounding.  In bits: a = 1.f
// 2^(E - 127) and 6 = 1.5 * 2^2, so the scale's byte (exponent + 127) is E - 2, one
// more where 1.f > 1.5.  A block with an infinity or a NaN gets the NaN scale, 255,
// and codes of 0.  Memory bounds both kernels, which read and write every value once:
// 16717 x 6144 from bf16 in 50 us, 5.2 TB/s, as fast as a copy, back in 36 us, 7.2 TB/s.
// A row of 4096 takes 4.2 us, as any launch does.
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
  uint32_t w __attribute__((ext_vector_type(4)));
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

// a wave's row and chunk of 512 elements, of at most 2^31 in all
struct Chunk {
  long unit, row;
  int c;
};
__device__ __forceinline__ Chunk chunk_of(long rows, int chunks) {
  const long unit = (long)block_id() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long row = (uint32_t)unit / (uint32_t)chunks;
  return {unit, row, (int)(unit - row * chunks)};
}

// A wave takes 512 elements of a row, 8 per lane: 4 lanes share a scale, and the
// wave's sixteen leave as one piece of 16 bytes.  (Two chunks a wave: 47 us for 50 at
// 16717 x 6144, but 5.1 for 4.9 at 4429 x 1536 and 84 for 80 in fp32.)
template <typename T>
__global__ __launch_bounds__(256) void quantize_fp4_kernel(const T* __restrict__ x, long rows, int K, int pitch, int chunks,
                                                           uint8_t* __restrict__ q, uint32_t* __restrict__ s) {
  const int lane = threadIdx.x & 63;
  const auto [unit, row, c] = chunk_of(rows, chunks);
  if (unit >= rows * chunks) return;
  const int k = c * 512 + lane * 8;
  float v[8];
  load8<T>(x + row * K + k, min(max(K - k, 0), 8), v);
  uint32_t a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(v[i]) & 0x7fffffff);
  a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0xb1, 0xf, 0xf, true));  // lanes 1, 0, 3, 2 of each four
  a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0x4e, 0xf, 0xf, true));  // 2, 3, 0, 1
  const uint32_t byte = scale_byte(a);
  const float inv = __uint_as_float((254 - byte) << 23);
  uint32_t w = 0;
  static_for<4>([&](auto ic) {
    constexpr int i = decltype(ic)::value;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2 * i] * inv, v[2 * i + 1] * inv, 1.0f, i);
  });
  if (byte == 255) w = 0;
  if (k < pitch * 2) *(uint32_t*)(q + row * pitch + c * 256 + lane * 4) = w;
  // block 4 i + j, whose first lane is 16 i + 4 j, is byte i of word j: the bytes of lanes 16 apart are joined
  uint32_t word = byte << (lane >> 4) * 8;
  const auto far = __builtin_amdgcn_permlane32_swap(word, word, false, false);
  word = far[0] | far[1];
  const auto near = __builtin_amdgcn_permlane16_swap(word, word, false, false);
  word = near[0] | near[1];
  if (lane < 16 && lane % 4 == 0) s[unit * 4 + lane / 4] = word;
}

// Back: a lane takes 16 bytes' worth of neighbouring elements of a row, in fp32 in two turns.  They are stored past the
// caches: through them 55 us for 36, in fp32 122 for 65.
template <typename T>
__global__ __launch_bounds__(256) void dequantize_fp4_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ s,
                                                             long rows, int K, int pitch, int chunks, T* __restrict__ y) {
  constexpr int E = 16 / sizeof(T);
  const int lane = threadIdx.x & 63;
  const auto [unit, row, c] = chunk_of(rows, chunks);
  if (unit >= rows * chunks) return;
#pragma unroll
  for (int h = 0; h < 8 / E; ++h) {
    const int at = h * 256 + lane * E, k = c * 512 + at, b = at >> 5;
    if (k >= K) return;
    const uint8_t* const from = q + row * pitch + c * 256 + at / 2;
    const uint32_t w = E == 8 ? *(const uint32_t*)from : *(const uint16_t*)from;
    const uint32_t byte = s[unit * 16 + (b & 3) * 4 + (b >> 2)];
    const float scale = __uint_as_float(byte == 0 ? 0x00400000 : byte == 255 ? 0x7fc00000 : byte << 23);
    float v[E];
    static_for<E / 2>([&](auto ic) {
      constexpr int i = decltype(ic)::value;
      const auto f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, i);
      v[2 * i] = f[0] * scale;
      v[2 * i + 1] = f[1] * scale;
    });
    T* const to = y + row * K + k;
    if (K - k >= E) {
      Bytes16<T> u;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) u.w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        else u.w[i] = __float_as_uint(v[i]);
      }
      __builtin_nontemporal_store(u.w, &((Bytes16<T>*)to)->w);
    } else {
#pragma unroll
      for (int i = 0; i < E - 1; ++i)
        if (i < K - k) to[i] = from_f32<T>(v[i]);
    }
  }
}

}  // namespace

hipError_t launch_quantize_fp4(int dtype, const void* x, long rows, int K, void* q, void* scales, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const int chunks = fp4_scale_pitch(K) / 16;
  const dim3 grid = grid_of((rows * chunks + 3) / 4);
  if (dtype == DIT_BF16)
    hipLaunchKernelGGL((quantize_fp4_kernel<bf16_t>), grid, dim3(256), 0, s, (const bf16_t*)x, rows, K, fp4_pitch(K), chunks,
                       (uint8_t*)q, (uint32_t*)scales);
  else
    hipLaunchKernelGGL((quantize_fp4_kernel<float>), grid, dim3(256), 0, s, (const float*)x, rows, K, fp4_pitch(K), chunks,
                       (uint8_t*)q, (uint32_t*)scales);
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
