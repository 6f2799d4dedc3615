// Products of block-scaled e4m3 matrices, Y = X W^T + b: X with a scale per
// 1 x 128, W with one per 128 x 128, both powers of two.
//
//   y[m, n] = sum_kb 2^(sx[m, kb] + sw[n / 128, kb] - 254) sum_{k in kb} x[m, k] w[n, k]  +  b[n]
//
// bf16 output: the 8-bit matrix cores, v_mfma_scale_f32_16x16x128_f8f6f4, whose
// K is one scale block and which apply both scales in the instruction (an
// operand's scale byte per row), so the sum needs no vector arithmetic at all.
// They align each 8 products to the largest of them and keep 14 bits there
// (measured: 2^p + 2^-6 loses its second term from p = 8 on within 8 products,
// and only at fp32's own limit across them); everything else is summed in fp32.
// Against 64 bits that is 1.3e-5 (norm) on normal values, a hundredth of the
// output's own rounding.
// fp32 output: the codes go through bf16 (exactly, scales included) to the bf16
// matrix cores, exact products with fp32 sums, at half the rate.
#include "device_common.h"

namespace dit {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

struct Fp8Problem {
  const uint8_t* x;    // [M][Kp]
  const uint8_t* xs;   // [M][pitch]
  const uint8_t* w;    // [N][Kp]
  const uint8_t* ws;   // [ceil(N / 128)][pitch]
  const void* bias;
  int bias_f32;
  void* y;
  int M, N, kb, pitch;
};

__device__ __forceinline__ float bias_at(const Fp8Problem& p, int n) {
  if (!p.bias) return 0.f;
  return p.bias_f32 ? ((const float*)p.bias)[n] : bf2f(((const bf16_t*)p.bias)[n]);
}

__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __uint_as_float(byte == 0 ? 0x400000u : byte << 23);  // 2^(byte - 127); 255: +inf, never written
}

// one lane's 32 codes as bf16 values, 8 to an operand
__device__ __forceinline__ void to_bf16(const uint4& lo, const uint4& hi, float scale, bf16x8_t* out) {
  const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * i + j], scale, false);
      const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[2 * i + j], scale, true);
      out[i][4 * j + 0] = a[0];
      out[i][4 * j + 1] = a[1];
      out[i][4 * j + 2] = b[0];
      out[i][4 * j + 3] = b[1];
    }
}

// 64 x 64 outputs per block, 32 x 32 per wave, operands straight from memory.
// W's rows are the matrix cores' rows, so a lane holds four neighbouring columns
// of one output row.
template <bool F32>
__global__ __launch_bounds__(256) void fp8_tile_kernel(const Fp8Problem p) {
  const int tiles_n = (p.N + 63) / 64;
  const int id = block_id();
  const int tm = id / tiles_n, tn = id - tm * tiles_n;
  if (tm * 64 >= p.M) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int m0 = tm * 64 + (wave >> 1) * 32, n0 = tn * 64 + (wave & 1) * 32;
  const long Kp = (long)p.kb * kFp8Block;
  const uint8_t *xr[2], *wr[2], *xsr[2], *wsr[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int m = min(m0 + i * 16 + (lane & 15), p.M - 1), n = min(n0 + i * 16 + (lane & 15), p.N - 1);
    xr[i] = p.x + m * Kp + (lane >> 4) * 32;
    wr[i] = p.w + n * Kp + (lane >> 4) * 32;
    xsr[i] = p.xs + (long)m * p.pitch;
    wsr[i] = p.ws + (long)(n >> 7) * p.pitch;
  }
  f32x4_t acc[2][2] = {};
  for (int kb = 0; kb < p.kb; ++kb) {
    uint4 x[2][2], w[2][2];
    int xs[2], ws[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        x[i][c] = ((const uint4*)(xr[i] + kb * 128))[c];
        w[i][c] = ((const uint4*)(wr[i] + kb * 128))[c];
      }
      xs[i] = xsr[i][kb];
      ws[i] = wsr[i][kb];
    }
    if constexpr (F32) {
      bf16x8_t xb[2][4], wb[2][4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        to_bf16(x[i][0], x[i][1], scale_of(xs[i]), xb[i]);
        to_bf16(w[i][0], w[i][1], scale_of(ws[i]), wb[i]);
      }
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[j][c], xb[i][c], acc[i][j], 0, 0, 0);
    } else {
      i32x8_t xv[2], wv[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        xv[i] = i32x8_t{(int)x[i][0].x, (int)x[i][0].y, (int)x[i][0].z, (int)x[i][0].w,
                        (int)x[i][1].x, (int)x[i][1].y, (int)x[i][1].z, (int)x[i][1].w};
        wv[i] = i32x8_t{(int)w[i][0].x, (int)w[i][0].y, (int)w[i][0].z, (int)w[i][0].w,
                        (int)w[i][1].x, (int)w[i][1].y, (int)w[i][1].z, (int)w[i][1].w};
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wv[j], xv[i], acc[i][j], 0, 0, 0, ws[j], 0, xs[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int m = m0 + i * 16 + (lane & 15);
    if (m >= p.M) continue;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int n = n0 + j * 16 + (lane >> 4) * 4 + r;
        if (n >= p.N) continue;
        const float v = acc[i][j][r] + bias_at(p, n);
        if constexpr (F32) ((float*)p.y)[(long)m * p.N + n] = v;
        else ((bf16_t*)p.y)[(long)m * p.N + n] = f2bf(v);
      }
  }
}

}  // namespace

hipError_t launch_gemm_fp8(int M, int N, int K, const void* x, const void* xs, const void* w, const void* ws,
                           const void* bias, int bias_dtype, void* y, int out_dtype, hipStream_t s) {
  if (M == 0) return hipSuccess;
  Fp8Problem p;
  p.x = (const uint8_t*)x;
  p.xs = (const uint8_t*)xs;
  p.w = (const uint8_t*)w;
  p.ws = (const uint8_t*)ws;
  p.bias = bias;
  p.bias_f32 = bias_dtype == DIT_F32;
  p.y = y;
  p.M = M;
  p.N = N;
  p.kb = fp8_k_blocks(K);
  p.pitch = fp8_scale_pitch(K);
  const long tiles = (long)((M + 63) / 64) * ((N + 63) / 64);
  if (out_dtype == DIT_F32)
    hipLaunchKernelGGL((fp8_tile_kernel<true>), grid_of(tiles), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((fp8_tile_kernel<false>), grid_of(tiles), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace dit
