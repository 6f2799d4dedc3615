// Products of microscaled e2m1 matrices, Y = X W^T + b, both with a power-of-two
// scale per 1 x 32:
//
//   y[m, n] = sum_b 2^(sx[m, b] + sw[n, b] - 254) sum_{k in b} x[m, k] w[n, k]  +  bias[n]
//
// on the 4-bit matrix cores, which apply the scales in the instruction: of
// v_mfma_scale_f32_16x16x128_f8f6f4 lane l holds row l % 16 and the block l / 16 of
// 128 elements, 16 bytes, and gives that block's scale byte.
#include "device_common.h"

namespace dit {

namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));

struct Fp4Problem {
  const uint8_t* x;   // [M][pitch]
  const uint8_t* xs;  // [M][spitch]
  const uint8_t* w;   // [N][pitch]
  const uint8_t* ws;  // [N][spitch]
  const void* bias;
  int bias_f32, out_f32;
  void* y;
  int M, N, pitch, spitch;
};

__device__ __forceinline__ float bias_at(const Fp4Problem& p, int n) {
  if (!p.bias) return 0.f;
  return p.bias_f32 ? ((const float*)p.bias)[n] : bf2f(((const bf16_t*)p.bias)[n]);
}

// c += x w of 128 elements, the scales in byte B of their words; only four of the operands' registers hold 4-bit codes
template <int B>
__device__ __forceinline__ f32x4_t mfma(const i32x4_t& w, const i32x4_t& x, const f32x4_t& c, int sw, int sx) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_shufflevector(w, w, 0, 1, 2, 3, 0, 1, 2, 3),
                                                          __builtin_shufflevector(x, x, 0, 1, 2, 3, 0, 1, 2, 3), c, 4, 4, B, sw,
                                                          B, sx);
}

constexpr int kGridRow4 = 22;

// 64 x 64 outputs per block of 4 waves, each 32 x 32, operands straight from memory
__global__ __launch_bounds__(256) void fp4_simple_kernel(const Fp4Problem p) {
  const long tn = (p.N + 63) / 64, tm = (p.M + 63) / 64, id = ((long)blockIdx.y << kGridRow4) + blockIdx.x;
  if (id >= tm * tn) return;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, lr = lane & 15, g = lane >> 4;
  const int m0 = (int)(id / tn) * 64 + (wv >> 1) * 32, n0 = (int)(id % tn) * 64 + (wv & 1) * 32;
  const uint8_t *x[2], *xs[2], *w[2], *ws[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const long m = min(m0 + i * 16 + lr, p.M - 1), n = min(n0 + i * 16 + lr, p.N - 1);
    x[i] = p.x + m * p.pitch + g * 16;
    xs[i] = p.xs + m * p.spitch + g * 4;
    w[i] = p.w + n * p.pitch + g * 16;
    ws[i] = p.ws + n * p.spitch + g * 4;
  }
  f32x4_t acc[2][2] = {};
  for (int k = 0; k < p.pitch; k += 256) {
    int sx[2], sw[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      sx[i] = *(const int*)(xs[i] + k / 16);
      sw[i] = *(const int*)(ws[i] + k / 16);
    }
    static_for<4>([&](auto sc) {
      constexpr int s = decltype(sc)::value;
      if (k + s * 64 < p.pitch) {
        i32x4_t xf[2], wf[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          xf[i] = *(const i32x4_t*)(x[i] + k + s * 64);
          wf[i] = *(const i32x4_t*)(w[i] + k + s * 64);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j) acc[i][j] = mfma<s>(wf[j], xf[i], acc[i][j], sw[j], sx[i]);
      }
    });
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const long m = m0 + i * 16 + lr;
        const int n = n0 + j * 16 + g * 4 + r;
        if (m >= p.M || n >= p.N) continue;
        const float v = acc[i][j][r] + bias_at(p, n);
        if (p.out_f32) ((float*)p.y)[m * p.N + n] = v;
        else ((bf16_t*)p.y)[m * p.N + n] = f2bf(v);
      }
}

}  // namespace

const char* gemm_fp4_config_name(int M, int N, int K, int out_dtype) { return "gemm_fp4"; }

hipError_t launch_gemm_fp4(int M, int N, int K, const void* x, const void* xs, const void* w, const void* ws,
                           const void* bias, int bias_dtype, void* y, int out_dtype, hipStream_t s) {
  if (M == 0) return hipSuccess;
  Fp4Problem p;
  p.x = (const uint8_t*)x;
  p.xs = (const uint8_t*)xs;
  p.w = (const uint8_t*)w;
  p.ws = (const uint8_t*)ws;
  p.bias = bias;
  p.bias_f32 = bias_dtype == DIT_F32;
  p.out_f32 = out_dtype == DIT_F32;
  p.y = y;
  p.M = M;
  p.N = N;
  p.pitch = fp4_pitch(K);
  p.spitch = fp4_scale_pitch(K);
  const long tiles = (((long)M + 63) / 64) * (((long)N + 63) / 64);
  const dim3 grid((unsigned)std::min(tiles, 1L << kGridRow4), (unsigned)((tiles - 1) >> kGridRow4) + 1);
  hipLaunchKernelGGL(fp4_simple_kernel, grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace dit
