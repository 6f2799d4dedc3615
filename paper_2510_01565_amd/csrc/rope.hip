// Rotary positions: pairs of dimensions of every head turned by position times
// frequency, (a, b) -> m (a cos - b sin, a sin + b cos).
//
// The angle is formed in 64 bits, in turns: pos * (w / 2 pi), of which the nearest
// whole number is taken off; what is left goes to fp32 and to sine and cosine of a
// multiple of pi.  A block forms the sines and cosines of its tokens' pairs once, in
// LDS, for all heads, while its first pieces are on their way.  Memory bounds it: x is
// read once and y written once, both past the caches: 56 us at 16391 tokens of 40 heads
// of 128, half of each turned, 6.0 TB/s; 62 with the loads behind the sines, 66 through
// the caches.  A single token takes 5.7 us, of which 4.2 is any launch's.
#include <math.h>

#include "device_common.h"

namespace dit {

namespace {

constexpr int kMaxPairs = DIT_ROPE_MAX_DIM / 2;
struct RopeArgs {
  const void* x;
  void* y;
  const int* pos;
  long ldx, ldy, rows;
  int heads, d, rot;
  float magnitude;
  double turns[kMaxPairs];  // w / (2 pi)
};

template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Bytes16 {
  uint32_t w __attribute__((ext_vector_type(4)));
};
template <typename T>
__device__ __forceinline__ void load16b(const T* x, float* v) {
  Bytes16<T> u;
  u.w = __builtin_nontemporal_load(&((const Bytes16<T>*)x)->w);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) {
      v[2 * i] = __uint_as_float(u.w[i] << 16);
      v[2 * i + 1] = __uint_as_float(u.w[i] & 0xffff0000);
    } else {
      v[i] = __uint_as_float(u.w[i]);
    }
  }
}
template <typename T>
__device__ __forceinline__ void store16b(T* y, const float* v) {
  Bytes16<T> u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 2) u.w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    else u.w[i] = __float_as_uint(v[i]);
  }
  __builtin_nontemporal_store(u.w, &((Bytes16<T>*)y)->w);
}

// A block takes a token.  WIDE: pieces of 16 bytes, where the turned part (each half of it, HALF) and the head are whole
// numbers of them; otherwise element by element.
template <typename T, bool HALF, bool WIDE>
__global__ __launch_bounds__(256) void rope_kernel(const RopeArgs a) {
  __shared__ float2 cs[kMaxPairs];
  const long row = block_id();
  if (row >= a.rows) return;
  const int pairs = a.rot / 2;
  const T* const x = (const T*)a.x + row * a.ldx;
  T* const y = (T*)a.y + row * a.ldy;
  constexpr int E = WIDE ? 16 / sizeof(T) : 1;  // elements of a piece
  constexpr int P = HALF ? E : WIDE ? E : 2;    // of what is loaded at once
  // a head's work: pieces of the turned part (of its first half, HALF), then pieces that are copied
  const int turned = HALF ? pairs / E : (WIDE ? a.rot / E : pairs), copied = x == y ? 0 : (a.d - a.rot) / E;
  const int per = turned + copied, units = a.heads * per;
  float p[P], q[P];
  int c, e;
  auto load = [&](int u) __attribute__((always_inline)) {
    const int h = u / per;
    c = u - h * per;
    e = h * a.d + (c >= turned ? a.rot + (c - turned) * E : c * P);
    if constexpr (WIDE) {
      load16b(x + e, p);
      if constexpr (HALF)
        if (c < turned) load16b(x + e + pairs, q);
    } else {
      p[0] = to_f32<T>(x[e]);
      if (c < turned) (HALF ? q[0] : p[P - 1]) = to_f32<T>(x[HALF ? e + pairs : e + 1]);
    }
  };
  auto turn = [&]() __attribute__((always_inline)) {
    if (c >= turned) {
      if constexpr (WIDE) store16b(y + e, p);
      else y[e] = from_f32<T>(p[0]);
    } else if constexpr (HALF) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float2 r = cs[c * E + i];
        const float b = p[i] * r.y + q[i] * r.x;
        p[i] = p[i] * r.x - q[i] * r.y;
        q[i] = b;
      }
      if constexpr (WIDE) {
        store16b(y + e, p);
        store16b(y + e + pairs, q);
      } else {
        y[e] = from_f32<T>(p[0]);
        y[e + pairs] = from_f32<T>(q[0]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < P; i += 2) {
        const float2 r = cs[c * (P / 2) + i / 2];
        const float b = p[i] * r.y + p[i + 1] * r.x;
        p[i] = p[i] * r.x - p[i + 1] * r.y;
        p[i + 1] = b;
      }
      if constexpr (WIDE) {
        store16b(y + e, p);
      } else {
        y[e] = from_f32<T>(p[0]);
        y[e + 1] = from_f32<T>(p[1]);
      }
    }
  };
  // the first loads are on their way while the sines are formed
  int u = threadIdx.x;
  if (u < units) load(u);
  const int pos = a.pos ? a.pos[row] : (int)row;
  for (int i = threadIdx.x; i < pairs; i += 256) {
    double t = (double)pos * a.turns[i];
    t -= rint(t);
    float s, c;
    sincospif(2.0f * (float)t, &s, &c);
    cs[i] = make_float2(c * a.magnitude, s * a.magnitude);
  }
  __syncthreads();
  while (u < units) {
    turn();
    u += 256;
    if (u < units) load(u);
  }
}

template <typename T, bool HALF>
void launch(const RopeArgs& a, hipStream_t s) {
  constexpr int E = 16 / sizeof(T);
  const bool wide = a.rot % (HALF ? 2 * E : E) == 0 && a.d % E == 0;
  const dim3 grid = grid_of(a.rows);
  if (wide) hipLaunchKernelGGL((rope_kernel<T, HALF, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((rope_kernel<T, HALF, false>), grid, dim3(256), 0, s, a);
}

}  // namespace

hipError_t launch_rope(int dtype, long rows, int heads, int d, int rot, int layout, const int* pos, const double* w,
                       float magnitude, const void* x, long ldx, void* y, long ldy, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  RopeArgs a;
  a.x = x;
  a.y = y;
  a.pos = pos;
  a.ldx = ldx;
  a.ldy = ldy;
  a.rows = rows;
  a.heads = heads;
  a.d = d;
  a.rot = rot;
  a.magnitude = magnitude;
  for (int i = 0; i < kMaxPairs; ++i) a.turns[i] = i < rot / 2 ? w[i] / (2 * M_PI) : 0.0;
  if (dtype == DIT_BF16) layout == DIT_ROPE_HALF ? launch<bf16_t, true>(a, s) : launch<bf16_t, false>(a, s);
  else layout == DIT_ROPE_HALF ? launch<float, true>(a, s) : launch<float, false>(a, s);
  return hipGetLastError();
}

}  // namespace dit
