// Attention over the key blocks that a cheap score selects.  A request's
// sequence is cut into blocks of kQB queries and kKB keys; for every head and
// query block a list names the key blocks it attends to.
//
// Selection: the score of (query block i, key block j) is the product of their
// means.  Means and products are in 64 bits: the answer is a list of indices,
// which must not depend on the order of a sum, and sums of 64 or 128 bf16 values
// in 64 bits are exact.  The best n of a row are found by the bits of the n-th
// largest score, from the highest down.
//
// Attention: online softmax over the listed blocks, in ascending order.
#include <float.h>
#include <math.h>

#include "device_common.h"

namespace dit {

namespace {

constexpr int kQB = kSparseQ, kKB = kSparseK;

// query block `row` (over all requests): its request and its index there
__device__ __forceinline__ int request_of(const int* off, int n, int row) {
  int r = 0;
  while (r + 1 < n && row >= off[r + 1]) ++r;
  return r;
}

// ---------------------------------------------------------------- means
// Block (unit, head): the mean of one block of keys or queries, 64 bits.
// Threads (token slot, 8 dimensions); the slots' sums meet in LDS.
template <typename T, int HD>
__global__ __launch_bounds__(256) void block_means_kernel(const T* __restrict__ q, const T* __restrict__ k, int heads,
                                                          const SparseMeta m, double* __restrict__ qm,
                                                          double* __restrict__ km) {
  constexpr int CH = HD / 8, SL = 256 / CH;
  __shared__ double part[SL][HD + 1];
  const int nkb = m.kb_off[m.n_req];
  int u = blockIdx.x;
  const int h = blockIdx.y;
  const bool keys = u < nkb;
  if (!keys) u -= nkb;
  const int* off = keys ? m.kb_off : m.qb_off;
  const int bs = keys ? kKB : kQB;
  const int r = request_of(off, m.n_req, u);
  const int L = m.off[r + 1] - m.off[r], t0 = (u - off[r]) * bs, n = min(bs, L - t0);
  const int c = threadIdx.x % CH, sl = threadIdx.x / CH;
  const T* x = (keys ? k : q) + ((long)(m.off[r] + t0) * heads + h) * HD + c * 8;
  double a[8] = {};
  for (int t = sl; t < n; t += SL) {
    const T* y = x + (long)t * heads * HD;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] += (double)to_f32<T>(y[i]);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) part[sl][c * 8 + i] = a[i];
  __syncthreads();
  if (threadIdx.x < HD) {
    double s = 0.0;
    for (int i = 0; i < SL; ++i) s += part[i][threadIdx.x];
    const long row = (long)h * off[m.n_req] + u;
    (keys ? km : qm)[row * HD + threadIdx.x] = s / n;
  }
}

// ---------------------------------------------------------------- selection
// order-preserving bits of a score: larger scores, larger keys; -0 as 0, NaN above all
__device__ __forceinline__ uint64_t score_key(double s) {
  if (s != s) return ~0ull - 1;
  s += 0.0;
  const uint64_t b = (uint64_t)__double_as_longlong(s);
  return b >> 63 ? ~b : b | (1ull << 63);
}

template <int HD>
__global__ __launch_bounds__(256) void select_blocks_kernel(const double* __restrict__ qm, const double* __restrict__ km,
                                                            const SparseMeta m, int text_first, int keep,
                                                            int* __restrict__ out) {
  __shared__ double qs[HD];
  __shared__ uint64_t key[kSparseMaxKeyBlocks];
  const int row = blockIdx.x, h = blockIdx.y;
  const int r = request_of(m.qb_off, m.n_req, row);
  const int n = m.kb_off[r + 1] - m.kb_off[r];
  const int nt = text_first ? (m.n_txt[r] + kKB - 1) / kKB : 0;
  const int tid = threadIdx.x;
  for (int i = tid; i < HD; i += 256) qs[i] = qm[((long)h * m.qb_off[m.n_req] + row) * HD + i];
  __syncthreads();
  for (int j = tid; j < n; j += 256) {
    const double* y = km + ((long)h * m.kb_off[m.n_req] + m.kb_off[r] + j) * HD;
    double s = 0.0;
    for (int i = 0; i < HD; ++i) s += qs[i] * y[i];
    key[j] = j < nt ? ~0ull : score_key(s);
  }
  __syncthreads();
  if (tid >= 64) return;
  int* o = out + ((long)h * m.qb_off[m.n_req] + row) * keep;
  const int lane = tid, want = min(keep, n);
  // t: the want-th largest key, bit by bit; done early when exactly `want` keys reach it
  uint64_t t = 0;
  if (want < n) {
    for (int bit = 63; bit >= 0; --bit) {
      const uint64_t c = t | 1ull << bit;
      int count = 0;
      for (int j = 0; j < n; j += 64) count += __popcll(__ballot(j + lane < n && key[min(j + lane, n - 1)] >= c));
      if (count >= want) t = c;
      if (count == want) break;
    }
  }
  int above = 0;
  for (int j = 0; j < n; j += 64) above += __popcll(__ballot(j + lane < n && key[min(j + lane, n - 1)] > t));
  int ties = want - above, at = 0;  // of the keys equal to t, the first `ties` belong to the answer
  for (int j = 0; j < n; j += 64) {
    const bool in = j + lane < n;
    const uint64_t k = key[min(j + lane, n - 1)];
    const uint64_t below = (1ull << lane) - 1;
    const uint64_t eq = __ballot(in && k == t);
    const bool take = in && (k > t || (k == t && __popcll(eq & below) < ties));
    const uint64_t tk = __ballot(take);
    if (take) o[at + __popcll(tk & below)] = j + lane;
    at += __popcll(tk);
    ties -= min(ties, (int)__popcll(eq));
  }
  for (int j = want + lane; j < keep; j += 64) o[j] = -1;
}

// ---------------------------------------------------------------- a query block's list
// The blocks that `keep` entries name, ascending and each once, in `list`;
// returns how many.  Entries outside [0, n) name none.  mask: kSparseMaxKeyBlocks bits.
__device__ __forceinline__ int read_list(const int* __restrict__ entries, int keep, int n, uint32_t* mask, uint16_t* list,
                                         int* count, int tid, int nt) {
  for (int i = tid; i < kSparseMaxKeyBlocks / 32; i += nt) mask[i] = 0;
  __syncthreads();
  for (int i = tid; i < keep; i += nt) {
    const uint32_t b = (uint32_t)entries[i];
    if (b < (uint32_t)n) atomicOr(&mask[b >> 5], 1u << (b & 31));
  }
  __syncthreads();
  static_assert(kSparseMaxKeyBlocks == 64 * 32, "one word per lane");
  if (tid < 64) {
    uint32_t w = mask[tid];
    int at = __popc(w);
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(at, o, 64);
      if (tid >= o) at += v;
    }
    if (tid == 63) *count = at;
    at -= __popc(w);
    for (; w; w &= w - 1) list[at++] = (uint16_t)(tid * 32 + __ffs(w) - 1);
  }
  __syncthreads();
  return *count;
}

struct SparseArgs {
  const void *q, *k, *v;
  void* o;
  const int* blocks;  // [heads][query blocks][keep]
  int keep, heads;
  float scale;
  SparseMeta meta;
};

// ---------------------------------------------------------------- bf16
// 4 waves x 32 queries.  S^T = K Q^T by v_mfma_f32_32x32x16_bf16: a lane holds
// the scores of query lane % 32 for half of the keys, and its probabilities are
// the B operand of O^T = V^T P^T.
template <int HD>
__global__ __launch_bounds__(256) void sparse_bf16_kernel(const SparseArgs a) {
  constexpr int CH = HD / 8, KP = HD + 8;  // row pitch of the tiles in LDS
  __shared__ uint4 ktile[kKB * KP / 8];
  __shared__ bf16_t vtile[kKB * KP];
  __shared__ uint32_t mask[kSparseMaxKeyBlocks / 32];
  __shared__ uint16_t list[kSparseMaxKeyBlocks];
  __shared__ int count;
  const SparseMeta& m = a.meta;
  const int nqb = m.qb_off[m.n_req];
  const int row = blockIdx.x, h = blockIdx.y;
  const int r = request_of(m.qb_off, m.n_req, row);
  const int L = m.off[r + 1] - m.off[r], q0 = (row - m.qb_off[r]) * kQB;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, hl = lane >> 5;
  const long tok = (long)a.heads * HD, base = (long)m.off[r] * tok + (long)h * HD;
  const bf16_t* Q = (const bf16_t*)a.q + base;
  const bf16_t* K = (const bf16_t*)a.k + base;
  const bf16_t* V = (const bf16_t*)a.v + base;
  const int cnt = read_list(a.blocks + ((long)h * nqb + row) * a.keep, a.keep, m.kb_off[r + 1] - m.kb_off[r], mask, list,
                            &count, tid, 256);
  const int qrow = q0 + wave * 32 + (lane & 31);
  bf16x8_t qf[HD / 16];
#pragma unroll
  for (int s = 0; s < HD / 16; ++s) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (qrow < L) u = *(const uint4*)(Q + qrow * tok + (s * 2 + hl) * 8);
    qf[s] = __builtin_bit_cast(bf16x8_t, u);
  }
  f32x16_t o[HD / 32] = {};
  float mx = -FLT_MAX, l = 0.f;
  const float sl2 = a.scale * 1.4426950408889634f;
  for (int t = 0; t < cnt; ++t) {
    const int k0 = list[t] * kKB;
    __syncthreads();
    for (int i = tid; i < kKB * CH; i += 256) {
      const int key = i / CH, c = i % CH;
      uint4 ku = make_uint4(0, 0, 0, 0), vu = ku;
      if (k0 + key < L) {
        ku = *(const uint4*)(K + (k0 + key) * tok + c * 8);
        vu = *(const uint4*)(V + (k0 + key) * tok + c * 8);
      }
      ktile[key * (KP / 8) + c] = ku;
      *(uint4*)&vtile[key * KP + c * 8] = vu;
    }
    __syncthreads();
    f32x16_t s[2] = {};
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, ktile[(b * 32 + (lane & 31)) * (KP / 8) + ks * 2 + hl]);
        s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], s[b], 0, 0, 0);
      }
    float tm = mx;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = k0 + b * 32 + (i >> 2) * 8 + hl * 4 + (i & 3);
        s[b][i] = key < L ? s[b][i] * sl2 : -INFINITY;
        tm = fmaxf(tm, s[b][i]);
      }
    tm = fmaxf(tm, __shfl_xor(tm, 32, 64));
    const float al = exp2f(mx - tm);
    mx = tm;
    l *= al;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] *= al;
#pragma unroll
    for (int g = 0; g < 4; ++g) {  // 16 keys at a time
      bf16x8_t pf;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const __bf16 p = (__bf16)exp2f(s[g >> 1][(g & 1) * 8 + i] - mx);
        pf[i] = p;
        l += (float)p;
      }
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) {
        bf16x8_t vf;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          vf[i] = __builtin_bit_cast(__bf16, vtile[(g * 16 + (i >> 2) * 8 + hl * 4 + (i & 3)) * KP + d * 32 + (lane & 31)]);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, o[d], 0, 0, 0);
      }
    }
  }
  l += __shfl_xor(l, 32, 64);
  if (qrow < L) {
    const float inv = cnt ? 1.0f / l : 0.f;
    bf16_t* og = (bf16_t*)a.o + base + qrow * tok;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        uint2 w;
        w.x = pack_bf16x2(o[d][g * 4 + 0] * inv, o[d][g * 4 + 1] * inv);
        w.y = pack_bf16x2(o[d][g * 4 + 2] * inv, o[d][g * 4 + 3] * inv);
        *(uint2*)(og + d * 32 + g * 8 + hl * 4) = w;
      }
  }
}

// ---------------------------------------------------------------- fp32 (head_dim 64)
// As the dense fp32 kernel: a block owns 16 queries, and of every listed key
// block each of its four waves takes 16 keys, with its own running max, sum and
// O, merged at the end in wave order.
constexpr int FD = 64, FQ = 16;

__global__ __launch_bounds__(256) void sparse_f32_kernel(const SparseArgs a) {
  __shared__ float osh[4][FQ][FD + 4];
  __shared__ float2 ml[4][FQ];
  __shared__ uint32_t mask[kSparseMaxKeyBlocks / 32];
  __shared__ uint16_t list[kSparseMaxKeyBlocks];
  __shared__ int count;
  const SparseMeta& m = a.meta;
  const int nqb = m.qb_off[m.n_req];
  const int row = blockIdx.x / (kQB / FQ), h = blockIdx.y;
  const int r = request_of(m.qb_off, m.n_req, row);
  const int L = m.off[r + 1] - m.off[r], q0 = (row - m.qb_off[r]) * kQB + blockIdx.x % (kQB / FQ) * FQ;
  if (q0 >= L) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, kq = lane >> 4;
  const long tok = (long)a.heads * FD, base = (long)m.off[r] * tok + (long)h * FD;
  const float *Q = (const float*)a.q + base, *K = (const float*)a.k + base, *V = (const float*)a.v + base;
  const int cnt = read_list(a.blocks + ((long)h * nqb + row) * a.keep, a.keep, m.kb_off[r + 1] - m.kb_off[r], mask, list,
                            &count, tid, 256);
  float4 q[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) q[c] = *(const float4*)(Q + min(q0 + lr, L - 1) * tok + c * 16 + kq * 4);
  const float sl2 = a.scale * 1.4426950408889634f;
  float mx = -FLT_MAX, l = 0.f;
  f32x4_t o[4] = {};
  for (int t = 0; t < cnt; ++t) {
    const int k0 = list[t] * kKB + wave * 16;
    float4 kf[4];
    float vf[4][4];
#pragma unroll
    for (int c = 0; c < 4; ++c) kf[c] = *(const float4*)(K + min(k0 + lr, L - 1) * tok + c * 16 + kq * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int c = 0; c < 4; ++c) vf[c][e] = k0 + kq * 4 + e < L ? V[(k0 + kq * 4 + e) * tok + c * 16 + lr] : 0.f;
    f32x4_t s0 = {}, s1 = {};
#pragma unroll
    for (int c = 0; c < 4; c += 2) {
      const float k0v[4] = {kf[c].x, kf[c].y, kf[c].z, kf[c].w}, q0v[4] = {q[c].x, q[c].y, q[c].z, q[c].w};
      const float k1v[4] = {kf[c + 1].x, kf[c + 1].y, kf[c + 1].z, kf[c + 1].w};
      const float q1v[4] = {q[c + 1].x, q[c + 1].y, q[c + 1].z, q[c + 1].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k0v[e], q0v[e], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k1v[e], q1v[e], s1, 0, 0, 0);
      }
    }
    float s[4], tm = mx;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[i] = k0 + kq * 4 + i < L ? (s0[i] + s1[i]) * sl2 : -INFINITY;
      tm = fmaxf(tm, s[i]);
    }
    tm = fmaxf(tm, __shfl_xor(tm, 16, 64));
    tm = fmaxf(tm, __shfl_xor(tm, 32, 64));
    const float al = exp2f(mx - tm);
    mx = tm;
    l *= al;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[i] = exp2f(s[i] - mx);
      l += s[i];
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[c][i] *= al;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int c = 0; c < 4; ++c) o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[c][e], s[e], o[c], 0, 0, 0);
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (kq == 0) ml[wave][lr] = make_float2(mx, l);
#pragma unroll
  for (int c = 0; c < 4; ++c) *(float4*)&osh[wave][lr][c * 16 + kq * 4] = make_float4(o[c][0], o[c][1], o[c][2], o[c][3]);
  __syncthreads();
  const int ql = tid >> 4, dd = (tid & 15) * 4, qrow = q0 + ql;
  if (qrow >= L) return;
  float mm = ml[0][ql].x;
#pragma unroll
  for (int w = 1; w < 4; ++w) mm = fmaxf(mm, ml[w][ql].x);
  float ls = 0.f;
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float wt = exp2f(ml[w][ql].x - mm);
    const float4 v = *(const float4*)&osh[w][ql][dd];
    ls = fmaf(wt, ml[w][ql].y, ls);
    y = make_float4(fmaf(wt, v.x, y.x), fmaf(wt, v.y, y.y), fmaf(wt, v.z, y.z), fmaf(wt, v.w, y.w));
  }
  const float inv = cnt ? 1.0f / ls : 0.f;
  *(float4*)((float*)a.o + base + qrow * tok + dd) = make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
}

}  // namespace

hipError_t launch_attention_select(int dtype, const void* q, const void* k, int heads, int head_dim, const SparseMeta& m,
                                   int text_first, int keep, double* qm, double* km, int* out, hipStream_t s) {
  const int nqb = m.qb_off[m.n_req], nkb = m.kb_off[m.n_req];
  const dim3 gm((unsigned)(nqb + nkb), (unsigned)heads), gs((unsigned)nqb, (unsigned)heads);
#define DIT_MEANS(T, HD)                                                                                            \
  hipLaunchKernelGGL((block_means_kernel<T, HD>), gm, dim3(256), 0, s, (const T*)q, (const T*)k, heads, m, qm, km)
  if (dtype == DIT_F32) DIT_MEANS(float, 64);
  else if (head_dim == 64) DIT_MEANS(bf16_t, 64);
  else DIT_MEANS(bf16_t, 128);
#undef DIT_MEANS
  if (head_dim == 64)
    hipLaunchKernelGGL(select_blocks_kernel<64>, gs, dim3(256), 0, s, qm, km, m, text_first, keep, out);
  else
    hipLaunchKernelGGL(select_blocks_kernel<128>, gs, dim3(256), 0, s, qm, km, m, text_first, keep, out);
  return hipGetLastError();
}

hipError_t launch_attention_sparse(int dtype, const void* q, const void* k, const void* v, const int* blocks, int keep,
                                   int heads, int head_dim, const SparseMeta& m, void* o, hipStream_t s) {
  SparseArgs a;
  a.q = q;
  a.k = k;
  a.v = v;
  a.o = o;
  a.blocks = blocks;
  a.keep = keep;
  a.heads = heads;
  a.scale = 1.0f / sqrtf((float)head_dim);
  a.meta = m;
  const int nqb = m.qb_off[m.n_req];
  if (dtype == DIT_F32)
    hipLaunchKernelGGL(sparse_f32_kernel, dim3((unsigned)nqb * (kQB / FQ), (unsigned)heads), dim3(256), 0, s, a);
  else if (head_dim == 64)
    hipLaunchKernelGGL(sparse_bf16_kernel<64>, dim3((unsigned)nqb, (unsigned)heads), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL(sparse_bf16_kernel<128>, dim3((unsigned)nqb, (unsigned)heads), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace dit
