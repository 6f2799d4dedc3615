// Attention over the key blocks that a cheap score selects.  A request's
// sequence is cut into blocks of kQB queries and kKB keys; for every head and
// query block a list names the key blocks it attends to.
//
// Selection: the score of (query block i, key block j) is the product of their
// means.  Means and products are in 64 bits: the answer is a list of indices, which
// roundings of 32 bits would change.  A mean's sum is exact for bf16 blocks whose
// magnitudes lie within 2^38 of each other; wider ones, fp32 inputs, the division of a
// shorter last block and the products round, in a fixed order, so that lists repeat, but
// two blocks of the same tokens in another order may differ in a last place.  The best n
// of a row are found by the bits of the n-th largest score, from the highest down.
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
// Where the mean of key block u (over all requests) has dimension d (even) of
// head h: in the order in which the matrix cores take it, 16 blocks at a time, so
// that the lanes of a wave load neighbouring words.  (From rows, 16 lanes would
// each start a row of their own: 80 accesses of the vector cache a load, 208 us
// at 516 x 1032 blocks and 24 heads.)
__device__ __forceinline__ long key_mean_at(const SparseMeta& m, int hd, int h, int u, int d) {
  const long tile = (long)h * ((m.kb_off[m.n_req] + 15) >> 4) + (u >> 4);
  return ((tile * (hd >> 3) + (d >> 3)) * 64 + (d >> 1 & 3) * 16 + (u & 15)) * 2;
}

// Block (key or query block, 512 columns of [heads, head_dim]): its mean, 64
// bits.  A wave reads 1 KB of a token's row at a time and takes every eighth
// token; the waves' sums meet in LDS.  Every element of Q and K is read once, and
// that bounds it: 170 us for 66048 tokens of 24 heads of 128, 4.8 TB/s, what a large
// copy reaches (4.8 - 5.4 by card, reads and writes).
template <typename T>
__global__ __launch_bounds__(512) void block_means_kernel(const T* __restrict__ q, const T* __restrict__ k, int heads,
                                                          int hd, const SparseMeta m, double* __restrict__ qm,
                                                          double* __restrict__ km) {
  __shared__ double part[8][8][65];
  const int nkb = m.kb_off[m.n_req];
  int u = blockIdx.x;
  const bool keys = u < nkb;
  if (!keys) u -= nkb;
  const int* off = keys ? m.kb_off : m.qb_off;
  const int bs = keys ? kKB : kQB;
  const int r = request_of(off, m.n_req, u);
  const int L = m.off[r + 1] - m.off[r], t0 = (u - off[r]) * bs, n = min(bs, L - t0);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int width = heads * hd, col = (blockIdx.y * 64 + lane) * 8;
  double a[8] = {};
  if (col < width) {
    const T* x = (keys ? k : q) + (long)(m.off[r] + t0) * width + col;
#pragma unroll 1
    for (int t = wave; t < n; t += 64) {
      float v[8][8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int tt = min(t + 8 * i, n - 1);  // past the end: the last token again, not added
        if constexpr (sizeof(T) == 2) {
          const uint4 w = *(const uint4*)(x + (long)tt * width);
          const uint32_t e[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            v[i][2 * c] = __uint_as_float(e[c] << 16);
            v[i][2 * c + 1] = __uint_as_float(e[c] & 0xffff0000u);
          }
        } else {
          *(float4*)&v[i][0] = ((const float4*)(x + (long)tt * width))[0];
          *(float4*)&v[i][4] = ((const float4*)(x + (long)tt * width))[1];
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (t + 8 * i < n) {
#pragma unroll
          for (int c = 0; c < 8; ++c) a[c] += (double)v[i][c];
        }
    }
  }
#pragma unroll
  for (int c = 0; c < 8; ++c) part[wave][c][lane] = a[c];
  __syncthreads();
  // two neighbouring columns per thread
  if (threadIdx.x >= 256) return;
  const int chunk = threadIdx.x >> 2, c = (threadIdx.x & 3) * 2, e = (blockIdx.y * 64 + chunk) * 8 + c;
  if (e >= width) return;
  double2 s = make_double2(0.0, 0.0);
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    s.x += part[w][c][chunk];
    s.y += part[w][c + 1][chunk];
  }
  const int h = e / hd, d = e - h * hd;
  const double2 mean = make_double2(s.x / n, s.y / n);
  if (keys) *(double2*)(km + key_mean_at(m, hd, h, u, d)) = mean;
  else *(double2*)(qm + ((long)h * m.qb_off[m.n_req] + u) * hd + d) = mean;
}

// ---------------------------------------------------------------- selection
// order-preserving bits of a score: larger scores, larger keys; -0 as 0, NaN above all; never 0
__device__ __forceinline__ uint64_t score_key(double s) {
  if (s != s) return ~0ull - 1;
  s += 0.0;
  const uint64_t b = (uint64_t)__double_as_longlong(s);
  return b >> 63 ? ~b : b | (1ull << 63);
}

struct SelectRows {
  int off[kMaxReq + 1];  // groups of query blocks of one request
};
typedef double f64x4_t __attribute__((ext_vector_type(4)));

// how many of the wave's keys are at least c (c > 0; a key that does not count is 0)
template <int NV>
__device__ __forceinline__ int count_from(const uint32_t* key, uint32_t c) {
  int count = 0;
#pragma unroll
  for (int v = 0; v < NV; ++v) count += __popcll(__ballot(key[v] >= c));
  return count;
}
// The largest t that at least `want` keys reach, bit by bit; *exact: exactly so many do (which ends the search early).
template <int NV>
__device__ __forceinline__ uint32_t nth_largest(const uint32_t* key, int want, bool* exact) {
  uint32_t t = 0;
  *exact = false;
  for (uint32_t bit = 1u << 31; bit; bit >>= 1) {
    const int count = count_from<NV>(key, t | bit);
    if (count >= want) t |= bit;
    if (count == want) {
      *exact = true;
      break;
    }
  }
  return t;
}
// the high word's score, its low word taken as 0
__device__ __forceinline__ double key_score(uint32_t hi) {
  const uint32_t b = hi >> 31 ? hi ^ 0x80000000u : ~hi;
  return __longlong_as_double((long long)((uint64_t)b << 32));
}
// A t that exactly `want` keys reach, by halving the interval of the scores: about
// as many steps as bits tell the want-th score from the next (10 of 1000 normal
// ones), where the search over the keys' bits also walks through the exponent.  0
// where it ends without one: equal high words, infinities, NaN.
template <int NV>
__device__ __forceinline__ uint32_t halve_scores(const uint32_t* key, int want) {
  uint32_t lo = ~0u, hi = 0;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    lo = min(lo, key[v] - 1);  // keys that do not count: the largest
    hi = max(hi, key[v]);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, 64));
    hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, 64));
  }
  double a = key_score(lo + 1), b = key_score(hi);
  for (int i = 0; i < 24; ++i) {
    const double mid = 0.5 * (a + b);
    if (!(mid > a && mid < b)) break;
    const uint32_t c = (uint32_t)(score_key(mid) >> 32);
    const int count = count_from<NV>(key, c);
    if (count == want) return c;
    if (count > want) a = mid;
    else b = mid;
  }
  return 0;
}

// NW waves, up to R query blocks of one request and head.  Scores by the 64-bit
// matrix cores (v_mfma_f64_16x16x4_f64: 16 key blocks x 16 query blocks; of every 8
// dimensions a lane quarter holds two, in the same order on both sides),
// kept in LDS as order-preserving integers, high and low words apart.  Then a
// wave takes a query block, 64 NV scores in registers, and finds the keep-th
// largest: by the high words, and by the low words among equal ones.
// 516 x 1032 scores of 24 heads of 128: 137 us, of which the matrix cores need 55
// (59 TFLOP/s); the rest is the search's counting, one block a CU (208 us with the
// key means in rows, 162 with a search by bits alone).  Small calls are latency:
// 35 x 70 scores of 24 heads about 6 us.
template <int HD, int NV, int R, int NW>
__global__ __launch_bounds__(NW * 64) void select_blocks_kernel(const double* __restrict__ qm,
                                                                const double* __restrict__ km, const SparseMeta m,
                                                                const SelectRows g, int text_first, int keep,
                                                                int* __restrict__ out) {
  constexpr int N = NV * 64;
  __shared__ uint32_t high[R][N], low[R][N];
  const int groups = g.off[m.n_req];
  // blocks of one XCD take consecutive units, head by head: its L2 holds their key means
  const int unit = xcd_remap(blockIdx.x, gridDim.x);
  const int h = unit / groups, id = unit - h * groups;
  const int r = request_of(g.off, m.n_req, id);
  const int row0 = m.qb_off[r] + (id - g.off[r]) * R, rows = min(R, m.qb_off[r + 1] - row0);
  const int n = m.kb_off[r + 1] - m.kb_off[r];
  const int nt = text_first ? (m.n_txt[r] + kKB - 1) / kKB : 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lr = lane & 15, lq = lane >> 4;
  {
    double2 q[HD / 8];
    const double* qs = qm + ((long)h * m.qb_off[m.n_req] + row0 + min(lr, rows - 1)) * HD + lq * 2;
#pragma unroll
    for (int i = 0; i < HD / 8; ++i) q[i] = *(const double2*)(qs + 8 * i);
    const int k0 = m.kb_off[r];
    const double* ks = km + key_mean_at(m, HD, h, 0, 0) + lane * 2;
    for (int t = (k0 >> 4) + wave; t * 16 < k0 + n; t += NW) {
      const double* y = ks + (long)t * HD * 16;
      f64x4_t s = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
      for (int i = 0; i < HD / 8; ++i) {
        const double2 kv = *(const double2*)(y + i * 128);
        s = __builtin_amdgcn_mfma_f64_16x16x4f64(kv.x, q[i].x, s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f64_16x16x4f64(kv.y, q[i].y, s, 0, 0, 0);
      }
      if (lr < rows)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = t * 16 + lq + 4 * e - k0;  // the first and the last tile hold other requests' blocks, too
          if (key >= 0 && key < n) {
            const uint64_t b = score_key(s[e]);
            high[lr][key] = (uint32_t)(b >> 32);
            low[lr][key] = (uint32_t)b;
          }
        }
    }
  }
  __syncthreads();
  const int want = min(keep, n);
  for (int row = wave; row < rows; row += NW) {
    int* o = out + ((long)h * m.qb_off[m.n_req] + row0 + row) * keep;
    // The text's blocks, then the best of the others: `best` of them.  Keys that take no part are 0.
    uint32_t hi[NV], lo[NV], t = 1, tl = 0;
    const int text = min(nt, want), best = want - text;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int key = v * 64 + lane;
      const bool in = key >= nt && key < n && best > 0;
      hi[v] = in ? high[row][key] : 0;
      lo[v] = in ? low[row][key] : 0;
    }
    bool exact = true;
    int ties = 0;  // of the keys equal to (t, tl), as many belong to the answer
    if (best > 0 && want < n) {
      t = halve_scores<NV>(hi, best);
      if (t == 0) t = nth_largest<NV>(hi, best, &exact);
    }
    if (!exact) {
      uint32_t l[NV];
#pragma unroll
      for (int v = 0; v < NV; ++v) l[v] = hi[v] == t ? lo[v] : 0;
      const int above = t == ~0u ? 0 : count_from<NV>(hi, t + 1);
      bool found;
      tl = nth_largest<NV>(l, best - above, &found);
      ties = best - above;
#pragma unroll
      for (int v = 0; v < NV; ++v) ties -= __popcll(__ballot(hi[v] == t && lo[v] > tl));
    }
    int at = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const uint64_t below = (1ull << lane) - 1;
      bool take = hi[v] >= t;
      if (!exact) {
        const bool same = hi[v] == t && lo[v] == tl;
        const uint64_t eq = __ballot(same);
        take = hi[v] > t || (hi[v] == t && lo[v] > tl) || (same && __popcll(eq & below) < ties);
        ties -= min(ties, (int)__popcll(eq));
      }
      take = take || v * 64 + lane < text;
      const uint64_t tk = __ballot(take);
      if (take) o[at + __popcll(tk & below)] = v * 64 + lane;
      at += __popcll(tk);
    }
    for (int j = want + lane; j < keep; j += 64) o[j] = -1;
  }
}

template <int HD, int NV, int R, int NW>
void launch_select(const double* qm, const double* km, int heads, const SparseMeta& m, int text_first, int keep, int* out,
                   hipStream_t s) {
  SelectRows g{};
  for (int r = 0; r < m.n_req; ++r) g.off[r + 1] = g.off[r] + (m.qb_off[r + 1] - m.qb_off[r] + R - 1) / R;
  hipLaunchKernelGGL((select_blocks_kernel<HD, NV, R, NW>), dim3((unsigned)g.off[m.n_req] * heads), dim3(NW * 64), 0, s,
                     qm, km, m, g, text_first, keep, out);
}

// Query blocks per thread block: 16, which fill the matrix cores' columns; 4 where
// the scores are few (under 2^19), which spreads them over more CUs; 8 where 16
// rows of scores exceed LDS.  Both launches of a call in us, 4 against 16 (query
// blocks times heads x key blocks): 840 x 70 14.4 against 20.4, 1512 x 125 20.5
// against 25.9, 4032 x 125 38.2 against 40.2; 8064 x 125 78.1 against 73.6, 3168 x
// 264 69.0 against 61.1, 12384 x 1032 453 against 302 (means 170 of it).  Past 320
// key blocks, 516 x 344 28.8 against 33.9 and 1032 x 344 equal: not worth a kernel.
// Up to 576 key blocks two thread blocks fit a CU, one searching while the other
// multiplies: 6768 x 563 135 us against 148 with room for 1088 each.
template <int HD>
void launch_select(const double* qm, const double* km, int heads, const SparseMeta& m, int text_first, int keep, int* out,
                   hipStream_t s) {
  int n = 0;
  for (int r = 0; r < m.n_req; ++r) n = std::max(n, m.kb_off[r + 1] - m.kb_off[r]);
  const bool few = (long)m.qb_off[m.n_req] * heads * n < 1 << 19;
  if (n <= 128) {
    if (few) launch_select<HD, 2, 4, 8>(qm, km, heads, m, text_first, keep, out, s);
    else launch_select<HD, 2, 16, 4>(qm, km, heads, m, text_first, keep, out, s);
  } else if (n <= 320) {
    if (few) launch_select<HD, 5, 4, 8>(qm, km, heads, m, text_first, keep, out, s);
    else launch_select<HD, 5, 16, 4>(qm, km, heads, m, text_first, keep, out, s);
  } else if (n <= 576) {
    launch_select<HD, 9, 16, 8>(qm, km, heads, m, text_first, keep, out, s);
  } else if (n <= 1088) {
    launch_select<HD, 17, 16, 16>(qm, km, heads, m, text_first, keep, out, s);
  } else {
    launch_select<HD, 32, 8, 16>(qm, km, heads, m, text_first, keep, out, s);
  }
}

// ---------------------------------------------------------------- a query block's list
// The blocks that `keep` entries name, ascending and each once, in `list`;
// returns how many.  Entries outside [0, n) name none.  Entries that ascend
// already, with none out of range but at the end, as the selection writes them,
// are taken as they stand (one barrier); others pass through a bit mask.
// scratch: a word for the count, one for each of up to 8 waves, kSparseMaxKeyBlocks bits.
__device__ __forceinline__ int read_list(const int* __restrict__ entries, int keep, int n, uint32_t* scratch, uint16_t* list,
                                         int tid, int nt) {
  uint32_t *const count = scratch, *const plain = scratch + 1, *const mask = scratch + 9;
  auto in_range = [&](int i) { return i < keep && (uint32_t)entries[min(i, keep - 1)] < (uint32_t)n; };
  bool ok = true;
  for (int i = tid; i < keep; i += nt) {
    const bool in = in_range(i);
    const int b = entries[i];
    if (in) {
      ok = ok && (i == 0 || (in_range(i - 1) && entries[i - 1] < b));
      list[i] = (uint16_t)b;
      if (!in_range(i + 1)) *count = i + 1;  // one thread of an ascending list
    } else if (i == 0) {
      *count = 0;
    }
  }
  const uint64_t all = __ballot(ok);
  if ((tid & 63) == 0) plain[tid >> 6] = all == __ballot(true);
  __syncthreads();
  uint32_t every = 1;
  for (int w = 0; w < nt / 64; ++w) every &= plain[w];
  if (every) return *count;
  __syncthreads();
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
constexpr int kListScratch = (9 + kSparseMaxKeyBlocks / 32) * 4;  // bytes

struct SparseArgs {
  const void *q, *k, *v;
  void* o;
  const int* blocks;  // [heads][query blocks][keep]
  int keep, heads;
  float scale;
  SparseMeta meta;
};

// ---------------------------------------------------------------- bf16
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));

// A query's running max is raised only when a tile's probabilities against it sum to
// more than 2^8 in one of its two lanes: up to there fp32 and bf16 hold them as well as
// any.  Each query decides for itself, so its bits do not depend on its neighbours.
constexpr float kLazyMax = 256.0f;

__device__ __forceinline__ void wait_vmcnt0_lgkmcnt0() { __builtin_amdgcn_s_waitcnt(7 << 4); }

// N MFMAs, each after R LDS reads of its own: the reads of A MFMAs stay ahead
template <int N, int R, int A>
__device__ __forceinline__ void read_ahead() {
  __builtin_amdgcn_sched_group_barrier(0x100, A * R, 0);
  static_for<N - A>([&](auto) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
  });
  __builtin_amdgcn_sched_group_barrier(0x008, A, 0);
}

// 4 waves x 32 queries.  S^T = K Q^T by v_mfma_f32_32x32x16_bf16: a lane holds
// the scores of query lane % 32 for half of the keys, and its probabilities are
// the B operand of O^T = V^T P^T.  K and V blocks arrive as they lie in memory,
// by direct-to-LDS loads into two stages, the next listed block's while this one
// is worked on; V is transposed on its way from LDS to the matrix cores
// (ds_read_b64_tr_b16: 16 lanes take a block of 4 keys x 16 dimensions, each lane
// the 4 keys of one dimension), so no copy of V is made and the keys a lane gets
// are those whose probabilities it holds.
//
// 16896 tokens, 24 heads of 128, lists of 33: 448 - 463 us, 0.95 - 0.98 PFLOP/s; three requests
// of 589 + 1357 + 4429 tokens, 12 heads of 64, lists of 16: 33.5 us.  The matrix cores are
// busy half of the time, vector arithmetic (an exponential, a multiply-add, a
// rounding and a sum per score) for most of the other; neither fewer LDS reads (64
// queries a wave, head_dim 64: 254 -> 266 us at 16896 tokens) nor a fourth wave per
// SIMD (247 -> 245) helps.
//
// KG = 2: two such groups of 4 waves halve the list between them, each with LDS
// stages of its own; the second hands its O, max and sum to the first through LDS
// at the end.
template <int HD, int KG>
__global__ __launch_bounds__(KG * 256) __attribute__((amdgpu_waves_per_eu(HD == 64 && KG == 1 ? 3 : 2)))
void sparse_bf16_kernel(const SparseArgs a) {
  constexpr int CH = HD / 8;           // 16-byte chunks of a row
  constexpr int RPI = 64 / CH;         // rows per wave load
  constexpr int NI = kKB / RPI / 4;    // loads of a tile per wave
  constexpr int ROWB = HD * 2, TILE = kKB * ROWB, STAGE = 2 * TILE;
  // [stage][K tile | V tile], then the list.  One array: with several the compiler waits for all loads ahead of every
  // read of LDS.
  constexpr int LIST = KG * 2 * STAGE, SCRATCH = LIST + kSparseMaxKeyBlocks * 2;
  __shared__ uint4 smem[(SCRATCH + kListScratch + 15) / 16];
  uint16_t* const list = (uint16_t*)((char*)smem + LIST);
  const SparseMeta& m = a.meta;
  const int nqb = m.qb_off[m.n_req];
  // blocks of one XCD take consecutive units, head by head: its L2 holds their K and V
  const int unit = xcd_remap(blockIdx.x, gridDim.x);
  const int h = unit / nqb, row = unit - h * nqb;
  const int r = request_of(m.qb_off, m.n_req, row);
  const int L = m.off[r + 1] - m.off[r], q0 = (row - m.qb_off[r]) * kQB, nkb = m.kb_off[r + 1] - m.kb_off[r];
  const int tid = threadIdx.x, lane = tid & 63, hl = lane >> 5;
  const int kg = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 8);     // key group
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) - kg * 4;        // of its group
  char* const lbase = (char*)smem + kg * 2 * STAGE;
  const long tok = (long)a.heads * HD, base = (long)m.off[r] * tok + (long)h * HD;
  const bf16_t* Q = (const bf16_t*)a.q + base;
  const bf16_t* K = (const bf16_t*)a.k + base;
  const bf16_t* V = (const bf16_t*)a.v + base;

  // slot of chunk c of K row `key`: the 16 rows of a fragment read lie in 16 different 16-byte bank groups
  auto kswz = [](int key, int c) { return HD == 128 ? c ^ (key & 15) : c ^ ((key >> 1) & 7); };
  // of V row `key`: the 64-byte segments of 4 neighbouring rows lie in 4 different quarters of the banks
  auto vswz = [](int key, int c) { return HD == 128 ? c ^ ((key & 3) << 2) : c ^ ((key & 2) << 1); };
  int ko[NI], vo[NI];  // global byte offsets of this lane's loads inside a tile
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int key = (wave * NI + i) * RPI + lane / CH;
    ko[i] = (key * (int)tok + kswz(key, lane % CH) * 8) * 2;
    vo[i] = (key * (int)tok + vswz(key, lane % CH) * 8) * 2;
  }
  auto tile_load = [&](int b, auto stc) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value;
    const int k0 = b * kKB;
    const int bytes = ((min(L - k0, kKB) - 1) * (int)tok + HD) * 2;  // keys past L read as zeros
    const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc((void*)(K + k0 * tok), (short)0, bytes, kBufferWord3);
    const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc((void*)(V + k0 * tok), (short)0, bytes, kBufferWord3);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int o = ko[i];
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rk, (__attribute__((address_space(3))) void*)(lbase + st * STAGE + (wave * NI + i) * 1024), 16, o, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int o = vo[i];
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rv, (__attribute__((address_space(3))) void*)(lbase + st * STAGE + TILE + (wave * NI + i) * 1024), 16, o, 0, 0, 0);
    }
  };
  auto block_at = [&](int i) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane((int)list[i]); };
  using S0 = std::integral_constant<int, 0>;
  using S1 = std::integral_constant<int, 1>;
  // the first block's loads ahead of the list, on the guess that it is the first entry
  const int* const entries = a.blocks + ((long)h * nqb + row) * a.keep;
  const int first = __builtin_amdgcn_readfirstlane(entries[0]);
  if ((uint32_t)first < (uint32_t)nkb && kg == 0) tile_load(first, S0{});
  const int qrow = q0 + wave * 32 + (lane & 31);
  bf16x8_t qf[HD / 16];
#pragma unroll
  for (int s = 0; s < HD / 16; ++s) {
    uint4 u = make_uint4(0, 0, 0, 0);
    if (qrow < L) u = *(const uint4*)(Q + qrow * tok + (s * 2 + hl) * 8);
    qf[s] = __builtin_bit_cast(bf16x8_t, u);
  }
  const int all = __builtin_amdgcn_readfirstlane(
      read_list(entries, a.keep, nkb, (uint32_t*)((char*)smem + SCRATCH), list, tid, KG * 256));
  // this group's part of the list: the first half, rounded up, or the rest
  const int half = (all + KG - 1) / KG, begin = kg * half, cnt = KG == 1 ? all : min(begin + half, all);
  if (begin < cnt && (kg > 0 || block_at(0) != first)) {
    wait_vmcnt0_lgkmcnt0();  // the guess lands first
    tile_load(block_at(begin), S0{});
  }

  f32x16_t o[HD / 32] = {};
  float mx = -FLT_MAX, l = 0.f;  // a finite start: keys whose scores are all -inf add nothing
  const float sl2 = a.scale * 1.4426950408889634f;
  // LDS byte offsets of this lane's fragment reads: K row lane % 32, chunk 2 ks + hl; V rows hl * 4 + lane % 16 / 4,
  // dimensions 32 db + lane / 16 % 2 * 16 + lane % 4 * 4
  int kf[HD / 16], vf[HD / 32];
#pragma unroll
  for (int ks = 0; ks < HD / 16; ++ks) kf[ks] = (lane & 31) * ROWB + kswz(lane & 31, ks * 2 + hl) * 16;
#pragma unroll
  for (int db = 0; db < HD / 32; ++db) {
    const int key = hl * 4 + (lane & 15) / 4;
    vf[db] = TILE + key * ROWB + vswz(key, db * 4 + (lane >> 4 & 1) * 2 + (lane & 3) / 2) * 16 + (lane & 1) * 8;
  }
  auto step = [&](int b, int next, auto stc, auto maskc) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value;
    if (next >= 0) tile_load(next, std::integral_constant<int, st ^ 1>{});
    f32x16_t s[2] = {};
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const bf16x8_t u = __builtin_bit_cast(bf16x8_t, *(const uint4*)(lbase + kf[ks] + st * STAGE + kb * 32 * ROWB));
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(u, qf[ks], s[kb], 0, 0, 0);
      }
    read_ahead<2 * HD / 16, 1, 4>();
    if constexpr (decltype(maskc)::value) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (b * kKB + kb * 32 + (i >> 2) * 8 + hl * 4 + (i & 3) >= L) s[kb][i] = -INFINITY;
    }
    // probabilities against the running max, rounded to bf16 in the order of the scores; the sum is of the rounded ones
    bf16x8_t pf[4];
    auto probabilities = [&]() __attribute__((always_inline)) {
      float t0 = 0.f, t1 = 0.f;
      const bf16x2_t one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = (g & 1) * 8 + 2 * e;
          const float p0 = __builtin_amdgcn_exp2f(fmaf(s[g >> 1][i], sl2, -mx));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(s[g >> 1][i + 1], sl2, -mx));
          const bf16x2_t pk = {(__bf16)p0, (__bf16)p1};
          if (e & 1) t1 = __builtin_amdgcn_fdot2_f32_bf16(pk, one, t1, false);
          else t0 = __builtin_amdgcn_fdot2_f32_bf16(pk, one, t0, false);
          w[e] = __builtin_bit_cast(uint32_t, pk);
        }
        pf[g] = __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3]));
      }
      return t0 + t1;
    };
    float t = probabilities();
    const bool high = !(t <= kLazyMax);
    if (__any(high)) {
      // a query's two lanes decide alike; the other queries keep their max, and with it their bits
      const bool raise = (int)high | __shfl_xor((int)high, 32, 64);  // every lane takes part in the exchange
      float tm = s[0][0];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) tm = fmaxf(tm, s[kb][i]);
      tm = fmaxf(mx, fmaxf(tm, __shfl_xor(tm, 32, 64)) * sl2);
      const float al = raise ? __builtin_amdgcn_exp2f(mx - tm) : 1.0f;
      mx = raise ? tm : mx;
      l *= al;
#pragma unroll
      for (int db = 0; db < HD / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= al;
      t = probabilities();
    }
    l += t;
#pragma unroll
    for (int g = 0; g < 4; ++g)
#pragma unroll
      for (int db = 0; db < HD / 32; ++db) {
        bf16x4_t v[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
          v[e] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
              (__attribute__((address_space(3))) bf16x4_t*)(lbase + vf[db] + st * STAGE + (g * 16 + e * 8) * ROWB));
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7), pf[g],
                                                        o[db], 0, 0, 0);
      }
    read_ahead<4 * HD / 32, 2, 2>();
    // this wave's loads have landed and its reads returned; behind the barrier everyone's have
    wait_vmcnt0_lgkmcnt0();
    asm volatile("s_barrier" ::: "memory");
  };
  wait_vmcnt0_lgkmcnt0();
  asm volatile("s_barrier" ::: "memory");
  using NoMask = std::false_type;
  using Mask = std::true_type;
  // only a request's last block, which is the last of its list, can hold keys past L
  const int whole = begin < cnt && L % kKB != 0 && block_at(cnt - 1) == nkb - 1 ? cnt - 1 : cnt;
  int j = begin, b = begin < cnt ? block_at(begin) : 0;
  auto after = [&](int i) __attribute__((always_inline)) { return i + 1 < cnt ? block_at(i + 1) : -1; };
  for (; j + 1 < whole; j += 2) {
    const int b1 = after(j);
    step(b, b1, S0{}, NoMask{});
    b = after(j + 1);
    step(b1, b, S1{}, NoMask{});
  }
  if (j < whole) {
    const int b1 = after(j);
    step(b, b1, S0{}, NoMask{});
    b = b1;
    ++j;
  }
  if (j < cnt) {
    if (((j - begin) & 1) == 0) step(b, -1, S0{}, Mask{});
    else step(b, -1, S1{}, Mask{});
  }
  if constexpr (KG > 1) {
    // at most one block fewer in the second group, which still meets the barrier
    if (cnt - begin < half) asm volatile("s_barrier" ::: "memory");
    // [wave][register][lane] over the tiles, which nobody reads any more
    constexpr int NR = HD / 2;
    static_assert(4 * (NR + 2) * 64 * 4 <= LIST, "merge LDS");
    float* const sh = (float*)smem + wave * (NR + 2) * 64 + lane;
    if (kg == 1) {
#pragma unroll
      for (int d = 0; d < HD / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) sh[(d * 16 + i) * 64] = o[d][i];
      sh[NR * 64] = mx;
      sh[(NR + 1) * 64] = l;
    }
    __syncthreads();
    if (kg == 1) return;
    // a group without a block has the lowest max, sum 0 and O 0
    const float m1 = sh[NR * 64], mm = fmaxf(mx, m1);
    const float a0 = __builtin_amdgcn_exp2f(mx - mm), a1 = __builtin_amdgcn_exp2f(m1 - mm);
    l = l * a0 + sh[(NR + 1) * 64] * a1;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = o[d][i] * a0 + sh[(d * 16 + i) * 64] * a1;
  }
  l += __shfl_xor(l, 32, 64);
  if (qrow < L) {
    const float inv = all ? 1.0f / l : 0.f;
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
// On the fp32 matrix cores (v_mfma_f32_16x16x4_f32).  A block owns 16 queries; of
// every listed key block each of its four waves takes 16 keys, with its own running
// max, sum and O, merged at the end in wave order.  K and V go straight from memory
// to registers, in 16-byte pieces: a lane's piece of V holds 4 neighbouring
// dimensions of a key, each a row of another MFMA.  The next block's K replaces
// this one's once the scores are done, its V once O is.
// Measured: 4429 tokens x 24 heads, lists of 18, 376 - 390 us (82 TF; 498 us with loads
// where they are used and V in single words), the dense kernel 75 TF; 288 tokens,
// lists of 2: 6.8 us.  32 queries a block halve the reads and measure the same
// (379; 589 tokens x 6 heads, lists of 8: 20.4 against 14.2): matrix cores and
// softmax bound it.
constexpr int FD = 64, FQ = 16;

__global__ __launch_bounds__(256) void sparse_f32_kernel(const SparseArgs a) {
  __shared__ float osh[4][FQ][FD + 4];
  __shared__ float2 ml[4][FQ];
  __shared__ uint32_t scratch[kListScratch / 4];
  __shared__ uint16_t list[kSparseMaxKeyBlocks];
  constexpr int PER = kQB / FQ;  // blocks of a query block
  const SparseMeta& m = a.meta;
  const int nqb = m.qb_off[m.n_req];
  const int row = blockIdx.x / PER, h = blockIdx.y;
  const int r = request_of(m.qb_off, m.n_req, row);
  const int L = m.off[r + 1] - m.off[r], q0 = (row - m.qb_off[r]) * kQB + blockIdx.x % PER * FQ;
  if (q0 >= L) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, kq = lane >> 4;
  const long tok = (long)a.heads * FD, base = (long)m.off[r] * tok + (long)h * FD;
  const float *Q = (const float*)a.q + base, *K = (const float*)a.k + base, *V = (const float*)a.v + base;
  float4 q[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) q[c] = *(const float4*)(Q + min(q0 + lr, L - 1) * tok + c * 16 + kq * 4);
  const int cnt = read_list(a.blocks + ((long)h * nqb + row) * a.keep, a.keep, m.kb_off[r + 1] - m.kb_off[r], scratch,
                            list, tid, 256);
  const float sl2 = a.scale * 1.4426950408889634f;
  float4 kf[4], vf[4];  // K: dims 16 c + 4 kq .. of key lr; V: dims 4 lr .. of key 4 kq + e (zeros past L)
  auto load_k = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < 4; ++c) kf[c] = *(const float4*)(K + min(k0 + lr, L - 1) * tok + c * 16 + kq * 4);
  };
  auto load_v = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int key = k0 + kq * 4 + e;
      vf[e] = *(const float4*)(V + min(key, L - 1) * tok + lr * 4);
      if (key >= L) vf[e] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
  };
  auto at = [](const float4& v, auto ec) __attribute__((always_inline)) {
    constexpr int e = decltype(ec)::value;
    return e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w;
  };
  float mx = -FLT_MAX, l = 0.f;
  f32x4_t o[4];  // element r of o[c]: dim 16 kq + 4 r + c of query lr
#pragma unroll
  for (int c = 0; c < 4; ++c) o[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (cnt > 0) {
    load_k(list[0] * kKB + wave * 16);
    load_v(list[0] * kKB + wave * 16);
  }
  for (int t = 0; t < cnt; ++t) {
    const int k0 = list[t] * kKB + wave * 16, next = t + 1 < cnt ? list[t + 1] * kKB + wave * 16 : -1;
    f32x4_t s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
    for (int c = 0; c < 4; c += 2)
      static_for<4>([&](auto ec) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(at(kf[c], ec), at(q[c], ec), s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(at(kf[c + 1], ec), at(q[c + 1], ec), s1, 0, 0, 0);
      });
    if (next >= 0) load_k(next);
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
      s[i] = exp2f(s[i] - tm);
      l += s[i];
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[c][i] *= al;
    static_for<4>([&](auto ec) {
      constexpr int e = decltype(ec)::value;
      static_for<4>([&](auto cc) {
        constexpr int c = decltype(cc)::value;
        o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(at(vf[e], cc), s[e], o[c], 0, 0, 0);
      });
    });
    if (next >= 0) load_v(next);
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (kq == 0) ml[wave][lr] = make_float2(mx, l);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *(float4*)&osh[wave][lr][kq * 16 + i * 4] = make_float4(o[0][i], o[1][i], o[2][i], o[3][i]);
  __syncthreads();
  // 16 lanes per query, 4 dims each.  A wave whose keys all lie past L has the lowest max, and weighs nothing.
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
  const dim3 grid((unsigned)(m.qb_off[m.n_req] + m.kb_off[m.n_req]), (unsigned)((heads * head_dim + 511) / 512));
  if (dtype == DIT_F32)
    hipLaunchKernelGGL(block_means_kernel<float>, grid, dim3(512), 0, s, (const float*)q, (const float*)k, heads, head_dim, m,
                       qm, km);
  else
    hipLaunchKernelGGL(block_means_kernel<bf16_t>, grid, dim3(512), 0, s, (const bf16_t*)q, (const bf16_t*)k, heads,
                       head_dim, m, qm, km);
  if (head_dim == 64) launch_select<64>(qm, km, heads, m, text_first, keep, out, s);
  else launch_select<128>(qm, km, heads, m, text_first, keep, out, s);
  return hipGetLastError();
}

// Two key groups where every block has a CU to itself and 8 blocks or more to
// attend to.  Measured, one group against two: 105 units of lists of 35, 44.1
// against 37.0 us; 189 of 60, 67.9 against 56.6; 210 of 12, 22.1 against 21.5; lists
// of 8 are equal (15.7).  Past 256 units the second group would wait for the first.
template <int HD>
static void launch_sparse(const SparseArgs& a, int nqb, hipStream_t s) {
  const unsigned units = (unsigned)nqb * a.heads;
  if (units <= 256 && a.keep >= 8)
    hipLaunchKernelGGL((sparse_bf16_kernel<HD, 2>), dim3(units), dim3(512), 0, s, a);
  else
    hipLaunchKernelGGL((sparse_bf16_kernel<HD, 1>), dim3(units), dim3(256), 0, s, a);
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
    launch_sparse<64>(a, nqb, s);
  else
    launch_sparse<128>(a, nqb, s);
  return hipGetLastError();
}

}  // namespace dit
