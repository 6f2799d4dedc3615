// Attention of packed sequences with grouped heads, causal or not,
// O = softmax(scale Q K^T) V, one pass over the keys with a running max and sum.
//
// The query heads of a group read the same keys, so they are rows of the same
// tiles: row i G + g of a sequence and key head is query i at the group's head g.
// A tile of keys is then loaded once for all of them, a tile of rows spans fewer
// positions (less of it is masked), and a single token fills as many rows as its
// group has heads.
//
// Row i G + g sees the first n_i keys: kv_len - q_len + i + 1 of them, none below
// zero, or all.  Keys past that get the score -inf.  Their values, which a product
// with a probability of 0 would let through where they are infinite or NaN, are
// looked at in the tiles that need a mask: such a tile is summed with zeros in their
// place, and they are added key by key to the rows that see them.
#include <float.h>
#include <math.h>

#include "device_common.h"

namespace dit {

namespace {

typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));

constexpr int kKeys = 64;  // of a tile

// A row's running max is raised only when a tile's probabilities against it sum to more than 2^8 in one of its two
// lanes: up to there fp32 and bf16 hold them as well as any.  Each row decides for itself.
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

// v, of an origin unknown to the compiler
__device__ __forceinline__ int opaque(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// the halves of a word of two bf16 values that are finite, zeros for the others
__device__ __forceinline__ uint32_t finite_halves(uint32_t w) {
  const uint32_t lo = (w & 0x7f80) == 0x7f80 ? 0 : w & 0xffff, hi = (w & 0x7f800000) == 0x7f800000 ? 0 : w & 0xffff0000;
  return lo | hi;
}
__device__ __forceinline__ bool is_finite(float v) { return (__float_as_uint(v) & 0x7f800000) != 0x7f800000; }

// the sequence of tile t: the last one that starts at or before it
__device__ __forceinline__ int sequence_of(const GroupedArgs& a, int t) {
  int n = 0;
#pragma unroll
  for (int b = 0; b < DIT_MAX_SEQUENCES; b += 64) {
    const int i = b + (threadIdx.x & 63);
    n += __popcll(__ballot(i < a.n_seq && a.tile_off[i] <= t));
  }
  return __builtin_amdgcn_readfirstlane(n - 1);
}

// keys that query i of sequence s sees
__device__ __forceinline__ int seen_by(const GroupedArgs& a, int s, int i) {
  return a.causal ? max(a.kv_len[s] - a.q_len[s] + i + 1, 0) : a.kv_len[s];
}

struct Unit {
  int s, h, row0, rows;     // sequence, key head, first row of the tile, rows of the sequence
  int begin, end, ranges;   // its range of the keys, and how many ranges the tile has
};
// key ranges that a sequence's tiles may have; a tile that sees fewer keys has fewer
__host__ __device__ __forceinline__ int ranges_of(const GroupedArgs& a, int s) {
  return a.kv_len[s] > a.chunk ? (a.kv_len[s] + a.chunk - 1) / a.chunk : 1;
}
// Unit `id` of tiles of `per` rows: key heads in turn, then the ranges of a tile; a sequence's last tile, which sees most,
// first.  The ranges of a tile are equal but for whole key tiles.  begin > end: a range that the tile does not have.
__device__ __forceinline__ Unit unit_of(const GroupedArgs& a, int id, int per) {
  Unit u;
  const int t = id / a.kv_heads;
  u.h = id - t * a.kv_heads;
  u.s = sequence_of(a, t);
  u.rows = a.q_len[u.s] * a.group;
  const int most = ranges_of(a, u.s), n = a.tile_off[u.s + 1] - 1 - t, tile = n / most, range = most - 1 - (n - tile * most);
  u.row0 = tile * per;
  const int seen = seen_by(a, u.s, (min(u.row0 + per, u.rows) - 1) / a.group);
  u.ranges = seen > a.chunk ? (seen + a.chunk - 1) / a.chunk : 1;
  const int len = ((seen + u.ranges - 1) / u.ranges + kKeys - 1) / kKeys * kKeys;
  u.begin = range * len;
  u.end = range < u.ranges ? min(u.begin + len, seen) : -1;
  return u;
}
// where a unit's partial results lie: O [rows of a tile][HD], unnormalised; behind all of them (max, sum) [rows of a tile]
__device__ __forceinline__ float* part_o(const GroupedArgs& a, int id, int per) { return a.part + (long)id * per * a.head_dim; }
__device__ __forceinline__ float2* part_ml(const GroupedArgs& a, int id, int per) {
  const long units = (long)a.tile_off[a.n_seq] * a.kv_heads;
  return (float2*)(a.part + units * per * a.head_dim) + (long)id * per;
}

// ---------------------------------------------------------------- bf16
// 4 waves x 32 rows.  S^T = K Q^T by v_mfma_f32_32x32x16_bf16: a lane holds the scores
// of row lane % 32 for half of the keys, and its probabilities are the B operand of
// O^T = V^T P^T.  K and V tiles arrive as they lie in memory, by direct-to-LDS loads
// into two stages; V is transposed on its way from LDS to the matrix cores.
// 16384 tokens of 32 heads of 128, causal, 1.9 ms, 1.15 PFLOP/s; without the softmax
// 1.64, without P V 1.23: matrix and vector instructions both, at the clock that the
// power leaves.  Twelve prompts of 1 to 4096 tokens, 24 heads of 64, 88 us, 0.8
// PFLOP/s: here the matrix cores are busy 34% of the time and the vector units, six
// issues a score, 49%.  A tile's scores, exponentials and products with V wait for each
// other, a barrier ends it, and 2.1 waves a SIMD, the launch's end counted in, are all
// there is to fill in.  Slower were two groups of waves that take turns at the two
// (2.12 ms: a wave alone on a SIMD issues vector instructions at half the rate of two),
// and a max that is looked at ahead of the exponentials (1.93 ms).
template <int HD>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(HD == 64 ? 3 : 2)))
void grouped_bf16_kernel(const GroupedArgs a) {
  constexpr int ROWS = 128;
  constexpr int CH = HD / 8;             // 16-byte chunks of a row
  constexpr int RPI = 64 / CH;           // rows per wave load
  constexpr int NI = kKeys / RPI / 4;    // loads of a tile per wave
  constexpr int ROWB = HD * 2, TILE = kKeys * ROWB, STAGE = 2 * TILE;
  __shared__ uint4 smem[2 * STAGE / 16];  // [stage][K tile | V tile]
  char* const lbase = (char*)smem;
  const int id = block_id();
  if (id >= a.tile_off[a.n_seq] * a.kv_heads) return;
  const Unit u = unit_of(a, id, ROWS);
  const int tid = threadIdx.x, lane = tid & 63, hl = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int L = a.kv_len[u.s], G = a.group;
  const int ld = (int)a.ldkv;
  const bf16_t* const K = (const bf16_t*)a.k + a.kv_row[u.s] * a.ldkv + (long)u.h * HD;
  const bf16_t* const V = (const bf16_t*)a.v + a.kv_row[u.s] * a.ldkv + (long)u.h * HD;
  const int last = u.rows - 1;
  if (u.end < 0) return;
  // key tiles from the range's first on: all, and those that every row sees
  const int first = u.begin / kKeys;
  const int tiles = (u.end + kKeys - 1) / kKeys;
  const int whole = min(seen_by(a, u.s, u.row0 / G), u.end) / kKeys;
  const int wave_seen = seen_by(a, u.s, min(u.row0 + wave * 32 + 31, last) / G);     // keys that some row of this wave sees

  // slot of chunk c of K row `key`: the 16 rows of a fragment read lie in 16 different 16-byte bank groups
  auto kswz = [](int key, int c) { return HD == 128 ? c ^ (key & 15) : c ^ ((key >> 1) & 7); };
  // of V row `key`: the 64-byte segments of 4 neighbouring rows lie in 4 different quarters of the banks
  auto vswz = [](int key, int c) { return HD == 128 ? c ^ ((key & 3) << 2) : c ^ ((key & 2) << 1); };
  int ko[NI], vo[NI];  // global byte offsets of this lane's loads inside a tile
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int key = (wave * NI + i) * RPI + lane / CH;
    ko[i] = (key * ld + kswz(key, lane % CH) * 8) * 2;
    vo[i] = (key * ld + vswz(key, lane % CH) * 8) * 2;
  }
  auto tile_load = [&](int j, int st) __attribute__((always_inline)) {
    const int k0 = j * kKeys;
    const int bytes = ((min(L - k0, kKeys) - 1) * ld + HD) * 2;  // keys past L read as zeros
    const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc((void*)(K + (long)k0 * ld), (short)0, bytes, kBufferWord3);
    const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc((void*)(V + (long)k0 * ld), (short)0, bytes, kBufferWord3);
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
  if (first < tiles) tile_load(first, 0);
  const int row = u.row0 + wave * 32 + (lane & 31), query = min(row, last) / G, head = u.h * G + min(row, last) - query * G;
  const int seen = seen_by(a, u.s, query);
  bf16x8_t qf[HD / 16];
  {
    const bf16_t* const Q = (const bf16_t*)a.q + (long)(a.q_off[u.s] + query) * a.ldq + (long)head * HD;
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) qf[s] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(Q + (s * 2 + hl) * 8));
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
  auto step = [&](int j, int st, auto maskc) __attribute__((always_inline)) {
    constexpr bool MASK = decltype(maskc)::value;
    if (j + 1 < tiles) tile_load(j + 1, st ^ 1);
    if (!MASK || j * kKeys < wave_seen) {
      f32x16_t s[2] = {};
#pragma unroll
      for (int ks = 0; ks < HD / 16; ++ks)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          const bf16x8_t f = __builtin_bit_cast(bf16x8_t, *(const uint4*)(lbase + kf[ks] + st * STAGE + kb * 32 * ROWB));
          s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, qf[ks], s[kb], 0, 0, 0);
        }
      read_ahead<2 * HD / 16, 1, 4>();
      if constexpr (MASK) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (j * kKeys + kb * 32 + (i >> 2) * 8 + hl * 4 + (i & 3) >= seen) s[kb][i] = -INFINITY;
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
        // a row's two lanes decide alike; the other rows keep their max, and with it their bits
        const bool raise = (int)high | __shfl_xor((int)high, 32, 64);  // every lane takes part in the exchange
        float tm = s[0][0];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) tm = fmaxf(tm, s[kb][i]);
        tm = fmaxf(tm, __shfl_xor(tm, 32, 64));
        tm = fmaxf(mx, tm * sl2);
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
      auto v_frag = [&](int g, int db) __attribute__((always_inline)) {
        bf16x4_t v[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
          v[e] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
              (__attribute__((address_space(3))) bf16x4_t*)(lbase + vf[db] + st * STAGE + (g * 16 + e * 8) * ROWB));
        return __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
      };
      bool plain = true;
      if constexpr (MASK) {
        // 0 times every value of the tile: NaN where one is not finite
        float z = 0.f;
        const bf16x2_t zero = {(__bf16)0.0f, (__bf16)0.0f};
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int db = 0; db < HD / 32; ++db) {
            const bf16x8_t f = v_frag(g, db);
#pragma unroll
            for (int e = 0; e < 8; e += 2) z = __builtin_amdgcn_fdot2_f32_bf16(bf16x2_t{f[e], f[e + 1]}, zero, z, false);
          }
        __builtin_amdgcn_sched_barrier(0);
        plain = !__any(z != z);
      }
      if (plain) {
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int db = 0; db < HD / 32; ++db)
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(g, db), pf[g], o[db], 0, 0, 0);
        read_ahead<4 * HD / 32, 2, 2>();
      } else {
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int db = 0; db < HD / 32; ++db) {
            uint4 w = __builtin_bit_cast(uint4, v_frag(g, db));
            w = make_uint4(finite_halves(w.x), finite_halves(w.y), finite_halves(w.z), finite_halves(w.w));
            o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, w), pf[g], o[db], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
          }
#pragma unroll 1
        for (int key = 0; key < kKeys; ++key) {
          // the row's probability of this key: register (key % 32 / 8) * 4 + key % 4 of block key / 32, lane half key / 4 % 2
          const int ln = opaque(lane);  // what depends on the lane alone is formed here, not held in registers over the tiles
          const int at = (key >> 5) * 16 + (key >> 3 & 3) * 4 + (key & 3);
          uint32_t w = 0;
          static_for<16>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            const uint4 q = __builtin_bit_cast(uint4, pf[i >> 2]);
            if (at >> 1 == i) w = (i & 3) == 0 ? q.x : (i & 3) == 1 ? q.y : (i & 3) == 2 ? q.z : q.w;
          });
          const float pr = __shfl(__uint_as_float(at & 1 ? w & 0xffff0000 : w << 16), (ln & 31) | (key >> 2 & 1) << 5, 64);
          const bool in = j * kKeys + key < seen;
#pragma unroll
          for (int db = 0; db < HD / 32; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int dim = db * 32 + q * 8 + (ln >> 5) * 4;
              const uint2 v = *(const uint2*)(lbase + st * STAGE + TILE + key * ROWB + vswz(key, dim / 8) * 16 + dim % 8 * 2);
              const float f[4] = {__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000), __uint_as_float(v.y << 16),
                                  __uint_as_float(v.y & 0xffff0000)};
#pragma unroll
              for (int r = 0; r < 4; ++r)
                o[db][q * 4 + r] = fmaf(pr, in && !is_finite(f[r]) ? f[r] : 0.f, o[db][q * 4 + r]);
              __builtin_amdgcn_sched_barrier(0);
            }
        }
      }
    }
    // this wave's loads have landed and its reads returned; behind the barrier everyone's have
    wait_vmcnt0_lgkmcnt0();
    asm volatile("s_barrier" ::: "memory");
  };
  wait_vmcnt0_lgkmcnt0();
  asm volatile("s_barrier" ::: "memory");
  using NoMask = std::false_type;
  using Mask = std::true_type;
  int j = first;
  for (; j + 1 < whole; j += 2) {
    step(j, 0, NoMask{});
    step(j + 1, 1, NoMask{});
  }
  if (j < whole) {
    step(j, 0, NoMask{});
    ++j;
  }
#pragma unroll 1
  for (; j < tiles; ++j) step(j, (j - first) & 1, Mask{});
  l += __shfl_xor(l, 32, 64);
  if (u.ranges > 1) {
    const int slot = wave * 32 + (lane & 31);
    float* const po = part_o(a, id, ROWS) + (long)slot * HD;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(float4*)(po + d * 32 + g * 8 + hl * 4) = make_float4(o[d][g * 4], o[d][g * 4 + 1], o[d][g * 4 + 2], o[d][g * 4 + 3]);
    if (hl == 0) part_ml(a, id, ROWS)[slot] = make_float2(mx, l);
  } else if (row <= last) {
    const float inv = seen > 0 ? 1.0f / l : 0.f;
    bf16_t* const og = (bf16_t*)a.o + (long)(a.q_off[u.s] + query) * a.ldo + (long)head * HD;
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
// On the fp32 matrix cores (v_mfma_f32_16x16x4_f32).  A block owns 16 rows; of every
// key tile each of its four waves takes 16 keys, with its own running max, sum and O,
// merged at the end in wave order.  K and V go straight from memory to registers, in
// 16-byte pieces: a lane's piece of V holds 4 neighbouring dimensions of a key, each a
// row of another MFMA.  The next tile's K replaces this one's once the scores are done,
// its V once O is.  Sixteen sequences of 1 to 16384 keys, 258 MB, 64 us, 4.1 TB/s.  The
// twelve prompts, 24 heads, 860 us, 82 TFLOP/s of the 157 that the matrix cores have:
// these are busy 53% of the time, the vector units 47%: the products, softmax and
// rescaled sums of 16 keys depend on each other, and 2.8 waves share a SIMD.
constexpr int FD = 64, FQ = 16;

__global__ __launch_bounds__(256) void grouped_f32_kernel(const GroupedArgs a) {
  __shared__ float osh[4][FQ][FD + 4];
  __shared__ float2 ml[4][FQ];
  const int id = block_id();
  if (id >= a.tile_off[a.n_seq] * a.kv_heads) return;
  const Unit u = unit_of(a, id, FQ);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, kq = lane >> 4;
  const int L = a.kv_len[u.s], G = a.group, last = u.rows - 1;
  const float* const K = (const float*)a.k + a.kv_row[u.s] * a.ldkv + (long)u.h * FD;
  const float* const V = (const float*)a.v + a.kv_row[u.s] * a.ldkv + (long)u.h * FD;
  if (u.end < 0) return;
  const int first = u.begin / kKeys;
  const int tiles = (u.end + kKeys - 1) / kKeys;
  const int least = seen_by(a, u.s, u.row0 / G);  // keys that every row sees
  const int row = min(u.row0 + lr, last), query = row / G;
  const int seen = seen_by(a, u.s, query);
  const float* const Q = (const float*)a.q + (long)(a.q_off[u.s] + query) * a.ldq + (long)(u.h * G + row - query * G) * FD;
  float4 q[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) q[c] = *(const float4*)(Q + c * 16 + kq * 4);
  const float sl2 = a.scale * 1.4426950408889634f;
  float4 kf[4], vf[4];  // K: dims 16 c + 4 kq .. of key lr; V: dims 4 lr .. of key 4 kq + e (zeros past L)
  auto load_k = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < 4; ++c) kf[c] = *(const float4*)(K + min(k0 + lr, L - 1) * a.ldkv + c * 16 + kq * 4);
  };
  auto load_v = [&](int k0) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int key = k0 + kq * 4 + e;
      vf[e] = *(const float4*)(V + min(key, L - 1) * a.ldkv + lr * 4);
      if (key >= L) vf[e] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
  };
  auto at = [](const float4& v, auto ec) __attribute__((always_inline)) {
    constexpr int e = decltype(ec)::value;
    return e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w;
  };
  float mx = -FLT_MAX, l = 0.f;
  f32x4_t o[4];  // element r of o[c]: dim 16 kq + 4 r + c of row lr
#pragma unroll
  for (int c = 0; c < 4; ++c) o[c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (first < tiles) {
    load_k(first * kKeys + wave * 16);
    load_v(first * kKeys + wave * 16);
  }
  for (int t = first; t < tiles; ++t) {
    const int k0 = t * kKeys + wave * 16, next = t + 1 < tiles ? k0 + kKeys : -1;
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
      s[i] = k0 + kq * 4 + i < seen ? (s0[i] + s1[i]) * sl2 : -INFINITY;
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
    bool plain = true;
    if (k0 + 16 > least) {  // a mask in this wave's keys
      float z = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) z += 0.f * vf[e].x + 0.f * vf[e].y + 0.f * vf[e].z + 0.f * vf[e].w;
      plain = !__any(z != z);
    }
    if (!plain) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        vf[e] = make_float4(is_finite(vf[e].x) ? vf[e].x : 0.f, is_finite(vf[e].y) ? vf[e].y : 0.f,
                            is_finite(vf[e].z) ? vf[e].z : 0.f, is_finite(vf[e].w) ? vf[e].w : 0.f);
    }
    static_for<4>([&](auto ec) {
      constexpr int e = decltype(ec)::value;
      static_for<4>([&](auto cc) {
        constexpr int c = decltype(cc)::value;
        o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(at(vf[e], cc), s[e], o[c], 0, 0, 0);
      });
    });
    if (!plain) {
#pragma unroll 1
      for (int key = 0; key < 16; ++key) {
        const int e = key & 3;
        const float pr = __shfl(e == 0 ? s[0] : e == 1 ? s[1] : e == 2 ? s[2] : s[3], lr + (key >> 2) * 16, 64);
        if (k0 + key < seen) {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float4 v = *(const float4*)(V + (k0 + key) * a.ldkv + kq * 16 + r * 4);
            if (!is_finite(v.x)) o[0][r] = fmaf(pr, v.x, o[0][r]);
            if (!is_finite(v.y)) o[1][r] = fmaf(pr, v.y, o[1][r]);
            if (!is_finite(v.z)) o[2][r] = fmaf(pr, v.z, o[2][r]);
            if (!is_finite(v.w)) o[3][r] = fmaf(pr, v.w, o[3][r]);
          }
        }
      }
    }
    if (next >= 0) load_v(next);
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (kq == 0) ml[wave][lr] = make_float2(mx, l);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    *(float4*)&osh[wave][lr][kq * 16 + i * 4] = make_float4(o[0][i], o[1][i], o[2][i], o[3][i]);
  __syncthreads();
  // 16 lanes per row, 4 dims each.  A wave whose keys are all masked has the lowest max, and weighs nothing.
  const int rl = tid >> 4, dd = (tid & 15) * 4, to = u.row0 + rl;
  if (to > last) return;  // (its partial results are not read either)
  float mm = ml[0][rl].x;
#pragma unroll
  for (int w = 1; w < 4; ++w) mm = fmaxf(mm, ml[w][rl].x);
  float ls = 0.f;
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float wt = exp2f(ml[w][rl].x - mm);
    const float4 v = *(const float4*)&osh[w][rl][dd];
    ls = fmaf(wt, ml[w][rl].y, ls);
    y = make_float4(fmaf(wt, v.x, y.x), fmaf(wt, v.y, y.y), fmaf(wt, v.z, y.z), fmaf(wt, v.w, y.w));
  }
  if (u.ranges > 1) {
    *(float4*)(part_o(a, id, FQ) + rl * FD + dd) = y;
    if (dd == 0) part_ml(a, id, FQ)[rl] = make_float2(mm, ls);
    return;
  }
  const int oq = to / G;
  const float inv = seen_by(a, u.s, oq) > 0 ? 1.0f / ls : 0.f;
  *(float4*)((float*)a.o + (long)(a.q_off[u.s] + oq) * a.ldo + (long)(u.h * G + to - oq * G) * FD + dd) =
      make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
}

// ---------------------------------------------------------------- bf16, few rows
// Sequences of at most 32 rows: one token, or a few, over a cache.  A block takes a
// range of the keys; its four waves take tiles of 32 keys in turn, each for all rows,
// with LDS, a running max, a sum and an O of its own: no barrier until they meet at the
// end.  A tile's K goes to registers whole, and the next tile's K into its place while
// the softmax runs; its V likewise, the next one's arriving beside the next scores.  So
// one place each is enough, two blocks share a CU, and what a CU has in flight is what
// its LDS holds.  The reads of K and V bound it, each once: sixteen sequences of 1 to
// 16384 keys, 8 key heads of 128, 258 MB, 54 us with the joining of the ranges, 4.8 TB/s
// (334 us by the kernel of many rows, whole sequences; 84 in ranges of 512 keys).
constexpr int kFewRows = 32, kFewKeys = 32, kFewWaves = 4;
constexpr int kStreamed = 2;  // a load's cache policy: not to be kept (58 us; kept 62)

__device__ __forceinline__ void wait_lgkmcnt0() { __builtin_amdgcn_s_waitcnt(0xc07f); }
template <int n>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(n >= 0 && n < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8));
}

template <int HD>
__global__ __launch_bounds__(kFewWaves * 64) __attribute__((amdgpu_waves_per_eu(2)))
void grouped_few_kernel(const GroupedArgs a) {
  constexpr int NW = kFewWaves;
  constexpr int CH = HD / 8, RPI = 64 / CH, NI = kFewKeys / RPI;  // chunks of a row, rows and number of loads of a tile
  constexpr int ROWB = HD * 2, TILE = kFewKeys * ROWB;
  constexpr int NR = HD / 2, MERGE = NW * (NR + 2) * 64 * 4;  // registers of O, bytes of all waves' results
  // [wave][K tile | V tile], then [wave][register][lane] of the results
  __shared__ uint4 smem[(MERGE > NW * 2 * TILE ? MERGE : NW * 2 * TILE) / 16];
  const int id = block_id();
  if (id >= a.tile_off[a.n_seq] * a.kv_heads) return;
  const Unit u = unit_of(a, id, kFewRows);
  if (u.end < 0) return;
  const int tid = threadIdx.x, lane = tid & 63, hl = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  char* const lbase = (char*)smem + wave * 2 * TILE;
  const int G = a.group, ld = (int)a.ldkv, last = u.rows - 1, end = u.end;
  const bf16_t* const K = (const bf16_t*)a.k + a.kv_row[u.s] * a.ldkv + (long)u.h * HD;
  const bf16_t* const V = (const bf16_t*)a.v + a.kv_row[u.s] * a.ldkv + (long)u.h * HD;
  const int least = min(seen_by(a, u.s, 0), end);  // keys that every row sees

  auto kswz = [](int key, int c) { return HD == 128 ? c ^ (key & 15) : c ^ ((key >> 1) & 7); };
  auto vswz = [](int key, int c) { return HD == 128 ? c ^ ((key & 3) << 2) : c ^ ((key & 2) << 1); };
  // keys k0 .. of a tile; keys past the range read as zeros, a tile past it touches no memory
  auto load = [&](const bf16_t* base, int k0, bool value) __attribute__((always_inline)) {
    const int n = min(end - k0, kFewKeys), bytes = __builtin_amdgcn_readfirstlane(n > 0 ? ((n - 1) * ld + HD) * 2 : 0);
    const __amdgpu_buffer_rsrc_t r =
        __builtin_amdgcn_make_buffer_rsrc((void*)(base + (long)(n > 0 ? k0 : 0) * ld), (short)0, bytes, kBufferWord3);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int key = i * RPI + lane / CH, c = value ? vswz(key, lane % CH) : kswz(key, lane % CH);
      const int o = (key * ld + c * 8) * 2;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          r, (__attribute__((address_space(3))) void*)(lbase + (value ? TILE : 0) + i * 1024), 16, o, 0, 0, kStreamed);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  const int row = lane & 31, query = min(row, last) / G, head = u.h * G + min(row, last) - query * G;
  const int seen = min(seen_by(a, u.s, query), end);
  bf16x8_t qf[HD / 16];
  {
    const bf16_t* const Q = (const bf16_t*)a.q + (long)(a.q_off[u.s] + query) * a.ldq + (long)head * HD;
#pragma unroll
    for (int s = 0; s < HD / 16; ++s) qf[s] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(Q + (s * 2 + hl) * 8));
  }
  __builtin_amdgcn_sched_barrier(0);
  const int k0 = u.begin + wave * kFewKeys;
  load(K, k0, false);
  load(V, k0, true);
  f32x16_t o[HD / 32] = {};
  float mx = -FLT_MAX, l = 0.f;
  const float sl2 = a.scale * 1.4426950408889634f;
  int kf[HD / 16], vf[HD / 32];
#pragma unroll
  for (int ks = 0; ks < HD / 16; ++ks) kf[ks] = (lane & 31) * ROWB + kswz(lane & 31, ks * 2 + hl) * 16;
#pragma unroll
  for (int db = 0; db < HD / 32; ++db) {
    const int key = hl * 4 + (lane & 15) / 4;
    vf[db] = TILE + key * ROWB + vswz(key, db * 4 + (lane >> 4 & 1) * 2 + (lane & 3) / 2) * 16 + (lane & 1) * 8;
  }
#pragma unroll 1
  for (int k = k0; k < end; k += NW * kFewKeys) {
    wait_vmcnt<NI>();  // this tile's K; its V may be on its way
    __builtin_amdgcn_sched_barrier(0);
    bf16x8_t kr[HD / 16];
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks) kr[ks] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(lbase + kf[ks]));
    wait_lgkmcnt0();  // read, before the next tile's K arrives here
    __builtin_amdgcn_sched_barrier(0);
    load(K, k + NW * kFewKeys, false);
    // two sums, whose products need not wait for each other
    f32x16_t s = {}, s1 = {};
#pragma unroll
    for (int ks = 0; ks < HD / 16; ks += 2) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kr[ks], qf[ks], s, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kr[ks + 1], qf[ks + 1], s1, 0, 0, 0);
    }
    s += s1;
    const bool mask = k + kFewKeys > least;
    if (mask) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (k + (i >> 2) * 8 + hl * 4 + (i & 3) >= seen) s[i] = -INFINITY;
    }
    bf16x8_t pf[2];
    auto probabilities = [&]() __attribute__((always_inline)) {
      float t0 = 0.f, t1 = 0.f;
      const bf16x2_t one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = g * 8 + 2 * e;
          const float p0 = __builtin_amdgcn_exp2f(fmaf(s[i], sl2, -mx));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(s[i + 1], sl2, -mx));
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
      const bool raise = (int)high | __shfl_xor((int)high, 32, 64);
      float tm = s[0];
#pragma unroll
      for (int i = 0; i < 16; ++i) tm = fmaxf(tm, s[i]);
      tm = fmaxf(tm, __shfl_xor(tm, 32, 64));
      tm = fmaxf(mx, tm * sl2);
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
    wait_vmcnt<NI>();  // this tile's V; the next one's K may be on its way
    __builtin_amdgcn_sched_barrier(0);
    bf16x8_t vr[2][HD / 32];
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int db = 0; db < HD / 32; ++db) {
        bf16x4_t v[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
          v[e] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
              (__attribute__((address_space(3))) bf16x4_t*)(lbase + vf[db] + (g * 16 + e * 8) * ROWB));
        vr[g][db] = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
      }
    if (mask) {
      float z = 0.f;
      const bf16x2_t zero = {(__bf16)0.0f, (__bf16)0.0f};
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int db = 0; db < HD / 32; ++db)
#pragma unroll
          for (int e = 0; e < 8; e += 2)
            z = __builtin_amdgcn_fdot2_f32_bf16(bf16x2_t{vr[g][db][e], vr[g][db][e + 1]}, zero, z, false);
      if (__any(z != z)) {
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int db = 0; db < HD / 32; ++db) {
            const uint4 w = __builtin_bit_cast(uint4, vr[g][db]);
            vr[g][db] = __builtin_bit_cast(
                bf16x8_t, make_uint4(finite_halves(w.x), finite_halves(w.y), finite_halves(w.z), finite_halves(w.w)));
          }
#pragma unroll 1
        for (int key = 0; key < kFewKeys; ++key) {
          // the row's probability of this key: register (key / 8) * 4 + key % 4 of lane half key / 4 % 2
          const int ln = opaque(lane), at = (key >> 3) * 4 + (key & 3);
          uint32_t w = 0;
          static_for<8>([&](auto ic) {
            constexpr int i = decltype(ic)::value;
            const uint4 q = __builtin_bit_cast(uint4, pf[i >> 2]);
            if (at >> 1 == i) w = (i & 3) == 0 ? q.x : (i & 3) == 1 ? q.y : (i & 3) == 2 ? q.z : q.w;
          });
          const float pr = __shfl(__uint_as_float(at & 1 ? w & 0xffff0000 : w << 16), (ln & 31) | (key >> 2 & 1) << 5, 64);
          const bool in = k + key < seen;
#pragma unroll
          for (int db = 0; db < HD / 32; ++db)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int dim = db * 32 + q * 8 + (ln >> 5) * 4;
              const uint2 v = *(const uint2*)(lbase + TILE + key * ROWB + vswz(key, dim / 8) * 16 + dim % 8 * 2);
              const float f[4] = {__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000), __uint_as_float(v.y << 16),
                                  __uint_as_float(v.y & 0xffff0000)};
#pragma unroll
              for (int r = 0; r < 4; ++r)
                o[db][q * 4 + r] = fmaf(pr, in && !is_finite(f[r]) ? f[r] : 0.f, o[db][q * 4 + r]);
            }
        }
      }
    }
    wait_lgkmcnt0();  // read, before the next tile's V arrives here
    __builtin_amdgcn_sched_barrier(0);
    load(V, k + NW * kFewKeys, true);
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int db = 0; db < HD / 32; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vr[g][db], pf[g], o[db], 0, 0, 0);
  }
  wait_vmcnt<0>();
  l += __shfl_xor(l, 32, 64);
  // All waves' results over the tiles, which are read no more; wave w joins dimensions 32 w .. in wave order.  A wave
  // without a key has the lowest max, sum 0 and O 0.
  __syncthreads();
  float* const sh = (float*)smem + lane;
  {
    float* const to = sh + wave * (NR + 2) * 64;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) to[(d * 16 + i) * 64] = o[d][i];
    to[NR * 64] = mx;
    to[(NR + 1) * 64] = l;
  }
  __syncthreads();
  if (wave >= HD / 32 || row > last) return;
  float mm = sh[NR * 64], sum = 0.f;
#pragma unroll
  for (int w = 1; w < NW; ++w) mm = fmaxf(mm, sh[(w * (NR + 2) + NR) * 64]);
  float y[16] = {};
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const float* const from = sh + w * (NR + 2) * 64;
    const float al = __builtin_amdgcn_exp2f(from[NR * 64] - mm);
    sum = fmaf(al, from[(NR + 1) * 64], sum);
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = fmaf(al, from[(wave * 16 + i) * 64], y[i]);
  }
  if (u.ranges > 1) {
    float* const po = part_o(a, id, kFewRows) + (long)row * HD + wave * 32 + hl * 4;
#pragma unroll
    for (int g = 0; g < 4; ++g) *(float4*)(po + g * 8) = make_float4(y[g * 4], y[g * 4 + 1], y[g * 4 + 2], y[g * 4 + 3]);
    if (wave == 0 && hl == 0) part_ml(a, id, kFewRows)[row] = make_float2(mm, sum);
    return;
  }
  const float inv = seen > 0 ? 1.0f / sum : 0.f;
  bf16_t* const og = (bf16_t*)a.o + (long)(a.q_off[u.s] + query) * a.ldo + (long)head * HD + wave * 32 + hl * 4;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    uint2 w;
    w.x = pack_bf16x2(y[g * 4 + 0] * inv, y[g * 4 + 1] * inv);
    w.y = pack_bf16x2(y[g * 4 + 2] * inv, y[g * 4 + 3] * inv);
    *(uint2*)(og + g * 8) = w;
  }
}

// ---------------------------------------------------------------- ranges of keys joined
// A row's ranges in their order; `t` of the HD / 4 threads that take 4 dimensions each.  FEW: tiles of kFewRows rows, one to
// a sequence, whose ranges may be many: a block takes one row, and its 8 groups of threads every 8th range each, which meet
// in LDS.  `rows` blocks to a sequence, as many as the longest has rows: kFewRows cost 3 of 57 us where each has four.
// Otherwise the block of a tile's first range takes the tile, 8 rows at a time.
struct Joined {
  float m, l;
  float4 y;
};
__device__ __forceinline__ Joined join_ranges(const float2* ml, const float* po, long ml_step, long o_step, int from, int to, int by) {
  Joined j = {-FLT_MAX, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll 4
  for (int i = from; i < to; i += by) j.m = fmaxf(j.m, ml[i * ml_step].x);
#pragma unroll 4
  for (int i = from; i < to; i += by) {
    const float2 x = ml[i * ml_step];
    const float4 v = *(const float4*)(po + i * o_step);
    const float al = exp2f(x.x - j.m);
    j.l = fmaf(al, x.y, j.l);
    j.y = make_float4(fmaf(al, v.x, j.y.x), fmaf(al, v.y, j.y.y), fmaf(al, v.z, j.y.z), fmaf(al, v.w, j.y.w));
  }
  return j;
}

template <typename T, int HD, bool FEW>
__global__ __launch_bounds__(HD * 2) void grouped_merge_kernel(const GroupedArgs a, int per, int rows) {
  constexpr int TPR = HD / 4, GROUPS = 8;
  __shared__ float4 part_y[FEW ? GROUPS : 1][TPR];
  __shared__ float2 part_m[FEW ? GROUPS : 1];
  int id = block_id();
  const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
  if constexpr (FEW) {
    const int s = id / (a.kv_heads * rows), h = id / rows % a.kv_heads;
    if (s >= a.n_seq) return;
    const int row = id % rows;
    id = a.tile_off[s] * a.kv_heads + h;
    const Unit u = unit_of(a, id, per);
    if (u.ranges == 1 || row >= u.rows) return;
    const long ml_step = (long)a.kv_heads * per, o_step = ml_step * HD;  // a tile's ranges are kv_heads units apart
    const Joined j = join_ranges(part_ml(a, id, per) + row, part_o(a, id, per) + (long)row * HD + t * 4, ml_step, o_step, g,
                                 u.ranges, GROUPS);
    part_y[g][t] = j.y;
    if (t == 0) part_m[g] = make_float2(j.m, j.l);
    __syncthreads();
    if (g > 0) return;
    float m = part_m[0].x, l = 0.f;
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) m = fmaxf(m, part_m[i].x);
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {  // a group without a range has the lowest max, and zeros
      const float al = exp2f(part_m[i].x - m);
      const float4 v = part_y[i][t];
      l = fmaf(al, part_m[i].y, l);
      y = make_float4(fmaf(al, v.x, y.x), fmaf(al, v.y, y.y), fmaf(al, v.z, y.z), fmaf(al, v.w, y.w));
    }
    const int query = row / a.group;
    const float inv = seen_by(a, u.s, query) > 0 ? 1.0f / l : 0.f;
    T* const o = (T*)a.o + (long)(a.q_off[u.s] + query) * a.ldo + (long)(u.h * a.group + row - query * a.group) * HD + t * 4;
    *(uint2*)o = make_uint2(pack_bf16x2(y.x * inv, y.y * inv), pack_bf16x2(y.z * inv, y.w * inv));
  } else {
    if (id >= a.tile_off[a.n_seq] * a.kv_heads) return;
    const Unit u = unit_of(a, id, per);
    if (u.ranges == 1 || u.begin > 0) return;
    const long ml_step = (long)a.kv_heads * per, o_step = ml_step * HD;
    for (int r = g; r < per && u.row0 + r < u.rows; r += GROUPS) {
      const Joined j = join_ranges(part_ml(a, id, per) + r, part_o(a, id, per) + (long)r * HD + t * 4, ml_step, o_step, 0,
                                   u.ranges, 1);
      const int row = u.row0 + r, query = row / a.group;
      const float inv = seen_by(a, u.s, query) > 0 ? 1.0f / j.l : 0.f;
      T* const o = (T*)a.o + (long)(a.q_off[u.s] + query) * a.ldo + (long)(u.h * a.group + row - query * a.group) * HD + t * 4;
      if constexpr (sizeof(T) == 2)
        *(uint2*)o = make_uint2(pack_bf16x2(j.y.x * inv, j.y.y * inv), pack_bf16x2(j.y.z * inv, j.y.w * inv));
      else
        *(float4*)o = make_float4(j.y.x * inv, j.y.y * inv, j.y.z * inv, j.y.w * inv);
    }
  }
}

// One launch: the sequences that one kernel takes, and its tiles and ranges.
struct Plan {
  GroupedArgs a;
  int per;         // rows of a tile
  long units;
  size_t bytes;    // of partial results
};
enum Kind { ROWS, FEW, F32 };

// The sequences of `in` that `kind` takes, cut into ranges where the launch is then modelled to end sooner.
constexpr size_t kMostBytes = 128 << 20;  // of partial results: a launch that would need more is not cut
Plan plan_of(const GroupedArgs& in, Kind kind, bool may_cut = true) {
  Plan p;
  p.a = in;
  GroupedArgs& a = p.a;
  p.per = kind == F32 ? FQ : kind == FEW ? kFewRows : 128;
  // Sequences of few rows have a kernel of their own, unless they are short and the other one is launched anyway: three
  // prompts of 1024 tokens with eight tokens over 500 keys each 26 us in one launch, 34 in two, over 2048 34 and 40, over
  // 4096 44 and 45 (the tokens alone 334 and 54 for sixteen of up to 16384).
  bool many = false;
  for (int i = 0; i < in.n_seq; ++i) many = many || (long)in.q_len[i] * in.group > kFewRows;
  a.n_seq = 0;
  for (int i = 0; i < in.n_seq; ++i) {
    const bool few = (long)in.q_len[i] * in.group <= kFewRows && !(many && in.kv_len[i] <= 2048);
    if (in.q_len[i] == 0 || (kind == FEW && !few) || (kind == ROWS && few)) continue;
    a.q_off[a.n_seq] = in.q_off[i];
    a.q_len[a.n_seq] = in.q_len[i];
    a.kv_len[a.n_seq] = in.kv_len[i];
    a.kv_row[a.n_seq] = in.kv_row[i];
    ++a.n_seq;
  }
  // Ranges as long as what one of 512 blocks (two to a CU) takes if all take the same, of 256 with many rows, and not below
  // `least`, as joining them takes another launch.  Whole, and in ranges: few rows, four sequences of 512 keys 8.8 us and
  // 12.1, of 1024 15.8 and 13.2; many rows, 300 queries over 2048 keys 39 and 47, 64 over 4096 67 and 43 (in ranges of 2048
  // keys 60, of 512 46).  One token over 4096 keys 13.5 in ranges of 256, 14.4 of 64.
  constexpr int kWhole = 1 << 30;
  double keys = 0;
  int longest = 0;
  for (int i = 0; i < a.n_seq; ++i) {
    keys += (double)(((long)a.q_len[i] * a.group + p.per - 1) / p.per) * a.kv_heads * a.kv_len[i];
    longest = std::max(longest, a.kv_len[i]);
  }
  const int least = kind == ROWS ? 1024 : 256, whole = kind == ROWS ? 2048 : 768;
  double even = fmax(keys / 512 * (kind == ROWS ? 2 : 1), least);
  // Many rows: no more than 256 blocks in the end (300 queries over 4096 keys 62 us, one range more to a tile 72), and no more
  // than 8 ranges of a tile, which one block joins (64 over 16384 69 us, 16 ranges 76, 4 ranges 87).  That is of 8 key heads;
  // fewer leave CUs idle: 33 rows and more of one tile and one key head are 8 blocks, a token of 40 heads to one key head over
  // 65536 keys 135 us, of 32, which the kernel for few rows takes, 20.
  if (kind == ROWS) even = fmax(longest / fmin(fmax(floor(longest / even), 1.0), 8.0), least);
  a.chunk = !may_cut || longest <= whole || even >= longest ? kWhole : ((int)even + kKeys - 1) / kKeys * kKeys;
  a.tile_off[0] = 0;
  bool cut = false;
  for (int i = 0; i < a.n_seq; ++i) {
    a.tile_off[i + 1] = a.tile_off[i] + (int)(((long)a.q_len[i] * a.group + p.per - 1) / p.per * ranges_of(a, i));
    cut = cut || ranges_of(a, i) > 1;
  }
  p.units = (long)a.tile_off[a.n_seq] * a.kv_heads;
  p.bytes = cut ? (size_t)p.units * p.per * (a.head_dim + 2) * 4 : 0;
  if (p.bytes > kMostBytes) return plan_of(in, kind, false);
  return p;
}

template <typename T, bool FEW_ROWS>
void launch_merge(const Plan& p, hipStream_t s) {
  if (p.bytes == 0) return;
  int rows = 0;  // of the sequence with most
  for (int i = 0; i < p.a.n_seq; ++i) rows = std::max(rows, p.a.q_len[i] * p.a.group);
  const dim3 grid = grid_of(FEW_ROWS ? (long)p.a.n_seq * p.a.kv_heads * rows : p.units);
  if (p.a.head_dim == 64) hipLaunchKernelGGL((grouped_merge_kernel<T, 64, FEW_ROWS>), grid, dim3(128), 0, s, p.a, p.per, rows);
  else hipLaunchKernelGGL((grouped_merge_kernel<T, 128, FEW_ROWS>), grid, dim3(256), 0, s, p.a, p.per, rows);
}

}  // namespace

size_t attention_grouped_bytes(int dtype, const GroupedArgs& a) {
  return dtype == DIT_F32 ? plan_of(a, F32).bytes : std::max(plan_of(a, FEW).bytes, plan_of(a, ROWS).bytes);
}

hipError_t launch_attention_grouped(int dtype, const GroupedArgs& a, hipStream_t s) {
  if (dtype == DIT_F32) {
    const Plan p = plan_of(a, F32);
    if (p.units == 0) return hipSuccess;
    hipLaunchKernelGGL(grouped_f32_kernel, grid_of(p.units), dim3(256), 0, s, p.a);
    launch_merge<float, false>(p, s);
    return hipGetLastError();
  }
  // one kernel after the other on the stream, and so on one workspace
  const Plan few = plan_of(a, FEW), rows = plan_of(a, ROWS);
  if (few.units > 0) {
    const dim3 grid = grid_of(few.units);
    if (a.head_dim == 64) hipLaunchKernelGGL((grouped_few_kernel<64>), grid, dim3(kFewWaves * 64), 0, s, few.a);
    else hipLaunchKernelGGL((grouped_few_kernel<128>), grid, dim3(kFewWaves * 64), 0, s, few.a);
    launch_merge<bf16_t, true>(few, s);
  }
  if (rows.units > 0) {
    const dim3 grid = grid_of(rows.units);
    if (a.head_dim == 64) hipLaunchKernelGGL((grouped_bf16_kernel<64>), grid, dim3(256), 0, s, rows.a);
    else hipLaunchKernelGGL((grouped_bf16_kernel<128>), grid, dim3(256), 0, s, rows.a);
    launch_merge<bf16_t, false>(rows, s);
  }
  return hipGetLastError();
}

}  // namespace dit
