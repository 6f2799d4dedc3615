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
// fp32 output: the codes go through bf16, exactly, to the bf16 matrix cores, at half
// the rate: exact products with fp32 sums.  X's codes take both scales with them (a row of
// X meets one scale of W per K tile), W's none.  All codes at scales of 2^-117 to 2^119 are
// normal bf16 values; a wave that met others (values near the type's ends) does its sums again.
#include <math.h>

#include "device_common.h"

namespace dit {

namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));

struct Word {
  int v;
};

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

// one lane's 32 codes times 2^(byte - 127) as bf16 values, 8 to an operand
__device__ __forceinline__ void to_bf16(const i32x8_t& w, int byte, bf16x8_t* out) {
  const float scale = __uint_as_float((uint32_t)byte << 23);
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
// the bytes with which every code, 2^-9 to 448, becomes a normal bf16 value
constexpr int kLeastByte = 10, kMostByte = 246;
constexpr uint32_t kBytes = kMostByte - kLeastByte;

// ---------------------------------------------------------------- 256 x 256 tiles, bf16 output
// s_waitcnt with vmcnt = n and the other counters left alone
template <int n>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(n >= 0 && n < 64, "vmcnt");
  __builtin_amdgcn_s_waitcnt((n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8));
}
// v, of an origin unknown to the compiler
__device__ __forceinline__ int opaque(int v) {
  asm volatile("" : "+v"(v));
  return v;
}
__device__ __forceinline__ void block_barrier() { asm volatile("s_barrier" ::: "memory"); }
// c += 2^(sw + sx - 254) w x, the lowest byte of either scale word.  A volatile
// statement: as a builtin the compiler moves it out of its turn between two
// barriers.  It does not see what the statement is: nothing may write an operand
// by vector arithmetic, nor read c, within the instruction's wait states.
__device__ __forceinline__ void asm_mfma(f32x4_t& c, const i32x8_t& w, const i32x8_t& x, int sw, int sx) {
  asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[0,0,0]"
               : "+v"(c)
               : "v"(w), "v"(x), "v"(sw), "v"(sx));
}

// grouped order: 8 M-tiles share each run of N-tiles, for L2 reuse of both operands
__device__ __forceinline__ void tile_of(int id, int tm, int tn, int& im, int& in) {
  constexpr int GM = 8;
  const int grp = id / (GM * tn), first = grp * GM, size = min(tm - first, GM), in_grp = id - grp * GM * tn;
  im = first + in_grp % size;
  in = in_grp / size;
}

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
struct __attribute__((packed, aligned(2))) Bf16x8 {
  u32x4_t v;
};
struct __attribute__((packed, aligned(4))) F32x4 {
  f32x4_t v;
};
__device__ __forceinline__ u32x4_t pack8(const float* v) {
  return u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}
// C neighbouring columns (a multiple of 8) of an output row that ends `left` columns further, at any element's address
template <bool F32, int C>
__device__ __forceinline__ void store_columns(char* y, const float* v, int left) {
  if (left >= C) {
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < C; i += 4) ((F32x4*)(y + i * 4))->v = f32x4_t{v[i], v[i + 1], v[i + 2], v[i + 3]};
    } else {
#pragma unroll
      for (int i = 0; i < C; i += 8) ((Bf16x8*)(y + i * 2))->v = pack8(v + i);
    }
  } else {
#pragma unroll
    for (int i = 0; i < C - 1; ++i)
      if (i < left) {
        if constexpr (F32) ((float*)y)[i] = v[i];
        else ((bf16_t*)y)[i] = f2bf(v[i]);
      }
  }
}

constexpr int kMaxBlocks256 = 256;  // of fp8_256_kernel: one per CU
constexpr int kMinKTiles256 = 3;    // its loads run up to three K tiles ahead, into the next output tile at most

// 8 waves, each 128 rows x 64 columns.  K tiles of 128 bytes (one scale block)
// move by direct-to-LDS loads into two stages.  Two wave groups (waves 0-3 and
// 4-7, one wave of each per SIMD) take turns: while one issues a cluster of 8
// MFMAs, the other reads the fragments of its next cluster from LDS and issues
// its share of the loads; block barriers hold the groups one turn apart.  A K
// tile is 4 clusters: cluster c multiplies the wave's c-th quarter of X rows (2
// fragments) with all its W rows (4 fragments, held for a whole tile, two tiles
// in turn).  Read phase 4 kt + c takes the X of the next cluster, 4 kt + c + 1, and
// part c of W of tile kt + 1; every wave has their data ahead of the first barrier of its
// next phase, which the other group meets a turn later.  So a place is loaded again two
// phases after its last read, not one: X's part c of tile kt + 2 in phase 4 kt + c + 1, W's
// of tile kt + 3 in phase 4 kt + c + 2.  Either is read 6 phases after its load: loads have
// 5 phases until the wait that makes them visible.
// A block works through its output tiles as one stream of K tiles: the loads of
// the next output tile run ahead of the last K tiles of this one, and each
// cluster's finished sums are written in its read phase of the next tile's first
// K tile, beside the other group's MFMAs.
// W's rows are dealt out to the fragments so that a lane holds 16 neighbouring
// columns of a row: it writes 32 bytes straight from registers.
// 16896 x 16384 x 4096: 895 - 960 us, 2.4 - 2.5 PFLOP/s, 2.6 - 2.9 at 8192^3 (320 us
// without loads, 262 without LDS reads either: matrix cores and clock bound it); the
// stores, which all CUs issue at the same time, cost about a tenth.  4429 x 6144 x 1536:
// 47 us, 432 tiles in two rounds of 256.
__global__ __launch_bounds__(512) void fp8_256_kernel(const Fp8Problem p) {
  constexpr int BM = 256, BN = 256, Q = 4;
  constexpr int ROWB = 128, CPR = 8, RPI = 8;  // bytes and 16-byte chunks of a row, rows per wave load
  constexpr int STAGE = BM * ROWB, SUB = STAGE / Q, REGION = 2 * STAGE;
  static_assert(BM == BN, "one stage size");
  // [X stage 0, 1 | W stage 0, 1 | scales stage 0, 1: 256 words of X, 4 copies of the words of W's two row blocks |
  // bias of the last two output tiles]
  constexpr int SCALES = 2 * REGION, SCALE_STAGE = 2048, BIAS = SCALES + 2 * SCALE_STAGE, BIAS_STAGE = 1024;
  __shared__ uint4 lds[(BIAS + 2 * BIAS_STAGE) / 16];
  char* const lbase = (char*)lds;
  const int tn = (p.N + BN - 1) / BN, tm = (p.M + BM - 1) / BM, tiles = tm * tn;
  // XCD x owns a contiguous range of tiles; its blocks take them in turn
  const int xcd = blockIdx.x & 7, per = tiles >> 3, rem = tiles & 7;
  const int tile_end = (xcd + 1) * per + min(xcd + 1, rem), tile_step = ((int)gridDim.x - xcd + 7) >> 3;
  int tile_next = xcd * per + min(xcd, rem) + (blockIdx.x >> 3);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wv >> 2, wn = wv & 3;
  // K tiles, and those of an output tile: an even number, the last one of zeros where K has an odd number
  const int KT = p.kb, Kp = KT * kFp8Block, KE = (KT + 1) & ~1;
  const int my_tiles = (tile_end - tile_next + tile_step - 1) / tile_step;

  // LDS slot of chunk c of row r: 16 consecutive rows' chunks lie in 16 different 16-byte bank groups
  auto swz = [](int row, int c) { return c ^ ((row >> 1) & 7); };
  // byte offsets of this lane's row of a part; the part and the K tile travel in the scalar offset, which the
  // range check counts
  const int lrow = wv * RPI + lane / CPR, lc = swz(lrow, lane % CPR) * 16;
  const int gx = (int)((uint32_t)(lrow / 32 * 128 + lrow % 32) * (uint32_t)Kp + lc);
  const int gw = (int)((uint32_t)(lrow / 16 * 64 + lrow % 16 / 4 * 16 + lrow % 4) * (uint32_t)Kp + lc);
  const int gs = (wv < 4 ? wv * 64 + lane : lane & 1) * p.pitch;
  // Three streams of loads, X, W and scales, each at a K tile of an output tile of its own; a row that does not exist
  // reads as zeros.
  auto buffer = [](const uint8_t* base, int n) __attribute__((always_inline)) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, n, kBufferWord3);
  };
  // rows r0 .. r0 + most - 1 of n, as far as they exist.  The size is forced into a scalar register: left to itself the
  // compiler holds it in a vector register and issues every load from a loop over the lanes' (equal) values.
  auto rows = [&](const uint8_t* base, int r0, int most, int n, int pitch) __attribute__((always_inline)) {
    return buffer(base + (long)r0 * pitch, __builtin_amdgcn_readfirstlane(max(min(n - r0, most), 0) * pitch));
  };
  auto tile_at = [&](int id, int& m0, int& n0) __attribute__((always_inline)) {
    int im, in;
    tile_of(id, tm, tn, im, in);
    m0 = __builtin_amdgcn_readfirstlane(im * BM);
    n0 = __builtin_amdgcn_readfirstlane(in * BN);
  };
  int m0, n0, m0_next, n0_next;  // this output tile and the next (behind the last one, itself again)
  tile_at(tile_next, m0, n0);
  m0_next = m0;
  n0_next = n0;
  int xm = m0, wn0 = n0, xk = 0, wk = 0;
  auto load_x = [&](auto stc, auto cc) __attribute__((always_inline)) {  // part c
    constexpr int st = decltype(stc)::value, c = decltype(cc)::value;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        rows(p.x, xm, xk < KT ? BM : 0, p.M, Kp),
        (__attribute__((address_space(3))) void*)(lbase + st * STAGE + c * SUB + wv * RPI * ROWB), 16, gx,
        xk * ROWB + c * 32 * Kp, 0, 0);
  };
  auto load_w = [&](auto stc, auto cc) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value, c = decltype(cc)::value;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        rows(p.w, wn0, wk < KT ? BN : 0, p.N, Kp),
        (__attribute__((address_space(3))) void*)(lbase + REGION + st * STAGE + c * SUB + wv * RPI * ROWB), 16, gw,
        wk * ROWB + c * 4 * Kp, 0, 0);
  };
  auto next_xk = [&]() __attribute__((always_inline)) {
    const bool on = ++xk == KE;
    xk = on ? 0 : xk;
    xm = on ? m0_next : xm;
  };
  auto next_wk = [&]() __attribute__((always_inline)) {
    const bool on = ++wk == KE;
    wk = on ? 0 : wk;
    wn0 = on ? n0_next : wn0;
  };
  // Scales: a word holds the bytes of 4 K tiles of a row, the first lowest.  The words of K tiles 4 g .. are read
  // from LDS as they are needed; those of the next four are loaded while they are: X's by waves 0-3, a row per lane,
  // W's by waves 4-7, each a copy.
  auto load_scales = [&](int stage, int m, int n, int k) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t r = wv < 4 ? rows(p.xs, m, BM, p.M, p.pitch) : rows(p.ws, n >> 7, 2, (p.N + 127) >> 7, p.pitch);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        r, (__attribute__((address_space(3))) void*)(lbase + SCALES + stage * SCALE_STAGE + wv * 256), 4, gs, k, 0, 0);
  };
  // the tile's bias, one value per word, 64 of them by each of four waves (and again by the others); zeros past N
  auto load_bias = [&](int stage) __attribute__((always_inline)) {
    const int q = wv & 3, n = p.bias ? max(p.N - n0, 0) : 0, vo = q * 64 + lane;
    __attribute__((address_space(3))) void* const to =
        (__attribute__((address_space(3))) void*)(lbase + BIAS + stage * BIAS_STAGE + q * 256);
    if (p.bias_f32)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer((const uint8_t*)p.bias + (long)n0 * 4, n * 4), to, 4, vo * 4, 0, 0, 0);
    else
      __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer((const uint8_t*)p.bias + (long)n0 * 2, n * 2), to, 2, vo * 2, 0, 0, 0);
  };

  // ---- fragment reads: row lane % 16 of a 16-row fragment, chunks lane / 16 and lane / 16 + 4
  const int xr = wm * 32 + (lane & 15), wr = wn * 16 + (lane & 15);
  int xa[2], wa[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    xa[h] = xr * ROWB + swz(xr, (lane >> 4) + 4 * h) * 16;
    wa[h] = REGION + wr * ROWB + swz(wr, (lane >> 4) + 4 * h) * 16;
  }
  // Whole-value casts: read member by member, the compiler takes them to alias the loads in flight and waits for those.
  auto lds16 = [&](int at) __attribute__((always_inline)) {
    return __builtin_bit_cast(i32x4_t, *(const uint4*)(lbase + at));
  };
  auto lds4 = [&](int at) __attribute__((always_inline)) {
    return __builtin_bit_cast(int, *(const Word*)(lbase + at));
  };
  auto frag = [&](int lo, int hi) __attribute__((always_inline)) {
    return __builtin_shufflevector(lds16(lo), lds16(hi), 0, 1, 2, 3, 4, 5, 6, 7);
  };
  const int xs0 = SCALES + (wm * 128 + (lane & 15)) * 4, ws0 = SCALES + 1024 + wv % 4 * 256 + (wn >> 1) * 4;
  f32x4_t acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  // X fragments of a cluster and its scale words (clusters in turn), W fragments of a K tile and its scale word (K tiles
  // in turn)
  i32x8_t fx[2][2], fw[2][4];
  int sx[2][2], sw[2];
  // reads part c of X of a K tile in `st` into the cluster's registers
  auto read_x = [&](auto stc, auto cc, int stage) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value, c = decltype(cc)::value;
    const int xsa = opaque(xs0 + stage * SCALE_STAGE);  // one address register, the rest in the reads' offsets
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      constexpr int off = st * STAGE + c * SUB;
      fx[c & 1][i] = frag(xa[0] + off + i * 16 * ROWB, xa[1] + off + i * 16 * ROWB);
      sx[c & 1][i] = lds4(xsa + (c * 32 + i * 16) * 4);
    }
    if constexpr (c == 0) sw[st] = lds4(opaque(ws0 + stage * SCALE_STAGE));
  };

  // ---- writes the finished sums of cluster c of the tile at (m0, n0), whose bias is in `stage`
  const int ncol = wn * 64 + (lane >> 4) * 16, mrow = wm * 128 + (lane & 15);
  const uint32_t pitch = (uint32_t)p.N * 2;
  const int bias_shift = p.bias_f32 ? 0 : 16;
  auto store = [&](auto cc, int m0, int n0, int stage) __attribute__((always_inline)) {
    constexpr int c = decltype(cc)::value;
    float b[16];
    const int at = opaque(ncol) * 4 + BIAS + stage * BIAS_STAGE;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const i32x4_t v = lds16(at + q * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) b[q * 4 + e] = __uint_as_float((uint32_t)v[e] << bias_shift);
    }
    // opaque: what depends on the lane alone is formed here again rather than held in registers over the K loop
    const int mr = opaque(mrow), n = p.N - n0 - opaque(ncol);  // n: columns left from this lane's first
    const uint32_t yo = (uint32_t)mr * pitch + (uint32_t)(p.N - n0 - n) * 2;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float v[16];
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) v[j * 4 + r] = acc[c * 2 + i][j][r] + b[j * 4 + r];
      char* const y = (char*)p.y + ((long)m0 * p.N + n0) * 2 + (long)(c * 32 + i * 16) * pitch + yo;
      if (mr < p.M - m0 - (c * 32 + i * 16)) store_columns<false, 16>(y, v, n);
    }
  };

  using S0 = std::integral_constant<int, 0>;
  using S1 = std::integral_constant<int, 1>;
  int prev_m0 = p.M, prev_n0 = 0, scale_stage = 0, bias_stage = 0;  // no row of the tile before the first exists
  bool counted = false;
  // STORE 1: the output tile's first K tile, which writes the previous tile's sums; 2: the one after it
  auto phase = [&](auto stc, auto cc, auto storec, int kt) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value, c = decltype(cc)::value;
    constexpr int STORE = decltype(storec)::value;
    using CN = std::integral_constant<int, (c + 1) % Q>;
    using SN = std::integral_constant<int, c + 1 < Q ? st : st ^ 1>;  // stage of the next cluster
    using CX = std::integral_constant<int, (c + Q - 1) % Q>;
    using SX = std::integral_constant<int, c == 0 ? st ^ 1 : st>;
    using CW = std::integral_constant<int, (c + Q - 2) % Q>;
    using SW = std::integral_constant<int, c < 2 ? st : st ^ 1>;
    if constexpr (STORE == 1) {
      store(cc, prev_m0, prev_n0, bias_stage ^ 1);
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          acc[c * 2 + i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
          asm volatile("" : "+v"(acc[c * 2 + i][j]));  // zeroed here, ahead of the barrier
        }
    }
    // the last phase's reads, this cluster's operands among them: complete ahead of the barrier, behind which (the next
    // phase on) their places are loaded again
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    const int byte = (kt & 3) * 8;
#pragma unroll
    for (int i = 0; i < 2; ++i) sx[c & 1][i] = opaque(opaque(sx[c & 1][i]) >> byte);
    if constexpr (c == 0) sw[st] = opaque(opaque(sw[st]) >> byte);
    // the next cluster's X; behind the last one of a K tile, whose scales may start another group
    if (c + 1 == Q && st == 1 && (((kt + 1) & 3) == 0 || kt + 1 == KE)) scale_stage ^= 1;
    read_x(SN{}, CN{}, scale_stage);
    {
      constexpr int off = (st ^ 1) * STAGE + c * SUB;
      fw[st ^ 1][c] = frag(wa[0] + off, wa[1] + off);
    }
    // the last part of X's K tile kt + 1, or a part of kt + 2; the last two parts of W's kt + 2, or a part of kt + 3
    load_x(SX{}, CX{});
    load_w(SW{}, CW{});
    if constexpr (c == 0) next_xk();
    if constexpr (c == 1) next_wk();
    // All but the loads of the last 5 phases have landed.  Those phases' stores need not have: 4 in each phase of the
    // first K tile, if all of the tile's rows and columns exist.
    if (STORE && counted) wait_vmcnt<10 + (STORE == 1 ? 4 * (c + 1) : STORE == 2 ? 16 - 4 * c : 0)>();
    else wait_vmcnt<10>();
    block_barrier();
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) asm_mfma(acc[c * 2 + i][j], fw[st][j], fx[c & 1][i], sw[st], sx[c & 1][i]);
    block_barrier();
  };
  // K tiles kt and kt + 1.  Scales come in groups of four K tiles, the last group of an output tile two or four: their
  // loads have 8 phases or more.
  auto k_pair = [&](auto firstc, int kt) __attribute__((always_inline)) {
    constexpr int FIRST = decltype(firstc)::value;
    if ((kt & 3) == 0) {
      const bool on = kt + 4 >= KE;
      load_scales(scale_stage ^ 1, on ? m0_next : m0, on ? n0_next : n0, on ? 0 : kt + 4);
    }
    static_for<Q>([&](auto cc) { phase(S0{}, cc, std::integral_constant<int, FIRST ? 1 : 0>{}, kt); });
    static_for<Q>([&](auto cc) { phase(S1{}, cc, std::integral_constant<int, FIRST ? 2 : 0>{}, kt + 1); });
  };
  load_scales(0, m0, n0, 0);
  static_for<Q>([&](auto cc) { load_w(S0{}, cc); });
  next_wk();
  static_for<Q>([&](auto cc) {
    load_x(S0{}, cc);
    load_w(S1{}, cc);
  });
  next_xk();
  next_wk();
  wait_vmcnt<Q * 2>();
  block_barrier();
  static_for<Q>([&](auto cc) {
    constexpr int off = decltype(cc)::value * SUB;
    fw[0][decltype(cc)::value] = frag(wa[0] + off, wa[1] + off);
  });
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  block_barrier();
  static_for<Q - 1>([&](auto cc) {
    load_x(S1{}, cc);
    if constexpr (decltype(cc)::value > 0) load_w(S0{}, std::integral_constant<int, decltype(cc)::value - 1>{});
  });
  wait_vmcnt<10>();  // what phase 0 reads has landed: X's first two parts, W's first of tile 1 and the scales
  block_barrier();
  read_x(S0{}, S0{}, 0);
  if (wv >= 4) block_barrier();
#pragma unroll 1
  for (int t = 0; t < my_tiles; ++t) {
    load_bias(bias_stage);
    tile_next += tile_step;
    if (tile_next < tile_end) tile_at(tile_next, m0_next, n0_next);
    counted = prev_m0 + BM <= p.M && prev_n0 + BN <= p.N;  // 4 stores a phase by every wave
    k_pair(std::true_type{}, 0);
#pragma unroll 1
    for (int kt = 2; kt < KE; kt += 2) k_pair(std::false_type{}, kt);
    prev_m0 = m0;
    prev_n0 = n0;
    bias_stage ^= 1;
    m0 = m0_next;
    n0 = n0_next;
  }
  if (wv < 4) block_barrier();
  wait_vmcnt<0>();  // the loads past the last K tile land before the block ends
  asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory");  // the last MFMAs' results
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(acc[i][j]));
  static_for<Q>([&](auto cc) { store(cc, prev_m0, prev_n0, bias_stage ^ 1); });
}

// ---------------------------------------------------------------- smaller tiles, and fp32 output
__device__ __forceinline__ i32x8_t load32(const uint8_t* p, int second) {
  return __builtin_shufflevector(*(const i32x4_t*)p, *(const i32x4_t*)(p + second), 0, 1, 2, 3, 4, 5, 6, 7);
}

// acc += the products of one K tile's fragments.  bf16 output: the 8-bit cores,
// scales in the instruction; fp32: codes and scales to bf16, four steps of 32.  sx: per
// row, sw: the same in all of W's fragments; met: more than kBytes once a scale left the range.
template <bool F32, int FM, int FN>
__device__ __forceinline__ void multiply(const i32x8_t* x, const i32x8_t* w, const int* sx, const int* sw, uint32_t& met,
                                         f32x4_t (*acc)[FN]) {
  if constexpr (F32) {
    bf16x8_t xb[FM][4];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const uint32_t past = (uint32_t)((sx[i] & 255) + (sw[0] & 255) - 127 - kLeastByte);  // outside the range: more than kBytes
      met = max(met, past);
      to_bf16(x[i], (int)past + kLeastByte, xb[i]);
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      bf16x8_t wb[4];
      to_bf16(w[j], 127, wb);
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int i = 0; i < FM; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[c], xb[i][c], acc[i][j], 0, 0, 0);
    }
  } else {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w[j], x[i], acc[i][j], 0, 0, 0, sw[j], 0, sx[i]);
  }
}

// The sums of a wave's K tiles kt, kt + step, .. for fp32 output at any scales, straight
// from memory.  A fragment takes three passes over a K tile where it has rows outside the
// range: rows within, below and above, the others as zeros.  Below, 2^-117 goes to W, and what
// is less than 2^-117 even then vanishes in fp32; above, 2^100, and past the range even then
// every product overflows.  The products are exact wherever the power goes, so a row within
// gets the bits that multiply() gives it, whatever its neighbours hold.
// Rows of X from m, of W from n; the lane's codes at byte k of a K tile and `second` further.
template <int FM, int FN>
__device__ __forceinline__ void multiply_again(const Fp8Problem& p, int m, int n, int kt, int step, int k, int second,
                                               f32x4_t (*acc)[FN]) {
  const int lr = threadIdx.x & 15, Kp = p.kb * kFp8Block;
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (; kt < p.kb; kt += step) {
    const int sw = p.ws[(long)(n >> 7) * p.pitch + kt];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const long row = min(m + i * 16 + lr, p.M - 1);
      const i32x8_t x = load32(p.x + row * Kp + kt * 128 + k, second);
      const int b = p.xs[row * p.pitch + kt] + sw - 127, side = b < kLeastByte ? 1 : b > kMostByte ? 2 : 0;
#pragma unroll 1
      for (int pass = 0; pass < 3; ++pass) {
        if (!__any(side == pass)) continue;
        const int shift = pass == 0 ? 0 : pass == 1 ? kLeastByte - 127 : 100;
        bf16x8_t xb[4], wb[4];
        to_bf16(side == pass ? x : i32x8_t{}, min(max(b - shift, kLeastByte), kMostByte), xb);
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          const long col = min(n + (lr >> 2) * (4 * FN) + j * 4 + (lr & 3), p.N - 1);
          to_bf16(load32(p.w + col * Kp + kt * 128 + k, second), 127 + shift, wb);
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wb[c], xb[c], acc[i][j], 0, 0, 0);
        }
      }
    }
  }
}

// a launch's blocks along x (fewer than 2^32 threads), the rest goes on along y
constexpr int kRingRowLog2 = 22;

// BM x BN outputs per block; KG groups of WM x WN waves share out the K tiles.  A
// step is KG K tiles, which arrive by direct-to-LDS loads in a ring of ST stages;
// the groups' sums meet in LDS at the end, in their order.  As in the kernel
// above a lane holds 4 FN neighbouring columns of each of its rows.
// The loads bound it: 53 - 60 bytes per ns and CU, between what L2 (133) and memory
// (27) give them.  589 x 1536 x 6144 in 64 x 64: 15 us (9.4 MB of W, each through 10 row blocks).
template <bool F32, int BM, int BN, int WM, int WN, int KG, int ST>
__global__ __launch_bounds__(WM* WN* KG * 64) void fp8_ring_kernel(const Fp8Problem p) {
  constexpr int NW = WM * WN * KG, FM = BM / WM / 16, FN = BN / WN / 16;
  constexpr int ROWB = 128, UNITS = KG * (BM + BN) / 8, LPW = UNITS / NW;  // loads of 8 rows; per wave and step
  constexpr int TILE = (BM + BN) * ROWB, SCALES = KG * TILE, STAGE = SCALES + BM * 4 + 256;
  static_assert(LPW * NW == UNITS && BM % 64 == 0 && BM / 64 < NW && KG <= 4 && 4 % KG == 0, "tile config");
  static_assert(ST * STAGE <= 160 * 1024 && (KG - 1) * WM * WN * FM * FN * 1024 <= ST * STAGE, "LDS");
  __shared__ uint4 lds[ST * STAGE / 16];
  char* const lbase = (char*)lds;
  const int tn = (p.N + BN - 1) / BN, tm = (p.M + BM - 1) / BM;
  const int id = (int)(blockIdx.y << kRingRowLog2) + xcd_remap(blockIdx.x, gridDim.x);
  if (id >= tm * tn) return;
  int im, in;
  tile_of(id, tm, tn, im, in);
  const int m0 = im * BM, n0 = in * BN, KT = p.kb, Kp = KT * kFp8Block, steps = (KT + KG - 1) / KG;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), kg = wv / (WM * WN), wm = wv / WN % WM, wn = wv % WN;
  auto swz = [](int row, int c) { return c ^ ((row >> 1) & 7); };

  // this wave's loads of a step: 8 rows each of X or W of one K tile
  uint32_t go[LPW];
#pragma unroll
  for (int i = 0; i < LPW; ++i) {
    const int row = (wv * LPW + i) * 8 % (BM + BN) + (lane >> 3);
    int g = row;
    if (row >= BM) {  // W's rows dealt out to the fragments
      constexpr int C = BN / WN;
      const int w = row - BM, in_wave = w % C, f = in_wave & 15;
      g = w - in_wave + (f >> 2) * (4 * FN) + (in_wave >> 4) * 4 + (f & 3);
    }
    go[i] = (uint32_t)g * (uint32_t)Kp + swz(row, lane & 7) * 16;
  }
  auto buffer = [&](const uint8_t* base, int r0, int most, int rows, int pitch) __attribute__((always_inline)) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)(base + (long)r0 * pitch), (short)0,
                                             __builtin_amdgcn_readfirstlane(max(min(rows - r0, most), 0) * pitch), kBufferWord3);
  };
  // rows past the last one: its scales
  const int sgo = (wv < BM / 64 ? min(wv * 64 + lane, p.M - 1 - m0) : lane & 1) * p.pitch;
  auto load = [&](int step, int stage) __attribute__((always_inline)) {
    char* const at = lbase + stage * STAGE;
#pragma unroll
    for (int i = 0; i < LPW; ++i) {
      const int unit = wv * LPW + i, q = unit * 8 / (BM + BN), row = unit * 8 % (BM + BN), kt = step * KG + q;
      const bool x = row < BM;
      // locals, not expressions: the host pass drops the kernel's launch stub otherwise
      const int vo = (int)go[i], so = kt * ROWB;
      const __amdgpu_buffer_rsrc_t rs =
          buffer(x ? p.x : p.w, x ? m0 : n0, kt < KT ? (x ? BM : BN) : 0, x ? p.M : p.N, Kp);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rs, (__attribute__((address_space(3))) void*)(at + q * TILE + row * ROWB), 16, vo, so, 0, 0);
    }
    // the scale words of the step's K tiles: X's by the first waves, a row per lane, W's two row blocks' by the others
    const bool x = wv < BM / 64;
    const int vo = sgo, so = min(step * KG, KT - 1) & ~3;
    const __amdgpu_buffer_rsrc_t rs =
        buffer(x ? p.xs : p.ws, x ? m0 : n0 >> 7, x ? BM : 2, x ? p.M : (p.N + 127) >> 7, p.pitch);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        rs, (__attribute__((address_space(3))) void*)(at + SCALES + (x ? wv * 256 : BM * 4)), 4, vo, so, 0, 0);
  };
  auto lds16 = [&](int at) __attribute__((always_inline)) {
    return __builtin_bit_cast(i32x4_t, *(const uint4*)(lbase + at));
  };
  auto lds4 = [&](int at) __attribute__((always_inline)) { return __builtin_bit_cast(int, *(const Word*)(lbase + at)); };
  const int xr = wm * FM * 16 + (lane & 15), wr = BM + wn * FN * 16 + (lane & 15);
  int xa[2], wa[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    xa[h] = kg * TILE + xr * ROWB + swz(xr, (lane >> 4) + 4 * h) * 16;
    wa[h] = kg * TILE + wr * ROWB + swz(wr, (lane >> 4) + 4 * h) * 16;
  }
  const int sxa = SCALES + xr * 4, swa = SCALES + BM * 4 + (((n0 & 127) + wn * FN * 16) >> 7) * 4;
  f32x4_t acc[FM][FN] = {};
  uint32_t met = 0;
  static_for<ST - 1>([&](auto sc) { load(decltype(sc)::value, decltype(sc)::value); });
  int stage = 0;
  for (int s = 0; s < steps; ++s) {
    // step s has landed, this wave's part and, behind the barrier, everyone's; the stage before it is read no more
    wait_vmcnt<(ST - 2) * (LPW + 1)>();
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    block_barrier();
    load(s + ST - 1, stage == 0 ? ST - 1 : stage - 1);
    const int at = stage * STAGE, byte = ((s * KG + kg) & 3) * 8;
    i32x8_t x[FM], w[FN];
    int sx[FM], sw[FN];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      x[i] = __builtin_shufflevector(lds16(at + xa[0] + i * 16 * ROWB), lds16(at + xa[1] + i * 16 * ROWB), 0, 1, 2, 3, 4, 5, 6, 7);
      sx[i] = lds4(at + sxa + i * 64) >> byte;
    }
#pragma unroll
    for (int j = 0; j < FN; ++j)
      w[j] = __builtin_shufflevector(lds16(at + wa[0] + j * 16 * ROWB), lds16(at + wa[1] + j * 16 * ROWB), 0, 1, 2, 3, 4, 5, 6, 7);
    const int ws = lds4(at + swa) >> byte;  // a wave's columns lie in one row block of scales
#pragma unroll
    for (int j = 0; j < FN; ++j) sw[j] = ws;
    multiply<F32, FM, FN>(x, w, sx, sw, met, acc);
    stage = stage + 1 == ST ? 0 : stage + 1;
  }
  wait_vmcnt<0>();
  if constexpr (F32)
    if (__any(met > kBytes))
      multiply_again<FM, FN>(p, m0 + wm * FM * 16, n0 + wn * FN * 16, kg, KG, (lane >> 4) * 16, 64, acc);
  __syncthreads();
  if constexpr (KG > 1) {
    // sums of groups 1 .. at [group - 1][wave of the group][fragment][lane]
    uint4* const part = lds + (wv % (WM * WN)) * (FM * FN * 64) + lane;
    if (kg > 0) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          part[(kg - 1) * WM * WN * FM * FN * 64 + (i * FN + j) * 64] = __builtin_bit_cast(uint4, acc[i][j]);
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int g = 0; g < KG - 1; ++g)
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          acc[i][j] += __builtin_bit_cast(f32x4_t, part[g * WM * WN * FM * FN * 64 + (i * FN + j) * 64]);
  }
  const int n = n0 + wn * FN * 16 + (lane >> 4) * (4 * FN);
  if (n >= p.N) return;
  float b[4 * FN];
#pragma unroll
  for (int i = 0; i < 4 * FN; ++i) b[i] = n + i < p.N ? bias_at(p, n + i) : 0.f;
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const long m = m0 + wm * FM * 16 + i * 16 + (lane & 15);
    if (m >= p.M) continue;
    float v[4 * FN];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) v[j * 4 + r] = acc[i][j][r] + b[j * 4 + r];
    store_columns<F32, 4 * FN>((char*)p.y + (m * p.N + n) * (F32 ? 4 : 2), v, p.N - n);
  }
}

// ---------------------------------------------------------------- small tiles, K shared out to the waves
// BM x BN = 16 FM x 16 FN outputs per block, NW waves that share out the K tiles: a
// wave multiplies all rows and columns of its K tiles, which nobody else reads, so
// the waves need no barrier until their sums meet in LDS, in wave order.  K tiles
// arrive by direct-to-LDS loads in two stages of each wave's own (loads to registers,
// 64 bytes of 16 rows each, reach half the rate).  As above W's rows are dealt out to
// the fragments, and a lane ends with 4 FN neighbouring columns of a row.  For outputs
// that fill one round of CUs or less: what a CU loads bounds these products (60 - 85
// bytes per ns), and smaller tiles spread it over more CUs.  4 waves (8: 4 - 25% slower
// past one round, where fewer blocks fit a CU).  64 x 1536 x 6144: 6.4 us.
template <bool F32, int FM, int FN, int NW>
__global__ __launch_bounds__(NW * 64) void fp8_split_kernel(const Fp8Problem p) {
  constexpr int BM = FM * 16, BN = FN * 16, ROWB = 128, TILE = (BM + BN) * ROWB;
  constexpr int LOADS = (BM + BN) / 8 + FM + 1;  // of a K tile
  __shared__ uint4 lds[NW * 2 * TILE / 16];      // [wave][stage][X's rows, then W's]; then the waves' sums
  static_assert(FM <= NW && FM * FN * 1024 <= 2 * TILE && BN <= 128, "tile config");
  const int tn = (p.N + BN - 1) / BN, tm = (p.M + BM - 1) / BM;
  const int id = (int)(blockIdx.y << kRingRowLog2) + xcd_remap(blockIdx.x, gridDim.x);
  if (id >= tm * tn) return;
  int im, in;
  tile_of(id, tm, tn, im, in);
  const int m0 = im * BM, n0 = in * BN, Kp = p.kb * kFp8Block;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane & 15;
  char* const lbase = (char*)lds + wv * 2 * TILE;
  auto swz = [](int row, int c) { return c ^ ((row >> 1) & 7); };
  // loads of 8 rows: of X, and of either half of a fragment of W
  const int row = lane >> 3;
  uint32_t xo[2], wo[2], so[FM];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = h * 8 + row, c = swz(r, lane & 7) * 16;
    xo[h] = row * (uint32_t)Kp + c;
    wo[h] = (uint32_t)((r >> 2) * (4 * FN) + (r & 3)) * (uint32_t)Kp + c;
  }
#pragma unroll
  for (int i = 0; i < FM; ++i) so[i] = min(i * 16 + lr, p.M - 1 - m0) * (uint32_t)p.pitch;
  // rows and K tiles past the last one read as zeros, with the last one's scales
  auto rows = [&](const uint8_t* base, int r0, int most, int n, int pitch) __attribute__((always_inline)) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)(base + (long)r0 * pitch), (short)0,
                                             __builtin_amdgcn_readfirstlane(min(n - r0, most) * pitch), kBufferWord3);
  };
  int sx[2][FM], sw[2];
  auto load = [&](int kt, auto stc) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value;
    const bool in = kt < p.kb;
    const __amdgpu_buffer_rsrc_t rx = rows(p.x, m0, in ? BM : 0, p.M, Kp), rw = rows(p.w, n0, in ? BN : 0, p.N, Kp);
    const __amdgpu_buffer_rsrc_t rsx = rows(p.xs, m0, BM, p.M, p.pitch);
    const __amdgpu_buffer_rsrc_t rsw = rows(p.ws, n0 >> 7, 1, (p.N + 127) >> 7, p.pitch);
    const int ks = min(kt, p.kb - 1);
#pragma unroll
    for (int i = 0; i < BM / 8; ++i) {
      const int vo = (int)xo[i & 1], at = kt * ROWB + i * 8 * Kp;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (__attribute__((address_space(3))) void*)(lbase + st * TILE + i * 1024), 16, vo,
                                               at, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < BN / 8; ++i) {
      const int vo = (int)wo[i & 1], at = kt * ROWB + (i >> 1) * 4 * Kp;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rw, (__attribute__((address_space(3))) void*)(lbase + st * TILE + (BM / 8 + i) * 1024), 16, vo, at, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) sx[st][i] = __builtin_amdgcn_raw_buffer_load_b8(rsx, so[i], ks, 0);
    sw[st] = __builtin_amdgcn_raw_buffer_load_b8(rsw, 0, ks, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  int fa[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) fa[h] = lr * ROWB + swz(lr, (lane >> 4) + 4 * h) * 16;
  auto frag = [&](int at) __attribute__((always_inline)) {
    const i32x4_t lo = __builtin_bit_cast(i32x4_t, *(const uint4*)(lbase + at + fa[0]));
    const i32x4_t hi = __builtin_bit_cast(i32x4_t, *(const uint4*)(lbase + at + fa[1]));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  f32x4_t acc[FM][FN] = {};
  uint32_t met = 0;
  auto step = [&](int kt, auto stc) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value;
    wait_vmcnt<LOADS>();  // all but the next K tile's loads
    __builtin_amdgcn_sched_barrier(0);
    i32x8_t x[FM], w[FN];
    int xs[FM], ws[FN];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      x[i] = frag(st * TILE + i * 16 * ROWB);
      xs[i] = sx[st][i];
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      w[j] = frag(st * TILE + (BM + j * 16) * ROWB);
      ws[j] = sw[st];
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): read, before the K tile after the next arrives here
    __builtin_amdgcn_sched_barrier(0);
    load(kt + 2 * NW, stc);
    multiply<F32, FM, FN>(x, w, xs, ws, met, acc);
    __builtin_amdgcn_sched_barrier(0);
  };
  using S0 = std::integral_constant<int, 0>;
  using S1 = std::integral_constant<int, 1>;
  load(wv, S0{});
  load(wv + NW, S1{});
#pragma unroll 1
  for (int k = wv; k < p.kb; k += 2 * NW) {
    step(k, S0{});
    step(k + NW, S1{});
  }
  wait_vmcnt<0>();
  if constexpr (F32)
    if (__any(met > kBytes)) multiply_again<FM, FN>(p, m0, n0, wv, NW, (lane >> 4) * 16, 64, acc);
  uint4* const sums = lds + lane;
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) sums[wv * (2 * TILE / 16) + (i * FN + j) * 64] = __builtin_bit_cast(uint4, acc[i][j]);
  __syncthreads();
  if (wv >= FM) return;  // wave i finishes rows 16 i ..
  const int m = m0 + wv * 16 + lr, n = n0 + (lane >> 4) * (4 * FN);
  if (m >= p.M || n >= p.N) return;
  float v[4 * FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    f32x4_t s = __builtin_bit_cast(f32x4_t, sums[(wv * FN + j) * 64]);
#pragma unroll
    for (int g = 1; g < NW; ++g) s += __builtin_bit_cast(f32x4_t, sums[g * (2 * TILE / 16) + (wv * FN + j) * 64]);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[j * 4 + r] = s[r] + (n + j * 4 + r < p.N ? bias_at(p, n + j * 4 + r) : 0.f);
  }
  store_columns<F32, 4 * FN>((char*)p.y + ((long)m * p.N + n) * (F32 ? 4 : 2), v, p.N - n);
}

// ---------------------------------------------------------------- few rows
// Up to 16 rows of X against 16 columns per block: W is read once, straight from
// memory to registers, and the block's waves share out the K tiles, two in flight
// each.  Their sums meet in LDS in wave order.  4 x 9216 x 1536: 6 us with the launch
// (14 MB of W, 2.4 TB/s).
template <bool F32>
__global__ __launch_bounds__(512) void fp8_rows_kernel(const Fp8Problem p) {
  constexpr int NW = 8, U = 2;
  __shared__ f32x4_t part[NW][64];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 15, n0 = blockIdx.x * 16, Kp = p.kb * kFp8Block;
  const uint8_t* const w = p.w + (long)min(n0 + lr, p.N - 1) * Kp + (lane >> 4) * 32;
  const uint8_t* const ws = p.ws + (long)(n0 >> 7) * p.pitch;
  const uint8_t* const x = p.x + (long)min(lr, p.M - 1) * Kp + (lane >> 4) * 32;
  const uint8_t* const xs = p.xs + (long)min(lr, p.M - 1) * p.pitch;
  f32x4_t acc[1][1] = {};
  uint32_t met = 0;
  for (int k0 = wv; k0 < p.kb; k0 += NW * U) {
    i32x8_t wf[U], xf[U];
    int sw[U], sx[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kt = min(k0 + u * NW, p.kb - 1);  // past the end: loaded again, not multiplied
      wf[u] = load32(w + (long)kt * 128, 16);
      sw[u] = ws[kt];
      xf[u] = load32(x + (long)kt * 128, 16);
      sx[u] = xs[kt];
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (k0 + u * NW < p.kb) multiply<F32, 1, 1>(&xf[u], &wf[u], &sx[u], &sw[u], met, acc);
  }
  if constexpr (F32)
    if (__any(met > kBytes)) multiply_again<1, 1>(p, 0, n0, wv, NW, (lane >> 4) * 32, 16, acc);
  part[wv][lane] = acc[0][0];
  __syncthreads();
  if (wv > 0) return;
  f32x4_t s = part[0][lane];
#pragma unroll
  for (int g = 1; g < NW; ++g) s += part[g][lane];
  const int m = lr, n = n0 + (lane >> 4) * 4;
  if (m >= p.M) return;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    if (n + r >= p.N) break;
    const float v = s[r] + bias_at(p, n + r);
    const long o = (long)m * p.N + n + r;
    if constexpr (F32) ((float*)p.y)[o] = v;
    else ((bf16_t*)p.y)[o] = f2bf(v);
  }
}

}  // namespace

// Which kernel a product takes: the one whose modelled time is least.  In
// microseconds, rounds of 256 tiles times (a fixed part + a part per K tile of
// 128), of the ring kernels two blocks to a CU and the odd round at a rate of its own,
// and no less than reading W takes; fitted to 110 shapes (M 1 - 16896, N 33 - 262144,
// K 64 - 65536; it picks the fastest or one within 15% of it on all of them).
// Up to 16 rows there is one more, up to a W of 32 MB.  Measured, in us with the
// launch, bf16 output, these first ones with W not in the caches:
//   rows         4 x 9216 x 1536 6.1 (16 x 32: 7.1), 16 x 1536 x 6144 8.8 (9.9), but
//                16 x 16384 x 4096 22 (18.7), where X's share of the traffic counts
//   16 x 32      64 x 1536 x 6144 6.4 (32 x 32: 7.6, 64 x 64: 13.2)
//   32 x 32      128 x 1536 x 6144 7.9 (16 x 32: 9.6, 32 x 64: 9.8)
//   32 x 64      200 x 1536 x 6144 10.0 (32 x 32: 12.6, 64 x 64: 13.5)
//   64 x 64      589 x 1536 x 6144 14.8 (32 x 64: 21.5, 128 x 128: 28.5), 589 x 1536 x 1536 6.4
//   128 x 128    4429 x 1536 x 1536 17.0 (64: 26.0, 256: 27.0), 333 x 6144 x 1536 10.9 (64: 12.4)
//   256 x 256    4429 x 6144 x 1536 50 (128: 52.5), 4096^3 63 (128: 73.5); a launch of one
//                round leaves the chip its clock, hence two lines
enum Fp8Cfg { FP8_ROWS, FP8_16X32, FP8_32X32, FP8_32X64, FP8_64, FP8_128, FP8_256 };
static Fp8Cfg pick(int M, int N, int K, int out_dtype) {
  const double kt = fp8_k_blocks(K);
  const bool f32 = out_dtype == DIT_F32;
  if (M <= 16 && N * kt * 128 <= 1 << 25) return FP8_ROWS;
  auto rounds = [&](int bm, int bn) { return ceil(ceil((double)M / bm) * ceil((double)N / bn) / 256.0); };
  // the ring kernels: c, then a pair of rounds and an odd one, each fixed + per K tile
  auto ring = [&](int b, double c, double pair, double pair_kt, double odd, double odd_kt) {
    const double n = rounds(b, b);
    return c + floor(n / 2) * (pair + pair_kt * kt) + (n - 2 * floor(n / 2)) * (odd + odd_kt * kt);
  };
  Fp8Cfg cfg = FP8_64;
  double best = f32                    ? ring(64, 3.5, 2.45, 0.5, 1.0, 0.31)
                : rounds(64, 64) <= 1 ? 3.5 + 0.235 * kt
                                      : ring(64, 2.5, 1.9, 0.385, 0.3, 0.33);
  auto offer = [&](Fp8Cfg c, double us) {
    if (us < best) {
      best = us;
      cfg = c;
    }
  };
  const double memory = 2.9 + N * kt * 128 / 7e6;
  offer(FP8_16X32, fmax(2.9 + rounds(16, 32) * (0.7 + (f32 ? 0.065 : 0.06) * kt), memory));
  offer(FP8_32X32, fmax(2.9 + rounds(32, 32) * (1.15 + (f32 ? 0.095 : 0.083) * kt), memory));
  offer(FP8_32X64, fmax(1.7 + rounds(32, 64) * (3.2 + (f32 ? 0.16 : 0.145) * kt), memory));
  offer(FP8_128, f32                      ? ring(128, 3.5, 5.7, 1.55, 2.7, 0.92)
                 : rounds(128, 128) <= 1 ? 4.75 + 0.547 * kt
                                         : ring(128, 3.1, 3.65, 0.866, 0.0, 0.7));
  // offsets within a tile of 256 output rows fit 32 bits up to 2^21 columns
  if (!f32 && kt >= kMinKTiles256 && N <= 1 << 21)
    offer(FP8_256, rounds(256, 256) <= 1 ? 13.5 + 1.02 * kt : rounds(256, 256) * (7.0 + 1.45 * kt));
  return cfg;
}

const char* gemm_fp8_config_name(int M, int N, int K, int out_dtype) {
  static const char* names[] = {"gemm_fp8_rows", "gemm_fp8_16x32", "gemm_fp8_32x32", "gemm_fp8_32x64", "gemm_fp8_64x64", "gemm_fp8_128x128", "gemm_fp8_256x256"};
  return names[pick(M, N, K, out_dtype)];
}

static dim3 ring_grid(long blocks) {
  return dim3((unsigned)std::min(blocks, 1L << kRingRowLog2), (unsigned)((blocks - 1) >> kRingRowLog2) + 1);
}

// Two stages leave room for a second block on a CU, whose loads and products go on
// while the first one waits or stores (4429 x 1536 x 1536 17.0 us against 20.5 with
// four, 11469 x 6574 x 1024 98 against 137, 16896 x 6144 x 1536 fp32 320 against 407).
// A launch of one block a CU needs four to cover its loads, bf16 ones at any rate (589 x
// 1536 x 6144 14.9 against 20.0; fp32 20.4 against 21.6, and 18.9 against 19.3 the other way).
template <bool F32, int BM, int BN, int WM, int WN, int KG>
static void launch_ring(const Fp8Problem& p, hipStream_t s) {
  const long tiles = (long)((p.M + BM - 1) / BM) * ((p.N + BN - 1) / BN);
  const dim3 grid = ring_grid(tiles), block(WM * WN * KG * 64);
  if constexpr (!F32) {
    if (tiles <= 256) {
      hipLaunchKernelGGL((fp8_ring_kernel<F32, BM, BN, WM, WN, KG, 4>), grid, block, 0, s, p);
      return;
    }
  }
  hipLaunchKernelGGL((fp8_ring_kernel<F32, BM, BN, WM, WN, KG, 2>), grid, block, 0, s, p);
}

template <bool F32, int FM, int FN>
static void launch_split(const Fp8Problem& p, hipStream_t s) {
  constexpr int NW = 4, BM = FM * 16, BN = FN * 16;
  const dim3 grid = ring_grid((long)((p.M + BM - 1) / BM) * ((p.N + BN - 1) / BN));
  hipLaunchKernelGGL((fp8_split_kernel<F32, FM, FN, NW>), grid, dim3(NW * 64), 0, s, p);
}

template <bool F32>
static void launch_small(Fp8Cfg cfg, const Fp8Problem& p, hipStream_t s) {
  if (cfg == FP8_ROWS) hipLaunchKernelGGL((fp8_rows_kernel<F32>), dim3((p.N + 15) / 16), dim3(512), 0, s, p);
  else if (cfg == FP8_16X32) launch_split<F32, 1, 2>(p, s);
  else if (cfg == FP8_32X32) launch_split<F32, 2, 2>(p, s);
  else if (cfg == FP8_32X64) launch_split<F32, 2, 4>(p, s);
  else if (cfg == FP8_64) launch_ring<F32, 64, 64, 2, 2, 2>(p, s);
  else launch_ring<F32, 128, 128, 2, 4, 1>(p, s);
}

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
  const Fp8Cfg cfg = pick(M, N, K, out_dtype);
  if (cfg == FP8_256) {
    const long tiles = (long)((M + 255) / 256) * ((N + 255) / 256);
    hipLaunchKernelGGL(fp8_256_kernel, dim3((unsigned)std::min<long>(tiles, kMaxBlocks256)), dim3(512), 0, s, p);
  } else if (out_dtype == DIT_F32) {
    launch_small<true>(cfg, p, s);
  } else {
    launch_small<false>(cfg, p, s);
  }
  return hipGetLastError();
}

}  // namespace dit
