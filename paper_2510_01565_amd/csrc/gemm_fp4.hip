// Products of microscaled e2m1 matrices, Y = X W^T + b, both with a power-of-two
// scale per 1 x 32:
//
//   y[m, n] = sum_b 2^(sx[m, b] + sw[n, b] - 254) sum_{k in b} x[m, k] w[n, k]  +  bias[n]
//
// on the 4-bit matrix cores, which apply the scales in the instruction.  Of
// v_mfma_scale_f32_16x16x128_f8f6f4 lane l holds row l % 16 and the block l / 16 of
// 128 elements, 16 bytes, of the 32x32x64 form row l % 32 and block l / 32 of 64, and
// gives that block's scale as a byte of a word.  A row's 16 scale bytes of 512
// elements are kept as four words, word j byte i for block 4 i + j: lane l of the
// smaller form takes word l / 16 for all four steps of 128, of the larger one words
// l / 32 and l / 32 + 2 for all eight of 64, the byte being a constant of the code.
// The products of a block are exact, as is their sum, which meets the other blocks'
// in fp32; both outputs take the same sums.
#include <math.h>

#include "device_common.h"

namespace dit {

namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));

struct Word {
  int v;
};

struct Fp4Problem {
  const uint8_t* x;   // [M][pitch]
  const uint8_t* xs;  // [M][spitch]
  const uint8_t* w;   // [N][pitch]
  const uint8_t* ws;  // [N][spitch]
  const void* bias;
  int bias_f32;
  void* y;
  int M, N, kt, pitch, spitch;  // kt: K tiles of 256 elements, 128 bytes
};

__device__ __forceinline__ float bias_at(const Fp4Problem& p, int n) {
  if (!p.bias) return 0.f;
  return p.bias_f32 ? ((const float*)p.bias)[n] : bf2f(((const bf16_t*)p.bias)[n]);
}

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
// c += w x (first: c = w x) of 64 elements, the scales in byte B of their words.  Volatile statements, which keep their
// places among the reads and loads between them.  The compiler does not see what they are: nothing may read c within the
// instruction's wait states.
#define FP4_MFMA(OUT, C, SEL)                                                                                         \
  asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, " C ", %3, %4 " SEL " cbsz:4 blgp:4"                      \
               : OUT(c)                                                                                               \
               : "v"(w), "v"(x), "v"(sw), "v"(sx))
#define FP4_MFMA_BYTES(OUT, C)                                                        \
  if constexpr (B == 0) FP4_MFMA(OUT, C, "op_sel:[0,0,0] op_sel_hi:[0,0,0]");          \
  else if constexpr (B == 1) FP4_MFMA(OUT, C, "op_sel:[1,1,0] op_sel_hi:[0,0,0]");     \
  else if constexpr (B == 2) FP4_MFMA(OUT, C, "op_sel:[0,0,0] op_sel_hi:[1,1,0]");     \
  else FP4_MFMA(OUT, C, "op_sel:[1,1,0] op_sel_hi:[1,1,0]")
template <int B>
__device__ __forceinline__ void asm_mfma(f32x16_t& c, const i32x4_t& w, const i32x4_t& x, int sw, int sx) {
  FP4_MFMA_BYTES("+a", "%0");
}
template <int B>
__device__ __forceinline__ void asm_mfma_first(f32x16_t& c, const i32x4_t& w, const i32x4_t& x, int sw, int sx) {
  FP4_MFMA_BYTES("=a", "0");
}

// grouped order: GM M-tiles share each run of N-tiles, for L2 reuse of both operands.  Groups, which XCDs go through side by
// side, start an eighth of the N-tiles apart: each part of W then comes from memory at its own time, most of it in the first
// rounds, and not at the same time for all, who wait for it in every round.  16896 x 16384 x 4096 behind a kernel that
// reads 256 MB 580 us for 668, 8192^3 277 for 290; with both operands still in the last cache the same.
// GM 4 for 256x256 tiles, 8 for smaller ones: the first behind the quantising of X 594 us (8: 612, 16: 634); 333 x 4096 x 4096
// 11.6 us (4: 12.3).
template <int GM>
__device__ __forceinline__ void tile_of(int id, int tm, int tn, int& im, int& in) {
  const int grp = id / (GM * tn), first = grp * GM, size = min(tm - first, GM), in_grp = id - grp * GM * tn;
  im = first + in_grp % size;
  in = (in_grp / size + grp * max(tn / 8, 1)) % tn;
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
__device__ __forceinline__ u32x4_t bits4(const float* v) {
  return u32x4_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
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

// 16 bytes of an output row that ends `left` columns further, at any element's address.  Past the caches, out of which the
// outputs would push the operands: 16896 x 16384 x 4096 572 us for 606, 4429 x 1536 x 1536 11.8 for 13.0.
template <bool F32>
__device__ __forceinline__ void store_chunk(char* y, const u32x4_t& w, int left) {
  constexpr int C = F32 ? 4 : 8;
  if (left >= C) {
    __builtin_nontemporal_store(w, &((Bf16x8*)y)->v);
  } else {
#pragma unroll
    for (int i = 0; i < C - 1; ++i)
      if (i < left) {
        if constexpr (F32) ((uint32_t*)y)[i] = w[i];
        else ((uint16_t*)y)[i] = (uint16_t)(w[i / 2] >> (i % 2 * 16));
      }
  }
}
// Lanes that differ in bits 3 and 4 and four registers change places: register k of lane (8 a + l), a < 4, is what register a
// of lane (8 k + l) was.
__device__ __forceinline__ void turn4(u32x4_t (&w)[4]) {
#pragma unroll
  for (int d = 0; d < 4; ++d) {
    uint32_t r[4];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const auto s = __builtin_amdgcn_permlane16_swap(w[k][d], w[k + 2][d], false, false);
      r[k] = s[0];
      r[k + 2] = s[1];
    }
#pragma unroll
    for (int k = 0; k < 4; k += 2) {  // row_ror:8, the upper or lower 8 lanes of each 16
      w[k][d] = __builtin_amdgcn_update_dpp(r[k], r[k + 1], 0x128, 0xf, 0xc, false);
      w[k + 1][d] = __builtin_amdgcn_update_dpp(r[k + 1], r[k], 0x128, 0xf, 0x3, false);
    }
  }
}

// ---------------------------------------------------------------- 256 x 256 tiles
constexpr int kMaxBlocks256 = 256;  // one per CU
constexpr int kStaggerKTiles = 8, kStaggerRounds = 6;
constexpr int kMinKTiles256 = 3;    // its loads run up to three K tiles ahead, into the next output tile at most

// 4 waves, one per SIMD, each 128 rows x 128 columns by 32x32x64 matrix instructions: 16
// sums of 16 registers each, in accumulation registers.  K tiles of 128 bytes (256
// elements) move by direct-to-LDS loads into two stages, each in parts: X's part c holds
// the c-th 32 rows of either wave row, W's part j fragment j of either wave column.  A K
// tile is 4 phases: phase c multiplies the wave's c-th 32 rows of X with all its rows of
// W (4 fragments of 4 steps, held for a whole tile, two tiles in turn), and between its
// 16 MFMAs reads the X of the next phase, fragment c of W of the next K tile, and issues
// its share of the loads.  One barrier ends a phase; ahead of it a wave's reads have
// returned, so a place is loaded again in the phase after its read: in phase 4 kt + c
// X's part c of tile kt + 2, and W's part c - 1 of tile kt + 3 (c = 0: part 3 of kt + 2).
// Both are read 7 phases after their load: loads have 6 phases.
// A block works through its output tiles as one stream of K tiles: the loads of the next
// output tile run ahead of the last K tiles of this one.  The finished sums of rows c are
// written between the MFMAs of the phase ahead of the one that starts them anew: rows 0
// in the last phase of the tile, 1 to 3 in the first three of the next.  W's rows are
// dealt out to the fragments so that a lane's and its neighbour's 16-byte chunks lie
// side by side; four chunks change places with those of the lanes of three other rows,
// and a store writes 128 bytes of each of 8 rows (16 bytes of each of 64 took 1068 us
// for 606 at 16896 x 16384 x 4096).
// 8192^3 248 us, 4.4 PFLOP/s; 16717 x 4096 x 16384 525 us; 16896 x 16384 x 4096 573 us;
// the same instructions without loads reach 6.7.  8 waves of 128 x 64, two on a SIMD, 268,
// 555 and 667 us: they read half as much again of LDS.  Here a phase's MFMAs issue back to
// back; its barrier, and the start and end of a block's work, take the rest.
template <bool F32>
__global__ __launch_bounds__(256) void fp4_256_kernel(const Fp4Problem p) {
  constexpr int BM = 256, BN = 256, Q = 4, NS = F32 ? 16 : 8;  // NS: stores of a phase
  constexpr int ROWB = 128;
  constexpr int STAGE = BM * ROWB, SUB = STAGE / Q, REGION = 2 * STAGE;
  // [X stage 0, 1 | W stage 0, 1 | scales stage 0, 1: 16 bytes of every row of X, then of W | bias of the last two output
  // tiles]
  constexpr int SCALES = 2 * REGION, SCALE_STAGE = 8192, BIAS = SCALES + 2 * SCALE_STAGE, BIAS_STAGE = 1024;
  __shared__ uint4 lds[(BIAS + 2 * BIAS_STAGE) / 16];
  char* const lbase = (char*)lds;
  const int tn = (p.N + BN - 1) / BN, tm = (p.M + BM - 1) / BM, tiles = tm * tn;
  // XCD x owns a contiguous range of tiles; its blocks take them in turn
  const int xcd = blockIdx.x & 7, per = tiles >> 3, rem = tiles & 7;
  const int tile_end = (xcd + 1) * per + min(xcd + 1, rem), tile_step = ((int)gridDim.x - xcd + 7) >> 3;
  int tile_next = xcd * per + min(xcd, rem) + (blockIdx.x >> 3);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wv >> 1, wn = wv & 1;
  // K tiles, and those of an output tile: an even number, the last one of zeros where K has an odd number
  const int KT = p.kt, Kp = p.pitch, KE = (KT + 1) & ~1;
  const int my_tiles = (tile_end - tile_next + tile_step - 1) / tile_step;

  // LDS slot of chunk c of row r: 16 consecutive rows' chunks lie in 16 different 16-byte bank groups
  auto swz = [](int row, int c) { return c ^ ((row >> 1) & 7); };
  // Byte offsets of this lane's row in the first of a wave's two loads of a part; the second takes rows 8 further, whose
  // slots differ in bit 2.  The part and the K tile travel in the scalar offset, which the range check counts.  Row i of
  // W's fragment j is column column(j) + HALF (i / 4 % 2) + 4 (i / 8) + i % 4 of its wave's 128.
  constexpr int HALF = F32 ? 16 : 32;
  constexpr auto column = [](int j) { return F32 ? j * 32 : j / 2 * 64 + j % 2 * 16; };
  const int lrow = wv * 16 + lane / 8, li = lrow & 31, lc = swz(lrow, lane % 8) * 16;
  const int gx = (int)((uint32_t)(lrow / 32 * 128 + li) * (uint32_t)Kp + lc);
  const int gw = (int)((uint32_t)(lrow / 32 * 128 + (li >> 2 & 1) * HALF + (li >> 3) * 4 + (li & 3)) * (uint32_t)Kp + lc);
  const int gs = (wv * 64 + lane) * p.spitch;
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
    tile_of<4>(id, tm, tn, im, in);
    m0 = __builtin_amdgcn_readfirstlane(im * BM);
    n0 = __builtin_amdgcn_readfirstlane(in * BN);
  };
  int m0, n0, m0_next, n0_next;  // this output tile and the next (behind the last one, itself again)
  tile_at(tile_next, m0, n0);
  m0_next = m0;
  n0_next = n0;
  int xm = m0, wn0 = n0, xk = 0, wk = 0;
  // half e of part c of the stream's K tile
  // (locals, not expressions, as the builtins' arguments: the host pass drops the kernel's launch stub otherwise)
  auto load_x = [&](auto stc, auto cc, auto ec) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value, c = decltype(cc)::value, e = decltype(ec)::value;
    const int vo = gx ^ (e * 64), so = xk * ROWB + (c * 32 + e * 8) * Kp;
    const __amdgpu_buffer_rsrc_t r = rows(p.x, xm, xk < KT ? BM : 0, p.M, Kp);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        r, (__attribute__((address_space(3))) void*)(lbase + st * STAGE + c * SUB + (wv * 2 + e) * 1024), 16, vo, so, 0, 0);
  };
  auto load_w = [&](auto stc, auto jc, auto ec) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value, j = decltype(jc)::value, e = decltype(ec)::value;
    const int vo = gw ^ (e * 64), so = wk * ROWB + (column(j) + e * 4) * Kp;
    const __amdgpu_buffer_rsrc_t r = rows(p.w, wn0, wk < KT ? BN : 0, p.N, Kp);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        r, (__attribute__((address_space(3))) void*)(lbase + REGION + st * STAGE + j * SUB + (wv * 2 + e) * 1024), 16, vo, so, 0, 0);
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
  // The scales of two K tiles, 512 elements, arrive together, 64 rows of X and 64 of W by each wave, and are read in the last
  // phase of the two K tiles before: their loads have 7 phases
  auto load_scales = [&](int stage, int m, int n, int k) __attribute__((always_inline)) {
    const int vo = gs, so = k * 8;
    const __amdgpu_buffer_rsrc_t rx = rows(p.xs, m, BM, p.M, p.spitch), rw = rows(p.ws, n, BN, p.N, p.spitch);
    char* const to = lbase + SCALES + stage * SCALE_STAGE + wv * 1024;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (__attribute__((address_space(3))) void*)to, 16, vo, so, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (__attribute__((address_space(3))) void*)(to + 4096), 16, vo, so, 0, 0);
  };
  // the tile's bias, one value per word; zeros past N
  auto load_bias = [&](int stage) __attribute__((always_inline)) {
    const int es = p.bias_f32 ? 4 : 2, n = p.bias ? max(p.N - n0, 0) * es : 0, vo = (wv * 64 + lane) * es;
    const __amdgpu_buffer_rsrc_t r = buffer((const uint8_t*)p.bias + (long)n0 * es, n);
    __attribute__((address_space(3))) void* const to =
        (__attribute__((address_space(3))) void*)(lbase + BIAS + stage * BIAS_STAGE + wv * 256);
    if (p.bias_f32) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 4, vo, 0, 0, 0);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 2, vo, 0, 0, 0);
  };

  // ---- fragment reads: row lane % 32 of a 32-row fragment, at step s chunk 2 s + lane / 32
  const int half = lane >> 5;
  const int xr = wm * 32 + (lane & 31), wr = wn * 32 + (lane & 31);
  const int xa = xr * ROWB + swz(xr, half) * 16, wa = REGION + wr * ROWB + swz(wr, half) * 16;
  // Whole-value casts: read member by member, the compiler takes them to alias the loads in flight and waits for those.
  auto lds16 = [&](int at) __attribute__((always_inline)) {
    return __builtin_bit_cast(i32x4_t, *(const uint4*)(lbase + at));
  };
  auto lds4 = [&](int at) __attribute__((always_inline)) {
    return __builtin_bit_cast(int, *(const Word*)(lbase + at));
  };
  const int xs0 = SCALES + (wm * 128 + (lane & 31)) * 16 + half * 4;
  const int ws0 = SCALES + 4096 + (wn * 128 + (lane >> 2 & 1) * HALF + (lane >> 3 & 3) * 4 + (lane & 3)) * 16 + half * 4;
  f32x16_t acc[Q][4];
  // X fragments of a phase and its scale words (phases in turn), W fragments of a K tile (K tiles in turn) and the scale
  // words of two K tiles, those of the next two arriving while the last phases still take the ones before
  i32x4_t fx[2][4], fw[2][4][4];
  int sx[2][2], sw[4][2], sw_next[4][2];
  auto read_x = [&](auto stc, auto cc, auto sc) __attribute__((always_inline)) {  // step s of part c
    constexpr int st = decltype(stc)::value, c = decltype(cc)::value, s = decltype(sc)::value;
    fx[c & 1][s] = lds16((xa ^ (s * 32)) + st * STAGE + c * SUB);
  };
  auto read_w = [&](auto stc, auto jc, auto sc) __attribute__((always_inline)) {  // step s of fragment j
    constexpr int st = decltype(stc)::value, j = decltype(jc)::value, s = decltype(sc)::value;
    fw[st][j][s] = lds16((wa ^ (s * 32)) + st * STAGE + j * SUB);
  };
  auto read_sx = [&](auto cc, int stage) __attribute__((always_inline)) {
    constexpr int c = decltype(cc)::value;
#pragma unroll
    for (int h = 0; h < 2; ++h) sx[c & 1][h] = lds4(xs0 + stage * SCALE_STAGE + c * 32 * 16 + h * 8);
  };
  auto read_sw = [&](auto jc, int stage) __attribute__((always_inline)) {
    constexpr int j = decltype(jc)::value;
#pragma unroll
    for (int h = 0; h < 2; ++h) sw_next[j][h] = lds4(ws0 + stage * SCALE_STAGE + column(j) * 16 + h * 8);
  };

  // The next two K tiles' words of W, ahead of a barrier: an MFMA reads what a vector instruction wrote two instructions
  // later at the earliest, which the compiler does not know of the statements.
  auto take_sw = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) sw[j][h] = sw_next[j][h];
    __builtin_amdgcn_sched_barrier(0);
  };

  // ---- the finished sums of rows c of the tile at (m0, n0), whose bias is in `stage`, in groups of four chunks of 16 bytes
  constexpr int ES = F32 ? 4 : 2, C = 16 / ES, GROUPS = NS / 4, STEPS = 16 / GROUPS;
  const uint32_t pitch = (uint32_t)p.N * ES;
  const int bias_shift = p.bias_f32 ? 0 : 16;
  u32x4_t out[4];
  auto take = [&](auto cc, auto gc, auto kc, int stage) __attribute__((always_inline)) {
    constexpr int c = decltype(cc)::value, g = decltype(gc)::value, k = decltype(kc)::value;
    constexpr int j = F32 ? g : 2 * g + k / 2, r0 = F32 ? 4 * k : k % 2 * 8;
    const int at = opaque(wn * 128 + half * HALF) * 4 + (column(j) + r0) * 4 + BIAS + stage * BIAS_STAGE;
    float v[C];
#pragma unroll
    for (int e = 0; e < C; e += 4) {
      const i32x4_t b = lds16(at + e * 4);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[e + r] = acc[c][j][r0 + e + r] + __uint_as_float((uint32_t)b[r] << bias_shift);
    }
    if constexpr (F32) out[k] = bits4(v);
    else out[k] = pack8(v);
  };
  auto put = [&](auto cc, auto gc, auto kc, int m0, int n0) __attribute__((always_inline)) {
    constexpr int c = decltype(cc)::value, g = decltype(gc)::value, k = decltype(kc)::value;
    const int mr = opaque(wm * 128 + (lane & 7)), nc = opaque(wn * 128 + half * HALF + (lane >> 3 & 3) * C);
    const uint32_t yo = (uint32_t)(mr + c * 32 + k * 8) * pitch + (uint32_t)(nc + g * 8 * C) * ES;
    char* const y = (char*)p.y + ((long)m0 * p.N + n0) * ES + yo;
    if (mr < p.M - m0 - c * 32 - k * 8) store_chunk<F32>(y, out[k], p.N - n0 - nc - g * 8 * C);
  };
  // step i of 16
  auto store = [&](auto cc, auto ic, int m0, int n0, int stage) __attribute__((always_inline)) {
    constexpr int i = decltype(ic)::value, n = 8 / STEPS;
    using G = std::integral_constant<int, i / STEPS>;
    static_for<n>([&](auto ec) {
      constexpr int at = i % STEPS * n + decltype(ec)::value;
      if constexpr (at < 4) take(cc, G{}, std::integral_constant<int, at>{}, stage);
      if constexpr (at == 3) turn4(out);
      if constexpr (at >= 4) put(cc, G{}, std::integral_constant<int, at - 4>{}, m0, n0);
    });
  };

  using S0 = std::integral_constant<int, 0>;
  using S1 = std::integral_constant<int, 1>;
  int prev_m0 = p.M, prev_n0 = 0, scale_stage = 0, bias_stage = 0;  // no row of the tile before the first exists
  bool counted = false;  // NS stores a phase by every wave
  // PAIR 1: the output tile's first two K tiles, which write rows 1 to 3 of the tile before; 2: its last two, the last
  // phase of which writes its rows 0
  auto phase = [&](auto stc, auto cc, auto pairc) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value, c = decltype(cc)::value, PAIR = decltype(pairc)::value;
    constexpr bool FIRST = PAIR == 1 && st == 0, STORE = (FIRST && c < 3) || (PAIR == 2 && st == 1 && c == 3);
    using CN = std::integral_constant<int, (c + 1) % Q>;
    using SN = std::integral_constant<int, c + 1 < Q ? st : st ^ 1>;  // stage of the next phase's X
    using CW = std::integral_constant<int, (c + Q - 1) % Q>;
    using SW = std::integral_constant<int, c == 0 ? st : st ^ 1>;
    using ST1 = std::integral_constant<int, st ^ 1>;
    // The sums to be written are read from here on only: the compiler does not know how long the statements that made them
    // run, and would take some right behind the last of those.
    if constexpr (STORE)
#pragma unroll
      for (int j = 0; j < 4; ++j) asm volatile("" : "+a"(acc[CN::value][j]));
    static_for<16>([&](auto ic) {
      constexpr int i = decltype(ic)::value, s = i / 4, j = i % 4;
      if constexpr (FIRST && s == 0) asm_mfma_first<st * 2>(acc[c][j], fw[st][j][s], fx[c & 1][s], sw[j][0], sx[c & 1][0]);
      else asm_mfma<st * 2 + s / 2>(acc[c][j], fw[st][j][s], fx[c & 1][s], sw[j][s & 1], sx[c & 1][s & 1]);
      using I4 = std::integral_constant<int, i % 4>;
      if constexpr (i < 4) read_x(SN{}, CN{}, I4{});
      else if constexpr (i < 8) read_w(ST1{}, cc, I4{});
      else if constexpr (i == 8) read_sx(CN{}, c + 1 == Q && st == 1 ? scale_stage ^ 1 : scale_stage);
      else if constexpr (i == 9 && st == 1 && c == 3) static_for<4>([&](auto jc) { read_sw(jc, scale_stage ^ 1); });
      else if constexpr (i == 10) load_x(stc, cc, S0{});
      else if constexpr (i == 11) load_x(stc, cc, S1{});
      else if constexpr (i == 12) load_w(SW{}, CW{}, S0{});
      else if constexpr (i == 13) load_w(SW{}, CW{}, S1{});
      if constexpr (STORE) {
        if constexpr (PAIR == 1) store(CN{}, ic, prev_m0, prev_n0, bias_stage ^ 1);
        else store(CN{}, ic, m0, n0, bias_stage);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (c == 0) next_wk();
    if constexpr (c == 3) next_xk();
    // All but the loads of the last 6 phases have landed.  Those phases' stores need not have: those of the tile's last phase
    // and of the first three of the next, if all of its rows and columns exist.
    constexpr int at = st * 4 + c;  // phase of the pair
    constexpr int n = PAIR == 1 ? (at < 3 ? at + 2 : at < 5 ? 4 : 8 - at) : PAIR == 2 && at == 7 ? 1 : 0;
    constexpr int most = 24 + n * NS < 62 ? 24 + n * NS : 62;  // (63 is no wait)
    if (n > 0 && counted) wait_vmcnt<most>();
    else wait_vmcnt<24>();
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    if constexpr (st == 1 && c == 3) take_sw();
    block_barrier();
  };
  auto k_pair = [&](auto pairc, int kt) __attribute__((always_inline)) {
    constexpr int PAIR = decltype(pairc)::value;
    const bool on = kt + 2 >= KE;
    load_scales(scale_stage ^ 1, on ? m0_next : m0, on ? n0_next : n0, on ? 0 : kt + 2);
    static_for<Q>([&](auto cc) { phase(S0{}, cc, pairc); });
    static_for<Q>([&](auto cc) {
      if constexpr (PAIR == 2 && decltype(cc)::value == 3) counted = m0 + BM <= p.M && n0 + BN <= p.N;
      phase(S1{}, cc, pairc);
    });
    scale_stage ^= 1;
  };
  using E0 = S0;
  using E1 = S1;
  auto both_x = [&](auto stc, auto cc) __attribute__((always_inline)) {
    load_x(stc, cc, E0{});
    load_x(stc, cc, E1{});
  };
  auto both_w = [&](auto stc, auto cc) __attribute__((always_inline)) {
    load_w(stc, cc, E0{});
    load_w(stc, cc, E1{});
  };
  using P1 = std::integral_constant<int, 1>;
  using P2 = std::integral_constant<int, 2>;
  using P3 = std::integral_constant<int, 3>;
  // Blocks that finish a tile at the same time write at the same time, and wait for it.  An XCD's 32 blocks start up to 6 us
  // apart where a block has several tiles of short K to win that back.  Quantising of X and product, in us, with it and with
  // the same code that starts at once: 16717 x 6144 x 1536 139 and 141, in fp32 160 and 169; 16717 x 6144 x 2048 166 and 167;
  // 16896 x 8192 x 2048 207 and 210; 16896 x 16384 x 1024 256 and 264; 24000 x 16384 x 800 348 and 358; 8192 x 16384 x 1024
  // 132 and 136, in fp32 x 2048 214 both; 20000 x 5000 x 1800 218 both; but 16384 x 6144 x 768, just six tiles a block, 105
  // and 102.  A card with faster memory gains half as much.  16896 x 16384 x 4096 617 and 609, and so long K starts at once.
  if (KT <= kStaggerKTiles && tiles >= kStaggerRounds * kMaxBlocks256)
    for (int i = (int)blockIdx.x >> 3; i > 0; --i) __builtin_amdgcn_s_sleep(6);
  // as 8 phases ahead of the first would have: those that load tile 0's and 1's places
  load_scales(0, m0, n0, 0);
  both_w(S0{}, S0{});
  both_w(S0{}, P1{});
  both_w(S0{}, P2{});
  both_x(S0{}, S0{});
  both_w(S0{}, P3{});
  next_wk();
  both_x(S0{}, P1{});
  both_w(S1{}, S0{});
  both_x(S0{}, P2{});
  both_w(S1{}, P1{});
  both_x(S0{}, P3{});
  both_w(S1{}, P2{});
  next_xk();
  both_x(S1{}, S0{});
  both_w(S1{}, P3{});
  next_wk();
  wait_vmcnt<16>();
  block_barrier();
  static_for<Q>([&](auto jc) {
    static_for<4>([&](auto sc) { read_w(S0{}, jc, sc); });
    read_sw(jc, 0);
  });
  static_for<4>([&](auto sc) { read_x(S0{}, S0{}, sc); });
  read_sx(S0{}, 0);
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  block_barrier();
  both_x(S1{}, P1{});
  both_w(S0{}, S0{});
  both_x(S1{}, P2{});
  both_w(S0{}, P1{});
  both_x(S1{}, P3{});
  both_w(S0{}, P2{});
  next_xk();
  wait_vmcnt<24>();  // what phase 0 reads has landed
  take_sw();
  block_barrier();
#pragma unroll 1
  for (int t = 0; t < my_tiles; ++t) {
    load_bias(bias_stage);
    tile_next += tile_step;
    if (tile_next < tile_end) tile_at(tile_next, m0_next, n0_next);
    k_pair(P1{}, 0);
#pragma unroll 1
    for (int kt = 2; kt < KE - 2; kt += 2) k_pair(S0{}, kt);
    k_pair(P2{}, KE - 2);
    prev_m0 = m0;
    prev_n0 = n0;
    bias_stage ^= 1;
    m0 = m0_next;
    n0 = n0_next;
  }
  wait_vmcnt<0>();  // the loads past the last K tile land before the block ends
  asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory");  // the last MFMAs' results
#pragma unroll
  for (int i = 1; i < Q; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) asm volatile("" : "+a"(acc[i][j]));
  static_for<Q - 1>([&](auto cc) {
    static_for<16>([&](auto ic) {
      store(std::integral_constant<int, decltype(cc)::value + 1>{}, ic, prev_m0, prev_n0, bias_stage ^ 1);
    });
  });
}

// ---------------------------------------------------------------- smaller tiles
// c += x w of 128 elements, the scales in byte B of their words; only four of an operand's registers hold 4-bit codes
template <int B>
__device__ __forceinline__ f32x4_t mfma(const i32x4_t& w, const i32x4_t& x, const f32x4_t& c, int sw, int sx) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_shufflevector(w, w, 0, 1, 2, 3, 0, 1, 2, 3),
                                                          __builtin_shufflevector(x, x, 0, 1, 2, 3, 0, 1, 2, 3), c, 4, 4, B, sw,
                                                          B, sx);
}
// acc += the products of one K tile's fragments, two steps of 128 elements; the scale bytes are the words' lower two
template <int FM, int FN>
__device__ __forceinline__ void multiply(const i32x4_t (*x)[2], const i32x4_t (*w)[2], const int* sx, const int* sw,
                                         f32x4_t (*acc)[FN]) {
  static_for<2>([&](auto sc) {
    constexpr int s = decltype(sc)::value;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = mfma<s>(w[j][s], x[i][s], acc[i][j], sw[j], sx[i]);
  });
}

// a launch's blocks along x (fewer than 2^32 threads), the rest goes on along y
constexpr int kRingRowLog2 = 22;

// BM x BN outputs per block; KG groups of WM x WN waves share out the K tiles.  A
// step is KG K tiles, which arrive by direct-to-LDS loads in a ring of ST stages;
// the groups' sums meet in LDS at the end, in their order.  For bf16 outputs W's rows are
// dealt out to the fragments so that a lane holds 8 neighbouring columns of each of its
// rows; fp32 ones fill 64 bytes of a row by four lanes as they are (dealt out likewise,
// and kept in the caches, 16717 x 6144 x 1536 took 165 us for 157).
// 64x64 with two groups: 10.5 us at 333 x 4096 x 4096, bound by the loads' latency over
// 8 steps.  128x128: 16.0 us at 1024 x 4096 x 4096, 2.1 PFLOP/s: 3.8 to start and end, and
// 0.67 a K tile, of which the MFMAs take 0.32.
template <bool F32, int BM, int BN, int WM, int WN, int KG, int ST>
__global__ __launch_bounds__(WM* WN* KG * 64) void fp4_ring_kernel(const Fp4Problem p) {
  constexpr int NW = WM * WN * KG, FM = BM / WM / 16, FN = BN / WN / 16;
  constexpr int ROWB = 128, UNITS = KG * (BM + BN) / 8, LPW = UNITS / NW;  // loads of 8 rows; per wave and step
  constexpr int SU = (BM + BN) / 64;  // loads of 64 rows' scales, by as many waves
  constexpr int TILE = (BM + BN) * ROWB, SCALES = KG * TILE, STAGE = SCALES + (BM + BN) * 16;
  static_assert(LPW * NW == UNITS && BM % 64 == 0 && BN % 64 == 0 && SU <= NW && KG <= 2, "tile config");
  static_assert(ST * STAGE <= 160 * 1024 && (KG - 1) * WM * WN * FM * FN * 1024 <= ST * STAGE, "LDS");
  static_assert(FN == 2, "a lane's 8 columns of a row make one store of bf16, two of fp32");
  __shared__ uint4 lds[ST * STAGE / 16];
  char* const lbase = (char*)lds;
  const int tn = (p.N + BN - 1) / BN, tm = (p.M + BM - 1) / BM;
  const int id = (int)(blockIdx.y << kRingRowLog2) + xcd_remap(blockIdx.x, gridDim.x);
  if (id >= tm * tn) return;
  int im, in;
  tile_of<8>(id, tm, tn, im, in);
  const int m0 = im * BM, n0 = in * BN, KT = p.kt, Kp = p.pitch, steps = (KT + KG - 1) / KG;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), kg = wv / (WM * WN), wm = wv / WN % WM, wn = wv % WN;
  auto swz = [](int row, int c) { return c ^ ((row >> 1) & 7); };
  // row of X or of W that lies in row `row` of a tile: X's as they come, W's, for bf16 outputs, dealt out to the fragments
  auto source = [](int row) {
    constexpr int C = BN / WN;
    const int w = row - BM, in_wave = w % C, f = in_wave & 15;
    if (row < BM || F32) return row < BM ? row : w;
    return w - in_wave + (f >> 2) * (4 * FN) + (in_wave >> 4) * 4 + (f & 3);
  };

  // this wave's loads of a step: 8 rows each of X or W of one K tile
  uint32_t go[LPW];
#pragma unroll
  for (int i = 0; i < LPW; ++i) {
    const int row = (wv * LPW + i) * 8 % (BM + BN) + (lane >> 3);
    go[i] = (uint32_t)source(row) * (uint32_t)Kp + swz(row, lane & 7) * 16;
  }
  auto buffer = [&](const uint8_t* base, int r0, int most, int rows, int pitch) __attribute__((always_inline)) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)(base + (long)r0 * pitch), (short)0,
                                             __builtin_amdgcn_readfirstlane(max(min(rows - r0, most), 0) * pitch), kBufferWord3);
  };
  const int sgo = source(min(wv, SU - 1) * 64 + lane) * p.spitch;
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
    // the scales of the 512 elements that the step lies in, a row per lane
    if (wv < SU) {
      const bool x = wv < BM / 64;
      const int vo = sgo, so = (min(step * KG, KT - 1) >> 1) * 16;
      const __amdgpu_buffer_rsrc_t rs = buffer(x ? p.xs : p.ws, x ? m0 : n0, x ? BM : BN, x ? p.M : p.N, p.spitch);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rs, (__attribute__((address_space(3))) void*)(at + SCALES + wv * 1024), 16, vo, so, 0, 0);
    }
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
  const int sxa = SCALES + xr * 16 + (lane >> 4) * 4, swa = SCALES + wr * 16 + (lane >> 4) * 4;
  f32x4_t acc[FM][FN] = {};
  static_for<ST - 1>([&](auto sc) { load(decltype(sc)::value, decltype(sc)::value); });
  int stage = 0;
  for (int s = 0; s < steps; ++s) {
    // step s has landed, this wave's part and, behind the barrier, everyone's; the stage before it is read no more
    if (wv < SU) wait_vmcnt<(ST - 2) * (LPW + 1)>();
    else wait_vmcnt<(ST - 2) * LPW>();
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    block_barrier();
    load(s + ST - 1, stage == 0 ? ST - 1 : stage - 1);
    const int at = stage * STAGE, shift = ((s * KG + kg) & 1) * 16;
    i32x4_t x[FM][2], w[FN][2];
    int sx[FM], sw[FN];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) x[i][h] = lds16(at + xa[h] + i * 16 * ROWB);
      sx[i] = lds4(at + sxa + i * 256) >> shift;
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
#pragma unroll
      for (int h = 0; h < 2; ++h) w[j][h] = lds16(at + wa[h] + j * 16 * ROWB);
      sw[j] = lds4(at + swa + j * 256) >> shift;
    }
    multiply<FM, FN>(x, w, sx, sw, acc);
    stage = stage + 1 == ST ? 0 : stage + 1;
  }
  wait_vmcnt<0>();
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
  // fragment j's four columns of a lane: 16 j from its first, so that four lanes' chunks of fp32 make 64 bytes, for bf16 4 j
  constexpr int STEP = F32 ? 16 : 4;
  const int n = n0 + wn * FN * 16 + (lane >> 4) * (F32 ? 4 : 4 * FN);
  float b[4 * FN];
#pragma unroll
  for (int i = 0; i < 4 * FN; ++i) {
    const int at = n + i / 4 * STEP + i % 4;
    b[i] = at < p.N ? bias_at(p, at) : 0.f;
  }
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const long m = m0 + wm * FM * 16 + i * 16 + (lane & 15);
    if (m >= p.M) continue;
    float v[4 * FN];
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) v[j * 4 + r] = acc[i][j][r] + b[j * 4 + r];
    char* const y = (char*)p.y + (m * p.N + n) * (F32 ? 4 : 2);
    if constexpr (F32) {
#pragma unroll
      for (int j = 0; j < FN; ++j) store_chunk<F32>(y + j * STEP * 4, bits4(v + j * 4), p.N - n - j * STEP);
    } else {
      store_chunk<F32>(y, pack8(v), p.N - n);
    }
  }
}

// ---------------------------------------------------------------- small tiles, K shared out to the waves
// BM x BN = 16 FM x 16 FN outputs per block, NW waves that share out the K tiles: a
// wave multiplies all rows and columns of its K tiles, which nobody else reads, so
// the waves need no barrier until their sums meet in LDS, in wave order.  K tiles
// arrive by direct-to-LDS loads in two stages of each wave's own, their scales in
// registers.  As above W's rows are dealt out to the fragments, and a lane ends with 4
// FN neighbouring columns of a row.  16x32 6.2 us at 33 x 1536 x 6144, 32x32 7.8 us at
// 128 x 1536 x 6144: the latency of a wave's 6 K tiles.
template <bool F32, int FM, int FN, int NW>
__global__ __launch_bounds__(NW * 64) void fp4_split_kernel(const Fp4Problem p) {
  constexpr int BM = FM * 16, BN = FN * 16, ROWB = 128, TILE = (BM + BN) * ROWB;
  constexpr int LOADS = (BM + BN) / 8 + FM + FN;  // of a K tile
  __shared__ uint4 lds[NW * 2 * TILE / 16];       // [wave][stage][X's rows, then W's]; then the waves' sums
  static_assert(FM <= NW && FM * FN * 1024 <= 2 * TILE, "tile config");
  const int tn = (p.N + BN - 1) / BN, tm = (p.M + BM - 1) / BM;
  const int id = (int)(blockIdx.y << kRingRowLog2) + xcd_remap(blockIdx.x, gridDim.x);
  if (id >= tm * tn) return;
  int im, in;
  tile_of<8>(id, tm, tn, im, in);
  const int m0 = im * BM, n0 = in * BN, Kp = p.pitch;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lr = lane & 15, g = lane >> 4;
  char* const lbase = (char*)lds + wv * 2 * TILE;
  auto swz = [](int row, int c) { return c ^ ((row >> 1) & 7); };
  // loads of 8 rows: of X, and of either half of a fragment of W
  const int row = lane >> 3;
  uint32_t xo[2], wo[2], xso[FM], wso[FN];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = h * 8 + row, c = swz(r, lane & 7) * 16;
    xo[h] = row * (uint32_t)Kp + c;
    wo[h] = (uint32_t)((r >> 2) * (4 * FN) + (r & 3)) * (uint32_t)Kp + c;
  }
  // rows past the last one: its scales
#pragma unroll
  for (int i = 0; i < FM; ++i) xso[i] = min(i * 16 + lr, p.M - 1 - m0) * (uint32_t)p.spitch + g * 4;
#pragma unroll
  for (int j = 0; j < FN; ++j) wso[j] = min((lr >> 2) * (4 * FN) + j * 4 + (lr & 3), p.N - 1 - n0) * (uint32_t)p.spitch + g * 4;
  // rows and K tiles past the last one read as zeros, with the last one's scales
  auto rows = [&](const uint8_t* base, int r0, int most, int n, int pitch) __attribute__((always_inline)) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)(base + (long)r0 * pitch), (short)0,
                                             __builtin_amdgcn_readfirstlane(min(n - r0, most) * pitch), kBufferWord3);
  };
  int sx[2][FM], sw[2][FN];
  auto load = [&](int kt, auto stc) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value;
    const bool in = kt < p.kt;
    const __amdgpu_buffer_rsrc_t rx = rows(p.x, m0, in ? BM : 0, p.M, Kp), rw = rows(p.w, n0, in ? BN : 0, p.N, Kp);
    const __amdgpu_buffer_rsrc_t rsx = rows(p.xs, m0, BM, p.M, p.spitch), rsw = rows(p.ws, n0, BN, p.N, p.spitch);
    const int ks = (min(kt, p.kt - 1) >> 1) * 16;
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
    for (int i = 0; i < FM; ++i) sx[st][i] = __builtin_amdgcn_raw_buffer_load_b32(rsx, xso[i], ks, 0);
#pragma unroll
    for (int j = 0; j < FN; ++j) sw[st][j] = __builtin_amdgcn_raw_buffer_load_b32(rsw, wso[j], ks, 0);
    __builtin_amdgcn_sched_barrier(0);
  };
  int fa[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) fa[h] = lr * ROWB + swz(lr, g + 4 * h) * 16;
  auto lds16 = [&](int at) __attribute__((always_inline)) {
    return __builtin_bit_cast(i32x4_t, *(const uint4*)(lbase + at));
  };
  f32x4_t acc[FM][FN] = {};
  auto step = [&](int kt, auto stc) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value;
    wait_vmcnt<LOADS>();  // all but the next K tile's loads
    __builtin_amdgcn_sched_barrier(0);
    i32x4_t x[FM][2], w[FN][2];
    int xs[FM], ws[FN];
    const int shift = (kt & 1) * 16;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) x[i][h] = lds16(st * TILE + i * 16 * ROWB + fa[h]);
      xs[i] = sx[st][i] >> shift;
    }
#pragma unroll
    for (int j = 0; j < FN; ++j) {
#pragma unroll
      for (int h = 0; h < 2; ++h) w[j][h] = lds16(st * TILE + (BM + j * 16) * ROWB + fa[h]);
      ws[j] = sw[st][j] >> shift;
    }
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): read, before the K tile after the next arrives here
    __builtin_amdgcn_sched_barrier(0);
    load(kt + 2 * NW, stc);
    multiply<FM, FN>(x, w, xs, ws, acc);
    __builtin_amdgcn_sched_barrier(0);
  };
  using S0 = std::integral_constant<int, 0>;
  using S1 = std::integral_constant<int, 1>;
  load(wv, S0{});
  load(wv + NW, S1{});
#pragma unroll 1
  for (int k = wv; k < p.kt; k += 2 * NW) {
    step(k, S0{});
    step(k + NW, S1{});
  }
  wait_vmcnt<0>();
  uint4* const sums = lds + lane;
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) sums[wv * (2 * TILE / 16) + (i * FN + j) * 64] = __builtin_bit_cast(uint4, acc[i][j]);
  __syncthreads();
  if (wv >= FM) return;  // wave i finishes rows 16 i ..
  const int m = m0 + wv * 16 + lr, n = n0 + g * (4 * FN);
  if (m >= p.M || n >= p.N) return;
  float v[4 * FN];
#pragma unroll
  for (int j = 0; j < FN; ++j) {
    f32x4_t s = __builtin_bit_cast(f32x4_t, sums[(wv * FN + j) * 64]);
#pragma unroll
    for (int q = 1; q < NW; ++q) s += __builtin_bit_cast(f32x4_t, sums[q * (2 * TILE / 16) + (wv * FN + j) * 64]);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[j * 4 + r] = s[r] + (n + j * 4 + r < p.N ? bias_at(p, n + j * 4 + r) : 0.f);
  }
  store_columns<F32, 4 * FN>((char*)p.y + ((long)m * p.N + n) * (F32 ? 4 : 2), v, p.N - n);
}

// ---------------------------------------------------------------- few rows
// Up to 16 rows of X against 16 columns per block: W is read once, straight from
// memory to registers, and the block's waves share out the K tiles, two in flight
// each.  Their sums meet in LDS in wave order.  4.5 us at 1 x 4096 x 4096, of which
// 4.2 is any launch's: 8.4 MB would pass in 1.6 from memory, here they come from the caches.
template <bool F32>
__global__ __launch_bounds__(512) void fp4_rows_kernel(const Fp4Problem p) {
  constexpr int NW = 8, U = 2;
  __shared__ f32x4_t part[NW][64];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 15, g = lane >> 4, n0 = blockIdx.x * 16;
  const long wrow = min(n0 + lr, p.N - 1), xrow = min(lr, p.M - 1);
  const uint8_t* const w = p.w + wrow * p.pitch + g * 16;
  const uint8_t* const ws = p.ws + wrow * p.spitch + g * 4;
  const uint8_t* const x = p.x + xrow * p.pitch + g * 16;
  const uint8_t* const xs = p.xs + xrow * p.spitch + g * 4;
  f32x4_t acc[1][1] = {};
  for (int k0 = wv; k0 < p.kt; k0 += NW * U) {
    int sw[U], sx[U];
    i32x4_t wf[U][1][2], xf[U][1][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kt = min(k0 + u * NW, p.kt - 1);  // past the end: loaded again, not multiplied
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        wf[u][0][h] = *(const i32x4_t*)(w + (long)kt * 128 + h * 64);
        xf[u][0][h] = *(const i32x4_t*)(x + (long)kt * 128 + h * 64);
      }
      sw[u] = *(const int*)(ws + (kt >> 1) * 16) >> (kt & 1) * 16;
      sx[u] = *(const int*)(xs + (kt >> 1) * 16) >> (kt & 1) * 16;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (k0 + u * NW < p.kt) multiply<1, 1>(xf[u], wf[u], &sx[u], &sw[u], acc);
  }
  part[wv][lane] = acc[0][0];
  __syncthreads();
  if (wv > 0) return;
  f32x4_t s = part[0][lane];
#pragma unroll
  for (int q = 1; q < NW; ++q) s += part[q][lane];
  const int m = lr, n = n0 + g * 4;
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

// Which kernel a product takes.  Up to 16 rows and 8 MB of W's codes, the one that streams W: 5.1 us for the best other's
// 5.3 at (M, N, K) = (16, 4096, 4096) and 6.1 for 6.3 at (16, 1536, 6144), but 13.2 for 8.6 at (16, 16384, 4096), as each
// of its blocks reads all of X.  Otherwise the one whose modelled time is least: a start and a cost of each round of
// blocks, per block and per K tile, in us, fitted to all kernels' times at 196 shapes of 1 to 16717 rows and both output
// types.  The kernel taken is 0.2% behind the best there on average, and at most 1% but for up to 15% at three shapes of 700
// columns in fp32, where 64x64 tiles are better than their rounds.  Around the changes, in us (the kernel
// taken first): (33, 1536, 6144) 16x32 6.3, 32x32 7.7, 64x64 8.6; (128, 1536, 6144) 32x32 7.8, 64x64 8.7, 16x32 10.3;
// (333, 4096, 4096) 64x64 10.4, 128x128 14.7, 32x32 26.5; (1024, 4096, 4096) 128x128 16.2, 64x64 20.9, 256x256 32.6;
// (8192, 4096, 4096) 256x256 79, 128x128 99, 64x64 150.
enum Fp4Cfg { FP4_ROWS, FP4_16X32, FP4_32X32, FP4_64, FP4_128, FP4_256 };
static Fp4Cfg pick(int M, int N, int K) {
  const double kt = fp4_pitch(K) / 128;
  if (M <= 16 && N * kt * 128 <= 1 << 23) return FP4_ROWS;
  auto rounds = [&](int bm, int bn) { return ceil(ceil((double)M / bm) * ceil((double)N / bn) / 256.0); };
  // two blocks share a CU from the second round on
  auto ring = [&](int b, double c, double pair, double pair_kt, double odd, double odd_kt) {
    const double n = rounds(b, b);
    return c + floor(n / 2) * (pair + pair_kt * kt) + (n - 2 * floor(n / 2)) * (odd + odd_kt * kt);
  };
  Fp4Cfg cfg = FP4_64;
  double best = rounds(64, 64) <= 1 ? 4.0 + 0.22 * kt : ring(64, 2.0, 1.76, 0.475, 0.0, 0.408);
  auto offer = [&](Fp4Cfg c, double us) {
    if (us < best) {
      best = us;
      cfg = c;
    }
  };
  const double memory = 3.3 + N * kt * 128 / 5.6e6;
  offer(FP4_16X32, fmax(3.0 + rounds(16, 32) * (0.94 + 0.12 * kt), memory));
  offer(FP4_32X32, fmax(3.2 + rounds(32, 32) * (1.18 + 0.144 * kt), memory));
  offer(FP4_128, rounds(128, 128) <= 1 ? 4.26 + 0.635 * kt : ring(128, 0.44, 5.7, 1.19, 0.74, 0.89));
  // offsets within a tile of 256 output rows fit 32 bits up to 2^21 columns
  if (kt >= kMinKTiles256 && N <= 1 << 21)
    offer(FP4_256, rounds(256, 256) <= 1 ? 21.4 + 0.95 * kt : rounds(256, 256) * (13.7 + 1.47 * kt));
  return cfg;
}

const char* gemm_fp4_config_name(int M, int N, int K) {
  static const char* names[] = {"gemm_fp4_rows", "gemm_fp4_16x32", "gemm_fp4_32x32", "gemm_fp4_64x64", "gemm_fp4_128x128", "gemm_fp4_256x256"};
  return names[pick(M, N, K)];
}

static dim3 ring_grid(long blocks) {
  return dim3((unsigned)std::min(blocks, 1L << kRingRowLog2), (unsigned)((blocks - 1) >> kRingRowLog2) + 1);
}

// Two stages leave room for a second block on a CU, whose loads and products go on while the first one waits or stores; a
// launch of one block a CU needs four to cover its loads.
template <bool F32, int BM, int BN, int WM, int WN, int KG>
static void launch_ring(const Fp4Problem& p, hipStream_t s) {
  const long tiles = (long)((p.M + BM - 1) / BM) * ((p.N + BN - 1) / BN);
  const dim3 grid = ring_grid(tiles), block(WM * WN * KG * 64);
  if (tiles <= 256) hipLaunchKernelGGL((fp4_ring_kernel<F32, BM, BN, WM, WN, KG, 4>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((fp4_ring_kernel<F32, BM, BN, WM, WN, KG, 2>), grid, block, 0, s, p);
}

template <bool F32, int FM, int FN>
static void launch_split(const Fp4Problem& p, hipStream_t s) {
  constexpr int NW = 4, BM = FM * 16, BN = FN * 16;
  const dim3 grid = ring_grid((long)((p.M + BM - 1) / BM) * ((p.N + BN - 1) / BN));
  hipLaunchKernelGGL((fp4_split_kernel<F32, FM, FN, NW>), grid, dim3(NW * 64), 0, s, p);
}

template <bool F32>
static void launch(Fp4Cfg cfg, const Fp4Problem& p, hipStream_t s) {
  if (cfg == FP4_256) {
    const long tiles = (long)((p.M + 255) / 256) * ((p.N + 255) / 256);
    hipLaunchKernelGGL(fp4_256_kernel<F32>, dim3((unsigned)std::min<long>(tiles, kMaxBlocks256)), dim3(256), 0, s, p);
  } else if (cfg == FP4_ROWS) hipLaunchKernelGGL((fp4_rows_kernel<F32>), dim3((p.N + 15) / 16), dim3(512), 0, s, p);
  else if (cfg == FP4_16X32) launch_split<F32, 1, 2>(p, s);
  else if (cfg == FP4_32X32) launch_split<F32, 2, 2>(p, s);
  else if (cfg == FP4_64) launch_ring<F32, 64, 64, 2, 2, 2>(p, s);
  else launch_ring<F32, 128, 128, 2, 4, 1>(p, s);
}

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
  p.y = y;
  p.M = M;
  p.N = N;
  p.pitch = fp4_pitch(K);
  p.kt = p.pitch / 128;
  p.spitch = fp4_scale_pitch(K);
  const Fp4Cfg cfg = pick(M, N, K);
  if (out_dtype == DIT_F32) launch<true>(cfg, p, s);
  else launch<false>(cfg, p, s);
  return hipGetLastError();
}

}  // namespace dit
