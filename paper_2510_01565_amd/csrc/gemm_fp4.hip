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
// The products of a block are exact, as is the sum of 8 of them; both outputs take
// the same sums.
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
// c += w x of 64 elements, the scales in byte B of their words.  A volatile statement: as a builtin the compiler moves it
// out of its turn between two barriers.  It does not see what the statement is: nothing may write an operand by vector
// arithmetic, nor read c, within the instruction's wait states.
template <int B>
__device__ __forceinline__ void asm_mfma(f32x16_t& c, const i32x4_t& w, const i32x4_t& x, int sw, int sx) {
  static_assert(B >= 0 && B < 4, "scale byte");
  if constexpr (B == 0)
    asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                 : "+v"(c) : "v"(w), "v"(x), "v"(sw), "v"(sx));
  else if constexpr (B == 1)
    asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                 : "+v"(c) : "v"(w), "v"(x), "v"(sw), "v"(sx));
  else if constexpr (B == 2)
    asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[0,0,0] op_sel_hi:[1,1,0] cbsz:4 blgp:4"
                 : "+v"(c) : "v"(w), "v"(x), "v"(sw), "v"(sx));
  else
    asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[1,1,0] op_sel_hi:[1,1,0] cbsz:4 blgp:4"
                 : "+v"(c) : "v"(w), "v"(x), "v"(sw), "v"(sx));
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

// ---------------------------------------------------------------- 256 x 256 tiles
constexpr int kMaxBlocks256 = 256;  // one per CU
constexpr int kMinKTiles256 = 3;    // its loads run up to three K tiles ahead, into the next output tile at most

// 8 waves, each 128 rows x 64 columns, by 32x32x64 matrix instructions.  K tiles of 128
// bytes (256 elements) move by direct-to-LDS loads into two stages.  Two wave groups
// (waves 0-3 and 4-7, one wave of each per SIMD) take turns: while one issues a cluster
// of 8 MFMAs, the other reads the fragments of its next cluster from LDS and issues its
// share of the loads; block barriers hold the groups one turn apart.  A K tile is 4
// clusters: cluster c multiplies the wave's c-th 32 rows of X with all its 64 rows of W
// (2 fragments of 4 steps each, held for a whole tile, two tiles in turn).  Read phase 4
// kt + c takes the X of the next cluster, 4 kt + c + 1, and of W of tile kt + 1 fragment
// c / 2, steps 2 (c % 2) and the next; every wave has their data ahead of the first
// barrier of its next phase, which the other group meets a turn later.  So a place is
// loaded again two phases after its last read: X's part c of tile kt + 2 in phase 4 kt +
// c + 1; W's parts 0 and 1, which hold fragment 0, of tile kt + 3 in phase 4 kt + 3, its
// parts 2 and 3, fragment 1, in phase 4 kt + 5.  X is read 6 phases after its load, W 5:
// loads have 4 phases until the wait that makes them visible.
// A block works through its output tiles as one stream of K tiles: the loads of the next
// output tile run ahead of the last K tiles of this one, and each cluster's finished sums
// are written in its read phase of the next tile's first K tile, beside the other group's
// MFMAs.  W's rows are dealt out to the fragments so that a lane holds 32 neighbouring
// columns of a row: it writes them straight from registers.
template <bool F32>
__global__ __launch_bounds__(512) void fp4_256_kernel(const Fp4Problem p) {
  constexpr int BM = 256, BN = 256, Q = 4, NS = F32 ? 8 : 4;  // NS: stores of a phase
  constexpr int ROWB = 128, CPR = 8, RPI = 8;  // bytes and 16-byte chunks of a row, rows per wave load
  constexpr int STAGE = BM * ROWB, SUB = STAGE / Q, REGION = 2 * STAGE;
  static_assert(BM == BN, "one stage size");
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
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wv >> 2, wn = wv & 3;
  // K tiles, and those of an output tile: an even number, the last one of zeros where K has an odd number
  const int KT = p.kt, Kp = p.pitch, KE = (KT + 1) & ~1;
  const int my_tiles = (tile_end - tile_next + tile_step - 1) / tile_step;

  // LDS slot of chunk c of row r: 16 consecutive rows' chunks lie in 16 different 16-byte bank groups
  auto swz = [](int row, int c) { return c ^ ((row >> 1) & 7); };
  // byte offsets of this lane's row of a part; the part and the K tile travel in the scalar offset, which the
  // range check counts.  X's part c: rows 32 c .. of either wave row.  W's part c: fragment c / 2 of wave columns 2 (c % 2)
  // and the next, row i of it being column 32 (i / 4 % 2) + 16 (c / 2) + 4 (i / 8) + i % 4 of its wave's 64.
  const int lrow = wv * RPI + lane / CPR, lc = swz(lrow, lane % CPR) * 16;
  const int gx = (int)((uint32_t)(lrow / 32 * 128 + lrow % 32) * (uint32_t)Kp + lc);
  const int gw = (int)((uint32_t)(lrow / 32 * 64 + (lrow >> 2 & 1) * 32 + (lrow % 32 >> 3) * 4 + lrow % 4) * (uint32_t)Kp + lc);
  const int gs = (wv % 4 * 64 + lane) * p.spitch;
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
  // (locals, not expressions, as the builtins' arguments: the host pass drops the kernel's launch stub otherwise)
  auto load_x = [&](auto stc, auto cc) __attribute__((always_inline)) {  // part c
    constexpr int st = decltype(stc)::value, c = decltype(cc)::value;
    const int vo = gx, so = xk * ROWB + c * 32 * Kp;
    const __amdgpu_buffer_rsrc_t r = rows(p.x, xm, xk < KT ? BM : 0, p.M, Kp);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        r, (__attribute__((address_space(3))) void*)(lbase + st * STAGE + c * SUB + wv * RPI * ROWB), 16, vo, so, 0, 0);
  };
  auto load_w = [&](auto stc, auto cc) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value, c = decltype(cc)::value;
    const int vo = gw, so = wk * ROWB + ((c & 1) * 128 + (c >> 1) * 16) * Kp;
    const __amdgpu_buffer_rsrc_t r = rows(p.w, wn0, wk < KT ? BN : 0, p.N, Kp);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        r, (__attribute__((address_space(3))) void*)(lbase + REGION + st * STAGE + c * SUB + wv * RPI * ROWB), 16, vo, so, 0, 0);
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
  // The scales of two K tiles, 512 elements, arrive together: X's rows by waves 0-3, W's by waves 4-7, a row per lane.
  auto load_scales = [&](int stage, int m, int n, int k) __attribute__((always_inline)) {
    const int vo = gs, so = k * 8;
    const __amdgpu_buffer_rsrc_t r = wv < 4 ? rows(p.xs, m, BM, p.M, p.spitch) : rows(p.ws, n, BN, p.N, p.spitch);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(
        r, (__attribute__((address_space(3))) void*)(lbase + SCALES + stage * SCALE_STAGE + wv * 1024), 16, vo, so, 0, 0);
  };
  // the tile's bias, one value per word, 64 of them by each of four waves (and again by the others); zeros past N
  auto load_bias = [&](int stage) __attribute__((always_inline)) {
    const int q = wv & 3, es = p.bias_f32 ? 4 : 2, n = p.bias ? max(p.N - n0, 0) * es : 0, vo = (q * 64 + lane) * es;
    const __amdgpu_buffer_rsrc_t r = buffer((const uint8_t*)p.bias + (long)n0 * es, n);
    __attribute__((address_space(3))) void* const to =
        (__attribute__((address_space(3))) void*)(lbase + BIAS + stage * BIAS_STAGE + q * 256);
    if (p.bias_f32) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 4, vo, 0, 0, 0);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 2, vo, 0, 0, 0);
  };

  // ---- fragment reads: row lane % 32 of a 32-row fragment, at step s chunk 2 s + lane / 32
  const int half = lane >> 5;
  const int xr = wm * 32 + (lane & 31), wr = (wn & 1) * 32 + (lane & 31);
  const int xa = xr * ROWB + swz(xr, half) * 16, wa = REGION + (wn >> 1) * SUB + wr * ROWB + swz(wr, half) * 16;
  // Whole-value casts: read member by member, the compiler takes them to alias the loads in flight and waits for those.
  auto lds16 = [&](int at) __attribute__((always_inline)) {
    return __builtin_bit_cast(i32x4_t, *(const uint4*)(lbase + at));
  };
  auto lds4 = [&](int at) __attribute__((always_inline)) {
    return __builtin_bit_cast(int, *(const Word*)(lbase + at));
  };
  const int xs0 = SCALES + (wm * 128 + (lane & 31)) * 16 + half * 4;
  const int ws0 = SCALES + 4096 + (wn * 64 + (lane >> 2 & 1) * 32 + (lane >> 3 & 3) * 4 + (lane & 3)) * 16 + half * 4;
  f32x16_t acc[Q][2];
#pragma unroll
  for (int i = 0; i < Q; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x16_t{};
  // X fragments of a cluster and its scale words (clusters in turn), W fragments of a K tile (K tiles in turn) and the scale
  // words of two K tiles
  i32x4_t fx[2][4], fw[2][2][4];
  int sx[2][2], sw[2][2];
  // reads part c of X of a K tile in `st` into the cluster's registers
  auto read_x = [&](auto stc, auto cc, int stage) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value, c = decltype(cc)::value;
    const int a = opaque(xa), xsa = opaque(xs0 + stage * SCALE_STAGE);
#pragma unroll
    for (int s = 0; s < 4; ++s) fx[c & 1][s] = lds16((a ^ (s * 32)) + st * STAGE + c * SUB);
#pragma unroll
    for (int h = 0; h < 2; ++h) sx[c & 1][h] = lds4(xsa + c * 32 * 16 + h * 8);
  };
  // reads fragment c / 2 of W of a K tile in `st`, steps 2 (c % 2) and the next
  auto read_w = [&](auto stc, auto cc) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value, c = decltype(cc)::value, j = c >> 1, s0 = (c & 1) * 2;
    const int a = opaque(wa);
#pragma unroll
    for (int s = s0; s < s0 + 2; ++s) fw[st][j][s] = lds16((a ^ (s * 32)) + st * STAGE + j * 2 * SUB);
  };
  // reads W's scale words of two K tiles, in the phase whose MFMAs are the first to take them: the last ones' still took
  // the words before
  auto read_sw = [&](int stage) __attribute__((always_inline)) {
    const int wsa = opaque(ws0 + stage * SCALE_STAGE);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h) sw[j][h] = lds4(wsa + j * 16 * 16 + h * 8);
  };

  // ---- writes the finished sums of cluster c of the tile at (m0, n0), whose bias is in `stage`
  const int ncol = wn * 64 + half * 32, mrow = wm * 128 + (lane & 31);
  constexpr int ES = F32 ? 4 : 2;
  const uint32_t pitch = (uint32_t)p.N * ES;
  const int bias_shift = p.bias_f32 ? 0 : 16;
  auto store = [&](auto cc, int m0, int n0, int stage) __attribute__((always_inline)) {
    constexpr int c = decltype(cc)::value;
    const int at = opaque(ncol) * 4 + BIAS + stage * BIAS_STAGE;
    // opaque: what depends on the lane alone is formed here again rather than held in registers over the K loop
    const int mr = opaque(mrow), n = p.N - n0 - opaque(ncol);  // n: columns left from this lane's first
    const uint32_t yo = (uint32_t)mr * pitch + (uint32_t)(p.N - n0 - n) * ES;
    char* const y = (char*)p.y + ((long)m0 * p.N + n0) * ES + (long)(c * 32) * pitch + yo;
    const bool row = mr < p.M - m0 - c * 32;
    auto columns = [&](int q, float* v) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        const i32x4_t b = lds16(at + (q * 8 + e) * 4);
#pragma unroll
        for (int r = 0; r < 4; ++r)
          v[e + r] = acc[c][q >> 1][(q & 1) * 8 + e + r] + __uint_as_float((uint32_t)b[r] << bias_shift);
      }
    };
    if (!row) return;
    float v[8];
    if (n >= 32) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        columns(q, v);
        store_columns<F32, 8>(y + q * 8 * ES, v, 8);
      }
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        columns(q, v);
        store_columns<F32, 8>(y + q * 8 * ES, v, n - q * 8);
      }
    }
  };

  using S0 = std::integral_constant<int, 0>;
  using S1 = std::integral_constant<int, 1>;
  int prev_m0 = p.M, prev_n0 = 0, scale_stage = 0, bias_stage = 0;  // no row of the tile before the first exists
  bool counted = false;
  // STORE 1: the output tile's first K tile, which writes the previous tile's sums; 2: the one after it
  auto phase = [&](auto stc, auto cc, auto storec) __attribute__((always_inline)) {
    constexpr int st = decltype(stc)::value, c = decltype(cc)::value;
    constexpr int STORE = decltype(storec)::value;
    using CN = std::integral_constant<int, (c + 1) % Q>;
    using SN = std::integral_constant<int, c + 1 < Q ? st : st ^ 1>;  // stage of the next cluster
    using CX = std::integral_constant<int, (c + Q - 1) % Q>;
    using SX = std::integral_constant<int, c == 0 ? st ^ 1 : st>;
    using SW = std::integral_constant<int, c < 2 ? st : st ^ 1>;
    if constexpr (STORE == 1) {
      store(cc, prev_m0, prev_n0, bias_stage ^ 1);
      // zeroed here, ahead of the barrier; as a value the compiler holds 16 registers of zeros for it
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float z;
          asm volatile("v_mov_b32 %0, 0" : "=v"(z));
          acc[c][j][i] = z;
        }
    }
    // the last phase's reads, this cluster's operands among them: complete ahead of the barrier, behind which (the next
    // phase on) their places are loaded again
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
    // the next cluster's X, behind the last one of two K tiles with the next scales; W of the next K tile
    if constexpr (c == 0 && st == 0) read_sw(scale_stage);
    read_x(SN{}, CN{}, c + 1 == Q && st == 1 ? scale_stage ^ 1 : scale_stage);
    read_w(std::integral_constant<int, st ^ 1>{}, cc);
    // the last part of X's K tile kt + 1, or a part of kt + 2; W's parts 2 and 3 of kt + 2, or 0 and 1 of kt + 3
    load_x(SX{}, CX{});
    if constexpr (c == 0) next_xk();
    if constexpr (c == 1) {
      load_w(SW{}, std::integral_constant<int, 2>{});
      load_w(SW{}, std::integral_constant<int, 3>{});
      next_wk();
    }
    if constexpr (c == 3) {
      load_w(SW{}, S0{});
      load_w(SW{}, S1{});
    }
    // All but the loads of the last 4 phases have landed.  Those phases' stores need not have: NS in each phase of the
    // first K tile, if all of the tile's rows and columns exist.
    if (STORE && counted) wait_vmcnt<8 + (STORE == 1 ? NS * (c + 1) : STORE == 2 ? NS * (3 - c) : 0)>();
    else wait_vmcnt<8>();
    block_barrier();
    static_for<4>([&](auto sc) {
      constexpr int s = decltype(sc)::value;
#pragma unroll
      for (int j = 0; j < 2; ++j)
        asm_mfma<st * 2 + s / 2>(acc[c][j], fw[st][j][s], fx[c & 1][s], sw[j][s & 1], sx[c & 1][s & 1]);
    });
    block_barrier();
  };
  // K tiles kt and kt + 1, whose scales came as one; the next ones' have 4 phases or more.
  auto k_pair = [&](auto firstc, int kt) __attribute__((always_inline)) {
    constexpr int FIRST = decltype(firstc)::value;
    const bool on = kt + 2 >= KE;
    load_scales(scale_stage ^ 1, on ? m0_next : m0, on ? n0_next : n0, on ? 0 : kt + 2);
    static_for<Q>([&](auto cc) { phase(S0{}, cc, std::integral_constant<int, FIRST ? 1 : 0>{}); });
    static_for<Q>([&](auto cc) { phase(S1{}, cc, std::integral_constant<int, FIRST ? 2 : 0>{}); });
    scale_stage ^= 1;
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
  static_for<Q>([&](auto cc) { read_w(S0{}, cc); });
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0)
  block_barrier();
  static_for<Q - 1>([&](auto cc) {
    load_x(S1{}, cc);
    if constexpr (decltype(cc)::value > 0) load_w(S0{}, std::integral_constant<int, decltype(cc)::value - 1>{});
  });
  wait_vmcnt<8>();  // what phase 0 reads has landed: X's first two parts, W's first two of tile 1 and the scales
  block_barrier();
  read_x(S0{}, S0{}, 0);
  if (wv >= 4) block_barrier();
#pragma unroll 1
  for (int t = 0; t < my_tiles; ++t) {
    load_bias(bias_stage);
    tile_next += tile_step;
    if (tile_next < tile_end) tile_at(tile_next, m0_next, n0_next);
    counted = prev_m0 + BM <= p.M && prev_n0 + BN <= p.N;  // NS stores a phase by every wave
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
  for (int i = 0; i < Q; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) asm volatile("" : "+v"(acc[i][j]));
  static_for<Q>([&](auto cc) { store(cc, prev_m0, prev_n0, bias_stage ^ 1); });
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
// the groups' sums meet in LDS at the end, in their order.  As in the kernel
// above a lane holds 4 FN neighbouring columns of each of its rows.
template <bool F32, int BM, int BN, int WM, int WN, int KG, int ST>
__global__ __launch_bounds__(WM* WN* KG * 64) void fp4_ring_kernel(const Fp4Problem p) {
  constexpr int NW = WM * WN * KG, FM = BM / WM / 16, FN = BN / WN / 16;
  constexpr int ROWB = 128, UNITS = KG * (BM + BN) / 8, LPW = UNITS / NW;  // loads of 8 rows; per wave and step
  constexpr int SU = (BM + BN) / 64;  // loads of 64 rows' scales, by as many waves
  constexpr int TILE = (BM + BN) * ROWB, SCALES = KG * TILE, STAGE = SCALES + (BM + BN) * 16;
  static_assert(LPW * NW == UNITS && BM % 64 == 0 && BN % 64 == 0 && SU <= NW && KG <= 2, "tile config");
  static_assert(ST * STAGE <= 160 * 1024 && (KG - 1) * WM * WN * FM * FN * 1024 <= ST * STAGE, "LDS");
  __shared__ uint4 lds[ST * STAGE / 16];
  char* const lbase = (char*)lds;
  const int tn = (p.N + BN - 1) / BN, tm = (p.M + BM - 1) / BM;
  const int id = (int)(blockIdx.y << kRingRowLog2) + xcd_remap(blockIdx.x, gridDim.x);
  if (id >= tm * tn) return;
  int im, in;
  tile_of(id, tm, tn, im, in);
  const int m0 = im * BM, n0 = in * BN, KT = p.kt, Kp = p.pitch, steps = (KT + KG - 1) / KG;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), kg = wv / (WM * WN), wm = wv / WN % WM, wn = wv % WN;
  auto swz = [](int row, int c) { return c ^ ((row >> 1) & 7); };
  // row of X or of W that lies in row `row` of a tile: X's as they come, W's dealt out to the fragments
  auto source = [](int row) {
    if (row < BM) return row;
    constexpr int C = BN / WN;
    const int w = row - BM, in_wave = w % C, f = in_wave & 15;
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
// arrive by direct-to-LDS loads in two stages of each wave's own, their scales in
// registers.  As above W's rows are dealt out to the fragments, and a lane ends with 4
// FN neighbouring columns of a row.
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
  tile_of(id, tm, tn, im, in);
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
// each.  Their sums meet in LDS in wave order.
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

// Which kernel a product takes: the one whose modelled time is least.
enum Fp4Cfg { FP4_ROWS, FP4_16X32, FP4_32X32, FP4_32X64, FP4_64, FP4_128, FP4_256, FP4_CFGS };
static Fp4Cfg pick(int M, int N, int K, int out_dtype) {
  const double kt = fp4_pitch(K) / 128;
#ifdef FP4_FORCE
  if (const char* e = getenv("FP4_CFG")) {
    const int c = atoi(e);
    if ((c != FP4_ROWS || M <= 16) && (c != FP4_256 || kt >= kMinKTiles256)) return (Fp4Cfg)c;
  }
#endif
  if (M <= 16 && N * kt * 128 <= 1 << 25) return FP4_ROWS;
  auto rounds = [&](int bm, int bn) { return ceil(ceil((double)M / bm) * ceil((double)N / bn) / 256.0); };
  auto ring = [&](int b, double c, double pair, double pair_kt, double odd, double odd_kt) {
    const double n = rounds(b, b);
    return c + floor(n / 2) * (pair + pair_kt * kt) + (n - 2 * floor(n / 2)) * (odd + odd_kt * kt);
  };
  Fp4Cfg cfg = FP4_64;
  double best = rounds(64, 64) <= 1 ? 3.5 + 0.235 * kt : ring(64, 2.5, 1.9, 0.385, 0.3, 0.33);
  auto offer = [&](Fp4Cfg c, double us) {
    if (us < best) {
      best = us;
      cfg = c;
    }
  };
  const double memory = 2.9 + N * kt * 128 / 7e6;
  offer(FP4_16X32, fmax(2.9 + rounds(16, 32) * (0.7 + 0.06 * kt), memory));
  offer(FP4_32X32, fmax(2.9 + rounds(32, 32) * (1.15 + 0.083 * kt), memory));
  offer(FP4_32X64, fmax(1.7 + rounds(32, 64) * (3.2 + 0.145 * kt), memory));
  offer(FP4_128, rounds(128, 128) <= 1 ? 4.75 + 0.547 * kt : ring(128, 3.1, 3.65, 0.866, 0.0, 0.7));
  // offsets within a tile of 256 output rows fit 32 bits up to 2^21 columns
  if (kt >= kMinKTiles256 && N <= 1 << 21)
    offer(FP4_256, rounds(256, 256) <= 1 ? 13.5 + 1.02 * kt : rounds(256, 256) * (7.0 + 1.45 * kt));
  return cfg;
}

const char* gemm_fp4_config_name(int M, int N, int K, int out_dtype) {
  static const char* names[] = {"gemm_fp4_rows", "gemm_fp4_16x32", "gemm_fp4_32x32", "gemm_fp4_32x64", "gemm_fp4_64x64", "gemm_fp4_128x128", "gemm_fp4_256x256"};
  return names[pick(M, N, K, out_dtype)];
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
    hipLaunchKernelGGL(fp4_256_kernel<F32>, dim3((unsigned)std::min<long>(tiles, kMaxBlocks256)), dim3(512), 0, s, p);
  } else if (cfg == FP4_ROWS) hipLaunchKernelGGL((fp4_rows_kernel<F32>), dim3((p.N + 15) / 16), dim3(512), 0, s, p);
  else if (cfg == FP4_16X32) launch_split<F32, 1, 2>(p, s);
  else if (cfg == FP4_32X32) launch_split<F32, 2, 2>(p, s);
  else if (cfg == FP4_32X64) launch_split<F32, 2, 4>(p, s);
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
  const Fp4Cfg cfg = pick(M, N, K, out_dtype);
  if (out_dtype == DIT_F32) launch<true>(cfg, p, s);
  else launch<false>(cfg, p, s);
  return hipGetLastError();
}

}  // namespace dit
