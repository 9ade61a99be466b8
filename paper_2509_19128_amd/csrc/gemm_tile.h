// A tile of a matrix product on the matrix cores, for the kernels that own one: operands' way from memory, main loop, stores.
#pragma once
#include "pl_common.h"

namespace pl {
namespace {

constexpr int BK = 64;          // k elements per main-loop step
constexpr int STAGES = 4;       // k-steps held: one is multiplied while three are on their way
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
// Of sixteen lanes with 4 x 16 values (four lanes to a row of 32 bytes), lane i gets column i.  (__restrict__: a read of LDS of which the compiler knows
// nothing waits for every load on its way there; this one it takes for apart from them, as it does ordinary reads, whose waits are written out.)
__device__ __forceinline__ s16x4 read_transposed(lds_s16x4 *__restrict__ p) {
#ifdef __HIP_DEVICE_COMPILE__
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(p);
#else
  return s16x4{};
#endif
}
// Cache policy of the W loads: non-temporal (2) for weights that are COLD, that is, cannot be in the 256 MB last-level cache
// from the pass before, in tiles whose W one wavefront reads (WM = 1): they have no second reader, and ordinary loads
// evict each other from L2 on the way.  SwiGLU of the 32B shape, 128 rows: 111.8 -> 98.7 us (5.7 TB/s); 7B shape, 19 rows,
// whole step -4 %; products at 256 rows -1 % (the second row tile's reader still finds W in L2; not where that tile
// or one of more is short: launch_gemm, launch_gemm_folded).  Where two wavefronts
// share W through the caches (WM = 2; 1.5B shape, 64 rows) they cost 3.5 % of the step, and a matrix that stays in the
// last-level cache between calls 5 to 30 % (55 MB, 3 rows: 11 -> 16 us).
template <int WM, bool COLD>
constexpr int W_CACHE = WM == 1 && COLD ? 2 : 0;

// A tile of the product: a workgroup of 4 wavefronts arranged WM x WN, each of which owns (AT*32) x (BT*32) outputs.
// W fragments go from memory to a ring of register stages, x tiles by direct loads to a ring of LDS stages (no registers
// and no store instructions on the way), both three k-steps ahead of the products that use them; nothing waits for
// younger loads, as loads complete in order and each wait names the number that may stay in flight.  What bounds a k-step is the
// larger of its MFMA time and of its bytes at what one compute unit gets from the caches (about 100 KB/us from L2, 45
// from HBM): cycles per k-step of a lone workgroup with W in L2, and of its MFMAs alone, 256x256 2260 and 2048, 128x256 1100 and 1024,
// 128x128 790 and 512 (with x through registers, a double-buffered LDS tile and a full wait at each barrier: 128x256 1680).
// On the full chip with random operands the clock settles so that about 1.5 PFLOP/s are left at the margin (256x256 tiles, 1024 rows:
// 1.42 us per k-step, 1.01 with operands of zeros).
// Row r of an LDS stage holds its eight 16-byte chunks at slots chunk ^ (r & 7): a direct load fills a KiB in lane order, 8 whole rows,
// and the reads of a fragment (one chunk of 32 rows) meet every bank once.
// The products are taken with W as the first operand: a lane ends with one row and groups of four consecutive columns.
// Other kinds than TILE_ROWS: TILE_INT8, codes in 8 bits (a k-step is 128 of them: strides count pairs) and sums in int32;
// TILE_COLS, x as the first operand, so that a lane ends with one column of W and groups of four consecutive rows of x;
// TILE_COLS_T, the same with x k-major in memory (a row of it is one k): a k-step's 64 rows of BM lie in LDS as they come, and transposing reads
// bring a lane its four k of one column, two reads per fragment.  Row k has its 16-byte chunks at slots chunk ^ 4 (k & 3), so that the four
// k rows of a read lie in different banks; TILE_ROWS_T, W first again, with x an operand-ordered image taken across: the image's k are rows of x, its rows
// are k.  LDS holds, for each chunk of eight rows of x, 64 k of 16 bytes, number m at slot m ^ 4 (chunk & 3), read by transposing too.
enum { TILE_ROWS, TILE_INT8, TILE_COLS, TILE_COLS_T, TILE_ROWS_T };
// W_ROWS (TILE_COLS): W's rows too as they lie, wherever each is: few, and found again in the caches.
template <int WM, int WN, int AT, int BT, bool COLD, int KIND = TILE_ROWS, bool W_ROWS = false>
struct Tile {
  static constexpr int BM = WM * AT * 32, BN = WN * BT * 32;
  static constexpr int XI = BM / 32, XH = (XI + 1) / 2, WI = BT * 4;   // loads of a wavefront per k-step: x (half of them XH), W
  static constexpr int STAGE = BM * BK, LDS = STAGES * STAGE;          // elements
  static constexpr int X_CACHE = KIND == TILE_COLS && COLD ? 2 : 0;   // (weights are x there; non-temporal where nothing reads them again)
  // Offsets of x held per lane: one per load; of the kinds that address whole tiles, those that differ by more than a number of rows, which a scalar
  // adds (their kernels have no register to spare: a spill in the main loop waits for every load in flight).
  static constexpr int XL = KIND == TILE_ROWS ? XI : KIND == TILE_ROWS_T ? 4 : KIND == TILE_COLS_T && BM == 256 ? 2 : 1;
  static constexpr bool TURNED = KIND == TILE_COLS_T || KIND == TILE_ROWS_T;   // two reads of LDS per fragment
  static_assert(WM * WN == 4 && BT <= 2, "tile");

  // where a tile's operands are
  struct Part {
    int x_lane[XL];        // per lane: byte offset of its row and chunk (rows beyond M repeat the last one)
    int x_k;               // byte offset of the first k
    uint32_t w_blk[BT];    // byte offset of the first W block
  };
  // Operand-ordered W: block (k-step, n / 32) is 4096 bytes: [j][lane][16 B], lane = half * 32 + row.
  // Blocks are k-step-major: workgroups walk K in step, so at any moment the whole chip reads one
  // contiguous plane of W and the traffic spreads over every HBM channel (with row-block-major
  // order all streams sit a multiple of 8 blocks apart and camp on a fraction of the channels).
  __amdgpu_buffer_rsrc_t rw, rx;   // one resource per operand; what is uniform across a wavefront is in scalar registers
  uint32_t w_plane;
  int wave, wm, wn, l, lrow, half, a_off[4];
  int w_lane[BT];                  // W_ROWS: byte offset of the lane's row and half
  int x_step, x_load;              // bytes from a k-step of x to the next, and from a wavefront's load of 64 chunks to the next (other kinds than TILE_ROWS)
  bf16_t *xs;
  typedef std::conditional_t<KIND == TILE_INT8, i32x16, f32x16> Acc;
  Acc acc[AT][BT];
  bf16x8 wf[STAGES][BT][4], af[2][AT];

  __device__ __forceinline__ void init(bf16_t *xs_, const bf16_t *X, const bf16_t *W, int M, int N, int K) {
    xs = xs_;
    l = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    wm = wave / WN; wn = wave % WN;
    lrow = l & 31; half = l >> 5;
    w_plane = (uint32_t)(N >> 5) * 4096u;
    rw = __builtin_amdgcn_make_buffer_rsrc((void *)W, 0, (int)((int64_t)N * K * 2), 0x00020000);
    rx = __builtin_amdgcn_make_buffer_rsrc((void *)X, 0, (int)((int64_t)M * K * 2), 0x00020000);
#pragma unroll
    for (int j = 0; j < 4; ++j) a_off[j] = (wm * AT * 32 + lrow) * BK + ((half * 4 + j) ^ (lrow & 7)) * 8;
  }
  __device__ __forceinline__ Part part(int n_tile0, int m0, int ks0, int M, int N, int K) const {
    Part p;
#pragma unroll
    for (int i = 0; i < XI; ++i)
      p.x_lane[i] = (min(m0 + (wave * XI + i) * 8 + (l >> 3), M - 1) * K + ((l & 7) ^ (l >> 3)) * 8) * 2;
    p.x_k = ks0 * BK * 2;
#pragma unroll
    for (int b = 0; b < BT; ++b)
      p.w_blk[b] = (uint32_t)ks0 * w_plane + (uint32_t)min(((n_tile0 + wn * BT * 32) >> 5) + b, (N >> 5) - 1) * 4096u;
    return p;
  }
  // The same for the other kinds, which take their operands tile by tile, from pointers of their own.
  __device__ __forceinline__ void init_at(bf16_t *xs_) {
    xs = xs_;
    l = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    wm = wave / WN; wn = wave % WN;
    lrow = l & 31; half = l >> 5;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (KIND == TILE_COLS_T) {   // (j: block of 32 rows of x, modulo 4)
        const int s = l & 15, chunk = wm * AT * 4 + j * 4 + ((l >> 4) & 1) * 2 + ((s & 3) >> 1);
        a_off[j] = (half * 32 + (s >> 2)) * BM + (chunk ^ (4 * (s >> 2))) * 8 + (s & 1) * 4;
      } else if constexpr (KIND == TILE_ROWS_T) {   // (j: the k's bits 2 and 3)
        const int s = l & 15, chunk = wm * AT * 4 + ((l >> 4) & 1) * 2 + ((s & 3) >> 1);
        a_off[j] = (chunk * 64 + half * 32 + ((j * 4) ^ (4 * (chunk & 3))) + (s >> 2)) * 8 + (s & 1) * 4;
      } else {
        a_off[j] = (wm * AT * 32 + lrow) * BK + ((half * 4 + j) ^ (lrow & 7)) * 8;
      }
    }
  }
  // W_ROWS: the rows within `bytes` from W on; row b of the lane at element `at` (negative: none, zeros)
  __device__ __forceinline__ void rows_w(const bf16_t *W, int bytes) { rw = __builtin_amdgcn_make_buffer_rsrc((void *)W, 0, bytes, 0x00020000); }
  __device__ __forceinline__ void row_w(int b, int at) { w_lane[b] = at < 0 ? 0x7fff0000 : at * 2 + half * 64; }
  // (What lies beyond an operand reads as 0 by the check of its resource's size, which takes lane and scalar offset together, a scalar offset beyond the
  // size too: measured for sizes from 0 to 3 GiB, offsets up to 4, into registers and into LDS.)
  // x: rows (TILE_COLS_T: k) ldx elements apart from X on, of which `rows` exist (further ones read as 0); TILE_ROWS_T: an image of ldx rows, from the plane at
  // X on, of which `rows` planes of 64 exist;
  // w: operand-ordered, `n` of its rows per plane and `planes` k-steps from W on (further ones read as 0), the tile's from w_row on.
  __device__ __forceinline__ Part part_at(const bf16_t *X, int64_t ldx, int rows, const bf16_t *W, int n, int planes, int w_row) {
    Part p;
    w_plane = (uint32_t)(n >> 5) * 4096u;
    if (!W_ROWS) rw = __builtin_amdgcn_make_buffer_rsrc((void *)W, 0, (int)((uint32_t)planes * w_plane), 0x00020000);
    const int64_t x_bytes = (int64_t)rows * ldx * (KIND == TILE_ROWS_T ? 128 : 2);
    rx = __builtin_amdgcn_make_buffer_rsrc((void *)X, 0, (int)(uint32_t)min(x_bytes, (int64_t)1 << 31), 0x00020000);
    constexpr int PER = KIND == TILE_COLS_T ? BM / 8 : BK / 8, ROWS = 64 / PER;   // chunks of a row (of 64 k or of BM columns), rows of a load
    static_assert(KIND != TILE_COLS_T || ROWS * XL == 4, "the slots of a row go by its number modulo 4");
    static_assert(KIND != TILE_ROWS_T || XI == 8, "a wavefront loads a plane's part of a k-step");
    x_step = KIND == TILE_COLS_T ? (int)(BK * 2 * ldx) : KIND == TILE_ROWS_T ? 2 * 4096 : BK * 2;
    x_load = KIND == TILE_ROWS_T ? (int)(ldx * 128) : (int)(ROWS * 2 * ldx);   // (TILE_ROWS_T: from a plane to the next)
#pragma unroll
    for (int i = 0; i < XL; ++i) {
      if constexpr (KIND == TILE_ROWS_T) {
        const int m = l ^ (4 * i);
        p.x_lane[i] = (m >> 5) * 4096 + (m & 31) * 16;
        continue;
      }
      const int k = l / PER;
      p.x_lane[i] = (int)(k * ldx * 2) + ((l % PER) ^ (KIND == TILE_COLS_T ? 4 * ((i * ROWS + k) & 3) : l / PER)) * 16;
    }
    p.x_k = 0;
#pragma unroll
    for (int b = 0; b < BT; ++b) p.w_blk[b] = (uint32_t)min(((w_row + wn * BT * 32) >> 5) + b, (n >> 5) - 1) * 4096u;
    return p;
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int a = 0; a < AT; ++a)
#pragma unroll
      for (int b = 0; b < BT; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[a][b][i] = 0;
  }
  __device__ __forceinline__ void load_x(const Part &p, int st, int ks, int i0, int i1) {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
    for (int i = i0; i < i1; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, (lds_void *)(xs + st * STAGE + (wave * XI + i) * 512), 16, p.x_lane[i % XL],
                                               KIND == TILE_ROWS     ? p.x_k + ks * (BK * 2)
                                               : KIND == TILE_ROWS_T ? ks * x_step + wave * x_load + (i & 3) * 1024 + (i >> 2) * 512
                                                                     : ks * x_step + (wave * XI + i) * x_load,
                                               0, X_CACHE);
#endif
  }
  __device__ __forceinline__ void load_w(const Part &p, int st, int ks, int b) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      wf[st][b][j] = __builtin_bit_cast(
          bf16x8, W_ROWS ? __builtin_amdgcn_raw_buffer_load_b128(rw, w_lane[b] + j * 16, ks * (BK * 2), 0)
                         : __builtin_amdgcn_raw_buffer_load_b128(rw, l * 16 + j * 1024, (int)(p.w_blk[b] + (uint32_t)ks * w_plane), W_CACHE<WM, COLD>));
  }
  __device__ __forceinline__ void load(const Part &p, int st, int ks) {
    load_x(p, st, ks, 0, XI);
#pragma unroll
    for (int b = 0; b < BT; ++b) load_w(p, st, ks, b);
  }
  __device__ __forceinline__ void read_a(int st, int j) {
#pragma unroll
    for (int a = 0; a < AT; ++a) {
      if constexpr (TURNED) {
#ifdef __HIP_DEVICE_COMPILE__
        bf16_t *at = xs + st * STAGE, *at_lo, *at_hi;
        if constexpr (KIND == TILE_COLS_T) {
          at_lo = at + a_off[a & 3] + (a >> 2) * 128 + j * 8 * BM;
          at_hi = at_lo + 4 * BM;
        } else {
          at_lo = at + a_off[(j & 1) * 2] + (j >> 1) * 128 + a * 2048;
          at_hi = at + a_off[(j & 1) * 2 + 1] + (j >> 1) * 128 + a * 2048;
        }
        const s16x4 lo = read_transposed((lds_s16x4 *)at_lo), hi = read_transposed((lds_s16x4 *)at_hi);
        af[j & 1][a] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#endif
      } else {
        af[j & 1][a] = *(const bf16x8 *)(xs + st * STAGE + a_off[j] + a * 32 * BK);
      }
    }
  }
  __device__ __forceinline__ void mma(int st, int j) {
#pragma unroll
    for (int a = 0; a < AT; ++a)
#pragma unroll
      for (int b = 0; b < BT; ++b)
#ifdef __HIP_DEVICE_COMPILE__
        if constexpr (KIND == TILE_INT8)
          acc[a][b] = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, wf[st][b][j]), __builtin_bit_cast(i32x4, af[j & 1][a]), acc[a][b], 0, 0, 0);
        else if constexpr (KIND == TILE_ROWS || KIND == TILE_ROWS_T)
          acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf[st][b][j], af[j & 1][a], acc[a][b], 0, 0, 0);
        else
          acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af[j & 1][a], wf[st][b][j], acc[a][b], 0, 0, 0);
#else
        ;
#endif
  }
  // all but the LEFT youngest loads have arrived, and this wavefront has its operands out of LDS; then the others too
  template <int LEFT>
  __device__ __forceinline__ void meet() {
#ifdef __HIP_DEVICE_COMPILE__
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"i"(LEFT) : "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
#endif
  }
  // no load is on its way to LDS any more
  __device__ __forceinline__ void drain() {
#ifdef __HIP_DEVICE_COMPILE__
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#endif
  }
  // Results for kernels that compute with them: one register at a time, from where the matrix cores have them.  (As ordinary operands whole accumulators are
  // copied, which pushes other registers out to memory.)  `settle` first: the wait states that a read behind the last product needs.
  __device__ __forceinline__ void settle() const {
#ifdef __HIP_DEVICE_COMPILE__
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
#endif
  }
  __device__ __forceinline__ auto result(int a, int b, int i) const {
    std::conditional_t<KIND == TILE_INT8, int32_t, float> v = 0;
#ifdef __HIP_DEVICE_COMPILE__
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(acc[a][b][i]));
#endif
    return v;
  }
  // Issue order of a quarter of a k-step: LDS reads (for the next quarter) and VM loads one by one between the products.
  template <int VM, bool READS>
  __device__ __forceinline__ void order() {
    constexpr int per = VM >= AT ? VM / AT : 1;
#pragma unroll
    for (int i = 0; i < AT; ++i) {
      if (READS) __builtin_amdgcn_sched_group_barrier(0x100, TURNED ? 2 : 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, BT, 0);
      if (VM >= AT || i * VM / AT != (i + 1) * VM / AT) __builtin_amdgcn_sched_group_barrier(0x020, per, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  // First three k-steps of a part into stages 0 .. 2, and the first operands out of LDS.
  __device__ __forceinline__ void begin(const Part &p) {
#pragma unroll
    for (int st = 0; st < STAGES - 1; ++st) load(p, st, st);
    meet<2 * (XI + WI) + WI>();
    read_a(0, 0);
  }
  // One k-step in stage U (k-step index mod 4).  LOAD: k-step ks of part p goes to the stage that the last one freed.
  // AFTER: k-steps that follow (3: three or more), whose loads stay in flight while the next stage is waited for.
  // The operands of the last quarter are read before that wait, those of the next k-step's first quarter behind it, so that the matrix
  // pipeline has a quarter's products to work on meanwhile.
  template <int U, bool LOAD, int AFTER>
  __device__ __forceinline__ void kstep(const Part &p, int ks) {
    constexpr int TO = (U + 3) & 3;
    read_a(U, 1);
    if (LOAD) load_x(p, TO, ks, 0, XH);
    mma(U, 0);
    order<LOAD ? XH : 0, true>();
    read_a(U, 2);
    if (LOAD) load_x(p, TO, ks, XH, XI);
    mma(U, 1);
    order<LOAD ? XI - XH : 0, true>();
    read_a(U, 3);
    if (LOAD) load_w(p, TO, ks, 0);
    mma(U, 2);
    order<LOAD ? 4 : 0, true>();
    if (AFTER > 0) {
      meet<AFTER == 1 ? WI : AFTER == 2 ? XI + 2 * WI : 2 * (XI + WI) + 4>();
      read_a((U + 1) & 3, 0);
    }
    if (LOAD && BT > 1) load_w(p, TO, ks, BT - 1);
    mma(U, 3);
    if (AFTER > 0) {
#pragma unroll
      for (int i = 0; i < AT; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, BT, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, TURNED ? 2 : 1, 0);
        if (LOAD && BT > 1 && (4 >= AT || i * 4 / AT != (i + 1) * 4 / AT)) __builtin_amdgcn_sched_group_barrier(0x020, 4 >= AT ? 4 / AT : 1, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  // k-steps ks .. ks + 3 of a part of more than ks + 7, and its last four
  __device__ __forceinline__ void four(const Part &p, int ks) {
    kstep<0, true, 3>(p, ks + 3);
    kstep<1, true, 3>(p, ks + 4);
    kstep<2, true, 3>(p, ks + 5);
    kstep<3, true, 3>(p, ks + 6);
  }
  __device__ __forceinline__ void last_four(const Part &p, int ks) {
    kstep<0, true, 3>(p, ks + 3);
    kstep<1, false, 2>(p, 0);
    kstep<2, false, 1>(p, 0);
    kstep<3, false, 0>(p, 0);
  }
  // accumulator register i of lane l is column (i / 4) * 8 + (l / 32) * 4 + i % 4, row l % 32
  // a 32 x 32 block so that the four lanes of a quad hold 64 bytes of a row: v[t] is row (l % 32 & ~3) + t, columns l / 32 * 16 + l % 4 * 4 on
  static __device__ __forceinline__ void by_rows(f32x4 (&v)[4], const f32x16 &c) {
#ifdef __HIP_DEVICE_COMPILE__
    const int odd = threadIdx.x & 1, high = threadIdx.x >> 1 & 1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
      auto halves = [&](float x, float y, uint32_t &a, uint32_t &b) {   // lanes 32 .. 63 of x against 0 .. 31 of y
        const u32x2 r = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false));
        a = r[0]; b = r[1];
      };
      uint32_t q[4];   // 16 columns of a row, in groups of four
      halves(c[e], c[8 + e], q[0], q[1]);
      halves(c[4 + e], c[12 + e], q[2], q[3]);
      // each lane reads its neighbour's registers before it chooses (a choice between reads would be a branch that leaves the neighbour out)
      uint32_t x[4], y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)q[k ^ 1], 0xB1, 0xf, 0xf, true);   // quad_perm 1 0 3 2
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = odd != (k & 1) ? x[k] : q[k];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)y[k ^ 2], 0x4E, 0xf, 0xf, true);   // quad_perm 2 3 0 1
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k][e] = __uint_as_float(high != (k >> 1) ? x[k] : y[k]);
    }
#endif
  }
  // fp32 sums: row stride ldy, columns counted from y_col0, columns below n_end (a multiple of 32).
  // Stores of 64 bytes of a row instead of 32 (a lane's own columns): LM head of the 7B shape, 256 rows, 322 -> 306 us, 7B QKV 22.6 -> 20.9,
  // 32B QKV, 128 rows, 22.3 -> 21.4.  Up to 64 rows the exchange costs more than it saves (1.5B QKV, 64 rows, 4.8 -> 5.0; a step of the tiny
  // shape 3 %).
  __device__ __forceinline__ void store(float *Y, int n_tile0, int m0, int M, int n_end, int64_t ldy, int y_col0) const {
    const int n0 = n_tile0 + wn * BT * 32;
#pragma unroll
    for (int a = 0; a < AT; ++a) {
      const int m = m0 + (wm * AT + a) * 32;
      if (m >= M) continue;
#pragma unroll
      for (int b = 0; b < BT; ++b) {
        if (n0 + b * 32 >= n_end) continue;
        if (M <= 64) {
          float *y = Y + (m + lrow) * ldy + (n0 + b * 32 + half * 4 - y_col0);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (m + lrow < M) *(f32x4 *)(y + i * 8) = f32x4{acc[a][b][4 * i], acc[a][b][4 * i + 1], acc[a][b][4 * i + 2], acc[a][b][4 * i + 3]};
          continue;
        }
        f32x4 v[4];
        by_rows(v, acc[a][b]);
        float *y = Y + (m + (lrow & ~3)) * ldy + (n0 + b * 32 + half * 16 + (lrow & 3) * 4 - y_col0);
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (m + (lrow & ~3) + t < M) *(f32x4 *)(y + t * ldy) = v[t];
#ifdef __HIP_DEVICE_COMPILE__
        __builtin_amdgcn_sched_barrier(0);   // (one block's registers at a time)
#endif
      }
    }
  }
  // SwiGLU of a 64-row block's gate and up halves: the two column tiles of a wavefront, or (BT = 1) the tiles of two
  // neighbours, which swap half of them through the LDS stages that nothing reads any more and take half of the block each.
  __device__ __forceinline__ void store_swiglu(bf16_t *Y, int n_tile0, int m0, int M, int n_end, int N) {
    static_assert(BT == 2 || WM == 1, "pairs");
    constexpr int NI = BT == 2 ? 4 : 2;   // groups of four columns per lane
    const int n0 = BT == 2 ? n_tile0 + wn * 64 : n_tile0 + (wn >> 1) * 64, i0 = BT == 2 ? 0 : (wn & 1) * 2;
    f32x4 *swap = (f32x4 *)xs + l;        // [wavefront][a][2][lane]: two stages at most, and the last k-step reads the fourth
    if (BT == 1) {
#pragma unroll
      for (int a = 0; a < AT; ++a)
#pragma unroll
        for (int i = 0; i < 2; ++i) {   // an even wavefront (gate) hands on its groups 2 and 3, an odd one (up) 0 and 1
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = wn & 1 ? acc[a][0][4 * i + e] : acc[a][0][4 * (i + 2) + e];
          swap[((wn * AT + a) * 2 + i) * 64] = v;
        }
      __syncthreads();
    }
    if (n0 >= n_end) return;
#pragma unroll
    for (int a = 0; a < AT; ++a) {
      const int m = m0 + (wm * AT + a) * 32 + lrow;
      bf16_t *y = Y + (int64_t)m * (N / 2) + (n0 >> 1) + half * 4;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        f32x4 gte, up;
        if (BT == 2) {
#pragma unroll
          for (int e = 0; e < 4; ++e) { gte[e] = acc[a][0][4 * i + e]; up[e] = acc[a][BT - 1][4 * i + e]; }
        } else {
          const f32x4 other = swap[(((wn ^ 1) * AT + a) * 2 + i) * 64];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float mine = wn & 1 ? acc[a][0][4 * (i + 2) + e] : acc[a][0][4 * i + e];
            gte[e] = wn & 1 ? other[e] : mine;
            up[e] = wn & 1 ? mine : other[e];
          }
        }
        bf16x4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = swiglu(gte[e], up[e]);
        if (m < M) *(bf16x4 *)(y + (i0 + i) * 8) = o;
      }
    }
  }
};

// A tile of a product: operands as Tile::part_at has them, its k-steps (a multiple of four), and where its results go.
struct Item {
  const bf16_t *x, *w;
  int64_t ldx;
  int x_rows, w_n, w_planes, w_row, ksteps;
  int kind, row0, col0;   // of the kernel's own
};

template <typename T>
__device__ __forceinline__ typename T::Part part_of(T &t, const Item &i) { return t.part_at(i.x, i.ldx, i.x_rows, i.w, i.w_n, i.w_planes, i.w_row); }

// One tile with the whole workgroup.
template <typename T>
__device__ __forceinline__ void one_tile(T &t, const Item &c) {
  const auto p = part_of(t, c);
  t.zero();
  t.begin(p);
  int ks = 0;
  for (; ks < c.ksteps - 4; ks += 4) t.four(p, ks);
  t.last_four(p, ks);
}

// Tiles one after the other, the next one's first k-steps under the last products of the one at hand.  take(item): the next tile, or false; a tile is
// known one tile ahead; ask() is called as a tile begins and told() near its end, with barriers between it and the take() behind it.  One loop of four k-steps for all of a tile: with last k-steps
// of their own, behind the loop, the accumulators move between the two, and what spills meanwhile waits for every load in flight.
template <typename T, typename Ask, typename Told, typename Take, typename Done>
__device__ __forceinline__ void walk(T &t, Ask ask, Told told, Take take, Done done) {
  Item c, d;
  if (!take(c)) return;
  d = c;   // behind the last tile: its own first k-steps again, which nothing reads
  bool more = take(d);
  auto p = part_of(t, c);
  t.zero();
  t.begin(p);
  ask();
  for (;;) {
    for (int ks = 0; ks >= 0;) {
      t.template kstep<0, true, 3>(p, ks + 3);
      ks += 4;
      int at = ks;
      if (ks >= c.ksteps) {
        p = part_of(t, d);
        at = 0;
        ks = -1;
        told();
      }
      t.template kstep<1, true, 3>(p, at);
      t.template kstep<2, true, 3>(p, at + 1);
      t.template kstep<3, true, 3>(p, at + 2);
    }
    // what `done` computes from the lane alone is not to be held in registers through the k-steps
    asm volatile("" : "+v"(t.lrow), "+v"(t.half));
    t.settle();
    done(c);
    if (!more) break;
    t.zero();
    c = d;
    more = take(d);
    ask();
  }
  t.drain();
}

// two registers of four consecutive results each (bf16) against those of the other half of the wavefront: eight consecutive ones
__device__ __forceinline__ uint4 eight(const uint32_t (&a)[2], const uint32_t (&b)[2]) {
#ifdef __HIP_DEVICE_COMPILE__
  typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
  const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false));
  const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false));
  return make_uint4(lo[0], hi[0], lo[1], hi[1]);
#else
  return uint4{};
#endif
}
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}
}  // namespace
}  // namespace pl
