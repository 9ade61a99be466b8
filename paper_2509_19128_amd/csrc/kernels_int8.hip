// Products in 8-bit integers: y = x W^T with a scale per row of x (token) and per row of W (channel).
//
// Quantisation of a row: scale = max |x| / 127 in fp32, code = the integer nearest to x / scale (ties to even), at most 127 in magnitude.  The
// quotient is rounded as if exact: the product is then the same for every implementation of that sentence.  Codes are multiplied and added up
// in int32 without error (127^2 K < 2^31), in any order and any number of slices, and a result is (float(sum) * scale of its token) * scale of
// its channel.
//
// The product is gemm_tile.h's, but for few rows (gemm_int8_few_kernel, gemm_int8_narrow_kernel): W's codes in operand order straight to the registers of the first operand, x's through LDS.  Bytes per k-step and cycles
// of a matrix instruction are those of the bf16 product at twice the k, so a byte of weights does twice the work in both bounds.
#include "gemm_tile.h"

#include <algorithm>

namespace pl {
namespace {

constexpr int DPP_ROR2 = 0x122;
constexpr int K_UNIT = 512;   // codes of four k-steps: rows of x are padded with zeros to a multiple, W reads as zeros there
constexpr int UNITS = 256;

// The integer nearest to x / s (ties to even; clamped): the rounded quotient may be one off next to a tie, and its remainder says so.  x - q s is
// exact: a multiple of the last place of s (of x where x is the smaller) and no larger than 2 s.
__device__ inline int quotient(float x, float s, float inv) {
  float q = fminf(fmaxf(rintf(x * inv), -127.f), 127.f);
  const float r = fmaf(-q, s, x), h = 0.5f * s;
  if (r > h || (r == h && ((int)q & 1))) q += 1.f;
  if (r < -h || (r == -h && ((int)q & 1))) q -= 1.f;
  return (int)fminf(fmaxf(q, -127.f), 127.f);
}
// What the codes of a row need, from its largest magnitude (infinity: a number that is none): the scale, and the factors of quotient().  Tiny rows: both
// sides of the quotient times a power of two, so that 1 / s is finite; they, zeros and rows that hold no numbers take the long way.
struct RowScale {
  float scale, s, inv, up;
  bool plain;
  __device__ inline explicit RowScale(float most) {
    const bool fine = most < INFINITY;
    scale = fine ? most / 127.f : NAN;
    plain = scale >= 0x1p-100f;
    up = plain ? 1.f : 0x1p100f;
    s = fine ? scale * up : 0.f;
    inv = s > 0.f ? 1.f / s : 0.f;
  }
  // The codes of four values, a byte each.  x / s + 1.5 2^23 in one rounding has the code in its last byte; where a remainder is half of s or more
  // the quotient was rounded next to a tie, and the careful one decides.
  __device__ __forceinline__ uint32_t four(float x0, float x1, float x2, float x3) const {
    constexpr float MAGIC = 12582912.f;
    const float t0 = fmaf(x0, inv, MAGIC), t1 = fmaf(x1, inv, MAGIC), t2 = fmaf(x2, inv, MAGIC), t3 = fmaf(x3, inv, MAGIC);
    const float r0 = fmaf(MAGIC - t0, s, x0), r1 = fmaf(MAGIC - t1, s, x1), r2 = fmaf(MAGIC - t2, s, x2), r3 = fmaf(MAGIC - t3, s, x3);
    const float r = fmaxf(fmaxf(fabsf(r0), fabsf(r1)), fmaxf(fabsf(r2), fabsf(r3)));
    if (plain && r < 0.5f * s) {
      const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(t1), __float_as_uint(t0), 0x0c0c0400u), hi = __builtin_amdgcn_perm(__float_as_uint(t3), __float_as_uint(t2), 0x0c0c0400u);
      return hi << 16 | lo;
    }
    if (!(inv > 0.f)) return 0;
    return ((uint32_t)quotient(x0 * up, s, inv) & 255u) | ((uint32_t)quotient(x1 * up, s, inv) & 255u) << 8 | ((uint32_t)quotient(x2 * up, s, inv) & 255u) << 16 |
           (uint32_t)quotient(x3 * up, s, inv) << 24;
  }
};
// COUNT consecutive values of a row
template <typename T, int COUNT>
struct Values {
  static constexpr int VECTORS = COUNT * sizeof(T) / 16;
  uint4 raw[VECTORS];
  __device__ __forceinline__ void load(const T *p) {
#pragma unroll
    for (int i = 0; i < VECTORS; ++i) raw[i] = ((const uint4 *)p)[i];
  }
  __device__ __forceinline__ float get(int i) const {
    constexpr int PER = 16 / sizeof(T);
    const uint4 u = raw[i / PER];
    const int w = i % PER * sizeof(T) / 4;
    const uint32_t d = w == 0 ? u.x : w == 1 ? u.y : w == 2 ? u.z : u.w;
    if constexpr (sizeof(T) == 4) return __uint_as_float(d);
    else return __uint_as_float(i & 1 ? d & 0xffff0000u : d << 16);
  }
  // The largest magnitude as an unsigned number, which orders bit patterns without sign as their values are, infinities and NaN last: one or two
  // instructions a value.  (bf16: two side by side.)
  struct Most {
    typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
    std::conditional_t<sizeof(T) == 4, uint32_t, u16x2> m{};
    __device__ __forceinline__ float value() const {   // infinity stands for NaN too
      uint32_t bits;
      if constexpr (sizeof(T) == 4) bits = m;
      else bits = (uint32_t)max(m[0], m[1]) << 16;
      return bits < 0x7f800000u ? __uint_as_float(bits) : INFINITY;
    }
  };
  __device__ __forceinline__ void most(Most &m) const {
#pragma unroll
    for (int i = 0; i < VECTORS * 4; ++i) {
      const uint4 u = raw[i / 4];
      const uint32_t d = i % 4 == 0 ? u.x : i % 4 == 1 ? u.y : i % 4 == 2 ? u.z : u.w;
      if constexpr (sizeof(T) == 4) m.m = max(m.m, d & 0x7fffffffu);
      else m.m = __builtin_elementwise_max(m.m, __builtin_bit_cast(typename Most::u16x2, d & 0x7fff7fffu));
    }
  }
  __device__ __forceinline__ void codes(const RowScale &r, uint32_t (&q)[COUNT / 4]) const {
#pragma unroll
    for (int w = 0; w < COUNT / 4; ++w) q[w] = r.four(get(w * 4), get(w * 4 + 1), get(w * 4 + 2), get(w * 4 + 3));
  }
};

// Codes of weights in operand order.  ROWS rows per workgroup: a 128-byte line of the image holds the same sixteen k of eight rows, and workgroups that share
// lines are on one XCD.  A lane keeps its values between the two passes where they fit into HELD pieces of sixteen.
template <typename T, int HELD, int ROWS>
__global__ __launch_bounds__(1024) void quantize_weights_kernel(const T *__restrict__ w, int64_t ldw, uint4 *__restrict__ q, float *__restrict__ scale, int N, int K) {
  const int r = threadIdx.x & (ROWS - 1), lanes = blockDim.x / ROWS, first = threadIdx.x / ROWS, pieces = K >> 4;
  int block = blockIdx.x;
  if constexpr (ROWS < 8) {   // (gridDim.x is a multiple of 8: N of 32)
    const int each = gridDim.x >> 3;
    block = (block & 7) * each + (block >> 3);
  }
  const int row = block * ROWS + r;
  w += row * ldw;
  Values<T, 16> held[HELD ? HELD : 1];
  typename Values<T, 16>::Most most;
  if constexpr (HELD > 0) {
#pragma unroll
    for (int u = 0; u < HELD; ++u)
      if (first + u * lanes < pieces) held[u].load(w + (first + u * lanes) * 16);
#pragma unroll
    for (int u = 0; u < HELD; ++u)
      if (first + u * lanes < pieces) held[u].most(most);
  } else {
    for (int p = first; p < pieces; p += lanes) {
      held[0].load(w + p * 16);
      held[0].most(most);
    }
  }
  __shared__ float part[16][ROWS];
  float m = most.value();
  if constexpr (ROWS < 4) m = fmaxf(m, dpp<DPP_ROR2>(m));
  if constexpr (ROWS < 8) m = fmaxf(m, dpp<DPP_ROR4>(m));
  m = fmaxf(m, dpp<DPP_ROR8>(m));
  m = with_xor16(m, OpMax{});
  m = with_xor32(m, OpMax{});
  if ((threadIdx.x & 63) < ROWS) part[threadIdx.x >> 6][r] = m;
  __syncthreads();
  for (int i = 0; i < (int)blockDim.x >> 6; ++i) m = fmaxf(m, part[i][r]);
  const RowScale rs(m);
  if (first == 0) scale[row] = rs.scale;
  auto store = [&](int p, const Values<T, 16> &v) {   // piece p is (k / 16): block p / 8, half (p / 4) % 2, quarter p % 4
    uint32_t c[4];
    v.codes(rs, c);
    q[(((int64_t)(p >> 3) * (N >> 5) + (row >> 5)) * 4 + (p & 3)) * 64 + ((p >> 2) & 1) * 32 + (row & 31)] = make_uint4(c[0], c[1], c[2], c[3]);
  };
  if constexpr (HELD > 0) {
#pragma unroll
    for (int u = 0; u < HELD; ++u)
      if (first + u * lanes < pieces) store(first + u * lanes, held[u]);
  } else {
    for (int p = first; p < pieces; p += lanes) {
      held[0].load(w + p * 16);
      store(p, held[0]);
    }
  }
}

// Codes of x, row-major, rows padded with zeros to k_pad, or (ORDERED) in operand order, `blocks` blocks of 32 rows.  A workgroup per row, eight values of a
// lane at a time.
// ROW_HELD: pieces that a lane holds between its two looks (1 / 2 / 4: products of 3001 rows of 2560 x 32768 436 / 423 / 412 us).
constexpr int ROW_HELD = 4;
template <bool ORDERED>
__global__ __launch_bounds__(1024) void quantize_rows_kernel(const bf16_t *__restrict__ x, int64_t ldx, uint2 *__restrict__ q, float *__restrict__ scale, int K, int k_pad, int blocks) {
  x += blockIdx.x * ldx;
  q += ORDERED ? (int64_t)(blockIdx.x >> 5) * 512 + (blockIdx.x & 31) * 2 : (int64_t)blockIdx.x * (k_pad >> 3);
  const int pieces = K >> 3, all = k_pad >> 3;
  Values<bf16_t, 8> v[ROW_HELD];
  Values<bf16_t, 8>::Most most;
#pragma unroll
  for (int u = 0; u < ROW_HELD; ++u)
    if (threadIdx.x + u * blockDim.x < pieces) v[u].load(x + (threadIdx.x + u * blockDim.x) * 8);
#pragma unroll
  for (int u = 0; u < ROW_HELD; ++u)
    if (threadIdx.x + u * blockDim.x < pieces) v[u].most(most);
  for (int p = threadIdx.x + ROW_HELD * blockDim.x; p < pieces; p += blockDim.x) {
    Values<bf16_t, 8> more;
    more.load(x + p * 8);
    more.most(most);
  }
  __shared__ float part[16];
  float m = wave_max(most.value());
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  for (int i = 0; i < (int)blockDim.x >> 6; ++i) m = fmaxf(m, part[i]);
  const RowScale rs(m);
  if (threadIdx.x == 0) scale[blockIdx.x] = rs.scale;
  auto store = [&](int p, const Values<bf16_t, 8> &from) {
    uint32_t c[2] = {0, 0};
    if (p < pieces) from.codes(rs, c);
    // (in order: eight codes of block p / 16, quarter p / 2 % 4, half p / 8 % 2)
    q[ORDERED ? (int64_t)(p >> 4) * blocks * 512 + ((p >> 1) & 3) * 128 + ((p >> 3) & 1) * 64 + (p & 1) : p] = make_uint2(c[0], c[1]);
  };
#pragma unroll
  for (int u = 0; u < ROW_HELD; ++u)
    if (threadIdx.x + u * blockDim.x < all) store(threadIdx.x + u * blockDim.x, v[u]);
  for (int p = threadIdx.x + ROW_HELD * blockDim.x; p < all; p += blockDim.x) {
    Values<bf16_t, 8> again;
    if (p < pieces) again.load(x + p * 8);
    store(p, again);
  }
}

struct Int8Params {
  const int8_t *xq, *wq;
  const float *sx, *sw;
  void *y;               // fp32 or bf16 [M][N], or int32 [splits][M][N]
  int M, N, K, k_pad, splits, slice;   // slice: k-steps of a K slice, a multiple of four
  int ncol, nrow;        // tiles
};
enum { OUT_F32, OUT_BF16, OUT_SLICES };

template <typename T>
__device__ __forceinline__ Item int8_item(const Int8Params &g, int rtile, int ctile, int split) {
  Item c;
  const int k0 = split * g.slice;
  c.kind = split; c.row0 = rtile * T::BM; c.col0 = ctile * T::BN;
  c.x = (const bf16_t *)(g.xq + (int64_t)c.row0 * g.k_pad + k0 * 128); c.ldx = g.k_pad >> 1; c.x_rows = min(g.M - c.row0, T::BM);
  c.w = (const bf16_t *)(g.wq + (int64_t)k0 * g.N * 128); c.w_n = g.N; c.w_planes = g.K / 128 - k0; c.w_row = c.col0;
  c.ksteps = min(g.slice, g.k_pad / 128 - k0);
  return c;
}

// results of a tile: a lane has one row and groups of four consecutive columns
template <int OUT, typename T, int WM, int WN, int AT, int BT>
__device__ __forceinline__ void int8_store(const T &t, const Int8Params &g, const Item &c) {
#pragma unroll
  for (int b = 0; b < BT; ++b) {
    const int n = c.col0 + (t.wn * BT + b) * 32;
    if (n >= g.N) continue;   // (uniform)
    f32x4 sw[4];
    if constexpr (OUT != OUT_SLICES) {
#pragma unroll
      for (int i = 0; i < 4; ++i) sw[i] = *(const f32x4 *)(g.sw + n + i * 8 + t.half * 4);
    }
#pragma unroll
    for (int a = 0; a < AT; ++a) {
      const int m = c.row0 + (t.wm * AT + a) * 32 + t.lrow;
      int32_t v[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if constexpr (AT * BT > 8) v[i] = t.result(a, b, i);
        else v[i] = t.acc[a][b][i];
      }
      const int64_t at = (int64_t)m * g.N + n;
      if constexpr (OUT == OUT_SLICES) {
        int32_t *y = (int32_t *)g.y + (int64_t)c.kind * g.M * g.N + at + t.half * 4;
        if (m < g.M) {
#pragma unroll
          for (int i = 0; i < 4; ++i) *(i32x4 *)(y + i * 8) = i32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
        }
      } else {
        const float sx = g.sx[min(m, g.M - 1)];
        f32x4 r[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) r[i][e] = (float)v[4 * i + e] * sx * sw[i][e];
        if constexpr (OUT == OUT_F32) {
          float *y = (float *)g.y + at + t.half * 4;
          if (m < g.M) {
#pragma unroll
            for (int i = 0; i < 4; ++i) *(f32x4 *)(y + i * 8) = r[i];
          }
        } else {
          bf16_t *y = (bf16_t *)g.y + at + t.half * 8;
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const uint32_t lo[2] = {two_bf16(r[2 * p][0], r[2 * p][1]), two_bf16(r[2 * p][2], r[2 * p][3])};
            const uint32_t hi[2] = {two_bf16(r[2 * p + 1][0], r[2 * p + 1][1]), two_bf16(r[2 * p + 1][2], r[2 * p + 1][3])};
            const uint4 o = eight(lo, hi);
            if (m < g.M) *(uint4 *)(y + p * 16) = o;
          }
        }
      }
#ifdef __HIP_DEVICE_COMPILE__
      __builtin_amdgcn_sched_barrier(0);   // (one block's registers at a time)
#endif
    }
  }
}

// A tile per workgroup; the row tiles of a column tile and slice sit 8 ids apart, so that they run on one XCD at the same time and share W's way there.
template <int WM, int WN, int AT, int BT, int OUT, bool COLD>
__global__ __launch_bounds__(256) void gemm_int8_kernel(Int8Params g) {
  typedef Tile<WM, WN, AT, BT, COLD, TILE_INT8> T;
  __shared__ __attribute__((aligned(1024))) bf16_t xs[T::LDS];
  const int item = (blockIdx.x / (8 * g.nrow)) * 8 + (blockIdx.x & 7), rtile = (blockIdx.x >> 3) % g.nrow;
  if (item >= g.ncol * g.splits) return;
  T t;
  t.init_at(xs);
  const Item c = int8_item<T>(g, rtile, item % g.ncol, item / g.ncol);
  one_tile(t, c);
  t.settle();
  int8_store<OUT, T, WM, WN, AT, BT>(t, g, c);
}

// 256 x 256 tiles one after the other, a workgroup per compute unit: XCD i walks the i-th eighth of them, column tile by column tile.
template <int OUT>
__global__ __launch_bounds__(256) void gemm_int8_rounds_kernel(Int8Params g) {
  typedef Tile<1, 4, 8, 2, false, TILE_INT8> T;
  __shared__ __attribute__((aligned(1024))) bf16_t xs[T::LDS];
  const int tiles = g.nrow * g.ncol, xcd = blockIdx.x & 7;
  int at = xcd * (tiles >> 3) + min(xcd, tiles & 7);
  const int end = at + (tiles >> 3) + (xcd < (tiles & 7) ? 1 : 0);
  at += blockIdx.x >> 3;
  T t;
  t.init_at(xs);
  walk(t, [] {}, [] {}, [&](Item &d) {
    if (at >= end) return false;
    d = int8_item<T>(g, at % g.nrow, at / g.nrow, 0);
    at += gridDim.x >> 3;
    return true;
  }, [&](const Item &c) { int8_store<OUT, T, 1, 4, 8, 2>(t, g, c); });
}

// K slices added up (exactly, whatever the order) and scaled, four columns per thread
template <typename T>
__global__ __launch_bounds__(256) void int8_slices_kernel(const i32x4 *__restrict__ parts, const float *__restrict__ sx, const float *__restrict__ sw, T *__restrict__ y, int splits,
                                                          int M, int N) {
  const int n = (blockIdx.x * 256 + threadIdx.x) * 4, m = blockIdx.y;
  if (n >= N) return;
  const i32x4 *p = parts + ((int64_t)m * N + n) / 4;
  i32x4 sum = {0, 0, 0, 0};
#pragma unroll 8
  for (int s = 0; s < splits; ++s) sum += p[(int64_t)s * M * (N / 4)];
  const float a = sx[m];
  const f32x4 b = *(const f32x4 *)(sw + n);
  f32x4 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = (float)sum[e] * a * b[e];
  if constexpr (sizeof(T) == 4) *(f32x4 *)(y + (int64_t)m * N + n) = r;
  else *(uint2 *)(y + (int64_t)m * N + n) = make_uint2(two_bf16(r[0], r[1]), two_bf16(r[2], r[3]));
}

// Few rows in one launch: a workgroup quantises them for itself into LDS, under its first loads of W, and walks blocks of 32 channels.  Its eight wavefronts
// take turns of 1 KiB of a block of W (32 channels x 2 x 16 k in operand order: one operand of a matrix instruction, straight from memory), the other
// operand comes from the codes in LDS; at a block's end their sums are added up in LDS.  Nothing but W's way from memory is left to bound it.
// ROWS (1, 2, 4): 8 / ROWS wavefronts quantise a row.
constexpr int FEW_AHEAD = 8;    // turns of a wavefront whose loads are in flight
constexpr int FEW_HELD = 8;     // pieces of eight values that a lane holds of a row between its two looks
template <int ROWS, typename T>
__global__ __launch_bounds__(512) void gemm_int8_few_kernel(const bf16_t *__restrict__ x, int64_t ldx, const int8_t *__restrict__ wq, const float *__restrict__ sw, T *__restrict__ y,
                                                            int M, int N, int K) {
  extern __shared__ __attribute__((aligned(16))) int8_t few_lds[];
  // scales and maxima, sums of the wavefronts [8][16][64], codes [M][K + 16] (16 bytes more per row: consecutive rows begin in other banks; 2 KB behind
  // the last row are read against zeros)
  float *scale = (float *)few_lds, *part = scale + 8;
  int32_t *sums = (int32_t *)(few_lds + 256);
  int8_t *codes = few_lds + 256 + 8 * 4096;
  const int l = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), turns = K >> 8, pitch = K + 16, blocks = N >> 5;
  // The turns of a wavefront, block after block, as one sequence: of each block a multiple of FEW_AHEAD, those behind K reading as zeros (2 GiB on,
  // behind the end of any W).  A turn's registers are filled for the turn FEW_AHEAD on as soon as it is done.
  const int turns_pad = (turns + FEW_AHEAD - 1) / FEW_AHEAD * FEW_AHEAD, step = N * 256;   // (bytes: 256 k on)
  const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc((void *)wq, 0, (int)((int64_t)N * K), 0x00020000);
  const int first = __builtin_amdgcn_readfirstlane((wave >> 2) * N * 128 + (wave & 3) * 1024);
  auto load = [&](int block, int t) {
    return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, t < turns ? l * 16 : INT32_MIN, t < turns ? first + block * 4096 + t * step : 0, 2));
  };
  i32x4 cur[FEW_AHEAD];
#pragma unroll
  for (int u = 0; u < FEW_AHEAD; ++u) cur[u] = load(blockIdx.x, u);

  {
    constexpr int WAVES = 8 / ROWS, LANES = 64 * WAVES;
    const int row = wave / WAVES, at = threadIdx.x & (LANES - 1), pieces = K >> 3;   // (a row beyond M: the last one again, into no one's place)
    const bf16_t *mine = x + min(row, M - 1) * ldx;
    Values<bf16_t, 8> v[FEW_HELD];
    Values<bf16_t, 8>::Most most;
#pragma unroll
    for (int u = 0; u < FEW_HELD; ++u)
      if (at + u * LANES < pieces) v[u].load(mine + (at + u * LANES) * 8);
#pragma unroll
    for (int u = 0; u < FEW_HELD; ++u)
      if (at + u * LANES < pieces) v[u].most(most);
    float m = wave_max(most.value());
    if (l == 0) part[wave] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) m = fmaxf(m, part[row * WAVES + i]);
    const RowScale rs(m);
    if (at == 0 && row < M) scale[row] = rs.scale;
#pragma unroll
    for (int u = 0; u < FEW_HELD; ++u)
      if (at + u * LANES < pieces && row < M) {
        uint32_t c[2];
        v[u].codes(rs, c);
        *(uint2 *)(codes + row * pitch + (at + u * LANES) * 8) = make_uint2(c[0], c[1]);
      }
    __syncthreads();
  }

  [[maybe_unused]] const int8_t *mine = codes + min(l & 31, M - 1) * pitch + (wave >> 2) * 128 + (l >> 5) * 64 + (wave & 3) * 16;
  for (int block = blockIdx.x; block < blocks; block += gridDim.x) {
    i32x16 sum;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] = 0;
    for (int t0 = 0; t0 < turns_pad; t0 += FEW_AHEAD) {
      const bool last = t0 + FEW_AHEAD == turns_pad;
      const int block_on = last ? min(block + (int)gridDim.x, blocks - 1) : block, t_on = last ? 0 : t0 + FEW_AHEAD;   // (behind the last block: any)
#pragma unroll
      for (int u = 0; u < FEW_AHEAD; ++u) {
#ifdef __HIP_DEVICE_COMPILE__
        sum = __builtin_amdgcn_mfma_i32_32x32x32_i8(cur[u], *(const i32x4 *)(mine + (t0 + u) * 256), sum, 0, 0, 0);
#endif
        cur[u] = load(block_on, t_on + u);
      }
    }
    // sums of a wavefront: register i of lane l is channel (i / 4) * 8 + (l / 32) * 4 + i % 4, row l % 32
    if ((l & 31) < ROWS) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sums[(wave * 16 + i) * 64 + l] = sum[i];
    }
    __syncthreads();
    if (threadIdx.x < 32 * ROWS) {
      const int r = threadIdx.x & (ROWS - 1), c = threadIdx.x / ROWS, i = (c >> 3) * 4 + (c & 3), n = block * 32 + c;   // (c: channel)
      int32_t s = 0;
#pragma unroll
      for (int w = 0; w < 8; ++w) s += sums[(w * 16 + i) * 64 + ((c >> 2) & 1) * 32 + r];
      if (r < M) y[(int64_t)r * N + n] = (T)((float)s * scale[r] * sw[n]);
    }
    __syncthreads();
  }
}

// Narrow outputs of few rows: a workgroup takes 16 channels over all of K, its eight wavefronts turns of 64 k (1 KiB of W, in four pieces) with the same k of
// x's codes, in operand order too, straight from memory; at the end their sums are added up in LDS.  No slices that a launch behind would add up.
// BLOCKS: of 16 rows.
template <int BLOCKS, bool COLD, typename T>
__global__ __launch_bounds__(512) void gemm_int8_narrow_kernel(const int8_t *__restrict__ xq, const int8_t *__restrict__ wq, const float *__restrict__ sx, const float *__restrict__ sw,
                                                               T *__restrict__ y, int M, int N, int K) {
  constexpr int AHEAD = BLOCKS > 1 ? 2 : 4, PAIRS = (BLOCKS + 1) / 2;   // (turns in flight per wavefront; 8: 1536 x 1536, 8 rows, 5.7 -> 6.6 us)
  __shared__ i32x4 sums[8][BLOCKS][64];
  const int l = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), planes = K >> 7, n0 = blockIdx.x * 16;
  const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc((void *)wq, 0, (int)((int64_t)N * K), 0x00020000);
  const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void *)xq, 0, PAIRS * 32 * K, 0x00020000);
  // a lane's sixteen k: quarter l / 16 of the half that its wavefront has of a plane of 128 (both operands' alike, so that which k these are is no matter)
  const int lane = (l >> 4) * 1024 + (l & 15) * 16, w_first = (n0 >> 5) * 4096 + (wave & 1) * 512 + ((n0 >> 4) & 1) * 256;
  i32x4 w[AHEAD], x[AHEAD][BLOCKS], sum[BLOCKS];
  auto load = [&](int u, int t) {   // (planes behind K: zeros, from 2 GiB on)
    const int plane = t * 4 + (wave >> 1), at = plane < planes ? lane : INT32_MIN;
    w[u] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rw, at, plane < planes ? w_first + plane * N * 128 : 0, COLD ? 2 : 0));
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
      x[u][b] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, at, plane < planes ? (plane * PAIRS + b / 2) * 4096 + (wave & 1) * 512 + (b & 1) * 256 : 0, 0));
  };
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) load(u, u);
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) sum[b] = i32x4{0, 0, 0, 0};
  for (int t = 0; t * 4 < planes; t += AHEAD)
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b) sum[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u], x[u][b], sum[b], 0, 0, 0);
#endif
      load(u, t + u + AHEAD);
    }
  // register i of lane l: channel l / 16 * 4 + i, row l % 16
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) sums[wave][b][l] = sum[b];
  __syncthreads();
  if (wave >= BLOCKS) return;
  i32x4 s = {0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < 8; ++k) s += sums[k][wave][l];
  const int m = wave * 16 + (l & 15), n = n0 + (l >> 4) * 4;
  if (m >= M) return;
  const float a = sx[m];
  f32x4 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = (float)s[e] * a * sw[n + e];
  T *to = y + (int64_t)m * N + n;
  if constexpr (sizeof(T) == 4) *(f32x4 *)to = r;
  else *(uint2 *)to = make_uint2(two_bf16(r[0], r[1]), two_bf16(r[2], r[3]));
}

int done() { return hipGetLastError() == hipSuccess ? 0 : -7; }
int64_t align256(int64_t b) { return (b + 255) / 256 * 256; }

// How a product is cut: tile shape and K slices.  Microseconds as measured: fixed + k-steps of a slice * (base + load * (fraction of the units at work) +
// more * (average beyond one workgroup per unit) + round * (workgroups of the fullest unit - 1)), out per MB of bf16 results, and with slices their
// launch and MB of sums.  Fitted to 2700 launches (the products of the 1.5B, 7B and 32B shapes and smaller ones, 1 to 3001 rows, 1 to 24 slices, weights
// not in the last-level cache): the choice takes 1.2 % more than the best measured one on average, 6 % in 95 of 100.
enum { I8_32x128, I8_64x128, I8_128x128, I8_128x256, I8_64x64, I8_ROUNDS, I8_FEW, I8_NARROW };
struct ShapeTime { int rows, cols; float fixed, base, load, more, round, slices, slice_mb, out_mb; };
constexpr ShapeTime SHAPES[] = {{32, 128, 5.29f, 0.275f, 0.137f, 0.128f, 0.217f, 4.46f, 0.203f, 0.f},   {64, 128, 5.88f, 0.324f, 0.197f, 0.155f, 0.25f, 3.67f, 0.371f, 0.f},
                                {128, 128, 7.75f, 0.359f, 0.289f, 0.278f, 0.313f, 2.88f, 0.386f, 0.098f}, {128, 256, 8.39f, 0.625f, 0.623f, 0.419f, 0.707f, 2.75f, 0.337f, 0.067f},
                                {64, 64, 5.53f, 0.21f, 0.117f, 0.123f, 0.17f, 2.6f, 0.434f, 0.f},          {256, 256, 21.f, 0.98f, 0.393f, 0.407f, 1.258f, 0.f, 0.f, 0.377f}};
struct Int8Plan { int shape, splits, slice; };
constexpr int K_SLICES_MOST = 24, SLICED_TILES_MOST = 600;   // (the latter: tiles times slices)
// gemm_int8_few_kernel, where a workgroup holds its rows in registers while it looks for their largest magnitudes: fixed (less 2 for the launches that the
// caller's thread does not make), the quantisation, and a workgroup's part of W at what a unit gets, or all of W.  us, measured so / in two launches: 1 row 3584 x 3584 7.5 / 10.4, 37888 x 3584 22.9 / 28.8 (so, on other cards, 20.6 and 21.3), 1536 x 8960
// 12.3 / 11.1, 5120 x 27648 26.6 / 29.0; 4 rows 3584 x 3584 9.4 / 10.7, 37888 x 3584 23.5 / 29.0; 8 rows (a wavefront each) 16.2 / 11.2 and 29.1 / 30.4.
int few_rows(int M) { return M > 2 ? 4 : M; }
bool few_fits(int M, int K) { return M <= 4 && few_rows(M) * K <= 512 * FEW_HELD * 8; }
float few_us(int M, int N, int K) {
  const float rounds = (N / 32 + 2 * UNITS - 1) / (2 * UNITS);
  return std::max(2.8f + 1.5e-4f * few_rows(M) * K + rounds * K * (32 / 45e3f), 1.f + (float)N * K * (1 / 6.4e6f));
}
// gemm_int8_narrow_kernel, a workgroup per unit at most.  us on the device, with slices or 64 x 64 tiles / so, weights from memory: 8 rows 1536 x 3584 10.6 / 7.5,
// 4096 x 3584 12.2 / 8.6, 4096 x 7168 14.8 / 12.1; 64 rows 2560 x 2560 11.6 / 9.5, 4096 x 5120 15.4 / 13.6, 2560 x 7168 16.1 / 16.3; in the cache: 8 rows
// 1536 x 8960 10.0 / 11.0, 4608 x 3584 (two on a unit) 9.8 / 9.9, 19 rows 10.4 / 11.4.
int row_blocks(int M) { return (M + 31) / 32; }
float narrow_us(int M, int N, int K) {
  if (M > 64 || N > 16 * UNITS) return 1e30f;
  return 3.7f + K * (0.5e-3f + 0.25e-3f * ((M + 15) / 16)) + 5e-8f * N * K;
}
Int8Plan int8_plan(int M, int N, int K) {
  const int groups = (K + K_UNIT - 1) / K_UNIT;
  const float mb = 1e-6f * M * N, few = few_fits(M, K) ? few_us(M, N, K) : 1e30f;
  Int8Plan best{-1, 1, 0};
  if (few < 8) return Int8Plan{I8_FEW, 1, 0};   // (two launches take no less)
  float best_us = 0;
  for (int shape = 0; shape <= I8_ROUNDS; ++shape) {
    const ShapeTime &f = SHAPES[shape];
    // tiles of mostly absent rows, and so many small ones that their W is read over and over, were not measured
    if ((f.rows > 64 && f.rows >= 4 * M) || (shape != I8_ROUNDS && (int64_t)f.rows * 24 < M)) continue;
    const int64_t tiles = (int64_t)((M + f.rows - 1) / f.rows) * ((N + f.cols - 1) / f.cols);
    for (int sp : {1, 2, 3, 4, 5, 6, 8, 9, 12, 16, K_SLICES_MOST}) {
      if (sp > groups || (sp > 1 && (shape == I8_ROUNDS || tiles * sp > SLICED_TILES_MOST))) break;
      const int per = (groups + sp - 1) / sp, splits = (groups + per - 1) / per;   // (no empty slice)
      const int64_t n = tiles * splits;
      const float r = n * (1.f / UNITS);
      float us = f.fixed + per * 4 * (f.base + f.load * std::min(r, 1.f) + f.more * std::max(r - 1, 0.f) + f.round * ((n + UNITS - 1) / UNITS - 1)) + f.out_mb * 2 * mb;
      if (splits > 1) us += f.slices + f.slice_mb * 4 * splits * mb;
      if (best.shape < 0 || us < best_us) {
        best = Int8Plan{shape, splits, per * 4};
        best_us = us;
      }
    }
  }
  if (few < best_us) best = Int8Plan{I8_FEW, 1, 0};
  if (narrow_us(M, N, K) < std::min(few, best_us)) best = Int8Plan{I8_NARROW, 1, 0};
  return best;
}

template <int WM, int WN, int AT, int BT>
void launch_shape(const Int8Params &g, int out, bool cold, hipStream_t s) {
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((g.ncol * g.splits + 7) / 8 * 8 * g.nrow), dim3(256), 0, s, g); };
  auto with = [&](auto COLD) {
    constexpr bool c = WM == 1 && decltype(COLD)::value;
    if (out == OUT_F32) launch(gemm_int8_kernel<WM, WN, AT, BT, OUT_F32, c>);
    else if (out == OUT_BF16) launch(gemm_int8_kernel<WM, WN, AT, BT, OUT_BF16, c>);
    else launch(gemm_int8_kernel<WM, WN, AT, BT, OUT_SLICES, c>);
  };
  if (cold) with(std::true_type{}); else with(std::false_type{});
}

template <typename T>
void launch_weights(const T *w, int64_t ldw, int8_t *q, float *scale, int N, int K, hipStream_t s) {
  // Lanes of a row so that it takes at most HELD pieces of a lane (more would not fit a lane's 128 registers); the longest rows are read twice.
  // us, with a product of eight rows behind, read twice by 128 lanes / held by 256 or 512: fp32 5120 x 27648 274 / 183, 1024 x 20480 54 / 32, bf16 5120 x
  // 27648 152 / 131.  Rows of a workgroup: whole lines, but workgroups of 1024 threads are alone on a unit and overlap nothing (eight rows of 128 lanes /
  // four: fp32 4128 x 8192 64 / 44, bf16 16384 x 8192 113 / 106), and few rows leave units without work (eight / two: bf16 512 x 1536 18.4 / 15.8;
  // four / two: bf16 3584 x 18944 67 / 60, but 5120 x 27648 131 / 140).
  constexpr int HELD = sizeof(T) == 4 ? 5 : 7;
  const int pieces = K / 16;
  int lanes = 32;
  while (lanes < 512 && pieces > lanes * HELD) lanes *= 2;
  auto launch = [&](auto ROWS) {
    auto with = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(N / ROWS.value), dim3(lanes * ROWS.value), 0, s, w, ldw, (uint4 *)q, scale, N, K); };
    if (pieces <= lanes * HELD) with(quantize_weights_kernel<T, HELD, ROWS.value>); else with(quantize_weights_kernel<T, 0, ROWS.value>);
  };
  const int rows = lanes <= 64 ? (N < 8 * UNITS ? 2 : 8) : lanes <= 256 && N >= 16 * UNITS ? 4 : 2;
  if (rows == 8) launch(std::integral_constant<int, 8>{});
  else if (rows == 4) launch(std::integral_constant<int, 4>{});
  else launch(std::integral_constant<int, 2>{});
}

}  // namespace

int launch_quantize_int8(const void *w, bool f32, int64_t ldw, int8_t *q, float *scale, int N, int K, hipStream_t s) {
  if (f32) launch_weights((const float *)w, ldw, q, scale, N, K, s);
  else launch_weights((const bf16_t *)w, ldw, q, scale, N, K, s);
  return done();
}

// Enough for every number of rows up to M: a program has one workspace for its largest batch, and fewer rows may take more slices.  With at most
// SLICED_TILES_MOST tiles times slices, slices times rows of tiles are at most that over the tiles of a row.
int64_t gemm_int8_workspace_bytes(int M, int N, int K) {
  const int groups = (K + K_UNIT - 1) / K_UNIT;
  const int64_t ordered = N <= 16 * UNITS ? (int64_t)row_blocks(std::min(M, 64)) * 32 * K : 0;
  int64_t sums = 0;
#pragma unroll
  for (int shape = 0; shape < I8_ROUNDS; ++shape) {
    const int most = SLICED_TILES_MOST / ((N + SHAPES[shape].cols - 1) / SHAPES[shape].cols), slices = std::min({most, groups, K_SLICES_MOST});
    if (slices > 1) sums = std::max(sums, std::min((int64_t)slices * M, (int64_t)most * SHAPES[shape].rows) * N);
  }
  return align256((int64_t)M * 4) + align256(std::max(ordered, (int64_t)M * groups * K_UNIT)) + sums * 4;
}

void gemm_int8_plan(int M, int N, int K, int32_t *kernel, int32_t *splits) {
  const Int8Plan p = int8_plan(M, N, K);
  *kernel = p.shape;
  *splits = p.splits;
}

int launch_gemm_int8(const bf16_t *x, int64_t ldx, const int8_t *wq, const float *sw, void *y, bool f32, int M, int N, int K, void *ws, hipStream_t s) {
  const Int8Plan plan = int8_plan(M, N, K);
  if (plan.shape == I8_FEW) {
    const int bytes = 256 + 8 * 4096 + M * (K + 16) + FEW_AHEAD * 256, grid = std::min(N / 32, 2 * UNITS);
    auto launch = [&](auto kernel, auto *out) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(512), bytes, s, x, ldx, wq, sw, out, M, N, K); };
    auto with = [&](auto *out) {
      typedef std::remove_pointer_t<decltype(out)> T;
      switch (few_rows(M)) {
        case 1: launch(gemm_int8_few_kernel<1, T>, out); break;
        case 2: launch(gemm_int8_few_kernel<2, T>, out); break;
        default: launch(gemm_int8_few_kernel<4, T>, out);
      }
    };
    if (f32) with((float *)y); else with((bf16_t *)y);
    return done();
  }
  const int k_pad = plan.shape == I8_NARROW ? K : (K + K_UNIT - 1) / K_UNIT * K_UNIT;
  float *sx = (float *)ws;
  int8_t *xq = (int8_t *)ws + align256((int64_t)M * 4);
  auto quantize = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3(M), dim3(std::min(1024, (K / 8 + 63) / 64 * 64)), 0, s, x, ldx, (uint2 *)xq, sx, K, k_pad, row_blocks(M));
  };
  if (plan.shape == I8_NARROW) {
    quantize(quantize_rows_kernel<true>);
    auto launch = [&](auto kernel, auto *out) { hipLaunchKernelGGL(kernel, dim3(N / 16), dim3(512), 0, s, xq, wq, sx, sw, out, M, N, K); };
    auto with = [&](auto *out, auto COLD) {
      typedef std::remove_pointer_t<decltype(out)> T;
      switch ((M + 15) / 16) {
        case 1: launch(gemm_int8_narrow_kernel<1, COLD.value, T>, out); break;
        case 2: launch(gemm_int8_narrow_kernel<2, COLD.value, T>, out); break;
        case 3: launch(gemm_int8_narrow_kernel<3, COLD.value, T>, out); break;
        default: launch(gemm_int8_narrow_kernel<4, COLD.value, T>, out);
      }
    };
    auto cold = [&](auto *out) {
      if ((int64_t)N * K > (8 << 20)) with(out, std::true_type{}); else with(out, std::false_type{});
    };
    if (f32) cold((float *)y); else cold((bf16_t *)y);
    return done();
  }
  quantize(quantize_rows_kernel<false>);
  int32_t *slices = (int32_t *)(xq + align256((int64_t)M * k_pad));
  Int8Params g{xq, wq, sx, sw, plan.splits > 1 ? (void *)slices : y, M, N, K, k_pad, plan.splits, plan.slice,
               (N + SHAPES[plan.shape].cols - 1) / SHAPES[plan.shape].cols, (M + SHAPES[plan.shape].rows - 1) / SHAPES[plan.shape].rows};
  const int out = plan.splits > 1 ? OUT_SLICES : f32 ? OUT_F32 : OUT_BF16;
  // Weights read once in the call, of a matrix so large that a model of such does not stay in the last-level cache between two steps, by non-temporal
  // loads: 1 row 55296 x 5120 52.8 -> 47.2 us, 37888 x 3584 33.9 -> 31.4, 128 rows 55296 x 5120 61.5 -> 57.2 (one matrix again and again out of the
  // cache: up to 10 % the other way, 37888 x 3584, 64 rows, 30 -> 33).
  const bool cold = g.nrow == 1 && (int64_t)N * K > (8 << 20);
  switch (plan.shape) {
    case I8_32x128: launch_shape<1, 4, 1, 1>(g, out, cold, s); break;
    case I8_64x128: launch_shape<1, 4, 2, 1>(g, out, cold, s); break;
    case I8_128x128: launch_shape<1, 4, 4, 1>(g, out, cold, s); break;
    case I8_128x256: launch_shape<1, 4, 4, 2>(g, out, cold, s); break;
    case I8_64x64: launch_shape<2, 2, 1, 1>(g, out, cold, s); break;
    default:
      if (out == OUT_F32) hipLaunchKernelGGL(gemm_int8_rounds_kernel<OUT_F32>, dim3(UNITS), dim3(256), 0, s, g);
      else hipLaunchKernelGGL(gemm_int8_rounds_kernel<OUT_BF16>, dim3(UNITS), dim3(256), 0, s, g);
  }
  if (plan.splits > 1) {
    const dim3 grid((N / 4 + 255) / 256, M);
    if (f32) hipLaunchKernelGGL(int8_slices_kernel<float>, grid, dim3(256), 0, s, (const i32x4 *)slices, sx, sw, (float *)y, plan.splits, M, N);
    else hipLaunchKernelGGL(int8_slices_kernel<bf16_t>, grid, dim3(256), 0, s, (const i32x4 *)slices, sx, sw, (bf16_t *)y, plan.splits, M, N);
  }
  return done();
}

}  // namespace pl
