// Products in 8-bit integers: y = x W^T with a scale per row of x (token) and per row of W (channel).
//
// Quantisation of a row: scale = max |x| / 127 in fp32, code = the integer nearest to x / scale (ties to even), at most 127 in magnitude.  The
// quotient is rounded as if exact: the product is then the same for every implementation of that sentence.  Codes are multiplied and added up
// in int32 without error (127^2 K < 2^31), in any order and any number of slices, and a result is (float(sum) * scale of its token) * scale of
// its channel.
//
// The product is gemm_tile.h's: W's codes in operand order straight to the registers of the first operand, x's through LDS.  Bytes per k-step and cycles
// of a matrix instruction are those of the bf16 product at twice the k, so a byte of weights does twice the work in both bounds.
#include "gemm_tile.h"

#include <algorithm>

namespace pl {
namespace {

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
// sides of the quotient times a power of two, so that 1 / s is finite.
struct RowScale {
  float scale, s, inv, up;
  __device__ inline explicit RowScale(float most) {
    const bool fine = most < INFINITY;
    scale = fine ? most / 127.f : NAN;
    up = scale < 0x1p-100f ? 0x1p100f : 1.f;
    s = fine ? scale * up : 0.f;
    inv = s > 0.f ? 1.f / s : 0.f;
  }
  __device__ inline int code(float x) const { return inv > 0.f ? quotient(x * up, s, inv) : 0; }
};
__device__ inline float magnitude(float x, float m) {   // infinity stands for NaN too
  const float a = fabsf(x);
  return a < INFINITY ? fmaxf(m, a) : INFINITY;
}
// sixteen values of a row
template <typename T>
struct Sixteen {
  uint4 raw[sizeof(T)];
  __device__ __forceinline__ void load(const T *p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) raw[i] = ((const uint4 *)p)[i];
  }
  __device__ __forceinline__ float get(int i) const { return (float)((const T *)raw)[i]; }
  __device__ __forceinline__ float most(float m) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) m = magnitude(get(i), m);
    return m;
  }
  __device__ __forceinline__ uint4 codes(const RowScale &r) const {
    uint32_t q[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      q[w] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) q[w] |= ((uint32_t)r.code(get(w * 4 + e)) & 255u) << (8 * e);
    }
    return make_uint4(q[0], q[1], q[2], q[3]);
  }
};

// Codes of weights in operand order.  Eight rows per workgroup: a 128-byte line of the image holds the same sixteen k of eight rows.  A lane keeps its
// values between the two passes where they fit into HELD pieces of sixteen.
template <typename T, int HELD>
__global__ __launch_bounds__(1024) void quantize_weights_kernel(const T *__restrict__ w, int64_t ldw, uint4 *__restrict__ q, float *__restrict__ scale, int N, int K) {
  const int r = threadIdx.x & 7, row = blockIdx.x * 8 + r, lanes = blockDim.x >> 3, first = threadIdx.x >> 3, pieces = K >> 4;
  w += row * ldw;
  Sixteen<T> held[HELD ? HELD : 1];
  float m = 0.f;
  if constexpr (HELD > 0) {
#pragma unroll
    for (int u = 0; u < HELD; ++u)
      if (first + u * lanes < pieces) held[u].load(w + (first + u * lanes) * 16);
#pragma unroll
    for (int u = 0; u < HELD; ++u)
      if (first + u * lanes < pieces) m = held[u].most(m);
  } else {
    for (int p = first; p < pieces; p += lanes) {
      held[0].load(w + p * 16);
      m = held[0].most(m);
    }
  }
  __shared__ float part[16][8];
  m = fmaxf(m, dpp<DPP_ROR8>(m));
  m = with_xor16(m, OpMax{});
  m = with_xor32(m, OpMax{});
  if ((threadIdx.x & 63) < 8) part[threadIdx.x >> 6][r] = m;
  __syncthreads();
  for (int i = 0; i < (int)blockDim.x >> 6; ++i) m = fmaxf(m, part[i][r]);
  const RowScale rs(m);
  if (first == 0) scale[row] = rs.scale;
  auto store = [&](int p, const Sixteen<T> &v) {   // piece p is (k / 16): block p / 8, half (p / 4) % 2, quarter p % 4
    q[(((int64_t)(p >> 3) * (N >> 5) + (row >> 5)) * 4 + (p & 3)) * 64 + ((p >> 2) & 1) * 32 + (row & 31)] = v.codes(rs);
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

// Codes of x, row-major, rows padded with zeros to k_pad.  A workgroup per row.
__global__ __launch_bounds__(1024) void quantize_rows_kernel(const bf16_t *__restrict__ x, int64_t ldx, uint4 *__restrict__ q, float *__restrict__ scale, int K, int k_pad) {
  x += blockIdx.x * ldx;
  q += (int64_t)blockIdx.x * (k_pad >> 4);
  const int pieces = K >> 4;
  Sixteen<bf16_t> v;
  float m = 0.f;
  for (int p = threadIdx.x; p < pieces; p += blockDim.x) {
    v.load(x + p * 16);
    m = v.most(m);
  }
  __shared__ float part[16];
  m = wave_max(m);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  for (int i = 0; i < (int)blockDim.x >> 6; ++i) m = fmaxf(m, part[i]);
  const RowScale rs(m);
  if (threadIdx.x == 0) scale[blockIdx.x] = rs.scale;
  for (int p = threadIdx.x; p < k_pad >> 4; p += blockDim.x) {
    if (p < pieces && pieces > (int)blockDim.x) v.load(x + p * 16);   // (otherwise the one piece is still here)
    q[p] = p < pieces ? v.codes(rs) : make_uint4(0, 0, 0, 0);
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
template <int WM, int WN, int AT, int BT, int OUT>
__global__ __launch_bounds__(256) void gemm_int8_kernel(Int8Params g) {
  typedef Tile<WM, WN, AT, BT, false, TILE_INT8> T;
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
  walk(t, [] {}, [&](Item &d) {
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

int done() { return hipGetLastError() == hipSuccess ? 0 : -7; }
int64_t align256(int64_t b) { return (b + 255) / 256 * 256; }

// How a product is cut: tile shape and K slices.
enum { I8_32x128, I8_64x128, I8_128x128, I8_128x256, I8_256x128, I8_64x64, I8_ROUNDS };
struct Int8Plan { int shape, splits, slice; };
constexpr int SHAPE_ROWS[] = {32, 64, 128, 128, 256, 64, 256}, SHAPE_COLS[] = {128, 128, 128, 256, 128, 64, 256};
Int8Plan int8_plan(int M, int N, int K) {
  const int groups = (K + K_UNIT - 1) / K_UNIT;
  int shape = M <= 32 ? I8_32x128 : M <= 64 ? I8_64x128 : M <= 128 ? I8_128x128 : M <= 256 ? I8_256x128 : I8_ROUNDS;
  int splits = 1;
  if (shape != I8_ROUNDS) {
    const int tiles = (M + SHAPE_ROWS[shape] - 1) / SHAPE_ROWS[shape] * ((N + SHAPE_COLS[shape] - 1) / SHAPE_COLS[shape]);
    splits = std::max(1, std::min(groups, UNITS / tiles));
  }
  const int per = (groups + splits - 1) / splits;
  return Int8Plan{shape, (groups + per - 1) / per, per * 4};   // (no empty slice)
}

template <int WM, int WN, int AT, int BT>
void launch_shape(const Int8Params &g, int out, hipStream_t s) {
  const dim3 grid((g.ncol * g.splits + 7) / 8 * 8 * g.nrow);
  if (out == OUT_F32) hipLaunchKernelGGL((gemm_int8_kernel<WM, WN, AT, BT, OUT_F32>), grid, dim3(256), 0, s, g);
  else if (out == OUT_BF16) hipLaunchKernelGGL((gemm_int8_kernel<WM, WN, AT, BT, OUT_BF16>), grid, dim3(256), 0, s, g);
  else hipLaunchKernelGGL((gemm_int8_kernel<WM, WN, AT, BT, OUT_SLICES>), grid, dim3(256), 0, s, g);
}

template <typename T>
void launch_weights(const T *w, int64_t ldw, int8_t *q, float *scale, int N, int K, hipStream_t s) {
  // lanes of a row so that it takes at most HELD pieces of a lane: 32, 64 or 128
  constexpr int HELD = sizeof(T) == 4 ? 4 : 8;
  const int pieces = K / 16, lanes = pieces <= 32 * HELD ? 32 : pieces <= 64 * HELD ? 64 : 128;
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(N / 8), dim3(lanes * 8), 0, s, w, ldw, (uint4 *)q, scale, N, K); };
  if (pieces <= lanes * HELD) launch(quantize_weights_kernel<T, HELD>);
  else launch(quantize_weights_kernel<T, 0>);
}

}  // namespace

int launch_quantize_int8(const void *w, bool f32, int64_t ldw, int8_t *q, float *scale, int N, int K, hipStream_t s) {
  if (f32) launch_weights((const float *)w, ldw, q, scale, N, K, s);
  else launch_weights((const bf16_t *)w, ldw, q, scale, N, K, s);
  return done();
}

int64_t gemm_int8_workspace_bytes(int M, int N, int K) {
  const Int8Plan p = int8_plan(M, N, K);
  return align256((int64_t)M * 4) + align256((int64_t)M * ((K + K_UNIT - 1) / K_UNIT * K_UNIT)) + (p.splits > 1 ? (int64_t)p.splits * M * N * 4 : 0);
}

int launch_gemm_int8(const bf16_t *x, int64_t ldx, const int8_t *wq, const float *sw, void *y, bool f32, int M, int N, int K, void *ws, hipStream_t s) {
  const Int8Plan plan = int8_plan(M, N, K);
  const int k_pad = (K + K_UNIT - 1) / K_UNIT * K_UNIT;
  float *sx = (float *)ws;
  int8_t *xq = (int8_t *)ws + align256((int64_t)M * 4);
  int32_t *slices = (int32_t *)(xq + align256((int64_t)M * k_pad));
  hipLaunchKernelGGL(quantize_rows_kernel, dim3(M), dim3(std::min(1024, (K / 16 + 63) / 64 * 64)), 0, s, x, ldx, (uint4 *)xq, sx, K, k_pad);
  Int8Params g{xq, wq, sx, sw, plan.splits > 1 ? (void *)slices : y, M, N, K, k_pad, plan.splits, plan.slice,
               (N + SHAPE_COLS[plan.shape] - 1) / SHAPE_COLS[plan.shape], (M + SHAPE_ROWS[plan.shape] - 1) / SHAPE_ROWS[plan.shape]};
  const int out = plan.splits > 1 ? OUT_SLICES : f32 ? OUT_F32 : OUT_BF16;
  switch (plan.shape) {
    case I8_32x128: launch_shape<1, 4, 1, 1>(g, out, s); break;
    case I8_64x128: launch_shape<1, 4, 2, 1>(g, out, s); break;
    case I8_128x128: launch_shape<1, 4, 4, 1>(g, out, s); break;
    case I8_128x256: launch_shape<1, 4, 4, 2>(g, out, s); break;
    case I8_256x128: launch_shape<1, 4, 8, 1>(g, out, s); break;
    case I8_64x64: launch_shape<2, 2, 1, 1>(g, out, s); break;
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
