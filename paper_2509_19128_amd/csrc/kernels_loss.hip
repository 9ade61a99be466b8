// Log-probabilities of given tokens under an LM head, and their gradient, without logits in memory.
//
//   z[t, v] = inv_t[t] * sum_k h[t, k] W[v, k],  lse[t] = log sum_v exp z[t, v],  logprob[t] = z[t, y_t] - lse[t]
//   G[t, v] = g[t] inv_t[t] (1[v = y_t] - exp(z[t, v] - lse[t])),  dh = G W,  dW = G^T h
//
// Four products on the matrix cores, all by the tiles of gemm_tile.h with x as the first operand, so that a lane ends with one column and
// many rows:
//   logits (forward, and again for the gradient)   x = W (rows v), w = h               a lane ends with one position and its logits
//   dh                                             x = W, k-major (rows d, k = v), w = G   a lane ends with one position and columns of dh
//   dW                                             x = h, k-major (rows d, k = t), w = G^T a lane ends with one vocabulary entry
// so W is read as it lies (row-major, no transposed copy), and what is reordered is small: h once per call, G where it is made.  A position's
// maximum and sum of exponentials are then sums over a lane's registers and one swap of halves.
//
// Positions without a target are left out from the start: the others are numbered, gathered and padded with zeros to whole tiles, and every
// kernel works on those ("rows" below); how many there are is known on the device only.
#include "gemm_tile.h"

#include <algorithm>

namespace pl {
namespace {

constexpr int GROUP = 64;           // vocabulary entries of a partial sum: the same whatever the tile, so that a position's result is too
constexpr int TILE_V = 256;         // vocabulary entries of a tile
constexpr int PIECE = 8192;         // rows of a forward pass: 8 bytes per row and group of partial sums
constexpr int UNITS = 256;          // workgroups of a kernel that walks tiles: one fills a compute unit
constexpr float LOG2E = 1.4426950408889634f;

struct Row { float inv_t, lse, scale; int32_t target; };   // scale = g inv_t; padding: all 0, target -1

// positions with a target in order, their number, the way back, and zeros for the others
__global__ __launch_bounds__(1024) void loss_rows_kernel(const int32_t *__restrict__ target, int32_t *__restrict__ count, int32_t *__restrict__ rows,
                                                         int32_t *__restrict__ place, float *__restrict__ logprob, float *__restrict__ lse, int n, int vocab) {
  __shared__ int32_t part[16];
  int base = 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int t0 = 0; t0 < n; t0 += 1024) {
    const int t = t0 + threadIdx.x;
    const bool in = t < n, has = in && (uint32_t)target[t] < (uint32_t)vocab;
    const uint64_t mask = __ballot(has);
    if (lane == 0) part[wave] = __popcll(mask);
    __syncthreads();
    int at = base, all = 0;
    for (int i = 0; i < 16; ++i) {
      if (i < wave) at += part[i];
      all += part[i];
    }
    at += __popcll(mask & (((uint64_t)1 << lane) - 1));
    if (has) rows[at] = t;
    if (in && place) place[t] = has ? at : -1;
    if (in && logprob && !has) logprob[t] = lse[t] = 0.f;
    base += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) *count = base;
}

struct Head {
  const bf16_t *h, *w;
  int64_t ldh, ldw;
  const int32_t *target;
  const float *inv_t, *lse, *g;   // inv_t, or lse and g, may be null
  const int32_t *rows, *count;
  int vocab, d;
};

// Rows [first, first + 32 * gridDim.x) in operand order (planes of 64 k, blocks of 32 rows; padding 0), as they are (copy, if any), and what
// the tiles want to know of each.
__global__ __launch_bounds__(256) void loss_gather_kernel(Head q, int first, bf16_t *__restrict__ op, bf16_t *__restrict__ copy, Row *__restrict__ info) {
  const int r0 = blockIdx.x * 32, count = *q.count - first, j = threadIdx.x >> 6, half = (threadIdx.x >> 5) & 1, r = r0 + (threadIdx.x & 31);
  const int k = blockIdx.y * 64 + half * 32 + j * 8, t = r < count ? q.rows[first + r] : -1;
  const uint4 v = t >= 0 ? *(const uint4 *)(q.h + t * q.ldh + k) : make_uint4(0, 0, 0, 0);
  *(uint4 *)(op + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2048 + threadIdx.x * 8) = v;
  if (copy) *(uint4 *)(copy + (int64_t)r * q.d + k) = v;
  if (blockIdx.y == 0 && threadIdx.x < 32) {
    Row i{0.f, 0.f, 0.f, -1};
    if (t >= 0) {
      i.inv_t = q.inv_t ? q.inv_t[t] : 1.f;
      if (q.g) { i.lse = q.lse[t]; i.scale = q.g[t] * i.inv_t; }
      i.target = q.target[t];
    }
    info[r] = i;
  }
}

// Logit tiles: 256 vocabulary entries from v_begin on x BN rows.  XCD i takes the i-th eighth of them; bands of 2048 rows, in a band vocabulary tile by
// vocabulary tile, so that an XCD's units share few operands at a time.
template <int BN>
struct LogitTiles {
  int nm, nv, at, end;
  __device__ __forceinline__ void init(int count, int n_v) {
    nm = (count + BN - 1) / BN; nv = (n_v + TILE_V - 1) / TILE_V;
    const int tiles = nm * nv, xcd = blockIdx.x & 7;
    at = xcd * (tiles >> 3) + min(xcd, tiles & 7);
    end = at + (tiles >> 3) + (xcd < (tiles & 7) ? 1 : 0);
    at += blockIdx.x >> 3;
  }
  __device__ __forceinline__ void place(int &mt, int &vt) const {
    constexpr int BAND = 2048 / BN;
    const int band = at / (BAND * nv), rest = at - band * BAND * nv, wide = min(BAND, nm - band * BAND);
    vt = rest / wide;
    mt = band * BAND + rest - vt * wide;
  }
};

template <typename T>
__device__ __forceinline__ Item logit_item(const Head &q, const bf16_t *op, int n_pad, int v_begin, int mt, int vt) {
  Item i;
  i.row0 = mt * T::BN; i.col0 = v_begin + vt * TILE_V; i.kind = 0;
  i.x = q.w + i.col0 * q.ldw; i.ldx = q.ldw; i.x_rows = min(q.vocab - i.col0, TILE_V);
  i.w = op; i.w_n = n_pad; i.w_planes = i.ksteps = q.d / BK; i.w_row = i.row0;
  return i;
}

// (max, sum of exponentials) of each row and group of vocabulary entries; the logit of the target from the tile that has it
template <int WM, int WN, int AT, int BT>
__global__ __launch_bounds__(256) void loss_forward_kernel(Head q, const bf16_t *__restrict__ op, const Row *__restrict__ info, float2 *__restrict__ parts, float *__restrict__ zt,
                                                           int first, int n_pad) {
  typedef Tile<WM, WN, AT, BT, false, TILE_COLS> T;
  __shared__ __attribute__((aligned(1024))) bf16_t xs[T::LDS];
  const int count = min(*q.count - first, n_pad);
  if (count <= 0) return;
  LogitTiles<T::BN> tiles;
  tiles.init(count, q.vocab);
  if (tiles.at >= tiles.end) return;
  T t;
  t.init_at(xs);
  walk(t, [] {}, [&](Item &d) {
    if (tiles.at >= tiles.end) return false;
    int mt, vt;
    tiles.place(mt, vt);
    d = logit_item<T>(q, op, n_pad, 0, mt, vt);
    tiles.at += gridDim.x >> 3;
    return true;
  }, [&](const Item &c) {
    const int v0 = c.col0 + t.wm * AT * 32;
#pragma unroll
    for (int b = 0; b < BT; ++b) {
      const int r = c.row0 + (t.wn * BT + b) * 32 + t.lrow;
      const Row row = info[r];
#pragma unroll
      for (int a = 0; a < AT; a += 2) {
        const int v = v0 + a * 32;   // a group
        float z[2][16];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) z[h][i] = t.result(a + h, b, i) * row.inv_t;
        if (v + GROUP > q.vocab) {   // (uniform: the last tile's entries beyond the vocabulary)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (h * 32 + (i >> 2) * 8 + (i & 3) >= q.vocab - v - t.half * 4) z[h][i] = -INFINITY;
        }
        const int y = row.target - v;
        if (__ballot(y >= 0 && y < GROUP)) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (y - t.half * 4 == h * 32 + (i >> 2) * 8 + (i & 3) && r < count) zt[r] = z[h][i];
        }
        float m = z[0][0];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) m = fmaxf(m, z[h][i]);
        m = with_xor32(m, OpMax{});
        float s = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) s += __builtin_amdgcn_exp2f((z[h][i] - m) * LOG2E);
        s = with_xor32(s, OpSum{});
        if (t.half == 0 && r < count && v < q.vocab) parts[(int64_t)(v / GROUP) * n_pad + r] = make_float2(m, s);
#ifdef __HIP_DEVICE_COMPILE__
        __builtin_amdgcn_sched_barrier(0);   // (one block's registers at a time)
#endif
      }
    }
  });
}

// The groups of 64 rows joined: sixteen wavefronts take every sixteenth group in order, then their sixteen results are joined in order.
__global__ __launch_bounds__(1024) void loss_merge_kernel(const float2 *__restrict__ parts, const float *__restrict__ zt, const int32_t *__restrict__ rows,
                                                          const int32_t *__restrict__ count, float *__restrict__ logprob, float *__restrict__ lse, int groups, int first,
                                                          int n_pad) {
  __shared__ float2 joined[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = blockIdx.x * 64 + lane, n = min(*count - first, n_pad);
  if ((int)blockIdx.x * 64 >= n) return;
  // (no entries: -inf, 0; NaN stays)
  auto join = [](float &m, float &s, float2 p) {
    const float top = p.x > m || p.x != p.x ? p.x : m;
    if (top == -INFINITY) return;
    s = s * __expf(m - top) + p.y * __expf(p.x - top);
    m = top;
  };
  float m = -INFINITY, s = 0.f;
  if (r < n)
    for (int g = wave; g < groups; g += 16 * 8) {
      float2 p[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) p[u] = g + u * 16 < groups ? parts[(int64_t)(g + u * 16) * n_pad + r] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int u = 0; u < 8; ++u) join(m, s, p[u]);
    }
  joined[wave][lane] = make_float2(m, s);
  __syncthreads();
  if (wave || r >= n) return;
  for (int i = 1; i < 16; ++i) join(m, s, joined[i][lane]);
  const float l = m + logf(s);
  const int t = rows[first + r];
  lse[t] = l;
  logprob[t] = zt[r] - l;
}

// a 32 x 32 block of results (a lane: one column, rows (i / 4) * 8 + half * 4 + i % 4) as two fragments of eight consecutive rows: 16 f + 8 half on
__device__ __forceinline__ void fragments(uint4 (&f)[2], const float (&v)[16]) {
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    uint32_t a[2], b[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      a[e] = two_bf16(v[8 * p + 2 * e], v[8 * p + 2 * e + 1]);
      b[e] = two_bf16(v[8 * p + 4 + 2 * e], v[8 * p + 4 + 2 * e + 1]);
    }
    f[p] = eight(a, b);
  }
}
// byte offset of fragment f of a 32 x 32 block in an operand-ordered image: row block `row`, 32-wide k block `k32`, rows n in all
__device__ __forceinline__ int64_t fragment_place(int row, int k32, int n, int f, int half, int lrow) {
  return ((((int64_t)(k32 >> 1) * (n >> 5) + row) * 4 + 2 * f + half) * 64 + (k32 & 1) * 32 + lrow) * 16;
}

// G of vocabulary entries [v_begin, v_begin + n_v), in operand order both ways: `by_row` for dh (a row's entries are its k) and `by_entry` for dW (an entry's
// rows are its k).  The second is the first's transpose by the matrix cores: a product with the unit matrix moves what a lane holds of a position
// to the lane of the entry, exactly.  Clears the tickets of the kernel behind.
template <int WM, int WN, int AT, int BT>
__global__ __launch_bounds__(256) void loss_grad_logits_kernel(Head q, const bf16_t *__restrict__ op, const Row *__restrict__ info, bf16_t *__restrict__ by_row, bf16_t *__restrict__ by_entry,
                                                               int v_begin, int n_v, int width, int n_pad, int32_t *__restrict__ tickets) {
  typedef Tile<WM, WN, AT, BT, false, TILE_COLS> T;
  __shared__ __attribute__((aligned(1024))) bf16_t xs[T::LDS];
  if (blockIdx.x == 0 && threadIdx.x < 8) tickets[threadIdx.x * 32] = 0;
  LogitTiles<T::BN> tiles;
  tiles.init(*q.count, n_v);
  if (tiles.at >= tiles.end) return;
  T t;
  t.init_at(xs);
  walk(t, [] {}, [&](Item &d) {
    if (tiles.at >= tiles.end) return false;
    int mt, vt;
    tiles.place(mt, vt);
    d = logit_item<T>(q, op, n_pad, v_begin, mt, vt);
    tiles.at += gridDim.x >> 3;
    return true;
  }, [&](const Item &c) {
    const int v0 = c.col0 + t.wm * AT * 32;
    bf16x8 unit[2];
#pragma unroll
    for (int f = 0; f < 2; ++f)
#pragma unroll
      for (int e = 0; e < 8; ++e) unit[f][e] = (bf16_t)(t.lrow - t.half * 8 == f * 16 + e ? 1.f : 0.f);
#pragma unroll
    for (int b = 0; b < BT; ++b) {
      const int m32 = (c.row0 >> 5) + t.wn * BT + b;
      const Row row = info[m32 * 32 + t.lrow];
#pragma unroll
      for (int a = 0; a < AT; ++a) {
        const int v = v0 + a * 32, v32 = (v - v_begin) >> 5, y = row.target - v;
        float G[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) G[i] = -row.scale * __builtin_amdgcn_exp2f((t.result(a, b, i) * row.inv_t - row.lse) * LOG2E);
        if (__ballot(y >= 0 && y < 32)) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (y - t.half * 4 == (i >> 2) * 8 + (i & 3)) G[i] += row.scale;
        }
        if (v + 32 > q.vocab) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if ((i >> 2) * 8 + (i & 3) >= q.vocab - v - t.half * 4) G[i] = 0.f;
        }
        uint4 f[2];
        fragments(f, G);
        if (by_row) {
#pragma unroll
          for (int k = 0; k < 2; ++k) *(uint4 *)((char *)by_row + fragment_place(m32, v32, n_pad, k, t.half, t.lrow)) = f[k];
        }
        if (by_entry) {
          f32x16 turned;
#pragma unroll
          for (int i = 0; i < 16; ++i) turned[i] = 0.f;
#ifdef __HIP_DEVICE_COMPILE__
#pragma unroll
          for (int k = 0; k < 2; ++k) turned = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, f[k]), unit[k], turned, 0, 0, 0);
#endif
          float G2[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) G2[i] = turned[i];
          fragments(f, G2);
#pragma unroll
          for (int k = 0; k < 2; ++k) *(uint4 *)((char *)by_entry + fragment_place(v32, m32, width, k, t.half, t.lrow)) = f[k];
        }
#ifdef __HIP_DEVICE_COMPILE__
        __builtin_amdgcn_sched_barrier(0);   // (one block's registers at a time)
#endif
      }
    }
  });
}

struct GradParams {
  const bf16_t *by_row, *by_entry, *copy;   // G both ways, h's rows
  float *dh32;                              // [slices][n_pad][d], or null: no dh
  bf16_t *dw;                               // or null
  int32_t *tickets;                         // eight, 128 bytes apart, zero
  int v_begin, n_v, width, n_pad, k_slice, tile_rows;   // k_slice: k-steps of a slice of dh; tile_rows: of the kernel that made G (rows beyond its last tile hold nothing)
};

// dh += G W and dW = G^T h of a piece of the vocabulary, 256 x 256 tiles of both in one launch: the units take them by tickets, those of dh, which
// are the longer ones, first, from their own XCD's eighth of each kind, then from the others'.
__global__ __launch_bounds__(256) void loss_grad_kernel(Head q, GradParams g) {
  typedef Tile<1, 4, 8, 2, false, TILE_COLS_T> T;
  // (one LDS object: of two the compiler would know that loads on their way to one may not be what a read of it wants, and wait for them all)
  __shared__ __attribute__((aligned(1024))) bf16_t xs[T::LDS + 4];
  typedef __attribute__((address_space(3))) volatile int32_t lds_int;
  lds_int *drawn = (lds_int *)(xs + T::LDS);
  const int count = *q.count, nd = q.d / 256, nm = (count + 255) / 256, nv = (g.n_v + TILE_V - 1) / TILE_V;
  const int planes = (count + g.tile_rows - 1) / g.tile_rows * g.tile_rows / BK;      // of by_entry that exist
  const int k_all = nv * (TILE_V / BK), k_slice = g.k_slice;
  const int n_dh = g.dh32 ? (k_all + k_slice - 1) / k_slice * nm * nd : 0, n_dw = g.dw ? nv * nd : 0;
  // the item of a ticket: eighth x of both kinds; -1: none left there
  auto first_of = [](int n, int x) { return x * (n >> 3) + min(x, n & 7); };
  auto draw = [&]() {   // one thread
    for (int k = 0; k < 8; ++k) {
      const int x = (blockIdx.x + k) & 7, a = first_of(n_dh, x), n_a = first_of(n_dh, x + 1) - a, b = first_of(n_dw, x), n_b = first_of(n_dw, x + 1) - b;
      if (n_a + n_b == 0) continue;
      const int i = __hip_atomic_fetch_add(&g.tickets[x * 32], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (i < n_a) return a + i;
      if (i < n_a + n_b) return n_dh + b + (i - n_a);
    }
    return -1;
  };
  auto item = [&](int i) {
    Item c;
    if (i < n_dh) {
      const int dt = i % nd, rest = i / nd, mt = rest % nm, k0 = rest / nm * k_slice;
      c.kind = 0; c.row0 = mt * 256; c.col0 = dt * 256; c.ksteps = min(k_slice, k_all - k0);
      const int v = g.v_begin + k0 * BK;
      c.x = q.w + v * q.ldw + c.col0; c.ldx = q.ldw; c.x_rows = min(q.vocab - v, c.ksteps * BK);
      c.w = g.by_row + (int64_t)k0 * (g.n_pad >> 5) * 2048; c.w_n = g.n_pad; c.w_planes = c.ksteps; c.w_row = c.row0;
      c.kind = rest / nm;
    } else {
      const int j = i - n_dh, dt = j % nd, vt = j / nd;
      c.kind = -1; c.row0 = vt * TILE_V; c.col0 = dt * 256; c.ksteps = max(4, (planes + 3) / 4 * 4);
      c.x = g.copy + c.col0; c.ldx = q.d; c.x_rows = g.n_pad;
      c.w = g.by_entry; c.w_n = g.width; c.w_planes = planes; c.w_row = c.row0;
    }
    return c;
  };
  if (threadIdx.x == 0) {
    drawn[0] = draw();
    drawn[1] = draw();
  }
  __syncthreads();
  if (drawn[0] < 0) return;
  T t;
  t.init_at(xs);
  int turn = 0;
  walk(t, [&] {
    if (threadIdx.x == 0) drawn[turn] = draw();   // for the tile behind the next: its place was read a tile ago, and is read again behind this tile's barriers
  }, [&](Item &d) {
    const int i = __builtin_amdgcn_readfirstlane(drawn[turn]);
    turn ^= 1;
    if (i < 0) return false;
    d = item(i);
    return true;
  }, [&](const Item &c) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int r = c.row0 + (t.wn * 2 + b) * 32 + t.lrow;
      if (c.kind >= 0) {
        float *o = g.dh32 + ((int64_t)c.kind * g.n_pad + r) * q.d + c.col0 + t.half * 4;
        if (r < count) {
#pragma unroll
          for (int a = 0; a < 8; ++a) {
            f32x4 sum[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = g.v_begin > 0 ? *(const f32x4 *)(o + a * 32 + i * 8) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *(f32x4 *)(o + a * 32 + i * 8) = sum[i] + f32x4{t.result(a, b, 4 * i), t.result(a, b, 4 * i + 1), t.result(a, b, 4 * i + 2), t.result(a, b, 4 * i + 3)};
#ifdef __HIP_DEVICE_COMPILE__
            __builtin_amdgcn_sched_barrier(0);   // (one block's registers at a time)
#endif
          }
        }
      } else {
        bf16_t *o = g.dw + (int64_t)(g.v_begin + r) * q.d + c.col0 + t.half * 8;
#pragma unroll
        for (int a = 0; a < 8; ++a) {
          float v[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = t.result(a, b, i);
          uint4 f[2];
          fragments(f, v);
          if (g.v_begin + r < q.vocab) {
#pragma unroll
            for (int k = 0; k < 2; ++k) *(uint4 *)(o + a * 32 + k * 16) = f[k];
          }
#ifdef __HIP_DEVICE_COMPILE__
          __builtin_amdgcn_sched_barrier(0);   // (one block's registers at a time)
#endif
        }
      }
    }
  });
}

// dh of every position: the slices of its row added up in order and rounded, or zeros
__global__ __launch_bounds__(256) void loss_round_kernel(const float *__restrict__ dh32, bf16_t *__restrict__ dh, const int32_t *__restrict__ place, int slices, int n_pad, int d) {
  const int t = blockIdx.x, k = (blockIdx.y * 256 + threadIdx.x) * 4, r = place[t];
  if (k >= d) return;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (r >= 0)
    for (int s = 0; s < slices; ++s) v += *(const f32x4 *)(dh32 + ((int64_t)s * n_pad + r) * d + k);
  bf16x4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = (bf16_t)v[e];
  *(bf16x4 *)(dh + (int64_t)t * d + k) = o;
}

int64_t align256(int64_t b) { return (b + 255) / 256 * 256; }
int padded(int n) { return (n + 255) / 256 * 256; }
int done() { return hipGetLastError() == hipSuccess ? 0 : -7; }

struct Carver {
  char *at;
  template <typename T>
  T *take(int64_t n) {
    T *p = (T *)at;
    at += align256(n * (int64_t)sizeof(T));
    return p;
  }
};

struct ForwardSpace {
  int32_t *count, *rows;
  Row *info;
  bf16_t *op;
  float *zt;
  float2 *parts;
  int n_pad, groups;
  int64_t bytes;
  ForwardSpace(void *ws, int n, int vocab, int d) {
    Carver c{(char *)ws};
    n_pad = padded(std::min(n, PIECE));
    groups = (vocab + GROUP - 1) / GROUP;
    count = c.take<int32_t>(1); rows = c.take<int32_t>(n); info = c.take<Row>(n_pad); op = c.take<bf16_t>((int64_t)n_pad * d);
    zt = c.take<float>(n_pad); parts = c.take<float2>((int64_t)groups * n_pad);
    bytes = c.at - (char *)ws;
  }
};

// Vocabulary entries of a piece of the gradient: G, both ways, in 256 MB (what the last-level cache holds), at least a tile, and W's part of it
// behind a 32-bit offset.
int grad_width(int n_pad, int vocab) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(((int64_t)vocab + 255) / 256, ((int64_t)64 << 20) / n_pad / 256)) * 256;
}
// Slices of dh along a piece's vocabulary: until there are as many tiles as units (each is 4 n d bytes, read and written per piece).
int grad_slices(int n_pad, int width, int d) {
  const int tiles = n_pad / 256 * (d / 256);
  return std::max(1, std::min({UNITS / tiles, width / 1024, 16}));
}

struct GradSpace {
  int32_t *count, *tickets, *rows, *place;
  Row *info;
  bf16_t *op, *copy, *by_row, *by_entry;
  float *dh32;
  int n_pad, width, slices;
  int64_t bytes;
  GradSpace(void *ws, int n, int vocab, int d) {
    Carver c{(char *)ws};
    n_pad = padded(n);
    width = grad_width(n_pad, vocab);
    slices = grad_slices(n_pad, width, d);
    count = c.take<int32_t>(1); tickets = c.take<int32_t>(8 * 32); rows = c.take<int32_t>(n); place = c.take<int32_t>(n); info = c.take<Row>(n_pad);
    op = c.take<bf16_t>((int64_t)n_pad * d); copy = c.take<bf16_t>((int64_t)n_pad * d);
    by_row = c.take<bf16_t>((int64_t)n_pad * width); by_entry = c.take<bf16_t>((int64_t)n_pad * width);
    dh32 = c.take<float>((int64_t)slices * n_pad * d);
    bytes = c.at - (char *)ws;
  }
};

// calls f(rows of a tile, a kernel's shape as constants)
template <typename F>
void with_shape(int n, bool narrow, F f) {
  using std::integral_constant;
  if (narrow && n <= 32) f(integral_constant<int, 4>{}, integral_constant<int, 1>{}, integral_constant<int, 2>{}, integral_constant<int, 1>{});
  else if (n <= 64) f(integral_constant<int, 4>{}, integral_constant<int, 1>{}, integral_constant<int, 2>{}, integral_constant<int, 2>{});
  else if (n <= 128) f(integral_constant<int, 2>{}, integral_constant<int, 2>{}, integral_constant<int, 4>{}, integral_constant<int, 2>{});
  else f(integral_constant<int, 1>{}, integral_constant<int, 4>{}, integral_constant<int, 8>{}, integral_constant<int, 2>{});
}

}  // namespace

int64_t token_logprob_workspace_bytes(int n, int vocab, int d) { return ForwardSpace(nullptr, n, vocab, d).bytes; }

int launch_token_logprob(const TokenLoss &p, float *logprob, float *lse, hipStream_t s) {
  const ForwardSpace w(p.workspace, p.n, p.vocab, p.d);
  const Head q{p.h, p.w, p.ldh, p.ldw, p.target, p.inv_t, nullptr, nullptr, w.rows, w.count, p.vocab, p.d};
  hipLaunchKernelGGL(loss_rows_kernel, dim3(1), dim3(1024), 0, s, p.target, w.count, w.rows, (int32_t *)nullptr, logprob, lse, p.n, p.vocab);
  for (int first = 0; first < p.n; first += PIECE) {
    hipLaunchKernelGGL(loss_gather_kernel, dim3(w.n_pad / 32, p.d / 64), dim3(256), 0, s, q, first, w.op, (bf16_t *)nullptr, w.info);
    with_shape(std::min(p.n - first, PIECE), true, [&](auto WM, auto WN, auto AT, auto BT) {
      hipLaunchKernelGGL((loss_forward_kernel<WM.value, WN.value, AT.value, BT.value>), dim3(UNITS), dim3(256), 0, s, q, w.op, w.info, w.parts, w.zt, first, w.n_pad);
    });
    hipLaunchKernelGGL(loss_merge_kernel, dim3(w.n_pad / 64), dim3(1024), 0, s, w.parts, w.zt, w.rows, w.count, logprob, lse, w.groups, first, w.n_pad);
  }
  return done();
}

int64_t token_logprob_grad_workspace_bytes(int n, int vocab, int d) { return GradSpace(nullptr, n, vocab, d).bytes; }

int launch_token_logprob_grad(const TokenLoss &p, const float *lse, const float *g, bf16_t *dh, bf16_t *dw, hipStream_t s) {
  const GradSpace w(p.workspace, p.n, p.vocab, p.d);
  const Head q{p.h, p.w, p.ldh, p.ldw, p.target, p.inv_t, lse, g, w.rows, w.count, p.vocab, p.d};
  hipLaunchKernelGGL(loss_rows_kernel, dim3(1), dim3(1024), 0, s, p.target, w.count, w.rows, w.place, (float *)nullptr, (float *)nullptr, p.n, p.vocab);
  hipLaunchKernelGGL(loss_gather_kernel, dim3(w.n_pad / 32, p.d / 64), dim3(256), 0, s, q, 0, w.op, w.copy, w.info);
  // (W's rows of a piece lie behind one 32-bit offset)
  const int width = (int)std::min<int64_t>(w.width, (((int64_t)1 << 30) / p.ldw) / 256 * 256);
  // tiles of a slice from the first piece, the largest: later ones have no slice that it has not
  const int first_tiles = (std::min(width, p.vocab) + TILE_V - 1) / TILE_V, slice_tiles = (first_tiles + w.slices - 1) / w.slices;
  with_shape(p.n, false, [&](auto WM, auto WN, auto AT, auto BT) {
    for (int v = 0; v < p.vocab; v += width) {
      const int n_v = std::min(width, p.vocab - v);
      hipLaunchKernelGGL((loss_grad_logits_kernel<WM.value, WN.value, AT.value, BT.value>), dim3(UNITS), dim3(256), 0, s, q, w.op, w.info, dh ? w.by_row : nullptr,
                         dw ? w.by_entry : nullptr, v, n_v, w.width, w.n_pad, w.tickets);
      const GradParams gp{w.by_row, w.by_entry, w.copy, dh ? w.dh32 : nullptr, dw, w.tickets, v, n_v, w.width, w.n_pad, slice_tiles * (TILE_V / BK), WN.value * BT.value * 32};
      hipLaunchKernelGGL(loss_grad_kernel, dim3(UNITS), dim3(256), 0, s, q, gp);
    }
  });
  if (dh) hipLaunchKernelGGL(loss_round_kernel, dim3(p.n, (p.d / 4 + 255) / 256), dim3(256), 0, s, w.dh32, dh, w.place, (first_tiles + slice_tiles - 1) / slice_tiles, w.n_pad, p.d);
  return done();
}

}  // namespace pl
