// Log-probabilities of given tokens under an LM head, and their gradient, without logits in memory.
//
//   z[t, v] = inv_t[t] * sum_k h[t, k] W[v, k],  lse[t] = log sum_v exp z[t, v],  logprob[t] = z[t, y_t] - lse[t]
//   G[t, v] = g[t] inv_t[t] (1[v = y_t] - exp(z[t, v] - lse[t])),  dh = G W,  dW = G^T h
//
// Four products on the matrix cores, by the tiles of gemm_tile.h:
//   logits (forward, and again for the gradient)   x = W (rows v), w = h               a lane ends with one position and its logits
//   dh                                             x = W, k-major (rows d, k = v), w = G   a lane ends with one position and columns of dh
//   dW                                             x = G, across (rows v, k = t), w = h^T  a lane ends with one vocabulary entry
// so W is read as it lies (row-major, no transposed copy), G is written once, in operand order, and what else is reordered is small: h and h^T, once per
// call.  A position's maximum and sum of exponentials are then sums over a lane's registers and one swap of halves.
//
// Positions without a target are left out from the start: the others are numbered, gathered and padded with zeros to whole tiles, and every
// kernel works on those ("rows" below); how many there are is known on the device only.
#include "gemm_tile.h"

#include <algorithm>

namespace pl {
namespace {

constexpr int GROUP = 64;           // vocabulary entries of a partial sum: the same whatever the tile, so that a position's result is too
constexpr int TILE_V = 256;         // vocabulary entries that the gradient is cut by
constexpr int PIECE = 8192;         // rows of a forward pass: 8 bytes per row and group of partial sums
constexpr int UNITS = 256;          // workgroups of a kernel that walks tiles: one fills a compute unit
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// What the tiles want of a row.  Forward: factor = inv_t log2(e), since exponentials are powers of two, scale = inv_t; gradient: factor = inv_t, lse,
// scale = g inv_t.
// Padding: all 0, target -1.
struct Row { float factor, lse, scale; int32_t target; };
__device__ inline float finite_or_nan(float x) { return fabsf(x) < INFINITY ? x : NAN; }
// (not negative: the largest product has the largest logit; for 0 the smallest number, whose multiple of any product is below 5e-7, but of -inf, an entry that is masked
// or beyond the vocabulary, -inf and not 0 * inf)
__device__ inline float temperature(float inv_t) { return inv_t >= 0.f && inv_t < INFINITY ? fmaxf(inv_t, 0x1p-149f) : NAN; }
// (finite, so that a difference of 0 stays one)
__device__ inline float logit_factor(float it) { return it * LOG2E < INFINITY ? it * LOG2E : it == it ? 0x1.fffffep127f : NAN; }

// The workgroup numbers the positions with a target in order: each(position, has, number) for every position; returns how many there are.
template <int THREADS, typename Each>
__device__ __forceinline__ int number_positions(const int32_t *__restrict__ target, int n, int vocab, Each each) {
  __shared__ int32_t part[THREADS / 64];
  int base = 0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int t0 = 0; t0 < n; t0 += THREADS) {
    const int t = t0 + threadIdx.x;
    const bool has = t < n && (uint32_t)target[t] < (uint32_t)vocab;
    const uint64_t mask = __ballot(has);
    if (lane == 0) part[wave] = __popcll(mask);
    __syncthreads();
    int at = base, all = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) {
      if (i < wave) at += part[i];
      all += part[i];
    }
    if (t < n) each(t, has, at + __popcll(mask & (((uint64_t)1 << lane) - 1)));
    base += all;
    __syncthreads();
  }
  return base;
}

// How many positions have a target, which the device finds out, and how the gradient is cut for so many rows: vocabulary tiles of a piece, tiles of a slice
// of dh along a piece, and slices.  A piece's G takes at most `most` tiles of 256 x 256 (or one vocabulary tile's); its tiles are whole rounds of the
// units where there are that many.  Slices of dh: until there are as many tiles as units (each is a sum of its own that is read and written per piece).
struct Cut {
  int count, nm, piece, slice, slices;
  static __host__ __device__ int slices_most(int nm, int d) {
    const int tiles = nm * (d / 256), s = tiles > 0 ? UNITS / tiles : 1;
    return s < 1 ? 1 : s > 16 ? 16 : s;
  }
  static __host__ __device__ Cut of(int count, int vocab, int d, int64_t ldw, int most) {
    Cut c;
    c.count = count;
    c.nm = (count + 255) / 256;
    const int tiles = (vocab + TILE_V - 1) / TILE_V, fit = most / (c.nm > 0 ? c.nm : 1), far = (1 << 22) / (int)ldw;   // (W's rows of a piece lie behind one 32-bit offset)
    int p = fit < far ? fit : far;
    if (c.nm > 0 && c.nm * p >= UNITS) p = c.nm * p / UNITS * UNITS / c.nm;
    if (p < 1) p = 1;
    c.piece = p < tiles ? p : tiles;
    const int s = slices_most(c.nm, d);
    c.slice = (c.piece + s - 1) / s;
    c.slices = (c.piece + c.slice - 1) / c.slice;
    return c;
  }
};

// What is known of the positions: how many have a target, which, and the way back (place, may be null); zeros for the others (logprob and lse may be null).
struct Positions {
  const int32_t *target;
  Cut *cut;
  int32_t *rows, *place;
  float *logprob, *lse;
  int n, vocab, d, most;
  int64_t ldw;
  __device__ __forceinline__ void note(int t, bool has, int number) const {
    if (has) rows[number] = t;
    if (place) place[t] = has ? number : -1;
    if (logprob && !has) logprob[t] = lse[t] = 0.f;
  }
};
__global__ __launch_bounds__(1024) void loss_rows_kernel(Positions q) {
  const int count = number_positions<1024>(q.target, q.n, q.vocab, [&](int t, bool has, int number) { q.note(t, has, number); });
  if (threadIdx.x == 0) *q.cut = Cut::of(count, q.vocab, q.d, q.ldw, q.most);
}

struct Head {
  const bf16_t *h, *w;
  int64_t ldh, ldw;
  const int32_t *target;
  const float *inv_t, *lse, *g;   // inv_t, or lse and g, may be null
  const int32_t *rows;
  const Cut *cut;
  int vocab, d;
};

// Rows [first, first + 32 * gridDim.x) in operand order (planes of 64 k, blocks of 32 rows; padding 0), their transpose in operand order (if any: planes
// of 64 rows, blocks of 32 k; `low`: rows below it a second time, so many rows on), and what the tiles want to know of each.  NUMBER: few positions, which every workgroup numbers for itself instead of a launch ahead.
template <bool NUMBER>
__global__ __launch_bounds__(256) void loss_gather_kernel(Head q, Positions at, int first, bf16_t *__restrict__ op, bf16_t *__restrict__ turned, int low,
                                                          Row *__restrict__ info) {
  const int r0 = blockIdx.x * 32, j = threadIdx.x >> 6, half = (threadIdx.x >> 5) & 1, r = r0 + (threadIdx.x & 31), k = blockIdx.y * 64 + half * 32 + j * 8;
  int t = -1;
  if constexpr (NUMBER) {
    __shared__ int32_t mine[32];
    if (threadIdx.x < 32) mine[threadIdx.x] = -1;
    __syncthreads();
    const bool note = blockIdx.x == 0 && blockIdx.y == 0;
    const int count = number_positions<256>(at.target, at.n, at.vocab, [&](int u, bool has, int number) {
      if (has && (uint32_t)(number - r0) < 32u) mine[number - r0] = u;
      if (note) at.note(u, has, number);
    });
    if (note && threadIdx.x == 0) *at.cut = Cut::of(count, at.vocab, at.d, at.ldw, at.most);
    t = mine[threadIdx.x & 31];   // (number_positions ends behind a barrier; n >= 1)
  } else if (r < q.cut->count - first) {
    t = q.rows[first + r];
  }
  const uint4 v = t >= 0 ? *(const uint4 *)(q.h + t * q.ldh + k) : make_uint4(0, 0, 0, 0);
  *(uint4 *)(op + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2048 + threadIdx.x * 8) = v;
  if (turned && (low == 0 || r0 < low)) {   // (uniform)
    __shared__ __attribute__((aligned(16))) bf16_t block[32][72];
    *(uint4 *)&block[threadIdx.x & 31][half * 32 + j * 8] = v;
    __syncthreads();
    const int c = threadIdx.x & 63;   // column, and eight rows from j * 8 on
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = block[j * 8 + e][c];
    const int k32 = (blockIdx.y * 64 + c) >> 5;
    for (int to = r0; to <= r0 + low; to += low ? low : 1)
      *(bf16x8 *)(turned + ((((int64_t)(to >> 6) * (q.d >> 5) + k32) * 4 + j) * 64 + ((to >> 5) & 1) * 32 + (c & 31)) * 8) = o;
  }
  if (blockIdx.y == 0 && threadIdx.x < 32) {
    Row i{0.f, 0.f, 0.f, -1};
    if (t >= 0) {
      const float inv_t = q.inv_t ? q.inv_t[t] : 1.f, it = temperature(inv_t);
      i.factor = logit_factor(it);
      i.scale = it;
      if (q.g) {
        i.factor = it;
        i.lse = finite_or_nan(q.lse[t]);
        i.scale = q.g[t] * inv_t;
      }
      i.target = q.target[t];
    }
    info[r] = i;
  }
}

// Logit tiles: BM vocabulary entries x BN rows.  XCD i takes the i-th eighth of them; bands of 2048 rows, in a band vocabulary tile by
// vocabulary tile, so that an XCD's units share few operands at a time.
template <int BM, int BN>
struct LogitTiles {
  int nm, nv, at, end;
  __device__ __forceinline__ void init(int count, int n_v) {
    nm = (count + BN - 1) / BN; nv = (n_v + BM - 1) / BM;
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
  i.row0 = mt * T::BN; i.col0 = v_begin + vt * T::BM; i.kind = 0;
  i.x = q.w + i.col0 * q.ldw; i.ldx = q.ldw; i.x_rows = __builtin_amdgcn_readfirstlane(max(0, min(q.vocab - i.col0, T::BM)));   // (a vector instruction may have made it: the loads want it in a scalar register)
  i.w = op; i.w_n = n_pad; i.w_planes = i.ksteps = q.d / BK; i.w_row = i.row0;
  return i;
}

// (max, sum of exponentials) of each row and group of vocabulary entries; the product of the target (with inv_t) from the tile that has it.  Maxima and the target's are
// kept as the products they are, and only their differences are scaled: the largest entry's is exactly 0 at any temperature, its exponential 1, so that no
// log-probability is above 0 and a certain token's is 0.  (A scaled maximum is rounded, by inv_t z 2^-24, and z inv_t - that is not 0.  An instruction a
// logit more than the multiply-add takes; us, with that / so: 4096 positions of 152064 x 3584 2807 / 2806, of 32000 x 256 118.4 / 117.4, 61 of 151936 x 1536
// 90.7 / 92.1.)
// COLD: one tile of rows, so that W is read once.
// DIRECT: few positions, which every workgroup numbers for itself and whose rows it takes as they lie, each lane from another: no launch ahead, and lanes
// without a row load nothing.  us, with the gather / so: tiny shape 14.6 / 12.1, 1.5B 4 positions 89.9 / 79.7, 32 90.3 / 87.5, 48 90.7 / 95.7; 152064 x
// 5120 4 positions 273 / 242 (6.4 TB/s), 32 273 / 273.
constexpr int DIRECT_MOST = 32;
template <int WM, int WN, int AT, int BT, bool COLD, bool DIRECT>
__global__ __launch_bounds__(256) void loss_forward_kernel(Head q, Positions at, const bf16_t *__restrict__ op, const Row *__restrict__ info, float2 *__restrict__ parts,
                                                           float2 *__restrict__ zt, int first, int n_pad) {
  typedef Tile<WM, WN, AT, BT, COLD, TILE_COLS, DIRECT> T;
  __shared__ __attribute__((aligned(1024))) bf16_t xs[T::LDS + (DIRECT ? 128 : 0)];
  int count;
  T t;
  t.init_at(xs);
  float inv_ts[BT];
  int target[BT];
  if constexpr (DIRECT) {
    typedef __attribute__((address_space(3))) int32_t lds_int;
    lds_int *mine = (lds_int *)(xs + T::LDS);
    const bool in = t.l < at.n, has = in && (uint32_t)at.target[in ? t.l : 0] < (uint32_t)q.vocab;
    const uint64_t mask = __ballot(has);
    const int number = __popcll(mask & (((uint64_t)1 << t.l) - 1));
    count = __popcll(mask);
    if (t.wave == 0) {
      if (has) mine[number] = t.l;
      if (blockIdx.x == 0) {
        if (in) at.note(t.l, has, number);
        if (t.l == 0) at.cut->count = count;
      }
    }
    __syncthreads();
    t.rows_w(q.h, (int)(((at.n - 1) * q.ldh + q.d) * 2));
#pragma unroll
    for (int b = 0; b < BT; ++b) {
      const int r = (t.wn * BT + b) * 32 + t.lrow, row = r < count ? mine[r] : -1;
      t.row_w(b, row < 0 ? -1 : (int)(row * q.ldh));
      inv_ts[b] = temperature(row >= 0 && q.inv_t ? q.inv_t[row] : 1.f);
      target[b] = row >= 0 ? q.target[row] : -1;
    }
  } else {
    count = min(q.cut->count - first, n_pad);
  }
  if (count <= 0) return;
  LogitTiles<T::BM, T::BN> tiles;
  tiles.init(count, q.vocab);
  if (tiles.at >= tiles.end) return;
  walk(t, [] {}, [] {}, [&](Item &d) {
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
      Row row;
      if constexpr (DIRECT) { row.factor = logit_factor(inv_ts[b]); row.scale = inv_ts[b]; row.target = target[b]; }
      else row = info[r];
#pragma unroll
      for (int a = 0; a < AT; a += 2) {
        const int v = v0 + a * 32;   // a group
        float z[2][16];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) z[h][i] = t.result(a + h, b, i);
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
              if (y - t.half * 4 == h * 32 + (i >> 2) * 8 + (i & 3) && r < count) zt[r] = make_float2(z[h][i], row.scale);
        }
        float m = z[0][0];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) m = fmaxf(m, z[h][i]);
        m = with_xor32(m, OpMax{});
        const float from = m == -INFINITY ? 0.f : m;   // (a group of -inf adds nothing: its exponentials are 0)
        float s = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) s += __builtin_amdgcn_exp2f((z[h][i] - from) * row.factor);
        s = with_xor32(s, OpSum{});
        if (t.half == 0 && r < count && v < q.vocab) parts[(int64_t)(v / GROUP) * n_pad + r] = make_float2(m, s);
#ifdef __HIP_DEVICE_COMPILE__
        __builtin_amdgcn_sched_barrier(0);   // (one block's registers at a time)
#endif
      }
    }
  });
}

// The groups of JOIN_ROWS rows joined, by JOIN threads per row: each takes every JOINth group in order, then their results are joined, sixteen at a time and
// the rest, in order.  (One number of threads for every call: a row's result is to be the same in all.)
constexpr int JOIN_ROWS = 8, JOIN = 1024 / JOIN_ROWS;
__global__ __launch_bounds__(1024) void loss_merge_kernel(const float2 *__restrict__ parts, const float2 *__restrict__ zt, const int32_t *__restrict__ rows,
                                                          const Cut *__restrict__ cut, float *__restrict__ logprob, float *__restrict__ lse, int groups, int first,
                                                          int n_pad) {
  __shared__ float2 joined[JOIN][JOIN_ROWS];
  const int row = threadIdx.x % JOIN_ROWS, at = threadIdx.x / JOIN_ROWS, r = blockIdx.x * JOIN_ROWS + row, n = min(cut->count - first, n_pad);
  if ((int)blockIdx.x * JOIN_ROWS >= n) return;
  const float2 of_target = r < n ? zt[r] : make_float2(0.f, 0.f);   // its product, and inv_t
  const float factor = logit_factor(of_target.y);
  // (no entries, or none but -inf: -inf, 0; NaN stays, in the maximum or in the sum)
  auto join = [&](float &m, float &s, float2 p) {
    const float top = p.x > m || p.x != p.x ? p.x : m;
    if (top == -INFINITY) {
      s += p.y;
      return;
    }
    s = s * __builtin_amdgcn_exp2f((m - top) * factor) + p.y * __builtin_amdgcn_exp2f((p.x - top) * factor);
    m = top;
  };
  const float2 none = make_float2(-INFINITY, 0.f);
  float m = -INFINITY, s = 0.f;
  for (int g = at; g < groups; g += JOIN * 4) {
    float2 p[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) p[u] = g + u * JOIN < groups && r < n ? parts[(int64_t)(g + u * JOIN) * n_pad + r] : none;
#pragma unroll
    for (int u = 0; u < 4; ++u) join(m, s, p[u]);
  }
  joined[at][row] = make_float2(m, s);
#pragma unroll
  for (int left = JOIN / 16, many = 16; left > 0; many = left, left = left > 1 ? 1 : 0) {
    __syncthreads();
    if (at < left) {
      m = -INFINITY; s = 0.f;
      for (int i = 0; i < many; ++i) join(m, s, joined[at * many + i][row]);
    }
    __syncthreads();
    if (at < left) joined[at][row] = make_float2(m, s);
  }
  if (at || r >= n) return;
  const float l = log2f(s) * LN2;   // (s >= 1: the largest entry's own exponential)
  const int t = rows[first + r];
  lse[t] = fmaf(of_target.y, m, l);
  logprob[t] = fmaf(of_target.y, of_target.x - m, -l);
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

// Few rows: one tile of them, and G in two terms.  A product of bf16 operands rounds each entry of G by up to 2^-8, and where the sums are of few
// large entries nothing averages that out; the remainders, as so many rows more, fill k-steps and columns that would be padding.  (Error of dh and dW
// over that of their own rounding, 33 positions: 1.15 to 1.63 -> 1.00.)  More rows have the one term: many positions are what a training step averages over anyway, and a
// second would double two of the three products (4096 positions of the 7B shape: 2.4e-3 of dh's and dW's norm, 1.7e-3 of it their own rounding).
constexpr int SPLIT_MOST = 128;

// G of a piece of the vocabulary, in operand order (a row's entries are its k; rows to whole tiles, then those of the remainders).  Clears the tickets of the
// kernel behind.
template <int WM, int WN, int AT, int BT>
__global__ __launch_bounds__(256) void loss_grad_logits_kernel(Head q, const bf16_t *__restrict__ op, const Row *__restrict__ info, bf16_t *__restrict__ G_out,
                                                               int index, int n_pad, int32_t *__restrict__ tickets) {
  typedef Tile<WM, WN, AT, BT, false, TILE_COLS> T;
  constexpr bool SPLIT = T::BN <= SPLIT_MOST;
  __shared__ __attribute__((aligned(1024))) bf16_t xs[T::LDS];
  if (blockIdx.x == 0 && threadIdx.x < 16) tickets[threadIdx.x * 32] = 0;
  const Cut cut = *q.cut;
  const int count = cut.count;
  const int64_t begin = (int64_t)index * cut.piece * TILE_V;
  if (begin >= q.vocab) return;
  const int v_begin = (int)begin, width = cut.piece * TILE_V, n_rows = SPLIT ? 2 * T::BN : (count + T::BN - 1) / T::BN * T::BN;
  LogitTiles<T::BM, T::BN> tiles;
  tiles.init(count, min(width, (q.vocab - v_begin + TILE_V - 1) / TILE_V * TILE_V));   // (zeros behind the vocabulary, to a whole tile of the products)
  if (tiles.at >= tiles.end) return;
  T t;
  t.init_at(xs);
  walk(t, [] {}, [] {}, [&](Item &d) {
    if (tiles.at >= tiles.end) return false;
    int mt, vt;
    tiles.place(mt, vt);
    d = logit_item<T>(q, op, n_pad, v_begin, mt, vt);
    tiles.at += gridDim.x >> 3;
    return true;
  }, [&](const Item &c) {
    const int v0 = c.col0 + t.wm * AT * 32;
#pragma unroll
    for (int b = 0; b < BT; ++b) {
      const int m32 = (c.row0 >> 5) + t.wn * BT + b;
      const Row row = info[m32 * 32 + t.lrow];
      // lse is a rounded number: a logit within half its last place is lse, as far as that says, and the probability 1, so that a certain token has no
      // gradient however large the logits are (otherwise 1.2e-6 of g at a logit of 20, but all of it and more from 1e7 on).  The multiple of inv_t is not
      // rounded before lse is taken off.  us, by one multiply-add and an exponential / so: 4096 positions of 152064 x 3584 8618 / 8653, 777 of 151936 x 1536
      // 668 / 677, 4096 of 32000 x 256 353 / 372.
      const float near = fabsf(row.lse) * 0x1p-24f;
      const uint32_t keep = row.target < 0 ? 0u : ~0u;   // (padding is 0 whatever W holds: its logits are NaN where a weight is infinite)
#pragma unroll
      for (int a = 0; a < AT; ++a) {
        const int v = v0 + a * 32, v32 = (v - v_begin) >> 5, y = row.target - v;
        float G[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float x = fmaf(t.result(a, b, i), row.factor, -row.lse);
          G[i] = -row.scale * __builtin_amdgcn_exp2f((fabsf(x) <= near ? 0.f : x) * LOG2E);
        }
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
        auto write = [&](int block) {
          uint4 f[2];
          fragments(f, G);
#pragma unroll
          for (int k = 0; k < 2; ++k)
            *(uint4 *)((char *)G_out + fragment_place(block, v32, n_rows, k, t.half, t.lrow)) = make_uint4(f[k].x & keep, f[k].y & keep, f[k].z & keep, f[k].w & keep);
        };
        write(m32);
        if constexpr (SPLIT) {
#pragma unroll
          for (int i = 0; i < 16; ++i) G[i] -= (float)(bf16_t)G[i];
          write(m32 + T::BN / 32);
        }
#ifdef __HIP_DEVICE_COMPILE__
        __builtin_amdgcn_sched_barrier(0);   // (one block's registers at a time)
#endif
      }
    }
  });
}

struct GradParams {
  const bf16_t *G, *turned;                 // G in operand order, h^T in operand order
  float *dh32;                              // [slices][rows, to a multiple of 256][d], or null: no dh
  bf16_t *dw;                               // or null
  int32_t *tickets;                         // sixteen, 128 bytes apart, zero: eight of each kind of tile
  int index, tile_rows, low;                // the piece; rows of a tile of the kernel that made G; where the remainders' rows begin, or 0: none
};

// Tiles that the units take by tickets, from their own XCD's eighth and, when that is done, from the others'.  The first ones are dealt without a ticket,
// one to each unit whose hands `before` tiles of another kind leave empty: of tiles as long as those of dh no unit is to take a second one while
// another has none.  One thread draws; the others read what it leaves in LDS.  A ticket is asked for as a tile begins and looked at when the
// tile is nearly done.
struct Lottery {
  int32_t *tickets;   // eight, 128 bytes apart
  int n, before, asked, from;
  bool own, any;      // tickets of this XCD's eighth, of any eighth may be left
  __device__ __forceinline__ Lottery(int32_t *t, int n_, int before_) : tickets(t), n(n_), before(before_), asked(0), from(0), own(true), any(false) {
    for (int x = 0; x < 8; ++x) any |= size(x) > dealt(x);
  }
  static __device__ __forceinline__ int first(int n, int x) { return x * (n >> 3) + min(x, n & 7); }
  __device__ __forceinline__ int size(int x) const { return first(n, x + 1) - first(n, x); }
  __device__ __forceinline__ int busy(int x) const { return first(before, x + 1) - first(before, x); }   // units of an XCD that hold another tile
  __device__ __forceinline__ int dealt(int x) const { return max(0, UNITS / 8 - busy(x)); }
  __device__ __forceinline__ int draw(int x) const {
    return size(x) <= dealt(x) ? size(x) : dealt(x) + __hip_atomic_fetch_add(&tickets[x * 32], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  // a tile of another eighth, or -1: an eighth that looks unfinished is asked, and one that was finished meanwhile looks so the next time
  __device__ __forceinline__ int steal() const {
    while (any) {
      int seen[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) seen[k] = __hip_atomic_load(&tickets[((blockIdx.x + k) & 7) * 32], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      int x = -1;
#pragma unroll
      for (int k = 7; k >= 0; --k) {
        const int y = (blockIdx.x + k) & 7;
        if (dealt(y) + seen[k] < size(y)) x = y;
      }
      if (x < 0) break;
      const int i = draw(x);
      if (i < size(x)) return first(n, x) + i;
    }
    return -1;
  }
  // the first two tiles
  template <typename Place>
  __device__ __forceinline__ void begin(Place place) {
    const int x = blockIdx.x & 7, turn = (int)(blockIdx.x >> 3) - busy(x);
    from = first(n, x);
    int a = -1;
    if (turn >= 0) {
      if (turn < size(x)) a = from + turn;
    } else {
      ask();
      a = told();
    }
    place(0, a);
    ask();
    place(1, a < 0 ? -1 : told());
  }
  __device__ __forceinline__ void ask() {
    if (own) asked = draw(blockIdx.x & 7);
  }
  __device__ __forceinline__ int told() {
    if (own && asked < size(blockIdx.x & 7)) return from + asked;
    own = false;
    return steal();
  }
};

// dh += G W and dW = G^T h of a piece of the vocabulary, 256 x 256 tiles, in one launch: first those of dh, which are the longer ones, then those of dW.
__global__ __launch_bounds__(256) void loss_grad_kernel(Head q, GradParams g) {
  typedef Tile<1, 4, 8, 2, false, TILE_COLS_T> TH;
  typedef Tile<1, 4, 8, 2, false, TILE_ROWS_T> TW;
  // (one LDS object: of two the compiler would know that loads on their way to one may not be what a read of it wants, and wait for them all)
  __shared__ __attribute__((aligned(1024))) bf16_t xs[TH::LDS + 4];
  typedef __attribute__((address_space(3))) volatile int32_t lds_int;
  lds_int *drawn = (lds_int *)(xs + TH::LDS);
  const Cut cut = *q.cut;
  const int count = cut.count, nd = q.d / 256;
  const int64_t begin = (int64_t)g.index * cut.piece * TILE_V;
  if (begin >= q.vocab) return;
  const int v_begin = (int)begin, nm = cut.nm, nv = min(cut.piece, (q.vocab - v_begin + TILE_V - 1) / TILE_V), n_rows = nm * 256;
  const int g_rows = g.low ? (count > 0 ? 2 * g.low : 0) : (count + g.tile_rows - 1) / g.tile_rows * g.tile_rows;   // of G (none: all of it reads as 0)
  const int64_t g_plane = (int64_t)g_rows * 64;
  const int k_all = nv * (TILE_V / BK), k_slice = cut.slice * (TILE_V / BK);
  // the walk over one kind of tile
  auto tiles = [&](auto &t, int n, int before, int32_t *tickets, auto item, auto done) {
    Lottery lots(tickets, n, before);
    const bool draws = threadIdx.x == 0;
    if (draws) lots.begin([&](int i, int v) { drawn[i] = v; });
    __syncthreads();
    t.init_at(xs);
    int turn = 0;
    walk(t, [&] {
      if (draws) lots.ask();
    }, [&] {
      if (draws) drawn[turn] = lots.told();   // for the tile behind the next; this place was read a tile ago
    }, [&](Item &d) {
      const int i = __builtin_amdgcn_readfirstlane(drawn[turn]);
      turn ^= 1;
      if (i < 0) return false;
      d = item(i);
      return true;
    }, done);
    __syncthreads();
  };
  const int n_dh = g.dh32 ? (k_all + k_slice - 1) / k_slice * nm * nd : 0;
  if (n_dh > 0) {
    TH t;
    tiles(t, n_dh, 0, g.tickets, [&](int i) {
      Item c;
      const int dt = i % nd, rest = i / nd, mt = rest % nm, k0 = rest / nm * k_slice, v = v_begin + k0 * BK;
      c.kind = rest / nm; c.row0 = mt * 256; c.col0 = dt * 256; c.ksteps = min(k_slice, k_all - k0);
      c.x = q.w + v * q.ldw + c.col0; c.ldx = q.ldw; c.x_rows = min(q.vocab - v, c.ksteps * BK);
      c.w = g.G + k0 * g_plane; c.w_n = g_rows; c.w_planes = c.ksteps; c.w_row = c.row0;
      return c;
    }, [&](const Item &c) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int r = c.row0 + (t.wn * 2 + b) * 32 + t.lrow;
        float *o = g.dh32 + ((int64_t)c.kind * n_rows + r) * q.d + c.col0 + t.half * 4;
        if (r < count || (g.low && r >= g.low && r - g.low < count)) {
#pragma unroll
          for (int a = 0; a < 8; ++a) {
            f32x4 sum[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = v_begin > 0 ? *(const f32x4 *)(o + a * 32 + i * 8) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; ++i)
              *(f32x4 *)(o + a * 32 + i * 8) = sum[i] + f32x4{t.result(a, b, 4 * i), t.result(a, b, 4 * i + 1), t.result(a, b, 4 * i + 2), t.result(a, b, 4 * i + 3)};
#ifdef __HIP_DEVICE_COMPILE__
            __builtin_amdgcn_sched_barrier(0);   // (one block's registers at a time)
#endif
          }
        }
      }
    });
  }
  if (g.dw) {
    // G's rows behind its last tile do not exist: the last k-steps take other entries' rows in their place, against zeros of h^T
    TW t;
    tiles(t, nv * nd, n_dh, g.tickets + 8 * 32, [&](int i) {
      Item c;
      const int dt = i % nd, vt = i / nd;
      c.kind = 0; c.row0 = vt * TILE_V; c.col0 = dt * 256; c.ksteps = max(4, (g_rows / BK + 3) / 4 * 4);
      c.x = g.G + vt * 4 * g_plane; c.ldx = g_rows; c.x_rows = (nv - vt) * 4;
      c.w = g.turned; c.w_n = q.d; c.w_planes = g_rows / BK; c.w_row = c.col0;
      return c;
    }, [&](const Item &c) {
      // (the stores that fill a line behind each other: 1.5B shape, 61 / 777 positions, 393 / 669 -> 357 / 647 us)
#pragma unroll
      for (int a = 0; a < 8; ++a) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int v = v_begin + c.row0 + a * 32 + t.lrow;
          float s[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = t.result(a, b, i);
          uint4 f[2];
          fragments(f, s);
          bf16_t *o = g.dw + (int64_t)v * q.d + c.col0 + (t.wn * 2 + b) * 32 + t.half * 8;
          if (v < q.vocab) {
#pragma unroll
            for (int k = 0; k < 2; ++k) *(uint4 *)(o + k * 16) = f[k];
          }
#ifdef __HIP_DEVICE_COMPILE__
          __builtin_amdgcn_sched_barrier(0);   // (one block's registers at a time)
#endif
        }
      }
    });
  }
}

// dh of every position: the slices of its row (and of its remainders' row) added up in order and rounded, or zeros
__global__ __launch_bounds__(256) void loss_round_kernel(const float *__restrict__ dh32, bf16_t *__restrict__ dh, const int32_t *__restrict__ place,
                                                         const Cut *__restrict__ cut, int d, int low) {
  const int t = blockIdx.x, k = (blockIdx.y * 256 + threadIdx.x) * 4, r = place[t];
  if (k >= d) return;
  const int slices = cut->slices, n_pad = cut->nm * 256;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (r >= 0)
    for (int rest = 0; rest <= low; rest += low ? low : 1) {   // (the remainders' row)
      const float *at = dh32 + (int64_t)(r + rest) * d + k;
#pragma unroll 8
      for (int s = 0; s < slices; ++s) v += *(const f32x4 *)(at + (int64_t)s * n_pad * d);
    }
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
  Cut *cut;
  int32_t *rows;
  Row *info;
  bf16_t *op;
  float2 *zt, *parts;
  int n_pad, groups;
  int64_t bytes;
  ForwardSpace(void *ws, int n, int vocab, int d) {
    Carver c{(char *)ws};
    n_pad = padded(std::min(n, PIECE));
    groups = (vocab + GROUP - 1) / GROUP;
    cut = c.take<Cut>(1); rows = c.take<int32_t>(n); info = c.take<Row>(n_pad); op = c.take<bf16_t>((int64_t)n_pad * d);
    zt = c.take<float2>(n_pad); parts = c.take<float2>((int64_t)groups * n_pad);
    bytes = c.at - (char *)ws;
  }
};

// Tiles of 256 x 256 of a piece's G.  More takes fewer launches whose last tiles leave units without work (7B shape, 3328
// rows, about 750 / 1500 / 3000 / 6000 of them: 9.79 / 8.71 / 8.49 / 8.40 ms), and memory.
constexpr int GRAD_MOST = 3000;
constexpr int NUMBER_MOST = 1024;   // positions that the gather's workgroups number for themselves

struct GradSpace {
  Cut *cut;
  int32_t *tickets, *rows, *place;
  Row *info;
  bf16_t *op, *turned, *G;
  float *dh32;
  int n_pad;
  int64_t bytes;
  GradSpace(void *ws, int n, int vocab, int d) {
    Carver c{(char *)ws};
    n_pad = padded(n);
    // the most that any number of rows asks for
    int64_t g = 0, sums = 0;
    for (int rows = 256; rows <= n_pad; rows += 256) {
      g = std::max(g, (int64_t)rows * Cut::of(rows, vocab, d, d, GRAD_MOST).piece * TILE_V);
      sums = std::max(sums, (int64_t)rows * Cut::slices_most(rows / 256, d));
    }
    cut = c.take<Cut>(1); tickets = c.take<int32_t>(16 * 32); rows = c.take<int32_t>(n); place = c.take<int32_t>(n); info = c.take<Row>(n_pad);
    op = c.take<bf16_t>((int64_t)n_pad * d); turned = c.take<bf16_t>((int64_t)n_pad * d);
    G = c.take<bf16_t>(g);
    dh32 = c.take<float>(sums * d);
    bytes = c.at - (char *)ws;
  }
};
// pieces that any number of rows asks for
int grad_pieces(int n_pad, int vocab, int d, int64_t ldw) {
  const int v_tiles = (vocab + TILE_V - 1) / TILE_V;
  int most = 1;
  for (int rows = 256; rows <= n_pad; rows += 256) {
    const int piece = Cut::of(rows, vocab, d, ldw, GRAD_MOST).piece;
    most = std::max(most, (v_tiles + piece - 1) / piece);
  }
  return most;
}

// Calls f(a kernel's shape as constants, workgroups) for logits of up to n rows.  Few rows stream W: tiles of 128 entries, of which two are on a unit and
// the last ones leave fewer units without work than 256 of them do (1.5B shape, 61 positions: 110 -> 96 us).
template <typename F>
void with_shape(int n, F f) {
  using std::integral_constant;
  if (n <= 64) f(integral_constant<int, 2>{}, integral_constant<int, 2>{}, integral_constant<int, 2>{}, integral_constant<int, 1>{}, 2 * UNITS);
  else if (n <= 128) f(integral_constant<int, 2>{}, integral_constant<int, 2>{}, integral_constant<int, 2>{}, integral_constant<int, 2>{}, 2 * UNITS);
  else f(integral_constant<int, 1>{}, integral_constant<int, 4>{}, integral_constant<int, 8>{}, integral_constant<int, 2>{}, UNITS);
}

}  // namespace

int64_t token_logprob_workspace_bytes(int n, int vocab, int d) { return ForwardSpace(nullptr, n, vocab, d).bytes; }

int launch_token_logprob(const TokenLoss &p, float *logprob, float *lse, hipStream_t s) {
  const ForwardSpace w(p.workspace, p.n, p.vocab, p.d);
  const Head q{p.h, p.w, p.ldh, p.ldw, p.target, p.inv_t, nullptr, nullptr, w.rows, w.cut, p.vocab, p.d};
  const Positions at{p.target, w.cut, w.rows, nullptr, logprob, lse, p.n, p.vocab, p.d, GRAD_MOST, p.ldw};
  const bool number = p.n <= NUMBER_MOST;
  auto merge = [&](int first) {
    hipLaunchKernelGGL(loss_merge_kernel, dim3((std::min(p.n - first, w.n_pad) + JOIN_ROWS - 1) / JOIN_ROWS), dim3(1024), 0, s, w.parts, w.zt, w.rows, w.cut, logprob, lse,
                       w.groups, first, w.n_pad);
  };
  if (p.n <= DIRECT_MOST && (p.n * p.ldh + p.d) * 2 < 0x7fff0000) {   // (rows behind one 32-bit offset)
    hipLaunchKernelGGL((loss_forward_kernel<2, 2, 2, 1, true, true>), dim3(2 * UNITS), dim3(256), 0, s, q, at, w.op, w.info, w.parts, w.zt, 0, w.n_pad);
    merge(0);
    return done();
  }
  if (!number) hipLaunchKernelGGL(loss_rows_kernel, dim3(1), dim3(1024), 0, s, at);
  for (int first = 0; first < p.n; first += PIECE) {
    auto gather = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(w.n_pad / 32, p.d / 64), dim3(256), 0, s, q, at, first, w.op, (bf16_t *)nullptr, 0, w.info); };
    if (number) gather(loss_gather_kernel<true>); else gather(loss_gather_kernel<false>);
    with_shape(std::min(p.n - first, PIECE), [&](auto WM, auto WN, auto AT, auto BT, int grid) {
      auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, s, q, at, w.op, w.info, w.parts, w.zt, first, w.n_pad); };
      constexpr bool once = WM.value > 1;   // (tiles of up to 128 rows: there is one of them)
      launch(loss_forward_kernel<WM.value, WN.value, AT.value, BT.value, once, false>);
    });
    merge(first);
  }
  return done();
}

int64_t token_logprob_grad_workspace_bytes(int n, int vocab, int d) { return GradSpace(nullptr, n, vocab, d).bytes; }

int launch_token_logprob_grad(const TokenLoss &p, const float *lse, const float *g, bf16_t *dh, bf16_t *dw, hipStream_t s) {
  const GradSpace w(p.workspace, p.n, p.vocab, p.d);
  const Head q{p.h, p.w, p.ldh, p.ldw, p.target, p.inv_t, lse, g, w.rows, w.cut, p.vocab, p.d};
  const Positions at{p.target, w.cut, w.rows, w.place, nullptr, nullptr, p.n, p.vocab, p.d, GRAD_MOST, p.ldw};
  const int low = p.n <= 64 ? 64 : p.n <= SPLIT_MOST ? SPLIT_MOST : 0;   // (a tile's rows: with_shape)
  const bool number = p.n <= NUMBER_MOST;
  if (!number) hipLaunchKernelGGL(loss_rows_kernel, dim3(1), dim3(1024), 0, s, at);
  auto gather = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(w.n_pad / 32, p.d / 64), dim3(256), 0, s, q, at, 0, w.op, w.turned, low, w.info); };
  if (number) gather(loss_gather_kernel<true>); else gather(loss_gather_kernel<false>);
  const int pieces = grad_pieces(w.n_pad, p.vocab, p.d, p.ldw);
  with_shape(p.n, [&](auto WM, auto WN, auto AT, auto BT, int grid) {
    for (int i = 0; i < pieces; ++i) {
      hipLaunchKernelGGL((loss_grad_logits_kernel<WM.value, WN.value, AT.value, BT.value>), dim3(grid), dim3(256), 0, s, q, w.op, w.info, w.G, i, w.n_pad, w.tickets);
      const GradParams gp{w.G, w.turned, dh ? w.dh32 : nullptr, dw, w.tickets, i, WN.value * BT.value * 32, low};
      hipLaunchKernelGGL(loss_grad_kernel, dim3(UNITS), dim3(256), 0, s, q, gp);
    }
  });
  if (dh)
    hipLaunchKernelGGL(loss_round_kernel, dim3(p.n, (p.d / 4 + 255) / 256), dim3(256), 0, s, w.dh32, dh, w.place, w.cut, p.d, low);
  return done();
}

}  // namespace pl
