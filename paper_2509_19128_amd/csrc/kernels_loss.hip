// Log-probabilities of given tokens under an LM head, and their gradient, without logits in memory.
//
//   z[t, v] = inv_t[t] * sum_k h[t, k] W[v, k],  lse[t] = log sum_v exp z[t, v],  logprob[t] = z[t, y_t] - lse[t]
//   G[t, v] = g[t] inv_t[t] (1[v = y_t] - exp(z[t, v] - lse[t])),  dh = G W,  dW = G^T h
//
// The vocabulary is walked in groups of 64 rows of W: a group leaves (max, sum of exponentials) per position, joined in order by a second
// kernel.  The gradient takes the vocabulary in chunks: G of a chunk goes to memory, then both products read it.
// Positions without a target are left out from the start: the others are numbered, and every kernel works on those.
#include "pl_common.h"

#include <algorithm>

namespace pl {
namespace {

constexpr int GROUP = 64;   // vocabulary rows of a partial sum

// positions with a target in order, their number, and zeros for the others
__global__ __launch_bounds__(1024) void loss_rows_kernel(const int32_t *__restrict__ target, int32_t *__restrict__ count, int32_t *__restrict__ rows,
                                                         float *__restrict__ logprob, float *__restrict__ lse, int n, int vocab) {
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
    if (has) rows[at + __popcll(mask & (((uint64_t)1 << lane) - 1))] = t;
    else if (in && logprob) logprob[t] = lse[t] = 0.f;
    base += all;
    __syncthreads();
  }
  if (threadIdx.x == 0) *count = base;
}

// C[i][j] = sum_k a(i, k) b(j, k) of a 64 x 64 tile; a thread ends with i = ty * 4 .. + 3, j = tx * 4 .. + 3
template <typename A, typename B>
__device__ void tile64(float (&c)[4][4], int K, A a, B b) {
  __shared__ float as[16][65], bs[16][65];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) c[i][j] = 0.f;
  for (int k0 = 0; k0 < K; k0 += 16) {
    for (int e = threadIdx.x; e < 1024; e += 256) {
      as[e & 15][e >> 4] = k0 + (e & 15) < K ? a(e >> 4, k0 + (e & 15)) : 0.f;
      bs[e & 15][e >> 4] = k0 + (e & 15) < K ? b(e >> 4, k0 + (e & 15)) : 0.f;
    }
    __syncthreads();
    for (int k = 0; k < 16; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) c[i][j] = fmaf(as[k][ty * 4 + i], bs[k][tx * 4 + j], c[i][j]);
    __syncthreads();
  }
}

struct Head {
  const bf16_t *h, *w;
  int64_t ldh, ldw;
  const int32_t *target, *rows, *count;
  const float *inv_t;
  int vocab, d;
};

// the logits of 64 vocabulary rows (ty) and 64 positions (tx)
__device__ void logits64(const Head &q, float (&c)[4][4], int v0, int r0) {
  const int count = *q.count;
  tile64(c, q.d, [&](int i, int k) { return v0 + i < q.vocab ? (float)q.w[(v0 + i) * q.ldw + k] : 0.f; },
         [&](int j, int k) { return r0 + j < count ? (float)q.h[q.rows[r0 + j] * q.ldh + k] : 0.f; });
  for (int j = 0; j < 4; ++j) {
    const int r = r0 + (threadIdx.x & 15) * 4 + j;
    const float it = r < count && q.inv_t ? q.inv_t[q.rows[r]] : 1.f;
    for (int i = 0; i < 4; ++i) c[i][j] *= it;
  }
}

__global__ __launch_bounds__(256) void logprob_kernel(Head q, float2 *__restrict__ parts, float *__restrict__ zt, int n) {
  const int v0 = blockIdx.x * GROUP, r0 = blockIdx.y * 64, count = *q.count;
  if (r0 >= count) return;
  __shared__ float zs[64][65];
  float c[4][4];
  logits64(q, c, v0, r0);
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) zs[(threadIdx.x >> 4) * 4 + i][(threadIdx.x & 15) * 4 + j] = c[i][j];
  __syncthreads();
  const int r = r0 + threadIdx.x, nv = min(GROUP, q.vocab - v0);
  if (threadIdx.x >= 64 || r >= count) return;
  float m = -INFINITY, s = 0.f;
  for (int i = 0; i < nv; ++i) m = fmaxf(m, zs[i][threadIdx.x]);
  for (int i = 0; i < nv; ++i) s += expf(zs[i][threadIdx.x] - m);
  parts[(int64_t)blockIdx.x * n + r] = make_float2(m, s);
  const int y = q.target[q.rows[r]] - v0;
  if (y >= 0 && y < nv) zt[r] = zs[y][threadIdx.x];
}

__global__ __launch_bounds__(64) void logprob_merge_kernel(const float2 *__restrict__ parts, const float *__restrict__ zt, const int32_t *__restrict__ rows,
                                                           const int32_t *__restrict__ count, float *__restrict__ logprob, float *__restrict__ lse, int groups, int n) {
  const int r = blockIdx.x * 64 + threadIdx.x;
  if (r >= *count) return;
  float m = -INFINITY, s = 0.f;
  for (int g = 0; g < groups; ++g) m = fmaxf(m, parts[(int64_t)g * n + r].x);
  for (int g = 0; g < groups; ++g) {
    const float2 p = parts[(int64_t)g * n + r];
    s += p.y * expf(p.x - m);
  }
  const float l = m + logf(s);
  lse[rows[r]] = l;
  logprob[rows[r]] = zt[r] - l;
}

// G of vocabulary rows [v_begin, v_begin + width), bf16 [count][width]
__global__ __launch_bounds__(256) void grad_logits_kernel(Head q, const float *__restrict__ lse, const float *__restrict__ g, bf16_t *__restrict__ G, int v_begin, int width) {
  const int v0 = v_begin + blockIdx.x * 64, r0 = blockIdx.y * 64, count = *q.count;
  if (r0 >= count) return;
  float c[4][4];
  logits64(q, c, v0, r0);
  for (int j = 0; j < 4; ++j) {
    const int r = r0 + (threadIdx.x & 15) * 4 + j;
    if (r >= count) continue;
    const int t = q.rows[r];
    const float gt = q.inv_t ? g[t] * q.inv_t[t] : g[t];
    for (int i = 0; i < 4; ++i) {
      const int v = v0 + (threadIdx.x >> 4) * 4 + i;
      if (v < min(q.vocab, v_begin + width)) G[(int64_t)r * width + (v - v_begin)] = (bf16_t)(gt * ((v == q.target[t] ? 1.f : 0.f) - expf(c[i][j] - lse[t])));
    }
  }
}

// dh[r] += G W over a chunk
__global__ __launch_bounds__(256) void grad_h_kernel(Head q, const bf16_t *__restrict__ G, float *__restrict__ dh32, int v_begin, int width, bool first) {
  const int d0 = blockIdx.x * 64, r0 = blockIdx.y * 64, count = *q.count, nv = min(width, q.vocab - v_begin);
  if (r0 >= count) return;
  float c[4][4];
  tile64(c, nv, [&](int i, int k) { return r0 + i < count ? (float)G[(int64_t)(r0 + i) * width + k] : 0.f; },
         [&](int j, int k) { return (float)q.w[(v_begin + k) * q.ldw + d0 + j]; });
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int r = r0 + (threadIdx.x >> 4) * 4 + i;
      float *o = dh32 + (int64_t)r * q.d + d0 + (threadIdx.x & 15) * 4 + j;
      if (r < count) *o = first ? c[i][j] : *o + c[i][j];
    }
}

// dW rows of a chunk
__global__ __launch_bounds__(256) void grad_w_kernel(Head q, const bf16_t *__restrict__ G, bf16_t *__restrict__ dw, int v_begin, int width) {
  const int d0 = blockIdx.x * 64, i0 = blockIdx.y * 64, count = *q.count, nv = min(width, q.vocab - v_begin);
  float c[4][4];
  tile64(c, count, [&](int i, int k) { return i0 + i < nv ? (float)G[(int64_t)k * width + i0 + i] : 0.f; },
         [&](int j, int k) { return (float)q.h[q.rows[k] * q.ldh + d0 + j]; });
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int v = i0 + (threadIdx.x >> 4) * 4 + i;
      if (v < nv) dw[(int64_t)(v_begin + v) * q.d + d0 + (threadIdx.x & 15) * 4 + j] = (bf16_t)c[i][j];
    }
}

__global__ __launch_bounds__(256) void clear_rows_kernel(bf16_t *__restrict__ dh, const int32_t *__restrict__ target, int d, int vocab) {
  if ((uint32_t)target[blockIdx.x] < (uint32_t)vocab) return;
  for (int k = threadIdx.x; k < d; k += 256) dh[(int64_t)blockIdx.x * d + k] = (bf16_t)0.f;
}
__global__ __launch_bounds__(256) void round_rows_kernel(const float *__restrict__ dh32, bf16_t *__restrict__ dh, const int32_t *__restrict__ rows,
                                                         const int32_t *__restrict__ count, int d) {
  if ((int)blockIdx.x >= *count) return;
  for (int k = threadIdx.x; k < d; k += 256) dh[(int64_t)rows[blockIdx.x] * d + k] = (bf16_t)dh32[(int64_t)blockIdx.x * d + k];
}

int64_t align256(int64_t b) { return (b + 255) / 256 * 256; }
int chunk_width(int n, int vocab) { return std::min((vocab + 255) / 256, std::max(1, (int)(((int64_t)64 << 20) / n / 256))) * 256; }
int done() { return hipGetLastError() == hipSuccess ? 0 : -7; }

}  // namespace

int64_t token_logprob_workspace_bytes(int n, int vocab, int d) {
  const int64_t groups = (vocab + GROUP - 1) / GROUP;
  return 256 + align256((int64_t)n * 4) * 2 + groups * n * 8;
}

int launch_token_logprob(const TokenLoss &p, float *logprob, float *lse, hipStream_t s) {
  char *ws = (char *)p.workspace;
  int32_t *count = (int32_t *)ws, *rows = (int32_t *)(ws + 256);
  float *zt = (float *)(ws + 256 + align256((int64_t)p.n * 4));
  float2 *parts = (float2 *)(ws + 256 + align256((int64_t)p.n * 4) * 2);
  const int groups = (p.vocab + GROUP - 1) / GROUP;
  const Head q{p.h, p.w, p.ldh, p.ldw, p.target, rows, count, p.inv_t, p.vocab, p.d};
  hipLaunchKernelGGL(loss_rows_kernel, dim3(1), dim3(1024), 0, s, p.target, count, rows, logprob, lse, p.n, p.vocab);
  hipLaunchKernelGGL(logprob_kernel, dim3(groups, (p.n + 63) / 64), dim3(256), 0, s, q, parts, zt, p.n);
  hipLaunchKernelGGL(logprob_merge_kernel, dim3((p.n + 63) / 64), dim3(64), 0, s, parts, zt, rows, count, logprob, lse, groups, p.n);
  return done();
}

int64_t token_logprob_grad_workspace_bytes(int n, int vocab, int d) {
  return 256 + align256((int64_t)n * 4) + align256((int64_t)n * d * 4) + (int64_t)n * chunk_width(n, vocab) * 2;
}

int launch_token_logprob_grad(const TokenLoss &p, const float *lse, const float *g, bf16_t *dh, bf16_t *dw, hipStream_t s) {
  char *ws = (char *)p.workspace;
  int32_t *count = (int32_t *)ws, *rows = (int32_t *)(ws + 256);
  float *dh32 = (float *)(ws + 256 + align256((int64_t)p.n * 4));
  bf16_t *G = (bf16_t *)(ws + 256 + align256((int64_t)p.n * 4) + align256((int64_t)p.n * p.d * 4));
  const int width = chunk_width(p.n, p.vocab), rt = (p.n + 63) / 64;
  const Head q{p.h, p.w, p.ldh, p.ldw, p.target, rows, count, p.inv_t, p.vocab, p.d};
  hipLaunchKernelGGL(loss_rows_kernel, dim3(1), dim3(1024), 0, s, p.target, count, rows, (float *)nullptr, (float *)nullptr, p.n, p.vocab);
  for (int v = 0; v < p.vocab; v += width) {
    hipLaunchKernelGGL(grad_logits_kernel, dim3(width / 64, rt), dim3(256), 0, s, q, lse, g, G, v, width);
    if (dh) hipLaunchKernelGGL(grad_h_kernel, dim3(p.d / 64, rt), dim3(256), 0, s, q, G, dh32, v, width, v == 0);
    if (dw) hipLaunchKernelGGL(grad_w_kernel, dim3(p.d / 64, width / 64), dim3(256), 0, s, q, G, dw, v, width);
  }
  if (dh) {
    hipLaunchKernelGGL(clear_rows_kernel, dim3(p.n), dim3(256), 0, s, dh, p.target, p.d, p.vocab);
    hipLaunchKernelGGL(round_rows_kernel, dim3(p.n), dim3(256), 0, s, dh32, dh, rows, count, p.d);
  }
  return done();
}

}  // namespace pl
