// Products in 8-bit integers: y = x W^T with a scale per row of x (token) and per row of W (channel).
//
// Quantisation of a row: scale = max |x| / 127 in fp32, code = the integer nearest to x / scale (ties to even), at most 127 in magnitude.  The
// quotient is rounded as if exact: the product is then the same for every implementation of that sentence.  Codes are multiplied and added up
// in int32 without error (127^2 K < 2^31), and a result is (float(sum) * scale of its token) * scale of its channel.
#include "pl_common.h"

namespace pl {
namespace {

// The integer nearest to x / s (ties to even; clamped): the rounded quotient may be one off next to a tie, and its remainder says so.  x - q s is
// exact: a multiple of the last place of s (of x where x is the smaller) and no larger than 2 s.
__device__ inline int quotient(float x, float s, float inv) {
  float q = fminf(fmaxf(rintf(x * inv), -127.f), 127.f);
  const float r = fmaf(-q, s, x), h = 0.5f * s;
  if (r > h || (r == h && ((int)q & 1))) q += 1.f;
  if (r < -h || (r == -h && ((int)q & 1))) q -= 1.f;
  return (int)fminf(fmaxf(q, -127.f), 127.f);
}

__device__ inline float value(const bf16_t *x, int64_t i) { return (float)x[i]; }
__device__ inline float value(const float *x, int64_t i) { return x[i]; }

// place of code (row, k) in an operand-ordered image of N rows: blocks of 32 rows x 128 k, k-block-major
__device__ inline int64_t operand_place(int row, int k, int N) {
  const int half = (k >> 6) & 1, j = (k >> 4) & 3;
  return (((int64_t)(k >> 7) * (N >> 5) + (row >> 5)) * 4 + j) * 1024 + (half * 32 + (row & 31)) * 16 + (k & 15);
}

template <typename T, bool OPERAND>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T *__restrict__ x, int64_t ldx, int8_t *__restrict__ q, float *__restrict__ scale, int N, int K) {
  const int row = blockIdx.x;
  x += row * ldx;
  __shared__ float part[4];
  float m = 0.f;
  bool odd = false;
  for (int k = threadIdx.x; k < K; k += 256) {
    const float a = fabsf(value(x, k));
    odd |= !(a < INFINITY);
    m = fmaxf(m, a);
  }
  m = wave_max(m);
  if (__ballot(odd)) m = INFINITY;
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
  const bool fine = m < INFINITY;
  const float s = m / 127.f, up = s < 0x1p-100f ? 0x1p100f : 1.f;   // (tiny rows: both sides times a power of two, so that 1 / s is finite)
  const float inv = fine && s > 0.f ? 1.f / (s * up) : 0.f;
  if (threadIdx.x == 0) scale[row] = fine ? s : NAN;
  for (int k = threadIdx.x; k < K; k += 256) {
    const int c = inv > 0.f ? quotient(value(x, k) * up, s * up, inv) : 0;
    q[OPERAND ? operand_place(row, k, N) : (int64_t)row * K + k] = (int8_t)c;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void gemm_int8_kernel(const int8_t *__restrict__ xq, const float *__restrict__ sx, const int8_t *__restrict__ wq,
                                                        const float *__restrict__ sw, T *__restrict__ y, int M, int N, int K) {
  const int n = blockIdx.x * 256 + threadIdx.x, m = blockIdx.y;
  if (n >= N) return;
  int32_t sum = 0;
  for (int k = 0; k < K; k += 16) {
    const int8_t *w = wq + operand_place(n, k, N), *x = xq + (int64_t)m * K + k;
    for (int e = 0; e < 16; ++e) sum += (int)x[e] * (int)w[e];
  }
  y[(int64_t)m * N + n] = (T)((float)sum * sx[m] * sw[n]);
}

}  // namespace

int launch_quantize_int8(const void *w, bool f32, int64_t ldw, int8_t *q, float *scale, int N, int K, hipStream_t s) {
  if (f32) hipLaunchKernelGGL((quantize_rows_kernel<float, true>), dim3(N), dim3(256), 0, s, (const float *)w, ldw, q, scale, N, K);
  else hipLaunchKernelGGL((quantize_rows_kernel<bf16_t, true>), dim3(N), dim3(256), 0, s, (const bf16_t *)w, ldw, q, scale, N, K);
  return hipGetLastError() == hipSuccess ? 0 : -7;
}

int64_t gemm_int8_workspace_bytes(int M, int N, int K) { return ((int64_t)M * 4 + 255) / 256 * 256 + (int64_t)M * K; }

int launch_gemm_int8(const bf16_t *x, int64_t ldx, const int8_t *wq, const float *sw, void *y, bool f32, int M, int N, int K, void *ws, hipStream_t s) {
  float *sx = (float *)ws;
  int8_t *xq = (int8_t *)ws + ((int64_t)M * 4 + 255) / 256 * 256;
  hipLaunchKernelGGL((quantize_rows_kernel<bf16_t, false>), dim3(M), dim3(256), 0, s, x, ldx, xq, sx, M, K);
  const dim3 grid((N + 255) / 256, M);
  if (f32) hipLaunchKernelGGL(gemm_int8_kernel<float>, grid, dim3(256), 0, s, xq, sx, wq, sw, (float *)y, M, N, K);
  else hipLaunchKernelGGL(gemm_int8_kernel<bf16_t>, grid, dim3(256), 0, s, xq, sx, wq, sw, (bf16_t *)y, M, N, K);
  return hipGetLastError() == hipSuccess ? 0 : -7;
}

}  // namespace pl
