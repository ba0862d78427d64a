// Dense projection: z = x W^T + bias, y = residual + act(z); gradients dx = dz W, dw = dz^T x, dbias = sum of dz's rows.
// One kernel of 64 x 64 tiles, fp32 FMAs on operands of any strides, serves the three products.
#include <algorithm>

#include "rr_device.h"

namespace rr {

namespace {

constexpr int LN_TILE = 64, LN_K = 16, LN_THREADS = 256;

// C[m, n] = sum_k A[m, k] B[n, k], operands with strides in elements.
struct LinearArgs {
  const void *A, *B;
  long long am, ak, bn, bk;
  int M, N, K;
  const float *bias;     // epilogue
  const void *residual;
  void *out, *pre;
  int act, Nout;         // RR_ACT_SWIGLU: column n < Nout of B is the gate's, n + Nout the up projection's
};

template <bool BF16>
__device__ inline float load_value(const void *p, long long i) {
  if (BF16) return __builtin_bit_cast(float, (u32) static_cast<const uint16_t *>(p)[i] << 16);
  return static_cast<const float *>(p)[i];
}
template <bool BF16>
__device__ inline void store_value(void *p, long long i, float v) {
  if (BF16) static_cast<uint16_t *>(p)[i] = (uint16_t)pack_bf16(v, 0.0f);
  else static_cast<float *>(p)[i] = v;
}

template <bool BF16, bool GATED>
__global__ __launch_bounds__(LN_THREADS) void linear_tile_kernel(LinearArgs P) {
  constexpr int NB = GATED ? 2 : 1;
  __shared__ float a[LN_K][LN_TILE + 1], b[NB][LN_K][LN_TILE + 1];
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const int m0 = blockIdx.y * LN_TILE, n0 = blockIdx.x * LN_TILE;
  float acc[NB][4][4] = {};
  for (int k0 = 0; k0 < P.K; k0 += LN_K) {
    for (int i = tid; i < LN_K * LN_TILE; i += LN_THREADS) {
      const int r = i / LN_K, k = i % LN_K;
      const bool kin = k0 + k < P.K;
      a[k][r] = kin && m0 + r < P.M ? load_value<BF16>(P.A, (m0 + r) * P.am + (k0 + k) * P.ak) : 0.0f;
#pragma unroll
      for (int q = 0; q < NB; ++q)
        b[q][k][r] = kin && n0 + r < P.N ? load_value<BF16>(P.B, (long long)(n0 + r + q * P.Nout) * P.bn + (k0 + k) * P.bk) : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < LN_K; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int q = 0; q < NB; ++q) acc[q][i][j] = fmaf(a[k][ty + 16 * i], b[q][k][tx + 16 * j], acc[q][i][j]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
      if (m >= P.M || n >= P.N) continue;
      float z[NB];
#pragma unroll
      for (int q = 0; q < NB; ++q) {
        z[q] = acc[q][i][j] + (P.bias ? P.bias[n + q * P.Nout] : 0.0f);
        if (P.pre) store_value<BF16>(P.pre, (long long)m * NB * P.Nout + n + q * P.Nout, z[q]);
      }
      float y = z[0];
      if (GATED) y = z[0] / (1.0f + expf(-z[0])) * z[NB - 1];
      else if (P.act == RR_ACT_GELU) y = gelu_erf(z[0]);
      const long long at = (long long)m * P.N + n;
      if (P.residual) y += load_value<BF16>(P.residual, at);
      store_value<BF16>(P.out, at, y);
    }
}

// dz = dy act'(z) and, per 64 columns, the column sums.
template <bool BF16>
__global__ __launch_bounds__(256) void linear_dz_kernel(const void *dy, const void *pre, int act, int M, int N, void *dz, float *dbias) {
  __shared__ double sums[2][4][kWave];
  const int lane = threadIdx.x & 63, part = threadIdx.x >> 6, n = blockIdx.x * kWave + lane;
  const bool gated = act == RR_ACT_SWIGLU;
  const int R = gated ? 2 * N : N;
  double s0 = 0.0, s1 = 0.0;
  if (n < N)
    for (int m = part; m < M; m += 4) {
      const float d = load_value<BF16>(dy, (long long)m * N + n);
      float g = d, u = 0.0f;
      if (act != RR_ACT_NONE) {
        const float z = load_value<BF16>(pre, (long long)m * R + n);
        if (gated) {
          const float up = load_value<BF16>(pre, (long long)m * R + N + n), t = 1.0f / (1.0f + expf(-z));
          g = d * up * t * (1.0f + z * (1.0f - t));
          u = d * z * t;
          if (dz) store_value<BF16>(dz, (long long)m * R + N + n, u);
        } else {
          g = d * (0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * 0.39894228040143268f * expf(-0.5f * z * z));
        }
        if (dz) store_value<BF16>(dz, (long long)m * R + n, g);
      }
      s0 += g;
      s1 += u;
    }
  sums[0][part][lane] = s0;
  sums[1][part][lane] = s1;
  __syncthreads();
  if (part > 0 || n >= N || !dbias) return;
  s0 = s1 = 0.0;
  for (int q = 0; q < 4; ++q) {
    s0 += sums[0][q][lane];
    s1 += sums[1][q][lane];
  }
  dbias[n] = (float)s0;
  if (gated) dbias[N + n] = (float)s1;
}

void launch_tile(bool bf16, bool gated, const LinearArgs &A, hipStream_t s) {
  const dim3 grid((A.N + LN_TILE - 1) / LN_TILE, (A.M + LN_TILE - 1) / LN_TILE);
  if (bf16 && gated) linear_tile_kernel<true, true><<<grid, LN_THREADS, 0, s>>>(A);
  else if (bf16) linear_tile_kernel<true, false><<<grid, LN_THREADS, 0, s>>>(A);
  else if (gated) linear_tile_kernel<false, true><<<grid, LN_THREADS, 0, s>>>(A);
  else linear_tile_kernel<false, false><<<grid, LN_THREADS, 0, s>>>(A);
}

int width(const rr_linear_config &c) { return c.act == RR_ACT_SWIGLU ? 2 * c.N : c.N; }

}  // namespace

size_t linear_workspace(const rr_linear_config &c, bool backward) {
  if (!backward || c.act == RR_ACT_NONE) return 256;
  return ((size_t)c.M * width(c) * (c.dtype == RR_BF16 ? 2 : 4) + 255) / 256 * 256;
}

hipError_t launch_linear(const rr_linear_config &c, const void *x, const void *w, const float *bias, const void *residual, void *y,
                         void *pre, void *, hipStream_t s) {
  const LinearArgs A{x, w, c.K, 1, c.K, 1, c.M, c.N, c.K, bias, residual, y, pre, c.act, c.N};
  prof_begin(K_LINEAR, s);
  launch_tile(c.dtype == RR_BF16, c.act == RR_ACT_SWIGLU, A, s);
  prof_end(K_LINEAR, s);
  return hipGetLastError();
}

hipError_t launch_linear_backward(const rr_linear_config &c, const void *x, const void *w, const void *pre, const void *dy, void *dx,
                                  void *dw, float *dbias, void *ws, hipStream_t s) {
  const bool bf16 = c.dtype == RR_BF16;
  const int R = width(c);
  const bool products = dx || dw;
  const void *dz = c.act == RR_ACT_NONE ? dy : ws;
  prof_begin(K_LINEAR_BWD, s);
  if (dbias || (products && c.act != RR_ACT_NONE)) {
    const dim3 grid((c.N + kWave - 1) / kWave);
    if (bf16) linear_dz_kernel<true><<<grid, 256, 0, s>>>(dy, pre, c.act, c.M, c.N, products ? ws : nullptr, dbias);
    else linear_dz_kernel<false><<<grid, 256, 0, s>>>(dy, pre, c.act, c.M, c.N, products ? ws : nullptr, dbias);
  }
  if (dx) launch_tile(bf16, false, LinearArgs{dz, w, R, 1, 1, c.K, c.M, c.K, R, nullptr, nullptr, dx, nullptr, RR_ACT_NONE, c.K}, s);
  if (dw) launch_tile(bf16, false, LinearArgs{dz, x, 1, R, 1, c.K, R, c.K, c.M, nullptr, nullptr, dw, nullptr, RR_ACT_NONE, c.K}, s);
  prof_end(K_LINEAR_BWD, s);
  return hipGetLastError();
}

}  // namespace rr
