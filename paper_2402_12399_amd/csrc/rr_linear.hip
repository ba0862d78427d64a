// Dense projection: z = x W^T + bias, y = residual + act(z); gradients dx = dz W, dw = dz^T x, dbias = sum of dz's rows.
//
// Every product is "A[rows, K] times B[N, K]^T" with K contiguous in both operands (rr_gemm.h):
//   forward  x, W                 dx  dz, W^T                 dw  dz^T, x^T
// bf16 tiles, and fp32 tiles that split their operands, read those of the gradients as they lie in memory ("turned" operands); for
// other fp32 kernels linear_turn_kernel writes the transposes.  It also makes dz from dy and the stored z, and sums its columns.
// Which kernel multiplies is a matter of estimated time (dense_plan): 256 x 256 tiles of the persistent kernel, smaller
// tiles, either with the summation cut into slices where the tiles alone would leave CUs idle (each slice's raw sums go
// to the workspace and linear_join_kernel adds them in order and does the epilogue), or, up to kFewRows rows,
// linear_rows_kernel.
#include "rr_gemm.h"

namespace rr {

namespace {

int width(const rr_linear_config &c) { return c.act == RR_ACT_SWIGLU ? 2 * c.N : c.N; }
int element(const rr_linear_config &c) { return c.dtype == RR_BF16 ? 2 : 4; }
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

template <bool BF16>
__device__ inline float load_value(const void *p, size_t i) {
  if (BF16) return __builtin_bit_cast(float, (u32) static_cast<const uint16_t *>(p)[i] << 16);
  return static_cast<const float *>(p)[i];
}

template <bool BF16>
__device__ inline void store_value(void *p, size_t i, float v) {
  if (BF16) static_cast<uint16_t *>(p)[i] = (uint16_t)pack_bf16(v, 0.0f);
  else static_cast<float *>(p)[i] = v;
}

// ------------------------------------------------------------------ few rows
// Up to kFewRows rows: the weights are read once and everything else is small.  A workgroup owns 16 columns (gated: of both
// halves of W), its waves take turns at chunks of 64 (fp32: 32) elements of the rows and load fragments straight from
// global memory, without LDS, chunks ahead; the waves' sums are added through LDS in order.
constexpr int kFewRows = 32;
constexpr int LR_NW = 8, LR_THREADS = LR_NW * 64;
[[maybe_unused]] constexpr int LR_AHEAD = 2;

template <bool BF16, bool GATED, int ACT, int MF>
__global__ __launch_bounds__(LR_THREADS, 4) void linear_rows_kernel(DenseArgs P) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int ES = BF16 ? 2 : 4, NB = GATED ? 2 : 1, CHUNK = 128;  // bytes of a row
  using Frag = typename std::conditional<BF16, bf16x8, f32x4>::type;
  __shared__ f32x4 red[LR_NW][MF * NB][64];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 15, q = lane >> 4;
  const int N = P.N, n0 = blockIdx.x * 16;
  const unsigned rowb = (unsigned)P.K * ES;
  const int chunks = (int)((rowb + CHUNK - 1) / CHUNK);
  auto rsrc = [](const void *base, size_t off, size_t range) {
    return __builtin_amdgcn_make_buffer_rsrc(static_cast<char *>(const_cast<void *>(base)) + off, 0,
                                             __builtin_amdgcn_readfirstlane((int)range), BUF_FLAGS);
  };
  // rows past the last one and pieces past a row's end read as zero
  const __amdgpu_buffer_rsrc_t rsA = rsrc(P.A, 0, (size_t)P.M * rowb);
  const size_t wrows = (size_t)min(16, N - n0) * rowb;
  const __amdgpu_buffer_rsrc_t rsB[2] = {rsrc(P.B0, (size_t)n0 * rowb, wrows), GATED ? rsrc(P.B1, (size_t)n0 * rowb, wrows) : rsA};
  constexpr unsigned PAST = 0x7ffffff0u;
  auto load = [](const __amdgpu_buffer_rsrc_t &rs, unsigned off) {
    return __builtin_bit_cast(Frag, __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0));
  };
  f32x4 acc[MF][NB];
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  Frag a[LR_AHEAD][2][MF], b[LR_AHEAD][2][NB];
  auto fetch = [&](int c, int slot) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const unsigned at = (unsigned)c * CHUNK + h * 64 + q * 16;
      const bool in = c < chunks && at < rowb;
#pragma unroll
      for (int j = 0; j < NB; ++j) b[slot][h][j] = load(rsB[j], in ? r * rowb + at : PAST);
#pragma unroll
      for (int i = 0; i < MF; ++i) a[slot][h][i] = load(rsA, in && i * 16 + r < P.M ? (i * 16 + r) * rowb + at : PAST);
    }
  };
#pragma unroll
  for (int s = 0; s < LR_AHEAD; ++s) {
    fetch(w + s * LR_NW, s);
    __builtin_amdgcn_sched_barrier(0);  // in this order, or the loop below waits for all of them at once (16 x 4096 -> 2 x 4096 16.8 us, 15.7 so)
  }
  for (int c = w; c < chunks; c += LR_AHEAD * LR_NW) {
#pragma unroll
    for (int s = 0; s < LR_AHEAD; ++s) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j) {
            // B fragment first, as in the other kernels: lane owns row (lane & 15), columns 4 * (lane >> 4) .. + 3
            if constexpr (BF16) {
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[s][h][j], a[s][h][i], acc[i][j], 0, 0, 0);
            } else {
#pragma unroll
              for (int u = 0; u < 4; ++u)
                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[s][h][j][u], a[s][h][i][u], acc[i][j], 0, 0, 0);
            }
          }
      fetch(c + (LR_AHEAD + s) * LR_NW, s);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int i = 0; i < MF; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) red[w][i * NB + j][lane] = acc[i][j];
  __syncthreads();
  if (w >= MF) return;
  f32x4 sum[1][NB];
#pragma unroll
  for (int j = 0; j < NB; ++j) {
    sum[0][j] = red[0][w * NB + j][lane];
#pragma unroll
    for (int s = 1; s < LR_NW; ++s) sum[0][j] += red[s][w * NB + j][lane];
  }
  store_dense<1, NB, 16, BF16, GATED, ACT>(sum, P, 0, w * 16 + r, P.M, n0, lane);
#endif
}

// ------------------------------------------------------------------ one to four rows
// As many dot products per row of W as there are rows of x: a wave takes VR rows of W (gated: VR / 2 of each half), a lane 16
// bytes of each in every chunk of 1 KB, and the lanes' sums are added at the end.  Every wave reads whole rows, so that
// also a narrow W is spread over the chip (16 columns a workgroup in the kernel above: 8192 -> 1024 fills 64 CUs).  Each row of W is met by all of
// x, out of the caches: from 3 rows of bf16 on the other kernels are faster (4 rows, 4096 -> 2 x 11008 41.6 -> 35.4 us, 11008 -> 4096 23.4 -> 18.8;
// 3 rows 36.3 -> 35.5, 9.1 -> 8.5 for 4096 -> 4096, though 8192 -> 1024 7.6 -> 8.2), from 5 of fp32 (4 rows, 4096 -> 4096 16.1 here, 18.1 there).
// W streams past the caches (see launch_dense_tiles): one row, 4096 -> 2 x 11008 30.5 -> 27.3 us (6.6 TB/s), 11008 -> 4096 20.4 -> 18.0; fp32
// 4096 -> 4096 13.8 -> 12.4.
constexpr int kVectorRows(bool bf16) { return bf16 ? 2 : 4; }
constexpr int LV_THREADS = 256, LV_ROWS = 2;
[[maybe_unused]] constexpr int LV_AHEAD = 4;

template <bool BF16, bool GATED, int ACT, int M>
__global__ __launch_bounds__(LV_THREADS) void linear_vector_kernel(DenseArgs P) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int ES = BF16 ? 2 : 4, PE = 16 / ES, VR = LV_ROWS;
  constexpr int VN = GATED ? VR / 2 : VR;  // output columns of a wave
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((blockIdx.x * LV_THREADS + threadIdx.x) >> 6);
  const int N = P.N, n0 = w * VN;
  if (n0 >= N) return;
  const unsigned rowb = (unsigned)P.K * ES;
  const int chunks = (int)((rowb + 1023) / 1024);
  const char *wrow[VR];
#pragma unroll
  for (int v = 0; v < VR; ++v)
    wrow[v] = static_cast<const char *>(GATED && v >= VN ? P.B1 : P.B0) + (size_t)(n0 + v % VN) * rowb;  // N % 8 == 0: all there
  auto rsrc = [&](const char *base) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base), 0, __builtin_amdgcn_readfirstlane((int)rowb), BUF_FLAGS);
  };
  using Quad = decltype(__builtin_amdgcn_raw_buffer_load_b128(rsrc(nullptr), 0u, 0, 0));
  auto value = [](const Quad &v, int i) {
    const u32 word = v[BF16 ? i >> 1 : i];  // (a copy: __builtin_bit_cast of a vector's element takes element 0, whichever it is)
    return __builtin_bit_cast(float, BF16 ? (i & 1 ? word & 0xffff0000u : word << 16) : word);
  };
  float acc[VR][M];
#pragma unroll
  for (int v = 0; v < VR; ++v)
#pragma unroll
    for (int m = 0; m < M; ++m) acc[v][m] = 0.0f;
  // past a row's end: out of range, zero
  for (int c0 = 0; c0 < chunks; c0 += LV_AHEAD) {
    Quad b[LV_AHEAD][VR], a[LV_AHEAD][M];
#pragma unroll
    for (int s = 0; s < LV_AHEAD; ++s) {
      const unsigned at = (unsigned)(c0 + s) * 1024 + lane * 16;
#pragma unroll
      for (int v = 0; v < VR; ++v) b[s][v] = __builtin_amdgcn_raw_buffer_load_b128(rsrc(wrow[v]), at, 0, BUF_STREAM);
#pragma unroll
      for (int m = 0; m < M; ++m) a[s][m] = __builtin_amdgcn_raw_buffer_load_b128(rsrc(static_cast<const char *>(P.A) + (size_t)m * rowb), at, 0, 0);
    }
#pragma unroll
    for (int s = 0; s < LV_AHEAD; ++s)
#pragma unroll
      for (int i = 0; i < PE; ++i)
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
          for (int v = 0; v < VR; ++v) acc[v][m] = fmaf(value(b[s][v], i), value(a[s][m], i), acc[v][m]);
  }
#pragma unroll
  for (int v = 0; v < VR; ++v)
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int o = kWave / 2; o > 0; o >>= 1) acc[v][m] += __shfl_xor(acc[v][m], o);
  // lane m * VN + v writes column n0 + v of row m
#pragma unroll
  for (int m = 0; m < M; ++m)
#pragma unroll
    for (int v = 0; v < VN; ++v) {
      if (lane != m * VN + v) continue;
      const int n = n0 + v, R = GATED ? 2 * N : N;
      const float g = acc[v][m] + (P.bias ? P.bias[n] : 0.0f);
      const float up = GATED ? acc[v + VR - VN][m] + (P.bias ? P.bias[N + n] : 0.0f) : 0.0f;
      float y = GATED ? dense_silu<BF16>(g) * up : ACT == RR_ACT_GELU ? dense_gelu<BF16>(g) : g;
      if (P.pre) {
        store_value<BF16>(P.pre, (size_t)m * R + n, g);
        if (GATED) store_value<BF16>(P.pre, (size_t)m * R + N + n, up);
      }
      if (P.residual) y += load_value<BF16>(P.residual, (size_t)m * N + n);
      store_value<BF16>(P.Cout, (size_t)m * N + n, y);
    }
#endif
}

// ------------------------------------------------------------------ joining slices
// Adds the slices' sums in order and does the epilogue; a thread owns four columns (gated: of both halves) and has the sums
// of kJoinAhead slices under way.
constexpr int kJoinAhead = 8;
template <bool BF16, bool GATED, int ACT>
__global__ __launch_bounds__(256) void linear_join_kernel(DenseArgs P) {
  const int N = P.N, R = GATED ? 2 * N : N, quads = N / 4;
  const size_t t = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (t >= (size_t)P.M * quads) return;
  const int row = (int)(t / quads), col = (int)(t - (size_t)row * quads) * 4;
  f32x4 acc[1][GATED ? 2 : 1];
#pragma unroll
  for (int j = 0; j < (GATED ? 2 : 1); ++j) {
    const float *at = P.part + (size_t)row * R + j * N + col;
    acc[0][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = 0; s0 < P.slices; s0 += kJoinAhead) {
      f32x4 v[kJoinAhead];
#pragma unroll
      for (int s = 0; s < kJoinAhead; ++s) {
        v[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (s0 + s < P.slices) v[s] = *reinterpret_cast<const f32x4 *>(at + (size_t)(s0 + s) * P.M * R);
      }
#pragma unroll
      for (int s = 0; s < kJoinAhead; ++s) acc[0][j] += v[s];
    }
  }
  DenseArgs Q = P;
  Q.part = nullptr;
  // lane 0 .. 15 of a fragment own its first four columns: the thread's four, as if it were such a lane
  store_dense<1, GATED ? 2 : 1, 16, BF16, GATED, ACT>(acc, Q, 0, row, P.M, col, 0);
}

// ------------------------------------------------------------------ dz, transposes, column sums
// A workgroup takes 64 columns of dy (or of x, or W: ACT none), 64 rows at a time (every gridDim.y-th tile of them), makes dz where there
// is an activation, and writes what is asked for: dz, the sums of its columns over all its rows, and (fp32; bf16 products read every
// operand as it lies) its transpose of row pitch LT >= M, zeros behind column M, through LDS.  A thread owns two neighbouring rows and eight
// columns.
// bf16: dz is rounded once before the products, whose matrix instructions read bf16; the column sums take it unrounded.  The gradients are then two
// roundings off, 2.3e-3 in norm, where the exact ones rounded once are 1.7e-3.  As two bf16 parts dz would double both summations: 8192 rows, 2048 ->
// 2 x 5632, the products 581 us, 1146 with twice the columns of dz.
// Bound by HBM: 8192 x 5632 bf16 SwiGLU, dz alone: 89 us, 461 MB, 5.2 TB/s.
struct TurnArgs {
  const void *src, *pre;  // [M, N], [M, R]
  void *dz;               // [M, R]
  float *turned;          // [R, LT]
  float *sums;            // [gridDim.y, R]
  int M, N, LT;
};
constexpr int TN_TILE = 64, TN_THREADS = 256;

template <bool BF16>
__device__ inline void load_eight(const void *p, size_t at, bool in, float (&v)[8]) {
  if constexpr (BF16) {
    uint4 q = make_uint4(0, 0, 0, 0);
    if (in) q = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + at);
    const u32 w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(float, i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);
  } else {
    f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f}, b = a;
    if (in) {
      const f32x4 *s = reinterpret_cast<const f32x4 *>(static_cast<const float *>(p) + at);
      a = s[0];
      b = s[1];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = a[i];
      v[4 + i] = b[i];
    }
  }
}
template <bool BF16>
__device__ inline void store_eight(void *p, size_t at, const float (&v)[8]) {
  if constexpr (BF16) {
    *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + at) =
        make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  } else {
    float4 *d = reinterpret_cast<float4 *>(static_cast<float *>(p) + at);
    d[0] = make_float4(v[0], v[1], v[2], v[3]);
    d[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// Derivative of z Phi(z): Phi(z) + z phi(z).  Phi(-|z|) = exp(-z^2/2) Q(1 / (1 + 0.4 |z| / sqrt 2)) / 2 with Q a polynomial of degree
// 8 fitted to exp(x^2) erfc(x) for x up to 9.5 so that Phi's absolute error is small: 2.5e-8 with these coefficients (of fp32, whose rounding is
// most of it); both terms share the exponential.  Computed in fp32 the slope is 4 u of 1 off at most.  (erff branches twice per element: 2001 x 2816 fp32 35 us, 22 so.)
__device__ inline float gelu_slope(float z) {
  const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.4f * 0.70710678118654752f, 1.0f)), e = exp_short(-0.5f * z * z);
  float q = 0.07846596f;
  q = fmaf(q, t, -0.41394132f);
  q = fmaf(q, t, 0.72221178f);
  q = fmaf(q, t, -0.41413307f);
  q = fmaf(q, t, 0.43398637f);
  q = fmaf(q, t, 0.13015456f);
  q = fmaf(q, t, 0.23855637f);
  q = fmaf(q, t, 0.22468223f);
  q = fmaf(q, t, 1.7079643e-05f);
  const float half = 0.5f * e * q;
  return fmaf(z * 0.39894228040143268f, e, z >= 0.0f ? 1.0f - half : half);
}

template <bool BF16, int ACT>
__global__ __launch_bounds__(TN_THREADS) void linear_turn_kernel(TurnArgs P) {
  constexpr int NB = ACT == RR_ACT_SWIGLU ? 2 : 1;
  __shared__ float part[TN_THREADS / kWave][TN_TILE];
  const int tid = threadIdx.x, piece = tid & 7, pair = tid >> 3, N = P.N, R = NB * N;
  const int n0 = blockIdx.x * TN_TILE, col = n0 + piece * 8, rows = !BF16 && P.turned ? max(P.M, P.LT) : P.M;
  float sum[NB][8];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[b][i] = 0.0f;
  for (int m0 = blockIdx.y * TN_TILE; m0 < rows; m0 += gridDim.y * TN_TILE) {
    const int row = m0 + 2 * pair;
    float v[NB][2][8], z[ACT == RR_ACT_NONE ? 1 : NB][2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool in = row + h < P.M && col < N;
      load_eight<BF16>(P.src, (size_t)(row + h) * N + col, in, v[0][h]);
      if constexpr (ACT != RR_ACT_NONE)
#pragma unroll
        for (int b = 0; b < NB; ++b) load_eight<BF16>(P.pre, (size_t)(row + h) * R + b * N + col, in, z[b][h]);
    }
    if constexpr (ACT != RR_ACT_NONE) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float d = v[0][h][i], g = z[0][h][i];
          if constexpr (NB == 2) {
            // silu' = t (1 + g (1 - t)), t = 1 / (1 + exp(-g))
            const float t = 1.0f / (1.0f + (BF16 ? __expf(-g) : expf(-g)));
            v[0][h][i] = d * z[NB - 1][h][i] * t * (1.0f + g * (1.0f - t));
            v[NB - 1][h][i] = d * g * t;
          } else {
            v[0][h][i] = d * gelu_slope(g);
          }
        }
        if (P.dz && row + h < P.M && col < N)
#pragma unroll
          for (int b = 0; b < NB; ++b) store_eight<BF16>(P.dz, (size_t)(row + h) * R + b * N + col, v[b][h]);
      }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int i = 0; i < 8; ++i) sum[b][i] += v[b][0][i] + v[b][1][i];
      if constexpr (!BF16) {
        if (!P.turned) continue;
        constexpr int PITCH = TN_TILE + 1, PIECES = TN_TILE / 4;  // words of a column in LDS: odd, so that no two lanes meet in a bank; 16-byte pieces
        __shared__ float tile[TN_TILE * PITCH];
        __syncthreads();  // the tile before this one has been read
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float *at = tile + (piece * 8 + i) * PITCH + 2 * pair;
          at[0] = v[b][0][i];
          at[1] = v[b][1][i];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < TN_TILE * PIECES / TN_THREADS; ++k) {
          const int p = k * TN_THREADS + tid, c = p / PIECES, q = p % PIECES;
          const float *at = tile + c * PITCH + q * 4;
          const int m = m0 + q * 4;
          if (n0 + c < N && m < P.LT)
            *reinterpret_cast<float4 *>(P.turned + (size_t)(b * N + n0 + c) * P.LT + m) = make_float4(at[0], at[1], at[2], at[3]);
        }
      }
    }
  }
  if (!P.sums) return;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float s = sum[b][i];
#pragma unroll
      for (int o = 8; o < kWave; o <<= 1) s += __shfl_xor(s, o);
      if ((tid & (kWave - 1)) < 8) part[tid >> 6][piece * 8 + i] = s;
    }
    __syncthreads();
    if (tid < TN_TILE && n0 + tid < N)
      P.sums[(size_t)blockIdx.y * R + b * N + n0 + tid] = (part[0][tid] + part[1][tid]) + (part[2][tid] + part[3][tid]);
    __syncthreads();
  }
}

// dbias from the sums of `blocks` workgroups, in order; a thread has LB_AHEAD of them under way.
constexpr int LB_PARTS = 16;
[[maybe_unused]] constexpr int LB_AHEAD = 8;
__global__ __launch_bounds__(LB_PARTS * kWave) void linear_bias_kernel(const float *sums, int blocks, int R, float *dbias) {
  __shared__ double part[LB_PARTS][kWave];
  const int lane = threadIdx.x & 63, q = threadIdx.x >> 6, n = blockIdx.x * kWave + lane;
  double s = 0.0;
  if (n < R)
    for (int i = q; i < blocks; i += LB_PARTS * LB_AHEAD) {
      float v[LB_AHEAD];
#pragma unroll
      for (int k = 0; k < LB_AHEAD; ++k) {
        v[k] = 0.0f;
        if (i + k * LB_PARTS < blocks) v[k] = sums[(size_t)(i + k * LB_PARTS) * R + n];
      }
#pragma unroll
      for (int k = 0; k < LB_AHEAD; ++k) s += (double)v[k];
    }
  part[q][lane] = s;
  __syncthreads();
  if (q > 0 || n >= R) return;
  s = 0.0;
#pragma unroll
  for (int k = 0; k < LB_PARTS; ++k) s += part[k][lane];
  dbias[n] = (float)s;
}

// ------------------------------------------------------------------ which kernel
constexpr int kMaxSlices = 16;
constexpr size_t kPartBytes = (size_t)128 << 20;  // most that slices' sums may take
size_t part_bytes(size_t M, size_t R, int slices) { return M * R * 4 * slices; }
// the workspace for them: of a product of M rows it also serves every product of fewer rows
size_t part_reserve(size_t M, size_t R) { return up256(std::min(part_bytes(M, R, kMaxSlices), kPartBytes)); }

struct DensePlan {
  int shape, slices;  // shape: FfnShape; -1: linear_rows_kernel
  float time;         // estimate, us
};
bool splits(const DensePlan &p) { return p.shape == FFN_S128 || p.shape == FFN_S64; }

// Times in us of a dense product's parts: a fit to 970 bf16 products (M 5 .. 16384, rows and columns 64 .. 11008) and 700 fp32
// ones, each timed in up to 34 pairs of shape and slices.  The plan is 1.2 % (fp32: 1.1 %) off the best pair on average, 1.4 %
// (1.4 %) on the quarter of them that the fit did not see; the worst of those by 24 % (21 %), most of them products of 4 us.  (The
// grouped GEMM's numbers, which expect ragged experts and weights from HBM: 7 %, the worst by 45 %.)  3 .. 32 rows of bf16 with W from HBM,
// 1744 products in random order: `rows`, `cold`, `alone` and `even` fitted to a third of those, 2.3 % off the best, 3.0 % on the rest.
struct DenseShape { float chunk, fixed, alone; };  // as ShapeInfo: of a chunk, of a tile, of a chunk with the CU to itself (split shapes; few rows)
struct DenseTimes {
  int first;             // FfnShape of shape[0]
  DenseShape shape[6];
  float fetch, stream;   // bytes per us that a CU gets of its operands, and all of them together
  float last, even;      // a last, partial round on top of its share; split shapes, few rows: weight of the exact number of rounds
  float launch, join, join_slice, join_bytes;  // of any kernel; of the joining one: itself, per slice, passes over the slices' sums
  float rows;            // linear_rows_kernel: start and end
  float cold;            // up to kFewRows rows: a chunk's time, W coming from HBM, over that of a product that finds its operands in the caches
};
constexpr DenseTimes kBf16Times{FFN_P256, {{1.37f, 0.02f}, {0.787f, 1.05f}, {0.506f, 0.73f}, {0.341f, 0.66f, 1.1f}, {0.273f, 0.73f, 0.47f}, {0.14f, 0.84f, 0.19f}},
                                153e3f, 10.1e6f, 0.98f, 0.5f, 2.6f, 1.7f, 0.15f, 2.3f, 0.8f, 1.39f};
constexpr DenseTimes kF32Times{FFN_S128, {{1.328f, 0.52f, 1.67f}, {0.738f, 0.24f, 0.99f}, {0.937f, 0.17f}, {0.521f, 0.19f}, {0.26f, 0.02f}, {0.0f, 0.0f}},
                               38e3f, 91e6f, 0.54f, 0.25f, 3.4f, 2.3f, 0.083f, 1.36f, 0.5f, 1.0f};
constexpr float kPersistentDense = 3.2f;  // the 256 x 256 kernel's start

// Estimated time of A[M, K] times B[N, K]^T (gated: of two such) in tiles of shape q with K cut into `slices`; < 0: not possible.
// turned: B, or both operands, lie the other way round (fp32: the price of transposes is gradient_plan's).
enum Turned { TURNED_NONE, TURNED_B, TURNED_BOTH };
float dense_cost(long long M, long long N, long long K, bool bf16, bool gated, Turned turned, int q, int slices) {
  constexpr int kCUs = 256;
  const DenseTimes &T = bf16 ? kBf16Times : kF32Times;
  const ShapeInfo &s = kShape[q];
  const DenseShape &c = T.shape[q - T.first];
  const int es = bf16 ? 2 : 4, ce = GB_ROW_BYTES / es, bn = gated ? s.brows / 2 : s.brows;
  const long long Ks = slices > 1 ? (K / slices + ce - 1) / ce * ce : K;
  if (slices > 1 && (Ks * slices < K || Ks * (slices - 1) >= K)) return -1.0f;
  const bool persistent = q == FFN_P256, split = q == FFN_S128 || q == FFN_S64;
  if (persistent && (!persistent_ok((int)Ks) || (slices > 1 && turned != TURNED_BOTH && Ks * slices != K))) return -1.0f;
  const int KT = (int)((Ks + ce - 1) / ce);
  if (split && KT < 5) return -1.0f;
  const long long mt = (M + s.bm - 1) / s.bm, nt = (N + bn - 1) / bn, tiles = mt * nt * slices, rounds = tiles / kCUs, left = tiles - rounds * kCUs;
  const size_t R = (size_t)N * (gated ? 2 : 1), part = part_bytes(M, R, slices);
  if (slices > 1 && part > kPartBytes) return -1.0f;
  const float stream = (float)((double)(M + R) * K * es + (double)M * N * es) / T.stream;
  const float fetch = (float)GB_ROW_BYTES * ((float)s.brows / mt + (float)s.bm / nt) / T.fetch;
  const bool few = bf16 && M <= kFewRows && turned == TURNED_NONE;  // W from HBM, read once
  const float chunk = std::max(c.chunk * (few ? T.cold : 1.0f), fetch);  // (turned operands: the same, 440 products)
  float busy = (float)rounds * (KT * chunk + c.fixed);
  if (split || (few && c.alone > 0.0f)) {
    const float all = (float)tiles / kCUs;
    busy = std::max((T.even * all + (1.0f - T.even) * ceilf(all)) * (KT * chunk + c.fixed), KT * c.alone + c.fixed);
  } else if (persistent) {
    busy += kPersistentDense;
    if (left > 0) busy += KT * std::max(chunk * kCutCost[std::min<long long>(kCUs / left, PK_MAX_CUT) - 1], fetch) + c.fixed;
  } else if (left > 0) {
    busy += (KT * chunk + c.fixed) * (rounds ? std::min(1.0f, (float)left / kCUs + T.last) : 1.0f);
  }
  float t = T.launch + std::max(busy, stream) + 0.1f * busy;
  if (slices > 1) t += T.join + T.join_slice * slices + T.join_bytes * (float)part / kHbm;
  return t;
}

// linear_rows_kernel: a workgroup reads its rows of W and all of A.
float rows_cost(long long M, long long N, long long K, bool bf16, bool gated) {
  const DenseTimes &T = bf16 ? kBf16Times : kF32Times;
  const int es = bf16 ? 2 : 4;
  const long long blocks = (N + 15) / 16, bytes = ((gated ? 32 : 16) + M) * K * es;
  constexpr float kAlone = 37e3f, kShared = 30e3f;  // bytes per us of a CU with one workgroup, with several
  return T.launch + T.rows + (float)((blocks + 255) / 256) * (float)bytes / (blocks > 256 ? kShared : kAlone);
}

// splits_only: of the shapes that split fp32 operands (time < 0: none can)
DensePlan dense_plan(long long M, long long N, long long K, bool bf16, bool gated, Turned turned, bool splits_only = false) {
  const bool tiles_only = splits_only || (bf16 && turned != TURNED_NONE);
  if (M <= kVectorRows(bf16) && !tiles_only) return {-1, 1, rows_cost(M, N, K, bf16, gated)};
  const int q0 = bf16 ? FFN_P256 : FFN_S128, q1 = bf16 ? FFN_32N : splits_only ? FFN_S64 : FFN_F32N;
  DensePlan best{q1, 1, -1.0f};
  if (M <= kFewRows && !tiles_only) best = {-1, 1, rows_cost(M, N, K, bf16, gated)};
  for (int q = q0; q <= q1; ++q) {
    if (q == FFN_F32) continue;  // (32 x 128 in fp32: the best estimate of one product in 5000, by nothing)
    const long long bn = gated ? kShape[q].brows / 2 : kShape[q].brows, tiles = (M + kShape[q].bm - 1) / kShape[q].bm * ((N + bn - 1) / bn);
    for (int s = 1; s <= kMaxSlices && (s == 1 || tiles * s <= 2048); ++s) {  // (eight rounds: slices even nothing out any more)
      const float t = dense_cost(M, N, K, bf16, gated, turned, q, s);
      if (t >= 0.0f && (best.time < 0.0f || t < best.time)) best = {q, s, t};
    }
  }
  return best;
}

// The gradients' products: whether the operands are read as they lie.
struct TurnedPlan {
  DensePlan plan;
  bool as_is;
};
// fp32: tiles that split their operands turn them too; of other kernels the transposes before them are a part of the price (16 x
// 4096 -> 4096: 74 us with a transpose of W for linear_rows_kernel, 58 in tiles of 64 rows; 818 x 5848 -> 88: 46, 42).
// `turned`: bytes that those read and write.
TurnedPlan gradient_plan(const DensePlan &as_is, const DensePlan &any, size_t turned) {
  if (as_is.time >= 0.0f && as_is.time <= any.time + kF32Times.launch + (float)turned / kHbm) return {as_is, true};
  return {any, false};
}
TurnedPlan plan_dx(const rr_linear_config &c, int R, bool bf16) {
  if (bf16) return {dense_plan(c.M, c.K, R, bf16, false, TURNED_B), true};
  return gradient_plan(dense_plan(c.M, c.K, R, bf16, false, TURNED_B, true), dense_plan(c.M, c.K, R, bf16, false, TURNED_B), (size_t)R * c.K * 8);
}
// LT: length of the transposes' rows, where they are made
TurnedPlan plan_dw(const rr_linear_config &c, int R, bool bf16, int LT) {
  if (bf16) return {dense_plan(R, c.K, c.M, bf16, false, TURNED_BOTH), true};
  return gradient_plan(dense_plan(R, c.K, c.M, bf16, false, TURNED_BOTH, true), dense_plan(R, c.K, LT, bf16, false, TURNED_BOTH),
                       (size_t)LT * (2 * c.K + R) * 4);
}

template <class S, bool GATED, int ACT, bool TA, bool TB>
void launch_dense_tiles(DenseArgs A, hipStream_t s) {
  constexpr int bn = GATED ? S::BROWS / 2 : S::BROWS;
  A.NT = (A.N + bn - 1) / bn;
  A.MT = (A.M + S::BM - 1) / S::BM;
  constexpr long long kRow = 1ll << 20;  // workgroups in a row of the grid, whole XCD runs (see gemm_tile_kernel)
  const long long tiles = (long long)A.NT * A.MT * A.slices;
  const dim3 grid((unsigned)((std::min(tiles, kRow) + 7) / 8 * 8), (unsigned)((tiles + kRow - 1) / kRow));
  // One tile of rows: each byte of W is read by one workgroup, once, and streams past the caches (ONCE).  in the same tiles 16 x 4096 -> 2 x 11008
  // 39.2 -> 35.3 us (5.1 TB/s), 32 x 11008 -> 4096 24.0 -> 22.5, 128 x 4096 -> 2 x 11008 49.4 -> 46.1; only if the last-level cache still holds a large W from
  // the call before it costs time (16 x 4096 -> 2 x 11008, 180 MB: 27.0 -> 35.5; of 34 MB and less: nothing).  More tiles of rows: 10 % either way, so
  // not; fp32: 1 %, so not.
  if constexpr (S::BF16 && !TB) {
    if (A.MT == 1) {
      gemm_tile_kernel<S, GATED, ACT, false, false, true, TA, TB, true><<<grid, S::THREADS, S::SMEM, s>>>(A);
      return;
    }
  }
  gemm_tile_kernel<S, GATED, ACT, false, false, true, TA, TB><<<grid, S::THREADS, S::SMEM, s>>>(A);
}

template <bool BF16, bool GATED, int ACT, bool TA = false, bool TB = false>
void launch_dense_shape(int shape, DenseArgs A, hipStream_t s) {
  if constexpr (BF16) {
    switch (shape) {
      case FFN_P256:
        A.NT = GATED ? (A.N + 127) / 128 : (A.N + 255) / 256;
        A.MT = (A.M + PK_BM - 1) / PK_BM;
        gemm_bf16_persistent_kernel<GATED, ACT, false, false, true, TA, TB><<<cu_count(), PK_THREADS, PK_SMEM, s>>>(A);
        break;
      case FFN_256: launch_dense_tiles<TileB256, GATED, ACT, TA, TB>(A, s); break;
      case FFN_128: launch_dense_tiles<TileB128, GATED, ACT, TA, TB>(A, s); break;
      case FFN_64: launch_dense_tiles<TileB64, GATED, ACT, TA, TB>(A, s); break;
      case FFN_32: launch_dense_tiles<TileB32, GATED, ACT, TA, TB>(A, s); break;
      default: launch_dense_tiles<TileB32n, GATED, ACT, TA, TB>(A, s); break;
    }
  } else {
    switch (shape) {
      case FFN_S128: launch_dense_tiles<TileS128, GATED, ACT, TA, TB>(A, s); break;
      case FFN_S64: launch_dense_tiles<TileS64, GATED, ACT, TA, TB>(A, s); break;
      case FFN_F64:
        if constexpr (!TB) launch_dense_tiles<TileF64, GATED, ACT, TA, TB>(A, s);
        break;
      default:
        if constexpr (!TB) launch_dense_tiles<TileF32n, GATED, ACT, TA, TB>(A, s);
        break;
    }
  }
}

// The product and its epilogue.  A.A, B0, B1, Cout, M, N, lda, ldb, Kall and the epilogue's pointers are set.
template <bool BF16, bool GATED, int ACT>
void launch_product(DenseArgs A, const DensePlan &plan, Turned turned, float *part, hipStream_t s) {
  constexpr int ce = GB_ROW_BYTES / (BF16 ? 2 : 4);
  A.slices = plan.slices;
  A.K = plan.slices > 1 ? (A.Kall / plan.slices + ce - 1) / ce * ce : A.Kall;
  A.part = plan.slices > 1 ? part : nullptr;
  if (plan.shape < 0) {
    if (A.M <= kVectorRows(BF16)) {
      const dim3 grid((A.N * (GATED ? 2 : 1) / LV_ROWS + LV_THREADS / kWave - 1) / (LV_THREADS / kWave));
      if (A.M == 1) linear_vector_kernel<BF16, GATED, ACT, 1><<<grid, LV_THREADS, 0, s>>>(A);
      if (A.M == 2) linear_vector_kernel<BF16, GATED, ACT, 2><<<grid, LV_THREADS, 0, s>>>(A);
      if constexpr (kVectorRows(BF16) > 2) {
        if (A.M == 3) linear_vector_kernel<BF16, GATED, ACT, 3><<<grid, LV_THREADS, 0, s>>>(A);
        if (A.M == 4) linear_vector_kernel<BF16, GATED, ACT, 4><<<grid, LV_THREADS, 0, s>>>(A);
      }
      return;
    }
    const dim3 grid((A.N + 15) / 16);
    if (A.M <= 16) linear_rows_kernel<BF16, GATED, ACT, 1><<<grid, LR_THREADS, 0, s>>>(A);
    else linear_rows_kernel<BF16, GATED, ACT, 2><<<grid, LR_THREADS, 0, s>>>(A);
    return;
  }
  if constexpr (!GATED && ACT < 0) {
    if (turned == TURNED_B) launch_dense_shape<BF16, GATED, ACT, false, true>(plan.shape, A, s);
    if (turned == TURNED_BOTH) launch_dense_shape<BF16, GATED, ACT, true, true>(plan.shape, A, s);
  }
  if (turned == TURNED_NONE) launch_dense_shape<BF16, GATED, ACT>(plan.shape, A, s);
  if (plan.slices > 1)
    linear_join_kernel<BF16, GATED, ACT><<<(unsigned)(((size_t)A.M * (A.N / 4) + 255) / 256), 256, 0, s>>>(A);
}

template <bool BF16>
void launch_forward(int act, const DenseArgs &A, float *part, hipStream_t s) {
  const DensePlan plan = dense_plan(A.M, A.N, A.Kall, BF16, act == RR_ACT_SWIGLU, TURNED_NONE);
  if (act == RR_ACT_SWIGLU) launch_product<BF16, true, -1>(A, plan, TURNED_NONE, part, s);
  else if (act == RR_ACT_GELU) launch_product<BF16, false, RR_ACT_GELU>(A, plan, TURNED_NONE, part, s);
  else launch_product<BF16, false, -1>(A, plan, TURNED_NONE, part, s);
}

// Workgroups that a column of them is cut into: one per 64 rows, or, where they leave sums, no more than keep the chip busy.
int turn_blocks(const TurnArgs &A) {
  const int rows = A.turned ? std::max(A.M, A.LT) : A.M, tiles = (rows + TN_TILE - 1) / TN_TILE;
  return A.sums ? std::min(tiles, std::max(64, 1024 / ((A.N + TN_TILE - 1) / TN_TILE))) : tiles;
}

template <bool BF16>
void launch_turn(int act, const TurnArgs &A, hipStream_t s) {
  const dim3 grid((A.N + TN_TILE - 1) / TN_TILE, turn_blocks(A));
  if (act == RR_ACT_SWIGLU) linear_turn_kernel<BF16, RR_ACT_SWIGLU><<<grid, TN_THREADS, 0, s>>>(A);
  else if (act == RR_ACT_GELU) linear_turn_kernel<BF16, RR_ACT_GELU><<<grid, TN_THREADS, 0, s>>>(A);
  else linear_turn_kernel<BF16, RR_ACT_NONE><<<grid, TN_THREADS, 0, s>>>(A);
}

// Workspace of the backward pass.
struct BackwardWork {
  void *dz;
  float *dz_turned, *x_turned, *w_turned;  // fp32 only
  float *sums, *part;
  int LT;  // row pitch of the transposes that are summed over rows: M and zeros up to whole chunks
  size_t bytes;
};
BackwardWork backward_work(const rr_linear_config &c, void *ws) {
  BackwardWork W;
  char *base = static_cast<char *>(ws);
  size_t off = 0;
  auto take = [&](size_t n) {
    void *p = base ? base + off : nullptr;
    off += up256(n);
    return p;
  };
  auto take_floats = [&](size_t n) { return static_cast<float *>(take(n * 4)); };
  const size_t R = width(c), es = element(c);
  W.LT = (c.M + 63) / 64 * 64;
  W.dz = take(c.act == RR_ACT_NONE ? 0 : (size_t)c.M * R * es);
  const bool turns = c.dtype != RR_BF16;
  W.dz_turned = take_floats(turns ? R * W.LT : 0);
  W.x_turned = take_floats(turns ? (size_t)c.K * W.LT : 0);
  W.w_turned = take_floats(turns ? (size_t)c.K * R : 0);
  W.sums = take_floats((size_t)(W.LT / TN_TILE) * R);
  W.part = static_cast<float *>(take(std::max(part_reserve(c.M, c.K), part_reserve(R, c.K))));
  W.bytes = off;
  return W;
}

}  // namespace

hipError_t linear_kernel_attributes() {
  hipError_t e = hipSuccess;
  auto set = [&e](auto kern, int bytes) {
    if (e == hipSuccess) e = set_lds(kern, bytes);
  };
  auto kinds = [&](auto tag) {
    using S = typename decltype(tag)::type;
    if constexpr (!std::is_same<S, TileF32>::value) {
      set(gemm_tile_kernel<S, true, -1, false, false, true>, S::SMEM);
      set(gemm_tile_kernel<S, false, RR_ACT_GELU, false, false, true>, S::SMEM);
      set(gemm_tile_kernel<S, false, -1, false, false, true>, S::SMEM);
    }
    if constexpr (S::BF16) {
      set(gemm_tile_kernel<S, true, -1, false, false, true, false, false, true>, S::SMEM);
      set(gemm_tile_kernel<S, false, RR_ACT_GELU, false, false, true, false, false, true>, S::SMEM);
      set(gemm_tile_kernel<S, false, -1, false, false, true, false, false, true>, S::SMEM);
    }
    if constexpr (S::MATH != TILE_F32) {
      set(gemm_tile_kernel<S, false, -1, false, false, true, false, true>, S::SMEM);
      set(gemm_tile_kernel<S, false, -1, false, false, true, true, true>, S::SMEM);
    }
  };
  for_each_tile_shape(kinds);
  set(gemm_bf16_persistent_kernel<true, -1, false, false, true>, PK_SMEM);
  set(gemm_bf16_persistent_kernel<false, RR_ACT_GELU, false, false, true>, PK_SMEM);
  set(gemm_bf16_persistent_kernel<false, -1, false, false, true>, PK_SMEM);
  set(gemm_bf16_persistent_kernel<false, -1, false, false, true, false, true>, PK_SMEM);
  set(gemm_bf16_persistent_kernel<false, -1, false, false, true, true, true>, PK_SMEM);
  return e;
}

void linear_describe(const rr_linear_config &c, LinearPlans *out) {
  const bool bf16 = c.dtype == RR_BF16;
  const int R = width(c);
  const DensePlan plan[3] = {dense_plan(c.M, c.N, c.K, bf16, c.act == RR_ACT_SWIGLU, TURNED_NONE),
                             plan_dx(c, R, bf16).plan, plan_dw(c, R, bf16, backward_work(c, nullptr).LT).plan};
  for (int i = 0; i < 3; ++i) {
    out->bm[i] = plan[i].shape < 0 ? 0 : kShape[plan[i].shape].bm;
    out->brows[i] = plan[i].shape < 0 ? 0 : kShape[plan[i].shape].brows;
    out->slices[i] = plan[i].slices;
    out->parts[i] = splits(plan[i]);
  }
}

void linear_cut(int m0, int rows, int cut, int part, int32_t *range) {
  const CutRows r = cut_rows(m0, rows, cut, part);
  range[0] = r.m0;
  range[1] = r.end;
}

size_t linear_workspace(const rr_linear_config &c, bool backward) {
  return backward ? backward_work(c, nullptr).bytes : std::max<size_t>(256, part_reserve(c.M, width(c)));
}

hipError_t launch_linear(const rr_linear_config &c, const void *x, const void *w, const float *bias, const void *residual, void *y,
                         void *pre, void *ws, hipStream_t s) {
  DenseArgs A{};
  A.A = x;
  A.B0 = w;
  A.B1 = static_cast<const char *>(w) + (size_t)c.N * c.K * element(c);
  A.Cout = y;
  A.M = c.M;
  A.N = c.N;
  A.lda = A.ldb = A.Kall = c.K;
  A.bias = bias;
  A.residual = residual;
  A.pre = pre;
  prof_begin(K_LINEAR, s);
  if (c.dtype == RR_BF16) launch_forward<true>(c.act, A, static_cast<float *>(ws), s);
  else launch_forward<false>(c.act, A, static_cast<float *>(ws), s);
  prof_end(K_LINEAR, s);
  return hipGetLastError();
}

hipError_t launch_linear_backward(const rr_linear_config &c, const void *x, const void *w, const void *pre, const void *dy, void *dx,
                                  void *dw, float *dbias, void *ws, hipStream_t s) {
  const bool bf16 = c.dtype == RR_BF16;
  const int R = width(c);
  const BackwardWork W = backward_work(c, ws);
  auto turn = [&](int act, const TurnArgs &A) {
    if (bf16) launch_turn<true>(act, A, s);
    else launch_turn<false>(act, A, s);
  };
  auto product = [&](const void *a, int lda, const void *b, int ldb, void *out, int M, int N, int K, const DensePlan &plan, Turned turned) {
    DenseArgs A{};
    A.A = a;
    A.B0 = A.B1 = b;
    A.Cout = out;
    A.M = M;
    A.N = N;
    A.lda = lda;
    A.ldb = ldb;
    A.Kall = K;
    if (bf16) launch_product<true, false, -1>(A, plan, turned, W.part, s);
    else launch_product<false, false, -1>(A, plan, turned, W.part, s);
  };
  const bool act = c.act != RR_ACT_NONE;
  const TurnedPlan px = plan_dx(c, R, bf16), pw = plan_dw(c, R, bf16, W.LT);
  const TurnArgs make{dy, pre, act && (dx || (dw && pw.as_is)) ? W.dz : nullptr, dw && !pw.as_is ? W.dz_turned : nullptr,
                      dbias ? W.sums : nullptr, c.M, c.N, W.LT};
  const void *dz = act ? W.dz : dy;
  prof_begin(K_LINEAR_BWD, s);
  if (make.dz || make.turned || make.sums) turn(c.act, make);
  if (dbias) linear_bias_kernel<<<(R + kWave - 1) / kWave, LB_PARTS * kWave, 0, s>>>(W.sums, turn_blocks(make), R, dbias);
  if (dx && px.as_is) {
    product(dz, R, w, c.K, dx, c.M, c.K, R, px.plan, TURNED_B);
  } else if (dx) {
    turn(RR_ACT_NONE, TurnArgs{w, nullptr, nullptr, W.w_turned, nullptr, R, c.K, R});
    product(dz, R, W.w_turned, R, dx, c.M, c.K, R, px.plan, TURNED_NONE);
  }
  if (dw && pw.as_is) {
    product(dz, R, x, c.K, dw, R, c.K, c.M, pw.plan, TURNED_BOTH);
  } else if (dw) {
    turn(RR_ACT_NONE, TurnArgs{x, nullptr, nullptr, W.x_turned, nullptr, c.M, c.K, W.LT});
    product(W.dz_turned, W.LT, W.x_turned, W.LT, dw, R, c.K, W.LT, pw.plan, TURNED_NONE);
  }
  prof_end(K_LINEAR_BWD, s);
  return hipGetLastError();
}

}  // namespace rr
