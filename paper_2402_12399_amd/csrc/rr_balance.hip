// Load-balance loss of the router, per-expert counts, and the gradient of the scores:
//   f_e = c_e / (k n),  P_e = (1/n) sum_t p_te,  loss = coef E sum_e f_e P_e,
//   dL/da_te = dloss coef E / n  p_te (f_e - sum_j f_j p_tj),  p_t = softmax(a_t) over all experts, n counted tokens.
//
// LANES lanes share a token's row, four experts each, so that a wave reads 64 / LANES rows at once; maximum and sum go over
// those lanes by shuffles.  A lane sums its four experts' probabilities over its rows in 64 bits and never touches memory
// for them; one record per workgroup (sums, counts, n) is added up in a fixed order by balance_finish, or by the workgroup
// itself where there is only one.  The gradient needs f, so it is a second pass over the scores: the probabilities are made
// again rather than stored.
// Bound by HBM and, a little below it, by the instructions of exponentials and reductions.  2^20 tokens, 64 experts, top-2: loss
// 55 us + 6 (281 MB, 4.6 TB/s; with expf, shuffles through LDS, a lane per row for the choices and one row at a time 135 + 30),
// gradient 84 us (537 MB, 6.4 TB/s), added to what is there 153 (805 MB, 5.3 TB/s).  1001 tokens, 16 experts: 6.4 and 3.8 us, one workgroup
// without records.
#include "rr_device.h"

namespace rr {

namespace {

constexpr int BL_THREADS = 1024, BL_MAX_BLOCKS = 256;  // the loss: few workgroups, so that few records are left
constexpr int BG_THREADS = 256;
constexpr int BL_UNROLL = 4;  // rows that a lane loads before it needs the first

// What a workgroup leaves: probabilities summed, choices (and, in the last column, tokens) counted.
struct BalanceRecords {
  double prob[BL_MAX_BLOCKS][kMaxE];
  int32_t count[BL_MAX_BLOCKS][kMaxE + 1];
};

struct BalanceArgs {
  const float *logits;
  const int32_t *rank_expert;
  const uint8_t *mask;
  int T, E, k;
  float coef;
  float *loss;
  int32_t *counts;
  float *mean_prob;
  BalanceRecords *records;
};

// The four experts of a lane: in a row (VEC: the row is read 16 bytes at a time) or LANES apart.
template <int LANES, bool VEC>
__device__ inline int expert_of(int lane, int j) {
  return VEC ? 4 * (lane & (LANES - 1)) + j : (lane & (LANES - 1)) + LANES * j;
}
template <int LANES, bool VEC>
__device__ inline void load_row(const float *row, int E, int lane, float (&a)[4]) {
  if (VEC) {
    const int e = expert_of<LANES, VEC>(lane, 0);
    const float4 v = e < E ? *reinterpret_cast<const float4 *>(row + e) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    a[0] = v.x; a[1] = v.y; a[2] = v.z; a[3] = v.w;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int e = expert_of<LANES, VEC>(lane, j);
      a[j] = e < E ? row[e] : -INFINITY;
    }
  }
}
// Reductions over the lanes of a row, by DPP: neighbours, pairs, then mirrored halves of 8 and of 16 lanes.
template <int CTRL>
__device__ inline float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int LANES>
__device__ inline float row_max(float v) {
  if (LANES >= 2) v = fmaxf(v, dpp<0xB1>(v));
  if (LANES >= 4) v = fmaxf(v, dpp<0x4E>(v));
  if (LANES >= 8) v = fmaxf(v, dpp<0x141>(v));
  if (LANES >= 16) v = fmaxf(v, dpp<0x140>(v));
  return v;
}
template <int LANES>
__device__ inline float row_sum(float v) {
  if (LANES >= 2) v += dpp<0xB1>(v);
  if (LANES >= 4) v += dpp<0x4E>(v);
  if (LANES >= 8) v += dpp<0x141>(v);
  if (LANES >= 16) v += dpp<0x140>(v);
  return v;
}
// Scores -> unnormalised probabilities; returns 1 / their sum (0 for a row of -infinity only).
template <int LANES>
__device__ inline float softmax_row(float (&a)[4]) {
  const float m = row_max<LANES>(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])));
  const float top = m == -INFINITY ? 0.0f : m;
#pragma unroll
  for (int j = 0; j < 4; ++j) a[j] = exp_short(a[j] - top);
  const float sum = row_sum<LANES>((a[0] + a[1]) + (a[2] + a[3]));
  const float r = __builtin_amdgcn_rcpf(sum);  // 1 ulp; a step of Newton's makes it half of one
  return sum == 0.0f ? 0.0f : fmaf(fmaf(-sum, r, 1.0f), r, r);
}

// One thread per expert, the first wave: loss and the outputs from the sums.
__device__ inline void write_balance(const BalanceArgs &A, double prob, int count, int tokens) {
  const int e = threadIdx.x;
  double term = 0.0;
  if (e < A.E) {
    const double mean = tokens > 0 ? prob / tokens : 0.0;
    term = tokens > 0 ? (double)count / ((double)A.k * tokens) * mean : 0.0;
    A.counts[e] = count;
    if (A.mean_prob) A.mean_prob[e] = (float)mean;
  }
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) term += __shfl_xor(term, o);
  if (e == 0) {
    A.loss[0] = (float)((double)A.coef * A.E * term);
    A.counts[A.E] = tokens;
  }
}

template <int LANES, bool VEC>
__global__ __launch_bounds__(BL_THREADS) void balance_loss_kernel(BalanceArgs A) {
  constexpr int ROWS = kWave / LANES, WAVES = BL_THREADS / kWave, U = BL_UNROLL, STEP = ROWS * U;
  __shared__ double sums[WAVES][kMaxE];
  __shared__ int32_t hist[kMaxE + 1];  // the last one: tokens
  const int tid = threadIdx.x, lane = tid & (kWave - 1), w = tid >> 6, E = A.E, k = A.k;
  if (tid <= kMaxE) hist[tid] = 0;
  __syncthreads();
  double prob[4] = {0.0, 0.0, 0.0, 0.0};
  int live = 0;
  const long long step = (long long)gridDim.x * WAVES * STEP;
  for (long long t0 = ((long long)blockIdx.x * WAVES + w) * STEP; t0 < A.T; t0 += step) {
    float a[U][4];
    bool counted[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long t = t0 + u * ROWS + lane / LANES;
      counted[u] = t < A.T && (!A.mask || A.mask[t]);
#pragma unroll
      for (int j = 0; j < 4; ++j) a[u][j] = 0.0f;
      if (counted[u]) load_row<LANES, VEC>(A.logits + (size_t)t * E, E, lane, a[u]);
    }
    // the choices of these rows: lane l looks at choice l % 4 of every 16th row
#pragma unroll
    for (int i = 0; i < STEP; i += kWave / kMaxK) {
      const long long t = t0 + i + (lane >> 2);
      const int r = lane & 3;
      if (i + (lane >> 2) < STEP && r < k && t < A.T && (!A.mask || A.mask[t])) {
        const int e = A.rank_expert[(size_t)t * (k + 1) + r];
        if (e >= 0 && e < E) atomicAdd(&hist[e], 1);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float inv = softmax_row<LANES>(a[u]);
      if (counted[u]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) prob[j] += (double)(a[u][j] * inv);
        ++live;
      }
    }
  }
#pragma unroll
  for (int o = kWave / 2; o >= LANES; o >>= 1)
#pragma unroll
    for (int j = 0; j < 4; ++j) prob[j] += __shfl_xor(prob[j], o);
  if (lane < LANES)
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[w][expert_of<LANES, VEC>(lane, j)] = prob[j];
  if ((lane & (LANES - 1)) == 0 && live) atomicAdd(&hist[kMaxE], live);
  __syncthreads();
  if (tid >= kWave) return;
  double total = 0.0;
  if (tid < E)
#pragma unroll
    for (int q = 0; q < WAVES; ++q) total += sums[q][tid];
  if (gridDim.x == 1) {
    write_balance(A, total, hist[tid], hist[kMaxE]);
    return;
  }
  A.records->prob[blockIdx.x][tid] = total;
  A.records->count[blockIdx.x][tid] = hist[tid];
  if (tid == 0) A.records->count[blockIdx.x][kMaxE] = hist[kMaxE];
}

// Adds up the records of n workgroups: thread (part, expert) takes every 16th of them, a batch of loads at a time, then the
// parts are added in order.
__global__ __launch_bounds__(1024) void balance_finish_kernel(BalanceArgs A, int n) {
  constexpr int PARTS = 1024 / kWave, BATCH = 16;
  __shared__ double sums[PARTS][kMaxE];
  __shared__ int32_t hist[PARTS][kMaxE], tokens[PARTS];
  const int e = threadIdx.x & (kWave - 1), part = threadIdx.x >> 6;
  double prob = 0.0;
  int count = 0, live = 0;
  for (int i0 = part; i0 < n; i0 += PARTS * BATCH) {
    double p[BATCH];
    int c[BATCH], l[BATCH];
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int i = min(i0 + b * PARTS, n - 1);
      p[b] = A.records->prob[i][e];
      c[b] = A.records->count[i][e];
      l[b] = A.records->count[i][kMaxE];
    }
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const bool in = i0 + b * PARTS < n;
      prob += in ? p[b] : 0.0;
      count += in ? c[b] : 0;
      live += in ? l[b] : 0;
    }
  }
  sums[part][e] = prob;
  hist[part][e] = count;
  if (e == 0) tokens[part] = live;
  __syncthreads();
  if (part > 0) return;
  prob = 0.0;
  count = live = 0;
#pragma unroll
  for (int q = 0; q < PARTS; ++q) {
    prob += sums[q][e];
    count += hist[q][e];
    live += tokens[q];
  }
  write_balance(A, prob, count, live);
}

// A sum that is not fused with the product before it: accumulating adds the very numbers that the call writes otherwise.
__device__ inline float add(float a, float b) {
#pragma clang fp contract(off)
  return a + b;
}

typedef float f32x4_t __attribute__((ext_vector_type(4)));
struct BalanceGradArgs {
  const float *logits;
  const int32_t *counts;
  const uint8_t *mask;
  int T, E, k;
  float coef;
  const float *dloss;
  float *dlogits;
  int stream;  // store past the caches
};

template <int LANES, bool VEC, bool ADD>
__global__ __launch_bounds__(BG_THREADS) void balance_grad_kernel(BalanceGradArgs A) {
  constexpr int ROWS = kWave / LANES, WAVES = BG_THREADS / kWave;
  const int lane = threadIdx.x & (kWave - 1), w = threadIdx.x >> 6, E = A.E;
  const int n = A.counts[E];
  const float each = n > 0 ? 1.0f / ((float)A.k * (float)n) : 0.0f;
  // (in 64 bits: dloss coef and coef E may lie outside fp32's range where the quotient does not)
  const float scale = n > 0 ? (float)((double)(A.dloss ? *A.dloss : 1.0f) * A.coef * E / n) : 0.0f;
  // f_e less the mean of all: the mean falls out of f_e - sum_j f_j p_tj, as the p_tj add up to 1, and with it goes most of what would
  // cancel where the experts are nearly balanced (all alike: zeros, not rounding errors).  Differences of whole numbers are exact.
  int32_t count[4], sum = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int e = expert_of<LANES, VEC>(lane, j);
    count[j] = e < E ? A.counts[e] : 0;
    sum += count[j];
  }
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) sum += __shfl_xor(sum, o);
  float f[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) f[j] = expert_of<LANES, VEC>(lane, j) < E ? (float)(count[j] - sum / E) * each : 0.0f;
  // from the last row to the first: the loss has just read the last ones, which the last-level cache still holds
  const int step = gridDim.x * WAVES * ROWS;
  for (int t0 = (blockIdx.x * WAVES + w) * ROWS; t0 < A.T; t0 += step) {
    const int t = A.T - 1 - t0 - lane / LANES;
    const bool in = t >= 0, counted = in && (!A.mask || A.mask[t]);
    float a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (counted) load_row<LANES, VEC>(A.logits + (size_t)t * E, E, lane, a);
    const float inv = softmax_row<LANES>(a);
    const float mean = row_sum<LANES>(f[0] * a[0] + f[1] * a[1] + f[2] * a[2] + f[3] * a[3]) * inv;
    if (ADD ? !counted : !in) continue;
    float *row = A.dlogits + (size_t)t * E;
    float g[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] = counted ? scale * (a[j] * inv) * (f[j] - mean) : 0.0f;
    if (VEC) {
      const int e = expert_of<LANES, VEC>(lane, 0);
      if (e < E) {
        float4 *at = reinterpret_cast<float4 *>(row + e);
        const float4 v = ADD ? *at : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (ADD) *at = make_float4(add(v.x, g[0]), add(v.y, g[1]), add(v.z, g[2]), add(v.w, g[3]));
        else if (A.stream) __builtin_nontemporal_store(f32x4_t{g[0], g[1], g[2], g[3]}, reinterpret_cast<f32x4_t *>(at));
        else *at = make_float4(g[0], g[1], g[2], g[3]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int e = expert_of<LANES, VEC>(lane, j);
        if (e < E) row[e] = ADD ? add(row[e], g[j]) : g[j];
      }
    }
  }
}

// Workgroups that take `rows` rows each at a time.
int balance_blocks(int T, int rows, int most) {
  const int blocks = (T + rows - 1) / rows;
  return blocks < most ? blocks : most;
}

bool aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <class F>
void with_lanes(int E, bool vec, F f) {
  auto pick = [&](auto v) {
    constexpr bool VEC = decltype(v)::value;
    if (E <= 4) f(std::integral_constant<int, 1>{}, std::integral_constant<bool, VEC>{});
    else if (E <= 8) f(std::integral_constant<int, 2>{}, std::integral_constant<bool, VEC>{});
    else if (E <= 16) f(std::integral_constant<int, 4>{}, std::integral_constant<bool, VEC>{});
    else if (E <= 32) f(std::integral_constant<int, 8>{}, std::integral_constant<bool, VEC>{});
    else f(std::integral_constant<int, 16>{}, std::integral_constant<bool, VEC>{});
  };
  if (vec) pick(std::true_type{});
  else pick(std::false_type{});
}

}  // namespace

size_t balance_workspace() { return (sizeof(BalanceRecords) + 255) / 256 * 256; }

hipError_t launch_balance_loss(int T, int E, int k, const float *logits, const int32_t *rank_expert, const uint8_t *mask, float coef,
                               float *loss, int32_t *counts, float *mean_prob, void *ws, hipStream_t s) {
  const BalanceArgs A{logits, rank_expert, mask, T, E, k, coef, loss, counts, mean_prob, static_cast<BalanceRecords *>(ws)};
  int blocks = 1;
  prof_begin(K_BALANCE, s);
  with_lanes(E, E % 4 == 0 && aligned(logits), [&](auto lanes, auto vec) {
    constexpr int LANES = decltype(lanes)::value;
    constexpr int rows = kWave / LANES * BL_UNROLL * (BL_THREADS / kWave);
    blocks = T <= 4 * rows ? 1 : balance_blocks(T, rows, BL_MAX_BLOCKS);
    balance_loss_kernel<LANES, decltype(vec)::value><<<blocks, BL_THREADS, 0, s>>>(A);
  });
  if (blocks > 1) balance_finish_kernel<<<1, 1024, 0, s>>>(A, blocks);
  prof_end(K_BALANCE, s);
  return hipGetLastError();
}

hipError_t launch_balance_grad(int T, int E, int k, const float *logits, const int32_t *counts, const uint8_t *mask, float coef,
                               const float *dloss, bool add, float *dlogits, hipStream_t s) {
  // Scores and gradient that the last-level cache does not hold together: the gradient goes past it, or its dirty lines are what
  // the next pass over the scores waits for.  2^20 tokens, 64 experts: loss 79 -> 55 us, gradient 88 -> 86 (without the order
  // of rows below: 94).  Smaller ones stay there for who reads them next.
  constexpr size_t kLastLevelBytes = (size_t)256 << 20;
  const BalanceGradArgs A{logits, counts, mask, T, E, k, coef, dloss, dlogits, 2 * (size_t)T * E * 4 > kLastLevelBytes};
  prof_begin(K_BALANCE_BWD, s);
  with_lanes(E, E % 4 == 0 && aligned(logits) && aligned(dlogits), [&](auto lanes, auto vec) {
    constexpr int LANES = decltype(lanes)::value;
    constexpr bool VEC = decltype(vec)::value;
    const int blocks = balance_blocks(T, kWave / LANES * (BG_THREADS / kWave), 1 << 14);
    if (add) balance_grad_kernel<LANES, VEC, true><<<blocks, BG_THREADS, 0, s>>>(A);
    else balance_grad_kernel<LANES, VEC, false><<<blocks, BG_THREADS, 0, s>>>(A);
  });
  prof_end(K_BALANCE_BWD, s);
  return hipGetLastError();
}

}  // namespace rr
