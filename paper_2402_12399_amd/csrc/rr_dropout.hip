// Dropout with the residual sum, and its gradient:
//   out_i = residual_i + (u_i >= m ? x_i s : 0)          dx_i = u_i >= m ? dout_i s : 0
// u_i: 16 bits of Philox4x32-10 at counter offset + i / 8 (rr_device.h).  The backward pass is the forward pass of dout without
// a residual.  A thread owns groups of 8 elements, one call of the generator each.
#include "rr_device.h"

namespace rr {

namespace {

constexpr int DR_THREADS = 256;

struct DropoutArgs {
  const void *x, *residual;
  void *out;
  long long n;
  u32 m;        // of 65536: numbers below are dropped
  float scale;  // 65536 / (65536 - m)
  unsigned long long seed, offset;
  const unsigned long long *device_offset;
};

// Eight elements: as many as a call of the generator serves.
template <bool BF16>
struct Group;
template <>
struct Group<true> {
  uint4 v;
  __device__ void load(const void *p, long long g) { v = static_cast<const uint4 *>(p)[g]; }
  __device__ void store(void *p, long long g) const { static_cast<uint4 *>(p)[g] = v; }
  __device__ float get(int i) const {
    const u32 w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
    return __builtin_bit_cast(float, i & 1 ? w & 0xffff0000u : w << 16);
  }
  __device__ void set(const float (&f)[8]) {
    v = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
  }
};
template <>
struct Group<false> {
  float4 a, b;
  __device__ void load(const void *p, long long g) {
    a = static_cast<const float4 *>(p)[2 * g];
    b = static_cast<const float4 *>(p)[2 * g + 1];
  }
  __device__ void store(void *p, long long g) const {
    static_cast<float4 *>(p)[2 * g] = a;
    static_cast<float4 *>(p)[2 * g + 1] = b;
  }
  __device__ float get(int i) const {
    const float4 &q = i < 4 ? a : b;
    const int j = i & 3;
    return j == 0 ? q.x : j == 1 ? q.y : j == 2 ? q.z : q.w;
  }
  __device__ void set(const float (&f)[8]) {
    a = make_float4(f[0], f[1], f[2], f[3]);
    b = make_float4(f[4], f[5], f[6], f[7]);
  }
};

// The last n % 8 elements, one by one.
template <bool BF16, bool RES>
__device__ void dropout_tail(const DropoutArgs &A, long long g, const u32 (&u)[4]) {
  for (int i = 0; g * 8 + i < A.n; ++i) {
    const long long at = g * 8 + i;
    const u32 word = i < 2 ? u[0] : i < 4 ? u[1] : i < 6 ? u[2] : u[3];
    const bool keep = (i & 1 ? word >> 16 : word & 0xffffu) >= A.m;
    if constexpr (BF16) {
      auto value = [](const void *p, long long k) { return __builtin_bit_cast(float, (u32) static_cast<const uint16_t *>(p)[k] << 16); };
      float f = keep ? value(A.x, at) * A.scale : 0.0f;
      if (RES) f += value(A.residual, at);
      static_cast<uint16_t *>(A.out)[at] = (uint16_t)pack_bf16(f, 0.0f);
    } else {
      float f = keep ? static_cast<const float *>(A.x)[at] * A.scale : 0.0f;
      if (RES) f += static_cast<const float *>(A.residual)[at];
      static_cast<float *>(A.out)[at] = f;
    }
  }
}

template <bool BF16, bool RES>
__global__ __launch_bounds__(DR_THREADS) void dropout_kernel(DropoutArgs A) {
  const long long whole = A.n >> 3, step = (long long)gridDim.x * DR_THREADS;
  const unsigned long long offset = A.offset + (A.device_offset ? *A.device_offset : 0ull);
  for (long long g = (long long)blockIdx.x * DR_THREADS + threadIdx.x; g * 8 < A.n; g += step) {
    u32 u[4] = {0u, 0u, 0u, 0u};
    if (A.m) philox4x32_10(offset + g, A.seed, u);
    if (g >= whole) {
      dropout_tail<BF16, RES>(A, g, u);
      break;
    }
    Group<BF16> x, r;
    x.load(A.x, g);
    if (RES) r.load(A.residual, g);
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const u32 h = i & 1 ? u[i >> 1] >> 16 : u[i >> 1] & 0xffffu;
      f[i] = h >= A.m ? x.get(i) * A.scale : 0.0f;
      if (RES) f[i] += r.get(i);
    }
    x.set(f);
    x.store(A.out, g);
  }
}

}  // namespace

hipError_t launch_dropout(long long n, int dtype, const void *x, const void *residual, u32 m, unsigned long long seed,
                          unsigned long long offset, const unsigned long long *device_offset, void *out, KernelId id, hipStream_t s) {
  const float scale = m < 65536u ? (float)(65536.0 / (65536.0 - m)) : 0.0f;
  const DropoutArgs A{x, residual, out, n, m, scale, seed, offset, device_offset};
  constexpr long long kMaxBlocks = 1 << 15;
  const long long blocks = (n + 8 * DR_THREADS - 1) / (8 * DR_THREADS);
  const dim3 grid((unsigned)(blocks < kMaxBlocks ? blocks : kMaxBlocks));
  prof_begin(id, s);
  if (dtype == RR_BF16) {
    if (residual) dropout_kernel<true, true><<<grid, DR_THREADS, 0, s>>>(A);
    else dropout_kernel<true, false><<<grid, DR_THREADS, 0, s>>>(A);
  } else {
    if (residual) dropout_kernel<false, true><<<grid, DR_THREADS, 0, s>>>(A);
    else dropout_kernel<false, false><<<grid, DR_THREADS, 0, s>>>(A);
  }
  prof_end(id, s);
  return hipGetLastError();
}

}  // namespace rr
