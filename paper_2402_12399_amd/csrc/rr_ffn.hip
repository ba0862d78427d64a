// Expert FFN as a grouped GEMM over the dispatched rows (Sec. 5.1: every expert is a LLaMA FFN):
//   up   : h[row, f] = silu(x[row] . W1_e[f]) * (x[row] . W3_e[f])      (SwiGLU)
//          h[row, f] = gelu(x[row] . W1_e[f])                            (GELU)
//   down : y[row, c] = h[row] . W2_e[c]
// Both are "A[rows,K] times B[N,K]^T" with K contiguous in both operands.  Rows of expert e are
// row_base[e] .. row_base[e+1]-1 and are cut into row tiles when the routing tables are built (TileInfo).
// The GEMM kernels themselves: rr_gemm.h.  Here: rows of 2^23 elements and more, which tiles a layer uses, the launches.
#include "rr_gemm.h"

namespace rr {

namespace {

// ------------------------------------------------------------------ rows or columns of 2^23 elements and more, bf16 and fp32
// The kernels of rr_gemm.h address a tile's rows with 32-bit byte offsets.  Past kLongRow elements this one takes over, with
// 64-bit addresses: 32 rows x 16 columns (gated: of both matrices) per workgroup, its waves split K, fragments come
// straight from global memory (a lane's 16 bytes are its operand, as above), the partial tiles are summed through
// LDS in a fixed order.  Bound by the latency of its loads; such layers are one or two tiles wide in the
// other dimension, so that splitting K is what fills the chip: 6 rows, 2 experts, 8 x 2^23 bf16: down 10.5 ms, up 5.5 (256 x 256
// tiles: 117 and 5.4); the layer of 2^23 x 24 in fp32 84 ms (64 x 64 tiles of FMAs: 1047).

template <bool BF16, bool GATED, int ACT, bool GATHER, bool DIRECT>
__global__ __launch_bounds__(LG_THREADS) void gemm_long_kernel(GemmArgs P) {
  constexpr int ES = BF16 ? 2 : 4, PE = 16 / ES, KM = 4 * PE, NB = GATED ? 2 : 1;
  using Frag = typename std::conditional<BF16, bf16x8, f32x4>::type;
  __shared__ float red[LG_NW][2 * NB * 4][64];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, r = lane & 15, q = lane >> 4;
  const int N = P.N, NT = P.NT;
  const long long K = P.K, t = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (t >= (long long)P.ctl[0] * NT) return;
  const TileInfo ti = P.tiles[t / NT];
  const int n0 = (int)(t % NT) * LG_COLS;
  const char *a[2], *b[NB];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int lr = min(ti.row0 + i * 16 + r, ti.rows - 1);  // rows past the last one repeat it and are not stored
    long long row = ti.rbase + lr;
    if (GATHER) row = P.row_token ? P.row_token[row] : (lr < ti.fill ? P.slot_token[(size_t)ti.expert * P.C + lr] : P.ir_token[ti.ir_offset + lr - ti.fill]);
    a[i] = static_cast<const char *>(P.A) + (size_t)row * K * ES;
  }
#pragma unroll
  for (int m = 0; m < NB; ++m)
    b[m] = static_cast<const char *>(m ? P.B1 : P.B0) + ((size_t)ti.expert * N + min(n0 + r, N - 1)) * K * ES;
  f32x4 acc[2][NB];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int m = 0; m < NB; ++m) acc[i][m] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  auto fetch = [&](long long k, Frag (&fa)[2], Frag (&fb)[NB]) {
    const bool in = k + q * PE < K;  // K % 8 == 0: a lane's piece is inside or outside as a whole
    const size_t off = (size_t)(in ? k + q * PE : 0) * ES;
    const Frag zero = {};
#pragma unroll
    for (int i = 0; i < 2; ++i) fa[i] = in ? *reinterpret_cast<const Frag *>(a[i] + off) : zero;
#pragma unroll
    for (int m = 0; m < NB; ++m) fb[m] = in ? *reinterpret_cast<const Frag *>(b[m] + off) : zero;
  };
  Frag fa[2], fb[NB], na[2], nb[NB];
  const long long step = (long long)LG_NW * KM;
  fetch((long long)w * KM, fa, fb);
  for (long long k = (long long)w * KM; k < K; k += step) {
    fetch(k + step, na, nb);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int m = 0; m < NB; ++m) {
        // B fragment first, as in the other kernels: lane owns row (lane & 15), columns 4 * (lane >> 4) .. + 3
        if constexpr (BF16) {
          acc[i][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[m], fa[i], acc[i][m], 0, 0, 0);
        } else {
#pragma unroll
          for (int u = 0; u < 4; ++u) acc[i][m] = __builtin_amdgcn_mfma_f32_16x16x4f32(fb[m][u], fa[i][u], acc[i][m], 0, 0, 0);
        }
      }
#pragma unroll
    for (int i = 0; i < 2; ++i) fa[i] = na[i];
#pragma unroll
    for (int m = 0; m < NB; ++m) fb[m] = nb[m];
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int m = 0; m < NB; ++m)
#pragma unroll
      for (int u = 0; u < 4; ++u) red[w][(i * NB + m) * 4 + u][lane] = acc[i][m][u];
  __syncthreads();
  if (tid >= LG_ROWS * LG_COLS) return;
  const int i = w >> 2, u = w & 3;  // wave w < 8 finishes element u of row fragment i
  float c[NB];
#pragma unroll
  for (int m = 0; m < NB; ++m) {
    c[m] = 0.0f;
#pragma unroll
    for (int s = 0; s < LG_NW; ++s) c[m] += red[s][(i * NB + m) * 4 + u][lane];
  }
  if (GATED) c[0] = (BF16 ? silu(c[0]) : c[0] / (1.0f + expf(-c[0]))) * c[NB - 1];
  if (ACT == RR_ACT_GELU) c[0] = gelu_erf(c[0]);
  const int row = ti.row0 + i * 16 + r, col = n0 + 4 * q + u;
  if (row >= ti.rows || col >= N) return;
  const int dest = DIRECT ? P.row_dest[ti.rbase + row] : -1;
  const size_t at = (size_t)(ti.rbase + row) * N + col, to = (size_t)max(dest, 0) * N + col;
  if constexpr (BF16) {
    const uint16_t v = (uint16_t)pack_bf16(c[0], 0.0f);
    static_cast<uint16_t *>(P.Cout)[at] = v;
    if (DIRECT && dest >= 0) static_cast<uint16_t *>(P.Out)[to] = v;
  } else {
    static_cast<float *>(P.Cout)[at] = c[0];
    if (DIRECT && dest >= 0) static_cast<float *>(P.Out)[to] = c[0];
  }
}

// Row tiles of height bm that the layer's rows are expected to make.
long long expected_row_tiles(const Dims &D, int bm) {
  // dispatched rows: the top-k assignments (a dropped token's re-routed row stands for its dropped ones)
  const long long want = (long long)D.T * D.k, R = want < D.Rmax ? want : D.Rmax, used = R < D.E ? R : D.E;
  if (used == 1) return (R + bm - 1) / bm;  // all rows are one expert's
  // a popular expert: its capacity and three times an even share of re-routed tokens; one expert in eight is one
  const long long popular = std::min((long long)D.T, D.C + (D.ir ? 3ll * D.T / D.E : 0)), n_popular = (used + 7) / 8;
  return 4 * R <= 3ll * bm * used ? used + n_popular * ((popular - 1) / bm) : R / bm + used / 2;
}

// Estimated time of a GEMM with tiles of shape q, us; < 0: not possible.  by_rows: 256 x 256 tiles of which only a share of
// the rows is there are priced like the parts of a cut tile (their K loop leaves the missing fragments out).
float shape_cost(const Dims &D, int K, int N, bool up, int q, bool by_rows = false) {
  constexpr int kCUs = 256;  // of the part: a host function, which cannot ask a device (the launch does, see cu_count)
  const bool bf16 = D.dtype == RR_BF16, gated = up && D.act == RR_ACT_SWIGLU;
  const ShapeInfo &s = kShape[q];
  if (q == FFN_P256 && !persistent_ok(K)) return -1.0f;
  const bool split = q == FFN_S128 || q == FFN_S64;
  const int es = bf16 ? 2 : 4, KT = (int)(((long long)K * es + GB_ROW_BYTES - 1) / GB_ROW_BYTES);
  // a tile's rows are addressed with 32-bit byte offsets (below kLongRow elements the narrowest shape always fits)
  if ((long long)K * std::max(s.bm, s.brows) * es >= 1ll << 31) return -1.0f;
  // fp32 rows of up to four chunks: fp32 MFMAs (a tile is mostly its start and end); longer ones: split operands or 32 x 64.  Past 2^20 split
  // tiles, passes of a tenth of a second, nothing was timed: fp32 MFMAs in any of their shapes, as for short rows.
  constexpr int kSplitChunks = 5;
  constexpr long long kSplitTiles = 1ll << 20;
  auto tiles_of = [&](int bm, int brows) { return expected_row_tiles(D, bm) * ((N + (gated ? brows / 2 : brows) - 1) / (gated ? brows / 2 : brows)); };
  const bool can_split = KT >= kSplitChunks && tiles_of(kShape[FFN_S128].bm, kShape[FFN_S128].brows) <= kSplitTiles;
  if (split && (!can_split || tiles_of(s.bm, s.brows) > kSplitTiles)) return -1.0f;
  if ((q == FFN_F64 || q == FFN_F32) && can_split) return -1.0f;
  const float used = (float)std::min<long long>({(long long)D.T * D.k, D.Rmax, D.E});
  const float stream = used * N * K * es * (gated ? 2 : 1) / kHbm;
  const int bn = gated ? s.brows / 2 : s.brows;
  const long long mt = expected_row_tiles(D, s.bm), tiles = mt * ((N + bn - 1) / bn), rounds = tiles / kCUs, left = tiles - rounds * kCUs;
  const float fetch = (float)(s.brows * GB_ROW_BYTES) / kCuFetch * used / (float)mt;
  const float filled = std::min(1.0f, (float)std::min<long long>((long long)D.T * D.k, D.Rmax) / (float)(mt * s.bm));
  const float fixed = s.fixed + filled * (up && q == FFN_256 ? kAct256 : (up && q == FFN_128 ? kAct128 : 0.0f));
  auto part_cost = [&](long long n) { return s.cost * kCutCost[std::min<long long>(n, PK_MAX_CUT) - 1]; };
  const float cost = by_rows ? part_cost((long long)(1.0f / filled)) : s.cost, chunk = std::max(cost, fetch);
  float busy = (float)rounds * (KT * chunk + fixed);
  if (split) {  // three or four workgroups per CU: their number evens out half of the last round
    const float all = (float)tiles / kCUs;
    busy = std::max((0.56f * all + 0.44f * ceilf(all)) * (KT * chunk + fixed), KT * s.alone + fixed);
  } else if (q == FFN_P256) {
    busy += kPersistentStart;
    if (left > 0) busy += KT * std::max(std::min(cost, part_cost(kCUs / left)), fetch) + fixed;
  } else if (left > 0) {  // several workgroups per CU: a round that is nearly empty runs partly under the one before
    busy += (KT * chunk + fixed) * (rounds ? std::min(1.0f, (float)left / kCUs + 0.5f) : 1.0f);
  }
  return std::max(busy, stream) + 0.1f * busy;
}

struct FfnPlan { FfnShape up, down; };
// The pair of shapes with the least cost.  Both GEMMs walk one table of row tiles, as high as the higher of the two: a
// lower shape cuts every row tile of the table (GemmArgs::sub) and launches a workgroup for the cuts that turn out
// to be empty too, about 30 ns each (300 tokens, up 2048 -> 5632: 32-row tiles in a table of 128 rows 269 us, 140 alone).
FfnPlan ffn_plan(const Dims &D) {
  if (std::max(D.d, D.F) >= kLongRow) return {FFN_LONG, FFN_LONG};
  constexpr float kEmpty = 0.031f;
  const int q0 = D.dtype == RR_BF16 ? FFN_P256 : FFN_S128, q1 = D.dtype == RR_BF16 ? FFN_32N : FFN_F32N;
  auto empty = [&](int q, int N, bool gated, int bm) {
    const ShapeInfo &s = kShape[q];
    const int bn = gated ? s.brows / 2 : s.brows;
    const long long cuts = expected_row_tiles(D, bm) * (bm / s.bm) - expected_row_tiles(D, s.bm);
    return kEmpty * (float)(std::max(0ll, cuts) * ((N + bn - 1) / bn));
  };
  // One GEMM in split tiles and the other, though it could be too, in 32 x 64 fp32 ones: only if well ahead.  256 tokens, 6 experts of
  // 77 - 123 rows, 1600 x 5696: 373 us, 329 in 32 x 64 tiles alone; 656 tokens, 12 experts, 1808 x 6632: 671, 642.  Of the 600 layers 23
  // are more than 2 % slower than in fp32 shapes without the margin (up to 12 %), 16 with it, and the mean of all gains 0.2 %.
  constexpr float kMixed = 1.1f;
  auto split = [](int q) { return q == FFN_S128 || q == FFN_S64; };
  FfnPlan best{(FfnShape)q1, (FfnShape)q1};
  float least = -1.0f, up[FFN_F32N + 1], down[FFN_F32N + 1];
  for (int q = q0; q <= q1; ++q) {
    up[q] = shape_cost(D, D.d, D.F, true, q);
    down[q] = shape_cost(D, D.F, D.d, false, q);
  }
  const bool both = D.dtype != RR_BF16 && up[FFN_S64] >= 0.0f && down[FFN_S64] >= 0.0f;
  for (int u = q0; u <= q1; ++u)
    for (int w = q0; w <= q1; ++w) {
      if (!(up[u] >= 0.0f) || !(down[w] >= 0.0f)) continue;
      const int bm = std::max(kShape[u].bm, kShape[w].bm);
      const float sure = both && split(u) != split(w) ? kMixed : 1.0f;
      const float cost = sure * (up[u] + down[w]) + empty(u, D.F, D.act == RR_ACT_SWIGLU, bm) + empty(w, D.d, false, bm);
      if (least < 0.0f || cost <= least) { least = cost; best = {(FfnShape)u, (FfnShape)w}; }
    }
  // Layers that their weights bound - more than the last-level cache holds, and some dozen to a tile's height of rows
  // for each expert: the estimate of lower tiles is at its weakest here, as an expert whose rows need one tile more
  // than expected reads its weights again (it knows no row counts).  One tile per expert, though mostly padding, does not care.
  // 1024 tokens, 32 experts, quotas, 3904 x 11840 SwiGLU: 1715 us in 32 x 128 tiles, 1486 in 256 x 256 ones; 896 tokens, 24
  // experts, 2112 x 6016: 462, 402.  Of 1300 layers timed in every pair of shapes 74 were more than 2 % slower than
  // in 256 x 256 tiles (30 more than 8 %), 47 and 13 with this rule; 5 lose by it, at most 9 %.
  constexpr float kSure = 0.85f;
  constexpr long long kLastLevelBytes = 256ll << 20;
  const long long R = std::min<long long>((long long)D.T * D.k, D.Rmax), used = std::min<long long>(R, D.E);
  if (D.dtype == RR_BF16 && up[FFN_P256] >= 0.0f && down[FFN_P256] >= 0.0f && R >= 24 * used && R <= 256 * used &&
      used * D.d * D.F * 2 >= kLastLevelBytes &&
      kSure * (shape_cost(D, D.d, D.F, true, FFN_P256, true) + shape_cost(D, D.F, D.d, false, FFN_P256, true)) < up[best.up] + down[best.down])
    best = {FFN_P256, FFN_P256};
  return best;
}

template <class F>
void for_each_tile_kernel(F f) {
  auto shape = [&](auto tag) {
    using S = typename decltype(tag)::type;
    if constexpr (S::BF16) {
      f(gemm_tile_kernel<S, true, RR_ACT_SWIGLU, true, false>, S::SMEM);
      f(gemm_tile_kernel<S, true, RR_ACT_SWIGLU, false, false>, S::SMEM);
    }
    f(gemm_tile_kernel<S, true, -1, true, false>, S::SMEM);
    f(gemm_tile_kernel<S, true, -1, false, false>, S::SMEM);
    f(gemm_tile_kernel<S, false, RR_ACT_GELU, true, false>, S::SMEM);
    f(gemm_tile_kernel<S, false, RR_ACT_GELU, false, false>, S::SMEM);
    f(gemm_tile_kernel<S, false, -1, false, true>, S::SMEM);
  };
  for_each_tile_shape(shape);
}

// bf16 SwiGLU layers whose activation is computed with a division, not the hardware's reciprocal
bool swiglu_divides(int K) { return K % GB_BK != 0 || K < 3 * GB_BK; }

// Grid of the small-tile kernel for `tiles` tiles: a grid dimension holds fewer than 2^32 threads (a layer of 2^20 fp32 tokens,
// d_ff 32768, in 32 x 64 outputs has 2^24 tiles of 256 threads), so more tiles make rows of whole XCD runs.
dim3 tile_grid(long long tiles) {
  constexpr long long kRow = 1ll << 20;
  return dim3((unsigned)((std::min(tiles, kRow) + 7) / 8 * 8), (unsigned)((tiles + kRow - 1) / kRow));
}
int column_tiles(const ShapeInfo &s, int N, bool gated) {
  const int bn = gated ? s.brows / 2 : s.brows;
  return (int)(((long long)N + bn - 1) / bn);
}

// One GEMM (UP or down) with tiles of shape S; grid: the most tiles there can be.
template <class S, bool UP>
void launch_tiles(const Dims &D, GemmArgs g, bool fuse, hipStream_t s) {
  const bool gated = UP && D.act == RR_ACT_SWIGLU;
  g.NT = column_tiles(ShapeInfo{S::BM, S::BROWS, 0.0f, 0.0f}, g.N, gated);
  g.sub = D.BM / S::BM;
  const dim3 grid = tile_grid((long long)g.NT * D.max_mtiles * g.sub);
  if constexpr (UP && S::BF16) {
    if (gated && swiglu_divides(g.K)) {
      if (fuse) gemm_tile_kernel<S, true, RR_ACT_SWIGLU, true, false><<<grid, S::THREADS, S::SMEM, s>>>(g);
      else gemm_tile_kernel<S, true, RR_ACT_SWIGLU, false, false><<<grid, S::THREADS, S::SMEM, s>>>(g);
      return;
    }
  }
  if constexpr (UP) {
    if (gated && fuse) gemm_tile_kernel<S, true, -1, true, false><<<grid, S::THREADS, S::SMEM, s>>>(g);
    else if (gated) gemm_tile_kernel<S, true, -1, false, false><<<grid, S::THREADS, S::SMEM, s>>>(g);
    else if (fuse) gemm_tile_kernel<S, false, RR_ACT_GELU, true, false><<<grid, S::THREADS, S::SMEM, s>>>(g);
    else gemm_tile_kernel<S, false, RR_ACT_GELU, false, false><<<grid, S::THREADS, S::SMEM, s>>>(g);
  } else {
    gemm_tile_kernel<S, false, -1, false, true><<<grid, S::THREADS, S::SMEM, s>>>(g);
  }
}

template <bool BF16, bool UP>
void launch_long(const Dims &D, GemmArgs g, bool fuse, hipStream_t s) {
  g.NT = (int)(((long long)g.N + LG_COLS - 1) / LG_COLS);
  const dim3 grid = tile_grid((long long)g.NT * D.max_mtiles);
  if constexpr (UP) {
    const bool gated = D.act == RR_ACT_SWIGLU;
    if (gated && fuse) gemm_long_kernel<BF16, true, -1, true, false><<<grid, LG_THREADS, 0, s>>>(g);
    else if (gated) gemm_long_kernel<BF16, true, -1, false, false><<<grid, LG_THREADS, 0, s>>>(g);
    else if (fuse) gemm_long_kernel<BF16, false, RR_ACT_GELU, true, false><<<grid, LG_THREADS, 0, s>>>(g);
    else gemm_long_kernel<BF16, false, RR_ACT_GELU, false, false><<<grid, LG_THREADS, 0, s>>>(g);
  } else {
    gemm_long_kernel<BF16, false, -1, false, true><<<grid, LG_THREADS, 0, s>>>(g);
  }
}

template <bool UP>
void launch_gemm(FfnShape shape, const Dims &D, GemmArgs g, bool fuse, hipStream_t s) {
  switch (shape) {
    case FFN_P256: {
      const bool gated = UP && D.act == RR_ACT_SWIGLU;
      g.NT = gated ? (g.N + 127) / 128 : (g.N + 255) / 256;
      const int cus = cu_count();
      if constexpr (UP) {
        const bool ragged = swiglu_divides(g.K);  // (ACT RR_ACT_SWIGLU: with the division)
        if (gated && fuse && ragged) gemm_bf16_persistent_kernel<true, RR_ACT_SWIGLU, true><<<cus, PK_THREADS, PK_SMEM, s>>>(g);
        else if (gated && ragged) gemm_bf16_persistent_kernel<true, RR_ACT_SWIGLU, false><<<cus, PK_THREADS, PK_SMEM, s>>>(g);
        else if (gated && fuse) gemm_bf16_persistent_kernel<true, -1, true><<<cus, PK_THREADS, PK_SMEM, s>>>(g);
        else if (gated) gemm_bf16_persistent_kernel<true, -1, false><<<cus, PK_THREADS, PK_SMEM, s>>>(g);
        else if (fuse) gemm_bf16_persistent_kernel<false, RR_ACT_GELU, true><<<cus, PK_THREADS, PK_SMEM, s>>>(g);
        else gemm_bf16_persistent_kernel<false, RR_ACT_GELU, false><<<cus, PK_THREADS, PK_SMEM, s>>>(g);
      } else {
        gemm_bf16_persistent_kernel<false, -1, false, true><<<cus, PK_THREADS, PK_SMEM, s>>>(g);
      }
      break;
    }
    case FFN_256: launch_tiles<TileB256, UP>(D, g, fuse, s); break;
    case FFN_128: launch_tiles<TileB128, UP>(D, g, fuse, s); break;
    case FFN_64: launch_tiles<TileB64, UP>(D, g, fuse, s); break;
    case FFN_32: launch_tiles<TileB32, UP>(D, g, fuse, s); break;
    case FFN_32N: launch_tiles<TileB32n, UP>(D, g, fuse, s); break;
    case FFN_S128: launch_tiles<TileS128, UP>(D, g, fuse, s); break;
    case FFN_S64: launch_tiles<TileS64, UP>(D, g, fuse, s); break;
    case FFN_F64: launch_tiles<TileF64, UP>(D, g, fuse, s); break;
    case FFN_F32: launch_tiles<TileF32, UP>(D, g, fuse, s); break;
    case FFN_F32N: launch_tiles<TileF32n, UP>(D, g, fuse, s); break;
    case FFN_LONG:
      if (D.dtype == RR_BF16) launch_long<true, UP>(D, g, fuse, s);
      else launch_long<false, UP>(D, g, fuse, s);
      break;
  }
}

}  // namespace

// The GEMM kernels use more dynamic LDS than the default limit.  Raising it is host-side set-up of the
// loaded code object on the current device (no stream work); the caller runs it once per device.
hipError_t ffn_kernel_attributes() {
  hipError_t e = hipSuccess;
  auto set = [&e](auto kern, int bytes) {
    if (e == hipSuccess) e = set_lds(kern, bytes);
  };
  set(gemm_bf16_persistent_kernel<true, RR_ACT_SWIGLU, true>, PK_SMEM);
  set(gemm_bf16_persistent_kernel<true, RR_ACT_SWIGLU, false>, PK_SMEM);
  set(gemm_bf16_persistent_kernel<true, -1, true>, PK_SMEM);
  set(gemm_bf16_persistent_kernel<true, -1, false>, PK_SMEM);
  set(gemm_bf16_persistent_kernel<false, RR_ACT_GELU, true>, PK_SMEM);
  set(gemm_bf16_persistent_kernel<false, RR_ACT_GELU, false>, PK_SMEM);
  set(gemm_bf16_persistent_kernel<false, -1, false, true>, PK_SMEM);
  for_each_tile_kernel(set);
  return e;
}

// Row-tile height of the layer's tile table: the higher of the two GEMMs' tiles.
int ffn_row_tile(const Dims &D) {
  const FfnPlan plan = ffn_plan(D);
  return std::max(kShape[plan.up].bm, kShape[plan.down].bm);
}

void ffn_describe(const Dims &D, FfnShapes *out) {
  const FfnPlan plan = ffn_plan(D);
  const FfnShape q[2] = {plan.up, plan.down};
  for (int i = 0; i < 2; ++i) {
    out->bm[i] = kShape[q[i]].bm;
    out->brows[i] = kShape[q[i]].brows;
    out->cost[i] = shape_cost(D, i ? D.F : D.d, i ? D.d : D.F, i == 0, q[i]);
  }
}

bool ffn_fuses_gather(const Dims &D) { return (long long)D.T * D.d * (D.dtype == RR_BF16 ? 2 : 4) < 0x7ffffff0ll; }

hipError_t launch_ffn(const Dims &D, const void *x, const rr_tables &tb, const void *w1, const void *w3,
                      const void *w2, const Work &W, void *out, hipStream_t s) {
  const bool fuse = ffn_fuses_gather(D);
  const FfnPlan plan = ffn_plan(D);
  const GemmArgs up{fuse ? x : W.x_disp, w1, w3, W.h, D.d, D.F, 0, 1, W.tiles, W.tile_ctl,
                    tb.slot_token, tb.ir_token, D.quota ? W.row_token : nullptr, D.C,
                    (long long)D.T * D.d * (D.dtype == RR_BF16 ? 2 : 4), nullptr, nullptr};
  const GemmArgs down{W.h, w2, nullptr, W.y, D.F, D.d, 0, 1, W.tiles, W.tile_ctl, nullptr, nullptr, nullptr, 0, 0, W.row_dest, out};
  prof_begin(K_FFN_UP, s);
  launch_gemm<true>(plan.up, D, up, fuse, s);
  prof_end(K_FFN_UP, s);
  prof_begin(K_FFN_DOWN, s);
  launch_gemm<false>(plan.down, D, down, fuse, s);
  prof_end(K_FFN_DOWN, s);
  return hipGetLastError();
}

}  // namespace rr
