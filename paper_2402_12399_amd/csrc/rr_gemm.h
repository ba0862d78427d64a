// Matrix products "A[rows, K] times B[N, K]^T" with K contiguous in both operands, fp32 accumulation: the kernels of the grouped
// expert GEMM (rr_ffn.hip) and of the dense projections (rr_linear.hip).
//
// Large bf16 layers: persistent kernel, one workgroup of 8 waves per CU, tiles of 256 x 256 staged rows
// dealt in an XCD-aware panel order (see "Tile order" in the kernel).
//   * v_mfma_f32_16x16x32_bf16, fp32 accumulate; 2 x 4 waves, wave tile 128 x 64; two waves per SIMD
//     so that one wave's LDS reads overlap the other's MFMAs.  (A loop of MFMAs alone on normally
//     distributed operands sustains 2030 TFLOP/s with this shape and 1330 with 32x32x16, 2470 and 1670
//     on zeros: the wide shape was the kernel's ceiling.)
//   * K advances in chunks of 64 through LDS rings - two 32 KB stages of A, three of B, 160 KB in all
//     - filled by buffer_load ... lds (16 bytes per lane straight into LDS, no staging registers);
//     the chunks of a workgroup's successive tiles form one stream.  A wave instruction fills 1 KB = 8
//     consecutive LDS rows (lane l -> row l/8, chunk position l%8), so the swizzle is applied on the
//     global side: the lane fetches the chunk that belongs at its position.  Rows past the end of
//     an operand read as zero (buffer range check): ragged tiles need no masks on the load side.
//   * LDS rows are 128 B; chunk c of row r sits at position c ^ ((r >> 1) & 7): conflict-free for
//     the 16 lanes x 16 B that the 64-bank LDS serves per cycle, for the DMA writes as well.
//   * The K loop is software-pipelined by hand (see k_loop): the compiler's own schedule waits for
//     every LDS read right before its first use.
//   * The up projection can read its A rows straight from x through the dispatch tables (GATHER):
//     the dispatch gather is then a per-lane row offset of the LDS DMA and costs no pass over HBM.
//   * The last round of tiles rarely fills the chip: where its tiles are at most half as many as the
//     workgroups they are cut by rows into up to eight parts (see "cut").  8 K tokens top-1, 2048 x 5632: down
//     projection 292 -> 249 us (384 tiles for 256 CUs); 4 K tokens 4096 x 11008, top-2: down 829 -> 695 (576 tiles).
//     The waves of a column take turns at the 16-row fragments, so that a short tile keeps all four SIMDs busy.
//   * While a tile's epilogue stores drain, the first K chunk of the workgroup's next tile is
//     already in flight (its tile id and table entries were fetched during the K loop).
// Layers with few rows or short rows, and all fp32 layers: gemm_tile_kernel, smaller tiles of several shapes
// (ffn_plan chooses the pair).
#pragma once

#include <algorithm>
#include <type_traits>

#include "rr_device.h"

namespace rr {

namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;

// Scheduling groups for the instruction scheduler (masks of sched_group_barrier: 0x008 MFMA,
// 0x100 LDS read, 0x020 global or buffer load).  They order the instructions of the surrounding
// scheduling region only; what the instructions compute is untouched.
// N times "one MFMA, then one LDS read":
template <int N>
__device__ __forceinline__ void sched_mfma_lds_read() {
  if constexpr (N > 0) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    sched_mfma_lds_read<N - 1>();
  }
}
// As many pairs of reads (turned operands):
template <int N>
__device__ __forceinline__ void sched_mfma_two_lds_reads() {
  if constexpr (N > 0) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    sched_mfma_two_lds_reads<N - 1>();
  }
}
// The step's R LDS reads and then its D LDS-DMA loads, each behind one of the step's first MFMAs.  The loads come last, as in
// the source: they write LDS, so the compiler moves no LDS read across them, and groups that ask for a load between two
// reads are not followed at all (the reads then run in one burst; 16384 tokens x 4096 x 11008: gate/up 4.66 -> 4.50 ms,
// down 2.34 -> 2.24, the MFMA pipe's share of the busy cycles 0.71 -> 0.77, the clock 1.75 -> 1.71 GHz).
// P: LDS reads behind one MFMA (turned operands take two reads per fragment).
template <int M, int R, int D, int P = 1>
__device__ __forceinline__ void sched_step() {
  if constexpr (M > 0 && R > 0) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, R < P ? R : P, 0);
    sched_step<M - 1, (R < P ? 0 : R - P), D, P>();
  } else if constexpr (M > 0 && D > 0) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
    sched_step<M - 1, 0, D - 1, P>();
  }
}

__device__ inline float silu(float g) { return g / (1.0f + __expf(-g)); }
// for results that are rounded to bf16 right away, in layers of whole K chunks, three at least (swiglu_divides): hardware
// reciprocal (1 ulp; 0 for arguments below -87.4, where the result is below 2e-36) instead of a division.  300 tokens, 2048 x
// 5632, 16 experts, 128 x 128 tiles: the layer 235 us, with the division 237.
__device__ inline float silu_fast(float g) { return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }

// (bf16 results: the exponential and the division of the hardware, 2 ulp together, are far below the rounding)
template <bool BF16>
__device__ inline float dense_silu(float g) {
  return BF16 ? silu(g) : g / (1.0f + expf(-g));
}

// g Phi(g) = max(g, 0) - |g| Phi(-|g|).  For results that are rounded to bf16: Phi(-|g|) = exp(-g^2 / 2) t R(t), t = 1 / (1 + 0.55 |g| / sqrt 2),
// R a polynomial of degree 5 fitted to exp(x^2) erfc(x) / (2 t) so that Phi's absolute error is small: 2.6e-8 with these coefficients, 1.5e-7
// computed in fp32, and the result's 2.5e-7.  No branches: 8192 rows, 2048 -> 11264: 57 us more than without an activation with erff, 25 so.
template <bool BF16>
__device__ inline float dense_gelu(float g) {
  if (!BF16) return gelu_erf(g);
  const float a = fminf(fabsf(g), 30.0f), t = __builtin_amdgcn_rcpf(fmaf(a, 0.55f * 0.70710678118654752f, 1.0f));
  const float e = __builtin_amdgcn_exp2f(g * g * (-0.5f * 1.44269504088896341f));  // (of g itself: NaN stays)
  float r = 0.0536629334f;
  r = fmaf(r, t, -0.259021938f);
  r = fmaf(r, t, 0.379861683f);
  r = fmaf(r, t, -0.0207166243f);
  r = fmaf(r, t, 0.195422441f);
  r = fmaf(r, t, 0.150791496f);
  return fmaf(-a, t * e * r, fmaxf(g, 0.0f));
}

constexpr int GB_BK = 64;             // bf16 elements per K chunk = 128 B per LDS row
constexpr int GB_ROW_BYTES = 128;
[[maybe_unused]] constexpr u32 BUF_FLAGS = 0x00020000; // raw buffer descriptor word 3 (32-bit data format)
[[maybe_unused]] constexpr int BUF_STREAM = 2;           // cache policy of a load: not kept for another reader (nontemporal)

struct GemmArgs {
  const void *A;        // [rows, K] dispatched rows; with GATHER: x [T, K]
  const void *B0;       // [E, N, K]
  const void *B1;       // [E, N, K] gated only
  void *Cout;           // [rows, N]
  int K, N;
  int NT;               // column tiles
  int sub;              // small-tile kernel: row tiles per row tile of the table
  const TileInfo *tiles;
  const int32_t *ctl;   // [0] number of row tiles
  // GATHER only
  const int32_t *slot_token, *ir_token;
  const int32_t *row_token;  // token of every dispatched row (per-group quotas), or NULL: rows are slots, then the Intra-GPU list
  int C;
  long long a_bytes;    // size of the A operand in bytes (buffer range of the gather)
  // DIRECT only (down projection): row_dest[row] = the token whose only processed row this is, else -1;
  // such a row is also stored as row row_dest[row] of Out, the layer's output (Eq. 2 with a single term)
  const int32_t *row_dest;
  void *Out;
};

// A dense product (rr_linear.hip): no table of tiles, rows 0 .. M - 1, and in place of the experts equal slices of the
// summation, whose raw sums go to `part` when there are several.
struct DenseArgs : GemmArgs {  // K: elements of a slice
  int M, MT;             // rows, row tiles
  int slices;
  int lda, ldb;          // elements between rows of A and of B (turned operands: of their memory)
  int Kall;              // elements of the whole summation
  const float *bias;     // [R], R = N, gated 2 N (B1 = B0 + N rows); or NULL
  const void *residual;  // [M, N] or NULL
  void *pre;             // [M, R] or NULL
  float *part;           // [slices, M, R] or NULL
};

// Two neighbouring 16x16 accumulators of a lane (four columns 4 * fg .. + 3 of column fragments j and j + 1, as bf16 pairs) ->
// eight columns in a row, eight_columns_at(fg) .. + 7 from fragment j on: lanes 16 apart exchange halves.  16384 tokens,
// 4096 x 11008, top-2: gate/up 4.47 -> 4.41 ms, down 2.25 -> 2.22; 8192 tokens, 2048 x 5632: down 272 -> 265 us.
__device__ __forceinline__ int eight_columns_at(int fg) { return (fg & 1) * 16 + (fg >> 1) * 8; }
__device__ __forceinline__ uint4 eight_columns(uint2 a, uint2 b) {
  const auto x = __builtin_amdgcn_permlane16_swap(a.x, b.x, false, false), y = __builtin_amdgcn_permlane16_swap(a.y, b.y, false, false);
  return make_uint4(x[0], y[0], x[1], y[1]);
}

// Epilogue of the persistent kernel, which multiplies with the operands swapped (B fragment first):
// the 16x16 accumulator then holds the transposed tile, i.e. a lane owns ONE output row (lane % 16 of
// the A fragment) and four consecutive columns, 4 * (lane / 16) .. + 3 of the B fragment; two accumulators make one
// 16-byte store per lane, 64 bytes of each of 16 rows.
// dest (DIRECT): per fragment row of this lane, the row of Ob that the same values are also stored to, or -1.
// The WAVES_M waves of a column take turns at the 16-row fragments of the tile.
template <int WM, int WN, int WAVES_M, bool GATED, int ACT, bool DIRECT = false>
__device__ inline void store_tile_t(f32x4 (&acc)[WM][WN], uint16_t *Cb, int rbase, int rows_e, int m0, int n0, int N,
                                    int wm, int wn, int lane, const int *dest = nullptr, uint16_t *Ob = nullptr) {
  constexpr int NJ = GATED ? WN / 2 : WN;  // output column fragments per wave
  const int fr = lane & 15, fg = lane >> 4;
  const int wrow0 = m0 + wm * 16, wcol0 = n0 + wn * NJ * 16;
  const bool cols_in = wcol0 + NJ * 16 <= N;  // N % 8 == 0: a group of eight columns is inside or outside as a whole
  const int ecol = eight_columns_at(fg);
#pragma unroll
  for (int i = 0; i < WM; ++i) {
    const int row = wrow0 + i * WAVES_M * 16 + fr;
    if (row >= rows_e) continue;
    uint16_t *prow = Cb + (size_t)(rbase + row) * N + wcol0 + ecol;
    uint16_t *orow = nullptr;
    if (DIRECT && dest[i] >= 0) orow = Ob + (size_t)dest[i] * N + wcol0 + ecol;
#pragma unroll
    for (int j = 0; j < NJ; j += 2) {
      uint2 v[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float c[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          c[u] = acc[i][j + h][u];
          if (GATED) c[u] = (ACT == RR_ACT_SWIGLU ? silu(c[u]) : silu_fast(c[u])) * acc[i][j + h + NJ][u];
          if (ACT == RR_ACT_GELU) c[u] = gelu_erf(c[u]);
        }
        v[h] = make_uint2(pack_bf16(c[0], c[1]), pack_bf16(c[2], c[3]));
      }
      const uint4 val = eight_columns(v[0], v[1]);
      if (cols_in || wcol0 + j * 16 + ecol < N) {
        *reinterpret_cast<uint4 *>(prow + j * 16) = val;
        if (DIRECT && orow) *reinterpret_cast<uint4 *>(orow + j * 16) = val;
      }
    }
  }
}

// Output of a dense product in the same layout: row fragment i is rows row0 + i * STEP (row0: of this lane), the wave's columns
// start at col0.  Gated: the first half of the column fragments are the gate's, the second the up projection's.
template <int WM, int WN, int STEP, bool BF16, bool GATED, int ACT>
__device__ inline void store_dense(f32x4 (&acc)[WM][WN], const DenseArgs &P, int slice, int row0, int rows_end, int col0, int lane) {
  constexpr int NJ = GATED ? WN / 2 : WN, ES = BF16 ? 2 : 4;
  constexpr bool PAIRS = BF16 && NJ % 2 == 0;
  const int fg = lane >> 4, N = P.N, R = GATED ? 2 * N : N;
  if (P.part) {
#pragma unroll
    for (int i = 0; i < WM; ++i) {
      const int row = row0 + i * STEP;
      if (row >= rows_end) continue;
      float *to = P.part + ((size_t)slice * P.M + row) * R;
#pragma unroll
      for (int j = 0; j < WN; ++j) {
        const int col = col0 + (j % NJ) * 16 + 4 * fg;
        if (col < N) *reinterpret_cast<f32x4 *>(to + (j >= NJ ? N : 0) + col) = acc[i][j];
      }
    }
    return;
  }
  f32x4 bias[WN];
#pragma unroll
  for (int j = 0; j < WN; ++j) {
    bias[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int col = col0 + (j % NJ) * 16 + 4 * fg;
    if (P.bias && col < N)
#pragma unroll
      for (int u = 0; u < 4; ++u) bias[j][u] = P.bias[(j >= NJ ? N : 0) + col + u];
  }
  // the residual of RH row fragments at a time is under way before the first is needed (the K loop's fragments are free by now)
  constexpr int RH = WM > 4 ? 4 : WM;
  using Res = typename std::conditional<BF16, uint2, float4>::type;
  Res res_raw[RH][NJ];
#pragma unroll
  for (int i = 0; i < WM; ++i) {
    if (P.residual && i % RH == 0) {
#pragma unroll
      for (int h = 0; h < RH; ++h)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const int row = row0 + (i + h) * STEP, col = col0 + j * 16 + 4 * fg;
          if (row < rows_end && col < N)
            res_raw[h][j] = *reinterpret_cast<const Res *>(static_cast<const char *>(P.residual) + ((size_t)row * N + col) * ES);
        }
    }
    const int row = row0 + i * STEP;
    if (row >= rows_end) continue;
    // four columns of fragment j at `at`, the start of a row; even: the fragment before it (PAIRS)
    auto put = [&](char *at, int j, const float (&c)[4], uint2 &even) {
      if constexpr (BF16) {
        const uint2 v = make_uint2(pack_bf16(c[0], c[1]), pack_bf16(c[2], c[3]));
        if constexpr (PAIRS) {
          if (j % 2 == 0) {
            even = v;
            return;
          }
          const uint4 both = eight_columns(even, v);
          const int col = col0 + (j - 1) * 16 + eight_columns_at(fg);
          if (col < N) *reinterpret_cast<uint4 *>(at + (size_t)col * ES) = both;
        } else {
          const int col = col0 + j * 16 + 4 * fg;
          if (col < N) *reinterpret_cast<uint2 *>(at + (size_t)col * ES) = v;
        }
      } else {
        const int col = col0 + j * 16 + 4 * fg;
        if (col < N) *reinterpret_cast<float4 *>(at + (size_t)col * ES) = make_float4(c[0], c[1], c[2], c[3]);
      }
    };
    uint2 even_y = make_uint2(0, 0), even_g = even_y, even_u = even_y;
    char *yrow = static_cast<char *>(P.Cout) + (size_t)row * N * ES, *prow = static_cast<char *>(P.pre) + (size_t)row * R * ES;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int col = col0 + j * 16 + 4 * fg;
      float g[4], up[4], y[4], res[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      if (P.residual && col < N) {
        const Res v = res_raw[i % RH][j];
        if constexpr (BF16) {
          res[0] = __builtin_bit_cast(float, v.x << 16);
          res[1] = __builtin_bit_cast(float, v.x & 0xffff0000u);
          res[2] = __builtin_bit_cast(float, v.y << 16);
          res[3] = __builtin_bit_cast(float, v.y & 0xffff0000u);
        } else {
          res[0] = v.x; res[1] = v.y; res[2] = v.z; res[3] = v.w;
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        g[u] = acc[i][j][u] + bias[j][u];
        up[u] = GATED ? acc[i][GATED ? j + NJ : j][u] + bias[GATED ? j + NJ : j][u] : 0.0f;
        y[u] = GATED ? dense_silu<BF16>(g[u]) * up[u] : ACT == RR_ACT_GELU ? dense_gelu<BF16>(g[u]) : g[u];
        y[u] += res[u];
      }
      if (P.pre) {
        put(prow, j, g, even_g);
        if (GATED) put(prow + (size_t)N * ES, j, up, even_u);
      }
      put(yrow, j, y, even_y);
    }
  }
}

__device__ inline int swz(int r) { return (r >> 1) & 7; }

// Barrier that publishes LDS-DMA data.  Before it signals, a wave's own buffer_load ... lds must
// have written LDS - all of them but the youngest YOUNGER, which belong to a later chunk (memory
// instructions complete in order) - and its own fragment reads of the stage that is about to be
// refilled must have returned (lgkmcnt 0).  Spelled out in assembly: the compiler's barrier waits
// for what its memory model takes for LDS traffic only, and when it does drain vmcnt it drains all.
template <int YOUNGER>
__device__ inline void dma_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(YOUNGER) : "memory");
}

// ------------------------------------------------------------------ bf16, persistent, LDS DMA
constexpr int PK_WAVES_M = 2, PK_WAVES_N = 4, PK_WM = 8, PK_WN = 4;  // waves, and 16-row fragments of a wave: 128 x 64
constexpr int PK_NW = PK_WAVES_M * PK_WAVES_N;
constexpr int PK_THREADS = PK_NW * 64;
constexpr int PK_BM = PK_WAVES_M * PK_WM * 16;     // 256
constexpr int PK_BROWS = PK_WAVES_N * PK_WN * 16;  // 256 staged B rows
constexpr int PK_A_STAGE = PK_BM * GB_ROW_BYTES, PK_B_STAGE = PK_BROWS * GB_ROW_BYTES;
[[maybe_unused]] constexpr int PK_MAX_CUT = 8;
constexpr int PK_A_STAGES = 2, PK_B_STAGES = 3;
constexpr int PK_B_BASE = PK_A_STAGES * PK_A_STAGE;
constexpr int PK_SMEM = PK_B_BASE + PK_B_STAGES * PK_B_STAGE;  // 160 KB: all of a CU's LDS
[[maybe_unused]] constexpr int PK_NI = (PK_BM + PK_BROWS) / 8 / PK_NW;  // 1 KB load instructions per wave per chunk
[[maybe_unused]] constexpr int PK_NIA = PK_BM / 8 / PK_NW;

// Part `part` of a tile of `rows` rows from m0 on that is cut into `cut`: an equal share in whole fragments of both waves, which may leave
// the last parts short or empty (m0 >= end).  No part passes the tile's end: a row computed twice adds its residual twice where y
// lies in the residual's place.
struct CutRows { int m0, end; };
__host__ __device__ inline CutRows cut_rows(int m0, int rows, int cut, int part) {
  const int h = (rows + cut * 32 - 1) / (cut * 32) * 32, a = part * h, b = a + h;
  return {m0 + a, m0 + (b < rows ? b : rows)};
}

// Turned operands (TA, TB; dense products, bf16): the summation runs down the memory's rows, as in dx = dz W and dw = dz^T x.  A
// chunk is then 64 memory rows of as many neighbouring columns as the tile has rows, staged as they lie (a DMA instruction fills
// 1 KB of them), and the fragments come out of LDS through ds_read_b64_tr_b16: 16 lanes name the 4 pieces of 8 bytes of each of
// 4 rows, and lane l gets column l of the four.  A lane's eight elements are two such reads, rows 8 g .. + 3 and + 4 .. + 7
// (g = lane / 16), as in an operand that is not turned.  32-byte unit c of staged row k sits at c ^ turn_swz(k): the eight rows that
// 32 lanes read at once then lie in different eighths of the 64 banks, whatever the row's length RB (64 to 512 bytes; four or two short
// rows share the banks).  Rows past the end of the summation read as zero (range check), columns past the operand's edge hold
// the next row's and are not stored.
template <int RB>
__device__ inline int turn_swz(int k) {
  return RB >= 256 ? (k & 3) | (k >> 1 & 4) : RB == 128 ? (k >> 1 & 1) | (k >> 2 & 2) : k >> 3 & 1;
}
typedef short i16x4 __attribute__((ext_vector_type(4)));
// This lane's place in a DMA instruction that fills staged rows from `first` on: its row, and the byte of the memory row it fetches.
template <int RB>
__device__ inline void turned_lane(int first, int lane, int &row, int &byte) {
  row = first + lane / (RB / 16);
  byte = ((lane % (RB / 16)) ^ turn_swz<RB>(row) << 1) * 16;
}
// This lane's first row of a 32 x 16 fragment of unit c.
template <int RB>
__device__ inline int turned_at(int c, int fr, int fg) {
  const int k = 8 * fg + (fr >> 2);
  return k * RB + (c ^ turn_swz<RB>(k)) * 32 + (fr & 3) * 8;
}
// A turned fragment of 32 x 16 elements whose first row of this lane is at `at` in LDS.  (__restrict__ is not about aliases here: it
// leaves a scope on the reads, without which the compiler takes them for possible readers of every DMA load under way and drains
// those, vmcnt(0), before each group of reads.)
template <int RB>
__device__ __forceinline__ bf16x8 read_turned(const char *__restrict__ at) {
#if defined(__HIP_DEVICE_COMPILE__)
  const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)at);
  const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(at + 4 * RB));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#else
  return bf16x8{};
#endif
}

template <bool GATED, int ACT, bool GATHER, bool DIRECT = false, bool DENSE = false, bool TA = false, bool TB = false>
__global__ __launch_bounds__(PK_THREADS) void gemm_bf16_persistent_kernel(typename std::conditional<DENSE, DenseArgs, GemmArgs>::type P) {
#if defined(__HIP_DEVICE_COMPILE__)  // buffer-resource and LDS-DMA builtins exist in the device pass only
  constexpr int WM = PK_WM, WN = PK_WN, NW = PK_NW, BM = PK_BM, NI = PK_NI, NIA = PK_NIA;
  constexpr int BN = GATED ? PK_BROWS / 2 : PK_BROWS;
  constexpr int NIB0 = BN / 8 / NW;
  static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "operand boundaries must fall between load instructions");
  static_assert(!(TA || TB) || (DENSE && !GATED && !GATHER));
  extern __shared__ __attribute__((aligned(16))) char smem[];

  const int K = P.K, N = P.N, NT = P.NT, KT = (K + GB_BK - 1) / GB_BK;
  // Tile order.  Workgroups are dealt to the 8 XCDs round-robin (workgroup g runs on XCD g % 8) and
  // each XCD has its own L2.  The tiles are numbered panel by panel - panels of pm x pn neighbouring
  // tiles (4 row tiles x 8 column tiles for 32 workgroups per XCD), column panels first, ragged at the
  // right and bottom edges of the tile grid - and each run of pm * pn consecutive numbers goes to the
  // workgroups of one XCD: a chunk of an A row tile is then fetched into that L2 once for pn tiles
  // and a chunk of a B column tile once for pm, instead of once per tile, and consecutive rounds of
  // an XCD stay on the same rows of the same expert.
  int MT;
  if constexpr (DENSE) MT = P.MT * P.slices;
  else MT = P.ctl[0];
  const int total = MT * NT;
  const int G = gridDim.x;
  const int nX = (G & 7) == 0 ? 8 : 1, S = G / nX;
  const int pn = (S & 7) == 0 ? 8 : 1, pm = S / pn;
  const int xcd = blockIdx.x % nX, slot = blockIdx.x / nX;
  const int PMf = MT / pm, PNf = NT / pn;  // full panel rows / columns
  // tile number k (panel order) -> linear index mt * NT + nt
  auto tile_at = [&](int k) {
    int qm = k / (pm * NT);
    if (qm > PMf) qm = PMf;
    const int r = k - qm * pm * NT, h = qm < PMf ? pm : MT - PMf * pm;
    int qn = r / (h * pn);
    if (qn > PNf) qn = PNf;
    const int r2 = r - qn * h * pn, wd = qn < PNf ? pn : NT - PNf * pn;
    const int dm = r2 / wd, dn = r2 - dm * wd;
    return (qm * pm + dm) * NT + qn * pn + dn;
  };
  // This workgroup's i-th tile is number (i * nX + xcd) * S + slot.  The tiles of the last, partial round are
  // spread over the XCDs and, where they are at most half as many as the workgroups, cut by rows into up to
  // PK_MAX_CUT parts that different workgroups take.
  const int rounds = total / G, left = total - rounds * G;
  const int cut = left > 0 ? min(G / left, PK_MAX_CUT) : 1;
  const int units = left * cut, per_xcd = (units + nX - 1) / nX;
  // tile of round i and, in the last round, which part of it; -1: none
  struct Unit { int L, part; };
  auto unit_at = [&](int i) {
    if (i < rounds) return Unit{tile_at((i * nX + xcd) * S + slot), -1};
    const int u = xcd * per_xcd + slot;
    if (i > rounds || slot >= per_xcd || u >= units) return Unit{-1, -1};
    return Unit{tile_at(rounds * G + u / cut), cut > 1 ? u % cut : -1};
  };
  int round = 0;
  Unit U = unit_at(0), U1 = unit_at(1), U2 = unit_at(2);  // this workgroup's current tile and the two after it
  if (U.L < 0) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);  // wave-uniform: keeps LDS-DMA addressing scalar
  const int wm = w / PK_WAVES_N, wn = w % PK_WAVES_N;
  const int fr = lane & 15, fg = lane >> 4;

  // fragment addressing (the same for every tile): lane reads row (lane & 15), chunk 4*ks + (lane >> 4)
  const int fsw = swz(fr);  // fragment rows start at multiples of 16, so the swizzle depends on fr only
  const int a_off = (wm * 16 + fr) * GB_ROW_BYTES;  // fragment i: + i * PK_WAVES_M * 16 rows
  // gated: the first half of a wave's column fragments are gate columns, the second the matching up columns
  const int b_off = (wn * (GATED ? WN / 2 : WN) * 16 + fr) * GB_ROW_BYTES;
  // turned operands: the lane's offset for fragment i (A: i % 4; the others are 256 bytes further), first row
  int a_turn[4], b_turn[WN];
  constexpr int TRB = PK_BM * 2;  // bytes of a staged row
  static_assert(PK_BROWS == PK_BM);
  if constexpr (TA || TB) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a_turn[i] = turned_at<TRB>(i * PK_WAVES_M + wm, fr, fg);
#pragma unroll
    for (int j = 0; j < WN; ++j) b_turn[j] = turned_at<TRB>(wn * WN + j, fr, fg);
  }
  auto b_frag = [&](int j) { return (GATED && j >= WN / 2 ? BN + (j - WN / 2) * 16 : j * 16) * GB_ROW_BYTES; };

  // per-tile state.  A tile's table entry is fetched two tiles ahead and (GATHER) its token indices
  // one tile ahead, as plain vector loads issued right after a tile's first barrier: they complete
  // in the shadow of the K loop (whose next barrier is a whole K chunk of MFMAs away) and are only
  // touched after it, so no tile ever waits for a table lookup.
  struct Info { int e, m0, rbase, rows_e, fill_e, iroff_e, n0; };
  // Load addressing.  Instruction i of wave w fills stage rows [8 q, 8 q + 8), q = i * NW + w: lane l
  // fetches row 8 q + l / 8.  The swizzle of that row, ((8 q + l / 8) >> 1) & 7, does not depend on i
  // (8 NW is a multiple of 16), so a lane's offsets into one operand differ by a wave-uniform row
  // step from one instruction to the next: one register per operand (A gathered: one per
  // instruction), the step added when the load is issued.
  static_assert((8 * NW) % 16 == 0, "swizzle must not depend on the instruction index");
  constexpr int NVA = GATHER ? NIA : 1;
  // A tile keeps the base and range of its operands; the buffer descriptors are put together from
  // them when loads are issued, through readfirstlane: a descriptor that the register allocator has
  // parked in vector registers would otherwise be treated as divergent and every load wrapped in a
  // waterfall loop.
  struct Tile {
    int e, m0, rbase, rows_e, n0, live;
    int va[NVA], vb;
    unsigned long long pa, pb0, pb1;
    int na, nb;
  };
  auto rsrc_of = [](unsigned long long base, int range) {
    const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)base);
    const unsigned hi = __builtin_amdgcn_readfirstlane((unsigned)(base >> 32));
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<char *>(((unsigned long long)hi << 32) | lo), 0,
                                             __builtin_amdgcn_readfirstlane(range), BUF_FLAGS);
  };
  const int lrow = w * 8 + (lane >> 3);            // stage row of this lane in instruction 0
  const int lcol = ((lane & 7) ^ swz(lrow)) * 16;  // byte position of its 16-byte chunk in the global row
  int lda = K, ldb = K;
  if constexpr (DENSE) {
    lda = P.lda;
    ldb = P.ldb;
  }
  // bytes between the rows of consecutive instructions
  const unsigned rstep = NW * (TA ? 2 : 8) * lda * 2, rstep_b = NW * (TB ? 2 : 8) * ldb * 2;
  int trow = 0, tcol = 0;  // turned: as lrow and lcol
  if constexpr (TA || TB) turned_lane<TRB>(w * 2, lane, trow, tcol);
  static_assert(NW * 2 % 16 == 0, "the swizzle of a turned operand must not depend on the instruction index");
  // this lane's piece of the last chunk lies past the end of the row (K no multiple of the chunk)
  const bool past = (KT - 1) * GB_BK * 2 + lcol >= K * 2;
  const char *Ab = static_cast<const char *>(P.A);
  auto raw_load = [&](int Lt, int4 &ra, int4 &rb) {
    if (DENSE) return;
    const int4 *q = reinterpret_cast<const int4 *>(P.tiles + Lt / NT);
    ra = q[0];
    rb = q[1];
  };
  auto finalize = [&](const Unit &u, const int4 &ra, const int4 &rb) {
    Info f;
    f.e = __builtin_amdgcn_readfirstlane(ra.x);
    f.m0 = __builtin_amdgcn_readfirstlane(ra.y);
    f.rbase = __builtin_amdgcn_readfirstlane(ra.z);
    f.rows_e = __builtin_amdgcn_readfirstlane(ra.w);
    f.fill_e = __builtin_amdgcn_readfirstlane(rb.x);
    f.iroff_e = __builtin_amdgcn_readfirstlane(rb.y);
    f.n0 = (u.L % NT) * BN;
    if constexpr (DENSE) {
      f.e = u.L / NT / P.MT;  // the slice
      f.m0 = (u.L / NT - f.e * P.MT) * BM;
      f.rbase = f.fill_e = f.iroff_e = 0;
      f.rows_e = P.M;
    }
    if (u.part >= 0) {
      const CutRows r = cut_rows(f.m0, min(BM, f.rows_e - f.m0), cut, u.part);
      f.m0 = r.m0;
      f.rows_e = r.end;
    }
    return f;
  };
  // the dispatch gather (Sec. 3: tokens travel to their experts): the tokens behind this lane's A
  // rows - occupied capacity slots first, then the expert's Intra-GPU rows; -1 = padding
  // Every lane always loads (rows past the expert's end read a valid dummy and are masked when the
  // offsets are built): the number of memory instructions per tile is then fixed, which the counted
  // waits of the K loop rely on.
  auto lookup_tokens = [&](const Info &f, int (&tok)[NIA]) {
#pragma unroll
    for (int i = 0; i < NIA; ++i) {
      const int lr = f.m0 + (i * NW + w) * 8 + (lane >> 3);  // row within the expert
      const int32_t *src = lr < f.fill_e ? P.slot_token + ((size_t)f.e * P.C + lr) : P.ir_token + (f.iroff_e + lr - f.fill_e);
      if (P.row_token) src = P.row_token + (f.rbase + lr);
      if (lr >= f.rows_e) src = P.slot_token;
      tok[i] = *src;
    }
  };
  auto make_tile = [&](const Info &f, const int (&tok)[NIA], Tile &t) {
    t.e = f.e; t.m0 = f.m0; t.rbase = f.rbase; t.rows_e = f.rows_e; t.n0 = f.n0;
    t.live = (min(BM, f.rows_e - f.m0) + PK_WAVES_M * 16 - 1) / (PK_WAVES_M * 16);
    if constexpr (DENSE) {  // operands that start at the tile's first row (turned: column) and the slice's first element
      const size_t k0 = (size_t)f.e * K, pa = (size_t)lda * 2, pb = (size_t)ldb * 2;
      t.pa = reinterpret_cast<unsigned long long>(Ab) + (TA ? k0 * pa + f.m0 * 2 : f.m0 * pa + k0 * 2);
      t.pb0 = reinterpret_cast<unsigned long long>(P.B0) + (TB ? k0 * pb + f.n0 * 2 : f.n0 * pb + k0 * 2);
      t.pb1 = GATED ? reinterpret_cast<unsigned long long>(P.B1) + f.n0 * pb + k0 * 2 : t.pb0;
      // bytes to the operand's end; turned: memory rows of the slice
      t.na = TA ? min(K, P.Kall - (int)k0) : (int)(min(BM, f.rows_e - f.m0) * pa - k0 * 2);
      t.nb = TB ? min(K, P.Kall - (int)k0) : (int)(min(BN, N - f.n0) * pb - k0 * 2);
      t.va[0] = TA ? trow * lda * 2 + tcol : lrow * lda * 2 + lcol;
      t.vb = TB ? trow * ldb * 2 + tcol : lrow * ldb * 2 + lcol;
      return;
    }
    const char *B0b = static_cast<const char *>(P.B0) + (size_t)f.e * N * K * 2;
    const char *B1b = GATED ? static_cast<const char *>(P.B1) + (size_t)f.e * N * K * 2 : B0b;
    if (GATHER) {
      t.pa = reinterpret_cast<unsigned long long>(Ab);
      t.na = (int)P.a_bytes;
    } else {
      t.pa = reinterpret_cast<unsigned long long>(Ab + (size_t)f.rbase * K * 2);
      t.na = (int)min((size_t)f.rows_e * K * 2, (size_t)0x7fffffff);
    }
    t.pb0 = reinterpret_cast<unsigned long long>(B0b);
    t.pb1 = reinterpret_cast<unsigned long long>(B1b);
    if (GATHER) {
#pragma unroll
      for (int i = 0; i < NVA; ++i) {
        const bool real = f.m0 + (i * NW + w) * 8 + (lane >> 3) < f.rows_e && tok[i] >= 0;
        t.va[i] = real ? tok[i] * K * 2 + lcol : 0x7ffffff0;  // padding: past the range, reads as zero
      }
    } else {
      t.va[0] = (f.m0 + lrow) * K * 2 + lcol;
    }
    t.vb = (f.n0 + lrow) * K * 2 + lcol;  // gate and up rows (GATED) sit at the same offsets of W1 and W3
  };
  // The stream of K chunks that the LDS rings are filled from: where the next chunk of A (NIA instructions
  // per wave) and of B (NIB) comes from.  It runs ahead of the multiplication into the next tile; past the
  // last tile its ranges are 0, so that every chunk issues the same number of loads.
  constexpr int NIB = NI - NIA;
  unsigned sva[NVA], svb;  // offsets of this lane
  int ska, skb, sna, snb;  // byte positions in K, ranges; turned: unused, memory rows left
  int scol_a = 0, scol_b = 0;  // turned: bytes of a memory row before the tile's first column
  unsigned long long spa, spb0, spb1;
  auto stream_a = [&](const Tile &t, bool real) {
#pragma unroll
    for (int i = 0; i < NVA; ++i) sva[i] = t.va[i];
    spa = t.pa;
    sna = real ? t.na : 0;
    ska = 0;
    if (TA) scol_a = t.m0 * 2;
  };
  auto stream_b = [&](const Tile &t, bool real) {
    svb = t.vb;
    spb0 = t.pb0;
    spb1 = t.pb1;
    snb = real ? (DENSE ? t.nb : N * K * 2) : 0;
    skb = 0;
    if (TB) scol_b = t.n0 * 2;
  };
  auto issue_a = [&](int stage) {
    char *st = smem + stage * PK_A_STAGE + w * 1024;
    // turned: the buffer is the chunk's memory rows, from the tile's first column on
    const __amdgpu_buffer_rsrc_t rsA = rsrc_of(spa, TA ? max(0, min(GB_BK, sna)) * lda * 2 - (sna > 0 ? scol_a : 0) : sna);
#pragma unroll
    for (int i = 0; i < NIA; ++i) {
      auto lp = (__attribute__((address_space(3))) void *)(st + i * NW * 1024);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsA, lp, 16, GATHER ? sva[i < NVA ? i : 0] : sva[0] + i * rstep, ska, 0, 0);
    }
    if constexpr (TA) {
      spa += (unsigned long long)lda * (GB_BK * 2);
      sna -= GB_BK;
    } else {
      ska += GB_BK * 2;
    }
  };
  auto issue_b = [&](int stage, int i0, int i1) {  // instructions i0 .. i1 - 1 of the chunk
    char *st = smem + PK_B_BASE + stage * PK_B_STAGE + w * 1024;
    const int rangeb = TB ? max(0, min(GB_BK, snb)) * ldb * 2 - (snb > 0 ? scol_b : 0) : snb;
    const __amdgpu_buffer_rsrc_t rsB0 = rsrc_of(spb0, rangeb), rsB1 = rsrc_of(spb1, rangeb);
#pragma unroll
    for (int i = 0; i < NIB; ++i) {
      if (i < i0 || i >= i1) continue;
      // which weight matrix instruction i reads is known at compile time
      auto lp = (__attribute__((address_space(3))) void *)(st + i * NW * 1024);
      if (!GATED || i < NIB0)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsB0, lp, 16, svb + i * rstep_b, skb, 0, 0);
      else
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsB1, lp, 16, svb + (i - NIB0) * rstep_b, skb, 0, 0);
    }
    if (i1 == NIB) {
      if constexpr (TB) {
        spb0 += (unsigned long long)ldb * (GB_BK * 2);
        snb -= GB_BK;
      } else {
        skb += GB_BK * 2;
      }
    }
  };
  auto next_b = [](int sb) { return sb == PK_B_STAGES - 1 ? 0 : sb + 1; };

  // LDS rings: A has two stages, B three (160 KB together).  The K chunks of a workgroup's tiles
  // form one stream (chunk KT of a tile is chunk 0 of its next tile).  While chunk c is multiplied,
  // A(c+1), B(c+1) and B(c+2) are in flight or landed: the weights, which stream from HBM, are
  // fetched two chunks ahead, the activations (mostly L2 hits: a row tile is shared by all column
  // tiles) one.  Each chunk issues A(c+1) and then B(c+2), so the barrier that publishes chunk c+1
  // waits for everything but the NIB youngest loads.  KT >= 3.
  f32x4 acc[WM][WN];
  Tile cur, nxt;
  Info info1{}, info2{};                              // table entries of this workgroup's next two tiles
  int4 ra2 = make_int4(0, 0, 0, 0), rb2 = ra2;        // raw table entry of the tile after next
  int tok1[NIA];        // token indices of the next tile's A rows
  int sa = 0, sb = 0;   // ring stages of the current chunk
  {
    int4 ra, rb;
    raw_load(U.L, ra, rb);
    const Info f0 = finalize(U, ra, rb);
    if (f0.m0 >= f0.rows_e) return;  // an empty part
    int tok0[NIA];
#pragma unroll
    for (int i = 0; i < NIA; ++i) tok0[i] = -1;
    if (GATHER) lookup_tokens(f0, tok0);
    make_tile(f0, tok0, cur);
    if (U1.L >= 0) {
      raw_load(U1.L, ra, rb);
      info1 = finalize(U1, ra, rb);
    }
    stream_a(cur, true);
    stream_b(cur, true);
    issue_a(sa);
    issue_b(sb, 0, NIB);
    issue_b(next_b(sb), 0, NIB);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NIB) : "memory");  // own A(0), B(0) have landed
  }
  while (true) {
    const bool have1 = U1.L >= 0 && info1.m0 < info1.rows_e;  // (only a workgroup's last tile can be an empty part)
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
      for (int j = 0; j < WN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // Everybody's A(0), B(0) have landed: each wave saw its own arrive before it stored the previous
    // tile's results, so the barrier itself waits for no memory operation (the stores and B(1) may
    // still be on their way).
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    // table lookups for the tiles to come, issued before this chunk's loads so that they are older
    // than anything a counted wait lets pass
    if (GATHER) lookup_tokens(info1, tok1);
    raw_load(U2.L >= 0 ? U2.L : U.L, ra2, rb2);
    int dest[WM];  // DIRECT: where the rows that this lane will store also go (this tile's, used in its epilogue)
#pragma unroll
    for (int i = 0; i < WM; ++i) {
      dest[i] = -1;
      if (DIRECT) {
        const int row = cur.m0 + (i * PK_WAVES_M + wm) * 16 + fr;
        dest[i] = P.row_dest[cur.rbase + min(row, cur.rows_e - 1)];
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    issue_a(sa ^ 1);
    issue_b(next_b(next_b(sb)), 0, NIB);

    // Ragged and cut row tiles: the two waves of a column take turns at the tile's 16-row fragments, and
    // the K loop comes in copies for 2, 4, 6 and 8 fragments per wave (branch-free, which keeps the counted
    // LDS waits exact), so a short tile costs MFMA time in proportion to its rows on all four SIMDs.
    auto k_loop = [&](auto live_tag) {
      // A chunk is four steps: k-step ks (of two), half hf of the wave's A rows.  A step multiplies half of the
      // A fragments with all B fragments of its k-step: 16 MFMAs in a full tile.
      constexpr int HM = decltype(live_tag)::value / 2, MF = HM * WN;
      constexpr int RA = TA ? 2 * HM : HM, RB = TB ? 2 * WN : WN, RP = TA || TB ? 2 : 1;  // LDS reads of a step
      bf16x8 af[2][HM], bfr[2][WN];
      auto load_a = [&](const char *sta, int ks, int hf) {
        const char *p = sta + a_off + (((4 * ks + fg) ^ fsw) << 4);
#pragma unroll
        for (int i = 0; i < HM; ++i)
          if constexpr (TA)
            af[hf][i] = read_turned<TRB>(sta + a_turn[(hf * HM + i) & 3] + (hf * HM + i) / 4 * 256 + ks * 32 * TRB);
          else
            af[hf][i] = *reinterpret_cast<const bf16x8 *>(p + (hf * HM + i) * PK_WAVES_M * 16 * GB_ROW_BYTES);
      };
      auto load_b = [&](const char *stb, int ks) {
        const char *p = stb + b_off + (((4 * ks + fg) ^ fsw) << 4);
#pragma unroll
        for (int j = 0; j < WN; ++j)
          if constexpr (TB) bfr[ks][j] = read_turned<TRB>(stb + b_turn[j] + ks * 32 * TRB);
          else bfr[ks][j] = *reinterpret_cast<const bf16x8 *>(p + b_frag(j));
      };
      auto mfma_step = [&](int ks, int hf) {
#pragma unroll
        for (int i = 0; i < HM; ++i)
#pragma unroll
          for (int j = 0; j < WN; ++j)
            // B fragment first: the accumulator holds the transposed tile (see store_tile_t)
            acc[hf * HM + i][j] =
                __builtin_amdgcn_mfma_f32_16x16x32_bf16(bfr[ks][j], af[hf][i], acc[hf * HM + i][j], 0, 0, 0);
      };
      // The chunk's LDS-DMA loads are spread over its steps, behind an MFMA each: A(kt+1) in the step
      // after the barrier, B(kt+2) in the two after it.  (All eight in one place - 64 per CU, 16 clocks of the
      // load unit each - kept the waves waiting at the issue: down projection at 8 K tokens x 5632 296 -> 275 us.
      // It takes straight-line code, hence the stream of chunks that runs past the tile's end.)
      // Software pipeline: the fragments that the NEXT step needs and this one does not hold are read
      // under the MFMAs of this one, one LDS read behind each of the first MFMAs.  (With all the reads in
      // front of the MFMAs the LDS pipe is asked for several KB per wave in one burst and is then idle
      // for the rest of the step; both waves of a SIMD doing so in turn leaves MFMA slots empty.)  The
      // last step of a chunk runs after the barrier; the global loads of the stream go behind its last
      // MFMAs.  The loop is rotated so that its body starts at the barrier (the compiler's wait
      // counting is exact only inside one basic block).
      // the first three steps of a chunk; the B loads of the stream ride in the first two of them
      auto steps = [&](const char *sta, const char *stb, auto dma_tag, int bstage) {
        constexpr bool DMA = decltype(dma_tag)::value;
        load_a(sta, 0, 1);
        if (DMA) issue_b(bstage, 0, NIB / 2);
        mfma_step(0, 0);
        sched_step<MF, RA, DMA ? NIB / 2 : 0, RP>();
        __builtin_amdgcn_sched_barrier(0);
        load_a(sta, 1, 0);
        load_b(stb, 1);
        if (DMA) issue_b(bstage, NIB / 2, NIB);
        mfma_step(0, 1);
        sched_step<MF, RA + RB, DMA ? NIB - NIB / 2 : 0, RP>();
        __builtin_amdgcn_sched_barrier(0);
        load_a(sta, 1, 1);
        mfma_step(1, 0);
        sched_step<MF, RA, 0, RP>();
        __builtin_amdgcn_sched_barrier(0);
      };
      const char *sta = smem + sa * PK_A_STAGE, *stb = smem + PK_B_BASE + sb * PK_B_STAGE;
      load_a(sta, 0, 0);
      load_b(stb, 0);
      steps(sta, stb, std::false_type{}, 0);
      // The looked-up values are consumed here, unconditionally, rather than where they are first
      // needed: in straight-line code after the lookups the compiler's wait for them is a counted
      // one (the A(1) and B(2) loads behind them stay in flight), and nothing it tracks is pending
      // when the loop is entered or the tile ends - there it would drain every outstanding load
      // and store.  Without a next tile the values are unused.
      make_tile(info1, tok1, nxt);
      info2 = finalize(U2.L >= 0 ? U2 : U, ra2, rb2);
      if (DIRECT) {  // consumed here like the other lookups, so that no load is pending when the loop is entered
#pragma unroll
        for (int i = 0; i < WM; ++i) asm volatile("" : "+v"(dest[i]));
      }
      for (int kt = 1; kt < KT; ++kt) {
        // the stream moves on to the next tile: A one chunk, B two chunks before this tile ends
        if (kt == KT - 2) stream_b(nxt, have1);
        if (kt == KT - 1) stream_a(nxt, have1);
        if (K % GB_BK) {  // in the last chunk of a row, pieces past its end are sent out of range: they read as zero
          if (!TB && kt == KT - 3 && past) svb = 0x7ffffff0;
          if (!TA && kt == KT - 2 && past) {
#pragma unroll
            for (int i = 0; i < NVA; ++i) sva[i] = 0x7ffffff0;
          }
        }
        // A(kt) and B(kt) have landed - the B issued after A(kt) may still be on its way - and
        // nobody reads the stages of chunk kt-1 any more
        dma_barrier<NIB>();
        sa ^= 1;
        sb = next_b(sb);
        sta = smem + sa * PK_A_STAGE;
        stb = smem + PK_B_BASE + sb * PK_B_STAGE;
        load_a(sta, 0, 0);
        load_b(stb, 0);
        issue_a(sa ^ 1);
        mfma_step(1, 1);  // last step of chunk kt-1
        sched_step<MF, RA + RB, NIA, RP>();
        __builtin_amdgcn_sched_barrier(0);
        steps(sta, stb, std::true_type{}, next_b(next_b(sb)));
      }
      mfma_step(1, 1);
    };
    const int live = cur.live;
    if (live > 6) k_loop(std::integral_constant<int, 8>{});
    else if (live > 4) k_loop(std::integral_constant<int, 6>{});
    else if (live > 2) k_loop(std::integral_constant<int, 4>{});
    else k_loop(std::integral_constant<int, 2>{});

    // own A(0), B(0) of the next tile have landed (they were issued one and two chunks ago), before
    // the stores below join the queue of outstanding memory operations
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(NIB) : "memory");
    sa ^= 1;
    sb = next_b(sb);
    if constexpr (DENSE)
      store_dense<WM, WN, PK_WAVES_M * 16, true, GATED, ACT>(acc, P, cur.e, cur.m0 + wm * 16 + fr, cur.rows_e,
                                                             cur.n0 + wn * (GATED ? WN / 2 : WN) * 16, lane);
    else
      store_tile_t<WM, WN, PK_WAVES_M, GATED, ACT, DIRECT>(acc, static_cast<uint16_t *>(P.Cout), cur.rbase, cur.rows_e, cur.m0, cur.n0,
                                               N, wm, wn, lane, dest, static_cast<uint16_t *>(P.Out));
    if (!have1) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the stream's loads past the last tile still write this LDS
      break;
    }
    cur = nxt;
    U = U1;
    U1 = U2;
    U2 = unit_at(++round + 2);
    info1 = info2;
  }
#endif
}

// Four fp32 values, times kSplitScale, as sums of three bf16 values, each the nearest of what the ones before it leave (8
// mantissa bits and a sign: three of them hold all 24): plane[p] gets part p of the four.  bf16 counts down to 2^-133, so the
// parts of values below 2^-110 would lose bits: the scale lifts fp32's smallest step, 2^-149, to there, and the sum of
// products is brought back by kSplitUnscale (powers of two: nothing is rounded).  Values from 2^89 and sums from 2^50 on
// become infinities and are computed again (see the end of the K loop).  2048 tokens, 1024 x 2816, 8 experts: 510 us without the
// scale (tokens at 2^-122: an error of 8e-4), 503 with it as a 4-byte multiplication and 4-byte subtractions, 519 as 8-byte ones.
// Conversions and subtractions only: v_dot2c_f32_bf16 with (-1, 0) would subtract a packed value from its fp32 one without unpacking
// it (7 instructions for two values, not 11 and the 2 of the scale), but does not run beside MFMAs (22 cycles each, v_sub_f32 8).
[[maybe_unused]] constexpr float kSplitScale = 0x1p39f, kSplitUnscale = 0x1p-78f;
__device__ __forceinline__ void split3(const f32x4 &x, float scale, uint2 (&plane)[3]) {
#pragma clang fp contract(off)  // (the first subtraction as a fused one is 8 bytes long too)
  u32 w[3][2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    float a = x[2 * q] * scale, b = x[2 * q + 1] * scale;
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      w[p][q] = pack_bf16(a, b);
      if (p < 2) {
        a -= __builtin_bit_cast(float, w[p][q] << 16);
        b -= __builtin_bit_cast(float, w[p][q] & 0xffff0000u);
      }
    }
  }
#pragma unroll
  for (int p = 0; p < 3; ++p) plane[p] = make_uint2(w[p][0], w[p][1]);
}

// ------------------------------------------------------------------ small tiles, bf16 and fp32, any K % 8 == 0
// Everything the 256 x 256 kernel is not made for: fp32 layers, row lengths that are no multiple of the
// K chunk or shorter than three of them, and batches whose experts get few rows.  One workgroup per tile,
// several workgroups per CU: one's epilogue, table lookups and barrier waits run under another's MFMAs.
//   * K advances in chunks of 128 bytes of every staged row through a ring of ST stages filled by
//     buffer_load ... lds with the same row layout and swizzle as above; a chunk is requested ST - 1 chunks
//     ahead, into the stage that the barrier at the top of the chunk has just freed, and every chunk
//     issues the same number of loads (past the end: out of range, which costs no traffic), so one
//     counted wait serves any K.  Pieces past the end of a row are sent out of range as well: they read as zero.
//   * bf16: v_mfma_f32_16x16x32_bf16.  fp32: v_mfma_f32_16x16x4_f32, fp32 products and accumulation; a
//     lane's 16-byte piece is its operand of four MFMAs - the K order inside a chunk is then a
//     permutation, the same for both operands.
//   * fp32 rows of five chunks and more that fill their tiles (TILE_SPLIT): every operand is split into three bf16 parts
//     that hold its 24 bits, and the six products down to 2^-18 of the leading one run on the bf16 pipe, accumulated in
//     fp32 (a split of Dekker's kind, as the router's; the three left out are up to 2^-24.2 of a product, so a lone product is
//     off by up to 0.94 ulp, where an fp32 MFMA rounds it to 0.5): 96 cycles of MFMAs per pair of fragments and chunk instead of 256.
//     The parts are made once per workgroup, on the way to LDS (a wave that splits its own fragments does it two to four
//     times over, and conversions run at half speed beside MFMAs: 285 us instead of 265 for the layer below).  Error
//     against 64 bits below that of the fp32 MFMAs, which round as often (1024 tokens, 1024 x 2816 SwiGLU 1.09e-6
//     of the output's norm, 1.29e-6; 4096 x 4096 1.80e-6, 2.09e-6; 64 x 128 GELU 1.8e-7, 2.6e-7).
//     Of 40 layers from 32 to 4096 wide none has a larger error; with tokens of one to four nonzero values 1.5 % at most, 2.5 % less on average.
//     3931 rows, 1024 x 2816 SwiGLU, 64 x 128 tiles: up 355 -> 284 us, down 187 - 208 -> 198 (530 tiles, two on a CU that holds four: too
//     little beside the barriers); 7900 rows, 2112 x 4224 GELU, 128 x 128: 1077 -> 745, 1075 -> 773.  Bound by the bf16 pipe (57 % of the cycles
//     at 2.03 GHz) and the splitting beside it.
// Measured, before (register-staged bf16 kernel, fp32 FMA kernel) -> now: 6161 rows, 1000 x 2728, bf16 GELU, down 118 -> 47 us
// (the up projection runs on 256 x 256 tiles: 163 -> 58); 3931 rows, 1024 x 2816, fp32 SwiGLU: up 612 -> 354 us (128 TFLOP/s; the fp32 MFMA pipe sustains 154),
// down 397 -> 184.  bf16 tiles of this size are bound by the operand bytes per flop (L2 -> LDS), fp32 ones by the MFMAs.
// WM x WN: 16-row fragments of a wave.
enum TileMath { TILE_BF16, TILE_F32, TILE_SPLIT };  // TILE_SPLIT: fp32 operands as three bf16 parts each
template <TileMath MATH_, int WAVES_M_, int WAVES_N_, int WM_, int WN_, int ST_, int OCC_>
struct TileShape {
  static constexpr TileMath MATH = MATH_;
  static constexpr bool BF16 = MATH == TILE_BF16;
  static constexpr int WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, WM = WM_, WN = WN_, ST = ST_, OCC = OCC_;
  static constexpr int NW = WAVES_M * WAVES_N, THREADS = NW * 64;
  static constexpr int BM = WAVES_M * WM * 16, BROWS = WAVES_N * WN * 16;
  static constexpr int STAGE = (BM + BROWS) * (MATH == TILE_SPLIT ? 3 * GB_ROW_BYTES / 2 : GB_ROW_BYTES), SMEM = ST * STAGE;
};

// ACT: RR_ACT_GELU, RR_ACT_SWIGLU (bf16: with the division), or -1.  ONCE: no other workgroup reads these rows of B.
template <class S, bool GATED, int ACT, bool GATHER, bool DIRECT, bool DENSE = false, bool TA = false, bool TB = false, bool ONCE = false>
__global__ __launch_bounds__(S::THREADS, S::OCC) void gemm_tile_kernel(typename std::conditional<DENSE, DenseArgs, GemmArgs>::type P) {
#if defined(__HIP_DEVICE_COMPILE__)
  constexpr int WM = S::WM, WN = S::WN, NW = S::NW, BM = S::BM, ST = S::ST;
  constexpr int BN = GATED ? S::BROWS / 2 : S::BROWS;
  constexpr int NIA = BM / 8 / NW, NIB = S::BROWS / 8 / NW, NI = NIA + NIB, NIB0 = BN / 8 / NW;
  constexpr int ES = S::BF16 ? 2 : 4, CE = GB_ROW_BYTES / ES, PE = 16 / ES;  // elements per chunk of a row, per piece
  static_assert(BM % (8 * NW) == 0 && BN % (8 * NW) == 0, "operand boundaries must fall between load instructions");
  static_assert((8 * NW) % 16 == 0, "swizzle must not depend on the instruction index");
  static_assert(!GATED || WN % 2 == 0, "a wave holds the gate and the up columns of its outputs");
  static_assert(!(TA || TB) || (DENSE && !GATED && !GATHER && S::MATH != TILE_F32));
  constexpr int kPanel = 8;  // row tiles that share a column tile of weights before the next column tile
  extern __shared__ __attribute__((aligned(16))) char smem[];

  // tile number: each XCD (workgroup g runs on XCD g % 8) takes a contiguous run; panels of kPanel row
  // tiles, column tiles inside a panel, row tiles inside a column: neighbours share weights
  // (the table's row tiles are P.sub times as high as this kernel's)
  int MT;
  if constexpr (DENSE) MT = P.MT * P.slices;
  else MT = P.ctl[0] * P.sub;
  const int NT = P.NT, total = MT * NT;
  const unsigned g = blockIdx.y * gridDim.x + blockIdx.x;  // rows of whole XCD runs (tile_grid)
  const int per = (total + 7) >> 3, run = (int)(g >> 3), t = (int)(g & 7) * per + run;
  if (run >= per || t >= total) return;
  const int panel = t / (kPanel * NT), r = t - panel * kPanel * NT, h = min(kPanel, MT - panel * kPanel);
  const int nt = r / h, mt = panel * kPanel + r - nt * h;
  TileInfo ti;
  int m0, K = P.K, LD = K, LDB = K, k0 = 0;
  if constexpr (DENSE) {
    const int slice = mt / P.MT;
    ti = TileInfo{slice, 0, 0, P.M, 0, 0, 0, 0};
    m0 = (mt - slice * P.MT) * BM;
    k0 = slice * K;
    K = min(K, P.Kall - k0);
    LD = P.lda;
    LDB = P.ldb;
  } else {
    ti = P.tiles[mt / P.sub];
    m0 = ti.row0 + mt % P.sub * BM;
  }
  if (m0 >= ti.rows) return;
  const int N = P.N, KT = (K + CE - 1) / CE;
  const int e = ti.expert, rbase = ti.rbase, rows_e = ti.rows, n0 = nt * BN;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = w / S::WAVES_N, wn = w % S::WAVES_N;
  const int fr = lane & 15, fg = lane >> 4;
  constexpr unsigned PAST = 0x7ffffff0u;  // past every operand's range: reads as zero

  // ---- operands: buffers that start at the tile's first row (GATHER: at x) and end with its last one
  const int lrow = w * 8 + (lane >> 3);            // stage row of this lane in instruction 0
  const int piece = S::MATH == TILE_SPLIT ? lane & 7 : (lane & 7) ^ swz(lrow);  // 16-byte piece of the row's chunk that belongs at its position
  const unsigned rowb = (unsigned)LD * ES;
  const unsigned rowbB = DENSE ? (unsigned)LDB * ES : rowb;
  const unsigned rstep = NW * 8 * rowb, rstepB = DENSE ? NW * 8 * rowbB : rstep;  // between the rows of consecutive instructions
  auto rsrc = [](const char *base, size_t off, long long range) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(base) + off, 0,
                                             __builtin_amdgcn_readfirstlane((int)range), BUF_FLAGS);
  };
  const size_t mat = (DENSE ? (size_t)k0 * ES : (size_t)e * N * K * ES) + (size_t)n0 * rowbB;
  const long long brange = (long long)min(BN, N - n0) * rowbB - k0 * ES;
  const __amdgpu_buffer_rsrc_t rsB0 = rsrc(static_cast<const char *>(P.B0), mat, brange);
  const __amdgpu_buffer_rsrc_t rsB1 = GATED ? rsrc(static_cast<const char *>(P.B1), mat, brange) : rsB0;
  const __amdgpu_buffer_rsrc_t rsA =
      GATHER ? rsrc(static_cast<const char *>(P.A), 0, P.a_bytes)
             : rsrc(static_cast<const char *>(P.A), (size_t)(rbase + m0) * rowb + k0 * ES, (long long)min(BM, rows_e - m0) * rowb - k0 * ES);
  auto load16 = [](const __amdgpu_buffer_rsrc_t &rs, unsigned off, int koff) {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, off, koff, 0));
  };
  auto token_of = [&](int lr) {  // row within the expert: capacity slots first, then its Intra-GPU rows
    const int32_t *src = lr < ti.fill ? P.slot_token + ((size_t)e * P.C + lr) : P.ir_token + (ti.ir_offset + lr - ti.fill);
    if (P.row_token) src = P.row_token + (rbase + lr);
    if (lr >= rows_e) src = P.slot_token;  // a valid dummy: the lookups of all instructions are in flight together
    return *src;
  };
  unsigned va[GATHER ? NIA : 1];
  if (GATHER) {
#pragma unroll
    for (int i = 0; i < NIA; ++i) va[i] = (unsigned)token_of(m0 + i * NW * 8 + lrow);
#pragma unroll
    for (int i = 0; i < NIA; ++i) va[i] = m0 + i * NW * 8 + lrow < rows_e ? va[i] * rowb + piece * 16 : PAST;
  } else {
    va[0] = lrow * rowb + piece * 16;
  }
  const unsigned vb = lrow * rowbB + piece * 16;
  // Turned operands: a chunk's rows are a buffer of their own, from the tile's first column on.  Offsets of this lane in instructions
  // 0 and 1 (the swizzle of two instructions apart is the same), bytes between instructions.
  constexpr int TRA = BM * 2, TRB = S::BROWS * 2, RPA = 1024 / TRA, RPB = 1024 / TRB;
  static_assert(!TA || !S::BF16 || NW * RPA % 8 == 0);
  static_assert(!TB || !S::BF16 || NW * RPB % 8 == 0);
  unsigned ta[2] = {0, 0}, tb[2] = {0, 0};
  if constexpr ((TA || TB) && S::BF16) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int row, byte;
      turned_lane<TRA>((i * NW + w) * RPA, lane, row, byte);
      ta[i] = (row - i * NW * RPA) * rowb + byte;
      turned_lane<TRB>((i * NW + w) * RPB, lane, row, byte);
      tb[i] = (row - i * NW * RPB) * rowbB + byte;
    }
  }
  auto turned_rsrc = [&](const void *base, int kt, unsigned pitch, int col) {
    const int rows = kt < KT ? min(CE, K - kt * CE) : 0;  // past the end: none
    return rsrc(static_cast<const char *>(base), (size_t)(k0 + min(kt, KT - 1) * CE) * pitch + col * ES,
                rows > 0 ? (long long)rows * pitch - col * ES : 0);
  };
  auto issue = [&](int kt, int stage) {
    char *st = smem + stage * S::STAGE + w * 1024;
    const bool past = kt * CE + piece * PE >= K;  // the last chunk of a ragged K, and chunks past the end
    const int koff = min(kt, KT - 1) * GB_ROW_BYTES;
    const __amdgpu_buffer_rsrc_t rsTB = TB ? turned_rsrc(P.B0, kt, rowbB, n0) : rsB0, rsTA = TA ? turned_rsrc(P.A, kt, rowb, m0) : rsA;
#pragma unroll
    for (int i = 0; i < NIB; ++i) {
      auto lp = (__attribute__((address_space(3))) void *)(st + BM * GB_ROW_BYTES + i * NW * 1024);
      if constexpr (TB) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsTB, lp, 16, tb[i & 1] + i * NW * RPB * rowbB, 0, 0, 0);
        continue;
      }
      const unsigned v = vb + (GATED && i >= NIB0 ? i - NIB0 : i) * rstepB;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(!GATED || i < NIB0 ? rsB0 : rsB1, lp, 16, past ? PAST : v, koff, 0, ONCE ? BUF_STREAM : 0);
    }
#pragma unroll
    for (int i = 0; i < NIA; ++i) {
      auto lp = (__attribute__((address_space(3))) void *)(st + i * NW * 1024);
      if constexpr (TA) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsTA, lp, 16, ta[i & 1] + i * NW * RPA * rowb, 0, 0, 0);
        continue;
      }
      const unsigned v = GATHER ? va[GATHER ? i : 0] : va[0] + i * rstep;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsA, lp, 16, past ? PAST : v, koff, 0, 0);
    }
  };

  // ---- fragments: lane reads row (lane & 15), piece 4 ks + (lane >> 4) of k-step ks (two per chunk)
  int a_off[WM], b_off[WN];
  const int fsw = swz(fr);  // fragment rows start at multiples of 16, so the swizzle depends on fr only
#pragma unroll
  for (int i = 0; i < WM; ++i) a_off[i] = ((wm * WM + i) * 16 + fr) * GB_ROW_BYTES;
#pragma unroll
  for (int j = 0; j < WN; ++j) {
    constexpr int H = WN / 2;
    int row = (wn * WN + j) * 16 + fr;
    if (GATED) row = (j < H) ? (wn * H + j) * 16 + fr : BN + (wn * H + (j - H)) * 16 + fr;
    b_off[j] = (BM + row) * GB_ROW_BYTES;
  }
  int a_turn[WM], b_turn[WN];
  if constexpr ((TA || TB) && S::BF16) {
#pragma unroll
    for (int i = 0; i < WM; ++i) a_turn[i] = turned_at<TRA>(wm * WM + i, fr, fg);
#pragma unroll
    for (int j = 0; j < WN; ++j) b_turn[j] = BM * GB_ROW_BYTES + turned_at<TRB>(wn * WN + j, fr, fg);
  }
  using Frag = typename std::conditional<S::BF16, bf16x8, f32x4>::type;
  f32x4 acc[WM][WN];
#pragma unroll
  for (int i = 0; i < WM; ++i)
#pragma unroll
    for (int j = 0; j < WN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  Frag af[2][WM], bfr[2][WN];
  auto load_frags = [&](const char *st, int ks) {
    const int pos = ((4 * ks + fg) ^ fsw) << 4;
#pragma unroll
    for (int i = 0; i < WM; ++i) {
      if constexpr (TA && S::BF16) af[ks][i] = read_turned<TRA>(st + a_turn[i] + ks * 32 * TRA);
      else af[ks][i] = *reinterpret_cast<const Frag *>(st + a_off[i] + pos);
    }
#pragma unroll
    for (int j = 0; j < WN; ++j) {
      if constexpr (TB && S::BF16) bfr[ks][j] = read_turned<TRB>(st + b_turn[j] + ks * 32 * TRB);
      else bfr[ks][j] = *reinterpret_cast<const Frag *>(st + b_off[j] + pos);
    }
  };
  // B fragment first: the accumulator holds the transposed tile, a lane owns row (lane & 15) of the A
  // fragment and four consecutive columns, 4 * (lane >> 4) .. + 3 of the B fragment
  auto mfma_step = [&](int ks) {
    if constexpr (S::BF16) {
#pragma unroll
      for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bfr[ks][j], af[ks][i], acc[i][j], 0, 0, 0);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < WM; ++i)
#pragma unroll
          for (int j = 0; j < WN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(bfr[ks][j][q], af[ks][i][q], acc[i][j], 0, 0, 0);
    }
  };

  if constexpr (S::MATH != TILE_SPLIT)
#pragma unroll
    for (int q = 0; q < ST - 1; ++q) issue(q, q);
  int dest[WM];
#pragma unroll
  for (int i = 0; i < WM; ++i) {
    dest[i] = -1;
    if (DIRECT) dest[i] = P.row_dest[rbase + min(m0 + (wm * WM + i) * 16 + fr, rows_e - 1)];
  }
  int cur = 0, fill = ST - 1;
  if constexpr (S::MATH == TILE_SPLIT) {
    // Chunks go through registers: a lane holds four elements of NI rows, splits them and writes 8 bytes to each of the
    // three planes in LDS, 64 bytes per row and chunk; the next chunk is requested before this one is multiplied.
    f32x4 raw[NI];
    // 16-byte piece c of a plane's row sits at c ^ ((row >> 2) & 3): the 16 rows of a fragment then fill all 64 banks
    constexpr int PLANE = (BM + S::BROWS) * GB_ROW_BYTES / 2;
    char *const wr = smem + lrow * 64 + (((piece >> 1) ^ ((lrow >> 2) & 3)) << 4) + (piece & 1) * 8;
    const int fpos = fr * 64 + ((fg ^ (fr >> 2)) << 4);
    // A turned operand (row k of the chunk holds the elements k of all rows): a lane reads four rows' elements of as many k as
    // it has instructions, a block that it turns by taking the registers the other way round.  Row r of such a plane sits at
    // (r & 3) * rows / 4 + (r >> 2), its piece c at c ^ (r & 3): a wave's writes, eight neighbours of a quarter, and a
    // fragment's reads both fill all banks.
    const int tca = (TA && NIA == 2 ? w & 1 : w) * 8 + (lane & 7), tka = (lane >> 3) + (TA && NIA == 2 ? (w >> 1) * 8 : 0);  // block: 4 rows; NIA k
    const int tcb = w * 8 + (lane & 7), tkb = lane >> 3;
    static_assert(!(TA || TB) || (NW == 4 && !GATED && !GATHER));
    static_assert(!TA || (NIA == 4 && BM == 128) || (NIA == 2 && BM == 64));
    static_assert(!TB || (NIB == 4 && S::BROWS == 128));
    auto fetch_turned = [&](f32x4 *r, int n, const __amdgpu_buffer_rsrc_t &rs, int k, int c, unsigned pitch) {
      unsigned at = k * n * pitch + c * 16;
      // Tiles of 64 rows add up the other offsets again for every chunk: kept in registers, they make others spill (20000 x 512 -> 512
      // 169 us, 159 so; 128 x 128 tiles, which spill two or three, lose 2 % by it)
      if (WM == 2) asm volatile("" : "+v"(at));
#pragma unroll
      for (int i = 0; i < n; ++i) r[i] = load16(rs, at + i * pitch, 0);
    };
    auto write_turned = [&](const f32x4 *r, int n, int region, int rows, int k, int c, float scale) {
      int base = c * 64 + (n == 4 ? ((k >> 1) << 4) + (k & 1) * 8 : ((k >> 2) << 4) + (k & 3) * 4);
      if (WM == 2) asm volatile("" : "+v"(base));  // likewise
#pragma unroll
      for (int j = 0; j < 4; j += n == 4 ? 1 : 2) {
        uint2 q[3];
        split3(n == 4 ? f32x4{r[0][j], r[1][j], r[n - 2][j], r[n - 1][j]} : f32x4{r[0][j], r[1][j], r[0][(j + 1) & 3], r[1][(j + 1) & 3]}, scale, q);
#pragma unroll
        for (int p = 0; p < 3; ++p) {
          const int at = region + p * PLANE + j * (rows / 4) * 64;
          if (n == 4) {
            *reinterpret_cast<uint2 *>(smem + (base ^ (j << 4)) + at) = q[p];
          } else {
            *reinterpret_cast<u32 *>(smem + (base ^ (j << 4)) + at) = q[p].x;
            *reinterpret_cast<u32 *>(smem + (base ^ ((j + 1) << 4)) + at + rows / 4 * 64) = q[p].y;
          }
        }
        if (WM == 4 && j % 2 == 1) __builtin_amdgcn_sched_barrier(0);
      }
    };
    const int tpos = (fr >> 2) * 64 + ((fg ^ (fr & 3)) << 4);
    auto fetch = [&](int kt) {
      const bool past = kt * CE + piece * PE >= K;
      const int koff = min(kt, KT - 1) * GB_ROW_BYTES;
      if constexpr (TB) {
        fetch_turned(raw + NIA, NIB, turned_rsrc(P.B0, kt, rowbB, n0), tkb, tcb, rowbB);
      } else {
#pragma unroll
        for (int i = 0; i < NIB; ++i) {
          const unsigned v = vb + (GATED && i >= NIB0 ? i - NIB0 : i) * rstepB;
          raw[NIA + i] = load16(!GATED || i < NIB0 ? rsB0 : rsB1, past ? PAST : v, koff);
        }
      }
      if constexpr (TA) {
        fetch_turned(raw, NIA, turned_rsrc(P.A, kt, rowb, m0), tka, tca, rowb);
      } else {
#pragma unroll
        for (int i = 0; i < NIA; ++i) {
          const unsigned v = GATHER ? va[GATHER ? i : 0] : va[0] + i * rstep;
          raw[i] = load16(rsA, past ? PAST : v, koff);
        }
      }
    };
    float scale;  // in a register: a multiplication of 4 bytes instead of 8
    asm("s_mov_b32 %0, %1" : "=s"(scale) : "i"(__builtin_bit_cast(int, kSplitScale)));
    fetch(0);
    for (int kt = 0; kt < KT; ++kt) {
      if (kt > 0) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // everybody has read chunk kt - 1
      if constexpr (TA) write_turned(raw, NIA, 0, BM, tka, tca, scale);
      if constexpr (TB) write_turned(raw + NIA, NIB, BM * 64, S::BROWS, tkb, tcb, scale);
#pragma unroll
      for (int i = TA ? NIA : 0; i < (TB ? NIA : NI); ++i) {
        uint2 q[3];
        split3(raw[i], scale, q);
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<uint2 *>(wr + p * PLANE + i * NW * 8 * 64) = q[p];
        // (128 x 128: all rows' parts at once do not fit the registers.  9048 tokens, 768 x 1344, 64 experts: 690 us, two rows at a time 662;
        // 64 x 128 has the room: 2048 tokens, 1024 x 2816, 8 experts 504, two rows at a time 514)
        if (WM == 4 && i % 2 == 1) __builtin_amdgcn_sched_barrier(0);
      }
      fetch(kt + 1);
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // chunk kt is written
      bf16x8 b3[WN][3];
#pragma unroll
      for (int j = 0; j < WN; ++j)
#pragma unroll
        for (int p = 0; p < 3; ++p)
          b3[j][p] = *reinterpret_cast<const bf16x8 *>(smem + p * PLANE + (TB ? (BM + (fr & 3) * (S::BROWS / 4) + (wn * WN + j) * 4) * 64 + tpos
                                                                              : (b_off[j] / GB_ROW_BYTES - fr) * 64 + fpos));
#pragma unroll
      for (int i = 0; i < WM; ++i) {
        bf16x8 a3[3];
#pragma unroll
        for (int p = 0; p < 3; ++p)
          a3[p] = *reinterpret_cast<const bf16x8 *>(smem + p * PLANE + (TA ? ((fr & 3) * (BM / 4) + (wm * WM + i) * 4) * 64 + tpos
                                                                           : (wm * WM + i) * 16 * 64 + fpos));
        // the products of parts down to 2^-18 of the leading one, smallest first
        constexpr int PA[6] = {2, 0, 1, 1, 0, 0}, PB[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
        for (int q = 0; q < 6; ++q)
#pragma unroll
          for (int j = 0; j < WN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b3[j][PB[q]], a3[PA[q]], acc[i][j], 0, 0, 0);
      }
    }
    auto four_of_turned = [&](const void *base, unsigned pitch, int k, int row, int rows) {
      f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (k + u < K && row < rows) v[u] = *reinterpret_cast<const float *>(static_cast<const char *>(base) + (size_t)(k0 + k + u) * pitch + (size_t)row * 4);
      return v;
    };
    // An infinity, or a value that the scale or bf16's rounding makes one, leaves NaN behind its first part: a fragment of
    // which any element is not finite is computed again from fp32 operands.
#pragma unroll
    for (int i = 0; i < WM; ++i) {
      const int arow = (wm * WM + i) * 16 + fr;  // of the tile
      unsigned ao = arow * rowb;
#pragma unroll
      for (int j = 0; j < WN; ++j) {
        bool finite = true;
#pragma unroll
        for (int u = 0; u < 4; ++u) finite = finite && __builtin_isfinite(acc[i][j][u]);
        if (__all(finite)) {
#pragma unroll
          for (int u = 0; u < 4; ++u) acc[i][j][u] *= kSplitUnscale;
          continue;
        }
        if (GATHER) ao = m0 + arow < rows_e ? (unsigned)token_of(m0 + arow) * rowb : PAST;
        const bool up = GATED && j >= WN / 2;
        const unsigned bo = (unsigned)(GATED ? (wn * (WN / 2) + j % (WN / 2)) * 16 + fr : (wn * WN + j) * 16 + fr) * rowb;
        f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int k = 0; k < K; k += 16) {
          const unsigned kb = (k + 4 * fg) * ES;
          const bool past = kb >= (unsigned)K * ES;
          f32x4 a, b;
          if constexpr (TA) a = four_of_turned(P.A, rowb, k + 4 * fg, m0 + arow, rows_e);
          else a = load16(rsA, past || ao == PAST ? PAST : ao + kb, 0);
          if constexpr (TB) b = four_of_turned(P.B0, rowbB, k + 4 * fg, n0 + (wn * WN + j) * 16 + fr, N);
          else b = load16(up ? rsB1 : rsB0, past ? PAST : bo + kb, 0);
#pragma unroll
          for (int u = 0; u < 4; ++u) c = __builtin_amdgcn_mfma_f32_16x16x4f32(b[u], a[u], c, 0, 0, 0);
        }
        acc[i][j] = c;
      }
    }
  } else {
    for (int kt = 0; kt < KT; ++kt) {
      // own loads of chunk kt have landed (ST - 2 younger chunks may be on their way), own reads of chunk kt - 1 too
      dma_barrier<(ST - 2) * NI>();
      const char *st = smem + cur * S::STAGE;
      // software pipeline: the fragments of the next k-step are read under the MFMAs of this one
      load_frags(st, 0);
      if (kt > 0) mfma_step(1);  // last k-step of chunk kt - 1
      issue(kt + ST - 1, fill);
      __builtin_amdgcn_sched_barrier(0);
      load_frags(st, 1);
      mfma_step(0);
      if constexpr (TA || TB) sched_mfma_two_lds_reads<(WM + WN < WM * WN ? WM + WN : WM * WN)>();
      else if constexpr (S::BF16) sched_mfma_lds_read<(WM + WN < WM * WN ? WM + WN : WM * WN)>();
      __builtin_amdgcn_sched_barrier(0);
      cur = cur == ST - 1 ? 0 : cur + 1;
      fill = fill == ST - 1 ? 0 : fill + 1;
    }
    mfma_step(1);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // loads past the last chunk still write this LDS

  // ---- epilogue
  constexpr int NJ = GATED ? WN / 2 : WN;
  if constexpr (DENSE) {
    store_dense<WM, WN, 16, S::BF16, GATED, ACT>(acc, P, e, m0 + wm * WM * 16 + fr, rows_e, n0 + wn * NJ * 16, lane);
    return;
  }
  const int wrow0 = m0 + wm * WM * 16, wcol0 = n0 + wn * NJ * 16 + 4 * fg;
#pragma unroll
  for (int i = 0; i < WM; ++i) {
    const int row = wrow0 + i * 16 + fr;
    if (row >= rows_e) continue;
    char *prow = static_cast<char *>(P.Cout) + (size_t)(rbase + row) * N * ES;
    char *orow = DIRECT && dest[i] >= 0 ? static_cast<char *>(P.Out) + (size_t)dest[i] * N * ES : nullptr;
    constexpr bool PAIRS = S::BF16 && NJ % 2 == 0;
    uint2 even = make_uint2(0, 0);  // PAIRS: the accumulator before this one
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int col = PAIRS ? wcol0 - 4 * fg + (j & ~1) * 16 + eight_columns_at(fg) : wcol0 + j * 16;
      float c[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        c[u] = acc[i][j][u];
        if (GATED) c[u] = (!S::BF16 ? c[u] / (1.0f + expf(-c[u])) : (ACT == RR_ACT_SWIGLU ? silu(c[u]) : silu_fast(c[u]))) * acc[i][j + NJ][u];
        if (ACT == RR_ACT_GELU) c[u] = gelu_erf(c[u]);
      }
      uint2 val2 = make_uint2(0, 0);
      uint4 val4 = make_uint4(0, 0, 0, 0);
      if constexpr (S::BF16) val2 = make_uint2(pack_bf16(c[0], c[1]), pack_bf16(c[2], c[3]));
      if constexpr (PAIRS) {
        if (j % 2 == 0) {
          even = val2;
          continue;
        }
        val4 = eight_columns(even, val2);
      }
      if (col < N) {  // N % 8 == 0: a group of four or eight columns is inside or outside as a whole
        if constexpr (PAIRS) {
          *reinterpret_cast<uint4 *>(prow + (size_t)col * ES) = val4;
          if (DIRECT && orow) *reinterpret_cast<uint4 *>(orow + (size_t)col * ES) = val4;
        } else if constexpr (S::BF16) {
          *reinterpret_cast<uint2 *>(prow + (size_t)col * ES) = val2;
          if (DIRECT && orow) *reinterpret_cast<uint2 *>(orow + (size_t)col * ES) = val2;
        } else {
          const float4 val = make_float4(c[0], c[1], c[2], c[3]);
          *reinterpret_cast<float4 *>(prow + (size_t)col * ES) = val;
          if (DIRECT && orow) *reinterpret_cast<float4 *>(orow + (size_t)col * ES) = val;
        }
      }
    }
  }
#endif
}

constexpr int kLongRow = 1 << 23;  // elements of a row, from which on rr_ffn.hip has a kernel of its own
constexpr int LG_NW = 16, LG_THREADS = LG_NW * 64, LG_ROWS = 32, LG_COLS = 16;

template <typename Kern>
hipError_t set_lds(Kern kern, int bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

int cu_count() {
  static const int n = [] {  // initialised once, thread-safe (C++11 static)
    int dev = 0, cus = 0;
    hipDeviceProp_t prop;
    if (hipGetDevice(&dev) == hipSuccess && hipGetDeviceProperties(&prop, dev) == hipSuccess) cus = prop.multiProcessorCount;
    return cus > 0 ? cus : 256;
  }();
  return n;
}

// Whole K chunks, at least three (the rings); a ragged row needs one more, so that its last chunk is requested inside the K loop.
bool persistent_ok(int K) { return K % GB_BK == 0 ? K >= 3 * GB_BK : K > 3 * GB_BK; }

//                         BF16   waves  frags ring waves per SIMD
using TileS128 = TileShape<TILE_SPLIT, 2, 2, 4, 4, 1, 3>;  // fp32, 128 rows x 128 staged weight rows
using TileS64 = TileShape<TILE_SPLIT, 2, 2, 2, 4, 1, 4>;   // fp32, 64 x 128
using TileF64 = TileShape<TILE_F32, 2, 2, 2, 4, 2, 2>;     // fp32, 64 x 128
using TileF32 = TileShape<TILE_F32, 2, 2, 1, 4, 2, 2>;     // fp32, 32 x 128
using TileF32n = TileShape<TILE_F32, 2, 2, 1, 2, 3, 2>;    // fp32, 32 x 64
using TileB256 = TileShape<TILE_BF16, 4, 2, 4, 4, 3, 2>;     // bf16, 256 x 128, 8 waves
using TileB128 = TileShape<TILE_BF16, 2, 4, 4, 2, 4, 2>;     // bf16, 128 x 128, 8 waves
using TileB64 = TileShape<TILE_BF16, 2, 2, 2, 4, 3, 2>;      // bf16, 64 x 128
using TileB32 = TileShape<TILE_BF16, 1, 2, 2, 4, 4, 2>;      // bf16, 32 x 128
using TileB32n = TileShape<TILE_BF16, 1, 2, 2, 2, 5, 2>;     // bf16, 32 x 64

template <class S>
struct Tag { using type = S; };

template <class F>
void for_each_tile_shape(F shape) {
  shape(Tag<TileS128>{});
  shape(Tag<TileS64>{});
  shape(Tag<TileF64>{});
  shape(Tag<TileF32>{});
  shape(Tag<TileF32n>{});
  shape(Tag<TileB256>{});
  shape(Tag<TileB128>{});
  shape(Tag<TileB64>{});
  shape(Tag<TileB32>{});
  shape(Tag<TileB32n>{});
}

static_assert(TileB32::BM == kMinRowTile && TileB32n::BM == kMinRowTile && TileF32::BM == kMinRowTile && TileF32n::BM == kMinRowTile && LG_ROWS == kMinRowTile);

// Which tiles a GEMM uses: the shape with the least estimated time.  A CU works through ceil(tiles / CUs) tiles of
// (K chunks x time of a chunk + prologue and epilogue); a chunk takes the longer of
//   cost     its MFMAs and LDS traffic, us per chunk with the CU full, and
//   fetch    its weight bytes that come from HBM (row tiles of one expert share them through L2) at kCuFetch: what
//            one CU sustains against HBM, however deep its ring (a 64 x 128 ring of 6 chunks is no faster than one
//            of 3), so weight-bound layers need their bytes spread evenly over the CUs;
// and no launch is faster than its weights at kHbm.  Large tiles move the fewest operand bytes per flop, small ones
// leave no CU idle.  Measured against the estimate, us: 300 tokens Zipf(1.1), 16 experts, down 5632 -> 2048:
// 32 x 128 92, 64 x 128 108 (one expert has more than 64 rows: 272 tiles), 128 x 128 74; fp32, up / down: 64 x 128
// 213 / 238, 32 x 128 188 / 213, 32 x 64 165 / 168; 16 tokens, 8 experts, down 11008 -> 4096: 32 x 128 141, 32 x 64 133;
// 8 experts 4096 x 11008, K = 11008: 1230 rows 256 x 256 256, 256 x 128 178, 64 x 128 255.
// fp32: the split shapes' numbers are a fit to 260 layers timed in every pair of shapes (1e8 to 5e11 flop).  Of 600 others (5e7 to 3e11)
// the plan is 1.2 % off the best pair on average and 8.5 % faster than the three fp32 shapes were; 16 are 2 - 7 % slower than
// those: their rows per expert are not what the estimate expects, or each weight serves a row or two.
enum FfnShape { FFN_P256, FFN_256, FFN_128, FFN_64, FFN_32, FFN_32N, FFN_S128, FFN_S64, FFN_F64, FFN_F32, FFN_F32N, FFN_LONG };
struct ShapeInfo { int bm, brows; float cost, fixed, alone; };  // alone: of a chunk, where the CU has one workgroup (0: cost)
constexpr ShapeInfo kShape[] = {{256, 256, 1.45f, 5.0f}, {256, 128, 1.0f, 3.0f}, {128, 128, 0.62f, 2.0f},
                                {64, 128, 0.5f, 1.0f},   {32, 128, 0.4f, 1.0f},  {32, 64, 0.3f, 0.3f},
                                {128, 128, 1.37f, 1.1f, 2.8f}, {64, 128, 0.74f, 1.0f, 2.2f},  {64, 128, 1.05f, 1.0f},  {32, 128, 0.5f, 0.7f},  {32, 64, 0.26f, 0.5f},
                                {LG_ROWS, LG_COLS, 0.0f, 0.0f}};
constexpr float kCuFetch = 26e3f, kHbm = 5.9e6f;  // bytes per us
// the 256 x 256 kernel: its start, and a chunk of a tile of which a 1 / n share of the rows is there, n = 1 .. PK_MAX_CUT
constexpr float kPersistentStart = 6.0f, kCutCost[] = {1.0f, 0.72f, 0.6f, 0.53f, 0.5f, 0.47f, 0.45f, 0.43f};
static_assert(sizeof(kCutCost) / sizeof(float) == PK_MAX_CUT);
// the activation of a tile whose workgroup has the CU to itself (256 x 256: in `fixed`; smaller ones overlap theirs)
constexpr float kAct256 = 4.0f, kAct128 = 3.0f;

}  // namespace

}  // namespace rr
