// The feed-forward block's products for few tokens.  Forward, reading the weights
// bounds them: no tiles and no LDS on the way, each weight goes from
// memory to the registers of the one wave that multiplies it.  Rows may start
// at any element.
//
// Up to 2 tokens a wave takes whole rows of the weights, 1 KB at a time, and
// adds in fp32.  Up to 16, 8 or 16 rows a workgroup on MFMA, whose waves take
// runs of K in turn; their sums meet in LDS, added in the waves' order.  Block
// of bf16, one token, 4096 x 11008 54 us (5.0 TB/s), 1600 x 6400 17 us (as tiles
// 78 and 37 us); 4 tokens 59 and 20, 16 tokens 76 and 24 us (tiles 79 and 37);
// 4 tokens by rows, four at a time, 76 us.
//
// h is rounded to the type between the products, as it is for more tokens: up to
// 2 tokens no matrix instruction asks for that, but every row's wave reads h
// whole, and one token's y does not change its precision with the batch.
#pragma once

#include "train_gemm.hpp"

namespace spardl_train {

constexpr int kFewTokens = 16;

// 8 elements from k on of a row of K, zero past its end.
template <typename T>
__device__ __forceinline__ s16x8 row8(const T* row, int k, int K) { return load_raw(row, k, K); }

// Column n of row m of the product.
template <typename T, Epi E>
__device__ __forceinline__ void finish1(const Product& p, int64_t m, int n, float v, float w) {
  if constexpr (E == Epi::Gate) {
    if (p.out2 && n < p.N) {
      ((T*)p.out2)[m * p.ld_io + n] = (T)v;
      ((T*)p.out3)[m * p.ld_io + n] = (T)w;
    }
    activate<1, false>(&v, p.act, &v, nullptr);
    v *= w;
  }
  ((T*)p.out)[m * p.ld_out + n] = (T)v;
}

// A row a wave (of each weight), TOKENS tokens.  Two loads of each in flight: four
// or eight are no faster at 4096 x 11008 (53.1, 53.0, 52.2 us) and slower at
// 1600 x 6400 (17.0, 17.7, 20.6).
template <typename T, int TOKENS, Epi E>
__global__ __launch_bounds__(256) void k_rows(Product p) {
  constexpr int W = E == Epi::Gate ? 2 : 1, UNROLL = 2;
  const int lane = threadIdx.x & 63, n = blockIdx.x * 4 + (threadIdx.x >> 6), K = p.K;
  if (n >= p.pad_n) return;
  const T* weight[W];
#pragma unroll
  for (int w = 0; w < W; ++w) weight[w] = (const T*)p.n[w].p + (int64_t)min(n, p.N - 1) * p.n[w].ld;
  const T* x[TOKENS];
#pragma unroll
  for (int t = 0; t < TOKENS; ++t) x[t] = (const T*)p.m[0].p + (int64_t)min(t, p.M - 1) * p.m[0].ld;
  float acc[W][TOKENS] = {};
  for (int k0 = 8 * lane; k0 < K; k0 += 512 * UNROLL) {
    s16x8 fw[UNROLL][W], fx[UNROLL][TOKENS];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int k = k0 + 512 * u;       // past K: zeros
#pragma unroll
      for (int w = 0; w < W; ++w) fw[u][w] = row8(weight[w], k, K);
#pragma unroll
      for (int t = 0; t < TOKENS; ++t) fx[u][t] = row8(x[t], k, K);
    }
    typedef typename Chunk<T>::Vec Vec;
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
#pragma unroll
      for (int t = 0; t < TOKENS; ++t) {
        const Vec a = __builtin_bit_cast(Vec, fx[u][t]);
#pragma unroll
        for (int w = 0; w < W; ++w) {
          const Vec b = __builtin_bit_cast(Vec, fw[u][w]);
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[w][t] = fmaf((float)a[i], (float)b[i], acc[w][t]);
        }
      }
  }
#pragma unroll
  for (int t = 0; t < TOKENS; ++t) {
    float v = wave_sum(acc[0][t]), w = W == 2 ? wave_sum(acc[W - 1][t]) : 0.f;
    if (n >= p.N) v = w = 0.f;          // columns past N took the last row's weights
    if (lane == 0 && t < p.M) finish1<T, E>(p, t, n, v, w);
  }
}

// The 16 slots of a matrix instruction's operand take RUNS runs of 32 along K of
// 16 / RUNS rows: slot s row s % ROWS of the weights or tokens, run s / ROWS.
// Of the product the blocks of equal runs count and are added up, the others are
// thrown away.  So a load reads 64 RUNS bytes of a row, and half the tokens take
// half the loads.  A workgroup takes PARTS x ROWS rows of the weights and SETS x
// ROWS tokens.  16 rows of 4096 x 11008 bf16, 8 tokens: 68 us with one run, 61
// with two; 16 tokens 76 and, as two sets of 8, 72, but 27 and 31 at 1600 x 6400.
// Fewer rows than CUs can share by 16 take 8 a workgroup: down of 1600 x 6400, 8
// tokens, 11.4 -> 8.4 us, 16 tokens 14.2 -> 11.6; 4096 x 11008 would lose, 61 -> 67.
// Four runs, or two groups of 16 rows a wave, were slower.
template <typename T, Epi E, int RUNS, int PARTS, int SETS>
__global__ __launch_bounds__(512) void k_few(Product p) {
  constexpr int W = E == Epi::Gate ? 2 : 1, WAVES = 8, UNROLL = 2, ROWS = 16 / RUNS;
  constexpr int COLS = PARTS * ROWS, TOKENS = SETS * ROWS, PITCH = COLS + 1;
  __shared__ float sums[WAVES][W * TOKENS * PITCH];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, slot = lane & 15;
  const int n0 = blockIdx.x * COLS, K = p.K, k_lane = 32 * (slot / ROWS) + 8 * (lane >> 4);
  const T* weight[W][PARTS];
#pragma unroll
  for (int w = 0; w < W; ++w)
#pragma unroll
    for (int j = 0; j < PARTS; ++j)
      weight[w][j] = (const T*)p.n[w].p + (int64_t)min(n0 + j * ROWS + slot % ROWS, p.N - 1) * p.n[w].ld;
  const T* x[SETS];
#pragma unroll
  for (int t = 0; t < SETS; ++t) x[t] = (const T*)p.m[0].p + (int64_t)min(t * ROWS + slot % ROWS, p.M - 1) * p.m[0].ld;
  f32x4 acc[W][PARTS][SETS] = {};
  const int units = (K + 32 * RUNS - 1) / (32 * RUNS);
  for (int c0 = wave; c0 < units; c0 += WAVES * UNROLL) {
    s16x8 fw[UNROLL][W][PARTS], fx[UNROLL][SETS];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int k = (c0 + u * WAVES) * 32 * RUNS + k_lane;       // past K: zeros
#pragma unroll
      for (int w = 0; w < W; ++w)
#pragma unroll
        for (int j = 0; j < PARTS; ++j) fw[u][w][j] = row8(weight[w][j], k, K);
#pragma unroll
      for (int t = 0; t < SETS; ++t) fx[u][t] = row8(x[t], k, K);
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
#pragma unroll
      for (int w = 0; w < W; ++w)
#pragma unroll
        for (int j = 0; j < PARTS; ++j)
#pragma unroll
          for (int t = 0; t < SETS; ++t) acc[w][j][t] = Mfma<T>::run(fw[u][w][j], fx[u][t], acc[w][j][t]);
  }
  // Lane l holds the weights' slots 4 (l / 16) .. + 3 of the tokens' slot l % 16:
  // a run on, both slots are ROWS further.
#pragma unroll
  for (int w = 0; w < W; ++w)
#pragma unroll
    for (int j = 0; j < PARTS; ++j)
#pragma unroll
      for (int t = 0; t < SETS; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float v = acc[w][j][t][i];
          if constexpr (RUNS == 2) v += __shfl(v, (lane + 16 * ROWS / 4 + ROWS) & 63);
          if (slot < ROWS && lane >> 4 < ROWS / 4)
            sums[wave][(w * TOKENS + t * ROWS + slot) * PITCH + j * ROWS + 4 * (lane >> 4) + i] = v;
        }
  __syncthreads();
  // eight columns of one token a thread
  const int token = threadIdx.x / (COLS / 8), col = threadIdx.x % (COLS / 8) * 8;
  if (token >= min(TOKENS, p.M) || n0 + col >= p.pad_n) return;
  float v[W][8] = {};
  for (int s = 0; s < WAVES; ++s)
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int i = 0; i < 8; ++i) v[w][i] += sums[s][(w * TOKENS + token) * PITCH + col + i];
  // columns past N took the last row's weights: finish8 clears or leaves them out
  finish8<T, E>(p, token, n0 + col, v[0], v[W - 1], Saved{});
}

template <typename T, Epi E>
hipError_t launch_few(const Product& p, hipStream_t s) {
  const dim3 rows((uint32_t)ceil_div(p.pad_n, 4)), groups((uint32_t)ceil_div(p.pad_n, 16)), halves((uint32_t)ceil_div(p.pad_n, 8));
  if (p.M == 1) k_rows<T, 1, E><<<rows, 256, 0, s>>>(p);
  else if (p.M == 2) k_rows<T, 2, E><<<rows, 256, 0, s>>>(p);
  // 8 rows a group where that gives no CU a second one
  else if (halves.x <= 256 && p.M <= 8) k_few<T, E, 2, 1, 1><<<halves, 512, 0, s>>>(p);
  else if (halves.x <= 256) k_few<T, E, 2, 1, 2><<<halves, 512, 0, s>>>(p);
  else if (p.M <= 8) k_few<T, E, 2, 2, 1><<<groups, 512, 0, s>>>(p);
  else k_few<T, E, 1, 1, 1><<<groups, 512, 0, s>>>(p);
  return launched();
}

// The weights' gradients from up to 32 tokens: one matrix instruction takes them
// all, and writing bounds the launch.  128 rows of a gradient a workgroup, 16 a
// wave, of 256 columns, whose tokens it turns over in LDS.  The first operand's
// slots take columns 8 (s / 4) + s % 4 and, for a second instruction, 4 further:
// so a lane holds eight columns of one row.  The three of 3584 x 3584 fp16, 2
// tokens: 18.7 us (4.1 TB/s), as tiles 34.8; the whole backward pass of 32 tokens,
// 1600 x 6400, 62 -> 55 us, 4096 x 11008 196 -> 170.
constexpr int kOuterTokens = 32, kOuterRows = 128, kOuterCols = 256;
template <typename T>
__global__ __launch_bounds__(512) void k_outer(Gemm g) {
  constexpr int PITCH = kOuterTokens + 8;        // 16-byte aligned, and spread over the banks
  __shared__ __attribute__((aligned(16))) short cols[kOuterCols * PITCH];
  int which = 0;
  while (which + 1 < g.products && (int)blockIdx.x >= g.p[which + 1].first) ++which;
  const Product& p = g.p[which];
  const int tile = blockIdx.x - p.first, tm = tile / p.tiles_n, n0 = tile % p.tiles_n * kOuterCols;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, slot = lane & 15, oct = lane >> 4;
  const int64_t m = (int64_t)tm * kOuterRows + wave * 16 + slot;
  for (int i = threadIdx.x; i < kOuterTokens * kOuterCols / 8; i += 512) {
    const int t = i % kOuterTokens, c = i / kOuterTokens * 8;
    s16x8 v = {};
    if (t < p.K && n0 + c < p.N) v = load_raw((const T*)p.n[0].p + t * p.n[0].ld, n0 + c, p.N);
#pragma unroll
    for (int j = 0; j < 8; ++j) cols[(c + j) * PITCH + t] = v[j];
  }
  s16x8 row = {};
  if (m < p.M) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (8 * oct + j < p.K) row[j] = ((const short*)p.m[0].p)[(8 * oct + j) * p.m[0].ld + m];
  }
  __syncthreads();
  // lanes past the last row hold columns all the same: only their stores stay out
#pragma unroll 2
  for (int c = 0; c < kOuterCols; c += 32) {
    const short* const at = cols + (c + 8 * (slot >> 2) + (slot & 3)) * PITCH + 8 * oct;
    f32x4 v[2];
    v[0] = Mfma<T>::run(*(const s16x8*)at, row, f32x4{});
    v[1] = Mfma<T>::run(*(const s16x8*)(at + 4 * PITCH), row, f32x4{});
    const int n = n0 + c + 8 * oct;
    if (m < p.M && n < p.N) finish8<T, Epi::Store>(p, m, n, (float*)v, nullptr, Saved{});
  }
}

template <typename T>
hipError_t launch_outer(Gemm& g, hipStream_t s) {
  g.tiles = 0;
  for (int i = 0; i < g.products; ++i) {
    Product& p = g.p[i];
    p.tiles_m = (int32_t)ceil_div(p.M, kOuterRows);
    p.tiles_n = (int32_t)ceil_div(p.N, kOuterCols);
    p.first = g.tiles;
    g.tiles += p.tiles_m * p.tiles_n;
  }
  if (g.tiles == 0) return hipSuccess;
  k_outer<T><<<dim3((uint32_t)g.tiles), 512, 0, s>>>(g);
  return launched();
}

}  // namespace spardl_train
