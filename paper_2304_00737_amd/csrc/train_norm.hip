// The residual RMS norm and its backward pass.  Both stream their rows once:
// a row lives in the registers of the threads that share it, so the bytes
// bound them (two rows in and two out forward, three in and one out backward).
// 16384 x 4096 bf16: forward 89 us, 6.0 TB/s; backward 105 us, 5.1 TB/s; fp32 179
// and 181 us.  Narrow rows do not fill their lanes, since a wave holds one row:
// 65536 x 256 bf16 (32 of 64 lanes) 32 and 50 us for 22 of bytes, x 64 (8 lanes)
// 24 and 40 for 5.4.

#include "train.hpp"

namespace spardl_train {

namespace {

// Threads that share a row, and 16-byte chunks that each of them holds.
template <typename T, int THREADS, int NCH>
struct RowShape {
  static constexpr int ROWS = THREADS == 64 ? 4 : 1;      // rows of a workgroup
  static constexpr int BLOCK = THREADS * ROWS;
  static constexpr int N = Chunk<T>::N;
};

template <typename T, int THREADS, int NCH>
__global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void k_rms_norm(
    const T* x, int64_t ld_x, const T* res, int64_t ld_res, const T* weight, T* sum, int64_t ld_sum, T* y,
    int64_t ld_y, float* rstd, int64_t rows, int dim, float eps) {
  using S = RowShape<T, THREADS, NCH>;
  __shared__ float lds[S::BLOCK / 64];
  const int t = threadIdx.x % THREADS;
  const int64_t row = (int64_t)blockIdx.x * S::ROWS + threadIdx.x / THREADS;
  if (row >= rows) return;    // whole waves: rows share no barrier when a workgroup holds several
  float v[NCH][S::N];
  float sq = 0.f;
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int e0 = (c * THREADS + t) * S::N;
    if (e0 < dim) load_chunk<T, true>(x + row * ld_x, e0, dim, 0.f, v[c]);
  }
  if (res) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e0 = (c * THREADS + t) * S::N;
      if (e0 >= dim) continue;
      float a[S::N];
      load_chunk<T, true>(res + row * ld_res, e0, dim, 0.f, a);
#pragma unroll
      for (int i = 0; i < S::N; ++i) v[c][i] += a[i];
    }
  }
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int e0 = (c * THREADS + t) * S::N;
    if (e0 >= dim) continue;
#pragma unroll
    for (int i = 0; i < S::N; ++i) sq = fmaf(v[c][i], v[c][i], sq);
    if (sum) store_chunk<T, true>(sum + row * ld_sum, e0, dim, v[c]);
  }
  sq = group_sum<THREADS>(sq, lds);
  const float r = rsqrtf(sq / (float)dim + eps);
#pragma unroll
  for (int c = 0; c < NCH; ++c) {
    const int e0 = (c * THREADS + t) * S::N;
    if (e0 >= dim) continue;
    float w[S::N];
    load_chunk(weight, e0, dim, 0.f, w);
#pragma unroll
    for (int i = 0; i < S::N; ++i) v[c][i] = v[c][i] * r * w[i];
    store_chunk<T, true>(y + row * ld_y, e0, dim, v[c]);
  }
  if (rstd && t == 0) rstd[row] = r;
}

template <int N>
__device__ __forceinline__ void store_chunk_f32(float* row, int e0, int dim, const float* v) {
#pragma unroll
  for (int i = 0; i < N; i += 4) store_chunk(row, e0 + i, dim, v + i);
}

// A workgroup walks rows b, b + grid, ..., and keeps its part of dweight in
// registers; part[b] receives it at the end, a workgroup's rows joined in LDS.  The next row is loaded, packed, while the
// present one is worked on, where a thread's share of two rows fits its
// registers (16384 x 4096 bf16: 111 us without, 102 with).  fp32 rows past 8192
// spill 17 registers a lane: 4096 x 16384 206 us for 173 of bytes.
template <typename T, int THREADS, int NCH>
__global__ __launch_bounds__(THREADS == 64 ? 256 : THREADS) void k_rms_norm_backward(
    const T* dy, int64_t ld_dy, const T* sum, int64_t ld_sum, const T* weight, const float* rstd, const T* dsum,
    int64_t ld_dsum, T* dx, int64_t ld_dx, float* part, int64_t rows, int dim) {
  using S = RowShape<T, THREADS, NCH>;
  using Vec = typename Chunk<T>::Vec;
  __shared__ float lds[2][S::BLOCK / 64];
  const int t = threadIdx.x % THREADS;
  const int64_t slot = (int64_t)blockIdx.x * S::ROWS + threadIdx.x / THREADS, stride = (int64_t)gridDim.x * S::ROWS;
  float dw[NCH][S::N] = {};
  constexpr bool AHEAD = THREADS < 1024;
  i32x4 w[NCH], next[3][NCH];
  float r = 0.f, r_next = 0.f;
#pragma unroll
  for (int c = 0; c < NCH; ++c) w[c] = load_packed(weight, (c * THREADS + t) * S::N, dim);
  auto load = [&](int64_t row) {
    r_next = rstd[row];
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e0 = (c * THREADS + t) * S::N;
      next[0][c] = load_packed<T, true>(dy + row * ld_dy, e0, dim);
      next[1][c] = load_packed<T, true>(sum + row * ld_sum, e0, dim);
      if (dsum) next[2][c] = load_packed<T, true>(dsum + row * ld_dsum, e0, dim);
    }
  };
#pragma unroll
  for (int c = 0; c < NCH; ++c) next[2][c] = i32x4{};
  if (AHEAD && slot < rows) load(slot);
  int turn = 0;
  for (int64_t row = slot; row < rows; row += stride, turn ^= 1) {
    if (!AHEAD) load(row);
    i32x4 here[3][NCH];
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
      for (int c = 0; c < NCH; ++c) here[k][c] = next[k][c];
    r = r_next;
    if (AHEAD && row + stride < rows) load(row + stride);
    float dot = 0.f;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const Vec vy = __builtin_bit_cast(Vec, here[0][c]), vx = __builtin_bit_cast(Vec, here[1][c]);
      const Vec vw = __builtin_bit_cast(Vec, w[c]);
#pragma unroll
      for (int i = 0; i < S::N; ++i) {
        const float y = (float)vy[i], xh = (float)vx[i] * r;
        dw[c][i] = fmaf(y, xh, dw[c][i]);
        dot = fmaf(y * (float)vw[i], xh, dot);
      }
    }
    dot = group_sum<THREADS>(dot, lds[turn]) / (float)dim;   // two turns: no thread still reads the last one's
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e0 = (c * THREADS + t) * S::N;
      if (e0 >= dim) continue;
      const Vec vy = __builtin_bit_cast(Vec, here[0][c]), vx = __builtin_bit_cast(Vec, here[1][c]);
      const Vec vw = __builtin_bit_cast(Vec, w[c]), vd = __builtin_bit_cast(Vec, here[2][c]);
      float g[S::N];
#pragma unroll
      for (int i = 0; i < S::N; ++i) g[i] = fmaf(r, (float)vy[i] * (float)vw[i] - (float)vx[i] * r * dot, (float)vd[i]);
      store_chunk<T, true>(dx + row * ld_dx, e0, dim, g);
    }
  }
  float* const to = part + (int64_t)blockIdx.x * dim;
  if constexpr (S::ROWS == 1) {
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const int e0 = (c * THREADS + t) * S::N;
      if (e0 < dim) store_chunk_f32<S::N>(to, e0, dim, dw[c]);
    }
  } else {
    __shared__ float rows_dw[S::ROWS][THREADS * NCH * S::N];
#pragma unroll
    for (int c = 0; c < NCH; ++c)
#pragma unroll
      for (int i = 0; i < S::N; ++i) rows_dw[threadIdx.x / THREADS][(c * THREADS + t) * S::N + i] = dw[c][i];
    __syncthreads();
    for (int i = threadIdx.x; i < dim; i += S::BLOCK) {
      float v = rows_dw[0][i];
#pragma unroll
      for (int k = 1; k < S::ROWS; ++k) v += rows_dw[k][i];
      to[i] = v;
    }
  }
}

// dweight[c] = sum over the slots of part[slot][c]: 32 columns and 32 runs of
// slots per workgroup, the runs added in order.
__global__ __launch_bounds__(1024) void k_column_sum(const float* part, float* out, int slots, int dim) {
  __shared__ float lds[32][33];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), run = threadIdx.x >> 5;
  const int per = (slots + 31) / 32;
  const int end = min(slots, (run + 1) * per);
  float v = 0.f;
  int i = run * per;
  if (col < dim) {
    for (; i + 8 <= end; i += 8) {           // eight loads under way
      float u[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) u[k] = part[(int64_t)(i + k) * dim + col];
#pragma unroll
      for (int k = 0; k < 8; ++k) v += u[k];
    }
    for (; i < end; ++i) v += part[(int64_t)i * dim + col];
  }
  lds[run][threadIdx.x & 31] = v;
  __syncthreads();
  if (run == 0 && col < dim) {
    v = 0.f;
    for (int k = 0; k < 32; ++k) v += lds[k][threadIdx.x];
    out[col] = v;
  }
}

// Calls f.template operator()<T, THREADS, NCH>() of the shape for rows of dim.
template <typename T, typename F>
void with_shape(int dim, F f) {
  const int chunks = (dim + Chunk<T>::N - 1) / Chunk<T>::N;
  if (chunks <= 64) f.template operator()<T, 64, 1>();
  else if (chunks <= 128) f.template operator()<T, 64, 2>();
  else if (chunks <= 256) f.template operator()<T, 256, 1>();
  else if (chunks <= 512) f.template operator()<T, 256, 2>();
  else if (chunks <= 1024) f.template operator()<T, 512, 2>();
  else if (chunks <= 2048) f.template operator()<T, 1024, 2>();
  else if constexpr (sizeof(T) == 4) f.template operator()<T, 1024, 4>();
}
template <typename F>
void with_type_and_shape(int32_t dtype, int dim, F f) {
  if (dtype == SPARDL_BF16) with_shape<bf16>(dim, f);
  else if (dtype == SPARDL_FP16) with_shape<fp16>(dim, f);
  else with_shape<float>(dim, f);
}

struct Forward {
  const void *x, *res, *weight;
  void *sum, *y;
  int64_t ld_x, ld_res, ld_sum, ld_y, rows;
  float* rstd;
  int dim;
  float eps;
  hipStream_t s;
  template <typename T, int THREADS, int NCH>
  void operator()() const {
    using S = RowShape<T, THREADS, NCH>;
    k_rms_norm<T, THREADS, NCH><<<dim3((uint32_t)ceil_div(rows, S::ROWS)), S::BLOCK, 0, s>>>(
        (const T*)x, ld_x, (const T*)res, ld_res, (const T*)weight, (T*)sum, ld_sum, (T*)y, ld_y, rstd, rows, dim, eps);
  }
};

// Workgroups of the backward pass at most, each with a row of partial weight
// gradients: short rows take more of them to keep the card's loads under way,
// long rows' partial sums cost as much as a few rows each.
template <int THREADS, int NCH>
constexpr int64_t kGroups = THREADS * NCH <= 256 ? 2048 : THREADS == 256 ? 1024 : THREADS == 512 ? 512 : 256;

template <typename F>
struct Groups {
  F see;
  template <typename T, int THREADS, int NCH>
  void operator()() const { see(kGroups<THREADS, NCH>); }
};
template <typename F>
Groups(F) -> Groups<F>;

struct Backward {
  const void *dy, *sum, *weight, *dsum;
  void* dx;
  int64_t ld_dy, ld_sum, ld_dsum, ld_dx, rows;
  const float* rstd;
  float *dweight, *part;
  int dim;
  hipStream_t s;
  template <typename T, int THREADS, int NCH>
  void operator()() const {
    using S = RowShape<T, THREADS, NCH>;
    const int64_t blocks = rows < 1 ? 1 : ceil_div(rows, S::ROWS), most = kGroups<THREADS, NCH>;
    const int64_t grid = blocks < most ? blocks : most;
    k_rms_norm_backward<T, THREADS, NCH><<<dim3((uint32_t)grid), S::BLOCK, 0, s>>>(
        (const T*)dy, ld_dy, (const T*)sum, ld_sum, (const T*)weight, rstd, (const T*)dsum, ld_dsum, (T*)dx, ld_dx,
        grid == 1 ? dweight : part, rows, dim);      // one workgroup: its sum is the gradient
    if (grid > 1) k_column_sum<<<dim3((uint32_t)ceil_div(dim, 32)), 1024, 0, s>>>(part, dweight, (int)grid, dim);
  }
};

}  // namespace

hipError_t launch_rms_norm(const void* x, int64_t ld_x, const void* res, int64_t ld_res, const void* weight, void* sum,
                           int64_t ld_sum, void* y, int64_t ld_y, float* rstd, int64_t rows, int32_t dim, float eps,
                           int32_t dtype, hipStream_t s) {
  if (rows == 0) return hipSuccess;
  auto at = [&](const void* p, int64_t ld, int64_t r) {
    return p ? (char*)p + r * ld * (dtype == SPARDL_FP32 ? 4 : 2) : nullptr;
  };
  for (int64_t r = 0; r < rows; r += kRowsPerLaunch)
    with_type_and_shape(dtype, dim, Forward{at(x, ld_x, r), at(res, ld_res, r), weight, at(sum, ld_sum, r), at(y, ld_y, r),
                                            ld_x, ld_res, ld_sum, ld_y,
                                            rows - r < kRowsPerLaunch ? rows - r : kRowsPerLaunch,
                                            rstd ? rstd + r : nullptr, dim, eps, s});
  return launched();
}

size_t rms_norm_ws(int64_t rows, int32_t dim) {
  // the largest of the types' shapes
  int64_t most = 0;
  auto see = [&](int64_t groups) { most = most > groups ? most : groups; };
  with_shape<bf16>(dim, Groups{see});
  with_shape<float>(dim, Groups{see});
  return align256((size_t)(rows < 1 ? 1 : rows < most ? rows : most) * dim * sizeof(float));
}

hipError_t launch_rms_norm_backward(const void* dy, int64_t ld_dy, const void* sum, int64_t ld_sum, const void* weight,
                                    const float* rstd, const void* dsum, int64_t ld_dsum, void* dx, int64_t ld_dx,
                                    float* dweight, int64_t rows, int32_t dim, int32_t dtype, void* ws, hipStream_t s) {
  with_type_and_shape(dtype, dim, Backward{dy, sum, weight, dsum, dx, ld_dy, ld_sum, ld_dsum, ld_dx, rows, rstd, dweight,
                                           (float*)ws, dim, s});
  return launched();
}

}  // namespace spardl_train
