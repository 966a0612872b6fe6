// Matrix products of the gated feed-forward block: one kernel template on
// MFMA 16x16x32, whose operands may each run along K (rows of K elements) or
// across it (K rows of the operand's extent), with the block's elementwise
// work in its epilogue.
//
// A workgroup computes a BM x BN tile of C[m][n] = sum over k of M(m,k) N(n,k)
// in K steps of 64.  Both operands' steps go straight from memory to LDS (16
// bytes a lane) into a ring of STAGES buffers, and a wave holds the fragments
// of one half step in registers while it multiplies the other half, so that
// one barrier per step remains, between its halves: after it the next step's
// data are in LDS and nobody reads this one's any more, so its buffer takes
// the loads of the step STAGES further on.
//
// LDS layout.  Along K: rows of 64 elements = 8 chunks of 16 bytes, chunk c of
// row r at place c ^ (r & 7), read by 16-byte loads.  Across K: 64 rows of the
// tile's extent, chunk c of row k at place c ^ f(k), read by the transposing
// 8-byte loads (16 lanes take 4 rows x 16 columns and get 4 k of one column
// each).  The exclusive-or spreads what a wave reads at once over all banks.
//
// What bounds it, at 8192 x 4096 x 11008 bf16: h w_down^T takes 600 us (1.23
// PFLOP/s, matrix cores busy 62 % at 2.0 GHz): 64 KB a step and CU from L2 into
// LDS, which alone take 0.5 to 0.6 us of the 1.65 us of a step.  (An earlier
// state of this kernel, in a run of its own: 573 us whole, 402 without its
// loads, 409 with half of them, 579 without its LDS reads.)  Weight gradients
// 1.74 ms (1.27), gradient of x 1.11 ms (1.33), gate and up 1.24 ms (1.20), the
// gate's backward product 0.79 ms (0.94, its epilogue moves 0.9 GB).  A lone
// tile of 128 on a CU: 6 us of launch, first loads and epilogue, and 0.5 us a
// step, of which the matrix cores take 0.24 and LDS reads 0.21; its waves wait
// for 40 % of their time, for LDS 4 to 8 %.
#pragma once

#include "train.hpp"

namespace spardl_train {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr int KSTEP = 64;          // elements of K per step

enum class Epi { Store, Gate, GateBackward };

struct Side {
  const void* p;
  int64_t ld;
};

// One product of a launch.  Two segments: K runs over (m[0], n[0]) and then
// (m[1], n[1]).  Epi::Gate: n[0] and n[1] are the two weights of one pass.
struct Product {
  Side m[2], n[2];
  int32_t M, N, K, segments;
  int32_t tiles_m, tiles_n;
  int32_t first;                   // its first tile among the launch's
  // epilogue
  void* out;                       // Store: the result.  GateBackward: dgate.  Gate: h
  void *out2, *out3;               // GateBackward: dup, h.  Gate: gate, up (may be null)
  const void *in, *in2;            // GateBackward: gate, up
  int64_t ld_out, ld_io;           // ld_io: Gate's gate and up, GateBackward's inputs
  int32_t pad_n;                   // columns up to here are written to out (and GateBackward's out2, out3)
  int32_t out_f32, accumulate, act;
};

struct Gemm {
  Product p[3];
  int32_t products, tiles;
  int32_t whole, splits;           // tiles from `whole` on are each cut into `splits` runs of K
  float* part;                     // splits > 1: [tile - whole][split][BM][BN]
};

template <typename T>
struct Mfma;
template <>
struct Mfma<bf16> {
  typedef bf16 V8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 run(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
  }
};
template <>
struct Mfma<fp16> {
  typedef fp16 V8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ f32x4 run(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V8, a), __builtin_bit_cast(V8, b), c, 0, 0, 0);
  }
};

// ---------------------------------------------------------------- epilogue

// a = act(g) and, with SLOPE, its derivative, for N values; in place of g too.
//
// The error function comes from erfc(x) = exp(-x^2) P(t), t = 1 / (1 + 0.38 x),
// x >= 0, with P fitted to exp(x^2) erfc(x) for the least relative error over
// [0, 14] (1.1e-6): the derivative needs the same exponential, and small tails
// keep their leading digits.
template <int N, bool SLOPE>
__device__ __forceinline__ void activate(const float* g, int act, float* a, float* slope) {
  if (act == SPARDL_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float t = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g[i] * -1.44269504f));
      a[i] = g[i] * t;
      if constexpr (SLOPE) slope[i] = fmaf(a[i], 1.f - t, t);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float z = g[i], t = __builtin_amdgcn_rcpf(fmaf(0.38f * 0.70710678f, fabsf(z), 1.f));
      const float e = __builtin_amdgcn_exp2f(z * z * -0.72134752f);
      float q = fmaf(t, -0.12541800737380981f, 0.33603665232658386f);
      q = fmaf(t, q, -0.06991185247898102f);
      q = fmaf(t, q, 0.2478320151567459f);
      q = fmaf(t, q, 0.1805957704782486f);
      q = fmaf(t, q, 0.21657703816890717f);
      q = fmaf(t, q, 0.21428734064102173f);
      const float tail = 0.5f * (q * t) * e, phi = z < 0.f ? tail : 1.f - tail;
      a[i] = z * phi;
      if constexpr (SLOPE) slope[i] = fmaf(z * 0.39894228f, e, phi);
    }
  }
}

// What GateBackward reads for columns n .. n + 7 of row m: gate and up.
struct Saved {
  s16x8 gate, up;
};
template <typename T>
__device__ __forceinline__ s16x8 load_raw(const T* row, int n, int end) {
  return __builtin_bit_cast(s16x8, load_packed(row, n, end));
}
template <typename T>
__device__ __forceinline__ Saved load_saved(const Product& p, int64_t m, int n) {
  return {load_raw((const T*)p.in + m * p.ld_io, n, p.N), load_raw((const T*)p.in2 + m * p.ld_io, n, p.N)};
}

// Zeros for what lies past the product's columns: there a row of infinities met the weights' padding, and its NaN
// would reach the whole row through the next product.
__device__ __forceinline__ void clear_padding(const Product& p, int n, float* v) {
  if (n + 8 <= p.N) return;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (n + i >= p.N) v[i] = 0.f;
}

// Columns n .. n + 7 of row m of the product: v (Gate: the gate's v, the up's w).
template <typename T, Epi E>
__device__ __forceinline__ void finish8(const Product& p, int64_t m, int n, float* v, const float* w, const Saved& io) {
  if constexpr (E == Epi::Store) {
    auto to = [&](auto* out) {
      auto* row = out + m * p.ld_out;
      constexpr int N = 16 / sizeof(*out);     // columns of one store
#pragma unroll
      for (int c = 0; c < 8; c += N) {
        if (p.accumulate) {
          float old[N];
          load_chunk(row, n + c, p.pad_n, 0.f, old);
#pragma unroll
          for (int i = 0; i < N; ++i) v[c + i] += old[i];
        }
        store_chunk(row, n + c, p.pad_n, v + c);
      }
    };
    if (p.out_f32) to((float*)p.out);
    else to((T*)p.out);
  } else if constexpr (E == Epi::Gate) {
    if (p.out2) {
      store_chunk((T*)p.out2 + m * p.ld_io, n, p.N, v);
      store_chunk((T*)p.out3 + m * p.ld_io, n, p.N, w);
    }
    activate<8, false>(v, p.act, v, nullptr);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= w[i];
    clear_padding(p, n, v);
    store_chunk((T*)p.out + m * p.ld_out, n, p.pad_n, v);
  } else {
    float g[8], u[8], h[8], slope[8];
    const auto gate = __builtin_bit_cast(typename Chunk<T>::Vec, io.gate);   // whole: an element's cast reads the first
    const auto up = __builtin_bit_cast(typename Chunk<T>::Vec, io.up);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      g[i] = (float)gate[i];
      u[i] = (float)up[i];
    }
    activate<8, true>(g, p.act, h, slope);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      g[i] = v[i] * u[i] * slope[i];
      const float a = h[i];
      h[i] = a * u[i];
      u[i] = v[i] * a;
    }
    clear_padding(p, n, g);
    clear_padding(p, n, u);
    clear_padding(p, n, h);
    store_chunk((T*)p.out + m * p.ld_out, n, p.pad_n, g);
    store_chunk((T*)p.out2 + m * p.ld_out, n, p.pad_n, u);
    store_chunk((T*)p.out3 + m * p.ld_out, n, p.pad_n, h);
  }
}

// ---------------------------------------------------------------- tiles

// Swizzle of row k of a tile that lies across K, CPR chunks a row.
template <int CPR>
__device__ __forceinline__ int across_place(int k) {
  return (2 * ((k & 3) | (((k >> 3) & 1) << 2))) & (CPR - 1);
}

// 16 bytes a lane from the buffer at voff + soff (0 past its end) to the LDS
// address dst + 16 * lane.  As a builtin the compiler would wait for it before
// any transposing read of LDS, whose place it does not tell apart: every wait
// for these loads is written out (landed_barrier).  Scalars that a vector
// instruction wrote take up to five wait states, M0 one.
__device__ __forceinline__ void load_to_lds(i32x4 buffer, int dst, int voff, int soff) {
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(voff), "s"(buffer), "s"(soff), "{m0}"(dst)
               : "memory");
}

// One operand's loads into LDS, a K step at a time, for one wave: rows (or,
// across K, columns) from r0 on; what lies outside the matrix reads as 0.  The
// contiguous extent (K, or across it R) is taken up to the next multiple of
// 8: the host passes rows that reach that far, zero past K.  The waves take
// loads of 1024 bytes in turn.  DUAL: 16 rows of the gate's weight, then the
// same 16 of the up's, and so on, so that a wave only ever loads one of them.
template <bool ALONG, bool DUAL, int EXTENT, int WAVES>
struct Loader {
  static constexpr int CPR = EXTENT / 8;                               // chunks a row, across K
  static constexpr int RPL = ALONG ? 8 : 64 / CPR;                     // rows a load
  static constexpr int LOADS = EXTENT * KSTEP * 2 / 1024 / WAVES;
  static constexpr int VOFFS = !ALONG && RPL * WAVES == 8 ? 2 : 1;     // swizzles that alternate with the load
  static_assert(ALONG || RPL * WAVES >= 8, "more swizzles than offsets");
  static_assert(!DUAL || WAVES % 4 == 0, "a wave loads from one weight");

  const char* at;      // the tile's first element of a step
  int64_t left;        // bytes from it to the end of the matrix
  int64_t step;        // bytes from one step to the next
  int stride;          // bytes from one load's rows to the next's
  int voff[VOFFS];

  __device__ __forceinline__ void start(const Side& q, int r0, int R, int k0, int K, int wave, int lane) {
    const int row_bytes = (int)q.ld * 2;
    if constexpr (ALONG) {
      at = (const char*)q.p + 2 * ((int64_t)r0 * q.ld + k0);
      left = 2 * ((int64_t)(R - 1 - r0) * q.ld + (((K + 7) & ~7) - k0));
      step = KSTEP * 2;
      const int row = DUAL ? (wave >> 2) * 16 + (wave & 1) * 8 + (lane >> 3) : wave * 8 + (lane >> 3);
      voff[0] = row * row_bytes + (((lane & 7) ^ (lane >> 3)) << 4);
      stride = (DUAL ? 4 : 8) * WAVES * row_bytes;
    } else {
      at = (const char*)q.p + 2 * ((int64_t)k0 * q.ld + r0);
      left = 2 * ((int64_t)(K - 1 - k0) * q.ld + (((R + 7) & ~7) - r0));
      step = (int64_t)KSTEP * row_bytes;
#pragma unroll
      for (int j = 0; j < VOFFS; ++j) {
        const int k = (j * WAVES + wave) * RPL + lane / CPR;
        voff[j] = (wave * RPL + lane / CPR) * row_bytes + (((lane % CPR) ^ across_place<CPR>(k)) << 4);
      }
      stride = WAVES * RPL * row_bytes;
    }
  }
  // Prepares a step's loads; k: elements of K from this step on, along K (the
  // last step may be short).  With more = false nothing is read from memory.
  __device__ __forceinline__ void begin(int lane, int k, bool more) {
    const int high = (int)(left >> 32);     // in 32-bit halves: scalar compares
    const uint32_t low = (uint32_t)left;
    buffer.x = (int)(uintptr_t)at;
    buffer.y = (int)((uintptr_t)at >> 32) & 0xffff;
    buffer.z = !more || high < 0 ? 0 : high > 0 || low > 0x7ffffff0u ? 0x7ffffff0 : (int)low;
    buffer.w = 0x00020000;
#pragma unroll
    for (int j = 0; j < VOFFS; ++j) off[j] = voff[j];
    if (ALONG && (((lane & 7) ^ (lane >> 3)) << 3) >= k) off[0] = 0x7ffffffc;      // past the buffer
    at += step;
    left -= step;
  }
  // Load j of the step, of LOADS.
  __device__ __forceinline__ void issue(int dst, int wave, int j) const {
    load_to_lds(buffer, dst + (j * WAVES + wave) * 1024, off[j % VOFFS], j * stride);
  }
  i32x4 buffer;
  int off[VOFFS];
};

// Fragment of 16 rows (from `first` on) and 32 k (half `half` of the step):
// lane l holds row l % 16, k = 8 (l / 16) .. + 7.
template <bool ALONG, int EXTENT>
__device__ __forceinline__ s16x8 read_fragment(const lds_char* tile, int first, int half, int lane) {
  typedef __attribute__((address_space(3))) const s16x8 lds_s16x8;
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  if constexpr (ALONG) {
    const int row = first + (lane & 15);
    return *(lds_s16x8*)(tile + row * 128 + (((half * 4 + (lane >> 4)) ^ (lane & 7)) << 4));
  } else {
    constexpr int CPR = EXTENT / 8;
    const int r = lane & 15, k = half * 32 + 8 * (lane >> 4) + (r >> 2);
    const int chunk = ((first >> 3) + ((r & 3) >> 1)) ^ across_place<CPR>(k);   // the same for k + 4
    const lds_char* at = tile + k * (EXTENT * 2) + chunk * 16 + (r & 1) * 8;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * (EXTENT * 2)));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}

// All but the wave's latest LEFT loads into LDS have landed, what it read from LDS is in its
// registers, and every wave has got here.  The waits are its own: no register
// depends on the loads, so a barrier alone would not wait for them.
template <int LEFT>
__device__ __forceinline__ void landed_barrier() {
  static_assert(LEFT < 64, "the counter's range");
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LEFT) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Tile of a launch that workgroup `id` computes.  Workgroups go to the eight
// XCDs in turn: each XCD gets a run of neighbouring tiles, so that its L2
// holds the rows and columns that they share.
__device__ __forceinline__ int spread(int id, int total) {
  const int q = total / 8, r = total % 8, x = id & 7;
  return x * q + min(x, r) + (id >> 3);
}

// A tile's product and place: eight tiles of m by all of n at a time.
struct Place {
  int which, tm, tn;
};
__device__ __forceinline__ Place place(const Gemm& g, int tile) {
  int which = 0;
  while (which + 1 < g.products && tile >= g.p[which + 1].first) ++which;
  const Product& p = g.p[which];
  tile -= p.first;
  const int group = tile / (8 * p.tiles_n), in_group = tile % (8 * p.tiles_n);
  const int height = min(8, p.tiles_m - group * 8);
  return {which, group * 8 + in_group % height, in_group / height};
}

template <typename T, int BM, int BN, int WM, int WN, int PER_CU, int STAGES, bool M_ALONG, bool N_ALONG, Epi E>
__global__ __launch_bounds__(64 * WM * WN, PER_CU * WM * WN / 4) void k_gemm(Gemm g) {
  constexpr bool DUAL = E == Epi::Gate;
  constexpr int WAVES = WM * WN, MF = BM / WM / 16, NF = BN / WN / 16;
  constexpr int M_BYTES = BM * KSTEP * 2, N_BYTES = BN * KSTEP * 2;
  // STAGES buffers of M's step, then of N's
  constexpr int STRIP = (BN / WN + 4) * 4;                 // a row of a wave's part, in fp32, for the epilogue
  __shared__ __attribute__((aligned(1024))) char lds[STAGES * (M_BYTES + N_BYTES)];
  lds_char* const base = (lds_char*)lds;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int id = blockIdx.x, tail = id - g.whole;
  const bool cut = tail >= 0 && g.splits > 1;
  const int job = tail < 0 ? spread(id, g.whole) : spread(tail, (g.tiles - g.whole) * g.splits);
  const int split = cut ? job % g.splits : 0, splits = cut ? g.splits : 1;
  const Place at = place(g, tail < 0 ? job : g.whole + job / g.splits);
  const Product& p = g.p[at.which];
  const int m0 = at.tm * BM, n0 = at.tn * (DUAL ? BN / 2 : BN);

  const int K = p.K, per_segment = (K + KSTEP - 1) / KSTEP, steps = per_segment * p.segments;
  const int t0 = (int)((int64_t)steps * split / splits), t1 = (int)((int64_t)steps * (split + 1) / splits);
  const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);

  Loader<M_ALONG, false, BM, WAVES> lm;
  Loader<N_ALONG, DUAL, BN, WAVES> ln;
  int next = t0, left_k = 0;         // the step to load next, and what its segment has left of K
  auto enter = [&](int seg) {
    const int k0 = (next - seg * per_segment) * KSTEP;
    left_k = K - k0;
    lm.start(p.m[seg], m0, p.M, k0, K, wave, lane);
    ln.start(DUAL ? p.n[(wave >> 1) & 1] : p.n[seg], n0, p.N, k0, K, wave, lane);
  };
  auto begin = [&](bool more) {       // the loads of step `next`
    if (next == per_segment && next < steps) enter(1);
    lm.begin(lane, left_k, more);
    ln.begin(lane, left_k, more);
    left_k -= KSTEP;
    ++next;
  };
  constexpr int LOADS_M = decltype(lm)::LOADS, LOADS = LOADS_M + decltype(ln)::LOADS, READS = MF + NF, PRODUCTS = MF * NF;
  const int base_at = (int)(uintptr_t)base;
  auto load = [&](int buffer, int j) {
    if (j < LOADS_M) lm.issue(base_at + buffer * M_BYTES, wave, j);
    else ln.issue(base_at + STAGES * M_BYTES + buffer * N_BYTES, wave, j - LOADS_M);
  };

  f32x4 acc[NF][MF] = {};
  s16x8 fm[2][MF], fn[2][NF];
  auto read = [&](int buffer, int half, int j) {
    if (j < NF) fn[half][j] = read_fragment<N_ALONG, BN>(base + STAGES * M_BYTES + buffer * N_BYTES, wn + 16 * j, half, lane);
    else fm[half][j - NF] = read_fragment<M_ALONG, BM>(base + buffer * M_BYTES, wm + 16 * (j - NF), half, lane);
  };
  // A half step: its products, and after each of the first of them one of
  // `loads` loads into `buffer`, then one read of the other half, from buffer
  // rb.  (Reads before loads: 8192 x 4096 x 11008, gradient of x 1153 us
  // instead of 1123; loads spread out over all products 1154.)
  auto half_step = [&](int half, int buffer, int loads, int rb) {
#pragma unroll
    for (int i = 0; i < NF; ++i)
#pragma unroll
      for (int j = 0; j < MF; ++j) {
        acc[i][j] = Mfma<T>::run(fn[half][i], fm[half][j], acc[i][j]);
        const int op = i * MF + j;
        if (op < loads + READS) {
          if (op < loads) load(buffer, op);
          else read(rb, half ^ 1, op - loads);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
    for (int op = PRODUCTS; op < loads + READS; ++op) {      // more of them than products
      if (op < loads) load(buffer, op);
      else read(rb, half ^ 1, op - loads);
    }
  };

  if (t0 < t1) {
    enter(t0 >= per_segment ? 1 : 0);
#pragma unroll
    for (int b = 0; b < STAGES; ++b) {
      begin(t0 + b < t1);
#pragma unroll
      for (int j = 0; j < LOADS; ++j) load(b, j);
    }
    landed_barrier<(STAGES - 1) * LOADS>();
#pragma unroll
    for (int j = 0; j < READS; ++j) read(0, 0, j);
    for (int t = t0; t < t1; t += STAGES) {
#pragma unroll
      for (int b = 0; b < STAGES; ++b) {        // unrolled: the buffers' places are constants
        if (t + b >= t1) break;
        half_step(0, 0, 0, b);
        begin(t + b + STAGES < t1);               // while the last reads and products are under way
        landed_barrier<(STAGES - 2) * LOADS>();   // the next step is in LDS, and every wave has read all of this one
        half_step(1, b, LOADS, (b + 1) % STAGES);   // after the last step: reads what an earlier one left, not used
      }
    }
  }

  // A wave's part leaves through LDS, BATCH strips of 16 rows at a time, so
  // that rows are written in runs of 16 bytes a lane.  One turn takes 64 runs;
  // what GateBackward reads is fetched AHEAD turns before its own.  (A loop:
  // unrolled it was no faster and three times the code.  GateBackward's 640 KB
  // per tile of 256 bound its epilogue: 40 us while all CUs are in it.)
  landed_barrier<0>();
  constexpr int BATCH = WAVES * 32 * STRIP <= STAGES * (M_BYTES + N_BYTES) ? 2 : 1;
  constexpr int COLS = DUAL ? BN / WN / 2 : BN / WN, OCT = COLS / 8, TURNS = 16 * OCT / 64, AHEAD = 3;
  static_assert(MF % BATCH == 0 && 16 * OCT % 64 == 0, "whole batches and turns");
  static_assert(WAVES * BATCH * 16 * STRIP <= STAGES * (M_BYTES + N_BYTES), "the epilogue fits the operands' LDS");
  float* const strip = (float*)(lds + wave * (BATCH * 16 * STRIP));
  const int row_in = lane / OCT, col = lane % OCT * 8;
  const int n = n0 + (DUAL ? wn / 2 : wn) + col;
  auto row_of = [&](int turn) { return wm + turn * (64 / OCT) + row_in; };
  auto fetch = [&](int turn) {
    const int64_t m = m0 + row_of(turn);
    return !cut && turn < MF * TURNS && m < p.M && n < p.N ? load_saved<T>(p, m, n) : Saved{};
  };
  Saved ahead[AHEAD] = {};
  if constexpr (E == Epi::GateBackward) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) ahead[k] = fetch(k);
  }
#pragma unroll
  for (int batch = 0; batch < MF; batch += BATCH) {
#pragma unroll
    for (int j = 0; j < BATCH; ++j)
#pragma unroll
      for (int i = 0; i < NF; ++i)
        *(f32x4*)(strip + (16 * j + (lane & 15)) * (STRIP / 4) + 16 * i + 4 * (lane >> 4)) = acc[i][batch + j];
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int k = 0; k < BATCH * TURNS; ++k) {
      const int turn = batch * TURNS + k;
      Saved io = {};
      if constexpr (E == Epi::GateBackward) {
        io = ahead[0];
#pragma unroll
        for (int i = 0; i + 1 < AHEAD; ++i) ahead[i] = ahead[i + 1];
        ahead[AHEAD - 1] = fetch(turn + AHEAD);
      }
      const int64_t m = m0 + row_of(turn);
      if (m >= p.M || n >= p.pad_n) continue;
      const float* from = strip + (k * (64 / OCT) + row_in) * (STRIP / 4) + (DUAL ? (col >> 4) * 32 + (col & 15) : col);
      float v[8], w[8];
      *(f32x4*)v = *(const f32x4*)from;
      *(f32x4*)(v + 4) = *(const f32x4*)(from + 4);
      if constexpr (DUAL) {
        *(f32x4*)w = *(const f32x4*)(from + 16);
        *(f32x4*)(w + 4) = *(const f32x4*)(from + 20);
      }
      if (cut) {
        float* to = g.part + ((int64_t)job * BM + row_of(turn)) * BN + (DUAL ? wn / 2 : wn) + col;
        *(f32x4*)to = *(f32x4*)v;
        *(f32x4*)(to + 4) = *(f32x4*)(v + 4);
        if constexpr (DUAL) {
          *(f32x4*)(to + BN / 2) = *(f32x4*)w;
          *(f32x4*)(to + BN / 2 + 4) = *(f32x4*)(w + 4);
        }
      } else {
        finish8<T, E>(p, m, n, v, w, io);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Joins the runs of the cut tiles in order and finishes as the product itself
// would.  A workgroup takes 2048 values' columns of one tile.
template <typename T, int BM, int BN, Epi E>
__global__ __launch_bounds__(256) void k_join(Gemm g) {
  constexpr bool DUAL = E == Epi::Gate;
  constexpr int COLS = DUAL ? BN / 2 : BN, OCT = COLS / 8, ROWS = 256 / OCT, PER_TILE = BM / ROWS;
  const int tile = blockIdx.x / PER_TILE, row = blockIdx.x % PER_TILE * ROWS + threadIdx.x / OCT, col = threadIdx.x % OCT * 8;
  const Place at = place(g, g.whole + tile);
  const Product& p = g.p[at.which];
  const int64_t m = (int64_t)at.tm * BM + row;
  const int n = at.tn * COLS + col;
  if (m >= p.M || n >= p.pad_n) return;
  f32x4 v[2] = {}, w[2] = {};
  Saved io = {};
  if constexpr (E == Epi::GateBackward) io = load_saved<T>(p, m, n);
#pragma unroll 4
  for (int s = 0; s < g.splits; ++s) {
    const float* from = g.part + (((int64_t)tile * g.splits + s) * BM + row) * BN + col;
    v[0] += *(const f32x4*)from;
    v[1] += *(const f32x4*)(from + 4);
    if constexpr (DUAL) {
      w[0] += *(const f32x4*)(from + COLS);
      w[1] += *(const f32x4*)(from + COLS + 4);
    }
  }
  finish8<T, E>(p, m, n, (float*)v, (const float*)w, io);
}

}  // namespace spardl_train
