// Host side of the gated feed-forward block for one element type: operands,
// workspace and launches.
#pragma once

#include "train_few.hpp"
#include "train_gemm.hpp"

namespace spardl_train {

inline int64_t round8(int64_t x) { return (x + 7) & ~(int64_t)7; }

// Copies of a call's operands whose rows do not take 16-byte accesses: rows of
// `cols` elements to rows of round8(cols), zero past cols, all in one launch.
struct PackJob {
  const void* src;
  void* dst;
  int64_t ld_src, rows;
  int32_t cols;
};
constexpr int kPackJobs = 5;
struct PackJobs {
  PackJob job[kPackJobs];
  int32_t count;
};
template <typename T>
__global__ __launch_bounds__(256) void k_pack(PackJobs p) {
  const PackJob& j = p.job[blockIdx.y];
  const int chunks = (j.cols + 7) / 8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < j.rows * chunks; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / chunks;
    const int e0 = (int)(i % chunks) * 8;
    ((i32x4*)j.dst)[i] = load_packed((const T*)j.src + r * j.ld_src, e0, j.cols);
  }
}

// Workspace of one call, carved front to back.
struct Carver {
  char* base;
  size_t used = 0;
  void* take(size_t bytes) {
    void* p = base + used;
    used += align256(bytes);
    return p;
  }
};

// Operands as the products take them: themselves where their rows are 16-byte
// aligned and a multiple of 8 long, else copies, which run() makes.
template <typename T>
struct Operands {
  Carver& ws;
  PackJobs jobs = {};
  Side operator()(const void* p, int64_t ld, int64_t rows, int32_t cols) {
    if (cols % 8 == 0 && rows_aligned(p, ld)) return {p, ld};
    void* to = ws.take((size_t)rows * round8(cols) * 2);
    if (rows > 0) jobs.job[jobs.count++] = {p, to, ld, rows, cols};
    return {to, round8(cols)};
  }
  void run(hipStream_t s) const {
    if (jobs.count == 0) return;
    int64_t most = 0;
    for (int i = 0; i < jobs.count; ++i) {
      const int64_t chunks = jobs.job[i].rows * ((jobs.job[i].cols + 7) / 8);
      most = most > chunks ? most : chunks;
    }
    const int64_t blocks = ceil_div(most, 256);
    k_pack<T><<<dim3((uint32_t)(blocks < 4096 ? blocks : 4096), (uint32_t)jobs.count), 256, 0, s>>>(jobs);
  }
};

// Tiles of a launch (256 or 128 square), and how many runs of K the tiles that
// do not fill a round of the card are cut into.
struct Plan {
  int tile, whole, splits;
  int64_t floats;      // of partial sums; 0: none
};

inline int64_t round_of(int tile) { return tile == 256 ? 256 : 512; }      // tiles that the card holds at once
template <Epi E>
int columns(int tile) { return E == Epi::Gate ? tile / 2 : tile; }         // of the product, in a tile

// A launch's tiles, the K steps of its longest product and the values of its results.
struct Extent {
  int64_t tiles, steps, values;
};
template <Epi E>
Extent extent(const Gemm& g, int tile) {
  Extent x = {};
  for (int i = 0; i < g.products; ++i) {
    const Product& p = g.p[i];
    x.tiles += ceil_div(p.M, tile) * ceil_div(p.pad_n, columns<E>(tile));
    x.values += (int64_t)p.M * p.pad_n * (E == Epi::Gate ? 2 : 1);
    const int64_t s = ceil_div(p.K, KSTEP) * p.segments;
    x.steps = x.steps > s ? x.steps : s;
  }
  return x;
}

// The plan of least estimated time, in us, from what was measured on products
// of 64 .. 8192 x 1600 .. 11008: a step of a tile of 256 (one workgroup a CU)
// takes 1.65, of tiles of 128 1.0 with two on a CU and alone 0.5 if both
// operands lie along K (25 steps of 128 x 1600 x 6400) and 0.6 if not (200
// steps of 2048 x 1600, the weights across K: 122); a round's start and
// epilogue 6 and 4, and 25 and 9 more where the epilogue reads and writes five
// matrices; joining cut tiles 5 and their bytes, read and written at 5e6 a us.
template <Epi E, bool ALONG>
Plan plan(Gemm& g) {
  Plan best = {0, 0, 1, 0};
  double least = 0;
  for (int tile = 128; tile <= 256; tile += 128) {
    const auto [tiles, steps, values] = extent<E>(g, tile);
    const int64_t slots = round_of(tile), full = tiles / slots, rest = tiles % slots;
    const bool big = tile == 256;
    const double step = big ? 1.65 : 1.0;
    const double ends = (big ? 6.0 : 4.0) + (E == Epi::GateBackward ? big ? 25.0 : 9.0 : 0.0);
    for (int splits = 1; splits == 1 || (rest * splits <= slots && steps >= 4 * splits); ++splits) {
      const double last = !big && rest * splits <= 256 && !full ? ALONG ? 0.5 : 0.6 : step;
      double us = (double)full * ((double)steps * step + ends);
      if (rest) us += (double)ceil_div(steps, splits) * last + (splits > 1 && E == Epi::GateBackward ? 6.0 : ends);
      if (splits > 1) us += 5.0 + 8.0 * (double)(rest * splits) / (double)tiles * (double)values / 5e6;
      if (best.tile == 0 || us < least) {
        least = us;
        best = {tile, (int)(splits > 1 ? full * slots : tiles), splits, splits > 1 ? rest * splits * tile * tile : 0};
      }
      if (!rest) break;
    }
  }
  g.tiles = 0;
  g.whole = best.whole;
  g.splits = best.splits;
  for (int i = 0; i < g.products; ++i) {
    Product& p = g.p[i];
    p.tiles_m = (int32_t)ceil_div(p.M, best.tile);
    p.tiles_n = (int32_t)ceil_div(p.pad_n, columns<E>(best.tile));
    p.first = g.tiles;
    g.tiles += p.tiles_m * p.tiles_n;
  }
  return best;
}

// Floats of partial sums that no plan passes, for these products or smaller
// ones: all runs of the cut tiles fit a round of the card, and a run is four
// steps at least.  A plan's own need falls where one more tile ends a round, so
// a workspace sized by it would not serve a shorter batch.
template <Epi E>
int64_t most_partials(const Gemm& g) {
  int64_t most = 0;
  for (int tile = 128; tile <= 256; tile += 128) {
    const Extent x = extent<E>(g, tile);
    const int64_t splits = x.steps / 4, runs = x.tiles * splits < round_of(tile) ? x.tiles * splits : round_of(tile);
    const int64_t floats = splits > 1 ? runs * tile * tile : 0;
    most = most > floats ? most : floats;
  }
  return most;
}

template <typename T, bool M_ALONG, bool N_ALONG, Epi E>
hipError_t launch_product(Gemm& g, Carver ws, hipStream_t s) {
  const Plan b = plan<E, M_ALONG && N_ALONG>(g);
  if (g.tiles == 0) return hipSuccess;
  g.part = b.floats ? (float*)ws.take((size_t)b.floats * 4) : nullptr;
  const int cut = g.tiles - g.whole;
  const dim3 grid((uint32_t)(g.whole + cut * g.splits));
  if (b.tile == 256) {
    k_gemm<T, 256, 256, 2, 4, 1, 2, M_ALONG, N_ALONG, E><<<grid, 512, 0, s>>>(g);
    if (cut) k_join<T, 256, 256, E><<<dim3((uint32_t)(cut * (E == Epi::Gate ? 16 : 32))), 256, 0, s>>>(g);
  } else {
    // Alone on its CU a tile takes twice the waves and buffers (128 x 1600 x 6400: 20.9 -> 17.8 us); two on a CU
    // have each other, and more waves read more of LDS (416 tiles of 25 steps: 51 us, on eight waves each 59).
    if (grid.x <= 256) k_gemm<T, 128, 128, 4, 2, 1, 4, M_ALONG, N_ALONG, E><<<grid, 512, 0, s>>>(g);
    else k_gemm<T, 128, 128, 2, 2, 2, 2, M_ALONG, N_ALONG, E><<<grid, 256, 0, s>>>(g);
    if (cut) k_join<T, 128, 128, E><<<dim3((uint32_t)(cut * (E == Epi::Gate ? 4 : 8))), 256, 0, s>>>(g);
  }
  return launched();
}

inline Product product(Side m, Side n, int64_t M, int32_t N, int64_t K) {
  Product p = {};
  p.m[0] = m;
  p.n[0] = n;
  p.M = (int32_t)M;
  p.N = N;
  p.K = (int32_t)K;
  p.segments = 1;
  p.pad_n = N;
  return p;
}

template <typename T>
hipError_t ffn_forward(const Ffn& f, void* ws, hipStream_t s) {
  if (f.tokens == 0) return hipSuccess;
  Carver c{(char*)ws};
  const int64_t Fp = round8(f.hidden);
  void* h = c.take((size_t)f.tokens * Fp * 2);
  const bool few = f.tokens <= kFewTokens;     // rows as they are: no copies
  Operands<T> operands{c};
  auto side = [&](const void* p, int64_t ld, int64_t rows, int32_t cols) {
    return few ? Side{p, ld} : operands(p, ld, rows, cols);
  };
  const Side x = side(f.x, f.ld_x, f.tokens, f.dim), wg = side(f.w_gate, f.ld_gate, f.hidden, f.dim);
  const Side wu = side(f.w_up, f.ld_up, f.hidden, f.dim), wd = side(f.w_down, f.ld_down, f.dim, f.hidden);
  operands.run(s);

  Gemm g = {};
  g.products = 1;
  Product& a = g.p[0] = product(x, wg, f.tokens, f.hidden, f.dim);
  a.n[1] = wu;
  a.out = h;
  a.ld_out = a.pad_n = (int32_t)Fp;
  a.out2 = f.gate;
  a.out3 = f.up;
  a.ld_io = f.ld_hidden;
  a.act = f.act;
  hipError_t e = few ? launch_few<T, Epi::Gate>(a, s) : launch_product<T, true, true, Epi::Gate>(g, c, s);
  if (e != hipSuccess) return e;

  g.p[0] = product({h, Fp}, wd, f.tokens, f.dim, f.hidden);
  g.p[0].out = f.y;
  g.p[0].ld_out = f.ld_y;
  return few ? launch_few<T, Epi::Store>(g.p[0], s) : launch_product<T, true, true, Epi::Store>(g, c, s);
}

template <typename T>
hipError_t ffn_backward(const Ffn& f, void* ws, hipStream_t s) {
  Carver c{(char*)ws};
  const int64_t Fp = round8(f.hidden);
  void* dg = c.take((size_t)f.tokens * Fp * 2);
  void* du = c.take((size_t)f.tokens * Fp * 2);
  void* h = c.take((size_t)f.tokens * Fp * 2);
  Operands<T> operands{c};
  const Side dy = operands(f.dy, f.ld_dy, f.tokens, f.dim), x = operands(f.x, f.ld_x, f.tokens, f.dim);
  const Side wd = operands(f.w_down, f.ld_down, f.dim, f.hidden);
  Side wg = {}, wu = {};
  if (f.dx) {
    wg = operands(f.w_gate, f.ld_gate, f.hidden, f.dim);
    wu = operands(f.w_up, f.ld_up, f.hidden, f.dim);
  }
  operands.run(s);

  Gemm g = {};
  hipError_t e;
  g.products = 1;
  Product& a = g.p[0] = product(dy, wd, f.tokens, f.hidden, f.dim);
  a.out = dg;
  a.out2 = du;
  a.out3 = h;
  a.ld_out = a.pad_n = (int32_t)Fp;
  a.in = f.gate;
  a.in2 = f.up;
  a.ld_io = f.ld_hidden;
  a.act = f.act;
  e = launch_product<T, true, false, Epi::GateBackward>(g, c, s);
  if (e != hipSuccess) return e;

  if (f.dx) {
    g.p[0] = product({dg, Fp}, wg, f.tokens, f.dim, f.hidden);
    g.p[0].segments = 2;
    g.p[0].m[1] = {du, Fp};
    g.p[0].n[1] = wu;
    g.p[0].out = f.dx;
    g.p[0].ld_out = f.ld_dx;
    e = launch_product<T, true, false, Epi::Store>(g, c, s);
    if (e != hipSuccess) return e;
  }

  g.products = 3;
  g.p[0] = product({dg, Fp}, x, f.hidden, f.dim, f.tokens);
  g.p[1] = product({du, Fp}, x, f.hidden, f.dim, f.tokens);
  g.p[2] = product(dy, {h, Fp}, f.dim, f.hidden, f.tokens);
  void* const out[3] = {f.dw_gate, f.dw_up, f.dw_down};
  const int64_t ld[3] = {f.ld_dgate, f.ld_dup, f.ld_ddown};
  const bool f32 = f.dw_dtype == SPARDL_FP32;
  for (int i = 0; i < 3; ++i) {
    g.p[i].out = out[i];
    g.p[i].ld_out = ld[i];
    g.p[i].out_f32 = f32;
    g.p[i].accumulate = f.accumulate;
  }
  if (f.tokens <= kOuterTokens) return launch_outer<T>(g, s);
  return launch_product<T, false, false, Epi::Store>(g, c, s);
}

}  // namespace spardl_train
