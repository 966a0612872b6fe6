// The distillation loss from a teacher's top logits, and its gradient.
//
// One pass over a row keeps the running maximum m and the running sum s of
// exp((z - m) / t), rescaled when m grows; the loss then needs m, s and the
// logits of the row's slots only, and the gradient a second look at the row.
// The logits' bytes bound it: V elements in, and V out for the gradient.
// With few rows each row is cut into segments, whose (m, s) are joined in
// order.  4096 x 50257 bf16, loss and gradient: 167 us, 4.9 TB/s (rows of odd
// pitch 197; fp32 437, 3.8 TB/s); 8192 x 131072 916 us, 4.7 TB/s (its
// exponentials take half the time of a row, and only partly that of its
// memory); gradient alone of 1000 x 32003 fp16 27 us.  The loss alone of 300 and
// 1000 rows of 50257 bf16 takes 13.5 and 24.8 us for 4.9 and 16.2 of reading:
// scan_row has about one load a wave under way.

#include "train.hpp"

namespace spardl_train {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kTop = SPARDL_DISTILL_MAX_TOP;

struct Running {
  float m, s;   // max, and sum of exp((z - m) / t); (-inf, 0) of nothing
};

// exp((z - m) / t) for a finite m, by exp2: c = log2(e) / t.  The difference
// comes first, so logits at the type's ends overflow to exp = 0, not to NaN.
__device__ __forceinline__ float term(float z, float m, float c) { return __builtin_amdgcn_exp2f((z - m) * c); }

// The same for many z and one m: exp2 of a fused z c - m c, which misses the
// factor by the rounding of m c alone; `missed` makes up for it.  That rounding
// is in the exponent, up to |m c| 2^-24: only while it stays below 1 are both
// factors near 1, past 126 one would be 0 and the other infinite.
struct Terms {
  float c, m, mc, missed;
  bool fused;
  __device__ __forceinline__ Terms(float m_, float c_) : c(c_), m(m_), mc(m_ * c_) {
    fused = fabsf(mc) < 16777216.f;
    missed = fused ? __builtin_amdgcn_exp2f(-fmaf(m, c, -mc)) : 1.f;
  }
  __device__ __forceinline__ float near(float z) const { return __builtin_amdgcn_exp2f(fmaf(z, c, -mc)); }
};

__device__ __forceinline__ Running join(Running a, Running b, float c) {
  const float m = fmaxf(a.m, b.m);
  const float at = m == -INFINITY ? 0.f : m;   // both empty: 0 + 0 and no NaN
  return {m, a.s * term(a.m, at, c) + b.s * term(b.m, at, c)};
}

template <int THREADS>
__device__ Running group_join(Running r, float c, Running* lds) {
#pragma unroll
  for (int o = 32; o; o >>= 1) r = join(r, {__shfl_xor(r.m, o), __shfl_xor(r.s, o)}, c);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = r;
  __syncthreads();
  r = lds[0];
#pragma unroll
  for (int i = 1; i < THREADS / 64; ++i) r = join(r, lds[i], c);
  return r;
}

template <typename T, int THREADS>
__device__ Running scan_row(const T* row, int64_t first, int64_t end, float c) {
  constexpr int N = Chunk<T>::N;
  Running r{-INFINITY, 0.f};
  for (int64_t e0 = first + (int64_t)threadIdx.x * N; e0 < end; e0 += THREADS * N) {
    float z[N];
    load_chunk(row, e0, end, -INFINITY, z);
    float top = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, z[i]);
    // most chunks leave the maximum as it is
    if (top > r.m) {
      r.s *= term(r.m, top, c);
      r.m = top;
    }
    const float at = r.m == -INFINITY ? 0.f : r.m;
#pragma unroll
    for (int i = 0; i < N; ++i) r.s += term(z[i], at, c);
  }
  return r;
}

// A row's list in LDS: token (-1: empty), probability, and what the loss needs.
struct List {
  int32_t idx[kTop];
  float p[kTop];
  float z[kTop];      // the student's logit of the token
  float red[16];
};

// Fetches a row's list and the student's logits of its tokens; without a loss
// only those of tokens in [first, end) are read.
template <typename T, int THREADS>
__device__ void fetch_list(List& L, const T* row, const int32_t* idx, const float* val, int vocab, int top,
                           bool want_loss, int64_t first, int64_t end) {
  for (int k = threadIdx.x; k < top; k += THREADS) {
    const int32_t v = idx[k];
    const bool used = v >= 0 && v < vocab;
    L.idx[k] = used ? v : -1;
    L.p[k] = used ? val[k] : -INFINITY;
    L.z[k] = used && (want_loss || (v >= first && v < end)) ? (float)row[v] : 0.f;
  }
}

// The list's probabilities, and whether the row has any slot; loss: the row's
// loss, valid in every thread.  A thread works on the slots that it fetched.
// The loss is t times the sum of p (t log p - t log q): 1 / t and t^2, which
// pass the range of 32 bits long before t does, occur nowhere.
template <int THREADS>
__device__ bool settle_list(List& L, int top, float t, Running q, bool want_loss, float* loss) {
  const float c = kLog2e / t;
  float m = -INFINITY;
  for (int k = threadIdx.x; k < top; k += THREADS) m = fmaxf(m, L.p[k]);    // a NaN shows in the sum below
  m = wave_max(m);
  if constexpr (THREADS > 64) {
    if ((threadIdx.x & 63) == 0) L.red[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) m = fmaxf(m, L.red[i]);
    __syncthreads();
  }
  bool any = m > -INFINITY;
  float total = 0.f;
  for (int k = threadIdx.x; k < top; k += THREADS) {
    const float u = L.p[k];
    total += u == -INFINITY ? 0.f : term(u, m, c);
  }
  total = group_sum<THREADS>(total, L.red);
  any = any || total != total;
  __syncthreads();
  const float inv = 1.f / total, logs = t * (logf(q.s) - logf(total));
  float sum = 0.f;
  for (int k = threadIdx.x; k < top; k += THREADS) {
    const float u = L.p[k];
    const float p = u == -INFINITY ? 0.f : term(u, m, c) * inv;
    L.p[k] = p;
    if (want_loss && !(p <= 0.f)) sum += p * (((u - m) - (L.z[k] - q.m)) + logs);
  }
  if (want_loss) *loss = any ? t * group_sum<THREADS>(sum, L.red) : 0.f;
  __syncthreads();
  return any;
}

// The list's tokens in [first, end), each from all of its slots, over what a
// first write put there; a barrier lies between the two.  A token may stand in
// several slots, so a slot looks at all of them: top^2 reads of LDS a row.  Step
// of 4096 x 50257 bf16, odd pitch: 197 us with 64 slots, 266 with 256, 1005 with
// 1024.
template <typename T, int THREADS>
__device__ void write_list(const List& L, T* out, int64_t first, int64_t end, int top, float c, Running q, float scale) {
  for (int k = threadIdx.x; k < top; k += THREADS) {
    const int32_t v = L.idx[k];
    if (v < first || v >= end) continue;
    float p = 0.f;
    for (int j = 0; j < top; ++j) p += L.idx[j] == v ? L.p[j] : 0.f;
    out[v] = (T)(scale * (term(L.z[k], q.m, c) / q.s - p));
  }
}

// dlogits[first .. end) of a row: scale (q - p).
template <typename T, int THREADS>
__device__ void write_gradient(const List& L, const T* row, T* out, int64_t first, int64_t end, int top, float t,
                               Running q, bool any, float dloss) {
  constexpr int N = Chunk<T>::N;
  const float c = kLog2e / t, scale = dloss * t;
  const Terms e(q.m, c);
  const float each = scale / q.s * e.missed;
  for (int64_t e0 = first + (int64_t)threadIdx.x * N; e0 < end; e0 += THREADS * N) {
    float z[N] = {};
    if (any) {
      load_chunk(row, e0, end, -INFINITY, z);
      if (e.fused) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = each * e.near(z[i]);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = each * term(z[i], q.m, c);
      }
    }
    store_chunk<T, true>(out, e0, end, z);
  }
  __syncthreads();
  if (any) write_list<T, THREADS>(L, out, first, end, top, c, q, scale);
}

// A row of no finite logit has no q.
__device__ __forceinline__ Running settled(Running r) {
  if (r.m == -INFINITY) r.s = NAN;
  return r;
}

// One workgroup per row: loss and stats, and the gradient where d.dlogits is set.
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void k_distill_row(Distill d) {
  __shared__ List L;
  __shared__ Running red[THREADS / 64];
  const int64_t r = blockIdx.x;
  const T* row = (const T*)d.logits + r * d.ld;
  const float c = kLog2e / d.temperature;
  fetch_list<T, THREADS>(L, row, d.top_idx + r * d.ld_top, d.top_val + r * d.ld_top, d.vocab, d.top, true, 0, d.vocab);
  const Running q = settled(group_join<THREADS>(scan_row<T, THREADS>(row, 0, d.vocab, c), c, red));
  float loss;
  const bool any = settle_list<THREADS>(L, d.top, d.temperature, q, true, &loss);
  if (threadIdx.x == 0) {
    d.loss[r] = loss;
    d.stats[2 * r] = q.m;
    d.stats[2 * r + 1] = q.s;
  }
  if (d.dlogits)
    write_gradient<T, THREADS>(L, row, (T*)d.dlogits + r * d.ld_d, 0, d.vocab, d.top, d.temperature, q, any,
                               d.dloss[r]);
}

// The same for a row of at most THREADS x NCH chunks, which stays in the
// registers of its workgroup between the two looks at it.  (1024 x 16 in fp16 and
// fp32 spills 12 registers a lane: 4096 x 131072 fp16 500 us, bf16 465.)  Chunks
// past the row's end cost their exponentials too: 4096 x 64000 bf16 326 us.
template <typename T, int THREADS, int NCH, int PER_CU>
__global__ __launch_bounds__(THREADS, PER_CU * THREADS / 256) void k_distill_held(Distill d) {
  constexpr int N = Chunk<T>::N;
  typedef typename Chunk<T>::Vec Vec;
  __shared__ List L;
  __shared__ Running red[THREADS / 64];
  const int64_t r = blockIdx.x;
  const T* row = (const T*)d.logits + r * d.ld;
  const float c = kLog2e / d.temperature;
  Vec held[NCH];
#pragma unroll
  for (int k = 0; k < NCH; ++k) {
    const int e0 = (k * THREADS + threadIdx.x) * N;
    if (e0 + N <= d.vocab) {
      // one place a thread, one scalar base a chunk
      __builtin_memcpy(&held[k], (const char*)(row + k * THREADS * N) + threadIdx.x * 16u, 16);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) held[k][i] = (T)-INFINITY;
      if (e0 < d.vocab)
#pragma unroll
        for (int i = 0; i < N - 1; ++i)
          if (e0 + i < d.vocab) held[k][i] = row[e0 + i];
    }
  }
  fetch_list<T, THREADS>(L, row, d.top_idx + r * d.ld_top, d.top_val + r * d.ld_top, d.vocab, d.top, true, 0, d.vocab);
  Running q{-INFINITY, 0.f};
#pragma unroll
  for (int k = 0; k < NCH; ++k)
#pragma unroll
    for (int i = 0; i < N; ++i) q.m = fmaxf(q.m, (float)held[k][i]);
  const float at = q.m == -INFINITY ? 0.f : q.m;
  // Three looks at the packed row: the compiler is not to keep the unpacked
  // one, which takes twice the registers, from one to the next.
  auto repack = [&]() {
#pragma unroll
    for (int k = 0; k < NCH; ++k) asm volatile("" : "+v"(held[k]));
  };
  repack();
  const Terms own(at, c);
  if (own.fused) {
    float s[2] = {};
#pragma unroll
    for (int k = 0; k < NCH; ++k)
#pragma unroll
      for (int i = 0; i < N; ++i) s[i & 1] += own.near((float)held[k][i]);
    q.s = (s[0] + s[1]) * own.missed;
  } else {
#pragma unroll
    for (int k = 0; k < NCH; ++k)
#pragma unroll
      for (int i = 0; i < N; ++i) q.s += term((float)held[k][i], at, c);
  }
  q = settled(group_join<THREADS>(q, c, red));
  float loss;
  const bool any = settle_list<THREADS>(L, d.top, d.temperature, q, true, &loss);
  if (threadIdx.x == 0) {
    d.loss[r] = loss;
    d.stats[2 * r] = q.m;
    d.stats[2 * r + 1] = q.s;
  }
  const float scale = d.dloss[r] * d.temperature;
  const Terms e(q.m, c);
  const float each = scale / q.s * e.missed;
  T* out = (T*)d.dlogits + r * d.ld_d;
  repack();
#pragma unroll
  for (int k = 0; k < NCH; ++k) {
    const int e0 = (k * THREADS + threadIdx.x) * N;
    if (e0 >= d.vocab) continue;
    float z[N];
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = 0.f;
    if (any && e.fused) {
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = each * e.near((float)held[k][i]);
    } else if (any) {
#pragma unroll
      for (int i = 0; i < N; ++i) z[i] = each * term((float)held[k][i], q.m, c);
    }
    if (e0 + N <= d.vocab) {
      Vec v;
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = (T)z[i];
      __builtin_nontemporal_store(v, (typename Chunk<T>::Loose*)((char*)(out + k * THREADS * N) + threadIdx.x * 16u));
    } else {
      store_chunk(out, e0, d.vocab, z);
    }
  }
  __syncthreads();
  if (any) write_list<T, THREADS>(L, out, 0, d.vocab, d.top, c, q, scale);
}

// (m, s) of each segment of a row.
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void k_distill_segment(Distill d, int segs, int64_t seg, Running* part) {
  __shared__ Running red[THREADS / 64];
  const int64_t r = blockIdx.x / segs, k = blockIdx.x % segs;
  const int64_t first = k * seg, end = min(first + seg, (int64_t)d.vocab);
  const float c = kLog2e / d.temperature;
  const Running q =
      group_join<THREADS>(scan_row<T, THREADS>((const T*)d.logits + r * d.ld, first, end, c), c, red);
  if (threadIdx.x == 0) part[blockIdx.x] = q;
}

// A segment of a row's gradient; with part also the loss and stats, by the
// row's first segment.  One segment and no gradient: the loss alone.
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void k_distill_finish(Distill d, int segs, int64_t seg, int parts,
                                                            const Running* part) {
  __shared__ List L;
  const int64_t r = blockIdx.x / segs, k = blockIdx.x % segs;
  const T* row = (const T*)d.logits + r * d.ld;
  const float c = kLog2e / d.temperature;
  const int64_t first = k * seg, end = min(first + seg, (int64_t)d.vocab);
  fetch_list<T, THREADS>(L, row, d.top_idx + r * d.ld_top, d.top_val + r * d.ld_top, d.vocab, d.top, part != nullptr,
                         first, end);
  Running q{-INFINITY, 0.f};
  if (part) {
    for (int i = 0; i < parts; ++i) q = join(q, part[r * parts + i], c);
    q = settled(q);
  } else {
    q = {d.stats[2 * r], d.stats[2 * r + 1]};
  }
  float loss;
  const bool any = settle_list<THREADS>(L, d.top, d.temperature, q, part != nullptr, &loss);
  if (part && k == 0 && threadIdx.x == 0) {
    d.loss[r] = loss;
    d.stats[2 * r] = q.m;
    d.stats[2 * r + 1] = q.s;
  }
  if (d.dlogits)
    write_gradient<T, THREADS>(L, row, (T*)d.dlogits + r * d.ld_d, first, end, d.top,
                                d.temperature, q, any, d.dloss[r]);
}

// Segments of a row: enough workgroups to fill the card, none below 2048
// logits.  1000 x 50257 bf16, backward: 38.9 us with two segments a row, 38.4
// with one; 300 rows 15.7 and 21.2, 64 rows 8.5 and 15.8.
constexpr int64_t kFill = 1024, kSegMin = 2048;
int64_t segments(int64_t rows, int32_t vocab) {
  const int64_t want = ceil_div(kFill, rows < 1 ? 1 : rows), most = ceil_div(vocab, kSegMin);
  return want < most ? want : most;
}

// Whether the loss takes one workgroup per row, in one launch, rather than
// segments in two.  bf16, us in one and in two: with the gradient, where a row
// fits a workgroup's registers, 64 rows of 8000 8.0 and 10.7, of 50257 13.7 and
// 14.2, of 131072 20.6 and 16.5; 128 rows 8.0 and 11.4, 14.4 and 16.3, 23.6 and
// 25.4; 1000 rows 11.4 and 17.6, 41 and 59, 123 and 149.  The loss alone, 64
// rows of 8000 7.1 and 10.2, 1000 rows 8.0 and 11.7, but 300 rows of 50257 16
// and 13, 1000 rows 31 and 24.
bool one_launch(const Distill& d, int64_t chunks) {
  if (d.rows >= 2 * kFill) return true;
  if (d.dlogits) return chunks <= 1024 * 16 && d.rows >= (chunks <= 512 * 13 ? 64 : 128);
  return d.rows >= 64 && d.vocab <= 16384;
}

template <typename T>
hipError_t launch(const Distill& d, void* ws, hipStream_t s) {
  const int64_t segs = segments(d.rows, d.vocab);
  constexpr int64_t N = Chunk<T>::N;
  const int64_t seg = ceil_div(ceil_div(d.vocab, segs), N) * N;
  const int64_t used = ceil_div(d.vocab, seg), chunks = ceil_div(d.vocab, N);
  Running* part = (Running*)ws;
  if (d.loss && (used == 1 || one_launch(d, chunks))) {
    const dim3 grid((uint32_t)d.rows);
    // threads and chunks a thread that hold a row, as few as do
    if (d.dlogits && chunks <= 256 * 4) k_distill_held<T, 256, 4, 4><<<grid, 256, 0, s>>>(d);
    else if (d.dlogits && chunks <= 512 * 4) k_distill_held<T, 512, 4, 3><<<grid, 512, 0, s>>>(d);
    else if (d.dlogits && chunks <= 512 * 8) k_distill_held<T, 512, 8, 3><<<grid, 512, 0, s>>>(d);
    else if (d.dlogits && chunks <= 512 * 13) k_distill_held<T, 512, 13, 2><<<grid, 512, 0, s>>>(d);
    else if (d.dlogits && chunks <= 1024 * 16) k_distill_held<T, 1024, 16, 1><<<grid, 1024, 0, s>>>(d);
    else if (d.vocab > 8192) k_distill_row<T, 1024><<<grid, 1024, 0, s>>>(d);
    else k_distill_row<T, 256><<<grid, 256, 0, s>>>(d);
    return launched();
  }
  if (d.loss) {
    k_distill_segment<T, 256><<<dim3((uint32_t)(d.rows * used)), 256, 0, s>>>(d, (int)used, seg, part);
    // Where the gradient replaces the logits, the loss is taken before any segment of them is gone.
    const bool apart = !d.dlogits || d.dlogits == d.logits;
    Distill f = d;
    if (apart) f.dlogits = nullptr;
    const int64_t out = apart ? 1 : used;
    k_distill_finish<T, 256><<<dim3((uint32_t)(d.rows * out)), 256, 0, s>>>(f, (int)out, apart ? d.vocab : seg,
                                                                            (int)used, part);
    if (!apart || !d.dlogits) return launched();
  }
  k_distill_finish<T, 256><<<dim3((uint32_t)(d.rows * used)), 256, 0, s>>>(d, (int)used, seg, 0, nullptr);
  return launched();
}

}  // namespace

size_t distill_ws(int64_t rows, int32_t vocab) {
  // For any number of rows up to these: r rows take r segments(r) parts, at most r + kFill - 1 of them and
  // at most as many as rows of segments of kSegMin have.
  const int64_t most = (rows < 1 ? 1 : rows) * ceil_div(vocab, kSegMin), parts = rows + kFill - 1;
  return align256((size_t)(parts < most ? parts : most) * sizeof(Running));
}

hipError_t launch_distill(const Distill& d, void* ws, hipStream_t s) {
  const int64_t size = d.dtype == SPARDL_FP32 ? 4 : 2;
  for (int64_t r = 0; r < d.rows; r += kRowsPerLaunch) {
    Distill part = d;
    part.rows = d.rows - r < kRowsPerLaunch ? d.rows - r : kRowsPerLaunch;
    part.logits = (const char*)d.logits + r * d.ld * size;
    part.top_idx = d.top_idx + r * d.ld_top;
    part.top_val = d.top_val + r * d.ld_top;
    part.loss = d.loss ? d.loss + r : nullptr;
    part.stats = d.stats + 2 * r;
    part.dloss = d.dloss ? d.dloss + r : nullptr;
    part.dlogits = d.dlogits ? (char*)d.dlogits + r * d.ld_d * size : nullptr;
    const hipError_t e = d.dtype == SPARDL_BF16   ? launch<bf16>(part, ws, s)
                         : d.dtype == SPARDL_FP16 ? launch<fp16>(part, ws, s)
                                                  : launch<float>(part, ws, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace spardl_train
