// The gated feed-forward block on bf16, and its workspace.

#include "train_ffn.hpp"

namespace spardl_train {

size_t gated_ffn_ws(int64_t tokens, int32_t dim, int32_t hidden, bool backward, bool unaligned) {
  const int64_t T = tokens, Dp = round8(dim), Fp = round8(hidden);
  size_t b = (backward ? 3 : 1) * align256((size_t)T * Fp * 2);
  // A few tokens' forward pass takes rows as they are and cuts no tiles.  A view has its room all the same, so
  // that whether one is taken does not depend on the number of tokens.
  const bool few = !backward && T <= kFewTokens;
  if (unaligned || (!few && (dim % 8 || hidden % 8))) {
    b += (backward ? 2 : 1) * align256((size_t)T * Dp * 2);
    b += 2 * align256((size_t)hidden * Dp * 2) + align256((size_t)dim * Fp * 2);
  }
  if (few) return b + 256;
  // the products' partial sums, one product at a time
  Gemm g = {};
  auto one = [&](int64_t M, int32_t N, int64_t K, int32_t segments) {
    g.products = 1;
    g.p[0] = product({}, {}, M, N, K);
    g.p[0].segments = segments;
  };
  int64_t most = 0;
  auto see = [&](int64_t floats) { most = most > floats ? most : floats; };
  if (!backward) {
    one(T, hidden, dim, 1);
    g.p[0].pad_n = (int32_t)Fp;
    see(most_partials<Epi::Gate>(g));
    one(T, dim, hidden, 1);
    see(most_partials<Epi::Store>(g));
  } else {
    one(T, hidden, dim, 1);
    g.p[0].pad_n = (int32_t)Fp;
    see(most_partials<Epi::GateBackward>(g));
    one(T, dim, hidden, 2);
    see(most_partials<Epi::Store>(g));
    if (T > kOuterTokens) {
      g.products = 3;
      g.p[0] = g.p[1] = product({}, {}, hidden, dim, T);
      g.p[2] = product({}, {}, dim, hidden, T);
      see(most_partials<Epi::Store>(g));
    }
  }
  return b + align256((size_t)most * 4) + 256;
}

hipError_t ffn_forward_bf16(const Ffn& f, void* ws, hipStream_t s) { return ffn_forward<bf16>(f, ws, s); }
hipError_t ffn_backward_bf16(const Ffn& f, void* ws, hipStream_t s) { return ffn_backward<bf16>(f, ws, s); }

}  // namespace spardl_train
