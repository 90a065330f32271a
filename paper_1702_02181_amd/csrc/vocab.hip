// Products of the vocabulary head on the matrix cores (gfx950):
//     logits   z = s W^T + b      s [M, H] states, W [V, H]: both operands run along K = H
//     states   ds = dz W          K = V: dz runs along K, W across it
//     weights  dW (+)= dz^T s     K = M: both operands run across K
//     bias     db (+)= sum_m dz
// The loop and its tiles are product.h's.

#include <hip/hip_runtime.h>

#include "product.h"

namespace fold {

namespace {

// Whether the two gradients of the backward share a launch, in the smallest tiles: batches of one tile row, and of two
// unless W is so large that reading it twice costs more than a launch (all three gradients, bf16: 33 x 300 x 20,000 26.6
// us in four launches, 19.0 in two; 100 x 1,024 x 32,000 48 us together, 26 + 37 apart; 100 x 2,048 x 40,000 136 apart;
// 100 x 4,096 x 32,000 276 and 212; in fp32, where the matrix cores bound it, 100 x 4,096 x 32,000 589 and 659).
bool together(int64_t M, int H, int V, int esize) {
  return M <= 64 || (M <= 128 && (esize == 4 || (int64_t)V * row_ld(H) <= (int64_t)1 << 25));
}
Shape logits_shape(int64_t M, int H, int V, int esize) {
  return shape_of(M, row_ld(V), row_ld(H) * esize / 128, esize, 2, 1);
}
Shape states_shape(int64_t M, int H, int V, int esize) {
  return shape_of(std::max<int64_t>(M, 1), row_ld(H), (int64_t)row_ld(V) * esize / 128, esize, 1, kPieces,
                  together(M, H, V, esize));
}

// both: in one launch with the states' gradient
Shape weights_shape(int64_t M, int H, int V, int esize, bool both) {
  const int lines = 128 / esize;
  return shape_of(V, row_ld(H), (M + lines - 1) / lines, esize, 1, 1, both);
}

}  // namespace

// Workgroups of the largest launch that a call makes: at most vocab_tiles (cheap, whatever the shapes), or counted.
int64_t vocab_tiles(int64_t M, int H, int V) {
  const int64_t h = tiles_of(row_ld(H), 1), v = tiles_of(row_ld(V), 1), m = std::max<int64_t>(tiles_of(M, 1), 1);
  return std::max(m * ((v + 1) / 2), std::max(v * h, m * h * kPieces));
}
int64_t vocab_logits_tiles(int dtype, int64_t M, int H, int V) {
  const Shape sh = logits_shape(M, H, V, dtype == FOLD_BF16 ? 2 : 4);
  return sh.mt * sh.nt;
}
int64_t vocab_backward_tiles(int dtype, int64_t M, int H, int V) {
  const int es = dtype == FOLD_BF16 ? 2 : 4;
  const Shape s1 = states_shape(M, H, V, es);
  const int64_t ds = s1.mt * s1.nt * s1.split;
  int64_t most = s1.split > 1 ? std::max(ds, (int64_t)join_blocks(s1.split, (size_t)M * row_ld(H))) : ds;
  const Shape s2 = weights_shape(M, H, V, es, false);
  most = std::max(most, s2.mt * s2.nt);
  if (together(M, H, V, es)) {
    const Shape s3 = weights_shape(M, H, V, es, true);
    most = std::max(most, ds + s3.mt * s3.nt);
  }
  return most;  // the bias sums' launches are smaller: at most 2^13 groups of columns
}

void launch_vocab_logits(int dtype, int64_t M, int H, int V, const void* s, const void* W, const float* bias,
                         int out_dtype, void* z, hipStream_t st) {
  if (M <= 0) return;
  ProfScope prof("vocab_logits", st);
  const int es = dtype == FOLD_BF16 ? 2 : 4, ldh = row_ld(H), ldv = row_ld(V);
  const Shape sh = logits_shape(M, H, V, es);
  const ProductArgs g{{s, M, ldh}, {W, V, ldh}, M, V, sh.mt, sh.nt, ldh * es / 128, 1, z, (size_t)ldv, ldv, bias, 0,
                      nullptr};
  if (dtype == FOLD_F32) launch<float, kAlong, kAlong, float>(g, sh, st);
  else if (out_dtype == FOLD_F32) launch<uint16_t, kAlong, kAlong, float>(g, sh, st);
  else launch<uint16_t, kAlong, kAlong, uint16_t>(g, sh, st);
}

size_t vocab_backward_bytes(int dtype, int64_t M, int H, int V) {
  const int es = dtype == FOLD_BF16 ? 2 : 4;
  const int n = states_shape(M, H, V, es).split, c = bias_chunks(M, V, es);
  // the two follow each other on the stream: one region serves both
  return std::max(n == 1 ? 0 : (size_t)n * M * row_ld(H), c == 1 ? 0 : (size_t)c * row_ld(V)) * sizeof(float);
}

void launch_vocab_backward(int dtype, int64_t M, int H, int V, const void* s, const void* W, const void* dz, float* ds,
                           float* dW, float* db, int add, void* ws, hipStream_t st) {
  const int es = dtype == FOLD_BF16 ? 2 : 4, ldh = row_ld(H), ldv = row_ld(V);
  const int kst = 128 / es;
  const int64_t stages = (M + kst - 1) / kst;
  const Shape s1 = states_shape(M, H, V, es);
  const bool both = ds && dW && M > 0 && together(M, H, V, es);
  const Shape s2 = weights_shape(M, H, V, es, both);
  // a few rows' sums come from the weights' product, whose tiles of the first column hold all of dz: where every stage is
  // loaded before its loop (two of 128 bytes, or three of 64, of which a whole one is two)
  float* sums = dW && stages <= (s2.wm == 4 ? 1 : 2) ? db : nullptr;
  ProductArgs states{{dz, M, ldv}, {W, V, ldh}, M, H, s1.mt, s1.nt, ldv * es / 128, s1.split,
                     s1.split > 1 ? ws : ds, (size_t)ldh, ldh, nullptr, 0, nullptr};
  ProductArgs weights{{dz, M, ldv}, {s, M, ldh}, V, H, s2.mt, s2.nt, (int)stages, 1, dW, (size_t)ldh, ldh, nullptr, add,
                      sums};
  if (both) {
    ProfScope prof("vocab_backward", st);
    const unsigned n1 = blocks_of(states), n2 = blocks_of(weights);
    if (dtype == FOLD_F32)
      hipLaunchKernelGGL(k_product_both<float>, dim3(n1 + n2), dim3(kThreads), 0, st, states, weights, n1);
    else
      hipLaunchKernelGGL(k_product_both<uint16_t>, dim3(n1 + n2), dim3(kThreads), 0, st, states, weights, n1);
  } else {
    if (ds && M > 0) {
      ProfScope prof("vocab_dstates", st);
      if (dtype == FOLD_F32) launch<float, kAlong, kAcross, float>(states, s1, st);
      else launch<uint16_t, kAlong, kAcross, float>(states, s1, st);
    }
    if (dW) {
      ProfScope prof("vocab_dweights", st);
      if (dtype == FOLD_F32) launch<float, kAcross, kAcross, float>(weights, s2, st);
      else launch<uint16_t, kAcross, kAcross, float>(weights, s2, st);
    }
  }
  if (ds && M > 0 && s1.split > 1) {
    ProfScope prof("vocab_dstates_join", st);
    join<true>(static_cast<const float*>(ws), s1.split, (size_t)M * ldh, (size_t)M * ldh, ds, 0, st);
  }
  if (db && !sums) {
    ProfScope prof("vocab_dbias", st);
    const int c = bias_chunks(M, V, es);
    float* part = static_cast<float*>(ws);
    const dim3 grid((unsigned)(((int64_t)ldv * es + 1023) / 1024 * c));
    if (dtype == FOLD_F32)
      hipLaunchKernelGGL(k_column_sums<float>, grid, dim3(256), 0, st, static_cast<const float*>(dz), M, V,
                         (size_t)ldv, c, part, db, add);
    else
      hipLaunchKernelGGL(k_column_sums<uint16_t>, grid, dim3(256), 0, st, static_cast<const uint16_t*>(dz), M, V,
                         (size_t)ldv, c, part, db, add);
    if (c > 1) join<false>(part, c, (size_t)ldv, (size_t)V, db, add, st);
  }
}

}  // namespace fold
