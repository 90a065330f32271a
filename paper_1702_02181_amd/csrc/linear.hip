// Linear layers over rows of node states (gfx950):
//     forward   out = act(x W^T + b) + r      x [M, K], W [N, K]: both operands run along K
//     backward  dz = dout act'(pre),  dx = dz W,  dW (+)= dz^T x,  db (+)= sum_m dz
// Many rows: product.h's tiles, the forward's with the activation and the residual on the way out.  Few rows: W is read once,
// straight into the matrix cores' registers, by enough waves for the whole chip.
// 16,384 x 4,096 x 1,024 bf16 with a residual: 135 us, 1,020 TFLOP/s (an 8,192^3 product of the library: 1,190); the gradient of
// 16,384 x 1,024 x 4,096 with gelu: 329 us, of which dz 80; 1 x 1,024 x 4,096: 3.8 us.

#include <hip/hip_runtime.h>

#include "product.h"

namespace fold {

namespace {

// ---- few rows -------------------------------------------------------------------------------------------------------

// What bounds a few rows is W's way through memory.  A workgroup takes 16 outputs; its WAVES waves cut K into chunks of 256
// bytes, of which a wave loads 16 rows of W (16 bytes a lane, four loads in flight) and the same columns of x, which come from
// the caches.  W's rows are the matrix instruction's rows, so a lane holds four neighbouring outputs of a row of x; the waves'
// sums meet in LDS and are added in their order.
constexpr int kFewRows = 64, kFewWaves = 8;

template <typename T, int MB, int ACT>
__global__ __launch_bounds__(64 * kFewWaves) void k_linear_few(const T* x, const T* W, const float* bias, const T* res,
                                                               T* out, T* pre, int M, int K, int N, int ldk, int ldn) {
  constexpr int EV = 16 / (int)sizeof(T), STEPS = 4;  // elements of 16 bytes; 64-byte steps of a chunk
  __shared__ float red[kFewWaves][MB * 16][17];
  const int lane = threadIdx.x & 63, wave = wave_id(), l16 = lane & 15, quad = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const T* w = W + (size_t)min(n0 + l16, N - 1) * ldk + quad * EV;
  const T* xr[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) xr[b] = x + (size_t)min(16 * b + l16, M - 1) * ldk + quad * EV;
  f32x4 acc[MB];
#pragma unroll
  for (int b = 0; b < MB; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = ldk / (4 * EV);  // whole: a row's stride is a multiple of 64 elements
  for (int s0 = wave * STEPS; s0 < steps; s0 += kFewWaves * STEPS) {
    uint4 a[STEPS], v[MB][STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const size_t at = (size_t)min(s0 + s, steps - 1) * 4 * EV;
      a[s] = *reinterpret_cast<const uint4*>(w + at);
#pragma unroll
      for (int b = 0; b < MB; ++b) v[b][s] = *reinterpret_cast<const uint4*>(xr[b] + at);
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      if (s0 + s >= steps) break;
#pragma unroll
      for (int b = 0; b < MB; ++b) {
        if constexpr (sizeof(T) == 2)
          acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[s]),
                                                           __builtin_bit_cast(bf16x8, v[b][s]), acc[b], 0, 0, 0);
        else
#pragma unroll
          for (int e = 0; e < 4; ++e)
            acc[b] = __builtin_amdgcn_mfma_f32_16x16x4f32(word(a[s], e), word(v[b][s], e), acc[b], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int b = 0; b < MB; ++b)
#pragma unroll
    for (int e = 0; e < 4; ++e) red[wave][16 * b + l16][4 * quad + e] = acc[b][e];
  __syncthreads();
  for (int i = threadIdx.x; i < MB * 256; i += 64 * kFewWaves) {
    const int m = i >> 4, n = n0 + (i & 15);
    if (m >= M || n >= ldn) continue;
    float z = n < N && bias ? bias[n] : 0.f;
#pragma unroll
    for (int wv = 0; wv < kFewWaves; ++wv) z += red[wv][m][i & 15];
    const size_t at = (size_t)m * ldn + n;
    if (pre) pre[at] = from_f32<T>(n < N ? z : 0.f);
    const float r = res ? to_f32<T>(res[at]) : 0.f;
    out[at] = from_f32<T>(n < N ? act_value<ACT, T>(z) + r : 0.f);
  }
}

// ---- few tiles: K in pieces ------------------------------------------------------------------------------------------------

// out = act(the pieces' sum + bias) + residual, four columns of a row a thread, eight pieces in flight
template <typename T, int ACT>
__global__ __launch_bounds__(256) void k_linear_join(const float* part, int pieces, int64_t M, int N, int ld, const float* bias,
                                                     const T* res, T* out, T* pre) {
  const size_t n = (size_t)M * ld, i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= n) return;
  const int col = (int)(i % (size_t)ld);
  typedef typename Four<T>::raw raw;
  float s[4] = {0.f, 0.f, 0.f, 0.f}, r[4] = {0.f, 0.f, 0.f, 0.f}, y[4];
  raw rr{};
  if (res) rr = *reinterpret_cast<const raw*>(res + i);
#pragma unroll
  for (int e = 0; e < 4; ++e) s[e] = bias && col + e < N ? bias[col + e] : 0.f;
  for (int p0 = 0; p0 < pieces; p0 += 8) {
    float4 v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const float4*>(part + (size_t)min(p0 + u, pieces - 1) * n + i);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const bool in = p0 + u < pieces;
      s[0] += in ? v[u].x : 0.f;
      s[1] += in ? v[u].y : 0.f;
      s[2] += in ? v[u].z : 0.f;
      s[3] += in ? v[u].w : 0.f;
    }
  }
  if (res) Four<T>::take(rr, r);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const bool in = col + e < N;
    y[e] = in ? act_value<ACT, T>(s[e]) + r[e] : 0.f;
    s[e] = in ? s[e] : 0.f;
  }
  if (pre) *reinterpret_cast<raw*>(pre + i) = Four<T>::give(s);
  *reinterpret_cast<raw*>(out + i) = Four<T>::give(y);
}

// ---- the gradient of the activation ------------------------------------------------------------------------------------

// dz = dout act'(pre), rounded to T as it enters its products beside W and x (in bf16 at most 2^-8 of each; fp32 products are
// sixteen times as long), and the rows' sums of dz before that.  A workgroup takes 64 16-byte vectors of columns of one
// of `chunks` pieces of the rows; its four waves take every fourth row, four of them in flight.  One piece writes db itself,
// more their sums to part [chunks][ld].
template <typename T, int ACT>
__global__ __launch_bounds__(256) void k_activation_back(const T* dout, const T* pre, T* dz, int64_t M, int N, size_t ld,
                                                         int chunks, float* part, float* db, int add) {
  constexpr int VEC = 16 / (int)sizeof(T), U = 4;
  __shared__ float red[4][64 * VEC + 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const size_t col = ((size_t)(blockIdx.x / chunks) * 64 + lane) * VEC;
  const int chunk = (int)(blockIdx.x % chunks);
  const int64_t per = (M + chunks - 1) / chunks, lo = min(chunk * per, M), hi = min(lo + per, M);
  float s[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) s[e] = 0.f;
  if (col < ld)
    for (int64_t m = lo + wave; m < hi; m += 4 * U) {
      uint4 d[U], z[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const size_t at = (size_t)min(m + 4 * u, hi - 1) * ld + col;
        d[u] = *reinterpret_cast<const uint4*>(dout + at);
        z[u] = *reinterpret_cast<const uint4*>(pre + at);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (m + 4 * u >= hi) break;
        const T *dv = reinterpret_cast<const T*>(&d[u]), *zv = reinterpret_cast<const T*>(&z[u]);
        uint4 o;
        T* ov = reinterpret_cast<T*>(&o);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float t = (int)col + e < N ? to_f32<T>(dv[e]) * act_slope<ACT, T>(to_f32<T>(zv[e])) : 0.f;
          s[e] += t;
          ov[e] = from_f32<T>(t);
        }
        *reinterpret_cast<uint4*>(dz + (size_t)(m + 4 * u) * ld + col) = o;
      }
    }
  if (!part && !db) return;
#pragma unroll
  for (int e = 0; e < VEC; ++e) red[wave][lane * VEC + e] = s[e];
  __syncthreads();
  const size_t c0 = (size_t)(blockIdx.x / chunks) * 64 * VEC;
  for (int i = threadIdx.x; i < 64 * VEC; i += 256) {
    if (c0 + i >= ld) break;
    const float t = (red[0][i] + red[1][i]) + (red[2][i] + red[3][i]);
    if (chunks > 1) part[(size_t)chunk * ld + c0 + i] = t;
    else if (c0 + i < (size_t)N) db[c0 + i] = add ? db[c0 + i] + t : t;
  }
}

// Pieces of the rows: eight workgroups a compute unit, whose arithmetic (some 30 instructions a value for gelu) then runs beside
// the others' loads, each with at least 16 rows.
int activation_chunks(int64_t M, int N, int es) {
  const int64_t groups = ((int64_t)row_ld(N) * es + 1023) / 1024;
  return (int)std::max<int64_t>(1, std::min<int64_t>({2048 / groups, M / 16, 256}));
}

// out (+)= the sum of the pieces in their order, eight loads in flight, rounded to OUT; n a multiple of 4
template <typename OUT>
__global__ __launch_bounds__(256) void k_join_as(const float* part, int pieces, size_t n, OUT* out, int add) {
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= n) return;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < pieces; p0 += 8) {
    float4 v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = *reinterpret_cast<const float4*>(part + (size_t)min(p0 + u, pieces - 1) * n + i);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const bool in = p0 + u < pieces;
      s[0] += in ? v[u].x : 0.f;
      s[1] += in ? v[u].y : 0.f;
      s[2] += in ? v[u].z : 0.f;
      s[3] += in ? v[u].w : 0.f;
    }
  }
  typedef typename Four<OUT>::raw raw;
  if (add) {
    float o[4];
    Four<OUT>::take(*reinterpret_cast<const raw*>(out + i), o);
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] += o[e];
  }
  *reinterpret_cast<raw*>(out + i) = Four<OUT>::give(s);
}

// ---- shapes ----------------------------------------------------------------------------------------------------------

// A compute unit that has one workgroup of 128 x 128 tiles alone waits for its loads: 16,384 x 1,024 x 4,096 bf16, dW in 256 of
// them 165 us, in 512 (two pieces) 142, in 256 of 256 x 256 (four pieces) 128.
constexpr double kAlone = 1.25;

Shape forward_shape(int64_t M, int K, int N, int es) {
  return shape_of(M, row_ld(N), row_ld(K) * es / 128, es, 2, kPieces, false, kAlone, true);
}
Shape dx_shape(int64_t M, int K, int N, int es) {
  return shape_of(std::max<int64_t>(M, 1), row_ld(K), (int64_t)row_ld(N) * es / 128, es, 1, kPieces, false, kAlone);
}
Shape dw_shape(int64_t M, int K, int N, int es) {
  const int lines = 128 / es;
  return shape_of(N, row_ld(K), std::max<int64_t>(1, (M + lines - 1) / lines), es, 1, kPieces, false, kAlone);
}

// Up to 64 rows go by k_linear_few while what a wave multiplies stays short: every block of 16 rows is multiplied along K / 8 by
// one wave.  Both ways, few rows and tiles: 1 x 4,096 x 4,096 bf16 9.1 and 11.9 us, 32 rows 15.7 and 12.7; 64 x 1,024 x 4,096 9.2
// and 11.1; 64 x 2,048 x 4,096 14.9 and 13.8; 1 x 16,384 x 1,024 22.5 and 12.8; fp32 1 x 4,096 x 4,096 21.4 and 25.8, 32 rows 28.5
// and 27.1; 64 x 1,024 x 4,096 16.6 and 17.7, 64 x 2,048 x 1,024 23.3 and 13.9.
bool few_rows(int64_t M, int K) {
  const int blocks = M <= 16 ? 1 : M <= 32 ? 2 : 4;
  return M <= kFewRows && row_ld(K) * blocks <= 4096;
}

template <typename T, int ACT>
void few(int M, int K, int N, const void* x, const void* W, const float* bias, const void* res, void* out, void* pre,
         hipStream_t st) {
  const int ldk = row_ld(K), ldn = row_ld(N), mb = (M + 15) / 16;
  const dim3 grid(ldn / 16), block(64 * kFewWaves);
  const auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, block, 0, st, static_cast<const T*>(x), static_cast<const T*>(W), bias,
                       static_cast<const T*>(res), static_cast<T*>(out), static_cast<T*>(pre), M, K, N, ldk, ldn);
  };
  if (mb <= 1) go(k_linear_few<T, 1, ACT>);
  else if (mb <= 2) go(k_linear_few<T, 2, ACT>);
  else go(k_linear_few<T, 4, ACT>);
}

template <typename T, int ACT>
void forward(int64_t M, int K, int N, const void* x, const void* W, const float* bias, const void* res, void* out,
             void* pre, void* ws, hipStream_t st) {
  if (few_rows(M, K)) return few<T, ACT>((int)M, K, N, x, W, bias, res, out, pre, st);
  const int es = sizeof(T), ldk = row_ld(K), ldn = row_ld(N);
  const Shape sh = forward_shape(M, K, N, es);
  ProductArgs g{{x, M, ldk}, {W, N, ldk}, M, N, sh.mt, sh.nt, ldk * es / 128, sh.split, out, (size_t)ldn, ldn, bias, 0, nullptr};
  if (sh.split > 1) {
    g.out = ws;
    g.bias = nullptr;
    launch<T, kAlong, kAlong, float>(g, sh, st);
    hipLaunchKernelGGL((k_linear_join<T, ACT>), dim3((unsigned)(((size_t)M * ldn + 1023) / 1024)), dim3(256), 0, st,
                       static_cast<const float*>(ws), sh.split, M, N, ldn, bias, static_cast<const T*>(res),
                       static_cast<T*>(out), static_cast<T*>(pre));
    return;
  }
  g.residual = res;
  g.pre = pre;
  if constexpr (ACT == FOLD_ACT_NONE)
    if (!res && !pre) return launch<T, kAlong, kAlong, T>(g, sh, st);
  launch<T, kAlong, kAlong, T, ACT>(g, sh, st);
}

// C of type OUT from a product whose K may be cut: the pieces' fp32 sums go through ws
template <typename T, int AD, typename OUT>
void cut_product(ProductArgs g, const Shape& sh, OUT* out, void* ws, int add, hipStream_t st) {
  if (sh.split == 1) {
    g.out = out;
    g.add = add;
    launch<T, AD, kAcross, OUT>(g, sh, st);
    return;
  }
  g.out = ws;
  launch<T, AD, kAcross, float>(g, sh, st);
  const size_t n = (size_t)g.M * g.ld;
  hipLaunchKernelGGL(k_join_as<OUT>, dim3((unsigned)((n + 1023) / 1024)), dim3(256), 0, st, static_cast<const float*>(ws),
                     sh.split, n, out, add);
}

// The two gradients of a small batch in one launch, in the smallest tiles: apart, each leaves much of the chip idle and has a
// launch's start to itself.  `first` workgroups (a multiple of 8) for dx, the rest for dW.
bool together(const Shape& dx, const Shape& dw) { return dx.wm == 1 && dw.wm == 1; }
template <typename T, typename OX, typename OW>
__global__ __launch_bounds__(kThreads, 2) void k_linear_both(ProductArgs states, ProductArgs weights, unsigned first) {
  __shared__ __attribute__((aligned(16))) ProductLds<1, 1, 128, 2> lds;
  if (blockIdx.x < first) product<T, kAlong, kAcross, OX, 1, 1, 128, 2>(states, blockIdx.x, lds);
  else product<T, kAcross, kAcross, OW, 1, 1, 128, 2>(weights, blockIdx.x - first, lds);
}
template <typename T, typename OX, typename OW>
void both_products(ProductArgs x, ProductArgs w, const Shape& s1, const Shape& s2, OX* dx, OW* dw, float* ws, int add,
                   hipStream_t st) {
  const size_t nx = (size_t)x.M * x.ld, nw = (size_t)w.M * w.ld;
  float* wpart = ws + (s1.split > 1 ? s1.split * nx : 0);
  x.out = s1.split > 1 ? static_cast<void*>(ws) : dx;
  w.out = s2.split > 1 ? static_cast<void*>(wpart) : dw;
  w.add = s2.split > 1 ? 0 : add;
  const unsigned n1 = blocks_of(x), n2 = blocks_of(w);
  const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(n1 + n2), dim3(kThreads), 0, st, x, w, n1); };
  if (s1.split > 1 && s2.split > 1) go(k_linear_both<T, float, float>);
  else if (s1.split > 1) go(k_linear_both<T, float, OW>);
  else if (s2.split > 1) go(k_linear_both<T, OX, float>);
  else go(k_linear_both<T, OX, OW>);
  if (s1.split > 1)
    hipLaunchKernelGGL(k_join_as<OX>, dim3((unsigned)((nx + 1023) / 1024)), dim3(256), 0, st, ws, s1.split, nx, dx, 0);
  if (s2.split > 1)
    hipLaunchKernelGGL(k_join_as<OW>, dim3((unsigned)((nw + 1023) / 1024)), dim3(256), 0, st, wpart, s2.split, nw, dw, add);
}

template <typename T>
void backward(int64_t M, int K, int N, const void* x, const void* W, int act, const void* pre, const void* dout, void* dpre,
              int dx_dtype, void* dx, int dw_dtype, void* dW, float* db, int add, void* ws, hipStream_t st) {
  const int es = sizeof(T), ldk = row_ld(K), ldn = row_ld(N);
  const T* dz = static_cast<const T*>(dout);
  if (act != FOLD_ACT_NONE || db) {
    ProfScope prof(act == FOLD_ACT_NONE ? "linear_dbias" : "linear_activation", st);
    const int c = act == FOLD_ACT_NONE ? bias_chunks(M, N, es) : activation_chunks(M, N, es);
    float* part = db && c > 1 ? static_cast<float*>(ws) : nullptr;
    const dim3 grid((unsigned)(((int64_t)ldn * es + 1023) / 1024 * c));
    const auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, dz, static_cast<const T*>(pre), static_cast<T*>(dpre), M, N,
                         (size_t)ldn, c, part, db, add);
    };
    if (act == FOLD_ACT_RELU) go(k_activation_back<T, FOLD_ACT_RELU>);
    else if (act == FOLD_ACT_TANH) go(k_activation_back<T, FOLD_ACT_TANH>);
    else if (act == FOLD_ACT_GELU) go(k_activation_back<T, FOLD_ACT_GELU>);
    else
      hipLaunchKernelGGL(k_column_sums<T>, grid, dim3(256), 0, st, dz, M, N, (size_t)ldn, c, part, db, add);
    if (part) join<false>(part, c, (size_t)ldn, (size_t)N, db, add, st);
    if (act != FOLD_ACT_NONE) dz = static_cast<const T*>(dpre);
  }
  const Shape s1 = dx_shape(M, K, N, es), s2 = dw_shape(M, K, N, es);
  const int lines = 128 / es;
  const ProductArgs states{{dz, M, ldn}, {W, N, ldk}, M, K, s1.mt, s1.nt, ldn * es / 128, s1.split, nullptr, (size_t)ldk, ldk,
                           nullptr, 0, nullptr};
  const ProductArgs weights{{dz, M, ldn}, {x, M, ldk}, N, K, s2.mt, s2.nt, (int)((M + lines - 1) / lines), s2.split, nullptr,
                            (size_t)ldk, ldk, nullptr, 0, nullptr};
  if (dx && dW && M > 0 && together(s1, s2)) {
    ProfScope prof("linear_dx_dw", st);
    const auto both = [&](auto* px, auto* pw) {
      both_products<T>(states, weights, s1, s2, px, pw, static_cast<float*>(ws), dw_dtype == FOLD_F32 ? add : 0, st);
    };
    if constexpr (sizeof(T) == 2) {
      T *tx = static_cast<T*>(dx), *tw = static_cast<T*>(dW);
      if (dx_dtype == FOLD_F32 && dw_dtype == FOLD_F32) both(static_cast<float*>(dx), static_cast<float*>(dW));
      else if (dx_dtype == FOLD_F32) both(static_cast<float*>(dx), tw);
      else if (dw_dtype == FOLD_F32) both(tx, static_cast<float*>(dW));
      else both(tx, tw);
    } else {
      both(static_cast<float*>(dx), static_cast<float*>(dW));
    }
    return;
  }
  if (dx && M > 0) {
    ProfScope prof("linear_dx", st);
    if (dx_dtype == FOLD_F32) cut_product<T, kAlong, float>(states, s1, static_cast<float*>(dx), ws, 0, st);
    else if constexpr (sizeof(T) == 2) cut_product<T, kAlong, uint16_t>(states, s1, static_cast<uint16_t*>(dx), ws, 0, st);
  }
  if (dW) {
    ProfScope prof("linear_dw", st);
    if (dw_dtype == FOLD_F32) cut_product<T, kAcross, float>(weights, s2, static_cast<float*>(dW), ws, add, st);
    else if constexpr (sizeof(T) == 2) cut_product<T, kAcross, uint16_t>(weights, s2, static_cast<uint16_t*>(dW), ws, 0, st);
  }
}

}  // namespace

int64_t linear_tiles(int dtype, int64_t M, int K, int N) {
  const Shape sh = forward_shape(M, K, N, dtype == FOLD_BF16 ? 2 : 4);
  if (few_rows(M, K)) return row_ld(N) / 16;
  return std::max(sh.mt * sh.nt * sh.split, sh.split > 1 ? M * row_ld(N) / 1024 + 1 : 0);
}
size_t linear_bytes(int dtype, int64_t M, int K, int N) {
  const Shape sh = forward_shape(M, K, N, dtype == FOLD_BF16 ? 2 : 4);
  return few_rows(M, K) || sh.split == 1 ? 0 : (size_t)sh.split * M * row_ld(N) * sizeof(float);
}
int64_t linear_backward_tiles(int dtype, int64_t M, int K, int N) {
  const int es = dtype == FOLD_BF16 ? 2 : 4;
  const Shape a = dx_shape(M, K, N, es), b = dw_shape(M, K, N, es);
  const int64_t join = ((int64_t)std::max(a.split > 1 ? (M + 1) * row_ld(K) : 0, b.split > 1 ? (int64_t)N * row_ld(K) : 0)) / 1024 + 1;
  return std::max(a.mt * a.nt * a.split + b.mt * b.nt * b.split, join);
}

void launch_linear(int dtype, int64_t M, int K, int N, const void* x, const void* W, const float* bias, int act,
                   const void* res, void* out, void* pre, void* ws, hipStream_t st) {
  if (M <= 0) return;
  ProfScope prof("linear", st);
  const auto go = [&](auto a) {
    constexpr int ACT = decltype(a)::value;
    if (dtype == FOLD_F32) forward<float, ACT>(M, K, N, x, W, bias, res, out, pre, ws, st);
    else forward<uint16_t, ACT>(M, K, N, x, W, bias, res, out, pre, ws, st);
  };
  if (act == FOLD_ACT_RELU) go(std::integral_constant<int, FOLD_ACT_RELU>());
  else if (act == FOLD_ACT_TANH) go(std::integral_constant<int, FOLD_ACT_TANH>());
  else if (act == FOLD_ACT_GELU) go(std::integral_constant<int, FOLD_ACT_GELU>());
  else go(std::integral_constant<int, FOLD_ACT_NONE>());
}

size_t linear_backward_bytes(int dtype, int64_t M, int K, int N) {
  const int es = dtype == FOLD_BF16 ? 2 : 4;
  const Shape a = dx_shape(M, K, N, es), b = dw_shape(M, K, N, es);
  const int c = std::max(bias_chunks(M, N, es), activation_chunks(M, N, es));
  // they follow each other on the stream, so one region serves all; in one launch either has its own
  const size_t dx = a.split > 1 ? (size_t)a.split * M * row_ld(K) : 0, dw = b.split > 1 ? (size_t)b.split * N * row_ld(K) : 0;
  return std::max({together(a, b) ? dx + dw : std::max(dx, dw), c > 1 ? (size_t)c * row_ld(N) : (size_t)0}) * sizeof(float);
}

void launch_linear_backward(int dtype, int64_t M, int K, int N, const void* x, const void* W, int act, const void* pre,
                            const void* dout, void* dpre, int dx_dtype, void* dx, int dw_dtype, void* dW, float* dbias,
                            int add, void* ws, hipStream_t st) {
  if (dtype == FOLD_F32)
    backward<float>(M, K, N, x, W, act, pre, dout, dpre, dx_dtype, dx, dw_dtype, dW, dbias, add, ws, st);
  else
    backward<uint16_t>(M, K, N, x, W, act, pre, dout, dpre, dx_dtype, dx, dw_dtype, dW, dbias, add, ws, st);
}

}  // namespace fold
