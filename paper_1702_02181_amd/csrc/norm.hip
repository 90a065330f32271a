// Layer norm of rows of node states, forward and backward (gfx950).
//     mean = (1/n) sum x,  rstd = (mean of (x - mean)^2 + eps)^-1/2,  xh = (x - mean) rstd,  y = gamma xh + beta
//     g = gamma dy,  dx = rstd (g - mean(g) - xh mean(g xh)) (+ residual),  dgamma = sum dy xh,  dbeta = sum dy
// HBM bounds both: a row is read once, into the registers of the LPR lanes that share it, NV vectors of 16 bytes a lane, and
// everything about it is computed there in fp32 (the deviations from the mean itself, not from a difference of sums).
// 131,072 x 1,024 bf16: 108 us, 5.0 TB/s; gradients of 65,536 x 1,024 bf16 with a residual: 108 us, 5.0 TB/s; of 55,911 x 512
// fp32: 67 us, 5.1 TB/s; a copy of 2 GiB: 4.96 TB/s.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "internal.h"
#include "mfma.h"

namespace fold {

namespace {

constexpr int kThreads = 256;

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
// the sum over W neighbouring lanes, the same in all of them
template <int W>
__device__ __forceinline__ float lanes_sum(float v) {
  v += dpp<0xb1>(v);                // lane ^ 1
  v += dpp<0x4e>(v);                // lane ^ 2
  v += dpp<0x141>(v);               // 7 - lane, of 8
  if constexpr (W > 8) v += dpp<0x140>(v);  // 15 - lane, of 16
  if constexpr (W > 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (W > 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}

// the same over the LPR lanes of a row; above 64 they are in several waves, which meet in `red` (one place a wave)
template <int LPR>
__device__ __forceinline__ float row_sum(float v, float* red) {
  v = lanes_sum<(LPR > 64 ? 64 : LPR)>(v);
  if constexpr (LPR > 64) {
    const int wave = threadIdx.x >> 6, first = wave & ~(LPR / 64 - 1);
    __syncthreads();  // the sum before this one has been read
    red[wave] = v;
    __syncthreads();
    v = red[first];
#pragma unroll
    for (int w = 1; w < LPR / 64; ++w) v += red[first + w];
  }
  return v;
}

// The values of a row that a lane holds: vector i is the row's vector i LPR + lane, VEC values from column (i LPR + lane) VEC.
template <typename T>
struct Vec {
  static constexpr int N = 16 / (int)sizeof(T);
  __device__ static __forceinline__ void take(const uint4& r, float (&v)[N]) {
    const T* e = reinterpret_cast<const T*>(&r);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = to_f32<T>(e[k]);
  }
  __device__ static __forceinline__ uint4 give(const float (&v)[N]) {
    uint4 r;
    T* e = reinterpret_cast<T*>(&r);
#pragma unroll
    for (int k = 0; k < N; ++k) e[k] = from_f32<T>(v[k]);
    return r;
  }
};

// columns col .. col + 3 of a vector of n values; 0 behind its end, `none` where there is no vector
__device__ __forceinline__ void load4(const float* p, int col, int n, float none, float (&v)[4]) {
  if (p && col + 4 <= n && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    const float4 w = *reinterpret_cast<const float4*>(p + col);
    v[0] = w.x;
    v[1] = w.y;
    v[2] = w.z;
    v[3] = w.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = col + e < n ? (p ? p[col + e] : none) : 0.f;
  }
}

struct NormArgs {
  const void* x;
  int64_t rows;
  int n, ld;
  const float *gamma, *beta;
  float eps;
  void* y;
  float *mean, *rstd;
};

template <typename T, int LPR, int NV>
__global__ __launch_bounds__(kThreads) void k_norm(NormArgs a) {
  using V = Vec<T>;
  constexpr int VEC = V::N, RPB = kThreads / LPR;
  __shared__ float red[kThreads / 64];
  const int gl = threadIdx.x % LPR, vecs = a.ld / VEC;
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / LPR;
  const T* x = static_cast<const T*>(a.x);
  const float n = (float)a.n;
  const bool tail = a.n < LPR * NV * VEC;  // (then what lies past the row's values is looked away from)
  auto load = [&](int64_t r, uint4 (&v)[NV]) {
    const uint4* p = reinterpret_cast<const uint4*>(x + (size_t)min(r, a.rows - 1) * a.ld);
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = p[min(i * LPR + gl, vecs - 1)];
  };
  uint4 raw[NV];
  load(row, raw);
  // weights stay in registers over the rows; zero past the last column, so that the pad columns come out as zero
  float g[NV][VEC], b[NV][VEC];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < VEC; e += 4) {
      float t[4], u[4];
      load4(a.gamma, (i * LPR + gl) * VEC + e, a.n, 1.f, t);
      load4(a.beta, (i * LPR + gl) * VEC + e, a.n, 0.f, u);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        g[i][e + k] = t[k];
        b[i][e + k] = u[k];
      }
    }
  // all waves of the workgroup take part in every round; rows behind the last one are the last one again, and not stored
  for (int64_t first = (int64_t)blockIdx.x * RPB; first < a.rows; first += step, row += step) {
    uint4 next[NV];
    load(row + step, next);
    float v[NV][VEC], sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      V::take(raw[i], v[i]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        if (tail) v[i][e] = (i * LPR + gl) * VEC + e < a.n ? v[i][e] : 0.f;
        sum += v[i][e];
      }
    }
    const float mean = row_sum<LPR>(sum, red) / n;
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        v[i][e] -= mean;
        if (tail) v[i][e] = (i * LPR + gl) * VEC + e < a.n ? v[i][e] : 0.f;
        sq += v[i][e] * v[i][e];
      }
    const float rstd = 1.f / sqrtf(row_sum<LPR>(sq, red) / n + a.eps);
    T* y = static_cast<T*>(a.y) + (size_t)row * a.ld;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        v[i][e] = v[i][e] * rstd * g[i][e] + b[i][e];
        if (tail) v[i][e] = (i * LPR + gl) * VEC + e < a.n ? v[i][e] : 0.f;
      }
      if (i * LPR + gl < vecs && row < a.rows) reinterpret_cast<uint4*>(y)[i * LPR + gl] = V::give(v[i]);
    }
    if (gl == 0 && row < a.rows) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = next[i];
  }
}

struct NormBackArgs {
  const void* x;
  int64_t rows;
  int n, ld;
  const float *gamma, *mean, *rstd;
  const void* dy;
  int dy_f32;          // dy is fp32 (where T is bf16)
  const void* residual;
  void* dx;            // or NULL
  int dx_f32, res_f32; // dx, the residual are fp32
  float* part;         // [blocks][2][ld]: the block's sums for gamma and beta; NULL: nobody wants them, or:
  float *dgamma, *dbeta;  // a single workgroup writes them itself
  int add;
};

// 16 bytes of T, or, where types are MIXED, perhaps the same values in fp32 (twice 16 bytes)
template <typename T, bool MIXED>
struct Pair {
  uint4 lo, hi[MIXED ? 1 : 0];
};
template <typename T, bool MIXED>
__device__ __forceinline__ Pair<T, MIXED> load_pair(const void* p, size_t row, int ld, int vec, bool f32) {
  Pair<T, MIXED> r;
  if (MIXED && f32) {
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + row * ld) + 2 * vec;
    r.lo = q[0];
    if constexpr (MIXED) r.hi[0] = q[1];
  } else {
    r.lo = reinterpret_cast<const uint4*>(static_cast<const T*>(p) + row * ld)[vec];
    if constexpr (MIXED) r.hi[0] = make_uint4(0, 0, 0, 0);
  }
  return r;
}
template <typename T, bool MIXED>
__device__ __forceinline__ void take_pair(const Pair<T, MIXED>& r, bool f32, float (&v)[Vec<T>::N]) {
  if constexpr (MIXED)
    if (f32) {
      const float* lo = reinterpret_cast<const float*>(&r.lo);
      const float* hi = reinterpret_cast<const float*>(&r.hi[0]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = lo[e];
        v[4 + e] = hi[e];
      }
      return;
    }
  Vec<T>::take(r.lo, v);
}

// A workgroup walks over rows of the whole matrix and keeps its sums for gamma and beta in registers until the end.
template <typename T, int LPR, int NV, bool MIXED>
__global__ __launch_bounds__(kThreads) void k_norm_back(NormBackArgs a) {
  using V = Vec<T>;
  constexpr int VEC = V::N, RPB = kThreads / LPR;
  __shared__ float red[2][LPR * NV * VEC], meet[kThreads / 64];
  const int gl = threadIdx.x % LPR, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, vecs = a.ld / VEC;
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / LPR;
  const T* x = static_cast<const T*>(a.x);
  const float n = (float)a.n;
  const bool dyf = a.dy_f32, dxf = a.dx_f32, resf = a.res_f32;
  uint4 raw[NV];
  Pair<T, MIXED> rdy[NV], rres[NV];
  float mean, rstd;
  const bool added = a.dx && a.residual, tail = a.n < LPR * NV * VEC;
  auto load = [&](int64_t at) {
    const size_t r = (size_t)min(at, a.rows - 1);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int vec = min(i * LPR + gl, vecs - 1);
      raw[i] = reinterpret_cast<const uint4*>(x + r * a.ld)[vec];
      rdy[i] = load_pair<T, MIXED>(a.dy, r, a.ld, vec, dyf);
      if (added) rres[i] = load_pair<T, MIXED>(a.residual, r, a.ld, vec, resf);
    }
    mean = a.mean[r];
    rstd = a.rstd[r];
  };
  load(row);
  float g[NV][VEC], dg[NV][VEC], db[NV][VEC];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < VEC; e += 4) {
      float t[4];
      load4(a.gamma, (i * LPR + gl) * VEC + e, a.n, 1.f, t);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        g[i][e + k] = t[k];
        dg[i][e + k] = db[i][e + k] = 0.f;
      }
    }
  for (int64_t first = (int64_t)blockIdx.x * RPB; first < a.rows; first += step, row += step) {
    float xh[NV][VEC], dy[NV][VEC], s1 = 0.f, s2 = 0.f;
    const float m = mean, rs = rstd;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      V::take(raw[i], xh[i]);
      take_pair<T, MIXED>(rdy[i], dyf, dy[i]);
    }
    Pair<T, MIXED> res[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) res[i] = rres[i];
    load(row + step);
    if (tail)  // what lies past the row's values, whatever it is
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const bool in = (i * LPR + gl) * VEC + e < a.n;
          xh[i][e] = in ? xh[i][e] : m;
          dy[i][e] = in ? dy[i][e] : 0.f;
        }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e) xh[i][e] = (xh[i][e] - m) * rs;
    if (row < a.rows)
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          dg[i][e] += dy[i][e] * xh[i][e];
          db[i][e] += dy[i][e];
        }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        dy[i][e] *= g[i][e];
        s1 += dy[i][e];
        s2 += dy[i][e] * xh[i][e];
      }
    if (!a.dx) continue;
    s1 = row_sum<LPR>(s1, meet) / n;
    s2 = row_sum<LPR>(s2, meet) / n;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int vec = i * LPR + gl;
      float r[VEC];
      if (added) take_pair<T, MIXED>(res[i], resf, r);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        dy[i][e] = rs * (dy[i][e] - s1 - xh[i][e] * s2);
        if (added) dy[i][e] += r[e];
        if (tail) dy[i][e] = vec * VEC + e < a.n ? dy[i][e] : 0.f;
      }
      if (vec >= vecs || row >= a.rows) continue;
      if (MIXED && dxf) {
        uint4* q = reinterpret_cast<uint4*>(static_cast<float*>(a.dx) + (size_t)row * a.ld) + 2 * vec;
        const float* d = dy[i];
        q[0] = make_uint4(__float_as_uint(d[0]), __float_as_uint(d[1]), __float_as_uint(d[2]), __float_as_uint(d[3]));
        q[1] = make_uint4(__float_as_uint(d[VEC - 4]), __float_as_uint(d[VEC - 3]), __float_as_uint(d[VEC - 2]),
                          __float_as_uint(d[VEC - 1]));
      } else {
        reinterpret_cast<uint4*>(static_cast<T*>(a.dx) + (size_t)row * a.ld)[vec] = V::give(dy[i]);
      }
    }
  }
  if (!a.part && !a.dgamma && !a.dbeta) return;
  // the wave's rows, then the four waves one after the other
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < VEC; ++e)
#pragma unroll
      for (int o = LPR; o < 64; o *= 2) {
        dg[i][e] += __shfl_xor(dg[i][e], o);
        db[i][e] += __shfl_xor(db[i][e], o);
      }
  constexpr int WPR = LPR > 64 ? LPR / 64 : 1;  // waves of a row
  for (int w = 0; w < kThreads / 64; w += WPR) {
    if (wave / WPR * WPR == w && lane < LPR)
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const int at = (i * LPR + gl) * VEC + e;
          red[0][at] = w == 0 ? dg[i][e] : red[0][at] + dg[i][e];
          red[1][at] = w == 0 ? db[i][e] : red[1][at] + db[i][e];
        }
    __syncthreads();
  }
  if (!a.part) {
    for (int c = threadIdx.x; c < a.n; c += kThreads) {
      if (a.dgamma) a.dgamma[c] = a.add ? a.dgamma[c] + red[0][c] : red[0][c];
      if (a.dbeta) a.dbeta[c] = a.add ? a.dbeta[c] + red[1][c] : red[1][c];
    }
    return;
  }
  for (int c = threadIdx.x; c < 2 * a.ld; c += kThreads)
    a.part[(size_t)blockIdx.x * 2 * a.ld + c] = c < a.ld ? red[0][c] : red[1][c - a.ld];
}

// dgamma and dbeta from the workgroups' sums [pieces][2][ld], in a fixed order: 8 lanes of four columns by 32 groups that
// take every 32nd piece and meet in LDS.
__global__ __launch_bounds__(kThreads) void k_norm_join(const float* part, int pieces, int ld, int n, float* dgamma,
                                                        float* dbeta, int add) {
  __shared__ float4 red[32][8];
  const int at = threadIdx.x & 7, group = threadIdx.x >> 3;
  const int c = (blockIdx.x * 8 + at) * 4;  // of 2 ld, a multiple of 32
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = group; p0 < pieces; p0 += 32 * 8) {  // eight loads in flight
    float4 v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      v[u] = *reinterpret_cast<const float4*>(part + (size_t)min(p0 + 32 * u, pieces - 1) * 2 * ld + c);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const bool in = p0 + 32 * u < pieces;
      s.x += in ? v[u].x : 0.f;
      s.y += in ? v[u].y : 0.f;
      s.z += in ? v[u].z : 0.f;
      s.w += in ? v[u].w : 0.f;
    }
  }
  red[group][at] = s;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  float t = 0.f;
  for (int g = 0; g < 32; ++g) t += reinterpret_cast<const float*>(red[g])[threadIdx.x];
  const int col = blockIdx.x * 32 + threadIdx.x, at_col = col < ld ? col : col - ld;
  float* out = col < ld ? dgamma : dbeta;
  if (out && at_col < n) out[at_col] = add ? out[at_col] + t : t;
}

// How a row lies over lanes: the fewest lanes that hold it in 24 values each (16 where the row fills them), so that the
// backward's seven arrays of that many registers leave two waves a SIMD and more.
struct Lanes {
  int lpr, nv;
};
Lanes lanes_of(int ld, int esize) {
  const int vecs = ld * esize / 16, most = 6 * esize / 4;
  int l = 8;
  while (l < kThreads && vecs > l * most) l *= 2;
  return {l, (vecs + l - 1) / l};
}

// Workgroups of the backward: what the chip holds at once, two a compute unit, three where registers allow it (bf16, 16
// values a lane), each with at least four rounds of rows.
int back_blocks(int64_t rows, const Lanes& l, int esize) {
  const int64_t rpb = kThreads / l.lpr, most = esize == 2 && l.nv <= 2 ? 768 : 512;
  return (int)std::max<int64_t>(1, std::min<int64_t>(most, (rows + 4 * rpb - 1) / (4 * rpb)));
}

// f(LPR, NV) for the smallest NV that is built
template <typename F, int L, int A, int B, int C>
void with_vectors(int nv, F& f) {
  if (nv <= A) f(std::integral_constant<int, L>(), std::integral_constant<int, A>());
  else if (nv <= B) f(std::integral_constant<int, L>(), std::integral_constant<int, B>());
  else f(std::integral_constant<int, L>(), std::integral_constant<int, C>());
}
template <typename T, class F>
void with_lanes(const Lanes& l, F&& f) {
  constexpr int W = sizeof(T) == 2 ? 1 : 2;  // vectors of 8 values
  switch (l.lpr) {
    case 8: return with_vectors<F, 8, W, 2 * W, 3 * W>(l.nv, f);
    case 16: return with_vectors<F, 16, 2 * W, 2 * W, 3 * W>(l.nv, f);
    case 32: return with_vectors<F, 32, 2 * W, 2 * W, 3 * W>(l.nv, f);
    case 64: return with_vectors<F, 64, 2 * W, 2 * W, 3 * W>(l.nv, f);
    case 128: return with_vectors<F, 128, 2 * W, 2 * W, 3 * W>(l.nv, f);
    default: return with_vectors<F, 256, 2 * W, 2 * W, 2 * W>(l.nv, f);
  }
}

template <typename T>
void norm_rows(const NormArgs& a, hipStream_t st) {
  with_lanes<T>(lanes_of(a.ld, sizeof(T)), [&](auto lpr, auto nv) {
    constexpr int RPB = kThreads / decltype(lpr)::value;
    const int64_t blocks = std::min<int64_t>((a.rows + RPB - 1) / RPB, 5 * 256);
    hipLaunchKernelGGL((k_norm<T, decltype(lpr)::value, decltype(nv)::value>), dim3((unsigned)blocks), dim3(kThreads), 0,
                       st, a);
  });
}
template <typename T>
void norm_rows_back(const NormBackArgs& a, int blocks, hipStream_t st) {
  with_lanes<T>(lanes_of(a.ld, sizeof(T)), [&](auto lpr, auto nv) {
    constexpr int L = decltype(lpr)::value, N = decltype(nv)::value;
    const dim3 grid((unsigned)blocks), block(kThreads);
    if constexpr (sizeof(T) == 2)
      if (a.dy_f32 || a.dx_f32 || (a.residual && a.res_f32)) {
        hipLaunchKernelGGL((k_norm_back<T, L, N, true>), grid, block, 0, st, a);
        return;
      }
    hipLaunchKernelGGL((k_norm_back<T, L, N, false>), grid, block, 0, st, a);
  });
}

}  // namespace

void launch_norm(int dtype, int64_t rows, int n, const void* x, const float* gamma, const float* beta, float eps, void* y,
                 float* mean, float* rstd, hipStream_t st) {
  if (rows <= 0) return;
  ProfScope prof("layer_norm", st);
  const NormArgs a{x, rows, n, row_ld(n), gamma, beta, eps, y, mean, rstd};
  if (dtype == FOLD_F32) norm_rows<float>(a, st);
  else norm_rows<uint16_t>(a, st);
}

size_t norm_backward_bytes(int dtype, int64_t rows, int n) {
  const int ld = row_ld(n), es = dtype == FOLD_BF16 ? 2 : 4, blocks = back_blocks(rows, lanes_of(ld, es), es);
  return blocks == 1 ? 0 : (size_t)blocks * 2 * ld * sizeof(float);
}

void launch_norm_backward(int dtype, int64_t rows, int n, const void* x, const float* gamma, const float* mean,
                          const float* rstd, int dy_dtype, const void* dy, int dx_dtype, int res_dtype, const void* residual,
                          void* dx, float* dgamma, float* dbeta, int add, void* ws, hipStream_t st) {
  const int ld = row_ld(n), es = dtype == FOLD_BF16 ? 2 : 4;
  const Lanes l = lanes_of(ld, es);
  const int blocks = rows > 0 ? back_blocks(rows, l, es) : 0;
  const bool sums = dgamma || dbeta;
  float* part = sums && blocks != 1 ? static_cast<float*>(ws) : nullptr;
  if (rows > 0) {
    ProfScope prof("layer_norm_back", st);
    const NormBackArgs a{x, rows, n, ld, gamma, mean, rstd, dy, dy_dtype == FOLD_F32, residual, dx, dx_dtype == FOLD_F32,
                         res_dtype == FOLD_F32, part, blocks == 1 ? dgamma : nullptr, blocks == 1 ? dbeta : nullptr, add};
    if (dtype == FOLD_F32) norm_rows_back<float>(a, blocks, st);
    else norm_rows_back<uint16_t>(a, blocks, st);
  }
  if (sums && blocks != 1) {
    ProfScope prof("layer_norm_join", st);
    hipLaunchKernelGGL(k_norm_join, dim3((unsigned)(2 * ld / 32)), dim3(kThreads), 0, st, part, blocks, ld, n, dgamma,
                       dbeta, add);
  }
}

}  // namespace fold
