// Products of the vocabulary head on the matrix cores (gfx950):
//     logits   z = s W^T + b      s [M, H] states, W [V, H]: both operands run along K = H
//     states   ds = dz W          K = V: dz runs along K, W across it
//     weights  dW (+)= dz^T s     K = M: both operands run across K
//     bias     db (+)= sum_m dz
// One kernel, k_product, computes C[m][n] = sum_k A(m, k) B(n, k) in 128 x 128 tiles for operands of either direction.

#include <hip/hip_runtime.h>

#include <algorithm>

#include "common.h"
#include "dma.h"
#include "internal.h"
#include "mfma.h"

namespace fold {

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 128;            // rows and columns of a workgroup's tile (waves 2 x 2, each 64 x 64)
constexpr int kStage = kTile * 128;   // bytes of one operand's stage: 64 bf16 or 32 fp32 values of K

// what every operand element outside its matrix is read from
__device__ __attribute__((aligned(16))) uint32_t g_zero[4];

// An operand as it lies in memory: `rows` lines of `ld` elements.  kAlong: line i holds element i's K values (and the
// pad columns up to ld are zero or meet zeros); kAcross: line k holds the K value k of every element.
enum { kAlong = 0, kAcross = 1 };
struct Operand {
  const void* p;
  int64_t lines;
  int ld;
};

// A stage in LDS.  kAlong: the row tiles of dma.h (row r's 16-byte unit u in slot 8 r + (u ^ swz(r))).  kAcross: K lines
// of 128 elements; bf16 fragments come from the transposing read, which takes 4 lines x 16 columns at a time, so line
// k's units are permuted by ^ 4 (k & 3) to put the 4 lines into different 64-byte bank ranges; fp32 fragments are one
// dword a lane, the two half waves read lines k and k + 16, whose units are permuted apart by ^ 8.
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4_t;
#define FOLD_LDS_AS __attribute__((address_space(3)))

template <typename T>
__device__ __forceinline__ int across_off(int k, int col) {
  if constexpr (sizeof(T) == 2) return k * 256 + (((col >> 3) ^ (4 * (k & 3))) << 4) + (col & 7) * 2;
  else return k * 512 + (((col >> 2) ^ (8 * ((k >> 4) & 1))) << 4) + (col & 3) * 4;
}

// One wave's loads of an operand's stages (4 instructions a stage).  e0: the tile's first element.
template <typename T, int DIR>
struct Loader {
  const char* base[4];
  int line[4];
  bool in[4];
  int64_t lines;
  size_t step;  // bytes from a stage to the next
  __device__ __forceinline__ Loader(const Operand& o, int64_t e0, int wave, int lane) {
    lines = o.lines;
    const char* p = static_cast<const char*>(o.p);
    const size_t lb = (size_t)o.ld * sizeof(T);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = 4 * wave + i;
      if constexpr (DIR == kAlong) {
        // elements behind the last are computed from the last one's values and never stored
        const int64_t e = min(e0 + 8 * t + row_of_lane(lane), o.lines - 1);
        base[i] = p + (size_t)e * lb + unit_of_lane(lane, t) * 16;
        line[i] = 0;
        in[i] = true;
        step = 128;
      } else if constexpr (sizeof(T) == 2) {
        line[i] = 4 * t + (lane >> 4);
        const int64_t col = e0 + 8 * ((lane & 15) ^ (4 * (line[i] & 3)));
        in[i] = col < o.ld;
        base[i] = p + (size_t)line[i] * lb + (size_t)col * 2;
        step = 64 * lb;
      } else {
        line[i] = 2 * t + (lane >> 5);
        const int64_t col = e0 + 4 * ((lane & 31) ^ (8 * ((line[i] >> 4) & 1)));
        in[i] = col < o.ld;
        base[i] = p + (size_t)line[i] * lb + (size_t)col * 4;
        step = 32 * lb;
      }
    }
  }
  __device__ __forceinline__ void issue(int64_t c, int wave, char* lds) const {
    constexpr int kLines = 128 / sizeof(T);  // K values of a stage
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const char* src = base[i] + (size_t)c * step;
      if constexpr (DIR == kAcross)
        src = in[i] && c * kLines + line[i] < lines ? src : reinterpret_cast<const char*>(g_zero);
      dma16(src, lds + (4 * wave + i) * 1024);
    }
  }
};

// The fragment of 32 elements from e0 of step s: bf16 K = 16 s + 8 (lane / 32) + 0 .. 7 (s < 4); fp32, four K values in
// one, K = 4 s + 16 (lane / 32) + 0 .. 3 (s < 4).
template <typename T, int DIR>
__device__ __forceinline__ uint4 fragment(const char* lds, int e0, int s, int lane) {
  const int h = lane >> 5, l32 = lane & 31;
  if constexpr (DIR == kAlong) {
    return *reinterpret_cast<const uint4*>(lds + rt_off(e0 + l32, sizeof(T) == 2 ? 2 * s + h : 4 * h + s));
  } else if constexpr (sizeof(T) == 2) {
    const int g = lane >> 4, gi = lane & 15;
    const int col = e0 + 16 * (g & 1) + 4 * (gi & 3), k = 16 * s + 8 * (g >> 1) + (gi >> 2);
    const bf16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((FOLD_LDS_AS bf16x4_t*)(lds + across_off<T>(k, col)));
    const bf16x4_t hi =
        __builtin_amdgcn_ds_read_tr16_b64_v4bf16((FOLD_LDS_AS bf16x4_t*)(lds + across_off<T>(k + 4, col)));
    const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
    return make_uint4(a.x, a.y, b.x, b.y);
  } else {
    uint4 r;
    uint32_t* w = &r.x;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w[e] = *reinterpret_cast<const uint32_t*>(lds + across_off<T>(4 * s + 16 * h + e, e0 + l32));
    return r;
  }
}

template <typename T, int AD, int BD>
__device__ __forceinline__ void product_stage(const char* As, const char* Bs, f32x16 (&acc)[2][2], int a0, int b0,
                                              int lane) {
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    uint4 a[2], b[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) a[i] = fragment<T, AD>(As, a0 + 32 * i, s, lane);
#pragma unroll
    for (int i = 0; i < 2; ++i) b[i] = fragment<T, BD>(Bs, b0 + 32 * i, s, lane);
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a[i]),
                                                              __builtin_bit_cast(bf16x8, b[j]), acc[i][j], 0, 0, 0);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float((&a[i].x)[e]),
                                                             __uint_as_float((&b[j].x)[e]), acc[i][j], 0, 0, 0);
    }
  }
}

struct ProductArgs {
  Operand a, b;
  int64_t M, N;       // elements of either operand
  int64_t mt, nt;     // tiles
  int nstage, split;  // stages of K, and the pieces they are cut into
  void* out;
  size_t ld;
  int64_t cols;       // columns of out that are written (pad columns up to it as zero)
  const float* bias;  // [N] or NULL
  int add;            // out += C, the pad columns left alone
};

// OUT: the element type of out; partial sums of a split go to out + piece * M * ld
template <typename T, int AD, int BD, typename OUT>
__global__ __launch_bounds__(kThreads) void k_product(ProductArgs g) {
  __shared__ __attribute__((aligned(16))) char A0[kStage], A1[kStage], B0[kStage], B1[kStage];
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const int wm = wave & 1, wn = wave >> 1;
  const int64_t tile = blockIdx.x / g.split;
  const int piece = (int)(blockIdx.x % g.split);
  const int64_t m0 = tile % g.mt * kTile, n0 = tile / g.mt * kTile;
  const int per = (g.nstage + g.split - 1) / g.split;
  const int c0 = min(piece * per, g.nstage), c1 = min(c0 + per, g.nstage);
  const Loader<T, AD> la(g.a, m0, wave, lane);
  const Loader<T, BD> lb(g.b, n0, wave, lane);
  f32x16 acc[2][2];
  zero_acc(acc);
  auto issue = [&](int c, char* A, char* B) {
    la.issue(c, wave, A);
    lb.issue(c, wave, B);
  };
  if (c0 < c1) {
    issue(c0, A0, B0);
    vm_wait();
    __syncthreads();
    int c = c0;
    for (; c + 2 <= c1; c += 2) {
      issue(c + 1, A1, B1);
      __builtin_amdgcn_sched_barrier(0);
      product_stage<T, AD, BD>(A0, B0, acc, wm * 64, wn * 64, lane);
      vm_wait();
      __syncthreads();
      if (c + 2 < c1) issue(c + 2, A0, B0);
      __builtin_amdgcn_sched_barrier(0);
      product_stage<T, AD, BD>(A1, B1, acc, wm * 64, wn * 64, lane);
      vm_wait();
      __syncthreads();
    }
    if (c < c1) product_stage<T, AD, BD>(A0, B0, acc, wm * 64, wn * 64, lane);
  }
  OUT* out = static_cast<OUT*>(g.out) + (size_t)piece * g.M * g.ld;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int64_t n = n0 + wn * 64 + j * 32 + (lane & 31);
    if (n >= g.cols || (g.add && n >= g.N)) continue;
    const float b = g.bias && n < g.N ? g.bias[n] : 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int64_t m = m0 + wm * 64 + i * 32 + acc_row(r, lane);
        if (m >= g.M) continue;
        OUT* o = out + (size_t)m * g.ld + n;
        float v = n < g.N ? acc[i][j][r] + b : 0.f;
        if constexpr (sizeof(OUT) == 4) v += g.add ? *o : 0.f;
        *o = from_f32<OUT>(v);
      }
  }
}

// out (+)= the sum of the pieces, in their order
__global__ __launch_bounds__(256) void k_join(const float* part, int pieces, size_t n, float* out) {
  const size_t step = (size_t)gridDim.x * 256 * 4;
  for (size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += step) {
    float4 s = *reinterpret_cast<const float4*>(part + i);
    for (int p = 1; p < pieces; ++p) {
      const float4 v = *reinterpret_cast<const float4*>(part + (size_t)p * n + i);
      s.x += v.x;
      s.y += v.y;
      s.z += v.z;
      s.w += v.w;
    }
    *reinterpret_cast<float4*>(out + i) = s;
  }
}

// db: sums over the rows, a workgroup per 64 columns; its four waves take every fourth row
template <typename T>
__global__ __launch_bounds__(256) void k_column_sums(const T* dz, int64_t M, int V, size_t ld, float* db, int add) {
  __shared__ float red[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = blockIdx.x * 64 + lane;
  float s = 0.f;
  for (int64_t m = wave; m < M; m += 4) s += to_f32<T>(dz[(size_t)m * ld + col]);
  red[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && col < V) {
    s = (red[0][lane] + red[1][lane]) + (red[2][lane] + red[3][lane]);
    db[col] = add ? db[col] + s : s;
  }
}

int64_t tiles(int64_t n) { return (n + kTile - 1) / kTile; }

// Pieces of K for the states' gradient: few tiles with a long K are cut until the chip has two workgroups a compute
// unit, each with at least 8 stages.
int split_of(int64_t M, int H, int V, int esize) {
  const int64_t t = std::max<int64_t>(1, tiles(M) * tiles(row_ld(H)));
  const int64_t nst = ((int64_t)row_ld(V) * esize + 127) / 128;
  return (int)std::max<int64_t>(1, std::min<int64_t>({512 / t, nst / 8, 64}));
}

template <typename T, int AD, int BD, typename OUT>
void launch(const ProductArgs& g, hipStream_t st) {
  hipLaunchKernelGGL((k_product<T, AD, BD, OUT>), dim3((unsigned)(g.mt * g.nt * g.split)), dim3(kThreads), 0, st, g);
}

}  // namespace

int64_t vocab_tiles(int64_t M, int H, int V) {
  const int64_t h = tiles(row_ld(H)), v = tiles(row_ld(V)), m = std::max<int64_t>(tiles(M), 1);
  return std::max(m * v, std::max(v * h, m * h * 64));
}

void launch_vocab_logits(int dtype, int64_t M, int H, int V, const void* s, const void* W, const float* bias,
                         int out_dtype, void* z, hipStream_t st) {
  if (M <= 0) return;
  ProfScope prof("vocab_logits", st);
  const int es = dtype == FOLD_BF16 ? 2 : 4, ldh = row_ld(H), ldv = row_ld(V);
  ProductArgs g{{s, M, ldh}, {W, V, ldh}, M, V, tiles(M), tiles(ldv), ldh * es / 128, 1, z, (size_t)ldv, ldv, bias, 0};
  if (dtype == FOLD_F32) launch<float, kAlong, kAlong, float>(g, st);
  else if (out_dtype == FOLD_F32) launch<uint16_t, kAlong, kAlong, float>(g, st);
  else launch<uint16_t, kAlong, kAlong, uint16_t>(g, st);
}

size_t vocab_backward_bytes(int dtype, int64_t M, int H, int V) {
  const int n = split_of(M, H, V, dtype == FOLD_BF16 ? 2 : 4);
  return n == 1 ? 0 : (size_t)n * M * row_ld(H) * sizeof(float);
}

void launch_vocab_backward(int dtype, int64_t M, int H, int V, const void* s, const void* W, const void* dz, float* ds,
                           float* dW, float* db, int add, void* ws, hipStream_t st) {
  const int es = dtype == FOLD_BF16 ? 2 : 4, ldh = row_ld(H), ldv = row_ld(V);
  const int kst = 128 / es;
  if (ds && M > 0) {
    ProfScope prof("vocab_dstates", st);
    const int n = split_of(M, H, V, es);
    ProductArgs g{{dz, M, ldv}, {W, V, ldh}, M, H, tiles(M), tiles(ldh), ldv * es / 128, n,
                  n > 1 ? ws : ds, (size_t)ldh, ldh, nullptr, 0};
    if (dtype == FOLD_F32) launch<float, kAlong, kAcross, float>(g, st);
    else launch<uint16_t, kAlong, kAcross, float>(g, st);
    if (n > 1) {
      const size_t total = (size_t)M * ldh;
      hipLaunchKernelGGL(k_join, dim3((unsigned)std::min<size_t>((total + 1023) / 1024, 4096)), dim3(256), 0, st,
                         static_cast<const float*>(ws), n, total, ds);
    }
  }
  if (dW) {
    ProfScope prof("vocab_dweights", st);
    ProductArgs g{{dz, M, ldv}, {s, M, ldh}, V, H, tiles(V), tiles(ldh), (int)((M + kst - 1) / kst), 1,
                  dW, (size_t)ldh, ldh, nullptr, add};
    if (dtype == FOLD_F32) launch<float, kAcross, kAcross, float>(g, st);
    else launch<uint16_t, kAcross, kAcross, float>(g, st);
  }
  if (db) {
    ProfScope prof("vocab_dbias", st);
    const dim3 grid((unsigned)(ldv / 64));
    if (dtype == FOLD_F32)
      hipLaunchKernelGGL(k_column_sums<float>, grid, dim3(256), 0, st, static_cast<const float*>(dz), M, V,
                         (size_t)ldv, db, add);
    else
      hipLaunchKernelGGL(k_column_sums<uint16_t>, grid, dim3(256), 0, st, static_cast<const uint16_t*>(dz), M, V,
                         (size_t)ldv, db, add);
  }
}

}  // namespace fold
