// Products of the vocabulary head on the matrix cores (gfx950):
//     logits   z = s W^T + b      s [M, H] states, W [V, H]: both operands run along K = H
//     states   ds = dz W          K = V: dz runs along K, W across it
//     weights  dW (+)= dz^T s     K = M: both operands run across K
//     bias     db (+)= sum_m dz
// One loop, product(), computes C[m][n] = sum_k A(m, k) B(n, k) for operands of either direction.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>

#include "common.h"
#include "dma.h"
#include "internal.h"
#include "mfma.h"
#include "wide.h"

namespace fold {

namespace {

constexpr int kThreads = 256;  // four waves, 2 x 2, each 32 WM rows x 32 WN columns of the tile

// what the K values past an operand's last line are read from
__device__ __attribute__((aligned(16))) uint32_t g_zero[4];

// An operand as it lies in memory: `lines` lines of `ld` elements.  kAlong: line i holds element i's K values (and the
// pad columns up to ld are zero or meet zeros); kAcross: line k holds the K value k of every element.
enum { kAlong = 0, kAcross = 1 };
struct Operand {
  const void* p;
  int64_t lines;
  int ld;
};

// A stage is KB bytes of K, 128 or 64: NS = KB / 32 steps of 16 bf16 or 8 fp32 values.  In LDS, kAlong: KB bytes an
// element, the 16-byte units permuted as in dma.h (128) or wide.h (64) so that 16 neighbouring elements' units fall in 16
// bank groups.  kAcross: lines of ELEMS elements; bf16 fragments come from the transposing read, which takes 4 lines x 16
// columns at a time, so line k's units are permuted by ^ 4 (k & 3) to put the 4 lines into different 64-byte bank ranges;
// fp32 fragments are one dword a lane, the two half waves read lines k and k + 4 NS, whose units are permuted apart by
// ^ 8.
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4_t;
#define FOLD_LDS_AS __attribute__((address_space(3)))

template <typename T, int ELEMS, int NS>
__device__ __forceinline__ int across_unit(int k, int u) {
  return u ^ (sizeof(T) == 2 ? 4 * (k & 3) % (ELEMS / 8) : 8 * ((k / (4 * NS)) & 1));
}
template <typename T, int ELEMS, int NS>
__device__ __forceinline__ int across_off(int k, int col) {
  constexpr int VEC = 16 / (int)sizeof(T);
  return k * (ELEMS * (int)sizeof(T)) + across_unit<T, ELEMS, NS>(k, col / VEC) * 16 + col % VEC * (int)sizeof(T);
}
template <int KB>
__device__ __forceinline__ int along_off(int r, int u) {
  return KB == 128 ? rt_off(r, u) : wide::off(r, u);
}

// lane l of the wave copies 16 bytes from base + off (its own offset) to lds + 16 l; not tracked by the compiler (see
// dma16_untracked)
__device__ __forceinline__ void dma16_at(const char* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
// the same with 4 bytes a lane, from its own address
__device__ __forceinline__ void dma4_at(const float* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(src) : "memory", "m0");
}
template <typename P>
__device__ __forceinline__ uint32_t lds_of(const P* p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(const FOLD_LDS_AS char*)reinterpret_cast<const char*>(p));
}

// One wave's loads of an operand's stages: NI instructions of 1 KB a stage, instruction t of the workgroup (NI a wave).
// e0: the tile's first element.  Elements past the operand's last one are read from a clamped place: they reach results
// that are not stored.
template <typename T, int DIR, int ELEMS, int KB>
struct Loader {
  static constexpr int NI = ELEMS * KB / 4096;
  static constexpr int LINES = KB / (int)sizeof(T);  // K values of a stage
  static constexpr int LL = ELEMS * sizeof(T) / 16;  // lanes of a line (kAcross)
  const char* p;      // the tile's corner at K = 0
  int64_t lines;
  size_t step;        // bytes from a stage to the next
  uint32_t off[NI];
  int line0;
  __device__ __forceinline__ Loader(const Operand& o, int64_t e0, int wave, int lane) {
    lines = o.lines;
    const size_t lb = (size_t)o.ld * sizeof(T);
    p = static_cast<const char*>(o.p) + (DIR == kAlong ? (size_t)e0 * lb : (size_t)e0 * sizeof(T));
    step = DIR == kAlong ? (size_t)KB : LINES * lb;
    line0 = wave * NI * (64 / LL) + lane / LL;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int t = wave * NI + i;
      if constexpr (DIR == kAlong) {
        const int r = KB == 128 ? 8 * t + row_of_lane(lane) : 16 * t + wide::lane_row(lane);
        const int u = KB == 128 ? unit_of_lane(lane, t) : wide::lane_unit(lane);
        const int64_t e = min(e0 + r, o.lines - 1) - e0;
        off[i] = (uint32_t)(e * (int64_t)lb) + u * 16;
      } else {
        const int line = t * (64 / LL) + lane / LL;
        const int u = across_unit<T, ELEMS, KB / 32>(line, lane % LL);
        const int64_t col = min(e0 + u * (int)(16 / sizeof(T)), (int64_t)o.ld - (int)(16 / sizeof(T))) - e0;
        off[i] = (uint32_t)(line * (int64_t)lb + col * (int64_t)sizeof(T));
      }
    }
  }
  // the stages whose lines are all there
  __device__ __forceinline__ int64_t whole() const { return DIR == kAlong ? INT64_MAX : lines / LINES; }
  __device__ __forceinline__ void issue(int64_t c, int wave, uint32_t lds) const {
    const char* src = p + (size_t)c * step;
    if (c < whole()) {
#pragma unroll
      for (int i = 0; i < NI; ++i) dma16_at(src, off[i], lds + (wave * NI + i) * 1024);
    } else {  // the last lines: zeros behind them
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const bool in = c * (int64_t)LINES + line0 + i * (64 / LL) < lines;
        const char* at = in ? src + off[i] : reinterpret_cast<const char*>(g_zero);
        asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds + (wave * NI + i) * 1024), "v"(at)
                     : "memory", "m0");
      }
    }
  }
};

// The fragment of 32 elements from e0 of step s < NS: bf16 K = 16 s + 8 (lane / 32) + 0 .. 7; fp32, four K values in one,
// K = 4 s + 4 NS (lane / 32) + 0 .. 3.
template <typename T, int DIR, int ELEMS, int KB>
__device__ __forceinline__ uint4 fragment(const char* lds, int e0, int s, int lane) {
  constexpr int NS = KB / 32;
  const int h = lane >> 5, l32 = lane & 31;
  if constexpr (DIR == kAlong) {
    return *reinterpret_cast<const uint4*>(lds + along_off<KB>(e0 + l32, sizeof(T) == 2 ? 2 * s + h : NS * h + s));
  } else if constexpr (sizeof(T) == 2) {
    const int g = lane >> 4, gi = lane & 15;
    const int col = e0 + 16 * (g & 1) + 4 * (gi & 3), k = 16 * s + 8 * (g >> 1) + (gi >> 2);
    const bf16x4_t lo =
        __builtin_amdgcn_ds_read_tr16_b64_v4bf16((FOLD_LDS_AS bf16x4_t*)(lds + across_off<T, ELEMS, NS>(k, col)));
    const bf16x4_t hi =
        __builtin_amdgcn_ds_read_tr16_b64_v4bf16((FOLD_LDS_AS bf16x4_t*)(lds + across_off<T, ELEMS, NS>(k + 4, col)));
    const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
    return make_uint4(a.x, a.y, b.x, b.y);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w[e] = *reinterpret_cast<const uint32_t*>(lds + across_off<T, ELEMS, NS>(4 * s + 4 * NS * h + e, e0 + l32));
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}

__device__ __forceinline__ float word(const uint4& v, int e) {
  return __uint_as_float(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w);
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
  float* sums;        // [M] (+)= the sums over K of A's elements, or NULL; A across, all of K loaded before the loop, no pieces
};

// a value that is the same in all lanes, on the scalar unit (divisions leave it)
__device__ __forceinline__ unsigned uniform(unsigned v) { return __builtin_amdgcn_readfirstlane(v); }

// Tiles go to the XCDs in runs, each run walking groups of 8 tile rows column by column: the workgroups that an XCD has
// at once then share their operands' stages in its L2 (32 of them: 8 x 4 tiles).
// (In 32 bits: a launch has fewer than 2^24 tiles.)
__device__ __forceinline__ void tile_at(const ProductArgs& g, unsigned t, unsigned& mt, unsigned& nt) {
  const unsigned whole = 8 * (unsigned)g.nt, group = uniform(t / whole), in = t - group * whole;
  const unsigned rows = min(8u, (unsigned)g.mt - 8 * group);
  nt = uniform(in / rows);
  mt = 8 * group + (in - nt * rows);
}
__device__ __forceinline__ bool tile_of(const ProductArgs& g, unsigned block, unsigned& mt, unsigned& nt,
                                        unsigned& piece) {
  const unsigned one = (unsigned)g.mt * (unsigned)g.nt, total = one * (unsigned)g.split, per = (total + 7) >> 3;
  const unsigned slot = block >> 3, at = (block & 7) * per + slot;
  if (slot >= per || at >= total) return false;
  piece = uniform(at / one);
  tile_at(g, at - piece * one, mt, nt);
  return true;
}

template <typename OUT>
__device__ __forceinline__ OUT* out_of(const ProductArgs& g, unsigned piece) {
  return static_cast<OUT*>(g.out) + (size_t)piece * g.M * g.ld;
}
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {  // rounded to nearest even, one instruction
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), bf16x2_t));
}

// The accumulators start from the bias of their columns (LDS, 32 WN of them): C's columns are on the accumulators' rows, so
// register 4 q + e of lane l is column 8 q + 4 (l / 32) + e of row l % 32.
template <int WM, int WN>
__device__ __forceinline__ void start_acc(f32x16 (&acc)[WM][WN], const float* bias, int lane) {
#pragma unroll
  for (int j = 0; j < WN; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float4 b = *reinterpret_cast<const float4*>(bias + 32 * j + 8 * q + 4 * (lane >> 5));
#pragma unroll
      for (int i = 0; i < WM; ++i) {
        acc[i][j][4 * q] = b.x;
        acc[i][j][4 * q + 1] = b.y;
        acc[i][j][4 * q + 2] = b.z;
        acc[i][j][4 * q + 3] = b.w;
      }
    }
}

// what a wave's lanes have written to LDS is there for its other lanes (LDS keeps a wave's order: nothing to wait for)
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_sched_barrier(0);
}

// One wave's part of a tile, WM x WN accumulators from row m0, column n0, to out, through images in LDS of 32 rows by 128
// bytes (rows 16 bytes apart in their banks), so that an instruction stores eight rows' whole lines.  Stored from the
// registers, 32 rows by 32 bytes, logits whose rows are a power of two apart queued in a few of the memory's channels:
// 8,192 x 32,768 bf16 at H = 1,024 took 980 us, at a vocabulary of 32,000 530 us.  For bf16 the half waves swap first: two
// neighbouring groups of 8 columns, 4 in either half, become 8 columns of one group a lane.  WHOLE: the part lies inside
// the matrix.
constexpr int kImageRow = 128 + 16, kImage = 32 * kImageRow;

template <typename OUT, int WM, int WN, bool WHOLE>
__device__ __forceinline__ void store_part(const ProductArgs& g, OUT* out, const f32x16 (&acc)[WM][WN], int rows, int vals,
                                           int cols, char* img, int lane) {
  constexpr int VEC = 16 / (int)sizeof(OUT), COLS = 128 / (int)sizeof(OUT), JG = COLS / 32 < WN ? COLS / 32 : WN;
  constexpr int LPR = 32 * JG / VEC;  // lanes of a row of the image
  const int h = lane >> 5, l32 = lane & 31;
#pragma unroll
  for (int i = 0; i < WM; ++i)
#pragma unroll
    for (int j0 = 0; j0 < WN; j0 += JG) {
#pragma unroll
      for (int j = j0; j < j0 + JG; ++j) {
        f32x16 c = acc[i][j];
        if constexpr (WM * WN >= 16) asm volatile("" : "+a"(c));  // stays in its accumulator registers until here
#pragma unroll
        for (int q = 0; q < 4; q += VEC / 4) {
          uint4 v;
          int n;
          if constexpr (sizeof(OUT) == 4) {
            n = 32 * (j - j0) + 8 * q + 4 * h;
            v = make_uint4(__float_as_uint(c[4 * q]), __float_as_uint(c[4 * q + 1]), __float_as_uint(c[4 * q + 2]),
                           __float_as_uint(c[4 * q + 3]));
          } else {
            n = 32 * (j - j0) + 8 * (q + h);
            const auto lo = __builtin_amdgcn_permlane32_swap(bf16_pair(c[4 * q], c[4 * q + 1]),
                                                             bf16_pair(c[4 * q + 4], c[4 * q + 5]), false, false);
            const auto hi = __builtin_amdgcn_permlane32_swap(bf16_pair(c[4 * q + 2], c[4 * q + 3]),
                                                             bf16_pair(c[4 * q + 6], c[4 * q + 7]), false, false);
            v = make_uint4(lo[0], hi[0], lo[1], hi[1]);
          }
          *reinterpret_cast<uint4*>(img + l32 * kImageRow + n * (int)sizeof(OUT)) = v;
        }
      }
      wave_fence();
#pragma unroll
      for (int x = 0; x < 32 * LPR / 64; ++x) {
        const int row = x * (64 / LPR) + lane / LPR, col = lane % LPR * VEC, n = 32 * j0 + col;
        uint4 v = *reinterpret_cast<const uint4*>(img + row * kImageRow + col * (int)sizeof(OUT));
        if constexpr (!WHOLE) {
          if (32 * i + row >= rows || n >= cols) continue;
          v = mask_tail<OUT>(v, max(vals - n, 0));
        }
        OUT* o = out + (size_t)(32 * i + row) * g.ld + n;
        if constexpr (sizeof(OUT) == 4) {
          if (g.add) {  // + 0 in the pad columns
            const float4 old = *reinterpret_cast<const float4*>(o);
            v.x = __float_as_uint(old.x + __uint_as_float(v.x));
            v.y = __float_as_uint(old.y + __uint_as_float(v.y));
            v.z = __float_as_uint(old.z + __uint_as_float(v.z));
            v.w = __float_as_uint(old.w + __uint_as_float(v.w));
          }
        }
        *reinterpret_cast<uint4*>(o) = v;
      }
      wave_fence();
    }
}

template <typename OUT, int WM, int WN>
__device__ __forceinline__ void store_tile(const ProductArgs& g, OUT* out, const f32x16 (&acc)[WM][WN], int64_t m0,
                                           int64_t n0, char* img, int lane) {
  // what of the part exists: rows, columns with a value, columns that are written
  const int rows = (int)min(g.M - m0, (int64_t)(32 * WM)), vals = (int)min(g.N - n0, (int64_t)(32 * WN));
  const int cols = (int)min(g.cols - n0, (int64_t)(32 * WN));
  out += (size_t)m0 * g.ld + n0;
  if (rows == 32 * WM && vals == 32 * WN) store_part<OUT, WM, WN, true>(g, out, acc, rows, vals, cols, img, lane);
  else store_part<OUT, WM, WN, false>(g, out, acc, rows, vals, cols, img, lane);
}

// One stage of the K loop: NS steps of MULS multiplications, placed one by one with what runs beside them.
//   load(s, f)   reads fragment f of the step after s (of the next stage after the last step)
//   meet()       the workgroup meets: everybody has read its fragments of this stage, the next stage has landed
//   put(d)       starts load d of a new stage
// The fragments are spread over a step, so that four waves' reads do not queue in LDS, the first needed first; the new
// stage's loads go out in the first step, into the slot that the last meeting freed (SLOTS > 2), or behind the meeting into
// this stage's own slot (SLOTS = 2).  A meeting follows the first multiplications of its step, which need the fragments
// read last.
template <int MULS, int FRAGS, int LOADS, int NS, int SLOTS, class MUL, class LOAD, class MEET, class PUT>
__device__ __forceinline__ void pipeline_stage(MUL&& multiply, LOAD&& load, MEET&& meet, PUT&& put) {
  constexpr int K = MULS < 16 ? MULS : 16, EACH = MULS / K;  // places of a step, multiplications of each
  constexpr int MEETING = K == 16 ? 4 : 0;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const bool last = s == NS - 1, loads = SLOTS > 2 ? s == 0 : last;
    const int from = last ? MEETING : 0, pfrom = SLOTS > 2 ? 0 : MEETING;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (last && k == MEETING) meet();
#pragma unroll
      for (int e = 0; e < EACH; ++e) multiply(s & 1, k * EACH + e);
#pragma unroll
      for (int f = 0; f < FRAGS; ++f)
        if (from + f * (K - from) / FRAGS == k) load(s, f);
#pragma unroll
      for (int d = 0; d < LOADS; ++d)
        if (loads && pfrom + (2 * d + 1) * (K - pfrom) / (2 * LOADS) == k) put(d);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// OUT: the element type of out; partial sums of a split go to out + piece * M * ld.
// The K loop keeps SLOTS stages in LDS and the fragments of two steps (16 bytes of K a lane) in registers: a step's
// multiplications run while the next step's fragments are read.
// block: this workgroup's place among the product's.
template <int WM, int WN, int KB, int SLOTS>
struct ProductLds {
  char stages[SLOTS * 64 * (WM + WN) * KB];
  float bias[64 * WN];
};
template <typename T, int AD, int BD, typename OUT, int WM, int WN, int KB, int SLOTS>
__device__ __forceinline__ void product(const ProductArgs& g, unsigned block, ProductLds<WM, WN, KB, SLOTS>& shared) {
  constexpr int EA = 64 * WM, EB = 64 * WN, STAGE = (EA + EB) * KB, NS = KB / 32;
  using LA = Loader<T, AD, EA, KB>;
  using LB = Loader<T, BD, EB, KB>;
  char* lds = shared.stages;
  float* bias = shared.bias;
  static_assert(EB <= kThreads, "one bias a thread");
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const int wm = wave & 1, wn = wave >> 1;
  unsigned mt, nt, piece;
  if (!tile_of(g, block, mt, nt, piece)) return;
  const int64_t m0 = (int64_t)mt * EA, n0 = (int64_t)nt * EB;
  const int per = (g.nstage + g.split - 1) / g.split;
  const int c0 = min((int)piece * per, g.nstage), c1 = min(c0 + per, g.nstage);
  const LA la(g.a, m0, wave, lane);
  const LB lb(g.b, n0, wave, lane);
  const uint32_t base = lds_of(lds);
  const bool sums = AD == kAcross && g.sums && nt == 0;  // column tid % EA of the tile, every kThreads / EA-th line
  float sum = 0.f;
  f32x16 acc[WM][WN];
  if (tid < EB) bias[tid] = g.bias && n0 + tid < g.N ? g.bias[n0 + tid] : 0.f;
  auto issue = [&](int c) {
    const uint32_t to = base + (c - c0) % SLOTS * STAGE;
    la.issue(c, wave, to);
    lb.issue(c, wave, to + EA * KB);
  };
  uint4 fa[2][WM], fb[2][WN];
  // the f-th fragment of step s of a slot into register set `set`
  auto load = [&](const char* slot, int s, int set, int f) {  // in the order of their first use
    const int i = f == 0 ? 0 : f - WN, j = f - 1;
    if (f == 0 || f > WN) fa[set][i] = fragment<T, AD, EA, KB>(slot, (wm * WM + i) * 32, s, lane);
    else fb[set][j] = fragment<T, BD, EB, KB>(slot + EA * KB, (wn * WN + j) * 32, s, lane);
  };
  // the k-th multiplication of a step.  C's columns are on the accumulators' rows: a lane holds four neighbouring
  // columns of one row of C
  constexpr int FRAGS = WM + WN, MULS = WM * WN * (sizeof(T) == 2 ? 1 : 4), LOADS = LA::NI + LB::NI;
  constexpr int AHEAD = SLOTS > 2 ? SLOTS - 1 : SLOTS;  // stages loaded before the loop, and ahead in it
  auto multiply = [&](int set, int k) {
    const int e = k / (WM * WN), i = k / WN % WM, j = k % WN;
    if constexpr (sizeof(T) == 2)
      acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fb[set][j]),
                                                          __builtin_bit_cast(bf16x8, fa[set][i]), acc[i][j], 0, 0, 0);
    else
      acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(word(fb[set][j], e), word(fa[set][i], e), acc[i][j], 0, 0, 0);
  };
  // waits until stage c is in LDS: at most the loads of the stages after it, of those that were issued, are outstanding
  static_assert(SLOTS == 2 || SLOTS == 4, "the waits below");
  auto landed = [&](int c, int issued) {
    const int behind = issued - 1 - c;
    if (SLOTS == 4 && behind >= 3) vm_wait_n<3 * LOADS>();
    else if (SLOTS == 4 && behind == 2) vm_wait_n<2 * LOADS>();
    else if (behind == 1) vm_wait_n<LOADS>();
    else vm_wait();
  };
  if (c0 == c1) {
    __syncthreads();
    start_acc(acc, bias + wn * 32 * WN, lane);
  } else {
    int issued = min(c0 + AHEAD, c1);
    for (int c = c0; c < issued; ++c) issue(c);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the bias
    landed(c0, issued);
    wg_barrier();
    start_acc(acc, bias + wn * 32 * WN, lane);
#pragma unroll
    for (int f = 0; f < FRAGS; ++f) load(lds, 0, 0, f);
    int c = c0;
    // the stages that start the load of a whole stage
    const int cw = (int)min((int64_t)c1, min(la.whole(), lb.whole())) - AHEAD;
    const char *pa = la.p + (size_t)(c0 + AHEAD) * la.step, *pb = lb.p + (size_t)(c0 + AHEAD) * lb.step;
    for (; c < cw; ++c) {
      const int at = (c - c0) % SLOTS * STAGE, next = (c + 1 - c0) % SLOTS * STAGE;
      const uint32_t to = base + (c - c0 + AHEAD) % SLOTS * STAGE;
      pipeline_stage<MULS, FRAGS, LOADS, NS, SLOTS>(
          multiply, [&](int s, int f) { load(lds + (s < NS - 1 ? at : next), (s + 1) % NS, (s + 1) & 1, f); },
          [&]() {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((SLOTS - 2) * LOADS) : "memory");
            wg_barrier();
          },
          [&](int d) {
            if (d < LA::NI) dma16_at(pa, la.off[d], to + (wave * LA::NI + d) * 1024);
            else dma16_at(pb, lb.off[d - LA::NI], to + EA * KB + (wave * LB::NI + d - LA::NI) * 1024);
          });
      pa += la.step;
      pb += lb.step;
    }
    issued = max(issued, min(c + AHEAD, c1));
    for (; c < c1; ++c) {
      const char *at = lds + (c - c0) % SLOTS * STAGE, *next = lds + (c + 1 - c0) % SLOTS * STAGE;
      if (SLOTS > 2 && issued < c1) issue(issued++);
      if constexpr (AD == kAcross)
        if (sums)
#pragma unroll 8
          for (int k = tid / EA; k < KB / (int)sizeof(T); k += kThreads / EA)
            sum += to_f32<T>(*reinterpret_cast<const T*>(at + across_off<T, EA, NS>(k, tid % EA)));
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        if (s == NS - 1 && c + 1 < c1) {
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          landed(c + 1, issued);
          wg_barrier();
          if (SLOTS == 2 && issued < c1) issue(issued++);
        }
        if (s < NS - 1 || c + 1 < c1)
#pragma unroll
          for (int f = 0; f < FRAGS; ++f) load(s < NS - 1 ? at : next, (s + 1) % NS, (s + 1) & 1, f);
#pragma unroll
        for (int k = 0; k < MULS; ++k) multiply(s & 1, k);
      }
    }
  }
  static_assert(SLOTS * STAGE >= 4 * kImage + kThreads * 4, "the images and sums lie where the stages were");
  __syncthreads();
  if constexpr (AD == kAcross)
    if (sums) {
      float* red = reinterpret_cast<float*>(lds + 4 * kImage);
      red[tid] = sum;
      __syncthreads();
      if (tid < EA && m0 + tid < g.M) {
        float t = red[tid];
#pragma unroll
        for (int w = 1; w < kThreads / EA; ++w) t += red[tid + w * EA];
        g.sums[m0 + tid] = g.add ? g.sums[m0 + tid] + t : t;
      }
    }
  store_tile<OUT, WM, WN>(g, out_of<OUT>(g, piece), acc, m0 + wm * 32 * WM, n0 + wn * 32 * WN, lds + wave * kImage, lane);
}

template <typename T, int AD, int BD, typename OUT, int WM, int WN, int KB, int SLOTS>
__global__ __launch_bounds__(kThreads, WM * WN >= 16 ? 1 : 2) void k_product(ProductArgs g) {
  __shared__ __attribute__((aligned(16))) ProductLds<WM, WN, KB, SLOTS> lds;
  product<T, AD, BD, OUT, WM, WN, KB, SLOTS>(g, blockIdx.x, lds);
}

// The states' and the weights' gradient of a small batch in one launch: `first` workgroups (a multiple of 8) for the
// states', the rest for the weights'.  Apart, each leaves most of the chip idle and has a launch's start to itself.
template <typename T>
__global__ __launch_bounds__(kThreads, 2) void k_product_both(ProductArgs states, ProductArgs weights, unsigned first) {
  __shared__ __attribute__((aligned(16))) ProductLds<1, 1, 128, 2> lds;
  if (blockIdx.x < first) product<T, kAlong, kAcross, float, 1, 1, 128, 2>(states, blockIdx.x, lds);
  else product<T, kAcross, kAcross, float, 1, 1, 128, 2>(weights, blockIdx.x - first, lds);
}

// The same product where both operands run along a short K (the logits: K = H) and there are many tiles: a workgroup per
// compute unit walks its tiles, and the stages of all of them are one stream through the slots.  While a tile's last stages
// are multiplied the first of the next tile and its bias are loaded, and they land while the tile is stored, so neither
// the first loads' latency nor the store's is waited for (8,192 x 1,024 x 32,000 bf16: 693 us with a workgroup a tile,
// 490 us so).  Needs at least SLOTS stages.
template <typename T, typename OUT>
__global__ __launch_bounds__(kThreads, 1) void k_product_chain(ProductArgs g) {
  g.add = 0;  // logits are written
  constexpr int WM = 4, WN = 4, KB = 64, SLOTS = 4;
  constexpr int EA = 64 * WM, EB = 64 * WN, STAGE = (EA + EB) * KB, NS = KB / 32;
  using LA = Loader<T, kAlong, EA, KB>;
  using LB = Loader<T, kAlong, EB, KB>;
  __shared__ __attribute__((aligned(16))) char lds[SLOTS * STAGE];
  __shared__ __attribute__((aligned(16))) char image[4 * kImage];
  __shared__ __attribute__((aligned(16))) float bias[2][EB];  // of the tile that is multiplied and of the next
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const int wm = wave & 1, wn = wave >> 1;
  const unsigned total = (unsigned)g.mt * (unsigned)g.nt, per = (total + 7) >> 3;
  const unsigned first = (blockIdx.x & 7) * per, slots = gridDim.x >> 3;
  unsigned slot = blockIdx.x >> 3, mt, nt;
  auto there = [&](unsigned s) { return s < per && first + s < total; };
  if (!there(slot)) return;
  const uint32_t base = lds_of(lds);
  tile_at(g, first + slot, mt, nt);
  int64_t m0 = (int64_t)mt * EA, n0 = (int64_t)nt * EB;
  LA la(g.a, m0, wave, lane);
  LB lb(g.b, n0, wave, lane);
  const int n = g.nstage;
  uint4 fa[2][WM], fb[2][WN];
  auto load = [&](const char* at, int s, int set, int f) {
    const int i = f == 0 ? 0 : f - WN, j = f - 1;
    if (f == 0 || f > WN) fa[set][i] = fragment<T, kAlong, EA, KB>(at, (wm * WM + i) * 32, s, lane);
    else fb[set][j] = fragment<T, kAlong, EB, KB>(at + EA * KB, (wn * WN + j) * 32, s, lane);
  };
  constexpr int FRAGS = WM + WN, MULS = WM * WN * (sizeof(T) == 2 ? 1 : 4), LOADS = LA::NI + LB::NI;
  f32x16 acc[WM][WN];
  auto multiply = [&](int set, int k) {
    const int e = k / (WM * WN), i = k / WN % WM, j = k % WN;
    if constexpr (sizeof(T) == 2)
      acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fb[set][j]),
                                                          __builtin_bit_cast(bf16x8, fa[set][i]), acc[i][j], 0, 0, 0);
    else
      acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(word(fb[set][j], e), word(fa[set][i], e), acc[i][j], 0, 0, 0);
  };
  const char *pa = la.p, *pb = lb.p;
  size_t step = la.step;  // of either operand
  auto put = [&](int d, uint32_t to) {
    if (d < LA::NI) dma16_at(pa, la.off[d], to + (wave * LA::NI + d) * 1024);
    else dma16_at(pb, lb.off[d - LA::NI], to + EA * KB + (wave * LB::NI + d - LA::NI) * 1024);
  };
  // columns that are not there get another one's bias, and are not stored; before a tile's first stage, so that it is there
  // when that is
  auto load_bias = [&](int buf) {
    if (g.bias) dma4_at(g.bias + min(n0 + tid, g.N - 1), lds_of(bias[buf]) + wave * 256);
  };
  if (!g.bias) bias[0][tid] = bias[1][tid] = 0.f;
  load_bias(0);
#pragma unroll
  for (int c = 0; c < SLOTS - 1; ++c) {
#pragma unroll
    for (int d = 0; d < LOADS; ++d) put(d, base + c * STAGE);
    pa += step;
    pb += step;
  }
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((SLOTS - 2) * LOADS) : "memory");
  wg_barrier();
#pragma unroll
  for (int f = 0; f < FRAGS; ++f) load(lds, 0, 0, f);
  // A wait for stage c lets only the loads of later stages be outstanding, and loads and stores are counted together and
  // complete in order.  After a tile that was stored whole, STORES store instructions lie between the loads of the next
  // tile's first stages and what comes later, so the next SLOTS - 2 waits may leave that many more (the counter holds 63).
  constexpr int STORES = WM * WN * 32 * 32 * (int)sizeof(OUT) / 1024;
  constexpr int WAIT = (SLOTS - 2) * LOADS, RELAXED = WAIT + STORES < 63 ? WAIT + STORES : 63;
  bool more = true;
  int loads = n - (SLOTS - 1), at = 0;  // stages still to load of the tile that is loaded; the slot that is read
  int relaxed = 0;
  for (int mine = 0;; mine ^= 1) {
    const int64_t m = m0, nn = n0;  // of the tile that is multiplied
    start_acc(acc, bias[mine] + wn * 32 * WN, lane);
    for (int c = 0; c < n; ++c) {
      if (loads == 0) {
        slot += slots;
        more = there(slot);
        if (more) {
          tile_at(g, first + slot, mt, nt);
          m0 = (int64_t)mt * EA;
          n0 = (int64_t)nt * EB;
          la = LA(g.a, m0, wave, lane);
          lb = LB(g.b, n0, wave, lane);
          pa = la.p;
          pb = lb.p;
          loads = n;
          load_bias(mine ^ 1);
        } else {  // nothing is left: the last stage's place again, which nobody reads
          pa -= step;
          pb -= step;
          step = 0;
          loads = SLOTS + 1;
        }
      }
      --loads;
      const int next = at == (SLOTS - 1) * STAGE ? 0 : at + STAGE;
      const uint32_t to = base + (at == 0 ? (SLOTS - 1) * STAGE : at - STAGE);
      pipeline_stage<MULS, FRAGS, LOADS, NS, SLOTS>(
          multiply, [&](int s, int f) { load(lds + (s < NS - 1 ? at : next), (s + 1) % NS, (s + 1) & 1, f); },
          [&]() {
            if (relaxed > 0) {
              --relaxed;
              asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(RELAXED) : "memory");
            } else {
              asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(WAIT) : "memory");
            }
            wg_barrier();
          },
          [&](int d) { put(d, to); });
      pa += step;
      pb += step;
      at = next;
    }
    store_tile<OUT, WM, WN>(g, static_cast<OUT*>(g.out), acc, m + wm * 32 * WM, nn + wn * 32 * WN, image + wave * kImage,
                            lane);
    if (!more) break;
    relaxed = m + EA <= g.M && nn + EB <= g.N ? SLOTS - 2 : 0;
  }
  vm_wait();  // no load outlives the workgroup's LDS
}

// out = the sum of the pieces, in an order that does not depend on scheduling: G thread groups of a workgroup take every
// G-th piece (eight loads in flight each) of 1,024 / G neighbouring values and meet in LDS.  G = 4 for many pieces, which
// few values are cut into (33 x 320 in 16 pieces: 1.7 us, 11 us with G = 1 and a load at a time), else 1 (8,192 x 1,024 in
// 2 pieces: 15 us, 23 us with G = 4).  VEC: out is 16-byte aligned and n = stride; otherwise n of the pieces' `stride`
// values are written, one by one, and added to out if `add`.
template <bool VEC, int G>
__global__ __launch_bounds__(256) void k_join(const float* part, int pieces, size_t stride, size_t n, float* out,
                                              int add) {
  constexpr int W = 256 / G, U = 8;
  __shared__ float4 red[G][W];
  const int at = threadIdx.x % W, group = threadIdx.x / W;
  const size_t i = ((size_t)blockIdx.x * W + at) * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  auto take = [&](const float4& v, bool in) {  // a piece that is not there adds an exact 0
    s.x += in ? v.x : 0.f;
    s.y += in ? v.y : 0.f;
    s.z += in ? v.z : 0.f;
    s.w += in ? v.w : 0.f;
  };
  if (i < stride) {
    if (G == 1 && pieces <= 2) {
      take(*reinterpret_cast<const float4*>(part + i), true);
      if (pieces == 2) take(*reinterpret_cast<const float4*>(part + stride + i), true);
    } else {
      for (int p0 = group; p0 < pieces; p0 += G * U) {
        float4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          v[u] = *reinterpret_cast<const float4*>(part + (size_t)min(p0 + G * u, pieces - 1) * stride + i);
#pragma unroll
        for (int u = 0; u < U; ++u) take(v[u], p0 + G * u < pieces);
      }
    }
  }
  if constexpr (G > 1) {
    red[group][at] = s;
    __syncthreads();
    if (group == 0)
#pragma unroll
      for (int w = 1; w < G; ++w) take(red[w][at], true);
  }
  if (group != 0 || i >= n) return;
  if constexpr (VEC) {
    *reinterpret_cast<float4*>(out + i) = s;
  } else {
    const float t[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e < n) out[i + e] = add ? out[i + e] + t[e] : t[e];
  }
}

size_t join_blocks(int pieces, size_t stride) { return pieces > 8 ? (stride + 255) / 256 : (stride + 1023) / 1024; }
template <bool VEC>
void join(const float* part, int pieces, size_t stride, size_t n, float* out, int add, hipStream_t st) {
  const dim3 grid((unsigned)join_blocks(pieces, stride));
  if (pieces > 8) hipLaunchKernelGGL((k_join<VEC, 4>), grid, dim3(256), 0, st, part, pieces, stride, n, out, add);
  else hipLaunchKernelGGL((k_join<VEC, 1>), grid, dim3(256), 0, st, part, pieces, stride, n, out, add);
}

// db: column sums.  A workgroup takes 64 16-byte vectors of columns of one of `chunks` pieces of the rows; its four waves
// take every fourth row, eight loads in flight each.  One piece writes db itself, more their sums to part [chunks][ld].
template <typename T>
__global__ __launch_bounds__(256) void k_column_sums(const T* dz, int64_t M, int V, size_t ld, int chunks, float* part,
                                                     float* db, int add) {
  constexpr int VEC = 16 / (int)sizeof(T), U = 8;
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
      uint4 r[U];
#pragma unroll
      for (int u = 0; u < U; ++u) r[u] = *reinterpret_cast<const uint4*>(dz + (size_t)min(m + 4 * u, hi - 1) * ld + col);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool in = m + 4 * u < hi;
        const T* x = reinterpret_cast<const T*>(&r[u]);
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[e] += in ? to_f32<T>(x[e]) : 0.f;
      }
    }
#pragma unroll
  for (int e = 0; e < VEC; ++e) red[wave][lane * VEC + e] = s[e];
  __syncthreads();
  const size_t c0 = (size_t)(blockIdx.x / chunks) * 64 * VEC;
  for (int i = threadIdx.x; i < 64 * VEC; i += 256) {
    if (c0 + i >= ld) break;
    const float t = (red[0][i] + red[1][i]) + (red[2][i] + red[3][i]);
    if (chunks > 1) part[(size_t)chunk * ld + c0 + i] = t;
    else if (c0 + i < (size_t)V) db[c0 + i] = add ? db[c0 + i] + t : t;
  }
}

// pieces of the rows for db: enough workgroups for the chip, each with at least 64 rows
int bias_chunks(int64_t M, int V, int esize) {
  const int64_t groups = ((int64_t)row_ld(V) * esize + 1023) / 1024;
  return (int)std::max<int64_t>(1, std::min<int64_t>({1024 / groups, M / 64, 64}));
}

// How a product is cut: tiles of 64 WM x 64 WN, and K into pieces.
struct Shape {
  int wm, wn, split;
  int64_t mt, nt;
};
int64_t tiles_of(int64_t n, int w) { return (n + 64 * w - 1) / (64 * w); }
constexpr int kPieces = 64;
constexpr int kUnits = 256;  // compute units

// The cut with the least expected time.  A compute unit gets ceil(tiles * pieces / 256) workgroups, whose time goes with
// their area and their share of K; a stage of 64 x 64 takes 0.11 us (bf16) or 0.49 us (fp32) at the rate of the largest
// tiles, and the smaller ones' operands cost more of LDS's bandwidth.  Measured at 8,192 x 1,024 x 32,000 bf16 against
// 256 x 256 tiles: 1.2 times the time for 128 x 128, 1.55 for 64 x 128, 2.2 for 64 x 64; in fp32 (2,048 rows), where the
// matrix cores bound all of them, 1.0, 1.03 and 1.06.  A workgroup's first loads and its store take about 2 us; pieces
// cost their sums' way through memory (4 TB/s) and a second launch (3 us).  What the rule gets (best and worst cut tried):
// states' gradient of 33 x 300 x 20,000 bf16 13 us (335), of 257 x 300 x 20,001 fp32 49 us (4,512), weights' gradient of
// 2,048 x 256 x 10,000 fp32 100 us (486).
// small: the smallest tile's columns / 64 (1 or 2); smallest: that tile alone
Shape shape_of(int64_t M, int64_t N, int64_t nstage, int esize, int small, int pieces, bool smallest = false) {
  static constexpr struct { int wm, wn; double bf16, f32; } kTiles[] = {
      {4, 4, 1.0, 1.0}, {2, 2, 1.2, 1.0}, {1, 2, 1.55, 1.03}, {1, 1, 2.2, 1.06}};
  Shape best{0, 0, 0, 0, 0};
  double least = 0;
  for (const auto& t : kTiles) {
    if ((t.wm == 1 && t.wn != small) || (smallest && t.wm != 1)) continue;
    const int64_t mt = tiles_of(M, t.wm), nt = tiles_of(N, t.wn);
    for (int p = 1; p <= pieces && (p == 1 || nstage / p >= 4); p *= 2) {
      const double rounds = (double)((mt * nt * p + kUnits - 1) / kUnits);
      const double stage = t.wm * t.wn * (esize == 2 ? 0.11 * t.bf16 : 0.49 * t.f32);
      double us = rounds * (stage * (double)((nstage + p - 1) / p) + 2.0 / (t.wm == 4 ? 1 : 2));
      if (p > 1) us += 3.0 + (double)(p + 1) * M * N * 4 / 4e6;
      if (best.wm == 0 || us < least) {
        least = us;
        best = Shape{t.wm, t.wn, p, mt, nt};
      }
    }
  }
  return best;
}
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

unsigned blocks_of(const ProductArgs& g) { return (unsigned)((g.mt * g.nt * g.split + 7) / 8 * 8); }

template <typename T, int AD, int BD, typename OUT>
void launch(ProductArgs g, const Shape& sh, hipStream_t st) {
  const dim3 grid(blocks_of(g));
  if (sh.wm == 4) {
    g.nstage *= 2;
    if constexpr (AD == kAlong && BD == kAlong)
      if (g.nstage >= 4 && g.mt * g.nt > kUnits) {
        hipLaunchKernelGGL((k_product_chain<T, OUT>), dim3(kUnits), dim3(kThreads), 0, st, g);
        return;
      }
    hipLaunchKernelGGL((k_product<T, AD, BD, OUT, 4, 4, 64, 4>), grid, dim3(kThreads), 0, st, g);
  } else if (sh.wm == 2) {
    hipLaunchKernelGGL((k_product<T, AD, BD, OUT, 2, 2, 128, 2>), grid, dim3(kThreads), 0, st, g);
  } else if constexpr (AD == kAlong && BD == kAlong) {
    hipLaunchKernelGGL((k_product<T, AD, BD, OUT, 1, 2, 128, 2>), grid, dim3(kThreads), 0, st, g);
  } else {
    hipLaunchKernelGGL((k_product<T, AD, BD, OUT, 1, 1, 128, 2>), grid, dim3(kThreads), 0, st, g);
  }
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
