// Cross attention on the matrix cores (gfx950), forward and backward.
//     s = scale q k^T,  p = softmax(s) over the keys that count,  o = p v,  lse = log sum exp s
//     dp = do v^T,  delta = sum_d do o = sum_j p dp,  ds = p (dp - delta),  dq = scale ds k,  dk = scale ds^T q,  dv = p^T do
// Rows are gathered by index into LDS by direct loads; a masked key's, and what lies past the end, come from a block of zeros.
// What bounds it: k and v on their way from HBM and the caches (256 sequences of 16 .. 256 rows against 64 .. 512 keys, 8 heads of
// 128 in bf16: 131 us, 110 without the products, 87 for its bytes at a copy's rate; 64 single rows against 512 .. 4,096 keys, 16
// heads of 64 on 4: 30 us and a join of 4, at 4.9 TB/s); in the gradient the exponentials beside the products and the loads (64
// sequences of 256 .. 512 rows against 256 .. 1,024 keys, 16 heads of 64: 379 us, 440 TFLOP/s); in fp32 the matrix cores.
//
// Products are 32 x 32 tiles with the axis of the softmax on the accumulators' rows: the forward computes s^T = k q^T, so a
// lane holds one query's column, its maximum, sum and rescaling are one value a lane, and p^T leaves the accumulators in the
// layout of the next product's operand: its K values (keys) are permuted, 4 h + 0..3 and 8 + 4 h + 0..3 of 16 for half wave h,
// and v's fragments are read in the same order.  The keys' gradient holds keys on the lanes and does the same along the
// queries.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "checks.h"
#include "common.h"
#include "cross.h"
#include "dma.h"
#include "internal.h"
#include "mfma.h"

namespace fold {

namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __attribute__((aligned(16))) uint32_t g_zero[4];

#define FOLD_LDS_AS __attribute__((address_space(3)))
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4_t;
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t{a, b}), bf16x2_t));
}
__device__ __forceinline__ float word(const uint4& v, int e) {
  return __uint_as_float(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w);
}
// the value of the other half wave's lane of the same column, with this lane's
__device__ __forceinline__ float halves_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// LDS that only this wave reads and writes: its direct loads have landed (vm_wait), its reads before them are done
__device__ __forceinline__ void wave_barrier_lds() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Values that were loaded before a loop are there: without it the compiler waits for them at their use inside the loop, where
// the wait takes the direct loads in flight with it.
template <int N>
__device__ __forceinline__ void arrived(uint4 (&v)[N]) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int i = 0; i < N; ++i) {
    u32x4 t = __builtin_bit_cast(u32x4, v[i]);
    asm volatile("" : "+v"(t));
    v[i] = __builtin_bit_cast(uint4, t);
  }
}
__device__ __forceinline__ void arrived(float& v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void arrived(int& v) { asm volatile("" : "+v"(v)); }

// ---- tiles in LDS ---------------------------------------------------------------------------------------------------

// A row of a tile is U 16-byte units; unit u of row r lies at r U + (u ^ f(r)).  f puts the same unit of 16 consecutive rows
// into 16 different bank groups (16-byte reads along the rows), and 64 bytes of 4 consecutive rows into different quarters of
// the banks (transposing reads across them).
template <int U>
__device__ __forceinline__ int swizzle(int r) {
  if constexpr (U % 16 == 0) return ((r & 3) << 2) | ((r >> 2) & 3);
  else if constexpr (U % 8 == 0) return ((r & 2) << 1) | ((r >> 2) & 3);
  else return (r >> 2) & 3;  // 4, 12
}
template <int U>
__device__ __forceinline__ int unit_at(int r, int u) {
  return (r * U + (u ^ swizzle<U>(r))) * 16;
}

// acc += A B for one step of 32 bytes of K (16 bf16 or 8 fp32 values; a half wave's 16 bytes are its own)
template <typename T>
__device__ __forceinline__ f32x16 step_mma(const uint4& a, const uint4& b, f32x16 c) {
  if constexpr (sizeof(T) == 2) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(word(a, e), word(b, e), c, 0, 0, 0);
  }
  return c;
}

// What leaves an accumulator as the next product's operand: 32 K values (the accumulator's rows) of the lane's column.  In bf16
// p and ds are rounded here, to nearest even (at most 2^-8 of each): the matrix cores multiply k, q, v and dout by operands of
// their own type, and what the rounding leaves would be a second product of the same length.
template <typename T>
struct Probs;
template <>
struct Probs<uint16_t> {
  uint4 v[2];
  __device__ __forceinline__ explicit Probs(const f32x16& p) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
      v[t] = make_uint4(bf16_pair(p[8 * t], p[8 * t + 1]), bf16_pair(p[8 * t + 2], p[8 * t + 3]),
                        bf16_pair(p[8 * t + 4], p[8 * t + 5]), bf16_pair(p[8 * t + 6], p[8 * t + 7]));
  }
};
template <>
struct Probs<float> {
  f32x16 v;
  __device__ __forceinline__ explicit Probs(const f32x16& p) : v(p) {}
};

// acc[db] += X^T P: X the tile's rows k0 .. k0 + 31 (K), its columns 32 db .. on the accumulators' rows
template <typename T, int U, int DB>
__device__ __forceinline__ void across_mma(const char* tile, int k0, const Probs<T>& p, f32x16 (&acc)[DB], int lane) {
  const int h = lane >> 5, l32 = lane & 31;
  if constexpr (sizeof(T) == 2) {
    const int g = lane >> 4, gi = lane & 15;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int k = k0 + 16 * t + 4 * h + (gi >> 2);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const int col = 32 * db + 16 * (g & 1) + 4 * (gi & 3);
        const int in = (col & 7) * 2, u = col >> 3;
        const bf16x4_t lo =
            __builtin_amdgcn_ds_read_tr16_b64_v4bf16((FOLD_LDS_AS bf16x4_t*)(tile + unit_at<U>(k, u) + in));
        const bf16x4_t hi =
            __builtin_amdgcn_ds_read_tr16_b64_v4bf16((FOLD_LDS_AS bf16x4_t*)(tile + unit_at<U>(k + 8, u) + in));
        const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, make_uint4(a.x, a.y, b.x, b.y)),
                                                          __builtin_bit_cast(bf16x8, p.v[t]), acc[db], 0, 0, 0);
      }
    }
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int k = k0 + 8 * (r >> 2) + 4 * h + (r & 3);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const float a = *reinterpret_cast<const float*>(tile + unit_at<U>(k, 8 * db + (l32 >> 2)) + (l32 & 3) * 4);
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p.v[r], acc[db], 0, 0, 0);
      }
    }
  }
}

// 16 bytes at an address that is a multiple of an element's size alone (global memory takes them at any)
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Loose {
  uint32_t w[4];
};
// 16 bytes of a row from element e0 (d elements are there), zero past its end.  Without whole units the last one is taken from
// the row's last 16 bytes and moved down: element by element, 61 chains of 615 rows against 65 keys, 4 heads of 50 in fp32,
// their gradients took 298 us.
template <typename T, bool VEC>
__device__ __forceinline__ uint4 row_unit(const T* row, int e0, int d) {
  constexpr int E = 16 / (int)sizeof(T);
  uint4 v = make_uint4(0, 0, 0, 0);
  if (e0 >= d) return v;
  if constexpr (VEC) {
    v = *reinterpret_cast<const uint4*>(row + e0);
  } else {
    uint64_t lo = 0, hi = 0;
    int by = 0;
    if (d >= E) {
      const int at = min(e0, d - E), bits = (e0 - at) * (int)sizeof(T) * 8;  // 0 .. 112
      const Loose<T> u = *reinterpret_cast<const Loose<T>*>(row + at);
      lo = (uint64_t)u.w[1] << 32 | u.w[0];
      hi = (uint64_t)u.w[3] << 32 | u.w[2];
      if (bits >= 64) lo = hi, hi = 0;
      by = bits & 63;
    } else {  // heads of less than 16 bytes: their only unit
#pragma unroll 1
      for (int e = d - 1; e >= 0; --e) {
        constexpr int B = 8 * (int)sizeof(T);
        hi = hi << B | lo >> (64 - B);
        lo = lo << B | (B == 16 ? reinterpret_cast<const uint16_t*>(row)[e] : __float_as_uint((float)row[e]));
      }
    }
    lo = lo >> by | hi << 1 << (63 - by);
    hi >>= by;
    v = make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
  }
  return v;
}

// a row whose number and whose bytes to the next fit 32 bits: one multiplication into 64
template <typename T>
__device__ __forceinline__ const T* row_at(const T* base, int row, uint32_t ldb) {
  return reinterpret_cast<const T*>(reinterpret_cast<const char*>(base) + (uint64_t)(uint32_t)row * ldb);
}

// One wave's share of the loads of a tile of ROWS rows that NW waves load together: NI instructions of 1 KB.
template <typename T, int DP, int ROWS, int NW, bool VEC>
struct TileLoader {
  static constexpr int U = DP * (int)sizeof(T) / 16, E = 16 / (int)sizeof(T), NI = ROWS * U / (64 * NW);
  static_assert(NI * 64 * NW == ROWS * U, "whole instructions");
  int part, lane;
  __device__ __forceinline__ TileLoader(int part_, int lane_) : part(part_), lane(lane_) {}
  __device__ __forceinline__ int place(int i) const { return (part * NI + i) * 64 + lane; }
  __device__ __forceinline__ int row(int i) const { return place(i) / U; }
  __device__ __forceinline__ int unit(int i) const { return place(i) % U ^ swizzle<U>(row(i)); }
  // idx[i]: the matrix row of tile row row(i), -1: zeros
  __device__ __forceinline__ void load(const T* base, uint32_t ldb, int d, const int (&idx)[NI], char* lds) const {
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int e0 = unit(i) * E;
        const void* src = idx[i] >= 0 && e0 < d ? static_cast<const void*>(row_at(base, idx[i], ldb) + e0)
                                                : static_cast<const void*>(g_zero);
        dma16_untracked(src, lds + (part * NI + i) * 1024);
      }
    } else {
      uint4 v[NI];
#pragma unroll
      for (int i = 0; i < NI; ++i)
        v[i] = idx[i] >= 0 ? row_unit<T, false>(row_at(base, idx[i], ldb), unit(i) * E, d) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < NI; ++i) *reinterpret_cast<uint4*>(lds + place(i) * 16) = v[i];
    }
  }
};

template <typename T, bool VEC>
__device__ __forceinline__ void store4(T* p, const float (&v)[4], int d0, int d) {
  if constexpr (VEC) {
    if (d0 >= d) return;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(p + d0) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
    else *reinterpret_cast<float4*>(p + d0) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (d0 + e < d) p[d0 + e] = from_f32<T>(v[e]);
  }
}

// A wave's 32 rows of a result, which lie on the accumulators' columns, to memory through an image in LDS of its own, so that an
// instruction stores whole rows: stored from the registers, 8 bytes of 32 rows at a time, the keys' gradient of 64 chains of
// 640 nodes, 16 heads of 64, spent more time on its stores than on its products.  row(r): where row r goes, NULL: nowhere.
template <typename T, int DP>
constexpr int image_row() { return DP * (int)sizeof(T) + 16; }
template <typename T, int DP>
constexpr int image_bytes() { return 32 * image_row<T, DP>(); }
template <typename T, int DP, bool VEC, class ROW>
__device__ __forceinline__ void store_image(const f32x16 (&acc)[DP / 32], float factor, int d, char* img, int lane, ROW&& row) {
  constexpr int U = DP * (int)sizeof(T) / 16, E = 16 / (int)sizeof(T);
  const int h = lane >> 5, l32 = lane & 31;
#pragma unroll
  for (int db = 0; db < DP / 32; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float w[4] = {acc[db][4 * j] * factor, acc[db][4 * j + 1] * factor, acc[db][4 * j + 2] * factor,
                          acc[db][4 * j + 3] * factor};
      store4<T, true>(reinterpret_cast<T*>(img + l32 * image_row<T, DP>()), w, 32 * db + 8 * j + 4 * h, DP);
    }
  wave_barrier_lds();
#pragma unroll 4
  for (int i = 0; i < 32 * U / 64; ++i) {
    const int at = i * 64 + lane, r = at / U, e0 = at % U * E;
    T* to = row(r);
    const uint4 v = *reinterpret_cast<const uint4*>(img + r * image_row<T, DP>() + at % U * 16);
    if (!to || e0 >= d) continue;
    if constexpr (VEC) {
      *reinterpret_cast<uint4*>(to + e0) = v;
    } else if (e0 + E <= d) {
      *reinterpret_cast<Loose<T>*>(to + e0) = Loose<T>{{v.x, v.y, v.z, v.w}};
    } else {
      const T* e = reinterpret_cast<const T*>(&v);
#pragma unroll
      for (int k = 0; k < E; ++k)
        if (e0 + k < d) to[e0 + k] = e[k];
    }
  }
  wave_barrier_lds();  // before the image is written again
}

struct Args {
  const void *q, *k, *v, *dout;
  uint32_t ldq, ldk, ldv, lddo;  // in bytes
  const int *q_row, *k_row;
  const uint8_t* mask;
  float scale;
  int heads, group, d;
  int slots;       // of a head
  unsigned magic;  // x / group = x * magic >> 20 for x < 2^10, group <= 256
  void *out, *out2;
  int64_t ldo, ldo2;
  float* lse;          // written by the forward, read by the backward
  const float* delta;  // [query rows][heads]
  float* part;
};
__device__ __forceinline__ int row_of(const int* list, int entry) { return list[entry]; }

// a workgroup's tile, with its head and its slot among all heads'
template <class Tile>
__device__ __forceinline__ Tile tile_of_head(const Tile* tiles, unsigned index, const Args& a) {
  Tile t = tiles[index];
  t.kv_head = blockIdx.y;
  if (t.slot >= 0) t.slot += blockIdx.y * a.slots;
  return t;
}

// the virtual row r of a tile: its query's list entry and its head
struct Virtual {
  int entry, head;
  __device__ __forceinline__ Virtual(const Args& a, int entry0, int head0, int kv_head, int r) {
    const int x = head0 + r, i = (int)((unsigned)x * a.magic >> 20);
    entry = entry0 + i;
    head = kv_head * a.group + (x - i * a.group);
  }
};

// ---- forward ----------------------------------------------------------------------------------------------------------

constexpr float kSlack = 8.f;  // the reference is moved when a row's maximum has grown by a factor of 2^8

template <int TK>
constexpr uint64_t all_keys() { return TK == 64 ? ~0ull : (1ull << TK) - 1; }

// A lane mask (on the scalar unit) of the keys that register r of block kb holds: key 8 (r / 4) + r % 4 in the lower half
// wave, 4 more in the upper.
__device__ __forceinline__ bool key_in(uint64_t bits, int kb, int r) {
  const int at = 32 * kb + 8 * (r >> 2) + (r & 3);
  const uint64_t lo = (bits >> at) & 1, hi = (bits >> (at + 4)) & 1;
  return __builtin_amdgcn_inverse_ballot_w64((0 - lo & 0xffffffffull) | (0 - hi) << 32);
}

// The tiles of a run of keys on their way into LDS.  A tile's row numbers and mask are fetched while the tile two before it is
// multiplied and looked at when its loads are issued, a tile later: a wait for them waits for the direct loads that were issued
// before them too.
template <typename T, int DP, int TK, int NW, bool VEC>
struct KeyFeed {
  using L = TileLoader<T, DP, TK, NW, VEC>;
  const Args& a;
  const L& ld;
  int k_begin, k_end;
  int idx[L::NI];
  uint8_t mk;  // of entry lane % TK
  __device__ __forceinline__ KeyFeed(const Args& a_, const QTile& t, const L& ld_)
      : a(a_), ld(ld_), k_begin(t.k_begin), k_end(t.k_end), mk(1) {}
  __device__ __forceinline__ void fetch(int tile) {
    const int k0 = k_begin + tile * TK;
#pragma unroll
    for (int i = 0; i < L::NI; ++i) idx[i] = row_of(a.k_row, min(k0 + ld.row(i), k_end - 1));
    if (a.mask) mk = a.mask[min(k0 + (ld.lane & (TK - 1)), k_end - 1)];
  }
  // starts the loads of the tile that was fetched; which of its keys count
  __device__ __forceinline__ uint64_t issue(int tile, const T* k, const T* v, char* kt, char* vt) {
#pragma unroll
    for (int i = 0; i < L::NI; ++i) arrived(idx[i]);
    const uint64_t bits = __ballot(ld.lane < TK && k_begin + tile * TK + ld.lane < k_end && mk != 0);
    if (bits != all_keys<TK>())
#pragma unroll
      for (int i = 0; i < L::NI; ++i) idx[i] = (bits >> ld.row(i)) & 1 ? idx[i] : -1;
    ld.load(k, a.ldk, a.d, idx, kt);
    ld.load(v, a.ldv, a.d, idx, vt);
    return bits;
  }
};

// one value per lane of the running softmax of the lane's query, in base 2
struct Running {
  float m = -INFINITY, l = 0.f;
};

// p^T of one tile from s^T (TK keys x 32 queries), and the accumulators' rescaling
template <int KB, int DB>
__device__ __forceinline__ void softmax_tile(f32x16 (&s)[KB], f32x16 (&o)[DB], Running& run, float c, uint64_t bits,
                                             uint64_t all) {
  if (bits != all) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = key_in(bits, kb, r) ? s[kb][r] : -INFINITY;
  }
  float top = s[0][0];
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) top = fmaxf(top, s[kb][r]);
  const float m2 = halves_max(top) * c;
  if (__any(m2 > run.m + kSlack)) {
    const float m = fmaxf(run.m, m2), alpha = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(run.m - m);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
    run.l *= alpha;
    run.m = m;
  }
  const float ref = run.m == -INFINITY ? 0.f : run.m;
  float sum = 0.f;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[kb][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][r], c, -ref));
      sum += s[kb][r];
    }
  run.l += sum;
}

template <int TK, typename T, int DP>
constexpr int tile_bytes() { return TK * DP * (int)sizeof(T); }

// Partial results of a slot: ROWS rows of DP values, then their m and l.
template <int DP>
constexpr int slot_floats(int rows) { return rows * (DP + 2); }

// NW = 4: a workgroup's four waves hold 32 virtual rows each and share the keys' tiles.  NW = 1: they hold the same 32 rows,
// every wave walks every fourth tile in LDS of its own, and they meet at the end.  Two tiles of keys and values lie in LDS:
// one is multiplied while the next is loaded.
template <typename T, int DP, int TK, int NW, bool VEC>
__global__ __launch_bounds__(kThreads, (DP * sizeof(T) > 256 ? 1 : 2)) void k_cross(const QTile* tiles, Args a) {
  constexpr int U = DP * (int)sizeof(T) / 16, NS = U / 2, DB = DP / 32, KB = TK / 32, TB = tile_bytes<TK, T, DP>();
  constexpr int E = 16 / (int)sizeof(T), ROWS = NW == 4 ? kCrossRows : kCrossFew;
  constexpr int BUF = 2 * TB;  // a tile of keys and one of values
  constexpr int MEET = NW == 1 ? 4 * 32 * (DP + 4) * 4 + 4 * 32 * 8 : 0;
  constexpr int IMAGES = NW == 4 ? 4 * image_bytes<T, DP>() : 0;
  constexpr int TILES = 2 * BUF * (NW == 1 ? 4 : 1), LDS = TILES > IMAGES ? TILES : IMAGES;
  __shared__ __attribute__((aligned(16))) char lds[LDS > MEET ? LDS : MEET];
  const QTile t = tile_of_head(tiles, blockIdx.x, a);
  if (t.rows == 0) return;
  const int lane = threadIdx.x & 63, wave = wave_id(), h = lane >> 5, l32 = lane & 31;
  const T* k = static_cast<const T*>(a.k) + t.kv_head * a.d;
  const T* v = static_cast<const T*>(a.v) + t.kv_head * a.d;
  const int first = NW == 4 ? 32 * wave : 0;
  const bool active = first < t.rows;
  const Virtual vr(a, t.entry, t.head0, t.kv_head, min(first + l32, t.rows - 1));
  const int qrow = row_of(a.q_row, vr.entry);
  const bool in = first + l32 < t.rows;
  uint4 qf[NS];
  {
    const T* q = row_at(static_cast<const T*>(a.q), qrow, a.ldq) + vr.head * a.d;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = row_unit<T, VEC>(q, (2 * s + h) * E, a.d);
  }
  f32x16 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[db][r] = 0.f;
  Running run;
  const float c = a.scale * kLog2e;
  using L = TileLoader<T, DP, TK, NW, VEC>;
  const L ld(NW == 4 ? wave : 0, lane);
  char* mine = lds + (NW == 4 ? 0 : wave * 2 * BUF);
  constexpr int STRIDE = NW == 4 ? 1 : 4;
  const int ntile = (t.k_end - t.k_begin + TK - 1) / TK;
  KeyFeed<T, DP, TK, NW, VEC> feed(a, t, ld);
  auto issue = [&](int tile, int buf) { return feed.issue(tile, k, v, mine + buf * BUF, mine + buf * BUF + TB); };
  int at = NW == 4 ? 0 : wave;
  uint64_t bits = 0;
  if (at < ntile) feed.fetch(at);
  arrived(qf);
  if (at < ntile) {
    bits = issue(at, 0);
    if (at + STRIDE < ntile) feed.fetch(at + STRIDE);
  }
  for (int buf = 0; at < ntile; at += STRIDE, buf ^= 1) {
    const uint64_t now = bits;
    vm_wait();
    if constexpr (NW == 4) __syncthreads();
    else wave_barrier_lds();
    if (at + STRIDE < ntile) {
      bits = issue(at + STRIDE, buf ^ 1);
      if (at + 2 * STRIDE < ntile) feed.fetch(at + 2 * STRIDE);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (!active) continue;
    const char *kt = mine + buf * BUF, *vt = kt + TB;
    f32x16 s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
      for (int st = 0; st < NS; ++st)
        s[kb] = step_mma<T>(*reinterpret_cast<const uint4*>(kt + unit_at<U>(32 * kb + l32, 2 * st + h)), qf[st], s[kb]);
    }
    softmax_tile<KB, DB>(s, o, run, c, now, all_keys<TK>());
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) across_mma<T, U, DB>(vt, 32 * kb, Probs<T>(s[kb]), o, lane);
  }
  run.l = halves_sum(run.l);
  T* out = static_cast<T*>(a.out);
  if constexpr (NW == 4) {
    __syncthreads();  // the images lie where the tiles were
    if (!active) return;
    if (t.slot >= 0) {
      if (!in) return;
      float* p = a.part + (size_t)t.slot * slot_floats<DP>(ROWS);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *reinterpret_cast<float4*>(p + (first + l32) * DP + 32 * db + 8 * j + 4 * h) =
              make_float4(o[db][4 * j], o[db][4 * j + 1], o[db][4 * j + 2], o[db][4 * j + 3]);
      if (h == 0) {
        p[ROWS * DP + first + l32] = run.m;
        p[ROWS * (DP + 1) + first + l32] = run.l;
      }
      return;
    }
    const float inv = run.l > 0.f || run.l != run.l ? 1.f / run.l : 0.f;
    store_image<T, DP, VEC>(o, inv, a.d, lds + wave * image_bytes<T, DP>(), lane, [&](int r) -> T* {
      if (first + r >= t.rows) return nullptr;
      const Virtual x(a, t.entry, t.head0, t.kv_head, first + r);
      return out + (int64_t)row_of(a.q_row, x.entry) * a.ldo + x.head * a.d;
    });
    if (h == 0 && in && a.lse)
      a.lse[(int64_t)qrow * a.heads + vr.head] = run.l == 0.f ? -INFINITY : (run.m + __builtin_amdgcn_logf(run.l)) * kLn2;
  } else {
    // the waves' rows meet in LDS: [wave][row][DP + 4], then m and l [wave][row]
    constexpr int RS = DP + 4;
    float* img = reinterpret_cast<float*>(lds);
    float* ms = img + 4 * 32 * RS;
    float* ls = ms + 128;
    __syncthreads();
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(img + (wave * 32 + l32) * RS + 32 * db + 8 * j + 4 * h) =
            make_float4(o[db][4 * j], o[db][4 * j + 1], o[db][4 * j + 2], o[db][4 * j + 3]);
    if (h == 0) {
      ms[wave * 32 + l32] = run.m;
      ls[wave * 32 + l32] = run.l;
    }
    __syncthreads();
    const int r = threadIdx.x >> 3, c0 = (threadIdx.x & 7) * 4;
    if (r >= t.rows) return;
    float m = -INFINITY, l = 0.f, f[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, ms[w * 32 + r]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      f[w] = ms[w * 32 + r] == -INFINITY ? (ls[w * 32 + r] == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(ms[w * 32 + r] - m);
      l += f[w] * ls[w * 32 + r];
    }
    const Virtual mv(a, t.entry, t.head0, t.kv_head, r);
    const int row = row_of(a.q_row, mv.entry);
    float* p = t.slot >= 0 ? a.part + (size_t)t.slot * slot_floats<DP>(ROWS) : nullptr;
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float4 y = *reinterpret_cast<const float4*>(img + (w * 32 + r) * RS + 32 * db + c0);
        x[0] += f[w] * y.x;
        x[1] += f[w] * y.y;
        x[2] += f[w] * y.z;
        x[3] += f[w] * y.w;
      }
      if (p) {
        *reinterpret_cast<float4*>(p + r * DP + 32 * db + c0) = make_float4(x[0], x[1], x[2], x[3]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] *= inv;
        store4<T, VEC>(out + (int64_t)row * a.ldo + mv.head * a.d, x, 32 * db + c0, a.d);
      }
    }
    if (c0 == 0) {
      if (p) {
        p[ROWS * DP + r] = m;
        p[ROWS * (DP + 1) + r] = l;
      } else if (a.lse) {
        a.lse[(int64_t)row * a.heads + mv.head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
      }
    }
  }
}

// The pieces of a tile joined, in their order: SOFTMAX, each with its m and l, or plain sums (times the scale).  Eight threads
// a row, 32 rows a workgroup, four pieces in flight.
template <typename T, int DP, int ROWS, bool SOFTMAX, bool VEC>
__global__ __launch_bounds__(kThreads) void k_cross_join(const QTile* tiles, Args a) {
  constexpr int DB = DP / 32, SF = slot_floats<DP>(ROWS), BLOCKS = ROWS / 32, F = 4;
  const QTile t = tile_of_head(tiles, blockIdx.x / BLOCKS, a);
  const int c0 = (threadIdx.x & 7) * 4, r = blockIdx.x % BLOCKS * 32 + (threadIdx.x >> 3);
  if (r >= t.rows) return;
  T* out = static_cast<T*>(a.out);
  const float* p = a.part + (size_t)t.slot * SF;
  float m = -INFINITY, l = 0.f;
  if (SOFTMAX)
    for (int i0 = 0; i0 < t.pieces; i0 += 2 * F) {
      float mi[2 * F];
#pragma unroll
      for (int u = 0; u < 2 * F; ++u) mi[u] = p[(size_t)min(i0 + u, t.pieces - 1) * SF + ROWS * DP + r];
#pragma unroll
      for (int u = 0; u < 2 * F; ++u) m = fmaxf(m, mi[u]);
    }
  float x[DB][4];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[db][e] = 0.f;
  for (int i0 = 0; i0 < t.pieces; i0 += F) {
    float mi[F], li[F];
    float4 y[F][DB];
#pragma unroll
    for (int u = 0; u < F; ++u) {
      const float* at = p + (size_t)min(i0 + u, t.pieces - 1) * SF;
      if (SOFTMAX) {
        mi[u] = at[ROWS * DP + r];
        li[u] = at[ROWS * (DP + 1) + r];
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) y[u][db] = *reinterpret_cast<const float4*>(at + r * DP + 32 * db + c0);
    }
#pragma unroll
    for (int u = 0; u < F; ++u) {
      if (i0 + u >= t.pieces) break;
      float f = 1.f;
      if (SOFTMAX) {
        f = mi[u] == -INFINITY ? (li[u] == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(mi[u] - m);
        l += f * li[u];
      }
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        x[db][0] += f * y[u][db].x;
        x[db][1] += f * y[u][db].y;
        x[db][2] += f * y[u][db].z;
        x[db][3] += f * y[u][db].w;
      }
    }
  }
  const Virtual v(a, t.entry, t.head0, t.kv_head, r);
  const int row = row_of(a.q_row, v.entry);
  const float inv = !SOFTMAX ? a.scale : l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[db][e] *= inv;
    store4<T, VEC>(out + (int64_t)row * a.ldo + v.head * a.d, x[db], 32 * db + c0, a.d);
  }
  if (SOFTMAX && c0 == 0 && a.lse)
    a.lse[(int64_t)row * a.heads + v.head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ---- backward ---------------------------------------------------------------------------------------------------------

// delta = sum_d dout out of rows and heads, out as it was rounded: eight lanes each
struct DeltaArgs {
  const void *out, *dout;
  int64_t ldo, lddo;
  const int *q_row, *entries;  // the rows' list entries, NULL: all
  int64_t n;                   // rows times heads
  int heads, d;
  float* delta;
};
template <typename T, bool VEC>
__device__ __forceinline__ void row_deltas(const DeltaArgs& a, unsigned block, unsigned blocks) {
  constexpr int E = 16 / (int)sizeof(T);
  for (int64_t at = (int64_t)block * (kThreads / 8) + (threadIdx.x >> 3); at < a.n; at += (int64_t)blocks * (kThreads / 8)) {
    const int i = (int)(at / a.heads), head = (int)(at - (int64_t)i * a.heads);
    const int row = row_of(a.q_row, a.entries ? a.entries[i] : i);
    const T *x = static_cast<const T*>(a.out) + (int64_t)row * a.ldo + head * a.d;
    const T* y = static_cast<const T*>(a.dout) + (int64_t)row * a.lddo + head * a.d;
    float s = 0.f;
    for (int e0 = (threadIdx.x & 7) * E; e0 < a.d; e0 += 8 * E) {
      const uint4 u = row_unit<T, VEC>(x, e0, a.d), w = row_unit<T, VEC>(y, e0, a.d);
#pragma unroll
      for (int e = 0; e < E; ++e)
        s += to_f32<T>(reinterpret_cast<const T*>(&u)[e]) * to_f32<T>(reinterpret_cast<const T*>(&w)[e]);
    }
#pragma unroll
    for (int o = 1; o < 8; o *= 2) s += __shfl_xor(s, o);  // (eight lanes are in or out together)
    if ((threadIdx.x & 7) == 0) a.delta[(int64_t)row * a.heads + head] = s;
  }
}
template <typename T, bool VEC>
__global__ __launch_bounds__(kThreads) void k_cross_delta(DeltaArgs a) {
  row_deltas<T, VEC>(a, blockIdx.x, gridDim.x);
}

// delta = sum_j p_j dp_j of rows whose source has up to 32 keys, a tile of them: the keys and values lie in LDS, a wave takes every
// fourth 32 rows and loads the next ones while it looks at the products.  Summed from the first key's dp on, whose products are
// those of the gradients bit for bit: a row that has one key has dp - delta = 0.  The launch's first `n` workgroups of a head; the
// rest take all other rows (256 sequences of 64 rows, 8 heads of 64 in bf16, gradients: with 16 keys each 47 us, from out 43; with 8
// and 100 keys in turn 59, from out 55).
template <typename T, int DP, bool VEC>
__global__ __launch_bounds__(kThreads, (DP * sizeof(T) <= 128 ? 4 : DP * sizeof(T) <= 256 ? 3 : 1)) void k_cross_delta_brief(
    const QTile* tiles, unsigned n, Args a, DeltaArgs others) {
  constexpr int TK = 32, U = DP * (int)sizeof(T) / 16, NS = U / 2, TB = tile_bytes<TK, T, DP>(), E = 16 / (int)sizeof(T);
  __shared__ __attribute__((aligned(16))) char lds[2 * TB];
  if (blockIdx.x >= n) {
    const unsigned more = gridDim.x - n;
    return row_deltas<T, VEC>(others, blockIdx.y * more + blockIdx.x - n, gridDim.y * more);
  }
  const QTile t = tile_of_head(tiles, blockIdx.x, a);
  const int lane = threadIdx.x & 63, wave = wave_id(), h = lane >> 5, l32 = lane & 31;
  const T* k = static_cast<const T*>(a.k) + t.kv_head * a.d;
  const T* v = static_cast<const T*>(a.v) + t.kv_head * a.d;
  using L = TileLoader<T, DP, TK, 2, VEC>;  // two waves load the keys, two the values
  const L ld(wave & 1, lane);
  int idx[L::NI];
#pragma unroll
  for (int i = 0; i < L::NI; ++i) idx[i] = row_of(a.k_row, min(t.k_begin + ld.row(i), t.k_end - 1));
  const uint8_t mk = a.mask ? a.mask[min(t.k_begin + l32, t.k_end - 1)] : 1;
  uint4 qf[NS], df[NS];
  int64_t stat = 0;
  float lse = 0.f;
  const auto load = [&](int first) __attribute__((always_inline)) {
    const Virtual vr(a, t.entry, t.head0, t.kv_head, min(first + l32, t.rows - 1));
    const int qrow = row_of(a.q_row, vr.entry);
    const T* q = row_at(static_cast<const T*>(a.q), qrow, a.ldq) + vr.head * a.d;
    const T* g = row_at(static_cast<const T*>(a.dout), qrow, a.lddo) + vr.head * a.d;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      qf[s] = row_unit<T, VEC>(q, (2 * s + h) * E, a.d);
      df[s] = row_unit<T, VEC>(g, (2 * s + h) * E, a.d);
    }
    stat = (int64_t)qrow * a.heads + vr.head;
    lse = a.lse[stat];
  };
  if (32 * wave < t.rows) load(32 * wave);
  const uint64_t bits = __ballot(lane < TK && t.k_begin + lane < t.k_end && mk != 0);
#pragma unroll
  for (int i = 0; i < L::NI; ++i) idx[i] = (bits >> ld.row(i)) & 1 ? idx[i] : -1;
  if (wave < 2) ld.load(k, a.ldk, a.d, idx, lds);
  else ld.load(v, a.ldv, a.d, idx, lds + TB);
  vm_wait();
  __syncthreads();
  const float c = a.scale * kLog2e;
  const int j = bits ? __builtin_ctzll(bits) : 0;  // the first key: register 4 (j / 8) + j % 4 of half (j / 4) % 2
  for (int first = 32 * wave; first < t.rows; first += 32 * (kThreads / 64)) {
    f32x16 s, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
    for (int st = 0; st < NS; ++st) {
      const int place = unit_at<U>(l32, 2 * st + h);
      s = step_mma<T>(*reinterpret_cast<const uint4*>(lds + place), qf[st], s);
      dp = step_mma<T>(*reinterpret_cast<const uint4*>(lds + TB + place), df[st], dp);
      if (st % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // (registers)
    }
    const float ref = lse == -INFINITY ? INFINITY : lse * kLog2e;
    const int64_t at = stat;
    if (first + 32 * (kThreads / 64) < t.rows) load(first + 32 * (kThreads / 64));
    float base = 0.f, sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) base = 8 * (r >> 2) + (r & 3) == (j & ~4) ? dp[r] : base;
    base = __shfl(base, l32 + 32 * ((j >> 2) & 1));
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float term = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -ref)) * (dp[r] - base);
      sum += key_in(bits, 0, r) ? term : 0.f;
    }
    sum = base + halves_sum(sum);
    if (h == 0 && first + l32 < t.rows) others.delta[at] = sum;
  }
}

// Waves a SIMD of the gradients: three for rows of 128 bytes (64 chains of 16 heads of 64 in bf16: 375 us, with two 390), two
// where 256 registers do (5 sequences of 265 .. 443 rows, 32 heads of 50 in fp32: 90 us, with one 113).
template <typename T, int DP>
constexpr int waves_back() { return DP * sizeof(T) <= 128 ? 3 : DP * sizeof(T) <= 192 || (sizeof(T) == 4 && DP == 64) ? 2 : 1; }
// Whether a lane keeps its fragments of v in LDS of its own: where registers are short (the widest fp32 heads, and where more
// than one wave a SIMD share them: 168 each, or 256).
template <typename T, int DP>
constexpr bool keep_values() { return DP * sizeof(T) > 384 || DP * sizeof(T) == 128 || waves_back<T, DP>() == 2; }
template <typename T, int DP, int TK>
struct BackLds {
  static constexpr int TILES = 4 * tile_bytes<TK, T, DP>(), IMAGES = 4 * image_bytes<T, DP>();
  __attribute__((aligned(16))) char tiles[TILES > IMAGES ? TILES : IMAGES];
  __attribute__((aligned(16))) float stats[2][2][TK];  // [buffer][lse in base 2, delta][row]
  uint4 kept[keep_values<T, DP>() ? 4 * (DP * sizeof(T) / 32) * 64 : 1];
};

// The queries' gradient of a tile of up to 32 rows: all four waves hold them, each takes 32 of 128 keys that lie in LDS, and
// their sums meet at the end.  With the rows in one wave the other three only load: 216 x 5 sequences of 5 .. 14 rows against
// 1,628 .. 2,262 keys, 5 heads of 50 in fp32, all gradients: 1,285 us, so 930.
template <typename T, int DP, bool VEC>
__device__ __forceinline__ void queries_back_few(const QTile& t, const Args& a, char* lds) {
  constexpr int U = DP * (int)sizeof(T) / 16, NS = U / 2, DB = DP / 32, KEYS = 128, TB = tile_bytes<KEYS, T, DP>();
  constexpr int E = 16 / (int)sizeof(T);
  const int lane = threadIdx.x & 63, wave = wave_id(), h = lane >> 5, l32 = lane & 31;
  const T* k = static_cast<const T*>(a.k) + t.kv_head * a.d;
  const T* v = static_cast<const T*>(a.v) + t.kv_head * a.d;
  uint4 qf[NS], df[NS];
  float ref, delta;
  {
    const Virtual vr(a, t.entry, t.head0, t.kv_head, min(l32, t.rows - 1));
    const int qrow = row_of(a.q_row, vr.entry);
    const T* q = row_at(static_cast<const T*>(a.q), qrow, a.ldq) + vr.head * a.d;
    const T* g = row_at(static_cast<const T*>(a.dout), qrow, a.lddo) + vr.head * a.d;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      qf[s] = row_unit<T, VEC>(q, (2 * s + h) * E, a.d);
      df[s] = row_unit<T, VEC>(g, (2 * s + h) * E, a.d);
    }
    const int64_t stat = (int64_t)qrow * a.heads + vr.head;
    delta = a.delta[stat];
    const float lse = a.lse[stat];
    ref = lse == -INFINITY ? INFINITY : lse * kLog2e;
  }
  f32x16 dq[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[db][r] = 0.f;
  const float c = a.scale * kLog2e;
  using L = TileLoader<T, DP, KEYS, 4, VEC>;
  const L ld(wave, lane);
  const char *kt = lds, *vt = lds + TB;
#pragma unroll 1
  for (int k0 = t.k_begin; k0 < t.k_end; k0 += KEYS) {
    if (k0 != t.k_begin) __syncthreads();  // the keys before have been read
    int idx[L::NI];
#pragma unroll
    for (int i = 0; i < L::NI; ++i) idx[i] = row_of(a.k_row, min(k0 + ld.row(i), t.k_end - 1));
    uint8_t m0 = 1, m1 = 1;
    if (a.mask) {
      m0 = a.mask[min(k0 + lane, t.k_end - 1)];
      m1 = a.mask[min(k0 + 64 + lane, t.k_end - 1)];
    }
    const uint64_t b0 = __ballot(k0 + lane < t.k_end && m0 != 0), b1 = __ballot(k0 + 64 + lane < t.k_end && m1 != 0);
    if ((b0 & b1) != ~0ull)
#pragma unroll
      for (int i = 0; i < L::NI; ++i) idx[i] = ((ld.row(i) < 64 ? b0 : b1) >> (ld.row(i) & 63)) & 1 ? idx[i] : -1;
    const uint64_t bits = ((wave < 2 ? b0 : b1) >> (32 * (wave & 1))) & all_keys<32>();
    ld.load(k, a.ldk, a.d, idx, lds);
    __builtin_amdgcn_sched_barrier(0);
    ld.load(v, a.ldv, a.d, idx, lds + TB);
    vm_wait();
    __syncthreads();
    if (bits == 0) continue;
    f32x16 s, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
    for (int st = 0; st < NS; ++st) {
      s = step_mma<T>(*reinterpret_cast<const uint4*>(kt + unit_at<U>(32 * wave + l32, 2 * st + h)), qf[st], s);
      dp = step_mma<T>(*reinterpret_cast<const uint4*>(vt + unit_at<U>(32 * wave + l32, 2 * st + h)), df[st], dp);
      if (st % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // (registers)
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -ref)) * (dp[r] - delta);
    if (bits != all_keys<32>())
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = key_in(bits, 0, r) ? s[r] : 0.f;
    across_mma<T, U, DB>(kt, 32 * wave, Probs<T>(s), dq, lane);
  }
  // [wave][row][DP], the 16-byte units of a row in an order of its own
  float* sums = reinterpret_cast<float*>(lds);
  const auto at = [&](int w, int r, int u) { return sums + ((w * 32 + r) * (DP / 4) + (u ^ (r & 7))) * 4; };
  __syncthreads();
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<float4*>(at(wave, l32, 8 * db + 2 * j + h)) =
          make_float4(dq[db][4 * j], dq[db][4 * j + 1], dq[db][4 * j + 2], dq[db][4 * j + 3]);
  __syncthreads();
  const int r = threadIdx.x >> 3;
  if (r >= t.rows) return;
  const Virtual vr(a, t.entry, t.head0, t.kv_head, r);
  const int row = row_of(a.q_row, vr.entry);
  const bool none = a.lse[(int64_t)row * a.heads + vr.head] == -INFINITY;  // a row without keys, whatever q and dout hold
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    const int u = 8 * db + (threadIdx.x & 7);
    float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float4 y = *reinterpret_cast<const float4*>(at(w, r, u));
      x[0] += y.x;
      x[1] += y.y;
      x[2] += y.z;
      x[3] += y.w;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = none ? 0.f : x[e];
    if (t.slot >= 0) {
      *reinterpret_cast<float4*>(a.part + (size_t)t.slot * slot_floats<DP>(kCrossRows) + r * DP + 4 * u) =
          make_float4(x[0], x[1], x[2], x[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] *= a.scale;
      store4<T, VEC>(static_cast<T*>(a.out) + (int64_t)row * a.ldo + vr.head * a.d, x, 4 * u, a.d);
    }
  }
}

// The queries' gradient: as the forward with four waves, p recomputed from lse, dq^T += k^T ds^T.
template <typename T, int DP, int TK, bool VEC>
__device__ __forceinline__ void queries_back(const QTile* tiles, unsigned index, const Args& a, char* lds) {
  constexpr int U = DP * (int)sizeof(T) / 16, NS = U / 2, DB = DP / 32, KB = TK / 32, TB = tile_bytes<TK, T, DP>();
  constexpr int E = 16 / (int)sizeof(T), BUF = 2 * TB;
  const QTile t = tile_of_head(tiles, index, a);
  if (t.rows == 0) return;
  if constexpr (DP * sizeof(T) <= 384 && (VEC || DP < 128))  // (the widest heads leave no registers for a second way)
    if (t.rows <= 32) return queries_back_few<T, DP, VEC>(t, a, lds);
  const int lane = threadIdx.x & 63, wave = wave_id(), h = lane >> 5, l32 = lane & 31;
  const T* k = static_cast<const T*>(a.k) + t.kv_head * a.d;
  const T* v = static_cast<const T*>(a.v) + t.kv_head * a.d;
  const int first = 32 * wave;
  const bool active = first < t.rows;
  const Virtual vr(a, t.entry, t.head0, t.kv_head, min(first + l32, t.rows - 1));
  const int qrow = row_of(a.q_row, vr.entry);
  uint4 qf[NS], df[NS];
  {
    const T* q = row_at(static_cast<const T*>(a.q), qrow, a.ldq) + vr.head * a.d;
    const T* g = row_at(static_cast<const T*>(a.dout), qrow, a.lddo) + vr.head * a.d;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      qf[s] = row_unit<T, VEC>(q, (2 * s + h) * E, a.d);
      df[s] = row_unit<T, VEC>(g, (2 * s + h) * E, a.d);
    }
  }
  const int64_t stat = (int64_t)qrow * a.heads + vr.head;
  float delta = a.delta[stat];
  const float lse = a.lse[stat];
  float ref = lse == -INFINITY ? INFINITY : lse * kLog2e;
  f32x16 dq[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[db][r] = 0.f;
  const float c = a.scale * kLog2e;
  using L = TileLoader<T, DP, TK, 4, VEC>;
  const L ld(wave, lane);
  const int ntile = (t.k_end - t.k_begin + TK - 1) / TK;
  KeyFeed<T, DP, TK, 4, VEC> feed(a, t, ld);
  auto issue = [&](int tile) { return feed.issue(tile, k, v, lds + (tile & 1) * BUF, lds + (tile & 1) * BUF + TB); };
  uint64_t bits = 0;
  if (ntile > 0) feed.fetch(0);
  arrived(qf);
  arrived(df);
  arrived(ref);
  arrived(delta);
  if (ntile > 0) {
    bits = issue(0);
    if (ntile > 1) feed.fetch(1);
  }
  for (int at = 0; at < ntile; ++at) {
    const uint64_t now = bits;
    vm_wait();
    __syncthreads();
    if (at + 1 < ntile) {
      bits = issue(at + 1);
      if (at + 2 < ntile) feed.fetch(at + 2);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (!active) continue;
    const char *kt = lds + (at & 1) * BUF, *vt = kt + TB;
#pragma unroll(DP * sizeof(T) == 128 ? 1 : KB)  // (168 registers a lane)
    for (int kb = 0; kb < KB; ++kb) {
      f32x16 s, dp;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        s = step_mma<T>(*reinterpret_cast<const uint4*>(kt + unit_at<U>(32 * kb + l32, 2 * st + h)), qf[st], s);
        dp = step_mma<T>(*reinterpret_cast<const uint4*>(vt + unit_at<U>(32 * kb + l32, 2 * st + h)), df[st], dp);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -ref)) * (dp[r] - delta);
      if (now != all_keys<TK>())
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = key_in(now, kb, r) ? s[r] : 0.f;
      across_mma<T, U, DB>(kt, 32 * kb, Probs<T>(s), dq, lane);
    }
  }
  __syncthreads();  // the images lie where the tiles were
  if (!active) return;
  if (lse == -INFINITY)  // a row without keys, whatever q and dout hold
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) dq[db][r] = 0.f;
  if (t.slot >= 0) {
    if (first + l32 >= t.rows) return;
    float* p = a.part + (size_t)t.slot * slot_floats<DP>(kCrossRows);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(p + (first + l32) * DP + 32 * db + 8 * j + 4 * h) =
            make_float4(dq[db][4 * j], dq[db][4 * j + 1], dq[db][4 * j + 2], dq[db][4 * j + 3]);
    return;
  }
  store_image<T, DP, VEC>(dq, a.scale, a.d, lds + wave * image_bytes<T, DP>(), lane, [&](int r) -> T* {
    if (first + r >= t.rows) return nullptr;
    const Virtual x(a, t.entry, t.head0, t.kv_head, first + r);
    return static_cast<T*>(a.out) + (int64_t)row_of(a.q_row, x.entry) * a.ldo + x.head * a.d;
  });
}

// The gradient of keys and values: a wave holds 32 keys on its lanes, k and v in registers, and walks the row tiles of the
// sequences that read them: dv^T += do^T p, dk^T += q^T ds.
template <typename T, int DP, int RQ, bool VEC>
__device__ __forceinline__ void keys_back(const KTile* tiles, const RTile* runs, unsigned index, const Args& a,
                                          BackLds<T, DP, RQ>& mem) {
  constexpr int U = DP * (int)sizeof(T) / 16, NS = U / 2, DB = DP / 32, QB = RQ / 32, TB = tile_bytes<RQ, T, DP>();
  constexpr int E = 16 / (int)sizeof(T), BUF = 2 * TB;
  constexpr bool KEEP = keep_values<T, DP>();
  char* lds = mem.tiles;
  auto& stats = mem.stats;
  auto& kept = mem.kept;
  const KTile t = tile_of_head(tiles, index, a);
  if (t.keys == 0) return;
  const int lane = threadIdx.x & 63, wave = wave_id(), h = lane >> 5, l32 = lane & 31;
  const int first = 32 * wave, mykey = first + l32;
  const bool active = first < t.keys;
  const int ke = t.k_begin + min(mykey, t.keys - 1);
  uint4 kf[NS], vf[KEEP ? 1 : NS];
  {
    const int krow = row_of(a.k_row, ke);
    const T* k = row_at(static_cast<const T*>(a.k), krow, a.ldk) + t.kv_head * a.d;
    const T* v = row_at(static_cast<const T*>(a.v), krow, a.ldv) + t.kv_head * a.d;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      kf[s] = row_unit<T, VEC>(k, (2 * s + h) * E, a.d);
      vf[KEEP ? 0 : s] = row_unit<T, VEC>(v, (2 * s + h) * E, a.d);
      if constexpr (KEEP) kept[(wave * NS + s) * 64 + lane] = vf[0];
    }
  }
  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) dk[db][r] = dv[db][r] = 0.f;
  const float c = a.scale * kLog2e;
  using L = TileLoader<T, DP, RQ, 4, VEC>;
  // (the lane's places are worked out again for every tile: registers are short in the loop)
  const auto loader = [&]() {
    int l = lane;
    arrived(l);
    return L(wave, l);
  };
  const T *q = static_cast<const T*>(a.q), *g = static_cast<const T*>(a.dout);
  // A row tile's row numbers are fetched while the tile two before it is multiplied, what they lead to (the loads into LDS,
  // lse and delta) a tile later, as in KeyFeed; wave 0's lanes also hold a row each for lse and delta.
  int idx[L::NI], head[L::NI], stat_row = 0, stat_head = 0, nrows = 0;
  float lse = 0.f, delta = 0.f;  // of row `lane` of the tile that was issued last
  bool there = false;
  RTile next = t.t_begin < t.t_end ? runs[t.t_begin] : RTile{};
  auto fetch = [&](int tile) {  // and the list's entry of the tile after it
    const L ld = loader();
    RTile rt;
    rt.entry = __builtin_amdgcn_readfirstlane(next.entry);
    rt.head0 = __builtin_amdgcn_readfirstlane(next.head0);
    rt.rows = __builtin_amdgcn_readfirstlane(next.rows);
    next = runs[min(tile + 1, t.t_end - 1)];
    nrows = rt.rows;
#pragma unroll
    for (int i = 0; i < L::NI; ++i) {
      const Virtual vr(a, rt.entry, rt.head0, t.kv_head, min(ld.row(i), rt.rows - 1));
      head[i] = vr.head * a.d;
      idx[i] = row_of(a.q_row, vr.entry);
    }
    if (wave == 0) {
      const Virtual vr(a, rt.entry, rt.head0, t.kv_head, min(lane & (RQ - 1), rt.rows - 1));
      stat_row = row_of(a.q_row, vr.entry);
      stat_head = vr.head;
    }
  };
  auto issue = [&](int buf) {
#pragma unroll
    for (int i = 0; i < L::NI; ++i) arrived(idx[i]);
    arrived(stat_row);
    const L ld = loader();
    char* to = lds + buf * BUF;
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < L::NI; ++i) {
        const int e0 = ld.unit(i) * E;
        const bool in = ld.row(i) < nrows && e0 < a.d;
        const void* z = g_zero;
        dma16_untracked(in ? row_at(q, idx[i], a.ldq) + head[i] + e0 : z, to + (ld.part * L::NI + i) * 1024);
        dma16_untracked(in ? row_at(g, idx[i], a.lddo) + head[i] + e0 : z, to + TB + (ld.part * L::NI + i) * 1024);
      }
    } else {
#pragma unroll
      for (int i = 0; i < L::NI; ++i) {
        uint4 x = make_uint4(0, 0, 0, 0), y = x;
        if (ld.row(i) < nrows) {
          x = row_unit<T, false>(row_at(q, idx[i], a.ldq) + head[i], ld.unit(i) * E, a.d);
          y = row_unit<T, false>(row_at(g, idx[i], a.lddo) + head[i], ld.unit(i) * E, a.d);
        }
        *reinterpret_cast<uint4*>(to + ld.place(i) * 16) = x;
        *reinterpret_cast<uint4*>(to + TB + ld.place(i) * 16) = y;
      }
    }
    if (wave == 0) {
      const int64_t at = (int64_t)stat_row * a.heads + stat_head;
      lse = a.lse[at];
      delta = a.delta[at];
      there = (lane & (RQ - 1)) < nrows;
    }
  };
  if (t.t_begin < t.t_end) fetch(t.t_begin);
  arrived(kf);
  if constexpr (!KEEP) arrived(vf);
  if (t.t_begin < t.t_end) {
    issue(0);
    if (t.t_begin + 1 < t.t_end) fetch(t.t_begin + 1);
  }
  for (int at = t.t_begin; at < t.t_end; ++at) {
    const int buf = (at - t.t_begin) & 1;
    if (wave == 0 && lane < RQ) {
      stats[buf][0][lane] = there && lse != -INFINITY ? lse * kLog2e : INFINITY;  // no row: p = 0
      stats[buf][1][lane] = there ? delta : 0.f;
    }
    vm_wait();
    __syncthreads();
    if (at + 1 < t.t_end) {
      issue(buf ^ 1);
      if (at + 2 < t.t_end) fetch(at + 2);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (!active) continue;
    const char *qt = lds + buf * BUF, *gt = qt + TB;
#pragma unroll 1
    for (int qb = 0; qb < QB; ++qb) {
      f32x16 s, dp;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
      for (int st = 0; st < NS; ++st) {
        s = step_mma<T>(*reinterpret_cast<const uint4*>(qt + unit_at<U>(32 * qb + l32, 2 * st + h)), kf[st], s);
        dp = step_mma<T>(*reinterpret_cast<const uint4*>(gt + unit_at<U>(32 * qb + l32, 2 * st + h)),
                         KEEP ? kept[(wave * NS + st) * 64 + lane] : vf[KEEP ? 0 : st], dp);
        if constexpr (KEEP)
          if (st % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // four steps' fragments in registers at a time
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 m = *reinterpret_cast<const float4*>(&stats[buf][0][32 * qb + 8 * j + 4 * h]);
        const float4 dl = *reinterpret_cast<const float4*>(&stats[buf][1][32 * qb + 8 * j + 4 * h]);
        const float ref[4] = {m.x, m.y, m.z, m.w}, del[4] = {dl.x, dl.y, dl.z, dl.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * j + e], c, -ref[e]));
          s[4 * j + e] = p;
          dp[4 * j + e] = p * (dp[4 * j + e] - del[e]);
        }
      }
      across_mma<T, U, DB>(gt, 32 * qb, Probs<T>(s), dv, lane);
      across_mma<T, U, DB>(qt, 32 * qb, Probs<T>(dp), dk, lane);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __syncthreads();  // the images lie where the tiles were
  if (!active) return;
  if (t.slot >= 0) {
    if (mykey >= t.keys) return;
    float* p = a.part + ((size_t)t.slot * kCrossKeys + mykey) * 2 * DP;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d0 = 32 * db + 8 * j + 4 * h;
        *reinterpret_cast<float4*>(p + d0) = make_float4(dk[db][4 * j], dk[db][4 * j + 1], dk[db][4 * j + 2], dk[db][4 * j + 3]);
        *reinterpret_cast<float4*>(p + DP + d0) =
            make_float4(dv[db][4 * j], dv[db][4 * j + 1], dv[db][4 * j + 2], dv[db][4 * j + 3]);
      }
    return;
  }
  if (a.mask && a.mask[ke] == 0)  // a key that does not count, whatever its row holds
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) dk[db][r] = dv[db][r] = 0.f;
  char* img = lds + wave * image_bytes<T, DP>();
  const auto place = [&](void* to, int64_t ldt) {
    return [=, &a, &t](int r) -> T* {
      if (first + r >= t.keys) return nullptr;
      return static_cast<T*>(to) + (int64_t)row_of(a.k_row, t.k_begin + first + r) * ldt + t.kv_head * a.d;
    };
  };
  if (a.out) store_image<T, DP, VEC>(dk, a.scale, a.d, img, lane, place(a.out, a.ldo));
  if (a.out2) store_image<T, DP, VEC>(dv, 1.f, a.d, img, lane, place(a.out2, a.ldo2));
}

// Both gradients in one launch: `nkeys` workgroups for the keys', the rest for the queries', which fill the end.  In two launches
// 16 sources of 3 .. 127 keys in fp32 took 86 us where one took 65, 64 chains of 16 heads 396 and 386.
template <typename T, int DP, int TK, bool VEC>
__global__ __launch_bounds__(kThreads, (waves_back<T, DP>())) void k_cross_back(const KTile* keys, const RTile* runs,
                                                                                        unsigned nkeys, Args ka,
                                                                                        const QTile* rows, Args qa) {
  typedef BackLds<T, DP, TK> Lds;
  constexpr int FEW = 2 * tile_bytes<128, T, DP>(), SUMS = 4 * 32 * DP * 4, LEAST = FEW > SUMS ? FEW : SUMS;
  __shared__ __attribute__((aligned(16))) char mem[sizeof(Lds) > LEAST ? sizeof(Lds) : LEAST];
  Lds& lds = *reinterpret_cast<Lds*>(mem);
  if (blockIdx.x < nkeys) keys_back<T, DP, TK, VEC>(keys, runs, blockIdx.x, ka, lds);
  else queries_back<T, DP, TK, VEC>(rows, blockIdx.x - nkeys, qa, mem);
}

// The pieces of a tile of keys summed in their order: eight threads a key, 32 keys a workgroup, eight pieces in flight; the
// launch's third dimension is dk and dv.
template <typename T, int DP, bool VEC>
__global__ __launch_bounds__(kThreads) void k_cross_join_keys(const KTile* tiles, Args a) {
  constexpr int BLOCKS = kCrossKeys / 32, F = 8;
  const KTile t = tile_of_head(tiles, blockIdx.x / BLOCKS, a);
  const int c0 = (threadIdx.x & 7) * 4, key = blockIdx.x % BLOCKS * 32 + (threadIdx.x >> 3), which = blockIdx.z;
  T* to = static_cast<T*>(which ? a.out2 : a.out);
  if (key >= t.keys || !to) return;
  const int ke = t.k_begin + key, krow = row_of(a.k_row, ke);
  const bool counts = !a.mask || a.mask[ke] != 0;
  to += (int64_t)krow * (which ? a.ldo2 : a.ldo) + t.kv_head * a.d;
  const float* p = a.part + ((size_t)t.slot * kCrossKeys + key) * 2 * DP + which * DP;
  for (int d0 = c0; d0 < DP; d0 += 32) {
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < t.pieces; i0 += F) {
      float4 y[F];
#pragma unroll
      for (int u = 0; u < F; ++u)
        y[u] = *reinterpret_cast<const float4*>(p + (size_t)min(i0 + u, t.pieces - 1) * kCrossKeys * 2 * DP + d0);
#pragma unroll
      for (int u = 0; u < F; ++u) {
        if (i0 + u >= t.pieces) break;
        x[0] += y[u].x;
        x[1] += y[u].y;
        x[2] += y[u].z;
        x[3] += y[u].w;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = counts ? x[e] * (which ? 1.f : a.scale) : 0.f;
    store4<T, VEC>(to, x, d0, a.d);
  }
}

// ---- launches ---------------------------------------------------------------------------------------------------------

template <typename T, int DP_>
struct Width {
  typedef T type;
  static constexpr int DP = DP_;
};
// f(Width<T, DP>) for the width that holds the heads
template <class F>
void with_width(int dtype, int d, F&& f) {
  const auto pick = [&](auto zero) {
    typedef decltype(zero) T;
    if (d <= 32) f(Width<T, 32>());
    else if (d <= 64) f(Width<T, 64>());
    else if (d <= 96) f(Width<T, 96>());
    else f(Width<T, 128>());
  };
  if (dtype == FOLD_F32) pick(float());
  else pick(uint16_t());
}
// whether the heads' rows of a matrix lie at multiples of 16 bytes
bool whole_units(const CrossMat& m, int d, int es) {
  return !m.p || ((reinterpret_cast<uintptr_t>(m.p) & 15) == 0 && m.ld * es % 16 == 0 && d * es % 16 == 0);
}

Args args_of(const Cross& c, const CrossMat& q, const CrossMat& k, const CrossMat& v, const uint8_t* mask, float scale) {
  Args a{};
  a.q = q.p;
  a.k = k.p;
  a.v = v.p;
  const int es = c.dtype == FOLD_BF16 ? 2 : 4;
  a.ldq = (uint32_t)(q.ld * es);
  a.ldk = (uint32_t)(k.ld * es);
  a.ldv = (uint32_t)(v.ld * es);
  a.q_row = c.q_row;
  a.k_row = c.k_row;
  a.mask = mask;
  a.scale = scale;
  a.heads = c.heads;
  a.group = c.group;
  a.d = c.head_dim;
  a.magic = (1u << 20) / (unsigned)c.group + 1;
  return a;
}

}  // namespace

size_t cross_forward_bytes(const Cross& c) {
  return (size_t)c.fslots * c.kv_heads * (c.few ? kCrossFew : kCrossRows) * (cross_padded(c.head_dim) + 2) * sizeof(float);
}
static size_t delta_floats(const Cross& c) { return ((size_t)c.query_rows * c.heads + 3) / 4 * 4; }
static size_t dq_floats(const Cross& c) {
  return (size_t)c.bslots * c.kv_heads * kCrossRows * (cross_padded(c.head_dim) + 2);
}
size_t cross_backward_bytes(const Cross& c) {
  const size_t dk = (size_t)c.kslots * c.kv_heads * kCrossKeys * 2 * cross_padded(c.head_dim);
  return (delta_floats(c) + dq_floats(c) + dk) * sizeof(float);
}

void launch_cross(const Cross& c, CrossMat q, CrossMat k, CrossMat v, const uint8_t* mask, float scale, void* out,
                  int64_t ldo, float* lse, void* ws, hipStream_t st) {
  if (c.nfwd == 0) return;
  Args a = args_of(c, q, k, v, mask, scale);
  a.out = out;
  a.ldo = ldo;
  a.lse = lse;
  a.slots = c.fslots;
  a.part = static_cast<float*>(ws);
  const int es = c.dtype == FOLD_BF16 ? 2 : 4, d = c.head_dim;
  const bool vec = whole_units(q, d, es) && whole_units(k, d, es) && whole_units(v, d, es) && whole_units({out, ldo}, d, es);
  with_width(c.dtype, d, [&](auto w) {
    typedef typename decltype(w)::type T;
    constexpr int DP = decltype(w)::DP, TK = sizeof(T) == 2 ? 64 : 32;
    const auto go = [&](auto vector) {
      constexpr bool VEC = decltype(vector)::value;
      {
        ProfScope prof("cross", st);
        if constexpr (DP * sizeof(T) <= kCrossFewBytes)
          if (c.few) hipLaunchKernelGGL((k_cross<T, DP, 32, 1, VEC>), dim3(c.nfwd, c.kv_heads), dim3(kThreads), 0, st, c.fwd, a);
        if (!c.few) hipLaunchKernelGGL((k_cross<T, DP, TK, 4, VEC>), dim3(c.nfwd, c.kv_heads), dim3(kThreads), 0, st, c.fwd, a);
      }
      if (c.nfjoin == 0) return;
      ProfScope prof("cross_join", st);
      if (c.few)
        hipLaunchKernelGGL((k_cross_join<T, DP, kCrossFew, true, VEC>), dim3(c.nfjoin, c.kv_heads), dim3(kThreads), 0, st, c.fjoin, a);
      else
        hipLaunchKernelGGL((k_cross_join<T, DP, kCrossRows, true, VEC>), dim3(c.nfjoin * (kCrossRows / 32), c.kv_heads), dim3(kThreads), 0, st, c.fjoin, a);
    };
    if (vec) go(std::true_type());
    else go(std::false_type());
  });
}

void launch_cross_backward(const Cross& c, CrossMat q, CrossMat k, CrossMat v, const uint8_t* mask, float scale, CrossMat out,
                           const float* lse, CrossMat dout, void* dq, int64_t lddq, void* dk, int64_t lddk, void* dv,
                           int64_t lddv, void* ws, hipStream_t st) {
  Args a = args_of(c, q, k, v, mask, scale);
  a.dout = dout.p;
  a.lddo = (uint32_t)(dout.ld * (c.dtype == FOLD_BF16 ? 2 : 4));
  a.lse = const_cast<float*>(lse);
  float* delta = static_cast<float*>(ws);
  a.delta = delta;
  a.part = delta + delta_floats(c);
  const int es = c.dtype == FOLD_BF16 ? 2 : 4, d = c.head_dim;
  const bool vec = whole_units(q, d, es) && whole_units(k, d, es) && whole_units(v, d, es) && whole_units(out, d, es) &&
                   whole_units(dout, d, es) && whole_units({dq, lddq}, d, es) && whole_units({dk, lddk}, d, es) &&
                   whole_units({dv, lddv}, d, es);
  with_width(c.dtype, d, [&](auto w) {
    typedef typename decltype(w)::type T;
    constexpr int DP = decltype(w)::DP, TK = sizeof(T) == 2 ? 64 : 32;
    const auto go = [&](auto vector) {
      constexpr bool VEC = decltype(vector)::value;
      const DeltaArgs da{out.p, dout.p, out.ld, dout.ld, c.q_row, c.others, (int64_t)c.nothers * c.heads, c.heads, d, delta};
      const int64_t blocks = std::min<int64_t>((da.n + 31) / 32, 1 << 20);
      if (c.nbrief > 0) {
        ProfScope prof("cross_delta", st);
        const int64_t more = std::min<int64_t>((blocks + c.kv_heads - 1) / c.kv_heads, kMaxTiles - c.nbrief);
        hipLaunchKernelGGL((k_cross_delta_brief<T, DP, VEC>), dim3((unsigned)(c.nbrief + more), c.kv_heads), dim3(kThreads), 0, st,
                           c.brief, (unsigned)c.nbrief, a, da);
      } else if (blocks > 0) {
        ProfScope prof("cross_delta", st);
        hipLaunchKernelGGL((k_cross_delta<T, VEC>), dim3((unsigned)blocks), dim3(kThreads), 0, st, da);
      }
      const bool rows = dq && c.nback > 0, keys = (dk || dv) && c.nkeys > 0;
      Args qa = a, ka = a;
      qa.out = dq;
      qa.slots = c.bslots;
      qa.ldo = lddq;
      ka.out = dk;
      ka.slots = c.kslots;
      ka.ldo = lddk;
      ka.out2 = dv;
      ka.ldo2 = lddv;
      ka.part = a.part + dq_floats(c);
      const unsigned nk = keys ? c.nkeys : 0, nq = rows ? c.nback : 0;
      if (nk + nq > 0) {
        ProfScope prof("cross_back", st);
        hipLaunchKernelGGL((k_cross_back<T, DP, TK, VEC>), dim3(nk + nq, c.kv_heads), dim3(kThreads), 0, st, c.keys, c.rows, nk,
                           ka, c.back, qa);
      }
      if (rows && c.nbjoin > 0) {
        ProfScope prof("cross_dq_join", st);
        hipLaunchKernelGGL((k_cross_join<T, DP, kCrossRows, false, VEC>), dim3(c.nbjoin * (kCrossRows / 32), c.kv_heads), dim3(kThreads), 0, st, c.bjoin, qa);
      }
      if (keys && c.nkjoin > 0) {
        ProfScope prof("cross_dkv_join", st);
        hipLaunchKernelGGL((k_cross_join_keys<T, DP, VEC>), dim3(c.nkjoin * (kCrossKeys / 32), c.kv_heads, 2), dim3(kThreads), 0, st, c.kjoin, ka);
      }
    };
    if (vec) go(std::true_type());
    else go(std::false_type());
  });
}

}  // namespace fold
