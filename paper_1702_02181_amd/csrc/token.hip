// Row operators over the logits of a vocabulary head (gfx950): log probabilities of given tokens with the entropy and
// the top alternatives of every row, and the distillation loss with its gradient.
//
// A row of V logits is read in 16-byte vectors.  Its softmax is kept in base 2: with L = log2 e and a reference m2,
// x = z L - m2 (one fma: every term of a row sees the same rounded m2, which cancels in p and in log p),
// s = sum 2^x, and for the entropy t = sum 2^x x.  Then log p = ln 2 (x - log2 s) and H = ln 2 (log2 s - t / s).
// Partial (m2, s, t) of threads, waves and segments of a row meet by the usual rescaling; all of it is fp32.
//
// m2 is the maximum's z L, rounded: the maximum's own x is that rounding's error, at most 1/2 while |m2| <= kScaled, but
// 440 at a maximum of 1e10, where 2^x is no longer finite.  So references are clamped to +-kScaled: what lies far below
// (whole vectors masked by -1e9, -1e30 or the type's lowest value) then has finite terms, which
// vanish beside larger logits as they should.  A row, or a segment of one, whose largest logit itself lies outside (`far`) is
// read once more, with x = (z - m) L: the difference is rounded by itself, so m's term is an exact 1.
// NaN reaches s by itself (the maximum ignores NaN); +inf and NaN make the row's results NaN; a row of -inf alone is
// empty.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "common.h"
#include "internal.h"
#include "mfma.h"

namespace fold {

namespace {

constexpr float kL2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kScaled = 16777216.f;  // 2^24, the largest reference: see above
constexpr float kNear = kScaled / kL2E;  // the largest |z| whose reference is not clamped, at temperature 1
constexpr float kFloor = -200.f;   // 2^-200 is 0 in fp32: bounds x where it is multiplied by 2^x
constexpr int kThreads = 256, kWaves = kThreads / 64;  // of a workgroup, where nothing else is said
constexpr int kUnroll = 4;         // vectors a thread has in flight
constexpr int kCap = 1024;         // candidates of a segment's top list held in LDS
constexpr int kMaxSegments = 64;   // of a row: a lane each

__device__ __forceinline__ float neg_inf() { return -__builtin_inff(); }
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_(float x) { return __builtin_amdgcn_logf(x); }

template <typename T>
__device__ __forceinline__ void unpack(uint4 r, float (&v)[16 / sizeof(T)]) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
__device__ __forceinline__ float wave_add(float v) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
  return v;
}
// over a workgroup of NW waves; red holds NW floats and is free again after the next barrier
template <int NW, class OP>
__device__ __forceinline__ float block_fold(float v, float* red, OP op) {
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float r = red[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) r = op(r, red[w]);
  return r;
}
template <int NW>
__device__ __forceinline__ float block_max(float v, float* red) {
  return block_fold<NW>(wave_max(v), red, [](float a, float b) { return fmaxf(a, b); });
}
template <int NW>
__device__ __forceinline__ float block_add(float v, float* red) {
  return block_fold<NW>(wave_add(v), red, [](float a, float b) { return a + b; });
}

// Order of the logits as whole numbers: larger is larger, -0 equals +0; with the column below it, the lowest index of
// equal logits is the largest key.  0 is no key.
__device__ __forceinline__ uint32_t order_of(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t o) {
  return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ uint64_t key_of(float z, int col) {
  return ((uint64_t)order_of(z) << 32) | (0xffffffffu - (uint32_t)col);
}

// One segment of a row: vectors [v0, v1) of the row, whose V columns end inside vector (V - 1) / VEC.
template <typename T>
struct Segment {
  static constexpr int VEC = 16 / sizeof(T);
  const uint4* row;
  int v0, v1, V;

  // f(vector index, its values, the number of them that are real), for every vector a thread has: kUnroll loads in flight,
  // from clamped addresses
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    for (int b = v0; b < v1; b += kThreads * kUnroll) {
      uint4 raw[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) raw[u] = row[min(b + u * kThreads + (int)threadIdx.x, v1 - 1)];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const int i = b + u * kThreads + (int)threadIdx.x;
        float v[VEC];
        unpack<T>(raw[u], v);
        f(i, v, i < v1 ? min(VEC, V - i * VEC) : 0);
      }
    }
  }

  // f(first vector, group of `kUnroll` vectors' values) while whole groups are left, then f1(vector, values) for the rest
  // one vector at a time, columns that are not there as -inf.  The groups need no test for the end.
  template <class F, class F1>
  __device__ __forceinline__ void groups(F&& f, F1&& f1) const {
    int b = v0;
    for (; b + kThreads * kUnroll < v1; b += kThreads * kUnroll) {
      uint4 raw[kUnroll];
      float v[kUnroll][VEC];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) raw[u] = row[b + u * kThreads + (int)threadIdx.x];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) unpack<T>(raw[u], v[u]);
      f(b + (int)threadIdx.x, v);
    }
    uint4 raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (b + u * kThreads < v1) raw[u] = row[min(b + u * kThreads + (int)threadIdx.x, v1 - 1)];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (b + u * kThreads >= v1) continue;
      const int i = b + u * kThreads + (int)threadIdx.x, have = i < v1 ? V - i * VEC : 0;
      float v[VEC];
      unpack<T>(raw[u], v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = e < have ? v[e] : neg_inf();
      f1(i, v);
    }
  }
};

template <int N>
__device__ __forceinline__ float max_of(const float (&v)[N]) {
  float m = v[0];
#pragma unroll
  for (int e = 1; e < N; ++e) m = fmaxf(m, v[e]);
  return m;
}

__host__ __device__ inline int vectors_of(int V, int vec) { return (V + vec - 1) / vec; }

template <typename T>
__device__ __forceinline__ Segment<T> segment_of(const T* z, size_t ld, int64_t p, int seg, int nseg, int V) {
  // pieces of whole 64-column blocks, so that a gradient of another type splits at the same columns; the last ones may
  // be empty
  const int nv = vectors_of(V, (16 / (int)sizeof(T))), block = 64 / (16 / (int)sizeof(T));
  const int per = ((nv + nseg - 1) / nseg + block - 1) / block * block;
  Segment<T> s;
  s.row = reinterpret_cast<const uint4*>(z + (size_t)p * ld);
  s.v0 = min(seg * per, nv);
  s.v1 = min(s.v0 + per, nv);
  s.V = V;
  return s;
}

// Softmax state of some logits of a row: the largest, the reference (in units of log2), sum 2^x, sum 2^x x.
struct Stat {
  float m, m2, s, t;
};

// The reference of a maximum at a factor c = L / T; near: kScaled over the largest factor of the row's sums.
// Rounded here: fused into the subtraction that follows, two references of the same maximum would differ by the product's
// rounding.
__device__ __forceinline__ float ref_of(float m, float c, float near) {
#pragma clang fp contract(off)
  return fminf(fmaxf(m, -near), near) * c;
}
__device__ __forceinline__ bool is_far(float m, float near) { return fabsf(m) > near && m != neg_inf(); }
// x of a logit seen from a far maximum: z - m rounded by itself
__device__ __forceinline__ float far_x(float z, float m, float c) {
#pragma clang fp contract(off)
  return (z - m) * c;
}

// s and t seen from a reference that is d lower than theirs
__device__ __forceinline__ void shift(Stat& a, float d) {
  const float f = exp2_(d);
  a.t = f * (a.t + fmaxf(d, kFloor) * a.s);
  a.s = f * a.s;
}
__device__ __forceinline__ void rebase(Stat& a, float m2) {
  shift(a, a.m2 - m2);
  a.m2 = m2;
}

// What a segment's sums are shifted by when it joins a row: the segment's largest logit m, the row's `row` >= m.  Near
// maxima refer to their rounded reference, far ones to themselves; one rounding in either case.  A segment without a
// logit above -inf has sums of 0 (or NaN) and stays as it is.
__device__ __forceinline__ float join_shift(float m, float row, float c, float near) {
  if (m == neg_inf()) return 0.f;
  const bool far = is_far(m, near);
  if (is_far(row, near)) return far ? far_x(m, row, c) : -__builtin_fmaf(row, c, -ref_of(m, c, near));
  return far ? __builtin_fmaf(m, c, -ref_of(row, c, near)) : ref_of(m, c, near) - ref_of(row, c, near);
}

// The state of a whole row from that of its segments: `bad` for NaN or +inf, `empty` for -inf alone.
struct RowState {
  float m, m2, s, t;
  bool bad, empty, far;
  __device__ __forceinline__ void close() {
    far = is_far(m, kNear);
    bad = !(s == s) || m == __builtin_inff();
    empty = !bad && m == neg_inf();
  }
  // log p of a logit of this row
  __device__ __forceinline__ float logp(float z) const {
    if (bad) return __builtin_nanf("");
    if (empty) return neg_inf();
    if (far || z < -1e30f) return (z - m) - kLn2 * log2_(s);
    return kLn2 * (__builtin_fmaf(z, kL2E, -m2) - log2_(s));
  }
  __device__ __forceinline__ float entropy() const {
    if (bad) return __builtin_nanf("");
    if (empty) return 0.f;
    return fmaxf(kLn2 * (log2_(s) - t / s), 0.f);
  }
};

// ---------------------------------------------------------------- top lists

// The K largest keys of cand[0 .. n), in order, into out[0 .. K) (0 where there are fewer).
__device__ __forceinline__ void rank_keys(const uint64_t* cand, int n, int K, uint64_t* out) {
  if ((int)threadIdx.x < K) out[threadIdx.x] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const uint64_t k = cand[i];
    int r = 0;
    for (int j = 0; j < n; ++j) r += cand[j] > k;
    if (r < K) out[r] = k;
  }
  __syncthreads();
}

// What a thread keeps of its vectors for the top list: its largest logit, the first vector of the group that holds it, and
// the largest of its other groups.
struct Best {
  float m, second;
  int first;
  __device__ __forceinline__ void meet(int i, float v) {
    const bool more = v > m;
    second = fmaxf(second, more ? m : v);
    first = more ? i : first;
    m = more ? v : m;
  }
};

struct TopLds {
  uint64_t cand[kCap + kMaxTopTokens];
  uint64_t out[kMaxTopTokens];
  uint32_t key[kThreads];
  unsigned hist[256];
  int vec[kCap];
  uint32_t tau;
  int n, vectors, bin, left;
};

// Adds one to hist[b] for every lane with `in`; lanes that all have the same bin add once (a row of equal logits).
__device__ __forceinline__ void count_bin(unsigned* hist, int b, bool in) {
  const uint64_t act = __ballot(in);
  if (act == 0) return;
  const int first = __builtin_amdgcn_readlane(b, __builtin_ctzll(act));
  if (__ballot(in && b == first) == act) {
    if ((threadIdx.x & 63) == 0) atomicAdd(&hist[first], (unsigned)__popcll(act));
  } else if (in) {
    atomicAdd(&hist[b], 1u);
  }
}

// The K largest keys of a segment, in order, in s.out.  A threshold first: the K-th largest of the 256 threads' maxima
// cannot exceed the K-th largest logit, and few logits reach it (about K where the large ones are spread over the
// threads).  They are found again by the threads whose maximum reaches it, mostly in the one group of vectors that holds
// it; a thread whose other groups reach it too reads all its vectors again (eight loads in flight).
// Where more than kCap do, either many equal the threshold: then the logits above it are the list's head and the rest is
// filled with the first ones that equal it, in the columns' order, which ends as soon as the list is full.  Or more than
// kCap are above it (all the large ones in few threads' columns): then the K-th largest key is found digit by digit, with
// one read of the segment a digit.
template <typename T>
__device__ void top_of_segment(const Segment<T>& seg, const Best& best, int K, TopLds& s) {
  constexpr int VEC = 16 / (int)sizeof(T), NW = kWaves;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t key = best.m > neg_inf() ? order_of(best.m) : 0u;
  s.key[tid] = key;
  __syncthreads();
  if (wave == 0) {
    uint32_t k[4], t = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) k[w] = s.key[w * 64 + lane];
    for (int b = 31; b >= 0; --b) {
      const uint32_t c = t | (1u << b);
      int n = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) n += __popcll(__ballot(k[w] >= c));
      if (n >= K) {
        t = c;
        if (n == K) break;
      }
    }
    if (lane == 0) s.tau = t;
  }
  __syncthreads();
  const uint32_t tau = s.tau;
  const bool mine = key >= tau && key != 0;
  const bool others = best.second > neg_inf() && order_of(best.second) >= tau;
  // The logits above the threshold, or that reach it, into s.cand [s.n]: first the vectors that hold one, found by the
  // threads whose maximum reaches it, then their logits, a vector a thread.  False if there is no room for all.
  auto collect = [&](bool above) {
    __syncthreads();
    if (tid == 0) s.n = s.vectors = 0;
    __syncthreads();
    auto look = [&](int i, const uint4& raw) __attribute__((always_inline)) {
      float v[VEC];
      unpack<T>(raw, v);
      float vm = neg_inf();
#pragma unroll
      for (int e = 0; e < VEC; ++e) vm = fmaxf(vm, i * VEC + e < seg.V ? v[e] : neg_inf());
      const uint32_t o = order_of(vm);
      if (i < seg.v1 && vm > neg_inf() && (above ? o > tau : o >= tau)) {
        const int at = atomicAdd(&s.vectors, 1);
        if (at < kCap) s.vec[at] = i;
      }
    };
    if (mine && !others) {
      // a group of the main part, or one vector of the rest (the others looked at with it do not reach the threshold)
      uint4 raw[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) raw[u] = seg.row[min(best.first + u * kThreads, seg.v1 - 1)];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) look(best.first + u * kThreads, raw[u]);
    }
    if (mine && others) {
      constexpr int U = 8;
      for (int b = seg.v0 + tid; b < seg.v1; b += kThreads * U) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = seg.row[min(b + u * kThreads, seg.v1 - 1)];
#pragma unroll
        for (int u = 0; u < U; ++u) look(b + u * kThreads, raw[u]);
      }
    }
    __syncthreads();
    const int n = s.vectors;
    if (n > kCap) return false;
    for (int j = tid; j < n; j += kThreads) {
      const int i = s.vec[j];
      float v[VEC];
      unpack<T>(seg.row[i], v);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const uint32_t o = order_of(v[e]);
        if (i * VEC + e < seg.V && v[e] > neg_inf() && (above ? o > tau : o >= tau)) {
          const int at = atomicAdd(&s.n, 1);
          if (at < kCap) s.cand[at] = key_of(v[e], i * VEC + e);
        }
      }
    }
    __syncthreads();
    return s.n <= kCap;
  };
  if (collect(false)) {  // the same for every thread, as below
  } else if (collect(true)) {
    const int above = s.n;
    int need = K - above;  // of the logits that equal the threshold
    for (int b = seg.v0; b < seg.v1 && need > 0; b += kThreads) {
      const int i = b + tid;
      float v[VEC];
      unpack<T>(seg.row[min(i, seg.v1 - 1)], v);
      int c = 0;
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        c += i < seg.v1 && i * VEC + e < seg.V && v[e] > neg_inf() && order_of(v[e]) == tau;
      // place among the chunk's: inclusive sums over the wave, then the waves before
      int before = c;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(before, d);
        before += lane >= d ? o : 0;
      }
      __syncthreads();
      if (lane == 63) s.hist[wave] = before;
      __syncthreads();
      int total = 0;
      before -= c;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        before += w < wave ? (int)s.hist[w] : 0;
        total += (int)s.hist[w];
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (i < seg.v1 && i * VEC + e < seg.V && v[e] > neg_inf() && order_of(v[e]) == tau) {
          if (before < need) s.cand[above + (K - above - need) + before] = key_of(v[e], i * VEC + e);
          ++before;
        }
      need -= min(need, total);
    }
    __syncthreads();
    if (tid == 0) s.n = max(above, K - need);
    __syncthreads();
  } else {
    __syncthreads();
    uint64_t prefix = 0;
    int left = K;
    for (int byte = 7; byte >= 0; --byte) {
      s.hist[tid] = 0;
      __syncthreads();
      seg.each([&](int i, float (&v)[VEC], int nv) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const uint64_t q = key_of(v[e], i * VEC + e);
          const bool same = byte == 7 || (q >> (8 * byte + 8)) == (prefix >> (8 * byte + 8));
          count_bin(s.hist, (int)(q >> (8 * byte)) & 255, e < nv && v[e] > neg_inf() && same);
        }
      });
      __syncthreads();
      if (tid == 0) {
        int b = 255, above = 0;
        while (b > 0 && above + (int)s.hist[b] < left) above += (int)s.hist[b--];
        s.bin = b;
        s.left = left - above;
      }
      __syncthreads();
      prefix |= (uint64_t)s.bin << (8 * byte);
      left = s.left;
      const int upto = K - left + (int)s.hist[s.bin];  // keys not below the prefix
      __syncthreads();
      if (upto <= kCap) break;
    }
    if (tid == 0) s.n = 0;
    __syncthreads();
    seg.each([&](int i, float (&v)[VEC], int nv) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const uint64_t q = key_of(v[e], i * VEC + e);
        if (e < nv && v[e] > neg_inf() && q >= prefix) {
          const int at = atomicAdd(&s.n, 1);
          if (at < kCap) s.cand[at] = q;
        }
      }
    });
    __syncthreads();
  }
  rank_keys(s.cand, min(s.n, kCap), K, s.out);
}

// ---------------------------------------------------------------- log probabilities

struct TokenArgs {
  int64_t row0;      // first row of this launch
  const int* order;  // row p's tokens and results are at order[p] (NULL: p)
  const void* logits;
  size_t ld;
  int V, J, K, nseg;
  const int* tokens;
  float *logp, *entropy;
  int* top_token;
  float* top_logp;
  Stat* part;          // [rows][nseg]
  uint64_t* part_key;  // [rows][nseg][K]
};

// One row's results from its state and its K sorted keys
template <typename T>
__device__ __forceinline__ void write_row(const TokenArgs& a, int64_t p, const RowState& r, const uint64_t* keys) {
  const size_t q = a.order ? (size_t)a.order[p] : (size_t)p;
  const T* row = static_cast<const T*>(a.logits) + (size_t)p * a.ld;
  for (int j = threadIdx.x; j < a.J; j += kThreads) {
    const int tok = a.tokens[q * a.J + j];
    a.logp[q * a.J + j] = tok >= 0 && tok < a.V ? r.logp(to_f32<T>(row[tok])) : 0.f;
  }
  if (threadIdx.x == 0 && a.entropy) a.entropy[q] = r.entropy();
  if ((int)threadIdx.x < a.K) {
    const uint64_t k = keys[threadIdx.x];
    const bool none = k == 0 || r.bad;
    a.top_token[q * a.K + threadIdx.x] = none ? -1 : (int)(0xffffffffu - (uint32_t)k);
    a.top_logp[q * a.K + threadIdx.x] = none && !r.bad ? neg_inf() : r.logp(logit_of((uint32_t)(k >> 32)));
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_token(TokenArgs a) {
  __shared__ float red[kWaves];
  __shared__ TopLds top;
  constexpr int VEC = 16 / (int)sizeof(T);
  const int64_t p = a.row0 + blockIdx.x / a.nseg;
  const int g = (int)(blockIdx.x % a.nseg);
  const Segment<T> seg = segment_of<T>(static_cast<const T*>(a.logits), a.ld, p, g, a.nseg, a.V);
  Stat st{neg_inf(), ref_of(neg_inf(), kL2E, kNear), 0.f, 0.f};
  Best best{neg_inf(), neg_inf(), seg.v0 + (int)threadIdx.x};
  auto add = [&](const float (&v)[VEC]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float x = __builtin_fmaf(v[e], kL2E, -st.m2), y = exp2_(x);
      st.s += y;
      st.t = __builtin_fmaf(y, fmaxf(x, kFloor), st.t);
    }
  };
  auto meet = [&](int i, float m) __attribute__((always_inline)) {
    best.meet(i, m);
    const float m2 = ref_of(best.m, kL2E, kNear);
    if (m2 > st.m2) rebase(st, m2);
  };
  seg.groups(
      [&](int i, float (&v)[kUnroll][VEC]) __attribute__((always_inline)) {
        float m[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) m[u] = max_of(v[u]);
        meet(i, max_of(m));
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) add(v[u]);
      },
      [&](int i, float (&v)[VEC]) __attribute__((always_inline)) {
        meet(i, max_of(v));
        add(v);
      });
  st.m = best.m;
  RowState r;
  r.m = block_max<kWaves>(st.m, red);
  r.m2 = ref_of(r.m, kL2E, kNear);
  if (is_far(r.m, kNear)) {
    st.s = st.t = 0.f;
    seg.each([&](int, float (&v)[VEC], int nv) {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (e < nv) {
          const float x = far_x(v[e], r.m, kL2E), y = exp2_(x);
          st.s += y;
          st.t = __builtin_fmaf(y, fmaxf(x, kFloor), st.t);
        }
    });
  } else {
    rebase(st, r.m2);
  }
  r.s = block_add<kWaves>(st.s, red);
  r.t = block_add<kWaves>(st.t, red);
  if (a.K > 0) top_of_segment<T>(seg, best, a.K, top);
  if (a.nseg == 1) {
    r.close();
    write_row<T>(a, p, r, top.out);
  } else {
    const size_t at = (size_t)p * a.nseg + g;
    if (threadIdx.x == 0) a.part[at] = Stat{r.m, r.m2, r.s, r.t};
    if ((int)threadIdx.x < a.K) a.part_key[at * a.K + threadIdx.x] = top.out[threadIdx.x];
  }
}

// The state of a row from its segments' (at most 64): every lane of every wave gets it.
__device__ __forceinline__ RowState join(const Stat* part, int nseg) {
  const int lane = threadIdx.x & 63;
  Stat st{neg_inf(), 0.f, 0.f, 0.f};
  if (lane < nseg) st = part[lane];
  RowState r;
  r.m = wave_max(st.m);
  r.m2 = ref_of(r.m, kL2E, kNear);
  shift(st, join_shift(st.m, r.m, kL2E, kNear));
  r.s = wave_add(st.s);
  r.t = wave_add(st.t);
  r.close();
  return r;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_token_join(TokenArgs a) {
  __shared__ uint64_t cand[kMaxSegments * kMaxTopTokens], out[kMaxTopTokens];
  __shared__ uint64_t first[kMaxSegments];
  __shared__ int n;
  const int64_t p = a.row0 + blockIdx.x;
  const RowState r = join(a.part + (size_t)p * a.nseg, a.nseg);
  if (a.K > 0) {
    // a threshold: the largest of the segments' last keys, and the K-th largest of their first ones
    const uint64_t* keys = a.part_key + (size_t)p * a.nseg * a.K;
    const int lane = threadIdx.x & 63;
    uint64_t f = 0, l = 0;
    if (lane < a.nseg) {
      f = keys[lane * a.K];
      l = keys[lane * a.K + a.K - 1];
    }
    if (threadIdx.x < 64) first[threadIdx.x] = f;
    if (threadIdx.x == 0) n = 0;
    __syncthreads();
    int rank = 0;
    for (int j = 0; j < a.nseg; ++j) rank += first[j] > f || (first[j] == f && j < lane);
    if (rank == a.K - 1 && lane < a.nseg) l = f > l ? f : l;
    uint64_t tau = l;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint64_t o = __shfl_xor((unsigned long long)tau, d);
      tau = o > tau ? o : tau;
    }
    for (int i = threadIdx.x; i < a.nseg * a.K; i += kThreads) {
      const uint64_t k = keys[i];
      if (k != 0 && k >= tau) cand[atomicAdd(&n, 1)] = k;
    }
    __syncthreads();
    rank_keys(cand, n, a.K, out);
  }
  write_row<T>(a, p, r, out);
}

// ---------------------------------------------------------------- distillation
// The gradient needs the softmax's sums before its first value, so a row is read twice or held.  k_distill_row holds a
// row in its workgroup's registers and so reads and writes memory once (8,192 x 32,000 bf16: 208 us, a copy of the logits
// 200; held in LDS, where two such rows fit a compute unit and every pass reads it, 263); longer rows, and long ones that
// are few, go through k_distill_stats (sums of segments) and k_distill_grad (joins them, reads its segment again, mostly
// from a cache).
// A row has two sums if the loss has both terms and T != 1; otherwise one serves, at T where there are soft targets and at
// 1 where there are none.  Exponentials (16 cycles a wave) would bound the kernel with two a logit in each of two passes,
// so for T = 2 and 4, the usual ones, those at temperature 1 are powers of the others: c, the references and x are then
// exact binary fractions of those at 1 (all references are clamped at the same logit), so 2^(x T) = (2^x)^T up to the
// product's rounding (8,192 x 32,000 bf16, in one run: 232 us with two exponentials, at T = 3, 210 at T = 2, 216 at T = 4,
// 210 with one sum; 8,192 x 10,000: 74, 67.5, 69 and 66; 2,048 x 72,000 fp32: 266, 256, 258 and 250).
// FORM: the sums a row has and how the second comes about.
enum { kOneSum = -1, kTwoSums = 0, kSquare = 1, kFourth = 2 };
// 2^x at temperature 1 from 2^x at T, which is 2 ^ FORM
template <int FORM>
__device__ __forceinline__ float power(float y) {
  return FORM == kSquare ? y * y : (y * y) * (y * y);
}

struct DistillArgs {
  int64_t row0;  // first row of this launch
  const int* order;
  const void* logits;
  size_t ld;
  int V, k, nseg;
  const int* teacher_token;   // [rows][k]
  const float* teacher_logit;
  const int* labels;          // [rows] or NULL
  float T, soft, hard, scale;
  float c;      // log2 e / the temperature of the soft term (of the only one, if there is one)
  float near;   // kScaled over the larger of c and log2 e
  float* row_loss;
  void* grad;   // [rows][ld] or NULL
  Stat* part;   // [rows][nseg]: s the sum at c, t the sum at temperature 1 (two sums)
  float* at;    // [rows][k + 1]: the logits of the teacher's tokens and of the label
};

static_assert(kMaxTeacherTokens == 256, "one entry a thread of the smallest workgroup");

// a row's targets: this thread's teacher entry, the label
struct Target {
  bool have;       // the entry counts
  int tok;         // its token
  float t;         // the teacher's logit
  int y;           // the label, or -1
  bool soft, any;  // the row has a teacher's entry; a target at all
};
__device__ __forceinline__ Target target_of(const DistillArgs& a, size_t q) {
  Target g{false, -1, neg_inf(), -1, false, false};
  if ((int)threadIdx.x < a.k) {
    g.tok = a.teacher_token[q * a.k + threadIdx.x];
    g.t = a.teacher_logit[q * a.k + threadIdx.x];
    g.have = g.tok >= 0 && g.tok < a.V && !(g.t == neg_inf());
  }
  if (a.labels) {
    const int y = a.labels[q];
    g.y = y >= 0 && y < a.V ? y : -1;
  }
  g.soft = __syncthreads_or(g.have) != 0;
  g.any = g.soft || g.y >= 0;
  return g;
}

// What a row's gradient and loss are made of, from its maximum and sums.
template <int FORM>
struct RowGrad {
  static constexpr bool TWO = FORM != kOneSum;
  float m, mc, m1, s, s1;  // the maximum; the references and sums at c and (two sums) at temperature 1
  float c, invT;
  float wa, wb, ga, gb;    // weights of the soft and hard term, and of 2^x in the gradient
  bool far, bad, empty;
  __device__ __forceinline__ void close(const DistillArgs& a, const Target& t) {
    c = a.c;
    invT = 1.f / a.T;
    far = is_far(m, a.near);
    bad = !(s == s) || m == __builtin_inff();
    empty = !bad && m == neg_inf();
    if (!TWO) s1 = s;
    wa = t.soft ? a.scale * a.soft * a.T : 0.f;
    wb = t.y >= 0 ? a.scale * a.hard : 0.f;
    const float nan = __builtin_nanf("");
    ga = bad ? nan : empty ? 0.f : TWO ? wa / s : (wa + wb) / s;
    gb = TWO ? (bad ? nan : empty ? 0.f : wb / s1) : 0.f;
  }
  // the gradient of a logit that is no target: 0 for -inf, in rows that are not bad
  __device__ __forceinline__ float dense(float z) const {
    const float y = exp2_(__builtin_fmaf(z, c, -mc));
    if constexpr (FORM == kOneSum) return ga * y;
    if constexpr (FORM == kTwoSums) return __builtin_fmaf(gb, exp2_(__builtin_fmaf(z, kL2E, -m1)), ga * y);
    if constexpr (FORM == kSquare) return y * __builtin_fmaf(gb, y, ga);
    return __builtin_fmaf(gb, power<FORM>(y), ga * y);
  }
  // the same in a row that is far or bad
  __device__ __forceinline__ float odd(float z) const {
    if (bad) return ga;
    const float y = ga * exp2_(far_x(z, m, c));
    return TWO ? __builtin_fmaf(gb, exp2_(far_x(z, m, kL2E)), y) : y;
  }
  __device__ __forceinline__ bool is_odd() const { return bad || far; }
  // the gradient of a target: soft and hard mass on it
  __device__ __forceinline__ float target(float z, float soft_mass, float hard_mass) const {
    if (empty) return 0.f;
    if (bad) return ga;
    const float pc = exp2_(far ? far_x(z, m, c) : __builtin_fmaf(z, c, -mc));
    const float p1 = !TWO ? pc : exp2_(far ? far_x(z, m, kL2E) : __builtin_fmaf(z, kL2E, -m1));
    return wa * (pc / s - soft_mass) + wb * (p1 / s1 - hard_mass);
  }
  // log p at a temperature (its factor, reference and sum)
  __device__ __forceinline__ float logp(float z, float f, float ref, float sum, float inv) const {
    if (bad) return __builtin_nanf("");
    if (empty) return neg_inf();
    if (far || z < -1e30f) return (z - m) * inv - kLn2 * log2_(sum);
    return kLn2 * (__builtin_fmaf(z, f, -ref) - log2_(sum));
  }
  __device__ __forceinline__ float logp_soft(float z) const { return logp(z, c, mc, s, invT); }
  __device__ __forceinline__ float logp_hard(float z) const {
    return TWO ? logp(z, kL2E, m1, s1, 1.f) : logp(z, c, mc, s, 1.f);
  }
};

// this thread's share of the soft term: q (log q - log p), q = e / es with e = exp(dt)
template <int FORM>
__device__ __forceinline__ float soft_loss(const DistillArgs& a, const RowGrad<FORM>& r, const Target& t, float q,
                                           float dt, float es, float z) {
  return t.have && q != 0.f && a.soft != 0.f ? q * (dt - logf(es) - r.logp_soft(z)) : 0.f;
}
// the loss of a row with a target from the sum of the shares
template <int FORM>
__device__ __forceinline__ float row_loss(const DistillArgs& a, const RowGrad<FORM>& r, const Target& t, float soft,
                                          float zy) {
  if (r.bad) return __builtin_nanf("");
  if (r.empty) return __builtin_inff();
  float loss = t.soft && a.soft != 0.f ? a.soft * a.T * a.T * soft : 0.f;
  if (t.y >= 0 && a.hard != 0.f) loss -= a.hard * r.logp_hard(zy);
  return loss;
}

// The targets' columns inside [lo, hi), written whole after everything else: the first entry of a token takes the mass of
// all its entries.  tok, mass: every entry's token (-1: does not count) and q.
template <typename G, int FORM>
__device__ __forceinline__ void write_targets(const DistillArgs& a, const RowGrad<FORM>& r, const Target& t,
                                              const int* tok, const float* mass, float zj, float zy, G* out, int lo,
                                              int hi) {
  if (t.have && t.tok >= lo && t.tok < hi) {
    float sum = 0.f;
    bool lead = true;
    for (int j = 0; j < a.k; ++j) {
      const bool same = tok[j] == t.tok;
      sum += same ? mass[j] : 0.f;
      lead = lead && !(same && j < (int)threadIdx.x);
    }
    if (lead) out[t.tok] = from_f32<G>(r.target(zj, sum, t.tok == t.y ? 1.f : 0.f));
  }
  if (threadIdx.x == 0 && t.y >= lo && t.y < hi) {
    bool seen = false;
    for (int j = 0; j < a.k; ++j) seen = seen || tok[j] == t.y;
    if (!seen) out[t.y] = from_f32<G>(r.target(zy, 0.f, 1.f));
  }
}

template <typename G>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{a, b}), b2));  // to nearest even
}
// N neighbouring gradients
template <typename G, int N>
__device__ __forceinline__ void store_grad(G* p, const float (&v)[N]) {
  if constexpr (sizeof(G) == 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
  } else if constexpr (N == 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2<G>(v[0], v[1]), pack2<G>(v[2], v[3]), pack2<G>(v[4], v[5]),
                                              pack2<G>(v[6], v[7]));
  } else {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack2<G>(v[0], v[1]), pack2<G>(v[2], v[3]));
  }
}

// a word of logits with those after its first `have` set to -inf
template <typename T>
__device__ __forceinline__ uint32_t first_of(uint32_t w, int have) {
  if constexpr (sizeof(T) == 4) return have > 0 ? w : 0xff800000u;
  return have > 1 ? w : have > 0 ? (w & 0xffffu) | 0xff800000u : 0xff80ff80u;
}

// A whole row by one workgroup, in its registers: NV vectors a thread, loaded once, the columns that are not there set to
// -inf (probability 0, gradient 0), then gone through three times (maximum, sums, gradient).
template <typename T, typename G, int FORM, int TH, int NV>
__global__ __launch_bounds__(TH, NV <= 9 ? 6 : 4) void k_distill_row(DistillArgs a) {
  constexpr int VEC = 16 / (int)sizeof(T), NW = TH / 64;
  constexpr bool TWO = FORM != kOneSum;
  __shared__ float red[6][NW];
  __shared__ int tok[kMaxTeacherTokens];
  __shared__ float mass[kMaxTeacherTokens];
  const int tid = threadIdx.x;
  const int64_t p = a.row0 + blockIdx.x;
  const size_t q = a.order ? (size_t)a.order[p] : (size_t)p;
  const T* row = static_cast<const T*>(a.logits) + (size_t)p * a.ld;
  G* out = a.grad ? static_cast<G*>(a.grad) + (size_t)p * a.ld : nullptr;
  const int nv = (int)(a.ld / VEC);
  uint4 raw[NV];
#pragma unroll
  for (int u = 0; u < NV; ++u)
    if (u * TH < nv) raw[u] = reinterpret_cast<const uint4*>(row)[min(u * TH + tid, nv - 1)];
  const Target t = target_of(a, q);
  if (!t.any) {
    if (tid == 0) a.row_loss[q] = 0.f;
    if (out) {
      const float z[VEC] = {};
      for (int i = tid; i < nv; i += TH) store_grad<G>(out + (size_t)i * VEC, z);
    }
    return;
  }
  const float zj = t.have ? to_f32<T>(row[t.tok]) : 0.f, zy = t.y >= 0 ? to_f32<T>(row[t.y]) : 0.f;
#pragma unroll
  for (int u = 0; u < NV; ++u)
    if (u * TH < nv && (u + 1) * TH * VEC > a.V) {  // the row ends here
      const int have = a.V - (u * TH + tid) * VEC;
      raw[u] = make_uint4(first_of<T>(raw[u].x, have), first_of<T>(raw[u].y, have - VEC / 4),
                          first_of<T>(raw[u].z, have - VEC / 2), first_of<T>(raw[u].w, have - 3 * VEC / 4));
    }
  auto all = [&](const float* x, bool max) {
    float r = x[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) r = max ? fmaxf(r, x[w]) : r + x[w];
    return r;
  };
  auto put = [&](float* x, float v) {
    if ((tid & 63) == 0) x[tid >> 6] = v;
  };
  // f(vector of the row, its values)
  auto pass = [&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < NV; ++u)
      if (u * TH < nv) {
        float v[VEC];
        unpack<T>(raw[u], v);
        f(u * TH + tid, v);
      }
  };
  float m = neg_inf();
  pass([&](int, float (&v)[VEC]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) m = fmaxf(m, v[e]);
  });
  put(red[0], wave_max(m));
  put(red[1], wave_max(t.have ? t.t : neg_inf()));
  __syncthreads();
  RowGrad<FORM> r;
  r.m = all(red[0], true);
  r.mc = ref_of(r.m, a.c, a.near);
  r.m1 = ref_of(r.m, kL2E, a.near);
  float s = 0.f, s1 = 0.f;
  if (is_far(r.m, a.near)) {
    pass([&](int, float (&v)[VEC]) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        s += exp2_(far_x(v[e], r.m, a.c));
        if constexpr (TWO) s1 += exp2_(far_x(v[e], r.m, kL2E));
      }
    });
  } else {
    pass([&](int, float (&v)[VEC]) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float y = exp2_(__builtin_fmaf(v[e], a.c, -r.mc));
        s += y;
        if constexpr (FORM == kTwoSums) s1 += exp2_(__builtin_fmaf(v[e], kL2E, -r.m1));
        else if constexpr (TWO) s1 += power<FORM>(y);
      }
    });
  }
  // teacher: q_j = softmax(t / T) over the entries that count
  const float dt = (t.t - all(red[1], true)) / a.T;
  const float ej = t.have ? expf(dt) : 0.f;
  put(red[2], wave_add(s));
  if constexpr (TWO) put(red[3], wave_add(s1));
  put(red[4], wave_add(ej));
  __syncthreads();
  r.s = all(red[2], false);
  r.s1 = TWO ? all(red[3], false) : r.s;
  r.close(a, t);
  const float es = all(red[4], false), qj = t.have ? ej / es : 0.f;
  if (tid < a.k) {
    tok[tid] = t.have ? t.tok : -1;
    mass[tid] = qj;
  }
  put(red[5], wave_add(soft_loss(a, r, t, qj, dt, es, zj)));
  if (out) {
    if (r.is_odd()) {
      pass([&](int i, float (&v)[VEC]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = i * VEC + e < a.V ? r.odd(v[e]) : 0.f;
        if (i < nv) store_grad<G>(out + (uint32_t)(i * VEC), v);
      });
    } else {
      pass([&](int i, float (&v)[VEC]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = r.dense(v[e]);
        if (i < nv) store_grad<G>(out + (uint32_t)(i * VEC), v);
      });
    }
  }
  __syncthreads();
  if (tid == 0) a.row_loss[q] = row_loss(a, r, t, all(red[5], false), zy);
  if (out) write_targets(a, r, t, tok, mass, zj, zy, out, 0, a.V);
}

// One segment's maximum and its sums
template <typename T, int FORM>
__global__ __launch_bounds__(kThreads) void k_distill_stats(DistillArgs a) {
  __shared__ float red[kWaves];
  constexpr int VEC = 16 / (int)sizeof(T);
  constexpr bool TWO = FORM != kOneSum;
  const int64_t p = a.row0 + blockIdx.x / a.nseg;
  const int g = (int)(blockIdx.x % a.nseg);
  const size_t q = a.order ? (size_t)a.order[p] : (size_t)p;
  const Target tg = target_of(a, q);
  if (!tg.any) return;
  const Segment<T> seg = segment_of<T>(static_cast<const T*>(a.logits), a.ld, p, g, a.nseg, a.V);
  if (g == 0) {
    const T* row = static_cast<const T*>(a.logits) + (size_t)p * a.ld;
    float* at = a.at + (size_t)p * (a.k + 1);
    if (tg.have) at[threadIdx.x] = to_f32<T>(row[tg.tok]);
    if (threadIdx.x == 0) at[a.k] = tg.y >= 0 ? to_f32<T>(row[tg.y]) : 0.f;
  }
  float m = neg_inf(), s = 0.f, s1 = 0.f, rc = ref_of(m, a.c, a.near), r1 = ref_of(m, kL2E, a.near);
  auto meet = [&](float vm) __attribute__((always_inline)) {
    if (vm > m) {
      m = vm;
      const float nc = ref_of(m, a.c, a.near), n1 = ref_of(m, kL2E, a.near);
      s *= exp2_(rc - nc);
      rc = nc;
      if constexpr (TWO) {
        s1 *= exp2_(r1 - n1);
        r1 = n1;
      }
    }
  };
  auto add = [&](const float (&v)[VEC]) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float y = exp2_(__builtin_fmaf(v[e], a.c, -rc));
      s += y;
      if constexpr (FORM == kTwoSums) s1 += exp2_(__builtin_fmaf(v[e], kL2E, -r1));
      else if constexpr (TWO) s1 += power<FORM>(y);
    }
  };
  seg.groups(
      [&](int, float (&v)[kUnroll][VEC]) __attribute__((always_inline)) {
        float vm[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) vm[u] = max_of(v[u]);
        meet(max_of(vm));
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) add(v[u]);
      },
      [&](int, float (&v)[VEC]) __attribute__((always_inline)) {
        meet(max_of(v));
        add(v);
      });
  const float M = block_max<kWaves>(m, red);
  if (is_far(M, a.near)) {
    s = s1 = 0.f;
    seg.each([&](int, float (&v)[VEC], int nv) {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (e < nv) {
          s += exp2_(far_x(v[e], M, a.c));
          if constexpr (TWO) s1 += exp2_(far_x(v[e], M, kL2E));
        }
    });
  } else {
    s *= exp2_(rc - ref_of(M, a.c, a.near));
    if constexpr (TWO) s1 *= exp2_(r1 - ref_of(M, kL2E, a.near));
  }
  const float S = block_add<kWaves>(s, red), S1 = TWO ? block_add<kWaves>(s1, red) : 0.f;
  if (threadIdx.x == 0) a.part[(size_t)p * a.nseg + g] = Stat{M, 0.f, S, S1};
}

// The loss of a row and one segment of its gradient
template <typename T, typename G, int FORM>
__global__ __launch_bounds__(kThreads) void k_distill_grad(DistillArgs a) {
  __shared__ float red[kWaves];
  __shared__ int tok[kMaxTeacherTokens];
  __shared__ float mass[kMaxTeacherTokens];
  constexpr int VEC = 16 / (int)sizeof(T);
  const int64_t p = a.row0 + blockIdx.x / a.nseg;
  const int g = (int)(blockIdx.x % a.nseg);
  const size_t q = a.order ? (size_t)a.order[p] : (size_t)p;
  const Target tg = target_of(a, q);
  const Segment<T> seg = segment_of<T>(static_cast<const T*>(a.logits), a.ld, p, g, a.nseg, a.V);
  G* out = a.grad ? static_cast<G*>(a.grad) + (size_t)p * a.ld : nullptr;
  // the segment that holds column V - 1 writes the pad columns too; the empty ones behind it write nothing
  const int first = seg.v0 * VEC, last = seg.v0 == seg.v1 ? 0 : seg.v1 * VEC >= a.V ? (int)a.ld : seg.v1 * VEC;
  if (!tg.any) {
    if (g == 0 && threadIdx.x == 0) a.row_loss[q] = 0.f;
    if (out) {
      const float z[8] = {};
      for (int col = first + (int)threadIdx.x * 8; col < last; col += kThreads * 8) store_grad<G>(out + col, z);
    }
    return;
  }
  const int lane = threadIdx.x & 63;
  Stat st{neg_inf(), 0.f, 0.f, 0.f};
  if (lane < a.nseg) st = a.part[(size_t)p * a.nseg + lane];
  RowGrad<FORM> r;
  r.m = wave_max(st.m);
  r.mc = ref_of(r.m, a.c, a.near);
  r.m1 = ref_of(r.m, kL2E, a.near);
  r.s = wave_add(st.s * exp2_(join_shift(st.m, r.m, a.c, a.near)));
  r.s1 = wave_add(st.t * exp2_(join_shift(st.m, r.m, kL2E, a.near)));
  r.close(a, tg);
  const float tm = block_max<kWaves>(tg.have ? tg.t : neg_inf(), red);
  const float dt = (tg.t - tm) / a.T, ej = tg.have ? expf(dt) : 0.f, es = block_add<kWaves>(ej, red);
  const float qj = tg.have ? ej / es : 0.f;
  const float* at = a.at + (size_t)p * (a.k + 1);
  const float zj = tg.have ? at[threadIdx.x] : 0.f, zy = at[a.k];
  if ((int)threadIdx.x < a.k) {
    tok[threadIdx.x] = tg.have ? tg.tok : -1;
    mass[threadIdx.x] = qj;
  }
  if (g == 0) {
    const float soft = block_add<kWaves>(soft_loss(a, r, tg, qj, dt, es, zj), red);
    if (threadIdx.x == 0) a.row_loss[q] = row_loss(a, r, tg, soft, zy);
  }
  if (!out) return;
  const T* row = static_cast<const T*>(a.logits) + (size_t)p * a.ld;
  auto write = [&](auto&& value) __attribute__((always_inline)) {
    constexpr int U = 4;  // groups of 8 columns in flight
    for (int b = first + (int)threadIdx.x * 8; b < last; b += kThreads * 8 * U) {
      uint4 raw[U][8 / VEC];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int h = 0; h < 8 / VEC; ++h)
          raw[u][h] = *reinterpret_cast<const uint4*>(row + min(b + u * kThreads * 8, last - 8) + h * VEC);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int col = b + u * kThreads * 8;
        if (col >= last) continue;
        float v[8];
#pragma unroll
        for (int h = 0; h < 8 / VEC; ++h) {
          float w[VEC];
          unpack<T>(raw[u][h], w);
#pragma unroll
          for (int e = 0; e < VEC; ++e) v[h * VEC + e] = col + h * VEC + e < a.V ? value(w[e]) : 0.f;
        }
        store_grad<G>(out + col, v);
      }
    }
  };
  if (r.is_odd()) write([&](float z) __attribute__((always_inline)) { return r.odd(z); });
  else write([&](float z) __attribute__((always_inline)) { return r.dense(z); });
  __syncthreads();
  write_targets(a, r, tg, tok, mass, zj, zy, out, first, last);
}

// Segments of a row.  A workgroup takes about 11 us for a row of 200 KB, which is what a row in segments and their join
// take together, so shorter rows stay whole; longer ones are cut into pieces of 32 KB, unless there are rows enough to
// fill the chip several times (one row of 131,072 fp32: 32 us whole, 12 us in 16; 64 rows: 34 and 16 us; 1,500 rows: 162
// and 154 us; at 16,384 rows of 50,000 two segments cost more than they save).
constexpr int kSegmentBytes = 32 * 1024, kWholeBytes = 224 * 1024, kRowsFull = 2048;
int segments(int64_t rows, int V, int esize) {
  const int64_t bytes = (int64_t)V * esize;
  if (bytes < kWholeBytes || rows >= kRowsFull) return 1;
  return (int)std::min<int64_t>((bytes + kSegmentBytes - 1) / kSegmentBytes, kMaxSegments);
}
// rows of one launch of `threads` a row: all its threads are counted in 32 bits
constexpr int kHeldThreads = 1024;  // the most that hold a row
constexpr int64_t rows_of_launch(int threads) { return ((int64_t)1 << 31) / threads; }
static_assert(rows_of_launch(kHeldThreads) * kHeldThreads <= (int64_t)UINT32_MAX &&
                  rows_of_launch(kMaxSegments * kThreads) >= 1, "a launch's threads");
// Two passes over a row that is not held; a workgroup per 32 KB (2,048 rows of 130,001 fp32: 600 us whole, 495 in 16).
int distill_segments(int64_t rows, int V, int esize) {
  const int64_t bytes = (int64_t)V * esize;
  return (int)std::min<int64_t>((bytes + kSegmentBytes - 1) / kSegmentBytes, kMaxSegments);
}

// Rows that a workgroup holds in its registers.  512 threads hold up to 144 KB, always; 1,024 hold up to 288 KB, one row to
// a compute unit, where rows fill the chip twice (2,048 x 72,000 fp32: 255 us held, 335 in segments; 2,048 x 131,072 bf16:
// 298 and 316; 300 rows: 60 and 49; 8 rows: 25 and 16).
constexpr int kHeldBytes = 144 * 1024, kRowsHeld = 512;
bool held(int64_t rows, int V, int esize) {
  return (size_t)row_ld(V) * esize <= (size_t)kHeldBytes * (rows >= kRowsHeld ? 2 : 1);
}

template <typename T>
void launch_token_rows(const TokenArgs& a, unsigned rows, hipStream_t st) {
  hipLaunchKernelGGL(k_token<T>, dim3(rows * a.nseg), dim3(kThreads), 0, st, a);
  if (a.nseg > 1) hipLaunchKernelGGL(k_token_join<T>, dim3(rows), dim3(kThreads), 0, st, a);
}

template <typename T, typename G, int FORM>
void launch_distill_form(const DistillArgs& a, unsigned rows, hipStream_t st) {
  if (a.nseg == 0) {
    // the smallest size that holds the row: registers decide how many rows a compute unit has at once
    const size_t bytes = a.ld * sizeof(T);
    const dim3 grid(rows);
    if (bytes <= 8 * 1024)
      hipLaunchKernelGGL((k_distill_row<T, G, FORM, 256, 2>), grid, dim3(256), 0, st, a);
    else if (bytes <= 16 * 1024)
      hipLaunchKernelGGL((k_distill_row<T, G, FORM, 256, 4>), grid, dim3(256), 0, st, a);
    else if (bytes <= 24 * 1024)
      hipLaunchKernelGGL((k_distill_row<T, G, FORM, 256, 6>), grid, dim3(256), 0, st, a);
    else if (bytes <= 36 * 1024)
      hipLaunchKernelGGL((k_distill_row<T, G, FORM, 256, 9>), grid, dim3(256), 0, st, a);
    else if (bytes <= 48 * 1024)
      hipLaunchKernelGGL((k_distill_row<T, G, FORM, 512, 6>), grid, dim3(512), 0, st, a);
    else if (bytes <= 72 * 1024)
      hipLaunchKernelGGL((k_distill_row<T, G, FORM, 512, 9>), grid, dim3(512), 0, st, a);
    else if (bytes <= 96 * 1024)
      hipLaunchKernelGGL((k_distill_row<T, G, FORM, 512, 12>), grid, dim3(512), 0, st, a);
    else if (bytes <= 144 * 1024)
      hipLaunchKernelGGL((k_distill_row<T, G, FORM, 512, 18>), grid, dim3(512), 0, st, a);
    else
      hipLaunchKernelGGL((k_distill_row<T, G, FORM, kHeldThreads, 18>), grid, dim3(kHeldThreads), 0, st, a);
    return;
  }
  hipLaunchKernelGGL((k_distill_stats<T, FORM>), dim3(rows * a.nseg), dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL((k_distill_grad<T, G, FORM>), dim3(rows * a.nseg), dim3(kThreads), 0, st, a);
}
template <typename T, typename G>
void launch_distill_rows(const DistillArgs& a, bool two, unsigned rows, hipStream_t st) {
  if (!two) launch_distill_form<T, G, kOneSum>(a, rows, st);
  else if (a.T == 2.f) launch_distill_form<T, G, kSquare>(a, rows, st);
  else if (a.T == 4.f) launch_distill_form<T, G, kFourth>(a, rows, st);
  else launch_distill_form<T, G, kTwoSums>(a, rows, st);
}

}  // namespace

size_t token_workspace_bytes(int dtype, int64_t rows, int V, int K) {
  const int n = segments(rows, V, dtype == FOLD_BF16 ? 2 : 4);
  return n == 1 ? 0 : (size_t)rows * n * (sizeof(Stat) + (size_t)K * sizeof(uint64_t));
}

size_t distill_workspace_bytes(int dtype, int64_t rows, int V, int k) {
  const int es = dtype == FOLD_BF16 ? 2 : 4;
  if (held(rows, V, es)) return 0;
  return (size_t)rows * (distill_segments(rows, V, es) * sizeof(Stat) + (size_t)(k + 1) * sizeof(float));
}

void launch_token(int dtype, const int* order, int64_t rows, int V, const void* logits, int J, const int* tokens,
                  float* logp, float* entropy, int K, int* top_token, float* top_logp, void* ws, hipStream_t st) {
  if (rows <= 0) return;
  ProfScope prof("token_logprobs", st);
  const int n = segments(rows, V, dtype == FOLD_BF16 ? 2 : 4);
  TokenArgs a{0, order, logits, (size_t)row_ld(V), V, J, K, n, tokens, logp, entropy, top_token, top_logp,
              static_cast<Stat*>(ws), reinterpret_cast<uint64_t*>(static_cast<Stat*>(ws) + (size_t)rows * n)};
  for (const int64_t most = rows_of_launch(n * kThreads); a.row0 < rows; a.row0 += most) {
    const unsigned r = (unsigned)std::min<int64_t>(rows - a.row0, most);
    if (dtype == FOLD_BF16) launch_token_rows<uint16_t>(a, r, st);
    else launch_token_rows<float>(a, r, st);
  }
}

void launch_distill(int dtype, const int* order, int64_t rows, int V, const void* logits, int k,
                    const int* teacher_token, const float* teacher_logit, const int* labels, float T, float soft,
                    float hard, float scale, float* row_loss, int grad_dtype, void* grad, void* ws, hipStream_t st) {
  if (rows <= 0) return;
  ProfScope prof("loss_distill", st);
  const int es = dtype == FOLD_BF16 ? 2 : 4;
  const int n = held(rows, V, es) ? 0 : distill_segments(rows, V, es);
  // one temperature serves unless both terms are there and differ
  const bool uses_soft = soft != 0.f && k > 0, uses_hard = hard != 0.f && labels;
  const bool two = uses_soft && uses_hard && T != 1.f;
  const float c = kL2E / (uses_soft ? T : 1.f);
  DistillArgs a{0, order, logits, (size_t)row_ld(V), V, k, n, teacher_token, teacher_logit, labels, T, soft, hard,
                scale, c, kScaled / std::max(c, kL2E), row_loss, grad, static_cast<Stat*>(ws),
                reinterpret_cast<float*>(static_cast<Stat*>(ws) + (size_t)rows * n)};
  for (const int64_t most = rows_of_launch(n == 0 ? kHeldThreads : n * kThreads); a.row0 < rows; a.row0 += most) {
    const unsigned r = (unsigned)std::min<int64_t>(rows - a.row0, most);
    if (dtype == FOLD_BF16) launch_distill_rows<uint16_t, uint16_t>(a, two, r, st);
    else if (grad_dtype == FOLD_BF16) launch_distill_rows<float, uint16_t>(a, two, r, st);
    else launch_distill_rows<float, float>(a, two, r, st);
  }
}

}  // namespace fold
