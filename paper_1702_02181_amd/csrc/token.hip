// Row operators over the logits of a vocabulary head (gfx950): log probabilities of given tokens with the entropy and
// the top alternatives of every row, and the distillation loss with its gradient.
//
// A row of V logits is read in 16-byte vectors.  Its softmax is kept in base 2: with L = log2 e and a reference m2,
// x = z L - m2 (one fma: every term of a row sees the same rounded m2, which cancels in p and in log p),
// s = sum 2^x, and for the entropy t = sum 2^x x.  Then log p = ln 2 (x - log2 s) and H = ln 2 (log2 s - t / s).
// Partial (m2, s, t) of threads, waves and segments of a row meet by the usual rescaling; all of it is fp32.
//
// Values that leave the range where z L is finite: a segment whose largest logit has |m| >= kFar (logits masked by the
// type's lowest value and nothing else there, for instance) is read once more and its s is the count of logits equal
// to m: every other one is at least an ulp of m (more than 1e28) below, so its probability is an exact 0.
// NaN reaches s by itself (the maximum ignores NaN); +inf and NaN make the row's results NaN; a row of -inf alone is
// empty.

#include <hip/hip_runtime.h>

#include <algorithm>

#include "common.h"
#include "internal.h"
#include "mfma.h"

namespace fold {

namespace {

constexpr float kL2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFar = 1e35f;      // |m| from here on: see above (z / T stays finite for T >= 1e-3)
constexpr float kFloor = -200.f;   // 2^-200 is 0 in fp32: bounds x where it is multiplied by 2^x
constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kUnroll = 4;         // vectors a thread has in flight
constexpr int kCap = 1024;         // candidates of a segment's top list held in LDS

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
// over the workgroup; red holds kWaves floats and is free again after the next barrier
__device__ __forceinline__ float block_max(float v, float* red) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float r = red[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) r = fmaxf(r, red[w]);
  return r;
}
__device__ __forceinline__ float block_add(float v, float* red) {
  v = wave_add(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  float r = red[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) r += red[w];
  return r;
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

  // f(vector index, its values, the number of them that are real): kUnroll loads in flight, from clamped addresses
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
};

__host__ __device__ inline int vectors_of(int V, int vec) { return (V + vec - 1) / vec; }

template <typename T>
__device__ __forceinline__ Segment<T> segment_of(const T* z, size_t ld, int64_t p, int seg, int nseg, int V) {
  // pieces of whole 64-column blocks, so that a gradient of another type splits at the same columns; the last ones may
  // be empty
  const int nv = vectors_of(V, Segment<T>::VEC), block = 64 / Segment<T>::VEC;
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

__device__ __forceinline__ float ref_of(float m, float c) { return fminf(fmaxf(m, -kFar), kFar) * c; }
__device__ __forceinline__ bool is_far(float m) { return fabsf(m) >= kFar && m != neg_inf(); }

// s and t seen from the reference m2
__device__ __forceinline__ void rebase(Stat& a, float m2) {
  const float d = fmaxf(a.m2 - m2, kFloor), f = exp2_(a.m2 - m2);
  a.t = f * (a.t + d * a.s);
  a.s = f * a.s;
  a.m2 = m2;
}

// The state of a whole row from that of its segments: `bad` for NaN or +inf, `empty` for -inf alone.
struct RowState {
  float m, m2, s, t;
  bool bad, empty, far;
  __device__ __forceinline__ void close() {
    far = is_far(m);
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
    return fmaxf(kLn2 * (far ? log2_(s) : log2_(s) - t / s), 0.f);
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

struct TopLds {
  uint64_t cand[kCap];
  uint64_t out[kMaxTopTokens];
  uint32_t key[kThreads];
  unsigned hist[256];
  int n, bin, left;
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

// The K largest keys of a segment, in order, in s.out.  m: the thread's own largest logit.  A threshold first: the K-th
// largest of the 256 threads' maxima cannot exceed the K-th largest logit, and few logits reach it (about K where the
// large ones are spread over the threads); they are found again in the segment, now in a cache, by the threads whose
// maximum reaches it.  Where more than kCap do (many equal logits, or all the large ones in few threads' columns), the
// K-th largest key is found digit by digit instead, with one read of the segment a digit.
template <typename T>
__device__ void top_of_segment(const Segment<T>& seg, float m, int K, TopLds& s) {
  const int tid = threadIdx.x, lane = tid & 63;
  s.key[tid] = m > neg_inf() ? order_of(m) : 0u;
  if (tid == 0) s.n = 0;
  __syncthreads();
  uint32_t k[kWaves], tau = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) k[w] = s.key[w * 64 + lane];
  for (int b = 31; b >= 0; --b) {
    const uint32_t c = tau | (1u << b);
    int n = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) n += __popcll(__ballot(k[w] >= c));
    if (n >= K) {
      tau = c;
      if (n == K) break;
    }
  }
  if (s.key[tid] >= tau && s.key[tid] != 0) {
    for (int i = seg.v0 + tid; i < seg.v1; i += kThreads) {
      float v[Segment<T>::VEC];
      unpack<T>(seg.row[i], v);
#pragma unroll
      for (int e = 0; e < Segment<T>::VEC; ++e) {
        const int col = i * Segment<T>::VEC + e;
        if (col < seg.V && v[e] > neg_inf() && order_of(v[e]) >= tau) {
          const int at = atomicAdd(&s.n, 1);
          if (at < kCap) s.cand[at] = key_of(v[e], col);
        }
      }
    }
  }
  __syncthreads();
  if (s.n > kCap) {  // the same for every thread
    uint64_t prefix = 0;
    int left = K;
    for (int byte = 7; byte >= 0; --byte) {
      s.hist[tid] = 0;
      __syncthreads();
      seg.each([&](int i, float (&v)[Segment<T>::VEC], int nv) {
#pragma unroll
        for (int e = 0; e < Segment<T>::VEC; ++e) {
          const uint64_t q = key_of(v[e], i * Segment<T>::VEC + e);
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
    seg.each([&](int i, float (&v)[Segment<T>::VEC], int nv) {
#pragma unroll
      for (int e = 0; e < Segment<T>::VEC; ++e) {
        const uint64_t q = key_of(v[e], i * Segment<T>::VEC + e);
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
  constexpr int VEC = Segment<T>::VEC;
  const int64_t p = a.row0 + blockIdx.x / a.nseg;
  const int g = (int)(blockIdx.x % a.nseg);
  const Segment<T> seg = segment_of<T>(static_cast<const T*>(a.logits), a.ld, p, g, a.nseg, a.V);
  Stat st{neg_inf(), -kFar * kL2E, 0.f, 0.f};
  seg.each([&](int, float (&v)[VEC], int nv) {
    if (nv < VEC)
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = e < nv ? v[e] : neg_inf();
    float vm = v[0];
#pragma unroll
    for (int e = 1; e < VEC; ++e) vm = fmaxf(vm, v[e]);
    st.m = fmaxf(st.m, vm);
    const float m2 = ref_of(st.m, kL2E);
    if (m2 > st.m2) rebase(st, m2);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float x = __builtin_fmaf(v[e], kL2E, -st.m2), y = exp2_(x);
      st.s += y;
      st.t = __builtin_fmaf(y, fmaxf(x, kFloor), st.t);
    }
  });
  const float mine = st.m;
  RowState r;
  r.m = block_max(st.m, red);
  r.m2 = ref_of(r.m, kL2E);
  rebase(st, r.m2);
  r.s = block_add(st.s, red);
  r.t = block_add(st.t, red);
  if (is_far(r.m)) {
    float n = 0.f;
    seg.each([&](int, float (&v)[VEC], int nv) {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (e < nv) n += v[e] == r.m ? 1.f : v[e] == v[e] ? 0.f : v[e];
    });
    r.s = block_add(n, red);
    r.t = 0.f;
  }
  if (a.K > 0) top_of_segment<T>(seg, mine, a.K, top);
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
  Stat st{neg_inf(), -kFar * kL2E, 0.f, 0.f};
  if (lane < nseg) st = part[lane];
  RowState r;
  r.m = wave_max(st.m);
  r.m2 = ref_of(r.m, kL2E);
  const bool nan = st.s != st.s;
  if (is_far(r.m) && st.m != r.m) st.s = nan ? st.s : 0.f;  // a segment below a far maximum has probability 0
  else rebase(st, r.m2);
  r.s = wave_add(st.s);
  r.t = wave_add(st.t);
  r.close();
  return r;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_token_join(TokenArgs a) {
  __shared__ uint64_t cand[64 * kMaxTopTokens], out[kMaxTopTokens];
  __shared__ uint64_t first[64];
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
  float* row_loss;
  void* grad;   // [rows][ld] or NULL
  Stat* part;   // [rows][nseg]: t holds the sum at temperature T
  float* at;    // [rows][k + 1]: the logits of the teacher's tokens and of the label
};

static_assert(kMaxTeacherTokens == kThreads, "one entry a thread");

// a row's targets: which entries count
struct Target {
  bool have;      // this thread's teacher entry counts
  int tok;        // its token
  float t;        // the teacher's logit
  int y;          // the label, or -1
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

// One segment's maximum and its sums at temperature 1 and T
template <typename T>
__global__ __launch_bounds__(kThreads) void k_distill_stats(DistillArgs a) {
  __shared__ float red[kWaves];
  constexpr int VEC = Segment<T>::VEC;
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
  const float c = kL2E / a.T;
  float m = neg_inf(), s1 = 0.f, sT = 0.f;
  float r1 = -kFar * kL2E, rT = -kFar * c;
  seg.each([&](int, float (&v)[VEC], int nv) {
    if (nv < VEC)
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = e < nv ? v[e] : neg_inf();
    float vm = v[0];
#pragma unroll
    for (int e = 1; e < VEC; ++e) vm = fmaxf(vm, v[e]);
    if (vm > m) {
      m = vm;
      const float n1 = ref_of(m, kL2E), nT = ref_of(m, c);
      s1 *= exp2_(r1 - n1);
      sT *= exp2_(rT - nT);
      r1 = n1;
      rT = nT;
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      s1 += exp2_(__builtin_fmaf(v[e], kL2E, -r1));
      sT += exp2_(__builtin_fmaf(v[e], c, -rT));
    }
  });
  const float M = block_max(m, red), M1 = ref_of(M, kL2E), MT = ref_of(M, c);
  float S1 = block_add(s1 * exp2_(r1 - M1), red), ST = block_add(sT * exp2_(rT - MT), red);
  if (is_far(M)) {
    float n = 0.f;
    seg.each([&](int, float (&v)[VEC], int nv) {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (e < nv) n += v[e] == M ? 1.f : v[e] == v[e] ? 0.f : v[e];
    });
    S1 = ST = block_add(n, red);
  }
  if (threadIdx.x == 0) a.part[(size_t)p * a.nseg + g] = Stat{M, M1, S1, ST};
}

template <typename T>
__device__ __forceinline__ void store_grad(T* p, const float (&v)[16 / sizeof(T)]) {
  uint4 w;
  if constexpr (sizeof(T) == 4) {
    w = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  } else {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = (uint32_t)f2bf(v[2 * i]) | ((uint32_t)f2bf(v[2 * i + 1]) << 16);
    w = make_uint4(u[0], u[1], u[2], u[3]);
  }
  *reinterpret_cast<uint4*>(p) = w;
}

// The loss of a row and one segment of its gradient
template <typename T, typename G>
__global__ __launch_bounds__(kThreads) void k_distill(DistillArgs a) {
  __shared__ float red[kWaves];
  __shared__ int tok[kMaxTeacherTokens];
  __shared__ float mass[kMaxTeacherTokens];
  constexpr int VEC = Segment<T>::VEC, GV = 16 / sizeof(G);
  const int64_t p = a.row0 + blockIdx.x / a.nseg;
  const int g = (int)(blockIdx.x % a.nseg);
  const size_t q = a.order ? (size_t)a.order[p] : (size_t)p;
  const Target tg = target_of(a, q);
  const Segment<T> seg = segment_of<T>(static_cast<const T*>(a.logits), a.ld, p, g, a.nseg, a.V);
  G* out = a.grad ? static_cast<G*>(a.grad) + (size_t)p * a.ld : nullptr;
  // the segment that holds column V - 1 writes the pad columns too; the empty ones behind it write nothing
  const int last = seg.v0 == seg.v1 ? 0 : seg.v1 * VEC >= a.V ? (int)a.ld : seg.v1 * VEC;
  if (!tg.any) {
    if (g == 0 && threadIdx.x == 0) a.row_loss[q] = 0.f;
    if (out)
      for (int col = seg.v0 * VEC + (int)threadIdx.x * GV; col < last; col += kThreads * GV)
        *reinterpret_cast<uint4*>(out + col) = make_uint4(0, 0, 0, 0);
    return;
  }
  // the row's sums at temperature 1 (s) and T (sT)
  const float c = kL2E / a.T;
  const int lane = threadIdx.x & 63;
  Stat st{neg_inf(), 0.f, 0.f, 0.f};
  if (lane < a.nseg) st = a.part[(size_t)p * a.nseg + lane];
  RowState r;
  r.m = wave_max(st.m);
  r.m2 = ref_of(r.m, kL2E);
  const float mT = ref_of(r.m, c);
  float f1 = exp2_(st.m2 - r.m2), fT = exp2_(ref_of(st.m, c) - mT);
  if (is_far(r.m)) f1 = fT = st.m == r.m ? 1.f : 0.f;
  r.s = wave_add(lane < a.nseg ? st.s * f1 : 0.f);
  const float sT = wave_add(lane < a.nseg ? st.t * fT : 0.f);
  r.t = 0.f;
  r.close();
  // teacher: q_j = softmax(t / T) over the entries that count
  const float tm = block_max(tg.have ? tg.t : neg_inf(), red);
  const float dt = (tg.t - tm) / a.T;
  const float e = tg.have ? expf(dt) : 0.f;
  const float es = block_add(e, red);
  const float qj = tg.have ? e / es : 0.f;
  const float* at = a.at + (size_t)p * (a.k + 1);
  const float zj = tg.have ? at[threadIdx.x] : 0.f, zy = at[a.k];
  if ((int)threadIdx.x < a.k) {
    tok[threadIdx.x] = tg.have ? tg.tok : -1;
    mass[threadIdx.x] = qj;
  }
  if (g == 0) {
    float lossj = 0.f;
    if (tg.have && qj != 0.f) {
      float lp;
      if (r.bad) lp = __builtin_nanf("");
      else if (r.empty) lp = neg_inf();
      else if (r.far || zj < -1e30f) lp = (zj - r.m) / a.T - kLn2 * log2_(sT);
      else lp = kLn2 * (__builtin_fmaf(zj, c, -mT) - log2_(sT));
      lossj = qj * (dt - logf(es) - lp);
    }
    float loss = a.soft * a.T * a.T * block_add(lossj, red);
    if (!tg.soft || a.soft == 0.f) loss = 0.f;
    if (tg.y >= 0 && a.hard != 0.f) loss -= a.hard * r.logp(zy);
    if (threadIdx.x == 0) a.row_loss[q] = loss;
  }
  if (!out) return;
  const float wa = tg.soft ? a.scale * a.soft * a.T : 0.f, wb = tg.y >= 0 ? a.scale * a.hard : 0.f;
  // weights of 2^x in the gradient; an empty row has none
  const float nan = __builtin_nanf("");
  const float ga = r.bad ? nan : r.empty ? 0.f : wa / sT, gb = r.bad ? nan : r.empty ? 0.f : wb / r.s;
  auto p1 = [&](float z) { return r.far ? (z == r.m ? 1.f : 0.f) : exp2_(__builtin_fmaf(z, kL2E, -r.m2)); };
  auto pT = [&](float z) { return r.far ? (z == r.m ? 1.f : 0.f) : exp2_(__builtin_fmaf(z, c, -mT)); };
  auto dense = [&](float z) { return ga * pT(z) + gb * p1(z); };
  const T* row = static_cast<const T*>(a.logits) + (size_t)p * a.ld;
  for (int col = seg.v0 * VEC + (int)threadIdx.x * 8; col < last; col += kThreads * 8) {
    float v[8];
#pragma unroll
    for (int h = 0; h < 8 / VEC; ++h) {
      float u[VEC];
      unpack<T>(*reinterpret_cast<const uint4*>(row + col + h * VEC), u);
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[h * VEC + i] = col + h * VEC + i < a.V ? dense(u[i]) : 0.f;
    }
#pragma unroll
    for (int h = 0; h < 8 / GV; ++h) {
      float u[GV];
#pragma unroll
      for (int i = 0; i < GV; ++i) u[i] = v[h * GV + i];
      store_grad<G>(out + col + h * GV, u);
    }
  }
  // the targets' columns once more, whole: the first entry of a token takes the mass of all its entries
  __syncthreads();
  const bool empty = r.empty;
  auto sparse = [&](int col, float z, float soft_mass, float hard_mass) {
    if (col < seg.v0 * VEC || col >= last) return;
    const float d = empty ? 0.f : r.bad ? nan
        : (wa / sT * pT(z) - wa * soft_mass) + (wb / r.s * p1(z) - wb * hard_mass);
    out[col] = from_f32<G>(d);
  };
  if (tg.have) {
    float sum = 0.f;
    bool lead = true;
    for (int j = 0; j < a.k; ++j) {
      if (tok[j] != tg.tok) continue;
      sum += mass[j];
      lead = lead && j >= (int)threadIdx.x;
    }
    if (lead) sparse(tg.tok, zj, sum, tg.tok == tg.y ? 1.f : 0.f);
  }
  if (threadIdx.x == 0 && tg.y >= 0) {
    bool seen = false;
    for (int j = 0; j < a.k; ++j) seen = seen || tok[j] == tg.y;
    if (!seen) sparse(tg.y, zy, 0.f, 1.f);
  }
}

// Segments of a row: rows alone fill the chip from kRowsFull on; below, a row is cut into pieces of at least kSegMin
// bytes, at most 64.
constexpr int kRowsFull = 1024, kSegMin = 16384;
constexpr int64_t kRowsLaunch = 1 << 22;  // rows of one launch: its threads are counted in 32 bits
int segments(int64_t rows, int V, int esize) {
  if (rows >= kRowsFull) return 1;
  const int64_t want = (kRowsFull + rows - 1) / std::max<int64_t>(rows, 1);
  const int64_t most = ((int64_t)V * esize + kSegMin - 1) / kSegMin;
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, most), 64));
}

}  // namespace

size_t token_workspace_bytes(int dtype, int64_t rows, int V, int K) {
  const int n = segments(rows, V, dtype == FOLD_BF16 ? 2 : 4);
  return n == 1 ? 0 : (size_t)rows * n * (sizeof(Stat) + (size_t)K * sizeof(uint64_t));
}

size_t distill_workspace_bytes(int dtype, int64_t rows, int V, int k) {
  const int n = segments(rows, V, dtype == FOLD_BF16 ? 2 : 4);
  return (size_t)rows * (n * sizeof(Stat) + (size_t)(k + 1) * sizeof(float));
}

void launch_token(int dtype, const int* order, int64_t rows, int V, const void* logits, int J, const int* tokens,
                  float* logp, float* entropy, int K, int* top_token, float* top_logp, void* ws, hipStream_t st) {
  if (rows <= 0) return;
  ProfScope prof("token_logprobs", st);
  const int n = segments(rows, V, dtype == FOLD_BF16 ? 2 : 4);
  TokenArgs a{0, order, logits, (size_t)row_ld(V), V, J, K, n, tokens, logp, entropy, top_token, top_logp,
              static_cast<Stat*>(ws), reinterpret_cast<uint64_t*>(static_cast<Stat*>(ws) + (size_t)rows * n)};
  for (; a.row0 < rows; a.row0 += kRowsLaunch) {
    const unsigned r = (unsigned)std::min<int64_t>(rows - a.row0, kRowsLaunch);
    if (dtype == FOLD_BF16) {
      hipLaunchKernelGGL(k_token<uint16_t>, dim3(r * n), dim3(kThreads), 0, st, a);
      if (n > 1) hipLaunchKernelGGL(k_token_join<uint16_t>, dim3(r), dim3(kThreads), 0, st, a);
    } else {
      hipLaunchKernelGGL(k_token<float>, dim3(r * n), dim3(kThreads), 0, st, a);
      if (n > 1) hipLaunchKernelGGL(k_token_join<float>, dim3(r), dim3(kThreads), 0, st, a);
    }
  }
}

void launch_distill(int dtype, const int* order, int64_t rows, int V, const void* logits, int k,
                    const int* teacher_token, const float* teacher_logit, const int* labels, float T, float soft,
                    float hard, float scale, float* row_loss, int grad_dtype, void* grad, void* ws, hipStream_t st) {
  if (rows <= 0) return;
  ProfScope prof("loss_distill", st);
  const int n = segments(rows, V, dtype == FOLD_BF16 ? 2 : 4);
  DistillArgs a{0, order, logits, (size_t)row_ld(V), V, k, n, teacher_token, teacher_logit, labels, T, soft, hard,
                scale, row_loss, grad, static_cast<Stat*>(ws),
                reinterpret_cast<float*>(static_cast<Stat*>(ws) + (size_t)rows * n)};
  for (; a.row0 < rows; a.row0 += kRowsLaunch) {
    const dim3 grid((unsigned)std::min<int64_t>(rows - a.row0, kRowsLaunch) * n);
    if (dtype == FOLD_BF16) {
      hipLaunchKernelGGL(k_distill_stats<uint16_t>, grid, dim3(kThreads), 0, st, a);
      hipLaunchKernelGGL((k_distill<uint16_t, uint16_t>), grid, dim3(kThreads), 0, st, a);
    } else {
      hipLaunchKernelGGL(k_distill_stats<float>, grid, dim3(kThreads), 0, st, a);
      if (grad_dtype == FOLD_BF16)
        hipLaunchKernelGGL((k_distill<float, uint16_t>), grid, dim3(kThreads), 0, st, a);
      else
        hipLaunchKernelGGL((k_distill<float, float>), grid, dim3(kThreads), 0, st, a);
    }
  }
}

}  // namespace fold
