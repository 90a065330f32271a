// Plans of cross attention: the lists are checked on the GPU, the workgroups are laid out on the host, whose copy of the
// sequences' lengths lets long ones be cut and the work be spread over the chip.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstring>
#include <string>
#include <vector>

#include "checks.h"
#include "common.h"
#include "cross.h"
#include "pool.h"

namespace fold {

namespace {

__global__ __launch_bounds__(256) void k_zero_words(uint32_t* p, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = 0;
}

// the arrays that the host looks at, and the error word, one after the other
__global__ __launch_bounds__(256) void k_collect(const int32_t* a, int64_t na, const int32_t* b, int64_t nb, const int32_t* c,
                                                 int64_t nc, const uint32_t* error, int32_t* out) {
  const int64_t n = na + nb + nc + 1;
  for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256)
    out[i] = i < na ? a[i] : i < na + nb ? b[i - na] : i < na + nb + nc ? c[i - na - nb] : (int32_t)*error;
}

// error bits: 1 a row out of range, 2 a row listed twice
__global__ __launch_bounds__(256) void k_check_rows(const int32_t* row, int n, int limit, uint32_t* seen, uint32_t* error,
                                                    int shift) {
  for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
    const int r = row[i];
    if (r < 0 || r >= limit) {
      atomicOr(error, 1u << shift);
    } else {
      const uint32_t bit = 1u << (r & 31);
      if (atomicOr(&seen[r >> 5], bit) & bit) atomicOr(error, 2u << shift);
    }
  }
}

__global__ __launch_bounds__(256) void k_identity(int32_t* row, int n) {
  for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) row[i] = (int32_t)i;
}

struct Range {
  int64_t begin, end;
  int64_t size() const { return end - begin; }
};

// Workgroups of a head in launch order.  The XCDs take them in turn and each has an L2 of its own, so the workgroups that read the same
// keys (or rows) follow each other on one XCD: chunks of a group go, the costliest first, to the XCD with the least work.
template <class Tile>
struct Spread {
  struct Chunk {
    size_t begin, end;
    int64_t cost;
  };
  std::vector<Tile> all;
  std::vector<int64_t> cost;
  std::vector<size_t> groups{0};  // where groups begin
  void add(const Tile& t, int64_t c) {
    all.push_back(t);
    cost.push_back(c + 64);  // a workgroup's own start and end
  }
  void close() {
    if (groups.back() != all.size()) groups.push_back(all.size());
  }
  std::vector<Tile> order() const {
    const size_t most = std::max<size_t>(1, std::min<size_t>(64, all.size() / 64));
    std::vector<Chunk> chunks;
    for (size_t g = 0; g + 1 < groups.size(); ++g)
      for (size_t b = groups[g]; b < groups[g + 1]; b += most) {
        Chunk c{b, std::min(b + most, groups[g + 1]), 0};
        for (size_t i = c.begin; i < c.end; ++i) c.cost += cost[i];
        chunks.push_back(c);
      }
    // the costliest workgroups first, so that short ones fill the end
    std::stable_sort(chunks.begin(), chunks.end(), [&](const Chunk& a, const Chunk& b) {
      return a.cost / (int64_t)(a.end - a.begin) > b.cost / (int64_t)(b.end - b.begin);
    });
    std::vector<std::vector<size_t>> lane(8);
    int64_t load[8] = {0};
    for (const Chunk& c : chunks) {
      int x = 0;
      for (int i = 1; i < 8; ++i)
        if (load[i] < load[x]) x = i;
      load[x] += c.cost;
      for (size_t i = c.begin; i < c.end; ++i) lane[x].push_back(i);
    }
    size_t deep = 0;
    for (const auto& l : lane) deep = std::max(deep, l.size());
    Tile none{};
    std::vector<Tile> out(deep * 8, none);
    for (int x = 0; x < 8; ++x)
      for (size_t i = 0; i < lane[x].size(); ++i) out[i * 8 + x] = all[lane[x][i]];
    return out;  // a multiple of 8: the tiles of every head go to the same XCDs
  }
};

// Keys (or rows) of a piece at least.  A piece costs its partial results' way through memory and a share of the join, a tile
// of 32 x 32 scores sixteen times as much on the matrix cores in fp32 as in bf16.  Gradient of 8 sequences of 428 .. 737 nodes
// against 358 .. 449, two heads of 128 in bf16: 50 us with 256, 67 with 128; of 18 of 172 .. 260 against 12 .. 33, two heads of
// 75 in fp32: 94 with 256, 58 with 128; of 27 sources of 216 .. 230 read by five of 361 .. 802 each, a head of 16 in fp32: 52
// with 256, 54 with 128, 63 with 64.
int min_piece(int dtype) { return dtype == FOLD_BF16 ? 256 : 128; }
constexpr int kWanted = 512;    // workgroups that fill the chip: two a compute unit

// The length of pieces: what spreads the work evenly over the wanted workgroups, where there are fewer tiles than that; with
// more tiles only one that is far longer than the others is cut.
int64_t piece_of(int64_t tiles, int64_t work, int unit, int least) {
  if (tiles == 0) return least;
  int64_t len = std::max<int64_t>(least, (work + kWanted - 1) / kWanted);
  if (tiles >= kWanted) len = std::max<int64_t>(len, 4 * (work / tiles));
  return (len + unit - 1) / unit * unit;
}

struct Lists {
  const std::vector<int32_t>&qp, &kp;
  int G, kv_heads, least;
  std::vector<int32_t> first, seqs;  // source e's query sequences: seqs[first[e]] .. ; the last entry: those without a source
  struct Run {
    const int32_t *b, *e;
    const int32_t* begin() const { return b; }
    const int32_t* end() const { return e; }
  };
  Run readers(int64_t e) const { return {seqs.data() + first[e], seqs.data() + first[e + 1]}; }
};

// tiles of `height` virtual rows (launched for every key head) in pieces of the keys; the tiles in pieces also go to `join`
void query_tiles(const Lists& l, int height, std::vector<QTile>* out, std::vector<QTile>* join, int* slots) {
  const int64_t sources = (int64_t)l.kp.size() - 1;
  int64_t tiles = 0, work = 0;
  const auto keys_of = [&](int64_t e) { return e < sources ? (int64_t)l.kp[e + 1] - l.kp[e] : 0; };
  const auto rows_of = [&](int b) { return ((int64_t)l.qp[b + 1] - l.qp[b]) * l.G; };
  for (int64_t e = 0; e <= sources; ++e)
    for (int b : l.readers(e)) {
      const int64_t n = (rows_of(b) + height - 1) / height * l.kv_heads;
      tiles += n;
      work += n * keys_of(e);
    }
  const int64_t piece = piece_of(tiles, work, 64, l.least);
  Spread<QTile> s;
  *slots = 0;
  for (int64_t e = 0; e <= sources; ++e) {
    const int64_t nk = keys_of(e), pieces = std::max<int64_t>(1, (nk + piece - 1) / piece);
    const int64_t each = ((nk + pieces - 1) / pieces + 63) / 64 * 64;
    const int n = (int)(each ? std::max<int64_t>(1, (nk + each - 1) / each) : 1);
    const int32_t k0 = e < sources ? l.kp[e] : 0;
    for (int b : l.readers(e))
      for (int64_t r = 0; r < rows_of(b); r += height) {
        QTile t{};
        t.entry = (int32_t)(l.qp[b] + r / l.G);
        t.head0 = (int32_t)(r % l.G);
        t.rows = (int32_t)std::min<int64_t>(height, rows_of(b) - r);
        for (int p = 0; p < n; ++p) {
          t.k_begin = (int32_t)(k0 + std::min<int64_t>(p * each, nk));
          t.k_end = (int32_t)(k0 + std::min<int64_t>((p + 1) * each, nk));
          t.slot = n > 1 ? *slots + p : -1;
          t.pieces = p == 0 ? n : 0;
          s.add(t, t.k_end - t.k_begin);
          if (n > 1 && p == 0) join->push_back(t);
        }
        if (n > 1) *slots += n;
      }
    s.close();
  }
  *out = s.order();
}

// tiles of the rows whose source has up to `most` keys, and the list entries of all others that read a key
void brief_tiles(const Lists& l, int most, std::vector<QTile>* tiles, std::vector<int32_t>* others) {
  const int64_t sources = (int64_t)l.kp.size() - 1;
  for (int64_t e = 0; e < sources; ++e) {
    const int64_t nk = (int64_t)l.kp[e + 1] - l.kp[e];
    if (nk == 0) continue;
    for (int b : l.readers(e)) {
      const int64_t n = ((int64_t)l.qp[b + 1] - l.qp[b]) * l.G;
      if (nk > most) {
        for (int32_t i = l.qp[b]; i < l.qp[b + 1]; ++i) others->push_back(i);
        continue;
      }
      for (int64_t r = 0; r < n; r += kCrossBriefRows)
        tiles->push_back(QTile{(int32_t)(l.qp[b] + r / l.G), (int32_t)(r % l.G),
                               (int32_t)std::min<int64_t>(kCrossBriefRows, n - r), 0, l.kp[e], l.kp[e + 1], -1, 0});
    }
  }
}

void key_tiles(const Lists& l, int height, std::vector<KTile>* out, std::vector<KTile>* join, std::vector<RTile>* rows,
               int* slots) {
  const int64_t sources = (int64_t)l.kp.size() - 1;
  std::vector<Range> runs(sources);
  int64_t tiles = 0, work = 0;
  for (int64_t e = 0; e < sources; ++e) {
    runs[e].begin = (int64_t)rows->size();
    for (int b : l.readers(e)) {
      const int64_t n = ((int64_t)l.qp[b + 1] - l.qp[b]) * l.G;
      for (int64_t r = 0; r < n; r += height)
        rows->push_back(RTile{(int32_t)(l.qp[b] + r / l.G), (int32_t)(r % l.G), (int32_t)std::min<int64_t>(height, n - r), 0});
    }
    runs[e].end = (int64_t)rows->size();
    const int64_t n = ((int64_t)l.kp[e + 1] - l.kp[e] + kCrossKeys - 1) / kCrossKeys * l.kv_heads;
    tiles += n;
    work += n * runs[e].size() * height;
  }
  const int64_t piece = piece_of(tiles, work, height, l.least) / height;  // row tiles
  Spread<KTile> s;
  *slots = 0;
  for (int64_t e = 0; e < sources; ++e) {
    const int64_t nr = runs[e].size(), pieces = std::max<int64_t>(1, (nr + piece - 1) / piece);
    const int64_t each = std::max<int64_t>(1, (nr + pieces - 1) / pieces);
    const int n = (int)std::max<int64_t>(1, (nr + each - 1) / each);
    for (int64_t k = l.kp[e]; k < l.kp[e + 1]; k += kCrossKeys) {
      KTile t{};
      t.k_begin = (int32_t)k;
      t.keys = (int32_t)std::min<int64_t>(kCrossKeys, l.kp[e + 1] - k);
      for (int p = 0; p < n; ++p) {
        t.t_begin = (int32_t)(runs[e].begin + std::min<int64_t>(p * each, nr));
        t.t_end = (int32_t)(runs[e].begin + std::min<int64_t>((p + 1) * each, nr));
        t.slot = n > 1 ? *slots + p : -1;
        t.pieces = p == 0 ? n : 0;
        s.add(t, (int64_t)(t.t_end - t.t_begin) * height);
        if (n > 1 && p == 0) join->push_back(t);
      }
      if (n > 1) *slots += n;
    }
    s.close();
  }
  *out = s.order();
}

// checks one of the ptr arrays; the total it ends at
bool check_ptr(const std::vector<int32_t>& p, int total) {
  if (p[0] != 0 || p.back() != total) return false;
  for (size_t i = 1; i < p.size(); ++i)
    if (p[i] < p[i - 1]) return false;
  return true;
}

// gives a temporary block back on every path, after its stream has finished with it
struct Block {
  int device;
  hipStream_t st;
  void* p = nullptr;
  ~Block() {
    if (p && hipStreamSynchronize(st) == hipSuccess) pool_free(device, p, false);
  }
};

unsigned grid_for(size_t n) { return (unsigned)std::max<size_t>(1, std::min<size_t>((n + 255) / 256, 2048)); }

}  // namespace

int32_t cross_create(const fold_cross_batch* b, hipStream_t st, fold_cross** out) {
  const std::string who("fold_cross_create");
  if (!known_type(b->dtype)) return api_fail(FOLD_E_INVALID, who + ": unknown dtype");
  if (b->heads < 1 || b->heads > 1024 || b->kv_heads < 1 || b->heads % b->kv_heads != 0 || b->heads / b->kv_heads > 256)
    return api_fail(FOLD_E_INVALID, who + ": heads must be 1 .. 1024, a multiple of kv_heads, at most 256 times");
  if (b->head_dim < 1 || b->head_dim > kCrossHeadDim) return api_fail(FOLD_E_INVALID, who + ": head_dim must be 1 .. 128");
  if (b->num_seqs < 0 || b->num_sources < 0 || b->num_queries < 0 || b->num_keys < 0 || b->num_query_rows < 0 ||
      b->num_key_rows < 0)
    return api_fail(FOLD_E_INVALID, who + ": negative count");
  if ((int64_t)b->num_queries * b->heads > INT32_MAX)
    return api_fail(FOLD_E_INVALID, who + ": queries times heads reach 2^31");
  // before a list is looked at: a tile holds at most kCrossKeys keys (kCrossRows rows), so these are too many tiles however they
  // fall into sequences.  What is left ends 1,024 entries below 2^31, and a list entry plus a tile fits 32 bits.
  const std::string many = who + ": too many tiles for one launch (sequences, rows and keys)";
  if (((int64_t)b->num_keys + kCrossKeys - 1) / kCrossKeys >= kMaxTiles ||
      ((int64_t)b->num_queries * (b->heads / b->kv_heads) + kCrossRows - 1) / kCrossRows >= kMaxTiles)
    return api_fail(FOLD_E_INVALID, many);
  if (!b->query_ptr || !b->key_ptr) return api_fail(FOLD_E_INVALID, who + ": NULL query_ptr or key_ptr");
  if (!b->source && b->num_seqs != b->num_sources)
    return api_fail(FOLD_E_INVALID, who + ": without `source` there is a key sequence for each query sequence");
  if (b->num_queries > b->num_query_rows || b->num_keys > b->num_key_rows)
    return api_fail(FOLD_E_INVALID, who + ": more rows are listed than there are");
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(st, &capture) == hipSuccess && capture != hipStreamCaptureStatusNone)
    return api_fail(FOLD_E_INVALID, who + ": the stream is being captured (a plan is made before)");
  (void)hipGetLastError();

  int device = 0;
  FOLD_HIP_CHECK(hipGetDevice(&device));
  const int64_t nq = (int64_t)b->num_seqs + 1, nk = (int64_t)b->num_sources + 1, ns = b->source ? b->num_seqs : 0;
  std::vector<int32_t> qp(nq), kp(nk), src(ns);
  uint32_t error = 0;
  const size_t qw = b->query_row ? ((size_t)b->num_query_rows + 31) / 32 : 0;
  const size_t kw = b->key_row ? ((size_t)b->num_key_rows + 31) / 32 : 0, n = (size_t)nq + nk + ns + 1;
  {
    Block tmp{device, st};
    tmp.p = pool_alloc(device, (64 + qw + kw + n) * sizeof(uint32_t), false);
    if (!tmp.p) return api_fail(FOLD_E_NOMEM, who + ": no device memory");
    uint32_t* words = static_cast<uint32_t*>(tmp.p);
    int32_t* lists = reinterpret_cast<int32_t*>(words + 64 + qw + kw);
    hipLaunchKernelGGL(k_zero_words, dim3(grid_for(64 + qw + kw)), dim3(256), 0, st, words, 64 + qw + kw);
    if (qw)
      hipLaunchKernelGGL(k_check_rows, dim3(grid_for(b->num_queries)), dim3(256), 0, st, b->query_row, b->num_queries,
                         b->num_query_rows, words + 64, words, 0);
    if (kw)
      hipLaunchKernelGGL(k_check_rows, dim3(grid_for(b->num_keys)), dim3(256), 0, st, b->key_row, b->num_keys,
                         b->num_key_rows, words + 64 + qw, words, 2);
    hipLaunchKernelGGL(k_collect, dim3(grid_for(n)), dim3(256), 0, st, b->query_ptr, nq, b->key_ptr, nk, b->source, ns, words,
                       lists);
    FOLD_HIP_CHECK(hipGetLastError());
    struct Stage {  // pinned, where the lists fit it
      int* p;
      ~Stage() { stage_free(p); }
    } stage{n <= kStageInts ? stage_alloc() : nullptr};
    std::vector<int32_t> far(stage.p ? 0 : n);
    int32_t* got = stage.p ? stage.p : far.data();
    if (hipMemcpyAsync(got, lists, n * sizeof(int32_t), hipMemcpyDeviceToHost, st) != hipSuccess ||
        hipStreamSynchronize(st) != hipSuccess)
      return api_fail(FOLD_E_DEVICE, who + ": the lists could not be read");
    std::copy(got, got + nq, qp.begin());
    std::copy(got + nq, got + nq + nk, kp.begin());
    std::copy(got + nq + nk, got + nq + nk + ns, src.begin());
    error = (uint32_t)got[n - 1];
  }
  if (!check_ptr(qp, b->num_queries)) return api_fail(FOLD_E_INVALID, who + ": query_ptr malformed");
  if (!check_ptr(kp, b->num_keys)) return api_fail(FOLD_E_INVALID, who + ": key_ptr malformed");
  if (error & 5) return api_fail(FOLD_E_INVALID, who + (error & 1 ? ": query_row" : ": key_row") + " out of range");
  if (error & 10) return api_fail(FOLD_E_INVALID, who + (error & 2 ? ": query_row" : ": key_row") + " lists a row twice");
  Lists l{qp, kp, b->heads / b->kv_heads, b->kv_heads, min_piece(b->dtype), {}, {}};
  const auto source_of = [&](int s) -> int64_t {
    const int e = b->source ? src[s] : s;
    return e < 0 ? b->num_sources : e;
  };
  l.first.assign((size_t)nk + 1, 0);
  for (int s = 0; s < b->num_seqs; ++s) {
    if (b->source && (src[s] < -1 || src[s] >= b->num_sources))
      return api_fail(FOLD_E_INVALID, who + ": source out of range");
    ++l.first[source_of(s) + 1];
  }
  int64_t key_tile_count = 0;
  for (int64_t e = 0; e < nk; ++e) {
    if (e < b->num_sources) key_tile_count += ((int64_t)kp[e + 1] - kp[e] + kCrossKeys - 1) / kCrossKeys;
    l.first[e + 1] += l.first[e];
  }
  if (key_tile_count >= kMaxTiles) return api_fail(FOLD_E_INVALID, many);
  l.seqs.resize(b->num_seqs);
  {
    std::vector<int32_t> at(l.first.begin(), l.first.end() - 1);
    for (int s = 0; s < b->num_seqs; ++s) l.seqs[at[source_of(s)]++] = s;
  }

  fold_cross* h = new fold_cross;
  Cross& c = h->c;
  struct Guard {
    fold_cross*& h;
    ~Guard() { cross_destroy(h); }
  } guard{h};
  c.device = device;
  c.dtype = b->dtype;
  c.heads = b->heads;
  c.kv_heads = b->kv_heads;
  c.head_dim = b->head_dim;
  c.group = l.G;
  c.num_seqs = b->num_seqs;
  c.num_sources = b->num_sources;
  c.num_queries = b->num_queries;
  c.num_keys = b->num_keys;
  c.query_rows = b->num_query_rows;
  c.key_rows = b->num_key_rows;
  // tiles of 32 rows where those of 128 would be mostly empty: 64 sequences against 500 keys, 8 heads of 64 in bf16, low and tall
  // tiles: 8 rows of 16 heads on 4 17.7 and 18.5 us, 16 rows 16.8 and 16.6, 64 rows 21.7 and 20.0; 96 rows against 2,000 keys 75.5
  // and 57.4.  Low tiles of bf16 heads above 64 leave one workgroup a compute unit, so where tall ones fill the chip twice over
  // they stay tall: 256 sequences, 8 heads of 128, single rows against 2,000 keys 379 and 361 us, 8 rows against 500 125 and 111;
  // 16 sequences 16.5 and 18.2
  int64_t tall = 0, low = 0, least_tiles = 0;
  for (int s = 0; s < b->num_seqs; ++s) {
    const int64_t n = (int64_t)(qp[s + 1] - qp[s]) * l.G, e = b->source ? src[s] : s;
    const int64_t keys = e < 0 ? 0 : kp[e + 1] - kp[e];
    least_tiles += (n + kCrossRows - 1) / kCrossRows;
    tall += (n + kCrossRows - 1) / kCrossRows * keys;
    low += (n + kCrossFew - 1) / kCrossFew * keys;
  }
  if (least_tiles >= kMaxTiles) return api_fail(FOLD_E_INVALID, many);
  const bool full = c.dtype == FOLD_BF16 && cross_padded(c.head_dim) > 64 && least_tiles * c.kv_heads >= 4 * 256;
  c.few = low < 2 * tall && !full && cross_padded(c.head_dim) * (c.dtype == FOLD_BF16 ? 2 : 4) <= kCrossFewBytes;
  std::vector<QTile> fwd, fjoin, back, bjoin;
  std::vector<KTile> keys, kjoin;
  std::vector<RTile> rows;
  query_tiles(l, c.few ? kCrossFew : kCrossRows, &fwd, &fjoin, &c.fslots);
  query_tiles(l, kCrossRows, &back, &bjoin, &c.bslots);
  key_tiles(l, c.dtype == FOLD_BF16 ? 64 : 32, &keys, &kjoin, &rows, &c.kslots);
  std::vector<QTile> brief;
  std::vector<int32_t> others;
  brief_tiles(l, cross_brief(c.dtype), &brief, &others);
  c.nothers = (int)others.size();
  if (c.nothers == c.num_queries) others.clear();  // all of them

  if ((int64_t)std::max({fwd.size(), back.size() + keys.size(), 4 * fjoin.size(), 4 * bjoin.size(), 4 * kjoin.size()}) >= kMaxTiles)
    return api_fail(FOLD_E_INVALID, many);
  // one image of all the lists, uploaded whole; the row numbers behind it are copied or made on the device
  std::vector<char> image;
  const auto place = [&](const void* data, size_t size) {
    const size_t at = image.size();
    image.resize(at + (size + 255) / 256 * 256);
    if (size) std::memcpy(image.data() + at, data, size);
    return at;
  };
  const size_t at_fwd = place(fwd.data(), fwd.size() * sizeof(QTile)), at_fj = place(fjoin.data(), fjoin.size() * sizeof(QTile)),
               at_back = place(back.data(), back.size() * sizeof(QTile)),
               at_bj = place(bjoin.data(), bjoin.size() * sizeof(QTile)),
               at_keys = place(keys.data(), keys.size() * sizeof(KTile)),
               at_kj = place(kjoin.data(), kjoin.size() * sizeof(KTile)),
               at_rows = place(rows.data(), rows.size() * sizeof(RTile)),
               at_brief = place(brief.data(), brief.size() * sizeof(QTile)),
               at_others = place(others.data(), others.size() * sizeof(int32_t));
  const size_t at_qr = image.size(), at_kr = at_qr + ((size_t)b->num_queries * 4 + 255) / 256 * 256;
  c.blob = pool_alloc(device, std::max<size_t>(at_kr + (size_t)b->num_keys * 4, 256), true);
  if (!c.blob) return api_fail(FOLD_E_NOMEM, who + ": no device memory");
  char* base = static_cast<char*>(c.blob);
  bool ok = image.empty() || hipMemcpyAsync(base, image.data(), image.size(), hipMemcpyHostToDevice, st) == hipSuccess;
  const auto keep = [&](size_t at, const int32_t* from, int count) {
    int32_t* to = reinterpret_cast<int32_t*>(base + at);
    if (count > 0 && from)
      ok = ok && hipMemcpyAsync(to, from, (size_t)count * 4, hipMemcpyDeviceToDevice, st) == hipSuccess;
    else if (count > 0)
      hipLaunchKernelGGL(k_identity, dim3(grid_for(count)), dim3(256), 0, st, to, count);
    return to;
  };
  c.q_row = keep(at_qr, b->query_row, b->num_queries);
  c.k_row = keep(at_kr, b->key_row, b->num_keys);
  if (!(hipStreamSynchronize(st) == hipSuccess && ok)) return api_fail(FOLD_E_DEVICE, who + ": the plan could not be written");
  c.fwd = reinterpret_cast<QTile*>(base + at_fwd);
  c.fjoin = reinterpret_cast<QTile*>(base + at_fj);
  c.back = reinterpret_cast<QTile*>(base + at_back);
  c.bjoin = reinterpret_cast<QTile*>(base + at_bj);
  c.keys = reinterpret_cast<KTile*>(base + at_keys);
  c.kjoin = reinterpret_cast<KTile*>(base + at_kj);
  c.rows = reinterpret_cast<RTile*>(base + at_rows);
  c.brief = reinterpret_cast<QTile*>(base + at_brief);
  c.others = others.empty() ? nullptr : reinterpret_cast<int32_t*>(base + at_others);
  c.nfwd = (int)fwd.size();
  c.nfjoin = (int)fjoin.size();
  c.nback = (int)back.size();
  c.nbjoin = (int)bjoin.size();
  c.nkeys = (int)keys.size();
  c.nkjoin = (int)kjoin.size();
  c.nrows = (int)rows.size();
  c.nbrief = (int)brief.size();
  *out = h;
  h = nullptr;
  return FOLD_OK;
}

void cross_destroy(fold_cross* h) {
  if (!h) return;
  if (h->c.blob) pool_free_after_wait(h->c.device, h->c.blob);
  delete h;
}

}  // namespace fold
