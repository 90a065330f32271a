// Cross attention: the plan of a batch (which rows attend to which, cut into workgroups) and its launches.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fold.h"

namespace fold {

// Rows of a tile are "virtual": virtual row r of a query sequence is its query r / G and head r % G of a key head's group of G,
// so that heads that share keys share the loads of them.

// A workgroup's part of the forward pass or of the queries' gradient: up to 128 (32) virtual rows against a run of keys.
struct QTile {
  int32_t entry;           // list entry of the first row's query
  int32_t head0;           // the first row's head within its group
  int32_t rows;            // 0: nothing to do
  int32_t kv_head;         // the launch's second dimension
  int32_t k_begin, k_end;  // list entries of the keys
  int32_t slot;            // of the partial results (of the first head; a head's follow another's), -1: the results themselves
  int32_t pieces;          // of the tile, by the tile's first piece (its slot is theirs); 0 otherwise
};

// A workgroup's part of the gradient of keys and values: up to 128 keys against a run of row tiles.
struct KTile {
  int32_t k_begin, keys;   // keys 0: nothing to do
  int32_t kv_head;
  int32_t t_begin, t_end;  // row tiles
  int32_t slot, pieces;
  int32_t pad;
};
struct RTile {
  int32_t entry, head0, rows, pad;
};

struct Cross {
  int device = 0;
  int dtype = 0, heads = 0, kv_heads = 0, head_dim = 0, group = 0;
  int num_seqs = 0, num_sources = 0, num_queries = 0, num_keys = 0, query_rows = 0, key_rows = 0;
  void* blob = nullptr;  // every device array below
  int32_t *q_row = nullptr, *k_row = nullptr;  // the row of every list entry
  QTile* fwd = nullptr;   // the forward's workgroups
  QTile* fjoin = nullptr; // tiles in pieces
  QTile* back = nullptr;  // the queries' gradient's
  QTile* bjoin = nullptr;
  KTile* keys = nullptr;  // the keys' and values' gradient's
  KTile* kjoin = nullptr;
  RTile* rows = nullptr;
  QTile* brief = nullptr;    // rows of sources whose few keys give delta
  int32_t* others = nullptr; // list entries of all other rows that read a key; NULL: all entries
  int nfwd = 0, nfjoin = 0, nback = 0, nbjoin = 0, nkeys = 0, nkjoin = 0, nrows = 0, nbrief = 0, nothers = 0;
  int fslots = 0, bslots = 0, kslots = 0;  // of a head
  bool few = false;  // the forward takes tiles of 32 rows whose four waves share them and cut the keys
};

constexpr int kCrossHeadDim = 128;
constexpr int kCrossRows = 128, kCrossFew = 32;  // virtual rows of a workgroup
constexpr int kCrossFewBytes = 256;              // of a row that the tiles of 32 rows take: eight tiles of 32 keys in LDS
constexpr int kCrossKeys = 128;                  // keys of a workgroup of the keys' gradient


// Sources of up to so many keys give delta = sum_j p_j dp_j themselves, in fp32, where more keys take it from the forward's rounded
// out.  Beside few keys dp - delta is small and out's rounding is not: relative errors (L2) of dq in bf16 from out and from the
// keys, 2 keys 3.7e-3 and 2.3e-3, 4 2.9e-3, 16 2.5e-3, 32 2.43e-3 and 2.37e-3, 256 2.41e-3 and 2.36e-3 (a rounding of the result
// alone is 1.7e-3).  In fp32 out's rounding is not the largest; a single key, whose gradient is exactly 0, is looked at there too.
inline int cross_brief(int dtype) { return dtype == FOLD_BF16 ? 32 : 1; }
constexpr int kCrossBriefRows = 512;  // virtual rows of a workgroup that sums them

inline int cross_padded(int d) { return (d + 31) / 32 * 32; }  // a head's columns as the kernels hold them: 32, 64, 96, 128

// a matrix of the call: rows `ld` elements apart
struct CrossMat {
  const void* p;
  int64_t ld;
};

int32_t cross_create(const fold_cross_batch* b, hipStream_t st, fold_cross** out);
void cross_destroy(fold_cross* h);
size_t cross_forward_bytes(const Cross& c);
size_t cross_backward_bytes(const Cross& c);
void launch_cross(const Cross& c, CrossMat q, CrossMat k, CrossMat v, const uint8_t* mask, float scale, void* out,
                  int64_t ldo, float* lse, void* ws, hipStream_t st);
void launch_cross_backward(const Cross& c, CrossMat q, CrossMat k, CrossMat v, const uint8_t* mask, float scale, CrossMat out,
                           const float* lse, CrossMat dout, void* dq, int64_t lddq, void* dk, int64_t lddk, void* dv,
                           int64_t lddv, void* ws, hipStream_t st);

}  // namespace fold

struct fold_cross {
  fold::Cross c;
};
