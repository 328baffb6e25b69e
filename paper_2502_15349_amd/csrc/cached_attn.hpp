// Launch interface of attention over the paged cache.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ae {

// One set of key lists that the kernel walks: the sequences' own pages, or the shared prefix.  Rows are the query rows of one k/v
// head; row r of a list is token (r / g) % n, head r % g of the group, of sequence r / (n g) (of the list's own sequence where
// there is one list per sequence).
struct CachedPart {
  const int32_t* table;    // page numbers, row stride table_width (prefix: one row)
  const int32_t* lengths;  // device, per sequence; null: every list is max_length long
  int table_width, max_length;
  int lists;               // sequences, or 1
  int rows;                // query rows of a list
  int row_tiles;           // ceil(rows / rows of a workgroup)
  int chunk, splits;       // keys of a workgroup (a multiple of 32), ceil(max_length / chunk)
  int slot0;               // first of the part's partial results
  int causal;              // the newest n tokens of the list are the queries' own
};

struct CachedParams {
  const __bf16* Q;
  int64_t qs[3];  // element strides {batch, head, token}
  void* O;
  int64_t os[3];
  float* stats;   // optional [B, H_q, n]
  const uint8_t *K, *V, *Ke, *Ve;
  int B, H_q, H_kv, g, n, page_shift, n_pages;
  float c;        // scale * log2(e)
  int out_bf16;
  float* ws_o;    // [slots, B H_q n, D_v], null: one workgroup sees all keys of a row and writes O
  float* ws_lse;  // [slots, B H_q n]
  CachedPart part;
};

struct CachedMerge {
  const float* ws_o;
  const float* ws_lse;
  void* O;
  int64_t os[3];
  float* stats;
  const int32_t* lengths;
  int B, H_q, n, d_v, out_bf16;
  int prefix_slots;             // these are all there
  int chunk, max_length;        // own slots: ceil(length / chunk) of them are there
};

int cached_rows_per_workgroup(int dqk, int dv, bool e4m3, int rows);
hipError_t launch_cached(const CachedParams& p, int dqk, int dv, bool e4m3, hipStream_t s);
constexpr int kPrefixRows = 256;  // rows of a workgroup of launch_prefix
hipError_t launch_prefix(const CachedParams& p, int dqk, int dv, bool e4m3, hipStream_t s);
hipError_t launch_cached_merge(const CachedMerge& p, hipStream_t s);

}  // namespace ae
