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
  int tile_rows;           // query rows of a workgroup (of a prefix in the own keys' launch: of whole sequences)
  int row_tiles;           // ceil(rows / tile_rows)
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
  int waves;      // wavefronts of a workgroup of launch_cached: 4 or 8
  // The parts that a launch walks: the own lists (part[0]), and in front of their workgroups the prefix's (part[1], 0 or
  // prefix_blocks workgroups), where that has few rows.
  CachedPart part[2];
  int prefix_blocks;
  // Partial results, where a row has more than one: slots [0, part[0].slot0) the prefix's, the others the own list's.
  float* ws_o;        // [slots, B H_q n, D_v], normalised
  float* ws_lse;      // [slots, B H_q n], log2 of the sum of weights
  int32_t* counters;  // [B * H_kv * row tiles], kCounterStride apart, of workgroups that are done, zero before and after the launch; null: no workgroup waits for others
};

// Workgroups of `units` pieces of work with `tiles` row tiles each, dealt to the XCDs (which take the workgroups of a launch in turn):
// tiles of a unit read the same keys and go to one XCD, one after the other, so that its L2 has them for the second; the tiles of
// what is left over from whole rounds of eight units are spread over all XCDs.  (161 sequences x 8 tokens x 8/1 heads, 64/64, behind
// 13658 keys in four ranges: 175 us with a unit to an XCD throughout, 94 so.)
constexpr int kXcds = 8;
inline int64_t dealt_workgroups(int64_t units, int64_t tiles) {
  return units / kXcds * kXcds * tiles + (units % kXcds * tiles + kXcds - 1) / kXcds * kXcds;
}
// Which one a workgroup is; false: none.
__device__ __forceinline__ bool dealt_to(int block, int units, int tiles, int& unit, int& tile) {
  const int xcd = block % kXcds, slot = block / kXcds, whole = units / kXcds * tiles;
  if (slot < whole) {
    unit = slot / tiles * kXcds + xcd;
    tile = slot % tiles;
    return true;
  }
  const int64_t rest = (int64_t)(units % kXcds) * tiles;
  const int item = (int)(xcd * rest / kXcds) + slot - whole;
  unit = units / kXcds * kXcds + item / tiles;
  tile = item % tiles;
  return item < (int)((xcd + 1) * rest / kXcds);
}

// Ints from one counter to the next: a cache line each (side by side, 1 x 16 heads x 7984 8-bit keys of 64 + 64 took 16.5 us instead of 12.1).
constexpr int kCounterStride = 32;
int cached_rows_per_workgroup(int rows);  // at most
// Workgroups of so many rows and wavefronts that a compute unit holds at a time.
int cached_residents(int dqk, int dv, bool e4m3, int rows, int waves);
hipError_t launch_cached(const CachedParams& p, int dqk, int dv, bool e4m3, hipStream_t s);
constexpr int kPrefixRows = 256;  // rows of a workgroup of launch_prefix, which walks part[1] alone
hipError_t launch_prefix(const CachedParams& p, int dqk, int dv, bool e4m3, hipStream_t s);
hipError_t launch_fill_zero(int32_t* at, int64_t n, hipStream_t s);

}  // namespace ae
