// What the kernels of attention over a paged cache share: the call's
// parameters, its blocks of queries, and which rows a block sees.
#pragma once

#include "heads.hpp"

namespace pf {

constexpr int kBlock = 16;      // rows per block: a page is a multiple of it
constexpr int kMaxSlices = 512;

struct PagedParams {
  const char* q;
  int64_t q_ts, q_hs;
  const char* k;
  const char* v;
  const int32_t* table;
  const int32_t* kv_len;
  const int32_t* cu;    // NULL: one token of every sequence
  int n_pages, page_size, max_pages, batch, n_tokens;
  FastDiv page_blocks;  // blocks per page
  int hq, hk, group;
  FastDiv fgroup, fhk, fslices, fblocks;  // fblocks: blocks of a sequence without cu
  int cols, tile_rows;  // queries of a workgroup, rows of a tile (both powers of two)
  int slices;           // at most
  FastDiv fmin_tiles;   // least tiles of a slice
  int window, sinks;    // window: INT32_MAX without one
  float scale_log2;
  void* out;
  float* lse;
  float* part_o;        // [n_tokens * hq, slices, D]
  float2* part_ml;      // [n_tokens * hq, slices]
};

// The new tokens of one sequence. Column x of a (sequence, K/V head) is token
// x / group, head x % group of the group.
struct Sequence {
  int seq;       // -1: none
  int t0;        // its first token in the call
  int cols;
  int row0;      // row of that token
  int most;      // rows that the table holds
  __device__ __forceinline__ void set(const PagedParams& p, int s) {
    seq = s;
    int n_new = 1;
    t0 = s;
    if (p.cu) {
      t0 = p.cu[s];
      n_new = p.cu[s + 1] - t0;
      if (t0 < 0 || n_new <= 0 || n_new > p.n_tokens - t0) {  // nothing there, or boundaries that are none
        seq = -1;
        n_new = 0;
      }
    }
    cols = n_new * p.group;
    const int64_t first = (int64_t)p.kv_len[s] - n_new;
    row0 = (int)(first < -n_new ? -n_new : first);
    most = p.max_pages * p.page_size;
  }
};

// Blocks of COLS columns: sequence s takes blocks cu[s] * group / COLS + s on,
// at least as many as its columns fill, so a block finds its sequence without
// a sum over the others.
template <int COLS>
__device__ __forceinline__ int first_block(const PagedParams& p, int s) {
  return p.cu ? (int)((int64_t)p.cu[s] * p.group / COLS) + s : s * ((p.group + COLS - 1) / COLS);
}
template <int COLS>
__device__ __forceinline__ int sequence_of_block(const PagedParams& p, int blk) {
  return p.cu ? find_run(p.batch, [&](int c) { return first_block<COLS>(p, c); }, blk) : p.fblocks.div(blk);
}
// Their number (n_tokens < 0: one token of every sequence).
inline int64_t col_blocks(int cols, int group, int64_t n_tokens, int batch) {
  return n_tokens < 0 ? (int64_t)batch * ((group + cols - 1) / cols) : n_tokens * group / cols + batch;
}

// The rows that a block of columns sees, as a list of tiles: those of the
// first rows, then those of the windows.
struct Sight {
  int first, top;   // rows of its first and last token
  int last;         // the last row that it sees: top, or the table's end (-1: none)
  int head_tiles;   // tiles that hold the first rows
  int gap;          // added to later tile numbers
  int tiles;
  __host__ __device__ __forceinline__ Sight(const PagedParams& p, const Sequence& sq, int x0, int cols, int tile_rows) {
    first = max(sq.row0 + p.fgroup.div(x0), 0);
    top = max(sq.row0 + p.fgroup.div(x0 + cols - 1), -1);
    last = min(top, sq.most - 1);
    const int lo = max(first - p.window + 1, 0), n = last + 1;
    head_tiles = (min(min(p.sinks, lo), sq.most) + tile_rows - 1) / tile_rows;  // (lengths may pass the table)
    gap = max(lo / tile_rows - head_tiles, 0);
    const int all = (n + tile_rows - 1) / tile_rows;  // (the windows may lie past the table's end)
    tiles = min(head_tiles, all) + max(all - head_tiles - gap, 0);
  }
  __host__ __device__ __forceinline__ int tile(int i) const { return i < head_tiles ? i : i + gap; }
  // As many slices as leave each min_tiles, all of the same size but the last.
  __host__ __device__ __forceinline__ int per_slice(const PagedParams& p) const {
    const int n = max(min(p.fmin_tiles.div(tiles), p.slices), 1);
    return max((tiles + n - 1) / n, 1);
  }
};

// The prompts' kernel (bf16): out and lse, or with slices > 1 partial results
// for the join.
hipError_t launch_paged_prompt(const PagedParams& p, int d, int64_t groups, hipStream_t s);

}  // namespace pf
