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
  // What only some calls have, behind the rest, which so comes in the fewest loads:
  // with these between (and a test for packed rows in Sequence::set) prompts of 4 x
  // 500 tokens behind 500 fp32 rows, 8 over 2 heads of 64, took 54.2 us for 53.2, 16 of
  // 32 behind 1,000, 32 over 8 heads of 128, 35.5 for 34.9.
  const uint8_t* k_scale;  // pages of 8 bits: scale bytes of the rows
  const uint8_t* v_scale;
  int64_t k_ts, k_hs, v_ts, v_hs;  // packed rows, no pages: strides in elements
};

// The new tokens of one sequence. Column x of a (sequence, K/V head) is token
// x / group, head x % group of the group.
struct Sequence {
  int seq;       // -1: none
  int t0;        // its first token in the call
  int cols;
  int row0;      // row of that token
  int most;      // rows that the table holds
  // PACKED: a sequence's tokens are its rows.
  template <bool PACKED = false>
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
    if constexpr (PACKED) {
      row0 = 0;
      most = INT32_MAX;
      return;
    }
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

// The head and the item of this workgroup among `per_head` of each of `hks`
// K/V heads, a launch of their product. Workgroups go to the XCDs in turn; a
// head's items stay on as few XCDs as its share of them (their L2s hold its
// rows), and every XCD gets every rank of them, heavy ones first. Rounds of a
// workgroup per CU go up and down the ranks in turn, so where most are resident
// at once a heavy one shares a CU with a light one (a prompt of 8,192 tokens, 16
// heads of 64, 1,040 workgroups: 178 us, all rounds down 193). Of more than six
// rounds all go down: what begins last is then lightest (32 over 8 heads of 128,
// 2,056 workgroups: 518 us, up and down 526).
struct Item {
  int hk, at;
  __device__ __forceinline__ Item(int hks, const FastDiv& fhk, int per_head) {
    constexpr int kCus = 32;  // of an XCD
    const int id = (int)blockIdx.x;
    int i, round;  // items of a head in a round
    if (hks % kNumXcd == 0) {  // an XCD takes its heads one after another
      const int local = id / kNumXcd, turn = local / per_head;
      hk = turn * kNumXcd + id % kNumXcd;
      i = local - turn * per_head;
      round = kCus;
    } else {  // all heads at once
      i = fhk.div(id);
      hk = id - i * hks;
      round = max(kCus * kNumXcd / hks, 1);
    }
    const int row = i / round, n = min(per_head - row * round, round);
    at = (row & 1) && (int)gridDim.x <= 6 * kCus * kNumXcd ? row * round + n - 1 - (i - row * round) : i;
  }
};

// f over the wave, of values that are not negative, in every lane.
template <class F>
__device__ __forceinline__ int over_wave(int v, F&& f) {
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true));  // row_shr 1, 2, 4, 8
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true));
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true));
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true));
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, true));  // row_bcast 15, 31
  v = f(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, true));
  return __builtin_amdgcn_readlane(v, kWave - 1);
}

// The r-th block of columns of up to 64 sequences, those that see most rows
// first, whatever their sequence: block b of a sequence whose first token is
// row0 has level row0 / (tokens of a block) + b + 1. seq < 0: there are no more.
template <bool PACKED>
struct Ranked {
  int seq, block;
  __device__ __forceinline__ Ranked(int r, int batch, int cols, const PagedParams& p) {
    const int lane = (int)(threadIdx.x & (kWave - 1));
    int c = 0, top = 0;  // blocks of the lane's sequence, the level of its last
    if (lane < batch) {
      Sequence x;
      x.set<PACKED>(p, lane);
      if (x.seq >= 0) {
        c = (x.cols + cols - 1) / cols;
        top = (int)min((int64_t)max(x.row0, 0) * p.group / cols, (int64_t)1 << 29) + c;
      }
    }
    // blocks of level l and more
    auto from = [&](int l) { return over_wave(min(max(top - l + 1, 0), c), [](int a, int b) { return a + b; }); };
    seq = -1;
    block = 0;
    if (from(1) <= r) return;
    int lo = 1, hi = over_wave(top, [](int a, int b) { return max(a, b); }) + 1;  // from(lo) > r >= from(hi)
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (from(mid) > r)
        lo = mid;
      else
        hi = mid;
    }
    uint64_t have = __builtin_amdgcn_ballot_w64(top >= lo && top - c < lo);
    for (int i = r - from(lo + 1); i > 0; --i) have &= have - 1;
    seq = __builtin_ctzll(have);
    block = lo - 1 - __builtin_amdgcn_readlane(top - c, seq);
  }
};

// Whether a launch deals its blocks so: it fills the chip (else all are resident
// at once), and blocks of several sequences differ in weight, without a window.
// In the order of the sequences the heavy blocks of the last begin last: four of
// 2,048 tokens, 16 heads of 128, 71 us, ranked 61.
__device__ __forceinline__ bool ranked(const PagedParams& p, int groups) {
  return p.batch > 1 && p.batch <= kWave && groups >= 512 && p.window == INT32_MAX;
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

// Where the rows of K and V are: pages in the rows' type, pages of 8 bits, or
// packed rows in the order of the tokens.
enum Source { kPages, kPages8, kPacked };

// Factor of a scale byte, 2^(byte - 127) for bytes of 1 .. 254, and of the row
// whose byte lies in a word of four rows'.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }
__device__ __forceinline__ float scale_in(uint32_t word, int row) {
  return scale_of(__builtin_amdgcn_ubfe(word, (row & 3) * 8, 8));
}

// Two neighbouring e4m3 values, the lower or the upper half of a word, times a
// power of two: exact in bf16 and in fp32 (scale bytes of 3 to 246).
template <bool UPPER>
__device__ __forceinline__ uint32_t bf16_pair_of(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, UPPER));
}

// The prompts' kernel (bf16): out and lse, or with slices > 1 partial results
// for the join.
void launch_prompt(const PagedParams& p, int d, Source from, int64_t groups, hipStream_t s);

}  // namespace pf
