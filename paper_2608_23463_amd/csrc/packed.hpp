// Attention over whole sequences that lie one after another ("packed"), in
// training: what its forward and backward kernels share.
#pragma once

#include "attention.hpp"
#include "paged.hpp"

namespace pf {

// A call's parameters as the kernels take them.
PagedParams packed_params(const HeadsDims& d, const PackedCall& c);

// The gradients' part of a call. PagedParams holds the rest (no pages: a
// sequence's tokens are its rows).
struct PackedGrads {
  const char* dout;
  int64_t do_ts, do_hs;
  char* dq;
  char* dk;
  char* dv;
  int64_t dq_ts, dq_hs, dk_ts, dk_hs, dv_ts, dv_hs;
  float2* stats;      // [hq, stat_rows]: log-sum in exp2 units, rowsum(dO * O)
  int64_t stat_rows;
  float scale;
  int key_blocks;     // of a K/V head
  // the queries of a block of keys are cut into at most `slices` runs of at
  // least min_tiles tiles, whose sums are joined
  int slices;
  FastDiv fslices, fmin_tiles;
  float* part;
};

// A sequence's statistics begin at a multiple of four, so tiles of them load in
// 16-byte pieces: its place goes by its first token and its number.
__host__ __device__ __forceinline__ int64_t stat_row(int first, int seq) { return ((int64_t)(first >> 2) + seq) * 4; }

// A tile of rows in LDS that is read by rows (operands over channels) and by
// channels (operands over rows), so its 16-byte chunks are swizzled for both.
// By rows 16 consecutive rows of one chunk fall into different slots of 256
// bytes; by channels, in bf16, so do 4 rows of 4 chunks.
template <typename T, int D>
struct BothWays {
  static constexpr int RB = D * (int)sizeof(T), CH = RB / 16;
  typedef typename Mma<T>::frag frag;
  static __device__ __forceinline__ int swz(int r, int c) {
    if constexpr (sizeof(T) == 4) return c ^ (r & 15);
    if constexpr (CH == 16) return c ^ ((r & 3) << 2 | ((r >> 2) & 3));
    return c ^ (((r >> 1) & 1) << 2 | ((r >> 2) & 3));
  }
  // Reads go by a lane's base offset, formed once: the swizzles of the steps are
  // exclusive ors with constants, as a row's bytes are a power of two.
  // Rows: lane % 32 of the tile, channels 16 kk + 8 (lane / 32) ..
  static __device__ __forceinline__ uint32_t row_base(int lane) {
    const int r = lane & 31, g = lane >> 5;
    return (uint32_t)(r * RB + swz(r, sizeof(T) == 2 ? g : 2 * g) * 16);
  }
  static __device__ __forceinline__ frag row(const char* t, uint32_t base, int kk) {
    if constexpr (sizeof(T) == 2) {
      return *reinterpret_cast<const bf16x8*>(t + (base ^ (uint32_t)(kk * 32)));
    } else {
      const f32x4 a = *reinterpret_cast<const f32x4*>(t + (base ^ (uint32_t)(kk * 64)));
      const f32x4 b = *reinterpret_cast<const f32x4*>(t + (base ^ (uint32_t)(kk * 64 + 16)));
      frag f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[e] = a[e];
        f[e + 4] = b[e];
      }
      return f;
    }
  }
  // Channels: 32 cb + lane % 32, rows 16 s + 4 (lane / 32) + {0..3, 8..11}, the
  // order in which a 32x32 result holds its rows. In bf16 lane i of 16 addresses
  // row i / 4 at channels 4 (i % 4) .. + 3 of the group's 16.
  static __device__ __forceinline__ uint32_t col_base(int lane) {
    const int g = lane >> 5;
    if constexpr (sizeof(T) == 2) {
      const int r = g * 4 + ((lane & 15) >> 2), ch = (lane & 16) + 4 * (lane & 3);
      return (uint32_t)(r * RB + swz(r, ch / 8) * 16 + ((ch / 4) & 1) * 8);
    } else {
      return (uint32_t)(g * 4 * RB + (((lane & 31) / 4) ^ (g * 4)) * 16 + (lane & 3) * 4);
    }
  }
  static __device__ __forceinline__ frag col(const char* t, uint32_t base, int s, int cb) {
    frag f;
    if constexpr (sizeof(T) == 2) {
      const char* u = t + s * 16 * RB;
      const auto a = __builtin_bit_cast(bf16x4, lds_read_tr16(u + (base ^ (uint32_t)(cb * 64))));
      const auto b = __builtin_bit_cast(bf16x4, lds_read_tr16(u + 8 * RB + (base ^ (uint32_t)(cb * 64 + 32))));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[e] = a[e];
        f[e + 4] = b[e];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = (i / 4) * 8 + i % 4;
        f[i] = *reinterpret_cast<const float*>(t + (s * 16 + r) * RB + (base ^ (uint32_t)(((cb * 8) ^ r) * 16)));
      }
    }
    return f;
  }
  // the other operand, of rows 16 s .. + 15 of a result
  static __device__ __forceinline__ frag operand(const f32x16& x, int s) {
    if constexpr (sizeof(T) == 2) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(x[s * 8 + 2 * i], x[s * 8 + 2 * i + 1]);
      return __builtin_bit_cast(bf16x8, w);
    } else {
      frag f;
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = x[s * 8 + i];
      return f;
    }
  }
  // Wave `wave`'s share of the loads of rows j0 .. j0 + ROWS - 1 of a tensor
  // whose row 0 is at `base`, strides in bytes; rows past `last` land as zeros,
  // and so do those up to `before` from `sinks` on.
  template <int ROWS>
  static __device__ __forceinline__ void load(const char* base, int64_t stride, int j0, int last, char* tile, int wave,
                                              int lane, int before = -1, int sinks = 0) {
    constexpr int kPer = ROWS * RB / 4096, kRows = 1024 / RB;
    static_assert(kPer >= 1, "every wave loads");
    const rsrc_t rs = make_rsrc_uniform(base + (int64_t)j0 * stride, kOOB - 1);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = wave * kPer + j, r = i * kRows + lane / CH;
      uint32_t off = (uint32_t)(r * (int)stride + swz(r, lane % CH) * 16);
      if (j0 + r > last || (j0 + r <= before && j0 + r >= sinks)) off = kOOB;
      buf_ld16_lds(rs, off, tile + i * 1024);
    }
  }
};

// Steps 0 .. N - 1 of a chain of matrix instructions, the operands of the next
// one on their way from LDS while one runs (left alone, the compiler reads each
// pair of operands where it is used and waits there).
template <int N, class Load, class Use>
__device__ __forceinline__ void pipelined(Load&& load, Use&& use) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i + 1 < N) load(i + 1, (i + 1) & 1);
    __builtin_amdgcn_sched_barrier(0);
    use(i, i & 1);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// The 128 columns (token, head of a K/V head's) of a workgroup: 32 per wave,
// one per lane pair.
constexpr int kPackedCols = 128;
struct Columns {
  bool any;       // whether the workgroup has columns
  Sequence sq;
  int hk, x0, cols;
  bool on;        // whether the lane has one
  int tok, head, row;
  __device__ __forceinline__ Columns(const PagedParams& p, int lane, int wave) {
    const int blocks = (int)gridDim.x / p.hk;
    const Item item(p.hk, p.fhk, blocks);
    hk = item.hk;
    // the columns that see most come first
    if (ranked(p, (int)gridDim.x)) {
      const Ranked<true> r(item.at, p.batch, kPackedCols, p);
      any = r.seq >= 0;
      sq.set<true>(p, any ? r.seq : 0);
      x0 = any ? r.block * kPackedCols : 0;
    } else {
      const int blk = blocks - 1 - item.at, s = sequence_of_block<kPackedCols>(p, blk);
      sq.set<true>(p, s);
      x0 = (blk - first_block<kPackedCols>(p, s)) * kPackedCols;
      any = sq.seq >= 0 && x0 >= 0 && x0 < sq.cols;
    }
    cols = any ? min(sq.cols - x0, kPackedCols) : 0;
    const int mine = wave * 32 + (lane & 31);
    on = mine < cols;
    const int x = on ? x0 + mine : any ? x0 : 0;
    tok = p.fgroup.div(x);
    head = hk * p.group + x - tok * p.group;
    row = on ? tok : -1;
  }
};

}  // namespace pf
