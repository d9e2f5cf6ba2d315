// Attention of prompts in bf16 (the mathematics and the columns are those of
// paged_attention.hip; here a workgroup has 128 of them). Its rows come from
// bf16 pages, from pages of 8 bits, or from the tokens' own rows (whole sequences
// in training). 8 bits take 20 to 25 per cent longer (five prompts of up to 1,800
// tokens behind up to 6,000 rows, 32 over 8 heads of 128, 389 us, 321 from bf16
// pages): their rows pass through registers and LDS stores.
//
// Bound by the matrix cores and the exponentials: 4 D flops per (column, row)
// that is seen. 128 columns per workgroup, 32 per wave; tiles of 64 rows of K
// and V land in two LDS stages by direct loads, 16 rows per wave (a page is a
// multiple of 16 rows, so a wave's rows lie in one page), in the chunk orders
// that the fragment reads want (lds_swz, vtr_swz). A wave forms
// S^T = K Q^T, so a lane holds one column and half of its scores, then
// O^T += V^T P^T: the score registers hold rows 4 g + {0..3, 8..11} of each 16,
// and the transposed reads of V take the rows in that same order, so P never
// leaves its registers. Q is not scaled beforehand (its bf16 would round):
// the scale is part of the one multiply-add in front of each exponential. Waves
// in their matrix phases go before those in their exponentials (8,192 tokens, 32
// over 8 heads of 128, 531 us, without it 551; packed 558 and 592).
//
// The weights are rounded to bf16 once: 2^-8 of each at most, independent of
// one another. With many rows that is as much as the rounding of the result, so
// the error is 1.4 times that of the rounded exact result (0.0022 to 0.0023 of
// it, and 0.0017). The two terms of the single-token kernel would bring it back to
// 0.0017 and add half again to the matrix work that bounds this one: 8,192
// tokens, 32 over 8 heads of 128, 693 us for 523, six prompts with a window of
// 700, 16 heads of 64, 51 for 44. A caller who wants them lays the call out for
// fewer tokens. The weights' sum is taken unrounded, in fp32.
#include "attention.hpp"
#include "paged.hpp"

namespace pf {

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;
constexpr int kColumns = 128;

// Three workgroups per CU at 64 channels (16 heads: six windowed prompts 41 us,
// with two 53, four of 4,096 tokens behind 16,384 rows 1,382 and 1,462; one of
// 8,192 tokens 179 and 196; 20 windowed sequences in training 113 and 134), two at
// 128, whose accumulators take the registers of a third.
template <int D, Source FROM>
__global__ void __launch_bounds__(kThreads, D == 64 ? 3 : 2) paged_prompt_kernel(PagedParams p) {
  constexpr int RB = D * 2, CH = RB / 16;     // bytes and 16-byte chunks of a row
  constexpr int kTileBytes = kTile * RB, kStage = 2 * kTileBytes;
  constexpr int kLoads = kBlock * RB / 1024;  // 1 KB loads of a wave's 16 rows
  constexpr int kRowsPerLoad = 1024 / RB;
  constexpr int kPerTile = kTile / kBlock, kAhead = kWave / kPerTile;
  __shared__ __attribute__((aligned(1024))) char smem[2 * kStage];

  // the blocks that see most rows come first
  const int total = (int)gridDim.x, blocks = p.fslices.div(total) / p.hk;
  const Item item(p.hk, p.fhk, blocks * p.slices);
  const int hk = item.hk, rank = p.fslices.div(item.at), slice = item.at - rank * p.slices;
  Sequence sq;
  int s, x0;
  if (ranked(p, total)) {
    const Ranked<FROM == kPacked> r(rank, p.batch, kColumns, p);
    if (r.seq < 0) return;
    s = r.seq;
    sq.set<FROM == kPacked>(p, s);
    x0 = r.block * kColumns;
  } else {
    const int blk = blocks - 1 - rank;
    s = sequence_of_block<kColumns>(p, blk);
    sq.set<FROM == kPacked>(p, s);
    x0 = (blk - first_block<kColumns>(p, s)) * kColumns;
    if (sq.seq < 0 || x0 < 0 || x0 >= sq.cols) return;
  }
  const int cols = min(sq.cols - x0, kColumns);
  const Sight sight(p, sq, x0, cols, kTile);
  const int per = sight.per_slice(p);
  const int first = slice * per, ntiles = min(per, sight.tiles - first);
  if (ntiles <= 0 && p.slices > 1) return;  // no rows: the join does not read this slice

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 5, col = lane & 31;

  // the lane's column, and the rows lo < j <= row that it sees; those of the
  // wave's first and last column bound what the wave can skip
  const int xw = x0 + wave * 32, mine = wave * 32 + col;
  const bool on = mine < cols;
  const int xm = on ? x0 + mine : x0, tok = p.fgroup.div(xm), head = hk * p.group + xm - tok * p.group;
  const int row = on ? max(sq.row0 + tok, -1) : -1, lo = row - p.window;
  const int wcols = min(cols - wave * 32, 32);  // <= 0: an idle wave
  const int wfirst = sq.row0 + p.fgroup.div(wcols > 0 ? xw : x0);
  const int wtop = wcols > 0 ? sq.row0 + p.fgroup.div(xw + wcols - 1) : -1, wlast = min(wtop, sight.last);
  const int wlow = max(wfirst, 0) - p.window;  // rows up to it are before every window of the wave
  const int whigh = max(wtop, 0) - p.window;  // rows past it are inside every one

  bf16x8 qf[D / 16];
  {
    const bf16* qp = reinterpret_cast<const bf16*>(p.q) + (int64_t)(sq.t0 + tok) * p.q_ts + (int64_t)head * p.q_hs;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      u32x4 t = {0u, 0u, 0u, 0u};
      if (on) t = ld16(qp + kk * 16 + g * 8);
      qf[kk] = __builtin_bit_cast(bf16x8, t);
    }
  }

  constexpr bool kPaged = FROM != kPacked;
  const int32_t* table = p.table + (int64_t)s * p.max_pages;
  const int page_rows = p.hk * p.page_size;  // a cache has fewer than 2^31 rows
  auto tile_row = [&](int t) { return sight.tile(first + t) * kTile; };
  // First cache rows of the blocks of 16 tiles, a block per lane: -1 where the
  // sequence or the table has none. One vector load for 16 tiles, on its way
  // as long beforehand: scalar lookups per tile would make every wait for an
  // LDS read wait for them too (8,192 tokens, 32 over 8 heads of 128: 610 us with
  // them, 523 so).
  auto blocks_of = [&](int t) -> int {
    const int tl = t + lane / kPerTile;
    const int blk16 = tile_row(min(tl, ntiles - 1)) / kBlock + lane % kPerTile;
    const int pg = p.page_blocks.div(blk16);
    const int id = table[min(pg, p.max_pages - 1)];
    const bool have = blk16 * kBlock <= sight.last && (unsigned)id < (unsigned)p.n_pages;
    return have ? id * page_rows + hk * p.page_size + (blk16 - pg * p.page_blocks.d) * kBlock : -1;
  };
  // value rows that no column sees land as zeros: whether a tile has none
  auto all_seen = [&](int r0) {
    return r0 + kTile - 1 <= sight.first && (r0 > sight.top - p.window || r0 + kTile <= p.sinks);
  };
  auto unseen = [&](int j) { return j > sight.last || (j <= sight.first - p.window && j >= p.sinks); };
  // Packed rows: starts the loads of a tile. Rows past the last that is seen
  // may be another sequence's or past the tensor's end.
  auto issue_packed = [&](int t, int stage) {
    const int r0 = tile_row(t), j0 = r0 + wave * kBlock;
    const bool all = all_seen(r0);
    const rsrc_t rk = make_rsrc_uniform(p.k + ((int64_t)(sq.t0 + j0) * p.k_ts + hk * p.k_hs) * 2, kOOB - 1);
    const rsrc_t rv = make_rsrc_uniform(p.v + ((int64_t)(sq.t0 + j0) * p.v_ts + hk * p.v_hs) * 2, kOOB - 1);
    char* st = smem + stage * kStage + wave * kBlock * RB;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int r = j * kRowsPerLoad + lane / CH, c = lane % CH;
      uint32_t off = (uint32_t)(r * (int)p.k_ts * 2 + lds_swz<CH>(wave * kBlock + r, c) * 16);
      if (!all && j0 + r > sight.last) off = kOOB;
      buf_ld16_lds(rk, off, st + j * 1024);
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int r = j * kRowsPerLoad + lane / CH, c = lane % CH;
      uint32_t off = (uint32_t)(r * (int)p.v_ts * 2 + vtr_swz<CH>(wave * kBlock + r, c) * 16);
      if (!all && unseen(j0 + r)) off = kOOB;
      buf_ld16_lds(rv, off, st + kTileBytes + j * 1024);
    }
  };
  // Pages of 8 bits: a tile's rows come into registers, 16 values per lane and
  // load, and are widened on their way to LDS, where the values are those of a
  // bf16 cache (a power of two times e4m3 is exact in bf16).
  constexpr int C8 = D / 16, kLoads8 = kBlock * C8 / kWave, kRows8 = kWave / C8;
  u32x4 raw_k[kLoads8], raw_v[kLoads8];
  uint32_t word_k[kLoads8], word_v[kLoads8];  // with the row's scale byte (a loaded byte would be waited for to be widened)
  auto fetch8 = [&](int t, int rows, int at) {
    const int r0 = tile_row(t);
    const int mine16 = __builtin_amdgcn_readlane(rows, at + wave);
    const bool all = all_seen(r0);
    const int64_t row = mine16 < 0 ? 0 : mine16;
    const uint32_t n = mine16 < 0 ? 0 : kBlock;
    const rsrc_t rk = make_rsrc_uniform(p.k + row * D, n * D), rv = make_rsrc_uniform(p.v + row * D, n * D);
    const rsrc_t sk = make_rsrc_uniform(p.k_scale + row, n), sv = make_rsrc_uniform(p.v_scale + row, n);
#pragma unroll
    for (int j = 0; j < kLoads8; ++j) {
      const int r = j * kRows8 + lane / C8, c = lane % C8;
      const bool none = !all && unseen(r0 + wave * kBlock + r);
      raw_k[j] = buf_ld16(rk, (uint32_t)(r * D + c * 16));
      raw_v[j] = buf_ld16(rv, none ? kOOB : (uint32_t)(r * D + c * 16));
      word_k[j] = __builtin_amdgcn_raw_buffer_load_b32(sk, r & ~3, 0, 0);
      word_v[j] = __builtin_amdgcn_raw_buffer_load_b32(sv, none ? kOOB : (uint32_t)(r & ~3), 0, 0);
    }
  };
  auto put8 = [&](int stage) {
    char* st = smem + stage * kStage;
#pragma unroll
    for (int j = 0; j < kLoads8; ++j) {
      const int r = wave * kBlock + j * kRows8 + lane / C8, c = lane % C8;
      const float fk = scale_in(word_k[j], r), fv = scale_in(word_v[j], r);
      u32x4 k[2], v[2];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        k[i / 2][i % 2 * 2] = bf16_pair_of<false>(raw_k[j][i], fk);
        k[i / 2][i % 2 * 2 + 1] = bf16_pair_of<true>(raw_k[j][i], fk);
        v[i / 2][i % 2 * 2] = bf16_pair_of<false>(raw_v[j][i], fv);
        v[i / 2][i % 2 * 2 + 1] = bf16_pair_of<true>(raw_v[j][i], fv);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        *reinterpret_cast<u32x4*>(st + r * RB + lds_swz<CH>(r, 2 * c + h) * 16) = k[h];
        *reinterpret_cast<u32x4*>(st + kTileBytes + r * RB + vtr_swz<CH>(r, 2 * c + h) * 16) = v[h];
      }
    }
  };
  // Starts the loads of a tile whose blocks are `rows`' from lane `at` on.
  auto issue = [&](int t, int stage, int rows, int at) {
    const int r0 = tile_row(t);
    const int mine16 = __builtin_amdgcn_readlane(rows, at + wave);
    // a block without a page lands as zeros too
    const bool all = all_seen(r0);
    const uint32_t bytes = mine16 < 0 ? 0 : kBlock * RB;
    const int64_t base = mine16 < 0 ? 0 : (int64_t)mine16 * RB;
    const rsrc_t rk = make_rsrc_uniform(p.k + base, bytes), rv = make_rsrc_uniform(p.v + base, bytes);
    char* st = smem + stage * kStage + wave * kBlock * RB;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int r = j * kRowsPerLoad + lane / CH, c = lane % CH;
      buf_ld16_lds(rk, (uint32_t)(r * RB + lds_swz<CH>(wave * kBlock + r, c) * 16), st + j * 1024);
    }
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int r = j * kRowsPerLoad + lane / CH, c = lane % CH;
      uint32_t off = (uint32_t)(r * RB + vtr_swz<CH>(wave * kBlock + r, c) * 16);
      if (!all && unseen(r0 + wave * kBlock + r)) off = kOOB;
      buf_ld16_lds(rv, off, st + kTileBytes + j * 1024);
    }
  };

  f32x16 o[D / 32];
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[cb][r] = 0.0f;
  // Scores in exp2 units against a reference: a real maximum of the lane
  // pair's first tile with a visible row, kept while the running sums stay
  // below 2^32, then raised: weights and sums of values of up to 2^80 are far
  // from fp32's end, also where 512 slices are joined, and a reference that is
  // near the maximum (the rows of a long cache add 2^10 to 2^20) stays.
  float mref = -INFINITY, lrun = 0.0f;
  bool have_ref = false;  // wave-uniform
  constexpr float kSumLimit = 4294967296.0f;  // 2^32

  int rows = -1, rows_next = -1;  // of 16 tiles, and of the 16 behind them
  if (ntiles > 0) {
    if constexpr (kPaged) {
      rows = blocks_of(0);
      rows_next = blocks_of(kAhead);
    }
    if constexpr (FROM == kPages) issue(0, 0, rows, 0);
    if constexpr (FROM == kPacked) issue_packed(0, 0);
    if constexpr (FROM == kPages8) {
      fetch8(0, rows, 0);
      put8(0);
    }
  }
  if constexpr (FROM == kPages8) {
    // the queries and table entries are there too, whatever the way here: else the
    // loop would wait for them, and with them for the rows on their way
    wait_vmcnt<0>();
    if (ntiles > 1) fetch8(1, rows, kPerTile);
  }
  for (int t = 0; t < ntiles; ++t) {
    const int r0 = tile_row(t), in = t % kAhead;
    if constexpr (FROM != kPages8) wait_vmcnt<0>();
    lds_barrier();  // tile t landed for all; every wave is done with tile t - 1
    const int gone =
        kPaged ? (int)(__builtin_amdgcn_ballot_w64(rows < 0) >> (in * kPerTile)) & ((1 << kPerTile) - 1) : 0;
    if (kPaged && in == kAhead - 1) {
      rows = rows_next;
      if (t + 1 + kAhead < ntiles) rows_next = blocks_of(t + 1 + kAhead);
    }
    if constexpr (FROM == kPages) {
      if (t + 1 < ntiles) issue(t + 1, (t + 1) & 1, rows, (t + 1) % kAhead * kPerTile);
    } else if constexpr (FROM == kPacked) {
      if (t + 1 < ntiles) issue_packed(t + 1, (t + 1) & 1);
    } else {  // the next tile's registers to LDS, and the one behind it into them
      if (t + 1 < ntiles) put8((t + 1) & 1);
      if (t + 2 < ntiles) fetch8(t + 2, in == kAhead - 2 ? rows_next : rows, (t + 2) % kAhead * kPerTile);
    }
    const char* sk = smem + (t & 1) * kStage;
    const char* sv = sk + kTileBytes;
    if (r0 > wlast || (r0 + kTile - 1 <= wlow && r0 >= p.sinks)) continue;  // wave-uniform: nothing it sees
    const bool whole = gone == 0 && r0 + kTile - 1 <= wfirst && (r0 > whigh || r0 + kTile <= p.sinks);
    f32x16 sc[2];
    auto scores = [&]() {
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[kb][r] = 0.0f;
        const int kr = kb * 32 + col;
        const char* krow = sk + kr * RB;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          sc[kb] = Mma<bf16>::mma(*reinterpret_cast<const bf16x8*>(krow + lds_swz<CH>(kr, kk * 2 + g) * 16), qf[kk], sc[kb]);
      }
      __builtin_amdgcn_s_setprio(0);
    };
    // V^T of rows 4 g + {0..3} and 8 + 4 g + {0..3} of 16, the order of the
    // scores. Lane i of a 16-lane group addresses row i / 4 at channels
    // 4 (i % 4) .. + 3 of the group's 16.
    auto values = [&](int kb, int s2, int cb) {
      const int k1 = kb * 32 + s2 * 16 + g * 4 + ((lane & 15) >> 2), ch = cb * 32 + (lane & 16) + 4 * (lane & 3);
      auto addr = [&](int key) { return sv + key * RB + vtr_swz<CH>(key, ch / 8) * 16 + ((ch / 4) & 1) * 8; };
      const auto a = __builtin_bit_cast(bf16x4, lds_read_tr16(addr(k1)));
      const auto b = __builtin_bit_cast(bf16x4, lds_read_tr16(addr(k1 + 8)));
      bf16x8 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[e] = a[e];
        v[e + 4] = b[e];
      }
      return v;
    };
    // scores scaled against `ref`; what is not seen counts for nothing
    auto against = [&](float ref) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[kb][r] = fmaf(sc[kb][r], p.scale_log2, -ref);
      if (whole) return;
      if (gone == 0 && r0 >= p.sinks) {  // the window's edges alone: one unsigned comparison
        const int past = row - r0;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if ((unsigned)(past - (kb * 32 + acc_row(r, lane))) >= (unsigned)p.window) sc[kb][r] = -INFINITY;
        return;
      }
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int in = kb * 32 + acc_row(r, lane), j = r0 + in;
          const bool seen = j <= row && (j > lo || j < p.sinks) && !((gone >> (in / kBlock)) & 1);
          if (!seen) sc[kb][r] = -INFINITY;
        }
    };
    auto exponentiate = [&]() {
      float ls[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = fast_exp2(sc[kb][r]);
          sc[kb][r] = e;
          ls[r & 3] += e;
        }
      return (ls[0] + ls[1]) + (ls[2] + ls[3]);
    };
    float tsum = 0.0f;
    bool redo = !have_ref;
    // of the first 16 rows, read while the exponentials are taken (rows of 8 bits on
    // their way take these registers)
    constexpr bool kEarly = FROM != kPages8;
    bf16x8 early[kEarly ? D / 32 : 1];
    auto products = [&]() {
      scores();
      if constexpr (kEarly)
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb) early[cb] = values(0, 0, cb);
    };
    if (have_ref && whole) {  // one run of instructions: products, reads and exponentials side by side
      products();
      float ls[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = fast_exp2(fmaf(sc[kb][r], p.scale_log2, -mref));
          sc[kb][r] = e;
          ls[r & 3] += e;
        }
      tsum = (ls[0] + ls[1]) + (ls[2] + ls[3]);
      redo = __builtin_amdgcn_ballot_w64(!(lrun + tsum <= kSumLimit)) != 0;
    } else if (have_ref) {
      products();
      against(mref);
      tsum = exponentiate();
      redo = __builtin_amdgcn_ballot_w64(!(lrun + tsum <= kSumLimit)) != 0;
    }
    if (redo) {  // wave-uniform: the first tile, a sum past the limit, or a lane's first row
      products();
      against(0.0f);
      float mt = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) mt = fmaxf(mt, sc[kb][r]);
      mt = fmaxf(mt, other_half(mt));
      const float ltot = lrun + other_half(lrun);
      const float mnew = fmaxf(mt, mref + fmaxf(0.0f, __log2f(ltot)));
      // nothing is accumulated while a lane has no reference
      const float a = mref == -INFINITY ? 0.0f : fast_exp2(mref - mnew);
      lrun *= a;
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[cb][r] *= a;
      mref = mnew;
      have_ref = true;
      const float ref = mnew == -INFINITY ? 0.0f : mnew;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[kb][r] -= ref;
      tsum = exponentiate();
    }
    lrun += tsum;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(sc[kb][s2 * 8 + 2 * i], sc[kb][s2 * 8 + 2 * i + 1]);
        const bf16x8 pb = __builtin_bit_cast(bf16x8, w);
#pragma unroll
        for (int cb = 0; cb < D / 32; ++cb)
          o[cb] = Mma<bf16>::mma(kEarly && kb == 0 && s2 == 0 ? early[kEarly ? cb : 0] : values(kb, s2, cb), pb, o[cb]);
      }
    __builtin_amdgcn_s_setprio(0);
  }

  const float l = lrun + other_half(lrun);
  if (!on) return;
  const int64_t orow = (int64_t)(sq.t0 + tok) * p.hq + head;
  const bool whole_row = p.slices == 1;
  const float f = !whole_row ? 1.0f : l > 0.0f ? 1.0f / l : l;  // nothing seen: zero (and a NaN stays one)
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const float v[4] = {o[cb][r] * f, o[cb][r + 1] * f, o[cb][r + 2] * f, o[cb][r + 3] * f};
      const int c = cb * 32 + acc_row(r, lane);
      if (whole_row)
        store4(static_cast<bf16*>(p.out) + orow * D + c, v);
      else
        store4(p.part_o + (orow * p.slices + slice) * D + c, v);
    }
  if (g != 0) return;
  if (!whole_row)
    p.part_ml[orow * p.slices + slice] = make_float2(mref, l);
  else if (p.lse)
    p.lse[orow] = (mref + __log2f(l)) * 0.69314718055994530942f;
}

}  // namespace

void launch_prompt(const PagedParams& p, int d, Source from, int64_t groups, hipStream_t s) {
  const dim3 grid((unsigned)(groups * p.slices));
  if (from == kPacked)
    d == 64 ? paged_prompt_kernel<64, kPacked><<<grid, kThreads, 0, s>>>(p)
            : paged_prompt_kernel<128, kPacked><<<grid, kThreads, 0, s>>>(p);
  else if (from == kPages8)
    d == 64 ? paged_prompt_kernel<64, kPages8><<<grid, kThreads, 0, s>>>(p)
            : paged_prompt_kernel<128, kPages8><<<grid, kThreads, 0, s>>>(p);
  else
    d == 64 ? paged_prompt_kernel<64, kPages><<<grid, kThreads, 0, s>>>(p)
            : paged_prompt_kernel<128, kPages><<<grid, kThreads, 0, s>>>(p);
}

}  // namespace pf
