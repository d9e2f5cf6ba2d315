// Gradients of causal attention over whole sequences that lie one after
// another.
//
//   p_ij = exp(scale q_i.k_j - lse_i) where i sees j, D_i = dO_i.O_i
//   dV_j = sum_i p_ij dO_i,  dS_ij = p_ij (dO_i.v_j - D_i)
//   dQ_i = scale sum_j dS_ij k_j,  dK_j = scale sum_i dS_ij q_i
// over the query heads of a K/V head too in dK and dV. The probabilities are
// formed again from the forward's log-sums. Two kernels and a join, no atomics:
// every gradient is written once, in the same order of additions in every run.
//  - packed_dq_kernel: 128 columns (token, head), 32 per wave; the tiles of keys
//    that they see. It forms D_i and leaves it, and lse_i, heads first.
//  - packed_dkdv_kernel: 128 keys of a K/V head, 32 per wave, one per lane
//    pair; the 32-query tiles that see them, head after head.
// A tile lies in LDS once, by rows; the products over channels read it by rows,
// those over positions by channels (in bf16 through transposing reads), so P
// and dS are operands in the registers where they were computed. In bf16 both
// are rounded to it, 2^-8 of each at most; sums are fp32.
//
// Bound by the matrix cores in bf16 at 128 channels, seven products for five (dQ's
// kernel forms scores and dP once more): 8 documents of up to 4,096 tokens, 32 over 8
// heads, 1,280 us, 880 TFLOP/s; by the exponentials too at 64 (8,192 tokens, 16
// heads, 586 us); small calls by the latency of three launches.
#include <algorithm>

#include "packed.hpp"
#include "trace.hpp"

namespace pf {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kKeys = 128;  // of a workgroup of dK and dV
constexpr int kQueries = 32;

template <typename T, int D>
__device__ __forceinline__ void store_rows(T* out, const f32x16 (&acc)[D / 32], float f, int lane) {
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const float x[4] = {acc[cb][r] * f, acc[cb][r + 1] * f, acc[cb][r + 2] * f, acc[cb][r + 3] * f};
      store4(out + cb * 32 + acc_row(r, lane), x);
    }
}

// The keys of a workgroup, and its run of the (head, tile of queries) list.
struct KeyBlock {
  bool any;
  Sequence sq;
  int hk, blk, s, n, k0;
  int last;        // the last query that sees one of the keys
  int tiles;       // of the queries up to it, per head
  int run, first;  // tiles of a slice, the first of this one
  int live;        // slices that have any
  // `slice`: the workgroup's, of z.slices
  __device__ __forceinline__ KeyBlock(const PagedParams& p, const PackedGrads& z, int hk_, int blk_, int slice)
      : hk(hk_), blk(blk_) {
    s = find_run(p.batch, [&](int c) { return p.cu[c] / kKeys + c; }, blk);
    sq.set<true>(p, s);
    n = sq.seq < 0 ? 0 : p.fgroup.div(sq.cols);
    k0 = (blk - (p.cu[s] / kKeys + s)) * kKeys;
    any = k0 >= 0 && k0 < n;
    if (!any) return;
    // the queries that see a key of the block: from its first key on, up to the
    // end of its last key's windows, or to the sequence's end for the first rows
    const int64_t reach = k0 < p.sinks ? n : min((int64_t)n, (int64_t)k0 + kKeys - 1 + p.window);
    last = (int)reach - 1;
    tiles = (last - k0) / kQueries + 1;
    const int all = tiles * p.group, cut = max(min(z.fmin_tiles.div(all), z.slices), 1);
    run = (all + cut - 1) / cut;
    live = (all + run - 1) / run;
    first = slice * run;
    run = min(run, all - first);
  }
};

// Where a lane's 4 D / 32 quads of a partial dK (which = 0) or dV lie.
template <int D>
__device__ __forceinline__ f32x4* part_of(const PackedGrads& z, const KeyBlock& b, int slice, int which, int wave, int lane) {
  const int64_t unit = ((int64_t)b.hk * z.key_blocks + b.blk) * z.slices + slice;
  return reinterpret_cast<f32x4*>(z.part) + ((unit * 2 + which) * kWaves + wave) * (D / 8) * kWave + lane;
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? (D == 64 ? 3 : 2) : 1)
packed_dkdv_kernel(PagedParams p, PackedGrads z) {
  typedef BothWays<T, D> Tl;
  typedef Mma<T> MM;
  constexpr int kTileBytes = kQueries * Tl::RB, kStage = 2 * kTileBytes + 1024, es = (int)sizeof(T);
  constexpr bool kHold = sizeof(T) == 4 || D == 64;  // the values in registers; else in LDS
  // two stages of Q, dO and statistics, then the values (one array: the compiler
  // would wait for loads in flight to one before it reads the other)
  __shared__ __attribute__((aligned(1024))) char smem[2 * kStage + (kHold ? 0 : kWaves * kTileBytes)];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5, col = lane & 31;
  const uint32_t rb = Tl::row_base(lane), cb0 = Tl::col_base(lane);

  const Item item(p.hk, p.fhk, z.key_blocks * z.slices);
  const int blk = z.fslices.div(item.at), slice = item.at - blk * z.slices;
  const KeyBlock b(p, z, item.hk, blk, slice);
  if (!b.any || b.run <= 0) return;
  const Sequence& sq = b.sq;
  const int hk = b.hk, k0 = b.k0, n = b.n;
  const int key = k0 + wave * 32 + col;
  const bool on = key < n;

  typename MM::frag kf[D / 16], vf[kHold ? D / 16 : 1];
  {
    const int64_t tok = sq.t0 + (on ? key : k0);
    const T* kp = reinterpret_cast<const T*>(p.k) + tok * p.k_ts + (int64_t)hk * p.k_hs;
    const T* vp = reinterpret_cast<const T*>(p.v) + tok * p.v_ts + (int64_t)hk * p.v_hs;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      kf[kk] = MM::load(kp + kk * 16 + g * 8);
      if constexpr (kHold) vf[kk] = MM::load(vp + kk * 16 + g * 8);
    }
    if constexpr (!kHold)
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
        Tl::template load<kQueries>(p.v + (sq.t0 * p.v_ts + hk * p.v_hs) * es, p.v_ts * es, k0 + w * 32, n - 1, smem + 2 * kStage + w * kTileBytes, wave,
                                    lane);
  }
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) dk[cb][r] = dv[cb][r] = 0.0f;

  const int wk0 = k0 + wave * 32;
  int ih = b.first / b.tiles, it = b.first - ih * b.tiles, ct = it;  // head and tile of the loads, tile in turn
  auto issue = [&](int stage) {
    const int q0 = k0 + (b.tiles - 1 - it) * kQueries, h = hk * p.group + ih;
    char* st = smem + stage * kStage;
    Tl::template load<kQueries>(p.q + (sq.t0 * p.q_ts + h * p.q_hs) * es, p.q_ts * es, q0, b.last, st, wave, lane);
    Tl::template load<kQueries>(z.dout + (sq.t0 * z.do_ts + h * z.do_hs) * es, z.do_ts * es, q0, b.last, st + kTileBytes,
                                wave, lane);
    if (wave == 0) {
      const rsrc_t rs = make_rsrc_uniform(z.stats + h * z.stat_rows + stat_row(sq.t0, b.s) + q0, kQueries * 8);
      buf_ld16_lds(rs, lane < kQueries / 2 ? lane * 16 : kOOB, st + 2 * kTileBytes);
    }
    if (++it == b.tiles) {
      it = 0;
      ++ih;
    }
  };
  issue(0);
  for (int t = 0; t < b.run; ++t) {
    wait_vmcnt<0>();
    lds_barrier();
    if (t + 1 < b.run) issue((t + 1) & 1);
    const int q0 = k0 + (b.tiles - 1 - ct) * kQueries;
    ct = ct + 1 == b.tiles ? 0 : ct + 1;
    // wave-uniform: the wave has no keys, or nothing of the tile sees them
    if (wk0 >= n || q0 + kQueries - 1 < wk0 || (q0 - p.window >= wk0 + 31 && wk0 >= p.sinks)) continue;
    const char* sq_ = smem + (t & 1) * kStage;
    const char* so = sq_ + kTileBytes;
    const float* st = reinterpret_cast<const float*>(so + kTileBytes);
    f32x16 sc, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = dp[r] = 0.0f;
    typename MM::frag fa[2], fb[2], fv[2];
    auto rows_of = [&](int kk, int u) {
      fa[u] = Tl::row(sq_, rb, kk);
      fb[u] = Tl::row(so, rb, kk);
      if constexpr (!kHold) fv[u] = Tl::row(smem + 2 * kStage + wave * kTileBytes, rb, kk);
    };
    auto cols_of = [&](int i, int u) {
      fa[u] = Tl::col(so, cb0, i / (D / 32), i % (D / 32));
      fb[u] = Tl::col(sq_, cb0, i / (D / 32), i % (D / 32));
    };
    __builtin_amdgcn_s_setprio(1);
    rows_of(0, 0);
    pipelined<D / 16>(rows_of, [&](int kk, int u) {
      sc = MM::mma(fa[u], kf[kk], sc);
      dp = MM::mma(fb[u], kHold ? vf[kHold ? kk : 0] : fv[u], dp);
    });
    __builtin_amdgcn_s_setprio(0);
    cols_of(0, 0);
    const bool whole = q0 >= wk0 + 31 && q0 + kQueries <= n && (q0 + kQueries - 1 - p.window < wk0 || wk0 + 31 < p.sinks);
#pragma unroll
    for (int r4 = 0; r4 < 16; r4 += 4) {
      const int i0 = acc_row(r4, lane);
      const f32x4 a = *reinterpret_cast<const f32x4*>(st + 2 * i0), c = *reinterpret_cast<const f32x4*>(st + 2 * i0 + 4);
      const float ls[4] = {a[0], a[2], c[0], c[2]}, de[4] = {a[1], a[3], c[1], c[3]};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sc[r4 + e] = fast_exp2(fmaf(sc[r4 + e], p.scale_log2, -ls[e]));
        dp[r4 + e] = sc[r4 + e] * (dp[r4 + e] - de[e]);
      }
    }
    if (!whole) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int i = q0 + acc_row(r, lane);
        const bool sees = (key <= i) & (i < n) & ((key > i - p.window) | (key < p.sinks));
        sc[r] = sees ? sc[r] : 0.0f;
        dp[r] = sees ? dp[r] : 0.0f;
      }
    }
    const typename MM::frag pf[2] = {Tl::operand(sc, 0), Tl::operand(sc, 1)};
    const typename MM::frag df[2] = {Tl::operand(dp, 0), Tl::operand(dp, 1)};
    __builtin_amdgcn_s_setprio(1);
    pipelined<D / 16>(cols_of, [&](int i, int u) {
      const int s2 = i / (D / 32), cb = i % (D / 32);
      dv[cb] = MM::mma(fa[u], pf[s2], dv[cb]);
      dk[cb] = MM::mma(fb[u], df[s2], dk[cb]);
    });
    __builtin_amdgcn_s_setprio(0);
  }
  if (b.live > 1) {
    f32x4* to[2] = {part_of<D>(z, b, slice, 0, wave, lane), part_of<D>(z, b, slice, 1, wave, lane)};
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        to[0][(cb * 4 + r) * kWave] = f32x4{dk[cb][4 * r], dk[cb][4 * r + 1], dk[cb][4 * r + 2], dk[cb][4 * r + 3]};
        to[1][(cb * 4 + r) * kWave] = f32x4{dv[cb][4 * r], dv[cb][4 * r + 1], dv[cb][4 * r + 2], dv[cb][4 * r + 3]};
      }
    return;
  }
  if (!on) return;
  const int64_t tok = sq.t0 + key;
  store_rows<T, D>(reinterpret_cast<T*>(z.dk) + tok * z.dk_ts + (int64_t)hk * z.dk_hs, dk, z.scale, lane);
  store_rows<T, D>(reinterpret_cast<T*>(z.dv) + tok * z.dv_ts + (int64_t)hk * z.dv_hs, dv, 1.0f, lane);
}

// Joins the slices of a block of keys in their order: a workgroup per 32
// channels of dK (y even) or dV, its lanes as above.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) packed_join_kernel(PagedParams p, PackedGrads z) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int blk = p.fhk.div((int)blockIdx.x), hk = (int)blockIdx.x - blk * p.hk;
  const KeyBlock b(p, z, hk, blk, 0);
  if (!b.any || b.live < 2) return;
  const int which = blockIdx.y & 1, cb = blockIdx.y / 2, key = b.k0 + wave * 32 + (lane & 31);
  f32x4 x[4] = {};
  for (int s = 0; s < b.live; ++s) {
    const f32x4* from = part_of<D>(z, b, s, which, wave, lane);
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] += from[(cb * 4 + r) * kWave];
  }
  if (key >= b.n) return;
  const int64_t tok = b.sq.t0 + key;
  T* out = which ? reinterpret_cast<T*>(z.dv) + tok * z.dv_ts + (int64_t)hk * z.dv_hs
                 : reinterpret_cast<T*>(z.dk) + tok * z.dk_ts + (int64_t)hk * z.dk_hs;
  const float f = which ? 1.0f : z.scale;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const float y[4] = {x[r][0] * f, x[r][1] * f, x[r][2] * f, x[r][3] * f};
    store4(out + cb * 32 + acc_row(4 * r, lane), y);
  }
}

// In bf16 D_i comes from the rounded O, an error as large as the others in the
// scores' gradients where a query sees few keys. But these add up to zero over
// a query's keys, so what they add up to corrects D: for the kernel of dK and dV,
// which runs behind this one, and where a workgroup sees few tiles for dQ too, by a
// pass beforehand. dQ's error over that of the rounded exact result, and the time of
// the whole backward (8,192 tokens, 32 over 8 heads of 128), with that pass over up to
// 4 tiles, 2 and none: documents of 64 tokens 1.415 and 138 us, the same, 1.60 and 134;
// of 320 1.424 and 190 us, 1.427 and 182, 1.54 and 179; of 512 1.423 and 266 us, 1.426
// and 240, 1.52 and 240; windows of 200 1.426 and 208 us, 1.433 and 187, 1.46 and 189.
// Over up to 5 and 8 the errors are those of 4, 1.41 being the two roundings' own.
constexpr int kFewTiles = 4;

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? (D == 64 ? 3 : 2) : 1) packed_dq_kernel(PagedParams p, PackedGrads z) {
  constexpr bool kCorrect = sizeof(T) == 2;
  typedef BothWays<T, D> Tl;
  typedef Mma<T> MM;
  constexpr int kRows = sizeof(T) == 2 ? 64 : 32, kTileBytes = kRows * Tl::RB, es = (int)sizeof(T);
  __shared__ __attribute__((aligned(1024))) char smem[2][2 * kTileBytes];  // K, V
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5;
  const uint32_t rb = Tl::row_base(lane), cb0 = Tl::col_base(lane);
  const Columns c(p, lane, wave);
  if (!c.any) return;
  const Sight sight(p, c.sq, c.x0, c.cols, kRows);
  const int lo = c.row - p.window;
  const int wcols = min(c.cols - wave * 32, 32);  // <= 0: an idle wave
  const int wfirst = p.fgroup.div(c.x0 + wave * 32), wtop = wcols > 0 ? p.fgroup.div(c.x0 + wave * 32 + wcols - 1) : -1;

  typename MM::frag qf[D / 16], of[D / 16];
  float2* const stat = z.stats + c.head * z.stat_rows + stat_row(c.sq.t0, c.sq.seq) + c.tok;
  float2 st;
  {
    const int64_t tok = c.sq.t0 + c.tok;
    const T* qp = reinterpret_cast<const T*>(p.q) + tok * p.q_ts + (int64_t)c.head * p.q_hs;
    const T* op = reinterpret_cast<const T*>(z.dout) + tok * z.do_ts + (int64_t)c.head * z.do_hs;
    const int64_t orow = tok * p.hq + c.head;
    const T* outp = reinterpret_cast<const T*>(p.out) + orow * D;
    float d = 0.0f;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      qf[kk] = MM::load(qp + kk * 16 + g * 8);
      of[kk] = MM::load(op + kk * 16 + g * 8);
      const typename MM::frag o = MM::load(outp + kk * 16 + g * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) d = fmaf(to_f32(o[e]), to_f32(of[kk][e]), d);
    }
    st = make_float2(p.lse[orow] * 1.4426950408889634f, d + other_half(d));
  }
  const char* k = p.k + (c.sq.t0 * p.k_ts + c.hk * p.k_hs) * es;
  const char* v = p.v + (c.sq.t0 * p.v_ts + c.hk * p.v_hs) * es;
  auto tile_row = [&](int t) { return sight.tile(t < sight.tiles ? t : t - sight.tiles) * kRows; };
  auto issue = [&](int t) {
    const int r0 = tile_row(t);
    Tl::template load<kRows>(k, p.k_ts * es, r0, sight.last, smem[t & 1], wave, lane, sight.first - p.window, p.sinks);
    Tl::template load<kRows>(v, p.v_ts * es, r0, sight.last, smem[t & 1] + kTileBytes, wave, lane);
  };
  f32x16 dq[D / 32];
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[cb][r] = 0.0f;
  // once more over few tiles: the first pass only corrects D
  const int total = kCorrect && sight.tiles <= kFewTiles ? 2 * sight.tiles : sight.tiles;
  const int last_pass = total - sight.tiles;
  float slip = 0.0f;  // sum of the column's dS so far
  issue(0);
  for (int t = 0; t < total; ++t) {
    wait_vmcnt<0>();
    lds_barrier();
    if (t + 1 < total) issue(t + 1);
    if (kCorrect && t == last_pass && t > 0) {
      st.y += slip + other_half(slip);
      slip = 0.0f;
    }
    const char* sk = smem[t & 1];
    const char* sv = sk + kTileBytes;
#pragma unroll
    for (int kb = 0; kb < kRows / 32; ++kb) {
      const int r0 = tile_row(t) + kb * 32;
      if (r0 > wtop || (r0 + 31 <= wfirst - p.window && r0 >= p.sinks)) continue;  // wave-uniform
      f32x16 sc, dp;
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = dp[r] = 0.0f;
      typename MM::frag fa[2], fb[2];
      auto rows_of = [&](int kk, int u) {
        fa[u] = Tl::row(sk + kb * 32 * Tl::RB, rb, kk);
        fb[u] = Tl::row(sv + kb * 32 * Tl::RB, rb, kk);
      };
      auto cols_of = [&](int i, int u) { fa[u] = Tl::col(sk + kb * 32 * Tl::RB, cb0, i / (D / 32), i % (D / 32)); };
      __builtin_amdgcn_s_setprio(1);
      rows_of(0, 0);
      pipelined<D / 16>(rows_of, [&](int kk, int u) {
        sc = MM::mma(fa[u], qf[kk], sc);
        dp = MM::mma(fb[u], of[kk], dp);
      });
      __builtin_amdgcn_s_setprio(0);
      cols_of(0, 0);
      const bool whole = r0 + 31 <= wfirst && (r0 > wtop - p.window || r0 + 32 <= p.sinks);
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = fast_exp2(fmaf(sc[r], p.scale_log2, -st.x)) * (dp[r] - st.y);
      if (!whole) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int j = r0 + acc_row(r, lane);
          const bool sees = (j <= c.row) & ((j > lo) | (j < p.sinks));
          sc[r] = sees ? sc[r] : 0.0f;
        }
      }
      if (kCorrect) {
        float add[4] = {};
#pragma unroll
        for (int r = 0; r < 16; ++r) add[r & 3] += sc[r];
        slip += (add[0] + add[1]) + (add[2] + add[3]);
        if (t < last_pass) continue;
      }
      const typename MM::frag df[2] = {Tl::operand(sc, 0), Tl::operand(sc, 1)};
      __builtin_amdgcn_s_setprio(1);
      pipelined<D / 16>(cols_of, [&](int i, int u) {
        const int cb = i % (D / 32);
        dq[cb] = MM::mma(fa[u], df[i / (D / 32)], dq[cb]);
      });
      __builtin_amdgcn_s_setprio(0);
    }
  }
  slip += other_half(slip);
  if (!c.on) return;
  if (g == 0) *stat = make_float2(st.x, st.y + slip);
  store_rows<T, D>(reinterpret_cast<T*>(z.dq) + (c.sq.t0 + c.tok) * z.dq_ts + (int64_t)c.head * z.dq_hs, dq, z.scale, lane);
}

// How the queries of a block of keys are cut where the blocks do not fill the
// chip: four workgroups per CU, of 8 tiles at least, 4 where they are few (two of
// up to 200 tokens, 8 over 2 heads of 128, 32 us for 42; 2,048 tokens, 32 over 8 heads
// of 128, 169 us, 352 whole, 208 in half as many of 32; 8,192 tokens, 4 heads of 64,
// 241, 378 and 272), in fp32 two, of 2 (seven documents of up to 500 tokens, window
// 100, 8 over 2 heads of 64: 96 us in slices of 8, 80 of 2). From one round of
// workgroups on, two slices of long lists (8,192 tokens, 32 over 8 heads of 128, 1,908
// us, 2,064 whole). Of several rounds, cuts cost more in partial sums than they even
// out (8 documents of up to 4,096 tokens, 32 over 8 heads of 128, 1,000 blocks: 792 us
// whole, 810 in two slices, 787 in up to four, and 23 and 56 us of joins; 8,192 tokens,
// 16 heads of 64, 329 and 338, 348), and so does dealing them by weight over the
// documents (907 us: probably their queries are no longer shared in an L2).
struct KeyPlan {
  int64_t groups;  // blocks of all heads
  int slices, min_tiles;
};
KeyPlan key_plan(const HeadsDims& d, int64_t n_tokens, int batch, int64_t max_len, int64_t window, int64_t sinks) {
  KeyPlan k;
  k.groups = packed_key_groups(d, n_tokens, batch);
  int64_t reach = std::min(max_len, n_tokens);
  if (window > 0 && sinks == 0) reach = std::min(reach, kKeys + std::min<int64_t>(window, INT32_MAX));
  const int64_t most = (reach + kQueries - 1) / kQueries * (d.hq / d.hk);  // tiles of a block
  const bool wide = d.esize == 2;
  k.min_tiles = k.groups >= 512 ? 128 : !wide ? 2 : k.groups < 64 ? 4 : 8;
  const int64_t want = k.groups >= 768 ? 1 : k.groups >= 512 ? 2 : ((wide ? 1024 : 512) + k.groups - 1) / k.groups;
  k.slices = (int)std::max<int64_t>(1, std::min<int64_t>({want, most / k.min_tiles, 64}));
  return k;
}

int64_t stat_rows(int64_t n_tokens, int batch) { return (n_tokens + 3) / 4 * 4 + 4 * (int64_t)batch + kQueries; }
size_t stat_bytes(const HeadsDims& d, int64_t n_tokens, int batch) {
  return ((size_t)d.hq * stat_rows(n_tokens, batch) * sizeof(float2) + 255) / 256 * 256;
}

template <typename T, int D>
hipError_t backward_on(const HeadsDims& d, const PagedParams& p, const PackedGrads& z, hipStream_t s) {
  hipError_t e = timed("packed_dq", s, [&] {
    packed_dq_kernel<T, D><<<dim3((unsigned)packed_groups(d, p.n_tokens, p.batch)), kThreads, 0, s>>>(p, z);
  });
  if (e != hipSuccess) return e;
  e = timed("packed_dkdv", s, [&] {
    packed_dkdv_kernel<T, D><<<dim3((unsigned)(z.key_blocks * d.hk * z.slices)), kThreads, 0, s>>>(p, z);
  });
  if (e != hipSuccess || z.slices == 1) return e;
  return timed("packed_join", s, [&] {
    packed_join_kernel<T, D><<<dim3((unsigned)(z.key_blocks * d.hk), D / 16), kThreads, 0, s>>>(p, z);
  });
}

}  // namespace

int64_t packed_key_groups(const HeadsDims& d, int64_t n_tokens, int batch) {
  return (n_tokens / kKeys + batch) * d.hk;
}

size_t packed_backward_ws(const HeadsDims& d, int64_t n_tokens, int batch, int64_t max_len, int64_t window, int64_t sinks) {
  const KeyPlan k = key_plan(d, n_tokens, batch, max_len, window, sinks);
  const size_t part = k.slices == 1 ? 0 : (size_t)k.groups * k.slices * 2 * kKeys * d.d * sizeof(float);
  return stat_bytes(d, n_tokens, batch) + part;
}

hipError_t launch_packed_backward(const HeadsDims& d, const PackedCall& c, const PackedOut& o, char* ws, hipStream_t s) {
  const PagedParams p = packed_params(d, c);
  const KeyPlan k = key_plan(d, c.n_tokens, c.batch, c.max_len, c.window, c.sinks);
  PackedGrads z{};
  z.dout = o.dout.p;
  z.do_ts = o.dout.ts;
  z.do_hs = o.dout.hs;
  z.dq = o.dq.p;
  z.dq_ts = o.dq.ts;
  z.dq_hs = o.dq.hs;
  z.dk = o.dk.p;
  z.dk_ts = o.dk.ts;
  z.dk_hs = o.dk.hs;
  z.dv = o.dv.p;
  z.dv_ts = o.dv.ts;
  z.dv_hs = o.dv.hs;
  z.stats = reinterpret_cast<float2*>(ws);
  z.stat_rows = stat_rows(c.n_tokens, c.batch);
  z.scale = c.scale;
  z.key_blocks = (int)(k.groups / d.hk);
  z.slices = k.slices;
  z.fslices = FastDiv(k.slices);
  z.fmin_tiles = FastDiv(k.min_tiles);
  z.part = reinterpret_cast<float*>(ws + stat_bytes(d, c.n_tokens, c.batch));
  if (d.esize == 2) return d.d == 64 ? backward_on<bf16, 64>(d, p, z, s) : backward_on<bf16, 128>(d, p, z, s);
  return d.d == 64 ? backward_on<float, 64>(d, p, z, s) : backward_on<float, 128>(d, p, z, s);
}

}  // namespace pf
