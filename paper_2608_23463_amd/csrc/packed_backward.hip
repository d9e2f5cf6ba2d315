// Gradients of causal attention over whole sequences that lie one after
// another.
//
//   p_ij = exp(scale q_i.k_j - lse_i) where i sees j, D_i = dO_i.O_i
//   dV_j = sum_i p_ij dO_i,  dS_ij = p_ij (dO_i.v_j - D_i)
//   dQ_i = scale sum_j dS_ij k_j,  dK_j = scale sum_i dS_ij q_i
// over the query heads of a K/V head too in dK and dV. The probabilities are
// formed again from the forward's log-sums. Three kernels, no atomics: every
// gradient is written once, in the same order of additions in every run.
//  - packed_stats_kernel: D_i, and lse_i in exp2 units, heads first.
//  - packed_dkdv_kernel: 128 keys of a K/V head, 32 per wave, one per lane
//    pair; the 32-query tiles that see them, head after head.
//  - packed_dq_kernel: 128 columns (token, head), 32 per wave; the tiles of keys
//    that they see.
// A tile lies in LDS once, by rows; the products over channels read it by rows,
// those over positions by channels (in bf16 through transposing reads), so P
// and dS are operands in the registers where they were computed. In bf16 both
// are rounded to it, 2^-8 of each at most; sums are fp32.
#include <algorithm>

#include "packed.hpp"
#include "trace.hpp"

namespace pf {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kKeys = 128;  // of a workgroup of dK and dV
constexpr int kQueries = 32;

// A wave per token: its place among the statistics, then its heads' rows.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) packed_stats_kernel(PagedParams p, PackedGrads z) {
  constexpr int LPR = D / 8;  // lanes of a row, eight channels each
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int tok = (int)blockIdx.x * kWaves + wave;
  if (tok >= p.n_tokens) return;
  const int s = find_run(p.batch, [&](int c) { return p.cu[c]; }, tok);
  Sequence sq;
  sq.set(p, s);
  const int i = tok - sq.t0;
  if (sq.seq < 0 || i < 0 || i >= sq.cols / p.group) return;
  const int64_t at = stat_row(sq.t0, s) + i;
  const int c = lane % LPR * 8;
  for (int h = lane / LPR; h < p.hq; h += kWave / LPR) {
    float a[8], b[8], d = 0.0f;
    load8(reinterpret_cast<const T*>(p.out) + ((int64_t)tok * p.hq + h) * D + c, a);
    load8(reinterpret_cast<const T*>(z.dout) + (int64_t)tok * z.do_ts + (int64_t)h * z.do_hs + c, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) d += a[e] * b[e];
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) d += __shfl_xor(d, o);
    if (lane % LPR == 0)
      z.stats[h * z.stat_rows + at] = make_float2(p.lse[(int64_t)tok * p.hq + h] * 1.4426950408889634f, d);
  }
}

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

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1) packed_dkdv_kernel(PagedParams p, PackedGrads z) {
  typedef BothWays<T, D> Tl;
  typedef Mma<T> MM;
  constexpr int kTileBytes = kQueries * Tl::RB, kStage = 2 * kTileBytes + 1024, es = (int)sizeof(T);
  __shared__ __attribute__((aligned(1024))) char smem[2][kStage];  // Q, dO, statistics
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5, col = lane & 31;

  const int at = xcd_run(), hk = z.fkey_blocks.div(at), blk = at - hk * z.key_blocks;
  const int s = find_run(p.batch, [&](int c) { return p.cu[c] / kKeys + c; }, blk);
  Sequence sq;
  sq.set(p, s);
  const int n = sq.seq < 0 ? 0 : sq.cols / p.group, k0 = (blk - (p.cu[s] / kKeys + s)) * kKeys;
  if (k0 < 0 || k0 >= n) return;
  const int key = k0 + wave * 32 + col;
  const bool on = key < n;

  typename MM::frag kf[D / 16], vf[D / 16];
  {
    const int64_t tok = sq.t0 + (on ? key : k0);
    const T* kp = reinterpret_cast<const T*>(p.k) + tok * p.k_ts + (int64_t)hk * p.k_hs;
    const T* vp = reinterpret_cast<const T*>(p.v) + tok * p.v_ts + (int64_t)hk * p.v_hs;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      kf[kk] = MM::load(kp + kk * 16 + g * 8);
      vf[kk] = MM::load(vp + kk * 16 + g * 8);
    }
  }
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) dk[cb][r] = dv[cb][r] = 0.0f;

  // the queries that see a key of the block: from its first key on, up to the
  // end of its last key's windows, or to the sequence's end for the first rows
  const int64_t reach = k0 < p.sinks ? n : min((int64_t)n, (int64_t)k0 + kKeys - 1 + p.window);
  const int tiles = ((int)reach - k0 + kQueries - 1) / kQueries, total = tiles * p.group;
  const int wk0 = k0 + wave * 32;
  int ih = 0, it = 0;  // head and tile of the loads
  auto issue = [&](int stage) {
    const int q0 = k0 + it * kQueries, h = hk * p.group + ih;
    char* st = smem[stage];
    Tl::template load<kQueries>(p.q + (sq.t0 * p.q_ts + h * p.q_hs) * es, p.q_ts * es, q0, n - 1, st, wave, lane);
    Tl::template load<kQueries>(z.dout + (sq.t0 * z.do_ts + h * z.do_hs) * es, z.do_ts * es, q0, n - 1, st + kTileBytes,
                                wave, lane);
    if (wave == 0) {
      const rsrc_t rs = make_rsrc_uniform(z.stats + h * z.stat_rows + stat_row(sq.t0, s) + q0, kQueries * 8);
      buf_ld16_lds(rs, lane < kQueries / 2 ? lane * 16 : kOOB, st + 2 * kTileBytes);
    }
    if (++it == tiles) {
      it = 0;
      ++ih;
    }
  };
  issue(0);
  int ct = 0;
  for (int t = 0; t < total; ++t) {
    wait_vmcnt<0>();
    lds_barrier();
    if (t + 1 < total) issue((t + 1) & 1);
    const int q0 = k0 + ct * kQueries;
    ct = ct + 1 == tiles ? 0 : ct + 1;
    // wave-uniform: nothing of the tile sees the wave's keys
    if (q0 + kQueries - 1 < wk0 || (q0 - p.window >= wk0 + 31 && wk0 >= p.sinks)) continue;
    const char* sq_ = smem[t & 1];
    const char* so = sq_ + kTileBytes;
    const float* st = reinterpret_cast<const float*>(so + kTileBytes);
    f32x16 sc, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = dp[r] = 0.0f;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      sc = MM::mma(Tl::row(sq_, col, kk, g), kf[kk], sc);
      dp = MM::mma(Tl::row(so, col, kk, g), vf[kk], dp);
    }
    const bool whole = q0 >= wk0 + 31 && q0 + kQueries <= n && (q0 + kQueries - 1 - p.window < wk0 || wk0 + 31 < p.sinks);
#pragma unroll
    for (int r4 = 0; r4 < 16; r4 += 4) {
      const int i0 = acc_row(r4, lane);
      const f32x4 a = *reinterpret_cast<const f32x4*>(st + 2 * i0), b = *reinterpret_cast<const f32x4*>(st + 2 * i0 + 4);
      const float ls[4] = {a[0], a[2], b[0], b[2]}, de[4] = {a[1], a[3], b[1], b[3]};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = q0 + i0 + e;
        float pr = fast_exp2(fmaf(sc[r4 + e], p.scale_log2, -ls[e]));
        float ds = pr * (dp[r4 + e] - de[e]);
        if (!whole && !(key <= i && i < n && (key > i - p.window || key < p.sinks))) pr = ds = 0.0f;
        sc[r4 + e] = pr;
        dp[r4 + e] = ds;
      }
    }
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
      const auto pf = Tl::operand(sc, s2), df = Tl::operand(dp, s2);
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb) {
        dv[cb] = MM::mma(Tl::col(so, s2 * 16, cb * 32, lane), pf, dv[cb]);
        dk[cb] = MM::mma(Tl::col(sq_, s2 * 16, cb * 32, lane), df, dk[cb]);
      }
    }
  }
  if (!on) return;
  const int64_t tok = sq.t0 + key;
  store_rows<T, D>(reinterpret_cast<T*>(z.dk) + tok * z.dk_ts + (int64_t)hk * z.dk_hs, dk, z.scale, lane);
  store_rows<T, D>(reinterpret_cast<T*>(z.dv) + tok * z.dv_ts + (int64_t)hk * z.dv_hs, dv, 1.0f, lane);
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) packed_dq_kernel(PagedParams p, PackedGrads z) {
  typedef BothWays<T, D> Tl;
  typedef Mma<T> MM;
  constexpr int kRows = 32, kTileBytes = kRows * Tl::RB, es = (int)sizeof(T);
  __shared__ __attribute__((aligned(1024))) char smem[2][2 * kTileBytes];  // K, V
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5, col = lane & 31;
  const Columns c(p, lane, wave);
  if (!c.any) return;
  const Sight sight(p, c.sq, c.x0, c.cols, kRows);
  const int lo = c.row - p.window;
  const int wcols = min(c.cols - wave * 32, 32);  // <= 0: an idle wave
  const int wfirst = p.fgroup.div(c.x0 + wave * 32), wtop = wcols > 0 ? p.fgroup.div(c.x0 + wave * 32 + wcols - 1) : -1;

  typename MM::frag qf[D / 16], of[D / 16];
  float2 st = make_float2(0.0f, 0.0f);
  {
    const int64_t tok = c.sq.t0 + c.tok;
    const T* qp = reinterpret_cast<const T*>(p.q) + tok * p.q_ts + (int64_t)c.head * p.q_hs;
    const T* op = reinterpret_cast<const T*>(z.dout) + tok * z.do_ts + (int64_t)c.head * z.do_hs;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      qf[kk] = MM::load(qp + kk * 16 + g * 8);
      of[kk] = MM::load(op + kk * 16 + g * 8);
    }
    st = z.stats[c.head * z.stat_rows + stat_row(c.sq.t0, c.sq.seq) + c.tok];
  }
  const char* k = p.k + (c.sq.t0 * p.k_ts + c.hk * p.k_hs) * es;
  const char* v = p.v + (c.sq.t0 * p.v_ts + c.hk * p.v_hs) * es;
  auto issue = [&](int t) {
    const int r0 = sight.tile(t) * kRows;
    Tl::template load<kRows>(k, p.k_ts * es, r0, sight.last, smem[t & 1], wave, lane);
    Tl::template load<kRows>(v, p.v_ts * es, r0, sight.last, smem[t & 1] + kTileBytes, wave, lane);
  };
  f32x16 dq[D / 32];
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) dq[cb][r] = 0.0f;
  issue(0);
  for (int t = 0; t < sight.tiles; ++t) {
    wait_vmcnt<0>();
    lds_barrier();
    if (t + 1 < sight.tiles) issue(t + 1);
    const int r0 = sight.tile(t) * kRows;
    if (r0 > wtop || (r0 + kRows - 1 <= wfirst - p.window && r0 >= p.sinks)) continue;  // wave-uniform
    const char* sk = smem[t & 1];
    const char* sv = sk + kTileBytes;
    f32x16 sc, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = dp[r] = 0.0f;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      sc = MM::mma(Tl::row(sk, col, kk, g), qf[kk], sc);
      dp = MM::mma(Tl::row(sv, col, kk, g), of[kk], dp);
    }
    const bool whole = r0 + kRows - 1 <= wfirst && (r0 > wtop - p.window || r0 + kRows <= p.sinks);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int j = r0 + acc_row(r, lane);
      float ds = fast_exp2(fmaf(sc[r], p.scale_log2, -st.x)) * (dp[r] - st.y);
      if (!whole && !(j <= c.row && (j > lo || j < p.sinks))) ds = 0.0f;
      sc[r] = ds;
    }
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2) {
      const auto df = Tl::operand(sc, s2);
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb) dq[cb] = MM::mma(Tl::col(sk, s2 * 16, cb * 32, lane), df, dq[cb]);
    }
  }
  if (!c.on) return;
  store_rows<T, D>(reinterpret_cast<T*>(z.dq) + (c.sq.t0 + c.tok) * z.dq_ts + (int64_t)c.head * z.dq_hs, dq, z.scale, lane);
}

template <typename T, int D>
hipError_t backward_on(const HeadsDims& d, const PagedParams& p, const PackedGrads& z, hipStream_t s) {
  hipError_t e = timed("packed_stats", s, [&] {
    packed_stats_kernel<T, D><<<dim3((unsigned)((p.n_tokens + kWaves - 1) / kWaves)), kThreads, 0, s>>>(p, z);
  });
  if (e != hipSuccess) return e;
  e = timed("packed_dkdv", s, [&] {
    packed_dkdv_kernel<T, D><<<dim3((unsigned)(z.key_blocks * d.hk)), kThreads, 0, s>>>(p, z);
  });
  if (e != hipSuccess) return e;
  return timed("packed_dq", s, [&] {
    packed_dq_kernel<T, D><<<dim3((unsigned)packed_groups(d, p.n_tokens, p.batch)), kThreads, 0, s>>>(p, z);
  });
}

int64_t stat_rows(int64_t n_tokens, int batch) { return (n_tokens + 3) / 4 * 4 + 4 * (int64_t)batch + kQueries; }

}  // namespace

int64_t packed_key_groups(const HeadsDims& d, int64_t n_tokens, int batch) {
  return (n_tokens / kKeys + batch) * d.hk;
}

size_t packed_backward_ws(const HeadsDims& d, int64_t n_tokens, int batch) {
  return (size_t)d.hq * stat_rows(n_tokens, batch) * sizeof(float2);
}

hipError_t launch_packed_backward(const HeadsDims& d, const PackedCall& c, const PackedOut& o, char* ws, hipStream_t s) {
  const PagedParams p = packed_params(d, c);
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
  z.key_blocks = (int)(packed_key_groups(d, c.n_tokens, c.batch) / d.hk);
  z.fkey_blocks = FastDiv(z.key_blocks);
  if (d.esize == 2) return d.d == 64 ? backward_on<bf16, 64>(d, p, z, s) : backward_on<bf16, 128>(d, p, z, s);
  return d.d == 64 ? backward_on<float, 64>(d, p, z, s) : backward_on<float, 128>(d, p, z, s);
}

}  // namespace pf
