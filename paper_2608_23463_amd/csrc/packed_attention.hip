// Causal attention over whole sequences that lie one after another, in
// training: forward in fp32, and the calls' layout. In bf16 the forward is the
// prompts' kernel over packed rows (paged_prompt.hip); the gradients are in
// packed_backward.hip.
//
//   o_i = sum_j softmax_j(scale q_i.k_j) v_j over j <= i of the token's own
//   sequence and, with a window, j > i - window or j < sinks.
#include <algorithm>

#include "packed.hpp"
#include "trace.hpp"

namespace pf {

namespace {

constexpr int kThreads = 256;
constexpr int kRows = 32;  // of a tile

// Bound by the fp32 matrix instructions: 4 D flops per (column, row) seen.
// S^T = K Q^T and O^T += V^T P^T as in the prompts' kernel; tiles of 32 rows in
// two LDS stages (4,096 tokens, 16 over 4 heads of 128, 638 us, 108 TFLOP/s).
template <int D>
__global__ void __launch_bounds__(kThreads, 2) packed_forward_kernel(PagedParams p) {
  typedef BothWays<float, D> Tl;
  typedef Mma<float> MM;
  constexpr int kTileBytes = kRows * Tl::RB;
  __shared__ __attribute__((aligned(1024))) char smem[2][2 * kTileBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 5;
  const uint32_t rb = Tl::row_base(lane), cb0 = Tl::col_base(lane);
  const Columns c(p, lane, wave);
  if (!c.any) return;
  const Sight sight(p, c.sq, c.x0, c.cols, kRows);
  const int lo = c.row - p.window;

  MM::frag qf[D / 16];
  {
    const float* qp = reinterpret_cast<const float*>(p.q) + (int64_t)(c.sq.t0 + c.tok) * p.q_ts + (int64_t)c.head * p.q_hs;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[kk][e] = 0.0f;
      if (c.on) qf[kk] = MM::load(qp + kk * 16 + g * 8);
    }
  }
  const char* k = p.k + (c.sq.t0 * p.k_ts + c.hk * p.k_hs) * 4;
  const char* v = p.v + (c.sq.t0 * p.v_ts + c.hk * p.v_hs) * 4;
  auto issue = [&](int t) {
    const int r0 = sight.tile(t) * kRows;
    Tl::template load<kRows>(k, p.k_ts * 4, r0, sight.last, smem[t & 1], wave, lane);
    Tl::template load<kRows>(v, p.v_ts * 4, r0, sight.last, smem[t & 1] + kTileBytes, wave, lane, sight.first - p.window,
                             p.sinks);
  };
  f32x16 o[D / 32];
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[cb][r] = 0.0f;
  float mx = -INFINITY, sum = 0.0f;

  issue(0);
  for (int t = 0; t < sight.tiles; ++t) {
    wait_vmcnt<0>();
    lds_barrier();
    if (t + 1 < sight.tiles) issue(t + 1);
    const int r0 = sight.tile(t) * kRows;
    const char* sk = smem[t & 1];
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.0f;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) s = MM::mma(Tl::row(sk, rb, kk), qf[kk], s);
    float top = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int j = r0 + acc_row(r, lane);
      s[r] = j <= c.row && (j > lo || j < p.sinks) ? s[r] * p.scale_log2 : -INFINITY;
      top = fmaxf(top, s[r]);
    }
    top = fmaxf(top, other_half(top));
    const float now = fmaxf(mx, top), ref = now == -INFINITY ? 0.0f : now;
    const float back = fast_exp2(mx - ref);
    mx = now;
    float add = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = fast_exp2(s[r] - ref);
      add += s[r];
    }
    sum = sum * back + add;
#pragma unroll
    for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[cb][r] *= back;
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb)
        o[cb] = MM::mma(Tl::col(sk + kTileBytes, cb0, s2, cb), Tl::operand(s, s2), o[cb]);
  }
  if (!c.on) return;
  const float l = sum + other_half(sum), f = l > 0.0f ? 1.0f / l : l;
  const int64_t orow = (int64_t)(c.sq.t0 + c.tok) * p.hq + c.head;
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const float x[4] = {o[cb][r] * f, o[cb][r + 1] * f, o[cb][r + 2] * f, o[cb][r + 3] * f};
      store4(static_cast<float*>(p.out) + orow * D + cb * 32 + acc_row(r, lane), x);
    }
  if (g == 0 && p.lse) p.lse[orow] = (mx + __log2f(l)) * 0.69314718055994530942f;
}

}  // namespace

hipError_t launch_packed_forward(const HeadsDims& d, const PackedCall& c, hipStream_t s) {
  const PagedParams p = packed_params(d, c);
  const int64_t groups = packed_groups(d, c.n_tokens, c.batch);
  return timed("packed_attention", s, [&] {
    if (d.esize == 2)
      launch_prompt(p, d.d, kPacked, groups, s);
    else if (d.d == 64)
      packed_forward_kernel<64><<<dim3((unsigned)groups), kThreads, 0, s>>>(p);
    else
      packed_forward_kernel<128><<<dim3((unsigned)groups), kThreads, 0, s>>>(p);
  });
}

int64_t packed_groups(const HeadsDims& d, int64_t n_tokens, int batch) {
  return col_blocks(kPackedCols, d.hq / d.hk, n_tokens, batch) * d.hk;
}

PagedParams packed_params(const HeadsDims& d, const PackedCall& c) {
  PagedParams p{};
  p.q = c.q.p;
  p.q_ts = c.q.ts;
  p.q_hs = c.q.hs;
  p.k = c.k.p;
  p.k_ts = c.k.ts;
  p.k_hs = c.k.hs;
  p.v = c.v.p;
  p.v_ts = c.v.ts;
  p.v_hs = c.v.hs;
  p.cu = c.cu;
  p.batch = c.batch;
  p.n_tokens = (int)c.n_tokens;
  p.hq = d.hq;
  p.hk = d.hk;
  p.group = d.hq / d.hk;
  p.fgroup = FastDiv(p.group);
  p.fhk = FastDiv(d.hk);
  p.cols = kPackedCols;
  p.slices = 1;
  p.fslices = FastDiv(1);
  p.fmin_tiles = FastDiv(1);
  p.window = c.window > 0 ? (int)std::min<int64_t>(c.window, INT32_MAX) : INT32_MAX;
  p.sinks = (int)std::min<int64_t>(c.sinks, INT32_MAX);
  p.scale_log2 = c.scale * 1.4426950408889634f;
  p.out = c.out;
  p.lse = c.lse;
  return p;
}

}  // namespace pf
