// Rows of an 8-bit cache back into the rows' type: codes times their row's power
// of two, exact in bf16 and in fp32. Bound by HBM: 1 + es bytes per element.
#include "paged.hpp"
#include "trace.hpp"

namespace pf {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kTokens = 4;  // of a wave

struct Read8Params {
  const char* k;
  const char* v;
  const uint8_t* k_scale;
  const uint8_t* v_scale;
  const int32_t* table;
  const int32_t* kv_len;
  const int32_t* cu;
  int n_pages, page_size, max_pages, batch, hk;
  FastDiv fpage, fhk;
  int64_t n;
  Rows k_out, v_out;
};

// A wave takes kTokens tokens, whose rows run through it D / 16 lanes each.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) paged_quant_read_kernel(Read8Params p) {
  constexpr int LPR = D / 16, RPP = kWave / LPR;
  __shared__ int64_t places[kWaves][kTokens];
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int64_t t0 = ((int64_t)blockIdx.x * kWaves + wave) * kTokens;
  const int tokens = (int)min((int64_t)kTokens, p.n - t0);
  if (tokens <= 0) return;  // waves share nothing: no barrier below
  for (int i = 0; i < tokens; ++i) {
    int at;
    const int64_t place = cache_place(p.cu, p.kv_len, p.table, p.batch, p.max_pages, p.n_pages, p.hk, p.fpage, t0 + i, &at);
    if (lane == 0) places[wave][i] = place;
  }
  __builtin_amdgcn_wave_barrier();
  const int rows = 2 * p.hk, c = lane % LPR * 16;
  for (int it = lane / LPR; it < tokens * rows; it += RPP) {
    const int u = p.fhk.div(it), tk = u / 2, h = it - u * p.hk;  // K's heads, then V's
    const int64_t place = places[wave][tk];
    if (place < 0) continue;
    const int64_t row = place + (int64_t)h * p.page_size;
    const u32x4 w = ld16((u & 1 ? p.v : p.k) + row * D + c);
    const float f = scale_of((u & 1 ? p.v_scale : p.k_scale)[row]);
    float x[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], f, false);
      const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i], f, true);
      x[4 * i] = a[0];
      x[4 * i + 1] = a[1];
      x[4 * i + 2] = b[0];
      x[4 * i + 3] = b[1];
    }
    const Rows& out = u & 1 ? p.v_out : p.k_out;
    T* dst = reinterpret_cast<T*>(out.p) + (t0 + tk) * out.ts + h * out.hs + c;
    store8(dst, x);
    store8(dst + 8, x + 8);
  }
}

template <typename T>
void read_on(const HeadsDims& d, const Read8Params& p, hipStream_t s) {
  const dim3 grid((unsigned)((p.n + kWaves * kTokens - 1) / (kWaves * kTokens)));
  if (d.d == 64)
    paged_quant_read_kernel<T, 64><<<grid, kThreads, 0, s>>>(p);
  else
    paged_quant_read_kernel<T, 128><<<grid, kThreads, 0, s>>>(p);
}

}  // namespace

hipError_t launch_paged_quant_read(const HeadsDims& d, const PagedDims& c, int64_t n, const int32_t* cu_tokens, const Rows& k_out,
                              const Rows& v_out, hipStream_t s) {
  Read8Params p{};
  p.k = c.k;
  p.v = c.v;
  p.k_scale = c.k_scale;
  p.v_scale = c.v_scale;
  p.table = c.table;
  p.kv_len = c.kv_len;
  p.cu = cu_tokens;
  p.n_pages = c.n_pages;
  p.page_size = c.page_size;
  p.max_pages = c.max_pages;
  p.batch = c.batch;
  p.hk = d.hk;
  p.fpage = FastDiv(c.page_size);
  p.fhk = FastDiv(d.hk);
  p.n = n;
  p.k_out = k_out;
  p.v_out = v_out;
  return timed("paged_quant_read", s, [&] { d.esize == 2 ? read_on<bf16>(d, p, s) : read_on<float>(d, p, s); });
}

}  // namespace pf
