// Rows of an 8-bit cache back into the rows' type: codes times their row's power
// of two, exact in bf16 and in fp32 (scale bytes of 3 to 246). Bound by HBM: 1 + es bytes per element
// (24 sequences of up to 7,000 rows, 8 heads of 128, 131 us, 4.9 TB/s; with 32 bytes of a
// lane's written side by side 160).
#include "paged.hpp"
#include "trace.hpp"

namespace pf {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kMostTokens = 4;  // of a wave

// A wave takes one token where its rows of K and V fill more than half of the four
// passes that load together, or where waves are few; else kMostTokens. 168,000 tokens
// of 2 x 64 in bf16 30 us (a token each 77), 4 x 128 104 (134), 12 x 64 168 (165), 16 x
// 64 223 (208), 8 x 128 in fp32 355 (337); 8,192 of 8 x 64 8.7 us (9.2), 4,096 of them 7.4
// (6.6), 150 6.2 (4.9).
constexpr int kManyTokens = 8192, kFewBytes = 1024;  // bytes of a token's K in the rows' type

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
  int tokens;  // of a wave
  Rows k_out, v_out;
};

// A wave takes up to kMostTokens consecutive tokens. A lane each finds a token's
// place, within the sequences of the first and the last; then the (token, head)
// rows run through the wave, 16 bytes of a lane's written at a
// time and four passes' loads on their way together.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) paged_quant_read_kernel(Read8Params p) {
  constexpr int VL = 16 / (int)sizeof(T);  // channels of a lane: 16 bytes written side by side
  constexpr int LPR = D / VL, RPP = kWave / LPR, kAhead = 4;
  typedef uint32_t Codes __attribute__((ext_vector_type(VL / 4)));
  __shared__ int64_t places[kWaves][kMostTokens];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int64_t t0 = ((int64_t)blockIdx.x * kWaves + wave) * p.tokens;
  const int tokens = (int)min((int64_t)p.tokens, p.n - t0);
  if (tokens <= 0) return;  // waves share nothing: no barrier below
  const int64_t mine = t0 + min(lane, tokens - 1);
  int s = (int)mine;
  if (p.cu) {
    auto first = [&](int c) { return p.cu[c]; };
    s = find_run(p.batch + 1, first, t0);
    // the last of s .. end that begins at or before the lane's token
    for (int end = tokens == 1 ? s : find_run(p.batch + 1, first, t0 + tokens - 1); s < end;) {
      const int mid = (s + end + 1) / 2;
      if (p.cu[mid] <= mine)
        s = mid;
      else
        end = mid - 1;
    }
  }
  if (lane < tokens) {
    int at;
    places[wave][lane] = place_in(p.cu, p.kv_len, p.table, p.batch, p.max_pages, p.n_pages, p.hk, p.fpage, mine, s, &at);
  }
  __builtin_amdgcn_wave_barrier();
  const int items = 2 * p.hk * tokens, c = lane % LPR * VL;
  for (int base = lane / LPR; base < items; base += kAhead * RPP) {
    Codes w[kAhead];
    uint32_t byte[kAhead];
    int64_t row[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int it = base + i * RPP, u = p.fhk.div(it), h = it - u * p.hk;  // K's heads of a token, then V's
      const int64_t place = it < items ? places[wave][u / 2] : -1;
      row[i] = place < 0 ? -1 : place + (int64_t)h * p.page_size;
      const int64_t from = max(row[i], (int64_t)0);
      w[i] = *reinterpret_cast<const Codes*>((u & 1 ? p.v : p.k) + from * D + c);
      byte[i] = (u & 1 ? p.v_scale : p.k_scale)[from];
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (row[i] < 0) continue;
      const int it = base + i * RPP, u = p.fhk.div(it), h = it - u * p.hk;
      const float f = scale_of(byte[i]);
      float x[VL];
#pragma unroll
      for (int j = 0; j < VL / 4; ++j) {
        const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i][j], f, false);
        const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[i][j], f, true);
        x[4 * j] = a[0];
        x[4 * j + 1] = a[1];
        x[4 * j + 2] = b[0];
        x[4 * j + 3] = b[1];
      }
      const Rows& out = u & 1 ? p.v_out : p.k_out;
      T* dst = reinterpret_cast<T*>(out.p) + (t0 + u / 2) * out.ts + h * out.hs + c;
      if constexpr (VL == 8)
        store8(dst, x);
      else
        store4(dst, x);
    }
  }
}

template <typename T>
void read_on(const HeadsDims& d, const Read8Params& p, hipStream_t s) {
  const dim3 grid((unsigned)((p.n + kWaves * p.tokens - 1) / (kWaves * p.tokens)));
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
  p.tokens = n >= kManyTokens && d.hk * d.d * d.esize <= kFewBytes ? kMostTokens : 1;
  p.k_out = k_out;
  p.v_out = v_out;
  return timed("paged_quant_read", s, [&] { d.esize == 2 ? read_on<bf16>(d, p, s) : read_on<float>(d, p, s); });
}

}  // namespace pf
