// Attention of ordinary tokens beside the proxies: queries and keys normed
// and turned by their positions, the paged cache they go to, and the attention
// of new tokens, one of every sequence or a prompt, over it.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime.h>

#include "../../include/proxyformer.h"
#include "common.hpp"

namespace pf {

// A tensor of rows [token, head, head_dim]; strides in elements.
struct Rows {
  char* p = nullptr;
  int64_t ts = 0, hs = 0;
};

// What the norm and the rotation need, as every kernel of them takes it.
struct HeadsDims {
  int hq, hk, d, esize;
  int norm;
  float eps;
  int rot;              // elements turned, a multiple of 16
  int pairs_style;      // PF_ROPE_PAIRS
  int axis_end[PF_MAX_AXES];  // first pair past each axis
  int n_axes;
};

struct HeadsWeights {
  const void* gamma_q;
  const void* gamma_k;
  const double* freqs;
};

struct PagedDims {
  char* k;
  char* v;
  uint8_t* k_scale;  // pages of 8 bits, else NULL
  uint8_t* v_scale;
  int n_pages, page_size;
  const int32_t* table;
  int max_pages;
  const int32_t* kv_len;
  int batch;
};

// A launch has fewer than 2^32 threads in a dimension: workgroups of 256 at most.
constexpr int64_t kMaxGroups = ((int64_t)1 << 24) - 1;
// Tokens of a call: four per workgroup at least.
constexpr int64_t kMaxTokens = 4 * kMaxGroups;

// The largest s < count with at(s) <= x, where at rises and at(0) <= x: the
// wave probes 64 places at a time, each time within the run that is left. Of
// boundaries that do not rise it is some s in range.
template <class F>
__device__ __forceinline__ int find_run(int count, F&& at, int64_t x) {
  const int lane = (int)(threadIdx.x & (kWave - 1));
  int s = 0;
  for (int n = count; n > 1;) {
    const int step = (n + kWave - 1) / kWave, c = lane * step;
    const bool below = c < n && at(s + (c < n ? c : 0)) <= x;
    const int k = max((int)__popcll(__ballot(below)) - 1, 0);
    s += k * step;
    n = min(step, n - k * step);
  }
  return __builtin_amdgcn_readfirstlane(s);
}

// Where token `tok` of a call, of sequence s, is in a cache: its row (head 0) in
// the pages, or -1 for one of no sequence or without a place; `at` is its row of
// the sequence, kv_len - new + i for the i-th new token.
__device__ __forceinline__ int64_t place_in(const int32_t* cu, const int32_t* kv_len, const int32_t* table, int batch,
                                            int max_pages, int n_pages, int hk, const FastDiv& fpage, int64_t tok, int s,
                                            int* at) {
  *at = 0;
  if (s >= batch || (cu && tok < cu[s])) return -1;
  const int64_t pos = cu ? (int64_t)kv_len[s] - cu[s + 1] + tok : (int64_t)kv_len[s] - 1;
  if (pos < 0 || pos >= (int64_t)max_pages * fpage.d) return -1;
  *at = (int)pos;
  const int pg = fpage.div((int)pos);
  const int id = table[(int64_t)s * max_pages + pg];
  return id >= 0 && id < n_pages ? (int64_t)id * hk * fpage.d + ((int)pos - pg * fpage.d) : -1;
}

// The same, with its sequence to be found (by the whole wave).
__device__ __forceinline__ int64_t cache_place(const int32_t* cu, const int32_t* kv_len, const int32_t* table, int batch,
                                               int max_pages, int n_pages, int hk, const FastDiv& fpage, int64_t tok,
                                               int* at) {
  return place_in(cu, kv_len, table, batch, max_pages, n_pages, hk, fpage, tok,
                  cu ? find_run(batch + 1, [&](int c) { return cu[c]; }, tok) : (int)tok, at);
}
int heads_dims(const pf_heads_config* c, HeadsDims* d, const char** why);

// Forward: q -> q_out, k -> k_out. n_tokens rows, positions [n_axes, n_tokens].
hipError_t launch_qk_forward(const HeadsDims& d, const HeadsWeights& w, int64_t n, const Rows& q, const Rows& k,
                             const int32_t* positions, const Rows& q_out, const Rows& k_out, hipStream_t s);
// Append: q (its p may be NULL) -> q_out, k and v -> the pages.
hipError_t launch_paged_append(const HeadsDims& d, const HeadsWeights& w, const PagedDims& c, int64_t n,
                               const int32_t* cu_tokens, const Rows& q, const Rows& k, const Rows& v,
                               const int32_t* positions, const Rows& q_out, hipStream_t s);
// 8-bit pages back into rows of the config's type: those that an append of the
// same tokens writes.
hipError_t launch_paged_quant_read(const HeadsDims& d, const PagedDims& c, int64_t n, const int32_t* cu_tokens, const Rows& k_out,
                              const Rows& v_out, hipStream_t s);
size_t qk_backward_ws(const HeadsDims& d, int64_t n);
hipError_t launch_qk_backward(const HeadsDims& d, const HeadsWeights& w, int64_t n, const Rows& q, const Rows& k,
                              const int32_t* positions, const Rows& dq_out, const Rows& dk_out, const Rows& dq,
                              const Rows& dk, float* dgamma_q, float* dgamma_k, float* ws, hipStream_t s);

// Attention over the cache: how its rows are cut. The tiles that a block of
// queries sees are cut into at most `slices` runs of at least `min_tiles`, by
// its own length.
struct PagedPlan {
  bool prompt;       // paged_prompt_kernel, or the one for single tokens
  int cols, tile_rows;
  int slices, min_tiles;
  int64_t groups;  // workgroups per slice
  size_t bytes;
};
PagedPlan paged_plan(const HeadsDims& d, int batch, int64_t n_tokens, bool ragged, int64_t max_new, int64_t max_kv_len,
                     int64_t window, int64_t sinks, bool bits8);
hipError_t launch_paged_attention(const HeadsDims& d, const PagedDims& c, const PagedPlan& pl, int64_t n_tokens,
                                  const int32_t* cu_tokens, const Rows& q, float scale, int64_t window, int64_t sinks,
                                  void* out, float* lse, char* ws, hipStream_t s);

// Attention over whole sequences that lie one after another.
struct PackedCall {
  int64_t n_tokens, max_len;
  const int32_t* cu;
  int batch;
  Rows q, k, v;
  int64_t window, sinks;
  float scale;
  void* out;   // the backward reads out and lse
  float* lse;
};
struct PackedOut {
  Rows dout, dq, dk, dv;
};
// Workgroups by columns and by keys.
int64_t packed_groups(const HeadsDims& d, int64_t n_tokens, int batch);
int64_t packed_key_groups(const HeadsDims& d, int64_t n_tokens, int batch);
size_t packed_backward_ws(const HeadsDims& d, int64_t n_tokens, int batch, int64_t max_len, int64_t window, int64_t sinks);
hipError_t launch_packed_forward(const HeadsDims& d, const PackedCall& c, hipStream_t s);
hipError_t launch_packed_backward(const HeadsDims& d, const PackedCall& c, const PackedOut& o, char* ws, hipStream_t s);

}  // namespace pf
