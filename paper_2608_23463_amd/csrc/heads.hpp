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

int heads_dims(const pf_heads_config* c, HeadsDims* d, const char** why);

// Forward: q -> q_out, k -> k_out. n_tokens rows, positions [n_axes, n_tokens].
hipError_t launch_qk_forward(const HeadsDims& d, const HeadsWeights& w, int64_t n, const Rows& q, const Rows& k,
                             const int32_t* positions, const Rows& q_out, const Rows& k_out, hipStream_t s);
// Append: q (its p may be NULL) -> q_out, k and v -> the pages.
hipError_t launch_paged_append(const HeadsDims& d, const HeadsWeights& w, const PagedDims& c, int64_t n,
                               const int32_t* cu_tokens, const Rows& q, const Rows& k, const Rows& v,
                               const int32_t* positions, const Rows& q_out, hipStream_t s);
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
                     int64_t window, int64_t sinks);
hipError_t launch_paged_attention(const HeadsDims& d, const PagedDims& c, const PagedPlan& pl, int64_t n_tokens,
                                  const int32_t* cu_tokens, const Rows& q, float scale, int64_t window, int64_t sinks,
                                  void* out, float* lse, char* ws, hipStream_t s);

}  // namespace pf
