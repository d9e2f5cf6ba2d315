// Queries and keys normed per head and turned by their positions: in training
// (forward, backward) and on the way into a paged cache (append).
//
//   z = x * rstd * gamma,  rstd = (mean(x^2) + eps)^-1/2   (without norm z = x)
//   pair (a, b) of the first rot elements, angle t = position * frequency:
//   y_a = z_a cos t - z_b sin t,  y_b = z_a sin t + z_b cos t
//
// A wave takes TPW consecutive tokens. It forms their cosines and sines once,
// one pair per lane, and keeps them in LDS for all heads of the tokens. Then
// the (token, head) rows of a tensor run through the wave in passes: D / 16
// lanes hold a row, 16 elements each, both members of eight pairs, so the
// rotation needs no exchange and the norm one sum over those lanes.
// Bound by HBM: every row is read and written once, in 16-byte accesses.
#include "heads.hpp"
#include "trace.hpp"

namespace pf {

int heads_dims(const pf_heads_config* c, HeadsDims* d, const char** why) {
  *why = "";
  if (!c) {
    *why = "config is NULL";
    return PF_ERR_INVALID_ARG;
  }
  if (c->dtype != PF_BF16 && c->dtype != PF_FP32) {
    *why = "dtype must be PF_BF16 or PF_FP32";
    return PF_ERR_INVALID_ARG;
  }
  if (c->n_heads < 1 || c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads != 0) {
    *why = "n_heads must be a positive multiple of n_kv_heads";
    return PF_ERR_INVALID_ARG;
  }
  if (c->n_heads > 4096) {
    *why = "more than 4096 heads";
    return PF_ERR_UNSUPPORTED;
  }
  if (c->head_dim != 64 && c->head_dim != 128) {
    *why = "head_dim must be 64 or 128";
    return PF_ERR_UNSUPPORTED;
  }
  if (c->norm != PF_NORM_NONE && c->norm != PF_NORM_RMS) {
    *why = "norm must be PF_NORM_NONE or PF_NORM_RMS";
    return PF_ERR_INVALID_ARG;
  }
  if (c->norm == PF_NORM_RMS && !(c->eps >= 0.0f && c->eps < 1e30f)) {
    *why = "eps must be finite and not negative";
    return PF_ERR_INVALID_ARG;
  }
  if (c->rot_dim < 0 || c->rot_dim > c->head_dim || c->rot_dim % 16 != 0) {
    *why = "rot_dim must be a multiple of 16 in 0..head_dim";
    return PF_ERR_INVALID_ARG;
  }
  if (c->rope_style != PF_ROPE_HALVES && c->rope_style != PF_ROPE_PAIRS) {
    *why = "rope_style must be PF_ROPE_HALVES or PF_ROPE_PAIRS";
    return PF_ERR_INVALID_ARG;
  }
  if (c->n_axes < 1 || c->n_axes > PF_MAX_AXES) {
    *why = "n_axes must be in 1..PF_MAX_AXES";
    return PF_ERR_INVALID_ARG;
  }
  int end = 0;
  for (int i = 0; i < PF_MAX_AXES; ++i) {
    if (i < c->n_axes) {
      if (c->axis_pairs[i] < 0 || c->axis_pairs[i] > c->rot_dim / 2) {
        *why = "axis_pairs must not be negative or above rot_dim / 2";
        return PF_ERR_INVALID_ARG;
      }
      end += c->axis_pairs[i];
    }
    d->axis_end[i] = end;
  }
  if (end != c->rot_dim / 2) {
    *why = "axis_pairs must add up to rot_dim / 2";
    return PF_ERR_INVALID_ARG;
  }
  d->hq = c->n_heads;
  d->hk = c->n_kv_heads;
  d->d = c->head_dim;
  d->esize = c->dtype == PF_BF16 ? 2 : 4;
  d->norm = c->norm;
  d->eps = c->eps;
  d->rot = c->rot_dim;
  d->pairs_style = c->rope_style == PF_ROPE_PAIRS;
  d->n_axes = c->n_axes;
  return PF_OK;
}

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;

struct TurnParams {
  const double* freqs;
  const int32_t* positions;  // [n_axes, n] or NULL (append: by the cache)
  int64_t n;
  int rot;
  int axis_end[PF_MAX_AXES];
};

// Rotation and norm of one launch.
struct QkParams {
  TurnParams turn;
  Rows q, k, v, q_out, k_out;
  const void* gamma_q;
  const void* gamma_k;
  int hq, hk;
  FastDiv fq, fk;
  float eps;
  int norm;
  FastDiv fparts;  // few tokens: waves of a token
  // append
  char* k_pages;
  char* v_pages;
  uint8_t* k_scale;  // pages of 8 bits
  uint8_t* v_scale;
  const int32_t* table;
  const int32_t* kv_len;
  const int32_t* cu;
  int n_pages, page_size, max_pages, batch;
  FastDiv fpage;
};

// Cosine and sine of position * frequency. Far positions need more than 32
// bits: a position of 2^20 in fp32 leaves an angle off by up to 2^-4. The
// angle is formed in revolutions in 64 bits (three roundings: 2^-51 of it) and
// its whole revolutions dropped there. What rounding the rest to fp32 leaves, up
// to 2^-26 of a revolution, is turned by to first order.
__device__ __forceinline__ float2 turn_of(double freq, int pos) {
  const double rev = (double)pos * freq * 0.15915494309189533577;
  const double part = rev - rint(rev);
  const float f = (float)part, rest = (float)((part - f) * 6.28318530717958647693);
  float s, c;
  sincospif(2.0f * f, &s, &c);
  return make_float2(c - rest * s, s + rest * c);
}

__device__ __forceinline__ int axis_of(const TurnParams& t, int pair) {
  int a = 0;
#pragma unroll
  for (int i = 0; i < PF_MAX_AXES - 1; ++i) a += pair >= t.axis_end[i];
  return a;
}

// Where a lane's 16 elements of a row sit. Chunk c of D / 16; `turned` tells
// whether its pairs are among the rotated ones.
//  halves: members of pair p at p and rot / 2 + p. The elements past rot are
//  split in halves the same way, so every chunk is two runs of eight.
//  pairs: members at 2p and 2p + 1, one run of sixteen.
template <int D, bool PAIRS>
struct Chunk {
  int a, b;
  bool turned;
  __device__ __forceinline__ Chunk(int c, int rot) {
    if (PAIRS) {
      a = 16 * c;
      b = a + 8;
      turned = a < rot;
    } else {
      turned = 16 * c < rot;
      const int e = turned ? 8 * c : 8 * c - rot / 2;
      a = turned ? e : rot + e;
      b = turned ? rot / 2 + e : rot + (D - rot) / 2 + e;
    }
  }
};

// Member registers of pair i of a lane: v[ia(i)], v[ib(i)].
template <bool PAIRS>
__device__ __forceinline__ constexpr int ia(int i) { return PAIRS ? 2 * i : i; }
template <bool PAIRS>
__device__ __forceinline__ constexpr int ib(int i) { return PAIRS ? 2 * i + 1 : 8 + i; }

template <bool PAIRS>
__device__ __forceinline__ void rotate(float* v, const float2* cs, bool turned, float sign) {
  if (!turned) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = v[ia<PAIRS>(i)], b = v[ib<PAIRS>(i)], c = cs[i].x, s = sign * cs[i].y;
    v[ia<PAIRS>(i)] = a * c - b * s;
    v[ib<PAIRS>(i)] = a * s + b * c;
  }
}

// Sum over the 4 or 8 neighbouring lanes of a row, on the VALU: each other
// lane of a pair, then of the two pairs, then (mirrored) of the two fours.
template <int CTRL>
__device__ __forceinline__ float add_lane(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ double add_lane(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_mov_dpp((int)(uint32_t)u, CTRL, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_mov_dpp((int)(uint32_t)(u >> 32), CTRL, 0xf, 0xf, true);
  return v + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int LPR, typename V>
__device__ __forceinline__ V row_sum(V v) {
  static_assert(LPR == 4 || LPR == 8, "lanes of a row");
  v = add_lane<0xb1>(v);              // quad_perm 1 0 3 2
  v = add_lane<0x4e>(v);              // quad_perm 2 3 0 1
  if (LPR == 8) v = add_lane<0x141>(v);  // row_half_mirror
  return v;
}

// Largest over those lanes, of values that are not negative (a lane outside the
// row would give zero).
template <int CTRL>
__device__ __forceinline__ float max_lane(float v) {
  return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true)));
}
template <int LPR>
__device__ __forceinline__ float row_max(float v) {
  static_assert(LPR == 4 || LPR == 8, "lanes of a row");
  v = max_lane<0xb1>(v);
  v = max_lane<0x4e>(v);
  if (LPR == 8) v = max_lane<0x141>(v);
  return v;
}

template <typename T>
__device__ __forceinline__ void load16(const T* p, int a, int b, Raw8<T>* r) {
  raw_load8(p + a, r[0]);
  raw_load8(p + b, r[1]);
}

// Position of token t of the launch on an axis.
__device__ __forceinline__ int position_of(const TurnParams& t, int64_t tok, int axis) {
  return t.positions[(int64_t)axis * t.n + tok];
}

// One tensor's rows of a launch: which = 0 queries, 1 keys, 2 values (append:
// copied as they are).
struct Tensor {
  Rows in, out;
  const void* gamma;
  int heads, which;
  FastDiv fd;
};
__device__ __forceinline__ Tensor tensor_of(const QkParams& p, int which) {
  return which == 0 ? Tensor{p.q, p.q_out, p.gamma_q, p.hq, 0, p.fq}
                    : which == 1 ? Tensor{p.k, p.k_out, p.gamma_k, p.hk, 1, p.fk} : Tensor{p.v, Rows{}, nullptr, p.hk, 2, p.fk};
}

template <typename T>
__device__ __forceinline__ void load_gain(const QkParams& p, const Tensor& x, int a, int b, float* g) {
  if (!p.norm || x.which == 2) return;
  if (x.gamma) {
    load8(static_cast<const T*>(x.gamma) + a, g);
    load8(static_cast<const T*>(x.gamma) + b, g + 8);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) g[i] = 1.0f;
  }
}

// What a launch does with the rows: turned ones to tensors, or keys and values
// into pages of the rows' type or of 8 bits.
enum Mode { kTurn, kAppend, kAppend8 };

// Norm and rotation of the lane's 16 elements of a row. FINE: for keys that are
// held in 8 bits, whose values next to a border each error on the way moves by a
// whole step: the norm in 64 bits, rounded to fp32, then the turn in 64 bits by a
// cosine and a sine in fp32, rounded to it again. Element after element: side by
// side the products would cost the registers of a workgroup (24 prompts of up to
// 2,600 tokens, 32 over 8 heads of 128, 190 us for 163, 152 in 32 bits).
template <int D, bool PAIRS, bool FINE>
__device__ __forceinline__ void norm_and_turn(const QkParams& p, int which, float* v, const float* g, const float2* cs,
                                              bool turned) {
  if (which == 2) return;
  if (FINE && which == 1) {
    if (p.norm) {
      double ss = 0.0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        ss += (double)v[i] * v[i];
        asm volatile("" : "+v"(ss));
      }
      // (the mean of squares may be past fp32's range where the row is not)
      const double r = rsqrt(row_sum<D / 16>(ss) * (1.0 / D) + p.eps);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float gain = g[i];
        asm volatile("" : "+v"(gain));  // widened here, not kept wide over the rows
        v[i] = (float)(v[i] * r * gain);
        asm volatile("" : "+v"(v[i]));
      }
    }
    if (turned)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double a = v[ia<PAIRS>(i)], b = v[ib<PAIRS>(i)], c = cs[i].x, s = cs[i].y;
        v[ia<PAIRS>(i)] = (float)(a * c - b * s);
        v[ib<PAIRS>(i)] = (float)(a * s + b * c);
        asm volatile("" : "+v"(v[ia<PAIRS>(i)]), "+v"(v[ib<PAIRS>(i)]));
      }
    return;
  }
  if (p.norm) {
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) ss += v[i] * v[i];
    const float rstd = rsqrtf(row_sum<D / 16>(ss) * (1.0f / D) + p.eps);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] *= rstd * g[i];
  }
  rotate<PAIRS>(v, cs, turned, 1.0f);
}

// Where a token of an append goes: its row (head 0) in the pages, or -1 for one
// of no sequence or without a place; `at` is its row of the sequence.
__device__ __forceinline__ int64_t place_of(const QkParams& p, int64_t tok, int* at) {
  return cache_place(p.cu, p.kv_len, p.table, p.batch, p.max_pages, p.n_pages, p.hk, p.fpage, tok, at);
}

// The lane's 16 elements of a row, turned, to their place: tensors, or pages
// where `place` is the token's row.
//
// In 8 bits a row is codes in e4m3, to nearest even, of x 2^-e with the smallest
// e that takes the row's largest finite magnitude to at most 448 (and at least
// -110), and e + 127 as a byte: the multiplication is exact, so each element is
// rounded once. A floating code needs no finer scale than a power of two: its
// steps go by the value. What is not finite is held as NaN.
template <typename T, int D, Mode MODE>
__device__ __forceinline__ void put_row(const QkParams& p, const Tensor& x, int64_t tok, int h, bool on, int64_t place,
                                        int a, int b, float* v) {
  if (MODE != kAppend8 || x.which == 0) {
    if (!on) return;
    T* dst = MODE == kTurn || x.which == 0
                 ? reinterpret_cast<T*>(x.out.p) + tok * x.out.ts + h * x.out.hs
                 : reinterpret_cast<T*>(x.which == 1 ? p.k_pages : p.v_pages) + (place + (int64_t)h * p.page_size) * D;
    store8(dst + a, v);
    store8(dst + b, v + 8);
    return;
  }
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float m = fabsf(v[i]);
    top = fmaxf(top, m < INFINITY ? m : 0.0f);
  }
  top = row_max<D / 16>(top);
  const uint32_t bits = __builtin_bit_cast(uint32_t, top);
  const int byte = max((int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0), 17);
  const float inv = __builtin_bit_cast(float, (uint32_t)(254 - byte) << 23);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = fabsf(v[4 * i + e]) < INFINITY ? v[4 * i + e] * inv : NAN;
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    c = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], c, true);
    w[i] = (uint32_t)c;
  }
  if (!on) return;
  const int64_t row = place + (int64_t)h * p.page_size;
  char* dst = (x.which == 1 ? p.k_pages : p.v_pages) + row * D;
  *reinterpret_cast<uint2*>(dst + a) = make_uint2(w[0], w[1]);
  *reinterpret_cast<uint2*>(dst + b) = make_uint2(w[2], w[3]);
  if (threadIdx.x % (D / 16) == 0) (x.which == 1 ? p.k_scale : p.v_scale)[row] = (uint8_t)byte;
}

// Many tokens: TPW of them per wave, all their rows.
template <typename T, int D, bool PAIRS, int TPW, Mode MODE>
__global__ void __launch_bounds__(kThreads) qk_forward_kernel(QkParams p) {
  constexpr bool APPEND = MODE != kTurn;
  constexpr int LPR = D / 16, RPP = kWave / LPR;  // lanes per row, rows per pass
  __shared__ float2 turns[kWaves][TPW][D / 2];
  __shared__ int64_t places[kWaves][TPW];
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int64_t t0 = ((int64_t)blockIdx.x * kWaves + wave) * TPW;
  const int tokens = (int)min((int64_t)TPW, p.turn.n - t0);
  if (tokens <= 0) return;  // waves share nothing: no barrier below
  const int row = lane / LPR;
  const Chunk<D, PAIRS> ch(lane % LPR, p.turn.rot);

  for (int i = 0; i < tokens; ++i) {
    int at = 0;
    if (APPEND) {
      const int64_t place = place_of(p, t0 + i, &at);
      if (lane == 0) places[wave][i] = place;
    }
    for (int pair = lane; pair < D / 2; pair += kWave) {
      float2 cs = make_float2(1.0f, 0.0f);
      if (pair < p.turn.rot / 2) {
        if (!APPEND || p.turn.positions) at = position_of(p.turn, t0 + i, axis_of(p.turn, pair));
        cs = turn_of(p.turn.freqs[pair], at);
      }
      turns[wave][i][pair] = cs;
    }
  }
  __builtin_amdgcn_wave_barrier();  // LDS of the wave's own: in order without a workgroup barrier

  for (int which = p.q.p ? 0 : 1; which < (APPEND ? 3 : 2); ++which) {
    const Tensor x = tensor_of(p, which);
    const int items = tokens * x.heads;
    float g[16];
    load_gain<T>(p, x, ch.a, ch.b, g);
    for (int base = 0; base < items; base += RPP) {
      const int it = base + row;
      const bool on = it < items;
      const int tk = on ? x.fd.div(it) : 0, h = on ? it - tk * x.heads : 0;
      float v[16];
      Raw8<T> r[2];
      load16(reinterpret_cast<const T*>(x.in.p) + (t0 + tk) * x.in.ts + h * x.in.hs, ch.a, ch.b, r);
      raw_to_f32(r[0], v);
      raw_to_f32(r[1], v + 8);
      norm_and_turn<D, PAIRS, MODE == kAppend8>(p, which, v, g, &turns[wave][tk][8 * (lane % LPR)], ch.turned);
      const int64_t place = APPEND ? places[wave][tk] : 0;
      put_row<T, D, MODE>(p, x, t0 + tk, h, on && place >= 0, place, ch.a, ch.b, v);
    }
  }
}

// Few tokens: a wave for every RPP rows of every token, whose loads are on
// their way while it finds the token's place and its turns.
template <typename T, int D, bool PAIRS, Mode MODE>
__global__ void __launch_bounds__(kThreads) qk_few_kernel(QkParams p) {
  constexpr bool APPEND = MODE != kTurn;
  constexpr int LPR = D / 16, RPP = kWave / LPR;
  __shared__ float2 turns[kWaves][D / 2];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int unit = (int)blockIdx.x * kWaves + wave;
  const int tok = p.fparts.div(unit);
  int part = unit - tok * p.fparts.d;
  if (tok >= p.turn.n) return;
  const int pq = p.q.p ? (p.hq + RPP - 1) / RPP : 0, pk = (p.hk + RPP - 1) / RPP;
  const int which = part < pq ? 0 : part < pq + pk ? 1 : 2;
  part -= which == 0 ? 0 : which == 1 ? pq : pq + pk;
  const Tensor x = tensor_of(p, which);
  const Chunk<D, PAIRS> ch(lane % LPR, p.turn.rot);
  const int h = part * RPP + lane / LPR;
  const bool on = h < x.heads;
  float g[16], v[16];
  Raw8<T> r[2];
  load16(reinterpret_cast<const T*>(x.in.p) + (int64_t)tok * x.in.ts + (on ? h : 0) * x.in.hs, ch.a, ch.b, r);
  load_gain<T>(p, x, ch.a, ch.b, g);
  int at = 0;
  const int64_t place = APPEND ? place_of(p, tok, &at) : 0;
  if (which < 2) {
    for (int pair = lane; pair < D / 2; pair += kWave) {
      float2 cs = make_float2(1.0f, 0.0f);
      if (pair < p.turn.rot / 2) {
        if (!APPEND || p.turn.positions) at = position_of(p.turn, tok, axis_of(p.turn, pair));
        cs = turn_of(p.turn.freqs[pair], at);
      }
      turns[wave][pair] = cs;
    }
    __builtin_amdgcn_wave_barrier();
  }
  raw_to_f32(r[0], v);
  raw_to_f32(r[1], v + 8);
  norm_and_turn<D, PAIRS, MODE == kAppend8>(p, which, v, g, &turns[wave][8 * (lane % LPR)], ch.turned);
  put_row<T, D, MODE>(p, x, tok, h, on && place >= 0, place, ch.a, ch.b, v);
}

struct QkBwdParams {
  TurnParams turn;
  Rows q, k, dqo, dko, dq, dk;
  const void* gamma_q;
  const void* gamma_k;
  int hq, hk;
  FastDiv fq, fk;
  float eps;
  int norm;
  float* part;  // [2][blocks][D]: gains' gradients of every workgroup
};

// dz = R(-t) dy; dgamma += dz * xn with xn = x rstd; g = dz gamma;
// dx = rstd (g - xn mean(g xn)). A lane keeps the gains' gradients of its 16
// elements over kGainRows of its rows; then its wave's lanes are joined and
// added to sums in 64 bits, so that the error does not grow with the tokens.
// The workgroups' sums are joined in a fixed order.
constexpr int kGainRows = 64;

template <typename T, int D, bool PAIRS, int TPW>
__global__ void __launch_bounds__(kThreads, 3) qk_backward_kernel(QkBwdParams p) {
  constexpr int LPR = D / 16, RPP = kWave / LPR;
  __shared__ float2 turns[kWaves][TPW][D / 2];
  __shared__ double sums[kWaves][2][D];
  __shared__ float gains[2][D];
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int row = lane / LPR;
  const Chunk<D, PAIRS> ch(lane % LPR, p.turn.rot);
  float acc[2][16] = {};
  int rows = 0;  // of a lane since the last fold, at most
  for (int i = threadIdx.x; i < 2 * D; i += kThreads) {
    const T* gamma = static_cast<const T*>(i < D ? p.gamma_q : p.gamma_k);
    gains[i / D][i % D] = p.norm && gamma ? to_f32(gamma[i % D]) : 1.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) sums[w][i / D][i % D] = 0.0;
  }
  __syncthreads();
  const int64_t step = (int64_t)gridDim.x * kWaves * TPW;
  for (int64_t t0 = ((int64_t)blockIdx.x * kWaves + wave) * TPW; t0 < p.turn.n; t0 += step) {
    const int tokens = (int)min((int64_t)TPW, p.turn.n - t0);
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int i = 0; i < tokens; ++i)
      for (int pair = lane; pair < D / 2; pair += kWave) {
        float2 cs = make_float2(1.0f, 0.0f);
        if (pair < p.turn.rot / 2)
          cs = turn_of(p.turn.freqs[pair], position_of(p.turn, t0 + i, axis_of(p.turn, pair)));
        turns[wave][i][pair] = cs;
      }
    __builtin_amdgcn_wave_barrier();
    auto run = [&](const Rows& x, const Rows& dy, const Rows& dx, const float* gain, int heads, const FastDiv& fd,
                   float* ac) {
      const int items = tokens * heads;
#pragma unroll 1
      for (int it = row; it < items; it += RPP) {  // a row's lanes are on or off together
        const int tk = fd.div(it), h = it - tk * heads;
        float dz[16];
        Raw8<T> r[2], rx[2];
        load16(reinterpret_cast<const T*>(dy.p) + (t0 + tk) * dy.ts + h * dy.hs, ch.a, ch.b, r);
        if (p.norm) load16(reinterpret_cast<const T*>(x.p) + (t0 + tk) * x.ts + h * x.hs, ch.a, ch.b, rx);
        raw_to_f32(r[0], dz);
        raw_to_f32(r[1], dz + 8);
        rotate<PAIRS>(dz, &turns[wave][tk][8 * (lane % LPR)], ch.turned, -1.0f);
        if (p.norm) {
          float xn[16];
          raw_to_f32(rx[0], xn);
          raw_to_f32(rx[1], xn + 8);
          float ss = 0.0f;
#pragma unroll
          for (int i = 0; i < 16; ++i) ss += xn[i] * xn[i];
          const float rstd = rsqrtf(row_sum<LPR>(ss) * (1.0f / D) + p.eps);
          // read here, not kept over the rows: with both tensors' gains in
          // registers fewer waves fit
          asm volatile("" ::: "memory");
          float g[16];
          load8(gain + ch.a, g);
          load8(gain + ch.b, g + 8);
          float dot = 0.0f;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            xn[i] *= rstd;
            ac[i] += dz[i] * xn[i];
            dz[i] *= g[i];
            dot += dz[i] * xn[i];
          }
          const float mean = row_sum<LPR>(dot) * (1.0f / D);
#pragma unroll
          for (int i = 0; i < 16; ++i) dz[i] = rstd * (dz[i] - xn[i] * mean);
        }
        T* dst = reinterpret_cast<T*>(dx.p) + (t0 + tk) * dx.ts + h * dx.hs;
        store8(dst + ch.a, dz);
        store8(dst + ch.b, dz + 8);
      }
    };
    run(p.q, p.dqo, p.dq, gains[0], p.hq, p.fq, acc[0]);
    run(p.k, p.dko, p.dk, gains[1], p.hk, p.fk, acc[1]);
    rows += (TPW * p.hq + RPP - 1) / RPP;
    if (p.part && (rows >= kGainRows || t0 + step >= p.turn.n)) {
      rows = 0;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
#pragma unroll
        for (int o = LPR; o < kWave; o <<= 1)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[w][i] += __shfl_xor(acc[w][i], o);
        if (row == 0)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            double* to = &sums[wave][w][half ? ch.b : ch.a];
            double v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = to[i] + acc[w][8 * half + i];
#pragma unroll
            for (int i = 0; i < 8; ++i) to[i] = v[i];
          }
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[w][i] = 0.0f;
      }
    }
  }
  if (!p.part) return;
  __syncthreads();
  if (threadIdx.x < 2 * D) {
    const int w = threadIdx.x / D, c = threadIdx.x % D;
    double v = 0.0;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) v += sums[k][w][c];
    p.part[((int64_t)w * gridDim.x + blockIdx.x) * D + c] = (float)v;
  }
}

// dgamma[w][c] = sum over the workgroups' rows, in a fixed order and 64 bits: 64
// columns per workgroup, 16 streams of rows joined through LDS, eight loads in
// flight in each (past the end the last row again: behind a condition each load
// would be waited for by itself).
__global__ void __launch_bounds__(1024) qk_gain_kernel(const float* part, int blocks, int D, float* dgq, float* dgk) {
  __shared__ double sums[16][64];
  const int w = blockIdx.y, c = blockIdx.x * 64 + (threadIdx.x & 63), st = threadIdx.x >> 6;
  const float* p = part + (int64_t)w * blocks * D + c;
  double v[8] = {};
  for (int b = st; b < blocks; b += 16 * 8) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = p[(int64_t)min(b + 16 * i, blocks - 1) * D];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += b + 16 * i < blocks ? (double)x[i] : 0.0;
  }
  sums[st][threadIdx.x & 63] = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
  __syncthreads();
  if (st == 0) {
    double all = 0.0;
#pragma unroll
    for (int i = 0; i < 16; ++i) all += sums[i][threadIdx.x];
    float* out = w ? dgk : dgq;
    if (out) out[c] = (float)all;
  }
}

TurnParams turn_params(const HeadsDims& d, const HeadsWeights& w, int64_t n, const int32_t* positions) {
  TurnParams t;
  t.freqs = w.freqs;
  t.positions = positions;
  t.n = n;
  t.rot = d.rot;
  for (int i = 0; i < PF_MAX_AXES; ++i) t.axis_end[i] = d.axis_end[i];
  return t;
}

// Tokens below which a wave takes one pass: 2,000 x (16 + 16) x 64 6.5 us (7.0
// with a wave per token), an append of 500 x (16 + 16 + 16) x 64 5.8 (7.6), of
// 4,000 x (32 + 8 + 8) x 128 22.7 (20.8).
constexpr int64_t kFewTokens = 2048;

template <typename T, int D, bool PAIRS, Mode MODE>
hipError_t forward_on(QkParams p, int64_t n, const char* label, hipStream_t s) {
  constexpr bool APPEND = MODE != kTurn;
  constexpr int RPP = kWave / (D / 16);
  return timed(label, s, [&] {
    if (n < kFewTokens) {
      const int pk = (p.hk + RPP - 1) / RPP;
      p.fparts = FastDiv((p.q.p ? (p.hq + RPP - 1) / RPP : 0) + (APPEND ? 2 * pk : pk));
      const int64_t units = n * p.fparts.d;
      qk_few_kernel<T, D, PAIRS, MODE><<<dim3((unsigned)((units + kWaves - 1) / kWaves)), kThreads, 0, s>>>(p);
    } else {
      // One token per wave while its rows fill the passes to two thirds: its
      // loads start earliest (65,536 x (16 + 4) x 128: 127 us, with four tokens
      // 136). With few heads, whose passes would run part empty, four
      // (100,000 x (4 + 1) x 64: 34 us, with one 79).
      const int passes = (p.q.p ? (p.hq + RPP - 1) / RPP : 0) + (APPEND ? 2 : 1) * ((p.hk + RPP - 1) / RPP);
      const int rows = (p.q.p ? p.hq : 0) + (APPEND ? 2 : 1) * p.hk;
      const bool single = 2 * passes * RPP <= 3 * rows;
      const int per = kWaves * (single ? 1 : 4);
      const dim3 grid((unsigned)((n + per - 1) / per));
      if (single)
        qk_forward_kernel<T, D, PAIRS, 1, MODE><<<grid, kThreads, 0, s>>>(p);
      else
        qk_forward_kernel<T, D, PAIRS, 4, MODE><<<grid, kThreads, 0, s>>>(p);
    }
  });
}

template <Mode MODE>
hipError_t forward_any(const HeadsDims& d, const QkParams& p, int64_t n, const char* label, hipStream_t s) {
  if (d.esize == 2) {
    if (d.d == 64)
      return d.pairs_style ? forward_on<bf16, 64, true, MODE>(p, n, label, s) : forward_on<bf16, 64, false, MODE>(p, n, label, s);
    return d.pairs_style ? forward_on<bf16, 128, true, MODE>(p, n, label, s) : forward_on<bf16, 128, false, MODE>(p, n, label, s);
  }
  if (d.d == 64)
    return d.pairs_style ? forward_on<float, 64, true, MODE>(p, n, label, s) : forward_on<float, 64, false, MODE>(p, n, label, s);
  return d.pairs_style ? forward_on<float, 128, true, MODE>(p, n, label, s) : forward_on<float, 128, false, MODE>(p, n, label, s);
}

QkParams qk_params(const HeadsDims& d, const HeadsWeights& w, int64_t n, const int32_t* positions) {
  QkParams p{};
  p.turn = turn_params(d, w, n, positions);
  p.gamma_q = w.gamma_q;
  p.gamma_k = w.gamma_k;
  p.hq = d.hq;
  p.hk = d.hk;
  p.fq = FastDiv(d.hq);
  p.fk = FastDiv(d.hk);
  p.eps = d.eps;
  p.norm = d.norm;
  return p;
}

// Tokens per wave and step of the backward: 65,536 x (16 + 16) x 64 161 us (157
// with one, 164 with four), 100,000 x (16 + 1) x 64 141 (155, 140), 5,003 x (8 +
// 2) x 128 fp32 26.7 (28.4, 27.4). Some calls would gain from another number: 500 x
// (16 + 16) x 64 12.3 (10.8, 15.7), 20,000 x (32 + 8) x 128 135 (129, 130), 100,000 x
// (4 + 1) x 64 85 (126, 62).
constexpr int kBwdTokens = 2;
// Workgroups at most, three per CU: 65,536 x (16 + 16) x 64 161 us (165 with 512,
// 168 with 1,536), 100,000 x (16 + 1) x 64 141 (157, 148), 20,000 x (32 + 8) x 128
// 135 (129, 139).
constexpr int kBwdBlocks = 768;

int bwd_blocks(int64_t n) {
  const int64_t per = (int64_t)kWaves * kBwdTokens;
  const int64_t b = (n + per - 1) / per;
  return (int)(b < kBwdBlocks ? b : kBwdBlocks);
}

template <typename T, int D, bool PAIRS>
void backward_on(const QkBwdParams& p, int64_t n, hipStream_t s) {
  qk_backward_kernel<T, D, PAIRS, kBwdTokens><<<dim3((unsigned)bwd_blocks(n)), kThreads, 0, s>>>(p);
}

}  // namespace

hipError_t launch_qk_forward(const HeadsDims& d, const HeadsWeights& w, int64_t n, const Rows& q, const Rows& k,
                             const int32_t* positions, const Rows& q_out, const Rows& k_out, hipStream_t s) {
  QkParams p = qk_params(d, w, n, positions);
  p.q = q;
  p.k = k;
  p.q_out = q_out;
  p.k_out = k_out;
  return forward_any<kTurn>(d, p, n, "qk_norm_rope", s);
}

hipError_t launch_paged_append(const HeadsDims& d, const HeadsWeights& w, const PagedDims& c, int64_t n,
                               const int32_t* cu_tokens, const Rows& q, const Rows& k, const Rows& v,
                               const int32_t* positions, const Rows& q_out, hipStream_t s) {
  QkParams p = qk_params(d, w, n, positions);
  p.q = q;
  p.k = k;
  p.v = v;
  p.q_out = q_out;
  p.k_pages = c.k;
  p.v_pages = c.v;
  p.table = c.table;
  p.kv_len = c.kv_len;
  p.cu = cu_tokens;
  p.n_pages = c.n_pages;
  p.page_size = c.page_size;
  p.max_pages = c.max_pages;
  p.batch = c.batch;
  p.fpage = FastDiv(c.page_size);
  p.k_scale = c.k_scale;
  p.v_scale = c.v_scale;
  return c.k_scale ? forward_any<kAppend8>(d, p, n, "paged_quant_append", s) : forward_any<kAppend>(d, p, n, "paged_append", s);
}

size_t qk_backward_ws(const HeadsDims& d, int64_t n) {
  return d.norm ? (size_t)2 * bwd_blocks(n) * d.d * sizeof(float) : 0;
}

hipError_t launch_qk_backward(const HeadsDims& d, const HeadsWeights& w, int64_t n, const Rows& q, const Rows& k,
                              const int32_t* positions, const Rows& dq_out, const Rows& dk_out, const Rows& dq,
                              const Rows& dk, float* dgamma_q, float* dgamma_k, float* ws, hipStream_t s) {
  QkBwdParams p{};
  p.turn = turn_params(d, w, n, positions);
  p.q = q;
  p.k = k;
  p.dqo = dq_out;
  p.dko = dk_out;
  p.dq = dq;
  p.dk = dk;
  p.gamma_q = w.gamma_q;
  p.gamma_k = w.gamma_k;
  p.hq = d.hq;
  p.hk = d.hk;
  p.fq = FastDiv(d.hq);
  p.fk = FastDiv(d.hk);
  p.eps = d.eps;
  p.norm = d.norm;
  const bool gains = d.norm && (dgamma_q || dgamma_k);
  p.part = gains ? ws : nullptr;
  hipError_t e = n == 0 ? hipSuccess : timed("qk_backward", s, [&] {
    if (d.esize == 2) {
      if (d.d == 64) d.pairs_style ? backward_on<bf16, 64, true>(p, n, s) : backward_on<bf16, 64, false>(p, n, s);
      else d.pairs_style ? backward_on<bf16, 128, true>(p, n, s) : backward_on<bf16, 128, false>(p, n, s);
    } else {
      if (d.d == 64) d.pairs_style ? backward_on<float, 64, true>(p, n, s) : backward_on<float, 64, false>(p, n, s);
      else d.pairs_style ? backward_on<float, 128, true>(p, n, s) : backward_on<float, 128, false>(p, n, s);
    }
  });
  if (e != hipSuccess || !gains) return e;
  return timed("qk_gains", s, [&] {
    qk_gain_kernel<<<dim3(d.d / 64, 2), 1024, 0, s>>>(ws, bwd_blocks(n), d.d, dgamma_q, dgamma_k);
  });
}

}  // namespace pf
