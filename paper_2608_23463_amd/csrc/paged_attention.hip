// Attention of new tokens, one of every sequence or a prompt, over a paged
// cache.
//
//   o = sum_j softmax_j(scale q.k_j) v_j over the rows j that a token at row r
//   of its sequence sees: j <= r and, with a window, j > r - window or j < sinks.
//
// paged_attention_kernel: tokens one by one are bound by HBM, every visible
// row of K and V read once and 4 D flops per query head and row against 2 D
// elements of a group of heads. The 16 columns of its matrix instructions are
// the queries that share K and V: the heads of a group, and tokens after one
// another where a group has fewer than 16. A row is fetched once for all of
// them, and the multiplications cost next to nothing beside the loads, however
// few of the columns are used. A (block of columns, K/V head, slice of the
// rows) is a workgroup; its four waves take tiles of 16 * NB rows in turn and
// each keeps its own running maximum and sum.
//
// Nothing passes through LDS on the way. The order in which a matrix
// instruction's k index runs is free as long as both operands agree, and so is
// the order of its m index as long as the results are stored by it:
//  - scores: S^T[row, column] = K Q^T, lane (m, g) = (lane % 16, lane / 16)
//    holds 16 bytes of K row m. The result leaves lane (n, g) with rows
//    4 g .. 4 g + 3 of every block of 16 for column n.
//  - values: O^T[d, column] += V^T P^T takes those rows in just that order as
//    its k index, so the probabilities are an operand where they were computed.
//    Lane (m, g) loads VE neighbouring channels VE m .. of the same rows, and
//    the e-th instruction takes channel e of every lane: its m index stands for
//    channel VE m + e. In bf16 one permute joins two rows of a channel.
//
// Pages of 8 bits: the codes become the values of a wider cache (a power of two
// times e4m3 is exact in bf16 and in fp32) where an instruction takes them; the
// rest is the same. 32 sequences of 16,384 rows, 16 heads of 64, 209 us, 368 over
// bf16 pages.
#include <algorithm>

#include "paged.hpp"
#include "trace.hpp"

namespace pf {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kCols = 16;  // queries of a workgroup

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// f over the four lanes l % 16, 16 + l % 16, .., the same in each of them.
template <class F>
__device__ __forceinline__ float over_rows(float x, F&& f) {
  uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  uint32_t e = a[0], o = a[1];  // a bit cast takes the elements as values, not the pair's start
  u = __builtin_bit_cast(uint32_t, f(__builtin_bit_cast(float, e), __builtin_bit_cast(float, o)));
  const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  e = b[0], o = b[1];
  return f(__builtin_bit_cast(float, e), __builtin_bit_cast(float, o));
}

template <typename T, int D, bool B8>
struct Tile;

// bf16: tiles of two blocks, one k step of the value product.
template <int D>
struct Tile<bf16, D, false> {
  typedef bf16 Stored;
  static constexpr int NB = 2, KS = D / 32, VE = D / 16, JJ = 1, NO = VE;
  static constexpr int kPerCu = D == 64 ? 4 : 3;  // workgroups that fit a CU's registers
  u32x4 k[NB][KS];
  uint32_t v[NB][4][VE / 2];
  __device__ __forceinline__ void load_k(int b, const bf16* row, int g) {
#pragma unroll
    for (int s = 0; s < KS; ++s) k[b][s] = ld16(row + (4 * s + g) * 8);
  }
  __device__ __forceinline__ void load_v(int b, int r, const bf16* row, int m) {
    if constexpr (VE == 8) {
      const u32x4 t = ld16(row + VE * m);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[b][r][i] = t[i];
    } else {
      const u32x2 t = *reinterpret_cast<const u32x2*>(row + VE * m);
      v[b][r][0] = t[0];
      v[b][r][1] = t[1];
    }
  }
  __device__ __forceinline__ void zero_v(int b, int r) {
#pragma unroll
    for (int i = 0; i < VE / 2; ++i) v[b][r][i] = 0;
  }
  struct Query {
    bf16x8 f[KS];
    __device__ __forceinline__ void load(const bf16* row, int g, bool on) {
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        u32x4 t = {0u, 0u, 0u, 0u};
        if (on) t = ld16(row + (4 * s + g) * 8);
        f[s] = __builtin_bit_cast(bf16x8, t);
      }
    }
  };
  __device__ __forceinline__ f32x4 scores(int b, const Query& q) const {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < KS; ++i)
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[b][i]), q.f[i], s, 0, 0, 0);
    return s;
  }
  // The probabilities enter as two bf16 terms, p = hi + lo: one would round
  // each to 2^-8 of itself, two keep 2^-16, and the second product is hidden
  // behind the loads.
  __device__ __forceinline__ void values(const float* p, f32x4* o) const {
    bf16x8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      hi[i] = (bf16)p[i];
      lo[i] = (bf16)(p[i] - (float)hi[i]);
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      u32x4 a;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; r += 2)
          a[2 * b + r / 2] =
              __builtin_amdgcn_perm(v[b][r + 1][e / 2], v[b][r][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
      const bf16x8 f = __builtin_bit_cast(bf16x8, a);
      o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, hi, o[e], 0, 0, 0);
      o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, lo, o[e], 0, 0, 0);
    }
  }
};

// fp32: four rows per k step. Tiles of one block at D = 128 keep two tiles in
// the registers.
template <int D>
struct Tile<float, D, false> {
  typedef float Stored;
  static constexpr int NB = D == 64 ? 2 : 1, KS = D / 16, VE = 4, JJ = D / 64, NO = 4 * JJ;
  static constexpr int kPerCu = 3;
  f32x4 k[NB][KS];
  f32x4 v[NB][4][JJ];
  __device__ __forceinline__ void load_k(int b, const float* row, int g) {
#pragma unroll
    for (int s = 0; s < KS; ++s) k[b][s] = *reinterpret_cast<const f32x4*>(row + 16 * s + 4 * g);
  }
  __device__ __forceinline__ void load_v(int b, int r, const float* row, int m) {
#pragma unroll
    for (int j = 0; j < JJ; ++j) v[b][r][j] = *reinterpret_cast<const f32x4*>(row + 64 * j + 4 * m);
  }
  __device__ __forceinline__ void zero_v(int b, int r) {
#pragma unroll
    for (int j = 0; j < JJ; ++j) v[b][r][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  struct Query {
    f32x4 f[KS];
    __device__ __forceinline__ void load(const float* row, int g, bool on) {
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        f[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (on) f[s] = *reinterpret_cast<const f32x4*>(row + 16 * s + 4 * g);
      }
    }
  };
  __device__ __forceinline__ f32x4 scores(int b, const Query& q) const {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < KS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[b][i][e], q.f[i][e], s, 0, 0, 0);
    return s;
  }
  __device__ __forceinline__ void values(const float* p, f32x4* o) const {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < JJ; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            o[4 * j + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[b][r][j][e], p[4 * b + r], o[4 * j + e], 0, 0, 0);
  }
};

// What rows of 8 bits share: a lane holds 16 channels of a row of K per load,
// and of V the D / 16 neighbouring channels that it holds in bf16 too. Values are
// widened where they are used, times their row's power of two: exact in bf16 and
// fp32. Tiles of two blocks (48 sequences of up to 9,000 rows, 32 over 8 heads of
// 128, 105 us, with four 144: their registers do not fit a third workgroup; 1M rows
// 397 and 517; 32 sequences of 16,384 rows, 16 heads of 64, 209 and 209).
template <int D>
struct Raw8Tile {
  typedef uint8_t Stored;
  static constexpr int NB = 2, KL = D / 64, VE = D / 16, JJ = 1, NO = VE;
  u32x4 k[NB][KL];
  uint32_t v[NB][4][VE / 4];
  uint32_t ks[NB], vs[NB];  // words with the scale byte of the lane's row of K, of its four rows of V
  __device__ __forceinline__ void load_k(int b, const uint8_t* row, int g) {
#pragma unroll
    for (int s = 0; s < KL; ++s) k[b][s] = ld16(row + (4 * s + g) * 16);
  }
  __device__ __forceinline__ void load_v(int b, int r, const uint8_t* row, int m) {
    if constexpr (VE == 8) {
      const u32x2 t = *reinterpret_cast<const u32x2*>(row + VE * m);
      v[b][r][0] = t[0];
      v[b][r][1] = t[1];
    } else {
      v[b][r][0] = *reinterpret_cast<const uint32_t*>(row + VE * m);
    }
  }
  __device__ __forceinline__ void zero_v(int b, int r) {
#pragma unroll
    for (int i = 0; i < VE / 4; ++i) v[b][r][i] = 0;
    vs[b] = (vs[b] & ~(255u << (8 * r))) | 127u << (8 * r);
  }
  __device__ __forceinline__ float k_scale(int b) const { return scale_in(ks[b], (int)threadIdx.x); }
  __device__ __forceinline__ float v_scale(int b, int r) const { return scale_in(vs[b], r); }
};

template <int D>
struct Tile<bf16, D, true> : Raw8Tile<D> {
  typedef Raw8Tile<D> R;
  using R::k, R::v, R::ks, R::vs;
  static constexpr int kPerCu = D == 64 ? 4 : 3;
  struct Query {
    bf16x8 f[2 * R::KL];
    __device__ __forceinline__ void load(const bf16* row, int g, bool on) {
#pragma unroll
      for (int s = 0; s < 2 * R::KL; ++s) {
        u32x4 t = {0u, 0u, 0u, 0u};
        if (on) t = ld16(row + (4 * (s / 2) + g) * 16 + s % 2 * 8);
        f[s] = __builtin_bit_cast(bf16x8, t);
      }
    }
  };
  __device__ __forceinline__ f32x4 scores(int b, const Query& q) const {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    const float f = R::k_scale(b);
#pragma unroll
    for (int i = 0; i < 2 * R::KL; ++i) {
      u32x4 a;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const uint32_t raw = k[b][i / 2][i % 2 * 2 + w];
        a[2 * w] = bf16_pair_of<false>(raw, f);
        a[2 * w + 1] = bf16_pair_of<true>(raw, f);
      }
      s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), q.f[i], s, 0, 0, 0);
    }
    return s;
  }
  // (the probabilities in two bf16 terms, as for a bf16 cache)
  template <int E>  // channels E and E + 1 of the lane's
  __device__ __forceinline__ void pair(int c, const bf16x8& hi, const bf16x8& lo, f32x4* o) const {
    u32x4 a, z;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 4; r += 2) {
        const uint32_t x = bf16_pair_of<(E & 2) != 0>(v[2 * c + b][r][E / 4], R::v_scale(2 * c + b, r));
        const uint32_t y = bf16_pair_of<(E & 2) != 0>(v[2 * c + b][r + 1][E / 4], R::v_scale(2 * c + b, r + 1));
        a[2 * b + r / 2] = __builtin_amdgcn_perm(y, x, 0x05040100u);
        z[2 * b + r / 2] = __builtin_amdgcn_perm(y, x, 0x07060302u);
      }
    const bf16x8 f0 = __builtin_bit_cast(bf16x8, a), f1 = __builtin_bit_cast(bf16x8, z);
    o[E] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f0, hi, o[E], 0, 0, 0);
    o[E + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f1, hi, o[E + 1], 0, 0, 0);
    o[E] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f0, lo, o[E], 0, 0, 0);
    o[E + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f1, lo, o[E + 1], 0, 0, 0);
  }
  __device__ __forceinline__ void values(const float* p, f32x4* o) const {
#pragma unroll
    for (int c = 0; c < R::NB / 2; ++c) {
      bf16x8 hi, lo;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        hi[i] = (bf16)p[8 * c + i];
        lo[i] = (bf16)(p[8 * c + i] - (float)hi[i]);
      }
      pair<0>(c, hi, lo, o);
      pair<2>(c, hi, lo, o);
      if constexpr (R::VE == 8) {
        pair<4>(c, hi, lo, o);
        pair<6>(c, hi, lo, o);
      }
    }
  }
};

template <int D>
struct Tile<float, D, true> : Raw8Tile<D> {
  typedef Raw8Tile<D> R;
  using R::k, R::v, R::ks, R::vs;
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  static constexpr int kPerCu = 3;
  struct Query {
    f32x4 f[4 * R::KL];
    __device__ __forceinline__ void load(const float* row, int g, bool on) {
#pragma unroll
      for (int s = 0; s < 4 * R::KL; ++s) {
        f[s] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (on) f[s] = *reinterpret_cast<const f32x4*>(row + (4 * (s / 4) + g) * 16 + s % 4 * 4);
      }
    }
  };
  __device__ __forceinline__ f32x4 scores(int b, const Query& q) const {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    const float f = R::k_scale(b);
#pragma unroll
    for (int i = 0; i < 4 * R::KL; ++i) {
      const uint32_t raw = k[b][i / 4][i % 4];
      const f32x2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(raw, f, false);
      const f32x2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(raw, f, true);
      s = __builtin_amdgcn_mfma_f32_16x16x4f32(x[0], q.f[i][0], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_16x16x4f32(x[1], q.f[i][1], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_16x16x4f32(y[0], q.f[i][2], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_16x16x4f32(y[1], q.f[i][3], s, 0, 0, 0);
    }
    return s;
  }
  __device__ __forceinline__ void values(const float* p, f32x4* o) const {
#pragma unroll
    for (int b = 0; b < R::NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float f = R::v_scale(b, r), w = p[4 * b + r];
#pragma unroll
        for (int i = 0; i < R::VE / 4; ++i) {
          const f32x2 x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v[b][r][i], f, false);
          const f32x2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v[b][r][i], f, true);
          o[4 * i] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[0], w, o[4 * i], 0, 0, 0);
          o[4 * i + 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[1], w, o[4 * i + 1], 0, 0, 0);
          o[4 * i + 2] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[0], w, o[4 * i + 2], 0, 0, 0);
          o[4 * i + 3] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[1], w, o[4 * i + 3], 0, 0, 0);
        }
      }
  }
};

template <typename T, int D, bool B8>
__global__ void __launch_bounds__(kThreads, (Tile<T, D, B8>::kPerCu)) paged_attention_kernel(PagedParams p) {
  typedef Tile<T, D, B8> Tl;
  typedef typename Tl::Stored Stored;
  constexpr int NB = Tl::NB, TR = NB * kBlock;
  __shared__ __attribute__((aligned(16))) float so[kWaves][kCols][D + 4];  // columns four banks apart
  __shared__ float sm[kWaves][kCols], sl[kWaves][kCols];

  // Slices fastest, then K/V heads, then blocks of columns; every group begins
  // at another slice. Workgroups go to the XCDs in turn, and short sequences
  // fill their first slices only: with eight slices in order most of the rows
  // would go to the first XCDs (64 sequences of up to 9,000 rows, 8 K/V heads of
  // 128: 243 us, and 210 so; with other numbers of slices no difference).
  const int id = (int)blockIdx.x, up = p.fslices.div(id);
  int slice = id - up * p.slices + up - p.fslices.div(up) * p.slices;
  slice -= slice >= p.slices ? p.slices : 0;
  const int blk = p.fhk.div(up), hk = up - blk * p.hk;
  const int s = sequence_of_block<kCols>(p, blk);
  Sequence sq;
  sq.set(p, s);
  const int x0 = (blk - first_block<kCols>(p, s)) * kCols;
  if (sq.seq < 0 || x0 < 0 || x0 >= sq.cols) return;
  const int cols = min(sq.cols - x0, kCols);
  const Sight sight(p, sq, x0, cols, TR);
  const int per = sight.per_slice(p);
  const int first = slice * per, last = min(first + per, sight.tiles);
  if (first >= last && p.slices > 1) return;  // no rows: the join does not read this slice

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave;
  const int m = lane % 16, g = lane / 16;

  // the lane's column: its query, and the rows lo < j <= row that it sees (the
  // table may end before its own)
  const int mx0 = x0 + (m < cols ? m : 0), tok = p.fgroup.div(mx0);
  const int own = m < cols ? max(sq.row0 + tok, -1) : -1, lo = own - p.window, row = min(own, sight.last);
  typename Tl::Query q;
  q.load(reinterpret_cast<const T*>(p.q) + (sq.t0 + tok) * p.q_ts + (int64_t)(hk * p.group + mx0 - tok * p.group) * p.q_hs,
         g, m < cols);

  const int32_t* table = p.table + (int64_t)s * p.max_pages;
  const int64_t page_rows = (int64_t)p.hk * p.page_size;
  const Stored* kp = reinterpret_cast<const Stored*>(p.k);
  const Stored* vp = reinterpret_cast<const Stored*>(p.v);

  // A tile's blocks: their table entries as they are, and their first slots.
  struct Place {
    int id[NB], slot[NB];
  };
  f32x4 o[Tl::NO];
#pragma unroll
  for (int i = 0; i < Tl::NO; ++i) o[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float mx = -INFINITY, sum = 0.0f;

  auto place = [&](int i) {
    Place w;
    const int blk = sight.tile(min(i, last - 1)) * NB;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int pg = min(p.page_blocks.div(blk + b), p.max_pages - 1);
      w.slot[b] = (blk + b - p.page_blocks.div(blk + b) * p.page_blocks.d) * kBlock;
      w.id[b] = table[pg];
    }
    return w;
  };
  // An entry that is no page reads page 0 instead, whose rows exist.
  auto is_page = [&](int id) { return (unsigned)id < (unsigned)p.n_pages; };
  auto base = [&](const Place& w, int b) {
    return (is_page(w.id[b]) ? w.id[b] : 0) * page_rows + (int64_t)hk * p.page_size + w.slot[b];
  };
  Tl t;
  auto fetch_k = [&](const Place& w) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      t.load_k(b, kp + base(w, b) * D + m * D, g);
      if constexpr (B8) t.ks[b] = *reinterpret_cast<const uint32_t*>(p.k_scale + base(w, b) + (m & ~3));
    }
  };
  auto fetch_v = [&](const Place& w) {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int r = 0; r < 4; ++r) t.load_v(b, r, vp + base(w, b) * D + (4 * g + r) * D, m);
      if constexpr (B8) t.vs[b] = *reinterpret_cast<const uint32_t*>(p.v_scale + base(w, b) + 4 * g);
    }
  };

  // The next tile's K is on its way from the moment the scores are formed and
  // its V from the products on, into the registers these leave; table entries
  // come a tile before that. Past the slice's end its last tile is fetched
  // again (a cache hit): behind a condition the compiler would have to wait for
  // every load at the next use.
  int i = first + wave;
  if (i < last) {
    Place w = place(i), next = place(i + kWaves);
    fetch_k(w);
    fetch_v(w);
    while (true) {
      const int row0 = sight.tile(i) * TR;
      f32x4 sc[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) sc[b] = t.scores(b, q);
      fetch_k(next);
      const Place after = place(i + 2 * kWaves);
      float pr[4 * NB];
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) pr[4 * b + r] = sc[b][r] * p.scale_log2;
      bool whole = row0 + TR - 1 <= min(sight.first, sight.last) && (row0 > sight.top - p.window || row0 + TR <= p.sinks);
#pragma unroll
      for (int b = 0; b < NB; ++b) whole = whole && is_page(w.id[b]);
      if (!whole) {
        // what is not seen counts for nothing, whatever its bits are
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int j = row0 + b * kBlock + 4 * g + r;
            const bool none = !is_page(w.id[b]);
            if (none || j > row || (j <= lo && j >= p.sinks)) pr[4 * b + r] = -INFINITY;
            if (none || j > sight.last || (j <= sight.first - p.window && j >= p.sinks)) t.zero_v(b, r);
          }
      }
      float top = pr[0];
#pragma unroll
      for (int r = 1; r < 4 * NB; ++r) top = fmaxf(top, pr[r]);
      top = over_rows(top, [](float a, float b) { return fmaxf(a, b); });
      const float now = fmaxf(mx, top);
      const float ref = now == -INFINITY ? 0.0f : now;
      const float back = fast_exp2(mx - ref);
      mx = now;
      float add = 0.0f;
#pragma unroll
      for (int r = 0; r < 4 * NB; ++r) {
        pr[r] = fast_exp2(pr[r] - ref);
        add += pr[r];
      }
      sum = sum * back + add;
#pragma unroll
      for (int k = 0; k < Tl::NO; ++k) o[k] *= back;
      t.values(pr, o);
      fetch_v(next);
      i += kWaves;
      if (i >= last) break;
      w = next;
      next = after;
    }
  }

  // join the four waves
  sum = over_rows(sum, [](float a, float b) { return a + b; });
  if (g == 0) {
    sm[wave][m] = mx;
    sl[wave][m] = sum;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int j = 0; j < Tl::JJ; ++j)
#pragma unroll
      for (int e = 0; e < Tl::VE; ++e) so[wave][m][64 * j + Tl::VE * (4 * g + r) + e] = o[j * Tl::VE + e][r];
  __syncthreads();
  constexpr int C4 = D / 4;
  for (int at = threadIdx.x; at < cols * C4; at += kThreads) {
    const int h = at / C4, c = (at % C4) * 4;
    float top = sm[0][h];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sm[w][h]);
    const float ref = top == -INFINITY ? 0.0f : top;
    float l = 0.0f;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = fast_exp2(sm[w][h] - ref);
      l += f * sl[w][h];
      acc += f * *reinterpret_cast<const f32x4*>(&so[w][h][c]);
    }
    const int tk = p.fgroup.div(x0 + h);
    const int64_t orow = (int64_t)(sq.t0 + tk) * p.hq + hk * p.group + (x0 + h - tk * p.group);
    if (p.slices == 1) {
      const float inv = l > 0.0f ? 1.0f / l : l;  // nothing seen: zero (and a NaN stays one)
      float res[4] = {acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
      store4(reinterpret_cast<T*>(p.out) + orow * D + c, res);
      if (p.lse && c == 0) p.lse[orow] = (top + __log2f(l)) * 0.69314718055994530942f;
    } else {
      *reinterpret_cast<f32x4*>(p.part_o + (orow * p.slices + slice) * D + c) = acc;
      if (c == 0) p.part_ml[orow * p.slices + slice] = make_float2(top, l);
    }
  }
}

// The slices that hold a (token, head)'s partial results, 0 .. live - 1 of its
// row; -1: a token behind the last sequence.
__device__ __forceinline__ int live_slices(const PagedParams& p, int row) {
  const int tok = row / p.hq, head = (row - tok * p.hq) % p.group;
  const int s0 = p.cu ? find_run(p.batch, [&](int c) { return p.cu[c]; }, tok) : tok;
  Sequence sq;
  sq.set(p, s0);
  const int x = (tok - sq.t0) * p.group + head;
  if (sq.seq < 0 || x < 0 || x >= sq.cols) return -1;
  const int x0 = x & -p.cols;  // its block's first column
  const Sight sight(p, sq, x0, min(sq.cols - x0, p.cols), p.tile_rows);
  const int per = sight.per_slice(p);
  return (sight.tiles + per - 1) / per;
}

// Joins the slices of a row in a fixed order, ROWS rows per workgroup: four of
// few slices, a wave each, or one of many. A lane takes four channels; the
// streams of slices are joined through LDS.
template <typename T, int D, int ROWS>
__global__ void __launch_bounds__(kThreads) paged_join_kernel(PagedParams p) {
  constexpr int C4 = D / 4, NS = kThreads / ROWS / C4;  // streams of a row
  __shared__ float so[ROWS][NS][D];
  __shared__ float sl[ROWS][NS];
  const int lane = threadIdx.x % kWave, at = threadIdx.x % (kThreads / ROWS), r = threadIdx.x / (kThreads / ROWS);
  const int row = __builtin_amdgcn_readfirstlane((int)blockIdx.x * ROWS + r);
  const int live = row < p.n_tokens * p.hq ? live_slices(p, row) : -1;
  const float2* ml = p.part_ml + (int64_t)row * p.slices;
  const float* po = p.part_o + (int64_t)row * p.slices * D;
  float top = -INFINITY;
  for (int s = lane; s < live; s += kWave) top = fmaxf(top, ml[s].x);
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
  const float ref = top == -INFINITY ? 0.0f : top;
  const int c = (at % C4) * 4, st = at / C4;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  float l = 0.0f;
  for (int s = st; s < live; s += NS) {
    const float2 x = ml[s];
    const float f = fast_exp2(x.x - ref);
    l += f * x.y;
    acc += f * *reinterpret_cast<const f32x4*>(po + (int64_t)s * D + c);
  }
  *reinterpret_cast<f32x4*>(&so[r][st][c]) = acc;
  if (c == 0) sl[r][st] = l;
  __syncthreads();
  if (st == 0 && live >= 0) {
    l = 0.0f;
    acc = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      l += sl[r][s];
      acc += *reinterpret_cast<const f32x4*>(&so[r][s][c]);
    }
    const float inv = l > 0.0f ? 1.0f / l : l;
    float res[4] = {acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv};
    store4(reinterpret_cast<T*>(p.out) + (int64_t)row * D + c, res);
    if (p.lse && c == 0) p.lse[row] = (top + __log2f(l)) * 0.69314718055994530942f;
  }
}

// Slices up to which a wave joins a row: the attention of 16 prompts of up to 40
// tokens, 32 heads, 3 slices takes 33 us (49 with a workgroup per row), of one
// token of 32 heads in 15 slices 13.2 us with a workgroup (14.5), in 64 21.8 (27.6).
constexpr int kFewSlices = 8;

template <typename T, int D, Source FROM>
hipError_t attention_on(const PagedParams& p, const PagedPlan& pl, hipStream_t s) {
  const bool tr = trace_on();
  hipError_t e;
  if (tr)
    trace_begin(FROM == kPages ? (pl.prompt ? "paged_prompt" : "paged_attention")
                               : (pl.prompt ? "paged_quant_prompt" : "paged_quant_attention"), s);
  if (pl.prompt)
    launch_prompt(p, D, FROM, pl.groups, s);
  else
    paged_attention_kernel<T, D, FROM == kPages8><<<dim3((unsigned)(pl.groups * pl.slices)), kThreads, 0, s>>>(p);
  e = hipGetLastError();
  if (tr) trace_end(s);
  if (e != hipSuccess || p.slices == 1) return e;
  if (tr) trace_begin("paged_join", s);
  const unsigned rows = (unsigned)(p.n_tokens * p.hq);
  if (p.slices <= kFewSlices)
    paged_join_kernel<T, D, 4><<<dim3((rows + 3) / 4), kThreads, 0, s>>>(p);
  else
    paged_join_kernel<T, D, 1><<<dim3(rows), kThreads, 0, s>>>(p);
  e = hipGetLastError();
  if (tr) trace_end(s);
  return e;
}

// New tokens of a sequence from which the prompt kernel runs. With a head per
// K/V head that is where the two kernels meet: 16 sequences behind 1,000 rows, 8
// heads of 128, 16 tokens 17.4 us (23.4 with the prompt kernel), 31 28.8 (24.6),
// 32 24.2 (28.2 without it), 64 30.4 (40.0). Heads that share K and V fill the
// prompt kernel's columns earlier, so it would be ahead from 8 tokens on with 4
// heads each (25.8, and 27.8) and from 4 on with 8 (25.6, and 27.9), but it rounds
// the weights to one bf16 term: fewer tokens keep the two terms.
constexpr int64_t kPromptTokens = 32;

}  // namespace

PagedPlan paged_plan(const HeadsDims& d, int batch, int64_t n_tokens, bool ragged, int64_t max_new, int64_t max_kv_len,
                     int64_t window, int64_t sinks, bool bits8) {
  PagedPlan pl;
  pl.prompt = d.esize == 2 && ragged && max_new >= kPromptTokens;
  pl.cols = pl.prompt ? 128 : kCols;
  pl.tile_rows = pl.prompt ? 64 : kBlock * (!bits8 && d.esize == 4 && d.d == 128 ? 1 : 2);
  window = std::min<int64_t>(window, INT32_MAX);
  sinks = std::min<int64_t>(sinks, INT32_MAX);
  max_new = std::min<int64_t>(max_new, n_tokens);
  int64_t rows = std::min<int64_t>(max_kv_len, INT32_MAX);
  if (window > 0) rows = std::min(rows, window + sinks + std::min<int64_t>(max_new, pl.cols) + 2 * pl.tile_rows);
  const int64_t tiles = std::max<int64_t>(1, (rows + pl.tile_rows - 1) / pl.tile_rows);
  pl.groups = col_blocks(pl.cols, d.hq / d.hk, ragged ? n_tokens : -1, batch) * d.hk;
  // Few groups: two workgroups per CU, if that leaves each enough tiles (fewer
  // and longer slices stream better: 8 K/V heads of 128 over 1M rows take 725 us
  // in 512 workgroups and 753 in 2,048, 4 sequences of up to 60,000 fp32 rows over 2
  // heads 52 and 58; 16 heads of 64 over 1,000 rows 10.0 us in slices of 8 tiles,
  // 11.2 of 16, 9.7 of 4, which costs calls of few rows a join). Where the groups
  // fill the chip by themselves, cuts only even out sequences of different
  // lengths, and short slices cost more than that gives: 48 sequences of up to
  // 9,000 rows, 8 K/V heads of 128, 201 us whole, 179 in two slices, 160 in slices
  // of 48 tiles, 158 of 24, 156 of 16; all of 4,100 rows 158, 150, 150, 155 and
  // 159; 64 sequences of up to 1,000 rows, 16 heads of 64, 29 us whole or of 24,
  // 43 of 16.
  const bool filled = pl.groups >= 256;
  const int64_t want = pl.prompt || !filled ? 512 : 4096;
  pl.min_tiles = pl.prompt ? 4 : pl.groups < 32 ? 8 : filled ? 24 : 16;
  int64_t s = std::min<int64_t>((want + pl.groups - 1) / pl.groups, tiles / pl.min_tiles);
  s = std::max<int64_t>(1, std::min<int64_t>(s, kMaxSlices));
  pl.slices = (int)s;
  pl.bytes = s == 1 ? 0 : (size_t)n_tokens * d.hq * s * (d.d * sizeof(float) + sizeof(float2));
  pl.bytes = (pl.bytes + 255) / 256 * 256;
  return pl;
}

hipError_t launch_paged_attention(const HeadsDims& d, const PagedDims& c, const PagedPlan& pl, int64_t n_tokens,
                                  const int32_t* cu_tokens, const Rows& q, float scale, int64_t window, int64_t sinks,
                                  void* out, float* lse, char* ws, hipStream_t s) {
  PagedParams p{};
  p.q = q.p;
  p.q_ts = q.ts;
  p.q_hs = q.hs;
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
  p.n_tokens = (int)n_tokens;
  p.page_blocks = FastDiv(c.page_size / kBlock);
  p.hq = d.hq;
  p.hk = d.hk;
  p.group = d.hq / d.hk;
  p.cols = pl.cols;
  p.tile_rows = pl.tile_rows;
  p.slices = pl.slices;
  p.fmin_tiles = FastDiv(pl.min_tiles);
  p.fslices = FastDiv(pl.slices);
  p.fhk = FastDiv(d.hk);
  p.fgroup = FastDiv(p.group);
  p.fblocks = FastDiv((p.group + kCols - 1) / kCols);
  p.window = window > 0 ? (int)std::min<int64_t>(window, INT32_MAX) : INT32_MAX;
  p.sinks = (int)std::min<int64_t>(sinks, INT32_MAX);
  p.scale_log2 = scale * 1.4426950408889634f;
  p.out = out;
  p.lse = lse;
  p.part_o = reinterpret_cast<float*>(ws);
  p.part_ml = reinterpret_cast<float2*>(ws + (size_t)n_tokens * d.hq * pl.slices * d.d * sizeof(float));
  if (c.k_scale) {
    if (d.esize == 2) return d.d == 64 ? attention_on<bf16, 64, kPages8>(p, pl, s) : attention_on<bf16, 128, kPages8>(p, pl, s);
    return d.d == 64 ? attention_on<float, 64, kPages8>(p, pl, s) : attention_on<float, 128, kPages8>(p, pl, s);
  }
  if (d.esize == 2) return d.d == 64 ? attention_on<bf16, 64, kPages>(p, pl, s) : attention_on<bf16, 128, kPages>(p, pl, s);
  return d.d == 64 ? attention_on<float, 64, kPages>(p, pl, s) : attention_on<float, 128, kPages>(p, pl, s);
}

}  // namespace pf
