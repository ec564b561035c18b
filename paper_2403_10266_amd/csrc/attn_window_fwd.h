// Kernels of attention with a window and first tokens that stay visible, over rows of a
// tensor (attn_window.hip) and over pages of a cache (attn_paged.hip):
//   o_i = sum_j softmax_j(scale q_i . k_j) v_j  over the keys that query i sees.
//
// One pass over the keys with the running maximum and sum of the softmax; both products
// on the matrix cores, computed transposed (keys on rows, queries on columns): a lane
// owns one column, so the statistics are per-lane scalars and the probabilities are the
// next product's operand as they stand.  Columns are the (query, head) pairs of one
// key/value head's group, heads fastest: a tile of keys serves the whole group, and a
// block of columns spans few positions, so that a narrow window leaves few keys.
// Only the tiles that a block of columns sees are visited, and only those on the
// window's edges are masked.
//
// Keys come in groups of 16 rows, each loaded by one wave, so that a group's page, its
// place and its scale are scalars.  e4m3 rows become bf16 on their way into LDS, exactly
// (the scales are powers of two); from there on there is one kernel for all caches.
#pragma once

#include <algorithm>

#include "attn_window.h"

namespace dsp {
namespace {

struct FwdParams {
  const void* q;
  const void* k;
  const void* v;
  void* o;
  float* lse;
  float* part;       // split keys: the columns' references, sums and rows of each work-group
  const int32_t* q_pos;
  const int32_t* kv_len;
  const int32_t* q_start;
  const int32_t* table;
  const float* k_scale;
  const float* v_scale;
  int64_t qs[3], ks[3], os[3];
  Window win;
  uint32_t X, H, Hkv, Lq, Lk, D;
  Divisor grp;       // heads of a key/value head's group
  uint32_t N, T, n_pages, max_pages, shift;   // pages
  Order order;       // many columns, rows of a tensor
  uint32_t n_blk;    // many columns, pages: blocks in all
  uint32_t few_cols; // many columns: units of at most so many are left to the other form
  uint32_t pieces, n_split, cblk;   // few columns: units times splits, blocks of 32 columns
  uint32_t block_cols;              // of a block, at most
  float c;           // scale * log2(e)
  bool vec;
};

// A sequence (or a unit of B X) and one of its key/value heads.
template <typename T, typename S, bool PAGED>
struct Unit {
  const T* q;        // column (query i, head hh of the group): q + i q_row + hh D
  T* o;
  float* lse;        // + i lse_i + hh lse_h
  int64_t q_row, o_row, lse_i, lse_h;
  int64_t p0;        // position of query 0
  int32_t nq, len;
  Source<S, PAGED> src;
};
template <typename T, typename S>
__device__ __forceinline__ Unit<T, S, false> unit(const FwdParams& p, uint32_t bx, uint32_t e, Unit<T, S, false>*) {
  Unit<T, S, false> u;
  const uint32_t b = bx / p.X, x = bx - b * p.X, h0 = e * p.grp.d;
  u.q = static_cast<const T*>(p.q) + (int64_t)b * p.qs[0] + (int64_t)x * p.qs[1] + (int64_t)h0 * p.D;
  u.o = static_cast<T*>(p.o) + (int64_t)b * p.os[0] + (int64_t)x * p.os[1] + (int64_t)h0 * p.D;
  u.lse = p.lse ? p.lse + ((uint64_t)bx * p.H + h0) * p.Lq : nullptr;
  u.q_row = p.qs[2], u.o_row = p.os[2], u.lse_i = 1, u.lse_h = p.Lq;
  u.p0 = first_position(p.q_pos, b);
  u.nq = (int32_t)p.Lq;
  u.len = (int32_t)length(p.kv_len, b, p.Lk);
  const int64_t at = (int64_t)b * p.ks[0] + (int64_t)x * p.ks[1] + (int64_t)e * p.D;
  u.src.k = static_cast<const S*>(p.k) + at;
  u.src.v = static_cast<const S*>(p.v) + at;
  u.src.row = p.ks[2];
  u.src.row_bytes = (uint32_t)p.ks[2] * (uint32_t)sizeof(S);
  return u;
}
template <typename T, typename S>
__device__ __forceinline__ Unit<T, S, true> unit(const FwdParams& p, uint32_t n, uint32_t e, Unit<T, S, true>*) {
  Unit<T, S, true> u;
  const Rows r = new_rows(p.q_start, n, p.T);
  const uint32_t h0 = e * p.grp.d;
  u.q = static_cast<const T*>(p.q) + (int64_t)r.first * p.qs[2] + (int64_t)h0 * p.D;
  u.o = static_cast<T*>(p.o) + (int64_t)r.first * p.os[2] + (int64_t)h0 * p.D;
  u.lse = p.lse ? p.lse + (uint64_t)r.first * p.H + h0 : nullptr;
  u.q_row = p.qs[2], u.o_row = p.os[2], u.lse_i = p.H, u.lse_h = 1;
  u.p0 = (int64_t)p.kv_len[n] - r.n;
  u.nq = min(r.n, (int32_t)p.Lq);
  u.len = (int32_t)length(p.kv_len, n, p.Lk);
  u.src.k = static_cast<const S*>(p.k) + (int64_t)e * p.ks[2];
  u.src.v = static_cast<const S*>(p.v) + (int64_t)e * p.ks[2];
  u.src.table = p.table + (uint64_t)n * p.max_pages;
  u.src.ks = p.k_scale ? p.k_scale + e : nullptr;
  u.src.vs = p.v_scale ? p.v_scale + e : nullptr;
  u.src.page = p.ks[0], u.src.row = p.ks[1];
  u.src.row_bytes = (uint32_t)p.ks[1] * (uint32_t)sizeof(S);
  u.src.n_pages = p.n_pages, u.src.n_heads = p.Hkv, u.src.shift = p.shift;
  return u;
}

// Clamps of this wave leave a NaN as it is (bit 8 of the mode register; set, they make it 0):
// a probability that fast() cuts with its exponential's clamp stays NaN.  A minimum for it
// costs 4% (8192 causal tokens 156 and 162 us).
__device__ __forceinline__ void keep_nan() {
  asm volatile("s_setreg_imm32_b32 hwreg(HW_REG_MODE, 8, 1), 0");
}

// The softmax of QT blocks of 32 columns over NKT blocks of 32 keys at a time, less a
// reference of each column (exp2 units).
//  * exact(): takes the tile's maxima and moves the references to them.
//  * fast() (LAZY, bf16: a reference off the maximum costs an exponent's last bits, fp32 results
//    1.3e-6 of their value at 64 off where exact() gives 2e-7): the references stay, kRoom above the maximum of the
//    tiles that set them, and probabilities are cut at 1, so that nothing stands between the exponentials and the
//    product with v.  A score above its reference shows afterwards, as a sum of a half or
//    more (probabilities below it add up to less, or are so many that the reference had better
//    move too); then, rarely, fix() moves the reference and adds to the tile's probabilities
//    what the cut took from them.
// The room bounds the values: sums are of 2^-kRoom v, and with 16 those of any v above 2^-110 keep
// fp32's normal range (with 64 above 2^-62 only), at the price of a fix for every 16 binary steps
// that the scores climb.
// Sums are those of the fp32 probabilities (of the rounded ones, which a column of ones in v
// would give with the product, the log-sum-exp would be off by their roundings: 9 times its
// bound at 64 keys).
template <typename T, int DC, int QT, int NKT, bool LAZY>
struct Softmax {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  static constexpr float kRoom = LAZY ? 16.0f : 0.0f;
  ColAcc<T, DC> o[QT];
  float ref[QT], sum[QT];   // the sum of this lane's keys
  bool set;                 // every column that sees a key has a reference

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int j = 0; j < QT; ++j) {
      o[j].zero();
      ref[j] = -INFINITY;
      sum[j] = 0.0f;
    }
    set = false;
  }
  // a column's sum over all keys
  __device__ __forceinline__ float total(int j) const { return sum[j] + swap_halves(sum[j]); }

  // Scores of the tile from key0 in exp2 units, less `minus`.  mask: some column does not
  // see some key of it; gone: bits of its groups of 16 keys that are not there.
  template <typename KF, typename Q>
  static __device__ __forceinline__ void scores(floatx16 (&s)[NKT][QT], const KF& kf, const Q& qf, int32_t key0, bool mask,
                                                uint32_t gone, float c, const Seen (&cols)[QT],
                                                const float (&minus)[QT], int lane) {
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int j = 0; j < QT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kt][j][r] = 0.0f;
#pragma unroll
    for (int st = 0; st < G::NS; ++st)
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) {
        const auto a = kf(kt, st);
#pragma unroll
        for (int j = 0; j < QT; ++j) s[kt][j] = M::mma(a, qf[j][st], s[kt][j]);
      }
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt) finish(s[kt], kt, key0, mask, gone, c, cols, minus, lane);
  }
  static __device__ __forceinline__ void scale(floatx16 (&s)[QT], float c, const float (&minus)[QT]) {
#pragma unroll
    for (int j = 0; j < QT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[j][r] = fmaf(s[j][r], c, -minus[j]);
  }
  // products of block kt made scores
  static __device__ __forceinline__ void finish(floatx16 (&s)[QT], int kt, int32_t key0, bool mask, uint32_t gone, float c,
                                                const Seen (&cols)[QT], const float (&minus)[QT], int lane) {
    scale(s, c, minus);
    if (!mask) return;
#pragma unroll
    for (int j = 0; j < QT; ++j) {
      uint32_t bits = block_bits(cols[j], kt, key0, gone) >> (4 * (lane >> 5));
      // formed again here: kept from fast() to fix() they take 32 registers, which spill (3.7 times the time)
      asm volatile("" : "+v"(bits));
#pragma unroll
      for (int r = 0; r < 16; ++r) s[j][r] = mask_bit(s[j][r], bits, 8 * (r / 4) + r % 4);
    }
  }
  // bit i: whether the column sees key key0 + 32 kt + i
  static __device__ __forceinline__ uint32_t block_bits(const Seen& col, int kt, int32_t key0, uint32_t gone) {
    const uint32_t lost = (gone >> (2 * kt) & 1 ? 0xFFFFu : 0u) | (gone >> (2 * kt) & 2 ? 0xFFFF0000u : 0u);
    return seen_bits(col, key0 + 32 * kt) & ~lost;
  }
  __device__ __forceinline__ void product(const T* vl, const ColB<T> (&pf)[NKT][QT], int lane) {
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int j = 0; j < QT; ++j) o[j].add(vl, 32 * kt, lane, pf[kt][j]);
  }

  // One tile: kf(kt, st) the fragments of its keys, vl its values in LDS.
  template <typename KF, typename Q>
  __device__ __forceinline__ void exact(const KF& kf, const T* vl, const Q& qf, int32_t key0, bool mask, uint32_t gone,
                                        float c, const Seen (&cols)[QT], int lane) {
    floatx16 s[NKT][QT];
    float zero[QT];
#pragma unroll
    for (int j = 0; j < QT; ++j) zero[j] = 0.0f;
    scores(s, kf, qf, key0, mask, gone, c, cols, zero, lane);
    ColB<T> pf[NKT][QT];
    bool all = true;
#pragma unroll
    for (int j = 0; j < QT; ++j) {
      float m = s[0][j][0];
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) m = fmaxf(m, s[kt][j][r]);
      m = fmaxf(fmaxf(m, swap_halves(m)) + kRoom, ref[j]);
      const float f = ref[j] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ref[j] - m);
      sum[j] *= f;
      o[j].scale(f, lane);
      ref[j] = m;
      const float by = m == -INFINITY ? 0.0f : m;   // nothing yet: every score is -inf
      float add = 0.0f;
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = __builtin_amdgcn_exp2f(s[kt][j][r] - by);
          add += e;
          pf[kt][j].set(r, e);
        }
      sum[j] += add;
      if constexpr (LAZY) {
        // a column that is not finite has all it will have: the others' way is the same
        add += swap_halves(add);
        all &= m != -INFINITY || !sees_any(cols[j]) || add != add;
      }
    }
    if constexpr (LAZY) set = __all(all);
    product(vl, pf, lane);
  }

  // Whether some column's reference has to move.  The operands of a block's products are
  // read from LDS ahead of them, a block of 32 keys at a time, in the order written here (the
  // fences keep it): left to itself the compiler reads each right before its MFMA, and a
  // wave waits for LDS sixteen times a tile.
  template <typename KF, typename Q>
  __device__ __forceinline__ bool fast(const KF& kf, const T* vl, const Q& qf, int32_t key0, bool mask, uint32_t gone,
                                       float c, const Seen (&cols)[QT], int lane) {
    float by[QT];
#pragma unroll
    for (int j = 0; j < QT; ++j) by[j] = ref[j] == -INFINITY ? 0.0f : ref[j];   // a column that sees nothing
    floatx16 s[NKT][QT];
    ColB<T> pf[NKT][QT];
    typename M::frag ka[NKT][G::NS];
#pragma unroll
    for (int st = 0; st < G::NS; ++st) ka[0][st] = kf(0, st);
    ColA<T, DC> va[NKT];
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt) {
      __builtin_amdgcn_sched_barrier(0);
      if (kt + 1 < NKT) {
#pragma unroll
        for (int st = 0; st < G::NS; ++st) ka[kt + 1][st] = kf(kt + 1, st);
      } else {
        va[0].load(vl, 0, lane);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < QT; ++j) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kt][j][r] = 0.0f;
      }
#pragma unroll
      for (int st = 0; st < G::NS; ++st)
#pragma unroll
        for (int j = 0; j < QT; ++j) s[kt][j] = M::mma(ka[kt][st], qf[j][st], s[kt][j]);
    }
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt) {
      scale(s[kt], c, by);
      if (kt + 1 < NKT) va[kt + 1].load(vl, 32 * (kt + 1), lane);
      cut(s[kt], pf[kt], kt, key0, mask, gone, cols, lane);
#pragma unroll
      for (int j = 0; j < QT; ++j) o[j].add(va[kt], pf[kt][j]);
    }
    bool over = false;
#pragma unroll
    for (int j = 0; j < QT; ++j) over |= sum[j] > 0.5f;
    return __any(over);
  }
  // The probabilities of block kt, cut at 1, summed.  Masked ones are taken out by bits after
  // the exponential (2 operations each; 5 by comparisons before it): cut, none is infinite.
  __device__ __forceinline__ void cut(const floatx16 (&s)[QT], ColB<T> (&pf)[QT], int kt, int32_t key0, bool mask,
                                      uint32_t gone, const Seen (&cols)[QT], int lane) {
    auto at = [&](int j, uint32_t bits, bool all) {
      float a = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float e = __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(s[j][r]), 0.0f, 1.0f);
        if (!all) e = keep_bit(e, bits, 8 * (r / 4) + r % 4);
        a += e;
        pf[j].set(r, e);
      }
      sum[j] += a;
    };
    if (!mask) {
#pragma unroll
      for (int j = 0; j < QT; ++j) at(j, 0, true);
      return;
    }
#pragma unroll
    for (int j = 0; j < QT; ++j) at(j, block_bits(cols[j], kt, key0, gone) >> (4 * (lane >> 5)), false);
  }

  // After fast() of the same tile: for each column with a score above its reference, the
  // reference goes d up, to that score and the room; sums are rescaled by 2^-d, and every
  // key gets the difference between its probability and the one that was added.  A column
  // whose sum passed a half by scores below its reference (one in the last binary step, or many further
  // down) goes up by the room, or every later step would come here again (4096 such keys: 185 us
  // instead of 88).
  template <typename KF, typename Q>
  __device__ __forceinline__ void fix(const KF& kf, const T* vl, const Q& qf, int32_t key0, bool mask, uint32_t gone,
                                      float c, const Seen (&cols)[QT], int lane) {
    floatx16 s[NKT][QT];
    float by[QT];
#pragma unroll
    for (int j = 0; j < QT; ++j) by[j] = ref[j] == -INFINITY ? 0.0f : ref[j];
    scores(s, kf, qf, key0, mask, gone, c, cols, by, lane);
    ColB<T> pf[NKT][QT];
#pragma unroll
    for (int j = 0; j < QT; ++j) {
      float m = s[0][j][0];
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) m = fmaxf(m, s[kt][j][r]);
      m = fmaxf(m, swap_halves(m));
      const float d = m > 0.0f || total(j) > 0.5f ? fmaxf(m, 0.0f) + kRoom : 0.0f;
      ref[j] = by[j] + d;
      const float f = __builtin_amdgcn_exp2f(-d);
      sum[j] *= f;
      o[j].scale(f, lane);
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float x = s[kt][j][r];
          const float e = x > 0.0f ? __builtin_amdgcn_exp2f(x - d) - f : 0.0f;
          sum[j] += e;
          pf[kt][j].set(r, e);
        }
    }
    product(vl, pf, lane);
  }
};

// What a block of columns does with a tile of KB keys: nothing, or with a mask, or all of it.
struct Edges {
  Seen first, last;
  __device__ __forceinline__ bool none(int32_t key0, int32_t n) const {
    return key0 >= last.sink && (key0 + n <= first.lo || key0 >= last.hi);
  }
  __device__ __forceinline__ bool all(int32_t key0, int32_t n) const {
    return key0 + n <= first.sink || (key0 >= last.lo && key0 + n <= first.hi);
  }
};
// The queries of columns n0 .. n1 from c0, as Edges.
template <typename U>
__device__ __forceinline__ Edges edges(const Window& w, const U& u, const Columns& c, uint32_t n0, uint32_t n1) {
  return {seen(w, u.p0 + c.query(n0), u.len), seen(w, u.p0 + c.query(n1), u.len)};
}

// The w-th block of `size` columns of all sequences' new tokens; n < 0: none.  The last block
// of a sequence, which has the most keys, comes first (8192 new tokens of one, 32 heads of 64:
// 336 us, 410 the other way round), and up to 64 sequences go by falling length, so that
// the longest passes do not start last: 64 chunks of 64 tokens over 300 to 8000 keys 251 us, 341 in the
// table's order, which more sequences keep; 64 prompts of up to 1500 tokens 406 and 394.  Every
// work-group finds its place anew, so one number for each sequence says where it stands (by two
// comparisons of lengths and lanes, not unrolled, the prompts took 474 us).
struct BlockOf {
  int32_t n, blk;
};
__device__ __forceinline__ BlockOf block_of(const FwdParams& p, uint32_t size, uint32_t w, int lane) {
  if (p.N <= 64) {
    const bool on = (uint32_t)lane < p.N;
    const uint32_t cols = on ? (uint32_t)min(new_rows(p.q_start, lane, p.T).n, (int32_t)p.Lq) * p.grp.d : 0u;
    const uint32_t len = on ? length(p.kv_len, lane, 1u << 25) : 0u;
    const uint32_t key = len << 6 | (63 - lane);   // an order of its own for each lane
    const uint32_t blocks = cols > p.few_cols ? (cols + size - 1) / size : 0;
    uint32_t first = 0;   // of the lane's sequence: the blocks of those before it
    for (uint32_t j = 0; j < p.N; j += 8) {
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) {
        const uint32_t theirs = __builtin_amdgcn_readlane(blocks, j + i);
        first += __builtin_amdgcn_readlane(key, j + i) > key ? theirs : 0u;
      }
    }
    const uint64_t it = __ballot(w >= first && w - first < blocks);
    if (!it) return {-1, 0};
    const int n = __ffsll((unsigned long long)it) - 1;
    const uint32_t f = __builtin_amdgcn_readlane(first, n), b = __builtin_amdgcn_readlane(blocks, n);
    return {n, (int32_t)(f + b - 1 - w)};
  }
  const int32_t n = (int32_t)__builtin_amdgcn_readfirstlane(piece_owner(p.q_start, p.N, p.T, p.grp.d, size, 1, w, lane));
  if ((int32_t)w < first_piece(p.q_start, n, p.T, p.grp.d, size, 1)) return {-1, 0};
  // a place past the sequence's blocks has no columns
  const int32_t blk = first_piece(p.q_start, n + 1, p.T, p.grp.d, size, 1) - 1 - (int32_t)w;
  return {blk < 0 ? -1 : n, blk};
}

// Many columns: QT blocks of 32 per wave, the keys in LDS tiles that all waves share,
// the next tile on its way in registers.  Vector units (busy 64%: for a score an exponential, its
// scaling, cut, sum and half a conversion) and matrix cores (38%) take turns, which together is the
// whole time: 8192 causal tokens, 32 heads of 64 over 8, window 2048, 159 us, 757 TFLOP/s of the
// 120 GF of its mask; without a window 318 us, 865 TFLOP/s.  In narrow windows waves wait for tiles
// that only their neighbours see (waits 50%): 8 x 16 units of 4096 x 72, window 257, 129 us.
template <typename T, typename S, bool PAGED, int DC, int NW, int QT, int KB, int NKT, int MINW>
__global__ __launch_bounds__(NW * 64, MINW) void window_fwd_kernel(FwdParams p) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  using U = Unit<T, S, PAGED>;
  using R = Rows16<T, S, DC>;
  constexpr int NT = NW * 64, CB = NW * 32 * QT, GR = KB / 16;
  constexpr int TILE = KB * G::P;
  constexpr int NL = 2 * GR / NW;   // a wave loads a group of 16 keys of K and V, or of one of them
  static_assert(NW == GR || NW == 2 * GR, "every wave loads the same");
  static_assert(NW * 32 <= 4 * KB && KB % (32 * NKT) == 0, "the output rows fit the tiles, a tile is whole steps");
  extern __shared__ __attribute__((aligned(16))) char smem[];
  T* lds = reinterpret_cast<T*>(smem);                       // [2][K, V][KB][P]
  uint32_t* gone = reinterpret_cast<uint32_t*>(lds + 4 * TILE);   // [2][GR]: pages that are not there

  keep_nan();
  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t un, e, blk;
  if constexpr (PAGED) {
    e = blockIdx.x % p.Hkv;
    const BlockOf at = block_of(p, CB, blockIdx.x / p.Hkv, lane);
    if (at.n < 0) return;
    un = (uint32_t)at.n, blk = (uint32_t)at.blk;
  } else {
    const Place pl = place(p.order);
    if (!pl.any) return;
    un = pl.bx, e = pl.h, blk = p.order.blocks - 1 - pl.block;
  }
  const U u = unit<T, S>(p, un, e, (U*)nullptr);
  const uint32_t cols = (uint32_t)u.nq * p.grp.d, c0 = blk * CB;
  if (c0 >= cols || cols <= p.few_cols) return;
  const int D = (int)p.D;
  const uint32_t nc = min(cols - c0, (uint32_t)CB);          // columns of the work-group
  const Columns cs(p.grp, c0);
  const Edges we = edges(p.win, u, cs, 0, nc - 1);
  const Tiles<KB> tiles(we.first, we.last);

  const typename R::Map map = R::map(D, u.src.row_bytes, lane);
  R rows[NL];
  float scale[NL];
  const int grp16 = 16 * (wave % GR);   // the wave's group in a tile
  const bool of_v = NL == 1 && wave >= GR;
  bool lost = false;
  int32_t id = -1;
  auto ask = [&](int32_t t) { id = t < tiles.n ? u.src.page_of(tiles.key0(t) + grp16, we.last.hi) : -1; };   // its page
  auto fetch = [&](int32_t t) {
    const int32_t key0 = tiles.key0(t) + grp16;
    const auto gp = u.src.group(key0, id);
    lost = gp.gone;
    const bool whole = !gp.gone && whole_group(we.first, we.last, key0);
    auto on = [&](int r) {
      const int32_t j = key0 + r;
      return !gp.gone && (j < we.last.sink || (j >= we.first.lo && j < we.last.hi));
    };
    rows[0].fetch(map, of_v ? gp.v : gp.k, D, p.vec, whole, on);
    scale[0] = of_v ? gp.vs : gp.ks;
    if constexpr (NL == 2) {
      rows[1].fetch(map, gp.v, D, p.vec, whole, on);
      scale[1] = gp.vs;
    }
  };
  auto stash = [&](int buf) {
    T* to = lds + buf * 2 * TILE + grp16 * G::P;
    rows[0].stash(map, to + (of_v ? TILE : 0), scale[0]);
    if constexpr (NL == 2) rows[1].stash(map, to + TILE, scale[1]);
    if (PAGED && !of_v && lane == 0) gone[buf * GR + wave % GR] = lost;
  };
  if (tiles.n) {
    ask(0);
    fetch(0);
    ask(1);
  }
  typename M::frag qf[QT][G::NS];
  Seen col[QT];
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    const uint32_t n = 32 * (wave * QT + j) + l32, i = cs.query(min(n, nc - 1)), hh = cs.head(n, i);
    row_frags<T, DC>(n < nc ? u.q + (int64_t)i * u.q_row + (int64_t)hh * D : nullptr, g, D, p.vec, qf[j]);
    col[j] = seen(p.win, u.p0 + i, u.len);
  }
  const uint32_t w0 = 32 * QT * wave;
  const bool on = w0 < nc;
  const Edges ed = edges(p.win, u, cs, min(w0, nc - 1), min(w0 + 32 * QT, nc) - 1);   // of the wave
  clear_cols<T, DC>(lds, 4 * KB, D, threadIdx.x, NT);
  if (tiles.n) stash(0);
  Softmax<T, DC, QT, NKT, sizeof(T) == 2> sm;
  sm.init();
  __syncthreads();
  // A tile's steps of 32 NKT keys: exact ones (fp32: all) until every column has a reference, then fast
  // ones, in a loop that the rare fix() stands outside of (inside, its registers weigh on it:
  // 8192 causal tokens 173 and 185 us).  Waves go from one loop to the other by themselves;
  // each meets every tile's barrier once.
  int32_t it = 0, k0 = 0;
  auto begin = [&]() __attribute__((always_inline)) {   // the tile after it sets out
    if (it + 1 >= tiles.n) return;
    fetch(it + 1);
    ask(it + 2);
  };
  auto advance = [&]() __attribute__((always_inline)) {
    k0 += 32 * NKT;
    if (k0 < KB) return;
    if (it + 1 < tiles.n) stash((it + 1) & 1);
    __syncthreads();
    k0 = 0;
    if (++it < tiles.n) begin();
  };
  // f(operands, values, first key, mask, keys not there) for a step that the wave's columns see
  auto step = [&](auto f) __attribute__((always_inline)) {
    const int32_t key0 = tiles.key0(it) + k0;
    if (!on || ed.none(key0, 32 * NKT)) return false;
    uint32_t lost_bits = 0;
    if constexpr (PAGED) {
      const uint32_t* flag = gone + (it & 1) * GR + k0 / 16;
#pragma unroll
      for (int i = 0; i < 2 * NKT; ++i) lost_bits |= flag[i] << i;
      lost_bits = __builtin_amdgcn_readfirstlane(lost_bits);
    }
    const T* ks = lds + (it & 1) * 2 * TILE + k0 * G::P;
    auto kf = [&](int kt, int st) {
      return *reinterpret_cast<const typename M::frag*>(ks + (32 * kt + l32) * G::P + 2 * G::E * st + G::E * g);
    };
    return f(kf, ks + TILE, key0, lost_bits || !ed.all(key0, 32 * NKT), lost_bits);
  };
  if (tiles.n) begin();
  while (it < tiles.n && !sm.set) {
    step([&](const auto& kf, const T* vl, int32_t key0, bool mask, uint32_t lost_bits) __attribute__((always_inline)) {
      sm.exact(kf, vl, qf, key0, mask, lost_bits, p.c, col, lane);
      return false;
    });
    advance();
  }
  if constexpr (sizeof(T) == 2) {
    while (it < tiles.n) {
      bool moved = false;
      for (; it < tiles.n && !moved;) {
        moved = step([&](const auto& kf, const T* vl, int32_t key0, bool mask, uint32_t lost_bits) __attribute__((always_inline)) {
          return sm.fast(kf, vl, qf, key0, mask, lost_bits, p.c, col, lane);
        });
        if (!moved) advance();
      }
      if (!moved) break;
      step([&](const auto& kf, const T* vl, int32_t key0, bool mask, uint32_t lost_bits) __attribute__((always_inline)) {
        sm.fix(kf, vl, qf, key0, mask, lost_bits, p.c, col, lane);
        return true;
      });
      advance();
    }
  }

#pragma unroll
  for (int j = 0; j < QT; ++j) {
    const float l = sm.total(j);
    sm.o[j].scale(l == 0.0f ? 0.0f : 1.0f / l, lane);
    const uint32_t j0 = 32 * (wave * QT + j);
    auto row = [&](int k) -> T* {
      const uint32_t n = j0 + k, i = cs.query(n);
      return n < nc ? u.o + (int64_t)i * u.o_row + (int64_t)cs.head(n, i) * D : nullptr;
    };
    if (p.vec) store_rows_lds<T, DC>(lds + wave * 32 * G::P, sm.o[j], lane, D, G::DP, row);
    else store_rows<T, DC>(sm.o[j], lane, D, false, row);
    const uint32_t n = j0 + l32, i = cs.query(n);
    if (u.lse && g == 0 && n < nc)
      u.lse[(int64_t)i * u.lse_i + (int64_t)cs.head(n, i) * u.lse_h] =
          l == 0.0f ? -INFINITY : kLn2 * (sm.ref[j] + log2f(l));
  }
}

// Short units: all keys of one in LDS at once, with one barrier, and a wave per 32 columns,
// which takes the blocks of 32 keys that it sees.  Memory bounds these: what counts is that
// a work-group asks for all of its rows at once.  1024 x 16 units of 128 x 72: 256 us, 4.8 TB/s
// (a copy: 5.1).
template <typename T, int DC, int NW, int KEYS, int MINW>
__global__ __launch_bounds__(NW * 64, MINW) void window_short_kernel(FwdParams p) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  using U = Unit<T, T, false>;
  using R = Rows16<T, T, DC>;
  constexpr int NT = NW * 64, GR = KEYS / 16, TILE = KEYS * G::P;
  constexpr int NL = 2 * GR / NW;   // group loads of a wave: K's groups, then V's
  static_assert(2 * GR % NW == 0 && NW * 32 <= 2 * KEYS, "every wave loads the same; the output rows fit");
  extern __shared__ __attribute__((aligned(16))) char smem[];
  T* kl = reinterpret_cast<T*>(smem);   // [K, V][KEYS][P]
  T* vl = kl + TILE;

  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Place pl = place(p.order);
  if (!pl.any) return;
  const U u = unit<T, T>(p, pl.bx, pl.h, (U*)nullptr);
  const uint32_t nc = (uint32_t)u.nq * p.grp.d;
  const int D = (int)p.D;
  const Columns cs(p.grp, 0);
  const Edges we = edges(p.win, u, cs, 0, nc - 1);
  const typename R::Map map = R::map(D, u.src.row_bytes, lane);
  R rows[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int li = wave + i * NW;
    const int32_t key0 = 16 * (li % GR);
    const auto gp = u.src.group(key0, 0);
    rows[i].fetch(map, li < GR ? gp.k : gp.v, D, p.vec, whole_group(we.first, we.last, key0), [&](int r) {
      const int32_t j = key0 + r;
      return j < we.last.sink || (j >= we.first.lo && j < we.last.hi);
    });
  }
  const uint32_t w0 = 32 * wave, n = w0 + l32, i = cs.query(min(n, nc - 1)), hh = cs.head(n, i);
  typename M::frag qf[1][G::NS];
  row_frags<T, DC>(n < nc ? u.q + (int64_t)i * u.q_row + (int64_t)hh * D : nullptr, g, D, p.vec, qf[0]);
  const Seen col[1] = {seen(p.win, u.p0 + i, u.len)};
  clear_cols<T, DC>(kl, 2 * KEYS, D, threadIdx.x, NT);
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int li = wave + i * NW;
    rows[i].stash(map, (li < GR ? kl : vl) + 16 * (li % GR) * G::P, 1.0f);
  }
  if constexpr (NW > 1) __syncthreads();
  else wave_order();
  Softmax<T, DC, 1, 1, false> sm;
  sm.init();
  if (w0 < nc) {
    const Edges ed = edges(p.win, u, cs, w0, min(w0 + 32, nc) - 1);
    for (int32_t key0 = 0; key0 < ed.last.hi; key0 += 32) {
      if (ed.none(key0, 32)) continue;
      sm.exact(
          [&](int, int st) {
            return *reinterpret_cast<const typename M::frag*>(kl + (key0 + l32) * G::P + 2 * G::E * st + G::E * g);
          },
          vl + key0 * G::P, qf, key0, !ed.all(key0, 32), 0, p.c, col, lane);
    }
  }
  const float l = sm.total(0);
  sm.o[0].scale(l == 0.0f ? 0.0f : 1.0f / l, lane);
  if constexpr (NW > 1) __syncthreads();   // the keys and values are done with
  else wave_order();
  auto row = [&](int k) -> T* {
    const uint32_t c = w0 + k, i = cs.query(c);
    return c < nc ? u.o + (int64_t)i * u.o_row + (int64_t)cs.head(c, i) * D : nullptr;
  };
  if (p.vec) store_rows_lds<T, DC>(kl + wave * 32 * G::P, sm.o[0], lane, D, G::DP, row);
  else store_rows<T, DC>(sm.o[0], lane, D, false, row);
  if (u.lse && g == 0 && n < nc)
    u.lse[(int64_t)i * u.lse_i + (int64_t)hh * u.lse_h] = l == 0.0f ? -INFINITY : kLn2 * (sm.ref[0] + log2f(l));
}

// Few columns: blocks of 32 of a unit's, the keys' tiles of 32 cut among work-groups and,
// inside one, among its waves, each with LDS rows of its own and no barrier until the
// waves' sums are joined.  A pass over a cache is bound by memory: what counts is how
// many waves a CU holds, that each has its next tile on its way, and that every load
// runs along rows.  2 tokens over 100000 keys, 32 heads of 128 over 8: 80 us and 8 for the join,
// 5.1 TB/s in the pass; 64 tokens over 8-bit caches of up to 16000 keys 166 us, 4.4 TB/s in the pass.
constexpr int kMinTiles = 4;   // of a work-group's wave, where the keys are cut
struct Cut {                   // tiles of each part, and parts that have any
  int32_t per, used;
};
__device__ __forceinline__ Cut cut(int32_t n, uint32_t n_split, int waves) {
  Cut c;
  const int32_t even = (n + (int32_t)n_split - 1) / (int32_t)n_split;
  c.per = (max(even, kMinTiles * waves) + waves - 1) / waves * waves;
  c.used = max((n + c.per - 1) / c.per, 1);
  return c;
}

template <typename T, typename S, bool PAGED, int DC, int NW, int MINW>
__global__ __launch_bounds__(NW * 64, MINW) void window_few_kernel(FwdParams p) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  using U = Unit<T, S, PAGED>;
  using R = Rows16<T, S, DC>;
  constexpr int TILE = 32 * G::P;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  T* kl = reinterpret_cast<T*>(smem) + wave * 2 * TILE;   // [NW][K, V][32][P]
  T* vl = kl + TILE;

  // an XCD takes the heads of a stretch of keys, which together read whole token rows, and the blocks of a head's columns
  const uint32_t he = p.Hkv * p.cblk, j8 = blockIdx.x >> 3, piece = j8 / he * 8 + (blockIdx.x & 7u);
  if (piece >= p.pieces) return;
  const uint32_t ec = j8 % he, e = ec / p.cblk, c0 = 32 * (ec - e * p.cblk);
  const uint32_t un = piece / p.n_split, split = piece - un * p.n_split;
  const U u = unit<T, S>(p, un, e, (U*)nullptr);
  const uint32_t cols = (uint32_t)u.nq * p.grp.d;
  if (c0 >= cols || cols > p.few_cols) return;
  const uint32_t nc = min(cols - c0, 32u);
  const int D = (int)p.D;
  const Columns cs(p.grp, c0);
  const Edges ed = edges(p.win, u, cs, 0, nc - 1);
  const Tiles<32> tiles(ed.first, ed.last);
  const Cut part = cut(tiles.n, p.n_split, NW);
  if ((int32_t)split >= part.used) return;
  const int32_t t1 = min(tiles.n, ((int32_t)split + 1) * part.per);

  const typename R::Map map = R::map(D, u.src.row_bytes, lane);
  R rk[2], rv[2];
  float ks[2], vs[2];
  int32_t id[2];
  uint32_t lost = 0;
  auto ask = [&](int32_t t) {
#pragma unroll
    for (int i = 0; i < 2; ++i) id[i] = u.src.page_of(tiles.key0(t) + 16 * i, t < t1 ? ed.last.hi : 0);
  };
  auto fetch = [&](int32_t t) {
    lost = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int32_t key0 = tiles.key0(t) + 16 * i;
      const auto gp = u.src.group(key0, id[i]);
      ks[i] = gp.ks, vs[i] = gp.vs;
      lost |= (gp.gone ? 1u : 0u) << i;
      auto on = [&](int r) {
        const int32_t j = key0 + r;
        return !gp.gone && (j < ed.last.sink || (j >= ed.first.lo && j < ed.last.hi));
      };
      const bool whole = !gp.gone && whole_group(ed.first, ed.last, key0);
      rk[i].fetch(map, gp.k, D, p.vec, whole, on);
      rv[i].fetch(map, gp.v, D, p.vec, whole, on);
    }
  };
  const int32_t mine = (int32_t)split * part.per + wave;
  if (mine < t1) {
    ask(mine);
    fetch(mine);
    ask(mine + NW);
  }
  clear_cols<T, DC>(kl, 64, D, lane, 64);
  const uint32_t ci = cs.query(min((uint32_t)l32, nc - 1)), ch = cs.head(l32, ci);
  typename M::frag qf[1][G::NS];
  row_frags<T, DC>((uint32_t)l32 < nc ? u.q + (int64_t)ci * u.q_row + (int64_t)ch * D : nullptr, g, D, p.vec, qf[0]);
  const Seen col[1] = {seen(p.win, u.p0 + ci, u.len)};

  Softmax<T, DC, 1, 1, false> sm;
  sm.init();
  for (int32_t t = mine; t < t1; t += NW) {
    wave_order();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      rk[i].stash(map, kl + 16 * i * G::P, ks[i]);
      rv[i].stash(map, vl + 16 * i * G::P, vs[i]);
    }
    const uint32_t was_lost = lost;
    wave_order();
    if (t + NW < t1) {
      fetch(t + NW);
      ask(t + 2 * NW);
    }
    const int32_t key0 = tiles.key0(t);
    sm.exact(
        [&](int, int st) {
          return *reinterpret_cast<const typename M::frag*>(kl + l32 * G::P + 2 * G::E * st + G::E * g);
        },
        vl, qf, key0, was_lost || !ed.all(key0, 32), was_lost, p.c, col, lane);
  }
  float l = sm.total(0);

  // the waves' columns meet at the largest of their references, and are added in the
  // waves' order; the tiles are done with
  auto out = [&](uint32_t n) {
    const uint32_t i = cs.query(n);
    return u.o + (int64_t)i * u.o_row + (int64_t)cs.head(n, i) * D;
  };
  auto put_lse = [&](uint32_t n, float m, float s) {
    const uint32_t i = cs.query(n);
    if (u.lse)
      u.lse[(int64_t)i * u.lse_i + (int64_t)cs.head(n, i) * u.lse_h] = s == 0.0f ? -INFINITY : kLn2 * (m + log2f(s));
  };
  __syncthreads();
  float* ms = reinterpret_cast<float*>(smem);   // [NW][32] references, [NW][32] sums, [2][32] joined
  if (g == 0) {
    ms[wave * 32 + l32] = sm.ref[0];
    ms[(NW + wave) * 32 + l32] = l;
  }
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < NW; ++w) top = fmaxf(top, ms[w * 32 + l32]);
  const float base = top == -INFINITY ? 0.0f : top;
  l = 0.0f;
#pragma unroll
  for (int w = 0; w < NW; ++w) l += __builtin_amdgcn_exp2f(ms[w * 32 + l32] - base) * ms[(NW + w) * 32 + l32];
  sm.o[0].scale(__builtin_amdgcn_exp2f(sm.ref[0] - base), lane);
  float* rows = ms + (2 * NW + 2) * 32;   // [NW][nc][DP]
  store_rows<T, DC>(sm.o[0], lane, G::DP, true, [&](int n) -> float* {
    return (uint32_t)n < nc ? rows + (wave * nc + n) * G::DP : nullptr;
  });
  if (wave == 0 && g == 0) {
    ms[2 * NW * 32 + l32] = top;
    ms[(2 * NW + 1) * 32 + l32] = l;
  }
  __syncthreads();
  // maxima, sums, rows of 32 columns
  float* to = p.part + (((uint64_t)un * he + ec) * p.n_split + split) * 32 * (2 + p.D);
  for (uint32_t i = threadIdx.x; i < nc * p.D; i += NW * 64) {
    const uint32_t n = i / p.D, d = i - n * p.D;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) v += rows[(w * nc + n) * G::DP + d];
    const float s = ms[(2 * NW + 1) * 32 + n];
    if (part.used > 1) to[64 + i] = v;
    else out(n)[d] = (T)(s == 0.0f ? 0.0f : v / s);
  }
  if (threadIdx.x < nc) {
    const float m = ms[2 * NW * 32 + threadIdx.x], s = ms[(2 * NW + 1) * 32 + threadIdx.x];
    if (part.used > 1) to[threadIdx.x] = m, to[32 + threadIdx.x] = s;
    else put_lse(threadIdx.x, m, s);
  }
}

// Joins the parts of one column: with their references m_s, sums l_s and rows o_s,
// o = sum 2^(m_s - m) o_s / sum 2^(m_s - m) l_s.  A work-group per column; 256 / DP groups
// of threads take every such part, and their sums are added in order.
constexpr int kMaxSplit = 512;
template <typename T, typename S, bool PAGED, int DP>
__global__ __launch_bounds__(256) void window_join_kernel(FwdParams p, int waves) {
  constexpr int GR = 256 / DP;
  __shared__ float f[kMaxSplit], red[256], m4[4];
  using U = Unit<T, S, PAGED>;
  const uint32_t he = p.Hkv * p.cblk, uec = blockIdx.x / p.block_cols, n = blockIdx.x - uec * p.block_cols;
  const uint32_t un = uec / he, ec = uec - un * he, e = ec / p.cblk, c0 = 32 * (ec - e * p.cblk);
  const U u = unit<T, S>(p, un, e, (U*)nullptr);
  const uint32_t cols = (uint32_t)u.nq * p.grp.d;
  if (c0 + n >= cols || cols > p.few_cols) return;
  const Columns cs(p.grp, c0);
  const Edges ed = edges(p.win, u, cs, 0, min(cols - c0, 32u) - 1);
  const Tiles<32> tiles(ed.first, ed.last);
  const uint32_t used = (uint32_t)cut(tiles.n, p.n_split, waves).used;
  if (used == 1) return;
  const uint32_t stride = 32 * (2 + p.D);
  const float* w = p.part + (uint64_t)uec * p.n_split * stride;
  float m = -INFINITY;
  for (uint32_t s = threadIdx.x; s < used; s += 256) {
    f[s] = w[(uint64_t)s * stride + n];
    m = fmaxf(m, f[s]);
  }
#pragma unroll
  for (int off = 32; off; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
  if ((threadIdx.x & 63) == 0) m4[threadIdx.x >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
  const float top = m == -INFINITY ? 0.0f : m;
  for (uint32_t s = threadIdx.x; s < used; s += 256) f[s] = __builtin_amdgcn_exp2f(f[s] - top);   // no keys: 0
  __syncthreads();
  const uint32_t d = threadIdx.x % DP, gr = threadIdx.x / DP;
  float a = 0.0f, l = 0.0f;
  if (d < p.D) {
#pragma unroll 4
    for (uint32_t s = gr; s < used; s += GR) {
      const float* ws = w + (uint64_t)s * stride;
      l += f[s] * ws[32 + n];
      a += f[s] * ws[64 + n * p.D + d];
    }
  }
  red[threadIdx.x] = a;
  __syncthreads();
  if (gr == 0) {
#pragma unroll
    for (int i = 1; i < GR; ++i) a += red[i * DP + d];
  }
  __syncthreads();
  red[threadIdx.x] = l;
  __syncthreads();
  if (gr || d >= p.D) return;
#pragma unroll
  for (int i = 1; i < GR; ++i) l += red[i * DP + d];
  const uint32_t i = cs.query(n), hh = cs.head(n, i);
  u.o[(int64_t)i * u.o_row + (int64_t)hh * p.D + d] = (T)(l == 0.0f ? 0.0f : a / l);
  if (u.lse && d == 0)
    u.lse[(int64_t)i * u.lse_i + (int64_t)hh * u.lse_h] = l == 0.0f ? -INFINITY : kLn2 * (top + log2f(l));
}

template <typename K>
int launch(K* kernel, int64_t blocks, int threads, size_t lds, FwdParams& p, hipStream_t s) {
  if (!grid_fits(blocks, threads)) return DSP_ERR_SHAPE;
  if (lds > 64 * 1024) {
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return DSP_ERR_HIP;
  }
  kernel<<<dim3((uint32_t)blocks), threads, lds, s>>>(p);
  return last_launch_status();
}

template <typename T, typename S, bool PAGED, int DC, int NW, int QT, int KB, int NKT, int MINW>
int start_many(FwdParams& p, const WindowArgs& a, hipStream_t s) {
  constexpr int CB = NW * 32 * QT;
  int64_t blocks;
  if (PAGED) {
    p.n_blk = (uint32_t)(a.T * p.grp.d / CB + a.B);
    blocks = (int64_t)p.n_blk * a.Hkv;
  } else {
    p.order = window_order(a, (a.Lq * p.grp.d + CB - 1) / CB, CB / p.grp.d + 1);
    blocks = order_blocks(p.order);
  }
  const size_t lds = (size_t)4 * KB * Geo<T, DC>::P * sizeof(T) + 2 * (KB / 16) * 4;
  return launch(window_fwd_kernel<T, S, PAGED, DC, NW, QT, KB, NKT, MINW>, blocks, NW * 64, lds, p, s);
}

template <typename T, int DC, int NW, int KEYS, int MINW>
int start_short(FwdParams& p, const WindowArgs& a, hipStream_t s) {
  p.order = make_order(a.B * a.X, a.Hkv, 1, 1, false);
  return launch(window_short_kernel<T, DC, NW, KEYS, MINW>, order_blocks(p.order), NW * 64,
                (size_t)2 * KEYS * Geo<T, DC>::P * sizeof(T), p, s);
}

template <typename T, typename S, bool PAGED, int DC, int NW>
int start_few(FwdParams& p, const WindowArgs& a, hipStream_t s) {
  constexpr int MINW = sizeof(T) == 4 ? 1 : DC <= 80 ? 3 : 2;
  size_t lds = (size_t)NW * 2 * 32 * Geo<T, DC>::P * sizeof(T);
  lds = std::max(lds, ((2 * NW + 2) * 32 + (size_t)NW * 32 * Geo<T, DC>::DP) * 4);
  const int64_t pieces = a.B * a.X * p.n_split;
  p.pieces = (uint32_t)pieces;
  int st = launch(window_few_kernel<T, S, PAGED, DC, NW, MINW>, (pieces + 7) / 8 * 8 * a.Hkv * p.cblk, NW * 64, lds, p, s);
  if (st != DSP_OK || p.n_split == 1) return st;
  p.block_cols = (uint32_t)std::min<int64_t>(a.Lq * p.grp.d, 32);
  const int64_t cols = a.B * a.X * a.Hkv * p.cblk * p.block_cols;   // few units: they are why the keys are split
  if (!grid_fits(cols, 256)) return DSP_ERR_SHAPE;
  if (a.D <= 64) window_join_kernel<T, S, PAGED, 64><<<dim3((uint32_t)cols), 256, 0, s>>>(p, NW);
  else window_join_kernel<T, S, PAGED, 128><<<dim3((uint32_t)cols), 256, 0, s>>>(p, NW);
  return last_launch_status();
}

// How a call is cut: whether units of few columns have a launch of their own, and into
// how many parts their keys go at most.
struct Choice {
  bool few, many;
  int64_t cblk, n_split;
};
inline Choice choose(const WindowArgs& a) {
  Choice c = {};
  const int64_t grp = a.H / a.Hkv, cols = a.Lq * grp, units = std::max<int64_t>(a.B * a.X * a.Hkv, 1);
  // keys that a block of columns can see
  int64_t keys = a.Lk;
  if (a.win.left >= 0 && a.win.right >= 0)
    keys = std::min<int64_t>(keys, (int64_t)a.win.left + a.win.right + a.win.sinks + 64);
  // More columns than a block has take several of this form where the other one, with whole
  // passes over the keys, would leave most of the chip idle: each block reads the keys again, out
  // of L2.  Heads of 64, groups of 4; blocks of all units, keys: this form and the other in us:
  // 16, 8000: 21 and 124; 128, 2000: 33 and 37; 256, 2000: 53 and 37; 512, 8000: 115 - 135 and
  // 146 - 173; 1024, 8000: 220 and 171; 16, 100000: 58 and 1760; 512, 100000: 842 and 2183 (keys from
  // the call before in the 256 MB cache; 16, 100000 with other keys in turn 73).
  const int64_t blocks = (cols + 31) / 32;
  c.cblk = cols > 32 && units * blocks <= std::min<int64_t>(512, keys / 16) ? blocks : 1;
  c.few = grp <= 32 || c.cblk > 1;
  c.many = cols > 32 * c.cblk;
  if (c.many && !(a.page_shift && a.B > 1)) c.few = false;
  c.n_split = 1;
  if (!c.few) return c;
  // One sequence's units are alike: as many work-groups as the chip holds at once (100000 keys
  // of 8 heads of 128: 87 us with 2 to a CU, 93 with 4, 104 with 8).  Sequences differ in
  // length: 8 to a CU (64 of up to 16000 keys in 8 bits, 8 heads of 64: 166 us; 178 with 6, 196
  // with 4, 174 with 16).
  const int64_t per_cu = a.B > 1 ? 8 : !a.bf16 ? 1 : a.D <= 64 ? 4 : a.D <= 80 ? 3 : 2;
  int64_t n = (256 * per_cu + units * c.cblk - 1) / (units * c.cblk);
  // a part's blocks and heads run on one XCD: as many parts for each of the eight
  if (c.cblk > 1) n = (n + 7) / 8 * 8;
  n = std::min<int64_t>({n, keys / 256, kMaxSplit});
  if (n > 1) c.n_split = n;
  return c;
}
inline size_t part_bytes(const WindowArgs& a) {
  const Choice c = choose(a);
  return c.n_split > 1 ? (size_t)(a.B * a.X * a.Hkv * c.cblk * c.n_split) * 32 * (2 + (size_t)a.D) * 4 : 0;
}

template <typename T, typename S, bool PAGED, int DC>
int start(FwdParams& p, const WindowArgs& a, const Choice& c, hipStream_t s) {
  p.few_cols = c.few ? (uint32_t)(32 * c.cblk) : 0;
  p.cblk = (uint32_t)c.cblk;
  p.n_split = (uint32_t)c.n_split;
  if (c.few) {
    if (int st = start_few<T, S, PAGED, DC, 4>(p, a, s)) return st;
  }
  if (!c.many) return DSP_OK;
  // Registers for three waves to a SIMD where they go without (many) spills, tiles of 64 keys
  // where they do not: 8 x 16 units of 4096 x 72, window 257, 144 us with three waves and 32
  // keys, 160 and 174 with two waves and 64 and 32; 32 heads of 8192 x 64, window 2048, 172 us
  // with three waves and 64 keys, 198 with 32; 16 of 8192 x 128, window 1024, with two waves 218
  // and 226.
  // Steps of 32 keys inside a tile of 64 above that: 209 us.
  constexpr bool B16 = sizeof(T) == 2, MID = DC > 64 && DC <= 80;
  return start_many<T, S, PAGED, DC, 4, 1, B16 && !MID ? 64 : 32, B16 && DC <= 64 ? 2 : 1, B16 ? (DC <= 80 ? 3 : 2) : 1>(p, a, s);
}

inline FwdParams params(const WindowArgs& a) {
  FwdParams p = {};
  p.q = a.q, p.k = a.k, p.v = a.v, p.o = a.o, p.lse = a.lse, p.part = a.workspace;
  p.q_pos = a.q_pos, p.kv_len = a.kv_len, p.q_start = a.q_start, p.table = a.table;
  p.k_scale = a.k_scale, p.v_scale = a.v_scale;
  for (int i = 0; i < 3; ++i) p.qs[i] = a.q_strides[i], p.ks[i] = a.kv_strides[i], p.os[i] = a.o_strides[i];
  p.win = a.win;
  p.X = (uint32_t)a.X, p.H = a.H, p.Hkv = a.Hkv, p.grp = divisor(a.H / a.Hkv), p.Lq = (uint32_t)a.Lq, p.Lk = (uint32_t)a.Lk;
  p.D = a.D;
  p.N = (uint32_t)a.B, p.T = (uint32_t)a.T, p.n_pages = (uint32_t)a.n_pages, p.max_pages = (uint32_t)a.max_pages;
  p.shift = a.page_shift;
  p.c = a.scale * kLog2e;
  p.vec = a.vec;
  return p;
}

}  // namespace
}  // namespace dsp
