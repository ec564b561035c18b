// Attention with a learned relative position bias by buckets (forward):
//   s_ij = scale q_i . k_j + bias[bucket(j - i - q_pos)][h],  o = softmax(s) v,
// over the keys inside kv_len and, when causal, not after the query.
//
// One pass over the keys with the running maximum and sum of the softmax; both
// products on the matrix cores, computed transposed (keys on rows, queries on
// columns) as in the plain kernels: a lane owns one query column, so the statistics
// are per-lane scalars and the probabilities are the next product's operand as they
// stand.  The scale and the bias meet the fp32 score in one fused multiply-add, so
// nothing of a score is rounded to bf16.
//
// The bias depends on the distance only.  A work-group keeps the part of the table it
// can need in LDS, one fp32 value per distance; a 32 x 32 block of scores is a band of
// 63 distances of it.  Blocks wholly past the table's end have one value, in a
// register; for long sequences that is nearly all of them, and the bias costs them
// nothing beyond the multiply-add that the scale needs anyway.
//
// The subtracted reference follows the running maximum lazily: it is the maximum of the
// first tile until a tile's probabilities sum to more than 2^16 (one comparison for
// each column and tile); only then are the tile's maxima taken and the sums rescaled.
//
// Few queries against many keys (a new token against a cache): the queries of a
// key/value head's group share one block of 32 columns, and the keys are cut among
// work-groups, whose unnormalised sums a second kernel joins.
//
// Measured in bf16, 16 heads of 72: 8 x 16 units of 4096 750-860 us with the card's clock
// (825-720 TFLOP/s): the matrix cores are busy 38%, the vector units 30%, waits take 30%;
// whether the reference moves is asked between a tile's exponentials and its second
// product, so none of the one runs under the other.  The plain attention, which multiplies
// first and corrects afterwards, takes 600-640 us.  1350 x 16 units of 49: 159-175 us (3.8-3.5
// TB/s; the plain attention 120); 1024 x 16 units of 32 66-71 us (4.3-4.6 TB/s, memory); a
// token against 4 caches of up to 50000 keys of 8 heads of 64 38 us and 4 for the join (5.3
// TB/s while it reads), against 2048 caches of up to 120 keys 50 us (4.9 TB/s).
#include <algorithm>
#include <type_traits>

#include "attn_relpos.h"

namespace dsp {
namespace {

// Whether a row's sum says that it has no keys: exactly 0.  By its bits, since a query
// that is not finite has a NaN there, which this file's comparisons may take either way.
__device__ __forceinline__ bool no_keys(float sum) { return __builtin_bit_cast(uint32_t, sum) == 0u; }

struct FwdParams {
  const void* q;
  const void* k;
  const void* v;
  void* o;
  float* lse;
  float* part;       // split keys: the columns' references, sums and rows of each work-group
  const int32_t* q_pos;
  const int32_t* kv_len;
  int64_t qs[3], ks[3], os[3];
  BiasArgs bias;
  uint32_t X, H, grp, Lq, Lk, n_split, split_keys, D;
  uint32_t sub;      // few queries: parts of a key/value head's group, of grp heads each
  Order order;       // many queries
  uint32_t pieces;   // few queries: (b, x) times splits
  uint32_t tab;      // distances of the LDS table, for each head of a work-group
  uint32_t cols;     // few queries: queries x grp
  float c;           // scale * log2(e)
  bool vec, causal;
};

// The softmax of QT blocks of 32 query columns over NKT blocks of 32 keys at a time.
// LAZY: the reference moves only when it has to (long runs of keys); otherwise every
// tile takes its maxima (few keys, and passes that memory bounds).
template <typename T, int DC, int QT, int NKT, bool LAZY>
struct Softmax {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  // a tile's sum of probabilities past this moves the reference: every probability
  // then stays below it, far inside both types' range
  static constexpr float kMove = 65536.0f;
  ColAcc<T, DC> o[QT];
  float ref[QT], sum[QT];   // exp2 units; the sum of this lane's keys
  bool set;                 // every column has a reference

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int j = 0; j < QT; ++j) {
      o[j].zero();
      ref[j] = -INFINITY;
      sum[j] = 0.0f;
    }
    set = false;
  }
  // what a tile of keys needs besides its LDS rows
  struct Keys {
    int32_t key0;           // its first key
    int32_t stop;           // keys of the work-group end here
    int32_t M;
    bool causal;
  };

  // scores of the tile in exp2 units, less `minus`
  template <typename KF, typename Q>
  static __device__ __forceinline__ void scores(floatx16 (&s)[NKT][QT], const KF& kf, const Q& qf, const Keys& k, float c,
                                         const int32_t (&first)[QT], const int32_t (&at)[QT],
                                         const float* const (&tab)[QT], const float (&left)[QT],
                                         const float (&right)[QT], const float (&minus)[QT], int lane) {
    const int g = lane >> 5;
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
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int j = 0; j < QT; ++j) {
        const int32_t key0 = k.key0 + 32 * kt;
        const int32_t d0 = key0 - first[j];
        if (d0 + 31 <= -k.M || d0 - 31 >= k.M) {
          const float t = (d0 < 0 ? left[j] : right[j]) - minus[j];
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kt][j][r] = fmaf(s[kt][j][r], c, t);
        } else {
          const float* tb = tab[j] + key0 + 4 * g;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kt][j][r] = fmaf(s[kt][j][r], c, tb[8 * (r / 4) + r % 4] - minus[j]);
        }
        if ((k.causal && d0 + 31 > 0) || key0 + 32 > k.stop) {
          const int32_t stop = k.causal ? min(k.stop, at[j] + 1) : k.stop;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (key0 + 8 * (r / 4) + 4 * g + r % 4 >= stop) s[kt][j][r] = -INFINITY;
        }
      }
  }

  // One tile: kf(kt, st) the fragments of its keys, vl its values in LDS; first[j] is the
  // position of block j's first query, at[j] of this lane's own, tab[j] the table at
  // its distance from key 0.
  template <typename KF, typename Q>
  __device__ __forceinline__ void step(const KF& kf, const T* vl, const Q& qf, const Keys& k, float c,
                                       const int32_t (&first)[QT], const int32_t (&at)[QT],
                                       const float* const (&tab)[QT], const float (&left)[QT],
                                       const float (&right)[QT], int lane) {
    ColB<T> pf[NKT][QT];
    float add[QT];
    bool move = !LAZY || !set;
    if (LAZY && set) {
      floatx16 s[NKT][QT];
      scores(s, kf, qf, k, c, first, at, tab, left, right, ref, lane);
      move = probabilities(s, pf, add);
    }
    if (!LAZY || __any(move)) {
      // the scores themselves, their maxima, and the sums moved to those
      floatx16 s[NKT][QT];
      float zero[QT];
#pragma unroll
      for (int j = 0; j < QT; ++j) zero[j] = 0.0f;
      scores(s, kf, qf, k, c, first, at, tab, left, right, zero, lane);
      bool all = true;
#pragma unroll
      for (int j = 0; j < QT; ++j) {
        float m = s[0][j][0];
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
          for (int r = 0; r < 16; ++r) m = fmaxf(m, s[kt][j][r]);
        m = fmaxf(fmaxf(m, swap_halves(m)), ref[j]);
        const float f = ref[j] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ref[j] - m);
        sum[j] *= f;
        o[j].scale(f, lane);
        ref[j] = m;
        all &= m != -INFINITY;
        const float by = m == -INFINITY ? 0.0f : m;   // nothing yet: every score is -inf
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kt][j][r] -= by;
      }
      set = __all(all);
      probabilities(s, pf, add);
    }
#pragma unroll
    for (int j = 0; j < QT; ++j) sum[j] += add[j];
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int j = 0; j < QT; ++j) o[j].add(vl, 32 * kt, lane, pf[kt][j]);
  }
  // exp2 of the scores, as operands and summed; whether some column's are too large
  static __device__ __forceinline__ bool probabilities(const floatx16 (&s)[NKT][QT], ColB<T> (&pf)[NKT][QT],
                                                       float (&add)[QT]) {
    bool over = false;
#pragma unroll
    for (int j = 0; j < QT; ++j) {
      float a = 0.0f;
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = __builtin_amdgcn_exp2f(s[kt][j][r]);
          a += e;
          pf[kt][j].set(r, e);
        }
      add[j] = a;
      over |= a > kMove;
    }
    return over;
  }
};

// Many queries: QT blocks of 32 queries of one head per wave, the keys in LDS tiles
// that all waves share, the next tile on its way in registers.
template <typename T, int DC, int NW, int QT, int KB, int NBUF, int MINW>
__global__ __launch_bounds__(NW * 64, MINW) void relpos_fwd_kernel(FwdParams p) {
  // NBUF == 1: one tile holds all keys
  using G = Geo<T, DC>;
  using M = Mx<T>;
  constexpr int NT = NW * 64, QB = NW * 32 * QT, NKT = KB / 32;
  constexpr int TILE = KB * G::P;
  static_assert(NW * QT * 32 <= NBUF * 2 * KB || QT > 1 || NW <= NBUF * 2 * NKT, "the output rows fit the tiles");
  extern __shared__ __attribute__((aligned(16))) char smem[];
  T* lds = reinterpret_cast<T*>(smem);                       // [NBUF][K, V][KB][P]
  float* tab = reinterpret_cast<float*>(lds + NBUF * 2 * TILE);

  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Place pl = place(p.order);
  if (!pl.any) return;
  // causal: the last queries have the most keys
  const uint32_t bx = pl.bx, h = pl.h, qb = p.causal ? p.order.blocks - 1 - pl.block : pl.block;
  const uint32_t b = bx / p.X, x = bx % p.X;
  const int D = (int)p.D;
  const int64_t k_at = (int64_t)b * p.ks[0] + (int64_t)x * p.ks[1] + (int64_t)(h / p.grp) * D;
  const T* kg = static_cast<const T*>(p.k) + k_at;
  const T* vg = static_cast<const T*>(p.v) + k_at;
  const T* qg = static_cast<const T*>(p.q) + (int64_t)b * p.qs[0] + (int64_t)x * p.qs[1] + (int64_t)h * D;

  const int32_t q0 = position(p.q_pos, b) + (int32_t)(qb * QB);   // position of the block's first query
  const uint32_t nq = min(p.Lq - qb * QB, (uint32_t)QB);
  uint32_t k1 = length(p.kv_len, b, p.Lk);
  if (p.causal) {
    const int32_t last = q0 + (int32_t)nq;   // keys before it
    k1 = last <= 0 ? 0u : min(k1, (uint32_t)last);
  }
  const uint32_t row_bytes = (uint32_t)p.ks[2] * (uint32_t)sizeof(T);
  using TileT = Tile<T, DC, KB, NT>;
  const typename TileT::Map map = TileT::map(D, row_bytes, threadIdx.x);
  TileT tk, tv;
  auto fetch = [&](uint32_t kb) {
    const uint32_t rows = kb < k1 ? min(k1 - kb, (uint32_t)KB) : 0u;
    tk.fetch(map, kg + (int64_t)kb * p.ks[2], rows, row_bytes, D, p.vec);
    tv.fetch(map, vg + (int64_t)kb * p.ks[2], rows, row_bytes, D, p.vec);
  };
  auto stash = [&](int buf) {
    tk.stash(map, lds + buf * 2 * TILE);
    tv.stash(map, lds + buf * 2 * TILE + TILE);
  };
  // the table: distances lo .. hi
  const int32_t lo = max(-(p.bias.M + kEdge), -(q0 + QB - 1));
  const int32_t hi = min(p.bias.M + kEdge, (int32_t)((k1 + KB - 1) / KB * KB) - 1 - q0);
  const int32_t n_tab = k1 ? hi - lo + 1 : 0;
  Table<T, NT> table;
  table.fetch(p.bias, lo, n_tab);
  const int32_t wq = q0 + 32 * QT * wave;   // the wave's first query
  typename M::frag qf[QT][G::NS];
  if constexpr (NBUF == 1) {
    // short units are bound by memory: Q, too, comes along its rows, through the
    // rows of V
    static_assert(QB == KB && QT == 1, "one tile of queries");
    const uint32_t q_row = (uint32_t)p.qs[2] * (uint32_t)sizeof(T);
    const typename TileT::Map mq = TileT::map(D, q_row, threadIdx.x);
    TileT tq;
    tq.fetch(mq, qg + (int64_t)(qb * QB) * p.qs[2], nq, q_row, D, p.vec);
    if (k1) fetch(0);
    clear_pad<T, DC>(lds, 2 * KB, D, threadIdx.x, NT);
    tq.stash(mq, lds + TILE);
    if (k1) tk.stash(map, lds);
    __syncthreads();
#pragma unroll
    for (int st = 0; st < G::NS; ++st)
      qf[0][st] = *reinterpret_cast<const typename M::frag*>(lds + TILE + (32 * wave + l32) * G::P + 2 * G::E * st +
                                                             G::E * g);
    __syncthreads();
    if (k1) tv.stash(map, lds + TILE);
  } else {
    if (k1) fetch(0);
#pragma unroll
    for (int j = 0; j < QT; ++j) {
      const uint32_t i = 32 * (wave * QT + j) + l32;
      row_frags<T, DC>(i < nq ? qg + (int64_t)(qb * QB + i) * p.qs[2] : nullptr, g, D, p.vec, qf[j]);
    }
    clear_pad<T, DC>(lds, NBUF * 2 * KB, D, threadIdx.x, NT);
    if (k1) stash(0);
  }
  table.build(p.bias, lo, n_tab, tab, 0, p.H, h, 1);
  float left[QT], right[QT];
  int32_t first[QT], at[QT];
  const float* tb[QT];
  left[0] = bias_at<T>(p.bias, p.H, h, -p.bias.M);
  right[0] = bias_at<T>(p.bias, p.H, h, p.bias.M);
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    left[j] = left[0], right[j] = right[0];
    first[j] = wq + 32 * j;
    at[j] = first[j] + l32;
    tb[j] = tab - lo - at[j];
  }
  Softmax<T, DC, QT, NKT, NBUF != 1> sm;
  sm.init();
  __syncthreads();
  const uint32_t n_it = (k1 + KB - 1) / KB;
  for (uint32_t it = 0; it < n_it; ++it) {
    const uint32_t kb = it * KB;
    const bool more = NBUF > 1 && it + 1 < n_it;
    if (more) fetch(kb + KB);
    const T* kl = lds + (NBUF > 1 ? (it & 1) : 0) * 2 * TILE;
    // queries of this wave are all before the tile, or past the end: nothing to do
    if (!(p.causal && (int32_t)kb > wq + 32 * QT - 1) && 32u * QT * wave < nq)
      sm.step(
          [&](int kt, int st) {
            return *reinterpret_cast<const typename M::frag*>(kl + (32 * kt + l32) * G::P + 2 * G::E * st + G::E * g);
          },
          kl + TILE, qf, {(int32_t)kb, (int32_t)k1, p.bias.M, p.causal}, p.c, first, at, tb, left, right, lane);
    if (more) stash((it + 1) & 1);
    __syncthreads();
  }

  T* og = static_cast<T*>(p.o) + (int64_t)b * p.os[0] + (int64_t)x * p.os[1] + (int64_t)h * D;
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    const float l = sm.sum[j] + swap_halves(sm.sum[j]);
    sm.o[j].scale(no_keys(l) ? 0.0f : 1.0f / l, lane);
    const uint32_t c0 = 32 * (wave * QT + j);
    auto row = [&](int n) -> T* { return c0 + n < nq ? og + (int64_t)(qb * QB + c0 + n) * p.os[2] : nullptr; };
    if (p.vec) store_rows_lds<T, DC>(lds + wave * 32 * G::P, sm.o[j], lane, D, G::DP, row);
    else store_rows<T, DC>(sm.o[j], lane, D, false, row);
    if (p.lse && g == 0 && c0 + l32 < nq)
      p.lse[((uint64_t)bx * p.H + h) * p.Lq + qb * QB + c0 + l32] = no_keys(l) ? -INFINITY : kLn2 * (sm.ref[j] + log2f(l));
  }
}

// Few queries: the queries of a key/value head's group (at most 32 in all) are the
// columns of one block.  Each wave takes every NW-th tile of 32 keys through LDS rows of
// its own, with no barrier until the waves' sums are joined.  A pass over a cache is
// bound by memory: what counts is how many waves a CU holds, that each has its next
// tile on its way, and that every load runs along rows (the operands' own layout,
// loaded directly, asks L2 for each line four times: 61 -> 81 us for the token
// against long caches).  ONE: the keys are one tile.
template <typename T, int DC, int NW, bool ONE, int MINW>
__global__ __launch_bounds__(NW * 64, MINW) void relpos_few_kernel(FwdParams p) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  constexpr int TILE = 32 * G::P;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  T* kl = reinterpret_cast<T*>(smem) + wave * 2 * TILE;   // [NW][K, V][32][P]
  T* vl = kl + TILE;
  float* tab = reinterpret_cast<float*>(reinterpret_cast<T*>(smem) + NW * 2 * TILE);

  // an XCD takes the heads of a stretch of keys, which together read whole token rows
  const uint32_t kvh = p.H / p.grp, j8 = blockIdx.x >> 3, piece = j8 / kvh * 8 + (blockIdx.x & 7u);
  if (piece >= p.pieces) return;
  const uint32_t e = j8 % kvh, split = piece % p.n_split, bx = piece / p.n_split, h0 = e * p.grp;
  const uint32_t b = bx / p.X, x = bx - b * p.X;
  const int D = (int)p.D;
  const int64_t k_at = (int64_t)b * p.ks[0] + (int64_t)x * p.ks[1] + (int64_t)(e / p.sub) * D;
  const T* kg = static_cast<const T*>(p.k) + k_at;
  const T* vg = static_cast<const T*>(p.v) + k_at;

  const int32_t q0 = position(p.q_pos, b);
  const uint32_t k0 = split * p.split_keys;
  uint32_t k1 = min(length(p.kv_len, b, p.Lk), k0 + p.split_keys);
  if (p.causal) {
    const int32_t last = q0 + (int32_t)p.Lq;
    k1 = last <= 0 ? 0u : min(k1, (uint32_t)last);
  }
  const uint32_t row_bytes = (uint32_t)p.ks[2] * (uint32_t)sizeof(T);
  using TileT = Tile<T, DC, 32, 64>;
  const typename TileT::Map map = TileT::map(D, row_bytes, lane);
  TileT tk, tv;
  auto fetch = [&](uint32_t kb) {
    const uint32_t rows = kb < k1 ? min(k1 - kb, 32u) : 0u;
    tk.fetch(map, kg + (int64_t)kb * p.ks[2], rows, row_bytes, D, p.vec);
    tv.fetch(map, vg + (int64_t)kb * p.ks[2], rows, row_bytes, D, p.vec);
  };
  const int32_t lo = max(-(p.bias.M + kEdge), (int32_t)k0 - (q0 + 31));
  const int32_t hi = min(p.bias.M + kEdge, (int32_t)(k0 + (max(k1, k0) - k0 + 31) / 32 * 32) - 1 - q0);
  const int32_t n_tab = k0 < k1 ? hi - lo + 1 : 0;
  Table<T, NW * 64> table;
  table.fetch(p.bias, lo, n_tab);
  // this lane's column: head ch of the group, query cq
  const uint32_t ch = min(l32 / p.Lq, p.grp - 1), cq = l32 - ch * p.Lq;
  const T* qg = static_cast<const T*>(p.q) + (int64_t)b * p.qs[0] + (int64_t)x * p.qs[1];
  auto at_row = [&](uint32_t hh, uint32_t i, int64_t rs) { return (int64_t)i * rs + (int64_t)(h0 + hh) * D; };
  // the columns' rows, on their way to LDS like the keys'
  constexpr int NQ = (32 * G::CHM + 63) / 64;
  u32x4 qp[NQ];
  const uint32_t chunks = (uint32_t)(D / G::E);
  if (p.vec)
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const uint32_t c = lane + 64 * i, col = c / chunks, hh = col / p.Lq;
      if (col < p.cols)
        qp[i] = *reinterpret_cast<const u32x4*>(qg + at_row(hh, col - hh * p.Lq, p.qs[2]) + (c - col * chunks) * G::E);
    }
  const uint32_t mine = k0 + 32 * wave;
  if (mine < k1) fetch(mine);
  clear_pad<T, DC>(kl, 64, D, lane, 64);
  typename M::frag qf[1][G::NS];
  if (p.vec) {
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const uint32_t c = lane + 64 * i, col = c / chunks;
      if (col < p.cols) *reinterpret_cast<u32x4*>(vl + col * G::P + (c - col * chunks) * G::E) = qp[i];
    }
    // columns past the last hold what the LDS held: their results are dropped
#pragma unroll
    for (int st = 0; st < G::NS; ++st)
      qf[0][st] = *reinterpret_cast<const typename M::frag*>(vl + l32 * G::P + 2 * G::E * st + G::E * g);
  } else {
    row_frags<T, DC>((uint32_t)l32 < p.cols ? qg + at_row(ch, cq, p.qs[2]) : nullptr, g, D, false, qf[0]);
  }
  table.build(p.bias, lo, n_tab, tab, p.tab, p.H, h0, p.grp);
  const float left[1] = {bias_at<T>(p.bias, p.H, h0 + ch, -p.bias.M)};
  const float right[1] = {bias_at<T>(p.bias, p.H, h0 + ch, p.bias.M)};
  const int32_t first[1] = {q0}, at[1] = {q0 + (int32_t)cq};
  const float* const tb[1] = {tab + (int64_t)ch * p.tab - lo - at[0]};

  Softmax<T, DC, 1, 1, false> sm;
  sm.init();
  __syncthreads();   // the table
  for (uint32_t kb = mine; kb < k1; kb += 32 * NW) {
    tk.stash(map, kl);
    tv.stash(map, vl);
    if (!ONE && kb + 32 * NW < k1) fetch(kb + 32 * NW);
    sm.step(
        [&](int, int st) {
          return *reinterpret_cast<const typename M::frag*>(kl + l32 * G::P + 2 * G::E * st + G::E * g);
        },
        vl, qf, {(int32_t)kb, (int32_t)k1, p.bias.M, p.causal}, p.c, first, at, tb, left, right, lane);
    if (ONE) break;
  }
  float l = sm.sum[0] + swap_halves(sm.sum[0]);

  T* og = static_cast<T*>(p.o) + (int64_t)b * p.os[0] + (int64_t)x * p.os[1];
  if constexpr (NW == 1) {
    sm.o[0].scale(no_keys(l) ? 0.0f : 1.0f / l, lane);
    auto row = [&](int n) -> T* {
      const uint32_t hh = (uint32_t)n / p.Lq;
      return (uint32_t)n < p.cols ? og + at_row(hh, n - hh * p.Lq, p.os[2]) : nullptr;
    };
    if (p.vec) store_rows_lds<T, DC>(vl, sm.o[0], lane, D, G::DP, row);
    else store_rows<T, DC>(sm.o[0], lane, D, false, row);
    if (p.lse && g == 0 && (uint32_t)l32 < p.cols)
      p.lse[((uint64_t)bx * p.H + h0 + ch) * p.Lq + cq] = no_keys(l) ? -INFINITY : kLn2 * (sm.ref[0] + log2f(l));
  } else {
    // the waves' columns meet at the largest of their references, and are added in
    // the waves' order; the tiles and the table are done with
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
    float* rows = ms + (2 * NW + 2) * 32;   // [NW][cols][DC]
    store_rows<T, DC>(sm.o[0], lane, G::DP, true, [&](int n) -> float* {
      return (uint32_t)n < p.cols ? rows + (wave * p.cols + n) * G::DP : nullptr;
    });
    if (wave == 0 && g == 0) {
      ms[2 * NW * 32 + l32] = top;
      ms[(2 * NW + 1) * 32 + l32] = l;
    }
    __syncthreads();
    float* part = p.part + ((uint64_t)(bx * kvh + e) * p.n_split + split) * p.cols * (2 + p.D);   // maxima, sums, rows
    for (uint32_t i = threadIdx.x; i < p.cols * p.D; i += NW * 64) {
      const uint32_t col = i / p.D, d = i - col * p.D;
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < NW; ++w) v += rows[(w * p.cols + col) * G::DP + d];
      if (p.n_split > 1) {
        part[2 * p.cols + i] = v;
      } else {
        const float s = ms[(2 * NW + 1) * 32 + col];
        const uint32_t hh = col / p.Lq;
        og[at_row(hh, col - hh * p.Lq, p.os[2]) + d] = (T)(no_keys(s) ? 0.0f : v / s);
      }
    }
    if (threadIdx.x < p.cols) {
      const float m = ms[2 * NW * 32 + threadIdx.x], s = ms[(2 * NW + 1) * 32 + threadIdx.x];
      if (p.n_split > 1) part[threadIdx.x] = m, part[p.cols + threadIdx.x] = s;
      else if (p.lse) {
        const uint32_t hh = threadIdx.x / p.Lq;
        p.lse[((uint64_t)bx * p.H + h0 + hh) * p.Lq + threadIdx.x - hh * p.Lq] =
            no_keys(s) ? -INFINITY : kLn2 * (m + log2f(s));
      }
    }
  }
}

// Joins the splits of one column: with their references m_s, sums l_s and rows o_s,
// o = sum 2^(m_s - m) o_s / sum 2^(m_s - m) l_s.  A work-group per column; 256 / DP
// groups of threads take every such split, and their sums are added in order.
constexpr int kMaxSplit = 512;
template <typename T, int DP>
__global__ __launch_bounds__(256) void relpos_join_kernel(FwdParams p) {
  constexpr int GR = 256 / DP;
  __shared__ float f[kMaxSplit], red[256], m4[4];
  const uint32_t unit = blockIdx.x / p.cols, col = blockIdx.x - unit * p.cols;
  const uint32_t stride = p.cols * (2 + p.D);
  const float* w = p.part + (uint64_t)unit * p.n_split * stride;
  float m = -INFINITY;
  for (uint32_t s = threadIdx.x; s < p.n_split; s += 256) {
    f[s] = w[(uint64_t)s * stride + col];
    m = fmaxf(m, f[s]);
  }
#pragma unroll
  for (int off = 32; off; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
  if ((threadIdx.x & 63) == 0) m4[threadIdx.x >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
  const float top = m == -INFINITY ? 0.0f : m;
  for (uint32_t s = threadIdx.x; s < p.n_split; s += 256) f[s] = __builtin_amdgcn_exp2f(f[s] - top);   // no keys: 0
  __syncthreads();
  const uint32_t d = threadIdx.x % DP, gr = threadIdx.x / DP;
  float a = 0.0f, l = 0.0f;
  if (d < p.D) {
#pragma unroll 4
    for (uint32_t s = gr; s < p.n_split; s += GR) {
      const float* ws = w + (uint64_t)s * stride;
      l += f[s] * ws[p.cols + col];
      a += f[s] * ws[2 * p.cols + col * p.D + d];
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
  const uint32_t kvh = p.H / p.grp, bx = unit / kvh, hh = col / p.Lq, i = col - hh * p.Lq;
  const uint32_t h = unit % kvh * p.grp + hh, b = bx / p.X, x = bx % p.X;
  static_cast<T*>(p.o)[(int64_t)b * p.os[0] + (int64_t)x * p.os[1] + (int64_t)i * p.os[2] + (int64_t)h * p.D + d] =
      (T)(no_keys(l) ? 0.0f : a / l);
  if (p.lse && d == 0) p.lse[((uint64_t)bx * p.H + h) * p.Lq + i] = no_keys(l) ? -INFINITY : kLn2 * (top + log2f(l));
}

struct Choice {
  bool few;
  int64_t n_split, split_keys;
};

// The few-queries form where a group's queries fit the 32 columns of a block (16384
// units of 32 queries 66 us, 92 by the form for many; 8192 units of one token 62 and 542).
// Its keys are cut while there are fewer work-groups than 8 for each CU (lengths differ,
// so more than the chip holds at once; 4, 8 and 16 are within 4% of each other), into
// pieces of at least 256 keys.
Choice choose(const RelposArgs& a) {
  Choice c = {};
  const int64_t grp = a.H / a.Hkv;
  c.n_split = 1;
  c.split_keys = a.Lk;
  c.few = a.Lq * grp <= 32;
  if (!c.few) return c;
  const int64_t units = std::max<int64_t>(a.B * a.X * a.Hkv, 1);
  const int64_t n = std::min<int64_t>({(256 * 8 + units - 1) / units, a.Lk / 256, kMaxSplit});
  if (n > 1) {
    c.split_keys = ((a.Lk + n - 1) / n + 127) / 128 * 128;
    c.n_split = (a.Lk + c.split_keys - 1) / c.split_keys;
  }
  return c;
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

template <typename T, int DC, int NW, int QT, int KB, int NBUF, int MINW>
int start_many(FwdParams& p, const RelposArgs& a, hipStream_t s) {
  constexpr int QB = NW * 32 * QT;
  p.order = make_order(a.B * a.X, a.Hkv, a.H / a.Hkv, (a.Lq + QB - 1) / QB, a.causal);
  p.tab = (uint32_t)std::min<int64_t>(2 * (p.bias.M + kEdge) + 1, QB + (a.Lk + KB - 1) / KB * KB);
  const size_t lds = (size_t)NBUF * 2 * KB * Geo<T, DC>::P * sizeof(T) + (size_t)p.tab * 4;
  return launch(relpos_fwd_kernel<T, DC, NW, QT, KB, NBUF, MINW>, order_blocks(p.order), NW * 64, lds, p, s);
}

template <typename T, int DC, int NW, bool ONE>
int start_few(FwdParams& p, const RelposArgs& a, hipStream_t s) {
  constexpr int MINW = sizeof(T) == 4 ? 1 : ONE ? (DC <= 80 ? 4 : DC <= 96 ? 3 : 2) : DC <= 80 ? 3 : 2;
  p.tab = (uint32_t)std::min<int64_t>(2 * (p.bias.M + kEdge) + 1, 32 + ((int64_t)p.split_keys + 31) / 32 * 32);
  // A group whose tables do not fit beside the tiles (long tables, many heads) is taken
  // in parts, each of which reads the keys; one head always fits.
  const uint32_t grp = p.grp;
  const size_t tiles = (size_t)NW * 2 * 32 * Geo<T, DC>::P * sizeof(T);
  p.sub = 1;
  while (grp % p.sub || tiles + (size_t)p.tab * (grp / p.sub) * 4 > 160 * 1024) ++p.sub;
  p.grp = grp / p.sub;
  p.cols = (uint32_t)a.Lq * p.grp;
  size_t lds = tiles + (size_t)p.tab * p.grp * 4;
  if (NW > 1) lds = std::max(lds, ((2 * NW + 2) * 32 + (size_t)NW * p.cols * Geo<T, DC>::DP) * 4);
  const int64_t pieces = a.B * a.X * p.n_split;
  p.pieces = (uint32_t)pieces;
  int st = launch(relpos_few_kernel<T, DC, NW, ONE, MINW>, (pieces + 7) / 8 * 8 * (a.H / p.grp), NW * 64, lds, p, s);
  if (st != DSP_OK || p.n_split == 1) return st;
  const int64_t cols = a.B * a.X * a.H * a.Lq;   // few units: they are why the keys are split
  if (a.D <= 64) relpos_join_kernel<T, 64><<<dim3((uint32_t)cols), 256, 0, s>>>(p);
  else relpos_join_kernel<T, 128><<<dim3((uint32_t)cols), 256, 0, s>>>(p);
  return last_launch_status();
}

template <typename T, int DC>
int start(FwdParams& p, const RelposArgs& a, bool few, hipStream_t s) {
  if (few) {
    // One wave and one tile where there is one (1600 units of 32 queries and keys 11 us,
    // four waves 21); a wave per unit, without the join, where the units alone fill the
    // chip, 12 waves to a CU, and their keys are few (8192 units of 120 keys 62 us
    // against 107 with four waves, 3200 of 200 39 against 47, of 400 78 and 77, of 2000
    // 372 and 322); two tiles at once (2400 units of 64 keys 19 against 27).
    const bool full = a.B * a.X * a.Hkv >= 256 * 12 && a.Lk <= 384;
    if (a.Lk <= 32) return start_few<T, DC, 1, true>(p, a, s);
    if (full) return start_few<T, DC, 1, false>(p, a, s);
    if (a.Lk <= 64) return start_few<T, DC, 2, true>(p, a, s);
    return start_few<T, DC, 4, false>(p, a, s);
  }
  constexpr bool B16 = sizeof(T) == 2;
  // one tile of keys (and of queries): 21600 units of 49 158 us, by the loop below 360
  if (a.Lq <= 64 && a.Lk <= 64) return start_many<T, DC, 2, 1, 64, 1, B16 ? (DC <= 80 ? 3 : 2) : 1>(p, a, s);
  // Long rows.  Heads of at most 64 columns: 4 waves of 32 queries, 3 of such work-groups
  // to a CU (8 x 16 units of 4096 x 64: 627 us; 8 waves of 64 queries 630, and 81 instead
  // of 60 us for 64 x 16 units of 300).  Wider heads have registers for 2 waves per SIMD,
  // and large blocks of queries, 64 to a wave up to 80 columns, ask less of LDS: 880 us
  // against 913 for 4096 x 72, 1160 against 1215 for 4096 x 128.  Where they leave CUs
  // idle or much of a block empty it is the other way round: 64 x 16 units of 300 x 72
  // 106 and 96, of 300 x 128 160 and 125, four units of 2000 x 96 60 and 55.
  if constexpr (B16 && DC > 64) {
    constexpr int QT = DC <= 80 ? 2 : 1;
    if (a.Lq >= 1024 && a.B * a.X * a.H * ((a.Lq + 256 * QT - 1) / (256 * QT)) >= 256)
      return start_many<T, DC, 8, QT, 64, 2, 2>(p, a, s);
  }
  return start_many<T, DC, 4, 1, B16 ? 64 : 32, 2, B16 ? (DC <= 64 ? 3 : 2) : 1>(p, a, s);
}

}  // namespace

int launch_attn_relpos(const RelposArgs& a, hipStream_t s) {
  const Choice c = choose(a);
  FwdParams p = {};
  p.q = a.q, p.k = a.k, p.v = a.v, p.o = a.o, p.lse = a.lse, p.part = a.workspace;
  p.q_pos = a.q_pos, p.kv_len = a.kv_len;
  for (int i = 0; i < 3; ++i) p.qs[i] = a.q_strides[i], p.ks[i] = a.kv_strides[i], p.os[i] = a.o_strides[i];
  p.bias = {a.bias, a.buckets, a.max_dist, a.n_buckets};
  p.X = (uint32_t)a.X, p.H = a.H, p.grp = a.H / a.Hkv, p.Lq = (uint32_t)a.Lq, p.Lk = (uint32_t)a.Lk, p.D = a.D;
  p.n_split = (uint32_t)c.n_split, p.split_keys = (uint32_t)c.split_keys;
  p.c = a.scale * kLog2e;
  p.vec = a.vec, p.causal = a.causal;
  if (a.bf16) {
    if (a.D <= 32) return start<bf16, 32>(p, a, c.few, s);
    if (a.D <= 48) return start<bf16, 48>(p, a, c.few, s);
    if (a.D <= 64) return start<bf16, 64>(p, a, c.few, s);
    if (a.D <= 72) return start<bf16, 72>(p, a, c.few, s);
    if (a.D <= 80) return start<bf16, 80>(p, a, c.few, s);
    if (a.D <= 96) return start<bf16, 96>(p, a, c.few, s);
    return start<bf16, 128>(p, a, c.few, s);
  }
  if (a.D <= 32) return start<float, 32>(p, a, c.few, s);
  if (a.D <= 64) return start<float, 64>(p, a, c.few, s);
  if (a.D <= 96) return start<float, 96>(p, a, c.few, s);
  return start<float, 128>(p, a, c.few, s);
}

size_t attn_relpos_workspace_bytes(const RelposArgs& a) {
  const Choice c = choose(a);
  return c.n_split > 1 ? (size_t)(a.B * a.X * a.H * c.n_split * a.Lq) * (2 + (size_t)a.D) * 4 : 0;
}

}  // namespace dsp
