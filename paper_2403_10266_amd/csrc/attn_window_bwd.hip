// Gradient of attention with a window and first tokens that stay visible.  With
//   z_ij = scale q_i . k_j over the keys j that query i sees,  P = softmax(z),
//   Delta_i = sum_d dO_id O_id,  dZ = P (dP - Delta),  dP = dO V^T:
//   dV = P^T dO,  dQ = scale dZ K,  dK = scale dZ^T Q.
// P is recomputed from the forward's row log-sum-exp.  Two kernels, both deterministic:
// the first owns blocks of (query, head) columns of a key/value head's group and visits
// the keys that they see (dQ and Delta = sum_j P dP, as O is rounded in bf16), the second owns blocks of keys and visits the
// queries that see them, head by head of the group (dK, dV).
//
// A first token that stays visible is seen by every later query, so its block of keys has
// a window's queries many times over.  Where units are few, those queries are cut into parts,
// work-groups of about a window's work whose fp32 sums a third kernel adds in order.
//
// P and dZ are rounded to bf16 for the products that take them as operands (the matrix
// cores' type; their sums are fp32).
#include <algorithm>

#include "attn_window.h"

namespace dsp {
namespace {

struct BwdParams {
  const void* q;
  const void* k;
  const void* v;
  const void* o;
  const void* dout;
  const float* lse;
  void* dq;
  void* dk;
  void* dv;
  float* delta;      // [B X H][Lq]
  float* part;       // sinks in several parts: [unit and head][block][part][dK, dV][keys][D]
  const int32_t* q_pos;
  const int32_t* kv_len;
  int64_t qs[3], ks[3], os[3];
  Window win;
  uint32_t X, H, Hkv, Lq, Lk, D;
  Divisor grp;
  Order order;
  uint32_t parts, sink_blocks;   // parts of the first blocks of keys (0: they are like the others, 1: they only go first)
  uint32_t sink_groups;          // work-groups for them, the first of the grid
  float c, scale;
  bool vec;
};

__device__ __forceinline__ int64_t bx_at(const BwdParams& p, uint32_t bx, const int64_t* st) {
  return (int64_t)(bx / p.X) * st[0] + (int64_t)(bx % p.X) * st[1];
}

// The operands of a block's products, read from LDS ahead of them: the order is the one
// written (in bf16, where a wave would otherwise wait for LDS before every MFMA).
template <typename T>
__device__ __forceinline__ void ahead() {
  if constexpr (sizeof(T) == 2) __builtin_amdgcn_sched_barrier(0);
}
template <typename T, int DC>
__device__ __forceinline__ void row_operand(const T* lds, int row0, int l32, int g, typename Mx<T>::frag (&a)[Geo<T, DC>::NS]) {
  using G = Geo<T, DC>;
#pragma unroll
  for (int st = 0; st < G::NS; ++st)
    a[st] = *reinterpret_cast<const typename Mx<T>::frag*>(lds + (row0 + l32) * G::P + 2 * G::E * st + G::E * g);
}
template <typename T, int DC>
__device__ __forceinline__ void row_product(floatx16& s, const typename Mx<T>::frag (&a)[Geo<T, DC>::NS],
                                            const typename Mx<T>::frag (&b)[Geo<T, DC>::NS]) {
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = 0.0f;
#pragma unroll
  for (int st = 0; st < Geo<T, DC>::NS; ++st) s = Mx<T>::mma(a[st], b[st], s);
}

// dQ and Delta: 32 columns per wave, keys on the rows of the products.  Chains of product,
// exponential and product bound it, at two waves to a SIMD, one for heads above 96 (matrix cores
// 22 - 26%, waits 36 - 45%): 8 x 16 units of 4096 x 72, window 257, 193 us; 4 sequences of 4000, 32
// heads of 64 over 8, window 501, 134 us (without the correction of Delta 186 and, with three waves, 102).
template <typename T, int DC, int NW, int KB, int MINW>
__global__ __launch_bounds__(NW * 64, MINW) void window_bwd_dq_kernel(BwdParams p) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  using R = Rows16<T, T, DC>;
  constexpr int NT = NW * 64, CB = NW * 32, NKT = KB / 32, GR = KB / 16, TILE = KB * G::P;
  constexpr int NL = 2 * GR / NW;
  static_assert(2 * GR % NW == 0 && NW <= 4 * NKT, "every wave loads the same; the output rows fit the tiles");
  extern __shared__ __attribute__((aligned(16))) char smem[];
  T* lds = reinterpret_cast<T*>(smem);   // [2][K, V][KB][P]

  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Place pl = place(p.order);
  if (!pl.any) return;
  const uint32_t bx = pl.bx, e = pl.h, blk = p.order.blocks - 1 - pl.block, b = bx / p.X;
  const uint32_t c0 = blk * CB, nc = min(p.Lq * p.grp.d - c0, (uint32_t)CB);
  const int D = (int)p.D;
  const int64_t k_at = bx_at(p, bx, p.ks) + (int64_t)e * D;
  const T* kg = static_cast<const T*>(p.k) + k_at;
  const T* vg = static_cast<const T*>(p.v) + k_at;
  const int32_t len = (int32_t)length(p.kv_len, b, p.Lk);
  const int64_t p0 = first_position(p.q_pos, b);
  const Columns cs(p.grp, c0);
  auto seen_by = [&](uint32_t n) { return seen(p.win, p0 + cs.query(min(n, nc - 1)), len); };
  const Seen first = seen_by(0), last = seen_by(CB - 1);
  const Tiles<KB> tiles(first, last);

  const uint32_t row_bytes = (uint32_t)p.ks[2] * (uint32_t)sizeof(T);
  const typename R::Map map = R::map(D, row_bytes, lane);
  R rows[NL];
  auto fetch = [&](int32_t t) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int li = wave + i * NW;
      const int32_t key0 = tiles.key0(t) + 16 * (li % GR);
      rows[i].fetch(map, (li < GR ? kg : vg) + (int64_t)key0 * p.ks[2], D, p.vec, whole_group(first, last, key0), [&](int r) {
        const int32_t j = key0 + r;
        return j < last.sink || (j >= first.lo && j < last.hi);
      });
    }
  };
  auto stash = [&](int buf) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int li = wave + i * NW;
      rows[i].stash(map, lds + buf * 2 * TILE + (li < GR ? 0 : TILE) + 16 * (li % GR) * G::P, 1.0f);
    }
  };
  if (tiles.n) fetch(0);
  const uint32_t n = 32 * wave + l32, qi = cs.query(min(n, nc - 1)), qh = e * p.grp.d + cs.head(min(n, nc - 1), qi);
  const bool on = n < nc;
  const int64_t q_at = bx_at(p, bx, p.qs), o_at = bx_at(p, bx, p.os);
  auto at = [&](const void* base, int64_t from, int64_t row) {
    return on ? static_cast<const T*>(base) + from + (int64_t)qi * row + (int64_t)qh * D : nullptr;
  };
  typename M::frag qf[G::NS], df[G::NS];
  row_frags<T, DC>(at(p.q, q_at, p.qs[2]), g, D, p.vec, qf);
  row_frags<T, DC>(at(p.dout, o_at, p.os[2]), g, D, p.vec, df);
  float delta = 0.0f;
  {
    typename M::frag of[G::NS];
    row_frags<T, DC>(at(p.o, o_at, p.os[2]), g, D, p.vec, of);
#pragma unroll
    for (int s = 0; s < G::NS; ++s)
#pragma unroll
      for (int k = 0; k < G::E; ++k) delta += (float)df[s][k] * (float)of[s][k];
    delta += swap_halves(delta);
  }
  const uint64_t stat = ((uint64_t)bx * p.H + qh) * p.Lq + qi;
  // a row that sees nothing, or past the end: P = exp2(-inf) = 0
  const float l = on ? p.lse[stat] : -INFINITY;
  const float lse2 = l == -INFINITY ? INFINITY : l * kLog2e;
  const Seen col = seen(p.win, p0 + qi, len);
  const Seen wf = seen_by(32 * wave), wl = seen_by(32 * wave + 31);
  const bool wave_on = 32 * wave < nc;
  clear_cols<T, DC>(lds, 4 * KB, D, threadIdx.x, NT);
  if (tiles.n) stash(0);
  __syncthreads();

  // bf16: Delta from the rounded o misses sum_j P dP by `off`, the sum of the column's dZ, and dQ by
  // off times sum_j P k_j: one more product, of operands that are there.  Without it dQ and dK err
  // 1.4 times as much where rows see few keys, and without limit where dP varies less over a row's
  // keys than o's rounding does.
  constexpr bool FIX = sizeof(T) == 2;
  ColAcc<T, DC> dq, pk;
  dq.zero();
  pk.zero();
  float off = 0.0f;
  for (int32_t it = 0; it < tiles.n; ++it) {
    const bool more = it + 1 < tiles.n;
    if (more) fetch(it + 1);
    const T* kl = lds + (it & 1) * 2 * TILE;
    const T* vl = kl + TILE;
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt) {
      const int32_t key0 = tiles.key0(it) + 32 * kt;
      if (!wave_on || (key0 >= wl.sink && (key0 + 32 <= wf.lo || key0 >= wl.hi))) continue;
      const bool mask = !(key0 + 32 <= wf.sink || (key0 >= wl.lo && key0 + 32 <= wf.hi));
      floatx16 s, dp;
      typename M::frag ka[G::NS], va[G::NS];
      row_operand<T, DC>(kl, 32 * kt, l32, g, ka);
      ahead<T>();
      row_product<T, DC>(s, ka, qf);
      row_operand<T, DC>(vl, 32 * kt, l32, g, va);
      ahead<T>();
      row_product<T, DC>(dp, va, df);
      ColA<T, DC> kt_a;
      kt_a.load(kl, 32 * kt, lane);
      ahead<T>();
      const uint32_t bits = mask ? seen_bits(col, key0) >> (4 * g) : ~0u;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], p.c, -lse2));
      if (mask) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = keep_bit(s[r], bits, 8 * (r / 4) + r % 4);
      }
      ColB<T> z, pb;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float dz = s[r] * (dp[r] - delta);
        z.set(r, dz);
        if constexpr (FIX) {
          off += dz;
          pb.set(r, s[r]);
        }
      }
      dq.add(kt_a, z);
      if constexpr (FIX) pk.add(kt_a, pb);
    }
    if (more) stash((it + 1) & 1);
    __syncthreads();
  }
  if constexpr (FIX) {
    off += swap_halves(off);
    dq.add(-off, pk, lane);
    delta += off;
  }
  if (on && g == 0) p.delta[stat] = delta;
  dq.scale(p.scale, lane);
  T* out = static_cast<T*>(p.dq) + q_at + (int64_t)e * p.grp.d * D;
  auto row = [&](int k) -> T* {
    const uint32_t n = 32 * wave + k, i = cs.query(n);
    return n < nc ? out + (int64_t)i * p.qs[2] + (int64_t)cs.head(n, i) * D : nullptr;
  };
  if (p.vec) store_rows_lds<T, DC>(lds + wave * 32 * G::P, dq, lane, D, G::DP, row);
  else store_rows<T, DC>(dq, lane, D, false, row);
}

// The queries that see key j: first <= i < end.
struct SeenBy {
  int32_t first, end;
};
__device__ __forceinline__ SeenBy seen_by(const Window& w, int64_t p0, int32_t n, int32_t len, int64_t j) {
  auto clamp = [n](int64_t v) { return (int32_t)(v < 0 ? 0 : v > n ? n : v); };
  SeenBy s;
  s.first = w.right < 0 ? 0 : clamp(j - w.right - p0);
  s.end = j >= len ? 0 : w.left < 0 || j < w.sinks ? n : clamp(j + w.left - p0 + 1);
  return s;
}

// dK and dV, over the queries of every head of the key/value head's group, in tiles of
// 32 QT: a wave per 32 keys, whose K, V and sums it holds (two waves to a SIMD that wait half of their
// time, and in the second call a grid that fills the chip one and a third times).  The same two calls:
// 223 and 177 us.
template <typename T, int DC, int KW, int QT, int MINW>
__global__ __launch_bounds__(KW * 64, MINW) void window_bwd_dkv_kernel(BwdParams p) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  constexpr int NT = KW * 64, QB = 32 * QT, TILE = QB * G::P, KEYS = 32 * KW;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  T* lds = reinterpret_cast<T*>(smem);                            // [2][Q, dO][QB][P]
  float* stat = reinterpret_cast<float*>(lds + 4 * TILE);         // [2][lse2, Delta][QB]

  const int lane0 = threadIdx.x & 63, lane = lane0, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t blk, bx, e, part = 0;
  const bool sink = blockIdx.x < p.sink_groups;
  if (sink) {
    const uint32_t u = blockIdx.x / p.parts, ub = u / p.sink_blocks;
    part = blockIdx.x - u * p.parts;
    blk = u - ub * p.sink_blocks;
    bx = ub / p.Hkv;
    e = ub - bx * p.Hkv;
  } else {
    const Place pl = place(p.order, blockIdx.x - p.sink_groups);
    if (!pl.any || (p.parts && pl.block < p.sink_blocks)) return;
    blk = pl.block, bx = pl.bx, e = pl.h;
  }
  const uint32_t b = bx / p.X;
  const int D = (int)p.D;
  const int64_t k_at = bx_at(p, bx, p.ks) + (int64_t)e * D;
  const int64_t q_bx = bx_at(p, bx, p.qs), o_bx = bx_at(p, bx, p.os);
  const int32_t first_key = (int32_t)(blk * KEYS), key = first_key + 32 * wave + l32;
  const int32_t len = (int32_t)length(p.kv_len, b, p.Lk);
  const int64_t p0 = first_position(p.q_pos, b);
  const SeenBy mine = seen_by(p.win, p0, (int32_t)p.Lq, len, key);
  // of the wave's keys: the tiles that any is seen from, and those that all are
  int32_t any0 = mine.first < mine.end ? mine.first : INT32_MAX, any1 = mine.end, all0 = mine.first, all1 = mine.end;
#pragma unroll
  for (int off = 16; off; off >>= 1) {
    any0 = min(any0, __shfl_xor(any0, off));
    any1 = max(any1, __shfl_xor(any1, off));
    all0 = max(all0, __shfl_xor(all0, off));
    all1 = min(all1, __shfl_xor(all1, off));
  }
  any0 = __builtin_amdgcn_readfirstlane(any0), any1 = __builtin_amdgcn_readfirstlane(any1);
  all0 = __builtin_amdgcn_readfirstlane(all0), all1 = __builtin_amdgcn_readfirstlane(all1);
  typename M::frag kf[G::NS], vf[G::NS];
  const bool there = mine.first < mine.end;   // a key that nothing sees may hold anything
  row_frags<T, DC>(there ? static_cast<const T*>(p.k) + k_at + (int64_t)key * p.ks[2] : nullptr, g, D, p.vec, kf);
  row_frags<T, DC>(there ? static_cast<const T*>(p.v) + k_at + (int64_t)key * p.ks[2] : nullptr, g, D, p.vec, vf);

  const uint32_t q_row = (uint32_t)p.qs[2] * (uint32_t)sizeof(T), o_row = (uint32_t)p.os[2] * (uint32_t)sizeof(T);
  using TileT = Tile<T, DC, QB, NT>;
  const typename TileT::Map mq = TileT::map(D, q_row, threadIdx.x), mo = TileT::map(D, o_row, threadIdx.x);
  TileT tq, to;
  static_assert(NT >= 2 * QB, "a statistic for each thread");
  float pre = 0.0f;
  clear_cols<T, DC>(lds, 4 * QB, D, threadIdx.x, NT);

  ColAcc<T, DC> dk, dv;
  dk.zero();
  dv.zero();
  // the tiles of queries that see the work-group's keys, head after head
  const int32_t key_end = min(first_key + KEYS, len);
  const SeenBy lowest = seen_by(p.win, p0, (int32_t)p.Lq, len, first_key);
  const SeenBy highest = seen_by(p.win, p0, (int32_t)p.Lq, len, (int64_t)key_end - 1);
  const int32_t q_end = first_key < key_end ? max(lowest.end, highest.end) : 0;
  const uint32_t it0 = (uint32_t)lowest.first / QB, n_it = q_end > lowest.first ? ((uint32_t)q_end + QB - 1) / QB - it0 : 0;
  uint32_t step = 0, steps = n_it * p.grp.d;
  if (sink) {
    const uint32_t per = (steps + p.parts - 1) / p.parts;
    step = min(part * per, steps);
    steps = min(step + per, steps);
  }
  uint32_t hh = n_it ? step / n_it : 0, it = step - hh * n_it;   // the step to fetch
  auto fetch = [&]() {
    const uint32_t h = e * p.grp.d + hh, q0 = (it0 + it) * QB, rows = min(p.Lq - q0, (uint32_t)QB);
    tq.fetch(mq, static_cast<const T*>(p.q) + q_bx + (int64_t)h * D + (int64_t)q0 * p.qs[2], rows, q_row, D, p.vec);
    to.fetch(mo, static_cast<const T*>(p.dout) + o_bx + (int64_t)h * D + (int64_t)q0 * p.os[2], rows, o_row, D, p.vec);
    if (threadIdx.x < 2 * QB) {
      const uint32_t i = threadIdx.x % QB;
      const bool is_delta = threadIdx.x >= QB;
      const uint64_t at = ((uint64_t)bx * p.H + h) * p.Lq + q0 + i;
      const float l = i < rows ? (is_delta ? p.delta : p.lse)[at] : is_delta ? 0.0f : -INFINITY;
      pre = is_delta ? l : l == -INFINITY ? INFINITY : l * kLog2e;
    }
  };
  auto stash = [&](int buf) {
    tq.stash(mq, lds + buf * 2 * TILE);
    to.stash(mo, lds + buf * 2 * TILE + TILE);
    if (threadIdx.x < 2 * QB) stat[buf * 2 * QB + threadIdx.x] = pre;
  };
  if (step < steps) {
    fetch();
    stash(0);
  }
  __syncthreads();
  for (int buf = 0; step < steps; ++step, buf ^= 1) {
    const int32_t qt0 = (int32_t)((it0 + it) * QB);   // the tile's first query
    const bool more = step + 1 < steps;
    if (++it == n_it) it = 0, ++hh;
    if (more) fetch();
    int lane = lane0;
    asm volatile("" : "+v"(lane));   // addresses made of it are cheaper to form again than to keep
    const int l32 = lane & 31, g = lane >> 5;
    const T* ql = lds + buf * 2 * TILE;
    const T* ol = ql + TILE;
    const float* sl = stat + buf * 2 * QB;
#pragma unroll
    for (int sub = 0; sub < QT; ++sub) {
      const int32_t q0 = qt0 + 32 * sub;
      if (q0 >= any1 || q0 + 32 <= any0) continue;
      const bool mask = q0 < all0 || q0 + 32 > all1;
      floatx16 s, dp;
      typename M::frag qa[G::NS], oa[G::NS];
      row_operand<T, DC>(ql, 32 * sub, l32, g, qa);
      row_operand<T, DC>(ol, 32 * sub, l32, g, oa);
      ahead<T>();
      row_product<T, DC>(s, qa, kf);
      ColA<T, DC> o_a, q_a;
      o_a.load(ol, 32 * sub, lane);
      ahead<T>();
      row_product<T, DC>(dp, oa, vf);
      // lane (n + 32 g): key n, queries 8 (r / 4) + 4 g + r % 4
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const floatx4 l = *reinterpret_cast<const floatx4*>(sl + 32 * sub + 8 * q + 4 * g);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[4 * q + j] = __builtin_amdgcn_exp2f(fmaf(s[4 * q + j], p.c, -l[j]));
      }
      if (mask) {
        const uint32_t bits = (low_bits(mine.end - q0) & ~low_bits(mine.first - q0)) >> (4 * g);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = keep_bit(s[r], bits, 8 * (r / 4) + r % 4);
      }
      ColB<T> pb, zb;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const floatx4 dl = *reinterpret_cast<const floatx4*>(sl + QB + 32 * sub + 8 * q + 4 * g);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          pb.set(4 * q + j, s[4 * q + j]);
          zb.set(4 * q + j, s[4 * q + j] * (dp[4 * q + j] - dl[j]));
        }
      }
      q_a.load(ql, 32 * sub, lane);
      ahead<T>();
      dv.add(o_a, pb);
      dk.add(q_a, zb);
    }
    if (more) stash(buf ^ 1);
    __syncthreads();
  }
  dk.scale(p.scale, lane);
  T* const out[2] = {static_cast<T*>(p.dk) + k_at, static_cast<T*>(p.dv) + k_at};
  float* const sums_at = p.part + ((((uint64_t)bx * p.Hkv + e) * p.sink_blocks + blk) * p.parts + part) * 2 * KEYS * p.D;
  const uint32_t k0 = first_key + 32 * wave;
  auto row = [&](T* base, int n) -> T* { return k0 + n < p.Lk ? base + (int64_t)(k0 + n) * p.ks[2] : nullptr; };
  auto part_row = [&](int which, int n) -> float* { return sums_at + ((uint64_t)which * KEYS + 32 * wave + n) * p.D; };
  if (sink && p.parts > 1) {
    const bool vec4 = p.D % 4 == 0;
    store_rows<T, DC>(dk, lane, D, vec4, [&](int n) { return part_row(0, n); });
    store_rows<T, DC>(dv, lane, D, vec4, [&](int n) { return part_row(1, n); });
  } else if (p.vec) {
    T* so = lds + wave * 32 * G::P;   // the tiles are done with
    static_assert(KW * 32 <= 4 * QB, "rows to write through");
    store_rows_lds<T, DC>(so, dk, lane, D, G::DP, [&](int n) { return row(out[0], n); });
    store_rows_lds<T, DC>(so, dv, lane, D, G::DP, [&](int n) { return row(out[1], n); });
  } else {
    store_rows<T, DC>(dk, lane, D, false, [&](int n) { return row(out[0], n); });
    store_rows<T, DC>(dv, lane, D, false, [&](int n) { return row(out[1], n); });
  }
}

// dK and dV of the first blocks of keys: their parts added in order.
template <typename T>
__global__ __launch_bounds__(256) void window_bwd_sink_kernel(BwdParams p, uint32_t keys) {
  const uint32_t ub = blockIdx.x / p.sink_blocks, blk = blockIdx.x - ub * p.sink_blocks;
  const uint32_t bx = ub / p.Hkv, e = ub - bx * p.Hkv, n = keys * p.D;
  const float* from = p.part + (uint64_t)blockIdx.x * p.parts * 2 * n;
  const int64_t k_at = bx_at(p, bx, p.ks) + (int64_t)e * p.D;
  for (uint32_t i = blockIdx.y * 256 + threadIdx.x; i < 2 * n; i += gridDim.y * 256) {
    float v = 0.0f;
#pragma unroll 8
    for (uint32_t s = 0; s < p.parts; ++s) v += from[(uint64_t)s * 2 * n + i];
    const uint32_t which = i >= n, at = i - which * n, key = at / p.D, d = at - key * p.D, j = blk * keys + key;
    if (j < p.Lk) (static_cast<T*>(which ? p.dv : p.dk) + k_at)[(int64_t)j * p.ks[2] + d] = (T)v;
  }
}

// Short units, of at most 32 NW keys and columns: one work-group reads each row once.  Wave w
// first takes columns 32 w .. against all keys, which lie in LDS (Delta = sum_j P dP, with
// no need of o, then dQ); then its Q and dO, which it held in registers as operands, take the
// place of the keys in LDS, it keeps keys 32 w .. in registers, and dK and dV follow with the
// scores computed the other way round.  Memory bounds those of one or two blocks: 1350 x 16 units of
// 49 x 72 265 us, 2048 x 16 of 32 254, 4.0 - 4.2 TB/s.  At 128 it is the scores, formed three times by
// two waves to a SIMD: 1024 x 16 units 665 us, 3.2 TB/s (940 with the two kernels for long units).
template <typename T, int DC, int NW, int MINW>
__global__ __launch_bounds__(NW * 64, MINW) void window_bwd_short_kernel(BwdParams p) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  using R = Rows16<T, T, DC>;
  constexpr int NT = NW * 64, N = NW * 32, TILE = N * G::P;
  constexpr int NL = 4;   // group loads of a wave: two of K, two of V
  extern __shared__ __attribute__((aligned(16))) char smem[];
  T* t0 = reinterpret_cast<T*>(smem);      // K, then Q: [N][P]
  T* t1 = t0 + TILE;                       // V, then dO
  float* st_lse = reinterpret_cast<float*>(t1 + TILE);   // [N], exp2 units
  float* st_del = st_lse + N;

  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Place pl = place(p.order);
  if (!pl.any) return;
  const uint32_t bx = pl.bx, e = pl.h, b = bx / p.X, nc = p.Lq * p.grp.d;
  const int D = (int)p.D;
  const int64_t k_at = bx_at(p, bx, p.ks) + (int64_t)e * D, q_at = bx_at(p, bx, p.qs), o_at = bx_at(p, bx, p.os);
  const int32_t len = (int32_t)length(p.kv_len, b, p.Lk);
  const int64_t p0 = first_position(p.q_pos, b);
  const Columns cs(p.grp, 0);
  const Seen first = seen(p.win, p0, len), last = seen(p.win, p0 + p.Lq - 1, len);
  const typename R::Map map = R::map(D, (uint32_t)p.ks[2] * (uint32_t)sizeof(T), lane);
  R rows[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int32_t key0 = 32 * wave + 16 * (i & 1);
    rows[i].fetch(map, static_cast<const T*>(i < 2 ? p.k : p.v) + k_at + (int64_t)key0 * p.ks[2], D, p.vec,
                  whole_group(first, last, key0), [&](int r) {
                    const int32_t j = key0 + r;
                    return j < last.sink || (j >= first.lo && j < last.hi);
                  });
  }
  const uint32_t w0 = 32 * wave, n = w0 + l32, qi = cs.query(min(n, nc - 1)), qh = e * p.grp.d + cs.head(min(n, nc - 1), qi);
  const bool on = n < nc;
  auto at = [&](const void* base, int64_t from, int64_t row) {
    return on ? static_cast<const T*>(base) + from + (int64_t)qi * row + (int64_t)qh * D : nullptr;
  };
  typename M::frag qf[G::NS], df[G::NS];
  row_frags<T, DC>(at(p.q, q_at, p.qs[2]), g, D, p.vec, qf);
  row_frags<T, DC>(at(p.dout, o_at, p.os[2]), g, D, p.vec, df);
  const float l = on ? p.lse[((uint64_t)bx * p.H + qh) * p.Lq + qi] : -INFINITY;
  const float lse2 = l == -INFINITY ? INFINITY : l * kLog2e;   // sees nothing, or past the end: P = 0
  const Seen col = seen(p.win, p0 + qi, len);
  clear_cols<T, DC>(t0, 2 * N, D, threadIdx.x, NT);
#pragma unroll
  for (int i = 0; i < NL; ++i) rows[i].stash(map, (i < 2 ? t0 : t1) + (32 * wave + 16 * (i & 1)) * G::P, 1.0f);
  __syncthreads();

  // columns against the keys
  const bool wave_on = w0 < nc;
  const Seen wf = seen(p.win, p0 + cs.query(min(w0, nc - 1)), len), wl = seen(p.win, p0 + cs.query(min(w0 + 31, nc - 1)), len);
  float delta = 0.0f;
  ColAcc<T, DC> dq;
  dq.zero();
  auto block = [&](int key0, floatx16& s, floatx16& dp) {   // P and dP
    typename M::frag a[G::NS];
    row_operand<T, DC>(t0, key0, l32, g, a);
    row_product<T, DC>(s, a, qf);
    row_operand<T, DC>(t1, key0, l32, g, a);
    row_product<T, DC>(dp, a, df);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], p.c, -lse2));
    if (!(key0 + 32 <= wf.sink || (key0 >= wl.lo && key0 + 32 <= wf.hi))) {
      const uint32_t bits = seen_bits(col, key0) >> (4 * g);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = keep_bit(s[r], bits, 8 * (r / 4) + r % 4);
    }
  };
  auto none = [&](int key0) { return !wave_on || (key0 >= wl.sink && (key0 + 32 <= wf.lo || key0 >= wl.hi)); };
  for (int key0 = 0; key0 < N; key0 += 32) {
    if (none(key0)) continue;
    floatx16 s, dp;
    block(key0, s, dp);
#pragma unroll
    for (int r = 0; r < 16; ++r) delta += s[r] * dp[r];
  }
  delta += swap_halves(delta);
  for (int key0 = 0; key0 < N; key0 += 32) {
    if (none(key0)) continue;
    floatx16 s, dp;
    block(key0, s, dp);
    ColB<T> z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z.set(r, s[r] * (dp[r] - delta));
    dq.add(t0, key0, lane, z);
  }
  if (g == 0) st_lse[n] = lse2, st_del[n] = delta;
  typename M::frag kf[G::NS], vf[G::NS];
  row_operand<T, DC>(t0, w0, l32, g, kf);
  row_operand<T, DC>(t1, w0, l32, g, vf);
  __syncthreads();   // the keys are done with
  dq.scale(p.scale, lane);
  T* out = static_cast<T*>(p.dq) + q_at + (int64_t)e * p.grp.d * D;
  auto q_row = [&](int k) -> T* {
    const uint32_t c = w0 + k, i = cs.query(c);
    return c < nc ? out + (int64_t)i * p.qs[2] + (int64_t)cs.head(c, i) * D : nullptr;
  };
  if (p.vec) store_rows_lds<T, DC>(t0 + w0 * G::P, dq, lane, D, G::DP, q_row);
  else store_rows<T, DC>(dq, lane, D, false, q_row);
  wave_order();
#pragma unroll
  for (int st = 0; st < G::NS; ++st) {
    const int to = (w0 + l32) * G::P + 2 * G::E * st + G::E * g;
    *reinterpret_cast<typename M::frag*>(t0 + to) = qf[st];
    *reinterpret_cast<typename M::frag*>(t1 + to) = df[st];
  }
  __syncthreads();

  // keys against the columns: key j's are those of the queries that see it
  const int32_t key = (int32_t)w0 + l32, grp = (int32_t)p.grp.d;
  const SeenBy mine = seen_by(p.win, p0, (int32_t)p.Lq, len, key);
  const int32_t c_first = mine.first * grp, c_end = mine.end * grp;
  ColAcc<T, DC> dk, dv;
  dk.zero();
  dv.zero();
  for (int c0 = 0; c0 < N; c0 += 32) {
    const uint32_t all = low_bits(c_end - c0) & ~low_bits(c_first - c0);
    if (c0 >= (int32_t)nc || !__any(all != 0)) continue;
    const uint32_t bits = all >> (4 * g);
    floatx16 s, dp;
    typename M::frag a[G::NS];
    row_operand<T, DC>(t0, c0, l32, g, a);
    row_product<T, DC>(s, a, kf);
    row_operand<T, DC>(t1, c0, l32, g, a);
    row_product<T, DC>(dp, a, vf);
    ColB<T> pb, zb;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const floatx4 ll = *reinterpret_cast<const floatx4*>(st_lse + c0 + 8 * q + 4 * g);
      const floatx4 dl = *reinterpret_cast<const floatx4*>(st_del + c0 + 8 * q + 4 * g);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float pr = keep_bit(__builtin_amdgcn_exp2f(fmaf(s[4 * q + j], p.c, -ll[j])), bits, 8 * q + j);
        pb.set(4 * q + j, pr);
        zb.set(4 * q + j, pr * (dp[4 * q + j] - dl[j]));
      }
    }
    dv.add(t1, c0, lane, pb);
    dk.add(t0, c0, lane, zb);
  }
  __syncthreads();   // Q and dO are done with
  dk.scale(p.scale, lane);
  auto k_row = [&](void* base) {
    return [&, base](int k) -> T* {
      const uint32_t r = w0 + k;
      return r < p.Lk ? static_cast<T*>(base) + k_at + (int64_t)r * p.ks[2] : nullptr;
    };
  };
  if (p.vec) {
    store_rows_lds<T, DC>(t0 + w0 * G::P, dk, lane, D, G::DP, k_row(p.dk));
    store_rows_lds<T, DC>(t1 + w0 * G::P, dv, lane, D, G::DP, k_row(p.dv));
  } else {
    store_rows<T, DC>(dk, lane, D, false, k_row(p.dk));
    store_rows<T, DC>(dv, lane, D, false, k_row(p.dv));
  }
}

template <typename K>
int lds_limit(K* kernel, size_t lds) {
  if (lds <= 64 * 1024) return DSP_OK;
  return hip_status(
      hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
}

constexpr int kDkvKeys = 128;   // of a work-group
// Parts of the first keys' queries: about a window's work each, and no more work-groups than the
// chip's 512 places for them: more only write and read more sums.  One part: the first blocks of keys
// start first and write their gradients themselves.  Gradients in us with any number of parts, 512
// work-groups, 256: 64 x 16 units of 8000 x 72, window 65, 4 sinks 6670 (2.4 GB of sums), 5470
// (none), 5490; 8 x 16 of 8000 x 64, window 201, 768 (172 MB), 710 (38), 698; 8 of 8000 x 64 with 2000
// sinks 237, 177, 209.
constexpr int64_t kPlaces = 512;
struct Sinks {
  int64_t blocks, parts;   // parts 0: these blocks of keys are like the others
};
Sinks sinks_of(const WindowArgs& a) {
  Sinks s = {0, 0};
  if (a.win.sinks == 0 || a.win.left < 0 || a.Lq == 0 || a.Lk == 0) return s;
  const int64_t band = (int64_t)a.win.left + (a.win.right < 0 ? a.Lq : a.win.right) + kDkvKeys + 64;
  const int64_t parts = std::min<int64_t>(a.Lq / std::max<int64_t>(band, 256), 64);
  if (parts < 2) return s;
  s.blocks = (std::min<int64_t>(a.win.sinks, a.Lk) + kDkvKeys - 1) / kDkvKeys;
  s.parts = std::min(parts, std::max<int64_t>(kPlaces / (a.B * a.X * a.Hkv * s.blocks), 1));
  return s;
}

template <typename T, int DC>
int start_dq(BwdParams& p, const WindowArgs& a, hipStream_t s) {
  constexpr int NW = 4, CB = 32 * NW, KB = 32, MINW = DC <= 96 ? 2 : 1;
  p.order = window_order(a, (a.Lq * p.grp.d + CB - 1) / CB, CB / p.grp.d + 1);
  const size_t lds = (size_t)4 * KB * Geo<T, DC>::P * sizeof(T);
  auto* kernel = window_bwd_dq_kernel<T, DC, NW, KB, MINW>;
  if (!grid_fits(order_blocks(p.order), NW * 64)) return DSP_ERR_SHAPE;
  if (int st = lds_limit(kernel, lds)) return st;
  kernel<<<dim3((uint32_t)order_blocks(p.order)), NW * 64, lds, s>>>(p);
  return last_launch_status();
}

template <typename T, int DC, int KW, int QT, int MINW>
int start_dkv(BwdParams& p, const WindowArgs& a, hipStream_t s) {
  static_assert(32 * KW == kDkvKeys, "the sinks' workspace");
  constexpr int QB = 32 * QT;
  p.order = window_order(a, (a.Lk + 32 * KW - 1) / (32 * KW), 32 * KW);
  const Sinks sk = sinks_of(a);
  p.parts = (uint32_t)sk.parts, p.sink_blocks = (uint32_t)sk.blocks;
  const int64_t first = a.B * a.X * a.Hkv * sk.blocks * sk.parts, blocks = first + order_blocks(p.order);
  if (!grid_fits(blocks, KW * 64)) return DSP_ERR_SHAPE;
  p.sink_groups = (uint32_t)first;
  const size_t lds = (size_t)4 * QB * Geo<T, DC>::P * sizeof(T) + (size_t)4 * QB * 4;
  auto* kernel = window_bwd_dkv_kernel<T, DC, KW, QT, MINW>;
  if (int st = lds_limit(kernel, lds)) return st;
  kernel<<<dim3((uint32_t)blocks), KW * 64, lds, s>>>(p);
  if (int st = last_launch_status()) return st;
  if (sk.parts <= 1) return DSP_OK;
  const int64_t ub = a.B * a.X * a.Hkv * sk.blocks;
  window_bwd_sink_kernel<T><<<dim3((uint32_t)ub, 32), 256, 0, s>>>(p, 32 * KW);   // few units and parts: latency counts
  return last_launch_status();
}

// Waves of the short form, 0: the unit is too long.
int short_waves(const WindowArgs& a) {
  const int64_t most = std::max<int64_t>(a.Lq * (a.H / a.Hkv), a.Lk);
  return a.Lq == 0 || a.Lk == 0 || most > 128 ? 0 : most <= 32 ? 1 : most <= 64 ? 2 : 4;
}
template <typename T, int DC, int NW, int MINW>
int start_short(BwdParams& p, const WindowArgs& a, hipStream_t s) {
  p.order = make_order(a.B * a.X, a.Hkv, 1, 1, false);
  const size_t lds = (size_t)2 * 32 * NW * Geo<T, DC>::P * sizeof(T) + (size_t)2 * 32 * NW * 4;
  auto* kernel = window_bwd_short_kernel<T, DC, NW, MINW>;
  if (!grid_fits(order_blocks(p.order), NW * 64)) return DSP_ERR_SHAPE;
  if (int st = lds_limit(kernel, lds)) return st;
  kernel<<<dim3((uint32_t)order_blocks(p.order)), NW * 64, lds, s>>>(p);
  return last_launch_status();
}

template <typename T, int DC>
int start(BwdParams& p, const WindowArgs& a, hipStream_t s) {
  constexpr int MS = sizeof(T) == 4 ? 1 : DC <= 48 ? 3 : DC <= 96 ? 2 : 1;
  switch (short_waves(a)) {
    case 1: return start_short<T, DC, 1, MS>(p, a, s);
    case 2: return start_short<T, DC, 2, MS>(p, a, s);
    case 4: return start_short<T, DC, 4, MS>(p, a, s);
  }
  if (a.Lq > 0)
    if (int st = start_dq<T, DC>(p, a, s)) return st;
  if (a.Lk == 0) return DSP_OK;
  constexpr bool B16 = sizeof(T) == 2;
  return start_dkv<T, DC, 4, B16 ? 2 : 1, B16 && DC <= 80 ? 2 : 1>(p, a, s);
}

}  // namespace

size_t attn_window_bwd_workspace_bytes(const WindowArgs& a) {
  if (short_waves(a)) return 0;
  const int64_t stats = (a.B * a.X * a.H * a.Lq + 63) / 64 * 64;
  const Sinks s = sinks_of(a);
  const int64_t groups = s.parts > 1 ? a.B * a.X * a.Hkv * s.blocks * s.parts : 0;
  return (size_t)(stats + groups * 2 * kDkvKeys * a.D) * 4;
}

int launch_attn_window_bwd(const WindowArgs& a, hipStream_t s) {
  BwdParams p = {};
  p.q = a.q, p.k = a.k, p.v = a.v, p.o = a.o, p.dout = a.dout, p.lse = a.lse;
  p.dq = a.dq, p.dk = a.dk, p.dv = a.dv;
  p.delta = a.workspace;
  p.part = a.workspace + (a.B * a.X * a.H * a.Lq + 63) / 64 * 64;
  p.q_pos = a.q_pos, p.kv_len = a.kv_len;
  for (int i = 0; i < 3; ++i) p.qs[i] = a.q_strides[i], p.ks[i] = a.kv_strides[i], p.os[i] = a.o_strides[i];
  p.win = a.win;
  p.X = (uint32_t)a.X, p.H = a.H, p.Hkv = a.Hkv, p.grp = divisor(a.H / a.Hkv), p.Lq = (uint32_t)a.Lq, p.Lk = (uint32_t)a.Lk;
  p.D = a.D;
  p.c = a.scale * kLog2e, p.scale = a.scale;
  p.vec = a.vec;
  if (a.bf16) {
    if (a.D <= 32) return start<bf16, 32>(p, a, s);
    if (a.D <= 48) return start<bf16, 48>(p, a, s);
    if (a.D <= 64) return start<bf16, 64>(p, a, s);
    if (a.D <= 80) return start<bf16, 80>(p, a, s);
    if (a.D <= 96) return start<bf16, 96>(p, a, s);
    return start<bf16, 128>(p, a, s);
  }
  if (a.D <= 32) return start<float, 32>(p, a, s);
  if (a.D <= 64) return start<float, 64>(p, a, s);
  if (a.D <= 96) return start<float, 96>(p, a, s);
  return start<float, 128>(p, a, s);
}

}  // namespace dsp
