// Gradient of attention with a learned relative position bias.  With
//   z_ij = scale q_i . k_j + bias[bucket(j - i - q_pos)][h],  P = softmax(z),
//   Delta_i = sum_j P_ij dP_ij = sum_d dO_id O_id,  dZ = P (dP - Delta),  dP = dO V^T:
//   dV = P^T dO,  dQ = scale dZ K,  dK = scale dZ^T Q,
//   dbias[t][h] = sum of dZ_ij over every (b, x, i, j) whose distance has bucket t.
// P is recomputed from the forward's row log-sum-exp.  Two kernels, both deterministic:
// the first owns blocks of queries and loops over the keys (dQ, Delta, dbias), the
// second owns blocks of keys and loops over the queries of its group's heads (dK, dV).
//
// dbias is a sum along diagonals of dZ.  Blocks wholly past the table's end add to one
// register per lane.  The others go through LDS: a wave writes its 32 x 32 block and
// reads it back along the diagonals, lane c the distance c - 31 from the block's, and
// adds the 63 sums to an array over the distances of its own (no atomics: LDS atomics
// took 85 ns an instruction here, half of the kernel's time).  A work-group stays with
// one head and runs through several blocks of queries, so the waves' arrays are folded
// once, in order; a last kernel adds the work-groups' sums in order and folds distances
// into buckets.
//
// P and dZ are rounded to bf16 for the products that take them as operands (the matrix
// cores' type; their sums are fp32), dbias sums dZ before that rounding.  Delta is formed
// from P and dP; only in fp32 and for units past 64 positions from the stored o.
//
// Measured in bf16: 32 heads of 64 over 8, 4 causal sequences of 2000, 1334, 667 and 0:
// dQ 189 us, dK and dV 215, dbias 6 (bound by a wave's chain of product, exponential and
// product, with two or three waves to a SIMD, the matrix cores busy 25-27%, waits 48%, and by
// causal blocks of unequal length); 8 x 16 units of 4096 x 72 4.1-4.3 ms in all (370 TFLOP/s
// of the gradient's 5 products; the plain gradient 2.3 ms); 1350 x 16 units of 49 x 72
// 367-390 us: seven passes over rows, 1.07 GB (by the counters 1.16), 2.7-2.9 TB/s, so not
// memory but a unit's chain of loads, two passes and stores, with three work-groups to a CU
// and nothing of the next unit on its way (waits 46%).
#include <algorithm>
#include <type_traits>

#include "attn_relpos.h"

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
  float* part;       // [H][parts][2 M + 1]
  const int32_t* q_pos;
  const int32_t* kv_len;
  int64_t qs[3], ks[3], os[3];
  BiasArgs bias;
  uint32_t X, H, grp, Lq, Lk, n_blk, D, BX, parts;
  Order order;       // dK, dV
  float c, scale;
  bool vec, causal;
};

__device__ __forceinline__ int64_t bx_at(const BwdParams& p, uint32_t bx, const int64_t* st) {
  return (int64_t)(bx / p.X) * st[0] + (int64_t)(bx % p.X) * st[1];
}

// The probabilities of a block with queries on rows and keys on columns, in place of its
// raw scores: lse2 (LDS) at this lane's first row, d0 the first key's place after the
// first query.  `key0`, len: keys from len on have none.
__device__ __forceinline__ void block_probabilities(const BwdParams& p, floatx16& s, const float* lse2,
                                                    const float* tab0, float left, float right, int32_t d0, int l32,
                                                    int g, uint32_t key0, uint32_t len) {
  const bool far = d0 + 31 <= -p.bias.M || d0 - 31 >= p.bias.M;
  const float t = d0 < 0 ? left : right;
  const float* tb = tab0 + d0 + l32 - 4 * g;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const floatx4 l = *reinterpret_cast<const floatx4*>(lse2 + 8 * q);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[4 * q + i] = fmaf(s[4 * q + i], p.c, (far ? t : tb[-(8 * q + i)]) - l[i]);
  }
  if (p.causal && d0 + 31 > 0) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (d0 + l32 > 8 * (r / 4) + 4 * g + r % 4) s[r] = -INFINITY;
  }
  if (key0 + 32 > len) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = key0 + l32 < len ? s[r] : -INFINITY;
  }
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(s[r]);
}

// Adds a block of dZ (lane (n + 32 g): query n, keys 8 (r / 4) + 4 g + r % 4) to the sums
// by distance: `at` is the sum of the first key's distance from the first query, `room`
// 32 rows of 32 floats of this wave's.  Row k is written rotated by k, so that column c
// holds the elements of two distances: k - q = -c where k <= q, and 32 - c past the wrap.
constexpr int kDiag = 32 * 32;
__device__ __forceinline__ void add_diagonals(float* at, float* room, const floatx16& z, int lane) {
  asm volatile("" : "+v"(lane));   // what is made of it below is not worth keeping in registers
  const int l32 = lane & 31, g = lane >> 5;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int k = 8 * (r / 4) + r % 4;
    room[(k + 4 * g) * 32 + ((l32 - 4 * g - k) & 31)] = z[r];
  }
  wave_order();
  // lane (c + 32 g): column c, rows 16 g ..; row k of it is query k + c, or k + c - 32
  float low = 0.0f, high = 0.0f;
  const int split = 32 - l32 - 16 * g;   // rows from here on have wrapped
  const float* from = room + 16 * g * 32 + l32;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float e = from[i * 32];
    low += i < split ? e : 0.0f;
    high += i < split ? 0.0f : e;
  }
  low += swap_halves(low);
  high += swap_halves(high);
  // distance -c from the first half's lanes, 32 - c (c > 0) from the second's
  if (g == 0) at[-l32] += low;
  else if (l32) at[32 - l32] += high;
  wave_order();
}

// A work-group's sums of one head into its part: the waves' arrays, the sums past
// the table's ends ([2][NT]) and the table's own entries past M, in a fixed order.
template <int NT>
__device__ __forceinline__ void fold_sums(const BwdParams& p, float* acc, int n_acc, const float* ends, uint32_t h,
                                          uint32_t part) {
  const int32_t near = p.bias.M + kEdge, n_tab = 2 * near + 1;
  for (int32_t e = threadIdx.x; e < n_tab; e += NT) {
    float v = acc[e];
    for (int w = 1; w < n_acc; ++w) v += acc[w * n_tab + e];
    acc[e] = v;
  }
  __syncthreads();
  const int32_t n_out = 2 * p.bias.M + 1;
  float* w = p.part + ((uint64_t)h * p.parts + part) * n_out;
  for (int32_t e = threadIdx.x; e < n_out; e += NT) {
    float v = acc[e + kEdge];
    if (e == 0) {
      for (int t = 0; t < NT; ++t) v += ends[t];
      for (int i = 0; i < kEdge; ++i) v += acc[i];
    }
    if (e == n_out - 1) {   // M = 0: both ends are the one distance
      for (int t = 0; t < NT; ++t) v += ends[NT + t];
      for (int i = 0; i < kEdge; ++i) v += acc[n_tab - 1 - i];
    }
    w[e] = v;
  }
}

// ---------------------------------------------------------------------------
// dQ, Delta and the sums of dZ by distance: 32 queries of one head per wave.  In bf16 the
// keys pass twice, first for Delta_i = sum_j P_ij dP_ij.  Taken from o, Delta would carry
// the rounding of o, and a bucket's sum, whose terms cancel (each row of dZ adds up to
// nothing), that rounding many times over: 5e-3 of dbias at 384 causal positions.  The
// first pass costs a third of the gradient: 4096 x 72 3.15 -> 4.2 ms.
template <typename T, int DC, int NW, int KB, int MINW>
__global__ __launch_bounds__(NW * 64, MINW) void relpos_bwd_dq_kernel(BwdParams p) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  constexpr int NT = NW * 64, QB = NW * 32, NKT = KB / 32, TILE = KB * G::P;
  constexpr bool TWICE = sizeof(T) == 2;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  T* lds = reinterpret_cast<T*>(smem);   // [2][K, V][KB][P]
  const int32_t near = p.bias.M + kEdge, n_tab = 2 * near + 1;
  float* room = reinterpret_cast<float*>(lds + 4 * TILE);  // [NW][kDiag]
  float* tab = room + NW * kDiag;                     // bias of distance d at near + d
  float* acc = tab + n_tab;                                // [NW][n_tab]: the waves' sums

  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // work-group -> (head, part): an XCD (work-groups i % 8) keeps to its own heads
  uint32_t h, part;
  if (p.H % 8 == 0) {
    const uint32_t hx = p.H / 8, r = blockIdx.x / 8;
    h = blockIdx.x % 8 * hx + r % hx;
    part = r / hx;
  } else {
    h = blockIdx.x % p.H;
    part = blockIdx.x / p.H;
  }
  const int D = (int)p.D;
  const uint32_t row_bytes = (uint32_t)p.ks[2] * (uint32_t)sizeof(T);
  using TileT = Tile<T, DC, KB, NT>;
  const typename TileT::Map map = TileT::map(D, row_bytes, threadIdx.x);
  TileT tk, tv;

  for (int32_t e = threadIdx.x; e < n_tab; e += NT) tab[e] = bias_at<T>(p.bias, p.H, h, e - near);
  for (int32_t e = threadIdx.x; e < NW * n_tab; e += NT) acc[e] = 0.0f;
  clear_pad<T, DC>(lds, 4 * KB, D, threadIdx.x, NT);
  const float left = bias_at<T>(p.bias, p.H, h, -p.bias.M), right = bias_at<T>(p.bias, p.H, h, p.bias.M);
  float* mine = acc + wave * n_tab + near;
  float sum_l = 0.0f, sum_r = 0.0f;

  // a work-group's items: with one each, the costly ones (causal: the last blocks of
  // every unit) come first
  const uint32_t n_items = p.BX * p.n_blk;
  for (uint32_t item = part; item < n_items; item += p.parts) {
    const uint32_t blk = p.n_blk - 1 - item / p.BX, bx = item - item / p.BX * p.BX;
    const uint32_t b = bx / p.X;
    const int64_t q_at = bx_at(p, bx, p.qs) + (int64_t)h * D, o_at = bx_at(p, bx, p.os) + (int64_t)h * D;
    const int64_t k_at = bx_at(p, bx, p.ks) + (int64_t)(h / p.grp) * D;
    const T* kg = static_cast<const T*>(p.k) + k_at;
    const T* vg = static_cast<const T*>(p.v) + k_at;
    const int32_t q0 = position(p.q_pos, b) + (int32_t)(blk * QB);
    uint32_t k1 = length(p.kv_len, b, p.Lk);
    if (p.causal) {
      const int32_t last = q0 + (int32_t)min(p.Lq - blk * QB, (uint32_t)QB);
      k1 = last <= 0 ? 0u : min(k1, (uint32_t)last);
    }
    auto fetch = [&](uint32_t kb) {
      const uint32_t rows = kb < k1 ? min(k1 - kb, (uint32_t)KB) : 0u;
      tk.fetch(map, kg + (int64_t)kb * p.ks[2], rows, row_bytes, D, p.vec);
      tv.fetch(map, vg + (int64_t)kb * p.ks[2], rows, row_bytes, D, p.vec);
    };
    auto stash = [&](int buf) {
      tk.stash(map, lds + buf * 2 * TILE);
      tv.stash(map, lds + buf * 2 * TILE + TILE);
    };
    if (k1) fetch(0);
    const uint32_t row = blk * QB + 32 * wave + l32;
    const bool on = row < p.Lq;
    typename M::frag qf[G::NS], df[G::NS];
    row_frags<T, DC>(on ? static_cast<const T*>(p.q) + q_at + (int64_t)row * p.qs[2] : nullptr, g, D, p.vec, qf);
    row_frags<T, DC>(on ? static_cast<const T*>(p.dout) + o_at + (int64_t)row * p.os[2] : nullptr, g, D, p.vec, df);
    float delta = 0.0f;
    if constexpr (!TWICE) {
      typename M::frag of[G::NS];
      row_frags<T, DC>(on ? static_cast<const T*>(p.o) + o_at + (int64_t)row * p.os[2] : nullptr, g, D, p.vec, of);
#pragma unroll
      for (int s = 0; s < G::NS; ++s)
#pragma unroll
        for (int e = 0; e < G::E; ++e) delta += (float)df[s][e] * (float)of[s][e];
      delta += swap_halves(delta);
    }
    const uint64_t stat = ((uint64_t)bx * p.H + h) * p.Lq + row;
    // a row without keys, or past the end: P = exp2(-inf) = 0
    const float l = on ? p.lse[stat] : -INFINITY;
    const float lse2 = l == -INFINITY ? INFINITY : l * kLog2e;
    __syncthreads();   // the buffers, the table and the sums are free and set
    if (k1) stash(0);
    __syncthreads();
    const uint32_t n_it = (k1 + KB - 1) / KB;
    const int32_t wq = q0 + 32 * wave;
    // S and dP of one block of 32 keys, S made the exponents of P; false: nothing to do
    auto block = [&](const T* kl, uint32_t kb, int kt, floatx16& s, floatx16& dp) {
      const T* vl = kl + TILE;
      const int32_t key0 = (int32_t)kb + 32 * kt, d0 = key0 - wq;
      if (key0 >= (int32_t)k1 || (p.causal && d0 > 31)) return false;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.0f;
#pragma unroll
      for (int st = 0; st < G::NS; ++st) {
        const int at = (32 * kt + l32) * G::P + 2 * G::E * st + G::E * g;
        s = M::mma(*reinterpret_cast<const typename M::frag*>(kl + at), qf[st], s);
        dp = M::mma(*reinterpret_cast<const typename M::frag*>(vl + at), df[st], dp);
      }
      if (d0 + 31 <= -p.bias.M || d0 - 31 >= p.bias.M) {
        const float t = (d0 < 0 ? left : right) - lse2;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], p.c, t);
      } else {
        const float* tb = tab + near + d0 + 4 * g - l32;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], p.c, tb[8 * (r / 4) + r % 4] - lse2);
      }
      if ((p.causal && d0 + 31 > 0) || key0 + 32 > (int32_t)k1) {
        const int32_t stop = (p.causal ? min((int32_t)k1, wq + l32 + 1) : (int32_t)k1) - key0 - 4 * g;
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (8 * (r / 4) + r % 4 >= stop) s[r] = -INFINITY;
      }
      return true;
    };
    if constexpr (TWICE) {
      for (uint32_t it = 0; it < n_it; ++it) {
        fetch(it + 1 < n_it ? (it + 1) * KB : 0);
        const T* kl = lds + (it & 1) * 2 * TILE;
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) {
          floatx16 s, dp;
          if (!block(kl, it * KB, kt, s, dp)) continue;
#pragma unroll
          for (int r = 0; r < 16; ++r) delta += __builtin_amdgcn_exp2f(s[r]) * dp[r];
        }
        stash((it + 1) & 1);
        __syncthreads();
      }
      delta += swap_halves(delta);
    }
    if (on && g == 0) p.delta[stat] = delta;
    ColAcc<T, DC> dq;
    dq.zero();
    const uint32_t odd = TWICE ? n_it & 1 : 0;   // the buffer of the first tile
    for (uint32_t it = 0; it < n_it; ++it) {
      const uint32_t kb = it * KB;
      const bool more = it + 1 < n_it;
      if (more) fetch(kb + KB);
      const T* kl = lds + ((it + odd) & 1) * 2 * TILE;
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt) {
        floatx16 s, dp;
        if (!block(kl, kb, kt, s, dp)) continue;
        const int32_t d0 = (int32_t)kb + 32 * kt - wq;
        ColB<T> z;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          dp[r] = __builtin_amdgcn_exp2f(s[r]) * (dp[r] - delta);
          z.set(r, dp[r]);
        }
        if (d0 + 31 <= -p.bias.M || d0 - 31 >= p.bias.M) {
          float v = 0.0f;
#pragma unroll
          for (int r = 0; r < 16; ++r) v += dp[r];
          if (d0 < 0) sum_l += v;
          else sum_r += v;
        } else {
          add_diagonals(mine + d0, room + wave * kDiag, dp, lane);
        }
        dq.add(kl, 32 * kt, lane, z);
      }
      if (more) stash((it + 1 + odd) & 1);
      __syncthreads();
    }
    dq.scale(p.scale, lane);
    T* out = static_cast<T*>(p.dq) + q_at;
    auto q_out = [&](int n) -> T* {
      const uint32_t r = blk * QB + 32 * wave + n;
      return r < p.Lq ? out + (int64_t)r * p.qs[2] : nullptr;
    };
    if (p.vec) store_rows_lds<T, DC>(lds + wave * 32 * G::P, dq, lane, D, D, q_out);   // this wave's rows of the tiles
    else store_rows<T, DC>(dq, lane, D, false, q_out);
  }

  __syncthreads();
  float* ends = room;   // [2][NT]
  ends[threadIdx.x] = sum_l;
  ends[NT + threadIdx.x] = sum_r;
  __syncthreads();
  fold_sums<NT>(p, acc, NW, ends, h, part);
}

// dbias[t][h]: the parts of each distance, then the distances of each bucket, in a fixed
// order: 4 interleaved runs of parts for each distance, 64 lanes to a bucket.
template <typename T>
__global__ __launch_bounds__(1024) void relpos_bias_grad_kernel(BwdParams p, T* dbias) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const uint32_t h = blockIdx.x;
  const int32_t n = 2 * p.bias.M + 1;
  float* sums = reinterpret_cast<float*>(smem);             // [4][n]
  int32_t* which = reinterpret_cast<int32_t*>(sums + 4 * n);  // [n]
  const float* w = p.part + (uint64_t)h * p.parts * n;
  for (int32_t e = threadIdx.x; e < n; e += 1024) which[e] = p.bias.buckets[e];
  const uint32_t run = threadIdx.x >> 8;
  for (int32_t e = threadIdx.x & 255; e < n; e += 256) {
    float v = 0.0f;
#pragma unroll 8
    for (uint32_t s = run; s < p.parts; s += 4) v += w[(uint64_t)s * n + e];
    sums[run * n + e] = v;
  }
  __syncthreads();
  for (int32_t e = threadIdx.x; e < n; e += 1024) sums[e] = (sums[e] + sums[n + e]) + (sums[2 * n + e] + sums[3 * n + e]);
  __syncthreads();
  const int lane = threadIdx.x & 63;
  for (int32_t t = threadIdx.x >> 6; t < p.bias.nb; t += 16) {
    float v = 0.0f;
    for (int32_t e = lane; e < n; e += 64) v += which[e] == t ? sums[e] : 0.0f;
#pragma unroll
    for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off);
    const bool masked = (float)static_cast<const T*>(p.bias.bias)[(int64_t)t * p.H + h] <= kMasked;
    if (lane == 0) dbias[(int64_t)t * p.H + h] = (T)(masked ? 0.0f : v);
  }
}

// ---------------------------------------------------------------------------
// dK and dV, over the queries of every head of the key/value head's group, in tiles of
// 32 QT: KW blocks of 32 keys, each tile's queries shared out among QS waves for each,
// whose sums are joined at the end.  More keys read the queries less often; more waves
// to a key make more work-groups, each shorter, which is what few, long, causal or
// ragged units need to fill the chip evenly.
template <typename T, int DC, int KW, int QS, int QT, int MINW>
__global__ __launch_bounds__(KW * QS * 64, MINW) void relpos_bwd_dkv_kernel(BwdParams p) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  constexpr int NT = KW * QS * 64, QB = 32 * QT, TILE = QB * G::P;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  T* lds = reinterpret_cast<T*>(smem);                            // [2][Q, dO][QB][P]
  float* stat = reinterpret_cast<float*>(lds + 4 * TILE);         // [2][lse2, Delta][QB]
  const int32_t near = p.bias.M + kEdge, n_tab = 2 * near + 1;
  float* tab = stat + 4 * QB;

  const int lane0 = threadIdx.x & 63, lane = lane0, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kw = wave / QS, qs = wave % QS;
  const Place pl = place(p.order);   // heads of the order: key/value heads
  if (!pl.any) return;
  const uint32_t blk = pl.block, bx = pl.bx, e = pl.h, b = bx / p.X;
  const int D = (int)p.D;
  const int64_t k_at = bx_at(p, bx, p.ks) + (int64_t)e * D;
  const int64_t q_bx = bx_at(p, bx, p.qs), o_bx = bx_at(p, bx, p.os);
  const uint32_t first_key = blk * 32 * KW, key0 = first_key + 32 * kw, key = key0 + l32;
  const uint32_t len = length(p.kv_len, b, p.Lk);
  const int32_t pos = position(p.q_pos, b);
  typename M::frag kf[G::NS], vf[G::NS];
  row_frags<T, DC>(key < len ? static_cast<const T*>(p.k) + k_at + (int64_t)key * p.ks[2] : nullptr, g, D, p.vec, kf);
  row_frags<T, DC>(key < len ? static_cast<const T*>(p.v) + k_at + (int64_t)key * p.ks[2] : nullptr, g, D, p.vec, vf);

  const uint32_t q_row = (uint32_t)p.qs[2] * (uint32_t)sizeof(T), o_row = (uint32_t)p.os[2] * (uint32_t)sizeof(T);
  using TileT = Tile<T, DC, QB, NT>;
  const typename TileT::Map mq = TileT::map(D, q_row, threadIdx.x), mo = TileT::map(D, o_row, threadIdx.x);
  TileT tq, to;
  static_assert(NT >= 2 * QB, "a statistic for each thread");
  float pre = 0.0f;
  clear_pad<T, DC>(lds, 4 * QB, D, threadIdx.x, NT);

  ColAcc<T, DC> dk, dv;
  dk.zero();
  dv.zero();
  // the first tile of queries that sees the work-group's first key
  const int32_t first = p.causal ? (int32_t)first_key - pos : 0;
  const uint32_t it0 = first > 0 ? (uint32_t)first / QB : 0u;
  const uint32_t n_it = (p.Lq + QB - 1) / QB;
  const bool any = first_key < len && it0 < n_it;
  for (uint32_t hh = 0; any && hh < p.grp; ++hh) {
    const uint32_t h = e * p.grp + hh;
    const T* qg = static_cast<const T*>(p.q) + q_bx + (int64_t)h * D;
    const T* og = static_cast<const T*>(p.dout) + o_bx + (int64_t)h * D;
    const uint64_t st0 = ((uint64_t)bx * p.H + h) * p.Lq;
    const float left = bias_at<T>(p.bias, p.H, h, -p.bias.M), right = bias_at<T>(p.bias, p.H, h, p.bias.M);
    auto fetch = [&](uint32_t it) {
      const uint32_t q0 = it * QB, rows = min(p.Lq - q0, (uint32_t)QB);
      tq.fetch(mq, qg + (int64_t)q0 * p.qs[2], rows, q_row, D, p.vec);
      to.fetch(mo, og + (int64_t)q0 * p.os[2], rows, o_row, D, p.vec);
      if (threadIdx.x < 2 * QB) {
        const uint32_t i = threadIdx.x % QB;
        const bool is_delta = threadIdx.x >= QB;
        const float l = i < rows ? (is_delta ? p.delta : p.lse)[st0 + q0 + i] : is_delta ? 0.0f : -INFINITY;
        pre = is_delta ? l : l == -INFINITY ? INFINITY : l * kLog2e;
      }
    };
    auto stash = [&](int buf) {
      tq.stash(mq, lds + buf * 2 * TILE);
      to.stash(mo, lds + buf * 2 * TILE + TILE);
      if (threadIdx.x < 2 * QB) stat[buf * 2 * QB + threadIdx.x] = pre;
    };
    fetch(it0);
    __syncthreads();   // the table and the buffers are free
    for (int32_t t = threadIdx.x; t < n_tab; t += NT) tab[t] = bias_at<T>(p.bias, p.H, h, t - near);
    stash(it0 & 1);
    __syncthreads();
    for (uint32_t it = it0; it < n_it; ++it) {
      const bool more = it + 1 < n_it;
      if (more) fetch(it + 1);
      int lane = lane0;
      asm volatile("" : "+v"(lane));
      const int l32 = lane & 31, g = lane >> 5;
      const T* ql = lds + (it & 1) * 2 * TILE;
      const T* ol = ql + TILE;
      const float* sl = stat + (it & 1) * 2 * QB;
#pragma unroll
      for (int i = 0; i < QT / QS; ++i) {
        const int sub = i * QS + qs;
        const int32_t q0 = pos + (int32_t)(it * QB) + 32 * sub;   // position of the block's first query
        if (key0 >= len || it * QB + 32 * sub >= p.Lq || (p.causal && (int32_t)key0 > q0 + 31)) continue;
        floatx16 s, dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.0f;
#pragma unroll
        for (int st = 0; st < G::NS; ++st) {
          const int at = (32 * sub + l32) * G::P + 2 * G::E * st + G::E * g;
          s = M::mma(*reinterpret_cast<const typename M::frag*>(ql + at), kf[st], s);
          dp = M::mma(*reinterpret_cast<const typename M::frag*>(ol + at), vf[st], dp);
        }
        // lane (n + 32 g): key n, queries 8 (r / 4) + 4 g + r % 4
        block_probabilities(p, s, sl + 32 * sub + 4 * g, tab + near, left, right, (int32_t)key0 - q0, l32, g, key0, len);
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
        dv.add(ol, 32 * sub, lane, pb);
        dk.add(ql, 32 * sub, lane, zb);
      }
      if (more) stash((it + 1) & 1);
      __syncthreads();
    }
  }
  dk.scale(p.scale, lane);
  T* const out[2] = {static_cast<T*>(p.dk) + k_at, static_cast<T*>(p.dv) + k_at};
  auto row = [&](T* base, int n) -> T* { return key0 + n < p.Lk ? base + (int64_t)(key0 + n) * p.ks[2] : nullptr; };
  if constexpr (QS == 1) {
    if (p.vec) {
      T* so = lds + wave * 32 * G::P;   // the tiles are done with
      static_assert(KW * 32 <= 4 * QB, "rows to write through");
      __syncthreads();
      store_rows_lds<T, DC>(so, dk, lane, D, G::DP, [&](int n) { return row(out[0], n); });
      store_rows_lds<T, DC>(so, dv, lane, D, G::DP, [&](int n) { return row(out[1], n); });
    } else {
      store_rows<T, DC>(dk, lane, D, false, [&](int n) { return row(out[0], n); });
      store_rows<T, DC>(dv, lane, D, false, [&](int n) { return row(out[1], n); });
    }
  } else {
    // the QS waves' sums of a key, added in order
    float* sums = reinterpret_cast<float*>(smem);   // [QS][KW * 32][DP]
    constexpr int W = G::DP, ROWS = KW * 32;
    static_assert((size_t)QS * ROWS * W * 4 <= (size_t)4 * TILE * sizeof(T), "the sums fit the tiles");
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
      store_rows<T, DC>(which ? dv : dk, lane, W, true, [&](int n) { return sums + (qs * ROWS + kw * 32 + n) * W; });
      __syncthreads();
      for (uint32_t i = threadIdx.x; i < ROWS * W / 4; i += NT) {
        const uint32_t n = i / (W / 4), d = i % (W / 4) * 4;
        floatx4 v = *reinterpret_cast<const floatx4*>(sums + n * W + d);
#pragma unroll
        for (int q = 1; q < QS; ++q) v += *reinterpret_cast<const floatx4*>(sums + (q * ROWS + n) * W + d);
        if (first_key + n < p.Lk)
          store4(out[which] + (int64_t)(first_key + n) * p.ks[2], (int)d, D, p.vec, v[0], v[1], v[2], v[3]);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Adds the gradients of keys 32 wave .. from one head's queries: rows of Q and dO in
// LDS, the keys' and values' in registers; tb0: the bias of distance 0.
template <typename T, int DC, int NB>
__device__ __forceinline__ void short_dkv(const BwdParams& p, const T* ql, const T* ol,
                                          const typename Mx<T>::frag (&kf)[Geo<T, DC>::NS],
                                          const typename Mx<T>::frag (&vf)[Geo<T, DC>::NS], const float* st_lse,
                                          const float* st_del, const float* tb0, int32_t q0, uint32_t len, int wave,
                                          int lane, ColAcc<T, DC>& dk, ColAcc<T, DC>& dv) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  const int l32 = lane & 31, g = lane >> 5;
  const float left = tb0[-p.bias.M], right = tb0[p.bias.M];
  if (32u * wave >= len) return;
#pragma unroll
  for (int qt = 0; qt < NB; ++qt) {
    const int32_t d0 = 32 * wave - q0 - 32 * qt;
    if (32u * qt >= p.Lq || (p.causal && d0 > 31)) continue;
    floatx16 s, dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.0f;
#pragma unroll
    for (int i = 0; i < G::NS; ++i) {
      const int at = (32 * qt + l32) * G::P + 2 * G::E * i + G::E * g;
      s = M::mma(*reinterpret_cast<const typename M::frag*>(ql + at), kf[i], s);
      dp = M::mma(*reinterpret_cast<const typename M::frag*>(ol + at), vf[i], dp);
    }
    block_probabilities(p, s, st_lse + 32 * qt + 4 * g, tb0, left, right, d0, l32, g, 32 * wave, len);
    ColB<T> pb, zb;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const floatx4 dl = *reinterpret_cast<const floatx4*>(st_del + 32 * qt + 8 * q + 4 * g);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        pb.set(4 * q + i, s[4 * q + i]);
        zb.set(4 * q + i, s[4 * q + i] * (dp[4 * q + i] - dl[i]));
      }
    }
    dv.add(ol, 32 * qt, lane, pb);
    dk.add(ql, 32 * qt, lane, zb);
  }
}
// and writes them, through LDS rows 32 wave .. of two tiles
template <typename T, int DC>
__device__ __forceinline__ void short_store(const BwdParams& p, T* kl, T* vl, int64_t k_at, int wave, int lane,
                                            ColAcc<T, DC>& dk, const ColAcc<T, DC>& dv) {
  using G = Geo<T, DC>;
  const int D = (int)p.D;
  dk.scale(p.scale, lane);
  auto out = [&](void* base) {
    return [&, base](int n) -> T* {
      const uint32_t r = 32 * wave + n;
      return r < p.Lk ? static_cast<T*>(base) + k_at + (int64_t)r * p.ks[2] : nullptr;
    };
  };
  if (p.vec) {
    store_rows_lds<T, DC>(kl + 32 * wave * G::P, dk, lane, D, D, out(p.dk));
    store_rows_lds<T, DC>(vl + 32 * wave * G::P, dv, lane, D, D, out(p.dv));
  } else {
    store_rows<T, DC>(dk, lane, D, false, out(p.dk));
    store_rows<T, DC>(dv, lane, D, false, out(p.dv));
  }
}

// Units of at most 32 NB queries and keys (temporal attention): one work-group holds a
// unit's Q, K, V and dO in LDS, so each row crosses HBM once.  Wave w first takes queries
// 32 w .. against all keys (dQ, dbias), with the whole row of P and dP in registers, so
// Delta_i = sum_j P_ij dP_ij needs no o and none of its rounding; then keys 32 w ..
// against all queries (dK, dV), with the scores computed again the other way round.
// A work-group stays with one head (which has keys of its own) and runs through units;
// a wave's dZ is summed over them in registers, element by element, and goes to the
// sums by distance only when the queries' first position changes and at the end.
// Where heads share keys (not OWN) dK and dV are sums over heads: they are left to
// relpos_bwd_short_dkv_kernel, and Delta goes to memory.
template <typename T, int DC, int NB, bool OWN, int MINW>
__global__ __launch_bounds__(NB * 64, MINW) void relpos_bwd_short_kernel(BwdParams p) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  constexpr int NT = NB * 64, R = NB * 32, TILE = R * G::P;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  T* kl = reinterpret_cast<T*>(smem);
  T* vl = kl + TILE;
  T* ql = vl + TILE;
  T* ol = ql + TILE;
  float* st_lse = reinterpret_cast<float*>(ol + TILE);    // [R]
  float* st_del = st_lse + R;                             // [R]
  const int32_t near = p.bias.M + kEdge, n_tab = 2 * near + 1;
  float* tab = st_del + R;                                // [n_tab]
  float* acc = tab + n_tab;                               // [NB][n_tab]: the waves' sums
  float* ends = acc + NB * n_tab;                         // [2][NT]: sums past the table's ends

  const int lane0 = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // work-group -> (head, part); an XCD takes whole token rows
  const uint32_t j8 = blockIdx.x >> 3;
  const uint32_t h = j8 % p.H, part = j8 / p.H * 8 + (blockIdx.x & 7u);
  const int D = (int)p.D;
  const uint32_t k_row = (uint32_t)p.ks[2] * (uint32_t)sizeof(T), q_row = (uint32_t)p.qs[2] * (uint32_t)sizeof(T),
                 o_row = (uint32_t)p.os[2] * (uint32_t)sizeof(T);
  using TileT = Tile<T, DC, R, NT>;
  const typename TileT::Map mk = TileT::map(D, k_row, threadIdx.x), mq = TileT::map(D, q_row, threadIdx.x),
                            mo = TileT::map(D, o_row, threadIdx.x);

  for (int32_t t = threadIdx.x; t < n_tab; t += NT) tab[t] = bias_at<T>(p.bias, p.H, h, t - near);
  for (int32_t t = threadIdx.x; t < NB * n_tab + 2 * NT; t += NT) acc[t] = 0.0f;   // and the ends
  clear_pad<T, DC>(kl, 4 * R, D, threadIdx.x, NT);

  floatx16 sum[NB];   // of dZ, queries 32 wave .. against keys 32 kt ..
#pragma unroll
  for (int kt = 0; kt < NB; ++kt)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[kt][r] = 0.0f;
  int32_t sum_q0 = 0;
  for (uint32_t bx = part;; bx += p.parts) {
    const bool done = bx >= p.BX;
    const uint32_t b = done ? 0 : bx / p.X;
    const int32_t q0 = position(p.q_pos, b);
    if (done || q0 != sum_q0) {
      __syncthreads();   // the sums by distance are set
      int lane = lane0;
      asm volatile("" : "+v"(lane));
      const int l32 = lane & 31, g = lane >> 5;
      float* mine = acc + wave * n_tab + near;
#pragma unroll
      for (int kt = 0; kt < NB; ++kt) {
        const int32_t d0 = 32 * kt - sum_q0 - 32 * wave;
        if (d0 + 31 <= -p.bias.M || d0 - 31 >= p.bias.M) {
          float v = 0.0f;
#pragma unroll
          for (int r = 0; r < 16; ++r) v += sum[kt][r];
          ends[(d0 < 0 ? 0 : NT) + threadIdx.x] += v;
        } else {
          // rare: one register of one half of the wave (32 distances) at a time
          float* to = mine + d0 + 4 * g - l32;
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              if (g == half) to[8 * (r / 4) + r % 4] += sum[kt][r];
              wave_order();
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[kt][r] = 0.0f;
      }
      sum_q0 = q0;
    }
    if (done) break;
    int lane = lane0;
    asm volatile("" : "+v"(lane));   // the addresses made of it are cheaper to form again than to keep over the loop
    const int l32 = lane & 31, g = lane >> 5;
    const uint32_t len = length(p.kv_len, b, p.Lk);
    const int64_t k_at = bx_at(p, bx, p.ks) + (int64_t)(OWN ? h : h / p.grp) * D,
                  q_at = bx_at(p, bx, p.qs) + (int64_t)h * D, o_at = bx_at(p, bx, p.os) + (int64_t)h * D;
    {
      TileT tk, tv, tq, to;
      tk.fetch(mk, static_cast<const T*>(p.k) + k_at, len, k_row, D, p.vec);
      tv.fetch(mk, static_cast<const T*>(p.v) + k_at, len, k_row, D, p.vec);
      tq.fetch(mq, static_cast<const T*>(p.q) + q_at, p.Lq, q_row, D, p.vec);
      to.fetch(mo, static_cast<const T*>(p.dout) + o_at, p.Lq, o_row, D, p.vec);
      float l = -INFINITY;
      if (threadIdx.x < p.Lq) l = p.lse[((uint64_t)bx * p.H + h) * p.Lq + threadIdx.x];
      __syncthreads();   // the rows are free
      tk.stash(mk, kl);
      tv.stash(mk, vl);
      tq.stash(mq, ql);
      to.stash(mo, ol);
      if (threadIdx.x < R) st_lse[threadIdx.x] = l == -INFINITY ? INFINITY : l * kLog2e;
    }
    __syncthreads();
    const float* tb0 = tab + near;
    const float left = tb0[-p.bias.M], right = tb0[p.bias.M];
    ColAcc<T, DC> dq;
    dq.zero();
    if (32u * wave < p.Lq) {
      const int32_t wq = q0 + 32 * wave;
      typename M::frag qf[G::NS], df[G::NS];
#pragma unroll
      for (int s = 0; s < G::NS; ++s) {
        const int at = (32 * wave + l32) * G::P + 2 * G::E * s + G::E * g;
        qf[s] = *reinterpret_cast<const typename M::frag*>(ql + at);
        df[s] = *reinterpret_cast<const typename M::frag*>(ol + at);
      }
      const float lse2 = st_lse[32 * wave + l32];
      floatx16 s[NB], dp[NB];
      float delta = 0.0f;
#pragma unroll
      for (int kt = 0; kt < NB; ++kt) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kt][r] = dp[kt][r] = 0.0f;
        if (32u * kt >= len) continue;
#pragma unroll
        for (int i = 0; i < G::NS; ++i) {
          const int at = (32 * kt + l32) * G::P + 2 * G::E * i + G::E * g;
          s[kt] = M::mma(*reinterpret_cast<const typename M::frag*>(kl + at), qf[i], s[kt]);
          dp[kt] = M::mma(*reinterpret_cast<const typename M::frag*>(vl + at), df[i], dp[kt]);
        }
        const int32_t d0 = 32 * kt - wq;
        if (d0 + 31 <= -p.bias.M || d0 - 31 >= p.bias.M) {
          const float t = (d0 < 0 ? left : right) - lse2;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kt][r] = fmaf(s[kt][r], p.c, t);
        } else {
          const float* tb = tb0 + d0 + 4 * g - l32;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kt][r] = fmaf(s[kt][r], p.c, tb[8 * (r / 4) + r % 4] - lse2);
        }
        if ((p.causal && d0 + 31 > 0) || 32u * kt + 32 > len) {
          const int32_t stop = p.causal ? min((int32_t)len, wq + l32 + 1) : (int32_t)len;
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (32 * kt + 8 * (r / 4) + 4 * g + r % 4 >= stop) s[kt][r] = -INFINITY;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[kt][r] = __builtin_amdgcn_exp2f(s[kt][r]);
          delta += s[kt][r] * dp[kt][r];
        }
      }
      delta += swap_halves(delta);
      if (OWN) {
        if (g == 0) st_del[32 * wave + l32] = delta;
      } else if (g == 0 && 32u * wave + l32 < p.Lq) {
        p.delta[((uint64_t)bx * p.H + h) * p.Lq + 32 * wave + l32] = delta;
      }
#pragma unroll
      for (int kt = 0; kt < NB; ++kt) {
        if (32u * kt >= len) continue;
        ColB<T> z;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float dz = s[kt][r] * (dp[kt][r] - delta);
          sum[kt][r] += dz;
          z.set(r, dz);
        }
        dq.add(kl, 32 * kt, lane, z);
      }
      dq.scale(p.scale, lane);
    }
    __syncthreads();   // Delta is there
    typename M::frag kf[G::NS], vf[G::NS];
    if constexpr (OWN) {
#pragma unroll
      for (int s = 0; s < G::NS; ++s) {
        const int at = (32 * wave + l32) * G::P + 2 * G::E * s + G::E * g;
        kf[s] = *reinterpret_cast<const typename M::frag*>(kl + at);
        vf[s] = *reinterpret_cast<const typename M::frag*>(vl + at);
      }
      __syncthreads();   // the rows of K are free
    }
    auto q_out = [&](int n) -> T* {
      const uint32_t r = 32 * wave + n;
      return r < p.Lq ? static_cast<T*>(p.dq) + q_at + (int64_t)r * p.qs[2] : nullptr;
    };
    if (p.vec) store_rows_lds<T, DC>(kl + 32 * wave * G::P, dq, lane, D, D, q_out);
    else store_rows<T, DC>(dq, lane, D, false, q_out);
    if constexpr (OWN) {
      ColAcc<T, DC> dk, dv;
      dk.zero();
      dv.zero();
      short_dkv<T, DC, NB>(p, ql, ol, kf, vf, st_lse, st_del, tb0, q0, len, wave, lane, dk, dv);
      // the rows of K and V serve to write: this wave's own, which it alone reads now
      short_store<T, DC>(p, kl, vl, k_at, wave, lane, dk, dv);
    }
  }
  __syncthreads();
  fold_sums<NT>(p, acc, NB, ends, h, part);
}

// dK and dV of short units whose keys several heads share: a work-group runs through
// units of one key/value head, whose heads' tables it keeps; wave w takes keys 32 w ..
// and adds up their gradients over the heads in registers.
template <typename T, int DC, int NB, int MINW>
__global__ __launch_bounds__(NB * 64, MINW) void relpos_bwd_short_dkv_kernel(BwdParams p, uint32_t parts) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  constexpr int NT = NB * 64, R = NB * 32, TILE = R * G::P;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  T* ql = reinterpret_cast<T*>(smem);                     // K at first
  T* ol = ql + TILE;                                      // V at first
  float* st_lse = reinterpret_cast<float*>(ol + TILE);    // [R]
  float* st_del = st_lse + R;                             // [R]
  const int32_t near = p.bias.M + kEdge, n_tab = 2 * near + 1;
  float* tab = st_del + R;                                // [grp][n_tab]
  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t kvh = p.H / p.grp, j8 = blockIdx.x >> 3;
  const uint32_t e = j8 % kvh, part = j8 / kvh * 8 + (blockIdx.x & 7u);
  const int D = (int)p.D;
  const uint32_t k_row = (uint32_t)p.ks[2] * (uint32_t)sizeof(T), q_row = (uint32_t)p.qs[2] * (uint32_t)sizeof(T),
                 o_row = (uint32_t)p.os[2] * (uint32_t)sizeof(T);
  using TileT = Tile<T, DC, R, NT>;
  const typename TileT::Map mk = TileT::map(D, k_row, threadIdx.x), mq = TileT::map(D, q_row, threadIdx.x),
                            mo = TileT::map(D, o_row, threadIdx.x);
  for (uint32_t hh = 0; hh < p.grp; ++hh)
    for (int32_t t = threadIdx.x; t < n_tab; t += NT)
      tab[hh * n_tab + t] = bias_at<T>(p.bias, p.H, e * p.grp + hh, t - near);
  clear_pad<T, DC>(ql, 2 * R, D, threadIdx.x, NT);
  for (uint32_t bx = part; bx < p.BX; bx += parts) {
    const uint32_t b = bx / p.X;
    const int32_t q0 = position(p.q_pos, b);
    const uint32_t len = length(p.kv_len, b, p.Lk);
    const int64_t k_at = bx_at(p, bx, p.ks) + (int64_t)e * D;
    TileT ta, tb;
    ta.fetch(mk, static_cast<const T*>(p.k) + k_at, len, k_row, D, p.vec);
    tb.fetch(mk, static_cast<const T*>(p.v) + k_at, len, k_row, D, p.vec);
    __syncthreads();   // the rows are free
    ta.stash(mk, ql);
    tb.stash(mk, ol);
    typename M::frag kf[G::NS], vf[G::NS];
    ColAcc<T, DC> dk, dv;
    dk.zero();
    dv.zero();
    for (uint32_t hh = 0; hh < p.grp; ++hh) {
      const uint32_t h = e * p.grp + hh;
      const int64_t q_at = bx_at(p, bx, p.qs) + (int64_t)h * D, o_at = bx_at(p, bx, p.os) + (int64_t)h * D;
      ta.fetch(mq, static_cast<const T*>(p.q) + q_at, p.Lq, q_row, D, p.vec);
      tb.fetch(mo, static_cast<const T*>(p.dout) + o_at, p.Lq, o_row, D, p.vec);
      float l = -INFINITY, del = 0.0f;
      if (threadIdx.x < p.Lq) {
        const uint64_t stat = ((uint64_t)bx * p.H + h) * p.Lq + threadIdx.x;
        l = p.lse[stat];
        del = p.delta[stat];
      }
      __syncthreads();   // K and V, or the last head's rows, are there
      if (hh == 0) {
#pragma unroll
        for (int s = 0; s < G::NS; ++s) {
          const int at = (32 * wave + l32) * G::P + 2 * G::E * s + G::E * g;
          kf[s] = *reinterpret_cast<const typename M::frag*>(ql + at);
          vf[s] = *reinterpret_cast<const typename M::frag*>(ol + at);
        }
        __syncthreads();   // and free
      }
      ta.stash(mq, ql);
      tb.stash(mo, ol);
      if (threadIdx.x < R) {
        st_lse[threadIdx.x] = l == -INFINITY ? INFINITY : l * kLog2e;
        st_del[threadIdx.x] = del;
      }
      __syncthreads();
      short_dkv<T, DC, NB>(p, ql, ol, kf, vf, st_lse, st_del, tab + hh * n_tab + near, q0, len, wave, lane, dk, dv);
    }
    __syncthreads();   // the rows serve to write
    short_store<T, DC>(p, ql, ol, k_at, wave, lane, dk, dv);
  }
}

constexpr int kDqWaves = 4;   // of a work-group of the dQ kernel, 32 queries each

// LDS of the short-unit kernel, and the blocks of 32 it takes the call with (0: not at
// all): at most 64 queries and keys (fp32 up to 64 wide: a wider one's rows and sums do
// not fit the registers); where heads share keys, tables of a group of 32 KB at most.
// Against the kernels for long units: 1350 x 16 units of 49 x 72 367-406 us and 1303 in all;
// heads that share keys, 2000 x 16 over 4 of 49 x 72, 467 and 1404.
size_t short_lds(const RelposArgs& a, int nb, int row_bytes) {
  const size_t n_tab = 2 * ((size_t)a.max_dist + kEdge) + 1;
  return (size_t)4 * 32 * nb * row_bytes + (size_t)2 * 32 * nb * 4 + (n_tab * (1 + nb) + 2 * 64 * nb) * 4;
}
int row_bytes_of(const RelposArgs& a) {
  const int dc = a.bf16 ? (a.D <= 32 ? 32 : a.D <= 48 ? 48 : a.D <= 64 ? 64 : a.D <= 80 ? 80 : a.D <= 96 ? 96 : 128)
                        : (a.D + 31) / 32 * 32;
  return a.bf16 ? (dc + 8) * 2 : (dc + 4) * 4;
}
size_t shared_tables(const RelposArgs& a) {
  return (size_t)(a.H / a.Hkv) * (2 * ((size_t)a.max_dist + kEdge) + 1) * 4;
}
int short_blocks(const RelposArgs& a) {
  const int64_t l = std::max(a.Lq, a.Lk);
  if (a.Lq == 0 || l > 64 || (!a.bf16 && a.D > 64)) return 0;
  if (a.H != a.Hkv && shared_tables(a) > 32 * 1024) return 0;
  return l <= 32 ? 1 : 2;
}
// Work-groups of a head (parts of its dbias): enough to fill the chip, no more than
// there is work.
int64_t parts_of(const RelposArgs& a) {
  if (const int nb = short_blocks(a)) {
    const int64_t per_cu = std::max<int64_t>(1, 160 * 1024 / (int64_t)short_lds(a, nb, row_bytes_of(a)));
    const int64_t want = (256 * std::min<int64_t>(per_cu, 8 / nb) + a.H - 1) / a.H;
    return (std::min(a.B * a.X, want) + 7) / 8 * 8;
  }
  constexpr int64_t qb = 32 * kDqWaves;
  const int64_t items = a.B * a.X * ((a.Lq + qb - 1) / qb);
  const int64_t want = (4096 + a.H - 1) / a.H;
  return std::max<int64_t>(1, std::min(items, want));
}

template <typename K>
int lds_limit(K* kernel, size_t lds) {
  if (lds <= 64 * 1024) return DSP_OK;
  return hip_status(
      hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
}

template <typename T>
int bias_grad(BwdParams& p, const RelposArgs& a, hipStream_t s) {
  const size_t n = 2 * (size_t)p.bias.M + 1;
  relpos_bias_grad_kernel<T><<<dim3(p.H), 1024, n * 5 * 4, s>>>(p, static_cast<T*>(a.dbias));
  return last_launch_status();
}

template <typename T, int DC, int NB>
int start_short(BwdParams& p, const RelposArgs& a, hipStream_t s) {
  constexpr int MINW = sizeof(T) == 2 && DC <= 96 ? 2 : 1;
  const bool own = a.H == a.Hkv;
  auto* kernel = own ? relpos_bwd_short_kernel<T, DC, NB, true, MINW> : relpos_bwd_short_kernel<T, DC, NB, false, MINW>;
  const size_t row = Geo<T, DC>::P * sizeof(T), lds = short_lds(a, NB, row);
  if (int st = lds_limit(kernel, lds)) return st;
  const int64_t blocks = (int64_t)p.parts * a.H;
  if (!grid_fits(blocks, NB * 64)) return DSP_ERR_SHAPE;
  kernel<<<dim3((uint32_t)blocks), NB * 64, lds, s>>>(p);
  if (int st = last_launch_status()) return st;
  if (!own) {
    auto* dkv = relpos_bwd_short_dkv_kernel<T, DC, NB, MINW>;
    const size_t dkv_lds = (size_t)2 * 32 * NB * (row + 4) + shared_tables(a);
    if (int st = lds_limit(dkv, dkv_lds)) return st;
    const int64_t per_cu = std::min<int64_t>(8 / NB, 160 * 1024 / dkv_lds);
    const int64_t want = (256 * per_cu + a.Hkv - 1) / a.Hkv;
    const int64_t parts = (std::min(a.B * a.X, want) + 7) / 8 * 8;
    if (!grid_fits(parts * a.Hkv, NB * 64)) return DSP_ERR_SHAPE;
    dkv<<<dim3((uint32_t)(parts * a.Hkv)), NB * 64, dkv_lds, s>>>(p, (uint32_t)parts);
    if (int st = last_launch_status()) return st;
  }
  return bias_grad<T>(p, a, s);
}

template <typename T, int DC, int NW>
int start_dq(BwdParams& p, const RelposArgs& a, hipStream_t s) {
  // 32 keys a tile and registers for two waves per SIMD against 64 keys, the whole
  // gradient: 32 heads of 2000 x 128 causal 787 and 1308 us, 16 of 72 321 and 314, 8 x 16
  // units of 4096 x 72 4200 and 4150.  Three waves for bf16 up to 64 columns: 32 heads of
  // 2000 x 64 causal 388 with 32 keys, 557 with 64, and 410 with two waves and either.  fp32
  // up to 96 columns with two waves and some spills is within 10% of one wave either way: 8 x
  // 16 units of 700 x 64 639 and 694, of 300 x 96 314 and 330, of 700 x 72 1020 and 938.
  constexpr int KB = 32, MINW = sizeof(T) == 2 && DC <= 64 ? 3 : sizeof(T) == 2 || DC <= 96 ? 2 : 1;
  const size_t n_tab = 2 * ((size_t)p.bias.M + kEdge) + 1;
  p.n_blk = (uint32_t)((a.Lq + 32 * NW - 1) / (32 * NW));
  const size_t lds = (size_t)4 * KB * Geo<T, DC>::P * sizeof(T) + (size_t)NW * kDiag * 4 + n_tab * 4 * (1 + NW);
  auto* kernel = relpos_bwd_dq_kernel<T, DC, NW, KB, MINW>;
  if (int st = lds_limit(kernel, lds)) return st;
  kernel<<<dim3(p.H * p.parts), NW * 64, lds, s>>>(p);
  return last_launch_status();
}

template <typename T, int DC, int KW, int QS, int QT>
int start_dkv(BwdParams& p, const RelposArgs& a, hipStream_t s) {
  constexpr int QB = 32 * QT;
  p.order = make_order(a.B * a.X, a.Hkv, 1, (a.Lk + 32 * KW - 1) / (32 * KW), a.causal);
  if (!grid_fits(order_blocks(p.order), KW * QS * 64)) return DSP_ERR_SHAPE;
  const size_t lds = (size_t)4 * QB * Geo<T, DC>::P * sizeof(T) + (size_t)4 * QB * 4 +
                     (2 * ((size_t)p.bias.M + kEdge) + 1) * 4;
  auto* kernel = relpos_bwd_dkv_kernel<T, DC, KW, QS, QT, KW * QS == 8 ? 2 : 1>;
  if (int st = lds_limit(kernel, lds)) return st;
  kernel<<<dim3((uint32_t)order_blocks(p.order)), KW * QS * 64, lds, s>>>(p);
  return last_launch_status();
}

template <typename T, int DC>
int start(BwdParams& p, const RelposArgs& a, hipStream_t s) {
  if constexpr (sizeof(T) == 2 || DC <= 64)
    if (const int nb = short_blocks(a)) return nb == 1 ? start_short<T, DC, 1>(p, a, s) : start_short<T, DC, 2>(p, a, s);
  if (a.Lq > 0) {
    if (int st = start_dq<T, DC, kDqWaves>(p, a, s)) return st;
  }
  if (int st = bias_grad<T>(p, a, s)) return st;
  if (a.Lk == 0) return DSP_OK;
  // The most keys to a work-group that still fill the chip, which holds 256 of eight
  // waves: once where units are alike, twice where masks or lengths may make them differ
  // (lengths lie on the device, so any that are given count).  Whole gradients with 8, 4 and
  // 2 blocks of keys: 4 x 2000 tokens, causal and ragged, 32 heads of 64 over 8 (256, 512 and
  // 1024 work-groups) 536, 417 and 463 us, 16 of 72 over 4 (half as many) 523, 395 and 323;
  // 64 units of 200, 16 heads of 72 over 4, not causal (256, 512, 1024) 205, 268 and 256, 16 x
  // 32 of 400 x 64 (1024 ..) 272, 325 and 373, 8 x 16 of 4096 x 72 4188, 4448 and 4950.
  auto fills = [&](int64_t keys) {
    return a.B * a.X * a.Hkv * ((a.Lk + keys - 1) / keys) >= (a.causal || a.kv_len ? 512 : 256);
  };
  if constexpr (sizeof(T) == 2 && DC <= 80) {
    if (fills(256)) return start_dkv<T, DC, 8, 1, 2>(p, a, s);
    if (fills(128)) return start_dkv<T, DC, 4, 2, 4>(p, a, s);
    return start_dkv<T, DC, 2, 4, 4>(p, a, s);
  } else {
    // wide heads and fp32: registers for four waves, in fp32 LDS for 64 queries
    if (fills(128)) return start_dkv<T, DC, 4, 1, sizeof(T) == 2 ? 2 : 1>(p, a, s);
    return start_dkv<T, DC, 2, 2, 2>(p, a, s);
  }
}

}  // namespace

size_t attn_relpos_bwd_workspace_bytes(const RelposArgs& a) {
  const int64_t stats = (a.B * a.X * a.H * a.Lq + 63) / 64 * 64;
  return (size_t)(stats + a.H * parts_of(a) * (2 * (int64_t)a.max_dist + 1)) * 4;
}

int launch_attn_relpos_bwd(const RelposArgs& a, hipStream_t s) {
  BwdParams p = {};
  p.q = a.q, p.k = a.k, p.v = a.v, p.o = a.o, p.dout = a.dout, p.lse = a.lse;
  p.dq = a.dq, p.dk = a.dk, p.dv = a.dv;
  p.delta = a.workspace;
  p.part = a.workspace + (a.B * a.X * a.H * a.Lq + 63) / 64 * 64;
  p.q_pos = a.q_pos, p.kv_len = a.kv_len;
  for (int i = 0; i < 3; ++i) p.qs[i] = a.q_strides[i], p.ks[i] = a.kv_strides[i], p.os[i] = a.o_strides[i];
  p.bias = {a.bias, a.buckets, a.max_dist, a.n_buckets};
  p.X = (uint32_t)a.X, p.H = a.H, p.grp = a.H / a.Hkv, p.Lq = (uint32_t)a.Lq, p.Lk = (uint32_t)a.Lk, p.D = a.D;
  p.BX = (uint32_t)(a.B * a.X);
  p.parts = a.Lq > 0 ? (uint32_t)parts_of(a) : 0;   // no queries: sums of nothing
  p.c = a.scale * kLog2e, p.scale = a.scale;
  p.vec = a.vec, p.causal = a.causal;
  if (a.bf16) {
    if (a.D <= 32) return start<bf16, 32>(p, a, s);
    if (a.D <= 48) return start<bf16, 48>(p, a, s);
    if (a.D <= 64) return start<bf16, 64>(p, a, s);
    if (a.D <= 72) return start<bf16, 72>(p, a, s);
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
