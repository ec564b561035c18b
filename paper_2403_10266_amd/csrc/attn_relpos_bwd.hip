// Gradient of attention with a learned relative position bias.  With
//   z_ij = scale q_i . k_j + bias[bucket(j - i - q_pos)][h],  P = softmax(z),
//   Delta_i = sum_d dO_id O_id,  dZ = P (dO V^T - Delta):
//   dV = P^T dO,  dQ = scale dZ K,  dK = scale dZ^T Q,
//   dbias[t][h] = sum of dZ_ij over every (b, x, i, j) whose distance has bucket t.
// P is recomputed from the forward's row log-sum-exp.  Two kernels, both deterministic:
// the first owns blocks of queries and loops over the keys (dQ, Delta, dbias), the
// second owns blocks of keys and loops over the queries of its group's heads (dK, dV).
//
// dbias is a sum along diagonals of dZ.  Blocks wholly past the table's end add to one
// register per lane.  In the others each lane adds its dZ to an LDS array over the
// distances; the array is private to a half of a wave, whose 32 lanes hold 32
// different distances of each register, so every element is added by one lane at a
// time in program order and the sum does not depend on timing.  A work-group stays
// with one head and runs through several blocks of queries, so the arrays are folded
// once; a last kernel adds the work-groups' sums in order and folds distances into
// buckets.
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
  uint32_t X, H, grp, Lq, Lk, n_blk, n_blocks, D, BX, parts;
  float c, scale;
  bool vec, causal;
};

__device__ __forceinline__ int64_t bx_at(const BwdParams& p, uint32_t bx, const int64_t* st) {
  return (int64_t)(bx / p.X) * st[0] + (int64_t)(bx % p.X) * st[1];
}

// ---------------------------------------------------------------------------
// dQ, Delta and the sums of dZ by distance: 32 queries of one head per wave.
template <typename T, int DC, int NW, int KB, int MINW>
__global__ __launch_bounds__(NW * 64, MINW) void relpos_bwd_dq_kernel(BwdParams p) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  constexpr int NT = NW * 64, QB = NW * 32, NKT = KB / 32, TILE = KB * G::P;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  T* lds = reinterpret_cast<T*>(smem);   // [2][K, V][KB][P]
  const int32_t near = p.bias.M + kEdge, n_tab = 2 * near + 1;
  float* tab = reinterpret_cast<float*>(lds + 4 * TILE);   // bias of distance d at near + d
  float* acc = tab + n_tab;                                // [2 NW][n_tab]: the half-waves' sums

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
  for (int32_t e = threadIdx.x; e < 2 * NW * n_tab; e += NT) acc[e] = 0.0f;
  clear_pad<T, DC>(lds, 4 * KB, D, threadIdx.x, NT);
  const float left = bias_at<T>(p.bias, p.H, h, -p.bias.M), right = bias_at<T>(p.bias, p.H, h, p.bias.M);
  float* mine = acc + (2 * wave + g) * n_tab + near;
  float sum_l = 0.0f, sum_r = 0.0f;

  const uint32_t n_items = p.BX * p.n_blk;
  for (uint32_t item = part; item < n_items; item += p.parts) {
    const uint32_t bx = item / p.n_blk;
    const uint32_t blk = p.causal ? p.n_blk - 1 - item % p.n_blk : item % p.n_blk;
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
      tk.fetch(map, kg + (int64_t)kb * p.ks[2], rows, row_bytes, D, p.vec, threadIdx.x);
      tv.fetch(map, vg + (int64_t)kb * p.ks[2], rows, row_bytes, D, p.vec, threadIdx.x);
    };
    auto stash = [&](int buf) {
      tk.stash(map, lds + buf * 2 * TILE, threadIdx.x);
      tv.stash(map, lds + buf * 2 * TILE + TILE, threadIdx.x);
    };
    if (k1) fetch(0);
    const uint32_t row = blk * QB + 32 * wave + l32;
    const bool on = row < p.Lq;
    typename M::frag qf[G::NS], df[G::NS], of[G::NS];
    row_frags<T, DC>(on ? static_cast<const T*>(p.q) + q_at + (int64_t)row * p.qs[2] : nullptr, g, D, p.vec, qf);
    row_frags<T, DC>(on ? static_cast<const T*>(p.dout) + o_at + (int64_t)row * p.os[2] : nullptr, g, D, p.vec, df);
    row_frags<T, DC>(on ? static_cast<const T*>(p.o) + o_at + (int64_t)row * p.os[2] : nullptr, g, D, p.vec, of);
    float delta = 0.0f;
#pragma unroll
    for (int s = 0; s < G::NS; ++s)
#pragma unroll
      for (int e = 0; e < G::E; ++e) delta += (float)df[s][e] * (float)of[s][e];
    delta += swap_halves(delta);
    const uint64_t stat = ((uint64_t)bx * p.H + h) * p.Lq + row;
    // a row without keys, or past the end: P = exp2(-inf) = 0
    const float l = on ? p.lse[stat] : -INFINITY;
    const float lse2 = l == -INFINITY ? INFINITY : l * kLog2e;
    if (on && g == 0) p.delta[stat] = delta;

    ColAcc<T, DC> dq;
    dq.zero();
    __syncthreads();   // the buffers, the table and the sums are free and set
    if (k1) stash(0);
    __syncthreads();
    const uint32_t n_it = (k1 + KB - 1) / KB;
    const int32_t wq = q0 + 32 * wave;
    for (uint32_t it = 0; it < n_it; ++it) {
      const uint32_t kb = it * KB;
      const bool more = it + 1 < n_it;
      if (more) fetch(kb + KB);
      const T* kl = lds + (it & 1) * 2 * TILE;
      const T* vl = kl + TILE;
      if (!(p.causal && (int32_t)kb > wq + 31)) {
        floatx16 s[NKT], dp[NKT];
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
          for (int r = 0; r < 16; ++r) s[kt][r] = dp[kt][r] = 0.0f;
#pragma unroll
        for (int st = 0; st < G::NS; ++st)
#pragma unroll
          for (int kt = 0; kt < NKT; ++kt) {
            const int at = (32 * kt + l32) * G::P + 2 * G::E * st + G::E * g;
            s[kt] = M::mma(*reinterpret_cast<const typename M::frag*>(kl + at), qf[st], s[kt]);
            dp[kt] = M::mma(*reinterpret_cast<const typename M::frag*>(vl + at), df[st], dp[kt]);
          }
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt) {
          const int32_t key0 = (int32_t)kb + 32 * kt, d0 = key0 - wq;
          const bool far = d0 + 31 <= -p.bias.M || d0 - 31 >= p.bias.M;
          const int32_t at = d0 + 4 * g - l32;   // the distance of register 0
          if (far) {
            const float t = (d0 < 0 ? left : right) - lse2;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kt][r] = fmaf(s[kt][r], p.c, t);
          } else {
            const float* tb = tab + near + at;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kt][r] = fmaf(s[kt][r], p.c, tb[8 * (r / 4) + r % 4] - lse2);
          }
          if ((p.causal && d0 + 31 > 0) || key0 + 32 > (int32_t)k1) {
            const int32_t stop = p.causal ? min((int32_t)k1, wq + l32 + 1) : (int32_t)k1;
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (key0 + 8 * (r / 4) + 4 * g + r % 4 >= stop) s[kt][r] = -INFINITY;
          }
          ColB<T> z;
          float row_z = 0.0f;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float dz = __builtin_amdgcn_exp2f(s[kt][r]) * (dp[kt][r] - delta);
            dp[kt][r] = dz;
            z.set(r, dz);
          }
          if (far) {
#pragma unroll
            for (int r = 0; r < 16; ++r) row_z += dp[kt][r];
            if (d0 < 0) sum_l += row_z;
            else sum_r += row_z;
          } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) atomicAdd(mine + at + 8 * (r / 4) + r % 4, dp[kt][r]);
          }
          dq.add(kl, 32 * kt, lane, z);
        }
      }
      if (more) stash((it + 1) & 1);
      __syncthreads();
    }
    dq.scale(p.scale, lane);
    T* out = static_cast<T*>(p.dq) + q_at;
    store_rows<T, DC>(dq, lane, D, p.vec, [&](int n) -> T* {
      const uint32_t r = blk * QB + 32 * wave + n;
      return r < p.Lq ? out + (int64_t)r * p.qs[2] : nullptr;
    });
  }

  // the work-group's sums: the half-waves' arrays, the far registers, and the ends
  // of the table past M, in a fixed order
  __syncthreads();
  float* far = reinterpret_cast<float*>(lds);   // [2][NT]
  far[threadIdx.x] = sum_l;
  far[NT + threadIdx.x] = sum_r;
  for (int32_t e = threadIdx.x; e < n_tab; e += NT) {
    float v = acc[e];
    for (int w = 1; w < 2 * NW; ++w) v += acc[w * n_tab + e];
    acc[e] = v;
  }
  __syncthreads();
  if (threadIdx.x < 2) {
    const int right_end = threadIdx.x;
    float v = 0.0f;
    for (int t = 0; t < NT; ++t) v += far[right_end * NT + t];
    for (int e = 0; e < kEdge; ++e) v += acc[right_end ? n_tab - 1 - e : e];
    // M = 0: both ends are the one distance
    if (p.bias.M == 0) far[2 * NT + right_end] = v;
    else acc[right_end ? near + p.bias.M : near - p.bias.M] += v;
  }
  __syncthreads();
  if (p.bias.M == 0 && threadIdx.x == 0) acc[near] += far[2 * NT] + far[2 * NT + 1];
  __syncthreads();
  const int32_t n_out = 2 * p.bias.M + 1;
  float* w = p.part + ((uint64_t)h * p.parts + part) * n_out;
  for (int32_t e = threadIdx.x; e < n_out; e += NT) w[e] = acc[e + kEdge];
}

// dbias[t][h]: the parts of each distance in order, then the distances of each bucket.
template <typename T>
__global__ __launch_bounds__(1024) void relpos_bias_grad_kernel(BwdParams p, T* dbias) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  float* sums = reinterpret_cast<float*>(smem);
  const uint32_t h = blockIdx.x;
  const int32_t n = 2 * p.bias.M + 1;
  const float* w = p.part + (uint64_t)h * p.parts * n;
  for (int32_t e = threadIdx.x; e < n; e += blockDim.x) {
    float v = 0.0f;
    for (uint32_t s = 0; s < p.parts; ++s) v += w[(uint64_t)s * n + e];
    sums[e] = v;
  }
  __syncthreads();
  for (int32_t t = threadIdx.x; t < p.bias.nb; t += blockDim.x) {
    float v = 0.0f;
    bool masked = (float)static_cast<const T*>(p.bias.bias)[(int64_t)t * p.H + h] <= kMasked;
    for (int32_t e = 0; e < n; ++e)
      if (p.bias.buckets[e] == t) v += sums[e];
    dbias[(int64_t)t * p.H + h] = (T)(masked ? 0.0f : v);
  }
}

// ---------------------------------------------------------------------------
// dK and dV: 32 keys of one key/value head per wave, over the queries of the group.
template <typename T, int DC, int NW, int QT, int MINW>
__global__ __launch_bounds__(NW * 64, MINW) void relpos_bwd_dkv_kernel(BwdParams p) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  constexpr int NT = NW * 64, QB = 32 * QT, TILE = QB * G::P;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  T* lds = reinterpret_cast<T*>(smem);                            // [2][Q, dO][QB][P]
  float* stat = reinterpret_cast<float*>(lds + 4 * TILE);         // [2][lse2, Delta][QB]
  const int32_t near = p.bias.M + kEdge, n_tab = 2 * near + 1;
  float* tab = stat + 4 * QB;

  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t bid = blockIdx.x;
  if ((p.n_blocks & 7u) == 0) bid = (bid & 7u) * (p.n_blocks >> 3) + (bid >> 3);
  const uint32_t unit = bid / p.n_blk, blk = bid - unit * p.n_blk;
  const uint32_t hkv = p.H / p.grp, bx = unit / hkv, e = unit % hkv, b = bx / p.X;
  const int D = (int)p.D;
  const int64_t k_at = bx_at(p, bx, p.ks) + (int64_t)e * D;
  const int64_t q_bx = bx_at(p, bx, p.qs), o_bx = bx_at(p, bx, p.os);
  const uint32_t key0 = blk * 32 * NW + 32 * wave, key = key0 + l32;
  const uint32_t len = length(p.kv_len, b, p.Lk);
  const int32_t pos = position(p.q_pos, b);
  const bool on = key < len;
  typename M::frag kf[G::NS], vf[G::NS];
  row_frags<T, DC>(on ? static_cast<const T*>(p.k) + k_at + (int64_t)key * p.ks[2] : nullptr, g, D, p.vec, kf);
  row_frags<T, DC>(on ? static_cast<const T*>(p.v) + k_at + (int64_t)key * p.ks[2] : nullptr, g, D, p.vec, vf);

  const uint32_t q_row = (uint32_t)p.qs[2] * (uint32_t)sizeof(T), o_row = (uint32_t)p.os[2] * (uint32_t)sizeof(T);
  using TileT = Tile<T, DC, QB, NT>;
  const typename TileT::Map mq = TileT::map(D, q_row, threadIdx.x), mo = TileT::map(D, o_row, threadIdx.x);
  TileT tq, to;
  float pre = 0.0f;
  clear_pad<T, DC>(lds, 4 * QB, D, threadIdx.x, NT);

  ColAcc<T, DC> dk, dv;
  dk.zero();
  dv.zero();
  // the first tile of queries that sees the work-group's first key
  const int32_t first = p.causal ? (int32_t)(blk * 32 * NW) - pos : 0;
  const uint32_t it0 = first > 0 ? (uint32_t)first / QB : 0u;
  const uint32_t n_it = (p.Lq + QB - 1) / QB;
  const bool any = blk * 32 * NW < len && it0 < n_it;
  for (uint32_t hh = 0; any && hh < p.grp; ++hh) {
    const uint32_t h = e * p.grp + hh;
    const T* qg = static_cast<const T*>(p.q) + q_bx + (int64_t)h * D;
    const T* og = static_cast<const T*>(p.dout) + o_bx + (int64_t)h * D;
    const uint64_t st0 = ((uint64_t)bx * p.H + h) * p.Lq;
    const float left = bias_at<T>(p.bias, p.H, h, -p.bias.M), right = bias_at<T>(p.bias, p.H, h, p.bias.M);
    auto fetch = [&](uint32_t it) {
      const uint32_t q0 = it * QB, rows = min(p.Lq - q0, (uint32_t)QB);
      tq.fetch(mq, qg + (int64_t)q0 * p.qs[2], rows, q_row, D, p.vec, threadIdx.x);
      to.fetch(mo, og + (int64_t)q0 * p.os[2], rows, o_row, D, p.vec, threadIdx.x);
      if (threadIdx.x < 2 * QB) {
        const uint32_t i = threadIdx.x % QB;
        const bool is_delta = threadIdx.x >= QB;
        const float l = i < rows ? (is_delta ? p.delta : p.lse)[st0 + q0 + i] : is_delta ? 0.0f : -INFINITY;
        pre = is_delta ? l : l == -INFINITY ? INFINITY : l * kLog2e;
      }
    };
    auto stash = [&](int buf) {
      tq.stash(mq, lds + buf * 2 * TILE, threadIdx.x);
      to.stash(mo, lds + buf * 2 * TILE + TILE, threadIdx.x);
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
      const T* ql = lds + (it & 1) * 2 * TILE;
      const T* ol = ql + TILE;
      const float* sl = stat + (it & 1) * 2 * QB;
#pragma unroll
      for (int sub = 0; sub < QT; ++sub) {
        const int32_t q0 = pos + (int32_t)(it * QB) + 32 * sub;   // position of the block's first query
        if (key0 >= len || (p.causal && (int32_t)key0 > q0 + 31)) continue;
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
        const int32_t d0 = (int32_t)key0 - q0;
        float lse2[16], dl[16];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const floatx4 a = *reinterpret_cast<const floatx4*>(sl + 32 * sub + 8 * q + 4 * g);
          const floatx4 d = *reinterpret_cast<const floatx4*>(sl + QB + 32 * sub + 8 * q + 4 * g);
#pragma unroll
          for (int i = 0; i < 4; ++i) lse2[4 * q + i] = a[i], dl[4 * q + i] = d[i];
        }
        if (d0 + 31 <= -p.bias.M || d0 - 31 >= p.bias.M) {
          const float t = d0 < 0 ? left : right;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], p.c, t - lse2[r]);
        } else {
          const float* tb = tab + near + d0 + l32 - 4 * g;
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = fmaf(s[r], p.c, tb[-(8 * (r / 4) + r % 4)] - lse2[r]);
        }
        if (p.causal && d0 + 31 > 0) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (d0 + l32 > 8 * (r / 4) + 4 * g + r % 4) s[r] = -INFINITY;
        }
        if (key0 + 32 > len) {
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = on ? s[r] : -INFINITY;
        }
        ColB<T> pb, zb;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e2 = __builtin_amdgcn_exp2f(s[r]);
          pb.set(r, e2);
          zb.set(r, e2 * (dp[r] - dl[r]));
        }
        dv.add(ol, 32 * sub, lane, pb);
        dk.add(ql, 32 * sub, lane, zb);
      }
      if (more) stash((it + 1) & 1);
      __syncthreads();
    }
  }
  dk.scale(p.scale, lane);
  T* ko = static_cast<T*>(p.dk) + k_at;
  T* vo = static_cast<T*>(p.dv) + k_at;
  store_rows<T, DC>(dk, lane, D, p.vec, [&](int n) { return key0 + n < p.Lk ? ko + (int64_t)(key0 + n) * p.ks[2] : nullptr; });
  store_rows<T, DC>(dv, lane, D, p.vec, [&](int n) { return key0 + n < p.Lk ? vo + (int64_t)(key0 + n) * p.ks[2] : nullptr; });
}

// Work-groups of a head: enough for the chip to hold two rounds of, no more than
// there are blocks of queries.
int64_t parts_of(const RelposArgs& a, int64_t qb) {
  const int64_t items = a.B * a.X * ((a.Lq + qb - 1) / qb);
  const int64_t want = (1024 + a.H - 1) / a.H;
  return std::max<int64_t>(1, std::min(items, want));
}
constexpr int kQB = 128;

template <typename K>
int lds_limit(K* kernel, size_t lds) {
  if (lds <= 64 * 1024) return DSP_OK;
  return hip_status(
      hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
}

template <typename T, int DC>
int start(BwdParams& p, const RelposArgs& a, hipStream_t s) {
  using G = Geo<T, DC>;
  constexpr int NW = 4, KB = 32;
  const size_t n_tab = 2 * ((size_t)p.bias.M + kEdge) + 1;
  if (a.Lq > 0) {
    p.n_blk = (uint32_t)((a.Lq + 32 * NW - 1) / (32 * NW));
    const size_t lds = (size_t)4 * KB * G::P * sizeof(T) + n_tab * 4 * (1 + 2 * NW);
    auto* kernel = relpos_bwd_dq_kernel<T, DC, NW, KB, 1>;
    if (int st = lds_limit(kernel, lds)) return st;
    kernel<<<dim3(p.H * p.parts), NW * 64, lds, s>>>(p);
    if (int st = last_launch_status()) return st;
  }
  relpos_bias_grad_kernel<T><<<dim3(p.H), 1024, (2 * (size_t)p.bias.M + 1) * 4, s>>>(p, static_cast<T*>(a.dbias));
  if (int st = last_launch_status()) return st;
  if (a.Lk > 0) {
    constexpr int QT = 1;
    p.n_blk = (uint32_t)((a.Lk + 32 * NW - 1) / (32 * NW));
    const int64_t blocks = a.B * a.X * a.Hkv * p.n_blk;
    if (!grid_fits(blocks, NW * 64)) return DSP_ERR_SHAPE;
    p.n_blocks = (uint32_t)blocks;
    const size_t lds = (size_t)4 * 32 * QT * G::P * sizeof(T) + (size_t)4 * 32 * QT * 4 + n_tab * 4;
    auto* kernel = relpos_bwd_dkv_kernel<T, DC, NW, QT, 1>;
    if (int st = lds_limit(kernel, lds)) return st;
    kernel<<<dim3(p.n_blocks), NW * 64, lds, s>>>(p);
  }
  return last_launch_status();
}

}  // namespace

size_t attn_relpos_bwd_workspace_bytes(const RelposArgs& a) {
  const int64_t stats = (a.B * a.X * a.H * a.Lq + 63) / 64 * 64;
  return (size_t)(stats + a.H * parts_of(a, kQB) * (2 * (int64_t)a.max_dist + 1)) * 4;
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
  p.parts = a.Lq > 0 ? (uint32_t)parts_of(a, kQB) : 0;   // no queries: sums of nothing
  p.c = a.scale * kLog2e, p.scale = a.scale;
  p.vec = a.vec, p.causal = a.causal;
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
