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
// The subtracted reference follows the running maximum lazily: it moves (and the sums
// are rescaled) only when a score exceeds it by 2^8, so the usual tile pays one
// comparison.
//
// Few queries against many keys (a new token against a cache): the queries of a
// key/value head's group share one block of 32 columns, and the keys are cut among
// work-groups, whose unnormalised sums a second kernel joins.
#include <algorithm>
#include <type_traits>

#include "attn_relpos.h"

namespace dsp {
namespace {

constexpr float kMove = 8.0f;   // exp2 units a score may exceed the reference by

struct FwdParams {
  const void* q;
  const void* k;
  const void* v;
  void* o;
  float* lse;
  float* part;   // split keys: per work-group 32 maxima, 32 sums, 32 rows of D
  const int32_t* q_pos;
  const int32_t* kv_len;
  int64_t qs[3], ks[3], os[3];
  BiasArgs bias;
  uint32_t X, H, grp, Lq, Lk, n_qb, n_split, split_keys, n_blocks, D;
  uint32_t tab;      // distances of the LDS table, for each head of a work-group
  uint32_t cols;     // packed: queries x group heads of a unit; 0: one head's queries
  float c;           // scale * log2(e)
  bool vec, vec_o, causal;
};

template <typename T, int DC, int NW, int QT, int KB, int NBUF, int MINW>
__global__ __launch_bounds__(NW * 64, MINW) void relpos_fwd_kernel(FwdParams p) {
  using G = Geo<T, DC>;
  using M = Mx<T>;
  constexpr int NT = NW * 64, QB = NW * 32 * QT, NKT = KB / 32;
  constexpr int TILE = KB * G::P;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  T* lds = reinterpret_cast<T*>(smem);                       // [NBUF][K, V][KB][P]
  float* tab = reinterpret_cast<float*>(lds + NBUF * 2 * TILE);

  const int lane = threadIdx.x & 63, l32 = lane & 31, g = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // work-group -> (unit, query block, split); each XCD takes a contiguous range
  uint32_t bid = blockIdx.x;
  if ((p.n_blocks & 7u) == 0) bid = (bid & 7u) * (p.n_blocks >> 3) + (bid >> 3);
  const uint32_t split = bid % p.n_split, ub = bid / p.n_split;
  const uint32_t unit = ub / p.n_qb;
  // causal: the last query blocks have the most keys and start first
  const uint32_t qb = p.causal ? p.n_qb - 1 - ub % p.n_qb : ub % p.n_qb;
  const uint32_t per_bx = p.cols ? p.H / p.grp : p.H;
  const uint32_t bx = unit / per_bx, h0 = p.cols ? unit % per_bx * p.grp : unit % per_bx;
  const uint32_t b = bx / p.X, x = bx % p.X;
  const int D = (int)p.D;
  const T* kg = static_cast<const T*>(p.k) + (int64_t)b * p.ks[0] + (int64_t)x * p.ks[1] + (int64_t)(h0 / p.grp) * D;
  const T* vg = static_cast<const T*>(p.v) + (kg - static_cast<const T*>(p.k));
  const T* qg = static_cast<const T*>(p.q) + (int64_t)b * p.qs[0] + (int64_t)x * p.qs[1] + (int64_t)h0 * D;

  const int32_t q0 = position(p.q_pos, b) + (int32_t)(qb * QB);   // position of the block's first query
  const uint32_t len = length(p.kv_len, b, p.Lk);
  const uint32_t nq = p.cols ? p.Lq : min(p.Lq - qb * QB, (uint32_t)QB);
  // keys [k0, k1) of this work-group: whole tiles from its split's first key on
  const uint32_t k0 = split * p.split_keys;
  uint32_t k1 = min(len, p.n_split > 1 ? k0 + p.split_keys : len);
  if (p.causal) {
    const int32_t last = q0 + (int32_t)nq;   // keys before it
    k1 = last <= 0 ? 0u : min(k1, (uint32_t)last);
  }
  const uint32_t row_bytes = (uint32_t)p.ks[2] * (uint32_t)sizeof(T);
  using TileT = Tile<T, DC, KB, NT>;
  const typename TileT::Map map = TileT::map(D, row_bytes);
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
  if (k0 < k1) fetch(k0);

  // the columns: head (in the unit) and query of this lane's column of tile j
  uint32_t ch[QT], cq[QT];
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    const uint32_t col = 32 * (wave * QT + j) + l32;
    ch[j] = p.cols ? min(col / p.Lq, p.grp - 1) : 0u;
    cq[j] = p.cols ? col - ch[j] * p.Lq : col;
  }
  auto row_at = [&](uint32_t c, uint32_t h, int64_t rs) { return (int64_t)(qb * QB + c) * rs + (int64_t)h * D; };
  typename M::frag qf[QT][G::NS];
#pragma unroll
  for (int j = 0; j < QT; ++j)
    row_frags<T, DC>(cq[j] < nq ? qg + row_at(cq[j], ch[j], p.qs[2]) : nullptr, g, D, p.vec, qf[j]);

  // the table: distances lo .. of each head of the work-group
  const int32_t kend = (int32_t)((k1 + KB - 1) / KB * KB);
  const int32_t lo = max(-(p.bias.M + kEdge), (int32_t)k0 - (q0 + QB - 1));
  const int32_t hi = min(p.bias.M + kEdge, kend - 1 - q0);
  const uint32_t nh = p.cols ? p.grp : 1;
  if (k0 < k1)
    for (uint32_t hh = 0; hh < nh; ++hh)
      for (int32_t d = lo + (int32_t)threadIdx.x; d <= hi; d += NT)
        tab[hh * p.tab + (uint32_t)(d - lo)] = bias_at<T>(p.bias, p.H, h0 + hh, d);
  float left[QT], right[QT];
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    left[j] = bias_at<T>(p.bias, p.H, h0 + ch[j], -p.bias.M);
    right[j] = bias_at<T>(p.bias, p.H, h0 + ch[j], p.bias.M);
  }

  ColAcc<T, DC> o[QT];
  float ref[QT], sum[QT];
  bool set[QT];
#pragma unroll
  for (int j = 0; j < QT; ++j) {
    o[j].zero();
    ref[j] = sum[j] = 0.0f;
    set[j] = false;
  }

  clear_pad<T, DC>(lds, NBUF * 2 * KB, D, NT);
  if (k0 < k1) stash(0);
  __syncthreads();
  const uint32_t n_it = k0 < k1 ? (k1 - k0 + KB - 1) / KB : 0;
  for (uint32_t it = 0; it < n_it; ++it) {
    const uint32_t kb = k0 + it * KB;
    const bool more = NBUF > 1 && it + 1 < n_it;
    if (more) fetch(kb + KB);
    const T* kl = lds + (NBUF > 1 ? (it & 1) : 0) * 2 * TILE;
    const T* vl = kl + TILE;
    // queries of this wave are all before the tile: nothing to see
    const int32_t wq = q0 + (p.cols ? 0 : 32 * QT * wave);          // the wave's first query
    const int32_t wl = wq + (p.cols ? (int32_t)p.Lq : 32 * QT) - 1;   // and its last
    if (!(p.causal && (int32_t)kb > wl)) {
      floatx16 s[NKT][QT];
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
          const auto a =
              *reinterpret_cast<const typename M::frag*>(kl + (32 * kt + l32) * G::P + 2 * G::E * st + G::E * g);
#pragma unroll
          for (int j = 0; j < QT; ++j) s[kt][j] = M::mma(a, qf[j][st], s[kt][j]);
        }
      // scores relative to the reference, in the exp2 domain
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int j = 0; j < QT; ++j) {
          const int32_t key0 = (int32_t)kb + 32 * kt;
          const int32_t bq = p.cols ? q0 : wq + 32 * j;   // the block's first query
          const int32_t d0 = key0 - bq;
          if (d0 + 31 <= -p.bias.M || d0 - 31 >= p.bias.M) {
            const float t = (d0 < 0 ? left[j] : right[j]) - ref[j];
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kt][j][r] = fmaf(s[kt][j][r], p.c, t);
          } else {
            const float* tb = tab + ch[j] * p.tab + (key0 + 4 * g - (q0 + (int32_t)cq[j]) - lo);
#pragma unroll
            for (int r = 0; r < 16; ++r)
              s[kt][j][r] = fmaf(s[kt][j][r], p.c, tb[8 * (r / 4) + r % 4] - ref[j]);
          }
          if ((p.causal && d0 + 31 > 0) || key0 + 32 > (int32_t)k1) {
            const int32_t stop = p.causal ? min((int32_t)k1, q0 + (int32_t)cq[j] + 1) : (int32_t)k1;
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (key0 + 8 * (r / 4) + 4 * g + r % 4 >= stop) s[kt][j][r] = -INFINITY;
          }
        }
      bool move = false;
      float top[QT];
#pragma unroll
      for (int j = 0; j < QT; ++j) {
        float m = s[0][j][0];
#pragma unroll
        for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
          for (int r = 0; r < 16; ++r) m = fmaxf(m, s[kt][j][r]);
        top[j] = fmaxf(m, swap_halves(m));
        move |= top[j] > (set[j] ? kMove : -INFINITY);
      }
      if (__any(move)) {
#pragma unroll
        for (int j = 0; j < QT; ++j) {
          const bool mv = top[j] > (set[j] ? kMove : -INFINITY);
          const float d = mv ? top[j] : 0.0f;
          const float f = mv && set[j] ? __builtin_amdgcn_exp2f(-d) : 1.0f;
          ref[j] += d;
          set[j] |= mv;
          sum[j] *= f;
          o[j].scale(f, lane);
#pragma unroll
          for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kt][j][r] -= d;
        }
      }
#pragma unroll
      for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
        for (int j = 0; j < QT; ++j) {
          ColB<T> pf;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float e = __builtin_amdgcn_exp2f(s[kt][j][r]);
            sum[j] += e;
            pf.set(r, e);
          }
          o[j].add(vl, 32 * kt, lane, pf);
        }
    }
    if (more) stash((it + 1) & 1);
    __syncthreads();
  }

#pragma unroll
  for (int j = 0; j < QT; ++j) {
    const float l = sum[j] + swap_halves(sum[j]);
    if (p.n_split > 1) {   // one block of columns: the sums as they are
      float* w = p.part + (uint64_t)(unit * p.n_split + split) * (64 + 32 * p.D);
      if (g == 0) {
        w[l32] = set[j] ? ref[j] : -INFINITY;
        w[32 + l32] = l;
      }
      store_rows<T, DC>(o[j], lane, D, false, [&](int n) { return w + 64 + n * (int)p.D; });
      continue;
    }
    o[j].scale(l > 0.0f ? 1.0f / l : 0.0f, lane);
    T* og = static_cast<T*>(p.o) + (int64_t)b * p.os[0] + (int64_t)x * p.os[1] + (int64_t)h0 * D;
    store_rows<T, DC>(o[j], lane, D, p.vec_o, [&](int n) -> T* {
      const uint32_t col = 32 * (wave * QT + j) + n;
      const uint32_t hh = p.cols ? col / p.Lq : 0, i = p.cols ? col - hh * p.Lq : col;
      return (p.cols ? col < p.cols : i < nq) ? og + row_at(i, hh, p.os[2]) : nullptr;
    });
    const bool mine = p.cols ? 32u * (wave * QT + j) + l32 < p.cols : cq[j] < nq;
    if (p.lse && g == 0 && mine)
      p.lse[((uint64_t)bx * p.H + h0 + ch[j]) * p.Lq + qb * QB + cq[j]] =
          l > 0.0f ? kLn2 * (ref[j] + log2f(l)) : -INFINITY;
  }
}

// Joins the splits of a unit's columns: with the splits' references m_s, sums l_s and
// rows o_s, o = sum 2^(m_s - m) o_s / sum 2^(m_s - m) l_s.  A wave per column.
template <typename T>
__global__ __launch_bounds__(256) void relpos_join_kernel(FwdParams p, uint32_t n_cols) {
  const uint32_t wid = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (wid >= n_cols) return;
  const uint32_t unit = wid / p.cols, col = wid - unit * p.cols;
  const uint32_t stride = 64 + 32 * p.D;
  const float* w = p.part + (uint64_t)unit * p.n_split * stride;
  float m = -INFINITY;
  for (uint32_t s = lane; s < p.n_split; s += 64) m = fmaxf(m, w[(uint64_t)s * stride + col]);
#pragma unroll
  for (int off = 32; off; off >>= 1) m = fmaxf(m, __shfl_xor(m, off));
  const float top = m == -INFINITY ? 0.0f : m;
  float l = 0.0f, a0 = 0.0f, a1 = 0.0f;
  for (uint32_t s = 0; s < p.n_split; ++s) {
    const float* ws = w + (uint64_t)s * stride;
    const float f = __builtin_amdgcn_exp2f(ws[col] - top);   // no keys: exp2(-inf) = 0
    l += f * ws[32 + col];
    const float* row = ws + 64 + col * p.D;
    if (lane < p.D) a0 += f * row[lane];
    if (lane + 64 < p.D) a1 += f * row[lane + 64];
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  const uint32_t kvh = p.H / p.grp, bx = unit / kvh, hh = col / p.Lq, i = col - hh * p.Lq;
  const uint32_t h = unit % kvh * p.grp + hh, b = bx / p.X, x = bx % p.X;
  T* o = static_cast<T*>(p.o) + (int64_t)b * p.os[0] + (int64_t)x * p.os[1] + (int64_t)i * p.os[2] + (int64_t)h * p.D;
  if (lane < p.D) o[lane] = (T)(a0 * inv);
  if (lane + 64 < p.D) o[lane + 64] = (T)(a1 * inv);
  if (p.lse && lane == 0) p.lse[((uint64_t)bx * p.H + h) * p.Lq + i] = l > 0.0f ? kLn2 * (top + log2f(l)) : -INFINITY;
}

struct Choice {
  bool pack;
  int64_t n_split, split_keys;
};

// Packed columns and split keys: the queries of a group share a block of 32 columns
// where they fit in one, and the keys are cut while there are fewer work-groups than
// the chip holds at once, into pieces of at least 256 keys.
Choice choose(const RelposArgs& a) {
  Choice c = {};
  const int64_t grp = a.H / a.Hkv;
  c.n_split = 1;
  c.split_keys = a.Lk;
  c.pack = a.Lq * grp <= 32 && a.Lq > 0;
  if (!c.pack) return c;
  const int64_t units = a.B * a.X * a.Hkv;
  const int64_t want = (256 * 6 + units - 1) / units;
  const int64_t n = std::min<int64_t>(std::min<int64_t>(want, (a.Lk + 255) / 256), 1024);
  if (n > 1) {
    c.split_keys = ((a.Lk + n - 1) / n + 63) / 64 * 64;
    c.n_split = (a.Lk + c.split_keys - 1) / c.split_keys;
  }
  return c;
}

template <typename T, int DC, int NW, int QT, int KB, int NBUF, int MINW>
int start(FwdParams& p, const RelposArgs& a, const Choice& c, hipStream_t s) {
  using G = Geo<T, DC>;
  constexpr int QB = NW * 32 * QT;
  const int64_t grp = a.H / a.Hkv;
  p.n_qb = (uint32_t)((a.Lq + QB - 1) / QB);
  if (p.cols) p.n_qb = 1;
  const int64_t span = QB + (a.Lk + KB - 1) / KB * KB;
  p.tab = (uint32_t)std::min<int64_t>(2 * (p.bias.M + kEdge) + 1, span);
  const size_t lds = (size_t)NBUF * 2 * KB * G::P * sizeof(T) + (size_t)p.tab * 4 * (p.cols ? grp : 1);
  const int64_t blocks = a.B * a.X * (p.cols ? a.Hkv : a.H) * p.n_qb * p.n_split;
  if (!grid_fits(blocks, NW * 64)) return DSP_ERR_SHAPE;
  p.n_blocks = (uint32_t)blocks;
  auto* kernel = relpos_fwd_kernel<T, DC, NW, QT, KB, NBUF, MINW>;
  if (lds > 64 * 1024) {
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return DSP_ERR_HIP;
  }
  kernel<<<dim3(p.n_blocks), NW * 64, lds, s>>>(p);
  int st = last_launch_status();
  if (st != DSP_OK || p.n_split == 1) return st;
  const int64_t cols = a.B * a.X * a.Hkv * p.cols;
  relpos_join_kernel<T><<<dim3((uint32_t)((cols + 3) / 4)), 256, 0, s>>>(p, (uint32_t)cols);
  return last_launch_status();
}

template <typename T, int DC>
int start_class(FwdParams& p, const RelposArgs& a, const Choice& c, hipStream_t s) {
  if (a.Lq <= 32 || p.cols) return start<T, DC, 1, 1, 32, 2, 1>(p, a, c, s);
  return start<T, DC, 4, 1, 32, 2, 1>(p, a, c, s);
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
  p.cols = c.pack ? (uint32_t)(a.Lq * p.grp) : 0;
  p.n_split = (uint32_t)c.n_split, p.split_keys = (uint32_t)c.split_keys;
  p.c = a.scale * kLog2e;
  p.vec = a.vec, p.vec_o = a.vec, p.causal = a.causal;
  if (a.bf16) {
    if (a.D <= 32) return start_class<bf16, 32>(p, a, c, s);
    if (a.D <= 48) return start_class<bf16, 48>(p, a, c, s);
    if (a.D <= 64) return start_class<bf16, 64>(p, a, c, s);
    if (a.D <= 80) return start_class<bf16, 80>(p, a, c, s);
    if (a.D <= 96) return start_class<bf16, 96>(p, a, c, s);
    return start_class<bf16, 128>(p, a, c, s);
  }
  if (a.D <= 32) return start_class<float, 32>(p, a, c, s);
  if (a.D <= 64) return start_class<float, 64>(p, a, c, s);
  if (a.D <= 96) return start_class<float, 96>(p, a, c, s);
  return start_class<float, 128>(p, a, c, s);
}

size_t attn_relpos_workspace_bytes(const RelposArgs& a) {
  const Choice c = choose(a);
  return c.n_split > 1 ? (size_t)(a.B * a.X * a.Hkv * c.n_split) * (64 + 32 * (size_t)a.D) * 4 : 0;
}

}  // namespace dsp
