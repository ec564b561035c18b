// Norm of queries and keys for each head, with the position rotation in the same
// pass, and its gradient.  For each token and head, x of width D:
//   n = g * x * r,  r = 1 / sqrt(mean(x^2) + eps)
//   y = R(p) n: for pair i of the first `rot` elements, with (c, s) = row p of
//       the table,  (a, b) -> (a c - b s, b c + a s).
// Gradient, with dn = R(p)^T dy (the turn back) and w = g * dn:
//   dg = sum over tokens and heads of dn * x * r,
//   dx = r * (w - x * r^2 * mean(w * x)).
// Everything between the loads and the stores is fp32; y and dx are rounded once.
//
// The pass is bound by HBM: each element is read once and written once (the
// gradient reads x and dy).  A row (one head of one token) is cut into chunks of
// 16 bytes, one per lane, and consecutive rows follow each other in a wave (seven
// rows of nine chunks at D = 72 in bf16), so a wave's loads cover one contiguous
// stretch of memory whatever D is.  The sums over a row are segmented wave
// reductions.  A chunk always holds whole pairs: adjacent pairs lie in one 16-byte
// run, pairs (i, i + rot/2) in two runs of 8 bytes, one of each half, so no lane
// needs another's elements.  A lane keeps its gains in registers and, for the
// gradient, its share of dg; the lanes' shares are added in a fixed order.
// Measured: 129600 tokens of 32 + 32 heads of 64 in bf16 400-410 us (5.3-5.2 TB/s, what a copy
// reaches), 32 x 1024 tokens of 16 + 16 of 72 71-73 us (4.3-4.1 TB/s; in fp32 136, 4.4),
// gradients of 13600 tokens of those 43-45 us and 4 for the gains (4.4-4.2 TB/s).
// Where the width, the rotation or an offset asks for it, a chunk is 8 or 4 bytes; what
// has no such chunk either takes a wave per row, element by element.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "dsp_internal.h"

namespace dsp {
namespace {

typedef __bf16 bf16;

constexpr int kNT = 256;   // threads of a work-group
// Row groups a wave has in flight.  129600 tokens of 64 heads of 64: 487, 430, 410 and
// 455 us for 1, 2, 4 and 8; gradients of 13600 tokens of 32 heads of 72: 57, 52, 56 and
// 62 us for 1, 2, 3 and 4 (170 registers from there on).
constexpr int unroll(bool bwd) { return bwd ? 2 : 4; }
constexpr int kMaxD = 256;

// n / d for n < 2^31 by a multiplication
struct FastDiv {
  uint32_t d, m, s;
};
FastDiv fast_div(uint32_t d) {
  uint32_t s = 0;
  while ((uint64_t(1) << s) < d) ++s;
  return {d, (uint32_t)(((uint64_t(1) << 32) * ((uint64_t(1) << s) - d)) / d + 1), s};
}
__device__ __forceinline__ uint32_t div(uint32_t n, const FastDiv& f) { return (__umulhi(n, f.m) + n) >> f.s; }

struct Side {  // queries or keys
  const void* x;
  const void* dy;  // gradient only
  void* y;         // y, or dx
  const void* g;   // gains, or null
  int64_t xs[3], ds[3], ys[3];  // element strides of x, dy and y along b, x, l
  FastDiv heads;
  uint32_t rows;   // tokens x heads
  uint32_t blocks;
};

struct NormParams {
  Side side[2];
  const float* cos;
  const float* sin;
  const int32_t* pos;  // [B][L], or null: position l
  float* part;         // gradient of the gains: [blocks of both sides][D], or null
  uint32_t P, R, D;
  uint32_t G, HP;      // lanes of a row, rows of a wave
  FastDiv L, X;
  float eps;
};

// E elements, and half of them: adjacent pairs lie in one run of E, pairs (i, i + rot/2)
// in two of E / 2
template <typename T, int E>
struct Vec {
  typedef T whole __attribute__((ext_vector_type(E)));
  typedef T half __attribute__((ext_vector_type(E / 2)));
};
template <typename T>
struct Vec<T, 2> {
  typedef T whole __attribute__((ext_vector_type(2)));
  typedef T half __attribute__((ext_vector_type(1)));
};

struct Where {
  uint32_t h, l, x, b;
};
__device__ __forceinline__ Where where(const NormParams& p, const Side& s, uint32_t row) {
  Where w;
  const uint32_t t = div(row, s.heads);
  w.h = row - t * s.heads.d;
  const uint32_t bx = div(t, p.L);
  w.l = t - bx * p.L.d;
  w.b = div(bx, p.X);
  w.x = bx - w.b * p.X.d;
  return w;
}
__device__ __forceinline__ int64_t at(const Where& w, const int64_t* st, uint32_t D) {
  return (int64_t)w.b * st[0] + (int64_t)w.x * st[1] + (int64_t)w.l * st[2] + (int64_t)w.h * D;
}
// the table's row of a token, or -1 where its position has none
__device__ __forceinline__ int64_t table_row(const NormParams& p, const Where& w) {
  if (!p.pos) return w.l;
  const int32_t q = p.pos[(int64_t)w.b * p.L.d + w.l];
  return (uint32_t)q < p.P ? q : -1;
}

// a lane's E elements as they lie, and in pair order: a[i], b[i] are the two of its
// i-th pair
template <typename T, int E, bool HALF>
struct Raw;
template <typename T, int E>
struct Raw<T, E, true> {
  using V = Vec<T, E>;
  typename V::half u, v;
  __device__ __forceinline__ void load(const T* x, uint32_t o0, uint32_t o1) {
    u = *reinterpret_cast<const typename V::half*>(x + o0);
    v = *reinterpret_cast<const typename V::half*>(x + o1);
  }
  __device__ __forceinline__ void pairs(float (&a)[E / 2], float (&b)[E / 2]) const {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) a[i] = (float)u[i], b[i] = (float)v[i];
  }
};
template <typename T, int E>
struct Raw<T, E, false> {
  using V = Vec<T, E>;
  typename V::whole u;
  __device__ __forceinline__ void load(const T* x, uint32_t o0, uint32_t) {
    u = *reinterpret_cast<const typename V::whole*>(x + o0);
  }
  __device__ __forceinline__ void pairs(float (&a)[E / 2], float (&b)[E / 2]) const {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) a[i] = (float)u[2 * i], b[i] = (float)u[2 * i + 1];
  }
};
template <typename T, int E, bool HALF>
__device__ __forceinline__ void store(T* y, uint32_t o0, uint32_t o1, const float (&a)[E / 2],
                                      const float (&b)[E / 2]) {
  using V = Vec<T, E>;
  if constexpr (HALF) {
    typename V::half u, v;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) u[i] = (T)a[i], v[i] = (T)b[i];
    *reinterpret_cast<typename V::half*>(y + o0) = u;
    *reinterpret_cast<typename V::half*>(y + o1) = v;
  } else {
    typename V::whole u;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) u[2 * i] = (T)a[i], u[2 * i + 1] = (T)b[i];
    *reinterpret_cast<typename V::whole*>(y + o0) = u;
  }
}

// sum over the G lanes of a row (j: this lane's place in it), in every one of them
__device__ __forceinline__ float row_sum(float v, uint32_t G, uint32_t j, int lane) {
  for (uint32_t off = 1; off < G; off <<= 1) {
    const float t = __shfl_down(v, off);
    v += j + off < G ? t : 0.0f;
  }
  return __shfl(v, lane - (int)j);
}

template <typename T, int E, bool HALF, bool BWD>
__global__ __launch_bounds__(kNT) void qk_norm_kernel(NormParams p) {
  constexpr int N = E / 2, kUnr = unroll(BWD);
  __shared__ float red[BWD ? kNT * E : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int which = blockIdx.x >= p.side[0].blocks;
  const Side& s = p.side[which];
  const uint32_t blk = blockIdx.x - (which ? p.side[0].blocks : 0);
  const uint32_t slot = lane / p.G, j = lane - slot * p.G;
  const bool on = slot < p.HP;
  const bool turns = E * j < p.R;  // R is a multiple of E
  const uint32_t o0 = HALF && turns ? N * j : E * j;
  const uint32_t o1 = HALF && turns ? p.R / 2 + N * j : E * j + N;
  const float inv_d = 1.0f / (float)p.D;

  float ga[N], gb[N], da[N], db[N];
#pragma unroll
  for (int i = 0; i < N; ++i) ga[i] = gb[i] = 1.0f, da[i] = db[i] = 0.0f;
  if (s.g) {
    Raw<T, E, HALF> raw;
    raw.load(static_cast<const T*>(s.g), o0, o1);
    raw.pairs(ga, gb);
  }

  typedef float fv __attribute__((ext_vector_type(N)));
  const uint32_t group = (kNT / 64) * p.HP * kUnr;  // rows of a work-group's pass
  for (uint64_t first = (uint64_t)blk * group; first < s.rows; first += (uint64_t)s.blocks * group) {
    // everything the rows need is asked for at once, without branches: rows past the
    // end repeat the last one and are not written
    Raw<T, E, HALF> rx[kUnr], ry[kUnr];
    fv c[kUnr], sn[kUnr];
    int64_t to[kUnr];
    bool ok[kUnr], known[kUnr];
#pragma unroll
    for (int u = 0; u < kUnr; ++u) {
      const uint64_t row = first + ((uint32_t)wave * kUnr + u) * p.HP + slot;
      ok[u] = on && row < s.rows;
      const Where w = where(p, s, row < s.rows ? (uint32_t)row : s.rows - 1);
      to[u] = at(w, s.ys, p.D);
      rx[u].load(static_cast<const T*>(s.x) + at(w, s.xs, p.D), o0, o1);
      if (BWD) ry[u].load(static_cast<const T*>(s.dy) + at(w, s.ds, p.D), o0, o1);
      known[u] = true;
      if (p.R) {
        const int64_t t = table_row(p, w);
        known[u] = t >= 0;
        const int64_t e = (known[u] ? t : 0) * (p.R / 2) + (turns ? N * j : 0);
        c[u] = *reinterpret_cast<const fv*>(p.cos + e);
        sn[u] = *reinterpret_cast<const fv*>(p.sin + e);
      }
    }
#pragma unroll
    for (int u = 0; u < kUnr; ++u) {
      float a[N], b[N], ya[N], yb[N];
      rx[u].pairs(a, b);
      if (BWD) ry[u].pairs(ya, yb);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        c[u][i] = !turns ? 1.0f : known[u] ? c[u][i] : NAN;
        sn[u][i] = !turns ? 0.0f : known[u] ? sn[u][i] : NAN;
      }
      float sq = 0.0f;
#pragma unroll
      for (int i = 0; i < N; ++i) sq += a[i] * a[i] + b[i] * b[i];
      float wx = 0.0f;
      if (BWD) {
#pragma unroll
        for (int i = 0; i < N; ++i) {  // dn, then w = g dn
          const float na = ya[i] * c[u][i] + yb[i] * sn[u][i];
          const float nb = yb[i] * c[u][i] - ya[i] * sn[u][i];
          ya[i] = na, yb[i] = nb;
          wx += ga[i] * na * a[i] + gb[i] * nb * b[i];
        }
        wx = row_sum(wx, p.G, j, lane);
      }
      sq = row_sum(sq, p.G, j, lane);
      const float r = 1.0f / sqrtf(sq * inv_d + p.eps);
      float oa[N], ob[N];
      if constexpr (BWD) {
        const float k = r * r * inv_d * wx;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          da[i] += ok[u] ? ya[i] * (a[i] * r) : 0.0f;
          db[i] += ok[u] ? yb[i] * (b[i] * r) : 0.0f;
          oa[i] = r * (ga[i] * ya[i] - a[i] * k);
          ob[i] = r * (gb[i] * yb[i] - b[i] * k);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float na = a[i] * r * ga[i], nb = b[i] * r * gb[i];
          oa[i] = na * c[u][i] - nb * sn[u][i];
          ob[i] = nb * c[u][i] + na * sn[u][i];
        }
      }
      if (ok[u]) store<T, E, HALF>(static_cast<T*>(s.y) + to[u], o0, o1, oa, ob);
    }
  }
  if constexpr (BWD) {
    if (!p.part) return;
    // the lanes' shares of dg: element e of chunk j from every slot of every wave
#pragma unroll
    for (int i = 0; i < N; ++i) {
      red[threadIdx.x * E + i] = on ? da[i] : 0.0f;
      red[threadIdx.x * E + N + i] = on ? db[i] : 0.0f;
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < p.D; e += kNT) {
      const uint32_t jj = e / E, i = e % E;  // chunk, element of its registers
      float v = 0.0f;
      for (int w = 0; w < kNT / 64; ++w)
        for (uint32_t sl = 0; sl < p.HP; ++sl) v += red[(w * 64 + sl * p.G + jj) * E + i];
      const bool half_turn = HALF && E * jj < p.R;
      // registers i < N hold the first elements of the pairs
      const uint32_t d = HALF ? (i < N ? (half_turn ? N * jj : E * jj) + i
                                       : (half_turn ? p.R / 2 + N * jj : E * jj + N) + i - N)
                              : E * jj + (i < N ? 2 * i : 2 * (i - N) + 1);
      p.part[(uint64_t)blockIdx.x * p.D + d] = v;
    }
  }
}

// The same pass for any width up to 256, rotation and alignment: a wave per row,
// lane e + 64 t the element d = e + 64 t with its pair's partner.
template <typename T, bool BWD>
__global__ __launch_bounds__(kNT) void qk_norm_any_kernel(NormParams p, int half) {
  constexpr int NE = kMaxD / 64;
  __shared__ float red[BWD ? (kNT / 64) * kMaxD : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int which = blockIdx.x >= p.side[0].blocks;
  const Side& s = p.side[which];
  const uint32_t blk = blockIdx.x - (which ? p.side[0].blocks : 0);
  const float inv_d = 1.0f / (float)p.D;
  uint32_t mate[NE], pair[NE];
  float sign[NE], g[NE], gm[NE], dg[NE];
#pragma unroll
  for (int t = 0; t < NE; ++t) {
    const uint32_t d = lane + 64 * t;
    const bool turns = d < p.R;
    const bool second = half ? d >= p.R / 2 : (d & 1);
    pair[t] = half ? (second ? d - p.R / 2 : d) : d / 2;
    mate[t] = !turns ? d : half ? (second ? d - p.R / 2 : d + p.R / 2) : (d ^ 1u);
    sign[t] = second ? 1.0f : -1.0f;
    const bool in = d < p.D;
    g[t] = s.g && in ? (float)static_cast<const T*>(s.g)[d] : 1.0f;
    gm[t] = s.g && in ? (float)static_cast<const T*>(s.g)[mate[t]] : 1.0f;
    dg[t] = 0.0f;
  }
  for (uint64_t row = (uint64_t)blk * (kNT / 64) + wave; row < s.rows; row += (uint64_t)s.blocks * (kNT / 64)) {
    const Where w = where(p, s, (uint32_t)row);
    const T* x = static_cast<const T*>(s.x) + at(w, s.xs, p.D);
    const T* dy = BWD ? static_cast<const T*>(s.dy) + at(w, s.ds, p.D) : nullptr;
    const int64_t tr = p.R ? table_row(p, w) : 0;
    float v[NE], vm[NE], u[NE], um[NE], c[NE], sn[NE], sq = 0.0f, wx = 0.0f;
#pragma unroll
    for (int t = 0; t < NE; ++t) {
      const uint32_t d = lane + 64 * t;
      v[t] = vm[t] = u[t] = um[t] = sn[t] = 0.0f;
      c[t] = 1.0f;
      if (d < p.D) {
        v[t] = (float)x[d];
        vm[t] = (float)x[mate[t]];
        if (BWD) u[t] = (float)dy[d], um[t] = (float)dy[mate[t]];
        if (d < p.R) {
          c[t] = tr >= 0 ? p.cos[tr * (p.R / 2) + pair[t]] : NAN;
          sn[t] = tr >= 0 ? p.sin[tr * (p.R / 2) + pair[t]] : NAN;
        }
      }
      sq += v[t] * v[t];
    }
    float dn[NE];
#pragma unroll
    for (int t = 0; t < NE; ++t) {
      dn[t] = u[t] * c[t] - sign[t] * um[t] * sn[t];
      wx += g[t] * dn[t] * v[t];
    }
#pragma unroll
    for (int off = 32; off; off >>= 1) {
      sq += __shfl_xor(sq, off);
      if (BWD) wx += __shfl_xor(wx, off);
    }
    const float r = 1.0f / sqrtf(sq * inv_d + p.eps);
    T* y = static_cast<T*>(s.y) + at(w, s.ys, p.D);
#pragma unroll
    for (int t = 0; t < NE; ++t) {
      const uint32_t d = lane + 64 * t;
      float o;
      if (BWD) {
        dg[t] += dn[t] * (v[t] * r);
        o = r * (g[t] * dn[t] - v[t] * (r * r * inv_d * wx));
      } else {
        o = v[t] * r * g[t] * c[t] + sign[t] * (vm[t] * r * gm[t]) * sn[t];
      }
      if (d < p.D) y[d] = (T)o;
    }
  }
  if constexpr (BWD) {
    if (!p.part) return;
#pragma unroll
    for (int t = 0; t < NE; ++t) red[wave * kMaxD + lane + 64 * t] = dg[t];
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < p.D; d += kNT) {
      float v = 0.0f;
      for (int w = 0; w < kNT / 64; ++w) v += red[w * kMaxD + d];
      p.part[(uint64_t)blockIdx.x * p.D + d] = v;
    }
  }
}

// dg[d] = sum over a side's work-groups of part[w][d], in a fixed order: 16 lanes
// of columns by 64 interleaved rows, then the 64 sums in turn.
__global__ __launch_bounds__(1024) void qk_norm_gain_kernel(const float* part, float* dgq, float* dgk, uint32_t bq,
                                                            uint32_t bk, uint32_t D) {
  __shared__ float red[64][17];
  const uint32_t col = threadIdx.x & 15, r = threadIdx.x >> 4, d = blockIdx.x * 16 + col;
  const bool key = blockIdx.y;
  float* dg = key ? dgk : dgq;
  if (!dg) return;
  const float* src = part + (key ? (uint64_t)bq * D : 0);
  const uint32_t n = key ? bk : bq;
  float v = 0.0f;
  if (d < D)
#pragma unroll 8
    for (uint32_t w = r; w < n; w += 64) v += src[(uint64_t)w * D + d];
  red[r][col] = v;
  __syncthreads();
  if (r == 0 && d < D) {
    for (int i = 1; i < 64; ++i) v += red[i][col];
    dg[d] = v;
  }
}

// work-groups a side's gradient runs on: enough to fill the chip, few enough
// that their shares of dg stay small
constexpr uint32_t kGradBlocks = 1024;

// The elements of a lane's chunk: 16 bytes' worth, or a half or a quarter of it where the
// width, the rotation or an alignment asks for it; 0: no such chunk (a lane for each
// element then).
int chunk(const QkNormArgs& a, bool bwd) {
  const int es = a.bf16 ? 2 : 4;
  for (int E = 16 / es; E >= 2; E /= 2) {
    if (a.D % E || a.rot % E || a.D / E > 64) continue;
    auto ok = [&](const void* ptr, const int64_t* st) {
      return reinterpret_cast<uintptr_t>(ptr) % (E * es) == 0 && st[0] % E == 0 && st[1] % E == 0 && st[2] % E == 0;
    };
    bool all = !a.rot || (reinterpret_cast<uintptr_t>(a.cos) % (2 * E) == 0 && reinterpret_cast<uintptr_t>(a.sin) % (2 * E) == 0);
    for (int i = 0; i < 2; ++i) {
      const QkNormSide& s = a.side[i];
      if (!s.heads) continue;
      all = all && ok(s.x, s.x_strides) && ok(s.y, s.y_strides) && (!bwd || ok(s.dy, s.dy_strides)) &&
            reinterpret_cast<uintptr_t>(s.gain) % (E * es) == 0;
    }
    if (all) return E;
  }
  return 0;
}

struct Plan {
  int E;
  uint32_t G, HP, blocks[2];
};
Plan plan(const QkNormArgs& a, bool bwd) {
  Plan r = {};
  r.E = chunk(a, bwd);
  r.G = r.E ? a.D / r.E : 64;
  r.HP = 64 / r.G;
  const int64_t per = r.E ? (kNT / 64) * r.HP * unroll(bwd) : kNT / 64;
  for (int i = 0; i < 2; ++i) {
    const int64_t rows = a.B * a.X * a.L * a.side[i].heads;
    int64_t n = (rows + per - 1) / per;
    n = std::min<int64_t>(n, bwd ? kGradBlocks : (int64_t(1) << 22));
    r.blocks[i] = (uint32_t)n;
  }
  return r;
}

template <typename T, int E>
void launch_chunks(const NormParams& p, dim3 grid, bool half, bool bwd, hipStream_t s) {
  if (half) {
    if (bwd) qk_norm_kernel<T, E, true, true><<<grid, kNT, 0, s>>>(p);
    else qk_norm_kernel<T, E, true, false><<<grid, kNT, 0, s>>>(p);
  } else {
    if (bwd) qk_norm_kernel<T, E, false, true><<<grid, kNT, 0, s>>>(p);
    else qk_norm_kernel<T, E, false, false><<<grid, kNT, 0, s>>>(p);
  }
}
template <typename T>
void launch(const NormParams& p, const Plan& pl, bool half, bool bwd, hipStream_t s) {
  const dim3 grid(pl.blocks[0] + pl.blocks[1]);
  if (pl.E == 8) {
    if constexpr (sizeof(T) == 2) launch_chunks<T, 8>(p, grid, half, bwd, s);
  } else if (pl.E == 4) {
    launch_chunks<T, 4>(p, grid, half, bwd, s);
  } else if (pl.E == 2) {
    launch_chunks<T, 2>(p, grid, half, bwd, s);
  } else if (bwd) {
    qk_norm_any_kernel<T, true><<<grid, kNT, 0, s>>>(p, half);
  } else {
    qk_norm_any_kernel<T, false><<<grid, kNT, 0, s>>>(p, half);
  }
}

}  // namespace

size_t qk_norm_workspace_bytes(int64_t tokens, int H, int Hkv, int D) {
  // at most kGradBlocks work-groups of each side, at least four rows in each
  auto n = [&](int64_t heads) { return std::min<int64_t>(kGradBlocks, (tokens * heads + 3) / 4); };
  return (size_t)(n(H) + n(Hkv)) * (size_t)D * 4;
}

int launch_qk_norm(const QkNormArgs& a, bool bwd, float* part, hipStream_t s) {
  const Plan pl = plan(a, bwd);
  NormParams p = {};
  for (int i = 0; i < 2; ++i) {
    const QkNormSide& in = a.side[i];
    Side& o = p.side[i];
    o.x = in.x, o.dy = in.dy, o.y = in.y, o.g = in.gain;
    for (int k = 0; k < 3; ++k) o.xs[k] = in.x_strides[k], o.ys[k] = in.y_strides[k], o.ds[k] = in.dy_strides[k];
    o.heads = fast_div(std::max(in.heads, 1));
    o.rows = (uint32_t)(a.B * a.X * a.L * in.heads);
    o.blocks = pl.blocks[i];
  }
  p.cos = a.cos, p.sin = a.sin, p.pos = a.pos;
  const bool gains = bwd && (a.side[0].dgain || a.side[1].dgain);
  p.part = gains ? part : nullptr;
  p.P = (uint32_t)a.P, p.R = a.rot, p.D = a.D, p.G = pl.G, p.HP = pl.HP;
  p.L = fast_div((uint32_t)std::max<int64_t>(a.L, 1)), p.X = fast_div((uint32_t)std::max<int64_t>(a.X, 1));
  p.eps = a.eps;
  if (pl.blocks[0] + pl.blocks[1] == 0) {
    // no rows
  } else if (a.bf16) launch<bf16>(p, pl, a.half, bwd, s);
  else launch<float>(p, pl, a.half, bwd, s);
  const int st = last_launch_status();
  if (st != DSP_OK || !gains) return st;
  qk_norm_gain_kernel<<<dim3((a.D + 15) / 16, 2), 1024, 0, s>>>(part, a.side[0].dgain, a.side[1].dgain, pl.blocks[0],
                                                                pl.blocks[1], a.D);
  return last_launch_status();
}

}  // namespace dsp
