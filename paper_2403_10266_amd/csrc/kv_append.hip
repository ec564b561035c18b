// New keys and values into a paged cache, keys (and queries) turned by position on the way:
//   y_a = x_a cos - x_b sin,  y_b = x_b cos + x_a sin
// for the pairs of a head's first `rot` elements, each product and the sum rounded to
// fp32 by itself, then once to the cache's type.
//
// Caches of the tokens' own type, and the queries, go by rows: a work-group takes up to
// 16 tokens of one sequence, whole rows of K, V and Q.  Memory bounds it: 16000 tokens, 16 heads
// of 72, K, V and Q, 56.5 us, 4.0 TB/s.
//
// In 8 bits (e4m3) a page has one scale for each head, the least power of two s with
// |x| <= 448 s for every token since the page's first slot was written.  A work-group takes
// one head of one page: it finds the new tokens' largest magnitude, rounds what the page
// holds again where s has grown (a power of two: nothing but a lost last bit near the
// least values), and writes.  Up to 1024 items of eight elements stay in registers between;
// those of larger pages are read and turned twice.  32 ragged chunks of up to 700 tokens 72 us,
// 3.6 TB/s; 64 single tokens 8 us.
#include <type_traits>

#include "attn_window.h"

namespace dsp {
namespace {

struct AppendParams {
  const void* k;
  const void* v;
  const void* q;
  void* yq;
  void* k_cache;
  void* v_cache;
  float* k_scale;
  float* v_scale;
  const int32_t* table;
  const int32_t* q_start;
  const int32_t* kv_len;
  const int32_t* pos;
  const float* cos;
  const float* sin;
  int64_t k_row, v_row, q_row, y_row, page_st, slot_st, head_st;
  uint32_t N, T, P, n_pages, max_pages, shift, H, Hkv, D, rot;
  Divisor items;         // of a head: 8 elements each
  int32_t row_tokens;    // of a work-group that goes by rows: 16 at most, so that they lie in two pages at most
  uint32_t rot_items;    // the first of them, whose elements turn
  uint32_t page_groups;  // work-groups that write pages of 8 bits; the others go by rows
  bool half, e4m3, vec;
};

constexpr int kItem = 8;
constexpr int kLeastExp = -64;   // of a scale

// Item c of a head: elements at() .. of it, four pairs in the part that turns.
struct Place8 {
  uint32_t a, b;    // first elements of its two halves of four
  bool turns;
};
__device__ __forceinline__ Place8 place8(const AppendParams& p, uint32_t c) {
  Place8 e;
  e.turns = c < p.rot_items;
  if (e.turns && p.half) {
    e.a = 4 * c;
    e.b = 4 * c + p.rot / 2;
  } else {
    e.a = e.turns ? 8 * c : p.rot + 8 * (c - p.rot_items);
    e.b = e.a + 4;
  }
  return e;
}
// whether its element t is one of the head's (rot and D may end inside an item)
__device__ __forceinline__ bool inside(const AppendParams& p, const Place8& e, int t) {
  if (!e.turns) return e.a + t < p.D;
  return p.half ? e.a + t % 4 < p.rot / 2 : e.a + t < p.rot;
}

template <typename T, bool VEC>
__device__ __forceinline__ void load8(const AppendParams& p, const T* head, const Place8& e, float (&x)[8]) {
  if constexpr (VEC) {
    if constexpr (sizeof(T) == 2) {
      uint2 lo, hi;
      if (e.b == e.a + 4) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(head + e.a);
        lo = {v[0], v[1]}, hi = {v[2], v[3]};
      } else {
        lo = *reinterpret_cast<const uint2*>(head + e.a), hi = *reinterpret_cast<const uint2*>(head + e.b);
      }
      const uint32_t w[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    } else {
      const floatx4 lo = *reinterpret_cast<const floatx4*>(head + e.a), hi = *reinterpret_cast<const floatx4*>(head + e.b);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = lo[i], x[4 + i] = hi[i];
    }
  } else {
#pragma unroll
    for (int t = 0; t < 8; ++t) x[t] = inside(p, e, t) ? (float)head[t < 4 ? e.a + t : e.b + t - 4] : 0.0f;
  }
}

// turns an item's four pairs by the angles of row `at` of the table (NaN if it has none)
template <bool VEC>
__device__ __forceinline__ void turn8(const AppendParams& p, const Place8& e, int64_t at, float (&x)[8]) {
  // no fused multiply-add: a value at the border of two codes falls the same way everywhere
#pragma clang fp contract(off)
  if (!e.turns) return;
  float c[4], s[4];
  const uint32_t first = p.half ? e.a : e.a / 2;   // pair
  if (at < 0 || at >= (int64_t)p.P) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = s[i] = __builtin_nanf("");
  } else {
    const float* cr = p.cos + at * (p.rot / 2) + first;
    const float* sr = p.sin + at * (p.rot / 2) + first;
    if constexpr (VEC) {
      const floatx4 cv = *reinterpret_cast<const floatx4*>(cr), sv = *reinterpret_cast<const floatx4*>(sr);
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = cv[i], s[i] = sv[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool in = first + i < p.rot / 2;
        c[i] = in ? cr[i] : 1.0f;
        s[i] = in ? sr[i] : 0.0f;
      }
    }
  }
  float a[4], b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float xa = p.half ? x[i] : x[2 * i], xb = p.half ? x[4 + i] : x[2 * i + 1];
    a[i] = xa * c[i] - xb * s[i];
    b[i] = xb * c[i] + xa * s[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = p.half ? a[i] : i % 2 ? b[i / 2] : a[i / 2];
    x[4 + i] = p.half ? b[i] : i % 2 ? b[2 + i / 2] : a[2 + i / 2];
  }
}

template <typename T, bool VEC>
__device__ __forceinline__ void store8(const AppendParams& p, T* head, const Place8& e, const float (&x)[8]) {
  if constexpr (VEC) {
    if constexpr (sizeof(T) == 2) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bf16x2 v = {(bf16)x[2 * i], (bf16)x[2 * i + 1]};
        w[i] = __builtin_bit_cast(uint32_t, v);
      }
      if (e.b == e.a + 4) {
        *reinterpret_cast<u32x4*>(head + e.a) = u32x4{w[0], w[1], w[2], w[3]};
      } else {
        *reinterpret_cast<uint2*>(head + e.a) = {w[0], w[1]};
        *reinterpret_cast<uint2*>(head + e.b) = {w[2], w[3]};
      }
    } else {
      *reinterpret_cast<floatx4*>(head + e.a) = floatx4{x[0], x[1], x[2], x[3]};
      *reinterpret_cast<floatx4*>(head + e.b) = floatx4{x[4], x[5], x[6], x[7]};
    }
  } else {
#pragma unroll
    for (int t = 0; t < 8; ++t)
      if (inside(p, e, t)) head[t < 4 ? e.a + t : e.b + t - 4] = (T)x[t];
  }
}

// e4m3 codes of an item over the scale 1 / inv.  What is not finite becomes NaN.
template <bool VEC>
__device__ __forceinline__ void store8_e4m3(const AppendParams& p, uint8_t* head, const Place8& e, const float (&x)[8],
                                            float inv) {
  float y[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) y[t] = fabsf(x[t]) < INFINITY ? x[t] * inv : __builtin_nanf("");
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h], y[4 * h + 1], 0, false);
    w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2], y[4 * h + 3], v, true);
  }
  if constexpr (VEC) {
    if (e.b == e.a + 4) {
      *reinterpret_cast<uint2*>(head + e.a) = {w[0], w[1]};
    } else {
      *reinterpret_cast<uint32_t*>(head + e.a) = w[0];
      *reinterpret_cast<uint32_t*>(head + e.b) = w[1];
    }
  } else {
#pragma unroll
    for (int t = 0; t < 8; ++t)
      if (inside(p, e, t)) head[t < 4 ? e.a + t : e.b + t - 4] = (uint8_t)(w[t / 4] >> (8 * (t % 4)));
  }
}

// the exponent of the least power of two s with top <= 448 s = 1.75 2^8 s
__device__ __forceinline__ int scale_exp(float top) {
  const uint32_t bits = __float_as_uint(top);
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(e, kLeastExp);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Rows: up to 16 tokens of one sequence, K, V and Q, or Q alone.  A thread takes four items
// at a time, so that their loads are under way together; the rows lie in at most two pages.
template <typename T, bool VEC, int NT>
__device__ __forceinline__ void append_rows(const AppendParams& p, uint32_t w) {
  constexpr int N = 4;
  const int lane = threadIdx.x & 63;
  const uint32_t n = __builtin_amdgcn_readfirstlane(piece_owner(p.q_start, p.N, p.T, 1, p.row_tokens, 1, w, lane));
  const int32_t blk = (int32_t)w - first_piece(p.q_start, n, p.T, 1, p.row_tokens, 1);
  const Rows r = new_rows(p.q_start, n, p.T);
  if (blk < 0 || blk * p.row_tokens >= r.n) return;
  const uint32_t count = (uint32_t)min(r.n - blk * p.row_tokens, p.row_tokens);
  const int64_t p0 = (int64_t)p.kv_len[n] - r.n + blk * p.row_tokens;   // position of the first
  const int64_t row0 = (int64_t)r.first + blk * p.row_tokens;
  const uint32_t kv_heads = p.e4m3 ? 0 : p.Hkv, per = (p.H + 2 * kv_heads) * p.items.d;
  const int64_t first_pi = p0 >> p.shift;
  auto page_at = [&](int64_t pi) {
    return kv_heads && pi >= 0 && pi < (int64_t)p.max_pages ? p.table[(uint64_t)n * p.max_pages + (uint64_t)pi] : -1;
  };
  const int32_t page0 = page_at(first_pi), page1 = page_at(first_pi + 1);

  uint32_t t = threadIdx.x / per, in_row = threadIdx.x - t * per;   // item
  while (t < count) {
    float x[N][8];
    Place8 e[N];
    T* to[N];
    int64_t at[N];       // the table's row, or kNoTurn
    constexpr int64_t kNoTurn = INT64_MIN;
#pragma unroll
    for (int q = 0; q < N; ++q) {
      to[q] = nullptr;
      at[q] = kNoTurn;
      if (t < count) {
        const uint32_t hh = p.items.of(in_row);
        e[q] = place8(p, in_row - hh * p.items.d);
        const int64_t row = row0 + t, pos = p0 + t;
        const bool is_q = hh < p.H, is_v = hh >= p.H + kv_heads;
        const uint32_t h = is_q ? hh : hh - p.H - (is_v ? kv_heads : 0);
        const T* from;
        if (is_q) {
          from = static_cast<const T*>(p.q) + row * p.q_row;
          to[q] = static_cast<T*>(p.yq) + row * p.y_row + (int64_t)h * p.D;
        } else {
          from = is_v ? static_cast<const T*>(p.v) + row * p.v_row : static_cast<const T*>(p.k) + row * p.k_row;
          const int32_t page = pos >> p.shift == first_pi ? page0 : page1;
          if ((uint32_t)page < p.n_pages)
            to[q] = static_cast<T*>(is_v ? p.v_cache : p.k_cache) + (int64_t)page * p.page_st +
                    (pos & ((1 << p.shift) - 1)) * p.slot_st + (int64_t)h * p.head_st;
        }
        if (!is_v && e[q].turns) at[q] = p.pos ? p.pos[row] : pos;
        load8<T, VEC>(p, from + (int64_t)h * p.D, e[q], x[q]);
        in_row += NT;
        while (in_row >= per) in_row -= per, ++t;
      }
    }
#pragma unroll
    for (int q = 0; q < N; ++q) {
      if (!to[q]) continue;
      if (at[q] != kNoTurn) turn8<VEC>(p, e[q], at[q], x[q]);
      store8<T, VEC>(p, to[q], e[q], x[q]);
    }
  }
}

// One head of K or V in one page of 8 bits.
template <bool VEC, int NT>
__device__ __forceinline__ void append_page(const AppendParams& p, uint32_t idx) {
  __shared__ float red[NT / 64];
  const int lane = threadIdx.x & 63;
  const uint32_t hw = idx % (2 * p.Hkv), w = idx / (2 * p.Hkv), h = hw >> 1;
  const bool is_v = hw & 1;
  const uint32_t size = 1u << p.shift;
  const uint32_t n = __builtin_amdgcn_readfirstlane(piece_owner(p.q_start, p.N, p.T, 1, size, 2, w, lane));
  const int32_t blk = (int32_t)w - first_piece(p.q_start, n, p.T, 1, size, 2);
  const Rows r = new_rows(p.q_start, n, p.T);
  if (blk < 0 || r.n == 0) return;
  const int64_t end = p.kv_len[n], p0 = end - r.n, from = p0 < 0 ? 0 : p0;
  const int64_t pi = (from >> p.shift) + blk, at0 = pi << p.shift;
  if (at0 >= end || pi >= (int64_t)p.max_pages) return;
  const int32_t page = p.table[(uint64_t)n * p.max_pages + (uint64_t)pi];
  if ((uint32_t)page >= p.n_pages) return;
  const uint32_t s0 = from > at0 ? (uint32_t)(from - at0) : 0u;          // slots that stay
  const uint32_t s1 = (uint32_t)min(end - at0, (int64_t)size);
  const int64_t row0 = r.first + (at0 - p0);                             // the row of slot 0
  const bf16* x0 = is_v ? static_cast<const bf16*>(p.v) : static_cast<const bf16*>(p.k);
  const int64_t x_row = is_v ? p.v_row : p.k_row;
  uint8_t* cache = static_cast<uint8_t*>(is_v ? p.v_cache : p.k_cache) + (int64_t)page * p.page_st + (int64_t)h * p.head_st;
  float* scale_at = (is_v ? p.v_scale : p.k_scale) + (uint64_t)page * p.Hkv + h;

  auto token = [&](uint32_t i, uint32_t* slot, Place8* e, float (&x)[8]) {   // item i of the new tokens
    const uint32_t t = p.items.of(i);
    *slot = s0 + t;
    *e = place8(p, i - t * p.items.d);
    const int64_t row = row0 + *slot;
    load8<bf16, VEC>(p, x0 + row * x_row + (int64_t)h * p.D, *e, x);
  };
  auto turn = [&](uint32_t slot, const Place8& e, float (&x)[8]) {
    if (!is_v) turn8<VEC>(p, e, p.pos ? p.pos[row0 + slot] : at0 + slot, x);
  };
  const uint32_t n_items = (s1 - s0) * p.items.d;
  float top = 0.0f;
  auto largest = [&](const float (&x)[8]) {
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const float m = fabsf(x[t]);
      if (m < INFINITY) top = fmaxf(top, m);
    }
  };
  // the thread's first items stay in registers, turned
  constexpr int N = 4;
  float x[N][8];
  Place8 e[N];
  uint32_t slot[N];
#pragma unroll
  for (int q = 0; q < N; ++q)
    if (threadIdx.x + q * NT < n_items) token(threadIdx.x + q * NT, &slot[q], &e[q], x[q]);
  const float was = s0 ? *scale_at : 0.0f;
#pragma unroll
  for (int q = 0; q < N; ++q)
    if (threadIdx.x + q * NT < n_items) {
      turn(slot[q], e[q], x[q]);
      largest(x[q]);
    }
  for (uint32_t i = threadIdx.x + N * NT; i < n_items; i += NT) {
    uint32_t sl;
    Place8 pl;
    float y[8];
    token(i, &sl, &pl, y);
    turn(sl, pl, y);
    largest(y);
  }
#pragma unroll
  for (int off = 32; off; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
  if (lane == 0) red[threadIdx.x >> 6] = top;
  __syncthreads();   // also: the scale is read before it is written
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) top = fmaxf(top, red[i]);
  float scale = pow2(scale_exp(top));
  if (s0) {
    if (was > scale && was < INFINITY) {
      scale = was;
    } else if (was > 0.0f && was < scale) {
      const float by = was / scale;   // what the page holds, rounded again
      for (uint32_t i = threadIdx.x; i < s0 * p.items.d; i += NT) {
        const uint32_t t = p.items.of(i);
        const Place8 e = place8(p, i - t * p.items.d);
        uint8_t* head = cache + (int64_t)t * p.slot_st;
        float x[8];
        if constexpr (VEC) {
          const uint32_t w2[2] = {*reinterpret_cast<const uint32_t*>(head + e.a), *reinterpret_cast<const uint32_t*>(head + e.b)};
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w2[q], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w2[q], true);
            x[4 * q] = lo[0], x[4 * q + 1] = lo[1], x[4 * q + 2] = hi[0], x[4 * q + 3] = hi[1];
          }
        } else {
#pragma unroll
          for (int q = 0; q < 8; ++q)
            x[q] = inside(p, e, q) ? __builtin_amdgcn_cvt_f32_fp8(head[q < 4 ? e.a + q : e.b + q - 4], 0) : 0.0f;
        }
        store8_e4m3<VEC>(p, head, e, x, by);
      }
    }
  }
  if (threadIdx.x == 0) *scale_at = scale;
  const float inv = 1.0f / scale;   // exact
#pragma unroll
  for (int q = 0; q < N; ++q)
    if (threadIdx.x + q * NT < n_items) store8_e4m3<VEC>(p, cache + (int64_t)slot[q] * p.slot_st, e[q], x[q], inv);
  for (uint32_t i = threadIdx.x + N * NT; i < n_items; i += NT) {
    uint32_t sl;
    Place8 pl;
    float y[8];
    token(i, &sl, &pl, y);
    turn(sl, pl, y);
    store8_e4m3<VEC>(p, cache + (int64_t)sl * p.slot_st, pl, y, inv);
  }
}

template <typename T, bool VEC, int NT>
__global__ __launch_bounds__(NT) void append_kernel(AppendParams p) {
  if constexpr (sizeof(T) == 2) {
    if (blockIdx.x < p.page_groups) {
      append_page<VEC, NT>(p, blockIdx.x);
      return;
    }
  }
  append_rows<T, VEC, NT>(p, blockIdx.x - p.page_groups);
}

template <typename T, bool VEC, int NT>
int run(AppendParams& p, hipStream_t s) {
  const int64_t pages = p.e4m3 ? ((int64_t)(p.T >> p.shift) + 2 * (int64_t)p.N) * 2 * p.Hkv : 0;
  const int64_t rows = p.H || !p.e4m3 ? (int64_t)p.T / p.row_tokens + p.N : 0;
  if (!grid_fits(pages + rows, NT)) return DSP_ERR_SHAPE;
  p.page_groups = (uint32_t)pages;
  if (pages + rows) append_kernel<T, VEC, NT><<<dim3((uint32_t)(pages + rows)), NT, 0, s>>>(p);
  return last_launch_status();
}

}  // namespace

int launch_kv_append(const AppendArgs& a, hipStream_t s) {
  AppendParams p = {};
  p.k = a.k, p.v = a.v, p.q = a.q, p.yq = a.yq, p.k_cache = a.k_cache, p.v_cache = a.v_cache;
  p.k_scale = a.k_scale, p.v_scale = a.v_scale, p.table = a.table, p.q_start = a.q_start, p.kv_len = a.kv_len;
  p.pos = a.pos, p.cos = a.cos, p.sin = a.sin;
  p.k_row = a.k_row, p.v_row = a.v_row, p.q_row = a.q_row, p.y_row = a.y_row;
  p.page_st = a.cache_strides[0], p.slot_st = a.cache_strides[1], p.head_st = a.cache_strides[2];
  p.N = (uint32_t)a.N, p.T = (uint32_t)a.T, p.P = (uint32_t)a.P, p.n_pages = (uint32_t)a.n_pages;
  p.max_pages = (uint32_t)a.max_pages, p.shift = a.page_shift;
  p.H = a.H, p.Hkv = a.Hkv, p.D = a.D, p.rot = a.rot;
  p.rot_items = (a.rot + kItem - 1) / kItem;
  p.items = divisor(p.rot_items + (a.D - a.rot + kItem - 1) / kItem);
  p.half = a.half, p.e4m3 = a.e4m3, p.vec = a.vec;
  p.row_tokens = 16;
  while (p.row_tokens > 1 && a.T / p.row_tokens < 4096) p.row_tokens /= 2;
  if (!a.bf16) return a.vec ? run<float, true, 256>(p, s) : run<float, false, 256>(p, s);
  return a.vec ? run<bf16, true, 256>(p, s) : run<bf16, false, 256>(p, s);
}

}  // namespace dsp
