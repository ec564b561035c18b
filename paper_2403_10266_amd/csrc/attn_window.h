// What windowed attention and attention over pages share (not installed): which keys a
// query sees, and loads of keys by groups of 16.
#pragma once

#include <type_traits>

#include "attn_tiles.h"

namespace dsp {
namespace {

// The position of a sequence's first query: any number of 32 bits, to be counted on in 64.
__device__ __forceinline__ int64_t first_position(const int32_t* q_pos, uint32_t b) { return q_pos ? q_pos[b] : 0; }

// A query at position p sees the keys j < sink and lo <= j < hi.  All three grow with p,
// so a block's first and last query bound what its queries see.
struct Seen {
  int32_t lo, hi, sink;
};
__device__ __forceinline__ Seen seen(const Window& w, int64_t p, int32_t len) {
  auto clamp = [len](int64_t v) { return (int32_t)(v < 0 ? 0 : v > len ? len : v); };
  Seen s;
  s.hi = w.right < 0 ? len : clamp(p + w.right + 1);
  s.lo = w.left < 0 ? 0 : clamp(p - w.left);
  s.sink = min(w.sinks, s.hi);
  return s;
}
// 16 keys from key0 that all, or some, of the queries between two see, in full
__device__ __forceinline__ bool whole_group(const Seen& first, const Seen& last, int32_t key0) {
  return key0 + 16 <= last.sink || (key0 >= first.lo && key0 + 16 <= last.hi);
}
// the lowest n bits
__device__ __forceinline__ uint32_t low_bits(int32_t n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }
// bit i: whether key key0 + i is seen
__device__ __forceinline__ uint32_t seen_bits(const Seen& s, int32_t key0) {
  return low_bits(s.sink - key0) | (low_bits(s.hi - key0) & ~low_bits(s.lo - key0));
}
// x where bit k (a constant) of bits is set, else 0, whatever x is: 2 operations
__device__ __forceinline__ float keep_bit(float x, uint32_t bits, int k) {
  return __uint_as_float(__float_as_uint(x) & (uint32_t)((int32_t)(bits << (31 - k)) >> 31));
}
__device__ __forceinline__ bool sees_any(const Seen& s) { return s.sink > 0 || s.lo < s.hi; }

// The keys that the queries between two see, in tiles of KB: `sinks` tiles from key 0,
// then the others from `band` on, a multiple of 16 (keys come in groups of 16).
template <int KB>
struct Tiles {
  int32_t sinks, band, n;
  __device__ __forceinline__ Tiles(const Seen& first, const Seen& last) {
    const int32_t lo = min(first.lo, last.hi) & ~15;
    sinks = (last.sink + KB - 1) / KB;
    band = lo;
    if (lo <= sinks * KB) sinks = band = 0;   // one run from key 0, if there are sinks
    if (last.sink == 0) sinks = 0, band = lo;
    n = sinks + (last.hi > band ? (last.hi - band + KB - 1) / KB : 0);
  }
  __device__ __forceinline__ int32_t key0(int32_t t) const { return t < sinks ? t * KB : band + (t - sinks) * KB; }
};

// x where bit k is set, else -inf: 2 operations
__device__ __forceinline__ float mask_bit(float x, uint32_t bits, int k) {
  const uint32_t t = (uint32_t)((int32_t)(bits << (31 - k)) >> 31);
  return __uint_as_float((__float_as_uint(x) & t) | (~t & 0xFF800000u));
}

// Division by a number below 2^15 that the host knows: exact for n up to 2^16 (and n d below
// 2^32), by one multiplication.
struct Divisor {
  uint32_t d, m;   // m = ceil(2^32 / d); 0 for d = 1
  __device__ __forceinline__ uint32_t of(uint32_t n) const { return m ? __umulhi(n, m) : n; }
};
inline Divisor divisor(uint32_t d) { return {d, d > 1 ? (uint32_t)(((uint64_t(1) << 32) + d - 1) / d) : 0u}; }

// Columns c0 + n (n below 2^15) of a unit as (query, head of the group) pairs.
struct Columns {
  Divisor grp;
  uint32_t i0, r0;   // of c0
  __device__ __forceinline__ Columns(const Divisor& g, uint32_t c0) : grp(g), i0(c0 / g.d), r0(c0 - c0 / g.d * g.d) {}
  __device__ __forceinline__ uint32_t query(uint32_t n) const { return i0 + grp.of(r0 + n); }
  __device__ __forceinline__ uint32_t head(uint32_t n, uint32_t query) const { return r0 + n - (query - i0) * grp.d; }
};

// zero in the columns D .. DP - 1 of `rows` LDS rows that the products take
template <typename T, int DC>
__device__ __forceinline__ void clear_cols(T* lds, int rows, int D, int tid, int nt) {
  using G = Geo<T, DC>;
  if (D >= G::DP) return;
  for (int r = tid; r < rows; r += nt)
    for (int c = (D + G::E - 1) / G::E * G::E; c < G::DP; c += G::E) *reinterpret_cast<u32x4*>(lds + r * G::P + c) = u32x4{0, 0, 0, 0};
}

// 16 keys of one tensor on their way from memory to LDS, by one wave: chunks of E
// elements (16 bytes in LDS), in memory S: T itself, or e4m3 (8 bytes), whose values times
// the page's scale, a power of two, are bf16 values exactly.  Rows that `on` leaves out
// and columns past D come as 0 (the columns are cleared once, by clear_cols).
template <typename T, typename S, int DC>
struct Rows16 {
  using G = Geo<T, DC>;
  static constexpr int E = G::E;
  static constexpr int STEP = 64 / G::CHM < 16 ? 64 / G::CHM : 16;   // rows of a pass, at least
  static constexpr int N = (16 + STEP - 1) / STEP;
  static constexpr uint32_t kNone = 0xFFFFFFF0u;   // an offset past the resource: 0
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  using R = std::conditional_t<sizeof(S) == 1, u32x2, u32x4>;
  R pre[N];

  struct Map {
    uint32_t at[N];           // byte offset of each pass's chunk, kNone for a lane without one
    uint32_t row, step;       // the first one's row, rows of a pass
    int to, col;              // element offset in LDS
  };
  static __device__ __forceinline__ Map map(int D, uint32_t row_bytes, uint32_t lane) {
    Map m;
    const uint32_t ch = (uint32_t)(D + E - 1) / E;
    m.step = min(64u / ch, 16u);
    m.row = lane / ch;
    const uint32_t col = lane - m.row * ch;
    if (m.row >= m.step) m.row = 16;   // a lane without chunks
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t row = m.row + i * m.step;
      m.at[i] = row < 16 ? row * row_bytes + col * (uint32_t)(E * sizeof(S)) : kNone;
    }
    m.col = (int)(col * E);
    m.to = (int)(m.row * G::P) + m.col;
    return m;
  }
  // whole: all 16 rows are taken, and nothing is asked of `on`
  template <typename F>
  __device__ __forceinline__ void fetch(const Map& m, const S* base, int D, bool vec, bool whole, F on) {
    const __amdgpu_buffer_rsrc_t rs = make_rsrc(base, 0x7FFFFFF0u);
    if (whole) {
#pragma unroll
      for (int i = 0; i < N; ++i) load(rs, i, m, m.at[i], D, vec);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) load(rs, i, m, on((int)(m.row + i * m.step)) ? m.at[i] : kNone, D, vec);
    }
  }
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rs, int i, const Map& m, uint32_t off, int D, bool vec) {
    if constexpr (sizeof(S) == 1) {
      pre[i] = __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, 0);
    } else if (sizeof(T) == 2 || vec) {
      pre[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        pre[i][e] = __builtin_amdgcn_raw_buffer_load_b32(rs, m.col + e < D && off != kNone ? off + 4u * e : kNone, 0, 0);
    }
  }
  __device__ __forceinline__ void stash(const Map& m, T* lds, float scale) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (m.row + i * m.step >= 16) continue;
      u32x4 w;
      if constexpr (sizeof(S) == 1) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          w[2 * h] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(pre[i][h], scale, false));
          w[2 * h + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(pre[i][h], scale, true));
        }
      } else {
        w = pre[i];
      }
      *reinterpret_cast<u32x4*>(lds + m.to + i * (int)m.step * G::P) = w;
    }
  }
};

// The keys and values of one sequence and key/value head, by groups of 16: rows of a
// tensor, or slots of pages (a page holds whole groups).  Three steps, so that a loop can
// take the first for later tiles ahead of time: the group's page, its places, the loads.
template <typename S, bool PAGED>
struct Source;
template <typename S>
struct Source<S, false> {
  const S* k;
  const S* v;
  int64_t row;      // elements
  uint32_t row_bytes;
  struct Group {
    const S* k;
    const S* v;
    float ks, vs;
    bool gone;
  };
  __device__ __forceinline__ int32_t page_of(int32_t, int32_t) const { return 0; }
  __device__ __forceinline__ Group group(int32_t key, int32_t) const {
    return {k + (int64_t)key * row, v + (int64_t)key * row, 1.0f, 1.0f, false};
  }
};
template <typename S>
struct Source<S, true> {
  const S* k;       // of the head
  const S* v;
  const int32_t* table;   // of the sequence
  const float* ks;  // of the head
  const float* vs;
  int64_t page, row;
  uint32_t row_bytes, n_pages, n_heads, shift;
  struct Group {
    const S* k;
    const S* v;
    float ks, vs;
    bool gone;      // no such page: its keys are not there
  };
  // keys at or past `end` are not asked for: the table may not reach them
  __device__ __forceinline__ int32_t page_of(int32_t key, int32_t end) const {
    return key < end ? table[(uint32_t)key >> shift] : -1;
  }
  __device__ __forceinline__ Group group(int32_t key, int32_t id) const {
    Group g;
    g.gone = (uint32_t)id >= n_pages;
    const int64_t at = g.gone ? 0 : (int64_t)id * page + (int64_t)((uint32_t)key & ((1u << shift) - 1)) * row;
    g.k = k + at;
    g.v = v + at;
    g.ks = g.vs = 1.0f;
    if constexpr (sizeof(S) == 1) {
      if (!g.gone) {
        g.ks = ks[(int64_t)id * n_heads];
        g.vs = vs[(int64_t)id * n_heads];
      }
    }
    return g;
  }
};

// Packed rows of new tokens: sequence n has rows first .. first + n - 1 of T.
struct Rows {
  int32_t first, n;
};
__device__ __forceinline__ int32_t start_row(const int32_t* q_start, uint32_t n, uint32_t T) {
  const int32_t v = q_start[n];
  return v < 0 ? 0 : v > (int32_t)T ? (int32_t)T : v;
}
__device__ __forceinline__ Rows new_rows(const int32_t* q_start, uint32_t n, uint32_t T) {
  const int32_t a = start_row(q_start, n, T), b = start_row(q_start, n + 1, T);
  return {a, max(b - a, 0)};
}
// Work over packed rows without a list made on the host: sequence n owns the pieces
// f(n) .. f(n + 1) - 1 with f(n) = grp q_start[n] / size + extra n, at least as many as
// its rows fill (size of them to a piece, in whole pieces for extra 1; a piece may also
// be cut at every size-th place of another count for extra 2).  The owner of piece w
// is found by 64 comparisons at a time.
__device__ __forceinline__ int32_t first_piece(const int32_t* q_start, uint32_t n, uint32_t T, uint32_t grp,
                                               uint32_t size, uint32_t extra) {
  return (int32_t)((uint32_t)start_row(q_start, n, T) * grp / size + extra * n);
}
__device__ __forceinline__ uint32_t piece_owner(const int32_t* q_start, uint32_t N, uint32_t T, uint32_t grp,
                                                uint32_t size, uint32_t extra, uint32_t w, int lane) {
  uint32_t lo = 0, count = N;
  while (count > 1) {
    const uint32_t step = (count + 63) / 64, i = lane * step;
    const bool at = i < count && first_piece(q_start, lo + i, T, grp, size, extra) <= (int32_t)w;
    const uint32_t k = (uint32_t)__popcll(__ballot(at)), skip = k ? (k - 1) * step : 0;
    lo += skip;
    count = min(step, count - skip);
  }
  return lo;
}

// The order of blocks of `rows` rows whose other side is a window of `span` rows more, where
// an XCD's L2 (4 MB) holds what the heads of such a block read; else that of whole sequences.
inline Order window_order(const WindowArgs& a, int64_t blocks, int64_t rows) {
  const int64_t es = a.bf16 ? 2 : 4;
  const int64_t span = a.win.left < 0 || a.win.right < 0 ? INT64_MAX / 4096 : (int64_t)a.win.left + a.win.right + 1;
  const int64_t bytes = (span + rows) * 2 * std::max(a.H, a.Hkv) * a.D * es;
  if (blocks > 2 && span < INT64_MAX / 4096 && bytes <= (int64_t(5) << 19)) return make_run_order(a.B * a.X, a.Hkv, blocks);
  return make_order(a.B * a.X, a.Hkv, 1, blocks, a.win.right >= 0 && a.win.left < 0);
}

}  // namespace
}  // namespace dsp
