// Tiles of the attention kernels that take masks and lengths (not installed): matrix
// fragments, loads, stores and the order of work, for bf16 and fp32.
//
// Both types run on 32 x 32 matrix instructions whose accumulator gives lane
// (n + 32 g) column n, rows 8 (r / 4) + 4 g + r % 4 for its registers r = 0 .. 15:
// bf16 on 32x32x16, fp32 on 32x32x2.  Tensors sit row-major in LDS.
//  * Row products (scores): A and B fragments are 16 bytes of a row, lane (n + 32 g)
//    holding row n, bytes 32 s + 16 g .. + 15 of step s.  A contraction may take its
//    terms in any order that both sides share, so in fp32 the four elements of a
//    fragment are four instructions.
//  * Column products (P V and the gradients'): the A operand is the tensor's
//    transpose, the B operand the accumulator of a row product as it stands (rounded
//    to bf16 for bf16), again in the row order that both sides share.
#pragma once

#include <math.h>

#include <algorithm>

#include "attn_bf16_common.h"
#include "dsp_internal.h"

namespace dsp {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <typename T>
struct Mx;
template <>
struct Mx<bf16> {
  static constexpr int E = 8;       // elements of 16 bytes
  typedef bf16x8 frag;
  static __device__ __forceinline__ floatx16 mma(frag a, frag b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mx<float> {
  static constexpr int E = 4;
  typedef floatx4 frag;
  static __device__ __forceinline__ floatx16 mma(frag a, frag b, floatx16 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
  }
};

// Head widths are rounded up to a class DC; columns D .. are zero in LDS.
template <typename T, int DC>
struct Geo {
  static constexpr int E = Mx<T>::E;
  static constexpr int DP = (DC + 15) / 16 * 16;       // columns the products take
  static constexpr int NS = DP / (2 * E);              // steps of a row product
  static constexpr bool SLAB = DP % 32 != 0;           // bf16: last 16 columns on 16x16x32
  static constexpr int NT = DP / 32;                   // 32-column tiles of a column product
  static constexpr int P = DP + E;                     // LDS row pitch: an odd number of 16 bytes
  static constexpr int CHM = DC / E;                   // 16-byte chunks of a row, at most
  static_assert(DC % 8 == 0 && (!SLAB || E == 8), "class");
};

// Between LDS accesses of different lanes of one wave to the same words: the hardware
// keeps their order; the compiler does where it cannot tell a lane's addresses apart,
// and has to be told to where it can.
__device__ __forceinline__ void wave_order() { asm volatile("" ::: "memory"); }

// A B operand of a column product made of a 32 x 32 accumulator
template <typename T>
struct ColB;
template <>
struct ColB<bf16> {
  bf16x8 v[2];
  __device__ __forceinline__ void set(int r, float x) { v[r / 8][r % 8] = (bf16)x; }
};
template <>
struct ColB<float> {
  floatx16 v;
  __device__ __forceinline__ void set(int r, float x) { v[r] = x; }
};

// acc[col][n] += sum over the 32 rows of t from row0 of t[row][col0 + col] b[row][n]
__device__ __forceinline__ floatx16 col_mma(const bf16* t, int pitch, int row0, int col0, int lane,
                                            const ColB<bf16>& b, floatx16 acc) {
  const int j16 = lane & 15, g = lane >> 5, mbase = 16 * ((lane >> 4) & 1);
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    const int row = row0 + 16 * kk + 4 * g + (j16 >> 2);
    const int col = col0 + mbase + 4 * (j16 & 3);
    const shortx4 lo = lds_read_tr(t + row * pitch + col);
    const shortx4 hi = lds_read_tr(t + (row + 8) * pitch + col);
    const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b.v[kk], acc, 0, 0, 0);
  }
  return acc;
}
__device__ __forceinline__ floatx16 col_mma(const float* t, int pitch, int row0, int col0, int lane,
                                            const ColB<float>& b, floatx16 acc) {
  const int l32 = lane & 31, g = lane >> 5;
#pragma unroll
  for (int r = 0; r < 16; ++r)
    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(t[(row0 + 8 * (r / 4) + 4 * g + r % 4) * pitch + col0 + l32], b.v[r],
                                               acc, 0, 0, 0);
  return acc;
}

// The last 16 columns (col0 ..) on 16x16x32: accumulator h holds columns col0 +
// 4 (lane / 16) + r of n = 16 h + lane % 16.  One permlane16 swap of the two 16-row
// halves of b gives the B operands, whose row order the A operand shares.
__device__ __forceinline__ void slab_mma(const bf16* t, int pitch, int row0, int col0, int lane,
                                         const ColB<bf16>& b, floatx4 (&acc)[2]) {
  const int j16 = lane & 15, c = lane >> 4;
  const int row = row0 + ((c & 1) ? 16 : 0) + ((c & 2) ? 4 : 0) + (j16 >> 2);
  const int col = col0 + 4 * (j16 & 3);
  const shortx4 lo = lds_read_tr(t + row * pitch + col);
  const shortx4 hi = lds_read_tr(t + (row + 8) * pitch + col);
  const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  const u32x4 x = __builtin_bit_cast(u32x4, b.v[0]), y = __builtin_bit_cast(u32x4, b.v[1]);
  u32x4 b0, b1;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const auto r = __builtin_amdgcn_permlane16_swap(x[w], y[w], false, false);
    b0[w] = r[0];
    b1[w] = r[1];
  }
  acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, b0), acc[0], 0, 0, 0);
  acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, __builtin_bit_cast(bf16x8, b1), acc[1], 0, 0, 0);
}

// The A operands of a column product over 32 rows of t from row0, read ahead of it.
template <typename T, int DC>
struct ColA;
template <int DC>
struct ColA<bf16, DC> {
  using G = Geo<bf16, DC>;
  bf16x8 t[G::NT > 0 ? G::NT : 1][2], s;
  static __device__ __forceinline__ bf16x8 read(const bf16* at) {
    const shortx4 lo = lds_read_tr(at), hi = lds_read_tr(at + 8 * G::P);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  __device__ __forceinline__ void load(const bf16* lds, int row0, int lane) {
    const int j16 = lane & 15, g = lane >> 5, c = lane >> 4;
    const bf16* at = lds + (row0 + 4 * g + (j16 >> 2)) * G::P + 16 * (c & 1) + 4 * (j16 & 3);
#pragma unroll
    for (int i = 0; i < G::NT; ++i)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) t[i][kk] = read(at + 16 * kk * G::P + 32 * i);
    if constexpr (G::SLAB)
      s = read(lds + (row0 + ((c & 1) ? 16 : 0) + ((c & 2) ? 4 : 0) + (j16 >> 2)) * G::P + 32 * G::NT + 4 * (j16 & 3));
  }
};
template <int DC>
struct ColA<float, DC> {   // fp32 reads them as it goes
  const float* lds;
  int row0, lane;
  __device__ __forceinline__ void load(const float* l, int r, int n) { lds = l, row0 = r, lane = n; }
};
// the slab's B operands (as in slab_mma)
__device__ __forceinline__ void slab_b(const ColB<bf16>& b, bf16x8 (&out)[2]) {
  const u32x4 x = __builtin_bit_cast(u32x4, b.v[0]), y = __builtin_bit_cast(u32x4, b.v[1]);
  u32x4 b0, b1;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const auto r = __builtin_amdgcn_permlane16_swap(x[w], y[w], false, false);
    b0[w] = r[0];
    b1[w] = r[1];
  }
  out[0] = __builtin_bit_cast(bf16x8, b0);
  out[1] = __builtin_bit_cast(bf16x8, b1);
}

// The accumulators of a column product for one 32-row block: its tiles and slab.
template <typename T, int DC>
struct ColAcc {
  using G = Geo<T, DC>;
  floatx16 t[G::NT > 0 ? G::NT : 1];
  floatx4 s[2];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < G::NT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) t[i][r] = 0.0f;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[h][r] = 0.0f;
  }
  __device__ __forceinline__ void add(const T* lds, int row0, int lane, const ColB<T>& b) {
#pragma unroll
    for (int i = 0; i < G::NT; ++i) t[i] = col_mma(lds, G::P, row0, 32 * i, lane, b, t[i]);
    if constexpr (G::SLAB) slab_mma(lds, G::P, row0, 32 * G::NT, lane, b, s);
  }
  __device__ __forceinline__ void add(const ColA<T, DC>& a, const ColB<T>& b) {
    if constexpr (sizeof(T) == 4) {
      add(a.lds, a.row0, a.lane, b);
    } else {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int i = 0; i < G::NT; ++i) t[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.t[i][kk], b.v[kk], t[i], 0, 0, 0);
      if constexpr (G::SLAB) {
        bf16x8 half[2];
        slab_b(b, half);
#pragma unroll
        for (int h = 0; h < 2; ++h) s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.s, half[h], s[h], 0, 0, 0);
      }
    }
  }
  // plus f times b, f what each lane holds for its own column n = lane % 32
  __device__ __forceinline__ void add(float f, const ColAcc& b, int lane) {
#pragma unroll
    for (int i = 0; i < G::NT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) t[i][r] = fmaf(f, b.t[i][r], t[i][r]);
    if constexpr (G::SLAB) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float fh = __shfl(f, 16 * h + (lane & 15));
#pragma unroll
        for (int r = 0; r < 4; ++r) s[h][r] = fmaf(fh, b.s[h][r], s[h][r]);
      }
    }
  }
  // times a factor that each lane holds for its own column n = lane % 32
  __device__ __forceinline__ void scale(float f, int lane) {
#pragma unroll
    for (int i = 0; i < G::NT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) t[i][r] *= f;
    if constexpr (G::SLAB) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float fh = __shfl(f, 16 * h + (lane & 15));
#pragma unroll
        for (int r = 0; r < 4; ++r) s[h][r] *= fh;
      }
    }
  }
};

// Stores four consecutive elements of a row from column d0, those below D.
__device__ __forceinline__ void store4(bf16* row, int d0, int D, bool, float a, float b, float c, float d) {
  if (d0 >= D) return;   // D is a multiple of 8
  const bf16x2 lo = {(bf16)a, (bf16)b}, hi = {(bf16)c, (bf16)d};
  uint2 w;
  w.x = __builtin_bit_cast(uint32_t, lo);
  w.y = __builtin_bit_cast(uint32_t, hi);
  *reinterpret_cast<uint2*>(row + d0) = w;
}
__device__ __forceinline__ void store4(float* row, int d0, int D, bool vec, float a, float b, float c, float d) {
  if (vec) {
    if (d0 < D) *reinterpret_cast<floatx4*>(row + d0) = floatx4{a, b, c, d};
    return;
  }
  if (d0 < D) row[d0] = a;
  if (d0 + 1 < D) row[d0 + 1] = b;
  if (d0 + 2 < D) row[d0 + 2] = c;
  if (d0 + 3 < D) row[d0 + 3] = d;
}

// Writes the rows of a ColAcc: `row_of(n)` gives column n's row, or null.
template <typename T, int DC, typename F>
__device__ __forceinline__ void store_rows(const ColAcc<T, DC>& a, int lane, int D, bool vec, F row_of) {
  using G = Geo<T, DC>;
  const int g = lane >> 5;
  auto* row = row_of(lane & 31);
  if (row) {
#pragma unroll
    for (int i = 0; i < G::NT; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        store4(row, 32 * i + 8 * q + 4 * g, D, vec, a.t[i][4 * q], a.t[i][4 * q + 1], a.t[i][4 * q + 2],
               a.t[i][4 * q + 3]);
  }
  if constexpr (G::SLAB) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      auto* rs = row_of(16 * h + (lane & 15));
      if (rs) store4(rs, 32 * G::NT + 4 * (lane >> 4), D, vec, a.s[h][0], a.s[h][1], a.s[h][2], a.s[h][3]);
    }
  }
}

// The same through LDS: `so` holds 32 rows of pitch P for this wave alone, and the rows
// leave as whole 16-byte chunks, consecutive lanes along a row (from the accumulators
// a store would write 8 or 16 bytes of 32 rows each).  cols: the columns written there,
// all (DP) where the rows are done with, D where a later tile takes them: past D lies its
// padding, cleared once, and a sum there is not 0 but NaN where an operand was not finite.
template <typename T, int DC, typename F>
__device__ __forceinline__ void store_rows_lds(T* so, const ColAcc<T, DC>& a, int lane, int D, int cols, F row_of) {
  using G = Geo<T, DC>;
  store_rows<T, DC>(a, lane, cols, true, [&](int n) { return so + n * G::P; });
  const int ch = D / G::E;   // whole chunks: the callers' rows are aligned
  int row = lane / ch, col = lane - row * ch;
  const int dr = 64 / ch, dc = 64 - dr * ch;
  for (int c = lane; c < 32 * ch; c += 64) {
    T* to = row_of(row);
    if (to) *reinterpret_cast<u32x4*>(to + col * G::E) = *reinterpret_cast<const u32x4*>(so + row * G::P + col * G::E);
    row += dr, col += dc;
    if (col >= ch) col -= ch, ++row;
  }
}

// The fragments of one row in registers, columns D .. as 0; row null: all 0.
template <typename T, int DC>
__device__ __forceinline__ void row_frags(const T* row, int g, int D, bool vec,
                                          typename Mx<T>::frag (&f)[Geo<T, DC>::NS]) {
  constexpr int E = Mx<T>::E;
#pragma unroll
  for (int s = 0; s < Geo<T, DC>::NS; ++s) {
    const int d = 2 * E * s + E * g;
#pragma unroll
    for (int e = 0; e < E; ++e) f[s][e] = (T)0.0f;
    if (!row) continue;
    if (vec) {
      if (d < D) f[s] = *reinterpret_cast<const typename Mx<T>::frag*>(row + d);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (d + e < D) f[s][e] = row[d + e];
    }
  }
}

// A tile of up to R rows of one tensor on its way from memory to LDS: NT threads (tid),
// 16-byte chunks, rows past `rows` and columns past D as 0 (the columns are cleared
// once, by clear_pad).  A thread keeps to one column of chunks and takes every n-th
// row, so its places are one offset and a scalar step.  vec: whole chunks at 16-byte
// offsets; otherwise (fp32) an element at a time.
template <typename T, int DC, int R, int NT>
struct Tile {
  using G = Geo<T, DC>;
  static constexpr int STEP = NT / G::CHM;               // rows of a pass, at least
  static constexpr int N = (R + STEP - 1) / STEP;
  u32x4 pre[N];

  // where this thread's chunks lie: byte offset in the tensor's rows, element offset in LDS
  struct Map {
    uint32_t at, row, step;   // step: rows of a pass
    int to, col;
  };
  static __device__ __forceinline__ Map map(int D, uint32_t row_bytes, uint32_t tid) {
    Map m;
    const uint32_t ch = (uint32_t)(D + G::E - 1) / G::E;
    m.step = min(NT / ch, (uint32_t)R);
    m.row = tid / ch;
    const uint32_t col = tid - m.row * ch;
    if (m.row >= m.step) m.row = R;   // a thread without chunks
    m.at = m.row * row_bytes + col * 16u;
    m.col = (int)(col * G::E);
    m.to = (int)(m.row * G::P) + m.col;
    return m;
  }
  __device__ __forceinline__ void fetch(const Map& m, const T* base, uint32_t rows, uint32_t row_bytes, int D,
                                        bool vec) {
    // an offset past the resource instead of a branch: all loads go out at once.  The
    // resource ends with the last row's last element, whatever the stride (0 included).
    const __amdgpu_buffer_rsrc_t rs = make_rsrc(base, rows ? (rows - 1) * row_bytes + (uint32_t)(D * sizeof(T)) : 0u);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t off = m.row + i * m.step < rows ? m.at + i * m.step * row_bytes : 0xFFFFFFF0u;
      if (sizeof(T) == 2 || vec) {
        pre[i] = __builtin_amdgcn_raw_buffer_load_b128(rs, off, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          pre[i][e] = __builtin_amdgcn_raw_buffer_load_b32(rs, m.col + e < D ? off + 4u * e : 0xFFFFFFF0u, 0, 0);
      }
    }
  }
  __device__ __forceinline__ void stash(const Map& m, T* lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (m.row + i * m.step < R) *reinterpret_cast<u32x4*>(lds + m.to + i * (int)m.step * G::P) = pre[i];
  }
};
// zero in columns D .. P - 1 of `rows` LDS rows (fp32: past the chunk that holds D - 1)
template <typename T, int DC>
__device__ __forceinline__ void clear_pad(T* lds, int rows, int D, int tid, int nt) {
  using G = Geo<T, DC>;
  const int d0 = (D + G::E - 1) / G::E * G::E, w = G::P - d0;
  for (int e = tid; e < rows * w; e += nt) lds[e / w * G::P + d0 + e % w] = (T)0.0f;
}

// Which work-group does what.  Work-group i runs on XCD i % 8, each with an L2 of its
// own.  Work comes in chunks that share cached rows: the heads of one key/value head's
// group, or of a whole token row where a unit has few blocks (heads lie side by side in
// a row's cache lines).  Chunk c goes to XCD c % 8, so that sequences of different
// lengths spread over all of them.  A chunk's blocks follow each other; where the
// blocks differ in cost (causal masks) every chunk's most costly ones come first.
// Whole token rows against single heads: 1350 x 16 units of 49 x 72 158 and 181 us,
// 400 x 16 of 100 145 and 156, 64 x 16 of 300 the same.
struct Order {
  uint32_t n_chunks, per_xcd;   // chunks in all, and (rounded up) of an XCD
  uint32_t heads, blocks;       // of a chunk: heads, blocks of each head
  uint32_t chunks_bx;           // chunks of one (b, x)
  bool costly_first;
  uint32_t run;                 // 0, or the other order below: n_chunks blocks, per_xcd runs of `run`
};
inline Order make_order(int64_t bx, int64_t groups, int64_t grp, int64_t blocks, bool costly_first) {
  const int64_t rows = blocks <= 2 && bx >= 64 ? groups : 1;   // key/value heads of a chunk
  Order o;
  o.chunks_bx = (uint32_t)(groups / rows);
  o.n_chunks = (uint32_t)(bx * o.chunks_bx);
  o.per_xcd = (o.n_chunks + 7) / 8;
  o.heads = (uint32_t)(rows * grp);
  o.blocks = (uint32_t)blocks;
  o.costly_first = costly_first;
  o.run = 0;
  return o;
}
// Blocks that see a window only: neighbouring blocks share rows, and the heads of a token
// share cache lines, so an XCD takes runs of neighbouring blocks, each with all its heads
// side by side; runs go to the XCDs in turn.
inline Order make_run_order(int64_t bx, int64_t heads, int64_t blocks) {
  Order o = {};
  o.n_chunks = (uint32_t)(bx * blocks);
  o.run = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(8, bx * blocks / 8));
  o.per_xcd = ((o.n_chunks + o.run - 1) / o.run + 7) / 8;
  o.heads = (uint32_t)heads;
  o.blocks = (uint32_t)blocks;
  o.chunks_bx = 1;
  return o;
}
inline int64_t order_blocks(const Order& o) {
  return (int64_t)8 * o.per_xcd * o.heads * (o.run ? o.run : o.blocks);
}
struct Place {
  uint32_t bx, h, block;   // block 0 is the most costly
  bool any;                // the grid is rounded up: nothing to do
};
__device__ __forceinline__ Place place(const Order& o, uint32_t i = blockIdx.x) {
  const uint32_t xcd = i & 7u, j = i >> 3;
  Place p;
  uint32_t local, head;
  if (o.run) {
    local = j / o.heads;
    const uint32_t k = local / o.run, block = (k * 8 + xcd) * o.run + local - k * o.run;
    p.h = j - local * o.heads;
    p.any = block < o.n_chunks;
    p.bx = block / o.blocks;
    p.block = block - p.bx * o.blocks;
    return p;
  }
  if (o.costly_first) {
    const uint32_t n = o.per_xcd * o.heads, r = j % n;
    p.block = j / n;
    local = r / o.heads;
    head = r - local * o.heads;
  } else {
    const uint32_t n = o.heads * o.blocks, r = j % n;
    local = j / n;
    head = r / o.blocks;
    p.block = r - head * o.blocks;
  }
  const uint32_t chunk = local * 8 + xcd;
  p.any = chunk < o.n_chunks;
  p.bx = chunk / o.chunks_bx;
  p.h = (chunk - p.bx * o.chunks_bx) * o.heads + head;
  return p;
}

// q_pos and kv_len come from the device: kept where differences cannot overflow
__device__ __forceinline__ int32_t position(const int32_t* q_pos, uint32_t b) {
  if (!q_pos) return 0;
  const int32_t v = q_pos[b];
  return v < -(1 << 30) ? -(1 << 30) : v > (1 << 30) ? (1 << 30) : v;
}
__device__ __forceinline__ uint32_t length(const int32_t* kv_len, uint32_t b, uint32_t Lk) {
  if (!kv_len) return Lk;
  const int32_t v = kv_len[b];
  return v < 0 ? 0u : (uint32_t)v < Lk ? (uint32_t)v : Lk;
}

}  // namespace
}  // namespace dsp
