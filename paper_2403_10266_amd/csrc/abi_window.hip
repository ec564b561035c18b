// C ABI of windowed attention and the paged cache: host-side argument validation and
// launches on the caller's stream.  Every entry point validates all of its arguments
// before it enqueues anything.
#include <math.h>

#include "abi_checks.h"
#include "dsp_internal.h"

using namespace dsp;

namespace {

constexpr int64_t kMaxL = int64_t(1) << 30;
constexpr int kMaxGroup = 1 << 15;   // query heads of a key/value head

// Sizes of dsp_attn_window that its workspaces depend on, checked.
int window_sizes(WindowArgs& a, int64_t B, int64_t X, int64_t Lq, int64_t Lk, int H, int Hkv, int D, int left,
                 int right, int sinks, int dtype) {
  if (!valid_dtype(dtype)) return DSP_ERR_DTYPE;
  if (B < 0 || X < 0 || Lq < 0 || Lk < 0 || H < 1 || Hkv < 1 || H % Hkv || H / Hkv >= kMaxGroup || D < 1 || D > kWindowMaxD)
    return DSP_ERR_SHAPE;
  if (dtype == DSP_BF16 && D % 8) return DSP_ERR_SHAPE;
  if (Lq >= kMaxL || Lk >= kMaxL) return DSP_ERR_SHAPE;
  if (sinks < 0) return DSP_ERR_ARG;
  int64_t units, n;
  if (!mul_ok(B, X, &units) || units >= kMaxL || !mul_ok(units, H, &n) || n >= (int64_t(1) << 31) || !mul_ok(n, Lq, &n) ||
      n > (int64_t(1) << 48) || Lq * (H / Hkv) >= (int64_t(1) << 31))
    return DSP_ERR_SHAPE;
  a.B = B, a.X = X, a.Lq = Lq, a.Lk = Lk, a.H = H, a.Hkv = Hkv, a.D = D;
  a.win = {left < 0 ? -1 : left, right < 0 ? -1 : right, sinks};
  a.bf16 = dtype == DSP_BF16;
  return DSP_OK;
}

int window_impl(WindowArgs& a, bool bwd, void* workspace, size_t ws_bytes, const int64_t* q_st, const int64_t* kv_st,
                const int64_t* o_st, float scale, int dtype, void* stream) {
  const int es = elem_size(dtype);
  if (!q_st || !kv_st || !o_st) return DSP_ERR_NULL;
  if (isnan(scale) || isinf(scale)) return DSP_ERR_ARG;
  for (int i = 0; i < 3; ++i)
    if (q_st[i] < 0 || kv_st[i] < 0 || o_st[i] < 0) return DSP_ERR_SHAPE;
  const bool no_units = a.B == 0 || a.X == 0;
  const bool no_q = no_units || a.Lq == 0, no_k = no_units || a.Lk == 0;
  if (bwd ? no_q && no_k : no_q) return DSP_OK;
  const void* q_side[] = {a.q, bwd ? a.dout : a.q, bwd ? a.o : a.q, bwd ? a.dq : a.o};
  const void* k_side[] = {a.k, a.v, bwd ? a.dk : a.k, bwd ? a.dv : a.v};
  for (const void* p : q_side)
    if (!no_q && !p) return DSP_ERR_NULL;
  for (const void* p : k_side)
    if (!no_k && !p) return DSP_ERR_NULL;
  if (bwd && !no_q && !a.lse) return DSP_ERR_NULL;
  if (!aligned(a.q_pos, 4) || !aligned(a.kv_len, 4) || !aligned(a.lse, 4)) return DSP_ERR_ALIGN;
  const int64_t wq = (int64_t)a.H * a.D, wk = (int64_t)a.Hkv * a.D;
  bool vec = a.D % (16 / es) == 0;
  auto side = [&](const void* const (&side)[4], const int64_t* st) {
    for (const void* p : side) {
      if (!aligned(p, es)) return false;
      vec = vec && aligned(p, 16);
    }
    for (int i = 0; i < 3; ++i) vec = vec && st[i] % (16 / es) == 0;
    return true;
  };
  if (!side(q_side, q_st) || !side(k_side, kv_st) || !side(q_side, o_st)) return DSP_ERR_ALIGN;
  if (dtype == DSP_BF16 && !vec) return DSP_ERR_ALIGN;
  if (!no_q && (!spans_ok(a.B, a.X, a.Lq, q_st) || !spans_ok(a.B, a.X, a.Lq, o_st))) return DSP_ERR_SHAPE;
  if (!no_k && !spans_ok(a.B, a.X, a.Lk, kv_st)) return DSP_ERR_SHAPE;
  for (int i = 0; i < 3; ++i) a.q_strides[i] = q_st[i], a.kv_strides[i] = kv_st[i], a.o_strides[i] = o_st[i];
  // the stride of a single row is never used as one; the kernels read whole rows by it
  if (a.Lq <= 1) a.q_strides[2] = a.o_strides[2] = wq;
  if (a.Lk <= 1) a.kv_strides[2] = wk;
  const int64_t far = (int64_t(1) << 31) / 64 / es;   // 64 rows lie within 2^31 bytes
  for (const int64_t* st : {a.q_strides, a.kv_strides, a.o_strides})
    if (st[2] >= far) return DSP_ERR_SHAPE;
  auto disjoint = [&](int64_t L, const int64_t* st, int64_t w) { return rows_disjoint(a.B, a.X, L, st, w); };
  const int64_t Lq = no_q ? 0 : a.Lq, Lk = no_k ? 0 : a.Lk;
  const int64_t *sq = a.q_strides, *sk = a.kv_strides, *so = a.o_strides;
  if (!bwd && !disjoint(a.Lq, so, wq)) return DSP_ERR_ARG;
  if (bwd && ((!no_q && !disjoint(a.Lq, sq, wq)) || (!no_k && !disjoint(a.Lk, sk, wk)))) return DSP_ERR_ARG;
  // every output is apart from every input and from the other outputs
  const Mem q = {a.q, sq, wq, Lq}, k = {a.k, sk, wk, Lk}, v = {a.v, sk, wk, Lk}, o = {a.o, so, wq, Lq};
  const Mem dout = {a.dout, so, wq, Lq}, dq = {a.dq, sq, wq, Lq}, dk = {a.dk, sk, wk, Lk}, dv = {a.dv, sk, wk, Lk};
  const Mem lse = mem_block(a.lse, a.B * a.X * a.H * Lq * 4), none = {};
  const Mem q_pos = mem_block(a.q_pos, a.B * 4), kv_len = mem_block(a.kv_len, a.B * 4);
  const Mem fwd_in[] = {q, k, v, q_pos, kv_len, none, none, none};
  const Mem bwd_in[] = {q, k, v, q_pos, kv_len, o, dout, lse};
  const Mem fwd_out[] = {o, lse, none}, bwd_out[] = {dq, dk, dv};
  const auto& in = bwd ? bwd_in : fwd_in;
  const auto& out = bwd ? bwd_out : fwd_out;
  auto clear = [&](const Mem& m, int others) {
    for (const Mem& i : in)
      if (!apart(m, i, a.B, a.X, es)) return false;
    for (int j = 0; j < others; ++j)
      if (!apart(m, out[j], a.B, a.X, es)) return false;
    return true;
  };
  for (int i = 0; i < 3; ++i)
    if (!clear(out[i], i)) return DSP_ERR_ARG;
  const size_t need = bwd ? attn_window_bwd_workspace_bytes(a) : attn_window_workspace_bytes(a);
  if (need && (!workspace || ws_bytes < need || !aligned(workspace, 16))) return DSP_ERR_WORKSPACE;
  if (need && !clear(mem_block(workspace, (int64_t)need), 3)) return DSP_ERR_ARG;
  a.workspace = static_cast<float*>(workspace);
  a.scale = scale > 0.0f ? scale : (float)(1.0 / sqrt((double)a.D));
  a.vec = vec;
  if (no_q) a.Lq = 0;
  if (no_k) a.Lk = 0;
  return bwd ? launch_attn_window_bwd(a, as_stream(stream)) : launch_attn_window(a, as_stream(stream));
}

// Two tensors of one layout, the second `off` >= 0 elements further, share no row of w
// elements.  Dimensions (extents e, strides s) by decreasing stride, from `at` on; where they
// do not nest the answer is no.
bool shifted_apart(const int64_t* e, const int64_t* s, int at, int64_t w, int64_t off) {
  if (at == 3) return off >= w;
  if (e[at] <= 1) return shifted_apart(e, s, at + 1, w, off);
  int64_t inner = w;
  for (int i = at + 1; i < 3; ++i) inner += (e[i] - 1) * s[i];
  if (off >= (e[at] - 1) * s[at] + inner) return true;
  if (inner > s[at]) return false;
  const int64_t steps = off / s[at], r = off - steps * s[at];
  if (r < inner && !shifted_apart(e, s, at + 1, w, r)) return false;
  if (r + inner > s[at] && steps + 1 < e[at] && !shifted_apart(e, s, at + 1, w, s[at] - r)) return false;
  return true;
}

struct Cache {
  int64_t e[3], st[3];   // pages, slots, heads
  int64_t bytes;         // from the first element to the last
  int es, shift;
};
// Checks the sizes of a paged cache and, where given, its layout.
int cache_layout(Cache& c, int64_t N, int64_t n_pages, int64_t max_pages, int page, int Hkv, int D, const int64_t* st,
                 int cache_dtype, int dtype) {
  if (!valid_dtype(dtype)) return DSP_ERR_DTYPE;
  if (cache_dtype != dtype && !(cache_dtype == DSP_E4M3 && dtype == DSP_BF16)) return DSP_ERR_DTYPE;
  if (N < 0 || n_pages < 0 || max_pages < 0 || N > (int64_t(1) << 20) || n_pages >= kMaxL) return DSP_ERR_SHAPE;
  if (page < 16 || page > 1024 || (page & (page - 1))) return DSP_ERR_SHAPE;
  if (max_pages * page >= kMaxL || max_pages >= kMaxL) return DSP_ERR_SHAPE;
  c.shift = 0;
  while ((1 << c.shift) < page) ++c.shift;
  c.es = cache_dtype == DSP_E4M3 ? 1 : elem_size(dtype);
  if (!st) return DSP_OK;   // sizes alone
  c.e[0] = n_pages, c.e[1] = page, c.e[2] = Hkv;
  for (int i = 0; i < 3; ++i) {
    c.st[i] = st[i];
    if (st[i] < 0 || (c.e[i] > 1 && st[i] == 0)) return DSP_ERR_SHAPE;
  }
  if (!n_pages) return DSP_OK;   // nothing to span: every token is dropped, no key is seen
  if (!spans_ok(n_pages, page, Hkv, st)) return DSP_ERR_SHAPE;
  if (st[1] >= (int64_t(1) << 31) / 64 / c.es) return DSP_ERR_SHAPE;   // 64 slots lie within 2^31 bytes
  if (!rows_disjoint(n_pages, page, Hkv, st, D)) return DSP_ERR_ARG;
  c.bytes = ((n_pages - 1) * st[0] + (page - 1) * st[1] + (Hkv - 1) * st[2] + D) * c.es;
  return DSP_OK;
}
bool caches_apart(const Cache& c, const void* k, const void* v, int D) {
  int64_t off = (intptr_t)v - (intptr_t)k;
  off = off < 0 ? -off : off;
  if (off % c.es) return off >= c.bytes;
  int64_t e[3] = {c.e[0], c.e[1], c.e[2]}, s[3] = {c.st[0], c.st[1], c.st[2]};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (s[j] > s[i]) { std::swap(s[i], s[j]); std::swap(e[i], e[j]); }
  return shifted_apart(e, s, 0, D, off / c.es);
}

int paged_sizes(WindowArgs& a, Cache& c, int64_t N, int64_t T, int64_t max_q, int64_t n_pages, int64_t max_pages, int page,
                int H, int Hkv, int D, const int64_t* st, int left, int right, int sinks, int cache_dtype, int dtype) {
  if (!valid_dtype(dtype)) return DSP_ERR_DTYPE;
  if (H < 1 || Hkv < 1 || H % Hkv || H / Hkv >= kMaxGroup || D < 1 || D > kWindowMaxD || T < 0 || max_q < 0)
    return DSP_ERR_SHAPE;
  if (dtype == DSP_BF16 && D % 8) return DSP_ERR_SHAPE;
  int64_t n;
  if (!mul_ok(T, H, &n) || n >= kMaxL) return DSP_ERR_SHAPE;
  if (int s = cache_layout(c, N, n_pages, max_pages, page, Hkv, D, st, cache_dtype, dtype)) return s;
  if (sinks < 0) return DSP_ERR_ARG;
  a.B = N, a.X = 1, a.T = T, a.Lq = std::min(max_q, T), a.Lk = n_pages ? max_pages * page : 0;
  a.H = H, a.Hkv = Hkv, a.D = D, a.n_pages = n_pages, a.max_pages = max_pages, a.page_shift = c.shift;
  a.win = {left < 0 ? -1 : left, right < 0 ? -1 : right, sinks};
  a.bf16 = dtype == DSP_BF16, a.e4m3 = cache_dtype == DSP_E4M3;
  return DSP_OK;
}

}  // namespace

extern "C" {

size_t dsp_attn_window_workspace_bytes(int64_t B, int64_t X, int64_t Lq, int64_t Lk, int H, int Hkv, int D, int left,
                                       int right, int sinks, int dtype) {
  WindowArgs a = {};
  if (window_sizes(a, B, X, Lq, Lk, H, Hkv, D, left, right, sinks, dtype) != DSP_OK || B == 0 || X == 0 || Lq == 0) return 0;
  return attn_window_workspace_bytes(a);
}

int dsp_attn_window(const void* q, const void* k, const void* v, void* o, float* lse, const int32_t* q_pos,
                    const int32_t* kv_len, int left, int right, int sinks, void* workspace, size_t ws_bytes, int64_t B,
                    int64_t X, int64_t Lq, int64_t Lk, int H, int Hkv, int D, const int64_t* q_strides,
                    const int64_t* kv_strides, const int64_t* o_strides, float scale, int dtype, void* stream) {
  WindowArgs a = {};
  if (int st = window_sizes(a, B, X, Lq, Lk, H, Hkv, D, left, right, sinks, dtype)) return st;
  a.q = q, a.k = k, a.v = v, a.o = o, a.lse = lse, a.q_pos = q_pos, a.kv_len = kv_len;
  return window_impl(a, false, workspace, ws_bytes, q_strides, kv_strides, o_strides, scale, dtype, stream);
}

size_t dsp_attn_window_bwd_workspace_bytes(int64_t B, int64_t X, int64_t Lq, int64_t Lk, int H, int Hkv, int D, int left,
                                           int right, int sinks, int dtype) {
  WindowArgs a = {};
  if (window_sizes(a, B, X, Lq, Lk, H, Hkv, D, left, right, sinks, dtype) != DSP_OK || B == 0 || X == 0) return 0;
  return attn_window_bwd_workspace_bytes(a);
}

int dsp_attn_window_bwd(const void* q, const void* k, const void* v, const void* o, const void* dout, const float* lse,
                        void* dq, void* dk, void* dv, const int32_t* q_pos, const int32_t* kv_len, int left, int right,
                        int sinks, void* workspace, size_t ws_bytes, int64_t B, int64_t X, int64_t Lq, int64_t Lk, int H,
                        int Hkv, int D, const int64_t* q_strides, const int64_t* kv_strides, const int64_t* o_strides,
                        float scale, int dtype, void* stream) {
  WindowArgs a = {};
  if (int st = window_sizes(a, B, X, Lq, Lk, H, Hkv, D, left, right, sinks, dtype)) return st;
  a.q = q, a.k = k, a.v = v, a.o = const_cast<void*>(o), a.dout = dout, a.lse = const_cast<float*>(lse);
  a.dq = dq, a.dk = dk, a.dv = dv, a.q_pos = q_pos, a.kv_len = kv_len;
  return window_impl(a, true, workspace, ws_bytes, q_strides, kv_strides, o_strides, scale, dtype, stream);
}

size_t dsp_attn_paged_workspace_bytes(int64_t N, int64_t T, int64_t max_q, int64_t n_pages, int64_t max_pages, int page,
                                      int H, int Hkv, int D, int left, int right, int sinks, int dtype) {
  WindowArgs a = {};
  Cache c = {};
  if (paged_sizes(a, c, N, T, max_q, n_pages, max_pages, page, H, Hkv, D, nullptr, left, right, sinks, dtype, dtype) != DSP_OK ||
      !a.B || !a.Lq)
    return 0;
  return attn_paged_workspace_bytes(a);
}

int dsp_attn_paged(const void* q, const void* k_cache, const void* v_cache, void* o, float* lse, const float* k_scale,
                   const float* v_scale, const int32_t* table, const int32_t* q_start, const int32_t* kv_len, int left,
                   int right, int sinks, void* workspace, size_t ws_bytes, int64_t N, int64_t T, int64_t max_q,
                   int64_t n_pages, int64_t max_pages, int page, int H, int Hkv, int D, int64_t q_stride,
                   const int64_t* cache_strides, int64_t o_stride, float scale, int cache_dtype, int dtype, void* stream) {
  WindowArgs a = {};
  Cache c = {};
  if (!cache_strides) return DSP_ERR_NULL;
  if (int st = paged_sizes(a, c, N, T, max_q, n_pages, max_pages, page, H, Hkv, D, cache_strides, left, right, sinks,
                           cache_dtype, dtype))
    return st;
  if (isnan(scale) || isinf(scale)) return DSP_ERR_ARG;
  if (q_stride < 0 || o_stride < 0) return DSP_ERR_SHAPE;
  if (!a.B || !a.Lq) return DSP_OK;
  const bool keys = a.Lk > 0;
  if (!q || !o || !q_start || !kv_len || (keys && (!k_cache || !v_cache || !table))) return DSP_ERR_NULL;
  if (keys && a.e4m3 && (!k_scale || !v_scale)) return DSP_ERR_NULL;
  const int es = elem_size(dtype);
  if (!aligned(q, es) || !aligned(o, es) || !aligned(k_cache, c.es) || !aligned(v_cache, c.es) || !aligned(lse, 4) ||
      !aligned(k_scale, 4) || !aligned(v_scale, 4) || !aligned(table, 4) || !aligned(q_start, 4) || !aligned(kv_len, 4))
    return DSP_ERR_ALIGN;
  // rows in chunks of 16 bytes, of 8 in caches of 8 bits
  const int per = 16 / es, chunk = a.e4m3 ? 8 : 16;
  a.vec = D % per == 0 && q_stride % per == 0 && o_stride % per == 0 && aligned(q, 16) && aligned(o, 16) &&
          aligned(k_cache, chunk) && aligned(v_cache, chunk);
  for (int i = 0; i < 3; ++i) a.vec = a.vec && (c.e[i] <= 1 || c.st[i] % per == 0);
  if (a.bf16 && !a.vec) return DSP_ERR_ALIGN;
  const int64_t w = (int64_t)H * D, row_q[3] = {0, 0, T > 1 ? q_stride : w}, row_o[3] = {0, 0, T > 1 ? o_stride : w};
  if (row_q[2] >= (int64_t(1) << 40) || row_o[2] >= (int64_t(1) << 40)) return DSP_ERR_SHAPE;
  if (row_o[2] < w) return DSP_ERR_ARG;
  for (int i = 0; i < 3; ++i) a.q_strides[i] = row_q[i], a.o_strides[i] = row_o[i], a.kv_strides[i] = c.st[i];
  a.q = q, a.k = k_cache, a.v = v_cache, a.o = o, a.lse = lse;
  a.k_scale = a.e4m3 ? k_scale : nullptr, a.v_scale = a.e4m3 ? v_scale : nullptr;
  a.table = table, a.q_start = q_start, a.kv_len = kv_len;
  // the outputs are apart from what is read and from one another
  const int64_t scales = a.e4m3 ? n_pages * Hkv * 4 : 0;
  const Mem in[] = {{q, row_q, w, T}, mem_block(k_cache, c.bytes), mem_block(v_cache, c.bytes), mem_block(k_scale, scales),
                    mem_block(v_scale, scales), mem_block(table, N * max_pages * 4), mem_block(q_start, (N + 1) * 4),
                    mem_block(kv_len, N * 4)};
  const Mem out[] = {{o, row_o, w, T}, mem_block(lse, T * H * 4)};
  auto clear = [&](const Mem& m, int others) {
    for (const Mem& i : in)
      if (!apart(m, i, 1, 1, es)) return false;
    for (int j = 0; j < others; ++j)
      if (!apart(m, out[j], 1, 1, es)) return false;
    return true;
  };
  for (int i = 0; i < 2; ++i)
    if (!clear(out[i], i)) return DSP_ERR_ARG;
  const size_t need = attn_paged_workspace_bytes(a);
  if (need && (!workspace || ws_bytes < need || !aligned(workspace, 16))) return DSP_ERR_WORKSPACE;
  if (need && !clear(mem_block(workspace, (int64_t)need), 2)) return DSP_ERR_ARG;
  a.workspace = static_cast<float*>(workspace);
  a.scale = scale > 0.0f ? scale : (float)(1.0 / sqrt((double)D));
  return launch_attn_paged(a, as_stream(stream));
}

int dsp_kv_append(const void* k, const void* v, const void* q, void* yq, void* k_cache, void* v_cache, float* k_scale,
                  float* v_scale, const int32_t* table, const int32_t* q_start, const int32_t* kv_len, const float* cos,
                  const float* sin, const int32_t* pos, int64_t P, int rot, int flags, int64_t N, int64_t T,
                  int64_t n_pages, int64_t max_pages, int page, int H, int Hkv, int D, int64_t k_stride, int64_t v_stride,
                  int64_t q_stride, int64_t yq_stride, const int64_t* cache_strides, int cache_dtype, int dtype,
                  void* stream) {
  Cache c = {};
  if (!cache_strides) return DSP_ERR_NULL;
  if (!valid_dtype(dtype)) return DSP_ERR_DTYPE;
  if (H < 0 || Hkv < 1 || D < 1 || D > 256 || T < 0 || rot < 0 || rot % 2 || rot > D) return DSP_ERR_SHAPE;
  int64_t n;
  if (!mul_ok(T, (int64_t)H + 2 * (int64_t)Hkv, &n) || n >= kMaxL || (int64_t)H + 2 * (int64_t)Hkv >= 2048) return DSP_ERR_SHAPE;
  if (int st = cache_layout(c, N, n_pages, max_pages, page, Hkv, D, cache_strides, cache_dtype, dtype)) return st;
  if (flags & ~DSP_ROPE_ADJACENT) return DSP_ERR_ARG;
  if (k_stride < 0 || v_stride < 0 || q_stride < 0 || yq_stride < 0) return DSP_ERR_SHAPE;
  if (!N || !T) return DSP_OK;
  if (rot && (P < 1 || P > INT32_MAX)) return DSP_ERR_SHAPE;
  const bool pages = n_pages && max_pages, e4m3 = cache_dtype == DSP_E4M3;
  if (!k || !v || !q_start || !kv_len || (H && (!q || !yq)) || (rot && (!cos || !sin))) return DSP_ERR_NULL;
  if (pages && (!k_cache || !v_cache || !table || (e4m3 && (!k_scale || !v_scale)))) return DSP_ERR_NULL;
  const int es = elem_size(dtype);
  for (const void* p : {k, v, H ? q : nullptr, H ? (const void*)yq : nullptr})
    if (!aligned(p, es)) return DSP_ERR_ALIGN;
  for (const void* p : {(const void*)k_cache, (const void*)v_cache})
    if (!aligned(p, c.es)) return DSP_ERR_ALIGN;
  for (const void* p : {(const void*)k_scale, (const void*)v_scale, (const void*)table, (const void*)q_start,
                        (const void*)kv_len, (const void*)cos, (const void*)sin, (const void*)pos})
    if (!aligned(p, 4)) return DSP_ERR_ALIGN;
  const int64_t wk = (int64_t)Hkv * D, wq = (int64_t)H * D;
  const int64_t sk[3] = {0, 0, T > 1 ? k_stride : wk}, sv[3] = {0, 0, T > 1 ? v_stride : wk};
  const int64_t sq[3] = {0, 0, T > 1 ? q_stride : wq}, sy[3] = {0, 0, T > 1 ? yq_stride : wq};
  for (const int64_t* st : {sk, sv, sq, sy})
    if (st[2] >= (int64_t(1) << 40)) return DSP_ERR_SHAPE;
  if (H && sy[2] < wq) return DSP_ERR_ARG;
  // whole items of eight elements, at most 16 bytes at a time
  auto whole = [](const void* p, int64_t st, int size) { return aligned(p, std::min(8 * size, 16)) && st % 8 == 0; };
  bool vec = D % 8 == 0 && rot % 8 == 0 && (!rot || (aligned(cos, 16) && aligned(sin, 16))) && whole(k, sk[2], es) &&
             whole(v, sv[2], es) && (!H || (whole(q, sq[2], es) && whole(yq, sy[2], es)));
  for (int i = 0; i < 3; ++i) vec = vec && whole(i ? v_cache : k_cache, c.e[i] <= 1 ? 0 : c.st[i], c.es);
  // what is written is apart from what is read and from one another; queries may stay in place
  const int64_t scales = e4m3 ? n_pages * Hkv * 4 : 0, angles = rot ? P * rot / 2 * 4 : 0;
  const Mem in[] = {{q, sq, wq, T}, {k, sk, wk, T}, {v, sv, wk, T}, mem_block(table, N * max_pages * 4),
                    mem_block(q_start, (N + 1) * 4), mem_block(kv_len, N * 4), mem_block(cos, angles),
                    mem_block(sin, angles), mem_block(rot ? pos : nullptr, T * 4)};
  const Mem out[] = {{yq, sy, wq, T}, mem_block(k_cache, c.bytes), mem_block(v_cache, c.bytes),
                     mem_block(e4m3 ? k_scale : nullptr, scales), mem_block(e4m3 ? v_scale : nullptr, scales)};
  for (int i = H ? 0 : 1; i < 5; ++i) {
    for (int j = H ? 0 : 1; j < 9; ++j) {
      const bool own = i == 0 && j == 0 && same_rows(yq, sy, q, sq, 1, 1, T);
      if (!own && !apart(out[i], in[j], 1, 1, es)) return DSP_ERR_ARG;
    }
    for (int j = H ? 0 : 1; j < i; ++j)
      if (!(i == 2 && j == 1) && !apart(out[i], out[j], 1, 1, es)) return DSP_ERR_ARG;
  }
  if (pages && !caches_apart(c, k_cache, v_cache, D)) return DSP_ERR_ARG;
  AppendArgs a = {};
  a.k = k, a.v = v, a.q = q, a.yq = yq, a.k_cache = k_cache, a.v_cache = v_cache, a.k_scale = k_scale, a.v_scale = v_scale;
  a.table = table, a.q_start = q_start, a.kv_len = kv_len, a.pos = rot ? pos : nullptr, a.cos = cos, a.sin = sin;
  a.N = N, a.T = T, a.P = P, a.n_pages = pages ? n_pages : 0, a.max_pages = pages ? max_pages : 0;
  a.k_row = sk[2], a.v_row = sv[2], a.q_row = sq[2], a.y_row = sy[2];
  for (int i = 0; i < 3; ++i) a.cache_strides[i] = c.st[i];
  a.H = H, a.Hkv = Hkv, a.D = D, a.rot = rot, a.page_shift = c.shift;
  a.half = !(flags & DSP_ROPE_ADJACENT), a.bf16 = dtype == DSP_BF16, a.e4m3 = e4m3, a.vec = vec;
  return launch_kv_append(a, as_stream(stream));
}

}  // extern "C"
