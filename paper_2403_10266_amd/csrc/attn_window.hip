// Attention with a window and first tokens that stay visible, over rows of tensors of any
// layout (the kernels: attn_window_fwd.h).
#include "attn_window_fwd.h"

namespace dsp {
namespace {

template <typename T, int DC>
int run(const WindowArgs& a, hipStream_t s) {
  FwdParams p = params(a);
  const int64_t cols = a.Lq * p.grp.d;
  constexpr bool B16 = sizeof(T) == 2;
  if (cols <= 32 && a.Lk <= 32) return start_short<T, DC, 1, 32, B16 ? (DC <= 80 ? 4 : 3) : 1>(p, a, s);
  if (cols <= 64 && a.Lk <= 64) return start_short<T, DC, 2, 64, B16 ? 3 : 1>(p, a, s);
  if (cols <= 128 && a.Lk <= 128) return start_short<T, DC, 4, 128, B16 ? (DC <= 96 ? 3 : 2) : 1>(p, a, s);
  return start<T, T, false, DC>(p, a, choose(a), s);
}

}  // namespace

int launch_attn_window(const WindowArgs& a, hipStream_t s) {
  if (a.bf16) {
    if (a.D <= 32) return run<bf16, 32>(a, s);
    if (a.D <= 48) return run<bf16, 48>(a, s);
    if (a.D <= 64) return run<bf16, 64>(a, s);
    if (a.D <= 72) return run<bf16, 72>(a, s);
    if (a.D <= 80) return run<bf16, 80>(a, s);
    if (a.D <= 96) return run<bf16, 96>(a, s);
    return run<bf16, 128>(a, s);
  }
  if (a.D <= 32) return run<float, 32>(a, s);
  if (a.D <= 64) return run<float, 64>(a, s);
  if (a.D <= 96) return run<float, 96>(a, s);
  return run<float, 128>(a, s);
}

size_t attn_window_workspace_bytes(const WindowArgs& a) { return part_bytes(a); }

}  // namespace dsp
