// Attention of packed new tokens over a cache of pages in bf16, fp32 or e4m3 (the kernels:
// attn_window_fwd.h).
#include "attn_window_fwd.h"

namespace dsp {
namespace {

template <typename T, typename S, int DC>
int run(const WindowArgs& a, hipStream_t s) {
  FwdParams p = params(a);
  return start<T, S, true, DC>(p, a, choose(a), s);
}
template <typename S>
int run_bf16(const WindowArgs& a, hipStream_t s) {
  if (a.D <= 32) return run<bf16, S, 32>(a, s);
  if (a.D <= 48) return run<bf16, S, 48>(a, s);
  if (a.D <= 64) return run<bf16, S, 64>(a, s);
  if (a.D <= 72) return run<bf16, S, 72>(a, s);
  if (a.D <= 80) return run<bf16, S, 80>(a, s);
  if (a.D <= 96) return run<bf16, S, 96>(a, s);
  return run<bf16, S, 128>(a, s);
}

}  // namespace

int launch_attn_paged(const WindowArgs& a, hipStream_t s) {
  if (a.bf16) return a.e4m3 ? run_bf16<uint8_t>(a, s) : run_bf16<bf16>(a, s);
  if (a.D <= 32) return run<float, float, 32>(a, s);
  if (a.D <= 64) return run<float, float, 64>(a, s);
  if (a.D <= 96) return run<float, float, 96>(a, s);
  return run<float, float, 128>(a, s);
}

size_t attn_paged_workspace_bytes(const WindowArgs& a) { return part_bytes(a); }

}  // namespace dsp
