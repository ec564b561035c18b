// Pieces shared by the forward and the gradient of attention with a relative
// position bias (not installed).
#pragma once

#include "attn_tiles.h"

namespace dsp {
namespace {

constexpr float kMasked = -1e30f;   // a bias this low takes its keys out

struct BiasArgs {
  const void* bias;        // [n_buckets][H]
  const int32_t* buckets;  // [2 M + 1]
  int32_t M, nb;
};
__device__ __forceinline__ int32_t bucket_at(const BiasArgs& b, int32_t d) {
  return b.buckets[(d < -b.M ? -b.M : d > b.M ? b.M : d) + b.M];
}
// the bias of bucket k, and of a distance, for head h in the exp2 domain
template <typename T>
__device__ __forceinline__ float bias_of(const BiasArgs& b, uint32_t H, uint32_t h, int32_t k) {
  const float v = (uint32_t)k < (uint32_t)b.nb ? (float)static_cast<const T*>(b.bias)[(int64_t)k * H + h] : 0.0f;
  return v <= kMasked ? -INFINITY : v * kLog2e;
}
template <typename T>
__device__ __forceinline__ float bias_at(const BiasArgs& b, uint32_t H, uint32_t h, int32_t d) {
  return bias_of<T>(b, H, h, bucket_at(b, d));
}
// The table of distances lo .. lo + n - 1 for nh heads from h0, `stride` apart in LDS, by
// NT threads.  Loads return in order: the buckets are asked for before a work-group's
// first keys and the biases after them, so that neither wait is added to the keys'.
template <typename T, int NT>
struct Table {
  static constexpr int N = NT < 128 ? 4 : 2;
  int32_t k[N];
  __device__ __forceinline__ void fetch(const BiasArgs& b, int32_t lo, int32_t n) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int32_t t = (int32_t)threadIdx.x + i * NT;
      k[i] = t < n ? bucket_at(b, lo + t) : -1;
    }
  }
  __device__ __forceinline__ void build(const BiasArgs& b, int32_t lo, int32_t n, float* tab, uint32_t stride,
                                        uint32_t H, uint32_t h0, uint32_t nh) const {
    for (uint32_t h4 = 0; h4 < nh; h4 += 4) {   // four heads' loads at a time
      float v[4][N];
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < N; ++i)
          v[q][i] = h4 + q < nh ? bias_of<T>(b, H, h0 + h4 + q, k[i]) : 0.0f;
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int32_t t = (int32_t)threadIdx.x + i * NT;
          if (t < n && h4 + q < nh) tab[(h4 + q) * stride + t] = v[q][i];
        }
    }
    for (int32_t t = (int32_t)threadIdx.x + N * NT; t < n; t += NT) {
      const int32_t far = bucket_at(b, lo + t);
      for (uint32_t hh = 0; hh < nh; ++hh) tab[hh * stride + t] = bias_of<T>(b, H, h0 + hh, far);
    }
  }
};
// A 32 x 32 block of scores whose keys start d0 positions after its queries holds the
// distances d0 - 31 .. d0 + 31.  Where they all lie at or past one end of the table
// the bias is one value; the other blocks' distances lie within M + kEdge.
constexpr int kEdge = 62;

}  // namespace
}  // namespace dsp
