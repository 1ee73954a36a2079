// Host-callable launchers of the sequence operators' kernels (blocknorm.hip,
// linear4.hip, scan.hip) and the device helpers they share.  A launcher
// enqueues on the given stream; none allocates or synchronises.
#pragma once

#include "gemm_common.hpp"
#include "kcommon.hpp"
#include "launch.hpp"

namespace sn {
namespace k {

// ------------------------------------------------------------------ norms around a block
struct NormArgs {
  int dtype, rdtype;  // rdtype -1: no residual
  int64_t rows;
  int dim, groups, kind, gate;
  float eps, scale;
  const float *post_w, *post_b, *pre_w, *pre_b, *scale_v;
  const void* x;
  int64_t xs;
  const void* g;
  int64_t gs;
  const void* r;
  int64_t rs;
  void* ro;
  int64_t ros;
  void* y;
  int64_t ys;
};
constexpr int kNormMaxDim = 32768;
void block_norm(const NormArgs& a, hipStream_t st);

// ------------------------------------------------------------------ products with 4-bit weights
struct Linear4Args {
  int dtype, act;
  int64_t m;
  int rows, cols, group;
  const uint8_t* q;   // [rows][ceil(cols / 2)]
  const f16* scale;   // [rows][groups]
  const uint8_t* zero;  // [rows][groups] or null
  const float* bias;    // [rows] or null
  const void* x;
  int64_t xs;
  void* y;
  int64_t ys;
};
void linear4(const Linear4Args& a, hipStream_t st);

// ------------------------------------------------------------------ device helpers
constexpr float kLog2e = 1.44269504088896340736f;

// v * sigmoid(v); exp2 overflows to infinity for v < -89, whose reciprocal is the limit 0
__device__ __forceinline__ float silu_f(float v) {
  return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * v));
}

// Whether an address or a byte count is a multiple of 16.
inline bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline bool al16(int64_t b) { return (b & 15) == 0; }

}  // namespace k
}  // namespace sn
