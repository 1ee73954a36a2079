// Norms of queries and keys for each head, with the position rotation in the
// same pass: x * rsqrt(mean(x^2) + eps) * w over a head's elements, then each
// pair (a, b) of its first `rot` elements turned by position * freq: a cos - b
// sin, b cos + a sin.  A turn is counted in 2^-64 of a circle, so that position
// times turn wraps to the angle with nothing lost at any position.
#include "attn.hpp"

namespace sn {
namespace k {

// A workgroup takes one token's heads, a wave one head after the other; lane l
// holds the pairs l, l + 64, ... of all of them, so their sines are made once.
constexpr int kHeadWaves = 4;
template <typename T, int NP>
__global__ __launch_bounds__(64 * kHeadWaves) void head_norm_kernel(HeadNormArgs a) {
  const int64_t token = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int D = a.dim, half = a.rot / 2;
  int ia[NP], ib[NP];  // a pair's elements, D: none
  float cs[NP], sn[NP];
  const int64_t pos = a.positions ? a.positions[token] : 0;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int j = lane + 64 * i;
    cs[i] = 1.f, sn[i] = 0.f;
    if (j < half) {
      ia[i] = a.pairs == 0 ? j : 2 * j;
      ib[i] = a.pairs == 0 ? j + half : 2 * j + 1;
      const long long t = (long long)((unsigned long long)pos * a.turn[j]);  // signed: -1/2 .. 1/2 of a circle
      sincospif((float)t * 0x1p-63f, &sn[i], &cs[i]);
    } else {
      ia[i] = min(a.rot + 2 * (j - half), D);
      ib[i] = min(a.rot + 2 * (j - half) + 1, D);
    }
  }
  const int all = a.heads + a.kv_heads;
  for (int h = blockIdx.y * kHeadWaves + wave; h < all; h += gridDim.y * kHeadWaves) {
    const bool key = h >= a.heads;
    const int hh = key ? h - a.heads : h;
    const T* x = (key ? static_cast<const T*>(a.k) + token * a.ks : static_cast<const T*>(a.q) + token * a.qs) + (int64_t)hh * D;
    T* y = (key ? static_cast<T*>(a.ko) + token * a.kos : static_cast<T*>(a.qo) + token * a.qos) + (int64_t)hh * D;
    const float* w = key ? a.k_w : a.q_w;
    float va[NP], vb[NP], s = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      va[i] = ia[i] < D ? to_f(x[ia[i]]) : 0.f;
      vb[i] = ib[i] < D ? to_f(x[ib[i]]) : 0.f;
      s = fmaf(va[i], va[i], fmaf(vb[i], vb[i], s));
    }
    float k = 1.f;
    if (a.norm) k = rsqrtf(wave_sum(s) / (float)D + a.eps);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      va[i] *= w && ia[i] < D ? k * w[ia[i]] : k;
      vb[i] *= w && ib[i] < D ? k * w[ib[i]] : k;
      if (ia[i] < D) y[ia[i]] = from_f<T>(va[i] * cs[i] - vb[i] * sn[i]);
      if (ib[i] < D) y[ib[i]] = from_f<T>(vb[i] * cs[i] + va[i] * sn[i]);
    }
  }
}

template <typename T>
static void launch_head_norm(const HeadNormArgs& a, hipStream_t st) {
  const int all = a.heads + a.kv_heads;
  // few tokens: a token's heads over several workgroups
  const int y = (int)std::min<int64_t>((all + kHeadWaves - 1) / kHeadWaves, std::max<int64_t>(1, 512 / a.tokens));
  const dim3 grid((unsigned)a.tokens, y), block(64 * kHeadWaves);
  if (a.dim <= 128) SN_LAUNCH((head_norm_kernel<T, 1>), grid, block, 0, st, a);
  else SN_LAUNCH((head_norm_kernel<T, 2>), grid, block, 0, st, a);
}

void head_norm(const HeadNormArgs& a, hipStream_t st) {
  check(a.dim >= 1 && a.dim <= 256 && a.rot >= 0 && a.rot <= a.dim && a.rot % 2 == 0 && a.heads + a.kv_heads >= 1 &&
            a.tokens >= 1 && a.tokens < (int64_t(1) << 24) && (a.rot == 0 || a.positions),
        "head norm shapes");
  if (a.dtype == 0) launch_head_norm<float>(a, st);
  else if (a.dtype == 1) launch_head_norm<f16>(a, st);
  else launch_head_norm<bf16>(a, st);
}

}  // namespace k
}  // namespace sn
