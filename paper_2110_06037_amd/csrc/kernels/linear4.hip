// Products with 4-bit weights and group scales.
//
// y[m][k] = act(sum_c x[m][c] s[k][c / g] (q[k][c] - z[k][c / g]) + b[k]): a
// wave per output feature and block of 8 rows of x; lanes take two features
// (one byte of codes) at a time.
#include "seq.hpp"

namespace sn {
namespace k {

template <typename T>
__global__ __launch_bounds__(256) void linear4_kernel(Linear4Args a) {
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= a.rows) return;
  const int64_t m0 = (int64_t)blockIdx.y * 8;
  const int pairs = (a.cols + 1) / 2, groups = (a.cols + a.group - 1) / a.group;
  const T* x = static_cast<const T*>(a.x);
  float acc[8] = {};
  for (int j = lane; j < pairs; j += 64) {
    const int c = 2 * j, g = c / a.group;
    const int64_t at = (int64_t)row * groups + g;
    const unsigned code = a.q[(int64_t)row * pairs + j];
    const float s = (float)a.scale[at];
    const int z = a.zero ? a.zero[at] : 8;
    const float w0 = s * (float)((int)(code & 15) - z), w1 = s * (float)((int)(code >> 4) - z);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (m0 + i < a.m) {
        const T* xp = x + (m0 + i) * a.xs + c;
        acc[i] = fmaf(to_f(xp[0]), w0, acc[i]);
        if (c + 1 < a.cols) acc[i] = fmaf(to_f(xp[1]), w1, acc[i]);
      }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float s = wave_sum(acc[i]);
    if (lane == i && m0 + i < a.m)
      static_cast<T*>(a.y)[(m0 + i) * a.ys + row] = from_f<T>(act_f(s + (a.bias ? a.bias[row] : 0.f), a.act));
  }
}

void linear4(const Linear4Args& a, hipStream_t st) {
  check(a.m >= 1 && a.rows >= 1 && a.cols >= 1 && a.group >= 2 && a.group % 2 == 0 && a.m <= 65535 * 8, "4-bit product shapes");
  const dim3 grid((a.rows + 3) / 4, (unsigned)((a.m + 7) / 8));
  if (a.dtype == 0) SN_LAUNCH((linear4_kernel<float>), grid, dim3(256), 0, st, a);
  else if (a.dtype == 1) SN_LAUNCH((linear4_kernel<f16>), grid, dim3(256), 0, st, a);
  else SN_LAUNCH((linear4_kernel<bf16>), grid, dim3(256), 0, st, a);
}

}  // namespace k
}  // namespace sn
