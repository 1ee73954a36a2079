// Norms before and after a block with its gate, scale and residual, one pass
// over the rows: t = norm(x * silu(g)) (or norm(x) * silu(g)), r' = r +
// scale * t, y = norm(r').  Every step is elementwise but the statistics, so
// a row is read once, held in registers in float32 through both norms, and
// written once; the layer norm's variance is summed from the centred
// registers.  Bound by memory, the bytes of x, g, r, r' and y: 8192 rows of
// 2048 in bf16 with a float32 residual, tensors beyond the caches, 42 us, 4.8
// TB/s, what a copy of gigabytes reaches; 4096 rows of 4096 gated in 8 groups
// 20.6 us, 4.9 TB/s.  Below some hundred rows the launch and two trips to memory
// and back (the row; behind its sums, the weights) remain: one row of 2048 2.5
// us.  (Weights read with the row instead: no difference at any of these.)
#include "seq.hpp"

namespace sn {
namespace k {

// How a thread reaches its chunks of 8 consecutive elements: whole and aligned
// to 16 bytes; at any element, a row's last one cut short; rows of fewer than 8
// elements, one by one.  (777 rows of 1023 in f16 with gate and residual: 5.9
// us against 7.4 with every element loaded by itself, 5000 rows without: 9.4
// against 14.4.)
enum { kAligned, kAnywhere, kSingle };

// 8 elements from any address (one or two loads: global memory takes them
// unaligned).
template <typename E>
__device__ __forceinline__ V8<E> ld8_any(const E* p) {
  V8<E> r;
  __builtin_memcpy(&r, p, sizeof(r));
  return r;
}
template <typename E>
__device__ __forceinline__ void st8_any(E* p, const V8<E>& r) {
  __builtin_memcpy(p, &r, sizeof(r));
}
// The chunk at c of a row (or vector) q of D elements, 0 past its end.  No load
// is behind a branch (its join would wait for it): a cut chunk is read as the
// row's last 8 elements and moved down.
template <int MODE, typename E>
__device__ __forceinline__ void chunk_get(const E* q, int c, int D, bool on, float (&v)[8]) {
  if constexpr (MODE == kAligned) {
    const V8<E> u = on && c < D ? ld8(q + c) : zero8<E>();
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = to_f(u.v[j]);
  } else if constexpr (MODE == kSingle) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = on && c + j < D ? to_f(q[c + j]) : 0.f;
  } else {
    const int cut = on ? min(max(c + 8 - D, 0), 8) : 8;
    const V8<E> u = ld8_any(q + min(c, D - 8));
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = to_f(u.v[j]);
#pragma unroll
    for (int s = 8; s > 0; s /= 2)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = cut & s ? j + s < 8 ? v[j + s] : 0.f : v[j];
  }
}
template <int MODE, typename E>
__device__ __forceinline__ void chunk_put(E* q, int c, int D, const float (&v)[8]) {
  V8<E> u;
#pragma unroll
  for (int j = 0; j < 8; ++j) u.v[j] = from_f<E>(v[j]);
  if constexpr (MODE == kAligned) {
    if (c < D) st8(q + c, u);
  } else {
    if (MODE == kAnywhere && c + 8 <= D) return st8_any(q + c, u);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c + j < D) q[c + j] = u.v[j];
  }
}

// WPR: waves per row; NV: chunks per thread.  A row of D elements fits when
// D <= 512 WPR NV.  As few waves as hold the row in one or two chunks: two for up
// to 1024 elements (5000 rows: 7.8 us against 9.7 with four, half of them idle);
// rows beyond 4096 take 16 waves rather than more registers.
template <typename T, typename R, int MODE, int WPR, int NV>
__global__ __launch_bounds__(WPR < 4 ? 256 : 64 * WPR) void block_norm_kernel(NormArgs a) {
  constexpr int TPR = 64 * WPR;
  constexpr int ROWS = WPR < 4 ? 4 / WPR : 1;
  __shared__ float red[4][ROWS][WPR];
  const int t = threadIdx.x % TPR;
  const int slot = threadIdx.x / TPR;
  const int D = a.dim / a.groups;
  const int64_t units = a.rows * a.groups;
  const int64_t unit = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * ROWS + slot;
  const bool on = unit < units;  // threads without a row take part in the barriers
  const int64_t row = on ? unit / a.groups : 0;
  const int col = on ? (int)(unit - row * a.groups) * D : 0;

  auto at = [&](int i) { return (i * TPR + t) * 8; };
  auto load = [&](auto* p, int64_t stride, float (&v)[NV][8]) {
    const auto* q = p + row * stride + col;
#pragma unroll
    for (int i = 0; i < NV; ++i) chunk_get<MODE>(q, at(i), D, on, v[i]);
  };
  auto store = [&](auto* p, int64_t stride, const float (&v)[NV][8]) {
    auto* q = p + row * stride + col;
    if (!on) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) chunk_put<MODE>(q, at(i), D, v[i]);
  };
  int phase = 0;
  auto total = [&](float s) {
    s = wave_sum(s);
    if constexpr (WPR > 1) {
      float* m = red[phase++][slot];
      if ((t & 63) == 0) m[t >> 6] = s;
      __syncthreads();
      s = 0.f;
#pragma unroll
      for (int w = 0; w < WPR; ++w) s += m[w];
    }
    return s;
  };
  // per-channel vectors, read where they are used (cached: all rows share them)
  auto vec = [&](const float* w, int c0, int i, float (&o)[8]) { chunk_get<MODE>(w + c0, at(i), D, true, o); };
  const float inv = 1.f / (float)D;
  auto norm = [&](float (&v)[NV][8], const float* w, const float* b, int c0) {
    if (a.kind == 1) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) s += v[i][j];
      const float mean = total(s) * inv;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = at(i) + j < D ? v[i][j] - mean : 0.f;
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fmaf(v[i][j], v[i][j], s);
    const float k = rsqrtf(fmaf(total(s), inv, a.eps));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float wv[8];
      vec(w, c0, i, wv);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= k * wv[j];
      if (b) {
        vec(b, c0, i, wv);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] += wv[j];
      }
    }
  };

  float v[NV][8], g[NV][8], r[NV][8];
  load(static_cast<const T*>(a.x), a.xs, v);
  if (a.gate) load(static_cast<const T*>(a.g), a.gs, g);
  if (a.rdtype >= 0) load(static_cast<const R*>(a.r), a.rs, r);
  if (a.gate == 1) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= silu_f(g[i][j]);
  }
  if (a.post_w) norm(v, a.post_w, a.post_b, col);
  if (a.gate == 2) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= silu_f(g[i][j]);
  }
  if (a.scale_v) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float sv[8];
      vec(a.scale_v, col, i, sv);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= sv[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= a.scale;
  }
  if (a.rdtype >= 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] += r[i][j];
    store(static_cast<R*>(a.ro), a.ros, v);
  }
  if (a.pre_w) norm(v, a.pre_w, a.pre_b, col);
  if (a.y) store(static_cast<T*>(a.y), a.ys, v);
}

template <typename T, typename R, int MODE>
static void launch_norm(const NormArgs& a, hipStream_t st) {
  const int D = a.dim / a.groups;
  const int64_t units = a.rows * a.groups;
  // in two dimensions: one takes fewer than 2^32 threads
  const auto grid = [&](int rows_per_block) {
    const int64_t blocks = (units + rows_per_block - 1) / rows_per_block, x = std::min<int64_t>(blocks, 1 << 20);
    return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
  };
  auto launch = [&](auto wpr, auto nv) {
    constexpr int WPR = decltype(wpr)::value, NV = decltype(nv)::value;
    SN_LAUNCH((block_norm_kernel<T, R, MODE, WPR, NV>), grid(WPR < 4 ? 4 / WPR : 1), dim3(WPR < 4 ? 256 : 64 * WPR), 0, st, a);
  };
#define SN_NORM(WPR, NV) launch(std::integral_constant<int, WPR>(), std::integral_constant<int, NV>())
  if constexpr (MODE == kSingle) {
    SN_NORM(1, 1);
  } else {
    if (D <= 512) SN_NORM(1, 1);
    else if (D <= 1024) SN_NORM(2, 1);
    else if (D <= 2048) SN_NORM(4, 1);
    else if (D <= 4096) SN_NORM(4, 2);
    else if (D <= 8192) SN_NORM(16, 1);
    else if (D <= 16384) SN_NORM(16, 2);
    else SN_NORM(16, 4);
  }
#undef SN_NORM
}

template <typename T, typename R>
static void launch_norm_v(const NormArgs& a, hipStream_t st) {
  // wide loads: every row of every tensor starts at a multiple of 16 bytes
  // (32-byte chunks of float32 go as two loads)
  const int D = a.dim / a.groups;
  const int e = sizeof(T), er = sizeof(R);
  bool vec = D % 8 == 0 && al16(a.x) && al16(a.xs * e);
  if (a.gate) vec = vec && al16(a.g) && al16(a.gs * e);
  if (a.rdtype >= 0) vec = vec && al16(a.r) && al16(a.rs * er) && al16(a.ro) && al16(a.ros * er);
  if (a.y) vec = vec && al16(a.y) && al16(a.ys * e);
  if (vec) launch_norm<T, R, kAligned>(a, st);
  else if (D >= 8) launch_norm<T, R, kAnywhere>(a, st);
  else launch_norm<T, R, kSingle>(a, st);
}

void block_norm(const NormArgs& a, hipStream_t st) {
  check(a.dim >= 1 && a.groups >= 1 && a.dim % a.groups == 0 && a.dim <= kNormMaxDim && a.rows >= 1 &&
            a.rows * a.groups < (int64_t(1) << 31) && (a.rdtype == -1 || a.rdtype == a.dtype || a.rdtype == 0),
        "norm shapes");
  if (a.dtype == 0) launch_norm_v<float, float>(a, st);
  else if (a.dtype == 1) a.rdtype == 0 ? launch_norm_v<f16, float>(a, st) : launch_norm_v<f16, f16>(a, st);
  else a.rdtype == 0 ? launch_norm_v<bf16, float>(a, st) : launch_norm_v<bf16, bf16>(a, st);
}

}  // namespace k
}  // namespace sn
