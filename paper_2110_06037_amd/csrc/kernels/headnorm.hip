// Norms of queries and keys for each head, with the position rotation in the
// same pass: x * rsqrt(mean(x^2) + eps) * w over a head's elements, then each
// pair (a, b) of its first `rot` elements turned by position * freq: a cos - b
// sin, b cos + a sin.  A turn is counted in 2^-64 of a circle, so that position
// times turn wraps to the angle with nothing lost at any position.  The sines of a
// token are made once, one a thread, and shared by all of its heads through LDS.
//
// Bound by memory where there are many tokens, the bytes of x and y once each: 4096 tokens of
// 40 heads of 128 in bf16 14.5 us, 5.8 TB/s, in float32 26.9, 6.2 TB/s; 16384 tokens 65 us,
// beyond the caches, 5.2 TB/s.  Below some hundred tokens the launch and two trips to memory
// remain (the row with its position, which the sines wait for; the weights are read beside
// them): one token 2.7 us.  Sizes that do not come in chunks of 4 elements (72 elements,
// of which 50 rotate, in f16) take single elements, 33 us for 4096 tokens.
#include "attn.hpp"

namespace sn {
namespace k {

constexpr int kHeadThreads = 256, kHeadTokens = 4, kHeadPairs = 128;

// The sum over the 1, 2, 4 .. 32 neighbouring lanes that share a row, in all of them.
__device__ __forceinline__ float sum_lanes(float v, int lanes) {
  if (lanes > 1) v += dpp_take<0xB1>(v);   // XOR 1
  if (lanes > 2) v += dpp_take<0x4E>(v);   // XOR 2
  if (lanes > 4) v += dpp_take<0x141>(v);  // the other quad of 8 lanes
  if (lanes > 8) v += dpp_take<0x140>(v);  // the other 8 of 16
  if (lanes > 16) v += __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), 0x401F));  // XOR 16
  return v;
}

// A workgroup takes some tokens, four where they fill the chip, so that the sines, the
// weights and the launch of a workgroup are paid once for 160 rows instead of 40 (4096 tokens
// 15.2 us, by single ones 17.3; 256 tokens 5.3 and 3.9); `lanes` threads a row (one head of one token), each
// two chunks of V elements: of the rotated pairs' two halves (HALVES), or one after the
// other; of what does not rotate likewise.
template <typename T, int V, bool HALVES>
__global__ __launch_bounds__(kHeadThreads) void head_norm_kernel(HeadNormArgs a) {
  __shared__ float sc[kHeadTokens][kHeadPairs], ss[kHeadTokens][kHeadPairs];
  const int tid = threadIdx.x, D = a.dim, half = a.rot / 2, all = a.heads + a.kv_heads;
  const int64_t token0 = (int64_t)blockIdx.x * a.tokens_each;
  const int tokens = (int)min<int64_t>(a.tokens_each, a.tokens - token0);
  const int slot = tid & (a.lanes - 1), step = kHeadThreads / a.lanes;
  // this thread's elements and pairs
  int ia, ib, pair;
  bool turned = true;
  if constexpr (HALVES) {
    const int c = slot * V;
    turned = c < half;
    ia = turned ? c : a.rot + (c - half);
    ib = turned ? c + half : a.rot + (D - a.rot) / 2 + (c - half);
    pair = turned ? c : 0;
  } else {
    ia = 2 * slot * V, ib = ia + V, pair = slot * V;
  }
  const bool on = 2 * slot * V < D;
  if (!on) ia = ib = 0;  // (loads are behind no branch, whose join would wait for them)

  // a row's elements, read one row ahead: the first while the sines are made
  const int rows = tokens * all, next = gridDim.y * step;
  T xa[V], xb[V];
  int row = blockIdx.y * step + tid / a.lanes;
  auto place = [&](int r, const void* q, int64_t qs, const void* k, int64_t ks) {
    const int tk = fdiv(r, a.all), h = r - tk * all;
    const int64_t token = token0 + tk;
    return h >= a.heads ? static_cast<const T*>(k) + token * ks + (int64_t)(h - a.heads) * D
                        : static_cast<const T*>(q) + token * qs + (int64_t)h * D;
  };
  auto fetch = [&](int r) {
    const T* x = place(min(r, rows - 1), a.q, a.qs, a.k, a.ks);
    __builtin_memcpy(xa, x + ia, sizeof(xa));
    __builtin_memcpy(xb, x + ib, sizeof(xb));
  };
  fetch(row);
  for (int i = tid; i < tokens * half; i += kHeadThreads) {
    const int tk = i / half, j = i - tk * half;
    const long long p = a.positions[token0 + tk];
    const long long t = (long long)((unsigned long long)p * a.turn[j]);  // signed: -1/2 .. 1/2 of a circle
    sincospif((float)t * 0x1p-63f, &ss[tk][j], &sc[tk][j]);
  }
  float wq[2][V], wk[2][V];
  __builtin_memcpy(wq[0], a.q_w + ia, sizeof(wq[0]));
  __builtin_memcpy(wq[1], a.q_w + ib, sizeof(wq[1]));
  __builtin_memcpy(wk[0], a.k_w + ia, sizeof(wk[0]));
  __builtin_memcpy(wk[1], a.k_w + ib, sizeof(wk[1]));
  __syncthreads();
  for (; row < rows; row += next) {
    const int tk = fdiv(row, a.all), h = row - tk * all;
    const bool key = h >= a.heads;
    T ta[V], tb[V];
    __builtin_memcpy(ta, xa, sizeof(ta));
    __builtin_memcpy(tb, xb, sizeof(tb));
    fetch(row + next);
    float va[V], vb[V], s = 0.f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      va[j] = on ? to_f(ta[j]) : 0.f, vb[j] = on ? to_f(tb[j]) : 0.f;
      s = fmaf(va[j], va[j], fmaf(vb[j], vb[j], s));
    }
    const float k = a.norm ? rsqrtf(sum_lanes(s, a.lanes) / (float)D + a.eps) : 1.f;
#pragma unroll
    for (int j = 0; j < V; ++j) va[j] *= k * (key ? wk : wq)[0][j], vb[j] *= k * (key ? wk : wq)[1][j];
    if constexpr (HALVES) {
      if (turned)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float c = sc[tk][pair + j], n = ss[tk][pair + j], u = va[j], w = vb[j];
          va[j] = u * c - w * n, vb[j] = w * c + u * n;
        }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (pair + j >= half) continue;
        const float c = sc[tk][pair + j], n = ss[tk][pair + j];
        float& u = 2 * j < V ? va[2 * j] : vb[2 * j - V];
        float& w = 2 * j < V ? va[2 * j + 1] : vb[2 * j + 1 - V];
        const float u0 = u, w0 = w;
        u = u0 * c - w0 * n, w = w0 * c + u0 * n;
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) ta[j] = from_f<T>(va[j]), tb[j] = from_f<T>(vb[j]);
    if (!on) continue;
    T* y = const_cast<T*>(place(row, a.qo, a.qos, a.ko, a.kos));
    __builtin_memcpy(y + ia, ta, sizeof(ta));
    __builtin_memcpy(y + ib, tb, sizeof(tb));
  }
}

// Sizes that do not come in such chunks: a wave takes one head after the other of a
// token, lane l the pairs l, l + 64, ... of all of them, by single elements.
constexpr int kHeadWaves = 4;
template <typename T, int NP>
__global__ __launch_bounds__(64 * kHeadWaves) void head_norm_any_kernel(HeadNormArgs a) {
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
      const float u = va[i] * (ia[i] < D ? k * w[ia[i]] : k), v = vb[i] * (ib[i] < D ? k * w[ib[i]] : k);
      const bool turned = lane + 64 * i < half;  // (others stay apart: 0 times what is not finite is NaN)
      if (ia[i] < D) y[ia[i]] = from_f<T>(turned ? u * cs[i] - v * sn[i] : u);
      if (ib[i] < D) y[ib[i]] = from_f<T>(turned ? v * cs[i] + u * sn[i] : v);
    }
  }
}

template <typename T, int V>
static void launch_head_norm(HeadNormArgs& a, hipStream_t st) {
  const int all = a.heads + a.kv_heads, slots = a.dim / (2 * V);
  a.all = make_fastdiv(all);
  a.lanes = 1;
  while (a.lanes < slots) a.lanes *= 2;
  a.tokens_each = a.tokens >= 256 * kHeadTokens ? kHeadTokens : 1;
  const int step = kHeadThreads / a.lanes;
  // few tokens: a token's heads over several workgroups (1024 of them rather than 256, for 256 tokens 3.9
  // us, 4.4; for 1024 tokens 6.4 and 8.1)
  const int64_t x = (a.tokens + a.tokens_each - 1) / a.tokens_each;
  const int y = (int)std::min<int64_t>((all + step - 1) / step, std::max<int64_t>(1, 1024 / x));
  const dim3 grid((unsigned)x, y), block(kHeadThreads);
  if (a.pairs == 0) SN_LAUNCH((head_norm_kernel<T, V, true>), grid, block, 0, st, a);
  else SN_LAUNCH((head_norm_kernel<T, V, false>), grid, block, 0, st, a);
}

template <typename T>
static void launch_head_norm(HeadNormArgs& a, hipStream_t st) {
  // whole chunks of V in each half of what rotates and of what does not
  auto fits = [&](int V) {
    return a.pairs == 0 ? a.rot / 2 % V == 0 && (a.dim - a.rot) % (2 * V) == 0 : a.dim % (2 * V) == 0;
  };
  if constexpr (sizeof(T) == 2)
    if (fits(8)) return launch_head_norm<T, 8>(a, st);
  if (fits(4)) return launch_head_norm<T, 4>(a, st);
  const int all = a.heads + a.kv_heads;
  const int y = (int)std::min<int64_t>((all + kHeadWaves - 1) / kHeadWaves, std::max<int64_t>(1, 512 / a.tokens));
  const dim3 grid((unsigned)a.tokens, y), block(64 * kHeadWaves);
  if (a.dim <= 128) SN_LAUNCH((head_norm_any_kernel<T, 1>), grid, block, 0, st, a);
  else SN_LAUNCH((head_norm_any_kernel<T, 2>), grid, block, 0, st, a);
}

void head_norm(const HeadNormArgs& args, hipStream_t st) {
  HeadNormArgs a = args;
  check(a.dim >= 1 && a.dim <= 2 * kHeadPairs && a.rot >= 0 && a.rot <= a.dim && a.rot % 2 == 0 && a.heads + a.kv_heads >= 1 &&
            a.tokens >= 1 && a.tokens < (int64_t(1) << 24) && (a.rot == 0 || a.positions),
        "head norm shapes");
  if (a.dtype == 0) launch_head_norm<float>(a, st);
  else if (a.dtype == 1) launch_head_norm<f16>(a, st);
  else launch_head_norm<bf16>(a, st);
}

}  // namespace k
}  // namespace sn
