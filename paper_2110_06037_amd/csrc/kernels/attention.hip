// Attention over the paged cache: row i of sequence b stands at position p =
// past[b] + i and its query heads see the positions max(0, p - window + 1) .. p,
// y = sum softmax(scale q k) v, with the running maximum and sum of one pass.
#include "attn.hpp"

namespace sn {
namespace k {

// A wave takes one head of one row, a lane the elements l, l + 64, ...
template <typename T, bool I8>
__global__ __launch_bounds__(64) void attention_kernel(AttnArgs a) {
  const CacheArgs& c = a.c;
  const int64_t row = blockIdx.x;
  const int h = blockIdx.y, lane = threadIdx.x, D = c.dim;
  const int kvh = h / (a.heads / c.kv_heads);
  const int b = seq_of(c, row);
  if (b < 0) return;
  int64_t first, end;
  seq_rows(c, b, first, end);
  const int past = min(c.past[b], kMaxPast);
  const T* q = static_cast<const T*>(a.q) + row * a.qs + (int64_t)h * D;
  T* y = static_cast<T*>(a.y) + row * a.ys + (int64_t)h * D;
  float qv[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -__builtin_huge_valf(), m0, l = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) qv[i] = lane + 64 * i < D ? to_f(q[lane + 64 * i]) * (a.scale * kLog2e) : 0.f;
  const int pos = past < 0 ? -1 : past + (int)(row - first);
  const int last = (int)min((int64_t)pos, ((int64_t)c.width << c.shift) - 1);
  for (int p = a.window ? max(0, pos - a.window + 1) : 0; p <= last; ++p) {
    const int page = page_of(c, b, p), slot = p & ((1 << c.shift) - 1);
    if (page < 0) continue;
    const int64_t ka = k_at(c, page, kvh, slot), va = v_at(c, page, kvh, slot);
    float kv[4], vv[4], s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = min(lane + 64 * i, D - 1);
      if constexpr (I8) {
        kv[i] = (float)static_cast<const int8_t*>(c.k)[ka + d];
        vv[i] = (float)static_cast<const int8_t*>(c.v)[va + d * kCacheTile];
      } else {
        kv[i] = to_f(static_cast<const T*>(c.k)[ka + d]);
        vv[i] = to_f(static_cast<const T*>(c.v)[va + d * kCacheTile]);
      }
      s = fmaf(qv[i], lane + 64 * i < D ? kv[i] : 0.f, s);
    }
    s = wave_sum(s);
    float vs = 1.f;
    if constexpr (I8) s *= c.ks[scale_at(c, page, kvh, slot)], vs = c.vs[scale_at(c, page, kvh, slot)];
    m0 = m, m = fmaxf(m, s);
    const float n = m == -__builtin_huge_valf() ? 0.f : m, f = __builtin_amdgcn_exp2f(m0 - n), e = __builtin_amdgcn_exp2f(s - n);
    l = l * f + e;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = o[i] * f + e * vs * vv[i];
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (lane + 64 * i < D) y[lane + 64 * i] = from_f<T>(o[i] * inv);
}

template <typename T>
static void launch_attention(const AttnArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)a.c.tokens, a.heads);
  if (a.c.i8) SN_LAUNCH((attention_kernel<T, true>), grid, dim3(64), 0, st, a);
  else SN_LAUNCH((attention_kernel<T, false>), grid, dim3(64), 0, st, a);
}

void attention(const AttnArgs& a, hipStream_t st) {
  const CacheArgs& c = a.c;
  check(c.dim >= 8 && c.dim <= 256 && c.dim % 8 == 0 && c.kv_heads >= 1 && a.heads % c.kv_heads == 0 && a.heads <= 65535 &&
            c.shift >= 4 && c.seqs >= 1 && c.tokens >= 1 && c.tokens < (1 << 26),
        "attention shapes");
  if (c.dtype == 0) launch_attention<float>(a, st);
  else if (c.dtype == 1) launch_attention<f16>(a, st);
  else launch_attention<bf16>(a, st);
}

}  // namespace k
}  // namespace sn
