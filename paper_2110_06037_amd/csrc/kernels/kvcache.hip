// The paged key-value cache: rows written to their pages, as they are or in 8
// bits, and read back.  In 8 bits a head's row has the scale s = max|x| * (1 / 127) in
// float32 and the codes nearest to x / s (ties to even).
#include "attn.hpp"

namespace sn {
namespace k {

// The integer nearest to x / s, ties to even, exactly: a rounded quotient is at
// most one off where it falls next to the middle of two, and r = x - c s, which
// float32 holds without rounding there, says on which side x lies.
__device__ __forceinline__ float code_of(float x, float s, float inv) {
  float c = rintf(x * inv);
  const float r = fmaf(-c, s, x), h = 0.5f * s;
  const bool odd = (int)c & 1;
  if (r > h || (r == h && odd)) c += 1.f;
  if (r < -h || (r == -h && odd)) c -= 1.f;
  return c;
}
// max|x| * (1 / 127); rows below 127 * 2^-120 count as zeros (code_of's steps stay exact),
// and a row with an infinity or a NaN has no numbers at all.
__device__ __forceinline__ float scale_of(float most, bool fine) {
  if (!fine) return __builtin_nanf("");
  const float s = most * (1.f / 127.f);
  return s < 0x1p-120f ? 0.f : s;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int i = 32; i; i >>= 1) v = fmaxf(v, __shfl_xor(v, i));
  return v;
}

// A wave takes one token's row of one head, of K or of V.
constexpr int kRowWaves = 4;
template <typename T, bool I8, bool WRITE>
__global__ __launch_bounds__(64 * kRowWaves) void cache_rows_kernel(CacheRows a) {
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & 63;
  const int64_t unit = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kRowWaves + (threadIdx.x >> 6);
  if (unit >= c.tokens * c.kv_heads) return;
  const int64_t row = unit / c.kv_heads;
  const int head = (int)(unit - row * c.kv_heads), D = c.dim;
  const int b = seq_of(c, row);
  if (b < 0) return;
  int64_t first, end;
  seq_rows(c, b, first, end);
  const int past = min(c.past[b], kMaxPast);
  const int pos = past < 0 ? -1 : past + (int)(row - first);
  const int page = page_of(c, b, pos);
  const int slot = pos & ((1 << c.shift) - 1);
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    T* x = which ? static_cast<T*>(a.v) + row * a.vrs : static_cast<T*>(a.k) + row * a.krs;
    x += (int64_t)head * D;
    const int64_t at = page < 0 ? 0 : which ? v_at(c, page, head, slot) : k_at(c, page, head, slot);
    const int step = which ? kCacheTile : 1;
    float* scale = which ? c.vs : c.ks;
    if constexpr (WRITE) {
      if (page < 0) continue;
      if constexpr (I8) {
        float v[4], most = 0.f;
        bool fine = true;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = lane + 64 * i < D ? to_f(x[lane + 64 * i]) : 0.f;
          most = fmaxf(most, fabsf(v[i]));
          fine = fine && __builtin_isfinite(v[i]);
        }
        const float s = scale_of(wave_max(most), __all(fine));
        const float inv = s > 0.f ? 1.f / s : 0.f;
        if (lane == 0) scale[scale_at(c, page, head, slot)] = s;
        int8_t* q = static_cast<int8_t*>(which ? c.v : c.k) + at;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (lane + 64 * i < D) q[(lane + 64 * i) * step] = s > 0.f ? (int8_t)(int)code_of(v[i], s, inv) : (int8_t)0;
      } else {
        T* q = static_cast<T*>(which ? c.v : c.k) + at;
        for (int d = lane; d < D; d += 64) q[d * step] = x[d];
      }
    } else {
      if constexpr (I8) {
        const float s = page < 0 ? 0.f : scale[scale_at(c, page, head, slot)];
        const int8_t* q = static_cast<const int8_t*>(which ? c.v : c.k) + at;
        for (int d = lane; d < D; d += 64) x[d] = from_f<T>(page < 0 ? 0.f : (float)q[d * step] * s);
      } else {
        const T* q = static_cast<const T*>(which ? c.v : c.k) + at;
        for (int d = lane; d < D; d += 64) x[d] = page < 0 ? (T)0.f : q[d * step];
      }
    }
  }
}

template <typename T, bool WRITE>
static void launch_rows(const CacheRows& a, hipStream_t st) {
  const int64_t blocks = (a.c.tokens * a.c.kv_heads + kRowWaves - 1) / kRowWaves, x = std::min<int64_t>(blocks, 1 << 20);
  const dim3 grid((unsigned)x, (unsigned)((blocks + x - 1) / x)), block(64 * kRowWaves);
  if (a.c.i8) SN_LAUNCH((cache_rows_kernel<T, true, WRITE>), grid, block, 0, st, a);
  else SN_LAUNCH((cache_rows_kernel<T, false, WRITE>), grid, block, 0, st, a);
}
template <bool WRITE>
static void cache_rows(const CacheRows& a, hipStream_t st) {
  const CacheArgs& c = a.c;
  check(c.dim >= 8 && c.dim <= 256 && c.dim % 8 == 0 && c.kv_heads >= 1 && c.shift >= 4 && c.seqs >= 1 && c.tokens >= 1 &&
            (c.tokens * c.kv_heads) >> 40 == 0,
        "cache shapes");
  if (c.dtype == 0) launch_rows<float, WRITE>(a, st);
  else if (c.dtype == 1) launch_rows<f16, WRITE>(a, st);
  else launch_rows<bf16, WRITE>(a, st);
}
void cache_write(const CacheRows& a, hipStream_t st) { cache_rows<true>(a, st); }
void cache_read(const CacheRows& a, hipStream_t st) { cache_rows<false>(a, st); }

}  // namespace k
}  // namespace sn
