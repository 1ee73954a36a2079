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

// The largest over the 1, 2, 4 .. 32 neighbouring lanes that share a row, in all of them.
__device__ __forceinline__ float max_lanes(float v, int lanes) {
  if (lanes > 1) v = fmaxf(v, dpp_take<0xB1>(v));   // XOR 1
  if (lanes > 2) v = fmaxf(v, dpp_take<0x4E>(v));   // XOR 2
  if (lanes > 4) v = fmaxf(v, dpp_take<0x141>(v));  // the other quad of 8 lanes
  if (lanes > 8) v = fmaxf(v, dpp_take<0x140>(v));  // the other 8 of 16
  if (lanes > 16) v = fmaxf(v, __shfl_xor(v, 16));
  return v;
}

// A wave takes one token's row of one head, of K and of V.
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

// Many rows: a workgroup takes the 16 positions of a sequence that V keeps together,
// of one head or, of small ones, some; K's rows in chunks of 8, V's through LDS,
// which turns them into rows of positions.  Positions that the call does not cover are left
// alone: of a tile of which it covers only some, elements are written one by one.
constexpr int kTileThreads = 256;
template <typename T, bool I8, bool WRITE>
__global__ __launch_bounds__(kTileThreads) void cache_tiles_kernel(CacheRows a) {
  typedef typename std::conditional<I8, int8_t, T>::type E;
  // [8 elements' chunk j][chunk][16 positions]: threads of a row's chunks next to each other
  __shared__ __attribute__((aligned(16))) E turn[8 * kTileThreads * 2];
  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, D = c.dim, chunks = D / 8;
  int b, tile, first, n;
  if (!find_rows(c, blockIdx.x, [&](int s, int rows) { return rows_tiles(c.past[s], rows); }, b, tile, first, n)) return;
  const int past = min(c.past[b], kMaxPast);
  const int pos0 = (max(past, 0) & ~15) + 16 * tile;  // of the tile
  const int page = past < 0 ? -1 : page_of(c, b, pos0);
  if (WRITE && page < 0) return;
  const int slot0 = pos0 & ((1 << c.shift) - 1);
  const bool whole = past >= 0 && pos0 >= past && pos0 + 16 <= past + n;
  // lanes of a row of 8-element chunks, rows of one head that lie 16 * lanes threads apart
  const int lanes = a.lanes, slots = kTileThreads / lanes, ch = tid & (lanes - 1);
  const bool key = blockIdx.z == 0;
  T* rows = static_cast<T*>(key ? a.k : a.v);
  const int64_t stride = key ? a.krs : a.vrs;
  E* store = static_cast<E*>(key ? c.k : c.v);
  float* scales = key ? c.ks : c.vs;
  const int heads = max(1, slots / 16);  // of a pass
  for (int pass = 0; pass < max(1, 16 / slots); ++pass) {
    const int u = pass * slots + tid / lanes, s = u & 15, hh = u >> 4;  // token of the tile, head of the group
    const int head = blockIdx.y * heads + hh;
    const bool on = ch < chunks && head < c.kv_heads;
    // rows of a slot without a sequence are counted from 0 (they are read as zeros)
    const int row = pos0 + s - max(past, 0);
    const bool mine = on && row >= 0 && row < n;
    T* x = rows + (int64_t)(first + row) * stride + (int64_t)head * D + 8 * ch;
    const int64_t at = ((((int64_t)max(page, 0) * c.kv_heads + min(head, c.kv_heads - 1)) << c.shift) + slot0);  // of the tile's rows
    if constexpr (WRITE) {
      V8<T> v = zero8<T>();
      if (mine) __builtin_memcpy(&v, x, sizeof(v));
      V8<E> q;
      if constexpr (I8) {
        float most = 0.f, f[8];
        bool fine = true;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = to_f(v.v[j]), most = fmaxf(most, fabsf(f[j])), fine = fine && __builtin_isfinite(f[j]);
        if (!fine) most = __builtin_huge_valf();
        most = max_lanes(most, lanes);
        const float sc = scale_of(most, __builtin_isfinite(most)), inv = sc > 0.f ? 1.f / sc : 0.f;
        if (mine && ch == 0) scales[at + s] = sc;
#pragma unroll
        for (int j = 0; j < 8; ++j) q.v[j] = sc > 0.f ? (int8_t)(int)code_of(f[j], sc, inv) : (int8_t)0;
      } else {
        q = v;
      }
      if (key) {
        if (mine) __builtin_memcpy(__builtin_assume_aligned(store + (at + s) * D + 8 * ch, 8), &q, sizeof(q));
      } else if (whole) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (on) turn[((hh * 8 + j) * lanes + ch) * 16 + s] = q.v[j];
      } else if (mine) {
#pragma unroll
        for (int j = 0; j < 8; ++j) store[at * D + (8 * ch + j) * 16 + s] = q.v[j];
      }
    } else if (key) {
      if (mine) {
        V8<T> v = zero8<T>();
        if (page >= 0) {
          V8<E> q;
          __builtin_memcpy(&q, __builtin_assume_aligned(store + (at + s) * D + 8 * ch, 8), sizeof(q));
          if constexpr (I8) {
            const float sc = scales[at + s];
#pragma unroll
            for (int j = 0; j < 8; ++j) v.v[j] = from_f<T>((float)q.v[j] * sc);
          } else {
            v = q;
          }
        }
        __builtin_memcpy(x, &v, sizeof(v));
      }
    }
  }
  if (key) return;
  // V: granules of 16 bytes between LDS and the tile's memory, of all heads of the group
  constexpr int GE = 16 / sizeof(E), VG = 16 / GE;  // positions of a granule, granules of an element
  auto each_granule = [&](auto f) {
    for (int g = tid; g < heads * D * VG; g += kTileThreads) {
      const int hh = g / (D * VG), e = g - hh * (D * VG), d = e / VG, part = e % VG, head = blockIdx.y * heads + hh;
      if (head >= c.kv_heads) break;
      const int64_t at = ((((int64_t)max(page, 0) * c.kv_heads + head) << c.shift) + slot0);
      f(turn + ((hh * 8 + (d & 7)) * lanes + (d >> 3)) * 16 + part * GE, store + at * D + d * 16 + part * GE);
    }
  };
  if constexpr (WRITE) {
    if (!whole) return;
    __syncthreads();
    each_granule([&](const E* from, E* to) { *reinterpret_cast<u32x4*>(to) = *reinterpret_cast<const u32x4*>(from); });
  } else {
    if (page >= 0) {
      each_granule([&](E* to, const E* from) { *reinterpret_cast<u32x4*>(to) = *reinterpret_cast<const u32x4*>(from); });
      __syncthreads();
    }
    for (int pass = 0; pass < max(1, 16 / slots); ++pass) {
      const int u = pass * slots + tid / lanes, s = u & 15, hh = u >> 4, head = blockIdx.y * heads + hh, row = pos0 + s - max(past, 0);
      if (ch >= chunks || head >= c.kv_heads || row < 0 || row >= n) continue;
      V8<T> v = zero8<T>();
      if (page >= 0) {
        const float sc = I8 ? scales[((((int64_t)page * c.kv_heads + head) << c.shift) + slot0) + s] : 1.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const E q = turn[((hh * 8 + j) * lanes + ch) * 16 + s];
          if constexpr (I8) v.v[j] = from_f<T>((float)q * sc);
          else v.v[j] = q;
        }
      }
      __builtin_memcpy(rows + (int64_t)(first + row) * stride + (int64_t)head * D + 8 * ch, &v, sizeof(v));
    }
  }
}

template <typename T, bool WRITE>
static void launch_rows(CacheRows& a, hipStream_t st) {
  const CacheArgs& c = a.c;
  // A tile of 16 positions for sequences of some rows each; single rows by waves.
  // (At 8 rows a sequence, half a tile, both take the same time.)
  const int64_t tiles = c.tokens / 16 + 2 * (int64_t)c.seqs;
  if (c.tokens >= 8 * (int64_t)c.seqs) {
    a.lanes = 1;
    while (a.lanes < c.dim / 8) a.lanes *= 2;
    const int heads = std::max(1, kTileThreads / a.lanes / 16);
    const dim3 grid((unsigned)tiles, (c.kv_heads + heads - 1) / heads, 2);
    if (c.i8) SN_LAUNCH((cache_tiles_kernel<T, true, WRITE>), grid, dim3(kTileThreads), 0, st, a);
    else SN_LAUNCH((cache_tiles_kernel<T, false, WRITE>), grid, dim3(kTileThreads), 0, st, a);
    return;
  }
  const int64_t blocks = (c.tokens * c.kv_heads + kRowWaves - 1) / kRowWaves, x = std::min<int64_t>(blocks, 1 << 20);
  const dim3 grid((unsigned)x, (unsigned)((blocks + x - 1) / x)), block(64 * kRowWaves);
  if (c.i8) SN_LAUNCH((cache_rows_kernel<T, true, WRITE>), grid, block, 0, st, a);
  else SN_LAUNCH((cache_rows_kernel<T, false, WRITE>), grid, block, 0, st, a);
}
template <bool WRITE>
static void cache_rows(const CacheRows& args, hipStream_t st) {
  CacheRows a = args;
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
