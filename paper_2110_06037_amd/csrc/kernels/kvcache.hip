// The paged key-value cache: rows written to their pages, as they are or in 8
// bits, and read back.  In 8 bits a head's row has the scale s = max|x| * (1 / 127) in
// float32 and the codes nearest to x / s (ties to even).
//
// Bound by memory where there are many rows: 16384 of 8 heads of 128 in bf16, written in 8
// bits and read back, are 202 MB in 43 us (4.7 TB/s), kept in bf16 44; 4096 rows 50 MB in 17.3 us and
// 14.6: a launch each way (2.3 us), the chain from past over the table to the page, and 6 us in all for
// the bytes at a copy's rate. Few rows are the launch and that chain: 8 rows 3.2 us to write, 3.1 to read.
#include "attn.hpp"

namespace sn {
namespace k {

// The integer nearest to x / s, ties to even, exactly, in the low 8 bits: x * inv is added
// to 1.5 * 2^23, whose last bit counts ones, so the sum rounds to an integer c. That is at most one
// off, where x / s falls next to the middle of two, and r = x - c s, which float32 holds
// without rounding, says on which side x lies: beyond half of s (an odd c: from there on), c is
// the neighbour's.
__device__ __forceinline__ unsigned code_of(float x, float s, float inv) {
  const float t = fmaf(x, inv, 12582912.f), r = fmaf(12582912.f - t, s, x);
  const unsigned c = __builtin_bit_cast(unsigned, t);
  const float half = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, 0.5f * s) - (c & 1u));
  return c + (fabsf(r) > half ? (__builtin_bit_cast(int, r) >> 31) | 1 : 0);
}
__device__ __forceinline__ V8<int8_t> codes_of(const float (&x)[8], float s, float inv) {
  V8<int8_t> q;
#pragma unroll
  for (int j = 0; j < 8; ++j) q.v[j] = (int8_t)code_of(x[j], s, inv);
  return q;
}
// The sizes of two numbers as integers of the same order, infinities and NaN behind all others.
template <typename T>
__device__ __forceinline__ unsigned size_of(const V8<T>& v) {
  unsigned most = 0;
  if constexpr (sizeof(T) == 2) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    const u32x4 w = __builtin_bit_cast(u32x4, v);
    u16x2 m = {0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[j] & 0x7fff7fffu));
    const unsigned short one = max(m[0], m[1]);
    most = __builtin_bit_cast(unsigned, to_f(__builtin_bit_cast(T, one)));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, __builtin_bit_cast(unsigned, v.v[j]) & 0x7fffffffu);
  }
  return most;
}
// max|x| * (1 / 127); rows below 127 * 2^-120 count as zeros (code_of's steps stay exact),
// and a row with an infinity or a NaN has no numbers at all.
__device__ __forceinline__ float scale_of(unsigned most) {
  if (most >= 0x7f800000u) return __builtin_nanf("");
  const float s = __builtin_bit_cast(float, most) * (1.f / 127.f);
  return s < 0x1p-120f ? 0.f : s;
}
// The largest over the 1, 2, 4 .. 64 neighbouring lanes that share a row, in all of them.
__device__ __forceinline__ unsigned max_lanes(unsigned v, int lanes) {
  auto take = [&](unsigned o) { v = max(v, o); };
  if (lanes > 1) take(__builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, false));   // XOR 1
  if (lanes > 2) take(__builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, false));   // XOR 2
  if (lanes > 4) take(__builtin_amdgcn_mov_dpp(v, 0x141, 0xF, 0xF, false));  // the other quad of 8 lanes
  if (lanes > 8) take(__builtin_amdgcn_mov_dpp(v, 0x140, 0xF, 0xF, false));  // the other 8 of 16
  if (lanes > 16) take(__shfl_xor(v, 16));
  if (lanes > 32) take(__shfl_xor(v, 32));
  return v;
}

// Single rows: a wave takes one token's row of one head, of K or of V, lane l the
// elements l, l + 64, ...; what it writes is read before the place is known.
constexpr int kRowWaves = 4;
template <typename T, bool I8, bool WRITE>
__global__ __launch_bounds__(64 * kRowWaves) void cache_rows_kernel(CacheRows a) {
  typedef typename std::conditional<I8, int8_t, T>::type E;
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & 63;
  const int64_t unit = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kRowWaves + (threadIdx.x >> 6);
  if (unit >= 2 * c.tokens * c.kv_heads) return;
  const bool key = unit & 1;
  const int64_t row = (unit >> 1) / c.kv_heads;
  const int head = (int)((unit >> 1) - row * c.kv_heads), D = c.dim;
  T* x = (key ? static_cast<T*>(a.k) + row * a.krs : static_cast<T*>(a.v) + row * a.vrs) + (int64_t)head * D;
  T t[4];
  if constexpr (WRITE) {
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = x[min(lane + 64 * i, D - 1)];
  }
  const int b = seq_of(c, row);
  if (b < 0) return;
  int64_t first, end;
  seq_rows(c, b, first, end);
  const int past = min(c.past[b], kMaxPast);
  const int pos = past < 0 ? -1 : past + (int)(row - first);
  const int page = page_of(c, b, pos), slot = pos & ((1 << c.shift) - 1);
  if (WRITE && page < 0) return;
  const int step = key ? 1 : kCacheTile;
  E* q = static_cast<E*>(key ? c.k : c.v) + (page < 0 ? 0 : key ? k_at(c, page, head, slot) : v_at(c, page, head, slot));
  float* scale = (key ? c.ks : c.vs) + (page < 0 || !I8 ? 0 : scale_at(c, page, head, slot));
  if constexpr (WRITE) {
    E e[4];
    if constexpr (I8) {
      unsigned most = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) most = max(most, __builtin_bit_cast(unsigned, to_f(t[i])) & 0x7fffffffu);
      const float s = scale_of(max_lanes(most, 64)), inv = s > 0.f ? 1.f / s : 0.f;
      if (lane == 0) *scale = s;
#pragma unroll
      for (int i = 0; i < 4; ++i) e[i] = s > 0.f ? (int8_t)code_of(to_f(t[i]), s, inv) : (int8_t)0;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) e[i] = t[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < D) q[(lane + 64 * i) * step] = e[i];
  } else {
    E e[4];
    float s = 0.f;
    if (page >= 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) e[i] = q[min(lane + 64 * i, D - 1) * step];
      if constexpr (I8) s = *scale;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (lane + 64 * i >= D) continue;
      if constexpr (I8) x[lane + 64 * i] = from_f<T>(page < 0 ? 0.f : (float)e[i] * s);
      else x[lane + 64 * i] = page < 0 ? (T)0.f : e[i];
    }
  }
}

// Many rows: a workgroup takes the 16 positions of a sequence that V keeps together, of
// K or of V, of one head or some; rows in chunks of 8 elements, and V's through LDS,
// which turns them into rows of positions.  Positions that the call does not cover are
// left alone: of a tile of which it covers only some, elements are written one by one.
// What a thread reads is all in flight at once.
constexpr int kTileThreads = 256;
constexpr int kTilePasses = 2;  // (4: the same for many rows, 3 us more for few)
template <typename T, bool I8, bool WRITE>
__global__ __launch_bounds__(kTileThreads) void cache_tiles_kernel(CacheRows a) {
  typedef typename std::conditional<I8, int8_t, T>::type E;
  constexpr int NP = kTilePasses, GE = 16 / sizeof(E), VG = 16 / GE;  // positions of a granule of 16 bytes, granules of an element
  constexpr int NG = NP * kTileThreads * 8 / GE / kTileThreads;
  // of each head [element % 8][element / 8][16 positions]: threads of a row lie next to each other
  __shared__ u32x4 turn[NP * kTileThreads * 8 / GE];
  E* te = reinterpret_cast<E*>(turn);
  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, D = c.dim, chunks = D / 8;
  int b, tile, first, n, past;
  if (c.offsets) {
    if (!find_rows(c, blockIdx.x, [&](int rows, int before) { return (int64_t)rows_tiles(before, rows); }, b, tile, first, n, past)) return;
  } else {  // sequences of equal lengths have the same bound of tiles each: no search
    // (4096 rows written and read 17.3 us, searched for 19.0)
    n = (int)c.each;
    const int of = n / 16 + 2;
    b = uniform(blockIdx.x / of);
    if (b >= c.seqs) return;
    tile = blockIdx.x - b * of, first = b * n, past = uniform(min(c.past[b], kMaxPast));
    if (tile >= rows_tiles(past, n)) return;
  }
  const int pos0 = (max(past, 0) & ~15) + 16 * tile;  // of the tile
  const int slot0 = pos0 & ((1 << c.shift) - 1);
  const bool whole = past >= 0 && pos0 >= past && pos0 + 16 <= past + n;
  const int row0 = pos0 - max(past, 0);  // of the sequence (a slot without one counts from 0, and reads zeros)
  const bool key = blockIdx.z == 0;
  T* rows = static_cast<T*>(key ? a.k : a.v);
  const int64_t stride = key ? a.krs : a.vrs;
  // a pass: `slots` rows of `lanes` threads each
  const int lanes = a.lanes, slots = kTileThreads / lanes, ch = tid & (lanes - 1), heads = NP * slots / 16, head0 = blockIdx.y * heads;
  auto at_pass = [&](int p, int& s, int& hh) {  // position in the tile, head of the group; whether the call has the row
    const int u = p * slots + tid / lanes;
    s = u & 15, hh = u >> 4;
    return ch < chunks && head0 + hh < c.kv_heads && row0 + s >= 0 && row0 + s < n;
  };
  auto row_at = [&](int s, int hh) { return rows + (int64_t)(first + row0 + s) * stride + (int64_t)(head0 + hh) * D + 8 * ch; };
  V8<T> v[NP];
  if constexpr (WRITE) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      int s, hh;
      v[p] = zero8<T>();
      if (at_pass(p, s, hh)) __builtin_memcpy(&v[p], row_at(s, hh), sizeof(v[p]));
    }
  }
  const int page = past < 0 ? -1 : page_of(c, b, pos0);
  if (WRITE && page < 0) return;
  E* store = static_cast<E*>(key ? c.k : c.v);
  float* scales = key ? c.ks : c.vs;
  auto tile_at = [&](int hh) { return ((((int64_t)max(page, 0) * c.kv_heads + head0 + hh) << c.shift) + slot0); };
  auto turned = [&](int s, int hh, int j) { return te + ((hh * 8 + j) * lanes + ch) * 16 + s; };
  // V's granules, all heads of the group one after the other: in LDS, in memory
  const int granules = min(heads, c.kv_heads - head0) * D * VG;
  auto granule = [&](int g, u32x4*& in_lds, u32x4*& in_memory) {
    const int hh = fdiv(g, a.head_granules), e = g - hh * (D * VG), d = e / VG, part = e % VG;
    in_lds = turn + ((hh * 8 + (d & 7)) * lanes + (d >> 3)) * VG + part;
    in_memory = reinterpret_cast<u32x4*>(store + tile_at(hh) * D + d * 16 + part * GE);
  };
  if constexpr (WRITE) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      int s, hh;
      const bool mine = at_pass(p, s, hh);
      V8<E> q;
      if constexpr (I8) {
        const float sc = scale_of(max_lanes(size_of(v[p]), lanes)), inv = sc > 0.f ? 1.f / sc : 0.f;
        if (mine && ch == 0) scales[tile_at(hh) + s] = sc;
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = to_f(v[p].v[j]);
        q = codes_of(f, sc, inv);
        if (!(sc > 0.f)) q = V8<int8_t>{};
      } else {
        q = v[p];
      }
      if (!mine) continue;
      if (key) {
        __builtin_memcpy(__builtin_assume_aligned(store + (tile_at(hh) + s) * D + 8 * ch, 8), &q, sizeof(q));
      } else if (whole) {
#pragma unroll
        for (int j = 0; j < 8; ++j) *turned(s, hh, j) = q.v[j];
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) store[tile_at(hh) * D + (8 * ch + j) * 16 + s] = q.v[j];
      }
    }
    if (key || !whole) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      u32x4 *l, *m;
      if (i * kTileThreads + tid >= granules) break;
      granule(i * kTileThreads + tid, l, m);
      *m = *l;
    }
  } else {
    V8<E> q[NP];
    float sc[NP];
    if (page >= 0) {
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        int s, hh;
        const bool mine = at_pass(p, s, hh);
        if (I8 && mine) sc[p] = scales[tile_at(hh) + s];
        if (key && mine) __builtin_memcpy(&q[p], __builtin_assume_aligned(store + (tile_at(hh) + s) * D + 8 * ch, 8), sizeof(q[p]));
      }
      if (!key) {
        u32x4 r[NG], *l, *m;
#pragma unroll
        for (int i = 0; i < NG; ++i)
          if (i * kTileThreads + tid < granules) granule(i * kTileThreads + tid, l, m), r[i] = *m;
#pragma unroll
        for (int i = 0; i < NG; ++i)
          if (i * kTileThreads + tid < granules) granule(i * kTileThreads + tid, l, m), *l = r[i];
        __syncthreads();
      }
    }
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      int s, hh;
      if (!at_pass(p, s, hh)) continue;
      V8<T> t = zero8<T>();
      if (page >= 0) {
        if (!key)
#pragma unroll
          for (int j = 0; j < 8; ++j) q[p].v[j] = *turned(s, hh, j);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if constexpr (I8) t.v[j] = from_f<T>((float)q[p].v[j] * sc[p]);
          else t.v[j] = q[p].v[j];
        }
      }
      __builtin_memcpy(row_at(s, hh), &t, sizeof(t));
    }
  }
}

template <typename T, bool WRITE>
static void launch_rows(CacheRows& a, hipStream_t st) {
  const CacheArgs& c = a.c;
  // Tiles of 16 positions for many rows of few sequences, single rows by waves.  (Written
  // and read back, 8 heads of 128 in 8 bits: 8 sequences of 16 rows 9.4 us by tiles, 6.3 by
  // rows; of 64 rows 10.1 and 10.9; of 512 rows 22 and 51; 64 of one row 12.4 and 5.7.)
  // Not for very many sequences: every workgroup counts tiles over them.
  if (c.tokens >= 4 * (int64_t)c.seqs && c.tokens * c.kv_heads >= 4096 && c.seqs <= 512) {
    const int64_t tiles = c.tokens / 16 + 2 * (int64_t)c.seqs;
    a.lanes = 1;
    while (a.lanes < c.dim / 8) a.lanes *= 2;
    a.head_granules = make_fastdiv(c.dim * (c.i8 ? 1 : (int)sizeof(T)));
    const int heads = kTilePasses * (kTileThreads / a.lanes) / 16;
    const dim3 grid((unsigned)tiles, (c.kv_heads + heads - 1) / heads, 2);
    if (c.i8) SN_LAUNCH((cache_tiles_kernel<T, true, WRITE>), grid, dim3(kTileThreads), 0, st, a);
    else SN_LAUNCH((cache_tiles_kernel<T, false, WRITE>), grid, dim3(kTileThreads), 0, st, a);
    return;
  }
  const int64_t blocks = (2 * c.tokens * c.kv_heads + kRowWaves - 1) / kRowWaves, x = std::min<int64_t>(blocks, 1 << 20);
  const dim3 grid((unsigned)x, (unsigned)((blocks + x - 1) / x)), block(64 * kRowWaves);
  if (c.i8) SN_LAUNCH((cache_rows_kernel<T, true, WRITE>), grid, block, 0, st, a);
  else SN_LAUNCH((cache_rows_kernel<T, false, WRITE>), grid, block, 0, st, a);
}
template <bool WRITE>
static void cache_rows(const CacheRows& args, hipStream_t st) {
  CacheRows a = args;
  const CacheArgs& c = a.c;
  check(c.dim >= 8 && c.dim <= 256 && c.dim % 8 == 0 && c.kv_heads >= 1 && c.shift >= 4 && c.seqs >= 1 && c.tokens >= 1 &&
            (c.tokens * c.kv_heads) >> 39 == 0,
        "cache shapes");
  if (c.dtype == 0) launch_rows<float, WRITE>(a, st);
  else if (c.dtype == 1) launch_rows<f16, WRITE>(a, st);
  else launch_rows<bf16, WRITE>(a, st);
}
void cache_write(const CacheRows& a, hipStream_t st) { cache_rows<true>(a, st); }
void cache_read(const CacheRows& a, hipStream_t st) { cache_rows<false>(a, st); }

}  // namespace k
}  // namespace sn
