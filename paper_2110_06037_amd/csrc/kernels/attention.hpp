// Attention over the paged cache: row i of sequence b stands at position p =
// past[b] + i and its query heads see the positions max(0, p - window + 1) .. p:
// y = sum exp(scale q k) v / sum exp(scale q k), in one pass over the keys with
// a running maximum.  Both kernels compute S^T = K Q^T and O^T = V^T P^T, so that a
// lane holds one query's scores and weights as the second product takes them:
// nothing moves between lanes but the maximum.  V lies in the cache with 16
// positions of an element together, which is that product's operand.
//
// attn_step_kernel: up to 16 query heads of one token; a wave reads K and V
// straight into the operands of 16 x 16 products.
// attn_run_kernel: 128 rows (a token's query heads of one key head are
// neighbours), a wave 32 of them in 32 x 32 products, K and V through LDS.
#pragma once

#include "attn.hpp"

namespace sn {
namespace k {

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// ------------------------------------------------------------------ operands
// 8 consecutive elements along the sum are one lane's operand: of one
// instruction in 16 bits, of eight in float32 (the sum's order does not matter as
// long as both operands have it).
template <typename T>
struct Frag;
template <>
struct Frag<bf16> {
  typedef bf16x8 type;
};
template <>
struct Frag<f16> {
  typedef f16x8 type;
};
template <>
struct Frag<float> {
  typedef f32x8 type;
};
__device__ __forceinline__ f32x4 mma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma16(f32x8 a, f32x8 b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ f32x16 mma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma32(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma32(f32x8 a, f32x8 b, f32x16 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

// 8 elements from any address that its elements allow.
template <typename E>
__device__ __forceinline__ V8<E> load8(const E* p) {
  V8<E> r;
  __builtin_memcpy(&r, p, sizeof(r));
  return r;
}
template <typename T>
__device__ __forceinline__ typename Frag<T>::type frag_of(const V8<T>& v) {
  return __builtin_bit_cast(typename Frag<T>::type, v);
}
// The integers that 8 codes are, exact in every type.
template <typename T>
__device__ __forceinline__ typename Frag<T>::type frag_of(const V8<int8_t>& v) {
  typename Frag<T>::type f;
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = (T)(float)v.v[j];
  return f;
}

// The larger of a lane's value and that of the lane 16 or 32 away; their sum.
__device__ __forceinline__ float max_x32(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
__device__ __forceinline__ float max_x16(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
__device__ __forceinline__ float sum_x32(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ __forceinline__ float sum_x16(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}

constexpr float kNone = -__builtin_huge_valf();  // a maximum of nothing
__device__ __forceinline__ float some(float m) { return m == kNone ? 0.f : m; }

// Whether this workgroup is the last of n at a counter, which it then clears.  What
// each has written before is seen by the last one afterwards.
__device__ __forceinline__ bool last_of(unsigned* count, unsigned n, int* shared) {
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    *shared = atomicAdd(count, 1u) + 1 == n;
    if (*shared) *count = 0;
  }
  __syncthreads();
  const bool last = *shared;
  if (last) __threadfence();
  return last;
}

// ------------------------------------------------------------------ single tokens
constexpr int kStepWaves = 4;
constexpr int kStepTarget = 512;  // workgroups that the keys of all sequences are spread over
constexpr int kStepLeast = 4;     // blocks of keys that a workgroup takes at least, one a wave
constexpr int kStepUnits = 1024;  // bound of the parts per head group (slots: twice as many)
template <typename T, bool I8, int DP>
constexpr int step_keys() {  // keys of a block that each quarter of a wave holds: K and V take up to 64 registers each
  return I8 || DP * sizeof(T) <= 256 ? 16 : 8;
}

// What one sequence has of keys in blocks of KB: none if there are none.
struct Span {
  int from, last;  // positions
  int block, blocks;
};
__device__ __forceinline__ Span step_span(const AttnArgs& a, int b, int KB) {
  const int past = a.c.past[b];
  Span s;
  s.from = a.window ? max(0, past - a.window + 1) : 0;
  s.last = min(past, (a.c.width << a.c.shift) - 1);
  s.block = s.from / KB;
  s.blocks = s.last < s.from ? 0 : s.last / KB - s.block + 1;
  return s;
}

// Which keys this workgroup takes.  The sequences' blocks, all together, are cut
// into parts of `per` blocks, about `units` of them, so that a batch of very
// different lengths is spread evenly with no length known to the host; every wave
// finds its workgroup's part by itself, 64 sequences at a time.
struct Part {
  int b, part, parts, slot, per;  // slot: this sequence's first place in the workspace
  Span s;
};
__device__ __forceinline__ bool step_part(const AttnArgs& a, int KB, int unit, Part& p) {
  const int lane = threadIdx.x & 63, seqs = a.c.seqs;
  int64_t total = 0;
  for (int base = 0; base < seqs; base += 64)
    if (base + lane < seqs) total += step_span(a, base + lane, KB).blocks;
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) total += __shfl_xor(total, i);
  const int per = (int)min<int64_t>(max<int64_t>((total + a.units - 1) / a.units, kStepLeast), 1 << 30);
  int before = 0;  // parts, and slots times 2^19, of the sequences before
  for (int base = 0; base < seqs; base += 64) {
    const int b = base + lane;
    const int n = b < seqs ? max(1, (step_span(a, b, KB).blocks + per - 1) / per) : 0;
    int sum = n + (n > 1 ? n << 19 : 0);
    const int own = sum;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
      const int up = __shfl_up(sum, i);
      if (lane >= i) sum += up;
    }
    const unsigned long long at = __ballot(unit < ((before + sum) & 0x7ffff));
    if (at) {
      const int l = __ffsll(at) - 1;
      p.b = base + l, p.parts = __shfl(n, l), p.per = per;
      const int first = __shfl(before + sum - own, l);
      p.part = unit - (first & 0x7ffff), p.slot = first >> 19;
      p.b = __builtin_amdgcn_readfirstlane(p.b), p.parts = __builtin_amdgcn_readfirstlane(p.parts);
      p.part = __builtin_amdgcn_readfirstlane(p.part), p.slot = __builtin_amdgcn_readfirstlane(p.slot);
      p.s = step_span(a, p.b, KB);
      return true;
    }
    before += __shfl(sum, 63);
  }
  return false;
}

template <typename T, bool I8, int DP, bool EXACT>
__global__ __launch_bounds__(64 * kStepWaves) void attn_step_kernel(AttnArgs a) {
  typedef typename std::conditional<I8, int8_t, T>::type E;                        // of the cache
  typedef typename std::conditional<I8 && sizeof(T) == 2, bf16, T>::type W;        // of the second product
  typedef typename Frag<T>::type FT;
  typedef typename Frag<W>::type FW;
  // Weights meet V in two parts of bf16 (16 bits; the range that weights with an
  // 8-bit row's scale in them may need), or once in f16, 2^14 times as large: only
  // weights below 2^-28 of the largest have fewer than 11 bits.
  constexpr bool SPLIT = std::is_same<W, bf16>::value;
  constexpr float LIFT = std::is_same<W, f16>::value ? 14.f : 0.f;
  constexpr int KPG = step_keys<T, I8, DP>(), KB = 4 * KPG, NT = KPG / 4, NU = KPG / 8, NS = DP / 32, ND = DP / 16;
  constexpr int OS = DP + 4;  // floats between the rows of `so`
  __shared__ float so[kStepWaves][16][OS], sm[kStepWaves][16], sl[kStepWaves][16];
  __shared__ int flag;
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
  const int D = EXACT ? DP : c.dim, head = blockIdx.y, each = a.heads / c.kv_heads;
  const int cols = min(16, each - (int)blockIdx.z * 16), qh = head * each + blockIdx.z * 16;
  Part p;
  if (!step_part(a, KB, blockIdx.x, p)) return;
  const int b = p.b;
  const int first = p.s.block + p.part * p.per, end = min(first + p.per, p.s.block + p.s.blocks);

  // this lane's keys: of K's rows 4 t + ..., of V 8 u + ...
  const int ko = KPG * (col >> 2), vo = KPG * g;
  const int kslot = (ko & 15) + (col & 3), vslot = vo & 15;
  const int mask = (1 << c.shift) - 1;
  auto page_at = [&](int block, int off) { return block < end ? page_of(c, b, block * KB + off) : -1; };

  FT q[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int d = 64 * (s >> 1) + 16 * g + 8 * (s & 1);
    V8<T> v = zero8<T>();
    if (col < cols && (EXACT || d < D)) v = load8(static_cast<const T*>(a.q) + b * a.qs + (int64_t)(qh + col) * D + d);
    q[s] = frag_of<T>(v);
    if (a.negative) q[s] = -q[s];
  }

  V8<E> kr[NT][NS], vr[ND][NU];
  float ks[I8 ? KPG : 1], vs[I8 ? KPG : 1];
  auto load_k = [&](int block, int page) {
    const int64_t row = ((((int64_t)max(page, 0) * c.kv_heads + head) << c.shift) + ((block * KB + (ko & ~15)) & mask) + kslot);
    const E* p0 = static_cast<const E*>(c.k) + row * D;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const int d = 64 * (s >> 1) + 16 * g + 8 * (s & 1);
        kr[t][s] = load8(p0 + (int64_t)(4 * t) * D + (EXACT || d < D ? d : 0));
      }
  };
  auto load_v = [&](int block, int page) {
    const int64_t row = ((((int64_t)max(page, 0) * c.kv_heads + head) << c.shift) + ((block * KB + (vo & ~15)) & mask));
    const E* p0 = static_cast<const E*>(c.v) + row * D + vslot;
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int u = 0; u < NU; ++u) vr[n][u] = load8(p0 + (EXACT ? 16 * n + col : min(16 * n + col, D - 1)) * 16 + 8 * u);
    if constexpr (I8) {
#pragma unroll
      for (int j = 0; j < KPG; j += 4) {
        __builtin_memcpy(&ks[j], c.ks + row + j, 16);
        __builtin_memcpy(&vs[j], c.vs + row + j, 16);
      }
    }
  };

  f32x4 o[ND];
#pragma unroll
  for (int n = 0; n < ND; ++n) o[n] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = kNone, l = 0.f;
  int block = first + wave;
  int kp = page_at(block, ko), vp = page_at(block, vo);
  int kp1 = page_at(block + kStepWaves, ko), vp1 = page_at(block + kStepWaves, vo);
  if (block < end) load_k(block, kp), load_v(block, vp);
  for (; block < end; block += kStepWaves) {
    const bool more = block + kStepWaves < end;
    f32x4 s[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        FT f = frag_of<T>(kr[t][i]);
        if constexpr (!EXACT)
          if (64 * (i >> 1) + 16 * g + 8 * (i & 1) >= D) f = FT{};
        s[t] = mma16(f, q[i], s[t]);
      }
    }
    if (more) load_k(block + kStepWaves, kp1);
    const int base = block * KB + vo;
    const bool there = vp >= 0;
    const bool full = block * KB >= p.s.from && block * KB + KB - 1 <= p.s.last && __all(there);
    float v[NT][4], top = kNone;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[t][i] = s[t][i] * (I8 ? ks[I8 ? 4 * t + i : 0] * a.scale2 : a.scale2);
    if (!full) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int pos = base + 4 * t + i;
          if (!there || pos < p.s.from || pos > p.s.last) v[t][i] = kNone;
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) top = fmaxf(top, v[t][i]);
    top = fmaxf(m, max_x32(max_x16(top)));
    if (__any(top > m)) {
      const float f = __builtin_amdgcn_exp2f(m - some(top));
      l *= f;
#pragma unroll
      for (int n = 0; n < ND; ++n) o[n] *= f;
      m = top;
    }
    const float ref = some(m) - LIFT;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[t][i] = __builtin_amdgcn_exp2f(v[t][i] - ref);
        l += v[t][i];
        if constexpr (I8) v[t][i] *= vs[4 * t + i];
      }
    if (!full) {  // what lies in places that are not seen takes no part, whatever it is
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int pos = base + 4 * t + i;
          if (!there || pos < p.s.from || pos > p.s.last) {
            v[t][i] = 0.f;
            if constexpr (!I8) {
#pragma unroll
              for (int n = 0; n < ND; ++n) vr[n][t >> 1].v[4 * (t & 1) + i] = (E)0.f;
            }
          }
        }
    }
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      FW hi, lo;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float w = v[2 * u + (j >> 2)][j & 3];
        hi[j] = (W)w;
        if constexpr (SPLIT) lo[j] = (W)(w - (float)hi[j]);
      }
#pragma unroll
      for (int n = 0; n < ND; ++n) {
        const FW f = frag_of<W>(vr[n][u]);
        o[n] = mma16(f, hi, o[n]);
        if constexpr (SPLIT) o[n] = mma16(f, lo, o[n]);
      }
    }
    kp = kp1, vp = vp1;
    if (more) load_v(block + kStepWaves, vp);
    kp1 = page_at(block + 2 * kStepWaves, ko), vp1 = page_at(block + 2 * kStepWaves, vo);
  }
  l = sum_x32(sum_x16(l));

  // the waves' results, together
  if (g == 0) sm[wave][col] = m, sl[wave][col] = l;
  if (col < cols)
#pragma unroll
    for (int n = 0; n < ND; ++n) *reinterpret_cast<f32x4*>(&so[wave][col][16 * n + 4 * g]) = o[n];
  __syncthreads();
  const int64_t slots = (int64_t)c.kv_heads * gridDim.z, at = (int64_t)head * gridDim.z + blockIdx.z;
  const int chunks = D / 4;
  float* wo = a.ws_o + ((p.slot + p.part) * slots + at) * 16 * DP;
  float* wm = a.ws_m + ((p.slot + p.part) * slots + at) * 32;
  for (int i = threadIdx.x; i < cols * chunks; i += 64 * kStepWaves) {
    const int r = i / chunks, d = 4 * (i - r * chunks);
    float top = kNone, sum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kStepWaves; ++w) top = fmaxf(top, sm[w][r]);
#pragma unroll
    for (int w = 0; w < kStepWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(sm[w][r] - some(top));
      sum += f * sl[w][r];
      acc += f * *reinterpret_cast<const f32x4*>(&so[w][r][d]);
    }
    if (p.parts == 1) {
      T* y = static_cast<T*>(a.y) + b * a.ys + (int64_t)(qh + r) * D + d;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      T t[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) t[j] = from_f<T>(acc[j] * inv);
      __builtin_memcpy(y, t, sizeof(t));
    } else {
      *reinterpret_cast<f32x4*>(wo + r * DP + d) = acc;
      if (d == 0) wm[r] = top, wm[16 + r] = sum;
    }
  }
  if (p.parts == 1) return;
  if (!last_of(a.count + p.slot * slots + at, p.parts, &flag)) return;
  // the last workgroup of a sequence joins its parts, in their order
  wo = a.ws_o + (p.slot * slots + at) * 16 * DP, wm = a.ws_m + (p.slot * slots + at) * 32;
  for (int i = threadIdx.x; i < cols * chunks; i += 64 * kStepWaves) {
    const int r = i / chunks, d = 4 * (i - r * chunks);
    float top = kNone, sum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < p.parts; ++k) top = fmaxf(top, wm[k * slots * 32 + r]);
    for (int k = 0; k < p.parts; ++k) {
      const float f = __builtin_amdgcn_exp2f(wm[k * slots * 32 + r] - some(top));
      sum += f * wm[k * slots * 32 + 16 + r];
      acc += f * *reinterpret_cast<const f32x4*>(wo + k * slots * 16 * DP + r * DP + d);
    }
    T* y = static_cast<T*>(a.y) + b * a.ys + (int64_t)(qh + r) * D + d;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T t[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) t[j] = from_f<T>(acc[j] * inv);
    __builtin_memcpy(y, t, sizeof(t));
  }
}

// ------------------------------------------------------------------ prompts
// A row of 8-bit values stands for code * s: its s goes as a power of two into the
// codes, which every type holds exactly (f16 from 2^-24 on), and the rest of it,
// 1 .. 2, into the weights, so that those are the only numbers that are rounded.
// The power is at most what a row of the type may have, so that codes stay numbers
// whatever lies where a scale that was never written would be.
template <typename T>
__device__ __forceinline__ float power_of(float s) {
  constexpr unsigned top = std::is_same<T, f16>::value ? 0x43800000u : 0x7b800000u;  // 2^8 (-128 lies in memory), 2^120
  return __builtin_bit_cast(float, min(max(__builtin_bit_cast(unsigned, s) & 0x7f800000u, 0x33800000u), top));
}
constexpr int kRunRows = 128;
constexpr int kRunParts = 512;  // workgroups that fewer tiles than half of it are split to
template <typename T>
constexpr int run_keys() {
  return sizeof(T) == 2 ? 64 : 32;
}

// The sequence and its tile of rows behind a number: tiles are counted over the sequences in order.
__device__ __forceinline__ bool run_tile(const CacheArgs& c, int each, int tile, int& b, int64_t& t, int64_t& first, int64_t& n) {
  const int lane = threadIdx.x & 63;
  int64_t before = 0;
  for (int base = 0; base < c.seqs; base += 64) {
    int64_t lo = 0, hi = 0;
    if (base + lane < c.seqs) seq_rows(c, base + lane, lo, hi);
    const int64_t own = ((hi - lo) * each + kRunRows - 1) / kRunRows;
    int64_t sum = own;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
      const int64_t up = __shfl_up(sum, i);
      if (lane >= i) sum += up;
    }
    const unsigned long long at = __ballot(tile < before + sum);
    if (at) {
      const int l = __ffsll(at) - 1;
      b = __builtin_amdgcn_readfirstlane(base + l);
      t = tile - __shfl(before + sum - own, l);
      first = __shfl(lo, l), n = __shfl(hi - lo, l);
      return true;
    }
    before += __shfl(sum, 63);
  }
  return false;
}

template <typename T, bool I8, int DP, bool EXACT>
__global__ __launch_bounds__(256, DP * sizeof(T) <= 256 ? 2 : 1) void attn_run_kernel(AttnArgs a) {
  typedef typename std::conditional<I8, int8_t, T>::type E;
  typedef typename Frag<T>::type F;
  constexpr int KB = run_keys<T>(), NK = KB / 32, NS = DP / 16, ND = DP / 32, NC = DP / 8, NL = KB * NC / 256;
  constexpr int KX = (NC < 16 ? NC : 16) - 1, VC = KB / 8, VX = VC - 1;
  // f16 weights are 2^6 times as large (2^14 at most, see kLazy)
  constexpr float LIFT = std::is_same<T, f16>::value ? 6.f : 0.f, kLazy = 8.f;
  __shared__ __attribute__((aligned(16))) T sk[2][KB * DP];
  __shared__ __attribute__((aligned(16))) T sv[2][KB * DP];
  __shared__ __attribute__((aligned(16))) float sks[2][I8 ? KB : 4], svs[2][I8 ? KB : 4];
  __shared__ int flag[2];
  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, h = lane >> 5;
  const int D = EXACT ? DP : c.dim, each = a.heads / c.kv_heads;
  // heads next to each other: workgroups of one head go to one XCD where 8 divides
  // their number.  The last tiles, which see the most keys, first.
  const int head = blockIdx.x % c.kv_heads, tiles = gridDim.x / c.kv_heads, tile = tiles - 1 - blockIdx.x / c.kv_heads;
  int b;
  int64_t t, row0, n;
  if (!run_tile(c, each, tile, b, t, row0, n)) return;
  const int past = min(c.past[b], kMaxPast);
  const int64_t rows = n * each, mine = t * kRunRows + 32 * wave + r;
  const int64_t rr = min(mine, rows - 1);  // rows behind the last one repeat it and are not stored
  const int token = (int)(rr / each), qh = head * each + (int)(rr - (int64_t)token * each);
  const int pos = past < 0 ? -1 : past + token;
  const int top_pos = __builtin_amdgcn_readlane(pos, 63), low_pos = __builtin_amdgcn_readfirstlane(pos);  // of the wave
  // the workgroup's keys, and this part's blocks of them
  const int64_t r0 = t * kRunRows, r1 = min(r0 + kRunRows, rows) - 1;
  const int pos0 = past < 0 ? -1 : past + (int)(r0 / each), pos1 = past < 0 ? -1 : past + (int)(r1 / each);
  const int from = a.window ? max(0, pos0 - a.window + 1) : 0, last = min(pos1, (c.width << c.shift) - 1);
  int first = from / KB, end = last < from ? first : last / KB + 1;
  if (gridDim.z > 1) {
    const int all = end - first, per = (all + gridDim.z - 1) / gridDim.z;
    first = min(end, first + (int)blockIdx.z * per), end = min(end, first + per);
  }
  const int mask = (1 << c.shift) - 1;

  F q[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int d = 16 * s + 8 * h;
    V8<T> v = zero8<T>();
    if (EXACT || d < D) v = load8(static_cast<const T*>(a.q) + (row0 + token) * a.qs + (int64_t)qh * D + d);
    q[s] = frag_of<T>(v);
    if (a.negative) q[s] = -q[s];
  }

  // lane i holds the page of the i-th 16 positions of a block
  auto pages_at = [&](int block) { return lane < KB / 16 && block < end ? page_of(c, b, block * KB + 16 * lane) : -1; };
  V8<E> kr[NL], vr[NL];
  float ksr = 0.f, vsr = 0.f, vpw[I8 ? NL : 1][8];
  auto load = [&](int block, int pages) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int x = tid + 256 * i;
      {
        const int key = x / NC, d = 8 * (x % NC), t16 = __builtin_amdgcn_readfirstlane(key / 16);
        const int page = max(0, __builtin_amdgcn_readlane(pages, t16));
        const E* p = static_cast<const E*>(c.k) +
                     ((((int64_t)page * c.kv_heads + head) << c.shift) + ((block * KB + 16 * t16) & mask)) * D;
        kr[i] = load8(p + (key & 15) * D + (EXACT || d < D ? d : 0));
      }
      {
        const int t16 = __builtin_amdgcn_readfirstlane(x / (2 * DP)), e = x % (2 * DP);
        const int page = max(0, __builtin_amdgcn_readlane(pages, t16));
        const int64_t at = (((int64_t)page * c.kv_heads + head) << c.shift) + ((block * KB + 16 * t16) & mask);
        vr[i] = load8(static_cast<const E*>(c.v) + at * D + (EXACT ? 8 * e : 8 * min(e, 2 * D - 1)));
        if constexpr (I8) __builtin_memcpy(vpw[i], c.vs + at + 8 * (e & 1), 32);
      }
    }
    if constexpr (I8)
      if (tid < KB) {
        const int page = max(0, __shfl(pages, tid / 16));
        const int64_t at = (((int64_t)page * c.kv_heads + head) << c.shift) + ((block * KB + tid) & mask);
        ksr = c.ks[at], vsr = c.vs[at];
      }
  };
  // Into LDS: K [key][element], V [element][key], the chunks of 8 of a row in an order
  // of the row's own, so that 8 lanes that read one chunk of 8 rows meet no bank twice.
  auto store = [&](int buf, int block, bool edge) {
    bool odd = false;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int x = tid + 256 * i;
      {
        const int key = x / NC, ch = x % NC;
        F f = frag_of<T>(kr[i]);
        if constexpr (!EXACT)
          if (8 * ch >= D) f = F{};
        *reinterpret_cast<F*>(&sk[buf][(key * NC + (ch ^ (key & KX))) * 8]) = f;
      }
      {
        const int t16 = x / (2 * DP), e = x % (2 * DP), d = e >> 1, ch = 2 * t16 + (e & 1);
        F f;
        if constexpr (I8) {
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = (T)((float)vr[i].v[j] * power_of<T>(vpw[i][j]));
        } else {
          f = frag_of<T>(vr[i]);
          if (edge && (EXACT || d < D))
#pragma unroll
            for (int j = 0; j < 8; ++j) odd = odd || !__builtin_isfinite((float)f[j]);
        }
        *reinterpret_cast<F*>(&sv[buf][(d * VC + (ch ^ (d & VX))) * 8]) = f;
      }
    }
    if constexpr (I8)
      if (tid < KB) sks[buf][tid] = ksr * a.scale2, svs[buf][tid] = vsr / power_of<T>(vsr);
    if (!I8 && edge && __any(odd) && lane == 0) flag[buf] = block + 1;  // (a block's own number: none is ever cleared)
  };
  // Whether every row of the workgroup sees every key of a block.
  auto edge_of = [&](int block, int pages) {
    return block * KB + KB - 1 > pos0 || (a.window && block * KB < pos1 - a.window + 1) ||
           __builtin_popcountll(__ballot(pages >= 0)) < KB / 16;
  };

  f32x16 o[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
  float m = kNone, l = 0.f;
  int pages = pages_at(first), pages1 = pages_at(first + 1);
  if (tid < 2) flag[tid] = 0;
  bool edge = edge_of(first, pages);
  if (first < end) {
    load(first, pages);
    __syncthreads();
    store(0, first, edge);
  }
  __syncthreads();
  for (int block = first; block < end; ++block) {
    const int buf = (block - first) & 1;
    const bool more = block + 1 < end;
    if (more) load(block + 1, pages1);
    const int pages2 = pages_at(block + 2);
    const bool odd = !I8 && edge && flag[buf] == block + 1;
    // (a wave whose rows see none of the block has nothing to do)
    if (block * KB <= top_pos && !(a.window && block * KB + KB - 1 < low_pos - a.window + 1)) {
      f32x16 s[NK];
#pragma unroll
      for (int i = 0; i < NK; ++i) {
#pragma unroll
        for (int j = 0; j < 16; ++j) s[i][j] = 0.f;
        // row r of the product is key r with bits 2 and 3 exchanged: a lane's 8
        // scores in a row are then those of 8 keys in a row
        const int key = 32 * i + ((r & 19) | ((r & 4) << 1) | ((r & 8) >> 1));
#pragma unroll
        for (int j = 0; j < NS; ++j)
          s[i] = mma32(*reinterpret_cast<const F*>(&sk[buf][(key * NC + ((2 * j + h) ^ (key & KX))) * 8]), q[j], s[i]);
      }
      if constexpr (I8) {
#pragma unroll
        for (int i = 0; i < NK; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) s[i][j] *= sks[buf][32 * i + 16 * (j >> 3) + 8 * h + (j & 7)];
      }
      if (edge) {
        const unsigned long long there = __ballot(pages >= 0);
#pragma unroll
        for (int i = 0; i < NK; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const int key = 32 * i + 16 * (j >> 3) + 8 * h + (j & 7), kpos = block * KB + key;
            const bool see = kpos <= pos && (!a.window || kpos > pos - a.window) && (there >> (2 * i + (j >> 3)) & 1);
            s[i][j] = see ? s[i][j] : kNone;
          }
      }
      const float mul = I8 ? 1.f : a.scale2;
      float top = kNone;
#pragma unroll
      for (int i = 0; i < NK; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) top = fmaxf(top, s[i][j]);
      top = max_x32(top) * mul;
      // the maximum moves only when it grew by 2^kLazy: sums stay far from their type's
      // ends (each row by itself: no row's result depends on its neighbours)
      if (__any(top > m + kLazy)) {
        const float now = top > m + kLazy ? top : m, f = __builtin_amdgcn_exp2f(m - some(now));
        l *= f;
#pragma unroll
        for (int i = 0; i < ND; ++i) o[i] *= f;
        m = now;
      }
      const float ref = LIFT - some(m);
#pragma unroll
      for (int i = 0; i < NK; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          s[i][j] = __builtin_amdgcn_exp2f(fmaf(s[i][j], mul, ref));
          l += s[i][j];
        }
      if constexpr (I8) {
#pragma unroll
        for (int i = 0; i < NK; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const float w = s[i][j] * svs[buf][32 * i + 16 * (j >> 3) + 8 * h + (j & 7)];
            s[i][j] = edge && s[i][j] == 0.f ? 0.f : w;  // (the scale of a place that is not seen may be NaN)
          }
      }
      if (I8 || !odd) {
#pragma unroll
        for (int kk = 0; kk < KB / 16; ++kk) {
          F w;
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] = (T)s[kk >> 1][8 * (kk & 1) + j];
#pragma unroll
          for (int i = 0; i < ND; ++i) {
            const int d = 32 * i + r;
            o[i] = mma32(*reinterpret_cast<const F*>(&sv[buf][(d * VC + ((2 * kk + h) ^ (d & VX))) * 8]), w, o[i]);
          }
        }
      } else {
        // A value that is not finite lies in a block that not every row sees whole
        // (0 times it would be NaN): the finite ones as ever, and the weights that
        // the others have, whose signs say what becomes of the sums.
        F w[KB / 16];
#pragma unroll
        for (int kk = 0; kk < KB / 16; ++kk)
#pragma unroll
          for (int j = 0; j < 8; ++j) w[kk][j] = (T)s[kk >> 1][8 * (kk & 1) + j];
#pragma unroll
        for (int i = 0; i < ND; ++i) {
          const int d = 32 * i + r;
          f32x16 up, down;
#pragma unroll
          for (int j = 0; j < 16; ++j) up[j] = down[j] = 0.f;
#pragma unroll
          for (int kk = 0; kk < KB / 16; ++kk) {
            const F v = *reinterpret_cast<const F*>(&sv[buf][(d * VC + ((2 * kk + h) ^ (d & VX))) * 8]);
            F fine, plus, minus;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const float x = (float)v[j];
              fine[j] = __builtin_isfinite(x) ? v[j] : (T)0.f;
              plus[j] = __builtin_isfinite(x) || x < 0.f ? (T)0.f : (T)1.f;
              minus[j] = __builtin_isfinite(x) || x > 0.f ? (T)0.f : (T)1.f;
            }
            o[i] = mma32(fine, w[kk], o[i]), up = mma32(plus, w[kk], up), down = mma32(minus, w[kk], down);
          }
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            if (up[j] > 0.f) o[i][j] += __builtin_huge_valf();
            if (down[j] > 0.f) o[i][j] -= __builtin_huge_valf();
          }
        }
      }
    }
    edge = edge_of(block + 1, pages1);
    pages = pages1, pages1 = pages2;
    if (more) store(buf ^ 1, block + 1, edge);
    __syncthreads();
  }
  l = sum_x32(l);

  if (gridDim.z > 1) {
    // parts: left in the lanes' order, joined by the tile's last workgroup in the parts' order
    const int64_t slot = (int64_t)blockIdx.x * gridDim.z;
    f32x4* wo = reinterpret_cast<f32x4*>(a.ws_o) + slot * (kRunRows * DP / 4) + tid;
    float* wm = a.ws_m + slot * (2 * 256) + tid;
    {
      f32x4* w0 = wo + blockIdx.z * (kRunRows * DP / 4);
#pragma unroll
      for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) w0[(4 * i + j) * 256] = f32x4{o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]};
      wm[blockIdx.z * 512] = m, wm[blockIdx.z * 512 + 256] = l;
    }
    if (!last_of(a.count + blockIdx.x, gridDim.z, &flag[0])) return;
    m = kNone;
    for (int z = 0; z < (int)gridDim.z; ++z) m = fmaxf(m, wm[z * 512]);
    l = 0.f;
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    for (int z = 0; z < (int)gridDim.z; ++z) {
      const float f = __builtin_amdgcn_exp2f(wm[z * 512] - some(m));
      l += f * wm[z * 512 + 256];
#pragma unroll
      for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 v = wo[z * (kRunRows * DP / 4) + (4 * i + j) * 256];
#pragma unroll
          for (int x = 0; x < 4; ++x) o[i][4 * j + x] += f * v[x];
        }
    }
  }
  if (mine >= rows) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* y = static_cast<T*>(a.y) + (row0 + token) * a.ys + (int64_t)qh * D;
#pragma unroll
  for (int i = 0; i < ND; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d = 32 * i + 8 * j + 4 * h;
      T v[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) v[x] = from_f<T>(o[i][4 * j + x] * inv);
      if (EXACT || d < D) __builtin_memcpy(y + d, v, sizeof(v));
    }
}

// ------------------------------------------------------------------ launches
template <typename T, bool I8, int DP, bool EXACT>
static void launch_step(AttnArgs& a, hipStream_t st) {
  const CacheArgs& c = a.c;
  constexpr int KB = 4 * step_keys<T, I8, DP>();
  const int each = a.heads / c.kv_heads, groups = (each + 15) / 16;
  const int64_t most = ((int64_t)c.width << c.shift) / KB + 1;  // blocks of one sequence
  a.units = (int)std::min<int64_t>(kStepUnits, (kStepTarget + (int64_t)c.kv_heads * groups - 1) / ((int64_t)c.kv_heads * groups));
  const int64_t parts = std::min<int64_t>(a.units + (int64_t)c.seqs, c.seqs * ((most + kStepLeast - 1) / kStepLeast));
  SN_LAUNCH((attn_step_kernel<T, I8, DP, EXACT>), dim3((unsigned)parts, c.kv_heads, groups), dim3(64 * kStepWaves), 0, st, a);
}

template <typename T, bool I8, int DP, bool EXACT>
static void launch_run(AttnArgs& a, hipStream_t st) {
  const CacheArgs& c = a.c;
  constexpr int KB = run_keys<T>();
  const int64_t wgs = attn_run_tiles(a) * c.kv_heads, blocks = (((int64_t)c.width << c.shift) + KB - 1) / KB;
  int64_t parts = 1;
  if (2 * wgs <= kRunParts) parts = std::max<int64_t>(1, std::min<int64_t>((kRunParts + wgs - 1) / wgs, blocks / 4));
  SN_LAUNCH((attn_run_kernel<T, I8, DP, EXACT>), dim3((unsigned)wgs, 1, (unsigned)parts), dim3(256), 0, st, a);
}

template <typename T>
static void launch_attention(AttnArgs& a, bool step, hipStream_t st) {
  auto sized = [&](auto i8, auto dp) {
    constexpr bool I8 = decltype(i8)::value;
    constexpr int DP = decltype(dp)::value;
    if (step) a.c.dim == DP ? launch_step<T, I8, DP, true>(a, st) : launch_step<T, I8, DP, false>(a, st);
    else a.c.dim == DP ? launch_run<T, I8, DP, true>(a, st) : launch_run<T, I8, DP, false>(a, st);
  };
  auto stored = [&](auto i8) {
    if (a.c.dim <= 64) sized(i8, std::integral_constant<int, 64>());
    else if (a.c.dim <= 128) sized(i8, std::integral_constant<int, 128>());
    else sized(i8, std::integral_constant<int, 256>());
  };
  if (a.c.i8) stored(std::true_type());
  else stored(std::false_type());
}

}  // namespace k
}  // namespace sn
