// Attention over the paged cache: row i of sequence b stands at position p =
// past[b] + i and its query heads see the positions max(0, p - window + 1) .. p:
// y = sum exp(scale q k) v / sum exp(scale q k), in one pass over the keys with
// a running maximum.  Both kernels compute S^T = K Q^T and O^T = V^T P^T, so that a
// lane holds one query's scores and weights as the second product takes them:
// nothing moves between lanes but the maximum.  V lies in the cache with 16
// positions of an element together, which is that product's operand.
//
// Scores, maxima, sums and outputs are float32; what is rounded besides the result are the
// weights: in f16 to 11 bits, lifted by a power of two (LIFT) so that small ones stay normal numbers;
// in bf16 by the step kernel to two bf16 parts, 16 bits, by the run kernel to one, 8 bits,
// as large as a rounding of bf16 values themselves.  (The float32 sum l takes them unrounded.)
//
// attn_step_kernel: up to 16 query heads of one token; a wave reads K and V
// straight into the operands of 16 x 16 products, since every key is used once and LDS
// would only be a detour.  Bound by the cache's bytes: 64 sequences of 2048 keys, 8 key heads of
// 128 in bf16 101 us, 5.3 TB/s; up to 8192 keys 197 us, 5.4 TB/s; 32 heads without
// groups 6.3 TB/s; in 8 bits, ragged to 8192 keys, 110 - 119 us, 4.6 - 5.0 TB/s, where vector
// instructions, codes turned into numbers first, take 44 % of the cycles.  64 of 2048 keys in
// float32 191 us; over 8 bits in f16 48, in float32 96.  Short ones are a chain of dependent steps:
// one sequence of 4096 keys 11.2 us, of which launch and plan some 3.2, queries and table 0.7, the
// keys 3.0, joining the waves 0.7, storing the part and counting it 1.7, joining the parts 2.3 and
// looking whether results are finite 0.3.  (Float32 of 136 to 248 elements spills 9 registers.)
// attn_run_kernel: 128 rows (a token's query heads of one key head are
// neighbours), a wave 32 of them in 32 x 32 products, K and V through LDS, where the
// four waves share them.  Bound by issue, of matrix products and of the softmax: 4096 rows of 32
// heads, 8 key heads of 128 in bf16, causal, 145 - 153 us, 137.5 GFLOP that count, 900 - 950
// TFLOP/s, a library product of 8192^3 1206.  Of the cycles of busy compute units the matrix pipes
// take 48 %, vector instructions (which start the products, too) 50, LDS 6, without a bank conflict;
// without its loads it takes 138 us, without its exponentials 139: two waves a SIMD, whose registers
// hold no more, cover one's softmax with the other's products in part.  Over a cache in 8 bits 180 -
// 187 us (f16 192 - 197): vector instructions 64 % of the cycles, products 35.
// Not faster (4096 rows, 162 us then): 32 keys a block and three waves a SIMD 171, a block's scores
// taken beside the last one's softmax 180, a queue of tiles 192, tiles in another order 174.
// Float32 goes through float32 products: 2048 rows 383 us, 90 TFLOP/s, the library's 154; over 8 bits 409.
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
  if constexpr (std::is_same<T, f16>::value) {
    // code + 128 as the last bits of 1024 .. 2047, whose step is 1; two at a time (4096 rows 218 -> 206 us)
    typedef f16 f16x2 __attribute__((ext_vector_type(2)));
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 w = __builtin_bit_cast(u32x2, v) ^ 0x80808080u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned two = __builtin_amdgcn_perm(0x64646464u, w[j >> 1], j & 1 ? 0x04030402u : 0x04010400u);
      const f16x2 c = __builtin_bit_cast(f16x2, two) - (f16)1152.f;
      f[2 * j] = c[0], f[2 * j + 1] = c[1];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (T)(float)v.v[j];
  }
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

// Values that are not finite.  A weight exp(..) is above zero however small it is, so an infinity that a
// row sees is its result's, and a NaN, or infinities of both signs, are NaN.  In float32 a weight may be
// 0, whose product with an infinity is NaN, as may be that of two parts of a weight; which it is would
// depend on where blocks, parts and tiles end.  So the products only say that there is something (a
// sum that is not finite stays so to the end), and whoever writes such a result looks through the
// values again: its class is that of the values that the row sees, whatever their weights, if those
// are numbers.  (Values in 8 bits have no infinities: a row that held one has a NaN for a scale.)
// The looking is in functions of its own, which read the kernel's arguments anew: inlined, its
// scalars cost the loops registers (4096 rows 147 -> 161 us, one token after 4095 10.9 -> 11.6).
typedef const __attribute__((address_space(4))) AttnArgs* KernelArgs;
__device__ __forceinline__ bool finite(float v) { return fabsf(v) < __builtin_huge_valf(); }
__device__ __forceinline__ float class_of(bool plus, bool minus) {  // NaN counts as both
  return (plus ? __builtin_huge_valf() : 0.f) - (minus ? __builtin_huge_valf() : 0.f);
}
// The class of element d of the values at the positions from .. last; 0 where all are finite.
template <typename T>
__device__ __attribute__((noinline)) float class_of_values(KernelArgs args, int b, int head, int d, int from, int last) {
  const CacheArgs c = ((const AttnArgs*)args)->c;
  bool plus = false, minus = false;
#pragma unroll 1
  for (int p = from & ~7; p <= last && !(plus && minus); p += 8) {
    const int page = page_of(c, b, p);
    if (page < 0) continue;
    const V8<T> v = load8(static_cast<const T*>(c.v) + v_at(c, page, head, p & ((1 << c.shift) - 1)) + 16 * d);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float f = to_f(v.v[j]);
      if (p + j >= from && p + j <= last && !finite(f)) plus |= !(f < 0.f), minus |= !(f > 0.f);
    }
  }
  return class_of(plus, minus);
}
// Whether there is a place at any of the positions from .. last.  A sum of weights is 0 where none is seen, and the
// result zeros, or where all scores that are seen are minus infinity: 0 / 0.
__device__ __forceinline__ bool sees_place(const CacheArgs& c, int b, int from, int last) {
#pragma unroll 1
  for (int p = from; p <= last; p = (p | ((1 << c.shift) - 1)) + 1)
    if (page_of(c, b, p) >= 0) return true;
  return false;
}
static __device__ __attribute__((noinline)) float inverse_of_0(KernelArgs args, int b, int from, int last) {
  const CacheArgs c = ((const AttnArgs*)args)->c;
  return sees_place(c, b, from, last) ? __builtin_nanf("") : 0.f;
}
// Which of the 32 keys from `base` on a row at `pos` sees.
__device__ __forceinline__ unsigned first_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }
__device__ __forceinline__ unsigned seen_keys(int base, int pos, int window) {
  return first_bits(pos - base + 1) & ~first_bits(window ? pos - window + 1 - base : 0);
}

// Parts of a sum that other workgroups read: stores and loads of the workspace go past
// the XCDs' own L2 caches (cache policy sc1), a workgroup's stores are complete
// before it counts itself in, so that no cache-wide fence is needed (with fences: 157
// us instead of 30 for 700 workgroups).
constexpr int kCoherent = 16;
struct Shared {
  __amdgpu_buffer_rsrc_t r;
  __device__ __forceinline__ Shared(const float* p) : r(make_rsrc(p, 0x7fffffff)) {}
  __device__ __forceinline__ void put4(int at, f32x4 v) const {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), r, 4 * at, 0, kCoherent);
  }
  __device__ __forceinline__ void put(int at, float v) const {
    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), r, 4 * at, 0, kCoherent);
  }
  __device__ __forceinline__ f32x4 get4(int at) const {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, 4 * at, 0, kCoherent));
  }
  __device__ __forceinline__ float get(int at) const {
    return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, 4 * at, 0, kCoherent));
  }
};
// Whether this workgroup is the last of n at a counter, which it then clears.
__device__ __forceinline__ bool last_of(unsigned* count, unsigned n, int* shared) {
  wait_vmcnt<0>();
  __syncthreads();
  if (threadIdx.x == 0) {
    *shared = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == n;
    if (*shared) __hip_atomic_exchange(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return *shared;
}

// Parts joined in their order, eight at a time, all of whose numbers are in flight.
struct Join {
  float ms[8], ls[8], top = kNone, sum = 0.f;
  f32x4 os[8], acc = {0.f, 0.f, 0.f, 0.f};
  template <typename Get>
  __device__ __forceinline__ void fetch(int first, int last, Get get) {
#pragma unroll
    for (int k = 0; k < 8; ++k) get(min(first + k, last), ms[k], ls[k], os[k]);
  }
  __device__ __forceinline__ void add(int first, int last) {
    float now = top;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (first + k > last) ms[k] = kNone;
      now = fmaxf(now, ms[k]);
    }
    const float f = __builtin_amdgcn_exp2f(top - some(now));
    sum *= f, acc *= f, top = now;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float w = __builtin_amdgcn_exp2f(ms[k] - some(now));
      if (first + k <= last) sum += w * ls[k], acc += w * os[k];
    }
  }
};

// ------------------------------------------------------------------ single tokens
constexpr int kStepWaves = 4;
// Blocks of keys of a workgroup where there are workgroups enough: one a wave.  (One sequence of 4096
// keys 11.2 us, with 2 blocks 13.2, with 8 11.9; 8 of 2048 16.5, 16.8, 19.9.)
constexpr int kStepLeast = 4;
constexpr int kStepUnits = 1024;  // bound of the workgroups per group of heads
// Workgroups that the keys of all sequences are spread over: one a compute unit, two
// where codes are turned into numbers.  (64 sequences of up to 8192 keys, 8 key heads of
// 128, in bf16 198 us with 256 and 204 with 512, in 8 bits 128 and 120; one of
// 32768 keys in bf16 29 and 33.5: fewer parts to join.)
// Two also where the tables say that each sequence can have some of its own (64 of 128 keys 9
// us, by parts of two sequences 11); more that end at once would put the others
// two on some units and none on others (64 of 2048 keys: 127 us, without them 101).
inline int step_units(const AttnArgs& a, int target) {
  const int64_t groups = (int64_t)a.c.kv_heads * ((a.heads / a.c.kv_heads + 15) / 16);
  return (int)std::min<int64_t>(kStepUnits, (target + groups - 1) / groups);
}
template <typename T, bool I8, int DP>
constexpr int step_keys() {  // keys of a block that each quarter of a wave holds: K and V take up to 64 registers each
  return I8 || DP * sizeof(T) <= 256 ? 16 : 8;
}

// What one sequence has of keys in blocks of KB; one block, of which nothing is seen, at least.
struct Span {
  int from, last;  // positions
  int block, blocks;
};
__device__ __forceinline__ Span step_span(const AttnArgs& a, int past, int KB) {
  Span s;
  s.from = a.window && past >= a.window ? past - a.window + 1 : 0;
  s.last = min(past, (a.c.width << a.c.shift) - 1);
  s.block = s.from / KB;
  s.blocks = s.last < s.from ? 1 : s.last / KB - s.block + 1;
  return s;
}

// Which keys this workgroup takes.  The blocks of all sequences stand in one row, which is
// cut into equal parts, so that a batch of very different lengths is spread evenly with no
// length known to the host; a part may begin and end inside sequences and hold
// several.  Where there are workgroups enough, each sequence begins a part of its own.
// Every wave finds its workgroup's part by itself, 64 sequences at a time.
struct Part {
  int per, begin, end;  // blocks of a part; this one's
  int pad;              // a sequence counts as a multiple of pad + 1 blocks
  int b, start, past;   // the sequence that it begins in, where that begins, and its positions
};
__device__ __forceinline__ bool step_part(const AttnArgs& a, int KB, int unit, Part& p) {
  const int lane = threadIdx.x & 63, seqs = a.c.seqs;
  int total = 0, padded = 0, own = 0, past = -1;
  for (int base = 0; base < seqs; base += 64) {
    past = a.c.past[min(base + lane, seqs - 1)];
    own = base + lane < seqs ? step_span(a, past, KB).blocks : 0;
    total += own, padded += (own + kStepLeast - 1) & -kStepLeast;
  }
  total = lane_of((int)scan_lanes(total), 63), padded = lane_of((int)scan_lanes(padded), 63);
  p.pad = 0, p.per = (total + a.units - 1) / a.units;
  if (padded <= kStepLeast * a.units) p.pad = kStepLeast - 1, p.per = kStepLeast, total = padded;
  p.begin = unit * p.per, p.end = min(p.begin + p.per, total);
  if (p.begin >= total) return false;
  int before = 0;
  for (int base = 0; base < seqs; base += 64) {
    if (seqs > 64) {
      past = a.c.past[min(base + lane, seqs - 1)];
      own = base + lane < seqs ? step_span(a, past, KB).blocks : 0;
    }
    const int n = (own + p.pad) & ~p.pad;
    const int sum = (int)scan_lanes(n);
    const unsigned long long at = __ballot(p.begin < before + sum);
    if (at) {
      const int l = __ffsll(at) - 1;
      p.b = base + l, p.start = before + lane_of(sum - n, l), p.past = lane_of(past, l);
      return true;
    }
    before += lane_of(sum, 63);
  }
  return false;
}

// (The least waves of the launch bounds keep 128 bf16 elements, at 257 registers, on two workgroups a unit.)
template <typename T, bool I8, int DP, bool EXACT>
__global__ __launch_bounds__(64 * kStepWaves, EXACT && DP <= 128 ? 2 : 1) void attn_step_kernel(AttnArgs a) {
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
  const int unit = blockIdx.x;
  Part p;
  if (!step_part(a, KB, unit, p)) return;

  // this lane's keys: of K's rows 4 t + ..., of V 8 u + ...
  const int ko = KPG * (col >> 2), vo = KPG * g;
  const int kslot = (ko & 15) + (col & 3), vslot = vo & 15;
  const int mask = (1 << c.shift) - 1;
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

  // the sequences, or parts of them, that this workgroup's blocks belong to
  for (;;) {
  const int b = p.b;
  const Span span = step_span(a, p.past, KB);
  // (without a page there is nothing to read, not even where nothing is seen)
  const int first = span.block + max(p.begin - p.start, 0), end = c.pages ? span.block + min(p.end - p.start, span.blocks) : 0;
  auto page_at = [&](int block, int off) { return block < end ? page_of(c, b, block * KB + off) : -1; };
  FT q[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int d = 64 * (s >> 1) + 16 * g + 8 * (s & 1);
    // (behind no branch, whose join would wait; columns without a head repeat the last one and are not stored)
    q[s] = frag_of<T>(load8(static_cast<const T*>(a.q) + b * a.qs + (int64_t)(qh + min(col, cols - 1)) * D + (EXACT || d < D ? d : 0)));
  }

  if constexpr (!EXACT) {
#pragma unroll
    for (int s = 0; s < NS; ++s)
      if (64 * (s >> 1) + 16 * g + 8 * (s & 1) >= D) q[s] = FT{};
  }
  const float scale = a.negative ? -a.scale2 : a.scale2;

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
    const bool full = block * KB >= span.from && block * KB + KB - 1 <= span.last && __all(there);
    float v[NT][4], top = kNone;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[t][i] = s[t][i] * (I8 ? ks[I8 ? 4 * t + i : 0] * scale : scale);
    if (!full) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int pos = base + 4 * t + i;
          if (!there || pos < span.from || pos > span.last) v[t][i] = kNone;
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
          if (!there || pos < span.from || pos > span.last) {
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
  if (p.start > p.begin) __syncthreads();  // (the last sequence's are read)
  if (g == 0) sm[wave][col] = m, sl[wave][col] = l;
  if (col < cols)
#pragma unroll
    for (int n = 0; n < ND; ++n) *reinterpret_cast<f32x4*>(&so[wave][col][16 * n + 4 * g]) = o[n];
  __syncthreads();
  // A sequence in several workgroups, unit0 .. unit1: each leaves its part in a slot, of
  // which it has one for a sequence that began before it and one for a sequence that
  // goes on behind it; the last one joins them, in their order.
  const int unit0 = p.start / p.per, unit1 = (p.start + span.blocks - 1) / p.per;
  const int slots = c.kv_heads * gridDim.z, at = head * gridDim.z + blockIdx.z;
  const Shared wo(a.ws_o), wm(a.ws_m);
  auto slot = [&](int u) { return (u == unit0 ? 2 * u + 1 : 2 * u) * slots + at; };
  constexpr int chunks = DP / 4;
  auto finish = [&](int r, int d, f32x4 acc, float sum) {
    float inv = 1.f / sum;
    if (sum == 0.f) inv = inverse_of_0((KernelArgs)__builtin_amdgcn_kernarg_segment_ptr(), b, span.from, span.last);
    if (!I8 && sum > 0.f && finite(sum) && !finite((acc[0] + acc[1]) + (acc[2] + acc[3])))
#pragma unroll 1
      for (int j = 0; j < 4; ++j) {
        const float is = class_of_values<T>((KernelArgs)__builtin_amdgcn_kernarg_segment_ptr(), b, head, d + j, span.from, span.last);
        if (is != 0.f) acc = f32x4{j == 0 ? is : acc[0], j == 1 ? is : acc[1], j == 2 ? is : acc[2], j == 3 ? is : acc[3]};
      }
    T v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = from_f<T>(acc[j] * inv);
    __builtin_memcpy(static_cast<T*>(a.y) + b * a.ys + (int64_t)(qh + r) * D + d, v, sizeof(v));
  };
  for (int i = threadIdx.x; i < cols * chunks; i += 64 * kStepWaves) {
    const int r = i / chunks, d = 4 * (i % chunks);
    if (!EXACT && d >= D) continue;
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
    if (unit0 == unit1) {
      finish(r, d, acc, sum);
    } else {
      wo.put4(slot(unit) * (16 * DP) + r * DP + d, acc);
      if (d == 0) wm.put(slot(unit) * 32 + r, top), wm.put(slot(unit) * 32 + 16 + r, sum);
    }
  }
  if (unit0 != unit1 && last_of(a.count + slot(unit0), unit1 - unit0 + 1, &flag)) {
    for (int i = threadIdx.x; i < cols * chunks; i += 64 * kStepWaves) {
      const int r = i / chunks, d = 4 * (i % chunks);
      if (!EXACT && d >= D) continue;
      Join parts;
      for (int u = unit0; u <= unit1; u += 8) {
        parts.fetch(u, unit1, [&](int from, float& ms, float& ls, f32x4& os) {
          const int at = slot(from);
          ms = wm.get(at * 32 + r), ls = wm.get(at * 32 + 16 + r), os = wo.get4(at * (16 * DP) + r * DP + d);
        });
        parts.add(u, unit1);
      }
      finish(r, d, parts.acc, parts.sum);
    }
  }
  p.start += (span.blocks + p.pad) & ~p.pad, ++p.b;
  if (p.start >= p.end) return;
  p.past = uniform(c.past[p.b]);
  }
}

// ------------------------------------------------------------------ prompts
// f16 weights of 8-bit rows, which stand for code * s: s goes as a power of two into the
// codes, which f16 holds exactly from 2^-24 on, and the rest of it, 1 .. 2, into the weights,
// so that those are the only numbers that are rounded, and in range.  (bf16 has the range for
// all of s in the weights.)  The power is at most a row's of f16 values, so that codes stay numbers whatever lies
// in a place that was never written, -128 with any scale.
__device__ __forceinline__ float power_of(float s) {
  return __builtin_bit_cast(float, min(max(__builtin_bit_cast(unsigned, s) & 0x7f800000u, 0x33800000u), 0x43800000u));  // 2^-24 .. 2^8
}
constexpr int kRunRows = 128;
// Workgroups that tiles are split to, along the keys, where they are no more than half of it: two a compute
// unit, as many as run at once.  (256 rows after 8192 keys, 8 key heads, 8 parts each: 59 us in bf16, 70 in 8 bits;
// to 256 workgroups 68 and 95, to 1024 73 and 81.)
constexpr int kRunParts = 512;
// How many parts a tile has: of four blocks each at least (512 rows, 8 blocks: 2 parts 17.9 us, 4
// parts 22.6; 16 rows after 8192 keys, 129 blocks: 32 parts 19.9, 16 parts 22.0, 64 parts 22.8).
inline int run_parts(int64_t blocks, int64_t wgs) {
  if (2 * wgs > kRunParts) return 1;
  return (int)std::max<int64_t>(1, std::min((kRunParts + wgs - 1) / wgs, blocks / 4));
}
// Few parts are joined by their tile's last workgroup, at 0.7 us a part, beside other tiles' work;
// many by a launch of their own, about 6 us.  (2 parts 17.6 us by the last workgroup, 20.1 by a launch; 4
// parts 22.2 and 24.3; 8 parts 58.2 and 53.0; 32 parts 35 and 19.7.)  Above 128 elements always by
// a launch: the registers of the other way cost every call there (4096 rows of 256 elements 222 and 195 us).
template <int DP>
constexpr bool run_joins(int parts) {
  return DP > 128 || parts >= 8;
}
template <typename T>
constexpr int run_keys() {
  return sizeof(T) == 2 ? 64 : 32;
}

// LDS direct load: 16 bytes a lane from the resource (beyond its range: zeros), whose
// offset is `offset` + `more`, to 1024 bytes at `to`.  (The compiler's own form makes every later read of the array wait for it; here the
// kernel waits itself, once a block.)
__device__ __forceinline__ u32x4 resource(const void* p, unsigned bytes) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return u32x4{(unsigned)at, (unsigned)(at >> 32) & 0xffffu, bytes, 0x00020000u};
}
__device__ __forceinline__ void lds_load(u32x4 rsrc, unsigned offset, unsigned more, const void* to) {
  const unsigned at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) const void*)to;
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(offset), "s"(rsrc), "s"(more), "s"(at)
               : "m0", "memory");
}

// The schedule of N products whose first operands come from LDS: reads go AHEAD of the
// products (16-bit types; the compiler's own order waits for nearly every read).
template <typename T, int N, int AHEAD>
__device__ __forceinline__ void reads_ahead() {
  if constexpr (sizeof(T) == 2) {
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);  // reads of LDS
#pragma unroll
    for (int i = 0; i < N - AHEAD; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // products
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
  }
}

// K and V of a block in LDS, in granules of 16 bytes: K [key][element], V as the
// cache has it, [16 keys][element][key].  The granules of a row lie in an order of
// the row's own, so that 16 lanes that read one of each of 16 rows meet none of the 64
// banks twice.
template <typename T, int DP>
struct RunTile {
  static constexpr int KB = run_keys<T>(), GE = 16 / sizeof(T), FG = 8 / GE;  // elements of a granule, granules of 8 elements
  static constexpr int KG = DP / GE, VG = 16 / GE;                            // granules of a key's row, of an element's 16 keys
  static constexpr int N = KB * DP / GE;                                      // of a block, each of K and V
  static __device__ __forceinline__ int k(int key, int g) { return key * KG + (g ^ (KG == 12 ? key >> 2 & 3 : KG < 16 ? key >> 1 & 7 : key & 15)); }
  static __device__ __forceinline__ int v_order(int d) { return sizeof(T) == 2 ? (d >> 3) & 1 : (d >> 2) & 3; }
  static __device__ __forceinline__ int v(int t16, int d, int g) { return (t16 * DP + d) * VG + (g ^ v_order(d)); }
};

// The rows of a tile: of sequence b the t-th 128.  False: there are fewer tiles.  In split calls
// sequences of equal lengths are found without looking at any (16 rows after 8192 keys 19.4 -> 18.5 us, 4
// after 4096 15.2 -> 14.3; others gain nothing, 4096 rows 154 -> 158).
__device__ __forceinline__ bool find_tile(const CacheArgs& c, int tile, int each, bool split, int& b, int& t, int& row0, int& n, int& past) {
  auto tiles = [&](int rows) { return ((int64_t)rows * each + kRunRows - 1) / kRunRows; };
  if (c.offsets || !split) return find_rows(c, tile, [&](int rows, int) { return tiles(rows); }, b, t, row0, n, past);
  n = (int)c.each;
  const int of = (int)tiles(n);
  b = uniform(tile / of);
  if (b >= c.seqs) return false;
  t = tile - b * of, row0 = b * n, past = uniform(min(c.past[b], kMaxPast));
  return true;
}
// The keys that a tile's rows see: positions of its first and last row, blocks of keys.
struct RunSpan {
  int pos0, pos1, first, end;
};
__device__ __forceinline__ RunSpan run_span(const AttnArgs& a, int t, int rows, int past, int KB) {
  RunSpan s;
  const int r0 = t * kRunRows, r1 = min(r0 + kRunRows, rows) - 1;
  s.pos0 = past < 0 ? -1 : past + uniform(fdiv(r0, a.each)), s.pos1 = past < 0 ? -1 : past + uniform(fdiv(r1, a.each));
  const int from = a.window ? max(0, s.pos0 - a.window + 1) : 0, last = min(s.pos1, (a.c.width << a.c.shift) - 1);
  s.first = from / KB, s.end = last < from ? s.first : last / KB + 1;
  return s;
}
// The launch's parts are as many as the table has room for; a tile uses as many as its keys make
// of four blocks at least (16 rows after none, in a table of 32768 positions, 15.5 -> 8.9 us,
// after 1000 15.2 -> 13.2; ragged lengths in f16 25.7 -> 22.7).
__device__ __forceinline__ int run_used(const RunSpan& s, int parts, int& per) {
  const int all = s.end - s.first;
  per = max(4, (all + parts - 1) / parts);
  return max(1, (all + per - 1) / per);
}
// Where a thread's sums of 4 elements of a part lie, and its maximum and sum of weights.
template <int DP>
__device__ __forceinline__ int run_o_at(int slot, int i) {
  return (slot * (DP / 8) + i) * 1024 + 4 * threadIdx.x;
}
__device__ __forceinline__ int run_m_at(int slot) { return slot * 512 + threadIdx.x; }

// The results of a tile's rows that have no weights, and the classes of those that are not finite, block by block as the
// products were taken.
template <typename T, bool I8, int DP>
__device__ __attribute__((noinline)) void run_again(KernelArgs args, int tile, bool split, float l, bool classes, unsigned* marks) {
  const AttnArgs a = *(const AttnArgs*)args;
  const CacheArgs& c = a.c;
  constexpr int KB = run_keys<T>(), GE = 16 / sizeof(T), VG = 16 / GE, NM = DP / 32;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, h = lane >> 5;
  const int D = c.dim, each = a.heads / c.kv_heads, head = blockIdx.x % c.kv_heads;
  int b, t, row0, n, past;
  if (!find_tile(c, tile, each, split, b, t, row0, n, past)) return;
  const int rows = n * each, mine = t * kRunRows + 32 * wave + r, token = fdiv(min(mine, rows - 1), a.each);
  const int pos = past < 0 ? -1 : past + token;
  T* y = static_cast<T*>(a.y) + (int64_t)(row0 + token) * a.ys + (int64_t)(head * each + mine - token * each) * D;
  if (mine < rows && l == 0.f && sees_place(c, b, a.window ? max(0, pos - a.window + 1) : 0, min(pos, (c.width << c.shift) - 1)))
    for (int d = 4 * h; d < D; d += 8)
#pragma unroll
      for (int j = 0; j < 4; ++j) y[d + j] = from_f<T>(__builtin_nanf(""));
  if (I8 || !classes) return;
  const RunSpan span = run_span(a, t, rows, past, KB);
  unsigned plus[NM], minus[NM];  // this lane's elements 32 i + 8 j + 4 h + x: bits 4 j + x
#pragma unroll
  for (int i = 0; i < NM; ++i) plus[i] = minus[i] = 0;
#pragma unroll 1
  for (int block = span.first; block < span.end; ++block) {
    __syncthreads();
    for (int i = tid; i < 4 * DP; i += 256) marks[i] = 0;
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < KB / GE * D; i += 256) {
      const int d = i / VG % D, key = i / (VG * D) * 16 + i % VG * GE, p = block * KB + key, page = page_of(c, b, p);
      if (page < 0) continue;
      T e[GE];
      __builtin_memcpy(e, static_cast<const T*>(c.v) + v_at(c, page, head, p & ((1 << c.shift) - 1)) + 16 * d, 16);
#pragma unroll
      for (int j = 0; j < GE; ++j) {
        const float v = (float)e[j];
        if (finite(v)) continue;
        if (!(v < 0.f)) atomicOr(&marks[4 * d + (key >> 5)], 1u << ((key & 31) + j));
        if (!(v > 0.f)) atomicOr(&marks[4 * d + 2 + (key >> 5)], 1u << ((key & 31) + j));
      }
    }
    __syncthreads();
    const unsigned seen0 = seen_keys(block * KB, pos, a.window), seen1 = KB > 32 ? seen_keys(block * KB + 32, pos, a.window) : 0u;
#pragma unroll
    for (int i = 0; i < NM; ++i)
#pragma unroll 1
      for (int j = 0; j < 16; ++j) {
        const unsigned* at = &marks[4 * (32 * i + 8 * (j >> 2) + 4 * h + (j & 3))];
        plus[i] |= (at[0] & seen0) | (at[1] & seen1) ? 1u << j : 0u;
        minus[i] |= (at[2] & seen0) | (at[3] & seen1) ? 1u << j : 0u;
      }
  }
  if (mine >= rows || !(l > 0.f && finite(l))) return;
#pragma unroll
  for (int i = 0; i < NM; ++i)
#pragma unroll 1
    for (int j = 0; j < 16; ++j)
      if ((plus[i] | minus[i]) >> j & 1) y[32 * i + 8 * (j >> 2) + 4 * h + (j & 3)] = from_f<T>(class_of(plus[i] >> j & 1, minus[i] >> j & 1));
}

template <typename T, bool I8, int DP, bool EXACT>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void attn_run_kernel(AttnArgs a) {
  typedef typename std::conditional<I8, int8_t, T>::type E;
  typedef typename Frag<T>::type F;
  typedef RunTile<T, DP> L;
  constexpr int KB = L::KB, NK = KB / 32, NS = DP / 16, ND = DP / 32, NG = L::N / 256, FG = L::FG;
  constexpr int NC = DP / 8, NL = KB * NC / 256;  // chunks of 8 elements (8-bit caches)
  constexpr bool POWER = I8 && std::is_same<T, f16>::value;  // see power_of
  // f16 weights are 2^6 times as large (2^14 at most, see kLazy)
  constexpr float LIFT = std::is_same<T, f16>::value ? 6.f : 0.f, kLazy = 8.f;
  __shared__ u32x4 sk[2 * L::N], sv[2 * L::N];
  __shared__ __attribute__((aligned(16))) float sks[2][I8 ? KB : 4], svs[2][I8 ? KB : 4];
  __shared__ F powers[POWER ? 4 * KB / 8 : 1];  // every wave's own
  __shared__ __attribute__((aligned(16))) unsigned marks[I8 ? 4 : DP * 4];  // of an element: 64 keys' bits, +inf or NaN; -inf or NaN
  __shared__ int flag[2], used, again[2];  // used: the tile's parts; again: rows without weights, results that are not finite
  const CacheArgs& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = lane & 31, h = lane >> 5;
  const int D = EXACT ? DP : c.dim, each = a.heads / c.kv_heads;
  // heads next to each other: workgroups of one head go to one XCD where 8 divides
  // their number.  The last tiles, which see the most keys, first.
  const int head = blockIdx.x % c.kv_heads, tiles = gridDim.x / c.kv_heads, tile = tiles - 1 - blockIdx.x / c.kv_heads;
  int b, t, row0, n, past;
  if (!find_tile(c, tile, each, gridDim.z > 1, b, t, row0, n, past)) return;
  const int rows = n * each, mine = t * kRunRows + 32 * wave + r;  // (below 2^31: the launcher's tiles)
  const int rr = min(mine, rows - 1);  // rows behind the last one repeat it and are not stored
  const int token = fdiv(rr, a.each), qh = head * each + rr - token * each;
  const int pos = past < 0 ? -1 : past + token;
  const int top_pos = __builtin_amdgcn_readlane(pos, 63), low_pos = uniform(pos);  // of the wave
  // the workgroup's keys, and this part's blocks of them
  const RunSpan span = run_span(a, t, rows, past, KB);
  const int pos0 = span.pos0, pos1 = span.pos1;
  int first = span.first, end = span.end;
  if (gridDim.z > 1) {
    int per;
    const int parts = run_used(span, gridDim.z, per);
    if (blockIdx.z >= parts) return;
    if (tid == 0) used = parts;
    first = min(end, first + (int)blockIdx.z * per), end = min(end, first + per);
  }
  const int mask = (1 << c.shift) - 1;

  F q[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int d = 16 * s + 8 * h;
    q[s] = frag_of<T>(load8(static_cast<const T*>(a.q) + (int64_t)(row0 + token) * a.qs + (int64_t)qh * D + (EXACT || d < D ? d : 0)));
    if (!EXACT && d >= D) q[s] = F{};
    if (a.negative) q[s] = -q[s];
  }

  // lane i holds the page of the i-th 16 positions of a block
  // (its entry of the table is read two blocks ahead, and looked at one block later)
  const int32_t* table = c.table + b * c.ts;
  auto entry_of = [&](int block) { return min(((block * KB) >> c.shift) + ((((block * KB) & mask) + 16 * min(lane, KB / 16 - 1)) >> c.shift), c.width - 1); };
  auto pages_of = [&](int block, int entry) {
    return lane < KB / 16 && block * KB + 16 * lane < c.width << c.shift && (unsigned)entry < (uint64_t)c.pages ? entry : -1;
  };
  // where the i-th 16 positions of a block lie, in rows of dim elements
  auto rows_at = [&](int block, int pages, int t16) {
    const int page = max(0, __builtin_amdgcn_readlane(pages, t16));
    return (((int64_t)page * c.kv_heads + head) << c.shift) + ((block * KB + 16 * t16) & mask);
  };
  const unsigned row_bytes = D * sizeof(E), page_bytes = (unsigned)(c.kv_heads << c.shift) * row_bytes, head_bytes = (head << c.shift) * row_bytes;

  // Caches in T: LDS direct loads.  A wave's i-th load fills the 64 granules from
  // 256 i + 64 wave on; all lie in one 16 positions.  This lane's granule is at an
  // offset from them that is the same in every block.
  unsigned koff[I8 ? 1 : NG], voff[I8 ? 1 : NG];
  if constexpr (!I8) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int x = 256 * i + tid, key = x / L::KG, kg = L::k(key, x % L::KG) % L::KG;
      koff[i] = EXACT || kg * L::GE < D ? (unsigned)(((key & 15) * D + kg * L::GE) * sizeof(T)) : kOOB;
      const int d = x / L::VG % DP, vg = x % L::VG ^ L::v_order(d);
      voff[i] = EXACT || d < D ? (unsigned)((d * 16 + vg * L::GE) * sizeof(T)) : kOOB;
    }
  }
  // 8-bit caches: through registers.
  V8<E> kr[I8 ? NL : 1], vr[I8 ? NL : 1];
  float ksr = 0.f, vsr = 0.f;
  auto load = [&](int block, int pages, int buf) {
    if constexpr (!I8) {
      // a 16 positions' place, and with pages of a whole block at least that of them all
      auto place = [&](int t16) {
        return (int64_t)((uint64_t)(unsigned)max(0, __builtin_amdgcn_readlane(pages, t16)) * page_bytes) + head_bytes +
               ((block * KB + 16 * t16) & mask) * row_bytes;
      };
      const unsigned to = buf * L::N + 64 * wave, tile_bytes = 16 * row_bytes;
      if (KB >> c.shift <= 1) {
        const int64_t o = place(0);
        const u32x4 rk = resource(static_cast<const char*>(c.k) + o, KB * row_bytes), rv = resource(static_cast<const char*>(c.v) + o, KB * row_bytes);
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const unsigned more = (256 * i + 64 * wave) / (16 * L::KG) * tile_bytes;
          lds_load(rk, koff[i], more, &sk[to + 256 * i]);
          lds_load(rv, voff[i], more, &sv[to + 256 * i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < NG; ++i) {
          const int64_t o = place((256 * i + 64 * wave) / (16 * L::KG));
          lds_load(resource(static_cast<const char*>(c.k) + o, tile_bytes), koff[i], 0, &sk[to + 256 * i]);
          lds_load(resource(static_cast<const char*>(c.v) + o, tile_bytes), voff[i], 0, &sv[to + 256 * i]);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int x = 256 * i + tid, w = 256 * i + 64 * wave;
        const int d = 8 * (x % NC), e = x % (2 * DP);
        kr[i] = load8(static_cast<const E*>(c.k) + (rows_at(block, pages, w / NC / 16) + (x / NC & 15)) * D + (EXACT || d < D ? d : 0));
        const int64_t at = rows_at(block, pages, w / (2 * DP));
        vr[i] = load8(static_cast<const E*>(c.v) + at * D + (EXACT ? 8 * e : 8 * min(e, 2 * D - 1)));
      }
      if (POWER || tid < KB) {
        const int key = tid & (KB - 1), page = max(0, __shfl(pages, key / 16));
        const int64_t at = (((int64_t)page * c.kv_heads + head) << c.shift) + ((block * KB + key) & mask);
        ksr = c.ks[at], vsr = c.vs[at];
      }
    }
  };
  auto put8 = [&](u32x4* to, int at0, int at1, const F& f) {
    const u32x4* p = reinterpret_cast<const u32x4*>(&f);
    to[at0] = p[0];
    if constexpr (FG == 2) to[at1] = p[1];
  };
  auto store = [&](int buf) {
    if constexpr (I8) {
      if constexpr (POWER) {
        reinterpret_cast<T*>(powers)[tid] = (T)power_of(vsr);  // (a wave holds all keys' scales)
        __builtin_amdgcn_wave_barrier();
      }
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int x = 256 * i + tid, key = x / NC, ch = x % NC;
        F f = frag_of<T>(kr[i]);
        if constexpr (!EXACT)
          if (8 * ch >= D) f = F{};
        put8(sk + buf * L::N, L::k(key, FG * ch), L::k(key, FG * ch + FG - 1), f);
        const int t16 = x / (2 * DP), e = x % (2 * DP), dd = e >> 1;
        F g = frag_of<T>(vr[i]);
        if constexpr (POWER) g *= powers[KB / 8 * wave + 2 * t16 + (e & 1)];
        put8(sv + buf * L::N, L::v(t16, dd, FG * (e & 1)), L::v(t16, dd, FG * (e & 1) + FG - 1), g);
      }
      if (tid < KB) sks[buf][tid] = ksr * a.scale2, svs[buf][tid] = POWER ? vsr / power_of(vsr) : vsr;
    }
  };
  auto k_frag = [&](int buf, int key, int ch) {
    F f;
    u32x4* p = reinterpret_cast<u32x4*>(&f);
#pragma unroll
    for (int i = 0; i < FG; ++i) p[i] = sk[buf * L::N + L::k(key, FG * ch + i)];
    return f;
  };
  auto v_frag = [&](int buf, int t16, int d) {
    F f;
    u32x4* p = reinterpret_cast<u32x4*>(&f);
#pragma unroll
    for (int i = 0; i < FG; ++i) p[i] = sv[buf * L::N + L::v(t16, d, FG * h + i)];
    return f;
  };

  // whether some row of the workgroup does not see some key of a block
  auto edge_of = [&](int block, int pages) {
    return block * KB + KB - 1 > pos0 || (a.window && block * KB < pos1 - a.window + 1) ||
           __builtin_popcountll(__ballot(pages >= 0)) < KB / 16;
  };
  // What a row does not see takes no part in it, whatever it is, but 0 times a value that
  // is not finite would: such blocks are looked through as they arrive, each thread
  // at what it has loaded.  (A flag holds a block's own number, so none is ever cleared.)
  auto look = [&](int block, int buf) {
    unsigned odd = 0;
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const u32x4 v = sv[buf * L::N + 256 * i + tid];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // an exponent of ones, and one more, carries into the sign
        constexpr unsigned E1 = std::is_same<T, f16>::value ? 0x7c007c00u : sizeof(T) == 2 ? 0x7f807f80u : 0x7f800000u;
        constexpr unsigned ONE = std::is_same<T, f16>::value ? 0x04000400u : sizeof(T) == 2 ? 0x00800080u : 0x00800000u;
        odd |= (v[j] & E1) + ONE;
      }
    }
    if (__any(odd & (sizeof(T) == 2 ? 0x80008000u : 0x80000000u)) && lane == 0) flag[buf] = block + 1;
  };

  f32x16 o[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i)
#pragma unroll
    for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
  float m = kNone, l = 0.f;
  int pages = -1, pages1 = -1;
  if (tid < 2) flag[tid] = 0, again[tid] = 0;
  if (first < end) {
    const int entry = table[entry_of(first)], entry1 = table[entry_of(first + 1)];
    pages = pages_of(first, entry), pages1 = pages_of(first + 1, entry1);
    load(first, pages, 0), store(0);
  }
  __syncthreads();  // (the flags are clear)
  wait_vmcnt<0>();
  if (!I8 && first < end && edge_of(first, pages)) look(first, 0);
  __syncthreads();
  for (int block = first; block < end; ++block) {
    const int buf = (block - first) & 1;
    const bool more = block + 1 < end;
    const int entry2 = table[entry_of(block + 2)];
    if (more) load(block + 1, pages1, buf ^ 1);
    const unsigned long long there = __ballot(pages >= 0);
    const bool edge = edge_of(block, pages);
    const bool odd = !I8 && edge && flag[buf] == block + 1;
    if (odd) {
      // Values that are not finite become zeros in LDS, with a bit that says where they
      // were: the rows that see them get a sum that is not finite after the product.
      for (int i = tid; i < DP * 4; i += 256) marks[i] = 0;
      lds_barrier();
#pragma unroll 1
      for (int i = 0; i < NG; ++i) {
        const int x = 256 * i + tid, d = x / L::VG % DP, key = x / (L::VG * DP) * 16 + (x % L::VG ^ L::v_order(d)) * L::GE;
        T e[L::GE];
        __builtin_memcpy(e, &sv[buf * L::N + x], 16);
#pragma unroll
        for (int j = 0; j < L::GE; ++j) {
          if (finite((float)e[j])) continue;
          atomicOr(&marks[4 * d + (key >> 5)], 1u << ((key & 31) + j));
          e[j] = (T)0.f;
        }
        __builtin_memcpy(&sv[buf * L::N + x], e, 16);
      }
      lds_barrier();
    }
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
        for (int j = 0; j < NS; ++j) s[i] = mma32(k_frag(buf, key, 2 * j + h), q[j], s[i]);
      }
      reads_ahead<T, NK * NS, 6>();
      if constexpr (I8) {
#pragma unroll
        for (int i = 0; i < NK; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) s[i][j] *= sks[buf][32 * i + 16 * (j >> 3) + 8 * h + (j & 7)];
      }
      if (edge) {
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
      float tops[4] = {kNone, kNone, kNone, kNone};
#pragma unroll
      for (int i = 0; i < NK; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) tops[j & 3] = fmaxf(tops[j & 3], s[i][j]);
      const float top = max_x32(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]))) * mul;
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
      float sums[4] = {l, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NK; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          s[i][j] = __builtin_amdgcn_exp2f(fmaf(s[i][j], mul, ref));
          sums[j & 3] += s[i][j];
        }
      l = (sums[0] + sums[1]) + (sums[2] + sums[3]);
      if constexpr (I8) {
#pragma unroll
        for (int i = 0; i < NK; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            s[i][j] *= svs[buf][32 * i + 16 * (j >> 3) + 8 * h + (j & 7)];
          }
        if (edge) {  // (the scale of a place that is not seen may be NaN)
#pragma unroll
          for (int i = 0; i < NK; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const int key = 32 * i + 16 * (j >> 3) + 8 * h + (j & 7), kpos = block * KB + key;
              const bool see = kpos <= pos && (!a.window || kpos > pos - a.window) && (there >> (2 * i + (j >> 3)) & 1);
              s[i][j] = see ? s[i][j] : 0.f;
            }
        }
      }
      // (the wave that multiplies goes first: the others have waits to fill; 4096 rows 162 -> 151 us)
      __builtin_amdgcn_s_setprio(1);
      F w[KB / 16];
#pragma unroll
      for (int kk = 0; kk < KB / 16; ++kk)
#pragma unroll
        for (int j = 0; j < 8; ++j) w[kk][j] = (T)s[kk >> 1][8 * (kk & 1) + j];
#pragma unroll
      for (int kk = 0; kk < KB / 16; ++kk)
#pragma unroll
        for (int i = 0; i < ND; ++i) o[i] = mma32(v_frag(buf, kk, 32 * i + r), w[kk], o[i]);
      reads_ahead<T, KB / 16 * ND, 4>();
      if (!I8) __builtin_amdgcn_s_setprio(0);
      if (odd) {
        // the keys that this row sees, against each element's marked ones
        unsigned seen[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < NK; ++i)
          seen[i] = seen_keys(block * KB + 32 * i, pos, a.window) & ((there >> (2 * i) & 1 ? 0xffffu : 0u) | (there >> (2 * i + 1) & 1 ? 0xffff0000u : 0u));
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            const unsigned* at = &marks[4 * (32 * i + 8 * (j >> 2) + 4 * h + (j & 3))];
            if ((at[0] & seen[0]) | (at[1] & seen[1])) o[i][j] += __builtin_huge_valf();
          }
      }
    }
    if (more) store(buf ^ 1);
    // (codes are turned into numbers before others' products go on: 4096 rows 200 -> 187 us)
    if (I8) __builtin_amdgcn_s_setprio(0);
    wait_vmcnt<0>();
    pages = pages1, pages1 = pages_of(block + 2, entry2);
    if (!I8 && more && edge_of(block + 1, pages)) look(block + 1, buf ^ 1);
    dma_barrier();
  }
  l = sum_x32(l);
  auto look_again = [&] {
    float odd[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) odd[j & 3] += o[i][j];
    const bool none = l == 0.f && pos >= 0 && mine < rows, odds = !I8 && l > 0.f && finite(l) && !finite((odd[0] + odd[1]) + (odd[2] + odd[3]));
    if (__any(none || odds)) {
      if (none) again[0] = 1;
      if (odds) again[1] = 1;
    }
  };
  const int parts = gridDim.z > 1 ? uniform(used) : 1;
  if (parts == 1) look_again();
  __syncthreads();

  if (parts > 1) {  // left in the lanes' order
    const int slot = blockIdx.x * gridDim.z;
    const Shared wo(a.ws_o), wm(a.ws_m);
    if (t * kRunRows + 32 * wave < rows) {
#pragma unroll
      for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          wo.put4(run_o_at<DP>(slot + blockIdx.z, 4 * i + j), f32x4{o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]});
      wm.put(run_m_at(slot + blockIdx.z), m), wm.put(run_m_at(slot + blockIdx.z) + 256, l);
    }
    if (run_joins<DP>(gridDim.z)) return;
    if constexpr (!run_joins<DP>(2)) {  // joined by the tile's last workgroup in the parts' order
      if (!last_of(a.count + blockIdx.x, parts, &flag[0])) return;
      const int there = t * kRunRows + 32 * wave < rows ? parts : 0;  // (a wave without rows left nothing)
      m = kNone;
#pragma unroll 4
      for (int z = 0; z < there; ++z) m = fmaxf(m, wm.get(run_m_at(slot + z)));
      l = 0.f;
#pragma unroll
      for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
      for (int z = 0; z < there; ++z) {
        const float f = __builtin_amdgcn_exp2f(wm.get(run_m_at(slot + z)) - some(m));
        l += f * wm.get(run_m_at(slot + z) + 256);
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const f32x4 v = wo.get4(run_o_at<DP>(slot + z, 4 * i + j));
#pragma unroll
            for (int x = 0; x < 4; ++x) o[i][4 * j + x] += f * v[x];
          }
      }
      look_again();
      __syncthreads();
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* y = static_cast<T*>(a.y) + (int64_t)(row0 + token) * a.ys + (int64_t)qh * D;
  if (mine < rows)
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
  if (uniform(again[0] | again[1])) run_again<T, I8, DP>((KernelArgs)__builtin_amdgcn_kernarg_segment_ptr(), tile, gridDim.z > 1, l, again[1], marks);
}

// The parts of a tile joined in their order, 4 elements of 128 rows at a time, each tile by as
// many workgroups as fill the chip.
template <typename T, int DP, bool EXACT>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, int parts) {
  const CacheArgs& c = a.c;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, h = lane >> 5;
  const int D = EXACT ? DP : c.dim, each = a.heads / c.kv_heads;
  const int head = blockIdx.x % c.kv_heads, tile = gridDim.x / c.kv_heads - 1 - blockIdx.x / c.kv_heads;
  int i = blockIdx.y;
  auto get = [&](int z, float& ms, float& ls, f32x4& os) {
    const int slot = blockIdx.x * parts + z;
    ms = a.ws_m[run_m_at(slot)], ls = a.ws_m[run_m_at(slot) + 256];
    os = *reinterpret_cast<const f32x4*>(a.ws_o + run_o_at<DP>(slot, i));
  };
  Join join;
  join.fetch(0, parts - 1, get);  // (before it is known whether the tile has rows: there is room for all)
  int b, t, row0, n, past;
  if (!find_tile(c, tile, each, true, b, t, row0, n, past)) return;
  const int mine = t * kRunRows + 32 * wave + r, token = fdiv(min(mine, n * each - 1), a.each);
  int per;
  const int used = run_used(run_span(a, t, n * each, past, run_keys<T>()), parts, per);
  if (used == 1 || mine >= n * each) return;  // (one: the rows are there)
  T* y = static_cast<T*>(a.y) + (int64_t)(row0 + token) * a.ys + (int64_t)(head * each + mine - token * each) * D;
  for (int z = 0;;) {
    join.add(z, used - 1);
    z += 8;
    if (z >= used) {
      const int d = 8 * i + 4 * h;
      const int pos = past < 0 ? -1 : past + token, from = a.window ? max(0, pos - a.window + 1) : 0, last = min(pos, (c.width << c.shift) - 1);
      if (!c.i8 && (EXACT || d < D) && join.sum > 0.f && finite(join.sum) && !finite((join.acc[0] + join.acc[1]) + (join.acc[2] + join.acc[3])))
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float is = class_of_values<T>((KernelArgs)__builtin_amdgcn_kernarg_segment_ptr(), b, head, d + x, from, last);
          if (is != 0.f) join.acc[x] = is;
        }
      float inv = 1.f / join.sum;
      if (join.sum == 0.f) inv = inverse_of_0((KernelArgs)__builtin_amdgcn_kernarg_segment_ptr(), b, from, last);
      T v[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) v[x] = from_f<T>(join.acc[x] * inv);
      if (EXACT || d < D) __builtin_memcpy(y + d, v, sizeof(v));
      if ((i += gridDim.y) >= DP / 8) return;
      join.top = kNone, join.sum = 0.f, join.acc = f32x4{0.f, 0.f, 0.f, 0.f}, z = 0;
    }
    join.fetch(z, used - 1, get);
  }
}

// ------------------------------------------------------------------ launches
template <typename T, bool I8, int DP, bool EXACT>
static void launch_step(AttnArgs& a, hipStream_t st) {
  const CacheArgs& c = a.c;
  constexpr int KB = 4 * step_keys<T, I8, DP>();
  const int each = a.heads / c.kv_heads, groups = (each + 15) / 16;
  const int64_t most = (((int64_t)c.width << c.shift) + KB - 1) / KB + 1;  // blocks of one sequence
  const int64_t own = c.seqs * ((most + kStepLeast - 1) / kStepLeast);     // parts, if each sequence has its own
  a.units = step_units(a, 512);
  if (!I8 && own > a.units) a.units = step_units(a, 256);
  const int64_t parts = std::min<int64_t>(a.units, own);
  SN_LAUNCH((attn_step_kernel<T, I8, DP, EXACT>), dim3((unsigned)parts, c.kv_heads, groups), dim3(64 * kStepWaves), 0, st, a);
}

template <typename T, bool I8, int DP, bool EXACT>
static void launch_run(AttnArgs& a, hipStream_t st) {
  const CacheArgs& c = a.c;
  constexpr int KB = run_keys<T>();
  const int64_t wgs = attn_run_tiles(a) * c.kv_heads, blocks = (((int64_t)c.width << c.shift) + KB - 1) / KB;
  a.each = make_fastdiv(a.heads / c.kv_heads);
  const int parts = (int)run_parts(blocks, wgs);
  SN_LAUNCH((attn_run_kernel<T, I8, DP, EXACT>), dim3((unsigned)wgs, 1, parts), dim3(256), 0, st, a);
  if (parts > 1 && run_joins<DP>(parts)) SN_LAUNCH((attn_join_kernel<T, DP, EXACT>), dim3((unsigned)wgs, (unsigned)std::min<int64_t>(DP / 8, std::max<int64_t>(1, 1024 / wgs))), dim3(256), 0, st, a, parts);
}

template <typename T>
static void launch_attention(AttnArgs& a, bool step, hipStream_t st) {
  auto sized = [&](auto i8, auto dp) {
    constexpr bool I8 = decltype(i8)::value;
    constexpr int DP = decltype(dp)::value;
    if constexpr (DP != 96)
      if (step) return a.c.dim == DP ? launch_step<T, I8, DP, true>(a, st) : launch_step<T, I8, DP, false>(a, st);
    a.c.dim == DP ? launch_run<T, I8, DP, true>(a, st) : launch_run<T, I8, DP, false>(a, st);
  };
  auto stored = [&](auto i8) {
    if (a.c.dim <= 64) return sized(i8, std::integral_constant<int, 64>());
    // prompts of 16-bit types, which the products bound: 4096 rows of 80 elements 140 -> 129 us,
    // in 8 bits 197 -> 166; steps are bound by bytes, which are the same
    if constexpr (sizeof(T) == 2)
      if (!step && a.c.dim <= 96) return sized(i8, std::integral_constant<int, 96>());
    if (a.c.dim <= 128) sized(i8, std::integral_constant<int, 128>());
    else sized(i8, std::integral_constant<int, 256>());
  };
  if (a.c.i8) stored(std::true_type());
  else stored(std::false_type());
}

}  // namespace k
}  // namespace sn
