// Selective state space scan with its short causal convolution.
//
// Per head, with running sums c_t of the log2 decays dt a inside a chunk of 64
// tokens, S[t][s] = C_t . B_s and Xd_s = dt_s X_s, the recurrence
// h_t = exp(dt_t a) h_{t-1} + Xd_t (outer) B_t, y_t = h_t C_t + d X_t is
//
//   y_t   = 2^{c_t} C_t h_0 + sum_{s <= t} S[t][s] 2^{c_t - c_s} Xd_s + d X_t
//   h_end = 2^{c_end} h_0 + sum_s 2^{c_end - c_s} B_s (outer) Xd_s
//
// i.e. three small matrix products per chunk and head on MFMA, chunk after
// chunk with the state in registers.  Sequences of many chunks are cut into
// segments so that few heads still fill the chip: a first pass finds the
// state that every segment adds, and the second pass starts every segment from
// its own state, summed up from those, by a small kernel if they are many.
//
// All decays are at most 1 (a <= 0).  c is held as hi + lo with hi in steps of
// 1/256, so that differences of hi are exact and those of lo small: a plain
// float32 sum would lose the differences of neighbours late in a chunk of
// strong decays.  A step's log2 decay counts as at least -1000: 2^-1000 is 0
// beside anything in float32, and 64 steps stay below 2^16, up to where float32
// holds every multiple of 1/256.
#include "seq.hpp"

namespace sn {
namespace k {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int Q = kScanChunk;
constexpr int kScanDt = kScanDtRow;

// ------------------------------------------------------------------ rows of a sequence
// First row and length of sequence b; offsets are clamped to the call's rows,
// so that no content of theirs leads outside.
struct Seq {
  int64_t first;
  int len;
};
__device__ __forceinline__ int64_t seq_start(const ScanArgs& a, int b) {
  if (!a.offsets) return (int64_t)b * a.each;
  const int64_t o = a.offsets[b];
  return o < 0 ? 0 : o > a.tokens ? a.tokens : o;
}
__device__ __forceinline__ Seq seq_of(const ScanArgs& a, int b) {
  Seq s;
  s.first = seq_start(a, b);
  const int64_t n = seq_start(a, b + 1) - s.first;
  s.len = n > 0 ? (int)n : 0;
  return s;
}
// Chunk c of sequence b has workspace slot first / 64 + b + c: a sequence of n
// rows has at most floor((first + n) / 64) - floor(first / 64) + 1 chunks, so
// slots of different sequences differ and stay below tokens / 64 + seqs + 1.
__device__ __forceinline__ int slot0_of(int64_t first, int b) { return (int)(first / Q) + b; }

// Likewise segment i of its sequence, of `per` chunks, has slot segment0 + i,
// below (tokens / 64 + seqs) / per + seqs + 1.
__device__ __forceinline__ int64_t segment0_of(const ScanArgs& a, int64_t first, int b) {
  return slot0_of(first, b) / a.per + b;
}

// Raw value of channel ch at time t of a sequence: before 0 from the window,
// past the end 0.
template <typename T>
__device__ __forceinline__ float raw_at(const ScanArgs& a, const Seq& s, int b, int t, int ch) {
  if (t >= s.len) return 0.f;
  if (t >= 0) return to_f(static_cast<const T*>(a.x)[(s.first + t) * a.xs + ch]);
  const int k = a.conv - 1 + t;
  return k < 0 || !a.window ? 0.f : to_f(static_cast<const T*>(a.window)[((int64_t)b * (a.conv - 1) + k) * a.chans + ch]);
}

// The convolution's sum over up to 4 taps, r[3] the newest value; taps that
// the layer does not have are not touched (their values may be NaN).
__device__ __forceinline__ float taps4(const float (&w)[4], float bias, float r0, float r1, float r2, float r3, int conv) {
  float u = fmaf(w[3], r3, bias);
  if (conv > 1) u = fmaf(w[2], r2, u);
  if (conv > 2) u = fmaf(w[1], r1, u);
  if (conv > 3) u = fmaf(w[0], r0, u);
  return u;
}

// ------------------------------------------------------------------ operands in two halves
// The matrix products run in f16 with float32 sums.  An operand is scaled by a
// power of two that brings its largest value below 2^14, and split in hi =
// f16(v) and lo = f16(v - hi).  hi hi + hi lo + lo hi then has 22 significant
// bits, float32's precision but for 2, at a third of the f16 rate, five times that
// of the float32 instructions.  Values have all 22 bits down to 2^-17 of the
// largest beside them, and fewer below: an error of 2^-39 of that.  It is taken
// over as little as shares a sum, from the values themselves (a product of maxima
// that lie in different rows would be far above any): a row of the mix; a
// column's state; a column's convolved values and, apart from them, those values
// times step and decay, in a chunk; B and C over a chunk of their group.
// Scales are kept as exponents: a product's comes off as their sum in one
// ldexp, where the product of two powers, or of two inverses, may leave
// float32's range.
__device__ __forceinline__ int exp_for(float m) {  // k with m 2^k in [2^13, 2^14), at most 126
  const int e = (__builtin_bit_cast(int, m) >> 23) & 255;
  return min(140 - e, 126);
}
__device__ __forceinline__ float pow2(int k) { return __builtin_bit_cast(float, (k + 127) << 23); }
struct HiLo {
  f16x8 hi, lo;
};
__device__ __forceinline__ HiLo split8(const float (&v)[8]) {
  HiLo r;
  u32x4 h;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    typedef f16 f16x2 __attribute__((ext_vector_type(2)));
    h[i] = __builtin_bit_cast(unsigned, f16x2{(f16)v[2 * i], (f16)v[2 * i + 1]});
    // lo is taken from the packed halves as they are: the compiler may fold the
    // product that makes v into one conversion of two (one rounding instead of
    // two), and near a tie hi and the hi that lo completes would differ
    unsigned one = h[i];
    asm("" : "+v"(one));
    h[i] = one;
  }
  r.hi = __builtin_bit_cast(f16x8, h);
#pragma unroll
  for (int i = 0; i < 8; ++i) r.lo[i] = (f16)(v[i] - (float)r.hi[i]);
  return r;
}
__device__ __forceinline__ f32x4 mul3(const HiLo& a, const HiLo& b, f32x4 c) {
  c = Mfma<f16>::run(a.lo, b.hi, c);
  c = Mfma<f16>::run(a.hi, b.lo, c);
  return Mfma<f16>::run(a.hi, b.hi, c);
}
// The larger of a running maximum and |v|, unless v is not finite.
__device__ __forceinline__ float max_finite(float m, float v) {
  v = fabsf(v);
  return v < INFINITY ? fmaxf(m, v) : m;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 32; d > 0; d /= 2) v = fmaxf(v, __shfl_xor(v, d));
  return v;
}
// Over the four lanes l % 16 + 16 i.  (A swap of v's halves, or rows of 16 lanes,
// with another register that holds v leaves each side's in one of the two.)
template <class F>
__device__ __forceinline__ unsigned over_rows(unsigned v, F f) {
  const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  const unsigned w = f((unsigned)a[0], (unsigned)a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
  return f((unsigned)b[0], (unsigned)b[1]);
}
// The largest of values >= 0 (as bits, which have the same order; a NaN counts as largest).
__device__ __forceinline__ float rows_max(float v) {
  return __builtin_bit_cast(float, over_rows(__builtin_bit_cast(unsigned, v), [](unsigned a, unsigned b) { return max(a, b); }));
}
__device__ __forceinline__ float rows_sum(float v) {
  return __builtin_bit_cast(float, over_rows(__builtin_bit_cast(unsigned, v), [](unsigned a, unsigned b) {
    return __builtin_bit_cast(unsigned, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
  }));
}

// ------------------------------------------------------------------ what all heads share
// grid (slots, groups + ceil(heads / 16) + copies).  The y index chooses: a
// group's B, C and S; 16 heads' step sizes and decays; a share of the windows'
// copy.  B and C go out as hi and lo in the order of the operands:
//   ws_c [slot][group][tb][q][hi, lo][lane][8]: t = 16 tb + lane % 16
//   ws_b [slot][group][nt][q][hi, lo][lane][8]: n = 16 nt + lane % 16
// with the 8 values of step q at 32 q + 4 (lane / 16) + {0..3, 16..19} of n or
// s: the order in which accumulator tiles hold rows.  S = C B^T in float32,
//   ws_s [slot][group][tb][sb <= tb][lane][4]: t = 16 tb + lane % 16, s = 16 sb + 4 (lane / 16) + 0..3.
// Once per chunk and group instead of once per wave of the heads.  Bound by
// latency: one workgroup per chunk and part, the raw rows from memory, then the
// convolution, the maxima and S one after the other, 11.5 us for 4096 tokens of
// 64 heads and one group.
constexpr int kPrep = 1024;
template <typename T, int NP>
__global__ __launch_bounds__(kPrep) void scan_prep_kernel(ScanArgs a) {
  extern __shared__ __attribute__((aligned(16))) float lds[];
  const int part = blockIdx.y, hb = (a.heads + 15) / 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (part >= a.groups + hb) {
    const int64_t n = (int64_t)a.seqs * (a.conv - 1) * a.chans, step = (int64_t)(gridDim.y - a.groups - hb) * gridDim.x * kPrep;
    const T* src = static_cast<const T*>(a.window);
    T* dst = static_cast<T*>(a.wcopy);
    for (int64_t i = ((int64_t)(part - a.groups - hb) * gridDim.x + blockIdx.x) * kPrep + threadIdx.x; i < n; i += step)
      dst[i] = src ? src[i] : from_f<T>(0.f);
    return;
  }
  // the sequence of this slot: the last one whose first slot is not above it
  const int slot = blockIdx.x;
  int lo = 0, hi = a.seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (slot0_of(seq_start(a, mid), mid) <= slot) lo = mid;
    else hi = mid - 1;
  }
  const int b = lo;
  const Seq s = seq_of(a, b);
  const int c = slot - slot0_of(s.first, b);
  if (c < 0 || c * Q >= s.len) return;
  const int t0 = c * Q;

  if (part >= a.groups) {  // ---- a wave per head, a lane per token
    const int h = (part - a.groups) * 16 + wave;
    if (h >= a.heads) return;
    const int t = t0 + lane;
    float dt = 0.f, inc = 0.f;
    if (t < s.len) {
      const float v = to_f(static_cast<const T*>(a.dt)[(s.first + t) * a.dts + h]) + a.dt_bias[h];
      dt = v > 20.f ? v : log1pf(expf(v));  // beyond 20 the difference is below a unit
      inc = dt * a.a2[h];
      if (inc < -1000.f) inc = -1000.f;  // still 0, and the sums' hi exact; NaN stays
    }
    float ch = rintf(inc * 256.f) * (1.f / 256.f), cl = inc - ch;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const float uh = __shfl_up(ch, d), ul = __shfl_up(cl, d);
      if (lane >= d) ch += uh, cl += ul;
    }
    const float eh = __shfl(ch, 63), el = __shfl(cl, 63);
    const float f = dt * __builtin_amdgcn_exp2f((eh - ch) + (el - cl));
    float* o = a.ws_dt + ((int64_t)slot * a.heads + h) * kScanDt;
    o[lane] = __builtin_amdgcn_exp2f(ch + cl);
    o[Q + lane] = ch;
    o[2 * Q + lane] = cl;
    o[3 * Q + lane] = dt;
    o[4 * Q + lane] = f;
    if (lane == 0) o[5 * Q] = eh + el;
    return;
  }

  // ---- B and C of one group
  const int N = a.state;
  constexpr int pitch = NP + 4, ITEMS = NP / 32;  // channels by 4 times per thread
  float* Cs = lds;                // [t][n]
  float* Bs = lds + Q * pitch;    // [t][n]
  float* red = Bs + Q * pitch;    // [2][waves]
  float mb = 0.f, mc = 0.f;
  float w[ITEMS][4], bias[ITEMS];
  T r[ITEMS][7];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {  // all loads first
    const int i = threadIdx.x + kPrep * k, e = i % (2 * NP), tq = i / (2 * NP) * 4;
    const int n = min(e % NP, N - 1), ch = a.heads * a.dim + (e >= NP ? a.groups * N : 0) + part * N + n;
    const T* x = static_cast<const T*>(a.x) + s.first * a.xs + ch;
#pragma unroll
    for (int j = 0; j < 7; ++j) r[k][j] = x[min(max(t0 + tq - 3 + j, 0), s.len - 1) * a.xs];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[k][j] = a.conv_w[j * a.chans + ch];
    bias[k] = a.conv_b[ch];
  }
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int i = threadIdx.x + kPrep * k, e = i % (2 * NP), tq = i / (2 * NP) * 4, n = e % NP;
    const bool isc = e >= NP;
    float v[7];
#pragma unroll
    for (int j = 0; j < 7; ++j) v[j] = to_f(r[k][j]);
    if (t0 + tq == 0) {
      const int ch = a.heads * a.dim + (isc ? a.groups * N : 0) + part * N + min(n, N - 1);
#pragma unroll
      for (int j = 0; j < 3; ++j) v[j] = raw_at<T>(a, s, b, j - 3, ch);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float u = 0.f;  // past the end, and in columns that only fill the tile
      if (t0 + tq + j < s.len && n < N) u = silu_f(taps4(w[k], bias[k], v[j], v[j + 1], v[j + 2], v[j + 3], a.conv));
      if (isc) mc = max_finite(mc, u);
      else mb = max_finite(mb, u);
      (isc ? Cs : Bs)[(tq + j) * pitch + n] = u;
    }
  }
  mb = wave_max(mb), mc = wave_max(mc);
  if (lane == 0) red[wave] = mb, red[kPrep / 64 + wave] = mc;
  __syncthreads();
  mb = wave_max(red[lane & 15]), mc = wave_max(red[16 + (lane & 15)]);
  const float sb_ = pow2(exp_for(mb)), sc_ = pow2(exp_for(mc));
  const int64_t sg = (int64_t)slot * a.groups + part;
  if (threadIdx.x == 0) a.ws_max[sg * kScanMax] = mb, a.ws_max[sg * kScanMax + 1] = mc;
  const int col = lane & 15, g = lane >> 4;
  f16* Cg = static_cast<f16*>(a.ws_c) + sg * Q * NP * 2;
  f16* Bg = static_cast<f16*>(a.ws_b) + sg * Q * NP * 2;
  constexpr int NQ = NP / 32;
  for (int f = wave; f < 4 * NQ + NP / 16 * 2; f += kPrep / 64) {
    const bool isc = f < 4 * NQ;
    float v[8];
    if (isc) {
      const int tb = f / NQ, q = f % NQ;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = sc_ * Cs[(16 * tb + col) * pitch + 32 * q + 4 * g + j + (j & 4) * 3];
    } else {
      const int nt = (f - 4 * NQ) >> 1, q = (f - 4 * NQ) & 1;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = sb_ * Bs[(32 * q + 4 * g + j + (j & 4) * 3) * pitch + 16 * nt + col];
    }
    const HiLo r = split8(v);
    f16* o = (isc ? Cg + f * 1024 : Bg + (f - 4 * NQ) * 1024) + lane * 8;
    *reinterpret_cast<f16x8*>(o) = r.hi;
    *reinterpret_cast<f16x8*>(o + 512) = r.lo;
  }
  const int tb = wave >> 2, sb = wave & 3;
  if (sb <= tb) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int n0 = 0; n0 < NP; n0 += 16) {
      const f32x4 bf = *reinterpret_cast<const f32x4*>(Bs + (16 * sb + col) * pitch + n0 + 4 * g);
      const f32x4 cf = *reinterpret_cast<const f32x4*>(Cs + (16 * tb + col) * pitch + n0 + 4 * g);
#pragma unroll
      for (int v = 0; v < 4; ++v) acc = Mfma<float>::run(bf[v], cf[v], acc);  // rows s, columns t
    }
    *reinterpret_cast<f32x4*>(a.ws_s + sg * kScanS + (tb * (tb + 1) / 2 + sb) * 256 + lane * 4) = acc;
  }
}

// ------------------------------------------------------------------ the heads
// A wave owns 16 columns p of one head and all N <= 16 NT state rows n: the
// state lives in NT accumulator tiles (lane: n = 16 nt + 4 (lane / 16) + v, p =
// p0 + lane % 16), whose layout is also that of the second operand
// of the product with C, so the state never leaves the registers; and a lane's
// convolution outputs (times 16 sb + 4 (lane / 16) + v, the same p) are the
// second operand of both other products.
// SEG: only the state that the segment adds (from zero; unless they are carried,
// segment 0 from the sequence's own, which it copies), no outputs.
// SHARE: the four waves of 64 columns of a head make its mix of a chunk's rows
// together.
//
// The waves of a workgroup share the group's C, B and S of a chunk in LDS, and
// each has its head's decays there, all brought by LDS direct loads while the
// chunk before (C, decays; with SHARE S) or the product with C (B; else S) is
// computed: two barriers per chunk, behind which one set has arrived and the
// other is free.  Bound by the latency of one chunk after the other: about 5 us
// for a lone wave, 1.5 more for each further wave of a SIMD, whose registers
// (178) leave room for two; 4096 tokens of 64 heads of 64 x 128 in bf16: 33 us
// for the first pass, 77 for the second, with matrix instructions in 16% of the
// cycles and other vector instructions in 37%; 8 sequences of 2048, which need no
// first pass, 275 us all told.  Twelve or sixteen waves were not faster.
// (Scales from products of maxima instead of from the values: 8 us less for the
// second pass, and rows of large values took the others' bits.)
//
// SEG up to 128 state rows has room for two chunks' B, and one barrier per chunk
// (33.5 us against 35.5; at 256 rows two chunks leave one workgroup per CU: 105
// us for the whole scan against 98).
constexpr int kScanWaves = 8;  // of a workgroup: 2 per SIMD
constexpr int kDtBytes = kScanDt * 4;
constexpr int kMaxBytes = kScanMax * 4;
constexpr int kMixBytes = 6 * (2048 + 64);  // a head's 6 operands of the mix of a chunk's rows, hi and lo, and their rows' scales
template <int NT, bool SEG>
constexpr bool scan_two() { return SEG && NT <= 8; }
template <int NT, bool SEG>
constexpr int scan_tiles() { return SEG ? (scan_two<NT, SEG>() ? 8192 : 4096) * NT : 8192 * NT + 10 * 1024; }
template <int NT, bool SHARE, bool SEG>
constexpr int scan_lds(int waves) {  // B, C, S, two sets of largest sizes, two decay rows per wave, the mix of every 4 waves
  return scan_tiles<NT, SEG>() + 2 * kMaxBytes + waves * 2 * kDtBytes + (SHARE && !SEG ? waves / 4 * kMixBytes : 0);
}
template <typename T, int NT, bool SHARE, bool SEG>
__global__ __launch_bounds__(64 * kScanWaves) void scan_main_kernel(ScanArgs a) {
  constexpr bool TWO = scan_two<NT, SEG>();
  extern __shared__ __attribute__((aligned(16))) char smem[];
  char* const ldsB = smem;
  char* const ldsC = smem + 4096 * NT;                    // not with SEG
  char* const ldsS = smem + 8192 * NT;                    // not with SEG
  const int waves = blockDim.x >> 6;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  // Sequences and then segments vary fastest over the workgroups, so that (with
  // 8 of them or a multiple) each XCD's L2 serves the chunks of its own.  With
  // offsets, segments vary slowest: most sequences have none of the later ones,
  // and workgroups without work at regular places leave whole shader engines
  // idle (8 sequences of 2048 rows: 981 us against 357).
  const int each = a.heads / a.groups, pblocks = (a.dim + 15) / 16;
  const int ublocks = (each * pblocks + waves - 1) / waves, yblocks = a.groups * ublocks;
  const unsigned rest = blockIdx.x / a.seqs;
  const int b = blockIdx.x % a.seqs;
  const int seg = a.offsets ? rest / yblocks : rest % a.segs, yb = a.offsets ? rest % yblocks : rest / a.segs;
  const int grp = yb / ublocks, unit_ = (yb % ublocks) * waves + wave;
  // a wave beyond the last unit works on the last one, for the barriers' sake, and stores nothing
  const bool live = unit_ < each * pblocks;
  const int unit = min(unit_, each * pblocks - 1);
  char* const ldsM = smem + scan_lds<NT, false, SEG>(waves) + (wave >> 2) * kMixBytes;  // with SHARE
  char* const ldsX = smem + scan_tiles<NT, SEG>();
  char* const ldsD = ldsX + 2 * kMaxBytes + wave * 2 * kDtBytes;
  const Seq s = seq_of(a, b);
  const int nc = (s.len + Q - 1) / Q;
  const int c0 = min(seg * a.per, nc), c1 = min(c0 + a.per, nc);
  const int N = a.state;
  constexpr int NP = 16 * NT;

  if (!SEG && a.window_out) {
    // the window after the last row, shared out over the sequence's workgroups
    const int64_t n = (int64_t)(a.conv - 1) * a.chans;
    const int blocks = a.segs * yblocks, me = yb * a.segs + seg;
    T* out = static_cast<T*>(a.window_out) + b * n;
    for (int64_t i = (int64_t)me * blockDim.x + threadIdx.x; i < n; i += (int64_t)blocks * blockDim.x) {
      const int k = (int)(i / a.chans), ch = (int)(i - (int64_t)k * a.chans), t = s.len - (a.conv - 1) + k;
      out[i] = t >= 0 ? static_cast<const T*>(a.x)[(s.first + t) * a.xs + ch]
                      : static_cast<const T*>(a.wcopy)[b * n + (int64_t)(a.conv - 1 + t) * a.chans + ch];
    }
  }
  const int h = grp * each + unit / pblocks;
  const int p0 = unit % pblocks * 16 + col;  // this lane's p
  const bool have = live && p0 < a.dim;      // whether it exists
  const int64_t hold = (int64_t)a.dim * N;

  f32x4 st[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) st[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
  // the lane's part of a head's state; what is outside it has an offset out of range
  auto at_state = [&](int nt, int v) {
    const int n = 16 * nt + 4 * g + v;
    return (int)(have && n < N ? ((unsigned)p0 * (unsigned)N + (unsigned)n) * 4u : kOOB);
  };
  auto load_state = [&](const float* p, f32x4 (&to)[NT]) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p, hold * 4);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      if (a.vec_state) {
        to[nt] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at_state(nt, 0), 0, 0));
      } else {
#pragma unroll
        for (int v = 0; v < 4; ++v)
          to[nt][v] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, at_state(nt, v), 0, 0));
      }
  };
  auto store_state = [&](float* p) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(p, hold * 4);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      if (a.vec_state) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, st[nt]), r, at_state(nt, 0), 0, 0);
      } else {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float one = st[nt][v];  // (a bit cast of the element itself reads element 0)
          __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, one), r, at_state(nt, v), 0, 0);
        }
      }
  };
  // the head's slot of segment i
  const int64_t head_seg0 = segment0_of(a, s.first, b) * a.heads + h;
  auto seg_slot = [&](int i) { return head_seg0 + (int64_t)i * a.heads; };
  auto seg_state = [&](int i) { return a.ws_seg + seg_slot(i) * hold; };
  // the whole workgroup: a segment that nothing follows (no one reads its
  // state), or behind the sequence's last one (which has no slot)
  if (SEG ? c1 >= nc : seg > 0 && c0 >= nc) return;
  // the lane's convolution
  const int ch0 = h * a.dim + p0;
  float w[4];
  const float cb = have ? a.conv_b[ch0] : 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = have ? a.conv_w[k * a.chans + ch0] : 0.f;
  const float dh = SEG ? 0.f : a.d[h];
  const unsigned rowb = (unsigned)a.xs * (unsigned)sizeof(T);
  const unsigned xoff = 4 * g * rowb + (unsigned)(h * a.dim + p0) * (unsigned)sizeof(T);
  float total = 0.f;  // log2 of the segment's decay
  const int slot0 = slot0_of(s.first, b);
  auto fetch = [&](char* to, const void* from, int kbytes) {  // shared by the waves, 1 KB an instruction
    const __amdgpu_buffer_rsrc_t r = make_rsrc(from, kbytes * 1024);
    for (int i = wave; i < kbytes; i += waves) dma16(r, to + i * 1024, lane * 16 + i * 1024, 0);
  };
  auto fetch_c = [&](int c) {  // C, the wave's decays, and S (its tiles on and below the diagonal, packed) with SHARE
    const int64_t sg = (int64_t)(slot0 + c) * a.groups + grp;
    if (!SEG) fetch(ldsC, static_cast<const char*>(a.ws_c) + sg * 4096 * NT, 4 * NT);
    if (!SEG && SHARE) fetch(ldsS, a.ws_s + sg * kScanS, 10);
    const __amdgpu_buffer_rsrc_t r = make_rsrc(a.ws_dt + ((int64_t)(slot0 + c) * a.heads + h) * kScanDt, kDtBytes);
    char* to = ldsD + (c & 1) * kDtBytes;
    dma16(r, to, lane * 16, 0);
    if (lane < (kDtBytes - 1024) / 16) dma16(r, to + 1024, lane * 16 + 1024, 0);
    if (wave == 0 && lane < kMaxBytes / 16)
      dma16(make_rsrc(a.ws_max + sg * kScanMax, kMaxBytes), ldsX + (c & 1) * kMaxBytes, lane * 16, 0);
  };
  auto fetch_b = [&](int c) {  // B, and S without SHARE
    const int64_t sg = (int64_t)(slot0 + c) * a.groups + grp;
    fetch(ldsB + (TWO ? (c & 1) * 4096 * NT : 0), static_cast<const char*>(a.ws_b) + sg * 4096 * NT, 4 * NT);
    if (!SEG && !SHARE) fetch(ldsS, a.ws_s + sg * kScanS, 10);
  };
  // Raw rows 16 sb + 4 g - 3 + k of a chunk; rows past the end (or before the
  // sequence) give zero, and so does a chunk past the segment.
  T raw[4][7];
  auto load_raw = [&](int c) {
    unsigned xo = xoff;  // per chunk: kept out of the loop, its 28 sums would fill the registers
    asm volatile("" : "+v"(xo));
    const int t0 = c * Q;
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(static_cast<const T*>(a.x) + (s.first + t0 - 3) * a.xs,
                                                c < c1 ? (long long)min(s.len - t0 + 3, Q + 3) * rowb : 0);
#pragma unroll
    for (int sb = 0; sb < 4; ++sb)
#pragma unroll
      for (int k = 0; k < 7; ++k) {
        const bool before = sb == 0 && k < 3 && c == 0 && g == 0;
        const unsigned row = xo + (16 * sb + k) * rowb;  // in the offset that the range check sees
        const unsigned o = before || !have ? kOOB : row;
        if constexpr (sizeof(T) == 2) {
          const uint16_t v = __builtin_amdgcn_raw_buffer_load_b16(rx, (int)o, 0, 0);
          __builtin_memcpy(&raw[sb][k], &v, 2);
        } else {
          const unsigned v = __builtin_amdgcn_raw_buffer_load_b32(rx, (int)o, 0, 0);
          __builtin_memcpy(&raw[sb][k], &v, 4);
        }
      }
  };
  // Accesses of a chunk that follow its loads of the next chunk's C and decays:
  // the raw rows, and the stores of y.
  constexpr int AFTER = 28 + (SEG ? 0 : 16);
  if (c0 < c1) fetch_c(c0), fetch_b(c0);
  if (!SEG) {
    const float* in = a.state_in ? a.state_in + ((int64_t)b * a.heads + h) * hold : nullptr;
    if (nc <= a.per) {
      if (in) load_state(in, st);
    } else if (seg == 0) {
      // the copy: by now the sequence's last segment may have written its state in place
      if (in) load_state(seg_state(0), st);
    } else {
      const int from = a.carried ? seg : 1;
      load_state(seg_state(from), st);
      for (int i = from + 1; i <= seg; ++i) {
        f32x4 add[NT];
        load_state(seg_state(i), add);
        const float f = __builtin_amdgcn_exp2f(a.ws_decay[seg_slot(i)]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int v = 0; v < 4; ++v) st[nt][v] = fmaf(st[nt][v], f, add[nt][v]);
      }
    }
  }
  load_raw(c0);
  if (SEG) {
    if (!a.carried && seg == 0 && a.state_in) {
      load_state(a.state_in + ((int64_t)b * a.heads + h) * hold, st);
      store_state(seg_state(0));
    }
  }
  wait_vmcnt<0>();
  dma_barrier();
  for (int c = c0; c < c1; ++c) {
    const int t0 = c * Q;
    const f16* Cg = reinterpret_cast<const f16*>(ldsC) + lane * 8;
    const f16* Bg = reinterpret_cast<const f16*>(ldsB + (TWO ? (c & 1) * 4096 * NT : 0)) + lane * 8;
    const float* Sg = reinterpret_cast<const float*>(ldsS) + lane * 4;
    const float* dtp = reinterpret_cast<const float*>(ldsD + (c & 1) * kDtBytes);
    // (from LDS: scalar loads here would hold up every wait for LDS)
    const float* maxes = reinterpret_cast<const float*>(ldsX + (c & 1) * kMaxBytes);
    float maxb, maxc, cend;
    auto scalars = [&] { maxb = maxes[0], maxc = maxes[1], cend = dtp[5 * Q]; };
    if constexpr (!SEG) scalars();
    f32x4 acc[4];
    int kh = 0;
    if constexpr (!SEG) {
      // ---- C times the state in front of the chunk
      float top = 0.f;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int v = 0; v < 4; ++v) top = fmaxf(top, fabsf(st[nt][v]));
      kh = exp_for(rows_max(top));
      const float sh = pow2(kh);
#pragma unroll
      for (int tb = 0; tb < 4; ++tb) acc[tb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int q = 0; q < NT / 2; ++q) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = sh * st[2 * q + (e >> 2)][e & 3];
        const HiLo hf = split8(v);
#pragma unroll
        for (int tb = 0; tb < 4; ++tb) {
          const f16* cp = Cg + (tb * (NT / 2) + q) * 1024;
          HiLo cf;
          cf.hi = *reinterpret_cast<const f16x8*>(cp);
          cf.lo = *reinterpret_cast<const f16x8*>(cp + 512);
          acc[tb] = mul3(cf, hf, acc[tb]);
        }
      }
    }
    // ---- convolution
    __builtin_amdgcn_sched_barrier(0);  // (the fences keep one phase's registers from another's)
    if (c == 0 && g == 0) {  // the window in front of the sequence
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const int i = a.conv - 4 + k;
        if (i >= 0 && have) raw[0][k] = static_cast<const T*>(a.wcopy)[((int64_t)b * (a.conv - 1) + i) * a.chans + ch0];
      }
    }
    float u[4][4], sq = 0.f;
    auto convolve = [&](int conv) {
#pragma unroll
      for (int sb = 0; sb < 4; ++sb) {
        float r[7];
#pragma unroll
        for (int k = 0; k < 7; ++k) r[k] = to_f(raw[sb][k]);
#pragma unroll
        for (int v = 0; v < 4; ++v) u[sb][v] = taps4(w, cb, r[v], r[v + 1], r[v + 2], r[v + 3], conv);
      }
    };
    if (a.conv == 4) convolve(4);  // without the tests for absent taps
    else convolve(a.conv);
#pragma unroll
    for (int sb = 0; sb < 4; ++sb)
#pragma unroll
      for (int v = 0; v < 4; ++v) u[sb][v] = silu_f(u[sb][v]);
    // The mix of rows 16 tb .. + 15 with rows 32 q .. + 31: S, the decay between
    // them and the step size, above the diagonal nothing; scaled by 2^k, a row's
    // own (the lane's: row 16 tb + lane % 16).
    auto mix = [&](int tb, int q, int& k) {
      const float th = dtp[Q + 16 * tb + col], tl = dtp[2 * Q + 16 * tb + col];
      float m[8], most = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int sb = 2 * q + i, at = 16 * sb + 4 * g;
        const f32x4 sh_ = *reinterpret_cast<const f32x4*>(dtp + Q + at);
        const f32x4 sl_ = *reinterpret_cast<const f32x4*>(dtp + 2 * Q + at);
        const f32x4 sd_ = *reinterpret_cast<const f32x4*>(dtp + 3 * Q + at);
        const f32x4 sv = *reinterpret_cast<const f32x4*>(Sg + (tb * (tb + 1) / 2 + min(sb, tb)) * 256);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float x = sv[v] * sd_[v] * __builtin_amdgcn_exp2f((th - sh_[v]) + (tl - sl_[v]));
          m[4 * i + v] = at + v > 16 * tb + col ? 0.f : x;
          most = fmaxf(most, fabsf(m[4 * i + v]));
        }
      }
      k = exp_for(rows_max(most));
      const float s = pow2(k);
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] *= s;
      return split8(m);
    };
    // [operand][hi, lo][lane], operand tb + 2 q; then [operand][16] scales
    f16x8* const mixes = reinterpret_cast<f16x8*>(ldsM) + lane;
    int* const mixk = reinterpret_cast<int*>(ldsM + 6 * 2048);
    if constexpr (SHARE && !SEG) {
      // the four waves of a head make 10 tiles, 2 or 3 each
      auto put = [&](int tb, int q) {
        int k;
        const HiLo m = mix(tb, q, k);
        mixes[(tb + 2 * q) * 128] = m.hi;
        mixes[(tb + 2 * q) * 128 + 64] = m.lo;
        if (g == 0) mixk[(tb + 2 * q) * 16 + col] = k;
      };
      const int w4 = wave & 3;
      put(w4 == 3 ? 2 : w4 == 0 ? 0 : w4 + 1, w4 == 3);
      if (w4 == 0) put(1, 0);
      if (w4 == 3) put(3, 1);
    }
    // Every wave's loads of B (and S) of this chunk and its share of the mix
    // have arrived, and C (and S) is free.  (TWO: everything of this chunk has,
    // and the other buffers are free.)
    wait_vmcnt<0>();
    dma_barrier();
    if (c + 1 < c1) {
      fetch_c(c + 1);
      if (TWO) fetch_b(c + 1);
    }
    // the AFTER accesses that follow stay behind these
    asm volatile("" ::: "memory");
    if constexpr (SEG) scalars();
    load_raw(c + 1);
    if (t0 + Q > s.len) {  // past the end: zero (a NaN would meet the zeros of earlier rows)
#pragma unroll
      for (int sb = 0; sb < 4; ++sb)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (t0 + 16 * sb + 4 * g + v >= s.len) u[sb][v] = 0.f;
    }
#pragma unroll
    for (int sb = 0; sb < 4; ++sb)
#pragma unroll
      for (int v = 0; v < 4; ++v) sq = fmaf(u[sb][v], u[sb][v], sq);
    // A column's largest value from its sum of squares: at most 2^3 too much.
    // A value that is not finite must not meet the zeros of earlier rows (0 *
    // NaN): it leaves the products, and its column is NaN from its row on.
    bool poison = false;
    float maxu = 0.f;
    int from = Q;
    if constexpr (!SEG) maxu = sqrtf(rows_sum(sq));
    if (__any(!(sq < INFINITY))) {  // or a value beyond 2^63
      float m = 0.f;
#pragma unroll
      for (int sb = 0; sb < 4; ++sb)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          m = max_finite(m, u[sb][v]);
          if (!(fabsf(u[sb][v]) < INFINITY)) {
            u[sb][v] = 0.f;
            from = min(from, 16 * sb + 4 * g + v);
          }
        }
      from = min(from, __shfl_xor(from, 16));
      from = min(from, __shfl_xor(from, 32));
      poison = __any(from < Q);
      m = rows_max(m);
      if (!(maxu < INFINITY)) maxu = m;
    }
    __builtin_amdgcn_sched_barrier(0);  // (the fences keep one phase's registers from another's)
    if constexpr (!SEG) {
      // ---- C h with the decay since the chunk's start, and the skip term
      const int ku = exp_for(maxu), kch = -(exp_for(maxc) + kh);
      const float su = pow2(ku);
#pragma unroll
      for (int tb = 0; tb < 4; ++tb) {
        const f32x4 e = *reinterpret_cast<const f32x4*>(dtp + 16 * tb + 4 * g);
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[tb][v] = fmaf(dh, u[tb][v], __builtin_ldexpf(acc[tb][v] * e[v], kch));
      }
      // ---- earlier rows of the chunk, and the row itself
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = su * u[2 * q + (i >> 2)][i & 3];
        const HiLo uf = split8(v);
#pragma unroll
        for (int tb = 2 * q; tb < 4; ++tb) {
          HiLo mf;
          i32x4 k;  // of rows 16 tb + 4 g + 0..3
          if constexpr (SHARE) {
            mf.hi = mixes[(tb + 2 * q) * 128];
            mf.lo = mixes[(tb + 2 * q) * 128 + 64];
            k = *reinterpret_cast<const i32x4*>(mixk + (tb + 2 * q) * 16 + 4 * g);
          } else {
            int own;
            mf = mix(tb, q, own);
#pragma unroll
            for (int v = 0; v < 4; ++v) k[v] = __shfl(own, 4 * g + v);
          }
          const f32x4 sum = mul3(mf, uf, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int v = 0; v < 4; ++v) acc[tb][v] += __builtin_ldexpf(sum[v], -(k[v] + ku));
        }
      }
      if (poison) {
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (16 * tb + 4 * g + v >= from) acc[tb][v] = NAN;
      }
      // stores past the last row (or column) are outside the range, and dropped
      const unsigned yrow = (unsigned)a.ys * (unsigned)sizeof(T);
      const __amdgpu_buffer_rsrc_t ry =
          make_rsrc(static_cast<T*>(a.y) + (s.first + t0) * a.ys, (long long)min(s.len - t0, Q) * yrow);
      unsigned yo = 4 * g * yrow + (unsigned)ch0 * (unsigned)sizeof(T);
      asm volatile("" : "+v"(yo));
#pragma unroll
      for (int tb = 0; tb < 4; ++tb)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const T o = from_f<T>(acc[tb][v]);
          const unsigned off = yo + (16 * tb + v) * yrow;
          const int to_ = (int)(have ? off : kOOB);
          if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, o), ry, to_, 0, 0);
          else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, o), ry, to_, 0, 0);
        }
    }
    // ---- the state after the chunk
    __builtin_amdgcn_sched_barrier(0);
    const float e = __builtin_amdgcn_exp2f(cend);
    float uf[4][4], most = 0.f;
#pragma unroll
    for (int sb = 0; sb < 4; ++sb) {
      const f32x4 f = *reinterpret_cast<const f32x4*>(dtp + 4 * Q + 16 * sb + 4 * g);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        uf[sb][v] = u[sb][v] * f[v];
        most = fmaxf(most, fabsf(uf[sb][v]));
      }
    }
    const int kf = exp_for(rows_max(most)), kadd = -(exp_for(maxb) + kf);
    const float sf = pow2(kf);
    HiLo xf[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = sf * uf[2 * q + (i >> 2)][i & 3];
      xf[q] = split8(v);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      f32x4 add = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const f16* bp = Bg + (nt * 2 + q) * 1024;
        HiLo bf;
        bf.hi = *reinterpret_cast<const f16x8*>(bp);
        bf.lo = *reinterpret_cast<const f16x8*>(bp + 512);
        add = mul3(bf, xf[q], add);
      }
#pragma unroll
      for (int v = 0; v < 4; ++v) st[nt][v] = fmaf(st[nt][v], e, __builtin_ldexpf(add[v], kadd));
    }
    total += cend;
    if (poison) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
        if (from < Q) st[nt] = f32x4{NAN, NAN, NAN, NAN};
    }
    if constexpr (!TWO) {
      // every wave's loads of C and its decays for the next chunk have arrived
      // (the newest AFTER are not among them), and B (and S) is free
      wait_vmcnt<AFTER>();
      dma_barrier();
      if (c + 1 < c1) fetch_b(c + 1);
    }
  }
  if (SEG) {
    store_state(seg_state(seg + 1));
    if (lane == 0 && live && unit % pblocks == 0) a.ws_decay[seg_slot(seg + 1)] = total;
  } else if (a.state_out && (c1 == nc && (c0 < c1 || seg == 0))) {
    // the segment with the sequence's last chunk (segment 0 of a sequence without rows)
    store_state(a.state_out + ((int64_t)b * a.heads + h) * hold);
  }
}

// States over the segments, if there are many: slot i, with what segment i - 1
// adds, takes the state in front of segment i.  Bound by one load after the
// other, each behind the store of the segment before it (8 segments of 64 heads
// of 64 x 128: 8 us).
__global__ __launch_bounds__(256) void scan_carry_kernel(ScanArgs a) {
  const int64_t hold = (int64_t)a.dim * a.state, e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int b = blockIdx.z, h = blockIdx.y;
  if (e >= hold) return;
  const Seq s = seq_of(a, b);
  const int nc = (s.len + Q - 1) / Q;
  if (a.per >= nc) return;  // one segment, from the sequence's own state
  const int64_t slot = segment0_of(a, s.first, b) * a.heads + h;
  float* p = a.ws_seg + slot * hold + e;
  float v = a.state_in ? a.state_in[((int64_t)b * a.heads + h) * hold + e] : 0.f;
  *p = v;
  for (int i = 1; i * a.per < nc; ++i) {
    p += a.heads * hold;
    v = fmaf(v, __builtin_amdgcn_exp2f(a.ws_decay[slot + (int64_t)i * a.heads]), *p);
    *p = v;
  }
}

// ------------------------------------------------------------------ one token per sequence
// grid (heads x splits of a head's rows p, sequences).  A quad of state columns
// per thread; L threads (a power of two) side by side hold a row.  The state
// is read first: its bytes bound the kernel.  The workgroups of a group all
// read the window of B and C; when it is updated in place, the last of them
// to have read it (counted per sequence and group) writes it.
// PASS: quads of a thread.  More share the convolution of B and C among more
// rows, fewer make more workgroups when there are few sequences.
// 64 heads of 64 x 128 in bf16: 64 sequences 61 us, 4.4 TB/s (a copy of gigabytes
// reaches 4.8); 8 sequences 12 us; one 5.8 us, most of it the launch and the way
// from the window over the convolution to the state.
template <typename T, int PASS>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanArgs a, int L, int splits) {
  __shared__ float sbc[2][256], sx[256 * PASS];
  __shared__ unsigned last;
  const int b = blockIdx.y, h = blockIdx.x / splits, split = blockIdx.x % splits;
  const int N = a.state, each = a.heads / a.groups, grp = h / each;
  const int rows = 256 / L, q = threadIdx.x % L, r = threadIdx.x / L;
  const int pb = split * rows * PASS, inner = a.heads * a.dim;
  const int64_t hold = (int64_t)a.dim * N, at = ((int64_t)b * a.heads + h) * hold;
  f32x4 st[PASS];
#pragma unroll
  for (int i = 0; i < PASS; ++i) {
    const int p = pb + i * rows + r, n = 4 * q;
    st[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (p < a.dim && n < N && a.state_in) {
      const float* sp = a.state_in + at + (int64_t)p * N + n;
      if (a.vec_state) st[i] = *reinterpret_cast<const f32x4*>(sp);
      else
#pragma unroll
        for (int v = 0; v < 4; ++v) st[i][v] = n + v < N ? sp[v] : 0.f;
    }
  }
  // channels of this workgroup: its p rows of X, then the group's B and C
  const int px = min(rows * PASS, a.dim - pb), items = px + 2 * N, keep = a.conv - 1;
  const T* win = static_cast<const T*>(a.window);
  T* wout = static_cast<T*>(a.window_out);
  const bool in_place = a.window_out == a.window;
  constexpr int ITEMS = PASS + 2;
  T now[ITEMS][4];  // raw values of the thread's channels, for the new window
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int it = i * 256 + threadIdx.x;
    if (it >= items) break;
    const int e = it - px;
    const int ch = it < px ? h * a.dim + pb + it : inner + (e < N ? grp * N + e : a.groups * N + grp * N + e - N);
    float w[4], v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int kk = k - (4 - a.conv);  // which of the conv values, oldest first
      now[i][k] = kk < 0 ? from_f<T>(0.f)
                  : kk == keep ? static_cast<const T*>(a.x)[b * a.xs + ch]
                  : win        ? win[((int64_t)b * keep + kk) * a.chans + ch]
                               : from_f<T>(0.f);
      w[k] = a.conv_w[k * a.chans + ch];
      v[k] = to_f(now[i][k]);
    }
    const float u = silu_f(taps4(w, a.conv_b[ch], v[0], v[1], v[2], v[3], a.conv));
    if (it < px) sx[it] = u;
    else if (e < N) sbc[0][e] = u;
    else sbc[1][e - N] = u;
    if (it < px && wout)  // only this thread touches the channel
#pragma unroll
      for (int k = 1; k < 4; ++k)
        if (k >= 4 - keep) wout[((int64_t)b * keep + k - 4 + keep) * a.chans + ch] = now[i][k];
  }
  const float v = to_f(static_cast<const T*>(a.dt)[b * a.dts + h]) + a.dt_bias[h];
  const float dt = v > 20.f ? v : log1pf(expf(v));
  const float decay = __builtin_amdgcn_exp2f(dt * a.a2[h]);
  __syncthreads();  // every read of the window has arrived, too
  if (wout && keep > 0) {
    if (in_place) {
      if (threadIdx.x == 0) {
        const unsigned n = (unsigned)(each * splits);
        unsigned* cnt = a.count + (int64_t)b * a.groups + grp;
        last = atomicAdd(cnt, 1u) + 1 == n;
        if (last) *cnt = 0;
      }
      __syncthreads();
    }
    if (in_place ? last != 0 : (h % each == 0 && split == 0)) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int e = i * 256 + (int)threadIdx.x - px;
        if (e < 0 || e >= 2 * N) continue;
        const int ch = inner + (e < N ? grp * N + e : a.groups * N + grp * N + e - N);
#pragma unroll
        for (int k = 1; k < 4; ++k)
          if (k >= 4 - keep) wout[((int64_t)b * keep + k - 4 + keep) * a.chans + ch] = now[i][k];
      }
    }
  }
  f32x4 B = {0.f, 0.f, 0.f, 0.f}, C = B;
  if (4 * q < N)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (4 * q + k < N) B[k] = sbc[0][4 * q + k], C[k] = sbc[1][4 * q + k];
#pragma unroll
  for (int i = 0; i < PASS; ++i) {
    const int p = pb + i * rows + r, n = 4 * q;
    const float x = p < a.dim ? sx[i * rows + r] : 0.f, xd = dt * x;
    float y = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      st[i][k] = fmaf(st[i][k], decay, xd * B[k]);
      if (n + k < N) y = fmaf(st[i][k], C[k], y);
    }
    for (int d = L / 2; d > 0; d /= 2) y += __shfl_xor(y, d);
    if (p < a.dim && n < N && a.state_out) {
      float* sp = a.state_out + at + (int64_t)p * N + n;
      if (a.vec_state) *reinterpret_cast<f32x4*>(sp) = st[i];
      else
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (n + k < N) sp[k] = st[i][k];
    }
    if (q == 0 && p < a.dim) static_cast<T*>(a.y)[b * a.ys + h * a.dim + p] = from_f<T>(fmaf(a.d[h], x, y));
  }
}

// ------------------------------------------------------------------ launchers
template <typename T, int NT, bool SHARE>
static void launch_main(const ScanArgs& a, hipStream_t st) {
  const int units = a.heads / a.groups * ((a.dim + 15) / 16), waves = std::min(kScanWaves, units);
  auto grid = [&](int w) { return dim3((unsigned)((int64_t)a.segs * a.seqs * a.groups * ((units + w - 1) / w))); };
  if (a.segs > 1) {
    // half the waves: three of its workgroups fit a CU
    const int ws = std::min(4, units);
    SN_LAUNCH((scan_main_kernel<T, NT, false, true>), grid(ws), dim3(64 * ws), (scan_lds<NT, false, true>(ws)), st, a);
    if (a.carried) SN_LAUNCH((scan_carry_kernel), dim3((a.dim * a.state + 255) / 256, a.heads, a.seqs), dim3(256), 0, st, a);
  }
  SN_LAUNCH((scan_main_kernel<T, NT, SHARE, false>), grid(waves), dim3(64 * waves), (scan_lds<NT, SHARE, false>(waves)), st, a);
}
template <typename T, bool SHARE>
static void launch_np(const ScanArgs& a, hipStream_t st) {
  if (a.np == 32) launch_main<T, 2, SHARE>(a, st);
  else if (a.np == 64) launch_main<T, 4, SHARE>(a, st);
  else if (a.np == 128) launch_main<T, 8, SHARE>(a, st);
  else if constexpr (!SHARE) launch_main<T, 16, SHARE>(a, st);
}

template <typename T>
static void launch_scan(ScanArgs a, hipStream_t st) {
  a.vec_state = a.state % 4 == 0 && al16(a.state_in) && al16(a.state_out) && al16(a.ws_seg);
  const int64_t slots = scan_slots(a.tokens, a.seqs);
  const int64_t copies = std::min<int64_t>(8, (int64_t)a.seqs * (a.conv - 1) * a.chans / (slots * kPrep) + 1);
  const dim3 grid((unsigned)slots, (unsigned)(a.groups + (a.heads + 15) / 16 + copies));
  const size_t lds = (2 * Q * (a.np + 4) + 2 * kPrep / 64) * sizeof(float);
  if (a.np == 32) SN_LAUNCH((scan_prep_kernel<T, 32>), grid, dim3(kPrep), lds, st, a);
  else if (a.np == 64) SN_LAUNCH((scan_prep_kernel<T, 64>), grid, dim3(kPrep), lds, st, a);
  else if (a.np == 128) SN_LAUNCH((scan_prep_kernel<T, 128>), grid, dim3(kPrep), lds, st, a);
  else SN_LAUNCH((scan_prep_kernel<T, 256>), grid, dim3(kPrep), lds, st, a);
  // with 64 columns per head or a multiple, four waves of one share its mix
  // (4096 tokens of 64 heads: 126 us against 135 for all launches; 3 x 511 of 24:
  // 41 against 44; 4096 of 32 x 128 x 16: 79 against 90); beside 256 state rows LDS has
  // no room for it
  if ((a.dim + 15) / 16 % 4 == 0 && a.np <= 128) launch_np<T, true>(a, st);
  else launch_np<T, false>(a, st);
}

constexpr int64_t kStepBlocks = 512;
template <typename T>
static void launch_step(ScanArgs a, hipStream_t st) {
  a.vec_state = a.state % 4 == 0 && al16(a.state_in) && al16(a.state_out);
  int L = 1;
  while (4 * L < a.state) L *= 2;
  auto splits = [&](int pass) { return (a.dim + pass * (256 / L) - 1) / (pass * (256 / L)); };
  // as many quads as a head has rows for, if that leaves kStepBlocks workgroups.
  // 64 heads of 64 x 128, us with two, four, eight quads: 1 sequence 5.9, 7.0, 9.7;
  // 4: 8.6, 8.5, 10.6; 8: 13.2, 11.1, 12.5; 16: 21.8, 19.8, 17.8; 64: 71, 58, 60
  auto fits = [&](int pass) {
    return pass * (256 / L) <= std::max(a.dim, 8) && (int64_t)a.seqs * a.heads * splits(pass) >= kStepBlocks;
  };
  auto grid = [&](int pass) { return dim3((unsigned)(a.heads * splits(pass)), a.seqs); };
  if (fits(8)) SN_LAUNCH((scan_step_kernel<T, 8>), grid(8), dim3(256), 0, st, a, L, splits(8));
  else if (fits(4)) SN_LAUNCH((scan_step_kernel<T, 4>), grid(4), dim3(256), 0, st, a, L, splits(4));
  else SN_LAUNCH((scan_step_kernel<T, 2>), grid(2), dim3(256), 0, st, a, L, splits(2));
}

// Up to this many state rows of segments, each segment finds the state in front
// of it from those that the earlier ones add by itself, instead of a launch that
// does so for all: 2 segments of 128 rows 47.1 -> 44.8 us, 4 of 64 43.5 -> 42.4,
// 8 of 16 (counted as 32) 83.2 -> 80.0; but 8 of 64 97.9 -> 98.7, 8 of 128 121.4
// -> 124.9 and 32 of 256 99 -> 186, a load's latency and more for each.
constexpr int kScanCarry = 256;

// Segments: as many chunks to each as leave kScanUnits waves, at least two (a
// segment's chunks but the last one's are read twice, and its state is written
// and read); one if there are more waves anyhow, or the states found no room.
// us with 1024, 2048, 4096 waves: 1024 tokens of 64 heads of 64 x 128 74, 67, 67;
// 4096 182, 120, 135; 16384 of 8 heads 114, 92, 121; 4096 of 24 heads of 64 x 64
// 73, 76, 70.
static void scan_split(ScanArgs& a) {
  a.each = a.tokens / a.seqs;
  const int64_t slots = scan_slots(a.tokens, a.seqs), units = (int64_t)a.heads * ((a.dim + 15) / 16);
  const int64_t chunks = ((a.offsets ? a.tokens : a.each) + Q - 1) / Q;  // the most that one sequence may have
  const int64_t hold = (int64_t)a.heads * a.dim * a.state;
  int64_t per = std::max<int64_t>(2, ((a.tokens + Q - 1) / Q * units + kScanUnits - 1) / kScanUnits);
  while (per < chunks && scan_segment_slots(slots, a.seqs, (int)per) * hold > a.seg_cap) ++per;
  a.per = (int)std::max<int64_t>(1, std::min(per, chunks));
  a.segs = (int)std::max<int64_t>(1, (chunks + a.per - 1) / a.per);
  a.carried = a.segs * a.np > kScanCarry;
}

void scan_run(const ScanArgs& in, hipStream_t st) {
  ScanArgs a = in;
  check(a.heads >= 1 && a.groups >= 1 && a.heads % a.groups == 0 && a.dim >= 1 && a.state >= 1 && a.state <= 256 &&
            a.conv >= 1 && a.conv <= 4 && a.seqs >= 1 && a.seqs <= 65535 && a.tokens >= 0,
        "scan shapes");
  scan_split(a);
  check((int64_t)a.segs * a.seqs * a.groups * ((a.heads / a.groups * (int64_t)((a.dim + 15) / 16) + 3) / 4) * 64 * kScanWaves <
            (int64_t(1) << 32),
        "scan of more workgroups than a launch takes");
  if (a.dtype == 0) launch_scan<float>(a, st);
  else if (a.dtype == 1) launch_scan<f16>(a, st);
  else launch_scan<bf16>(a, st);
}

void scan_step(const ScanArgs& a, hipStream_t st) {
  check(a.heads >= 1 && a.groups >= 1 && a.heads % a.groups == 0 && a.dim >= 1 && a.state >= 1 && a.state <= 256 &&
            a.conv >= 1 && a.conv <= 4 && a.seqs >= 1 && a.seqs <= 65535 && a.tokens == a.seqs,
        "scan step shapes");
  if (a.dtype == 0) launch_step<float>(a, st);
  else if (a.dtype == 1) launch_step<f16>(a, st);
  else launch_step<bf16>(a, st);
}

}  // namespace k
}  // namespace sn
