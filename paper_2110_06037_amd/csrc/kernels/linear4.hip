// Products with 4-bit weights and group scales on MFMA.
//
//   y[m][k] = act(sum_c x[m][c] s[k][c / g] (q[k][c] - z[k][c / g]) + b[k])
//
// The weights are laid out once (linear4_pack) in the order in which MFMA's
// second operand wants them: a block of 16 features k by 128 inputs c is 1 KB,
// lane l holding feature l % 16 and the inputs 32 i + 8 (l / 16) + 0..7 of
// step i in its i-th dword.  A wave reads a block as one run of 16 bytes per
// lane, and no weight passes through LDS.
//
// Codes become 16-bit floats by or-ing them into the low mantissa bits of a
// constant (two weights per instruction).  f16: 1024 + q or 64 + q, less 1024 +
// z or 64 + z in one packed subtraction: q - z exactly.  bf16: 128 + q, and
// the 128 + z come off the sums instead, (128 + z) sum_c x[m][c], with the
// sums over x from an MFMA against ones: cheaper than any exact form, at a
// cost of 2^-24 * 143 of the terms' sizes in float32, far below a bf16
// rounding.  float32: x as the exact sum of three bf16 parts, which are three
// rows of the first operand, times q - z exactly in bf16.  Products are exact,
// sums float32; a group's scale multiplies the float32 sum of its run.
#include "seq.hpp"

namespace sn {
namespace k {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------ layout
// One thread per dword of codes; scales and zero points per run of 32 GS
// inputs: [block row][block column][16 features][4 / GS].
__global__ __launch_bounds__(256) void linear4_pack_kernel(const uint8_t* q, const f16* scale, const uint8_t* zero,
                                                           int rows, int cols, int group, int gs, unsigned* wq, f16* ws,
                                                           uint8_t* wz) {
  const int cbs = (cols + 127) / 128, groups = (cols + group - 1) / group, pairs = (cols + 1) / 2;
  const int64_t total = (int64_t)((rows + 15) / 16) * cbs * 256, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  const int step = (int)(i & 3), lane = (int)(i >> 2) & 63;
  const int64_t blk = i >> 8;
  const int row = (int)(blk / cbs) * 16 + (lane & 15), c0 = (int)(blk % cbs) * 128;
  const int c = c0 + 32 * step + 8 * (lane >> 4);
  unsigned w = 0;
  for (int e = 0; e < 8; ++e) {
    unsigned code = 8;  // meets an input of zero, or is of no feature
    if (row < rows && c + e < cols) code = q[(int64_t)row * pairs + (c + e) / 2] >> (4 * ((c + e) & 1)) & 15;
    // dword bits: inputs 0, 2, 4, 6 from the low half up, 1, 3, 5, 7 from the high half
    w |= code << (4 * (e / 2) + 16 * (e & 1));
  }
  wq[i] = w;
  const int runs = 4 / gs;
  if (step < runs && lane < 16) {
    const int cr = c0 + 32 * gs * step;
    const bool in = row < rows && cr < cols;
    const int64_t from = (int64_t)row * groups + cr / group, to = (blk * 16 + lane) * runs + step;
    ws[to] = in ? scale[from] : (f16)0.f;
    if (wz) wz[to] = in ? zero[from] : 8;
  }
}

// ------------------------------------------------------------------ weights to floats
// v_and_or_b32 takes one scalar: the mask stays in a register
__device__ __forceinline__ unsigned and_or(unsigned w, unsigned mask, unsigned magic) { return (w & mask) | magic; }

__device__ __forceinline__ f16x8 deq_f16(unsigned w, f16x2 z1024, f16x2 z64) {
  f16x2 r[4];
  r[0] = __builtin_bit_cast(f16x2, and_or(w, 0x000f000fu, 0x64006400u)) - z1024;
  r[1] = __builtin_bit_cast(f16x2, and_or(w, 0x00f000f0u, 0x54005400u)) - z64;
  w >>= 8;
  r[2] = __builtin_bit_cast(f16x2, and_or(w, 0x000f000fu, 0x64006400u)) - z1024;
  r[3] = __builtin_bit_cast(f16x2, and_or(w, 0x00f000f0u, 0x54005400u)) - z64;
  return __builtin_bit_cast(f16x8, r);
}
__device__ __forceinline__ bf16x8 deq_bf16_128(unsigned w) {  // 128 + q
  u32x4 r;
  r[0] = and_or(w, 0x000f000fu, 0x43004300u);
  r[1] = and_or(w >> 4, 0x000f000fu, 0x43004300u);
  r[2] = and_or(w >> 8, 0x000f000fu, 0x43004300u);
  r[3] = and_or(w >> 12, 0x000f000fu, 0x43004300u);
  return __builtin_bit_cast(bf16x8, r);
}
// q - z: the two halves of a pair are the high halves of the floats 128 + q
__device__ __forceinline__ bf16x8 deq_bf16(unsigned w, float z128) {
  u32x4 r = __builtin_bit_cast(u32x4, deq_bf16_128(w));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float lo = __builtin_bit_cast(float, r[i] << 16) - z128, hi = __builtin_bit_cast(float, r[i] & 0xffff0000u) - z128;
    r[i] = __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, hi), __builtin_bit_cast(unsigned, lo), 0x07060302u);
  }
  return __builtin_bit_cast(bf16x8, r);
}

// ------------------------------------------------------------------ inputs
// 8 consecutive inputs of a row from c on, 0 past its end; vec: aligned, and
// whole chunks of 8.
template <typename T>
__device__ __forceinline__ V8<T> ld_x(const T* row, int c, int cols, bool vec) {
  if (vec) return c < cols ? ld8(row + c) : zero8<T>();
  V8<T> r;
#pragma unroll
  for (int j = 0; j < 8; ++j) r.v[j] = c + j < cols ? row[c + j] : (T)0.f;
  return r;
}
// Part 0, 1 or 2 of float32 values as bf16: the leading 8 significant bits,
// the next 8, the last 8, each the value less the parts before it (exact).
__device__ __forceinline__ float rest_f(float x) {
  const float top = __builtin_bit_cast(float, __builtin_bit_cast(unsigned, x) & 0xffff0000u);
  return x == top ? 0.f : x - top;  // an infinity has no rest
}
__device__ __forceinline__ bf16x8 top_bf16(const float (&v)[8]) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r[i] = __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, v[2 * i + 1]), __builtin_bit_cast(unsigned, v[2 * i]), 0x07060302u);
  return __builtin_bit_cast(bf16x8, r);
}
// A NaN whose set bits all lie in the low half would read as an infinity
__device__ __forceinline__ float quiet(float x) { return x == x ? x : NAN; }
__device__ __forceinline__ bf16x8 part_of(V8<float> x, int part) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float v = quiet(x.v[j]);
    const float r1 = rest_f(v), r2 = rest_f(r1);
    x.v[j] = part == 0 ? v : part == 1 ? r1 : part == 2 ? r2 : 0.f;
  }
  return top_bf16(x.v);
}

template <typename T>
struct Op4 {
  typedef typename std::conditional<std::is_same<T, f16>::value, f16, bf16>::type E;  // MFMA's element
  typedef typename Mfma<E>::frag frag;
};

// ------------------------------------------------------------------ few rows
// A workgroup owns 16 features; its waves take the blocks of 128 inputs in
// turn, U at a time with all their loads in flight, and their sums meet in
// LDS.  x goes from global memory (its rows are shared by all workgroups and
// stay in the caches) straight to the first operand: row r = 4 g + v of it is
// row 4 v + g of x, so that up to 4 rows have all their sums in element v = 0
// (MV = 1); in float32 v is the part and g the row.
template <typename T, int NB, int MV, int GS>
__global__ __launch_bounds__(1024) void linear4_rows_kernel(Linear4Args a) {
  typedef typename Op4<T>::E E;
  typedef typename Op4<T>::frag frag;
  constexpr bool F32 = std::is_same<T, float>::value;
  constexpr bool BIASED = std::is_same<T, bf16>::value;
  constexpr int RUNS = 4 / GS, U = NB >= 4 ? 2 : 4;
  constexpr int PER = F32 ? 4 : 4 * MV;  // rows of x per block of the first operand
  constexpr int NV = F32 ? 1 : MV;       // results per lane and block
  extern __shared__ float red[];         // [wave][NB][NV][64]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int col = lane & 15, g = lane >> 4, xr = lane & 15;
  const int cbs = (a.cols + 127) / 128;
  const int64_t blk0 = (int64_t)blockIdx.x * cbs;
  const u32x4* wq = reinterpret_cast<const u32x4*>(a.wq) + blk0 * 64 + lane;
  const f16* ws = a.ws + (blk0 * 16 + col) * RUNS;
  const uint8_t* wz = a.wz ? a.wz + (blk0 * 16 + col) * RUNS : nullptr;
  // this lane's rows of x
  const T* x = static_cast<const T*>(a.x);
  const T* xrow[NB];
  bool on[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int v = xr & 3;
    const int64_t m = (int64_t)(blockIdx.y * NB + nb) * PER + (F32 ? xr >> 2 : 4 * v + (xr >> 2));
    on[nb] = m < a.m && v < (F32 ? 3 : MV);
    xrow[nb] = x + (on[nb] ? m : 0) * a.xs;
  }
  float tot[NB][NV] = {};
  const frag ones = __builtin_bit_cast(frag, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
  for (int c0 = wave; c0 < cbs; c0 += waves * U) {
    u32x4 w[U];
    f16 sc[U][RUNS];
    uint8_t zp[U][RUNS];
    V8<T> xv[U][NB][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int cb = c0 + u * waves;
      if (cb >= cbs) break;
      w[u] = __builtin_nontemporal_load(wq + (int64_t)cb * 64);
      __builtin_memcpy(sc[u], ws + (int64_t)cb * 16 * RUNS, 2 * RUNS);
      if (wz) __builtin_memcpy(zp[u], wz + (int64_t)cb * 16 * RUNS, RUNS);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          xv[u][nb][i] = on[nb] ? ld_x(xrow[nb], cb * 128 + 32 * i + 8 * g, a.cols, a.vec_x) : zero8<T>();
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int cb = c0 + u * waves;
      if (cb >= cbs) break;
#pragma unroll
      for (int run = 0; run < RUNS; ++run) {
        const float s = (float)sc[u][run], z = wz ? (float)zp[u][run] : 8.f;
        const f16 z1024 = (f16)(1024.f + z), z64 = (f16)(64.f + z);
        f32x4 acc[NB], xs[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[nb] = xs[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = run * GS; i < (run + 1) * GS; ++i) {
          frag wf;
          if constexpr (F32) wf = deq_bf16(w[u][i], 128.f + z);
          else if constexpr (BIASED) wf = deq_bf16_128(w[u][i]);
          else wf = deq_f16(w[u][i], f16x2{z1024, z1024}, f16x2{z64, z64});
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            frag xf;
            if constexpr (F32) xf = part_of(xv[u][nb][i], xr & 3);
            else xf = __builtin_bit_cast(frag, xv[u][nb][i]);
            acc[nb] = Mfma<E>::run(xf, wf, acc[nb]);
            if constexpr (BIASED) xs[nb] = Mfma<E>::run(xf, ones, xs[nb]);
          }
        }
        if constexpr (F32) {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) tot[nb][0] = fmaf(s, acc[nb][0] + (acc[nb][1] + acc[nb][2]), tot[nb][0]);
        } else if constexpr (BIASED) {
          // an infinity among the biased products (or a finite sum beyond the
          // range that only the bias brings there): the run again with q - z
          bool over = false;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int v = 0; v < NV; ++v) over = over || !(fabsf(acc[nb][v]) < INFINITY);
          float zz = 128.f + z;
          if (__any(over)) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) acc[nb] = xs[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = run * GS; i < (run + 1) * GS; ++i)
#pragma unroll
              for (int nb = 0; nb < NB; ++nb)
                acc[nb] = Mfma<E>::run(__builtin_bit_cast(frag, xv[u][nb][i]), deq_bf16(w[u][i], zz), acc[nb]);
          }
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int v = 0; v < NV; ++v) tot[nb][v] = fmaf(s, fmaf(-zz, xs[nb][v], acc[nb][v]), tot[nb][v]);
        } else {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int v = 0; v < NV; ++v) tot[nb][v] = fmaf(s, acc[nb][v], tot[nb][v]);
        }
      }
    }
  }
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int v = 0; v < NV; ++v) red[((wave * NB + nb) * NV + v) * 64 + lane] = tot[nb][v];
  __syncthreads();
  for (int i = threadIdx.x; i < NB * NV * 64; i += blockDim.x) {
    float s = 0.f;
    for (int w = 0; w < waves; ++w) s += red[w * NB * NV * 64 + i];
    const int l = i & 63, v = (i >> 6) % NV, nb = (i >> 6) / NV;
    const int64_t m = (int64_t)(blockIdx.y * NB + nb) * PER + (F32 ? l >> 4 : 4 * v + (l >> 4));
    const int k = blockIdx.x * 16 + (l & 15);
    if (m < a.m && k < a.rows)
      static_cast<T*>(a.y)[m * a.ys + k] = from_f<T>(act_f(s + (a.bias ? a.bias[k] : 0.f), a.act));
  }
}

// ------------------------------------------------------------------ many rows
// Tile of 64 rows of x by 64 RB features: each of 4 waves owns 16 RB features
// and all 64 rows, so no weight is turned into floats twice in a workgroup,
// and x alone goes through LDS, in the first operand's order (a wave loads its
// 16 rows of the next 128 inputs into registers while the current ones are
// multiplied).  bf16: the wave that loads 16 rows sums them against ones; the
// sums wait in LDS and the bias comes off at the end, as one more product.
template <typename T, int RB, int GS>
__global__ __launch_bounds__(256) void linear4_tile_kernel(Linear4Args a, int tiles_m, int tiles_n) {
  typedef typename Op4<T>::E E;
  typedef typename Op4<T>::frag frag;
  constexpr bool F32 = std::is_same<T, float>::value;
  constexpr bool BIASED = std::is_same<T, bf16>::value;
  constexpr int RUNS = 4 / GS, PARTS = F32 ? 3 : 1;
  extern __shared__ char smem[];
  // [stage][part][row block][step][lane] of 16 bytes, then the bias sums
  frag* xt = reinterpret_cast<frag*>(smem);
  constexpr int STAGE = PARTS * 4 * 4 * 64;
  float* xsum = reinterpret_cast<float*>(xt + 2 * STAGE);  // [run][64]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int cbs = (a.cols + 127) / 128, rbs = (a.rows + 15) / 16;
  int mt, nt;
  tile_of(blockIdx.x, tiles_m, tiles_n, mt, nt);
  const int64_t m0 = (int64_t)mt * 64;
  const T* xrow = static_cast<const T*>(a.x) + min(m0 + 16 * wave + col, a.m - 1) * a.xs;  // rows past m: any row's values
  const int rb0 = (nt * 4 + wave) * RB;
  int64_t blk[RB];  // first block of each of the wave's rows of blocks (past the last: the last's, not stored)
#pragma unroll
  for (int r = 0; r < RB; ++r) blk[r] = (int64_t)min(rb0 + r, rbs - 1) * cbs;
  f32x4 tot[4][RB];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int r = 0; r < RB; ++r) tot[i][r] = f32x4{0.f, 0.f, 0.f, 0.f};
  const frag ones = __builtin_bit_cast(frag, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
  V8<T> xn[4];
  u32x4 wn[RB];
  auto load = [&](int cb) {
#pragma unroll
    for (int r = 0; r < RB; ++r) wn[r] = (reinterpret_cast<const u32x4*>(a.wq) + (blk[r] + cb) * 64)[lane];
#pragma unroll
    for (int i = 0; i < 4; ++i) xn[i] = ld_x(xrow, cb * 128 + 32 * i + 8 * g, a.cols, a.vec_x);
  };
  auto put = [&](int stage, int cb) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (F32) {
#pragma unroll
        for (int p = 0; p < 3; ++p) xt[stage * STAGE + ((p * 4 + wave) * 4 + i) * 64 + lane] = part_of(xn[i], p);
      } else {
        xt[stage * STAGE + (wave * 4 + i) * 64 + lane] = __builtin_bit_cast(frag, xn[i]);
      }
    }
    if constexpr (BIASED) {
#pragma unroll
      for (int run = 0; run < RUNS; ++run) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = run * GS; i < (run + 1) * GS; ++i) s = Mfma<E>::run(__builtin_bit_cast(frag, xn[i]), ones, s);
        if (col == 0) *reinterpret_cast<f32x4*>(xsum + (cb * RUNS + run) * 64 + 16 * wave + 4 * g) = s;
      }
    }
  };
  load(0);
  put(0, 0);
  for (int cb = 0; cb < cbs; ++cb) {
    u32x4 w[RB];
    f16 sc[RB][RUNS];
    uint8_t zp[RB][RUNS];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      w[r] = wn[r];
      __builtin_memcpy(sc[r], a.ws + ((blk[r] + cb) * 16 + col) * RUNS, 2 * RUNS);
      if (a.wz) __builtin_memcpy(zp[r], a.wz + ((blk[r] + cb) * 16 + col) * RUNS, RUNS);
    }
    lds_barrier();  // the stage is written, and the other one no longer read
    if (cb + 1 < cbs) load(cb + 1);
    const frag* xc = xt + (cb & 1) * STAGE + lane;
#pragma unroll
    for (int run = 0; run < RUNS; ++run) {
      f32x4 acc[4][RB];
#pragma unroll
      for (int mi = 0; mi < 4; ++mi)
#pragma unroll
        for (int r = 0; r < RB; ++r) acc[mi][r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = run * GS; i < (run + 1) * GS; ++i) {
        frag wf[RB];
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          const float z = a.wz ? (float)zp[r][run] : 8.f;
          if constexpr (F32) {
            wf[r] = deq_bf16(w[r][i], 128.f + z);
          } else if constexpr (BIASED) {
            wf[r] = deq_bf16_128(w[r][i]);
          } else {
            const f16 z1024 = (f16)(1024.f + z), z64 = (f16)(64.f + z);
            wf[r] = deq_f16(w[r][i], f16x2{z1024, z1024}, f16x2{z64, z64});
          }
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
          for (int mi = 0; mi < 4; ++mi) {
            const frag xf = xc[((p * 4 + mi) * 4 + i) * 64];
#pragma unroll
            for (int r = 0; r < RB; ++r) acc[mi][r] = Mfma<E>::run(xf, wf[r], acc[mi][r]);
          }
      }
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        const float s = (float)sc[r][run];
#pragma unroll
        for (int mi = 0; mi < 4; ++mi)
#pragma unroll
          for (int v = 0; v < 4; ++v) tot[mi][r][v] = fmaf(s, acc[mi][r][v], tot[mi][r][v]);
      }
    }
    if (cb + 1 < cbs) put((cb + 1) & 1, cb + 1);
  }
  if constexpr (BIASED) {
    __syncthreads();
    for (int cb = 0; cb < cbs; ++cb)
#pragma unroll
      for (int run = 0; run < RUNS; ++run) {
        f32x4 xs[4];
#pragma unroll
        for (int mi = 0; mi < 4; ++mi) xs[mi] = *reinterpret_cast<const f32x4*>(xsum + (cb * RUNS + run) * 64 + 16 * mi + 4 * g);
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          const int64_t at = ((blk[r] + cb) * 16 + col) * RUNS + run;
          const float zs = (128.f + (a.wz ? (float)a.wz[at] : 8.f)) * (float)a.ws[at];
#pragma unroll
          for (int mi = 0; mi < 4; ++mi)
#pragma unroll
            for (int v = 0; v < 4; ++v) tot[mi][r][v] = fmaf(-zs, xs[mi][v], tot[mi][r][v]);
        }
      }
    // rows with an infinity or a NaN (or beyond the range by the bias alone)
    // again, with q - z, input by input
    bool over = false;
#pragma unroll
    for (int mi = 0; mi < 4; ++mi)
#pragma unroll
      for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int v = 0; v < 4; ++v) over = over || !(fabsf(tot[mi][r][v]) < INFINITY);
    if (__any(over)) {
#pragma unroll
      for (int mi = 0; mi < 4; ++mi)
#pragma unroll
        for (int r = 0; r < RB; ++r)
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            if (fabsf(tot[mi][r][v]) < INFINITY) continue;
            const int64_t m = min(m0 + 16 * mi + 4 * g + v, a.m - 1);
            const T* xp = static_cast<const T*>(a.x) + m * a.xs;
            float sum = 0.f;
            for (int c = 0; c < a.cols; ++c) {
              const int64_t b = blk[r] + c / 128, at = (b * 16 + col) * RUNS + c % 128 / (32 * GS);
              const unsigned dw = a.wq[(b * 64 + col + 16 * (c % 32 / 8)) * 4 + c % 128 / 32];
              const float q = (float)(dw >> (4 * (c % 8 / 2) + 16 * (c & 1)) & 15);
              sum = fmaf(to_f(xp[c]), (q - (a.wz ? (float)a.wz[at] : 8.f)) * (float)a.ws[at], sum);
            }
            tot[mi][r][v] = sum;
          }
    }
  }
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    const int k = (rb0 + r) * 16 + col;
    if (k >= a.rows) continue;
    const float b = a.bias ? a.bias[k] : 0.f;
#pragma unroll
    for (int mi = 0; mi < 4; ++mi)
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int64_t m = m0 + 16 * mi + 4 * g + v;
        if (m < a.m) static_cast<T*>(a.y)[m * a.ys + k] = from_f<T>(act_f(tot[mi][r][v] + b, a.act));
      }
  }
}

// ------------------------------------------------------------------ launchers
int linear4_gs(int group) { return group % 128 == 0 ? 4 : group % 64 == 0 ? 2 : 1; }
int64_t linear4_blocks(int rows, int cols) { return (int64_t)((rows + 15) / 16) * ((cols + 127) / 128); }

void linear4_pack(const uint8_t* q, const f16* scale, const uint8_t* zero, int rows, int cols, int group, unsigned* wq,
                  f16* ws, uint8_t* wz, hipStream_t st) {
  const int64_t blocks = linear4_blocks(rows, cols);
  check(blocks < (int64_t(1) << 31), "4-bit weights");
  SN_LAUNCH(linear4_pack_kernel, dim3((unsigned)blocks), dim3(256), 0, st, q, scale, zero, rows, cols, group,
            linear4_gs(group), wq, ws, wz);
}

template <typename T, int NB, int MV, int GS>
static void launch_rows(const Linear4Args& a, hipStream_t st) {
  constexpr int PER = std::is_same<T, float>::value ? 4 : 4 * MV, NV = std::is_same<T, float>::value ? 1 : MV;
  const int cbs = (a.cols + 127) / 128;
  const int waves = cbs <= 4 ? 4 : cbs <= 64 ? 8 : 16;
  const dim3 grid((a.rows + 15) / 16, (unsigned)((a.m + NB * PER - 1) / (NB * PER)));
  SN_LAUNCH((linear4_rows_kernel<T, NB, MV, GS>), grid, dim3(64 * waves), waves * NB * NV * 256, st, a);
}

template <typename T, int RB, int GS>
static void launch_tile(const Linear4Args& a, hipStream_t st) {
  const int tm = (int)((a.m + 63) / 64), tn = (a.rows + 64 * RB - 1) / (64 * RB), cbs = (a.cols + 127) / 128;
  const int parts = std::is_same<T, float>::value ? 3 : 1;
  const size_t lds = 2 * parts * 16384 + (std::is_same<T, bf16>::value ? (size_t)cbs * (4 / GS) * 256 : 0);
  SN_LAUNCH((linear4_tile_kernel<T, RB, GS>), dim3((unsigned)(tm * tn)), dim3(256), lds, st, a, tm, tn);
}

template <typename T, int GS>
static void launch_linear4(const Linear4Args& a, hipStream_t st) {
  constexpr bool F32 = std::is_same<T, float>::value;
  // the tile kernel keeps the sums of bf16 inputs in LDS: 64 KB less its stages
  const bool fits = !std::is_same<T, bf16>::value || (int64_t)((a.cols + 127) / 128) * (4 / GS) <= 128;
  if (a.m > (F32 ? 16 : 64) && fits) {
    if ((a.m + 63) / 64 * ((a.rows + 255) / 256) >= 256) launch_tile<T, 4, GS>(a, st);
    else launch_tile<T, 1, GS>(a, st);
    return;
  }
  if constexpr (F32) {
    if (a.m <= 4) launch_rows<T, 1, 1, GS>(a, st);
    else if (a.m <= 8) launch_rows<T, 2, 1, GS>(a, st);
    else launch_rows<T, 4, 1, GS>(a, st);
  } else {
    if (a.m <= 4) launch_rows<T, 1, 1, GS>(a, st);
    else if (a.m <= 16) launch_rows<T, 1, 4, GS>(a, st);
    else if (a.m <= 32) launch_rows<T, 2, 4, GS>(a, st);
    else launch_rows<T, 4, 4, GS>(a, st);
  }
}

void linear4(const Linear4Args& in, hipStream_t st) {
  Linear4Args a = in;
  check(a.m >= 1 && a.rows >= 1 && a.cols >= 1 && a.group >= 32 && a.group % 32 == 0 && a.m <= 65535 * 4, "4-bit product shapes");
  const int e = a.dtype == 0 ? 4 : 2;
  a.vec_x = a.cols % 8 == 0 && al16(a.x) && al16(a.xs * e);
#define SN_L4(T)                                         \
  switch (linear4_gs(a.group)) {                         \
    case 4: launch_linear4<T, 4>(a, st); break;          \
    case 2: launch_linear4<T, 2>(a, st); break;          \
    default: launch_linear4<T, 1>(a, st); break;         \
  }
  if (a.dtype == 0) SN_L4(float)
  else if (a.dtype == 1) SN_L4(f16)
  else SN_L4(bf16)
#undef SN_L4
}

}  // namespace k
}  // namespace sn
