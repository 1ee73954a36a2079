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
// Codes become 16-bit floats by or-ing them into the mantissa of a constant, two
// weights per instruction (the published way from small integers to floats
// without a conversion).  f16: 1024 + q or 64 + q, less 1024 + z or 64 + z in
// one packed subtraction: q - z exactly.  bf16: 16 + q (the code in bits 3 to 6
// of 7), and the 16 + z come off the sums instead, (16 + z) sum_c x[m][c], with
// the sums over x from an MFMA against ones: cheaper than any exact form.  The
// sums that carry it are float32 and at most 31 times their inputs' sizes; it
// comes off after every run (few rows) or every 4 runs (many), so that no sum
// of a whole row carries it: with inputs of one sign, 2048 of them and results
// of 0, errors of 1.5 * 2^-24 of the terms' sizes in the root mean square (few
// rows: 0.05).  float32: x as the exact sum of three bf16 parts, which are three
// rows of the first operand, times q - z exactly in bf16.  Products are exact,
// sums float32; a group's scale multiplies the float32 sum of its run.
#include "seq.hpp"

namespace sn {
namespace k {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// ------------------------------------------------------------------ layout
// One thread per dword of codes; per run of 32 GS inputs a word of scale (low
// half, binary16) and zero point: [block row][block column][16 features][4 / GS].
__global__ __launch_bounds__(256) void linear4_pack_kernel(const uint8_t* q, const f16* scale, const uint8_t* zero,
                                                           int rows, int cols, int group, int gs, int up,
                                                           unsigned* wq, unsigned* ws) {
  // (a group may be nearly 2^31 wide: unsigned, the sum does not overflow)
  const int cbs = (cols + 127) / 128, groups = ((unsigned)cols + (unsigned)group - 1) / group, pairs = (cols + 1) / 2;
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
  wq[i] = up ? w << up | w >> (32 - up) : w;  // rotated to where bf16 wants the first pair
  const int runs = 4 / gs;
  if (step < runs && lane < 16) {
    const int cr = c0 + 32 * gs * step;
    const bool in = row < rows && cr < cols;
    const int64_t from = (int64_t)row * groups + cr / group, to = (blk * 16 + lane) * runs + step;
    ws[to] = in ? __builtin_bit_cast(uint16_t, scale[from]) | (unsigned)(zero ? zero[from] : 8) << 16 : 0u;
  }
}

// ------------------------------------------------------------------ weights to floats
// A constant in a vector register whose value the compiler does not see: (w &
// mask) | it is one v_and_or_b32 then (of two known constants the compiler
// makes two instructions with literals).
__device__ __forceinline__ unsigned vconst(unsigned v) {
  asm("" : "+v"(v));
  return v;
}
__device__ __forceinline__ float act4(float v, int act) {  // a NaN stays one
  if (act != ACT_NONE && v < 0.f) v = 0.f;
  return act == ACT_RELU6 && v > 6.f ? 6.f : v;
}
// A run's scale and zero point.
struct Run4 {
  float s, z;
  unsigned z1024, z64;  // pairs of 1024 + z and 64 + z in f16
  __device__ __forceinline__ explicit Run4(unsigned w) {
    s = (float)__builtin_bit_cast(f16, (uint16_t)w);
    const unsigned zi = w >> 16, zz = zi | (w & 0xffff0000u);
    z = (float)zi;
    z1024 = zz | 0x64006400u;
    z64 = zz << 4 | 0x54005400u;
  }
};
// The or-ed bits of 1024 + q and 64 + q, or of 16 + q (both halves of a pair).
struct Magic {
  unsigned a, b;
};
template <typename T>
__device__ __forceinline__ Magic magic4() {
  return std::is_same<T, f16>::value ? Magic{vconst(0x64006400u), vconst(0x54005400u)} : Magic{vconst(0x41804180u), 0u};
}
__device__ __forceinline__ f16x8 deq_f16(unsigned w, const Run4& c, const Magic& k) {  // q - z
  const f16x2 a = __builtin_bit_cast(f16x2, c.z1024), b = __builtin_bit_cast(f16x2, c.z64);
  f16x2 r[4];
  r[0] = __builtin_bit_cast(f16x2, (w & 0x000f000fu) | k.a) - a;
  r[1] = __builtin_bit_cast(f16x2, (w & 0x00f000f0u) | k.b) - b;
  w >>= 8;
  r[2] = __builtin_bit_cast(f16x2, (w & 0x000f000fu) | k.a) - a;
  r[3] = __builtin_bit_cast(f16x2, (w & 0x00f000f0u) | k.b) - b;
  return __builtin_bit_cast(f16x8, r);
}
constexpr int kUpBf16 = 3;   // bits that the dwords are rotated up by
constexpr float kOff = 16.f;  // of the codes
__device__ __forceinline__ bf16x8 deq_bf16_off(unsigned w, const Magic& k) {  // 16 + q
  u32x4 r;
  r[0] = (w & 0x00780078u) | k.a;
  r[1] = ((w >> 4) & 0x00780078u) | k.a;
  r[2] = ((w >> 8) & 0x00780078u) | k.a;
  r[3] = (__builtin_amdgcn_alignbit(w, w, 12) & 0x00780078u) | k.a;
  return __builtin_bit_cast(bf16x8, r);
}
// q - z: the two halves of a pair are the high halves of the floats 16 + q
__device__ __forceinline__ bf16x8 deq_bf16(unsigned w, float zoff, const Magic& k) {
  u32x4 r = __builtin_bit_cast(u32x4, deq_bf16_off(w, k));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float lo = __builtin_bit_cast(float, r[i] << 16) - zoff, hi = __builtin_bit_cast(float, r[i] & 0xffff0000u) - zoff;
    r[i] = __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, hi), __builtin_bit_cast(unsigned, lo), 0x07060302u);
  }
  return __builtin_bit_cast(bf16x8, r);
}
template <typename T>
__device__ __forceinline__ auto deq4(unsigned w, const Run4& c, const Magic& k) {
  if constexpr (std::is_same<T, float>::value) return deq_bf16(w, kOff + c.z, k);
  else if constexpr (std::is_same<T, bf16>::value) return deq_bf16_off(w, k);
  else return deq_f16(w, c, k);
}

// ------------------------------------------------------------------ inputs
// 8 consecutive inputs c .. c + 7 of a row of x, 0 past its end.  VX: rows of
// whole aligned chunks below 2 GiB from the resource's base, one or two wide
// loads (a resource's loads outside its range give zero); else element by
// element.
template <typename T, bool VX>
struct XRow {
  __amdgpu_buffer_rsrc_t rs;
  const T* row;
  unsigned off;  // of the row, in bytes (kOOB: a row of zeros)
  __device__ __forceinline__ V8<T> get(int c, int cols) const {
    V8<T> r;
    if constexpr (VX) {
      const unsigned o = c < cols ? off + (unsigned)c * (unsigned)sizeof(T) : kOOB;
      u32x4 u[sizeof(T) / 2];
      u[0] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)o, 0, 0));
      if constexpr (sizeof(T) == 4) u[1] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)o, 16, 0));
      __builtin_memcpy(&r, u, sizeof(r));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) r.v[j] = off != kOOB && c + j < cols ? row[c + j] : (T)0.f;
    }
    return r;
  }
};

// Part 0, 1 or 2 of float32 values as bf16: the leading 8 significant bits,
// the next 8, the last 8, each the value less the parts before it (exact).
// The masks are 0 for what is not taken off, so a lane's part is data, not a
// choice among three results: 6 instructions a value instead of 14 (5 rows of
// 2048 inputs and 1000 features: 10.4 -> 5.9 us; 16 rows, 8512 features: 48 ->
// 22).  An infinity has no rest, and a NaN is one in part 0 alone (its set bits
// may all lie in the low half).
struct Part {
  unsigned first, second;
  float odd;
  __device__ __forceinline__ explicit Part(int p)
      : first(p > 0 ? 0xffff0000u : 0u), second(p > 1 ? 0xffff0000u : 0u), odd(p > 0 ? 0.f : NAN) {}
};
__device__ __forceinline__ bf16x8 top_bf16(const float (&v)[8]) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r[i] = __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, v[2 * i + 1]), __builtin_bit_cast(unsigned, v[2 * i]), 0x07060302u);
  return __builtin_bit_cast(bf16x8, r);
}
__device__ __forceinline__ bf16x8 part_of(V8<float> x, const Part& p) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float v = x.v[j];
    v -= __builtin_bit_cast(float, __builtin_bit_cast(unsigned, v) & p.first);
    v -= __builtin_bit_cast(float, __builtin_bit_cast(unsigned, v) & p.second);
    x.v[j] = v == v ? v : p.odd;
  }
  return top_bf16(x.v);
}

// The words of a feature's runs in a block.
template <int RUNS>
__device__ __forceinline__ void ld_runs(__amdgpu_buffer_rsrc_t rs, int voff, int soff, unsigned (&o)[RUNS]) {
  if constexpr (RUNS == 1) {
    o[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, voff, soff, 0);
  } else if constexpr (RUNS == 2) {
    const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, voff, soff, 0));
    o[0] = v[0], o[1] = v[1];
  } else {
    const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, voff, soff, 0));
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = v[i];
  }
}

template <typename T>
struct Op4 {
  typedef typename std::conditional<std::is_same<T, f16>::value, f16, bf16>::type E;  // MFMA's element
  typedef typename Mfma<E>::frag frag;
};

// ------------------------------------------------------------------ few rows
// A workgroup owns 16 R features; its waves take the blocks of 128 inputs in
// turn, U at a time with all their loads in flight, and their sums meet in
// LDS.  x goes from global memory (its rows are shared by all workgroups and
// stay in the caches) straight to the first operand: row r = 4 g + v of it is
// row 4 v + g of x, so that up to 4 rows have all their sums in element v = 0
// (MV = 1); in float32 v is the part and g the row.
//
// Bound by the weights' bytes, and by the one trip to memory that every wave
// makes: 4 rows of 4096 inputs and 16384 features in f16, weights from HBM, 10.0
// us, 3.5 TB/s; one row in bf16 8.9 us, 3.9 TB/s; of 2048 inputs and 8512 features
// 5.3 us, of which an empty launch is 2.3.
template <typename T, int NB, int MV, int GS, bool VX, int R, int U>
__global__ __launch_bounds__(R == 1 && NB < 4 ? 1024 : 512) void linear4_rows_kernel(Linear4Args a) {
  typedef typename Op4<T>::E E;
  typedef typename Op4<T>::frag frag;
  constexpr bool F32 = std::is_same<T, float>::value;
  constexpr bool BIASED = std::is_same<T, bf16>::value;
  constexpr int RUNS = 4 / GS;
  constexpr int PER = F32 ? 4 : 4 * MV;  // rows of x per block of the first operand
  constexpr int NV = F32 ? 1 : MV;       // results per lane and block
  extern __shared__ float red[];         // [wave][R][NB][NV][64]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int col = lane & 15, g = lane >> 4, xr = lane & 15;
  const int cbs = (a.cols + 127) / 128, rbs = (a.rows + 15) / 16;
  const int rb0 = blockIdx.x * R;
  // loads outside a row of blocks give zero, and meet inputs of zero (the whole
  // offset in the operand that the range check compares)
  __amdgpu_buffer_rsrc_t rw[R], rs[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t blk = (int64_t)min(rb0 + r, rbs - 1) * cbs;
    rw[r] = make_rsrc(a.wq + blk * 256, (long long)cbs * 1024);
    rs[r] = make_rsrc(a.ws + blk * 16 * RUNS, (long long)cbs * 64 * RUNS);
  }
  // this lane's rows of x
  const int rows_x = (int)a.m;  // at most NB PER
  const T* xb = static_cast<const T*>(a.x);
  XRow<T, VX> xrow[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int v = xr & 3, m = nb * PER + (F32 ? xr >> 2 : 4 * v + (xr >> 2));
    const bool on = m < rows_x && v < (F32 ? 3 : MV);
    if constexpr (VX) xrow[nb].rs = make_rsrc(xb, ((rows_x - 1) * a.xs + a.cols) * (int)sizeof(T));
    xrow[nb].row = xb + (on ? m * a.xs : 0);
    xrow[nb].off = on ? VX ? (unsigned)(m * a.xs) * (unsigned)sizeof(T) : 0u : kOOB;
  }
  float tot[R][NB][NV] = {};
  const Magic magic = magic4<T>();
  const Part part(xr & 3);  // float32
  const frag ones = __builtin_bit_cast(frag, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
  for (int c0 = wave; c0 < cbs; c0 += waves * U) {
    u32x4 w[U][R];
    unsigned sc[U][R][RUNS];
    V8<T> xv[U][NB][4];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < R; ++r)  // read once: not kept in the caches for others
        w[u][r] = __builtin_bit_cast(
            u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw[r], lane * 16 + (c0 + u * waves) * 1024, 0, 2));
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i) xv[u][nb][i] = xrow[nb].get((c0 + u * waves) * 128 + 32 * i + 8 * g, a.cols);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        ld_runs<RUNS>(rs[r], col * 4 * RUNS + (c0 + u * waves) * 64 * RUNS, 0, sc[u][r]);
      }
    // all of the loads first (4096 x 16384, 4 rows of f16: 13.4 -> 10.2 us; left
    // to the compiler for bf16, where it hides them better by itself: 8.9
    // against 9.9 us)
    if constexpr (!BIASED) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int run = 0; run < RUNS; ++run) {
        frag xf[NB][GS];
        f32x4 xs[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          xs[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < GS; ++i) {
            if constexpr (F32) xf[nb][i] = part_of(xv[u][nb][run * GS + i], part);
            else xf[nb][i] = __builtin_bit_cast(frag, xv[u][nb][run * GS + i]);
            if constexpr (BIASED) xs[nb] = Mfma<E>::run(xf[nb][i], ones, xs[nb]);
          }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const Run4 rc(sc[u][r][run]);
          const float s = rc.s;
          f32x4 acc[NB];
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) acc[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < GS; ++i) {
            const frag wf = deq4<T>(w[u][r][run * GS + i], rc, magic);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) acc[nb] = Mfma<E>::run(xf[nb][i], wf, acc[nb]);
          }
          if constexpr (F32) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) tot[r][nb][0] = fmaf(s, acc[nb][0] + (acc[nb][1] + acc[nb][2]), tot[r][nb][0]);
          } else if constexpr (BIASED) {
            // an infinity among the biased products (or a finite sum beyond
            // the range that only the bias brings there): again with q - z
            bool over = false;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int v = 0; v < NV; ++v) over = over || !(fabsf(acc[nb][v]) < INFINITY);
            const float zz = kOff + rc.z;
            if (__any(over)) {
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) {
                f32x4 again = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < GS; ++i) again = Mfma<E>::run(xf[nb][i], deq_bf16(w[u][r][run * GS + i], zz, magic), again);
#pragma unroll
                for (int v = 0; v < NV; ++v) tot[r][nb][v] = fmaf(s, again[v], tot[r][nb][v]);
              }
            } else {
#pragma unroll
              for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int v = 0; v < NV; ++v) tot[r][nb][v] = fmaf(s, fmaf(-zz, xs[nb][v], acc[nb][v]), tot[r][nb][v]);
            }
          } else {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int v = 0; v < NV; ++v) tot[r][nb][v] = fmaf(s, acc[nb][v], tot[r][nb][v]);
          }
        }
      }
    }
  }
  constexpr int SUMS = R * NB * NV * 64;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int v = 0; v < NV; ++v) red[wave * SUMS + ((r * NB + nb) * NV + v) * 64 + lane] = tot[r][nb][v];
  __syncthreads();
  for (int i = threadIdx.x; i < SUMS; i += blockDim.x) {
    float s = 0.f;
    for (int w = 0; w < waves; ++w) s += red[w * SUMS + i];
    const int l = i & 63, v = (i >> 6) % NV, nb = (i >> 6) / NV % NB, r = (i >> 6) / (NV * NB);
    const int m = nb * PER + (F32 ? l >> 4 : 4 * v + (l >> 4)), k = (rb0 + r) * 16 + (l & 15);
    if (m < rows_x && k < a.rows)
      static_cast<T*>(a.y)[m * a.ys + k] = from_f<T>(act4(s + (a.bias ? a.bias[k] : 0.f), a.act));
  }
}

// ------------------------------------------------------------------ many rows
constexpr int kL4Stages = 3;
// Tile of 64 rows of x by 64 RB features: each of 4 waves owns 16 RB features
// and all 64 rows, so no weight is turned into floats twice in a workgroup,
// and x alone goes through LDS, in the first operand's order.  DMA (16-bit
// types, wide rows): LDS direct loads, three blocks of 128 inputs in a ring,
// two blocks ahead; else through registers, one block ahead (float32 is split
// into its parts there).  bf16: sums against ones, each wave for 16 of the rows,
// meet in LDS, and after every 4 runs the bias comes off as one more matrix
// product in float32, whose 4 steps are the runs.
//
// Bound by instruction issue: matrix instructions fill a third of the cycles, the
// codes' way to floats and the runs' scales another third (counted); HBM
// traffic is small.  1500 rows of 2048 inputs
// and 8512 features: 76 us in bf16, 690 TFLOP/s (a plain library
// product of 8192^3 reaches 1236); 344 us in float32.  (The bias off the whole
// sums at the end, from sums over x that wait in LDS, was 3 us faster, with ten
// times the error, and had no room for rows of more than 128 runs.)
template <typename T, int RB, int GS, bool VX>
__global__ __launch_bounds__(256, 2) void linear4_tile_kernel(Linear4Args a, int tiles_m, int tiles_n) {
  typedef typename Op4<T>::E E;
  typedef typename Op4<T>::frag frag;
  constexpr bool F32 = std::is_same<T, float>::value, BIASED = std::is_same<T, bf16>::value;
  constexpr bool DMA = VX && !F32;
  constexpr int RUNS = 4 / GS, PARTS = F32 ? 3 : 1;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  // [stage][part][row][slot] of 16 bytes, then (bf16) the sums over x of the last
  // 8 runs, and each wave's words of the last 4 (in registers they spilled)
  frag* xt = reinterpret_cast<frag*>(smem);
  constexpr int STAGE = PARTS * 4 * 4 * 64, STAGES = DMA ? kL4Stages : 2;
  float* xsum = reinterpret_cast<float*>(xt + STAGES * STAGE);  // [run % 8][64]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;
  const int cbs = (a.cols + 127) / 128, rbs = (a.rows + 15) / 16;
  int mt, nt;
  tile_of(blockIdx.x, tiles_m, tiles_n, mt, nt);
  const int64_t m0 = (int64_t)mt * 64, left = a.m - m0;
  // A stage of x in LDS: 64 rows of 16 slots of 8 inputs, chunk j of row m in
  // slot j ^ (m % 16), so that both the loads (16 lanes to a row) and the
  // operand reads (16 lanes to a column of chunks) meet all banks once.  This
  // lane loads chunk (lane % 16) ^ (m % 16) of rows m = 16 wave + 4 i + lane / 16
  // (past the last: the last one's values, not stored).
  const T* xb = static_cast<const T*>(a.x) + m0 * a.xs;
  XRow<T, VX> xrow[4];
  int xchunk[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = 4 * i + g, mx = (int)min((int64_t)(16 * wave + m), left - 1);
    if constexpr (VX) xrow[i].rs = make_rsrc(xb, ((min(left, (int64_t)64) - 1) * a.xs + a.cols) * (int)sizeof(T));
    xrow[i].row = xb + mx * a.xs;
    xrow[i].off = VX ? (unsigned)(mx * a.xs) * (unsigned)sizeof(T) : 0u;
    xchunk[i] = 8 * (col ^ m);
  }
  const int rb0 = (nt * 4 + wave) * RB;
  // the wave's rows of blocks (past the last: the last one's, not stored)
  __amdgpu_buffer_rsrc_t rw[RB], rs[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    const int64_t blk = (int64_t)min(rb0 + r, rbs - 1) * cbs;
    rw[r] = make_rsrc(a.wq + blk * 256, (long long)cbs * 1024);
    rs[r] = make_rsrc(a.ws + blk * 16 * RUNS, (long long)cbs * 64 * RUNS);
  }
  f32x4 tot[4][RB];  // [i]: row block (wave + i) % 4, so that each wave's own sums are those of i = 0
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int r = 0; r < RB; ++r) tot[i][r] = f32x4{0.f, 0.f, 0.f, 0.f};
  const Magic magic = magic4<T>();
  const frag ones = __builtin_bit_cast(frag, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
  const int runs = cbs * RUNS;
  constexpr int WORDS = 4 * RB * 16;
  unsigned* const words = reinterpret_cast<unsigned*>(xsum + 8 * 64) + wave * RB * 16;  // [run % 4][wave][RB][16]
  // The bias of runs q .. q + 3 off the sums (those behind the last do not count).
  auto settle = [&](int q) {
    if constexpr (BIASED) {
      int l = lane;
      if constexpr (BIASED) asm volatile("" : "+v"(l));
      const int run = q + (l >> 4), c = l & 15;
      const bool on = run < runs;
      float xs[4];
#pragma unroll
      for (int mi = 0; mi < 4; ++mi) xs[mi] = on ? xsum[(run & 7) * 64 + 16 * ((wave + mi) & 3) + c] : 0.f;
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        const Run4 rc(words[(l >> 4) * WORDS + r * 16 + c]);
        const float zs = on ? -(kOff + rc.z) * rc.s : 0.f;
#pragma unroll
        for (int mi = 0; mi < 4; ++mi) tot[mi][r] = Mfma<float>::run(xs[mi], zs, tot[mi][r]);
      }
    }
  };
  // Behind the barrier in front of a block: the blocks before it have left 4 new runs.
  auto settle_before = [&](int cb) {
    if (cb > 0 && cb * RUNS % 4 == 0) settle(cb * RUNS - 4);
  };
  V8<T> xn[DMA ? 1 : 4];
  struct W {
    u32x4 q[RB];
    unsigned s[RB][RUNS];
  };
  auto load_w = [&](int cb, W& w) {
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      w.q[r] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rw[r], lane * 16, cb * 1024, 0));
      ld_runs<RUNS>(rs[r], col * 4 * RUNS, cb * 64 * RUNS, w.s[r]);
    }
  };
  auto load_x = [&](int cb) {  // registers, or LDS stage cb % STAGES
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = cb * 128 + xchunk[i];
      if constexpr (DMA) {
        const unsigned o = c < a.cols ? xrow[i].off + (unsigned)c * 2u : kOOB;
        dma16(xrow[i].rs, reinterpret_cast<char*>(xt + (cb % STAGES) * STAGE + (wave * 4 + i) * 64), o, 0);
      } else {
        xn[i] = xrow[i].get(c, a.cols);
      }
    }
  };
  auto put = [&](int cb) {
    if constexpr (!DMA)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        frag* to = xt + (cb % STAGES) * STAGE + (wave * 4 + i) * 64 + lane;
        if constexpr (F32) {
#pragma unroll
          for (int p = 0; p < 3; ++p) to[p * 16 * 64] = part_of(xn[i], Part(p));
        } else {
          *to = __builtin_bit_cast(frag, xn[i]);
        }
      }
  };
  auto multiply = [&](int cb, const W& w) {
    int l = lane;
    if constexpr (BIASED) asm volatile("" : "+v"(l));  // 16 addresses that would stay in registers through the loop
    const frag* xc = xt + (cb % STAGES) * STAGE + (l & 15) * 16;
    auto xfrag = [&](int p, int mi, int i) { return xc[(p * 4 + ((wave + mi) & 3)) * 256 + ((4 * i + (l >> 4)) ^ (l & 15))]; };
#pragma unroll
    for (int run = 0; run < RUNS; ++run) {
      f32x4 acc[4][RB], xs = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int mi = 0; mi < 4; ++mi)
#pragma unroll
        for (int r = 0; r < RB; ++r) acc[mi][r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = run * GS; i < (run + 1) * GS; ++i) {
        frag wf[RB];
#pragma unroll
        for (int r = 0; r < RB; ++r) wf[r] = deq4<T>(w.q[r][i], Run4(w.s[r][run]), magic);
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
          for (int mi = 0; mi < 4; ++mi) {
            const frag xf = xfrag(p, mi, i);
            if (BIASED && mi == 0) xs = Mfma<E>::run(xf, ones, xs);
#pragma unroll
            for (int r = 0; r < RB; ++r) acc[mi][r] = Mfma<E>::run(xf, wf[r], acc[mi][r]);
          }
      }
      if constexpr (BIASED) {
        if (col == 0) *reinterpret_cast<f32x4*>(xsum + ((cb * RUNS + run) & 7) * 64 + 16 * wave + 4 * g) = xs;
        if (g == 0)
#pragma unroll
          for (int r = 0; r < RB; ++r) words[((cb * RUNS + run) & 3) * WORDS + r * 16 + col] = w.s[r][run];
      }
#pragma unroll
      for (int mi = 0; mi < 4; ++mi)
#pragma unroll
        for (int r = 0; r < RB; ++r) {
          const float s = Run4(w.s[r][run]).s;
#pragma unroll
          for (int v = 0; v < 4; ++v) tot[mi][r][v] = fmaf(s, acc[mi][r][v], tot[mi][r][v]);
        }
      if (RUNS > 1) __builtin_amdgcn_sched_barrier(0);  // one run's registers at a time
    }
  };
  if constexpr (DMA) {
    // the weights one block ahead (behind the last: the last one's again, not
    // used; the block is in the scalar offset, which no range check need see), x
    // two; past the last block: zeros
    W w0, w1;
    load_x(0), load_w(0, w0), load_x(1);
    auto block = [&](int cb, const W& now, W& next) {
      // x of the block is in LDS once all but the 4 loads of the next block's
      // x have arrived; behind the barrier every wave's are, and the stage of
      // block cb + 2 is no longer read
      wait_vmcnt<4>();
      dma_barrier();
      load_w(min(cb + 1, cbs - 1), next), load_x(cb + 2);
      settle_before(cb);
      multiply(cb, now);
    };
    for (int cb = 0; cb < cbs; cb += 2) {
      block(cb, w0, w1);
      if (cb + 1 < cbs) block(cb + 1, w1, w0);
    }
  } else {
    W w0, w1;
    load_x(0), load_w(0, w0);
    put(0);
    for (int cb = 0; cb < cbs; cb += 2) {
      lds_barrier();  // the stage is written, and the other one no longer read
      if (cb + 1 < cbs) load_x(cb + 1), load_w(cb + 1, w1);
      settle_before(cb);
      multiply(cb, w0);
      if (cb + 1 >= cbs) break;
      put(cb + 1);
      lds_barrier();
      if (cb + 2 < cbs) load_x(cb + 2), load_w(cb + 2, w0);
      settle_before(cb + 1);
      multiply(cb + 1, w1);
      if (cb + 2 < cbs) put(cb + 2);
    }
  }
  if constexpr (BIASED) {
    __syncthreads();
    settle((cbs - 1) * RUNS / 4 * 4);
  }
  // The results leave through LDS, as rows of 64 RB features: wide stores
  // (straight from the accumulators they would be runs of 16 features, a third
  // of the time at 2048 inputs).
  constexpr int WIDE = 64 * RB, PITCH = WIDE + 16 / sizeof(T);
  T* out = reinterpret_cast<T*>(smem);  // [row][feature], in place of the stages
  wait_vmcnt<0>();
  __syncthreads();  // nothing is on its way to the stages, and no one reads them
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    const int k = (rb0 + r) * 16 + col;
    const float b = a.bias && k < a.rows ? a.bias[k] : 0.f;
#pragma unroll
    for (int mi = 0; mi < 4; ++mi)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        out[(16 * ((wave + mi) & 3) + 4 * g + v) * PITCH + (wave * RB + r) * 16 + col] = from_f<T>(act4(tot[mi][r][v] + b, a.act));
  }
  if constexpr (BIASED) {
    // sums that are not finite (an infinity or a NaN of x, or beyond the range
    // by the bias alone) again, with q - z, input by input
    uint64_t odd = 0;
#pragma unroll
    for (int mi = 0; mi < 4; ++mi)
#pragma unroll
      for (int r = 0; r < RB; ++r)
#pragma unroll
        for (int v = 0; v < 4; ++v) odd |= (uint64_t)!(fabsf(tot[mi][r][v]) < INFINITY) << ((mi * RB + r) * 4 + v);
    while (odd) {
      const int e = __builtin_ctzll(odd), v = e & 3, r = (e >> 2) % RB, mi = (e >> 2) / RB;
      odd &= odd - 1;
      const int m = 16 * ((wave + mi) & 3) + 4 * g + v, k = (rb0 + r) * 16 + col;
      if (m >= left || k >= a.rows) continue;
      const int64_t blk = (int64_t)(rb0 + r) * cbs;
      const T* x = xb + m * a.xs;
      float sum = 0.f;
      for (int c = 0; c < a.cols; ++c) {
        const int64_t b = blk + c / 128;
        const Run4 rc(a.ws[(b * 16 + col) * RUNS + c % 128 / (32 * GS)]);
        const unsigned dw = a.wq[(b * 64 + col + 16 * (c % 32 / 8)) * 4 + c % 128 / 32];
        const unsigned code = __builtin_amdgcn_alignbit(dw, dw, kUpBf16 + 4 * (c % 8 / 2) + 16 * (c & 1)) & 15;
        sum = fmaf(to_f(x[c]), ((float)code - rc.z) * rc.s, sum);
      }
      out[m * PITCH + (wave * RB + r) * 16 + col] = from_f<T>(act4(sum + (a.bias ? a.bias[k] : 0.f), a.act));
    }
  }
  __syncthreads();
  const int k0 = nt * WIDE, rows = (int)min(left, (int64_t)64), wide = min(WIDE, a.rows - k0);
  T* y = static_cast<T*>(a.y) + m0 * a.ys + k0;
  if (a.vec_y) {
    constexpr int PER16 = 16 / sizeof(T), CH = WIDE / PER16;
    for (int i = threadIdx.x; i < rows * CH; i += 256) {
      const int m = i / CH, c = i % CH * PER16;
      if (c < wide) *reinterpret_cast<u32x4*>(y + m * a.ys + c) = *reinterpret_cast<const u32x4*>(out + m * PITCH + c);
    }
  } else {
    for (int i = threadIdx.x; i < rows * WIDE; i += 256) {
      const int m = i / WIDE, c = i % WIDE;
      if (c < wide) y[m * a.ys + c] = out[m * PITCH + c];
    }
  }
}

// ------------------------------------------------------------------ launchers
int linear4_gs(int group) { return group % 128 == 0 ? 4 : group % 64 == 0 ? 2 : 1; }
int64_t linear4_blocks(int rows, int cols) { return (int64_t)((rows + 15) / 16) * ((cols + 127) / 128); }

void linear4_pack(int dtype, const uint8_t* q, const f16* scale, const uint8_t* zero, int rows, int cols, int group,
                  unsigned* wq, unsigned* ws, hipStream_t st) {
  const int64_t blocks = linear4_blocks(rows, cols);
  check(blocks < (int64_t(1) << 31), "4-bit weights");
  SN_LAUNCH(linear4_pack_kernel, dim3((unsigned)blocks), dim3(256), 0, st, q, scale, zero, rows, cols, group,
            linear4_gs(group), dtype == 1 ? 0 : kUpBf16, wq, ws);
}

template <typename T, int NB, int MV, int GS, bool VX, int R, int U>
static void launch_rows_u(const Linear4Args& a, hipStream_t st) {
  constexpr int PER = std::is_same<T, float>::value ? 4 : 4 * MV, NV = std::is_same<T, float>::value ? 1 : MV;
  const int cbs = (a.cols + 127) / 128;
  // one row of blocks per workgroup: few features, so more waves for each
  const int waves = std::min(R == 1 && NB < 4 ? 16 : 8, (cbs + U - 1) / U);
  const dim3 grid((a.rows + 16 * R - 1) / (16 * R));
  check(a.m <= NB * PER, "rows of a few-row 4-bit product");
  SN_LAUNCH((linear4_rows_kernel<T, NB, MV, GS, VX, R, U>), grid, dim3(64 * waves), waves * R * NB * NV * 256, st, a);
}
template <typename T, int NB, int MV, int GS, bool VX>
static void launch_rows(const Linear4Args& a, hipStream_t st) {
  // Several rows of blocks per workgroup share the loads of x (and its sums),
  // as long as the workgroups still fill the chip.
  if constexpr (VX) {
    constexpr int U = NB == 1 ? 2 : 1;
    const int rbs = (a.rows + 15) / 16;
    if (rbs >= (NB == 1 ? 1024 : 512)) return launch_rows_u<T, NB, MV, GS, VX, NB == 4 ? 2 : 4, U>(a, st);
    if constexpr (NB == 1)
      if (rbs >= 512) return launch_rows_u<T, NB, MV, GS, VX, 2, U>(a, st);
  }
  launch_rows_u<T, NB, MV, GS, VX, 1, 1>(a, st);
}

template <typename T, int RB, int GS, bool VX>
static void launch_tile(const Linear4Args& a, hipStream_t st) {
  const int tm = (int)((a.m + 63) / 64), tn = (a.rows + 64 * RB - 1) / (64 * RB);
  constexpr bool F32 = std::is_same<T, float>::value, DMA = VX && !F32;
  const size_t lds = (DMA ? kL4Stages : 2) * (F32 ? 3 : 1) * 16384 +
                     (std::is_same<T, bf16>::value ? 8 * 256 + 4 * 4 * RB * 64 : 0);
  SN_LAUNCH((linear4_tile_kernel<T, RB, GS, VX>), dim3((unsigned)(tm * tn)), dim3(256), lds, st, a, tm, tn);
}

template <typename T, int GS, bool VX>
static void launch_linear4(const Linear4Args& a, hipStream_t st) {
  constexpr bool F32 = std::is_same<T, float>::value;
  if (a.m > (F32 ? 16 : 32)) {
    // as wide as registers allow (more runs in a block, or parts, take more of
    // them), if the tiles still fill the chip
    constexpr int RB = F32 ? GS == 4 ? 2 : 1 : GS == 4 && VX ? 4 : GS == 1 && !VX ? 1 : 2;
    if ((a.m + 63) / 64 * ((a.rows + 64 * RB - 1) / (64 * RB)) >= 256) launch_tile<T, RB, GS, VX>(a, st);
    else launch_tile<T, 1, GS, VX>(a, st);
    return;
  }
  if constexpr (F32) {
    if (a.m <= 4) launch_rows<T, 1, 1, GS, VX>(a, st);
    else if (a.m <= 8) launch_rows<T, 2, 1, GS, VX>(a, st);
    else launch_rows<T, 4, 1, GS, VX>(a, st);
  } else {
    if (a.m <= 4) launch_rows<T, 1, 1, GS, VX>(a, st);
    else if (a.m <= 16) launch_rows<T, 1, 4, GS, VX>(a, st);
    else launch_rows<T, 2, 4, GS, VX>(a, st);
  }
}

void linear4(const Linear4Args& in, hipStream_t st) {
  Linear4Args a = in;
  check(a.m >= 1 && a.rows >= 1 && a.cols >= 1 && a.group >= 32 && a.group % 32 == 0 && a.m <= 65535 * 4, "4-bit product shapes");
  const int e = a.dtype == 0 ? 4 : 2;
  a.vec_y = a.rows % (16 / e) == 0 && al16(a.y) && al16(a.ys * e);
  // wide loads of x: whole aligned chunks of 8, and 64 rows within a resource
  const bool vx = a.cols % 8 == 0 && al16(a.x) && al16(a.xs * e) && (64 * a.xs + a.cols) * e < (int64_t)kOOB;
#define SN_L4(T)                                                                                  \
  switch (linear4_gs(a.group)) {                                                                  \
    case 4: vx ? launch_linear4<T, 4, true>(a, st) : launch_linear4<T, 4, false>(a, st); break; \
    case 2: vx ? launch_linear4<T, 2, true>(a, st) : launch_linear4<T, 2, false>(a, st); break; \
    default: vx ? launch_linear4<T, 1, true>(a, st) : launch_linear4<T, 1, false>(a, st); break; \
  }
  if (a.dtype == 0) SN_L4(float)
  else if (a.dtype == 1) SN_L4(f16)
  else SN_L4(bf16)
#undef SN_L4
}

}  // namespace k
}  // namespace sn
