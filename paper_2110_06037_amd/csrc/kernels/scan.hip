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
// state that every segment adds, a small kernel carries the states over the
// segments, and the second pass starts every segment from its own state.
//
// All decays are at most 1 (a <= 0).  c is held as hi + lo with hi in steps of
// 1/256, so that differences of hi are exact and those of lo small: a plain
// float32 sum would lose the differences of neighbours late in a chunk of
// strong decays.
#include "seq.hpp"

namespace sn {
namespace k {

constexpr int Q = kScanChunk;

// ------------------------------------------------------------------ rows of a sequence
// First row and length of sequence b; offsets are clamped to the call's rows,
// so that no content of theirs leads outside.
struct Seq {
  int64_t first;
  int len;
};
__device__ __forceinline__ int64_t seq_start(const ScanArgs& a, int b) {
  if (!a.offsets) return (int64_t)b * (a.tokens / a.seqs);
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

// ------------------------------------------------------------------ what all heads share
// grid (slots, groups + ceil(heads / 4) + 1).  The y index chooses: a group's
// B, C and S; four heads' step sizes and running sums; the window's copy of
// sequence x.
template <typename T>
__global__ __launch_bounds__(256) void scan_prep_kernel(ScanArgs a) {
  const int part = blockIdx.y, hb = (a.heads + 3) / 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (part == a.groups + hb) {
    const int b = blockIdx.x;
    const int64_t n = (int64_t)(a.conv - 1) * a.chans;
    if (b >= a.seqs) return;
    const T* src = static_cast<const T*>(a.window);
    T* dst = static_cast<T*>(a.wcopy) + b * n;
    for (int64_t i = threadIdx.x; i < n; i += 256) dst[i] = src ? src[b * n + i] : from_f<T>(0.f);
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
    const int h = (part - a.groups) * 4 + wave;
    if (h >= a.heads) return;
    const int t = t0 + lane;
    float dt = 0.f, inc = 0.f;
    if (t < s.len) {
      const float v = to_f(static_cast<const T*>(a.dt)[(s.first + t) * a.dts + h]) + a.dt_bias[h];
      dt = v > 20.f ? v : log1pf(expf(v));  // beyond 20 the difference is below a unit
      inc = dt * a.a2[h];
      if (inc < -1e4f) inc = -1e4f;  // 2^-1e4 is 0: keeps the sums finite, NaN stays
    }
    float ch = rintf(inc * 256.f) * (1.f / 256.f), cl = inc - ch;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const float uh = __shfl_up(ch, d), ul = __shfl_up(cl, d);
      if (lane >= d) ch += uh, cl += ul;
    }
    float* o = a.ws_dt + ((int64_t)slot * a.heads + h) * 3 * Q;
    o[lane] = dt;
    o[Q + lane] = ch;
    o[2 * Q + lane] = cl;
    return;
  }

  // ---- B and C of one group: convolution, then S = C B^T
  const int N = a.state, NP = a.np;
  float* C = a.ws_c + ((int64_t)slot * a.groups + part) * Q * NP;   // [t][n]
  float* B = a.ws_b + ((int64_t)slot * a.groups + part) * Q * NP;   // [n][t]
  float* S = a.ws_s + ((int64_t)slot * a.groups + part) * Q * Q;    // [t][s]
  for (int i = threadIdx.x; i < 2 * NP * (Q / 4); i += 256) {
    const int e = i % (2 * NP), tq = i / (2 * NP) * 4;
    const bool isc = e >= NP;
    const int n = isc ? e - NP : e;
    float u[4] = {0.f, 0.f, 0.f, 0.f};
    if (n < N) {
      const int ch = a.heads * a.dim + (isc ? a.groups * N : 0) + part * N + n;
      float w[4], r[7];
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = a.conv_w[k * a.chans + ch];
#pragma unroll
      for (int k = 0; k < 7; ++k) r[k] = raw_at<T>(a, s, b, t0 + tq - 3 + k, ch);
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (t0 + tq + v < s.len) u[v] = silu_f(taps4(w, a.conv_b[ch], r[v], r[v + 1], r[v + 2], r[v + 3], a.conv));
    }
    if (isc) {
#pragma unroll
      for (int v = 0; v < 4; ++v) C[(tq + v) * NP + n] = u[v];
    } else {
      *reinterpret_cast<f32x4*>(B + n * Q + tq) = f32x4{u[0], u[1], u[2], u[3]};
    }
  }
  __syncthreads();
  const int col = lane & 15, g = lane >> 4, tb = wave;
  for (int sb = 0; sb <= tb; ++sb) {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int n0 = 0; n0 < NP; n0 += 16) {
      const f32x4 cf = *reinterpret_cast<const f32x4*>(C + (16 * tb + col) * NP + n0 + 4 * g);
#pragma unroll
      for (int v = 0; v < 4; ++v)
        acc = Mfma<float>::run(cf[v], B[(n0 + 4 * g + v) * Q + 16 * sb + col], acc);
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) S[(16 * tb + 4 * g + v) * Q + 16 * sb + col] = acc[v];
  }
}

// ------------------------------------------------------------------ the heads
// A wave owns 16 PT columns p of one head and all N <= 16 NT state rows n: the
// state lives in PT NT accumulator tiles (lane: n = 16 nt + 4 (lane / 16) + v,
// p = p0 + PT (lane % 16) + j), whose layout is also that of the second
// operand of the product with C, so the state never leaves the registers;
// and a lane's convolution outputs (times 16 sb + 4 (lane / 16) + v, the
// same p) are the second operand of both other products.  PT consecutive p
// per lane make its row accesses vectors.
// SEG: only the state that the segment adds (from zero), no outputs.
template <typename T, int PT>
__device__ __forceinline__ void ld_p(const T* p, int n, bool vec, float (&o)[PT]) {
  if (vec && n >= PT) {
    T v[PT];
    __builtin_memcpy(v, __builtin_assume_aligned(p, sizeof(T) * PT), sizeof(T) * PT);
#pragma unroll
    for (int j = 0; j < PT; ++j) o[j] = to_f(v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < PT; ++j) o[j] = j < n ? to_f(p[j]) : 0.f;
  }
}

template <typename T, int NT, int PT, bool SEG>
__global__ __launch_bounds__(256) void scan_main_kernel(ScanArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, g = lane >> 4;
  const int b = blockIdx.z, seg = blockIdx.y;
  const int each = a.heads / a.groups, pblocks = (a.dim + 16 * PT - 1) / (16 * PT);
  const int ublocks = (each * pblocks + 3) / 4;
  const int grp = blockIdx.x / ublocks, unit = (blockIdx.x % ublocks) * 4 + wave;
  const Seq s = seq_of(a, b);
  const int nc = (s.len + Q - 1) / Q, per = (nc + a.segs - 1) / a.segs;
  const int c0 = min(seg * per, nc), c1 = min(c0 + per, nc);
  const int NP = a.np, N = a.state;

  if (!SEG && a.window_out) {
    // the window after the last row, shared out over the sequence's workgroups
    const int64_t n = (int64_t)(a.conv - 1) * a.chans;
    const int blocks = gridDim.x * gridDim.y, me = blockIdx.y * gridDim.x + blockIdx.x;
    T* out = static_cast<T*>(a.window_out) + b * n;
    for (int64_t i = (int64_t)me * 256 + threadIdx.x; i < n; i += (int64_t)blocks * 256) {
      const int k = (int)(i / a.chans), ch = (int)(i - (int64_t)k * a.chans), t = s.len - (a.conv - 1) + k;
      out[i] = t >= 0 ? static_cast<const T*>(a.x)[(s.first + t) * a.xs + ch]
                      : static_cast<const T*>(a.wcopy)[b * n + (int64_t)(a.conv - 1 + t) * a.chans + ch];
    }
  }
  if (unit >= each * pblocks) return;
  const int h = grp * each + unit / pblocks;
  const int p0 = (unit % pblocks) * 16 * PT + PT * col;  // this lane's first p
  const int pn = a.dim - p0;                             // and how many of its PT exist (<= 0: none)
  const int64_t hold = (int64_t)a.dim * N;

  f32x4 st[NT][PT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int j = 0; j < PT; ++j) st[nt][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto state_rw = [&](auto* p, auto&& f) {  // f(element pointer, tile register) over the lane's state
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < PT; ++j) {
        const int n = 16 * nt + 4 * g;
        auto* q = p + (int64_t)(p0 + j) * N + n;
        if (j < pn && n < N) f(q, st[nt][j], n);
      }
  };
  auto load = [&](const float* q, f32x4& r, int n) {
    if (a.vec_state) r = *reinterpret_cast<const f32x4*>(q);
    else
#pragma unroll
      for (int v = 0; v < 4; ++v) r[v] = n + v < N ? q[v] : 0.f;
  };
  auto store = [&](float* q, f32x4& r, int n) {
    if (a.vec_state) *reinterpret_cast<f32x4*>(q) = r;
    else
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (n + v < N) q[v] = r[v];
  };
  float* segst = a.ws_seg + (((int64_t)b * a.segs + seg) * a.heads + h) * hold;
  if (SEG) {
    if (c1 >= nc) return;  // nothing follows: no one reads this segment's state
  } else if (a.segs > 1) {
    state_rw(static_cast<const float*>(segst), load);
  } else if (a.state_in) {
    state_rw(a.state_in + ((int64_t)b * a.heads + h) * hold, load);
  }

  // the lane's convolution
  const int ch0 = h * a.dim + p0;
  float w[4][PT], cb[PT];
#pragma unroll
  for (int j = 0; j < PT; ++j) {
    cb[j] = j < pn ? a.conv_b[ch0 + j] : 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k][j] = j < pn ? a.conv_w[k * a.chans + ch0 + j] : 0.f;
  }
  const float dh = a.d[h];
  float total = 0.f;  // log2 of the segment's decay
  for (int c = c0; c < c1; ++c) {
    const int slot = slot0_of(s.first, b) + c, t0 = c * Q;
    const float* Cm = a.ws_c + ((int64_t)slot * a.groups + grp) * Q * NP;
    const float* Bm = a.ws_b + ((int64_t)slot * a.groups + grp) * Q * NP;
    const float* Sm = a.ws_s + ((int64_t)slot * a.groups + grp) * Q * Q;
    const float* dtp = a.ws_dt + ((int64_t)slot * a.heads + h) * 3 * Q;
    // convolution outputs and Xd of the lane's 16 times
    float u[4][PT][4], xd[4][PT][4];
    float odd = 0.f;  // NaN if some Xd is not finite
#pragma unroll
    for (int sb = 0; sb < 4; ++sb) {
      float r[7][PT];
#pragma unroll
      for (int k = 0; k < 7; ++k) {
        const int t = t0 + 16 * sb + 4 * g - 3 + k;
        if (t >= 0 && t < s.len) {
          ld_p<T, PT>(static_cast<const T*>(a.x) + (s.first + t) * a.xs + ch0, pn, a.vec_x, r[k]);
        } else if (t < 0 && a.conv - 1 + t >= 0) {
          ld_p<T, PT>(static_cast<const T*>(a.wcopy) + ((int64_t)b * (a.conv - 1) + a.conv - 1 + t) * a.chans + ch0, pn,
                      false, r[k]);
        } else {
#pragma unroll
          for (int j = 0; j < PT; ++j) r[k][j] = 0.f;
        }
      }
      const f32x4 dt = *reinterpret_cast<const f32x4*>(dtp + 16 * sb + 4 * g);
#pragma unroll
      for (int j = 0; j < PT; ++j) {
        const float wj[4] = {w[0][j], w[1][j], w[2][j], w[3][j]};
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          u[sb][j][v] = silu_f(taps4(wj, cb[j], r[v][j], r[v + 1][j], r[v + 2][j], r[v + 3][j], a.conv));
          const float x = t0 + 16 * sb + 4 * g + v < s.len ? u[sb][j][v] * dt[v] : 0.f;
          xd[sb][j][v] = x;
          odd = fmaf(x, 0.f, odd);
        }
      }
    }
    // A value that is not finite must not meet the zeros of earlier rows (0 *
    // NaN): it leaves the products, and its column is NaN from its row on.
    int from[PT];
#pragma unroll
    for (int j = 0; j < PT; ++j) from[j] = Q;
    const bool poison = __any(odd != 0.f);
    if (poison) {
#pragma unroll
      for (int j = 0; j < PT; ++j) {
#pragma unroll
        for (int sb = 0; sb < 4; ++sb)
#pragma unroll
          for (int v = 0; v < 4; ++v)
            if (!(fabsf(xd[sb][j][v]) < INFINITY)) {
              xd[sb][j][v] = 0.f;
              from[j] = min(from[j], 16 * sb + 4 * g + v);
            }
        from[j] = min(from[j], __shfl_xor(from[j], 16));
        from[j] = min(from[j], __shfl_xor(from[j], 32));
      }
    }
    const float eh = dtp[2 * Q - 1], el = dtp[3 * Q - 1];  // c at the chunk's end
    if constexpr (!SEG) {
#pragma unroll
      for (int tb = 0; tb < 4; ++tb) {
        f32x4 acc[PT];
#pragma unroll
        for (int j = 0; j < PT; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const f32x4 cf = *reinterpret_cast<const f32x4*>(Cm + (16 * tb + col) * NP + 16 * nt + 4 * g);
#pragma unroll
          for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int j = 0; j < PT; ++j) acc[j] = Mfma<float>::run(cf[v], st[nt][j][v], acc[j]);
        }
        const f32x4 rh = *reinterpret_cast<const f32x4*>(dtp + Q + 16 * tb + 4 * g);
        const f32x4 rl = *reinterpret_cast<const f32x4*>(dtp + 2 * Q + 16 * tb + 4 * g);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float e = __builtin_amdgcn_exp2f(rh[v] + rl[v]);
#pragma unroll
          for (int j = 0; j < PT; ++j) acc[j][v] *= e;
        }
        const int tr = 16 * tb + col;  // the row of the first operand that this lane holds
        const float th = dtp[Q + tr], tl = dtp[2 * Q + tr];
#pragma unroll
        for (int sb = 0; sb <= tb; ++sb) {
          const f32x4 sv = *reinterpret_cast<const f32x4*>(Sm + tr * Q + 16 * sb + 4 * g);
          const f32x4 sh = *reinterpret_cast<const f32x4*>(dtp + Q + 16 * sb + 4 * g);
          const f32x4 sl = *reinterpret_cast<const f32x4*>(dtp + 2 * Q + 16 * sb + 4 * g);
#pragma unroll
          for (int v = 0; v < 4; ++v) {
            const float m =
                16 * sb + 4 * g + v <= tr ? sv[v] * __builtin_amdgcn_exp2f((th - sh[v]) + (tl - sl[v])) : 0.f;
#pragma unroll
            for (int j = 0; j < PT; ++j) acc[j] = Mfma<float>::run(m, xd[sb][j][v], acc[j]);
          }
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const int t = 16 * tb + 4 * g + v;
          T o[PT];
#pragma unroll
          for (int j = 0; j < PT; ++j) {
            float y = fmaf(dh, u[tb][j][v], acc[j][v]);
            if (t >= from[j]) y = NAN;
            o[j] = from_f<T>(y);
          }
          if (t0 + t < s.len) {
            T* yp = static_cast<T*>(a.y) + (s.first + t0 + t) * a.ys + ch0;
            if (a.vec_y && pn >= PT) {
              __builtin_memcpy(__builtin_assume_aligned(yp, sizeof(T) * PT), o, sizeof(T) * PT);
            } else {
#pragma unroll
              for (int j = 0; j < PT; ++j)
                if (j < pn) yp[j] = o[j];
            }
          }
        }
      }
    }
    // the state after the chunk
    const float e = __builtin_amdgcn_exp2f(eh + el);
    total += eh + el;
#pragma unroll
    for (int sb = 0; sb < 4; ++sb) {
      const f32x4 sh = *reinterpret_cast<const f32x4*>(dtp + Q + 16 * sb + 4 * g);
      const f32x4 sl = *reinterpret_cast<const f32x4*>(dtp + 2 * Q + 16 * sb + 4 * g);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const float f = __builtin_amdgcn_exp2f((eh - sh[v]) + (el - sl[v]));
#pragma unroll
        for (int j = 0; j < PT; ++j) xd[sb][j][v] *= f;
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int j = 0; j < PT; ++j) st[nt][j] *= e;
#pragma unroll
      for (int sb = 0; sb < 4; ++sb) {
        const f32x4 bf = *reinterpret_cast<const f32x4*>(Bm + (16 * nt + col) * Q + 16 * sb + 4 * g);
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
          for (int j = 0; j < PT; ++j) st[nt][j] = Mfma<float>::run(bf[v], xd[sb][j][v], st[nt][j]);
      }
    }
    if (poison) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < PT; ++j)
          if (from[j] < Q) st[nt][j] = f32x4{NAN, NAN, NAN, NAN};
    }
  }
  if (SEG) {
    state_rw(segst, store);
    if (lane == 0 && unit % pblocks == 0) a.ws_decay[((int64_t)b * a.segs + seg) * a.heads + h] = total;
  } else if (a.state_out && (c1 == nc && (c0 < c1 || seg == 0))) {
    // the segment with the sequence's last chunk (segment 0 of a sequence without rows)
    state_rw(a.state_out + ((int64_t)b * a.heads + h) * hold, store);
  }
}

// States over the segments: slot i of a head's segments takes the state in
// front of segment i.  Segments after the sequence's end are not read.
__global__ __launch_bounds__(256) void scan_carry_kernel(ScanArgs a) {
  const int64_t hold = (int64_t)a.dim * a.state, e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int b = blockIdx.z, h = blockIdx.y;
  if (e >= hold) return;
  const int nc = (seq_of(a, b).len + Q - 1) / Q, per = (nc + a.segs - 1) / a.segs;
  float v = a.state_in ? a.state_in[((int64_t)b * a.heads + h) * hold + e] : 0.f;
  for (int i = 0; i < a.segs; ++i) {
    float* p = a.ws_seg + (((int64_t)b * a.segs + i) * a.heads + h) * hold + e;
    const bool more = (i + 1) * per < nc;  // another segment follows with chunks of its own
    float add = 0.f, f = 0.f;
    if (more) add = *p, f = __builtin_amdgcn_exp2f(a.ws_decay[((int64_t)b * a.segs + i) * a.heads + h]);
    *p = v;
    if (!more) return;
    v = fmaf(v, f, add);
  }
}

// ------------------------------------------------------------------ one token per sequence
// grid (heads x splits of a head's rows p, sequences).  A quad of state columns
// per thread; L threads (a power of two) side by side hold a row.  The state
// is read first: its bytes bound the kernel.  The workgroups of a group all
// read the window of B and C; when it is updated in place, the last of them
// to have read it (counted per sequence and group) writes it.
template <typename T>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanArgs a, int L, int splits) {
  constexpr int PASS = 2;
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
  T now[4][4];  // raw values of the thread's channels, for the new window
  constexpr int ITEMS = 4;
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
template <typename T, int NT, int PT>
static void launch_main(const ScanArgs& a, hipStream_t st) {
  const int each = a.heads / a.groups, pblocks = (a.dim + 16 * PT - 1) / (16 * PT);
  const dim3 grid(a.groups * ((each * pblocks + 3) / 4), a.segs, a.seqs);
  if (a.segs > 1) {
    SN_LAUNCH((scan_main_kernel<T, NT, PT, true>), grid, dim3(256), 0, st, a);
    SN_LAUNCH((scan_carry_kernel), dim3((a.dim * a.state + 255) / 256, a.heads, a.seqs), dim3(256), 0, st, a);
  }
  SN_LAUNCH((scan_main_kernel<T, NT, PT, false>), grid, dim3(256), 0, st, a);
}

template <typename T>
static void launch_scan(ScanArgs a, hipStream_t st) {
  constexpr int PT = 4;
  a.vec_state = a.state % 4 == 0 && al16(a.state_in) && al16(a.state_out) && al16(a.ws_seg);
  // a lane's PT values of a row go as one vector: rows and heads on its alignment
  const int64_t v = sizeof(T) * PT;
  auto ok = [&](const void* p, int64_t stride) {
    return reinterpret_cast<uintptr_t>(p) % v == 0 && stride * sizeof(T) % v == 0 && a.dim % PT == 0;
  };
  a.vec_x = ok(a.x, a.xs), a.vec_y = ok(a.y, a.ys);
  const int64_t slots = scan_slots(a.tokens, a.seqs);
  SN_LAUNCH((scan_prep_kernel<T>), dim3((unsigned)slots, a.groups + (a.heads + 3) / 4 + 1), dim3(256), 0, st, a);
  if (a.np <= 32) launch_main<T, 2, PT>(a, st);
  else if (a.np <= 64) launch_main<T, 4, PT>(a, st);
  else if (a.np <= 128) launch_main<T, 8, PT>(a, st);
  else launch_main<T, 16, PT>(a, st);
}

template <typename T>
static void launch_step(ScanArgs a, hipStream_t st) {
  a.vec_state = a.state % 4 == 0 && al16(a.state_in) && al16(a.state_out);
  int L = 1;
  while (4 * L < a.state) L *= 2;
  const int rows = 2 * (256 / L), splits = (a.dim + rows - 1) / rows;
  SN_LAUNCH((scan_step_kernel<T>), dim3((unsigned)(a.heads * splits), a.seqs), dim3(256), 0, st, a, L, splits);
}

static int scan_segments(const ScanArgs& a) {
  // waves of a pass: units of 64 columns per head and sequence; segments until
  // about 1024 of them (one per SIMD) run, each at least two chunks
  const int64_t units = (int64_t)a.seqs * a.heads * ((a.dim + 63) / 64);
  const int64_t chunks = (a.tokens + Q - 1) / Q;  // the most that one sequence may have
  const int64_t want = std::min<int64_t>((kScanUnits + units - 1) / units, chunks / 2);
  return (int)std::max<int64_t>(1, want);
}

void scan_run(const ScanArgs& in, hipStream_t st) {
  ScanArgs a = in;
  check(a.heads >= 1 && a.groups >= 1 && a.heads % a.groups == 0 && a.dim >= 1 && a.state >= 1 && a.state <= 256 &&
            a.conv >= 1 && a.conv <= 4 && a.seqs >= 1 && a.seqs <= 65535 && a.tokens >= 0,
        "scan shapes");
  a.segs = scan_segments(a);
  check(a.segs == 1 || a.seqs * (int64_t)a.segs * a.heads * a.dim * a.state <= a.seg_cap, "scan segments");
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
