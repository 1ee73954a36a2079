// Host-callable launchers of the sequence operators' kernels (blocknorm.hip,
// linear4.hip, scan.hip) and the device helpers they share.  A launcher
// enqueues on the given stream; none allocates or synchronises.
#pragma once

#include <algorithm>

#include "gemm_common.hpp"
#include "kcommon.hpp"
#include "launch.hpp"

namespace sn {
namespace k {

// ------------------------------------------------------------------ norms around a block
struct NormArgs {
  int dtype, rdtype;  // rdtype -1: no residual
  int64_t rows;
  int dim, groups, kind, gate;
  float eps, scale;
  const float *post_w, *post_b, *pre_w, *pre_b, *scale_v;
  const void* x;
  int64_t xs;
  const void* g;
  int64_t gs;
  const void* r;
  int64_t rs;
  void* ro;
  int64_t ros;
  void* y;
  int64_t ys;
};
constexpr int kNormMaxDim = 32768;
void block_norm(const NormArgs& a, hipStream_t st);

// ------------------------------------------------------------------ products with 4-bit weights
struct Linear4Args {
  int dtype, act;
  int64_t m;
  int rows, cols, group;
  const unsigned* wq;  // codes, and scales with zero points, in the kernels' order (linear4_pack)
  const unsigned* ws;
  const float* bias;  // [rows] or null
  const void* x;
  int64_t xs;
  void* y;
  int64_t ys;
  bool vec_y;  // wide stores (set by the launcher)
};
// Blocks of 16 features by 128 inputs: 256 dwords of codes each, and
// 64 / linear4_gs words of scale and zero point.
int64_t linear4_blocks(int rows, int cols);
int linear4_gs(int group);  // steps of 32 inputs that share a scale
void linear4_pack(int dtype, const uint8_t* q, const f16* scale, const uint8_t* zero, int rows, int cols, int group,
                  unsigned* wq, unsigned* ws, hipStream_t st);
void linear4(const Linear4Args& a, hipStream_t st);

// ------------------------------------------------------------------ selective scan
constexpr int kScanChunk = 64;     // tokens per chunk
constexpr int kScanUnits = 2048;   // waves that a pass is cut into segments for
constexpr int kScanDtRow = 5 * kScanChunk + 4;  // floats per head and chunk of ws_dt
constexpr int kScanMax = 4;                      // floats per group and chunk of ws_max
constexpr int kScanS = 10 * 256;                 // floats per group and chunk of ws_s
struct ScanArgs {
  int dtype, heads, dim, groups, state, conv, chans;  // dim: of a head
  int np;  // state columns that the workspace's rows hold (scan_np)
  // weights
  const float* conv_w;  // [4][chans], the last conv rows used
  const float* conv_b;  // [chans]
  const float* a2;      // [heads], a log2(e)
  const float* d;       // [heads]
  const float* dt_bias;
  // workspace
  void* ws_c;      // [slot][group] C of a chunk, 2 x 64 np f16 (scan_prep_kernel)
  void* ws_b;      // [slot][group] B of a chunk, likewise
  float* ws_s;     // [slot][group] C B^T, its 10 tiles on and below the diagonal
  float* ws_max;   // [slot][group][kScanMax] largest sizes in B and C
  float* ws_dt;    // [slot][head][kScanDtRow]: 64 each of the decay since the chunk's start, its log2 as
                   // hi and lo, the step size, the step size times the decay to the chunk's end; then
                   // the chunk's log2 decay
  float* ws_seg;   // [segment slot][head][dim][state]: slot 0 of a sequence its state before the call, slot i + 1
                   // what segment i adds
  float* ws_decay; // [segment slot][head], likewise: log2 of segment i's decay
  void* wcopy;     // [seq][conv - 1][chans]    the window before the call
  unsigned* count; // [seq][group], zero between calls
  int64_t seg_cap; // elements of ws_seg
  // call
  int seqs;
  int segs, per;  // segments of the longest sequence, chunks of a segment (set by the launcher)
  bool carried;   // states over the segments by a launch of their own (set by the launcher)
  int64_t each;  // rows per sequence without offsets (set by the launcher)
  int64_t tokens;
  const int32_t* offsets;
  const void* x;
  int64_t xs;
  const void* dt;
  int64_t dts;
  const void* window;
  const float* state_in;
  void* y;
  int64_t ys;
  void* window_out;
  float* state_out;
  bool vec_state;  // wide accesses of the state (set by the launcher)
};
inline int scan_np(int state) { return state <= 32 ? 32 : state <= 64 ? 64 : state <= 128 ? 128 : 256; }
inline int64_t scan_slots(int64_t tokens, int seqs) { return tokens / kScanChunk + seqs + 1; }
inline int64_t scan_segment_slots(int64_t slots, int seqs, int per) { return slots / per + seqs + 1; }
void scan_run(const ScanArgs& a, hipStream_t st);
void scan_step(const ScanArgs& a, hipStream_t st);

// ------------------------------------------------------------------ device helpers
constexpr float kLog2e = 1.44269504088896340736f;

// v * sigmoid(v); exp2 overflows to infinity for v < -89, whose reciprocal is the limit 0
__device__ __forceinline__ float silu_f(float v) {
  return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * v));
}

// Whether an address or a byte count is a multiple of 16.
inline bool al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline bool al16(int64_t b) { return (b & 15) == 0; }

}  // namespace k
}  // namespace sn
