// Host-callable launchers of the attention operators' kernels (headnorm.hip,
// kvcache.hip, attention.hip) and the device helpers they share.  A launcher
// enqueues on the given stream; none allocates or synchronises.
#pragma once

#include "seq.hpp"

namespace sn {
namespace k {

// ------------------------------------------------------------------ norms of heads with the position rotation
struct HeadNormArgs {
  int dtype, heads, kv_heads, dim, rot, pairs, norm;
  float eps;
  const float *q_w, *k_w;          // [dim]
  const unsigned long long* turn;  // [rot / 2] turns per position, the fraction times 2^64
  int64_t tokens;
  const int32_t* positions;
  const void* q;
  int64_t qs;
  const void* k;
  int64_t ks;
  void* qo;
  int64_t qos;
  void* ko;
  int64_t kos;
  // set by the launcher
  FastDiv all;               // by the heads of a token
  int lanes, tokens_each;  // threads of a row, tokens of a workgroup
};
void head_norm(const HeadNormArgs& a, hipStream_t st);

// ------------------------------------------------------------------ paged cache
constexpr int kCacheTile = 16;           // positions that V keeps together
constexpr int kMaxPositions = 1 << 29;   // of a table, and of a window
constexpr int kMaxPast = 1 << 30;        // past counts as this at most: such rows see no window of a table
struct CacheArgs {
  int dtype, kv_heads, dim, shift;  // shift: log2 of a page's positions
  bool i8;
  int64_t pages;
  void* k;    // [page][kv head][position][dim]
  void* v;    // [page][kv head][position / 16][dim][position % 16]
  float* ks;  // [page][kv head][position]
  float* vs;
  int seqs, width;
  const int32_t* table;
  int64_t ts;
  const int32_t* past;
  int64_t tokens;
  const int32_t* offsets;
  int64_t each;  // rows per sequence without offsets
};
struct CacheRows {
  CacheArgs c;
  void* k;  // [tokens][kv_heads * dim]: read by a write, written by a read
  int64_t krs;
  void* v;
  int64_t vrs;
  // set by the launcher
  int lanes;              // threads of a row
  FastDiv head_granules;  // by the 16 bytes that V has of a head's 16 positions
};
void cache_write(const CacheRows& a, hipStream_t st);
void cache_read(const CacheRows& a, hipStream_t st);

// ------------------------------------------------------------------ attention over the cache
struct AttnArgs {
  CacheArgs c;
  int heads, window;
  float scale;
  const void* q;
  int64_t qs;
  void* y;
  int64_t ys;
  // workspace (attn_workspace)
  float* ws_o;      // parts' sums of weighted values
  float* ws_m;      // their maxima and sums of weights
  unsigned* count;  // parts that are done, zero between calls
  // set by the launchers
  float scale2;   // |scale| log2(e)
  bool negative;  // scale < 0
  int units;      // parts that a step's keys are cut into at most
  FastDiv each;   // by the query heads of a key head
};
int64_t attn_run_tiles(const AttnArgs& a);  // bound of a prompt call's tiles of rows, per key head
bool step_keys_fit(const CacheArgs& c);  // the keys of a step's sequences, in blocks of 32, are below 2^30
void attn_workspace(const AttnArgs& a, int64_t& o, int64_t& m, int64_t& counts);
void attn_run(AttnArgs a, hipStream_t st);
void attn_step(AttnArgs a, hipStream_t st);
void attention_f32(AttnArgs& a, bool step, hipStream_t st);
void attention_f16(AttnArgs& a, bool step, hipStream_t st);
void attention_bf16(AttnArgs& a, bool step, hipStream_t st);

// ------------------------------------------------------------------ device helpers
// The rows of sequence b: [first, end), within the call's rows.
__device__ __forceinline__ void seq_rows(const CacheArgs& c, int b, int64_t& first, int64_t& end) {
  if (c.offsets) {
    first = min((int64_t)max(c.offsets[b], 0), c.tokens);
    end = max(first, min((int64_t)max(c.offsets[b + 1], 0), c.tokens));
  } else {
    first = b * c.each;
    end = first + c.each;
  }
}
// The sequence of a row, -1 for rows of none.
__device__ __forceinline__ int seq_of(const CacheArgs& c, int64_t row) {
  if (!c.offsets) return (int)(row / c.each);
  int lo = 0, hi = c.seqs;  // the last b with offsets[b] <= row
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (c.offsets[mid] <= row) lo = mid;
    else hi = mid;
  }
  return c.offsets[lo] <= row && row < c.offsets[lo + 1] ? lo : -1;
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int lane_of(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }  // (of a uniform lane)
// The sum over this lane and those before it, at most 2^32 - 1.
__device__ __forceinline__ unsigned scan_lanes(unsigned v) {
#define SN_SCAN(CTRL, ROWS) v = __builtin_elementwise_add_sat(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false))
  SN_SCAN(0x111, 0xF);  // 1, 2, 4, 8 lanes before, within 16
  SN_SCAN(0x112, 0xF);
  SN_SCAN(0x114, 0xF);
  SN_SCAN(0x118, 0xF);
  SN_SCAN(0x142, 0xA);  // the last of 16 to the next 16
  SN_SCAN(0x143, 0xC);  // the last of 32 to the next 32
#undef SN_SCAN
  return v;
}
// Units of work are counted over the sequences in order, count(rows, past) of each: the
// sequence behind the number `unit`, the unit's number in it, the sequence's rows and past.
// (Every wave for itself, 64 sequences at a time.  Offsets that fall may count more units than
// there are: sums stop at the top of their range, and stay in order.)  False: there are fewer units.
template <typename F>
__device__ __forceinline__ bool find_rows(const CacheArgs& c, unsigned unit, F count, int& b, int& at, int& first, int& rows, int& past) {
  const int lane = threadIdx.x & 63;
  unsigned before = 0;
  for (int base = 0; base < c.seqs; base += 64) {
    int64_t lo, hi;
    const int own_past = min(c.past[min(base + lane, c.seqs - 1)], kMaxPast);
    seq_rows(c, min(base + lane, c.seqs - 1), lo, hi);
    const unsigned own = base + lane < c.seqs ? (unsigned)count((int)(hi - lo), own_past) : 0;
    const unsigned sum = __builtin_elementwise_add_sat(before, scan_lanes(own));
    const unsigned long long in = __ballot(unit < sum);
    if (in) {
      const int l = __ffsll(in) - 1;
      b = base + l, at = (int)(unit - (l ? (unsigned)lane_of((int)sum, l - 1) : before));
      first = lane_of((int)lo, l), rows = lane_of((int)(hi - lo), l), past = lane_of(own_past, l);
      return true;
    }
    before = (unsigned)lane_of((int)sum, 63);
  }
  return false;
}
// How many groups of 16 positions `rows` rows after `past` lie in.
__device__ __forceinline__ int rows_tiles(int past, int rows) {
  const int p = max(past, 0) & 15;
  return rows ? (p + rows + 15) >> 4 : 0;
}
// The page that holds a position of sequence b, -1 if none does.
__device__ __forceinline__ int page_of(const CacheArgs& c, int b, int pos) {
  const int i = pos >> c.shift;
  if (pos < 0 || i >= c.width) return -1;
  const int page = c.table[b * c.ts + i];
  return (unsigned)page < (uint64_t)c.pages ? page : -1;
}
// Where a position's row of K and its elements of V begin (V: 16 apart), and its scales.
__device__ __forceinline__ int64_t k_at(const CacheArgs& c, int page, int head, int slot) {
  return ((((int64_t)page * c.kv_heads + head) << c.shift) + slot) * c.dim;
}
__device__ __forceinline__ int64_t v_at(const CacheArgs& c, int page, int head, int slot) {
  return ((((int64_t)page * c.kv_heads + head) << c.shift) + (slot & ~15)) * c.dim + (slot & 15);
}
__device__ __forceinline__ int64_t scale_at(const CacheArgs& c, int page, int head, int slot) {
  return (((int64_t)page * c.kv_heads + head) << c.shift) + slot;
}

}  // namespace k
}  // namespace sn
