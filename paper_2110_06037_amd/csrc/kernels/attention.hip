// Attention over the paged cache: which kernel a call takes, and its workspace.
#include "attention.hpp"

namespace sn {
namespace k {

bool step_keys_fit(const CacheArgs& c) { return c.seqs * ((((int64_t)c.width << c.shift) >> 5) + 2) < (int64_t(1) << 30); }

int64_t attn_run_tiles(const AttnArgs& a) {
  const int each = a.heads / a.c.kv_heads;
  return a.c.tokens * each / kRunRows + a.c.seqs;
}

// Elements of ws_o, ws_m and count that any call of a handle needs.
void attn_workspace(const AttnArgs& a, int64_t& o, int64_t& m, int64_t& counts) {
  const int64_t DP = a.c.dim <= 64 ? 64 : a.c.dim <= 128 ? 128 : 256;
  const int64_t groups = (int64_t)a.c.kv_heads * ((a.heads / a.c.kv_heads + 15) / 16);
  const int64_t units = step_units(a, 512);
  // step: two slots a workgroup; run: at most kRunParts + kRunParts / 2 parts of tiles, which number kRunParts / 2 at most
  const int64_t step = units > 1 ? 2 * units * groups : 0, run = kRunParts + kRunParts / 2;
  o = std::max(step * 16 * DP, run * kRunRows * DP);
  m = std::max(step * 32, run * 512);
  counts = std::max<int64_t>(step, kRunParts);
}

static void attention(AttnArgs& a, bool step, hipStream_t st) {
  const CacheArgs& c = a.c;
  check(c.dim >= 8 && c.dim <= 256 && c.dim % 8 == 0 && c.kv_heads >= 1 && a.heads % c.kv_heads == 0 && a.heads <= 65535 &&
            c.shift >= 4 && c.shift <= 12 && c.seqs >= 1 && c.seqs <= 65535 && c.tokens >= 1 && c.width >= 0 &&
            ((int64_t)c.width << c.shift) <= kMaxPositions && a.window >= 0 && a.window <= kMaxPositions,
        "attention shapes");
  // without a page there is no position
  if (c.pages == 0) a.c.width = 0;
  // a scale of 0: all weights are equal, and masked scores stay minus infinity
  const float s = fabsf(a.scale) * kLog2e;
  a.scale2 = s > 0.f ? s : 0x1p-149f;
  a.negative = a.scale < 0.f;
  if (c.dtype == 0) attention_f32(a, step, st);
  else if (c.dtype == 1) attention_f16(a, step, st);
  else attention_bf16(a, step, st);
}

void attn_run(AttnArgs a, hipStream_t st) {
  check(attn_run_tiles(a) * a.c.kv_heads < (int64_t(1) << 24), "attention tiles");
  attention(a, false, st);
}
void attn_step(AttnArgs a, hipStream_t st) {
  check(a.c.tokens == a.c.seqs && !a.c.offsets && step_keys_fit(a.c), "attention step");
  attention(a, true, st);
}

}  // namespace k
}  // namespace sn
