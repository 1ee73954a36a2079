// Attention operators of the C ABI: handles, argument checks, and the calls of
// the kernels' launchers.
#include <memory>

#include "api_guard.hpp"
#include "kernels/attn.hpp"
#include "seqop.hpp"

using namespace sn;

namespace {

struct HeadNormOp : sn_op {
  k::HeadNormArgs a{};
  using sn_op::sn_op;
};
struct CacheOp : sn_op {
  k::CacheArgs c{};
  using sn_op::sn_op;
};
struct AttnOp : sn_op {
  k::AttnArgs a{};
  int max_seqs = 0;
  int64_t max_tokens = 0;
  using sn_op::sn_op;
};

k::CacheArgs cache_of(const sn_cache_desc& d) {
  check_dtype(d.dtype);
  if (d.store != SN_STORE_SAME && d.store != SN_STORE_I8) fail(SN_E_INVALID, "unknown store");
  if (d.kv_heads < 1 || d.kv_heads > 4096) fail(SN_E_SHAPE, "kv_heads must be in 1..4096");
  if (d.head_dim < 1) fail(SN_E_SHAPE, "head_dim must be positive");
  if (d.head_dim % 8 || d.head_dim > 256) fail(SN_E_UNSUPPORTED, "head_dim must be a multiple of 8 up to 256");
  if (d.page < 16 || d.page > 4096 || (d.page & (d.page - 1))) fail(SN_E_SHAPE, "page must be a power of two in 16..4096");
  k::CacheArgs c{};
  c.dtype = d.dtype, c.i8 = d.store == SN_STORE_I8, c.kv_heads = d.kv_heads, c.dim = d.head_dim;
  while ((1 << c.shift) < d.page) ++c.shift;
  // (places within a page are 32-bit offsets)
  if ((int64_t)d.kv_heads * d.page * d.head_dim * (c.i8 ? 1 : dtype_size(d.dtype)) >> 31) fail(SN_E_UNSUPPORTED, "a page of 2^31 bytes or more");
  return c;
}

void check_aligned(const void* p, size_t to, const char* what) {
  if (reinterpret_cast<uintptr_t>(p) % to) fail(SN_E_INVALID, std::string(what) + " is not aligned");
}

// The call's cache and sequences, checked.
k::CacheArgs cache_args(k::CacheArgs c, const sn_cache_io* io, bool step) {
  if (!io) fail(SN_E_INVALID, "null arguments");
  if (io->seqs < 0 || io->seqs > 65535) fail(SN_E_SHAPE, "seqs must be in 0..65535");
  if (io->tokens < 0 || io->tokens > (1 << 26)) fail(SN_E_SHAPE, "tokens must be in 0..2^26");
  if (io->seqs == 0 && io->tokens) fail(SN_E_SHAPE, "tokens without a sequence");
  if (step && (io->tokens != io->seqs || io->offsets)) fail(SN_E_SHAPE, "a step takes one token per sequence");
  if (io->seqs && !io->offsets && io->tokens % io->seqs) fail(SN_E_SHAPE, "tokens are no multiple of seqs, and there are no offsets");
  if (io->pages < 0 || io->pages >> 31) fail(SN_E_SHAPE, "pages must be in 0..2^31 - 1");
  if ((io->pages * c.kv_heads << c.shift) >> 40) fail(SN_E_SHAPE, "more than 2^40 rows of heads in the cache");
  if (io->width < 0 || ((int64_t)io->width << c.shift) > k::kMaxPositions) fail(SN_E_SHAPE, "width * page must be in 0..2^29");
  if (io->pages && (!io->k || !io->v || (c.i8 && (!io->k_scale || !io->v_scale)))) fail(SN_E_INVALID, "the cache's memory is null");
  if (!c.i8 && (io->k_scale || io->v_scale)) fail(SN_E_INVALID, "scales given to a cache without them");
  check_aligned(io->k, 16, "the cache's k");
  check_aligned(io->v, 16, "the cache's v");
  for (const void* p : {(const void*)io->k_scale, (const void*)io->v_scale, (const void*)io->offsets}) check_aligned(p, 4, "a scale or offset");
  if (io->width && io->seqs && !io->table) fail(SN_E_INVALID, "table is null");
  check_aligned(io->table, 4, "table");
  if (io->table_stride < 0 || io->table_stride > (int64_t(1) << 40)) fail(SN_E_SHAPE, "table: row stride out of range");
  c.ts = io->table_stride;  // (rows that are read only may lie in each other)
  check_rows(io->past, io->seqs, io->seqs ? 1 : 0, io->seqs, SN_F32, "past");
  c.pages = io->pages, c.k = io->k, c.v = io->v, c.ks = io->k_scale, c.vs = io->v_scale;
  c.seqs = io->seqs, c.width = io->width, c.table = io->table, c.past = io->past;
  c.tokens = io->tokens, c.offsets = io->offsets, c.each = io->seqs ? io->tokens / io->seqs : 0;
  return c;
}

// The places of the call's lists, and of the cache's memory.
struct CachePlaces {
  Place table, past, offsets, k, v, ks, vs;
  explicit CachePlaces(const k::CacheArgs& c)
      : table(c.table, c.width && c.seqs ? 4 * ((c.seqs - 1) * c.ts + c.width) : 0), past(c.past, 4 * (int64_t)c.seqs),
        offsets(c.offsets, c.offsets ? 4 * ((int64_t)c.seqs + 1) : 0), k(c.k, rows(c) * c.dim * element(c)),
        v(c.v, rows(c) * c.dim * element(c)), ks(c.ks, c.i8 ? rows(c) * 4 : 0), vs(c.vs, c.i8 ? rows(c) * 4 : 0) {}
  static int64_t rows(const k::CacheArgs& c) { return (c.pages * c.kv_heads) << c.shift; }
  static int element(const k::CacheArgs& c) { return c.i8 ? 1 : dtype_size(c.dtype); }
};

k::CacheRows row_args(CacheOp& op, const sn_cache_io* io, const void* kp, int64_t k_stride, const void* vp, int64_t v_stride) {
  k::CacheRows a{};
  a.c = cache_args(op.c, io, false);
  const int64_t n = (int64_t)a.c.kv_heads * a.c.dim;
  a.krs = check_rows(kp, k_stride, a.c.tokens, n, a.c.dtype, "k");
  a.vrs = check_rows(vp, v_stride, a.c.tokens, n, a.c.dtype, "v");
  a.k = const_cast<void*>(kp), a.v = const_cast<void*>(vp);
  return a;
}

int attn_call(sn_op* p, const sn_cache_io* io, const void* q, int64_t q_stride, void* y, int64_t y_stride, void* stream, bool step) {
  return guarded([&] {
    AttnOp& op = op_of<AttnOp>(p, OP_ATTENTION);
    k::AttnArgs a = op.a;
    a.c = cache_args(a.c, io, step);
    if (a.c.seqs > op.max_seqs) fail(SN_E_SHAPE, "seqs outside the handle's range");
    if (a.c.tokens > op.max_tokens) fail(SN_E_SHAPE, "tokens outside the handle's range");
    const int64_t n = (int64_t)a.heads * a.c.dim;
    a.qs = check_rows(q, q_stride, a.c.tokens, n, a.c.dtype, "q");
    a.ys = check_rows(y, y_stride, a.c.tokens, n, a.c.dtype, "y");
    if (!step && k::attn_run_tiles(a) * a.c.kv_heads >> 24) fail(SN_E_UNSUPPORTED, "tokens * heads above 2^31 - 128 * seqs * kv_heads");
    if (step && !k::step_keys_fit(a.c)) fail(SN_E_UNSUPPORTED, "seqs * (width * page + 64) of a step not below 2^35");
    need_device(op);
    if (!a.c.tokens) return;
    const int e = dtype_size(a.c.dtype);
    const CachePlaces m(a.c);
    check_apart(Place(y, a.c.tokens, n, a.ys, e), "y",
                {Place(q, a.c.tokens, n, a.qs, e), m.table, m.past, m.offsets, m.k, m.v, m.ks, m.vs});
    a.q = q, a.y = y;
    OnDevice on(op.device);
    step ? k::attn_step(a, static_cast<hipStream_t>(stream)) : k::attn_run(a, static_cast<hipStream_t>(stream));
    HIPCHK(hipGetLastError());
  });
}

}  // namespace

extern "C" {

int sn_headnorm_create(const sn_headnorm_desc* desc, const float* q_w, const float* k_w, const double* freq,
                       int32_t device, sn_op** out) {
  return guarded([&] {
    if (!out) fail(SN_E_INVALID, "null output pointer");
    *out = nullptr;
    if (!desc) fail(SN_E_INVALID, "null description");
    const sn_headnorm_desc& d = *desc;
    check_dtype(d.dtype);
    if (d.heads < 0 || d.kv_heads < 0 || (int64_t)d.heads + d.kv_heads < 1 || d.heads > 65535 || d.kv_heads > 65535)
      fail(SN_E_SHAPE, "heads and kv_heads must be in 0..65535, one of them positive");
    if (d.head_dim < 1 || d.head_dim > 256) fail(SN_E_SHAPE, "head_dim must be in 1..256");
    if (d.rot < 0 || d.rot > d.head_dim || d.rot % 2) fail(SN_E_SHAPE, "rot must be even and at most head_dim");
    if (d.pairs != SN_PAIRS_HALVES && d.pairs != SN_PAIRS_NEIGHBOURS) fail(SN_E_INVALID, "unknown pairs");
    if (d.norm != 0 && d.norm != 1) fail(SN_E_INVALID, "norm must be 0 or 1");
    if (!(d.eps > 0.f) || !std::isfinite(d.eps)) fail(SN_E_INVALID, "eps must be positive and finite");
    if (!d.norm && (q_w || k_w)) fail(SN_E_INVALID, "weights without a norm");
    if (d.rot && !freq) fail(SN_E_INVALID, "freq is null");
    std::vector<unsigned long long> turn(d.rot / 2);
    for (int i = 0; i < d.rot / 2; ++i) {
      if (!(std::fabs(freq[i]) < 1048576.0)) fail(SN_E_INVALID, "freq has a value outside +-2^20");
      // turns per position; whole turns change nothing
      const long double t = (long double)freq[i] / 6.283185307179586476925286766559005768L;
      turn[i] = (unsigned long long)std::min(ldexpl(t - floorl(t), 64), 18446744073709551615.0L);
    }
    check_device(device);
    std::unique_ptr<HeadNormOp> op(new HeadNormOp(OP_HEADNORM, device));
    k::HeadNormArgs& a = op->a;
    a.dtype = d.dtype, a.heads = d.heads, a.kv_heads = d.kv_heads, a.dim = d.head_dim, a.rot = d.rot;
    a.pairs = d.pairs, a.norm = d.norm, a.eps = d.eps;
    if (device >= 0) {
      OnDevice on(device);
      const std::vector<float> ones(d.head_dim, 1.f);
      a.q_w = op->upload(q_w ? q_w : ones.data(), d.head_dim), a.k_w = op->upload(k_w ? k_w : ones.data(), d.head_dim);
      a.turn = op->upload(turn.data(), turn.size());
    }
    *out = op.release();
  });
}

int sn_headnorm_run(sn_op* p, int64_t tokens, const int32_t* positions, const void* q, int64_t q_stride,
                    const void* kp, int64_t k_stride, void* q_out, int64_t q_out_stride, void* k_out,
                    int64_t k_out_stride, void* stream) {
  return guarded([&] {
    HeadNormOp& op = op_of<HeadNormOp>(p, OP_HEADNORM);
    k::HeadNormArgs a = op.a;
    if (tokens < 0 || tokens >= (1 << 24)) fail(SN_E_SHAPE, "tokens must be in 0..2^24 - 1");
    const int64_t nq = (int64_t)a.heads * a.dim, nk = (int64_t)a.kv_heads * a.dim;
    const int64_t tq = a.heads ? tokens : 0, tk = a.kv_heads ? tokens : 0;
    if ((!a.heads && (q || q_out)) || (!a.kv_heads && (kp || k_out))) fail(SN_E_INVALID, "rows given for heads that the handle does not have");
    a.qs = check_rows(q, q_stride, tq, nq, a.dtype, "q");
    a.ks = check_rows(kp, k_stride, tk, nk, a.dtype, "k");
    a.qos = check_rows(q_out, q_out_stride, tq, nq, a.dtype, "q_out");
    a.kos = check_rows(k_out, k_out_stride, tk, nk, a.dtype, "k_out");
    if (a.rot) check_rows(positions, tokens, tokens ? 1 : 0, tokens, SN_F32, "positions");
    else if (positions) fail(SN_E_INVALID, "positions given to a handle without a rotation");
    if (q && q == q_out && a.qs != a.qos) fail(SN_E_SHAPE, "q in place needs one stride");
    if (kp && kp == k_out && a.ks != a.kos) fail(SN_E_SHAPE, "k in place needs one stride");
    need_device(op);
    if (!tokens) return;
    const int e = dtype_size(a.dtype);
    const Place pq(q, tq, nq, a.qs, e), pk(kp, tk, nk, a.ks, e), pp(positions, positions ? 4 * tokens : 0);
    const Place oq(q_out, tq, nq, a.qos, e), ok(k_out, tk, nk, a.kos, e);
    check_apart(oq, "q_out", {pq}, true);
    check_apart(ok, "k_out", {pk}, true);
    check_apart(oq, "q_out", {pk, pp, ok});
    check_apart(ok, "k_out", {pq, pp});
    a.tokens = tokens, a.positions = positions;
    a.q = q, a.k = kp, a.qo = q_out, a.ko = k_out;
    OnDevice on(op.device);
    k::head_norm(a, static_cast<hipStream_t>(stream));
    HIPCHK(hipGetLastError());
  });
}

int sn_cache_create(const sn_cache_desc* desc, int32_t device, sn_op** out) {
  return guarded([&] {
    if (!out) fail(SN_E_INVALID, "null output pointer");
    *out = nullptr;
    if (!desc) fail(SN_E_INVALID, "null description");
    const k::CacheArgs c = cache_of(*desc);
    check_device(device);
    std::unique_ptr<CacheOp> op(new CacheOp(OP_CACHE, device));
    op->c = c;
    *out = op.release();
  });
}

int sn_cache_write(sn_op* p, const sn_cache_io* io, const void* kp, int64_t k_stride, const void* vp, int64_t v_stride,
                   void* stream) {
  return guarded([&] {
    CacheOp& op = op_of<CacheOp>(p, OP_CACHE);
    const k::CacheRows a = row_args(op, io, kp, k_stride, vp, v_stride);
    need_device(op);
    if (!a.c.tokens || !a.c.pages) return;
    const int e = dtype_size(a.c.dtype);
    const int64_t n = (int64_t)a.c.kv_heads * a.c.dim;
    const CachePlaces m(a.c);
    const Place rk(kp, a.c.tokens, n, a.krs, e), rv(vp, a.c.tokens, n, a.vrs, e);
    check_apart(m.k, "the cache's k", {rk, rv, m.table, m.past, m.offsets, m.v, m.ks, m.vs});
    check_apart(m.v, "the cache's v", {rk, rv, m.table, m.past, m.offsets, m.ks, m.vs});
    check_apart(m.ks, "the cache's k_scale", {rk, rv, m.table, m.past, m.offsets, m.vs});
    check_apart(m.vs, "the cache's v_scale", {rk, rv, m.table, m.past, m.offsets});
    OnDevice on(op.device);
    k::cache_write(a, static_cast<hipStream_t>(stream));
    HIPCHK(hipGetLastError());
  });
}

int sn_cache_read(sn_op* p, const sn_cache_io* io, void* kp, int64_t k_stride, void* vp, int64_t v_stride, void* stream) {
  return guarded([&] {
    CacheOp& op = op_of<CacheOp>(p, OP_CACHE);
    const k::CacheRows a = row_args(op, io, kp, k_stride, vp, v_stride);
    need_device(op);
    if (!a.c.tokens) return;
    const int e = dtype_size(a.c.dtype);
    const int64_t n = (int64_t)a.c.kv_heads * a.c.dim;
    const CachePlaces m(a.c);
    const Place rk(kp, a.c.tokens, n, a.krs, e), rv(vp, a.c.tokens, n, a.vrs, e);
    check_apart(rk, "k", {m.table, m.past, m.offsets, m.k, m.v, m.ks, m.vs, rv});
    check_apart(rv, "v", {m.table, m.past, m.offsets, m.k, m.v, m.ks, m.vs});
    OnDevice on(op.device);
    k::cache_read(a, static_cast<hipStream_t>(stream));
    HIPCHK(hipGetLastError());
  });
}

int sn_attn_create(const sn_attn_desc* desc, int32_t device, sn_op** out) {
  return guarded([&] {
    if (!out) fail(SN_E_INVALID, "null output pointer");
    *out = nullptr;
    if (!desc) fail(SN_E_INVALID, "null description");
    const sn_attn_desc& d = *desc;
    const k::CacheArgs c = cache_of(d.cache);
    if (d.heads < 1 || d.heads > 65535 || d.heads % c.kv_heads) fail(SN_E_SHAPE, "heads must be a multiple of kv_heads up to 65535");
    if (d.window < 0 || d.window > k::kMaxPositions) fail(SN_E_SHAPE, "window must be in 0..2^29");
    if (!std::isfinite(d.scale)) fail(SN_E_INVALID, "scale must be finite");
    if (d.max_seqs < 1 || d.max_seqs > 65535) fail(SN_E_SHAPE, "max_seqs must be in 1..65535");
    if (d.max_tokens < 1 || d.max_tokens > (1 << 26)) fail(SN_E_SHAPE, "max_tokens must be in 1..2^26");
    check_device(device);
    std::unique_ptr<AttnOp> op(new AttnOp(OP_ATTENTION, device));
    op->max_seqs = d.max_seqs, op->max_tokens = std::max<int64_t>(d.max_tokens, d.max_seqs);
    op->a.c = c, op->a.heads = d.heads, op->a.window = d.window, op->a.scale = d.scale;
    if (device >= 0) {
      OnDevice on(device);
      int64_t o, m, counts;
      k::attn_workspace(op->a, o, m, counts);
      op->a.ws_o = static_cast<float*>(op->alloc(o * sizeof(float)));
      op->a.ws_m = static_cast<float*>(op->alloc(m * sizeof(float)));
      op->a.count = static_cast<unsigned*>(op->alloc(counts * sizeof(unsigned)));
      HIPCHK(hipMemset(op->a.count, 0, counts * sizeof(unsigned)));
      HIPCHK(hipDeviceSynchronize());
    }
    *out = op.release();
  });
}

int sn_attn_run(sn_op* op, const sn_cache_io* io, const void* q, int64_t q_stride, void* y, int64_t y_stride, void* stream) {
  return attn_call(op, io, q, q_stride, y, y_stride, stream, false);
}

int sn_attn_step(sn_op* op, const sn_cache_io* io, const void* q, int64_t q_stride, void* y, int64_t y_stride, void* stream) {
  return attn_call(op, io, q, q_stride, y, y_stride, stream, true);
}

}  // extern "C"
