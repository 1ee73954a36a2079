// Sequence operators of the C ABI: handles with their weights and
// workspaces, argument checks, and the calls of the kernels' launchers.
#include <memory>

#include "api_guard.hpp"
#include "kernels/seq.hpp"
#include "seqop.hpp"

using namespace sn;

namespace {

// ------------------------------------------------------------------ norms
struct NormOp : sn_op {
  k::NormArgs a{};
  using sn_op::sn_op;
};

// ------------------------------------------------------------------ 4-bit products
struct Linear4Op : sn_op {
  k::Linear4Args a{};
  using sn_op::sn_op;
};

// ------------------------------------------------------------------ scan
struct ScanOp : sn_op {
  k::ScanArgs a{};
  int max_seqs = 0;
  int64_t max_tokens = 0;
  using sn_op::sn_op;
};

// Either one tensor or two that do not touch.
void check_in_out(const void* in, const void* out, int64_t bytes, const char* what) {
  const uintptr_t i = reinterpret_cast<uintptr_t>(in), o = reinterpret_cast<uintptr_t>(out);
  if (in && out && i != o && i < o + bytes && o < i + bytes)
    fail(SN_E_INVALID, std::string(what) + " overlaps its input without being it");
}

// The call's arguments, checked.
k::ScanArgs scan_args(const ScanOp& op, const sn_scan_io* io, bool step) {
  if (!io) fail(SN_E_INVALID, "null arguments");
  k::ScanArgs a = op.a;
  const int e = dtype_size(a.dtype);
  if (io->seqs < 0 || io->seqs > op.max_seqs) fail(SN_E_SHAPE, "seqs outside the handle's range");
  if (io->tokens < 0 || io->tokens > op.max_tokens) fail(SN_E_SHAPE, "tokens outside the handle's range");
  if (io->seqs == 0 && io->tokens) fail(SN_E_SHAPE, "tokens without a sequence");
  if (step && (io->tokens != io->seqs || io->offsets)) fail(SN_E_SHAPE, "a step takes one token per sequence");
  if (io->seqs && !io->offsets && io->tokens % io->seqs)
    fail(SN_E_SHAPE, "tokens are no multiple of seqs, and there are no offsets");
  a.xs = check_rows(io->x, io->x_stride, io->tokens, a.chans, a.dtype, "x");
  a.dts = check_rows(io->dt, io->dt_stride, io->tokens, a.heads, a.dtype, "dt");
  a.ys = check_rows(io->y, io->y_stride, io->tokens, (int64_t)a.heads * a.dim, a.dtype, "y");
  // 67 rows of x and 64 of y are addressed with 32-bit offsets
  if (std::max(a.xs, a.ys) * e * 68 >= (int64_t(1) << 31)) fail(SN_E_UNSUPPORTED, "row stride above 2^31 / 68 bytes");
  for (const void* p : {io->window, (const void*)io->window_out})
    if (reinterpret_cast<uintptr_t>(p) % e) fail(SN_E_INVALID, "window is not aligned to its elements");
  for (const void* p : {(const void*)io->state, (const void*)io->state_out, (const void*)io->offsets})
    if (reinterpret_cast<uintptr_t>(p) % 4) fail(SN_E_INVALID, "state or offsets are not aligned to 4 bytes");
  check_in_out(io->window, io->window_out, (int64_t)io->seqs * (a.conv - 1) * a.chans * e, "window_out");
  check_in_out(io->state, io->state_out, (int64_t)io->seqs * a.heads * a.dim * a.state * 4, "state_out");
  a.seqs = io->seqs, a.tokens = io->tokens, a.offsets = io->offsets;
  a.x = io->x, a.dt = io->dt, a.y = io->y;
  a.window = io->window, a.window_out = a.conv > 1 ? io->window_out : nullptr;
  a.state_in = io->state, a.state_out = io->state_out;
  return a;
}

// What a call writes lies apart from what it reads (windows and states may be
// updated in place: check_in_out).
void check_scan_apart(const k::ScanArgs& a, const sn_scan_io& io) {
  const int e = dtype_size(a.dtype);
  const int64_t wbytes = (int64_t)a.seqs * (a.conv - 1) * a.chans * e, hbytes = (int64_t)a.seqs * a.heads * a.dim * a.state * 4;
  const Place x(io.x, a.tokens, a.chans, a.xs, e), dt(io.dt, a.tokens, a.heads, a.dts, e);
  const Place y(io.y, a.tokens, (int64_t)a.heads * a.dim, a.ys, e), offsets(io.offsets, 4 * ((int64_t)a.seqs + 1));
  const Place w(io.window, wbytes), wo(io.window_out, wbytes), h(io.state, hbytes), ho(io.state_out, hbytes);
  check_apart(y, "y", {x, dt, offsets, w, wo, h, ho});
  check_apart(wo, "window_out", {x, dt, offsets, h, ho});
  check_apart(ho, "state_out", {x, dt, offsets, w});
}

}  // namespace

extern "C" {

void sn_op_destroy(sn_op* op) {
  try {
    delete op;
  } catch (...) {
  }
}

int sn_norm_create(const sn_norm_desc* desc, const float* post_w, const float* post_b, const float* pre_w,
                   const float* pre_b, const float* scale_v, int32_t device, sn_op** out) {
  return guarded([&] {
    if (!out) fail(SN_E_INVALID, "null output pointer");
    *out = nullptr;
    if (!desc) fail(SN_E_INVALID, "null description");
    const sn_norm_desc& d = *desc;
    check_dtype(d.dtype);
    if (d.res_dtype != -1 && d.res_dtype != d.dtype && d.res_dtype != SN_F32)
      fail(SN_E_INVALID, "res_dtype is the dtype, SN_F32 or -1");
    if (d.dim < 1 || d.dim > k::kNormMaxDim) fail(SN_E_SHAPE, "dim must be in 1..32768");
    if (d.groups < 1 || d.dim % d.groups) fail(SN_E_SHAPE, "groups must divide dim");
    if (d.groups > 1 && pre_w) fail(SN_E_UNSUPPORTED, "groups above 1 need a post norm alone");
    if (d.kind != SN_NORM_RMS && d.kind != SN_NORM_LAYER) fail(SN_E_INVALID, "unknown norm kind");
    if (d.gate < SN_GATE_NONE || d.gate > SN_GATE_AFTER) fail(SN_E_INVALID, "unknown gate");
    if (!(d.eps > 0.f) || !std::isfinite(d.eps)) fail(SN_E_INVALID, "eps must be positive and finite");
    if (!std::isfinite(d.scale)) fail(SN_E_INVALID, "scale must be finite");
    if ((post_b && !post_w) || (pre_b && !pre_w)) fail(SN_E_INVALID, "a norm's bias needs its weight");
    check_device(device);
    std::unique_ptr<NormOp> op(new NormOp(OP_NORM, device));
    k::NormArgs& a = op->a;
    a.dtype = d.dtype, a.rdtype = d.res_dtype, a.dim = d.dim, a.groups = d.groups, a.kind = d.kind, a.gate = d.gate;
    a.eps = d.eps, a.scale = d.scale;
    if (device >= 0) {
      OnDevice on(device);
      a.post_w = op->upload(post_w, d.dim), a.post_b = op->upload(post_b, d.dim);
      a.pre_w = op->upload(pre_w, d.dim), a.pre_b = op->upload(pre_b, d.dim);
      a.scale_v = op->upload(scale_v, d.dim);
    } else {
      a.pre_w = pre_w;  // only whether it is there counts
    }
    *out = op.release();
  });
}

int sn_norm_run(sn_op* p, int64_t rows, const void* x, int64_t x_stride, const void* gate, int64_t gate_stride,
                const void* res, int64_t res_stride, void* res_out, int64_t res_out_stride, void* y,
                int64_t y_stride, void* stream) {
  return guarded([&] {
    NormOp& op = op_of<NormOp>(p, OP_NORM);
    k::NormArgs a = op.a;
    if (rows < 0 || rows >= (int64_t(1) << 31) || rows * a.groups >= (int64_t(1) << 31)) fail(SN_E_SHAPE, "rows out of range");
    const bool has_y = a.pre_w || a.rdtype < 0;
    a.xs = check_rows(x, x_stride, rows, a.dim, a.dtype, "x");
    if (a.gate) a.gs = check_rows(gate, gate_stride, rows, a.dim, a.dtype, "gate");
    else if (gate) fail(SN_E_INVALID, "a gate given to a handle without one");
    if (a.rdtype >= 0) {
      a.rs = check_rows(res, res_stride, rows, a.dim, a.rdtype, "res");
      a.ros = check_rows(res_out, res_out_stride, rows, a.dim, a.rdtype, "res_out");
      if (res == res_out && a.rs != a.ros) fail(SN_E_SHAPE, "res in place needs one stride");
    } else if (res || res_out) {
      fail(SN_E_INVALID, "a residual given to a handle without one");
    }
    if (has_y) a.ys = check_rows(y, y_stride, rows, a.dim, a.dtype, "y");
    else if (y) fail(SN_E_INVALID, "y given to a handle without a pre norm (its output is res_out)");
    if (y && y == x && a.xs != a.ys) fail(SN_E_SHAPE, "y in place needs one stride");
    need_device(op);
    if (!rows) return;
    const int e = dtype_size(a.dtype), er = dtype_size(std::max(a.rdtype, 0));
    const Place px(x, rows, a.dim, a.xs, e), pg(gate, rows, a.dim, a.gs, e), pr(res, rows, a.dim, a.rs, er);
    const Place py(y, rows, a.dim, a.ys, e), pro(res_out, rows, a.dim, a.ros, er);
    check_apart(py, "y", {px, pg, pr}, true);
    check_apart(pro, "res_out", {px, pg, pr}, true);
    check_apart(py, "y", {pro});
    a.rows = rows;
    a.x = x, a.g = gate, a.r = res, a.ro = res_out, a.y = y;
    OnDevice on(op.device);
    k::block_norm(a, static_cast<hipStream_t>(stream));
    HIPCHK(hipGetLastError());
  });
}

int sn_qlinear_create(const sn_qlinear_desc* desc, const uint8_t* q, const uint16_t* scale, const uint8_t* zero,
                      const float* bias, int32_t device, sn_op** out) {
  return guarded([&] {
    if (!out) fail(SN_E_INVALID, "null output pointer");
    *out = nullptr;
    if (!desc || !q || !scale) fail(SN_E_INVALID, "null description, codes or scales");
    const sn_qlinear_desc& d = *desc;
    check_dtype(d.dtype);
    if (d.rows < 1 || d.cols < 1) fail(SN_E_SHAPE, "rows and cols must be positive");
    if (d.rows > (1 << 24) || d.cols > (1 << 20)) fail(SN_E_UNSUPPORTED, "more than 2^24 rows or 2^20 cols");
    // (one launch lays them out, with fewer than 2^32 threads)
    if (k::linear4_blocks(d.rows, d.cols) >= (int64_t(1) << 24)) fail(SN_E_UNSUPPORTED, "more than 2^24 blocks of 2048 weights");
    if (d.group < 32 || d.group % 32) fail(SN_E_SHAPE, "group must be a multiple of 32");
    if (d.act < SN_ACT_NONE || d.act > SN_ACT_RELU6) fail(SN_E_INVALID, "unknown activation");
    const int64_t groups = (d.cols + (int64_t)d.group - 1) / d.group;
    const int64_t n = d.rows * groups;
    for (int64_t i = 0; i < n; ++i)
      if ((scale[i] & 0x7c00) == 0x7c00) fail(SN_E_INVALID, "a scale is not finite");
    for (int64_t i = 0; zero && i < n; ++i)
      if (zero[i] > 15) fail(SN_E_INVALID, "a zero point above 15");
    check_finite(bias, d.rows, "bias");
    check_device(device);
    std::unique_ptr<Linear4Op> op(new Linear4Op(OP_LINEAR4, device));
    k::Linear4Args& a = op->a;
    a.dtype = d.dtype, a.act = d.act, a.rows = d.rows, a.cols = d.cols, a.group = d.group;
    if (device >= 0) {
      OnDevice on(device);
      // the caller's arrays, and from them the kernels' order
      sn_op raw(OP_LINEAR4, device);
      const uint8_t* rq = raw.upload(q, (size_t)d.rows * ((d.cols + 1) / 2));
      const uint16_t* rs = raw.upload(scale, n);
      const uint8_t* rz = raw.upload(zero, n);
      const int64_t blocks = k::linear4_blocks(d.rows, d.cols), scales = blocks * 64 / k::linear4_gs(d.group);
      unsigned* wq = static_cast<unsigned*>(op->alloc(blocks * 1024));
      unsigned* ws = static_cast<unsigned*>(op->alloc(scales * 4));
      k::linear4_pack(d.dtype, rq, reinterpret_cast<const k::f16*>(rs), rz, d.rows, d.cols, d.group, wq, ws, nullptr);
      HIPCHK(hipGetLastError());
      a.wq = wq, a.ws = ws;
      a.bias = op->upload(bias, d.rows);
      HIPCHK(hipDeviceSynchronize());
    }
    *out = op.release();
  });
}

int sn_qlinear_run(sn_op* p, int64_t m, const void* x, int64_t x_stride, void* y, int64_t y_stride, void* stream) {
  return guarded([&] {
    Linear4Op& op = op_of<Linear4Op>(p, OP_LINEAR4);
    k::Linear4Args a = op.a;
    if (m < 0 || m > 65535 * 4) fail(SN_E_SHAPE, "m must be in 0..262140");
    a.xs = check_rows(x, x_stride, m, a.cols, a.dtype, "x");
    a.ys = check_rows(y, y_stride, m, a.rows, a.dtype, "y");
    need_device(op);
    if (!m) return;
    const int e = dtype_size(a.dtype);
    check_apart(Place(y, m, a.rows, a.ys, e), "y", {Place(x, m, a.cols, a.xs, e)});
    a.m = m, a.x = x, a.y = y;
    OnDevice on(op.device);
    k::linear4(a, static_cast<hipStream_t>(stream));
    HIPCHK(hipGetLastError());
  });
}

int sn_scan_create(const sn_scan_desc* desc, const float* conv_w, const float* conv_b, const float* a_,
                   const float* d_, const float* dt_bias, int32_t device, sn_op** out) {
  return guarded([&] {
    if (!out) fail(SN_E_INVALID, "null output pointer");
    *out = nullptr;
    if (!desc || !conv_w || !a_) fail(SN_E_INVALID, "null description, conv_w or a");
    const sn_scan_desc& d = *desc;
    check_dtype(d.dtype);
    if (d.heads < 1 || d.head_dim < 1 || d.groups < 1 || d.state < 1) fail(SN_E_SHAPE, "sizes must be positive");
    if (d.heads % d.groups) fail(SN_E_SHAPE, "groups must divide heads");
    if (d.groups > 16384) fail(SN_E_UNSUPPORTED, "more than 16384 groups");
    if (d.state > 256) fail(SN_E_UNSUPPORTED, "state above 256");
    if (d.conv < 1 || d.conv > 4) fail(SN_E_UNSUPPORTED, "conv must be in 1..4");
    const int64_t chans = (int64_t)d.heads * d.head_dim + 2 * (int64_t)d.groups * d.state;
    if (d.heads > 65535 || d.head_dim > 65535 || chans > (1 << 24)) fail(SN_E_UNSUPPORTED, "more than 2^24 channels");
    if (d.max_seqs < 1 || d.max_seqs > 65535) fail(SN_E_SHAPE, "max_seqs must be in 1..65535");
    if (d.max_tokens < 1 || d.max_tokens > (1 << 27)) fail(SN_E_SHAPE, "max_tokens must be in 1..2^27");
    check_finite(conv_w, chans * d.conv, "conv_w");
    check_finite(conv_b, chans, "conv_b");
    check_finite(a_, d.heads, "a");
    check_finite(d_, d.heads, "d");
    check_finite(dt_bias, d.heads, "dt_bias");
    for (int h = 0; h < d.heads; ++h)
      if (a_[h] > 0.f) fail(SN_E_INVALID, "a has a positive value (states would grow)");
    check_device(device);
    std::unique_ptr<ScanOp> op(new ScanOp(OP_SCAN, device));
    op->max_seqs = d.max_seqs, op->max_tokens = d.max_tokens;
    k::ScanArgs& a = op->a;
    a.dtype = d.dtype, a.heads = d.heads, a.dim = d.head_dim, a.groups = d.groups, a.state = d.state;
    a.conv = d.conv, a.chans = (int)chans, a.np = k::scan_np(d.state);
    if (device >= 0) {
      OnDevice on(device);
      std::vector<float> w(4 * chans, 0.f), zeros(chans, 0.f), a2(d.heads);
      for (int64_t c = 0; c < chans; ++c)
        for (int j = 0; j < d.conv; ++j) w[(4 - d.conv + j) * chans + c] = conv_w[c * d.conv + j];
      for (int h = 0; h < d.heads; ++h) a2[h] = (float)((double)a_[h] * 1.4426950408889634074);
      a.conv_w = op->upload(w.data(), w.size());
      a.conv_b = op->upload(conv_b ? conv_b : zeros.data(), chans);
      a.a2 = op->upload(a2.data(), d.heads);
      a.d = op->upload(d_ ? d_ : zeros.data(), d.heads);
      a.dt_bias = op->upload(dt_bias ? dt_bias : zeros.data(), d.heads);
      const int64_t slots = k::scan_slots(d.max_tokens, d.max_seqs), Q = k::kScanChunk;
      auto floats = [&](int64_t n) { return static_cast<float*>(op->alloc(n * 4)); };
      a.ws_c = op->alloc(slots * d.groups * Q * a.np * 4);
      a.ws_b = op->alloc(slots * d.groups * Q * a.np * 4);
      a.ws_s = floats(slots * d.groups * k::kScanS);
      a.ws_max = floats(slots * d.groups * k::kScanMax);
      a.ws_dt = floats(slots * d.heads * k::kScanDtRow);
      // segments' states: kScanUnits waves of 16 columns and as much again for
      // the sequences' last ones, if calls can be so long (two chunks at least)
      const int64_t hold = (int64_t)d.heads * d.head_dim * d.state, most = k::scan_segment_slots(slots, d.max_seqs, 2);
      a.seg_cap = std::min(int64_t(2) * k::kScanUnits * 16 * d.state, most * hold);
      a.ws_seg = floats(a.seg_cap);
      a.ws_decay = floats(std::max<int64_t>(1, a.seg_cap / hold) * d.heads);
      a.wcopy = op->alloc(d.max_seqs * (d.conv - 1) * chans * dtype_size(d.dtype));
      const size_t counters = (size_t)d.max_seqs * d.groups * sizeof(unsigned);
      a.count = static_cast<unsigned*>(op->alloc(counters));
      HIPCHK(hipMemset(a.count, 0, counters));
      HIPCHK(hipDeviceSynchronize());
    }
    *out = op.release();
  });
}

int sn_scan_run(sn_op* p, const sn_scan_io* io, void* stream) {
  return guarded([&] {
    ScanOp& op = op_of<ScanOp>(p, OP_SCAN);
    const k::ScanArgs a = scan_args(op, io, false);
    need_device(op);
    if (!a.seqs) return;
    check_scan_apart(a, *io);
    OnDevice on(op.device);
    k::scan_run(a, static_cast<hipStream_t>(stream));
    HIPCHK(hipGetLastError());
  });
}

int sn_scan_step(sn_op* p, const sn_scan_io* io, void* stream) {
  return guarded([&] {
    ScanOp& op = op_of<ScanOp>(p, OP_SCAN);
    const k::ScanArgs a = scan_args(op, io, true);
    need_device(op);
    if (!a.seqs) return;
    check_scan_apart(a, *io);
    OnDevice on(op.device);
    k::scan_step(a, static_cast<hipStream_t>(stream));
    HIPCHK(hipGetLastError());
  });
}

}  // extern "C"
