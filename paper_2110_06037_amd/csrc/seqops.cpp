// Sequence operators of the C ABI: handles with their weights and
// workspaces, argument checks, and the calls of the kernels' launchers.
#include <hip/hip_runtime.h>

#include <cmath>
#include <memory>

#include "api_guard.hpp"
#include "core.hpp"
#include "kernels/seq.hpp"

using namespace sn;

#define HIPCHK(expr)                                                                        \
  do {                                                                                      \
    hipError_t e_ = (expr);                                                                 \
    if (e_ != hipSuccess) fail(SN_E_DEVICE, std::string(#expr) + ": " + hipGetErrorString(e_)); \
  } while (0)

enum OpKind { OP_NORM, OP_LINEAR4 };

struct sn_op {
  const OpKind kind;
  const int device;
  std::vector<void*> owned;  // device memory
  sn_op(OpKind k, int dev) : kind(k), device(dev) {}
  virtual ~sn_op() {
    if (owned.empty()) return;
    int cur = 0;
    (void)hipGetDevice(&cur);
    (void)hipSetDevice(device);
    for (void* p : owned) (void)hipFree(p);
    (void)hipSetDevice(cur);
  }
  void* alloc(size_t bytes) {
    void* p = nullptr;
    const hipError_t e = hipMalloc(&p, std::max<size_t>(bytes, 256));
    if (e == hipErrorOutOfMemory) (void)hipGetLastError();
    if (e != hipSuccess) fail(SN_E_DEVICE, std::string("hipMalloc: ") + hipGetErrorString(e));
    owned.push_back(p);
    return p;
  }
  template <typename V>
  V* upload(const V* host, size_t n, size_t padded = 0) {
    if (!host) return nullptr;
    V* p = static_cast<V*>(alloc(std::max(n, padded) * sizeof(V)));
    if (padded > n) HIPCHK(hipMemset(p + n, 0, (padded - n) * sizeof(V)));
    HIPCHK(hipMemcpy(p, host, n * sizeof(V), hipMemcpyHostToDevice));
    return p;
  }
};

namespace {

// The handle's device for the length of a call; the caller's afterwards.
struct OnDevice {
  int before = -1;
  explicit OnDevice(int device) {
    int cur = 0;
    HIPCHK(hipGetDevice(&cur));
    if (cur == device) return;
    HIPCHK(hipSetDevice(device));
    before = cur;
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

void check_device(int device) {
  if (device < -1) fail(SN_E_INVALID, "device must be >= -1");
  if (device < 0) return;
  int n = 0;
  HIPCHK(hipGetDeviceCount(&n));
  if (device >= n) fail(SN_E_DEVICE, "no such HIP device");
}

void check_dtype(int dtype) {
  if (dtype < SN_F32 || dtype > SN_BF16) fail(SN_E_INVALID, "unknown dtype");
}

void check_finite(const float* v, int64_t n, const char* what) {
  for (int64_t i = 0; v && i < n; ++i)
    if (!std::isfinite(v[i])) fail(SN_E_INVALID, std::string(what) + " has a value that is not finite");
}

template <class Op>
Op& op_of(sn_op* p, OpKind kind) {
  if (!p) fail(SN_E_INVALID, "null operator pointer");
  if (p->kind != kind) fail(SN_E_INVALID, "the handle is of another operator");
  return *static_cast<Op*>(p);
}

// A tensor of `rows` rows of `n` elements: given, rows that do not overlap,
// elements on their own alignment.
void check_rows(const void* p, int64_t stride, int64_t rows, int64_t n, int dtype, const char* what) {
  if (rows == 0) return;
  if (!p) fail(SN_E_INVALID, std::string(what) + " is null");
  if (rows > 1 && stride < n) fail(SN_E_SHAPE, std::string(what) + ": row stride below the row's length");
  if (stride < 0 || stride > (int64_t(1) << 40)) fail(SN_E_SHAPE, std::string(what) + ": row stride out of range");
  if (reinterpret_cast<uintptr_t>(p) % dtype_size(dtype)) fail(SN_E_INVALID, std::string(what) + " is not aligned to its elements");
}

void need_device(const sn_op& op) {
  if (op.device < 0) fail(SN_E_DEVICE, "host-only handle cannot run");
}

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
    check_rows(x, x_stride, rows, a.dim, a.dtype, "x");
    if (a.gate) check_rows(gate, gate_stride, rows, a.dim, a.dtype, "gate");
    else if (gate) fail(SN_E_INVALID, "a gate given to a handle without one");
    if (a.rdtype >= 0) {
      check_rows(res, res_stride, rows, a.dim, a.rdtype, "res");
      check_rows(res_out, res_out_stride, rows, a.dim, a.rdtype, "res_out");
      if (res == res_out && res_stride != res_out_stride) fail(SN_E_SHAPE, "res in place needs one stride");
    } else if (res || res_out) {
      fail(SN_E_INVALID, "a residual given to a handle without one");
    }
    if (has_y) check_rows(y, y_stride, rows, a.dim, a.dtype, "y");
    else if (y) fail(SN_E_INVALID, "y given to a handle without a pre norm (its output is res_out)");
    if (y && y == x && x_stride != y_stride) fail(SN_E_SHAPE, "y in place needs one stride");
    need_device(op);
    if (!rows) return;
    a.rows = rows;
    a.x = x, a.xs = x_stride, a.g = gate, a.gs = gate_stride, a.r = res, a.rs = res_stride;
    a.ro = res_out, a.ros = res_out_stride, a.y = y, a.ys = y_stride;
    OnDevice on(op.device);
    k::block_norm(a, static_cast<hipStream_t>(stream));
    HIPCHK(hipGetLastError());
  });
}

int sn_linear4_create(const sn_linear4_desc* desc, const uint8_t* q, const uint16_t* scale, const uint8_t* zero,
                      const float* bias, int32_t device, sn_op** out) {
  return guarded([&] {
    if (!out) fail(SN_E_INVALID, "null output pointer");
    *out = nullptr;
    if (!desc || !q || !scale) fail(SN_E_INVALID, "null description, codes or scales");
    const sn_linear4_desc& d = *desc;
    check_dtype(d.dtype);
    if (d.rows < 1 || d.cols < 1) fail(SN_E_SHAPE, "rows and cols must be positive");
    if (d.rows > (1 << 24) || d.cols > (1 << 20)) fail(SN_E_UNSUPPORTED, "more than 2^24 rows or 2^20 cols");
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
      a.q = op->upload(q, (size_t)d.rows * ((d.cols + 1) / 2));
      a.scale = reinterpret_cast<const k::f16*>(op->upload(scale, n));
      a.zero = op->upload(zero, n);
      a.bias = op->upload(bias, d.rows);
    }
    *out = op.release();
  });
}

int sn_linear4_run(sn_op* p, int64_t m, const void* x, int64_t x_stride, void* y, int64_t y_stride, void* stream) {
  return guarded([&] {
    Linear4Op& op = op_of<Linear4Op>(p, OP_LINEAR4);
    k::Linear4Args a = op.a;
    if (m < 0 || m > 65535 * 8) fail(SN_E_SHAPE, "m must be in 0..524280");
    check_rows(x, x_stride, m, a.cols, a.dtype, "x");
    check_rows(y, y_stride, m, a.rows, a.dtype, "y");
    need_device(op);
    if (!m) return;
    a.m = m, a.x = x, a.xs = x_stride, a.y = y, a.ys = y_stride;
    OnDevice on(op.device);
    k::linear4(a, static_cast<hipStream_t>(stream));
    HIPCHK(hipGetLastError());
  });
}

}  // extern "C"
