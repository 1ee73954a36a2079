// What the sequence and attention operators of the C ABI share: the handle with
// its device memory, and the checks of a call's arguments.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "core.hpp"

#define HIPCHK(expr)                                                                        \
  do {                                                                                      \
    hipError_t e_ = (expr);                                                                 \
    if (e_ != hipSuccess) sn::fail(SN_E_DEVICE, std::string(#expr) + ": " + hipGetErrorString(e_)); \
  } while (0)

enum OpKind { OP_NORM, OP_LINEAR4, OP_SCAN, OP_HEADNORM, OP_CACHE, OP_ATTENTION };

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
    if (e != hipSuccess) sn::fail(SN_E_DEVICE, std::string("hipMalloc: ") + hipGetErrorString(e));
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

namespace sn {

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

inline void check_device(int device) {
  if (device < -1) fail(SN_E_INVALID, "device must be >= -1");
  if (device < 0) return;
  int n = 0;
  HIPCHK(hipGetDeviceCount(&n));
  if (device >= n) fail(SN_E_DEVICE, "no such HIP device");
}

inline void check_dtype(int dtype) {
  if (dtype < SN_F32 || dtype > SN_BF16) fail(SN_E_INVALID, "unknown dtype");
}

inline void check_finite(const float* v, int64_t n, const char* what) {
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
// elements on their own alignment.  Returns the stride to use: that of one row
// means nothing to the caller, but the kernels' ranges are made from it.
inline int64_t check_rows(const void* p, int64_t stride, int64_t rows, int64_t n, int dtype, const char* what) {
  if (rows == 0) return n;
  if (!p) fail(SN_E_INVALID, std::string(what) + " is null");
  if (rows == 1) stride = n;
  if (stride < n) fail(SN_E_SHAPE, std::string(what) + ": row stride below the row's length");
  if (stride > (int64_t(1) << 40)) fail(SN_E_SHAPE, std::string(what) + ": row stride out of range");
  if (reinterpret_cast<uintptr_t>(p) % dtype_size(dtype)) fail(SN_E_INVALID, std::string(what) + " is not aligned to its elements");
  return stride;
}

// A tensor's place in memory: `rows` rows of `bytes`, `step` bytes apart.
struct Place {
  uintptr_t at;
  int64_t rows, bytes, step;
  Place(const void* p, int64_t rows, int64_t n, int64_t stride, int64_t e)
      : at(reinterpret_cast<uintptr_t>(p)), rows(p ? rows : 0), bytes(n * e), step(stride * e) {}
  Place(const void* p, int64_t n) : Place(p, n > 0, n, n, 1) {}  // in one piece
  uintptr_t end() const { return at + (rows - 1) * step + bytes; }
  bool same(const Place& o) const { return at == o.at && rows == o.rows && bytes == o.bytes && step == o.step; }
};

// Whether two tensors share a byte.  Rows of one step may lie between each
// other's (slices of one wider tensor); of two steps, overlapping ranges count.
inline bool meet(const Place& a, const Place& b) {
  if (!a.rows || !b.rows || a.end() <= b.at || b.end() <= a.at) return false;
  if (a.rows == 1 && b.rows == 1) return true;
  const int64_t step = a.rows == 1 ? b.step : a.step;
  if (a.rows > 1 && b.rows > 1 && a.step != b.step) return true;
  const int64_t d = ((int64_t)(b.at - a.at) % step + step) % step;
  return d < a.bytes || d + b.bytes > step;
}

// Other workgroups read an input while an output is written: none may lie in
// an input, but for `in_place` kernels, where every element is read by the thread
// that writes it, as the same tensor.
inline void check_apart(const Place& out, const char* what, std::initializer_list<Place> others, bool in_place = false) {
  for (const Place& o : others)
    if (meet(out, o) && !(in_place && out.same(o))) fail(SN_E_INVALID, std::string(what) + " overlaps another tensor of the call");
}

inline void need_device(const sn_op& op) {
  if (op.device < 0) fail(SN_E_DEVICE, "host-only handle cannot run");
}

}  // namespace sn
