// The C boundary of the library: status codes out, no exception across.
#pragma once

#include <new>
#include <string>

#include "core.hpp"

namespace sn {

// description of this thread's last failure (sn_last_error)
inline std::string& api_error() {
  static thread_local std::string e;
  return e;
}

template <class F>
int guarded(F&& f) {
  try {
    f();
    return SN_OK;
  } catch (const Error& e) {
    api_error() = e.what();
    return e.code;
  } catch (const std::bad_alloc&) {
    api_error() = "out of host memory";
    return SN_E_INTERNAL;
  } catch (const std::exception& e) {
    api_error() = e.what();
    return SN_E_INTERNAL;
  } catch (...) {
    api_error() = "unknown error";
    return SN_E_INTERNAL;
  }
}

}  // namespace sn
