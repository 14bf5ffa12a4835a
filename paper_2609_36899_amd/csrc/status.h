// The C ABI's error report: sets this thread's last_error() message and
// returns the code.
#pragma once

#include <string>

namespace pdec {

int fail(int code, const std::string& msg);

}  // namespace pdec

#define HIP_OR_FAIL(expr)                                                                \
  do {                                                                                   \
    hipError_t e_ = (expr);                                                              \
    if (e_ != hipSuccess)                                                                \
      return pdec::fail(PDEC_HIP_ERROR, std::string(#expr) + ": " + hipGetErrorString(e_)); \
  } while (0)
