// The dynamic-LDS limits that kernels have been given: plain bookkeeping for allow_dynamic_lds
// and for host code.
#pragma once

#include <map>
#include <utility>

namespace aqlm {

// A limit is a property of a kernel on a device, and setting it replaces what was set before: calls that need less
// must not lower it for those that needed more.
struct LdsLimits {
  std::map<std::pair<const void*, int>, int> most;

  // Calls set() (0: done) where the kernel has not been given this much on the device yet.
  template <typename F>
  auto allow(const void* kern, int dev, int bytes, F set) -> decltype(set()) {
    int& held = most[{kern, dev}];
    if (bytes <= held) return decltype(set())(0);
    const auto e = set();
    if (e == decltype(set())(0)) held = bytes;
    return e;
  }
};

}  // namespace aqlm
