// The thread-local error message of the C ABI (fcg_last_error), shared by the
// library's host translation units.
#pragma once

#include <exception>
#include <string>

#include "fcg.h"

namespace fcg {
// Record msg as the calling thread's last error and return s.
fcg_status report(fcg_status s, const std::string& msg);

// Body of an entry point that allocates: a host allocation that fails becomes a
// status (whose message is short enough to need none itself).
template <typename F>
fcg_status guarded(F&& f) {
  try {
    return f();
  } catch (const std::exception&) {
    return report(FCG_ENOMEM, "host allocation");
  }
}
}  // namespace fcg
