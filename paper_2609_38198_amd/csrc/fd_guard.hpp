// The guard of a C entry point: no exception crosses the ABI, and every failure
// becomes a status with a message.
#pragma once

#include <exception>
#include <string>

#include "fd_internal.hpp"

namespace fd {

template <class F>
inline fd_status guarded(F&& f) {
  try {
    f();
    set_error("");
    return FD_OK;
  } catch (const Error& e) {
    set_error(e.msg);
    return e.status;
  } catch (const std::exception& e) {
    set_error(std::string("internal error: ") + e.what());
    return FD_ERR_HIP;
  } catch (...) {
    set_error("internal error");
    return FD_ERR_HIP;
  }
}

}  // namespace fd
