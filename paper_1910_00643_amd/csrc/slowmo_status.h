// What every C entry point outside slowmo_api.cpp shares: the thread's error message and a
// wall that no exception passes.
#pragma once
#include <hip/hip_runtime.h>

#include <exception>
#include <new>
#include <string>

#include "../../include/slowmo.h"

namespace slowmo {

// Sets the message that slowmo_last_error(NULL) returns and hands `st` back.
slowmo_status fail_thread(slowmo_status st, const char *msg) noexcept;
slowmo_status fail_thread_hip(hipError_t e, const char *what) noexcept;

template <typename F>
slowmo_status walled(F &&body) noexcept {
  try {
    return body();
  } catch (const std::bad_alloc &) {
    return fail_thread(SLOWMO_ERR_NOMEM, "host allocation failed");
  } catch (const std::exception &e) {
    return fail_thread(SLOWMO_ERR_ARG, e.what());
  } catch (...) {
    return fail_thread(SLOWMO_ERR_ARG, "unexpected exception");
  }
}

}  // namespace slowmo
