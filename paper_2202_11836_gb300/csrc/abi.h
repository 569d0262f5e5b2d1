// What every C entry point is wrapped in: no C++ exception crosses the ABI.
#pragma once
#include <exception>
#include <new>

#define ABI_GUARD_BEGIN try {
#define ABI_GUARD_END                                              \
  }                                                                \
  catch (const std::bad_alloc&) {                                  \
    set_error("host allocation failed");                           \
    return SKY_ERR_OOM;                                            \
  }                                                                \
  catch (const std::exception& ex) {                               \
    set_error("internal error: %s", ex.what());                    \
    return SKY_ERR_CUDA;                                           \
  }                                                                \
  catch (...) {                                                    \
    set_error("internal error");                                   \
    return SKY_ERR_CUDA;                                           \
  }
