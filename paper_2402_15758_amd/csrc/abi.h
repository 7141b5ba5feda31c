// What the C ABI's entry points share: the status they return, the calling
// thread's last message, and the checks that raise them.
#pragma once
#include <hip/hip_runtime.h>

#include <exception>
#include <stdexcept>
#include <string>

#include "chimera.h"

// The library's own: a program or another library may have a g_err too.
extern thread_local __attribute__((visibility("hidden"))) std::string g_err;

namespace {

struct Err : std::runtime_error {
  chimera_status st;
  Err(chimera_status s, const std::string& m) : std::runtime_error(m), st(s) {}
};

#define HIPCK(x)                                                                          \
  do {                                                                                    \
    hipError_t e_ = (x);                                                                  \
    if (e_ != hipSuccess) throw Err(CHIMERA_EHIP, std::string(#x) + ": " + hipGetErrorString(e_)); \
  } while (0)
#define REQUIRE(c, st, msg) \
  do {                      \
    if (!(c)) throw Err(st, msg); \
  } while (0)

template <class F>
chimera_status guard(F&& f) {
  try {
    f();
    return CHIMERA_OK;
  } catch (const Err& e) {
    g_err = e.what();
    return e.st;
  } catch (const std::exception& e) {
    g_err = e.what();
    return CHIMERA_EINVAL;
  } catch (...) {
    g_err = "unknown error";
    return CHIMERA_EINVAL;
  }
}

size_t esize(int dt) { return dt == CHIMERA_BF16 ? 2 : 4; }

// Row capacity of a tiled GEMM-input buffer that may hold up to m rows: a
// launch with m rows reads 16-row tiles in groups of 1, 2 or 4.
// Rows of an activation buffer: whole tiles of the GEMM row blocks that
// read it (16, 32, 64, then 128-row blocks).
int mcap(int m) { return m <= 16 ? 16 : (m <= 32 ? 32 : (m <= 64 ? 64 : (m + 127) / 128 * 128)); }

}  // namespace
