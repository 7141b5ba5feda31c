// Checks that the C ABI's operators share.
#pragma once
#include "abi.h"

namespace {

int64_t round256(int64_t b) { return (b + 255) / 256 * 256; }

void check_dtype(int32_t dtype) {
  REQUIRE(dtype == CHIMERA_F32 || dtype == CHIMERA_BF16, CHIMERA_EINVAL, "dtype");
}
void check_aligned(const void* p, const char* what) {
  REQUIRE(((uintptr_t)p & 15) == 0, CHIMERA_EINVAL, std::string(what) + " must be 16-byte aligned");
}
// The caller's stream must belong to the current device: the kernels are
// launched there.
hipStream_t check_stream(void* stream) {
  hipStream_t st = (hipStream_t)stream;
  if (st != nullptr) {
    hipDevice_t on = 0;
    int dev = 0;
    HIPCK(hipStreamGetDevice(st, &on));
    HIPCK(hipGetDevice(&dev));
    REQUIRE((int)on == dev, CHIMERA_EINVAL, "the stream belongs to another device than the current one");
  }
  return st;
}

}  // namespace
