// Checks of arguments that the entry points share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool head_dim_ok(int d) { return d == 64 || d == 128 || d == 256; }

// A sticky error left on this thread by earlier, unrelated HIP work would otherwise be reported by the
// first hipGetLastError() after our own launch and be mistaken for ours.
void forget_stale_hip_error() { (void)hipGetLastError(); }

}  // namespace
