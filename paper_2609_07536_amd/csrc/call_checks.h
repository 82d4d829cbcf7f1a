// What the calls of moe_experts.h check and return on the host.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "moe_experts.h"

namespace {

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline bool type_ok(int32_t t) { return t == MOE_BF16 || t == MOE_F32; }
inline size_t type_size(int32_t t) { return t == MOE_BF16 ? 2 : 4; }
inline int done() { return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP; }

}  // namespace
