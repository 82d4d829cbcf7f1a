// Bits of a workspace's status word (its first), which moe_gemm2_status reads.
#pragma once

#include <cstdint>

constexpr uint32_t kStBadRouting = 1u;
constexpr uint32_t kStTimeout = 2u;
