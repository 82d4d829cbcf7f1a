// A workgroup's unit (tile) of a grouped GEMM, found from the expert offsets.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "status_bits.h"

namespace {

// The rows of 64 K experts from e0 on, K neighbouring ones in each lane, by one
// round trip (with K = 1 alone, E = 1024 experts took a wave 16 of them for each
// tile: the stage of H = 1024, I = 256, 16 rows each 316 us, now 151).  Clamped as
// in load_experts; experts past E are empty.
template <int K>
struct ExpertRows {
  int start[K], count[K];
  bool bad;   // this lane's offsets are not a non-decreasing prefix of [0, rows]
  __device__ __forceinline__ ExpertRows(const int32_t* offsets, long long rows, int E, int e0) {
    const int e = e0 + K * (threadIdx.x & 63), cap = (int)rows;
    int off[K + 1];
#pragma unroll
    for (int i = 0; i <= K; ++i) off[i] = offsets[min(e + i, E)];
    bad = e == 0 && off[0] != 0;
#pragma unroll
    for (int i = 0; i < K; ++i) {
      bad |= off[i + 1] < off[i] || off[i + 1] > cap;
      start[i] = min(max(off[i], 0), cap);
      count[i] = max(min(off[i + 1], cap) - start[i], 0);   // (experts past E: off[i + 1] is off[i])
    }
  }
  template <class Units>
  __device__ __forceinline__ int sum(Units units) const {   // of this lane's experts
    int n = 0;
#pragma unroll
    for (int i = 0; i < K; ++i) n += units(count[i]);
    return n;
  }
};

// An expert's rows, its first m-unit and how many it has.
struct ExpertUnit {
  int e, start, count, first, n;
};
// The expert that holds m-unit mt of the chunk at e0, which starts at m-unit
// `carry`; v: the inclusive prefix of the lanes' sums.
template <int K, class Units>
__device__ __forceinline__ ExpertUnit find_expert(const ExpertRows<K>& r, int e0, int mt, Units units,
                                                  int carry, int v) {
  // the first lane whose prefix passes mt, and its expert that does
  const int l = (int)__builtin_ctzll(__ballot(carry + v > mt));
  int k = 0, first = carry + v - r.sum(units), start = r.start[0], count = r.count[0], n = units(count);
#pragma unroll
  for (int i = 1; i < K; ++i)
    if (mt >= first + n) {
      first += n;
      k = i, start = r.start[i], count = r.count[i], n = units(count);
    }
  return {e0 + K * l + __builtin_amdgcn_readlane(k, l), __builtin_amdgcn_readlane(start, l),
          __builtin_amdgcn_readlane(count, l), __builtin_amdgcn_readlane(first, l),
          __builtin_amdgcn_readlane(n, l)};
}

// Inclusive, over the lanes: within rows of 16 by shifts, then each row's sum to the
// next one's and the first half's to the second's (data-parallel primitives: each
// step is one addition, where a shuffle through LDS takes 100 cycles).
template <int kCtrl, int kRows>
__device__ __forceinline__ int prefix_step(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, kCtrl, kRows, 0xf, false);
}
__device__ __forceinline__ int wave_prefix(int v) {
  v = prefix_step<0x111, 0xf>(v);   // row_shr 1, 2, 4, 8
  v = prefix_step<0x112, 0xf>(v);
  v = prefix_step<0x114, 0xf>(v);
  v = prefix_step<0x118, 0xf>(v);
  v = prefix_step<0x142, 0xa>(v);   // row_bcast 15 into rows 1 and 3
  return prefix_step<0x143, 0xc>(v);   // row_bcast 31 into rows 2 and 3
}

struct SmallUnit {
  int e, r0, rows_valid, n0;
  bool ok;
};

// This workgroup's unit (expert -> n-tile -> m-tile; consecutive units of an
// XCD are neighbours), by each wave for itself.
template <int BM, int BN, int K>
__device__ __forceinline__ SmallUnit small_unit_of(const int32_t* offsets, long long rows, int E, int NT,
                                                   uint32_t* status, int* rows_dev) {
  constexpr int kChunk = 64 * K;
  auto tiles = [](int count) { return (count + BM - 1) / BM; };
  ExpertRows<K> r(offsets, rows, E, 0);
  bool bad = r.bad;
  int mine = r.sum(tiles), e0 = 0;
  for (int e = kChunk; e < E; e += kChunk) {   // (the last chunk stays in r)
    r = ExpertRows<K>(offsets, rows, E, e0 = e);
    bad |= r.bad;
    mine += r.sum(tiles);
  }
  // the last row: the end of the last lane's last expert, empty or not
  *rows_dev = __builtin_amdgcn_readlane(r.start[K - 1] + r.count[K - 1], 63);
  if (bad && blockIdx.x == 0 && status)   // (the caller may have none)
    __hip_atomic_fetch_or(status, kStBadRouting, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  int v = wave_prefix(mine);
  SmallUnit u = {0, 0, 0, 0, false};
  const int b = blockIdx.x;
  const long long units = (long long)__builtin_amdgcn_readlane(v, 63) * NT;
  const long long chunk = (units + 7) >> 3;
  const long long unit = (long long)(b & 7) * chunk + (b >> 3);
  u.ok = (b >> 3) < chunk && unit < units;
  if (!u.ok) return u;
  const int mt = (int)(unit / NT);
  int carry = 0;
  if (E > kChunk) {
    for (e0 = 0;; e0 += kChunk) {
      r = ExpertRows<K>(offsets, rows, E, e0);
      v = wave_prefix(r.sum(tiles));
      const int sum = __builtin_amdgcn_readlane(v, 63);
      if (mt < carry + sum) break;
      carry += sum;
      u.ok = e0 + kChunk < E;   // (always: mt is below their sum)
      if (!u.ok) return u;
    }
  }
  const ExpertUnit x = find_expert(r, e0, mt, tiles, carry, v);
  const int within = (int)(unit - (long long)x.first * NT);
  const int nt = within / x.n;
  const int mi = within - nt * x.n;
  u.e = x.e;
  u.n0 = nt * BN;
  u.r0 = x.start + mi * BM;
  u.rows_valid = min(BM, x.count - mi * BM);
  return u;
}
template <int BM, int BN>
__device__ __forceinline__ SmallUnit small_unit(const int32_t* offsets, long long rows, int E, int NT,
                                                uint32_t* status, int* rows_dev) {
  return E <= 64    ? small_unit_of<BM, BN, 1>(offsets, rows, E, NT, status, rows_dev)
         : E <= 128 ? small_unit_of<BM, BN, 2>(offsets, rows, E, NT, status, rows_dev)
                    : small_unit_of<BM, BN, 4>(offsets, rows, E, NT, status, rows_dev);
}

}  // namespace
