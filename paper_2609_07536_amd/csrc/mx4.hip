// Microscaled 4-bit floating point on gfx950: quantisation of activations and
// weights, and the experts' products (C ABI and format: moe_experts.h).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstddef>
#include <cstdint>
#include <type_traits>
#include <utility>

#include "call_checks.h"
#include "expert_units.h"
#include "lds_loads.h"
#include "moe_experts.h"
#include "status_bits.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 32;         // elements that share a scale
constexpr int kBlockBytes = 16;    // their codes
constexpr int kMaxExperts = 1024;

__host__ __device__ inline int blocks_of(int K) { return (K + kBlock - 1) / kBlock; }
__host__ __device__ inline int scale_pitch(int K) { return (blocks_of(K) + 3) / 4 * 4; }

// ---- quantisation -------------------------------------------------------------
//
// A block's scale byte comes from the bits of its largest magnitude alone: the
// exponent field less 2 (not below 0), 255 where that is an infinity or NaN.
// The conversion instruction divides by the scale, rounds to the nearest code
// (ties to even) and saturates, two values at a time.

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  const int e = (int)(top >> 23);
  return e == 255 ? 255u : (uint32_t)max(e - 2, 0);
}
// 2^(byte - 127) (byte 0: a subnormal)
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __uint_as_float(byte == 0 ? 0x00400000u : byte << 23);
}
// eight codes, the first in the lowest bits
__device__ __forceinline__ uint32_t codes8(const float (&v)[8], uint32_t byte) {
  const float s = scale_of(byte);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
  return byte == 255 ? 0 : c;
}

// V elements, aligned to one
template <class T, int V>
struct Mem {
  typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
// p[0..8), zeros from n on
template <class T>
__device__ __forceinline__ void load8(const T* p, int n, float (&v)[8]) {
  if (n >= 8) {
    const auto x = *(const typename Mem<T, 8>::type*)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? (float)p[i] : 0.f;
  }
}
// V values to p[0..min(n, V))
template <int V, class T>
__device__ __forceinline__ void store_few(T* p, int n, const float (&v)[8]) {
  if (n >= V) {
    T __attribute__((ext_vector_type(V))) x;
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (T)v[i];
    *(typename Mem<T, V>::type*)p = x;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) p[i] = (T)v[i];
  }
}

template <int kCtrl>
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, kCtrl, 0xf, 0xf, true));
}

// Eight elements a thread, four neighbouring threads a block: every thread's
// load and store is one of the wave's contiguous ones.  Bound by memory: 16384 x
// 2048 bf16 (85 MB with the codes) 19.1 us, 4.5 TB/s; 16 rows 2.5 us, latency.
template <class T>
__global__ void __launch_bounds__(256) mx4_quantize_kernel(const T* x, uint8_t* codes, uint8_t* scales,
                                                           long long rows, int K) {
  const int per_row = blocks_of(K) * 4;   // threads of a row
  const long long base = (long long)blockIdx.x * 256;
  const long long row0 = base / per_row;
  const uint32_t i = (uint32_t)(base - row0 * per_row) + threadIdx.x;
  const uint32_t down = i / (uint32_t)per_row;
  const long long row = row0 + down;
  const int c = (int)(i - down * (uint32_t)per_row);
  const bool in = row < rows;
  float v[8] = {};
  if (in) load8(x + row * K + 8 * c, K - 8 * c, v);
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, magnitude(v[j]));
  top = quad_max<0xb1>(top);   // lanes 1 0 3 2
  top = quad_max<0x4e>(top);   // lanes 2 3 0 1
  if (!in) return;
  const uint32_t byte = scale_byte(top);
  *(uint32_t*)(codes + row * (per_row * 4ll) + 4 * c) = codes8(v, byte);
  if ((c & 3) == 0) {
    const int kb = c >> 2, KS = scale_pitch(K), KB = per_row >> 2;
    uint8_t* s = scales + row * KS + kb;
    *s = (uint8_t)byte;
    if (kb == KB - 1)
      for (int j = 1; kb + j < KS; ++j) s[j] = 0;
  }
}

// w [E, K, N] to codes and scales of [E, N, K].  A workgroup takes 128 columns
// and 256 of K: a thread's two columns over the 32 of K of a block, so a block's
// largest magnitude needs no other lane; the codes leave through LDS as 128
// contiguous bytes per column.  30 experts of 704 x 2048 in bf16 (110 MB with the
// codes) 31.5 us with 32 loads of a thread in flight (51.9 with a test before each
// load): 3.5 TB/s, where a copy reaches 4.9.  What takes the rest is not known.
constexpr int kWCols = 128, kWBlocks = 8;
template <class T>
__global__ void __launch_bounds__(256) mx4_quantize_weights_kernel(const T* w, uint8_t* codes, uint8_t* scales,
                                                                   int K, int N, int k_tiles, int n_tiles) {
  __shared__ __align__(16) uint8_t c[kWCols * kWBlocks * kBlockBytes];
  __shared__ __align__(8) uint8_t s[kWCols * kWBlocks];
  const int KB = blocks_of(K), KS = scale_pitch(K);
  const uint32_t unit = blockIdx.x;
  const int kt = unit % (uint32_t)k_tiles, nt = unit / (uint32_t)k_tiles % (uint32_t)n_tiles;
  const long long e = unit / (uint32_t)k_tiles / (uint32_t)n_tiles;
  const int n0 = nt * kWCols, b0 = kt * kWBlocks;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = n0 + 2 * lane;
  const T* src = w + e * K * N + n;
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const int b = wave + 4 * p, k0 = (b0 + b) * kBlock;
    float v[2][kBlock];
    if (k0 + kBlock <= K && n0 + kWCols <= N) {   // a whole block of whole columns: no load waits for a test
#pragma unroll
      for (int k = 0; k < kBlock; ++k) {
        const auto x = *(const typename Mem<T, 2>::type*)(src + (long long)(k0 + k) * N);
        v[0][k] = (float)x[0];
        v[1][k] = (float)x[1];
      }
    } else
#pragma unroll
    for (int k = 0; k < kBlock; ++k) {
      v[0][k] = v[1][k] = 0.f;
      if (k0 + k < K && n < N) {
        const T* q = src + (long long)(k0 + k) * N;
        if (n + 1 < N) {
          const auto x = *(const typename Mem<T, 2>::type*)q;
          v[0][k] = (float)x[0];
          v[1][k] = (float)x[1];
        } else {
          v[0][k] = (float)q[0];
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < kBlock; ++k) top = max(top, magnitude(v[j][k]));
      const uint32_t byte = k0 < K ? scale_byte(top) : 0;
      u32x4 q;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = v[j][8 * i + k];
        q[i] = codes8(o, byte);
      }
      const int r = 2 * lane + j;
      // (chunk swizzled by the column pair: the lanes' columns are 256 bytes apart)
      *(u32x4*)(c + r * (kWBlocks * kBlockBytes) + ((b ^ (lane & 7)) * kBlockBytes)) = q;
      s[r * kWBlocks + b] = (uint8_t)byte;
    }
  }
  __syncthreads();
#pragma unroll
  for (int p = 0; p < kWCols * kWBlocks / 256; ++p) {
    const int i = p * 256 + (int)threadIdx.x, r = i / kWBlocks, b = i % kWBlocks;
    if (n0 + r < N && b0 + b < KB)
      *(u32x4*)(codes + ((e * N + n0 + r) * KB + b0 + b) * (long long)kBlockBytes) =
          *(const u32x4*)(c + r * (kWBlocks * kBlockBytes) + ((b ^ ((r >> 1) & 7)) * kBlockBytes));
  }
  const int r = (int)threadIdx.x >> 1, b = ((int)threadIdx.x & 1) * 4;   // four scales a thread
  if (n0 + r < N && b0 + b < KS)
    *(uint32_t*)(scales + (e * N + n0 + r) * KS + b0 + b) = *(const uint32_t*)(s + r * kWBlocks + b);
}

// Bound by memory: 30 x 2048 x 704 to bf16 18.5 us, just after the codes were written
// (they come from the caches).
template <class T>
__global__ void __launch_bounds__(256) mx4_dequantize_kernel(const uint8_t* codes, const uint8_t* scales, T* out,
                                                             long long rows, int K) {
  const int per_row = (K + 7) / 8;   // threads of a row, eight elements each
  const long long base = (long long)blockIdx.x * 256;
  const long long row0 = base / per_row;
  const uint32_t i = (uint32_t)(base - row0 * per_row) + threadIdx.x;
  const uint32_t down = i / (uint32_t)per_row;
  const long long row = row0 + down;
  const int c = (int)(i - down * (uint32_t)per_row);
  if (row >= rows) return;
  const uint32_t q = *(const uint32_t*)(codes + row * (blocks_of(K) * (long long)kBlockBytes) + 4 * c);
  const uint32_t byte = scales[row * scale_pitch(K) + (c >> 2)];
  const float s = scale_of(byte);
  const f32x2 a[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 1),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, s, 3)};
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = byte == 255 ? __builtin_nanf("") : a[j >> 1][j & 1];
  store_few<8>(out + row * K + 8 * c, K - 8 * c, v);
}

// ---- the experts' products -------------------------------------------------------
//
// A workgroup takes a tile of BM rows of one expert by BN of its weights' rows.
// Both operands are rows of codes along K, so a stage of 128 of K is 64 bytes of
// each, loaded straight into an LDS ring; a lane's operand of the 16x16x128
// scaled matrix instruction is one block: 16 bytes of codes and one scale byte
// (with operands of random codes this form reaches 7.2 PFLOP/s, 32x32x64 6.4).
// The weights are the instruction's first operand, so a lane ends up with
// columns of one row of the output.  The instruction multiplies the codes exactly
// and sums in fp32; out is rounded to bf16 once, since the next product or the
// combine takes bf16.
//
// What bounds large calls: 98304 rows (32 experts, K 2048, N 1408 with SwiGLU, 567
// GFLOP) 208 us, 2.7 PFLOP/s, 38% of what the instruction reaches.  The loop over K is
// two thirds of that (16 stages of 256 x 256 some 26 000 clocks, the matrix instructions
// alone 16 400), the rest a finished tile's stores and the next one's start.  The
// down-projection (K 704, N 2048, 283 GFLOP, 464 MB) takes 212 us, 2.2 times its bytes
// at a copy's rate: a tile has only six stages for its 128 KB of output, and the
// non-temporal figures below point to the way out.  That the start waits for the
// stores (loads and stores are counted in order) is not what costs: stores left under way
// during the next tile's first two stages, with exact counts, gave the same outputs at
// 196 -> 198 us up, 217 -> 213 down (311 -> 307 with the combine).
//
// The stores are ordinary ones.  Non-temporal ones are faster alone (16384 tokens,
// up 200 -> 189 us, down 226 -> 165) and slower with who reads them next (up and
// quantisation 227 -> 233, down and combine 321 -> 343; 4096 tokens down and combine
// 88 -> 105), which then finds less in the caches.

struct MxArgs {
  const uint8_t* a;          // [a_rows, KB, 16]
  const uint8_t* as;         // [a_rows, KS]
  const uint8_t* w;          // [E, N, KB, 16]
  const uint8_t* ws;         // [E, N, KS]
  const int32_t* offsets;    // [E + 1]
  const int32_t* row_ids;    // [rows] or null: row r is a's row r
  __bf16* out;               // [rows, NO]
  uint8_t *oc, *os;          // or that in 4 bits: [rows, OB, 16], [rows, OS]
  uint32_t* status;          // or null
  long long rows;
  int a_rows, K, N, E, KB, KS;
  int NO;                    // columns of out: N, or N / 2 with SwiGLU
  int OB, OS;                // their blocks and scales
  int NT;                    // tiles along them
  int most;                  // tiles that the host counted on (launch_product)
};

// z / (1 + exp(-z)) by the reciprocal instruction (1 ulp): a full division is ten
// instructions of each output.
__device__ __forceinline__ float silu(float z) { return z * __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

// BM rows by BN weight rows, WM x WN waves, a ring of four stages with D of them
// ahead, R workgroups per CU.  Scales come 16 bytes of a row (four stages' worth, a
// quad) at a time, with the first stage that they are for.
template <int BM_, int BN_, int WM_, int WN_, int D_, int R_>
struct MxTile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, D = D_, R = R_;
  static constexpr int S = 4;
  static constexpr int NW = WM * WN, kThr = NW * 64;
  static constexpr int MB = BM / WM / 16, NB = BN / WN / 16;   // a wave's 16 x 16 blocks
  static constexpr int LA = MB > 4 ? 3 : MB / 2;               // blocks of a that are read ahead
  static constexpr int kRows = BM + BN;
  static constexpr int kStage = kRows * 64;                    // bytes: 4 blocks of each row
  static constexpr int LPS = kStage / 1024 / NW;               // 1 KB loads per wave and stage
  static constexpr int kQuad = kRows * 16;                     // bytes of scales of four stages
  static constexpr int QL = kRows / 64;                        // 1 KB loads of a quad
  static constexpr int SL = (QL + NW - 1) / NW;                // ... per wave (the last ones twice)
  static constexpr int kScales = S * kStage;                   // two quads
  static constexpr int kIds = kScales + 2 * kQuad;             // the next tile's rows of a
  static constexpr int kLds = kIds + BM * 4;
  // loads of a wave that stage j adds (j % 4 matters)
  static constexpr int loads(int j) { return LPS + (j % 4 == 0 ? SL : 0); }
  // loads after stage j + 1's while stage j is multiplied
  static constexpr int newer(int j) { return (D > 2 ? loads(j + 2) : 0) + (D > 3 ? loads(j + 3) : 0); }
  static_assert(D >= 2 && D <= S, "ring");
  static_assert(BM % (16 * NW) == 0 && BN % (16 * NW) == 0 && BM % 64 == 0 && BN % 64 == 0, "loads per wave");
  static_assert(BM <= 256, "one load of row ids");
  static_assert(MB % 2 == 0 && NB % 2 == 0, "blocks");
  static_assert(S * LPS + SL <= 63, "vmcnt range");
  static_assert(R * (kLds + 4 * (kMaxExperts + 2)) <= 160 * 1024, "LDS");
};

// Position of 16-byte chunk c (0..3) of a row within the row's 64 bytes, by two bits q
// of the row.  A 16-byte read is served to 16 lanes at a time, lanes 0-3, 12-15, 20-23
// and 24-27 first; with lane = i + 16 c and q = i / 4 these fall on distinct banks
// (measured: 4.7 cycles an instruction, as for a linear read; 8.4 with c ^ q).
__device__ __forceinline__ int swz(int q, int c) { return c ^ (((q ^ (q << 1)) & 2) | ((q >> 1) & 1)); }

typedef const __attribute__((address_space(3))) uint8_t lds_u8;
typedef const __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef const __attribute__((address_space(3))) uint32_t lds_u32;

// f(0) .. f(N - 1), the index as a constant
template <int N, class F, int... I>
__device__ __forceinline__ void static_for_each(F& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>()), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F f) {
  static_for_each<N>(f, std::make_integer_sequence<int, N>());
}

// (Whole numbers only: copies of a bool and its padding end up in memory.)
struct Tile {
  int e, r0, rows_valid, n0, ok;
};
template <int BM>
__device__ __forceinline__ int tiles_of(int r0, int r1) { return (max(r1 - r0, 0) + BM - 1) / BM; }
// Tile `unit` (expert -> kGroup tiles of columns -> rows -> columns), by each wave for
// itself; row(i), i <= E: expert i's first row (row(E): the end of the last one).
// Four tiles of columns at a time: their weights stay in the L2 while the rows come by
// (16384 tokens, against all columns of a row first: up 195 -> 191 us, down 225 -> 222).
constexpr int kGroup = 4;
template <int BM, int BNO, class Row>
__device__ __forceinline__ Tile unit_at(const MxArgs& a, int unit, Row row) {
  const int lane = threadIdx.x & 63;
  int before = 0;   // tiles of the experts up to e0
  for (int e0 = 0;; e0 += 64) {
    const int r0 = row(min(e0 + lane, a.E)), r1 = row(min(e0 + lane + 1, a.E));
    const int t = tiles_of<BM>(r0, r1), end = before + wave_prefix(t);
    const uint64_t past = __ballot((long long)end * a.NT > unit);
    if (past == 0) {
      if (e0 + 64 >= a.E) return {0, 0, 0, 0, 0};
      before = __builtin_amdgcn_readlane(end, 63);
      continue;
    }
    const int i = (int)__builtin_ctzll(past);
    const int n = __builtin_amdgcn_readlane(t, i), within = unit - (__builtin_amdgcn_readlane(end, i) - n) * a.NT;
    const int group = within / (n * kGroup), left = within - group * (n * kGroup);
    const int wide = min(kGroup, a.NT - group * kGroup), mi = left / wide, nt = group * kGroup + left - mi * wide;
    const int start = __builtin_amdgcn_readlane(r0, i) + mi * BM;
    return {e0 + i, start, min(BM, __builtin_amdgcn_readlane(r1, i) - start), nt * BNO, 1};
  }
}
// All tiles.  Offsets are clamped as in ExpertRows; bad ones are flagged, and where they
// make ranges overlap no more tiles run than there are without.
template <int BM>
__device__ __forceinline__ int all_tiles(const MxArgs& a) {
  const int lane = threadIdx.x & 63, cap = (int)a.rows;
  long long tiles = 0;   // of rows
  bool bad = false;
  for (int e0 = 0; e0 < a.E; e0 += 64) {
    const int e = e0 + lane, o0 = a.offsets[min(e, a.E)], o1 = a.offsets[min(e + 1, a.E)];
    bad |= (e == 0 && o0 != 0) || o1 < o0 || o1 > cap;
    tiles += __builtin_amdgcn_readlane(wave_prefix(tiles_of<BM>(min(max(o0, 0), cap), min(max(o1, 0), cap))), 63);
  }
  if (bad && a.status && blockIdx.x == 0)
    __hip_atomic_fetch_or(a.status, kStBadRouting, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return (int)min(tiles * a.NT, (long long)a.most);
}

// kCodes (with SwiGLU): the output, rounded to bf16 as it would be stored, leaves in 4
// bits, as mx4_quantize_kernel makes them: four lanes hold a block's 32 columns.  The
// layer, replayed from a graph, against a launch that reads the bf16 and quantises it
// (32 experts of 2048 x 704, top 6): 1024 tokens 56.5 -> 53.5 us, 4096 156.8 -> 144.3, 16384
// 547.9 -> 539.7; over four shapes 1.5 to 8% less.  Thin kernels hold 16 columns a wave,
// half a block, and leave it to that launch.
template <class C, bool kSwiglu, bool kCodes>
__global__ void __launch_bounds__(C::kThr, C::R * C::NW / 4) mx4_product_kernel(MxArgs a) {
#define MX_INLINE __attribute__((always_inline))
  __shared__ __align__(1024) uint8_t smem[C::kLds];
  __shared__ int expert_row[kMaxExperts + 1];   // each expert's first row, for the tiles after the first
  constexpr int BNO = kSwiglu ? C::BN / 2 : C::BN;   // output columns of a tile
  static_assert(!kSwiglu || C::NB % 4 == 0, "a wave has pairs of gate and of up blocks");
  static_assert(!kCodes || (kSwiglu && BNO % kBlock == 0), "whole blocks");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // this workgroup's tiles: every step-th of an XCD's contiguous share
  const int units = all_tiles<C::BM>(a), share = (units + 7) >> 3;
  const int step = gridDim.x >> 3;
  int unit = (blockIdx.x & 7) * share + (blockIdx.x >> 3);
  const int last = min(((int)(blockIdx.x & 7) + 1) * share, units);
  if (unit >= last) return;
  auto row_at = [&](int e) MX_INLINE { return min(max(a.offsets[e], 0), (int)a.rows); };
  Tile u = unit_at<C::BM, BNO>(a, unit, row_at);
  for (int e = threadIdx.x; e <= a.E; e += C::kThr) expert_row[e] = row_at(e);

  const uint32_t lds = lds_addr(smem);
  lds_u8* base = (lds_u8*)(uintptr_t)lds;
  const uint32_t pitch = (uint32_t)a.KB * kBlockBytes;
  const int KT = (a.KB + 3) / 4;
  const i32x4 ra = buffer_rsrc(a.a, (long long)a.a_rows * pitch), ras = buffer_rsrc(a.as, (long long)a.a_rows * a.KS);
  i32x4 rw, rws;

  // a tile's row ids, four a lane (by a resource of the tile's own: an offset from the
  // first row's would pass 32 bits)
  auto issue_ids = [&](const Tile& t) MX_INLINE {
    if (a.row_ids && wave == 0 && 4 * lane < C::BM)
      dma16(buffer_rsrc(a.row_ids + t.r0, 4ll * t.rows_valid), 16u * (uint32_t)lane, lds + C::kIds);
  };
  // tile row i (BM rows of a, then BN of w) to its row in memory, or -1
  auto row_of = [&](const Tile& t, int i) MX_INLINE -> int {
    if (i < C::BM) {
      if (i >= t.rows_valid) return -1;
      const int id = a.row_ids ? *(const __attribute__((address_space(3))) int*)(base + C::kIds + 4 * i) : t.r0 + i;
      if (id >= 0 && id < a.a_rows) return id;
      if (a.status && a.row_ids) __hip_atomic_fetch_or(a.status, kStBadRouting, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      return -1;
    }
    const int j = i - C::BM;
    if (!kSwiglu) return t.n0 + j < a.N ? t.n0 + j : -1;
    const int n = t.n0 + (j < BNO ? j : j - BNO);
    return n < a.NO ? (j < BNO ? n : a.NO + n) : -1;
  };
  // This lane's part of its wave's loads: load q is 16 rows of a stage, a's for the
  // first ones; a load of scales is 64 rows of a quad.  Rows of a are swizzled by bits
  // 2 and 3, rows of w by bits 3 and 4 (lw below).
  constexpr int kLoadsA = C::BM / 16 / C::NW;
  auto load_row = [&](int q, int ln) MX_INLINE { return (q * C::NW + wave) * 16 + (ln >> 2); };
  auto load_chunk = [&](int q, int ln) MX_INLINE {
    const int i = load_row(q, ln);
    return swz((q < kLoadsA ? i >> 2 : i >> 3) & 3, ln & 3);
  };
  // (what is computed from this copy stays where it is used: hoisted out of the
  // loops it would take the registers that the loop over K needs)
  auto lane_here = [&]() MX_INLINE {
    int v = lane;
    asm volatile("" : "+v"(v));
    return v;
  };
  auto scale_load = [&](int q) MX_INLINE { return (q * C::NW + wave) % C::QL; };
  uint32_t off[C::LPS], soff[C::SL];
  auto set_tile = [&](const Tile& t) MX_INLINE {
    rw = buffer_rsrc(a.w + t.e * ((long long)a.N * pitch), (long long)a.N * pitch);
    rws = buffer_rsrc(a.ws + (long long)t.e * a.N * a.KS, (long long)a.N * a.KS);
    const int ln = lane_here();
#pragma unroll
    for (int q = 0; q < C::LPS; ++q) {
      const int r = row_of(t, load_row(q, ln));
      off[q] = r < 0 ? kOutOfRange : (uint32_t)r * pitch + load_chunk(q, ln) * kBlockBytes;
    }
#pragma unroll
    for (int q = 0; q < C::SL; ++q) {
      const int r = row_of(t, scale_load(q) * 64 + ln);
      soff[q] = r < 0 ? kOutOfRange : (uint32_t)r * (uint32_t)a.KS;
    }
  };
  // load q of stage kt, to its slot of the ring; what lies past the end is set out
  // of range beforehand (cut_k) and loads zeros
  const uint32_t ldsw = lds + (uint32_t)wave * 1024;
  auto issue = [&](auto q, auto slot, uint32_t k) MX_INLINE {   // k: 64 bytes a stage, 0 past the end
    constexpr int Q = decltype(q)::value;
    dma16_at<decltype(slot)::value * C::kStage + Q * C::NW * 1024>(Q < kLoadsA ? ra : rw, off[Q], ldsw, k);
  };
  auto cut_k = [&](int kt) MX_INLINE {
    const int ln = lane_here();
#pragma unroll
    for (int q = 0; q < C::LPS; ++q)
      if (4 * kt + load_chunk(q, ln) >= a.KB) off[q] = kOutOfRange;
  };
  auto issue_scales = [&](int q, int kt) MX_INLINE {   // of the quad from stage kt on
    const int i = scale_load(q);
    const bool in = kt < KT;
    dma16(64 * i < C::BM ? ras : rws, in ? soff[q] : kOutOfRange,
          lds + (uint32_t)(C::kScales + ((kt >> 2) & 1) * C::kQuad + i * 1024), in ? 4u * (uint32_t)kt : 0);
  };

  const int wm0 = (wave / C::WN) * C::MB * 16, wn = wave % C::WN;
  // first tile row of pair p of this wave's blocks of w: with SwiGLU half are gate, half up
  auto w_row = [&](int p) MX_INLINE {
    return C::BM + (kSwiglu ? (p < C::NB / 4 ? (wn * (C::NB / 4) + p) * 32 : BNO + (wn * (C::NB / 4) + p - C::NB / 4) * 32)
                            : (wn * (C::NB / 2) + p) * 32);
  };
  const int l = lane & 15, g = lane >> 4;   // the instruction's row, and block of its 128 of K
  // the row of its pair that a lane brings for block f of the two, so that its
  // accumulators of both are columns 8 g .. 8 g + 7 of one output row
  const int lw = 8 * (l >> 2) + (l & 3);
  // where a lane's codes and scales are: a's and w's, plus constants (two bases for
  // codes, an offset in an instruction ends at 64 KB)
  const int wave_w = wn * (kSwiglu ? C::NB / 4 : C::NB / 2) * 32 + lw;   // (4 f rows leave bits 3, 4 alone)
  lds_u8* const pa = base + (wm0 + l) * 64 + swz(l >> 2, g) * 16;
  lds_u8* const pw = base + wave_w * 64 + swz(l >> 2, g) * 16;
  // a lane without a block in the last stage has codes of zeros and takes the scale
  // of the stage's first block, whatever pad bytes hold
  const int back = 4 * (KT - 1) + g < a.KB ? 0 : g;
  lds_u8 *qa, *qw;

  // 16 bytes of codes and a scale: a lane's block of a 16-row operand
  struct Frag {
    u32x4 v;
    int s;
  };
  // tile row of block nb of w, less what differs between waves and lanes
  auto w_const = [](int nb) MX_INLINE {
    const int p = nb >> 1;
    return C::BM + (kSwiglu && p >= C::NB / 4 ? BNO + (p - C::NB / 4) * 32 : p * 32) + 4 * (nb & 1);
  };
  auto read_a = [&](int mb, int slot, int stage4) MX_INLINE -> Frag {   // stage4: of its quad
    const int at = slot * C::kStage + mb * 1024;
    return {*(lds_u32x4*)((at < 65536 ? pa : pa + 65536) + (at < 65536 ? at : at - 65536)), qa[stage4 * 4 + mb * 256]};
  };
  auto read_w = [&](int nb, int slot, int stage4) MX_INLINE -> Frag {
    const int r = w_const(nb), at = slot * C::kStage + r * 64;
    return {*(lds_u32x4*)((at < 65536 ? pw : pw + 65536) + (at < 65536 ? at : at - 65536)), qw[stage4 * 4 + r * 16]};
  };

  f32x4 acc[C::NB][C::MB];
  Tile done = u;   // the tile in acc
  done.ok = 0;
  issue_ids(u);
  for (;;) {
    waitcnt_vm<0>();   // u's row ids (and loads past the end of the last tile, which write to LDS as well)
    block_barrier();
    if (u.ok) set_tile(u);
    // The ring is free: u's first stages land while the last tile is stored, a load
    // or two and then the stores of 16 of its rows (each lane's: eight neighbouring
    // columns, 16 bytes, at a time).
    constexpr int kFirst = C::D * C::LPS;
    const int ln = lane_here();
    static_for<C::MB>([&](auto m) MX_INLINE {
      constexpr int mb = decltype(m)::value;
      if (u.ok) {
        if constexpr (mb == 0)
#pragma unroll
          for (int q = 0; q < C::SL; ++q) issue_scales(q, 0);
        constexpr int i0 = mb * kFirst / C::MB, i1 = (mb + 1) * kFirst / C::MB;
        static_for<i1 - i0>([&](auto i) MX_INLINE {
          constexpr int at = i0 + decltype(i)::value, kt = at / C::LPS, q = at % C::LPS;
          if (q == 0 && kt >= KT - 1) cut_k(kt);
          issue(std::integral_constant<int, q>(), std::integral_constant<int, kt>(), kt < KT ? 64u * kt : 0);
        });
      }
      const int row = wm0 + mb * 16 + (ln & 15);
      if constexpr (kCodes) {
        if (done.ok) {   // (all lanes: a block's four exchange their largest magnitudes)
#pragma unroll
          for (int p = 0; p < C::NB / 4; ++p) {
            const int b0 = done.n0 + w_row(p) - C::BM, n = b0 + 8 * (ln >> 4), block = b0 / kBlock;
            float v[8];
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float x = silu(acc[2 * p + i / 4][mb][i % 4]) * acc[C::NB / 2 + 2 * p + i / 4][mb][i % 4];
              v[i] = n + i < a.NO ? (float)(__bf16)x : 0.f;   // (past them a NaN of a's would come through)
              top = max(top, magnitude(v[i]));
            }
            top = max(top, (uint32_t)__shfl_xor((int)top, 16));
            top = max(top, (uint32_t)__shfl_xor((int)top, 32));
            const uint32_t byte = scale_byte(top);
            if (row < done.rows_valid && block < a.OB) {
              const long long r = done.r0 + row;
              *(uint32_t*)(a.oc + (r * a.OB + block) * kBlockBytes + 4 * (ln >> 4)) = codes8(v, byte);
              if (ln < 16) {
                uint8_t* s = a.os + r * a.OS + block;
                *s = (uint8_t)byte;
                if (block == a.OB - 1)
                  for (int j = 1; block + j < a.OS; ++j) s[j] = 0;
              }
            }
          }
        }
      } else if (done.ok && row < done.rows_valid) {
        __bf16* o = a.out + (long long)(done.r0 + row) * a.NO;
#pragma unroll
        for (int p = 0; p < (kSwiglu ? C::NB / 4 : C::NB / 2); ++p) {
          float v[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            v[i] = acc[2 * p + i / 4][mb][i % 4];
            if (kSwiglu) v[i] = silu(v[i]) * acc[C::NB / 2 + 2 * p + i / 4][mb][i % 4];
          }
          const int n = done.n0 + w_row(p) - C::BM + 8 * (ln >> 4);
          if (n < a.NO) store_few<8>(o + n, a.NO - n, v);
        }
      }
    });
    if (!u.ok) break;
    Tile next = u;
    unit += step;
    next.ok = unit < last;
    if (next.ok) next = unit_at<C::BM, BNO>(a, unit, [&](int e) MX_INLINE { return expert_row[e]; });
#pragma unroll
    for (int nb = 0; nb < C::NB; ++nb)
#pragma unroll
      for (int mb = 0; mb < C::MB; ++mb) acc[nb][mb] = f32x4{0.f, 0.f, 0.f, 0.f};

    waitcnt_vm<(C::D - 1) * C::LPS>();   // stage 0 and its scales
    block_barrier();
    if (next.ok) issue_ids(next);   // (this tile's have been read)
    // w's blocks of a stage stay in registers for it, a's come by one after the
    // other, read LA ahead.  Once the last is on its way the stage's slot is free:
    // the next stage goes out, and the first operands of stage kt + 1 are read, so that
    // products are left to issue after the barrier, with the reads and loads spread
    // between them.  Four stages at a time: slots, parities and places are
    // constants, so that hardly a vector instruction is left beside the products
    // (two waves share a SIMD's issue: 100 such instructions a stage cost a
    // quarter of its time).
    qa = base + C::kScales + (wm0 + l) * 16 + g - (KT == 1 ? back : 0);
    qw = base + C::kScales + wave_w * 16 + g - (KT == 1 ? back : 0);
    int other = C::kQuad;   // from this quad of scales to the next
    Frag w[2][C::NB], x[C::MB];
#pragma unroll
    for (int nb = 0; nb < C::NB; ++nb) w[0][nb] = read_w(nb, 0, 0);
#pragma unroll
    for (int mb = 0; mb < C::LA; ++mb) x[mb] = read_a(mb, 0, 0);
    auto stage = [&](auto pos, int kt) MX_INLINE {
      constexpr int J = decltype(pos)::value, kNext = (J + 1) % 4, kLate = C::MB - C::LA;
      if (kt + C::D >= KT - 1) cut_k(kt + C::D);
      const uint32_t k = kt + C::D < KT ? 64u * (uint32_t)(kt + C::D) : 0;
      static_for<C::MB>([&](auto m) MX_INLINE {
        constexpr int mb = decltype(m)::value;
        if constexpr (mb < kLate) {
          x[mb + C::LA] = read_a(mb + C::LA, J % C::S, J);
        } else {
          if constexpr (mb == kLate) {   // the blocks from here on are multiplied after the barrier
            // stage kt + 1 has landed, and this one's last reads
            waitcnt_vm<C::newer(J)>();
            block_barrier();
            if ((J + C::D) % 4 == 0)
#pragma unroll
              for (int q = 0; q < C::SL; ++q) issue_scales(q, kt + C::D);
            if (J == 3) qa += other, qw += other, other = -other;
            if (kt + 1 == KT - 1) qa -= back, qw -= back;
          }
          x[mb - kLate] = read_a(mb - kLate, kNext % C::S, kNext);
        }
        static_for<C::NB>([&](auto n) MX_INLINE {
          constexpr int nb = decltype(n)::value;
          const Frag &p = w[J & 1][nb], &q = x[mb];
          acc[nb][mb] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
              i32x8{(int)p.v[0], (int)p.v[1], (int)p.v[2], (int)p.v[3], 0, 0, 0, 0},
              i32x8{(int)q.v[0], (int)q.v[1], (int)q.v[2], (int)q.v[3], 0, 0, 0, 0}, acc[nb][mb], 4, 4, 0, p.s, 0, q.s);
          if constexpr (mb >= kLate) {   // (kSteps products: the next w, and the loads, spread over them)
            constexpr int kSteps = C::LA * C::NB, i = (mb - kLate) * C::NB + nb;
            constexpr int o0 = i * C::NB / kSteps, o1 = (i + 1) * C::NB / kSteps;
            static_for<o1 - o0>([&](auto o) MX_INLINE { w[kNext & 1][o0 + o] = read_w(o0 + o, kNext % C::S, kNext); });
            constexpr int q0 = i * C::LPS / kSteps, q1 = (i + 1) * C::LPS / kSteps;
            static_for<q1 - q0>([&](auto o) MX_INLINE {
              issue(std::integral_constant<int, q0 + decltype(o)::value>(), std::integral_constant<int, (J + C::D) % C::S>(), k);
            });
          }
        });
        __builtin_amdgcn_sched_barrier(0);   // (else the products all move behind the barrier)
      });
    };
    for (int kt = 0;;) {
      stage(std::integral_constant<int, 0>(), kt);
      if (++kt >= KT) break;
      stage(std::integral_constant<int, 1>(), kt);
      if (++kt >= KT) break;
      stage(std::integral_constant<int, 2>(), kt);
      if (++kt >= KT) break;
      stage(std::integral_constant<int, 3>(), kt);
      if (++kt >= KT) break;
    }
    done = u;
    u = next;
  }
#undef MX_INLINE
}

// ---- few rows per expert ------------------------------------------------------------
//
// Such a call reads each weight for a handful of rows: it is bound by the stream
// of the weights, and at the smallest by how soon that stream starts.  So a
// wave loads its weights straight into registers, all of 128 KC of K at once (16
// weight rows, 64 bytes of each, an instruction), while the rows of a, shared
// by the workgroup's waves, go to LDS; no ring, one barrier per segment.
// The 16x16x128 instruction then takes 16 weight rows and 16 rows of a.
// Measured: 1 token (9.2 MB of weights and scales) 5.9 us: the launch, and one after
// the other the loads of the offsets, the unit's way through memory (20 bytes of scratch
// a lane), the row ids and the weights; 64 tokens (26.6 MB) 8.7 us, 3.0 TB/s.

__device__ __forceinline__ u32x4 buffer_load16(__amdgpu_buffer_rsrc_t r, uint32_t off) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, 0));
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t load_rsrc(const void* base, long long bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, (int)(bytes > 0x7fffffffLL ? 0x7fffffffLL : bytes), 0x00020000);
}

// 16 MB rows of a; a wave's 32 weight rows (with SwiGLU 16 gate and 16 up ones);
// NW waves; KC stages of 128 of K in registers at a time
template <int MB_, int KC_, int NW_>
struct MxThin {
  static constexpr int MB = MB_, KC = KC_, NW = NW_, kThr = 64 * NW;
  static constexpr int BM = 16 * MB, BN = 32 * NW;
  static constexpr int kCodes = BM * 64 * KC;                       // LDS bytes
  static constexpr int kSegs = (KC + 15) / 16, kScales = BM * 64 * kSegs;   // (64 bytes a row and 16 stages)
  static_assert(KC * MB % NW == 0, "loads per wave");
  static_assert(KC % 4 == 0, "scales are loaded 16 bytes at a time");
};

template <class C, bool kSwiglu>
__global__ void __launch_bounds__(C::kThr) mx4_thin_kernel(MxArgs a) {
  __shared__ __align__(1024) uint8_t smem[C::kCodes + C::kScales];
  constexpr int BNO = kSwiglu ? C::BN / 2 : C::BN;
  int rows_dev;
  const SmallUnit u = small_unit<C::BM, BNO>(a.offsets, a.rows, a.E, a.NT, a.status, &rows_dev);
  if (!u.ok) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int l = lane & 15, g = lane >> 4;   // the instruction's row, and block of its 128 of K
  const uint32_t lds = lds_addr(smem), lds_s = lds + C::kCodes;
  const long long pitch = (long long)a.KB * kBlockBytes;
  const i32x4 ra = buffer_rsrc(a.a, a.a_rows * pitch), ras = buffer_rsrc(a.as, (long long)a.a_rows * a.KS);
  const auto rw = load_rsrc(a.w + u.e * (a.N * pitch), a.N * pitch);
  const auto rws = load_rsrc(a.ws + (long long)u.e * a.N * a.KS, (long long)a.N * a.KS);
  const int KT = (a.KB + 3) / 4;

  // a's rows for this lane's LDS loads (16 rows, 64 bytes of each, a load)
  uint32_t off[C::MB], soff[C::MB];
  const int ca = swz(lane >> 4, lane & 3);
#pragma unroll
  for (int mb = 0; mb < C::MB; ++mb) {
    const int i = 16 * mb + (lane >> 2);
    int r = -1;
    if (i < u.rows_valid) {
      r = u.r0 + i;
      if (a.row_ids) {
        r = a.row_ids[r];
        if ((r < 0 || r >= a.a_rows) && a.status)
          __hip_atomic_fetch_or(a.status, kStBadRouting, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      if (r >= a.a_rows) r = -1;
    }
    off[mb] = r < 0 ? kOutOfRange : (uint32_t)(r * pitch) + ca * kBlockBytes;
    soff[mb] = r < 0 ? kOutOfRange : (uint32_t)((long long)r * a.KS) + ca * 16;
  }
  // this lane's weight rows: block f's instruction row l.  Plain: columns 8 (l / 4) +
  // 4 f + l % 4 of the wave's 32, so that a lane ends up with 8 neighbouring ones
  const int n0 = u.n0 + wave * (BNO / C::NW);
  uint32_t woff[2], wsoff[2];
#pragma unroll
  for (int f = 0; f < 2; ++f) {
    const int n = n0 + (kSwiglu ? l : 8 * (l >> 2) + 4 * f + (l & 3));
    const int r = kSwiglu && f ? a.NO + n : n;
    woff[f] = n < a.NO ? (uint32_t)(r * pitch) + g * kBlockBytes : kOutOfRange;
    wsoff[f] = n < a.NO ? (uint32_t)((long long)r * a.KS) : kOutOfRange;
  }
  const uint32_t tail = (a.KB & 3) ? (1u << (8 * (a.KB & 3))) - 1 : ~0u;   // scales of the last stage

  f32x4 acc[2][C::MB];
#pragma unroll
  for (int f = 0; f < 2; ++f)
#pragma unroll
    for (int mb = 0; mb < C::MB; ++mb) acc[f][mb] = f32x4{0.f, 0.f, 0.f, 0.f};

  lds_u8* base = (lds_u8*)(uintptr_t)lds;
  lds_u8* sbase = (lds_u8*)(uintptr_t)lds_s;
  for (int kt0 = 0; kt0 < KT; kt0 += C::KC) {
    if (kt0) block_barrier();   // the segment before has been read
#pragma unroll
    for (int j = 0; j < C::KC * C::MB / C::NW; ++j) {
      const int q = wave + C::NW * j;
      const int mb = q % C::MB, kt = kt0 + q / C::MB;   // (uniform)
      uint32_t o = off[0];
#pragma unroll
      for (int i = 1; i < C::MB; ++i) o = mb == i ? off[i] : o;
      dma16(ra, o != kOutOfRange && 4 * kt + ca < a.KB ? o + 64u * (uint32_t)kt : kOutOfRange,
            lds + (uint32_t)((q / C::MB * C::MB + mb) * 1024));
    }
    for (int q = wave; q < C::kSegs * C::MB; q += C::NW) {
      const int mb = q % C::MB, seg = q / C::MB;   // 64 bytes of scales a row: 16 stages
      uint32_t o = soff[0];
#pragma unroll
      for (int i = 1; i < C::MB; ++i) o = mb == i ? soff[i] : o;
      const int k = 4 * kt0 + 64 * seg;
      if (C::KC >= 16 || 4 * ca < C::KC)   // (lanes past a shorter segment: not in LDS)
        dma16(ras, o != kOutOfRange && k + 16 * ca < a.KS ? o + (uint32_t)k : kOutOfRange, lds_s + (uint32_t)(q * 1024));
    }
    u32x4 w[2][C::KC], ws[2][C::KC / 4];
#pragma unroll
    for (int f = 0; f < 2; ++f) {
#pragma unroll
      for (int k = 0; k < C::KC / 4; ++k)
        ws[f][k] = buffer_load16(rws, wsoff[f] != kOutOfRange && 4 * (kt0 + 4 * k) < a.KS ? wsoff[f] + 4u * (uint32_t)(kt0 + 4 * k) : kOutOfRange);
    }
#pragma unroll
    for (int k = 0; k < C::KC; ++k)
#pragma unroll
      for (int f = 0; f < 2; ++f)
        w[f][k] = buffer_load16(rw, woff[f] != kOutOfRange && 4 * (kt0 + k) + g < a.KB ? woff[f] + 64u * (uint32_t)(kt0 + k) : kOutOfRange);
    waitcnt_vm<2 * C::KC + 2 * (C::KC / 4)>();   // a's loads, which were issued first
    block_barrier();
#pragma unroll
    for (int k = 0; k < C::KC; ++k) {
      if (kt0 + k >= KT) break;
      const uint32_t mask = kt0 + k == KT - 1 ? tail : ~0u;
      int sw[2];
#pragma unroll
      for (int f = 0; f < 2; ++f) sw[f] = (int)((ws[f][k / 4][k % 4] & mask) >> (8 * g));
#pragma unroll
      for (int mb = 0; mb < C::MB; ++mb) {
        const u32x4 v = *(lds_u32x4*)(base + (k * C::MB + mb) * 1024 + l * 64 + swz(l >> 2, g) * 16);
        const uint32_t s = *(lds_u32*)(sbase + (k / 16 * C::MB + mb) * 1024 + l * 64 + swz(l >> 2, (k % 16) / 4) * 16 + 4 * (k % 4));
        const i32x8 fa = {(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const i32x8 fw = {(int)w[f][k][0], (int)w[f][k][1], (int)w[f][k][2], (int)w[f][k][3], 0, 0, 0, 0};
          acc[f][mb] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw, fa, acc[f][mb], 4, 4, 0, sw[f], 0,
                                                                        (int)((s & mask) >> (8 * g)));
        }
      }
    }
  }

#pragma unroll
  for (int mb = 0; mb < C::MB; ++mb) {
    const int row = 16 * mb + l;
    if (row >= u.rows_valid) continue;
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = acc[0][mb][i], y = acc[1][mb][i];
      v[i] = kSwiglu ? silu(x) * y : x;
      v[4 + i] = y;
    }
    const int n = n0 + (kSwiglu ? 4 : 8) * g;
    if (n < a.NO) store_few<kSwiglu ? 4 : 8>(a.out + (long long)(u.r0 + row) * a.NO + n, a.NO - n, v);
  }
}

// ---- host --------------------------------------------------------------------------

constexpr long long kMaxGrid = (1 << 24) - 1;   // workgroups of 256 threads: a launch's threads stay below 2^32
constexpr int kMaxSize = INT32_MAX - 256;        // of what is counted in 32 bits in steps of up to 256

int check_rows(const void* wide, size_t wide_align, const void* codes, const void* scales, int64_t rows, int32_t K) {
  if (rows < 0 || K < 1) return MOE_ERR_INVALID_ARG;
  if (K > kMaxSize) return MOE_ERR_UNSUPPORTED;
  if (rows > 0 && (!wide || !codes || !scales)) return MOE_ERR_INVALID_ARG;
  if (!aligned(wide, wide_align) || !aligned(codes, 16) || !aligned(scales, 4)) return MOE_ERR_ALIGNMENT;
  return MOE_OK;
}

// As many tiles of bm rows as there can be, in eight equal shares (one of each XCD).
long long most_tiles(const MxArgs& a, int bm, int nt) {
  const long long n = a.E < a.rows ? a.E : a.rows;
  return (((a.rows - n) / bm + n) * nt + 7) / 8 * 8;
}

// Workgroups that take several tiles: as many as are resident at once, and not more
// than there can be tiles.
constexpr int kCus = 256;
template <class C>
int launch_product(MxArgs a, bool swiglu, hipStream_t s) {
  const int bno = swiglu ? C::BN / 2 : C::BN;
  a.NT = (a.NO + bno - 1) / bno;
  const long long most = most_tiles(a, C::BM, a.NT);
  if (most > INT32_MAX / 2) return MOE_ERR_UNSUPPORTED;
  a.most = (int)most;
  const unsigned grid = (unsigned)(most < C::R * kCus ? most : C::R * kCus);
  if (a.oc) mx4_product_kernel<C, true, true><<<grid, C::kThr, 0, s>>>(a);
  else if (swiglu) mx4_product_kernel<C, true, false><<<grid, C::kThr, 0, s>>>(a);
  else mx4_product_kernel<C, false, false><<<grid, C::kThr, 0, s>>>(a);
  return done();
}

template <class C>
int launch_thin(MxArgs a, bool swiglu, hipStream_t s) {
  const int bno = swiglu ? C::BN / 2 : C::BN;
  a.NT = (a.NO + bno - 1) / bno;
  const unsigned grid = (unsigned)most_tiles(a, C::BM, a.NT);
  if (swiglu) mx4_thin_kernel<C, true><<<grid, C::kThr, 0, s>>>(a);
  else mx4_thin_kernel<C, false><<<grid, C::kThr, 0, s>>>(a);
  return done();
}

// Which tiles: each kind's price in us, from what the host knows (rows, experts,
// sizes; not the counts per expert, which are taken as an even spread's): a call's
// latency and its tiles' share of the CUs, each with a part per stage of 128 of K.
// Fitted to 150 measured calls of each kind (E 8 to 256, 1 to 8192 tokens, K 256 to
// 4096, N 512 to 4096, uniform and Zipf 1.0); the kind with the least price is on average
// 3% and at most 19% slower than the fastest one.  (Also measured: waves in twos and fours
// for 16 and 32 rows, and 128 x 256 tiles: within 0.5% of this on average.)
struct Price {
  int rows, cols;                      // of a tile, cols in rows of w
  double call, call_k, tile, tile_k;   // us, per stage of K; tiles: for one on every CU
  int column_tiles(const MxArgs& a, bool swiglu) const {
    const int bno = swiglu ? cols / 2 : cols;
    return (a.NO + bno - 1) / bno;
  }
  // Thin kernels: a workgroup of 2 cols threads for each tile, of which a launch has less
  // than 2^32, and sums of the experts' tiles that stay in 32 bits whatever the offsets are.
  bool fits(const MxArgs& a, bool swiglu) const {
    return most_tiles(a, rows, column_tiles(a, swiglu)) * 2 * cols < 1ll << 32 && (a.rows / rows + 1) * a.E <= INT32_MAX;
  }
  double of(const MxArgs& a, bool swiglu) const {
    const double mean = (double)a.rows / a.E, hit = a.E * (1 - std::exp(-mean)), KT = (a.KB + 3) / 4;
    const double per = mean / rows + 0.5;   // ragged ends: half a tile
    const double m = std::fmin((double)a.rows, mean > 0.5 * rows ? hit * std::fmax(1.0, per) : hit);
    return call + call_k * KT + m * column_tiles(a, swiglu) / kCus * (tile + tile_k * KT);
  }
};

constexpr int kFirstTile = 4;   // the kinds from here on are tiles, those before are thin
int kind_of(const MxArgs& a, bool swiglu) {
  static constexpr Price kPrices[] = {{16, 32, 2.96, 0.075, 0.07, 0.0756},   {16, 32, 3.32, 0.043, 0.272, 0.0709},
                                      {32, 64, 2.94, 0.127, 0.347, 0.140},   {64, 128, 3.14, 0.216, 1.025, 0.302},
                                      {128, 128, 4.17, 0.201, 1.875, 0.310}, {256, 256, 5.61, 0.402, 8.038, 0.582}};
  int best = 5;
  double least = kPrices[5].of(a, swiglu);
  for (int i = 4; i >= 0; --i) {
    if (i < kFirstTile && !kPrices[i].fits(a, swiglu)) continue;
    const double p = kPrices[i].of(a, swiglu);
    if (p <= least) least = p, best = i;
  }
  return best;
}

int launch(const MxArgs& a, bool swiglu, int kind, hipStream_t s) {
  switch (kind) {
    case 0: return launch_thin<MxThin<1, 8, 1>>(a, swiglu, s);
    case 1: return launch_thin<MxThin<1, 16, 1>>(a, swiglu, s);
    case 2: return launch_thin<MxThin<2, 8, 2>>(a, swiglu, s);
    case 3: return launch_thin<MxThin<4, 8, 4>>(a, swiglu, s);
    case 4: return launch_product<MxTile<128, 128, 2, 2, 3, 2>>(a, swiglu, s);
    default: return launch_product<MxTile<256, 256, 2, 4, 3, 1>>(a, swiglu, s);
  }
}

}  // namespace

extern "C" int moe_mx4_quantize(const void* x, void* codes, void* scales, int64_t rows, int32_t K, int32_t x_type,
                                void* stream) {
  if (!type_ok(x_type)) return MOE_ERR_INVALID_ARG;
  const int bad = check_rows(x, type_size(x_type), codes, scales, rows, K);
  if (bad) return bad;
  if (rows == 0) return MOE_OK;
  const long long per_row = blocks_of(K) * 4ll;
  if (rows > kMaxGrid * 256 / per_row) return MOE_ERR_UNSUPPORTED;
  const unsigned grid = (unsigned)((rows * per_row + 255) / 256);
  const hipStream_t s = (hipStream_t)stream;
  if (x_type == MOE_BF16)
    mx4_quantize_kernel<<<grid, 256, 0, s>>>((const __bf16*)x, (uint8_t*)codes, (uint8_t*)scales, rows, K);
  else
    mx4_quantize_kernel<<<grid, 256, 0, s>>>((const float*)x, (uint8_t*)codes, (uint8_t*)scales, rows, K);
  return done();
}

extern "C" int moe_mx4_quantize_weights(const void* w, void* codes, void* scales, int32_t E, int32_t K, int32_t N,
                                        int32_t w_type, void* stream) {
  if (!type_ok(w_type) || E < 1 || N < 1) return MOE_ERR_INVALID_ARG;
  if (N > kMaxSize) return MOE_ERR_UNSUPPORTED;
  const int bad = check_rows(w, type_size(w_type), codes, scales, 1, K);
  if (bad) return bad;
  const long long kt = (blocks_of(K) + kWBlocks - 1) / kWBlocks, nt = ((long long)N + kWCols - 1) / kWCols;
  if (kt * nt > kMaxGrid / E) return MOE_ERR_UNSUPPORTED;
  const unsigned grid = (unsigned)(kt * nt * E);
  const hipStream_t s = (hipStream_t)stream;
  if (w_type == MOE_BF16)
    mx4_quantize_weights_kernel<<<grid, 256, 0, s>>>((const __bf16*)w, (uint8_t*)codes, (uint8_t*)scales, K, N,
                                                     (int)kt, (int)nt);
  else
    mx4_quantize_weights_kernel<<<grid, 256, 0, s>>>((const float*)w, (uint8_t*)codes, (uint8_t*)scales, K, N,
                                                     (int)kt, (int)nt);
  return done();
}

extern "C" int moe_mx4_dequantize(const void* codes, const void* scales, void* out, int64_t rows, int32_t K,
                                  int32_t out_type, void* stream) {
  if (!type_ok(out_type)) return MOE_ERR_INVALID_ARG;
  const int bad = check_rows(out, type_size(out_type), codes, scales, rows, K);
  if (bad) return bad;
  if (rows == 0) return MOE_OK;
  const long long per_row = (K + 7) / 8;
  if (rows > kMaxGrid * 256 / per_row) return MOE_ERR_UNSUPPORTED;
  const unsigned grid = (unsigned)((rows * per_row + 255) / 256);
  const hipStream_t s = (hipStream_t)stream;
  if (out_type == MOE_BF16)
    mx4_dequantize_kernel<<<grid, 256, 0, s>>>((const uint8_t*)codes, (const uint8_t*)scales, (__bf16*)out, rows, K);
  else
    mx4_dequantize_kernel<<<grid, 256, 0, s>>>((const uint8_t*)codes, (const uint8_t*)scales, (float*)out, rows, K);
  return done();
}

namespace {

// moe_mx4_product, or with oc and os, where the call's tiles can, its output in 4 bits;
// *in_codes: whether it is.
int product(const void* a_codes, const void* a_scales, const void* w_codes, const void* w_scales,
            const int32_t* expert_offsets, const int32_t* row_ids, void* out, void* oc, void* os, bool* in_codes,
            int64_t a_rows, int64_t rows, int32_t K, int32_t N, int32_t E, bool swiglu, void* workspace, void* stream) {
  MxArgs a = {};
  a.a = (const uint8_t*)a_codes;
  a.as = (const uint8_t*)a_scales;
  a.w = (const uint8_t*)w_codes;
  a.ws = (const uint8_t*)w_scales;
  a.offsets = expert_offsets;
  a.row_ids = row_ids;
  a.out = (__bf16*)out;
  a.status = (uint32_t*)workspace;
  a.rows = rows;
  a.a_rows = (int)a_rows;
  a.K = K;
  a.N = N;
  a.E = E;
  a.KB = blocks_of(K);
  a.KS = scale_pitch(K);
  a.NO = swiglu ? N / 2 : N;
  const int kind = kind_of(a, swiglu);
  if (oc && kind >= kFirstTile) {
    a.oc = (uint8_t*)oc;
    a.os = (uint8_t*)os;
    a.OB = blocks_of(a.NO);
    a.OS = scale_pitch(a.NO);
    *in_codes = true;
  }
  return launch(a, swiglu, kind, (hipStream_t)stream);
}

}  // namespace

extern "C" int moe_mx4_product(const void* a_codes, const void* a_scales, const void* w_codes, const void* w_scales,
                               const int32_t* expert_offsets, const int32_t* row_ids, void* out, int64_t a_rows,
                               int64_t rows, int32_t K, int32_t N, int32_t E, int32_t swiglu, void* workspace,
                               void* stream) {
  if (a_rows < 0 || rows < 0 || K < 1 || N < 1 || E < 1 || (swiglu && N % 2)) return MOE_ERR_INVALID_ARG;
  const long long pitch = ((long long)K + kBlock - 1) / kBlock * kBlockBytes;
  if (E > kMaxExperts || rows > kMaxSize || K > kMaxSize || pitch * N > INT32_MAX || (a_rows > 0 && pitch > INT32_MAX / a_rows))
    return MOE_ERR_UNSUPPORTED;
  if (rows > 0 && (!a_codes || !a_scales || !w_codes || !w_scales || !expert_offsets || !out)) return MOE_ERR_INVALID_ARG;
  if (!aligned(a_codes, 16) || !aligned(w_codes, 16) || !aligned(a_scales, 4) || !aligned(w_scales, 4) ||
      !aligned(expert_offsets, 4) || !aligned(row_ids, 4) || !aligned(out, 2) || !aligned(workspace, 256))
    return MOE_ERR_ALIGNMENT;
  if (rows == 0) return MOE_OK;
  if (a_rows == 0) return MOE_ERR_INVALID_ARG;
  return product(a_codes, a_scales, w_codes, w_scales, expert_offsets, row_ids, out, nullptr, nullptr, nullptr, a_rows, rows,
                 K, N, E, swiglu != 0, workspace, stream);
}

namespace {

// The layer's scratch: activations in 4 bits and in bf16, each from a 256-byte line on.
struct LayerScratch {
  size_t hc, hs, x, xc, xs, y, bytes;
};
bool layer_scratch(int32_t T, int32_t H, int32_t I, int32_t topk, LayerScratch* l) {
  if (T < 0 || H < 1 || I < 1 || topk < 1 || topk > 64 || H > kMaxSize || I > kMaxSize) return false;
  const size_t rows = (size_t)T * topk;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  l->hc = take((size_t)T * blocks_of(H) * kBlockBytes);
  l->hs = take((size_t)T * scale_pitch(H));
  l->x = take(rows * I * 2);
  l->xc = take(rows * blocks_of(I) * kBlockBytes);
  l->xs = take(rows * scale_pitch(I));
  l->y = take(rows * H * 2);
  l->bytes = at;
  return true;
}

}  // namespace

extern "C" size_t moe_mx4_layer_scratch_size(int32_t T, int32_t H, int32_t I, int32_t topk) {
  LayerScratch l;
  return layer_scratch(T, H, I, topk, &l) ? l.bytes : 0;
}

extern "C" int moe_mx4_layer_forward(const void* hidden, const void* w1_codes, const void* w1_scales,
                                     const void* w2_codes, const void* w2_scales, const int32_t* expert_offsets,
                                     const int32_t* token_ids, const int32_t* slot_rows, const float* gates, void* out,
                                     int32_t T, int32_t H, int32_t I, int32_t E, int32_t topk, int32_t out_type,
                                     void* scratch, size_t scratch_bytes, void* workspace, void* stream) {
  LayerScratch l;
  if (T < 0 || H < 1 || I < 1 || E < 1 || topk < 1 || !type_ok(out_type)) return MOE_ERR_INVALID_ARG;
  if (!layer_scratch(T, H, I, topk, &l) || I > INT32_MAX / 2 || (long long)T * topk > kMaxSize) return MOE_ERR_UNSUPPORTED;
  if (T == 0) return MOE_OK;
  // (everything is looked at before the first launch)
  if (!hidden || !w1_codes || !w1_scales || !w2_codes || !w2_scales || !expert_offsets || !token_ids || !slot_rows ||
      !gates || !out)
    return MOE_ERR_INVALID_ARG;
  if (!scratch || scratch_bytes < l.bytes) return MOE_ERR_WORKSPACE;
  if (!aligned(hidden, 2) || !aligned(w1_codes, 16) || !aligned(w1_scales, 4) || !aligned(w2_codes, 16) ||
      !aligned(w2_scales, 4) || !aligned(expert_offsets, 4) || !aligned(token_ids, 4) || !aligned(slot_rows, 4) ||
      !aligned(gates, 4) || !aligned(out, type_size(out_type)) || !aligned(scratch, 16) || !aligned(workspace, 256))
    return MOE_ERR_ALIGNMENT;
  const long long rows = (long long)T * topk, ph = (long long)blocks_of(H) * kBlockBytes,
                  pi = (long long)blocks_of(I) * kBlockBytes;
  if (E > kMaxExperts || ph * T > INT32_MAX || ph * 2 * I > INT32_MAX || pi * rows > INT32_MAX || pi * H > INT32_MAX)
    return MOE_ERR_UNSUPPORTED;
  uint8_t* s = (uint8_t*)scratch;
  int r = moe_mx4_quantize(hidden, s + l.hc, s + l.hs, T, H, MOE_BF16, stream);
  bool in_codes = false;   // up-projection tiles quantise what they hold; thin ones leave it to a launch
  if (r == MOE_OK)
    r = product(s + l.hc, s + l.hs, w1_codes, w1_scales, expert_offsets, token_ids, s + l.x, s + l.xc, s + l.xs,
                &in_codes, T, rows, H, 2 * I, E, true, workspace, stream);
  if (r == MOE_OK && !in_codes) r = moe_mx4_quantize(s + l.x, s + l.xc, s + l.xs, rows, I, MOE_BF16, stream);
  if (r == MOE_OK)
    r = moe_mx4_product(s + l.xc, s + l.xs, w2_codes, w2_scales, expert_offsets, nullptr, s + l.y, rows, rows, I, H, E,
                        0, workspace, stream);
  if (r == MOE_OK)
    r = moe_combine_rows(s + l.y, slot_rows, gates, out, T, topk, rows, H, MOE_BF16, out_type, workspace, stream);
  return r;
}
