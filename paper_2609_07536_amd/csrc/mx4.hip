// Microscaled 4-bit floating point on gfx950: quantisation of activations and
// weights, and the experts' products (C ABI and format: moe_experts.h).
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <type_traits>

#include "expert_units.h"
#include "lds_loads.h"
#include "moe_experts.h"
#include "status_bits.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 32;         // elements that share a scale
constexpr int kBlockBytes = 16;    // their codes

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
template <class T>
__device__ __forceinline__ void store8(T* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    T __attribute__((ext_vector_type(8))) x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (T)v[i];
    *(typename Mem<T, 8>::type*)p = x;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (T)v[i];
  }
}

template <int kCtrl>
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, kCtrl, 0xf, 0xf, true));
}

// Eight elements a thread, four neighbouring threads a block: every thread's
// load and store is one of the wave's contiguous ones.
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
// contiguous bytes per column.
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
  store8(out + row * K + 8 * c, K - 8 * c, v);
}

// ---- the experts' products -------------------------------------------------------
//
// A workgroup takes a tile of BM rows of one expert by BN of its weights' rows.
// Both operands are rows of codes along K, so a stage of 128 of K is 64 bytes of
// each, loaded straight into an LDS ring; a lane's operand of the 32x32x64
// scaled matrix instruction is one block: 16 bytes of codes and one scale byte.
// The weights are the instruction's first operand, so a lane ends up with
// columns of one row of the output.

struct MxArgs {
  const uint8_t* a;          // [a_rows, KB, 16]
  const uint8_t* as;         // [a_rows, KS]
  const uint8_t* w;          // [E, N, KB, 16]
  const uint8_t* ws;         // [E, N, KS]
  const int32_t* offsets;    // [E + 1]
  const int32_t* row_ids;    // [rows] or null: row r is a's row r
  __bf16* out;               // [rows, NO]
  uint32_t* status;          // or null
  long long rows;
  int a_rows, K, N, E, KB, KS;
  int NO;                    // columns of out: N, or N / 2 with SwiGLU
  int NT;                    // tiles along them
};

// BM rows by BN weight rows, WM x WN waves, a ring of S stages
template <int BM_, int BN_, int WM_, int WN_, int S_>
struct MxTile {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, S = S_;
  static constexpr int NW = WM * WN, kThr = NW * 64;
  static constexpr int MB = BM / WM / 32, NB = BN / WN / 32;   // a wave's 32 x 32 blocks
  static constexpr int kRows = BM + BN;
  static constexpr int kStage = kRows * 64;                    // bytes: 4 blocks of each row
  static constexpr int LPS = kStage / 1024 / NW;               // 1 KB loads per wave and stage
  static constexpr int kSeg = 16;                              // stages whose scales are in LDS together
  static constexpr int kScaleRow = kSeg * 4;                   // as many bytes as a stage's row
  static constexpr int kScales = kRows * kScaleRow;
  static_assert(kStage % (1024 * NW) == 0 && MB >= 1 && NB >= 1, "loads per wave");
  static_assert((S - 2) * LPS <= 63 && S >= 2, "vmcnt range");
  static_assert(S * kStage + kScales <= 160 * 1024, "LDS");
};

// Position of 16-byte chunk c (0..3) of row r within the row's 64 bytes: the 16
// rows that a read touches at once then fall on distinct banks.
__device__ __forceinline__ int swz(int r, int c) { return c ^ ((r >> 2) & 3); }

typedef const __attribute__((address_space(3))) uint8_t lds_u8;
typedef const __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef const __attribute__((address_space(3))) uint32_t lds_u32;

template <class C, bool kSwiglu>
__global__ void __launch_bounds__(C::kThr) mx4_product_kernel(MxArgs a) {
  __shared__ __align__(1024) uint8_t smem[C::S * C::kStage + C::kScales];
  constexpr int BNO = kSwiglu ? C::BN / 2 : C::BN;   // output columns of a tile
  int rows_dev;
  const SmallUnit u = small_unit<C::BM, BNO>(a.offsets, a.rows, a.E, a.NT, a.status, &rows_dev);
  if (!u.ok) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t lds = lds_addr(smem), lds_s = lds + C::S * C::kStage;
  const long long pitch = (long long)a.KB * kBlockBytes;
  const i32x4 ra = buffer_rsrc(a.a, a.a_rows * pitch), ras = buffer_rsrc(a.as, (long long)a.a_rows * a.KS);
  const i32x4 rw = buffer_rsrc(a.w + u.e * (a.N * pitch), a.N * pitch);
  const i32x4 rws = buffer_rsrc(a.ws + (long long)u.e * a.N * a.KS, (long long)a.N * a.KS);

  // tile row i (BM rows of a, then BN of w) to its row in memory, or -1
  auto row_of = [&](int i) -> int {
    if (i < C::BM) {
      if (i >= u.rows_valid) return -1;
      const int r = u.r0 + i;
      if (!a.row_ids) return r < a.a_rows ? r : -1;
      const int id = a.row_ids[r];
      if (id < 0 || id >= a.a_rows) {
        if (a.status) __hip_atomic_fetch_or(a.status, kStBadRouting, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        return -1;
      }
      return id;
    }
    const int j = i - C::BM;
    if (!kSwiglu) return u.n0 + j < a.N ? u.n0 + j : -1;
    const int n = u.n0 + (j < BNO ? j : j - BNO);
    return n < a.NO ? (j < BNO ? n : a.NO + n) : -1;
  };
  // this lane's part of its wave's loads: a load is 16 rows of a stage
  uint32_t off[C::LPS], soff[C::LPS];
  int chunk[C::LPS];
#pragma unroll
  for (int q = 0; q < C::LPS; ++q) {
    const int i = (C::LPS * wave + q) * 16 + (lane >> 2), r = row_of(i);
    chunk[q] = swz(i, lane & 3);
    off[q] = r < 0 ? kOutOfRange : (uint32_t)(r * pitch) + chunk[q] * kBlockBytes;
    // (scales: the same rows in the same order, 16 bytes of a row's 64 a lane)
    soff[q] = r < 0 ? kOutOfRange : (uint32_t)((long long)r * a.KS) + chunk[q] * 16;
  }
  const int KT = (a.KB + 3) / 4;
  auto issue = [&](int kt, int slot) {
#pragma unroll
    for (int q = 0; q < C::LPS; ++q) {
      const bool in = off[q] != kOutOfRange && 4 * kt + chunk[q] < a.KB;
      const int i = (C::LPS * wave + q) * 16;   // uniform: a's rows or w's
      dma16(i < C::BM ? ra : rw, in ? off[q] + 64u * (uint32_t)kt : kOutOfRange,
            lds + (uint32_t)(slot * C::kStage + i * 64));
    }
  };
  auto issue_scales = [&](int seg) {
#pragma unroll
    for (int q = 0; q < C::LPS; ++q) {
      const uint32_t k = (uint32_t)(seg * C::kScaleRow);
      const bool in = soff[q] != kOutOfRange && (int)k + chunk[q] * 16 < a.KS;
      const int i = (C::LPS * wave + q) * 16;
      dma16(i < C::BM ? ras : rws, in ? soff[q] + k : kOutOfRange, lds_s + (uint32_t)(i * 64));
    }
  };

  const int wm0 = (wave / C::WN) * C::MB * 32, wn = wave % C::WN;
  // tile rows of this wave's block of w: with SwiGLU its first half gate, the other up
  auto w_row = [&](int nb) {
    return kSwiglu ? (nb < C::NB / 2 ? (wn * (C::NB / 2) + nb) * 32 : BNO + (wn * (C::NB / 2) + nb - C::NB / 2) * 32)
                   : (wn * C::NB + nb) * 32;
  };
  const int h = lane >> 5, l = lane & 31;
  // the row of w that a lane brings as row l of the instruction, so that its
  // accumulators 8c .. 8c + 7 are columns 16c + 8h .. of one output row
  const int lw = 16 * (l >> 4) + 8 * ((l >> 2) & 1) + 4 * ((l >> 3) & 1) + (l & 3);
  const uint32_t tail = (a.KB & 3) ? (1u << (8 * (a.KB & 3))) - 1 : ~0u;   // scales of the last stage

  f32x16 acc[C::NB][C::MB];
#pragma unroll
  for (int nb = 0; nb < C::NB; ++nb)
#pragma unroll
    for (int mb = 0; mb < C::MB; ++mb)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[nb][mb][i] = 0.f;

  issue_scales(0);
#pragma unroll
  for (int s = 0; s < C::S - 1; ++s) issue(s, s);
  int slot = 0;
  for (int kt = 0; kt < KT; ++kt) {
    waitcnt_vm<(C::S - 2) * C::LPS>();
    block_barrier();
    if (kt > 0 && kt % C::kSeg == 0) {   // the next segment's scales (a reduction over 2048)
      issue_scales(kt / C::kSeg);
      waitcnt_vm<0>();
      block_barrier();
    }
    issue(kt + C::S - 1, (slot + C::S - 1) % C::S);   // (past the end: nothing is read)
    lds_u8* base = (lds_u8*)(uintptr_t)(lds + (uint32_t)(slot * C::kStage));
    lds_u8* sbase = (lds_u8*)(uintptr_t)lds_s;
    const uint32_t mask = kt == KT - 1 ? tail : ~0u;
    const int sc = (kt % C::kSeg) >> 2, sb = (kt & 3) * 4;   // the stage's dword of a scale row
    uint32_t sa[C::MB], sw[C::NB];
#pragma unroll
    for (int mb = 0; mb < C::MB; ++mb) {
      const int r = wm0 + mb * 32 + l;
      sa[mb] = (*(lds_u32*)(sbase + r * 64 + swz(r, sc) * 16 + sb) & mask) >> (8 * h);
    }
#pragma unroll
    for (int nb = 0; nb < C::NB; ++nb) {
      const int r = C::BM + w_row(nb) + lw;
      sw[nb] = (*(lds_u32*)(sbase + r * 64 + swz(r, sc) * 16 + sb) & mask) >> (8 * h);
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      i32x8 fa[C::MB], fw[C::NB];
#pragma unroll
      for (int mb = 0; mb < C::MB; ++mb) {
        const int r = wm0 + mb * 32 + l;
        const u32x4 v = *(lds_u32x4*)(base + r * 64 + swz(r, 2 * ks + h) * 16);
        fa[mb] = i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
      }
#pragma unroll
      for (int nb = 0; nb < C::NB; ++nb) {
        const int r = C::BM + w_row(nb) + lw;
        const u32x4 v = *(lds_u32x4*)(base + r * 64 + swz(r, 2 * ks + h) * 16);
        fw[nb] = i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
      }
#pragma unroll
      for (int nb = 0; nb < C::NB; ++nb)
#pragma unroll
        for (int mb = 0; mb < C::MB; ++mb)
          acc[nb][mb] = ks == 0 ? __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fw[nb], fa[mb], acc[nb][mb], 4, 4, 0,
                                                                                   (int)sw[nb], 0, (int)sa[mb])
                                : __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fw[nb], fa[mb], acc[nb][mb], 4, 4, 2,
                                                                                   (int)sw[nb], 2, (int)sa[mb]);
    }
    slot = slot + 1 == C::S ? 0 : slot + 1;
  }
  waitcnt_vm<0>();   // (the loads past the end write to LDS as well)

  // each lane's rows: eight columns, one 16-byte store, at a time
#pragma unroll
  for (int mb = 0; mb < C::MB; ++mb) {
    const int row = wm0 + mb * 32 + l;
    if (row >= u.rows_valid) continue;
    __bf16* o = a.out + (long long)(u.r0 + row) * a.NO;
#pragma unroll
    for (int nb = 0; nb < (kSwiglu ? C::NB / 2 : C::NB); ++nb)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          v[i] = acc[nb][mb][8 * c + i];
          if (kSwiglu) {
            const float up = acc[nb + C::NB / 2][mb][8 * c + i];
            v[i] = v[i] / (1.f + __expf(-v[i])) * up;
          }
        }
        const int n = u.n0 + (kSwiglu ? (wn * (C::NB / 2) + nb) * 32 : w_row(nb)) + 16 * c + 8 * h;
        if (n < a.NO) store8(o + n, a.NO - n, v);
      }
  }
}

// ---- host --------------------------------------------------------------------------

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
bool type_ok(int32_t t) { return t == MOE_BF16 || t == MOE_F32; }
size_t type_size(int32_t t) { return t == MOE_BF16 ? 2 : 4; }
int done() { return hipGetLastError() == hipSuccess ? MOE_OK : MOE_ERR_HIP; }

constexpr long long kMaxGrid = 1 << 24;   // workgroups of 256 threads: a launch's threads stay below 2^32

int check_rows(const void* wide, size_t wide_align, const void* codes, const void* scales, int64_t rows, int32_t K) {
  if (rows < 0 || K < 1) return MOE_ERR_INVALID_ARG;
  if (K > INT32_MAX - 256) return MOE_ERR_UNSUPPORTED;
  if (rows > 0 && (!wide || !codes || !scales)) return MOE_ERR_INVALID_ARG;
  if (!aligned(wide, wide_align) || !aligned(codes, 16) || !aligned(scales, 4)) return MOE_ERR_ALIGNMENT;
  return MOE_OK;
}

template <class C>
int launch_product(MxArgs a, bool swiglu, hipStream_t s) {
  const int bno = swiglu ? C::BN / 2 : C::BN;
  a.NT = (a.NO + bno - 1) / bno;
  // the most tiles that `rows` rows in at most min(E, rows) experts make, in eight equal shares
  const long long n = a.E < a.rows ? a.E : a.rows;
  const long long grid = (((a.rows - n) / C::BM + n) * a.NT + 7) / 8 * 8;
  if (grid * C::kThr >= 1ll << 32) return MOE_ERR_UNSUPPORTED;
  if (swiglu) mx4_product_kernel<C, true><<<(unsigned)grid, C::kThr, 0, s>>>(a);
  else mx4_product_kernel<C, false><<<(unsigned)grid, C::kThr, 0, s>>>(a);
  return done();
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

extern "C" int moe_mx4_product(const void* a_codes, const void* a_scales, const void* w_codes, const void* w_scales,
                               const int32_t* expert_offsets, const int32_t* row_ids, void* out, int64_t a_rows,
                               int64_t rows, int32_t K, int32_t N, int32_t E, int32_t swiglu, void* workspace,
                               void* stream) {
  if (a_rows < 0 || rows < 0 || K < 1 || N < 1 || E < 1 || (swiglu && N % 2)) return MOE_ERR_INVALID_ARG;
  const long long pitch = ((long long)K + kBlock - 1) / kBlock * kBlockBytes;
  if (E > 1024 || rows > INT32_MAX || pitch * N > INT32_MAX || (a_rows > 0 && pitch > INT32_MAX / a_rows))
    return MOE_ERR_UNSUPPORTED;
  if (rows > 0 && (!a_codes || !a_scales || !w_codes || !w_scales || !expert_offsets || !out)) return MOE_ERR_INVALID_ARG;
  if (!aligned(a_codes, 16) || !aligned(w_codes, 16) || !aligned(a_scales, 4) || !aligned(w_scales, 4) ||
      !aligned(expert_offsets, 4) || !aligned(row_ids, 4) || !aligned(out, 2) || !aligned(workspace, 256))
    return MOE_ERR_ALIGNMENT;
  if (rows == 0) return MOE_OK;
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
  const hipStream_t s = (hipStream_t)stream;
  const long long mean = rows / E;
  if (mean >= 128) return launch_product<MxTile<256, 256, 2, 4, 3>>(a, swiglu, s);
  return launch_product<MxTile<64, 128, 1, 2, 3>>(a, swiglu, s);
}
