// The post-router layer for a few tokens in two launches, for gfx950 (C ABI: moe_block.h).
//
// A token's row is a row of the 16x16x32 matrix instruction, so one instruction
// takes all tokens through 32 of K and 16 columns of an expert's weights.  Weights go
// straight from memory to registers, each read once (but 4-bit ones of the first launch once for
// seven tokens, where there are more than eight), with no stop in LDS: what bounds the
// layer is their stream, and the first launch's loads need nothing but the choice itself.
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "call_checks.h"
#include "lds_loads.h"
#include "moe_block.h"

namespace {

constexpr int kMaxTopk = 64, kMaxExperts = 1024;
constexpr int kMaxWidth = 1 << 22;   // H and I
constexpr int kMaxShares = 16;       // workgroups that share a tile of the second launch
constexpr int kBlock = 32;   // elements of an mx4 block

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4_2 __attribute__((ext_vector_type(4), aligned(2)));

// What the first launch leaves for the second of a unit (a slot that is the first to name
// its expert, or an expert where there are more slots than experts): the expert or -1, the
// tokens that name it and the sum of each one's gates, in slot order.  The activation of
// token t for it is row T unit + t of `act`, in two parts of bf16 whose sum has 16 bits of
// mantissa: rounded to one, it would add as much to the layer's error as a bf16 output does.
struct Hit {
  int32_t e;
  uint32_t tokens;
  float gate[MOE_FEW_TOKENS];
};

struct FewArgs {
  const __bf16* x;
  const uint8_t *w1, *w1_scales, *w2, *w2_scales;   // bf16 or codes
  const int32_t* ids;
  const float* gates;
  void* out;
  Hit* hits;         // [units]
  __bf16* act;       // [T units][2][pitch]
  float* parts;      // [shares][T][H], where the second launch has several shares
  uint32_t* count;   // [tiles of the second launch]: shares that are there
  int T, H, I, E, topk, first, slots, units, pitch;
  int tiles, out_tiles, shares;   // (tiles: of a unit of the first launch)
  bool out16;
};

__device__ __forceinline__ int expert_of(const FewArgs& a, int id) {
  const int64_t e = (int64_t)id - a.first;
  return e >= 0 && e < a.E ? (int)e : -1;
}

// ---- operands ----------------------------------------------------------------------
//
// Weights come by buffer loads: past an expert's last row they read zeros, so no step
// needs a test.  Offsets are below 2^31; kOutOfRange is past every extent.
typedef __amdgpu_buffer_rsrc_t Buffer;
__device__ __forceinline__ Buffer buffer(const void* p, long long bytes) {
  const uint64_t b = (uint64_t)(uintptr_t)p;
  const uint64_t u = ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(b >> 32)) << 32) |
                     (uint32_t)__builtin_amdgcn_readfirstlane((int)b);
  return __builtin_amdgcn_make_buffer_rsrc((void*)(uintptr_t)u, 0, __builtin_amdgcn_readfirstlane((int)bytes),
                                           0x00020000);   // (raw 32-bit data)
}
__device__ __forceinline__ u32x4 load16(Buffer b, uint32_t at) { return __builtin_amdgcn_raw_buffer_load_b128(b, at, 0, 0); }

__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// bf16 weights, [K, columns]: a lane takes four neighbouring columns of eight rows of K, so
// that sixteen lanes read whole 128-byte lines, and eight elements of a token's row.  The
// matrix instruction takes a column's eight values: one permutation for two of them.
struct Bf16Step {
  u32x2 w[8];
  u32x4 x;
  __device__ __forceinline__ void load(Buffer b, uint32_t at, uint32_t pitch) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __builtin_amdgcn_raw_buffer_load_b64(b, at + i * pitch, 0, 0);
  }
  __device__ __forceinline__ u32x4 column(int c) const {
    u32x4 v;
#pragma unroll
    for (int p = 0; p < 4; ++p)
      v[p] = __builtin_amdgcn_perm(w[2 * p + 1][c / 2], w[2 * p][c / 2], c % 2 ? 0x07060302u : 0x05040100u);
    return v;
  }
};
// A wave's n steps, the loads of two of them under way; a step past the end is loads of
// nothing and products of zeros, without a branch, so that the waits stay exact.
template <class Step, class Load, class Use>
__device__ __forceinline__ void run_steps(int n, Load load, Use use) {
  Step b[2];
  load(b[0], 0);
  load(b[1], 1);
  int i = 0;
  for (; i + 2 < n; i += 2) {
    use(b[0], i);
    load(b[0], i + 2);
    use(b[1], i + 1);
    load(b[1], i + 3);
  }
  use(b[0], i);
  use(b[1], i + 1);
}

// Weights in mx4, N rows of codes along K: a wave's step is 16 blocks (512 of K), a lane's
// four of them of each row.  The scales of a row's 16 blocks come by one load and the
// tokens' elements through LDS, a row of them by one load: four loads of elements for every
// load of codes, most of them of tokens that do not name the expert, and one of a scale
// byte took half of the time (46 MB in 18.4 us, 10.9 without them).
constexpr int kStepBlocks = 16, kStepK = kStepBlocks * kBlock;
constexpr int kStepBytes = 2 * kStepK + 16;   // of a token's row in LDS (rows start four banks apart)
template <int N>
struct Mx4Step {
  u32x4 codes[N][4], scale[N];
  // row r of KB blocks and KS scale bytes, from block kb0 on
  __device__ __forceinline__ void load(int n, Buffer c, Buffer s, uint32_t r, int kb0, int KB, int KS, bool in) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int kb = kb0 + 4 * j + g;
      codes[n][j] = load16(c, in && kb < KB ? (r * KB + kb) * 16 : kOutOfRange);
    }
    if (KS >= kStepBlocks) {   // (the last 16 bytes of the row at most)
      scale[n] = load16(s, in ? r * KS + min(kb0, KS - kStepBlocks) : kOutOfRange);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        scale[n][j] = __builtin_amdgcn_raw_buffer_load_b32(s, in && 4 * j < KS ? r * KS + 4 * j : kOutOfRange, 0, 0);
    }
  }
  // brings the scales of blocks kb0 + 4 j .. into scale[n][j], zeros for blocks past the row's
  // (their bytes in memory are anything, and 255 would make NaN of codes of zeros)
  __device__ __forceinline__ void align(int kb0, int KB, int KS) {
    for (int past = kb0 + kStepBlocks - KS; KS >= kStepBlocks && past > 0; past -= 4)
#pragma unroll
      for (int n = 0; n < N; ++n) scale[n] = u32x4{scale[n][1], scale[n][2], scale[n][3], 0};
    if (kb0 + kStepBlocks > KB) {   // (uniform)
      const int first = kb0 + (int)((threadIdx.x & 63) >> 4);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < N; ++n) scale[n][j] = first + 4 * j < KB ? scale[n][j] : 0;
    }
  }
  __device__ __forceinline__ uint32_t byte(int n, int j) const {
    return (scale[n][j] >> (((threadIdx.x & 63) >> 4) * 8)) & 255;
  }
  // eight values (what a code stands for is exact in bf16)
  __device__ __forceinline__ u32x4 eight(int n, int j, int q) const {
    const uint32_t b = byte(n, j);
    const float s = __uint_as_float(b == 0 ? 0x00400000u : b << 23);
    const uint32_t c = codes[n][j][q];
    return {__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2)),
            __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3))};
  }
  // whether one of the lane's blocks is NaN
  __device__ __forceinline__ bool bad(int n) const {
    bool r = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) r |= byte(n, j) == 255;
    return r;
  }
};
// v, or NaN where a lane of the same column had a NaN block (its 32 operands are anything).
__device__ __forceinline__ f32x4 with_nan(f32x4 v, bool bad) {
  const uint64_t m = __ballot(bad);
  if (m) {   // (uniform, and rare)
    if ((m >> (threadIdx.x & 15)) & 0x0001000100010001ull) v = f32x4{1.f, 1.f, 1.f, 1.f} * __builtin_nanf("");
  }
  return v;
}

// Eight elements of a row of K from k on, zeros past its end, for any K.
__device__ __forceinline__ u32x4 row8(const __bf16* row, int k, int K) {
  u32x4 v = {0, 0, 0, 0};
  if (k + 8 <= K) {
    v = *(const u32x4_2*)(row + k);
  } else if (k < K) {
    const uint16_t* q = (const uint16_t*)row + k;
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (k + i < K) v[i / 2] |= (uint32_t)q[i] << (16 * (i % 2));
  }
  return v;
}
// 512 elements from k on of a row (of K) to a row of the wave's LDS, zeros past its end.
// kOdd: K is no multiple of 32, and the row may start at any element.
template <bool kOdd>
__device__ __forceinline__ void row_to_lds(uint8_t* lds, i32x4 rsrc, const __bf16* x, int at, int k, int K) {
  const int lane = threadIdx.x & 63;
  k += 8 * lane;
  if constexpr (kOdd)
    *(u32x4*)(lds + 16 * lane) = row8(x + at, k, K);
  else
    dma16(rsrc, k < K ? 2u * (at + k) : kOutOfRange, lds_addr(lds));
}
// Before a wave's rows in LDS are written again: what was there has been read.
__device__ __forceinline__ void rows_read() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// The four operands of eight of block 4 j + g of the lane's row.
__device__ __forceinline__ u32x4 row_operand(const uint8_t* lds, int row, int j, int q) {
  return *(const u32x4*)(lds + row * kStepBytes + (4 * j + (int)((threadIdx.x & 63) >> 4)) * 2 * kBlock + 16 * q);
}

// ---- the first launch ------------------------------------------------------------------

// A workgroup's expert and the tokens that name it (bit t); false: nothing to do.  The
// workgroup's own slot comes first, by itself; then lane t looks through token t's slots, eight
// at a time, whose loads (the eighth's in a branch) are under way together.
__device__ __forceinline__ bool few_unit(const FewArgs& a, int u, int* e, uint32_t* tokens) {
  const int t = threadIdx.x & 63;
  const bool by_slot = a.slots <= a.E;
  const int32_t* p = a.ids + min(t, a.T - 1) * a.topk;
  const int own = a.ids[by_slot ? u : 0];
  int at = -1;   // token t's first slot that names the expert
  *e = 0;
  for (int j0 = 0; j0 < a.topk; j0 += 8) {
    int id[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) id[i] = p[min(j0 + i, a.topk - 1)];
    *e = by_slot ? expert_of(a, own) : u;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (at < 0 && j0 + i < a.topk && expert_of(a, id[i]) == *e) at = t * a.topk + j0 + i;
  }
  *tokens = (uint32_t)__ballot(t < a.T && at >= 0);
  if (*e < 0 || *tokens == 0) return false;
  // (the first slot that names the expert has it)
  return !by_slot || __builtin_amdgcn_readlane(at, (int)__builtin_ctz(*tokens)) == u;
}

// What the second launch needs of a unit, by the unit's first workgroup.
__device__ __forceinline__ void write_hit(const FewArgs& a, int u, int e, uint32_t tokens) {
  const int t = threadIdx.x;
  if (t < MOE_FEW_TOKENS) {
    float g = 0.f;
    if ((tokens >> t) & 1)
      for (int j = 0; j < a.topk; ++j)
        if (expert_of(a, a.ids[t * a.topk + j]) == e) g += a.gates[t * a.topk + j];
    a.hits[u].gate[t] = g;
  }
  if (t == 0) {
    a.hits[u].e = e;
    a.hits[u].tokens = tokens;
  }
}

// The unit and tile of a workgroup, and what every first launch does besides; false: nothing
// to do.
__device__ __forceinline__ bool begin_up(const FewArgs& a, int* unit, int* tile, int* e, uint32_t* tokens) {
  *unit = blockIdx.x / a.tiles;
  *tile = blockIdx.x - *unit * a.tiles;
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < a.out_tiles; i += blockDim.x) a.count[i] = 0;
  if (few_unit(a, *unit, e, tokens)) return true;
  if (*tile == 0) write_hit(a, *unit, -1, 0);
  return false;
}

// The lane's sums of column n to the wave's LDS [16 tokens][columns].
template <int COLS>
__device__ __forceinline__ void put_column(float (*sums)[COLS], int n, f32x4 v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < 4; ++i) sums[4 * (lane >> 4) + i][n] = v[i];
}

// silu(gate) * up of the waves' sums, `pitch` floats apart, in fp32.
template <int W, int COLS>
__device__ __forceinline__ float swiglu(const float* sums, int pitch, int t, int g, int u) {
  float x = 0.f, y = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    x += sums[w * pitch + t * COLS + g];
    y += sums[w * pitch + t * COLS + u];
  }
  return x / (1.f + expf(-x)) * y;
}

// An element of a token's activation, in its two parts.
__device__ __forceinline__ void put_act(const FewArgs& a, int unit, int t, int o, float v) {
  const __bf16 hi = (__bf16)v;
  const float rest = v - (float)hi;
  __bf16* p = a.act + ((long long)a.T * unit + t) * 2 * a.pitch + o;
  p[0] = hi;
  p[a.pitch] = (__bf16)(fabsf(rest) < __builtin_inff() ? rest : 0.f);   // (of an infinity there is no rest)
}

// 64 packed columns (32 outputs), the waves taking every W-th 32 of K.  Bound by the stream of
// the weights: 16 tokens, 32 experts of 2048 x 704, 34 us for 185 MB (5.4 TB/s); one token, 6
// experts, 9 to 10 us for 35 MB, a quarter of it the launch (sixteen waves a workgroup, for twice
// the loads under way: equal).
constexpr int kCols = 64;
template <int W>
__global__ void __launch_bounds__(64 * W) few_up_kernel(FewArgs a) {
  __shared__ float lds[W][16][kCols];
  int unit, tile, e;
  uint32_t tokens;
  if (!begin_up(a, &unit, &tile, &e, &tokens)) return;
  const int wave = threadIdx.x >> 6, n = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
  const int N = 2 * a.I, col = tile * kCols + 4 * n;
  const bool mine = (tokens >> n) & 1;
  const long long bytes = 2LL * a.H * N;
  const Buffer w = buffer(a.w1 + e * bytes, bytes), x = buffer(a.x, 2LL * a.T * a.H);
  const uint32_t pitch = 2 * N;
  f32x4 acc[4] = {};
  const int steps = (a.H + 31) / 32;
  run_steps<Bf16Step>(
      (steps - wave + W - 1) / W,
      [&](Bf16Step& b, int i) {
        const int k = (wave + i * W) * 32 + g * 8;
        b.load(w, k < a.H && col < N ? k * pitch + 2 * col : kOutOfRange, pitch);
        b.x = load16(x, k < a.H && mine ? 2u * (n * a.H + k) : kOutOfRange);
      },
      [&](const Bf16Step& b, int) {
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] = mfma(b.x, b.column(c), acc[c]);
      });
#pragma unroll
  for (int c = 0; c < 4; ++c) put_column(lds[wave], 4 * n + c, acc[c]);
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * kCols / 2; i += 64 * W) {
    const int t = i / (kCols / 2), c = i % (kCols / 2), at = c / 16 * 32 + c % 16, o = tile * (kCols / 2) + c;
    if (((tokens >> t) & 1) && o < a.I)
      put_act(a, unit, t, o, swiglu<W, kCols>(lds[0][0], 16 * kCols, t, at, at + 16));
  }
  if (tile == 0) write_hit(a, unit, e, tokens);
}

// 16 outputs (their gate and their up rows), the waves taking every W-th 16 blocks of K.
// R: rows of LDS for tokens.  With more than eight tokens (kMany) those that name the expert, R
// at a time, each R another pass over the expert's codes: more than seven of sixteen are rare,
// and a row for each of sixteen leaves a CU half of the waves (11 experts of 1352 x 336, whole
// layer of 9 and 16 tokens 15.2 and 16.5 us so, 12.1 and 13.2 now; 32 of 2048 x 704 27.2 and 29.6,
// 26.2 and 29.1; 1024 x 512, top 8, 16 tokens 17.2 and 17.8; all passes on registers in one loop
// 30 and more).  One token, 6 experts of 2048 x 704: 7.3 us for 9 MB, one step a wave, that is
// the launch and a chain of loads, each waited for before the next: the own slot, the tokens' slots,
// the tokens' rows, and the codes and scales, which the two ways to load scales (load()) keep apart;
// then the sum over waves.  8 tokens, 24 experts:
// some 15 us for 37 MB.
template <int R, int W, bool kMany, bool kOdd>
__global__ void __launch_bounds__(64 * W) few_up_mx4_kernel(FewArgs a) {
  // (a wave's sums take the place of its rows, so that a CU holds four workgroups of R = 8
  // instead of three: the layer of 8 tokens, 32 experts of 1024 x 512, top 8, 19.7 -> 16.4 us;
  // with kMany they are needed while rows are)
  constexpr int kSums = 16 * 32 * (int)sizeof(float), kRows = R * kStepBytes;
  __shared__ __attribute__((aligned(16))) uint8_t lds[W][kMany ? kRows + kSums : kRows];
  static_assert(kRows >= kSums, "room for the sums");
  int unit, tile, e;
  uint32_t tokens;
  if (!begin_up(a, &unit, &tile, &e, &tokens)) return;
  const int wave = threadIdx.x >> 6, n = threadIdx.x & 15;
  uint8_t* const rows = lds[wave];
  const int KB = (a.H + kBlock - 1) / kBlock, KS = (KB + 3) / 4 * 4, col = tile * 16 + n;
  const long long codes = 2LL * a.I * KB * 16, scales = 2LL * a.I * KS;
  const Buffer wc = buffer(a.w1 + e * codes, codes), ws = buffer(a.w1_scales + e * scales, scales);
  const i32x4 rsrc = buffer_rsrc(a.x, 2LL * a.T * a.H);
  float (*const sums)[32] = (float (*)[32])(kMany ? rows + kRows : rows);
  const int row = min(n, R - 1);
  uint32_t left = tokens;
#pragma unroll 1
  do {
    // up to R tokens, those with the R lowest numbers (kMany), each in a row of its own
    uint32_t these = left;
    if (kMany) {
#pragma unroll
      for (int r = 0; r < R; ++r) left &= left - 1;
      these &= ~left;
    }
    f32x4 acc[2] = {};   // gate and up
    bool bad[2] = {};
    for (int kb0 = wave * kStepBlocks; kb0 < KB; kb0 += W * kStepBlocks) {
      Mx4Step<2> b;
      // (rows of tokens that do not name the expert hold anything: they make results that nobody takes)
      rows_read();
      int r = 0;
      for (uint32_t m = these; m; m &= m - 1, ++r) {
        const int t = __builtin_ctz(m);
        row_to_lds<kOdd>(rows + (kMany ? r : t) * kStepBytes, rsrc, a.x, t * a.H, kb0 * kBlock, a.H);
      }
#pragma unroll
      for (int m = 0; m < 2; ++m) b.load(m, wc, ws, col + m * a.I, kb0, KB, KS, col < a.I);
      waitcnt_vm<0>();
      asm volatile("" ::: "memory");
      b.align(kb0, KB, KS);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const u32x4 v = row_operand(rows, row, j, q);
#pragma unroll
          for (int m = 0; m < 2; ++m) acc[m] = mfma(v, b.eight(m, j, q), acc[m]);
        }
#pragma unroll
      for (int m = 0; m < 2; ++m) bad[m] |= b.bad(m);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) acc[m] = with_nan(acc[m], bad[m]);
    if (kMany) {
      int token[4] = {-1, -1, -1, -1};   // of the lane's rows 4 g + i
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int t = these ? __builtin_ctz(these) : -1;
        these &= these - 1;
        token[r % 4] = r / 4 == (threadIdx.x & 63) >> 4 ? t : token[r % 4];
      }
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (token[i] >= 0) sums[token[i]][16 * m + n] = acc[m][i];
    } else {
#pragma unroll
      for (int m = 0; m < 2; ++m) put_column(sums, 16 * m + n, acc[m]);
    }
  } while (kMany && left);
  __syncthreads();
  for (int i = threadIdx.x; i < 256; i += 64 * W) {
    const int t = i / 16, c = i % 16, o = tile * 16 + c;
    if (((tokens >> t) & 1) && o < a.pitch)
      put_act(a, unit, t, o, o < a.I ? swiglu<W, 32>(sums[0] - wave * (int)(sizeof(lds[0]) / 4), sizeof(lds[0]) / 4, t, c, c + 16) : 0.f);
  }
  if (tile == 0) write_hit(a, unit, e, tokens);
}

// ---- the second launch -------------------------------------------------------------------
//
// A workgroup takes a tile of out's columns through a share of the hit experts' K; the
// waves of a tile's workgroups share it evenly.  A wave adds an expert's part to its sums,
// weighted and only for the tokens that name it, before it goes on to the next; the waves'
// sums are joined in LDS, and the shares' by the last of a tile's workgroups to end, both
// in a fixed order.

// The hit experts, in the order of their units, to `hits`: the expert, and its tokens with
// the unit in the high half.  Returns how many.
template <int W>
__device__ __forceinline__ int list_hits(const FewArgs& a, int2* hits) {
  __shared__ int ends[W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int n = 0;
  for (int u0 = 0; u0 < a.units; u0 += 64 * W) {
    const int u = u0 + threadIdx.x;
    int2 h = {-1, 0};
    if (u < a.units) h = *(const int2*)&a.hits[u];
    const uint64_t m = __ballot(h.x >= 0);
    if (lane == 0) ends[wave] = __popcll(m);
    __syncthreads();
    int before = n;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      before += w < wave ? ends[w] : 0;
      n += ends[w];
    }
    if (h.x >= 0) hits[before + __popcll(m & ((1ull << lane) - 1))] = {h.x, h.y | u << 16};
    __syncthreads();
  }
  return n;
}

// A wave's steps s0 .. s1 of the n experts' `steps` each, and where they begin.
struct Part {
  int s0, s1, u, s;
  template <int W>
  static __device__ __forceinline__ Part of(int n, int steps, int share, int shares, int wave) {
    const int all = shares * W, mine = share * W + wave, total = n * steps, each = total / all, more = total - each * all;
    Part p;
    p.s0 = mine * each + min(mine, more);
    p.s1 = p.s0 + each + (mine < more);
    p.u = p.s0 / steps;
    p.s = p.s0 - p.u * steps;
    return p;
  }
};

__device__ __forceinline__ void put_out(const FewArgs& a, int t, int o, float v) {
  if (a.out16)
    ((__bf16*)a.out)[(long long)t * a.H + o] = (__bf16)v;
  else
    ((float*)a.out)[(long long)t * a.H + o] = v;
}

// The waves' sums of COLS columns from LDS, and the shares', to out.
template <int W, int COLS>
__device__ __forceinline__ void join_sums(const FewArgs& a, const float (*lds)[16][COLS], int share, int tile) {
  __shared__ bool last;
  __syncthreads();
  for (int i = threadIdx.x; i < a.T * COLS; i += 64 * W) {
    const int t = i / COLS, c = i % COLS, o = tile * COLS + c;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += lds[w][t][c];
    if (o < a.H) {
      if (a.shares == 1)
        put_out(a, t, o, v);
      else
        __hip_atomic_store(a.parts + ((long long)share * a.T + t) * a.H + o, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  if (a.shares == 1) return;
  // A share's sums have left for good before it counts itself: they are stored past the L2
  // (as agent-scope atomics), so that each wave waits for its own stores and no cache is
  // written back (a release fence by every wave took 25 us).
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0)
    last = __hip_atomic_fetch_add(a.count + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.shares - 1;
  __syncthreads();
  if (!last) return;
  for (int i = threadIdx.x; i < a.T * COLS; i += 64 * W) {
    const int t = i / COLS, c = i % COLS, o = tile * COLS + c;
    if (o >= a.H) continue;
    const float* p = a.parts + (long long)t * a.H + o;
    const long long pitch = (long long)a.T * a.H;
    float part[8], v = 0.f;   // (eight of them on their way together)
    for (int p0 = 0; p0 < a.shares; p0 += 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (p0 + i < a.shares) part[i] = __hip_atomic_load(p + (p0 + i) * pitch, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (p0 + i < a.shares) v += part[i];
    }
    put_out(a, t, o, v);
  }
}

// Up to eight tokens: rows 0 to 7 of the matrix instruction are one part of their
// activations, rows 8 to 15 the other; more tokens (kMany): an instruction for each part.  Bound
// by the stream of the weights: 16 tokens, 32 experts of 2048 x 704, 22 us for 92 MB (4.2 TB/s);
// one token, 6 experts, 7.6 us for 17 MB, where the launch, the list of the hit experts and the
// shares' join are the most of it.
template <int W, bool kMany>
__global__ void __launch_bounds__(64 * W) few_down_kernel(FewArgs a) {
  __shared__ float lds[W][16][kCols];
  __shared__ int2 hits[kMaxExperts];
  struct Step : Bf16Step {
    u32x4 rest;
  };
  const int share = blockIdx.x / a.out_tiles, tile = blockIdx.x - share * a.out_tiles;
  const int wave = threadIdx.x >> 6, n = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
  const int col = tile * kCols + 4 * n, steps = (a.I + 31) / 32;
  const int token = kMany ? n : n & 7, part = kMany ? 0 : n >> 3, row0 = kMany ? 4 * g : 4 * (g & 1);
  const Part p = Part::of<W>(list_hits<W>(a, hits), steps, share, a.shares, wave);
  f32x4 acc[4] = {}, sum[4] = {}, gate = {};
  uint32_t named = 0;   // the tokens of the four rows that name the expert
  auto load_gates = [&](int2 h) {
    named = (uint32_t)h.y >> row0;
#pragma unroll
    for (int i = 0; i < 4; ++i) gate[i] = a.hits[(uint32_t)h.y >> 16].gate[row0 + i];
  };
  int load_u = p.u, load_s = p.s, u = p.u, s = p.s;   // the places of the next load and the next products
  if (p.s0 < p.s1) {
    load_gates(hits[u]);
    run_steps<Step>(
        p.s1 - p.s0,
        [&](Step& b, int i) {
          const bool live = p.s0 + i < p.s1;
          const int2 h = hits[live ? load_u : p.u];
          const int e = __builtin_amdgcn_readfirstlane(h.x);
          const uint32_t tokens = __builtin_amdgcn_readfirstlane(h.y);
          const long long bytes = 2LL * a.I * a.H;
          const int k = load_s * 32 + g * 8;
          const bool in = live && k < a.I;
          b.load(buffer(a.w2 + e * bytes, bytes), in && col < a.H ? (uint32_t)(k * a.H + col) * 2 : kOutOfRange, 2 * a.H);
          const Buffer x = buffer(a.act + (long long)a.T * (tokens >> 16) * 2 * a.pitch, 4LL * a.T * a.pitch);
          const uint32_t at = in && ((tokens >> token) & 1) ? 2u * ((2 * token + part) * a.pitch + k) : kOutOfRange;
          b.x = load16(x, at);
          if (kMany) b.rest = load16(x, at + 2 * a.pitch);
          if (++load_s == steps) load_s = 0, ++load_u;
        },
        [&](const Step& b, int i) {
          const int at = p.s0 + i;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const u32x4 w = b.column(c);
            acc[c] = mfma(b.x, w, acc[c]);
            if (kMany) acc[c] = mfma(b.rest, w, acc[c]);
          }
          if (at < p.s1 && (s + 1 == steps || at + 1 == p.s1)) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                sum[c][j] = (named >> j) & 1 ? fmaf(gate[j], acc[c][j], sum[c][j]) : sum[c][j];
                acc[c][j] = 0.f;
              }
            if (at + 1 < p.s1) load_gates(hits[u + 1]);
          }
          if (++s == steps) s = 0, ++u;
        });
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    if (!kMany) {   // the other part's sums are 32 lanes away
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[c][i] += __shfl_xor(sum[c][i], 32);
    }
    if (kMany || g < 2) put_column(lds[wave], 4 * n + c, sum[c]);
  }
  join_sums<W>(a, lds, share, tile);
}

// Weights in mx4: 16 columns, a wave's step as in the first launch.  R tokens (up to eight)
// at a time, rows 0 to 7 of the matrix instruction one part of their activations and rows 8
// to 15 the other: the tokens that name the expert, one after the other, so that more than R
// of them, which take another pass over the codes that are there, are rare.  16 tokens, 32
// experts of 2048 x 704: 13.7 us for 25 MB, one token 5.6 us: bound by latency, one to four steps
// a wave between the list and the join, each waiting for its codes and scales before it asks for the
// tokens' rows (the next step's codes under way while a step is worked
// on: equal, the other waves hide it).
template <int R, int W, int kPasses>
__global__ void __launch_bounds__(64 * W) few_down_mx4_kernel(FewArgs a) {
  __shared__ float lds[W][16][16];
  __shared__ int2 hits[kMaxExperts];
  __shared__ __attribute__((aligned(16))) uint8_t rows[W][2 * R * kStepBytes];
  const int share = blockIdx.x / a.out_tiles, tile = blockIdx.x - share * a.out_tiles;
  const int wave = threadIdx.x >> 6, n = threadIdx.x & 15, g = (threadIdx.x & 63) >> 4;
  const int KB = a.pitch / kBlock, KS = (KB + 3) / 4 * 4, col = tile * 16 + n;
  const int steps = (KB + kStepBlocks - 1) / kStepBlocks;
  const int row = min(n & 7, R - 1) + (n >> 3) * R;   // of LDS, of this lane's operands
  const long long codes = 16LL * a.H * KB, scales = (long long)a.H * KS;
  const Part p = Part::of<W>(list_hits<W>(a, hits), steps, share, a.shares, wave);
#pragma unroll
  for (int i = 0; i < 4; ++i) lds[wave][4 * g + i][n] = 0.f;
  f32x4 acc[kPasses] = {};
  bool bad = false;
  int u = p.u, s = p.s;
  for (int at = p.s0; at < p.s1; ++at) {
    const int2 h = hits[u];
    const int e = __builtin_amdgcn_readfirstlane(h.x), kb0 = s * kStepBlocks;
    const uint32_t tokens = __builtin_amdgcn_readfirstlane(h.y), unit = tokens >> 16;
    const __bf16* x = a.act + (long long)a.T * unit * 2 * a.pitch;
    const i32x4 rsrc = buffer_rsrc(x, 4LL * a.T * a.pitch);
    Mx4Step<1> b;
    b.load(0, buffer(a.w2 + e * codes, codes), buffer(a.w2_scales + e * scales, scales), col, kb0, KB, KS, col < a.H);
    const bool ends = s + 1 == steps || at + 1 == p.s1;
    uint32_t m = tokens & 0xffff;
#pragma unroll
    for (int pass = 0; pass < kPasses; ++pass) {
      if (m == 0) break;
      rows_read();
      // the pass's tokens, each also in the lanes that have its results (rows 4 g + i, g < 2)
      int token[4] = {0, 0, 0, 0};
      uint32_t there = 0;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (m == 0) break;
        const int t = __builtin_ctz(m);
        m &= m - 1;
        row_to_lds<false>(rows[wave] + r * kStepBytes, rsrc, x, 2 * t * a.pitch, kb0 * kBlock, a.pitch);
        row_to_lds<false>(rows[wave] + (R + r) * kStepBytes, rsrc, x, (2 * t + 1) * a.pitch, kb0 * kBlock, a.pitch);
        token[r % 4] = r / 4 == (g & 1) ? t : token[r % 4];
        there |= 1u << r;
      }
      float gate[4];
      if (ends) {
#pragma unroll
        for (int i = 0; i < 4; ++i) gate[i] = a.hits[unit].gate[token[i]];
      }
      waitcnt_vm<0>();
      asm volatile("" ::: "memory");
      if (pass == 0) b.align(kb0, KB, KS);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[pass] = mfma(row_operand(rows[wave], row, j, q), b.eight(0, j, q), acc[pass]);
      if (pass == 0) bad |= b.bad(0);
      if (ends) {
        const f32x4 v = with_nan(acc[pass], bad);
        acc[pass] = f32x4{};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float both = v[i] + __shfl_xor(v[i], 32);   // the other part's
          if (g < 2 && ((there >> (4 * g + i)) & 1)) lds[wave][token[i]][n] = fmaf(gate[i], both, lds[wave][token[i]][n]);
        }
      }
    }
    if (ends) bad = false;
    if (++s == steps) s = 0, ++u;
  }
  join_sums<W>(a, lds, share, tile);
}

// ---- host ----------------------------------------------------------------------------------

int act_pitch(int I) { return (I + kBlock - 1) / kBlock * kBlock; }
size_t up16(size_t n) { return (n + 15) / 16 * 16; }

// The second launch: columns of a tile, waves of a workgroup, and the shares of a tile's
// work: as many as there are CUs for, while every wave keeps a step.  (us, 32 experts, top 6,
// 2048 x 704: bf16, one token 12.6, 9.6, 7.8, 7.6 with 1, 2, 4, 8 shares, 16 tokens 96, 54, 31,
// 22; mx4, 16 tokens 17.7 and 13.7 with 1 and 2.)  Sixteen only with four steps a wave, and
// slots enough that most units are hit: the whole layer, 32 experts, top 8, 1024 x 512 in bf16,
// with 8 and 16: one token 13.7 and 15.5, five 21.6 and 22.7, eight 26.7 and 25.2, sixteen 32.9
// and 30.8.
struct Down {
  int cols, waves, tiles, shares;
};
Down down_of(bool mx4, int T, int H, int I, int units, int topk) {
  Down d;
  d.cols = mx4 ? 16 : kCols;
  d.waves = mx4 && T <= 4 ? 16 : 8;
  d.tiles = (H + d.cols - 1) / d.cols;
  const int k = mx4 ? kStepK : 32;
  const long long steps = (long long)units * ((I + k - 1) / k);
  d.shares = 1;
  while (d.shares < 8 && 2 * d.shares * d.tiles <= 256 && steps >= 2 * d.shares * d.waves) d.shares *= 2;
  if (d.shares == 8 && 16 * d.tiles <= 256 && steps >= 64 * d.waves && T * topk >= 2 * units) d.shares = kMaxShares;
  return d;
}

// Scratch: the units, the activations, the shares' counts and their sums.
struct Layout {
  size_t act, count, parts, bytes;
};
Layout layout_of(int T, int H, int I, int E, int topk) {
  const size_t units = T * topk < E ? T * topk : E;
  Layout l;
  l.act = up16(units * sizeof(Hit));
  l.count = l.act + up16(units * T * 2 * act_pitch(I) * sizeof(__bf16));
  l.parts = l.count + up16((size_t)(H + 15) / 16 * sizeof(uint32_t));
  size_t parts = 0;
  for (const bool mx4 : {false, true}) {
    const Down d = down_of(mx4, T, H, I, (int)units, topk);
    const size_t n = d.shares > 1 ? (size_t)d.shares * T * H * sizeof(float) : 0;
    parts = n > parts ? n : parts;
  }
  l.bytes = l.parts + up16(parts);
  return l;
}

int few(bool mx4, const void* hidden, const void* w1, const void* w1_scales, const void* w2, const void* w2_scales,
        const int32_t* ids, const float* gates, void* out, int32_t T, int32_t H, int32_t I, int32_t E, int32_t topk,
        int32_t first, int32_t out_type, void* scratch, size_t scratch_bytes, void* stream) {
  if (T < 0 || H < 1 || I < 1 || E < 1 || topk < 1 || !type_ok(out_type)) return MOE_ERR_INVALID_ARG;
  if (T > MOE_FEW_TOKENS || topk > kMaxTopk || E > kMaxExperts || H > kMaxWidth || I > kMaxWidth)
    return MOE_ERR_UNSUPPORTED;
  if (!mx4 && (H % 8 || I % 16 || 4LL * H * I > INT32_MAX)) return MOE_ERR_UNSUPPORTED;
  const long long kb1 = (H + 31LL) / 32, kb2 = (I + 31LL) / 32;
  if (mx4 && (32LL * I * kb1 > INT32_MAX || 16LL * H * kb2 > INT32_MAX)) return MOE_ERR_UNSUPPORTED;
  const int units = T * topk < E ? T * topk : E;
  // (a launch holds fewer than 2^32 threads)
  if ((long long)units * (act_pitch(I) / 16) > (1 << 22)) return MOE_ERR_UNSUPPORTED;
  if (T == 0) return MOE_OK;
  if (!hidden || !w1 || !w2 || !ids || !gates || !out || (mx4 && (!w1_scales || !w2_scales))) return MOE_ERR_INVALID_ARG;
  const Layout l = layout_of(T, H, I, E, topk);
  if (!scratch || scratch_bytes < l.bytes) return MOE_ERR_WORKSPACE;
  if (!aligned(hidden, 16) || !aligned(w1, 16) || !aligned(w2, 16) || !aligned(ids, 4) || !aligned(gates, 4) ||
      !aligned(out, type_size(out_type)) || !aligned(scratch, 16))
    return MOE_ERR_ALIGNMENT;
  if (mx4 && (!aligned(w1_scales, 4) || !aligned(w2_scales, 4))) return MOE_ERR_ALIGNMENT;
  for (const void* in : {hidden, w1, w1_scales, w2, w2_scales, (const void*)ids, (const void*)gates, (const void*)scratch})
    if (out == in) return MOE_ERR_INVALID_ARG;
  FewArgs a = {};
  a.x = (const __bf16*)hidden;
  a.w1 = (const uint8_t*)w1, a.w1_scales = (const uint8_t*)w1_scales;
  a.w2 = (const uint8_t*)w2, a.w2_scales = (const uint8_t*)w2_scales;
  a.ids = ids, a.gates = gates, a.out = out;
  a.hits = (Hit*)scratch;
  a.act = (__bf16*)((char*)scratch + l.act);
  a.count = (uint32_t*)((char*)scratch + l.count);
  a.parts = (float*)((char*)scratch + l.parts);
  a.T = T, a.H = H, a.I = I, a.E = E, a.topk = topk, a.first = first;
  a.slots = T * topk, a.units = units, a.pitch = act_pitch(I), a.out16 = out_type == MOE_BF16;
  const Down d = down_of(mx4, T, H, I, units, topk);
  a.out_tiles = d.tiles, a.shares = d.shares;
  const hipStream_t s = (hipStream_t)stream;
  // Variants by the rows that tokens take in LDS, which bounds how many waves a CU holds; seven
  // with the sums beside them are what four workgroups of the first launch have room for.
  const bool odd = H % kBlock != 0;
  if (!mx4) {
    a.tiles = (2 * I + kCols - 1) / kCols;
    few_up_kernel<8><<<(unsigned)(units * a.tiles), 64 * 8, 0, s>>>(a);
  } else {
    a.tiles = a.pitch / 16;
    auto up = T <= 4   ? (odd ? few_up_mx4_kernel<4, 4, false, true> : few_up_mx4_kernel<4, 4, false, false>)
              : T <= 8 ? (odd ? few_up_mx4_kernel<8, 4, false, true> : few_up_mx4_kernel<8, 4, false, false>)
                       : (odd ? few_up_mx4_kernel<7, 4, true, true> : few_up_mx4_kernel<7, 4, true, false>);
    up<<<(unsigned)(units * a.tiles), 64 * 4, 0, s>>>(a);
  }
  if (hipGetLastError() != hipSuccess) return MOE_ERR_HIP;
  auto down = !mx4     ? (T <= 8 ? few_down_kernel<8, false> : few_down_kernel<8, true>)
              : T <= 4 ? few_down_mx4_kernel<4, 16, 1>
              : T <= 8 ? few_down_mx4_kernel<8, 8, 1>
                       : few_down_mx4_kernel<8, 8, 2>;
  down<<<(unsigned)(d.tiles * d.shares), 64 * d.waves, 0, s>>>(a);
  return done();
}

}  // namespace

extern "C" size_t moe_few_scratch_size(int32_t T, int32_t H, int32_t I, int32_t E, int32_t topk) {
  if (T < 1 || T > MOE_FEW_TOKENS || H < 1 || H > kMaxWidth || I < 1 || I > kMaxWidth || E < 1 || E > kMaxExperts ||
      topk < 1 || topk > kMaxTopk)
    return 0;
  return layout_of(T, H, I, E, topk).bytes;
}

extern "C" int moe_few_forward(const void* hidden, const void* w1, const void* w2, const int32_t* ids,
                               const float* gates, void* out, int32_t T, int32_t H, int32_t I, int32_t E,
                               int32_t topk, int32_t first_expert, int32_t out_type, void* scratch,
                               size_t scratch_bytes, void* stream) {
  return few(false, hidden, w1, nullptr, w2, nullptr, ids, gates, out, T, H, I, E, topk, first_expert, out_type, scratch,
             scratch_bytes, stream);
}

extern "C" int moe_few_forward_mx4(const void* hidden, const void* w1_codes, const void* w1_scales,
                                   const void* w2_codes, const void* w2_scales, const int32_t* ids,
                                   const float* gates, void* out, int32_t T, int32_t H, int32_t I, int32_t E,
                                   int32_t topk, int32_t first_expert, int32_t out_type, void* scratch,
                                   size_t scratch_bytes, void* stream) {
  return few(true, hidden, w1_codes, w1_scales, w2_codes, w2_scales, ids, gates, out, T, H, I, E, topk, first_expert,
             out_type, scratch, scratch_bytes, stream);
}
