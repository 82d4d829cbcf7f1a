// The post-router layer for a few tokens in two launches, for gfx950 (C ABI: moe_block.h).
//
// A token's row is a row of the 16x16x32 matrix instruction, so one instruction
// takes all tokens through 32 of K and 16 columns of an expert's weights.  Weights go
// straight from memory to registers, each read once, with no stop in LDS: what bounds the
// layer is their stream, and the first launch's loads need nothing but the choice itself.
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "call_checks.h"
#include "moe_block.h"

namespace {

constexpr int kMaxTopk = 64, kMaxExperts = 1024;
constexpr int kMaxSlots = MOE_FEW_TOKENS * kMaxTopk;
constexpr int kMaxWidth = 1 << 22;   // H and I
constexpr int kBlock = 32;   // elements of an mx4 block

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_2 __attribute__((ext_vector_type(4), aligned(2)));

// What the first launch leaves for the second: the hit experts in the order of their
// first slots, and for each token that names one the row of its activation (the first of
// its slots that does) and the sum of their gates, in slot order.
struct Hit {
  int32_t e, pad[3];
  int32_t row[MOE_FEW_TOKENS];   // or -1
  float gate[MOE_FEW_TOKENS];
};
struct Plan {
  int32_t n, pad[15];
  Hit hit[1];
};

struct FewArgs {
  const __bf16* x;
  const uint8_t *w1, *w1_scales, *w2, *w2_scales;   // bf16 or codes
  const int32_t* ids;
  const float* gates;
  void* out;
  Plan* plan;
  __bf16* act;   // [slots][pitch]
  int T, H, I, E, topk, first, slots, pitch;
  int tiles;     // of an expert's columns (first launch)
  bool out16;
};

__device__ __forceinline__ int expert_of(const FewArgs& a, int id) {
  const int64_t e = (int64_t)id - a.first;
  return e >= 0 && e < a.E ? (int)e : -1;
}

// ---- operands ----------------------------------------------------------------------

// Eight elements of a row from k on, zeros past its end.
__device__ __forceinline__ bf16x8 row8(const __bf16* row, int k, int K) {
  u32x4 v = {0, 0, 0, 0};
  if (k + 8 <= K) {
    v = *(const u32x4_2*)(row + k);
  } else if (k < K) {
    const uint16_t* q = (const uint16_t*)row + k;
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (k + i < K) v[i / 2] |= (uint32_t)q[i] << (16 * (i % 2));
  }
  return __builtin_bit_cast(bf16x8, v);
}

// C neighbouring columns of a row of bf16 weights.
template <int C>
struct Cols {
  uint32_t d[C / 2];
};
template <int C>
__device__ __forceinline__ Cols<C> load_cols(const __bf16* p) {
  Cols<C> r;
  if constexpr (C == 8) {
    const u32x4 v = *(const u32x4*)p;
    r.d[0] = v[0], r.d[1] = v[1], r.d[2] = v[2], r.d[3] = v[3];
  } else if constexpr (C == 4) {
    const u32x2 v = *(const u32x2*)p;
    r.d[0] = v[0], r.d[1] = v[1];
  } else {
    r.d[0] = *(const uint32_t*)p;
  }
  return r;
}

// Where a lane's part of the products lies: with D > 1, the 16 rows are D times 16 / D
// tokens and the 16 columns D times 16 / D columns, each time another 32 of K: the D blocks
// on the diagonal are products (their sum is the result), the others are not used.
template <int D>
struct Lane {
  static constexpr int tokens = 16 / D;
  int l, g, at, part;   // lane, group of 8 of K, token (A) or column (B), diagonal block
  __device__ __forceinline__ Lane() {
    l = threadIdx.x & 63;
    g = l >> 4;
    at = l & (tokens - 1);
    part = (l & 15) / tokens;
  }
};

// Eight rows of K by C columns of bf16 weights, and what the matrix instruction takes of
// them: a column's eight values, by one permutation for two of them.
template <int C>
struct Weights {
  Cols<C> r[8];
  __device__ __forceinline__ void load(const __bf16* w, long long pitch, bool in) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (in) {
        r[i] = load_cols<C>(w + i * pitch);
      } else {
#pragma unroll
        for (int j = 0; j < C / 2; ++j) r[i].d[j] = 0;
      }
    }
  }
  __device__ __forceinline__ bf16x8 column(int c) const {
    u32x4 v;
#pragma unroll
    for (int p = 0; p < 4; ++p)
      v[p] = __builtin_amdgcn_perm(r[2 * p + 1].d[c / 2], r[2 * p].d[c / 2], c % 2 ? 0x07060302u : 0x05040100u);
    return __builtin_bit_cast(bf16x8, v);
  }
};

// A block of 32 mx4 values as four operands of eight (what a code stands for is exact in
// bf16).
struct Block {
  u32x4 codes;
  uint32_t byte;
  __device__ __forceinline__ void load(const uint8_t* c, const uint8_t* s, bool in) {
    codes = {0, 0, 0, 0};
    byte = 0;
    if (in) {
      codes = *(const u32x4*)c;
      byte = *s;
    }
  }
  __device__ __forceinline__ bf16x8 eight(int q) const {
    const float s = __uint_as_float(byte == 0 ? 0x00400000u : byte << 23);
    const bf16x2 p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[q], s, 0),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[q], s, 1),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[q], s, 2),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[q], s, 3)};
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = byte == 255 ? 0x7fc07fc0u : __builtin_bit_cast(uint32_t, p[i]);
    return __builtin_bit_cast(bf16x8, v);
  }
};

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// ---- the first launch ------------------------------------------------------------------

// The plan, by the launch's last workgroup.
__device__ void make_plan(const FewArgs& a) {
  __shared__ int32_t ids[kMaxSlots], index[kMaxExperts];
  __shared__ float gates[kMaxSlots];
  __shared__ int n;
  const int tid = threadIdx.x, threads = blockDim.x;
  for (int e = tid; e < a.E; e += threads) index[e] = INT32_MAX;
  for (int s = tid; s < a.slots; s += threads) {
    ids[s] = expert_of(a, a.ids[s]);
    gates[s] = a.gates[s];
  }
  __syncthreads();
  for (int s = tid; s < a.slots; s += threads)
    if (ids[s] >= 0) atomicMin(&index[ids[s]], s);
  __syncthreads();
  if (tid < 64) {   // the experts in the order of their first slots
    int at = 0;
    for (int s0 = 0; s0 < a.slots; s0 += 64) {
      const int s = s0 + tid, e = s < a.slots ? ids[s] : -1;
      const bool leads = e >= 0 && index[e] == s;
      const uint64_t m = __ballot(leads);
      if (leads) a.plan->hit[at + __popcll(m & ((1ull << tid) - 1))].e = e;
      at += __popcll(m);
    }
    if (tid == 0) a.plan->n = n = at;
  }
  __syncthreads();
  // (a leader's place again, by counting, where its token's rows and gates are filled in)
  for (int i = tid; i < n * MOE_FEW_TOKENS; i += threads) {
    Hit* h = &a.plan->hit[i / MOE_FEW_TOKENS];
    const int t = i % MOE_FEW_TOKENS, e = h->e;
    int row = -1;
    float g = 0.f;
    if (t < a.T)
      for (int j = 0; j < a.topk; ++j)
        if (ids[t * a.topk + j] == e) {
          row = row < 0 ? t * a.topk + j : row;
          g += gates[t * a.topk + j];
        }
    h->row[t] = row;
    h->gate[t] = g;
  }
}

// A workgroup's expert and tile; the rows of the activation that its tokens have in
// it (lane t of each wave; -1: not this expert's).  False: nothing to do.
__device__ __forceinline__ bool few_unit(const FewArgs& a, int* e, int* tile, int* row) {
  const int lane = threadIdx.x & 63;
  const int u = blockIdx.x / a.tiles;
  *tile = blockIdx.x - u * a.tiles;
  const bool by_slot = a.slots <= a.E;
  *e = by_slot ? expert_of(a, a.ids[u]) : u;
  if (*e < 0) return false;
  if (by_slot) {   // the first slot that names the expert has it
    bool other = false;
    for (int s = lane; s < u; s += 64) other |= expert_of(a, a.ids[s]) == *e;
    if (__ballot(other)) return false;
  }
  *row = -1;
  if (lane < a.T)
    for (int j = a.topk - 1; j >= 0; --j)
      if (expert_of(a, a.ids[lane * a.topk + j]) == *e) *row = lane * a.topk + j;
  return __ballot(*row >= 0) != 0;
}

template <int D>
__device__ __forceinline__ float swiglu_sum(const float* lds, int parts, int pitch, int g, int u) {
  float x = 0.f, y = 0.f;
  for (int p = 0; p < parts; ++p) {
    x += lds[p * pitch + g];
    y += lds[p * pitch + u];
  }
  return x / (1.f + expf(-x)) * y;
}

template <int C, int D, int W>
__global__ void __launch_bounds__(64 * W) few_up_kernel(FewArgs a) {
  if (blockIdx.x == gridDim.x - 1) return make_plan(a);
  constexpr int TOK = 16 / D, COLS = TOK * C;
  __shared__ float lds[W * D][TOK][COLS];
  __shared__ int rows[64];
  int e, tile, row;
  if (!few_unit(a, &e, &tile, &row)) return;
  if (threadIdx.x < 64) rows[threadIdx.x] = row;
  const Lane<D> ln;
  const int wave = threadIdx.x >> 6, N = 2 * a.I;
  const int mine = __shfl(row, ln.at);   // of this lane's token
  const __bf16* x = a.x + (long long)ln.at * a.H;
  const int col = tile * COLS + ln.at * C;
  const __bf16* w = (const __bf16*)a.w1 + (long long)e * a.H * N + col;
  f32x4 acc[C] = {};
  const int steps = (a.H + 32 * D - 1) / (32 * D);
  for (int s = wave; s < steps; s += W) {
    const int k = (s * D + ln.part) * 32 + ln.g * 8;
    Weights<C> b;
    b.load(w + (long long)k * N, N, k < a.H && col < N);
    bf16x8 v = {};
    if (mine >= 0) v = row8(x, k, a.H);
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] = mfma(v, b.column(c), acc[c]);
  }
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * ln.g + i;
      if (r / TOK == ln.part) lds[wave * D + ln.part][r % TOK][ln.at * C + c] = acc[c][i];
    }
  __syncthreads();
  for (int i = threadIdx.x; i < TOK * COLS / 2; i += 64 * W) {
    const int t = i / (COLS / 2), c = i % (COLS / 2), at = c / 16 * 32 + c % 16;
    const float v = swiglu_sum<D>(&lds[0][t][0], W * D, TOK * COLS, at, at + 16);
    const int r = rows[t];
    const int o = tile * (COLS / 2) + c;
    if (r >= 0 && o < a.I) a.act[(long long)r * a.pitch + o] = (__bf16)v;
  }
}

// Weights in mx4: TOK outputs a workgroup, their gate and their up rows.
template <int D, int W>
__global__ void __launch_bounds__(64 * W) few_up_mx4_kernel(FewArgs a) {
  if (blockIdx.x == gridDim.x - 1) return make_plan(a);
  constexpr int TOK = 16 / D;
  __shared__ float lds[W * D][TOK][2 * TOK];
  __shared__ int rows[64];
  int e, tile, row;
  if (!few_unit(a, &e, &tile, &row)) return;
  if (threadIdx.x < 64) rows[threadIdx.x] = row;
  const Lane<D> ln;
  const int wave = threadIdx.x >> 6;
  const int KB = (a.H + kBlock - 1) / kBlock, KS = (KB + 3) / 4 * 4;
  const int mine = __shfl(row, ln.at);
  const __bf16* x = a.x + (long long)ln.at * a.H;
  const int col = tile * TOK + ln.at;
  const long long rg = (long long)e * 2 * a.I + col, ru = rg + a.I;
  f32x4 ag = {}, au = {};
  const int steps = (KB + 4 * D - 1) / (4 * D);
  for (int s = wave; s < steps; s += W) {
    const int kb = (s * D + ln.part) * 4 + ln.g;
    const bool in = kb < KB && col < a.I;
    Block bg, bu;
    bg.load(a.w1 + (rg * KB + kb) * 16, a.w1_scales + rg * KS + kb, in);
    bu.load(a.w1 + (ru * KB + kb) * 16, a.w1_scales + ru * KS + kb, in);
    bf16x8 v[4] = {};
    if (mine >= 0) {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = row8(x, kb * kBlock + 8 * q, a.H);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      ag = mfma(v[q], bg.eight(q), ag);
      au = mfma(v[q], bu.eight(q), au);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 4 * ln.g + i;
    if (r / TOK == ln.part) {
      lds[wave * D + ln.part][r % TOK][ln.at] = ag[i];
      lds[wave * D + ln.part][r % TOK][TOK + ln.at] = au[i];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < TOK * TOK; i += 64 * W) {
    const int t = i / TOK, c = i % TOK;
    const float v = swiglu_sum<D>(&lds[0][t][0], W * D, 2 * TOK * TOK, c, TOK + c);
    const int r = rows[t];
    const int o = tile * TOK + c;
    if (r >= 0 && o < a.pitch) a.act[(long long)r * a.pitch + o] = (__bf16)(o < a.I ? v : 0.f);
  }
}

// ---- the second launch -------------------------------------------------------------------
//
// A workgroup takes a tile of out's columns through every hit expert; its waves share the
// experts' K.  A wave adds an expert's part to its sums, weighted and only for the tokens
// that name it, before it goes on to the next; the waves' sums are joined in LDS, in order.
template <int C, int D, int W, bool kMx4>
__global__ void __launch_bounds__(64 * W) few_down_kernel(FewArgs a) {
  constexpr int TOK = 16 / D, COLS = TOK * C;
  __shared__ float lds[W * D][TOK][COLS];
  const Lane<D> ln;
  const int wave = threadIdx.x >> 6;
  const int col = blockIdx.x * COLS + ln.at * C;
  const int KB = (a.I + kBlock - 1) / kBlock, KS = (KB + 3) / 4 * 4;
  const int steps = kMx4 ? (KB + 4 * D - 1) / (4 * D) : (a.I + 32 * D - 1) / (32 * D);
  const int n = a.plan->n;
  const int s0 = (int)((long long)n * steps * wave / W), s1 = (int)((long long)n * steps * (wave + 1) / W);
  f32x4 acc[C] = {}, sum[C] = {};
  int u = s0 / steps, s = s0 - u * steps;
  for (int at = s0; at < s1; ++at) {
    const Hit* h = &a.plan->hit[u];
    const int e = h->e, row = h->row[ln.at];
    const __bf16* x = a.act + (long long)row * a.pitch;
    if constexpr (kMx4) {
      const int kb = (s * D + ln.part) * 4 + ln.g;
      const long long r = (long long)e * a.H + col;
      Block b;
      b.load(a.w2 + (r * KB + kb) * 16, a.w2_scales + r * KS + kb, kb < KB && col < a.H);
      bf16x8 v[4] = {};
      if (row >= 0 && kb < KB) {
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = row8(x, kb * kBlock + 8 * q, a.pitch);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[0] = mfma(v[q], b.eight(q), acc[0]);
    } else {
      const int k = (s * D + ln.part) * 32 + ln.g * 8;
      Weights<C> b;
      b.load((const __bf16*)a.w2 + ((long long)e * a.I + k) * a.H + col, a.H, k < a.I && col < a.H);
      bf16x8 v = {};
      if (row >= 0) v = row8(x, k, a.I);
#pragma unroll
      for (int c = 0; c < C; ++c) acc[c] = mfma(v, b.column(c), acc[c]);
    }
    if (++s == steps || at + 1 == s1) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int t = (4 * ln.g + i) % TOK;
        const bool on = h->row[t] >= 0;
        const float g = h->gate[t];
#pragma unroll
        for (int c = 0; c < C; ++c) {
          sum[c][i] = on ? fmaf(g, acc[c][i], sum[c][i]) : sum[c][i];
          acc[c][i] = 0.f;
        }
      }
      s = 0;
      ++u;
    }
  }
#pragma unroll
  for (int c = 0; c < C; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * ln.g + i;
      if (r / TOK == ln.part) lds[wave * D + ln.part][r % TOK][ln.at * C + c] = sum[c][i];
    }
  __syncthreads();
  for (int i = threadIdx.x; i < TOK * COLS; i += 64 * W) {
    const int t = i / COLS, c = i % COLS, o = blockIdx.x * COLS + c;
    float v = 0.f;
    for (int p = 0; p < W * D; ++p) v += lds[p][t][c];
    if (t < a.T && o < a.H) {
      if (a.out16)
        ((__bf16*)a.out)[(long long)t * a.H + o] = (__bf16)v;
      else
        ((float*)a.out)[(long long)t * a.H + o] = v;
    }
  }
}

// ---- host ----------------------------------------------------------------------------------

size_t plan_bytes(int slots) {
  return sizeof(Plan) - sizeof(Hit) + sizeof(Hit) * (size_t)(slots < kMaxExperts ? slots : kMaxExperts);
}
int act_pitch(int I) { return (I + kBlock - 1) / kBlock * kBlock; }

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
  if (!scratch || scratch_bytes < moe_few_scratch_size(T, I, topk)) return MOE_ERR_WORKSPACE;
  if (!aligned(hidden, 2) || !aligned(w1, 16) || !aligned(w2, 16) || !aligned(ids, 4) || !aligned(gates, 4) ||
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
  a.plan = (Plan*)scratch;
  a.act = (__bf16*)((char*)scratch + plan_bytes(T * topk));
  a.T = T, a.H = H, a.I = I, a.E = E, a.topk = topk, a.first = first;
  a.slots = T * topk, a.pitch = act_pitch(I), a.out16 = out_type == MOE_BF16;
  const hipStream_t s = (hipStream_t)stream;
  if (mx4) {
    a.tiles = (a.pitch + 15) / 16;
    few_up_mx4_kernel<1, 8><<<(unsigned)(units * a.tiles + 1), 512, 0, s>>>(a);
    if (hipGetLastError() != hipSuccess) return MOE_ERR_HIP;
    few_down_kernel<1, 1, 16, true><<<(unsigned)((H + 15) / 16), 1024, 0, s>>>(a);
  } else {
    a.tiles = (2 * I + 31) / 32;
    few_up_kernel<2, 1, 8><<<(unsigned)(units * a.tiles + 1), 512, 0, s>>>(a);
    if (hipGetLastError() != hipSuccess) return MOE_ERR_HIP;
    few_down_kernel<2, 1, 16, false><<<(unsigned)((H + 31) / 32), 1024, 0, s>>>(a);
  }
  return done();
}

}  // namespace

extern "C" size_t moe_few_scratch_size(int32_t T, int32_t I, int32_t topk) {
  if (T < 1 || T > MOE_FEW_TOKENS || I < 1 || I > kMaxWidth || topk < 1 || topk > kMaxTopk) return 0;
  return plan_bytes(T * topk) + (size_t)T * topk * act_pitch(I) * sizeof(__bf16);
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
