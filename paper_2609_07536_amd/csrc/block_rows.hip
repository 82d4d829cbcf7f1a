// The router's choice, and the residual join with the norms on both sides, with
// their gradients, for gfx950 (C ABI: moe_block.h).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstddef>
#include <cstdint>

#include "call_checks.h"
#include "moe_block.h"
#include "status_bits.h"

namespace {

// ---- sums and maxima over lanes ------------------------------------------------
//
// Within rows of 16 lanes by data-parallel primitives (exchanges with the lane 1 and 2
// away, then the mirrored half row and row: every lane ends up with the result), over
// the rows of a wave by shuffles.  The order is fixed.
template <int kCtrl>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), kCtrl, 0xf, 0xf, true));
}
template <int kCtrl>
__device__ __forceinline__ int dpp(int v) {
  return __builtin_amdgcn_update_dpp(0, v, kCtrl, 0xf, 0xf, true);
}
template <int L, class T, class Op>
__device__ __forceinline__ T over_lanes(T v, Op op) {
  v = op(v, dpp<0xb1>(v));                     // quad_perm 1 0 3 2
  v = op(v, dpp<0x4e>(v));                     // quad_perm 2 3 0 1
  if (L >= 8) v = op(v, dpp<0x141>(v));        // row_half_mirror
  if (L >= 16) v = op(v, dpp<0x140>(v));       // row_mirror
  if (L >= 64) {
    v = op(v, __shfl_xor(v, 16));
    v = op(v, __shfl_xor(v, 32));
  }
  return v;
}
template <int L>
__device__ __forceinline__ float sum_of(float v) {
  return over_lanes<L>(v, [](float a, float b) { return a + b; });
}
template <int L>
__device__ __forceinline__ float max_of(float v) {
  return over_lanes<L>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int L>
__device__ __forceinline__ int min_of(int v) {
  return over_lanes<L>(v, [](int a, int b) { return min(a, b); });
}

// ---- the router's choice ---------------------------------------------------------
//
// L lanes take a token, R logits each in chunks of four (16 bytes of fp32): lane l
// holds experts 4 (q L + l) + i.  A slot is the group's largest key, then the lowest
// expert that has it; its lane notes the slot and strikes the key out.
constexpr float kNone = -__builtin_inff();
constexpr int kMaxTopk = 64, kMaxExperts = 1024;

template <class T, int L, int R>
__device__ __forceinline__ void load_logits(const T* p, int E, int l, float (&v)[R]) {
  typedef T mem __attribute__((ext_vector_type(4), aligned(sizeof(T))));
#pragma unroll
  for (int q = 0; q < R / 4; ++q) {
    const int e = 4 * (q * L + l);
    if (e + 4 <= E) {
      const mem m = *(const mem*)(p + e);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * q + i] = (float)m[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * q + i] = e + i < E ? (float)p[e + i] : kNone;
    }
  }
}

__device__ __forceinline__ float sigmoid(float x) { return 1.f / (1.f + expf(-x)); }

// A float's bits in an order that integers compare by (NaN aside).
__device__ __forceinline__ int ordered(float v) {
  const int b = __float_as_int(v);
  return b ^ ((b >> 31) & 0x7fffffff);
}

// Bound by the instructions of the rounds: for each logit of a lane two comparisons and two
// selections (16384 tokens, 8 of 256 experts by sixteen lanes a token: a call takes 10.8 us,
// of which the launch and 18 MB are some 5, and 9.3 of bf16 logits; by eight lanes 11.2; a
// threshold found bit by bit over a wave's counts 15).  The chosen go through LDS to the lanes
// that take their scores: slot j is lane j % L's.
template <class T, int L, int R>
__global__ void __launch_bounds__(256) choose_kernel(const T* logits, const float* bias, int32_t* ids, float* gates,
                                                     long long first, int tokens, int E, int topk, bool softmax,
                                                     bool renorm, float scale) {
  __shared__ int32_t lds_id[256 / L][kMaxTopk];
  __shared__ float lds_x[256 / L][kMaxTopk];
  const int l = threadIdx.x % L, group = threadIdx.x / L;
  const long long t0 = first + (long long)blockIdx.x * (256 / L) + group;
  const bool in = t0 < tokens, all = softmax && !renorm;
  const long long t = in ? t0 : tokens - 1;   // (groups past the last token do its work again, and write nothing)
  float v[R], b[R];
  load_logits<T, L, R>(logits + t * E, E, l, v);
  if (bias) load_logits<float, L, R>(bias, E, l, b);
  float shift = kNone, sum = 0.f;
  if (all) {   // (kNone, which is past E too, adds nothing)
#pragma unroll
    for (int r = 0; r < R; ++r) shift = fmaxf(shift, v[r]);
    shift = max_of<L>(shift);
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (v[r] != kNone) sum += expf(v[r] - shift);
  }
  const int none = ordered(kNone);
  int key[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float k = (bias ? v[r] + b[r] : v[r]) + 0.f;   // (+ 0: -0 and 0 are equal)
    key[r] = k > kNone ? ordered(k) : none;
  }
  for (int j = l; j < topk; j += L) lds_id[group][j] = -1;
  for (int n = 0; n < topk; ++n) {
    int best = key[0];
#pragma unroll
    for (int r = 1; r < R; ++r) best = max(best, key[r]);
    best = over_lanes<L>(best, [](int x, int y) { return max(x, y); });
    const uint64_t live = __ballot(best > none);
    if (live == 0) break;   // no token of the wave has another
    int e = INT32_MAX;
#pragma unroll
    for (int r = R - 1; r >= 0; --r) e = key[r] == best ? 4 * (r / 4 * L + l) + r % 4 : e;
    e = best > none ? e : INT32_MAX;
    // more lanes than tokens have it: equal keys, of which the lower expert's goes first
    if (__popcll(__ballot(e != INT32_MAX)) * L != __popcll(live)) {
      const int least = min_of<L>(e);
      e = e == least ? e : INT32_MAX;
    }
    if (e != INT32_MAX) lds_id[group][n] = e;
#pragma unroll
    for (int r = 0; r < R; ++r) key[r] = e == 4 * (r / 4 * L + l) + r % 4 ? none : key[r];
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // (a wave reads what it wrote)
  if (!all) {
    for (int j = l; j < topk; j += L) {
      const int e = lds_id[group][j];
      const float x = e < 0 ? kNone : (float)logits[t * E + e];
      lds_x[group][j] = x;
      shift = fmaxf(shift, softmax ? x : fminf(x, 0.f));
    }
    shift = max_of<L>(shift);
  }
  for (int j = l; j < topk; j += L) {
    const int e = lds_id[group][j];
    const float x = !all ? lds_x[group][j] : e < 0 ? kNone : (float)logits[t * E + e];
    // (renormalised sigmoids by their ratio to the largest: none is lost to underflow)
    const float p = e < 0     ? 0.f
        : softmax ? expf(x - shift)
        : renorm  ? expf(fminf(x, 0.f) - shift) / (1.f + expf(-fabsf(x)))
                  : sigmoid(x);
    if (renorm) sum += p;
    lds_x[group][j] = p;
  }
  sum = sum_of<L>(sum);
  const float f = softmax || renorm ? scale / sum : scale;
  if (!in) return;
  for (int j = l; j < topk; j += L) {
    const int e = lds_id[group][j];
    ids[t * topk + j] = e;
    gates[t * topk + j] = e < 0 ? 0.f : lds_x[group][j] * f;
  }
}

// With q_j the gates over `scale`, the chosen slots' gradients g_j, and G = sum q_j g_j:
//   softmax over all e     s p_e ([e chosen] g - G)
//   renormalised softmax   s q_e (g - G), chosen e only
//   ... sigmoid            s q_e (1 - p_e) (g - G)
//   sigmoid                s p_e (1 - p_e) g
// An expert that several slots name enters by its number of slots `cnt` and their sum.
// A token's logits, and in the end its gradients, stay in the registers of its lanes.  Bound by
// latency at training's sizes (8192 tokens, 4 of 30 experts: 5.3 us for 2.2 MB, and the same for
// 1.2 MB in bf16, half of it the launch): the flag of a bad id stands between a slot's loads and
// the next one's, so that the slots' are waited for one after the other.
template <class T, int L, int R>
__global__ void __launch_bounds__(256) choose_grad_kernel(const float* dgates, const T* logits, const int32_t* ids,
                                                          T* dlogits, long long first, int tokens, int E, int topk, bool softmax,
                                                          bool renorm, float scale, uint32_t* status) {
  const int l = threadIdx.x % L;
  const long long t0 = first + (long long)blockIdx.x * (256 / L) + threadIdx.x / L;
  const bool in = t0 < tokens;
  const long long t = in ? t0 : tokens - 1;
  float v[R], g[R];
  int cnt[R];
  load_logits<T, L, R>(logits + t * E, E, l, v);
#pragma unroll
  for (int r = 0; r < R; ++r) g[r] = 0.f, cnt[r] = 0;
  int some = 0;
  for (int j = 0; j < topk; ++j) {
    const int id = ids[t * topk + j];
    const float d = dgates[t * topk + j];
    if ((id < -1 || id >= E) && status)
      __hip_atomic_fetch_or(status, kStBadRouting, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (id < 0 || id >= E) continue;
    some = 1;
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (id == 4 * (r / 4 * L + l) + r % 4) {
        g[r] += d;
        ++cnt[r];
      }
  }
  const bool all = softmax && !renorm;
  float shift = kNone, p[R], sum = 0.f, dot = 0.f;
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (all || cnt[r] > 0) shift = fmaxf(shift, softmax || !renorm ? v[r] : fminf(v[r], 0.f));
  shift = max_of<L>(shift);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int e = 4 * (r / 4 * L + l) + r % 4;
    p[r] = 0.f;
    if (all ? some && e < E : cnt[r] > 0) {
      p[r] = softmax ? expf(v[r] - shift)
             : renorm ? expf(fminf(v[r], 0.f) - shift) / (1.f + expf(-fabsf(v[r])))
                      : sigmoid(v[r]);
      sum += all ? p[r] : cnt[r] * p[r];
    }
  }
  sum = sum_of<L>(sum);
  const float inv = softmax || renorm ? (some ? 1.f / sum : 0.f) : 1.f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    p[r] *= inv;
    if (cnt[r] > 0) dot += p[r] * g[r];
  }
  dot = sum_of<L>(dot);
  if (!in) return;
  typedef T mem __attribute__((ext_vector_type(4), aligned(sizeof(T))));
#pragma unroll
  for (int q = 0; q < R / 4; ++q) {
    const int e = 4 * (q * L + l);
    float d[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * q + i;
      d[i] = 0.f;
      if (all ? some != 0 : cnt[r] > 0) {
        const float sg = softmax ? 1.f : sigmoid(-v[r]);   // 1 - p
        d[i] = all      ? p[r] * (g[r] - dot)
               : renorm ? p[r] * sg * (g[r] - cnt[r] * dot)
                        : p[r] * sg * g[r];
        d[i] *= scale;
      }
    }
    if (e + 4 <= E) {
      mem m;
#pragma unroll
      for (int i = 0; i < 4; ++i) m[i] = (T)d[i];
      *(mem*)(dlogits + t * E + e) = m;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (e + i < E) dlogits[t * E + e + i] = (T)d[i];
    }
  }
}

// ---- rows of the residual stream -----------------------------------------------------

// Eight elements of a row as they lie in memory, bf16 in `a` alone: loaded together
// whatever their types are, and converted where they are used.
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_4 __attribute__((ext_vector_type(4), aligned(4)));
struct Raw {
  u32x4 a, b;
};
// Columns c .. c + 7 of a row of H that starts at element `row`, zeros past its end.  The
// lanes at the end of a row load its last eight, and floats() shifts them down: single
// elements in a branch of their own make the wave wait there, tensor after tensor, and a
// shift right after the load makes it wait for that.  Rows of fewer than eight are left to
// floats().
__device__ __forceinline__ Raw load8(const void* p, bool bf16, long long row, int c, int H) {
  Raw r = {{0, 0, 0, 0}, {0, 0, 0, 0}};
  const int at = min(c, H - 8);
  if (c - at < 8 && at >= 0) {
    if (bf16) {
      r.a = *(const u32x4_2*)((const uint16_t*)p + row + at);
    } else {
      r.a = *(const u32x4_4*)((const uint32_t*)p + row + at);
      r.b = *(const u32x4_4*)((const uint32_t*)p + row + at + 4);
    }
  }
  return r;
}
// the same as floats, from what load8 gave for them
__device__ __forceinline__ void floats(Raw r, bool bf16, const void* p, long long row, int c, int H, float (&v)[8]) {
  if (H % 8) {   // (uniform)
    const int s = c - min(c, H - 8);
    if (H < 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        v[i] = i >= H - c ? 0.f
               : bf16     ? __uint_as_float((uint32_t)((const uint16_t*)p)[row + c + i] << 16)
                          : ((const float*)p)[row + c + i];
      return;
    }
    if (bf16) {
      if (s & 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.a[i] = r.a[i] >> 16 | (i < 3 ? r.a[(i + 1) % 4] << 16 : 0);
      }
      if (s & 2) r.a = u32x4{r.a[1], r.a[2], r.a[3], 0};
      if (s & 4) r.a = u32x4{r.a[2], r.a[3], 0, 0};
    } else {
      if (s & 1) r.a = u32x4{r.a[1], r.a[2], r.a[3], r.b[0]}, r.b = u32x4{r.b[1], r.b[2], r.b[3], 0};
      if (s & 2) r.a = u32x4{r.a[2], r.a[3], r.b[0], r.b[1]}, r.b = u32x4{r.b[2], r.b[3], 0, 0};
      if (s & 4) r.a = r.b, r.b = u32x4{0, 0, 0, 0};
    }
  }
  if (bf16) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(r.a[i] << 16);
      v[2 * i + 1] = __uint_as_float(r.a[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(i < 4 ? r.a[i % 4] : r.b[i % 4]);
  }
}
__device__ __forceinline__ void floats_of(const void* p, bool bf16, int c, int H, float (&v)[8]) {
  floats(load8(p, bf16, 0, c, H), bf16, p, 0, c, H, v);
}
__device__ __forceinline__ Raw raw(const float (&v)[8], bool bf16) {
  Raw r;
  if (bf16) {
    typedef __bf16 b16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const b16x2 h = {(__bf16)v[2 * i], (__bf16)v[2 * i + 1]};
      r.a[i] = __builtin_bit_cast(uint32_t, h);
      r.b[i] = 0;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r.a[i] = __float_as_uint(v[i]);
      r.b[i] = __float_as_uint(v[i + 4]);
    }
  }
  return r;
}
__device__ __forceinline__ void store8(void* p, bool bf16, long long at, int n, const Raw& r) {
  if (n >= 8) {
    if (bf16) {
      *(u32x4_2*)((uint16_t*)p + at) = r.a;
    } else {
      *(u32x4_4*)((uint32_t*)p + at) = r.a;
      *(u32x4_4*)((uint32_t*)p + at + 4) = r.b;
    }
  } else if (n > 0) {
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < n) {
        if (bf16)
          ((uint16_t*)p)[at + i] = (uint16_t)(r.a[i / 2] >> (16 * (i % 2)));
        else
          ((uint32_t*)p)[at + i] = i < 4 ? r.a[i % 4] : r.b[i % 4];
      }
  }
}
__device__ __forceinline__ float element(const void* p, bool bf16, long long at) {
  return bf16 ? __uint_as_float((uint32_t)((const uint16_t*)p)[at] << 16) : ((const float*)p)[at];
}

// The random words of columns 4 block .. 4 block + 3 of a row (the multipliers and key
// steps are the published ones).
__device__ __forceinline__ void philox(uint32_t block, uint32_t row, uint64_t offset, uint64_t seed, uint32_t (&w)[4]) {
  uint32_t c0 = block, c1 = row, c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  w[0] = c0, w[1] = c1, w[2] = c2, w[3] = c3;
}

struct JoinArgs {
  const void *h, *y, *after, *gate, *before, *dx, *dz;   // (the gradient: h is x, the joined stream)
  const uint64_t* rng;
  void *x, *z, *dh, *dy;
  float *d_after, *d_gate, *d_before, *parts;
  int T, H;
  bool h16, y16, z16, w16;
  int gate_kind;
  float scale, keep, eps;   // keep: 1 / (1 - p)
  uint32_t least;           // least random word of a kept element
  bool drop;
};

// x + factor drop(v), columns c .. c + 7 of row t (c a multiple of 8): where it drops x stays,
// also with a factor that is no finite number (a gate of tokens is in it).
__device__ __forceinline__ void drop8(const JoinArgs& a, uint64_t seed, uint64_t offset, long long t, int c, float factor,
                                      const float (&v)[8], float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i % 4 == 0) philox((uint32_t)(c / 4 + i / 4), (uint32_t)t, offset, seed, w);
    x[i] = w[i % 4] >= a.least ? fmaf(factor, v[i] * a.keep, x[i]) : x[i];
  }
}

// Sums of n values over a row's threads: NT, or as many waves fewer as its columns need.
template <int NT, int n>
__device__ __forceinline__ void row_sums(float (&v)[n], float* lds) {
#pragma unroll
  for (int i = 0; i < n; ++i) v[i] = sum_of<64>(v[i]);
  if (NT == 64) return;
  const int wave = threadIdx.x / 64, waves = blockDim.x / 64;
  __syncthreads();   // (the last sums have been read)
  if (threadIdx.x % 64 == 0) {
#pragma unroll
    for (int i = 0; i < n; ++i) lds[i * (NT / 64) + wave] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < n; ++i) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) s += w < waves ? lds[i * (NT / 64) + w] : 0.f;
    v[i] = s;
  }
}

// A workgroup takes a row, U chunks of eight columns a thread, all of it in registers:
// every tensor is read and written once.  Bound by memory: 16384 rows of 2048, h, x and z in
// bf16 and y in fp32, 60 us for 336 MB (5.6 TB/s; a large copy 4.9); 4096 rows of 4096, 2048 of 8192
// and 1024 of 16384, all in bf16, 29, 34 and 33 us for 134 MB.  A few rows by latency: one 2.6 us;
// 777 of 1352 with the norm after the block, a gate of tokens and dropout 5.9: the weights' loads
// and the random numbers, which wait for no sum, stand behind the sums all the same.
template <int NT, int U>
__global__ void __launch_bounds__(NT) join_kernel(JoinArgs a, long long first) {
  __shared__ float lds[NT / 64];
  const long long t = first + blockIdx.x, row = t * a.H;
  uint64_t seed = 0, offset = 0;
  Raw rh[U], ry[U];
  int n[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = 8 * (u * NT + (int)threadIdx.x);
    n[u] = min(8, a.H - c);
    if (a.y) ry[u] = load8(a.y, a.y16, row, c, a.H);
    if (a.h) rh[u] = load8(a.h, a.h16, row, c, a.H);
  }
  if (a.drop) seed = a.rng[0], offset = a.rng[1];
  float factor = a.scale;
  if (a.y && a.gate_kind == MOE_GATE_TOKEN) factor *= element(a.gate, a.w16, t);
  float r = 1.f;
  if (a.after) {
    float s[1] = {0.f};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float y[8];
      floats(ry[u], a.y16, a.y, row, 8 * (u * NT + (int)threadIdx.x), a.H, y);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] = fmaf(y[i], y[i], s[0]);
    }
    row_sums<NT>(s, lds);
    r = rsqrtf(s[0] / a.H + a.eps);
  }
  float x[U][8], s[1] = {0.f};
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = 8 * (u * NT + (int)threadIdx.x);
    if (a.h)
      floats(rh[u], a.h16, a.h, row, c, a.H, x[u]);
    else
#pragma unroll
      for (int i = 0; i < 8; ++i) x[u][i] = 0.f;
    if (a.y) {
      float v[8], w[8];
      floats(ry[u], a.y16, a.y, row, c, a.H, v);
      if (a.after) {
        floats_of(a.after, a.w16, c, a.H, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = v[i] * r * w[i];
      }
      if (a.gate_kind == MOE_GATE_CHANNEL) {
        floats_of(a.gate, a.w16, c, a.H, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= w[i];
      }
      if (a.drop)
        drop8(a, seed, offset, t, c, factor, v, x[u]);
      else
#pragma unroll
        for (int i = 0; i < 8; ++i) x[u][i] = fmaf(factor, v[i], x[u][i]);
      const Raw o = raw(x[u], a.h16);
      store8(a.x, a.h16, row + c, n[u], o);
      if (a.h16) {   // the norm's x is the one that is kept
#pragma unroll
        for (int i = 0; i < 8; ++i) x[u][i] = __uint_as_float(i % 2 ? o.a[i / 2] & 0xffff0000u : o.a[i / 2] << 16);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) s[0] = fmaf(x[u][i], x[u][i], s[0]);
  }
  if (!a.before) return;
  row_sums<NT>(s, lds);
  r = rsqrtf(s[0] / a.H + a.eps);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int c = 8 * (u * NT + (int)threadIdx.x);
    float w[8];
    floats_of(a.before, a.w16, c, a.H, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] *= x[u][i] * r;
    store8(a.z, a.z16, row + c, n[u], raw(w, a.z16));
  }
}

// The gradient: with v = dz before, r the norm's factor and D = dx + r (v - x r^2
// mean(x v)), dh = D, da = scale drop(D), db = gate da, and dy is db or, by the same
// formula, its way back through the norm after the block.  Workgroup g takes rows g,
// g + G, ..., four columns a thread (so that what a thread keeps fits its registers); its sums
// over rows of the columns' gradients go to `parts` [array][G][H] and are added up by a second
// launch, always in the same order.  Rows of up to 4096 columns keep these sums, and the weights,
// in registers, and ask for the next row before they work on one.  That row is under way
// meanwhile where all that is read is bf16; an fp32 tensor's settle() may leave loads of its own
// for the first sum over the row (rows of fewer than four columns), a bf16 gate of tokens is
// converted where it is loaded, and with either the compiler waits for all loads there.  Longer
// rows (kLong) keep the sums in LDS and load weights and columns again.  Bound by memory: 8192
// rows of 2048 in bf16 with the norm before, 33.0 us and 4.6 for the second launch, 168 MB (5.1 TB/s);
// with an fp32 stream and y 57.1 and 4.7, 302 MB (5.3).  4096 rows of 4096 in bf16 36.0 and 4.6 for the
// same 168 MB, but 2048 of 8192, whose columns come twice, 68.8 and 4.8.  777 rows of 1351 in fp32 with
// everything, 14.5 and 4.2 for 23 MB, by latency: two rows a workgroup, each waited for, with two
// sums over the row and the random numbers one after the other.
// Types are the kernel's own (B16: bf16, else fp32), so that a row is as few registers as it
// is bytes; kY: with a norm after the block or a gate (else y is not read).
template <bool B16>
struct Four;
template <>
struct Four<true> {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  typedef uint32_t u32x2_2 __attribute__((ext_vector_type(2), aligned(2)));
  u32x2 a;
  // columns c .. c + 3 of a row that starts at element `row`, as load8 and floats do it
  __device__ __forceinline__ void load(const void* p, long long row, int c, int H) {
    const int at = min(c, H - 4);
    a = u32x2{0, 0};
    if (c - at < 4 && at >= 0) a = *(const u32x2_2*)((const uint16_t*)p + row + at);
  }
  // (where the row's end is no multiple of four; the loads have to be there)
  __device__ __forceinline__ void settle(const void* p, long long row, int c, int H) {
    uint64_t v = (uint64_t)a[1] << 32 | a[0];
    if (H < 4) {
      v = 0;
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < H - c) v |= (uint64_t)((const uint16_t*)p)[row + c + i] << (16 * i);
    } else {
      v >>= 16 * ((c - min(c, H - 4)) & 3);
    }
    a = u32x2{(uint32_t)v, (uint32_t)(v >> 32)};
  }
  __device__ __forceinline__ f32x4 get() const {
    return {__uint_as_float(a[0] << 16), __uint_as_float(a[0] & 0xffff0000u), __uint_as_float(a[1] << 16),
            __uint_as_float(a[1] & 0xffff0000u)};
  }
  static __device__ __forceinline__ void put(void* p, long long at, int n, f32x4 v) {
    __bf16* q = (__bf16*)p + at;
    typedef __bf16 b16x4 __attribute__((ext_vector_type(4)));
    typedef __bf16 b16x4_2 __attribute__((ext_vector_type(4), aligned(2)));
    if (n >= 4) {
      *(b16x4_2*)q = b16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]};
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < n) q[i] = (__bf16)v[i];
    }
  }
};
template <>
struct Four<false> {
  typedef float f32x4_4 __attribute__((ext_vector_type(4), aligned(4)));
  f32x4 a;
  __device__ __forceinline__ void load(const void* p, long long row, int c, int H) {
    const int at = min(c, H - 4);
    a = f32x4{0.f, 0.f, 0.f, 0.f};
    if (c - at < 4 && at >= 0) a = *(const f32x4_4*)((const float*)p + row + at);
  }
  __device__ __forceinline__ void settle(const void* p, long long row, int c, int H) {
    if (H < 4) {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < H - c) a[i] = ((const float*)p)[row + c + i];
    } else {
      const int s = c - min(c, H - 4);
      if (s & 1) a = f32x4{a[1], a[2], a[3], 0.f};
      if (s & 2) a = f32x4{a[2], a[3], 0.f, 0.f};
    }
  }
  __device__ __forceinline__ f32x4 get() const { return a; }
  static __device__ __forceinline__ void put(void* p, long long at, int n, f32x4 v) {
    float* q = (float*)p + at;
    if (n >= 4) {
      *(f32x4_4*)q = v;
    } else {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (i < n) q[i] = v[i];
    }
  }
};
// Four weights of either type: loaded with others, converted where they are used.
struct FourWeights {
  Four<true> b;
  Four<false> f;
  __device__ __forceinline__ void load(const void* p, bool bf16, int c, int H) {
    if (bf16) b.load(p, 0, c, H);
    else f.load(p, 0, c, H);
  }
  __device__ __forceinline__ f32x4 get(const void* p, bool bf16, int c, int H) {
    if (bf16) {
      if (H % 4) b.settle(p, 0, c, H);
      return b.get();
    }
    if (H % 4) f.settle(p, 0, c, H);
    return f.get();
  }
};

enum { kAfterSum, kGateSum, kBeforeSum, kSums };
// How many of the columns' sums a launch for long rows has LDS for, beside a row.
constexpr int sums_of(int U) { return U > 2 ? 1 : 3; }

// (four waves a SIMD, 128 registers; two where a thread keeps eight columns)
template <int NT, int U, bool H16, bool Y16, bool Z16, bool kY>
__global__ void __launch_bounds__(NT, NT == 1024 || U == 1 ? 4 : 2) join_grad_kernel(JoinArgs a) {
  constexpr bool kLong = NT == 1024;
  __shared__ float lds[3 * NT / 64];
  __shared__ f32x4 long_sums[kLong ? sums_of(U) : 1][kLong ? U * NT : 1], long_d[kLong && kY ? U * NT : 1];
  uint64_t seed = 0, offset = 0;
  if (a.drop) seed = a.rng[0], offset = a.rng[1];
  const bool norm_x = a.before && a.dz, token = kY && a.gate_kind == MOE_GATE_TOKEN,
             channel = kY && a.gate_kind == MOE_GATE_CHANNEL, after = kY && a.after;
  const bool want[kSums] = {after && a.d_after, channel && a.d_gate, norm_x && a.d_before};
  const int place[kSums] = {0, want[0], want[0] + want[1]};   // of each sum that is wanted
  const void* const weights[kSums] = {a.after, a.gate, a.before};
  const bool use[kSums] = {after, channel, norm_x};
  f32x4 sum[kSums][kLong ? 1 : U] = {};
  const int c0 = 4 * (int)threadIdx.x;
  // the weights of four columns: kept, or (long rows) loaded with the columns
  struct Weights {
    f32x4 w[kSums];
  };
  Weights kept[kLong ? 1 : U];
  FourWeights raw_w[kSums];
  auto load_weights = [&](int u, bool first) {   // first: of those that the first pass over a row needs
#pragma unroll
    for (int k = 0; k < kSums; ++k)
      if (use[k] && (k == kBeforeSum || !first)) raw_w[k].load(weights[k], a.w16, 4 * NT * u + c0, a.H);
  };
  auto get_weights = [&](int u, bool first) {
    Weights o;
#pragma unroll
    for (int k = 0; k < kSums; ++k)
      o.w[k] = use[k] && (k == kBeforeSum || !first) ? raw_w[k].get(weights[k], a.w16, 4 * NT * u + c0, a.H)
                                                     : f32x4{1.f, 1.f, 1.f, 1.f};
    return o;
  };
  auto add = [&](int k, int u, f32x4 v) {
    if (!kLong) sum[k][kLong ? 0 : u] += v;
    else if (want[k]) long_sums[place[k]][u * NT + threadIdx.x] += v;
  };
  struct Rows {   // four of the thread's columns, and the row's gate
    Four<H16> d, x;
    Four<Z16> z;
    Four<Y16> y;
    float gate;
  } next[kLong ? 1 : U], now[kLong ? 1 : U];
  auto load = [&](Rows& o, long long t, int u) {
    const int c = 4 * NT * u + c0;
    const long long row = t * a.H;
    if (norm_x) {
      o.x.load(a.h, row, c, a.H);
      o.z.load(a.dz, row, c, a.H);
    }
    if (kY) o.y.load(a.y, row, c, a.H);
    if (a.dx) o.d.load(a.dx, row, c, a.H);
    if (token) o.gate = element(a.gate, a.w16, t);
  };
  // (a long row's columns come again for each use, by loops that stay loops: unrolled they
  // take more registers than there are)
  constexpr int kUnroll = kLong ? 1 : U;
  auto settle = [&](Rows& o, long long t, int u) {
    const int c = 4 * NT * u + c0;
    const long long row = t * a.H;
    if (norm_x) {
      o.x.settle(a.h, row, c, a.H);
      o.z.settle(a.dz, row, c, a.H);
    }
    if (kY) o.y.settle(a.y, row, c, a.H);
    if (a.dx) o.d.settle(a.dx, row, c, a.H);
  };
  auto columns = [&](long long t, int u, bool first) -> const Rows& {
    if (kLong) {
      load(now[0], t, u);
      load_weights(u, first);
      if (a.H % 4) settle(now[0], t, u);
      kept[0] = get_weights(u, first);
    }
    return now[kLong ? 0 : u];
  };
  auto prefetch = [&](long long t) {
    if (kLong || t >= a.T) return;
#pragma unroll
    for (int u = 0; u < (kLong ? 1 : U); ++u) load(next[u], t, u);
  };
  prefetch(blockIdx.x);
  if (kLong) {
    for (int k = 0; k < sums_of(U); ++k)
#pragma unroll
      for (int u = 0; u < U; ++u) long_sums[k][u * NT + threadIdx.x] = f32x4{0.f, 0.f, 0.f, 0.f};
  } else {
#pragma unroll
    for (int u = 0; u < (kLong ? 1 : U); ++u) {
      load_weights(u, false);
      kept[u] = get_weights(u, false);
    }
  }
  for (long long t = blockIdx.x; t < a.T; t += gridDim.x) {
#pragma unroll
    for (int u = 0; u < (kLong ? 1 : U); ++u) {
      now[u] = next[u];
      if (!kLong && a.H % 4) settle(now[u], t, u);
    }
    prefetch(t + gridDim.x);
    float s[3] = {0.f, 0.f, 0.f};   // of x^2, x v, y^2
#pragma unroll kUnroll
    for (int u = 0; u < U; ++u) {
      const Rows& row = columns(t, u, true);
      if (norm_x) {
        const f32x4 x = row.x.get(), v = row.z.get() * kept[kLong ? 0 : u].w[kBeforeSum];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[0] = fmaf(x[i], x[i], s[0]);
          s[1] = fmaf(x[i], v[i], s[1]);
        }
      }
      if (after) {
        const f32x4 y = row.y.get();
#pragma unroll
        for (int i = 0; i < 4; ++i) s[2] = fmaf(y[i], y[i], s[2]);
      }
    }
    row_sums<NT>(s, lds);
    const float r = rsqrtf(s[0] / a.H + a.eps), m = r * r * (s[1] / a.H);
    const float q = after ? rsqrtf(s[2] / a.H + a.eps) : 1.f;
    f32x4 short_d[kLong ? 1 : U];
    float s2[2] = {0.f, 0.f};   // of y v of the norm after the block, and da b
#pragma unroll kUnroll
    for (int u = 0; u < U; ++u) {
      const int c = 4 * NT * u + c0;
      const long long at = t * a.H + c;
      const Rows& row = columns(t, u, false);
      f32x4 d = a.dx ? row.d.get() : f32x4{0.f, 0.f, 0.f, 0.f};
      if (norm_x) {
        const f32x4 x = row.x.get(), z = row.z.get(), v = z * kept[kLong ? 0 : u].w[kBeforeSum];
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = fmaf(r, fmaf(-m, x[i], v[i]), d[i]);
        add(kBeforeSum, u, z * (x * r));
      }
      if (a.dh) Four<H16>::put(a.dh, at, a.H - c, d);
      d *= a.scale;
      if (a.drop) {
        uint32_t word[4];
        philox((uint32_t)(c / 4), (uint32_t)t, offset, seed, word);
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = word[i] >= a.least ? d[i] * a.keep : 0.f;
      }
      if (kY) {
        const f32x4 y = row.y.get(), yn = y * q;
        const f32x4 wa = kept[kLong ? 0 : u].w[kAfterSum], da = d, b = yn * wa;
        if (channel) {
          add(kGateSum, u, da * b);
          d *= kept[kLong ? 0 : u].w[kGateSum];
        } else if (token) {
#pragma unroll
          for (int i = 0; i < 4; ++i) s2[1] = fmaf(da[i], b[i], s2[1]);
          d *= row.gate;
        }
        if (after) {
          add(kAfterSum, u, d * yn);
          d *= wa;
#pragma unroll
          for (int i = 0; i < 4; ++i) s2[0] = fmaf(d[i], y[i], s2[0]);
        }
        if (kLong) long_d[u * NT + threadIdx.x] = d;
        else short_d[kLong ? 0 : u] = d;
      } else if (a.dy) {
        Four<Y16>::put(a.dy, at, a.H - c, d);
      }
    }
    if (!kY) continue;
    float k = 0.f;
    if (after || token) {
      row_sums<NT>(s2, lds);
      if (token && a.d_gate && threadIdx.x == 0) a.d_gate[t] = s2[1];
      k = q * q * (s2[0] / a.H);
    }
    if (!a.dy) continue;
#pragma unroll kUnroll
    for (int u = 0; u < U; ++u) {
      const int c = 4 * NT * u + c0;
      f32x4 d = kLong ? long_d[u * NT + threadIdx.x] : short_d[kLong ? 0 : u];
      if (after) {
        if (kLong) {
          now[0].y.load(a.y, t * a.H, c, a.H);
          if (a.H % 4) now[0].y.settle(a.y, t * a.H, c, a.H);
        }
        const f32x4 y = now[kLong ? 0 : u].y.get();
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = q * fmaf(-k, y[i], d[i]);
      }
      Four<Y16>::put(a.dy, t * a.H + c, a.H - c, d);
    }
  }
  // the columns' sums: this workgroup's part of each, or the whole where it is the only one
  // (a sum that the call has no terms for is zeros)
  float* const outs[kSums] = {a.d_after, a.gate_kind == MOE_GATE_CHANNEL ? a.d_gate : nullptr, a.d_before};
  long long skip = 0;
#pragma unroll
  for (int k = 0; k < kSums; ++k) {
    if (!outs[k]) continue;
    float* const p = gridDim.x > 1 ? a.parts + skip + (long long)blockIdx.x * a.H : outs[k];
    skip += (long long)gridDim.x * a.H;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = 4 * NT * u + c0;
      const f32x4 v = !kLong ? sum[k][kLong ? 0 : u] : want[k] ? long_sums[place[k]][u * NT + threadIdx.x] : f32x4{0.f, 0.f, 0.f, 0.f};
      if (c < a.H) Four<false>::put(p, c, a.H - c, v);
    }
  }
}

// parts [array][G][H] to the arrays' sums: a workgroup takes 32 columns of an array, 32
// threads a column.
__global__ void __launch_bounds__(1024) column_sums_kernel(const float* parts, float* o0, float* o1, float* o2, int G,
                                                           int H) {
  __shared__ float lds[32][33];
  const int c = threadIdx.x % 32, k = threadIdx.x / 32;
  const long long col = (long long)blockIdx.x * 32 + c;
  const float* p = parts + (long long)blockIdx.y * G * H;
  float s = 0.f;
  if (col < H) {
#pragma unroll 8
    for (int g = k; g < G; g += 32) s += p[(long long)g * H + col];
  }
  lds[k][c] = s;
  __syncthreads();
  if (k == 0 && col < H) {
    s = 0.f;
    for (int i = 0; i < 32; ++i) s += lds[i][c];
    (blockIdx.y == 0 ? o0 : blockIdx.y == 1 ? o1 : o2)[col] = s;
  }
}

// ---- host -------------------------------------------------------------------------

constexpr int kMaxWidth = 16384;

int check_choice(const void* logits, int32_t T, int32_t E, int32_t topk, int32_t type, int32_t score) {
  if (T < 0 || E < 1 || topk < 1 || topk > E || !type_ok(type) || (score != MOE_SOFTMAX && score != MOE_SIGMOID))
    return MOE_ERR_INVALID_ARG;
  if (E > kMaxExperts || topk > kMaxTopk) return MOE_ERR_UNSUPPORTED;
  if (T > 0 && !logits) return MOE_ERR_INVALID_ARG;
  return aligned(logits, type_size(type)) ? MOE_OK : MOE_ERR_ALIGNMENT;
}

// The lanes of a token and the logits of a lane for E experts: f(L, R) as types.
template <int L, int R>
struct Shape {
  static constexpr int lanes = L, each = R;
};
template <class F>
void with_shape(int E, F f) {
  if (E <= 32) f(Shape<8, 4>());
  else if (E <= 64) f(Shape<16, 4>());
  else if (E <= 128) f(Shape<16, 8>());
  else if (E <= 256) f(Shape<16, 16>());
  else if (E <= 512) f(Shape<64, 8>());
  else f(Shape<64, 16>());
}

template <class F>
void with_choice(int E, F f) {
  if (E <= 16) f(Shape<4, 4>());
  else if (E <= 32) f(Shape<8, 4>());
  else if (E <= 64) f(Shape<8, 8>());
  else if (E <= 128) f(Shape<8, 16>());
  else if (E <= 256) f(Shape<16, 16>());
  else if (E <= 512) f(Shape<16, 32>());
  else f(Shape<64, 16>());
}

// Launches of at most 2^20 workgroups (a launch holds fewer than 2^32 threads), `per` tokens
// each: f(first token, workgroups).
template <class F>
void in_launches(int32_t T, int per, F f) {
  const long long most = (long long)per << 20;
  for (long long t = 0; t < T; t += most) f(t, (unsigned)(((T - t < most ? T - t : most) + per - 1) / per));
}

int check_join(const JoinArgs& a, int32_t T, int32_t H, int32_t h_type, int32_t y_type, int32_t z_type,
               int32_t w_type, int32_t gate_kind, double drop) {
  if (T < 0 || H < 1 || !type_ok(h_type) || !type_ok(y_type) || !type_ok(z_type) || !type_ok(w_type) ||
      gate_kind < MOE_GATE_NONE || gate_kind > MOE_GATE_CHANNEL || !(drop >= 0.0 && drop < 1.0))
    return MOE_ERR_INVALID_ARG;
  if (H > kMaxWidth) return MOE_ERR_UNSUPPORTED;
  if (gate_kind == MOE_GATE_CHANNEL && !a.gate) return MOE_ERR_INVALID_ARG;
  if (T > 0) {   // (tensors of no rows may have no address)
    if ((gate_kind == MOE_GATE_TOKEN && !a.gate) || (drop > 0.0 && !a.rng)) return MOE_ERR_INVALID_ARG;
    if (!a.y && (a.after || gate_kind != MOE_GATE_NONE || drop > 0.0)) return MOE_ERR_INVALID_ARG;
  }
  const size_t h = type_size(h_type), y = type_size(y_type), z = type_size(z_type), w = type_size(w_type);
  if (!aligned(a.h, h) || !aligned(a.x, h) || !aligned(a.dx, h) || !aligned(a.dh, h) || !aligned(a.y, y) ||
      !aligned(a.dy, y) || !aligned(a.z, z) || !aligned(a.dz, z) || !aligned(a.after, w) || !aligned(a.gate, w) ||
      !aligned(a.before, w) || !aligned(a.rng, 8) || !aligned(a.d_after, 4) || !aligned(a.d_gate, 4) ||
      !aligned(a.d_before, 4))
    return MOE_ERR_ALIGNMENT;
  return MOE_OK;
}
void set_common(JoinArgs* a, int32_t T, int32_t H, int32_t h_type, int32_t y_type, int32_t z_type, int32_t w_type,
                int32_t gate_kind, float scale, double drop, float eps) {
  a->T = T, a->H = H;
  a->h16 = h_type == MOE_BF16, a->y16 = y_type == MOE_BF16, a->z16 = z_type == MOE_BF16, a->w16 = w_type == MOE_BF16;
  a->gate_kind = gate_kind;
  a->scale = scale, a->eps = eps;
  a->drop = drop > 0.0;
  a->keep = (float)(1.0 / (1.0 - drop));
  a->least = (uint32_t)std::floor(drop * 4294967296.0);
}
bool same(const void* p, const void* q) { return p && p == q; }

// Threads of a row and chunks of a thread: f(NT, U) as types (Shape).
template <class F>
void with_row(int H, F f) {
  if (H <= 512) f(Shape<64, 1>());
  else if (H <= 2048) f(Shape<256, 1>());
  else if (H <= 8192) f(Shape<1024, 1>());
  else f(Shape<1024, 2>());
}
template <class F>
void with_grad_row(int H, F f) {
  if (H <= 256) f(Shape<64, 1>());
  else if (H <= 1024) f(Shape<256, 1>());
  else if (H <= 2048) f(Shape<512, 1>());
  else if (H <= 4096) f(Shape<512, 2>());
  else if (H <= 8192) f(Shape<1024, 2>());
  else f(Shape<1024, 4>());
}
// The threads that a launch of them needs, where each takes `each` columns once.
template <class S>
int threads_of(S, int H, int each) {
  return S::each > 1 ? S::lanes : (H + 64 * each - 1) / (64 * each) * 64;
}
// Workgroups of the gradient: enough to fill the card, few enough that their parts are
// small beside the rows.
int grad_groups(int T, int H) {
  const int most = H <= 256 ? 2048 : H <= 1024 ? 1024 : H <= 2048 ? 512 : 256;
  const int rows = T / 2 + T % 2;   // two rows a workgroup, where there are few
  return rows < most ? (rows < 1 ? 1 : rows) : most;
}

}  // namespace

extern "C" int moe_choose(const void* logits, const float* bias, int32_t* ids, float* gates, int32_t T, int32_t E,
                          int32_t topk, int32_t logits_type, int32_t score, int32_t renormalize, float scale,
                          void* stream) {
  const int bad = check_choice(logits, T, E, topk, logits_type, score);
  if (bad) return bad;
  if (T == 0) return MOE_OK;
  if (!ids || !gates) return MOE_ERR_INVALID_ARG;
  if (!aligned(bias, 4) || !aligned(ids, 4) || !aligned(gates, 4)) return MOE_ERR_ALIGNMENT;
  if (logits == (const void*)ids || logits == (const void*)gates || (void*)ids == (void*)gates || bias == gates ||
      same(bias, ids))
    return MOE_ERR_INVALID_ARG;
  const hipStream_t s = (hipStream_t)stream;
  with_choice(E, [&](auto shape) {
    constexpr int L = decltype(shape)::lanes, R = decltype(shape)::each, per = 256 / L;
    in_launches(T, per, [&](long long first, unsigned blocks) {
      if (logits_type == MOE_BF16)
        choose_kernel<__bf16, L, R><<<blocks, 256, 0, s>>>((const __bf16*)logits, bias, ids, gates, first, T, E, topk,
                                                           score == MOE_SOFTMAX, renormalize != 0, scale);
      else
        choose_kernel<float, L, R><<<blocks, 256, 0, s>>>((const float*)logits, bias, ids, gates, first, T, E, topk,
                                                          score == MOE_SOFTMAX, renormalize != 0, scale);
    });
  });
  return done();
}

extern "C" int moe_choose_grad(const float* dgates, const void* logits, const int32_t* ids, void* dlogits, int32_t T,
                               int32_t E, int32_t topk, int32_t logits_type, int32_t score, int32_t renormalize,
                               float scale, void* workspace, void* stream) {
  const int bad = check_choice(logits, T, E, topk, logits_type, score);
  if (bad) return bad;
  if (T == 0) return MOE_OK;
  if (!dgates || !ids || !dlogits) return MOE_ERR_INVALID_ARG;
  if (!aligned(dgates, 4) || !aligned(ids, 4) || !aligned(dlogits, type_size(logits_type)) || !aligned(workspace, 256))
    return MOE_ERR_ALIGNMENT;
  if (dlogits == logits || dlogits == (const void*)dgates || dlogits == (const void*)ids) return MOE_ERR_INVALID_ARG;
  const hipStream_t s = (hipStream_t)stream;
  uint32_t* st = (uint32_t*)workspace;
  with_shape(E, [&](auto shape) {
    constexpr int L = decltype(shape)::lanes, R = decltype(shape)::each, per = 256 / L;
    in_launches(T, per, [&](long long first, unsigned blocks) {
      if (logits_type == MOE_BF16)
        choose_grad_kernel<__bf16, L, R><<<blocks, 256, 0, s>>>(dgates, (const __bf16*)logits, ids, (__bf16*)dlogits,
                                                                first, T, E, topk, score == MOE_SOFTMAX,
                                                                renormalize != 0, scale, st);
      else
        choose_grad_kernel<float, L, R><<<blocks, 256, 0, s>>>(dgates, (const float*)logits, ids, (float*)dlogits,
                                                               first, T, E, topk, score == MOE_SOFTMAX,
                                                               renormalize != 0, scale, st);
    });
  });
  return done();
}

extern "C" int moe_join(const void* h, const void* y, const void* after, const void* gate, const void* before,
                        const uint64_t* rng, void* x, void* z, int32_t T, int32_t H, int32_t h_type, int32_t y_type,
                        int32_t z_type, int32_t w_type, int32_t gate_kind, float scale, double drop, float eps,
                        void* stream) {
  JoinArgs a = {};
  a.h = h, a.y = y, a.after = after, a.gate = gate, a.before = before, a.rng = rng, a.x = x, a.z = z;
  const int bad = check_join(a, T, H, h_type, y_type, z_type, w_type, gate_kind, drop);
  if (bad) return bad;
  if (T == 0) return MOE_OK;
  if ((!h && !y) || (y && !x) || (before && !z) || (!y && !before)) return MOE_ERR_INVALID_ARG;
  if (!y) a.x = nullptr;
  if (!before) a.z = nullptr;
  for (const void* in : {y, after, gate, before, (const void*)rng})   // (x may be h)
    if (same(a.z, in) || same(a.x, in)) return MOE_ERR_INVALID_ARG;
  if (same(a.z, h) || same(a.x, a.z)) return MOE_ERR_INVALID_ARG;
  set_common(&a, T, H, h_type, y_type, z_type, w_type, gate_kind, scale, drop, eps);
  const hipStream_t s = (hipStream_t)stream;
  with_row(H, [&](auto shape) {
    constexpr int NT = decltype(shape)::lanes, U = decltype(shape)::each;
    const int threads = threads_of(shape, H, 8);
    in_launches(T, 1, [&](long long first, unsigned blocks) { join_kernel<NT, U><<<blocks, threads, 0, s>>>(a, first); });
  });
  return done();
}

extern "C" size_t moe_join_grad_scratch_size(int32_t T, int32_t H) {
  if (T < 0 || H < 1 || H > kMaxWidth) return 0;
  const int G = grad_groups(T, H);
  return G > 1 ? (size_t)G * H * 3 * sizeof(float) : 0;
}

extern "C" int moe_join_grad(const void* dx, const void* dz, const void* x, const void* y, const void* after,
                             const void* gate, const void* before, const uint64_t* rng, void* dh, void* dy,
                             float* d_after, float* d_gate, float* d_before, int32_t T, int32_t H, int32_t h_type,
                             int32_t y_type, int32_t z_type, int32_t w_type, int32_t gate_kind, float scale,
                             double drop, float eps, void* scratch, size_t scratch_bytes, void* stream) {
  JoinArgs a = {};
  const bool reads_y = after || gate_kind != MOE_GATE_NONE;
  a.dx = dx, a.dz = dz, a.h = x, a.after = after, a.gate = gate, a.before = before, a.rng = rng;
  a.dh = dh, a.dy = dy, a.d_after = d_after, a.d_gate = d_gate, a.d_before = d_before;
  a.y = y || reads_y ? y : dy;   // (that there was one is all that matters)
  const int bad = check_join(a, T, H, h_type, y_type, z_type, w_type, gate_kind, drop);
  if (bad) return bad;
  if ((d_after && !after) || (d_before && !before) || (d_gate && gate_kind == MOE_GATE_NONE)) return MOE_ERR_INVALID_ARG;
  if (T > 0 && ((!dx && !dz) || (dz && (!before || !x)) || (dy && !a.y))) return MOE_ERR_INVALID_ARG;
  const void* outs[5] = {dh, dy, d_after, d_gate, d_before};
  for (const void* o : outs)
    for (const void* in : {dz, x, y, after, gate, before, (const void*)rng})
      if (same(o, in)) return MOE_ERR_INVALID_ARG;
  for (int i = 1; i < 5; ++i)   // (dh may be dx)
    if (same(outs[i], dx)) return MOE_ERR_INVALID_ARG;
  for (int i = 0; i < 5; ++i)
    for (int j = 0; j < i; ++j)
      if (same(outs[i], outs[j])) return MOE_ERR_INVALID_ARG;
  set_common(&a, T, H, h_type, y_type, z_type, w_type, gate_kind, scale, drop, eps);
  const int G = grad_groups(T, H);
  const bool channel = gate_kind == MOE_GATE_CHANNEL && d_gate;
  const int arrays = (d_after != nullptr) + channel + (d_before != nullptr);
  if (T == 0 && arrays == 0) return MOE_OK;
  if (G > 1 && arrays > 0) {
    if (!scratch || scratch_bytes < moe_join_grad_scratch_size(T, H)) return MOE_ERR_WORKSPACE;
    if (!aligned(scratch, 16)) return MOE_ERR_ALIGNMENT;
    a.parts = (float*)scratch;
  }
  if (T == 0) a.drop = false;
  const hipStream_t s = (hipStream_t)stream;
  auto launch = [&](const JoinArgs& a) {
    with_grad_row(H, [&](auto shape) {
      constexpr int NT = decltype(shape)::lanes, U = decltype(shape)::each;
      const int threads = threads_of(shape, H, 4);
#define MOE_GRAD(H16, Y16, Z16)                                                      \
  reads_y ? join_grad_kernel<NT, U, H16, Y16, Z16, true><<<(unsigned)G, threads, 0, s>>>(a) \
          : join_grad_kernel<NT, U, H16, Y16, Z16, false><<<(unsigned)G, threads, 0, s>>>(a)
      switch (4 * a.h16 + 2 * a.y16 + a.z16) {
        case 0: MOE_GRAD(false, false, false); break;
        case 1: MOE_GRAD(false, false, true); break;
        case 2: MOE_GRAD(false, true, false); break;
        case 3: MOE_GRAD(false, true, true); break;
        case 4: MOE_GRAD(true, false, false); break;
        case 5: MOE_GRAD(true, false, true); break;
        case 6: MOE_GRAD(true, true, false); break;
        default: MOE_GRAD(true, true, true); break;
      }
#undef MOE_GRAD
    });
    return hipGetLastError() == hipSuccess;
  };
  // LDS holds one of the columns' sums of the longest rows: the others by launches of their own,
  // before dh, which may be dx, is written
  float** const sums[3] = {&a.d_after, channel ? &a.d_gate : nullptr, &a.d_before};
  int left = arrays;
  for (int k = 2; H > 8192 && k >= 0 && left > 1; --k) {
    if (!sums[k] || !*sums[k]) continue;
    JoinArgs b = a;
    b.dh = b.dy = nullptr;
    b.d_after = k == 0 ? a.d_after : nullptr;
    b.d_gate = k == 1 ? a.d_gate : nullptr;
    b.d_before = k == 2 ? a.d_before : nullptr;
    *sums[k] = nullptr;
    --left;
    if (a.parts) b.parts = a.parts + (long long)left * G * H;
    if (!launch(b)) return MOE_ERR_HIP;
  }
  if (!launch(a)) return MOE_ERR_HIP;
  if (G > 1 && arrays > 0) {
    float* o[3] = {nullptr, nullptr, nullptr};
    int n = 0;
    if (d_after) o[n++] = d_after;
    if (channel) o[n++] = d_gate;
    if (d_before) o[n++] = d_before;
    column_sums_kernel<<<dim3((unsigned)((H + 31) / 32), (unsigned)arrays), 1024, 0, s>>>(a.parts, o[0], o[1], o[2], G,
                                                                                          H);
  }
  return done();
}

extern "C" int moe_block_abi_version(void) { return 100; }
