// Tokens sorted by expert, their rows' way to the experts and back, and the
// gradients of that way, for gfx950 (C ABI: moe_experts.h).
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "call_checks.h"
#include "expert_units.h"
#include "moe_experts.h"
#include "status_bits.h"

namespace {

constexpr int kMaxTopk = 64;      // a wave holds a token's slots, one a lane
constexpr int kMaxExperts = 1024;

// ---- the sort ------------------------------------------------------------------
//
// A counting sort by expert: counts, their prefix, places.  A slot's place
// within its expert is the slots of that expert before it: those of earlier
// chunks and earlier waves (counted), those of earlier rounds of its wave (a
// running count in LDS, which only that wave touches) and those of lower lanes
// (a ballot per bit of the expert id gives the lanes with the same id).  No
// atomic decides an order, so the sort is stable and repeatable.
//
// Up to kOneLaunch slots one workgroup does it all.  Beyond, a first launch
// counts each chunk's experts and a second places the chunks, each workgroup
// adding up all chunks' counts for itself, from the L2s: up to 64 KB in chunks of 512
// and 1024 slots, at most 1 MB (256 chunks of 1024 experts) in larger ones.  Two
// launches without waits between workgroups.  Latency bounds both ways (98304 slots
// move 2 MB, 0.4 us of a copy): 6 slots of 32 experts take 3.0 us of GPU time, 98304
// slots of 32 experts 3.0 + 6.9, 131072 of 256 3.0 + 13.3; with many chunks of many
// experts the counts do: 524288 slots of 1024 experts, 256 MB of them, 5.0 + 69.
constexpr int kOneLaunch = 4096;
constexpr int kOneThreads = 1024;
constexpr int kPlaceThreads = 256;
// Slots of a chunk: as few as spread the work over many CUs, while what every
// workgroup adds up (chunks times experts) stays small.  Measured (us a call, replayed
// from a graph, 512 / 1024 / 2048 slots): 98304 slots of 32 experts 8.9 / 10.2 / 12.3, 262144 of 64 15.2 / 12.5 /
// 13.0, 131072 of 256 20.8 / 15.9 / 15.2, 65536 of 1024 38 / 27 / 23.
constexpr int kLeastChunk = 512, kChunk = 2048;   // (past kChunk: times what keeps them at most kMaxChunks)
constexpr int kMaxChunks = 256;
constexpr long long kMaxCounts = 16384;

struct SortArgs {
  const int32_t* ids;
  const float* gates;
  int32_t* offsets;
  int32_t* token_ids;
  float* gate_w;
  int32_t* slot_rows;
  uint32_t* counts;      // [chunks][E], two launches only
  int slots, topk, E, first, id_bits;
  int chunk, chunks;     // slots of a chunk (a multiple of 512)
};

// the expert of an id, or -1
__device__ __forceinline__ int expert_of(const SortArgs& a, int id) {
  const int64_t e = (int64_t)id - a.first;
  return e >= 0 && e < a.E ? (int)e : -1;
}

// A wave's rounds of 64 slots, R of them by loads that are in flight together (one
// after the other they took 8 of a large batch's 13 us).
constexpr int kRounds = 8;
// (end: of the wave's slots; lanes past it load the last one again)
template <int R, class T>
__device__ __forceinline__ void load_rounds(const T* p, int s, int end, T (&v)[R]) {
  const int first = s - (int)(threadIdx.x & 63);
#pragma unroll
  for (int r = 0; r < R; ++r)
    if (first + 64 * r < end) v[r] = p[min(s + 64 * r, end - 1)];
}

// the lanes that hold the same e (0 <= e < 2^bits) as this one, among `live`
__device__ __forceinline__ uint64_t same_expert(int e, uint64_t live, int bits) {
  uint64_t m = live;
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((e >> b) & 1);
    m &= ((e >> b) & 1) ? set : ~set;
  }
  return m;
}

__global__ void __launch_bounds__(kPlaceThreads) sort_count_kernel(SortArgs a) {
  __shared__ uint32_t n[kMaxExperts];
  for (int e = threadIdx.x; e < a.E; e += kPlaceThreads) n[e] = 0;
  __syncthreads();
  const int s0 = blockIdx.x * a.chunk, s1 = min(s0 + a.chunk, a.slots);
  const int wave = threadIdx.x >> 6, per = a.chunk / (kPlaceThreads / 64);
  const int w1 = min(s0 + (wave + 1) * per, s1);
  for (int s = s0 + wave * per + (int)(threadIdx.x & 63); s - (int)(threadIdx.x & 63) < w1; s += 64 * kRounds) {
    int id[kRounds];
    load_rounds<kRounds>(a.ids, s, w1, id);
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      const int e = s + 64 * r < w1 ? expert_of(a, id[r]) : -1;
      if (e >= 0) atomicAdd(&n[e], 1u);
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kPlaceThreads)
    a.counts[(size_t)blockIdx.x * a.E + e] = n[e];
}

// A count in LDS that one wave's lanes hand on among themselves: the next
// round reads what a lane of this one wrote.
__device__ __forceinline__ uint32_t lds_get(uint32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
__device__ __forceinline__ void lds_put(uint32_t* p, uint32_t v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

// kParts: wave parts times experts that fit (a workgroup has as many waves as that allows)
template <int kMaxThreads, int kParts, bool kOne>
__global__ void __launch_bounds__(kMaxThreads) sort_place_kernel(SortArgs a) {
  __shared__ uint32_t part[kParts];          // [wave][E]: slots in the wave's part, then its next row
  __shared__ uint32_t first[kMaxExperts];    // the expert's slots, then its first row in this chunk
  __shared__ uint32_t before[kMaxExperts];   // its slots in earlier chunks
  __shared__ uint32_t live;                  // rows of all experts
  const int tid = threadIdx.x, threads = blockDim.x, lane = tid & 63, wave = tid >> 6;
  const int waves = threads >> 6;
  for (int i = tid; i < waves * a.E; i += threads) part[i] = 0;
  for (int e = tid; e < a.E; e += threads) first[e] = before[e] = 0;
  __syncthreads();

  // the wave's part of the chunk, in whole rounds of 64 slots
  const int s0 = blockIdx.x * a.chunk, s1 = min(s0 + a.chunk, a.slots);
  const int per = (a.chunk / 64 + waves - 1) / waves * 64;
  const int w0 = min(s0 + wave * per, s1), w1 = min(w0 + per, s1);
  uint32_t* mine = part + wave * a.E;
  constexpr int R = kOne ? kRounds / 2 : kRounds;   // (a single workgroup has at most as many)
  for (int s = w0 + lane; s - lane < w1; s += 64 * R) {
    int id[R];
    load_rounds<R>(a.ids, s, w1, id);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int e = s + 64 * r < w1 ? expert_of(a, id[r]) : -1;
      if (e >= 0) atomicAdd(&mine[e], 1u);
    }
  }
  if (!kOne) {
    // a thread adds up one expert's counts over every groups-th chunk
    const int groups = max(1, threads / a.E);
    for (int i = tid; i < groups * a.E; i += threads) {
      const int e = i % a.E;
      uint32_t n = 0, b = 0;
#pragma unroll 8
      for (int c = i / a.E; c < a.chunks; c += groups) {
        const uint32_t v = a.counts[(size_t)c * a.E + e];
        n += v;
        b += c < (int)blockIdx.x ? v : 0;
      }
      atomicAdd(&first[e], n);
      atomicAdd(&before[e], b);
    }
  }
  __syncthreads();
  if (kOne) {
    for (int e = tid; e < a.E; e += threads) {
      uint32_t n = 0;
      for (int w = 0; w < waves; ++w) n += part[w * a.E + e];
      first[e] = n;
    }
    __syncthreads();
  }
  if (wave == 0) {   // the experts' first rows
    const int each = (a.E + 63) / 64;
    const int e0 = min(lane * each, a.E), e1 = min(e0 + each, a.E);
    uint32_t n = 0;
    for (int e = e0; e < e1; ++e) n += first[e];
    const uint32_t end = (uint32_t)wave_prefix((int)n);
    uint32_t at = end - n;
    for (int e = e0; e < e1; ++e) {
      const uint32_t c = first[e];
      if (blockIdx.x == 0) a.offsets[e] = (int32_t)at;
      first[e] = at + before[e];
      at += c;
    }
    if (lane == 63) {
      live = end;
      if (blockIdx.x == 0) a.offsets[a.E] = (int32_t)end;
    }
  }
  __syncthreads();
  for (int e = tid; e < a.E; e += threads) {
    uint32_t at = first[e];
    for (int w = 0; w < waves; ++w) {
      const uint32_t n = part[w * a.E + e];
      part[w * a.E + e] = at;
      at += n;
    }
  }
  __syncthreads();
  const int rows = (int)live;
  for (int s0r = w0 + lane; s0r - lane < w1; s0r += 64 * R) {
    int id[R];
    float gate[R];
    load_rounds<R>(a.ids, s0r, w1, id);
    load_rounds<R>(a.gates, s0r, w1, gate);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int s = s0r + 64 * r;
      if (s - lane >= w1) break;   // (uniform)
      const int e = s < w1 ? expert_of(a, id[r]) : -1;
      const uint64_t same = same_expert(e, __ballot(e >= 0), a.id_bits);
      int row = -1;
      if (e >= 0) {
        const uint32_t at = lds_get(&mine[e]);
        const uint64_t lower = same & ((1ull << lane) - 1);
        row = (int)at + __popcll(lower);
        __builtin_amdgcn_wave_barrier();
        if (lower == 0) lds_put(&mine[e], at + __popcll(same));
        __builtin_amdgcn_wave_barrier();
        a.token_ids[row] = s / a.topk;
        a.gate_w[row] = gate[r];
      }
      if (s < w1) {
        a.slot_rows[s] = row;
        if (s >= rows) {   // past the last row
          a.token_ids[s] = -1;
          a.gate_w[s] = 0.f;
        }
      }
    }
  }
}

// ---- rows ------------------------------------------------------------------------
//
// One wave takes a token and 64 chunks of its columns (V elements a lane, 16
// bytes of bf16): the token's row is read once, or written once, and its
// slots' rows are found by one load of slot_rows that the lanes share.  The
// last chunk of a row that is no whole number of chunks starts V elements
// before the row's end and overlaps the one before, so no size needs single
// elements (rows shorter than a chunk take V = 1), and the loads need no more
// alignment than their elements have.

// A token's slots, one a lane: rows in range, and which lanes have one.
struct Slots {
  int row;
  uint64_t mask;
};
__device__ __forceinline__ Slots token_slots(const int32_t* slot_rows, long long t, int topk,
                                             long long rows, uint32_t* status) {
  const int lane = threadIdx.x & 63;
  int r = -1;
  if (lane < topk) r = slot_rows[t * topk + lane];
  const bool bad = r < -1 || r >= rows;
  if (bad) {
    r = -1;
    if (status) __hip_atomic_fetch_or(status, kStBadRouting, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  return {r, __ballot(r >= 0)};
}

// V elements of T in registers, and as they lie in memory (aligned to an element)
template <class T, int V>
struct Chunk {
  typedef T reg __attribute__((ext_vector_type(V)));
  typedef T mem __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};
template <class T, int V>
using Reg = typename Chunk<T, V>::reg;
template <class T, int V>
__device__ __forceinline__ Reg<T, V> load(const T* p) {
  return *(const typename Chunk<T, V>::mem*)p;
}
template <class T, int V>
__device__ __forceinline__ void store(T* p, Reg<T, V> v) {
  *(typename Chunk<T, V>::mem*)p = v;
}

// the wave's token and the first of its columns; false past the last token
template <int kCols>
__device__ __forceinline__ bool unit_at(long long unit, int T, int blocks, long long* t, long long* c) {
  *t = unit / blocks;
  *c = (unit - *t * blocks) * kCols;
  return *t < T;
}

// V: bytes of a chunk (16, or 1 for shorter rows); U chunks a lane.  Bound by memory;
// a small call by latency: 777 tokens to their rows, 7.8 MB, 3.7 us.
template <int V, int U>
__global__ void __launch_bounds__(256) dispatch_kernel(const uint8_t* x, const int32_t* slot_rows,
                                                       uint8_t* out, int T, int topk, long long rows,
                                                       long long width, int blocks, uint32_t* status) {
  const int lane = threadIdx.x & 63;
  const long long stride = (long long)gridDim.x * 4;
  for (long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);; unit += stride) {
    long long t, c0;
    if (!unit_at<64 * V * U>(unit, T, blocks, &t, &c0)) break;
    const Slots sl = token_slots(slot_rows, t, topk, rows, status);
    Reg<uint8_t, V> v[U];
    long long c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      c[u] = c0 + (long long)(u * 64 + lane) * V;
      const bool in = c[u] < width;
      c[u] = in ? min(c[u], width - V) : -1;
      if (in) v[u] = load<uint8_t, V>(x + t * width + c[u]);
    }
    for (uint64_t m = sl.mask; m; m &= m - 1) {
      uint8_t* o = out + (long long)__builtin_amdgcn_readlane(sl.row, (int)__builtin_ctzll(m)) * width;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c[u] >= 0) store<uint8_t, V>(o + c[u], v[u]);
    }
  }
}

// Sums of a token's rows, weighted (combine) or not (the dispatch's gradient), in fp32
// in slot order, rounded once.  Bound by memory: every row is read once, in batches of
// eight loads; the dispatch's gradient of 8192 tokens moves 168 MB in 32.9 us, 5.1 TB/s (a
// copy reaches 4.9); 64 tokens combine in 3.4 us, latency.
constexpr int kBatch = 8;   // rows whose loads are in flight together
template <class In, class Out, bool kWeighted, int V>
__global__ void __launch_bounds__(256) sum_rows_kernel(const In* y, const int32_t* slot_rows,
                                                       const float* gates, Out* out, int T, int topk,
                                                       long long rows, int H, int blocks,
                                                       uint32_t* status) {
  const int lane = threadIdx.x & 63;
  const long long stride = (long long)gridDim.x * 4;
  for (long long unit = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);; unit += stride) {
    long long t, c0;
    if (!unit_at<64 * V>(unit, T, blocks, &t, &c0)) break;
    const Slots sl = token_slots(slot_rows, t, topk, rows, status);
    float gate = 1.f;
    if (kWeighted && lane < topk) gate = gates[t * topk + lane];
    const long long c1 = c0 + lane * V;
    const bool in = c1 < H;
    const long long c = in ? min(c1, (long long)H - V) : 0;
    float acc[V] = {};
    uint64_t m = sl.mask;
    while (m) {
      Reg<In, V> v[kBatch];
      const int n = min(kBatch, (int)__popcll(m));
      uint64_t q = m;
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (u < n) {
          const long long r = __builtin_amdgcn_readlane(sl.row, (int)__builtin_ctzll(q));
          v[u] = load<In, V>(y + r * H + c);
          q &= q - 1;
        }
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (u < n) {
          const float g = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(gate), (int)__builtin_ctzll(m)));
#pragma unroll
          for (int i = 0; i < V; ++i) acc[i] = kWeighted ? fmaf(g, (float)v[u][i], acc[i]) : acc[i] + (float)v[u][i];
          m &= m - 1;
        }
    }
    Reg<Out, V> o;
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = (Out)acc[i];
    if (in) store<Out, V>(out + t * H + c, o);
  }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// A wave takes a token: dout's columns stay in registers (64 V U of them at a
// time) while its slots' rows of y come by and their gradients leave.  dgates' sum
// is fp32, the lanes' parts joined in a fixed order; dy is rounded once.  Bound by
// memory: y read and dy written once, 941 MB for 16384 tokens in 188 us, 5.0 TB/s.
template <class DOut, class Y, int V, int U>
__global__ void __launch_bounds__(256) combine_grad_kernel(const DOut* dout, const Y* y,
                                                           const int32_t* slot_rows, const float* gates,
                                                           Y* dy, float* dgates, int T, int topk,
                                                           long long rows, int H, uint32_t* status) {
  const int lane = threadIdx.x & 63;
  const long long stride = (long long)gridDim.x * 4;
  for (long long t = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); t < T; t += stride) {
    const Slots sl = token_slots(slot_rows, t, topk, rows, status);
    float gate = 0.f, dgate = 0.f;
    if (lane < topk) gate = gates[t * topk + lane];
    for (int c0 = 0; c0 < H; c0 += 64 * V * U) {
      float d[U][V];
      int c[U], skip[U];   // of a chunk's elements the first `skip` belong to the chunk before
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c1 = c0 + (u * 64 + lane) * V;
        c[u] = c1 < H ? min(c1, H - V) : -1;
        skip[u] = c1 - c[u];
        Reg<DOut, V> v;
        if (c[u] >= 0) v = load<DOut, V>(dout + t * H + c[u]);
#pragma unroll
        for (int i = 0; i < V; ++i) d[u][i] = c[u] >= 0 ? (float)v[i] : 0.f;
      }
      for (uint64_t m = sl.mask; m; m &= m - 1) {
        const int j = (int)__builtin_ctzll(m);
        const long long r = (long long)__builtin_amdgcn_readlane(sl.row, j) * H;
        const float g = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(gate), j));
        Reg<Y, V> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (c[u] >= 0) v[u] = load<Y, V>(y + r + c[u]);
        float dot = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (c[u] >= 0) {
            Reg<Y, V> o;
#pragma unroll
            for (int i = 0; i < V; ++i) {
              if (i >= skip[u]) dot = fmaf((float)v[u][i], d[u][i], dot);
              o[i] = (Y)(g * d[u][i]);
            }
            store<Y, V>(dy + r + c[u], o);
          }
        dot = wave_sum(dot);
        if (lane == j) dgate += dot;
      }
    }
    if (lane < topk) dgates[t * topk + lane] = dgate;
  }
}

// ---- host -------------------------------------------------------------------------

// Workgroups of four waves, one unit a wave; past kMaxBlocks of them each wave takes several.
constexpr long long kMaxBlocks = 1 << 20;
unsigned blocks_for(long long units) {
  const long long n = (units + 3) / 4;
  return (unsigned)(n < kMaxBlocks ? n : kMaxBlocks);
}

// Columns that the kernels count in 32 bits, with what lies past the last step of theirs.
constexpr int64_t kMaxColumns = INT32_MAX - 4096;

// What the row operators have in common.
int check_rows(const int32_t* slot_rows, int32_t T, int32_t topk, int64_t rows, int64_t width,
               const void* workspace) {
  if (T < 0 || rows < 0 || width < 1 || topk < 1) return MOE_ERR_INVALID_ARG;
  if (topk > kMaxTopk || rows > INT32_MAX || width > INT32_MAX) return MOE_ERR_UNSUPPORTED;
  if (T > 0 && !slot_rows) return MOE_ERR_INVALID_ARG;
  if (!aligned(slot_rows, 4) || !aligned(workspace, 256)) return MOE_ERR_ALIGNMENT;
  return MOE_OK;
}

struct SortPlan {
  long long slots;
  int chunk, chunks;
};
bool sort_plan(int32_t T, int32_t topk, int32_t E, SortPlan* p) {
  if (T < 0 || topk < 1 || topk > kMaxTopk || E < 1 || E > kMaxExperts) return false;
  p->slots = (long long)T * topk;
  if (p->slots > INT32_MAX - (1 << 24)) return false;   // (indices past the last chunk stay below 2^31)
  const long long spread = (long long)kChunk * kMaxChunks;
  p->chunk = kChunk * (int)((p->slots + spread - 1) / spread);
  for (int c = kLeastChunk; c < kChunk; c *= 2)
    if ((p->slots + c - 1) / c * E <= kMaxCounts) {
      p->chunk = c;
      break;
    }
  if (p->slots <= kOneLaunch) p->chunk = kOneLaunch;
  p->chunks = p->slots <= kOneLaunch ? 1 : (int)((p->slots + p->chunk - 1) / p->chunk);
  return true;
}

template <class In, class Out, bool kWeighted>
int launch_sum_rows(const void* y, const int32_t* slot_rows, const float* gates, void* out, int T, int topk,
                    long long rows, int H, uint32_t* status, hipStream_t s) {
  constexpr int V = 8;
  if (H >= V) {
    const int blocks = (H + 64 * V - 1) / (64 * V);
    sum_rows_kernel<In, Out, kWeighted, V><<<blocks_for((long long)T * blocks), 256, 0, s>>>(
        (const In*)y, slot_rows, gates, (Out*)out, T, topk, rows, H, blocks, status);
  } else {
    sum_rows_kernel<In, Out, kWeighted, 1><<<blocks_for(T), 256, 0, s>>>(
        (const In*)y, slot_rows, gates, (Out*)out, T, topk, rows, H, 1, status);
  }
  return done();
}

int sum_rows(bool weighted, const void* y, const int32_t* slot_rows, const float* gates, void* out, int32_t T,
             int32_t topk, int64_t rows, int32_t H, int32_t y_type, int32_t out_type, void* workspace,
             void* stream) {
  const int bad = check_rows(slot_rows, T, topk, rows, H, workspace);
  if (bad) return bad;
  if (H > kMaxColumns) return MOE_ERR_UNSUPPORTED;
  if (!type_ok(y_type) || !type_ok(out_type)) return MOE_ERR_INVALID_ARG;
  if (T == 0) return MOE_OK;
  if (!out || (rows > 0 && !y) || (weighted && !gates)) return MOE_ERR_INVALID_ARG;
  if (!aligned(y, type_size(y_type)) || !aligned(out, type_size(out_type)) || !aligned(gates, 4)) return MOE_ERR_ALIGNMENT;
  if (rows > 0 && y == out) return MOE_ERR_INVALID_ARG;
  const hipStream_t s = (hipStream_t)stream;
  uint32_t* st = (uint32_t*)workspace;
#define MOE_SUM_ROWS(In, Out)                                                                          \
  return weighted ? launch_sum_rows<In, Out, true>(y, slot_rows, gates, out, T, topk, rows, H, st, s) \
                  : launch_sum_rows<In, Out, false>(y, slot_rows, nullptr, out, T, topk, rows, H, st, s)
  if (y_type == MOE_BF16 && out_type == MOE_BF16) MOE_SUM_ROWS(__bf16, __bf16);
  if (y_type == MOE_BF16) MOE_SUM_ROWS(__bf16, float);
  if (out_type == MOE_BF16) MOE_SUM_ROWS(float, __bf16);
  MOE_SUM_ROWS(float, float);
#undef MOE_SUM_ROWS
}

template <class DOut, class Y>
int launch_combine_grad(const void* dout, const void* y, const int32_t* slot_rows, const float* gates, void* dy,
                        float* dgates, int T, int topk, long long rows, int H, uint32_t* st, hipStream_t s) {
  const unsigned blocks = blocks_for(T);
#define MOE_COMBINE_GRAD(V, U)                                                                             \
  combine_grad_kernel<DOut, Y, V, U><<<blocks, 256, 0, s>>>((const DOut*)dout, (const Y*)y, slot_rows,     \
                                                             gates, (Y*)dy, dgates, T, topk, rows, H, st)
  if (H < 8) MOE_COMBINE_GRAD(1, 1);
  else if (H <= 512) MOE_COMBINE_GRAD(8, 1);
  else MOE_COMBINE_GRAD(8, 4);
#undef MOE_COMBINE_GRAD
  return done();
}

}  // namespace

extern "C" size_t moe_sort_scratch_size(int32_t T, int32_t topk, int32_t E) {
  SortPlan p;
  if (!sort_plan(T, topk, E, &p) || p.chunks <= 1) return 0;
  return (size_t)p.chunks * E * sizeof(uint32_t);
}

extern "C" int moe_sort_by_expert(const int32_t* expert_ids, const float* gates, int32_t* expert_offsets,
                                  int32_t* token_ids, float* gate_w, int32_t* slot_rows, int32_t T,
                                  int32_t topk, int32_t E, int32_t first_expert, void* scratch,
                                  size_t scratch_bytes, void* stream) {
  if (T < 0 || topk < 1 || E < 1) return MOE_ERR_INVALID_ARG;
  SortPlan p;
  if (!sort_plan(T, topk, E, &p)) return MOE_ERR_UNSUPPORTED;
  if (!expert_offsets || (T > 0 && (!expert_ids || !gates || !token_ids || !gate_w || !slot_rows)))
    return MOE_ERR_INVALID_ARG;
  for (const void* q : {(const void*)expert_ids, (const void*)gates, (const void*)expert_offsets,
                        (const void*)token_ids, (const void*)gate_w, (const void*)slot_rows, (const void*)scratch})
    if (!aligned(q, 4)) return MOE_ERR_ALIGNMENT;
  const size_t need = moe_sort_scratch_size(T, topk, E);
  if (need > 0 && (!scratch || scratch_bytes < need)) return MOE_ERR_WORKSPACE;
  int bits = 0;
  while ((1 << bits) < E) ++bits;
  const SortArgs a = {expert_ids, gates, expert_offsets, token_ids, gate_w, slot_rows, (uint32_t*)scratch,
                      (int)p.slots, topk, E, first_expert, bits, p.chunk, p.chunks};
  const hipStream_t s = (hipStream_t)stream;
  if (p.chunks == 1) {
    constexpr int kParts = 8192;
    int waves = (int)((p.slots + 63) / 64);
    waves = waves < 1 ? 1 : waves;
    waves = waves < kOneThreads / 64 ? waves : kOneThreads / 64;
    waves = waves < kParts / E ? waves : kParts / E;
    SortArgs one = a;
    one.chunk = waves * 64 * (int)((p.slots + waves * 64 - 1) / (waves * 64));
    sort_place_kernel<kOneThreads, kParts, true><<<1, waves * 64, 0, s>>>(one);
    return done();
  }
  sort_count_kernel<<<p.chunks, kPlaceThreads, 0, s>>>(a);
  if (hipGetLastError() != hipSuccess) return MOE_ERR_HIP;
  sort_place_kernel<kPlaceThreads, kPlaceThreads / 64 * kMaxExperts, false><<<p.chunks, kPlaceThreads, 0, s>>>(a);
  return done();
}

extern "C" int moe_dispatch_rows(const void* x, const int32_t* slot_rows, void* out, int32_t T, int32_t topk,
                                 int64_t rows, int64_t row_bytes, void* workspace, void* stream) {
  const int bad = check_rows(slot_rows, T, topk, rows, row_bytes, workspace);
  if (bad) return bad;
  if (T == 0 || rows == 0) return MOE_OK;
  if (!x || !out || x == out) return MOE_ERR_INVALID_ARG;
  const hipStream_t s = (hipStream_t)stream;
  uint32_t* st = (uint32_t*)workspace;
#define MOE_DISPATCH(V, U)                                                                                \
  const int blocks = (int)((row_bytes + 64 * V * U - 1) / (64 * V * U));                                  \
  dispatch_kernel<V, U><<<blocks_for((long long)T * blocks), 256, 0, s>>>(                                \
      (const uint8_t*)x, slot_rows, (uint8_t*)out, T, topk, rows, row_bytes, blocks, st)
  if (row_bytes >= 16) {
    MOE_DISPATCH(16, 2);
  } else {
    MOE_DISPATCH(1, 1);
  }
#undef MOE_DISPATCH
  return done();
}

extern "C" int moe_dispatch_rows_grad(const void* d, const int32_t* slot_rows, void* dx, int32_t T, int32_t topk,
                                      int64_t rows, int32_t H, int32_t d_type, int32_t dx_type, void* workspace,
                                      void* stream) {
  return sum_rows(false, d, slot_rows, nullptr, dx, T, topk, rows, H, d_type, dx_type, workspace, stream);
}

extern "C" int moe_combine_rows(const void* y, const int32_t* slot_rows, const float* gates, void* out, int32_t T,
                                int32_t topk, int64_t rows, int32_t H, int32_t y_type, int32_t out_type,
                                void* workspace, void* stream) {
  return sum_rows(true, y, slot_rows, gates, out, T, topk, rows, H, y_type, out_type, workspace, stream);
}

extern "C" int moe_combine_rows_grad(const void* dout, const void* y, const int32_t* slot_rows, const float* gates,
                                     void* dy, float* dgates, int32_t T, int32_t topk, int64_t rows, int32_t H,
                                     int32_t dout_type, int32_t y_type, void* workspace, void* stream) {
  const int bad = check_rows(slot_rows, T, topk, rows, H, workspace);
  if (bad) return bad;
  if (H > kMaxColumns) return MOE_ERR_UNSUPPORTED;
  if (!type_ok(dout_type) || !type_ok(y_type)) return MOE_ERR_INVALID_ARG;
  if (T == 0) return MOE_OK;
  if (!dout || !gates || !dgates || (rows > 0 && (!y || !dy))) return MOE_ERR_INVALID_ARG;
  if (!aligned(dout, type_size(dout_type)) || !aligned(y, type_size(y_type)) || !aligned(dy, type_size(y_type)) ||
      !aligned(gates, 4) || !aligned(dgates, 4))
    return MOE_ERR_ALIGNMENT;
  if (rows > 0 && dout == dy) return MOE_ERR_INVALID_ARG;
  const hipStream_t s = (hipStream_t)stream;
  uint32_t* st = (uint32_t*)workspace;
#define MOE_GRAD(DOut, Y) \
  return launch_combine_grad<DOut, Y>(dout, y, slot_rows, gates, dy, dgates, T, topk, rows, H, st, s)
  if (dout_type == MOE_BF16 && y_type == MOE_BF16) MOE_GRAD(__bf16, __bf16);
  if (dout_type == MOE_BF16) MOE_GRAD(__bf16, float);
  if (y_type == MOE_BF16) MOE_GRAD(float, __bf16);
  MOE_GRAD(float, float);
#undef MOE_GRAD
}

extern "C" int moe_experts_abi_version(void) { return 100; }
