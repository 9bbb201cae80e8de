// What the router's kernels and the gradient's share: see route.hip and route_groups.hip for the methods.
#pragma once

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "tacg_internal.h"

namespace tacg {

struct RouteArgs {
  const void* logits;
  int64_t stride_layer, stride_token;            // elements
  int64_t n_tokens;
  int32_t n_layers, E, k, F, rows;               // rows: of a workgroup's run
  int32_t softmax, renorm, vec;                  // vec: bytes that a load may take at a time
  // groups of experts (1: no limit), how many are kept, by how many of their best; e * group_mul >> 16 = e / group_size
  int32_t groups, top_groups, group_best, group_size;
  uint32_t group_mul;
  int32_t group_pairs;                           // neighbouring 16-byte chunks of a group, two by two; 0: not a whole number
  int32_t group_lanes;                           // lanes of a row that share a group then
  float scale;
  const float* bias;                             // [L][E] or null
  int16_t* trace;
  float* gate;
  float* norm;                                   // [L][N] or null
  float* mass;                                   // workspace: [slots][E]
  uint32_t* count;                               // [slots][E]
  double* squares;                               // [slots]
  uint32_t* routed;                              // [slots]
  uint32_t* arrived;                             // [F][L], for route_reduce
  uint32_t* err;
  // first run and first token of each family; a lane each reads a pair
  int32_t run_off[TACG_MAX_FAMILIES + 1];
  int64_t fam_off[TACG_MAX_FAMILIES + 1];
};

// The rows of a selection that groups limit (route_groups.hip).
void start_route_groups(const RouteArgs& a, int32_t dtype, bool bal, dim3 grid, hipStream_t stream);

namespace {

constexpr int kRowLanes = 8;                     // lanes that share a row
constexpr int kRouteThreads = 256;
constexpr int kRouteWaves = kRouteThreads / 64;
constexpr int kRowsPerPass = kRouteThreads / kRowLanes;
constexpr float kNone = -INFINITY;

struct BackArgs {
  const void* logits;
  int64_t stride_layer, stride_token;
  int64_t n_tokens;
  int32_t n_layers, E, k, F, rows, softmax, renorm, vec;
  float scale;
  const int16_t* trace;
  const float* norm;
  const uint32_t* D;                             // [F][L][E] or null
  const uint32_t* tokens;                        // [F][L] or null
  const float* grad_gate;                        // [L][N][k] or null
  const float* grad_balance;                     // [F][L] or null
  const float* grad_z;                           // [F][L] or null
  void* grad;                                    // [L][N][E]
  int32_t run_off[TACG_MAX_FAMILIES + 1];
  int64_t fam_off[TACG_MAX_FAMILIES + 1];
};

struct Bf16 { uint16_t bits; };
struct F16 { uint16_t bits; };

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(Bf16 x) { return __uint_as_float(static_cast<uint32_t>(x.bits) << 16); }
__device__ __forceinline__ float widen(F16 x) { return static_cast<float>(__builtin_bit_cast(_Float16, x.bits)); }

// One rounding, to nearest even, of the finished 32-bit value.
__device__ __forceinline__ void narrow(float v, float& o) { o = v; }
__device__ __forceinline__ void narrow(float v, Bf16& o) { o.bits = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v)); }
__device__ __forceinline__ void narrow(float v, F16& o) { o.bits = __builtin_bit_cast(uint16_t, static_cast<_Float16>(v)); }

template <class T>
constexpr int kChunk = 16 / sizeof(T);           // elements of a 16-byte chunk

// A lane's elements of a row: chunk c of the lane starts at element (c * 8 + lane) * kChunk.  Elements past E come as -inf.
// vec: 16 or 8 where every row starts at a multiple of it and holds a whole number of such pieces, else the element's size.
template <class T, int CH>
__device__ __forceinline__ void load_row(const T* row, int sub, int E, int vec, float (&x)[CH * kChunk<T>]) {
  constexpr int V = kChunk<T>;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int at = (c * kRowLanes + sub) * V;
    alignas(16) T piece[V];
    if (vec == 16) {
      if (at < E) *reinterpret_cast<uint4*>(piece) = *reinterpret_cast<const uint4*>(row + at);
#pragma unroll
      for (int j = 0; j < V; ++j) x[c * V + j] = at < E ? widen(piece[j]) : kNone;
    } else if (vec == 8) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int a = at + h * (V / 2);
        if (a < E) *reinterpret_cast<uint2*>(piece + h * (V / 2)) = *reinterpret_cast<const uint2*>(row + a);
#pragma unroll
        for (int j = 0; j < V / 2; ++j) x[c * V + h * (V / 2) + j] = a < E ? widen(piece[h * (V / 2) + j]) : kNone;
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) x[c * V + j] = at + j < E ? widen(row[at + j]) : kNone;
    }
  }
}

template <class T, int CH>
__device__ __forceinline__ void store_row(T* row, int sub, int E, int vec, const float (&x)[CH * kChunk<T>]) {
  constexpr int V = kChunk<T>;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int at = (c * kRowLanes + sub) * V;
    alignas(16) T piece[V];
#pragma unroll
    for (int j = 0; j < V; ++j) narrow(x[c * V + j], piece[j]);
    if (vec == 16) {
      if (at < E) *reinterpret_cast<uint4*>(row + at) = *reinterpret_cast<uint4*>(piece);
    } else if (vec == 8) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (at + h * (V / 2) < E)
          *reinterpret_cast<uint2*>(row + at + h * (V / 2)) = *reinterpret_cast<uint2*>(piece + h * (V / 2));
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (at + j < E) row[at + j] = piece[j];
    }
  }
}

// Exchanges within the eight lanes of a row: with the lane whose number differs in bit 0, in bit 1, in all three.
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kMirror = 0x141;
template <int CTRL>
__device__ __forceinline__ int across(int v) {
  return __builtin_amdgcn_mov_dpp(v, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ float across(float v) {
  return __int_as_float(across<CTRL>(__float_as_int(v)));
}

// The instructions themselves: what they return for a NaN does not matter here, and fmaxf() first quiets every operand.
__device__ __forceinline__ float vmax(float a, float b) {
  float o;
  asm("v_max_f32 %0, %1, %2" : "=v"(o) : "v"(a), "v"(b));
  return o;
}
__device__ __forceinline__ float vmin(float a, float b) {
  float o;
  asm("v_min_f32 %0, %1, %2" : "=v"(o) : "v"(a), "v"(b));
  return o;
}
__device__ __forceinline__ float vmax3(float a, float b, float c) {
  float o;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(o) : "v"(a), "v"(b), "v"(c));
  return o;
}

__device__ __forceinline__ float row_max(float v) {
  v = vmax(v, across<kSwap1>(v));
  v = vmax(v, across<kSwap2>(v));
  return vmax(v, across<kMirror>(v));
}
__device__ __forceinline__ float row_sum(float v) {
  v += across<kSwap1>(v);
  v += across<kSwap2>(v);
  return v + across<kMirror>(v);
}

// v_rcp_f32 is within one unit in the last place; an exact division would cost ten instructions.
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }

__device__ __forceinline__ void order(float& a, float& b) {  // the larger one first
  const float hi = vmax(a, b);
  b = vmin(a, b);
  a = hi;
}
// Sorts a sequence that rises and then falls (or the other way), largest first.
template <int N>
__device__ __forceinline__ void sort_bitonic(float* a) {
  if constexpr (N > 1) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) order(a[i], a[i + N / 2]);
    sort_bitonic<N / 2>(a);
    sort_bitonic<N / 2>(a + N / 2);
  }
}
// Batcher's odd-even merge sort, largest first: 19 exchanges for eight.
template <int N>
__device__ __forceinline__ void sort_all(float (&a)[N]) {
#pragma unroll
  for (int p = 1; p < N; p *= 2)
#pragma unroll
    for (int d = p; d >= 1; d /= 2)
#pragma unroll
      for (int j = d % p; j + d < N; j += 2 * d)
#pragma unroll
        for (int i = j; i < j + d && i + d < N; ++i)
          if (i / (2 * p) == (i + d) / (2 * p)) order(a[i], a[i + d]);
}
// The N largest of the sorted lists of this lane and another; sorted again, or (LAST) only the smallest of them.
template <int N, int CTRL, bool LAST>
__device__ __forceinline__ float merge(float (&a)[N]) {
  float b[N];
#pragma unroll
  for (int i = 0; i < N; ++i) b[i] = vmax(a[i], across<CTRL>(a[N - 1 - i]));
  float low = b[0];
  if constexpr (LAST) {
#pragma unroll
    for (int i = 1; i < N; ++i) low = vmin(low, b[i]);
  } else {
    sort_bitonic<N>(b);
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = b[i];
  }
  return low;
}

// The KL-th largest of the maxima of the row's groups (-inf if there are fewer), and the largest.  Group j of a lane: elements
// j, j + G, j + 2 G, ...: neighbouring experts lie in different ones.
template <int KL, int M>
__device__ __forceinline__ float lower_bound(const float (&y)[M], float& top) {
  constexpr int G = M < 8 ? M : 8;
  float m[G], a[KL];
#pragma unroll
  for (int j = 0; j < G; ++j) {
    if constexpr (M / G == 4) m[j] = vmax(vmax3(y[j], y[j + G], y[j + 2 * G]), y[j + 3 * G]);
    else if constexpr (M / G == 2) m[j] = vmax(y[j], y[j + G]);
    else m[j] = y[j];
  }
  sort_all(m);
#pragma unroll
  for (int i = 0; i < KL; ++i) a[i] = i < G ? m[i < G ? i : 0] : kNone;
  merge<KL, kSwap1, false>(a);
  merge<KL, kSwap2, false>(a);
  top = vmax(a[0], across<kMirror>(a[0]));
  return merge<KL, kMirror, true>(a);
}

// Bit M - 1 - i of the mask: y[i] >= bound.
template <int M>
__device__ __forceinline__ uint32_t at_least(const float (&y)[M], float bound) {
  uint32_t mask = 0;
#pragma unroll
  for (int i = 0; i < M; ++i)
    asm("v_cmp_ge_f32 vcc, %1, %2\n\tv_addc_co_u32 %0, vcc, %0, %0, vcc" : "+v"(mask) : "v"(y[i]), "v"(bound) : "vcc");
  return mask;
}

// A list entry: orders by value, equal values by id, the lower one first.
__device__ __forceinline__ double entry_of(float v, int e) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, static_cast<double>(v + 0.0f));  // -0 and +0 are equal
  return __builtin_bit_cast(double, bits | static_cast<uint32_t>(v < 0.0f ? e : 255 - e));
}
__device__ __forceinline__ int expert_of(double entry) {  // the id of a list entry, whose value is static_cast<float>(entry)
  const int low = static_cast<int>(__builtin_bit_cast(uint64_t, entry) & 255u);
  return entry < 0.0 ? low : 255 - low;
}
struct Run {
  int family;
  int64_t first, last;  // tokens
  bool start;           // the family's first run
};
template <class Args>
__device__ __forceinline__ Run run_of(const Args& a, int run) {
  const int lane = threadIdx.x & 63;  // a lane per family, all tables read at once
  const int next = a.run_off[lane + 1], first = a.run_off[lane];
  const int64_t from = a.fam_off[lane], to = a.fam_off[lane + 1];
  const int f = __popcll(__ballot(lane < a.F && run >= next));
  auto of = [&](int64_t v) {
    return static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v >> 32), f))) << 32 |
                                static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), f)));
  };
  Run r;
  r.family = f;
  const int before = run - __builtin_amdgcn_readlane(first, f);
  r.start = before == 0;
  r.first = of(from) + static_cast<int64_t>(before) * a.rows;
  const int64_t end = r.first + a.rows, last = of(to);
  r.last = end < last ? end : last;
  return r;
}

// Sum over the eight rows of a wave.
__device__ __forceinline__ float rows_sum(float v) {
  v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x128, 0xf, 0xf, true));  // rotated by 8 within 16
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

template <class T, int CH>
__device__ __forceinline__ int element(int i, int sub) {  // the id of a lane's i-th element
  return ((i / kChunk<T>) * kRowLanes + sub) * kChunk<T> + i % kChunk<T>;
}


}  // namespace
}  // namespace tacg
