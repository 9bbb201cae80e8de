// The router's kernel and what it shares with the gradient's: see route.hip for the method.
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
  int32_t groups, top_groups, group_size, group_best;
  int32_t group_chunks;                          // 16-byte chunks of a group, 0 where a chunk may hold two groups' experts
  int32_t group_lanes;                           // lanes of a row that share a group then
  uint32_t group_mul;                            // e * group_mul >> 16 = e / group_size
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

// Rows of a selection that groups limit: in a unit of its own.
void start_route_groups(const RouteArgs& a, int32_t dtype, bool bal, dim3 grid, hipStream_t stream);

namespace {

constexpr int kRowLanes = 8;                     // lanes that share a row
constexpr int kRouteThreads = 256;
constexpr int kRouteWaves = kRouteThreads / 64;
constexpr int kRowsPerPass = kRouteThreads / kRowLanes;
constexpr float kNone = -INFINITY;

// How near two values v = s + bias, or sums of two, may be for 32 bits to hold them in another order.  `bias` bounds their biases' magnitude, so
// s <= |v| + bias.  A score is exp of a difference d <= 0, or nearly: the argument is off by |d| 2^-23, the exp and, for the softmax, the
// sum of all of them by 2^-19 more, so s is off by s 2^-18 while s > 2^-11 (|d| < 8) and by s 2^-15 at least down to the smallest.
__device__ __forceinline__ float near_by(float v, float bias) {
  const float s = fabsf(v) + bias;
  return 0x1p-17f * s + 0x1p-14f * fminf(s, 0x1p-11f) + FLT_MIN;
}

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
__device__ __forceinline__ double entry_of(double v, int e) {  // the same of 64-bit values, less their last eight bits
  const uint64_t bits = __builtin_bit_cast(uint64_t, v + 0.0) & ~uint64_t(0xff);
  return __builtin_bit_cast(double, bits | static_cast<uint32_t>(v < 0.0 ? e : 255 - e));
}
__device__ __forceinline__ int id_of(double entry) {
  const uint64_t bits = __builtin_bit_cast(uint64_t, entry);
  const int low = static_cast<int>(bits & 0xff);
  return bits >> 63 ? low : 255 - low;
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

// grid: (runs, layers).  KL: the smallest of 4, 8 and 16 that is not below k.
template <class T, int CH, int KL, bool BAL, bool BIAS, bool GROUPS>
__global__ __launch_bounds__(kRouteThreads, 2) void route_main(RouteArgs a) {
  constexpr int V = kChunk<T>, M = CH * V, KS = (KL + kRowLanes - 1) / kRowLanes;
  constexpr int kList = KL < 8 ? 16 : 2 * KL;  // elements of a row's list
  __shared__ double list[kRowsPerPass][kList];
  __shared__ alignas(16) float copy[kRowsPerPass][M * kRowLanes + 4];  // the rows' logits: rows in different banks
  __shared__ float2 chosen[kRowsPerPass][KS * kRowLanes];
  __shared__ uint32_t count[BAL ? TACG_MAX_EXPERTS : 1];
  __shared__ float mass[BAL ? kRouteWaves : 1][BAL ? TACG_MAX_EXPERTS : 1];
  __shared__ float squares[kRouteWaves];
  __shared__ uint32_t routed[kRouteWaves];
  // GROUPS: the two largest values of each chunk of a row (rows in different banks, two by two), the groups' scores, and the chosen
  // experts' values in order
  constexpr int kPairs = CH * kRowLanes, kPairStride = (kPairs + 15) / 16 * 16 + 8;
  __shared__ float2 two[GROUPS ? kRowsPerPass : 1][GROUPS ? kPairStride : 1];
  __shared__ float group_score[GROUPS ? kRowsPerPass : 1][GROUPS ? TACG_MAX_GROUPS + 1 : 1];
  __shared__ double group_score64[GROUPS ? kRowsPerPass : 1][GROUPS ? TACG_MAX_GROUPS + 1 : 1];
  __shared__ alignas(16) float bias_of[GROUPS && BIAS ? TACG_MAX_EXPERTS : 4];  // the layer's
  __shared__ float ranked[GROUPS && BIAS ? kRowsPerPass : 1][GROUPS && BIAS ? KL + 2 : 1];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, sub = lane & (kRowLanes - 1);
  const int l = blockIdx.y;
  const Run run = run_of(a, blockIdx.x);
  const int E = a.E, k = a.k;
  const T* layer = static_cast<const T*>(a.logits) + l * a.stride_layer;
  double* mine = list[tid >> 3];
  float2* slots = chosen[tid >> 3];
  float* logit = copy[tid >> 3];
  float acc[BAL ? M : 1];
  float sq = 0.0f;
  uint32_t live = 0;
  if (BAL) {
#pragma unroll
    for (int i = 0; i < (BAL ? M : 1); ++i) acc[i] = 0.0f;
    for (int e = tid; e < E; e += kRouteThreads) count[e] = 0;
    if (tid == 0 && run.start) a.arrived[static_cast<int64_t>(run.family) * a.n_layers + l] = 0;
    __syncthreads();
  }
  if constexpr (GROUPS && BIAS) {
    for (int e = tid; e < TACG_MAX_EXPERTS; e += kRouteThreads) bias_of[e] = e < E ? a.bias[l * E + e] : 0.0f;
    __syncthreads();
  }
  auto bias_at = [&](int e) {
    if constexpr (GROUPS) return bias_of[e];
    else return a.bias[l * E + e];
  };
  // whether the sum over all experts is needed
  const bool all = BAL || BIAS || a.norm != nullptr || (a.softmax && !a.renorm);
  for (int64_t base = run.first; base < run.last; base += kRowsPerPass) {
    const int64_t t = base + (tid >> 3);
    const bool in = t < run.last;
    const T* row = layer + (in ? t : run.first) * a.stride_token;
    float x[M];
    load_row<T, CH>(row, sub, E, a.vec, x);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < M; i += 2) bad |= __builtin_isunordered(x[i], x[i + 1]);
    float top, bound = 0.0f;
    if constexpr (BIAS || GROUPS) {
      top = x[0];
#pragma unroll
      for (int i = 1; i < M; ++i) top = vmax(top, x[i]);
      top = row_max(top);
    } else {
      bound = lower_bound<KL>(x, top);
    }
    bad |= top == INFINITY;
    if (__any(bad)) {  // a NaN or +inf: the row is not routed
      const uint64_t m = __ballot(bad) >> (lane & ~(kRowLanes - 1));
      if ((m & 0xff) != 0) {
        if (in && sub == 0) atomicOr(a.err, TACG_ERR_VALUE);
        top = bound = kNone;
#pragma unroll
        for (int i = 0; i < M; ++i) x[i] = kNone;
      }
    }
#pragma unroll
    for (int i = 0; i < M; i += 4)
      *reinterpret_cast<float4*>(logit + element<T, CH>(i, sub)) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const bool some = top > kNone;
    uint32_t mask = 0;
    // GROUPS: the groups that the selection keeps, a bit each
    uint32_t kept = 0;
    double inverse64 = 1.0;
    const float from = some ? top : 0.0f;
    auto value64 = [&](float v, int e) {
      double s = a.softmax ? exp(static_cast<double>(v) - static_cast<double>(from)) * inverse64 : 1.0 / (1.0 + exp(-static_cast<double>(v)));
      if constexpr (BIAS) s += static_cast<double>(bias_of[e]);
      return s;
    };
    auto allowed = [&](int e) { return (kept >> (((e * a.group_mul) >> 16) & 31)) & 1u; };
    // the sum of all scores, in 64 bits: where a bias is added to them
    auto total64 = [&] {
      if (!BIAS || !a.softmax) return;
      double sum = 0.0;
      for (int e = sub; e < E; e += kRowLanes) sum += exp(static_cast<double>(logit[e]) - static_cast<double>(from));
#pragma unroll
      for (int o = 1; o < kRowLanes; o <<= 1) sum += __shfl_xor(sum, o, 64);
      inverse64 = sum > 0.0 ? 1.0 / sum : 0.0;
    };
    // the groups that are kept, of the values y (logits, or scores with a bias; -inf: not available)
    auto keep_groups = [&](const float (&y)[M], float most_bias, auto value32) {
      // the sum of a group's best values from the best logits; those of a bias are there
      auto sum32 = [&](float first, float second) {
        if (BIAS) return a.group_best > 1 && second > kNone ? first + second : first;
        if (a.group_best == 1 || first == kNone) return first;
        auto s = [&](float v) { return v == kNone ? 0.0f : a.softmax ? __expf(v - from) : sigmoid(v); };
        return s(first) + s(second);
      };
      auto take = [&](float& first, float& second, float f, float s) {
        second = vmax3(vmin(first, f), second, s);
        first = vmax(first, f);
      };
      float* score = group_score[tid >> 3];
      float2* pairs = two[tid >> 3];
      if (a.group_chunks > 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          float first = y[c * V], second = kNone;
#pragma unroll
          for (int i = 1; i < V; ++i) {
            second = vmax(second, vmin(first, y[c * V + i]));
            first = vmax(first, y[c * V + i]);
          }
          pairs[c * kRowLanes + sub] = make_float2(first, second);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int n = a.group_chunks;
        for (int g = sub; g < a.groups; g += kRowLanes) {
          float first = kNone, second = kNone;
          int i = sub % n;  // lanes start in different banks
          for (int c = 0; c < n; ++c) {
            const float2 v = pairs[g * n + i];
            take(first, second, v.x, v.y);
            i = i + 1 == n ? 0 : i + 1;
          }
          score[g] = sum32(first, second);
        }
      } else {
        const int lanes = a.group_lanes, part = sub & (lanes - 1);
        for (int g = lanes > 1 ? sub / lanes : sub; g < a.groups; g += kRowLanes) {
          float first = kNone, second = kNone;
          for (int e = g * a.group_size + part; e < (g + 1) * a.group_size; e += lanes)
            if (logit[e] > kNone) take(first, second, value32(logit[e], e), kNone);
          if (lanes > 1) take(first, second, across<kSwap1>(first), across<kSwap1>(second));
          if (lanes > 2) take(first, second, across<kSwap2>(first), across<kSwap2>(second));
          score[g] = sum32(first, second);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      kept = 0;
      bool near = false;
      const bool exact = !BIAS && a.group_best == 1;  // logits
      for (int g = sub; g < a.groups; g += kRowLanes) {
        const float own = score[g], margin = near_by(own, 2.0f * most_bias);
        int better = 0;
        for (int h = 0; h < a.groups; ++h) {
          const float d = score[h] - own;
          better += score[h] > own || (score[h] == own && h < g);
          near |= !exact && h != g && fabsf(d) <= margin;
        }
        if (own > kNone && better < a.top_groups) kept |= 1u << g;
      }
      if (__any(near)) {
        total64();
        double* score64 = group_score64[tid >> 3];
        for (int g = sub; g < a.groups; g += kRowLanes) {
          double first = -INFINITY, second = -INFINITY;
          for (int e = g * a.group_size; e < (g + 1) * a.group_size; ++e) {
            if (!(logit[e] > kNone)) continue;
            const double v = value64(logit[e], e);
            if (v > first) second = first, first = v;
            else if (v > second) second = v;
          }
          score64[g] = a.group_best > 1 && second > -INFINITY ? first + second : first;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        kept = 0;
        for (int g = sub; g < a.groups; g += kRowLanes) {
          int better = 0;
          for (int h = 0; h < a.groups; ++h) better += score64[h] > score64[g] || (score64[h] == score64[g] && h < g);
          if (score64[g] > -INFINITY && better < a.top_groups) kept |= 1u << g;
        }
      }
      kept |= across<kSwap1>(static_cast<int>(kept));
      kept |= across<kSwap2>(static_cast<int>(kept));
      kept |= across<kMirror>(static_cast<int>(kept));
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    // y without the experts of other groups
    auto limit = [&](float (&y)[M]) {
      if (a.group_chunks > 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const bool in = allowed((c * kRowLanes + sub) * V);
#pragma unroll
          for (int i = 0; i < V; ++i) y[c * V + i] = in ? y[c * V + i] : kNone;
        }
      } else {
#pragma unroll
        for (int i = 0; i < M; ++i) y[i] = allowed(element<T, CH>(i, sub)) ? y[i] : kNone;
      }
    };
    if constexpr (GROUPS && !BIAS) {
      keep_groups(x, 0.0f, [](float v, int) { return v; });
      float y[M], unused;
#pragma unroll
      for (int i = 0; i < M; ++i) y[i] = x[i];
      limit(y);
      bound = lower_bound<KL>(y, unused);
      mask = at_least(y, vmax(bound, -FLT_MAX));
    }
    if constexpr (!BIAS && !GROUPS) mask = at_least(x, vmax(bound, -FLT_MAX));
    // scores: exp(x - top) (softmax, to be divided by their sum) or the sigmoid, in place of the logits
    const float shift = some ? top : 0.0f;
    float total = 0.0f, inverse = 0.0f, widest = 0.0f;
    if (all) {
      uint32_t away = 0;  // BIAS: which logits are -inf
      if constexpr (BIAS) away = ~at_least(x, -FLT_MAX);
      if (a.softmax) {
#pragma unroll
        for (int i = 0; i < M; ++i) x[i] = __expf(x[i] - shift), total += x[i];
      } else {
#pragma unroll
        for (int i = 0; i < M; ++i) x[i] = sigmoid(x[i]), total += x[i];
      }
      total = row_sum(total);
      inverse = total > 0.0f ? 1.0f / total : 0.0f;
      if (BAL && in) {
#pragma unroll
        for (int i = 0; i < (BAL ? M : 1); ++i) acc[i] += x[i] * inverse;
      }
      if constexpr (BIAS) {
        const float f = a.softmax ? inverse : 1.0f;
        float most_bias = 0.0f;
#pragma unroll
        for (int i = 0; i < M; ++i) {
          const int e = element<T, CH>(i, sub);
          const float b = bias_at(GROUPS ? e : e < E ? e : 0);
          if constexpr (GROUPS) most_bias = fmaxf(most_bias, fabsf(b));
          x[i] = (away >> (M - 1 - i)) & 1u ? kNone : x[i] * f + b;
        }
        if constexpr (GROUPS) {
          most_bias = row_max(most_bias);
          keep_groups(x, most_bias, [&](float v, int e) { return (a.softmax ? __expf(v - shift) * inverse : sigmoid(v)) + bias_of[e]; });
          limit(x);
          widest = most_bias;
        }
        float unused;
        bound = lower_bound<KL>(x, unused);
        if constexpr (GROUPS) bound -= near_by(bound, most_bias);
        mask = at_least(x, vmax(bound, -FLT_MAX));
      }
    }
    // what the selection orders by, of one expert
    using Key = std::conditional_t<GROUPS && BIAS, double, float>;
    auto value = [&](float v, int e) {
      if constexpr (BIAS) v = (a.softmax ? __expf(v - shift) * inverse : sigmoid(v)) + bias_at(e);
      return v;
    };
    auto order_by = [&](float v, int e) {
      if constexpr (GROUPS && BIAS) return value64(v, e);
      else return value(v, e);
    };
    // the list: each lane's elements after those of the lanes before it
    int n = __popc(mask), before = 0;
    {
      int o = across<kSwap1>(n);
      before += sub & 1 ? o : 0;
      n += o;
      o = across<kSwap2>(n);
      before += sub & 2 ? o : 0;
      n += o;
      o = across<kMirror>(n);
      before += sub & 4 ? o : 0;
      n += o;
    }
    int most = 0;  // of the wave's rows
#pragma unroll
    for (int r = 0; r < 64; r += kRowLanes) {
      const int v = __builtin_amdgcn_readlane(n, r);
      most = v > most ? v : most;
    }
    int id[KS];   // of slots sub, sub + 8: expert and its logit
    float w[KS];
#pragma unroll
    for (int q = 0; q < KS; ++q) id[q] = -1, w[q] = kNone;
    if (most <= kList) {
      int32_t* ids = reinterpret_cast<int32_t*>(mine);  // before the entries
#pragma unroll
      for (int q = 0; q < KS; ++q) slots[sub + q * kRowLanes] = make_float2(__int_as_float(-1), kNone);
      if constexpr (M <= 8) {
#pragma unroll
        for (int i = 0; i < M; ++i)
          if ((mask >> (M - 1 - i)) & 1u) ids[before++] = element<T, CH>(i, sub);
      } else {
        while (__any(mask != 0)) {
          if (mask != 0) {
            const int i = __clz(mask) - (32 - M);
            mask &= ~(1u << (M - 1 - i));
            ids[before++] = element<T, CH>(i, sub);
          }
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      // entries sub, sub + 8, ... of the lane; those past the end order behind all others
      auto place = [&](auto entries, auto value_of) {
        constexpr int N = entries.value;
        constexpr bool again = std::is_same_v<decltype(value_of(0.0f, 0)), double>;  // the ids are those of the entries before
        int e[N], larger[N];
        float x[N];
        double own[N];
#pragma unroll
        for (int q = 0; q < N; ++q) {
          const bool have = sub + q * kRowLanes < n;
          e[q] = !have ? 0 : again ? id_of(mine[sub + q * kRowLanes]) : ids[sub + q * kRowLanes];
          x[q] = logit[e[q]];
          own[q] = have ? entry_of(value_of(x[q], e[q]), e[q]) : -INFINITY;
          larger[q] = 0;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int q = 0; q < N; ++q) mine[sub + q * kRowLanes] = own[q];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int first = 0; first < N * kRowLanes; first += kRowLanes) {
          double other[kRowLanes];
#pragma unroll
          for (int i = 0; i < kRowLanes; ++i) other[i] = mine[first + i];
#pragma unroll
          for (int i = 0; i < kRowLanes; ++i)
#pragma unroll
            for (int q = 0; q < N; ++q) larger[q] += other[i] > own[q];
        }
#pragma unroll
        for (int q = 0; q < N; ++q)
          if (sub + q * kRowLanes < n && larger[q] < k) slots[larger[q]] = make_float2(__int_as_float(e[q]), x[q]);
        if constexpr (GROUPS && BIAS && !again) {
#pragma unroll
          for (int q = 0; q < N; ++q)
            if (sub + q * kRowLanes < n && larger[q] <= k) ranked[tid >> 3][larger[q]] = static_cast<float>(own[q]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      };
      auto place_all = [&](auto value_of) {
        if constexpr (KL == 16) {
          if (most <= 3 * kRowLanes) place(std::integral_constant<int, 3>(), value_of);
          else place(std::integral_constant<int, 4>(), value_of);
        } else {
          if (most <= kRowLanes) place(std::integral_constant<int, 1>(), value_of);
          else place(std::integral_constant<int, 2>(), value_of);
        }
      };
      if constexpr (GROUPS && BIAS) {
        float* order = ranked[tid >> 3];
        for (int j = sub; j <= k; j += kRowLanes) order[j] = kNone;
        place_all(value);
        // neighbours that 32 bits may hold in another order, the first that is not chosen among them
        bool near = false;
        for (int j = sub; j < k; j += kRowLanes)
          near |= order[j + 1] > kNone && order[j] - order[j + 1] <= near_by(order[j], widest);
        if (__any(near)) {
          total64();
          place_all(value64);
        }
      } else {
        place_all(value);
      }
#pragma unroll
      for (int q = 0; q < KS; ++q) {
        const float2 v = slots[sub + q * kRowLanes];
        id[q] = __float_as_int(v.x);
        w[q] = v.y;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    } else {
      // k passes: the best after the last winner in (value descending, id ascending)
      if constexpr (GROUPS && BIAS) total64();
      Key last = INFINITY;
      int last_e = -1;
      for (int j = 0; j < k; ++j) {
        Key best = kNone;
        int at = 0x7fffffff;
        for (int i = 0; i < M; ++i) {
          const int e = element<T, CH>(i, sub);
          if (e >= E || (GROUPS && !allowed(e))) continue;
          const Key v = logit[e] > kNone ? order_by(logit[e], e) : static_cast<Key>(kNone);
          const bool after = v < last || (v == last && e > last_e);
          if (after && v > best) best = v, at = e;
        }
#pragma unroll
        for (int o = 1; o < kRowLanes; o <<= 1) {
          const Key v = __shfl_xor(best, o, 64);
          const int e = __shfl_xor(at, o, 64);
          if (v > best || (v == best && e < at)) best = v, at = e;
        }
#pragma unroll
        for (int q = 0; q < KS; ++q)
          if (j == sub + q * kRowLanes && best > kNone) id[q] = at, w[q] = logit[at];
        last = best;
        last_e = best > kNone ? at : 0x7fffffff;
      }
    }
    // gates of the selected
    if (a.softmax) {
      float high = shift;
      if (BIAS && a.renorm) {
        high = kNone;
#pragma unroll
        for (int q = 0; q < KS; ++q) high = vmax(high, w[q]);
        high = row_max(high);
        high = high == kNone ? 0.0f : high;
      }
#pragma unroll
      for (int q = 0; q < KS; ++q) w[q] = __expf(w[q] - high);
    } else {
#pragma unroll
      for (int q = 0; q < KS; ++q) w[q] = sigmoid(w[q]);
    }
    float factor = 1.0f;
    if (a.renorm) {
      float part = 0.0f;
#pragma unroll
      for (int q = 0; q < KS; ++q) part += w[q];
      part = row_sum(part);
      factor = part > 0.0f ? 1.0f / part : 0.0f;
    } else if (a.softmax) {
      factor = inverse;
    }
    const int64_t at = static_cast<int64_t>(l) * a.n_tokens + t;
    if (in) {
#pragma unroll
      for (int q = 0; q < KS; ++q) {
        const int j = sub + q * kRowLanes;
        if (j < k) {
          a.trace[at * k + j] = static_cast<int16_t>(id[q]);
          a.gate[at * k + j] = w[q] * factor * a.scale;  // the share first: factor * scale may be more than 32 bits hold
          if (BAL && id[q] >= 0) atomicAdd(&count[id[q]], 1u);
        }
      }
    }
    if (all) {
      const float norm = a.softmax ? (some ? top + __logf(total) : kNone) : total;
      if (a.norm != nullptr && in && sub == 0) a.norm[at] = norm;
      if (BAL && in && some && sub == 0) {
        live += 1;
        if (a.softmax) sq += norm * norm;
      }
    }
  }
  if (!BAL) return;
  // the run's sums: rows of a wave, then the waves in order
#pragma unroll
  for (int i = 0; i < (BAL ? M : 1); ++i) {
    acc[i] = rows_sum(acc[i]);
    const int e = element<T, CH>(i, sub);
    if (lane < kRowLanes && e < E) mass[wave][e] = acc[i];
  }
  sq = rows_sum(sq);
#pragma unroll
  for (int o = kRowLanes; o < 64; o <<= 1) live += __shfl_xor(live, o, 64);
  if (lane == 0) squares[wave] = sq, routed[wave] = live;
  barrier_after_lds_atomics();
  const int64_t slot = static_cast<int64_t>(l) * gridDim.x + blockIdx.x;
  for (int e = tid; e < E; e += kRouteThreads) {
    float m = mass[0][e];
#pragma unroll
    for (int w = 1; w < (BAL ? kRouteWaves : 1); ++w) m += mass[w][e];
    a.mass[slot * E + e] = m;
    a.count[slot * E + e] = count[e];
  }
  if (tid == 0) {
    double s = 0.0;
    uint32_t n = 0;
#pragma unroll
    for (int w = 0; w < kRouteWaves; ++w) s += squares[w], n += routed[w];
    a.squares[slot] = s;
    a.routed[slot] = n;
  }
}

template <class T, int CH, int KL, bool GROUPS>
void start_main(const RouteArgs& a, bool bal, dim3 grid, hipStream_t s) {
  auto* kernel = a.bias != nullptr ? (bal ? route_main<T, CH, KL, true, true, GROUPS> : route_main<T, CH, KL, false, true, GROUPS>)
                                   : (bal ? route_main<T, CH, KL, true, false, GROUPS> : route_main<T, CH, KL, false, false, GROUPS>);
  kernel<<<grid, kRouteThreads, 0, s>>>(a);
}

template <class T, int CH, bool GROUPS>
void start_main(const RouteArgs& a, bool bal, dim3 grid, hipStream_t s) {
  if (a.k <= 4) start_main<T, CH, 4, GROUPS>(a, bal, grid, s);
  else if (a.k <= 8) start_main<T, CH, 8, GROUPS>(a, bal, grid, s);
  else start_main<T, CH, 16, GROUPS>(a, bal, grid, s);
}

template <class T, bool GROUPS>
void start_main(const RouteArgs& a, bool bal, dim3 grid, hipStream_t s) {
  const int chunks = (a.E + kChunk<T> * kRowLanes - 1) / (kChunk<T> * kRowLanes);
  if constexpr (sizeof(T) == 2) {
    if (chunks <= 1) return start_main<T, 1, GROUPS>(a, bal, grid, s);
  }
  if (chunks <= 2) return start_main<T, 2, GROUPS>(a, bal, grid, s);
  if (chunks <= 4) return start_main<T, 4, GROUPS>(a, bal, grid, s);
  if constexpr (sizeof(T) == 4) start_main<T, 8, GROUPS>(a, bal, grid, s);
}

// All of a call's rows, by the type of its logits.
template <bool GROUPS>
void start_rows(const RouteArgs& a, int32_t dtype, bool bal, dim3 grid, hipStream_t s) {
  if (dtype == TACG_F32) start_main<float, GROUPS>(a, bal, grid, s);
  else if (dtype == TACG_BF16) start_main<Bf16, GROUPS>(a, bal, grid, s);
  else start_main<F16, GROUPS>(a, bal, grid, s);
}

}  // namespace
}  // namespace tacg
