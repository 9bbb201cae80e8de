// The router of a mixture-of-experts layer: top-k experts and gates from logits, per-expert counts and the balance and z losses
// of every (family, layer) segment, and the gradient of gates and losses to the logits.
//
// A row is the E logits of one token at one layer.  Eight lanes share a row, so a wave holds eight rows; lane i of a row owns
// the 16-byte chunks i, i + 8, i + 16, ... of it, as 32-bit floats in registers.  With s the scores (softmax, or sigmoid) and
// s' = s (softmax) or s / sum s (sigmoid), a segment of T rows with D_e selections and M_e = sum_t s'_e(t) has
//   balance = E / (k T^2) sum_e D_e M_e,   z = 1/T sum_t lse_t^2.
//
// route_main: one pass over the logits.  Selection in a row:
//   * a lane's elements fall into up to eight groups; the k-th largest (4th, 8th or 16th, by the kernel's variant) of the row's group
//     maxima, found by sorting networks within and merges across the lanes, is a lower bound of the k-th largest logit that few
//     more than k elements reach;
//   * those elements' values, with the id below the value's last bit (32-bit value and id in a 64-bit float), go to a list in LDS;
//   * the place of each is the number of larger ones in the list.
//   A row with more such elements than the list holds (many equal ones) is selected by k passes over it instead.  (k passes for every
//   row: 966 us where this takes 140, 58 layers of 8155 rows of 256 in 32 bits with sigmoid scores, counts and loss.)
//   A workgroup takes a run of rows of one segment; its sums of s' (32 bits over a run, then 64), counts, rows and squares go to a
//   slot of the workspace, and route_reduce adds a segment's slots in order in 64 bits, so that results do not depend on the
//   order of execution.  Bound by instruction issue with counts and loss (about 880 vector instructions per eight rows of 256, VALU
//   busy 0.7 of the time, 3.6 TB/s); the selection alone is near memory (48 x 4101 rows of 128: 27 us, 4.1 TB/s).
// route_back: one pass over logits and gradient; with c = d loss / d s' (a constant of the segment) and u the gradient of the scores
//   through the gates, softmax: dx = s (c + u - sum s (c + u) + 2 gz lse / T), sigmoid: dx = (1 - s) (s' (c - sum s' c) + u s).  u s has
//   k entries a row: they are laid into a row of LDS, where each lane reads its own experts' back.  The softmax is computed again, from
//   differences to the row's largest.  Bound by memory: 58 layers of 8155 rows of 256 in 227 us, 4.4 TB/s read and written (a copy
//   reaches 4.8); sigmoid the same.
// Both take rows in pieces of 16 or 8 bytes where every row starts at a multiple of them and holds a whole number, else element by element,
// which costs most: 58 layers of 8155 rows of 255 with sums 223 us (of 256: 140), in 16 bits 312 (148); gradient 476 us (227), in 16 bits
// 476 (177); 48 x 4101 rows of 127, selection alone, 33 us (29), in 16 bits 43 (28).
// With a bias the scores of all experts come before the selection, and the bias is read again in each pass: 48 us against 29 for
// 48 x 4101 rows of 128, 296 against 140 for 58 x 8155 of 256 with sums.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "tacg_internal.h"

namespace tacg {
namespace {

constexpr int kRowLanes = 8;                     // lanes that share a row
constexpr int kRouteThreads = 256;
constexpr int kRouteWaves = kRouteThreads / 64;
constexpr int kRowsPerPass = kRouteThreads / kRowLanes;
constexpr float kNone = -INFINITY;

struct RouteArgs {
  const void* logits;
  int64_t stride_layer, stride_token;            // elements
  int64_t n_tokens;
  int32_t n_layers, E, k, F, rows;               // rows: of a workgroup's run
  int32_t softmax, renorm, vec;                  // vec: bytes that a load may take at a time
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
template <class T, int CH, int KL, bool BAL, bool BIAS>
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
    if constexpr (BIAS) {
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
    if constexpr (!BIAS) mask = at_least(x, vmax(bound, -FLT_MAX));
    // scores: exp(x - top) (softmax, to be divided by their sum) or the sigmoid, in place of the logits
    const float shift = some ? top : 0.0f;
    float total = 0.0f, inverse = 0.0f;
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
#pragma unroll
        for (int i = 0; i < M; ++i) {
          const int e = element<T, CH>(i, sub);
          x[i] = (away >> (M - 1 - i)) & 1u ? kNone : x[i] * f + a.bias[l * E + (e < E ? e : 0)];
        }
        float unused;
        bound = lower_bound<KL>(x, unused);
        mask = at_least(x, vmax(bound, -FLT_MAX));
      }
    }
    // what the selection orders by, of one expert
    auto value = [&](float v, int e) {
      if constexpr (BIAS) v = (a.softmax ? __expf(v - shift) * inverse : sigmoid(v)) + a.bias[l * E + e];
      return v;
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
      auto place = [&](auto entries) {
        constexpr int N = entries.value;
        int e[N], larger[N];
        float x[N];
        double own[N];
#pragma unroll
        for (int q = 0; q < N; ++q) {
          const bool have = sub + q * kRowLanes < n;
          e[q] = have ? ids[sub + q * kRowLanes] : 0;
          x[q] = logit[e[q]];
          own[q] = have ? entry_of(value(x[q], e[q]), e[q]) : -INFINITY;
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
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      };
      if constexpr (KL == 16) {
        if (most <= 3 * kRowLanes) place(std::integral_constant<int, 3>());
        else place(std::integral_constant<int, 4>());
      } else {
        if (most <= kRowLanes) place(std::integral_constant<int, 1>());
        else place(std::integral_constant<int, 2>());
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
      float last = INFINITY;
      int last_e = -1;
      for (int j = 0; j < k; ++j) {
        float best = kNone;
        int at = 0x7fffffff;
        for (int i = 0; i < M; ++i) {
          const int e = element<T, CH>(i, sub);
          if (e >= E) continue;
          const float v = logit[e] > kNone ? value(logit[e], e) : kNone;
          const bool after = v < last || (v == last && e > last_e);
          if (after && v > best) best = v, at = e;
        }
#pragma unroll
        for (int o = 1; o < kRowLanes; o <<= 1) {
          const float v = __shfl_xor(best, o, 64);
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

struct ReduceArgs {
  const float* mass;
  const uint32_t* count;
  const double* squares;
  const uint32_t* routed;
  double* part;        // [F][L][blocks of experts]
  uint32_t* arrived;   // [F][L], cleared by route_main (or, without runs, not needed)
  int32_t runs, L, E, k;
  uint32_t* D;
  uint32_t* tokens;
  float* balance;
  float* z;
  int32_t run_off[TACG_MAX_FAMILIES + 1];
};

// grid: (families, layers, blocks of EXPERTS experts).  The threads of a workgroup share the runs of a segment.  The last
// workgroup of a segment to arrive adds up the blocks' parts, in order.
template <int EXPERTS>
__global__ __launch_bounds__(kRouteThreads) void route_reduce(ReduceArgs a) {
  constexpr int kReduceExperts = EXPERTS, kReduceSlices = kRouteThreads / EXPERTS;
  __shared__ double mass[kReduceSlices][kReduceExperts];
  __shared__ uint32_t count[kReduceSlices][kReduceExperts];
  __shared__ double waves[kRouteWaves];
  __shared__ bool last;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int f = blockIdx.x, l = blockIdx.y, slice = tid / kReduceExperts, own = tid % kReduceExperts;
  const int e = blockIdx.z * kReduceExperts + own;
  const int64_t segment = static_cast<int64_t>(f) * a.L + l, from = static_cast<int64_t>(l) * a.runs;
  const int begin = a.run_off[f], end = a.run_off[f + 1];
  double m = 0.0;
  uint32_t c = 0;
  if (e < a.E) {
#pragma unroll 4
    for (int r = begin + slice; r < end; r += kReduceSlices) {
      m += a.mass[(from + r) * a.E + e];
      c += a.count[(from + r) * a.E + e];
    }
  }
  mass[slice][own] = m;
  count[slice][own] = c;
  __syncthreads();
  double v = 0.0;
  if (slice == 0 && e < a.E) {
    m = 0.0;
    c = 0;
#pragma unroll
    for (int s = 0; s < kReduceSlices; ++s) m += mass[s][own], c += count[s][own];
    a.D[segment * a.E + e] = c;
    v = m * c;
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  if (lane == 0) waves[wave] = v;
  __syncthreads();
  if (wave == 0) {
    if (lane == 0) {
      v = 0.0;
#pragma unroll
      for (int w = 0; w < kRouteWaves; ++w) v += waves[w];
      bool done = true;
      if (gridDim.z > 1) {
        a.part[segment * gridDim.z + blockIdx.z] = v;
        __threadfence();
        done = begin == end || atomicAdd(&a.arrived[segment], 1u) == gridDim.z - 1;
        __threadfence();
      } else {
        waves[0] = v;
      }
      last = done;
    }
  }
  __syncthreads();
  if (!last || wave != 0) return;
  double s = 0.0, b = 0.0;
  uint32_t n = 0;
#pragma unroll 2
  for (int r = begin + lane; r < end; r += 64) s += a.squares[from + r], n += a.routed[from + r];
  if (begin < end && gridDim.z > 1 && lane < static_cast<int>(gridDim.z))
    b = __hip_atomic_load(&a.part[segment * gridDim.z + lane], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (gridDim.z == 1 && lane == 0) b = waves[0];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    s += __shfl_xor(s, o, 64);
    b += __shfl_xor(b, o, 64);
    n += __shfl_xor(n, o, 64);
  }
  if (lane == 0) {
    const double rows = n;
    a.tokens[segment] = n;
    a.balance[segment] = n ? static_cast<float>(b * a.E / (a.k * rows * rows)) : 0.0f;
    if (a.z != nullptr) a.z[segment] = n ? static_cast<float>(s / rows) : 0.0f;
  }
}

template <class T, int CH, int KS>
__global__ __launch_bounds__(kRouteThreads) void route_back(BackArgs a) {
  constexpr int V = kChunk<T>, M = CH * V, kStride = M * kRowLanes + 32;
  __shared__ float sparse[kRowsPerPass][kStride];  // u s of a row's selected experts, else 0
  const int tid = threadIdx.x, lane = tid & 63, sub = lane & (kRowLanes - 1);
  const int l = blockIdx.y;
  const Run run = run_of(a, blockIdx.x);
  const int E = a.E, k = a.k;
  const int64_t segment = static_cast<int64_t>(run.family) * a.n_layers + l;
  const T* layer = static_cast<const T*>(a.logits) + l * a.stride_layer;
  float* mine = sparse[tid >> 3];
  for (int i = sub; i < kStride; i += kRowLanes) mine[i] = 0.0f;
  float c[M], zc = 0.0f;
  {
    const float n = a.tokens != nullptr ? static_cast<float>(a.tokens[segment]) : 0.0f;
    const float b = a.grad_balance != nullptr && n > 0.0f ? a.grad_balance[segment] * E / (k * n * n) : 0.0f;
    if (a.grad_z != nullptr && n > 0.0f) zc = a.grad_z[segment] * 2.0f / n;
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const int e = ((i / V) * kRowLanes + sub) * V + i % V;
      c[i] = b != 0.0f && e < E ? b * static_cast<float>(a.D[segment * E + e]) : 0.0f;
    }
  }
  for (int64_t base = run.first; base < run.last; base += kRowsPerPass) {
    const int64_t t = base + (tid >> 3);
    const bool in = t < run.last;
    const int64_t at = static_cast<int64_t>(l) * a.n_tokens + (in ? t : run.first);
    const T* row = layer + (in ? t : run.first) * a.stride_token;
    float p[M];
    load_row<T, CH>(row, sub, E, a.vec, p);
    const float norm = a.norm[at];
    const bool live = a.softmax ? norm > kNone : norm > 0.0f;
    int id[KS];
    float u[KS], s[KS];
#pragma unroll
    for (int q = 0; q < KS; ++q) {
      const int j = sub + q * kRowLanes;
      id[q] = -1;
      u[q] = s[q] = 0.0f;
      if (a.grad_gate != nullptr && j < k) {
        id[q] = a.trace[at * k + j];
        if (static_cast<uint32_t>(id[q]) >= static_cast<uint32_t>(E)) id[q] = -1;
        if (id[q] >= 0) {
          u[q] = a.grad_gate[at * k + j];
          s[q] = widen(row[id[q]]);
        }
      }
    }
    // softmax from differences to the row's largest: a normaliser of magnitude 1e4 would leave errors of 1e-3 in its exp
    float top = kNone, inverse = 0.0f;
    if (a.softmax) {
#pragma unroll
      for (int i = 0; i < M; ++i) top = fmaxf(top, p[i]);
      top = row_max(top);
      float total = 0.0f;
#pragma unroll
      for (int i = 0; i < M; ++i) {
        p[i] = live ? __expf(p[i] - top) : 0.0f;
        total += p[i];
      }
      total = row_sum(total);
      inverse = live ? 1.0f / total : 0.0f;
    }
    // scores s of the selected, and the gradient u of the scores through the gates, times s.  Sums of scores are divided by first: shares are
    // numbers up to 1, while a reciprocal or a score alone, multiplied, may leave the range of 32 bits
    if (a.softmax) {
      float high = top;
      if (a.renorm) {
        high = kNone;
#pragma unroll
        for (int q = 0; q < KS; ++q) high = fmaxf(high, id[q] >= 0 ? s[q] : kNone);
        high = row_max(high);
      }
#pragma unroll
      for (int q = 0; q < KS; ++q) s[q] = id[q] >= 0 ? __expf(s[q] - high) * (a.renorm ? 1.0f : inverse) : 0.0f;
    } else {
#pragma unroll
      for (int q = 0; q < KS; ++q) s[q] = id[q] >= 0 ? sigmoid(s[q]) : 0.0f;
    }
    float su = 0.0f;  // softmax without renormalisation: sum of u s
    if (a.renorm) {
      float part = 0.0f, mean = 0.0f;
#pragma unroll
      for (int q = 0; q < KS; ++q) part += s[q];
      part = row_sum(part);
      const float inv = part > 0.0f ? 1.0f / part : 0.0f;
#pragma unroll
      for (int q = 0; q < KS; ++q) s[q] *= inv, mean += s[q] * u[q];
      mean = row_sum(mean);
#pragma unroll
      for (int q = 0; q < KS; ++q) u[q] = a.scale * (u[q] - mean) * s[q];
    } else {
#pragma unroll
      for (int q = 0; q < KS; ++q) u[q] = a.scale * u[q] * s[q], su += u[q];
      if (a.softmax) su = row_sum(su);
    }
#pragma unroll
    for (int q = 0; q < KS; ++q)
      if (id[q] >= 0) mine[id[q]] = u[q];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // all experts of the row
    float dot = 0.0f;
    if (a.softmax) {
#pragma unroll
      for (int i = 0; i < M; ++i) {
        p[i] *= inverse;
        dot += p[i] * c[i];
      }
      dot = row_sum(dot);
      const float sub_all = (live ? zc * norm : 0.0f) - dot - (a.renorm ? 0.0f : su);
#pragma unroll
      for (int i = 0; i < M; ++i) p[i] = p[i] * (c[i] + sub_all) + mine[element<T, CH>(i, sub)];
    } else {
      const float inv = live ? 1.0f / norm : 0.0f;
#pragma unroll
      for (int i = 0; i < M; ++i) {
        p[i] = live ? sigmoid(p[i]) : 0.0f;  // a row that is not routed may hold a NaN
        dot += p[i] * inv * c[i];
      }
      dot = row_sum(dot);
#pragma unroll
      for (int i = 0; i < M; ++i) p[i] = (1.0f - p[i]) * (p[i] * inv * (c[i] - dot) + mine[element<T, CH>(i, sub)]);
    }
    if (in) store_row<T, CH>(static_cast<T*>(a.grad) + at * E, sub, E, a.vec, p);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int q = 0; q < KS; ++q)
      if (id[q] >= 0) mine[id[q]] = 0.0f;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// Bytes that a load of a row's piece may take: rows start at a multiple of them and hold a whole number of pieces.
int piece_bytes(const void* base, int64_t stride_layer, int64_t stride_token, int32_t E, int size) {
  for (int b = 16; b >= 8; b /= 2) {
    const int64_t n = b / size;
    if (reinterpret_cast<uintptr_t>(base) % b == 0 && stride_layer % n == 0 && stride_token % n == 0 && E % n == 0)
      return b;
  }
  return size;
}

int dtype_size(int32_t dtype) { return dtype == TACG_F32 ? 4 : 2; }

// Rows of a workgroup's run, whole passes: eight workgroups a CU (58 layers of 8155 rows of 256 with sums: 129 us, with two a CU 145),
// of at least two passes where the sums of a run go to a slot (24 layers of 2046 rows of 60: 14.7 us, with one 15.6).
int run_rows(int64_t total_rows, bool sums) {
  int64_t r = total_rows / (256 * 8);
  r = (r + kRowsPerPass - 1) / kRowsPerPass * kRowsPerPass;
  return static_cast<int>(std::min<int64_t>(std::max<int64_t>(r, sums ? 2 * kRowsPerPass : kRowsPerPass), 512));
}

// Workgroups per segment of the reduction: several where the segments have many runs, which one workgroup would take too long for (one
// layer of 8192 rows of 256: 50 us with one, 17 with eight); else one, as the fences between them cost more than they give (58
// layers of 16 families of 2 runs: 362 us against 129; 24 of 6 families of 6 runs: 25 against 15).
int reduce_blocks(int64_t n_tokens, int32_t n_layers, int32_t n_experts, int32_t n_fam) {
  return n_tokens / run_rows(n_tokens * n_layers, true) >= 16 * n_fam ? (n_experts + 31) / 32 : 1;
}

template <class Args>
int fill_runs(Args& a, const int64_t* fam_off_host, int32_t n_fam, int rows) {
  int64_t runs = 0;
  a.rows = rows;
  for (int f = 0; f < n_fam; ++f) {
    a.fam_off[f] = fam_off_host[f];
    a.run_off[f] = static_cast<int32_t>(runs);
    runs += (fam_off_host[f + 1] - fam_off_host[f] + rows - 1) / rows;
  }
  a.fam_off[n_fam] = fam_off_host[n_fam];
  a.run_off[n_fam] = static_cast<int32_t>(runs);
  return static_cast<int>(runs);
}

template <class T, int CH, int KL>
void start_main(const RouteArgs& a, bool bal, dim3 grid, hipStream_t s) {
  auto* kernel = a.bias != nullptr ? (bal ? route_main<T, CH, KL, true, true> : route_main<T, CH, KL, false, true>)
                                   : (bal ? route_main<T, CH, KL, true, false> : route_main<T, CH, KL, false, false>);
  kernel<<<grid, kRouteThreads, 0, s>>>(a);
}

template <class T, int CH>
void start_main(const RouteArgs& a, bool bal, dim3 grid, hipStream_t s) {
  if (a.k <= 4) start_main<T, CH, 4>(a, bal, grid, s);
  else if (a.k <= 8) start_main<T, CH, 8>(a, bal, grid, s);
  else start_main<T, CH, 16>(a, bal, grid, s);
}

template <class T>
void start_main(const RouteArgs& a, bool bal, dim3 grid, hipStream_t s) {
  const int chunks = (a.E + kChunk<T> * kRowLanes - 1) / (kChunk<T> * kRowLanes);
  if constexpr (sizeof(T) == 2) {
    if (chunks <= 1) return start_main<T, 1>(a, bal, grid, s);
  }
  if (chunks <= 2) return start_main<T, 2>(a, bal, grid, s);
  if (chunks <= 4) return start_main<T, 4>(a, bal, grid, s);
  if constexpr (sizeof(T) == 4) start_main<T, 8>(a, bal, grid, s);
}

template <class T, int CH>
void start_back(const BackArgs& a, dim3 grid, hipStream_t s) {
  auto* kernel = a.k > kRowLanes ? route_back<T, CH, 2> : route_back<T, CH, 1>;
  kernel<<<grid, kRouteThreads, 0, s>>>(a);
}

template <class T>
void start_back(const BackArgs& a, dim3 grid, hipStream_t s) {
  const int chunks = (a.E + kChunk<T> * kRowLanes - 1) / (kChunk<T> * kRowLanes);
  if (chunks <= 1) start_back<T, 1>(a, grid, s);
  else if (chunks <= 2) start_back<T, 2>(a, grid, s);
  else if (chunks <= 4) start_back<T, 4>(a, grid, s);
  else if constexpr (sizeof(T) == 4) start_back<T, 8>(a, grid, s);
}

}  // namespace

size_t route_workspace(int64_t n_tokens, int32_t n_layers, int32_t n_experts, int32_t n_fam) {
  const int rows = run_rows(n_tokens * n_layers, true);
  const size_t slots = static_cast<size_t>(n_layers) * static_cast<size_t>(n_tokens / rows + n_fam);
  const size_t segments = static_cast<size_t>(n_layers) * n_fam;
  return 2 * align256(slots * n_experts * 4) + align256(slots * 8) + align256(slots * 4) +
         align256(segments * reduce_blocks(n_tokens, n_layers, n_experts, n_fam) * 8) + align256(segments * 4);
}

int launch_route(const void* logits, int32_t dtype, int64_t stride_layer, int64_t stride_token, int64_t n_tokens,
                 int32_t n_layers, int32_t top_k, int32_t n_experts, const int64_t* fam_off_host, int32_t n_fam,
                 int32_t score, const float* bias, bool renorm, float scale, int16_t* trace, float* gate, float* norm,
                 uint32_t* D, uint32_t* tokens, float* balance, float* z, uint32_t* d_err, void* workspace,
                 hipStream_t stream) {
  const bool bal = D != nullptr;
  RouteArgs a{};
  a.logits = logits;
  a.stride_layer = stride_layer;
  a.stride_token = stride_token;
  a.n_tokens = n_tokens;
  a.n_layers = n_layers;
  a.E = n_experts;
  a.k = top_k;
  a.F = n_fam;
  a.softmax = score == TACG_SOFTMAX;
  a.renorm = renorm;
  a.scale = scale;
  a.bias = bias;
  a.trace = trace;
  a.gate = gate;
  a.norm = norm;
  a.err = d_err;
  a.vec = piece_bytes(logits, stride_layer, stride_token, n_experts, dtype_size(dtype));
  const int runs = fill_runs(a, fam_off_host, n_fam, run_rows(n_tokens * n_layers, bal));
  double* part = nullptr;
  if (bal) {
    Carver w{static_cast<char*>(workspace), 0};
    const size_t slots = static_cast<size_t>(n_layers) * runs;
    a.mass = w.take<float>(slots * n_experts);
    a.count = w.take<uint32_t>(slots * n_experts);
    a.squares = w.take<double>(slots);
    a.routed = w.take<uint32_t>(slots);
    part = w.take<double>(static_cast<size_t>(n_layers) * n_fam * reduce_blocks(n_tokens, n_layers, n_experts, n_fam));
    a.arrived = w.take<uint32_t>(static_cast<size_t>(n_layers) * n_fam);
  }
  if (runs > 0) {
    const dim3 grid(runs, n_layers);
    if (dtype == TACG_F32) start_main<float>(a, bal, grid, stream);
    else if (dtype == TACG_BF16) start_main<Bf16>(a, bal, grid, stream);
    else start_main<F16>(a, bal, grid, stream);
    if (hipGetLastError() != hipSuccess) return TACG_E_DEVICE;
  }
  if (bal) {
    ReduceArgs r{};
    r.mass = a.mass;
    r.count = a.count;
    r.squares = a.squares;
    r.routed = a.routed;
    r.part = part;
    r.arrived = a.arrived;
    r.runs = runs;
    r.L = n_layers;
    r.E = n_experts;
    r.k = top_k;
    r.D = D;
    r.tokens = tokens;
    r.balance = balance;
    r.z = z;
    for (int f = 0; f <= n_fam; ++f) r.run_off[f] = a.run_off[f];
    const int blocks = reduce_blocks(n_tokens, n_layers, n_experts, n_fam);
    const dim3 grid(n_fam, n_layers, blocks);
    if (blocks > 1 || n_experts <= 32) route_reduce<32><<<grid, kRouteThreads, 0, stream>>>(r);
    else route_reduce<TACG_MAX_EXPERTS><<<grid, kRouteThreads, 0, stream>>>(r);
    if (hipGetLastError() != hipSuccess) return TACG_E_DEVICE;
  }
  return TACG_OK;
}

int launch_route_backward(const void* logits, int32_t dtype, int64_t stride_layer, int64_t stride_token,
                          int64_t n_tokens, int32_t n_layers, int32_t top_k, int32_t n_experts,
                          const int64_t* fam_off_host, int32_t n_fam, int32_t score, bool renorm, float scale,
                          const int16_t* trace, const float* norm, const uint32_t* D, const uint32_t* tokens,
                          const float* grad_gate, const float* grad_balance, const float* grad_z, void* grad_logits,
                          hipStream_t stream) {
  BackArgs a{};
  a.logits = logits;
  a.stride_layer = stride_layer;
  a.stride_token = stride_token;
  a.n_tokens = n_tokens;
  a.n_layers = n_layers;
  a.E = n_experts;
  a.k = top_k;
  a.F = n_fam;
  a.softmax = score == TACG_SOFTMAX;
  a.renorm = renorm;
  a.scale = scale;
  a.trace = trace;
  a.norm = norm;
  a.D = D;
  a.tokens = tokens;
  a.grad_gate = grad_gate;
  a.grad_balance = grad_balance;
  a.grad_z = grad_z;
  a.grad = grad_logits;
  const int size = dtype_size(dtype);
  a.vec = std::min(piece_bytes(logits, stride_layer, stride_token, n_experts, size),
                   piece_bytes(grad_logits, 0, 0, n_experts, size));
  const int runs = fill_runs(a, fam_off_host, n_fam, run_rows(n_tokens * n_layers, false));
  if (runs == 0) return TACG_OK;
  const dim3 grid(runs, n_layers);
  if (dtype == TACG_F32) start_back<float>(a, grid, stream);
  else if (dtype == TACG_BF16) start_back<Bf16>(a, grid, stream);
  else start_back<F16>(a, grid, stream);
  return hipGetLastError() == hipSuccess ? TACG_OK : TACG_E_DEVICE;
}

}  // namespace tacg
