// The router whose selection is limited to the best groups of experts (route.hip: the router, its sums and its gradient).
//
// A row's lanes, its list and the sums of a run are those of route_main.  Before the list, the two largest values of every pair of
// neighbouring 16-byte chunks go to LDS, a lane adds up a group's from there, and ranks it among the others.  Without a bias the values
// are the logits, and only the best two of a group become scores.  All of it in 32 bits.
// Rows whose order 32 bits may hold wrongly are left out, and taken again at the end, a wave a row, in 64 bits: where two groups' sums lie
// nearer than near_by(), or, with a bias, two neighbours of those that are chosen, or the last of them and any that is not, unless their
// logits and biases are equal; and rows with more large values than the list holds.  Kept apart from the loop, so that neither its registers nor its
// time suffer (in the loop: 58 layers of 8155 rows of 256 in 32 bits, biased sigmoid scores, top-8 in four of eight groups, 261 us against
// 232 at that time).
// Those rows now: 190 us, 2.7 TB/s, where all in 64 bits took 717; with sums and 4077 rows 137 us.  Bound by instruction issue (1237
// vector instructions per eight rows, a fifth of them for the sigmoids, half of whose time is exp and reciprocal) and by waits for LDS: three
// waves a SIMD, by registers (168) and LDS (50 KB).  With sums of biased scores fourteen registers spill, which costs less than the third
// wave gives (137 against 185).
#include "route_kernels.h"

namespace tacg {
namespace {

// How near two values v = s + bias, or sums of two, may be for 32 bits to hold them in another order.  `bias` bounds their biases' magnitude, so
// s <= |v| + bias.  A score is exp of a difference or logit d <= 0, or nearly: its argument is off by |d| 2^-24 twice, the exp by 2^-23.  While
// s > 2^-11 (|d| < 8) that is 2^-20.2; a sigmoid adds 2^-22 for sum and reciprocal (and less of the exp, the nearer it is to 1), a softmax
// 2^-18.9 for the additions of the sum of all.  Down to the smallest s it is 2^-16 of s.  v is rounded once more.  Twice that, for two values:
__device__ __forceinline__ float near_by(float v, float bias, bool softmax) {
  const float s = fabsf(v) + bias;
  return (softmax ? 0x1p-17f : 0x1.4p-19f) * s + 0x1p-15f * fminf(s, 0x1p-11f) + FLT_MIN;
}

// What all lanes of a wave make of their values, of N words each: merge(a, b) brings b into a.  Exchanges within 2, 4, 8 and 16 lanes, then
// between rows and halves, where both sides' values come at once.
template <int N, class Merge>
__device__ __forceinline__ void wave_merge(int (&v)[N], Merge merge) {
  int o[N];
  auto dpp = [&](auto control) {
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = across<decltype(control)::value>(v[i]);
    merge(v, o);
  };
  dpp(std::integral_constant<int, kSwap1>());
  dpp(std::integral_constant<int, kSwap2>());
  dpp(std::integral_constant<int, kMirror>());
  dpp(std::integral_constant<int, 0x140>());  // mirrored within 16
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const auto r = __builtin_amdgcn_permlane16_swap(static_cast<uint32_t>(v[i]), static_cast<uint32_t>(v[i]), false, false);
    v[i] = static_cast<int>(r[0]);
    o[i] = static_cast<int>(r[1]);
  }
  merge(v, o);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const auto r = __builtin_amdgcn_permlane32_swap(static_cast<uint32_t>(v[i]), static_cast<uint32_t>(v[i]), false, false);
    v[i] = static_cast<int>(r[0]);
    o[i] = static_cast<int>(r[1]);
  }
  merge(v, o);
}
__device__ __forceinline__ float wave_sum(float x) {
  int v[1] = {__float_as_int(x)};
  wave_merge(v, [](int (&a)[1], const int (&b)[1]) { a[0] = __float_as_int(__int_as_float(a[0]) + __int_as_float(b[0])); });
  return __int_as_float(v[0]);
}
__device__ __forceinline__ float wave_max(float x) {
  int v[1] = {__float_as_int(x)};
  wave_merge(v, [](int (&a)[1], const int (&b)[1]) { a[0] = __float_as_int(fmaxf(__int_as_float(a[0]), __int_as_float(b[0]))); });
  return __int_as_float(v[0]);
}
__device__ __forceinline__ double double_of(int low, int high) { return __hiloint2double(high, low); }
__device__ __forceinline__ double wave_sum(double x) {
  int v[2] = {__double2loint(x), __double2hiint(x)};
  wave_merge(v, [](int (&a)[2], const int (&b)[2]) {
    const double s = double_of(a[0], a[1]) + double_of(b[0], b[1]);
    a[0] = __double2loint(s), a[1] = __double2hiint(s);
  });
  return double_of(v[0], v[1]);
}

// One row by a wave, in 64 bits: lane i has the experts i, i + 64, ...  Not unrolled: few rows come here.
template <class T, bool BIAS>
__device__ void exact_row(const RouteArgs& a, const T* row, const float* bias, int64_t at, uint32_t* count) {
  constexpr int M = TACG_MAX_EXPERTS / 64;
  const int lane = threadIdx.x & 63, E = a.E, k = a.k;
  float x[M], top = kNone, total = 0.0f;
#pragma unroll
  for (int i = 0; i < M; ++i) {
    x[i] = lane + 64 * i < E ? widen(row[lane + 64 * i]) : kNone;
    top = vmax(top, x[i]);
  }
  top = wave_max(top);
  const float from = top > kNone ? top : 0.0f;
  double v[M], sum = 0.0;
#pragma unroll
  for (int i = 0; i < M; ++i) {
    const double d = static_cast<double>(x[i]);
    v[i] = a.softmax ? exp(d - static_cast<double>(from)) : 1.0 / (1.0 + exp(-d));
    sum += v[i];
    total += __expf(x[i] - from);
  }
  total = wave_sum(total);
  if (BIAS && a.softmax) {
    sum = wave_sum(sum);
#pragma unroll
    for (int i = 0; i < M; ++i) v[i] *= sum > 0.0 ? 1.0 / sum : 0.0;
  }
#pragma unroll
  for (int i = 0; i < M; ++i) {
    if constexpr (BIAS) v[i] += static_cast<double>(bias[lane + 64 * i]);
    else if (a.group_best == 1) v[i] = static_cast<double>(x[i]);
    if (!(x[i] > kNone)) v[i] = -INFINITY;
  }
  double score = -INFINITY;  // of group `lane`
#pragma unroll 1
  for (int g = 0; g < a.groups; ++g) {
    double first = -INFINITY, second = -INFINITY;
#pragma unroll
    for (int i = 0; i < M; ++i) {
      const double u = static_cast<int>(((lane + 64 * i) * a.group_mul) >> 16) == g ? v[i] : -INFINITY;
      second = fmax(second, fmin(first, u));
      first = fmax(first, u);
    }
    int two[4] = {__double2loint(first), __double2hiint(first), __double2loint(second), __double2hiint(second)};
    wave_merge(two, [](int (&p)[4], const int (&q)[4]) {
      const double f = double_of(p[0], p[1]), s = double_of(p[2], p[3]), of = double_of(q[0], q[1]), os = double_of(q[2], q[3]);
      const double high = fmax(f, of), low = fmax(fmin(f, of), fmax(s, os));
      p[0] = __double2loint(high), p[1] = __double2hiint(high), p[2] = __double2loint(low), p[3] = __double2hiint(low);
    });
    first = double_of(two[0], two[1]);
    second = double_of(two[2], two[3]);
    if (lane == g) score = a.group_best > 1 && second > -INFINITY ? first + second : first;
  }
  int better = 0;
#pragma unroll 1
  for (int h = 0; h < a.groups; ++h) {
    const double s = __shfl(score, h, 64);
    better += s > score || (s == score && h < lane);
  }
  const uint64_t kept = __ballot(lane < a.groups && score > -INFINITY && better < a.top_groups);
#pragma unroll
  for (int i = 0; i < M; ++i) {
    if constexpr (!BIAS) v[i] = static_cast<double>(x[i]);
    const uint32_t g = ((lane + 64 * i) * a.group_mul) >> 16;
    if (!(x[i] > kNone) || !((kept >> (g & 63)) & 1)) v[i] = -INFINITY;
  }
  int id = -1;  // of slot `lane`
  float w = kNone;
#pragma unroll 1
  for (int j = 0; j < k; ++j) {
    double best = -INFINITY;
    int e = 0x7fffffff;
    float logit = kNone;
#pragma unroll
    for (int i = 0; i < M; ++i)
      if (v[i] > best) best = v[i], e = lane + 64 * i, logit = x[i];
    int winner[4] = {__double2loint(best), __double2hiint(best), e, __float_as_int(logit)};
    wave_merge(winner, [](int (&p)[4], const int (&q)[4]) {
      const double u = double_of(p[0], p[1]), o = double_of(q[0], q[1]);
      const bool other = o > u || (o == u && q[2] < p[2]);
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = other ? q[i] : p[i];
    });
    best = double_of(winner[0], winner[1]);
    e = winner[2];
    logit = __int_as_float(winner[3]);
    if (!(best > -INFINITY)) break;
#pragma unroll
    for (int i = 0; i < M; ++i)
      if (e == lane + 64 * i) v[i] = -INFINITY;
    if (lane == j) id = e, w = logit;
  }
  if (a.softmax) {
    const float high = BIAS && a.renorm ? wave_max(w) : from;
    w = __expf(w - (high == kNone ? 0.0f : high));
  } else {
    w = sigmoid(w);
  }
  float factor = 1.0f;
  if (a.renorm) {
    const float part = wave_sum(lane < k ? w : 0.0f);
    factor = part > 0.0f ? 1.0f / part : 0.0f;
  } else if (a.softmax) {
    factor = total > 0.0f ? 1.0f / total : 0.0f;
  }
  if (lane < k) {
    a.trace[at * k + lane] = static_cast<int16_t>(id);
    a.gate[at * k + lane] = w * factor * a.scale;
    if (count != nullptr && id >= 0) atomicAdd(&count[id], 1u);
  }
}

// grid: (runs, layers).  KL: the smallest of 4, 8 and 16 that is not below k.
template <class T, int CH, int KL, bool BAL, bool BIAS>
__global__ __launch_bounds__(kRouteThreads, 3) void route_grouped(RouteArgs a) {
  constexpr int V = kChunk<T>, M = CH * V, KS = (KL + kRowLanes - 1) / kRowLanes;
  constexpr int kList = KL < 8 ? 16 : 2 * KL;  // elements of a row's list
  constexpr int kPairs = CH * kRowLanes / 2, kPairStride = (kPairs + 15) / 16 * 16 + 8;
  constexpr int kRunRows = 512;
  // of a row, one after another: the two largest values of each pair of its chunks (two rows' in all banks); then the list
  union Row {
    struct {
      float2 two[kPairStride];
      float border[2];
    };
    struct {
      double list[kList];
      float2 chosen[KS * kRowLanes];
      float ranked[KL + 1];
    } after;
  };
  __shared__ Row rows[kRowsPerPass];
  __shared__ alignas(16) float copy[kRowsPerPass][M * kRowLanes + 4];  // the rows' logits: rows in different banks
  __shared__ alignas(16) float group_score[kRowsPerPass][TACG_MAX_GROUPS + 4];
  __shared__ alignas(16) float bias_of[BIAS ? TACG_MAX_EXPERTS : 4];   // the layer's
  __shared__ uint16_t hard_rows[kRunRows];                             // left for the end
  __shared__ int n_hard;
  __shared__ uint32_t count[BAL ? TACG_MAX_EXPERTS : 1];
  __shared__ float squares[kRouteWaves];
  __shared__ uint32_t routed[kRouteWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, sub = lane & (kRowLanes - 1);
  const int l = blockIdx.y;
  const Run run = run_of(a, blockIdx.x);
  const int E = a.E, k = a.k;
  const T* layer = static_cast<const T*>(a.logits) + l * a.stride_layer;
  double* mine = rows[tid >> 3].after.list;
  float2* slots = rows[tid >> 3].after.chosen;
  float* logit = copy[tid >> 3];
  float acc[BAL ? M : 1];
  float sq = 0.0f;
  uint32_t live = 0;
#pragma unroll
  for (int i = 0; i < (BAL ? M : 1); ++i) acc[i] = 0.0f;
  if (tid == 0) n_hard = 0;
  if (BAL) {
    for (int e = tid; e < E; e += kRouteThreads) count[e] = 0;
    if (tid == 0 && run.start) a.arrived[static_cast<int64_t>(run.family) * a.n_layers + l] = 0;
  }
  float most_bias = 0.0f;
  if constexpr (BIAS) {
    for (int e = tid; e < TACG_MAX_EXPERTS; e += kRouteThreads) bias_of[e] = e < E ? a.bias[l * E + e] : 0.0f;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TACG_MAX_EXPERTS; i += 64) most_bias = fmaxf(most_bias, fabsf(bias_of[lane + i]));
    most_bias = wave_max(most_bias);
  }
  __syncthreads();
  // whether the sum over all experts is needed
  const bool all = BAL || BIAS || a.norm != nullptr || (a.softmax && !a.renorm);
  const bool whole = a.vec == 16 && E == M * kRowLanes;  // no lane has less than all its chunks
  for (int64_t base = run.first; base < run.last; base += kRowsPerPass) {
    const int64_t t = base + (tid >> 3);
    const bool in = t < run.last;
    const T* row = layer + (in ? t : run.first) * a.stride_token;
    float x[M];
    if (whole) load_row<T, CH>(row, sub, M * kRowLanes, 16, x);
    else load_row<T, CH>(row, sub, E, a.vec, x);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < M; i += 2) bad |= __builtin_isunordered(x[i], x[i + 1]);
    float top = x[0];
#pragma unroll
    for (int i = 1; i < M; ++i) top = vmax(top, x[i]);
    top = row_max(top);
    bad |= top == INFINITY;
    if (__any(bad)) {  // a NaN or +inf: the row is not routed
      const uint64_t m = __ballot(bad) >> (lane & ~(kRowLanes - 1));
      if ((m & 0xff) != 0) {
        if (in && sub == 0) atomicOr(a.err, TACG_ERR_VALUE);
        top = kNone;
#pragma unroll
        for (int i = 0; i < M; ++i) x[i] = kNone;
      }
    }
#pragma unroll
    for (int i = 0; i < M; i += 4)
      *reinterpret_cast<float4*>(logit + element<T, CH>(i, sub)) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const bool some = top > kNone;
    const float shift = some ? top : 0.0f;
    float total = 0.0f, inverse = 0.0f;
    // without a bias the logits order; scores are of their own
    auto scores = [&](float (&s)[M]) {
      if (a.softmax) {
#pragma unroll
        for (int i = 0; i < M; ++i) s[i] = __expf(x[i] - shift), total += s[i];
      } else {
#pragma unroll
        for (int i = 0; i < M; ++i) s[i] = sigmoid(x[i]), total += s[i];
      }
      total = row_sum(total);
      inverse = total > 0.0f ? 1.0f / total : 0.0f;
      if (BAL && in) {
#pragma unroll
        for (int i = 0; i < (BAL ? M : 1); ++i) acc[i] += s[i] * inverse;
      }
    };
    if constexpr (BIAS) {
      float s[M];
      scores(s);
      const float f = a.softmax ? inverse : 1.0f;
#pragma unroll
      for (int i = 0; i < M; i += 4) {
        const float4 b = *reinterpret_cast<const float4*>(bias_of + element<T, CH>(i, sub));
        x[i] = x[i] > kNone ? s[i] * f + b.x : kNone;
        x[i + 1] = x[i + 1] > kNone ? s[i + 1] * f + b.y : kNone;
        x[i + 2] = x[i + 2] > kNone ? s[i + 2] * f + b.z : kNone;
        x[i + 3] = x[i + 3] > kNone ? s[i + 3] * f + b.w : kNone;
      }
    } else if (all) {
      float s[M];
      scores(s);
    }
    // what the selection orders by, of one expert
    auto value = [&](float v, int e) {
      if constexpr (BIAS) v = (a.softmax ? __expf(v - shift) * inverse : sigmoid(v)) + bias_of[e];
      return v;
    };
    // ---- the groups that are kept, a bit each
    uint32_t kept = 0;
    bool hard = false;
    {
      auto take = [](float& first, float& second, float f, float s) {
        second = vmax3(vmin(first, f), second, s);
        first = vmax(first, f);
      };
      float* score = group_score[tid >> 3];
      float2* pairs = rows[tid >> 3].two;
      for (int g = a.groups + sub; g < ((a.groups + 7) & ~7); g += kRowLanes) score[g] = kNone;
      auto keep = [&](int g, float first, float second) {
        if constexpr (BIAS) {
          score[g] = a.group_best > 1 && second > kNone ? first + second : first;
        } else {  // logits: their scores are added
          auto s = [&](float v) { return v == kNone ? 0.0f : a.softmax ? __expf(v - shift) : sigmoid(v); };
          score[g] = a.group_best == 1 || first == kNone ? first : s(first) + s(second);
        }
      };
      if (a.group_pairs > 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          float first = vmax(x[c * V], x[c * V + 1]), second = vmin(x[c * V], x[c * V + 1]);
#pragma unroll
          for (int i = 2; i < V; i += 2) take(first, second, vmax(x[c * V + i], x[c * V + i + 1]), vmin(x[c * V + i], x[c * V + i + 1]));
          take(first, second, across<kSwap1>(first), across<kSwap1>(second));
          pairs[(c * kRowLanes + sub) / 2] = make_float2(first, second);  // both lanes write the same
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const int n = a.group_pairs;
        for (int g = sub; g < a.groups; g += kRowLanes) {
          float first = kNone, second = kNone;
          for (int c = 0; c < n; c += 4) {
            float2 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int at = c + (n % 4 == 0 ? (i + sub) & 3 : i);  // lanes start in different banks
              v[i] = at < n ? pairs[g * n + at] : make_float2(kNone, kNone);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) take(first, second, v[i].x, v[i].y);
          }
          keep(g, first, second);
        }
      } else {
        const int lanes = a.group_lanes, part = sub & (lanes - 1);
        for (int g = lanes == 4 ? sub >> 2 : lanes == 2 ? sub >> 1 : sub; g < a.groups; g += kRowLanes) {
          float first = kNone, second = kNone;
          for (int e = g * a.group_size + part; e < (g + 1) * a.group_size; e += lanes)
            if (logit[e] > kNone) take(first, second, value(logit[e], e), kNone);
          if (lanes > 1) take(first, second, across<kSwap1>(first), across<kSwap1>(second));
          if (lanes > 2) take(first, second, across<kSwap2>(first), across<kSwap2>(second));
          keep(g, first, second);
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      float* border = rows[tid >> 3].border;  // the last that is kept, and the first that is not
      for (int g = sub; g < a.groups; g += kRowLanes) {
        const float own = score[g];
        int better = 0;
        for (int h = 0; h < a.groups; h += 8) {  // those past the last are -inf
          float s[8];
          *reinterpret_cast<float4*>(s) = *reinterpret_cast<const float4*>(score + h);
          *reinterpret_cast<float4*>(s + 4) = *reinterpret_cast<const float4*>(score + h + 4);
#pragma unroll
          for (int i = 0; i < 8; ++i) better += s[i] > own || (s[i] == own && h + i < g);
        }
        if (own > kNone && better < a.top_groups) kept |= 1u << g;
        const int at = better - a.top_groups + 1;
        if (at == 0 || at == 1) border[at] = own;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if ((BIAS || a.group_best > 1) && a.top_groups < a.groups)  // else logits, in their order
        hard = border[1] > kNone && border[0] - border[1] <= near_by(border[0], 2.0f * most_bias, a.softmax);
      kept |= across<kSwap1>(static_cast<int>(kept));
      kept |= across<kSwap2>(static_cast<int>(kept));
      kept |= across<kMirror>(static_cast<int>(kept));
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    auto allowed = [&](int e) { return (kept >> (((e * a.group_mul) >> 16) & 31)) & 1u; };
    if (a.group_pairs > 0) {
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const bool is = allowed((c * kRowLanes + sub) * V);
#pragma unroll
        for (int i = 0; i < V; ++i) x[c * V + i] = is ? x[c * V + i] : kNone;
      }
    } else {
      int from = sub;
      asm volatile("" : "+v"(from));  // or each element's group would stay in a register throughout
#pragma unroll
      for (int i = 0; i < M; ++i) x[i] = allowed(element<T, CH>(i, from)) ? x[i] : kNone;
    }
    // ---- the list: elements that reach a lower bound of the k-th largest, each lane's after those of the lanes before it
    float unused, bound = lower_bound<KL>(x, unused);
    if constexpr (BIAS) bound -= near_by(bound, most_bias, a.softmax);
    uint32_t mask = at_least(x, vmax(bound, -FLT_MAX));
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
    if (n > kList) hard = true, n = 0, mask = 0;
    int most = 0;  // of the wave's rows
#pragma unroll
    for (int r = 0; r < 64; r += kRowLanes) {
      const int v = __builtin_amdgcn_readlane(n, r);
      most = v > most ? v : most;
    }
    int32_t* ids = reinterpret_cast<int32_t*>(mine);  // before the entries
    float* order = rows[tid >> 3].after.ranked;
#pragma unroll
    for (int q = 0; q < KS; ++q) slots[sub + q * kRowLanes] = make_float2(__int_as_float(-1), kNone);
    if constexpr (BIAS)
      for (int j = sub; j <= k; j += kRowLanes) order[j] = kNone;
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
      float y[N], v[N];
      double own[N];
#pragma unroll
      for (int q = 0; q < N; ++q) {
        const bool have = sub + q * kRowLanes < n;
        e[q] = have ? ids[sub + q * kRowLanes] : 0;
        y[q] = logit[e[q]];
        v[q] = value(y[q], e[q]);
        own[q] = have ? entry_of(v[q], e[q]) : -INFINITY;
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
      for (int q = 0; q < N; ++q) {
        if (sub + q * kRowLanes >= n) continue;
        if (larger[q] < k) slots[larger[q]] = make_float2(__int_as_float(e[q]), y[q]);
        if (BIAS && larger[q] <= k) order[larger[q]] = v[q];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    if constexpr (KL == 16) {
      if (most <= 3 * kRowLanes) place(std::integral_constant<int, 3>());
      else place(std::integral_constant<int, 4>());
    } else {
      if (most <= kRowLanes) place(std::integral_constant<int, 1>());
      else place(std::integral_constant<int, 2>());
    }
    int id[KS];   // of slots sub, sub + 8: expert and its logit
    float w[KS];
    bool doubt = false;
    auto close = [&](int j) { return order[j + 1] > kNone && order[j] - order[j + 1] <= near_by(order[j], most_bias, a.softmax); };
#pragma unroll
    for (int q = 0; q < KS; ++q) {
      const int j = sub + q * kRowLanes;
      const float2 v = slots[j];
      id[q] = __float_as_int(v.x);
      w[q] = v.y;
      if (BIAS && j < k) doubt |= close(j);
    }
    if (BIAS && __any(doubt)) {  // equal logits with equal biases are equal, and in their order
      auto differ = [&](int e, int f) { return logit[e] != logit[f] || bias_of[e] != bias_of[f]; };
      for (int j = sub; j + 1 < k; j += kRowLanes)
        if (close(j)) hard |= differ(__float_as_int(slots[j].x), __float_as_int(slots[j + 1].x));
      if (close(k - 1)) {  // one that is as near to the last chosen may stand behind equal ones: all that are not chosen
        const int e = __float_as_int(slots[k - 1].x);
        const float last = order[k - 1], near = near_by(last, most_bias, a.softmax);
        for (int i = sub; i < n; i += kRowLanes) {
          const double u = mine[i];
          const float v = static_cast<float>(u);
          if (v <= last && last - v <= near) hard |= differ(e, expert_of(u));
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (__any(hard)) {
      hard = ((__ballot(hard) >> (lane & ~(kRowLanes - 1))) & 0xff) != 0;
      if (hard && in && sub == 0) hard_rows[atomicAdd(&n_hard, 1)] = static_cast<uint16_t>(t - run.first);
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
    if (in && !hard) {
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
  barrier_after_lds_atomics();
  // the run's sums: rows of a wave, then the waves in order
  constexpr int kMass = M * kRowLanes;
  float* sums = &copy[0][0];  // the logits are of no use any more
  if (BAL) {
#pragma unroll
    for (int i = 0; i < (BAL ? M : 1); ++i) {
      acc[i] = rows_sum(acc[i]);
      if (lane < kRowLanes) sums[wave * kMass + element<T, CH>(i, sub)] = acc[i];
    }
    sq = rows_sum(sq);
#pragma unroll
    for (int o = kRowLanes; o < 64; o <<= 1) live += __shfl_xor(live, o, 64);
    if (lane == 0) squares[wave] = sq, routed[wave] = live;
  }
  for (int i = wave; i < n_hard; i += kRouteWaves) {
    const int64_t t = run.first + hard_rows[i];
    exact_row<T, BIAS>(a, layer + t * a.stride_token, bias_of, static_cast<int64_t>(l) * a.n_tokens + t, BAL ? count : nullptr);
  }
  if (!BAL) return;
  barrier_after_lds_atomics();
  const int64_t slot = static_cast<int64_t>(l) * gridDim.x + blockIdx.x;
  for (int e = tid; e < E; e += kRouteThreads) {
    float m = sums[e];
#pragma unroll
    for (int w = 1; w < kRouteWaves; ++w) m += sums[w * kMass + e];
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

template <class T, int CH, int KL>
void start(const RouteArgs& a, bool bal, dim3 grid, hipStream_t s) {
  auto* kernel = a.bias != nullptr ? (bal ? route_grouped<T, CH, KL, true, true> : route_grouped<T, CH, KL, false, true>)
                                   : (bal ? route_grouped<T, CH, KL, true, false> : route_grouped<T, CH, KL, false, false>);
  kernel<<<grid, kRouteThreads, 0, s>>>(a);
}

template <class T, int CH>
void start(const RouteArgs& a, bool bal, dim3 grid, hipStream_t s) {
  if (a.k <= 4) start<T, CH, 4>(a, bal, grid, s);
  else if (a.k <= 8) start<T, CH, 8>(a, bal, grid, s);
  else start<T, CH, 16>(a, bal, grid, s);
}

template <class T>
void start(const RouteArgs& a, bool bal, dim3 grid, hipStream_t s) {
  const int chunks = (a.E + kChunk<T> * kRowLanes - 1) / (kChunk<T> * kRowLanes);
  if constexpr (sizeof(T) == 2) {
    if (chunks <= 1) return start<T, 1>(a, bal, grid, s);
  }
  if (chunks <= 2) return start<T, 2>(a, bal, grid, s);
  if (chunks <= 4) return start<T, 4>(a, bal, grid, s);
  if constexpr (sizeof(T) == 4) start<T, 8>(a, bal, grid, s);
}

}  // namespace

void start_route_groups(const RouteArgs& a, int32_t dtype, bool bal, dim3 grid, hipStream_t stream) {
  if (dtype == TACG_F32) start<float>(a, bal, grid, stream);
  else if (dtype == TACG_BF16) start<Bf16>(a, bal, grid, stream);
  else start<F16>(a, bal, grid, stream);
}

}  // namespace tacg
