// Products of the experts' weights in 4 bits with the tokens routed to them.
//
//   W[h][n][c] = scale[h][n][c / group] * (level[h][n][c] - zero[h][n][c / group]),   zero = 8 where none is given.
//
// q4_pack_kernel: levels, scales and zeros of a weight matrix, a lane per 32 columns (16 bytes of levels).
//
// The products run on the matrix cores, with tokens as rows and weight rows as columns of v_mfma_f32_16x16x32: lane n + 16 q supplies
// columns 8 q .. 8 q + 7 of weight row n and of token n, and holds the sums of weight row n with tokens 4 q .. 4 q + 3.  A step is 128
// columns of 16 weight rows: a lane loads 16 bytes, columns 32 q .. 32 q + 31 of its row, and two exchanges of half and quarter waves
// give it the words of the four products of the step, each of 32 columns.  (Without the exchange the tokens' loads would be spread over
// four times as many cache lines.)  A level becomes a 16-bit float by an OR into the mantissa: 128 + level (bfloat16) or
// 1024 + level (float16), both exact; the float16 one is then brought to level - zero by one exact packed subtraction, the bfloat16
// one after the product: sum (level - zero) x = sum (128 + level) x - (128 + zero) sum x, with sum x from a product with ones.
// The eight levels of a word come out in the order 0 4 1 5 2 6 3 7, so the tokens' values are put in that order too.  The scale of a
// group is applied in 32 bits to the group's sum.
//
// The waves of a workgroup take the steps of its 16 RT weight rows in turn and add their sums up in LDS, in order.
// q4_tiles: a workgroup finds the tokens of its expert by itself (no launch before it): with few (token, slot) pairs it is the one of
//   the first pair of that expert, with many there is a workgroup for each held expert.
// q4_sum_token: few pairs, summed over a token's experts: a workgroup takes all experts of one token, the steps of all of them in turn.
// q4_combine: sums the 32-bit products of many pairs over the slots of a token.
#include <algorithm>
#include <cmath>

#include "tacg_internal.h"

namespace tacg {
namespace {

constexpr int kPiece = 32;  // columns of 16 bytes of levels

struct Q4Args {
  const void* x;
  int64_t x_token, x_slot;  // strides in elements
  int64_t n_tokens;
  int32_t k, E, H, N, K, group, n_groups, pieces, mode;
  const int16_t* ids;
  const int32_t* slot;      // [E] or null
  const uint8_t* q;
  const void* scales;
  const uint8_t* zeros;     // or null
  const float* gate;        // [T][k] or null
  int32_t few;              // few pairs: a workgroup per pair and block of rows
  float* part;              // [T][k][N], or null
  void* out;
  uint32_t* err;
};

__device__ __forceinline__ float widen(__bf16 v) { return static_cast<float>(v); }
__device__ __forceinline__ float widen(_Float16 v) { return static_cast<float>(v); }
__device__ __forceinline__ float widen(float v) { return v; }

// Where the weights of an expert id are held: -1 for none (an unused slot, an expert of another GPU), below -1 for an invalid entry.
constexpr int kBadId = -2, kBadTable = -3;
__device__ __forceinline__ int place_of(const Q4Args& a, int e) {
  const int h = a.slot != nullptr ? a.slot[e] : e;
  return h < 0 ? -1 : h < a.H ? h : kBadTable;
}
__device__ __forceinline__ void report(const Q4Args& a, int h) {
  if (h == kBadId) atomicOr(a.err, TACG_ERR_ID_RANGE);
  if (h == kBadTable) atomicOr(a.err, TACG_ERR_TABLE);
}

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kStep = 128;       // columns of a step
constexpr int kScan = 8192;      // pairs that a workgroup looks through

typedef __attribute__((ext_vector_type(4))) float float4v;
typedef __attribute__((ext_vector_type(4))) uint32_t uint4v;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;

__device__ __forceinline__ float4v mfma(const uint4v& tokens, const uint4v& weights, float4v c, __bf16) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, tokens), __builtin_bit_cast(bf16x8, weights),
                                                 c, 0, 0, 0);
}
__device__ __forceinline__ float4v mfma(const uint4v& tokens, const uint4v& weights, float4v c, _Float16) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, tokens), __builtin_bit_cast(f16x8, weights),
                                                c, 0, 0, 0);
}

// 16-bit floats of the eight levels of a word, in the order 0 4 1 5 2 6 3 7: 128 + level.
__device__ __forceinline__ uint4v spread(uint32_t w, uint32_t, __bf16) {
  constexpr uint32_t kMask = 0x000f000fu, kBase = 0x43004300u;
  return uint4v{(w & kMask) | kBase, ((w >> 4) & kMask) | kBase, ((w >> 8) & kMask) | kBase, ((w >> 12) & kMask) | kBase};
}
// The same as level - zero; `minus` holds -(1024 + zero) twice.
__device__ __forceinline__ uint4v spread(uint32_t w, uint32_t minus, _Float16) {
  constexpr uint32_t kMask = 0x000f000fu, kBase = 0x64006400u;
  const f16x2 m = __builtin_bit_cast(f16x2, minus);
  uint4v o;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    o[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, ((w >> (4 * i)) & kMask) | kBase) + m);
  return o;
}

// One step's operands of a lane, as loaded.  PER: groups of a step.
template <class T, int RT, int TT, int PER>
struct Operands {
  uint4v w[RT];
  T scale[RT][PER];
  uint8_t zero[RT][PER];
  uint4v x[TT][4];
};

// row: first byte-piece index of each weight row; x: the lane's token rows, null where there is none.
template <class T, int RT, int TT, int PER>
__device__ __forceinline__ void load_step(const Q4Args& a, int s, int quarter, const int64_t (&row)[RT],
                                          const T* const (&x)[TT], Operands<T, RT, TT, PER>& o) {
  int piece = 4 * s + quarter;  // past the end the tokens' values are 0: any levels do
  piece = piece < a.pieces ? piece : a.pieces - 1;
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    o.w[i] = reinterpret_cast<const uint4v*>(a.q)[row[i] * a.pieces + piece];
#pragma unroll
    for (int g = 0; g < PER; ++g) {
      int at = PER == 1 ? s * kStep / a.group : s * PER + g;
      at = at < a.n_groups ? at : a.n_groups - 1;
      o.scale[i][g] = static_cast<const T*>(a.scales)[row[i] * a.n_groups + at];
      o.zero[i][g] = a.zeros != nullptr ? a.zeros[row[i] * a.n_groups + at] : 8;
    }
  }
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = s * kStep + 32 * i + 8 * quarter;
      o.x[t][i] = uint4v{0, 0, 0, 0};
      if (x[t] != nullptr) {
        if (c + 8 <= a.K) {
          __builtin_memcpy(&o.x[t][i], x[t] + c, 16);  // rows need not be aligned to more than an element
        } else if (c < a.K) {
          T v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = c + j < a.K ? x[t][c + j] : static_cast<T>(0.0f);
          __builtin_memcpy(&o.x[t][i], v, 16);
        }
      }
    }
}

// sum += factor * scale * (level - zero) . x of one step.
template <class T, int RT, int TT, int PER>
__device__ __forceinline__ void add_step(const Operands<T, RT, TT, PER>& o, float factor, float4v (&sum)[RT][TT]) {
  constexpr bool kLate = sizeof(T) == 2 && __is_same(T, __bf16);  // the zero is taken off the sums
  constexpr int kRun = 4 / PER;                                   // products of a group
  uint4v x[TT][4];
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4v v = o.x[t][i];
      x[t][i] = uint4v{__builtin_amdgcn_perm(v[2], v[0], 0x05040100u), __builtin_amdgcn_perm(v[2], v[0], 0x07060302u),
                       __builtin_amdgcn_perm(v[3], v[1], 0x05040100u), __builtin_amdgcn_perm(v[3], v[1], 0x07060302u)};
    }
  uint32_t w[RT][4];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const auto a = __builtin_amdgcn_permlane32_swap(o.w[r][0], o.w[r][2], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(o.w[r][1], o.w[r][3], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    const auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    w[r][0] = c[0];
    w[r][1] = c[1];
    w[r][2] = d[0];
    w[r][3] = d[1];
  }
#pragma unroll
  for (int g = 0; g < PER; ++g) {
    float4v all[TT], part[RT][TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      all[t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
      if (kLate) {
        constexpr uint32_t kOnes = 0x3f803f80u;
#pragma unroll
        for (int i = g * kRun; i < (g + 1) * kRun; ++i) all[t] = mfma(x[t][i], uint4v{kOnes, kOnes, kOnes, kOnes}, all[t], T());
      }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const uint32_t minus = 0xe400u + o.zero[r][g];  // -(1024 + zero) in float16
#pragma unroll
      for (int t = 0; t < TT; ++t) part[r][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = g * kRun; i < (g + 1) * kRun; ++i) {
        const uint4v v = spread(w[r][i], minus | minus << 16, T());
#pragma unroll
        for (int t = 0; t < TT; ++t) part[r][t] = mfma(x[t][i], v, part[r][t], T());
      }
      const float scale = static_cast<float>(o.scale[r][g]) * factor;
      const float zero = 128.0f + static_cast<float>(o.zero[r][g]);
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float v = kLate ? part[r][t][j] - zero * all[t][j] : part[r][t][j];
          sum[r][t][j] += scale * v;
        }
    }
  }
}

__device__ __forceinline__ float silu(float v) { return v / (1.0f + __expf(-v)); }

// Adds the waves' sums of 16 tokens up in order; out(token, column) takes the value of each.
template <int RT, int WIDTH, class Out>
__device__ __forceinline__ void join(float (&red)[kWaves][16][RT * 16 + 4], const float4v (&mine)[RT], bool glu, Out out) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int j = 0; j < 4; ++j) red[wave][4 * (lane >> 4) + j][16 * r + (lane & 15)] = mine[r][j];
  __syncthreads();
  for (int i = tid; i < 16 * WIDTH; i += kThreads) {
    const int t = i / WIDTH, n = i % WIDTH;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += red[w][t][n];
    if (glu) {
      float u = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) u += red[w][t][n + WIDTH];
      v = silu(v) * u;
    }
    out(t, n, v);
  }
}

__device__ __forceinline__ int look_up(const Q4Args& a, const int16_t* place, int id) {
  return static_cast<uint32_t>(id) < static_cast<uint32_t>(a.E) ? place[id] : id == -1 ? -1 : kBadId;
}
__device__ __forceinline__ int served_by(const Q4Args& a, const int16_t* place, int id) {
  const int h = look_up(a, place, id);
  return h < 0 ? -1 : h;
}

// Where the pairs from `from` on, `n` of them, that matrix `h` serves (h = -1: that no matrix serves) stand in the list, in order.
__device__ __forceinline__ int list_pairs(const Q4Args& a, int64_t from, int n, int h, const int16_t* place,
                                          uint16_t* list, int (&total)[kWaves]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int each = (n + kThreads - 1) / kThreads;
  const int first = tid * each, last = first + each < n ? first + each : n;
  int mine = 0;
  for (int i = first; i < last; ++i) mine += served_by(a, place, a.ids[from + i]) == h;
  int at = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(at, o, 64);
    if (lane >= o) at += v;
  }
  if (lane == 63) total[wave] = at;
  __syncthreads();
  at -= mine;
  int all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) at += total[w];
    all += total[w];
  }
  if (mine > 0)
    for (int i = first; i < last; ++i)
      if (served_by(a, place, a.ids[from + i]) == h) list[at++] = static_cast<uint16_t>(i);
  __syncthreads();
  return all;
}

// grid: (blocks of 16 RT weight rows; GLU: of half as many output columns, few pairs: pairs, many: held experts and one for the pairs
// that none serves, runs of kScan pairs).
template <class T, bool GLU, int RT, int TT, int PER>
__global__ __launch_bounds__(kThreads) void q4_tiles(Q4Args a) {
  constexpr int kWidth = GLU ? RT * 8 : RT * 16;  // output columns of a workgroup
  __shared__ float red[kWaves][16][RT * 16 + 4];
  __shared__ uint16_t list[kScan];
  __shared__ int16_t place[TACG_MAX_EXPERTS];
  __shared__ int total[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, quarter = lane >> 4;
  const int64_t pairs = a.n_tokens * a.k, from = static_cast<int64_t>(blockIdx.z) * kScan;
  const int n = static_cast<int>(pairs - from < kScan ? pairs - from : kScan);
  for (int e = tid; e < a.E; e += kThreads) place[e] = static_cast<int16_t>(place_of(a, e));
  __syncthreads();
  int h;
  if (a.few) {
    h = look_up(a, place, a.ids[blockIdx.y]);
    if (blockIdx.x == 0 && tid == 0) report(a, h);
    h = h < 0 ? -1 : h;
  } else {
    h = static_cast<int>(blockIdx.y) < a.H ? static_cast<int>(blockIdx.y) : -1;
    if (h < 0 && blockIdx.x == 0)
      for (int i = tid; i < n; i += kThreads) report(a, look_up(a, place, a.ids[from + i]));
  }
  const int count = list_pairs(a, from, n, h, place, list, total);
  if (count == 0 || (a.few && list[0] != blockIdx.y)) return;
  const int column = blockIdx.x * kWidth;
  const int width = GLU ? a.N / 2 : a.N;
  T* out = static_cast<T*>(a.out);
  if (h < 0) {
    if (a.mode == TACG_Q4_SUM) return;
    for (int64_t i = tid; i < static_cast<int64_t>(count) * kWidth; i += kThreads) {
      const int c = column + static_cast<int>(i % kWidth);
      if (c < width) out[(from + list[i / kWidth]) * width + c] = static_cast<T>(0.0f);
    }
    return;
  }
  int64_t row[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    int v = column + 16 * (GLU ? r % (RT / 2) : r) + (lane & 15);
    v = v < width ? v : width - 1;
    row[r] = static_cast<int64_t>(h) * a.N + v + (GLU && r >= RT / 2 ? width : 0);
  }
  const int steps = (a.K + kStep - 1) / kStep;
  for (int base = 0; base < count; base += 16 * TT) {
    const T* x[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int i = base + 16 * t + (lane & 15);
      const uint32_t pair = static_cast<uint32_t>(from) + (i < count ? list[i] : 0);
      const uint32_t token = pair / a.k, j = pair % a.k;
      x[t] = i < count ? static_cast<const T*>(a.x) + token * a.x_token + j * a.x_slot : nullptr;
    }
    float4v sum[RT][TT];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int t = 0; t < TT; ++t) sum[r][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    if (wave < steps) {
      Operands<T, RT, TT, PER> now, next;
      load_step(a, wave, quarter, row, x, now);
      for (int s = wave; s < steps; s += kWaves) {
        if (s + kWaves < steps) load_step(a, s + kWaves, quarter, row, x, next);
        add_step(now, 1.0f, sum);
        now = next;
      }
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      float4v mine[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) mine[r] = sum[r][t];
      join<RT, kWidth>(red, mine, GLU, [&](int token, int c, float v) {
        const int i = base + 16 * t + token;
        if (i >= count || column + c >= width) return;
        const int64_t at = (from + list[i]) * width + column + c;
        if (a.mode == TACG_Q4_SUM) a.part[at] = v;
        else out[at] = static_cast<T>(v);
      });
    }
  }
}

// grid: (blocks of 16 RT weight rows, tokens).
template <class T, int RT, int PER>
__global__ __launch_bounds__(kThreads) void q4_sum_token(Q4Args a) {
  __shared__ float red[kWaves][16][RT * 16 + 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, quarter = lane >> 4;
  __shared__ int held_at[TACG_MAX_TOPK], slots[TACG_MAX_TOPK], count;
  const int64_t t = blockIdx.y;
  if (wave == 0) {  // the served slots, in order
    int h = -1;
    if (lane < a.k) {
      const int id = a.ids[t * a.k + lane];
      h = static_cast<uint32_t>(id) < static_cast<uint32_t>(a.E) ? place_of(a, id) : id == -1 ? -1 : kBadId;
      if (blockIdx.x == 0) report(a, h);
    }
    const uint64_t some = __ballot(h >= 0);
    if (h >= 0) {
      const int at = __popcll(some & ((1ull << lane) - 1));
      held_at[at] = h;
      slots[at] = lane;
    }
    if (lane == 0) count = __popcll(some);
  }
  __syncthreads();
  const int served = count;
  const int column = blockIdx.x * RT * 16;
  const int steps = (a.K + kStep - 1) / kStep, items = served * steps;
  float4v sum[RT][1];
#pragma unroll
  for (int r = 0; r < RT; ++r) sum[r][0] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
  Operands<T, RT, 1, PER> now, next;
  float gate = 0.0f, gate_next = 0.0f;
  auto load = [&](int i, Operands<T, RT, 1, PER>& o, float& g) {
    const int j = i / steps;
    int64_t row[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int v = column + 16 * r + (lane & 15);
      row[r] = static_cast<int64_t>(held_at[j]) * a.N + (v < a.N ? v : a.N - 1);
    }
    const T* x[1] = {(lane & 15) == 0 ? static_cast<const T*>(a.x) + t * a.x_token + slots[j] * a.x_slot : nullptr};
    load_step(a, i % steps, quarter, row, x, o);
    g = a.gate[t * a.k + slots[j]];
  };
  if (wave < items) {
    load(wave, now, gate);
    for (int i = wave; i < items; i += kWaves) {
      if (i + kWaves < items) load(i + kWaves, next, gate_next);
      add_step(now, gate, sum);
      now = next;
      gate = gate_next;
    }
  }
  float4v mine[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) mine[r] = sum[r][0];
  join<RT, RT * 16>(red, mine, false, [&](int token, int c, float v) {
    if (token == 0 && column + c < a.N) static_cast<T*>(a.out)[t * a.N + column + c] = static_cast<T>(v);
  });
}

// grid: (blocks of output columns, tokens).
template <class T>
__global__ __launch_bounds__(256) void q4_combine(Q4Args a) {
  const int n = blockIdx.x * 256 + threadIdx.x;
  if (n >= a.N) return;
  for (int64_t t = blockIdx.y; t < a.n_tokens; t += gridDim.y) {
    float y = 0.0f;
    for (int j = 0; j < a.k; ++j) {
      const int id = a.ids[t * a.k + j];
      if (static_cast<uint32_t>(id) < static_cast<uint32_t>(a.E) && place_of(a, id) >= 0)
        y += a.gate[t * a.k + j] * a.part[(t * a.k + j) * a.N + n];
    }
    static_cast<T*>(a.out)[t * a.N + n] = static_cast<T>(y);
  }
}

struct PackArgs {
  const void* w;
  int64_t stride, rows;
  int32_t K, group, n_groups, pieces;
  uint8_t* q;
  void* scales;
  uint8_t* zeros;
  uint32_t* err;
};

// A lane per 32 columns; group / 32 neighbouring lanes hold a group.  A row's pieces are padded to whole groups of lanes.
template <class T, class S>
__global__ __launch_bounds__(256) void q4_pack_kernel(PackArgs a) {
  const int lanes = a.group / kPiece;
  const int per_row = a.n_groups * lanes;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t r = i / per_row;
  const int p = static_cast<int>(i % per_row);
  const bool in = r < a.rows;
  const T* w = static_cast<const T*>(a.w) + r * a.stride;
  float v[kPiece], lo = 0.0f, hi = 0.0f;
  bool bad = false;
#pragma unroll
  for (int j = 0; j < kPiece; ++j) {
    const int c = p * kPiece + j;
    v[j] = in && c < a.K ? widen(w[c]) : 0.0f;
    bad |= !(fabsf(v[j]) < INFINITY);
    lo = fminf(lo, v[j]);
    hi = fmaxf(hi, v[j]);
  }
  for (int o = 1; o < lanes; o <<= 1) {
    lo = fminf(lo, __shfl_xor(lo, o, 64));
    hi = fmaxf(hi, __shfl_xor(hi, o, 64));
  }
  const S scale = static_cast<S>(a.zeros != nullptr ? (hi - lo) / 15.0f : fmaxf(-lo, hi) / 7.0f);
  const float s = widen(scale);
  if (!(s < INFINITY)) bad = true;
  if (in && bad) atomicOr(a.err, TACG_ERR_VALUE);
  const float zero = a.zeros == nullptr ? 8.0f : s > 0.0f ? fminf(fmaxf(rintf(-lo / s), 0.0f), 15.0f) : 8.0f;
  uint32_t word[4] = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < kPiece; ++j) {
    const float level = s > 0.0f ? fminf(fmaxf(rintf(v[j] / s) + zero, 0.0f), 15.0f) : zero;
    word[j / 8] |= static_cast<uint32_t>(level) << (4 * (j % 8));
  }
  if (!in) return;
  if (p < a.pieces) reinterpret_cast<uint4*>(a.q)[r * a.pieces + p] = make_uint4(word[0], word[1], word[2], word[3]);
  if (p % lanes == 0) {
    const int64_t g = r * a.n_groups + p / lanes;
    static_cast<S*>(a.scales)[g] = scale;
    if (a.zeros != nullptr) a.zeros[g] = static_cast<uint8_t>(zero);
  }
}

template <class T>
void start_pack(const PackArgs& a, int32_t scale_dtype, hipStream_t stream) {
  const int64_t lanes = a.rows * a.n_groups * (a.group / kPiece);
  const dim3 grid(static_cast<uint32_t>((lanes + 255) / 256));
  if (scale_dtype == TACG_BF16) q4_pack_kernel<T, __bf16><<<grid, 256, 0, stream>>>(a);
  else q4_pack_kernel<T, _Float16><<<grid, 256, 0, stream>>>(a);
}

}  // namespace

int launch_q4_pack(const void* w, int32_t dtype, int64_t n_rows, int32_t n_cols, int64_t stride, int32_t group,
                   int32_t scale_dtype, uint8_t* q, void* scales, uint8_t* zeros, uint32_t* d_err, hipStream_t stream) {
  PackArgs a{};
  a.w = w;
  a.stride = stride;
  a.rows = n_rows;
  a.K = n_cols;
  a.group = group;
  a.n_groups = (n_cols + group - 1) / group;
  a.pieces = (n_cols + kPiece - 1) / kPiece;
  a.q = q;
  a.scales = scales;
  a.zeros = zeros;
  a.err = d_err;
  if (dtype == TACG_F32) start_pack<float>(a, scale_dtype, stream);
  else if (dtype == TACG_BF16) start_pack<__bf16>(a, scale_dtype, stream);
  else start_pack<_Float16>(a, scale_dtype, stream);
  return hipGetLastError() == hipSuccess ? TACG_OK : TACG_E_DEVICE;
}

// Few pairs: most have an expert of their own, so a workgroup per pair leaves little to share and wastes none on experts without tokens.
static bool few_pairs(int64_t pairs, int32_t n_experts) { return pairs <= n_experts; }

size_t expert_q4_workspace(int64_t n_tokens, int32_t top_k, int32_t n_experts, int32_t n_rows, int32_t n_cols,
                           int32_t mode) {
  (void)n_cols;
  const int64_t pairs = n_tokens * top_k;
  if (mode != TACG_Q4_SUM || few_pairs(pairs, n_experts)) return 0;
  return align256(static_cast<size_t>(pairs) * n_rows * sizeof(float));
}

namespace {

template <class T, bool GLU, int RT, int TT>
void start_tiles(const Q4Args& a, hipStream_t stream) {
  const int64_t pairs = a.n_tokens * a.k;
  const int width = GLU ? a.N / 2 : a.N, block = GLU ? RT * 8 : RT * 16;
  const dim3 grid((width + block - 1) / block, a.few ? static_cast<uint32_t>(pairs) : a.H + 1,
                  static_cast<uint32_t>((pairs + kScan - 1) / kScan));
  if (a.group == 32) q4_tiles<T, GLU, RT, TT, 4><<<grid, kThreads, 0, stream>>>(a);
  else if (a.group == 64) q4_tiles<T, GLU, RT, TT, 2><<<grid, kThreads, 0, stream>>>(a);
  else q4_tiles<T, GLU, RT, TT, 1><<<grid, kThreads, 0, stream>>>(a);
}

template <class T>
void start(const Q4Args& a, hipStream_t stream) {
  if (a.few && a.mode == TACG_Q4_SUM) {
    const dim3 grid((a.N + 15) / 16, static_cast<uint32_t>(a.n_tokens));
    if (a.group == 32) q4_sum_token<T, 1, 4><<<grid, kThreads, 0, stream>>>(a);
    else if (a.group == 64) q4_sum_token<T, 1, 2><<<grid, kThreads, 0, stream>>>(a);
    else q4_sum_token<T, 1, 1><<<grid, kThreads, 0, stream>>>(a);
    return;
  }
  const bool glu = a.mode == TACG_Q4_GLU;
  const bool two = !a.few && a.n_tokens * a.k > 10 * static_cast<int64_t>(a.E);
  if (glu) two ? start_tiles<T, true, 4, 2>(a, stream) : start_tiles<T, true, 2, 1>(a, stream);
  else two ? start_tiles<T, false, 4, 2>(a, stream) : start_tiles<T, false, 2, 1>(a, stream);
  if (a.mode == TACG_Q4_SUM)
    q4_combine<T><<<dim3((a.N + 255) / 256, static_cast<uint32_t>(std::min<int64_t>(a.n_tokens, 65535))), 256, 0, stream>>>(a);
}

}  // namespace

int launch_expert_q4(const void* x, int32_t dtype, int64_t x_stride_token, int64_t x_stride_slot, int64_t n_tokens,
                     int32_t top_k, int32_t n_experts, const int16_t* ids, const int32_t* slot_of_expert,
                     int32_t n_held, const uint8_t* q, const void* scales, const uint8_t* zeros, int32_t group,
                     int32_t n_rows, int32_t n_cols, int32_t mode, const float* gate, void* out, uint32_t* d_err,
                     void* workspace, hipStream_t stream) {
  Q4Args a{};
  a.x = x;
  a.x_token = x_stride_token;
  a.x_slot = x_stride_slot;
  a.n_tokens = n_tokens;
  a.k = top_k;
  a.E = n_experts;
  a.H = n_held;
  a.N = n_rows;
  a.K = n_cols;
  a.group = group;
  a.n_groups = (n_cols + group - 1) / group;
  a.pieces = (n_cols + kPiece - 1) / kPiece;
  a.mode = mode;
  a.ids = ids;
  a.slot = slot_of_expert;
  a.q = q;
  a.scales = scales;
  a.zeros = zeros;
  a.gate = gate;
  a.out = out;
  a.err = d_err;
  a.few = few_pairs(n_tokens * top_k, n_experts);
  a.part = static_cast<float*>(workspace);
  if (dtype == TACG_BF16) start<__bf16>(a, stream);
  else start<_Float16>(a, stream);
  return hipGetLastError() == hipSuccess ? TACG_OK : TACG_E_DEVICE;
}

}  // namespace tacg
