// Products of the experts' weights in 4 bits with the tokens routed to them.
//
//   W[h][n][c] = scale[h][n][c / group] * (level[h][n][c] - zero[h][n][c / group]),   zero = 8 where none is given.
//
// The products run on the matrix cores, with tokens as rows and weight rows as columns of v_mfma_f32_16x16x32: lane n + 16 q supplies
// columns 8 q .. 8 q + 7 of weight row n and of token n, and holds the sums of weight row n with tokens 4 q .. 4 q + 3.  A step is 256
// columns of 16 weight rows: a lane loads twice 16 bytes, columns 32 q .. 32 q + 31 of 128, and exchanges of half and quarter waves
// give it the words of the step's products, each of 32 columns.  (Without the exchange the tokens' loads would be spread over
// four times as many cache lines.)  A level becomes a 16-bit float by an AND-OR into the mantissa, as offset + level, which is exact; the
// offset and the zero are taken off the group's sum:  sum (level - zero) x = sum (offset + level) x - (offset + zero) sum x,  with sum x
// from a product with ones.  The eight levels of a word come out in the order 0 4 1 5 2 6 3 7, so the tokens' values are put in
// that order too.  The scale of a group is applied in 32 bits to the group's sum.
//
// q4_tiles: many (token, slot) pairs.  A workgroup takes an expert and a block of its weight rows and finds the expert's tokens by itself
//   (no launch before it); every wave has rows of its own, and the tokens' values come through LDS.  512 tokens through 256 experts of
//   2048 x 4096, top-8, gated: 281 us, 4.0 TB/s of weights (the same loads without the products: 253; a copy reaches 4.8 TB/s); bound
//   by the latency of a step (LDS, products, barrier) that two waves a SIMD do not quite hide.  32 tokens through 128 experts
//   of 1536 x 2048: 63 us, 3.1 TB/s, where a workgroup has eight steps in all.  A second step of weights in flight cost more in
//   registers than it gave (77 and 331 us).  Where experts and columns alone leave processors idle, several workgroups share an
//   expert's tokens: a token's place in its tile, and so its bits, stay the same.
// q4_few: few pairs.  A workgroup takes 16 weight rows (gated: 16 pairs of them) of the expert of one pair, or, summed, of all experts of a
//   token; its waves take the steps in turn and add their sums up in LDS, in order.  One token through six experts of 2048 x 2048:
//   8.2 us; through eight of 4096 x 2048, summed: 11 us, 3.4 TB/s; bound by latency: a wave has one to four steps.
#pragma once

#include <type_traits>

#include "tacg_internal.h"

namespace tacg {

// Few pairs: most have an expert of their own, so a workgroup per pair (or token) leaves little to share and wastes none on experts
// without tokens.  Measured, few against many in us: gated, 128 experts of 1536 x 2048, top-8: 20.1 / 30.4 at 4 tokens, 29.9 / 30.4
// at 6, 36.2 / 30.7 at 8; 60 experts of 2048 x 2048, top-4: 14.1 / 23.0 at 4, 20.6 / 23.2 at 6, 25.5 / 23.5 at 8.  Each: 22.6 / 30.1,
// 31.3 / 30.3, 39.4 / 30.9; 16.3 / 23.1, 21.8 / 23.2, 28.1 / 23.6.  Summed (2048 x 1024): 31.3 / 33.7 at 16 tokens of 128 experts,
// 56.0 / 37.1 at 32; 17.7 / 21.2 at 15 of 60, 17.9 / 21.8 at 16, 32.9 / 22.7 at 32.
// The rule goes by the pairs alone, so it is not the faster one everywhere: 256 experts of 2048 x 1024, top-8, 8 tokens: gated 37.1 / 26.4, each
// 44.3 / 26.0; summed, 256 of 4096 x 2048, 32 tokens: 233 / 179.  An expert's pairs go two at a time: 100 pairs that all choose one of
// 256 experts of 2048 x 2048: gated 122 / 74.6, each 71.8 / 74.3.
inline bool q4_few_pairs(int64_t pairs, int32_t n_experts, int32_t mode) {
  return mode == TACG_Q4_SUM ? pairs <= n_experts : 5 * pairs <= 2 * static_cast<int64_t>(n_experts);
}

constexpr int kPiece = 32;  // columns of 16 bytes of levels

struct Q4Args {
  const void* x;
  int64_t x_token, x_slot;  // strides in elements
  int64_t n_tokens;
  int32_t k, E, H, N, K, group, n_groups, pieces, mode;
  int32_t shares;           // workgroups that take an expert's tiles of tokens in turn (many pairs)
  const int16_t* ids;
  const int32_t* slot;      // [E] or null
  const uint8_t* q;
  const void* scales;
  const uint8_t* zeros;     // or null
  const float* gate;        // [T][k] or null
  float* part;              // [T][k][N], or null
  void* out;
  uint32_t* err;
};


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

constexpr int kStep = 256;       // columns of a step
constexpr int kBlocks = kStep / 32;
constexpr int kScan = 4096;      // pairs that a workgroup looks through

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

// 16-bit floats offset + level of the eight levels of a word, in the order 0 4 1 5 2 6 3 7: four bits under the mantissa's bit of
// weight 1.  A level in bits 4 to 7 needs an offset of 64 in float16, in bits 0 to 3 one of 1024, which would cost the sums four bits.
template <class T>
constexpr float kOffset = __is_same(T, __bf16) ? 128.0f : 64.0f;
// The four bits of each half, in a vector register that the compiler takes for a variable: an AND-OR takes one scalar operand, and with two
// known ones it becomes two instructions.
template <class T>
__device__ __forceinline__ uint32_t level_mask() {
  return __builtin_amdgcn_mbcnt_lo(0, __is_same(T, __bf16) ? 0x000f000fu : 0x00f000f0u);
}
template <class T>
__device__ __forceinline__ uint4v spread(uint32_t w, uint32_t mask) {
  if constexpr (__is_same(T, __bf16)) {
    constexpr uint32_t kBase = 0x43004300u;
    return uint4v{(w & mask) | kBase, ((w >> 4) & mask) | kBase, ((w >> 8) & mask) | kBase, ((w >> 12) & mask) | kBase};
  } else {
    constexpr uint32_t kBase = 0x54005400u;
    return uint4v{((w << 4) & mask) | kBase, (w & mask) | kBase, ((w >> 4) & mask) | kBase, ((w >> 8) & mask) | kBase};
  }
}

// The matrix that a workgroup reads, and where a lane's rows lie in it.
template <class T, int RT>
struct Rows {
  const char* level;
  const T* scale;
  const uint8_t* zero;
  uint32_t at[RT];  // row
};

// A step's weights of a lane, as loaded.  GROUPS: scale groups of a step, two scales and four zeros to a word.  ZEROS: whether zeros are
// given (a choice at run time would merge two values after their load, and so wait for it there).
template <class T, int RT, int GROUPS, bool ZEROS>
struct Weights {
  uint4v level[RT][2];
  uint32_t scale[RT][(GROUPS + 1) / 2];
  uint32_t zero[ZEROS ? RT : 1][(GROUPS + 3) / 4];
};

template <class T, int RT>
__device__ __forceinline__ Rows<T, RT> rows_of(const Q4Args& a, int h) {
  const int64_t first = static_cast<int64_t>(h < 0 ? 0 : h) * a.N;
  Rows<T, RT> o;
  o.level = reinterpret_cast<const char*>(a.q) + first * a.pieces * 16;
  o.scale = static_cast<const T*>(a.scales) + first * a.n_groups;
  o.zero = a.zeros + first * a.n_groups;
  return o;
}

// The words of N values of a row's groups from `first` on; past the row's end any that can be read safely (the tokens' values are 0 there).
// WHOLE: none lies past it.
template <int N, bool WHOLE, class V, int W>
__device__ __forceinline__ void load_groups(const V* row, int first, int n_groups, uint32_t (&o)[W]) {
  constexpr int kBits = 8 * sizeof(V);
  if constexpr (WHOLE) {
    if constexpr (N * sizeof(V) < 4) {
      o[0] = 0;
      __builtin_memcpy(o, row + first, N * sizeof(V));
    } else {
      __builtin_memcpy(o, row + first, sizeof(o));
    }
  } else if (n_groups >= N) {
    const int from = first + N <= n_groups ? first : n_groups - N, skip = (first - from) * kBits;
    if constexpr (N * sizeof(V) < 4) {
      o[0] = 0;
      __builtin_memcpy(o, row + from, N * sizeof(V));
    } else {
      __builtin_memcpy(o, row + from, sizeof(o));
    }
    if (skip > 0) {  // the last step: bring the first group to the front
#pragma unroll
      for (int w = 0; w < W; ++w) {
        uint32_t v = 0;
#pragma unroll
        for (int u = 0; u + w < W; ++u) {
          const int by = skip - 32 * u;
          if (by >= 0 && by < 32) v = o[w + u] >> by;
          if (by < 0 && by > -32) v |= o[w + u] << -by;
        }
        o[w] = v;
      }
    }
  } else {
#pragma unroll
    for (int w = 0; w < W; ++w) o[w] = 0;
#pragma unroll
    for (int g = 0; g < N; ++g) {
      V v = row[first + g < n_groups ? first + g : n_groups - 1];
      uint32_t bits = 0;
      __builtin_memcpy(&bits, &v, sizeof(V));
      o[g * kBits / 32] |= bits << (g * kBits % 32);
    }
  }
}

// group: the lane's first one.  WHOLE: the step ends before the columns do.  A choice at run time would make the compiler wait for the fewest loads that either way issues.
template <bool WHOLE, class T, int RT, int GROUPS, bool ZEROS>
__device__ __forceinline__ void load_weights(const Q4Args& a, int column, int quarter, int group, const Rows<T, RT>& rows,
                                             Weights<T, RT, GROUPS, ZEROS>& o) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int piece = column / kPiece + 4 * i + quarter;  // past the end the tokens' values are 0: any levels do
    if (!WHOLE) piece = piece < a.pieces ? piece : a.pieces - 1;
#pragma unroll
    for (int r = 0; r < RT; ++r)
      o.level[r][i] = *reinterpret_cast<const uint4v*>(rows.level + 16u * (rows.at[r] * a.pieces + piece));
  }
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    load_groups<GROUPS, WHOLE>(rows.scale + rows.at[r] * a.n_groups, group, a.n_groups, o.scale[r]);
    if constexpr (ZEROS) load_groups<GROUPS, WHOLE>(rows.zero + rows.at[r] * a.n_groups, group, a.n_groups, o.zero[r]);
  }
}

// Eight values of a token from column c on, 0 past the columns' end.
template <bool WHOLE, class T>
__device__ __forceinline__ uint4v load_token(const Q4Args& a, const T* x, int c) {
  uint4v o = {0, 0, 0, 0};
  if (WHOLE || c + 8 <= a.K) {
    __builtin_memcpy(&o, x + c, 16);  // rows need not be aligned to more than an element
  } else if (c < a.K) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint16_t v = 0;
      if (c + j < a.K) __builtin_memcpy(&v, x + c + j, 2);
      o[j / 2] |= static_cast<uint32_t>(v) << (16 * (j % 2));
    }
  }
  return o;
}

// The order in which spread() gives the levels.
__device__ __forceinline__ uint4v in_order(const uint4v& v) {
  return uint4v{__builtin_amdgcn_perm(v[2], v[0], 0x05040100u), __builtin_amdgcn_perm(v[2], v[0], 0x07060302u),
                __builtin_amdgcn_perm(v[3], v[1], 0x05040100u), __builtin_amdgcn_perm(v[3], v[1], 0x07060302u)};
}

template <class T>
__device__ __forceinline__ float half_of(uint32_t word, int i) {
  return static_cast<float>(__builtin_bit_cast(T, static_cast<uint16_t>(word >> (16 * i))));
}

// The words of the lane's row in the order of the step's products.
template <class T, int RT, int GROUPS, bool ZEROS>
__device__ __forceinline__ void exchange(const Weights<T, RT, GROUPS, ZEROS>& o, uint32_t (&w)[RT][kBlocks]) {
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4v l = o.level[r][i];
      const auto a = __builtin_amdgcn_permlane32_swap(l[0], l[2], false, false);
      const auto b = __builtin_amdgcn_permlane32_swap(l[1], l[3], false, false);
      const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
      const auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
      w[r][4 * i] = c[0];
      w[r][4 * i + 1] = c[1];
      w[r][4 * i + 2] = d[0];
      w[r][4 * i + 3] = d[1];
    }
}

// One in all columns (zeros given), or -(offset + 8): what takes the offset off.
template <class T, bool ZEROS>
__device__ __forceinline__ uint4v ones() {
  constexpr uint32_t kOne = __is_same(T, __bf16) ? (ZEROS ? 0x3f80u : 0xc308u) : (ZEROS ? 0x3c00u : 0xd480u);
  constexpr uint32_t kTwo = kOne | kOne << 16;
  return uint4v{kTwo, kTwo, kTwo, kTwo};
}

// sum += factor * scale * (level - zero) . x of one step; tokens(t, i): the lane's ordered values of block i of token tile t.
template <class T, int RT, int TT, int GROUPS, bool ZEROS, class Tokens>
__device__ __forceinline__ void add_step(const Weights<T, RT, GROUPS, ZEROS>& o, Tokens tokens, float factor,
                                         float4v (&sum)[RT][TT]) {
  constexpr int kRun = kBlocks / GROUPS;  // products of a group
  const uint32_t mask = level_mask<T>();
  uint32_t w[RT][kBlocks];
  exchange(o, w);
#pragma unroll
  for (int g = 0; g < GROUPS; ++g) {
    float4v all[TT], part[RT][TT];
    uint4v x[TT][kRun];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      all[t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        x[t][i] = tokens(t, g * kRun + i);
        all[t] = mfma(x[t][i], ones<T, ZEROS>(), all[t], T());
      }
#pragma unroll
      for (int r = 0; r < RT; ++r) part[r][t] = ZEROS ? float4v{0.0f, 0.0f, 0.0f, 0.0f} : all[t];
    }
#pragma unroll
    for (int i = 0; i < kRun; ++i)
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const uint4v v = spread<T>(w[r][g * kRun + i], mask);
#pragma unroll
        for (int t = 0; t < TT; ++t) part[r][t] = mfma(x[t][i], v, part[r][t], T());
      }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const float scale = half_of<T>(o.scale[r][g / 2], g % 2) * factor;
      const float zero = ZEROS ? kOffset<T> + static_cast<float>((o.zero[ZEROS ? r : 0][g / 4] >> (8 * (g % 4))) & 255u) : 0.0f;
#pragma unroll
      for (int t = 0; t < TT; ++t) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[r][t][j] += scale * (ZEROS ? part[r][t][j] - zero * all[t][j] : part[r][t][j]);
        asm volatile("" : "+v"(sum[r][t]));  // here, and not with the other groups: all their products would not fit the registers
      }
    }
  }
}

// One or two tokens: the 16 rows of a product hold the eight blocks of a step of each, lane n + 16 q the columns 8 q .. 8 q + 7 of block n & 7
// of token n >> 3, and the product with the weights of block i is right in its rows i and 8 + i.  One read of the tokens serves
// the step's products, one product gives the sums of x of all blocks, and a lane has a quarter of the results to scale: those of
// blocks 4 (q & 1) .. of token q >> 1.  The weights hold the lane's groups alone.
constexpr int rows_groups(int groups) { return groups > 1 ? groups / 2 : 1; }
__device__ __forceinline__ int rows_group(int groups, int column, int quarter) {
  return column * groups / kStep + (groups > 1 ? (quarter & 1) * (groups / 2) : 0);
}
template <class T, int RT, int GROUPS, bool ZEROS>
__device__ __forceinline__ void add_rows(const Weights<T, RT, GROUPS, ZEROS>& o, const uint4v& x, bool upper, float factor,
                                         float (&sum)[RT]) {
  const float4v none = {0.0f, 0.0f, 0.0f, 0.0f};
  const uint32_t mask = level_mask<T>();
  const float4v all = mfma(x, ones<T, ZEROS>(), none, T());
  uint32_t w[RT][kBlocks];
  exchange(o, w);
#pragma unroll
  for (int r = 0; r < RT; ++r) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float low = mfma(x, spread<T>(w[r][j], mask), ZEROS ? none : all, T())[j];
      const float high = mfma(x, spread<T>(w[r][j + 4], mask), ZEROS ? none : all, T())[j];
      const int g = j * GROUPS / 4;
      float v = upper ? high : low;
      if (ZEROS) v -= (kOffset<T> + static_cast<float>((o.zero[ZEROS ? r : 0][g / 4] >> (8 * (g % 4))) & 255u)) * all[j];
      sum[r] += half_of<T>(o.scale[r][g / 2], g % 2) * factor * v;
      if (j % 2 == 1) asm volatile("" : "+v"(sum[r]));  // here: all products of the step would not fit the registers
    }
  }
}
// The two quarters of a token together.
__device__ __forceinline__ float rows_total(float v) {
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

__device__ __forceinline__ float silu(float v) { return v / (1.0f + __expf(-v)); }

__device__ __forceinline__ int look_up(const Q4Args& a, const int16_t* place, int id) {
  return static_cast<uint32_t>(id) < static_cast<uint32_t>(a.E) ? place[id] : id == -1 ? -1 : kBadId;
}
__device__ __forceinline__ int served_by(const Q4Args& a, const int16_t* place, int id) {
  const int h = look_up(a, place, id);
  return h < 0 ? -1 : h;
}

// Where the pairs from `from` on, `n` of them, that matrix `h` serves (h = -1: that no matrix serves) stand in the list, in order.
// A thread takes 8 V neighbouring ids, all loaded before the first is looked at.
template <int V, int WAVES>
__device__ __forceinline__ int list_pairs(const Q4Args& a, int64_t from, int n, int h, const int16_t* place,
                                          uint16_t* list, int (&total)[WAVES]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int first = tid * 8 * V;
  int16_t ids[8 * V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int16_t* p = a.ids + from + first + 8 * v;
    if (first + 8 * v + 8 <= n) {
      __builtin_memcpy(ids + 8 * v, p, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) ids[8 * v + i] = first + 8 * v + i < n ? p[i] : -1;
    }
  }
  uint32_t mine = 0;
#pragma unroll
  for (int i = 0; i < 8 * V; ++i) mine |= (first + i < n && served_by(a, place, ids[i]) == h ? 1u : 0u) << i;
  int at = __popc(mine);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(at, o, 64);
    if (lane >= o) at += v;
  }
  if (lane == 63) total[wave] = at;
  __syncthreads();
  at -= __popc(mine);
  int all = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w < wave) at += total[w];
    all += total[w];
  }
  while (mine != 0) {
    list[at++] = static_cast<uint16_t>(first + __ffs(mine) - 1);
    mine &= mine - 1;
  }
  __syncthreads();
  return all;
}

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kTokenBytes = kStep * 2 + 16;  // of a token's step in LDS: 16 tokens' pieces lie in different banks

// RAGGED: the columns are no whole number of groups, or less than a step.  Otherwise the last step starts where it still has kStep
// columns, with the tokens' values of those that the step before has had as 0: no load needs a bound.
template <bool RAGGED>
__device__ __forceinline__ int first_column(const Q4Args& a, int s) {
  const int c = s * kStep;
  return RAGGED || c + kStep <= a.K ? c : a.K - kStep;
}

// Tokens base .. of a workgroup's list, 16 TT at most (TT = 0: one or two), with its weight rows: every wave has rows of its own; the
// tokens' values come through LDS, a step ahead, in two buffers.
template <class T, bool GLU, int RT, int TT, int GROUPS, bool ZEROS, bool RAGGED>
__device__ __forceinline__ void tokens_with_rows(const Q4Args& a, const Rows<T, RT>& rows, const uint16_t* list, int64_t from,
                                                 int base, int count, int column, char (*held)[kTokenBytes]) {
  constexpr bool kFew = TT == 0;
  constexpr int kTiles = kFew ? 1 : TT, kTokens = kFew ? 2 : 16 * TT;
  constexpr int kHeld = kFew ? rows_groups(GROUPS) : GROUPS;  // groups of a step that a lane needs
  constexpr int kLoads = (kTokens + 7) / 8;  // 16-byte pieces of a step's tokens that a thread brings
  const int tid = threadIdx.x, lane = tid & 63, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int width = GLU ? a.N / 2 : a.N;
  const int row = lane & 15;
  const bool brings = kTokens >= 8 || (tid >> 5) < kTokens;
  const T* x[kLoads];
  uint4v piece[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int at = base + 8 * i + (tid >> 5);  // past the last token: its values again, for sums that nobody takes
    const uint32_t pair = static_cast<uint32_t>(from) + list[at < count ? at : count - 1];
    const uint32_t t = pair / a.k, j = pair % a.k;
    x[i] = static_cast<const T*>(a.x) + t * a.x_token + j * a.x_slot;
  }
  const int last = RAGGED ? a.K / kStep - 1 : (a.K + kStep - 1) / kStep - 1;  // of the steps without a columns' end
  auto fetch = [&](auto whole, int s) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) piece[i] = load_token<whole.value>(a, x[i], first_column<RAGGED>(a, s) + 8 * (tid & 31));
  };
  auto buffer = [&](int s, int t) { return held[(s & 1) * kTokens + t]; };
  auto stage = [&](int s) {
    if (!RAGGED && s == last && first_column<RAGGED>(a, s) + 8 * (tid & 31) < s * kStep) {  // columns of the step before
#pragma unroll
      for (int i = 0; i < kLoads; ++i) piece[i] = uint4v{0, 0, 0, 0};
    }
    if (brings) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        *reinterpret_cast<uint4v*>(buffer(s, 8 * i + (tid >> 5)) + 16 * (tid & 31)) = in_order(piece[i]);
    }
  };
  float4v sum[RT][kTiles];
  float few[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    few[r] = 0.0f;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) sum[r][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
  }
  Weights<T, RT, kHeld, ZEROS> now, next;
  auto load = [&](auto whole, int s, auto& w) {
    const int c = first_column<RAGGED>(a, s);
    load_weights<whole.value>(a, c, quarter, kFew ? rows_group(GROUPS, c, quarter) : c * GROUPS / kStep, rows, w);
  };
  auto add = [&](int s) {
    if constexpr (kFew) {
      add_rows(now, *reinterpret_cast<const uint4v*>(buffer(s, row >> 3) + 64 * (row & 7) + 16 * quarter), (quarter & 1) != 0,
               1.0f, few);
    } else {
      add_step<T, RT, kTiles, GROUPS, ZEROS>(now, [&](int t, int i) {
        return *reinterpret_cast<const uint4v*>(buffer(s, 16 * t + row) + 64 * i + 16 * quarter);
      }, 1.0f, sum);
    }
  };
  const std::true_type whole;
  if (last >= 0) {
    fetch(whole, 0);
    load(whole, 0, now);
    stage(0);
    fetch(whole, last < 1 ? last : 1);
  }
  __syncthreads();
  for (int s = 0; s <= last; ++s) {  // what is brought after the last step is not used
    load(whole, s < last ? s + 1 : last, next);
    add(s);
    stage(s + 1);
    fetch(whole, s + 2 <= last ? s + 2 : last);
    __syncthreads();
    now = next;
  }
  if (RAGGED && (last + 1) * kStep < a.K) {
    fetch(std::false_type(), last + 1);
    load(std::false_type(), last + 1, now);
    stage(last + 1);
    __syncthreads();
    add(last + 1);
  }
  __syncthreads();  // the buffers are free for the next tokens
  constexpr int kRows = GLU ? RT / 2 : RT;
  T* out = static_cast<T*>(a.out);
  if constexpr (kFew) {
#pragma unroll
    for (int r = 0; r < RT; ++r) few[r] = rows_total(few[r]);
  }
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int j = 0; j < (kFew ? 1 : 4); ++j) {
      const int i = base + (kFew ? quarter >> 1 : 16 * t + 4 * quarter + j);
      if (i >= count || (kFew && (quarter & 1) != 0)) continue;
      const int64_t at = (from + list[i]) * width;
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const int c = column + wave * 16 * kRows + 16 * r + row;
        if (c >= width) continue;
        float v = kFew ? few[r] : sum[r][t][j];
        if constexpr (GLU) v = silu(v) * (kFew ? few[r + kRows] : sum[r + kRows][t][j]);
        if (a.mode == TACG_Q4_SUM) a.part[at + c] = v;
        else out[at + c] = static_cast<T>(v);
      }
    }
}

// Many pairs.  grid: (blocks of a workgroup's output columns, held experts and one for the pairs that none serves, runs of kScan pairs
// times shares of the tiles of tokens).
template <class T, bool GLU, int RT, int TT, int GROUPS, bool ZEROS, bool RAGGED>
__global__ __launch_bounds__(kThreads, TT == 1 ? 3 : 2) void q4_tiles(Q4Args a) {
  constexpr int kOut = GLU ? RT * 8 : RT * 16;  // output columns of a wave
  constexpr int kWidth = kOut * kWaves;         // of the workgroup
  __shared__ alignas(16) char held[2 * 16 * TT][kTokenBytes];
  __shared__ uint16_t list[kScan];
  __shared__ int16_t place[TACG_MAX_EXPERTS];
  __shared__ int total[kWaves];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t pairs = a.n_tokens * a.k, from = static_cast<int64_t>(blockIdx.z / a.shares) * kScan;
  const int share = blockIdx.z % a.shares;
  const int n = static_cast<int>(pairs - from < kScan ? pairs - from : kScan);
  for (int e = tid; e < a.E; e += kThreads) place[e] = static_cast<int16_t>(place_of(a, e));
  const int h = static_cast<int>(blockIdx.y) < a.H ? static_cast<int>(blockIdx.y) : -1;
  const int column = blockIdx.x * kWidth;
  const int width = GLU ? a.N / 2 : a.N;
  __syncthreads();
  const int count = n <= kThreads * 8 ? list_pairs<1>(a, from, n, h, place, list, total)
                                      : list_pairs<2>(a, from, n, h, place, list, total);
  if (h < 0) {
    if (blockIdx.x == 0 && share == 0)
      for (int i = tid; i < n; i += kThreads) report(a, look_up(a, place, a.ids[from + i]));
    if (a.mode == TACG_Q4_SUM) return;
    auto clear = [&](auto value) {  // three of four of 4096 pairs of 1024 columns: 16 bytes at a time 16.5 us a call, one value at a time 57
      constexpr int kEach = sizeof(value) / sizeof(T), kRow = kWidth / kEach;
      for (int i = share * kThreads + tid; i < count * kRow; i += a.shares * kThreads) {
        const int c = column + i % kRow * kEach;
        if (c < width) *reinterpret_cast<decltype(value)*>(static_cast<T*>(a.out) + (from + list[i / kRow]) * width + c) = value;
      }
    };
    if (width % 8 == 0 && reinterpret_cast<uintptr_t>(a.out) % 16 == 0) clear(uint4v{0, 0, 0, 0});
    else clear(static_cast<T>(0.0f));
    return;
  }
  Rows<T, RT> rows = rows_of<T, RT>(a, h);
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    int v = column + wave * kOut + 16 * (GLU ? r % (RT / 2) : r) + (lane & 15);
    v = v < width ? v : width - 1;
    rows.at[r] = v + (GLU && r >= RT / 2 ? width : 0);
  }
  for (int base = share * 16 * TT; base < count; base += a.shares * 16 * TT) {
    const int left = count - base;
    if (TT == 2 && left > 16) tokens_with_rows<T, GLU, RT, TT, GROUPS, ZEROS, RAGGED>(a, rows, list, from, base, count, column, held);
    else if (left > 2) tokens_with_rows<T, GLU, RT, 1, GROUPS, ZEROS, RAGGED>(a, rows, list, from, base, count, column, held);
    else tokens_with_rows<T, GLU, RT, 0, GROUPS, ZEROS, RAGGED>(a, rows, list, from, base, count, column, held);
  }
}

// Few pairs.  The waves of a workgroup share its weight rows and take the steps in turn; their sums are added up in LDS, in order.
// grid: (blocks of 16 output columns; EACH and GLU: pairs, of which the first of each expert serves all of them, SUM: tokens).
template <class T, int MODE, int WAVES, int GROUPS, bool ZEROS, bool RAGGED>
__global__ __launch_bounds__(WAVES * 64, 4) void q4_few(Q4Args a) {
  constexpr bool GLU = MODE == TACG_Q4_GLU, SUM = MODE == TACG_Q4_SUM;
  constexpr int RT = GLU ? 2 : 1;
  constexpr int kTokens = SUM ? 1 : 2;
  __shared__ float red[WAVES][kTokens][RT * 16];
  __shared__ uint16_t list[TACG_MAX_EXPERTS];
  __shared__ int16_t place[TACG_MAX_EXPERTS];
  __shared__ int total[WAVES];
  const int tid = threadIdx.x, lane = tid & 63, quarter = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int width = GLU ? a.N / 2 : a.N;
  const int n = blockIdx.x * 16 + (lane & 15), column = n < width ? n : width - 1;
  const int steps = (a.K + kStep - 1) / kStep;
  T* out = static_cast<T*>(a.out);
  int h = -1, count;
  if constexpr (SUM) {  // list: the token's served slots, place: their matrices
    if (wave == 0) {
      int p = -1;
      if (lane < a.k) {
        const int id = a.ids[blockIdx.y * a.k + lane];
        p = static_cast<uint32_t>(id) < static_cast<uint32_t>(a.E) ? place_of(a, id) : id == -1 ? -1 : kBadId;
        if (blockIdx.x == 0) report(a, p);
      }
      const uint64_t some = __ballot(p >= 0);
      if (p >= 0) {
        const int at = __popcll(some & ((1ull << lane) - 1));
        place[at] = static_cast<int16_t>(p);
        list[at] = static_cast<uint16_t>(lane);
      }
      if (lane == 0) total[0] = __popcll(some);
    }
    __syncthreads();
    count = total[0];
  } else {
    for (int e = tid; e < a.E; e += WAVES * 64) place[e] = static_cast<int16_t>(place_of(a, e));
    __syncthreads();
    h = look_up(a, place, a.ids[blockIdx.y]);
    if (blockIdx.x == 0 && tid == 0) report(a, h);
    h = h < 0 ? -1 : h;
    count = list_pairs<1>(a, 0, static_cast<int>(a.n_tokens * a.k), h, place, list, total);
    if (list[0] != blockIdx.y) return;
    if (h < 0) {
      for (int i = tid; i < 16 * count; i += WAVES * 64)
        if (blockIdx.x * 16 + i % 16 < width)
          out[static_cast<int64_t>(list[i / 16]) * width + blockIdx.x * 16 + i % 16] = static_cast<T>(0.0f);
      return;
    }
  }
  const int items = SUM ? count * steps : steps;
  Rows<T, RT> rows = rows_of<T, RT>(a, h);
  rows.at[0] = column;
  if constexpr (GLU) rows.at[1] = column + width;
  for (int base = 0; base < (SUM ? 1 : count); base += 2) {
    const T* x = static_cast<const T*>(a.x);
    if constexpr (SUM) {
      x += blockIdx.y * a.x_token;
    } else {
      const int i = base + ((lane >> 3) & 1);  // past the last token: its values again, for sums that nobody takes
      const uint32_t pair = list[i < count ? i : count - 1];
      x += static_cast<int64_t>(pair / a.k) * a.x_token + static_cast<int64_t>(pair % a.k) * a.x_slot;
    }
    float sum[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) sum[r] = 0.0f;
    Weights<T, RT, rows_groups(GROUPS), ZEROS> now, next;
    uint4v piece, piece_next;
    float factor = 1.0f, factor_next = 1.0f;
    int skip = 0, skip_next = 0;  // columns of a step that the step before has had
    auto load = [&](int i, auto& w, uint4v& v, float& f, int& skip) {
      int s = i;
      const T* token = x;
      if constexpr (SUM) {
        const int j = i / steps, slot = __builtin_amdgcn_readfirstlane(list[j]);
        s = i - j * steps;
        rows = rows_of<T, RT>(a, __builtin_amdgcn_readfirstlane(place[j]));
        rows.at[0] = column;
        f = a.gate[blockIdx.y * a.k + slot];
        token += slot * a.x_slot;
      }
      const int from = first_column<RAGGED>(a, s), c = from + 32 * (lane & 7) + 8 * quarter;
      const int group = rows_group(GROUPS, from, quarter);
      if (!RAGGED || (s + 1) * kStep <= a.K) {
        v = load_token<true>(a, token, c);
        load_weights<true>(a, from, quarter, group, rows, w);
      } else {
        v = load_token<false>(a, token, c);
        load_weights<false>(a, from, quarter, group, rows, w);
      }
      skip = s * kStep - from;
    };
    if (wave < items) load(wave, now, piece, factor, skip);
    for (int i = wave; i < items; i += WAVES) {
      if (i + WAVES < items) load(i + WAVES, next, piece_next, factor_next, skip_next);
      if (!RAGGED && 32 * (lane & 7) + 8 * quarter < skip) piece = uint4v{0, 0, 0, 0};
      add_rows(now, in_order(piece), (quarter & 1) != 0, factor, sum);
      skip = skip_next;
      now = next;
      piece = piece_next;
      factor = factor_next;
    }
    if (base > 0) __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      sum[r] = rows_total(sum[r]);
      if ((quarter & 1) == 0 && (quarter >> 1) < kTokens) red[wave][quarter >> 1][16 * r + (lane & 15)] = sum[r];
    }
    __syncthreads();
    if (tid < 16 * kTokens) {
      const int t = tid / 16, c = blockIdx.x * 16 + tid % 16;
      if (c < width && (SUM || base + t < count)) {
        float y = 0.0f, u = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          y += red[w][t][tid % 16];
          if (GLU) u += red[w][t][tid % 16 + (GLU ? 16 : 0)];
        }
        const int64_t at = SUM ? blockIdx.y : list[base + t];
        out[at * width + c] = static_cast<T>(GLU ? silu(y) * u : y);
      }
    }
  }
}

// launch(groups of a step, whether zeros are given)
template <class Launch>
void by_weights(const Q4Args& a, Launch launch) {
  auto with = [&](auto groups) {
    if (a.zeros != nullptr) launch(groups, std::true_type());
    else launch(groups, std::false_type());
  };
  if (a.group == 32) with(std::integral_constant<int, 8>());
  else if (a.group == 64) with(std::integral_constant<int, 4>());
  else if (a.group == 128) with(std::integral_constant<int, 2>());
  else with(std::integral_constant<int, 1>());
}

// Shares of an expert's tiles of tokens: a grid that leaves processors idle spreads them, up to 512 workgroups, and as many as twice
// the mean of an expert's tokens fills.  One share against this rule in us, 512 tokens: each, 8 experts of 1024 x 2048, top-2:
// 45.7 / 22.6; gated, 2048 x 2048: 59.8 / 29.2 (a limit of 256: 38.8, of 1024: 32.4), 4096 x 2048: 62.2 / 42.6 (61.1, 47.9).
inline int32_t q4_shares(int64_t workgroups, int64_t pairs, int32_t n_experts, int32_t tokens) {
  const int64_t fills = 512 / workgroups, tiles = (2 * pairs / n_experts + tokens - 1) / tokens;
  const int64_t shares = fills < tiles ? fills : tiles;
  return static_cast<int32_t>(shares < 1 ? 1 : shares);
}

template <class T, bool RAGGED, bool GLU, int RT, int TT>
void start_tiles(Q4Args a, hipStream_t stream) {
  const int64_t pairs = a.n_tokens * a.k;
  const int width = GLU ? a.N / 2 : a.N, block = (GLU ? RT * 8 : RT * 16) * kWaves;
  const int64_t runs = (pairs + kScan - 1) / kScan, columns = (width + block - 1) / block;
  a.shares = q4_shares(columns * (a.H > 0 ? a.H : 1) * runs, pairs < kScan ? pairs : kScan, a.E, 16 * TT);
  const dim3 grid(static_cast<uint32_t>(columns), a.H + 1, static_cast<uint32_t>(runs * a.shares));
  by_weights(a, [&](auto groups, auto zeros) {
    q4_tiles<T, GLU, RT, TT, groups.value, zeros.value, RAGGED><<<grid, kThreads, 0, stream>>>(a);
  });
}

template <class T, bool RAGGED, int MODE, int WAVES>
void start_few(const Q4Args& a, hipStream_t stream) {
  const int width = MODE == TACG_Q4_GLU ? a.N / 2 : a.N;
  const dim3 grid((width + 15) / 16, static_cast<uint32_t>(MODE == TACG_Q4_SUM ? a.n_tokens : a.n_tokens * a.k));
  by_weights(a, [&](auto groups, auto zeros) {
    q4_few<T, MODE, WAVES, groups.value, zeros.value, RAGGED><<<grid, WAVES * 64, 0, stream>>>(a);
  });
}

template <class T, bool RAGGED>
void q4_start(const Q4Args& a, hipStream_t stream) {
  const int64_t pairs = a.n_tokens * a.k;
  const bool glu = a.mode == TACG_Q4_GLU;
  if (q4_few_pairs(pairs, a.E, a.mode)) {
    if (a.mode == TACG_Q4_SUM) start_few<T, RAGGED, TACG_Q4_SUM, 16>(a, stream);
    else if (glu) start_few<T, RAGGED, TACG_Q4_GLU, 8>(a, stream);
    else start_few<T, RAGGED, TACG_Q4_EACH, 8>(a, stream);
    return;
  }
  // Two tiles of tokens from ten an expert on: with 2048 x 2048 and 128 experts 72.9 us against 70.1 at ten, 85 / 71 at twelve,
  // 104 / 73 at sixteen (one against two tiles), below it the other way: 66.1 / 69.2 at eight.
  // Rows of a wave, by the workgroups of 256 rows that there are: 64 from 512 on with two tiles of tokens (36.5 us against 43.1
  // with 32; at 256: 23.6 / 22.1), 16 below 128 (13.3 against 16.3 with 32 at 64; at 256: 30.4 / 21.9), else 32.
  const int64_t wide = static_cast<int64_t>(a.H) * ((a.N + 255) / 256);
  const bool two = pairs > 10 * static_cast<int64_t>(a.E);
  if constexpr (!RAGGED) {
    if (two && wide >= 512) return glu ? start_tiles<T, RAGGED, true, 4, 2>(a, stream) : start_tiles<T, RAGGED, false, 4, 2>(a, stream);
    if (!glu && wide < 128) return two ? start_tiles<T, RAGGED, false, 1, 2>(a, stream) : start_tiles<T, RAGGED, false, 1, 1>(a, stream);
  }
  if (two) glu ? start_tiles<T, RAGGED, true, 2, 2>(a, stream) : start_tiles<T, RAGGED, false, 2, 2>(a, stream);
  else glu ? start_tiles<T, RAGGED, true, 2, 1>(a, stream) : start_tiles<T, RAGGED, false, 2, 1>(a, stream);
}

}  // namespace tacg
