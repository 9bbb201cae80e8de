// Products in 8-bit integers with a scale for each token and for each weight row, for the experts of a GPU.
//
//   x[t][c] ~ sx[t] * qx[t][c],  W[n][c] ~ sw[n] * qw[n][c],  W[n] . x[t] ~ sw[n] * sx[t] * (sum over c of qw qx)
//
// with levels -127..127, half to even, of 127 x / max |x|.  The sum is exact in 32 bits: its magnitude is at most 65536 * 2^14 = 2^30.
//
// Weights lie in tiles of 16 rows x 64 columns (tacg_i8_pack), so that a wave's load of 1 KB is one operand of v_mfma_i32_16x16x64: lane n + 16 q
// supplies columns 16 q .. 16 q + 15 of row n, and of token n, and holds the sums of rows 4 q .. 4 q + 3 with token n.  Rows and tokens are
// padded to 64 columns with zeros, so no product has a bound.
//
// i8_prepare: levels of the tokens, a wave a row, kept in registers between the search for the largest and the rounding (8192 x 4096 in
//   bfloat16: 23 us, 4.4 TB/s, a part from the last-level cache; rows of more than 4096 columns are read twice: 8192 x 7168 53 us, 3.3 TB/s),
//   and in the same launch the pairs in the order of their matrices (Plan; 32768 pairs of 128 matrices: 10 us, latency of one reading;
//   bound by the longer of both).
// i8_few, i8_few_sum: few pairs, one launch.  One token through six gated matrices of 2816 x 2048: 8.8 us, 3.9 TB/s; through eight of 4096 x
//   1024, summed: 8.3 us; bound by latency: each wave has eight (sixteen) steps, behind the list of the pairs and the rounding.
// i8_stream: few pairs a matrix.  16 tokens, top-8, through 128 gated matrices of 1536 x 2048, of which they meet about 82: 46 us, 5.6 TB/s of
//   weights; bound by memory.
// i8_tiles: many.  64 tokens through those matrices: 74 us, 5.4 TB/s; bound by memory.  4096 x 4096 x 8192: 124 us, 2.2e15 operations/s
//   (torch's int8 product of 8192^3 reaches 2.1e15); 4096 tokens, top-8, through the 128 matrices: 150 us, 1.4e15.  The matrix cores are
//   busy half of the time; the caches give a CU 24 KB for each 64 columns of a tile, 11 TB/s in all (their first level is active 0.8 of the
//   time), and random levels draw so much power that the clock falls from 2.4 to 2.0 GHz (the same product of zeros: 119 us against 162, run
//   after run).
// i8_combine: sums over the slots of a token, in order; 8190 tokens of 4096 columns, one of eight GPUs: 55 us, 3.7 TB/s; bound by memory.
// i8_pack_kernel: 64 matrices of 2048 x 2048 in bfloat16 in 266 us, 3 TB/s; each row is read twice.
#include <algorithm>
#include <cmath>
#include <type_traits>
#include <utility>

#include "tacg_internal.h"

namespace tacg {
namespace {

typedef __attribute__((ext_vector_type(4))) int int4v;

constexpr int kTileRows = 16, kTileCols = 64, kTileBytes = kTileRows * kTileCols, kPiece = 16;

struct I8Args {
  const int8_t* x;          // levels
  const void* tokens;       // few pairs: x as the caller has it, and its strides in elements
  const float* x_scale;
  int64_t x_token, x_slot;  // strides of the levels, in bytes
  int64_t n_tokens;
  int32_t k, E, H, N, K, row_tiles, col_tiles, mode, out_dtype, slots;  // slots: whether every slot has its own x
  uint32_t over_k;          // the high half of pair * over_k is pair / k (0 for k = 1): pairs are below 2^27, k up to 16
  const int16_t* ids;       // or null: slot j takes matrix j
  const int32_t* slot;      // [E] or null
  const int8_t* w;
  const float* w_scale;
  const float* gate;        // [T][k] or null: 1
  float* part;              // [T][k][N]: the products of the pairs that are summed later, or null
  void* out;
  uint32_t* err;
};

__device__ __forceinline__ int token_index(const I8Args& a, int pair) {
  return a.over_k != 0 ? static_cast<int>(__umulhi(static_cast<uint32_t>(pair), a.over_k)) : pair;
}

constexpr int kBadId = -2, kBadTable = -3;

// Where the matrix of pair (t, j) lies: -1 for a slot that is served elsewhere, below for invalid entries.
__device__ __forceinline__ int place_of(const I8Args& a, int64_t pair, int j) {
  if (a.ids == nullptr) return j;
  const int e = a.ids[pair];
  if (e == -1) return -1;
  if (static_cast<uint32_t>(e) >= static_cast<uint32_t>(a.E)) return kBadId;
  const int h = a.slot != nullptr ? a.slot[e] : e;
  return h < 0 ? -1 : h < a.H ? h : kBadTable;
}

__device__ __forceinline__ void store(void* p, int64_t i, float v, int dtype) {
  if (dtype == TACG_F32) static_cast<float*>(p)[i] = v;
  else if (dtype == TACG_BF16) static_cast<__bf16*>(p)[i] = static_cast<__bf16>(v);
  else static_cast<_Float16*>(p)[i] = static_cast<_Float16>(v);
}

// Rounding to levels: 127 x / top, both brought to the range of top first.  127 x is exact for values of 16 bits, and the quotient is
// corrected to the nearest 32-bit number, which is exact where it lies half way between two levels.
struct Rounder {
  int exponent;
  float top, inverse;  // top in [0.5, 1)
  __device__ __forceinline__ explicit Rounder(float largest) {
    exponent = largest > 0.0f ? __builtin_amdgcn_frexp_expf(largest) : 0;
    top = largest > 0.0f ? ldexpf(largest, -exponent) : 1.0f;
    inverse = __builtin_amdgcn_rcpf(top);
  }
  // 1.5 * 2^23 + level: the level is the low byte
  __device__ __forceinline__ uint32_t operator()(float x) const {
    const float v = 127.0f * ldexpf(x, -exponent);
    float q = v * inverse;
    q = fmaf(fmaf(-q, top, v), inverse, q);
    return __float_as_uint(q + 12582912.0f);
  }
};

// A lane's values of a row: pieces of eight, 64 lanes after another.
constexpr int kChunk = 8, kWaveChunk = 64 * kChunk;

template <int DTYPE>
__device__ __forceinline__ void load_chunk(const void* x, int64_t first, int c, int K, float (&v)[kChunk]) {
  using T = std::conditional_t<DTYPE == TACG_F32, float, std::conditional_t<DTYPE == TACG_BF16, __bf16, _Float16>>;
  const T* p = static_cast<const T*>(x) + first + c;
  if (c + kChunk <= K) {
    T piece[kChunk];
    __builtin_memcpy(piece, p, sizeof(piece));  // rows need not start at multiples of 16 bytes
#pragma unroll
    for (int i = 0; i < kChunk; ++i) v[i] = static_cast<float>(piece[i]);
  } else {
#pragma unroll
    for (int i = 0; i < kChunk; ++i) v[i] = c + i < K ? static_cast<float>(p[i]) : 0.0f;
  }
}
__device__ __forceinline__ uint32_t largest(const float (&v)[kChunk], uint32_t m) {
#pragma unroll
  for (int i = 0; i < kChunk; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  return m;
}
__device__ __forceinline__ uint2 levels_of(const Rounder& level, const float (&v)[kChunk], bool bad) {
  uint32_t o[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t lo = __builtin_amdgcn_perm(level(v[4 * h + 1]), level(v[4 * h]), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(level(v[4 * h + 3]), level(v[4 * h + 2]), 0x04000c0cu);
    o[h] = bad ? 0u : lo | hi;
  }
  return make_uint2(o[0], o[1]);
}

struct TokenArgs {
  const void* x;
  int64_t stride_token, stride_slot, rows;
  int32_t K, Kp, k;    // k: rows of a token
  int8_t* q;
  float* scale;
  uint32_t* err;
};

// One row by one wave.  CH: pieces of a lane that stay in registers; 0: the row is read twice.
template <int DTYPE, int CH>
__device__ __forceinline__ void round_row(const TokenArgs& a, int64_t r, int lane) {
  const int64_t first = a.k == 1 ? r * a.stride_token : r / a.k * a.stride_token + r % a.k * a.stride_slot;
  uint32_t m = 0;  // magnitudes order as their bits, and what is not finite is above all others
  float v[CH ? CH : 1][kChunk];
  if constexpr (CH > 0) {
#pragma unroll
    for (int c = 0; c < CH; ++c) load_chunk<DTYPE>(a.x, first, c * kWaveChunk + lane * kChunk, a.K, v[c]);
#pragma unroll
    for (int c = 0; c < CH; ++c) m = largest(v[c], m);
  } else {
    for (int c = lane * kChunk; c < a.K; c += kWaveChunk) {
      load_chunk<DTYPE>(a.x, first, c, a.K, v[0]);
      m = largest(v[0], m);
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), o, 64)));
  const bool bad = m >= 0x7f800000u;
  const Rounder level(bad ? 0.0f : __uint_as_float(m));
  int8_t* q = a.q + r * a.Kp;
  if constexpr (CH > 0) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = c * kWaveChunk + lane * kChunk;
      if (at < a.Kp) *reinterpret_cast<uint2*>(q + at) = levels_of(level, v[c], bad);
    }
  } else {
    for (int at = lane * kChunk; at < a.Kp; at += kWaveChunk) {
      load_chunk<DTYPE>(a.x, first, at, a.K, v[0]);
      *reinterpret_cast<uint2*>(q + at) = levels_of(level, v[0], bad);
    }
  }
  if (lane == 0) {
    a.scale[r] = bad ? NAN : __uint_as_float(m) / 127.0f;
    if (bad) atomicOr(a.err, TACG_ERR_VALUE);
  }
}

struct PackArgs {
  const void* w;
  int64_t tiles;  // of 16 rows, of all matrices
  int32_t N, K, row_tiles, col_tiles;
  int8_t* q;
  float* scale;
  uint32_t* err;
};

// grid: tiles of 16 rows; 16 lanes a row.
template <int DTYPE>
__global__ __launch_bounds__(256) void i8_pack_kernel(PackArgs a) {
  const int tid = threadIdx.x, r = tid >> 4, sub = tid & 15;
  for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const int64_t h = tile / a.row_tiles;
    const int n = static_cast<int>(tile % a.row_tiles) * kTileRows + r;
    const bool in = n < a.N;
    const int64_t row = h * a.N + n;
    uint32_t m = 0;
    float v[kChunk] = {};
    if (in)
      for (int c = sub * kChunk; c < a.K; c += 16 * kChunk) {
        load_chunk<DTYPE>(a.w, row * a.K, c, a.K, v);
        m = largest(v, m);
      }
    for (int o = 8; o >= 1; o >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), o, 64)));
    const bool bad = m >= 0x7f800000u;
    const Rounder level(bad ? 0.0f : __uint_as_float(m));
    int8_t* out = a.q + tile * a.col_tiles * kTileBytes + r * kPiece;
    for (int c = sub * kChunk; c < a.col_tiles * kTileCols; c += 16 * kChunk) {
      if (in) load_chunk<DTYPE>(a.w, row * a.K, c, a.K, v);
      *reinterpret_cast<uint2*>(out + static_cast<int64_t>(c / kPiece) * kTileRows * kPiece + c % kPiece) = levels_of(level, v, bad || !in);
    }
    if (in && sub == 0) {
      a.scale[row] = bad ? NAN : __uint_as_float(m) / 127.0f;
      if (bad) atomicOr(a.err, TACG_ERR_VALUE);
    }
  }
}


// ---- the order of the pairs -------------------------------------------------------------------

// The pairs served here by their matrix: order[first[h] .. first[h + 1]) are those of matrix h.  The
// tiles of `tile` pairs of matrix h have the numbers first[h] / tile + h and following: no two matrices share one, and no matrix
// needs to know the others' tiles (with fewer pairs than matrices, first[h] and following).  tiles[i] = matrix and first pair of tile i, or -1, up to number(first[H], H).
struct Plan {
  int32_t* order;
  int32_t* first;     // [H + 1]
  int2* tiles;
  int32_t tile, n_tiles;
  int32_t sparse;     // fewer pairs than matrices
  int32_t by_rows;    // which units a die takes
  __host__ __device__ int number(int first, int h) const { return sparse ? first : first / tile + h; }
};

constexpr int kScan = 8, kBatch = 4, kSegment = 2;  // pairs of a load, loads of a batch, batches whose pairs are remembered

// One workgroup per matrix looks through all pairs: none waits for another, and no launch is
// needed to add up counts.  Up to 64 pairs a lane are read once, with a bit in LDS for each; more are read twice.
template <int THREADS>
__device__ void plan_block(const I8Args& a, const Plan& p, int h) {
  constexpr int kBatchPairs = THREADS * kScan * kBatch, kSegmentPairs = kBatchPairs * kSegment;
  __shared__ int place[TACG_MAX_EXPERTS];
  __shared__ int lower, equal, cursor;
  __shared__ uint32_t own[kSegment][THREADS];  // a lane reads what it wrote itself
  const int tid = threadIdx.x;
  const int pairs = static_cast<int>(a.n_tokens * a.k);
  if (tid == 0) lower = equal = cursor = 0;
  if (tid < a.E) {
    const int v = a.slot != nullptr ? a.slot[tid] : tid;
    place[tid] = v < 0 ? -1 : v < a.H ? v : kBadTable;
  }
  __syncthreads();
  uint32_t bad = 0;
  int below = 0;
  // the lane's pairs of a batch: base + i * 2048 + tid * 8 and the seven behind it, a bit each
  auto batch = [&](int base) {
    int4v id[kBatch];  // eight ids each
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int at = base + (i * THREADS + tid) * kScan;
      id[i] = int4v{-1, -1, -1, -1};
      if (at + kScan <= pairs) __builtin_memcpy(&id[i], a.ids + at, 16);
      else if (at < pairs)
#pragma unroll
        for (int e = 0; e < kScan; ++e)
          if (at + e < pairs) id[i][e / 2] = e % 2 ? (id[i][e / 2] & 0xffff) | (a.ids[at + e] << 16) : (id[i][e / 2] & ~0xffff) | (a.ids[at + e] & 0xffff);
    }
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int at = base + (i * THREADS + tid) * kScan;
#pragma unroll
      for (int e = 0; e < kScan; ++e) {
        const int id16 = e % 2 ? id[i][e / 2] >> 16 : static_cast<int16_t>(id[i][e / 2]);
        const bool in = static_cast<uint32_t>(id16) < static_cast<uint32_t>(a.E);
        int v = place[in ? id16 : 0];
        if (!in) v = id16 == -1 ? -1 : kBadId;
        bad |= v == kBadId ? TACG_ERR_ID_RANGE : v == kBadTable ? TACG_ERR_TABLE : 0u;
        below += v >= 0 && v < h;
        mine |= static_cast<uint32_t>(v == h) << (i * kScan + e);  // pairs past the last have the id -1
      }
    }
    return mine;
  };
  int count = 0;
  for (int base = 0; base < pairs; base += kBatchPairs) {
    const uint32_t m = batch(base);
    own[base / kBatchPairs % kSegment][tid] = m;
    count += __popc(m);
  }
  const int mine = count;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    below += __shfl_xor(below, o, 64);
    count += __shfl_xor(count, o, 64);
  }
  if ((tid & 63) == 0) {
    atomicAdd(&lower, below);
    atomicAdd(&equal, count);
  }
  if (h == 0 && bad != 0) atomicOr(a.err, bad);
  barrier_after_lds_atomics();
  const int from = lower;
  count = equal;
  int at = from + (mine > 0 ? atomicAdd(&cursor, mine) : 0);  // the order of a matrix' pairs does not matter to any result
  for (int base = 0; base < pairs && count > 0; base += kBatchPairs) {
    for (uint32_t m = pairs > kSegmentPairs ? batch(base) : own[base / kBatchPairs][tid]; m != 0; m &= m - 1) {
      const int bit = __ffs(m) - 1;
      p.order[at++] = base + (bit / kScan * THREADS + tid) * kScan + bit % kScan;
    }
  }
  const int begin = p.number(from, h);
  const int end = h < a.H ? p.number(from + count, h + 1) : begin;  // without any matrix there are no tiles
  for (int i = begin + tid; i < end; i += THREADS) {
    const int start = from + (i - begin) * p.tile;
    p.tiles[i] = start < from + count ? make_int2(h, start) : make_int2(-1, 0);
  }
  if (tid == 0) {
    p.first[h] = from;
    if (h == a.H - 1) p.first[a.H] = from + count;
  }
}

// grid: n_plan workgroups for the order of the pairs, then workgroups whose waves take a row of tokens each, or (skip > 0, rows are pairs)
// those of `skip` rows that are served here.
template <int DTYPE, int CH, int THREADS>
__global__ __launch_bounds__(THREADS) void i8_prepare(TokenArgs t, I8Args a, Plan p, int n_plan, int skip) {
  if (static_cast<int>(blockIdx.x) < n_plan) {
    plan_block<THREADS>(a, p, blockIdx.x);
    return;
  }
  const int lane = threadIdx.x & 63;
  const int64_t step = static_cast<int64_t>(gridDim.x - n_plan) * (THREADS / 64);
  const int64_t own = static_cast<int64_t>(blockIdx.x - n_plan) * (THREADS / 64) + (threadIdx.x >> 6);
  if (skip == 0) {
    for (int64_t r = own; r < t.rows; r += step) round_row<DTYPE, CH>(t, r, lane);
    return;
  }
  for (int64_t base = own * skip; base < t.rows; base += step * skip) {
    uint64_t served = __ballot(lane < skip && base + lane < t.rows && place_of(a, min(base + lane, t.rows - 1), 0) >= 0);
    for (; served != 0; served &= served - 1) round_row<DTYPE, CH>(t, base + __ffsll(static_cast<unsigned long long>(served)) - 1, lane);
  }
}

// ---- products ----------------------------------------------------------------------------------

constexpr int kManyTile = 128, kFewTile = 32;  // pairs of a tile

constexpr int kWaves = 4;
// A block of 16 tokens in LDS: 16 bytes of each after another, for each quarter of the 64 columns.  Quarters are 18 * 16 bytes apart and the
// steps 16 more, as lanes that write different quarters of a token would meet the same banks: conflicts of a product of 4096 x 4096 x 8192
// 3.3e4 cycles a CU of 2.5e5 (20 * 16 and 32: 4.9e4), which is not what bounds it.
constexpr int kPieceBytes = 18 * 16, kBlockBytes = 4 * kPieceBytes;

// What a lane does of its part of a tile's results: 4 consecutive rows of a token.
__device__ __forceinline__ void put(const I8Args& a, int64_t row, int n, int width, const float (&y)[4], void* out, int dtype) {
  const int64_t at = row * width + n;
  if (n + 4 <= width && width % 4 == 0) {
    if (dtype == TACG_F32) {
      float4 v = make_float4(y[0], y[1], y[2], y[3]);
      __builtin_memcpy(static_cast<float*>(out) + at, &v, 16);
    } else if (dtype == TACG_BF16) {
      __bf16 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = static_cast<__bf16>(y[i]);
      __builtin_memcpy(static_cast<__bf16*>(out) + at, v, 8);
    } else {
      _Float16 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = static_cast<_Float16>(y[i]);
      __builtin_memcpy(static_cast<_Float16*>(out) + at, v, 8);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < width) store(out, at + i, y[i], dtype);
  }
}

struct Unit {
  int h, first, count;  // matrix, its tile's first pair in the order and number of pairs
  int n0;               // first output column
};

__device__ __forceinline__ int pair_of(const I8Args& a, const Plan& p, const Unit& u, int i) {
  return a.ids == nullptr ? (u.first + i) * a.k + u.h : p.order[u.first + i];
}

// Where a lane's piece of a block of 16 weight rows lies in its matrix: its row's 16 bytes of the tile's first 64 columns.  Gated: RF / 2
// blocks of gate rows and the same rows of the other kind after each.
template <int RF>
__device__ __forceinline__ void weight_rows(const I8Args& a, int n0, bool glu, int width, uint32_t (&at)[RF]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < RF; ++i) {
    int row = min(n0 + (glu ? i / 2 : i) * kTileRows, width - 1) + (lane & 15) + (glu && (i & 1) ? width : 0);
    row = min(row, a.row_tiles * kTileRows - 1);
    at[i] = static_cast<uint32_t>(row / kTileRows) * a.col_tiles * kTileBytes + (lane >> 4) * 256 + row % kTileRows * kPiece;
  }
}

__device__ __forceinline__ const char* matrix_of(const I8Args& a, int h) {
  return reinterpret_cast<const char*>(a.w) + static_cast<int64_t>(h) * a.row_tiles * a.col_tiles * kTileBytes;
}
__device__ __forceinline__ const int8_t* token_of(const I8Args& a, int pair) {
  const int t = token_index(a, pair);
  return a.x + t * a.x_token + (pair - t * a.k) * a.x_slot;
}
__device__ __forceinline__ int4v load16(const void* p) { return *static_cast<const int4v*>(p); }
__device__ __forceinline__ int4v load_once(const void* p) { return __builtin_nontemporal_load(static_cast<const int4v*>(p)); }

// f(integral_constant 0), f(1), ... f(N - 1): what a loop of so many steps is not unrolled to.
template <class F, int... I>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>()), ...);
}

// Results of a wave: lane n + 16 q holds rows 4 q .. 4 q + 3 of a block for token n.
// pair_at(i): the pair of the tile's token i; scale_at(i, pair): the scale of its levels.
template <int RF, int JT, class Pair, class Scale>
__device__ __forceinline__ void finish(const I8Args& a, const Unit& u, int n0, const int4v (&acc)[RF][JT], Pair pair_at, Scale scale_at) {
  const int lane = threadIdx.x & 63;
  const bool glu = a.mode == TACG_Q4_GLU;
  const int width = glu ? a.N / 2 : a.N;
  const float* sw = a.w_scale + static_cast<int64_t>(u.h) * a.N;
  float scale[RF][4];
#pragma unroll
  for (int i = 0; i < RF; ++i) {
    const int n = n0 + (glu ? i / 2 : i) * kTileRows + (lane >> 4) * 4;
    const float* from = sw + (glu && (i & 1) ? width : 0);
    if (n + 4 <= width) __builtin_memcpy(scale[i], from + n, 16);
    else
#pragma unroll
      for (int r = 0; r < 4; ++r) scale[i][r] = from[min(n + r, width - 1)];
  }
  const bool part = a.mode == TACG_Q4_SUM && a.part != nullptr;
  void* out = part ? a.part : a.out;
  const int dtype = part ? TACG_F32 : a.out_dtype;
  each_of(std::make_integer_sequence<int, JT>(), [&](auto block) {
    constexpr int j = decltype(block)::value;
    const int i0 = j * 16 + (lane & 15);
    if (i0 >= u.count) return;
    const int pair = pair_at(i0);
    const float sx = scale_at(i0, pair);
    const float gate = a.mode == TACG_Q4_SUM && !part && a.gate != nullptr ? a.gate[pair] : 1.0f;
    if (glu) {
      if constexpr (RF > 1) {
#pragma unroll
        for (int i = 0; i < RF / 2; ++i) {
          const int n = n0 + i * kTileRows + (lane >> 4) * 4;
          float y[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float g = static_cast<float>(acc[2 * i][j][r]) * (sx * scale[2 * i][r]);
            const float v = static_cast<float>(acc[2 * i + 1][j][r]) * (sx * scale[2 * i + 1][r]);
            y[r] = g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * v;  // the reciprocal is within one unit in the last place
          }
          if (n < width) put(a, pair, n, width, y, out, dtype);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < RF; ++i) {
        const int n = n0 + i * kTileRows + (lane >> 4) * 4;
        float y[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] = static_cast<float>(acc[i][j][r]) * (sx * scale[i][r]) * gate;
        if (n < width) put(a, pair, n, width, y, out, dtype);
      }
    }
  });
}

template <int RF, int JT>
__device__ __forceinline__ void finish(const I8Args& a, const Plan& p, const Unit& u, int n0, const int4v (&acc)[RF][JT]) {
  finish(a, u, n0, acc, [&](int i) { return pair_of(a, p, u, i); },
         [&](int, int pair) { return a.x_scale[a.slots ? pair : token_index(a, pair)]; });
}

// Many tokens: a wave has 64 weight rows and all tokens of the tile, JT blocks of 16.  Weights go from memory to the registers of the wave that
// needs them, three steps of 64 columns ahead.  Tokens go through LDS, whole lines of 128 bytes for two steps at a time, and from
// there two blocks ahead.
template <int JT>
__device__ __forceinline__ void tile_product(const I8Args& a, const Plan& p, const Unit& u, char* lds) {
  constexpr int RF = 4, AHEAD = 2, kLoads = JT / 2;  // loads of a wave for two steps: eight tokens each
  constexpr int kHalf = JT * kBlockBytes + 16;       // LDS of a step
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool glu = a.mode == TACG_Q4_GLU;
  const int width = glu ? a.N / 2 : a.N;
  const int n0 = u.n0 + wave * (glu ? RF / 2 : RF) * kTileRows;
  const char* w = matrix_of(a, u.h);
  uint32_t at[RF];
  weight_rows<RF>(a, n0, glu, width, at);
  uint32_t token[kLoads];  // in pieces of 16 bytes
#pragma unroll
  for (int i = 0; i < kLoads; ++i)
    token[i] = static_cast<uint32_t>((token_of(a, pair_of(a, p, u, min((wave + i * kWaves) * 8 + (lane >> 3), u.count - 1))) - a.x) / kPiece);
  int4v acc[RF][JT];
#pragma unroll
  for (int i = 0; i < RF; ++i)
#pragma unroll
    for (int j = 0; j < JT; ++j) acc[i][j] = int4v{0, 0, 0, 0};
  const int last = a.col_tiles - 1;
  auto load_weights = [&](int c, int4v (&v)[RF]) {
    const uint32_t from = static_cast<uint32_t>(min(c, last)) * kTileBytes;
#pragma unroll
    for (int i = 0; i < RF; ++i) v[i] = load16(w + (at[i] + from));
  };
  int4v tk[kLoads];
  auto load_tokens = [&](int c) {  // for steps c and c + 1; past the last column its own bytes again
    const int from = min(c * kTileCols + (lane & 7) * kPiece, last * kTileCols + (lane & 3) * kPiece);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) tk[i] = load16(a.x + static_cast<uint64_t>(token[i]) * kPiece + from);
  };
  auto keep_tokens = [&](int c) {
    char* to = lds + ((c >> 1) & 1) * (2 * kHalf) + ((lane >> 2) & 1) * kHalf + (lane & 3) * kPieceBytes;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = (wave + i * kWaves) * 8 + (lane >> 3);
      *reinterpret_cast<int4v*>(to + (row >> 4) * kBlockBytes + (row & 15) * 16) = tk[i];
    }
  };
  int4v w0[RF], w1[RF], w2[RF], w3[RF];
  load_tokens(0);
  load_weights(0, w0);
  load_weights(1, w1);
  load_weights(2, w2);
  keep_tokens(0);
  auto multiply = [&](int c, const int4v (&now)[RF]) {
    const char* from = lds + ((c >> 1) & 1) * (2 * kHalf) + (c & 1) * kHalf + (lane >> 4) * kPieceBytes + (lane & 15) * 16;
    int4v t[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) t[j] = load16(from + j * kBlockBytes);
#pragma unroll
    for (int j = 0; j < JT; ++j) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < RF; ++i) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(now[i], t[j % AHEAD], acc[i][j], 0, 0, 0);
      if (j + AHEAD < JT) t[j % AHEAD] = load16(from + (j + AHEAD) * kBlockBytes);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // two steps: `first` holds the weights of the earlier one and takes those of step c + 4, `third` those of c + 3
  auto pair_of_steps = [&](int c, int4v (&first)[RF], const int4v (&second)[RF], int4v (&third)[RF]) {
    __syncthreads();
    load_tokens(c + 2);
    load_weights(c + 3, third);
    if (c <= last) multiply(c, first);
    load_weights(c + 4, first);
    if (c + 1 <= last) multiply(c + 1, second);
    keep_tokens(c + 2);
  };
  for (int c = 0; c <= last; c += 4) {
    pair_of_steps(c, w0, w1, w3);
    pair_of_steps(c + 2, w2, w3, w1);
  }
  finish<RF, JT>(a, p, u, n0, acc);
}

// Few tokens: the time is that of the weights' loads.  A wave has RF blocks of 16 weight rows; weights and tokens go straight to its
// registers, DEPTH steps of 64 columns ahead, without a barrier.  SPLIT: the four waves have the same rows and a quarter of the
// columns each, and add their (exact) sums up in LDS.
template <int RF, int JT, bool SPLIT>
__device__ __forceinline__ void stream_product(const I8Args& a, const Plan& p, const Unit& u, int4v* lds) {
  constexpr int DEPTH = 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool glu = a.mode == TACG_Q4_GLU;
  const int width = glu ? a.N / 2 : a.N;
  const int n0 = u.n0 + (SPLIT ? 0 : wave * (glu ? RF / 2 : RF) * kTileRows);
  const char* w = matrix_of(a, u.h);
  uint32_t at[RF];
  weight_rows<RF>(a, n0, glu, width, at);
  const int8_t* token[JT];
#pragma unroll
  for (int j = 0; j < JT; ++j) token[j] = token_of(a, pair_of(a, p, u, min(j * 16 + (lane & 15), u.count - 1))) + (lane >> 4) * kPiece;
  int4v acc[RF][JT];
#pragma unroll
  for (int i = 0; i < RF; ++i)
#pragma unroll
    for (int j = 0; j < JT; ++j) acc[i][j] = int4v{0, 0, 0, 0};
  const int begin = SPLIT ? a.col_tiles * wave / kWaves : 0, end = SPLIT ? a.col_tiles * (wave + 1) / kWaves : a.col_tiles;
  int4v v[DEPTH][RF], t[DEPTH][JT];
  auto load = [&](int c, int d) {
    const uint32_t from = static_cast<uint32_t>(c) * kTileBytes;
#pragma unroll
    for (int i = 0; i < RF; ++i) v[d][i] = load16(w + (at[i] + from));
#pragma unroll
    for (int j = 0; j < JT; ++j) t[d][j] = load16(token[j] + c * kTileCols);
  };
  auto multiply = [&](int d) {
#pragma unroll
    for (int j = 0; j < JT; ++j)
#pragma unroll
      for (int i = 0; i < RF; ++i) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[d][i], t[d][j], acc[i][j], 0, 0, 0);
  };
  const int last = max(end - 1, 0);
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) load(min(begin + d, last), d);
  int c = begin;
  for (; c + 2 * DEPTH <= end; c += DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      multiply(d);
      load(c + d + DEPTH, d);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // the last ones: DEPTH or more, unless there are fewer in all
#pragma unroll
  for (int d = 0; d < DEPTH; ++d)
    if (c + d < end) {
      multiply(d);
      if (c + d + DEPTH < end) load(c + d + DEPTH, d);
    }
  c += DEPTH;
#pragma unroll
  for (int d = 0; d < DEPTH; ++d)
    if (c + d < end) multiply(d);
  if constexpr (SPLIT) {
    if (wave > 0) {
#pragma unroll
      for (int i = 0; i < RF; ++i)
#pragma unroll
        for (int j = 0; j < JT; ++j) lds[((wave - 1) * RF * JT + i * JT + j) * 64 + lane] = acc[i][j];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int o = 0; o < kWaves - 1; ++o)
#pragma unroll
      for (int i = 0; i < RF; ++i)
#pragma unroll
        for (int j = 0; j < JT; ++j) acc[i][j] += lds[(o * RF * JT + i * JT + j) * 64 + lane];
  }
  finish<RF, JT>(a, p, u, n0, acc);
}

// What is served elsewhere is 0.  A wave takes 64 pairs at a time.
__device__ __forceinline__ void clear_block(const I8Args& a, int block, int blocks) {
  const int width = a.mode == TACG_Q4_GLU ? a.N / 2 : a.N, size = a.out_dtype == TACG_F32 ? 4 : 2;
  const int64_t bytes = static_cast<int64_t>(width) * size;
  const int lane = threadIdx.x & 63, pairs = static_cast<int>(a.n_tokens) * a.k;
  for (int base = (block * kWaves + (threadIdx.x >> 6)) * 64; base < pairs; base += blocks * kWaves * 64) {
    uint64_t away = __ballot(base + lane < pairs && place_of(a, min(base + lane, pairs - 1), 0) < 0);
    for (; away != 0; away &= away - 1) {
      char* row = static_cast<char*>(a.out) + (base + __ffsll(static_cast<unsigned long long>(away)) - 1) * bytes;
      const int64_t head = min(bytes, static_cast<int64_t>(-reinterpret_cast<uintptr_t>(row) & 15)), body = (bytes - head) / 16;
      if (lane < head / 2) reinterpret_cast<int16_t*>(row)[lane] = 0;
      for (int64_t c = lane; c < body; c += 64) reinterpret_cast<int4*>(row + head)[c] = make_int4(0, 0, 0, 0);
      const int64_t done = head + body * 16;
      if (lane < (bytes - done) / 2) reinterpret_cast<int16_t*>(row + done)[lane] = 0;
    }
  }
}

// The unit of a workgroup: a tile of pairs and a block of `rows` output columns.  Workgroups go to the eight dies in turn, and what a die reads
// twice should come from its own cache.  A run of units for each die, all blocks of a tile after another; or (by_rows, where a matrix has
// more tiles than one and the blocks are a multiple of eight, of 16 at least) the same blocks of all tiles to the same die, which also gives the
// dies the same work: 8190 pairs of 32 matrices of 4096 x 2048 137 us from 147.
__device__ __forceinline__ bool unit_of(const I8Args& a, const Plan& p, int blocks, int rows, int clear, Unit& u) {
  // tiles that there are: those of pairs served here
  const int total = (a.ids == nullptr ? p.n_tiles : p.number(__builtin_amdgcn_readfirstlane(p.first[a.H]), a.H)) * blocks;
  int w = blockIdx.x;
  if (w >= total) {
    const int all = p.n_tiles * blocks;
    if (w >= all) clear_block(a, w - all, clear);
    return false;
  }
  const int share = total / 8;
  if (!p.by_rows && w < share * 8) w = (w & 7) * share + (w >> 3);
  const int tile = w / blocks;
  u.n0 = (w - tile * blocks) * rows;
  if (a.ids == nullptr) {
    const int per = (static_cast<int>(a.n_tokens) + p.tile - 1) / p.tile;
    u.h = tile / per;
    u.first = (tile - u.h * per) * p.tile;
    u.count = static_cast<int>(a.n_tokens) - u.first;
  } else {
    const int2 t = p.tiles[tile];
    u.h = __builtin_amdgcn_readfirstlane(t.x);
    u.first = __builtin_amdgcn_readfirstlane(t.y);
    if (u.h < 0) return false;
    u.count = __builtin_amdgcn_readfirstlane(p.first[u.h + 1]) - u.first;
  }
  u.count = min(u.count, p.tile);
  return true;
}

// grid: tiles of pairs x blocks of output columns, then `clear` workgroups.
__global__ __launch_bounds__(256, 2) void i8_tiles(I8Args a, Plan p, int blocks, int rows, int clear) {
  __shared__ alignas(16) char lds[4 * (kManyTile / 16 * kBlockBytes + 16)];
  Unit u;
  if (!unit_of(a, p, blocks, rows, clear, u)) return;
  const int jt = (u.count + 15) / 16;
  if (jt > 6) tile_product<8>(a, p, u, lds);
  else if (jt > 4) tile_product<6>(a, p, u, lds);
  else if (jt > 2) tile_product<4>(a, p, u, lds);
  else tile_product<2>(a, p, u, lds);
}

template <int RF, bool SPLIT>
__global__ __launch_bounds__(256, 2) void i8_stream(I8Args a, Plan p, int blocks, int rows, int clear) {
  __shared__ int4v lds[SPLIT ? (kWaves - 1) * RF * 2 * 64 : 1];
  Unit u;
  if (!unit_of(a, p, blocks, rows, clear, u)) return;
  if (u.count > 16) stream_product<RF, 2, SPLIT>(a, p, u, lds);
  else stream_product<RF, 1, SPLIT>(a, p, u, lds);
}

// ---- few pairs: one launch ---------------------------------------------------------------------
//
// Every workgroup looks at all pairs (up to 64, a lane each) and rounds the tokens that it needs by itself, into LDS: no launch before it.

constexpr int kFewPairs = 64;

// A row of x, in the caller's type, as levels in LDS (col_tiles * 64 bytes) by LANES lanes of which this is number i; 256: the workgroup.
// The scale comes back.
template <int DTYPE, int LANES>
__device__ __forceinline__ float round_to_lds(const I8Args& a, int64_t first, int64_t scale_at, char* to, uint32_t* most, int i, bool report) {
  const int width = a.col_tiles * kTileCols;
  if constexpr (DTYPE == TACG_I8) {
    for (int c = i * 16; c < width; c += LANES * 16) *reinterpret_cast<int4v*>(to + c) = load16(static_cast<const int8_t*>(a.tokens) + first + c);
    return a.x_scale[scale_at];
  } else {
    constexpr int kStep = LANES * kChunk;
    float kept[2][kChunk], v[kChunk];
    uint32_t m = 0;
#pragma unroll
    for (int s = 0; s < 2; ++s) load_chunk<DTYPE>(a.tokens, first, s * kStep + i * kChunk, a.K, kept[s]);
#pragma unroll
    for (int s = 0; s < 2; ++s) m = largest(kept[s], m);
    for (int c = 2 * kStep + i * kChunk; c < a.K; c += kStep) {
      load_chunk<DTYPE>(a.tokens, first, c, a.K, v);
      m = largest(v, m);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), o, 64)));
    if constexpr (LANES > 64) {
      if ((i & 63) == 0) most[i >> 6] = m;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < LANES / 64; ++w) m = max(m, most[w]);
      __syncthreads();
    }
    const bool bad = m >= 0x7f800000u;
    const Rounder level(bad ? 0.0f : __uint_as_float(m));
#pragma unroll
    for (int s = 0; s < 2; ++s)
      if (s * kStep + i * kChunk < width) *reinterpret_cast<uint2*>(to + s * kStep + i * kChunk) = levels_of(level, kept[s], bad);
    for (int c = 2 * kStep + i * kChunk; c < width; c += kStep) {
      load_chunk<DTYPE>(a.tokens, first, c, a.K, v);
      *reinterpret_cast<uint2*>(to + c) = levels_of(level, v, bad);
    }
    if (bad && report && i == 0) atomicOr(a.err, TACG_ERR_VALUE);
    return bad ? NAN : __uint_as_float(m) / 127.0f;
  }
}

// The lane's pair, of up to 64: where its matrix lies.  The first workgroup along the rows reports what is invalid.
__device__ __forceinline__ int lane_place(const I8Args& a, bool report) {
  const int lane = threadIdx.x & 63, pairs = static_cast<int>(a.n_tokens) * a.k;
  int h = -1;
  if (lane < pairs) h = place_of(a, lane, lane - token_index(a, lane) * a.k);
  if (report && threadIdx.x < 64 && h < -1) atomicOr(a.err, h == kBadId ? TACG_ERR_ID_RANGE : TACG_ERR_TABLE);
  return h;
}

// Each and gated products: grid (blocks of 32 weight rows, pairs).  The workgroup of the first pair of a matrix takes all its pairs, 16 at a
// time; its four waves have a quarter of the columns each.  lds: rows of levels, `stride` bytes apart, as many as 16 pairs of a matrix can
// have: one for each of up to 16 pairs, or, with one x for all slots, for each of up to 16 tokens (few_of).
template <int DTYPE>
__global__ __launch_bounds__(256, 2) void i8_few(I8Args a, int rows, int stride) {
  constexpr int RF = 2, DEPTH = 4;
  extern __shared__ int4v levels_lds[];
  char* levels = reinterpret_cast<char*>(levels_lds);
  __shared__ int4v sums[(kWaves - 1) * RF * 64];
  __shared__ int list[kFewPairs];
  __shared__ float scales[kFewPairs];
  __shared__ uint32_t most[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool glu = a.mode == TACG_Q4_GLU;
  const int width = glu ? a.N / 2 : a.N;
  const int place = lane_place(a, blockIdx.x == 0 && blockIdx.y == 0);
  Unit u;
  u.n0 = blockIdx.x * rows;
  u.h = __builtin_amdgcn_readlane(place, blockIdx.y);
  u.first = 0;
  if (u.h < 0) {
    for (int n = u.n0 + tid; n < min(u.n0 + rows, width); n += 256) store(a.out, static_cast<int64_t>(blockIdx.y) * width + n, 0.0f, a.out_dtype);
    return;
  }
  const uint64_t same = __ballot(place == u.h);
  if ((same & ((uint64_t(1) << blockIdx.y) - 1)) != 0) return;
  u.count = __popcll(same);
  if (place == u.h && wave == 0) list[__popcll(same & ((uint64_t(1) << lane) - 1))] = lane;
  const char* w = matrix_of(a, u.h);
  uint32_t at[RF];
  weight_rows<RF>(a, u.n0, glu, width, at);
  const int begin = a.col_tiles * wave / kWaves, end = a.col_tiles * (wave + 1) / kWaves, last = max(end - 1, 0);
  int4v v[DEPTH][RF];
  auto load = [&](int c, int d) {
#pragma unroll
    for (int i = 0; i < RF; ++i) v[d][i] = load16(w + (at[i] + static_cast<uint32_t>(c) * kTileBytes));
  };
#pragma unroll
  for (int d = 0; d < DEPTH; ++d) load(min(begin + d, last), d);  // before the tokens are there
  __syncthreads();
  // 16 tokens at a time
  for (int first = 0; first < u.count; first += 16) {
    const int n = min(u.count - first, 16);
    // a row of levels for each slot's x, or for each token: its pairs (an expert that it has twice, two experts with one matrix) are neighbours
    uint32_t starts = 0;  // bit r: pair r is the first of a row
    float s = 0.0f;
    for (int r = 0, before = -1; r < n; ++r) {
      const int pair = __builtin_amdgcn_readfirstlane(list[first + r]), t = token_index(a, pair);
      if (a.slots || t != before) {
        s = round_to_lds<DTYPE, 256>(a, t * a.x_token + (pair - t * a.k) * a.x_slot, a.slots ? pair : t, levels + __popc(starts) * stride, most,
                                     tid, blockIdx.x == 0);
        starts |= 1u << r;
        before = t;
      }
      if (tid == 0) scales[r] = s;
    }
    __syncthreads();
    const char* token = levels + (__popc(starts & ((2u << min(lane & 15, n - 1)) - 1)) - 1) * stride + (lane >> 4) * kPiece;
    int4v acc[RF][1] = {};
    auto multiply = [&](int c, int d) {
      const int4v t = load16(token + c * kTileCols);
#pragma unroll
      for (int i = 0; i < RF; ++i) acc[i][0] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[d][i], t, acc[i][0], 0, 0, 0);
    };
    if (first > 0) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) load(min(begin + d, last), d);
    }
    int c = begin;
    for (; c + 2 * DEPTH <= end; c += DEPTH) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        multiply(c + d, d);
        load(c + d + DEPTH, d);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (c + d < end) {
        multiply(c + d, d);
        if (c + d + DEPTH < end) load(c + d + DEPTH, d);
      }
    c += DEPTH;
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (c + d < end) multiply(c + d, d);
    if (wave > 0) {
#pragma unroll
      for (int i = 0; i < RF; ++i) sums[((wave - 1) * RF + i) * 64 + lane] = acc[i][0];
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int o = 0; o < kWaves - 1; ++o)
#pragma unroll
        for (int i = 0; i < RF; ++i) acc[i][0] += sums[(o * RF + i) * 64 + lane];
      Unit part = u;
      part.count = n;
      finish(a, part, u.n0, acc, [&](int i) { return list[first + i]; }, [&](int i, int) { return scales[i]; });
    }
    __syncthreads();
  }
}

// Sums over a token's experts: grid (blocks of 16 weight rows, tokens), eight waves.  A wave rounds the x of one slot after another; then the
// steps of all served slots are shared evenly, and a slot's (exact) sums meet in LDS.
template <int DTYPE>
__global__ __launch_bounds__(512, 2) void i8_few_sum(I8Args a, int stride) {
  constexpr int DEPTH = 8, kAll = 8;
  extern __shared__ int4v levels_lds[];
  char* levels = reinterpret_cast<char*>(levels_lds);
  __shared__ int sums[TACG_MAX_TOPK][kTileRows];
  __shared__ float scales[TACG_MAX_TOPK];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int place = lane_place(a, blockIdx.x == 0 && blockIdx.y == 0);
  const int t0 = blockIdx.y * a.k, n0 = blockIdx.x * kTileRows;
  const uint64_t served = (__ballot(place >= 0) >> t0) & ((uint64_t(1) << a.k) - 1);
  for (int i = tid; i < TACG_MAX_TOPK * kTileRows; i += 512) sums[i / kTileRows][i % kTileRows] = 0;
  // the wave's steps, and the weights of the first of them, which come while the tokens are rounded
  const int slots = __popcll(served), all = slots * a.col_tiles, begin = all * wave / kAll, end = all * (wave + 1) / kAll;
  const int row = min(n0 + (lane & 15), a.row_tiles * kTileRows - 1);
  const uint32_t at = static_cast<uint32_t>(row / kTileRows) * a.col_tiles * kTileBytes + (lane >> 4) * 256 + row % kTileRows * kPiece;
  uint64_t left = served;
  int slot = 0, stop = 0;
  const char* w = nullptr;
  int4v v[DEPTH];
  auto load = [&](int c) {
    if (c >= stop) {  // the matrix of another slot
      while (c >= (slot + 1) * a.col_tiles) left &= left - 1, ++slot;
      w = matrix_of(a, __builtin_amdgcn_readlane(place, t0 + __ffsll(static_cast<unsigned long long>(left)) - 1));
      stop = min(end, (slot + 1) * a.col_tiles);
    }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)  // read once: not kept in the caches (8.3 us against 9.5 at one token and eight matrices of 4096 x 1024)
      v[d] = load_once(w + (at + static_cast<uint32_t>(min(c + d, stop - 1) - slot * a.col_tiles) * kTileBytes));
  };
  if (begin < end) load(begin);
  int s0 = 0;
  for (uint64_t m = served; m != 0; m &= m - 1, ++s0) {
    const int j = __ffsll(static_cast<unsigned long long>(m)) - 1;
    if ((!a.slots && s0 > 0) || s0 % kAll != wave) continue;  // one x for all slots, or one each
    const float s = round_to_lds<DTYPE, 64>(a, blockIdx.y * a.x_token + j * a.x_slot, a.slots ? t0 + j : blockIdx.y, levels + s0 * stride,
                                            nullptr, lane, blockIdx.x == 0);
    if (lane == 0) scales[s0] = s;
  }
  __syncthreads();
  int4v acc = {0, 0, 0, 0};
  for (int c = begin; c < end;) {
    const char* token = levels + (a.slots ? slot : 0) * stride + (lane >> 4) * kPiece - slot * a.col_tiles * kTileCols;
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
      if (c + d < stop) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[d], load16(token + (c + d) * kTileCols), acc, 0, 0, 0);
    c = min(c + DEPTH, stop);
    if (c == stop) {
      if ((lane & 15) == 0) {
#pragma unroll
        for (int r = 0; r < 4; ++r) atomicAdd(&sums[slot][(lane >> 4) * 4 + r], acc[r]);
      }
      acc = int4v{0, 0, 0, 0};
    }
    if (c < end) load(c);
  }
  barrier_after_lds_atomics();
  const int n = n0 + tid;
  if (tid >= kTileRows || n >= a.N) return;
  float y = 0.0f;
  int s = 0;
  for (uint64_t m = served; m != 0; m &= m - 1, ++s) {
    const int j = __ffsll(static_cast<unsigned long long>(m)) - 1, h = __builtin_amdgcn_readlane(place, t0 + j);
    const float v = static_cast<float>(sums[s][tid]) * (scales[a.slots ? s : 0] * a.w_scale[static_cast<int64_t>(h) * a.N + n]);
    y += (a.gate != nullptr ? a.gate[t0 + j] : 1.0f) * v;
  }
  store(a.out, static_cast<int64_t>(blockIdx.y) * a.N + n, y, a.out_dtype);
}

// Sums over the slots of a token, in order.  grid: (blocks of 1024 output columns, tokens).
__global__ __launch_bounds__(256) void i8_combine(I8Args a) {
  const int n = (blockIdx.x * 256 + threadIdx.x) * 4, lane = threadIdx.x & 63;
  for (int64_t t = blockIdx.y; t < a.n_tokens; t += gridDim.y) {
    // a lane per slot: which are served here, and their gates
    const int64_t own = t * a.k + min(lane, a.k - 1);
    const float gate = a.gate != nullptr ? a.gate[own] : 1.0f;
    uint64_t served = __ballot(lane < a.k && place_of(a, own, lane) >= 0);
    float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    while (served != 0) {
      const int j = __ffsll(static_cast<unsigned long long>(served)) - 1;
      served &= served - 1;
      const float g = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(gate), j));
      const float* v = a.part + (t * a.k + j) * a.N + n;
      float f[4];
      if (n + 4 <= a.N) __builtin_memcpy(f, v, 16);
      else
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = n + i < a.N ? v[i] : 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] += g * f[i];
    }
    if (n < a.N) put(a, t, n, a.N, y, a.out, a.out_dtype);
  }
}

template <int DTYPE, int THREADS>
void start_prepare(const TokenArgs& t, const I8Args& a, const Plan& p, int n_plan, int skip, hipStream_t stream) {
  constexpr int kRows = THREADS / 64;
  const int per = std::max(skip, 1);
  const dim3 grid(static_cast<uint32_t>(n_plan + std::min<int64_t>((t.rows + kRows * per - 1) / (kRows * per), 1 << 20)));
  auto* kernel = t.K <= kWaveChunk       ? i8_prepare<DTYPE, 1, THREADS>
                 : t.K <= 2 * kWaveChunk ? i8_prepare<DTYPE, 2, THREADS>
                 : t.K <= 4 * kWaveChunk ? i8_prepare<DTYPE, 4, THREADS>
                 : t.K <= 8 * kWaveChunk ? i8_prepare<DTYPE, 8, THREADS>
                                         : i8_prepare<DTYPE, 0, THREADS>;
  kernel<<<grid, THREADS, 0, stream>>>(t, a, p, n_plan, skip);
}

// Many pairs are looked through by more threads.
template <int DTYPE>
void start_prepare(const TokenArgs& t, const I8Args& a, const Plan& p, int n_plan, int skip, hipStream_t stream) {
  if (n_plan > 0 && a.n_tokens * a.k > 8192) start_prepare<DTYPE, 1024>(t, a, p, n_plan, skip, stream);
  else start_prepare<DTYPE, 256>(t, a, p, n_plan, skip, stream);
}

void start_prepare(const TokenArgs& t, int32_t dtype, const I8Args& a, const Plan& p, int n_plan, int skip, hipStream_t stream) {
  if (dtype == TACG_F32) start_prepare<TACG_F32>(t, a, p, n_plan, skip, stream);
  else if (dtype == TACG_BF16) start_prepare<TACG_BF16>(t, a, p, n_plan, skip, stream);
  else start_prepare<TACG_F16>(t, a, p, n_plan, skip, stream);
}

TokenArgs token_args(const void* x, int64_t stride_token, int64_t stride_slot, int64_t n_rows, int32_t rows_of_token, int32_t n_cols,
                     int8_t* q, float* scale, uint32_t* d_err) {
  TokenArgs t{};
  t.x = x;
  t.stride_token = stride_token;
  t.stride_slot = stride_slot;
  t.rows = n_rows;
  t.k = rows_of_token;
  t.K = n_cols;
  t.Kp = (n_cols + kTileCols - 1) / kTileCols * kTileCols;
  t.q = q;
  t.scale = scale;
  t.err = d_err;
  return t;
}

// Pairs of a tile.  So few a matrix, on average, that their time is that of the weights' loads, or so few workgroups that
// most processors would idle: 32, streamed (calls in a row, streamed / tiles in us: gated, 128 experts of 1536 x 2048, top-8: 51 / 55 at 16
// tokens, 72 / 71 at 32, 81 / 78 at 64, 104 / 87 at 512; one matrix of 4096 x 4096: 13 / 20 at 16, 16 / 27 at 64; 200 tokens, top-4,
// 15 of 60 of 2048 x 1408, summed: 21.0 / 22.1).  Else as many as a wave has registers for, or
// fewer where that leaves fewer processors idle.  A processor's time is that of its workgroups' tokens and, for the start and the end of
// each, of 128 tokens more if it has one, 45 if one of them works while another waits (at 2048 columns; measured on grids of 64 to 4500
// workgroups).  In us, 128 / 96 / 64 pairs: 3001 tokens through one gated matrix of 4096 x 2048: 42 / 38 / 40; 800 through 8 of 4096 x
// 2048: 35 / 30 / 36; 1500, top-2, through 16 of 2048 x 2048: 44 / 39 / 33; 8000, top-6, through 64 gated of 2816 x 2048: 336 / 355 / 402.
int tile_of(int64_t pairs, int32_t n_experts, int32_t n_held, int32_t n_rows, int32_t n_cols, bool shared) {
  const int64_t blocks = (n_rows + 4 * kWaves * kTileRows - 1) / (4 * kWaves * kTileRows);
  const double here = static_cast<double>(pairs) * n_held / n_experts;  // on average
  const double grid = (here / 64 + 0.5 * n_held) * blocks;
  if (pairs <= 3 * static_cast<int64_t>(n_experts) || grid < 64 || (grid < 128 && here <= 14.0 * n_held)) return kFewTile;
  int best = kManyTile;
  double least = 0.0;
  for (int tile = kManyTile; tile >= 64; tile -= 32) {
    const double tiles = shared ? static_cast<double>((pairs / n_held + tile - 1) / tile * n_held) : here / tile + 0.5 * n_held;
    const double each = std::ceil(tiles * blocks / 256), cost = each * (tile + (each > 1.0 ? 45.0 : 128.0) * 2048 / n_cols);
    if (tile == kManyTile || cost < 0.95 * least) best = tile, least = cost;
  }
  return best;
}

// Few pairs, whose tokens' levels find room in LDS: one launch, as long as the tokens of a matrix, which are rounded one after another, are few
// too, and, summed, few tokens read the same weights.  One launch / two or three, calls in a row from Python, in us: gated, 6 of 64 experts of
// 2816 x 2048: 10.1 / 13.9 at one token, 33 / 39 at 8; 2 of 8 of 4096 x 2048: 10.1 / 13.6, 17.3 / 21.9 at 8, 23.2 / 19.5 at 16; one of 4096 x 4096:
// 9.5 / 13.1, 11.6 / 13.0 at 4, 13.8 / 13.1 at 6; summed, 8 of 256 of 4096 x 1024: 10.8 / 17.5, 48 / 51 at 8; 2 of 8 of 4096 x 2048: 15.9 / 19.5 at 4,
// 22.5 / 20.0 at 6.  Replayed from a graph, where launches cost less, the same but for one of 4096 x 4096 at 4 tokens: 11.5 / 9.7.  Rows of
// levels are 16 bytes further apart than they are long, so that the same column of neighbours lies in different banks.
struct Few {
  bool is;
  int stride;
  uint32_t lds;
};
Few few_of(int64_t n_tokens, int32_t top_k, int32_t n_experts, int32_t n_cols, int32_t mode, bool slots) {
  Few f{};
  const int64_t pairs = n_tokens * top_k;
  f.stride = (n_cols + kTileCols - 1) / kTileCols * kTileCols + 16;
  const int64_t rows = mode == TACG_Q4_SUM ? (slots ? top_k : 1) : std::min<int64_t>(n_tokens * (slots ? top_k : 1), 16);
  const bool alone = mode == TACG_Q4_SUM ? pairs <= kFewPairs && n_tokens <= std::max(4, n_experts / top_k)
                                         : pairs <= 48 && pairs <= 4 * static_cast<int64_t>(n_experts);
  f.is = alone && rows * f.stride <= 49152;
  f.lds = static_cast<uint32_t>(rows * f.stride);
  return f;
}

template <int DTYPE>
void start_few(const I8Args& a, const Few& f, hipStream_t stream) {
  if (a.mode == TACG_Q4_SUM) {
    i8_few_sum<DTYPE><<<dim3(a.row_tiles, static_cast<uint32_t>(a.n_tokens)), 512, f.lds, stream>>>(a, f.stride);
    return;
  }
  const int width = a.mode == TACG_Q4_GLU ? a.N / 2 : a.N, rows = a.mode == TACG_Q4_GLU ? kTileRows : 2 * kTileRows;
  i8_few<DTYPE><<<dim3((width + rows - 1) / rows, static_cast<uint32_t>(a.n_tokens * a.k)), 256, f.lds, stream>>>(a, rows, f.stride);
}

// The parts of a call's workspace.
struct Space {
  int8_t* levels;
  float* scales;
  float* part;
  Plan plan;
  size_t bytes;
};

Space space_of(void* base, int64_t n_tokens, int32_t top_k, int32_t n_experts, int32_t n_held, int32_t n_rows, int32_t n_cols, int32_t mode, int32_t dtype,
               bool slots, bool shared) {
  Space s{};
  if (few_of(n_tokens, top_k, n_experts, n_cols, mode, slots).is) return s;
  Carver ws{static_cast<char*>(base), 0};
  const int64_t pairs = n_tokens * top_k, rows = slots ? pairs : n_tokens;
  if (dtype != TACG_I8) {
    s.levels = ws.take<int8_t>(rows * ((n_cols + kTileCols - 1) / kTileCols * kTileCols));
    s.scales = ws.take<float>(rows);
  }
  s.plan.tile = tile_of(pairs, n_experts, n_held, n_rows, n_cols, shared);  // `shared` does not change the bytes
  s.plan.sparse = pairs <= n_held;
  s.plan.n_tiles = s.plan.sparse ? static_cast<int32_t>(pairs) : static_cast<int32_t>(pairs / s.plan.tile + n_held);
  s.plan.order = ws.take<int32_t>(pairs);
  s.plan.first = ws.take<int32_t>(n_held + 1);
  s.plan.tiles = ws.take<int2>(pairs / kFewTile + n_held);  // whatever the tile is
  if (mode == TACG_Q4_SUM && top_k > 1) s.part = ws.take<float>(pairs * n_rows);
  s.bytes = ws.used;
  return s;
}

}  // namespace

int launch_i8_pack(const void* w, int32_t dtype, int64_t n_matrices, int32_t n_rows, int32_t n_cols, int8_t* q, float* scale,
                   uint32_t* d_err, hipStream_t stream) {
  PackArgs a{};
  a.w = w;
  a.N = n_rows;
  a.K = n_cols;
  a.row_tiles = (n_rows + kTileRows - 1) / kTileRows;
  a.col_tiles = (n_cols + kTileCols - 1) / kTileCols;
  a.tiles = n_matrices * a.row_tiles;
  a.q = q;
  a.scale = scale;
  a.err = d_err;
  const dim3 grid(static_cast<uint32_t>(std::min<int64_t>(a.tiles, 1 << 20)));
  if (dtype == TACG_F32) i8_pack_kernel<TACG_F32><<<grid, 256, 0, stream>>>(a);
  else if (dtype == TACG_BF16) i8_pack_kernel<TACG_BF16><<<grid, 256, 0, stream>>>(a);
  else i8_pack_kernel<TACG_F16><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? TACG_OK : TACG_E_DEVICE;
}

int launch_token_i8(const void* x, int32_t dtype, int64_t row_stride, int64_t n_rows, int32_t n_cols, int8_t* q, float* scale,
                    uint32_t* d_err, hipStream_t stream) {
  start_prepare(token_args(x, row_stride, 0, n_rows, 1, n_cols, q, scale, d_err), dtype, I8Args{}, Plan{}, 0, 0, stream);
  return hipGetLastError() == hipSuccess ? TACG_OK : TACG_E_DEVICE;
}

size_t expert_i8_workspace(int64_t n_tokens, int32_t top_k, int32_t n_experts, int32_t n_held, int32_t n_rows, int32_t n_cols,
                           int32_t mode, int32_t dtype, bool slots) {
  return space_of(nullptr, n_tokens, top_k, n_experts, n_held, n_rows, n_cols, mode, dtype, slots, false).bytes;
}

int launch_expert_i8(const void* x, int32_t dtype, const float* x_scale, int64_t stride_token, int64_t stride_slot, int64_t n_tokens,
                     int32_t top_k, int32_t n_experts, const int16_t* ids, const int32_t* slot_of_expert, int32_t n_held,
                     const int8_t* w, const float* w_scale, int32_t n_rows, int32_t n_cols, int32_t mode, const float* gate,
                     void* out, int32_t out_dtype, uint32_t* d_err, void* workspace, hipStream_t stream) {
  const bool slots = stride_slot != 0;
  Space s = space_of(workspace, n_tokens, top_k, ids != nullptr ? n_experts : n_held, n_held, n_rows, n_cols, mode, dtype, slots, ids == nullptr);
  I8Args a{};
  a.n_tokens = n_tokens;
  a.k = top_k;
  a.over_k = top_k > 1 ? static_cast<uint32_t>((0x100000000u + top_k - 1) / top_k) : 0;
  a.E = n_experts;
  a.H = n_held;
  a.N = n_rows;
  a.K = n_cols;
  a.row_tiles = (n_rows + kTileRows - 1) / kTileRows;
  a.col_tiles = (n_cols + kTileCols - 1) / kTileCols;
  a.mode = mode;
  a.out_dtype = out_dtype;
  a.slots = slots;
  a.ids = ids;
  a.slot = slot_of_expert;
  a.w = w;
  a.w_scale = w_scale;
  a.gate = gate;
  a.part = s.part;
  a.out = out;
  a.err = d_err;
  const Few few_pairs = few_of(n_tokens, top_k, ids != nullptr ? n_experts : n_held, n_cols, mode, slots);
  if (few_pairs.is) {
    a.tokens = x;
    a.x_scale = x_scale;
    a.x_token = stride_token;
    a.x_slot = stride_slot;
    if (dtype == TACG_I8) start_few<TACG_I8>(a, few_pairs, stream);
    else if (dtype == TACG_F32) start_few<TACG_F32>(a, few_pairs, stream);
    else if (dtype == TACG_BF16) start_few<TACG_BF16>(a, few_pairs, stream);
    else start_few<TACG_F16>(a, few_pairs, stream);
    return hipGetLastError() == hipSuccess ? TACG_OK : TACG_E_DEVICE;
  }
  // tokens are found by 32-bit numbers of their 16-byte pieces
  const int64_t row = static_cast<int64_t>(a.col_tiles) * kTileCols;
  const double span = dtype == TACG_I8 ? static_cast<double>(n_tokens) * stride_token + static_cast<double>(top_k) * stride_slot + row
                                       : static_cast<double>(n_tokens) * (slots ? top_k : 1) * row;
  if (span >= 0x1p36) return TACG_E_UNSUPPORTED;
  // rows of a workgroup: fewer where the grid would leave processors idle
  const bool few = s.plan.tile == kFewTile;
  const int64_t busy = ids == nullptr ? (n_tokens + s.plan.tile - 1) / s.plan.tile * n_held
                                      : std::min<int64_t>(n_tokens * top_k, n_held + n_tokens * top_k / s.plan.tile);
  int frags = 4 * kWaves;
  bool split = false;
  if (few) {
    if (busy * n_rows < 256 * 8 * 64) frags = 2, split = true;
    else if (busy * n_rows < 256 * 12 * 64) frags = 2 * kWaves;
  }
  const int width = mode == TACG_Q4_GLU ? n_rows / 2 : n_rows, per = frags * kTileRows / (mode == TACG_Q4_GLU ? 2 : 1);
  const int blocks = (width + per - 1) / per;
  if (ids == nullptr) s.plan.n_tiles = static_cast<int>((n_tokens + s.plan.tile - 1) / s.plan.tile) * n_held;
  s.plan.by_rows = blocks % 8 == 0 && blocks >= 16 &&
                   static_cast<double>(n_tokens) * top_k >= 1.5 * s.plan.tile * (ids != nullptr ? n_experts : n_held);
  const int clear = ids != nullptr && s.part == nullptr ? static_cast<int>(std::min<int64_t>((n_tokens * top_k + 255) / 256, 512)) : 0;
  const int64_t grid = static_cast<int64_t>(s.plan.n_tiles) * blocks + clear;
  if (grid >= (int64_t(1) << 32) / 256) return TACG_E_UNSUPPORTED;  // threads that a launch holds; so large a grid has tiles of 64 pairs or more
  const int n_plan = ids != nullptr ? std::max(n_held, 1) : 0;
  if (dtype == TACG_I8) {
    a.x = static_cast<const int8_t*>(x);
    a.x_scale = x_scale;
    a.x_token = stride_token;
    a.x_slot = stride_slot;
    if (n_plan > 0) start_prepare(TokenArgs{}, TACG_BF16, a, s.plan, n_plan, 0, stream);
  } else {
    const int64_t width = static_cast<int64_t>(a.col_tiles) * kTileCols;
    const int64_t rows = n_tokens * (slots ? top_k : 1);
    const TokenArgs t = token_args(x, stride_token, stride_slot, rows, slots ? top_k : 1, n_cols, s.levels, s.scales, d_err);
    a.x = s.levels;
    a.x_scale = s.scales;
    a.x_token = width * (slots ? top_k : 1);
    a.x_slot = slots ? width : 0;
    const int skip = slots && ids != nullptr ? static_cast<int>(std::min<int64_t>(rows / 8192 + 1, 64)) : 0;
    start_prepare(t, dtype, a, s.plan, n_plan, skip, stream);
  }
  if (hipGetLastError() != hipSuccess) return TACG_E_DEVICE;
  if (grid > 0) {
    auto* kernel = !few ? i8_tiles : split ? i8_stream<2, true> : frags == 2 * kWaves ? i8_stream<2, false> : i8_stream<4, false>;
    kernel<<<static_cast<uint32_t>(grid), 256, 0, stream>>>(a, s.plan, blocks, per, clear);
  }
  if (s.part != nullptr) {
    const dim3 sums((n_rows + 1023) / 1024, static_cast<uint32_t>(std::min<int64_t>(n_tokens, 65535)));
    i8_combine<<<sums, 256, 0, stream>>>(a);
  }
  return hipGetLastError() == hipSuccess ? TACG_OK : TACG_E_DEVICE;
}

}  // namespace tacg
