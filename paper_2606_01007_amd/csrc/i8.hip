// Products in 8-bit integers with a scale for each token and for each weight row, for the experts of a GPU.
//
//   x[t][c] ~ sx[t] * qx[t][c],  W[n][c] ~ sw[n] * qw[n][c],  W[n] . x[t] ~ sw[n] * sx[t] * (sum over c of qw qx)
//
// with levels -127..127, half to even, of 127 x / max |x|.  The sum is exact in 32 bits: its magnitude is at most 65536 * 2^14 = 2^30.
//
// i8_tokens: levels and scales of tokens, a workgroup per row.
// i8_pack_kernel: the same of weights, into the tiles that the products read: 16 rows x 64 columns, 16 bytes of each row after another.
// i8_product: a lane per weight row, a workgroup per (token, slot), or summed per token.
#include <algorithm>
#include <cmath>

#include "tacg_internal.h"

namespace tacg {
namespace {

constexpr int kTileRows = 16, kTileCols = 64, kTileBytes = kTileRows * kTileCols, kPiece = 16;

struct I8Args {
  const int8_t* x;          // levels
  const float* x_scale;
  int64_t x_token, x_slot;  // strides of the levels, in bytes
  int64_t n_tokens;
  int32_t k, E, H, N, row_tiles, col_tiles, mode, out_dtype, slots;  // slots: whether every slot has its own x
  const int16_t* ids;       // or null: slot j takes matrix j
  const int32_t* slot;      // [E] or null
  const int8_t* w;
  const float* w_scale;
  const float* gate;        // [T][k] or null: 1
  void* out;
  uint32_t* err;
};

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

template <int DTYPE>
__device__ __forceinline__ float load(const void* p, int64_t i) {
  if constexpr (DTYPE == TACG_F32) return static_cast<const float*>(p)[i];
  else if constexpr (DTYPE == TACG_BF16) return static_cast<float>(static_cast<const __bf16*>(p)[i]);
  else return static_cast<float>(static_cast<const _Float16*>(p)[i]);
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

struct TokenArgs {
  const void* x;
  int64_t stride_token, stride_slot, rows;
  int32_t K, Kp, k;    // k: rows of a token
  int8_t* q;
  float* scale;
  uint32_t* err;
};

// grid: rows.
template <int DTYPE>
__global__ __launch_bounds__(256) void i8_tokens(TokenArgs a) {
  __shared__ uint32_t most[4];
  const int tid = threadIdx.x;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const int64_t first = r / a.k * a.stride_token + r % a.k * a.stride_slot;
    uint32_t m = 0;  // magnitudes order as their bits, and what is not finite is above all others
    for (int c = tid; c < a.K; c += 256) m = max(m, __float_as_uint(load<DTYPE>(a.x, first + c)) & 0x7fffffffu);
    for (int o = 32; o >= 1; o >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), o, 64)));
    if ((tid & 63) == 0) most[tid >> 6] = m;
    __syncthreads();
    m = max(max(most[0], most[1]), max(most[2], most[3]));
    const bool bad = m >= 0x7f800000u;
    const Rounder level(bad ? 0.0f : __uint_as_float(m));
    for (int c = tid; c < a.Kp; c += 256)
      a.q[r * a.Kp + c] = c < a.K && !bad ? static_cast<int8_t>(level(load<DTYPE>(a.x, first + c)) & 0xffu) : int8_t(0);
    if (tid == 0) {
      a.scale[r] = bad ? NAN : __uint_as_float(m) / 127.0f;
      if (bad) atomicOr(a.err, TACG_ERR_VALUE);
    }
    __syncthreads();
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
    if (in)
      for (int c = sub; c < a.K; c += 16) m = max(m, __float_as_uint(load<DTYPE>(a.w, row * a.K + c)) & 0x7fffffffu);
    for (int o = 8; o >= 1; o >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), o, 64)));
    const bool bad = m >= 0x7f800000u;
    const Rounder level(bad ? 0.0f : __uint_as_float(m));
    int8_t* out = a.q + tile * a.col_tiles * kTileBytes + r * kPiece + sub;
    for (int p = 0; p < a.col_tiles * (kTileCols / kPiece); ++p) {
      const int c = p * kPiece + sub;
      out[static_cast<int64_t>(p) * kTileRows * kPiece] =
          in && c < a.K && !bad ? static_cast<int8_t>(level(load<DTYPE>(a.w, row * a.K + c)) & 0xffu) : int8_t(0);
    }
    if (in && sub == 0) {
      a.scale[row] = bad ? NAN : __uint_as_float(m) / 127.0f;
      if (bad) atomicOr(a.err, TACG_ERR_VALUE);
    }
  }
}

__device__ __forceinline__ const int4* row_of(const I8Args& a, int h, int n) {
  return reinterpret_cast<const int4*>(a.w + (static_cast<int64_t>(h) * a.row_tiles + n / kTileRows) * a.col_tiles * kTileBytes) +
         n % kTileRows;
}

// A weight row's sum with a token's levels.
__device__ __forceinline__ int dot(const I8Args& a, int h, int n, const int8_t* levels) {
  const int4* w = row_of(a, h, n);
  const int4* x = reinterpret_cast<const int4*>(levels);
  int s = 0;
  for (int p = 0; p < a.col_tiles * (kTileCols / kPiece); ++p) {
    const int4 u = w[static_cast<int64_t>(p) * kTileRows], v = x[p];
    s = __builtin_amdgcn_sdot4(u.x, v.x, s, false);
    s = __builtin_amdgcn_sdot4(u.y, v.y, s, false);
    s = __builtin_amdgcn_sdot4(u.z, v.z, s, false);
    s = __builtin_amdgcn_sdot4(u.w, v.w, s, false);
  }
  return s;
}

// grid: (blocks of 256 output columns, pairs or, summed, tokens).
__global__ __launch_bounds__(256) void i8_product(I8Args a) {
  const bool sum = a.mode == TACG_Q4_SUM, glu = a.mode == TACG_Q4_GLU;
  const int width = glu ? a.N / 2 : a.N, n = blockIdx.x * 256 + threadIdx.x;
  const int64_t units = sum ? a.n_tokens : a.n_tokens * a.k;
  for (int64_t u = blockIdx.y; u < units; u += gridDim.y) {
    float y = 0.0f;
    for (int i = 0; i < (sum ? a.k : 1); ++i) {
      const int64_t t = sum ? u : u / a.k;
      const int j = sum ? i : static_cast<int>(u % a.k);
      const int64_t pair = t * a.k + j;
      const int h = place_of(a, pair, j);
      if (h < 0) {
        if (h < -1 && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.err, h == kBadId ? TACG_ERR_ID_RANGE : TACG_ERR_TABLE);
        continue;
      }
      if (n >= width) continue;
      const int8_t* levels = a.x + t * a.x_token + j * a.x_slot;
      const float sx = a.x_scale[a.slots ? pair : t];
      const float* sw = a.w_scale + static_cast<int64_t>(h) * a.N;
      float v = static_cast<float>(dot(a, h, n, levels)) * (sx * sw[n]);
      if (glu) {
        const float up = static_cast<float>(dot(a, h, n + width, levels)) * (sx * sw[n + width]);
        v = v / (1.0f + __expf(-v)) * up;
      }
      if (sum) y += (a.gate != nullptr ? a.gate[pair] : 1.0f) * v;
      else y = v;
    }
    if (n < width) store(a.out, u * width + n, y, a.out_dtype);
  }
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

int launch_token_i8(const void* x, int32_t dtype, int64_t stride_token, int64_t stride_slot, int64_t n_rows, int32_t rows_of_token,
                    int32_t n_cols, int8_t* q, float* scale, uint32_t* d_err, hipStream_t stream) {
  TokenArgs a{};
  a.x = x;
  a.stride_token = stride_token;
  a.stride_slot = stride_slot;
  a.rows = n_rows;
  a.k = rows_of_token;
  a.K = n_cols;
  a.Kp = (n_cols + kTileCols - 1) / kTileCols * kTileCols;
  a.q = q;
  a.scale = scale;
  a.err = d_err;
  const dim3 grid(static_cast<uint32_t>(std::min<int64_t>(n_rows, 1 << 20)));
  if (dtype == TACG_F32) i8_tokens<TACG_F32><<<grid, 256, 0, stream>>>(a);
  else if (dtype == TACG_BF16) i8_tokens<TACG_BF16><<<grid, 256, 0, stream>>>(a);
  else i8_tokens<TACG_F16><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? TACG_OK : TACG_E_DEVICE;
}

size_t expert_i8_workspace(int64_t n_tokens, int32_t top_k, int32_t n_cols, int32_t dtype, bool slots) {
  if (dtype == TACG_I8) return 0;
  const size_t rows = static_cast<size_t>(n_tokens) * (slots ? top_k : 1);
  return align256(rows * ((n_cols + kTileCols - 1) / kTileCols * kTileCols)) + align256(rows * sizeof(float));
}

int launch_expert_i8(const void* x, int32_t dtype, const float* x_scale, int64_t stride_token, int64_t stride_slot, int64_t n_tokens,
                     int32_t top_k, int32_t n_experts, const int16_t* ids, const int32_t* slot_of_expert, int32_t n_held,
                     const int8_t* w, const float* w_scale, int32_t n_rows, int32_t n_cols, int32_t mode, const float* gate,
                     void* out, int32_t out_dtype, uint32_t* d_err, void* workspace, hipStream_t stream) {
  I8Args a{};
  const bool slots = stride_slot != 0;
  a.n_tokens = n_tokens;
  a.k = top_k;
  a.E = n_experts;
  a.H = n_held;
  a.N = n_rows;
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
  a.out = out;
  a.err = d_err;
  if (dtype == TACG_I8) {
    a.x = static_cast<const int8_t*>(x);
    a.x_scale = x_scale;
    a.x_token = stride_token;
    a.x_slot = stride_slot;
  } else {
    Carver ws{static_cast<char*>(workspace), 0};
    const int64_t rows = n_tokens * (slots ? top_k : 1), width = static_cast<int64_t>(a.col_tiles) * kTileCols;
    int8_t* q = ws.take<int8_t>(rows * width);
    float* scale = ws.take<float>(rows);
    const int rc = launch_token_i8(x, dtype, stride_token, stride_slot, rows, slots ? top_k : 1, n_cols, q, scale, d_err, stream);
    if (rc != TACG_OK) return rc;
    a.x = q;
    a.x_scale = scale;
    a.x_token = width * (slots ? top_k : 1);
    a.x_slot = slots ? width : 0;
  }
  const int64_t units = mode == TACG_Q4_SUM ? n_tokens : n_tokens * top_k;
  const int width = mode == TACG_Q4_GLU ? n_rows / 2 : n_rows;
  const dim3 grid((width + 255) / 256, static_cast<uint32_t>(std::min<int64_t>(units, 65535)));
  i8_product<<<grid, 256, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? TACG_OK : TACG_E_DEVICE;
}

}  // namespace tacg
