// Products of the experts' weights in 4 bits with the tokens routed to them.
//
//   W[h][n][c] = scale[h][n][c / group] * (level[h][n][c] - zero[h][n][c / group]),   zero = 8 where none is given.
//
// q4_pack_kernel: levels, scales and zeros of a weight matrix, a lane per 32 columns (16 bytes of levels).
// q4_simple: a wave per output value; every lane takes 32 columns at a time and sums level * x and x in 32 bits; scale and zero are
//   applied to the two sums of a piece, which lies in one group.
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
  void* out;
  uint32_t* err;
};

__device__ __forceinline__ float widen(__bf16 v) { return static_cast<float>(v); }
__device__ __forceinline__ float widen(_Float16 v) { return static_cast<float>(v); }
__device__ __forceinline__ float widen(float v) { return v; }

// Where the weights of an expert id are held: -1 for none (an unused slot, an expert of another GPU, an invalid entry).
__device__ __forceinline__ int held_of(const Q4Args& a, int id) {
  if (id < 0 || id >= a.E) {
    if (id != -1) atomicOr(a.err, TACG_ERR_ID_RANGE);
    return -1;
  }
  const int h = a.slot != nullptr ? a.slot[id] : id;
  if (h >= a.H) {
    atomicOr(a.err, TACG_ERR_TABLE);
    return -1;
  }
  return h < 0 ? -1 : h;
}

template <class T>
__device__ __forceinline__ float wave_dot(const Q4Args& a, int h, int n, const T* x, int lane) {
  const int64_t r = static_cast<int64_t>(h) * a.N + n;
  const uint4* q = reinterpret_cast<const uint4*>(a.q) + r * a.pieces;
  const T* scales = static_cast<const T*>(a.scales) + r * a.n_groups;
  float sum = 0.0f;
  for (int p = lane; p < a.pieces; p += 64) {
    const uint4 w = q[p];
    const uint32_t word[4] = {w.x, w.y, w.z, w.w};
    float dot = 0.0f, all = 0.0f;
#pragma unroll
    for (int i = 0; i < kPiece; ++i) {
      const int c = p * kPiece + i;
      const float v = c < a.K ? widen(x[c]) : 0.0f;
      dot += static_cast<float>((word[i / 8] >> (4 * (i % 8))) & 15u) * v;
      all += v;
    }
    const int g = p * kPiece / a.group;
    const float zero = a.zeros != nullptr ? static_cast<float>(a.zeros[r * a.n_groups + g]) : 8.0f;
    sum += widen(scales[g]) * (dot - zero * all);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
  return sum;
}

// grid: (output columns / 4, slots or tokens, blocks of them); a wave per output.
template <class T>
__global__ __launch_bounds__(256) void q4_simple(Q4Args a) {
  const int lane = threadIdx.x & 63;
  const int width = a.mode == TACG_Q4_GLU ? a.N / 2 : a.N;
  const int n = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (n >= width) return;
  const T* x = static_cast<const T*>(a.x);
  T* out = static_cast<T*>(a.out);
  const int64_t items = a.mode == TACG_Q4_SUM ? a.n_tokens : a.n_tokens * a.k;
  for (int64_t i = blockIdx.y; i < items; i += gridDim.y) {
    float y = 0.0f;
    if (a.mode == TACG_Q4_SUM) {
      for (int j = 0; j < a.k; ++j) {
        const int h = held_of(a, a.ids[i * a.k + j]);
        if (h >= 0) y += a.gate[i * a.k + j] * wave_dot(a, h, n, x + i * a.x_token + j * a.x_slot, lane);
      }
    } else {
      const int h = held_of(a, a.ids[i]);
      if (h >= 0) {
        const T* v = x + (i / a.k) * a.x_token + (i % a.k) * a.x_slot;
        y = wave_dot(a, h, n, v, lane);
        if (a.mode == TACG_Q4_GLU) y = y / (1.0f + __expf(-y)) * wave_dot(a, h, n + width, v, lane);
      }
    }
    if (lane == 0) out[i * width + n] = static_cast<T>(y);
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

size_t expert_q4_workspace(int64_t, int32_t, int32_t, int32_t, int32_t, int32_t) { return 0; }

int launch_expert_q4(const void* x, int32_t dtype, int64_t x_stride_token, int64_t x_stride_slot, int64_t n_tokens,
                     int32_t top_k, int32_t n_experts, const int16_t* ids, const int32_t* slot_of_expert,
                     int32_t n_held, const uint8_t* q, const void* scales, const uint8_t* zeros, int32_t group,
                     int32_t n_rows, int32_t n_cols, int32_t mode, const float* gate, void* out, uint32_t* d_err,
                     void* workspace, hipStream_t stream) {
  (void)workspace;
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
  const int width = mode == TACG_Q4_GLU ? n_rows / 2 : n_rows;
  const int64_t items = mode == TACG_Q4_SUM ? n_tokens : n_tokens * top_k;
  const dim3 grid((width + 3) / 4, static_cast<uint32_t>(std::min<int64_t>(items, 65535)));
  if (dtype == TACG_BF16) q4_simple<__bf16><<<grid, 256, 0, stream>>>(a);
  else q4_simple<_Float16><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? TACG_OK : TACG_E_DEVICE;
}

}  // namespace tacg
