// Weights in 4 bits: packing, and the host side of the experts' products (kernels: q4_kernels.h).
//
// q4_pack_kernel: levels, scales and zeros of a weight matrix, a lane per 32 columns (16 bytes of levels), read one by one; done once
//   per weight.  64 matrices of 2048 x 2048 in bfloat16: 548 us, a quarter of what a copy reaches; bound by its loads of 2 bytes.
// q4_combine: sums the 32-bit products of many pairs over the slots of a token.
#include <algorithm>
#include <cmath>

#include "q4_kernels.h"

namespace tacg {

extern template void q4_start<__bf16, false>(const Q4Args& a, hipStream_t stream);
extern template void q4_start<__bf16, true>(const Q4Args& a, hipStream_t stream);
extern template void q4_start<_Float16, false>(const Q4Args& a, hipStream_t stream);
extern template void q4_start<_Float16, true>(const Q4Args& a, hipStream_t stream);

namespace {

__device__ __forceinline__ float widen(__bf16 v) { return static_cast<float>(v); }
__device__ __forceinline__ float widen(_Float16 v) { return static_cast<float>(v); }
__device__ __forceinline__ float widen(float v) { return v; }

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

size_t expert_q4_workspace(int64_t n_tokens, int32_t top_k, int32_t n_experts, int32_t n_rows, int32_t n_cols,
                           int32_t mode) {
  (void)n_cols;
  const int64_t pairs = n_tokens * top_k;
  if (mode != TACG_Q4_SUM || q4_few_pairs(pairs, n_experts, mode)) return 0;
  return align256(static_cast<size_t>(pairs) * n_rows * sizeof(float));
}

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
  a.part = static_cast<float*>(workspace);
  const bool ragged = n_cols % group != 0 || n_cols < kStep;
  if (dtype == TACG_BF16) ragged ? q4_start<__bf16, true>(a, stream) : q4_start<__bf16, false>(a, stream);
  else ragged ? q4_start<_Float16, true>(a, stream) : q4_start<_Float16, false>(a, stream);
  if (mode == TACG_Q4_SUM && !q4_few_pairs(n_tokens * top_k, n_experts, mode)) {
    const dim3 grid((n_rows + 255) / 256, static_cast<uint32_t>(std::min<int64_t>(n_tokens, 65535)));
    if (dtype == TACG_BF16) q4_combine<__bf16><<<grid, 256, 0, stream>>>(a);
    else q4_combine<_Float16><<<grid, 256, 0, stream>>>(a);
  }
  return hipGetLastError() == hipSuccess ? TACG_OK : TACG_E_DEVICE;
}

}  // namespace tacg
