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
#include "route_kernels.h"

namespace tacg {
namespace {
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
                 int32_t score, const float* bias, bool renorm, float scale, int32_t n_groups, int32_t top_groups,
                 int32_t group_best, int16_t* trace, float* gate, float* norm,
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
  a.groups = n_groups;
  a.top_groups = top_groups;
  a.group_size = n_experts / n_groups;
  a.group_best = group_best;
  const int chunk = 16 / dtype_size(dtype);
  a.group_chunks = a.group_size % chunk == 0 ? a.group_size / chunk : 0;
  a.group_lanes = n_groups <= 2 ? 4 : n_groups <= 4 ? 2 : 1;
  a.group_mul = (65536 + a.group_size - 1) / a.group_size;
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
    if (a.groups > 1) start_route_groups(a, dtype, bal, grid, stream);
    else start_rows<false>(a, dtype, bal, grid, stream);
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
