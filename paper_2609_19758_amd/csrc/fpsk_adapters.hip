// Low-rank adapters of many requests added to a shared projection's product (gfx950).
//
//   Y_i = out(C_i + s_a (X_i A_a^T) B_a^T),  a = index_i
//
// C (t x n FP32) is the verified product X W^T of the shared weight, A count x r x k and
// B count x n x r the adapters' factors, s their scales.  index -1: no adapter, Y_i = out(C_i).
// Any other index outside [0, count) makes the row NaN, so that it cannot pass unseen.
#include "fpsk_layers.h"

#include <algorithm>

namespace fpsk {

namespace {

struct AdapterArgs {
  const float* C;
  const uint16_t* X;
  const uint16_t* A;
  const uint16_t* B;
  const int32_t* index;
  const float* scale;
  int64_t t, k, n;
  int count, rank;
  float* V;                // t x rank: X_i A_a^T
  void* Y;
  int half;                // Y in the half format
};

// V, one row per wave.
template <int DT>
__global__ __launch_bounds__(kThreads) void shrink_kernel(AdapterArgs a) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 4 + wave; i < a.t;
       i += static_cast<int64_t>(gridDim.x) * 4) {
    const int which = a.index[i];
    if (which < 0 || which >= a.count) continue;
    const uint16_t* x = a.X + i * a.k;
    for (int j = 0; j < a.rank; ++j) {
      const uint16_t* w = a.A + (static_cast<int64_t>(which) * a.rank + j) * a.k;
      float s = 0.0f;
      for (int64_t e = lane; e < a.k; e += 64) s += from_half<DT>(x[e]) * from_half<DT>(w[e]);
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
      if (lane == 0) a.V[i * a.rank + j] = s;
    }
  }
}

// Y, one element a thread.
template <int DT>
__global__ __launch_bounds__(kThreads) void expand_kernel(AdapterArgs a) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  for (int64_t o = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; o < a.t * a.n; o += step) {
    const int64_t i = o / a.n, j = o - i * a.n;
    const int which = a.index[i];
    float y = a.C[o];
    if (which >= 0 && which < a.count) {
      const uint16_t* b = a.B + (static_cast<int64_t>(which) * a.n + j) * a.rank;
      float s = 0.0f;
      for (int e = 0; e < a.rank; ++e) s += a.V[i * a.rank + e] * from_half<DT>(b[e]);
      y += a.scale[which] * s;
    } else if (which != -1) {
      y = __builtin_nanf("");
    }
    if (a.half) {
      static_cast<uint16_t*>(a.Y)[o] = to_half<DT>(y);
    } else {
      static_cast<float*>(a.Y)[o] = y;
    }
  }
}

bool adapter_dims(int64_t t, int64_t k, int64_t n, int32_t count, int32_t rank) {
  const double most = 1099511627776.0;
  return t >= 0 && t < kDimLimit && k >= 1 && k < kDimLimit && n >= 1 && n < kDimLimit && count >= 1 &&
         rank >= 1 && rank <= 256 && static_cast<double>(t) * k <= most &&
         static_cast<double>(t) * n <= most && static_cast<double>(count) * rank * k <= most &&
         static_cast<double>(count) * rank * n <= most;
}

}  // namespace

}  // namespace fpsk

using namespace fpsk;

extern "C" {

int64_t fpsketch_adapters_workspace(int64_t t, int64_t k, int64_t n, int32_t count, int32_t rank) {
  return adapter_dims(t, k, n, count, rank) ? 4 * t * rank : 0;
}

fpsketch_status fpsketch_adapters(const float* C, const void* X, const void* A, const void* B,
                                  const int32_t* index, const float* scale, int64_t t, int64_t k,
                                  int64_t n, int32_t count, int32_t rank, fpsketch_dtype dtype,
                                  void* Y, fpsketch_dtype y_dtype, void* workspace,
                                  int64_t workspace_bytes, void* stream) {
  if (!half_type(dtype)) return layer_error(FPSK_EDTYPE, "fpsketch_adapters: X, A and B are FP16 or BF16");
  if (y_dtype != dtype && y_dtype != FPSK_F32) return layer_error(FPSK_EDTYPE, "fpsketch_adapters: Y has the half format of X, or FP32");
  if (!adapter_dims(t, k, n, count, rank)) return layer_error(FPSK_ESHAPE, "fpsketch_adapters: dimensions (rank 1 to 256)");
  if (t == 0) return FPSK_OK;
  if (C == nullptr || X == nullptr || A == nullptr || B == nullptr || index == nullptr || scale == nullptr || Y == nullptr) {
    return layer_error(FPSK_EINVAL, "fpsketch_adapters: null pointer");
  }
  const bool half = y_dtype != FPSK_F32;
  if (!aligned(C, 4) || !aligned(X, 2) || !aligned(A, 2) || !aligned(B, 2) || !aligned(index, 4) ||
      !aligned(scale, 4) || !aligned(Y, half ? 2 : 4)) {
    return layer_error(FPSK_EINVAL, "fpsketch_adapters: a pointer is not aligned to its elements");
  }
  int cus = 0;
  const fpsketch_status s = layer_device(&cus);
  if (s != FPSK_OK) return s;
  const int64_t need = fpsketch_adapters_workspace(t, k, n, count, rank);
  if (workspace == nullptr || workspace_bytes < need || !aligned(workspace, 16)) {
    return layer_error(FPSK_EINVAL, "fpsketch_adapters: workspace smaller than fpsketch_adapters_workspace, or not aligned to 16 bytes");
  }
  const Span in[] = {{C, 4 * t * n}, {X, 2 * t * k}, {A, int64_t{2} * count * rank * k},
                     {B, int64_t{2} * count * rank * n}, {index, 4 * t}, {scale, int64_t{4} * count}};
  const Span out[] = {{Y, (half ? 2 : 4) * t * n}, {workspace, need}};
  if (!disjoint(in, out)) return layer_error(FPSK_EINVAL, "fpsketch_adapters: an output overlaps another argument");
  AdapterArgs a{};
  a.C = C;
  a.X = static_cast<const uint16_t*>(X);
  a.A = static_cast<const uint16_t*>(A);
  a.B = static_cast<const uint16_t*>(B);
  a.index = index;
  a.scale = scale;
  a.t = t;
  a.k = k;
  a.n = n;
  a.count = count;
  a.rank = rank;
  a.V = static_cast<float*>(workspace);
  a.Y = Y;
  a.half = half;
  const auto st = static_cast<hipStream_t>(stream);
  const dim3 g1(static_cast<unsigned>(std::min<int64_t>((t + 3) / 4, 65536)));
  const dim3 g2(static_cast<unsigned>(std::min<int64_t>((t * n + kThreads - 1) / kThreads, 16384)));
  hipError_t e = dtype == FPSK_BF16
                     ? launch_k(shrink_kernel<1>, g1, dim3(kThreads), 0, st, nullptr, nullptr, a)
                     : launch_k(shrink_kernel<0>, g1, dim3(kThreads), 0, st, nullptr, nullptr, a);
  if (e == hipSuccess) {
    e = dtype == FPSK_BF16
            ? launch_k(expand_kernel<1>, g2, dim3(kThreads), 0, st, nullptr, nullptr, a)
            : launch_k(expand_kernel<0>, g2, dim3(kThreads), 0, st, nullptr, nullptr, a);
  }
  return launched(e, "fpsketch_adapters");
}

}  // extern "C"
