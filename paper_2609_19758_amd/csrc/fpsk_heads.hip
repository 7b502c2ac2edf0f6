// Query, key and value heads from a delivered QKV product (gfx950).
//
// A row of the product C (t x (hq + 2 hkv) hd, FP32) holds a token's query heads, key heads and
// value heads.  For a query or key head x with gains g and a position p:
//   y = g x / sqrt(mean x^2 + eps)             (left out without gains)
//   the first rd entries of y are rotated in pairs by the angles p w_i, i < rd / 2:
//     (a, b) -> (a cos - b sin, b cos + a sin), pairs (i, i + rd / 2) or (2i, 2i + 1)
// and rounded once; value heads are rounded only.  With r = 1 / sqrt(mean x^2 + eps) and u the
// gradient of y (the output's, rotated back), the backward pass is
//   dg = sum u x r,   dx = r (g u - x r^2 mean(x g u)).
#include "fpsk_layers.h"

#include <algorithm>

namespace fpsk {

namespace {

constexpr int kMaxHead = 512;

struct HeadArgs {
  const float* C;
  int64_t t;
  int hq, hkv, hd, rd;
  int inter;               // pairs (2i, 2i + 1)
  const float* gq;
  const float* gk;
  float eps;
  const int64_t* pos;
  const float* freq;
  uint16_t* q;
  uint16_t* k;
  uint16_t* v;
  // backward
  const uint16_t* dq;
  const uint16_t* dk;
  const uint16_t* dv;
  uint16_t* dC;
  float* part;             // work-groups x 2 x hd partial gain gradients (q, k)
  float* dgq;
  float* dgk;
  int groups;
};

// cos and sin of p w.  The angle is formed and reduced in FP64: at positions of a million its
// FP32 product is off by a tenth of a turn.  What is left, at most half a turn, is exact enough in
// FP32 (2^-23 absolute) for results that are rounded to a half format.
__device__ __forceinline__ void angle(int64_t p, float w, float* c, float* s) {
  const double a = static_cast<double>(p) * static_cast<double>(w);
  const double n = rint(a * 0.15915494309189535);                 // turns
  const float r = static_cast<float>(fma(-n, 2.4492935982947064e-16, fma(-n, 6.283185307179586, a)));
  sincosf(r, s, c);
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// One token per work-group, one head per wave at a time.
template <int DT>
__global__ __launch_bounds__(kThreads) void heads_kernel(HeadArgs a) {
  __shared__ float cs[kMaxHead / 2], sn[kMaxHead / 2];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int half = a.rd / 2, width = a.hq + 2 * a.hkv;
  for (int64_t i = blockIdx.x; i < a.t; i += gridDim.x) {
    __syncthreads();
    for (int p = threadIdx.x; p < half; p += kThreads) angle(a.pos[i], a.freq[p], &cs[p], &sn[p]);
    __syncthreads();
    for (int h = wave; h < width; h += kThreads / 64) {
      const float* x = a.C + (i * width + h) * a.hd;
      const bool isq = h < a.hq, isk = !isq && h < a.hq + a.hkv;
      uint16_t* y = isq   ? a.q + (i * a.hq + h) * a.hd
                    : isk ? a.k + (i * a.hkv + h - a.hq) * a.hd
                          : a.v + (i * a.hkv + h - a.hq - a.hkv) * a.hd;
      if (!isq && !isk) {
        for (int e = lane; e < a.hd; e += 64) y[e] = to_half<DT>(x[e]);
        continue;
      }
      const float* g = isq ? a.gq : a.gk;
      float r = 1.0f;
      if (g != nullptr) {
        float s = 0.0f;
        for (int e = lane; e < a.hd; e += 64) s += x[e] * x[e];
        r = 1.0f / sqrtf(wave_sum(s) / static_cast<float>(a.hd) + a.eps);
      }
      for (int p = lane; p < half; p += 64) {
        const int e0 = a.inter ? 2 * p : p, e1 = a.inter ? 2 * p + 1 : p + half;
        float u = x[e0], w = x[e1];
        if (g != nullptr) {
          u *= r * g[e0];
          w *= r * g[e1];
        }
        y[e0] = to_half<DT>(u * cs[p] - w * sn[p]);
        y[e1] = to_half<DT>(w * cs[p] + u * sn[p]);
      }
      for (int e = a.rd + lane; e < a.hd; e += 64) {
        y[e] = to_half<DT>(g != nullptr ? x[e] * r * g[e] : x[e]);
      }
    }
  }
}

// The backward pass; the gradients of the gains are summed per work-group in LDS, every wave on
// columns of its own, in the order of its heads.
template <int DT>
__global__ __launch_bounds__(kThreads) void heads_grad_kernel(HeadArgs a) {
  __shared__ float cs[kMaxHead / 2], sn[kMaxHead / 2];
  __shared__ float sums[4][2][kMaxHead];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int half = a.rd / 2, width = a.hq + 2 * a.hkv;
  for (int e = lane; e < kMaxHead; e += 64) sums[wave][0][e] = sums[wave][1][e] = 0.0f;
  for (int64_t i = blockIdx.x; i < a.t; i += gridDim.x) {
    __syncthreads();
    for (int p = threadIdx.x; p < half; p += kThreads) angle(a.pos[i], a.freq[p], &cs[p], &sn[p]);
    __syncthreads();
    for (int h = wave; h < width; h += kThreads / 64) {
      const bool isq = h < a.hq, isk = !isq && h < a.hq + a.hkv;
      const uint16_t* dy = isq   ? a.dq + (i * a.hq + h) * a.hd
                           : isk ? a.dk + (i * a.hkv + h - a.hq) * a.hd
                                 : a.dv + (i * a.hkv + h - a.hq - a.hkv) * a.hd;
      uint16_t* dx = a.dC + (i * width + h) * a.hd;
      if (!isq && !isk) {
        for (int e = lane; e < a.hd; e += 64) dx[e] = dy[e];
        continue;
      }
      const float* g = isq ? a.gq : a.gk;
      const float* x = a.C + (i * width + h) * a.hd;
      // entry e of the gradient rotated back
      auto back = [&](int e) {
        if (e >= a.rd) return from_half<DT>(dy[e]);
        const int p = a.inter ? e >> 1 : (e < half ? e : e - half);
        const bool first = a.inter ? (e & 1) == 0 : e < half;
        const int o = a.inter ? e ^ 1 : (first ? e + half : e - half);
        const float m = from_half<DT>(dy[e]), n = from_half<DT>(dy[o]);
        return first ? m * cs[p] + n * sn[p] : m * cs[p] - n * sn[p];
      };
      if (g == nullptr) {
        for (int e = lane; e < a.hd; e += 64) dx[e] = to_half<DT>(back(e));
        continue;
      }
      float ss = 0.0f, xu = 0.0f;
      for (int e = lane; e < a.hd; e += 64) {
        ss += x[e] * x[e];
        xu += x[e] * g[e] * back(e);
      }
      const float n = static_cast<float>(a.hd);
      const float r = 1.0f / sqrtf(wave_sum(ss) / n + a.eps);
      const float c = r * r * wave_sum(xu) / n;
      float* sum = sums[wave][isq ? 0 : 1];
      for (int e = lane; e < a.hd; e += 64) {
        const float u = back(e);
        dx[e] = to_half<DT>(r * (g[e] * u - x[e] * c));
        sum[e] += u * x[e] * r;
      }
    }
  }
  if (a.gq == nullptr) return;
  __syncthreads();
  for (int e = threadIdx.x; e < 2 * a.hd; e += kThreads) {
    const int w = e / a.hd, j = e % a.hd;
    a.part[static_cast<int64_t>(blockIdx.x) * 2 * a.hd + e] =
        (sums[0][w][j] + sums[1][w][j]) + (sums[2][w][j] + sums[3][w][j]);
  }
}

// The gains' gradients: the work-groups' sums in order, one entry per wave.
__global__ __launch_bounds__(64) void gains_kernel(HeadArgs a) {
  const int e = blockIdx.x, lane = threadIdx.x;
  double s = 0.0;
  for (int g = lane; g < a.groups; g += 64) s += a.part[static_cast<int64_t>(g) * 2 * a.hd + e];
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (lane == 0) {
    if (e < a.hd) {
      a.dgq[e] = static_cast<float>(s);
    } else {
      a.dgk[e - a.hd] = static_cast<float>(s);
    }
  }
}

// ---- host ------------------------------------------------------------------------------------

bool heads_dims(int64_t t, int hq, int hkv, int hd) {
  return t >= 0 && t < kDimLimit && hq >= 1 && hkv >= 1 && hd >= 1 && hd <= kMaxHead &&
         hq <= 65536 && hkv <= 65536 &&
         static_cast<double>(t) * (hq + 2.0 * hkv) * hd <= 1099511627776.0;
}

int grad_groups(int64_t t, int cus) { return static_cast<int>(std::min<int64_t>(t, 4 * cus)); }

// What both directions check; nothing launched on an error.
fpsketch_status heads_check(const char* who, int64_t t, int hq, int hkv, int hd, const float* gq,
                            const float* gk, double eps, const int64_t* pos, const float* freq,
                            int rd, int pairs, fpsketch_dtype dtype) {
  char msg[160];
  auto bad = [&](fpsketch_status s, const char* what) {
    std::snprintf(msg, sizeof(msg), "%s: %s", who, what);
    return layer_error(s, msg);
  };
  if (!half_type(dtype)) return bad(FPSK_EDTYPE, "the heads are FP16 or BF16");
  if (!heads_dims(t, hq, hkv, hd)) return bad(FPSK_ESHAPE, "dimensions (a head has 1 to 512 entries)");
  if (rd < 0 || rd > hd || rd % 2 != 0) return bad(FPSK_EINVAL, "rd must be even and at most hd");
  if (pairs != FPSK_PAIRS_HALF && pairs != FPSK_PAIRS_INTERLEAVED) return bad(FPSK_EINVAL, "unknown pairs");
  if ((gq == nullptr) != (gk == nullptr)) return bad(FPSK_EINVAL, "gains for queries or keys only");
  if (gq != nullptr && !(eps >= 0.0 && std::isfinite(eps))) return bad(FPSK_EINVAL, "eps must be finite and not negative");
  if (rd > 0 && t > 0 && (pos == nullptr || freq == nullptr)) return bad(FPSK_EINVAL, "null pos or freq");
  if (!aligned(gq, 4) || !aligned(gk, 4) || !aligned(pos, 8) || !aligned(freq, 4)) {
    return bad(FPSK_EINVAL, "a pointer is not aligned to its elements");
  }
  return FPSK_OK;
}

}  // namespace

}  // namespace fpsk

using namespace fpsk;

extern "C" {

fpsketch_status fpsketch_heads(const float* C, int64_t t, int32_t hq, int32_t hkv, int32_t hd,
                               const float* gq, const float* gk, double eps, const int64_t* pos,
                               const float* freq, int32_t rd, int32_t pairs, fpsketch_dtype dtype,
                               void* q, void* k, void* v, void* stream) {
  fpsketch_status s = heads_check("fpsketch_heads", t, hq, hkv, hd, gq, gk, eps, pos, freq, rd, pairs, dtype);
  if (s != FPSK_OK) return s;
  if (t == 0) return FPSK_OK;
  if (C == nullptr || q == nullptr || k == nullptr || v == nullptr) return layer_error(FPSK_EINVAL, "fpsketch_heads: null pointer");
  if (!aligned(C, 4) || !aligned(q, 2) || !aligned(k, 2) || !aligned(v, 2)) {
    return layer_error(FPSK_EINVAL, "fpsketch_heads: a pointer is not aligned to its elements");
  }
  int cus = 0;
  s = layer_device(&cus);
  if (s != FPSK_OK) return s;
  const int64_t nq = 2 * t * hq * hd, nk = 2 * t * hkv * hd;
  const Span in[] = {{C, 2 * (nq + 2 * nk)}, {gq, 4 * hd}, {gk, 4 * hd}, {pos, rd > 0 ? 8 * t : 0}, {freq, 2 * rd}};
  const Span out[] = {{q, nq}, {k, nk}, {v, nk}};
  if (!disjoint(in, out)) return layer_error(FPSK_EINVAL, "fpsketch_heads: an output overlaps another argument");
  HeadArgs a{};
  a.C = C;
  a.t = t;
  a.hq = hq;
  a.hkv = hkv;
  a.hd = hd;
  a.rd = rd;
  a.inter = pairs == FPSK_PAIRS_INTERLEAVED;
  a.gq = gq;
  a.gk = gk;
  a.eps = static_cast<float>(eps);
  a.pos = pos;
  a.freq = freq;
  a.q = static_cast<uint16_t*>(q);
  a.k = static_cast<uint16_t*>(k);
  a.v = static_cast<uint16_t*>(v);
  const auto st = static_cast<hipStream_t>(stream);
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(t, 1 << 20)));
  return launched(dtype == FPSK_BF16
                      ? launch_k(heads_kernel<1>, grid, dim3(kThreads), 0, st, nullptr, nullptr, a)
                      : launch_k(heads_kernel<0>, grid, dim3(kThreads), 0, st, nullptr, nullptr, a),
                  "fpsketch_heads");
}

int64_t fpsketch_heads_grad_workspace(int64_t t, int32_t hq, int32_t hkv, int32_t hd) {
  int cus = 0;
  if (!heads_dims(t, hq, hkv, hd) || t == 0 || layer_device(&cus) != FPSK_OK) return 0;
  return int64_t{8} * grad_groups(t, cus) * hd;
}

fpsketch_status fpsketch_heads_grad(const void* dq, const void* dk, const void* dv, const float* C,
                                    int64_t t, int32_t hq, int32_t hkv, int32_t hd, const float* gq,
                                    const float* gk, double eps, const int64_t* pos,
                                    const float* freq, int32_t rd, int32_t pairs,
                                    fpsketch_dtype dtype, void* dC, float* dgq, float* dgk,
                                    void* workspace, int64_t workspace_bytes, void* stream) {
  fpsketch_status s = heads_check("fpsketch_heads_grad", t, hq, hkv, hd, gq, gk, eps, pos, freq, rd, pairs, dtype);
  if (s != FPSK_OK) return s;
  const bool norm = gq != nullptr;
  if (t > 0 && (dq == nullptr || dk == nullptr || dv == nullptr || dC == nullptr || (norm && C == nullptr))) {
    return layer_error(FPSK_EINVAL, "fpsketch_heads_grad: null pointer");
  }
  if (norm && (dgq == nullptr || dgk == nullptr)) return layer_error(FPSK_EINVAL, "fpsketch_heads_grad: null gradient of the gains");
  if (!aligned(C, 4) || !aligned(dq, 2) || !aligned(dk, 2) || !aligned(dv, 2) || !aligned(dC, 2) ||
      !aligned(dgq, 4) || !aligned(dgk, 4)) {
    return layer_error(FPSK_EINVAL, "fpsketch_heads_grad: a pointer is not aligned to its elements");
  }
  int cus = 0;
  s = layer_device(&cus);
  if (s != FPSK_OK) return s;
  const int groups = grad_groups(t, cus);
  const int64_t need = norm ? int64_t{8} * groups * hd : 0;
  if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned(workspace, 16))) {
    return layer_error(FPSK_EINVAL, "fpsketch_heads_grad: workspace smaller than fpsketch_heads_grad_workspace, or not aligned to 16 bytes");
  }
  const int64_t nq = 2 * t * hq * hd, nk = 2 * t * hkv * hd;
  const Span in[] = {{dq, nq}, {dk, nk}, {dv, nk}, {norm ? C : nullptr, 2 * (nq + 2 * nk)}, {gq, 4 * hd},
                     {gk, 4 * hd}, {pos, rd > 0 ? 8 * t : 0}, {freq, 2 * rd}};
  const Span out[] = {{dC, nq + 2 * nk}, {norm ? dgq : nullptr, 4 * hd}, {norm ? dgk : nullptr, 4 * hd}, {workspace, need}};
  if (!disjoint(in, out)) return layer_error(FPSK_EINVAL, "fpsketch_heads_grad: an output overlaps another argument");
  HeadArgs a{};
  a.C = C;
  a.t = t;
  a.hq = hq;
  a.hkv = hkv;
  a.hd = hd;
  a.rd = rd;
  a.inter = pairs == FPSK_PAIRS_INTERLEAVED;
  a.gq = gq;
  a.gk = gk;
  a.eps = static_cast<float>(eps);
  a.pos = pos;
  a.freq = freq;
  a.dq = static_cast<const uint16_t*>(dq);
  a.dk = static_cast<const uint16_t*>(dk);
  a.dv = static_cast<const uint16_t*>(dv);
  a.dC = static_cast<uint16_t*>(dC);
  a.part = static_cast<float*>(workspace);
  a.dgq = dgq;
  a.dgk = dgk;
  a.groups = groups;
  const auto st = static_cast<hipStream_t>(stream);
  hipError_t e = hipSuccess;
  if (t > 0) {
    const dim3 grid(static_cast<unsigned>(groups));
    e = dtype == FPSK_BF16
            ? launch_k(heads_grad_kernel<1>, grid, dim3(kThreads), 0, st, nullptr, nullptr, a)
            : launch_k(heads_grad_kernel<0>, grid, dim3(kThreads), 0, st, nullptr, nullptr, a);
  }
  if (e == hipSuccess && norm) {
    e = launch_k(gains_kernel, dim3(static_cast<unsigned>(2 * hd)), dim3(64), 0, st, nullptr, nullptr, a);
  }
  return launched(e, "fpsketch_heads_grad");
}

}  // extern "C"
