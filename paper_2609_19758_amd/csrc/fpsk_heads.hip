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
#include <cfloat>

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
  float* part;             // 2 x hd x work-groups: partial gain gradients (q, k)
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

// Heads whose entries come in whole groups: hd and rd multiples of 8 (loads and stores of 8 and 16
// bytes at element alignment, which gfx950 takes).  LPH lanes take a head, 8 entries each: the groups
// of 4 that rotate with each other (4u and rd / 2 + 4u, or 8u and 8u + 4 with interleaved pairs), or 8
// neighbours past rd.  A lane meets the same entries in every head, so gains and angles stay in its
// registers, and nothing passes through LDS (8191 tokens of 120 heads of 128: 144 us, 340 us in the
// kernel for any size below).
struct Unit {
  int e0, e1;              // its groups of 4
  bool turns;
};

__device__ __forceinline__ Unit unit_of(const HeadArgs& a, int u) {
  if (!a.inter && 8 * u < a.rd) return {4 * u, a.rd / 2 + 4 * u, true};
  return {8 * u, 8 * u + 4, 8 * u < a.rd};
}

template <int LPH>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int o = LPH / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// (x0, x1) turned by the angles of (c, s): pairs (x0[e], x1[e]), or neighbours.
__device__ __forceinline__ void turn(bool inter, f32x4 c, f32x4 s, f32x4& x0, f32x4& x1) {
  if (inter) {
    const f32x4 a = x0, b = x1;
    x0 = f32x4{a[0] * c[0] - a[1] * s[0], a[1] * c[0] + a[0] * s[0], a[2] * c[1] - a[3] * s[1], a[3] * c[1] + a[2] * s[1]};
    x1 = f32x4{b[0] * c[2] - b[1] * s[2], b[1] * c[2] + b[0] * s[2], b[2] * c[3] - b[3] * s[3], b[3] * c[3] + b[2] * s[3]};
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float p = x0[e], q = x1[e];
      x0[e] = p * c[e] - q * s[e];
      x1[e] = q * c[e] + p * s[e];
    }
  }
}

__device__ __forceinline__ void unit_angles(const HeadArgs& a, int64_t i, int u, f32x4& c, f32x4& s) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float x, y;
    angle(a.pos[i], a.freq[4 * u + e], &x, &y);
    c[e] = x;
    s[e] = y;
  }
}

template <int DT>
__device__ __forceinline__ void put4(uint16_t* y, f32x4 x) {
  *reinterpret_cast<u16x4_a2*>(y) = to_half4<DT>(x[0], x[1], x[2], x[3]);
}

// One token per work-group, or part of its heads (gridDim.y parts): bound by reading C and writing
// the heads (8191 x 120 x 128: 5.2 TB/s, a copy's rate).  A wave takes 64 / LPH heads at a time, the
// next ones under way.
template <int DT, int LPH, bool NORM>
__global__ __launch_bounds__(kThreads) void heads_vec_kernel(HeadArgs a) {
  constexpr int HPW = 64 / LPH;
  const int lane = threadIdx.x & 63, u = lane % LPH, units = a.hd / 8;
  const int nq = a.hq, nk = a.hq + a.hkv, width = a.hq + 2 * a.hkv;
  const int step = 4 * gridDim.y * HPW;
  const int h0 = (blockIdx.y * 4 + (threadIdx.x >> 6)) * HPW + lane / LPH;
  const bool live = u < units;
  const Unit t = unit_of(a, live ? u : 0);
  f32x4 gq[2], gk[2];
  if constexpr (NORM) {
    gq[0] = *reinterpret_cast<const f32x4_a4*>(a.gq + t.e0);
    gq[1] = *reinterpret_cast<const f32x4_a4*>(a.gq + t.e1);
    gk[0] = *reinterpret_cast<const f32x4_a4*>(a.gk + t.e0);
    gk[1] = *reinterpret_cast<const f32x4_a4*>(a.gk + t.e1);
  }
  for (int64_t i = blockIdx.x; i < a.t; i += gridDim.x) {
    const float* row = a.C + i * width * a.hd;
    f32x4 n0, n1;
    auto fetch = [&](int h) {                // (past the last head: that one again)
      const float* x = row + static_cast<int64_t>(h < width ? h : width - 1) * a.hd;
      n0 = *reinterpret_cast<const f32x4_a4*>(x + t.e0);
      n1 = *reinterpret_cast<const f32x4_a4*>(x + t.e1);
    };
    fetch(h0);
    f32x4 c = {1.0f, 1.0f, 1.0f, 1.0f}, s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (t.turns) unit_angles(a, i, u, c, s);
    for (int h = h0; h - lane / LPH < width; h += step) {
      f32x4 x0 = n0, x1 = n1;
      fetch(h + step);
      if constexpr (NORM) {
        float ss = 0.0f;
        if (live) {
#pragma unroll
          for (int e = 0; e < 4; ++e) ss += x0[e] * x0[e] + x1[e] * x1[e];
        }
        const float r = 1.0f / sqrtf(head_sum<LPH>(ss) / static_cast<float>(a.hd) + a.eps);
        if (h < nk) {
          x0 *= r * (h < nq ? gq[0] : gk[0]);
          x1 *= r * (h < nq ? gq[1] : gk[1]);
        }
      }
      if (h < nk && t.turns) turn(a.inter, c, s, x0, x1);
      if (!live || h >= width) continue;
      uint16_t* y = h < nq   ? a.q + (i * a.hq + h) * a.hd
                    : h < nk ? a.k + (i * a.hkv + h - nq) * a.hd
                             : a.v + (i * a.hkv + h - nk) * a.hd;
      put4<DT>(y + t.e0, x0);
      put4<DT>(y + t.e1, x1);
    }
  }
}

// The backward pass likewise; a lane sums its entries of the gains' gradients over all its heads, the
// work-group's lanes meet in LDS at the end.  4096 x 48 x 128: 42 us, 4.4 TB/s (157 us in the kernel for
// any size); bound by memory and the two sums across lanes per head.
template <int DT, int LPH, bool NORM>
__global__ __launch_bounds__(kThreads, 4) void heads_grad_vec_kernel(HeadArgs a) {
  constexpr int HPW = 64 / LPH;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, u = lane % LPH, units = a.hd / 8;
  const int nq = a.hq, nk = a.hq + a.hkv, width = a.hq + 2 * a.hkv;
  const int h0 = wave * HPW + lane / LPH;
  const bool live = u < units;
  const Unit t = unit_of(a, live ? u : 0);
  f32x4 gq[2], gk[2], dq[2] = {}, dk[2] = {};
  if constexpr (NORM) {
    gq[0] = *reinterpret_cast<const f32x4_a4*>(a.gq + t.e0);
    gq[1] = *reinterpret_cast<const f32x4_a4*>(a.gq + t.e1);
    gk[0] = *reinterpret_cast<const f32x4_a4*>(a.gk + t.e0);
    gk[1] = *reinterpret_cast<const f32x4_a4*>(a.gk + t.e1);
  }
  for (int64_t i = blockIdx.x; i < a.t; i += gridDim.x) {
    f32x4 n0 = {}, n1 = {};
    u16x4 m0, m1;
    auto fetch = [&](int h_) {               // (past the last head: that one again; C has no use in v)
      const int h = h_ < width ? h_ : width - 1;
      const uint16_t* dy = h < nq   ? a.dq + (i * a.hq + h) * a.hd
                           : h < nk ? a.dk + (i * a.hkv + h - nq) * a.hd
                                    : a.dv + (i * a.hkv + h - nk) * a.hd;
      m0 = *reinterpret_cast<const u16x4_a2*>(dy + t.e0);
      m1 = *reinterpret_cast<const u16x4_a2*>(dy + t.e1);
      if constexpr (NORM) {
        const float* x = a.C + (i * width + (h < nk ? h : nk - 1)) * a.hd;
        n0 = *reinterpret_cast<const f32x4_a4*>(x + t.e0);
        n1 = *reinterpret_cast<const f32x4_a4*>(x + t.e1);
      }
    };
    fetch(h0);
    f32x4 c = {1.0f, 1.0f, 1.0f, 1.0f}, s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (t.turns) unit_angles(a, i, u, c, s);
    for (int h = h0; h - lane / LPH < width; h += 4 * HPW) {
      const f32x4 x0 = n0, x1 = n1;
      const u16x4 y0 = m0, y1 = m1;
      fetch(h + 4 * HPW);
      f32x4 u0, u1;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        u0[e] = from_half<DT>(y0[e]);
        u1[e] = from_half<DT>(y1[e]);
      }
      if (h < nk && t.turns) turn(a.inter, c, -s, u0, u1);
      if constexpr (NORM) {
        const f32x4 g0 = h < nq ? gq[0] : gk[0], g1 = h < nq ? gq[1] : gk[1];
        float ss = 0.0f, xu = 0.0f;
        if (live) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            ss += x0[e] * x0[e] + x1[e] * x1[e];
            xu += x0[e] * g0[e] * u0[e] + x1[e] * g1[e] * u1[e];
          }
        }
        const float n = static_cast<float>(a.hd);
        const float r = 1.0f / sqrtf(head_sum<LPH>(ss) / n + a.eps);
        const float f = r * r * head_sum<LPH>(xu) / n;
        if (h < nk) {
          const f32x4 d0 = u0 * x0 * r, d1 = u1 * x1 * r;
          if (h < nq) {
            dq[0] += d0;
            dq[1] += d1;
          } else {
            dk[0] += d0;
            dk[1] += d1;
          }
          u0 = r * (g0 * u0 - x0 * f);
          u1 = r * (g1 * u1 - x1 * f);
        }
      }
      if (!live || h >= width) continue;
      uint16_t* dx = a.dC + (i * width + h) * a.hd;
      if (h < nk) {
        put4<DT>(dx + t.e0, u0);
        put4<DT>(dx + t.e1, u1);
      } else {
        *reinterpret_cast<u16x4_a2*>(dx + t.e0) = y0;
        *reinterpret_cast<u16x4_a2*>(dx + t.e1) = y1;
      }
    }
  }
  if constexpr (NORM) {
    __shared__ float sums[4][2][kMaxHead];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        f32x4 d = w == 0 ? dq[b] : dk[b];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
          for (int o = LPH; o < 64; o <<= 1) d[e] += __shfl_xor(d[e], o, 64);
          if (live && lane < LPH) sums[wave][w][(b == 0 ? t.e0 : t.e1) + e] = d[e];
        }
      }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * a.hd; e += kThreads) {
      const int w = e / a.hd, j = e % a.hd;
      a.part[static_cast<int64_t>(e) * a.groups + blockIdx.x] =
          (sums[0][w][j] + sums[1][w][j]) + (sums[2][w][j] + sums[3][w][j]);
    }
  }
}

// Any head size: one token per work-group, one head per wave at a time.
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
    a.part[static_cast<int64_t>(e) * a.groups + blockIdx.x] =
        (sums[0][w][j] + sums[1][w][j]) + (sums[2][w][j] + sums[3][w][j]);
  }
}

// The gains' gradients: the work-groups' sums, one entry per work-group.
__global__ __launch_bounds__(kThreads) void gains_kernel(HeadArgs a) {
  __shared__ double sums[kThreads / 64];
  const float* p = a.part + static_cast<int64_t>(blockIdx.x) * a.groups;
  double s = 0.0;
#pragma unroll 4
  for (int g = threadIdx.x; g < a.groups; g += kThreads) s += p[g];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    const int e = blockIdx.x;
    (e < a.hd ? a.dgq[e] : a.dgk[e - a.hd]) = static_cast<float>((sums[0] + sums[1]) + (sums[2] + sums[3]));
  }
}

// ---- host ------------------------------------------------------------------------------------

// Whole groups: what the vector kernels take.
bool whole(int hd, int rd) { return hd % 8 == 0 && rd % 8 == 0; }

template <int DT, int LPH>
hipError_t launch_vec(const HeadArgs& a, bool backward, dim3 grid, hipStream_t st) {
  if (backward) {
    if (a.gq != nullptr) return launch_k(heads_grad_vec_kernel<DT, LPH, true>, grid, dim3(kThreads), 0, st, nullptr, nullptr, a);
    return launch_k(heads_grad_vec_kernel<DT, LPH, false>, grid, dim3(kThreads), 0, st, nullptr, nullptr, a);
  }
  if (a.gq != nullptr) return launch_k(heads_vec_kernel<DT, LPH, true>, grid, dim3(kThreads), 0, st, nullptr, nullptr, a);
  return launch_k(heads_vec_kernel<DT, LPH, false>, grid, dim3(kThreads), 0, st, nullptr, nullptr, a);
}

int lanes_of(int hd) { return hd <= 64 ? 8 : hd <= 128 ? 16 : hd <= 256 ? 32 : 64; }

template <int DT>
hipError_t launch_heads(const HeadArgs& a, bool backward, bool vec, dim3 grid, hipStream_t st) {
  if (!vec) {
    if (backward) return launch_k(heads_grad_kernel<DT>, grid, dim3(kThreads), 0, st, nullptr, nullptr, a);
    return launch_k(heads_kernel<DT>, grid, dim3(kThreads), 0, st, nullptr, nullptr, a);
  }
  switch (lanes_of(a.hd)) {
    case 8: return launch_vec<DT, 8>(a, backward, grid, st);
    case 16: return launch_vec<DT, 16>(a, backward, grid, st);
    case 32: return launch_vec<DT, 32>(a, backward, grid, st);
    default: return launch_vec<DT, 64>(a, backward, grid, st);
  }
}

bool heads_dims(int64_t t, int hq, int hkv, int hd) {
  return t >= 0 && t < kDimLimit && hq >= 1 && hkv >= 1 && hd >= 1 && hd <= kMaxHead &&
         hq <= 65536 && hkv <= 65536 &&
         static_cast<double>(t) * (hq + 2.0 * hkv) * hd <= 1099511627776.0;
}

// Work-groups of the backward pass: 4 per compute unit, as many as are resident (44 us at 4096 tokens;
// 2 take 52 us, 8 take 47).
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
  // eps is held in FP32.  Below its normal numbers it would vanish, and a head of zeros with it become NaN, or
  // the square of its reciprocal root pass FP32.
  if (gq != nullptr && !(eps == 0.0 || (eps >= FLT_MIN && eps <= FLT_MAX))) {
    return bad(FPSK_EINVAL, "eps must be zero or a positive normal number of FP32");
  }
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
  const bool vec = whole(hd, rd);
  dim3 grid(static_cast<unsigned>(std::min<int64_t>(t, 1 << 20)));
  if (vec && t < 2 * cus) {
    // few tokens: a work-group for every round of heads, up to 2 for each compute unit (48 heads at 48
    // tokens: 5.4 us with one work-group a token, 4.1 with three; at 500 tokens 7.2 and 8.7)
    const int rounds = (hq + 2 * hkv + 4 * (64 / lanes_of(hd)) - 1) / (4 * (64 / lanes_of(hd)));
    grid.y = static_cast<unsigned>(std::max<int64_t>(1, std::min<int64_t>(rounds, 2 * cus / t)));
  }
  return launched(dtype == FPSK_BF16 ? launch_heads<1>(a, false, vec, grid, st)
                                     : launch_heads<0>(a, false, vec, grid, st),
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
    const bool vec = whole(hd, rd);
    e = dtype == FPSK_BF16 ? launch_heads<1>(a, true, vec, grid, st) : launch_heads<0>(a, true, vec, grid, st);
  }
  if (e == hipSuccess && norm) {
    e = launch_k(gains_kernel, dim3(static_cast<unsigned>(2 * hd)), dim3(kThreads), 0, st, nullptr, nullptr, a);
  }
  return launched(e, "fpsketch_heads_grad");
}

}  // extern "C"
