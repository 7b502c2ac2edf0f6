// Shared by the operators around a delivered product (fpsk_gated.hip, fpsk_adapters.hip,
// fpsk_heads.hip): vector types of the matrix instructions, rounding to the half formats, ragged
// loads, activations, and the argument checks of their C entry points.
#pragma once

#include <cmath>
#include <cstdint>
#include <cstdio>

#include "../../include/fpsketch.h"
#include "fpsk_device.h"

namespace fpsk {

// fpsk_host.hip: keeps the detail of fpsketch_last_error and returns the status.
fpsketch_status layer_error(fpsketch_status s, const char* detail) noexcept;

typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
typedef u16x4 u16x4_a2 __attribute__((aligned(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// D += X Y on 16 x 16 x 32: lane l holds X[l % 16][8 (l / 16) + e] and Y[8 (l / 16) + e][l % 16],
// e < 8, and D[4 (l / 16) + r][l % 16], r < 4.
template <int DT>
__device__ __forceinline__ f32x4 mfma32(u32x4 x, u32x4 y, f32x4 d) {
  if constexpr (DT == 1) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x),
                                                   __builtin_bit_cast(bf16x8, y), d, 0, 0, 0);
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x),
                                                  __builtin_bit_cast(f16x8, y), d, 0, 0, 0);
  }
}

// Round to nearest even.
template <int DT>
__device__ __forceinline__ uint16_t to_half(float x) {
  if constexpr (DT == 1) {
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
  } else {
    return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x));
  }
}

template <int DT>
__device__ __forceinline__ float from_half(uint16_t h) {
  return lo_half<DT>(h);
}

template <int DT>
__device__ __forceinline__ u16x4 to_half4(float a, float b, float c, float d) {
  return u16x4{to_half<DT>(a), to_half<DT>(b), to_half<DT>(c), to_half<DT>(d)};
}

// Elements off .. off + 7 of an array of total >= 8 half words, zero from the nv-th on (nv <= 0:
// all; off may then lie outside).  One 16-byte load at element alignment without a branch: near the
// end of the array the last whole group is loaded and moved down.
__device__ __forceinline__ u32x4 load_ragged(const uint16_t* X, int64_t off, int64_t nv,
                                             int64_t total) {
  const int64_t last = total - 8, o = off < 0 || nv <= 0 ? 0 : (off < last ? off : last);
  u32x4 v = *reinterpret_cast<const u32x4_a2*>(X + o);
  const int s = nv <= 0 ? 0 : static_cast<int>(off - o);
  if (s & 1) {
    v = u32x4{(v[0] >> 16) | (v[1] << 16), (v[1] >> 16) | (v[2] << 16),
              (v[2] >> 16) | (v[3] << 16), v[3] >> 16};
  }
  if (s & 2) v = u32x4{v[1], v[2], v[3], 0u};
  if (s & 4) v = u32x4{v[2], v[3], 0u, 0u};
  return v & rag_keep(0, nv);
}

// Row-major operands streamed by one wave for itself: blocks of 16 rows, 64 k a stage, by loads that go
// straight to LDS.  Eight lanes read a row's 128-byte line; as fragments (a lane 16 bytes of its own
// row) the same bytes cost the address unit a cycle a lane, four times as many, which bounded these
// kernels at 16 bytes a cycle and compute unit.  16-byte group c of row r is kept at c ^ ((r / 2) % 8),
// so that a fragment's reads cover all banks.  Rows of whole groups on 16-byte boundaries, ld at most
// kMaxLd; k past the end reads zeros (an offset that the buffer's bounds turn into zeros).
constexpr int64_t kMaxLd = int64_t{1} << 22;
constexpr uint32_t kBound = 1u << 31, kOutside = ~15u;   // bytes of a buffer; an offset past them
constexpr int kStreamK = 64;

template <int BLOCKS>
struct WaveRows {
  static constexpr int kBytes = BLOCKS * 16 * kStreamK * 2;   // a stage
  static constexpr int kLoads = 2 * BLOCKS;
  const char* base[BLOCKS];
  uint32_t at[BLOCKS][2];
  int kk;                  // k of the lane's group in rows 0 .. 7, with bit 5 the other way in 8 .. 15

  // Block b: the 16 rows from `first` of a matrix of `rows`; rows past the end repeat the last one.
  __device__ __forceinline__ void set(int b, const uint16_t* x, int64_t first, int64_t rows, int64_t ld) {
    const int lane = threadIdx.x & 63;
    const int64_t from = first < rows ? first : rows - 1;
    base[b] = reinterpret_cast<const char*>(x + from * ld);
    kk = 8 * ((lane & 7) ^ (lane >> 4));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t r = 8 * i + (lane >> 3), in = from + r < rows ? r : rows - 1 - from;
      at[b][i] = static_cast<uint32_t>(2 * (in * ld + (kk ^ (32 * i))));
    }
  }

  __device__ __forceinline__ void load(char* lds, int64_t k0, int64_t K) const {
    const int left = static_cast<int>(K - k0 < kStreamK ? K - k0 : kStreamK);
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      const char* from = base[b] + (left > 0 ? 2 * k0 : 0);
      const __amdgpu_buffer_rsrc_t buffer =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(from), 0, kBound, 0x00027000);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            buffer, (__attribute__((address_space(3))) void*)(lds + (2 * b + i) * 1024), 16,
            (kk ^ (32 * i)) < left ? at[b][i] : kOutside, 0, 0, 0);
      }
    }
  }

  // Fragment of block b, k = 32 ks .. 32 ks + 31 of the stage.
  static __device__ __forceinline__ u32x4 frag(const char* lds, int b, int ks) {
    const int lane = threadIdx.x & 63, r = lane & 15;
    return *reinterpret_cast<const u32x4*>(lds + b * 2048 + r * 128 + (((4 * ks + (lane >> 4)) ^ (r >> 1)) << 4));
  }
};

// Waits until at most `left` of this wave's loads to LDS are under way.
template <int left>
__device__ __forceinline__ void stage_here() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(left) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// acc[i][j] += F_j X_i^T over k in [k0, k1), X_i and F_j blocks of 16 rows: a wave's own product, three
// stages in its parts of r0, r1 and r2, two of them under way.
template <int DT, int MT, int NT>
__device__ __forceinline__ void wave_product(const WaveRows<MT>& x, const WaveRows<NT>& f, char* r0, char* r1,
                                             char* r2, int64_t k0, int64_t k1, f32x4 (&acc)[MT][NT]) {
  constexpr int kLoads = WaveRows<MT>::kLoads + WaveRows<NT>::kLoads;
  auto load = [&](char* lds, int64_t k) {
    x.load(lds, k, k1);
    f.load(lds + WaveRows<MT>::kBytes, k, k1);
    __builtin_amdgcn_sched_barrier(0);
  };
  auto step = [&](char* lds, int64_t next) {
    stage_here<2 * kLoads>();
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      u32x4 fx[MT], ff[NT];
#pragma unroll
      for (int i = 0; i < MT; ++i) fx[i] = WaveRows<MT>::frag(lds, i, ks);
#pragma unroll
      for (int j = 0; j < NT; ++j) ff[j] = WaveRows<NT>::frag(lds + WaveRows<MT>::kBytes, j, ks);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = mfma32<DT>(ff[j], fx[i], acc[i][j]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    load(lds, next);                       // (the fragments are in registers)
  };
  if (k0 < k1) {
    load(r0, k0);
    load(r1, k0 + kStreamK);
    load(r2, k0 + 2 * kStreamK);
    for (int64_t k = k0; k < k1; k += 3 * kStreamK) {   // (past k1 the stages hold zeros)
      step(r0, k + 3 * kStreamK);
      step(r1, k + 4 * kStreamK);
      step(r2, k + 5 * kStreamK);
    }
  }
  stage_here<0>();                         // no load outlives the product
}

// 1 / (1 + e^-x).  The hardware's exponential and reciprocal are within a few units of FP32's last
// place, far below the half formats' half step that every result here is rounded by.
__device__ __forceinline__ float sigmoid(float x) {
  return __builtin_amdgcn_rcpf(1.0f + __expf(-x));
}

// The activations act(x) of the gated block: 0 silu x s(x); 1 gelu x Phi(x), with Phi from erfc so
// that the far negative side does not cancel; 2 its tanh form, 0.5 (1 + tanh y) = s(2 y).
constexpr float kSqrtHalf = 0.70710678118654752f;
constexpr float kGeluC = 1.5957691216057308f;     // 2 sqrt(2 / pi)
constexpr float kGeluA = 0.044715f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;

template <int ACT>
__device__ __forceinline__ float act_gate(float x) {   // act(x) = x act_gate(x)
  if constexpr (ACT == 0) return sigmoid(x);
  if constexpr (ACT == 1) return 0.5f * erfcf(-kSqrtHalf * x);
  return sigmoid(kGeluC * (x + kGeluA * x * x * x));
}

// act'(x) given s = act_gate(x).  Where s has reached 0 or 1 the second term has vanished; it is
// left out there because its factors overflow first.
template <int ACT>
__device__ __forceinline__ float act_slope(float x, float s) {
  if constexpr (ACT == 0) return (s == 0.0f || s == 1.0f) ? s : s + x * s * (1.0f - s);
  if constexpr (ACT == 1) {
    const float e = x * x;
    return e > 200.0f ? s : s + x * kInvSqrt2Pi * __expf(-0.5f * e);
  }
  return (s == 0.0f || s == 1.0f)
             ? s
             : s + x * s * (1.0f - s) * kGeluC * (1.0f + 3.0f * kGeluA * x * x);
}

// ---- host side of the entry points ---------------------------------------------------------

constexpr int64_t kDimLimit = int64_t{1} << 31;

struct Span {
  const void* p;
  int64_t bytes;
};

inline bool overlap(const Span& a, const Span& b) {
  if (a.p == nullptr || b.p == nullptr || a.bytes <= 0 || b.bytes <= 0) return false;
  const auto x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return x < y + static_cast<uintptr_t>(b.bytes) && y < x + static_cast<uintptr_t>(a.bytes);
}

// Every output clear of every input and of the other outputs.
template <int NI, int NO>
bool disjoint(const Span (&in)[NI], const Span (&out)[NO]) {
  for (int o = 0; o < NO; ++o) {
    for (int i = 0; i < NI; ++i) {
      if (overlap(out[o], in[i])) return false;
    }
    for (int p = 0; p < o; ++p) {
      if (overlap(out[o], out[p])) return false;
    }
  }
  return true;
}

inline bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

inline bool half_type(fpsketch_dtype t) { return t == FPSK_F16 || t == FPSK_BF16; }

// Multiprocessors of the current device in *cus; FPSK_ENODEV unless it is a gfx950.
fpsketch_status layer_device(int* cus) noexcept;

// The status of an operator whose launches ended with e.
inline fpsketch_status launched(hipError_t e, const char* where) noexcept {
  if (e == hipSuccess) return FPSK_OK;
  char msg[160];
  std::snprintf(msg, sizeof(msg), "%s: %s", where, hipGetErrorString(e));
  return layer_error(e == hipErrorOutOfMemory ? FPSK_ENOMEM : FPSK_EHIP, msg);
}

}  // namespace fpsk
