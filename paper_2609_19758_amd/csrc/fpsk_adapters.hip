// Low-rank adapters of many requests added to a shared projection's product (gfx950).
//
//   Y_i = out(C_i + s_a (X_i A_a^T) B_a^T),  a = index_i
//
// C (t x n FP32) is the verified product X W^T of the shared weight, A count x r x k and
// B count x n x r the adapters' factors, s their scales.  index -1: no adapter, Y_i = out(C_i).
// Any other index outside [0, count) makes the row NaN, so that it cannot pass unseen.
#include "fpsk_layers.h"

#include <algorithm>
#include <type_traits>

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
  float* V;                // splits x t x ldv: partial sums of X_i A_a^T (ldv: rank in whole groups of 4)
  int ldv;
  void* Y;
  int64_t tiles;
  int ways;                // work-groups that share a tile's adapters
  int splits;              // parts of k
  int blocks;              // rank blocks (shrink), or work-groups that share a tile's columns (expand)
};

// Both kernels take tiles of neighbouring rows as they come, in turn over the adapters that a tile's
// rows name: an adapter's factor multiplies the whole tile on the matrix cores, and only its own rows
// are kept.  The rows of a request are neighbours, so a prompt's tile names one adapter or two and no
// sorting of rows is needed before; a decode tile names up to 16, which `ways` work-groups take in turn
// (48 tokens of 24 adapters: 14.9 us, 41.0 with one work-group to a tile).  What a tile costs grows with the
// adapters it names: 256 tokens of 64 adapters take 36 us one by one and 15 us in 16 runs.
//
// each(a, mask): a the adapter (-1: none, count: invalid), mask its rows in the tile.
template <int TR, typename F>
__device__ __forceinline__ void for_adapters(const AdapterArgs& a, int64_t row0, int way, F each) {
  const int lane = threadIdx.x & 63;
  const bool live = lane < TR && row0 + lane < a.t;
  int which = live ? a.index[row0 + lane] : -1;
  if (which < -1 || which > a.count) which = a.count;
  uint64_t left = __ballot(live);
  for (int c = 0; left != 0; ++c) {
    const int b = __builtin_amdgcn_readlane(which, __builtin_ctzll(left));
    const uint64_t mask = __ballot(live && which == b);
    if (c % a.ways == way) each(b, mask);
    left &= ~mask;
  }
}

constexpr int kShrinkWaves = 4;
constexpr int kMaxSplits = 8;

// What both forms of the first product do with a work-group: a tile of 16 MT rows, a block of 16 NT
// ranks and a part of k; within it every wave a run of k.
struct ShrinkPart {
  int split, r0, way;
  int64_t row0;
};

template <int TR, int RB>
__device__ __forceinline__ ShrinkPart shrink_part(const AdapterArgs& a) {
  ShrinkPart p;
  unsigned b = blockIdx.x;
  p.split = b % a.splits;
  b /= a.splits;
  p.r0 = b % a.blocks * RB;
  b /= a.blocks;
  const auto tiles = static_cast<unsigned>(a.tiles);
  p.row0 = static_cast<int64_t>(b % tiles) * TR;
  p.way = static_cast<int>(b / tiles);     // last: most tiles name one adapter only
  return p;
}

// The waves' sums to V, rows of the adapter only.
template <int TR, int RB>
__device__ __forceinline__ void shrink_store(const AdapterArgs& a, const ShrinkPart& p, uint64_t mask,
                                             float (*red)[TR][RB + 4]) {
  for (int e = threadIdx.x; e < TR * RB; e += 64 * kShrinkWaves) {
    const int r = e / RB, c = e % RB;
    if (((mask >> r) & 1) != 0 && p.r0 + c < a.rank) {
      float v = 0.0f;
#pragma unroll
      for (int w = 0; w < kShrinkWaves; ++w) v += red[w][r][c];
      a.V[(static_cast<int64_t>(p.split) * a.t + p.row0 + r) * a.ldv + p.r0 + c] = v;
    }
  }
}

// V = X A^T, both streamed through LDS; the parts of k are added by the next kernel, in order.  Bound
// by reading X and by how few bytes of it the factor's rows leave room for under way: 4093 x 11008 at
// rank 64 takes 39 us (2.3 TB/s of X; 106 MB come from memory for 90 of X), 31.8 us where every tile names one
// adapter; more parts of k or two work-groups to every tile take longer (75.5 us for both kernels, 83.6 and
// 79.3).  48 x 4096 at rank 16, 24 adapters: 6.0 us.
template <int DT, int MT, int NT>
__global__ __launch_bounds__(64 * kShrinkWaves) void shrink_kernel(AdapterArgs a) {
  constexpr int TR = 16 * MT, RB = 16 * NT, kBytes = WaveRows<MT>::kBytes + WaveRows<NT>::kBytes;
  __shared__ __attribute__((aligned(16))) char b0[kShrinkWaves * kBytes];
  __shared__ __attribute__((aligned(16))) char b1[kShrinkWaves * kBytes];
  __shared__ __attribute__((aligned(16))) char b2[kShrinkWaves * kBytes];
  static_assert(sizeof(float) * kShrinkWaves * TR * (RB + 4) <= sizeof(b0), "the waves' sums take the place of b0");
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4;
  const ShrinkPart p = shrink_part<TR, RB>(a);
  const int64_t steps = (a.k + kStreamK - 1) / kStreamK, parts = static_cast<int64_t>(kShrinkWaves) * a.splits;
  const int64_t run = (steps + parts - 1) / parts * kStreamK, k0 = (p.split * kShrinkWaves + wave) * run;
  const int64_t k1 = k0 + run < a.k ? k0 + run : a.k;
  for_adapters<TR>(a, p.row0, p.way, [&](int which, uint64_t mask) {
    if (which < 0 || which >= a.count) return;
    WaveRows<MT> x;
    WaveRows<NT> f;
#pragma unroll
    for (int i = 0; i < MT; ++i) x.set(i, a.X, p.row0 + 16 * i, a.t, a.k);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      f.set(j, a.A + static_cast<int64_t>(which) * a.rank * a.k, p.r0 + 16 * j, a.rank, a.k);
    }
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    __syncthreads();                       // the sums of the adapter before
    wave_product<DT, MT, NT>(x, f, b0 + wave * kBytes, b1 + wave * kBytes, b2 + wave * kBytes, k0, k1, acc);
    __syncthreads();
    auto red = reinterpret_cast<float(*)[TR][RB + 4]>(b0);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        *reinterpret_cast<f32x4*>(&red[wave][16 * i + (lane & 15)][16 * j + 4 * g]) = acc[i][j];
      }
    }
    __syncthreads();
    shrink_store<TR, RB>(a, p, mask, red);
  });
}

// The same for any alignment: fragments straight from memory, a wave's 64 k per step as 32 bytes a lane,
// with the next step's loads in flight during the products.
template <int DT, int MT, int NT>
__global__ __launch_bounds__(64 * kShrinkWaves) void shrink_ragged_kernel(AdapterArgs a) {
  constexpr int TR = 16 * MT, RB = 16 * NT;
  __shared__ __attribute__((aligned(16))) float red[kShrinkWaves][TR][RB + 4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g = lane >> 4;
  const ShrinkPart p = shrink_part<TR, RB>(a);
  const int64_t row0 = p.row0;
  const int r0 = p.r0, split = p.split;
  const int64_t steps = a.k / 64;                  // whole ones

  for_adapters<TR>(a, row0, p.way, [&](int which, uint64_t mask) {
    if (which < 0 || which >= a.count) return;
    // rows and ranks past the end repeat the last one; their sums are not stored
    int64_t xo[MT], ao[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int64_t r = row0 + 16 * i + (lane & 15);
      xo[i] = (r < a.t ? r : a.t - 1) * a.k + 16 * g;
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int r = r0 + 16 * j + (lane & 15);
      ao[j] = (static_cast<int64_t>(which) * a.rank + (r < a.rank ? r : a.rank - 1)) * a.k + 16 * g;
    }
    const int64_t xall = a.t * a.k, aall = static_cast<int64_t>(a.count) * a.rank * a.k;
    u32x4 x[2][MT][2], f[2][NT][2];
    auto fetch = [&](int b, int64_t s) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t k0 = 64 * s + 8 * h;
#pragma unroll
        for (int i = 0; i < MT; ++i) x[b][i][h] = *reinterpret_cast<const u32x4_a2*>(a.X + xo[i] + k0);
#pragma unroll
        for (int j = 0; j < NT; ++j) f[b][j][h] = *reinterpret_cast<const u32x4_a2*>(a.A + ao[j] + k0);
      }
      __builtin_amdgcn_sched_barrier(0);   // (else the loads sink to where they are used)
    };
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    auto multiply = [&](int b) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
          for (int j = 0; j < NT; ++j) acc[i][j] = mfma32<DT>(f[b][j][h], x[b][i][h], acc[i][j]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    // Unconditional loads: behind a branch the compiler waits for the step ahead too.  A wave past
    // its last step reads that one again.
    const int64_t turn = split * kShrinkWaves + __builtin_amdgcn_readfirstlane(wave);
    const int64_t parts = static_cast<int64_t>(kShrinkWaves) * a.splits, run = (steps + parts - 1) / parts;
    int64_t s = turn * run < steps ? turn * run : steps, left = steps - s < run ? steps - s : run;
    if (left > 0) {
      const int64_t last = s + left - 1;
      fetch(0, s);
      for (; left > 1; left -= 2, s += 2) {
        fetch(1, s + 1);
        multiply(0);
        fetch(0, s + 2 < last ? s + 2 : last);
        multiply(1);
      }
      if (left == 1) multiply(0);
    }
    if (turn == parts - 1 && 64 * steps < a.k) {  // the broken last step
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t k0 = 64 * steps + 8 * h, nv = a.k - k0 - 16 * g;
#pragma unroll
        for (int i = 0; i < MT; ++i) x[0][i][h] = load_ragged(a.X, xo[i] + k0, nv, xall);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const u32x4 w = load_ragged(a.A, ao[j] + k0, nv, aall);
#pragma unroll
          for (int i = 0; i < MT; ++i) acc[i][j] = mfma32<DT>(w, x[0][i][h], acc[i][j]);
        }
      }
    }
    __syncthreads();                       // the sums of the adapter before
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        *reinterpret_cast<f32x4*>(&red[wave][16 * i + (lane & 15)][16 * j + 4 * g]) = acc[i][j];
      }
    }
    __syncthreads();
    shrink_store<TR, RB>(a, p, mask, red);
  });
}

constexpr int kColumns = 128;   // of a work-group at a time, 32 per wave

// A rank sum in three half words, whose sum it is with all of its 24 bits: 8 each in BF16; in FP16 11
// each, the later two 2^12 times as large, so that they are in FP16's range wherever the first is (sums are
// scaled to below 2^15 before).
constexpr int kWords = 3;
template <int DT>
constexpr float kLater = DT == 0 ? 4096.0f : 1.0f;

template <int DT>
__device__ __forceinline__ void split_words(float s, uint16_t (&w)[kWords]) {
  w[0] = to_half<DT>(s);
  const bool finite = fabsf(s) < __builtin_inff();
  // (BF16: a finite sum that would round to infinity keeps the largest number as its first word)
  if (DT == 1 && (w[0] & 0x7fffu) == 0x7f80u && finite) w[0] -= 1;
  float rest = s - from_half<DT>(w[0]);    // (exact, as is each one after it)
  rest *= kLater<DT>;
#pragma unroll
  for (int i = 1; i < kWords; ++i) {
    w[i] = finite ? to_half<DT>(rest) : uint16_t{0};
    rest -= from_half<DT>(w[i]);
  }
}

// Y = C + s V B^T on a tile of 16 MT rows.  Bound by C
// and Y, whose loads and stores are whole lines: the columns of a 32-wide block are dealt to two
// products so that a lane holds 8 neighbours of one row.  V enters the matrix cores as half words
// (split_words) against the exact factor B; in FP16 a row is first scaled by a power of two that puts its
// largest sum at 2^14, and its later words have sums of their own.  4093 x 4096 at rank 64 in FP16: 36.4 us,
// 2.8 TB/s (36.3 with two words, which lose bits; 8192 x 11008 at rank 128 207 and 198, 4096 x 4096 at rank 256 90
// and 79); 48 x 4096 at rank 16, 24 adapters, in BF16: 8.9 us (8.7).
//
// WHOLE: the rank is a multiple of 8, so that a group of 8 ranks lies in a row of B or outside.
template <int DT, int MT, bool HALF, bool WHOLE>
__global__ __launch_bounds__(kThreads) void expand_kernel(AdapterArgs a) {
  constexpr int TR = 16 * MT, PER = kThreads / TR;      // threads per row of V
  constexpr int W = kWords;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int rp = (a.rank + 31) / 32 * 32, ld = rp + 8;  // ranks as the products take them
  uint16_t* words = reinterpret_cast<uint16_t*>(smem);  // W x TR x ld
  float* back = reinterpret_cast<float*>(words + W * TR * ld);   // TR: what undoes the scaling
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4;
  unsigned b = blockIdx.x;
  const int64_t c0 = static_cast<int64_t>(b % a.blocks) * kColumns;
  b /= a.blocks;
  const int64_t row0 = static_cast<int64_t>(b % a.tiles) * TR;
  const int way = static_cast<int>(b / a.tiles);

  for_adapters<TR>(a, row0, way, [&](int which, uint64_t mask) {
    const bool mine = which >= 0 && which < a.count;
    const int64_t base = static_cast<int64_t>(which) * a.n, all = static_cast<int64_t>(a.count) * a.n * a.rank;
    float scale = 0.0f, undo[MT] = {};
    if (mine) {
      __syncthreads();                     // the V of the adapter before
      const int r = threadIdx.x / PER, p = threadIdx.x % PER;
      const bool own = ((mask >> r) & 1) != 0;
      const float* v = a.V + (own ? row0 + r : row0) * a.ldv;
      uint16_t *first = words + r * ld, *second = first + TR * ld;
      const int64_t part = a.t * a.ldv;
      float top = 0.0f;
#pragma unroll 2
      for (int c = 4 * p; c < rp; c += 4 * PER) {
        f32x4 w[kMaxSplits];               // all loads in flight, then the sum in order
#pragma unroll
        for (int q = 0; q < kMaxSplits; ++q) {
          w[q] = *reinterpret_cast<const f32x4*>(v + (q < a.splits ? q * part : 0) + (c < a.ldv ? c : 0));
        }
        f32x4 sum = w[0];
#pragma unroll
        for (int q = 1; q < kMaxSplits; ++q) {
          if (q < a.splits) sum += w[q];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (!own || c + e >= a.rank) sum[e] = 0.0f;
          if (fabsf(sum[e]) < __builtin_inff()) top = fmaxf(top, fabsf(sum[e]));
        }
        // (until the row's scale is known, the two halves of its bits in the places of its first words)
        const u32x4 bits = __builtin_bit_cast(u32x4, sum);
        *reinterpret_cast<u16x4*>(first + c) = __builtin_convertvector(bits >> 16, u16x4);
        *reinterpret_cast<u16x4*>(second + c) = __builtin_convertvector(bits & 0xffffu, u16x4);
      }
      float up = 1.0f, down = 1.0f;
      if constexpr (DT == 0) {
#pragma unroll
        for (int o = PER / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, PER));
        if (top > 0.0f) {                  // (of the finite ones: they stay in range beside an infinite one)
          int e = ilogbf(top) - 14;
          e = e < -126 ? -126 : e;
          up = ldexpf(1.0f, -e);
          down = ldexpf(1.0f, e);
        }
      }
      for (int c = 4 * p; c < rp; c += 4 * PER) {
        const u16x4 top16 = *reinterpret_cast<const u16x4*>(first + c), low16 = *reinterpret_cast<const u16x4*>(second + c);
        u16x4 word[W];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint16_t w[W];
          split_words<DT>(__uint_as_float(static_cast<uint32_t>(top16[e]) << 16 | low16[e]) * up, w);
#pragma unroll
          for (int i = 0; i < W; ++i) word[i][e] = w[i];
        }
#pragma unroll
        for (int i = 0; i < W; ++i) *reinterpret_cast<u16x4*>(first + i * TR * ld + c) = word[i];
      }
      if (p == 0) back[r] = down;
      __syncthreads();
      scale = a.scale[which];
#pragma unroll
      for (int i = 0; i < MT; ++i) undo[i] = back[16 * i + (lane & 15)];
    }

    // FULL: the wave's 32 columns all lie in the row.
    auto columns = [&](int64_t n0, auto full) {
      constexpr bool FULL = decltype(full)::value;
      u32x4 f[2];
      auto fetch = [&](int s) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          // row i of the product's 16 is column 8 (i / 4) + 4 h + i % 4 of the block
          const int64_t col = n0 + 8 * ((lane & 15) >> 2) + 4 * h + (lane & 3);
          const bool ok = (FULL || col < a.n) && s + 8 * g < a.rank;
          const int64_t at = (base + col) * a.rank + s + 8 * g;
          if constexpr (WHOLE) {
            f[h] = *reinterpret_cast<const u32x4_a2*>(a.B + (ok ? at : 0));
            if (!ok) f[h] = u32x4{0u, 0u, 0u, 0u};
          } else {
            f[h] = load_ragged(a.B, at, ok ? a.rank - s - 8 * g : 0, all);
          }
        }
      };
      if (mine) fetch(0);
      const int64_t col = n0 + 8 * g;
      f32x4 y[MT][2];
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const int64_t r = row0 + 16 * i + (lane & 15);
        const float* c = a.C + (r < a.t ? r : a.t - 1) * a.n;
        if constexpr (FULL) {              // (rows of other adapters too: they are not stored here)
          y[i][0] = *reinterpret_cast<const f32x4_a4*>(c + col);
          y[i][1] = *reinterpret_cast<const f32x4_a4*>(c + col + 4);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) y[i][e / 4][e % 4] = col + e < a.n ? c[col + e] : 0.0f;
        }
      }
      if (mine) {
        // The later words: summed over all ranks in one row of blocks, per 32 ranks in two (over all of them
        // 4093 x 4096 in FP16 takes 72 registers and 40 us, not 64 and 36; 48 tokens take 8.9 us, per 32 ranks 10.4).
        // Against an infinite entry of B they are infinite with any sign or NaN, where the first words' sum is what
        // the whole one would be.
        f32x4 acc[MT][2] = {}, later[2] = {};
        auto add_later = [&](int i) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float l = fabsf(later[e / 4][e % 4]) < __builtin_inff() ? later[e / 4][e % 4] : 0.0f;
            acc[i][e / 4][e % 4] = fmaf(l, 1.0f / kLater<DT>, acc[i][e / 4][e % 4]);
          }
        };
        for (int s = 0; s < rp; s += 32) {
          if (s > 0) fetch(s);
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            const int at = (16 * i + (lane & 15)) * ld + s + 8 * g;
            if constexpr (MT > 1) later[0] = later[1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = W - 1; w >= 0; --w) {
              const u32x4 v = *reinterpret_cast<const u32x4*>(words + w * TR * ld + at);
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                f32x4& to = w > 0 ? later[h] : acc[i][h];
                to = mfma32<DT>(f[h], v, to);
              }
            }
            if constexpr (MT > 1) add_later(i);
          }
        }
        if constexpr (MT == 1) add_later(0);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float v = acc[i][e / 4][e % 4];
            if constexpr (DT == 0) v *= undo[i];
            y[i][e / 4][e % 4] = fmaf(v, scale, y[i][e / 4][e % 4]);
          }
        }
      } else if (which >= 0) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
          for (int e = 0; e < 8; ++e) y[i][e / 4][e % 4] = __builtin_nanf("");
        }
      }
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        if (((mask >> (16 * i + (lane & 15))) & 1) == 0) continue;
        const int64_t o = (row0 + 16 * i + (lane & 15)) * a.n;
        const f32x4 u = y[i][0], v = y[i][1];
        if constexpr (HALF) {
          auto* w = static_cast<uint16_t*>(a.Y) + o;
          const u16x4 p = to_half4<DT>(u[0], u[1], u[2], u[3]), r = to_half4<DT>(v[0], v[1], v[2], v[3]);
          if (FULL) {
            const u32x2 pw = __builtin_bit_cast(u32x2, p), rw = __builtin_bit_cast(u32x2, r);
            *reinterpret_cast<u32x4_a2*>(w + col) = u32x4{pw[0], pw[1], rw[0], rw[1]};
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              if (col + e < a.n) w[col + e] = e < 4 ? p[e] : r[e - 4];
            }
          }
        } else {
          float* w = static_cast<float*>(a.Y) + o;
          if (FULL) {
            *reinterpret_cast<f32x4_a4*>(w + col) = u;
            *reinterpret_cast<f32x4_a4*>(w + col + 4) = v;
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              if (col + e < a.n) w[col + e] = e < 4 ? u[e] : v[e - 4];
            }
          }
        }
      }
    };
    // (a tile's work-groups walk its columns side by side; with a run of columns each, their lines of C
    // lie far apart at any one time: 319 against 267 us at 8192 x 11008 with 28 blocks of columns each)
    for (int64_t n0 = c0 + 32 * wave; n0 < a.n; n0 += int64_t{kColumns} * a.blocks) {
      if (n0 + 32 <= a.n) {
        columns(n0, std::true_type{});
      } else {
        columns(n0, std::false_type{});
      }
    }
  });
}

// Operands of fewer than 8 elements, which the 16-byte loads above do not fit: one output a thread.
template <int DT>
__global__ __launch_bounds__(kThreads) void tiny_kernel(AdapterArgs a, int half) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  for (int64_t o = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; o < a.t * a.n; o += step) {
    const int64_t i = o / a.n, j = o - i * a.n;
    const int which = a.index[i];
    float y = a.C[o];
    if (which >= 0 && which < a.count) {
      float s = 0.0f;
      for (int e = 0; e < a.rank; ++e) {
        const int64_t f = static_cast<int64_t>(which) * a.rank + e;
        float v = 0.0f;
        for (int64_t c = 0; c < a.k; ++c) v = fmaf(from_half<DT>(a.X[i * a.k + c]), from_half<DT>(a.A[f * a.k + c]), v);
        s = fmaf(v, from_half<DT>(a.B[(static_cast<int64_t>(which) * a.n + j) * a.rank + e]), s);
      }
      y = fmaf(a.scale[which], s, y);
    } else if (which != -1) {
      y = __builtin_nanf("");
    }
    if (half) {
      static_cast<uint16_t*>(a.Y)[o] = to_half<DT>(y);
    } else {
      static_cast<float*>(a.Y)[o] = y;
    }
  }
}

// ---- host ------------------------------------------------------------------------------------

// How the work is cut: tiles of 32 rows in long batches (each factor is then read from L2 half as
// often: 4093 tokens at rank 64 take 76 us, 92 in tiles of 16; 1500 at rank 16 24.4 and 26.6), of 16 in
// short ones (48 tokens 15.2 us, 18.3 in tiles of 32); k in up to 8 parts while the tiles do not give
// every compute unit two work-groups (4093 tokens without parts 80 us); and as many work-groups to a
// tile's adapters as that leaves room for.
struct Plan {
  int mt;                  // 16-row blocks of a tile
  int64_t tiles;
  int splits, ways, nt, rank_blocks, ldv;   // of the first product (the second's: launch_expand)
  bool direct;
};

// Work-groups to a tile's adapters, where there are `groups` with one each.
int ways_of(int mt, int64_t groups, int count, int cus) {
  const int64_t most = std::min<int64_t>(16 * mt, int64_t{count} + 2);
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(most, 2 * cus / groups)));
}

Plan plan_of(int64_t t, int64_t k, int count, int rank, bool direct, int cus) {
  Plan p;
  p.direct = direct;
  p.nt = rank <= 16 ? 1 : rank <= 32 ? 2 : 4;
  p.rank_blocks = (rank + 16 * p.nt - 1) / (16 * p.nt);
  p.ldv = (rank + 3) / 4 * 4;
  p.mt = t > 1024 ? 2 : 1;
  p.tiles = (t + 16 * p.mt - 1) / (16 * p.mt);
  const int64_t steps = (k + 63) / 64, groups = p.tiles * p.rank_blocks;
  p.splits = static_cast<int>(
      std::max<int64_t>(1, std::min<int64_t>({2 * cus / groups, steps / kShrinkWaves, int64_t{kMaxSplits}})));
  p.ways = ways_of(p.mt, groups * p.splits, count, cus);
  return p;
}

int64_t space_of(const Plan& p, int64_t t) { return int64_t{4} * p.splits * t * p.ldv; }

template <int DT, int MT, int NT>
hipError_t launch_shrink(const AdapterArgs& a, bool direct, hipStream_t st) {
  const dim3 grid(static_cast<unsigned>(a.tiles * a.ways * a.blocks * a.splits)), block(64 * kShrinkWaves);
  if (direct) {
    FPSK_LAUNCH((shrink_kernel<DT, MT, NT>), grid, block, 0, st, a);
  } else {
    FPSK_LAUNCH((shrink_ragged_kernel<DT, MT, NT>), grid, block, 0, st, a);
  }
  return hipSuccess;
}

template <int DT, int MT>
hipError_t launch_shrink(AdapterArgs a, const Plan& p, hipStream_t st) {
  a.ways = p.ways;
  a.blocks = p.rank_blocks;
  if (p.nt == 1) return launch_shrink<DT, MT, 1>(a, p.direct, st);
  if (p.nt == 2) return launch_shrink<DT, MT, 2>(a, p.direct, st);
  return launch_shrink<DT, MT, 4>(a, p.direct, st);
}

template <int DT, int MT, bool HALF, bool WHOLE>
hipError_t launch_expand(AdapterArgs a, int cus, hipStream_t st) {
  const auto kernel = expand_kernel<DT, MT, HALF, WHOLE>;
  // A work-group forms the tile's V once for all its columns: so many of them that three work-groups
  // are left for every compute unit, but no more than the rank is worth, since later work-groups even
  // out what is left at the end (8192 x 11008: rank 128 273 us without that bound, 207 us; rank 16 157
  // and 142 us; with one block each rank 256 at 4096 x 4096 takes 102 us, not 90).
  const int64_t steps = (a.n + kColumns - 1) / kColumns;
  const int64_t each = std::max<int64_t>(1, std::min<int64_t>({steps, a.tiles * steps / (3 * cus), a.rank / 32}));
  a.blocks = static_cast<int>((steps + each - 1) / each);
  a.ways = ways_of(MT, a.tiles * a.blocks, a.count, 4 * cus);
  const int rp = (a.rank + 31) / 32 * 32;
  const size_t lds = static_cast<size_t>(16 * MT) * (2 * kWords * (rp + 8) + 4);   // (at most 50816 bytes)
  const dim3 grid(static_cast<unsigned>(a.tiles * a.ways * a.blocks)), block(kThreads);
  FPSK_LAUNCH(kernel, grid, block, lds, st, a);
  return hipSuccess;
}

template <int DT, int MT>
hipError_t launch_adapters(AdapterArgs a, const Plan& p, bool half, int cus, hipStream_t st) {
  a.tiles = p.tiles;
  const hipError_t e = launch_shrink<DT, MT>(a, p, st);
  if (e != hipSuccess) return e;
  if (a.rank % 8 == 0) return half ? launch_expand<DT, MT, true, true>(a, cus, st) : launch_expand<DT, MT, false, true>(a, cus, st);
  return half ? launch_expand<DT, MT, true, false>(a, cus, st) : launch_expand<DT, MT, false, false>(a, cus, st);
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
  int cus = 0;
  if (!adapter_dims(t, k, n, count, rank) || t == 0 || layer_device(&cus) != FPSK_OK) return 0;
  return space_of(plan_of(t, k, count, rank, false, cus), t);
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
  const Plan p = plan_of(t, k, count, rank, k % 8 == 0 && k <= kMaxLd && aligned(X, 16) && aligned(A, 16), cus);
  const int64_t need = space_of(p, t);
  // work-groups of the two launches
  if (static_cast<double>(p.tiles) * p.ways * p.rank_blocks * p.splits * kThreads >= 4294967296.0 ||
      (static_cast<double>(p.tiles) * ((n + 127) / 128) + 64.0 * cus) * kThreads >= 4294967296.0) {
    return layer_error(FPSK_ESHAPE, "fpsketch_adapters: too many tiles");
  }
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
  a.ldv = p.ldv;
  a.splits = p.splits;
  a.Y = Y;
  const auto st = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (t * k < 8 || k * rank * count < 8 || n * rank * count < 8) {
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((t * n + kThreads - 1) / kThreads, 4096)));
    e = dtype == FPSK_BF16 ? launch_k(tiny_kernel<1>, grid, dim3(kThreads), 0, st, nullptr, nullptr, a, int{half})
                           : launch_k(tiny_kernel<0>, grid, dim3(kThreads), 0, st, nullptr, nullptr, a, int{half});
  } else if (dtype == FPSK_BF16) {
    e = p.mt == 2 ? launch_adapters<1, 2>(a, p, half, cus, st) : launch_adapters<1, 1>(a, p, half, cus, st);
  } else {
    e = p.mt == 2 ? launch_adapters<0, 2>(a, p, half, cus, st) : launch_adapters<0, 1>(a, p, half, cus, st);
  }
  return launched(e, "fpsketch_adapters");
}

}  // extern "C"
