// The gated feed-forward block around a delivered product (gfx950).
//
//   P = X W^T          X t x d, W 2f x d (f gate rows, then f up rows), FP32 sums
//   H = act(G) U       G = P[:, :f], U = P[:, f:], rounded once to the half format
//   dP = [dH U act'(G), dH act(G)]
//   dX = dP W, dW = dP^T X
//
// All three products are taken by mm_tile (mm_kernel, and mm_pair_kernel for two at once): a work-group takes a
// tile of the output over K in steps of 64, both operands' tiles in LDS (two buffers), every wave a part of the tile in FP32
// accumulators of the 16 x 16 x 32 matrix instruction.  An operand's tile is kept as it is stored:
//   row-major (K contiguous)   rows of 64 k, read as 16-byte fragments;
//   K-major (the product runs along the stored rows, W in dP W, both operands in dP^T X)
//                              rows of one k, read with the transposing LDS read, which gives a
//                              lane four k of one column: no operand is transposed in memory.
// The activation's operands meet in one lane (gate and up rows take turns in a tile), so H is formed from
// the accumulators while P is stored, and a verified block costs one pass over X, W, P and H.
// 4096 x 4096 x 11008 BF16 (P and H): 668 to 677 us, 1.10 PFLOP/s; a library product alone takes 693 us there.
// dX and dW at 2048 x 4096 x 11008: 683 to 690 us, 1.07 PFLOP/s (library products 355 and 319 us).
//
// Beside it: few_kernel up to 16 tokens; mm_ragged_kernel, the same tiles through registers, where operands off
// 16-byte groups are not worth the padded copies of pad_kernel; tiny_kernel where an operand has fewer than 8
// elements; and mm_sum_kernel, which adds the parts of a product whose K is cut.
#include "fpsk_layers.h"

#include <algorithm>

namespace fpsk {

namespace {

constexpr int kBK = 64;
constexpr int kFew = 16;       // tokens up to which the gated block streams W into fragments

struct MmArgs {
  const uint16_t* A;       // M x K, or K x M (K-major)
  const uint16_t* B;       // N x K, or K x N (K-major)
  int64_t M, N, K;
  int64_t lda, ldb;        // elements from row to row as stored
  int64_t f;               // gated: N = 2f
  float* out;              // M x N (gated: may be null)
  uint16_t* H;             // gated: M x f
  float* part;             // splits x M x N partial products, splits > 1
  int64_t tiles_m, tiles_n;
  int splits;
  int64_t kslice;          // k per split, a multiple of kBK
};

// One operand's tile: R rows (row-major) or columns (K-major) by kBK, loaded by NT threads.
//
// In LDS, 16-byte groups are permuted within a row so that a wave's reads spread over the banks:
// row-major group c of row r at c ^ ((r / 2) % 8) (the 16 rows of a fragment then cover all banks);
// K-major the 32-byte pair s of row k at s ^ hash(k), which separates the 8 rows that half a wave
// reads.
//
// GATE: tile rows are taken in blocks of 16, gate and up rows in turn, so that a wave holds both
// halves of the same columns of H.
template <int R, int NT, bool KM, bool GATE>
struct Tile {
  static constexpr int kLoads = R * 8 / NT;       // 16-byte groups per thread
  static constexpr int kBytes = R * kBK * 2;
  const uint16_t* X;
  int64_t ld, lim, total;
  int64_t off[kLoads];     // element offset of the group at k = 0; < 0: outside
  int kk[kLoads];          // its k

  static __device__ __forceinline__ int hash(int k) { return (k & 3) | ((k >> 1) & 4); }

  __device__ void init(const uint16_t* x, int64_t r0, int64_t rows, int64_t ld_, int64_t f,
                       int64_t total_) {
    X = x;
    ld = ld_;
    lim = rows;
    total = total_;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int L = i * NT + static_cast<int>(threadIdx.x);
      if constexpr (KM) {
        const int k = L / (R / 8), slot = L % (R / 8);
        const int c = (((slot >> 1) ^ hash(k)) << 1) | (slot & 1);
        const int64_t n = r0 + 8 * c;
        kk[i] = k;
        off[i] = n < rows ? static_cast<int64_t>(k) * ld + n : -1;
      } else {
        const int r = L >> 3, c = (L & 7) ^ ((r >> 1) & 7);
        int64_t row = r0 + r;
        bool ok = row < rows;
        if constexpr (GATE) {
          const int64_t j = r0 + ((r >> 5) << 4) + (r & 15);   // r0: the tile's first column of H
          ok = j < f;
          row = j + ((r >> 4) & 1) * f;
        }
        kk[i] = 8 * c;
        off[i] = ok ? row * ld + 8 * c : -1;
      }
    }
  }

  // Group i at k0 .. k0 + kBK (< K), zero outside.
  __device__ __forceinline__ u32x4 group(int i, int64_t k0, int64_t K) const {
    const int64_t k = k0 + kk[i];
    if constexpr (KM) {
      const int64_t o = off[i] + k0 * ld;
      const int64_t n = off[i] - static_cast<int64_t>(kk[i]) * ld;
      return load_ragged(X, o, off[i] >= 0 && k < K ? lim - n : 0, total);
    } else {
      return load_ragged(X, off[i] + k0, off[i] >= 0 ? K - k : 0, total);
    }
  }

  static __device__ __forceinline__ void put(char* lds, int i, u32x4 v) {
    *reinterpret_cast<u32x4*>(lds + (i * NT + static_cast<int>(threadIdx.x)) * 16) = v;
  }

  // Fragment of rows (columns) n0 .. n0 + 15 and k = 32 ks .. 32 ks + 31.
  static __device__ __forceinline__ u32x4 frag(const char* lds, int n0, int ks) {
    const int lane = threadIdx.x & 63;
    if constexpr (KM) {
      // (each address in one step from the array: behind a second one the compiler no longer sees
      // which buffer is read, and waits for the loads into the other)
      const int h = ((lane >> 2) & 3) | (((lane >> 4) & 1) << 2);
      const int at = (32 * ks + 8 * (lane >> 4) + ((lane & 15) >> 2)) * (2 * R) + (((n0 >> 4) ^ h) << 5) + 8 * (lane & 3);
      typedef __attribute__((address_space(3))) s16x4* lp;
      const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(lds + at)));
      const u32x2 b = __builtin_bit_cast(
          u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(lds + (at + 8 * R))));
      return u32x4{a[0], a[1], b[0], b[1]};
    } else {
      const int r = n0 + (lane & 15), c = 4 * ks + (lane >> 4);
      return *reinterpret_cast<const u32x4*>(lds + r * 128 + ((c ^ ((r >> 1) & 7)) << 4));
    }
  }
};

// A stage: the same tile filled by loads that go straight to LDS: 16-byte groups on 16-byte
// boundaries (rows a multiple of 8 long), 32-bit offsets within the tile (ld at most kMaxLd).  A
// wave's 64 groups land in order, so the permutation is in the addresses.  Rows past the end repeat
// the last one, whose products are not stored; for k past K the offset is one that the buffer's
// bounds turn into zeros.
template <int R, int NT, bool KM, bool GATE>
struct Stage {
  typedef Tile<R, NT, KM, GATE> T;
  static constexpr int kBytes = R * kBK * 2;
  static constexpr int kLoads = R * kBK / 8 / NT;
  static constexpr int kRows = 8 * NT / R;   // K-major: k rows per load
  static_assert(kLoads >= 1 && NT % 128 == 0 && (KM ? kRows : NT / 8) % 16 == 0,
                "the permutation is the same for every load");
  const char* base;        // the wave's tile at k = 0
  int64_t step;            // bytes from one k to the next
  uint32_t at[KM ? 1 : kLoads];
  uint32_t rows_on;        // K-major: bytes from one load's rows to the next's
  int kk;                  // k of the first group (K-major: kRows on with each load)

  // rows: of the matrix, or K-major its columns as stored (ld).
  __device__ void init(const uint16_t* x, int64_t r0, int64_t rows, int64_t ld, int64_t f) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), L = threadIdx.x;
    // gate or up rows: 16 tile rows each in turn, 8 to a wave
    const int64_t first = GATE ? r0 + ((wave >> 1) & 1) * f : r0;
    base = reinterpret_cast<const char*>(x + (KM ? r0 : first * ld));
    step = KM ? 2 * ld : 2;
    rows_on = static_cast<uint32_t>(2 * kRows * ld);
    if constexpr (KM) {
      kk = L / (R / 8);
      const int slot = L % (R / 8);
      const int c = (((slot >> 1) ^ T::hash(kk)) << 1) | (slot & 1);
      at[0] = static_cast<uint32_t>(2 * (kk * ld + (r0 + 8 * c < rows ? 8 * c : rows - 8 - r0)));
    } else {
      const int c = (L & 7) ^ ((L >> 4) & 7);
      kk = 8 * c;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = (i * NT + L) >> 3;
        const int64_t j = GATE ? ((r >> 5) << 4) + (r & 15) : r, lim = GATE ? f : rows;
        at[i] = static_cast<uint32_t>(2 * ((r0 + j < lim ? j : lim - 1 - r0) * ld + 8 * c));
      }
    }
  }

  // The stage at k0, zeros from K on (all of it where k0 >= K).
  __device__ __forceinline__ void load(char* lds, int64_t k0, int64_t K) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int left = static_cast<int>(K - k0 < kBK ? K - k0 : kBK);
    // (past K the base itself must not run on: nothing is read there, but it stays an address)
    const char* from = base + (left > 0 ? k0 : 0) * step;
    const __amdgpu_buffer_rsrc_t buffer =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(from), 0, kBound, 0x00027000);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int k = kk + (KM ? i * kRows : 0);
      const uint32_t o = at[KM ? 0 : i] + (KM ? i * rows_on : 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          buffer, (__attribute__((address_space(3))) void*)(lds + (i * NT + 64 * wave) * 16), 16,
          k < left ? o : kOutside, 0, 0, 0);
    }
  }
};

template <int ACT>
__device__ __forceinline__ float gate_up(float g, float u) {
  return g * act_gate<ACT>(g) * u;
}

template <int DT>
__device__ __forceinline__ float gate_up(int act, float g, float u) {
  return act == 0 ? gate_up<0>(g, u) : act == 1 ? gate_up<1>(g, u) : gate_up<2>(g, u);
}

// Four neighbours of a row of n, at column j.
__device__ __forceinline__ void store4(float* row, int64_t j, int64_t n, f32x4 v, bool vec) {
  if (vec && j + 3 < n) {
    *reinterpret_cast<f32x4*>(row + j) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (j + e < n) row[j + e] = v[e];
    }
  }
}

__device__ __forceinline__ void store4h(uint16_t* row, int64_t j, int64_t n, u16x4 v, bool vec) {
  if (vec && j + 3 < n) {
    *reinterpret_cast<u16x4*>(row + j) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (j + e < n) row[j + e] = v[e];
    }
  }
}

// Work-groups are dealt to the 8 XCDs in turn: with this order each XCD gets neighbours among `count`.
__device__ __forceinline__ uint32_t by_xcd(uint32_t b, uint32_t count) {
  const uint32_t per = count / 8;
  return b < 8 * per ? (b % 8) * per + b / 8 : b;
}

// Each XCD gets neighbouring tiles, in bands of 4 rows
// of tiles, so that its L2 holds the operands' tiles that they share (2048 x 16384 x 8192: bands of 8
// rows 468 us, of 4 rows 448; 4096 x 22016 x 4096: 16 rows 717, 4 rows 661).
__device__ __forceinline__ void tile_of(uint32_t b, uint32_t tm, uint32_t tn, uint32_t* m, uint32_t* n) {
  b = by_xcd(b, tm * tn);
  const uint32_t band = b / (4 * tn), first = 4 * band;
  const uint32_t height = tm - first < 4 ? tm - first : 4;
  const uint32_t in = b - band * 4 * tn;
  *n = in / height;
  *m = first + in - *n * height;
}

// Accumulators of a wave: BM / WM x BN / WN of the tile.
template <int DT, int BM, int BN, int WM, int WN, bool AKM, bool BKM, bool GATED>
struct Wave {
  static constexpr int NT = 64 * WM * WN;
  static constexpr int MT = BM / WM / 16, NTL = BN / WN / 16;
  typedef Tile<BM, NT, AKM, false> TA;
  typedef Tile<BN, NT, BKM, GATED> TB;
  f32x4 acc[MT][NTL];
  int wm, wn;

  __device__ void init() {
    const int wave = threadIdx.x >> 6;
    wm = (wave / WN) * (BM / WM);
    wn = (wave % WN) * (BN / WN);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
      for (int j = 0; j < NTL; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
  }

  __device__ __forceinline__ void multiply(const char* la, const char* lb) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      u32x4 fb[NTL];
#pragma unroll
      for (int j = 0; j < NTL; ++j) fb[j] = TB::frag(lb, wn + 16 * j, ks);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const u32x4 fa = TA::frag(la, wm + 16 * i, ks);
#pragma unroll
        for (int j = 0; j < NTL; ++j) acc[i][j] = mfma32<DT>(fb[j], fa, acc[i][j]);
      }
    }
  }

  // The same with a row block's fragment read two blocks ahead of its products, and the second half's
  // fragments of B during the last blocks of the first; the barriers keep the scheduler from moving
  // the reads down to their use, where the matrix cores would wait for LDS (796 -> 747 us at 4096 x
  // 4096 x 22016).
  __device__ __forceinline__ void multiply_ahead(const char* la, const char* lb) {
    static_assert(MT >= NTL && MT > 2, "");
    u32x4 fa[3], fb[2][NTL];
#pragma unroll
    for (int j = 0; j < NTL; ++j) fb[0][j] = TB::frag(lb, wn + 16 * j, 0);
    fa[0] = TA::frag(la, wm, 0);
    fa[1] = TA::frag(la, wm + 16, 0);
#pragma unroll
    for (int g = 0; g < 2 * MT; ++g) {
      const int ks = g / MT, i = g % MT, next = g + 2;
      if (next < 2 * MT) fa[next % 3] = TA::frag(la, wm + 16 * (next % MT), next / MT);
      if (ks == 0 && i >= MT - NTL) fb[1][i - (MT - NTL)] = TB::frag(lb, wn + 16 * (i - (MT - NTL)), 1);
#pragma unroll
      for (int j = 0; j < NTL; ++j) acc[i][j] = mfma32<DT>(fb[ks][j], fa[g % 3], acc[i][j]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // lane l: row l % 16, columns 4 (l / 16) .. + 3 of every 16 x 16 block
  __device__ void store(const MmArgs& a, int64_t m0, int64_t n0, int64_t split, int act) const {
    const int lane = threadIdx.x & 63;
    float* out = a.splits > 1 ? a.part + split * a.M * a.N : a.out;
    const bool vec = (a.N & 3) == 0 && (reinterpret_cast<uintptr_t>(out) & 15u) == 0 &&
                     (!GATED || (a.f & 3) == 0);
    const bool vec_h = GATED && (a.f & 3) == 0 && (reinterpret_cast<uintptr_t>(a.H) & 7u) == 0;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int64_t m = m0 + wm + 16 * i + (lane & 15);
      if (m >= a.M) continue;
      if constexpr (GATED) {
#pragma unroll
        for (int j = 0; j < NTL; j += 2) {
          const int64_t n = n0 + ((wn + 16 * j) >> 1) + 4 * (lane >> 4);
          const f32x4 g = acc[i][j], u = acc[i][j + 1];
          if (out != nullptr) {
            store4(out + m * a.N, n, a.f, g, vec);
            store4(out + m * a.N + a.f, n, a.f, u, vec);
          }
          if (a.splits == 1) {
            store4h(a.H + m * a.f, n, a.f,
                    to_half4<DT>(gate_up<DT>(act, g[0], u[0]), gate_up<DT>(act, g[1], u[1]),
                                 gate_up<DT>(act, g[2], u[2]), gate_up<DT>(act, g[3], u[3])),
                    vec_h);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < NTL; ++j) {
          store4(out + m * a.N, n0 + wn + 16 * j + 4 * (lane >> 4), a.N, acc[i][j], vec);
        }
      }
    }
  }
};

// A work-group's part of the product.
struct Part {
  int64_t m0, n0, k0, k1, split;
};

template <int BM, int BN, bool GATED>
__device__ __forceinline__ Part part_of(const MmArgs& a, uint32_t block) {
  // (32 bits: a launch has fewer work-groups, and 64-bit divisions are long)
  const auto rows = static_cast<uint32_t>(a.tiles_m), cols = static_cast<uint32_t>(a.tiles_n);
  const uint32_t split = block / (rows * cols);
  uint32_t tm, tn;
  tile_of(block - split * rows * cols, rows, cols, &tm, &tn);
  Part p;
  p.split = split;
  p.m0 = static_cast<int64_t>(tm) * BM;
  p.n0 = static_cast<int64_t>(tn) * (GATED ? BN / 2 : BN);
  p.k0 = p.split * a.kslice;
  p.k1 = p.k0 + a.kslice < a.K ? p.k0 + a.kslice : a.K;
  return p;
}

// Any alignment: the operands' tiles pass through registers, whose loads are two to four instructions a
// group (worth_copies has the times of both kernels).
template <int DT, int BM, int BN, int WM, int WN, bool AKM, bool BKM, bool GATED>
__global__ __launch_bounds__(64 * WM * WN, 2) void mm_ragged_kernel(MmArgs a, int act) {
  typedef Wave<DT, BM, BN, WM, WN, AKM, BKM, GATED> W;
  typedef typename W::TA TA;
  typedef typename W::TB TB;
  __shared__ __attribute__((aligned(16))) char lds_a[2][TA::kBytes];
  __shared__ __attribute__((aligned(16))) char lds_b[2][TB::kBytes];
  const Part p = part_of<BM, BN, GATED>(a, blockIdx.x);
  TA ta;
  TB tb;
  ta.init(a.A, p.m0, a.M, AKM ? a.M : a.K, 0, a.M * a.K);
  tb.init(a.B, p.n0, a.N, BKM ? a.N : a.K, a.f, a.N * a.K);
  W w;
  w.init();
  u32x4 ra[TA::kLoads], rb[TB::kLoads];
  auto fetch = [&](int64_t k) {
#pragma unroll
    for (int i = 0; i < TA::kLoads; ++i) ra[i] = ta.group(i, k, p.k1);
#pragma unroll
    for (int i = 0; i < TB::kLoads; ++i) rb[i] = tb.group(i, k, p.k1);
  };
  auto keep = [&](int buf) {
#pragma unroll
    for (int i = 0; i < TA::kLoads; ++i) TA::put(lds_a[buf], i, ra[i]);
#pragma unroll
    for (int i = 0; i < TB::kLoads; ++i) TB::put(lds_b[buf], i, rb[i]);
  };
  int buf = 0;
  if (p.k0 < p.k1) {
    fetch(p.k0);
    keep(0);
  }
  for (int64_t k = p.k0; k < p.k1; k += kBK) {
    __syncthreads();
    const bool more = k + kBK < p.k1;
    if (more) fetch(k + kBK);
    w.multiply(lds_a[buf], lds_b[buf]);
    if (more) keep(buf ^ 1);
    buf ^= 1;
  }
  w.store(a, p.m0, p.n0, p.split, act);
}

// Waits until at most `left` of this wave's loads to LDS are under way, then for the work-group.
template <int left>
__device__ __forceinline__ void stages_ready() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(left) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Whole 16-byte groups, two buffers of 64 k: the next step's loads are under way during this one's
// products.  A buffer is an array of its own, so that the compiler knows loads into one apart from
// reads of the other.  A step of a 256 x 256 tile takes 1.66 us, a rate of 1.29 PFLOP/s (a library product of 8192
// x 8192 x 8192 reaches 1.23 to FP32).  By the counters at 4096 x 22016 x 4096 a compute unit has work for 88 % of
// the launch (6 rounds of work-groups for 5.4), and then its matrix cores are busy for 57 % of the time and LDS for
// 21 %, without bank conflicts: no unit is full, the steps wait for their loads at the barriers.  There,
// loads spread between the products take longer (670 -> 735 us), as do non-temporal stores (674 -> 680)
// and tiles of the last round in halves (667 -> 676).
template <int DT, int BM, int BN, int WM, int WN, bool AKM, bool BKM, bool GATED>
__device__ __forceinline__ void mm_tile(const MmArgs& a, int act, uint32_t block, char* a0, char* b0,
                                        char* a1, char* b1) {
  typedef Wave<DT, BM, BN, WM, WN, AKM, BKM, GATED> W;
  typedef Stage<BM, W::NT, AKM, false> SA;
  typedef Stage<BN, W::NT, BKM, GATED> SB;
  const Part p = part_of<BM, BN, GATED>(a, block);
  SA sa;
  SB sb;
  sa.init(a.A, p.m0, AKM ? a.lda : a.M, a.lda, 0);
  sb.init(a.B, p.n0, BKM ? a.ldb : a.N, a.ldb, a.f);
  W w;
  w.init();
  auto load = [&](char* la, char* lb, int64_t k) {
    sa.load(la, k, p.k1);
    sb.load(lb, k, p.k1);
    __builtin_amdgcn_sched_barrier(0);     // (else the loads sink to the end of the products)
  };
  load(a0, b0, p.k0);
  int64_t k = p.k0;
  for (; k + kBK < p.k1; k += 2 * kBK) {   // (loads past K fill a buffer with zeros)
    stages_ready<0>();
    load(a1, b1, k + kBK);
    w.multiply_ahead(a0, b0);
    stages_ready<0>();
    load(a0, b0, k + 2 * kBK);
    w.multiply_ahead(a1, b1);
  }
  stages_ready<0>();                       // no load outlives the kernel
  if (k < p.k1) w.multiply_ahead(a0, b0);
  w.store(a, p.m0, p.n0, p.split, act);
}

template <int DT, int BM, int BN, int WM, int WN, bool AKM, bool BKM, bool GATED>
__global__ __launch_bounds__(64 * WM * WN, 2) void mm_kernel(MmArgs a, int act) {
  __shared__ __attribute__((aligned(16))) char a0[BM * kBK * 2];
  __shared__ __attribute__((aligned(16))) char b0[BN * kBK * 2];
  __shared__ __attribute__((aligned(16))) char a1[BM * kBK * 2];
  __shared__ __attribute__((aligned(16))) char b1[BN * kBK * 2];
  mm_tile<DT, BM, BN, WM, WN, AKM, BKM, GATED>(a, act, blockIdx.x, a0, b0, a1, b1);
}

// dX and dW in one launch: tiles of 128 x 128 are taken where they do not fill the chip for long, and
// two launches would leave it part empty twice (1000 x 512 x 1024: 32 us in two, 20 us; 333 x 1000 x
// 2731 with its padded copies: 36 and 28 us).
template <int DT>
__global__ __launch_bounds__(256, 2) void mm_pair_kernel(MmArgs dx, MmArgs dw, uint32_t first) {
  __shared__ __attribute__((aligned(16))) char a0[128 * kBK * 2];
  __shared__ __attribute__((aligned(16))) char b0[128 * kBK * 2];
  __shared__ __attribute__((aligned(16))) char a1[128 * kBK * 2];
  __shared__ __attribute__((aligned(16))) char b1[128 * kBK * 2];
  if (blockIdx.x < first) {
    mm_tile<DT, 128, 128, 2, 2, false, true, false>(dx, 0, blockIdx.x, a0, b0, a1, b1);
  } else {
    mm_tile<DT, 128, 128, 2, 2, true, true, false>(dw, 0, blockIdx.x - first, a0, b0, a1, b1);
  }
}

// Up to 16 tokens: bound by reading W once.  A work-group takes 16 columns of H and all tokens; each
// wave streams a run of k of its gate rows, up rows and tokens, and the waves' sums meet in LDS.
// 1 x 4096 x 11008: 32.4 us, 5.6 TB/s of W; 16 tokens: 36 us, 48 us in mm_kernel, which keeps fewer
// bytes under way (17 tokens: 48 us).
template <int DT>
__global__ __launch_bounds__(kThreads) void few_kernel(MmArgs a, int act) {
  constexpr int kWaves = kThreads / 64, kBytes = WaveRows<1>::kBytes + WaveRows<2>::kBytes;
  __shared__ __attribute__((aligned(16))) char r0[kWaves * kBytes];
  __shared__ __attribute__((aligned(16))) char r1[kWaves * kBytes];
  __shared__ __attribute__((aligned(16))) char r2[kWaves * kBytes];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4;
  const int64_t j0 = static_cast<int64_t>(blockIdx.x) * 16;
  WaveRows<1> x;
  WaveRows<2> w;
  x.set(0, a.A, 0, a.M, a.lda);
  w.set(0, a.B, j0, a.f, a.ldb);
  w.set(1, a.B + a.f * a.ldb, j0, a.f, a.ldb);
  f32x4 acc[1][2] = {};
  const int64_t steps = (a.K + kStreamK - 1) / kStreamK, run = (steps + kWaves - 1) / kWaves * kStreamK;
  const int64_t k0 = wave * run, k1 = k0 + run < a.K ? k0 + run : a.K;
  wave_product<DT, 1, 2>(x, w, r0 + wave * kBytes, r1 + wave * kBytes, r2 + wave * kBytes, k0, k1, acc);
  __syncthreads();
  static_assert(sizeof(float) * kWaves * kFew * 36 <= sizeof(r0), "the waves' sums take the place of r0");
  auto red = reinterpret_cast<float(*)[kFew][36]>(r0);
#pragma unroll
  for (int u = 0; u < 2; ++u) *reinterpret_cast<f32x4*>(&red[wave][lane & 15][16 * u + 4 * g]) = acc[0][u];
  __syncthreads();
  const int r = threadIdx.x / 16, c = threadIdx.x % 16;
  if (r >= a.M || j0 + c >= a.f) return;
  float gate = 0.0f, up = 0.0f;
#pragma unroll
  for (int v = 0; v < kWaves; ++v) {
    gate += red[v][r][c];
    up += red[v][r][16 + c];
  }
  if (a.out != nullptr) {
    a.out[r * a.N + j0 + c] = gate;
    a.out[r * a.N + a.f + j0 + c] = up;
  }
  a.H[r * a.f + j0 + c] = to_half<DT>(gate_up<DT>(act, gate, up));
}

// A product with an operand of fewer than 8 elements, which 16-byte loads do not fit: one output
// (gated: one of H) a thread.  sa, sb: strides of A and B along k, ra, rb along their rows.
template <int DT, bool GATED>
__global__ __launch_bounds__(kThreads) void tiny_kernel(MmArgs a, int64_t ra, int64_t sa, int64_t rb,
                                                        int64_t sb, int act) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  const int64_t cols = GATED ? a.f : a.N;
  for (int64_t o = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; o < a.M * cols; o += step) {
    const int64_t m = o / cols, n = o - m * cols;
    float v[2] = {0.0f, 0.0f};
    for (int h = 0; h < (GATED ? 2 : 1); ++h) {
      for (int64_t k = 0; k < a.K; ++k) {
        v[h] = fmaf(from_half<DT>(a.A[m * ra + k * sa]), from_half<DT>(a.B[(n + h * a.f) * rb + k * sb]), v[h]);
      }
      if (a.out != nullptr) a.out[m * a.N + n + h * a.f] = v[h];
    }
    if constexpr (GATED) a.H[o] = to_half<DT>(gate_up<DT>(act, v[0], v[1]));
  }
}

// Copies with rows padded by zeros to whole 16-byte groups, for the loads that go straight to LDS: up
// to three matrices in one launch, a group a thread.
struct PadArgs {
  const uint16_t* src[3];
  uint16_t* dst[3];
  int64_t rows[3], cols[3];
};

__device__ __host__ inline int64_t padded(int64_t cols) { return (cols + 7) / 8 * 8; }

__global__ __launch_bounds__(kThreads) void pad_kernel(PadArgs a) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  for (int m = 0; m < 3; ++m) {
    const int64_t groups = padded(a.cols[m]) / 8, total = a.rows[m] * a.cols[m];
    for (int64_t o = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; o < a.rows[m] * groups; o += step) {
      const int64_t r = o / groups, c = 8 * (o - r * groups);
      u32x4 v = {0u, 0u, 0u, 0u};
      if (total >= 8) {
        v = load_ragged(a.src[m], r * a.cols[m] + c, a.cols[m] - c, total);
      } else {
        for (int e = 0; e < 8; ++e) {
          if (c + e < a.cols[m]) {
            v[e / 2] |= static_cast<uint32_t>(a.src[m][r * a.cols[m] + c + e]) << (16 * (e & 1));
          }
        }
      }
      *reinterpret_cast<u32x4*>(a.dst[m] + 8 * o) = v;
    }
  }
}

// The sum of the partial products in the order of the splits: V neighbours a thread (gated: of H, and
// the same of both halves of P).  V = 4 where rows are whole groups of 4.
template <int V>
__device__ __forceinline__ void add_parts(const MmArgs& a, int64_t at, float (&v)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = 0.0f;
  const int64_t size = a.M * a.N;
#pragma unroll 4
  for (int s = 0; s < a.splits; ++s) {
    const float* p = a.part + s * size + at;
    if constexpr (V == 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += x[e];
    } else {
      v[0] += p[0];
    }
  }
}

template <int V>
__device__ __forceinline__ void put_floats(float* to, const float (&v)[V]) {
  if constexpr (V == 4) {
    *reinterpret_cast<f32x4_a4*>(to) = f32x4{v[0], v[1], v[2], v[3]};
  } else {
    to[0] = v[0];
  }
}

template <int DT, bool GATED, int V>
__global__ __launch_bounds__(kThreads) void mm_sum_kernel(MmArgs a, int act) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  const int64_t cols = GATED ? a.f : a.N, count = a.M * cols / V;
  for (int64_t o = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; o < count; o += step) {
    if constexpr (GATED) {
      const int64_t m = V * o / cols, at = m * a.N + (V * o - m * cols);
      float g[V], u[V];
      add_parts<V>(a, at, g);
      add_parts<V>(a, at + a.f, u);
      if (a.out != nullptr) {
        put_floats<V>(a.out + at, g);
        put_floats<V>(a.out + at + a.f, u);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) a.H[V * o + e] = to_half<DT>(gate_up<DT>(act, g[e], u[e]));
    } else {
      float v[V];
      add_parts<V>(a, V * o, v);
      put_floats<V>(a.out + V * o, v);
    }
  }
}

// H = act(G) U from a delivered product, one element a thread: bound by reading P and writing H (2048 x
// 11008: 45.8 us, 4.9 TB/s of a copy's 5.15).
template <int DT>
__global__ __launch_bounds__(kThreads) void narrow_kernel(const float* P, int64_t t, int64_t f,
                                                          int act, uint16_t* H) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * kThreads;
  for (int64_t o = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; o < t * f; o += step) {
    const int64_t m = o / f, at = 2 * m * f + (o - m * f);
    H[o] = to_half<DT>(gate_up<DT>(act, P[at], P[at + f]));
  }
}

template <int ACT>
__device__ __forceinline__ void grads(float g, float u, float dh, float* dg, float* du) {
  const float s = act_gate<ACT>(g);
  *dg = dh * u * act_slope<ACT>(g, s);
  *du = dh * g * s;
}

// dP of a 64 x 64 block of H: bound by its loads and stores (14 bytes an entry of H, 18 with the
// transpose).  A thread takes 4 x 4 entries, all loads at once, and turns them in registers for the
// transpose, whose rows then leave LDS as whole lines.  2048 x 11008 with the transpose: 84 us, 4.8
// TB/s of a copy's 5.15; 1531 x 13824, whose transposed rows begin inside lines: 83 us, 4.6 TB/s (without
// the transpose 56 us, 5.3 TB/s).  Strips of tokens whose lines meet in LDS are no faster (99 us), nor
// blocks of 128 tokens (105).
//
// Blocks are taken in bands of `band` columns of blocks, down a band; xcd: neighbours on one XCD.
template <int DT, int ACT>
__global__ __launch_bounds__(kThreads) void grad_kernel(const uint16_t* dH, const float* P, int64_t t,
                                                        int64_t f, uint16_t* dP, uint16_t* dPt,
                                                        uint32_t blocks_t, uint32_t band, bool xcd) {
  constexpr int kEdge = 64;
  __shared__ __attribute__((aligned(16))) uint16_t tile[2][kEdge][kEdge + 4];   // columns x tokens
  const uint32_t blocks_f = gridDim.x / blocks_t, b = xcd ? by_xcd(blockIdx.x, gridDim.x) : blockIdx.x;
  const uint32_t first = b / (band * blocks_t) * band, width = blocks_f - first < band ? blocks_f - first : band;
  const uint32_t in = b - first * blocks_t, m = in / width;
  const int64_t m0 = static_cast<int64_t>(m) * kEdge, j0 = static_cast<int64_t>(first + in - m * width) * kEdge;
  const int x = 4 * (threadIdx.x & 15), y = 4 * (threadIdx.x >> 4);
  const bool whole = j0 + x + 3 < f;       // (tokens past the last one: that one again, not stored)
  f32x4 g[4], u[4];
  u16x4 h[4];
  if (whole) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t m = m0 + y + r < t ? m0 + y + r : t - 1, at = 2 * m * f + j0 + x;
      g[r] = *reinterpret_cast<const f32x4_a4*>(P + at);
      u[r] = *reinterpret_cast<const f32x4_a4*>(P + at + f);
      h[r] = *reinterpret_cast<const u16x4_a2*>(dH + m * f + j0 + x);
    }
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t m = m0 + y + r < t ? m0 + y + r : t - 1, j = j0 + x + e;
        g[r][e] = j < f ? P[2 * m * f + j] : 0.0f;
        u[r][e] = j < f ? P[2 * m * f + f + j] : 0.0f;
        h[r][e] = j < f ? dH[m * f + j] : uint16_t{0};
      }
    }
  }
  u16x4 hg[4], hu[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float dg, du;
      grads<ACT>(g[r][e], u[r][e], from_half<DT>(h[r][e]), &dg, &du);
      hg[r][e] = to_half<DT>(dg);
      hu[r][e] = to_half<DT>(du);
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int64_t m = m0 + y + r, at = 2 * m * f + j0 + x;
    if (m >= t) continue;
    if (whole) {
      *reinterpret_cast<u16x4_a2*>(dP + at) = hg[r];
      *reinterpret_cast<u16x4_a2*>(dP + at + f) = hu[r];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (j0 + x + e < f) {
          dP[at + e] = hg[r][e];
          dP[at + f + e] = hu[r][e];
        }
      }
    }
  }
  if (dPt == nullptr) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    *reinterpret_cast<u16x4*>(&tile[0][x + e][y]) = u16x4{hg[0][e], hg[1][e], hg[2][e], hg[3][e]};
    *reinterpret_cast<u16x4*>(&tile[1][x + e][y]) = u16x4{hu[0][e], hu[1][e], hu[2][e], hu[3][e]};
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int half = i & 1, c = (threadIdx.x >> 4) + 16 * (i >> 1);
    const u16x4 v = *reinterpret_cast<const u16x4*>(&tile[half][c][x]);
    const int64_t j = j0 + c, m = m0 + x;
    if (j >= f) continue;
    uint16_t* to = dPt + (j + half * f) * t + m;
    if (m + 3 < t) {
      *reinterpret_cast<u16x4_a2*>(to) = v;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (m + e < t) to[e] = v[e];
      }
    }
  }
}

template <int DT>
hipError_t launch_grad(const uint16_t* dH, const float* P, int64_t t, int64_t f, int act, uint16_t* dP,
                       uint16_t* dPt, hipStream_t st) {
  const auto bt = static_cast<uint32_t>((t + 63) / 64), bf = static_cast<uint32_t>((f + 63) / 64);
  const bool odd_t = dPt != nullptr && (t % 64 != 0 || !aligned(dPt, 128)), odd_f = f % 64 != 0 || !aligned(dP, 128);
  // Where rows do not begin on 128-byte lines, neighbours share lines, which are written once if they meet in
  // one L2: columns of blocks one after the other per XCD for the transpose's rows (1531 x 13824: 99 us in
  // rows of blocks, 83), rows of blocks for dP's (1024 x 13001: 67 and 55), bands of 8 columns for both
  // (1000 x 13001: 79 and 61).  On lines, rows of blocks over all XCDs (1536 x 13824: 76, 80 in columns).
  const uint32_t band = odd_t ? (odd_f ? 8 : 1) : bf;
  const dim3 grid(bf * bt);
  if (act == FPSK_SILU) FPSK_LAUNCH((grad_kernel<DT, 0>), grid, dim3(kThreads), 0, st, dH, P, t, f, dP, dPt, bt, band, odd_t || odd_f);
  if (act == FPSK_GELU) FPSK_LAUNCH((grad_kernel<DT, 1>), grid, dim3(kThreads), 0, st, dH, P, t, f, dP, dPt, bt, band, odd_t || odd_f);
  if (act == FPSK_GELU_TANH) FPSK_LAUNCH((grad_kernel<DT, 2>), grid, dim3(kThreads), 0, st, dH, P, t, f, dP, dPt, bt, band, odd_t || odd_f);
  return hipSuccess;
}

// ---- host ------------------------------------------------------------------------------------

// How a product is cut: tiles of 256 x 256 (one work-group a compute unit) or 128 x 128 (two), and K
// in parts where the tiles alone would leave compute units idle.
struct Cut {
  bool big, direct, few;
  int64_t tiles_m, tiles_n, kslice;
  int splits;
};

// Microseconds that a product of M x N takes in `tiles` tiles and `splits` parts of `per` steps, by
// what the kernels measure: a step of 64 k takes 1.66 us in a tile of 256, 1.1 us in two of 128 side by
// side and 0.6 us in one alone (2.8 and 2.35 us through registers, where it waits for its own loads); a
// round of work-groups begins and ends in 5 and 3 us; operands come from memory at 4.3 TB/s, 3.4 with a
// single tile of 128 per compute unit; and parts are written, read and added at 5 TB/s in a launch of 3 us.
// (4096 x 22016 x 4096: 667 us, measured 672; 500 x 22016 x 4096: 111 and 110, where 256-tiles in two parts
// take 145 and 128-tiles 144; 1000 x 8192 x 4096: 73 and 67, in 256-tiles 79 in two parts, 93 in one; 67 x
// 27648 x 5120: 75 and 72, 86 in one part; 130 x 8192 x 4095 through registers: 55 and 56, 85 in
// two parts.)
double cost(bool big, bool direct, double M, double N, double K, int64_t tiles, int64_t splits, int64_t per,
            int cus) {
  const int64_t groups = tiles * splits, slots = big ? cus : 2 * cus, rest = groups % slots;
  const double steps = static_cast<double>(per);
  const double round = big ? 1.66 * steps + 5 : (direct ? 1.1 : 2.8) * steps + 3;
  double c = static_cast<double>(groups / slots) * round;
  if (rest > 0) c += big || rest > cus ? round : (direct ? 0.6 : 2.35) * steps + 3;
  c = std::max(c, 2e-6 * K * (M + N) / (big || groups > cus ? 4.3 : 3.4));
  return splits == 1 ? c : c + 3 + 8e-6 / 5 * static_cast<double>(splits) * M * N;
}

// cols: columns of the product, or of H (two of the product each).
Cut cut_of(int64_t M, int64_t cols, bool gated, bool few, int64_t K, bool direct, int cus) {
  Cut c;
  c.direct = direct;
  c.big = false;
  c.few = few;
  c.tiles_m = 1;
  c.tiles_n = (cols + 15) / 16;
  c.kslice = K;
  c.splits = 1;
  if (few) return c;
  const int64_t steps = std::max<int64_t>(1, (K + kBK - 1) / kBK);
  double best = -1.0;
  for (const bool big : {true, false}) {
    if (big && !direct) continue;
    const int64_t edge = big ? 256 : 128, per_n = gated ? edge / 2 : edge;
    const int64_t tm = (M + edge - 1) / edge, tn = (cols + per_n - 1) / per_n;
    // up to 32 parts of at least 4 steps, while those before leave compute units free
    const int64_t most = std::min<int64_t>({32, std::max<int64_t>(1, steps / 4), 1 + 2 * cus / (tm * tn)});
    for (int64_t s = 1; s <= most; ++s) {
      const int64_t per = (steps + s - 1) / s, parts = (steps + per - 1) / per;
      const double t = cost(big, direct, static_cast<double>(M), static_cast<double>(gated ? 2 * cols : cols),
                            static_cast<double>(K), tm * tn, parts, per, cus);
      if (best >= 0.0 && t >= best) continue;
      best = t;
      c.big = big;
      c.tiles_m = tm;
      c.tiles_n = tn;
      c.kslice = per * kBK;
      c.splits = static_cast<int>(parts);
    }
  }
  return c;
}

// K in fewer parts, but two, where another product of the same launch leaves `room` work-groups only
// (500 x 2048 x 2048: 42 us with each product cut for itself, 33 us).
void fewer_parts(Cut& c, int64_t K, int64_t room) {
  const int64_t most = std::max<int64_t>(2, room / (c.tiles_m * c.tiles_n));
  if (c.splits <= most) return;
  const int64_t steps = (K + kBK - 1) / kBK, per = (steps + most - 1) / most;
  c.kslice = per * kBK;
  c.splits = static_cast<int>((steps + per - 1) / per);
}

// An operand that the loads to LDS fit as it is: rows of whole 16-byte groups on 16-byte boundaries.
bool fits(const void* p, int64_t ld) { return ld % 8 == 0 && aligned(p, 16); }

// Whether a product is worth padded copies of the `elements` that do not fit: small ones, whose copy is
// one short launch (gated 400 x 1023 x 1000: 23 us either way), and those with the work to make up for it
// (4095 x 4096: 71 against 98 us through registers at 300 tokens, but 56 and 59 us at 200, 55 and 56 at 130 and
// 43 against 31 us at 20).
bool worth_copies(int64_t elements, int64_t M, int64_t N, int64_t K) {
  return elements <= int64_t{1} << 22 || 256.0 * static_cast<double>(elements) <= static_cast<double>(M) * N * K;
}

// The workspace of a call in the order it is handed out; addresses only where there is one.
struct Space {
  char* base;
  int64_t used = 0;
  void* take(int64_t bytes) {
    void* p = base == nullptr ? nullptr : base + used;
    used += (bytes + 15) / 16 * 16;
    return p;
  }
};

// An operand of a call: as it is, or its padded copy.
struct Operand {
  const uint16_t* p;
  int64_t rows, cols, ld;
  bool fit;
};

Operand operand(const void* p, int64_t rows, int64_t cols) {
  return {static_cast<const uint16_t*>(p), rows, cols, cols, fits(p, cols)};
}

// Gives x a padded copy: its place in the workspace and its part in the launch that fills it.
void copy_padded(Operand& x, Space& space, PadArgs& pad, int& pads) {
  if (x.fit) return;
  x.ld = padded(x.cols);
  auto* to = static_cast<uint16_t*>(space.take(2 * x.rows * x.ld));
  pad.src[pads] = x.p;
  pad.dst[pads] = to;
  pad.rows[pads] = x.rows;
  pad.cols[pads] = x.cols;
  ++pads;
  x.p = to;
  x.fit = true;
}

hipError_t launch_pad(const PadArgs& pad, int pads, hipStream_t st) {
  if (pads == 0) return hipSuccess;
  int64_t most = 0;
  for (int m = 0; m < pads; ++m) most = std::max(most, pad.rows[m] * padded(pad.cols[m]) / 8);
  if (most == 0) return hipSuccess;
  const auto grid = static_cast<unsigned>(std::min<int64_t>((most + kThreads - 1) / kThreads, 8192));
  FPSK_LAUNCH(pad_kernel, dim3(grid), dim3(kThreads), 0, st, pad);
  return hipSuccess;
}

MmArgs cut(MmArgs a, const Cut& c) {
  a.tiles_m = c.tiles_m;
  a.tiles_n = c.tiles_n;
  a.splits = c.splits;
  a.kslice = c.kslice;
  return a;
}

template <int DT, bool GATED>
hipError_t launch_sum(const MmArgs& a, const Cut& c, int act, hipStream_t st) {
  if (c.splits > 1) {
    const int64_t count = a.M * (GATED ? a.f : a.N);
    const bool four = (GATED ? a.f : a.M * a.N) % 4 == 0;
    const auto g = static_cast<unsigned>(std::min<int64_t>((count / (four ? 4 : 1) + kThreads - 1) / kThreads, 8192));
    if (four) {
      FPSK_LAUNCH((mm_sum_kernel<DT, GATED, 4>), dim3(g), dim3(kThreads), 0, st, a, act);
    } else {
      FPSK_LAUNCH((mm_sum_kernel<DT, GATED, 1>), dim3(g), dim3(kThreads), 0, st, a, act);
    }
  }
  return hipSuccess;
}

template <int DT, bool AKM, bool BKM, bool GATED>
hipError_t launch_mm(MmArgs a, const Cut& c, int act, hipStream_t st) {
  a = cut(a, c);
  if (!c.direct && !c.few && a.K > 0 && (a.M * a.K < 8 || a.N * a.K < 8)) {
    const int64_t count = a.M * (GATED ? a.f : a.N);
    const auto g = static_cast<unsigned>(std::min<int64_t>((count + kThreads - 1) / kThreads, 8192));
    FPSK_LAUNCH((tiny_kernel<DT, GATED>), dim3(g), dim3(kThreads), 0, st, a, AKM ? 1 : a.K,
                AKM ? a.M : 1, BKM ? 1 : a.K, BKM ? a.N : 1, act);
    return hipSuccess;
  }
  if constexpr (GATED) {
    if (c.few) {
      FPSK_LAUNCH(few_kernel<DT>, dim3(static_cast<unsigned>(c.tiles_n)), dim3(kThreads), 0, st, a, act);
      return hipSuccess;
    }
  }
  const dim3 grid(static_cast<unsigned>(c.tiles_m * c.tiles_n * c.splits));
  if (c.big) {
    FPSK_LAUNCH((mm_kernel<DT, 256, 256, 2, 4, AKM, BKM, GATED>), grid, dim3(512), 0, st, a, act);
  } else if (c.direct) {
    FPSK_LAUNCH((mm_kernel<DT, 128, 128, 2, 2, AKM, BKM, GATED>), grid, dim3(256), 0, st, a, act);
  } else {
    FPSK_LAUNCH((mm_ragged_kernel<DT, 128, 128, 2, 2, AKM, BKM, GATED>), grid, dim3(256), 0, st, a, act);
  }
  return launch_sum<DT, GATED>(a, c, act, st);
}

template <int DT>
hipError_t launch_pair(MmArgs x, const Cut& cx, MmArgs w, const Cut& cw, hipStream_t st) {
  x = cut(x, cx);
  w = cut(w, cw);
  const auto first = static_cast<unsigned>(cx.tiles_m * cx.tiles_n * cx.splits);
  const auto second = static_cast<unsigned>(cw.tiles_m * cw.tiles_n * cw.splits);
  FPSK_LAUNCH(mm_pair_kernel<DT>, dim3(first + second), dim3(256), 0, st, x, w, first);
  const hipError_t e = launch_sum<DT, false>(x, cx, 0, st);
  return e != hipSuccess ? e : launch_sum<DT, false>(w, cw, 0, st);
}

bool dims_ok(int64_t t, int64_t d, int64_t f) {
  if (t < 0 || d < 1 || f < 1 || t >= kDimLimit || d > kMaxLd || 2 * f > kMaxLd) return false;
  // element counts stay inside 2^40, and the tiles of a product inside one launch
  const double most = 1099511627776.0;
  const double td = static_cast<double>(t) * static_cast<double>(d);
  const double tf = 2.0 * static_cast<double>(t) * static_cast<double>(f);
  const double df = 2.0 * static_cast<double>(d) * static_cast<double>(f);
  return td <= most && tf <= most && df <= most;
}

bool launch_fits(const Cut& c) {
  return static_cast<double>(c.tiles_m) * c.tiles_n * c.splits * 512.0 < 4294967296.0;
}

int64_t part_bytes(const Cut& c, int64_t M, int64_t N) {
  return c.splits > 1 ? static_cast<int64_t>(c.splits) * M * N * 4 : 0;
}

// What a call of fpsketch_gated does, and the workspace it takes.
struct GatedPlan {
  Operand x, w;
  PadArgs pad{};
  int pads = 0;
  Cut cut;
  float* part;
  int64_t bytes;
};

GatedPlan plan_gated(const void* X, const void* W, int64_t t, int64_t d, int64_t f, void* workspace, int cus) {
  GatedPlan g;
  Space space{static_cast<char*>(workspace)};
  g.x = operand(X, t, d);
  g.w = operand(W, 2 * f, d);
  const int64_t odd = (g.x.fit ? 0 : t * d) + (g.w.fit ? 0 : 2 * f * d);
  if (worth_copies(odd, t, 2 * f, d)) {
    copy_padded(g.x, space, g.pad, g.pads);
    copy_padded(g.w, space, g.pad, g.pads);
  }
  const bool fit = g.x.fit && g.w.fit;
  g.cut = cut_of(t, f, true, fit && t <= kFew, d, fit, cus);
  g.part = static_cast<float*>(space.take(part_bytes(g.cut, t, 2 * f)));
  g.bytes = space.used;
  return g;
}

// The same for fpsketch_gated_products.  Two products that run one after the other share the room for
// their parts.
struct ProductsPlan {
  Operand p, x, w, xw;     // dP, X, W; dP as dX takes it
  PadArgs pad{};
  int pads = 0;
  Cut dx, dw;
  bool pair;
  float *part_x, *part_w;
  int64_t bytes;
};

ProductsPlan plan_products(const void* dP, const void* X, const void* W, int64_t t, int64_t d, int64_t f,
                           bool need_dx, bool need_dw, void* workspace, int cus) {
  ProductsPlan g;
  Space space{static_cast<char*>(workspace)};
  g.p = operand(dP, t, 2 * f);
  g.x = operand(X, t, d);
  g.w = operand(W, 2 * f, d);
  // How each is computed does not depend on whether the other is asked for, so that it has the same
  // bits either way.
  const int64_t odd_p = g.p.fit ? 0 : 2 * t * f;
  const bool direct_x = worth_copies(odd_p + (g.w.fit ? 0 : 2 * f * d), t, d, 2 * f);
  const bool direct_w = worth_copies(odd_p + (g.x.fit ? 0 : t * d), 2 * f, d, t);
  g.dx = cut_of(std::max<int64_t>(t, 1), d, false, false, 2 * f, direct_x, cus);
  g.dw = cut_of(2 * f, d, false, false, t, direct_w, cus);
  const bool take_x = need_dx && t > 0 && direct_x, take_w = need_dw && direct_w;
  const Operand p = g.p;
  if (take_x || take_w) copy_padded(g.p, space, g.pad, g.pads);   // once for both
  g.xw = take_x ? g.p : p;
  if (!take_w) g.p = p;
  if (take_x) copy_padded(g.w, space, g.pad, g.pads);
  if (take_w) copy_padded(g.x, space, g.pad, g.pads);
  const bool share = direct_x && direct_w && !g.dx.big && !g.dw.big;   // a launch, where both are asked for
  if (share) {
    fewer_parts(g.dx, 2 * f, 2 * cus - g.dw.tiles_m * g.dw.tiles_n);
    fewer_parts(g.dw, t, 2 * cus - g.dx.tiles_m * g.dx.tiles_n);
  }
  g.pair = take_x && take_w && share;
  const int64_t px = need_dx && t > 0 ? part_bytes(g.dx, t, d) : 0, pw = need_dw ? part_bytes(g.dw, 2 * f, d) : 0;
  if (g.pair) {
    g.part_x = static_cast<float*>(space.take(px));
    g.part_w = static_cast<float*>(space.take(pw));
  } else {
    g.part_x = g.part_w = static_cast<float*>(space.take(std::max(px, pw)));
  }
  g.bytes = space.used;
  return g;
}

bool workspace_ok(const void* workspace, int64_t bytes, int64_t need) {
  return need == 0 || (workspace != nullptr && bytes >= need && aligned(workspace, 16));
}

}  // namespace

}  // namespace fpsk

using namespace fpsk;

extern "C" {

int64_t fpsketch_gated_workspace(const void* X, const void* W, int64_t t, int64_t d, int64_t f) {
  int cus = 0;
  if (!dims_ok(t, d, f) || t == 0 || layer_device(&cus) != FPSK_OK) return 0;
  return plan_gated(X, W, t, d, f, nullptr, cus).bytes;
}

fpsketch_status fpsketch_gated(const void* X, const void* W, int64_t t, int64_t d, int64_t f,
                               fpsketch_dtype dtype, fpsketch_act act, void* H, float* P,
                               void* workspace, int64_t workspace_bytes, void* stream) {
  if (!half_type(dtype)) return layer_error(FPSK_EDTYPE, "fpsketch_gated: X, W and H are FP16 or BF16");
  if (act < FPSK_SILU || act > FPSK_GELU_TANH) return layer_error(FPSK_EINVAL, "fpsketch_gated: unknown activation");
  if (!dims_ok(t, d, f)) return layer_error(FPSK_ESHAPE, "fpsketch_gated: dimensions");
  if (t == 0) return FPSK_OK;
  if (X == nullptr || W == nullptr || H == nullptr) return layer_error(FPSK_EINVAL, "fpsketch_gated: null pointer");
  if (!aligned(X, 2) || !aligned(W, 2) || !aligned(H, 2) || !aligned(P, 4)) {
    return layer_error(FPSK_EINVAL, "fpsketch_gated: a pointer is not aligned to its elements");
  }
  int cus = 0;
  const fpsketch_status s = layer_device(&cus);
  if (s != FPSK_OK) return s;
  const GatedPlan g = plan_gated(X, W, t, d, f, workspace, cus);
  if (!launch_fits(g.cut)) return layer_error(FPSK_ESHAPE, "fpsketch_gated: too many tiles");
  if (!workspace_ok(workspace, workspace_bytes, g.bytes)) {
    return layer_error(FPSK_EINVAL, "fpsketch_gated: workspace smaller than fpsketch_gated_workspace, or not aligned to 16 bytes");
  }
  const Span in[] = {{X, 2 * t * d}, {W, 4 * f * d}};
  const Span out[] = {{H, 2 * t * f}, {P, 8 * t * f}, {workspace, g.bytes}};
  if (!disjoint(in, out)) return layer_error(FPSK_EINVAL, "fpsketch_gated: an output overlaps another argument");
  MmArgs a{};
  a.A = g.x.p;
  a.B = g.w.p;
  a.M = t;
  a.N = 2 * f;
  a.K = d;
  a.lda = g.x.ld;
  a.ldb = g.w.ld;
  a.f = f;
  a.out = P;
  a.H = static_cast<uint16_t*>(H);
  a.part = g.part;
  const auto st = static_cast<hipStream_t>(stream);
  hipError_t e = launch_pad(g.pad, g.pads, st);
  if (e == hipSuccess) {
    e = dtype == FPSK_BF16 ? launch_mm<1, false, false, true>(a, g.cut, act, st)
                           : launch_mm<0, false, false, true>(a, g.cut, act, st);
  }
  return launched(e, "fpsketch_gated");
}

fpsketch_status fpsketch_gated_narrow(const float* P, int64_t t, int64_t f, fpsketch_dtype dtype,
                                      fpsketch_act act, void* H, void* stream) {
  if (!half_type(dtype)) return layer_error(FPSK_EDTYPE, "fpsketch_gated_narrow: H is FP16 or BF16");
  if (act < FPSK_SILU || act > FPSK_GELU_TANH) return layer_error(FPSK_EINVAL, "fpsketch_gated_narrow: unknown activation");
  if (!dims_ok(t, 1, f)) return layer_error(FPSK_ESHAPE, "fpsketch_gated_narrow: dimensions");
  if (t == 0) return FPSK_OK;
  if (P == nullptr || H == nullptr) return layer_error(FPSK_EINVAL, "fpsketch_gated_narrow: null pointer");
  if (!aligned(P, 4) || !aligned(H, 2)) {
    return layer_error(FPSK_EINVAL, "fpsketch_gated_narrow: a pointer is not aligned to its elements");
  }
  int cus = 0;
  const fpsketch_status s = layer_device(&cus);
  if (s != FPSK_OK) return s;
  const Span in[] = {{P, 8 * t * f}};
  const Span out[] = {{H, 2 * t * f}};
  if (!disjoint(in, out)) return layer_error(FPSK_EINVAL, "fpsketch_gated_narrow: H overlaps P");
  const auto st = static_cast<hipStream_t>(stream);
  const auto grid = static_cast<unsigned>(std::min<int64_t>((t * f + kThreads - 1) / kThreads, 16384));
  auto* h = static_cast<uint16_t*>(H);
  return launched(dtype == FPSK_BF16
                      ? launch_k(narrow_kernel<1>, dim3(grid), dim3(kThreads), 0, st, nullptr, nullptr,
                                 P, t, f, static_cast<int>(act), h)
                      : launch_k(narrow_kernel<0>, dim3(grid), dim3(kThreads), 0, st, nullptr, nullptr,
                                 P, t, f, static_cast<int>(act), h),
                  "fpsketch_gated_narrow");
}

fpsketch_status fpsketch_gated_grad(const void* dH, const float* P, int64_t t, int64_t f,
                                    fpsketch_dtype dtype, fpsketch_act act, void* dP, void* dPt,
                                    void* stream) {
  if (!half_type(dtype)) return layer_error(FPSK_EDTYPE, "fpsketch_gated_grad: dH and dP are FP16 or BF16");
  if (act < FPSK_SILU || act > FPSK_GELU_TANH) return layer_error(FPSK_EINVAL, "fpsketch_gated_grad: unknown activation");
  if (!dims_ok(t, 1, f)) return layer_error(FPSK_ESHAPE, "fpsketch_gated_grad: dimensions");
  if (t == 0) return FPSK_OK;
  if (dH == nullptr || P == nullptr || dP == nullptr) return layer_error(FPSK_EINVAL, "fpsketch_gated_grad: null pointer");
  if (!aligned(P, 4) || !aligned(dH, 2) || !aligned(dP, 2) || !aligned(dPt, 2)) {
    return layer_error(FPSK_EINVAL, "fpsketch_gated_grad: a pointer is not aligned to its elements");
  }
  int cus = 0;
  const fpsketch_status s = layer_device(&cus);
  if (s != FPSK_OK) return s;
  const Span in[] = {{dH, 2 * t * f}, {P, 8 * t * f}};
  const Span out[] = {{dP, 4 * t * f}, {dPt, 4 * t * f}};
  if (!disjoint(in, out)) return layer_error(FPSK_EINVAL, "fpsketch_gated_grad: an output overlaps another argument");
  if (static_cast<double>((f + 63) / 64) * ((t + 63) / 64) * kThreads >= 4294967296.0) {
    return layer_error(FPSK_ESHAPE, "fpsketch_gated_grad: too many blocks");
  }
  const auto st = static_cast<hipStream_t>(stream);
  const auto* dh = static_cast<const uint16_t*>(dH);
  auto *o = static_cast<uint16_t*>(dP), *ot = static_cast<uint16_t*>(dPt);
  return launched(dtype == FPSK_BF16 ? launch_grad<1>(dh, P, t, f, act, o, ot, st)
                                     : launch_grad<0>(dh, P, t, f, act, o, ot, st),
                  "fpsketch_gated_grad");
}

int64_t fpsketch_gated_products_workspace(const void* dP, const void* X, const void* W, int64_t t,
                                          int64_t d, int64_t f, int32_t need_dx, int32_t need_dw) {
  int cus = 0;
  if (!dims_ok(t, d, f) || layer_device(&cus) != FPSK_OK) return 0;
  return plan_products(dP, X, W, t, d, f, need_dx != 0, need_dw != 0, nullptr, cus).bytes;
}

fpsketch_status fpsketch_gated_products(const void* dP, const void* X, const void* W, int64_t t,
                                        int64_t d, int64_t f, fpsketch_dtype dtype, float* dX,
                                        float* dW, void* workspace, int64_t workspace_bytes,
                                        void* stream) {
  if (!half_type(dtype)) return layer_error(FPSK_EDTYPE, "fpsketch_gated_products: dP, X and W are FP16 or BF16");
  if (!dims_ok(t, d, f)) return layer_error(FPSK_ESHAPE, "fpsketch_gated_products: dimensions");
  if (dX == nullptr && dW == nullptr && t > 0) return layer_error(FPSK_EINVAL, "fpsketch_gated_products: no output");
  if ((t > 0 && dP == nullptr) || (t > 0 && dW != nullptr && X == nullptr) ||
      (t > 0 && dX != nullptr && W == nullptr)) {
    return layer_error(FPSK_EINVAL, "fpsketch_gated_products: null pointer");
  }
  if (!aligned(dP, 2) || !aligned(X, 2) || !aligned(W, 2) || !aligned(dX, 4) || !aligned(dW, 4)) {
    return layer_error(FPSK_EINVAL, "fpsketch_gated_products: a pointer is not aligned to its elements");
  }
  int cus = 0;
  const fpsketch_status s = layer_device(&cus);
  if (s != FPSK_OK) return s;
  const bool need_dx = dX != nullptr, need_dw = dW != nullptr;
  const ProductsPlan g = plan_products(dP, X, W, t, d, f, need_dx, need_dw, workspace, cus);
  if ((need_dx && !launch_fits(g.dx)) || (need_dw && !launch_fits(g.dw))) {
    return layer_error(FPSK_ESHAPE, "fpsketch_gated_products: too many tiles");
  }
  if (!workspace_ok(workspace, workspace_bytes, g.bytes)) {
    return layer_error(FPSK_EINVAL, "fpsketch_gated_products: workspace smaller than fpsketch_gated_products_workspace, or not aligned to 16 bytes");
  }
  const Span in[] = {{dP, 4 * t * f}, {X, 2 * t * d}, {W, 4 * f * d}};
  const Span out[] = {{dX, 4 * t * d}, {dW, 8 * f * d}, {workspace, g.bytes}};
  if (!disjoint(in, out)) return layer_error(FPSK_EINVAL, "fpsketch_gated_products: an output overlaps another argument");
  const auto st = static_cast<hipStream_t>(stream);
  hipError_t e = launch_pad(g.pad, g.pads, st);
  MmArgs x{}, w{};
  x.A = g.xw.p;
  x.B = g.w.p;
  x.M = t;
  x.N = d;
  x.K = 2 * f;
  x.lda = g.xw.ld;
  x.ldb = g.w.ld;
  x.out = dX;
  x.part = g.part_x;
  w.A = g.p.p;
  w.B = g.x.p;
  w.M = 2 * f;
  w.N = d;
  w.K = t;
  w.lda = g.p.ld;
  w.ldb = g.x.ld;
  w.out = dW;
  w.part = g.part_w;
  const bool bf16 = dtype == FPSK_BF16;
  if (e == hipSuccess && g.pair) {
    e = bf16 ? launch_pair<1>(x, g.dx, w, g.dw, st) : launch_pair<0>(x, g.dx, w, g.dw, st);
    return launched(e, "fpsketch_gated_products");
  }
  if (e == hipSuccess && need_dx && t > 0) {
    e = bf16 ? launch_mm<1, false, true, false>(x, g.dx, 0, st) : launch_mm<0, false, true, false>(x, g.dx, 0, st);
  }
  if (e == hipSuccess && need_dw) {
    e = bf16 ? launch_mm<1, true, true, false>(w, g.dw, 0, st) : launch_mm<0, true, true, false>(w, g.dw, 0, st);
  }
  return launched(e, "fpsketch_gated_products");
}

}  // extern "C"
