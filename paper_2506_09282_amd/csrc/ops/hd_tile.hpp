// A workgroup's tile of a matrix product on the matrix instructions,
//   c[m][n] = sum_k a(m, k) b(n, k),
// shared by the operators whose products have many rows on both sides.
//
// An operand lies in memory with its reduction contiguous (kRows: row m holds k), with its
// reduction as rows (kCols: row k holds m), or as an 8-bit weight image (kImage). A stage is
// 128 bytes of the reduction of every row (64 bf16, 32 fp32, 128 int8 values). It goes through
// registers into one of two buffers in LDS while the other is multiplied, so that rows of any
// alignment, ends of rows and rows that take no part cost nothing but their own loads.
//
// In LDS a kRows operand is [row][8 pieces of 16 bytes], piece j at j ^ (row & 7): a lane's
// operand of the 32 x 32 instruction is one piece, and the 64 pieces of a read spread over all
// banks. A kCols operand is [k][R values] as in memory; bf16 takes its operands with transposing
// reads (16 lanes read 4 rows of 16 values and get 4 values of one column each), fp32, whose
// instruction takes one k from a lane, with plain ones.
#pragma once

#include "hd_ops.hpp"

namespace hd {
namespace ops {
namespace tile {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_a1 __attribute__((aligned(1)));
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));
typedef u32x4 u32x4_a1 __attribute__((aligned(1)));

enum Kind { kRows, kCols, kImage };

struct Operand {
  const void* p;         // row 0
  int64_t ld;            // elements from row to row
  int64_t extent;        // rows of the tile's own dimension
  const uint64_t* live;  // kCols: a bit for each k that takes part (null: all do); the
                         // others' rows are not looked at and count as 0
};

// Strides up to this keep a tile's offsets in 32 bits.
constexpr int64_t kMaxStride = int64_t(1) << 22;

struct Bf16 {
  typedef bf16raw elem;
  typedef u32x4_a2 piece;
  typedef f32x16 acc;
  static constexpr int kEs = 2, kBk = 64;
  static __device__ __forceinline__ void mfma(acc& c, const u32x4& a, const u32x4& b) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
struct F32 {
  typedef float elem;
  typedef u32x4_a4 piece;
  typedef f32x16 acc;
  static constexpr int kEs = 4, kBk = 32;
  static __device__ __forceinline__ void mfma(acc& c, const u32x4& a, const u32x4& b) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0,
                                               0, 0);
  }
};
struct I8 {
  typedef int8_t elem;
  typedef u32x4_a1 piece;
  typedef i32x16 acc;
  static constexpr int kEs = 1, kBk = 128;
  static __device__ __forceinline__ void mfma(acc& c, const u32x4& a, const u32x4& b) {
    c = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a),
                                              __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};

// The first `valid` elements at p, zeros behind them.
template <class P>
__device__ __forceinline__ u32x4 load_part(const char* p, int valid) {
  u32x4 v = {0u, 0u, 0u, 0u};
  constexpr int kE = 16 / P::kEs;
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    if (e >= valid) break;
    uint32_t x;
    if constexpr (P::kEs == 4)
      x = reinterpret_cast<const uint32_t*>(p)[e];
    else if constexpr (P::kEs == 2)
      x = reinterpret_cast<const uint16_t*>(p)[e];
    else
      x = reinterpret_cast<const uint8_t*>(p)[e];
    v[e * P::kEs / 4] |= x << (8 * (e * P::kEs % 4));
  }
  return v;
}

// How pieces of a kCols row k are moved, so that rows read together use different banks.
template <class P, int R>
__device__ __forceinline__ int col_swizzle(int k) {
  if constexpr (P::kEs == 4)
    return R >= 64 ? ((k >> 2) & 1) * 8 : 0;
  else
    return R >= 128 ? (k & 3) * 4 : R == 64 ? ((k >> 1) & 1) * 4 : 0;
}

// One operand's way from memory to LDS: R rows (or columns) by T threads.
template <class P, int KIND, int R, int T>
struct Loader {
  static constexpr int kE = 16 / P::kEs;
  static constexpr int kPasses = R * 8 / T;
  static constexpr int kAcross = KIND == kCols ? R / kE : 8;  // pieces of a row
  static constexpr int kStep = T / kAcross;                   // rows of a pass
  static_assert(kPasses >= 1 && T % kAcross == 0, "");
  static constexpr int kBytes = R * 128;  // of a stage

  const char* base;  // kRows: the tile's first row; kCols: its first column of k = 0
  int64_t ld;        // bytes
  const uint64_t* live;
  uint32_t off[kPasses];
  int lds_at, row, cols;
  bool inside;  // every column of the tile exists
  u32x4 reg[kPasses];

  __device__ __forceinline__ Loader(const Operand& o, int64_t at, int tid) {
    ld = o.ld * P::kEs;
    live = o.live;
    row = tid / kAcross;
    const int piece = tid % kAcross;
    if constexpr (KIND == kImage) {
      // a wave's load is a block of 32 outputs x 32 inputs: lane l holds output l % 32,
      // inputs 16 (l / 32) ... of it; ld: blocks of 32 inputs
      const int lane = tid & 63, wave = tid >> 6;
      base = reinterpret_cast<const char*>(o.p);
#pragma unroll
      for (int p = 0; p < kPasses; ++p) {
        const int block = p * (T / 64) + wave;  // of the stage: (outputs / 32, inputs / 32)
        const int64_t tiles = cdiv(o.extent, 32);
        int64_t t = at / 32 + block / 4;
        t = t < tiles ? t : tiles - 1;
        off[p] = 0;
        reg[p] = u32x4{0u, 0u, 0u, 0u};
        first[p] = (t * o.ld + block % 4) * 1024 + lane * 16;
      }
      row = lane & 31;
      cols = lane >> 5;
      lds_at = 0;
      inside = true;
      return;
    }
    if constexpr (KIND == kRows) {
      base = reinterpret_cast<const char*>(o.p) + at * ld;
      const int64_t last = o.extent - 1 - at;
#pragma unroll
      for (int p = 0; p < kPasses; ++p) {
        const int r = p * kStep + row;
        off[p] = (uint32_t)(r < last ? r : last) * (uint32_t)ld + piece * 16;
      }
      cols = piece * kE;  // its place in the stage
      lds_at = row * 128 + ((piece ^ (row & 7)) << 4);
      inside = true;
    } else {
      base = reinterpret_cast<const char*>(o.p) + at * P::kEs;
      const int64_t left = o.extent - at - piece * kE;
      cols = left > kE ? kE : left < 0 ? 0 : (int)left;
      inside = o.extent - at >= R;
#pragma unroll
      for (int p = 0; p < kPasses; ++p)
        off[p] = (uint32_t)(p * kStep + row) * (uint32_t)ld + piece * 16;
      lds_at = 0;
    }
  }
  int64_t first[KIND == kImage ? kPasses : 1];

  __device__ __forceinline__ u32x4 whole(const char* p) const {
    return *reinterpret_cast<const typename P::piece*>(p);
  }

  // Stage [k, min(k + kBk, end)) to registers.
  __device__ __forceinline__ void load(int64_t k, int64_t end) {
    if constexpr (KIND == kImage) {
#pragma unroll
      for (int p = 0; p < kPasses; ++p)  // (an image's reduction is whole stages)
        reg[p] = *reinterpret_cast<const u32x4*>(base + first[p] + k * 32);
    } else if constexpr (KIND == kRows) {
      const char* at = base + k * P::kEs;
      if (k + P::kBk <= end) {
#pragma unroll
        for (int p = 0; p < kPasses; ++p) reg[p] = whole(at + off[p]);
      } else {
        const int64_t left = end - k - cols;
#pragma unroll
        for (int p = 0; p < kPasses; ++p)
          reg[p] = left >= kE ? whole(at + off[p]) : load_part<P>(at + off[p], (int)left);
      }
    } else {
      const char* at = base + k * ld;
      if (inside && !live && k + P::kBk <= end) {
#pragma unroll
        for (int p = 0; p < kPasses; ++p) reg[p] = whole(at + off[p]);
      } else {
        uint64_t bits = live ? live[k >> 6] >> (k & 63) : ~uint64_t(0);
        const int64_t left = end - k;
        if (left < 64) bits &= (uint64_t(1) << left) - 1;
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
          u32x4 v = {0u, 0u, 0u, 0u};
          if (bits >> (p * kStep + row) & 1)
            v = cols == kE ? whole(at + off[p]) : load_part<P>(at + off[p], cols);
          reg[p] = v;
        }
      }
    }
  }

  // Those registers to the operand's part of a buffer.
  __device__ __forceinline__ void store(char* lds, int tid) const {
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      int at;
      if constexpr (KIND == kImage) {
        const int block = p * (T / 64) + (tid >> 6);
        const int r = block / 4 * 32 + row;
        at = r * 128 + (((block % 4 * 2 + cols) ^ (r & 7)) << 4);
      } else if constexpr (KIND == kRows) {
        at = lds_at + p * kStep * 128;
      } else {
        const int k = p * kStep + row;
        at = k * R * P::kEs + (((tid % kAcross) ^ col_swizzle<P, R>(k)) << 4);
      }
      *reinterpret_cast<u32x4*>(lds + at) = reg[p];
    }
  }
};

// A lane's operand: rows 32 * sub ... of the tile, quarter kk of the stage.
template <class P, int KIND, int R>
__device__ __forceinline__ u32x4 fragment(const char* lds, int sub, int kk, int lane) {
  const int half = lane >> 5;
  if constexpr (KIND != kCols) {
    const int row = sub * 32 + (lane & 31);
    return *reinterpret_cast<const u32x4*>(lds + row * 128 +
                                           (((2 * kk + half) ^ (lane & 7)) << 4));
  } else if constexpr (P::kEs == 2) {
    const int i = lane & 15, piece = sub * 4 + ((lane >> 4) & 1) * 2 + ((i & 3) >> 1);
    const int k = kk * 16 + half * 8 + (i >> 2);
    u32x4 v;
#pragma unroll
    for (int j = 0; j < 2; ++j) {  // (k + 4 moves pieces as k does)
      const char* at = lds + (k + 4 * j) * R * 2 + ((piece ^ col_swizzle<P, R>(k + 4 * j)) << 4) +
                       (i & 1) * 8;
      const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4*)(at));
      const u32x2 y = __builtin_bit_cast(u32x2, x);
      v[2 * j] = y[0];
      v[2 * j + 1] = y[1];
    }
    return v;
  } else {
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int k = (2 * kk + half) * 4 + e;
      const int piece = (sub * 8 + ((lane & 31) >> 2)) ^ col_swizzle<P, R>(k);
      v[e] = *reinterpret_cast<const uint32_t*>(lds + k * R * 4 + piece * 16 + (lane & 3) * 4);
    }
    return v;
  }
}

// BM x BN by WM x WN waves. Of a wave's accumulators c[i][j], register r of lane l is
//   m = 32 (wave row * MT + i) + 8 (r / 4) + 4 (l / 32) + r % 4,  n = 32 (...) + l % 32.
template <class P_, int AK, int BK_, int BM_, int BN_, int WM_, int WN_>
struct Tile {
  typedef P_ P;
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, T = 64 * WM * WN;
  static constexpr int MT = BM / WM / 32, NT = BN / WN / 32;
  static constexpr int kStage = (BM + BN) * 128, kLds = 2 * kStage;
  typedef typename P::acc Acc;

  // The sum over k in [k0, k1). All threads of the workgroup; ends with a barrier.
  static __device__ __forceinline__ void product(const Operand& a, const Operand& b, int64_t m0,
                                                 int64_t n0, int64_t k0, int64_t k1, char* lds,
                                                 Acc (&c)[MT][NT]) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = wave / WN, wn = wave % WN;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) c[i][j][r] = 0;
    if (k0 >= k1) return;
    Loader<P, AK, BM, T> la(a, m0, tid);
    Loader<P, BK_, BN, T> lb(b, n0, tid);
    la.load(k0, k1);
    lb.load(k0, k1);
    la.store(lds, tid);
    lb.store(lds + BM * 128, tid);
    __syncthreads();
    int cur = 0;
    for (int64_t k = k0; k < k1; k += P::kBk) {
      const bool more = k + P::kBk < k1;
      if (more) {
        la.load(k + P::kBk, k1);
        lb.load(k + P::kBk, k1);
      }
      const char* at = lds + cur * kStage;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        u32x4 fa[MT], fb[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) fa[i] = fragment<P, AK, BM>(at, wm * MT + i, kk, lane);
#pragma unroll
        for (int j = 0; j < NT; ++j)
          fb[j] = fragment<P, BK_, BN>(at + BM * 128, wn * NT + j, kk, lane);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int j = 0; j < NT; ++j) P::mfma(c[i][j], fa[i], fb[j]);
      }
      cur ^= 1;
      if (more) {
        la.store(lds + cur * kStage, tid);
        lb.store(lds + cur * kStage + BM * 128, tid);
      }
      __syncthreads();
    }
  }
};

// Workgroup b of n takes this place in the order of the work, so that the workgroups of one
// die (b % 8), which share an L2, have neighbouring places.
__device__ __forceinline__ uint32_t die_order(uint32_t b, uint32_t n) {
  const uint32_t x = b & 7, each = n >> 3, more = n & 7;
  return x * each + (x < more ? x : more) + (b >> 3);
}

// Place `id` in an mt x nt grid of tiles: eight tiles of n side by side, then m, so that
// neighbouring places share rows of both operands.
__device__ __forceinline__ void tile_at(uint32_t id, uint32_t mt, uint32_t nt, uint32_t& mi,
                                        uint32_t& ni) {
  const uint32_t g = id / (8 * mt), first = 8 * g;
  const uint32_t wide = nt - first < 8 ? nt - first : 8;
  const uint32_t at = id - g * 8 * mt;
  ni = first + at % wide;
  mi = at / wide;
}

// ---- host: which tile, and how many parts of the reduction -----------------------
enum Shape { k256, k128, k32x128, k128x32 };

struct Plan {
  Shape shape;
  int64_t mt, nt;   // tiles
  int64_t splits;   // parts of the reduction
  int64_t each;     // values of k of a part (a multiple of 128)
};

// For [M][N] sums over K: the large tile where there is one for every compute unit, narrow
// ones where a side is short, and parts of the reduction where that leaves the chip idle.
inline Plan plan(int64_t M, int64_t N, int64_t K) {
  Plan p;
  int64_t slots;  // workgroups that the chip holds at once
  if (M <= 32) {
    p = {k32x128, 1, cdiv(N, 128), 1, 0};
    slots = 768;
  } else if (N <= 32) {
    p = {k128x32, cdiv(M, 128), 1, 1, 0};
    slots = 768;
  } else if (cdiv(M, 256) * cdiv(N, 256) >= 192) {
    p = {k256, cdiv(M, 256), cdiv(N, 256), 1, 0};
    slots = 256;
  } else {
    p = {k128, cdiv(M, 128), cdiv(N, 128), 1, 0};
    slots = 512;
  }
  const int64_t tiles = p.mt * p.nt;
  const int64_t most = cdiv(K, 256);  // at least two stages or so to a part
  if (2 * tiles <= slots && p.shape != k256) {
    p.splits = slots / tiles;
    if (p.splits > most) p.splits = most;
  }
  p.each = cdiv(cdiv(K, p.splits), 128) * 128;
  p.splits = cdiv(K, p.each);
  return p;
}

}  // namespace tile
}  // namespace ops
}  // namespace hd
