// A workgroup's tile of a matrix product on the matrix instructions,
//   c[m][n] = sum_k a(m, k) b(n, k),
// shared by the operators whose products have many rows on both sides.
//
// An operand lies in memory with its reduction contiguous (kRows: row m holds k), with its
// reduction as rows (kCols: row k holds m), or as an 8-bit weight image (kImage). A stage is
// 128 bytes of the reduction of every row (64 bf16, 32 fp32, 128 int8 values; 64 bytes of fp32 in
// three parts). It goes through
// registers into one of two buffers in LDS while the other is multiplied, so that rows of any
// alignment, ends of rows and rows that take no part cost nothing but their own loads.
//
// In LDS a kRows operand is [row][8 pieces of 16 bytes], piece j at j ^ (row / 2 % 8): a lane's
// operand of the 32 x 32 instruction is one piece, and 16 lanes' pieces, of 16 rows, lie in all 64
// banks (with j ^ (row % 8) two at a time share theirs: 37% of the LDS's cycles). A kCols operand
// is [k][R values] as in memory; bf16 takes its operands with transposing reads (16 lanes read 4
// rows of 16 values and get 4 values of one column each), fp32, whose instruction takes one k
// from a lane, with plain ones.
//
// The large tile (256 x 256, eight waves of 128 x 64) keeps the matrix units busy for 57% of the
// cycles in bf16 and 44% in int8, LDS for 35% in both, without bank conflicts in bf16. No unit is
// full: its waves wait for 29 and 33% of their time, half of that for LDS, and meet at each stage's
// barrier. It is not memory (with every load from a cache's hot lines 4096 x 131072 by 4096 bf16
// took 3.73 ms instead of 3.87) and not the distance of the reads alone (reading operands a quarter
// ahead changed nothing). Measured: that product with the epilogue of a cross entropy 3.7 to 3.9 ms
// (1.12 to 1.19 PFLOP/s; a library product of 8192^3 1.22 to 1.26), int8 8192 x 4096 x 16384 0.57 to
// 0.6 ms (1.8 to 1.9 POP/s), fp32 in three parts 777 x 2047 x 32003 0.60 to 0.63 ms (160 to 170
// TFLOP/s; fp32's own instruction 1.02 ms). Ranges are those of several cards.
#pragma once

#include <type_traits>

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
  int64_t rest = 0;      // a product's first operand: bytes from its values to what their type's
                         // rounding left of them, which is multiplied too (0: nothing)
};

// Strides up to this keep a tile's offsets in 32 bits.
constexpr int64_t kMaxStride = int64_t(1) << 22;

struct Bf16 {
  typedef bf16raw elem;
  typedef u32x4_a2 piece;
  typedef f32x16 acc;
  static constexpr int kEs = 2, kBk = 64, kParts = 1;
  static __device__ __forceinline__ void mfma(acc& c, const u32x4& a, const u32x4& b) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
struct F32 {
  typedef float elem;
  typedef u32x4_a4 piece;
  typedef f32x16 acc;
  static constexpr int kEs = 4, kBk = 32, kParts = 1;
  static __device__ __forceinline__ void mfma(acc& c, const u32x4& a, const u32x4& b) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0,
                                               0, 0);
  }
};
// fp32 as the exact sum of three bf16 values: the upper half of its bits, the rest rounded to
// bf16, and what is left (8 bits; exact but for bits below 2^-133). Six of the nine products of
// parts are summed; those left out are within 2^-22 of the whole and of either sign. That is
// six bf16 instructions for 16 values of k, where fp32's own take twice as long. An infinity
// has no such parts and counts as NaN.
struct X3 {
  typedef float elem;
  typedef u32x4_a4 piece;
  typedef f32x16 acc;
  static constexpr int kEs = 4, kBk = 16, kParts = 3;
  static __device__ __forceinline__ void mfma(acc& c, const u32x4& a, const u32x4& b) {
    Bf16::mfma(c, a, b);
  }
  // Four values to two words of each part.
  static __device__ __forceinline__ void split(const u32x4& v, u32x2 (&part)[3]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t x = v[2 * h], y = v[2 * h + 1];
      part[0][h] = __builtin_amdgcn_perm(y, x, 0x07060302);  // the upper halves
      const float rx = __uint_as_float(x) - __uint_as_float(x & 0xffff0000u);
      const float ry = __uint_as_float(y) - __uint_as_float(y & 0xffff0000u);
      const bf16x2 m = {(__bf16)rx, (__bf16)ry};
      const uint32_t mid = __builtin_bit_cast(uint32_t, m);
      part[1][h] = mid;
      const bf16x2 l = {(__bf16)(rx - __uint_as_float(mid << 16)),
                        (__bf16)(ry - __uint_as_float(mid & 0xffff0000u))};
      part[2][h] = __builtin_bit_cast(uint32_t, l);
    }
  }
};
struct I8 {
  typedef int8_t elem;
  typedef u32x4_a1 piece;
  typedef i32x16 acc;
  static constexpr int kEs = 1, kBk = 128, kParts = 1;
  static __device__ __forceinline__ void mfma(acc& c, const u32x4& a, const u32x4& b) {
    c = __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a),
                                              __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};

// The first `valid` elements at p, zeros behind them. With `back`, the elements before p are there
// too, and one load takes those that end with the last valid one (BACK: not in the large tile,
// whose registers are full).
template <class P, bool BACK>
__device__ __forceinline__ u32x4 load_part(const char* p, int valid, bool back) {
  constexpr int kE = 16 / P::kEs;
  u32x4 v = {0u, 0u, 0u, 0u};
  if (valid <= 0) return v;
  if (BACK && back) {
    const int bytes = (kE - valid) * P::kEs;  // under 16
    v = *reinterpret_cast<const typename P::piece*>(p - bytes);
    uint64_t lo = (uint64_t)v[1] << 32 | v[0], hi = (uint64_t)v[3] << 32 | v[2];
    const int s = 8 * (bytes & 7);
    if (bytes & 8) {
      lo = hi;
      hi = 0;
    }
    lo = lo >> s | (s ? hi << (64 - s) : 0);
    hi >>= s;
    return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
  }
  // (a loop, not 16 bytes' worth of straight code: it is rare, and short kernels wait for code)
  uint64_t lo = 0, hi = 0;
#pragma unroll 1
  for (int e = valid - 1; e >= 0; --e) {
    uint32_t x;
    if constexpr (P::kEs == 4)
      x = reinterpret_cast<const uint32_t*>(p)[e];
    else if constexpr (P::kEs == 2)
      x = reinterpret_cast<const uint16_t*>(p)[e];
    else
      x = reinterpret_cast<const uint8_t*>(p)[e];
    hi = hi << (8 * P::kEs) | lo >> (64 - 8 * P::kEs);
    lo = lo << (8 * P::kEs) | x;
  }
  return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// How pieces of a kCols row k are moved, so that rows read together use different banks.
template <class P, int R>
__device__ __forceinline__ int col_swizzle(int k) {
  if constexpr (P::kEs == 4)
    return R >= 64 ? ((k >> 2) & 1) * 8 : 0;
  else
    return R >= 128 ? (k & 3) * 4 : R == 64 ? ((k >> 1) & 1) * 4 : 0;
}

// One operand's way from memory to LDS: R rows (or columns) by T threads. ONCE: past the caches.
template <class P, int KIND, int R, int T, int RING, bool ONCE>
struct Loader {
  static constexpr int kE = 16 / P::kEs;
  static constexpr int kAcross = KIND == kCols ? R / kE : P::kBk / kE;  // pieces of a row
  static constexpr int kStep = T / kAcross;                             // rows of a pass
  static constexpr int kPasses = (KIND == kCols ? P::kBk : R) / kStep;
  static_assert(kPasses >= 1 && T % kAcross == 0, "");

  const char* base;  // kRows: the tile's first row; kCols: its first column of k = 0
  int64_t ld;        // bytes
  const uint64_t* live;
  uint32_t off[KIND == kCols ? 1 : kPasses];
  int lds_at, row, cols;
  bool back;  // kCols: the elements before a piece are the row's
  u32x4 ring[RING][kPasses];  // stages on their way

  __device__ __forceinline__ Loader(const Operand& o, int64_t at, int tid) {
    ld = o.ld * P::kEs;
    live = o.live;
    row = tid / kAcross;
    const int piece = tid % kAcross;
    if constexpr (KIND == kImage) {
      // a wave's load is a block of 32 outputs x 32 inputs: lane l holds output l % 32,
      // inputs 16 (l / 32) ... of it; ld: blocks of 32 inputs
      const int lane = tid & 63, wave = tid >> 6;
      base = reinterpret_cast<const char*>(o.p) + at / 32 * o.ld * 1024;
      const int64_t last = cdiv(o.extent - at, 32) - 1;
#pragma unroll
      for (int p = 0; p < kPasses; ++p) {
        const int block = p * (T / 64) + wave;  // of the stage: (outputs / 32, inputs / 32)
        const int t = block / 4 < last ? block / 4 : (int)last;
        off[p] = ((uint32_t)t * (uint32_t)o.ld + block % 4) * 1024 + lane * 16;
      }
      row = lane & 31;
      cols = lane >> 5;
      lds_at = 0;
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
      lds_at = row * 128 + ((piece ^ ((row >> 1) & 7)) << 4);
    } else {
      base = reinterpret_cast<const char*>(o.p) + at * P::kEs;
      const int64_t last = (o.extent - 1 - at) / kE;  // the last piece with a column that exists
      const int mine = piece < last ? piece : (int)last;
      const int64_t left = o.extent - at - mine * kE;
      cols = left > kE ? kE : (int)left;
      back = at + mine * kE >= kE;
      off[0] = (uint32_t)row * (uint32_t)ld + mine * 16;  // of pass 0
      lds_at = 0;
    }
  }
  __device__ __forceinline__ u32x4 whole(const char* p) const {
    return *reinterpret_cast<const typename P::piece*>(p);
  }
  // reg[p] = piece(p) for every pass, past the caches where that pays.
  template <class F>
  __device__ __forceinline__ void pieces(u32x4 (&reg)[kPasses], F piece) const {
#pragma unroll
    for (int p = 0; p < kPasses; ++p)
      reg[p] = ONCE ? __builtin_nontemporal_load(
                          reinterpret_cast<const typename P::piece*>(piece(p)))
                    : whole(piece(p));
  }

  // Stage [k, min(k + kBk, end)) to a slot of the ring.
  __device__ __forceinline__ void load(int64_t k, int64_t end, int slot, int64_t more = 0) {
    u32x4(&reg)[kPasses] = ring[slot];
    if constexpr (KIND == kImage) {
#pragma unroll
      for (int p = 0; p < kPasses; ++p)  // (an image's reduction is whole stages)
        reg[p] = *reinterpret_cast<const u32x4*>(base + k * 32 + off[p]);
    } else if constexpr (KIND == kRows) {
      const char* at = base + k * P::kEs + more;
      if (k + P::kBk <= end) {
        pieces(reg, [&](int p) { return at + off[p]; });
      } else {
        const int64_t left = end - k - cols;
#pragma unroll
        for (int p = 0; p < kPasses; ++p)
          reg[p] = left >= kE ? whole(at + off[p])
                             : load_part<P, (RING > 1)>(at + off[p], (int)left, k + cols >= kE);
      }
    } else {
      const char* at = base + k * ld + more;
      const uint64_t bits = live ? live[k >> 6] >> (k & 63) : ~uint64_t(0);
      if (k + P::kBk + kE <= end) {
        // (a piece across the row's end runs into the next rows, of which there are enough: what
        // it takes from there are columns that nobody looks at)
        const uint64_t mine = bits >> row;
        pieces(reg, [&](int p) { return at + p * kStep * ld + off[0]; });
        if (live) {
#pragma unroll
          for (int p = 0; p < kPasses; ++p)
            if (!(mine >> (p * kStep) & 1)) reg[p] = u32x4{0u, 0u, 0u, 0u};
        }
      } else {
        const int left = end - k < 64 ? (int)(end - k) : 64;
        const uint64_t mine = (left < 64 ? bits & ((uint64_t(1) << left) - 1) : bits) >> row;
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
          u32x4 v = {0u, 0u, 0u, 0u};
          if (mine >> (p * kStep) & 1)
            v = cols == kE ? whole(at + p * kStep * ld + off[0])
                           : load_part<P, (RING > 1)>(at + p * kStep * ld + off[0], cols, back);
          reg[p] = v;
        }
      }
    }
  }

  // Those registers to the operand's part of a buffer.
  __device__ __forceinline__ void store(char* lds, int tid, int slot) const {
    const u32x4(&reg)[kPasses] = ring[slot];
    if constexpr (P::kParts == 3) {
      const int piece = tid % kAcross;
#pragma unroll
      for (int p = 0; p < kPasses; ++p) {
        u32x2 part[3];
        X3::split(reg[p], part);
        const int r = p * kStep + row;
        const int at = KIND == kRows
                           ? r * 32 + (((piece >> 1) ^ ((r >> 3) & 1)) << 4) + (piece & 1) * 8
                           : r * R * 2 + (((piece >> 1) ^ col_swizzle<Bf16, R>(r)) << 4) +
                                 (piece & 1) * 8;
#pragma unroll
        for (int q = 0; q < 3; ++q) *reinterpret_cast<u32x2*>(lds + q * R * 32 + at) = part[q];
      }
      return;
    }
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      int at;
      if constexpr (KIND == kImage) {
        const int block = p * (T / 64) + (tid >> 6);
        const int r = block / 4 * 32 + row;
        at = r * 128 + (((block % 4 * 2 + cols) ^ ((r >> 1) & 7)) << 4);
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

// A lane's operand: rows 32 * sub ... of the tile, quarter kk of the stage (or the part kk of it).
template <class P, int KIND, int R>
__device__ __forceinline__ u32x4 fragment(const char* lds, int sub, int kk, int lane) {
  const int half = lane >> 5;
  if constexpr (P::kParts == 3 && KIND == kRows) {  // (kk: the part)
    const int row = sub * 32 + (lane & 31);
    return *reinterpret_cast<const u32x4*>(lds + kk * R * 32 + row * 32 +
                                           ((half ^ ((lane >> 3) & 1)) << 4));
  } else if constexpr (P::kParts == 3) {
    return fragment<Bf16, kCols, R>(lds + kk * R * 32, sub, 0, lane);
  } else if constexpr (KIND != kCols) {
    const int row = sub * 32 + (lane & 31);
    return *reinterpret_cast<const u32x4*>(lds + row * 128 +
                                           (((2 * kk + half) ^ ((lane >> 1) & 7)) << 4));
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
// ONCE: the wide operand of a narrow tile goes past the caches.
template <class P_, int AK, int BK_, int BM_, int BN_, int WM_, int WN_, bool ONCE = false>
struct Tile {
  typedef P_ P;
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, T = 64 * WM * WN;
  static constexpr int MT = BM / WM / 32, NT = BN / WN / 32;
  static constexpr int kRowBytes = P::kParts == 3 ? 96 : 128;  // of a stage
  static constexpr int kStage = (BM + BN) * kRowBytes, kLds = 2 * kStage;
  // Operands in registers: the parts, or a quarter of a stage (reading one quarter while another
  // is multiplied took as many registers again and gained nothing: two waves share a SIMD).
  static constexpr int kSets = P::kParts;
  // Stages loaded ahead: as many as the registers hold. The large tile has the time of a whole
  // stage (over 2000 cycles) for each load; smaller ones, and short reductions, wait for memory.
  static constexpr int kRing = BM * BN > 128 * 128                       ? 1
                               : BM * BN == 128 * 128 && P::kParts == 3 ? 3
                                                                        : 2;
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
    Loader<P, AK, BM, T, kRing, (ONCE && BN == 32)> la(a, m0, tid);
    Loader<P, BK_, BN, T, kRing, (ONCE && BM == 32)> lb(b, n0, tid);
    // (stages are counted in 32 bits: a reduction is far shorter)
    // With a rest each stage comes twice, the second time with the rest of a's values (and b's
    // again, from a cache).
    const int twice = a.rest != 0;
    const int stages = (int)((k1 - k0 + P::kBk - 1) / P::kBk) << twice;
    auto load = [&](int s, int slot) {
      const int64_t k = k0 + (int64_t)(s >> twice) * P::kBk;
      la.load(k, k1, slot, s & twice ? a.rest : 0);
      lb.load(k, k1, slot);
    };
    auto store = [&](char* to, int slot) {
      la.store(to, tid, slot);
      lb.store(to + BM * kRowBytes, tid, slot);
    };
    u32x4 fa[kSets][MT], fb[kSets][NT];
    auto read = [&](int to, const char* at, int kk) {
#pragma unroll
      for (int i = 0; i < MT; ++i) fa[to][i] = fragment<P, AK, BM>(at, wm * MT + i, kk, lane);
#pragma unroll
      for (int j = 0; j < NT; ++j)
        fb[to][j] = fragment<P, BK_, BN>(at + BM * kRowBytes, wn * NT + j, kk, lane);
    };
    auto multiply = [&](int of_a, int of_b) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) P::mfma(c[i][j], fa[of_a][i], fb[of_b][j]);
    };
    // Stage s goes to LDS from slot s % kRing while stage s - 1 is multiplied, and stage
    // s + kRing is then loaded into that slot.
    load(0, 0);
#pragma unroll
    for (int u = 1; u < kRing; ++u)
      if (u < stages) load(u, u);
    store(lds, 0);
    if (kRing < stages) load(kRing, 0);
    __syncthreads();
    auto step = [&](int s, int u) {
      const char* at = lds + (s & 1) * kStage;
      char* other = lds + ((s & 1) ^ 1) * kStage;
      const int slot = (u + 1) % kRing;
      auto next = [&] {
        if (s + 1 < stages) {
          store(other, slot);
          if (s + 1 + kRing < stages) load(s + 1 + kRing, slot);
        }
      };
      if constexpr (P::kParts == 3) {
#pragma unroll
        for (int q = 0; q < 3; ++q) read(q, at, q);
        multiply(2, 0);  // parts' products, the smallest first
        multiply(1, 1);
        multiply(0, 2);
        next();
        multiply(1, 0);
        multiply(0, 1);
        multiply(0, 0);
        __syncthreads();
      } else {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          read(0, at, kk);
          if (kk == 2) next();
          // (the next stage is there, and the rest of this one is in registers)
          if (kk == 3) __syncthreads();
          multiply(0, 0);
        }
      }
    };
    // (no way out of a round: its last steps are passed over)
    for (int s0 = 0; s0 < stages; s0 += kRing) {
#pragma unroll
      for (int u = 0; u < kRing; ++u)
        if (s0 + u < stages) step(s0 + u, u);
    }
    __syncthreads();
  }

  // f(m, n, four values of row m from column n on) for all of the tile, a wave's lanes side by side
  // along the rows. The sums change lanes through the wave's own part of LDS.
  template <class F>
  static __device__ __forceinline__ void rows_out(const Acc (&c)[MT][NT], char* lds, int64_t m0,
                                                  int64_t n0, F f) {
    typedef std::remove_reference_t<decltype(c[0][0][0] + 0)> E;
    typedef E Four __attribute__((ext_vector_type(4)));
    constexpr int kPitch = NT * 32 + 8;  // (rows four apart lie half the banks apart)
    static_assert(WM * WN * 32 * kPitch * 4 <= kLds, "");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    E* mine = reinterpret_cast<E*>(lds) + wave * 32 * kPitch;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      // (a wave's LDS accesses are done in order)
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          mine[((r / 4) * 8 + half * 4 + r % 4) * kPitch + j * 32 + (lane & 31)] = c[i][j][r];
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      const int64_t m = m0 + (wave / WN * MT + i) * 32, n = n0 + wave % WN * NT * 32;
#pragma unroll 2
      for (int q = lane; q < 32 * NT * 8; q += 64) {
        const int row = q / (NT * 8), col = q % (NT * 8) * 4;
        f(m + row, n + col, *reinterpret_cast<const Four*>(mine + row * kPitch + col));
      }
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
enum Shape { k256, k128, k32x256, k256x32 };

struct Plan {
  Shape shape;
  int64_t mt, nt;   // tiles
  int64_t splits;   // parts of the reduction
  int64_t each;     // values of k of a part (a multiple of 128)
};

// Whether the wide operand of a narrow tile goes past the caches: each of its values passes one
// workgroup, once (twice where the other operand has a rest: 16384 x 10240 bf16 under 26 classes 150
// us instead of 166 through the caches), but where lines hold parts of two rows or stages, those take it from the cache
// (16384 x 10240 fp32 under 26 classes: 114 us instead of 130; 100003 rows of 2000 bytes: 66
// instead of 55).
inline bool once(const Plan& p, const Operand& a, const Operand& b, int es) {
  if ((p.shape != k32x256 && p.shape != k256x32) || a.rest) return false;
  const Operand& wide = p.shape == k32x256 ? b : a;
  return ((uintptr_t)wide.p | (uintptr_t)(wide.ld * es)) % 128 == 0;
}

// Whether the large tile, one to a compute unit, finishes before the tile of a quarter of its size,
// two to a unit, which takes 5/8 of the time (4096 x 4096 by 2048 bf16, one round and two: 67 us
// instead of 83; 4096 x 5120, two and three: 118 instead of 103).
inline bool large_pays(int64_t M, int64_t N) {
  return 8 * cdiv(cdiv(M, 256) * cdiv(N, 256), 256) <= 5 * cdiv(cdiv(M, 128) * cdiv(N, 128), 512);
}

// For [M][N] sums over K: the large tile or the one of a quarter of its size, narrow ones where a
// side is short, and parts of the reduction where that leaves the chip idle.
inline Plan plan(int64_t M, int64_t N, int64_t K) {
  Plan p;
  int64_t slots;  // workgroups that the chip holds at once
  if (M <= 32) {
    p = {k32x256, 1, cdiv(N, 256), 1, 0};
    slots = 512;
  } else if (N <= 32) {
    p = {k256x32, cdiv(M, 256), 1, 1, 0};
    slots = 512;
  } else if (large_pays(M, N)) {
    p = {k256, cdiv(M, 256), cdiv(N, 256), 1, 0};
    slots = 256;
  } else {
    p = {k128, cdiv(M, 128), cdiv(N, 128), 1, 0};
    slots = 512;
  }
  const int64_t tiles = p.mt * p.nt;
  const int64_t most = cdiv(K, 128);
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
