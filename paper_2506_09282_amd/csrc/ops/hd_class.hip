// Softmax cross entropy of given classes straight from encodings H[N][D] and class vectors
// C[K][D], and its gradient, without the scores S = H C^T ever being kept:
//
//   s_k = <H_n, C_k>,  m = max s_k,  L = log sum exp(scale (s_k - m)),
//   loss = L - scale (s_y - m)
//   dS = g scale (p - 1[k = y]),  p = exp(scale (s_k - m) - L);   dH = dS C,  dC = dS^T H
//
// A tile of scores stays in its workgroup's registers: the forward pass leaves of it each row's
// maximum and sum over the tile's classes (joined by a second launch) and the score asked for; the
// backward pass computes it again and leaves dS, of as many classes at a time as fit
// kPieceBytes, which the two products then read. Classes are the instruction's rows, so
// that a lane holds 16 classes of one sample and most of a row's maximum and sum needs no
// exchange between lanes.
//
// Many classes are bound by the large tile's pace: a forward pass of 4096 x 131072 by 4096 bf16 takes 3.7 to
// 3.9 ms, a backward pass of 4096 x 65536 by 4096 10.2 to 10.6 ms (1.04 to 1.08 PFLOP/s of its five
// products, two of them for the rest of dS). Few
// classes are bound by reading H, once forward and twice backward: 16384 x 10240 fp32 under 26
// classes 114 and 258 us (5.9 and 5.2 TB/s).
//
// Where there are too few tiles for the chip (few rows and classes), the reduction over D is
// split and the parts of the (then small) score matrix go through the workspace.
#include <type_traits>

#include "hd_tile.hpp"

namespace hd {
namespace ops {

namespace {

using tile::Bf16;
using tile::die_order;
using tile::F32;
using tile::kCols;
using tile::kRows;
using tile::Operand;
using tile::Plan;
using tile::Tile;
using tile::tile_at;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kThreads = 256;

// Scores' gradients kept at a time, in whole tiles of 256 classes (1 KiB a row at least, which is more
// than this from 131072 rows on). 128 MiB stay in the last cache (256 MB) between the launch that
// writes them and the two that read them.
constexpr int64_t kPieceBytes = int64_t(128) << 20;

// bf16 values that hold one of dS: two for the bf16 products, within 2^-16 of it. One is not enough
// at any size: while the class vectors are nearly equal (before the first refining step) every row's dS
// is rounded alike, and the gradients cancel what the encodings, or the class vectors, have in
// common, but not what was rounded off with it (4096 rows with a shared component under 10 equal
// classes: errors of dC 31 times its own rounding). The second value costs the products a second
// pass over each stage (4096 x 65536 by 4096 10.2 ms instead of 6.3; 16384 x 10240 under 26 classes,
// their gradient alone, 150 us instead of 123).
template <typename T>
constexpr int kValues = sizeof(T) == 2 ? 2 : 1;

struct Scores {  // of the classes [0, K) of a piece
  Operand H, C;
  const int32_t* y;
  const uint64_t* open;  // a bit for each class (null: all are open)
  float scale;
  int64_t N, D, K;
  int64_t first;  // the piece's first class (of y)
  uint32_t mt, nt;
};

// Of 32 classes from k on, those that take part.
__device__ __forceinline__ uint32_t open_bits(const Scores& a, int64_t k) {
  const int64_t left = a.K - k;
  if (left <= 0) return 0u;
  uint32_t bits = left < 32 ? (1u << left) - 1u : ~0u;
  if (a.open) bits &= (uint32_t)(a.open[k >> 6] >> (k & 32));
  return bits;
}

__device__ __forceinline__ bool asked(int32_t y, int64_t K) { return y >= 0 && y < K; }

// A row's maximum and sum of exp2(c (s - m)) over two sets of classes.
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2, float c) {
  const float top = fmaxf(m, m2);
  const float at = top == -INFINITY ? 0.0f : top;  // (nothing takes part: sums of 0 stay 0)
  s = s * exp2f(c * (m - at)) + s2 * exp2f(c * (m2 - at));
  m = top;
}

// m and log of the sum to what the caller gets; NaN and +inf among the scores give NaN.
__device__ __forceinline__ void finish_row(float m, float s, float target, bool asks, float scale,
                                           float* loss, float* stats) {
  float L = logf(s), at = m;
  if (m == -INFINITY && s == 0.0f) {  // no class
    L = 0.0f;
    *loss = asks ? INFINITY : 0.0f;
  } else {
    if (s != s || m == INFINITY) at = L = NAN;
    *loss = asks ? L - scale * (target - at) : 0.0f;
  }
  stats[0] = at;
  stats[1] = L;
}

// ---- forward ----------------------------------------------------------------------

// parts[n][class tile] = {maximum, sum}, target[n] = the score asked for.
template <class TL>
__global__ __launch_bounds__(TL::T, 2) void class_loss_kernel(
    Scores a, float2* __restrict__ parts, float* __restrict__ target) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  uint32_t mi, ni;
  tile_at(die_order(blockIdx.x, gridDim.x), a.mt, a.nt, mi, ni);
  const int64_t m0 = (int64_t)mi * TL::BM, n0 = (int64_t)ni * TL::BN;
  typename TL::Acc c[TL::MT][TL::NT];
  TL::product(a.C, a.H, m0, n0, 0, a.D, lds, c);

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const int wm = wave / TL::WN, wn = wave % TL::WN;
  const float scale2 = a.scale * kLog2e;
  const bool all_open = !a.open && m0 + TL::BM <= a.K;
  float2* part = reinterpret_cast<float2*>(lds);  // [WM][BN]
#pragma unroll
  for (int j = 0; j < TL::NT; ++j) {
    const int col = (wn * TL::NT + j) * 32 + (lane & 31);
    const int64_t n = n0 + col;
    const int32_t y = n < a.N ? a.y[n] : -1;
    const int64_t at = (int64_t)y - m0 - wm * TL::MT * 32;
    const bool here = y >= 0 && y < a.K && at >= 0 && at < TL::MT * 32;
    if (!all_open) {
#pragma unroll
      for (int i = 0; i < TL::MT; ++i) {
        uint32_t bits = open_bits(a, m0 + (wm * TL::MT + i) * 32) >> (4 * half);
        // (worked out for each column again: kept, the lanes' conditions fill the registers)
        asm volatile("" : "+v"(bits));
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (!(bits >> ((r / 4) * 8 + r % 4) & 1)) c[i][j][r] = -INFINITY;
      }
    }
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < TL::MT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) m = fmaxf(m, c[i][j][r]);
    if (here) {  // one of the two lanes of a sample holds the score asked for
      int place = (int)at;
      place = ((place >> 2) & 1) == half ? (place >> 5) * 16 + ((place & 31) >> 3) * 4 + (place & 3)
                                         : -1;
      asm volatile("" : "+v"(place));
      float t = 0.0f;
#pragma unroll
      for (int i = 0; i < TL::MT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) t = place == i * 16 + r ? c[i][j][r] : t;
      if (place >= 0) target[n] = t;
    }
    const float base = m == -INFINITY ? 0.0f : m;
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < TL::MT; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) s += exp2f(scale2 * (c[i][j][r] - base));
    join(m, s, lane_xor<32>(m), lane_xor<32>(s), scale2);
    if (half == 0) part[wm * TL::BN + col] = make_float2(m, s);
  }
  __syncthreads();
  for (int col = threadIdx.x; col < TL::BN; col += TL::T) {
    float2 x = part[col];
#pragma unroll
    for (int w = 1; w < TL::WM; ++w) {
      const float2 z = part[w * TL::BN + col];
      join(x.x, x.y, z.x, z.y, scale2);
    }
    if (n0 + col < a.N) parts[(n0 + col) * a.mt + mi] = x;
  }
}

// A wave joins the parts of a row.
__global__ __launch_bounds__(kThreads) void class_join_kernel(
    const float2* __restrict__ parts, const float* __restrict__ target,
    const int32_t* __restrict__ y, int64_t N, int64_t K, int tiles, float scale,
    float* __restrict__ loss, float* __restrict__ stats) {
  const int64_t n = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
  if (n >= N) return;
  const int lane = threadIdx.x & 63;
  const float scale2 = scale * kLog2e;
  float m = -INFINITY, s = 0.0f;
  for (int t = lane; t < tiles; t += 64) {
    const float2 x = parts[n * tiles + t];
    join(m, s, x.x, x.y, scale2);
  }
  join(m, s, lane_xor<1>(m), lane_xor<1>(s), scale2);
  join(m, s, lane_xor<2>(m), lane_xor<2>(s), scale2);
  join(m, s, lane_xor<4>(m), lane_xor<4>(s), scale2);
  join(m, s, lane_xor<8>(m), lane_xor<8>(s), scale2);
  join(m, s, lane_xor<16>(m), lane_xor<16>(s), scale2);
  join(m, s, lane_xor<32>(m), lane_xor<32>(s), scale2);
  if (lane == 0) {
    const bool asks = asked(y[n], K);
    finish_row(m, s, asks ? target[n] : 0.0f, asks, scale, loss + n, stats + 2 * n);
  }
}

// ---- the scores in parts of D, where there are few ----------------------------------

// out[part][n][class], rows of mt * BM classes.
template <class TL>
__global__ __launch_bounds__(TL::T, 2) void class_scores_kernel(Scores a, int64_t each,
                                                                float* __restrict__ out) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const uint32_t tiles = a.mt * a.nt;
  const uint32_t id = die_order(blockIdx.x, gridDim.x), part = id / tiles;
  uint32_t mi, ni;
  tile_at(id % tiles, a.mt, a.nt, mi, ni);
  const int64_t m0 = (int64_t)mi * TL::BM, n0 = (int64_t)ni * TL::BN;
  const int64_t k0 = part * each, k1 = k0 + each < a.D ? k0 + each : a.D;
  typename TL::Acc c[TL::MT][TL::NT];
  TL::product(a.C, a.H, m0, n0, k0, k1, lds, c);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const int wm = wave / TL::WN, wn = wave % TL::WN;
  const int64_t ld = (int64_t)a.mt * TL::BM;
#pragma unroll
  for (int j = 0; j < TL::NT; ++j) {
    const int64_t n = n0 + (wn * TL::NT + j) * 32 + (lane & 31);
    if (n >= a.N) continue;
    float* row = out + ((int64_t)part * a.N + n) * ld + m0 + wm * TL::MT * 32 + half * 4;
#pragma unroll
    for (int i = 0; i < TL::MT; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(row + i * 32 + q * 8) =
            f32x4{c[i][j][4 * q], c[i][j][4 * q + 1], c[i][j][4 * q + 2], c[i][j][4 * q + 3]};
  }
}

struct Parts {
  const float* p;  // [count][N][ld], ld a multiple of 4
  int64_t ld, N;
  int count;
};
// Four scores of a row, of every `step`-th part from `first` on.
__device__ __forceinline__ f32x4 scores_of(const Parts& s, int64_t n, int64_t k, int first,
                                           int step) {
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  const float* at = s.p + (first * s.N + n) * s.ld + k;
#pragma unroll 8
  for (int i = first; i < s.count; i += step, at += step * s.N * s.ld)
    v += *reinterpret_cast<const f32x4*>(at);
  return v;
}
// The sum over PG groups of threads that each hold every PG-th part; `lane` of `lanes` in a
// group. All threads call it; the first group has the sums.
template <int PG>
__device__ __forceinline__ f32x4 join_groups(f32x4 v, int group, int lane, int lanes, f32x4* lds) {
  if constexpr (PG > 1) {
    lds[group * lanes + lane] = v;
    __syncthreads();
    if (group == 0) {
#pragma unroll
      for (int g = 1; g < PG; ++g) v += lds[g * lanes + lane];
    }
  }
  return v;
}

// A bit for each of four classes from k on that takes part. (Without a branch: this compiler has
// lost the values of short-circuited conditions that write parts of a vector.)
__device__ __forceinline__ uint32_t open4(const uint8_t* mask, int64_t k, int64_t K) {
  uint32_t bits = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t at = k + e < K ? k + e : K - 1;
    const uint32_t open = mask ? (uint32_t)(mask[at] != 0) : 1u;
    bits |= (open & (uint32_t)(k + e < K)) << e;
  }
  return bits;
}

// m and s of a row over 2^x neighbouring lanes.
template <int LANES>
__device__ __forceinline__ void join_lanes(float& m, float& s, float c) {
  join(m, s, lane_xor<1>(m), lane_xor<1>(s), c);
  join(m, s, lane_xor<2>(m), lane_xor<2>(s), c);
  join(m, s, lane_xor<4>(m), lane_xor<4>(s), c);
  if constexpr (LANES > 8) {
    join(m, s, lane_xor<8>(m), lane_xor<8>(s), c);
    join(m, s, lane_xor<16>(m), lane_xor<16>(s), c);
    join(m, s, lane_xor<32>(m), lane_xor<32>(s), c);
  }
}

// A row's loss from the parts of its scores. G lanes take four classes each (G = 256: kChunk classes
// of the row, one of gridDim.y pieces that class_join_kernel joins; else G lanes cover the row), PG
// groups of them share the parts.
constexpr int64_t kChunk = 4096;

template <int G, int PG>
__global__ __launch_bounds__(kThreads) void class_rows_kernel(
    Parts sc, const int32_t* __restrict__ y, const uint8_t* __restrict__ mask, int64_t K,
    float scale, float* __restrict__ loss, float* __restrict__ stats, float2* __restrict__ pieces,
    float* __restrict__ targets) {
  constexpr int kRowsOf = kThreads / (G * PG);
  __shared__ f32x4 sums[PG > 1 ? kThreads : 1];
  __shared__ float2 part[kThreads / 64];
  __shared__ float target[kRowsOf];
  const int lane = threadIdx.x % G, group = threadIdx.x / G % PG, row = threadIdx.x / (G * PG);
  const int64_t at = (int64_t)blockIdx.x * kRowsOf + row;
  const bool there = at < sc.N;  // (all threads meet at the barriers)
  const int64_t n = there ? at : sc.N - 1;
  const int32_t yn = y[n];
  const bool asks = asked(yn, K);
  const float scale2 = scale * kLog2e;
  float m = -INFINITY, s = 0.0f;
  const int64_t k1 = G > 64 && (blockIdx.y + 1) * kChunk < K ? (blockIdx.y + 1) * kChunk : K;
  for (int64_t k0 = G > 64 ? blockIdx.y * kChunk : 0; k0 < k1; k0 += 4 * G) {
    const int64_t k = k0 + 4 * lane;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (k < K) v = scores_of(sc, n, k, group, PG);
    v = join_groups<PG>(v, group, lane, G, sums);
    const uint32_t bits = open4(mask, k, K);
    float x[4], top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = bits >> e & 1 ? v[e] : -INFINITY;
      top = fmaxf(top, x[e]);
    }
    const int64_t place = (int64_t)yn - k;
    if (asks & (group == 0) & (place >= 0) & (place < 4)) {
      const float t = place < 2 ? (place == 0 ? x[0] : x[1]) : (place == 2 ? x[2] : x[3]);
      if (G > 64 && pieces)
        targets[n] = t;
      else
        target[row] = t;
    }
    const float base = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) sum += exp2f(scale2 * (x[e] - base));
    join(m, s, top, sum, scale2);
  }
  join_lanes<(G < 64 ? G : 64)>(m, s, scale2);
  if constexpr (G > 64)
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = make_float2(m, s);
  __syncthreads();
  if constexpr (G > 64) {
    m = part[0].x;
    s = part[0].y;
    for (int w = 1; w < kThreads / 64; ++w) join(m, s, part[w].x, part[w].y, scale2);
  }
  if (G > 64 && pieces) {
    if (threadIdx.x == 0) pieces[n * gridDim.y + blockIdx.y] = make_float2(m, s);
  } else if (there && lane == 0 && group == 0)
    finish_row(m, s, asks ? target[row] : 0.0f, asks, scale, loss + n, stats + 2 * n);
}

// ---- backward: the scores' gradient ---------------------------------------------------

struct RowGrad {
  float m, shift, g;  // p = exp2(c (s - m) - shift), dS = g (p - 1[k = y])
  int64_t y;          // of the piece; far outside where no class is asked for
  bool on;
};
__device__ __forceinline__ RowGrad row_grad(const Scores& a, const float* stats, const float* g,
                                            int64_t K_all, int64_t n) {
  RowGrad r;
  const float m = stats[2 * n];
  r.on = asked(a.y[n], K_all);
  r.m = m == -INFINITY ? 0.0f : m;
  r.shift = stats[2 * n + 1] * kLog2e;
  r.g = g[n] * a.scale;
  r.y = (int64_t)a.y[n] - a.first;
  return r;
}
__device__ __forceinline__ float score_grad(const RowGrad& r, float s, int64_t k, bool open,
                                            float scale2) {
  // a score of -inf takes no part: its p is 0, also where it is asked for
  float p = exp2f(scale2 * (s - r.m) - r.shift);
  if (k == r.y && s != -INFINITY) p -= 1.0f;
  return r.on && open ? r.g * p : 0.0f;
}

// What a value's rounding to bf16 leaves of it (nothing of an infinity, which stays one).
__device__ __forceinline__ float rest_of(float d) {
  const float hi = bf16_to_f32(to_bf16(d));
  return fabsf(hi) == INFINITY ? 0.0f : d - hi;
}

// dS[value][n][class] of a piece, rows of ld elements.
template <class TL>
__global__ __launch_bounds__(TL::T, 2) void class_dscores_kernel(
    Scores a, int64_t K_all, const float* __restrict__ stats, const float* __restrict__ g,
    typename TL::P::elem* __restrict__ dS, int64_t ld) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  uint32_t mi, ni;
  tile_at(die_order(blockIdx.x, gridDim.x), a.mt, a.nt, mi, ni);
  const int64_t m0 = (int64_t)mi * TL::BM, n0 = (int64_t)ni * TL::BN;
  typename TL::Acc c[TL::MT][TL::NT];
  TL::product(a.C, a.H, m0, n0, 0, a.D, lds, c);
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));  // (nothing of what follows is worked out before the product)
  const int lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  const int wm = wave / TL::WN, wn = wave % TL::WN;
  const float scale2 = a.scale * kLog2e;
  typedef typename TL::P::elem T;
  // [32 samples][up to 256 bytes of the wave's classes, first values before second], so that the
  // stores run along the rows
  constexpr int kV = kValues<T>, kMost = 256 / (32 * sizeof(T) * kV);
  constexpr int kTiles = TL::MT > kMost ? kMost : TL::MT;
  constexpr int kAcross = kTiles * 32, kPitch = kV * kAcross + 16 / sizeof(T);
  static_assert(TL::MT % kTiles == 0 && TL::WM * TL::WN * 32 * kPitch * sizeof(T) <= TL::kLds, "");
  T* mine = reinterpret_cast<T*>(lds) + wave * 32 * kPitch;
#pragma unroll
  for (int j = 0; j < TL::NT; ++j) {
    const int64_t nw = n0 + (wn * TL::NT + j) * 32, n = nw + (lane & 31);
    const RowGrad row = row_grad(a, stats, g, K_all, n < a.N ? n : a.N - 1);
#pragma unroll
    for (int i0 = 0; i0 < TL::MT; i0 += kTiles) {
      const int64_t first = m0 + (wm * TL::MT + i0) * 32;
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        uint32_t bits = open_bits(a, first + i * 32);
        asm volatile("" : "+v"(bits));  // (worked out for each column again)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int at = q * 8 + half * 4 + e;
            v[e] = score_grad(row, c[i0 + i][j][4 * q + e], first + i * 32 + at, bits >> at & 1,
                              scale2);
          }
          const int at = (lane & 31) * kPitch + i * 32 + q * 8 + half * 4;
          store_four(mine, at, v, 4);
          if constexpr (kV > 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = rest_of(v[e]);
            store_four(mine, at + kAcross, v, 4);
          }
          __builtin_amdgcn_sched_barrier(0);  // (four at a time: the registers hold the sums)
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      // (ld is a multiple of 8: a piece of 16 bytes fits or begins past it)
      constexpr int kE = 16 / sizeof(T), kPieces = kAcross / kE;
      int q0 = threadIdx.x & 63;
      asm volatile("" : "+v"(q0));
#pragma unroll 1
      for (int q = q0; q < 32 * kV * kPieces; q += 64) {
        const int r = q / (kV * kPieces), piece = q % (kV * kPieces);
        const int value = piece / kPieces, k = piece % kPieces * kE;
        if (nw + r < a.N && first + k < ld)
          *reinterpret_cast<u32x4*>(dS + (value * a.N + nw + r) * ld + first + k) =
              *reinterpret_cast<const u32x4*>(mine + r * kPitch + value * kAcross + k);
      }
    }
  }
}

// Bits of the rows that ask for a class (word w of them), then of the open classes; a wave to a
// word. Either may be null.
__device__ __forceinline__ void write_bits(int64_t w, const int32_t* y, int64_t N, uint64_t* rows,
                                           const uint8_t* mask, int64_t K, uint64_t* classes) {
  const int lane = threadIdx.x & 63;
  const int64_t row_words = rows ? cdiv(N, 64) : 0;
  if (w < row_words) {
    const int64_t n = w * 64 + lane;
    const uint64_t b = __builtin_amdgcn_ballot_w64(n < N && asked(y[n], K));
    if (lane == 0) rows[w] = b;
    return;
  }
  w -= row_words;
  if (!classes || w >= cdiv(K, 64)) return;
  const int64_t k = w * 64 + lane;
  const uint64_t b = __builtin_amdgcn_ballot_w64(k < K && mask[k] != 0);
  if (lane == 0) classes[w] = b;
}
__global__ __launch_bounds__(kThreads) void class_bits_kernel(const int32_t* __restrict__ y,
                                                              int64_t N, uint64_t* rows,
                                                              const uint8_t* __restrict__ mask,
                                                              int64_t K, uint64_t* classes) {
  write_bits((int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6), y, N, rows, mask, K,
             classes);
}

// dS from the parts of the scores (all classes); a thread takes four classes of a row, PG groups
// of threads share the parts. The blocks behind them write the bits.
template <typename T, int PG>
__global__ __launch_bounds__(kThreads) void class_dscores_parts_kernel(
    Scores a, Parts sc, const float* __restrict__ stats, const float* __restrict__ g,
    T* __restrict__ dS, int64_t ld, const uint8_t* __restrict__ mask, uint32_t blocks, uint64_t* rows,
    uint64_t* classes) {
  constexpr int kLanes = kThreads / PG;
  __shared__ f32x4 sums[PG > 1 ? kThreads : 1];
  if (blockIdx.x >= blocks) {
    write_bits((int64_t)(blockIdx.x - blocks) * (kThreads / 64) + (threadIdx.x >> 6), a.y, a.N,
               rows, mask, a.K, classes);
    return;
  }
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const int64_t at = (int64_t)blockIdx.x * kLanes + lane, quads = ld / 4;
  const int64_t n = at / quads, k = (at - n * quads) * 4;
  const bool there = n < a.N;
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  if (there && k < a.K) v = scores_of(sc, n, k, group, PG);
  v = join_groups<PG>(v, group, lane, kLanes, sums);
  if (!there || group != 0) return;
  const RowGrad row = row_grad(a, stats, g, a.K, n);
  const uint32_t bits = open4(mask, k, a.K);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float d = score_grad(row, v[e], k + e, bits >> e & 1, a.scale * kLog2e);
    store_elem(dS, n * ld + k + e, d);
    if (kValues<T> > 1)
      store_elem(dS, (a.N + n) * ld + k + e, rest_of(d));
  }
}

// ---- backward: the products -------------------------------------------------------------

// Where a product goes: its part of the reduction to parts[part][M][N], or, added to
// `before` where there is one, to sums (fp32) or out. All are contiguous.
struct Out {
  void* out;
  float *sums, *parts;
  const float* before;
  int64_t M, N;
};

template <typename T>
__device__ __forceinline__ void put(const Out& o, int64_t at, f32x4 v, int64_t n) {
  if (o.before) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += o.before[e < n ? at + e : at];
  }
  if (o.sums)
    store_four(o.sums, at, v, n);
  else
    store_four(reinterpret_cast<T*>(o.out), at, v, n);
}

struct Product {  // out = a b over K, tile by tile and part by part
  Operand a, b;
  int64_t K, each;
  uint32_t mt, nt;
  Out o;
};

template <class TL>
__device__ __forceinline__ void product_tile(const Product& p, uint32_t id, char* lds) {
  const uint32_t tiles = p.mt * p.nt, part = id / tiles;
  uint32_t mi, ni;
  tile_at(id % tiles, p.mt, p.nt, mi, ni);
  const int64_t m0 = (int64_t)mi * TL::BM, n0 = (int64_t)ni * TL::BN;
  const int64_t k0 = part * p.each, k1 = k0 + p.each < p.K ? k0 + p.each : p.K;
  typename TL::Acc c[TL::MT][TL::NT];
  TL::product(p.a, p.b, m0, n0, k0, k1, lds, c);
  const Out& o = p.o;
  float* to = o.parts ? o.parts + (int64_t)part * o.M * o.N : nullptr;
  TL::rows_out(c, lds, m0, n0, [&](int64_t m, int64_t n, const f32x4& v) {
    if (m >= o.M || n >= o.N) return;
    if (to)
      store_four(to, m * o.N + n, v, o.N - n);
    else
      put<typename TL::P::elem>(o, m * o.N + n, v, o.N - n);
  });
}

template <class TL>
__global__ __launch_bounds__(TL::T, 2) void class_product_kernel(Product p) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  product_tile<TL>(p, die_order(blockIdx.x, gridDim.x), lds);
}

// Two products in one launch: the first `blocks` workgroups take p's tiles, the others q's.
template <class TL, class TQ>
__global__ __launch_bounds__(TL::T, 2) void class_products_kernel(Product p, uint32_t blocks,
                                                                  Product q) {
  static_assert(TL::T == TQ::T, "");
  extern __shared__ __attribute__((aligned(16))) char lds[];
  if (blockIdx.x < blocks)
    product_tile<TL>(p, blockIdx.x, lds);
  else
    product_tile<TQ>(q, blockIdx.x - blocks, lds);
}

// The parts' sum, four values to a thread, the parts shared by PG groups of threads.
template <typename T, int PG>
__global__ __launch_bounds__(kThreads) void class_sum_kernel(Out o, int count, uint32_t blocks,
                                                             Out o2, int count2) {
  constexpr int kLanes = kThreads / PG;
  __shared__ f32x4 sums[PG > 1 ? kThreads : 1];
  const bool second = blockIdx.x >= blocks;  // (another sum behind the first)
  if (second) {
    o = o2;
    count = count2;
  }
  const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
  const int64_t each = o.M * o.N;
  const int64_t at = ((int64_t)(blockIdx.x - (second ? blocks : 0)) * kLanes + lane) * 4;
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  if (at + 4 <= each) {
    const float* p = o.parts + group * each + at;
#pragma unroll 8
    for (int i = group; i < count; i += PG, p += PG * each)
      v += *reinterpret_cast<const f32x4_a4*>(p);
  } else if (at < each) {
    for (int i = group; i < count; i += PG) {
      const float* p = o.parts + i * each + at;
      v += f32x4{p[0], at + 1 < each ? p[1] : 0.0f, at + 2 < each ? p[2] : 0.0f, 0.0f};
    }
  }
  v = join_groups<PG>(v, group, lane, kLanes, sums);
  if (group == 0 && at < each) put<T>(o, at, v, each - at);
}

// ---- host -------------------------------------------------------------------------------

template <auto KERNEL>
hipError_t allow_lds(int bytes) {
  static PerDeviceOnce once;
  return once_per_device(once, [&] {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL),
                               hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  });
}

template <auto KERNEL, class TL, typename... A>
hipError_t launch_tiles(int64_t blocks, hipStream_t stream, A... args) {
  const hipError_t e = allow_lds<KERNEL>(TL::kLds);
  if (e != hipSuccess) return e;
  KERNEL<<<dim3((uint32_t)blocks), dim3(TL::T), TL::kLds, stream>>>(args...);
  return hipGetLastError();
}

// f is called with the tile of a plan.
template <class P, int AK, int BK, class F>
hipError_t with_tile(const Plan& p, const Operand& a, const Operand& b, F f) {
  // fp32 on the bf16 instruction where the matrix instructions bound the tile
  typedef std::conditional_t<std::is_same_v<P, F32>, tile::X3, P> Q;
  const bool once = tile::once(p, a, b, P::kEs);
  switch (p.shape) {
    case tile::k256: return f(Tile<Q, AK, BK, 256, 256, 2, 4>());
    case tile::k128: return f(Tile<Q, AK, BK, 128, 128, 2, 2>());
    case tile::k32x256:
      return once ? f(Tile<P, AK, BK, 32, 256, 1, 4, true>()) : f(Tile<P, AK, BK, 32, 256, 1, 4>());
    default:
      return once ? f(Tile<P, AK, BK, 256, 32, 4, 1, true>()) : f(Tile<P, AK, BK, 256, 32, 4, 1>());
  }
}

int64_t tile_m(const Plan& p) {
  return p.shape == tile::k32x256 ? 32 : p.shape == tile::k128 ? 128 : 256;
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

// How a call cuts its classes: one piece where the scores go through the workspace in
// parts, else as many classes as kPieceBytes hold.
int64_t piece_of(int64_t N, int64_t K, int64_t each) {
  int64_t k = kPieceBytes / (N * each) / 256 * 256;
  if (k < 256) k = 256;
  return k < K ? k : K;
}

struct LossPlace {
  Plan s;
  size_t open, parts, pieces, target, total;
};
LossPlace loss_place(int64_t N, int64_t D, int64_t K) {
  LossPlace w;
  w.s = tile::plan(K, N, D);
  w.open = 0;
  w.parts = up((size_t)cdiv(K, 64) * 8);
  if (w.s.splits > 1) {
    w.pieces = w.parts + up((size_t)w.s.splits * N * w.s.mt * tile_m(w.s) * 4);
    w.target = w.pieces + up((size_t)N * cdiv(K, kChunk) * 8);
    w.total = w.target + up((size_t)N * 4);
  } else {
    w.pieces = w.target = w.parts + up((size_t)N * w.s.mt * 8);
    w.total = w.target + up((size_t)N * 4);
  }
  return w;
}

struct GradPlace {
  int64_t piece, ld;  // classes at a time, and of a row of dS
  size_t rows, open, dS, scores, sums, parts, total;
};
template <typename T>
GradPlace grad_place(int64_t N, int64_t D, int64_t K, bool dH, bool dC) {
  GradPlace w;
  constexpr int64_t kEach = kValues<T> * sizeof(T);  // bytes of one of dS
  const Plan s = tile::plan(K, N, D);
  w.piece = s.splits > 1 ? K : piece_of(N, K, kEach);
  w.ld = cdiv(w.piece, 8) * 8;
  w.rows = 0;
  w.open = up((size_t)cdiv(N, 64) * 8);
  w.dS = w.open + up((size_t)cdiv(K, 64) * 8);
  w.scores = w.dS + up((size_t)N * w.ld * kEach);
  size_t at = w.scores;
  if (s.splits > 1) at += up((size_t)s.splits * N * s.mt * tile_m(s) * 4);
  w.sums = at;
  if (dH && w.piece < K) at += up((size_t)N * D * 4);
  w.parts = at;
  // (the last piece may be short, and its products split further)
  size_t most = 0;
  for (int64_t k : {w.piece, K - (K - 1) / w.piece * w.piece}) {
    const Plan h = tile::plan(N, D, k), c = tile::plan(k, D, N);
    most = std::max(most, (size_t)((dH && h.splits > 1 ? h.splits * N * D : 0) +
                                   (dC && c.splits > 1 ? c.splits * k * D : 0)) * 4);
  }
  w.total = at + up(most);
  return w;
}

template <class P>
hipError_t run_scores(const Scores& a, const Plan& p, float* parts, hipStream_t stream) {
  return with_tile<P, kRows, kRows>(p, a.C, a.H, [&](auto t) {
    typedef decltype(t) TL;
    if constexpr (TL::BM * TL::BN > 128 * 128)
      return hipErrorInvalidValue;  // (the large tile is not split)
    else
      return launch_tiles<class_scores_kernel<TL>, TL>(p.mt * p.nt * p.splits, stream, a, p.each,
                                                       parts);
  });
}

template <class P>
hipError_t run_loss(const ClassArgs& c, float* loss, float* stats, char* ws, hipStream_t stream) {
  const LossPlace w = loss_place(c.N, c.D, c.K);
  hipError_t e;
  uint64_t* open = nullptr;
  if (c.mask && w.s.splits == 1) {
    open = reinterpret_cast<uint64_t*>(ws + w.open);
    class_bits_kernel<<<dim3((uint32_t)cdiv(cdiv(c.K, 64), kThreads / 64)), dim3(kThreads), 0,
                        stream>>>(nullptr, 0, nullptr, c.mask, c.K, open);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  const Scores a{{c.H, c.ldh, c.N, nullptr}, {c.C, c.ldc, c.K, nullptr}, c.y, open, c.scale,
                 c.N, c.D, c.K, 0, (uint32_t)w.s.mt, (uint32_t)w.s.nt};
  const int64_t tiles = w.s.mt * w.s.nt;
  float* parts = reinterpret_cast<float*>(ws + w.parts);
  if (w.s.splits == 1) {
    float* target = reinterpret_cast<float*>(ws + w.target);
    e = with_tile<P, kRows, kRows>(w.s, a.C, a.H, [&](auto t) {
      typedef decltype(t) TL;
      return launch_tiles<class_loss_kernel<TL>, TL>(tiles, stream, a,
                                                     reinterpret_cast<float2*>(parts), target);
    });
    if (e != hipSuccess) return e;
    class_join_kernel<<<dim3((uint32_t)cdiv(c.N, kThreads / 64)), dim3(kThreads), 0, stream>>>(
        reinterpret_cast<const float2*>(parts), target, c.y, c.N, c.K, (int)w.s.mt, c.scale, loss,
        stats);
    return hipGetLastError();
  }
  if ((e = run_scores<P>(a, w.s, parts, stream)) != hipSuccess) return e;
  const Parts sc{parts, w.s.mt * tile_m(w.s), c.N, (int)w.s.splits};
  const int chunks = c.K > 256 ? (int)cdiv(c.K, kChunk) : 1;
  float2* pieces = chunks > 1 ? reinterpret_cast<float2*>(ws + w.pieces) : nullptr;
  float* targets = reinterpret_cast<float*>(ws + w.target);
  auto rows = [&](auto* kernel, int each) {
    kernel<<<dim3((uint32_t)cdiv(c.N, each), (uint32_t)chunks), dim3(kThreads), 0, stream>>>(
        sc, c.y, c.mask, c.K, c.scale, loss, stats, pieces, targets);
    return hipGetLastError();
  };
  // Many parts are those of few rows: a workgroup to a row shares them.
  const bool many = sc.count > 8;
  if (c.K <= 32)
    return many ? rows(class_rows_kernel<8, 32>, 1) : rows(class_rows_kernel<8, 1>, 32);
  if (c.K <= 256)
    return many ? rows(class_rows_kernel<64, 4>, 1) : rows(class_rows_kernel<64, 1>, 4);
  e = rows(class_rows_kernel<256, 1>, 1);
  if (e != hipSuccess || chunks == 1) return e;
  class_join_kernel<<<dim3((uint32_t)cdiv(c.N, kThreads / 64)), dim3(kThreads), 0, stream>>>(
      pieces, targets, c.y, c.N, c.K, chunks, c.scale, loss, stats);
  return hipGetLastError();
}

struct Job {
  Plan plan;
  Product p;
  int64_t blocks() const { return plan.mt * plan.nt * plan.splits; }
};
Job job(const Operand& a, const Operand& b, int64_t K, Out o, float* parts) {
  const Plan p = tile::plan(o.M, o.N, K);
  if (p.splits > 1) o.parts = parts;
  return {p, {a, b, K, p.each, (uint32_t)p.mt, (uint32_t)p.nt, o}};
}

template <class P>
hipError_t sum_parts(const Job* x, const Job* y, hipStream_t stream) {
  typedef typename P::elem T;
  if (x && x->plan.splits == 1) x = nullptr;
  if (y && y->plan.splits == 1) y = nullptr;
  if (!x) std::swap(x, y);
  if (!x) return hipSuccess;
  const int count = (int)x->plan.splits, count2 = y ? (int)y->plan.splits : 0;
  const Out o = x->p.o, o2 = y ? y->p.o : o;
  auto sum = [&](auto* kernel, int groups) {
    const int64_t each = 4 * kThreads / groups;
    const int64_t blocks = cdiv(o.M * o.N, each), more = y ? cdiv(o2.M * o2.N, each) : 0;
    kernel<<<dim3((uint32_t)(blocks + more)), dim3(kThreads), 0, stream>>>(
        o, count, (uint32_t)blocks, o2, count2);
    return hipGetLastError();
  };
  return std::max(count, count2) > 8 ? sum(class_sum_kernel<T, 8>, 8)
                                     : sum(class_sum_kernel<T, 1>, 1);
}

template <class P, int AK, int BK>
hipError_t run_product(const Job& w, hipStream_t stream) {
  return with_tile<P, AK, BK>(w.plan, w.p.a, w.p.b, [&](auto t) {
    typedef decltype(t) TL;
    return launch_tiles<class_product_kernel<TL>, TL>(w.blocks(), stream, w.p);
  });
}

// Both gradients' products. Short ones share a launch, in which neither waits for the other's last
// tiles (300 rows by 20 classes, D = 512: 26 us a call instead of 33; 64 by 100, D = 10240: 28 instead of
// 38; the large tile and long products gain nothing).
constexpr int64_t kSharedBlocks = 1024;
template <class P>
hipError_t run_products(const Job* c, const Job* h, hipStream_t stream) {
  hipError_t e;
  if (c && h && c->blocks() + h->blocks() <= kSharedBlocks && c->plan.shape != tile::k256 &&
      h->plan.shape != tile::k256 && c->plan.shape != tile::k256x32 &&
      h->plan.shape != tile::k256x32) {
    typedef std::conditional_t<std::is_same_v<P, F32>, tile::X3, P> Q;
    typedef Tile<Q, kCols, kCols, 128, 128, 2, 2> C128;
    typedef Tile<P, kCols, kCols, 32, 256, 1, 4> C32;
    typedef Tile<Q, kRows, kCols, 128, 128, 2, 2> H128;
    typedef Tile<P, kRows, kCols, 32, 256, 1, 4> H32;
    auto both = [&](auto t, auto u) {
      typedef decltype(t) TC;
      typedef decltype(u) TH;
      constexpr int kLds = TC::kLds > TH::kLds ? TC::kLds : TH::kLds;
      const hipError_t err = allow_lds<class_products_kernel<TC, TH>>(kLds);
      if (err != hipSuccess) return err;
      class_products_kernel<TC, TH>
          <<<dim3((uint32_t)(c->blocks() + h->blocks())), dim3(TC::T), kLds, stream>>>(
              c->p, (uint32_t)c->blocks(), h->p);
      return hipGetLastError();
    };
    const bool c32 = c->plan.shape == tile::k32x256, h32 = h->plan.shape == tile::k32x256;
    e = c32 ? h32 ? both(C32(), H32()) : both(C32(), H128())
            : h32 ? both(C128(), H32()) : both(C128(), H128());
    return e != hipSuccess ? e : sum_parts<P>(c, h, stream);
  }
  if (c) {
    if ((e = run_product<P, kCols, kCols>(*c, stream)) != hipSuccess) return e;
    if ((e = sum_parts<P>(c, nullptr, stream)) != hipSuccess) return e;
  }
  if (!h) return hipSuccess;
  e = run_product<P, kRows, kCols>(*h, stream);
  return e != hipSuccess ? e : sum_parts<P>(h, nullptr, stream);
}

template <class P>
hipError_t run_grad(const ClassArgs& c, const float* stats, const float* g, void* dH, void* dC,
                    char* ws, hipStream_t stream) {
  typedef typename P::elem T;
  const GradPlace w = grad_place<T>(c.N, c.D, c.K, dH != nullptr, dC != nullptr);
  uint64_t* rows = reinterpret_cast<uint64_t*>(ws + w.rows);
  uint64_t* open = reinterpret_cast<uint64_t*>(ws + w.open);
  if (!dC) rows = nullptr;
  if (!c.mask) open = nullptr;
  // (in one piece the scores' parts may be summed by a launch that writes the bits too)
  const Plan whole = tile::plan(c.K, c.N, c.D);
  const uint32_t bit_blocks = (uint32_t)cdiv((rows ? cdiv(c.N, 64) : 0) + (open ? cdiv(c.K, 64) : 0),
                                             kThreads / 64);
  hipError_t e;
  if (whole.splits == 1 && bit_blocks) {
    class_bits_kernel<<<dim3(bit_blocks), dim3(kThreads), 0, stream>>>(c.y, c.N, rows, c.mask, c.K,
                                                                       open);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  T* dS = reinterpret_cast<T*>(ws + w.dS);
  float* sums = reinterpret_cast<float*>(ws + w.sums);
  float* parts = reinterpret_cast<float*>(ws + w.parts);
  for (int64_t first = 0; first < c.K; first += w.piece) {
    const int64_t K = std::min(w.piece, c.K - first);
    const bool last = first + K == c.K;
    const uint64_t* part_open = open ? open + first / 64 : nullptr;
    const T* C = reinterpret_cast<const T*>(c.C) + first * c.ldc;
    Plan s = tile::plan(K, c.N, c.D);
    const int64_t tiles = s.mt * s.nt;
    if (w.piece < c.K) s.splits = 1;  // (a short last piece is computed whole)
    const Scores a{{c.H, c.ldh, c.N, nullptr}, {C, c.ldc, K, nullptr}, c.y, part_open, c.scale,
                   c.N, c.D, K, first, (uint32_t)s.mt, (uint32_t)s.nt};
    if (s.splits == 1) {
      e = with_tile<P, kRows, kRows>(s, a.C, a.H, [&](auto t) {
        typedef decltype(t) TL;
        return launch_tiles<class_dscores_kernel<TL>, TL>(tiles, stream, a, c.K, stats, g, dS,
                                                          w.ld);
      });
    } else {
      float* scores = reinterpret_cast<float*>(ws + w.scores);
      if ((e = run_scores<P>(a, s, scores, stream)) != hipSuccess) return e;
      const Parts sc{scores, s.mt * tile_m(s), c.N, (int)s.splits};
      auto sum = [&](auto* kernel, int groups) {
        const uint32_t blocks = (uint32_t)cdiv(c.N * w.ld / 4, kThreads / groups);
        kernel<<<dim3(blocks + bit_blocks), dim3(kThreads), 0, stream>>>(
            a, sc, stats, g, dS, w.ld, c.mask, blocks, rows, open);
        return hipGetLastError();
      };
      e = sc.count > 8 ? sum(class_dscores_parts_kernel<T, 8>, 8)
                       : sum(class_dscores_parts_kernel<T, 1>, 1);
    }
    if (e != hipSuccess) return e;
    const Out oc{reinterpret_cast<T*>(dC) + first * c.D, nullptr, nullptr, nullptr, K, c.D};
    const Out oh{dH, last ? nullptr : sums, nullptr, first ? sums : nullptr, c.N, c.D};
    const int64_t rest = kValues<T> > 1 ? c.N * w.ld * P::kEs : 0;
    const Job jc = job({dS, w.ld, K, nullptr, rest}, {c.H, c.ldh, c.D, rows}, c.N, oc, parts);
    const Job jh = job({dS, w.ld, c.N, nullptr, rest}, {C, c.ldc, c.D, part_open}, K, oh,
                       parts + (dC && jc.plan.splits > 1 ? jc.plan.splits * K * c.D : 0));
    if ((e = run_products<P>(dC ? &jc : nullptr, dH ? &jh : nullptr, stream)) != hipSuccess)
      return e;
  }
  return hipSuccess;
}

}  // namespace

size_t class_loss_ws_bytes(int64_t N, int64_t D, int64_t K) { return loss_place(N, D, K).total; }
size_t class_grad_ws_bytes(int64_t N, int64_t D, int64_t K, int dt, bool dH, bool dC) {
  return (dt == 0 ? grad_place<float>(N, D, K, dH, dC) : grad_place<bf16raw>(N, D, K, dH, dC)).total;
}

hipError_t launch_class_loss(const ClassArgs& a, float* loss, float* stats, void* workspace,
                             hipStream_t stream) {
  char* ws = reinterpret_cast<char*>(workspace);
  return a.dt == 0 ? run_loss<F32>(a, loss, stats, ws, stream)
                   : run_loss<Bf16>(a, loss, stats, ws, stream);
}
hipError_t launch_class_loss_grad(const ClassArgs& a, const float* stats, const float* g_loss,
                                  void* dH, void* dC, void* workspace, hipStream_t stream) {
  char* ws = reinterpret_cast<char*>(workspace);
  return a.dt == 0 ? run_grad<F32>(a, stats, g_loss, dH, dC, ws, stream)
                   : run_grad<Bf16>(a, stats, g_loss, dH, dC, ws, stream);
}

}  // namespace ops
}  // namespace hd
