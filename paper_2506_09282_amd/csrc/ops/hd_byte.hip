// Products in 8-bit integers with a scale for each row of X and each output:
//
//   s_n = max_i |X[n][i]| / 127,  q = rint(X / s_n),  Y[n][o] = act(s_n t_o sum_i q[n][i] w[o][i])
//
// The sum is exact in int32 (at most 2^17 - 1 inputs), the scales are applied to it in 64 bits and
// the result is rounded once. The scales stand outside the reduction, so the int8 matrix
// instruction takes the codes as they are.
//
// Weights are laid out once, in blocks of 32 outputs x 32 inputs in the operand order of the
// 32 x 32 x 32 instruction: lane l of a wave's 1 KiB load holds inputs 16 (l / 32) ... of output
// l % 32. The blocks of 32 outputs follow each other along the inputs, filled up with zeros to
// whole stages of 128 inputs; the outputs' scales follow the codes.
//
// Up to 64 rows are bound by reading the weights once (1 x 4096 x 14336 bf16 11 to 12 us a call, 32 rows
// 16 to 17 us, of which the product takes 12 to 14: 4.4 TB/s), more by the tile's own pace (8192 x 4096
// x 16384: 0.59 to 0.63 ms, 30 us of them the rows' codes).
#include "hd_tile.hpp"

namespace hd {
namespace ops {

namespace {

using tile::die_order;
using tile::I8;
using tile::kImage;
using tile::kRows;
using tile::Operand;
using tile::Plan;
using tile::Tile;
using tile::tile_at;

constexpr int kThreads = 256;
constexpr float kInv127 = 1.0f / 127.0f;

size_t up(size_t n) { return (n + 255) / 256 * 256; }

// The code of x under the reciprocal scale r.
__device__ __forceinline__ int8_t code_of(float x, float r) {
  return (int8_t)fminf(fmaxf(rintf(x * r), -127.0f), 127.0f);
}
// A scale from the largest size of its values (+inf, also for NaN, where one is not finite).
struct ScaleOf {
  float s, r;
  __device__ __forceinline__ explicit ScaleOf(float top) {
    if (top < INFINITY) {
      s = top * kInv127;
      r = 1.0f / s;
      if (!(r < INFINITY)) r = 0.0f;
    } else {
      s = NAN;
      r = 0.0f;
    }
  }
};
__device__ __forceinline__ float size_of(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : INFINITY;  // (NaN too)
}
__device__ __forceinline__ int8_t coded(float x, const ScaleOf& sc) {
  return sc.s == sc.s ? code_of(x, sc.r) : (int8_t)0;
}

__device__ __forceinline__ float block_max(float v, float* part) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, kWave));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
}

// ---- weights -----------------------------------------------------------------------

// A thread takes 16 inputs of an output: codes as given, or X's under the output's scale.
__global__ __launch_bounds__(kThreads) void byte_pack_kernel(const int8_t* __restrict__ codes,
                                                             const float* __restrict__ scales,
                                                             int64_t O, int64_t I,
                                                             int64_t blocks,  // of 32 inputs
                                                             char* __restrict__ image,
                                                             float* __restrict__ image_scales) {
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t tiles = cdiv(O, 32);
  if (at >= tiles * blocks * 64) return;
  const int lane = (int)(at & 63);
  const int64_t b = at >> 6, t = b / blocks, s = b - t * blocks;
  const int64_t o = t * 32 + (lane & 31), i0 = s * 32 + (lane >> 5) * 16;
  u32x4 v = {0u, 0u, 0u, 0u};
  if (o < O) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (i0 + e < I) v[e / 4] |= (uint32_t)(uint8_t)codes[o * I + i0 + e] << (8 * (e & 3));
  }
  reinterpret_cast<u32x4*>(image)[at] = v;
  if (s == 0 && lane < 32) image_scales[o] = o < O ? scales[o] : 0.0f;
}

// The outputs' scales: a workgroup to a row of W, or to 64 columns of it.
template <typename T>
__global__ __launch_bounds__(kThreads) void byte_scales_kernel(const T* __restrict__ W, int64_t ldw,
                                                               bool in_rows, int64_t O, int64_t I,
                                                               float* __restrict__ scales) {
  __shared__ float part[kThreads];
  if (!in_rows) {
    const int64_t o = blockIdx.x;
    float top = 0.0f;
    for (int64_t i = threadIdx.x; i < I; i += kThreads)
      top = fmaxf(top, size_of(load_elem(W, o * ldw + i)));
    top = block_max(top, part);
    if (threadIdx.x == 0) scales[o] = ScaleOf(top).s;
    return;
  }
  const int64_t o = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
  float top = 0.0f;
  if (o < O)
    for (int64_t i = threadIdx.x >> 6; i < I; i += kThreads / 64)
      top = fmaxf(top, size_of(load_elem(W, i * ldw + o)));
  part[threadIdx.x] = top;
  __syncthreads();
  if (threadIdx.x < 64 && o < O) {
    for (int w = 1; w < kThreads / 64; ++w) top = fmaxf(top, part[w * 64 + threadIdx.x]);
    scales[o] = ScaleOf(top).s;
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void byte_codes_kernel(const T* __restrict__ W, int64_t ldw,
                                                              bool in_rows, int64_t O, int64_t I,
                                                              int64_t blocks,
                                                              char* __restrict__ image,
                                                              float* __restrict__ scales) {
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t tiles = cdiv(O, 32);
  if (at >= tiles * blocks * 64) return;
  const int lane = (int)(at & 63);
  const int64_t b = at >> 6, t = b / blocks, s = b - t * blocks;
  const int64_t o = t * 32 + (lane & 31), i0 = s * 32 + (lane >> 5) * 16;
  u32x4 v = {0u, 0u, 0u, 0u};
  if (o < O) {
    const float scale = scales[o];
    float r = 1.0f / scale;
    if (!(r < INFINITY)) r = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (i0 + e < I && scale == scale) {
        const float x = load_elem(W, in_rows ? (i0 + e) * ldw + o : o * ldw + i0 + e);
        v[e / 4] |= (uint32_t)(uint8_t)code_of(x, r) << (8 * (e & 3));
      }
  } else if (s == 0 && lane < 32) {
    scales[o] = 0.0f;
  }
  reinterpret_cast<u32x4*>(image)[at] = v;
}

__global__ __launch_bounds__(kThreads) void byte_unpack_kernel(const char* __restrict__ image,
                                                               const float* __restrict__ scales,
                                                               int64_t O, int64_t I,
                                                               int64_t blocks,
                                                               float* __restrict__ W) {
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t tiles = cdiv(O, 32);
  if (at >= tiles * blocks * 64) return;
  const int lane = (int)(at & 63);
  const int64_t b = at >> 6, t = b / blocks, s = b - t * blocks;
  const int64_t o = t * 32 + (lane & 31), i0 = s * 32 + (lane >> 5) * 16;
  if (o >= O) return;
  const u32x4 v = reinterpret_cast<const u32x4*>(image)[at];
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (i0 + e < I) W[o * I + i0 + e] = (float)(int8_t)(v[e / 4] >> (8 * (e & 3))) * scales[o];
}

// ---- rows of X -----------------------------------------------------------------------

__device__ __forceinline__ f32x4 load4_any(const float* p) {
  return *reinterpret_cast<const f32x4_a4*>(p);
}
__device__ __forceinline__ f32x4 load4_any(const bf16raw* p) {
  typedef u32x2 u32x2_a2 __attribute__((aligned(2)));
  const u32x2 w = *reinterpret_cast<const u32x2_a2*>(p);
  return f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u),
               __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u)};
}
// Sixteen inputs from i on, 0 past the row's end.
template <typename T>
__device__ __forceinline__ void load16(const T* x, int64_t i, int64_t I, float (&v)[16]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int64_t at = i + 4 * q;
    f32x4 w = {0.0f, 0.0f, 0.0f, 0.0f};
    if (at + 4 <= I) {
      w = load4_any(x + at);
    } else if (at < I) {  // (loads past the end repeat the last input)
      const float a = load_elem(x, at), b = load_elem(x, at + 1 < I ? at + 1 : at),
                  c = load_elem(x, at + 2 < I ? at + 2 : at);
      w = f32x4{a, at + 1 < I ? b : 0.0f, at + 2 < I ? c : 0.0f, 0.0f};
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * q + e] = w[e];
  }
}
__device__ __forceinline__ float size16(const float (&v)[16]) {
  float top = 0.0f;
#pragma unroll
  for (int e = 0; e < 16; ++e) top = fmaxf(top, size_of(v[e]));
  return top;
}
__device__ __forceinline__ u32x4 code16(const float (&v)[16], const ScaleOf& sc) {
  u32x4 w;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t x = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) x |= (uint32_t)(uint8_t)coded(v[4 * q + e], sc) << (8 * e);
    w[q] = x;
  }
  return w;
}

// A row's scale, and its codes 16 by 16 to put(piece, codes), by T threads; the first kHeld * T
// pieces are read once (8192 inputs or more).
template <int T, typename X, class Put>
__device__ __forceinline__ ScaleOf code_row(const X* x, int64_t I, int64_t pieces, float* part,
                                            Put put) {
  constexpr int kHeld = T >= 1024 ? 1 : 2;
  float v[kHeld][16];
  float top = 0.0f;
#pragma unroll
  for (int h = 0; h < kHeld; ++h) {
    const int64_t p = threadIdx.x + h * T;
    load16(x, 16 * p, I, v[h]);
    top = fmaxf(top, size16(v[h]));
  }
  for (int64_t p = threadIdx.x + kHeld * T; p < pieces; p += T) {
    float w[16];
    load16(x, 16 * p, I, w);
    top = fmaxf(top, size16(w));
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < T / 64; ++w) top = fmaxf(top, part[w]);
  const ScaleOf sc(top);
#pragma unroll
  for (int h = 0; h < kHeld; ++h) {
    const int64_t p = threadIdx.x + h * T;
    if (p < pieces) put(p, code16(v[h], sc));
  }
  for (int64_t p = threadIdx.x + kHeld * T; p < pieces; p += T) {
    float w[16];
    load16(x, 16 * p, I, w);
    put(p, code16(w, sc));
  }
  __syncthreads();  // (`part` may be used again)
  return sc;
}

// Codes of a row by a workgroup: rows of `width` codes, a multiple of 16, zeros from I on;
// or, with kOperand, as the products' operand, in blocks of 32 rows x 32 inputs like the weights'.
template <typename T, bool kOperand, int THREADS>
__global__ __launch_bounds__(THREADS) void byte_rows_kernel(const T* __restrict__ X, int64_t ldx,
                                                             int64_t I, int64_t width,
                                                             int8_t* __restrict__ codes,
                                                             float* __restrict__ scales) {
  __shared__ float part[THREADS / 64];
  const int64_t n = blockIdx.x;
  u32x4* out = reinterpret_cast<u32x4*>(codes);
  const int64_t first = kOperand ? n / 32 * (width / 32) * 64 + n % 32 : n * (width / 16);
  const ScaleOf sc =
      code_row<THREADS>(X + n * ldx, I, width / 16, part, [&](int64_t p, const u32x4& w) {
        out[first + (kOperand ? (p >> 1) * 64 + (p & 1) * 32 : p)] = w;
      });
  if (threadIdx.x == 0) scales[n] = sc.s;
}

// The same for rows of any width (the caller's), a byte at a time.
template <typename T>
__global__ __launch_bounds__(kThreads) void byte_rows_out_kernel(const T* __restrict__ X,
                                                                 int64_t ldx, int64_t I,
                                                                 int8_t* __restrict__ codes,
                                                                 float* __restrict__ scales) {
  __shared__ float part[kThreads / 64];
  const int64_t n = blockIdx.x;
  int8_t* out = codes + n * I;
  const ScaleOf sc =
      code_row<kThreads>(X + n * ldx, I, cdiv(I, 16), part, [&](int64_t p, const u32x4& w) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (16 * p + e < I) out[16 * p + e] = (int8_t)(w[e / 4] >> (8 * (e & 3)));
      });
  if (threadIdx.x == 0) scales[n] = sc.s;
}

// Given codes as the products' operand: a thread takes 16 inputs of a row.
__global__ __launch_bounds__(kThreads) void byte_operand_kernel(const int8_t* __restrict__ X,
                                                                int64_t ldx, int64_t N, int64_t I,
                                                                int64_t width,
                                                                u32x4* __restrict__ out) {
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x, pieces = width / 16;
  const int64_t n = at / pieces, p = at - n * pieces;
  if (n >= N) return;
  u32x4 v = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int64_t i = 16 * p + e;
    const uint32_t x = (uint8_t)X[n * ldx + (i < I ? i : I - 1)];
    v[e / 4] |= (i < I ? x : 0u) << (8 * (e & 3));
  }
  out[n / 32 * (width / 32) * 64 + (p >> 1) * 64 + (p & 1) * 32 + n % 32] = v;
}

// ---- the product -----------------------------------------------------------------------

struct Result {
  const float *row_scales, *scales;  // row_scales null: 1
  void* Y;
  int64_t ldy, N, O;
  int y_dt, act;
  int32_t* parts;  // [part][N][O]: sums of parts of the reduction
};

__device__ __forceinline__ float result(const Result& o, int64_t col, int32_t sum,
                                        double row_scale) {
  const double v = (double)sum * (double)o.scales[col] * row_scale;
  return o.act ? (float)v : v >= 0.0 ? 1.0f : -1.0f;
}
__device__ __forceinline__ void put(const Result& o, int64_t n, int64_t col, int32_t sum,
                                    double row_scale) {
  const float y = result(o, col, sum, row_scale);
  if (o.y_dt == 0)
    reinterpret_cast<float*>(o.Y)[n * o.ldy + col] = y;
  else
    reinterpret_cast<bf16raw*>(o.Y)[n * o.ldy + col] = to_bf16(y);
}

template <class TL>
__global__ __launch_bounds__(TL::T, 2) void byte_product_kernel(Operand a, Operand b, int64_t K,
                                                                int64_t each, uint32_t mt,
                                                                uint32_t nt, Result o) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const uint32_t tiles = mt * nt;
  const uint32_t id = die_order(blockIdx.x, gridDim.x), part = id / tiles;
  uint32_t mi, ni;
  tile_at(id % tiles, mt, nt, mi, ni);
  const int64_t m0 = (int64_t)mi * TL::BM, n0 = (int64_t)ni * TL::BN;
  const int64_t k0 = part * each, k1 = k0 + each < K ? k0 + each : K;
  typename TL::Acc c[TL::MT][TL::NT];
  TL::product(a, b, m0, n0, k0, k1, lds, c);
  int32_t* to = o.parts ? o.parts + (int64_t)part * o.N * o.O : nullptr;
  TL::rows_out(c, lds, m0, n0, [&](int64_t n, int64_t col, const i32x4& v) {
    if (n >= o.N || col >= o.O) return;
    if (to) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < o.O) to[n * o.O + col + e] = v[e];
      return;
    }
    const double row_scale = o.row_scales ? (double)o.row_scales[n] : 1.0;
    f32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e)  // (the image's scales go on to whole blocks of 32 outputs)
      y[e] = result(o, col + e, v[e], row_scale);
    if (o.y_dt == 0)
      store_four(reinterpret_cast<float*>(o.Y), n * o.ldy + col, y, o.O - col);
    else
      store_four(reinterpret_cast<bf16raw*>(o.Y), n * o.ldy + col, y, o.O - col);
  });
}

__global__ __launch_bounds__(kThreads) void byte_sum_kernel(Result o, int count) {
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x, each = o.N * o.O;
  if (at >= each) return;
  int32_t v = 0;
  for (int i = 0; i < count; ++i) v += o.parts[i * each + at];
  const int64_t n = at / o.O;
  put(o, n, at - n * o.O, v, o.row_scales ? (double)o.row_scales[n] : 1.0);
}

// ---- the product of few rows ------------------------------------------------------------
//
// The weights are read once and bound the call. A workgroup takes 32 outputs; its W waves take every
// W-th block of their inputs, straight into registers in operand order, several blocks
// ahead, and add up in LDS. X lies laid out as the other operand in memory (read by every
// workgroup from the L2), or, where it is short, each workgroup codes it for itself
// in LDS, which saves a launch.

constexpr int kFewRows = 64;  // (64 x 4096 x 14336: 21 us instead of 36 by tiles)
// (4096 x 14336: one row 12 us instead of 16 by two launches, two 14 instead of 16; four 17 and 16)
constexpr int64_t kOwnRows = 2, kOwnValues = 16384;  // of X, which a workgroup codes for itself

struct Few {
  const void* X;  // X as given (kOwn), or its codes as operands
  int64_t ldx, N, I, O;
  int64_t blocks;  // of 32 inputs
  const u32x4* image;
};

template <int RT, int W, bool kOwn, typename T>
__global__ __launch_bounds__(64 * W) void byte_few_kernel(Few f, Result o) {
  constexpr int kAhead = RT == 1 ? 8 : 6;
  extern __shared__ __attribute__((aligned(16))) char lds[];
  __shared__ float part[W];
  __shared__ float own_scales[kOwn ? 32 : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const int64_t tile = blockIdx.x;
  const u32x4* w = f.image + tile * f.blocks * 64 + lane;
  const int64_t pieces = f.blocks * 2;
  // this wave's blocks: wave, wave + W, ...
  const int count = (int)((f.blocks - wave + W - 1) / W);

  u32x4 wr[kAhead], xr[kOwn ? 1 : kAhead][RT];
  // codes of the lane's row: rows that are not there repeat the first (their sums go nowhere)
  const int row = (lane & 31) < f.N ? lane & 31 : 0;
  const u32x4* own = reinterpret_cast<const u32x4*>(lds) + row * pieces + half;
  const u32x4* x = reinterpret_cast<const u32x4*>(f.X) + lane;
  auto load_w = [&](int slot, int i) {
    wr[slot] = __builtin_nontemporal_load(w + (int64_t)(wave + i * W) * 64);
  };
  auto load_x = [&](int slot, int i) {
    const int64_t b = wave + i * W;
#pragma unroll
    for (int t = 0; t < RT; ++t) xr[slot][t] = x[(t * f.blocks + b) * 64];
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u)
    if (u < count) load_w(u, u);
  if constexpr (kOwn) {
    u32x4* to = reinterpret_cast<u32x4*>(lds);
    for (int n = 0; n < f.N; ++n) {
      const ScaleOf sc =
          code_row<64 * W>(reinterpret_cast<const T*>(f.X) + n * f.ldx, f.I, pieces, part,
                           [&](int64_t p, const u32x4& v) { to[n * pieces + p] = v; });
      if (threadIdx.x == 0) own_scales[n] = sc.s;
    }
    __syncthreads();
  } else {
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (u < count) load_x(u, u);
  }
  i32x16 c[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) c[t][r] = 0;
  for (int i0 = 0; i0 < count; i0 += kAhead) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int i = i0 + u;
      if (i < count) {
        if constexpr (kOwn) {
          I8::mfma(c[0], own[(wave + i * W) * 2], wr[u]);
        } else {
#pragma unroll
          for (int t = 0; t < RT; ++t) I8::mfma(c[t], xr[u][t], wr[u]);
        }
        if (i + kAhead < count) {
          load_w(u, i + kAhead);
          if constexpr (!kOwn) load_x(u, i + kAhead);
        }
      }
    }
  }
  if constexpr (kOwn) __syncthreads();  // (the codes are read)
  // [wave][row of 32 RT][32 outputs]
  int32_t* sums = reinterpret_cast<int32_t*>(lds);
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      sums[(wave * RT * 32 + t * 32 + (r / 4) * 8 + half * 4 + r % 4) * 32 + (lane & 31)] = c[t][r];
  __syncthreads();
  for (int at = threadIdx.x; at < RT * 1024; at += 64 * W) {
    const int64_t n = at >> 5, col = tile * 32 + (at & 31);
    int32_t v = 0;
#pragma unroll
    for (int k = 0; k < W; ++k) v += sums[k * RT * 1024 + at];
    if (n < f.N && col < o.O)
      put(o, n, col, v, kOwn ? (double)own_scales[n] : o.row_scales ? (double)o.row_scales[n] : 1.0);
  }
}

// ---- host -------------------------------------------------------------------------------

int64_t blocks_of(int64_t I) { return cdiv(I, 128) * 4; }
size_t codes_bytes(int64_t O, int64_t I) { return (size_t)(cdiv(O, 32) * blocks_of(I)) * 1024; }

template <auto KERNEL>
hipError_t allow_lds(int bytes) {
  static PerDeviceOnce once;
  return once_per_device(once, [&] {
    return hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL),
                               hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  });
}

template <class TL>
hipError_t launch(const Plan& p, const Operand& a, const Operand& b, int64_t K, const Result& o,
                  hipStream_t stream) {
  const hipError_t e = allow_lds<byte_product_kernel<TL>>(TL::kLds);
  if (e != hipSuccess) return e;
  byte_product_kernel<TL>
      <<<dim3((uint32_t)(p.mt * p.nt * p.splits)), dim3(TL::T), TL::kLds, stream>>>(
          a, b, K, p.each, (uint32_t)p.mt, (uint32_t)p.nt, o);
  return hipGetLastError();
}

struct Place {
  Plan p;
  int64_t width;  // of a row of codes
  bool few, own;  // the product of few rows; coding X for itself
  size_t scales, codes, parts, total;
};
Place place(int64_t N, int64_t O, int64_t I, bool given) {
  Place w;
  w.width = cdiv(I, 128) * 128;
  w.few = N <= kFewRows;
  w.own = w.few && !given && N <= kOwnRows && N * w.width <= kOwnValues;
  w.p = tile::plan(N, O, w.width);
  w.scales = w.codes = w.parts = w.total = 0;
  if (w.own) return w;
  if (!given) w.codes = up((size_t)N * 4);
  w.parts = w.codes;
  if (!given || w.few) w.parts += up((size_t)((w.few ? cdiv(N, 32) * 32 : N) * w.width));
  w.total = w.parts;
  if (!w.few && w.p.splits > 1) w.total += up((size_t)(w.p.splits * N * O) * 4);
  return w;
}

template <typename T>
hipError_t quantize(const void* W, int64_t ldw, bool in_rows, int64_t O, int64_t I, char* image,
                    hipStream_t stream) {
  const int64_t blocks = blocks_of(I);
  float* scales = reinterpret_cast<float*>(image + codes_bytes(O, I));
  byte_scales_kernel<T><<<dim3((uint32_t)(in_rows ? cdiv(O, 64) : O)), dim3(kThreads), 0, stream>>>(
      reinterpret_cast<const T*>(W), ldw, in_rows, O, I, scales);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  byte_codes_kernel<T>
      <<<dim3((uint32_t)cdiv(cdiv(O, 32) * blocks * 64, kThreads)), dim3(kThreads), 0, stream>>>(
          reinterpret_cast<const T*>(W), ldw, in_rows, O, I, blocks, image, scales);
  return hipGetLastError();
}

template <bool kOperand, typename T>
hipError_t rows(const void* X, int64_t ldx, int64_t N, int64_t I, int64_t width, int8_t* codes,
                float* scales, hipStream_t stream) {
  const T* x = reinterpret_cast<const T*>(X);
  if (width <= 2048)  // (a wave holds such a row)
    byte_rows_kernel<T, kOperand, 64>
        <<<dim3((uint32_t)N), dim3(64), 0, stream>>>(x, ldx, I, width, codes, scales);
  else
    byte_rows_kernel<T, kOperand, kThreads>
        <<<dim3((uint32_t)N), dim3(kThreads), 0, stream>>>(x, ldx, I, width, codes, scales);
  return hipGetLastError();
}

template <int RT, int W, bool kOwn, typename T>
hipError_t launch_few(const Few& f, const Result& o, hipStream_t stream) {
  constexpr int kLds = W * RT * 4096;  // the waves' sums; before them, kOwn's codes
  static_assert(!kOwn || kOwnValues <= kLds, "");
  const hipError_t e = allow_lds<byte_few_kernel<RT, W, kOwn, T>>(kLds);
  if (e != hipSuccess) return e;
  byte_few_kernel<RT, W, kOwn, T>
      <<<dim3((uint32_t)cdiv(f.O, 32)), dim3(64 * W), kLds, stream>>>(f, o);
  return hipGetLastError();
}
// More waves to 32 outputs where there are too few of these for the chip and the inputs are many; but
// more than four code a row for themselves no faster, and 16 are one workgroup to a unit (us a
// call by 4, 8 and 16 waves: 32 x 4096 x 14336 17.2, 16.9, 18.1; 16 x 16000 x 100 26.2, 23.1,
// 23.0; 16 x 1000 x 50000 16.2, 17.6, 22.7; 1 x 4096 x 14336, coded by itself, 12.3, 15.9, 15.2).
template <bool kOwn, typename T>
hipError_t few(const Few& f, const Result& o, hipStream_t stream) {
  const int64_t tiles = cdiv(f.O, 32);
  const int waves = f.blocks < 64 || tiles > (kOwn ? 256 : 1024) ? 4 : tiles > 256 ? 8 : 16;
  if (f.N <= 32)
    return waves == 16  ? launch_few<1, 16, kOwn, T>(f, o, stream)
           : waves == 8 ? launch_few<1, 8, kOwn, T>(f, o, stream)
                        : launch_few<1, 4, kOwn, T>(f, o, stream);
  if constexpr (kOwn)
    return hipErrorInvalidValue;
  else
    return waves == 16  ? launch_few<2, 16, kOwn, T>(f, o, stream)
           : waves == 8 ? launch_few<2, 8, kOwn, T>(f, o, stream)
                        : launch_few<2, 4, kOwn, T>(f, o, stream);
}

}  // namespace

size_t byte_image_bytes(int64_t O, int64_t I) {
  return codes_bytes(O, I) + up((size_t)cdiv(O, 32) * 32 * 4);
}

hipError_t launch_byte_pack(const int8_t* codes, const float* scales, int64_t O, int64_t I,
                            void* image, hipStream_t stream) {
  const int64_t blocks = blocks_of(I);
  char* im = reinterpret_cast<char*>(image);
  byte_pack_kernel<<<dim3((uint32_t)cdiv(cdiv(O, 32) * blocks * 64, kThreads)), dim3(kThreads), 0,
                     stream>>>(codes, scales, O, I, blocks, im,
                               reinterpret_cast<float*>(im + codes_bytes(O, I)));
  return hipGetLastError();
}

hipError_t launch_byte_quantize(const void* W, int64_t ldw, bool in_rows, int64_t O, int64_t I,
                                int dt, void* image, hipStream_t stream) {
  char* im = reinterpret_cast<char*>(image);
  return dt == 0 ? quantize<float>(W, ldw, in_rows, O, I, im, stream)
                 : quantize<bf16raw>(W, ldw, in_rows, O, I, im, stream);
}

hipError_t launch_byte_unpack(const void* image, float* W, int64_t O, int64_t I,
                              hipStream_t stream) {
  const int64_t blocks = blocks_of(I);
  const char* im = reinterpret_cast<const char*>(image);
  byte_unpack_kernel<<<dim3((uint32_t)cdiv(cdiv(O, 32) * blocks * 64, kThreads)), dim3(kThreads),
                       0, stream>>>(im, reinterpret_cast<const float*>(im + codes_bytes(O, I)), O,
                                    I, blocks, W);
  return hipGetLastError();
}

hipError_t launch_byte_rows(const void* X, int64_t ldx, int64_t N, int64_t I, int dt,
                            int8_t* codes, float* scales, hipStream_t stream) {
  if (dt == 0)
    byte_rows_out_kernel<float><<<dim3((uint32_t)N), dim3(kThreads), 0, stream>>>(
        reinterpret_cast<const float*>(X), ldx, I, codes, scales);
  else
    byte_rows_out_kernel<bf16raw><<<dim3((uint32_t)N), dim3(kThreads), 0, stream>>>(
        reinterpret_cast<const bf16raw*>(X), ldx, I, codes, scales);
  return hipGetLastError();
}

size_t byte_ws_bytes(int64_t N, int64_t O, int64_t I, int x_dt) {
  return place(N, O, I, x_dt == 2).total;
}

hipError_t launch_byte_product(const void* X, int64_t ldx, const float* row_scales,
                               const void* image, void* Y, int64_t ldy, int64_t N, int64_t O,
                               int64_t I, int x_dt, int y_dt, int act, void* workspace,
                               hipStream_t stream) {
  const bool given = x_dt == 2;
  const Place w = place(N, O, I, given);
  char* ws = reinterpret_cast<char*>(workspace);
  const char* im = reinterpret_cast<const char*>(image);
  const u32x4* image_codes = reinterpret_cast<const u32x4*>(im);
  Result o{row_scales, reinterpret_cast<const float*>(im + codes_bytes(O, I)), Y, ldy, N, O,
           y_dt, act, nullptr};
  const int64_t blocks = blocks_of(I);
  if (w.own) {
    const Few f{X, ldx, N, I, O, blocks, image_codes};
    return x_dt == 0 ? few<true, float>(f, o, stream) : few<true, bf16raw>(f, o, stream);
  }
  int8_t* codes = reinterpret_cast<int8_t*>(ws + w.codes);
  float* scales = reinterpret_cast<float*>(ws + w.scales);
  if (!given) o.row_scales = scales;
  hipError_t e;
  if (w.few) {
    if (given) {
      byte_operand_kernel<<<dim3((uint32_t)cdiv(N * (w.width / 16), kThreads)), dim3(kThreads), 0,
                            stream>>>(reinterpret_cast<const int8_t*>(X), ldx, N, I, w.width,
                                      reinterpret_cast<u32x4*>(codes));
      e = hipGetLastError();
    } else {
      e = x_dt == 0 ? rows<true, float>(X, ldx, N, I, w.width, codes, scales, stream)
                    : rows<true, bf16raw>(X, ldx, N, I, w.width, codes, scales, stream);
    }
    if (e != hipSuccess) return e;
    const Few f{codes, 0, N, I, O, blocks, image_codes};
    return few<false, float>(f, o, stream);
  }
  Operand a{X, ldx, N, nullptr};
  int64_t K = I;
  if (!given) {
    e = x_dt == 0 ? rows<false, float>(X, ldx, N, I, w.width, codes, scales, stream)
                  : rows<false, bf16raw>(X, ldx, N, I, w.width, codes, scales, stream);
    if (e != hipSuccess) return e;
    a = {codes, w.width, N, nullptr};
    K = w.width;
  }
  const Operand b{im, blocks, O, nullptr};
  if (w.p.splits > 1) o.parts = reinterpret_cast<int32_t*>(ws + w.parts);
  switch (w.p.shape) {
    case tile::k256: e = launch<Tile<I8, kRows, kImage, 256, 256, 2, 4>>(w.p, a, b, K, o, stream); break;
    case tile::k128: e = launch<Tile<I8, kRows, kImage, 128, 128, 2, 2>>(w.p, a, b, K, o, stream); break;
    default: e = launch<Tile<I8, kRows, kImage, 256, 32, 4, 1>>(w.p, a, b, K, o, stream);
  }
  if (e != hipSuccess || w.p.splits == 1) return e;
  byte_sum_kernel<<<dim3((uint32_t)cdiv(N * O, kThreads)), dim3(kThreads), 0, stream>>>(
      o, (int)w.p.splits);
  return hipGetLastError();
}

}  // namespace ops
}  // namespace hd
