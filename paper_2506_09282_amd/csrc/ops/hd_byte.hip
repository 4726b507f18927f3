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

// Codes of a row by a workgroup, zeros from I to width.
template <typename T>
__global__ __launch_bounds__(kThreads) void byte_rows_kernel(const T* __restrict__ X, int64_t ldx,
                                                             int64_t I, int64_t width,
                                                             int8_t* __restrict__ codes,
                                                             float* __restrict__ scales) {
  __shared__ float part[kThreads / 64];
  const int64_t n = blockIdx.x;
  const T* x = X + n * ldx;
  float top = 0.0f;
  for (int64_t i = threadIdx.x; i < I; i += kThreads) top = fmaxf(top, size_of(load_elem(x, i)));
  const ScaleOf sc(block_max(top, part));
  for (int64_t i = threadIdx.x; i < width; i += kThreads)
    codes[n * width + i] = i < I ? coded(load_elem(x, i), sc) : (int8_t)0;
  if (threadIdx.x == 0) scales[n] = sc.s;
}

// ---- the product -----------------------------------------------------------------------

struct Result {
  const float *row_scales, *scales;  // row_scales null: 1
  void* Y;
  int64_t ldy, N, O;
  int y_dt, act;
  int32_t* parts;  // [part][N][O]: sums of parts of the reduction
};

__device__ __forceinline__ void put(const Result& o, int64_t n, int64_t col, int32_t sum) {
  double v = (double)sum * (double)o.scales[col];
  if (o.row_scales) v *= (double)o.row_scales[n];
  const float y = o.act ? (float)v : v >= 0.0 ? 1.0f : -1.0f;
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
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const int wm = wave / TL::WN, wn = wave % TL::WN;
#pragma unroll
  for (int i = 0; i < TL::MT; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int64_t n = m0 + (wm * TL::MT + i) * 32 + (r / 4) * 8 + half * 4 + r % 4;
      if (n >= o.N) continue;
#pragma unroll
      for (int j = 0; j < TL::NT; ++j) {
        const int64_t col = n0 + (wn * TL::NT + j) * 32 + (lane & 31);
        if (col >= o.O) continue;
        if (o.parts)
          o.parts[((int64_t)part * o.N + n) * o.O + col] = c[i][j][r];
        else
          put(o, n, col, c[i][j][r]);
      }
    }
}

__global__ __launch_bounds__(kThreads) void byte_sum_kernel(Result o, int count) {
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x, each = o.N * o.O;
  if (at >= each) return;
  int32_t v = 0;
  for (int i = 0; i < count; ++i) v += o.parts[i * each + at];
  const int64_t n = at / o.O;
  put(o, n, at - n * o.O, v);
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
  size_t scales, codes, parts, total;
};
Place place(int64_t N, int64_t O, int64_t I, bool given) {
  Place w;
  w.width = cdiv(I, 128) * 128;
  w.p = tile::plan(N, O, w.width);
  w.scales = 0;
  w.codes = given ? 0 : up((size_t)N * 4);
  w.parts = w.codes + (given ? 0 : up((size_t)(N * w.width)));
  w.total = w.parts + (w.p.splits > 1 ? up((size_t)(w.p.splits * N * O) * 4) : 0);
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

template <typename T>
hipError_t rows(const void* X, int64_t ldx, int64_t N, int64_t I, int64_t width, int8_t* codes,
                float* scales, hipStream_t stream) {
  byte_rows_kernel<T><<<dim3((uint32_t)N), dim3(kThreads), 0, stream>>>(
      reinterpret_cast<const T*>(X), ldx, I, width, codes, scales);
  return hipGetLastError();
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
  return dt == 0 ? rows<float>(X, ldx, N, I, I, codes, scales, stream)
                 : rows<bf16raw>(X, ldx, N, I, I, codes, scales, stream);
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
  Operand a{X, ldx, N, nullptr};
  hipError_t e;
  int64_t K = I;
  if (!given) {
    int8_t* codes = reinterpret_cast<int8_t*>(ws + w.codes);
    float* scales = reinterpret_cast<float*>(ws + w.scales);
    e = x_dt == 0 ? rows<float>(X, ldx, N, I, w.width, codes, scales, stream)
                  : rows<bf16raw>(X, ldx, N, I, w.width, codes, scales, stream);
    if (e != hipSuccess) return e;
    a = {codes, w.width, N, nullptr};
    row_scales = scales;
    K = w.width;
  }
  const Operand b{im, blocks_of(I), O, nullptr};
  Result o{row_scales, reinterpret_cast<const float*>(im + codes_bytes(O, I)), Y, ldy, N, O,
           y_dt, act, nullptr};
  if (w.p.splits > 1) o.parts = reinterpret_cast<int32_t*>(ws + w.parts);
  switch (w.p.shape) {
    case tile::k256: e = launch<Tile<I8, kRows, kImage, 256, 256, 2, 4>>(w.p, a, b, K, o, stream); break;
    case tile::k128: e = launch<Tile<I8, kRows, kImage, 128, 128, 2, 2>>(w.p, a, b, K, o, stream); break;
    case tile::k32x128: e = launch<Tile<I8, kRows, kImage, 32, 128, 1, 4>>(w.p, a, b, K, o, stream); break;
    default: e = launch<Tile<I8, kRows, kImage, 128, 32, 4, 1>>(w.p, a, b, K, o, stream);
  }
  if (e != hipSuccess || w.p.splits == 1) return e;
  byte_sum_kernel<<<dim3((uint32_t)cdiv(N * O, kThreads)), dim3(kThreads), 0, stream>>>(
      o, (int)w.p.splits);
  return hipGetLastError();
}

}  // namespace ops
}  // namespace hd
