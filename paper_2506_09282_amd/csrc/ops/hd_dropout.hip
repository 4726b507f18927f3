// Dropout from a counter-based generator: the mask is a function of the key, the step and a
// value's place, so it is never stored, and the backward pass computes it again.
//
// Philox 4x32 with 10 rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as
// 1, 2, 3", 2011): columns 4j ... 4j + 3 of row n take the four words of the counter {j, n, step
// low, step high} under the key {seed low, seed high}. A value is dropped where its word is
// below p 2^32.
//
// Bound by memory: 16384 x 10240 fp32, 1.34 GB, in 218 to 230 us (5.8 to 6.2 TB/s). The 20 products of
// a counter's rounds, at a quarter of the vector units' rate, take about as long as moving
// bf16 does, and run beside it. A small call (33 x 4097) is the host's 7 us; the kernel takes 3.
#include "hd_ops.hpp"

namespace hd {
namespace ops {

namespace {

typedef u32x4 u32x4_a4 __attribute__((aligned(4)));

constexpr int kThreads = 256;
constexpr int kEach = 8;  // values of a thread: two counters

struct Draw {
  uint32_t k0, k1;
  uint64_t step;
  const uint64_t* step_at;  // device memory: added to step (null: 0)
  uint32_t below;           // words under it are dropped
  bool all;                 // every value is
  float scale;
};

__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t a = (uint64_t)0xD2511F53u * c[0], b = (uint64_t)0xCD9E8D57u * c[2];
    const uint32_t h0 = (uint32_t)(b >> 32) ^ c[1] ^ k0, h1 = (uint32_t)(a >> 32) ^ c[3] ^ k1;
    c[0] = h0;
    c[1] = (uint32_t)b;
    c[2] = h1;
    c[3] = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

__device__ __forceinline__ void load8(const float* p, float (&v)[kEach]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x4 x = *reinterpret_cast<const f32x4_a4*>(p + 4 * h);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * h + e] = x[e];
  }
}
__device__ __forceinline__ void load8(const bf16raw* p, float (&v)[kEach]) {
  const u32x4 x = *reinterpret_cast<const u32x4_a2*>(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[2 * e] = __uint_as_float(x[e] << 16);
    v[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ void store8(float* p, const float (&v)[kEach]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    *reinterpret_cast<f32x4_a4*>(p + 4 * h) =
        f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
}
__device__ __forceinline__ void store8(bf16raw* p, const float (&v)[kEach]) {
  u32x4 x;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = to_bf16(v[2 * e]) | (uint32_t)to_bf16(v[2 * e + 1]) << 16;
  *reinterpret_cast<u32x4_a2*>(p) = x;
}

// A block takes 2^across pieces of 8 columns by 256 >> across rows.
template <typename T>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const T* X, int64_t ldx, T* Y,
                                                           int64_t ldy, int64_t N, int64_t D,
                                                           int across, Draw w) {
  const uint64_t step = w.step + (w.step_at ? *w.step_at : 0);
  const int64_t piece = ((int64_t)blockIdx.x << across) + (threadIdx.x & ((1 << across) - 1));
  const int64_t d = piece * kEach;
  if (d >= D) return;
  const int rows = kThreads >> across;
  for (int64_t n = (int64_t)blockIdx.y * rows + (threadIdx.x >> across); n < N;
       n += (int64_t)gridDim.y * rows) {
    const T* x = X + n * ldx + d;
    T* y = Y + n * ldy + d;
    const bool whole = d + kEach <= D;
    float v[kEach];
    if (whole) {
      load8(x, v);
    } else {
#pragma unroll
      for (int e = 0; e < kEach; ++e) v[e] = d + e < D ? load_elem(x, e) : 0.0f;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t c[4] = {(uint32_t)(2 * piece + h), (uint32_t)n, (uint32_t)step,
                       (uint32_t)(step >> 32)};
      philox(c, w.k0, w.k1);
#pragma unroll
      for (int e = 0; e < 4; ++e)  // (chosen, not multiplied: what is dropped may be NaN)
        v[4 * h + e] = !w.all && c[e] >= w.below ? v[4 * h + e] * w.scale : 0.0f;
    }
    if (whole) {
      store8(y, v);
    } else {
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (d + e < D) store_elem(y, e, v[e]);
    }
  }
}

template <typename T>
hipError_t run(const void* X, int64_t ldx, void* Y, int64_t ldy, int64_t N, int64_t D,
               const Draw& w, hipStream_t stream) {
  const int64_t pieces = cdiv(D, kEach);
  int across = 0;
  while (across < 8 && (int64_t(1) << across) < pieces) ++across;
  const int64_t x = cdiv(pieces, int64_t(1) << across), rows = kThreads >> across;
  // (a launch has fewer than 2^32 threads: beyond them a block walks over rows)
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(65535, (int64_t(1) << 23) / x));
  const int64_t y = std::min(cdiv(N, rows), most);
  dropout_kernel<T><<<dim3((uint32_t)x, (uint32_t)y), dim3(kThreads), 0, stream>>>(
      reinterpret_cast<const T*>(X), ldx, reinterpret_cast<T*>(Y), ldy, N, D, across, w);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const void* X, int64_t ldx, void* Y, int64_t ldy, int64_t N, int64_t D,
                          uint64_t below, float scale, uint64_t seed, uint64_t step,
                          const uint64_t* step_at, int dt, hipStream_t stream) {
  const Draw w{(uint32_t)seed, (uint32_t)(seed >> 32), step, step_at, (uint32_t)below,
               below > 0xffffffffu, scale};
  return dt == 0 ? run<float>(X, ldx, Y, ldy, N, D, w, stream)
                 : run<bf16raw>(X, ldx, Y, ldy, N, D, w, stream);
}

}  // namespace ops
}  // namespace hd
