// Host-side declarations of the operators behind answers and learning (4-bit
// products, log probabilities, 8-bit checkpoints), and the device helpers they
// share.
#pragma once

#include "../hd_common.hpp"
#include "../hd_internal.hpp"

namespace hd {
namespace ops {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// the same vectors where rows start at any element
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));

// Round to nearest even to bfloat16's bits (NaN stays NaN).
__device__ __forceinline__ bf16raw to_bf16(float v) {
  const __bf16 b = (__bf16)v;
  return __builtin_bit_cast(bf16raw, b);
}
__device__ __forceinline__ void store_elem(float* p, int64_t i, float v) { p[i] = v; }
__device__ __forceinline__ void store_elem(bf16raw* p, int64_t i, float v) { p[i] = to_bf16(v); }

// Up to four values of a row from place i on (n of them), wherever rows start.
__device__ __forceinline__ void store_four(float* p, int64_t i, const f32x4& v, int64_t n) {
  if (n >= 4) {
    *reinterpret_cast<f32x4_a4*>(p + i) = v;
  } else {
    if (n > 0) p[i] = v[0];
    if (n > 1) p[i + 1] = v[1];
    if (n > 2) p[i + 2] = v[2];
  }
}
__device__ __forceinline__ void store_four(bf16raw* p, int64_t i, const f32x4& v, int64_t n) {
  typedef u32x2 u32x2_a2 __attribute__((aligned(2)));
  if (n >= 4) {
    *reinterpret_cast<u32x2_a2*>(p + i) = u32x2{to_bf16(v[0]) | (uint32_t)to_bf16(v[1]) << 16,
                                                to_bf16(v[2]) | (uint32_t)to_bf16(v[3]) << 16};
  } else {
    if (n > 0) p[i] = to_bf16(v[0]);
    if (n > 1) p[i + 1] = to_bf16(v[1]);
    if (n > 2) p[i + 2] = to_bf16(v[2]);
  }
}

// The value of lane ^ OFF, in the vector ALU alone (a shuffle through LDS takes several
// times as long, and the sorts and sums across lanes are chains of these).
template <int OFF>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
  static_assert(OFF == 1 || OFF == 2 || OFF == 4 || OFF == 8 || OFF == 16 || OFF == 32, "");
  if constexpr (OFF == 1) return __builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true);
  if constexpr (OFF == 2) return __builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true);
  if constexpr (OFF == 4) {  // lane ^ 7 (half a row mirrored), then ^ 3
    const int m = __builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true);
    return __builtin_amdgcn_mov_dpp(m, 0x1b, 0xf, 0xf, true);
  }
  if constexpr (OFF == 8) return __builtin_amdgcn_mov_dpp((int)v, 0x128, 0xf, 0xf, true);
  if constexpr (OFF == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return (threadIdx.x & 16) ? r[0] : r[1];
  }
  if constexpr (OFF == 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return (threadIdx.x & 32) ? r[0] : r[1];
  }
}
template <int OFF>
__device__ __forceinline__ float lane_xor(float v) {
  return __uint_as_float(lane_xor<OFF>(__float_as_uint(v)));
}
template <int OFF>
__device__ __forceinline__ uint64_t lane_xor(uint64_t v) {
  return (uint64_t)lane_xor<OFF>((uint32_t)(v >> 32)) << 32 | lane_xor<OFF>((uint32_t)v);
}

// ---- products with 4-bit weights (hd_nibble.hip) ---------------------------
struct NibbleLayout {
  int64_t otiles, itiles;           // tiles of 16 outputs, of 128 inputs
  size_t scales, zeros, total;      // byte offsets of the sections, size of the image
};
NibbleLayout nibble_layout(int64_t O, int64_t I, int G);
hipError_t launch_nibble_pack(const uint8_t* codes, const bf16raw* scales, const uint8_t* zeros,
                              int64_t O, int64_t I, int G, void* image, hipStream_t stream);
hipError_t launch_nibble_quantize(const void* W, int64_t ldw, bool in_rows, int64_t O, int64_t I,
                                  int G, bool with_zeros, int dt, void* image,
                                  hipStream_t stream);
hipError_t launch_nibble_unpack(const void* image, float* W, int64_t O, int64_t I, int G,
                                bool with_zeros, hipStream_t stream);
hipError_t launch_nibble_product(const void* X, int64_t ldx, const void* image, void* Y,
                                 int64_t ldy, int64_t N, int64_t O, int64_t I, int G,
                                 bool with_zeros, int x_dt, int y_dt, int act, void* workspace,
                                 hipStream_t stream);
size_t nibble_ws_bytes(int64_t N, int64_t I, int x_dt);  // of launch_nibble_product

// ---- log probabilities (hd_logprobs.hip) ------------------------------------
constexpr int kMaxTop = 32;  // alternatives of a row
struct LogprobsArgs {
  const void* scores;
  int64_t ld;
  const uint8_t* mask;  // may be null; row stride ldm (0: one mask for all rows)
  int64_t ldm;
  const int32_t* y;
  float scale;
  int64_t N, K;
  int dt;
};
size_t logprobs_ws_bytes(int64_t N, int64_t K, int dt);
hipError_t launch_logprobs(const LogprobsArgs& a, float* logp, float* entropy, float* stats,
                           int32_t* ids, float* top_logp, int top, void* workspace,
                           hipStream_t stream);
hipError_t launch_logprobs_grad(const LogprobsArgs& a, const float* stats, const float* entropy,
                                const float* g_logp, const float* g_entropy, void* dscores,
                                int64_t ldd, hipStream_t stream);

// ---- checkpoints in 8 bits (hd_ckpt.hip) -------------------------------------
constexpr int kCkptRows = 64;  // rows of one group
size_t ckpt_image_bytes(int64_t N, int64_t D);
hipError_t launch_ckpt_store(const void* H, int64_t ldh, int64_t N, int64_t D, int dt,
                             void* image, hipStream_t stream);
hipError_t launch_ckpt_load(const void* image, void* H, int64_t ldh, int64_t N, int64_t D, int dt,
                            hipStream_t stream);
size_t ckpt_grad_ws_bytes(int64_t N, int64_t D, int64_t K, int dt);
hipError_t launch_ckpt_class_grad(const void* dS, int64_t lds, const void* image, float* dC,
                                  int64_t N, int64_t D, int64_t K, int dt, bool accumulate,
                                  void* workspace, hipStream_t stream);

// ---- cross entropy of class scores that are never kept (hd_class.hip) ---------
struct ClassArgs {
  const void* H;
  int64_t ldh;
  const void* C;
  int64_t ldc;
  const uint8_t* mask;  // [K], may be null
  const int32_t* y;
  float scale;
  int64_t N, D, K;
  int dt;
};
size_t class_loss_ws_bytes(int64_t N, int64_t D, int64_t K);
hipError_t launch_class_loss(const ClassArgs& a, float* loss, float* stats, void* workspace,
                             hipStream_t stream);
size_t class_grad_ws_bytes(int64_t N, int64_t D, int64_t K, int dt, bool dH, bool dC);
hipError_t launch_class_loss_grad(const ClassArgs& a, const float* stats, const float* g_loss,
                                  void* dH, void* dC, void* workspace, hipStream_t stream);

// ---- products with 8-bit weights (hd_byte.hip) --------------------------------
size_t byte_image_bytes(int64_t O, int64_t I);
hipError_t launch_byte_pack(const int8_t* codes, const float* scales, int64_t O, int64_t I,
                            void* image, hipStream_t stream);
hipError_t launch_byte_quantize(const void* W, int64_t ldw, bool in_rows, int64_t O, int64_t I,
                                int dt, void* image, hipStream_t stream);
hipError_t launch_byte_unpack(const void* image, float* W, int64_t O, int64_t I,
                              hipStream_t stream);
hipError_t launch_byte_rows(const void* X, int64_t ldx, int64_t N, int64_t I, int dt,
                            int8_t* codes, float* scales, hipStream_t stream);
size_t byte_ws_bytes(int64_t N, int64_t O, int64_t I, int x_dt);
hipError_t launch_byte_product(const void* X, int64_t ldx, const float* row_scales,
                               const void* image, void* Y, int64_t ldy, int64_t N, int64_t O,
                               int64_t I, int x_dt, int y_dt, int act, void* workspace,
                               hipStream_t stream);

// ---- dropout (hd_dropout.hip) ----------------------------------------------------
// Values whose random word is under `below` (up to 2^32: all) are dropped.
hipError_t launch_dropout(const void* X, int64_t ldx, void* Y, int64_t ldy, int64_t N, int64_t D,
                          uint64_t below, float scale, uint64_t seed, uint64_t step,
                          const uint64_t* step_at, int dt, hipStream_t stream);

}  // namespace ops
}  // namespace hd
