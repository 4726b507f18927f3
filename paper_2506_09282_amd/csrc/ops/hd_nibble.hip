// Products with 4-bit weights and group scales:
//   Y[n,o] = act( sum_i X[n,i] * s[o,g] * (q[o,i] - z[o,g]) ),   g = i / G,
// q in 0..15, z = 8 where the weights have no zero points.
//
// One pass over the weights is what bounds it: O*I/2 bytes of codes and two (with
// zero points three) bytes a group, against X and Y, which are small. The codes go
// to the bf16 matrix instruction, which costs the same for 1 and for 16 rows of X:
// * the zero point is taken off the codes, whose differences q - z are exact in bf16: signed
//   bytes, a conversion each and a byte permutation for two (`codes_less_zero`). A sum over
//   a group holds the products themselves and is added to the output's with s in fp32;
// * bf16 results of bf16 X take a shorter way. A byte that holds a code 0..15 is, read as fp8
//   e4m3, the number q * 2^-9 (0..7 are its subnormals, 8..15 its first binade), so two masks
//   and a shift split eight codes and four conversions make eight bf16 values, exact.
//   sum x*q starts from -z * sum x, which a constant operand gives once for all tiles of
//   outputs, in the lanes that need it. Over an X of one sign both are larger than their
//   difference, and so are fp32's roundings: measured, X uniform in 0..1, at most 2^-26 of
//   sum |x| z s (784 inputs, G = 64; 2^-28 for 16384, G = 128). Of a result in bf16, whose own
//   rounding is 2^-9, that is less from one code in 16384 on that is off its zero point; a row
//   with none gives such a number instead of 0. Results that stay in fp32, or whose sign is
//   taken, do not go this way (1 x 16384 x 57344 bf16, inside a graph: G = 128 79.6 us so, 85 with
//   exact differences; G = 64 with zero points 96 and 109; 32 x 3072 x 10240 13.1 and 13.5);
// * fp32 X is the exact sum of three bf16 values (its 24 bits cut in three), one
//   matrix instruction each. Products of 4 and 8 bits are exact in fp32.
//
// Layout: a tile is 16 outputs x 128 inputs, 1 KiB of codes, one 16-byte load for
// each lane. Lane l holds output l % 16 and, in dword s, inputs 32 s + 8 (l / 16) + e,
// e = 0..7, code e in the nibble 2 e (e < 4) or 2 e - 7: the operand order of
// v_mfma_f32_16x16x32_bf16. Tiles of one 16-output row follow each other, so a wave
// reads 1 KiB runs. Scales and zero points lie as the result's lanes need them:
// [output tile][input tile][l / 16][group][4 outputs].
//
// A workgroup takes TD output tiles, its waves every W-th input tile, and the waves'
// sums are added in LDS in a fixed order. Waves share outputs and not inputs, because
// one row of X leaves nothing else to fill the chip with: 57344 outputs are 1792 workgroups
// at TD = 2, 1000 outputs 32.
//
// Measured (kernel): bf16 1 x 16384 x 57344, G = 128, 484 MB: 77 to 80 us, 6.1 to 6.3 TB/s, where
// reading alone gives 7.1 (the vector units are busy for 57% of the time, the matrix units for
// 26%; 57344 x 16384 codes are fetched once, 497 MB in all); fp32 136 us a call. fp32
// 1 x 561 x 10240, 3.3 MB: 5.4 us, a launch and one round of loads. bf16 32 x 3072 x 10240, 18
// MB: 10.7 to 11.2 us, a launch, six rounds of loads for each wave, and 63 MB of X from the L2.
#include "hd_ops.hpp"

namespace hd {
namespace ops {

namespace {

constexpr int kTileI = 128, kTileO = 16;

__host__ __device__ inline NibbleLayout layout_of(int64_t O, int64_t I, int G) {
  NibbleLayout L;
  L.otiles = cdiv(O, kTileO);
  L.itiles = cdiv(I, kTileI);
  const int64_t tiles = L.otiles * L.itiles, groups = tiles * (kTileI / G) * kTileO;
  L.scales = (size_t)tiles * 1024;
  L.zeros = L.scales + ((size_t)groups * 2 + 255) / 256 * 256;
  L.total = L.zeros + ((size_t)groups + 255) / 256 * 256;
  return L;
}

// Nibble of element e (0..7) of a lane's dword.
__host__ __device__ constexpr int nibble_of(int e) { return e < 4 ? 2 * e : 2 * e - 7; }

// Index of (output o, group g of the row) in the scale and zero-point sections.
__device__ __forceinline__ int64_t group_index(int64_t o, int64_t g, int64_t itiles, int gpt) {
  const int64_t tile = (o / kTileO) * itiles + g / gpt;
  const int r = (int)(o % kTileO);
  return ((tile * 4 + r / 4) * gpt + g % gpt) * 4 + r % 4;
}

// ---- layout ------------------------------------------------------------------

// Half a dword's codes to every other nibble.
__device__ __forceinline__ uint32_t spread(uint32_t v) {
  v = (v | v << 8) & 0x00ff00ffu;
  return (v | v << 4) & 0x0f0f0f0fu;
}

// `words`: rows start at multiples of four bytes, so a dword's codes are one in them too.
__global__ __launch_bounds__(256) void nibble_pack_kernel(const uint8_t* __restrict__ codes,
                                                          int64_t O, int64_t I, int64_t itiles,
                                                          int words, int64_t total,
                                                          uint32_t* out) {
  // one dword: eight codes of one output
  for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < total;
       w += (int64_t)gridDim.x * 256) {
    const int s = (int)(w & 3), lane = (int)(w >> 2) & 63;
    const int64_t tile = w >> 8;
    const int64_t o = tile / itiles * kTileO + lane % 16;
    const int64_t i0 = tile % itiles * kTileI + 32 * s + 8 * (lane / 16);
    const uint8_t* row = codes + o * cdiv(I, 2);
    uint32_t v = 0;
    if (words && o < O && i0 + 8 <= I) {
      const uint32_t q = *reinterpret_cast<const uint32_t*>(row + i0 / 2);
      out[w] = spread(q & 0xffffu) | spread(q >> 16) << 4;
      continue;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (o < O && i0 + e < I)
        v |= (uint32_t)((row[(i0 + e) / 2] >> (4 * (e & 1))) & 15) << (4 * nibble_of(e));
    out[w] = v;
  }
}

__global__ __launch_bounds__(256) void nibble_pack_groups_kernel(
    const bf16raw* __restrict__ scales, const uint8_t* __restrict__ zeros, int64_t O,
    int64_t groups, int64_t itiles, int gpt, int64_t total, bf16raw* out_s, uint8_t* out_z) {
  for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < total;
       w += (int64_t)gridDim.x * 256) {
    const int r = (int)(w % 4), gg = (int)(w / 4 % gpt), quad = (int)(w / 4 / gpt % 4);
    const int64_t tile = w / (16 * gpt);
    const int64_t o = tile / itiles * kTileO + 4 * quad + r, g = tile % itiles * gpt + gg;
    const bool in = o < O && g < groups;
    out_s[w] = in ? scales[o * groups + g] : (bf16raw)0;
    out_z[w] = in && zeros ? (uint8_t)(zeros[o * groups + g] & 15) : (uint8_t)8;
  }
}

// One wave quantises one tile: lane l the elements it will hold. W is [O][I]
// (in_rows false) or [I][O].
template <typename T>
__global__ __launch_bounds__(64) void nibble_quantize_kernel(const T* __restrict__ W, int64_t ldw,
                                                             int in_rows, int64_t O, int64_t I,
                                                             int64_t itiles, int gpt,
                                                             int with_zeros, u32x4* out,
                                                             bf16raw* out_s, uint8_t* out_z) {
  const int lane = threadIdx.x;
  const int64_t tile = blockIdx.x;
  const int64_t o = tile / itiles * kTileO + lane % 16;
  const int64_t i0 = tile % itiles * kTileI + 8 * (lane / 16);
  float v[4][8];
  float lo[4], hi[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    lo[s] = 0.0f, hi[s] = 0.0f;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int64_t i = i0 + 32 * s + e;
      v[s][e] = (o < O && i < I) ? load_elem(W, in_rows ? i * ldw + o : o * ldw + i) : 0.0f;
      lo[s] = fminf(lo[s], v[s][e]);
      hi[s] = fmaxf(hi[s], v[s][e]);
      bad |= v[s][e] != v[s][e];
    }
    if (bad) lo[s] = -INFINITY;  // NaN: the group's scale is no number either
#pragma unroll
    for (int off = 16; off < 64; off <<= 1) {  // the four lanes of one output
      lo[s] = fminf(lo[s], __shfl_xor(lo[s], off, kWave));
      hi[s] = fmaxf(hi[s], __shfl_xor(hi[s], off, kWave));
    }
  }
  const int per = 4 / gpt;  // steps of one group
  u32x4 packed;
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    float l = 0.0f, h = 0.0f;
    for (int t = s / per * per; t < s / per * per + per; ++t) {
      // (t is small and known after unrolling for each gpt)
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (u == t) l = fminf(l, lo[u]), h = fmaxf(h, hi[u]);
    }
    float span = with_zeros ? (h - l) / 15.0f : fmaxf(h, -l) / 7.0f;
    if (with_zeros && h < INFINITY && l > -INFINITY && !(span < INFINITY))
      span = h / 15.0f - l / 15.0f;  // (the difference alone is past fp32's range)
    bf16raw sb = to_bf16(span);  // the codes are taken by the scale that is kept
    const float sc = bf16_to_f32(sb);
    const bool bad = !(sc < INFINITY);
    if (bad) sb = 0x7fc0;  // NaN
    // a scale below 2^-128 has no inverse in fp32: its weights, 2^4 times as large at most, are
    // moved up first, which is exact
    const float up = sc < 0x1p-126f ? 0x1p24f : 1.0f;
    const float r = sc > 0.0f && !bad ? 1.0f / (sc * up) : 0.0f;
    const float z = with_zeros ? fminf(fmaxf(rintf(-l * up * r), 0.0f), 15.0f) : 8.0f;
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float q = fminf(fmaxf(rintf(v[s][e] * up * r) + z, 0.0f), 15.0f);
      w |= (uint32_t)q << (4 * nibble_of(e));
    }
    packed[s] = w;
    if (s % per == 0 && lane < 16) {
      const int64_t at = ((tile * 4 + lane / 4) * gpt + s / per) * 4 + lane % 4;
      out_s[at] = sb;
      out_z[at] = (uint8_t)z;
    }
  }
  out[tile * 64 + lane] = packed;
}

__device__ __forceinline__ float weight_at(const uint8_t* image, const bf16raw* scales,
                                           const uint8_t* zeros, int64_t o, int64_t i,
                                           int64_t itiles, int gpt, bool with_zeros) {
  const int64_t tile = (o / kTileO) * itiles + i / kTileI;
  const int in = (int)(i % kTileI), e = in % 8;
  const int lane = (int)(o % kTileO) + 16 * (in % 32 / 8);
  const uint32_t w = reinterpret_cast<const uint32_t*>(image)[(tile * 64 + lane) * 4 + in / 32];
  const int q = (int)(w >> (4 * nibble_of(e))) & 15;
  const int64_t at = group_index(o, i / (kTileI / gpt), itiles, gpt);
  const int z = with_zeros ? (int)zeros[at] : 8;
  return (float)(q - z) * bf16_to_f32(scales[at]);
}

__global__ __launch_bounds__(256) void nibble_unpack_kernel(const uint8_t* image,
                                                            const bf16raw* scales,
                                                            const uint8_t* zeros, float* W,
                                                            int64_t O, int64_t I, int64_t itiles,
                                                            int gpt, int with_zeros) {
  for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < O * I;
       w += (int64_t)gridDim.x * 256)
    W[w] = weight_at(image, scales, zeros, w / I, w % I, itiles, gpt, with_zeros != 0);
}

// ---- product -----------------------------------------------------------------

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

// Eight codes of a dword as bf16 values 0..15.
__device__ __forceinline__ bf16x8 codes_bf16(uint32_t w) {
  const uint32_t lo = w & 0x0f0f0f0fu, hi = (w >> 4) & 0x0f0f0f0fu;
  u32x4 v;
  v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, false));
  v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, true));
  v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, false));
  v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, true));
  return as_bf16x8(v);
}

// Upper halves of two words, a below b.
__device__ __forceinline__ uint32_t upper2(uint32_t a, uint32_t b) {
  return __builtin_amdgcn_perm(b, a, 0x07060302u);
}

// Eight codes of a dword less their zero point, as bf16: q - z with ZERO, where `less` holds
// 128 - z in each byte; else 16 (q - 8), a code moved to the upper half of its byte. Either is
// a signed byte, whose float has its bits in the upper half.
constexpr float kExactUnit = 0.0625f;  // of the latter
template <bool ZERO>
__device__ __forceinline__ bf16x8 codes_less_zero(uint32_t w, uint32_t less) {
  uint32_t lo, hi;
  if (ZERO) {
    lo = ((w & 0x0f0f0f0fu) + less) ^ 0x80808080u;
    hi = (((w >> 4) & 0x0f0f0f0fu) + less) ^ 0x80808080u;
  } else {
    lo = ((w << 4) ^ 0x80808080u) & 0xf0f0f0f0u;
    hi = (w ^ 0x80808080u) & 0xf0f0f0f0u;
  }
  float f[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[e] = (float)(int8_t)(lo >> (8 * e));
    f[4 + e] = (float)(int8_t)(hi >> (8 * e));
  }
  u32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    v[e] = upper2(__float_as_uint(f[2 * e]), __float_as_uint(f[2 * e + 1]));
  return as_bf16x8(v);
}

// Eight elements of X from column i, as PARTS bf16 operands: bf16 as they are, fp32
// cut in three (each part the upper 16 bits of what is left: exact, and of no
// larger magnitude, so nothing overflows; an infinity's rest is NaN, and such
// outputs are taken again one by one). Columns past I are zero.
template <typename T>
struct XLoad;
template <>
struct XLoad<bf16raw> {
  static constexpr int kParts = 1;
  u32x4 v;
  __device__ __forceinline__ void full(const bf16raw* p) {
    v = *reinterpret_cast<const u32x4_a2*>(p);
  }
  __device__ __forceinline__ void tail(const bf16raw* row, int64_t i, int64_t I) {
    uint32_t u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = row[i + e < I ? i + e : I - 1];
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = i + e < I ? u[e] : 0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = u[2 * e] | u[2 * e + 1] << 16;
  }
  __device__ __forceinline__ void parts(bf16x8 (&out)[1]) const { out[0] = as_bf16x8(v); }
};
template <>
struct XLoad<float> {
  static constexpr int kParts = 3;
  float v[8];
  __device__ __forceinline__ void full(const float* p) {
    const f32x4 a = *reinterpret_cast<const f32x4_a4*>(p);
    const f32x4 b = *reinterpret_cast<const f32x4_a4*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
  }
  __device__ __forceinline__ void tail(const float* row, int64_t i, int64_t I) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = row[i + e < I ? i + e : I - 1];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = i + e < I ? v[e] : 0.0f;
  }
  __device__ __forceinline__ void parts(bf16x8 (&out)[3]) const {
    u32x4 w[3];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float a = v[2 * e], b = v[2 * e + 1];
#pragma unroll
      for (int p = 0; p < 3; ++p) {
        const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
        w[p][e] = upper2(ua, ub);
        a -= __uint_as_float(ua & 0xffff0000u);
        b -= __uint_as_float(ub & 0xffff0000u);
      }
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) out[p] = as_bf16x8(w[p]);
  }
};

// One output by itself, by a whole wave, for those that are not finite: the formula in
// 64 bits, in which no partial sum overflows. The same in all lanes.
template <typename T>
__device__ __noinline__ float product_one(const T* x, const uint8_t* image, const bf16raw* scales,
                                          const uint8_t* zeros, int64_t o, int64_t I,
                                          int64_t itiles, int gpt, bool with_zeros) {
  double y = 0.0;
  for (int64_t i = threadIdx.x & 63; i < I; i += 64)
    y = fma((double)load_elem(x, i),
            (double)weight_at(image, scales, zeros, o, i, itiles, gpt, with_zeros), y);
  for (int off = 1; off < 64; off <<= 1) y += __shfl_xor(y, off, kWave);
  return (float)y;
}

// What a wave loads of an input tile: codes, scales and zero points of TD output
// tiles, and X.
template <int GPT, bool ZERO, int TD>
struct WeightFrag {
  u32x4 code[TD];
  u32x2 sc[TD][GPT];
  uint32_t zp[TD][ZERO ? GPT : 1];
};

// Large matrices are read once and do not fit the caches: their loads pass by
// (STREAM). Reading alone reaches 6.3 TB/s with ordinary loads and 7.1 so.
template <bool STREAM, typename V>
__device__ __forceinline__ V load_weights(const V* p) {
  if constexpr (STREAM)
    return __builtin_nontemporal_load(p);
  else
    return *p;
}

// Eight inputs from column 8 ch of a row, as operands.
template <typename T>
__device__ __forceinline__ void x_operands(const T* row, int64_t ch, int64_t I,
                                           bf16x8 (&out)[XLoad<T>::kParts]) {
  XLoad<T> v;
  if (8 * ch + 8 <= I)
    v.full(row + 8 * ch);
  else
    v.tail(row, 8 * ch, I);
  v.parts(out);
}

// X as operands in memory: [input tile][tile of 16 rows][step][part][lane]. Rows past N
// are zero. A workgroup lays out an input tile (x) of 16 rows (y).
template <typename T>
__global__ __launch_bounds__(256) void nibble_x_kernel(const T* __restrict__ X, int64_t ldx,
                                                       int64_t N, int64_t I, bf16x8* out) {
  constexpr int P = XLoad<T>::kParts;
  const int lane = threadIdx.x & 63, s = threadIdx.x >> 6;
  const int64_t it = blockIdx.x, nt = blockIdx.y, n = nt * 16 + lane % 16;
  bf16x8 parts[P] = {};
  if (n < N) x_operands(X + n * ldx, it * 16 + 4 * s + lane / 16, I, parts);
#pragma unroll
  for (int p = 0; p < P; ++p)
    out[(((it * gridDim.y + nt) * 4 + s) * P + p) * 64 + lane] = parts[p];
}

// NT tiles of 16 rows of X, TD tiles of 16 outputs, GPT groups in an input tile.
// XLDS (NT = 1): the workgroup first lays X out in LDS as operands, [input tile][step][part]
// [l / 16][row]; the lanes of columns past N read the last row's. Otherwise nibble_x_kernel
// has done so in memory (xop): a wave's load is 1 KiB in a row, where reading the rows
// of X themselves meets few of the L2's channels (strides of powers of two) and
// takes as long for one row as for sixteen.
// EXACT: zero points are taken off the codes, else off the sums (bf16 X and Y alone).
template <typename T, int GPT, bool ZERO, int NT, int TD, bool STREAM, bool XLDS, bool EXACT>
__global__ __launch_bounds__(512) void nibble_product_kernel(
    const T* __restrict__ X, int64_t ldx, const bf16x8* __restrict__ xop, int ntiles,
    const uint8_t* __restrict__ image, int64_t scales_at, int64_t zeros_at, void* __restrict__ Y,
    int64_t ldy, int64_t N, int64_t O, int64_t I, int64_t otiles, int itiles, int y_dt, int act) {
  constexpr int P = XLoad<T>::kParts;
  constexpr int STEPS = 4 / GPT;  // matrix steps of 32 inputs in a group
  typedef WeightFrag<GPT, ZERO, TD> Frag;
  extern __shared__ f32x4 sums[];  // [waves][TD][NT][64]; XLDS: X first
  // (the wave's number in a scalar register: addresses of its tiles too)
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int col = lane & 15, quad = lane >> 4;
  // the workgroups of one set of output tiles follow each other
  const int nblocks = (ntiles + NT - 1) / NT;
  const int64_t ot0 = (int64_t)(blockIdx.x / nblocks) * TD;
  const int nt0 = (int)(blockIdx.x % nblocks) * NT;
  const bf16raw* scales = reinterpret_cast<const bf16raw*>(image + scales_at);
  const uint8_t* zeros = image + zeros_at;

  // per output tile, the row of input tiles (tiles past the last repeat it)
  int64_t row[TD];
#pragma unroll
  for (int d = 0; d < TD; ++d) row[d] = (ot0 + d < otiles ? ot0 + d : otiles - 1) * itiles;

  f32x4 acc[TD][NT];
#pragma unroll
  for (int d = 0; d < TD; ++d)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[d][t] = f32x4{0, 0, 0, 0};
  u32x4 ones_w;
#pragma unroll
  for (int e = 0; e < 4; ++e) ones_w[e] = ZERO ? 0x3f803f80u : 0xc100c100u;  // 1, or -8
  const bf16x8 ones = as_bf16x8(ones_w);

  auto load = [&](int it, Frag& f) {
#pragma unroll
    for (int d = 0; d < TD; ++d) {
      const int64_t tile = row[d] + it;
      f.code[d] = load_weights<STREAM>(reinterpret_cast<const u32x4*>(image + tile * 1024) + lane);
#pragma unroll
      for (int g = 0; g < GPT; ++g) {
        f.sc[d][g] = load_weights<STREAM>(
            reinterpret_cast<const u32x2*>(scales + tile * (16 * GPT)) + quad * GPT + g);
        if (ZERO && EXACT)  // of the output whose codes the lane holds
          f.zp[d][g] = load_weights<STREAM>(zeros + tile * (16 * GPT) +
                                            ((col / 4) * GPT + g) * 4 + col % 4);
        else if (ZERO)  // of the four whose sums it will hold
          f.zp[d][g] = load_weights<STREAM>(
              reinterpret_cast<const uint32_t*>(zeros + tile * (16 * GPT)) + quad * GPT + g);
      }
    }
  };
  struct Operands {
    bf16x8 v[XLDS ? 1 : NT][4][P];
  };
  auto load_x = [&](int it, Operands& x) {
#pragma unroll
    for (int t = 0; t < (XLDS ? 0 : NT); ++t) {
      const int nt = nt0 + t < ntiles ? nt0 + t : ntiles - 1;  // (never written)
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int p = 0; p < P; ++p)
          x.v[t][s][p] = xop[((((int64_t)it * ntiles + nt) * 4 + s) * P + p) * 64 + lane];
    }
  };
  const bf16x8* xs = reinterpret_cast<const bf16x8*>(sums);
  const int lds_rows = N - 16 * nt0 < 16 ? (int)(N - 16 * nt0) : 16;  // of X in LDS
  // what the sums of x q start from: -z sum x
  auto start = [](const Frag& f, int d, int g, int r, float one) {
    return ZERO ? -(float)((f.zp[d][g] >> (8 * r)) & 255u) * one : one;
  };
  auto multiply = [&](const Frag& f, const Operands& x, int it) {
#pragma unroll
    for (int g = 0; g < GPT; ++g) {
      bf16x8 xp[STEPS][NT][P];
      f32x4 one[NT];  // -8 sum x, or sum x
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        one[t] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
          for (int p = 0; p < P; ++p) {
            if constexpr (XLDS)
              xp[s][t][p] = xs[((it * 4 + g * STEPS + s) * P + p) * 4 * lds_rows];
            else
              xp[s][t][p] = x.v[t][g * STEPS + s][p];
            if (!EXACT)
              one[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, xp[s][t][p], one[t], 0, 0, 0);
          }
      }
#pragma unroll
      for (int d = 0; d < TD; ++d) {
        f32x4 sum[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            sum[t][r] = EXACT ? 0.0f : start(f, d, g, r, one[t][r]);
        uint32_t less = 0;
        if (ZERO && EXACT) less = 0x80808080u - __builtin_amdgcn_perm(0, f.zp[d][g], 0u);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
          const uint32_t w = f.code[d][g * STEPS + s];
          const bf16x8 q = EXACT ? codes_less_zero<ZERO>(w, less) : codes_bf16(w);
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int p = 0; p < P; ++p)
              sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q, xp[s][t][p], sum[t], 0, 0, 0);
        }
        const u32x2 sc = f.sc[d][g];
        const float sf[4] = {__uint_as_float(sc[0] << 16), __uint_as_float(sc[0] & 0xffff0000u),
                             __uint_as_float(sc[1] << 16), __uint_as_float(sc[1] & 0xffff0000u)};
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[d][t][r] = fmaf(sf[r], sum[t][r], acc[d][t][r]);
      }
    }
  };

  // Two tiles' registers: one tile's loads are in flight while the other is multiplied.
  // They are issued without a condition, past the end for the last tile again, so that a
  // wait covers only the older ones; the scheduling barriers keep the compiler from
  // sinking them to their uses.
  const int own = itiles > wave ? (itiles - wave + waves - 1) / waves : 0;
  auto nth = [&](int i) { return wave + waves * (i < own ? i : own - 1); };
  Frag f[2];
  Operands x[2];
  if (own > 0) {
    load(nth(0), f[0]);
    load_x(nth(0), x[0]);
  }
  if (XLDS) {
    const int rows = lds_rows, chunks = itiles * 16;  // of eight inputs
    bf16x8* dst = reinterpret_cast<bf16x8*>(sums);
    for (int c = threadIdx.x; c < chunks * rows; c += blockDim.x) {
      const int n = c / chunks, ch = c % chunks;
      bf16x8 parts[P];
      x_operands(X + (16 * nt0 + n) * ldx, ch, I, parts);
#pragma unroll
      for (int p = 0; p < P; ++p) dst[((ch / 4 * P + p) * 4 + ch % 4) * rows + n] = parts[p];
    }
    __syncthreads();
    xs += quad * rows + (col < rows ? col : rows - 1);
  }
  if (own > 0) {
    int i = 0;
    for (; i + 2 <= own; i += 2) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        load(nth(i + r + 1), f[1 - r]);
        load_x(nth(i + r + 1), x[1 - r]);
        __builtin_amdgcn_sched_barrier(0);
        multiply(f[r], x[r], nth(i + r));
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (i < own) multiply(f[0], x[0], nth(i));
  }

  if (XLDS) __syncthreads();  // X is no longer read
  const int64_t n0 = (int64_t)nt0 * 16;
#pragma unroll
  for (int d = 0; d < TD; ++d)
#pragma unroll
    for (int t = 0; t < NT; ++t) sums[((wave * TD + d) * NT + t) * 64 + lane] = acc[d][t];
  __syncthreads();
  for (int j = wave; j < TD * NT; j += waves) {
    const int d = j / NT, t = j % NT;
    f32x4 y = sums[j * 64 + lane];
    for (int w = 1; w < waves; ++w) y += sums[(w * TD * NT + j) * 64 + lane];
    const int64_t n = n0 + 16 * t + col;
    const int64_t o0 = (ot0 + d) * kTileO + 4 * quad;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t o = o0 + r;
      const bool live = n < N && o < O;
      float v = EXACT && !ZERO ? y[r] * kExactUnit : y[r];
      // Not finite: an infinity or NaN in X, or a part of the sum past the range that the
      // whole stays within. Taken again as the formula says.
      for (uint64_t again = __ballot(live && !(fabsf(v) < INFINITY)); again; again &= again - 1) {
        const int from = (int)__builtin_ctzll(again);
        const int64_t nf = n0 + 16 * t + from % 16, of = (ot0 + d) * kTileO + 4 * (from / 16) + r;
        const float w = product_one(X + nf * ldx, image, scales, zeros, of, I, (int64_t)itiles,
                                    GPT, ZERO);
        if (lane == from) v = w;
      }
      if (!live) continue;
      v = activate(v, act);
      if (y_dt == 0)
        static_cast<float*>(Y)[n * ldy + o] = v;
      else
        static_cast<bf16raw*>(Y)[n * ldy + o] = to_bf16(v);
    }
  }
}

// X in LDS: two workgroups to a compute unit, or (fp32, of whose kernels a compute unit
// holds one workgroup anyway) one.
constexpr size_t kXLds = 64 * 1024, kXLdsOne = 128 * 1024;

struct ProductArgs {
  const void* X;
  int64_t ldx;
  const bf16x8* xop;  // X laid out
  const uint8_t* image;
  void* Y;
  int64_t ldy, N, O, I;
  NibbleLayout L;
  int lds_tiles, y_dt, act;
  bool exact;
  hipStream_t stream;
};

constexpr int64_t kMaxThreads = (int64_t(1) << 32) - 1;  // of a launch

constexpr int parts_of(int x_dt) { return x_dt == 0 ? 3 : 1; }

// Bytes of X as operands in LDS, up to 16 rows.
size_t x_lds_bytes(int64_t N, int64_t itiles, int x_dt) {
  return (size_t)(N < 16 ? N : 16) * itiles * 256 * parts_of(x_dt);
}
bool x_in_lds(int64_t N, int64_t itiles, int x_dt) {
  return N <= 16 && x_lds_bytes(N, itiles, x_dt) <= kXLds;
}

// Output tiles of a workgroup that keeps X in LDS; 0: X is laid out in memory. Each workgroup
// lays X out again, so where it fills half of the LDS (fp32; bf16 gains nothing) that pays if
// all of them run at once (1 x 16384 x 700: 18.5 us, with X in memory 24.1; 4 x 4096 x 10240 in
// three tiles: 11.6 and 14.4; but 4 x 4096 x 28672 in four: 26.3 and 21.6), and for one row always,
// which X in memory holds sixteen times (1 x 16384 x 57344: 136 and 154).
int lds_tiles(int64_t N, int64_t otiles, int64_t itiles, int x_dt) {
  if (x_in_lds(N, itiles, x_dt)) return 2;
  // More rows: each workgroup a tile of 16, where the workgroups run at once and together
  // lay out little, for a launch less of the host's time (20 x 1000 x 8192 bf16: 9.1 us a call,
  // with X in memory 10.8; fp32 64 x 617 x 4096 8.9 and 11.1, 64 x 1280 x 2000 8.8 and 11.0, though
  // inside a graph 8.7 and 7.4, 8.0 and 7.1; but 64 x 2000 x 4096 bf16 12.8 and 11.4,
  // 20 x 617 x 10240 fp32 13.3 and 11.0).
  const size_t bytes = x_lds_bytes(N, itiles, x_dt);
  const int64_t cus = num_cus();
  if (N > 16) {
    const int64_t groups = cdiv(otiles, 2) * cdiv(N, 16);
    const bool fits = bytes <= kXLds ? groups <= 2 * cus
                                     : x_dt == 0 && bytes <= kXLdsOne && groups <= cus;
    return fits && groups * itiles <= 16 * cus ? 2 : 0;
  }
  if (x_dt != 0 || bytes > kXLdsOne) return 0;
  for (int tiles = 2; tiles <= 4; ++tiles)
    if (cdiv(otiles, tiles) <= cus) return tiles;
  return N == 1 ? 4 : 0;
}

template <typename T, int GPT, bool ZERO, int NT, int TD, bool STREAM, bool XLDS, bool EXACT>
hipError_t launch_product_kernel(const ProductArgs& a) {
  // Eight waves share the input tiles; without X in LDS four where two row tiles or four output
  // tiles take more than 128 registers, so that two or three workgroups of them fit where one
  // of eight would (32 x 3072 x 10240: 12.4 us with eight, 11.2 with four; fp32 32 x 8192 x
  // 16384, four output tiles: 43.6 and 40.9).
  const int most = !XLDS && (NT == 2 || TD > 2) ? 4 : 8;
  const int waves = a.L.itiles < most ? (int)a.L.itiles : most;
  const int ntiles = (int)cdiv(a.N, 16);
  size_t lds = sizeof(f32x4) * 64 * TD * NT * waves;
  if (XLDS) {
    const size_t x = x_lds_bytes(a.N, a.L.itiles, sizeof(T) == 4 ? 0 : 1);
    if (x > lds) lds = x;
  }
  const auto kernel = nibble_product_kernel<T, GPT, ZERO, NT, TD, STREAM, XLDS, EXACT>;
  if (lds > 64 * 1024) {  // above the default limit: raised once per device and kernel
    static PerDeviceOnce once;
    const hipError_t e = once_per_device(once, [&] {
      return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                 hipFuncAttributeMaxDynamicSharedMemorySize, (int)kXLdsOne);
    });
    if (e != hipSuccess) return e;
  }
  // A launch holds fewer than 2^32 threads; outputs past those of the first take more. (The
  // offsets of scales and zero points count from the codes that a launch begins at.)
  const int64_t rows = cdiv(ntiles, NT), step = kMaxThreads / (64 * waves * rows) * TD;
  for (int64_t t0 = 0; t0 < a.L.otiles; t0 += step) {
    const int64_t tiles = t0 * a.L.itiles, left = a.L.otiles - t0;
    const int64_t here = left < step ? left : step;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(cdiv(here, TD) * rows)), dim3(64 * waves), lds,
                       a.stream, static_cast<const T*>(a.X), a.ldx, a.xop, ntiles,
                       a.image + tiles * 1024,
                       (int64_t)a.L.scales + tiles * (16 * GPT * 2 - 1024),
                       (int64_t)a.L.zeros + tiles * (16 * GPT - 1024),
                       static_cast<char*>(a.Y) + t0 * kTileO * (a.y_dt == 0 ? 4 : 2), a.ldy, a.N,
                       a.O - t0 * kTileO < here * kTileO ? a.O - t0 * kTileO : here * kTileO, a.I,
                       here, (int)a.L.itiles, a.y_dt, a.act);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T, int GPT, bool ZERO, int NT, int TD, bool STREAM, bool XLDS>
hipError_t launch_product_as(const ProductArgs& a) {
  if constexpr (sizeof(T) == 2)
    if (!a.exact) return launch_product_kernel<T, GPT, ZERO, NT, TD, STREAM, XLDS, false>(a);
  return launch_product_kernel<T, GPT, ZERO, NT, TD, STREAM, XLDS, true>(a);
}

// Above three quarters of the 256 MiB cache that the dies share a matrix does not stay there
// from call to call, and loads that pass by are faster (one row of bf16, 16384 inputs: 470 MB of
// codes 84.0 us a call instead of 86.3, 235 MB 47.4 instead of 50.0); below they would lose
// what stays (134 MB: 26.2 instead of 24.5).
constexpr size_t kStreamBytes = size_t(192) << 20;

// X laid out in memory is read once for each workgroup's output tiles, and that weighs more
// than the codes: four tiles (WIDE) instead of two halve it, but leave half the workgroups.
// * fp32: where two tiles make more workgroups than compute units, of which each holds
//   one (16 x 4096 x 10240: 14.7 us, with two tiles 18.0; 64 x 4096 x 16384: 42 and 61; but 16 x
//   4096 x 8192, 256 workgroups: 14.3 and 11.9);
// * bf16: where four tiles leave 7/4 workgroups for each compute unit, and two input tiles for
//   each wave (32 x 8192 x 28672: 32.7 us, with two 37.9; 64 x 8192 x 16384: 31.4 and 38.2; but 64
//   x 8192 x 12288, 384 workgroups: 36 and 34).
// The zero points of groups of 32 leave registers for three in fp32 and, with two row tiles,
// for two.
template <typename T, int GPT, bool ZERO, int NT, bool STREAM>
hipError_t launch_product_laid(const ProductArgs& a) {
  constexpr int WIDE = !(GPT == 4 && ZERO) ? 4 : NT == 2 ? 2 : sizeof(T) == 4 ? 3 : 4;
  const int64_t rows = cdiv(a.N, 16 * NT), cus = num_cus();
  const bool wide = sizeof(T) == 4 ? cdiv(a.L.otiles, 2) * rows > cus
                                   : cdiv(a.L.otiles, 4) * rows >= 7 * cus / 4 && a.L.itiles >= 8;
  if constexpr (WIDE > 2)
    if (wide) return launch_product_as<T, GPT, ZERO, NT, WIDE, STREAM, false>(a);
  return launch_product_as<T, GPT, ZERO, NT, 2, STREAM, false>(a);
}

template <typename T, int GPT, bool ZERO>
hipError_t launch_product_rows(const ProductArgs& a) {
  const bool stream = a.L.scales > kStreamBytes;
  if constexpr (sizeof(T) == 4) {
    // (codes past the caches have more output tiles than three of them to a compute unit)
    if (a.lds_tiles == 4)
      return stream ? launch_product_as<T, GPT, ZERO, 1, 4, true, true>(a)
                    : launch_product_as<T, GPT, ZERO, 1, 4, false, true>(a);
    if (a.lds_tiles == 3) return launch_product_as<T, GPT, ZERO, 1, 3, false, true>(a);
  }
  if (a.lds_tiles == 2)
    return stream ? launch_product_as<T, GPT, ZERO, 1, 2, true, true>(a)
                  : launch_product_as<T, GPT, ZERO, 1, 2, false, true>(a);
  if (a.N <= 16 && stream) return launch_product_laid<T, GPT, ZERO, 1, true>(a);
  // (fp32's three parts of two row tiles would not fit the registers)
  if (a.N <= 16 || sizeof(T) == 4) return launch_product_laid<T, GPT, ZERO, 1, false>(a);
  if constexpr (sizeof(T) == 2) return launch_product_laid<T, GPT, ZERO, 2, false>(a);
}

template <typename T>
hipError_t launch_product_typed(const ProductArgs& a, int G, bool zero) {
  switch (G) {
    case 32:
      return zero ? launch_product_rows<T, 4, true>(a) : launch_product_rows<T, 4, false>(a);
    case 64:
      return zero ? launch_product_rows<T, 2, true>(a) : launch_product_rows<T, 2, false>(a);
    default:
      return zero ? launch_product_rows<T, 1, true>(a) : launch_product_rows<T, 1, false>(a);
  }
}

unsigned blocks_for(int64_t total) {
  const int64_t g = cdiv(total, 256);
  return (unsigned)(g < 65536 ? g : 65536);
}

}  // namespace

NibbleLayout nibble_layout(int64_t O, int64_t I, int G) { return layout_of(O, I, G); }

hipError_t launch_nibble_pack(const uint8_t* codes, const bf16raw* scales, const uint8_t* zeros,
                              int64_t O, int64_t I, int G, void* image, hipStream_t stream) {
  const NibbleLayout L = layout_of(O, I, G);
  uint8_t* im = static_cast<uint8_t*>(image);
  const int gpt = kTileI / G;
  const int64_t words = L.otiles * L.itiles * 256, groups = L.otiles * L.itiles * gpt * kTileO;
  const bool aligned = (uintptr_t)codes % 4 == 0 && cdiv(I, 2) % 4 == 0;
  hipLaunchKernelGGL(nibble_pack_kernel, dim3(blocks_for(words)), dim3(256), 0, stream, codes, O,
                     I, L.itiles, (int)aligned, words, reinterpret_cast<uint32_t*>(im));
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(nibble_pack_groups_kernel, dim3(blocks_for(groups)), dim3(256), 0, stream,
                     scales, zeros, O, cdiv(I, G), L.itiles, gpt, groups,
                     reinterpret_cast<bf16raw*>(im + L.scales), im + L.zeros);
  return hipGetLastError();
}

hipError_t launch_nibble_quantize(const void* W, int64_t ldw, bool in_rows, int64_t O, int64_t I,
                                  int G, bool with_zeros, int dt, void* image,
                                  hipStream_t stream) {
  const NibbleLayout L = layout_of(O, I, G);
  uint8_t* im = static_cast<uint8_t*>(image);
  const dim3 grid((unsigned)(L.otiles * L.itiles));
  bf16raw* s = reinterpret_cast<bf16raw*>(im + L.scales);
  if (dt == 0)
    hipLaunchKernelGGL(nibble_quantize_kernel<float>, grid, dim3(64), 0, stream,
                       static_cast<const float*>(W), ldw, (int)in_rows, O, I, L.itiles,
                       kTileI / G, (int)with_zeros, reinterpret_cast<u32x4*>(im), s,
                       im + L.zeros);
  else
    hipLaunchKernelGGL(nibble_quantize_kernel<bf16raw>, grid, dim3(64), 0, stream,
                       static_cast<const bf16raw*>(W), ldw, (int)in_rows, O, I, L.itiles,
                       kTileI / G, (int)with_zeros, reinterpret_cast<u32x4*>(im), s,
                       im + L.zeros);
  return hipGetLastError();
}

hipError_t launch_nibble_unpack(const void* image, float* W, int64_t O, int64_t I, int G,
                                bool with_zeros, hipStream_t stream) {
  const NibbleLayout L = layout_of(O, I, G);
  const uint8_t* im = static_cast<const uint8_t*>(image);
  hipLaunchKernelGGL(nibble_unpack_kernel, dim3(blocks_for(O * I)), dim3(256), 0, stream, im,
                     reinterpret_cast<const bf16raw*>(im + L.scales), im + L.zeros, W, O, I,
                     L.itiles, kTileI / G, (int)with_zeros);
  return hipGetLastError();
}

size_t nibble_ws_bytes(int64_t N, int64_t I, int x_dt) {
  const int64_t itiles = cdiv(I, kTileI);
  if (x_in_lds(N, itiles, x_dt)) return 0;
  return (size_t)cdiv(N, 16) * itiles * 4096 * parts_of(x_dt);
}

hipError_t launch_nibble_product(const void* X, int64_t ldx, const void* image, void* Y,
                                 int64_t ldy, int64_t N, int64_t O, int64_t I, int G,
                                 bool with_zeros, int x_dt, int y_dt, int act, void* workspace,
                                 hipStream_t stream) {
  ProductArgs a{X,   ldx, nullptr, static_cast<const uint8_t*>(image), Y,  ldy, N, O,
                I,   layout_of(O, I, G), 0, y_dt, act, x_dt == 0 || y_dt == 0 || act == 0, stream};
  a.lds_tiles = lds_tiles(N, a.L.otiles, a.L.itiles, x_dt);
  if (a.lds_tiles == 0) {
    bf16x8* xop = static_cast<bf16x8*>(workspace);
    const int ntiles = (int)cdiv(N, 16);
    const dim3 grid((unsigned)a.L.itiles, (unsigned)ntiles), block(256);
    if (x_dt == 0)
      hipLaunchKernelGGL(nibble_x_kernel<float>, grid, block, 0, stream,
                         static_cast<const float*>(X), ldx, N, I, xop);
    else
      hipLaunchKernelGGL(nibble_x_kernel<bf16raw>, grid, block, 0, stream,
                         static_cast<const bf16raw*>(X), ldx, N, I, xop);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    a.xop = xop;
  }
  return x_dt == 0 ? launch_product_typed<float>(a, G, with_zeros)
                   : launch_product_typed<bf16raw>(a, G, with_zeros);
}

}  // namespace ops
}  // namespace hd
