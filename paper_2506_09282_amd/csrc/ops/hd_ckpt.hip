// Activations kept in 8 bits, and the class vectors' gradient read from them.
//
// A group is kCkptRows rows of one column d:
//   s = max |x| / 127 (times the fp32 nearest to 1/127),  q = rint(x * (1/s)) in -127..127,
// and a kept value stands for q * s. Columns, not rows, share a scale, because
// activations differ in size from channel to channel. A group that holds an
// infinity or NaN is kept as NaN.
//
//   dC[k,d] = sum over groups b of s[b,d] * sum_{n in b} dS[n,k] q[n,d]
//
// The column scale leaves the product's reduction (over n) alone: q goes to the
// bf16 matrix instruction as it is (8 bits, exact), bf16 dS too, and fp32 dS as
// the exact sum of three bf16 values; s multiplies the finished group in fp32. What bounds
// it is reading q once, N*D bytes, while K is small.
//
// Layout: [group of rows][16 rows of the group][column][16 bytes], then the scales
// [group][column]. A lane's 16-byte load is 16 rows of a column, half an operand pair of
// v_mfma_f32_32x32x16_bf16, neighbouring lanes are neighbouring columns, and
// storing is coalesced too. dS is first cut and laid out as the other
// operand (a small launch), so that the product's loop holds no transposition; in a short
// call each workgroup does that for itself.
//
// Measured: 4096 x 10240 fp32 kept 33.9 us (kernel; 212 MB, 6.3 TB/s) and taken back 30.8 (6.9
// TB/s), as a copy with such loads and stores. Gradient, 65536 x 10240 x 26 fp32: 164 to 177 us for
// a call's three launches in a row of calls (the product alone 174 to 192 under the profiler),
// where reading the 713 MB takes 100. Three matrix instructions for each step, a fifth of their
// rows past the 26 classes, keep the matrix units busy for 44% of the time and the bytes' way
// to bf16 the vector units for 44%: both run beside the loads, but hardly beside each other.
// 2999 x 10000 x 100 bf16, 36 MB: 21 to 23 us, of 29 for the call; 24 MB of partial sums of six
// slices are written beside them and read again by the join.
#include <type_traits>

#include "hd_ops.hpp"

namespace hd {
namespace ops {

namespace {

constexpr int kRows = kCkptRows;
constexpr float kInv127 = 1.0f / 127.0f;

__host__ __device__ inline int64_t groups_of(int64_t N) { return cdiv(N, kRows); }
__host__ __device__ inline int64_t scales_at(int64_t N, int64_t D) {
  return (groups_of(N) * kRows * D + 255) / 256 * 256;
}

// ---- store and load --------------------------------------------------------------

// How a lane's four columns of 256 lie. Where rows start at multiples of 16 bytes (8 in
// bf16) they are neighbours, in one load; elsewhere they are 64 apart and each load of a
// wave is a run, which is faster than wide loads across the lines' ends (1999 x 4097
// bf16 kept: 11.8 us wide, 9.4 so). ..Once: past the caches (kStreamBytes) rows pass once and do
// not stay there, the kept values, a quarter or half as large, do (4096 x 10240 fp32, 168 MB,
// kept and taken back: 70.3 us instead of 81.5; 84 MB: 37.1 instead of 35.9; 65536 x 1001 fp32
// kept: 68 instead of 106; 16384 x 8000 taken back: 97 instead of 120).
enum Columns { kApart, kApartOnce, kNear, kNearOnce };
constexpr bool near(int m) { return m == kNear || m == kNearOnce; }
constexpr bool once(int m) { return m == kApartOnce || m == kNearOnce; }
constexpr int64_t kStreamBytes = int64_t(96) << 20;

template <int M>
__device__ __forceinline__ int64_t column_of(int64_t d0, int lane, int c) {
  return near(M) ? d0 + 4 * lane + c : d0 + 64 * c + lane;
}

template <bool ONCE, typename T>
__device__ __forceinline__ float load_row1(const T* p) {
  const T x = ONCE ? __builtin_nontemporal_load(p) : *p;
  return load_elem(&x, 0);
}
template <bool ONCE>
__device__ __forceinline__ void load_row4(const float* p, float (&v)[4]) {
  const f32x4* at = reinterpret_cast<const f32x4*>(p);
  const f32x4 x = ONCE ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
  for (int c = 0; c < 4; ++c) v[c] = x[c];
}
template <bool ONCE>
__device__ __forceinline__ void load_row4(const bf16raw* p, float (&v)[4]) {
  const u32x2* at = reinterpret_cast<const u32x2*>(p);
  const u32x2 x = ONCE ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
  for (int c = 0; c < 4; ++c)
    v[c] = __uint_as_float(c % 2 ? x[c / 2] & 0xffff0000u : x[c / 2] << 16);
}
template <bool ONCE>
__device__ __forceinline__ void store_row4(float* p, const float (&v)[4]) {
  f32x4* at = reinterpret_cast<f32x4*>(p);
  const f32x4 x = {v[0], v[1], v[2], v[3]};
  if (ONCE)
    __builtin_nontemporal_store(x, at);
  else
    *at = x;
}
template <bool ONCE>
__device__ __forceinline__ void store_row4(bf16raw* p, const float (&v)[4]) {
  u32x2* at = reinterpret_cast<u32x2*>(p);
  const u32x2 x = {(uint32_t)to_bf16(v[0]) | (uint32_t)to_bf16(v[1]) << 16,
                   (uint32_t)to_bf16(v[2]) | (uint32_t)to_bf16(v[3]) << 16};
  if (ONCE)
    __builtin_nontemporal_store(x, at);
  else
    *at = x;
}

// A workgroup takes a group of 256 columns: a wave 16 of its rows, a lane four
// columns; the waves' largest values meet in LDS.
template <typename T, int M>
__global__ __launch_bounds__(256) void ckpt_store_kernel(const T* __restrict__ H, int64_t ldh,
                                                         int64_t N, int64_t D, u32x4* out,
                                                         float* out_s) {
  __shared__ u32x4 tops[4][64];
  const int lane = threadIdx.x & 63, ch = threadIdx.x >> 6;
  const int64_t d0 = (int64_t)blockIdx.x * 256, b = blockIdx.y;
  const int64_t n0 = b * kRows + 16 * ch;
  float v[16][4];
  // rows and columns past the end read the last one again, so that no load waits on a branch
  const T* col[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int64_t d = column_of<M>(d0, lane, c);
    col[c] = H + (d < D ? d : D - 1);
  }
  if (near(M) && d0 + 256 <= D) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
      load_row4<once(M)>(col[0] + (n0 + r < N ? n0 + r : N - 1) * ldh, v[r]);
  } else if (near(M) && D % 4 == 0) {  // a lane's four columns are all there or all past D
    const T* four = H + (d0 + 4 * lane < D ? d0 + 4 * lane : D - 4);
#pragma unroll
    for (int r = 0; r < 16; ++r)
      load_row4<once(M)>(four + (n0 + r < N ? n0 + r : N - 1) * ldh, v[r]);
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        v[r][c] = load_row1<once(M)>(col[c] + (n0 + r < N ? n0 + r : N - 1) * ldh);
  }
  if (n0 + 16 > N) {
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int c = 0; c < 4; ++c) v[r][c] = n0 + r < N ? v[r][c] : 0.0f;
  }
  u32x4 top = {0, 0, 0, 0};  // as bits, an infinity and NaN are larger than any number
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t a = __float_as_uint(v[r][c]) & 0x7fffffffu;
      top[c] = a > top[c] ? a : top[c];
    }
  tops[ch][lane] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const u32x4 t = tops[w][lane];
#pragma unroll
    for (int c = 0; c < 4; ++c) top[c] = t[c] > top[c] ? t[c] : top[c];
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int64_t d = column_of<M>(d0, lane, c);
    const bool bad = top[c] >= 0x7f800000u;
    const float s = __uint_as_float(top[c]) * kInv127;
    float inv = 1.0f / s;
    if (bad || !(inv < INFINITY)) inv = 0.0f;  // 0, or too small for its inverse: kept as 0
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float q = rintf((bad ? 0.0f : v[4 * i + e][c]) * inv);
        w[i] |= ((uint32_t)(int)fminf(fmaxf(q, -127.0f), 127.0f) & 255u) << (8 * e);
      }
    }
    if (d < D) {
      out[(b * 4 + ch) * D + d] = w;
      if (ch == 0) out_s[b * D + d] = bad ? NAN : s;
    }
  }
}

// A lane takes 16 rows of four columns.
template <typename T, int M>
__global__ __launch_bounds__(256) void ckpt_load_kernel(const u32x4* __restrict__ q,
                                                        const float* __restrict__ scale, T* H,
                                                        int64_t ldh, int64_t N, int64_t D) {
  const int lane = threadIdx.x & 63, ch = threadIdx.x >> 6;
  const int64_t d0 = (int64_t)blockIdx.x * 256, b = blockIdx.y;
  const int64_t n0 = b * kRows + 16 * ch;
  u32x4 w[4];
  float s[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int64_t d = column_of<M>(d0, lane, c), in = d < D ? d : D - 1;
    w[c] = q[(b * 4 + ch) * D + in];
    s[c] = scale[b * D + in];
  }
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    if (n0 + e >= N) break;
    float v[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) v[c] = (float)(int8_t)(w[c][e / 4] >> (8 * (e % 4))) * s[c];
    T* row = H + (n0 + e) * ldh;
    if (near(M) && (d0 + 256 <= D || D % 4 == 0)) {
      if (d0 + 4 * lane < D) store_row4<once(M)>(row + d0 + 4 * lane, v);
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int64_t d = column_of<M>(d0, lane, c);
        if (d < D) store_elem(row, d, v[c]);
      }
    }
  }
}

bool rows_aligned(const void* rows, int64_t ld, int dt) {
  return (uintptr_t)rows % (dt == 0 ? 16 : 8) == 0 && ld % 4 == 0;
}
Columns columns_of(const void* rows, int64_t ld, int64_t N, int64_t D, int dt) {
  const bool past = N * D * (dt == 0 ? 4 : 2) > kStreamBytes;
  // (fewer columns than a workgroup's would leave lanes of every load without work)
  if (rows_aligned(rows, ld, dt) && D >= 256) return past ? kNearOnce : kNear;
  return past ? kApartOnce : kApart;
}

// ---- the other operand --------------------------------------------------------------

// dS as operand fragments: [group][tile of 32 rows][8 rows of half a wave: p, j]
// [part][lane][16 bytes]; lane l holds row l % 32 of the tile, samples 32 p + 16 (l / 32)
// + 8 j + e. A row of the operand is a class; with few classes (FOLD) the three parts of
// fp32 are rows of their own, [part][class], which fills the tiles better.
constexpr int kSteps = kRows / 16;  // matrix steps of a group

// Eight values as P parts of an operand, or (FOLD) as the one part `part` (past 2: none).
template <typename T, int P, bool FOLD>
__device__ __forceinline__ void cut(float (&v)[8], int part, u32x4 (&out)[P]) {
#pragma unroll
  for (int p = 0; p < (FOLD ? 3 : P); ++p) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t a = __float_as_uint(v[2 * e]), c = __float_as_uint(v[2 * e + 1]);
      w[e] = __builtin_amdgcn_perm(c, a, 0x07060302u);
      // what is left; nothing of an infinity or NaN, whose first part says all
      v[2 * e] = (a & 0x7f800000u) == 0x7f800000u ? 0.0f
                                                  : v[2 * e] - __uint_as_float(a & 0xffff0000u);
      v[2 * e + 1] = (c & 0x7f800000u) == 0x7f800000u
                         ? 0.0f
                         : v[2 * e + 1] - __uint_as_float(c & 0xffff0000u);
      // (a NaN whose upper half alone would read as an infinity)
      if (sizeof(T) == 4 && p == 0) {
        if ((a & 0x7fffffffu) > 0x7f800000u) w[e] |= 0x00000040u;
        if ((c & 0x7fffffffu) > 0x7f800000u) w[e] |= 0x00400000u;
      }
    }
    if (!FOLD)
      out[p] = w;
    else if (p == part || p == 0)
      out[0] = w;
  }
}

// Where a lane's fragment comes from: its class (K: none), part and first sample.
struct Source {
  int k, part, n0;  // n0 within the group
};
template <bool FOLD>
__device__ __forceinline__ Source source_of(int kt, int step, int lane, int K) {
  const int row = 32 * kt + lane % 32;
  const int n0 = 32 * (step / 2) + 16 * (lane / 32) + 8 * (step % 2);
  if (FOLD) return {row < 3 * K ? row % K : K, row / K, n0};
  return {row < K ? row : K, 0, n0};
}

template <typename T, int P, bool FOLD>
__global__ __launch_bounds__(256) void ckpt_grad_operand_kernel(const T* __restrict__ dS,
                                                                int64_t lds, int64_t N, int K,
                                                                int ktiles, int64_t total,
                                                                u32x4* out) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= total) return;
  const int lane = (int)(at & 63), step = (int)(at >> 6) % kSteps;
  const int64_t bt = (at >> 6) / kSteps;
  const Source from = source_of<FOLD>((int)(bt % ktiles), step, lane, K);
  const int64_t n0 = bt / ktiles * kRows + from.n0;
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e)
    v[e] = (from.k < K && n0 + e < N) ? load_elem(dS, (n0 + e) * lds + from.k) : 0.0f;
  u32x4 w[P];
  cut<T, P, FOLD>(v, from.part, w);
#pragma unroll
  for (int p = 0; p < P; ++p) out[((bt * kSteps + step) * P + p) * 64 + lane] = w[p];
}

// ---- the gradient -----------------------------------------------------------------

__device__ __forceinline__ bf16x8 bytes_bf16(uint32_t a, uint32_t b) {
  u32x4 v;
  float f[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[e] = (float)(int8_t)(a >> (8 * e));
    f[4 + e] = (float)(int8_t)(b >> (8 * e));
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    v[e] = __builtin_amdgcn_perm(__float_as_uint(f[2 * e + 1]), __float_as_uint(f[2 * e]),
                                 0x07060302u);
  return __builtin_bit_cast(bf16x8, v);
}

constexpr int kFoldRow = 33;  // floats of a row in LDS

// W waves, each with DT tiles of 32 columns and KT tiles of 32 classes over a slice of the
// groups; they share the dS operand of R groups at a time through LDS. The next loads (the
// next group's kept values to registers, the next R operands on their way to the other
// half of LDS) are in flight while one group is multiplied; they are issued without a
// condition, past the end for the last group again, so that a wait covers only the
// older ones.
// T is u32x4 where dS has been laid out, else the type of dS's rows, which the workgroup
// then cuts by itself.
template <typename T, int P, int KT, int DT, int W, int R, bool FOLD, bool STREAM>
__global__ __launch_bounds__(64 * W, 2) void ckpt_class_grad_kernel(
    const u32x4* __restrict__ q, const float* __restrict__ scale, const T* __restrict__ ds,
    int64_t lds, int64_t N, float* __restrict__ out, int64_t D, int K, int ktiles, int64_t groups,
    int64_t per_slice, int64_t slice_stride, int accumulate) {
  constexpr bool ROWS = sizeof(T) < 16;
  constexpr int FRAGS = KT * kSteps * P * 64;  // 16-byte fragments of a group's operand
  // fragments that a thread brings: whole ones, or all parts of PER of them
  constexpr int THREADS = 64 * W, BRING = R * FRAGS / (ROWS ? P : 1);
  constexpr int PER = (BRING + THREADS - 1) / THREADS;
  extern __shared__ u32x4 op[];  // [2][R][FRAGS]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 31, half = lane >> 5;
  const int64_t d0 = ((int64_t)blockIdx.x * W + wave) * (32 * DT);
  const int kt0 = blockIdx.y * KT;
  const int64_t b0 = (int64_t)blockIdx.z * per_slice;
  const int own = (int)(b0 + per_slice < groups ? per_slice : groups - b0);
  int64_t dcol[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) {
    const int64_t d = d0 + 32 * t + col;
    dcol[t] = d < D ? d : D - 1;  // columns past D: any, never written
  }
  f32x16 acc[KT][DT];
#pragma unroll
  for (int k = 0; k < KT; ++k)
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[k][t][r] = 0.0f;

  struct Kept {
    u32x4 w[DT][2];
    float s[DT];
  };
  u32x4 stage[ROWS ? 1 : PER];
  T raw[ROWS ? PER : 1][8];
  auto group = [&](int i) { return b0 + (i < own ? i : own - 1); };
  auto fetch = [&](int64_t b, Kept& f) {
#pragma unroll
    for (int t = 0; t < DT; ++t) {
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const u32x4* at = q + (b * 4 + 2 * p + half) * D + dcol[t];
        f.w[t][p] = STREAM ? __builtin_nontemporal_load(at) : *at;
      }
      f.s[t] = scale[b * D + dcol[t]];
    }
  };
  auto fetch_op = [&](int i0) {  // the operands of groups i0 .. i0 + R - 1
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      int at = threadIdx.x + THREADS * i;
      if (BRING % THREADS != 0 && at >= BRING) at = BRING - 1;
      const int64_t b = group(i0 + at / (BRING / R));
      at %= BRING / R;
      if constexpr (ROWS) {
        const Source from = source_of<FOLD>(kt0 + at / (kSteps * 64), at / 64 % kSteps, at % 64, K);
        const T* col = ds + (from.k < K ? from.k : 0);
        const int64_t n0 = b * kRows + from.n0;
#pragma unroll
        for (int e = 0; e < 8; ++e) raw[i][e] = col[(n0 + e < N ? n0 + e : N - 1) * lds];
      } else {
        // class tiles past the last repeat it (their results are not written)
        const int k = at / (kSteps * P * 64);
        const int kt = kt0 + k < ktiles ? kt0 + k : ktiles - 1;
        stage[i] = ds[(b * ktiles + kt) * (kSteps * P * 64) + at % (kSteps * P * 64)];
      }
    }
  };
  auto put = [&](int buf, int i0) {  // what fetch_op(i0) brought
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = threadIdx.x + THREADS * i;
      if (BRING % THREADS != 0 && at >= BRING) continue;
      if constexpr (ROWS) {
        const int part_of = at % (BRING / R);
        const Source from =
            source_of<FOLD>(kt0 + part_of / (kSteps * 64), part_of / 64 % kSteps, part_of % 64, K);
        const int64_t n0 = group(i0 + at / (BRING / R)) * kRows + from.n0;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[e] = from.k < K && n0 + e < N ? load_elem(&raw[i][e], 0) : 0.0f;
        u32x4 w[P];
        cut<T, P, FOLD>(v, from.part, w);
#pragma unroll
        for (int p = 0; p < P; ++p) op[buf * (R * FRAGS) + (at / 64 * P + p) * 64 + at % 64] = w[p];
      } else {
        op[buf * (R * FRAGS) + at] = stage[i];
      }
    }
  };
  auto multiply = [&](const Kept& f, int buf) {
    bf16x8 qb[DT][kSteps];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
        qb[t][i] = bytes_bf16(f.w[t][i / 2][2 * (i % 2)], f.w[t][i / 2][2 * (i % 2) + 1]);
#pragma unroll
    for (int k = 0; k < KT; ++k) {
      f32x16 g[DT];
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) g[t][r] = 0.0f;
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const u32x4 a = op[buf * FRAGS + ((k * kSteps + i) * P + p) * 64 + lane];
#pragma unroll
          for (int t = 0; t < DT; ++t)
            g[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), qb[t][i],
                                                           g[t], 0, 0, 0);
        }
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[k][t][r] = fmaf(f.s[t], g[t][r], acc[k][t][r]);
    }
  };
  Kept f[2];
  fetch_op(0);
  fetch(group(0), f[0]);
  put(0, 0);
  __syncthreads();
  int i = 0, buf = 0;
  for (; i + 2 <= own; i += 2) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      // (the operand first: the kept values may stay in flight longer)
      if (r % R == 0) fetch_op(i + r + R);
      fetch(group(i + r + 1), f[1 - r]);
      __builtin_amdgcn_sched_barrier(0);  // (or the loads sink to their uses)
      multiply(f[r], buf * R + r % R);
      __builtin_amdgcn_sched_barrier(0);
      if (r % R == R - 1) {
        buf ^= 1;
        put(buf, i + r + 1);
        __syncthreads();
      }
    }
  }
  if (i < own) multiply(f[0], buf * R);

  float* dst = out + (int64_t)blockIdx.z * slice_stride;
  if constexpr (FOLD) {  // a class is the sum of three rows
    float* rows = reinterpret_cast<float*>(op) + wave * (KT * 32 * kFoldRow);
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      __syncthreads();  // (the operand, or the tile before, is read)
#pragma unroll
      for (int k = 0; k < KT; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          rows[(32 * k + 8 * (r / 4) + 4 * half + r % 4) * kFoldRow + col] = acc[k][t][r];
      __syncthreads();
      for (int i = lane; i < 32 * K; i += 64) {
        const int k = i / 32;
        const int64_t d = d0 + 32 * t + i % 32;
        const float* at = rows + k * kFoldRow + i % 32;
        const float v = at[0] + at[K * kFoldRow] + at[2 * K * kFoldRow];
        if (d < D) dst[k * D + d] = accumulate ? dst[k * D + d] + v : v;
      }
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < KT; ++k)
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const int64_t d = d0 + 32 * t + col;
      if (d >= D) continue;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int cls = 32 * (kt0 + k) + 8 * (r / 4) + 4 * half + r % 4;
        if (cls >= K) continue;
        float* at = dst + (int64_t)cls * D + d;
        *at = accumulate ? *at + acc[k][t][r] : acc[k][t][r];
      }
    }
}

// The slices' sums, added in order; eight loads in flight.
__global__ __launch_bounds__(256) void ckpt_grad_join_kernel(const float* __restrict__ part,
                                                             float* __restrict__ dC,
                                                             int64_t total, int slices,
                                                             int accumulate) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= total) return;
  float v = 0.0f;
  for (int s = 0; s < slices; s += 8) {
    float p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = part[(s + j < slices ? s + j : slices - 1) * total + i];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (s + j < slices) v += p[j];
  }
  dC[i] = accumulate ? dC[i] + v : v;
}

struct GradPlan {
  bool rows;                  // dS as it is, not laid out first
  bool fold;                  // fp32's parts as rows of their own
  int parts, ktiles;          // of a row's operand; tiles of 32 rows
  int kt, dt, waves;          // row tiles and column tiles of a wave; waves
  int kblocks;                // workgroups along K
  int64_t dblocks, per_slice;
  int slices;
  size_t operand, total;  // bytes of the dS operand, and with the partial sums
};

// Eight waves share an operand of three parts (65536 x 10240 x 26: 173 us, four waves
// 180); four are better where it is one (bf16, K = 10: 122 us, eight 143).
constexpr int waves_of(int parts) { return parts == 3 ? 8 : 4; }
// Column tiles of a wave: two read the operand half as often, where the sums of all
// class tiles leave the registers for it.
constexpr int dtiles_of(int kt) { return kt == 1 ? 2 : 1; }
// Groups between two barriers: two where the operand's halves fit LDS.
constexpr int round_of(int parts, int kt) { return parts * kt <= 6 ? 2 : 1; }

// Values up to which a workgroup cuts dS by itself (see grad_plan).
constexpr int64_t kRowsParts = int64_t(32) << 20, kRowsFold = int64_t(16) << 20;

GradPlan grad_plan(int64_t N, int64_t D, int64_t K, int dt) {
  GradPlan p;
  // Three rows for each class where that is one tile instead of three parts of one
  // (65536 x 10240 x 10: 127 us instead of 151) or four tiles instead of six parts (32768 x
  // 10240 x 40: 136 instead of 147); two tiles instead of three parts lose (K = 20: 170 instead
  // of 160), each side in the tiling that its count of parts and tiles gives it below: four waves
  // of one column tile against eight of two. (Two tiles in the tiling of the other side were
  // not measured.)
  p.fold = dt == 0 && (K <= 10 || (K > 32 && K <= 42));
  // A short call saves the launch that lays dS out; each workgroup then cuts all classes of its
  // groups by itself, which pays while there are few (K = 26, D = 10000, fp32: 1000 rows 15.0
  // us instead of 16.3, 4096 rows 27.1 either way, 65536 182 instead of 167; bf16: 300
  // rows 8.7 instead of 10.6; K = 6: 1000 rows 11.7 instead of 14.1, 2000 14.7 instead of
  // 14.2). Two class tiles are too many loads for it (2999 x 10000 x 60 bf16: 24 instead of 21).
  p.rows = K <= 32 && N * D <= (p.fold ? kRowsFold : kRowsParts);
  p.parts = dt == 0 && !p.fold ? 3 : 1;
  p.ktiles = (int)cdiv(p.fold ? 3 * K : K, 32);
  // the classes of one workgroup: up to 128, which read the kept values once
  p.kt = p.ktiles < 4 ? p.ktiles : 4;
  p.dt = dtiles_of(p.kt);
  p.waves = waves_of(p.parts);
  p.kblocks = (int)cdiv(p.ktiles, p.kt);
  p.dblocks = cdiv(D, p.waves * 32 * p.dt);
  // Two workgroups for each compute unit; a slice of at least four groups, since its
  // partial sums are written and read again.
  const int64_t groups = groups_of(N);
  int64_t slices = 2 * (int64_t)num_cus() / (p.dblocks * p.kblocks);
  if (slices > groups / 4) slices = groups / 4;
  // (two slices of several class tiles are not worth the partial sums: 700 x 10000 x 100 bf16 23.6
  // us, one 19.6, 520 x 16384 x 60 19.5 and 11.9; three parts, or one tile, are: 700 x 10000
  // x 26 fp32 17.1 and 21.0)
  if (slices < 1 || (slices == 2 && p.parts == 1 && p.kt > 1)) slices = 1;
  p.per_slice = cdiv(groups, slices);
  p.slices = (int)cdiv(groups, p.per_slice);
  p.operand = p.rows ? 0 : (size_t)groups * p.ktiles * kSteps * p.parts * 1024;
  p.total = p.operand + (p.slices > 1 ? (size_t)p.slices * K * D * 4 : 0);
  return p;
}

// Kept values past the caches, which do not stay there (bf16, K = 10: 671 MB 123 us instead of
// 138, 168 MB 39.0 instead of 42.6; 84 MB are the same either way).
constexpr int64_t kStreamKept = int64_t(96) << 20;

struct GradArgs {
  const void* dS;
  int64_t lds;
  const u32x4* q;
  const float* scale;
  const u32x4* operand;  // dS laid out
  float* out;
  int64_t N, D;
  int K;
  bool accumulate;
  hipStream_t stream;
};

template <typename T, int P, int KT, bool FOLD, bool STREAM>
hipError_t launch_grad_as(const GradPlan& p, const GradArgs& a, const T* ds) {
  constexpr int W = waves_of(P), R = round_of(P, KT);
  constexpr int op_lds = 2 * R * KT * kSteps * P * 1024, fold_lds = W * KT * 32 * kFoldRow * 4;
  constexpr int lds = FOLD && fold_lds > op_lds ? fold_lds : op_lds;
  const auto kernel = ckpt_class_grad_kernel<T, P, KT, dtiles_of(KT), W, R, FOLD, STREAM>;
  if (lds > 64 * 1024) {  // above the default limit: raised once per device and kernel
    static PerDeviceOnce once;
    const hipError_t e = once_per_device(once, [&] {
      return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    });
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)p.dblocks, (unsigned)p.kblocks, (unsigned)p.slices),
                     dim3(64 * W), lds, a.stream, a.q, a.scale, ds, a.lds, a.N, a.out, a.D, a.K,
                     p.ktiles, groups_of(a.N), p.per_slice, (int64_t)a.K * a.D,
                     (int)(a.accumulate && p.slices == 1));
  return hipGetLastError();
}

template <typename T, int P, int KT, bool FOLD>
hipError_t launch_grad_kernel(const GradPlan& p, const GradArgs& a) {
  if constexpr (KT == 1)
    if (p.rows) return launch_grad_as<T, P, KT, FOLD, false>(p, a, static_cast<const T*>(a.dS));
  // (where one workgroup reads each of them)
  if (groups_of(a.N) * kRows * a.D > kStreamKept && p.kblocks == 1)
    return launch_grad_as<u32x4, P, KT, FOLD, true>(p, a, a.operand);
  return launch_grad_as<u32x4, P, KT, FOLD, false>(p, a, a.operand);
}

template <typename T>
hipError_t launch_grad_typed(const void* dS, int64_t lds, const void* image, float* dC, int64_t N,
                             int64_t D, int64_t K, bool accumulate, const GradPlan& p,
                             void* workspace, hipStream_t stream) {
  u32x4* operand = static_cast<u32x4*>(workspace);
  float* part = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.operand);
  hipError_t e;
  if (!p.rows) {
    const int64_t total = groups_of(N) * p.ktiles * kSteps * 64;
    auto lay_out = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)cdiv(total, 256)), dim3(256), 0, stream,
                         static_cast<const T*>(dS), lds, N, (int)K, p.ktiles, total, operand);
    };
    if constexpr (sizeof(T) == 4)
      p.fold ? lay_out(ckpt_grad_operand_kernel<T, 1, true>)
             : lay_out(ckpt_grad_operand_kernel<T, 3, false>);
    else
      lay_out(ckpt_grad_operand_kernel<T, 1, false>);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const GradArgs a{dS, lds, static_cast<const u32x4*>(image),
                   reinterpret_cast<const float*>(static_cast<const char*>(image) +
                                                  scales_at(N, D)),
                   operand, p.slices > 1 ? part : dC, N, D, (int)K, accumulate, stream};
  if constexpr (sizeof(T) == 4) {
    if (p.fold)
      e = p.kt == 1 ? launch_grad_kernel<T, 1, 1, true>(p, a)
                    : launch_grad_kernel<T, 1, 4, true>(p, a);
    else
      e = p.kt == 1   ? launch_grad_kernel<T, 3, 1, false>(p, a)
          : p.kt == 2 ? launch_grad_kernel<T, 3, 2, false>(p, a)
          : p.kt == 3 ? launch_grad_kernel<T, 3, 3, false>(p, a)
                      : launch_grad_kernel<T, 3, 4, false>(p, a);
  } else {
    e = p.kt == 1   ? launch_grad_kernel<T, 1, 1, false>(p, a)
        : p.kt == 2 ? launch_grad_kernel<T, 1, 2, false>(p, a)
        : p.kt == 3 ? launch_grad_kernel<T, 1, 3, false>(p, a)
                    : launch_grad_kernel<T, 1, 4, false>(p, a);
  }
  if (e != hipSuccess || p.slices == 1) return e;
  hipLaunchKernelGGL(ckpt_grad_join_kernel, dim3((unsigned)cdiv(K * D, 256)), dim3(256), 0, stream,
                     part, dC, K * D, p.slices, (int)accumulate);
  return hipGetLastError();
}

}  // namespace

size_t ckpt_image_bytes(int64_t N, int64_t D) {
  return (size_t)scales_at(N, D) + (size_t)(groups_of(N) * D) * 4;
}

hipError_t launch_ckpt_store(const void* H, int64_t ldh, int64_t N, int64_t D, int dt,
                             void* image, hipStream_t stream) {
  u32x4* q = static_cast<u32x4*>(image);
  float* s = reinterpret_cast<float*>(static_cast<char*>(image) + scales_at(N, D));
  const dim3 grid((unsigned)cdiv(D, 256), (unsigned)groups_of(N)), block(256);
  auto go = [&](auto kernel, auto* rows) {
    hipLaunchKernelGGL(kernel, grid, block, 0, stream, rows, ldh, N, D, q, s);
  };
  auto typed = [&](auto* rows) {
    typedef std::remove_const_t<std::remove_pointer_t<decltype(rows)>> T;
    switch (columns_of(rows, ldh, N, D, dt)) {
      case kApart: return go(ckpt_store_kernel<T, kApart>, rows);
      case kApartOnce: return go(ckpt_store_kernel<T, kApartOnce>, rows);
      case kNear: return go(ckpt_store_kernel<T, kNear>, rows);
      case kNearOnce: return go(ckpt_store_kernel<T, kNearOnce>, rows);
    }
  };
  dt == 0 ? typed(static_cast<const float*>(H)) : typed(static_cast<const bf16raw*>(H));
  return hipGetLastError();
}

hipError_t launch_ckpt_load(const void* image, void* H, int64_t ldh, int64_t N, int64_t D, int dt,
                            hipStream_t stream) {
  const u32x4* q = static_cast<const u32x4*>(image);
  const float* s =
      reinterpret_cast<const float*>(static_cast<const char*>(image) + scales_at(N, D));
  const dim3 grid((unsigned)cdiv(D, 256), (unsigned)groups_of(N)), block(256);
  auto go = [&](auto kernel, auto* rows) {
    hipLaunchKernelGGL(kernel, grid, block, 0, stream, q, s, rows, ldh, N, D);
  };
  auto typed = [&](auto* rows) {
    typedef std::remove_pointer_t<decltype(rows)> T;
    switch (columns_of(rows, ldh, N, D, dt)) {
      case kApart:  // (narrow stores are ordinary ones)
      case kApartOnce: return go(ckpt_load_kernel<T, kApart>, rows);
      case kNear: return go(ckpt_load_kernel<T, kNear>, rows);
      case kNearOnce: return go(ckpt_load_kernel<T, kNearOnce>, rows);
    }
  };
  dt == 0 ? typed(static_cast<float*>(H)) : typed(static_cast<bf16raw*>(H));
  return hipGetLastError();
}

size_t ckpt_grad_ws_bytes(int64_t N, int64_t D, int64_t K, int dt) {
  return grad_plan(N, D, K, dt).total;
}

hipError_t launch_ckpt_class_grad(const void* dS, int64_t lds, const void* image, float* dC,
                                  int64_t N, int64_t D, int64_t K, int dt, bool accumulate,
                                  void* workspace, hipStream_t stream) {
  const GradPlan p = grad_plan(N, D, K, dt);
  return dt == 0 ? launch_grad_typed<float>(dS, lds, image, dC, N, D, K, accumulate, p, workspace,
                                            stream)
                 : launch_grad_typed<bf16raw>(dS, lds, image, dC, N, D, K, accumulate, p,
                                              workspace, stream);
}

}  // namespace ops
}  // namespace hd
