// Log probabilities of given classes, with the entropy and the best alternatives:
//   t_k = scale (s_k - m) - L,  m = max s,  L = log sum_k exp(scale (s_k - m)),
//   logp = t_y,  entropy = -sum_k exp(t_k) t_k,  the T largest t with their classes
// and the gradient of g logp + h entropy with respect to s:
//   scale ( g (1[k=y] - p_k) - h p_k (t_k + entropy) ),  p = exp(t).
//
// The scores are read once: each thread keeps a running maximum, the sum of
// exp and the sum of z exp(z), both rescaled when its maximum grows (all in fp32), so reading
// the scores is the bound. The two halves m and L are kept apart,
// because scale * m can be large against the differences that matter.
//
// What is masked, and -inf, contributes nothing whatever it holds. NaN or +inf among
// the rest make the row's floats NaN and its alternatives -1.
//
// Alternatives: a score and its class make one 64-bit key, ordered by score and then by
// lower class, so the choice is exact and does not depend on the order of the
// work. In a long row each wave keeps a sorted list of keys, one in each lane; a chunk
// whose largest score does not beat the list's T-th (almost every chunk) costs one
// comparison.
//
// * up to kShortK classes: LPR lanes hold a row in registers.
// * more: a wave walks a row, or a workgroup does, or a part of it, where there are fewer rows
//   than the chip has room for; the last workgroup to finish joins the parts in order.
// The gradient is a pass over the elements: statistics and entropy are its inputs, so it
// reads each score once and needs no reduction.
//
// Measured: 65536 x 26 fp32 top 3, 9.7 MB: kernel 6.8 us, launch and the selection of
// three among eight lanes. 1 x 131072 fp32 top 20: kernel 11 to 12 us, 64 parts of one step: a
// load, a sort, a ticket and the join of 64 lists, each waiting for the one before. 2048 x 100003
// bf16 top 8 with a mask of bytes, 615 MB: 127 to 136 us in a row of calls (138 to 150 under the
// profiler), 4.5 to 4.9 TB/s; the vector units, busy for 86% of the time, bound it: 16
// instructions an element, 9 where rows start at words and no mask is given. Gradient, 4096 x 65536
// bf16, 1.07 GB: 193 to 199 us in a row of calls (193 to 211 under the profiler), 5.4 to 5.6
// TB/s, against 5.6 to 6.4 for a copy with such loads and stores.
#include "hd_ops.hpp"

// A product that is rounded is meant to be (q = fl(c m) is taken off itself below); what is
// to be fused is written so.
#pragma clang fp contract(off)

namespace hd {
namespace ops {

namespace {

constexpr int kShortK = 1024;
constexpr int kLongThreads = 256;
constexpr int64_t kWaveBytes = 48 * 1024;  // of a row that one wave may take
// 16-byte chunks that a thread takes in a step: two of bf16, whose work for each byte
// is twice fp32's (4096 x 65536 top 4: 121 us with one, 116 with two; fp32 2048 x 100003 133
// with one, 151 with two), and where rows are split, which leaves a wave one step and
// its list one sort.
constexpr int chunks_of(int esize, bool split) { return esize == 4 && !split ? 1 : 2; }
// Past the caches (256 MiB that the dies share): loads and stores that do not stay there
// (bf16 scores, top 8: 410 MB 92.7 us instead of 93.8, but 134 MB 36.5 instead of 34.9). The
// gradient counts the scores and itself (537 MB each 193 us instead of 206, 134 MB each 49
// instead of 52).
constexpr int64_t kStreamBytes = int64_t(192) << 20;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kLowest = -3.402823466e38f;
constexpr float kUnder = -300.0f;  // 2^kUnder is 0: keeps 0 * -inf out of the sums

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Keys: larger is better. 0 stands for no class.
__device__ __forceinline__ uint64_t key_of(float s, uint32_t k) {
  uint32_t b = __float_as_uint(s + 0.0f);  // -0 and +0 are one score
  b ^= (b >> 31) ? 0xffffffffu : 0x80000000u;
  return (uint64_t)b << 32 | (uint32_t)~k;
}
__device__ __forceinline__ float order_score(uint32_t b) {
  return __uint_as_float(b ^ ((b >> 31) ? 0x80000000u : 0xffffffffu));
}
// The largest score below the one whose order is b (for comparisons, in which both zeros
// are one).
__device__ __forceinline__ float score_below(uint32_t b) {
  return order_score(b == 0x80000000u ? b - 2 : b - 1);
}
__device__ __forceinline__ float key_score(uint64_t key) {
  return order_score((uint32_t)(key >> 32));
}
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint64_t min64(uint64_t a, uint64_t b) { return a < b ? a : b; }

// The running statistics of a part of a row, in powers of two: z_k = c s_k - q with
// c = scale log2(e) and q = c m rounded to fp32, one fused multiply-add. m is the largest
// score, at least the lowest finite number (so that an -inf stays below it); sum is 0
// only where nothing was there. At the row's largest score z is what q was rounded by, up to
// half a unit in q's last place: 1/2 below kFar, but past it soon more than exp2 holds. There
// (`far`) z is c (s - m), whose difference is exact for neighbours, and q stands for 0 in it.
struct Stats {
  float m, q, sum, ez;  // ez: sum of z 2^z
};
constexpr float kFar = 16777216.0f;  // 2^24
__device__ __forceinline__ bool far_of(float q) { return !(fabsf(q) < kFar); }
__device__ __forceinline__ Stats stats_none(float c) {
  return Stats{kLowest, kLowest * c, 0.0f, 0.0f};
}
// How far, in powers of two, a's reference lies above that of m (q = fl(c m)): at most 0, or
// what q and a.q were rounded by. A reference is q, or where that is far c m itself.
__device__ __forceinline__ float stats_step(const Stats& a, float m, float q, float c) {
  float d = a.q - q;
  if (far_of(q) || far_of(a.q)) {
    d = (a.m - m) * c;
    if (!far_of(a.q)) d += fmaf(-a.m, c, a.q);
    if (!far_of(q)) d += fmaf(m, c, -q);
  }
  return fmaxf(d, kUnder);
}
__device__ __forceinline__ void stats_raise(Stats& a, float m, float c) {
  const float q = m * c, d = stats_step(a, m, q, c), f = exp2_fast(d);
  a.ez = f * fmaf(d, a.sum, a.ez);
  a.sum *= f;
  a.m = m;
  a.q = q;
}
__device__ __forceinline__ void stats_add_z(Stats& a, float z) {
  const float e = exp2_fast(z);
  a.sum += e;
  a.ez = fmaf(e, fmaxf(z, kUnder), a.ez);  // (NaN is in e)
}
template <int LEN>
__device__ __forceinline__ void stats_add(Stats& a, const float (&s)[LEN], float c) {
  if (far_of(a.q)) {
#pragma unroll
    for (int e = 0; e < LEN; ++e) stats_add_z(a, (s[e] - a.m) * c);
  } else {
#pragma unroll
    for (int e = 0; e < LEN; ++e) stats_add_z(a, fmaf(s[e], c, -a.q));
  }
}
// Over LANES neighbouring lanes; both lanes of a pair add the same two numbers.
template <int LANES, int OFF = 1>
__device__ __forceinline__ float max_across(float v) {
  if constexpr (OFF < LANES) return max_across<LANES, 2 * OFF>(fmaxf(v, lane_xor<OFF>(v)));
  return v;
}
template <int LANES, int OFF = 1>
__device__ __forceinline__ float sum_across(float v) {
  if constexpr (OFF < LANES) return sum_across<LANES, 2 * OFF>(v + lane_xor<OFF>(v));
  return v;
}
template <int LANES, int OFF = 1>
__device__ __forceinline__ uint32_t min_across(uint32_t v) {
  if constexpr (OFF < LANES) {
    const uint32_t w = lane_xor<OFF>(v);
    return min_across<LANES, 2 * OFF>(v < w ? v : w);
  }
  return v;
}

template <int LANES>
__device__ __forceinline__ Stats stats_across(Stats a, float c) {
  stats_raise(a, max_across<LANES>(a.m), c);
  a.sum = sum_across<LANES>(a.sum);
  a.ez = sum_across<LANES>(a.ez);
  return a;
}

struct Row {  // a finished row
  float m, logsum, entropy;
  bool none, bad;
};
__device__ __forceinline__ Row finish(Stats a, float c) {
  Row r;
  r.none = a.sum == 0.0f;
  r.bad = a.sum != a.sum;
  // the sum is of 2^(c s - q): log sum exp scale (s - m) has q - c m, what q was rounded
  // by, added
  const float log_z = logf(a.sum);
  r.logsum = r.none ? 0.0f : far_of(a.q) ? log_z : fmaf(fmaf(-a.m, c, a.q), kLn2, log_z);
  r.m = r.none ? -INFINITY : r.bad ? NAN : a.m;
  r.entropy = r.none ? 0.0f : log_z - (a.ez * kLn2) / a.sum;
  return r;
}
// log probability of a score in a finished row
__device__ __forceinline__ float logp_of(const Row& r, float s, float scale) {
  if (r.bad) return NAN;
  if (r.none || s == -INFINITY) return -INFINITY;
  return (s - r.m) * scale - r.logsum;
}

struct Out {
  float *logp, *entropy, *stats;
  int32_t* ids;
  float* top_logp;
  int top;
};

template <typename T>
__device__ __forceinline__ void write_row(const Row& r, const T* row, const uint8_t* mrow,
                                          const int32_t* y, int64_t n, int64_t K, float scale,
                                          const Out& o) {
  if (y) {
    const int64_t k = y[n];
    float lp = 0.0f;  // no class asked for
    if (k >= 0 && k < K) {
      const bool on = !mrow || mrow[k];
      lp = logp_of(r, on ? load_elem(row, k) : -INFINITY, scale);
    }
    o.logp[n] = lp;
  }
  o.entropy[n] = r.bad ? NAN : r.entropy;
  o.stats[2 * n] = r.m;
  o.stats[2 * n + 1] = r.bad ? NAN : r.logsum;
}
__device__ __forceinline__ void write_top(const Row& r, uint64_t key, int64_t n, int j,
                                          float scale, const Out& o) {
  const bool there = key != 0 && !r.bad;
  o.ids[n * o.top + j] = there ? (int32_t)~(uint32_t)key : -1;
  o.top_logp[n * o.top + j] =
      r.bad ? NAN : there ? logp_of(r, key_score(key), scale) : -INFINITY;
}

// ---- lists of the best keys --------------------------------------------------------

// Compare and exchange with lane ^ OFF within blocks of SIZE lanes, of which every other
// is sorted the other way round.
template <int SIZE, int OFF>
__device__ __forceinline__ uint64_t exchange(uint64_t v, int lane) {
  const uint64_t w = lane_xor<OFF>(v);
  const bool keep_max = ((lane & OFF) == 0) == (SIZE == 64 || (lane & SIZE) == 0);
  return keep_max ? max64(v, w) : min64(v, w);
}
template <int SIZE, int OFF>
__device__ __forceinline__ uint64_t merge(uint64_t v, int lane) {
  v = exchange<SIZE, OFF>(v, lane);
  if constexpr (OFF > 1) return merge<SIZE, OFF / 2>(v, lane);
  return v;
}
// Sorts one key per lane, largest first.
template <int SIZE = 2>
__device__ __forceinline__ uint64_t sort64(uint64_t v, int lane) {
  v = merge<SIZE, SIZE / 2>(v, lane);
  if constexpr (SIZE < 64) return sort64<2 * SIZE>(v, lane);
  return v;
}
// Lanes 0..31 hold a list, largest first, and lanes 32..63 another, smallest
// first: the 64 keys, largest first.
__device__ __forceinline__ uint64_t merge64(uint64_t v, int lane) { return merge<64, 32>(v, lane); }

// A wave's sorted list: lane j holds the (j+1)-th best key seen.
struct TopList {
  uint64_t key;
  float bar;  // a score has to beat this to enter the first `top`
};
__device__ __forceinline__ uint64_t lane_key(uint64_t v, int lane) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
  return (uint64_t)hi << 32 | lo;
}
// Inserts a key that is the same in all lanes.
__device__ __forceinline__ uint64_t list_insert(uint64_t list, uint64_t key, int lane) {
  const int at = __popcll(__ballot(list > key));
  const int lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)list, 0x138, 0xf, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(list >> 32), 0x138, 0xf, 0xf, false);
  const uint64_t up = (uint64_t)(uint32_t)hi << 32 | (uint32_t)lo;  // the lane below
  return lane < at ? list : lane == at ? key : up;
}

// ---- short rows ----------------------------------------------------------------

// LPR lanes to a row, VPL scores in each lane (class lane + LPR j).
template <typename T, int LPR, int VPL>
__global__ __launch_bounds__(256) void logprobs_short_kernel(LogprobsArgs a, Out o) {
  const int lane = threadIdx.x & (LPR - 1);
  const int64_t n = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
  const bool live = n < a.N;
  const int64_t nn = live ? n : a.N - 1;  // lanes past the end follow along and write nothing
  const T* row = static_cast<const T*>(a.scores) + nn * a.ld;
  const uint8_t* mrow = a.mask ? a.mask + nn * a.ldm : nullptr;
  const int K = (int)a.K;
  const float c = a.scale * kLog2e;
  float v[VPL];
  Stats st = stats_none(c);
#pragma unroll
  for (int j = 0; j < VPL; ++j) {
    const int k = lane + LPR * j;
    v[j] = k < K ? load_elem(row, k) : -INFINITY;
    if (mrow && k < K && !mrow[k]) v[j] = -INFINITY;
    st.m = fmaxf(st.m, v[j]);
  }
  st.m = max_across<LPR>(st.m);
  st.q = st.m * c;
  stats_add(st, v, c);
  st.sum = sum_across<LPR>(st.sum);
  st.ez = sum_across<LPR>(st.ez);
  const Row r = finish(st, c);
  if (live && lane == 0) write_row(r, row, mrow, a.y, n, a.K, a.scale, o);
  if (o.top == 0) return;
  if constexpr (LPR == 64) {
    // As in a long row: the T-th largest of the lanes' maxima is a bar, and what is not below
    // it enters a list.
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < VPL; ++j) m = fmaxf(m, v[j]);
    const uint64_t bar = lane_key(sort64(m > -INFINITY ? key_of(m, 0) : 0, lane), o.top - 1);
    const float low = bar ? score_below((uint32_t)(bar >> 32)) : -INFINITY;
    uint64_t list = 0;
#pragma unroll
    for (int j = 0; j < VPL; ++j)
      for (uint64_t pass = __ballot(v[j] > low); pass; pass &= pass - 1) {
        const int from = (int)__builtin_ctzll(pass);
        const float s =
            __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v[j]), from));
        list = list_insert(list, key_of(s, (uint32_t)(from + LPR * j)), lane);
      }
    if (live && lane < o.top) write_top(r, list, n, lane, a.scale, o);
  } else {
    // The best score, then the lowest class that has it, T times.
    for (int t = 0; t < o.top; ++t) {
      float m = -INFINITY;
#pragma unroll
      for (int j = 0; j < VPL; ++j) m = fmaxf(m, v[j]);
      m = max_across<LPR>(m);
      uint32_t k = ~0u;
#pragma unroll
      for (int j = VPL - 1; j >= 0; --j) k = v[j] == m ? (uint32_t)(lane + LPR * j) : k;
      k = min_across<LPR>(k);
#pragma unroll
      for (int j = 0; j < VPL; ++j)
        if (k == (uint32_t)(lane + LPR * j)) v[j] = -INFINITY;
      if (live && lane == 0) write_top(r, m > -INFINITY ? key_of(m, k) : 0, n, t, a.scale, o);
    }
  }
}

// ---- long rows -----------------------------------------------------------------

template <typename T>
struct Chunk {  // 16 bytes of scores
  static constexpr int kLen = 16 / (int)sizeof(T);
};

// A chunk on its way: its words, and the mask's.
template <typename T, bool MASK, bool STREAM>
struct Flight {
  static constexpr int LEN = Chunk<T>::kLen;
  u32x4 w;
  uint32_t m[MASK ? LEN / 4 : 1];
  __device__ __forceinline__ void load(const T* p, const uint8_t* mp) {
    typedef uint32_t m_a __attribute__((aligned(1)));
    if constexpr (STREAM)
      w = __builtin_nontemporal_load(reinterpret_cast<const u32x4_a2*>(p));
    else
      w = *reinterpret_cast<const u32x4_a2*>(p);
    if (MASK) {
#pragma unroll
      for (int i = 0; i < LEN / 4; ++i)
        m[i] = STREAM ? __builtin_nontemporal_load(reinterpret_cast<const m_a*>(mp) + i)
                      : reinterpret_cast<const m_a*>(mp)[i];
    }
  }
  __device__ __forceinline__ void scores(float* v) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int e = 0; e < LEN; ++e) {
        v[e] = __uint_as_float(w[e]);
        if (MASK && !(m[0] & (255u << (8 * e)))) v[e] = -INFINITY;
      }
    } else {
#pragma unroll
      for (int e = 0; e < LEN / 2; ++e) {
        uint32_t u = w[e];
        if (MASK) {
          // bit 7 of each byte: not 0; spread over the halves of a word by v_perm's sign
          // selectors (bytes 1 and 3 of either operand)
          const uint32_t f = ((m[e / 2] & 0x7f7f7f7fu) + 0x7f7f7f7fu) | m[e / 2];
          const uint32_t on =
              __builtin_amdgcn_perm(f, f << 8, e % 2 ? 0x0b0b0909u : 0x0a0a0808u);
          u = (u & on) | (0xff80ff80u & ~on);  // bf16 -inf
        }
        v[2 * e] = __uint_as_float(u << 16);
        v[2 * e + 1] = __uint_as_float(u & 0xffff0000u);
      }
    }
  }
};

// The value of the next lane (any in lane 63).
__device__ __forceinline__ uint32_t lane_next(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x130, 0xf, 0xf, true);
}

// A whole wave's chunks, neighbours in memory, whose row starts between two words (bf16 rows of
// odd length, masks of any): loads at the words before, which are as fast as aligned ones,
// then each lane moves its words up and takes what is missing from the next lane; lane 63
// loads its last values by themselves. `up` and `mup` are how many bytes before.
template <typename T, bool MASK, bool STREAM>
struct WaveFlight {
  Flight<T, MASK, STREAM> f;
  uint32_t last, mlast;  // lane 63's
  __device__ __forceinline__ void load(const T* p, const uint8_t* mp, uint32_t up, uint32_t mup,
                                       int lane) {
    constexpr int LEN = Chunk<T>::kLen;
    typedef uint32_t m_a __attribute__((aligned(1)));
    f.load(reinterpret_cast<const T*>(reinterpret_cast<const char*>(p) - up),
           MASK ? mp - mup : nullptr);
    if (up | mup) {
      if (lane == 63) {
        if (sizeof(T) == 2) last = reinterpret_cast<const bf16raw*>(p)[LEN - 1];
        if (MASK) mlast = *reinterpret_cast<const m_a*>(mp + LEN - 4);
      }
    }
  }
  __device__ __forceinline__ void settle(uint32_t up, uint32_t mup, int lane) {
    if (!(up | mup)) return;
    if constexpr (sizeof(T) == 2) {
      uint32_t next = lane_next(f.w[0]);
      next = lane == 63 ? last : next;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        f.w[e] = __builtin_amdgcn_alignbyte(e < 3 ? f.w[e + 1] : next, f.w[e], up);
    }
    if constexpr (MASK) {
      constexpr int M = Chunk<T>::kLen / 4;
      const uint32_t next = lane_next(f.m[0]);
#pragma unroll
      for (int e = 0; e < M; ++e)
        f.m[e] = __builtin_amdgcn_alignbyte(e < M - 1 ? f.m[e + 1] : next, f.m[e], mup);
      if (lane == 63) f.m[M - 1] = mlast;
    }
  }
};

// Joins the waves' statistics and lists of a workgroup; the result is whole in wave 0.
template <bool TOP, int WAVES>
__device__ __forceinline__ void join_waves(Stats& st, uint64_t& list, float c, int lane, int wave,
                                           Stats* sh_st, uint64_t* sh_key) {
  if (lane == 0) sh_st[wave] = st;
  if (TOP && lane < kMaxTop) sh_key[wave * kMaxTop + lane] = list;
  __syncthreads();
  if (wave != 0) return;
  st = stats_across<WAVES>(sh_st[lane % WAVES], c);
  if (TOP)
    for (int w = 1; w < WAVES; ++w) {
      const uint64_t other = sh_key[w * kMaxTop + (63 - lane) % kMaxTop];
      list = merge64(lane < kMaxTop ? list : other, lane);
    }
}

// Workspace of a split call: a counter for each row, then for each (row, part)
// kPartWords words: m, sum, ez, and the list's keys.
constexpr int kPartWords = 4 + 2 * kMaxTop;
constexpr int kMaxParts = 64;
struct Split {
  int parts;         // of a row
  int64_t part_len;  // scores in a part, a multiple of the step of a workgroup
  uint32_t *tickets, *words;
};

// Words that pass between workgroups: device-scope stores, performed before the writer
// takes its ticket, and device-scope loads after the last ticket. (Unlike exchanges, the
// loads of all parts are in flight together.)
__device__ __forceinline__ uint32_t get_word(const uint32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void put_word(uint32_t* p, uint32_t v) {
  __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ uint64_t get_key(const uint32_t* p) {
  return __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED,
                           __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void put_key(uint32_t* p, uint64_t v) {
  __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v, __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}

template <typename T, bool TOP, bool MASK, bool STREAM, int kChunks, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void logprobs_long_kernel(LogprobsArgs a, Out o,
                                                                   Split sp) {
  constexpr int LEN = Chunk<T>::kLen, kThreads = 64 * WAVES;
  constexpr int VALS = kChunks * LEN;
  __shared__ Stats sh_st[WAVES];
  __shared__ uint64_t sh_key[WAVES * kMaxTop];
  __shared__ uint32_t sh_last, sh_bar;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n = blockIdx.x / sp.parts;
  const int part = (int)(blockIdx.x % sp.parts);
  const T* row = static_cast<const T*>(a.scores) + n * a.ld;
  const uint8_t* mrow = MASK ? a.mask + n * a.ldm : nullptr;
  const float c = a.scale * kLog2e;
  const int64_t k_end = (part + 1) * sp.part_len < a.K ? (part + 1) * sp.part_len : a.K;

  if (TOP) {
    if (threadIdx.x == 0) sh_bar = 0;
    __syncthreads();
  }
  Stats st = stats_none(c);
  TopList list{0, -INFINITY};
  constexpr int ROUND = kThreads * LEN, STEP = kChunks * ROUND;
  auto class_of = [](int e) { return (uint32_t)(e / LEN * ROUND + e % LEN); };
  auto add = [&](float(&v)[VALS], uint32_t id0) {  // id0: the class of v[0]
    float m = v[0];
#pragma unroll
    for (int e = 1; e < VALS; ++e) m = fmaxf(m, v[e]);
    if (m > st.m) stats_raise(st, m, c);
    stats_add(st, v, c);
    if (!TOP || !__ballot(m > list.bar)) return;
    // What is below any wave's T-th score cannot be among the T best of the row. (Looked
    // up only here: in every step it would cost more than it saves.)
    const uint32_t shared_bar = *(volatile uint32_t*)&sh_bar;
    if (shared_bar) list.bar = fmaxf(list.bar, score_below(shared_bar));
    float bar = list.bar;
    if (!__ballot(m > bar)) return;
    if (bar == -INFINITY) {
      // Fewer than T so far. The lanes' largest go in together, sorted; then their T-th is a
      // bar for the rest (or a whole chunk would pass one by one).
      int at = 0;
#pragma unroll
      for (int e = VALS - 1; e >= 0; --e) at = v[e] == m ? e : at;
      const uint64_t fresh = sort64(m > -INFINITY ? key_of(m, id0 + class_of(at)) : 0, lane);
      const uint64_t held = lane_xor<32>(lane_xor<16>(lane_xor<8>(
          lane_xor<4>(lane_xor<2>(lane_xor<1>(list.key))))));  // the other way round
      list.key = merge64(lane < kMaxTop ? fresh : held, lane);
      const uint64_t s = lane_key(list.key, o.top - 1);
      if (s) bar = score_below((uint32_t)(s >> 32));
#pragma unroll
      for (int e = 0; e < VALS; ++e) v[e] = e == at ? -INFINITY : v[e];
    }
#pragma unroll
    for (int e = 0; e < VALS; ++e)
      for (uint64_t pass = __ballot(v[e] > bar); pass; pass &= pass - 1) {
        const int from = (int)__builtin_ctzll(pass);
        const float s =
            __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v[e]), from));
        const uint32_t id = (uint32_t)__builtin_amdgcn_readlane((int)id0, from) + class_of(e);
        list.key = list_insert(list.key, key_of(s, id), lane);
      }
    const uint64_t last = lane_key(list.key, o.top - 1);
    if (last) {
      list.bar = fmaxf(list.bar, key_score(last));
      if (lane == 0) atomicMax(&sh_bar, (uint32_t)(last >> 32));
    }
  };
  // Whole steps, the next one's loads in flight while one is worked on (past the end the
  // last one's again, so that they need no condition), then the step that ends inside. Steps
  // are counted from the row's start wherever it lies, so that a result does not depend
  // on alignment. Classes come in ascending order, so that of equal scores the
  // one already listed is the lower class.
  const int64_t k_begin = part * sp.part_len, whole = (k_end - k_begin) / STEP;
  const int64_t steps = cdiv(k_end - k_begin, STEP);
  // (a row's first word may begin before it where a row is before it)
  const bool inside = n > 0 || part > 0;
  const uint32_t up = sizeof(T) == 2 && inside ? (uint32_t)((uintptr_t)(row + k_begin) & 2) : 0;
  const uint32_t mup = MASK && (part > 0 || (n > 0 && a.ldm > 0))
                           ? (uint32_t)((uintptr_t)(mrow + k_begin) & 3)
                           : 0;
  WaveFlight<T, MASK, STREAM> flight[kChunks];
  auto place = [&](int64_t i, int u) {
    return k_begin + i * STEP + u * ROUND + (int64_t)threadIdx.x * LEN;
  };
  auto fetch = [&](int64_t i) {
#pragma unroll
    for (int u = 0; u < kChunks; ++u) {
      const int64_t k = place(i < whole ? i : whole - 1, u);
      flight[u].load(row + k, MASK ? mrow + k : nullptr, up, mup, lane);
    }
  };
  if (whole > 0) fetch(0);
  for (int64_t i = 0; i < steps; ++i) {
    float v[VALS];
    if (i < whole) {
#pragma unroll
      for (int u = 0; u < kChunks; ++u) {
        flight[u].settle(up, mup, lane);
        flight[u].f.scores(v + u * LEN);
      }
      fetch(i + 1);
      __builtin_amdgcn_sched_barrier(0);  // (or the loads sink below the work)
    } else {
#pragma unroll
      for (int u = 0; u < kChunks; ++u) {
        const int64_t k = place(i, u);
        if (k + LEN <= k_end) {
          flight[u].f.load(row + k, MASK ? mrow + k : nullptr);
          flight[u].f.scores(v + u * LEN);
        } else {
#pragma unroll
          for (int e = 0; e < LEN; ++e) {
            const bool in = k + e < k_end && (!MASK || mrow[k + e]);
            v[u * LEN + e] = in ? load_elem(row, k + e) : -INFINITY;
          }
        }
      }
    }
    add(v, (uint32_t)place(i, 0));
  }
  st = stats_across<64>(st, c);
  join_waves<TOP, WAVES>(st, list.key, c, lane, wave, sh_st, sh_key);

  if (sp.parts > 1) {
    uint32_t* mine = sp.words + ((int64_t)n * sp.parts + part) * kPartWords;
    if (wave == 0) {
      if (lane == 0) {
        put_word(mine, __float_as_uint(st.m));
        put_word(mine + 1, __float_as_uint(st.sum));
        put_word(mine + 2, __float_as_uint(st.ez));
      }
      if (TOP && lane < o.top) put_key(mine + 4 + 2 * lane, list.key);
      wait_own_memory_ops();
      if (lane == 0) sh_last = take_ticket(sp.tickets + n) == (uint32_t)sp.parts - 1;
    }
    __syncthreads();
    if (!sh_last) return;
    if (threadIdx.x == 0) reset_counter(sp.tickets + n);
    uint32_t* words = sp.words + (int64_t)n * sp.parts * kPartWords;
    if (wave == 0) {
      // lane p holds part p
      uint32_t* w = words + (int64_t)lane * kPartWords;
      uint64_t keys[kMaxTop] = {}, first = 0;
      const int each = TOP ? 64 / sp.parts : 0;  // keys of a part that begin the list
      st = stats_none(c);
      if (lane < sp.parts) {
        st.m = __uint_as_float(get_word(w));
        st.q = st.m * c;
        st.sum = __uint_as_float(get_word(w + 1));
        st.ez = __uint_as_float(get_word(w + 2));
        if (TOP) {
#pragma unroll
          for (int t = 0; t < kMaxTop; ++t)
            if (t >= each && t < o.top) keys[t] = get_key(w + 4 + 2 * t);
        }
      }
      if (TOP && lane < each * sp.parts && lane / sp.parts < o.top)
        first = get_key(words + (int64_t)(lane % sp.parts) * kPartWords + 4 +
                        2 * (lane / sp.parts));
      st = stats_across<64>(st, c);
      if (TOP) {
        // The parts' best, up to 64 together, sorted, begin the list; its T-th is a bar for the
        // rest. (With one of each part ten parts' 320 keys would pass one by one: 1 x 20000
        // top 32, 31 us.)
        list.key = sort64(first, lane);
        const uint64_t bar = lane_key(list.key, o.top - 1);
#pragma unroll
        for (int t = 1; t < kMaxTop; ++t) {
          for (uint64_t pass = __ballot(keys[t] > bar); pass; pass &= pass - 1)
            list.key = list_insert(list.key, lane_key(keys[t], (int)__builtin_ctzll(pass)), lane);
        }
      }
    }
    // all is read: left zeroed (plain stores, which the end of the launch makes visible)
    __syncthreads();
    for (int64_t i = threadIdx.x; i < (int64_t)sp.parts * kPartWords; i += kThreads)
      words[i] = 0;
  }
  if (wave != 0) return;
  const Row r = finish(st, c);
  if (lane == 0) write_row(r, row, mrow, a.y, n, a.K, a.scale, o);
  if (TOP && lane < o.top) write_top(r, list.key, n, lane, a.scale, o);
}

// Parts of a row: enough workgroups for every compute unit to hold two.
Split split_of(int64_t N, int64_t K, int esize) {
  Split s{1, 0, nullptr, nullptr};
  const int64_t step = (int64_t)kLongThreads * chunks_of(esize, true) * (16 / esize);
  const int64_t steps = cdiv(K, step);
  int64_t parts = cdiv(2 * (int64_t)num_cus(), N);
  if (parts > kMaxParts) parts = kMaxParts;
  if (parts > steps) parts = steps;
  const int64_t per = cdiv(steps, parts);
  s.parts = (int)cdiv(steps, per);
  s.part_len = per * step;
  return s;
}
constexpr size_t kAlign = 256;
size_t tickets_bytes(int64_t N) { return ((size_t)N * 4 + kAlign - 1) / kAlign * kAlign; }

template <typename T, int LPR, int VPL>
hipError_t launch_short(const LogprobsArgs& a, const Out& o, hipStream_t stream) {
  hipLaunchKernelGGL((logprobs_short_kernel<T, LPR, VPL>),
                     dim3((unsigned)cdiv(a.N, 256 / LPR)), dim3(256), 0, stream, a, o);
  return hipGetLastError();
}

template <typename T, bool STREAM, int C, int WAVES>
hipError_t launch_long(const LogprobsArgs& a, const Out& o, Split s, hipStream_t stream) {
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.N * s.parts)), dim3(64 * WAVES), 0, stream, a, o,
                       s);
    return hipGetLastError();
  };
  if (o.top)
    return a.mask ? go(logprobs_long_kernel<T, true, true, STREAM, C, WAVES>)
                  : go(logprobs_long_kernel<T, true, false, STREAM, C, WAVES>);
  return a.mask ? go(logprobs_long_kernel<T, false, true, STREAM, C, WAVES>)
                : go(logprobs_long_kernel<T, false, false, STREAM, C, WAVES>);
}

template <typename T>
hipError_t launch_typed(const LogprobsArgs& a, const Out& o, Split s, hipStream_t stream) {
  // Where few rows ask for many alternatives a wave takes a row: the T rounds of the narrower
  // forms are steps that wait for each other (1000 x 100, kernel: top 32 7.4 us instead of
  // 12.6, top 8 4.9 instead of 5.7, top 3 4.4 instead of 4.1; 8000 x 100 top 32 17.6 instead of 14.8).
  if (o.top >= 8 && a.K <= 64 * 4 && a.N <= 8 * (int64_t)num_cus())
    return launch_short<T, 64, 4>(a, o, stream);
  if (a.K <= 8 * 4) return launch_short<T, 8, 4>(a, o, stream);
  if (a.K <= 16 * 8) return launch_short<T, 16, 8>(a, o, stream);
  if (a.K <= 16 * 16) return launch_short<T, 16, 16>(a, o, stream);
  if (a.K <= kShortK) return launch_short<T, 64, 16>(a, o, stream);
  const bool stream_by = a.N * a.K * (int64_t)sizeof(T) > kStreamBytes;
  constexpr int C1 = chunks_of(sizeof(T), false), C2 = chunks_of(sizeof(T), true);
  if (s.parts > 1) return launch_long<T, false, C2, 4>(a, o, s, stream);
  // A wave takes a row where there are enough: four waves start, join and sort their lists
  // for a few steps each (30000 x 3000 fp32 top 5: 112 us, four 192; bf16 70 and 157; top 32 185 and
  // 335; but 1100 x 3000 fp32, kernel: 15.3 and 12.2). In long rows four waves
  // of a row are better (6000 x 16000 fp32 top 5: 115 and 107).
  if (a.K * (int64_t)sizeof(T) <= kWaveBytes && a.N >= 7 * (int64_t)num_cus())
    return stream_by ? launch_long<T, true, C1, 1>(a, o, s, stream)
                     : launch_long<T, false, C1, 1>(a, o, s, stream);
  return stream_by ? launch_long<T, true, C1, 4>(a, o, s, stream)
                   : launch_long<T, false, C1, 4>(a, o, s, stream);
}

// ---- gradient --------------------------------------------------------------------

struct GradRow {
  float m, logsum, entropy, g, h;
  int32_t y;
};
__device__ __forceinline__ GradRow grad_row(const LogprobsArgs& a, const float* stats,
                                            const float* entropy, const float* g_logp,
                                            const float* g_entropy, int64_t n) {
  GradRow r;
  r.m = stats[2 * n];
  r.logsum = stats[2 * n + 1];
  r.entropy = entropy[n];
  r.y = a.y ? a.y[n] : -1;
  r.g = g_logp && r.y >= 0 && r.y < a.K ? g_logp[n] : 0.0f;
  r.h = g_entropy ? g_entropy[n] : 0.0f;
  if (r.m == -INFINITY) r.m = 0.0f;  // an empty row: every p below is 0
  return r;
}
__device__ __forceinline__ float grad_of(const GradRow& r, float s, int32_t k, float scale) {
  float t = (s - r.m) * scale - r.logsum;
  if (t < -1000.0f) t = -1000.0f;  // p is 0 either way, and 0 * t too; NaN stays
  const float p = exp2_fast(t * kLog2e);
  float d = -p * (r.g + r.h * (t + r.entropy));
  if (k == r.y && s > -INFINITY) d += r.g;
  return d * scale;
}

// A thread takes LEN classes of one row. ROWS: a workgroup works within a row (blockIdx.y),
// else a thread finds its row.
template <typename T, bool MASK, bool ROWS, bool STREAM>
__global__ __launch_bounds__(256) void logprobs_grad_kernel(
    LogprobsArgs a, const float* __restrict__ stats, const float* __restrict__ entropy,
    const float* __restrict__ g_logp, const float* __restrict__ g_entropy, T* out, int64_t ldd,
    uint32_t chunks) {
  constexpr int LEN = Chunk<T>::kLen;
  int64_t n;
  uint32_t ch;
  if (ROWS) {
    n = blockIdx.x / cdiv(chunks, 256);
    ch = (uint32_t)(blockIdx.x % (uint32_t)cdiv(chunks, 256)) * 256 + threadIdx.x;
  } else {
    const uint64_t at = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    n = (int64_t)(at / chunks);
    ch = (uint32_t)(at % chunks);
  }
  if (n >= a.N || ch >= chunks) return;
  const GradRow r = grad_row(a, stats, entropy, g_logp, g_entropy, n);
  const int64_t k = (int64_t)ch * LEN;
  const T* row = static_cast<const T*>(a.scores) + n * a.ld + k;
  const uint8_t* mrow = MASK ? a.mask + n * a.ldm + k : nullptr;
  T* dst = out + n * ldd + k;
  if (k + LEN <= a.K) {
    Flight<T, MASK, STREAM> f;
    f.load(row, mrow);
    float v[LEN];
    f.scores(v);
    u32x4 d;
#pragma unroll
    for (int e = 0; e < LEN; ++e) v[e] = grad_of(r, v[e], (int32_t)(k + e), a.scale);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 4)
        d[e] = __float_as_uint(v[e]);
      else
        d[e] = (uint32_t)to_bf16(v[2 * e]) | (uint32_t)to_bf16(v[2 * e + 1]) << 16;
    }
    if constexpr (STREAM)
      __builtin_nontemporal_store(d, reinterpret_cast<u32x4_a2*>(dst));
    else
      *reinterpret_cast<u32x4_a2*>(dst) = d;
  } else {
    for (int e = 0; k + e < a.K; ++e) {
      const float s = !MASK || mrow[e] ? load_elem(row, e) : -INFINITY;
      store_elem(dst, e, grad_of(r, s, (int32_t)(k + e), a.scale));
    }
  }
}

template <typename T>
hipError_t launch_grad(const LogprobsArgs& a, const float* stats, const float* entropy,
                       const float* g_logp, const float* g_entropy, void* out, int64_t ldd,
                       hipStream_t stream) {
  const uint32_t chunks = (uint32_t)cdiv(a.K, Chunk<T>::kLen);
  T* d = static_cast<T*>(out);
  // a row of 256 chunks fills a workgroup
  const bool rows = chunks >= 256;
  const int64_t blocks = rows ? a.N * cdiv(chunks, 256) : cdiv(a.N * chunks, 256);
  const dim3 grid((unsigned)blocks), block(256);
  const bool stream_by = 2 * a.N * a.K * (int64_t)sizeof(T) > kStreamBytes;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, stats, entropy, g_logp, g_entropy, d,
                       ldd, chunks);
  };
  if (rows && stream_by) {
    if (a.mask) go(logprobs_grad_kernel<T, true, true, true>);
    else go(logprobs_grad_kernel<T, false, true, true>);
  } else if (rows) {
    if (a.mask) go(logprobs_grad_kernel<T, true, true, false>);
    else go(logprobs_grad_kernel<T, false, true, false>);
  } else {
    if (a.mask) go(logprobs_grad_kernel<T, true, false, false>);
    else go(logprobs_grad_kernel<T, false, false, false>);
  }
  return hipGetLastError();
}

constexpr int64_t kMaxRows = int64_t(1) << 21;  // of a launch

LogprobsArgs rows_from(const LogprobsArgs& a, int64_t n0, int64_t most) {
  LogprobsArgs r = a;
  r.scores = static_cast<const char*>(a.scores) + n0 * a.ld * (a.dt == 0 ? 4 : 2);
  if (a.mask) r.mask = a.mask + n0 * a.ldm;
  if (a.y) r.y = a.y + n0;
  r.N = a.N - n0 < most ? a.N - n0 : most;
  return r;
}

}  // namespace

size_t logprobs_ws_bytes(int64_t N, int64_t K, int dt) {
  if (K <= kShortK) return 0;
  const Split s = split_of(N, K, dt == 0 ? 4 : 2);
  if (s.parts == 1) return 0;
  return tickets_bytes(N) + (size_t)N * s.parts * kPartWords * 4;
}

hipError_t launch_logprobs(const LogprobsArgs& all, float* logp, float* entropy, float* stats,
                           int32_t* ids, float* top_logp, int top, void* workspace,
                           hipStream_t stream) {
  Split s = split_of(all.N, all.K, all.dt == 0 ? 4 : 2);  // (one part where N > kMaxRows)
  s.tickets = static_cast<uint32_t*>(workspace);
  s.words = reinterpret_cast<uint32_t*>(static_cast<char*>(workspace) + tickets_bytes(all.N));
  // a launch holds at most 2^32 threads
  for (int64_t n0 = 0; n0 < all.N; n0 += kMaxRows) {
    const LogprobsArgs a = rows_from(all, n0, kMaxRows);
    const Out o{logp ? logp + n0 : nullptr, entropy + n0, stats + 2 * n0,
                ids ? ids + n0 * top : nullptr, top_logp ? top_logp + n0 * top : nullptr, top};
    const hipError_t e = a.dt == 0 ? launch_typed<float>(a, o, s, stream)
                                   : launch_typed<bf16raw>(a, o, s, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_logprobs_grad(const LogprobsArgs& all, const float* stats,
                                const float* entropy, const float* g_logp,
                                const float* g_entropy, void* dscores, int64_t ldd,
                                hipStream_t stream) {
  // (a row takes up to 2^20 workgroups)
  const int64_t per = cdiv(all.K, 256 * 4), step = per > 4 ? (kMaxRows * 4) / per : kMaxRows;
  for (int64_t n0 = 0; n0 < all.N; n0 += step) {
    const LogprobsArgs a = rows_from(all, n0, step);
    const float *st = stats + 2 * n0, *en = entropy + n0, *gl = g_logp ? g_logp + n0 : nullptr,
                *ge = g_entropy ? g_entropy + n0 : nullptr;
    const hipError_t e =
        a.dt == 0 ? launch_grad<float>(a, st, en, gl, ge, static_cast<float*>(dscores) + n0 * ldd,
                                       ldd, stream)
                  : launch_grad<bf16raw>(a, st, en, gl, ge,
                                         static_cast<bf16raw*>(dscores) + n0 * ldd, ldd, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace ops
}  // namespace hd
