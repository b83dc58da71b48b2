// Sampling: one token per row of logits, from the min-p safe set, the top_k largest of it and of these the fewest that hold top_p
// of their mass, at a temperature, by a given random number.
//
// Every one of the three filters keeps the front of the row in falling order (equal logits by index), so what is kept is one
// cut: the logits above a value `v` and, of those equal to it, the ones up to an index.  Nothing is sorted but the logits around the
// cut, 2,048 at most:
//
//   1  the row streams past once: its maximum, the sum of e^{(z - m) / T} without the maximum's own terms (so that ln of the whole
//      sum keeps its digits where one token has all the mass), a sum for each piece of the row, and the maximum of each 32-byte
//      granule, which stays in shared memory.  What follows reads only the granules that can matter, from L2
//   2  for each of top_k and top_p: a histogram of the logits' distances from the maximum (whole numbers: the order of the
//      additions does not matter) brackets the cut, the logits in the bracket go to a list in shared memory that is sorted, and
//      the cut is where the running sum, in double, passes its aim.  A bracket too full for the list is cut again by the logits'
//      bits, down to a single value if need be
//   3  sums in double of what is kept, in the order of the indices, piece by piece; the piece in which the running sum passes
//      u times the whole is walked to the token
//
// Which token falls on which side of a border is decided in double.  Where a sum over the whole row is the border, float32's
// is tried first: it is good to error(), and mostly nothing lies so near the border that this matters.  With few rows the blocks
// of a cluster share a row and exchange sums through shared memory.
//
// Bound by instruction issue (three cycles of five) and by the waits of a row's phases, not by HBM; at 64 registers a thread, which two
// blocks an SM want, some 870 bytes a thread are spilled.  1,024 rows of 151,936 bfloat16 (311 MB, 47 us at 6.6 TB/s)
// take 122 us for the largest logit, 173 to 182 with nothing cut, 334 to 339 with a min-p set of 80 % of the row, 307 with top_k 50 and 518 to 540 with
// top_p 0.95, whose rows are read four times, once only a quarter of them.  Of a top_p row's some 200 thousand cycles, two
// rows an SM, the first sweep has 50, the quarter's histogram and its window 33, the sum behind the window with its list 80, the sort
// 20.  One row of that length takes 19 to 50 us by eight blocks.
#include <cmath>
#include <type_traits>

#include "dvp_common.cuh"

namespace dvp {
namespace sample {

constexpr int kThreads = 512, kWarps = kThreads / 32;  // two blocks an SM (1,024 rows, top_p 0.95: three of 256 threads were 1,093 us, two of 512 891)
constexpr int kBins = 2048, kList = 2048;
constexpr int kTable = 64;
constexpr int kParts = 64;          // sums that a warp keeps of its part of the row, of one piece or several each
constexpr int kMostBounds = 32768;  // granules whose maximum is held: 64 KB
constexpr float kLowest = -3.402823466e38f;
constexpr double kRound = 5.9604644775390625e-08;  // 2^-24, half a step of float32
constexpr int kNoIndex = 0x7fffffff;
constexpr long long kMostRows = 0x0fffffffLL, kMostLogits = 0x7fff0000LL;

struct Params {
  const void *logits;
  const float *uniform, *temperature_rows, *top_p_rows, *rho_rows;
  const int *top_k_rows;
  double temperature, top_p, rho;
  long long top_k;
  void *ids;
  float *logp, *logp_mp;
  int *count;
  long long T, V, ld;
  int id_is_i32, log_blocks;
  int bounds;  // granules of a block's part whose maxima are held, 0: too many
  unsigned int *bounds_status;  // the bounds-checking build's status word; unused otherwise
};

// What a block tells the others of its row.
struct Slot {
  double a;
  float m;
  int i;
};

template <typename T>
struct Shared {
  static constexpr int kPiece = 32 * 32 / sizeof(T);  // logits of 32 granules
  uint64_t list[kList];
  uint32_t hist[kBins];
  union {
    struct {
      float value[kWarps][kPiece];  // a warp's logits that matter, side by side
      uint16_t place[kWarps][kPiece];
    } compact;
    uint64_t sorted[kList];
  };
  double part[kWarps][kParts];  // of the last sum over the row; of the first sweep float32 pairs: a maximum, the sum against it
  double tail[kWarps][kParts];  // of the same parts what lies behind the cut
  double table[kTable];  // 2^(i / kTable)
  double chunk[kWarps];  // the warps' parts of a sum over the row
  double group[32];      // sums of 32 neighbouring logits
  double warp_a[kWarps], warp_b[kWarps];
  float warp_m[kWarps];
  uint32_t warp_n[kWarps];
  Slot slot[2];
  uint32_t list_n, counter[3];
  uint32_t pick_lo, pick_hi, pick_last;  // of the histogram's bins; the last that holds anything, then what pick_lo to pick_hi hold
};

// A logit's place in the order as an unsigned number; the zeros are one.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t b = __float_as_uint(z + 0.f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}

__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Inclusive sums over the lanes.
template <typename N>
__device__ __forceinline__ N warp_scan(N v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const N u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  return v;
}

struct Words {
  uint32_t w[8];
};
// A granule at the row's ends: what lies outside the row is -inf.
template <typename T>
__device__ __noinline__ Words load_end(const T *z, int at, int V) {
  Words r;
  const uint16_t *h = reinterpret_cast<const uint16_t *>(z);
  const uint32_t none = std::is_same<T, __half>::value ? 0xfc00u : 0xff80u;
#pragma unroll 1
  for (int i = 0; i < 8; ++i) {
    if constexpr (sizeof(T) == 4) {
      r.w[i] = at + i >= 0 && at + i < V ? __float_as_uint(z[at + i]) : 0xff800000u;
    } else {
      const int a = at + 2 * i;
      r.w[i] = (a >= 0 && a < V ? h[a] : none) | (a + 1 >= 0 && a + 1 < V ? h[a + 1] : none) << 16;
    }
  }
  return r;
}

// Two float32 in 64 bits, which one instruction adds or multiplies.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
  return v;
}
__device__ __forceinline__ void apart(uint64_t v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t v;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t v;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t v;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
  return v;
}

// Two neighbouring logits of a granule's eight words.
template <typename T>
__device__ __forceinline__ void two_of(const uint32_t (&w)[8], int i, float &lo, float &hi) {
  if constexpr (sizeof(T) == 4) {
    lo = __uint_as_float(w[2 * i]), hi = __uint_as_float(w[2 * i + 1]);
  } else if constexpr (std::is_same<T, __half>::value) {
    const float2 f = __half22float2(reinterpret_cast<const __half2 &>(w[i]));
    lo = f.x, hi = f.y;
  } else {
    lo = __uint_as_float(w[i] << 16), hi = __uint_as_float(w[i] & 0xffff0000u);
  }
}

template <typename T>
struct Row {
  static constexpr int kPer = 32 / sizeof(T);  // logits of a granule
  using Shared = sample::Shared<T>;
  bool bounded;  // the granules' maxima are held
  const T *z;
  int V, off;                    // off: logits of the first granule that lie in front of the row
  int seg0, segs, all_segs;      // the block's pieces of 32 granules, the row's
  int first, mine;               // of the block's pieces, the warp's
  int log_q;                     // pieces of a part: 2^log_q
  int blocks, rank, turn;
  int warp, lane;
  double inv_t;
  float c, c_rest;  // log2(e) / temperature, and what float32 leaves of it
  float m;  // the row's maximum
  // what is kept so far
  float cut_v;
  int cut_i;
#ifdef DVP_DEBUG_BOUNDS
  bool replaced = false;  // the first sweep's sums: a pass has put its own in their place
#endif
  __device__ __forceinline__ void replace() {
#ifdef DVP_DEBUG_BOUNDS
    replaced = true;
#endif
  }

  // The block's shared memory, by its own name wherever it is used: through a pointer that is handed on, every access would be one of
  // the general kind.
  __device__ __forceinline__ static Shared *sh() {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    return reinterpret_cast<Shared *>(smem_raw);
  }
  // The granules' maxima: bfloat16, rounded up.
  __device__ __forceinline__ static uint16_t *bounds() { return reinterpret_cast<uint16_t *>(sh() + 1); }

  __device__ __forceinline__ void meet() const {
    if (blocks > 1) {
      __syncwarp();
      asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
      asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
      __syncthreads();
    }
  }
  __device__ __forceinline__ const Shared *of(int r) const {
    return static_cast<const Shared *>(__cluster_map_shared_rank(sh(), (unsigned)r));
  }
  // Every block's value to all of them.  Two slots in turn: whoever writes one again has met the others since they read it.
  __device__ __forceinline__ void tell(double a, float m_, int i) {
    turn ^= 1;
    if (threadIdx.x == 0) sh()->slot[turn] = Slot{a, m_, i};
    meet();
  }
  __device__ __forceinline__ Slot told(int r) const { return r == rank ? sh()->slot[turn] : of(r)->slot[turn]; }

  __device__ __forceinline__ int first_of(int seg) const { return ((seg0 + seg) * 32 + lane) * kPer - off; }
  // A lane's granule of a piece; what lies outside the row is -inf.
  __device__ __forceinline__ void load(int seg, uint32_t (&w)[8]) const {
    const int at = first_of(seg);
    if (at >= 0 && at + kPer <= V) {
      ld_stream32(z + at, w);
    } else {
      const Words r = load_end(z, at, V);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = r.w[i];
    }
  }

  // e^{(x - m) / T} to some 2^-50.  With y = (x - m) / T and k the whole number next to 64 y / ln 2, r = y - k ln 2 / 64 is at most
  // ln 2 / 128, where six terms of the series leave 4e-17; e^y = 2^(k / 64) e^r, the fraction of the power from the table: eleven
  // operations in double.
  __device__ __forceinline__ double weight(float x) const { return power(((double)x - (double)m) * inv_t); }
  __device__ __forceinline__ double power(double y) const {
    const double big = 6755399441055744.0;  // 1.5 2^52: adding it leaves the whole number in the low bits
    const double shifted = fma(y, 92.33248261689366, big);
    const int k = __double2loint(shifted);
    const double r = fma(shifted - big, -0.010830424696249145, y);
    double e = fma(r, 1.0 / 120.0, 1.0 / 24.0);
    e = fma(e, r, 1.0 / 6.0);
    e = fma(e, r, 0.5);
    e = fma(e, r, 1.0);
    const double q = sh()->table[k & (kTable - 1)];
    e = fma(e * r, q, q);
    const double w = __hiloint2double(__double2hiint(e) + (k >> 6) * (1 << 20), __double2loint(e));
    return y > -700.0 ? w : 0.0;
  }
  __device__ __forceinline__ bool kept(float x, int i) const { return x > cut_v || (x == cut_v && i <= cut_i); }

  // ---- 1: the maximum, the sum beside it, the number of tokens that cannot be drawn
  // Lanes of a warp share the maximum that they have met, so that a larger one, which they turn to together, is rare.  The warps'
  // sums stay in `chunk`, against the row's maximum.
  struct First {
    float tm;
    double s, n;
    int gone;
  };
  __device__ __noinline__ static First first_sweep(const Row row) { return row.sweep_all(); }
  __device__ __forceinline__ First sweep_all() const {
    float tm = kNegInf, n = 0.f;  // the lane's terms: n of e^0, and s
    double s = 0.0;
    int gone = 0;                          // logits of -inf
    float of_part = 0.f;                   // the part's terms so far
    double *parts = sh()->part[warp];
    constexpr int U = 2;
    uint32_t next[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u < mine) load(first + u, next[u]);
    for (int i0 = 0; i0 < mine; i0 += U) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i0 + u >= mine) break;
        const int seg = first + i0 + u;
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = next[u][k];
        float hi, lo;
        extremes(w, hi, lo);
        if (i0 + u + U < mine) load(seg + U, next[u]);
        if (bounded) {
          const uint32_t b = __float_as_uint(hi);
          bounds()[seg * 32 + lane] = (uint16_t)(((b & 0x80000000u) ? b : b + 0xffffu) >> 16);
        }
        if (__any_sync(0xffffffffu, lo == kNegInf)) {
#pragma unroll
          for (int j = 0; j < kPer / 2; ++j) {
            float a, b;
            two_of<T>(w, j, a, b);
            gone += (a == kNegInf) + (b == kNegInf);
          }
        }
        const float top = warp_max(hi);
        const float ref = fmaxf(fmaxf(tm, top), kLowest);
        const bool largest = top >= tm && top > kNegInf;
        if (largest && top > tm) {
          if (tm > kNegInf) {
            const double f = power(((double)tm - (double)top) * inv_t);
            s = (s + (double)n) * f;
            of_part *= (float)f;
          } else {
            of_part = 0.f;  // as n, it has counted what is -inf so far as the largest
          }
          n = 0.f;
          tm = top;
        }
        // terms of the largest are counted; what is -inf, or too far below for the arithmetic, is left out
        if (largest || __any_sync(0xffffffffu, !((lo - ref) * c > -1e4f))) {
          unsigned out = 0;
          float same = 0.f;
#pragma unroll
          for (int j = 0; j < kPer / 2; ++j) {
            float a, b;
            two_of<T>(w, j, a, b);
            same += (a == tm ? 1.f : 0.f) + (b == tm ? 1.f : 0.f);
            out |= (a == ref || (a - ref) * c < -1e4f ? 1u : 0u) << (2 * j) | (b == ref || (b - ref) * c < -1e4f ? 1u : 0u) << (2 * j + 1);
          }
          const float g = terms<true>(w, ref, out);
          s += (double)g;
          n += same;
          of_part += g + same;
        } else {
          const float g = terms<false>(w, ref, 0);
          s += (double)g;
          of_part += g;
        }
        const int i = i0 + u;
        if (((i + 1) & ((1 << log_q) - 1)) == 0 || i + 1 == mine) {
          of_part = warp_sum(of_part);
          if (lane == 0) parts[i >> log_q] = __hiloint2double(__float_as_int(tm), __float_as_int(of_part));
          of_part = 0.f;
        }
      }
    }
    return First{tm, warp_sum(s), warp_sum((double)n), (int)__reduce_add_sync(0xffffffffu, gone)};
  }
  __device__ void stats(double &rest, int &masked) {
    const First f = first_sweep(*this);
    if (lane == 0) {
      sh()->warp_m[warp] = f.tm;
      sh()->warp_a[warp] = f.s;
      sh()->warp_b[warp] = f.n;
      sh()->warp_n[warp] = (uint32_t)f.gone;
    }
    __syncthreads();
    combine(kWarps, sh()->warp_m[lane & (kWarps - 1)], sh()->warp_a[lane & (kWarps - 1)], sh()->warp_b[lane & (kWarps - 1)], m, rest);
    masked = __reduce_add_sync(0xffffffffu, lane < kWarps ? (int)sh()->warp_n[lane & (kWarps - 1)] : 0);
    if (blocks > 1) {
      tell(rest, m, masked);
      const Slot o = told(lane & (blocks - 1));
      combine(blocks, o.m, o.a, 1.0, m, rest);
      masked = __reduce_add_sync(0xffffffffu, lane < blocks ? o.i : 0);
    }
    masked -= all_segs * 32 * kPer - V;  // what lies outside the row
    if (threadIdx.x < kWarps) {
      const float mi = sh()->warp_m[threadIdx.x];
      sh()->chunk[threadIdx.x] =
          mi > kNegInf ? (sh()->warp_a[threadIdx.x] + sh()->warp_b[threadIdx.x]) * power(((double)mi - (double)m) * inv_t) : 0.0;
    }
    __syncthreads();
  }
  // The largest and the least of a granule; those of 16 bits two at a time.
  __device__ __forceinline__ static void extremes(const uint32_t (&w)[8], float &hi, float &lo) {
    if constexpr (sizeof(T) == 4) {
      hi = lo = __uint_as_float(w[0]);
#pragma unroll
      for (int j = 1; j < kPer; ++j) hi = fmaxf(hi, __uint_as_float(w[j])), lo = fminf(lo, __uint_as_float(w[j]));
    } else {
      using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
      T2 a = reinterpret_cast<const T2 &>(w[0]), b = a;
#pragma unroll
      for (int i = 1; i < 8; ++i) {
        const T2 v = reinterpret_cast<const T2 &>(w[i]);
        a = __hmax2(a, v), b = __hmin2(b, v);
      }
      hi = fmaxf(Storage<T>::widen(a.x), Storage<T>::widen(a.y));
      lo = fminf(Storage<T>::widen(b.x), Storage<T>::widen(b.y));
    }
    hi = fmaxf(hi, kNegInf);  // a granule of NaN
  }
  // Sums a + b e^0 against maxima of their own, those of lanes 0 to n - 1, to one against the largest, which is left out once.
  __device__ __forceinline__ void combine(int n, float mi, double a, double b, float &m_out, double &rest) const {
    const bool has = lane < n;
    const float mm = warp_max(has ? mi : kNegInf);
    const unsigned top = __ballot_sync(0xffffffffu, has && mi == mm && mm > kNegInf);
    double v = 0.0;
    if (has) {
      if (top >> lane & 1)
        v = a + (b - (lane == __ffs(top) - 1 ? 1.0 : 0.0));
      else  // nothing or NaN where there is no maximum
        v = mi > kNegInf ? (a + b) * power(((double)mi - (double)mm) * inv_t) : a;
    }
    m_out = mm;
    rest = warp_sum(v);
  }
  // The sum of 2^{(x - ref) c} over a granule, without the logits in `out`.  The roundings of the product and of c are made good to
  // first order: 2^{a + r} = 2^a (1 + r ln 2).
  template <bool kOut>
  __device__ __forceinline__ float terms(const uint32_t (&w)[8], float ref, unsigned out) const {
    const uint64_t minus = pair(-ref, -ref), up = pair(c, c), down = pair(-c, -c), rest = pair(c_rest, c_rest);
    const uint64_t ln2 = pair(0.6931471805599453f, 0.6931471805599453f);
    uint64_t sum[2];
#pragma unroll
    for (int j = 0; j < kPer / 2; ++j) {
      float lo, hi;
      two_of<T>(w, j, lo, hi);
      const uint64_t d = add2(pair(lo, hi), minus), a = mul2(d, down), r = fma2(d, rest, fma2(d, up, a));
      apart(a, lo, hi);
      const uint64_t p = pair(ex2(-lo), ex2(-hi));
      uint64_t e = fma2(p, mul2(r, ln2), p);
      if constexpr (kOut) {
        apart(e, lo, hi);
        e = pair(out >> (2 * j) & 1 ? 0.f : lo, out >> (2 * j + 1) & 1 ? 0.f : hi);
      }
      sum[j & 1] = j < 2 ? e : add2(sum[j & 1], e);
    }
    float lo, hi;
    apart(add2(sum[0], sum[1]), lo, hi);
    return lo + hi;
  }
  // How far a sum S of terms(), of the row or any of its logits, can be off.  With p_k a logit's share of S, its exponent is
  // -log2 p_k - log2 S, and the mean of these at most the entropy, log2 V, less log2 S.  A difference is rounded once: ln 2 times that
  // mean, times 2^-24; the exponential is good to 4, what is left of product and c to 1, and a granule's additions take 5 at most.
  // It grows with S.
  __device__ __forceinline__ double error(double sum) const {
    const int bits = 32 - __clz(V) + max(0, 1023 - (int)(__double2hiint(sum) >> 20 & 0x7ff));
    return (11.0 + 0.6932 * (double)bits) * kRound * sum;
  }

  // A bit for each of a granule's logits that is at least v; those of 16 bits are compared two at a time, with the least value of
  // the type that is.
  __device__ __forceinline__ static unsigned from(const uint32_t (&w)[8], float v) {
    unsigned mask = 0;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) mask |= __uint_as_float(w[j]) >= v ? 1u << j : 0u;
    } else {
      using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
      T2 least;
      if constexpr (std::is_same<T, __half>::value)
        least.x = least.y = __float2half_ru(v);
      else
        least.x = least.y = __float2bfloat16_ru(v);
#pragma unroll
      for (int i = 0; i < 8; ++i) mask |= __hge2_mask(reinterpret_cast<const T2 &>(w[i]), least) & (1u << (2 * i) | 1u << (17 + 2 * i));
      mask = (mask | mask >> 16) & 0xffff;
    }
    return mask;
  }

  // The same for logits above v, with the largest value of the type that is not above it.
  __device__ __forceinline__ static unsigned over(const uint32_t (&w)[8], float v) {
    unsigned mask = 0;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) mask |= __uint_as_float(w[j]) > v ? 1u << j : 0u;
    } else {
      using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
      T2 most;
      if constexpr (std::is_same<T, __half>::value)
        most.x = most.y = __float2half_rd(v);
      else
        most.x = most.y = __float2bfloat16_rd(v);
#pragma unroll
      for (int i = 0; i < 8; ++i) mask |= __hgt2_mask(reinterpret_cast<const T2 &>(w[i]), most) & (1u << (2 * i) | 1u << (17 + 2 * i));
      mask = (mask | mask >> 16) & 0xffff;
    }
    return mask;
  }
  // A granule with `far` in the place of logits of at least v and below itself.
  __device__ __forceinline__ static void clamp(const uint32_t (&w)[8], float v, T far, uint32_t (&to)[8]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        const float x = __uint_as_float(w[j]);
        to[j] = __float_as_uint(x >= v ? far : fmaxf(x, far));
      }
    } else {
      using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
      T2 least, lowest;
      if constexpr (std::is_same<T, __half>::value)
        least.x = least.y = __float2half_ru(v);
      else
        least.x = least.y = __float2bfloat16_ru(v);
      lowest.x = lowest.y = far;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const T2 x = reinterpret_cast<const T2 &>(w[i]), raised = __hmax2(x, lowest);
        const uint32_t mask = __hge2_mask(x, least);
        to[i] = (reinterpret_cast<const uint32_t &>(lowest) & mask) | (reinterpret_cast<const uint32_t &>(raised) & ~mask);
      }
    }
  }

  // Of the warp's pieces i0 to i0 + 31 those with a granule that reaches `v`: a bit each.
  __device__ __forceinline__ unsigned hot_pieces(int i0, float v) const {
    const int n = min(32, mine - i0);
    if (!bounded) return n >= 32 ? 0xffffffffu : (1u << n) - 1u;
    const uint16_t *b = bounds() + (first + i0) * 32 + lane;
    unsigned hot = 0;
#pragma unroll 4
    for (int i = 0; i < n; ++i)
      if (__any_sync(0xffffffffu, __uint_as_float((uint32_t)b[i * 32] << 16) >= v)) hot |= 1u << i;
    return hot;
  }
  // Calls f(i, w) for the warp's pieces with a granule that reaches `v`, the next one's load under way; of every 32 those in `of`.
  template <typename F>
  __device__ __forceinline__ void each_hot(float v, F f, unsigned of = 0xffffffffu) const {
#pragma unroll 1
    for (int i0 = 0; i0 < mine; i0 += 32) {
      unsigned hot = hot_pieces(i0, v) & of;
      uint32_t next[8];
      if (hot) load(first + i0 + __ffs(hot) - 1, next);
#pragma unroll 1
      while (hot) {
        const int i = i0 + __ffs(hot) - 1;
        hot &= hot - 1;
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = next[j];
        if (hot) load(first + i0 + __ffs(hot) - 1, next);
        f(i, w);
      }
    }
  }

  // What a pass over the row looks for: the logits above `v`, those equal to it up to index `i`, none above `most`.  Of these the
  // ones above `split` are summed up; the others go where `rest` says.
  enum Rest { kNone, kFirst, kBinsOfKeys, kToList };
  struct Pass {
    float v;
    int i;
    float most, split;
    bool weights;  // sums of weights, else of ones
    Rest rest;
    uint32_t k_hi;   // kBinsOfKeys
    int shift;
  };
  // What `chunk` and the parts have of what is kept: see select().
  enum Sums { kStale, kTail, kExact };
  // What is kept, none below `from`.
  __device__ __forceinline__ Pass of_kept(float from) const {
    return Pass{fmaxf(from, cut_v), from > cut_v ? kNoIndex : cut_i, -kNegInf, kNegInf, true, kNone, 0, 0};
  }
  struct Sum {
    double all;  // over the row
    int n;       // their number; kFirst: the first index
  };
  // Reads the granules that can hold such a logit.  A piece's logits that matter are put side by side first: they are few, and
  // each lane by itself would form exponentials for one or two lanes at a time.  Leaves the warps' sums in `chunk` and tells the
  // blocks theirs; the order of the additions is fixed.
  __device__ __noinline__ static Sum pass(Row row, const Pass a) {
    float *value = sh()->compact.value[row.warp];
    uint16_t *place = sh()->compact.place[row.warp];
    double acc = 0.0;
    double *parts = sh()->part[row.warp];
    int n = 0, best = kNoIndex;
    const bool plain = a.i == kNoIndex && a.most == -kNegInf;
    for (int q = row.lane; q < kParts; q += 32) parts[q] = 0.0;
    __syncwarp();
    row.each_hot(a.v, [&](int i, const uint32_t (&w)[8]) {
      const int i0 = row.first_of(row.first + i), base = i0 - row.lane * kPer;
      unsigned mask = from(w, a.v);
      if (!plain) {
#pragma unroll
        for (int j = 0; j < kPer / 2; ++j) {
          float lo, hi;
          two_of<T>(w, j, lo, hi);
          if (!(lo <= a.most && (lo > a.v || i0 + 2 * j <= a.i))) mask &= ~(1u << (2 * j));
          if (!(hi <= a.most && (hi > a.v || i0 + 2 * j + 1 <= a.i))) mask &= ~(2u << (2 * j));
        }
      }
      if (!__any_sync(0xffffffffu, mask != 0)) return;
      const int own = __popc(mask), up_to = warp_scan(own), all = __shfl_sync(0xffffffffu, up_to, 31);
      double of_piece = 0.0;
      int at = up_to - own;
      if (a.rest == kNone) {
        // sums alone: two side by side, as one exponential is a long chain
#pragma unroll
        for (int j = 0; j < kPer / 2; ++j) {
          float lo, hi;
          two_of<T>(w, j, lo, hi);
          if (mask >> (2 * j) & 1) value[at++] = lo;
          if (mask >> (2 * j + 1) & 1) value[at++] = hi;
        }
        __syncwarp();
        if (!a.weights) {
          of_piece += (double)own;
        } else {
#pragma unroll 1
          for (int e = row.lane; e < all; e += 64) {
            const double one = row.weight(value[e]), two = row.weight(e + 32 < all ? value[e + 32] : kNegInf);
            of_piece += one + two;
          }
        }
        n += own;
      } else {
#pragma unroll
        for (int j = 0; j < kPer / 2; ++j) {
          float lo, hi;
          two_of<T>(w, j, lo, hi);
          if (mask >> (2 * j) & 1) {
            value[at] = lo;
            place[at++] = (uint16_t)(row.lane * kPer + 2 * j);
          }
          if (mask >> (2 * j + 1) & 1) {
            value[at] = hi;
            place[at++] = (uint16_t)(row.lane * kPer + 2 * j + 1);
          }
        }
        __syncwarp();
#pragma unroll 1
        for (int e = row.lane; e < all; e += 32) {
          const float v = value[e];
          if (v > a.split) {
            of_piece += a.weights ? row.weight(v) : 1.0;
            ++n;
          } else {
            const int at_row = base + place[e];
            if (a.rest == kFirst) {
              best = min(best, at_row);
            } else if (a.rest == kBinsOfKeys) {
              atomicAdd(&sh()->hist[(a.k_hi - key_of(v)) >> a.shift], 1u);
            } else if (a.rest == kToList) {
              row.to_list(v, at_row);
            }
          }
        }
      }
      __syncwarp();
      if (a.rest != kFirst && a.rest != kBinsOfKeys) {
        of_piece = warp_sum(of_piece);
        if (row.lane == 0) parts[i >> row.log_q] += of_piece;
        acc += of_piece;
      } else if (__any_sync(0xffffffffu, of_piece != 0.0)) {
        acc += warp_sum(of_piece);
      }
    });
    return row.joined(acc, a.rest == kFirst ? best : n, a.rest == kFirst);
  }
  // The warps' sums to `chunk`, the blocks' to each other; `first`: the least of their n, else the sum.
  __device__ __forceinline__ Sum joined(double acc, int n, bool first) {
    n = first ? __reduce_min_sync(0xffffffffu, n) : __reduce_add_sync(0xffffffffu, n);
    __syncthreads();  // chunk and warp_n have been read
    if (lane == 0) {
      sh()->chunk[warp] = acc;
      sh()->warp_n[warp] = (uint32_t)n;
    }
    __syncthreads();
    const int ns = (int)sh()->warp_n[lane & (kWarps - 1)];
    n = first ? __reduce_min_sync(0xffffffffu, ns) : __reduce_add_sync(0xffffffffu, lane < kWarps ? ns : 0);
    Sum r;
    r.all = warp_sum(lane < kWarps ? sh()->chunk[lane & (kWarps - 1)] : 0.0);
    r.n = n;
    if (blocks > 1) {
      turn ^= 1;
      if (threadIdx.x == 0) sh()->slot[turn] = Slot{r.all, 0.f, n};
      meet();
      const Slot o = told(lane & (blocks - 1));
      r.all = warp_sum(lane < blocks ? o.a : 0.0);
      r.n = first ? __reduce_min_sync(0xffffffffu, o.i) : __reduce_add_sync(0xffffffffu, lane < blocks ? o.i : 0);
    }
    return r;
  }
  __device__ __forceinline__ Sum sum(const Pass &a) {
    const Sum r = pass(*this, a);
    if (blocks > 1) turn ^= 1;  // as the pass has told the blocks
    replace();
    return r;
  }
  // The histogram of the distances of what is kept, none below `low`: most of a row's logits, one by one.
  __device__ __noinline__ static void bins_of_distance(Row row, float low, float per, unsigned of) {
    uint32_t *hist = row.sh()->hist;
    const bool plain = low > row.cut_v || row.cut_i == kNoIndex;
    const float v = fmaxf(low, row.cut_v);
    row.each_hot(v, [&](int i, const uint32_t (&w)[8]) {
      const int i0 = row.first_of(row.first + i);
#pragma unroll
      for (int j = 0; j < kPer / 2; ++j) {
        float lo, hi;
        two_of<T>(w, j, lo, hi);
        if (lo >= v && (plain || row.kept(lo, i0 + 2 * j))) atomicAdd(&hist[row.bin_of(lo, per)], 1u);
        if (hi >= v && (plain || row.kept(hi, i0 + 2 * j + 1))) atomicAdd(&hist[row.bin_of(hi, per)], 1u);
      }
    }, of);
  }
  // The sum of the warps' parts that lie in `chunk`.
  __device__ __forceinline__ double sum_of_chunks() {
    double v = warp_sum(lane < kWarps ? sh()->chunk[lane & (kWarps - 1)] : 0.0);
    if (blocks > 1) {
      tell(v, 0.f, 0);
      v = warp_sum(lane < blocks ? told(lane & (blocks - 1)).a : 0.0);
    }
    return v;
  }
  // The whole row's, in double, with nothing to leave out: a logit of -inf has no weight by itself.  Many exponentials side by side, since
  // one is a long chain (151,936 logits by one block of an SM: 46 us, as a pass 80).
  __device__ __noinline__ static Sum sweep_whole(Row row) {
    double *parts = sh()->part[row.warp];
    for (int q = row.lane; q < kParts; q += 32) parts[q] = 0.0;
    __syncwarp();
    double acc = 0.0;
#pragma unroll 1
    for (int i = 0; i < row.mine; ++i) {
      uint32_t w[8];
      row.load(row.first + i, w);
      double of_piece = 0.0;
#pragma unroll
      for (int j = 0; j < kPer / 2; ++j) {
        float lo, hi;
        two_of<T>(w, j, lo, hi);
        of_piece += row.weight(lo) + row.weight(hi);
      }
      of_piece = warp_sum(of_piece);
      if (row.lane == 0) parts[i >> row.log_q] += of_piece;
      acc += of_piece;
    }
    return row.joined(acc, 0, false);
  }
  __device__ __forceinline__ double whole() {
    const double all = sweep_whole(*this).all;
    if (blocks > 1) turn ^= 1;  // as the sweep has told the blocks
    replace();
    return all;
  }

  // The index at which the running sum of a pass `a` over the row passes `aim`, where the warps' parts lie in `chunk` and the blocks'
  // have been told: the first that it looks for where it does, or the last of those with something where rounding leaves none.
  // Known to the block that has it alone; the others get -2.  `unsure`: how far the parts may be off; then the answer is
  // kNoIndex where that matters, known to all.
  // `have`: the parts are sums of the pass (kExact), or those of the first sweep, of which `behind` is known to lie behind the cut
  // (kTail): their own roundings come to `unsure` then.
  __device__ __noinline__ static int find(Row row, const Pass a, double aim, double unsure, Sums have, double behind) {
    const int lane = row.lane, blocks = row.blocks;
    const auto amount = [&](float x, int i) {
      if (!(x >= a.v && x <= a.most && (x > a.v || i <= a.i))) return 0.0;
      return a.weights ? row.weight(x) : 1.0;
    };
    // where the running sum, `run` in front of lane 0, passes: the lane, or the last with something (-1); moves `run` in front of it
    bool hit = true;
    const auto passes = [&](double part, double &run) {
      const double up_to = warp_scan(part);
      const unsigned over = __ballot_sync(0xffffffffu, run + up_to > aim && part > 0.0), some = __ballot_sync(0xffffffffu, part > 0.0);
      const int who = over ? __ffs(over) - 1 : 31 - __clz(some);
      hit = over != 0;
      if (who >= 0) run += __shfl_sync(0xffffffffu, up_to - part, who);
      return who;
    };
    double run = 0.0;
    int owner = 0;
    if (blocks > 1) owner = max(0, passes(lane < blocks ? row.told(lane & (blocks - 1)).a : 0.0, run));
    int at = -2;
    if (owner == row.rank) {
      // the warp whose part it is
      const int of_warp = max(0, passes(lane < kWarps ? sh()->chunk[lane & (kWarps - 1)] : 0.0, run));
      // a lane's float32 sum has two additions and a product by a rounded factor a piece, and five additions join the lanes
      if (have == kTail) unsure += (double)(6 + (4 << row.log_q)) * kRound * (sh()->chunk[of_warp] + 2.0 * behind);
      const int per = (row.segs + kWarps - 1) / kWarps, s0 = of_warp * per, s1 = min(row.segs, s0 + per);
      // its parts, every warp alike
      int part_of = 0, piece = -1;
      {
        const int parts = (s1 - s0 + (1 << row.log_q) - 1) >> row.log_q;
        const double *stored = sh()->part[of_warp];
        double run_last = run;
#pragma unroll 1
        for (int q = 0; q < parts && piece < 0; q += 32) {
          double part = q + lane < parts ? stored[q + lane] : 0.0;
          if (have == kTail && q + lane < parts) {
            const float top = __int_as_float(__double2hiint(part));
            part = top > kNegInf ? (double)__int_as_float(__double2loint(part)) * row.power(((double)top - (double)row.m) * row.inv_t) : 0.0;
            if (behind > 0.0) part = fmax(0.0, part - sh()->tail[of_warp][q + lane]);
          }
          const double end = run + warp_sum(part);
          const int who = passes(part, run);
          if (who >= 0) {
            part_of = q + who;
            run_last = run;
            if (hit) piece = part_of;
          }
          run = end;
        }
        run = run_last;
      }
      int last = s0 + (part_of << row.log_q);
      if (row.log_q > 0) {
        // the part's pieces one by one
        const int end = min(s1, last + (1 << row.log_q));
        double run_last = run;
        bool found_piece = false;
#pragma unroll 1
        for (int seg = last; seg < end && !found_piece; ++seg) {
          double g = 0.0;
#pragma unroll 1
          for (int j = 0; j < kPer; ++j) {
            const int i = row.first_of(seg) - lane * kPer + lane + 32 * j;
            if (i >= 0 && i < row.V) g += amount(Storage<T>::widen(row.z[i]), i);
          }
          g = warp_sum(g);
          if (g > 0.0) {
            last = seg;
            run_last = run;
            found_piece = run + g > aim;
          }
          run += g;
        }
        run = run_last;
        if (!found_piece) piece = -1;
      }
      bool clear = piece >= 0;
      // its 32s of logits, a warp each, then the logit
      const int i0 = row.first_of(last) - lane * kPer;
      const auto term = [&](int group) {
        const int i = i0 + group * 32 + lane;
        return i >= 0 && i < row.V ? amount(Storage<T>::widen(row.z[i]), i) : 0.0;
      };
#pragma unroll 1
      for (int g = row.warp; g < kPer; g += kWarps) {
        const double all = warp_sum(term(g));
        if (lane == 0) sh()->group[g] = all;
      }
      __syncthreads();
      const int group = max(0, passes(lane < kPer ? sh()->group[lane] : 0.0, run));
      clear = clear && hit;
      const double g = term(group);
      const int who = max(0, passes(g, run));
      const double v = __shfl_sync(0xffffffffu, g, who);
      at = min(max(i0 + group * 32 + who, 0), row.V - 1);
      if (unsure > 0.0 && !(clear && hit && run + unsure <= aim && run + v - unsure > aim)) at = kNoIndex;
    }
    return at;
  }
  // find(), and whether it failed, known to all blocks; `everywhere`: the index too.
  __device__ __forceinline__ int found(const Pass &a, double aim, double unsure, bool everywhere, Sums have, double behind) {
#ifdef DVP_DEBUG_BOUNDS
    bounds_ok(have == kTail && replaced ? 1 : 0, 1, DVP_STALE_SUMS);
#endif
    int at = find(*this, a, aim, unsure, have, behind);
    if ((everywhere || unsure > 0.0) && blocks > 1) {
      tell(0.0, 0.f, at);
      const int any = __reduce_max_sync(0xffffffffu, told(lane & (blocks - 1)).i);
      if (everywhere || any == kNoIndex) at = any;
    }
    return at;
  }

  // ---- 2: the cut
  // Logits in the order of the row lie in bins by their distance from the maximum; the last bin has all from kBins - 1 on.
  __device__ __forceinline__ int bin_of(float x, float per) const {
    return min(kBins - 1, __float2int_rz((m - x) * per));  // the conversion saturates; infinity times 0 is bin 0 as all the others
  }

  // A lower bound of the k-th largest logit from the granules' maxima: where k granules reach up to a value, k logits do.
  __device__ float floor_of(long long k) {
    float low = cut_v;
    const int n = segs * 16;  // pairs
    if (bounded && k <= 2 * n) {
      if (threadIdx.x < 3) sh()->counter[threadIdx.x] = 0;
      __syncthreads();
      const uint32_t *pairs = reinterpret_cast<const uint32_t *>(bounds());
      uint32_t lo = 0, hi = 0xffff;  // of the order: the largest b that k bounds reach
      for (int round = 0; lo < hi; ++round) {
        const uint32_t mid = (lo + hi + 1) >> 1;
        // of the order, and so of the values: bounds of the least such value and above, two at a time
        const float v = value_of(mid << 16 | (mid & 0x8000u ? 0u : 0xffffu));
        __nv_bfloat162 least;
        least.x = least.y = __ushort_as_bfloat16((unsigned short)(__float_as_uint(v) >> 16));
        int two = 0;
        for (int i = threadIdx.x; i < n; i += kThreads) two += __hge2_mask(reinterpret_cast<const __nv_bfloat162 &>(pairs[i]), least) & 0x10001u;
        int reach = (two & 0xffff) + (two >> 16);
        reach = __reduce_add_sync(0xffffffffu, reach);
        // three counters in turn: one is added to, one is read, one is cleared for the next
        if (lane == 0 && reach) atomicAdd(&sh()->counter[round % 3], (uint32_t)reach);
        if (threadIdx.x == 0) sh()->counter[(round + 1) % 3] = 0;
        __syncthreads();
        if ((long long)sh()->counter[round % 3] >= k)
          lo = mid;
        else
          hi = mid - 1;
      }
      // a bound that was rounded up is above the bfloat16 in front of it
      const uint32_t b = std::is_same<T, __nv_bfloat16>::value ? lo : lo ? lo - 1 : 0;
      const float v = value_of(b << 16);
      if (v == v) low = fmaxf(low, v);
    }
    if (blocks > 1) {
      tell(0.0, low, 0);
      low = warp_max(told(lane & (blocks - 1)).m);
    }
    return low;
  }

  // Moves the cut to the last logit, in falling order, before which less than share * all lies; weights: sums of weights, else
  // of ones.  Logits below `floor` are known to lie behind it.  `all`: the amount in the whole row, good to `unsure`, of which at
  // most `below` lies below `floor`.  Returns what `chunk` and the parts have then, with `n_kept` the number that is kept: kTail, the
  // first sweep's parts and `tail` of them what is not kept; kExact, sums of what is kept in double; kStale, neither, and `n_kept` is
  // left to whoever forms them.
  __device__ Sums select(bool weights, double share, double all, double unsure, float floor, double below, int &n_kept) {
    double aim = share * all;
    const float span = floor > 0.5f * kLowest ? m - floor : (float)(40.0 / inv_t);
    const float most = (float)(kBins - 2) / span, per = span > 0.f && most < 1e30f ? most : 0.f;  // 0: all in one bin
    // level 0: bins of distance; from level 1 on logits from `low` to `high`, in bins by their keys
    float low = floor, high = m;
    uint32_t n_in = 0;
    // A histogram of all that can matter costs more than reading the row again.  Where a warp has pieces enough, one of a quarter
    // of them guesses where the cut is, and what is found there shows whether it was right (1,024 rows, top_p 0.95: from all pieces
    // 891 us, an eighth of them 847, whose windows are wider, a quarter 709).
    bool guess = unsure > 0.0 && all_segs >= 16 * kWarps * blocks;
    bool replaced = false;  // the first sweep's sums: a pass has put its own in their place
    if (guess) {
      for (int i = threadIdx.x; i < kBins; i += kThreads) sh()->hist[i] = 0;
      __syncthreads();
      bins_of_distance(*this, low, per, 0x11111111u << (warp & 3));
      meet();
      window((1.0 - share) * all, below, per);
      n_in = sh()->pick_last;
      guess = n_in <= kList * 7 / 8 && per > 0.f;
      if (guess) edges(sh()->pick_lo, sh()->pick_hi, per, low, high);
      meet();  // the histograms have been read
    }
    // Bounds by the bins' edges need not say where among many bins the cut lies (an aim next to the sum of what lies far in front of the
    // rest, say), and say no more at the next level.  That one is for the lower half of the bins then, from `half` down, and its
    // sum of what lies above says whether the cut is there at all.
    bool halve = false;
    float half = 0.f;
    // from the second level on every one divides the keys by 64, or the next one by 2: 2^32 of them want fewer than 70
#pragma unroll 1
    for (int level = guess ? 1 : 0; level < 70; ++level) {
      const float top = high;
      if (halve) high = half;
      const uint32_t k_lo = key_of(low), k_hi = key_of(high), width = k_hi - k_lo;
      const int shift = max(0, 21 - __clz(width));  // (width >> shift) < kBins
      const bool gather = level > 0 && n_in <= kList;
      // where the bracket has one value, its logits are taken by their index
      const bool ties = level > 0 && !gather && width == 0 && !halve;
      if (level == 2 && !gather && unsure > 0.0) {  // a flat row: bins of single values want the aim itself
        all = whole();
        aim = share * all;
        unsure = 0.0;
      }
      __syncthreads();
      for (int i = threadIdx.x; i < kBins; i += kThreads) sh()->hist[i] = 0;
      if (threadIdx.x == 0) sh()->list_n = 0;
      __syncthreads();
      Pass a = of_kept(low);
      // weights are summed up in any case: they are wanted next
      a.split = high;  // only the logits above; what is cut already lies at the bracket's end or behind it
      a.rest = ties ? kNone : gather ? kToList : kBinsOfKeys;
      if (ties) a.v = high, a.i = -1;
      a.k_hi = k_hi;
      a.shift = shift;
      Sum sums = {0.0, 0};
      double above = 0.0;
      double tail = 0.0;
      int n_not = 0;
      if (level == 0) {
        bins_of_distance(*this, low, per, 0xffffffffu);
        meet();
      } else if (gather && unsure > 0.0) {
        const Behind b = behind(low, high);
        tail = b.sum, n_not = b.n_not;
      } else {
        sums = sum(a);
        replaced = true;
        above = weights ? sums.all : (double)sums.n;
      }
      if (halve) {
        halve = false;
        if (above >= aim) {
          low = value_of(k_hi + 1);
          high = top;
          continue;
        }
      }
      if (ties) {
        // kept are the first r with above + (r - 1) w < aim
        const double w = weights ? weight(high) : 1.0;
        const auto number = [&](double to) {
          double r = fmin((double)n_in, fmax(1.0, ceil((to - above) / w)));
          if (r > 1.0 && !(above + (r - 1.0) * w < to))
            r -= 1.0;
          else if (r < (double)n_in && above + r * w < to)
            r += 1.0;
          return r;
        };
        const double r = number(aim);
        a = of_kept(high);
        a.most = high;
        a.weights = false;
        sum(a);
        cut_i = found(a, r - 0.5, 0.0, true, kExact, 0.0);
        cut_v = high;
        return kStale;
      }
      if (gather) {
        // all blocks' lists in one, alike in every block
        int n = 0;
#pragma unroll 1
        for (int r = 0; r < blocks; ++r) {
          const Shared *o = r == rank ? sh() : of(r);
          const int k = (int)o->list_n;
          if (n + k <= kList)
            for (int i = threadIdx.x; i < k; i += kThreads) sh()->sorted[n + i] = o->list[i];
          n += k;
        }
        if (blocks > 1) meet();  // the lists have been read
        if (n > kList && !guess) {  // more on the bracket's edge than its bins had
          n_in = (uint32_t)n;
          continue;
        }
        if (n <= kList) sort_list(n, k_lo, k_hi);
        int last;
        Sums have = kExact;
        if (unsure > 0.0) {
          // Kept is what has more than (1 - share) all at and behind it.  Of that side's sums, the whole's and the tail's, float32's
          // errors are the smaller by 1 - share; mostly nothing lies so near the border that they matter.
          const Border at = n <= kList ? cut_from_list(true, n, tail - (1.0 - share) * all, true, (1.0 - share) * unsure + error(tail), last)
                                       : kOutside;
          if (at == kOutside && guess) {
            guess = false;  // the long way then
            low = floor, high = m;
            level = -1;
            continue;
          }
          have = replaced ? kStale : kTail;  // what lies behind says what is kept of the first sweep's sums, and only of them
          if (at != kClear) {
            for (int i = threadIdx.x; i < n; i += kThreads) sh()->list[i] = sh()->sorted[i];  // passes take their place
            __syncthreads();
            aim = share * whole();
            a.v = high;
            a.i = -1;
            a.rest = kNone;
            sums = sum(a);
            for (int i = threadIdx.x; i < n; i += kThreads) sh()->sorted[i] = sh()->list[i];
            __syncthreads();
            cut_from_list(true, n, aim - sums.all, false, 0.0, last);
            have = kExact;
          }
        } else {
          cut_from_list(weights, n, aim - above, false, 0.0, last);
        }
        set_cut(last);
        if (have != kStale) {
          // The list's logits: those behind the cut go to the tail, or the kept ones to the exact sums, of the warp that has their
          // pieces and of their part.
          // Whole numbers of 2^-52 of the largest are added, in any order.
          static_assert(kBins * sizeof(uint32_t) == kWarps * kParts * sizeof(uint64_t), "the sums lie in the histogram");
          unsigned long long *sums_of = reinterpret_cast<unsigned long long *>(sh()->hist);
          const int each = (segs + kWarps - 1) / kWarps;
          const int from = have == kTail ? last + 1 : 0, to = have == kTail ? n : last + 1;
          for (int i = threadIdx.x; i < kWarps * kParts; i += kThreads) sums_of[i] = 0;
          __syncthreads();
          const double largest = from < to ? weight(value_of(~(uint32_t)(sh()->sorted[from] >> 32))) : 1.0;
          const double up = 4503599627370496.0 / fmax(largest, 1e-290);
          for (int i = from + threadIdx.x; i < to; i += kThreads) {
            const uint64_t item = sh()->sorted[i];
            const int piece = (int)((uint32_t)item + off) / (32 * kPer) - seg0;
            if (piece < 0 || piece >= segs) continue;
            const int of = piece / each;
            atomicAdd(&sums_of[of * kParts + ((piece - of * each) >> log_q)],
                      (unsigned long long)__double2ll_rn(weight(value_of(~(uint32_t)(item >> 32))) * up));
          }
          __syncthreads();
          double acc = 0.0;
          for (int q = lane; q < kParts; q += 32) {
            const double v = (double)sums_of[warp * kParts + q] * (fmax(largest, 1e-290) * 2.220446049250313e-16);
            acc += v;
            if (have == kTail)
              sh()->tail[warp][q] += v;
            else
              sh()->part[warp][q] += v;
          }
          acc = warp_sum(acc);
          if (lane == 0) sh()->chunk[warp] += have == kTail ? -(sh()->warp_b[warp] + acc) : acc;
          n_kept = have == kTail ? n_not - (n - 1 - last) : sums.n + last + 1;
          __syncthreads();
        }
        return have;
      }
      bracket(weights, level, aim, above, all, share * unsure, below, unsure, per, k_lo, k_hi, shift);
      const uint32_t lo = sh()->pick_lo, hi = sh()->pick_hi;
      n_in = sh()->pick_last;
      meet();  // the histograms have been read
      if (n_in == 0) return kStale;  // less than the aim in all: everything stays
      if (level == 0) {
        edges(lo, hi, per, low, high);
      } else {
        low = fmaxf(low, value_of(edge_of(k_lo, k_hi, hi, shift)));
        high = value_of(k_hi - (lo << shift));
        halve = weights && unsure == 0.0 && shift > 0 && hi - lo >= kBins / 64 && n_in > kList;
        half = value_of(edge_of(k_lo, k_hi, (lo + hi) / 2, shift) - 1);
      }
    }
    return kStale;
  }
  // The values, from low to high, that the logits in bins lo to hi can have; 2^-20 covers the roundings of the distance.
  __device__ __forceinline__ void edges(uint32_t lo, uint32_t hi, float per, float &low, float &high) const {
    const double slack = 9.5367431640625e-7;
    if (!(per > 0.f)) return;
    high = fminf(m, __double2float_ru((double)m - (double)lo / per * (1.0 - slack)));
    if (hi < kBins - 1) low = fmaxf(low, __double2float_rd((double)m - ((double)hi + 1.0) / per * (1.0 + slack)));
  }
  // From the histograms of a quarter of the row: the bins in which the sum over what lies behind can fall below `end`, within three
  // standard deviations and 0.5 %: pick_lo to pick_hi, which may have pick_last logits.  Every block alike.
  __device__ void window(double end, double below, float per) {
    constexpr int kOwn = kBins / kThreads;
    uint32_t n[kOwn];
    float w[kOwn], sum = 0.f, squares = 0.f;
    bins_of_row(n);
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      w[j] = ex2(-((float)(threadIdx.x * kOwn + j) + 0.5f) / per * c);
      sum += (float)n[j] * w[j];
      squares += (float)n[j] * w[j] * w[j];
    }
    const float sum_up = warp_scan(sum), squares_up = warp_scan(squares);
    __syncthreads();
    if (lane == 31) {
      sh()->warp_a[warp] = (double)sum_up;
      sh()->warp_b[warp] = (double)squares_up;
    }
    if (threadIdx.x == 0) sh()->pick_lo = sh()->pick_hi = kBins - 1;
    __syncthreads();
    // what lies behind this thread's bins: all, less what lies in front of them and in them
    float behind_w = 0.f, behind_s = 0.f;
    for (int v = warp; v < kWarps; ++v) behind_w += (float)sh()->warp_a[v], behind_s += (float)sh()->warp_b[v];
    behind_w -= sum_up - sum;
    behind_s -= squares_up - squares;
    uint32_t lo = kBins, hi = kBins;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      behind_w -= (float)n[j] * w[j];
      behind_s -= (float)n[j] * w[j] * w[j];
      const float off = 3.f * sqrtf(12.f * fmaxf(behind_s, 0.f)) + 0.005f * (float)end + (float)below;
      if (4.f * behind_w - off < (float)end) lo = min(lo, threadIdx.x * kOwn + j);
      if (4.f * behind_w + off < (float)end) hi = min(hi, threadIdx.x * kOwn + j);
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_min_sync(0xffffffffu, hi);
    if (lane == 0) {
      if (lo < (uint32_t)kBins) atomicMin(&sh()->pick_lo, lo);
      if (hi < (uint32_t)kBins) atomicMin(&sh()->pick_hi, hi);
    }
    __syncthreads();
    lo = sh()->pick_lo, hi = sh()->pick_hi;
    uint32_t inside = 0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const uint32_t b = threadIdx.x * kOwn + j;
      if (b >= lo && b <= hi) inside += n[j];
    }
    inside = __reduce_add_sync(0xffffffffu, inside);
    if (threadIdx.x == 0) sh()->pick_last = 0;
    __syncthreads();
    if (lane == 0 && inside) atomicAdd(&sh()->pick_last, 4 * inside);
    __syncthreads();
  }
  // The row's numbers in the thread's bins.
  __device__ __forceinline__ void bins_of_row(uint32_t (&n)[kBins / kThreads]) const {
    constexpr int kOwn = kBins / kThreads;
    static_assert(kOwn % 4 == 0, "bins are read four at a time");
#pragma unroll
    for (int j = 0; j < kOwn; ++j) n[j] = 0;
#pragma unroll 1
    for (int r = 0; r < blocks; ++r) {
      const uint32_t *hist = (r ? of((rank + r) & (blocks - 1)) : sh())->hist + threadIdx.x * kOwn;
#pragma unroll
      for (int j = 0; j < kOwn; j += 4) {
        const uint4 q = *reinterpret_cast<const uint4 *>(hist + j);
        n[j] += q.x, n[j + 1] += q.y, n[j + 2] += q.z, n[j + 3] += q.w;
      }
    }
  }
  __device__ __forceinline__ void set_cut(int last) {
    const uint64_t item = sh()->sorted[last];
    cut_v = value_of(~(uint32_t)(item >> 32));
    cut_i = (int)(uint32_t)item;
  }
  __device__ __forceinline__ void to_list(float x, int i) const {
    const uint32_t to = atomicAdd(&sh()->list_n, 1u);
    if (to < kList) sh()->list[to] = (uint64_t)(~key_of(x)) << 32 | (uint32_t)i;
  }
  // Of a row that nothing is cut from: the float32 sum of the weights of logits below `low`, with what lies from there to `high` to
  // the list.  Leaves `chunk` alone.
  struct Behind {
    double sum;
    int n_not;  // logits that are not behind
  };
  __device__ __noinline__ static Behind behind_of_warp(const Row row, float low, float high) { return row.sweep_behind(low, high); }
  __device__ __forceinline__ Behind sweep_behind(float low, float high) const {
    double s = 0.0;
    int n_not = 0;
    double *tails = sh()->tail[warp];
    for (int q = lane; q < kParts; q += 32) tails[q] = 0.0;
    __syncwarp();
    // a logit without weight, which takes the place of what is not behind and of all that lies below it
    const T far = Storage<T>::narrow(m - 1000.f / c);
    const float at_far = (Storage<T>::widen(far) - m) * c;
    const bool clamped = at_far < -200.f && at_far > -5000.f;
    // granules with something for the list: few, so they wait until a warp's lanes can take one each
    constexpr int kMost = Shared::kPiece;
    uint32_t *granule = reinterpret_cast<uint32_t *>(sh()->compact.value[warp]);
    uint16_t *which = sh()->compact.place[warp];
    int waiting = 0;
    const auto drain = [&] {
      __syncwarp();
#pragma unroll 1
      for (int e = lane; e < waiting; e += 32) {
        const int i0 = (int)((seg0 + first) * 32 + granule[e]) * kPer - off;
#pragma unroll 1
        for (unsigned mask = which[e]; mask; mask &= mask - 1) {
          const int i = i0 + __ffs(mask) - 1;
          to_list(Storage<T>::widen(z[i]), i);
        }
      }
      __syncwarp();
      waiting = 0;
    };
    // one piece on its way (1,024 rows, top_p 0.95: 529 us; two 533, three 607, for want of registers)
    uint32_t next[8];
    if (mine > 0) load(first, next);
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
      uint32_t w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = next[j];
      if (i + 1 < mine) load(first + i + 1, next);
      const unsigned from_low = from(w, low), in = from_low & ~over(w, high);
      n_not += __popc(from_low);
      float g;
      if (clamped) {
        uint32_t v[8];
        clamp(w, low, far, v);
        g = terms<false>(v, m, 0);
      } else {
        unsigned out = 0;
#pragma unroll
        for (int j = 0; j < kPer / 2; ++j) {
          float a, b;
          two_of<T>(w, j, a, b);
          out |= ((a - m) * c < -1e4f ? 1u : 0u) << (2 * j) | ((b - m) * c < -1e4f ? 1u : 0u) << (2 * j + 1);
        }
        g = terms<true>(w, m, out | from_low);
      }
      g = warp_sum(g);
      if (lane == 0) {
        tails[i >> log_q] += (double)g;
        s += (double)g;
      }
      const unsigned some = __ballot_sync(0xffffffffu, in != 0);
      if (in != 0) {
        const int at = waiting + __popc(some & ((1u << lane) - 1u));
        granule[at] = (uint32_t)(i * 32 + lane);
        which[at] = (uint16_t)in;
      }
      waiting += __popc(some);
      if (waiting > kMost - 32) drain();
    }
    drain();
    return Behind{__shfl_sync(0xffffffffu, s, 0), (int)__reduce_add_sync(0xffffffffu, n_not)};
  }
  // The warps' sums stay in warp_b.
  __device__ Behind behind(float low, float high) {
    const Behind w = behind_of_warp(*this, low, high);
    __syncthreads();
    if (lane == 0) {
      sh()->warp_b[warp] = w.sum;
      sh()->warp_n[warp] = (uint32_t)w.n_not;
    }
    __syncthreads();
    Behind r;
    r.sum = warp_sum(lane < kWarps ? sh()->warp_b[lane & (kWarps - 1)] : 0.0);
    r.n_not = (int)__reduce_add_sync(0xffffffffu, lane < kWarps ? sh()->warp_n[lane & (kWarps - 1)] : 0u);
    if (blocks > 1) {
      tell(r.sum, 0.f, r.n_not);
      const Slot o = told(lane & (blocks - 1));
      r.sum = warp_sum(lane < blocks ? o.a : 0.0);
      r.n_not = (int)__reduce_add_sync(0xffffffffu, lane < blocks ? o.i : 0);
    }
    return r;
  }
  // The least key of bin b, of keys from k_lo to k_hi: bin 0 has the largest.
  __device__ __forceinline__ static uint32_t edge_of(uint32_t k_lo, uint32_t k_hi, uint32_t b, int shift) {
    const int64_t least = (int64_t)k_hi - (int64_t)(((uint64_t)b + 1) << shift) + 1;
    return least > (int64_t)k_lo ? (uint32_t)least : k_lo;
  }

  // Which of the histograms' bins can hold the cut, whose aim is good to `unsure`: pick_lo to pick_hi, which have pick_last logits (0:
  // all of it lies in front of the aim).  Every block alike.
  __device__ void bracket(bool weights, int level, double aim, double above, double all, double unsure, double below, double all_unsure, float per,
                          uint32_t k_lo, uint32_t k_hi, int shift) {
    constexpr int kOwn = kBins / kThreads;
    // where a bin holds one value, its bounds are one
    const bool sharp = !weights || (level > 1 && shift == 0);
    uint32_t n[kOwn];
    double least[kOwn], most[kOwn], least_sum = 0.0, most_sum = 0.0;
    bins_of_row(n);
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const uint32_t b = threadIdx.x * kOwn + j;
      least[j] = most[j] = (double)n[j];
      if (weights && n[j]) {
        if (level == 0) {
          // the bin's distances from the maximum; 2^-20 and 1e-5 cover the roundings
          const float near = (float)b / per * (1.f - 1e-6f), far = ((float)b + 1.f) / per * (1.f + 1e-6f);
          most[j] *= per > 0.f ? (double)ex2(-near * c) * (1.0 + 1e-5) : 1.0;
          least[j] *= b == kBins - 1 || per == 0.f ? 0.0 : (double)ex2(-far * c) * (1.0 - 1e-5);
        } else {
          const double near = (double)m - (double)value_of(k_hi - (b << shift));
          const double far = (double)m - (double)value_of(edge_of(k_lo, k_hi, b, shift));
          most[j] *= power(-near * inv_t);
          least[j] = sharp ? most[j] : least[j] * power(-far * inv_t);
        }
      }
      least_sum += least[j];
      most_sum += most[j];
    }
    const double least_up = warp_scan(least_sum), most_up = warp_scan(most_sum);
    __syncthreads();
    if (lane == 31) {
      sh()->warp_a[warp] = least_up;
      sh()->warp_b[warp] = most_up;
    }
    if (threadIdx.x == 0) {
      sh()->pick_lo = kBins;   // the first bin up to which there can be as much as the aim
      sh()->pick_hi = kBins;   // the first up to which there is
      sh()->pick_last = 0;     // the last that holds anything
    }
    __syncthreads();
    // the warps in front of this one, and all
    const double la = warp_scan(lane < kWarps ? sh()->warp_a[lane & (kWarps - 1)] : 0.0);
    const double lb = warp_scan(lane < kWarps ? sh()->warp_b[lane & (kWarps - 1)] : 0.0);
    const double a_before = __shfl_sync(0xffffffffu, la, max(warp - 1, 0)), b_before = __shfl_sync(0xffffffffu, lb, max(warp - 1, 0));
    double least_run = above + (warp ? a_before : 0.0) + (least_up - least_sum);
    double most_run = above + (warp ? b_before : 0.0) + (most_up - most_sum);
    const double least_all = above + __shfl_sync(0xffffffffu, la, 31), most_all = above + below + __shfl_sync(0xffffffffu, lb, 31);
    uint32_t first_lo = kBins, first_hi = kBins, last_any = 0;
    // A bin's edges bound its weights to a percent or so.  Over the whole row (level 0) the bounds on what lies behind a bin,
    // taken from the known whole, are the closer ones where the aim is near it: 1.5 % of the last twentieth for a top_p of 0.95
    const double eps = sharp ? 0.0 : 1e-11 * all + unsure;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const uint32_t b = threadIdx.x * kOwn + j;
      least_run += least[j];
      most_run += most[j];
      if (!n[j]) continue;
      last_any = b;
      double high = most_run, low = sharp ? most_run : least_run;
      if (!sharp && level == 0) {
        high = fmin(high, all + all_unsure - (least_all - least_run));
        low = fmax(low, all - all_unsure - (most_all - most_run));
      }
      if (high >= aim - eps) first_lo = min(first_lo, b);
      if (low >= aim + eps) first_hi = min(first_hi, b);
    }
    first_lo = __reduce_min_sync(0xffffffffu, first_lo);
    first_hi = __reduce_min_sync(0xffffffffu, first_hi);
    last_any = __reduce_max_sync(0xffffffffu, last_any);
    if (lane == 0) {
      if (first_lo < (uint32_t)kBins) atomicMin(&sh()->pick_lo, first_lo);
      if (first_hi < (uint32_t)kBins) atomicMin(&sh()->pick_hi, first_hi);
      if (last_any) atomicMax(&sh()->pick_last, last_any);
    }
    __syncthreads();
    uint32_t lo = sh()->pick_lo, hi = min(sh()->pick_hi, sh()->pick_last);
    if (level > 0 && lo == kBins) lo = hi = sh()->pick_last;  // the cut is in the bracket: what is missing is a rounding
    // logits in bins lo to hi
    uint32_t inside = 0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const uint32_t b = threadIdx.x * kOwn + j;
      if (lo < (uint32_t)kBins && b >= lo && b <= hi) inside += n[j];
    }
    inside = __reduce_add_sync(0xffffffffu, inside);
    __syncthreads();
    if (threadIdx.x == 0) {
      sh()->pick_lo = lo;
      sh()->pick_hi = hi;
      sh()->pick_last = 0;
    }
    __syncthreads();
    if (lane == 0 && inside) atomicAdd(&sh()->pick_last, inside);
    __syncthreads();
  }

  // Sorts the n items of `sorted`, logits of keys from k_lo to k_hi: falling logits, rising indices.  Where a logit's place among
  // those keys and its index fit 32 bits, which they do for most lists of 16-bit logits, these are sorted: half of the shuffles, and
  // a comparison is one instruction (some 1,700 logits, two rows an SM: 20 thousand cycles, with 64 bits 48).
  __device__ void sort_list(int n, uint32_t k_lo, uint32_t k_hi) {
    __syncthreads();
    constexpr int kLow = sizeof(T) == 4 ? 0 : std::is_same<T, __half>::value ? 13 : 16;  // of a key: all 0 or, below zero, all 1
    const int of_index = 32 - __clz(V), of_key = 32 - __clz((k_hi >> kLow) - (k_lo >> kLow));
    if (of_index + of_key <= 32) {
      sort_items<uint32_t>(n, [&](uint64_t item) {
        return of_key ? ((k_hi >> kLow) - (~(uint32_t)(item >> 32) >> kLow)) << of_index | (uint32_t)item : (uint32_t)item;
      }, [&](uint32_t x) {
        uint32_t key = (k_hi >> kLow) - (of_key ? x >> of_index : 0u);
        key = key << kLow | (key >> (31 - kLow) & 1 ? 0u : (1u << kLow) - 1u);
        return (uint64_t)(~key) << 32 | (of_key ? x & ((1u << of_index) - 1u) : x);
      });
    } else {
      sort_items<uint64_t>(n, [](uint64_t item) { return item; }, [](uint64_t x) { return x; });
    }
  }
  // Four neighbouring items a thread, or one: partners lie in the same thread, the same warp or, farther away, in shared memory.
  template <typename K, typename Pack, typename Unpack>
  __device__ __forceinline__ void sort_items(int n, Pack pack, Unpack unpack) {
    static_assert(kList <= 4 * kThreads, "items of a thread");
    if (n <= kThreads)
      sort_by<K, 1>(n, pack, unpack);
    else
      sort_by<K, 4>(n, pack, unpack);
  }
  template <typename K, int kOwn, typename Pack, typename Unpack>
  __device__ __forceinline__ void sort_by(int n, Pack pack, Unpack unpack) {
    K *const items = reinterpret_cast<K *>(sh()->sorted);
    const int i0 = threadIdx.x * kOwn;
    K x[kOwn];
#pragma unroll
    for (int q = 0; q < kOwn; ++q) x[q] = i0 + q < n ? pack(sh()->sorted[i0 + q]) : ~(K)0;
    int size = 32 * kOwn;
    while (size < n) size <<= 1;
    const bool in = (i0 & ~(32 * kOwn - 1)) < size;
    const auto swap = [](K &a, K &b, bool rising) {
      const K least = a < b ? a : b, most = a < b ? b : a;
      a = rising ? least : most, b = rising ? most : least;
    };
#pragma unroll 1
    for (int k = 2; k <= size; k <<= 1) {
#pragma unroll 1
      for (int j = k >> 1; j >= kOwn; j >>= 1) {
        const bool small = ((i0 & j) == 0) == ((i0 & k) == 0);  // the thread's items take the smaller of the two
        K y[kOwn];
        if (j >= 32 * kOwn) {
          __syncthreads();
#pragma unroll
          for (int q = 0; q < kOwn; ++q)
            if (in) items[i0 + q] = x[q];
          __syncthreads();
#pragma unroll
          for (int q = 0; q < kOwn; ++q) y[q] = in ? items[(i0 ^ j) + q] : x[q];
        } else {
#pragma unroll
          for (int q = 0; q < kOwn; ++q) y[q] = __shfl_xor_sync(0xffffffffu, x[q], j / kOwn);
        }
#pragma unroll
        for (int q = 0; q < kOwn; ++q) x[q] = small ? (x[q] < y[q] ? x[q] : y[q]) : (x[q] < y[q] ? y[q] : x[q]);
      }
      if constexpr (kOwn == 4) {
        if (k >= 4) {
          swap(x[0], x[2], (i0 & k) == 0);
          swap(x[1], x[3], (i0 & k) == 0);
        }
        swap(x[0], x[1], (i0 & k) == 0);
        swap(x[2], x[3], ((i0 + 2) & k) == 0);
      }
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kOwn; ++q)
      if (i0 + q < n) sh()->sorted[i0 + q] = unpack(x[q]);
    __syncthreads();
  }
  // The last of the sorted list before which less than the aim lies, and whether that is so for every aim within `unsure`: kClear;
  // kNear, not; kOutside, the cut need not be in the list at all.  `from_end`: the aim is against the list's sum.
  enum Border { kClear, kNear, kOutside };
  __device__ Border cut_from_list(bool weights, int n, double aim, bool from_end, double unsure, int &last) {
    constexpr int kOwn = kList / kThreads;
    double w[kOwn], sum = 0.0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const int i = threadIdx.x * kOwn + j;
      w[j] = i < n ? weights ? weight(value_of(~(uint32_t)(sh()->sorted[i] >> 32))) : 1.0 : 0.0;
      sum += w[j];
    }
    const double up_to = warp_scan(sum);
    __syncthreads();
    if (lane == 31) sh()->warp_a[warp] = up_to;
    __syncthreads();
    const double la = warp_scan(lane < kWarps ? sh()->warp_a[lane & (kWarps - 1)] : 0.0), before = __shfl_sync(0xffffffffu, la, max(warp - 1, 0));
    double run = (warp ? before : 0.0) + (up_to - sum);
    if (from_end) aim += __shfl_sync(0xffffffffu, la, 31);
    int in_front = 0, near = 0, outside = unsure > 0.0 && (n == 0 || !(aim > unsure));  // of the list, before which less than the aim lies: its front
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const int i = threadIdx.x * kOwn + j;
      in_front += i < n && (run < aim || i == 0);
      // the list holds the cut where its first logit is kept, and its end is behind the aim
      near |= unsure > 0.0 && i < n && i > 0 && fabs(run - aim) <= unsure;
      run += w[j];
      outside |= unsure > 0.0 && i == n - 1 && run - aim <= unsure;
    }
    in_front = __reduce_add_sync(0xffffffffu, in_front);
    if (lane == 0) sh()->warp_n[warp] = (uint32_t)in_front;
    near = __syncthreads_or(near);
    outside = __syncthreads_or(outside);
    last = (int)__reduce_add_sync(0xffffffffu, lane < kWarps ? sh()->warp_n[lane & (kWarps - 1)] : 0u) - 1;
    __syncthreads();  // warp_n and warp_a have been read
    return outside ? kOutside : near ? kNear : kClear;
  }
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const Params p) {
  DVP_BOUNDS_BEGIN(p.bounds_status);
  Row<T> row;
  row.bounded = p.bounds != 0;
  row.warp = threadIdx.x >> 5;
  row.lane = threadIdx.x & 31;
  row.blocks = 1 << p.log_blocks;
  row.rank = blockIdx.x & (row.blocks - 1);
  const long long t = blockIdx.x >> p.log_blocks;
  row.z = static_cast<const T *>(p.logits) + t * p.ld;
  row.V = (int)p.V;
  constexpr int kPer = Row<T>::kPer;
  row.off = (int)((reinterpret_cast<uintptr_t>(row.z) & 31) / sizeof(T));
  const long long segs = ((row.off + p.V + kPer - 1) / kPer + 31) / 32, each = (segs + row.blocks - 1) >> p.log_blocks;
  row.all_segs = (int)segs;
  row.seg0 = (int)(each * row.rank);
  row.segs = (int)max(0LL, min(each, segs - row.seg0));
  const int each_warp = (row.segs + kWarps - 1) / kWarps;
  row.first = row.warp * each_warp;
  row.mine = max(0, min(each_warp, row.segs - row.first));
  row.turn = 0;
  row.log_q = 0;
  while (((each_warp + (1 << row.log_q) - 1) >> row.log_q) > kParts) ++row.log_q;

  // the row's settings
  double temperature = p.temperature_rows ? (double)p.temperature_rows[t] : p.temperature;
  double top_p = p.top_p_rows ? (double)p.top_p_rows[t] : p.top_p, rho = p.rho_rows ? (double)p.rho_rows[t] : p.rho;
  long long top_k = p.top_k_rows ? (long long)p.top_k_rows[t] : p.top_k;
  float u = p.uniform[t];
  u = u > 0.f ? fminf(u, 0.999999940395355224609375f) : 0.f;
  bool valid = temperature >= 0.0 && temperature <= 1.2676506002282294e30 && top_p == top_p && rho == rho;
  if (temperature < 7.888609052210118e-31 || top_p <= 0.0) top_k = 1;
  if (!(temperature >= 7.888609052210118e-31) || !valid) temperature = 1.0;
  rho = fmin(rho, 1.0);
  const bool top_k_one = top_k == 1;
  row.inv_t = 1.0 / temperature;
  row.c = (float)(1.4426950408889634 * row.inv_t);
  row.c_rest = (float)(1.4426950408889634 * row.inv_t - (double)row.c);

  if (threadIdx.x < kTable) row.sh()->table[threadIdx.x] = exp2((double)threadIdx.x / kTable);
  __syncthreads();
  double rest;
  int masked;
  row.stats(rest, masked);
  valid = valid && row.m > kNegInf && row.m < -kNegInf && rest == rest;
  int id = -1, count = 0;
  double kept_rest = 0.0;
  if (valid) {
    row.cut_v = rho > 0.0 ? fmaxf(kLowest, __double2float_ru((double)row.m + temperature * log(rho))) : kLowest;
    row.cut_i = kNoIndex;
    if (top_k_one) {
      typename Row<T>::Pass a = row.of_kept(row.m);
      a.split = -kNegInf;
      a.rest = Row<T>::kFirst;
      id = row.sum(a).n;
      count = 1;
    } else {
      bool whole = row.cut_v == kLowest;  // nothing is cut: the sums of the first sweep are those of what is kept
      typename Row<T>::Sums have = Row<T>::kStale;
#pragma unroll 1
      for (int step = 0; step < 2; ++step) {  // top_k, then top_p
        const bool weights = step == 1;
        if (weights ? !(top_p < 1.0) : !(top_k > 0 && top_k < p.V - masked)) continue;
        double share = 1.0, all = (double)top_k, unsure = 0.0, below = 0.0;
        float floor;
        if (weights) {
          share = top_p;
          all = rest + 1.0;
          if (whole)
            unsure = row.error(all);
          else
            all = row.sum(row.of_kept(kLowest)).all;
          // logits whose weight is under a V-th of 0.03 (1 - top_p) of the whole hold less than that much together
          below = 0.003 * (1.0 - top_p) * all;
          floor = fmaxf(row.cut_v, __double2float_rd((double)row.m + temperature * log(below / (double)p.V)));
          below *= 1.001;
        } else {
          floor = row.floor_of(top_k);
        }
        have = row.select(weights, share, all, unsure, floor, below, count);
        whole = false;
      }
      // by float32's sums of the first sweep, of what is kept or of all where nothing is cut, unless the border is too near for them
      const bool was_whole = whole;
      if (whole) {
        have = Row<T>::kTail;
        count = (int)p.V - masked;
      }
      double all;
      id = kNoIndex;
#pragma unroll 1
      while (id == kNoIndex) {
        double unsure = 0.0, behind = 0.0;
        if (have != Row<T>::kStale) {
          all = row.sum_of_chunks();
          // a logarithm near zero wants all of its sum's digits, and a small part of the row has the whole row's errors
          if (have == Row<T>::kTail && !was_whole && !(all > 1.5 && row.error(rest + 1.0) + row.error(rest + 1.0 - all) < 4e-6 * all)) {
            have = Row<T>::kStale;
            continue;
          }
          if (have == Row<T>::kTail) {
            // Of a sum P in front of the token and S behind it, u (P + S) is off by as much of P's error as P itself but for 1 - u of
            // it, and by u of S's.  What is below float32's range is in the last term
            behind = was_whole ? 0.0 : fmax(0.0, rest + 1.0 - all);
            unsure = (1.0 - u) * row.error(u * all + behind) + u * row.error((1.0 - u) * all + behind) + row.error(behind) + 1e-12 * all;
          }
        } else if (was_whole) {
          all = row.whole();
        } else {
          const typename Row<T>::Sum r = row.sum(row.of_kept(kLowest));
          all = r.all;
          count = r.n;
        }
        id = row.found(row.of_kept(kLowest), (double)u * all, unsure, false, have, behind);
        if (id == kNoIndex) have = Row<T>::kStale;
      }
      kept_rest = was_whole ? rest : all - 1.0;
    }
  }
  // the block that has the token writes
  if (threadIdx.x == 0 && (id >= 0 ? top_k_one ? row.rank == 0 : true : id == -1 && row.rank == 0)) {
    if (p.id_is_i32)
      static_cast<int *>(p.ids)[t] = id;
    else
      static_cast<long long *>(p.ids)[t] = id;
    const float nan = __int_as_float(0x7fc00000);
    const double x = id >= 0 ? ((double)Storage<T>::widen(row.z[id]) - (double)row.m) * row.inv_t : 0.0;
#pragma unroll 1
    for (int side = 0; side < 2; ++side) {
      float *to = side ? p.logp_mp : p.logp;
      if (to) to[t] = id >= 0 ? (float)(x - log1p(side ? kept_rest : rest)) : nan;
    }
    if (p.count) p.count[t] = count;
  }
  if (row.blocks > 1) row.meet();  // nobody leaves while its shared memory is read
}

// ---- host --------------------------------------------------------------------------------------------------------------

// Blocks that share a row; the limits are those of a chip of 148 SMs.  More of them shorten the sweeps and lengthen what they do together, and clusters of eight find room
// for fewer of them at a time.  1 / 2 / 4 / 8 blocks a row, us a call, of bfloat16:
//   4 x 151,936, top_p 0.95    110 / 78 / 55 / 51       74 x 151,936, top_p 0.95   226 / 142 / 127 / 185
//   64 x 151,936, nothing cut   71 / 52 / 36 / 42       148 x 151,936, top_k 50     65 / 76 / 171 / 287
//   16 x 32,768, top_p 0.95     55 / 53 / 48 / 51       16 x 8,192, top_k 50        34 / 41 / 41 / 52
// so two where the chip holds them all, four and eight where that leaves room, and as long as each has 16 KB.
inline int choose_blocks(long long T, long long row_bytes) {
  const auto room = [&](int blocks, long long most) { return T * blocks <= most && row_bytes >= blocks * 16LL * 1024; };
  return room(8, 128) ? 3 : room(4, 256) ? 2 : room(2, 296) ? 1 : 0;
}

template <typename T>
cudaError_t launch(const dvp_sample_args *a, Params p, cudaStream_t stream) {
  if (a->launch_hint) {
    for (p.log_blocks = 0; (1u << p.log_blocks) < a->launch_hint;) ++p.log_blocks;
  } else {
    p.log_blocks = choose_blocks(a->T, a->V * (long long)sizeof(T));
  }
  const int blocks = 1 << p.log_blocks;
  // granules of a block's part: whole pieces of 32, for a row that begins anywhere in its first granule
  const long long per = 32 / sizeof(T), segs = ((per - 1 + a->V + per - 1) / per + 31) / 32;
  const long long granules = (segs + blocks - 1) / blocks * 32;
  p.bounds = granules <= kMostBounds ? (int)granules : 0;
  const size_t smem = sizeof(Shared<T>) + (size_t)p.bounds * 2;
  auto kernel = sample_kernel<T>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(sizeof(Shared<T>) + kMostBounds * 2));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a->T << p.log_blocks), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)blocks;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = blocks > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

}  // namespace sample
}  // namespace dvp

extern "C" int dvp_sample(const dvp_sample_args *a) {
  using namespace dvp::sample;
  if (!a || a->struct_size != sizeof(dvp_sample_args)) return DVP_ERR_INVALID_ARG;
  if (a->logits_dtype != DVP_F32 && a->logits_dtype != DVP_BF16 && a->logits_dtype != DVP_F16) return DVP_ERR_UNSUPPORTED;
  if (a->id_dtype != DVP_ID_I64 && a->id_dtype != DVP_ID_I32) return DVP_ERR_UNSUPPORTED;
  if (a->T < 0 || a->V < 1 || a->ld < a->V) return DVP_ERR_INVALID_ARG;
  if (a->T > kMostRows || a->V > kMostLogits) return DVP_ERR_UNSUPPORTED;
  const uint32_t h = a->launch_hint;
  if (h != 0 && h != 1 && h != 2 && h != 4 && h != 8) return DVP_ERR_INVALID_ARG;
  const double least = 7.888609052210118e-31, most = 1.2676506002282294e30;  // 2^-100, 2^100
  if (!a->temperature_rows && !(a->temperature == 0.0 || (a->temperature >= least && a->temperature <= most))) return DVP_ERR_INVALID_ARG;
  if (!a->rho_rows && !(a->rho >= 0.0 && a->rho <= 1.0)) return DVP_ERR_INVALID_ARG;
  if (!a->top_p_rows && !(a->top_p >= 0.0)) return DVP_ERR_INVALID_ARG;
  if (a->T == 0) return DVP_OK;
  if (!a->logits || !a->uniform || !a->ids) return DVP_ERR_INVALID_ARG;
  Params p{a->logits, a->uniform, a->temperature_rows, a->top_p_rows, a->rho_rows, a->top_k_rows, a->temperature, a->top_p, a->rho,
           a->top_k, a->ids, a->logp, a->logp_mp, a->count, a->T, a->V, a->ld, a->id_dtype == DVP_ID_I32, 0, 0, dvp::bounds_status_word()};
  const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
  const cudaError_t e = a->logits_dtype == DVP_F32    ? launch<float>(a, p, stream)
                        : a->logits_dtype == DVP_BF16 ? launch<__nv_bfloat16>(a, p, stream)
                                                      : launch<__half>(a, p, stream);
  return e == cudaSuccess ? DVP_OK : DVP_ERR_CUDA;
}
