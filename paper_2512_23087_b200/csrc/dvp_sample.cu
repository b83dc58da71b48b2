// Sampling: one token per row of logits, from the min-p safe set, the top_k largest of it and of these the fewest that hold top_p
// of their mass, at a temperature, by a given random number.
//
// Every one of the three filters keeps the front of the row in falling order (equal logits by index), so what is kept is one
// cut: the logits above a value `v` and, of those equal to it, the ones up to an index.  Nothing is sorted but a few hundred
// logits around the cut:
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
// is tried first: it is good to `eps`, and mostly nothing lies so near the border that this matters.  With few rows the blocks
// of a cluster share a row and exchange sums through shared memory.
#include <cmath>
#include <type_traits>

#include "dvp_common.cuh"

namespace dvp {
namespace sample {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kBins = 2048, kList = 2048;
constexpr int kTable = 64, kCompact = 256;
constexpr int kSegs = 512;          // sums of pieces in the walk to the token
constexpr int kMostBounds = 32768;  // granules whose maximum is held: 64 KB
constexpr float kLowest = -3.402823466e38f;
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
};

// What a block tells the others of its row.
struct Slot {
  double a;
  float m;
  int i;
};

struct Shared {
  uint64_t list[kList];
  uint64_t sorted[kList];
  uint32_t hist[kBins];
  union {
    float compact[kWarps][kCompact];  // a warp's logits that matter, side by side
    double seg[kSegs];
  };
  double table[kTable];  // 2^(i / kTable)
  double chunk[kWarps];  // the warps' parts of a sum over the row
  double warp_a[kWarps], warp_b[kWarps];
  float warp_m[kWarps];
  uint32_t warp_n[kWarps];
  Slot slot[2];
  uint32_t list_n, counter[3];
  uint32_t pick_lo, pick_hi, pick_last;  // of the histogram's bins; the last that holds anything, then what pick_lo to pick_hi hold
  int unclear;  // whether another cut is possible for a sum that the row can have
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

// The eight words of a granule as logits.
template <typename T>
__device__ __forceinline__ void widen(const uint32_t (&w)[8], float (&x)[32 / sizeof(T)]) {
  Storage<T>::unpack(make_uint4(w[0], w[1], w[2], w[3]), x);
  Storage<T>::unpack(make_uint4(w[4], w[5], w[6], w[7]), x + 16 / sizeof(T));
}

template <typename T>
struct Row {
  static constexpr int kPer = 32 / sizeof(T);  // logits of a granule
  Shared *sh;
  uint16_t *bounds;  // bfloat16, rounded up; NULL: none
  const T *z;
  int V, off;                    // off: logits of the first granule that lie in front of the row
  int seg0, segs, all_segs;      // the block's pieces of 32 granules, the row's
  int first, mine;               // of the block's pieces, the warp's
  int blocks, rank, turn;
  int warp, lane;
  double inv_t;
  float c;  // log2(e) / temperature
  float m;  // the row's maximum
  // what is kept so far
  float cut_v;
  int cut_i;

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
    return static_cast<const Shared *>(__cluster_map_shared_rank(sh, (unsigned)r));
  }
  // Every block's value to all of them.  Two slots in turn: whoever writes one again has met the others since they read it.
  __device__ __forceinline__ void tell(double a, float m_, int i) {
    turn ^= 1;
    if (threadIdx.x == 0) sh->slot[turn] = Slot{a, m_, i};
    meet();
  }
  __device__ __forceinline__ Slot told(int r) const { return r == rank ? sh->slot[turn] : of(r)->slot[turn]; }

  __device__ __forceinline__ int first_of(int seg) const { return ((seg0 + seg) * 32 + lane) * kPer - off; }
  // A lane's granule of a piece; what lies outside the row is -inf.
  __device__ __forceinline__ void load(int seg, uint32_t (&w)[8]) const {
    const int at = first_of(seg);
    if (at >= 0 && at + kPer <= V) {
      ld_stream32(z + at, w);
    } else {
      const uint16_t *h = reinterpret_cast<const uint16_t *>(z);
      const uint32_t none = std::is_same<T, __half>::value ? 0xfc00u : 0xff80u;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4) {
          w[i] = at + i >= 0 && at + i < V ? __float_as_uint(z[at + i]) : 0xff800000u;
        } else {
          const int a = at + 2 * i;
          w[i] = (a >= 0 && a < V ? h[a] : none) | (a + 1 >= 0 && a + 1 < V ? h[a + 1] : none) << 16;
        }
      }
    }
  }

  // e^{(x - m) / T} to some 2^-50.  With y = (x - m) / T and k the whole number next to 64 y / ln 2, r = y - k ln 2 / 64 is at most
  // ln 2 / 128, where six terms of the series leave 4e-17; e^y = 2^(k / 64) e^r, the fraction of the power from the table: eleven
  // operations in double.
  __device__ __forceinline__ double weight(float x) const {
    const double y = ((double)x - (double)m) * inv_t;
    const double big = 6755399441055744.0;  // 1.5 2^52: adding it leaves the whole number in the low bits
    const double shifted = fma(y, 92.33248261689366, big);
    const int k = __double2loint(shifted);
    const double r = fma(shifted - big, -0.010830424696249145, y);
    double e = fma(r, 1.0 / 120.0, 1.0 / 24.0);
    e = fma(e, r, 1.0 / 6.0);
    e = fma(e, r, 0.5);
    e = fma(e, r, 1.0);
    const double q = sh->table[k & (kTable - 1)];
    e = fma(e * r, q, q);
    const double w = __hiloint2double(__double2hiint(e) + (k >> 6) * (1 << 20), __double2loint(e));
    return y > -700.0 ? w : 0.0;
  }
  __device__ __forceinline__ bool kept(float x, int i) const { return x > cut_v || (x == cut_v && i <= cut_i); }

  // ---- 1: the maximum, the sum beside it, the number of tokens that cannot be drawn
  // Lanes of a warp share the maximum that they have met, so that a larger one, which they turn to together, is rare.  The warps'
  // sums stay in `chunk`, against the row's maximum.
  __device__ void stats(double &rest, int &masked) {
    float tm = kNegInf, s = 0.f, n = 0.f;  // the lane's terms: n of e^0, and s
    int gone = 0;                          // logits of -inf
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
        float x[kPer], hi, lo;
        widen<T>(next[u], x);
        extremes(next[u], x, hi, lo);
        if (i0 + u + U < mine) load(seg + U, next[u]);
        if (bounds) {
          const uint32_t b = __float_as_uint(hi);
          bounds[seg * 32 + lane] = (uint16_t)(((b & 0x80000000u) ? b : b + 0xffffu) >> 16);
        }
        if (__any_sync(0xffffffffu, lo == kNegInf)) {
#pragma unroll
          for (int j = 0; j < kPer; ++j) gone += x[j] == kNegInf;
        }
        const float top = warp_max(hi);
        float g = 0.f;
        if (top >= tm && top > kNegInf) {
          if (top > tm) {
            s = (s + n) * ex2((tm - top) * c);
            n = 0.f;
            tm = top;
          }
#pragma unroll
          for (int j = 0; j < kPer; ++j) {
            if (x[j] == tm)
              n += 1.f;
            else
              g += ex2((x[j] - tm) * c);
          }
        } else {
          const float ref = fmaxf(tm, kLowest);
#pragma unroll
          for (int j = 0; j < kPer; ++j) g += ex2((x[j] - ref) * c);
        }
        s += g;
      }
    }
    const double ws = warp_sum((double)s), wn = warp_sum((double)n);
    gone = __reduce_add_sync(0xffffffffu, gone);
    if (lane == 0) {
      sh->warp_m[warp] = tm;
      sh->warp_a[warp] = ws;
      sh->warp_b[warp] = wn;
      sh->warp_n[warp] = (uint32_t)gone;
    }
    __syncthreads();
    combine(kWarps, sh->warp_m[lane & (kWarps - 1)], sh->warp_a[lane & (kWarps - 1)], sh->warp_b[lane & (kWarps - 1)], m, rest);
    masked = __reduce_add_sync(0xffffffffu, lane < kWarps ? (int)sh->warp_n[lane & (kWarps - 1)] : 0);
    if (blocks > 1) {
      tell(rest, m, masked);
      const Slot o = told(lane & (blocks - 1));
      combine(blocks, o.m, o.a, 1.0, m, rest);
      masked = __reduce_add_sync(0xffffffffu, lane < blocks ? o.i : 0);
    }
    masked -= all_segs * 32 * kPer - V;  // what lies outside the row
    if (threadIdx.x < kWarps) {
      const float mi = sh->warp_m[threadIdx.x];
      sh->chunk[threadIdx.x] = mi > kNegInf ? (sh->warp_a[threadIdx.x] + sh->warp_b[threadIdx.x]) * exp2(((double)mi - (double)m) * (double)c) : 0.0;
    }
    __syncthreads();
  }
  // The largest and the least of a granule; those of 16 bits two at a time.
  __device__ __forceinline__ static void extremes(const uint32_t (&w)[8], const float (&x)[kPer], float &hi, float &lo) {
    if constexpr (sizeof(T) == 4) {
      hi = x[0], lo = x[0];
#pragma unroll
      for (int j = 1; j < kPer; ++j) hi = fmaxf(hi, x[j]), lo = fminf(lo, x[j]);
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
        v = mi > kNegInf ? (a + b) * exp2(((double)mi - (double)mm) * (double)c) : a;
    }
    m_out = mm;
    rest = warp_sum(v);
  }
  // How far the float32 sums of stats() can be off, relative to the whole.  A term 2^a: a passes three roundings of 2^-24 of
  // itself; terms below 2^-32 of the largest hold 2^-32 V of the whole at most, so |a| counts with less than 33, 33 * 3 ln 2 = 69 times
  // 2^-24; the exponential 4 times, and a lane's chain of additions of kPer + the granules that it takes, and ten beside it.
  __device__ __forceinline__ double eps() const { return (double)(90 + kPer + (all_segs / (blocks * kWarps) + 2)) * 5.9604644775390625e-08; }

  // Calls f(x, i0) for the warp's pieces, each lane with its granule (-inf in those that hold nothing from `floor` on).  f is
  // called by whole warps.
  template <typename F>
  __device__ __forceinline__ void sweep(float floor, F f) const {
    constexpr int U = 2;
    for (int i0 = 0; i0 < mine; i0 += U) {
      uint32_t w[U][8];
      bool any[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int seg = first + i0 + u;
        const bool hot = i0 + u < mine && (!bounds || __uint_as_float((uint32_t)bounds[seg * 32 + lane] << 16) >= floor);
        any[u] = __any_sync(0xffffffffu, hot);
        if (hot) {
          load(seg, w[u]);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) w[u][i] = std::is_same<T, float>::value ? 0xff800000u : std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u;
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!any[u]) continue;
        float x[kPer];
        widen<T>(w[u], x);
        f(x, first_of(first + i0 + u));
      }
    }
  }
  // Adds to `acc` the amounts, and to `n` the number, of a warp's granules' logits that `want` asks for, 32 side by side where they
  // are few: each lane by itself would form exponentials for one or two lanes at a time.
  template <bool kWeights, typename Want>
  __device__ __forceinline__ void add(const float (&x)[kPer], int i0, Want want, double &acc, int &n) const {
    unsigned mask = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) mask |= want(x[j], i0 + j) ? 1u << j : 0u;
    const int own = __popc(mask);
    n += own;
    if constexpr (kWeights) {
      const int all = __reduce_add_sync(0xffffffffu, own);
      if (all == 0) return;
      if (all <= kCompact) {
        float *to = sh->compact[warp];
        int at = warp_scan(own) - own;
#pragma unroll
        for (int j = 0; j < kPer; ++j)
          if (mask >> j & 1) to[at++] = x[j];
        __syncwarp();
        for (int i = lane; i < all; i += 32) acc += weight(to[i]);
        __syncwarp();
      } else {
#pragma unroll
        for (int j = 0; j < kPer; ++j)
          if (mask >> j & 1) acc += weight(x[j]);
      }
    }
  }
  // Leaves the warp's amounts in `chunk`; the block's number in all threads.
  template <bool kWeights>
  __device__ int end_of_sum(double acc, int n) {
    n = __reduce_add_sync(0xffffffffu, n);
    const double sum = kWeights ? warp_sum(acc) : (double)n;
    __syncthreads();  // chunk and warp_n have been read
    if (lane == 0) {
      sh->chunk[warp] = sum;
      sh->warp_n[warp] = (uint32_t)n;
    }
    __syncthreads();
    return __reduce_add_sync(0xffffffffu, lane < kWarps ? (int)sh->warp_n[lane & (kWarps - 1)] : 0);
  }
  // The sum of the warps' parts, the block's in a fixed order and the row's, with the row's number; tells the blocks both.
  __device__ __forceinline__ double sum_of_row(int n, int &all_n) {
    double v = warp_sum(lane < kWarps ? sh->chunk[lane & (kWarps - 1)] : 0.0);
    all_n = n;
    if (blocks > 1) {
      tell(v, 0.f, n);
      const Slot o = told(lane & (blocks - 1));
      v = warp_sum(lane < blocks ? o.a : 0.0);
      all_n = __reduce_add_sync(0xffffffffu, lane < blocks ? o.i : 0);
    }
    return v;
  }
  // The sum of the weights that `want` asks for, in double.
  template <typename Want>
  __device__ double sum_of(float floor, Want want, int &all_n) {
    double acc = 0.0;
    int n = 0;
    sweep(floor, [&](const float (&x)[kPer], int i0) { add<true>(x, i0, want, acc, n); });
    n = end_of_sum<true>(acc, n);
    return sum_of_row(n, all_n);
  }
  // The whole row's.
  __device__ double whole() {
    int n;
    return sum_of(kLowest, [](float x, int) { return x > kNegInf; }, n);
  }

  // The first index of the maximum.
  __device__ int first_of_max() {
    int best = kNoIndex;
    sweep(m, [&](const float (&x)[kPer], int i0) {
#pragma unroll
      for (int j = kPer - 1; j >= 0; --j)
        if (x[j] == m) best = min(best, i0 + j);
    });
    best = __reduce_min_sync(0xffffffffu, best);
    __syncthreads();
    if (lane == 0) sh->warp_n[warp] = (uint32_t)best;
    __syncthreads();
    best = __reduce_min_sync(0xffffffffu, lane < kWarps ? (int)sh->warp_n[lane & (kWarps - 1)] : kNoIndex);
    if (blocks > 1) {
      tell(0.0, 0.f, best);
      best = __reduce_min_sync(0xffffffffu, told(lane & (blocks - 1)).i);
    }
    return best;
  }

  // The index at which the running sum over the row passes `aim`, where the warps' parts lie in `chunk` and the blocks' have been told
  // (sum_of_row): the first in `want` where it does, or the last of those with something where rounding leaves none.  Known to
  // the block that has it alone; the others get -2.  `unsure`: how far the running sums may be off; then the answer is
  // kNoIndex where that matters, known to all.
  template <bool kWeights, typename Want>
  __device__ int find(double aim, Want want, double unsure = 0.0) {
    const auto amount = [&](float x) { return kWeights ? weight(x) : 1.0; };
    int owner = 0;
    double before = 0.0;
    if (blocks > 1) {
      const double part = lane < blocks ? told(lane & (blocks - 1)).a : 0.0, up_to = warp_scan(part);
      const unsigned passes = __ballot_sync(0xffffffffu, lane < blocks && up_to > aim && part > 0.0);
      const unsigned any = __ballot_sync(0xffffffffu, part > 0.0);
      owner = passes ? __ffs(passes) - 1 : 31 - __clz(any);
      before = __shfl_sync(0xffffffffu, up_to - part, owner);
    }
    int at = -2;
    if (owner == rank) {
      // the warp whose part it is
      const double part = lane < kWarps ? sh->chunk[lane & (kWarps - 1)] : 0.0, up_to = warp_scan(part);
      const unsigned passes = __ballot_sync(0xffffffffu, lane < kWarps && before + up_to > aim && part > 0.0);
      const unsigned any = __ballot_sync(0xffffffffu, part > 0.0);
      const int of_warp = passes ? __ffs(passes) - 1 : 31 - __clz(any);
      double run = before + __shfl_sync(0xffffffffu, up_to - part, of_warp);
      const int per = (segs + kWarps - 1) / kWarps, s0 = of_warp * per, s1 = min(segs, s0 + per);
      // its pieces' sums, by all warps, kSegs at a time
      int piece = -1, last = -1;
      double run_last = run;
      for (int p0 = s0; p0 < s1 && piece < 0; p0 += kSegs) {
        const int p1 = min(s1, p0 + kSegs);
        __syncthreads();
        for (int seg = p0 + warp; seg < p1; seg += kWarps) {
          uint32_t w[8];
          load(seg, w);
          float x[kPer];
          widen<T>(w, x);
          const int i0 = first_of(seg);
          double g = 0.0;
#pragma unroll
          for (int j = 0; j < kPer; ++j)
            if (want(x[j], i0 + j)) g += amount(x[j]);
          g = warp_sum(g);
          if (lane == 0) sh->seg[seg - p0] = g;
        }
        __syncthreads();
        // every warp alike
        for (int q = p0; q < p1 && piece < 0; q += 32) {
          const double part = q + lane < p1 ? sh->seg[q + lane - p0] : 0.0, up = warp_scan(part);
          const unsigned hit = __ballot_sync(0xffffffffu, run + up > aim && part > 0.0), some = __ballot_sync(0xffffffffu, part > 0.0);
          const int who = hit ? __ffs(hit) - 1 : some ? 31 - __clz(some) : -1;
          if (who >= 0) {
            last = q + who;
            run_last = run + __shfl_sync(0xffffffffu, up - part, who);
            if (hit) piece = last;
          }
          run += __shfl_sync(0xffffffffu, up, 31);
        }
      }
      bool clear = piece >= 0;
      // the granule, then the logit: a lane each
      run = run_last;
      last = max(last, s0);
      uint32_t w[8];
      load(last, w);
      float x[kPer];
      widen<T>(w, x);
      int i0 = first_of(last);
      double g = 0.0;
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (want(x[j], i0 + j)) g += amount(x[j]);
      double up = warp_scan(g);
      unsigned hit = __ballot_sync(0xffffffffu, run + up > aim && g > 0.0);
      unsigned some = __ballot_sync(0xffffffffu, g > 0.0);
      int who = max(0, hit ? __ffs(hit) - 1 : 31 - __clz(some));
      clear = clear && hit;
      run += __shfl_sync(0xffffffffu, up - g, who);
      i0 = __shfl_sync(0xffffffffu, i0, who);
      const int i = i0 + lane;
      const float v = lane < kPer && i >= 0 && i < V ? Storage<T>::widen(z[i]) : kNegInf;
      g = v > kNegInf && want(v, i) ? amount(v) : 0.0;
      up = warp_scan(g);
      hit = __ballot_sync(0xffffffffu, run + up > aim && g > 0.0);
      some = __ballot_sync(0xffffffffu, g > 0.0);
      who = max(0, hit ? __ffs(hit) - 1 : 31 - __clz(some));
      const double low = run + __shfl_sync(0xffffffffu, up - g, who), high = run + __shfl_sync(0xffffffffu, up, who);
      at = min(max(i0 + who, 0), V - 1);
      if (unsure > 0.0 && !(clear && hit && low + unsure <= aim && high - unsure > aim)) at = kNoIndex;
    }
    if (unsure > 0.0 && blocks > 1) {
      tell(0.0, 0.f, at);
      if (told(owner).i == kNoIndex) return kNoIndex;
    }
    return at;
  }
  // find(), known to all blocks.
  template <bool kWeights, typename Want>
  __device__ int find_for_all(double aim, Want want) {
    int at = find<kWeights>(aim, want);
    if (blocks > 1) {
      tell(0.0, 0.f, at);
      at = __reduce_max_sync(0xffffffffu, told(lane & (blocks - 1)).i);
    }
    return at;
  }

  // ---- 2: the cut
  // Logits in the order of the row lie in bins by their distance from the maximum; the last bin has all from kBins - 1 on.
  __device__ __forceinline__ int bin_of(float x, float per) const {
    return min(kBins - 1, __float2int_rz(fminf(fminf(m - x, -kLowest) * per, 1e9f)));
  }

  // A lower bound of the k-th largest logit from the granules' maxima: where k granules reach up to a value, k logits do.
  __device__ float floor_of(long long k) {
    float low = cut_v;
    const int n = segs * 16;  // pairs
    if (bounds && k <= 2 * n) {
      if (threadIdx.x < 3) sh->counter[threadIdx.x] = 0;
      __syncthreads();
      const uint32_t *pairs = reinterpret_cast<const uint32_t *>(bounds);
      uint32_t lo = 0, hi = 0xffff;  // of the order: the largest b that k bounds reach
      for (int round = 0; lo < hi; ++round) {
        const uint32_t mid = (lo + hi + 1) >> 1;
        // of the order, and so of the values: bounds of the least such value and above
        const float v = value_of(mid << 16 | (mid & 0x8000u ? 0u : 0xffffu));
        int reach = 0;
        for (int i = threadIdx.x; i < n; i += kThreads) {
          const uint32_t two = pairs[i];
          reach += (__uint_as_float(two << 16) >= v) + (__uint_as_float(two & 0xffff0000u) >= v);
        }
        reach = __reduce_add_sync(0xffffffffu, reach);
        // three counters in turn: one is added to, one is read, one is cleared for the next
        if (lane == 0 && reach) atomicAdd(&sh->counter[round % 3], (uint32_t)reach);
        if (threadIdx.x == 0) sh->counter[(round + 1) % 3] = 0;
        __syncthreads();
        if ((long long)sh->counter[round % 3] >= k)
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

  // Moves the cut to the last logit, in falling order, before which less than share * all lies; kWeights: sums of weights, else
  // of ones.  Logits below `floor` are known to lie behind it.  `all`: the amount in the whole row, good to `unsure`, of which at
  // most `below` lies below `floor`.  Returns whether the weights of what is kept lie in `chunk` and their number in `n`.
  template <bool kWeights>
  __device__ bool select(double share, double all, double unsure, float floor, double below, int &n_kept) {
    const auto amount = [&](float x) { return kWeights ? weight(x) : 1.0; };
    double aim = share * all;
    const float span = floor > 0.5f * kLowest ? m - floor : (float)(40.0 / inv_t);
    const float most = (float)(kBins - 2) / span, per = span > 0.f && most < 1e30f ? most : 0.f;  // 0: all in one bin
    // level 0: bins of distance; from level 1 on logits from `low` to `high`, in bins by their keys
    float low = floor, high = m;
    uint32_t n_in = 0;
    // every level divides the keys by 2,048, at the latest from the eighth on: eleven are the most
    for (int level = 0; level < 16; ++level) {
      const uint32_t k_lo = key_of(low), k_hi = key_of(high), width = k_hi - k_lo;
      const int shift = max(0, 21 - __clz(width));  // (width >> shift) < kBins
      const bool gather = level > 0 && n_in <= kList;
      // where the bracket has one value, its logits are taken by their index
      const bool ties = level > 0 && !gather && width == 0;
      if (level == 2 && !gather && unsure > 0.0) {  // a flat row: bins of single values want the aim itself
        all = whole();
        aim = share * all;
        unsure = 0.0;
      }
      __syncthreads();
      if (!gather)
        for (int i = threadIdx.x; i < kBins; i += kThreads) sh->hist[i] = 0;
      if (threadIdx.x == 0) sh->list_n = 0;
      __syncthreads();
      double above = 0.0;
      int n_above = 0, n_block = 0;
      if (level == 0) {
        sweep(low, [&](const float (&x)[kPer], int i0) {
#pragma unroll
          for (int j = 0; j < kPer; ++j)
            if (x[j] >= low && kept(x[j], i0 + j)) atomicAdd(&sh->hist[bin_of(x[j], per)], 1u);
        });
        meet();
      } else {
        // the amount in front of the bracket, and the bracket's logits in bins or in the list
        double acc = 0.0;
        sweep(low, [&](const float (&x)[kPer], int i0) {
          // what is cut already lies at the bracket's end or behind it
          add<kWeights>(x, i0, [&](float v, int) { return v > high; }, acc, n_block);
          if (ties) return;
#pragma unroll
          for (int j = 0; j < kPer; ++j) {
            if (!(x[j] >= low && x[j] <= high && kept(x[j], i0 + j))) continue;
            if (gather) {
              const uint32_t at = atomicAdd(&sh->list_n, 1u);
              if (at < kList) sh->list[at] = (uint64_t)(~key_of(x[j])) << 32 | (uint32_t)(i0 + j);
            } else {
              atomicAdd(&sh->hist[(k_hi - key_of(x[j])) >> shift], 1u);
            }
          }
        });
        n_block = end_of_sum<kWeights>(acc, n_block);
        above = sum_of_row(n_block, n_above);
      }
      if (ties) {
        // kept are the first r with above + (r - 1) w < aim
        const double w = amount(high);
        const auto number = [&](double to) {
          double r = fmin((double)n_in, fmax(1.0, ceil((to - above) / w)));
          if (r > 1.0 && !(above + (r - 1.0) * w < to))
            r -= 1.0;
          else if (r < (double)n_in && above + r * w < to)
            r += 1.0;
          return r;
        };
        double r = number(aim);
        if (unsure > 0.0 && number(share * (all - unsure)) != number(share * (all + unsure))) r = number(share * whole());
        const auto tie = [&](float x, int i) { return x == high && kept(x, i); };
        double acc = 0.0;
        int n = 0, row_n;
        sweep(high, [&](const float (&x)[kPer], int i0) { add<false>(x, i0, tie, acc, n); });
        n = end_of_sum<false>(acc, n);
        sum_of_row(n, row_n);
        const int at = find_for_all<false>(r - 0.5, tie);
        cut_v = high;
        cut_i = at;
        return false;
      }
      if (gather) {
        // all blocks' lists in one, alike in every block
        int n = 0;
        if (blocks == 1) {
          n = (int)sh->list_n;
          if (n <= kList)
            for (int i = threadIdx.x; i < n; i += kThreads) sh->sorted[i] = sh->list[i];
        } else {
          for (int r = 0; r < blocks; ++r) {
            const Shared *o = of(r);
            const int k = (int)o->list_n;
            if (n + k <= kList)
              for (int i = threadIdx.x; i < k; i += kThreads) sh->sorted[n + i] = o->list[i];
            n += k;
          }
          meet();  // the lists have been read
        }
        if (n > kList) {  // more on the bracket's edge than its bins had
          n_in = (uint32_t)n;
          continue;
        }
        sort_list(n);
        int last;
        double list_sum;
        if (!cut_from_list<kWeights>(n, aim, share * unsure, above, last, list_sum)) {
          // the float32 sum is not enough: what lies behind the bracket in float32 again, beside the rest in double, mostly is
          const double tail = behind(low);
          if (!cut_from_list<kWeights>(n, share * (above + list_sum + tail), 4.0 * share * tail * eps() /* exponents of up to 126 */,
                                       above, last, list_sum)) {
            // the sum of what is above is in `chunk` no more
            const double exact = whole();
            cut_from_list<kWeights>(n, share * exact, 0.0, above, last, list_sum);
            set_cut(last);
            return false;
          }
        }
        set_cut(last);
        if (!kWeights) return false;
        // the list's kept logits to the warps that have their pieces
        const int each = (segs + kWarps - 1) / kWarps;
        const int lo_i = (seg0 + warp * each) * 32 * kPer - off, hi_i = (seg0 + min(segs, (warp + 1) * each)) * 32 * kPer - off;
        double acc = 0.0;
        for (int i = lane; i <= last; i += 32) {
          const uint64_t item = sh->sorted[i];
          const int at = (int)(uint32_t)item;
          if (at >= lo_i && at < hi_i) acc += weight(value_of(~(uint32_t)(item >> 32)));
        }
        acc = warp_sum(acc);
        if (lane == 0) sh->chunk[warp] += acc;
        n_kept = n_above + last + 1;
        __syncthreads();
        return true;
      }
      bracket<kWeights>(level, aim, above, all, share * unsure, below, unsure, per, k_lo, k_hi, shift);
      const uint32_t lo = sh->pick_lo, hi = sh->pick_hi;
      n_in = sh->pick_last;
      meet();  // the histograms have been read
      if (n_in == 0) return false;  // less than the aim in all: everything stays
      if (level == 0) {
        // the values that the bins' logits can have; 2^-20 covers the roundings of the distance
        const double slack = 9.5367431640625e-7;
        if (per > 0.f) {
          high = fminf(m, __double2float_ru((double)m - (double)lo / per * (1.0 - slack)));
          if (hi < kBins - 1) low = fmaxf(low, __double2float_rd((double)m - ((double)hi + 1.0) / per * (1.0 + slack)));
        }
      } else {
        low = fmaxf(low, value_of(edge_of(k_lo, k_hi, hi, shift)));
        high = value_of(k_hi - (lo << shift));
      }
    }
    return false;
  }
  __device__ __forceinline__ void set_cut(int last) {
    const uint64_t item = sh->sorted[last];
    cut_v = value_of(~(uint32_t)(item >> 32));
    cut_i = (int)(uint32_t)item;
  }
  // The float32 sum of the weights of logits below `low`, of a row that nothing is cut from.  Leaves `chunk` alone.
  __device__ double behind(float low) {
    float s = 0.f;
    sweep(kLowest, [&](const float (&x)[kPer], int) {
      float g = 0.f;
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (x[j] < low) g += ex2((x[j] - m) * c);
      s += g;
    });
    const double ws = warp_sum((double)s);
    __syncthreads();
    if (lane == 0) sh->warp_a[warp] = ws;
    __syncthreads();
    double own = warp_sum(lane < kWarps ? sh->warp_a[lane & (kWarps - 1)] : 0.0);
    if (blocks > 1) {
      tell(own, 0.f, 0);
      own = warp_sum(lane < blocks ? told(lane & (blocks - 1)).a : 0.0);
    }
    return own;
  }

  // The least key of bin b, of keys from k_lo to k_hi: bin 0 has the largest.
  __device__ __forceinline__ static uint32_t edge_of(uint32_t k_lo, uint32_t k_hi, uint32_t b, int shift) {
    const int64_t least = (int64_t)k_hi - (int64_t)(((uint64_t)b + 1) << shift) + 1;
    return least > (int64_t)k_lo ? (uint32_t)least : k_lo;
  }

  // Which of the histograms' bins can hold the cut, whose aim is good to `unsure`: pick_lo to pick_hi, which have pick_last logits (0:
  // all of it lies in front of the aim).  Every block alike.
  template <bool kWeights>
  __device__ void bracket(int level, double aim, double above, double all, double unsure, double below, double all_unsure, float per,
                          uint32_t k_lo, uint32_t k_hi, int shift) {
    constexpr int kOwn = kBins / kThreads;
    // where a bin holds one value, or the bracket would not get smaller, the larger bound decides
    const bool sharp = !kWeights || level >= 8 || (level > 1 && shift == 0);
    uint32_t n[kOwn], n_sum = 0;
    double least[kOwn], most[kOwn], least_sum = 0.0, most_sum = 0.0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) n[j] = sh->hist[threadIdx.x * kOwn + j];
    for (int r = 1; r < blocks; ++r) {
      const Shared *o = of((rank + r) & (blocks - 1));
#pragma unroll
      for (int j = 0; j < kOwn; ++j) n[j] += o->hist[threadIdx.x * kOwn + j];
    }
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const uint32_t b = threadIdx.x * kOwn + j;
      least[j] = most[j] = (double)n[j];
      if (kWeights && n[j]) {
        double far, near;  // the bin's distances from the maximum
        if (level == 0) {
          const double slack = 9.5367431640625e-7;
          near = per > 0.f ? (double)b / per * (1.0 - slack) : 0.0;
          far = b == kBins - 1 || per == 0.f ? __longlong_as_double(0x7ff0000000000000LL) : ((double)b + 1.0) / per * (1.0 + slack);
        } else {
          near = (double)m - (double)value_of(k_hi - (b << shift));
          far = (double)m - (double)value_of(edge_of(k_lo, k_hi, b, shift));
        }
        most[j] *= exp(-near * inv_t);
        least[j] = sharp ? most[j] : least[j] * exp(-far * inv_t);
      }
      n_sum += n[j];
      least_sum += least[j];
      most_sum += most[j];
    }
    const uint32_t n_up = warp_scan(n_sum);
    const double least_up = warp_scan(least_sum), most_up = warp_scan(most_sum);
    __syncthreads();
    if (lane == 31) {
      sh->warp_n[warp] = n_up;
      sh->warp_a[warp] = least_up;
      sh->warp_b[warp] = most_up;
    }
    if (threadIdx.x == 0) {
      sh->pick_lo = kBins;   // the first bin up to which there can be as much as the aim
      sh->pick_hi = kBins;   // the first up to which there is
      sh->pick_last = 0;     // the last that holds anything
    }
    __syncthreads();
    double least_run = above + least_up - least_sum, most_run = above + most_up - most_sum, least_all = above, most_all = above + below;
    for (int w = 0; w < kWarps; ++w) {
      const double a = sh->warp_a[w], b = sh->warp_b[w];
      if (w < warp) {
        least_run += a;
        most_run += b;
      }
      least_all += a;
      most_all += b;
    }
    // A bin's edges bound its weights to a percent or so.  Over the whole row (level 0) the bounds on what lies behind a bin,
    // taken from the known whole, are the closer ones where the aim is near it: 1.5 % of the last twentieth for a top_p of 0.95
    const double eps = sharp ? 0.0 : 1e-11 * all + unsure;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const uint32_t b = threadIdx.x * kOwn + j;
      least_run += least[j];
      most_run += most[j];
      if (!n[j]) continue;
      atomicMax(&sh->pick_last, b);
      double high = most_run, low = sharp ? most_run : least_run;
      if (!sharp && level == 0) {
        high = fmin(high, all + all_unsure - (least_all - least_run));
        low = fmax(low, all - all_unsure - (most_all - most_run));
      }
      if (high >= aim - eps) atomicMin(&sh->pick_lo, b);
      if (low >= aim + eps) atomicMin(&sh->pick_hi, b);
    }
    __syncthreads();
    uint32_t lo = sh->pick_lo, hi = min(sh->pick_hi, (uint32_t)kBins - 1);
    if (level > 0 && lo == kBins) lo = hi = sh->pick_last;  // the cut is in the bracket: what is missing is a rounding
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
      sh->pick_lo = lo;
      sh->pick_hi = hi;
      sh->pick_last = 0;
    }
    __syncthreads();
    if (lane == 0 && inside) atomicAdd(&sh->pick_last, inside);
    __syncthreads();
  }

  // Sorts the n items of `sorted`: falling logits, rising indices.
  __device__ void sort_list(int n) {
    int size = 32;
    while (size < n) size <<= 1;
    for (int i = n + threadIdx.x; i < size; i += kThreads) sh->sorted[i] = ~0ull;
    __syncthreads();
    for (int k = 2; k <= size; k <<= 1)
      for (int j = k >> 1; j > 0; j >>= 1) {
        for (int t = threadIdx.x; t < size / 2; t += kThreads) {
          const int a = (t & ~(j - 1)) * 2 + (t & (j - 1)), b = a + j;
          const uint64_t x = sh->sorted[a], y = sh->sorted[b];
          if ((x > y) == ((a & k) == 0)) {
            sh->sorted[a] = y;
            sh->sorted[b] = x;
          }
        }
        __syncthreads();
      }
  }
  // The last of the sorted list before which less than the aim lies; returns whether that is so for every aim within `unsure`.
  template <bool kWeights>
  __device__ bool cut_from_list(int n, double aim, double unsure, double above, int &last, double &list_sum) {
    constexpr int kOwn = kList / kThreads;
    double w[kOwn], sum = 0.0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const int i = threadIdx.x * kOwn + j;
      w[j] = i < n ? kWeights ? weight(value_of(~(uint32_t)(sh->sorted[i] >> 32))) : 1.0 : 0.0;
      sum += w[j];
    }
    const double up_to = warp_scan(sum);
    __syncthreads();
    if (lane == 31) sh->warp_a[warp] = up_to;
    if (threadIdx.x == 0) {
      sh->pick_last = 0;
      sh->unclear = 0;
    }
    __syncthreads();
    double run = above + up_to - sum, all = 0.0;
    for (int v = 0; v < kWarps; ++v) {
      const double a = sh->warp_a[v];
      if (v < warp) run += a;
      all += a;
    }
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const int i = threadIdx.x * kOwn + j;
      if (i < n && (run < aim || i == 0)) atomicMax(&sh->pick_last, (uint32_t)i);
      // the bracket holds the cut: its first logit is kept, and its end is behind the aim
      if (unsure > 0.0 && i < n && i > 0 && fabs(run - aim) <= unsure) sh->unclear = 1;
      run += w[j];
      if (unsure > 0.0 && i == n - 1 && run - aim <= unsure) sh->unclear = 1;
    }
    __syncthreads();
    last = (int)sh->pick_last;
    list_sum = all;
    return sh->unclear == 0;
  }
};

template <typename T>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const Params p) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Row<T> row;
  row.sh = reinterpret_cast<Shared *>(smem_raw);
  row.bounds = p.bounds ? reinterpret_cast<uint16_t *>(smem_raw + sizeof(Shared)) : nullptr;
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

  if (threadIdx.x < kTable) row.sh->table[threadIdx.x] = exp2((double)threadIdx.x / kTable);
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
      id = row.first_of_max();
      count = 1;
    } else {
      const auto kept = [&](float x, int i) { return row.kept(x, i); };
      bool whole = row.cut_v == kLowest;  // nothing is cut: the sums of the first sweep are those of what is kept
      bool have = false;                  // the sums of what is kept lie in `chunk`
      if (top_k > 0 && top_k < p.V - masked) {
        row.template select<false>(1.0, (double)top_k, 0.0, row.floor_of(top_k), 0.0, count);
        whole = false;
      }
      if (top_p < 1.0) {
        const double all = whole ? rest + 1.0 : row.sum_of(row.cut_v, kept, count), unsure = whole ? row.eps() * all : 0.0;
        // logits whose weight is under a V-th of 0.03 (1 - top_p) of the whole hold less than that much together
        const double below = 0.03 * (1.0 - top_p) * all;
        const float floor = __double2float_rd((double)row.m + temperature * log(below / (double)p.V));
        have = row.template select<true>(top_p, all, unsure, fmaxf(row.cut_v, floor), below * 1.001, count);
        whole = false;
      }
      double all;
      if (whole) {
        // by the warps' float32 sums, unless the border is too near for them
        int n;
        all = row.sum_of_row(0, n);
        id = row.template find<true>((double)u * all, kept, 2.0 * row.eps() * all);
        count = (int)p.V - masked;
      }
      if (!whole || id == kNoIndex) {
        if (have) {
          int n;
          all = row.sum_of_row(0, n);
        } else {
          all = row.sum_of(row.cut_v, kept, count);
        }
        id = row.template find<true>((double)u * all, kept);
      }
      kept_rest = whole ? rest : all - 1.0;
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
    if (p.logp) p.logp[t] = id >= 0 ? (float)(x - log1p(rest)) : nan;
    if (p.logp_mp) p.logp_mp[t] = id >= 0 ? (float)(x - log1p(kept_rest)) : nan;
    if (p.count) p.count[t] = count;
  }
  if (row.blocks > 1) row.meet();  // nobody leaves while its shared memory is read
}

// ---- host --------------------------------------------------------------------------------------------------------------

// Blocks that share a row: as many as the chip has room for beside the other rows, while each has work.
inline int choose_blocks(long long T, long long row_bytes) {
  int log_blocks = 0;
  while (log_blocks < 3 && (T << (log_blocks + 1)) <= 296 && (row_bytes >> (log_blocks + 1)) >= 16 * 1024) ++log_blocks;
  return log_blocks;
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
  const size_t smem = sizeof(Shared) + (size_t)p.bounds * 2;
  auto kernel = sample_kernel<T>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(sizeof(Shared) + kMostBounds * 2));
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
           a->top_k, a->ids, a->logp, a->logp_mp, a->count, a->T, a->V, a->ld, a->id_dtype == DVP_ID_I32, 0, 0};
  const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
  const cudaError_t e = a->logits_dtype == DVP_F32    ? launch<float>(a, p, stream)
                        : a->logits_dtype == DVP_BF16 ? launch<__nv_bfloat16>(a, p, stream)
                                                      : launch<__half>(a, p, stream);
  return e == cudaSuccess ? DVP_OK : DVP_ERR_CUDA;
}
