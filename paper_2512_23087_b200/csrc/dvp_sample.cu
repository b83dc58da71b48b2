// Sampling: one token per row of logits, from the min-p safe set, the top_k largest of it and of these the fewest that hold top_p
// of their mass, at a temperature, by a given random number.
//
// Every one of the three filters keeps the front of the row in falling order (equal logits by index), so what is kept is one
// cut: the logits above a value `v` and, of those equal to it, the ones up to an index.  Nothing is sorted but a few hundred
// logits around the cut:
//
//   1  the row streams past once: its maximum, the sum of e^{(z - m) / T} without the maximum's own terms (so that ln of the whole
//      sum keeps its digits where one token has all the mass), and the maximum of each 32-byte granule, which stays in shared
//      memory.  What follows reads only the granules that can matter, from L2
//   2  for each of top_k and top_p: a histogram of the logits' distances from the maximum (whole numbers: the order of the
//      additions does not matter) brackets the cut, the logits in the bracket go to a list in shared memory that is sorted, and
//      the cut is where the running sum, in double, passes its aim.  A bracket too full for the list is cut again by the logits'
//      bits, down to a single value if need be
//   3  sums in double of what is kept, in the order of the indices, piece by piece; the piece in which the running sum passes
//      u times the whole is walked to the token
//
// Decisions rest on sums in double: which token falls on which side of a border does not depend on how the row is divided
// among threads and blocks.  With few rows the blocks of a cluster share a row and exchange sums through shared memory.
#include <cmath>
#include <type_traits>

#include "dvp_common.cuh"

namespace dvp {
namespace sample {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kEntries = 1024;  // pieces of a block's part of the row, whole warps' loads, that have a sum of their own
constexpr int kBins = 2048, kList = 2048;
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

struct Shared {
  double entry[kEntries];
  uint64_t list[kList];
  uint32_t hist[kBins];
  double warp_a[kWarps], warp_b[kWarps];
  float warp_m[kWarps];
  uint32_t warp_n[kWarps];
  // read and written by the other blocks of the row
  double part_a, part_b;
  float part_m;
  int part_i;
  uint32_t list_n;
  double pick_a;
  uint32_t pick_lo, pick_hi, pick_n;
  float cut_v;
  int cut_i;
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

template <typename T>
struct Row {
  static constexpr int kPer = 32 / sizeof(T);  // logits of a granule
  Shared *sh;
  uint16_t *bounds;  // bfloat16, rounded up; NULL: none
  const T *z;
  int V, off;     // logits of the first granule that lie in front of the row
  int seg0, segs;  // the block's pieces of 32 granules
  int log_q, entries;  // pieces of an entry (2^log_q); entries
  int blocks, rank;
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
  __device__ __forceinline__ Shared *of(int r) const {
    return static_cast<Shared *>(__cluster_map_shared_rank(sh, (unsigned)r));
  }

  __device__ __forceinline__ int first_of(int seg) const { return ((seg0 + seg) * 32 + lane) * kPer - off; }
  __device__ __forceinline__ void load(int seg, float (&x)[kPer]) const {
    const int at = first_of(seg);
    if (at >= 0 && at + kPer <= V) {
      uint32_t w[8];
      ld_stream32(z + at, w);
      Storage<T>::unpack(make_uint4(w[0], w[1], w[2], w[3]), x);
      Storage<T>::unpack(make_uint4(w[4], w[5], w[6], w[7]), x + kPer / 2);
    } else {
#pragma unroll
      for (int j = 0; j < kPer; ++j) x[j] = at + j >= 0 && at + j < V ? Storage<T>::widen(z[at + j]) : kNegInf;
    }
  }
  __device__ __forceinline__ double weight(float x) const { return exp(((double)x - (double)m) * inv_t); }
  __device__ __forceinline__ bool kept(float x, int i) const { return x > cut_v || (x == cut_v && i <= cut_i); }

  // ---- 1: the maximum, the sum beside it
  // Lanes of a warp share the maximum that they have met, so that a larger one, which they turn to together, is rare.
  __device__ void stats(double &rest) {
    float tm = kNegInf, s = 0.f, n = 0.f;  // terms: n of e^0, and s
    const int mine = entries > warp ? ((entries - 1 - warp) / kWarps + 1) << log_q : 0;
    constexpr int U = 2;
    for (int i0 = 0; i0 < mine; i0 += U) {
      float x[U][kPer];
      int seg[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u;
        seg[u] = ((warp + (i >> log_q) * kWarps) << log_q) + (i & ((1 << log_q) - 1));
        if (i < mine && seg[u] < segs) {
          load(seg[u], x[u]);
        } else {
          seg[u] = -1;
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (seg[u] < 0) continue;
        float hi = kNegInf;
#pragma unroll
        for (int j = 0; j < kPer; ++j) hi = fmaxf(hi, x[u][j]);
        if (bounds) {
          const uint32_t b = __float_as_uint(hi);
          bounds[seg[u] * 32 + lane] = (uint16_t)(((b & 0x80000000u) ? b : b + 0xffffu) >> 16);
        }
        const float top = warp_max(hi);
        if (top >= tm && top > kNegInf) {
          if (top > tm) {
            s = (s + n) * ex2((tm - top) * c);
            n = 0.f;
            tm = top;
          }
#pragma unroll
          for (int j = 0; j < kPer; ++j) {
            if (x[u][j] == tm)
              n += 1.f;
            else
              s += ex2((x[u][j] - tm) * c);
          }
        } else {
          const float ref = fmaxf(tm, kLowest);
#pragma unroll
          for (int j = 0; j < kPer; ++j) s += ex2((x[u][j] - ref) * c);
        }
      }
    }
    const double ws = warp_sum((double)s), wn = warp_sum((double)n);
    if (lane == 0) {
      sh->warp_m[warp] = tm;
      sh->warp_a[warp] = ws;
      sh->warp_b[warp] = wn;
    }
    __syncthreads();
    combine(kWarps, [&](int i, float &mi, double &a, double &b) {
      mi = sh->warp_m[i], a = sh->warp_a[i], b = sh->warp_b[i];
    }, m, rest);
    if (blocks > 1) {
      if (threadIdx.x == 0) {
        sh->part_m = m;
        sh->part_a = rest;
      }
      meet();
      combine(blocks, [&](int i, float &mi, double &a, double &b) {
        const Shared *o = of(i);
        mi = o->part_m, a = o->part_a, b = 1.0;
      }, m, rest);
    }
  }
  // Sums a + b e^0 against maxima of their own to one against the largest, which is left out once.
  template <typename Get>
  __device__ __forceinline__ void combine(int n, Get get, float &m_out, double &rest) const {
    float mm = kNegInf, mi;
    double a, b, sum = 0.0;
    for (int i = 0; i < n; ++i) {
      get(i, mi, a, b);
      mm = fmaxf(mm, mi);
    }
    bool left_out = false;
    for (int i = 0; i < n; ++i) {
      get(i, mi, a, b);
      if (mi == mm && mm > kNegInf) {
        if (!left_out) b -= 1.0;
        left_out = true;
        sum += a + b;
      } else if (mi > kNegInf) {
        sum += (a + b) * exp2(((double)mi - (double)mm) * (double)c);
      } else {
        sum += a;  // nothing, or NaN
      }
    }
    m_out = mm;
    rest = sum;
  }

  // Calls f(seg, x, i0) for the pieces of the warp's entries, each lane with its granule (-inf in those that hold nothing from
  // `floor` on), and end(entry) behind the last piece of each.  f and end are called by whole warps.
  template <typename F, typename End>
  __device__ __forceinline__ void sweep(float floor, F f, End end) const {
    for (int e = warp; e < entries; e += kWarps) {
      const int s0 = e << log_q, s1 = min(segs, s0 + (1 << log_q));
      for (int seg = s0; seg < s1; ++seg) {
        const bool hot = !bounds || __uint_as_float((uint32_t)bounds[seg * 32 + lane] << 16) >= floor;
        if (!__any_sync(0xffffffffu, hot)) continue;
        float x[kPer];
        if (hot) {
          load(seg, x);
        } else {
#pragma unroll
          for (int j = 0; j < kPer; ++j) x[j] = kNegInf;
        }
        f(x, first_of(seg));
      }
      end(e);
    }
  }

  // The first index of the maximum.
  __device__ int first_of_max() {
    int best = kNoIndex;
    sweep(m, [&](const float (&x)[kPer], int i0) {
#pragma unroll
      for (int j = kPer - 1; j >= 0; --j)
        if (x[j] == m) best = min(best, i0 + j);
    }, [](int) {});
    best = __reduce_min_sync(0xffffffffu, best);
    if (threadIdx.x == 0) sh->part_i = kNoIndex;
    __syncthreads();
    if (lane == 0) atomicMin(&sh->part_i, best);
    meet();
    for (int r = 0; r < blocks; ++r) best = min(best, of(r)->part_i);
    return best;
  }

  // Sums over the entries' sums: every entry the sum up to and with it; returns the block's.
  __device__ double scan_entries() {
    __syncthreads();
    const int i = 2 * threadIdx.x;
    const double a = i < entries ? sh->entry[i] : 0.0, b = i + 1 < entries ? sh->entry[i + 1] : 0.0;
    const double up_to = warp_scan(a + b);
    if (lane == 31) sh->warp_a[warp] = up_to;
    __syncthreads();
    double before = 0.0;
    for (int w = 0; w < warp; ++w) before += sh->warp_a[w];
    double all = before;
    for (int w = warp; w < kWarps; ++w) all += sh->warp_a[w];
    const double first = before + up_to - b;
    if (i < entries) sh->entry[i] = first;
    if (i + 1 < entries) sh->entry[i + 1] = before + up_to;
    __syncthreads();
    return all;
  }

  // The sum of f(x, i) over the row, in double and a fixed order; each entry's running sum stays in the block.
  template <typename F>
  __device__ double sum_of(float floor, F f, double *before_block = nullptr, double *block_sum = nullptr) {
    for (int e = threadIdx.x; e < entries; e += kThreads) sh->entry[e] = 0.0;
    __syncthreads();
    double acc = 0.0;
    sweep(floor, [&](const float (&x)[kPer], int i0) {
#pragma unroll
      for (int j = 0; j < kPer; ++j) acc += f(x[j], i0 + j);
    }, [&](int e) {
      if (!__any_sync(0xffffffffu, acc != 0.0)) return;
      const double s = warp_sum(acc);
      if (lane == 0) sh->entry[e] = s;
      acc = 0.0;
    });
    const double own = scan_entries();
    if (block_sum) *block_sum = own;
    if (blocks == 1) {
      if (before_block) *before_block = 0.0;
      return own;
    }
    if (threadIdx.x == 0) sh->part_a = own;
    meet();
    double all = 0.0;
    for (int r = 0; r < blocks; ++r) {
      if (r == rank && before_block) *before_block = all;
      all += of(r)->part_a;
    }
    meet();  // part_a may be written again
    return all;
  }

  // The first index at which the running sum of f passes `aim`; the last with f > 0 where none does.  Every thread of the
  // row has the answer.
  template <typename F>
  __device__ int locate(float floor, F f, double share, bool share_is_aim, double *total) {
    double before, own;
    const double all = sum_of(floor, f, &before, &own);
    if (total) *total = all;
    const double aim = share_is_aim ? share : share * all;
    // the block and the entry: the first that passes, or the last with anything
    if (threadIdx.x == 0) sh->part_i = -1;
    if (threadIdx.x == 0) sh->pick_n = 0;
    int owner = -1;
    {
      double run = 0.0;
      int last = 0;
      for (int r = 0; r < blocks; ++r) {
        const double s = blocks == 1 ? own : of(r)->part_a;
        run += s;
        if (s > 0.0) last = r;
        if (owner < 0 && run > aim) owner = r;
      }
      if (owner < 0) owner = last;
    }
    __syncthreads();
    if (owner == rank) {
      // one entry in the block is the one: found by the threads, walked by the first warp
      for (int e = threadIdx.x; e < entries; e += kThreads) {
        const double up_to = sh->entry[e], low = e ? sh->entry[e - 1] : 0.0;
        if (up_to > low && before + up_to > aim && !(before + low > aim && low > 0.0)) atomicMax(&sh->pick_n, (uint32_t)e + 1);
      }
      __syncthreads();
      if (warp == 0) {
        int e = (int)sh->pick_n - 1;
        if (e < 0) {  // rounding: the last that has anything
          e = entries - 1;
          while (e > 0 && !(sh->entry[e] > sh->entry[e - 1])) --e;
        }
        double run = before + (e ? sh->entry[e - 1] : 0.0);
        int found = -1, last = -1;
        const int s0 = e << log_q, s1 = min(segs, s0 + (1 << log_q));
        for (int seg = s0; seg < s1 && found < 0; ++seg) {
          float x[kPer];
          load(seg, x);
          const int i0 = first_of(seg);
          double g = 0.0;
#pragma unroll
          for (int j = 0; j < kPer; ++j) g += f(x[j], i0 + j);
          const double up_to = warp_scan(g);
          const unsigned passes = __ballot_sync(0xffffffffu, run + up_to > aim && g > 0.0);
          const unsigned any = __ballot_sync(0xffffffffu, g > 0.0);
          const int who = passes ? __ffs(passes) - 1 : any ? 31 - __clz(any) : -1;
          if (who >= 0) {
            int at = -1;
            if (lane == who) {
              double r = run + up_to - g;
#pragma unroll
              for (int j = 0; j < kPer; ++j) {
                const double v = f(x[j], i0 + j);
                if (v > 0.0 && !(at >= 0 && r > aim)) at = i0 + j;
                r += v;
              }
            }
            at = __shfl_sync(0xffffffffu, at, who);
            last = at;
            if (passes) found = at;
          }
          run += __shfl_sync(0xffffffffu, up_to, 31);
        }
        if (lane == 0) sh->part_i = found >= 0 ? found : last;
      }
    }
    meet();
    const int at = of(owner)->part_i;
    meet();
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
    const int n = segs * 32;
    if (bounds && k <= n) {
      uint32_t lo = 0, hi = 0xffff;  // of the order: the largest b that k bounds reach
      while (lo < hi) {
        const uint32_t mid = (lo + hi + 1) >> 1;
        int mine = 0;
        for (int i = threadIdx.x; i < n; i += kThreads) mine += (key_of(__uint_as_float((uint32_t)bounds[i] << 16)) >> 16) >= mid;
        mine = __reduce_add_sync(0xffffffffu, mine);
        __syncthreads();
        if (lane == 0) sh->warp_n[warp] = (uint32_t)mine;
        __syncthreads();
        long long all = 0;
        for (int w = 0; w < kWarps; ++w) all += sh->warp_n[w];
        if (all >= k)
          lo = mid;
        else
          hi = mid - 1;
      }
      // a bound that was rounded up is above the bfloat16 in front of it
      const uint32_t b = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? lo : lo ? lo - 1 : 0;
      const float v = value_of(b << 16);
      if (v == v) low = fmaxf(low, v);
    }
    if (blocks > 1) {
      if (threadIdx.x == 0) sh->part_m = low;
      meet();
      for (int r = 0; r < blocks; ++r) low = fmaxf(low, of(r)->part_m);
      meet();
    }
    return low;
  }

  // Moves the cut to the last logit, in falling order, before which less than `aim` lies; kWeights: sums of weights, else of
  // ones.  Logits below `floor` are known to lie behind it.  `all`: the amount in the whole row, of which at most `below` lies
  // below `floor`.
  template <bool kWeights>
  __device__ void select(double aim, float floor, double all, double below) {
    const auto amount = [&](float x) { return kWeights ? weight(x) : 1.0; };
    const float span = floor > 0.5f * kLowest ? m - floor : (float)(40.0 / inv_t);
    const float want = (float)(kBins - 2) / span, per = span > 0.f && want < 1e30f ? want : 0.f;  // 0: all in one bin
    // level 0: bins of distance; from level 1 on the bracket is bins [b_lo, b_hi] and keys [k_lo, k_hi], cut by keys
    uint32_t b_lo = 0, b_hi = 0, k_lo = key_of(kLowest), k_hi = key_of(m), n_in = 0;
    // every level divides the keys by 2,048, at the latest from the eighth on: eleven are the most
    for (int level = 0; level < 16; ++level) {
      const bool gather = level > 0 && n_in <= kList;
      const uint32_t width = k_hi - k_lo;
      const int shift = max(0, 21 - __clz(width));  // (width >> shift) < kBins
      // where the bracket has one value, its logits are taken by their index
      const bool ties = level > 0 && !gather && width == 0;
      for (int i = threadIdx.x; i < kBins; i += kThreads) sh->hist[i] = 0;
      if (threadIdx.x == 0) sh->list_n = 0;
      meet();
      // the amount in front of the bracket, and the bracket's logits in bins or in the list
      const double above = sum_of(floor, [&](float x, int i) {
        if (!kept(x, i) || !(x >= floor)) return 0.0;
        const uint32_t key = key_of(x), b = (uint32_t)bin_of(x, per);
        if (level == 0) {
          atomicAdd(&sh->hist[b], 1u);
          return 0.0;
        }
        if (b < b_lo || (b <= b_hi && key > k_hi)) return amount(x);
        if (b > b_hi || key < k_lo) return 0.0;
        if (gather) {
          Shared *o = of(0);
          const uint32_t at = atomicAdd(&o->list_n, 1u);
          if (at < kList) o->list[at] = (uint64_t)(~key) << 32 | (uint32_t)i;
        } else if (!ties) {
          atomicAdd(&sh->hist[(k_hi - key) >> shift], 1u);
        }
        return 0.0;
      });
      meet();
      if (ties) {
        // kept are the first r with above + (r - 1) w < aim
        const float v = value_of(k_lo);
        const double w = amount(v);
        double r = fmin((double)n_in, fmax(1.0, ceil((aim - above) / w)));
        if (r > 1.0 && !(above + (r - 1.0) * w < aim))
          r -= 1.0;
        else if (r < (double)n_in && above + r * w < aim)
          r += 1.0;
        const int at = locate(v, [&](float x, int i) { return x == v && kept(x, i) ? 1.0 : 0.0; }, r - 0.5, true, nullptr);
        cut_v = v;
        cut_i = at;
        return;
      }
      if (rank == 0) {
        if (gather)
          cut_from_list<kWeights>(aim, above);
        else
          bracket<kWeights>(level, aim, above, all, below, per, k_lo, k_hi, shift);
      }
      meet();
      const Shared *o = of(0);
      if (gather) {
        cut_v = o->cut_v;
        cut_i = o->cut_i;
        meet();
        return;
      }
      const uint32_t lo = o->pick_lo, hi = o->pick_hi;
      n_in = o->pick_n;
      meet();
      if (n_in == 0) return;  // less than the aim in all: everything stays
      if (level == 0) {
        b_lo = lo, b_hi = hi;
        // keys that the bins' logits can have; 2^-20 covers the roundings of the distance
        const double slack = 9.5367431640625e-7;
        if (per > 0.f) {
          k_hi = key_of(__double2float_ru((double)m - (double)lo / per * (1.0 - slack)));
          if (hi < kBins - 1) k_lo = key_of(__double2float_rd((double)m - ((double)hi + 1.0) / per * (1.0 + slack)));
        }
      } else {
        k_lo = edge_of(k_lo, k_hi, hi, shift);
        k_hi -= lo << shift;
      }
    }
  }

  // The least key of bin b, of keys from k_lo to k_hi: bin 0 has the largest.
  __device__ __forceinline__ static uint32_t edge_of(uint32_t k_lo, uint32_t k_hi, uint32_t b, int shift) {
    const int64_t least = (int64_t)k_hi - (int64_t)(((uint64_t)b + 1) << shift) + 1;
    return least > (int64_t)k_lo ? (uint32_t)least : k_lo;
  }

  // The first block: which of the histogram's bins can hold the cut.  pick_n = 0: all of it lies in front of the aim.
  template <bool kWeights>
  __device__ void bracket(int level, double aim, double above, double all, double below, float per, uint32_t k_lo, uint32_t k_hi,
                          int shift) {
    constexpr int kOwn = kBins / kThreads;
    uint32_t n[kOwn], n_sum = 0;
    double least[kOwn], most[kOwn], least_sum = 0.0, most_sum = 0.0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const uint32_t b = threadIdx.x * kOwn + j;
      n[j] = sh->hist[b];
      for (int r = 1; r < blocks; ++r) n[j] += of(r)->hist[b];
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
        // where a bin holds one value, or the bracket would not get smaller, the larger of the two decides
        most[j] *= exp(-near * inv_t);
        least[j] = level >= 8 || (level > 0 && shift == 0) ? most[j] : least[j] * exp(-far * inv_t);
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
      sh->pick_lo = kBins;  // the first bin up to which there can be as much as the aim
      sh->pick_hi = kBins;  // the first up to which there is
      sh->part_i = 0;       // the last that holds anything
    }
    __syncthreads();
    uint32_t n_run = n_up - n_sum;
    double least_run = above + least_up - least_sum, most_run = above + most_up - most_sum, least_all = above, most_all = above + below;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) {
        n_run += sh->warp_n[w];
        least_run += sh->warp_a[w];
        most_run += sh->warp_b[w];
      }
      least_all += sh->warp_a[w];
      most_all += sh->warp_b[w];
    }
    // A bin's edges bound its weights to a percent or so.  Over the whole row (level 0) the bounds on what lies behind a bin,
    // taken from the known whole, are the closer ones where the aim is near it: 1.5 % of the last twentieth for a top_p of 0.95
    const bool sharp = !kWeights || level >= 8 || (level > 0 && shift == 0);
    const double eps = sharp ? 0.0 : 1e-11 * all;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const uint32_t b = threadIdx.x * kOwn + j;
      n_run += n[j];
      least_run += least[j];
      most_run += most[j];
      if (n[j]) atomicMax(&sh->part_i, (int)b);
      double high = most_run, low = sharp ? most_run : least_run;
      if (!sharp && level == 0) {
        high = fmin(high, all - (least_all - least_run));
        low = fmax(low, all - (most_all - most_run));
      }
      if (n[j] && high >= aim - eps) atomicMin(&sh->pick_lo, b);
      if (n[j] && low >= aim + eps) atomicMin(&sh->pick_hi, b);
    }
    __syncthreads();
    uint32_t lo = sh->pick_lo;
    uint32_t hi = min(sh->pick_hi, (uint32_t)kBins - 1);
    if (level > 0 && lo == kBins) lo = hi = (uint32_t)sh->part_i;  // the cut is in the bracket: what is missing is a rounding
    __syncthreads();
    // logits in bins lo to hi
    uint32_t inside = 0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const uint32_t b = threadIdx.x * kOwn + j;
      if (lo < (uint32_t)kBins && b >= lo && b <= hi) inside += n[j];
    }
    inside = __reduce_add_sync(0xffffffffu, inside);
    if (lane == 0) sh->warp_n[warp] = inside;
    __syncthreads();
    if (threadIdx.x == 0) {
      uint32_t all = 0;
      for (int w = 0; w < kWarps; ++w) all += sh->warp_n[w];
      sh->pick_n = all;
      sh->pick_lo = lo;
      sh->pick_hi = hi;
    }
    __syncthreads();
  }

  // The first block: sorts the list (falling logits, rising indices) and finds its last logit before which less than the aim lies.
  template <bool kWeights>
  __device__ void cut_from_list(double aim, double above) {
    const int n = min((int)sh->list_n, kList);
    int size = 32;
    while (size < n) size <<= 1;
    for (int i = n + threadIdx.x; i < size; i += kThreads) sh->list[i] = ~0ull;
    __syncthreads();
    for (int k = 2; k <= size; k <<= 1)
      for (int j = k >> 1; j > 0; j >>= 1) {
        for (int t = threadIdx.x; t < size / 2; t += kThreads) {
          const int a = (t & ~(j - 1)) * 2 + (t & (j - 1)), b = a + j;
          const uint64_t x = sh->list[a], y = sh->list[b];
          if ((x > y) == ((a & k) == 0)) {
            sh->list[a] = y;
            sh->list[b] = x;
          }
        }
        __syncthreads();
      }
    constexpr int kOwn = kList / kThreads;
    double w[kOwn], sum = 0.0;
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const int i = threadIdx.x * kOwn + j;
      w[j] = i < n ? kWeights ? weight(value_of(~(uint32_t)(sh->list[i] >> 32))) : 1.0 : 0.0;
      sum += w[j];
    }
    const double up_to = warp_scan(sum);
    if (lane == 31) sh->warp_a[warp] = up_to;
    if (threadIdx.x == 0) sh->pick_n = 0;
    __syncthreads();
    double run = above + up_to - sum;
    for (int v = 0; v < warp; ++v) run += sh->warp_a[v];
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      const int i = threadIdx.x * kOwn + j;
      if (i < n && (run < aim || i == 0)) atomicMax(&sh->pick_n, (uint32_t)i);
      run += w[j];
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      const uint64_t last = sh->list[sh->pick_n];
      sh->cut_v = value_of(~(uint32_t)(last >> 32));
      sh->cut_i = (int)(uint32_t)last;
    }
    __syncthreads();
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
  row.seg0 = (int)(each * row.rank);
  row.segs = (int)max(0LL, min(each, segs - row.seg0));
  row.log_q = 0;
  while (((row.segs + (1 << row.log_q) - 1) >> row.log_q) > kEntries) ++row.log_q;
  row.entries = (row.segs + (1 << row.log_q) - 1) >> row.log_q;

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
  row.inv_t = 1.0 / temperature;
  row.c = (float)(1.4426950408889634 * row.inv_t);

  double rest;
  row.stats(rest);
  valid = valid && row.m > kNegInf && row.m < -kNegInf && rest == rest;
  int id = -1, count = 0;
  double kept_rest = 0.0;
  if (valid) {
    row.cut_v = rho > 0.0 ? fmaxf(kLowest, __double2float_ru((double)row.m + temperature * log(rho))) : kLowest;
    row.cut_i = kNoIndex;
    if (top_k == 1) {
      id = row.first_of_max();
      count = 1;
    } else {
      if (top_k > 0 && top_k < p.V) row.template select<false>((double)top_k, row.floor_of(top_k), 0.0, 0.0);
      if (top_p < 1.0) {
        const float from = row.cut_v;
        const double all = row.sum_of(from, [&](float x, int i) { return row.kept(x, i) ? row.weight(x) : 0.0; });
        // logits whose weight is under a V-th of 0.01 (1 - top_p) of the whole hold less than that much together
        const double below = 0.01 * (1.0 - top_p) * all;
        row.template select<true>(top_p * all, fmaxf(from, __double2float_rd((double)row.m + temperature * log(below / (double)p.V))), all,
                                  below * 1.001);
      }
      // what is kept: the token, the sum and the number
      int n = 0;
      double all;
      id = row.locate(row.cut_v, [&](float x, int i) { return row.kept(x, i) ? row.weight(x) : 0.0; }, (double)u, false, &all);
      kept_rest = all - 1.0;
      row.sweep(row.cut_v, [&](const float (&x)[kPer], int i0) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) n += row.kept(x[j], i0 + j) && x[j] > kNegInf;
      }, [](int) {});
      n = __reduce_add_sync(0xffffffffu, n);
      if (threadIdx.x == 0) row.sh->part_i = 0;
      __syncthreads();
      if (row.lane == 0) atomicAdd(&row.sh->part_i, n);
      row.meet();
      for (int r = 0; r < row.blocks; ++r) count += row.of(r)->part_i;
    }
  }
  if (row.rank == 0 && threadIdx.x == 0) {
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
