// Root-mean-square norm with the residual's addition, its output in the model's type or in 8 bits with a scale for each
// block of 128 columns, and its backward pass.
//
//   h = x + r,  s = (mean h^2 + eps)^(-1/2),  y = h s w;      8 bits: c = max(max |y|, 2^-96) / 448 a block, q = e4m3(y / c)
//   g = dy w,   dx = s (g - h s^2 mean(g h)) (+ dr),          dw = sum_t dy h s
//
// Both are bound by HBM: a row's threads hold it in registers between the sum and the output, so every matrix passes
// once.  Rows that vectors of eight elements do not fit (width, stride or base) have kernels of their own, which read a row
// twice, element by element.
#include <atomic>
#include <cmath>

#include "dvp_common.cuh"
#include "dvp_fp8.cuh"

namespace dvp {
namespace norm {

constexpr int kBlockCols = 128;  // columns that share a scale
constexpr int kVec = 8;          // elements of a vector: 16 bytes of a 16-bit type, 32 of float32, 8 of e4m3
constexpr int kMaxPartials = 592;               // rows of partial sums of dw: one a block and row side by side, for 148 SMs four an SM

struct Params {
  const void *x, *r, *w;
  void *r_out, *out;
  float *scale, *rstd;
  long long T, H, ld_x, ld_r, ld_r_out, ld_out, ld_scale;
  float inv_h, eps;
  int w_f32;
};

// Eight neighbouring elements as they lie.  Not through the read-only path: an output may take the place of an input, whose
// elements the same thread has read.
template <typename T>
struct Raw {
  uint32_t w[2 * sizeof(T)];
  __device__ __forceinline__ void load(const T *p) {
    if constexpr (sizeof(T) == 4)
      asm volatile("ld.global.L1::no_allocate.v8.u32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                   : "l"(p)
                   : "memory");
    else
      asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                   : "l"(p)
                   : "memory");
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int j = 0; j < (int)(2 * sizeof(T)); ++j) w[j] = 0;
  }
  __device__ __forceinline__ void widen(float (&v)[8]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j]);
    } else {
      Storage<T>::unpack(make_uint4(w[0], w[1], w[2], w[3]), v);
    }
  }
};
template <typename T>
__device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[j]);
    st_stream32(p, w);
  } else {
    store_grads<T, 8>(p, v);
  }
}
// Weights: read by every row, so they stay in L1.  Loads by __ldg, which promises that nothing writes there, were executed ahead of
// the comparison with the row's end: a float32 weight of one element was read by a whole block.  Ordinary loads are not.
template <typename T>
__device__ __forceinline__ void load_weights8(const void *w, int w_f32, long long c, float (&v)[8]) {
  if (sizeof(T) == 4 || w_f32) {
    const float4 *q = reinterpret_cast<const float4 *>(static_cast<const float *>(w) + c);
    const float4 a = q[0], b = q[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else if constexpr (sizeof(T) == 2) {
    Storage<T>::unpack(*reinterpret_cast<const uint4 *>(static_cast<const T *>(w) + c), v);
  }
}
template <typename T>
__device__ __forceinline__ float load_weight(const void *w, int w_f32, long long c) {
  return sizeof(T) == 4 || w_f32 ? static_cast<const float *>(w)[c] : Storage<T>::widen(static_cast<const T *>(w)[c]);
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The sum over the `tpr` threads (whole warps) of each of the block's rows; `part`: 32 floats that no earlier sum is read
// from any more.  Every thread of the block takes part.
__device__ __forceinline__ float row_sum(float v, int tpr, float *part) {
  v = warp_sum(v);
  if (tpr == 32) return v;
  const int warp = threadIdx.x >> 5, warps = tpr >> 5, first = warp / warps * warps;
  if ((threadIdx.x & 31) == 0) part[warp] = v;
  __syncthreads();
  if (warps == 8 || warps == 16) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      if (i >= warps) break;
      const float4 q = *reinterpret_cast<const float4 *>(part + first + i);
      s += (q.x + q.y) + (q.z + q.w);
    }
    return s;
  }
  float s = 0.f;
  for (int i = 0; i < warps; ++i) s += part[first + i];
  return s;
}

// ---- rows in vectors ---------------------------------------------------------------------------------------------------

// A block's rows are blockIdx.x * rpb + i * gridDim.x * rpb: the next is on its way while one is summed up and stored, so that loads
// never pause (16,384 x 4,096 bfloat16 to 8 bits, with approximate quotients and roots: 103 us, with one row a block and nothing on its
// way 139; as it is now 113, 4.2 TB/s: instructions issue in 0.59 of the cycles, and warps wait for loads and for the row's chain).
template <typename T, typename TOut, int kPer>
__global__ void __launch_bounds__(kPer == 4 ? 512 : 256, kPer == 1 ? 4 : kPer == 2 ? 3 : 1) rms_norm_kernel(const Params p, const int tpr) {
  __shared__ __align__(16) float part[2][32];
  const int lane_of_row = threadIdx.x % tpr, rpb = blockDim.x / tpr;
  const long long step = (long long)gridDim.x * rpb;
  // rows on their way: two where their registers are few
  constexpr int kAhead = kPer == 1 && sizeof(T) == 2 ? 2 : 1;
  Raw<T> x[kAhead][kPer], r[kAhead][kPer];
  const auto column = [&](int i) { return ((long long)lane_of_row + (long long)i * tpr) * kVec; };
  long long t = (long long)blockIdx.x * rpb + threadIdx.x / tpr;
  // the row to fetch next, and this one's outputs, at the thread's first column
  const T *x_at = static_cast<const T *>(p.x) + t * p.ld_x + column(0), *r_at = static_cast<const T *>(p.r) + t * p.ld_r + column(0);
  T *h_at = static_cast<T *>(p.r_out) + t * p.ld_r_out + column(0);
  TOut *y_at = static_cast<TOut *>(p.out) + t * p.ld_out + column(0);
  bool in[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) in[i] = column(i) < p.H;
  const bool has_r = p.r != nullptr, has_h = p.r_out != nullptr;
  const int across = tpr * kVec;
  const auto fetch = [&](Raw<T> (&x)[kPer], Raw<T> (&r)[kPer], bool live) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (live && in[i]) {
        x[i].load(x_at + i * across);
        if (has_r) r[i].load(r_at + i * across);
      } else {
        x[i].zero();
        r[i].zero();
      }
    }
    x_at += step * p.ld_x;
    r_at += step * p.ld_r;
  };
#pragma unroll
  for (int a = 0; a < kAhead; ++a) fetch(x[a], r[a], t + a * step < p.T);
  int turn = 0;
  for (long long first = (long long)blockIdx.x * rpb; first < p.T; first += step, t += step, turn ^= 1) {
    const bool live = t < p.T;
    float h[kPer][kVec], sum = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      x[0][i].widen(h[i]);
      if (has_r) {
        float v[kVec];
        r[0][i].widen(v);
#pragma unroll
        for (int j = 0; j < kVec; ++j) h[i][j] += v[j];
      }
#pragma unroll
      for (int j = 0; j < kVec; ++j) sum = fmaf(h[i][j], h[i][j], sum);
    }
#pragma unroll
    for (int a = 0; a + 1 < kAhead; ++a)
#pragma unroll
      for (int i = 0; i < kPer; ++i) x[a][i] = x[a + 1][i], r[a][i] = r[a + 1][i];
    if (first + kAhead * step < p.T) fetch(x[kAhead - 1], r[kAhead - 1], t + kAhead * step < p.T);
    const float s = 1.f / sqrtf(fmaf(row_sum(sum, tpr, part[turn]), p.inv_h, p.eps));  // two sets: see the backward kernel
    if (live && lane_of_row == 0 && p.rstd) p.rstd[t] = s;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const bool here = live && in[i];
      if (has_h && here) store8(h_at + i * across, h[i]);
      float w[kVec], y[kVec];
      if (here) {
        load_weights8<T>(p.w, p.w_f32, column(i), w);
      } else {
#pragma unroll
        for (int j = 0; j < kVec; ++j) w[j] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < kVec; ++j) y[j] = h[i][j] * s * w[j];
      if constexpr (sizeof(TOut) == 1) {
        // sixteen neighbouring lanes hold a block of 128 columns
        float a = fp8::kLeastAmax;
#pragma unroll
        for (int j = 0; j < kVec; ++j) a = fmaxf(a, fabsf(y[j]));
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
        const float scale = fp8::scale_of(a);
        if (here) {
          if ((threadIdx.x & 15) == 0) p.scale[t * p.ld_scale + column(i) / kBlockCols] = scale;
          uint32_t q[2];
          fp8::quotients<kVec>(y, scale, q);
          st_stream8(y_at + i * across, make_uint2(q[0], q[1]));
        }
      } else if (here) {
        store8(y_at + i * across, y);
      }
    }
    h_at += step * p.ld_r_out;
    y_at += step * p.ld_out;
  }
}

// ---- rows of any layout ------------------------------------------------------------------------------------------------

constexpr int kAnyThreads = 256;

__device__ __forceinline__ float block_sum(float v, float *part) {
  v = warp_sum(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kAnyThreads / 32; ++i) s += part[i];
  return s;
}

// A warp takes whole blocks of 128 columns, four a lane, in both sweeps alike: what takes an input's place is written by the
// thread that has read it last.  (Kept in registers between the sweeps, 32 a thread, the rows were slower: 1,111 x 5,003 float16 16.4 us a
// call, read twice 12.3, as twice as many blocks fit an SM.)
template <typename T, typename TOut>
__global__ void __launch_bounds__(kAnyThreads) rms_norm_any_kernel(const Params p) {
  __shared__ float part[kAnyThreads / 32];
  constexpr int kWarps = kAnyThreads / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long blocks = (p.H + kBlockCols - 1) / kBlockCols;
  for (long long t = blockIdx.x; t < p.T; t += gridDim.x) {
    const T *x = static_cast<const T *>(p.x) + t * p.ld_x;
    const T *r = p.r ? static_cast<const T *>(p.r) + t * p.ld_r : nullptr;
    const auto entry = [&](long long c) { return Storage<T>::widen(x[c]) + (r ? Storage<T>::widen(r[c]) : 0.f); };
    const auto column = [&](long long b, int j) { return b * kBlockCols + j * 32 + lane; };
    float sum = 0.f;
    for (long long b = warp; b < blocks; b += kWarps)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const long long c = column(b, j);
        const float v = c < p.H ? entry(c) : 0.f;
        sum = fmaf(v, v, sum);
      }
    const float s = 1.f / sqrtf(fmaf(block_sum(sum, part), p.inv_h, p.eps));
    if (threadIdx.x == 0 && p.rstd) p.rstd[t] = s;
    for (long long b = warp; b < blocks; b += kWarps) {
      float h[4], y[4], a = fp8::kLeastAmax;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const long long c = column(b, j);
        h[j] = c < p.H ? entry(c) : 0.f;
        y[j] = c < p.H ? h[j] * s * load_weight<T>(p.w, p.w_f32, c) : 0.f;
        a = fmaxf(a, fabsf(y[j]));
      }
      uint32_t q[1] = {0};
      if constexpr (sizeof(TOut) == 1) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, o));
        const float scale = fp8::scale_of(a);
        fp8::quotients<4>(y, scale, q);
        if (lane == 0) p.scale[t * p.ld_scale + b] = scale;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const long long c = column(b, j);
        if (c >= p.H) continue;
        if (p.r_out) static_cast<T *>(p.r_out)[t * p.ld_r_out + c] = Storage<T>::narrow(h[j]);
        if constexpr (sizeof(TOut) == 1)
          static_cast<uint8_t *>(p.out)[t * p.ld_out + c] = (uint8_t)(q[0] >> (8 * j));
        else
          static_cast<TOut *>(p.out)[t * p.ld_out + c] = Storage<TOut>::narrow(y[j]);
      }
    }
  }
}

// ---- backward ----------------------------------------------------------------------------------------------------------

struct BackParams {
  const void *dy, *h, *w, *dr;
  const float *rstd;
  void *dx;
  float *partial;  // [gridDim.x, H]: the blocks' sums of dy h s; NULL without d_weight
  long long T, H, ld_dy, ld_h, ld_dr, ld_dx;
  float inv_h;
  int w_f32;
};

// A block's rows are blockIdx.x * rpb + i * gridDim.x * rpb: its threads keep their columns, and with them the sums of dw.  Bound by
// HBM: 16,384 x 4,096 bfloat16 with float32 dy, dr and dw 122 to 131 us, 671 MB at 5.1 to 5.5 TB/s; without the next row on its way 166, with its
// addresses formed anew for each row 131.  The sum of the partial rows is a launch of its own, some 5 us of a call's.
// Four vectors a thread (8,200 to 16,384 columns) spill some 600 bytes at 128 registers: 4,096 x 16,384 192 us, 3.5 TB/s.  Rows of up
// to 256 columns lie eight a block side by side, and the workspace's 592 rows allow 74 such blocks: 32,768 x 128 44 us, 1 TB/s.
template <typename T, typename TD, int kPer>
__global__ void __launch_bounds__(512, kPer == 1 ? 2 : 1) rms_norm_backward_kernel(const BackParams p, const int tpr) {
  __shared__ __align__(16) float part[2][32];
  const int lane_of_row = threadIdx.x % tpr, rpb = blockDim.x / tpr, row_of_block = threadIdx.x / tpr;
  float w[kPer][kVec], dw[kPer][kVec];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const long long c = ((long long)lane_of_row + (long long)i * tpr) * kVec;
#pragma unroll
    for (int j = 0; j < kVec; ++j) w[i][j] = dw[i][j] = 0.f;
    if (c < p.H) load_weights8<T>(p.w, p.w_f32, c, w[i]);
  }
  const long long step = (long long)gridDim.x * rpb;
  Raw<T> h_raw[kPer], r_raw[kPer];
  Raw<TD> d_raw[kPer];
  const auto fetch = [&](long long t) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const long long c = ((long long)lane_of_row + (long long)i * tpr) * kVec;
      if (t < p.T && c < p.H) {
        d_raw[i].load(static_cast<const TD *>(p.dy) + t * p.ld_dy + c);
        h_raw[i].load(static_cast<const T *>(p.h) + t * p.ld_h + c);
        if (p.dr) r_raw[i].load(static_cast<const T *>(p.dr) + t * p.ld_dr + c);
      } else {
        d_raw[i].zero();
        h_raw[i].zero();
        r_raw[i].zero();
      }
    }
  };
  constexpr bool kAhead = kPer < 4;  // four vectors a thread leave no registers for the next row
  long long t = (long long)blockIdx.x * rpb + row_of_block;
  if (kAhead) fetch(t);
  float s_next = t < p.T ? p.rstd[t] : 0.f;
  int turn = 0;
  for (long long first = (long long)blockIdx.x * rpb; first < p.T; first += step, t += step, turn ^= 1) {
    const bool live = t < p.T;
    const float s = s_next;
    if (!kAhead) fetch(t);
    float h[kPer][kVec], d[kPer][kVec], r[kPer][kVec];
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      h_raw[i].widen(h[i]);
      d_raw[i].widen(d[i]);
      if (p.dr) r_raw[i].widen(r[i]);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        dw[i][j] = fmaf(d[i][j] * s, h[i][j], dw[i][j]);
        d[i][j] *= w[i][j];
        dot = fmaf(d[i][j], h[i][j], dot);
      }
    }
    if (first + step < p.T) {
      if (kAhead) fetch(t + step);
      s_next = t + step < p.T ? p.rstd[t + step] : 0.f;
    }
    dot = row_sum(dot, tpr, part[turn]);  // two sets: one is read while the next row's is written
    const float k = dot * p.inv_h * s * s;
    if (p.dx && live) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const long long c = ((long long)lane_of_row + (long long)i * tpr) * kVec;
        if (c >= p.H) continue;
        float o[kVec];
#pragma unroll
        for (int j = 0; j < kVec; ++j) o[j] = s * fmaf(-k, h[i][j], d[i][j]) + (p.dr ? r[i][j] : 0.f);
        store8(static_cast<T *>(p.dx) + t * p.ld_dx + c, o);
      }
    }
  }
  if (!p.partial) return;
  // the rows that a block works on side by side have a row of partial sums each
  float *to = p.partial + ((long long)blockIdx.x * rpb + row_of_block) * p.H;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const long long c = ((long long)lane_of_row + (long long)i * tpr) * kVec;
    if (c < p.H)
#pragma unroll
      for (int j = 0; j < kVec; j += 4)
        *reinterpret_cast<float4 *>(to + c + j) = make_float4(dw[i][j], dw[i][j + 1], dw[i][j + 2], dw[i][j + 3]);
  }
}

template <typename T, typename TD>
__global__ void __launch_bounds__(kAnyThreads) rms_norm_backward_any_kernel(const BackParams p) {
  __shared__ float part[kAnyThreads / 32];
  float *to = p.partial ? p.partial + (long long)blockIdx.x * p.H : nullptr;
  for (long long t = blockIdx.x; t < p.T; t += gridDim.x) {
    const TD *dy = static_cast<const TD *>(p.dy) + t * p.ld_dy;
    const T *h = static_cast<const T *>(p.h) + t * p.ld_h;
    const float s = p.rstd[t];
    float dot = 0.f;
    for (long long c = threadIdx.x; c < p.H; c += kAnyThreads)
      dot = fmaf(Storage<TD>::widen(dy[c]) * load_weight<T>(p.w, p.w_f32, c), Storage<T>::widen(h[c]), dot);
    const float k = block_sum(dot, part) * p.inv_h * s * s;
    for (long long c = threadIdx.x; c < p.H; c += kAnyThreads) {
      const float d = Storage<TD>::widen(dy[c]), hc = Storage<T>::widen(h[c]);
      // a thread has the same columns in every row: it adds to what it has written itself
      if (to) to[c] = fmaf(d * s, hc, t == blockIdx.x ? 0.f : to[c]);
      if (!p.dx) continue;
      float o = s * fmaf(-k, hc, d * load_weight<T>(p.w, p.w_f32, c));
      if (p.dr) o += Storage<T>::widen(static_cast<const T *>(p.dr)[t * p.ld_dr + c]);
      static_cast<T *>(p.dx)[t * p.ld_dx + c] = Storage<T>::narrow(o);
    }
  }
}

// dw (+)= the sum of the partial rows: 32 columns a block, eight threads a column, in a fixed order.
__global__ void __launch_bounds__(256) sum_partials_kernel(const float *partial, int rows, long long H, float *dw,
                                                           int accumulate) {
  __shared__ float part[8][33];
  const int col = threadIdx.x & 31, slice = threadIdx.x >> 5;
  const long long c = (long long)blockIdx.x * 32 + col;
  float v = 0.f;
  if (c < H)
    for (int r = slice; r < rows; r += 8) v += partial[(long long)r * H + c];
  part[slice][col] = v;
  __syncthreads();
  if (slice == 0 && c < H) {
#pragma unroll
    for (int i = 1; i < 8; ++i) v += part[i][col];
    dw[c] = accumulate ? dw[c] + v : v;
  }
}

// ---- host --------------------------------------------------------------------------------------------------------------

inline bool dtype_ok(int d) { return d == DVP_F32 || d == DVP_BF16 || d == DVP_F16; }
inline long long size_of(int d) { return d == DVP_F32 ? 4 : d == DVP_E4M3 ? 1 : 2; }
// Rows of vectors: every row begins on the boundary of eight elements.
inline bool vectors(const void *base, long long ld, int dtype) {
  return !base || ((uintptr_t)base % (8 * size_of(dtype)) == 0 && ld % kVec == 0);
}
// float32 weights are read in 16 bytes.
inline bool weight_vectors(const void *w) { return (uintptr_t)w % 16 == 0; }

struct Shape {
  int per, tpr, rpb;  // vectors a thread, threads a row, rows a block
};
// Forward, one vector a thread up to 256 threads a row, then two (16,384 x 4,096 to 8 bits, approximate quotients: 103 us, one vector and 512 threads
// 114), then four; backward, whose threads hold a row of dw too, 512.  per = 0: too long for the registers, or no vector at all.
inline Shape shape_of(long long H, bool backward) {
  const long long nv = H / kVec;
  const int per = nv < 1 ? 0 : nv <= (backward ? 512 : 256) ? 1 : nv <= (backward ? 1024 : 512) ? 2 : nv <= 2048 ? 4 : 0;
  if (!per) return {0, 0, 0};
  const int tpr = (int)(((nv + per - 1) / per + 31) / 32 * 32);
  return {per, tpr, tpr >= 256 ? 1 : 256 / tpr};
}
// Blocks that the chip holds at once: what a kernel's registers allow, asked for once a kernel and number of threads.
template <typename Kernel>
int resident(Kernel kernel, std::atomic<int> (&known)[33], int threads, int sms) {
  int blocks = known[threads / 32].load(std::memory_order_relaxed);
  if (blocks == 0) {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, kernel, threads, 0) != cudaSuccess || blocks < 1) blocks = 1;
    known[threads / 32].store(blocks, std::memory_order_relaxed);
  }
  return blocks * sms;
}
inline int sm_count() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) return 148;
  return sms;
}

// Calls f with a value of the storage type that `d` names.
template <typename F>
cudaError_t by_type(int d, F f) {
  if (d == DVP_F32) return f(float());
  if (d == DVP_BF16) return f(__nv_bfloat16());
  return f(__half());
}

template <typename T, typename TOut>
cudaError_t launch_forward(const Params &p, bool fast, cudaStream_t stream) {
  const Shape sh = shape_of(p.H, false);
  if (fast && sh.per) {
    const int block = sh.tpr * sh.rpb;
    const long long want = (p.T + sh.rpb - 1) / sh.rpb;
    static std::atomic<int> known[5][33];
    const auto go = [&](auto kernel) {
      const long long most = resident(kernel, known[sh.per], block, sm_count());
      kernel<<<(unsigned)(want < most ? want : most), block, 0, stream>>>(p, sh.tpr);
    };
    if (sh.per == 1)
      go(rms_norm_kernel<T, TOut, 1>);
    else if (sh.per == 2)
      go(rms_norm_kernel<T, TOut, 2>);
    else
      go(rms_norm_kernel<T, TOut, 4>);
  } else {
    rms_norm_any_kernel<T, TOut><<<(unsigned)p.T, kAnyThreads, 0, stream>>>(p);
  }
  return cudaGetLastError();
}

// Blocks of the backward kernel: what the chip holds at once and the workspace has rows for, no more than there are rows.
inline int backward_blocks(long long T, int rpb, int most_blocks) {
  const long long want = (T + rpb - 1) / rpb, room = kMaxPartials / rpb;
  const long long n = want < room ? want : room;
  return (int)(n < most_blocks ? n : most_blocks);
}

template <typename T, typename TD>
cudaError_t launch_backward(const BackParams &p, bool fast, float *dw, int accumulate, cudaStream_t stream) {
  const Shape sh = shape_of(p.H, true);
  int rows;
  if (fast && sh.per) {
    const int block = sh.tpr * sh.rpb;
    static std::atomic<int> known[5][33];
    const auto go = [&](auto kernel) {
      const int grid = backward_blocks(p.T, sh.rpb, resident(kernel, known[sh.per], block, sm_count()));
      rows = grid * sh.rpb;
      kernel<<<grid, block, 0, stream>>>(p, sh.tpr);
    };
    if (sh.per == 1)
      go(rms_norm_backward_kernel<T, TD, 1>);
    else if (sh.per == 2)
      go(rms_norm_backward_kernel<T, TD, 2>);
    else
      go(rms_norm_backward_kernel<T, TD, 4>);
  } else {
    rows = backward_blocks(p.T, 1, kMaxPartials);
    rms_norm_backward_any_kernel<T, TD><<<rows, kAnyThreads, 0, stream>>>(p);
  }
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || !dw) return e;
  sum_partials_kernel<<<(unsigned)((p.H + 31) / 32), 256, 0, stream>>>(p.partial, rows, p.H, dw, accumulate);
  return cudaGetLastError();
}

// Whatever layout the pointers turn out to have: the most partial rows of both kinds of kernel.
size_t backward_workspace(const dvp_rms_norm_backward_args *a) {
  if (!a || a->struct_size != sizeof(*a) || a->T < 0 || a->H < 1 || !a->d_weight) return 0;
  return (size_t)(a->T < kMaxPartials ? (a->T + 7) / 8 * 8 : kMaxPartials) * (size_t)a->H * sizeof(float);
}

constexpr long long kMost = 0x7fffff00LL;

}  // namespace norm

size_t rms_norm_backward_workspace(const void *args) {
  return norm::backward_workspace(static_cast<const dvp_rms_norm_backward_args *>(args));
}

}  // namespace dvp

extern "C" {

int dvp_rms_norm(const dvp_rms_norm_args *a) {
  using namespace dvp;
  using namespace dvp::norm;
  if (!a || a->struct_size != sizeof(dvp_rms_norm_args)) return DVP_ERR_INVALID_ARG;
  if (!dtype_ok(a->x_dtype) || (a->weight_dtype != a->x_dtype && a->weight_dtype != DVP_F32)) return DVP_ERR_UNSUPPORTED;
  const bool fp8 = a->out_dtype == DVP_E4M3;
  if (!fp8 && !dtype_ok(a->out_dtype)) return DVP_ERR_UNSUPPORTED;
  if (a->T < 0 || a->H < 1 || !(a->eps >= 0.0 && std::isfinite(a->eps))) return DVP_ERR_INVALID_ARG;
  if (a->T > kMost || a->H > kMost) return DVP_ERR_UNSUPPORTED;
  if ((a->scale != nullptr) != fp8 && a->T > 0) return DVP_ERR_INVALID_ARG;
  if (a->T == 0) return DVP_OK;
  if (!a->x || !a->weight || !a->out || a->ld_x < a->H || a->ld_out < a->H) return DVP_ERR_INVALID_ARG;
  if ((a->residual && a->ld_residual < a->H) || (a->residual_out && a->ld_residual_out < a->H)) return DVP_ERR_INVALID_ARG;
  if (fp8 && a->ld_scale < (a->H + kBlockCols - 1) / kBlockCols) return DVP_ERR_INVALID_ARG;
  Params p{a->x, a->residual, a->weight, a->residual_out, a->out, a->scale, a->rstd, a->T, a->H, a->ld_x, a->ld_residual,
           a->ld_residual_out, a->ld_out, a->ld_scale, (float)(1.0 / (double)a->H), (float)a->eps, a->weight_dtype == DVP_F32};
  const bool fast = a->H % kVec == 0 && vectors(a->x, a->ld_x, a->x_dtype) && vectors(a->residual, a->ld_residual, a->x_dtype) &&
                    vectors(a->residual_out, a->ld_residual_out, a->x_dtype) && vectors(a->out, a->ld_out, a->out_dtype) &&
                    weight_vectors(a->weight);
  const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
  const cudaError_t e = by_type(a->x_dtype, [&](auto x) {
    using T = decltype(x);
    if (fp8) return launch_forward<T, uint8_t>(p, fast, stream);
    return by_type(a->out_dtype, [&](auto o) { return launch_forward<T, decltype(o)>(p, fast, stream); });
  });
  return e == cudaSuccess ? DVP_OK : DVP_ERR_CUDA;
}

int dvp_rms_norm_backward(const dvp_rms_norm_backward_args *a) {
  using namespace dvp;
  using namespace dvp::norm;
  if (!a || a->struct_size != sizeof(dvp_rms_norm_backward_args)) return DVP_ERR_INVALID_ARG;
  if (!dtype_ok(a->h_dtype) || !dtype_ok(a->dy_dtype) || (a->weight_dtype != a->h_dtype && a->weight_dtype != DVP_F32))
    return DVP_ERR_UNSUPPORTED;
  if (a->T < 0 || a->H < 1) return DVP_ERR_INVALID_ARG;
  if (a->T > kMost || a->H > kMost) return DVP_ERR_UNSUPPORTED;
  const cudaStream_t stream = static_cast<cudaStream_t>(a->stream);
  if (a->T == 0) {
    if (!a->d_weight || a->accumulate_dw) return DVP_OK;
    return cudaMemsetAsync(a->d_weight, 0, (size_t)a->H * sizeof(float), stream) == cudaSuccess ? DVP_OK : DVP_ERR_CUDA;
  }
  if (!a->dy || !a->h || !a->weight || !a->rstd || (!a->d_x && !a->d_weight)) return DVP_ERR_INVALID_ARG;
  if (a->ld_dy < a->H || a->ld_h < a->H || (a->d_residual && a->ld_d_residual < a->H) || (a->d_x && a->ld_d_x < a->H))
    return DVP_ERR_INVALID_ARG;
  if (a->d_weight && (!a->workspace || (uintptr_t)a->workspace % 256 || a->workspace_bytes < backward_workspace(a)))
    return DVP_ERR_WORKSPACE;
  BackParams p{a->dy, a->h, a->weight, a->d_x ? a->d_residual : nullptr, a->rstd, a->d_x,
               a->d_weight ? static_cast<float *>(a->workspace) : nullptr, a->T, a->H, a->ld_dy, a->ld_h, a->ld_d_residual,
               a->ld_d_x, (float)(1.0 / (double)a->H), a->weight_dtype == DVP_F32};
  const bool fast = a->H % kVec == 0 && vectors(a->dy, a->ld_dy, a->dy_dtype) && vectors(a->h, a->ld_h, a->h_dtype) &&
                    vectors(a->d_residual, a->ld_d_residual, a->h_dtype) && vectors(a->d_x, a->ld_d_x, a->h_dtype) &&
                    weight_vectors(a->weight);
  const cudaError_t e = by_type(a->h_dtype, [&](auto h) {
    return by_type(a->dy_dtype, [&](auto d) {
      return launch_backward<decltype(h), decltype(d)>(p, fast, a->d_weight, a->accumulate_dw, stream);
    });
  });
  return e == cudaSuccess ? DVP_OK : DVP_ERR_CUDA;
}

}  // extern "C"
