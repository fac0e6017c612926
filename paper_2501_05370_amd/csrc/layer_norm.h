// Layer norm over rows of d, forward and backward (sdden_layernorm_*).
//
//   xh = (x - mean) r,  r = 1 / sqrt(mean((x - mean)^2) + eps),  y = xh w + b
//   g = dy w:  dx = r (g - mean(g) - xh mean(g xh)) [+ dres],   dw = sum over rows dy xh,   db = sum over rows dy
//
// Bound by HBM: each row is read once and kept in registers (E elements per thread of the TPR threads that share a row), so the
// variance is the two-pass one, the sum of (x - m)^2 around the finished mean m, at no further traffic; everything between the
// loads and the stores is fp32.  m carries the roundings of a sum as large as the row's offset, so the sum of (x - m), taken with
// that of the squares, gives what it is off by (without it, rows at 1000 times their deviation had more than 1e-5 of it in every
// y).  Rows longer than the widest register form are walked in three passes, out of L2.
// Measured: 7680 fp32 rows of 12288 to bf16 121 us (4.7 TB/s; a copy by rows reaches 5.4), 16384 bf16 rows of 4096 forward 54 us
// (5.0 TB/s), backward with dres 99 us (5.4 TB/s, part of x still cached) and 7 us for the weights' gradients; one row 4 us.
// The weights' gradients need a sum over all rows: a workgroup walks rows blockIdx, blockIdx + grid, ... with its columns'
// sums in registers and leaves one partial row; reduce_partials_kernel adds those up in a fixed order (no atomics: the
// same bits every time).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "sd_lanes.h"

namespace lnorm {

struct Args {
  int R, d;
  const void *x, *dy, *dres;
  void* y;                      // forward: y; backward: dx
  int64_t ldx, lddy, lddres, ldy;
  const float *w, *b;           // may be null
  float* mean;                  // forward: out or null; backward: in
  float* rstd;
  float eps;
  float* partial;               // backward: [2, grid, d] or null
  const int32_t* count;         // forward: rows that count, at most R (device; null: R)
};

// V elements as they lie in memory, and as floats.
template <int V, typename T>
struct Raw {
  typedef T vec __attribute__((ext_vector_type(V), aligned(V * sizeof(T) < 16 ? V * sizeof(T) : 16)));
  typename std::conditional<V == 1, T, vec>::type v;
  __device__ __forceinline__ void load(const T* p) { v = *reinterpret_cast<const decltype(v)*>(p); }
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (V == 1) return static_cast<float>(v);
    else return static_cast<float>(v[e]);
  }
};

template <int V, typename T>
__device__ __forceinline__ void load(const T* p, float (&v)[V]) {
  Raw<V, T> r;
  r.load(p);
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = r[e];
}

// KEEP: into the caches, for the kernel that reads it next; else past them.  (A template: the compiler would make one ordinary
// store of the two sides of a branch.)
template <int V, bool KEEP, typename T>
__device__ __forceinline__ void store(T* p, const float (&v)[V]) {
  typedef typename Raw<V, T>::vec vec;
  if constexpr (V == 1) {
    *p = static_cast<T>(v[0]);
  } else {
    vec t;
#pragma unroll
    for (int e = 0; e < V; ++e) t[e] = static_cast<T>(v[e]);
    if constexpr (KEEP) *reinterpret_cast<vec*>(p) = t;
    else __builtin_nontemporal_store(t, reinterpret_cast<vec*>(p));
  }
}

using sdlane::wave_sum;

// Sum of a, or sums of a and b, over the TPR threads of a row; `slot` alternates between calls so that one barrier per call is enough.
template <int TPR>
__device__ __forceinline__ void row_sum(float& a, float2 (&red)[2][16], int slot) {
  a = wave_sum(a);
  if constexpr (TPR > 64) {
    constexpr int NW = TPR / 64;
    if ((threadIdx.x & 63) == 0) red[slot][threadIdx.x >> 6].x = a;
    __syncthreads();
    a = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) a += red[slot][w].x;
  }
}

template <int TPR>
__device__ __forceinline__ void row_sum2(float& a, float& b, float2 (&red)[2][16], int slot) {
  a = wave_sum(a);
  b = wave_sum(b);
  if constexpr (TPR > 64) {
    constexpr int NW = TPR / 64;
    if ((threadIdx.x & 63) == 0) red[slot][threadIdx.x >> 6] = make_float2(a, b);
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      a += red[slot][w].x;
      b += red[slot][w].y;
    }
  }
}

// From the mean square around a value that the mean is `off` from.  (A NaN stays one.)
__device__ __forceinline__ float rstd_of(float square, float off, float eps) {
  const float var = square - off * off;
  return 1.0f / sqrtf((var < 0.f ? 0.f : var) + eps);
}

constexpr int threads_of(int tpr) { return tpr < 256 ? 256 : tpr; }

// Columns of a thread: chunk c of V elements starts at (c * TPR + lane of the row) * V.
template <int TPR, int E, int V, bool KEEP, typename TX, typename TY>
__global__ __launch_bounds__(threads_of(TPR)) void forward_kernel(Args p) {
  if (p.count) p.R = *p.count < p.R ? *p.count : p.R;
  constexpr int C = E / V, RPB = threads_of(TPR) / TPR;
  __shared__ float2 red[2][16];
  const int t = threadIdx.x % TPR;
  const float inv_d = 1.0f / static_cast<float>(p.d);
  float w[C][V], b[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * TPR + t) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) w[c][e] = 1.f, b[c][e] = 0.f;
    if (col < p.d) {
      if (p.w) load<V>(p.w + col, w[c]);
      if (p.b) load<V>(p.b + col, b[c]);
    }
  }
  Raw<V, TX> raw[C];                    // the row that comes next: it is on its way during the sums and stores of this one
  auto fetch = [&](int64_t r) {
    const TX* x = static_cast<const TX*>(p.x) + r * p.ldx;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if ((c * TPR + t) * V < p.d) raw[c].load(x + (c * TPR + t) * V);
  };
  int64_t r = static_cast<int64_t>(blockIdx.x) * RPB + threadIdx.x / TPR;
  if (r < p.R) fetch(r);
  for (; r < p.R; r += static_cast<int64_t>(gridDim.x) * RPB) {
    float v[C][V];
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if ((c * TPR + t) * V < p.d) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          v[c][e] = raw[c][e];
          s += v[c][e];
        }
      }
    const int64_t next = r + static_cast<int64_t>(gridDim.x) * RPB;
    if (next < p.R) fetch(next);
    row_sum<TPR>(s, red, 0);
    const float about = s * inv_d;
    float q = 0.f, rest = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
      if ((c * TPR + t) * V < p.d) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          v[c][e] -= about;
          q += v[c][e] * v[c][e];
          rest += v[c][e];
        }
      }
    row_sum2<TPR>(q, rest, red, 1);
    const float off = rest * inv_d, rstd = rstd_of(q * inv_d, off, p.eps);
    if (t == 0 && p.mean) {
      p.mean[r] = about + off;
      p.rstd[r] = rstd;
    }
    TY* y = static_cast<TY*>(p.y) + r * p.ldy;
    const float shift = -off * rstd;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * TPR + t) * V;
      if (col < p.d) {
#pragma unroll
        for (int e = 0; e < V; ++e) v[c][e] = __builtin_fmaf(__builtin_fmaf(v[c][e], rstd, shift), w[c][e], b[c][e]);
        store<V, KEEP>(y + col, v[c]);
      }
    }
  }
}

// Rows of any length: three walks over the row, the second and third out of L2.
template <typename TX, typename TY>
__global__ __launch_bounds__(1024) void forward_long_kernel(Args p) {
  if (p.count) p.R = *p.count < p.R ? *p.count : p.R;
  __shared__ float2 red[2][16];
  for (int64_t r = blockIdx.x; r < p.R; r += gridDim.x) {
    const TX* x = static_cast<const TX*>(p.x) + r * p.ldx;
    TY* y = static_cast<TY*>(p.y) + r * p.ldy;
    float s = 0.f, q = 0.f;
    for (int c = threadIdx.x; c < p.d; c += 1024) s += static_cast<float>(x[c]);
    row_sum<1024>(s, red, 0);
    const float about = s / static_cast<float>(p.d);
    float rest = 0.f;
    for (int c = threadIdx.x; c < p.d; c += 1024) {
      const float v = static_cast<float>(x[c]) - about;
      q += v * v;
      rest += v;
    }
    row_sum2<1024>(q, rest, red, 1);
    const float off = rest / static_cast<float>(p.d), rstd = rstd_of(q / static_cast<float>(p.d), off, p.eps);
    if (threadIdx.x == 0 && p.mean) {
      p.mean[r] = about + off;
      p.rstd[r] = rstd;
    }
    for (int c = threadIdx.x; c < p.d; c += 1024) {
      const float w = p.w ? p.w[c] : 1.f, b = p.b ? p.b[c] : 0.f;
      y[c] = static_cast<TY>((static_cast<float>(x[c]) - about - off) * rstd * w + b);
    }
  }
}

// TY is dy's type, TX that of x, dres and dx.
template <int TPR, int E, int V, bool KEEP, typename TX, typename TY>
__global__ __launch_bounds__(threads_of(TPR)) void backward_kernel(Args p) {
  constexpr int C = E / V, RPB = threads_of(TPR) / TPR;
  __shared__ float2 red[2][16];
  __shared__ float fold[RPB > 1 ? (RPB - 1) * TPR * 2 : 1];
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const float inv_d = 1.0f / static_cast<float>(p.d);
  float w[C][V], dw[C][V], db[C][V];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * TPR + t) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) w[c][e] = 1.f, dw[c][e] = 0.f, db[c][e] = 0.f;
    if (col < p.d && p.w) load<V>(p.w + col, w[c]);
  }
  int slot = 0;
  for (int64_t r = static_cast<int64_t>(blockIdx.x) * RPB + sub; r < p.R; r += static_cast<int64_t>(gridDim.x) * RPB) {
    const TX* x = static_cast<const TX*>(p.x) + r * p.ldx;
    const TY* dy = static_cast<const TY*>(p.dy) + r * p.lddy;
    const float mean = p.mean[r], rstd = p.rstd[r];
    const TX* dres = p.dres ? static_cast<const TX*>(p.dres) + r * p.lddres : nullptr;
    Raw<V, TX> add[C];
    float xh[C][V], g[C][V];
    float sg = 0.f, sgx = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * TPR + t) * V;
      if (col < p.d) {
        load<V>(x + col, xh[c]);
        load<V>(dy + col, g[c]);
        if (dres) add[c].load(dres + col);
      }
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
      if ((c * TPR + t) * V < p.d) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
          xh[c][e] = (xh[c][e] - mean) * rstd;
          dw[c][e] += g[c][e] * xh[c][e];
          db[c][e] += g[c][e];
          g[c][e] *= w[c][e];
          sg += g[c][e];
          sgx += g[c][e] * xh[c][e];
        }
      }
    row_sum2<TPR>(sg, sgx, red, slot);
    slot ^= 1;
    sg *= inv_d;
    sgx *= inv_d;
    TX* dx = static_cast<TX*>(p.y) + r * p.ldy;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = (c * TPR + t) * V;
      if (col < p.d) {
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = rstd * (g[c][e] - sg - xh[c][e] * sgx);
        if (dres) {
#pragma unroll
          for (int e = 0; e < V; ++e) o[e] += add[c][e];
        }
        store<V, KEEP>(dx + col, o);
      }
    }
  }
  if (!p.partial) return;
  float* pw = p.partial + static_cast<int64_t>(blockIdx.x) * p.d;
  float* pb = pw + static_cast<int64_t>(gridDim.x) * p.d;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int col = (c * TPR + t) * V;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      float sw = dw[c][e], sb = db[c][e];
      if constexpr (RPB > 1) {          // several rows at a time: their sums meet in LDS first
        __syncthreads();
        if (sub > 0) {
          fold[((sub - 1) * TPR + t) * 2] = sw;
          fold[((sub - 1) * TPR + t) * 2 + 1] = sb;
        }
        __syncthreads();
        if (sub == 0) {
#pragma unroll
          for (int i = 0; i < RPB - 1; ++i) {
            sw += fold[(i * TPR + t) * 2];
            sb += fold[(i * TPR + t) * 2 + 1];
          }
        }
      }
      if (sub == 0 && col < p.d) {
        pw[col + e] = sw;
        pb[col + e] = sb;
      }
    }
  }
}

// Rows of any length, dx only; the weights' gradients are those of long_partials_kernel.
template <typename TX, typename TY>
__global__ __launch_bounds__(1024) void backward_long_kernel(Args p) {
  __shared__ float2 red[2][16];
  int slot = 0;
  for (int64_t r = blockIdx.x; r < p.R; r += gridDim.x) {
    const TX* x = static_cast<const TX*>(p.x) + r * p.ldx;
    const TY* dy = static_cast<const TY*>(p.dy) + r * p.lddy;
    const float mean = p.mean[r], rstd = p.rstd[r];
    float sg = 0.f, sgx = 0.f;
    for (int c = threadIdx.x; c < p.d; c += 1024) {
      const float g = static_cast<float>(dy[c]) * (p.w ? p.w[c] : 1.f);
      sg += g;
      sgx += g * ((static_cast<float>(x[c]) - mean) * rstd);
    }
    row_sum2<1024>(sg, sgx, red, slot);
    slot ^= 1;
    sg /= static_cast<float>(p.d);
    sgx /= static_cast<float>(p.d);
    TX* dx = static_cast<TX*>(p.y) + r * p.ldy;
    const TX* dres = p.dres ? static_cast<const TX*>(p.dres) + r * p.lddres : nullptr;
    for (int c = threadIdx.x; c < p.d; c += 1024) {
      const float g = static_cast<float>(dy[c]) * (p.w ? p.w[c] : 1.f);
      const float o = rstd * (g - sg - (static_cast<float>(x[c]) - mean) * rstd * sgx);
      dx[c] = static_cast<TX>(o + (dres ? static_cast<float>(dres[c]) : 0.f));
    }
  }
}

// Partial row blockIdx.y of long rows' weight gradients: rows blockIdx.y, + gridDim.y, ... of 256 columns per workgroup.
template <typename TX, typename TY>
__global__ __launch_bounds__(256) void long_partials_kernel(Args p) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= p.d) return;
  float sw = 0.f, sb = 0.f;
  for (int64_t r = blockIdx.y; r < p.R; r += gridDim.y) {
    const float v = static_cast<float>(static_cast<const TY*>(p.dy)[r * p.lddy + c]);
    sw += v * ((static_cast<float>(static_cast<const TX*>(p.x)[r * p.ldx + c]) - p.mean[r]) * p.rstd[r]);
    sb += v;
  }
  p.partial[static_cast<int64_t>(blockIdx.y) * p.d + c] = sw;
  p.partial[static_cast<int64_t>(gridDim.y + blockIdx.y) * p.d + c] = sb;
}

// dw[0..d) and db[0..d): sums of the P partial rows; 32 columns x 32 shares of the rows at a time per workgroup, eight loads of a
// share in flight.  Bound by latency: 1024 partial rows of 4096 (33 MB, just written) in 7 us.
constexpr int kReduceCols = 32;
// Workgroups of 1024 threads for d columns; a grid has to stay below 2^32 threads, so they walk the columns of wide rows.
inline unsigned reduce_grid(int d) { return d < kReduceCols << 20 ? (d + kReduceCols - 1) / kReduceCols : 1 << 20; }

__global__ __launch_bounds__(1024) void reduce_partials_kernel(const float* __restrict__ partial, int P, int d, float* __restrict__ dw,
                                                               float* __restrict__ db) {
  constexpr int kCols = kReduceCols, kShares = 32, kBatch = 8;
  __shared__ float sum[kShares][kCols + 1];
  const int lane = threadIdx.x % kCols, share = threadIdx.x / kCols;
  float* out = blockIdx.y ? db : dw;
  if (!out) return;
  for (int64_t col0 = static_cast<int64_t>(blockIdx.x) * kCols; col0 < d; col0 += static_cast<int64_t>(gridDim.x) * kCols) {
    const int64_t col = col0 + lane;
    const float* p = partial + static_cast<int64_t>(blockIdx.y) * P * d + (col < d ? col : d - 1);
    float s = 0.f;
    for (int i = share; i < P; i += kShares * kBatch) {
      float v[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) v[k] = i + k * kShares < P ? p[static_cast<int64_t>(i + k * kShares) * d] : 0.f;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) s += v[k];
    }
    sum[share][lane] = s;
    __syncthreads();
    if (share == 0 && col < d) {
      s = 0.f;
#pragma unroll
      for (int i = 0; i < kShares; ++i) s += sum[i][lane];
      out[col] = s;
    }
    __syncthreads();                     // the next columns' sums take these ones' place
  }
}

}  // namespace lnorm
