// Rows times a matrix kept in 4 bits:  Y[r, n] = sum_k X[r, k] (q[n, k] - 8) s[n, k / group]  (+ bias), fp32 sums.
//
// What bounds a call of few rows is reading the weights once, here half a byte each plus one bf16 scale per group; with many rows
// it is the matrix cores.  Both kernels work on the bf16 matrix cores with the weights exactly as stored and scale the fp32
// sum of a group, so nothing is rounded but the sums:
//   unpacking   a byte 0 .. 15 read as an 8-bit float (e4m3) is q 2^-9: the subnormals and the first binade are one linear
//               scale.  The hardware's conversion of two such bytes to two bf16 with a scale of 2^9 gives q exactly: 7
//               instructions per 8 weights (two masks, a shift, four conversions)
//   the -8      the sum of a group starts from -8 sum(x), which matrix instructions with a constant operand leave in just the
//               layout of the sum; one such chain serves all the columns a wavefront computes on the same rows.  (Summed by the
//               vector units as the rows are written to LDS, 512 rows x 4096 x 12288 take 92 us instead of 81: those bound the call.)
//   fp32 rows   are three bf16 pieces (8 + 8 + 8 bits: exact while the last bit is a normal bf16 number, |x| >= 2^-103) that take
//               three rows of the tile; the epilogue adds them up
//   range       a group's sum holds up to 8 |x| from its start and 15 |x| from the products, unscaled: 24 sum |x| < 2^128
// The order of a sum is the same everywhere: within a group along k, the groups of the blocks b = i, i + 8, i + 16, ... (128 k
// each) in that order for i = 0 .. 7, and then those eight sums; so a row's result does not depend on the call it is part of.
//
// Measured, us (matrices rotating through 75 MB, so from the memory-side cache at best): 12288 x 4096 (26 MB) one bf16 row 8.3, one
// fp32 row 10.9, 64 bf16 rows 28; 4096 x 12288 19 rows 17, 512 rows 81 (0.63 PFLOP/s of products, and half as many again for the -8), 512 fp32
// rows 267.  Registers: few_kernel<4, 1, 1, bf16, 16, 1> spills 44 bytes a lane, <2, 2, 1, rounded, 8, 2> 12, many_kernel<2, bf16> 20.
//
// Layout (made once, at create): 16 columns x 128 k are one block of 1 KiB, in which lane (l16, lq) finds its 16 bytes: dword
// j holds column l16, k = 32 j + 8 lq .. + 7, elements 0..3 in the low halves of its bytes and 4..7 in the high ones.  The blocks
// of 16 columns follow each other along k, their scales likewise as [128 / group][16] bf16 per block.  Columns and k past the
// ends are q = 8 with scale 0.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "layer_gemm.h"
#include "lds_ring.h"
#include "q4_shape.h"

namespace q4 {

using lgemm::bf16x4;
using lgemm::bf16x8;
using lgemm::f32x4;
using lgemm::u32x2;
using lgemm::u32x4;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// How rows enter: as they are, fp32 exactly (three pieces), fp32 rounded to bf16 first (a denoiser's call of up to 32 rows).
enum Rows { kBf16 = 0, kF32 = 1, kF32Rounded = 2 };
__host__ __device__ constexpr int pieces(int rows) { return rows == kF32 ? 3 : 1; }

struct Args {
  const u32x4* W;            // [ntiles, kblocks, 64]
  const uint16_t* S;         // [ntiles, kblocks, groups per block, 16] bf16
  int N, K, ntiles, kblocks;
  const void* X;
  int64_t ldx;
  int R;
  int group0;                // many_kernel: the launch's first group of rows
  const float* bias;         // [N], per-step table [T, N] with krow, or null
  void* Y;
  int64_t ldy;
  bool y_f32, vec_out;
  // evaluation of a denoiser: dense row m is source row rowidx[m] (X and Y, as flagged), m < *count
  const int32_t *rowidx, *count, *krow;
  bool gather, scatter, silu;
};

__device__ __forceinline__ bf16x8 unpack(uint32_t w) {
  const uint32_t lo = w & 0x0F0F0F0Fu, hi = (w >> 4) & 0x0F0F0F0Fu;
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.f, true);
  const bf16x4 l = __builtin_shufflevector(a, b, 0, 1, 2, 3), h = __builtin_shufflevector(c, d, 0, 1, 2, 3);
  return __builtin_shufflevector(l, h, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ f32x4 scales4(u32x2 s) {
  return f32x4{__uint_as_float(s[0] << 16), __uint_as_float(s[0] & 0xFFFF0000u), __uint_as_float(s[1] << 16), __uint_as_float(s[1] & 0xFFFF0000u)};
}

__device__ __forceinline__ f32x4 add_scaled(f32x4 a, f32x4 s, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) a[e] = __builtin_fmaf(s[e], c[e], a[e]);
  return a;
}

__device__ __forceinline__ bf16x8 minus8() {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = static_cast<__bf16>(-8.f);
  return v;
}

constexpr int kShares = 8;       // partial sums of an output, see the top
constexpr int kManyRows = 64;    // tile rows of many_kernel

// Eight values of a row from k on; past K they are 0.
struct F32x8 {
  f32x4 v[2];
  __device__ __forceinline__ f32x4& operator[](int i) { return v[i]; }
  __device__ __forceinline__ const f32x4& operator[](int i) const { return v[i]; }
};

template <int ROWS>
struct Chunk {
  typedef typename std::conditional<ROWS == kBf16, bf16x8, F32x8>::type Raw;
};

// It is loaded without a branch, 16 bytes at a time wherever the row starts (the hardware takes any alignment of the element type),
// from the row's last eight values where it ends behind K; in the last block finish_chunk replaces what such a load brought.
template <int ROWS>
__device__ __forceinline__ void load_chunk(const Args& p, int64_t src, int k, typename Chunk<ROWS>::Raw& v) {
  if (p.K < 8) return;                             // uniform; finish_chunk loads it
  typedef __bf16 any8 __attribute__((ext_vector_type(8), aligned(2)));
  typedef float any4 __attribute__((ext_vector_type(4), aligned(4)));
  const int at = k + 8 <= p.K ? k : p.K - 8;
  if constexpr (ROWS == kBf16) {
    v = *reinterpret_cast<const any8*>(static_cast<const __bf16*>(p.X) + src * p.ldx + at);
  } else {
    const float* x = static_cast<const float*>(p.X) + src * p.ldx + at;
    v[0] = *reinterpret_cast<const any4*>(x);
    v[1] = *reinterpret_cast<const any4*>(x + 4);
  }
}

template <int ROWS>
__device__ __forceinline__ void finish_chunk(const Args& p, int64_t src, int k, typename Chunk<ROWS>::Raw& v) {
  typedef typename std::conditional<ROWS == kBf16, __bf16, float>::type T;
  if (k + 8 <= p.K) return;
  const T* x = static_cast<const T*>(p.X) + src * p.ldx;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const T there = x[k + e < p.K ? k + e : p.K - 1], t = k + e < p.K ? there : static_cast<T>(0.f);
    if constexpr (ROWS == kBf16) v[e] = t;
    else v[e >> 2][e & 3] = t;
  }
}

// A row of 128 k is 256 bytes of LDS, all 64 banks: chunk c (8 k) of row v lies at c ^ (v & 15), so that a fragment read (16 rows,
// one chunk) and a row's write (one row, 16 chunks) both meet 16 different places.
__device__ __forceinline__ int lds_chunk(int v, int c) { return v * 256 + ((c ^ (v & 15)) << 4); }

// Writes the chunk's pieces into the rows pieces * row + 0 .. of the panel.
template <int ROWS>
__device__ __forceinline__ void put_chunk(unsigned char* panel, int row, int c, const typename Chunk<ROWS>::Raw& v) {
  if constexpr (ROWS == kBf16) {
    *reinterpret_cast<bf16x8*>(panel + lds_chunk(row, c)) = v;
  } else {
    bf16x8 hi, mid, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = v[e >> 2][e & 3];
      hi[e] = static_cast<__bf16>(x);
      if constexpr (ROWS == kF32) {
        const float r = x - static_cast<float>(hi[e]);
        mid[e] = static_cast<__bf16>(r);
        lo[e] = static_cast<__bf16>(r - static_cast<float>(mid[e]));
      }
    }
    const int first = ROWS == kF32 ? 3 * row : row;
    *reinterpret_cast<bf16x8*>(panel + lds_chunk(first, c)) = hi;
    if constexpr (ROWS == kF32) {
      *reinterpret_cast<bf16x8*>(panel + lds_chunk(first + 1, c)) = mid;
      *reinterpret_cast<bf16x8*>(panel + lds_chunk(first + 2, c)) = lo;
    }
  }
}

__device__ __forceinline__ bf16x8 get_fragment(const unsigned char* panel, int row0, int j, int l16, int lq) {
  return *reinterpret_cast<const bf16x8*>(panel + lds_chunk(row0 + l16, 4 * j + lq));
}

// One output row's columns n .. n + 3.
__device__ __forceinline__ void finish4(const Args& p, int m, int n, f32x4 c) {
  const int src = p.rowidx ? p.rowidx[m] : m;
  if (p.bias) {
    const float* b = p.krow ? p.bias + static_cast<int64_t>(p.krow[src]) * p.N : p.bias;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (n + e < p.N) c[e] += b[n + e];
  }
  if (p.silu) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c[e] *= lgemm::sigmoid(c[e]);
  }
  const int64_t at = static_cast<int64_t>(p.scatter ? src : m) * p.ldy + n;
  if (p.y_f32) {
    float* y = static_cast<float*>(p.Y) + at;
    if (p.vec_out && n + 4 <= p.N) {
      *reinterpret_cast<f32x4*>(y) = c;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < p.N) y[e] = c[e];
    }
  } else {
    __bf16* y = static_cast<__bf16*>(p.Y) + at;
    if (p.vec_out && n + 4 <= p.N) {
      *reinterpret_cast<u32x2*>(y) = lgemm::pack_bf16(c);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n + e < p.N) y[e] = static_cast<__bf16>(c[e]);
    }
  }
}

// ------------------------------------------------------------------------------------------------ few rows
// A workgroup computes 16 NT columns of up to 16 MT tile rows; its eight wavefronts take the blocks of 128 k in turn (together they
// stream the columns' blocks as they lie), each with its own panel of rows in LDS, and their sums meet in LDS at the end, in order.
// Weights and rows (XC chunks of 8 per lane: 4 XC rows) are requested PF blocks ahead in registers, PF being what these hold: both alike, as loads
// return in order and waiting for a row would wait for every weight requested before it.  There is no barrier in the loop.  Tile rows
// that no row of the call fills hold whatever was there: their sums are not used.
template <int MT, int NT, int GPB, int ROWS, int XC, int PF>
__global__ __launch_bounds__(64 * kShares) void few_kernel(Args p) {
  constexpr int NW = kShares, PIECES = pieces(ROWS), kRealRows = 16 * MT / PIECES, kChunks = XC;
  constexpr int kPanel = 16 * MT * 256;
  static_assert(4 * XC <= kRealRows + 3, "rows");
  static_assert(MT * NT * 16 * 64 <= kPanel, "the sums take the panels' place");
  __shared__ __align__(1024) unsigned char lds[NW * kPanel];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), l16 = lane & 15, lq = lane >> 4;
  const int tile0 = blockIdx.x * NT;
  const int row0 = blockIdx.y * kRealRows, M = (p.count ? (*p.count < p.R ? *p.count : p.R) : p.R) - row0;
  const int rows = M < kRealRows ? M : kRealRows;
  if (rows <= 0) return;
  unsigned char* panel = lds + wave * kPanel;
  const bf16x8 m8 = minus8();

  const u32x4* W[NT];
  const uint16_t* S[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t tile = tile0 + n < p.ntiles ? tile0 + n : p.ntiles - 1;
    W[n] = p.W + tile * p.kblocks * 64 + lane;
    S[n] = p.S + tile * p.kblocks * GPB * 16 + 4 * lq;
  }
  u32x4 w[PF][NT];
  u32x2 s[PF][NT][GPB];
  // what lies past the last block is requested again instead: no branch between the loads, which the compiler could only wait out
  auto fetch_weights = [&](int b, u32x4 (&w)[NT], u32x2 (&s)[NT][GPB]) {
    b = b < p.kblocks ? b : p.kblocks - 1;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      w[n] = W[n][static_cast<int64_t>(b) * 64];
#pragma unroll
      for (int g = 0; g < GPB; ++g) s[n][g] = *reinterpret_cast<const u32x2*>(S[n] + (static_cast<int64_t>(b) * GPB + g) * 16);
    }
  };
  int src[kChunks];
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    const int r = (64 * i + lane) >> 4, row = r < rows ? r : rows - 1;
    src[i] = p.gather ? p.rowidx[row0 + row] : row0 + row;
  }
  typedef typename Chunk<ROWS>::Raw Raw;
  Raw x[PF][kChunks];
  auto fetch_rows = [&](int b, Raw (&x)[kChunks]) {
    b = b < p.kblocks ? b : p.kblocks - 1;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) load_chunk<ROWS>(p, src[i], 128 * b + 8 * l16, x[i]);
  };
#pragma unroll
  for (int i = 0; i < PF; ++i) {
    fetch_weights(wave + i * NW, w[i], s[i]);
    fetch_rows(wave + i * NW, x[i]);
  }
  f32x4 acc[MT][NT] = {};
  for (int b0 = wave; b0 < p.kblocks; b0 += PF * NW) {
#pragma unroll
    for (int i = 0; i < PF; ++i) {
      const int b = b0 + i * NW;
      if (b >= p.kblocks) break;
      if (128 * b + 128 > p.K) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) finish_chunk<ROWS>(p, src[c], 128 * b + 8 * l16, x[i][c]);
      }
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
        if (4 * XC <= kRealRows || (64 * c + lane) >> 4 < kRealRows) put_chunk<ROWS>(panel, (64 * c + lane) >> 4, l16, x[i][c]);
      fetch_rows(b + PF * NW, x[i]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int g = 0; g < GPB; ++g) {
        constexpr int J = 4 / GPB;
        bf16x8 xf[MT][J];
        f32x4 c[MT][NT];
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            xf[m][j] = get_fragment(panel, 16 * m, g * J + j, l16, lq);
            c[m][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(m8, xf[m][j], j ? c[m][0] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
          }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int n = 1; n < NT; ++n) c[m][n] = c[m][0];
#pragma unroll
        for (int j = 0; j < J; ++j) {
          bf16x8 wf[NT];
#pragma unroll
          for (int n = 0; n < NT; ++n) wf[n] = unpack(w[i][n][g * J + j]);
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) c[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[n], xf[m][j], c[m][n], 0, 0, 0);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const f32x4 sc = scales4(s[i][n][g]);
#pragma unroll
          for (int m = 0; m < MT; ++m) acc[m][n] = add_scaled(acc[m][n], sc, c[m][n]);
        }
        if (GPB > 1) __builtin_amdgcn_sched_barrier(0);     // the groups one after the other: registers
      }
      fetch_weights(b + PF * NW, w[i], s[i]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }

  // lane (l16, lq) holds columns 4 lq .. + 3 of tile row 16 m + l16
  __syncthreads();
  f32x4* parts = reinterpret_cast<f32x4*>(lds);              // [wavefront][tile row][4 NT]
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n) parts[((wave * MT + m) * 16 + l16) * 4 * NT + 4 * n + lq] = acc[m][n];
  __syncthreads();
  for (int e = t; e < rows * 4 * NT; e += 64 * NW) {
    const int r = e / (4 * NT), q = e % (4 * NT);
    f32x4 c{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
      f32x4 piece{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NW; ++i) piece += parts[(i * 16 * MT + PIECES * r + k) * 4 * NT + q];
      c += piece;
    }
    const int n = 16 * tile0 + 4 * q;
    if (n < p.N) finish4(p, row0 + r, n, c);
  }
}

// ------------------------------------------------------------------------------------------------ many rows
// 64 tile rows x 128 columns, four wavefronts of 64 x 32, two workgroups to a CU whose phases overlap (one for groups of 32,
// whose registers two do not leave); the rows of a block of 128 k
// are staged through registers (where fp32 ones are split) into one of two LDS panels while the other is multiplied; weights go from memory into registers
// two blocks ahead, as rows do, and are unpacked by the wavefronts that multiply them.
template <int GPB, int ROWS>
__global__ __launch_bounds__(256, GPB < 4 ? 2 : 1) void many_kernel(Args p) {
  constexpr int kRows = kManyRows, kPanel = kRows * 256, PIECES = pieces(ROWS), kRealRows = kRows / PIECES;
  constexpr int kChunks = (kRealRows * 16 + 255) / 256;
  __shared__ __align__(1024) unsigned char lds[2 * kPanel];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), l16 = lane & 15, lq = lane >> 4;
  const int wn = wave;
  const int M = p.count ? (*p.count < p.R ? *p.count : p.R) : p.R;
  // the row groups of 128 columns run on the same XCD, one after the other: its L2 serves the weights to all but the first
  const int coltiles = (p.ntiles + 7) / 8, groups = gridDim.x / ((coltiles + 7) / 8 * 8), id = blockIdx.x >> 3;
  const int ct = (id / groups) * 8 + (blockIdx.x & 7), group = p.group0 + id % groups;
  const int row0 = group * kRealRows, rows = M - row0 < kRealRows ? M - row0 : kRealRows;
  if (ct >= coltiles || rows <= 0) return;
  typedef typename Chunk<ROWS>::Raw Raw;
  Raw x[2][kChunks];
  int src[kChunks];
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    int r = (256 * i + t) >> 4;
    if (r >= rows) r = rows - 1;                 // rows past the last repeat it: their sums are not used
    src[i] = p.gather ? p.rowidx[row0 + r] : row0 + r;
  }
  int64_t at[2];                                 // first block of this wavefront's 2 x 16 columns
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int nt = ct * 8 + wn * 2 + n;
    at[n] = static_cast<int64_t>(nt < p.ntiles ? nt : p.ntiles - 1) * p.kblocks;
  }
  u32x4 w[2][2];
  u32x2 s[2][2][GPB];
  // the blocks in the order of the sum, for the multiplication (b) and, ahead of it, for the loads of rows and weights; past the
  // last block some block is requested again: no branch between the loads, which the compiler could only wait out
  auto advance = [&](int b) {
    const int next = b + kShares < p.kblocks ? b + kShares : b % kShares + 1;
    return next < p.kblocks ? next : b;
  };
  int bx = 0, bw = 0, b = 0;
  auto fetch_rows = [&](Raw (&x)[kChunks]) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) load_chunk<ROWS>(p, src[i], 128 * bx + 8 * l16, x[i]);
    bx = advance(bx);
  };
  auto put_rows = [&](int h, int block, Raw (&x)[kChunks]) {
    if (128 * block + 128 > p.K) {
#pragma unroll
      for (int i = 0; i < kChunks; ++i) finish_chunk<ROWS>(p, src[i], 128 * block + 8 * l16, x[i]);
    }
#pragma unroll
    for (int i = 0; i < kChunks; ++i)
      if (256 * kChunks <= 16 * kRealRows || (256 * i + t) >> 4 < kRealRows) put_chunk<ROWS>(lds + h * kPanel, (256 * i + t) >> 4, l16, x[i]);
  };
  auto fetch_weights = [&](u32x4 (&w)[2], u32x2 (&s)[2][GPB]) {
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      w[n] = p.W[(at[n] + bw) * 64 + lane];
#pragma unroll
      for (int g = 0; g < GPB; ++g) s[n][g] = *reinterpret_cast<const u32x2*>(p.S + ((at[n] + bw) * GPB + g) * 16 + 4 * lq);
    }
    bw = advance(bw);
  };
  f32x4 acc[4][2] = {}, total[4][2] = {};
  const bf16x8 m8 = minus8();
  fetch_rows(x[0]);
  fetch_weights(w[0], s[0]);
  fetch_rows(x[1]);
  fetch_weights(w[1], s[1]);
  put_rows(0, 0, x[0]);
  fetch_rows(x[0]);
  __syncthreads();
  // step i of the sum from panel i & 1; the next step's rows, requested two steps ago, are written to the other panel meanwhile
  auto step = [&](int i, int h) {
    const int next = advance(b);
    put_rows(h ^ 1, next, x[h ^ 1]);             // (after the last step: not read)
    fetch_rows(x[h ^ 1]);
    const unsigned char* panel = lds + h * kPanel;
#pragma unroll
    for (int g = 0; g < GPB; ++g) {
      constexpr int J = 4 / GPB;
      bf16x8 xf[4][J];
      f32x4 c[4][2];
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          xf[m][j] = get_fragment(panel, 16 * m, g * J + j, l16, lq);
          c[m][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(m8, xf[m][j], j ? c[m][0] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
        }
#pragma unroll
      for (int m = 0; m < 4; ++m) c[m][1] = c[m][0];
      // eight independent chains side by side
#pragma unroll
      for (int j = 0; j < J; ++j) {
        bf16x8 wf[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) wf[n] = unpack(w[h][n][g * J + j]);
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
          for (int n = 0; n < 2; ++n) c[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[n], xf[m][j], c[m][n], 0, 0, 0);
      }
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const f32x4 sc = scales4(s[h][n][g]);
#pragma unroll
        for (int m = 0; m < 4; ++m) acc[m][n] = add_scaled(acc[m][n], sc, c[m][n]);
      }
      if (GPB > 1) __builtin_amdgcn_sched_barrier(0);       // the groups one after the other: registers
    }
    fetch_weights(w[h], s[h]);
    if (b + kShares >= p.kblocks) {              // the last block of a share: its sum is complete
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          total[m][n] += acc[m][n];
          acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    b = next;
    ldsring::barrier_keep_loads();               // __syncthreads would wait for the loads in flight
  };
  for (int i = 0; i < p.kblocks; i += 2) {
    step(i, 0);
    if (i + 1 < p.kblocks) step(i + 1, 1);
  }
  if constexpr (PIECES == 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 16 * i + l16;
      if (r >= rows) continue;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int col = (ct * 8 + wn * 2 + n) * 16 + 4 * lq;
        if (col < p.N) finish4(p, row0 + r, col, total[i][n]);
      }
    }
  } else {
    // the pieces of a row are neighbouring tile rows: the panels' 32 KiB hold the tile for their sum
    f32x4* parts = reinterpret_cast<f32x4*>(lds);            // [tile row][32 groups of 4 columns]
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int n = 0; n < 2; ++n) parts[(16 * i + l16) * 32 + (wn * 2 + n) * 4 + lq] = total[i][n];
    __syncthreads();
    for (int e = t; e < rows * 32; e += 256) {
      const int r = e >> 5, q = e & 31, col = ct * 128 + 4 * q;
      f32x4 c{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < PIECES; ++k) c += parts[(PIECES * r + k) * 32 + q];
      if (col < p.N) finish4(p, row0 + r, col, c);
    }
  }
}

// ------------------------------------------------------------------------------------------------ layout
// q [N, ceil(K / 2)] (even k in the low half of a byte) and s [N, ceil(K / group)] -> W and S above; one thread at a time per 16 bytes of W.
__global__ __launch_bounds__(256) void pack_kernel(const uint8_t* __restrict__ q, const uint16_t* __restrict__ s, int N, int K, int group,
                                                   int gpb, int ntiles, int kblocks, u32x4* __restrict__ W, uint16_t* __restrict__ S) {
  const int64_t rowbytes = (K + 1) / 2, groups = groups_of(K, group), total = static_cast<int64_t>(ntiles) * kblocks * 64;
  for (int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; id < total; id += static_cast<int64_t>(gridDim.x) * 256) {
    const int lane = static_cast<int>(id & 63), l16 = lane & 15, lq = lane >> 4;
    const int64_t block = id >> 6;
    const int nt = static_cast<int>(block / kblocks), b = static_cast<int>(block % kblocks);
    const int n = nt * 16 + l16;
    u32x4 out;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t v = 0;
      for (int e = 0; e < 8; ++e) {
        const int k = 128 * b + 32 * j + 8 * lq + e;
        uint32_t x = 8;
        if (n < N && k < K) {
          const uint8_t byte = q[n * rowbytes + (k >> 1)];
          x = k & 1 ? byte >> 4 : byte & 15;
        }
        v |= x << (8 * (e & 3) + 4 * (e >> 2));
      }
      out[j] = v;
    }
    W[id] = out;
    // lq is the group within the block where it has one
    if (lq < gpb) {
      const int k = 128 * b + (128 / gpb) * lq;
      S[(block * gpb + lq) * 16 + l16] = n < N && k < K ? s[n * groups + k / group] : static_cast<uint16_t>(0);
    }
  }
}

}  // namespace q4
