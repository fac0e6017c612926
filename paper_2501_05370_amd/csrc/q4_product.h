// Rows times a matrix kept in 4 bits:  Y[r, n] = sum_k X[r, k] (q[n, k] - 8) s[n, k / group]  (+ bias), fp32 sums.
//
// What bounds a call of few rows is reading the weights once, here half a byte each plus one bf16 scale per group; with many rows
// it is the matrix cores.  Both kernels work on the bf16 matrix cores with the weights exactly as stored and scale the fp32
// sum of a group, so nothing is rounded but the sums:
//   unpacking   a byte 0 .. 15 read as an 8-bit float (e4m3) is q 2^-9: the subnormals and the first binade are one linear
//               scale.  The hardware's conversion of two such bytes to two bf16 with a scale of 2^9 gives q exactly: 7
//               instructions per 8 weights (two masks, a shift, four conversions)
//   the -8      the sum of a group starts from -8 sum(x), which a matrix instruction with a constant operand leaves in just the
//               layout of the sum; one such chain serves every 16 columns a wavefront computes on the same rows
//   fp32 rows   are three bf16 pieces (8 + 8 + 8 bits: exact) that take three rows of the tile; the epilogue adds them up
// The order of a sum is the same everywhere: within a group along k, the groups of the blocks b = i, i + 8, i + 16, ... (128 k
// each) in that order for i = 0 .. 7, and then those eight sums; so a row's result does not depend on the call it is part of.
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

namespace q4 {

using lgemm::bf16x4;
using lgemm::bf16x8;
using lgemm::f32x4;
using lgemm::u32x2;
using lgemm::u32x4;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// How rows enter: as they are, fp32 exactly (three pieces), fp32 rounded to bf16 first.
enum Rows { kBf16 = 0, kF32 = 1, kF32Rounded = 2 };
__host__ __device__ constexpr int pieces(int rows) { return rows == kF32 ? 3 : 1; }

struct Args {
  const u32x4* W;            // [ntiles, kblocks, 64]
  const uint16_t* S;         // [ntiles, kblocks, groups per block, 16] bf16
  int N, K, ntiles, kblocks;
  const void* X;
  int64_t ldx;
  int R;
  bool vec;                  // rows and strides allow 16-byte loads
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

constexpr int kShares = 8;       // partial sums of an output, see the top

// Eight values of a row from k on; past K they are 0.
template <int ROWS>
struct Chunk {
  typedef typename std::conditional<ROWS == kBf16, bf16x8, f32x4[2]>::type Raw;
};

template <int ROWS>
__device__ __forceinline__ void load_chunk(const Args& p, int64_t src, int k, typename Chunk<ROWS>::Raw& v) {
  if constexpr (ROWS == kBf16) {
    const __bf16* x = static_cast<const __bf16*>(p.X) + src * p.ldx + k;
    if (p.vec && k + 8 <= p.K) {
      v = *reinterpret_cast<const bf16x8*>(x);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = k + e < p.K ? x[e] : static_cast<__bf16>(0.f);
    }
  } else {
    const float* x = static_cast<const float*>(p.X) + src * p.ldx + k;
    if (p.vec && k + 8 <= p.K) {
      v[0] = *reinterpret_cast<const f32x4*>(x);
      v[1] = *reinterpret_cast<const f32x4*>(x + 4);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e >> 2][e & 3] = k + e < p.K ? x[e] : 0.f;
    }
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
    if constexpr (ROWS == kF32) {
      *reinterpret_cast<bf16x8*>(panel + lds_chunk(3 * row, c)) = hi;
      *reinterpret_cast<bf16x8*>(panel + lds_chunk(3 * row + 1, c)) = mid;
      *reinterpret_cast<bf16x8*>(panel + lds_chunk(3 * row + 2, c)) = lo;
    } else {
      *reinterpret_cast<bf16x8*>(panel + lds_chunk(row, c)) = hi;
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

constexpr float kMinus8 = -8.f;
__device__ __forceinline__ bf16x8 minus8() {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = static_cast<__bf16>(kMinus8);
  return v;
}

// ------------------------------------------------------------------------------------------------ few rows
// A workgroup computes 16 columns of up to 16 MT tile rows; its eight wavefronts take the blocks of 128 k in turn (together they
// stream the columns' blocks as they lie), each with its own panel of rows in LDS, and their sums meet in LDS at the end, in order.
// Weights are requested two blocks ahead, rows one, in registers: there is no barrier in the loop.
template <int MT, int GPB, int ROWS>
__global__ __launch_bounds__(512) void few_kernel(Args p) {
  constexpr int NW = kShares, kPanel = 16 * MT * 256, PIECES = pieces(ROWS), kRealRows = 16 * MT / PIECES;
  constexpr int kChunks = (kRealRows * 16 + 63) / 64;       // chunks of a block per lane
  __shared__ __align__(1024) unsigned char lds[NW * kPanel];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), l16 = lane & 15, lq = lane >> 4;
  // the row groups of a tile run on the same XCD, one after the other: its L2 serves the weights to all but the first
  const int groups = gridDim.x / ((p.ntiles + 7) / 8 * 8), id = blockIdx.x >> 3;
  const int tile = (id / groups) * 8 + (blockIdx.x & 7), group = id % groups;
  if (tile >= p.ntiles) return;
  const int M = p.count ? *p.count : p.R;
  const int row0 = group * kRealRows, rows = M - row0 < kRealRows ? M - row0 : kRealRows;
  if (rows <= 0) return;
  unsigned char* panel = lds + wave * kPanel;
  for (int i = lane; i < kPanel / 16; i += 64) *reinterpret_cast<u32x4*>(panel + 16 * i) = u32x4{0, 0, 0, 0};

  int src[kChunks];
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    const int r = (64 * i + lane) >> 4;
    src[i] = r < rows ? (p.gather ? p.rowidx[row0 + r] : row0 + r) : -1;
  }
  typedef typename Chunk<ROWS>::Raw Raw;
  Raw x[kChunks];
  auto fetch_rows = [&](int b) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i)
      if (src[i] >= 0) load_chunk<ROWS>(p, src[i], 128 * b + 8 * l16, x[i]);
  };
  const u32x4* W = p.W + (static_cast<int64_t>(tile) * p.kblocks) * 64 + lane;
  const uint16_t* S = p.S + static_cast<int64_t>(tile) * p.kblocks * GPB * 16 + 4 * lq;
  u32x4 w0{}, w1{}, w2{};
  u32x2 s0[GPB] = {}, s1[GPB] = {}, s2[GPB] = {};
  auto fetch_weights = [&](int b, u32x4& w, u32x2 (&s)[GPB]) {
    if (b < p.kblocks) {
      w = W[static_cast<int64_t>(b) * 64];
#pragma unroll
      for (int g = 0; g < GPB; ++g) s[g] = *reinterpret_cast<const u32x2*>(S + (static_cast<int64_t>(b) * GPB + g) * 16);
    }
  };
  f32x4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  int b = wave;
  fetch_weights(b, w0, s0);
  fetch_weights(b + NW, w1, s1);
  if (b < p.kblocks) fetch_rows(b);
  const bf16x8 m8 = minus8();
  for (; b < p.kblocks; b += NW) {
    fetch_weights(b + 2 * NW, w2, s2);
#pragma unroll
    for (int i = 0; i < kChunks; ++i)
      if (src[i] >= 0) put_chunk<ROWS>(panel, (64 * i + lane) >> 4, l16, x[i]);
    if (b + NW < p.kblocks) fetch_rows(b + NW);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int g = 0; g < GPB; ++g) {
      constexpr int J = 4 / GPB;
      bf16x8 wf[J];
#pragma unroll
      for (int j = 0; j < J; ++j) wf[j] = unpack(w0[g * J + j]);
      const f32x4 s = scales4(s0[g]);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        bf16x8 xf[J];
        f32x4 c{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < J; ++j) xf[j] = get_fragment(panel, 16 * i, g * J + j, l16, lq);
#pragma unroll
        for (int j = 0; j < J; ++j) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(m8, xf[j], c, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < J; ++j) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[j], xf[j], c, 0, 0, 0);
        acc[i] = add_scaled(acc[i], s, c);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    w0 = w1;
    w1 = w2;
#pragma unroll
    for (int g = 0; g < GPB; ++g) {
      s0[g] = s1[g];
      s1[g] = s2[g];
    }
  }

  // lane (l16, lq) holds columns 4 lq .. + 3 of tile row 16 i + l16
  __syncthreads();
  f32x4* sums = reinterpret_cast<f32x4*>(lds);               // [wavefront][tile row][4]
#pragma unroll
  for (int i = 0; i < MT; ++i) sums[(wave * 16 * MT + 16 * i + l16) * 4 + lq] = acc[i];
  __syncthreads();
  for (int e = t; e < rows * 4; e += 512) {
    const int r = e >> 2, q = e & 3;
    f32x4 c{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < PIECES; ++k) {
      f32x4 piece{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NW; ++i) piece += sums[(i * 16 * MT + PIECES * r + k) * 4 + q];
      c += piece;
    }
    const int n = 16 * tile + 4 * q;
    if (n < p.N) finish4(p, row0 + r, n, c);
  }
}

// ------------------------------------------------------------------------------------------------ many rows
// 128 tile rows x 128 columns, four wavefronts of 64 x 64; the rows of a block of 128 k are staged through registers (where fp32
// ones are split) into one of two LDS panels while the other is multiplied, weights go from memory into registers and are unpacked
// by the wavefront that multiplies them, a block ahead.
template <int GPB, int ROWS>
__global__ __launch_bounds__(256) void many_kernel(Args p) {
  constexpr int kPanel = 128 * 256, PIECES = pieces(ROWS), kRealRows = 128 / PIECES;
  constexpr int kChunks = (kRealRows * 16 + 255) / 256;
  __shared__ __align__(1024) unsigned char lds[2 * kPanel];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), l16 = lane & 15, lq = lane >> 4;
  const int wm = wave >> 1, wn = wave & 1;
  const int M = p.count ? *p.count : p.R;
  const int coltiles = (p.ntiles + 7) / 8, groups = gridDim.x / ((coltiles + 7) / 8 * 8), id = blockIdx.x >> 3;
  const int ct = (id / groups) * 8 + (blockIdx.x & 7), group = id % groups;
  const int row0 = group * kRealRows, rows = M - row0 < kRealRows ? M - row0 : kRealRows;
  if (ct >= coltiles || rows <= 0) return;
  typedef typename Chunk<ROWS>::Raw Raw;
  Raw x[kChunks];
  int src[kChunks];
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    int r = (256 * i + t) >> 4;
    if (r >= rows) r = rows - 1;                 // rows past the last repeat it: their sums are not stored
    src[i] = p.gather ? p.rowidx[row0 + r] : row0 + r;
  }
  if (PIECES * kRealRows < 128)                  // tile rows that no piece fills
    for (int i = t; i < (128 - PIECES * kRealRows) * 16; i += 256)
#pragma unroll
      for (int h = 0; h < 2; ++h) *reinterpret_cast<u32x4*>(lds + h * kPanel + PIECES * kRealRows * 256 + 16 * i) = u32x4{0, 0, 0, 0};
  auto fetch_rows = [&](int b) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) load_chunk<ROWS>(p, src[i], 128 * b + 8 * l16, x[i]);
  };
  auto put_rows = [&](int h) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i)
      if ((256 * i + t) >> 4 < kRealRows) put_chunk<ROWS>(lds + h * kPanel, (256 * i + t) >> 4, l16, x[i]);
  };
  u32x4 w[4], wnext[4];
  u32x2 s[4][GPB], snext[4][GPB];
  auto fetch_weights = [&](int b, u32x4 (&w)[4], u32x2 (&s)[4][GPB]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int nt = ct * 8 + wn * 4 + i;
      if (nt >= p.ntiles) nt = p.ntiles - 1;
      const int64_t at = static_cast<int64_t>(nt) * p.kblocks + b;
      w[i] = p.W[at * 64 + lane];
#pragma unroll
      for (int g = 0; g < GPB; ++g) s[i][g] = *reinterpret_cast<const u32x2*>(p.S + (at * GPB + g) * 16 + 4 * lq);
    }
  };
  f32x4 acc[4][4], total[4][4];
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i >> 2][i & 3] = total[i >> 2][i & 3] = f32x4{0.f, 0.f, 0.f, 0.f};
  fetch_rows(0);
  fetch_weights(0, w, s);
  put_rows(0);
  __syncthreads();
  const bf16x8 m8 = minus8();
  for (int b = 0, step = 0; step < p.kblocks; ++step) {
    int next = b + kShares;                      // the last block of a share: its sum is complete
    const bool share_ends = next >= p.kblocks, more = step + 1 < p.kblocks;
    if (share_ends) next = b % kShares + 1;
    if (more) {
      fetch_rows(next);
      fetch_weights(next, wnext, snext);
    }
    const unsigned char* panel = lds + (step & 1) * kPanel;
#pragma unroll
    for (int g = 0; g < GPB; ++g) {
      constexpr int J = 4 / GPB;
      bf16x8 xf[4][J];
      f32x4 c0[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        c0[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < J; ++j) {
          xf[i][j] = get_fragment(panel, wm * 64 + 16 * i, g * J + j, l16, lq);
          c0[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(m8, xf[i][j], c0[i], 0, 0, 0);
        }
      }
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        bf16x8 wf[J];
#pragma unroll
        for (int j = 0; j < J; ++j) wf[j] = unpack(w[n][g * J + j]);
        const f32x4 sc = scales4(s[n][g]);
        f32x4 c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = c0[i];
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) c[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[j], xf[i][j], c[i], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i][n] = add_scaled(acc[i][n], sc, c[i]);
      }
    }
    if (share_ends) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          total[i][n] += acc[i][n];
          acc[i][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    b = next;
    if (more) {
      put_rows((step + 1) & 1);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = wnext[i];
#pragma unroll
        for (int g = 0; g < GPB; ++g) s[i][g] = snext[i][g];
      }
    }
    __syncthreads();
  }
  if constexpr (PIECES == 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = wm * 64 + 16 * i + l16;
      if (r >= rows) continue;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        const int col = (ct * 8 + wn * 4 + n) * 16 + 4 * lq;
        if (col < p.N) finish4(p, row0 + r, col, total[i][n]);
      }
    }
  } else {
    // the pieces of a row are neighbouring tile rows: 64 KiB of LDS hold the tile for the sum
    f32x4* sums = reinterpret_cast<f32x4*>(lds);             // [tile row][32 groups of 4 columns]
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int n = 0; n < 4; ++n) sums[(wm * 64 + 16 * i + l16) * 32 + (wn * 4 + n) * 4 + lq] = total[i][n];
    __syncthreads();
    for (int e = t; e < rows * 32; e += 256) {
      const int r = e >> 5, q = e & 31, col = ct * 128 + 4 * q;
      const f32x4 c = (sums[(3 * r) * 32 + q] + sums[(3 * r + 1) * 32 + q]) + sums[(3 * r + 2) * 32 + q];
      if (col < p.N) finish4(p, row0 + r, col, c);
    }
  }
}

// ------------------------------------------------------------------------------------------------ layout
// q [N, ceil(K / 2)] (even k in the low half of a byte) and s [N, ceil(K / group)] -> W and S above; one thread per 16 bytes of W.
__global__ __launch_bounds__(256) void pack_kernel(const uint8_t* __restrict__ q, const uint16_t* __restrict__ s, int N, int K, int group,
                                                   int gpb, int ntiles, int kblocks, u32x4* __restrict__ W, uint16_t* __restrict__ S) {
  const int64_t id = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (id >= static_cast<int64_t>(ntiles) * kblocks * 64) return;
  const int lane = static_cast<int>(id & 63), l16 = lane & 15, lq = lane >> 4;
  const int64_t block = id >> 6;
  const int nt = static_cast<int>(block / kblocks), b = static_cast<int>(block % kblocks);
  const int n = nt * 16 + l16;
  const int64_t rowbytes = (K + 1) / 2;
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
    const int64_t groups = (K + group - 1) / group;
    S[(block * gpb + lq) * 16 + l16] = n < N && k < K ? s[n * groups + k / group] : static_cast<uint16_t>(0);
  }
}

}  // namespace q4
