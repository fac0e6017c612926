// bf16 products of the gated feed-forward block and of its backward pass:  C[M,N] = sum_k A(m,k) B(n,k)  with fp32 sums.
//
// The block's weights are kept once, row = output feature, and forward and backward contract them over different axes, so an
// operand comes in one of two layouts:
//   kAlong   k runs along a row of memory:   (i, k) at i * ld + k        (rows times weights: X Wg^T, A Wd^T, the dY of dY Wd)
//   kAcross  k is the row of memory:         (i, k) at k * ld + i        (weights transposed: dY Wd, dG Wg; both in dG^T X)
// Neither is ever transposed in memory: a kAcross panel lies in LDS as it lies in memory, k by k, and its fragments are read
// with the transposing LDS read (ds_read_b64_tr_b16: 16 lanes point at 4 k x 16 i and get back 4 k of one i each).
//
// LDS panels of HB rows (i) x 64 k, filled by direct global->LDS loads of 1 KiB per wavefront (16 bytes per lane, lane-linear),
// so permutations against bank conflicts are applied to the lanes' global addresses:
//   kAlong   row i is 128 bytes, its 16-byte chunk c at position c ^ ((i >> 1) & 7): a fragment read (16 rows, one chunk) meets
//            every 16-byte column of the 64 banks once
//   kAcross  row k is 2 HB bytes, its 32-byte segment s at position s ^ f(k).  A transposing read serves 32 lanes at a time:
//            k = 0..3 and 8..11 of a step (then 4..7 and 12..15, ...), f gives those eight rows different segments modulo
//            256 bytes:  HB = 128: f = (k & 3) | (k >> 1 & 4);  HB = 64 (two rows per 256 bytes): f = (k >> 1 & 1) | (k >> 2 & 2)
// Ends: rows i past the end repeat the last one (their outputs are not stored, and an output takes nothing from another row);
// k past the end is loaded from 16 zero bytes in both operands, so whatever lies there (NaN included) stays out of the sums.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "lds_ring.h"

namespace lgemm {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

enum Layout { kAlong = 0, kAcross = 1 };
enum Epilogue {
  kGate,      // two products side by side: hidden = f(g) u in bf16, g and u in fp32 where asked for
  kStore,     // C in bf16 or fp32, plus a residual of the same type where asked for
  kGateGrad   // C = gradient of the hidden row: dG = C u f'(g), dU = C f(g) in bf16
};
enum Act { kSilu = 0, kGelu = 1 };

// Up to three products of one launch (the three weight gradients), or one.
struct Problem {
  const uint16_t* A[2];   // second pointer: the second K range (kStore), e.g. dX = dG Wg + dU Wu
  const uint16_t* B[2];   // kGate: gate and up weights; else as A
  int64_t lda, ldb;       // elements between rows of memory
  int M, N, K;            // K of one range; kGate: N is the hidden width
  int ranges;             // K ranges (1 or 2)
  void* out;              // kStore: C; kGate: hidden; kGateGrad: dG
  void* out2;             // kGateGrad: dU
  float* gates[2];        // kGate (out, or null) and kGateGrad (in): g and u
  const void* res;        // kStore: added to C, or null; same type and stride as out
  int64_t ldo;            // elements between rows of out / out2
  const int32_t* count;   // rows that count, at most M (device; null: M)
  const int32_t* rowidx;  // kStore: row m of C goes to row rowidx[m] of out (null: m); res is in the order of C
  int out_f32;            // kStore: type of out and res
  int tiles_m, tiles_n, tile0;
};

struct Args {
  Problem p[3];
  int problems, tiles;
  int act;
};

static __device__ const u32x4 g_zeros = {0, 0, 0, 0};

__device__ __forceinline__ float sigmoid(float x) { return __frcp_rn(1.0f + __expf(-x)); }

// f(g) and, for the backward pass, f'(g).  SiLU: g s, s + g s (1 - s).  GELU: g P, P + g p with the normal distribution's
// integral P (the library's erff) and density p.
__device__ __forceinline__ void activation(int act, float g, float& f, float& df) {
  if (act == kSilu) {
    const float s = sigmoid(g);
    f = g * s;
    df = s + f * (1.0f - s);
  } else {
    const float P = 0.5f * (1.0f + erff(g * 0.70710678118654752f));
    f = g * P;
    df = P + g * 0.39894228040143268f * __expf(-0.5f * g * g);
  }
}

__device__ __forceinline__ u32x2 pack_bf16(f32x4 v) {
  bf16x4 b;
#pragma unroll
  for (int e = 0; e < 4; ++e) b[e] = static_cast<__bf16>(v[e]);
  return __builtin_bit_cast(u32x2, b);
}

// ------------------------------------------------------------------------------------------------ panels
template <int HB>
__device__ __forceinline__ int segment_shift(int k) {
  return HB == 128 ? ((k & 3) | ((k >> 1) & 4)) : (((k >> 1) & 1) | ((k >> 2) & 2));
}

// Byte offset (from the panel's first element of the slice) of what this lane brings with load u of the panel, and its k.
template <int LAY, int HB>
__device__ __forceinline__ void lane_source(int u, int lane, int valid, int64_t ld, uint32_t& off, int& k) {
  if constexpr (LAY == kAlong) {
    const int row = 8 * u + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
    off = static_cast<uint32_t>((row < valid ? row : valid - 1) * ld * 2) + 16 * chunk;
    k = 8 * chunk;
  } else {
    constexpr int kChunks = HB / 8, kRowsPerLoad = 64 / kChunks;
    k = kRowsPerLoad * u + lane / kChunks;
    const int pos = lane % kChunks;
    const int col = (((pos >> 1) ^ segment_shift<HB>(k)) * 2 + (pos & 1)) * 8;
    off = static_cast<uint32_t>(k * ld * 2) + 2 * (col < valid ? col : valid - 8);
  }
}

typedef __attribute__((address_space(3))) unsigned char* lds_bytes;
typedef __attribute__((address_space(3))) void* lds_ptr;
typedef const __attribute__((address_space(1))) void* gbl_ptr;

// One load of a panel: `base` (uniform) is its first element at this slice, `left` the k's that remain from there.
__device__ __forceinline__ void load_panel(const unsigned char* base, uint32_t off, int k, int left, unsigned char* dst) {
  if (left >= 64) {
    __builtin_amdgcn_global_load_lds((gbl_ptr)(base + off), (lds_ptr)dst, 16, 0, 0);
  } else {
    const unsigned char* src = k < left ? base + off : reinterpret_cast<const unsigned char*>(&g_zeros);
    __builtin_amdgcn_global_load_lds((gbl_ptr)src, (lds_ptr)dst, 16, 0, 0);
  }
}

// Fragment of 16 rows i0 .. i0 + 15 (i0 a multiple of 16) at k step ks (32 wide): lane (l16, lq) gets row i0 + l16,
// k = 32 ks + 8 lq .. + 7.
template <int LAY, int HB>
__device__ __forceinline__ bf16x8 read_fragment(const unsigned char* panel, int i0, int ks, int l16, int lq) {
  if constexpr (LAY == kAlong) {
    const int row = i0 + l16;
    return *reinterpret_cast<const bf16x8*>(panel + row * 128 + (((4 * ks + lq) ^ (l16 >> 1)) << 4));
  } else {
    typedef __attribute__((address_space(3))) bf16x4* lds_b4;
    const int k = 32 * ks + 8 * lq + (l16 >> 2);            // k & 4 == 0: the second read's shift is the same
    const unsigned char* at = panel + k * (2 * HB) + (((i0 >> 4) ^ segment_shift<HB>(k)) << 5) + (l16 & 3) * 8;
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_b4)(at));
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_b4)(at + 4 * (2 * HB)));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}

// ------------------------------------------------------------------------------------------------ epilogue
// One row's four consecutive columns; kGate: g and u of the same four hidden columns.
template <int EPI>
__device__ __forceinline__ void store4(const Problem& p, int act, int64_t m, int n, f32x4 c, f32x4 c2) {
  int64_t at = m * p.ldo + n;
  if constexpr (EPI == kGate) {
    if (p.gates[0]) {
      const int64_t gat = m * p.N + n;
      *reinterpret_cast<f32x4*>(p.gates[0] + gat) = c;
      *reinterpret_cast<f32x4*>(p.gates[1] + gat) = c2;
    }
    f32x4 h;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float f, df;
      activation(act, c[e], f, df);
      h[e] = f * c2[e];
    }
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + at) = pack_bf16(h);
  } else if constexpr (EPI == kGateGrad) {
    const int64_t gat = m * p.N + n;
    const f32x4 g = *reinterpret_cast<const f32x4*>(p.gates[0] + gat), u = *reinterpret_cast<const f32x4*>(p.gates[1] + gat);
    f32x4 dg, du;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float f, df;
      activation(act, g[e], f, df);
      dg[e] = c[e] * u[e] * df;
      du[e] = c[e] * f;
    }
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + at) = pack_bf16(dg);
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out2) + at) = pack_bf16(du);
  } else {
    const int64_t rat = at;
    if (p.rowidx) at = static_cast<int64_t>(p.rowidx[m]) * p.ldo + n;
    if (p.out_f32) {
      if (p.res) c += *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.res) + rat);
      *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + at) = c;
    } else {
      if (p.res) {
        const bf16x4 r = *reinterpret_cast<const bf16x4*>(static_cast<const uint16_t*>(p.res) + rat);
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] += static_cast<float>(r[e]);
      }
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + at) = pack_bf16(c);
    }
  }
}

// Tile (tm, tn) of a workgroup.  Workgroups go round the eight XCDs, each with an L2 of its own: an XCD gets a contiguous
// share of the tiles, and walks it in patches of PM x PN tiles whose panels its L2 then serves.
template <int PM, int PN>
__device__ __forceinline__ bool pick_tile(const Args& a, int& which, int& tm, int& tn) {
  const int per_xcd = (a.tiles + 7) / 8;
  const int L = (blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
  if (blockIdx.x / 8 >= per_xcd || L >= a.tiles) return false;
  which = 0;
  if (a.problems > 1 && L >= a.p[1].tile0) which = 1;
  if (a.problems > 2 && L >= a.p[2].tile0) which = 2;
  const Problem& p = a.p[which];
  int l = L - p.tile0;
  // full rows of patches first come PM tiles high; the last one is as high as what is left
  const int band = l / (PM * p.tiles_n), h = p.tiles_m - band * PM < PM ? p.tiles_m - band * PM : PM;
  l -= band * PM * p.tiles_n;
  const int patch = l / (h * PN), left = p.tiles_n - patch * PN, w = left < PN ? left : PN;
  l -= patch * h * PN;
  tm = band * PM + l % h;
  tn = patch * PN + l / h;
  return w > 0;
}

// What a wavefront loads of one panel and where it comes from.
template <int LAY, int HB>
__device__ __forceinline__ const unsigned char* panel_base(const uint16_t* M, int64_t ld, int i0) {
  return reinterpret_cast<const unsigned char*>(M + (LAY == kAlong ? static_cast<int64_t>(i0) * ld : static_cast<int64_t>(i0)));
}

// ------------------------------------------------------------------------------------------------ 128 x 128 tile
// Four wavefronts of 64 x 64 (as 2 x 2 blocks of 32 x 32, one per pair of half panels, so that kGate's two products meet in
// one lane), two LDS stages of 32 KiB: two workgroups share a CU.
template <int EPI, int LA, int LB>
__global__ __launch_bounds__(256) void kernel128(Args a) {
  constexpr int HB = 64, kPanel = HB * 128, kStage = 4 * kPanel;
  __shared__ __align__(1024) unsigned char lds[2 * kStage];
  int which, tm, tn;
  if (!pick_tile<8, 8>(a, which, tm, tn)) return;
  const Problem& p = a.p[which];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave >> 1, wn = wave & 1, l16 = lane & 15, lq = lane >> 4;
  const int M = p.count ? (*p.count < p.M ? *p.count : p.M) : p.M;
  if (tm * 2 * HB >= M) return;
  const int m0 = tm * 2 * HB, n0 = tn * (EPI == kGate ? HB : 2 * HB);
  const int slices = (p.K + 63) / 64, nk = slices * p.ranges;

  // Wavefront w fills one panel per stage: A0, A1, B0, B1 (eight loads of 1 KiB).
  const bool is_b = wave >= 2;
  const int64_t ld = is_b ? p.ldb : p.lda;
  int i0, valid;
  if (!is_b) {
    i0 = m0 + wave * HB;
    valid = M - i0;
  } else {
    i0 = EPI == kGate ? n0 : n0 + (wave - 2) * HB;
    valid = p.N - i0;
  }
  if (valid <= 0) {               // a half panel past the end repeats the tile's first rows
    i0 = is_b ? n0 : m0;
    valid = (is_b ? p.N : M) - i0;
  }
  const uint16_t* src[2];
  src[0] = is_b ? (EPI == kGate ? p.B[wave - 2] : p.B[0]) : p.A[0];
  src[1] = is_b ? (EPI == kGate ? p.B[wave - 2] : p.B[1]) : p.A[1];
  auto fetch = [&](auto lay, int stage, int s) {
    constexpr int LAY = decltype(lay)::value;
    const int r = s >= slices, k0 = 64 * (s - r * slices);
    const unsigned char* base = panel_base<LAY, HB>(r ? src[1] : src[0], ld, i0) + static_cast<int64_t>(k0) * (LAY == kAlong ? 2 : 2 * ld);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      uint32_t off;
      int k;
      lane_source<LAY, HB>(u, lane, valid, ld, off, k);
      load_panel(base, off, k, p.K - k0, lds + stage * kStage + wave * kPanel + u * 1024);
    }
  };
  auto fetch_stage = [&](int stage, int s) {
    if (is_b) fetch(std::integral_constant<int, LB>{}, stage, s);
    else fetch(std::integral_constant<int, LA>{}, stage, s);
  };

  f32x4 acc[2][2][2][2];          // [A half][row block][B half][column block]
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i >> 3][(i >> 2) & 1][(i >> 1) & 1][i & 1] = f32x4{0.f, 0.f, 0.f, 0.f};

  if (nk > 0) fetch_stage(0, 0);
  for (int s = 0; s < nk; ++s) {
    const int stage = s & 1;
    if (s + 1 < nk) {
      fetch_stage(stage ^ 1, s + 1);
      ldsring::wait_loads<8>();
    } else {
      ldsring::wait_loads<0>();
    }
    ldsring::barrier_keep_loads();
    const unsigned char* base = lds + stage * kStage;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bf16x8 fa[2][2], fb[2][2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          fa[h][b] = read_fragment<LA, HB>(base + h * kPanel, wm * 32 + b * 16, ks, l16, lq);
          fb[h][b] = read_fragment<LB, HB>(base + (2 + h) * kPanel, wn * 32 + b * 16, ks, l16, lq);
        }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int ra = 0; ra < 2; ++ra)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int rb = 0; rb < 2; ++rb)
              acc[i][ra][j][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j][rb], fa[i][ra], acc[i][ra][j][rb], 0, 0, 0);
    }
    ldsring::barrier_keep_loads();          // every wavefront has read the stage: the next round may refill it
  }

#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int ra = 0; ra < 2; ++ra) {
      const int m = m0 + i * HB + wm * 32 + ra * 16 + l16;
      if (m >= M) continue;
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) {
        const int n = n0 + wn * 32 + rb * 16 + 4 * lq;
        if constexpr (EPI == kGate) {
          if (n < p.N) store4<EPI>(p, a.act, m, n, acc[i][ra][0][rb], acc[i][ra][1][rb]);
        } else {
          if (n < p.N) store4<EPI>(p, a.act, m, n, acc[i][ra][0][rb], acc[i][ra][0][rb]);
          if (n + HB < p.N) store4<EPI>(p, a.act, m, n + HB, acc[i][ra][1][rb], acc[i][ra][1][rb]);
        }
      }
    }
}

template <int EPI, int LA, int LB>
hipError_t launch(Args& a, hipStream_t st) {
  int total = 0;
  for (int i = 0; i < a.problems; ++i) {
    Problem& p = a.p[i];
    p.tiles_m = (p.M + 127) / 128;
    p.tiles_n = EPI == kGate ? (p.N + 63) / 64 : (p.N + 127) / 128;
    p.tile0 = total;
    total += p.tiles_m * p.tiles_n;
  }
  a.tiles = total;
  if (total == 0) return hipSuccess;
  hipLaunchKernelGGL((kernel128<EPI, LA, LB>), dim3((total + 7) / 8 * 8), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace lgemm
