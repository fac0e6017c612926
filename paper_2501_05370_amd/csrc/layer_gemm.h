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
//            256 bytes:  HB = 128: f = (k & 3) | (k >> 1 & 4);  HB = 64 (two rows per 256 bytes): f = (k >> 1 & 1) | (k >> 2 & 2);
//            HB = 32 (four rows): f = k >> 3 & 1
// Every kernel below sums an output over k in one chain of 16x16x32 instructions and in order, whatever its tile: a row's result
// does not depend on how many rows a call has (tested; the instruction set does not promise it).
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
// integral P and density p.  P's tail is e^(-g^2 / 2) t A(t), t = 1 / (1 + 0.27 |g|): all its digits wherever the exponential has
// them, where (1 + erf(g / sqrt 2)) / 2 has none left below g = -5, and the exponential is p's.  A: least squares in the relative error,
// reweighted towards the smallest largest one, over |g| <= 14.5 where the tail leaves fp32; 2.4e-8 off at most, 4e-7 evaluated in fp32.
__device__ __forceinline__ void activation(int act, float g, float& f, float& df) {
  if (act == kSilu) {
    const float s = sigmoid(g);
    f = g * s;
    df = s + f * (1.0f - s);
  } else {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.27f, __builtin_fabsf(g), 1.0f)), e = __expf(-0.5f * g * g);
    float a = 0.028961092233657837f;
    a = __builtin_fmaf(a, t, -0.12648582458496094f);
    a = __builtin_fmaf(a, t, 0.16978608071804047f);
    a = __builtin_fmaf(a, t, -0.06921068578958511f);
    a = __builtin_fmaf(a, t, 0.10782558470964432f);
    a = __builtin_fmaf(a, t, 0.07204962521791458f);
    a = __builtin_fmaf(a, t, 0.10181060433387756f);
    a = __builtin_fmaf(a, t, 0.10754287242889404f);
    a = __builtin_fmaf(a, t, 0.10772065818309784f);
    const float tail = e * (t * a), P = g < 0.0f ? tail : 1.0f - tail;
    f = g * P;
    df = P + g * 0.39894228040143268f * e;
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
  return HB == 128 ? ((k & 3) | ((k >> 1) & 4)) : HB == 64 ? (((k >> 1) & 1) | ((k >> 2) & 2)) : ((k >> 3) & 1);
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

// A wavefront's fragments of two half panels of HB = 32 RB rows (f[(h RB + b) 2 + ks]: half h, block b of 16 rows, k step ks of 32):
// lane (l16, lq) gets row l16 of the block, k = 32 ks + 8 lq .. + 7.  `first`: the wavefront's first 16-row block in a half panel.
template <int LAY, int HB>
__device__ __forceinline__ void read_fragments(const unsigned char* panels, int first, int l16, int lq, bf16x8 (&f)[HB / 8]) {
  constexpr int RB = HB / 32;
  if constexpr (LAY == kAlong) {
#pragma unroll
    for (int i = 0; i < 4 * RB; ++i) {
      const int h = i / (2 * RB), b = (i >> 1) % RB, ks = i & 1;
      f[i] = *reinterpret_cast<const bf16x8*>(panels + h * HB * 128 + ((first + b) * 16 + l16) * 128 + (((4 * ks + lq) ^ (l16 >> 1)) << 4));
    }
  } else {
    // the reads and their wait are one block: the builtin would wait for every direct load in flight as well
    const int k = 8 * lq + (l16 >> 2);                      // + 32 ks, + 4: the shift is the same
    const uint32_t at = (uint32_t)(uintptr_t)((lds_bytes)panels) + k * 2 * HB + (l16 & 3) * 8;
    const uint32_t a0 = at + ((first ^ segment_shift<HB>(k)) << 5);
    u32x2 r[8 * RB];
#define LG_TWO(x, y, ad, o1, o2) "ds_read_b64_tr_b16 %" #x ", %" #ad " offset:" #o1 "\n\tds_read_b64_tr_b16 %" #y ", %" #ad " offset:" #o2 "\n\t"
#define LG_OUT8 "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
    if constexpr (RB == 2) {
      const uint32_t a1 = at + (((first + 1) ^ segment_shift<HB>(k)) << 5);
      asm volatile(LG_TWO(0, 1, 16, 0, 512) LG_TWO(2, 3, 16, 4096, 4608) LG_TWO(4, 5, 17, 0, 512) LG_TWO(6, 7, 17, 4096, 4608)
                   LG_TWO(8, 9, 16, 8192, 8704) LG_TWO(10, 11, 16, 12288, 12800) LG_TWO(12, 13, 17, 8192, 8704) LG_TWO(14, 15, 17, 12288, 12800)
                   "s_waitcnt lgkmcnt(0)"
                   : LG_OUT8, "=&v"(r[8]), "=&v"(r[9]), "=&v"(r[10]), "=&v"(r[11]), "=&v"(r[12]), "=&v"(r[13]), "=&v"(r[14]), "=&v"(r[15])
                   : "v"(a0), "v"(a1) : "memory");
    } else {
      asm volatile(LG_TWO(0, 1, 8, 0, 256) LG_TWO(2, 3, 8, 2048, 2304) LG_TWO(4, 5, 8, 4096, 4352) LG_TWO(6, 7, 8, 6144, 6400)
                   "s_waitcnt lgkmcnt(0)"
                   : LG_OUT8 : "v"(a0) : "memory");
    }
#undef LG_TWO
#undef LG_OUT8
#pragma unroll
    for (int i = 0; i < 4 * RB; ++i) f[i] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(r[2 * i], r[2 * i + 1], 0, 1, 2, 3));
  }
}

// ------------------------------------------------------------------------------------------------ epilogue
// hidden, dG and dU are rounded to bf16 because the product that follows takes its operands so: half the bytes, and one pass of the matrix
// cores where fp32 rows would need three.  g and u stay fp32 for the backward pass.  Y is then off by 0.0024 of its norm where one rounding
// of the result alone leaves 0.0017.
__device__ __forceinline__ void store_gate_grad(const Problem& p, int act, int64_t m, int n, f32x4 c, f32x4 g, f32x4 u) {
  f32x4 dg, du;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float f, df;
    activation(act, g[e], f, df);
    dg[e] = c[e] * u[e] * df;
    du[e] = c[e] * f;
  }
  const int64_t at = m * p.ldo + n;
  *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out) + at) = pack_bf16(dg);
  *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.out2) + at) = pack_bf16(du);
}

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
    store_gate_grad(p, act, m, n, c, *reinterpret_cast<const f32x4*>(p.gates[0] + gat), *reinterpret_cast<const f32x4*>(p.gates[1] + gat));
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

// ------------------------------------------------------------------------------------------------ small tiles
// 2 HB x 2 HB outputs by four wavefronts (of 2 x 2 blocks, one per pair of half panels, so that kGate's two products meet in one
// lane) and a ring of NS stages: HB = 64, 32 KiB a stage, two stages so that two workgroups share a CU, or four where there is one
// per CU or fewer; HB = 32, 16 KiB a stage, for products whose larger tiles would leave most CUs without one.
template <int EPI, int LA, int LB, int HB, int NS>
__global__ __launch_bounds__(256) void tile_kernel(Args a) {
  constexpr int kPanel = HB * 128, kStage = 4 * kPanel, RB = HB / 32, kOps = HB / 8;
  __shared__ __align__(1024) unsigned char lds[NS * kStage];
  int which, tm, tn;
  if (!pick_tile<8, 8>(a, which, tm, tn)) return;
  const Problem& p = a.p[which];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave >> 1, wn = wave & 1, l16 = lane & 15, lq = lane >> 4;
  const int M = p.count ? (*p.count < p.M ? *p.count : p.M) : p.M;
  if (tm * 2 * HB >= M) return;
  const int m0 = tm * 2 * HB, n0 = tn * (EPI == kGate ? HB : 2 * HB);
  const int slices = (p.K + 63) / 64, nk = slices * p.ranges;

  // Wavefront w fills one half panel per stage: A0, A1, B0, B1 (HB / 8 loads of 1 KiB).
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
    for (int u = 0; u < kOps; ++u) {
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

  f32x4 acc[2][RB][2][RB] = {};   // [A half][row block][B half][column block]

#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (s < nk) fetch_stage(s, s);
  int stage = 0, free_stage = NS - 1;
  for (int s = 0; s < nk; ++s) {
    // stage s has landed for this wavefront, and past the barrier for all, which have read stage s - 1: its place is refilled
    ldsring::wait_stages<kOps, NS - 2>(nk - 1 - s);
    ldsring::barrier_keep_loads();
    if (s + NS - 1 < nk) fetch_stage(free_stage, s + NS - 1);
    const unsigned char* base = lds + stage * kStage;
    bf16x8 fa[4 * RB], fb[4 * RB];
    read_fragments<LA, HB>(base, RB * wm, l16, lq, fa);
    read_fragments<LB, HB>(base + 2 * kPanel, RB * wn, l16, lq, fb);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int ra = 0; ra < RB; ++ra)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
              acc[i][ra][j][rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[(j * RB + rb) * 2 + ks], fa[(i * RB + ra) * 2 + ks], acc[i][ra][j][rb], 0, 0, 0);
    free_stage = stage;
    stage = stage + 1 == NS ? 0 : stage + 1;
  }

#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int ra = 0; ra < RB; ++ra) {
      const int m = m0 + i * HB + (wm * RB + ra) * 16 + l16;
      if (m >= M) continue;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int n = n0 + (wn * RB + rb) * 16 + 4 * lq;
        if constexpr (EPI == kGate) {
          if (n < p.N) store4<EPI>(p, a.act, m, n, acc[i][ra][0][rb], acc[i][ra][1][rb]);
        } else {
          if (n < p.N) store4<EPI>(p, a.act, m, n, acc[i][ra][0][rb], acc[i][ra][0][rb]);
          if (n + HB < p.N) store4<EPI>(p, a.act, m, n + HB, acc[i][ra][1][rb], acc[i][ra][1][rb]);
        }
      }
    }
}

// ------------------------------------------------------------------------------------------------ 256 x 256 tile
// The two wavefronts of a SIMD belong to two groups that run one phase apart: while one issues the 16 matrix instructions of a
// 64 x 32 quadrant of its 128 x 64 share, the other reads the next fragments and requests two direct loads; a workgroup
// barrier ends every phase.  (The schedule of mlp_gemm_pp.h, whose comment has its hazard table, over half panels of either
// layout: a tile's A0 / A1 are its first and last 128 rows, B0 / B1 its first and last 128 columns -- kGate: gate and up weights
// of the same 128 hidden columns -- so that a region is one panel whatever its layout.)
//   slice s, quadrants (A0,B0) (A0,B1) (A1,B1) (A1,B0); memory phases 0..3 read A0, B1, A1 and the next slice's B0 and refill,
//   with slice s + 2, the panel that both groups have just read for the last time: B0, A0, B1, A1.
// A memory phase is one asm block: its LDS reads, its two loads, then the wait for the reads and for the panel that is read
// next (12 younger loads may be outstanding), so that no register is in flight where the compiler could move it.  The builtin for
// the transposing read would wait for every load in flight.  The block sets m0 (the loads' place in LDS) itself; nothing behind it
// reads an older value: the builtin loads, which set their own, all come before the loop.
// 128 KiB of LDS, one workgroup per CU.  Bound by the clock that the power allows (the loop is that of mlp_gemm_pp.h) and, where an
// epilogue moves fp32 gates, by HBM while the matrix cores wait.  PFLOP/s: 7680 rows, d = 12288, H = 4096 first products 1.38, last
// 1.45; 8192 rows, d = 4096, H = 11008 with gates kept (0.9 GB written) 1.24, last 1.38, dA with the gates' gradients (0.7 GB read,
// 0.4 written) 0.86, dX 1.40, the three weight gradients in one launch 1.20 (2064 tiles: the ninth round of 256 is nearly empty).
template <int OFF, bool LD, int W>
__device__ __forceinline__ void phase_along8(u32x4 (&f)[8], uint32_t ad0, uint32_t ad1, const void* g0, const void* g1, uint32_t m0, uint32_t m1) {
#define LG_READS                                                                                                        \
  "ds_read_b128 %0, %8 offset:%10\n\tds_read_b128 %1, %9 offset:%10\n\tds_read_b128 %2, %8 offset:%11\n\t"               \
  "ds_read_b128 %3, %9 offset:%11\n\tds_read_b128 %4, %8 offset:%12\n\tds_read_b128 %5, %9 offset:%12\n\t"               \
  "ds_read_b128 %6, %8 offset:%13\n\tds_read_b128 %7, %9 offset:%13\n\t"
#define LG_OUT "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3]), "=&v"(f[4]), "=&v"(f[5]), "=&v"(f[6]), "=&v"(f[7])
#define LG_IN "v"(ad0), "v"(ad1), "n"(OFF), "n"(OFF + 2048), "n"(OFF + 4096), "n"(OFF + 6144), "n"(W)
  if constexpr (LD)
    asm volatile(LG_READS "s_mov_b32 m0, %17\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %15, off\n\ts_mov_b32 m0, %18\n\ts_nop 0\n\t"
                          "global_load_lds_dwordx4 %16, off\n\ts_waitcnt vmcnt(%14) lgkmcnt(0)"
                 : LG_OUT : LG_IN, "v"(g0), "v"(g1), "s"(m0), "s"(m1) : "memory");
  else
    asm volatile(LG_READS "s_waitcnt vmcnt(%14) lgkmcnt(0)" : LG_OUT : LG_IN : "memory");
#undef LG_READS
#undef LG_OUT
#undef LG_IN
}

template <int OFF, bool LD, int W>
__device__ __forceinline__ void phase_along4(u32x4 (&f)[4], uint32_t ad0, uint32_t ad1, const void* g0, const void* g1, uint32_t m0, uint32_t m1) {
#define LG_READS                                                                                           \
  "ds_read_b128 %0, %4 offset:%6\n\tds_read_b128 %1, %5 offset:%6\n\tds_read_b128 %2, %4 offset:%7\n\t"     \
  "ds_read_b128 %3, %5 offset:%7\n\t"
#define LG_OUT "=&v"(f[0]), "=&v"(f[1]), "=&v"(f[2]), "=&v"(f[3])
#define LG_IN "v"(ad0), "v"(ad1), "n"(OFF), "n"(OFF + 2048), "n"(W)
  if constexpr (LD)
    asm volatile(LG_READS "s_mov_b32 m0, %11\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %9, off\n\ts_mov_b32 m0, %12\n\ts_nop 0\n\t"
                          "global_load_lds_dwordx4 %10, off\n\ts_waitcnt vmcnt(%8) lgkmcnt(0)"
                 : LG_OUT : LG_IN, "v"(g0), "v"(g1), "s"(m0), "s"(m1) : "memory");
  else
    asm volatile(LG_READS "s_waitcnt vmcnt(%8) lgkmcnt(0)" : LG_OUT : LG_IN : "memory");
#undef LG_READS
#undef LG_OUT
#undef LG_IN
}

// 8 transposing reads: two blocks of 16 (address registers ad0, ad1), both k steps, both halves of 4 k.
// f[2 b + ks] of the caller; OFF: stage and panel.
template <int OFF, bool LD, int W>
__device__ __forceinline__ void phase_across4(u32x4 (&f)[4], uint32_t ad0, uint32_t ad1, const void* g0, const void* g1, uint32_t m0, uint32_t m1) {
  u32x2 r[8];
#define LG_READS                                                                                                        \
  "ds_read_b64_tr_b16 %0, %8 offset:%10\n\tds_read_b64_tr_b16 %1, %8 offset:%11\n\tds_read_b64_tr_b16 %2, %8 offset:%12\n\t" \
  "ds_read_b64_tr_b16 %3, %8 offset:%13\n\tds_read_b64_tr_b16 %4, %9 offset:%10\n\tds_read_b64_tr_b16 %5, %9 offset:%11\n\t" \
  "ds_read_b64_tr_b16 %6, %9 offset:%12\n\tds_read_b64_tr_b16 %7, %9 offset:%13\n\t"
#define LG_OUT "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
#define LG_IN "v"(ad0), "v"(ad1), "n"(OFF), "n"(OFF + 1024), "n"(OFF + 8192), "n"(OFF + 9216), "n"(W)
  if constexpr (LD)
    asm volatile(LG_READS "s_mov_b32 m0, %17\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %15, off\n\ts_mov_b32 m0, %18\n\ts_nop 0\n\t"
                          "global_load_lds_dwordx4 %16, off\n\ts_waitcnt vmcnt(%14) lgkmcnt(0)"
                 : LG_OUT : LG_IN, "v"(g0), "v"(g1), "s"(m0), "s"(m1) : "memory");
  else
    asm volatile(LG_READS "s_waitcnt vmcnt(%14) lgkmcnt(0)" : LG_OUT : LG_IN : "memory");
#undef LG_READS
#undef LG_OUT
#undef LG_IN
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = __builtin_shufflevector(r[2 * i], r[2 * i + 1], 0, 1, 2, 3);
}

template <int OFF, bool LD, int W>
__device__ __forceinline__ void phase_across8(u32x4 (&f)[8], const uint32_t (&ad)[4], const void* g0, const void* g1, uint32_t m0, uint32_t m1) {
  u32x2 r[16];
#define LG_FOUR(a, b, c, d, ad) \
  "ds_read_b64_tr_b16 %" #a ", %" #ad " offset:%20\n\tds_read_b64_tr_b16 %" #b ", %" #ad " offset:%21\n\tds_read_b64_tr_b16 %" #c ", %" #ad \
  " offset:%22\n\tds_read_b64_tr_b16 %" #d ", %" #ad " offset:%23\n\t"
#define LG_READS LG_FOUR(0, 1, 2, 3, 16) LG_FOUR(4, 5, 6, 7, 17) LG_FOUR(8, 9, 10, 11, 18) LG_FOUR(12, 13, 14, 15, 19)
#define LG_OUT                                                                                                                 \
  "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7]), "=&v"(r[8]), "=&v"(r[9]), \
      "=&v"(r[10]), "=&v"(r[11]), "=&v"(r[12]), "=&v"(r[13]), "=&v"(r[14]), "=&v"(r[15])
#define LG_IN "v"(ad[0]), "v"(ad[1]), "v"(ad[2]), "v"(ad[3]), "n"(OFF), "n"(OFF + 1024), "n"(OFF + 8192), "n"(OFF + 9216), "n"(W)
  if constexpr (LD)
    asm volatile(LG_READS "s_mov_b32 m0, %27\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %25, off\n\ts_mov_b32 m0, %28\n\ts_nop 0\n\t"
                          "global_load_lds_dwordx4 %26, off\n\ts_waitcnt vmcnt(%24) lgkmcnt(0)"
                 : LG_OUT : LG_IN, "v"(g0), "v"(g1), "s"(m0), "s"(m1) : "memory");
  else
    asm volatile(LG_READS "s_waitcnt vmcnt(%24) lgkmcnt(0)" : LG_OUT : LG_IN : "memory");
#undef LG_FOUR
#undef LG_READS
#undef LG_OUT
#undef LG_IN
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = __builtin_shufflevector(r[2 * i], r[2 * i + 1], 0, 1, 2, 3);
}

template <int EPI, int LA, int LB>
__global__ __launch_bounds__(512) void kernel256(Args a) {
  constexpr int HB = 128, kPanel = HB * 128;       // A stage s at 2 s kPanel, B stage s at 4 kPanel + 2 s kPanel
  __shared__ __align__(1024) unsigned char lds[8 * kPanel];
  int which, tm, tn;
  if (!pick_tile<4, 8>(a, which, tm, tn)) return;
  const Problem& p = a.p[which];
  const int M = p.count ? (*p.count < p.M ? *p.count : p.M) : p.M;
  const int m0 = tm * 2 * HB;
  if (m0 >= M) return;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave >> 2, wn = wave & 3, l16 = lane & 15, lq = lane >> 4;
  const int n0 = tn * (EPI == kGate ? HB : 2 * HB);
  const int K = p.K, slices = (K + 63) / 64;
  const int nk = (slices * p.ranges + 1) / 2 * 2 > 2 ? (slices * p.ranges + 1) / 2 * 2 : 2;   // even; slices past the end are zeros

  // this wavefront's loads u = 2 wave, 2 wave + 1 of the panels A0, A1, B0, B1
  uint32_t off[4][2];
  int kl[2][2];                                    // the lanes' k within a slice: of A and of B panels
  const unsigned char* base[4][2];                 // [panel][K range], uniform
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int am = m0 + h * HB, bn = EPI == kGate ? n0 : n0 + h * HB;
    int av = M - am, bv = p.N - bn;
    if (av <= 0) { am = m0; av = M - am; }         // a half panel past the end repeats the first one
    if (bv <= 0) { bn = n0; bv = p.N - bn; }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      lane_source<LA, HB>(2 * wave + e, lane, av, p.lda, off[h][e], kl[0][e]);
      lane_source<LB, HB>(2 * wave + e, lane, bv, p.ldb, off[2 + h][e], kl[1][e]);
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      base[h][r] = panel_base<LA, HB>(p.A[r < p.ranges ? r : 0], p.lda, am);
      base[2 + h][r] = panel_base<LB, HB>(EPI == kGate ? p.B[h] : p.B[r < p.ranges ? r : 0], p.ldb, bn);
    }
  }
  const int64_t stepa = LA == kAlong ? 128 : 128 * p.lda, stepb = LB == kAlong ? 128 : 128 * p.ldb;
  const uint32_t lds0 = (uint32_t)(uintptr_t)((lds_bytes)lds);

  // where this lane reads its fragments
  uint32_t a_ad[4], b_ad[2];
  if constexpr (LA == kAlong) {
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) a_ad[ks] = a_ad[2 + ks] = lds0 + (wm * 64 + l16) * 128 + (((4 * ks + lq) ^ (l16 >> 1)) << 4);
  } else {
#pragma unroll
    for (int b = 0; b < 4; ++b)
      a_ad[b] = lds0 + (8 * lq + (l16 >> 2)) * 256 + (((wm * 4 + b) ^ segment_shift<HB>(8 * lq + (l16 >> 2))) << 5) + (l16 & 3) * 8;
  }
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    if constexpr (LB == kAlong)
      b_ad[b] = lds0 + 4 * kPanel + (wn * 32 + l16) * 128 + (((4 * b + lq) ^ (l16 >> 1)) << 4);
    else
      b_ad[b] = lds0 + 4 * kPanel + (8 * lq + (l16 >> 2)) * 256 + (((wn * 2 + b) ^ segment_shift<HB>(8 * lq + (l16 >> 2))) << 5) + (l16 & 3) * 8;
  }

  f32x4 acc[2][4][2][2];                           // [A half][row block][B half][column block]
#pragma unroll
  for (int i = 0; i < 32; ++i) acc[i >> 4][(i >> 2) & 3][(i >> 1) & 1][i & 1] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 fa[8], bx[4], by[4];

  const unsigned char* zeros = reinterpret_cast<const unsigned char*>(&g_zeros);
  // addresses of this lane's two loads of panel P (0, 1: A0, A1; 2, 3: B0, B1) for slice s
#define LG_SRC(P, s, g0, g1)                                                                        \
  const unsigned char *g0, *g1;                                                                     \
  {                                                                                                 \
    const int r_ = (s) >= slices && p_ranges == 2, k0_ = 64 * ((s) - (r_ ? slices : 0)), left_ = K - k0_; \
    const unsigned char* b_ = (r_ ? base[P][1] : base[P][0]) + static_cast<int64_t>((s) - (r_ ? slices : 0)) * ((P) < 2 ? stepa : stepb); \
    g0 = kl[(P) / 2][0] < left_ ? b_ + off[P][0] : zeros;                                           \
    g1 = kl[(P) / 2][1] < left_ ? b_ + off[P][1] : zeros;                                           \
  }
  const int p_ranges = p.ranges;
  const uint32_t dst = lds0 + 2 * wave * 1024;
#define LG_DST(P, st) (dst + ((P) < 2 ? (st) * 2 * kPanel + (P) * kPanel : 4 * kPanel + (st) * 2 * kPanel + ((P) - 2) * kPanel))
#define LG_LOAD(P, st, s)                                                                                              \
  do {                                                                                                                 \
    LG_SRC(P, s, g0, g1);                                                                                              \
    __builtin_amdgcn_global_load_lds((gbl_ptr)g0, (lds_ptr)(lds + (LG_DST(P, st) - lds0)), 16, 0, 0);                   \
    __builtin_amdgcn_global_load_lds((gbl_ptr)g1, (lds_ptr)(lds + (LG_DST(P, st) - lds0) + 1024), 16, 0, 0);            \
  } while (0)
#define LG_PHASE_END()                        \
  do {                                        \
    __builtin_amdgcn_sched_barrier(0);        \
    asm volatile("s_barrier" ::: "memory");   \
    __builtin_amdgcn_sched_barrier(0);        \
  } while (0)
  // memory phase: fragments of A half h, or of B half h into F, from stage st; loads of panel P for slice s into stage ldst
#define LG_MEM_A(h, st, P, ldst, s, LD, W)                                                                                       \
  do {                                                                                                                           \
    LG_SRC(P, s, g0, g1);                                                                                                        \
    if constexpr (LA == kAlong)                                                                                                  \
      phase_along8<(st) * 2 * kPanel + (h) * kPanel, LD, W>(fa, a_ad[0], a_ad[1], g0, g1, LG_DST(P, ldst), LG_DST(P, ldst) + 1024);  \
    else                                                                                                                         \
      phase_across8<(st) * 2 * kPanel + (h) * kPanel, LD, W>(fa, a_ad, g0, g1, LG_DST(P, ldst), LG_DST(P, ldst) + 1024);             \
    LG_PHASE_END();                                                                                                              \
  } while (0)
#define LG_MEM_B(F, h, st, P, ldst, s, LD, W)                                                                                    \
  do {                                                                                                                           \
    LG_SRC(P, s, g0, g1);                                                                                                        \
    if constexpr (LB == kAlong)                                                                                                  \
      phase_along4<(st) * 2 * kPanel + (h) * kPanel, LD, W>(F, b_ad[0], b_ad[1], g0, g1, LG_DST(P, ldst), LG_DST(P, ldst) + 1024);   \
    else                                                                                                                         \
      phase_across4<(st) * 2 * kPanel + (h) * kPanel, LD, W>(F, b_ad[0], b_ad[1], g0, g1, LG_DST(P, ldst), LG_DST(P, ldst) + 1024);  \
    LG_PHASE_END();                                                                                                              \
  } while (0)
#define LG_COMPUTE(i, j, F)                                                                                              \
  do {                                                                                                                   \
    __builtin_amdgcn_s_setprio(1);                                                                                       \
    _Pragma("unroll") for (int ks_ = 0; ks_ < 2; ++ks_)                                                                  \
        _Pragma("unroll") for (int ta_ = 0; ta_ < 4; ++ta_)                                                              \
            _Pragma("unroll") for (int tb_ = 0; tb_ < 2; ++tb_)                                                          \
                acc[i][ta_][j][tb_] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(                                           \
                    __builtin_bit_cast(bf16x8, F[2 * tb_ + ks_]), __builtin_bit_cast(bf16x8, fa[2 * ta_ + ks_]),         \
                    acc[i][ta_][j][tb_], 0, 0, 0);                                                                       \
    __builtin_amdgcn_s_setprio(0);                                                                                       \
    LG_PHASE_END();                                                                                                      \
  } while (0)
  // One slice in stage st: X holds its B0 on entry, Y the next slice's B0 on exit (NX).
#define LG_SLICE(st, X, Y, s2, LD, NX, W0, W1, W2, W3)                                                  \
  do {                                                                                                  \
    LG_MEM_A(0, st, 2, st, s2, LD, W0);                                                                 \
    LG_COMPUTE(0, 0, X);                                                                                \
    LG_MEM_B(Y, 1, st, 0, st, s2, LD, W1);                                                              \
    LG_COMPUTE(0, 1, Y);                                                                                \
    LG_MEM_A(1, st, 3, st, s2, LD, W2);                                                                 \
    LG_COMPUTE(1, 1, Y);                                                                                \
    if (NX) LG_MEM_B(Y, 0, (st) ^ 1, 1, st, s2, LD, W3);                                                \
    else LG_PHASE_END();                                                                                \
    LG_COMPUTE(1, 0, X);                                                                                \
  } while (0)

  LG_LOAD(2, 0, 0); LG_LOAD(0, 0, 0); LG_LOAD(3, 0, 0); LG_LOAD(1, 0, 0);
  LG_LOAD(2, 1, 1); LG_LOAD(0, 1, 1); LG_LOAD(3, 1, 1); LG_LOAD(1, 1, 1);
  ldsring::wait_loads<8>();                        // slice 0 has landed
  ldsring::barrier_keep_loads();
  if constexpr (LB == kAlong) phase_along4<0, false, 8>(bx, b_ad[0], b_ad[1], nullptr, nullptr, 0, 0);
  else phase_across4<0, false, 8>(bx, b_ad[0], b_ad[1], nullptr, nullptr, 0, 0);
  LG_PHASE_END();                                  // every wavefront holds its B0 of slice 0: that panel may be refilled
  if (wm == 1) LG_PHASE_END();                     // the second group runs one phase behind
  int s = 0;
  for (; s + 3 < nk; s += 2) {
    LG_SLICE(0, bx, by, s + 2, true, true, 12, 12, 12, 12);
    LG_SLICE(1, by, bx, s + 3, true, true, 12, 12, 12, 12);
  }
  LG_SLICE(0, bx, by, 0, false, true, 10, 8, 6, 4);
  LG_SLICE(1, by, bx, 0, false, false, 2, 0, 0, 0);
  if (wm == 0) LG_PHASE_END();                     // equal numbers of barriers
#undef LG_SLICE
#undef LG_COMPUTE
#undef LG_MEM_A
#undef LG_MEM_B
#undef LG_PHASE_END
#undef LG_LOAD
#undef LG_DST
#undef LG_SRC

  if constexpr (EPI == kGateGrad) {
    // g and u of a block of 16 rows are requested while the block before it is computed and stored (a store could alias them for
    // the compiler, which would wait): 8192 rows, d = 4096, H = 11008 860 us, without it 900
    auto row_of = [&](int b) { return m0 + (b >> 2) * HB + wm * 64 + (b & 3) * 16 + l16; };
    auto col_of = [&](int c) { return n0 + (c >> 1) * HB + wn * 32 + (c & 1) * 16 + 4 * lq; };
    f32x4 g[2][4], u[2][4];
    auto request = [&](int b, f32x4 (&g)[4], f32x4 (&u)[4]) {
      const int64_t m = row_of(b) < M ? row_of(b) : M - 1;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int64_t at = m * p.N + (col_of(c) < p.N ? col_of(c) : 0);
        g[c] = *reinterpret_cast<const f32x4*>(p.gates[0] + at);
        u[c] = *reinterpret_cast<const f32x4*>(p.gates[1] + at);
      }
    };
    request(0, g[0], u[0]);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      if (b < 7) request(b + 1, g[(b + 1) & 1], u[(b + 1) & 1]);
      if (row_of(b) < M) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (col_of(c) < p.N) store_gate_grad(p, a.act, row_of(b), col_of(c), acc[b >> 2][b & 3][c >> 1][c & 1], g[b & 1][c], u[b & 1][c]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int ra = 0; ra < 4; ++ra) {
        const int m = m0 + i * HB + wm * 64 + ra * 16 + l16;
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
}

// ------------------------------------------------------------------------------------------------ few rows
// Up to 16 MT rows: what bounds the call is reading the weights once, and the tiles above would leave that to N / 128 workgroups.
// Here a workgroup computes 16 outputs (kGate: 16 of both products; WT = 2: 32) of every row, in the same order of k as the
// tiles -- the same bits -- with one wavefront per 16 rows and product, and keeps RING - 1 stages of 128 k on their way in a
// ring in LDS.  A stage holds the weights' rows and XR rows of the call, 256 bytes each, chunk c of row r at c ^ (r & 15); its
// loads are dealt to the wavefronts.  Rows the call does not have are not loaded, and what lies in their place reaches only sums
// that nobody stores.
template <int EPI, int MT, int WT, int XR, int RING>
__global__ __launch_bounds__(64 * MT * (EPI == kGate ? 2 : 1)) void few_kernel(Args a) {
  constexpr int G = EPI == kGate ? 2 : 1, NW = MT * G, kW = 16 * WT * G, kStage = (kW + XR) * 256, kOps = (kW + XR) / 4 / NW;
  static_assert((kW + XR) / 4 % NW == 0 && RING * kOps < 64 && RING * kStage <= 160 * 1024, "ring");
  static_assert((EPI != kGate || WT == 1) && XR <= 16 * MT && (XR == 16 * MT || MT == 1), "shape");
  __shared__ __align__(1024) unsigned char ring[RING * kStage];
  const Problem& p = a.p[0];
  const int M = p.count ? (*p.count < p.M ? *p.count : p.M) : p.M;
  if (M <= 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, lq = lane >> 4;
  const int mt = wave % MT, g = wave / MT;         // this wavefront's 16 rows and product
  const int n0 = blockIdx.x * 16 * WT, K = p.K, nk = (K + 127) / 128;
  const unsigned char* zeros = reinterpret_cast<const unsigned char*>(&g_zeros);
  // load u of a stage brings its rows 4 u .. 4 u + 3 (weights, then the call's): this lane row 4 u + lq, position l16
  const unsigned char* src[kOps];
  int kl[kOps];
  bool live[kOps];
#pragma unroll
  for (int i = 0; i < kOps; ++i) {
    const int row = 4 * (i * NW + wave) + lq, chunk = l16 ^ (row & 15);
    kl[i] = 8 * chunk;
    if (row < kW) {
      int n = n0 + row % (16 * WT);
      if (n >= p.N) n = p.N - 1;
      src[i] = reinterpret_cast<const unsigned char*>((row < 16 * WT ? p.B[0] : p.B[1]) + static_cast<int64_t>(n) * p.ldb + 8 * chunk);
      live[i] = true;
    } else {
      src[i] = reinterpret_cast<const unsigned char*>(p.A[0] + (row - kW) * p.lda + 8 * chunk);
      live[i] = row - kW < M;
    }
  }
  auto fetch = [&](int slot, int s) {
    const int left = K - 128 * s;
    const int64_t at = static_cast<int64_t>(s) * 256;
#pragma unroll
    for (int i = 0; i < kOps; ++i) {
      const unsigned char* from = src[i] + at;
      if (left < 128 && kl[i] >= left) from = zeros;
      // rows past M: the first lane loads zeros, so that a stage is always the same number of loads
      if ((i * NW + NW - 1) * 4 >= kW) {
        if (!live[i]) from = zeros;
        if (live[i] || lane == 0)
          __builtin_amdgcn_global_load_lds((gbl_ptr)from, (lds_ptr)(ring + slot * kStage + (i * NW + wave) * 1024), 16, 0, 0);
      } else {
        __builtin_amdgcn_global_load_lds((gbl_ptr)from, (lds_ptr)(ring + slot * kStage + (i * NW + wave) * 1024), 16, 0, 0);
      }
    }
  };
#pragma unroll
  for (int s = 0; s < RING; ++s)
    if (s < nk) fetch(s, s);
  f32x4 acc[WT];
#pragma unroll
  for (int j = 0; j < WT; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int xrow = XR < 16 ? l16 % XR : 16 * mt + l16;
  struct Fragments {
    bf16x8 w[4][WT], x[4];
  };
  auto read = [&](int slot, Fragments& f) {
    const unsigned char* base = ring + slot * kStage;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int n = 0; n < WT; ++n)
        f.w[j][n] = *reinterpret_cast<const bf16x8*>(base + (g * WT + n) * 4096 + l16 * 256 + (((4 * j + lq) ^ l16) << 4));
      f.x[j] = *reinterpret_cast<const bf16x8*>(base + kW * 256 + xrow * 256 + (((4 * j + lq) ^ (xrow & 15)) << 4));
    }
  };
  auto join = [&]() {                              // the reads of this wavefront are done, and past it those of all
    if (NW > 1) ldsring::barrier_keep_loads();
    else ldsring::wait_reads();
  };
  Fragments now, next;
  ldsring::wait_stages<kOps, RING - 1>(nk - 1);
  join();
  read(0, now);
  int slot = 0;
  for (int s = 0; s < nk; ++s) {
    const int after = slot + 1 == RING ? 0 : slot + 1;
    // stage s + 1 has landed for this wavefront, and past the barrier for all; stage s is in registers and its slot free
    ldsring::wait_stages<kOps, RING - 2>(nk - 2 - s > 0 ? nk - 2 - s : 0);
    join();
    if (s + 1 < nk) read(after, next);
    if (s + RING < nk) fetch(slot, s + RING);
    __builtin_amdgcn_sched_barrier(0);             // both are on their way before the products
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int n = 0; n < WT; ++n) acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(now.w[j][n], now.x[j], acc[n], 0, 0, 0);
    now = next;
    slot = after;
  }
  f32x4 up{0.f, 0.f, 0.f, 0.f};
  if constexpr (EPI == kGate) {                    // the up product comes over from its wavefront
    __syncthreads();
    f32x4* sums = reinterpret_cast<f32x4*>(ring);
    if (g == 1) sums[mt * 64 + lane] = acc[0];
    __syncthreads();
    if (g == 1) return;
    up = sums[mt * 64 + lane];
  }
  const int row = 16 * mt + l16;
  if (row >= M) return;
#pragma unroll
  for (int n = 0; n < WT; ++n) {
    const int col = n0 + 16 * n + 4 * lq;
    if (col < p.N) store4<EPI>(p, a.act, row, col, acc[n], up);
  }
}

template <int EPI, int MT, int WT, int XR, int RING>
hipError_t launch_few(const Args& a, hipStream_t st) {
  hipLaunchKernelGGL((few_kernel<EPI, MT, WT, XR, RING>), dim3((a.p[0].N + 16 * WT - 1) / (16 * WT)), dim3(64 * MT * (EPI == kGate ? 2 : 1)), 0,
                     st, a);
  return hipGetLastError();
}

// Calls of up to 64 rows.  The ring is as deep as the LDS of a CU allows for the workgroups that share it.  us, both products
// (302 MB of weights at d = 12288, H = 4096): 1 row 39 + 22 (5 TB/s), 16 rows 43 + 24, 32 rows 48 + 25, 64 rows 59 + 32, where the
// tiles below take 144 + 52 for any of them; H = 11008, d = 4096: 1 row 34 + 27, 64 rows 48 + 45 (72 + 112).
template <int EPI>
hipError_t launch_few_rows(const Args& a, hipStream_t st) {
  const int M = a.p[0].M, tiles = (a.p[0].N + 15) / 16;
  const bool one = tiles <= 256;                   // one workgroup per CU
  if constexpr (EPI == kGate) {
    if (M <= 8) return one ? launch_few<EPI, 1, 1, 8, 12>(a, st) : launch_few<EPI, 1, 1, 8, 5>(a, st);
    if (M <= 16) return one ? launch_few<EPI, 1, 1, 16, 10>(a, st) : launch_few<EPI, 1, 1, 16, 4>(a, st);
    if (M <= 32) return one ? launch_few<EPI, 2, 1, 32, 9>(a, st) : launch_few<EPI, 2, 1, 32, 3>(a, st);
    return one ? launch_few<EPI, 4, 1, 64, 6>(a, st) : launch_few<EPI, 4, 1, 64, 3>(a, st);
  } else {
    if (M <= 4) return one ? launch_few<EPI, 1, 1, 4, 12>(a, st) : launch_few<EPI, 1, 1, 4, 10>(a, st);
    if (M <= 16) return one ? launch_few<EPI, 1, 1, 16, 7>(a, st) : launch_few<EPI, 1, 1, 16, 6>(a, st);
    if (M <= 32) return one ? launch_few<EPI, 2, 1, 32, 9>(a, st) : launch_few<EPI, 2, 1, 32, 4>(a, st);
    return one ? launch_few<EPI, 4, 1, 64, 7>(a, st) : launch_few<EPI, 4, 2, 64, 3>(a, st);
  }
}

// Tiles of edge T over all problems; sets their numbers.
template <int EPI>
int count_tiles(Args& a, int T) {
  int total = 0;
  for (int i = 0; i < a.problems; ++i) {
    Problem& p = a.p[i];
    const int tn = EPI == kGate ? T / 2 : T;
    p.tiles_m = (p.M + T - 1) / T;
    p.tiles_n = (p.N + tn - 1) / tn;
    p.tile0 = total;
    total += p.tiles_m * p.tiles_n;
  }
  return a.tiles = total;
}

template <int EPI, int LA, int LB>
hipError_t launch(Args& a, hipStream_t st) {
  if constexpr (EPI != kGateGrad && LA == kAlong && LB == kAlong) {
    if (a.p[0].M > 0 && a.p[0].M <= 64) return launch_few_rows<EPI>(a, st);
  }
  const int t256 = count_tiles<EPI>(a, 256);
  if (t256 == 0) return hipSuccess;
  // The tile, by how well the launch fills the 256 CUs (all of them give the same bits).  256 x 256 has the highest rate per CU
  // and a CU to itself: where its rounds of 256 workgroups are at least 60 % full.  64 x 64 where 128 x 128 would leave half of
  // the CUs idle, or, with short sums, one workgroup on each with nothing to overlap its start and its epilogue with.  us, 64 x 64 / 128 x 128:
  //   first products, d = 12288, H = 4096   129 rows (128 tiles of 128) 100 / 140   300 rows (192) 158 / 139   512 rows (256) 212 / 144
  //   last product, H = 11008, d = 4096     129 rows (64) 70 / 112   512 rows (128) 96 / 115
  //   weight gradients, d = H = 1024        1024 rows (192) 15.7 / 18.5   1500 rows (192) 21.0 / 24.2;   d = 1024, H = 2048, 2048 rows (384) 47 / 35
  //   first products, d = 520, H = 1352     777 rows (154) 13.4 / 17.5;   d = H = 512, 4096 rows (256) 14.5 / 14.6
  if (10 * static_cast<int64_t>(t256) >= 6 * ((t256 + 255) / 256) * int64_t{256}) {
    hipLaunchKernelGGL((kernel256<EPI, LA, LB>), dim3((t256 + 7) / 8 * 8), dim3(512), 0, st, a);
    return hipGetLastError();
  }
  const int t128 = count_tiles<EPI>(a, 128);
  if (t128 <= 128 || (t128 <= 256 && static_cast<int64_t>(a.p[0].K) * a.p[0].ranges <= 2048)) {
    const int t64 = count_tiles<EPI>(a, 64);
    hipLaunchKernelGGL((tile_kernel<EPI, LA, LB, 32, 3>), dim3((t64 + 7) / 8 * 8), dim3(256), 0, st, a);
  } else if (t128 <= 256) {
    hipLaunchKernelGGL((tile_kernel<EPI, LA, LB, 64, 4>), dim3((t128 + 7) / 8 * 8), dim3(256), 0, st, a);
  } else {
    hipLaunchKernelGGL((tile_kernel<EPI, LA, LB, 64, 2>), dim3((t128 + 7) / 8 * 8), dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace lgemm
