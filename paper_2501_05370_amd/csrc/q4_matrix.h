// The device copy of a 4-bit matrix in the layout of q4_product.h, and the choice of the kernel for a call.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>

#include "q4_product.h"

namespace q4 {

constexpr int kMaxDim = 1 << 20;

constexpr int kRoundedRows = 32;      // most rows of a call with kF32Rounded

template <int MT, int GPB, int ROWS, int XC, int PF>
hipError_t launch_few(const Args& a, int R, hipStream_t st) {
  // 32 columns a workgroup where that still gives every CU one: the rows' panel is written once for both.  us, 32 / 16 columns, 4096 x 12288:
  // 32 staged rows, groups of 64 19.0 / 22.5; one row, groups of 32 15.8 / 12.6 (registers for one workgroup per CU)
  if constexpr (MT <= 2 && GPB <= 2) {
    if (a.ntiles >= 512) {                   // (one group of rows: see launch_rows)
      hipLaunchKernelGGL((few_kernel<MT, 2, GPB, ROWS, XC, PF>), dim3((a.ntiles + 1) / 2), dim3(64 * kShares), 0, st, a);
      return hipGetLastError();
    }
  }
  constexpr int kRows = 16 * MT / pieces(ROWS);
  hipLaunchKernelGGL((few_kernel<MT, 1, GPB, ROWS, XC, PF>), dim3(a.ntiles, (R + kRows - 1) / kRows), dim3(64 * kShares), 0, st, a);
  return hipGetLastError();
}

template <int GPB, int ROWS>
hipError_t launch_rows(const Args& a, int R, hipStream_t st) {
  constexpr int P = pieces(ROWS);
  if (R <= 4) return launch_few<1, GPB, ROWS, 1, 4>(a, R, st);
  // A lane stages one row in four: a tile of 16 rows has a form that stages 8, one of 32 a form that stages 24.  us with / without (the
  // whole tile's form, which takes the same time for any rows of it), bf16, 12288 x 4096 (groups of 128):
  // 8 rows 8.8 / 11.7, 19 rows 14.2 / 16.3; 4096 x 12288 (groups of 64): 8 rows 12.6 / 15.6, 19 rows 17.3 / 18.9
  if constexpr (P == 1) {
    if (R <= 8) return launch_few<1, GPB, ROWS, 2, 4>(a, R, st);
    if (R > 16 && R <= 24) return launch_few<2, GPB, ROWS, 6, 2>(a, R, st);
  }
  if (R <= 16 / P) return launch_few<1, GPB, ROWS, (16 / P + 3) / 4, ROWS == kF32Rounded ? 3 : 4>(a, R, st);
  if (R <= 32 / P) return launch_few<2, GPB, ROWS, (32 / P + 3) / 4, 2>(a, R, st);
  if constexpr (ROWS == kF32Rounded) {
    return hipErrorInvalidValue;
  } else {
    // More than 32 tile rows: groups of 64 with either kernel.  A workgroup of few_kernel (16 columns, one to a CU) takes an eighth of
    // the blocks of 128 k per wavefront, 2.1 us each and 2.5 us around them; one of many_kernel (128 columns, two to a CU, one for groups of 32)
    // all of them at 1 us (1.5).  us measured (bf16 rows), few / many:  12288 x 4096, 64 rows 28 / 89, 128 rows 57 / 90, 192 rows 83 / 92;  4096 x 4096, 64 rows
    // 13 / 38;  4096 x 12288, 64 rows 34 / 35, 128 rows 68 / 35.  fp32 rows (three tile rows each):  12288 x 4096, 21 rows 37 / 116, 42 rows
    // 68 / 116, 64 rows 124 / 118;  4096 x 12288, 21 rows 40 / 43, 42 rows 77 / 45;  4096 x 4096, groups of 64, 42 rows 28 / 46, 64 rows 53 / 46,
    // groups of 32, 64 rows 56 / 61, 128 rows 96 / 61;  the rule takes the shorter time in each.
    const int64_t row_groups = (R + 64 / P - 1) / (64 / P), few = row_groups * a.ntiles, many = row_groups * ((a.ntiles + 7) / 8);
    const double few_us = static_cast<double>((few + 255) / 256) * (2.1 * ((a.kblocks + kShares - 1) / kShares) + 2.5);
    const double many_us = GPB < 4 ? static_cast<double>((many + 511) / 512) * a.kblocks : 1.5 * static_cast<double>((many + 255) / 256) * a.kblocks;
    if (few_us < 1.1 * many_us && row_groups < 65536) return launch_few<4, GPB, ROWS, (64 / P + 3) / 4, ROWS == kF32 ? 2 : 1>(a, R, st);
    Args part = a;
    const int64_t most = many_groups(a.ntiles);
    for (int64_t g = 0; g < row_groups; g += most) {
      part.group0 = static_cast<int>(g);
      const int64_t groups = std::min(most, row_groups - g);
      hipLaunchKernelGGL((many_kernel<GPB, ROWS>), dim3(static_cast<unsigned>(many_columns(a.ntiles) * groups)), dim3(256), 0, st, part);
      if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
  }
}

template <int ROWS>
hipError_t launch_gpb(const Args& a, int gpb, int R, hipStream_t st) {
  return gpb == 1 ? launch_rows<1, ROWS>(a, R, st) : gpb == 2 ? launch_rows<2, ROWS>(a, R, st) : launch_rows<4, ROWS>(a, R, st);
}

}  // namespace q4

struct sdden_q4 {
  int N = 0, K = 0, gpb = 1, ntiles = 0, kblocks = 0, device = 0;
  q4::u32x4* W = nullptr;
  uint16_t* S = nullptr;

  ~sdden_q4() {
    if (W) (void)hipFree(W);
    if (S) (void)hipFree(S);
  }

  // Copies and lays out the host's matrix on the current device; waits for it (setup).
  hipError_t upload(int n, int k, int group, const uint8_t* q, const uint16_t* scale) {
    N = n;
    K = k;
    gpb = group >= 128 ? 1 : 128 / group;
    ntiles = (N + 15) / 16;
    kblocks = (K + 127) / 128;
    const size_t blocks = static_cast<size_t>(ntiles) * kblocks, qbytes = static_cast<size_t>(N) * ((K + 1) / 2);
    const size_t sbytes = static_cast<size_t>(N) * q4::groups_of(K, group) * 2;
    uint8_t* dq = nullptr;
    uint16_t* ds = nullptr;
    hipError_t e = hipGetDevice(&device);
    if (e == hipSuccess) e = hipMalloc(&W, blocks * 1024);
    if (e == hipSuccess) e = hipMalloc(&S, blocks * gpb * 32);
    if (e == hipSuccess) e = hipMalloc(&dq, qbytes);
    if (e == hipSuccess) e = hipMalloc(&ds, sbytes);
    if (e == hipSuccess) e = hipMemcpy(dq, q, qbytes, hipMemcpyHostToDevice);
    if (e == hipSuccess) e = hipMemcpy(ds, scale, sbytes, hipMemcpyHostToDevice);
    if (e == hipSuccess) {
      hipLaunchKernelGGL(q4::pack_kernel, dim3(q4::pack_grid(static_cast<int64_t>(blocks))), dim3(256), 0, nullptr, dq, ds, N, K, group,
                         gpb, ntiles, kblocks, W, S);
      e = hipGetLastError();
    }
    if (e == hipSuccess) e = hipStreamSynchronize(nullptr);      // callers' streams need not wait for the null stream
    if (dq) (void)hipFree(dq);
    if (ds) (void)hipFree(ds);
    return e;
  }

  void fill(q4::Args& a) const {
    a.W = W;
    a.S = S;
    a.N = N;
    a.K = K;
    a.ntiles = ntiles;
    a.kblocks = kblocks;
  }

  hipError_t launch(const q4::Args& a, int R, int rows, hipStream_t st) const {
    if (rows == q4::kBf16) return q4::launch_gpb<q4::kBf16>(a, gpb, R, st);
    if (rows == q4::kF32) return q4::launch_gpb<q4::kF32>(a, gpb, R, st);
    return q4::launch_gpb<q4::kF32Rounded>(a, gpb, R, st);
  }
};
