// The device copy of a 4-bit matrix in the layout of q4_product.h, and the choice of the kernel for a call.
#pragma once
#include <hip/hip_runtime.h>

#include "q4_product.h"

namespace q4 {

constexpr int kMaxDim = 1 << 20;

constexpr int kRoundedRows = 32;      // most rows of a call with kF32Rounded

template <int MT, int GPB, int ROWS, int XC, int PF, bool VEC>
hipError_t launch_few(const Args& a, int R, hipStream_t st) {
  // 32 columns a workgroup where that still gives every CU one: the rows' panel is written once for both.  us, 32 / 16 columns, 4096 x 12288:
  // 19 rows, groups of 64 19.0 / 22.5; one row, groups of 32 15.8 / 12.6 (registers for one workgroup per CU)
  if constexpr (MT <= 2 && GPB <= 2 && VEC) {
    if (a.ntiles >= 512) {                   // (one group of rows: see launch_rows)
      hipLaunchKernelGGL((few_kernel<MT, 2, GPB, ROWS, XC, PF, VEC>), dim3((a.ntiles + 1) / 2), dim3(64 * kShares), 0, st, a);
      return hipGetLastError();
    }
  }
  constexpr int kRows = 16 * MT / pieces(ROWS);
  hipLaunchKernelGGL((few_kernel<MT, 1, GPB, ROWS, XC, PF, VEC>), dim3(a.ntiles, (R + kRows - 1) / kRows), dim3(64 * kShares), 0, st, a);
  return hipGetLastError();
}

template <int GPB, int ROWS, bool VEC>
hipError_t launch_rows(const Args& a, int R, hipStream_t st) {
  constexpr int P = pieces(ROWS);
  if (R <= 4) return launch_few<1, GPB, ROWS, 1, VEC ? 4 : 2, VEC>(a, R, st);
  if (R <= 16 / P) return launch_few<1, GPB, ROWS, (16 / P + 3) / 4, VEC ? ROWS == kF32Rounded ? 3 : 4 : 1, VEC>(a, R, st);
  if (R <= 32 / P) return launch_few<2, GPB, ROWS, (32 / P + 3) / 4, VEC ? 2 : 1, VEC>(a, R, st);
  if constexpr (ROWS == kF32Rounded) {
    return hipErrorInvalidValue;
  } else {
    // Up to three groups of 64 tile rows where 16 columns make at most one workgroup per CU: many_kernel has N / 128 workgroups for 64
    // tile rows then, and its time is that of one, us (bf16 rows, few / many): 12288 x 4096 64 rows 28 / 89, 128 rows 57 / 90;
    // 4096 x 4096 13 / 38.  With more columns it fills the chip: 4096 x 12288 64 rows 34 / 35, 128 rows 68 / 35.
    if (R <= 64 / P || (R <= 3 * (64 / P) && a.ntiles <= 256))
      return launch_few<4, GPB, ROWS, (64 / P + 3) / 4, ROWS == kF32 && VEC ? 2 : 1, VEC>(a, R, st);
    const int64_t grid = static_cast<int64_t>(((a.ntiles + 7) / 8 + 7) / 8 * 8) * ((R + kManyRows / P - 1) / (kManyRows / P));
    if (grid > (int64_t{1} << 30)) return hipErrorInvalidValue;
    hipLaunchKernelGGL((many_kernel<GPB, ROWS, VEC>), dim3(static_cast<unsigned>(grid)), dim3(256), 0, st, a);
    return hipGetLastError();
  }
}

template <int GPB, int ROWS>
hipError_t launch_vec(const Args& a, int R, hipStream_t st) {
  return a.vec && a.K % 8 == 0 ? launch_rows<GPB, ROWS, true>(a, R, st) : launch_rows<GPB, ROWS, false>(a, R, st);
}

template <int ROWS>
hipError_t launch_gpb(const Args& a, int gpb, int R, hipStream_t st) {
  return gpb == 1 ? launch_vec<1, ROWS>(a, R, st) : gpb == 2 ? launch_vec<2, ROWS>(a, R, st) : launch_vec<4, ROWS>(a, R, st);
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
    const size_t sbytes = static_cast<size_t>(N) * ((K + group - 1) / group) * 2;
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
      hipLaunchKernelGGL(q4::pack_kernel, dim3(static_cast<unsigned>((blocks * 64 + 255) / 256)), dim3(256), 0, nullptr, dq, ds, N, K, group,
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
