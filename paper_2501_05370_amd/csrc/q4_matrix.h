// The device copy of a 4-bit matrix in the layout of q4_product.h, and the choice of the kernel for a call.
#pragma once
#include <hip/hip_runtime.h>

#include "q4_product.h"

namespace q4 {

constexpr int kMaxDim = 1 << 20;

template <int GPB, int ROWS>
hipError_t launch_rows(const Args& a, int R, hipStream_t st) {
  constexpr int P = pieces(ROWS);
  const unsigned tiles = static_cast<unsigned>((a.ntiles + 7) / 8 * 8);
  if (R <= 64 / P) {
    if (R <= 16 / P) hipLaunchKernelGGL((few_kernel<1, GPB, ROWS>), dim3(tiles), dim3(512), 0, st, a);
    else if (R <= 32 / P) hipLaunchKernelGGL((few_kernel<2, GPB, ROWS>), dim3(tiles), dim3(512), 0, st, a);
    else hipLaunchKernelGGL((few_kernel<4, GPB, ROWS>), dim3(tiles), dim3(512), 0, st, a);
  } else {
    const int64_t grid = static_cast<int64_t>(((a.ntiles + 7) / 8 + 7) / 8 * 8) * ((R + 128 / P - 1) / (128 / P));
    if (grid > (int64_t{1} << 30)) return hipErrorInvalidValue;
    hipLaunchKernelGGL((many_kernel<GPB, ROWS>), dim3(static_cast<unsigned>(grid)), dim3(256), 0, st, a);
  }
  return hipGetLastError();
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
