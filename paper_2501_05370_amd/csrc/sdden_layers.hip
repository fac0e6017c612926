// The layers of row networks behind sdden.h: layer norm (layer_norm.h) and the gated feed-forward block (layer_gemm.h), each
// forward and backward.  Plain calls without a handle: the caller owns every buffer, nothing is kept between calls.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <exception>
#include <memory>
#include <vector>

#include "layer_gemm.h"
#include "layer_norm.h"
#include "sdden_internal.h"
#include "sdden_rows.h"
#include "time_table.h"

namespace {

#define LAYER_ERR sdi::g_den_create_error

bool type_ok(int32_t t) { return t == SDDEN_F32 || t == SDDEN_BF16; }
bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
size_t size_of(int32_t t) { return t == SDDEN_F32 ? 4 : 2; }

// ------------------------------------------------------------------------------------------------ layer norm
constexpr int32_t kMaxRows = 1 << 30, kMaxWidth = 1 << 30;       // of a call: sums of sizes stay within 32 bits

// Threads per row and elements per thread by width: a wavefront up to 1024 columns (four rows to a workgroup), then the
// smallest workgroup whose registers hold the row in the forward pass.  The backward pass holds x, dy, the weight and two sums of
// each column, and some of its forms spill: 1024 threads, element by element (40 to 68 bytes a lane) and with bf16 x and fp32 dy (36),
// 512 threads element by element with mixed types (36 and 92).  4096 rows forward and backward, us: 16384 columns bf16 200, with
// fp32 dy 254; 16383 columns 327, fp32 367; 12287 columns, mixed types 404 to 449, bf16 (no spill) 383: there the single elements cost
// more than the spills.
enum Width { kWave, k256, k512, k1024, kLong };
Width width_of(int d) { return d <= 1024 ? kWave : d <= 4096 ? k256 : d <= 12288 ? k512 : d <= 16384 ? k1024 : kLong; }

// Partial rows of the weights' gradients: as many workgroups as walk the rows.  16384 rows of 4096: 1024 workgroups 101 + 7 us (the
// second for adding the partial rows up), 512 147 + 5.
int partial_rows(int R, int d) {
  if (d > 16384) return std::min(R, 64);
  if (d <= 1024) return std::min(R / 4 + (R % 4 != 0), 1024);
  return std::min(R, d <= 4096 ? 1024 : 512);
}

// Outputs of more than this are stored past the caches: of an output that would fill them the next kernel finds little, and the
// inputs, which a backward pass reads again, stay.  Forward and backward of 16384 bf16 rows of 4096 in turn: 57 + 101 us, through
// the caches 58 + 125.
constexpr int64_t kKeepBytes = int64_t{32} << 20;

template <int V, bool KEEP, typename TX, typename TY>
void norm_forward_kept(const lnorm::Args& a, hipStream_t st) {
  const int R = a.R;
  switch (width_of(a.d)) {
    case kWave: hipLaunchKernelGGL((lnorm::forward_kernel<64, 16, V, KEEP, TX, TY>), dim3(std::min((R + 3) / 4, 2048)), dim3(256), 0, st, a); break;
    case k256: hipLaunchKernelGGL((lnorm::forward_kernel<256, 16, V, KEEP, TX, TY>), dim3(std::min(R, 2048)), dim3(256), 0, st, a); break;
    case k512: hipLaunchKernelGGL((lnorm::forward_kernel<512, 24, V, KEEP, TX, TY>), dim3(std::min(R, 1024)), dim3(512), 0, st, a); break;
    case k1024: hipLaunchKernelGGL((lnorm::forward_kernel<1024, 16, V, KEEP, TX, TY>), dim3(std::min(R, 512)), dim3(1024), 0, st, a); break;
    default: hipLaunchKernelGGL((lnorm::forward_long_kernel<TX, TY>), dim3(std::min(R, 512)), dim3(1024), 0, st, a); break;
  }
}

template <int V, bool KEEP, typename TX, typename TY>
void norm_backward_kept(const lnorm::Args& a, int P, hipStream_t st) {
  switch (width_of(a.d)) {
    case kWave: hipLaunchKernelGGL((lnorm::backward_kernel<64, 16, V, KEEP, TX, TY>), dim3(P), dim3(256), 0, st, a); break;
    case k256: hipLaunchKernelGGL((lnorm::backward_kernel<256, 16, V, KEEP, TX, TY>), dim3(P), dim3(256), 0, st, a); break;
    case k512: hipLaunchKernelGGL((lnorm::backward_kernel<512, 24, V, KEEP, TX, TY>), dim3(P), dim3(512), 0, st, a); break;
    case k1024: hipLaunchKernelGGL((lnorm::backward_kernel<1024, 16, V, KEEP, TX, TY>), dim3(P), dim3(1024), 0, st, a); break;
    default:
      hipLaunchKernelGGL((lnorm::backward_long_kernel<TX, TY>), dim3(std::min(a.R, 512)), dim3(1024), 0, st, a);
      if (a.partial) hipLaunchKernelGGL((lnorm::long_partials_kernel<TX, TY>), dim3((a.d + 255) / 256, P), dim3(256), 0, st, a);
      break;
  }
}

// (element by element, or long: always kept)
template <int V, typename TX, typename TY>
void norm_forward(const lnorm::Args& a, hipStream_t st) {
  if (V > 1 && static_cast<int64_t>(a.R) * a.d * static_cast<int64_t>(sizeof(TY)) > kKeepBytes) norm_forward_kept<V, V == 1, TX, TY>(a, st);
  else norm_forward_kept<V, true, TX, TY>(a, st);
}

template <int V, typename TX, typename TY>
void norm_backward(const lnorm::Args& a, int P, hipStream_t st) {
  if (V > 1 && static_cast<int64_t>(a.R) * a.d * static_cast<int64_t>(sizeof(TX)) > kKeepBytes) norm_backward_kept<V, V == 1, TX, TY>(a, P, st);
  else norm_backward_kept<V, true, TX, TY>(a, P, st);
}

// Calls `go` with the vector width and the two types of the call as template arguments.
template <typename F>
void by_type(int vec, int32_t tx, int32_t ty, F&& go) {
  using V1 = std::integral_constant<int, 1>;
  using V4 = std::integral_constant<int, 4>;
  using V8 = std::integral_constant<int, 8>;
  const float f = 0.f;
  const __bf16 b = static_cast<__bf16>(0.f);
  if (tx == SDDEN_BF16 && ty == SDDEN_BF16) {
    if (vec == 8) go(V8{}, b, b);
    else go(V1{}, b, b);
  } else if (vec == 1) {
    if (tx == SDDEN_F32 && ty == SDDEN_F32) go(V1{}, f, f);
    else if (tx == SDDEN_F32) go(V1{}, f, b);
    else go(V1{}, b, f);
  } else {
    if (tx == SDDEN_F32 && ty == SDDEN_F32) go(V4{}, f, f);
    else if (tx == SDDEN_F32) go(V4{}, f, b);
    else go(V4{}, b, f);
  }
}

// 16-byte accesses (8 elements where both types are bf16, else 4) where every row and vector starts on such a boundary, else one
// element at a time.  (The kernels' choice, not the hardware's, which takes any alignment of the element type.)  16384 bf16 rows of
// 4096 / 4095: forward 43 / 49 us, forward and backward 157 / 516.
int vector_width(int32_t d, int32_t tx, int32_t ty, std::initializer_list<int64_t> strides, std::initializer_list<const void*> ptrs) {
  const int vec = tx == SDDEN_BF16 && ty == SDDEN_BF16 ? 8 : 4;
  if (d % vec) return 1;
  for (int64_t s : strides)
    if (s % vec) return 1;
  for (const void* p : ptrs)
    if (!sdi::aligned16(p)) return 1;
  return vec;
}

// ------------------------------------------------------------------------------------------------ gated block
constexpr int64_t kMaxStride = int64_t{1} << 23;     // 128 rows of an operand stay within 32-bit offsets

int check_gated(const char* what, int32_t R, int32_t d, int32_t H, int32_t act, const uint16_t* X, int64_t x_stride, const uint16_t* Wg,
                const uint16_t* Wu, const uint16_t* Wd) {
  if (R < 0 || d <= 0 || H <= 0 || (act != SDDEN_SILU && act != SDDEN_GELU) || !Wg || !Wu || !Wd || (R > 0 && !X))
    return sdi::fail(LAYER_ERR, SD_ERR_ARG, "%s: bad argument", what);
  if (d % 8 || H % 8)
    return sdi::fail(LAYER_ERR, SD_ERR_UNSUPPORTED, "%s: d=%d and H=%d must be multiples of 8", what, d, H);
  if (x_stride < d || x_stride % 8 || x_stride > kMaxStride || d > kMaxStride || H > kMaxStride)
    return sdi::fail(LAYER_ERR, SD_ERR_ARG, "%s: x_stride=%lld must be a multiple of 8 from d=%d to %lld", what,
                     static_cast<long long>(x_stride), d, static_cast<long long>(kMaxStride));
  const int64_t tiles = (static_cast<int64_t>(R) + 127) / 128 * ((std::max(d, H) + 63) / 64), wtiles = (static_cast<int64_t>(d) + 127) / 128 * ((H + 127) / 128);
  if (R > kMaxRows || tiles > (1 << 28) || wtiles > (1 << 26))
    return sdi::fail(LAYER_ERR, SD_ERR_UNSUPPORTED, "%s: R=%d rows of d=%d, H=%d are too many for one call", what, R, d, H);
  if (!sdi::aligned16(X) || !sdi::aligned16(Wg) || !sdi::aligned16(Wu) || !sdi::aligned16(Wd))
    return sdi::fail(LAYER_ERR, SD_ERR_ARG, "%s: X and the weights must be 16-byte aligned", what);
  return SD_OK;
}

int done(const char* what, hipError_t e) {
  if (e != hipSuccess) return sdi::fail(LAYER_ERR, SD_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return SD_OK;
}

}  // namespace

extern "C" {

size_t sdden_layernorm_workspace_bytes(int32_t R, int32_t d) {
  if (R <= 0 || d <= 0) return 0;
  return static_cast<size_t>(partial_rows(R, d)) * d * 2 * sizeof(float);
}

int sdden_layernorm_forward(int32_t R, int32_t d, const void* x, int32_t x_type, int64_t x_stride, const float* weight, const float* bias,
                            float eps, void* y, int32_t y_type, int64_t y_stride, float* mean, float* rstd, void* stream) {
  const char* what = "sdden_layernorm_forward";
  if (R < 0 || d <= 0 || !type_ok(x_type) || !type_ok(y_type) || x_stride < d || y_stride < d || (R > 0 && (!x || !y)) || !mean != !rstd)
    return sdi::fail(LAYER_ERR, SD_ERR_ARG, "%s: bad argument", what);
  if (!(eps >= 0.f) || std::isinf(eps)) return sdi::fail(LAYER_ERR, SD_ERR_ARG, "%s: eps must be finite and not negative", what);
  if (!aligned_to(x, size_of(x_type)) || !aligned_to(y, size_of(y_type)) || !aligned_to(weight, 4) || !aligned_to(bias, 4) ||
      !aligned_to(mean, 4) || !aligned_to(rstd, 4))
    return sdi::fail(LAYER_ERR, SD_ERR_ARG, "%s: a pointer is not aligned to its element type", what);
  if (R > kMaxRows || d > kMaxWidth) return sdi::fail(LAYER_ERR, SD_ERR_UNSUPPORTED, "%s: R=%d and d=%d must not exceed 2^30", what, R, d);
  if (R == 0) return SD_OK;
  lnorm::Args a{};
  a.R = R; a.d = d; a.x = x; a.ldx = x_stride; a.y = y; a.ldy = y_stride; a.w = weight; a.b = bias; a.mean = mean; a.rstd = rstd; a.eps = eps;
  const int vec = vector_width(d, x_type, y_type, {x_stride, y_stride}, {x, y, weight, bias});
  by_type(vec, x_type, y_type, [&](auto v, auto tx, auto ty) { norm_forward<decltype(v)::value, decltype(tx), decltype(ty)>(a, static_cast<hipStream_t>(stream)); });
  return done(what, hipGetLastError());
}

int sdden_layernorm_backward(int32_t R, int32_t d, const void* dy, int32_t dy_type, int64_t dy_stride, const void* x, int32_t x_type,
                             int64_t x_stride, const float* weight, const float* mean, const float* rstd, const void* dres,
                             int64_t dres_stride, void* dx, int64_t dx_stride, float* dweight, float* dbias, void* workspace,
                             size_t workspace_bytes, void* stream) {
  const char* what = "sdden_layernorm_backward";
  if (R < 0 || d <= 0 || !type_ok(x_type) || !type_ok(dy_type) || x_stride < d || dy_stride < d || dx_stride < d || (dres && dres_stride < d) ||
      (R > 0 && (!x || !dy || !dx || !mean || !rstd)))
    return sdi::fail(LAYER_ERR, SD_ERR_ARG, "%s: bad argument", what);
  if (!aligned_to(x, size_of(x_type)) || !aligned_to(dx, size_of(x_type)) || !aligned_to(dres, size_of(x_type)) ||
      !aligned_to(dy, size_of(dy_type)) || !aligned_to(weight, 4) || !aligned_to(mean, 4) || !aligned_to(rstd, 4) ||
      !aligned_to(dweight, 4) || !aligned_to(dbias, 4) || !aligned_to(workspace, 4))
    return sdi::fail(LAYER_ERR, SD_ERR_ARG, "%s: a pointer is not aligned to its element type", what);
  if (R > kMaxRows || d > kMaxWidth) return sdi::fail(LAYER_ERR, SD_ERR_UNSUPPORTED, "%s: R=%d and d=%d must not exceed 2^30", what, R, d);
  const bool grads = dweight || dbias;
  if (grads && R > 0 && (!workspace || workspace_bytes < sdden_layernorm_workspace_bytes(R, d)))
    return sdi::fail(LAYER_ERR, SD_ERR_WORKSPACE, "%s: dweight and dbias need %zu bytes of workspace, got %zu", what,
                     sdden_layernorm_workspace_bytes(R, d), workspace ? workspace_bytes : 0);
  lnorm::Args a{};
  a.R = R; a.d = d; a.x = x; a.ldx = x_stride; a.dy = dy; a.lddy = dy_stride; a.dres = dres; a.lddres = dres ? dres_stride : 0;
  a.y = dx; a.ldy = dx_stride; a.w = weight; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.partial = grads ? static_cast<float*>(workspace) : nullptr;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int P = R > 0 ? partial_rows(R, d) : 0;
  if (R > 0) {
    const int vec = vector_width(d, x_type, dy_type, {x_stride, dy_stride, dx_stride, a.lddres}, {x, dy, dx, dres, weight});
    by_type(vec, x_type, dy_type, [&](auto v, auto tx, auto ty) { norm_backward<decltype(v)::value, decltype(tx), decltype(ty)>(a, P, st); });
  }
  if (grads)
    hipLaunchKernelGGL(lnorm::reduce_partials_kernel, dim3(lnorm::reduce_grid(d), 2), dim3(1024), 0, st, a.partial, P, d, dweight, dbias);
  return done(what, hipGetLastError());
}

size_t sdden_gated_workspace_bytes(int32_t R, int32_t d, int32_t H) {
  if (R <= 0 || d <= 0 || H <= 0) return 0;
  return static_cast<size_t>(R) * H * 2 * sizeof(uint16_t);            // dG, dU
}

int sdden_gated_forward(int32_t R, int32_t d, int32_t H, int32_t act, const uint16_t* X, int64_t x_stride, const uint16_t* Wg,
                        const uint16_t* Wu, const uint16_t* Wd, const void* res, void* Y, int32_t y_type, int64_t y_stride,
                        uint16_t* hidden, float* gates, void* stream) {
  const char* what = "sdden_gated_forward";
  if (int rc = check_gated(what, R, d, H, act, X, x_stride, Wg, Wu, Wd)) return rc;
  if (!type_ok(y_type) || (R > 0 && (!Y || !hidden)) || y_stride < d || y_stride % 8 || y_stride > kMaxStride)
    return sdi::fail(LAYER_ERR, SD_ERR_ARG, "%s: bad argument (Y, y_type, y_stride a multiple of 8 and at least d, hidden)", what);
  if (!sdi::aligned16(Y) || !sdi::aligned16(res) || !sdi::aligned16(hidden) || !sdi::aligned16(gates))
    return sdi::fail(LAYER_ERR, SD_ERR_ARG, "%s: Y, res, hidden and gates must be 16-byte aligned", what);
  if (R == 0) return SD_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  lgemm::Args a{};
  a.problems = 1;
  a.act = act;
  lgemm::Problem& p = a.p[0];
  p.A[0] = X; p.lda = x_stride; p.B[0] = Wg; p.B[1] = Wu; p.ldb = d; p.M = R; p.N = H; p.K = d; p.ranges = 1;
  p.out = hidden; p.ldo = H;
  if (gates) { p.gates[0] = gates; p.gates[1] = gates + static_cast<int64_t>(R) * H; }
  hipError_t e = lgemm::launch<lgemm::kGate, lgemm::kAlong, lgemm::kAlong>(a, st);
  if (e != hipSuccess) return done(what, e);
  p = lgemm::Problem{};
  p.A[0] = hidden; p.lda = H; p.B[0] = Wd; p.ldb = H; p.M = R; p.N = d; p.K = H; p.ranges = 1;
  p.out = Y; p.ldo = y_stride; p.res = res; p.out_f32 = y_type == SDDEN_F32;
  return done(what, lgemm::launch<lgemm::kStore, lgemm::kAlong, lgemm::kAlong>(a, st));
}

int sdden_gated_backward(int32_t R, int32_t d, int32_t H, int32_t act, const uint16_t* dY, int64_t dy_stride, const uint16_t* X,
                         int64_t x_stride, const uint16_t* Wg, const uint16_t* Wu, const uint16_t* Wd, const float* gates,
                         const uint16_t* hidden, uint16_t* dX, int64_t dx_stride, void* dWg, void* dWu, void* dWd, int32_t dw_type,
                         void* workspace, size_t workspace_bytes, void* stream) {
  const char* what = "sdden_gated_backward";
  if (int rc = check_gated(what, R, d, H, act, X, x_stride, Wg, Wu, Wd)) return rc;
  const bool weights = dWg || dWu || dWd;
  if ((R > 0 && (!dY || !gates || !hidden)) || dy_stride < d || dy_stride % 8 || dy_stride > kMaxStride ||
      (dX && (dx_stride < d || dx_stride % 8 || dx_stride > kMaxStride)) || !type_ok(dw_type) || (!dX && !weights))
    return sdi::fail(LAYER_ERR, SD_ERR_ARG, "%s: bad argument (pointers, strides multiples of 8 and at least d, dw_type)", what);
  if (weights && (!dWg || !dWu || !dWd))
    return sdi::fail(LAYER_ERR, SD_ERR_ARG, "%s: dWg, dWu and dWd are computed together: give all three or none", what);
  for (const void* q : {static_cast<const void*>(dY), static_cast<const void*>(gates), static_cast<const void*>(hidden),
                        static_cast<const void*>(dX), static_cast<const void*>(dWg), static_cast<const void*>(dWu),
                        static_cast<const void*>(dWd), static_cast<const void*>(workspace)})
    if (!sdi::aligned16(q)) return sdi::fail(LAYER_ERR, SD_ERR_ARG, "%s: every buffer must be 16-byte aligned", what);
  if (R > 0 && (!workspace || workspace_bytes < sdden_gated_workspace_bytes(R, d, H)))
    return sdi::fail(LAYER_ERR, SD_ERR_WORKSPACE, "%s: needs %zu bytes of workspace, got %zu", what, sdden_gated_workspace_bytes(R, d, H),
                     workspace ? workspace_bytes : 0);
  hipStream_t st = static_cast<hipStream_t>(stream);
  uint16_t* dG = static_cast<uint16_t*>(workspace);
  uint16_t* dU = dG + static_cast<int64_t>(R) * H;
  float* g = const_cast<float*>(gates);
  if (R > 0) {
    lgemm::Args a{};
    a.problems = 1;
    a.act = act;
    lgemm::Problem& p = a.p[0];
    p.A[0] = dY; p.lda = dy_stride; p.B[0] = Wd; p.ldb = H; p.M = R; p.N = H; p.K = d; p.ranges = 1;
    p.out = dG; p.out2 = dU; p.ldo = H; p.gates[0] = g; p.gates[1] = g + static_cast<int64_t>(R) * H;
    hipError_t e = lgemm::launch<lgemm::kGateGrad, lgemm::kAlong, lgemm::kAcross>(a, st);
    if (e != hipSuccess) return done(what, e);
    if (dX) {
      p = lgemm::Problem{};
      p.A[0] = dG; p.A[1] = dU; p.lda = H; p.B[0] = Wg; p.B[1] = Wu; p.ldb = d; p.M = R; p.N = d; p.K = H; p.ranges = 2;
      p.out = dX; p.ldo = dx_stride;
      e = lgemm::launch<lgemm::kStore, lgemm::kAlong, lgemm::kAcross>(a, st);
      if (e != hipSuccess) return done(what, e);
    }
  }
  if (weights) {
    lgemm::Args a{};
    a.problems = 3;
    for (int i = 0; i < 3; ++i) {
      lgemm::Problem& p = a.p[i];
      p.K = R; p.ranges = 1; p.out_f32 = dw_type == SDDEN_F32;
      if (i < 2) {
        p.A[0] = i ? dU : dG; p.lda = H; p.B[0] = X; p.ldb = x_stride; p.M = H; p.N = d; p.out = i ? dWu : dWg; p.ldo = d;
      } else {
        p.A[0] = dY; p.lda = dy_stride; p.B[0] = hidden; p.ldb = H; p.M = d; p.N = H; p.out = dWd; p.ldo = H;
      }
    }
    return done(what, lgemm::launch<lgemm::kStore, lgemm::kAcross, lgemm::kAcross>(a, st));
  }
  return SD_OK;
}

}  // extern "C"

// ------------------------------------------------------------------------------------------------ a denoiser of such layers
// D(x, k) = h_L,  h_0 = x + e_k,  h_{l+1} = h_l + FF_l(LN_l(h_l)): the residual stream stays fp32, the block's rows are bf16.
// Data flow per call: compaction of the unmasked rows; gather_add (h_0); per block the norm, the two first products with the
// activation, and the last product, which adds the stream in place and in the last block scatters to the source rows.
namespace {

// h[m] = X[rowidx[m]] + table[krow[rowidx[m]]], 4 elements per thread and step
__global__ __launch_bounds__(256) void gather_add_kernel(const float* __restrict__ X, const float* __restrict__ table,
                                                         const int32_t* __restrict__ rowidx, const int32_t* __restrict__ krow,
                                                         const int32_t* __restrict__ count, float* __restrict__ h, int d) {
  const int per_row = d / 4;
  const int64_t total = static_cast<int64_t>(*count) * per_row;
  for (int64_t g = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; g < total; g += static_cast<int64_t>(gridDim.x) * 256) {
    const int m = static_cast<int>(g / per_row), c = static_cast<int>(g % per_row) * 4, src = rowidx[m];
    const lgemm::f32x4 x = *reinterpret_cast<const lgemm::f32x4*>(X + static_cast<int64_t>(src) * d + c);
    const lgemm::f32x4 e = *reinterpret_cast<const lgemm::f32x4*>(table + static_cast<int64_t>(krow[src]) * d + c);
    *reinterpret_cast<lgemm::f32x4*>(h + static_cast<int64_t>(m) * d + c) = x + e;
  }
}

struct GatedDenoiser final : sdden {
  int H = 0, blocks = 0, act = 0, cap_rows = 0;
  float eps = 0.f;
  float *table = nullptr, *nw = nullptr, *nb = nullptr;              // [T,d], [blocks,d], [blocks,d]
  uint16_t *Wg = nullptr, *Wu = nullptr, *Wd = nullptr;              // [blocks,H,d] x 2, [blocks,d,H]
  int32_t *rowidx = nullptr, *count = nullptr;
  float* h = nullptr;
  uint16_t *n = nullptr, *hidden = nullptr;

  ~GatedDenoiser() override {
    for (void* q : {static_cast<void*>(table), static_cast<void*>(nw), static_cast<void*>(nb), static_cast<void*>(Wg),
                    static_cast<void*>(Wu), static_cast<void*>(Wd), static_cast<void*>(rowidx), static_cast<void*>(count),
                    static_cast<void*>(h), static_cast<void*>(n), static_cast<void*>(hidden)})
      if (q) (void)hipFree(q);
  }

  int reserve(int R) override {
    if (R <= cap_rows) return SD_OK;
    for (void* q : {static_cast<void*>(rowidx), static_cast<void*>(h), static_cast<void*>(n), static_cast<void*>(hidden)})
      if (q) (void)hipFree(q);
    rowidx = nullptr; h = nullptr; n = hidden = nullptr; cap_rows = 0;
    const size_t rows = static_cast<size_t>(R);
    SD_HIP_TRY(err, hipMalloc(&rowidx, 4 * rows));
    SD_HIP_TRY(err, hipMalloc(&h, 4 * rows * d));
    SD_HIP_TRY(err, hipMalloc(&n, 2 * rows * d));
    SD_HIP_TRY(err, hipMalloc(&hidden, 2 * rows * H));
    if (!count) SD_HIP_TRY(err, hipMalloc(&count, 4));
    cap_rows = R;
    return SD_OK;
  }

  int eval(int R, const float* X, const int32_t* krow, float* out, hipStream_t st) override {
    if (R > cap_rows)
      return sdi::fail(err, SD_ERR_WORKSPACE, "sdden_eval(gated): %d rows exceed the %d reserved (sdden_reserve)", R, cap_rows);
    if (!sdi::aligned16(X) || !sdi::aligned16(out))
      return sdi::fail(err, SD_ERR_ARG, "sdden_eval(gated): X and out must be 16-byte aligned");
    hipLaunchKernelGGL(sdrows::compact_rows_kernel, dim3(sdrows::compact_rows_grid(R)), dim3(sdrows::kScan), 0, st, krow, rowidx, count,
                       active, rows_per_chain, R, T);
    const int64_t chunks = static_cast<int64_t>(R) * (d / 4);
    hipLaunchKernelGGL(gather_add_kernel, dim3(static_cast<unsigned>(std::min<int64_t>((chunks + 255) / 256, 256 * 32))), dim3(256), 0, st, X,
                       table, rowidx, krow, count, h, d);
    for (int l = 0; l < blocks; ++l) {
      lnorm::Args a{};
      a.R = R; a.d = d; a.x = h; a.ldx = d; a.y = n; a.ldy = d; a.eps = eps; a.count = count;
      a.w = nw + static_cast<int64_t>(l) * d;
      a.b = nb + static_cast<int64_t>(l) * d;
      prof.mark(1, st);
      by_type(4, SDDEN_F32, SDDEN_BF16, [&](auto v, auto tx, auto ty) { norm_forward<decltype(v)::value, decltype(tx), decltype(ty)>(a, st); });
      prof.mark(1, st);
      const int64_t wl = static_cast<int64_t>(l) * H * d;
      lgemm::Args g{};
      g.problems = 1;
      g.act = act;
      lgemm::Problem& p = g.p[0];
      p.A[0] = n; p.lda = d; p.B[0] = Wg + wl; p.B[1] = Wu + wl; p.ldb = d; p.M = R; p.N = H; p.K = d; p.ranges = 1;
      p.out = hidden; p.ldo = H; p.count = count;
      prof.mark(2, st);
      SD_HIP_TRY(err, (lgemm::launch<lgemm::kGate, lgemm::kAlong, lgemm::kAlong>(g, st)));
      prof.mark(2, st);
      p = lgemm::Problem{};
      p.A[0] = hidden; p.lda = H; p.B[0] = Wd + wl; p.ldb = H; p.M = R; p.N = d; p.K = H; p.ranges = 1;
      p.res = h; p.out_f32 = 1; p.ldo = d; p.count = count;
      const bool last = l == blocks - 1;
      p.out = last ? out : h;
      p.rowidx = last ? rowidx : nullptr;
      prof.mark(3, st);
      SD_HIP_TRY(err, (lgemm::launch<lgemm::kStore, lgemm::kAlong, lgemm::kAlong>(g, st)));
      prof.mark(3, st);
    }
    SD_HIP_TRY(err, hipGetLastError());
    return SD_OK;
  }
};

}  // namespace

extern "C" int sdden_gated_create(int32_t d, int32_t H, int32_t E, int32_t blocks, int32_t act, const uint16_t* We, const float* be,
                                  const float* norm_weight, const float* norm_bias, float eps, const uint16_t* Wg, const uint16_t* Wu,
                                  const uint16_t* Wd, int32_t T, int32_t Rmax, sdden** out) try {
  const char* what = "sdden_gated_create";
  if ((E > 0 && !We) || !be || !norm_weight || !norm_bias || !Wg || !Wu || !Wd || !out || d <= 0 || H <= 0 || E < 0 || (E & 1) || blocks <= 0 ||
      T <= 0 || Rmax <= 0 || (act != SDDEN_SILU && act != SDDEN_GELU) || !(eps >= 0.f) || std::isinf(eps))
    return sdi::fail(LAYER_ERR, SD_ERR_ARG, "%s: bad argument", what);
  if (d % 8 || H % 8 || d > kMaxStride || H > kMaxStride)
    return sdi::fail(LAYER_ERR, SD_ERR_UNSUPPORTED, "%s: d=%d and H=%d must be multiples of 8 up to %lld", what, d, H,
                     static_cast<long long>(kMaxStride));
  std::unique_ptr<GatedDenoiser> m(new GatedDenoiser);
  m->d = d; m->T = T; m->H = H; m->blocks = blocks; m->act = act; m->eps = eps;
  const std::vector<float> table = sdtime::table(T, d, E, be, We);
  hipError_t e = hipSuccess;
  auto up = [&](auto** dst, const void* src, size_t bytes) {
    if (e == hipSuccess) e = hipMalloc(reinterpret_cast<void**>(dst), bytes);
    if (e == hipSuccess) e = hipMemcpy(*dst, src, bytes, hipMemcpyHostToDevice);
  };
  const size_t vec = static_cast<size_t>(blocks) * d * 4, mat = static_cast<size_t>(blocks) * d * H * 2;
  up(&m->table, table.data(), table.size() * 4);
  up(&m->nw, norm_weight, vec);
  up(&m->nb, norm_bias, vec);
  up(&m->Wg, Wg, mat);
  up(&m->Wu, Wu, mat);
  up(&m->Wd, Wd, mat);
  if (e != hipSuccess) return sdi::fail(LAYER_ERR, SD_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  if (int rc = m->reserve(Rmax)) {
    LAYER_ERR = m->err;
    return rc;
  }
  *out = m.release();
  return SD_OK;
} catch (const std::exception& ex) {
  return sdi::fail(LAYER_ERR, SD_ERR_ARG, "sdden_gated_create: %s", ex.what());
}
