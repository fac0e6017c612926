// Matrices kept in 4 bits with group scales (sdden_q4_*); kernels and layout in q4_product.h.
#include <hip/hip_runtime.h>

#include <new>

#include "q4_matrix.h"
#include "sdden_internal.h"

#define Q4_ERR sdi::g_den_create_error

extern "C" {

int sdden_q4_create(int32_t N, int32_t K, int32_t group, const uint8_t* q, const uint16_t* scale, sdden_q4** out) {
  const char* what = "sdden_q4_create";
  if (!out || !q || !scale || N <= 0 || K <= 0) return sdi::fail(Q4_ERR, SD_ERR_ARG, "%s: bad argument", what);
  if (group != 32 && group != 64 && (group <= 0 || group % 128))
    return sdi::fail(Q4_ERR, SD_ERR_UNSUPPORTED, "%s: group=%d must be 32, 64 or a multiple of 128", what, group);
  if (N > q4::kMaxDim || K > q4::kMaxDim)
    return sdi::fail(Q4_ERR, SD_ERR_UNSUPPORTED, "%s: N=%d and K=%d must not exceed %d", what, N, K, q4::kMaxDim);
  sdden_q4* m = new (std::nothrow) sdden_q4;
  if (!m) return sdi::fail(Q4_ERR, SD_ERR_ARG, "%s: out of host memory", what);
  const hipError_t e = m->upload(N, K, group, q, scale);
  if (e != hipSuccess) {
    delete m;
    return sdi::fail(Q4_ERR, SD_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  }
  *out = m;
  return SD_OK;
}

int sdden_q4_eval(const sdden_q4* m, int32_t R, const void* X, int32_t x_type, int64_t x_stride, const float* bias, void* Y,
                  int32_t y_type, int64_t y_stride, void* stream) {
  const char* what = "sdden_q4_eval";
  if (!m || R < 0 || (R > 0 && (!X || !Y)) || (x_type != SDDEN_F32 && x_type != SDDEN_BF16) || (y_type != SDDEN_F32 && y_type != SDDEN_BF16) ||
      x_stride < m->K || y_stride < m->N)
    return sdi::fail(Q4_ERR, SD_ERR_ARG, "%s: bad argument", what);
  if ((reinterpret_cast<uintptr_t>(X) & (x_type == SDDEN_F32 ? 3 : 1)) || (reinterpret_cast<uintptr_t>(Y) & (y_type == SDDEN_F32 ? 3 : 1)) ||
      (reinterpret_cast<uintptr_t>(bias) & 3))
    return sdi::fail(Q4_ERR, SD_ERR_ARG, "%s: a pointer is not aligned to its element type", what);
  int device = -1;
  if (hipGetDevice(&device) != hipSuccess || device != m->device)
    return sdi::fail(Q4_ERR, SD_ERR_ARG, "%s: the matrix lies on device %d, the current device is %d", what, m->device, device);
  if (R == 0) return SD_OK;
  q4::Args a{};
  m->fill(a);
  a.X = X; a.ldx = x_stride; a.R = R;
  a.vec = sdi::aligned16(X) && x_stride % (x_type == SDDEN_F32 ? 4 : 8) == 0;
  a.bias = bias;
  a.Y = Y; a.ldy = y_stride; a.y_f32 = y_type == SDDEN_F32;
  a.vec_out = sdi::aligned16(Y) && y_stride % 4 == 0;
  const hipError_t e = m->launch(a, R, x_type == SDDEN_F32 ? q4::kF32 : q4::kBf16, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return sdi::fail(Q4_ERR, SD_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return SD_OK;
}

int sdden_q4_destroy(sdden_q4* m) {
  if (!m) return SD_ERR_ARG;
  delete m;
  return SD_OK;
}

}  // extern "C"
