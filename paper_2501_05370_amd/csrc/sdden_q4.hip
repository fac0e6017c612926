// Matrices kept in 4 bits with group scales (sdden_q4_*); kernels and layout in q4_product.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <memory>
#include <new>
#include <vector>

#include "q4_matrix.h"
#include "sdden_internal.h"
#include "sdden_rows.h"
#include "time_table.h"

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
  if (R > (1 << 30)) return sdi::fail(Q4_ERR, SD_ERR_UNSUPPORTED, "%s: R=%d must not exceed 2^30", what, R);
  int device = -1;
  if (hipGetDevice(&device) != hipSuccess || device != m->device)
    return sdi::fail(Q4_ERR, SD_ERR_ARG, "%s: the matrix lies on device %d, the current device is %d", what, m->device, device);
  if (R == 0) return SD_OK;
  q4::Args a{};
  m->fill(a);
  a.X = X; a.ldx = x_stride; a.R = R;
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

// ------------------------------------------------------------------------------------------------ the MLP denoiser in 4 bits
// The network of sdden_mlp.hip with its three matrices in 4 bits, as a draft model that reads a quarter of the target's bytes:
//   compact_rows     unmasked rows -> dense list
//   product 1        H1 = silu(X Q1 + tb[krow])    rows gathered from the caller's bf16 image, or rounded to bf16 as they enter
//                    (more than 32 rows: by gather_round)
//   product 2        H2 = silu(H1 Q2 + b2)
//   product 3        out[rowidx] = H2 Q3 + b3       fp32
namespace {

float bf16_round(float x) {          // to nearest even; finite values only
  uint32_t u;
  std::memcpy(&u, &x, 4);
  u = (u + 0x7FFFu + ((u >> 16) & 1u)) & 0xFFFF0000u;
  std::memcpy(&x, &u, 4);
  return x;
}

bool all_finite(const uint16_t* W, size_t n) {
  bool ok = true;
  for (size_t i = 0; i < n; ++i) ok &= (W[i] & 0x7F80u) != 0x7F80u;
  return ok;
}

// W [K, N] bf16, finite (row = input) -> q [N, ceil(K/2)], scale [N, ceil(K/group)]: scale = bf16(max |w| / 7) over the group's
// inputs, q = round(w / scale) + 8 within 0..15; a group of zeros has scale 0 and q = 8.
void quantize(const uint16_t* W, int K, int N, int group, std::vector<uint8_t>& q, std::vector<uint16_t>& scale) {
  const int groups = q4::groups_of(K, group);
  const size_t rowbytes = (static_cast<size_t>(K) + 1) / 2;
  q.assign(static_cast<size_t>(N) * rowbytes, 0);
  scale.assign(static_cast<size_t>(N) * groups, 0);
  constexpr int NB = 64;              // columns at a time: a row's 128 bytes are read together
  for (int n0 = 0; n0 < N; n0 += NB) {
    const int nb = std::min(NB, N - n0);
    for (int g = 0; g < groups; ++g) {
      const int k0 = g * group, k1 = std::min(K, k0 + group);
      float amax[NB] = {}, s[NB];
      for (int k = k0; k < k1; ++k)
        for (int i = 0; i < nb; ++i) amax[i] = std::max(amax[i], std::fabs(sdtime::bf16_bits_to_float(W[static_cast<size_t>(k) * N + n0 + i])));
      for (int i = 0; i < nb; ++i) {
        s[i] = bf16_round(amax[i] / 7.0f);
        uint32_t u;
        std::memcpy(&u, &s[i], 4);
        scale[static_cast<size_t>(n0 + i) * groups + g] = static_cast<uint16_t>(u >> 16);
      }
      for (int k = k0; k < k1; ++k)
        for (int i = 0; i < nb; ++i) {
          const float w = sdtime::bf16_bits_to_float(W[static_cast<size_t>(k) * N + n0 + i]);
          const float v = s[i] > 0.f ? std::nearbyint(w / s[i]) : 0.f;
          const int c = static_cast<int>(std::min(7.f, std::max(-8.f, v))) + 8;
          q[(n0 + i) * rowbytes + (k >> 1)] |= static_cast<uint8_t>(k & 1 ? c << 4 : c);
        }
    }
  }
}

// Xb[m] = X[rowidx[m]] rounded to bf16, rows of ld (16 bytes) apart
__global__ __launch_bounds__(256) void gather_round_kernel(const float* __restrict__ X, const int32_t* __restrict__ rowidx,
                                                           const int32_t* __restrict__ count, uint16_t* __restrict__ Xb, int d, int64_t ld) {
  const int per_row = (d + 3) / 4;
  const int64_t total = static_cast<int64_t>(*count) * per_row;
  for (int64_t g = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; g < total; g += static_cast<int64_t>(gridDim.x) * 256) {
    const int m = static_cast<int>(g / per_row), c = static_cast<int>(g % per_row) * 4;
    const float* x = X + static_cast<int64_t>(rowidx[m]) * d + c;
    q4::f32x4 v{0.f, 0.f, 0.f, 0.f};
    if (d % 4 == 0) {
      v = *reinterpret_cast<const q4::f32x4*>(x);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < d) v[e] = x[e];
    }
    *reinterpret_cast<q4::u32x2*>(Xb + m * ld + c) = lgemm::pack_bf16(v);
  }
}

struct Mlp4Denoiser final : sdden {
  int H = 0, cap_rows = 0;
  sdden_q4 Q1, Q2, Q3;
  float *tb = nullptr, *b2 = nullptr, *b3 = nullptr;      // [T,H], [H], [d]
  int32_t *rowidx = nullptr, *count = nullptr;
  uint16_t *Xb = nullptr, *H1 = nullptr, *H2 = nullptr;
  int64_t ldx = 0, ldh = 0;                               // rows of Xb, of H1 and H2 start on 16 bytes

  ~Mlp4Denoiser() override {
    for (void* p : {static_cast<void*>(tb), static_cast<void*>(b2), static_cast<void*>(b3), static_cast<void*>(rowidx),
                    static_cast<void*>(count), static_cast<void*>(Xb), static_cast<void*>(H1), static_cast<void*>(H2)})
      if (p) (void)hipFree(p);
  }

  int reserve(int R) override {
    if (R <= cap_rows) return SD_OK;
    for (void* p : {static_cast<void*>(rowidx), static_cast<void*>(Xb), static_cast<void*>(H1), static_cast<void*>(H2)})
      if (p) (void)hipFree(p);
    rowidx = nullptr; Xb = H1 = H2 = nullptr; cap_rows = 0;
    ldx = (d + 7) / 8 * 8;
    ldh = (H + 7) / 8 * 8;
    SD_HIP_TRY(err, hipMalloc(&rowidx, 4 * static_cast<size_t>(R)));
    if (R > q4::kRoundedRows) SD_HIP_TRY(err, hipMalloc(&Xb, 2 * static_cast<size_t>(R) * ldx));
    SD_HIP_TRY(err, hipMalloc(&H1, 2 * static_cast<size_t>(R) * ldh));
    SD_HIP_TRY(err, hipMalloc(&H2, 2 * static_cast<size_t>(R) * ldh));
    if (!count) SD_HIP_TRY(err, hipMalloc(&count, 4));
    cap_rows = R;
    return SD_OK;
  }

  int eval(int R, const float* X, const int32_t* krow, float* out, hipStream_t st) override { return go(R, X, nullptr, krow, out, st); }
  int eval_mirror(int R, const float* X, const uint16_t* Xb, const int32_t* krow, float* out, hipStream_t st) override {
    return go(R, X, Xb, krow, out, st);
  }

  int go(int R, const float* X, const uint16_t* image, const int32_t* krow, float* out, hipStream_t st) {
    if (R > cap_rows)
      return sdi::fail(err, SD_ERR_WORKSPACE, "sdden_eval(mlp4): %d rows exceed the %d reserved (sdden_reserve)", R, cap_rows);
    if (!sdi::aligned16(X) || !sdi::aligned16(out) || !sdi::aligned16(image))
      return sdi::fail(err, SD_ERR_ARG, "sdden_eval(mlp4): X, its image and out must be 16-byte aligned");
    hipLaunchKernelGGL(sdrows::compact_rows_kernel, dim3(sdrows::compact_rows_grid(R)), dim3(sdrows::kScan), 0, st, krow, rowidx, count,
                       active, rows_per_chain, R, T);
    q4::Args a{};
    Q1.fill(a);
    a.R = R;
    int form = q4::kBf16;
    if (image) {
      a.X = image; a.ldx = d; a.gather = true;
    } else if (R <= q4::kRoundedRows) {
      a.X = X; a.ldx = d; a.gather = true;
      form = q4::kF32Rounded;
    } else {
      const int64_t chunks = static_cast<int64_t>(R) * ((d + 3) / 4);
      hipLaunchKernelGGL(gather_round_kernel, dim3(static_cast<unsigned>(std::min<int64_t>((chunks + 255) / 256, 256 * 32))), dim3(256), 0, st, X,
                         rowidx, count, Xb, d, ldx);
      a.X = Xb; a.ldx = ldx;
    }
    a.bias = tb; a.krow = krow; a.rowidx = rowidx; a.count = count; a.silu = true;
    a.Y = H1; a.ldy = ldh; a.vec_out = true;
    prof.mark(1, st);
    SD_HIP_TRY(err, Q1.launch(a, R, form, st));
    prof.mark(1, st);
    a = q4::Args{};
    Q2.fill(a);
    a.X = H1; a.ldx = ldh; a.R = R; a.bias = b2; a.count = count; a.silu = true; a.Y = H2; a.ldy = ldh; a.vec_out = true;
    prof.mark(2, st);
    SD_HIP_TRY(err, Q2.launch(a, R, q4::kBf16, st));
    prof.mark(2, st);
    a = q4::Args{};
    Q3.fill(a);
    a.X = H2; a.ldx = ldh; a.R = R; a.bias = b3; a.count = count; a.rowidx = rowidx; a.scatter = true;
    a.Y = out; a.ldy = d; a.y_f32 = true; a.vec_out = d % 4 == 0;
    prof.mark(3, st);
    SD_HIP_TRY(err, Q3.launch(a, R, q4::kBf16, st));
    prof.mark(3, st);
    SD_HIP_TRY(err, hipGetLastError());
    return SD_OK;
  }
};

}  // namespace

extern "C" int sdden_mlp4_create(int32_t d, int32_t H, int32_t E, int32_t group, const uint16_t* W1, const float* b1, const uint16_t* W2,
                                 const float* b2, const uint16_t* W3, const float* b3, int32_t T, int32_t Rmax, sdden** out) try {
  const char* what = "sdden_mlp4_create";
  if (!W1 || !b1 || !W2 || !b2 || !W3 || !b3 || !out || d <= 0 || H <= 0 || E < 0 || (E & 1) || T <= 0 || Rmax <= 0)
    return sdi::fail(Q4_ERR, SD_ERR_ARG, "%s: bad argument", what);
  if ((group != 32 && group != 64 && (group <= 0 || group % 128)) || d > q4::kMaxDim || H > q4::kMaxDim)
    return sdi::fail(Q4_ERR, SD_ERR_UNSUPPORTED, "%s: group=%d must be 32, 64 or a multiple of 128, d=%d and H=%d at most %d", what, group, d, H,
                     q4::kMaxDim);
  // 4 bits have no infinity and no NaN to stand for one: a broken network would become a plausible one
  const struct { const uint16_t* W; size_t n; const char* name; } matrices[] = {
      {W1, static_cast<size_t>(d) * H, "W1"}, {W2, static_cast<size_t>(H) * H, "W2"}, {W3, static_cast<size_t>(H) * d, "W3"}};
  for (const auto& w : matrices)
    if (!all_finite(w.W, w.n)) return sdi::fail(Q4_ERR, SD_ERR_ARG, "%s: %s has weights that are not finite", what, w.name);
  std::unique_ptr<Mlp4Denoiser> m(new Mlp4Denoiser);
  m->d = d; m->T = T; m->H = H;
  const std::vector<float> tb = sdtime::table(T, H, E, b1, W1 + static_cast<size_t>(d) * H);
  hipError_t e = hipSuccess;
  std::vector<uint8_t> q;
  std::vector<uint16_t> s;
  auto matrix = [&](sdden_q4& M, const uint16_t* W, int K, int N) {
    if (e != hipSuccess) return;
    quantize(W, K, N, group, q, s);
    e = M.upload(N, K, group, q.data(), s.data());
  };
  auto up = [&](float** dst, const float* src, size_t n) {
    if (e == hipSuccess) e = hipMalloc(reinterpret_cast<void**>(dst), 4 * n);
    if (e == hipSuccess) e = hipMemcpy(*dst, src, 4 * n, hipMemcpyHostToDevice);
  };
  up(&m->tb, tb.data(), tb.size());
  up(&m->b2, b2, H);
  up(&m->b3, b3, d);
  matrix(m->Q1, W1, d, H);
  matrix(m->Q2, W2, H, H);
  matrix(m->Q3, W3, H, d);
  if (e != hipSuccess) return sdi::fail(Q4_ERR, SD_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  if (int rc = m->reserve(Rmax)) {
    Q4_ERR = m->err;
    return rc;
  }
  *out = m.release();
  return SD_OK;
} catch (const std::exception& ex) {
  return sdi::fail(Q4_ERR, SD_ERR_ARG, "sdden_mlp4_create: %s", ex.what());
}
