// Host: the sinusoidal time embedding of every chain step through its weight rows, as a table added to a layer's input.
#pragma once
#include <cmath>
#include <cstdint>
#include <cstring>
#include <vector>

namespace sdtime {

inline float bf16_bits_to_float(uint16_t b) {
  const uint32_t u = static_cast<uint32_t>(b) << 16;
  float f;
  std::memcpy(&f, &u, 4);
  return f;
}

// table[k] = bias + emb(k) . W for k < T;  W [E, H] bf16, emb = [sin(k w_i) ; cos(k w_i)], w_i = 10000^(-2i/E)
inline std::vector<float> table(int T, int H, int E, const float* bias, const uint16_t* W) {
  std::vector<float> tb(static_cast<size_t>(T) * H);
  const int half = E / 2;
  std::vector<double> emb(E > 0 ? E : 1), row(H);
  for (int k = 0; k < T; ++k) {
    for (int i = 0; i < half; ++i) {
      const double w = std::pow(10000.0, -static_cast<double>(i) / half);
      emb[i] = std::sin(k * w);
      emb[half + i] = std::cos(k * w);
    }
    for (int n = 0; n < H; ++n) row[n] = bias[n];
    for (int e = 0; e < E; ++e) {
      const uint16_t* wrow = W + static_cast<size_t>(e) * H;
      const double ev = emb[e];
      for (int n = 0; n < H; ++n) row[n] += ev * bf16_bits_to_float(wrow[n]);
    }
    for (int n = 0; n < H; ++n) tb[static_cast<size_t>(k) * H + n] = static_cast<float>(row[n]);
  }
  return tb;
}

}  // namespace sdtime
