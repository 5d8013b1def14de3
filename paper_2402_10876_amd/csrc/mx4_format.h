// Internal: the microscaled 4-bit format on the host (plain arithmetic, also built without HIP).
//
// 32 consecutive rows of a column are a block: 32 values of e2m1 (sign, two bits of exponent, one of mantissa:
// 0, 0.5, 1, 1.5, 2, 3, 4, 6) times one power of two, held as its exponent plus 127 in a byte.
//   exponent : floor(log2 of the largest magnitude) - 2, so that the largest lands in [4, 8); a block of zeros: 0
//   value    : x / 2^exponent to the nearest of the format, ties to the even code, past 6 to 6; the sign stays
// The values of a block are fp16 numbers again (a value is a multiple of the input's own spacing or of a quarter of the
// largest magnitude's), and making a block of them a second time gives the same block: its largest is 4 or 6 still.
#pragma once
#include <stdint.h>
#include <string.h>

namespace twg {

constexpr int MX4_BLOCK = 32;
constexpr int MX4_ONE = 127;            // scale byte of 2^0
constexpr int MX4_NAN = 255;            // a block that holds an infinity or NaN (made by the device quantiser only)

inline float mx4_bits_to_float(uint32_t u) {
  float f;
  memcpy(&f, &u, 4);
  return f;
}
// Magnitude of an fp16 bit pattern (finite): an exact product, subnormal numbers included.
inline float mx4_magnitude(uint16_t h) { return mx4_bits_to_float((uint32_t)(h & 0x7fff) << 13) * 0x1p112f; }

// Scale byte of a block whose largest magnitude has the fp16 bits `top` (finite).
inline uint8_t mx4_scale_of(uint16_t top) {
  const float f = mx4_magnitude(top);
  if (f == 0.f) return MX4_ONE;
  uint32_t u;
  memcpy(&u, &f, 4);
  return (uint8_t)((u >> 23) - 2);      // (the exponent's field is 127 + floor(log2))
}
// What a block with this scale byte multiplies its values with.
inline float mx4_factor(uint8_t scale) { return mx4_bits_to_float((uint32_t)(254 - scale) << 23); }
// Code of an fp16 value in a block with this factor: the number of midpoints below it, a midpoint itself counting
// where the code above is the even one.
inline uint8_t mx4_code(uint16_t h, float factor) {
  const float t = mx4_magnitude(h) * factor;
  const int c = (t > 0.25f) + (t >= 0.75f) + (t > 1.25f) + (t >= 1.75f) + (t > 2.5f) + (t >= 3.5f) + (t > 5.f);
  return (uint8_t)(c | (h >> 15 << 3));
}
// fp16 bits of a code in a block with this scale byte (any that mx4_scale_of gives).
inline uint16_t mx4_value(uint8_t code, uint8_t scale) {
  static const float grid[8] = {0.f, 0.5f, 1.f, 1.5f, 2.f, 3.f, 4.f, 6.f};
  const float v = grid[code & 7] * mx4_bits_to_float((uint32_t)scale << 23);
  const uint16_t sign = (uint16_t)((code & 8) << 12);
  if (v < 0x1p-14f) return (uint16_t)(sign | (uint16_t)(v * 0x1p24f));       // a whole number of 2^-24
  uint32_t u;
  memcpy(&u, &v, 4);
  return (uint16_t)(sign | ((u >> 13) - (112u << 10)));
}

}  // namespace twg
