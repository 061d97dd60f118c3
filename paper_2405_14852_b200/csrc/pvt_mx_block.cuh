// Quantisation of one block of a row to 4-bit block floating point, for the kernels that write such matrices.
//
// Elements.  Under e8m0 the scale is a power of two, so x / scale is exact and the conversion rounds once.  Under e4m3 the
// quotient x / (scale tensor_scale) is rounded before it is converted, which could carry it over a border between two
// elements; it is therefore converted twice, a little larger and a little smaller than computed (2^-20; its error is below
// 2^-22), and only where the two disagree are the borders themselves compared, in binary64, where their products with scale
// and tensor_scale are exact (2 + 4 + 24 significant bits).  The scale's own rounding is settled the same way.
#pragma once

#include "pvt_mx.cuh"

#ifdef __CUDACC__
namespace pvt {
namespace mx {
namespace {

constexpr float kMore = 1.00000095367431640625f, kLess = 0.99999904632568359375f;  // 1 + 2^-20, 1 - 2^-20

// two conversions of eight values each side by side: code of v[0] in the lowest four bits
__device__ __forceinline__ uint32_t e2m1_codes(const float* v) {
  uint32_t d;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(d)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return d;
}

// the element nearest to |x| / d, by its borders: n from (n - 1/2) on, in the order of codes
__device__ __noinline__ uint32_t e2m1_exact(float x, double d) {
  const double a = fabs((double)x);
  uint32_t n = 0;
  n += a > 0.25 * d;
  n += a >= 0.75 * d;
  n += a > 1.25 * d;
  n += a >= 1.75 * d;
  n += a > 2.5 * d;
  n += a >= 3.5 * d;
  n += a > 5.0 * d;
  return n | (__float_as_uint(x) >> 31 << 3);
}

// the e4m3 number nearest to amax / six_ts (at most 448), ties to the even one: by its midpoints, exact in binary64
__device__ __noinline__ uint32_t e4m3_exact(float amax, double six_ts) {
  uint16_t two;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(0.0f), "f"((float)((double)amax / six_ts)));
  const uint32_t c = two & 127u;  // rounded twice: it may be the neighbour
  const double v = e4m3_value(c), a = amax;
  if (c < 126) {
    const double mid = 0.5 * (v + (double)e4m3_value(c + 1)) * six_ts;
    if (a > mid || (a == mid && (c & 1))) return c + 1;
  }
  if (c > 0) {
    const double mid = 0.5 * (v + (double)e4m3_value(c - 1)) * six_ts;
    if (a < mid || (a == mid && (c & 1))) return c - 1;
  }
  return c;
}
// The same by the quotient a little larger and a little smaller than computed, where that decides it (and 6 tensor_scale and its
// reciprocal are normal numbers).
__device__ __forceinline__ uint32_t e4m3_scale(float amax, float ts, float inv) {
  const float q = amax * inv;
  uint16_t two;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(q * kLess), "f"(q * kMore));
  return (two >> 8) == (two & 255u) && inv > 1e-37f && inv < 1e38f ? two & 127u : e4m3_exact(amax, 6.0 * (double)ts);
}

// The span's elements from one of two orders to the other: eight consecutive ones in a lane, and (rows that no wide access can
// take) element 32 i + lane in place i of a lane.  Eight numbers are padded to nine: no bank is met twice either way.
template <bool TO_ROWS>
__device__ __forceinline__ void turn(float* buffer, float* v, uint32_t lane) {
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t at = TO_ROWS ? 8 * lane + i : 32 * i + lane;
    buffer[at + at / 8] = v[i];
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t at = TO_ROWS ? 32 * i + lane : 8 * lane + i;
    v[i] = buffer[at + at / 8];
  }
}

// what a tensor scale comes to
struct TensorScale {
  float ts = 1.0f, inv_six = 1.0f / 6.0f;
  bool bad = false;
  __device__ __forceinline__ explicit TensorScale(const float* p) {
    if (!p) return;
    ts = *p;
    bad = !(ts > 0.0f && ts < __uint_as_float(0x7f800000u));
    inv_six = 1.0f / (6.0f * ts);
  }
};
// The scale byte of a block, from the bits of its largest magnitude, and the codes of a lane's E elements of it.
template <int FMT, int E>
__device__ __forceinline__ uint32_t quantize_block(float* v, uint32_t top, const TensorScale& t, uint32_t* word) {
  const bool bad = top >= 0x7f800000u || t.bad;
  uint32_t byte;
#pragma unroll
  for (int w = 0; w < E / 8; ++w) word[w] = 0;
  if (FMT == PVT_MX_E8M0_32) {
    // floor(log2 a) - 2, biased; numbers below 2^-126 have a scale of 2^-127 in any case
    const int e = max((int)(top >> 23) - 2, 0);
    byte = bad ? 255u : (uint32_t)e;
    const float inv = __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
    for (int i = 0; i < E; i += 2) set2(v + i, mul2(two(v + i), both(inv)));
    if (!bad) {
#pragma unroll
      for (int w = 0; w < E / 8; ++w) word[w] = e2m1_codes(v + 8 * w);
    }
  } else {
    byte = bad ? 127u : e4m3_scale(__uint_as_float(top), t.ts, t.inv_six);
    if (!bad && byte) {
      const float s = e4m3_float(byte), d = s * t.ts;
      float r;
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d));
      const float more = r * kMore, less = r * kLess;
      // where d or r leave the range of normal numbers every element is compared with its borders
      const bool all = !(d >= 1e-30f && d <= 1e30f);
#pragma unroll
      for (int w = 0; w < E / 8; ++w) {
        float hi[8], lo[8];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const float2 x = two(v + 8 * w + i);
          set2(hi + i, mul2(x, both(more))), set2(lo + i, mul2(x, both(less)));
        }
        word[w] = e2m1_codes(hi);
        const uint32_t differ = all ? 0xffffffffu : word[w] ^ e2m1_codes(lo);
        if (differ) {
          const double dd = (double)s * (double)t.ts;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (differ >> (4 * i) & 15u) word[w] = (word[w] & ~(15u << (4 * i))) | e2m1_exact(v[8 * w + i], dd) << (4 * i);
        }
      }
    }
  }
  return byte;
}

// a matrix that a kernel writes, or none (codes null)
struct Held {
  uint8_t *codes, *scales;
  const float* tensor_scale;
  int64_t ld;
  uint32_t cols, tiles;  // tiles of scales, of a strip
  int32_t format;
};
inline Held held(const pvt_mx& m) {
  return Held{m.codes, m.scales, m.tensor_scale, m.ld, (uint32_t)m.cols, strip_tiles(m.cols, block_of(m.format)), m.format};
}

// A row's eight neighbouring values of each lane, from column c0 = 8 lane + a multiple of 256 (or of 128, in sixteen lanes) on, into
// codes and scales.  here: the row exists; listed: it has scales (those of rows and blocks that do not exist are 0).
template <int FMT>
__device__ __forceinline__ void put_eight(const Held& m, uint32_t row, uint32_t c0, bool here, bool listed, const TensorScale& t,
                                          float* v) {
  constexpr uint32_t LANES = FMT == PVT_MX_E8M0_32 ? 4 : 2;  // of a block
  const uint32_t lane = threadIdx.x & 31, block = c0 / (8 * LANES);
  uint32_t word;
  if (c0 + 8 > m.cols) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c0 + i >= m.cols) v[i] = 0.0f;
  }
  uint32_t top = top_of8(v);
#pragma unroll
  for (uint32_t d = 1; d < LANES; d *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
  uint32_t byte = quantize_block<FMT, 8>(v, top, t, &word);
  if (c0 >= m.cols || !here) byte = 0;  // no such block
  uint32_t four = byte | __shfl_down_sync(0xffffffffu, byte, LANES) << 8;
  four |= __shfl_down_sync(0xffffffffu, four, 2 * LANES) << 16;
  if (lane % (4 * LANES) == 0 && listed && block / 4 < m.tiles) *reinterpret_cast<uint32_t*>(m.scales + scale_at(row, block, m.tiles)) = four;
  if (!here || c0 >= m.cols) return;
  uint8_t* const to = m.codes + (int64_t)row * m.ld + c0 / 2;
  if (c0 + 8 <= m.cols) {
    *reinterpret_cast<uint32_t*>(to) = word;
  } else {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i)
      if (2 * i < m.cols - c0) to[i] = (uint8_t)(word >> (8 * i));
  }
}

}  // namespace
}  // namespace mx
}  // namespace pvt
#endif
