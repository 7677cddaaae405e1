// Device helpers for 8-bit pages: e4m3 codes, the blocks' scales, addresses.
#pragma once
#include <cuda_fp8.h>

#include "hg_rows.cuh"

namespace hg {

// Powers of two are compared and inverted by their exponent field.  448, e4m3's largest, is 1.75 * 2^8.
constexpr int kLeastField = 1, kMostField = 253;  // 2^-126 and 2^126: their inverses are normal too

// Exponent field of the least power of two s with |x| <= 448 s for the largest |x|, given by its bits (finite).
__device__ __forceinline__ int needed_field(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return max(e, kLeastField);
}
// That of a stored scale, raised to a power of two.
__device__ __forceinline__ int stored_field(float s) {
  return min(max((int)((__float_as_uint(s) & 0x7fffffffu) + 0x7fffffu >> 23), kLeastField), kMostField);
}
__device__ __forceinline__ float power_of_field(int field) { return __uint_as_float((uint32_t)field << 23); }
__device__ __forceinline__ float inverse_of_field(int field) { return __uint_as_float((uint32_t)(254 - field) << 23); }

// |x| as it counts for a scale: NaN and infinities do not.
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}

// Codes of (a, b) * inv; an infinity becomes NaN, which stays one.
__device__ __forceinline__ uint32_t encode2(float a, float b, float inv) {
  a = fabsf(a) < INFINITY ? a * inv : NAN;
  b = fabsf(b) < INFINITY ? b * inv : NAN;
  return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint2 encode8(const float* x, float inv) {
  return make_uint2(encode2(x[0], x[1], inv) | encode2(x[2], x[3], inv) << 16,
                    encode2(x[4], x[5], inv) | encode2(x[6], x[7], inv) << 16);
}

// The two codes of a word's lower half, and of its upper half, as FP16, exactly.  (One instruction each: through the
// conversion functions of the headers, halves taken apart and put together again, 32 tokens of the decode took 925
// instructions of a warp, 640 this way: 32 requests of 8,577 tokens 140 -> 118 us.)
__device__ __forceinline__ void decode4(uint32_t w, uint32_t& lower, uint32_t& upper) {
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}\n"
      : "=r"(lower), "=r"(upper)
      : "r"(w));
}
__device__ __forceinline__ void decode8(uint2 codes, float* x) {
  const uint32_t w[2] = {codes.x, codes.y};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t lower, upper;
    decode4(w[i], lower, upper);
    const float2 a = half2_bits_to_float2(lower), b = half2_bits_to_float2(upper);
    x[4 * i] = a.x;
    x[4 * i + 1] = a.y;
    x[4 * i + 2] = b.x;
    x[4 * i + 3] = b.y;
  }
}
// Codes times `ratio`, as codes again.
__device__ __forceinline__ uint2 recode8(uint2 codes, float ratio) {
  float x[8];
  decode8(codes, x);
  return encode8(x, ratio);
}

// A lane's 16 channels of a row in binary32: lo's eight, then hi's; turned where `g` is given.
template <bool F16>
__device__ __forceinline__ void row_values(const uint4& lo, const uint4& hi, const LaneAngles* g, bool interleaved,
                                           float (&x)[16]) {
  const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 f = unpack2<F16>(w[i]);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
  if (!g) return;
  const float cs[8] = {g->cos[0].x, g->cos[0].y, g->cos[0].z, g->cos[0].w, g->cos[1].x, g->cos[1].y, g->cos[1].z, g->cos[1].w};
  const float sn[8] = {g->sin[0].x, g->sin[0].y, g->sin[0].z, g->sin[0].w, g->sin[1].x, g->sin[1].y, g->sin[1].z, g->sin[1].w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (interleaved) turn(x[2 * i], x[2 * i + 1], cs[i], sn[i]);
    else turn(x[i], x[8 + i], cs[i], sn[i]);
  }
}
template <bool F16>
__device__ __forceinline__ uint4 pack8(const float* x) {
  return make_uint4(pack2<F16>(x[0], x[1]), pack2<F16>(x[2], x[3]), pack2<F16>(x[4], x[5]), pack2<F16>(x[6], x[7]));
}

// 16 channels side by side: one store of a whole sector where the row lies so.
__device__ __forceinline__ void store16(uint16_t* dst, const uint4& lo, const uint4& hi) {
  if ((reinterpret_cast<uintptr_t>(dst) & 31u) == 0) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};\n" ::"l"(dst), "r"(lo.x), "r"(lo.y), "r"(lo.z),
                 "r"(lo.w), "r"(hi.x), "r"(hi.y), "r"(hi.z), "r"(hi.w)
                 : "memory");
  } else {
    *reinterpret_cast<uint4*>(dst) = lo;
    *reinterpret_cast<uint4*>(dst + 8) = hi;
  }
}

// x, or the 16-bit type's largest value where it is beyond; NaN stays.
template <bool F16>
constexpr float kMost16 = F16 ? 65504.f : 0x1.fep127f;
template <bool F16>
__device__ __forceinline__ float in_range(float x) {
  return x > kMost16<F16> ? kMost16<F16> : x < -kMost16<F16> ? -kMost16<F16> : x;
}

// Byte offset of a token's codes in the pool; index of its block's scale.
__device__ __forceinline__ int64_t code_row(const PagePool8& p, int page, int in_page, int head) {
  return page * p.page_stride + head * p.head_stride + in_page * p.token_stride;
}
__device__ __forceinline__ int64_t scale_at(const PagePool8& p, int page, int in_page, int head) {
  return (((int64_t)page * p.heads + head) << (p.page_shift - kBlock8Shift)) + (in_page >> kBlock8Shift);
}
// Page of a request's token; -1 where its place is outside the table or the page outside the pool.
__device__ __forceinline__ int page_of(const PagePool8& p, const int* table_row, int table_stride, int token) {
  const int at = token >> p.page_shift;
  if (token < 0 || at >= table_stride) return -1;
  const int page = table_row[at];
  return page >= 0 && page < p.num_pages ? page : -1;
}

}  // namespace hg
