// Device helpers for 16-bit rows: two channels of a word to binary32 and back, the position rotation, page addresses.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hg_attention.h"
#include "hg_common.cuh"
#include "hg_mma.cuh"

namespace hg {

template <bool F16>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if (F16) return half2_bits_to_float2(w);
  float2 f;
  bf16x2_to_f32(w, f.x, f.y);
  return f;
}
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return F16 ? pack_half2(lo, hi) : pack_bf16x2(lo, hi);
}

// Probabilities are held as 2^kLift e^(s - m) for the second product; a running maximum m may stay 2^kRescale behind, so the
// largest are 2^(kLift + kRescale).  FP16 ends at 2^-25: lifted by 2^7, below 65,504 still, terms down to 2^-32 of the
// largest are kept, where many small ones make up a part of a row.  BF16 reaches down to 2^-133 as it is.
constexpr float kRescale = 8.0f;
template <bool F16>
constexpr float kLift = F16 ? 7.0f : 0.0f;

// A row's 128 channels are divided among 8 lanes, 16 channels each, so that a lane holds whole pairs: with `half` =
// rot_dim / 2, lane c < half / 8 has the pairs [8c, 8c + 8), the others 16 channels that pass.  The lane's channels are
// [lo, lo + 8) and [hi, hi + 8).
struct LaneChannels {
  int lo, hi;
  bool turns;
};
__device__ __forceinline__ LaneChannels lane_channels(const Rotation& r, int c, bool rotate) {
  if (rotate && 8 * c < r.half && !r.interleaved) return {8 * c, r.half + 8 * c, true};
  // neighbours as pairs: channels [16c, 16c + 16); past the rotated ones likewise
  return {16 * c, 16 * c + 8, rotate && 8 * c < r.half};
}

// Cosines and sines of a token's pairs [8c, 8c + 8).
struct LaneAngles {
  float4 cos[2], sin[2];
};
__device__ __forceinline__ LaneAngles lane_angles(const Rotation& r, int c, int token) {
  const int part = 8 * c < r.end0 ? 0 : 8 * c < r.end1 ? 1 : 2;
  int pos = r.positions[(int64_t)part * r.position_stride + token];
  pos = min(max(pos, 0), r.table_len - 1);
  const float4* row = reinterpret_cast<const float4*>(r.table + (int64_t)pos * (2 * r.half));
  LaneAngles a;
  a.cos[0] = row[2 * c];
  a.cos[1] = row[2 * c + 1];
  a.sin[0] = row[r.half / 4 + 2 * c];
  a.sin[1] = row[r.half / 4 + 2 * c + 1];
  return a;
}

// (a c - b s, b c + a s) in binary32: the products that are subtracted or added last are part of an FMA.
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float x = fmaf(a, c, -(b * s));
  b = fmaf(b, c, a * s);
  a = x;
}

template <bool F16>
__device__ __forceinline__ void rotate_lane(uint4& lo, uint4& hi, const LaneAngles& g, bool interleaved) {
  uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  const float cs[8] = {g.cos[0].x, g.cos[0].y, g.cos[0].z, g.cos[0].w, g.cos[1].x, g.cos[1].y, g.cos[1].z, g.cos[1].w};
  const float sn[8] = {g.sin[0].x, g.sin[0].y, g.sin[0].z, g.sin[0].w, g.sin[1].x, g.sin[1].y, g.sin[1].z, g.sin[1].w};
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float2 x = unpack2<F16>(w[i]);
      turn(x.x, x.y, cs[i], sn[i]);
      w[i] = pack2<F16>(x.x, x.y);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float2 a = unpack2<F16>(w[i]), b = unpack2<F16>(w[4 + i]);
      turn(a.x, b.x, cs[2 * i], sn[2 * i]);
      turn(a.y, b.y, cs[2 * i + 1], sn[2 * i + 1]);
      w[i] = pack2<F16>(a.x, a.y);
      w[4 + i] = pack2<F16>(b.x, b.y);
    }
  }
  lo = make_uint4(w[0], w[1], w[2], w[3]);
  hi = make_uint4(w[4], w[5], w[6], w[7]);
}

// Element offset of a token's row in the pool.
__device__ __forceinline__ int64_t page_row(const PagePool& p, int page, int in_page, int head) {
  return page * p.page_stride + head * p.head_stride + in_page * p.token_stride;
}

}  // namespace hg
