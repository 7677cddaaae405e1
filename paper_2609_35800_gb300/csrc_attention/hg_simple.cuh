// Attention of one query row by one warp, key after key: the plainest form of the online softmax.
#pragma once
#include "hg_rows.cuh"

namespace hg {

struct RowState {
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};  // lane: channels 4 lane ..
};

template <bool F16>
__device__ __forceinline__ float4 lane_channels4(const uint16_t* row, int lane) {
  const uint2 w = ldg8(row + 4 * lane);
  const float2 a = unpack2<F16>(w.x), b = unpack2<F16>(w.y);
  return make_float4(a.x, a.y, b.x, b.y);
}

// One key: q is scaled by log2(e) times the softmax scale.
template <bool F16>
__device__ __forceinline__ void attend_key(RowState& st, const float4& q, float scale, const uint16_t* k,
                                           const uint16_t* v, int lane) {
  const float4 x = lane_channels4<F16>(k, lane), y = lane_channels4<F16>(v, lane);
  const float s = warp_sum(q.x * x.x + q.y * x.y + q.z * x.z + q.w * x.w) * scale;
  const float m = fmaxf(st.m, s), base = m == -INFINITY ? 0.f : m;
  const float keep = expf(st.m - base), p = expf(s - base);
  st.m = m;
  st.l = st.l * keep + p;
  st.o[0] = st.o[0] * keep + p * y.x;
  st.o[1] = st.o[1] * keep + p * y.y;
  st.o[2] = st.o[2] * keep + p * y.z;
  st.o[3] = st.o[3] * keep + p * y.w;
}

template <bool F16>
__device__ __forceinline__ void store_row(const RowState& st, uint16_t* out, float* lse, int lane, bool empty) {
  const float r = empty ? 0.f : 1.0f / st.l;
  *reinterpret_cast<uint2*>(out + 4 * lane) =
      make_uint2(pack2<F16>(st.o[0] * r, st.o[1] * r), pack2<F16>(st.o[2] * r, st.o[3] * r));
  if (lse && lane == 0) *lse = st.m + logf(st.l);
}

}  // namespace hg
