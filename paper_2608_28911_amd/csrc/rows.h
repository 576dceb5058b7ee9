// rows.h -- device helpers of the kernels that take rows of 16-bit values into pages
// (paged.hip, latent.hip): conversions, and turning rows by their positions.
#pragma once
#include <hip/hip_fp16.h>

#include "paged.h"

namespace semkv {
namespace {

__device__ inline float h2f(uint32_t b) { return __half2float(__ushort_as_half(uint16_t(b))); }
__device__ inline uint32_t f2h(float f) { return __half_as_ushort(__float2half_rn(f)); }

__device__ inline bool finite(float x) { return fabsf(x) < INFINITY; }     // false for NaN

template <int BF>
__device__ inline void unpack2(uint32_t d, float& a, float& b) {
  if constexpr (BF) {
    a = __uint_as_float(d << 16);
    b = __uint_as_float(d & 0xFFFF0000u);
  } else {
    a = h2f(d & 0xFFFFu);
    b = h2f(d >> 16);
  }
}

// The position that slot `slot` of the page is turned by.
__device__ inline int32_t position_of(const RotaryArgs& rot, const PageWork& w, int slot) {
  return rot.positions ? rot.positions[w.row0 + slot] : w.first + slot;
}

// Cosines and sines of the page's rows, [slot][pair], by the whole workgroup of
// 256; the room between rows keeps a row's 16-byte reads aligned and neighbouring
// rows' in different banks.
__host__ __device__ constexpr int turns_pitch(int d) { return d / 2 + 2; }
template <int D>
__device__ inline void make_turns(const RotaryArgs& rot, const PageWork& w, float2* turns) {
  const int half = rot.dim / 2, n = (w.hi - w.lo) * half;
  for (int i = threadIdx.x; i < n; i += 256) {
    const int slot = w.lo + i / half, pair = i % half;
    turns[slot * turns_pitch(D) + pair] = turn_of(position_of(rot, w, slot), rot.freqs[pair]);
  }
}

__device__ inline uint32_t pack2(float x, float y, bool bf16) {
  if (!bf16) return f2h(x) | f2h(y) << 16;
  uint32_t b[2] = {__float_as_uint(x), __float_as_uint(y)};
#pragma unroll
  for (int e = 0; e < 2; ++e)
    b[e] = (b[e] & 0x7FFFFFFFu) > 0x7F800000u ? 0x7FC0u : (b[e] + 0x7FFFu + ((b[e] >> 16) & 1u)) >> 16;
  return b[0] | b[1] << 16;
}

// Sixteen channels of a row turned, or as they are from rot.dim on: unit u is the
// pairs 8u .. 8u+7, then channels 16u .. 16u+15; p[0] goes to channels at .. at+7,
// p[1] to bt .. bt+7.  Both halves of a pair are one thread's, so that they may go
// where they came from.
template <int BF>
__device__ inline void turn_unit(const RotaryArgs& rot, const uint16_t* from, const float2* turns, int u, uint4 (&out)[2], int& at,
                                 int& bt) {
  const bool turned = 16 * u < rot.dim, halves = turned && !rot.interleaved;
  at = halves ? 8 * u : 16 * u;
  bt = halves ? 8 * u + rot.dim / 2 : 16 * u + 8;
  out[0] = *reinterpret_cast<const uint4*>(from + at);
  out[1] = *reinterpret_cast<const uint4*>(from + bt);
  if (!turned) return;
  const uint32_t p[8] = {out[0].x, out[0].y, out[0].z, out[0].w, out[1].x, out[1].y, out[1].z, out[1].w};
  float x[16], y[16];
#pragma unroll
  for (int e = 0; e < 8; ++e) unpack2<BF>(p[e], x[2 * e], x[2 * e + 1]);
  const float4* t = reinterpret_cast<const float4*>(turns + 8 * u);
  if (halves) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float4 v = t[i / 2];
      y[i] = turned_x(x[i], x[8 + i], make_float2(v.x, v.y));
      y[8 + i] = turned_y(x[i], x[8 + i], make_float2(v.x, v.y));
      y[i + 1] = turned_x(x[i + 1], x[9 + i], make_float2(v.z, v.w));
      y[9 + i] = turned_y(x[i + 1], x[9 + i], make_float2(v.z, v.w));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float4 v = t[i / 2];
      y[2 * i] = turned_x(x[2 * i], x[2 * i + 1], make_float2(v.x, v.y));
      y[2 * i + 1] = turned_y(x[2 * i], x[2 * i + 1], make_float2(v.x, v.y));
      y[2 * i + 2] = turned_x(x[2 * i + 2], x[2 * i + 3], make_float2(v.z, v.w));
      y[2 * i + 3] = turned_y(x[2 * i + 2], x[2 * i + 3], make_float2(v.z, v.w));
    }
  }
  uint32_t o[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = pack2(y[2 * e], y[2 * e + 1], BF);
  out[0] = make_uint4(o[0], o[1], o[2], o[3]);
  out[1] = make_uint4(o[4], o[5], o[6], o[7]);
}

}  // namespace
}  // namespace semkv
