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
// 256: a lane keeps its pair, a wave takes as many rows at a time as it has lanes
// for.  The room between rows keeps a row's 16-byte reads aligned and neighbouring
// rows' in different banks.
__host__ __device__ constexpr int turns_pitch(int d) { return d / 2 + 2; }
template <int D>
__device__ inline void make_turns(const RotaryArgs& rot, const PageWork& w, float2* turns) {
  const int half = rot.dim / 2, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;   // half: 64 at most
  const int rows = 64 / half, row = lane / half, pair = lane - row * half;
  if (row >= rows) return;
  const float f = rot.freqs[pair];
  for (int slot = w.lo + wave * rows + row; slot < w.hi; slot += 4 * rows)
    turns[slot * turns_pitch(D) + pair] = turn_of(position_of(rot, w, slot), f);
}

// Two values rounded to the type (nearest, ties to even) by the converts.
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
template <int BF>
__device__ inline uint32_t pack2(float x, float y) {
  if constexpr (BF) return __builtin_bit_cast(uint32_t, bf2v{__bf16(x), __bf16(y)});
  else return __builtin_bit_cast(uint32_t, half2v{_Float16(x), _Float16(y)});
}

// Sixteen channels of a row to be turned, or kept from rot.dim on: unit u is the
// pairs 8u .. 8u+7, then channels 16u .. 16u+15.  Both halves of a pair are one
// thread's, so that they may go back where they came from.
struct Unit { int at, bt; };     // channels at .. at+7, bt .. bt+7
__device__ inline Unit unit_of(const RotaryArgs& rot, int u) {
  const bool halves = 16 * u < rot.dim && !rot.interleaved;
  return {halves ? 8 * u : 16 * u, halves ? 8 * u + rot.dim / 2 : 16 * u + 8};
}

template <int BF>
__device__ inline void turn_unit(const RotaryArgs& rot, const float2* turns, int u, uint4 (&v)[2]) {
  if (16 * u >= rot.dim) return;
  const uint32_t p[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
  float x[16], y[16];
#pragma unroll
  for (int e = 0; e < 8; ++e) unpack2<BF>(p[e], x[2 * e], x[2 * e + 1]);
  const float4* t = reinterpret_cast<const float4*>(turns + 8 * u);
  if (!rot.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float4 w = t[i / 2];
      y[i] = turned_x(x[i], x[8 + i], make_float2(w.x, w.y));
      y[8 + i] = turned_y(x[i], x[8 + i], make_float2(w.x, w.y));
      y[i + 1] = turned_x(x[i + 1], x[9 + i], make_float2(w.z, w.w));
      y[9 + i] = turned_y(x[i + 1], x[9 + i], make_float2(w.z, w.w));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float4 w = t[i / 2];
      y[2 * i] = turned_x(x[2 * i], x[2 * i + 1], make_float2(w.x, w.y));
      y[2 * i + 1] = turned_y(x[2 * i], x[2 * i + 1], make_float2(w.x, w.y));
      y[2 * i + 2] = turned_x(x[2 * i + 2], x[2 * i + 3], make_float2(w.z, w.w));
      y[2 * i + 3] = turned_y(x[2 * i + 2], x[2 * i + 3], make_float2(w.z, w.w));
    }
  }
  uint32_t o[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = pack2<BF>(y[2 * e], y[2 * e + 1]);
  v[0] = make_uint4(o[0], o[1], o[2], o[3]);
  v[1] = make_uint4(o[4], o[5], o[6], o[7]);
}

// The query rows of a page, heads h0 .. h0 + heads - 1 of `units` units, turned by a
// workgroup of 256: a thread keeps its unit and head, and steps over rows, kAhead of
// them loaded before the first is stored.  Bound by vector instructions beside
// memory: 12 for each two pairs, unpacked, turned and rounded; the places of every
// unit worked out by divisions would be as many again.
constexpr int kAhead = 2;
template <int BF, int PITCH>
__device__ inline void turn_queries(const RotaryArgs& rot, const PageWork& w, const uint16_t* q, int64_t qT, int64_t qH, uint16_t* out,
                                    int64_t oT, int64_t oH, int h0, int heads, int units, const float2* turns) {
  const int all = heads * units, rows = all < 256 ? 256 / all : 1;      // units of a row, rows at a time
  for (int i0 = 0; i0 < all; i0 += 256) {
    const int row = all < 256 ? int(uint32_t(threadIdx.x) / uint32_t(all)) : 0, i = i0 + int(threadIdx.x) - row * all;
    if (row >= rows || i >= all) continue;
    const int h = int(uint32_t(i) / uint32_t(units)), u = i - h * units;
    const Unit c = unit_of(rot, u);
    const int first = w.lo + row, last = w.hi - 1;
    const uint16_t* from = q + w.row0 * qT + (h0 + h) * qH;
    uint16_t* to = out + w.row0 * oT + (h0 + h) * oH;
    for (int s0 = first; s0 <= last; s0 += rows * kAhead) {
      uint4 v[kAhead][2];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const uint16_t* x = from + min(s0 + k * rows, last) * qT;
        v[k][0] = *reinterpret_cast<const uint4*>(x + c.at);
        v[k][1] = *reinterpret_cast<const uint4*>(x + c.bt);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int slot = s0 + k * rows;
        if (slot > last) break;
        turn_unit<BF>(rot, turns + slot * PITCH, u, v[k]);
        *reinterpret_cast<uint4*>(to + slot * oT + c.at) = v[k][0];
        *reinterpret_cast<uint4*>(to + slot * oT + c.bt) = v[k][1];
      }
    }
  }
}

}  // namespace
}  // namespace semkv
