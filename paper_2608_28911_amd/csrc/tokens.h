// tokens.h -- device helpers of the kernels that read rows of logits (logprob.hip,
// beam.hip): loads, a lane's running sums, and the keys of the largest logits kept
// in order across the lanes of a wave.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace semkv {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

template <int DT>
struct Elem { static constexpr int size = DT == 2 ? 4 : 2, vec = 16 / size; };

template <int DT>
__device__ inline float load1(const void* row, int64_t i) {
  if constexpr (DT == 2) return static_cast<const float*>(row)[i];
  const uint32_t b = static_cast<const uint16_t*>(row)[i];
  if constexpr (DT == 0) return __half2float(__ushort_as_half(uint16_t(b)));
  return __uint_as_float(b << 16);
}

template <int DT>
__device__ inline void unpack(const uint4& v, float (&x)[Elem<DT>::vec]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (DT == 2) {
      x[e] = __uint_as_float(w[e]);
    } else if constexpr (DT == 1) {
      x[2 * e] = __uint_as_float(w[e] << 16);
      x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
    } else {
      x[2 * e] = __half2float(__ushort_as_half(uint16_t(w[e] & 0xFFFFu)));
      x[2 * e + 1] = __half2float(__ushort_as_half(uint16_t(w[e] >> 16)));
    }
  }
}

// Running sums of a lane, relative to its maximum.  The floor below keeps the
// maximum finite where every logit so far is -inf.
constexpr float kFloor = -3.4028234663852886e38f;
struct Sums { float m, S, T; };

__device__ inline float exp_of(float y) { return __builtin_amdgcn_exp2f(y * kLog2e); }

// x contributes e^(x-m) and e^(x-m)(x-m), 0 and 0 where x is -inf (the clamp
// keeps 0 * inf out of T; a NaN stays one through p)
__device__ inline void add(Sums& a, float x) {
  const float y = x - a.m, p = exp_of(y);
  a.S += p;
  a.T = fmaf(p, fmaxf(y, -200.0f), a.T);
}

__device__ inline void raise(Sums& a, float m) {          // m >= a.m
  const float d = a.m - m, f = exp_of(d);
  a.T = f * fmaf(a.S, fmaxf(d, -200.0f), a.T);
  a.S *= f;
  a.m = m;
}

// Within 16 lanes by DPP moves, then rows of 16 lanes are exchanged in
// registers; every lane has the result.
template <class F>
__device__ inline float over_wave(float x, F f) {
  auto dpp = [](float v, auto ctrl) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), decltype(ctrl)::value, 0xF, 0xF, true));
  };
  x = f(x, dpp(x, std::integral_constant<int, 0xB1>{}));     // lane xor 1
  x = f(x, dpp(x, std::integral_constant<int, 0x4E>{}));     // lane xor 2
  x = f(x, dpp(x, std::integral_constant<int, 0x141>{}));    // mirror of 8 lanes
  x = f(x, dpp(x, std::integral_constant<int, 0x140>{}));    // mirror of 16
  const uint32_t u = __float_as_uint(x);
  const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t y = __float_as_uint(f(__uint_as_float(p[0]), __uint_as_float(p[1])));
  const auto q = __builtin_amdgcn_permlane32_swap(y, y, false, false);
  return f(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

// The lanes' states joined, in every lane.
__device__ inline Sums join_wave(Sums s) {
  raise(s, over_wave(s.m, [](float a, float b) { return fmaxf(a, b); }));
  auto add = [](float a, float b) { return a + b; };
  return {s.m, over_wave(s.S, add), over_wave(s.T, add)};
}

// Order of logits as unsigned integers: NaN above everything, -0 as +0; 0 is
// below every logit.
__device__ inline uint32_t order_of(float x) {
  if (x != x) return ~0u;
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The wave's kept keys, descending over lanes 0 .. k-1: lane i holds the i-th.
struct Kept {
  uint32_t hi, lo;                       // order, complemented index
  __device__ bool above(uint32_t h, uint32_t l) const { return hi > h || (hi == h && lo > l); }
};
__device__ inline void keep(Kept& s, uint32_t h, uint32_t l, int lane) {   // h, l uniform
  const int at = __popcll(__ballot(s.above(h, l)));       // kept keys above it come first
  // the lane below's keys: a DPP move along the wave
  const uint32_t uh = __builtin_amdgcn_mov_dpp(int(s.hi), 0x138, 0xF, 0xF, true), ul = __builtin_amdgcn_mov_dpp(int(s.lo), 0x138, 0xF, 0xF, true);
  if (lane == at) {
    s.hi = h;
    s.lo = l;
  } else if (lane > at) {
    s.hi = uh;
    s.lo = ul;
  }
}
// The keys of lanes with `may` into the kept ones.  Those that no longer beat
// the last kept one drop out at every insertion.
__device__ inline void keep_all(Kept& s, bool may, uint32_t h, uint32_t l, int k, int lane) {
  while (true) {
    const uint32_t th = __builtin_amdgcn_readlane(s.hi, k - 1), tlo = __builtin_amdgcn_readlane(s.lo, k - 1);
    const uint64_t who = __ballot(may && (h > th || (h == th && l > tlo)));
    if (!who) return;
    const int from = __ffsll((unsigned long long)who) - 1;
    keep(s, __builtin_amdgcn_readlane(h, from), __builtin_amdgcn_readlane(l, from), lane);
    may = may && lane != from;
  }
}

__device__ inline float logit_of(uint32_t order) {
  return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order);
}

// The k-th largest of the lanes' orders (its upper 16 bits): as many lanes hold
// a logit that is no smaller, so a row's k likeliest are not below it.
__device__ inline uint32_t kth_order(uint32_t h, int k) {
  uint32_t t = 0;
#pragma unroll
  for (int b = 31; b >= 16; --b)
    if (__popcll(__ballot(h >= (t | 1u << b))) >= k) t |= 1u << b;
  return t;
}

}  // namespace
}  // namespace semkv
