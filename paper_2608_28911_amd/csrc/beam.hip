// beam.hip -- beam search's choice on gfx950: of a group's beams b with scores a_b
// and logits x_b, the k candidates (b, v) of the largest
//   t(b, v) = a_b + x_b[v] - ln sum_u exp x_b[u],
// equal ones by lower (b, v).
//
// Within a row t follows x, so one pass over the logits keeps a row's k largest by
// (x, v) and its sum of exponentials, and candidates of different rows meet only
// afterwards, k of each.  There the order can hang on the last place: a lane's sums
// are kept, joined and scaled, their logarithm is taken and t is worked out in 64 bits.
// What is fp32 are the exponentials and the sum of a vector's: (2.23 ln V + 5) 2^-24 of
// ln sum at most (e^-y is off by its argument's roundings, 2.23 y 2^-24, and a step of
// the power of two; y, which the exponentials weigh, is no more than the row's entropy
// on average; three additions), 2e-6 for 160000 logits, 2e-8 where roundings go either
// way.  (With a lane's sums in fp32 it grows with V: 7e-6 where many small exponentials
// stand beside a large one.)
#include "paged.h"
#include "tokens.h"

namespace semkv {
namespace {

constexpr int kMostEach = 4;                     // candidates of a group (64 beams' 64 at most) to a thread that chooses

constexpr int kAtOnce = 8, kSure = 120;          // keys of a row's splits that a lane takes at once; those that a wave counts into order

// Partial of one split of a row: m and pad, S (64 bits), then the kept keys.
__host__ __device__ constexpr int partial_words(int k) { return 4 + 2 * k; }

// e^d for d <= 0 (sums below a larger maximum), to 4e-13: 2^k times the series of what
// is left, |r| <= ln 2 / 2, as far as r^10/10!.  (Every wave comes by here: with exp()
// 0.3 to 1.1 us a call more.)
__device__ inline double exp_below(double d) {
  d = fmax(d, -1000.0);                           // 0 from there on
  const double k = rint(d * 1.4426950408889634), r = fma(k, -0.6931471805599453, d);
  double e = 1.0 / 3628800;
  e = fma(e, r, 1.0 / 362880);
  e = fma(e, r, 1.0 / 40320);
  e = fma(e, r, 1.0 / 5040);
  e = fma(e, r, 1.0 / 720);
  e = fma(e, r, 1.0 / 120);
  e = fma(e, r, 1.0 / 24);
  e = fma(e, r, 1.0 / 6);
  e = fma(e, r, 0.5);
  e = fma(e, r, 1.0);
  e = fma(e, r, 1.0);
  return ldexp(e, int(k));
}

struct Row { float m; double S; };                // a lane's maximum, and sum e^(x-m)

__device__ inline void raise(Row& a, float m) {   // m >= a.m
  a.S *= exp_below(double(a.m) - double(m));
  a.m = m;
}

// The lanes' sum, in every lane, as over_wave.
__device__ inline double sum_wave(double x) {
  auto with = [](double v, auto move) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = move(uint32_t(u)), hi = move(uint32_t(u >> 32));
    return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
  };
  auto dpp = [](auto ctrl) {
    return [](uint32_t v) { return uint32_t(__builtin_amdgcn_mov_dpp(int(v), decltype(ctrl)::value, 0xF, 0xF, true)); };
  };
  x += with(x, dpp(std::integral_constant<int, 0xB1>{}));    // lane xor 1
  x += with(x, dpp(std::integral_constant<int, 0x4E>{}));    // lane xor 2
  x += with(x, dpp(std::integral_constant<int, 0x141>{}));   // mirror of 8 lanes
  x += with(x, dpp(std::integral_constant<int, 0x140>{}));   // mirror of 16
  // rows of 16 lanes, and halves of the wave, are exchanged
  auto pair = [](double v, auto swap) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const auto lo = swap(uint32_t(u)), hi = swap(uint32_t(u >> 32));
    return __builtin_bit_cast(double, uint64_t(hi[0]) << 32 | lo[0]) + __builtin_bit_cast(double, uint64_t(hi[1]) << 32 | lo[1]);
  };
  x = pair(x, [](uint32_t v) { return __builtin_amdgcn_permlane16_swap(v, v, false, false); });
  return pair(x, [](uint32_t v) { return __builtin_amdgcn_permlane32_swap(v, v, false, false); });
}

// 16 bytes from an element's address (global loads need no more on gfx950).
template <int DT>
__device__ inline uint4 load_anywhere(const char* p) {
  uint4 v;
  __builtin_memcpy(&v, __builtin_assume_aligned(p, Elem<DT>::size), 16);
  return v;
}

// One workgroup takes a row, or a share of one where there are few.  The pass only
// sums and keeps each lane's largest logit; the k-th largest of these, over the
// workgroup, bounds what it can keep, and the few lanes that reach it (k, and what
// ties) are looked through again, a lane's vectors across the wave; what reaches the
// bound is put in order by counting.  (A list kept on the way took 33 us for 256 rows
// of 128000 fp16 logits and k = 8, half of its vector instructions insertions; now 18.9 to
// 19.3, of which 12 go with the logits, 5.4 TB/s.)
template <int DT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void beam_rows_kernel(BeamArgs a) {
  constexpr int V = Elem<DT>::vec, NT = 64 * WAVES, U = 4;
  __shared__ double sm_S[WAVES];
  __shared__ uint32_t sm_most[NT];
  __shared__ uint32_t sm_hi[NT], sm_lo[NT];                  // a wave's candidates: 64 of them
  __shared__ int sm_n[WAVES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  const float score = a.scores[row];
  const int ended = a.ended ? a.ended[row] : 0;
  const int64_t g = row / a.width;
  const char* x = static_cast<const char*>(a.x) + (g * a.s_group + (row - g * a.width) * a.s_beam) * Elem<DT>::size;
  // vectors from the row's first element on, wherever that lies: rows of the same
  // logits have the same sum to the last bit, and their candidates stay equal
  const int64_t vecs = a.vocab / V;
  const int64_t v0 = vecs * blockIdx.y / a.nsplit, v1 = vecs * (blockIdx.y + 1) / a.nsplit;
  // a beam that has no candidates of its own row may have no logits in memory: looked at
  // before the first load (the places above are worked out meanwhile)
  if (score == -INFINITY || ended) return;
  Row s = {kFloor, 0.0};
  const int k = a.k;

  // what is behind the last whole vector
  const int64_t tail = vecs * V + lane;
  const bool ends = blockIdx.y + 1 == a.nsplit && wave == 0 && tail < a.vocab;
  const float last = ends ? load1<DT>(x, tail) : -INFINITY;

  uint4 next[U];
  auto load = [&](int64_t v) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = v + u * NT;
      if (at < v1) next[u] = load_anywhere<DT>(x + 16 * at);
    }
  };
  // `count` vectors to the sum: the maximum of all, then each one's exponentials (in some
  // lane of a wave the maximum rises nearly every time, which is 20 instructions in 64
  // bits: with a vector at a time 256 rows of 128000 take 2.3 us more)
  auto sum = [&](auto count, const uint4* w) __attribute__((always_inline)) {
    constexpr int N = decltype(count)::value;
    float e[N][V], mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      unpack<DT>(w[u], e[u]);
#pragma unroll
      for (int i = 0; i < V; ++i) mx = fmaxf(mx, e[u][i]);
    }
    if (mx > s.m) raise(s, mx);
#pragma unroll
    for (int u = 0; u < N; ++u) {
      float p[V];
#pragma unroll
      for (int i = 0; i < V; ++i) p[i] = exp_of(e[u][i] - s.m);
#pragma unroll
      for (int d = V / 2; d > 0; d /= 2)
#pragma unroll
        for (int i = 0; i < d; ++i) p[i] += p[i + d];
      s.S += double(p[0]);
    }
  };
  load(v0 + tid);
  for (int64_t v = v0 + tid; v < v1; v += NT * U) {
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = next[u];
    load(v + NT * U);                                        // under way while these are looked at
    if (v + NT * (U - 1) < v1) {
      sum(std::integral_constant<int, U>{}, w);
    } else {
#pragma unroll
      for (int u = 0; u < U - 1; ++u)
        if (v + u * NT < v1) sum(std::integral_constant<int, 1>{}, w + u);
    }
  }
  if (last > s.m) raise(s, last);
  s.S += ends ? double(exp_of(last - s.m)) : 0.0;

  // the bound: of the lanes' largest, in the order of their upper 16 bits
  sm_most[tid] = order_of(s.m);
  __syncthreads();
  uint32_t most[WAVES], least = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) most[w] = sm_most[64 * w + lane];
  // the lanes' sums relative to the workgroup's maximum
  float m = logit_of(most[0]);
#pragma unroll
  for (int w = 1; w < WAVES; ++w) m = fmaxf(m, logit_of(most[w]));
  m = over_wave(m, [](float p, float q) { return fmaxf(p, q); });
  const float own = s.m;
  raise(s, m);
  const double S = sum_wave(s.S);
  if (lane == 0) sm_S[wave] = S;
#pragma unroll
  for (int b = 31; b >= 16; --b) {
    int n = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) n += __popcll(__ballot(most[w] >= (least | 1u << b)));
    if (n >= k) least |= 1u << b;
  }
  const float bound = least > order_of(-INFINITY) ? logit_of(least) : kFloor;   // -inf is no candidate
  // f(may, order, complemented index): every logit of this wave that reaches the bound
  auto visit = [&](auto f) {
    uint64_t who = __ballot(own >= bound);
    while (who) {                                            // four lanes' vectors at a time
      constexpr int B = 4;
      int from[B];
#pragma unroll
      for (int i = 0; i < B; ++i) {
        from[i] = who ? __ffsll((unsigned long long)who) - 1 : -1;
        who &= who - 1;
      }
      for (int64_t j0 = 0; v0 + 64 * wave + j0 * NT < v1; j0 += 64) {
        uint4 w[B];
        bool in[B];
#pragma unroll
        for (int i = 0; i < B; ++i) {
          const int64_t at = v0 + 64 * wave + from[i] + (j0 + lane) * NT;
          in[i] = from[i] >= 0 && at < v1;
          if (in[i]) w[i] = load_anywhere<DT>(x + 16 * at);
        }
#pragma unroll
        for (int i = 0; i < B; ++i) {
          if (from[i] < 0) break;
          float e[V];
          unpack<DT>(w[i], e);
#pragma unroll
          for (int d = 0; d < V; ++d) {
            const bool may = in[i] && e[d] >= bound;
            if (__any(may)) f(may, order_of(e[d]), ~uint32_t((v0 + 64 * wave + from[i] + (j0 + lane) * NT) * V + d));
          }
        }
      }
    }
    if (__any(ends && last >= bound)) f(ends && last >= bound, order_of(last), ~uint32_t(tail));
  };
  int n = 0;
  visit([&](bool may, uint32_t h, uint32_t l) {
    const uint64_t m = __ballot(may);
    const int at = n + int(__builtin_amdgcn_mbcnt_hi(uint32_t(m >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(m), 0)));
    if (may && at < 64) {
      sm_hi[64 * wave + at] = h;
      sm_lo[64 * wave + at] = l;
    }
    n += __popcll(m);
  });
  if (n > 64) {                                              // ties: a list in order, of the first k
    Kept kept = {0u, 0u};
    visit([&](bool may, uint32_t h, uint32_t l) { keep_all(kept, may, h, l, k, lane); });
    sm_hi[64 * wave + lane] = kept.hi;
    sm_lo[64 * wave + lane] = kept.lo;
    n = k;
  }
  if (lane == 0) sm_n[wave] = n;
  __syncthreads();
  // every candidate counts those before it: its place
  uint32_t* p = reinterpret_cast<uint32_t*>(a.ws) + (row * a.nsplit + blockIdx.y) * partial_words(k);
  const uint32_t h = sm_hi[tid], l = sm_lo[tid];
  int place = 0, all = 0;
  for (int w = 0; w < WAVES; ++w) {
    const int c = sm_n[w];
    all += c;
    for (int i = 0; i < c; ++i) {
      const uint32_t hi = sm_hi[64 * w + i], lo = sm_lo[64 * w + i];
      place += hi > h || (hi == h && lo > l);
    }
  }
  if (lane < n && place < k) {
    p[4 + 2 * place] = h;
    p[5 + 2 * place] = l;
  }
  for (int i = all + tid; i < k; i += NT) p[4 + 2 * i] = p[5 + 2 * i] = 0;
  if (tid == 0) {
    double all = sm_S[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) all += sm_S[w];
    p[0] = __float_as_uint(m);
    *reinterpret_cast<double*>(p + 2) = all;
  }
}

// LDS accesses of the wave's other lanes before what follows.
__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// One workgroup chooses a group's candidates: its waves (one for each beam, 16 at
// most) join the rows' splits, each row's list is in order, and the lists are joined
// by places: a candidate's is its own in its list and the number of those before it in
// the other (64 beams of 64: six joins; counting in all 63 other lists at once took 300
// us).
template <bool MANY>
__global__ __launch_bounds__(1024) void beam_choose_kernel(BeamArgs a) {
  extern __shared__ double sm_t[];                   // [width][k]
  uint2* sm_sure = reinterpret_cast<uint2*>(sm_t + a.width * a.k);         // [waves][kSure], and later
  uint16_t* sm_i = reinterpret_cast<uint16_t*>(sm_sure);                   // [width][k]: no more than 256 a wave
  int32_t* sm_v = reinterpret_cast<int32_t*>(sm_sure + (blockDim.x >> 6) * kSure);   // [width][k]
  __shared__ int sm_bad, sm_n;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = a.k, threads = blockDim.x;
  const int64_t g = blockIdx.x;
  if (tid == 0) sm_bad = sm_n = 0;
  __syncthreads();
  for (int b = wave; b < a.width; b += threads >> 6) {
    const int64_t row = g * a.width + b;
    const float score = a.scores[row];
    const int ended = a.ended ? a.ended[row] : 0;
    // all of these are under way before the first is looked at (what is not read of a
    // row that has no candidates is not used)
    const uint32_t* p = reinterpret_cast<const uint32_t*>(a.ws) + row * a.nsplit * partial_words(k);
    const int total = a.nsplit * k;
    auto key = [&](int at, uint32_t& h, uint32_t& l) {
      const int sp = at / k, j = at - sp * k;
      const bool valid = at < total;
      const uint32_t* q = p + (valid ? sp * partial_words(k) + 4 + 2 * j : 0);
      h = q[0];
      l = q[1];
      if (!valid) h = l = 0;
    };
    constexpr int N = MANY ? kAtOnce : 1;
    uint32_t h[N], l[N];
    const uint32_t* own = p + min(lane, a.nsplit - 1) * partial_words(k);
    const float own_m = lane < a.nsplit ? __uint_as_float(own[0]) : kFloor;
    const double own_S = *reinterpret_cast<const double*>(own + 2);
    key(lane, h[0], l[0]);
    double t = -INFINITY;
    int32_t v = 0;
    bool bad = !(score < INFINITY);
    if (ended) {
      if (lane == 0) t = double(score);
      v = a.pad;
    } else if (score != -INFINITY) {
#pragma unroll
      for (int c = 1; c < N; ++c) {
        h[c] = l[c] = 0;
        if (64 * c < total) key(64 * c + lane, h[c], l[c]);
      }
      float m = own_m;
      for (int i = lane + 64; i < a.nsplit; i += 64) m = fmaxf(m, __uint_as_float(p[i * partial_words(k)]));
      m = over_wave(m, [](float x, float y) { return fmaxf(x, y); });
      double S = lane < a.nsplit ? own_S * exp_below(double(own_m) - double(m)) : 0.0;
      for (int i = lane + 64; i < a.nsplit; i += 64) {
        const uint32_t* q = p + i * partial_words(k);
        S += *reinterpret_cast<const double*>(q + 2) * exp_below(double(__uint_as_float(q[0])) - double(m));
      }
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) S += __shfl_xor(S, d);
      Kept kept = {h[0], l[0]};                      // one split: its keys are in order
      if (!MANY && a.nsplit > 1) {
        kept = {0u, 0u};
        const uint32_t least = kth_order(h[0], k);   // of the first 64 keys, which the rest cannot lower
        for (int i = 0; i < total; i += 64) {
          if (i) key(i + lane, h[0], l[0]);
          keep_all(kept, h[0] != 0 && h[0] >= least, h[0], l[0], k, lane);
        }
      }
      if (MANY) {
        // keys that reach the k-th largest of the first ones are counted into order; where
        // ties are more than there is room for, a list is kept
        uint32_t least = 0;
#pragma unroll
        for (int b = 31; b >= 16; --b) {
          int n = 0;
#pragma unroll
          for (int c = 0; c < N; ++c) n += __popcll(__ballot(h[c] >= (least | 1u << b)));
          if (n >= k) least |= 1u << b;
        }
        uint2* sure = sm_sure + wave * kSure;
        int n = 0;
        auto take = [&](uint32_t h, uint32_t l) {
          const bool may = h != 0 && h >= least;
          const uint64_t who = __ballot(may);
          const int at = n + int(__builtin_amdgcn_mbcnt_hi(uint32_t(who >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(who), 0)));
          if (may && at < kSure) sure[at] = make_uint2(h, l);
          n += __popcll(who);
        };
#pragma unroll
        for (int c = 0; c < N; ++c) take(h[c], l[c]);
        for (int i = 64 * N; i < total; i += 64) {
          uint32_t hi, lo;
          key(i + lane, hi, lo);
          take(hi, lo);
        }
        if (n <= kSure) {
          wave_sync();
          const uint2 x = sure[min(lane, kSure - 1)], y = sure[min(64 + lane, kSure - 1)];
          int px = 0, py = 0;
#pragma unroll 4
          for (int i = 0; i < n; ++i) {
            const uint2 z = sure[i];
            px += z.x > x.x || (z.x == x.x && z.y > x.y);
            py += z.x > y.x || (z.x == y.x && z.y > y.y);
          }
          wave_sync();
          if (lane < n) sure[px] = x;
          if (64 + lane < n) sure[py] = y;
          wave_sync();
          const uint2 z = sure[lane];
          kept = lane < n ? Kept{z.x, z.y} : Kept{0u, 0u};
          wave_sync();                               // (the wave's next beam)
        } else {
          kept = {0u, 0u};
          for (int i = 0; i < total; i += 64) {
            uint32_t hi, lo;
            key(i + lane, hi, lo);
            keep_all(kept, hi != 0 && hi >= least, hi, lo, k, lane);
          }
        }
      }
      // a row without any logit above -inf has no candidates; a NaN or +inf is reported
      const double lse = double(m) + log(S);
      const bool some = S > 0.0;
      bad = bad || !(S < INFINITY);
      const float x = kept.hi ? logit_of(kept.hi) : -INFINITY;
      if (some && x > -INFINITY) {
        t = double(score) + (double(x) - lse);
        v = int32_t(~kept.lo);
      }
    }
    if (bad && lane == 0) sm_bad = 1;
    if (lane < k) {
      sm_t[b * k + lane] = t;
      sm_v[b * k + lane] = v;
    }
    const uint64_t there = __ballot(lane < k && t > -INFINITY);
    if (lane == 0) atomicAdd(&sm_n, __popcll(there));
  }
  __syncthreads();
  const bool bad = sm_bad != 0;
  const int n = bad ? 0 : sm_n;
  for (int i = n + tid; i < k; i += threads) {       // fewer candidates than wanted
    a.out_scores[g * k + i] = bad ? NAN : -INFINITY;
    a.parents[g * k + i] = -1;
    a.tokens[g * k + i] = -1;
  }
  if (bad) return;
  auto put = [&](int place, double t, int i) {       // candidate i of the lists
    a.out_scores[g * k + place] = float(t);
    a.parents[g * k + place] = int32_t(g * a.width + i / k);
    a.tokens[g * k + place] = sm_v[i];
  };
  if (a.width * k <= 128) {                          // few: a candidate counts all that are before it
    for (int i = tid; i < a.width * k; i += threads) {
      const double t = sm_t[i];
      if (!(t > -INFINITY)) continue;
      int place = 0;
#pragma unroll 4
      for (int j = 0; j < a.width * k; ++j) place += sm_t[j] > t || (sm_t[j] == t && j < i);
      if (place < k) put(place, t, i);
    }
    return;
  }
  // lists of k in order, joined two by two; equal ones: the lower beams' first
  for (int i = tid; i < a.width * k; i += threads) sm_i[i] = uint16_t(i);
  __syncthreads();
  for (int s = 1; s < a.width; s <<= 1) {
    const int pairs = (a.width + s - 1) / (2 * s);   // of lists 2 p s and 2 p s + s
    double t[kMostEach];
    int i[kMostEach], to[kMostEach];
#pragma unroll
    for (int e = 0; e < kMostEach; ++e) {
      const int at = tid + e * threads;
      to[e] = -1;
      if (at >= pairs * 2 * k) continue;
      const int pair = int(uint32_t(at) / uint32_t(2 * k)), r = at - pair * 2 * k, upper = r >= k, j = r - upper * k;
      const int own = (2 * pair + upper) * s * k, other = (2 * pair + 1 - upper) * s * k;
      t[e] = sm_t[own + j];
      i[e] = sm_i[own + j];
      int lo = 0, hi = k - j;                        // entries of the other list before it; at k places it is out
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        const double u = sm_t[other + mid];
        if (u > t[e] || (u == t[e] && upper)) lo = mid + 1;
        else hi = mid;
      }
      if (j + lo < k) to[e] = 2 * pair * s * k + j + lo;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kMostEach; ++e)
      if (to[e] >= 0) {
        sm_t[to[e]] = t[e];
        sm_i[to[e]] = uint16_t(i[e]);
      }
    __syncthreads();
  }
  if (tid < k && sm_t[tid] > -INFINITY) put(tid, sm_t[tid], sm_i[tid]);
}

// Splits of a row: enough workgroups for the chip where there are few rows, each
// with 8192 logits at least: a workgroup's fixed part (launch, first logits, bound,
// second look, order) is 7 us.  (1024 workgroups for 256 rows of 128000: 26.2 us a
// call instead of 25.0, 2048: 28.6.)
int splits(int64_t rows, int64_t vocab) {
  int64_t n = 512 / rows;
  if (n > vocab / 8192) n = vocab / 8192;
  return n < 1 ? 1 : int(n);
}

}  // namespace

size_t beam_select_workspace(int64_t rows, int64_t vocab, int k) {
  return size_t(rows) * splits(rows, vocab) * partial_words(k) * 4;
}

int launch_beam_select(BeamArgs a, hipStream_t s) {
  const int64_t rows = a.groups * a.width;
  a.nsplit = splits(rows, a.vocab);
  const dim3 grid(unsigned(rows), unsigned(a.nsplit));
  if (a.dtype == 0) hipLaunchKernelGGL((beam_rows_kernel<0, 4>), grid, dim3(256), 0, s, a);
  else if (a.dtype == 1) hipLaunchKernelGGL((beam_rows_kernel<1, 4>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((beam_rows_kernel<2, 4>), grid, dim3(256), 0, s, a);
  const int waves = a.width < 16 ? a.width : 16;
  const size_t lds = size_t(a.width) * a.k * 12 + size_t(waves) * kSure * 8;
  // many keys of a row's splits are counted, few put into a list one after another (8 beams'
  // 32 best, 384 keys each: 40 us a call in a list, 28 counted; 4 beams' 4 best, 60 keys:
  // 11.7 and 14.2)
  if (a.nsplit * a.k > 128) hipLaunchKernelGGL((beam_choose_kernel<true>), dim3(unsigned(a.groups)), dim3(64 * waves), lds, s, a);
  else hipLaunchKernelGGL((beam_choose_kernel<false>), dim3(unsigned(a.groups)), dim3(64 * waves), lds, s, a);
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

}  // namespace semkv
