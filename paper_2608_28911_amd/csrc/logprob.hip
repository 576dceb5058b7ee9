// logprob.hip -- log probabilities of given tokens, entropies and the likeliest
// tokens of rows of logits on gfx950: the self-information indicator of
// Sec. 3.3 for the ranking (Eq. 4-5), and what a serving program returns.
//
// One pass over a row: each lane keeps its running maximum m and, relative to
// it, S = sum e^(x-m) and T = sum e^(x-m) (x-m) in fp32 (the entropy is
// ln S - T/S); the lanes' states join at the end.  Memory-bound: a logit is
// read once (4096 rows of 128000 fp16 logits 185 us, 5.7 TB/s; 4 rows, 15 workgroups
// each, with five alternatives 9.8 us and 4.4 for their merge, which latency
// bounds).  A workgroup of 4 waves takes a row, or a share of one where there are
// few.  The likeliest tokens are kept sorted across the lanes of a wave,
// as 64-bit keys of the logit's order and the complemented index; a vector of
// logits is looked at again only if its maximum beats the wave's last kept one,
// which happens k ln(n/k) times for n logits in random order.
#include "paged.h"
#include "tokens.h"

namespace semkv {
namespace {

constexpr int kTopMax = 32;

// Partial of one split of a row: m, S, T, then the kept keys.
__host__ __device__ constexpr int partial_words(int top) { return 4 + 2 * top; }

// A row's target and its logit.
struct Given { int64_t target; float x; };
__device__ inline Given given(const TokenArgs& a, int64_t row) {
  Given g = {-1, 0.0f};
  if (!a.logp) return g;
  const int b = int(row / a.T);
  const int64_t t = row - b * a.T;
  g.target = a.targets[b * a.t_batch + t * a.t_token];
  if (g.target >= 0 && g.target < a.vocab) {
    const char* p = static_cast<const char*>(a.x) + (b * a.s_batch + t * a.s_token) * (a.dtype == 2 ? 4 : 2);
    g.x = a.dtype == 2 ? load1<2>(p, g.target) : a.dtype == 1 ? load1<1>(p, g.target) : load1<0>(p, g.target);
  }
  return g;
}

__device__ inline void finish(const TokenArgs& a, int64_t row, const Given& g, const Sums& s) {
  const int b = int(row / a.T);
  const int64_t t = row - b * a.T, at = b * a.o_batch + t * a.o_token;
  const float ln = __builtin_logf(s.S);
  const bool fine = s.S > 0.0f && s.S < INFINITY;         // not NaN either
  if (a.entropy) a.entropy[at] = fine ? ln - s.T / s.S : NAN;
  if (a.logp) {
    const float v = g.target >= 0 && g.target < a.vocab && fine ? (g.x - s.m) - ln : NAN;
    a.logp[at] = g.target == -1 ? 0.0f : a.negate ? -v : v;
  }
}

__device__ inline void finish_top(const TokenArgs& a, int64_t row, const Sums& s, uint32_t h, uint32_t l, int i) {
  const bool fine = s.S > 0.0f && s.S < INFINITY;
  const int64_t at = row * a.top + i;
  a.top_logp[at] = fine ? (logit_of(h) - s.m) - __builtin_logf(s.S) : NAN;
  a.top_ids[at] = fine ? int32_t(~l) : -1;
}

template <int DT, int WAVES, bool TOP>
__global__ __launch_bounds__(64 * WAVES) void token_logprobs_kernel(TokenArgs a) {
  constexpr int V = Elem<DT>::vec, NT = 64 * WAVES, U = 4;
  __shared__ Sums sm[WAVES];
  __shared__ uint32_t sm_hi[WAVES * kTopMax], sm_lo[WAVES * kTopMax];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  const int b = int(row / a.T);
  const int64_t t = row - b * a.T;
  const char* x = static_cast<const char*>(a.x) + (b * a.s_batch + t * a.s_token) * Elem<DT>::size;
  // the split's elements [i0, i1): whole vectors between the row's 16-byte
  // boundaries, single elements at its two ends
  const int64_t off = (16 - (reinterpret_cast<uintptr_t>(x) & 15)) % 16 / Elem<DT>::size;
  const int64_t head = off < a.vocab ? off : a.vocab;
  const int64_t vecs = (a.vocab - head) / V;
  const int64_t v0 = vecs * blockIdx.y / a.nsplit, v1 = vecs * (blockIdx.y + 1) / a.nsplit;
  const uint4* xv = reinterpret_cast<const uint4*>(x + head * Elem<DT>::size);
  Sums s = {kFloor, 0.0f, 0.0f};
  Kept kept = {0u, 0u};
  const int k = a.top;
  uint32_t last = 0;                     // order of the wave's last kept key

  auto single = [&](int64_t i, bool valid) {
    const float e = valid ? load1<DT>(x, i) : -INFINITY;
    if (fmaxf(e, kFloor) > s.m) raise(s, fmaxf(e, kFloor));
    if (valid) add(s, e);
    if constexpr (TOP) {
      const uint32_t h = valid ? order_of(e) : 0u;
      keep_all(kept, valid, h, ~uint32_t(i), k, lane);
      last = __builtin_amdgcn_readlane(kept.hi, k - 1);
    }
  };
  // the ends, shorter than a vector: the first split takes the row's head
  // before and the last its tail after its vectors, so that a wave meets its
  // logits in ascending order (but for those of one vector instruction)
  if (blockIdx.y == 0 && wave == 0) single(lane, lane < head);

  for (int64_t v = v0 + tid - lane; v < v1; v += NT * U) {   // wave-uniform bound
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = v + lane + u * NT;
      if (at < v1) w[u] = xv[at];
    }
    float e[U][V], mx[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool valid = v + lane + u * NT < v1;
      unpack<DT>(w[u], e[u]);
      mx[u] = -INFINITY;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (!valid) e[u][i] = -INFINITY;
        mx[u] = fmaxf(mx[u], e[u][i]);
      }
      const float m = fmaxf(mx[u], s.m);
      if (m > s.m) raise(s, m);
#pragma unroll
      for (int i = 0; i < V; ++i) add(s, e[u][i]);
    }
    if constexpr (TOP) {
      // a row with a NaN is reported by its sum: what is kept of it does not matter
      uint32_t most = 0;
#pragma unroll
      for (int u = 0; u < U; ++u) most = max(most, v + lane + u * NT < v1 ? order_of(mx[u]) : 0u);
      if (__any(most > last)) {
        // while the list fills, the lanes' maxima bound what it can end with
        const uint32_t least = max(last, kth_order(most, k));
        const float bound = least > order_of(-INFINITY) ? logit_of(least) : -INFINITY;   // the same order, as a logit
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int64_t at = v + lane + u * NT;
          if (!__any(at < v1 && mx[u] >= bound)) continue;
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const bool may = at < v1 && e[u][i] >= bound;
            if (__any(may)) keep_all(kept, may, order_of(e[u][i]), ~uint32_t(head + at * V + i), k, lane);
          }
        }
        last = __builtin_amdgcn_readlane(kept.hi, k - 1);
      }
    }
  }

  const int64_t tail = head + vecs * V;
  if (blockIdx.y + 1 == a.nsplit && wave == 0) single(tail + lane, tail + lane < a.vocab);

  s = join_wave(s);
  if (lane == 0) sm[wave] = s;
  if (TOP && lane < k) {
    sm_hi[wave * k + lane] = kept.hi;
    sm_lo[wave * k + lane] = kept.lo;
  }
  __syncthreads();
  if (wave != 0) return;
  const Given g = a.nsplit == 1 ? given(a, row) : Given{-1, 0.0f};
  s = join_wave(lane < WAVES ? sm[lane] : Sums{kFloor, 0.0f, 0.0f});
  if constexpr (TOP) {
    for (int i = k; i < WAVES * k; i += 64) {              // the other waves' keys into wave 0's
      const bool valid = i + lane < WAVES * k;
      const uint32_t h = valid ? sm_hi[i + lane] : 0u, l = valid ? sm_lo[i + lane] : 0u;
      keep_all(kept, valid, h, l, k, lane);
    }
  }
  if (a.nsplit > 1) {
    uint32_t* p = reinterpret_cast<uint32_t*>(a.ws) + (row * a.nsplit + blockIdx.y) * partial_words(a.top);
    if (lane == 0) {
      p[0] = __float_as_uint(s.m);
      p[1] = __float_as_uint(s.S);
      p[2] = __float_as_uint(s.T);
    }
    if (TOP && lane < k) {
      p[4 + 2 * lane] = kept.hi;
      p[5 + 2 * lane] = kept.lo;
    }
    return;
  }
  if (lane == 0) finish(a, row, g, s);
  if (TOP && lane < k) finish_top(a, row, s, kept.hi, kept.lo, lane);
}

// The splits of a row joined, a wave each: everything it needs is loaded first.
__global__ __launch_bounds__(64) void token_merge_kernel(TokenArgs a) {
  const int lane = threadIdx.x, k = a.top;
  const int64_t row = blockIdx.x;
  const uint32_t* p = reinterpret_cast<const uint32_t*>(a.ws) + row * a.nsplit * partial_words(k);
  auto key = [&](int at, uint32_t& h, uint32_t& l) {
    const int sp = at / max(k, 1), j = at - sp * k;
    const bool valid = at < a.nsplit * k;
    const uint32_t* q = p + (valid ? sp * partial_words(k) + 4 + 2 * j : 0);
    h = q[0];
    l = q[1];
    if (!valid) h = l = 0;
  };
  uint32_t h, l;
  key(lane, h, l);
  const Given g = given(a, row);
  Sums s = {kFloor, 0.0f, 0.0f};
  for (int i = lane; i < a.nsplit; i += 64) {
    const uint32_t* q = p + i * partial_words(k);
    Sums t = {__uint_as_float(q[0]), __uint_as_float(q[1]), __uint_as_float(q[2])};
    const float m = fmaxf(s.m, t.m);
    raise(s, m);
    raise(t, m);
    s.S += t.S;
    s.T += t.T;
  }
  s = join_wave(s);
  if (lane == 0) finish(a, row, g, s);
  if (k == 0) return;
  Kept kept = {0u, 0u};
  const uint32_t least = kth_order(h, k);          // of the first 64 keys, which the rest cannot lower
  for (int i = 0; i < a.nsplit * k; i += 64) {
    if (i) key(i + lane, h, l);
    keep_all(kept, h != 0 && h >= least, h, l, k, lane);
  }
  if (lane < k) finish_top(a, row, s, kept.hi, kept.lo, lane);
}

// Splits of a row: enough workgroups for the chip where there are few rows,
// each with 8192 logits at least.
int splits(int64_t rows, int64_t vocab) {
  int64_t n = 512 / rows;
  if (n > vocab / 8192) n = vocab / 8192;
  return n < 1 ? 1 : int(n);
}

template <int DT, int WAVES>
void launch(const TokenArgs& a, dim3 grid, hipStream_t s) {
  if (a.top) hipLaunchKernelGGL((token_logprobs_kernel<DT, WAVES, true>), grid, dim3(64 * WAVES), 0, s, a);
  else hipLaunchKernelGGL((token_logprobs_kernel<DT, WAVES, false>), grid, dim3(64 * WAVES), 0, s, a);
}

}  // namespace

size_t token_logprobs_workspace(int64_t rows, int64_t vocab, int top) {
  const int n = splits(rows, vocab);
  return n < 2 ? 0 : size_t(rows) * n * partial_words(top) * 4;
}

int launch_token_logprobs(TokenArgs a, hipStream_t s) {
  const int64_t rows = int64_t(a.batch) * a.T;
  a.nsplit = splits(rows, a.vocab);
  const dim3 grid(unsigned(rows), unsigned(a.nsplit));
  if (a.dtype == 0) launch<0, 4>(a, grid, s);
  else if (a.dtype == 1) launch<1, 4>(a, grid, s);
  else launch<2, 4>(a, grid, s);
  if (a.nsplit > 1) hipLaunchKernelGGL(token_merge_kernel, dim3(unsigned(rows)), dim3(64), 0, s, a);
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

}  // namespace semkv
