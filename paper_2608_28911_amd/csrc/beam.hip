// beam.hip -- beam search's choice on gfx950: of a group's beams b with scores a_b
// and logits x_b, the k candidates (b, v) of the largest
//   t(b, v) = a_b + x_b[v] - ln sum_u exp x_b[u],
// equal ones by lower (b, v).
//
// Within a row t follows x, so one pass over the logits keeps a row's k largest by
// (x, v) and its sum of exponentials, and candidates of different rows meet only
// afterwards, k of each.  There the order can hang on the last place: rows' sums
// are joined, their logarithm is taken and t is worked out in 64 bits (a lane's
// own sums are fp32, a vector of logits at a time: 2e-8 of ln sum in all).
#include "paged.h"
#include "tokens.h"

namespace semkv {
namespace {

constexpr int kMostKept = 64, kMostBeams = 64;   // candidates of a group, its beams

// Partial of one split of a row: m and pad, S (64 bits), then the kept keys.
__host__ __device__ constexpr int partial_words(int k) { return 4 + 2 * k; }

struct Row { float m, S; };                       // a lane's maximum, and sum e^(x-m)

__device__ inline void raise(Row& a, float m) {   // m >= a.m
  a.S *= exp_of(a.m - m);
  a.m = m;
}

// A beam that has candidates of its own row.
__device__ inline bool reads_row(const BeamArgs& a, int64_t row) {
  return a.scores[row] != -INFINITY && !(a.ended && a.ended[row]);
}

// 16 bytes from an element's address (global loads need no more on gfx950).
template <int DT>
__device__ inline uint4 load_anywhere(const char* p) {
  uint4 v;
  __builtin_memcpy(&v, __builtin_assume_aligned(p, Elem<DT>::size), 16);
  return v;
}

// One workgroup takes a row, or a share of one where there are few.
template <int DT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void beam_rows_kernel(BeamArgs a) {
  constexpr int V = Elem<DT>::vec, NT = 64 * WAVES, U = 4;
  __shared__ Row sm[WAVES];
  __shared__ uint32_t sm_hi[WAVES * kMostKept], sm_lo[WAVES * kMostKept];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = blockIdx.x;
  if (!reads_row(a, row)) return;
  const int64_t g = row / a.width;
  const char* x = static_cast<const char*>(a.x) + (g * a.s_group + (row - g * a.width) * a.s_beam) * Elem<DT>::size;
  // vectors from the row's first element on, wherever that lies: rows of the same
  // logits have the same sum to the last bit, and their candidates stay equal
  const int64_t vecs = a.vocab / V;
  const int64_t v0 = vecs * blockIdx.y / a.nsplit, v1 = vecs * (blockIdx.y + 1) / a.nsplit;
  Row s = {kFloor, 0.0f};
  Kept kept = {0u, 0u};
  const int k = a.k;
  uint32_t last = 0;                     // order of the wave's last kept key

  auto single = [&](int64_t i, bool valid) {
    const float e = valid ? load1<DT>(x, i) : -INFINITY;
    if (e > s.m) raise(s, e);
    s.S += valid ? exp_of(e - s.m) : 0.0f;
    keep_all(kept, valid, valid ? order_of(e) : 0u, ~uint32_t(i), k, lane);
    last = __builtin_amdgcn_readlane(kept.hi, k - 1);
  };
  for (int64_t v = v0 + tid - lane; v < v1; v += NT * U) {   // wave-uniform bound
    uint4 w[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = v + lane + u * NT;
      if (at < v1) w[u] = load_anywhere<DT>(x + 16 * at);
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
      if (mx[u] > s.m) raise(s, mx[u]);
      float p[V];
#pragma unroll
      for (int i = 0; i < V; ++i) p[i] = exp_of(e[u][i] - s.m);
#pragma unroll
      for (int d = V / 2; d > 0; d /= 2)
#pragma unroll
        for (int i = 0; i < d; ++i) p[i] += p[i + d];
      s.S += p[0];
    }
    uint32_t most = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) most = max(most, v + lane + u * NT < v1 ? order_of(mx[u]) : 0u);
    if (__any(most > last)) {
      // while the list fills, the lanes' maxima bound what it can end with
      const uint32_t least = max(last, kth_order(most, k));
      const float bound = least > order_of(-INFINITY) ? logit_of(least) : -INFINITY;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t at = v + lane + u * NT;
        if (!__any(at < v1 && mx[u] >= bound)) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const bool may = at < v1 && e[u][i] >= bound;
          if (__any(may)) keep_all(kept, may, order_of(e[u][i]), ~uint32_t(at * V + i), k, lane);
        }
      }
      last = __builtin_amdgcn_readlane(kept.hi, k - 1);
    }
  }

  const int64_t tail = vecs * V;
  if (blockIdx.y + 1 == a.nsplit && wave == 0) single(tail + lane, tail + lane < a.vocab);

  // the lanes' sums relative to the wave's maximum
  auto add = [](float p, float q) { return p + q; };
  raise(s, over_wave(s.m, [](float p, float q) { return fmaxf(p, q); }));
  s.S = over_wave(s.S, add);
  if (lane == 0) sm[wave] = s;
  if (lane < k) {
    sm_hi[wave * k + lane] = kept.hi;
    sm_lo[wave * k + lane] = kept.lo;
  }
  __syncthreads();
  if (wave != 0) return;
  for (int i = k; i < WAVES * k; i += 64) {                // the other waves' keys into wave 0's
    const bool valid = i + lane < WAVES * k;
    const uint32_t h = valid ? sm_hi[i + lane] : 0u, l = valid ? sm_lo[i + lane] : 0u;
    keep_all(kept, valid, h, l, k, lane);
  }
  uint32_t* p = reinterpret_cast<uint32_t*>(a.ws) + (row * a.nsplit + blockIdx.y) * partial_words(k);
  if (lane == 0) {
    float m = sm[0].m;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m = fmaxf(m, sm[w].m);
    double S = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) S += double(sm[w].S) * double(exp_of(sm[w].m - m));
    p[0] = __float_as_uint(m);
    *reinterpret_cast<double*>(p + 2) = S;
  }
  if (lane < k) {
    p[4 + 2 * lane] = kept.hi;
    p[5 + 2 * lane] = kept.lo;
  }
}

// One workgroup chooses a group's candidates: its waves join the rows' splits,
// a row at a time each, and every kept candidate counts those before it in each
// row's list, which is in order: its place.
__global__ __launch_bounds__(256) void beam_choose_kernel(BeamArgs a) {
  __shared__ double sm_t[kMostBeams * kMostKept];
  __shared__ int32_t sm_v[kMostBeams * kMostKept];
  __shared__ int sm_bad, sm_n;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, k = a.k;
  const int64_t g = blockIdx.x;
  if (tid == 0) sm_bad = sm_n = 0;
  __syncthreads();
  for (int b = wave; b < a.width; b += 4) {
    const int64_t row = g * a.width + b;
    const float score = a.scores[row];
    double t = -INFINITY;
    int32_t v = 0;
    bool bad = !(score < INFINITY);
    if (a.ended && a.ended[row]) {
      if (lane == 0) t = double(score);
      v = a.pad;
    } else if (score != -INFINITY) {
      const uint32_t* p = reinterpret_cast<const uint32_t*>(a.ws) + row * a.nsplit * partial_words(k);
      auto key = [&](int at, uint32_t& h, uint32_t& l) {
        const int sp = at / k, j = at - sp * k;
        const bool valid = at < a.nsplit * k;
        const uint32_t* q = p + (valid ? sp * partial_words(k) + 4 + 2 * j : 0);
        h = q[0];
        l = q[1];
        if (!valid) h = l = 0;
      };
      uint32_t h, l;
      key(lane, h, l);
      float m = kFloor;
      for (int i = lane; i < a.nsplit; i += 64) m = fmaxf(m, __uint_as_float(p[i * partial_words(k)]));
      m = over_wave(m, [](float x, float y) { return fmaxf(x, y); });
      double S = 0.0;
      for (int i = lane; i < a.nsplit; i += 64) {
        const uint32_t* q = p + i * partial_words(k);
        S += *reinterpret_cast<const double*>(q + 2) * double(exp_of(__uint_as_float(q[0]) - m));
      }
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) S += __shfl_xor(S, d);
      Kept kept = {0u, 0u};
      const uint32_t least = kth_order(h, k);        // of the first 64 keys, which the rest cannot lower
      for (int i = 0; i < a.nsplit * k; i += 64) {
        if (i) key(i + lane, h, l);
        keep_all(kept, h != 0 && h >= least, h, l, k, lane);
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
  for (int i = n + tid; i < k; i += 256) {           // fewer candidates than wanted
    a.out_scores[g * k + i] = bad ? NAN : -INFINITY;
    a.parents[g * k + i] = -1;
    a.tokens[g * k + i] = -1;
  }
  if (bad) return;
  for (int i = tid; i < a.width * k; i += 256) {
    const double t = sm_t[i];
    if (!(t > -INFINITY)) continue;
    const int mine = i / k;
    int place = i - mine * k;                        // what is before it in its own list
    for (int b = 0; b < a.width && place < k; ++b) {
      if (b == mine) continue;
      int lo = 0, hi = k;                            // entries before: larger, or equal and of a lower beam
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        const double u = sm_t[b * k + mid];
        if (u > t || (u == t && b < mine)) lo = mid + 1;
        else hi = mid;
      }
      place += lo;
    }
    if (place >= k) continue;
    a.out_scores[g * k + place] = float(t);
    a.parents[g * k + place] = int32_t(g * a.width + mine);
    a.tokens[g * k + place] = sm_v[i];
  }
}

// Splits of a row: enough workgroups for the chip where there are few rows,
// each with 8192 logits at least.
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
  hipLaunchKernelGGL(beam_choose_kernel, dim3(unsigned(a.groups)), dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

}  // namespace semkv
