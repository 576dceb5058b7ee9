// latent_attn.hip -- causal attention of every query head over one latent vector a
// token on gfx950: x = scale (q_h . c_t + qr_h . r_t), out = softmax(x) c.
//
// All heads of a token's row meet the same latents, so rows of (token, head) make
// the tiles of both products on v_mfma_f32_16x16x32: a workgroup takes 16 RT rows
// and a run of the sequence's pages, half a page (a unit of 32 tokens) at a time,
// which lies in LDS once for both:
//   scores  C[16 tokens][16 rows] = latents . q        a wave: 16 rows (RT = 4),
//                                                      or 16 of the tokens
//   values  C[16 channels][16 rows] = latents^T . p    a wave: a quarter of the
//                                                      channels, every row
// Scores, statistics and sums are fp32; the weights enter the second product in the
// latents' type (bf16 by 2^-8 of each at most, fp16 2^-11), relative to a running
// reference M of their row, which is moved only where a unit would pass it by 2^5;
// fp16 weights are 2^10 at the reference, so that they keep their bits down to 2^-24
// of it.
#include <hip/hip_fp16.h>

#include "paged.h"

namespace semkv {
namespace {

typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

constexpr int kUnit = 32;                  // tokens of a unit
constexpr int kSlots = 512, kMostSplits = 64, kLeast = 2;   // workgroups that units are shared out to, splits of a tile, units of a split
constexpr int kTileWords = 4;              // words of a tile's description
constexpr float kLag = 5.0f;
__host__ __device__ constexpr float head_of(bool bf) { return bf ? 0.0f : 10.0f; }

__host__ __device__ constexpr int partial_floats(int latent) { return latent + 4; }   // a row's sums, M and l

// The product of 32 channels or tokens.
template <int BF>
__device__ inline float4v mfma(const uint4& a, const uint4& b, float4v c) {
  if constexpr (BF)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8v, a), __builtin_bit_cast(bf8v, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8v, a), __builtin_bit_cast(half8v, b), c, 0, 0, 0);
}

__device__ inline uint32_t pack2(float x, float y, bool bf16) {
  if (!bf16) return uint32_t(__half_as_ushort(__float2half_rn(x))) | uint32_t(__half_as_ushort(__float2half_rn(y))) << 16;
  uint32_t b[2] = {__float_as_uint(x), __float_as_uint(y)};
#pragma unroll
  for (int e = 0; e < 2; ++e)
    b[e] = (b[e] & 0x7FFFFFFFu) > 0x7F800000u ? 0x7FC0u : (b[e] + 0x7FFFu + ((b[e] >> 16) & 1u)) >> 16;
  return b[0] | b[1] << 16;
}

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Over the four lanes of a row (16 apart).
template <class F>
__device__ inline float over_row(float x, F f) {
  const uint32_t u = __float_as_uint(x);
  const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t y = __float_as_uint(f(__uint_as_float(p[0]), __uint_as_float(p[1])));
  const auto q = __builtin_amdgcn_permlane32_swap(y, y, false, false);
  return f(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ inline float row_max(float x) { return over_row(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ inline float row_sum(float x) { return over_row(x, [](float a, float b) { return a + b; }); }

__device__ inline int wave_sum(int x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  return __builtin_amdgcn_readfirstlane(x);
}

// What a workgroup works on: a tile of a sequence's rows of (token, head), and a
// share of the units that it sees.
struct Tile {
  int seq, len, row0, count;         // sequence (-1: none), its tokens, its first row of the call, and rows
  int rows, first;                   // rows of (token, head), and the first of the tile's
  int seen, units;                   // tokens that the tile's last row sees, and their units
  int splits, split;                 // workgroups that share them, this one's place
  int slot, stride;                  // this workgroup's partial, and how far the tile's partials lie apart
  int tile, tiles;                   // number of the tile in the call; tiles of the call
};

// The units of a call are shared out by what the sequences really hold, so that
// no more workgroups are made than wanted (a.target; a partial each): a share is
// the call's tiles times units over the wanted workgroups, and grows until they
// suffice.  Where sequences pass 64, or that does not settle, so many are wanted
// less the tiles: each tile's last share is the only one that is not full.
// Consecutive shares of one split go to tiles of the same units: the workgroups
// of an XCD (every eighth) take consecutive ones, and find each other's units in
// its L2.
template <int ROWS>
__device__ inline Tile tile_of(const LatentAttnArgs& a, int block, int lane) {
  struct Share { int first, count, len, tiles, units; };
  auto share = [&](int s0, int& reached) {
    Share k;
    const SeqRows m = lane_rows(a.c, a.r, s0, lane, reached, k.len);
    k.first = m.first;
    k.count = m.count;
    k.tiles = int(uint32_t(m.count * a.n_heads + ROWS - 1) / uint32_t(ROWS));
    k.units = (k.len + kUnit - 1) / kUnit;
    return k;
  };
  int reached = 0;
  Share mine = share(0, reached);
  const int reached64 = reached;
  int64_t work = int64_t(mine.tiles) * mine.units;
  int tiles = mine.tiles;
  for (int s0 = 64; s0 < a.r.n_seqs; s0 += 64) {
    const Share k = share(s0, reached);
    work += int64_t(k.tiles) * k.units;
    tiles += k.tiles;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) work += __shfl_xor(work, d);
  tiles = wave_sum(tiles);
  const uint32_t wl = __builtin_amdgcn_readfirstlane(int(work)), wh = __builtin_amdgcn_readfirstlane(int(work >> 32));
  const bool far = wh || wl >> 31 || a.target <= tiles;        // many tiles: a workgroup each
  int chunk = INT32_MAX / 2;
  if (!far) {
    auto even = [&](int n) { return max(int((wl + uint32_t(n) - 1u) / uint32_t(n)), kLeast); };
    chunk = even(a.target);
    bool fits = false;
    if (a.r.n_seqs <= 64) {
#pragma unroll 1
      for (int tries = 0; tries < 4 && !fits; ++tries) {
        const int made = wave_sum(mine.tiles * min(int(uint32_t(mine.units + chunk - 1) / uint32_t(chunk)), kMostSplits));
        fits = made <= a.target;
        if (!fits) chunk = int(float(chunk) * float(made) / float(a.target)) + 1;
      }
    }
    if (!fits) chunk = even(a.target - tiles);
  }
  auto splits_of = [&](int units) { return max(min(int(uint32_t(units + chunk - 1) / uint32_t(chunk)), kMostSplits), 1); };
  int made = 0;
  for (int s0 = 0, r = 0; s0 < a.r.n_seqs; s0 += 64) {
    const Share k = s0 ? share(s0, r) : mine;
    if (!s0) r = reached64;
    made += wave_sum(k.tiles * splits_of(k.units));
  }
  const int per = (made + 7) / 8, flat = (block & 7) * per + (block >> 3);
  Tile k;
  k.seq = -1;
  k.tiles = tiles;
  if (block >> 3 >= per || flat >= made) return k;
  int before = 0, tbefore = 0;
  reached = reached64;
  for (int s0 = 0; s0 < a.r.n_seqs; s0 += 64) {
    if (s0) mine = share(s0, reached);
    const int splits = splits_of(mine.units), n = mine.tiles * splits;
    int incl = n, tincl = mine.tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int up = __shfl_up(incl, d), tup = __shfl_up(tincl, d);
      if (lane >= d) {
        incl += up;
        tincl += tup;
      }
    }
    const uint64_t above = __ballot(before + incl > flat);
    if (above) {
      const int l = __ffsll((unsigned long long)above) - 1;
      const int start = before + __builtin_amdgcn_readlane(incl - n, l), at = flat - start;
      const int own = __builtin_amdgcn_readlane(mine.tiles, l);
      k.splits = __builtin_amdgcn_readlane(splits, l);
      k.split = int(uint32_t(at) / uint32_t(own));
      const int t = at - k.split * own;
      k.seq = s0 + l;
      k.tile = tbefore + __builtin_amdgcn_readlane(tincl, l) - own + t;
      k.first = (own - 1 - t) * ROWS;                  // the last rows, which see the most, first
      k.row0 = __builtin_amdgcn_readlane(mine.first, l);
      k.count = __builtin_amdgcn_readlane(mine.count, l);
      k.len = __builtin_amdgcn_readlane(mine.len, l);
      k.slot = flat;
      k.stride = own;
      break;
    }
    before += __builtin_amdgcn_readlane(incl, 63);
    tbefore += __builtin_amdgcn_readlane(tincl, 63);
  }
  if (k.seq < 0) return k;
  k.rows = k.count * a.n_heads;
  const int last = int(uint32_t(min(k.first + ROWS, k.rows) - 1) / uint32_t(a.n_heads));      // row of the call
  k.seen = max(k.len - k.count + last + 1, 0);
  k.units = (k.seen + kUnit - 1) / kUnit;
  return k;
}

// Where 16 bytes (chunk) of a token's row lie in LDS: rotated within 256 bytes by
// the token, so that 16 tokens' same chunk, and the eight tokens whose 32 bytes a
// transposing read takes together, lie in different banks.
template <int L>
__device__ inline int latent_place(int t, int chunk) { return t * 2 * L + ((chunk ^ (t & 15)) << 4); }
template <int RP>
__device__ inline int rope_place(int t, int chunk) {
  return t * 2 * RP + ((chunk ^ (RP == 64 ? (t >> 1) & 7 : (t >> 2) & 3)) << 4);
}

// A unit's tokens in the order of the second product's operands: lane group g's
// elements e are tokens 8 g + 2 (e mod 4) + e div 4.
__device__ inline int token_of(int g, int e) { return 8 * g + 2 * (e & 3) + (e >> 2); }

template <int L, int RP, int BF, int RT>
__global__ __launch_bounds__(256, 1) void latent_attn_kernel(LatentAttnArgs a) {
  constexpr int ROWS = 16 * RT, KL = L / 32, KR = RP / 32, CT = L / 64, NQ = RT == 4 ? 2 : 1;   // NQ: token tiles of a wave's scores
  constexpr float HEAD = head_of(BF);
  __shared__ __align__(16) uint8_t sm_c[kUnit * L * 2];
  __shared__ __align__(16) uint8_t sm_r[kUnit * RP * 2];
  __shared__ __align__(16) uint4 sm_p[ROWS][4];
  __shared__ float sm_max[2][ROWS], sm_alpha[ROWS], sm_l[2][ROWS], sm_m[ROWS];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
  const PagedView& c = a.c;
  if (blockIdx.x == gridDim.x - 1)
    for (int s = tid; s < a.r.n_seqs; s += 256)
      if (starts_bad(a.r, s)) atomicOr(c.status, kBad);
  const Tile tl = tile_of<ROWS>(a, blockIdx.x, lane);
  int32_t* about = reinterpret_cast<int32_t*>(a.ws);      // of every tile: its first partial, how far they lie apart, their number
  if (a.target > 0 && tid == 0 && int(blockIdx.x) < a.target && int(blockIdx.x) >= tl.tiles) about[kTileWords * blockIdx.x + 2] = 0;
  if (tl.seq < 0) return;

  // rows of this wave's scores: tile wave mod RT; and its token tile
  const int rt0 = wave % RT, tt0 = RT == 4 ? 0 : wave / RT;
  const bool scores = RT == 4 || tt0 < 2;
  const int m0 = tl.len - tl.count;
  auto row_of = [&](int rt) { return min(tl.first + 16 * rt + n, tl.rows - 1); };
  uint4 q[KL + KR];
  int limit;                                              // the last token that the lane's row sees
  {
    const int row = row_of(rt0), i = int(uint32_t(row) / uint32_t(a.n_heads)), h = row - i * a.n_heads;
    const uint16_t* src = a.q + int64_t(tl.row0 + i) * a.qT + h * a.qH + 8 * g;
    const uint16_t* more = a.q_rope + int64_t(tl.row0 + i) * a.rT + h * a.rH + 8 * g;
#pragma unroll
    for (int k = 0; k < KL; ++k) q[k] = *reinterpret_cast<const uint4*>(src + 32 * k);
#pragma unroll
    for (int k = 0; k < KR; ++k) q[KL + k] = *reinterpret_cast<const uint4*>(more + 32 * k);
    limit = m0 + i;
  }
  const int all_see = m0 + int(uint32_t(tl.first) / uint32_t(a.n_heads));   // what the tile's first row sees, every row does
  const int u0 = int(int64_t(tl.units) * tl.split / tl.splits), u1 = int(int64_t(tl.units) * (tl.split + 1) / tl.splits);
  const int32_t* table = c.table + int64_t(tl.seq) * c.seq_pages;

  float4v o[RT][CT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int k = 0; k < CT; ++k) o[r][k] = float4v{0, 0, 0, 0};
  float M = -INFINITY, l = 0.0f;

#pragma unroll 1
  for (int u = u0; u < u1; ++u) {
    const int page = __builtin_amdgcn_readfirstlane(table[u >> 1]);
    if (page < 0) continue;                               // missing: not cached
    const uint16_t* rec = reinterpret_cast<const uint16_t*>(paged_record_at(c, page, a.layer, 0));
    const int t0 = (u & 1) * kUnit, most = min(tl.seen - 1 - u * kUnit, kUnit - 1);   // past the last token: the last again, with no weight
    __syncthreads();
    for (int i = tid; i < kUnit * L / 8; i += 256) {
      const int t = i / (L / 8), ch = i % (L / 8);
      *reinterpret_cast<uint4*>(sm_c + latent_place<L>(t, ch)) =
          reinterpret_cast<const uint4*>(rec + (t0 + min(t, most)) * L)[ch];
    }
    for (int i = tid; i < kUnit * RP / 8; i += 256) {
      const int t = i / (RP / 8), ch = i % (RP / 8);
      *reinterpret_cast<uint4*>(sm_r + rope_place<RP>(t, ch)) =
          reinterpret_cast<const uint4*>(rec + kPage * L + (t0 + min(t, most)) * RP)[ch];
    }
    __syncthreads();

    float4v x[NQ];
    float mx = -INFINITY;
    if (scores) {
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        const int t = 16 * (tt0 + j) + n;
        x[j] = float4v{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KL; ++k)
          x[j] = mfma<BF>(*reinterpret_cast<const uint4*>(sm_c + latent_place<L>(t, 4 * k + g)), q[k], x[j]);
#pragma unroll
        for (int k = 0; k < KR; ++k)
          x[j] = mfma<BF>(*reinterpret_cast<const uint4*>(sm_r + rope_place<RP>(t, 4 * k + g)), q[KL + k], x[j]);
        x[j] *= a.scale_log2e;
        if (u * kUnit + kUnit - 1 > all_see) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (u * kUnit + 16 * (tt0 + j) + 4 * g + e > limit) x[j][e] = -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, x[j][e]);
      }
      mx = row_max(mx);
    }
    if constexpr (RT < 4) {                               // two waves hold a row's tokens
      if (scores && g == 0) sm_max[tt0][16 * rt0 + n] = mx;
      __syncthreads();
      if (scores) mx = fmaxf(sm_max[0][16 * rt0 + n], sm_max[1][16 * rt0 + n]);
    }
    if (scores) {
      const float Mn = mx > M + kLag || M == -INFINITY ? fmaxf(mx, M) : M;
      const float alpha = M == -INFINITY || Mn == M ? 1.0f : exp2_fast(M - Mn);
      M = Mn;
      l *= alpha;
      const float ref = M == -INFINITY ? 0.0f : M - HEAD;
#pragma unroll
      for (int j = 0; j < NQ; ++j) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          p[e] = exp2_fast(x[j][e] - ref);
          l += p[e];
        }
        // tokens 16 (tt0 + j) + 4 g + e, in the order of token_of
        uint32_t* to = reinterpret_cast<uint32_t*>(&sm_p[16 * rt0 + n][2 * (tt0 + j) + (g >> 1)]);
        to[g & 1] = pack2(p[0], p[2], BF);
        to[2 + (g & 1)] = pack2(p[1], p[3], BF);
      }
      if (g == 0 && tt0 == 0) sm_alpha[16 * rt0 + n] = alpha;
    }
    __syncthreads();

    uint4 p[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      p[r] = sm_p[16 * r + n][g];
      const float alpha = sm_alpha[16 * r + n];
      if (__any(alpha != 1.0f)) {
#pragma unroll
        for (int k = 0; k < CT; ++k) o[r][k] *= alpha;
      }
    }
#pragma unroll
    for (int k = 0; k < CT; ++k) {
      const int ch = 16 * (wave * CT + k) + n;
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t lo = *reinterpret_cast<const uint16_t*>(sm_c + latent_place<L>(token_of(g, 2 * e), ch >> 3) + 2 * (ch & 7));
        const uint32_t hi = *reinterpret_cast<const uint16_t*>(sm_c + latent_place<L>(token_of(g, 2 * e + 1), ch >> 3) + 2 * (ch & 7));
        w[e] = lo | hi << 16;
      }
      const uint4 v = make_uint4(w[0], w[1], w[2], w[3]);
#pragma unroll
      for (int r = 0; r < RT; ++r) o[r][k] = mfma<BF>(v, p[r], o[r][k]);
    }
  }

  // the rows' statistics to every wave
  if (scores) {
    l = row_sum(l);
    if (g == 0) {
      sm_l[tt0][16 * rt0 + n] = l;
      if (tt0 == 0) sm_m[16 * rt0 + n] = M;
    }
  }
  __syncthreads();
  float* part = a.ws + kTileWords * kSlots + int64_t(tl.slot) * ROWS * partial_floats(L);
  if (tl.splits > 1 && tl.split == 0 && tid == 0) {
    about[kTileWords * tl.tile] = tl.slot;
    about[kTileWords * tl.tile + 1] = tl.stride;
    about[kTileWords * tl.tile + 2] = tl.splits;
    about[kTileWords * tl.tile + 3] = tl.row0 * a.n_heads + tl.first;
  }
  if (a.target > 0 && tl.splits == 1 && tid == 0) about[kTileWords * tl.tile + 2] = 0;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = tl.first + 16 * r + n;
    const float L0 = sm_l[0][16 * r + n] + (RT < 4 ? sm_l[1][16 * r + n] : 0.0f), Mr = sm_m[16 * r + n];
    if (tl.splits > 1) {
      float* to = part + (16 * r + n) * partial_floats(L);
#pragma unroll
      for (int k = 0; k < CT; ++k) *reinterpret_cast<float4v*>(to + 16 * (wave * CT + k) + 4 * g) = o[r][k];
      if (wave == 0 && g == 0) {
        to[L] = Mr;
        to[L + 1] = row < tl.rows ? L0 : 0.0f;
        to[L + 2] = row < tl.rows ? 1.0f : 0.0f;
      }
    } else if (row < tl.rows) {
      const int64_t at = int64_t(tl.row0) * a.n_heads + row;
      const float f = L0 == 0.0f ? 0.0f : 1.0f / L0;      // no token: zeros
#pragma unroll
      for (int k = 0; k < CT; ++k) {
        const float4v v = o[r][k] * f;
        *reinterpret_cast<uint2*>(a.out + at * L + 16 * (wave * CT + k) + 4 * g) = make_uint2(pack2(v[0], v[1], BF), pack2(v[2], v[3], BF));
      }
      if (a.lse && wave == 0 && g == 0) a.lse[at] = L0 == 0.0f ? -INFINITY : (Mr - HEAD + __builtin_log2f(L0)) * 0.69314718055994531f;
    }
  }
}

// The splits of a tile joined: a workgroup a row, a thread 4 channels.
template <int L, int BF>
__global__ __launch_bounds__(L / 4) void latent_join_kernel(LatentAttnArgs a, int rows) {
  constexpr float HEAD = head_of(BF);
  const int32_t* about = reinterpret_cast<const int32_t*>(a.ws) + kTileWords * blockIdx.x;
  const int splits = about[2];
  if (splits < 2) return;
  const int slot = about[0], stride = about[1], r = blockIdx.y, ch = 4 * threadIdx.x;
  const float* part = a.ws + kTileWords * kSlots + (int64_t(slot) * rows + r) * partial_floats(L);
  const int64_t step = int64_t(stride) * rows * partial_floats(L);
  if (part[L + 2] == 0.0f) return;                        // past the sequence's rows
  float M = -INFINITY;
  for (int s = 0; s < splits; ++s) M = fmaxf(M, part[s * step + L]);
  float sum = 0.0f;
  float4v v = float4v{0, 0, 0, 0};
  for (int s = 0; s < splits; ++s) {
    const float m = part[s * step + L], f = m == -INFINITY ? 1.0f : exp2_fast(m - M);   // nothing seen: zeros, or NaN
    sum = fmaf(part[s * step + L + 1], f, sum);
    v += *reinterpret_cast<const float4v*>(part + s * step + ch) * f;
  }
  const int64_t at = int64_t(about[3]) + r;
  v *= sum == 0.0f ? 0.0f : 1.0f / sum;
  *reinterpret_cast<uint2*>(a.out + at * L + ch) = make_uint2(pack2(v[0], v[1], BF), pack2(v[2], v[3], BF));
  if (a.lse && threadIdx.x == 0) a.lse[at] = sum == 0.0f ? -INFINITY : (M - HEAD + __builtin_log2f(sum)) * 0.69314718055994531f;
}

template <int L, int RP, int BF, int RT>
int launch(LatentAttnArgs a, hipStream_t s) {
  constexpr int ROWS = 16 * RT;
  // tiles of the call: a whole tile's rows each, and one more a sequence
  const int64_t whole = a.r.n_rows * ((a.n_heads + ROWS - 1) / ROWS);
  int64_t tiles = a.r.n_rows * a.n_heads / ROWS + a.r.n_seqs;
  if (tiles > whole) tiles = whole;
  if (tiles >= (int64_t(1) << 23)) return -2;      // a grid's threads are counted in 32 bits
  const bool split = tiles < kSlots;
  a.target = split ? kSlots : 0;
  const unsigned grid = split ? kSlots : unsigned((tiles + 7) / 8 * 8);
  hipLaunchKernelGGL((latent_attn_kernel<L, RP, BF, RT>), dim3(grid), dim3(256), 0, s, a);
  if (split) hipLaunchKernelGGL((latent_join_kernel<L, BF>), dim3(unsigned(tiles), ROWS), dim3(L / 4), 0, s, a, ROWS);
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

template <int L, int RP, int BF>
int launch_rows(const LatentAttnArgs& a, hipStream_t s) {
  const int64_t rows = (a.r.n_rows * a.n_heads + a.r.n_seqs - 1) / a.r.n_seqs;   // of a sequence, on average
  if (rows <= 16) return launch<L, RP, BF, 1>(a, s);
  if (rows <= 32) return launch<L, RP, BF, 2>(a, s);
  return launch<L, RP, BF, 4>(a, s);
}

template <int L, int RP>
int launch_type(const LatentAttnArgs& a, hipStream_t s) {
  return a.bf16 ? launch_rows<L, RP, 1>(a, s) : launch_rows<L, RP, 0>(a, s);
}

}  // namespace

// descriptions of the tiles, and kSlots partials of the widest tile
size_t latent_attn_workspace(int latent) { return size_t(kTileWords * kSlots + kSlots * 64 * partial_floats(latent)) * 4; }

int launch_latent_attn(LatentAttnArgs a, size_t ws_bytes, hipStream_t s) {
  if (ws_bytes < latent_attn_workspace(a.c.latent)) return -1;
  if (a.c.latent == 512) return a.c.rope == 64 ? launch_type<512, 64>(a, s) : launch_type<512, 32>(a, s);
  return a.c.rope == 64 ? launch_type<256, 64>(a, s) : launch_type<256, 32>(a, s);
}

}  // namespace semkv
