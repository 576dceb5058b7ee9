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
constexpr int kBufferWord3 = 0x00020000;   // raw buffer of 32-bit elements (gfx9 family)
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

// Two values rounded to the type (nearest, ties to even).
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
template <int BF>
__device__ inline uint32_t pack2(float x, float y) {
  if constexpr (BF) return __builtin_bit_cast(uint32_t, bf2v{__bf16(x), __bf16(y)});
  else return __builtin_bit_cast(uint32_t, half2v{_Float16(x), _Float16(y)});
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

// Over the wave, in every lane.
template <class F>
__device__ inline float over_wave(float x, F f) {
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) x = f(x, __shfl_xor(x, d));
  return over_row(x, f);
}

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

// The second product's operand of latents has channels along lanes and tokens in a
// lane: 16 lanes read 8 bytes each, four tokens' 16 channels, and get them turned
// (lane i: channel i of the four tokens).  Lane group g's elements are tokens
// 8 g + 2 j, then 8 g + 2 j + 1.
typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v lds_short4v;
__device__ inline uint2 turned4(const uint8_t* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v*)p));
}

// The workgroup's LDS: two units' latents and key parts, each an array of its own, so
// that reads of one do not wait for the loads of the other.
typedef __attribute__((address_space(3))) void lds_void;

// A store to LDS while loads into it are under way, for which the compiler would
// have it wait; they go elsewhere.  Counted by meet().
__device__ inline void put_lds(void* p, uint32_t v) {
  __asm__ volatile("ds_write_b32 %0, %1" : : "v"(uint32_t(uintptr_t((lds_void*)p))), "v"(v) : "memory");
}
__device__ inline void put_lds(void* p, float v) { put_lds(p, __float_as_uint(v)); }

// Earlier LDS accesses before later ones of the other waves.  Loads into LDS that are
// under way stay so (a fence would wait for them).
__device__ inline void meet() { __asm__ volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }
// The same, this wave's loads into LDS among what comes before.
__device__ inline void meet_loaded() { __asm__ volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

// A lane's number that the compiler works out anew where it is used: places made
// from it are not kept in registers over the loop, where they would be spilled.
__device__ inline int anew(int x) {
  __asm__ volatile("" : "+v"(x));
  return x;
}

// A unit from its record straight into LDS, 1 KB a wave's load.  Lane i's 16 bytes
// go to chunk i of the 64 chunks; from which chunk it takes them makes the places above.
template <int L, int RP>
__device__ __forceinline__ void load_unit(const PagedView& c, int layer, int page, int half, int most, int wave, int lane, uint8_t* sm_c,
                                          uint8_t* sm_r) {
  constexpr int PER = 512 / L, N = kUnit / (4 * PER);      // tokens of a load, loads of a wave
  const uint8_t* rec = paged_record_at(c, page, layer, 0);
  const auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(rec), 0, 2 * kPage * (L + RP), kBufferWord3);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int t = (4 * i + wave) * PER + (PER > 1 ? lane >> 5 : 0), ch = lane & (L / 8 - 1);
    const int from = (half * kUnit + min(t, most)) * 2 * L, at = (ch ^ (t & 15)) << 4;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(sm_c + (4 * i + wave) * 1024), 16, PER > 1 ? from + at : at,
                                             PER > 1 ? 0 : __builtin_amdgcn_readfirstlane(from), 0, 0);
  }
  if (wave * 1024 < kUnit * RP * 2) {
    constexpr int CH = RP / 8;
    const int t = wave * (64 / CH) + lane / CH, ch = lane & (CH - 1);
    const int at = (half * kUnit + min(t, most)) * 2 * RP + ((ch ^ (RP == 64 ? (t >> 1) & 7 : (t >> 2) & 3)) << 4);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(sm_r + wave * 1024), 16, at, 2 * kPage * L, 0, 0);
  }
}

template <int L, int RP, int BF, int RT>
__global__ __launch_bounds__(256, 2) void latent_attn_kernel(LatentAttnArgs a) {
  constexpr int ROWS = 16 * RT, KL = L / 32, KR = RP / 32, CT = L / 64, NQ = RT == 4 ? 2 : 1;   // NQ: token tiles of a wave's scores
  constexpr float HEAD = head_of(BF);
  __shared__ __align__(1024) uint8_t sm_c0[kUnit * L * 2], sm_c1[kUnit * L * 2];
  __shared__ __align__(1024) uint8_t sm_r0[kUnit * RP * 2], sm_r1[kUnit * RP * 2];
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
  const int u1 = int(int64_t(tl.units) * (tl.split + 1) / tl.splits);
  // (no kernel writes the table while this one runs: scalar loads)
  typedef const __attribute__((address_space(4))) int32_t* scalar_words;
  const scalar_words table = scalar_words(uintptr_t(c.table + int64_t(tl.seq) * c.seq_pages));
  int page = -1;
  auto find = [&](int u) {                                // the next unit whose page is there
    for (; u < u1; ++u) {
      page = table[u >> 1];
      if (page >= 0) break;
    }
    return u;
  };
  // past the last token that the tile sees: that one again, with no weight
  auto load = [&](int u, uint8_t* sm_c, uint8_t* sm_r) {
    load_unit<L, RP>(c, a.layer, page, u & 1, min(tl.seen - 1 - u * kUnit, kUnit - 1), wave, anew(lane), sm_c, sm_r);
  };
  int u = find(int(int64_t(tl.units) * tl.split / tl.splits));
  if (u < u1) load(u, sm_c0, sm_r0);
  int next = find(u + 1);                                 // the unit after u, and in `page` its page

  uint4 q[KL + KR];
  int limit;                                              // the last token that the lane's row sees
  {
    const int row = min(tl.first + 16 * rt0 + n, tl.rows - 1), i = int(uint32_t(row) / uint32_t(a.n_heads)), h = row - i * a.n_heads;
    const uint16_t* src = a.q + int64_t(tl.row0 + i) * a.qT + h * a.qH + 8 * g;
    const uint16_t* more = a.q_rope + int64_t(tl.row0 + i) * a.rT + h * a.rH + 8 * g;
#pragma unroll
    for (int k = 0; k < KL; ++k) q[k] = *reinterpret_cast<const uint4*>(src + 32 * k);
#pragma unroll
    for (int k = 0; k < KR; ++k) q[KL + k] = *reinterpret_cast<const uint4*>(more + 32 * k);
    limit = m0 + i;
  }
  const int all_see = m0 + int(uint32_t(tl.first) / uint32_t(a.n_heads));   // what the tile's first row sees, every row does

  float4v o[RT][CT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int k = 0; k < CT; ++k) o[r][k] = float4v{0, 0, 0, 0};
  float M = -INFINITY, l = 0.0f;
  // places that the lane reads: of its token's chunks g, g + 4, ... (every fourth
  // lies 256 bytes on), and of the channels that transposing reads take
  const int vt = 8 * g + 2 * (n >> 2), vs = ((n >> 1) & 1) ^ (vt & 15);
  const int qat = latent_place<L>(n, g), vat = vt * 2 * L + (((2 * CT * wave) ^ vs) << 4) + 8 * (n & 1);

  auto step = [&](const uint8_t* sm_c, const uint8_t* sm_r, uint8_t* next_c, uint8_t* next_r) __attribute__((always_inline)) {
    meet_loaded();
    const int at = u;
    u = next;
    if (u < u1) load(u, next_c, next_r);
    const int after = table[min(u + 1, u1 - 1) >> 1];

    float4v x[NQ];
    float mx = -INFINITY;
    if (scores) {
      const int qp = anew(qat), tile = 16 * tt0;
#pragma unroll
      for (int j = 0; j < NQ; ++j) x[j] = float4v{0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < KL; ++k)
#pragma unroll
        for (int j = 0; j < NQ; ++j)
          x[j] = mfma<BF>(*reinterpret_cast<const uint4*>(sm_c + (qp ^ (k & 3) << 6) + (k >> 2) * 256 + (tile + 16 * j) * 2 * L), q[k], x[j]);
#pragma unroll
      for (int k = 0; k < KR; ++k)
#pragma unroll
        for (int j = 0; j < NQ; ++j)
          x[j] = mfma<BF>(*reinterpret_cast<const uint4*>(sm_r + rope_place<RP>(tile + 16 * j + n, 4 * k + g)), q[KL + k], x[j]);
      // reads a few products ahead
      constexpr int AHEAD = 4 / NQ;
      __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * NQ, 0);
#pragma unroll
      for (int k = 0; k < KL + KR - AHEAD; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, NQ, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, NQ, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, AHEAD * NQ, 0);
#pragma unroll
      for (int j = 0; j < NQ; ++j) x[j] *= a.scale_log2e;
      if (at * kUnit + kUnit - 1 > all_see) {
#pragma unroll
        for (int j = 0; j < NQ; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (at * kUnit + tile + 16 * j + 4 * g + e > limit) x[j][e] = -INFINITY;
      }
#pragma unroll
      for (int j = 0; j < NQ; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, x[j][e]);
      mx = row_max(mx);
    }
    if constexpr (RT < 4) {                               // two waves hold a row's tokens
      if (scores && g == 0) put_lds(&sm_max[tt0][16 * rt0 + n], mx);
      meet();
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
        // tokens 16 (tt0 + j) + 4 g + e, in the order of turned4
        uint32_t* to = reinterpret_cast<uint32_t*>(&sm_p[16 * rt0 + n][2 * (tt0 + j) + (g >> 1)]);
        put_lds(to + (g & 1), pack2<BF>(p[0], p[2]));
        put_lds(to + 2 + (g & 1), pack2<BF>(p[1], p[3]));
      }
      if (g == 0 && tt0 == 0) put_lds(&sm_alpha[16 * rt0 + n], alpha);
    }
    meet();
    page = after;
    next = u + 1;
    if (page < 0) next = find(u + 1);

    uint4 p[RT];
    float alpha[RT];
    bool moved = false;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      p[r] = sm_p[16 * r + n][g];
      alpha[r] = sm_alpha[16 * r + n];
      moved = moved || alpha[r] != 1.0f;
    }
    if (__any(moved)) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int k = 0; k < CT; ++k) o[r][k] *= alpha[r];
    }
    const int vp = anew(vat);
#pragma unroll
    for (int k = 0; k < CT; ++k) {
      const uint2 lo = turned4(sm_c + (vp ^ k << 5)), hi = turned4(sm_c + (vp ^ (k << 5 | 16)) + 2 * L);
      const uint4 v = make_uint4(lo.x, lo.y, hi.x, hi.y);
#pragma unroll
      for (int r = 0; r < RT; ++r) o[r][k] = mfma<BF>(v, p[r], o[r][k]);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int k = 0; k < CT - 2; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x008, RT, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 2 * RT, 0);
  };
#pragma unroll 1
  while (u < u1) {
    step(sm_c0, sm_r0, sm_c1, sm_r1);
    if (u >= u1) break;
    step(sm_c1, sm_r1, sm_c0, sm_r0);
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
        *reinterpret_cast<uint2*>(a.out + at * L + 16 * (wave * CT + k) + 4 * g) = make_uint2(pack2<BF>(v[0], v[1]), pack2<BF>(v[2], v[3]));
      }
      if (a.lse && wave == 0 && g == 0) a.lse[at] = L0 == 0.0f ? -INFINITY : (Mr - HEAD + __builtin_log2f(L0)) * 0.69314718055994531f;
    }
  }
}

// The splits of a tile joined: a workgroup a row.  A lane takes a split's M and sum,
// so that their weights are there after one round trip; then the threads of a group
// (4 channels each) take every GROUPS-th split, B of them in flight.  (With a loop over
// splits that waits for each, 35 us instead of 8 for 115 rows of four sequences in 64 splits.)
template <int L, int BF>
__global__ __launch_bounds__(256) void latent_join_kernel(LatentAttnArgs a, int rows) {
  constexpr float HEAD = head_of(BF);
  constexpr int LPR = L / 4, GROUPS = 256 / LPR, B = 8;
  __shared__ float sm_f[kMostSplits];
  __shared__ __align__(16) float4v sm_v[GROUPS - 1][LPR];
  const int32_t* about = reinterpret_cast<const int32_t*>(a.ws) + kTileWords * blockIdx.x;
  const int splits = about[2];
  if (splits < 2) return;
  const int tid = threadIdx.x, lane = tid & 63, r = blockIdx.y;
  const int64_t step = int64_t(about[1]) * rows * partial_floats(L);
  const float* part = a.ws + kTileWords * kSlots + (int64_t(about[0]) * rows + r) * partial_floats(L);
  const float* mine = part + min(lane, splits - 1) * step + L;
  const float m = mine[0], l = lane < splits ? mine[1] : 0.0f;
  if (mine[2] == 0.0f) return;                            // past the sequence's rows
  const float M = over_wave(lane < splits ? m : -INFINITY, [](float x, float y) { return fmaxf(x, y); });
  const float f = m == -INFINITY ? 1.0f : exp2_fast(m - M);    // nothing seen: zeros, or NaN
  const float sum = over_wave(l * f, [](float x, float y) { return x + y; });
  if (tid < kMostSplits) sm_f[lane] = lane < splits ? f : 0.0f;
  __syncthreads();
  const int group = tid / LPR, ch = 4 * (tid % LPR);
  float4v v = float4v{0, 0, 0, 0};
  for (int s0 = group; s0 < splits; s0 += GROUPS * B) {
    float4v x[B];
#pragma unroll
    for (int k = 0; k < B; ++k) x[k] = *reinterpret_cast<const float4v*>(part + min(s0 + k * GROUPS, splits - 1) * step + ch);
#pragma unroll
    for (int k = 0; k < B; ++k)
      if (s0 + k * GROUPS < splits) v += x[k] * sm_f[s0 + k * GROUPS];
  }
  if (group > 0) sm_v[group - 1][tid % LPR] = v;
  __syncthreads();
  if (group > 0) return;
#pragma unroll
  for (int k = 0; k < GROUPS - 1; ++k) v += sm_v[k][tid];
  const int64_t at = int64_t(about[3]) + r;
  v *= sum == 0.0f ? 0.0f : 1.0f / sum;
  *reinterpret_cast<uint2*>(a.out + at * L + ch) = make_uint2(pack2<BF>(v[0], v[1]), pack2<BF>(v[2], v[3]));
  if (a.lse && tid == 0) a.lse[at] = sum == 0.0f ? -INFINITY : (M - HEAD + __builtin_log2f(sum)) * 0.69314718055994531f;
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
  if (split) hipLaunchKernelGGL((latent_join_kernel<L, BF>), dim3(unsigned(tiles), ROWS), dim3(256), 0, s, a, ROWS);
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
