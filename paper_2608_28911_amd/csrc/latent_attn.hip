// latent_attn.hip -- causal attention of every query head over one latent vector a
// token on gfx950: x = scale (q_h . c_t + qr_h . r_t), out = softmax(x) c.
//
// All heads of a token's row meet the same latents, so rows of (token, head) make
// the tiles of both products on v_mfma_f32_16x16x32: a workgroup takes 16 RT rows
// and a run of the sequence's pages, half a page (a unit of 32 tokens) at a time,
// which lies in LDS once for both:
//   scores  C[16 tokens][16 rows] = latents . q        a wave has 16 rows (64 rows);
//                                                      16 rows and 16 tokens (32);
//                                                      16 tokens, half the channels (16)
//   values  C[16 channels][16 rows] = latents^T . p    a wave has a quarter of the
//                                                      channels, and every row
// With 64 rows a wave works out its rows' weights, which cross through LDS.  With
// fewer the scores do, and every wave works out all weights: its lanes then hold them
// in the second product's layout, and there is one wait less between the products (one
// token of 16 heads over 2048: 11.9 us with weights through LDS, 10.8 so; over 32768
// 21.2 and 19.4; with halves of the channels for 32 rows too, LDS holds one workgroup
// a CU, and 16 sequences of 16384 tokens with 32 heads take 82 us, not 72).
// Scores, statistics and sums are fp32; the weights enter the second product in the
// latents' type (bf16 by 2^-8 of each at most, fp16 2^-11), relative to a running
// reference M of their row, which is moved only where a unit would pass it by 2^5;
// fp16 weights are 2^10 at the reference, so that they keep their bits down to 2^-24
// of it.
//
// 512 tokens of 16 heads over 16384 take 281 us (1.06 PFLOP/s): LDS is busy 43 % of
// the time by address and some 20 more under loads, beside matrix cores at 51 %.  16
// single tokens over up to 16384 read at 4.2 TB/s (55 us a call, on states in turn).
// 128 heads of 8 sequences over 16384, 64 us, and five tokens of 4 over 32768, 41, have
// 20 us that do not grow with the tokens: the splits' partials go to memory and back
// (59 and 30 MB), and a launch joins them.
#include <hip/hip_fp16.h>

#include <type_traits>

#include "paged.h"

namespace semkv {
namespace {

typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

constexpr int kUnit = 32;                  // tokens of a unit
constexpr int kBlock = 1024 + 32;          // bytes of LDS for 1 KB of latents
// workgroups that units are shared out to, splits of a tile (one token of 16 heads over
// 131072 so reads at 3.7 TB/s), units of a split
constexpr int kSlots = 512, kMostSplits = 128, kLeast = 2;
constexpr int kTileWords = 4;              // words of a tile's description
constexpr int kBufferWord3 = 0x00020000;   // raw buffer of 32-bit elements (gfx9 family)
constexpr float kLag = 5.0f;
__host__ __device__ constexpr float head_of(bool bf) { return bf ? 0.0f : 10.0f; }

// A partial: sums as the lanes of the second product hold them, [row tile][16
// channels][lane][4], so that their stores and the join's loads are of 1 KB in a row (by
// rows 2 us more for 59 MB); then M, sum and whether it is one, of each row.
__host__ __device__ constexpr int partial_floats(int latent) { return latent + 4; }   // of a row

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

// Sums of the lanes up to each one, by DPP moves: within rows of 16 lanes, then each
// row's last sum into the next rows.
__device__ inline int scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);     // lane - 1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);     // lane - 2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);     // lane - 4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);     // lane - 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);    // lane 15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);    // lane 31 into rows 2 and 3
  return x;
}
__device__ inline int wave_sum(int x) { return __builtin_amdgcn_readlane(scan(x), 63); }

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
// the call's tiles times units over the wanted workgroups, at least what makes a
// split worth its joining, and grows until they suffice.  Where sequences pass 64, or
// that does not settle, so many are wanted less the tiles: each tile's last share is
// the only one that is not full.
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
  // (below 2^30 where it is used: fewer than kSlots tiles of 2^21 units at most)
  uint32_t work = uint32_t(mine.tiles) * uint32_t(mine.units);
  int tiles = mine.tiles;
  for (int s0 = 64; s0 < a.r.n_seqs; s0 += 64) {
    const Share k = share(s0, reached);
    work += uint32_t(k.tiles) * uint32_t(k.units);
    tiles += k.tiles;
  }
  work = uint32_t(wave_sum(int(work)));
  tiles = wave_sum(tiles);
  int chunk = INT32_MAX / 2;                                   // many tiles: a workgroup each
  // (a tile that sees nothing has a workgroup too, for its zeros)
  auto splits_of = [&](int units) { return max(min(int(uint32_t(units + chunk - 1) / uint32_t(chunk)), kMostSplits), 1); };
  if (tiles < a.target) {
    // A split costs its partial's way to memory and back (64 rows of 512 channels 50 ns
    // beside all others', 16 rows 13) where a unit takes a workgroup 2 us: of units u a
    // split and W in all, u 2 us + W/u 50 ns is least at u^2 = W 50 ns / 2 us.  (8
    // sequences of 2048 tokens with 128 heads 36 us without this, 29; 16 with 16 heads
    // 22 and 18.)
    const int least = max(kLeast, int(__builtin_sqrtf(float(work) * (ROWS == 64 ? 0.04f : 0.02f))));
    auto even = [&](int n) { return max(int((work + uint32_t(n) - 1u) / uint32_t(n)), least); };
    chunk = even(a.target);
    bool fits = false;
    if (a.r.n_seqs <= 64) {
#pragma unroll 1
      for (int tries = 0; tries < 4 && !fits; ++tries) {
        const int made = wave_sum(mine.tiles * splits_of(mine.units));
        fits = made <= a.target;
        if (!fits) chunk = int(float(chunk) * float(made) / float(a.target)) + 1;
      }
    }
    if (!fits) chunk = even(a.target - tiles);
  }
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
    const int incl = scan(n), tincl = scan(mine.tiles);
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

// Where 16 bytes (chunk) of a token's row lie in LDS.  Latents: in blocks of 1 KB, as a
// load leaves them (a token of 512, two of 256), a block 32 bytes further round the
// banks than the one before; of two tokens in a block the second's chunks have bit 3
// changed.  So the 16 lanes that a 16-byte read takes at once (0 to 3, 12 to 15, 20 to
// 27 of each half wave, and the rest: eight tokens' chunk c, eight others' c + 1), and
// the 32 that a transposing read does (eight tokens in a row, 32 bytes each), read
// different banks, and channels further on are a constant further on.  (With blocks
// 16 bytes apart the reads conflict: 53 million cycles of it in a chunk of 512 tokens,
// 6 as it is.)  Key
// parts: rotated by the token.
template <int L>
__host__ __device__ constexpr int latents_bytes() { return kUnit * L / 512 * kBlock; }
template <int L>
__device__ inline int latent_place(int t, int chunk) {
  if constexpr (L == 512) return t * kBlock + (chunk << 4);
  else return (t >> 1) * kBlock + (t & 1) * 512 + ((chunk ^ (t & 1) << 3) << 4);
}
template <int RP>
__device__ inline int rope_place(int t, int chunk) {
  return t * 2 * RP + ((chunk ^ (RP == 64 ? (t >> 1) & 7 : (t >> 2) & 3)) << 4);
}

// The same for a row's weights, 16 bytes for each lane group: 5 % of a chunk's time.
__device__ inline int weights_place(int row, int group) { return group ^ (row >> 3 << 1); }

// The second product's operand of latents has channels along lanes and tokens in a
// lane: 16 lanes read 8 bytes each, four tokens' 16 channels, and get them turned
// (lane i: channel i of the four tokens).  Lane group g's elements are four tokens in a
// row, and four further on.
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
__device__ inline void put_lds(void* p, float4v v) {
  __asm__ volatile("ds_write_b128 %0, %1" : : "v"(uint32_t(uintptr_t((lds_void*)p))), "v"(v) : "memory");
}
__device__ inline void put_lds(void* p, uint2 v) {
  __asm__ volatile("ds_write_b64 %0, %1" : : "v"(uint32_t(uintptr_t((lds_void*)p))), "v"(uint64_t(v.y) << 32 | v.x) : "memory");
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

// A unit from its record straight into LDS, 1 KB a wave's load; from which chunk a
// lane takes its 16 bytes makes the places above.
template <int L, int RP>
__device__ __forceinline__ void load_unit(const PagedView& c, int layer, int page, int half, int most, int wave, int lane, uint8_t* sm_c,
                                          uint8_t* sm_r) {
  constexpr int PER = 512 / L, N = kUnit / (4 * PER);      // tokens of a load, loads of a wave
  const uint8_t* rec = paged_record_at(c, page, layer, 0);
  const auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(rec), 0, 2 * kPage * (L + RP), kBufferWord3);
  const int sub = PER > 1 ? lane >> 5 : 0, at = ((lane & (L / 8 - 1)) ^ sub << 3) << 4;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int block = 4 * i + wave;
    uint8_t* to = sm_c + block * kBlock;
    if constexpr (PER == 1)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)to, 16, at, (half * kUnit + min(block, most)) * 2 * L, 0, 0);
    else
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)to, 16, min(2 * block + sub, most) * 2 * L + at, half * kUnit * 2 * L, 0, 0);
  }
  if (wave * 1024 < kUnit * RP * 2) {
    constexpr int CH = RP / 8;
    const int t = wave * (64 / CH) + lane / CH, rc = lane & (CH - 1);
    const int rat = min(t, most) * 2 * RP + ((rc ^ (RP == 64 ? (t >> 1) & 7 : (t >> 2) & 3)) << 4);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)(sm_r + wave * 1024), 16, rat, 2 * kPage * L + half * kUnit * 2 * RP, 0, 0);
  }
}

template <int L, int RP, int BF, int RT>
__global__ __launch_bounds__(256, 2) void latent_attn_kernel(LatentAttnArgs a) {
  constexpr int ROWS = 16 * RT, KL = L / 32, KR = RP / 32, CT = L / 64, NQ = RT == 4 ? 2 : 1;   // NQ: tiles of a wave's scores
  constexpr int KT = KL + KR, PARTS = RT == 1 ? 2 : 1, KH = (KT + PARTS - 1) / PARTS;            // products a score, and a wave's part of them
  constexpr int RW = RT == 4 ? 1 : RT;                                                           // row tiles that a wave works out weights of
  constexpr float HEAD = head_of(BF);
  __shared__ __align__(64) uint8_t sm_c0[latents_bytes<L>()], sm_c1[latents_bytes<L>()];
  __shared__ __align__(64) uint8_t sm_r0[kUnit * RP * 2], sm_r1[kUnit * RP * 2];
  __shared__ __align__(16) uint4 sm_p[RT == 4 ? ROWS : 1][4];
  __shared__ float sm_alpha[ROWS], sm_l[ROWS], sm_m[ROWS];
  __shared__ __align__(16) uint32_t sm_moved[4];
  __shared__ __align__(16) float4v sm_x[PARTS][RT == 4 ? 1 : RT][2][RT == 4 ? 1 : 64];           // [part][row tile][token tile][lane]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
  const PagedView& c = a.c;
  if (blockIdx.x == gridDim.x - 1)
    for (int s = tid; s < a.r.n_seqs; s += 256)
      if (starts_bad(a.r, s)) atomicOr(c.status, kBad);
  const Tile tl = tile_of<ROWS>(a, blockIdx.x, lane);
  int32_t* about = reinterpret_cast<int32_t*>(a.ws);      // of every tile: its first partial, how far they lie apart, their number
  if (a.target > 0 && tid == 0 && int(blockIdx.x) < a.target && int(blockIdx.x) >= tl.tiles) about[kTileWords * blockIdx.x + 2] = 0;
  if (tl.seq < 0) return;

  // this wave's scores: of row tile rt0, from token tile tt0 on, part `part` of the channels
  const int rt0 = wave % RT, tt0 = RT == 4 ? 0 : RT == 2 ? wave >> 1 : wave & 1, part = RT == 1 ? wave >> 1 : 0;
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

  uint4 q[KH];
  int limit[RW];                                          // the last token that the lane's rows see
#pragma unroll
  for (int r = 0; r < RW; ++r) limit[r] = m0 + int(uint32_t(min(tl.first + 16 * (RT == 4 ? rt0 : r) + n, tl.rows - 1)) / uint32_t(a.n_heads));
  {
    const int row = min(tl.first + 16 * rt0 + n, tl.rows - 1), i = int(uint32_t(row) / uint32_t(a.n_heads)), h = row - i * a.n_heads;
    const uint16_t* src = a.q + int64_t(tl.row0 + i) * a.qT + h * a.qH + 8 * g;
    const uint16_t* more = a.q_rope + int64_t(tl.row0 + i) * a.rT + h * a.rH + 8 * g;
    auto queries = [&](auto from) __attribute__((always_inline)) {
      constexpr int FROM = decltype(from)::value;
#pragma unroll
      for (int k = FROM; k < FROM + KH && k < KT; ++k) q[k - FROM] = *reinterpret_cast<const uint4*>(k < KL ? src + 32 * k : more + 32 * (k - KL));
    };
    if (PARTS == 1 || part == 0) queries(std::integral_constant<int, 0>{});
    else queries(std::integral_constant<int, KH>{});
  }
  const int all_see = m0 + int(uint32_t(tl.first) / uint32_t(a.n_heads));   // what the tile's first row sees, every row does

  float4v o[RT][CT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int k = 0; k < CT; ++k) o[r][k] = float4v{0, 0, 0, 0};
  float M[RW], l[RW];
#pragma unroll
  for (int r = 0; r < RW; ++r) {
    M[r] = -INFINITY;
    l[r] = 0.0f;
  }
  // places that the lane reads: of its token's chunk g (every fourth further on is
  // 64 bytes further on, but for bit 3), and what it takes for the transposing reads
  const int qat = latent_place<L>(n, g), qat8 = latent_place<L>(n, g + 8) - 128;    // L == 512: the same
  const int vt = RT == 4 ? 16 * (g >> 1) + 4 * (g & 1) : 4 * g;             // the operand's first token: those + 8, or + 16, follow
  const int vat = latent_place<L>(vt + (n >> 2), 2 * CT * wave + ((n >> 1) & 1)) + 8 * (n & 1);

  // a row's weights of 8 of the unit's tokens, from scores x; the factor of the sums so far
  auto weigh = [&](float (&x)[8], float mx, float& M, float& l, uint4& p) __attribute__((always_inline)) {
    mx = row_max(mx) * a.scale_log2e;
    const float Mn = mx > M + kLag || M == -INFINITY ? fmaxf(mx, M) : M;
    const float alpha = M == -INFINITY || Mn == M ? 1.0f : exp2_fast(M - Mn);
    M = Mn;
    l *= alpha;
    const float ref = M == -INFINITY ? 0.0f : M - HEAD;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = exp2_fast(fmaf(x[e], a.scale_log2e, -ref));
      l += x[e];
    }
    p = make_uint4(pack2<BF>(x[0], x[1]), pack2<BF>(x[2], x[3]), pack2<BF>(x[4], x[5]), pack2<BF>(x[6], x[7]));
    return alpha;
  };
  // scores of tokens 4 g + i and 16 + 4 g + i of unit `at`, without those that the row does not see, and their maximum
  auto seen_of = [&](float (&x)[8], int at, int limit) __attribute__((always_inline)) {
    if (at * kUnit + kUnit - 1 > all_see) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at * kUnit + 16 * (e >> 2) + 4 * g + (e & 3) > limit) x[e] = -INFINITY;
    }
    float mx = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) mx = fmaxf(mx, x[e]);
    return mx;
  };

  auto step = [&](const uint8_t* sm_c, const uint8_t* sm_r, uint8_t* next_c, uint8_t* next_r) __attribute__((always_inline)) {
    meet_loaded();
    const int at = u;
    u = next;
    const int after = table[min(u + 1, u1 - 1) >> 1];
    if (u < u1) load(u, next_c, next_r);

    // two sums for each tile where the tile is the wave's only one: products that wait
    // for each other take twice as long
    constexpr int CH = NQ == 1 ? 2 : 1;
    float4v x[NQ][CH];
    auto products = [&](auto from) __attribute__((always_inline)) {
      constexpr int FROM = decltype(from)::value, N = KT - FROM < KH ? KT - FROM : KH;
      __builtin_amdgcn_s_setprio(1);
      const int tile = 16 * tt0;
#pragma unroll
      for (int k = FROM; k < FROM + N; ++k)
#pragma unroll
        for (int j = 0; j < NQ; ++j) {
          const uint8_t* at = k < KL ? sm_c + (L == 512 || !(k & 2) ? qat : qat8) + k * 64 + (tile + 16 * j) * (kBlock * L / 512)
                                     : sm_r + rope_place<RP>(tile + 16 * j + n, 4 * (k - KL) + g);
          const int i = (k - FROM) % CH;
          x[j][i] = mfma<BF>(*reinterpret_cast<const uint4*>(at), q[k - FROM], k - FROM < CH ? float4v{0, 0, 0, 0} : x[j][i]);
        }
      // reads a few products ahead
      constexpr int AHEAD = 4 / NQ;
      __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * NQ, 0);
#pragma unroll
      for (int k = 0; k < N - AHEAD; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, NQ, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, NQ, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, AHEAD * NQ, 0);
      __builtin_amdgcn_s_setprio(0);
    };
    uint4 p[RT];
    float alpha[RT];
    bool moved = false;
    if constexpr (RT == 4) {
      products(std::integral_constant<int, 0>{});
      float y[8] = {x[0][0][0], x[0][0][1], x[0][0][2], x[0][0][3], x[1][0][0], x[1][0][1], x[1][0][2], x[1][0][3]};
      uint4 w;
      const float mx = seen_of(y, at, limit[0]), f = weigh(y, mx, M[0], l[0], w);
      // tokens 4 g + i and 16 + 4 g + i, to where the lanes of the second product take them
#pragma unroll
      for (int j = 0; j < 2; ++j)
        put_lds(reinterpret_cast<uint2*>(&sm_p[16 * rt0 + n][weights_place(n, 2 * j + (g & 1))]) + (g >> 1), j ? make_uint2(w.z, w.w) : make_uint2(w.x, w.y));
      const bool any = __any(f != 1.0f);                   // rows whose reference has moved
      if (any && g == 0) put_lds(&sm_alpha[16 * rt0 + n], f);
      if (lane == 0) put_lds(&sm_moved[rt0], any ? 1u : 0u);
    } else {
      if (PARTS == 1 || part == 0) products(std::integral_constant<int, 0>{});
      else products(std::integral_constant<int, KH>{});
#pragma unroll
      for (int j = 0; j < NQ; ++j) put_lds(&sm_x[part][rt0][tt0 + j][lane], CH == 2 ? x[j][0] + x[j][CH - 1] : x[j][0]);
    }
    meet();
    page = after;
    next = u + 1;
    if (page < 0) next = find(u + 1);
    if constexpr (RT == 4) {
#pragma unroll
      for (int r = 0; r < RT; ++r) p[r] = sm_p[16 * r + n][weights_place(n, g)];
      const uint4 which = *reinterpret_cast<const uint4*>(sm_moved);
      moved = __builtin_amdgcn_readfirstlane(which.x | which.y | which.z | which.w);
      if (moved) {
        const uint32_t w[4] = {which.x, which.y, which.z, which.w};
#pragma unroll
        for (int r = 0; r < RT; ++r) alpha[r] = w[r] ? sm_alpha[16 * r + n] : 1.0f;
      }
    } else {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        float4v y0 = sm_x[0][r][0][lane], y1 = sm_x[0][r][1][lane];
        if constexpr (PARTS == 2) {
          y0 += sm_x[1][r][0][lane];
          y1 += sm_x[1][r][1][lane];
        }
        float y[8] = {y0[0], y0[1], y0[2], y0[3], y1[0], y1[1], y1[2], y1[3]};
        const float mx = seen_of(y, at, limit[r]);
        alpha[r] = weigh(y, mx, M[r], l[r], p[r]);
        moved = moved || alpha[r] != 1.0f;
      }
      moved = __any(moved);
    }
    if (moved) {
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int k = 0; k < CT; ++k) o[r][k] *= alpha[r];
    }
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int k = 0; k < CT; ++k) {
      const uint2 lo = turned4(sm_c + vat + 32 * k), hi = turned4(sm_c + vat + (RT == 4 ? 8 : 16) * (kBlock * L / 512) + 32 * k);
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
    __builtin_amdgcn_s_setprio(0);
  };
#pragma unroll 1
  while (u < u1) {
    step(sm_c0, sm_r0, sm_c1, sm_r1);
    if (u >= u1) break;
    step(sm_c1, sm_r1, sm_c0, sm_r0);
  }

  // the rows' statistics to every wave
#pragma unroll
  for (int r = 0; r < RW; ++r) l[r] = row_sum(l[r]);
  if constexpr (RT == 4) {
    if (g == 0) {
      sm_l[16 * rt0 + n] = l[0];
      sm_m[16 * rt0 + n] = M[0];
    }
    __syncthreads();
  }
  float* sums = a.ws + kTileWords * kSlots + int64_t(tl.slot) * ROWS * partial_floats(L);
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
    const float L0 = RT == 4 ? sm_l[16 * r + n] : l[r % RW], Mr = RT == 4 ? sm_m[16 * r + n] : M[r % RW];
    if (tl.splits > 1) {
#pragma unroll
      for (int k = 0; k < CT; ++k) *reinterpret_cast<float4v*>(sums + (r * (L / 16) + wave * CT + k) * 256 + 4 * lane) = o[r][k];
      if (wave == 0 && g == 0)
        *reinterpret_cast<float4v*>(sums + ROWS * L + 4 * (16 * r + n)) = row < tl.rows ? float4v{Mr, L0, 1.0f, 0.0f} : float4v{Mr, 0.0f, 0.0f, 0.0f};
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

// The splits of a tile joined: 16 rows by 16 channels are a wave's, or SHARE waves',
// of which each takes every SHARE-th split.  A thread takes M and sum of some splits of
// a row, so that their weights are there after one round trip; of the sums B are in
// flight before these are worked out.  (With a loop over splits that waits for each,
// 35 us instead of 8 for 115 rows of four sequences in 64.)
template <int L, int BF, int SHARE>
__global__ __launch_bounds__(SHARE == 1 ? 256 : 64 * SHARE) void latent_join_kernel(LatentAttnArgs a, int rows) {
  constexpr float HEAD = head_of(BF);
  constexpr int WAVES = SHARE == 1 ? 4 : SHARE, PER = 4 * WAVES, NS = kMostSplits / PER, B = 8;   // PER: splits whose M a pass takes
  __shared__ float sm_f[kMostSplits][16], sm_m[WAVES][16], sm_s[WAVES][16], sm_there[16];
  __shared__ __align__(16) float4v sm_v[WAVES - 1][SHARE == 1 ? 1 : 64];
  const int32_t* about = reinterpret_cast<const int32_t*>(a.ws) + kTileWords * blockIdx.x;
  const int splits = about[2];
  if (splits < 2) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, g = lane >> 4;
  const int t = SHARE == 1 ? 4 * int(blockIdx.z) + wave : int(blockIdx.z), first = SHARE == 1 ? 0 : wave;
  const int64_t step = int64_t(about[1]) * rows * partial_floats(L);
  const float* part = a.ws + kTileWords * kSlots + int64_t(about[0]) * rows * partial_floats(L);
  const float* stats = part + rows * L + 4 * (16 * int(blockIdx.y) + n);
  const float* sums = part + (int(blockIdx.y) * (L / 16) + t) * 256 + 4 * lane;
  const int own = tid >> 4;
  float4v st[NS];
#pragma unroll
  for (int i = 0; i < NS; ++i)
    if (PER * i < splits) st[i] = *reinterpret_cast<const float4v*>(stats + min(own + PER * i, splits - 1) * step);
  float4v x[B];
  auto load = [&](int s0) {
#pragma unroll
    for (int k = 0; k < B; ++k)
      if (s0 + k * SHARE < splits) x[k] = *reinterpret_cast<const float4v*>(sums + (s0 + k * SHARE) * step);
  };
  load(first);
  float mx = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int i = 0; i < NS; ++i)
    if (PER * i < splits) mx = fmaxf(mx, st[i][0]);        // (the last split more than once: the same maximum)
  mx = row_max(mx);
  if (g == 0) sm_m[wave][n] = mx;
  if (own == 0) sm_there[n] = st[0][2];
  __syncthreads();
  float M = sm_m[0][n];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) M = fmaxf(M, sm_m[w][n]);
#pragma unroll
  for (int i = 0; i < NS; ++i)
    if (own + PER * i < splits) {
      const float f = st[i][0] == -INFINITY ? 1.0f : exp2_fast(st[i][0] - M);    // nothing seen: zeros, or NaN
      sm_f[own + PER * i][n] = f;
      sum += st[i][1] * f;
    }
  sum = row_sum(sum);
  if (g == 0) sm_s[wave][n] = sum;
  __syncthreads();
  sum = sm_s[0][n];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) sum += sm_s[w][n];
  float4v v = float4v{0, 0, 0, 0};
  for (int s0 = first; s0 < splits; s0 += SHARE * B) {
    if (s0 != first) load(s0);
#pragma unroll
    for (int k = 0; k < B; ++k)
      if (s0 + k * SHARE < splits) v += x[k] * sm_f[s0 + k * SHARE][n];
  }
  if constexpr (SHARE > 1) {
    if (wave > 0) sm_v[wave - 1][lane] = v;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int k = 0; k < SHARE - 1; ++k) v += sm_v[k][lane];
  }
  if (sm_there[n] == 0.0f) return;                         // past the sequence's rows
  const int64_t at = int64_t(about[3]) + 16 * int(blockIdx.y) + n;
  v *= sum == 0.0f ? 0.0f : 1.0f / sum;
  *reinterpret_cast<uint2*>(a.out + at * L + 16 * t + 4 * g) = make_uint2(pack2<BF>(v[0], v[1]), pack2<BF>(v[2], v[3]));
  if (a.lse && t == 0 && g == 0) a.lse[at] = sum == 0.0f ? -INFINITY : (M - HEAD + __builtin_log2f(sum)) * 0.69314718055994531f;
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
  if (split) {
    // blocks of 16 rows by 16 channels: where these are too few for the chip's loads, more
    // waves share one's splits (one token over 32768, 32 blocks of 128 splits: 21.5 us with
    // 4 waves, 18.9 with 16; 64 sequences of 2048, 2048 blocks: 33.6 with 4, 32.9 with one,
    // 44 with 16)
    const int64_t blocks = tiles * (RT * L / 16);
    if (blocks <= 128) hipLaunchKernelGGL((latent_join_kernel<L, BF, 16>), dim3(unsigned(tiles), RT, L / 16), dim3(1024), 0, s, a, ROWS);
    else if (blocks <= 1024) hipLaunchKernelGGL((latent_join_kernel<L, BF, 4>), dim3(unsigned(tiles), RT, L / 16), dim3(256), 0, s, a, ROWS);
    else hipLaunchKernelGGL((latent_join_kernel<L, BF, 1>), dim3(unsigned(tiles), RT, L / 64), dim3(256), 0, s, a, ROWS);
  }
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

// The tiles' height by the rows that a slot of the call has on average, those without
// any among them: starts are on the device.  (What that misses: 60 tokens of 16 heads
// over 16384 take 57 us as the only slot, in 64-row tiles, and 87 among 64, in 16-row
// ones; a chunk of 512 beside 15 single tokens 328, the two apart 264 + 54.)
template <int L, int RP, int BF>
int launch_rows(const LatentAttnArgs& a, hipStream_t s) {
  const int64_t rows = (a.r.n_rows * a.n_heads + a.r.n_seqs - 1) / a.r.n_seqs;
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
