// paged_attn.hip -- causal attention over the paged 4-bit cache on gfx950.
//
// Rows of one (sequence, kv head): row r is query head r mod gqa of the
// sequence's row r div gqa.  A workgroup takes 16 NR rows and a run of the
// sequence's pages, its waves one page (a record of 64 tokens) at a time.
//
// Both products run on v_mfma_f32_16x16x32_f16 with nothing dequantized:
//   scores  C[16 tokens][16 rows] = codes . q,   x = s_t (c.q) + z_t (sum q)
//   values  C[16 channels][16 rows] = codes . w, w = p_t s_t, and the zeros'
//           share sum_t p_t z_t is kept apart in fp32
// A code enters as the half with its bits at 3..6 (c 2^-21, a subnormal) or
// 7..10 (c 2^-17): a shift for two words of two and an AND each, and the other
// operand carries the 1/16 of the second kind.  (The matrix unit aligns its
// products by the operands' exponents as written: the lower a subnormal's
// bits, the fewer of its product are kept.  With the codes at bits 0..3 and
// 4..7, one shift less, the error of a score was some 20 times this.)  A lane's
// 16-byte loads of a record are its operands but for that, and the scores'
// layout (lane: row lane mod 16, tokens 4 (lane div 16) + i) is the values'
// operand layout, since the words of V hold their tokens in that order: the
// weights go from one product to the next in registers.
//
// What bounds it (8 kv heads of 128 channels, 4 query heads each, one group a
// row): a batch of long contexts memory, 16 sequences of 8 to 16k tokens 50 us, 4.4
// TB/s (43 while their 218 MB stay in the last-level cache); one sequence latency,
// 2k tokens 9.5 us, 32k 14.6 (by builds that leave parts out, when it took 15 to
// 16: 2.5 with the launch until a workgroup knows its tile, 5 for its pages, 2.7 to
// join the splits); chunks vector instructions, 65 % of whose issue slots are taken,
// beside 34 % of the matrix cores': 2048 tokens over 16k 705 us, 828 TFLOP/s.  With
// groups of 64 and 32 75 % and 82 % (847 and 1215 us), and at 64 channels 74 % (a
// 4096-token prompt 130 us): a score takes the same vector instructions for half the
// products, and each further group its own scale and zero.
//
// Softmax: one pass with a running reference M per row, the largest x + e of the
// tokens that the row has seen, where 2^e bounds the token's V scale, so that w =
// 2^(x - M + 10) s_t lies within fp16 whatever the scales; it is moved only when a
// record would pass it by 2^5.  A token that the row does not see, or that is of
// no weight, has no part in it, however large its V; of several channel groups
// each has its scales taken relative to its own largest so far, 2^E_j.  Scores,
// sums, the zeros' share and the accumulators are fp32; w is rounded to fp16
// (nearest), and the share that the rounding takes from the middle of the codes'
// range (7.5) is given back through the zeros' sum, which leaves an error relative
// to the values' spread within their group.
#include <hip/hip_fp16.h>

#include "paged.h"

namespace semkv {
namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

// Workgroups of 4 waves that pages are shared out to (2 a compute unit).  Where
// a tile is split, ceil(pages / chunk) is below twice pages / chunk: at most 2
// kSlots partials, of which each tile's first also names its counter of
// finished splits, each on a 256-byte line at the workspace's head.
constexpr int kLeast = 4, kWhole = 8, kMostSplits = 64;
constexpr int kSlots = 512, kCounterStride = 64, kCounterWords = 2 * kSlots * kCounterStride;
constexpr int kBufferWord3 = 0x00020000;   // raw buffer of 32-bit elements (gfx9 family)
// fp16 weights: 2^10 at the reference, which may lag a record by 2^5 (below
// 65504), so that a weight (a sixteenth of it in every second slot) keeps its 11
// bits down to 2^-20 of the largest
constexpr float kHead = 10.0f, kLag = 5.0f;
constexpr int kSpread = 5;                 // exponents of a page's V scales that lie close together (w keeps its bits to 2^-15 then)

// 8 codes of a word as fp16: slots 0, 1, 4, 5 as c 2^-21, slots 2, 3, 6, 7 as c 2^-17
constexpr float kCode = 0x1p21f;
__device__ inline half8v codes8(uint32_t w) {
  const uint32_t l = w << 3, h = w >> 5;
  const uint4 v = make_uint4(l & 0x00780078u, l & 0x07800780u, h & 0x00780078u, h & 0x07800780u);
  return __builtin_bit_cast(half8v, v);
}
// codes of 128, as normal numbers: for the sums of the other operand
constexpr float kSum = 0x1p14f;
__device__ inline half8v sums8(bool some) {
  const uint32_t l = some ? 0x04000400u : 0u, h = some ? 0x14001400u : 0u;
  return __builtin_bit_cast(half8v, make_uint4(l, h, l, h));
}

__device__ inline float lo16(uint32_t m) { return float(__builtin_bit_cast(half2v, m)[0]); }
__device__ inline float hi16(uint32_t m) { return float(__builtin_bit_cast(half2v, m)[1]); }

// Over the four lanes of a row (16 apart): rows of 16 lanes are exchanged in
// registers, so that lane groups 0 and 1, 2 and 3, then both pairs meet.
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

// Ranges of V scales: the largest's fp16 bits in the lower half, and in the upper
// one the negative of the smallest's, which is 0 for a scale of 0 (a token that
// adds nothing) and the larger the smaller another one is.
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
__device__ inline ushort2v halves(uint32_t x) { return __builtin_bit_cast(ushort2v, x); }
__device__ inline uint32_t word(ushort2v x) { return __builtin_bit_cast(uint32_t, x); }
__device__ inline uint32_t wider(uint32_t x, uint32_t y) { return word(__builtin_elementwise_max(halves(x), halves(y))); }
__device__ inline uint32_t range_of(const uint32_t (&m)[4]) {     // of metadata words
  const uint32_t a = __builtin_amdgcn_perm(m[1], m[0], 0x05040100u), b = __builtin_amdgcn_perm(m[3], m[2], 0x05040100u);
  const uint32_t hi = wider(a, b), lo = wider(word(-halves(a)), word(-halves(b)));
  return wider(__builtin_amdgcn_perm(lo, hi, 0x05040100u), __builtin_amdgcn_perm(lo, hi, 0x07060302u));
}
__device__ inline uint32_t range_over_16(uint32_t x) {            // of 16 lanes, by DPP moves
  x = wider(x, uint32_t(__builtin_amdgcn_mov_dpp(int(x), 0xB1, 0xF, 0xF, true)));    // lane xor 1
  x = wider(x, uint32_t(__builtin_amdgcn_mov_dpp(int(x), 0x4E, 0xF, 0xF, true)));    // lane xor 2
  x = wider(x, uint32_t(__builtin_amdgcn_mov_dpp(int(x), 0x141, 0xF, 0xF, true)));   // mirror of 8 lanes
  return wider(x, uint32_t(__builtin_amdgcn_mov_dpp(int(x), 0x140, 0xF, 0xF, true)));   // mirror of 16
}
// e with scale < 2^e: at most twice too large, for subnormals up to 2^10 times
__device__ inline int exponent_of(uint32_t scale) { return int(scale >> 10) - 14; }
// the range of exponents e - kSpread to e
__device__ inline uint32_t limits_of(int e) {
  const uint32_t low = uint32_t(max(e + 14 - kSpread, 0)) << 10;
  return uint32_t(e + 14) << 10 | 0x3FFu | (low ? 0x10000u - low : 0xFFFFu) << 16;
}
__device__ inline bool passes(uint32_t range, uint32_t limits) {
  return word(__builtin_elementwise_sub_sat(halves(range), halves(limits))) != 0;
}

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// LDS that only one wave uses: its lanes' earlier accesses before its later ones
__device__ inline void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// What a workgroup works on: a tile of a sequence's rows, and a share of the
// pages that it sees.
struct Tile {
  int seq, len, row0, count;         // sequence, its tokens, its first row of the call, and rows
  int rows, first;                   // rows of (token, head), and the first of the tile's
  int pages, splits, split;          // pages the tile's last row sees, workgroups that share them, this one's place
  int part;                          // the tile's first partial and its counter
};

// The pages of a call are shared out by what the sequences really hold: the
// call's tiles times pages over the workgroups wanted for a kv head (a.target)
// make a share (`chunk`), which grows until as many workgroups do: one more
// than fit the chip at once costs as much as filling it again (4 x 32k tokens, 8
// waves a workgroup: 27 us instead of 41).  A sequence is split where it holds
// more than a share and kWhole pages, into kMostSplits at most: joining costs
// 2 us (500 tokens 7.0 us whole, 8.8 in two) and 0.05 more for each split.
__device__ inline int splits_of(int pages, int chunk) {
  if (pages <= max(chunk, kWhole)) return 1;
  const int share = max(chunk, (pages + kMostSplits - 1) / kMostSplits);
  return int(uint32_t(pages + share - 1) / uint32_t(share));
}

// A workgroup finds its tile from its flat index by a prefix sum over the
// sequences, 64 at a time.
template <int ROWS>
__device__ inline Tile tile_of(const PagedAttnArgs& a, int flat, int lane) {
  struct Share { int first, count, len, tiles, pages; };
  auto share = [&](int s0, int& reached) {
    Share k;
    const SeqRows m = lane_rows(a.c, a.r, s0, lane, reached, k.len);
    k.first = m.first;
    k.count = m.count;
    k.tiles = (m.count * a.gqa + ROWS - 1) / ROWS;
    k.pages = (k.len + kPage - 1) / kPage;
    return k;
  };
  int reached = 0;
  Share mine = share(0, reached);
  const int reached64 = reached;
  int64_t work = int64_t(mine.tiles) * mine.pages;
  for (int s0 = 64; s0 < a.r.n_seqs; s0 += 64) {
    const Share k = share(s0, reached);
    work += int64_t(k.tiles) * k.pages;
  }
  const int width = min(a.r.n_seqs, 64);           // lanes that hold a sequence
  for (int d = 1; d < width; d <<= 1) work += __shfl_xor(work, d);
  const uint32_t wl = __builtin_amdgcn_readfirstlane(int(work)), wh = __builtin_amdgcn_readfirstlane(int(work >> 32));
  // past 2^31 pages (never few tiles): one workgroup a tile
  const int even = wh || wl >> 31 ? INT32_MAX / 2 : int((wl + uint32_t(a.target) - 1u) / uint32_t(a.target));
  int chunk = max(even, kLeast);
  if (a.r.n_seqs > 1 && a.r.n_seqs <= 64) {
    int tiles = mine.tiles;
    for (int d = 1; d < width; d <<= 1) tiles += __shfl_xor(tiles, d);
    const int limit = max(a.target, 2 * __builtin_amdgcn_readfirstlane(tiles));
#pragma unroll 1
    for (int tries = 0; tries < 3; ++tries) {
      int made = mine.tiles * splits_of(mine.pages, chunk);
      for (int d = 1; d < width; d <<= 1) made += __shfl_xor(made, d);
      made = __builtin_amdgcn_readfirstlane(made);
      if (made <= limit) break;
      chunk = int(float(chunk) * float(made) / float(limit)) + 1;
    }
  }
  Tile k;
  k.seq = -1;
  int before = 0, parts = 0, sp = 1;
  reached = reached64;
  for (int s0 = 0; s0 < a.r.n_seqs; s0 += 64) {
    if (s0) mine = share(s0, reached);
    const int splits = splits_of(mine.pages, chunk);
    const int n = mine.tiles * splits, held = splits > 1 ? n : 0;
    int incl = n, pincl = held;
    for (int d = 1; d < width; d <<= 1) {
      const int up = __shfl_up(incl, d), pup = __shfl_up(pincl, d);
      if (lane >= d) {
        incl += up;
        pincl += pup;
      }
    }
    const uint64_t above = __ballot(before + incl > flat);
    if (above) {
      const int l = __ffsll((unsigned long long)above) - 1;
      const int at = flat - before - __builtin_amdgcn_readlane(incl - n, l);
      sp = __builtin_amdgcn_readlane(splits, l);
      const int t = int(uint32_t(at) / uint32_t(sp)), tiles = __builtin_amdgcn_readlane(mine.tiles, l);
      k.seq = s0 + l;
      k.split = at - t * sp;
      k.part = parts + __builtin_amdgcn_readlane(pincl - held, l) + t * sp;
      k.first = (tiles - 1 - t) * ROWS;            // the last rows, which see the most, first
      k.row0 = __builtin_amdgcn_readlane(mine.first, l);
      k.count = __builtin_amdgcn_readlane(mine.count, l);
      k.len = __builtin_amdgcn_readlane(mine.len, l);
      break;
    }
    before += __builtin_amdgcn_readlane(incl, 63);
    parts += __builtin_amdgcn_readlane(pincl, 63);
  }
  if (k.seq < 0) return k;
  k.rows = k.count * a.gqa;
  const int last = int(uint32_t(min(k.first + ROWS, k.rows) - 1) / uint32_t(a.gqa));      // row of the call
  const int seen = k.len - k.count + last + 1;
  k.pages = seen > 0 ? (seen + kPage - 1) / kPage : 0;
  k.splits = min(splits_of(k.pages, chunk), sp);
  return k;
}

__device__ inline uint32_t pack_out(float x, float y, bool bf16) {
  if (!bf16) return __builtin_bit_cast(uint32_t, half2v{_Float16(x), _Float16(y)});
  uint32_t b[2] = {__float_as_uint(x), __float_as_uint(y)};
#pragma unroll
  for (int e = 0; e < 2; ++e)
    b[e] = (b[e] & 0x7FFFFFFFu) > 0x7F800000u ? 0x7FC0u : (b[e] + 0x7FFFu + ((b[e] >> 16) & 1u)) >> 16;
  return b[0] | b[1] << 16;
}

// A store that another XCD's workgroups see
__device__ inline void store_far(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Four channels of an output row: sums v and l relative to the reference M.
template <int D>
__device__ inline void put_row(const PagedAttnArgs& a, const Tile& tl, int head, int row, int ch, float M, float L, float4v v) {
  const int i = row / a.gqa, g = row - i * a.gqa;
  const int64_t at = int64_t(tl.row0 + i) * a.c.n_kv_heads * a.gqa + head * a.gqa + g;
  v *= L == 0.0f ? 0.0f : 1.0f / L;                // no token: zeros
  *reinterpret_cast<uint2*>(a.out + at * D + ch) = make_uint2(pack_out(v[0], v[1], a.bf16), pack_out(v[2], v[3], a.bf16));
  if (ch == 0 && a.lse) a.lse[at] = L == 0.0f ? -INFINITY : (M - kHead + __builtin_log2f(L)) * 0.69314718055994531f;
}

// What a wave knows of its pages' V scales.  E: exponents of the groups' scales by
// which weights and sums are scaled (one group: none).  limits: range that a lane
// expects of the scales it holds; at first that of values of ordinary size (2^-6
// to 1), so that the first page needs no set-up.  bound: of the exponents within
// the limits, less E.  apart: the present page's exponents differ by more than
// kSpread.
template <int NG>
struct Scales {
  int E[NG];
  uint32_t limits;
  float bound;
  bool apart;
};

// Each group's V scales seldom leave the range that an earlier page set.  Where
// they do, it is set anew, and E raised if need be.  FIRST: the lane that the
// first group's range begins at, the next group's 16 lanes on; lanes that hold
// none have limits that nothing passes.
template <int NG, int NR, int NC, int FIRST>
__device__ __forceinline__ void look(Scales<NG>& sc, uint32_t range, bool holds, int kg, float4v (&o)[NR][NC], float4v (&ws)[NR]) {
  if (__builtin_expect(!__any(passes(range, sc.limits)), 1)) return;
  range = range_over_16(range);
  int most = -64, least = 64;                      // of the page's exponents, less E
  float fall[NG];
  bool rise = false;
#pragma unroll
  for (int j = 0; j < NG; ++j) {
    const uint32_t both = __builtin_amdgcn_readlane(range, FIRST + 16 * j);
    const int hi = exponent_of(both & 0xFFFFu), lo = both >> 16 ? exponent_of(0x10000u - (both >> 16)) : 64;
    fall[j] = __builtin_ldexpf(1.0f, min(sc.E[j] - hi, 0));
    if (NG > 1 && hi > sc.E[j]) {
      sc.E[j] = hi;
      rise = true;
    }
    most = max(most, hi - sc.E[j]);
    least = min(least, lo - sc.E[j]);
    if (kg % NG == j) sc.limits = limits_of(hi);
  }
  if (!holds) sc.limits = ~0u;
  if (rise) {                                      // the groups' sums so far are of the lower ones
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        ws[r] *= kg == j ? fall[j] : 1.0f;
#pragma unroll
        for (int ct = j * (NC / NG); ct < (j + 1) * (NC / NG); ++ct) o[r][ct] *= fall[j];
      }
  }
  sc.bound = float(most);
  sc.apart = most - least > kSpread;
}

// Partial of one split: each row's D sums, its M and l.
template <int D>
constexpr int partial_floats(int rows) { return rows * (D + 4); }

// SHARE: every wave has rows of its own and all walk the tile's pages together,
// each decoding a part of a page's codes into LDS for the others: a quarter of
// the decoding, for calls whose tiles fill the chip.  Otherwise the waves share
// rows and take pages in turn.
template <int D, int G, int NR, int NW, bool SHARE>
__global__ __launch_bounds__(64 * NW, 2) void paged_attn_kernel(PagedAttnArgs a) {
  constexpr int NK = D / 32, NC = D / 16, NG = D / G, KG = G / 32, CG = G / 16, ROWS = 16 * NR * (SHARE ? NW : 1);
  constexpr int CB = paged_code_bytes(D), NP = D / 32;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, kg = lane >> 4;
  const PagedView& c = a.c;
  const int head = blockIdx.x % c.n_kv_heads;
  if (blockIdx.x == gridDim.x - 1)                 // (the last workgroup: seldom one with a tile)
    for (int s = threadIdx.x; s < a.r.n_seqs; s += 64 * NW)
      if (starts_bad(a.r, s)) atomicOr(c.status, 4);
  const Tile tl = tile_of<ROWS>(a, blockIdx.x / c.n_kv_heads, lane);
  const int split = tl.split;
  if (tl.seq < 0 || split >= tl.splits) return;

  // the rows' queries, and behind them the wave's first record: in flight together
  uint4 qw[NR][NK];
  const int m0 = tl.len - tl.count, first = tl.first + (SHARE ? 16 * NR * wave : 0);   // the wave's first row
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int row = first + 16 * r + n < tl.rows ? first + 16 * r + n : tl.first;
    const int i = int(uint32_t(row) / uint32_t(a.gqa)), g = row - i * a.gqa;
    const uint16_t* src = a.q + int64_t(tl.row0 + i) * a.sT + int64_t(head * a.gqa + g) * a.sH + 8 * kg;
#pragma unroll
    for (int k = 0; k < NK; ++k) qw[r][k] = *reinterpret_cast<const uint4*>(src + 32 * k);
  }
  // the first row sees the least: pages up to here need no mask
  const int all_see = m0 + int(uint32_t(first) / uint32_t(a.gqa));
  const int each = int(uint32_t(tl.pages + tl.splits - 1) / uint32_t(tl.splits));
  const int p0 = split * each, p1 = min(p0 + each, tl.pages);
  const int32_t* table = c.table + int64_t(tl.seq) * c.seq_pages;
  // A wave's next record is loaded piece by piece as soon as the current one's
  // piece has been used; past its last page, and for a page that is missing,
  // the descriptor's size is 0 and the loads return zeros.
  auto page_at = [&](int p) { return p < p1 ? __builtin_amdgcn_readfirstlane(table[p]) : -1; };
  auto record = [&](int page) {
    return __builtin_amdgcn_make_buffer_rsrc(paged_record_at(c, max(page, 0), a.layer, head), 0,
                                             page < 0 ? 0 : paged_record(D, G), kBufferWord3);
  };
  auto load = [&](const __amdgpu_buffer_rsrc_t& rs, int offset) {
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rs, 16 * lane + offset, 0, 0));
  };
  // Metadata goes through LDS (16 lanes share a token's), a region for each
  // wave; with SHARE a region for each of two pages, and the operands with it
  constexpr int META = 32 * NG, MV = (META + 63) / 64;   // 16-byte words of it, and loads of a wave
  constexpr int FK = SHARE ? 4 * NK : 1, FV = SHARE ? 2 * NC : 1;
  __shared__ __align__(16) uint4 sm_meta[SHARE ? 2 : NW][META];
  __shared__ __align__(16) half8v sm_k[SHARE ? 2 : 1][FK][64], sm_v[SHARE ? 2 : 1][FV][64];
  // with SHARE a wave decodes pieces wave, wave + NW, ... of K's and then V's
  constexpr int MINE = SHARE ? 2 * NP / NW : 1;
  static_assert(!SHARE || (2 * NP % NW == 0 && NW >= 2), "pieces of a page");
  uint4 kw[SHARE ? 1 : NP], vw[SHARE ? 1 : NP], mw[SHARE ? 1 : MV], pw[MINE];
  int page, next;
  auto load_shared = [&](const __amdgpu_buffer_rsrc_t& rs) {
#pragma unroll
    for (int i = 0; i < MINE; ++i) pw[i] = load(rs, 1024 * (wave + NW * i));
    if (wave < MV) mw[0] = load(rs, 2 * CB + 1024 * wave);
  };
  // what was loaded of page p to its place; `have` tokens of the sequence are cached
  auto stage_shared = [&](int p, int have) {
    const int buf = p & 1;
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
      const int piece = wave + NW * i;
      half8v* to = piece < NP ? &sm_k[buf][4 * piece & (FK - 1)][lane] : &sm_v[buf][4 * (piece - NP) & (FV - 1)][lane];
      const uint32_t d[4] = {pw[i].x, pw[i].y, pw[i].z, pw[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) to[64 * e] = codes8(d[e]);
    }
    if (wave < MV && 64 * wave + lane < META) {
      const int at = 64 * wave + lane, t = p * kPage + 4 * (at & 15);
      uint32_t m[4] = {mw[0].x, mw[0].y, mw[0].z, mw[0].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) m[e] = at < 16 * NG || t + e < have ? m[e] : 0u;
      sm_meta[buf][at] = make_uint4(m[0], m[1], m[2], m[3]);
    }
  };
  if constexpr (SHARE) {
    page = page_at(0);
    next = page_at(1);
    load_shared(record(page));
  } else {
    page = page_at(p0 + wave);
    next = page_at(p0 + wave + NW);
    const auto rs = record(page);
#pragma unroll
    for (int i = 0; i < MV; ++i) mw[i] = load(rs, 2 * CB + 1024 * i);
#pragma unroll
    for (int i = 0; i < NP; ++i) kw[i] = load(rs, 1024 * i);
#pragma unroll
    for (int i = 0; i < NP; ++i) vw[i] = load(rs, CB + 1024 * i);
  }

  // the rows' queries as fp16 operands, each row scaled by a power of two so
  // that its largest value lies in [2^14, 2^15); slots 2, 3, 6, 7 carry 1/16
  half8v qf[NR][NK];
  float qs[NR][NG], cf[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const bool valid = first + 16 * r + n < tl.rows;
    uint32_t d[4 * NK];
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const uint4 v = qw[r][k];
      d[4 * k] = valid ? v.x : 0u;
      d[4 * k + 1] = valid ? v.y : 0u;
      d[4 * k + 2] = valid ? v.z : 0u;
      d[4 * k + 3] = valid ? v.w : 0u;
    }
    float x[NK][8], mx = 0.0f;
    if (a.bf16) {
#pragma unroll
      for (int i = 0; i < 8 * NK; ++i) x[i >> 3][i & 7] = __uint_as_float(i & 1 ? d[i >> 1] & 0xFFFF0000u : d[i >> 1] << 16);
    } else {
#pragma unroll
      for (int i = 0; i < 8 * NK; ++i) x[i >> 3][i & 7] = i & 1 ? hi16(d[i >> 1]) : lo16(d[i >> 1]);
    }
#pragma unroll
    for (int k = 0; k < NK; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) mx = fmaxf(mx, fabsf(x[k][e]));
    mx = row_max(mx);
    const int ex = mx > 0.0f ? min(max(15 - __builtin_amdgcn_frexp_expf(mx), -100), 126) : 0;
    const float up = __builtin_ldexpf(1.0f, ex), up4 = __builtin_ldexpf(1.0f, ex - 4);
    cf[r] = fmaxf(__builtin_ldexpf(a.scale_log2e * kCode, -ex), 0x1p-126f);
#pragma unroll
    for (int k = 0; k < NK; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[r][k][e] = _Float16(x[k][e] * (e & 2 ? up4 : up));
    // sum q of each group, in the scores' units
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      float4v acc = float4v{0, 0, 0, 0};
#pragma unroll
      for (int k = j * KG; k < (j + 1) * KG; ++k) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(sums8(true), qf[r][k], acc, 0, 0, 0);
      qs[r][j] = acc[0] * (kSum / kCode);
    }
  }

  float4v o[NR][NC], ws[NR];                       // ws: lane group kg holds group kg's (one group: every lane)
  float M[NR], l[NR], az[NR][NG];
  // lanes whose metadata (of the last load) are V's
  auto holds_v = [&] { return SHARE || (64 * (MV - 1) + lane >= 16 * NG && 64 * (MV - 1) + lane < META); };
  Scales<NG> sc;
#pragma unroll
  for (int j = 0; j < NG; ++j) sc.E[j] = 0;
  sc.limits = holds_v() ? limits_of(0) : ~0u;
  sc.bound = 0.0f;
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    M[r] = -INFINITY;
    l[r] = 0.0f;
#pragma unroll
    for (int j = 0; j < NG; ++j) az[r][j] = 0.0f;
    ws[r] = float4v{0, 0, 0, 0};
#pragma unroll
    for (int ct = 0; ct < NC; ++ct) o[r][ct] = float4v{0, 0, 0, 0};
  }

  if constexpr (SHARE) {
    stage_shared(0, page < 0 ? 0 : tl.len);
    load_shared(record(next));
  }
  // pages that the wave's last row sees (SHARE: it then only decodes)
  const int last_seen = m0 + int(uint32_t(min(first + 16 * NR, tl.rows) - 1) / uint32_t(a.gqa));
  for (int p = SHARE ? 0 : p0 + wave; p < p1; p += SHARE ? 1 : NW) {
    const auto rs = record(next);
    const int have = page < 0 ? 0 : tl.len;        // tokens of a missing page are past the end
    uint32_t range = 0;                            // of the V scales that the lane holds
    const uint4* kmeta;                            // [group][tile][4 tokens of kg]
    if constexpr (SHARE) {
      __syncthreads();                             // page p is staged, page p - 1 has been used
      if (p + 1 < p1) {
        const int after = page_at(p + 2);
        stage_shared(p + 1, next < 0 ? 0 : tl.len);
        load_shared(record(after));
        page = next;
        next = after;
      }
      if (first >= tl.rows || p * kPage > last_seen) continue;
      kmeta = sm_meta[p & 1] + kg;
      const uint4 mv = sm_meta[p & 1][16 * NG + (lane & (16 * NG - 1))];
      const uint32_t m[4] = {mv.x, mv.y, mv.z, mv.w};
      range = range_of(m);
    } else {
      page = next;
      next = page_at(p + 2 * NW);
      // a lane holds 4 tokens of a group, first K's groups, then V's.  V's for
      // tokens past the sequence's end, which may be anything, become 0; the
      // others' range enters the softmax's reference
#pragma unroll
      for (int i = 0; i < MV; ++i) {
        const int at = 64 * i + lane, t = p * kPage + 4 * (at & 15);
        uint32_t m[4] = {mw[i].x, mw[i].y, mw[i].z, mw[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) m[e] = at < 16 * NG || t + e < have ? m[e] : 0u;
        range = range_of(m);                       // the last load is V's
        if (META % 64 == 0 || at < META) sm_meta[wave][at] = make_uint4(m[0], m[1], m[2], m[3]);
      }
      wave_order();
      kmeta = sm_meta[wave] + kg;
    }
    const uint4* vmeta = kmeta + 16 * NG;

    // (SHARE has nothing to load before the scores, which hide this look's wait
    // for LDS: before them it costs a chunk 1 %, a prompt at D = 64 2.5 %.  With four
    // groups it is the other way round)
    constexpr bool kLookLate = SHARE && NG < 4;
    constexpr int kFirstV = SHARE ? 0 : 16 * NG & 63;
    sc.apart = false;
    if constexpr (!kLookLate) look<NG, NR, NC, kFirstV>(sc, range, holds_v(), kg, o, ws);

    // scores (a wave with matrix instructions to issue goes first, here and from
    // the first 32 tokens' values on: without the latter 722 us instead of 698 for
    // 2048 tokens over 16k)
    __builtin_amdgcn_s_setprio(1);
    float4v x[NR][4];
    const uint32_t* kd = reinterpret_cast<const uint32_t*>(kw);
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) {
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        float4v acc[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) acc[r] = float4v{0, 0, 0, 0};
#pragma unroll
        for (int k = j * KG; k < (j + 1) * KG; ++k) {
          const half8v A = SHARE ? sm_k[p & 1][(tt * NK + k) & (FK - 1)][lane] : codes8(kd[SHARE ? 0 : tt * NK + k]);
#pragma unroll
          for (int r = 0; r < NR; ++r) acc[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A, qf[r][k], acc[r], 0, 0, 0);
        }
        const uint4 mk = kmeta[j * 16 + tt * 4];
        const uint32_t m[4] = {mk.x, mk.y, mk.z, mk.w};
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float s = lo16(m[e]), z = hi16(m[e]);
            const float y = fmaf(z, qs[r][j], j == 0 ? 0.0f : x[r][tt][e]);   // (from the half as it is)
            x[r][tt][e] = fmaf(s, acc[r][e], y);
          }
      }
      if (NG > 1) __builtin_amdgcn_sched_barrier(0);   // else the metadata of every tile is read at once, and spilled
    }
    __builtin_amdgcn_s_setprio(0);
    if constexpr (!SHARE) {
#pragma unroll
      for (int i = 0; i < NP; ++i) kw[i] = load(rs, 1024 * i);
#pragma unroll
      for (int i = 0; i < MV; ++i) mw[i] = load(rs, 2 * CB + 1024 * i);
    }
    const int t0 = p * kPage + 4 * kg;             // the lane's first token
    if (p * kPage + kPage - 1 > all_see || have == 0) {   // not every row sees every token
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        // the last token the row sees; worked out here, not kept in a register
        int row = first + 16 * r + n;
        __asm__ volatile("" : "+v"(row));
        const int seen = m0 + int(uint32_t(min(row, tl.rows - 1)) / uint32_t(a.gqa));
#pragma unroll
        for (int tt = 0; tt < 4; ++tt)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[r][tt][e] = t0 + 16 * tt + e > min(seen, have - 1) ? -INFINITY : x[r][tt][e];
      }
    }

    if constexpr (kLookLate) look<NG, NR, NC, kFirstV>(sc, range, holds_v(), kg, o, ws);

    // the page's part of the reference.  Where its exponents lie close together,
    // the largest x plus their bound is at most 2^kSpread too large; else each
    // token's own counts, of several groups (relative to E_j) the largest (where
    // every page needs that: 2048 tokens over 16k 833 us, else 697; one token over
    // 32k 15.4 and 14.3).
    float ref[NR];
    bool move = false;
    float cand[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      float mx = x[r][0][0];
#pragma unroll
      for (int tt = 0; tt < 4; ++tt)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, x[r][tt][e]);
      cand[r] = fmaf(row_max(mx), cf[r], sc.bound);
    }
    if (sc.apart) {
#pragma unroll
      for (int r = 0; r < NR; ++r) cand[r] = -INFINITY;
#pragma unroll
      for (int tt = 0; tt < 4; ++tt) {
        int ex[4] = {-64, -64, -64, -64};
#pragma unroll
        for (int j = 0; j < NG; ++j) {
          const uint4 mv = vmeta[j * 16 + tt * 4];
          const uint32_t m[4] = {mv.x, mv.y, mv.z, mv.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) ex[e] = max(ex[e], exponent_of(m[e] & 0xFFFFu) - sc.E[j]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int r = 0; r < NR; ++r) cand[r] = fmaxf(cand[r], fmaf(x[r][tt][e], cf[r], float(ex[e])));
      }
#pragma unroll
      for (int r = 0; r < NR; ++r) cand[r] = row_max(cand[r]);
    }
#pragma unroll
    for (int r = 0; r < NR; ++r) move |= cand[r] > M[r] + kLag;
    if (__any(move)) {
#pragma unroll
      for (int r = 0; r < NR; ++r) {
        const float Mn = fmaxf(M[r], cand[r]);
        const float f = M[r] == -INFINITY ? 0.0f : exp2_fast(M[r] - Mn);
        M[r] = Mn;
        l[r] *= f;
#pragma unroll
        for (int j = 0; j < NG; ++j) az[r][j] *= f;
        ws[r] *= f;
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) o[r][ct] *= f;
      }
    }
#pragma unroll
    for (int r = 0; r < NR; ++r) ref[r] = M[r] == -INFINITY ? 0.0f : M[r] - kHead;

    // weights of 32 tokens, then their products, twice: vector and matrix
    // instructions of a SIMD's two waves meet oftener (740 us became 698)
    const uint32_t* vd = reinterpret_cast<const uint32_t*>(vw);
    float down[NG];
#pragma unroll
    for (int j = 0; j < NG; ++j) down[j] = __builtin_ldexpf(1.0f, -sc.E[j]);
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      // sums of the rounded weights (of several groups, each in its own four
      // rows of the result)
      const half8v ones = sums8(NG == 1 || n >> 2 == j);
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        half8v wf[NR];
#pragma unroll
        for (int tt = 2 * st; tt < 2 * st + 2; ++tt) {
          const uint4 mv = vmeta[j * 16 + tt * 4];
          const uint32_t m[4] = {mv.x, mv.y, mv.z, mv.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float s = lo16(m[e]), mid = fmaf(7.5f, s, hi16(m[e]));
            const float ss = NG > 1 ? s * (e & 2 ? down[j] * 0.0625f : down[j]) : e & 2 ? s * 0.0625f : s;
#pragma unroll
            for (int r = 0; r < NR; ++r) {
              if (j == 0) {
                x[r][tt][e] = exp2_fast(fmaf(x[r][tt][e], cf[r], -ref[r]));
                l[r] += x[r][tt][e];
              }
              wf[r][4 * (tt & 1) + e] = _Float16(x[r][tt][e] * ss);
              az[r][j] = fmaf(x[r][tt][e], mid, az[r][j]);   // the zeros' share
            }
          }
        }
        if (NG > 1) __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int r = 0; r < NR; ++r) ws[r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, wf[r], ws[r], 0, 0, 0);
#pragma unroll
        for (int ct = j * CG; ct < (j + 1) * CG; ++ct) {
          const half8v A = SHARE ? sm_v[p & 1][(ct * 2 + st) & (FV - 1)][lane] : codes8(vd[SHARE ? 0 : ct * 2 + st]);
#pragma unroll
          for (int r = 0; r < NR; ++r) o[r][ct] = __builtin_amdgcn_mfma_f32_16x16x32_f16(A, wf[r], o[r][ct], 0, 0, 0);
        }
      }
    }
    __builtin_amdgcn_s_setprio(0);
    if constexpr (!SHARE) {
#pragma unroll
      for (int i = 0; i < NP; ++i) vw[i] = load(rs, CB + 1024 * i);
      wave_order();                                // the metadata has been read
    }
  }

  // the waves' states merge in LDS, 16 rows at a time; then the tile's output,
  // or the split's partial
  // (the lane's number made anew: kept over the loop it would be spilled)
  const int lane2 = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0)), tid = 64 * wave + lane2;
  const int n2 = lane2 & 15, kg2 = lane2 >> 4;
  float up[NG];
#pragma unroll
  for (int j = 0; j < NG; ++j) up[j] = __builtin_ldexpf(1.0f, sc.E[j]);
  if constexpr (SHARE) {                           // the wave's rows are whole
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      const float L = row_sum(l[r]);
#pragma unroll
      for (int j = 0; j < NG; ++j) {
        const float w = NG == 1 ? ws[r][0] : __shfl(ws[r][0], 16 * j + n2);
        az[r][j] = fmaf(w, -7.5f * kSum * up[j], row_sum(az[r][j]));
      }
      if (first + 16 * r + n2 >= tl.rows) continue;
#pragma unroll
      for (int ct = 0; ct < NC; ++ct)
        put_row<D>(a, tl, head, first + 16 * r + n2, 16 * ct + 4 * kg2, M[r], L, o[r][ct] * (kCode * up[ct / CG]) + az[r][ct / CG]);
    }
    return;
  }
  constexpr int PITCH = D + 4, LPR = D / 4, NT = 64 * NW;   // LPR: threads of an output row
  __shared__ float sm_m[NW][ROWS], sm_l[NW][ROWS];
  __shared__ __align__(16) float sm_o[NW][16][PITCH];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    l[r] = row_sum(l[r]);
#pragma unroll
    for (int j = 0; j < NG; ++j) {
      // the zeros' share, less what the rounded weights give to 7.5
      const float w = NG == 1 ? ws[r][0] : __shfl(ws[r][0], 16 * j + n2);
      az[r][j] = fmaf(w, -7.5f * kSum * up[j], row_sum(az[r][j]));
    }
    if (kg2 == 0) {
      sm_m[wave][16 * r + n2] = M[r];
      sm_l[wave][16 * r + n2] = l[r];
    }
  }
  __syncthreads();
  const int64_t unit = int64_t(head) * 2 * a.target + tl.part;     // partials of a kv head: below 2 target
  float* parts = a.ws + kCounterWords + unit * partial_floats<D>(ROWS);
  const int rows = min(tl.rows - tl.first, ROWS);
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    if (16 * r >= rows) break;
    float Mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) Mx = fmaxf(Mx, sm_m[w][16 * r + n2]);
    // a row without a token keeps its NaN, if it has one, and zeros else
    const float f = M[r] == -INFINITY ? 1.0f : exp2_fast(M[r] - Mx);
    if (16 * r + n2 < rows) {
#pragma unroll
      for (int ct = 0; ct < NC; ++ct)
        *reinterpret_cast<float4v*>(&sm_o[wave][n2][16 * ct + 4 * kg2]) = (o[r][ct] * (kCode * up[ct / CG]) + az[r][ct / CG]) * f;
    }
    __syncthreads();
    for (int at = tid; at < min(rows - 16 * r, 16) * LPR; at += NT) {
      const int rr = at / LPR, ch = at % LPR * 4;
      float My = -INFINITY, L = 0.0f;
#pragma unroll
      for (int w = 0; w < NW; ++w) My = fmaxf(My, sm_m[w][16 * r + rr]);
      float4v v = float4v{0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float mw = sm_m[w][16 * r + rr], lw = sm_l[w][16 * r + rr];
        L += mw == -INFINITY ? lw : lw * exp2_fast(mw - My);
        v += *reinterpret_cast<const float4v*>(&sm_o[w][rr][ch]);
      }
      if (tl.splits > 1) {
        float* row = parts + split * partial_floats<D>(ROWS) + (16 * r + rr) * (D + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) store_far(row + ch + e, v[e]);
        if (ch == 0) {
          store_far(row + D, My);
          store_far(row + D + 1, L);
        }
      } else {
        put_row<D>(a, tl, head, tl.first + 16 * r + rr, ch, My, L, v);
      }
    }
    __syncthreads();
  }
  if (tl.splits < 2) return;

  // The last workgroup of the tile to arrive joins the splits.  Partials cross
  // XCDs, whose L2s are apart: they are stored and loaded past them, and every
  // thread's stores are complete before its workgroup is counted.
  __shared__ int sm_last;
  __asm__ volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0) {
    uint32_t* counter = reinterpret_cast<uint32_t*>(a.ws) + unit * kCounterStride;
    const uint32_t before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sm_last = before + 1 == uint32_t(tl.splits);
    if (sm_last) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!sm_last) return;
  __asm__ volatile("" ::: "memory");
  // NT/LPR rows at once: where there are fewer, the rest share a row's splits
  const int lanes = rows >= NT / LPR ? 1 : NT / LPR / rows;       // threads to a (row, 4 channels)
  const int at0 = tid / LPR, ch = tid % LPR * 4, part0 = at0 % lanes;
  constexpr int kFar = 16;                                        // cache policy sc1, as agent-scope loads
  const auto far = __builtin_amdgcn_make_buffer_rsrc(parts, 0, tl.splits * partial_floats<D>(ROWS) * 4, kBufferWord3);
  float* sm_j = &sm_o[0][0][0];                                   // [row][lane of it][D + 4]
  static_assert(NT / LPR * (D + 4) <= NW * 16 * PITCH, "join scratch");
  for (int row0 = 0; row0 < rows; row0 += NT / LPR) {
    const int rr = row0 + at0 / lanes;
    const bool mine = rr < rows;
    constexpr int B = 8;                                          // splits in flight
    float My = -INFINITY, L = 0.0f;
    float4v v = float4v{0, 0, 0, 0};
    for (int s0 = part0; mine && s0 < tl.splits; s0 += lanes * B) {
      float m[B], ls[B];
      float4v x[B];
#pragma unroll
      for (int k = 0; k < B; ++k) {
        // past the last split: the last again, with no weight
        const int off = (min(s0 + k * lanes, tl.splits - 1) * partial_floats<D>(ROWS) + rr * (D + 4)) * 4;
        const auto ml = __builtin_amdgcn_raw_buffer_load_b64(far, off + D * 4, 0, kFar);
        m[k] = __uint_as_float(ml[0]);
        ls[k] = __uint_as_float(ml[1]);
        x[k] = __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(far, off + ch * 4, 0, kFar));
      }
      float Mn = My;
#pragma unroll
      for (int k = 0; k < B; ++k) Mn = fmaxf(Mn, m[k]);
      const float keep = My == -INFINITY ? 1.0f : exp2_fast(My - Mn);
      L *= keep;
      v *= keep;
#pragma unroll
      for (int k = 0; k < B; ++k) {
        if (s0 + k * lanes >= tl.splits) continue;
        const float f = m[k] == -INFINITY ? 1.0f : exp2_fast(m[k] - Mn);   // nothing seen: zeros (or NaN)
        L = fmaf(ls[k], f, L);
        v += x[k] * f;
      }
      My = Mn;
    }
    if (lanes > 1) {
      __syncthreads();
      float* j = sm_j + at0 * (D + 4);
      *reinterpret_cast<float4v*>(j + ch) = v;
      if (ch == 0) {
        j[D] = My;
        j[D + 1] = L;
      }
      __syncthreads();
      if (part0 != 0 || !mine) continue;
      float Mn = My;
      for (int k = 1; k < lanes; ++k) Mn = fmaxf(Mn, j[k * (D + 4) + D]);
      const float keep = My == -INFINITY ? 1.0f : exp2_fast(My - Mn);
      L *= keep;
      v *= keep;
      for (int k = 1; k < lanes; ++k) {
        const float mk = j[k * (D + 4) + D], f = mk == -INFINITY ? 1.0f : exp2_fast(mk - Mn);
        L = fmaf(j[k * (D + 4) + D + 1], f, L);
        v += *reinterpret_cast<const float4v*>(j + k * (D + 4) + ch) * f;
      }
      My = Mn;
    }
    if (mine) put_row<D>(a, tl, head, tl.first + rr, ch, My, L, v);
  }
}

template <int D, int G, int NR, int NW, bool SHARE = false>
int launch(PagedAttnArgs a, hipStream_t s) {
  // tiles of the call: a whole tile's rows each, and one more a sequence
  constexpr int ROWS = 16 * NR * (SHARE ? NW : 1);
  const int64_t whole = a.r.n_rows * ((a.gqa + ROWS - 1) / ROWS);
  int64_t tiles = a.r.n_rows * a.gqa / ROWS + a.r.n_seqs;
  if (tiles > whole) tiles = whole;
  const int64_t units = tiles * a.c.n_kv_heads;
  if (units >= (int64_t(1) << 22)) return -2;      // a grid's threads are counted in 32 bits
  int64_t wanted = kSlots * 4 / NW / a.c.n_kv_heads;
  if (wanted < 1) wanted = 1;
  if (SHARE) wanted = 1;                           // no tile is split
  a.target = int(wanted);
  // every tile, and a share of the wanted ones where pages are split
  int64_t grid = tiles + wanted;
  if (SHARE || a.c.seq_pages <= kWhole) grid = tiles;
  hipLaunchKernelGGL((paged_attn_kernel<D, G, NR, NW, SHARE>), dim3(unsigned(grid * a.c.n_kv_heads)), dim3(64 * NW), 0, s, a);
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

template <int D, int G>
int launch_rows(const PagedAttnArgs& a, hipStream_t s) {
  const int64_t rows = (a.r.n_rows * a.gqa + a.r.n_seqs - 1) / a.r.n_seqs;   // of a sequence, on average
  // A workgroup of 8 waves for a single sequence: half as many splits to join
  // (one token over 32k tokens 14.9 us, with 4 waves 17.7); else of 4, two of
  // which hide each other's beginnings and ends (8 x 4k tokens 14.1, 21.5).  By
  // the table's width, since the host knows no length: a short sequence in a wide
  // table loses by it (2k tokens in a table of 512 pages 10.4, with 4 waves 9.4)
  if (rows <= 16 && a.r.n_seqs == 1 && a.c.seq_pages > 64) return launch<D, G, 1, 8>(a, s);
  if (rows <= 16) return launch<D, G, 1, 4>(a, s);
  // as above: 5 tokens of 4 x 32k, with 8 waves 35.5 us, with 4 42.6; 8 chunks
  // of 64 tokens, which fill the chip, 65.5 and 56.7
  if (rows * a.r.n_seqs * a.c.n_kv_heads <= 32 * 128) return launch<D, G, 2, 8>(a, s);
  // Decoding shared by a workgroup's waves, which make a tile of four times the
  // rows and is not split, where such tiles give every compute unit two (4 prompts
  // of 1024 tokens 84 us, 118 apart; a 2048-token chunk over 16k, 512 workgroups,
  // 697 and 725; but 8 chunks of 64 tokens, 128 workgroups, 126 and 59) and are
  // more than half full (64 x 20 tokens over 500 36 and 52, over 4k 164 and 159;
  // 64 x 16 35 and 41, but 163 and 119; 64 x 5 over 500 28 and 21, over 8k 266 and
  // 125).  By the average: the host knows no starts, and a call that is a large
  // chunk and a few single tokens over long contexts is not recognised (2048 over
  // 16k and 15 x 1 over 16k 1177, apart 865; the two in calls of their own 775)
  if (rows > 64 && (a.r.n_rows * a.gqa / 128 + a.r.n_seqs) * a.c.n_kv_heads >= 512) return launch<D, G, 2, 4, true>(a, s);
  return launch<D, G, 2, 4>(a, s);
}

}  // namespace

// counters, and 2 kSlots partials of the widest tile for each kv head
size_t paged_attn_workspace(int d) { return size_t(kCounterWords + 2 * kSlots * 32 * (d + 4)) * 4; }

int launch_paged_attn(PagedAttnArgs a, size_t ws_bytes, hipStream_t s) {
  if (ws_bytes < paged_attn_workspace(a.c.dim)) return -1;
  if (a.c.dim == 128) {
    if (a.c.group == 128) return launch_rows<128, 128>(a, s);
    if (a.c.group == 64) return launch_rows<128, 64>(a, s);
    return launch_rows<128, 32>(a, s);
  }
  if (a.c.group == 64) return launch_rows<64, 64>(a, s);
  return launch_rows<64, 32>(a, s);
}

}  // namespace semkv
