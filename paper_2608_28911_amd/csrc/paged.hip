// paged.hip -- the paged 4-bit cache on gfx950: quantizing rows into pages,
// reading them back, and the calls on page tables (assign, reserve, fork,
// compact).
//
// Page tables are kept on the device, so that a captured loop can take pages
// as it grows; their calls are a few microseconds of latency each (kernel
// times, 16 slots of 33 pages: reserve 5.3 us, the copies of 10 shared pages of
// 557 KB 4.0, fork 3.0 + 3.1; a launch alone is 2.2).  The calls on rows are
// memory-bound from some thousand rows on (8 kv heads, D = G = 128, fp16): 76000
// rows are written in 88 us (4.5 TB/s of rows in and records out) and read in 75
// (5.2 TB/s); 15600 of 62000 tokens of 4 layers move in 77 us; one row of each of
// 16 sequences is written in 3.5 us.  With 32 query heads beside them and K turned on
// the way, 76000 rows (D = G = 64) take 186 us (4.4 TB/s), a row of each of 16
// sequences 4.2.
#include <type_traits>

#include "paged.h"
#include "rows.h"

namespace semkv {
namespace {

// ---- page tables ---------------------------------------------------------

__device__ inline int div_up(int a, int b) { return (a + b - 1) / b; }

// Exclusive sum over the 1024 threads of the workgroup; `total` for all.
__device__ inline int block_scan(int x, int* waves, int& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int incl = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int up = __shfl_up(incl, d);
    if (lane >= d) incl += up;
  }
  __syncthreads();                      // `waves` may still be read from an earlier call
  if (lane == 63) waves[w] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int v = waves[i];
    before += i < w ? v : 0;
    total += v;
  }
  return before + incl - x;
}

// Takes the `want` lowest-numbered free pages into list[0 .. want): their bits
// are cleared and their counts set to 1.  False, and nothing done, if there
// are fewer.  Called by a whole 1024-thread workgroup; each thread owns a run
// of bitmap words, and a prefix sum of their set bits says which pages of the
// list are its own: no atomics, and the same pages every time.
__device__ inline bool take_pages(const PagedView& c, int want, int* waves) {
  const int words = (c.n_pages + 31) / 32, per = (words + 1023) / 1024;
  const int w0 = threadIdx.x * per, w1 = min(w0 + per, words);
  int n = 0;
  for (int w = w0; w < w1; ++w) n += __popc(c.free[w]);
  int total;
  int at = block_scan(n, waves, total);
  if (total < want) return false;
  for (int w = w0; w < w1 && at < want; ++w) {
    uint32_t bits = c.free[w];
    while (bits && at < want) {
      const int p = 32 * w + __ffs(bits) - 1;
      bits &= bits - 1;
      c.list[at++] = p;
      c.refs[p] = 1;
    }
    c.free[w] = bits;
  }
  return true;
}

// One slot more or less that holds page p.
__device__ inline void hold(const PagedView& c, int p) { atomicAdd(c.refs + p, 1); }
__device__ inline void release(const PagedView& c, int p) {
  if (atomicSub(c.refs + p, 1) == 1) atomicOr(c.free + (p >> 5), 1u << (p & 31));
}

// Every page free; `tables`: every sequence empty too.
__global__ __launch_bounds__(256) void paged_clear_kernel(PagedView c, int tables) {
  const int64_t i0 = int64_t(blockIdx.x) * 256 + threadIdx.x, step = int64_t(gridDim.x) * 256;
  if (tables) {
    for (int64_t i = i0; i < int64_t(c.max_seqs) * c.seq_pages; i += step) c.table[i] = -1;
    for (int64_t i = i0; i < c.max_seqs; i += step) c.lens[i] = 0;
  }
  for (int64_t i = i0; i < c.n_pages; i += step) c.refs[i] = 0;
  for (int64_t i = i0; i < c.max_seqs; i += step) c.cow[2 * i] = -1;
  const int words = (c.n_pages + 31) / 32;
  for (int64_t i = i0; i < words; i += step) {
    const int left = c.n_pages - int(32 * i);
    c.free[i] = left >= 32 ? ~0u : (1u << left) - 1u;
  }
  if (i0 == 0) *c.stalled = 0;
}

// The caller's tables, where every page is free (paged_clear_kernel): entries
// in use are copied and counted.  `lens` and `table` may be the cache's own: a
// thread reads the one entry that it writes, and a length that is the cache's
// own is written back as it was.
__global__ __launch_bounds__(256) void paged_assign_kernel(PagedView c, const int32_t* lens, const int32_t* table) {
  const int s = blockIdx.y, col = blockIdx.x * 256 + threadIdx.x;
  const int given = lens[s], most = kPage * c.seq_pages;
  const int len = min(max(given, 0), most);
  if (col == 0) {
    c.lens[s] = len;
    if (len != given) atomicOr(c.status, kBad);
  }
  if (col >= c.seq_pages) return;
  const int64_t at = int64_t(s) * c.seq_pages + col;
  const bool used = col < div_up(len, kPage);
  const int p = used ? table[at] : -1;
  const bool there = p >= 0 && p < c.n_pages;
  c.table[at] = there ? p : -1;
  if (!there) {
    if (used) atomicOr(c.status, kBad);
    return;
  }
  hold(c, p);
  atomicAnd(c.free + (p >> 5), ~(1u << (p & 31)));
}

// One workgroup, a thread for each slot: who needs how many pages (a prefix sum
// places them), who must copy a shared last page, then one thread for each page
// taken, which finds its slot by bisection.
__global__ __launch_bounds__(1024) void paged_reserve_kernel(PagedView c, const int32_t* n_new) {
  __shared__ int waves[16];
  __shared__ int last_of[kMaxSeqs];     // shared last page that sequence s grows into, -1: none
  __shared__ int base_of[kMaxSeqs + 1], held_of[kMaxSeqs];
  __shared__ int full;
  const int t = threadIdx.x;
  const bool mine = t < c.max_seqs;
  int len = 0, n = 0, last = -1, count = 0;
  bool fits = true;
  if (mine) {
    len = c.lens[t];
    n = n_new[t];
    if (n < 0) {
      atomicOr(c.status, kBad);
      n = 0;
    }
    fits = n <= kPage * c.seq_pages - len;
    if (fits && n > 0 && len % kPage != 0) {
      last = c.table[int64_t(t) * c.seq_pages + len / kPage];
      if (last >= 0) count = c.refs[last];
    }
  }
  if (count < 2) last = -1;
  last_of[t] = last;
  if (t == 0) full = 0;
  __syncthreads();
  if (!fits) full = 1;
  bool copy = false;
  if (last >= 0) {                      // others hold it: all but the lowest if every one grows
    int same = 0, lower = 0;
    for (int s = 0; s < c.max_seqs; ++s) {
      const int is = last_of[s] == last;
      same += is;
      lower += s < t ? is : 0;
    }
    copy = same != count || lower > 0;
  }
  __syncthreads();
  const bool no_room = full != 0;
  const int held = div_up(len, kPage), want = no_room ? 0 : div_up(len + n, kPage);
  const int need = no_room ? 0 : want - held + copy;
  int total;
  const int base = block_scan(need, waves, total);
  if (t < c.max_seqs) c.cow[2 * t] = -1;
  if (no_room || !take_pages(c, total, waves)) {
    if (t == 0) {
      *c.stalled = 1;
      atomicOr(c.status, kNoPages);
    }
    return;
  }
  base_of[t] = base;
  held_of[t] = held - copy;             // the entry that the sequence's first page goes to
  if (t == 0) {
    base_of[kMaxSeqs] = total;
    *c.stalled = 0;
  }
  __threadfence_block();
  __syncthreads();
  if (copy) {
    c.cow[2 * t] = last;
    c.cow[2 * t + 1] = c.list[base];
    atomicSub(c.refs + last, 1);
  }
  for (int r = t; r < total; r += 1024) {
    int lo = 0, hi = kMaxSeqs;          // the last sequence whose base is at most r
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (base_of[mid] <= r) lo = mid;
      else hi = mid;
    }
    c.table[int64_t(lo) * c.seq_pages + held_of[lo] + (r - base_of[lo])] = c.list[r];
  }
  if (mine) c.lens[t] = len + n;
}

// The copies of shared last pages: 16 KB a workgroup, every load in flight.
constexpr int kCopyVecs = 1024;
__global__ __launch_bounds__(256) void paged_copy_kernel(PagedView c) {
  const int s = blockIdx.y, src = c.cow[2 * s];
  if (src < 0) return;
  const int64_t bytes = int64_t(c.record) * c.n_layers * c.n_kv_heads, last = bytes / 16 - 1;
  const uint4* from = reinterpret_cast<const uint4*>(c.pool + src * bytes);
  uint4* to = reinterpret_cast<uint4*>(c.pool + c.cow[2 * s + 1] * bytes);
  const int64_t i0 = int64_t(blockIdx.x) * kCopyVecs + threadIdx.x;
  const int64_t i1 = min(i0 + 256, last), i2 = min(i0 + 512, last), i3 = min(i0 + 768, last);   // the last may be copied again
  if (i0 > last) return;
  const uint4 v0 = from[i0], v1 = from[i1], v2 = from[i2], v3 = from[i3];
  to[i0] = v0;
  to[i1] = v1;
  to[i2] = v2;
  to[i3] = v3;
}

// fork, first half: the new rows, and a count more for each page that a
// changed slot takes over.  The second half (paged_install_kernel) counts down
// what the slots held before, so no page is free in between.
__global__ __launch_bounds__(256) void paged_fork_kernel(PagedView c, const int32_t* parent) {
  const int s = blockIdx.y, col = blockIdx.x * 256 + threadIdx.x;
  int p = parent[s];
  const bool bad = p < -1 || p >= c.max_seqs;
  if (bad) p = s;
  if (col == 0) {
    if (bad) atomicOr(c.status, kBad);
    c.changed[s] = p != s;
    c.new_lens[s] = p < 0 ? 0 : c.lens[p];
  }
  if (p == s || col >= c.seq_pages) return;
  const int page = p < 0 ? -1 : c.table[int64_t(p) * c.seq_pages + col];
  c.new_table[int64_t(s) * c.seq_pages + col] = page;
  if (page >= 0) hold(c, page);
}

// The new rows of the changed slots; `listed`: row s is the run of `list` from
// base[s] (compact), else new_table's row (fork).
__global__ __launch_bounds__(256) void paged_install_kernel(PagedView c, int listed) {
  const int s = blockIdx.y, col = blockIdx.x * 256 + threadIdx.x;
  if (!c.changed[s] || col >= c.seq_pages) return;
  const int64_t at = int64_t(s) * c.seq_pages + col;
  const int len = c.new_lens[s], old = c.table[at];
  int page;
  if (listed) page = col < div_up(len, kPage) ? c.list[c.base[s] + col] : -1;
  else page = c.new_table[at];
  c.table[at] = page;
  if (old >= 0) release(c, old);
  if (col == 0) c.lens[s] = len;
}

// compact, first step: which slots change, and their fresh pages.
__global__ __launch_bounds__(1024) void paged_plan_kernel(PagedView c, const int32_t* n_keep, int64_t ld) {
  __shared__ int waves[16];
  const int t = threadIdx.x;
  int n = -1;
  if (t < c.max_seqs) {
    n = n_keep[t];
    if (n < -1 || n > ld || n > int64_t(kPage) * c.seq_pages) {
      atomicOr(c.status, kBad);
      n = -1;
    }
  }
  int total;
  const int base = block_scan(n > 0 ? div_up(n, kPage) : 0, waves, total);
  const bool ok = take_pages(c, total, waves);
  if (!ok && t == 0) atomicOr(c.status, kNoPages);
  if (t < c.max_seqs) {
    c.changed[t] = ok && n >= 0;
    c.new_lens[t] = n;
    c.base[t] = base;
  }
}

// compact, second step: one workgroup builds one record of a fresh page.  A
// K row is 32 D/16 bytes in four places (lane groups), of 16 bytes at D = 128
// and 8 at 64, each moved whole.  A V piece of 16 bytes holds two channels
// (D/32 pieces of 64 lanes) of the 16 tokens whose (t div 4) mod 4 is its lane
// group; a thread builds one of the destination from one load for each of its
// tokens, neighbouring lanes of neighbouring channels.  Memory-bound: tokens
// are in ascending order, so their loads meet the same lines in the L1 (with a
// load for each nibble's word 125 us instead of 77).
template <int D>
__global__ __launch_bounds__(256) void paged_move_kernel(PagedView c, const int32_t* keep, int64_t ld) {
  constexpr int KI = D / 32;                       // K words of a row and lane
  constexpr int CB = paged_code_bytes(D);
  __shared__ const uint8_t* rec_of[kPage];         // record of each kept token, null: none
  __shared__ int slot_of[kPage];
  const int s = blockIdx.y, tid = threadIdx.x;
  const int layer = blockIdx.z / c.n_kv_heads, head = blockIdx.z % c.n_kv_heads;
  if (!c.changed[s]) return;
  const int n = c.new_lens[s], first = blockIdx.x * kPage;
  if (first >= n) return;
  if (tid < kPage) {
    const uint8_t* rec = nullptr;
    int slot = 0;
    if (first + tid < n) {
      const int pos = keep[s * ld + first + tid];
      const int p = pos >= 0 && pos < c.lens[s] ? c.table[int64_t(s) * c.seq_pages + pos / kPage] : -1;
      if (p >= 0) {
        rec = paged_record_at(c, p, layer, head);
        slot = pos % kPage;
      } else if (layer == 0 && head == 0) {
        atomicOr(c.status, kBad);
      }
    }
    rec_of[tid] = rec;
    slot_of[tid] = slot;
  }
  __syncthreads();
  uint8_t* out = paged_record_at(c, c.list[c.base[s] + blockIdx.x], layer, head);
  {
    using Row = typename std::conditional<D == 128, uint4, uint2>::type;
    const int t = tid & 63, g = tid >> 6;          // token, lane group
    const uint8_t* rec = rec_of[t];
    const int st = slot_of[t];
    // word tile * KI, lane 16 g + t mod 16: piece, lane, word
    auto at = [&](int slot) { return (((slot / 16) * KI >> 2) * 64 + 16 * g + (slot & 15)) * 4 + ((slot / 16) * KI & 3); };
    Row v = {};
    if (rec) v = *reinterpret_cast<const Row*>(reinterpret_cast<const uint32_t*>(rec) + at(st));
    *reinterpret_cast<Row*>(reinterpret_cast<uint32_t*>(out) + at(t)) = v;
  }
  for (int i = tid; i < 64 * KI; i += 256) {       // piece and lane of V
    const int lane = i & 63, piece = i >> 6, t0 = 4 * (lane >> 4);
    uint32_t w[4] = {0, 0, 0, 0};                  // channels 32 piece + m and + 16, tokens 0..31 and 32..63
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const int t = t0 + 16 * (k >> 2) + (k & 3), j = ((k >> 2) & 1) * 4 + (k & 3), sh = 4 * (j >> 1) + 16 * (j & 1);
      const uint8_t* rec = rec_of[t];
      const int st = slot_of[t], sj = ((st >> 4) & 1) * 4 + (st & 3), ssh = 4 * (sj >> 1) + 16 * (sj & 1);
      uint4 v = make_uint4(0, 0, 0, 0);
      if (rec) v = reinterpret_cast<const uint4*>(rec + CB)[piece * 64 + ((st >> 2) & 3) * 16 + (lane & 15)];
      const uint32_t lo = st >> 5 ? v.y : v.x, hi = st >> 5 ? v.w : v.z;
      w[k >> 3] |= ((lo >> ssh) & 15u) << sh;
      w[2 + (k >> 3)] |= ((hi >> ssh) & 15u) << sh;
    }
    reinterpret_cast<uint4*>(out + CB)[i] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  // metadata: [K or V][group][token]
  uint32_t* om = reinterpret_cast<uint32_t*>(out + 2 * CB);
  const int groups = 2 * (D / c.group);
  for (int i = tid; i < groups * kPage; i += 256) {
    const int t = i & 63;
    const uint8_t* rec = rec_of[t];
    om[i] = rec ? reinterpret_cast<const uint32_t*>(rec + 2 * CB)[(i & ~63) + slot_of[t]] : 0u;
  }
}

// The same for a cache of latents, whose tokens are whole rows (15600 of 62000 tokens of
// 4 layers, 512 + 64 channels: 40 us with the other steps, 3.6 TB/s in and out).
__global__ __launch_bounds__(256) void latent_move_kernel(PagedView c, const int32_t* keep, int64_t ld) {
  const int s = blockIdx.y, layer = blockIdx.z;
  if (!c.changed[s]) return;
  const int n = c.new_lens[s], first = blockIdx.x * kPage;
  if (first >= n) return;
  uint4* out = reinterpret_cast<uint4*>(paged_record_at(c, c.list[c.base[s] + blockIdx.x], layer, 0));
  const int wide = c.latent / 8, more = c.rope / 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int t = wave; t < kPage; t += 4) {
    const int pos = first + t < n ? keep[s * ld + first + t] : -1;
    const int p = pos >= 0 && pos < c.lens[s] ? c.table[int64_t(s) * c.seq_pages + pos / kPage] : -1;
    if (p < 0 && first + t < n && layer == 0 && lane == 0) atomicOr(c.status, kBad);
    const uint4* from = reinterpret_cast<const uint4*>(paged_record_at(c, max(p, 0), layer, 0));
    uint4 v = make_uint4(0, 0, 0, 0), r = v;
    if (p >= 0 && lane < wide) v = from[pos % kPage * wide + lane];
    if (p >= 0 && lane < more) r = from[kPage * wide + pos % kPage * more + lane];
    if (lane < wide) out[t * wide + lane] = v;
    if (lane < more) out[kPage * wide + t * more + lane] = r;
  }
}

// ---- rows ----------------------------------------------------------------

// Group parameters as fp16, saturated, and a code against the stored pair.
struct Affine {
  uint32_t bits;               // scale | zero << 16
  float zero, inv;
  __device__ Affine(float mn, float mx) {
    const uint32_t zb = f2h(fminf(fmaxf(mn, -65504.0f), 65504.0f) + 0.0f);
    zero = h2f(zb);
    const uint32_t sb = f2h(fminf(fmaxf((mx - zero) / 15.0f, 0.0f), 65504.0f));
    const float scale = h2f(sb);
    inv = scale > 0.0f ? 1.0f / scale : 0.0f;
    bits = sb | zb << 16;
  }
  // x's code into byte e of w: clamped, then rounded (to nearest, ties to even)
  // by the convert
  __device__ uint32_t code(float x, int e, uint32_t w) const {
    return __builtin_amdgcn_cvt_pk_u8_f32(__builtin_amdgcn_fmed3f((x - zero) * inv, 0.0f, 15.0f), e, w);
  }
};

// f over runs of N = 2, 4, 8, 16, 32 or 64 lanes, in all of them: DPP moves
// within 16 lanes, rows of 16 exchanged in registers beyond.
template <int N, class F>
__device__ inline float over_lanes(float x, F f) {
  auto dpp = [](float v, auto ctrl) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), decltype(ctrl)::value, 0xF, 0xF, true));
  };
  x = f(x, dpp(x, std::integral_constant<int, 0xB1>{}));                   // lane xor 1
  if constexpr (N >= 4) x = f(x, dpp(x, std::integral_constant<int, 0x4E>{}));     // lane xor 2
  if constexpr (N >= 8) x = f(x, dpp(x, std::integral_constant<int, 0x141>{}));    // mirror of 8 lanes
  if constexpr (N >= 16) x = f(x, dpp(x, std::integral_constant<int, 0x140>{}));   // mirror of 16
  if constexpr (N >= 32) {
    const uint32_t u = __float_as_uint(x);
    const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    x = f(__uint_as_float(p[0]), __uint_as_float(p[1]));
  }
  if constexpr (N >= 64) {
    const uint32_t u = __float_as_uint(x);
    const auto p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    x = f(__uint_as_float(p[0]), __uint_as_float(p[1]));
  }
  return x;
}
template <int N>
__device__ inline float min_over(float x) { return over_lanes<N>(x, [](float a, float b) { return fminf(a, b); }); }
template <int N>
__device__ inline float max_over(float x) { return over_lanes<N>(x, [](float a, float b) { return fmaxf(a, b); }); }

// Whether every lane of this lane's run of N says so.
template <int N>
__device__ inline bool all_of(bool ok) {
  const uint64_t bad = __ballot(!ok);
  if constexpr (N == 64) return bad == 0;
  else return (bad >> (threadIdx.x & 63 & ~(N - 1)) & ((uint64_t(1) << N) - 1)) == 0;
}

// A page's only row of the call (a generated token): one wave, two channels a
// lane.  A K word is four lanes'; a V word is one channel of 8 tokens, of which
// the row's nibble is replaced.
template <int D, int G, int BF, bool ROT>
__device__ inline void write_row(const PagedWriteArgs& a, const RotaryArgs& rot, const PageWork& w, uint8_t* rec, int z, int kv,
                                 int holders, int head) {
  constexpr int CB = paged_code_bytes(D), KI = D / 32;
  const int lane = threadIdx.x & 63, slot = w.lo;
  const bool on = lane < D / 2;
  const int ch = on ? 2 * lane : 0;
  const uint16_t* X = kv ? a.V : a.K;
  const uint16_t* row = X + int64_t(z) * a.sL + (w.row0 + slot) * a.sT + head * a.sH;
  const uint32_t d = *reinterpret_cast<const uint32_t*>(row + ch);
  const bool turned = ROT && kv == 0 && ch < rot.dim;
  const bool second = ch >= rot.dim / 2;             // of the halves, where those are the pairs
  uint32_t other = 0;
  float2 t0 = make_float2(0.0f, 0.0f), t1 = t0;
  if (turned) {
    const int32_t pos = position_of(rot, w, slot);
    if (rot.interleaved) {
      t0 = turn_of(pos, rot.freqs[ch / 2]);
    } else {
      const int pair = second ? ch - rot.dim / 2 : ch;
      other = *reinterpret_cast<const uint32_t*>(row + (second ? pair : ch + rot.dim / 2));
      t0 = turn_of(pos, rot.freqs[pair]);
      t1 = turn_of(pos, rot.freqs[pair + 1]);
    }
  }
  uint32_t* words = reinterpret_cast<uint32_t*>(rec + kv * CB);
  const int xv = (ch / 16) * 2 + slot / 32;
  uint32_t* vw = words + ((xv >> 2) * 64 + ((slot >> 2) & 3) * 16 + (ch & 15)) * 4 + (xv & 3);
  uint32_t old0 = 0, old1 = 0;
  if (kv) {
    old0 = vw[0];
    old1 = vw[4];
  }
  if (w.page < 0 || holders > 1) {
    if (lane == 0) atomicOr(a.c.status, kBad);
    return;
  }
  float x0, x1;
  unpack2<BF>(d, x0, x1);
  if (turned) {
    if (rot.interleaved) {
      const float x = turned_x(x0, x1, t0);
      x1 = turned_y(x0, x1, t0);
      x0 = x;
    } else {
      float y0, y1;
      unpack2<BF>(other, y0, y1);
      x0 = second ? turned_y(y0, x0, t0) : turned_x(x0, y0, t0);
      x1 = second ? turned_y(y1, x1, t1) : turned_x(x1, y1, t1);
    }
  }
  const bool ok = all_of<G / 2>(finite(x0) && finite(x1));
  const Affine q(min_over<G / 2>(fminf(x0, x1)), max_over<G / 2>(fmaxf(x0, x1)));
  const uint32_t c0 = ok ? q.code(x0, 0, 0u) : 0u, c1 = ok ? q.code(x1, 0, 0u) : 0u;
  if (!ok && on) atomicOr(a.c.status, kNonfinite);
  if (on && ch % G == 0)
    reinterpret_cast<uint32_t*>(rec + 2 * CB + kv * paged_meta_bytes(D, G))[ch / G * kPage + slot] = ok ? q.bits : 0u;
  if (kv) {
    const int j = ((slot >> 4) & 1) * 4 + (slot & 3), sh = 4 * (j >> 1) + 16 * (j & 1);
    if (on) {
      vw[0] = (old0 & ~(15u << sh)) | c0 << sh;
      vw[4] = (old1 & ~(15u << sh)) | c1 << sh;
    }
  } else {
    int v = int(c0 << (4 * (lane & 3)) | c1 << (4 * (lane & 3) + 16));     // slots 2 (lane mod 4) and + 1
    v |= __builtin_amdgcn_mov_dpp(v, 0xB1, 0xF, 0xF, true);
    v |= __builtin_amdgcn_mov_dpp(v, 0x4E, 0xF, 0xF, true);
    const int xk = (slot / 16) * KI + ch / 32;
    if (on && (lane & 3) == 0) words[((xk >> 2) * 64 + (lane >> 2 & 3) * 16 + (slot & 15)) * 4 + (xk & 3)] = uint32_t(v);
  }
}

// Channels at .. at + D/4 - 1 of a row, x, turned; `row` is the whole row in memory,
// which holds the other halves of the pairs (the same lines again, from the L1).
// A lane's channels from rot.dim on stay.
template <int D, int BF>
__device__ __forceinline__ void turn_lane(const RotaryArgs& rot, const uint16_t* row, const float2* turns, int at, float (&x)[D / 4]) {
  constexpr int Q = D / 4;
  const int half = rot.dim / 2;                          // a multiple of 8
#pragma unroll
  for (int i = 0; i < Q; i += 8) {                       // eight channels at a time
    if (at + i < rot.dim) {
      const bool second = !rot.interleaved && at + i >= half;
      const int pair = rot.interleaved ? (at + i) / 2 : second ? at + i - half : at + i;
      if (rot.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const float4 t = *reinterpret_cast<const float4*>(turns + pair + e);
          const float2 ta = make_float2(t.x, t.y), tb = make_float2(t.z, t.w);
          const float a = turned_x(x[i + 2 * e], x[i + 2 * e + 1], ta), b = turned_x(x[i + 2 * e + 2], x[i + 2 * e + 3], tb);
          x[i + 2 * e + 1] = turned_y(x[i + 2 * e], x[i + 2 * e + 1], ta);
          x[i + 2 * e + 3] = turned_y(x[i + 2 * e + 2], x[i + 2 * e + 3], tb);
          x[i + 2 * e] = a;
          x[i + 2 * e + 2] = b;
        }
      } else {
        // y of the pair is x c + (its other half) s, x the same with -s
        const uint4 o = *reinterpret_cast<const uint4*>(row + (second ? pair : pair + half));
        const uint32_t d[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 t = *reinterpret_cast<const float4*>(turns + pair + 2 * e);
          const float sa = second ? t.y : -t.y, sb = second ? t.w : -t.w;
          float y0, y1;
          unpack2<BF>(d[e], y0, y1);
          const float p0 = x[i + 2 * e] * t.x, p1 = x[i + 2 * e + 1] * t.z, q0 = y0 * sa, q1 = y1 * sb;
          x[i + 2 * e] = p0 + q0;
          x[i + 2 * e + 1] = p1 + q1;
        }
      }
    }
  }
}

// One workgroup quantizes the rows of one (page, layer, kv head): K and then
// V, or one of them (a.parts == 2, where there are few pages).
// Four lanes own a token row, D/4 channels each (with 16 lanes a row, loads
// coalesce better, but a group's parameters, two divisions, are worked out in
// four times as many lanes: 140 us instead of 110 for 76000 rows of 8 heads);
// the codes go to LDS as bytes and come out as the words of the record's
// layout.  A page that the rows fill only in part keeps its other rows: K
// words belong to one row, V words hold 8 tokens and are merged with what is
// there.
template <int D, int G, int BF, bool ROT>
__device__ __forceinline__ void write_page(const PagedWriteArgs& a, const RotaryArgs& rot, const PageWork& w, uint8_t* codes, float2* turns,
                                           int zblock, int parts, int head) {
  constexpr int Q = D / 4;                               // channels of a lane
  constexpr int LG = G / Q > 1 ? G / Q : 1;              // lanes of a group
  constexpr int GQ = Q / G > 1 ? Q / G : 1, N = Q / GQ;  // groups of a lane, channels of each
  constexpr int CB = paged_code_bytes(D), KI = D / 32, PITCH = D + 4;
  const PagedView& c = a.c;
  const int tid = threadIdx.x, slot = tid >> 2, q = tid & 3;
  const int z = parts == 2 ? zblock >> 1 : zblock, layer = a.layer0 + z;
  const int kv0 = parts == 2 ? zblock & 1 : 0, kv1 = parts == 2 ? kv0 : 1;
  const int holders = c.refs[max(w.page, 0)];
  uint8_t* rec = paged_record_at(c, max(w.page, 0), layer, head);
  if (w.hi - w.lo == 1) {
    const int kv = kv0 + (tid >> 6);               // a wave each
    if (kv <= kv1) write_row<D, G, BF, ROT>(a, rot, w, rec, z, kv, holders, head);
    return;
  }
  // the rows are loaded before the page's holders are looked at; slots that
  // are no rows of the call load the first's
  const bool mine = slot >= w.lo && slot < w.hi;
  const int64_t from = int64_t(z) * a.sL + (w.row0 + (mine ? slot : w.lo)) * a.sT + head * a.sH + q * Q;
  uint4 in[Q / 8];
#pragma unroll
  for (int i = 0; i < Q / 8; ++i) in[i] = reinterpret_cast<const uint4*>((kv0 ? a.V : a.K) + from)[i];
  if (w.page < 0 || holders > 1) {
    if (tid == 0) atomicOr(c.status, kBad);
    return;
  }
  if constexpr (ROT) {
    if (kv0 == 0) {
      make_turns<D>(rot, w, turns);
      __syncthreads();
    }
  }
  bool bad = false;
#pragma unroll 1
  for (int kv = kv0; kv <= kv1; ++kv) {
    uint32_t* meta = reinterpret_cast<uint32_t*>(rec + 2 * CB + kv * paged_meta_bytes(D, G));
    float x[Q];
#pragma unroll
    for (int i = 0; i < Q / 8; ++i) {
      const uint32_t d[4] = {in[i].x, in[i].y, in[i].z, in[i].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) unpack2<BF>(d[e], x[8 * i + 2 * e], x[8 * i + 2 * e + 1]);
    }
    if constexpr (ROT) {
      if (kv == 0 && q * Q < rot.dim) turn_lane<D, BF>(rot, a.K + from - q * Q, turns + (mine ? slot : w.lo) * turns_pitch(D), q * Q, x);
    }
    if (kv < kv1) {                                      // V's row while K's is worked on
#pragma unroll
      for (int i = 0; i < Q / 8; ++i) in[i] = reinterpret_cast<const uint4*>(a.V + from)[i];
    } else if (kv > kv0) {
      __syncthreads();                                   // K's codes have been read
    }
#pragma unroll
    for (int g = 0; g < GQ; ++g) {
      float mn = x[g * N], mx = mn, nan = 0.0f * mn;
#pragma unroll
      for (int i = 1; i < N; ++i) {
        mn = fminf(mn, x[g * N + i]);
        mx = fmaxf(mx, x[g * N + i]);
        nan = fmaf(x[g * N + i], 0.0f, nan);             // 0, or NaN once a value is not finite
      }
      const bool ok = all_of<LG>(nan == 0.0f);
      const Affine p(LG > 1 ? min_over<LG>(mn) : mn, LG > 1 ? max_over<LG>(mx) : mx);
      bad |= mine && !ok;
#pragma unroll
      for (int i = 0; i < N; i += 4) {
        uint32_t pack = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) pack = p.code(x[g * N + i + e], e, pack);
        *reinterpret_cast<uint32_t*>(codes + slot * PITCH + q * Q + g * N + i) = ok ? pack : 0u;
      }
      if (mine && q % LG == 0) meta[((q * Q) / G + g) * kPage + slot] = ok ? p.bits : 0u;
    }
    __syncthreads();
    uint32_t* words = reinterpret_cast<uint32_t*>(rec + kv * CB);
    const bool whole = w.lo == 0 && w.hi == kPage;
    for (int i = tid; i < kPage * D / 8; i += 256) {
      const int lane = (i >> 2) & 63, x4 = 4 * (i >> 8) + (i & 3);
      if (kv == 0) {
        const int t = 16 * (x4 / KI) + (lane & 15);
        if (t < w.lo || t >= w.hi) continue;
        const uint32_t* p = reinterpret_cast<const uint32_t*>(codes + t * PITCH + 32 * (x4 % KI) + 8 * (lane >> 4));
        // codes 0 .. 3 of a dword as nibbles 0, 2 in its first byte and 1, 3 in
        // its second; the even ones of both dwords make the lower half
        const uint32_t lo = p[0] | p[0] >> 12, hi = p[1] | p[1] >> 12;
        words[i] = __builtin_amdgcn_perm(hi, lo, 0x05010400u);
      } else {
        const int vch = 16 * (x4 >> 1) + (lane & 15), t0 = 32 * (x4 & 1) + 4 * (lane >> 4);
        uint32_t v = 0, mask = ~0u;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          v |= uint32_t(codes[(t0 + 16 * (j >> 2) + (j & 3)) * PITCH + vch]) << (4 * (j >> 1) + 16 * (j & 1));
        if (!whole) {
          mask = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (uint32_t(t0 + 16 * (j >> 2) + (j & 3) - w.lo) < uint32_t(w.hi - w.lo)) mask |= 15u << (4 * (j >> 1) + 16 * (j & 1));
          v &= mask;
        }
        if (mask == ~0u) words[i] = v;
        else if (mask) words[i] = (words[i] & ~mask) | v;
      }
    }
  }
  if (bad) atomicOr(c.status, kNonfinite);
}

template <int D, int G, int BF>
__global__ __launch_bounds__(256) void paged_write_kernel(PagedWriteArgs a) {
  __shared__ __align__(16) uint8_t codes[kPage * (D + 4)];
  if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) check_rows(a.c, a.r);
  const int stalled = *a.c.stalled;
  const PageWork w = page_work(a.c, a.r, blockIdx.x);
  if (w.seq < 0 || stalled) return;
  write_page<D, G, BF, false>(a, RotaryArgs{}, w, codes, nullptr, blockIdx.z, a.parts, blockIdx.y);
}

// Write with the rotation on the way.  The workgroups of a page: for each kv head
// its K, turned before it is quantized, and its V, as above; and as many or more for
// the queries, each a share of the page's rows with every head, which lie together in
// memory and turn alike (a share of the heads with every row instead: 217 us for
// 76000 rows of 8 kv heads and 32 query heads of 64 channels, not 186).  Of those 186
// us 63 are K's and V's (written without a turn 42), the rest the queries' (a copy of
// them 110: memory); 2048 rows of 128 channels 12.7 us (K and V 10).  Several heads to
// a workgroup, which would share their cosines, spill.
template <int D, int G, int BF>
__global__ __launch_bounds__(256, D == 128 ? 3 : 5) void paged_append_kernel(PagedAppendArgs a) {
  __shared__ __align__(16) uint8_t codes[kPage * (D + 4)];
  __shared__ __align__(16) float2 turns[kPage * turns_pitch(D)];
  if (int(blockIdx.z) < a.w.parts) {
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) check_rows(a.w.c, a.w.r);
    const int stalled = *a.w.c.stalled;
    const PageWork w = page_work(a.w.c, a.w.r, blockIdx.x);
    if (w.seq < 0 || stalled) return;
    write_page<D, G, BF, true>(a.w, a.rot, w, codes, turns, blockIdx.z, a.w.parts, blockIdx.y);
    return;
  }
  PageWork w = uniform(page_work(a.w.c, a.w.r, blockIdx.x));
  const int shares = int(gridDim.y) * (int(gridDim.z) - a.w.parts);
  const int share = (int(blockIdx.z) - a.w.parts) * int(gridDim.y) + int(blockIdx.y);
  if (w.seq < 0) {
    // rows before their sequence's first token have no position that the cache knows:
    // their queries are zeros
    early_rows(a.w.c, a.w.r, share, shares, [&](int64_t row) {
#pragma unroll 1
      for (int j = 8 * threadIdx.x; j < a.gqa * a.w.c.n_kv_heads * D; j += 8 * 256)
        *reinterpret_cast<uint4*>(a.q_out + row * a.oT + j / D * a.oH + j % D) = make_uint4(0, 0, 0, 0);
    });
    return;
  }
  const int rows = w.hi - w.lo, lo = w.lo;
  w.hi = lo + rows * (share + 1) / shares;
  w.lo = lo + rows * share / shares;
  if (w.lo >= w.hi) return;
  make_turns<D>(a.rot, w, turns);
  __syncthreads();
  turn_queries<BF, turns_pitch(D)>(a.rot, w, a.q, a.qT, a.qH, a.q_out, a.oT, a.oH, 0, a.w.c.n_kv_heads * a.gqa, D / 16, turns);
}

// One workgroup returns the rows of one (page, layer, kv head): the record
// goes to LDS, a row's values leave in 16-byte stores of neighbouring lanes (with
// a quarter row to a lane 120 us instead of 75).  Memory-bound.
template <int DT>
__device__ inline void store8(void* p, int64_t at, const float (&v)[8]) {
  if constexpr (DT == 2) {
    float4* o = reinterpret_cast<float4*>(static_cast<float*>(p) + at);
    o[0] = make_float4(v[0], v[1], v[2], v[3]);
    o[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t b[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if constexpr (DT == 0) {
          b[e] = f2h(v[2 * i + e]);
        } else {                                   // finite: round to nearest even
          const uint32_t u = __float_as_uint(v[2 * i + e]);
          b[e] = (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
        }
      }
      w[i] = b[0] | b[1] << 16;
    }
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + at) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// The record's words in LDS, with room between runs of 32 and of 256 words so
// that the lanes of a row's neighbouring channels read from different banks.
__device__ inline int spread(int word) { return word + (word >> 5) * 4 + (word >> 8) * 8; }

template <int D, int DT>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedReadArgs a) {
  constexpr int CB = paged_code_bytes(D), KI = D / 32, LPR = D / 8;   // LPR: threads of a row, 8 channels each
  constexpr int WORDS = paged_record(D, 32) / 4;
  __shared__ __align__(16) uint32_t rec[WORDS + WORDS / 32 * 4 + WORDS / 256 * 8];
  const PagedView& c = a.c;
  const int tid = threadIdx.x;
  const int layer = a.layer0 + blockIdx.z, head = blockIdx.y;
  if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) check_rows(c, a.r);
  const PageWork w = page_work(c, a.r, blockIdx.x);
  if (w.seq < 0) {                                 // rows before their sequence's first token: zeros
    early_rows(c, a.r, 0, 1, [&](int64_t row) {
      const float zeros[8] = {};
      if (tid < 2 * LPR)
        store8<DT>(tid < LPR ? a.K : a.V, ((int64_t(blockIdx.z) * a.r.n_rows + row) * c.n_kv_heads + head) * D + tid % LPR * 8, zeros);
    });
    return;
  }
  const uint4* src = reinterpret_cast<const uint4*>(paged_record_at(c, max(w.page, 0), layer, head));
  for (int i = tid; i < c.record / 16; i += 256)
    *reinterpret_cast<uint4*>(rec + spread(4 * i)) = w.page >= 0 ? src[i] : make_uint4(0, 0, 0, 0);
  __syncthreads();
  const int groups = D / c.group, ch = tid % LPR * 8;
  for (int slot = tid / LPR; slot < kPage; slot += 256 / LPR) {
    if (slot < w.lo || slot >= w.hi) continue;
    const int64_t at = ((int64_t(blockIdx.z) * a.r.n_rows + w.row0 + slot) * c.n_kv_heads + head) * D + ch;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      const uint32_t m = rec[spread(2 * CB / 4 + (kv * groups + ch / c.group) * kPage + slot)];
      const float sc = h2f(m & 0xFFFFu), z = h2f(m >> 16);
      float v[8];
      if (kv == 0) {
        const int x = (slot / 16) * KI + ch / 32;
        const uint32_t word = rec[spread(((x >> 2) * 64 + ((ch & 31) >> 3) * 16 + (slot & 15)) * 4 + (x & 3))];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(float((word >> (4 * (j >> 1) + 16 * (j & 1))) & 15u), sc, z);
      } else {
        const int x = (ch / 16) * 2 + slot / 32, j = ((slot >> 4) & 1) * 4 + (slot & 3);
        const int sh = 4 * (j >> 1) + 16 * (j & 1);
        // 8 channels: within 32 words
        const uint32_t* p = rec + spread(CB / 4 + ((x >> 2) * 64 + ((slot >> 2) & 3) * 16 + (ch & 15)) * 4 + (x & 3));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(float((p[4 * e] >> sh) & 15u), sc, z);
      }
      store8<DT>(kv ? a.V : a.K, at, v);
    }
  }
}

inline int done() { return hipGetLastError() == hipSuccess ? 0 : -5; }

inline dim3 table_grid(const PagedView& c) { return dim3(unsigned((c.seq_pages + 255) / 256), unsigned(c.max_seqs)); }

}  // namespace

int launch_paged_clear(const PagedView& c, int tables, hipStream_t s) {
  int64_t n = tables ? int64_t(c.max_seqs) * c.seq_pages : c.max_seqs;
  if (n < c.n_pages) n = c.n_pages;
  const int64_t blocks = (n + 255) / 256;
  hipLaunchKernelGGL(paged_clear_kernel, dim3(unsigned(blocks < 2048 ? blocks : 2048)), dim3(256), 0, s, c, tables);
  return done();
}

int launch_paged_assign(const PagedView& c, const int32_t* lens, const int32_t* table, hipStream_t s) {
  const int st = launch_paged_clear(c, 0, s);
  if (st) return st;
  hipLaunchKernelGGL(paged_assign_kernel, table_grid(c), dim3(256), 0, s, c, lens, table);
  return done();
}

int launch_paged_reserve(const PagedView& c, const int32_t* n_new, hipStream_t s) {
  hipLaunchKernelGGL(paged_reserve_kernel, dim3(1), dim3(1024), 0, s, c, n_new);
  const int64_t vecs = int64_t(c.record) * c.n_layers * c.n_kv_heads / 16;
  hipLaunchKernelGGL(paged_copy_kernel, dim3(unsigned((vecs + kCopyVecs - 1) / kCopyVecs), unsigned(c.max_seqs)), dim3(256), 0, s, c);
  return done();
}

int launch_paged_fork(const PagedView& c, const int32_t* parent, hipStream_t s) {
  hipLaunchKernelGGL(paged_fork_kernel, table_grid(c), dim3(256), 0, s, c, parent);
  hipLaunchKernelGGL(paged_install_kernel, table_grid(c), dim3(256), 0, s, c, 0);
  return done();
}

int launch_paged_compact(const PagedView& c, const int32_t* keep, int64_t ld, const int32_t* n_keep, hipStream_t s) {
  hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(1024), 0, s, c, n_keep, ld);
  int64_t pages = (ld + kPage - 1) / kPage;
  if (pages > c.seq_pages) pages = c.seq_pages;
  if (pages > 0) {
    const dim3 grid(unsigned(pages), unsigned(c.max_seqs), unsigned(c.n_layers * c.n_kv_heads));
    if (c.latent) hipLaunchKernelGGL(latent_move_kernel, grid, dim3(256), 0, s, c, keep, ld);
    else if (c.dim == 128) hipLaunchKernelGGL((paged_move_kernel<128>), grid, dim3(256), 0, s, c, keep, ld);
    else hipLaunchKernelGGL((paged_move_kernel<64>), grid, dim3(256), 0, s, c, keep, ld);
  }
  hipLaunchKernelGGL(paged_install_kernel, table_grid(c), dim3(256), 0, s, c, 1);
  return done();
}

template <int D, int G>
static void write_of(const PagedWriteArgs& a, dim3 grid, hipStream_t s) {
  if (a.bf16) hipLaunchKernelGGL((paged_write_kernel<D, G, 1>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((paged_write_kernel<D, G, 0>), grid, dim3(256), 0, s, a);
}

int launch_paged_write(PagedWriteArgs a, hipStream_t s) {
  // K and V in workgroups of their own where there are few: 2048 rows of 8
  // heads 6.4 us, 7.3 together; 16384 rows 26.4, 24.5; 76000 rows 104, 87.5
  const int64_t bound = touched_bound(a.r);
  a.parts = bound * a.c.n_kv_heads * a.layers < 2048 ? 2 : 1;
  const dim3 grid(unsigned(bound), unsigned(a.c.n_kv_heads), unsigned(a.parts * a.layers));
  if (a.c.dim == 128) {
    if (a.c.group == 128) write_of<128, 128>(a, grid, s);
    else if (a.c.group == 64) write_of<128, 64>(a, grid, s);
    else write_of<128, 32>(a, grid, s);
  } else {
    if (a.c.group == 64) write_of<64, 64>(a, grid, s);
    else write_of<64, 32>(a, grid, s);
  }
  return done();
}

template <int D, int G>
static void append_of(const PagedAppendArgs& a, dim3 grid, hipStream_t s) {
  if (a.w.bf16) hipLaunchKernelGGL((paged_append_kernel<D, G, 1>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((paged_append_kernel<D, G, 0>), grid, dim3(256), 0, s, a);
}

int launch_paged_append(PagedAppendArgs a, hipStream_t s) {
  const PagedView& c = a.w.c;
  const int64_t bound = touched_bound(a.w.r);
  a.w.parts = bound * c.n_kv_heads < 2048 ? 2 : 1;
  // the queries' shares: as many as there are kv heads, or a multiple of four rows each
  // where these and the pages are few (512 rows of 64 query heads to one kv head, with
  // their reading: 51 us in 9 workgroups, 14 so; 2 kv heads and 32: 20, 13)
  int64_t more = 0;
  if (a.q) {
    const int64_t most = a.w.r.n_rows / bound / (4 * c.n_kv_heads);
    more = 2048 / (bound * c.n_kv_heads);
    if (more > most) more = most;
    if (more < 1) more = 1;
  }
  const dim3 grid(unsigned(bound), unsigned(c.n_kv_heads), unsigned(a.w.parts + more));
  if (c.dim == 128) {
    if (c.group == 128) append_of<128, 128>(a, grid, s);
    else if (c.group == 64) append_of<128, 64>(a, grid, s);
    else append_of<128, 32>(a, grid, s);
  } else {
    if (c.group == 64) append_of<64, 64>(a, grid, s);
    else append_of<64, 32>(a, grid, s);
  }
  return done();
}

template <int D>
static void read_of(const PagedReadArgs& a, dim3 grid, hipStream_t s) {
  if (a.dtype == 0) hipLaunchKernelGGL((paged_read_kernel<D, 0>), grid, dim3(256), 0, s, a);
  else if (a.dtype == 1) hipLaunchKernelGGL((paged_read_kernel<D, 1>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((paged_read_kernel<D, 2>), grid, dim3(256), 0, s, a);
}

int launch_paged_read(const PagedReadArgs& a, hipStream_t s) {
  const dim3 grid(unsigned(touched_bound(a.r)), unsigned(a.c.n_kv_heads), unsigned(a.layers));
  if (a.c.dim == 128) read_of<128>(a, grid, s);
  else read_of<64>(a, grid, s);
  return done();
}

}  // namespace semkv
