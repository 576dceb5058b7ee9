// latent.hip -- the paged cache of latents on gfx950: rows into pages, and back.
//
// A token is one vector for all heads: a latent part (key and value) and a key
// part that is turned by its position, both kept in 16 bits.  A page holds 64
// tokens of every layer: [64][latent], then [64][rope].  Both calls move rows and
// are memory-bound: 28000 rows of 512 + 64 channels and 16 heads' query parts are taken
// in 39 us (4.6 TB/s in and out), and read back in 12 (from the last-level cache).
#include "paged.h"
#include "rows.h"

namespace semkv {
namespace {

__device__ inline uint16_t* latent_at(const PagedView& c, int page, int layer) {
  return reinterpret_cast<uint16_t*>(paged_record_at(c, page, layer, 0));
}

// Whether eight 16-bit values are all finite: exponents below the type's last.
template <int BF>
__device__ inline bool finite8(const uint4& v) {
  constexpr uint32_t E = BF ? 0x7F80u : 0x7C00u;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  bool ok = true;
#pragma unroll
  for (int e = 0; e < 4; ++e) ok = ok && (w[e] & E) != E && (w[e] >> 16 & E) != E;
  return ok;
}

constexpr int kParts = 4;        // workgroups that share a page's latents
constexpr int kQueryHeads = 32;  // query heads of a workgroup
constexpr int kQueryBlocks = 2048;   // workgroups that queries are shared out to

// The workgroups of a page: kParts for its latents and key parts, a wave a row,
// then those of the queries: kQueryHeads heads and a share of the rows each.
template <int L, int BF>
__global__ __launch_bounds__(256) void latent_append_kernel(LatentAppendArgs a) {
  constexpr int LANES = L / 8;                             // 16 bytes a lane
  __shared__ __align__(16) float2 turns[kPage * turns_pitch(64)];
  const PagedView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int units = c.rope / 16;
  if (blockIdx.x == 0 && blockIdx.y == 0) check_rows(c, a.r);
  if (int(blockIdx.y) < kParts) {
    const int stalled = *c.stalled;
    const PageWork w = page_work(c, a.r, blockIdx.x);
    if (w.seq < 0 || stalled) return;
    // the slots of this workgroup
    const int lo = max(w.lo, kPage / kParts * int(blockIdx.y)), hi = min(w.hi, kPage / kParts * int(blockIdx.y + 1));
    if (lo >= hi) return;
    if (w.page < 0 || c.refs[w.page] > 1) {
      if (tid == 0) atomicOr(c.status, kBad);
      return;
    }
    PageWork mine = w;
    mine.lo = lo;
    mine.hi = hi;
    // a wave's rows, all loaded before the first is looked at
    constexpr int ROWS = kPage / kParts / 4;
    const bool holds = lane < LANES, turns_one = lane < units;
    const Unit place = unit_of(a.rot, lane);
    uint4 v[ROWS], p[ROWS][2];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const int64_t row = w.row0 + min(lo + wave + 4 * k, hi - 1);
      v[k] = p[k][0] = p[k][1] = make_uint4(0, 0, 0, 0);
      if (holds) v[k] = reinterpret_cast<const uint4*>(a.C + row * a.cT)[lane];
      if (turns_one) {
        p[k][0] = *reinterpret_cast<const uint4*>(a.R + row * a.rT + place.at);
        p[k][1] = *reinterpret_cast<const uint4*>(a.R + row * a.rT + place.bt);
      }
    }
    make_turns<64>(a.rot, mine, turns);
    __syncthreads();
    uint16_t* to = latent_at(c, w.page, a.layer);
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const int slot = lo + wave + 4 * k;
      if (slot >= hi) break;
      if (turns_one) turn_unit<BF>(a.rot, turns + slot * turns_pitch(64), lane, p[k]);
      // a token with a value that is not finite is kept as zeros: a weight of 0
      // times it would be NaN in the sums of every row
      const bool ok = !__any(!finite8<BF>(v[k]) || !finite8<BF>(p[k][0]) || !finite8<BF>(p[k][1]));
      if (!ok) {
        v[k] = p[k][0] = p[k][1] = make_uint4(0, 0, 0, 0);
        if (lane == 0) atomicOr(c.status, kNonfinite);
      }
      if (holds) reinterpret_cast<uint4*>(to + slot * L)[lane] = v[k];
      if (turns_one) {
        uint16_t* r = to + kPage * L + slot * c.rope;
        *reinterpret_cast<uint4*>(r + place.at) = p[k][0];
        *reinterpret_cast<uint4*>(r + place.bt) = p[k][1];
      }
    }
    return;
  }
  // the queries of kQueryHeads heads, a share of the page's rows
  const int slice = (int(blockIdx.y) - kParts) / a.q_shares, share = int(blockIdx.y) - kParts - slice * a.q_shares;
  const int h0 = slice * kQueryHeads, heads = min(a.n_heads - h0, kQueryHeads);
  PageWork w = page_work(c, a.r, blockIdx.x);
  if (w.seq < 0) {                                                       // rows before their sequence's first token: zeros
    early_rows(c, a.r, share, a.q_shares, [&](int64_t row) {
      for (int j = 8 * tid; j < heads * c.rope; j += 8 * 256)
        *reinterpret_cast<uint4*>(a.q_out + row * a.oT + (h0 + j / c.rope) * a.oH + j % c.rope) = make_uint4(0, 0, 0, 0);
    });
    return;
  }
  const int rows = w.hi - w.lo, lo = w.lo;
  w.hi = lo + rows * (share + 1) / a.q_shares;
  w.lo = lo + rows * share / a.q_shares;
  if (w.lo >= w.hi) return;
  make_turns<64>(a.rot, w, turns);
  __syncthreads();
  turn_queries<BF, turns_pitch(64)>(a.rot, w, a.q, a.qT, a.qH, a.q_out, a.oT, a.oH, h0, heads, units, turns);
}

// A wave a row: zeros where its page is missing.
__global__ __launch_bounds__(256) void latent_read_kernel(LatentReadArgs a) {
  const PagedView& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lanes = c.latent / 8, more = c.rope / 8;
  auto put = [&](int64_t row, const uint16_t* page, int slot) {
    uint4 v = make_uint4(0, 0, 0, 0), r = v;
    if (page && lane < lanes) v = reinterpret_cast<const uint4*>(page + slot * c.latent)[lane];
    if (page && lane < more) r = reinterpret_cast<const uint4*>(page + kPage * c.latent + slot * c.rope)[lane];
    if (lane < lanes) reinterpret_cast<uint4*>(a.C + row * c.latent)[lane] = v;
    if (lane < more) reinterpret_cast<uint4*>(a.R + row * c.rope)[lane] = r;
  };
  if (blockIdx.x == 0 && blockIdx.y == 0) check_rows(c, a.r);
  const PageWork w = page_work(c, a.r, blockIdx.x);
  if (w.seq < 0) {                                         // rows before their sequence's first token
    early_rows(c, a.r, int(blockIdx.y), kParts, [&](int64_t row) {
      if (wave == 0) put(row, nullptr, 0);
    });
    return;
  }
  const uint16_t* page = w.page < 0 ? nullptr : latent_at(c, w.page, a.layer);
  const int lo = max(w.lo, kPage / kParts * int(blockIdx.y)), hi = min(w.hi, kPage / kParts * int(blockIdx.y + 1));
  for (int slot = lo + wave; slot < hi; slot += 4) put(w.row0 + slot, page, slot);
}

}  // namespace

template <int L>
static void append_of(const LatentAppendArgs& a, dim3 grid, hipStream_t s) {
  if (a.bf16) hipLaunchKernelGGL((latent_append_kernel<L, 1>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((latent_append_kernel<L, 0>), grid, dim3(256), 0, s, a);
}

int launch_latent_append(LatentAppendArgs a, hipStream_t s) {
  const int slices = a.q ? (a.n_heads + kQueryHeads - 1) / kQueryHeads : 0;
  // the queries' workgroups: a few for each CU where there are few pages, of eight rows at
  // least (a page's rows to each: 716 rows of 128 heads, with their reading, 23.6 us and
  // not 15.1; 28000 of 16 heads, 54.7 and not 50.5)
  const int64_t pages = touched_bound(a.r), rows = a.r.n_rows / pages;
  int64_t shares = kQueryBlocks / (pages * (slices ? slices : 1));
  if (shares > rows / 8) shares = rows / 8;
  a.q_shares = shares < 1 ? 1 : int(shares);
  const dim3 grid(unsigned(pages), unsigned(kParts + slices * a.q_shares));
  if (a.c.latent == 512) append_of<512>(a, grid, s);
  else append_of<256>(a, grid, s);
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

int launch_latent_read(const LatentReadArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(latent_read_kernel, dim3(unsigned(touched_bound(a.r)), kParts), dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

}  // namespace semkv
