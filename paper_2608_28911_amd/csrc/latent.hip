// latent.hip -- the paged cache of latents on gfx950: rows into pages, and back.
//
// A token is one vector for all heads: a latent part (key and value) and a key
// part that is turned by its position, both kept in 16 bits.  A page holds 64
// tokens of every layer: [64][latent], then [64][rope].  Both calls move rows and
// are memory-bound.
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

// The workgroups of a page: kParts for its latents and key parts, a wave a row,
// then those of the queries.
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
    make_turns<64>(a.rot, mine, turns);
    __syncthreads();
    uint16_t* to = latent_at(c, w.page, a.layer);
    for (int slot = lo + wave; slot < hi; slot += 4) {
      const int64_t row = w.row0 + slot;
      const bool holds = lane < LANES, turns_one = lane < units;
      uint4 v = make_uint4(0, 0, 0, 0), p[2] = {v, v};
      if (holds) v = reinterpret_cast<const uint4*>(a.C + row * a.cT)[lane];
      int at = 0, bt = 0;
      if (turns_one) turn_unit<BF>(a.rot, a.R + row * a.rT, turns + slot * turns_pitch(64), lane, p, at, bt);
      // a token with a value that is not finite is kept as zeros: a weight of 0
      // times it would be NaN in the sums of every row
      const bool ok = !__any(!finite8<BF>(v) || !finite8<BF>(p[0]) || !finite8<BF>(p[1]));
      if (!ok) {
        v = p[0] = p[1] = make_uint4(0, 0, 0, 0);
        if (lane == 0) atomicOr(c.status, kNonfinite);
      }
      if (holds) reinterpret_cast<uint4*>(to + slot * L)[lane] = v;
      if (turns_one) {
        uint16_t* r = to + kPage * L + slot * c.rope;
        *reinterpret_cast<uint4*>(r + at) = p[0];
        *reinterpret_cast<uint4*>(r + bt) = p[1];
      }
    }
    return;
  }
  // the queries of kQueryHeads heads
  const int h0 = (int(blockIdx.y) - kParts) * kQueryHeads, heads = min(a.n_heads - h0, kQueryHeads);
  if (blockIdx.x == 0 && tid < 64) {                       // rows before their sequence's first token: zeros
    int reached = 0;
    for (int s0 = 0; s0 < a.r.n_seqs; s0 += 64) {
      int len;
      const SeqRows m = lane_rows(c, a.r, s0, lane, reached, len);
      for (int i = 0; i < m.count - len; ++i)
        for (int j = 0; j < heads * c.rope; j += 8)
          *reinterpret_cast<uint4*>(a.q_out + int64_t(m.first + i) * a.oT + (h0 + j / c.rope) * a.oH + j % c.rope) = make_uint4(0, 0, 0, 0);
    }
  }
  const PageWork w = page_work(c, a.r, blockIdx.x);
  if (w.seq < 0) return;
  make_turns<64>(a.rot, w, turns);
  __syncthreads();
  const int n = (w.hi - w.lo) * heads * units;
  for (int i = tid; i < n; i += 256) {
    const int u = i % units, h = h0 + i / units % heads, slot = w.lo + i / (units * heads);
    const int64_t row = w.row0 + slot;
    uint4 p[2];
    int at, bt;
    turn_unit<BF>(a.rot, a.q + row * a.qT + h * a.qH, turns + slot * turns_pitch(64), u, p, at, bt);
    uint16_t* to = a.q_out + row * a.oT + h * a.oH;
    *reinterpret_cast<uint4*>(to + at) = p[0];
    *reinterpret_cast<uint4*>(to + bt) = p[1];
  }
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
  if (blockIdx.x == 0 && blockIdx.y == 0) {
    check_rows(c, a.r);
    if (wave == 0) {                                       // rows before their sequence's first token
      int reached = 0;
      for (int s0 = 0; s0 < a.r.n_seqs; s0 += 64) {
        int len;
        const SeqRows m = lane_rows(c, a.r, s0, lane, reached, len);
        for (int l = 0; l < 64; ++l) {
          const int first = __builtin_amdgcn_readlane(m.first, l);
          const int early = __builtin_amdgcn_readlane(m.count - len, l), count = __builtin_amdgcn_readlane(m.count, l);
          for (int i = 0; i < min(early, count); ++i) put(first + i, nullptr, 0);
        }
      }
    }
  }
  const PageWork w = page_work(c, a.r, blockIdx.x);
  if (w.seq < 0) return;
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

int launch_latent_append(const LatentAppendArgs& a, hipStream_t s) {
  const int slices = a.q ? (a.n_heads + kQueryHeads - 1) / kQueryHeads : 0;
  const dim3 grid(unsigned(touched_bound(a.r)), unsigned(kParts + slices));
  if (a.c.latent == 512) append_of<512>(a, grid, s);
  else append_of<256>(a, grid, s);
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

int launch_latent_read(const LatentReadArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(latent_read_kernel, dim3(unsigned(touched_bound(a.r)), kParts), dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? 0 : -5;
}

}  // namespace semkv
