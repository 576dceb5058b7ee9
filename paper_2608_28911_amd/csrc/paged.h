// paged.h -- argument blocks and device helpers shared by the kernels of the
// paged 4-bit cache (paged.hip, paged_attn.hip) and their host API
// (paged_api.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace semkv {

constexpr int kPage = 64;        // tokens of a page
constexpr int kMaxSeqs = 1024;   // sequence slots: one thread of a workgroup each

__host__ __device__ constexpr int paged_code_bytes(int d) { return 32 * d; }              // K or V codes of a record
__host__ __device__ constexpr int paged_meta_bytes(int d, int g) { return d / g * 256; }  // K or V metadata
__host__ __device__ constexpr int paged_record(int d, int g) {
  return 2 * paged_code_bytes(d) + 2 * paged_meta_bytes(d, g);
}

// The cache as kernels see it: pool, and the parts of the state buffer.
struct PagedView {
  uint8_t* pool;
  int32_t* stalled;              // not 0: the last reserve found no pages
  int32_t* lens;                 // [max_seqs]
  int32_t* table;                // [max_seqs][seq_pages]
  int32_t* refs;                 // [n_pages]
  uint32_t* free;                // bitmap of the free pages
  // scratch of the page calls
  int32_t* new_lens;             // [max_seqs]
  int32_t* changed;              // [max_seqs]
  int32_t* cow;                  // [max_seqs][2]: page to copy and its copy, -1: none
  int32_t* base;                 // [max_seqs]: first entry of `list` that sequence s takes
  int32_t* list;                 // [n_pages]: pages taken by this call
  int32_t* new_table;            // [max_seqs][seq_pages]
  int32_t* status;
  int32_t n_layers, n_kv_heads, n_pages, max_seqs, seq_pages, dim, group, record;
};

__device__ inline uint8_t* paged_record_at(const PagedView& c, int page, int layer, int head) {
  return c.pool + ((int64_t(page) * c.n_layers + layer) * c.n_kv_heads + head) * c.record;
}

// The rows of a call: sequence s has rows starts[s] .. starts[s+1]-1.
struct PagedRows {
  const int32_t* starts;
  int32_t n_seqs;
  int64_t n_rows;
};

struct PagedWriteArgs {
  PagedView c;
  PagedRows r;
  const uint16_t* K; const uint16_t* V;
  int64_t sL, sT, sH;
  int32_t layer0, layers, bf16, parts;
};

struct PagedReadArgs {
  PagedView c;
  PagedRows r;
  void* K; void* V;
  int32_t layer0, layers, dtype;
};

struct PagedAttnArgs {
  PagedView c;
  PagedRows r;
  const uint16_t* q;
  int64_t sT, sH;
  int32_t layer, bf16, gqa, target;
  float scale_log2e;
  uint16_t* out;
  float* lse;
  float* ws;
};

struct TokenArgs {
  const void* x;
  int32_t dtype, batch, top, negate, nsplit;
  int64_t T, vocab, s_batch, s_token;
  const int64_t* targets;
  int64_t t_batch, t_token;
  float* logp; float* entropy;
  int64_t o_batch, o_token;
  float* top_logp; int32_t* top_ids;
  float* ws;
};

// A sequence's share of a call's rows; count 0 where it has none.
struct SeqRows { int32_t first, count; };

// The rows of sequences s0 .. s0+63, one to a lane of the wave.  A sequence has
// none where its starts descend or pass the rows there are, nor where they begin
// before an earlier sequence's rows end: no row is two sequences', and no call
// has more rows in all than the host counted for its grid (a tile of which only
// some workgroups existed would leave its counter behind).  reached: where the
// rows of the sequences before s0 end; moved past these where more follow.  len:
// the sequence's tokens.  All three loads are under way before the first is
// looked at (a row of each of 16 sequences is read in 4.1 us, with loads behind
// conditions in 4.5).
__device__ inline SeqRows lane_rows(const PagedView& c, const PagedRows& r, int s0, int lane, int& reached, int& len) {
  const bool mine = s0 + lane < r.n_seqs;
  const int s = min(s0 + lane, r.n_seqs - 1), rows = int(r.n_rows);
  const int32_t a = r.starts[s], b = r.starts[s + 1];
  len = c.lens[s];
  bool ok = mine && a >= 0 && b > a && b <= rows;
  int end = b;                          // of this and the earlier sequences' rows, where starts ascend
  if (__builtin_expect(__any(a < reached || b < a || b > rows), 0)) {
    end = ok ? b : 0;
#pragma unroll 1
    for (int d = 1; d < 64; d <<= 1) end = max(end, __shfl_up(end, d));
    const int before = __shfl_up(end, 1);
    ok = ok && a >= max(reached, lane ? before : 0);
  }
  if (s0 + 64 < r.n_seqs) reached = max(reached, __builtin_amdgcn_readlane(end, 63));
  return {a, ok ? b - a : 0};
}

// Starts that descend, or pass the rows there are.
__device__ inline bool starts_bad(const PagedRows& r, int s) {
  const int32_t a = r.starts[s], b = r.starts[s + 1];
  return a < 0 || b < a || b > r.n_rows;
}

// Which sequence's tile a flat index names, where a sequence of `len` tokens
// and `count` rows has tiles(len, count) of them; and its rows and tokens.  The
// whole wave counts 64 sequences at a time.  -1 past the last.
template <class F>
__device__ inline int find_tile(const PagedView& c, const PagedRows& r, int flat, int lane, F tiles, int& tile, SeqRows& rows,
                                int& len) {
  int before = 0, reached = 0;
  for (int s0 = 0; s0 < r.n_seqs; s0 += 64) {
    int own;
    const SeqRows mine = lane_rows(c, r, s0, lane, reached, own);
    int n = tiles(own, mine.count), incl = n;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int up = __shfl_up(incl, d);
      if (lane >= d) incl += up;
    }
    const uint64_t above = __ballot(before + incl > flat);
    if (above) {
      const int l = __ffsll((unsigned long long)above) - 1;
      const int start = before + __shfl(incl - n, l);
      tile = flat - start;
      rows = {__builtin_amdgcn_readlane(mine.first, l), __builtin_amdgcn_readlane(mine.count, l)};
      len = __builtin_amdgcn_readlane(own, l);
      return __builtin_amdgcn_readfirstlane(s0 + l);
    }
    before += __shfl(incl, 63);
  }
  tile = 0;
  return -1;
}

int launch_paged_clear(const PagedView& c, int tables, hipStream_t s);
int launch_paged_assign(const PagedView& c, const int32_t* lens, const int32_t* table, hipStream_t s);
int launch_paged_reserve(const PagedView& c, const int32_t* n_new, hipStream_t s);
int launch_paged_fork(const PagedView& c, const int32_t* parent, hipStream_t s);
int launch_paged_compact(const PagedView& c, const int32_t* keep, int64_t ld, const int32_t* n_keep, hipStream_t s);
int launch_paged_write(PagedWriteArgs a, hipStream_t s);
int launch_paged_read(const PagedReadArgs& a, hipStream_t s);
size_t paged_attn_workspace(int d);
int launch_paged_attn(PagedAttnArgs a, size_t ws_bytes, hipStream_t s);
size_t token_logprobs_workspace(int64_t rows, int64_t vocab, int top);
int launch_token_logprobs(TokenArgs a, hipStream_t s);

}  // namespace semkv
