// paged_api.hip -- host side of the paged 4-bit cache and of token scoring:
// validation, buffer geometry and launches.  Nothing here allocates or
// synchronizes.
#include <math.h>
#include <string.h>

#include "paged.h"
#include "semkv.h"

using namespace semkv;

namespace {

int64_t round64(int64_t words) { return (words + 63) / 64 * 64; }

PagedView view(const semkv_paged* c) {
  PagedView v;
  memset(&v, 0, sizeof(v));
  const semkv_paged_config& k = c->cfg;
  v.pool = c->pool;
  v.stalled = c->state;
  v.lens = c->state + c->sz.lens_word;
  v.table = c->state + c->sz.table_word;
  v.refs = c->state + c->sz.refs_word;
  v.free = reinterpret_cast<uint32_t*>(c->state + c->sz.free_word);
  int32_t* scratch = c->state + c->sz.scratch_word;
  const int64_t seqs = round64(k.max_seqs);
  v.new_lens = scratch;
  v.changed = scratch + seqs;
  v.base = scratch + 2 * seqs;
  v.cow = scratch + 3 * seqs;
  v.list = scratch + 5 * seqs;
  v.new_table = v.list + round64(k.n_pages);
  v.status = c->status;
  v.n_layers = k.n_layers;
  v.n_kv_heads = k.n_kv_heads;
  v.n_pages = k.n_pages;
  v.max_seqs = k.max_seqs;
  v.seq_pages = k.seq_pages;
  v.dim = k.head_dim;
  v.group = k.group;
  v.record = int32_t(c->sz.record_bytes);
  return v;
}

// The rows of a call: 0 if they can be, 1 if there is none, else a status.
int rows_of(const semkv_paged* c, const int32_t* starts, int32_t n_seqs, int64_t n_rows, PagedRows* r) {
  if (n_seqs < 0 || n_seqs > c->cfg.max_seqs || n_rows < 0) return SEMKV_EINVAL;
  if (n_rows > (int64_t(1) << 28)) return SEMKV_EUNSUPPORTED;   // grids of one workgroup a page
  if (n_seqs == 0 || n_rows == 0) return 1;
  if (!starts || (uintptr_t(starts) & 3)) return SEMKV_EINVAL;
  r->starts = starts;
  r->n_seqs = n_seqs;
  r->n_rows = n_rows;
  return 0;
}

// Whether n words at p lie, in part at least, in words [word, end) of the state.
bool inside(const semkv_paged* c, const int32_t* p, int64_t n, int64_t word, int64_t end) {
  const uintptr_t a = uintptr_t(p), state = uintptr_t(c->state);
  return n > 0 && a < state + 4 * end && a + 4 * n > state + 4 * word;
}

// An argument of reserve, fork or compact in what follows the tables, which
// their kernels write while others of their workgroups still read arguments.
// (Lengths and tables are written last: an argument may lie there.)
bool scratched(const semkv_paged* c, const int32_t* p, int64_t n) {
  return inside(c, p, n, c->sz.refs_word, int64_t(c->sz.state_bytes / 4));
}

constexpr int64_t kMaxRows = (int64_t(1) << 24) - 1;

bool layer_ok(const semkv_paged* c, int32_t layer, int32_t least) { return layer >= least && layer < c->cfg.n_layers; }

}  // namespace

extern "C" {

int semkv_paged_cache_sizes(const semkv_paged_config* cfg, semkv_paged_sizes* out) {
  if (!cfg || !out) return SEMKV_EINVAL;
  const semkv_paged_config& k = *cfg;
  if (k.n_layers < 1 || k.n_kv_heads < 1 || k.n_q_heads < 1 || k.n_pages < 1 || k.max_seqs < 1 || k.seq_pages < 1)
    return SEMKV_EINVAL;
  if (k.n_q_heads % k.n_kv_heads || k.n_q_heads / k.n_kv_heads > 64) return SEMKV_EUNSUPPORTED;
  if (k.head_dim != 64 && k.head_dim != 128) return SEMKV_EUNSUPPORTED;
  if ((k.group != 32 && k.group != 64 && k.group != 128) || k.group > k.head_dim) return SEMKV_EUNSUPPORTED;
  if (k.n_pages > (1 << 20) || k.max_seqs > kMaxSeqs || k.seq_pages > (1 << 20)) return SEMKV_EUNSUPPORTED;
  if (int64_t(k.max_seqs) * k.seq_pages > (int64_t(1) << 28)) return SEMKV_EUNSUPPORTED;
  if (int64_t(k.n_layers) * k.n_kv_heads > 65535) return SEMKV_EUNSUPPORTED;
  memset(out, 0, sizeof(*out));
  out->record_bytes = paged_record(k.head_dim, k.group);
  out->page_bytes = out->record_bytes * k.n_layers * k.n_kv_heads;
  out->pool_bytes = size_t(out->page_bytes) * k.n_pages;
  const int64_t table = round64(int64_t(k.max_seqs) * k.seq_pages), seqs = round64(k.max_seqs), pages = round64(k.n_pages);
  out->lens_word = 64;
  out->table_word = out->lens_word + seqs;
  out->refs_word = out->table_word + table;
  out->free_word = out->refs_word + pages;
  out->scratch_word = out->free_word + round64((k.n_pages + 31) / 32);
  out->state_bytes = size_t(out->scratch_word + 5 * seqs + pages + table) * 4;
  out->workspace_bytes = paged_attn_workspace(k.head_dim);
  return SEMKV_OK;
}

int semkv_paged_init(semkv_paged* c, const semkv_paged_config* cfg, void* pool, int32_t* state, int32_t* status,
                     hipStream_t stream) {
  if (!c || !cfg) return SEMKV_EINVAL;
  semkv_paged_sizes sz;
  const int st = semkv_paged_cache_sizes(cfg, &sz);
  if (st) return st;
  if (!pool || !state || !status) return SEMKV_EINVAL;
  if ((uintptr_t(pool) | uintptr_t(state)) & 15 || (uintptr_t(status) & 3)) return SEMKV_EINVAL;
  memset(c, 0, sizeof(*c));
  c->cfg = *cfg;
  c->sz = sz;
  c->pool = static_cast<uint8_t*>(pool);
  c->state = state;
  c->status = status;
  return launch_paged_clear(view(c), 1, stream);
}

int semkv_paged_assign(semkv_paged* c, const int32_t* lens, const int32_t* table, hipStream_t stream) {
  if (!c || !lens || !table) return SEMKV_EINVAL;
  if ((uintptr_t(lens) | uintptr_t(table)) & 3) return SEMKV_EINVAL;
  const PagedView v = view(c);
  const int64_t end = int64_t(c->sz.state_bytes / 4);
  if (lens != v.lens && inside(c, lens, v.max_seqs, 0, end)) return SEMKV_EINVAL;
  if (table != v.table && inside(c, table, int64_t(v.max_seqs) * v.seq_pages, 0, end)) return SEMKV_EINVAL;
  return launch_paged_assign(v, lens, table, stream);
}

int semkv_paged_reserve(semkv_paged* c, const int32_t* n_new, hipStream_t stream) {
  if (!c || !n_new || (uintptr_t(n_new) & 3) || scratched(c, n_new, c->cfg.max_seqs)) return SEMKV_EINVAL;
  return launch_paged_reserve(view(c), n_new, stream);
}

int semkv_paged_fork(semkv_paged* c, const int32_t* parent, hipStream_t stream) {
  if (!c || !parent || (uintptr_t(parent) & 3) || scratched(c, parent, c->cfg.max_seqs)) return SEMKV_EINVAL;
  return launch_paged_fork(view(c), parent, stream);
}

int semkv_paged_compact(semkv_paged* c, const int32_t* keep, int64_t ld_keep, const int32_t* n_keep, hipStream_t stream) {
  if (!c || !n_keep || ld_keep < 0 || (ld_keep > 0 && !keep)) return SEMKV_EINVAL;
  if ((uintptr_t(keep) | uintptr_t(n_keep)) & 3) return SEMKV_EINVAL;
  const int64_t ld = ld_keep < (int64_t(1) << 40) ? ld_keep : int64_t(1) << 40;
  if (scratched(c, keep, ld * c->cfg.max_seqs) || scratched(c, n_keep, c->cfg.max_seqs)) return SEMKV_EINVAL;
  return launch_paged_compact(view(c), keep, ld_keep, n_keep, stream);
}

int semkv_paged_write(semkv_paged* c, int32_t layer, const void* K, const void* V, int32_t dtype, int64_t sL, int64_t sT,
                      int64_t sH, const int32_t* starts, int32_t n_seqs, int64_t n_rows, hipStream_t stream) {
  if (!c || !layer_ok(c, layer, -1)) return SEMKV_EINVAL;
  if (dtype != SEMKV_DTYPE_F16 && dtype != SEMKV_DTYPE_BF16) return SEMKV_EINVAL;
  PagedWriteArgs a;
  memset(&a, 0, sizeof(a));
  const int st = rows_of(c, starts, n_seqs, n_rows, &a.r);
  if (st) return st < 0 ? st : SEMKV_OK;
  if (!K || !V || ((uintptr_t(K) | uintptr_t(V)) & 15) || ((sT | sH | (layer < 0 ? sL : 0)) & 7)) return SEMKV_EINVAL;
  a.c = view(c);
  a.K = static_cast<const uint16_t*>(K);
  a.V = static_cast<const uint16_t*>(V);
  a.sL = sL;
  a.sT = sT;
  a.sH = sH;
  a.layer0 = layer < 0 ? 0 : layer;
  a.layers = layer < 0 ? c->cfg.n_layers : 1;
  a.bf16 = dtype == SEMKV_DTYPE_BF16;
  return launch_paged_write(a, stream);
}

int semkv_paged_read(const semkv_paged* c, int32_t layer, void* K, void* V, int32_t dtype, const int32_t* starts,
                     int32_t n_seqs, int64_t n_rows, hipStream_t stream) {
  if (!c || !layer_ok(c, layer, -1)) return SEMKV_EINVAL;
  if (dtype != SEMKV_DTYPE_F16 && dtype != SEMKV_DTYPE_BF16 && dtype != SEMKV_DTYPE_F32) return SEMKV_EINVAL;
  PagedReadArgs a;
  memset(&a, 0, sizeof(a));
  const int st = rows_of(c, starts, n_seqs, n_rows, &a.r);
  if (st) return st < 0 ? st : SEMKV_OK;
  if (!K || !V || ((uintptr_t(K) | uintptr_t(V)) & 15)) return SEMKV_EINVAL;
  a.c = view(c);
  a.K = K;
  a.V = V;
  a.layer0 = layer < 0 ? 0 : layer;
  a.layers = layer < 0 ? c->cfg.n_layers : 1;
  a.dtype = dtype;
  return launch_paged_read(a, stream);
}

int semkv_paged_attn(const semkv_paged* c, int32_t layer, const void* q, int32_t dtype, int64_t sT, int64_t sH,
                     float scale, const int32_t* starts, int32_t n_seqs, int64_t n_rows, void* out, float* lse,
                     void* workspace, size_t ws_bytes, hipStream_t stream) {
  if (!c || !layer_ok(c, layer, 0)) return SEMKV_EINVAL;
  if (dtype != SEMKV_DTYPE_F16 && dtype != SEMKV_DTYPE_BF16) return SEMKV_EINVAL;
  if (!(scale > 0.0f) || !isfinite(scale)) return SEMKV_EINVAL;
  PagedAttnArgs a;
  memset(&a, 0, sizeof(a));
  const int st = rows_of(c, starts, n_seqs, n_rows, &a.r);
  if (st) return st < 0 ? st : SEMKV_OK;
  if (!q || !out || !workspace) return SEMKV_EINVAL;
  if (((uintptr_t(q) | uintptr_t(out) | uintptr_t(workspace)) & 15) || (uintptr_t(lse) & 3) || ((sT | sH) & 7))
    return SEMKV_EINVAL;
  a.c = view(c);
  a.q = static_cast<const uint16_t*>(q);
  a.sT = sT;
  a.sH = sH;
  a.layer = layer;
  a.bf16 = dtype == SEMKV_DTYPE_BF16;
  a.gqa = c->cfg.n_q_heads / c->cfg.n_kv_heads;
  a.scale_log2e = float(double(scale) * 1.4426950408889634);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.ws = static_cast<float*>(workspace);
  return launch_paged_attn(a, ws_bytes, stream);
}

int semkv_token_logprobs_workspace(int64_t rows, int64_t vocab, int32_t top, size_t* bytes) {
  if (!bytes || rows < 0 || vocab < 1 || top < 0 || top > 32 || top > vocab) return SEMKV_EINVAL;
  *bytes = rows == 0 ? 0 : token_logprobs_workspace(rows, vocab, top);
  return SEMKV_OK;
}

int semkv_token_logprobs(const void* logits, int32_t dtype, int32_t batch, int64_t T, int64_t vocab, int64_t s_batch,
                         int64_t s_token, const int64_t* targets, int64_t t_batch, int64_t t_token, int32_t negate,
                         float* logp, float* entropy, int64_t o_batch, int64_t o_token, int32_t top, float* top_logp,
                         int32_t* top_ids, void* workspace, size_t ws_bytes, hipStream_t stream) {
  if (dtype != SEMKV_DTYPE_F16 && dtype != SEMKV_DTYPE_BF16 && dtype != SEMKV_DTYPE_F32) return SEMKV_EINVAL;
  if (batch < 0 || T < 0 || vocab < 1 || top < 0 || top > 32 || top > vocab) return SEMKV_EINVAL;
  if (batch == 0 || T == 0) return SEMKV_OK;
  if (vocab > INT32_MAX || T > kMaxRows || batch > kMaxRows / T) return SEMKV_EUNSUPPORTED;   // one workgroup a row
  if (!logits || (logp && !targets) || (top > 0 && (!top_logp || !top_ids))) return SEMKV_EINVAL;
  if (uintptr_t(logits) & (dtype == SEMKV_DTYPE_F32 ? 3 : 1)) return SEMKV_EINVAL;
  if ((uintptr_t(logp) | uintptr_t(entropy) | uintptr_t(top_logp) | uintptr_t(top_ids) | uintptr_t(workspace)) & 3) return SEMKV_EINVAL;
  if (uintptr_t(targets) & 7) return SEMKV_EINVAL;
  const size_t need = token_logprobs_workspace(int64_t(batch) * T, vocab, top);
  if (need && (!workspace || ws_bytes < need)) return SEMKV_EINVAL;
  TokenArgs a;
  memset(&a, 0, sizeof(a));
  a.x = logits;
  a.dtype = dtype;
  a.batch = batch;
  a.top = top;
  a.negate = negate != 0;
  a.T = T;
  a.vocab = vocab;
  a.s_batch = s_batch;
  a.s_token = s_token;
  a.targets = targets;
  a.t_batch = t_batch;
  a.t_token = t_token;
  a.logp = logp;
  a.entropy = entropy;
  a.o_batch = o_batch;
  a.o_token = o_token;
  a.top_logp = top_logp;
  a.top_ids = top_ids;
  a.ws = static_cast<float*>(workspace);
  return launch_token_logprobs(a, stream);
}

}  // extern "C"
