// paged_api.hip -- host side of the paged caches (4-bit, latents), of token scoring
// and of beam search's choice: validation, buffer geometry and launches.  Nothing
// here allocates or synchronizes.
#include <math.h>
#include <string.h>

#include "paged.h"
#include "semkv.h"

using namespace semkv;

namespace {

int64_t round64(int64_t words) { return (words + 63) / 64 * 64; }

// The parts that both kinds of cache have.
template <class C>
PagedView common_view(const C* c) {
  PagedView v;
  memset(&v, 0, sizeof(v));
  const auto& k = c->cfg;
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
  v.n_pages = k.n_pages;
  v.max_seqs = k.max_seqs;
  v.seq_pages = k.seq_pages;
  v.record = int32_t(c->sz.record_bytes);
  return v;
}

PagedView view(const semkv_paged* c) {
  PagedView v = common_view(c);
  v.n_kv_heads = c->cfg.n_kv_heads;
  v.dim = c->cfg.head_dim;
  v.group = c->cfg.group;
  return v;
}

PagedView view(const semkv_latent* c) {
  PagedView v = common_view(c);
  v.n_kv_heads = 1;
  v.latent = c->cfg.latent;
  v.rope = c->cfg.rope;
  return v;
}

// The rows of a call: 0 if they can be, 1 if there is none, else a status.
template <class C>
int rows_of(const C* c, const int32_t* starts, int32_t n_seqs, int64_t n_rows, PagedRows* r) {
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
template <class C>
bool inside(const C* c, const int32_t* p, int64_t n, int64_t word, int64_t end) {
  const uintptr_t a = uintptr_t(p), state = uintptr_t(c->state);
  return n > 0 && a < state + 4 * end && a + 4 * n > state + 4 * word;
}

// An argument of reserve, fork or compact in what follows the tables, which
// their kernels write while others of their workgroups still read arguments.
// (Lengths and tables are written last: an argument may lie there.)
template <class C>
bool scratched(const C* c, const int32_t* p, int64_t n) {
  return inside(c, p, n, c->sz.refs_word, int64_t(c->sz.state_bytes / 4));
}

constexpr int64_t kMaxRows = (int64_t(1) << 24) - 1;

template <class C>
bool layer_ok(const C* c, int32_t layer, int32_t least) { return layer >= least && layer < c->cfg.n_layers; }

// What sizes have in common: of pages of page_bytes, and the state.
int common_sizes(int32_t n_pages, int32_t max_seqs, int32_t seq_pages, int64_t page_bytes, semkv_paged_sizes* out) {
  if (n_pages > (1 << 20) || max_seqs > kMaxSeqs || seq_pages > (1 << 20)) return SEMKV_EUNSUPPORTED;
  if (int64_t(max_seqs) * seq_pages > (int64_t(1) << 28)) return SEMKV_EUNSUPPORTED;
  out->page_bytes = page_bytes;
  out->pool_bytes = size_t(page_bytes) * n_pages;
  const int64_t table = round64(int64_t(max_seqs) * seq_pages), seqs = round64(max_seqs), pages = round64(n_pages);
  out->lens_word = 64;
  out->table_word = out->lens_word + seqs;
  out->refs_word = out->table_word + table;
  out->free_word = out->refs_word + pages;
  out->scratch_word = out->free_word + round64((n_pages + 31) / 32);
  out->state_bytes = size_t(out->scratch_word + 5 * seqs + pages + table) * 4;
  return SEMKV_OK;
}

template <class C, class K>
int init(C* c, const K* cfg, const semkv_paged_sizes& sz, void* pool, int32_t* state, int32_t* status, hipStream_t stream) {
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

template <class C>
int assign(C* c, const int32_t* lens, const int32_t* table, hipStream_t stream) {
  if (!c || !lens || !table) return SEMKV_EINVAL;
  if ((uintptr_t(lens) | uintptr_t(table)) & 3) return SEMKV_EINVAL;
  const PagedView v = view(c);
  const int64_t end = int64_t(c->sz.state_bytes / 4);
  if (lens != v.lens && inside(c, lens, v.max_seqs, 0, end)) return SEMKV_EINVAL;
  if (table != v.table && inside(c, table, int64_t(v.max_seqs) * v.seq_pages, 0, end)) return SEMKV_EINVAL;
  return launch_paged_assign(v, lens, table, stream);
}

template <class C>
int reserve(C* c, const int32_t* n_new, hipStream_t stream) {
  if (!c || !n_new || (uintptr_t(n_new) & 3) || scratched(c, n_new, c->cfg.max_seqs)) return SEMKV_EINVAL;
  return launch_paged_reserve(view(c), n_new, stream);
}

template <class C>
int fork(C* c, const int32_t* parent, hipStream_t stream) {
  if (!c || !parent || (uintptr_t(parent) & 3) || scratched(c, parent, c->cfg.max_seqs)) return SEMKV_EINVAL;
  return launch_paged_fork(view(c), parent, stream);
}

template <class C>
int compact(C* c, const int32_t* keep, int64_t ld_keep, const int32_t* n_keep, hipStream_t stream) {
  if (!c || !n_keep || ld_keep < 0 || (ld_keep > 0 && !keep)) return SEMKV_EINVAL;
  if ((uintptr_t(keep) | uintptr_t(n_keep)) & 3) return SEMKV_EINVAL;
  const int64_t ld = ld_keep < (int64_t(1) << 40) ? ld_keep : int64_t(1) << 40;
  if (scratched(c, keep, ld * c->cfg.max_seqs) || scratched(c, n_keep, c->cfg.max_seqs)) return SEMKV_EINVAL;
  return launch_paged_compact(view(c), keep, ld_keep, n_keep, stream);
}

// Whether a rotation of heads of `dim` channels can be: 0, or a status.
int rotary_of(const semkv_rotary* rot, int32_t dim, RotaryArgs* out) {
  if (!rot || !rot->freqs || ((uintptr_t(rot->freqs) | uintptr_t(rot->positions)) & 3)) return SEMKV_EINVAL;
  if (rot->dim < 16 || rot->dim > dim || rot->dim % 16) return SEMKV_EUNSUPPORTED;
  out->freqs = rot->freqs;
  out->positions = rot->positions;
  out->dim = rot->dim;
  out->interleaved = rot->interleaved != 0;
  return SEMKV_OK;
}

// Queries that an append turns: both places given, aligned, or neither.
bool queries_ok(const void* q, int64_t qT, int64_t qH, const void* out, int64_t oT, int64_t oH) {
  if (!q) return true;
  return out && !((uintptr_t(q) | uintptr_t(out)) & 15) && !((qT | qH | oT | oH) & 7);
}

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
  if (int64_t(k.n_layers) * k.n_kv_heads > 65535) return SEMKV_EUNSUPPORTED;
  memset(out, 0, sizeof(*out));
  const int record = paged_record(k.head_dim, k.group);
  const int st = common_sizes(k.n_pages, k.max_seqs, k.seq_pages, int64_t(record) * k.n_layers * k.n_kv_heads, out);
  if (st) return st;
  out->record_bytes = record;
  out->workspace_bytes = paged_attn_workspace(k.head_dim);
  return SEMKV_OK;
}

int semkv_paged_init(semkv_paged* c, const semkv_paged_config* cfg, void* pool, int32_t* state, int32_t* status,
                     hipStream_t stream) {
  if (!c || !cfg) return SEMKV_EINVAL;
  semkv_paged_sizes sz;
  const int st = semkv_paged_cache_sizes(cfg, &sz);
  if (st) return st;
  return init(c, cfg, sz, pool, state, status, stream);
}

int semkv_paged_assign(semkv_paged* c, const int32_t* lens, const int32_t* table, hipStream_t stream) {
  return assign(c, lens, table, stream);
}

int semkv_paged_reserve(semkv_paged* c, const int32_t* n_new, hipStream_t stream) { return reserve(c, n_new, stream); }

int semkv_paged_fork(semkv_paged* c, const int32_t* parent, hipStream_t stream) { return fork(c, parent, stream); }

int semkv_paged_compact(semkv_paged* c, const int32_t* keep, int64_t ld_keep, const int32_t* n_keep, hipStream_t stream) {
  return compact(c, keep, ld_keep, n_keep, stream);
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

int semkv_paged_append(semkv_paged* c, int32_t layer, const void* K, const void* V, int32_t dtype, int64_t sT, int64_t sH,
                       const void* q, int64_t qT, int64_t qH, void* q_out, int64_t oT, int64_t oH, const semkv_rotary* rot,
                       const int32_t* starts, int32_t n_seqs, int64_t n_rows, hipStream_t stream) {
  if (!c || !layer_ok(c, layer, 0)) return SEMKV_EINVAL;
  if (dtype != SEMKV_DTYPE_F16 && dtype != SEMKV_DTYPE_BF16) return SEMKV_EINVAL;
  PagedAppendArgs a;
  memset(&a, 0, sizeof(a));
  int st = rotary_of(rot, c->cfg.head_dim, &a.rot);
  if (st) return st;
  st = rows_of(c, starts, n_seqs, n_rows, &a.w.r);
  if (st) return st < 0 ? st : SEMKV_OK;
  if (!K || !V || ((uintptr_t(K) | uintptr_t(V)) & 15) || ((sT | sH) & 7)) return SEMKV_EINVAL;
  if (!queries_ok(q, qT, qH, q_out, oT, oH)) return SEMKV_EINVAL;
  a.w.c = view(c);
  a.w.K = static_cast<const uint16_t*>(K);
  a.w.V = static_cast<const uint16_t*>(V);
  a.w.sT = sT;
  a.w.sH = sH;
  a.w.layer0 = layer;
  a.w.layers = 1;
  a.w.bf16 = dtype == SEMKV_DTYPE_BF16;
  a.q = static_cast<const uint16_t*>(q);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.qT = qT;
  a.qH = qH;
  a.oT = oT;
  a.oH = oH;
  a.gqa = c->cfg.n_q_heads / c->cfg.n_kv_heads;
  return launch_paged_append(a, stream);
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

int semkv_latent_cache_sizes(const semkv_latent_config* cfg, semkv_paged_sizes* out) {
  if (!cfg || !out) return SEMKV_EINVAL;
  const semkv_latent_config& k = *cfg;
  if (k.n_layers < 1 || k.n_heads < 1 || k.n_pages < 1 || k.max_seqs < 1 || k.seq_pages < 1) return SEMKV_EINVAL;
  if (k.dtype != SEMKV_DTYPE_F16 && k.dtype != SEMKV_DTYPE_BF16) return SEMKV_EINVAL;
  if ((k.latent != 256 && k.latent != 512) || (k.rope != 32 && k.rope != 64)) return SEMKV_EUNSUPPORTED;
  if (k.n_heads > 128 || k.n_layers > 65535) return SEMKV_EUNSUPPORTED;
  memset(out, 0, sizeof(*out));
  const int record = 2 * kPage * (k.latent + k.rope);
  const int st = common_sizes(k.n_pages, k.max_seqs, k.seq_pages, int64_t(record) * k.n_layers, out);
  if (st) return st;
  out->record_bytes = record;
  out->workspace_bytes = latent_attn_workspace(k.latent);
  return SEMKV_OK;
}

int semkv_latent_init(semkv_latent* c, const semkv_latent_config* cfg, void* pool, int32_t* state, int32_t* status,
                      hipStream_t stream) {
  if (!c || !cfg) return SEMKV_EINVAL;
  semkv_paged_sizes sz;
  const int st = semkv_latent_cache_sizes(cfg, &sz);
  if (st) return st;
  return init(c, cfg, sz, pool, state, status, stream);
}

int semkv_latent_assign(semkv_latent* c, const int32_t* lens, const int32_t* table, hipStream_t stream) {
  return assign(c, lens, table, stream);
}

int semkv_latent_reserve(semkv_latent* c, const int32_t* n_new, hipStream_t stream) { return reserve(c, n_new, stream); }

int semkv_latent_fork(semkv_latent* c, const int32_t* parent, hipStream_t stream) { return fork(c, parent, stream); }

int semkv_latent_compact(semkv_latent* c, const int32_t* keep, int64_t ld_keep, const int32_t* n_keep, hipStream_t stream) {
  return compact(c, keep, ld_keep, n_keep, stream);
}

int semkv_latent_append(semkv_latent* c, int32_t layer, const void* C, int64_t cT, const void* R, int64_t rT, const void* q,
                        int64_t qT, int64_t qH, void* q_out, int64_t oT, int64_t oH, const semkv_rotary* rot,
                        const int32_t* starts, int32_t n_seqs, int64_t n_rows, hipStream_t stream) {
  if (!c || !layer_ok(c, layer, 0)) return SEMKV_EINVAL;
  LatentAppendArgs a;
  memset(&a, 0, sizeof(a));
  int st = rotary_of(rot, c->cfg.rope, &a.rot);
  if (st) return st;
  st = rows_of(c, starts, n_seqs, n_rows, &a.r);
  if (st) return st < 0 ? st : SEMKV_OK;
  if (!C || !R || ((uintptr_t(C) | uintptr_t(R)) & 15) || ((cT | rT) & 7)) return SEMKV_EINVAL;
  if (!queries_ok(q, qT, qH, q_out, oT, oH)) return SEMKV_EINVAL;
  a.c = view(c);
  a.C = static_cast<const uint16_t*>(C);
  a.R = static_cast<const uint16_t*>(R);
  a.cT = cT;
  a.rT = rT;
  a.q = static_cast<const uint16_t*>(q);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.qT = qT;
  a.qH = qH;
  a.oT = oT;
  a.oH = oH;
  a.n_heads = c->cfg.n_heads;
  a.layer = layer;
  a.bf16 = c->cfg.dtype == SEMKV_DTYPE_BF16;
  return launch_latent_append(a, stream);
}

int semkv_latent_read(const semkv_latent* c, int32_t layer, void* C, void* R, const int32_t* starts, int32_t n_seqs,
                      int64_t n_rows, hipStream_t stream) {
  if (!c || !layer_ok(c, layer, 0)) return SEMKV_EINVAL;
  LatentReadArgs a;
  memset(&a, 0, sizeof(a));
  const int st = rows_of(c, starts, n_seqs, n_rows, &a.r);
  if (st) return st < 0 ? st : SEMKV_OK;
  if (!C || !R || ((uintptr_t(C) | uintptr_t(R)) & 15)) return SEMKV_EINVAL;
  a.c = view(c);
  a.C = static_cast<uint16_t*>(C);
  a.R = static_cast<uint16_t*>(R);
  a.layer = layer;
  return launch_latent_read(a, stream);
}

int semkv_latent_attn(const semkv_latent* c, int32_t layer, const void* q, int64_t qT, int64_t qH, const void* q_rope, int64_t rT,
                      int64_t rH, float scale, const int32_t* starts, int32_t n_seqs, int64_t n_rows, void* out, float* lse,
                      void* workspace, size_t ws_bytes, hipStream_t stream) {
  if (!c || !layer_ok(c, layer, 0)) return SEMKV_EINVAL;
  if (!(scale > 0.0f) || !isfinite(scale)) return SEMKV_EINVAL;
  LatentAttnArgs a;
  memset(&a, 0, sizeof(a));
  const int st = rows_of(c, starts, n_seqs, n_rows, &a.r);
  if (st) return st < 0 ? st : SEMKV_OK;
  if (!q || !q_rope || !out || !workspace) return SEMKV_EINVAL;
  if (((uintptr_t(q) | uintptr_t(q_rope) | uintptr_t(out) | uintptr_t(workspace)) & 15) || (uintptr_t(lse) & 3)) return SEMKV_EINVAL;
  if ((qT | qH | rT | rH) & 7) return SEMKV_EINVAL;
  a.c = view(c);
  a.q = static_cast<const uint16_t*>(q);
  a.q_rope = static_cast<const uint16_t*>(q_rope);
  a.qT = qT;
  a.qH = qH;
  a.rT = rT;
  a.rH = rH;
  a.n_heads = c->cfg.n_heads;
  a.layer = layer;
  a.bf16 = c->cfg.dtype == SEMKV_DTYPE_BF16;
  a.scale_log2e = float(double(scale) * 1.4426950408889634);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.ws = static_cast<float*>(workspace);
  return launch_latent_attn(a, ws_bytes, stream);
}

int semkv_beam_select_workspace(int64_t groups, int32_t width, int64_t vocab, int32_t k, size_t* bytes) {
  if (!bytes || groups < 0 || width < 1 || vocab < 1 || k < 1) return SEMKV_EINVAL;
  if (width > 64 || k > 64 || vocab > INT32_MAX || groups > kMaxRows / width) return SEMKV_EUNSUPPORTED;
  *bytes = groups == 0 ? 0 : beam_select_workspace(groups * width, vocab, k);
  return SEMKV_OK;
}

int semkv_beam_select(const void* logits, int32_t dtype, int64_t groups, int32_t width, int64_t vocab, int64_t s_group,
                      int64_t s_beam, const float* scores, const int32_t* ended, int32_t pad, int32_t k, float* out_scores,
                      int32_t* parents, int32_t* tokens, void* workspace, size_t ws_bytes, hipStream_t stream) {
  if (dtype != SEMKV_DTYPE_F16 && dtype != SEMKV_DTYPE_BF16 && dtype != SEMKV_DTYPE_F32) return SEMKV_EINVAL;
  size_t need;
  const int st = semkv_beam_select_workspace(groups, width, vocab, k, &need);
  if (st) return st;
  if (groups == 0) return SEMKV_OK;
  if (!logits || !scores || !out_scores || !parents || !tokens || !workspace || ws_bytes < need) return SEMKV_EINVAL;
  if (uintptr_t(logits) & (dtype == SEMKV_DTYPE_F32 ? 3 : 1)) return SEMKV_EINVAL;
  if ((uintptr_t(scores) | uintptr_t(ended) | uintptr_t(out_scores) | uintptr_t(parents) | uintptr_t(tokens)) & 3) return SEMKV_EINVAL;
  if (uintptr_t(workspace) & 15) return SEMKV_EINVAL;
  BeamArgs a;
  memset(&a, 0, sizeof(a));
  a.x = logits;
  a.dtype = dtype;
  a.width = width;
  a.k = k;
  a.pad = pad;
  a.groups = groups;
  a.vocab = vocab;
  a.s_group = s_group;
  a.s_beam = s_beam;
  a.scores = scores;
  a.ended = ended;
  a.out_scores = out_scores;
  a.parents = parents;
  a.tokens = tokens;
  a.ws = static_cast<float*>(workspace);
  return launch_beam_select(a, stream);
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
