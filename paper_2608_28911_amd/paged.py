"""Python binding of the paged 4-bit cache and of token scoring.

As the rest of the binding it only marshals arguments: torch supplies device
memory and the current stream, the library's kernels do the work.  Calls
enqueue on the current stream of the cache's device and read nothing back, so
they can be captured into graphs.
"""
import ctypes
import functools

from . import _abi
from ._abi import check, lib

_DTYPES = None


def _code(dtype, what, floats=False):
    """The library's code of a torch dtype; fp32 only where it is taken."""
    global _DTYPES
    if _DTYPES is None:
        import torch
        _DTYPES = {torch.float16: _abi.DTYPE_F16, torch.bfloat16: _abi.DTYPE_BF16, torch.float32: _abi.DTYPE_F32}
    code = _DTYPES.get(dtype)
    if code is None or (code == _abi.DTYPE_F32 and not floats):
        raise ValueError("%s: dtype %s is not supported" % (what, dtype))
    return code


def _need(ok, what, *args):
    if not ok:
        raise ValueError(what % tuple(list(a) if isinstance(a, tuple) else a for a in args))


def _int32():
    if _torch is None:
        _setup()
    return _torch.int32


_torch = None


def _setup():
    """torch's functions that every call needs, looked up once: the current
    device, and a device's current stream as an integer.  _torch says that they
    are there, and is set last: another thread may be looking."""
    global _torch, _device, _stream_of
    import torch
    _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _stream_of = raw or (lambda i: torch.cuda.current_stream(i).cuda_stream)
    _torch = torch


def _enqueue(index, f, what, *args):
    """f(*args, stream) with device `index` current, on its current stream."""
    _need(index >= 0, "%s: the buffers must be on a GPU", what)
    if _torch is None:
        _setup()
    if _device() == index:
        st = f(*args, _stream_of(index))
    else:
        with _torch.cuda.device(index):
            st = f(*args, _stream_of(index))
    if st:
        check(st, what)


def make_paged_config(n_layers, n_kv_heads, n_q_heads, n_pages, max_seqs, seq_pages, head_dim=128,
                      group=128) -> _abi.PagedConfig:
    return _abi.PagedConfig(n_layers=n_layers, n_kv_heads=n_kv_heads, n_q_heads=n_q_heads, head_dim=head_dim, group=group,
                            n_pages=n_pages, max_seqs=max_seqs, seq_pages=seq_pages)


def paged_sizes(cfg: _abi.PagedConfig) -> _abi.PagedSizes:
    s = _abi.PagedSizes()
    check(lib().semkv_paged_cache_sizes(ctypes.byref(cfg), ctypes.byref(s)), "semkv_paged_cache_sizes")
    return s


class PagedKV4:
    """A KV cache held in 4 bits, in pages of 64 tokens, for sequences of their
    own lengths (include/semkv.h says what each call does).

    The pool may be given (uint8, pool_bytes of paged_sizes(cfg), any shape):
    a program then keeps its own view of the pages.  Every other buffer is the
    cache's; the workspace has its full size from the start, so that a graph
    that holds its address stays valid."""

    def __init__(self, cfg: _abi.PagedConfig, pool=None, device="cuda"):
        import torch
        self.cfg = cfg
        self.sz = z = paged_sizes(cfg)
        dev = pool.device if pool is not None else torch.device(device)
        if dev.type == "cuda" and dev.index is None:
            dev = torch.device("cuda", torch.cuda.current_device())
        self.device = dev
        self._at = dev.index if dev.type == "cuda" else -1    # as Tensor.get_device() says it
        if pool is None:
            pool = torch.empty(z.pool_bytes, dtype=torch.uint8, device=dev)
        _need(pool.dtype == torch.uint8 and pool.is_contiguous() and pool.numel() == z.pool_bytes,
              "pool: contiguous uint8 of %d bytes" % z.pool_bytes)
        self.pool = pool
        self.state = s = torch.zeros(z.state_bytes // 4, dtype=torch.int32, device=dev)
        self.status_word = torch.zeros(4, dtype=torch.int32, device=dev)
        self.ws = torch.zeros(z.workspace_bytes // 4, dtype=torch.float32, device=dev)
        self.c = _abi.Paged()
        self._ref = ctypes.byref(self.c)
        self._lib = lib()
        # what every call reads of the configuration, as plain integers
        self._layers, self._heads, self._q_heads, self._dim = cfg.n_layers, cfg.n_kv_heads, cfg.n_q_heads, cfg.head_dim
        self._seqs, self._width, self._scale = cfg.max_seqs, cfg.seq_pages, cfg.head_dim ** -0.5
        _enqueue(self._at, self._lib.semkv_paged_init, "semkv_paged_init", self._ref, ctypes.byref(cfg), pool.data_ptr(),
                 s.data_ptr(), self.status_word.data_ptr())
        self.lens = s[z.lens_word:z.lens_word + self._seqs]               # tokens of each slot
        self.table = s[z.table_word:z.table_word + self._seqs * self._width].view(self._seqs, self._width)  # its pages, -1: none
        self.refs = s[z.refs_word:z.refs_word + cfg.n_pages]              # table entries that name a page
        self.stalled = s[:1]                                              # not 0: the last reserve failed

    # -- checks ------------------------------------------------------------
    def _ints(self, t, what, *shape):
        _need(t.dtype == _int32() and t.get_device() == self._at and t.shape == shape and t.is_contiguous(),
              "%s: contiguous int32 of shape %s on %s", what, shape, self.device)
        return t.data_ptr()

    def _starts(self, t):
        n = t.numel()
        _need(t.dtype == _int32() and t.get_device() == self._at and t.dim() == 1 and t.is_contiguous()
              and 1 <= n <= self._seqs + 1, "starts: contiguous int32 of n_seqs + 1 values on %s", self.device)
        return t.data_ptr(), n - 1

    # -- pages -------------------------------------------------------------
    def assign(self, lens, table):
        """Take over lengths [max_seqs] and page tables [max_seqs, seq_pages], int32; either may be the cache's own
        (shorter lengths over self.table drop the sequences' last tokens)."""
        _enqueue(self._at, self._lib.semkv_paged_assign, "semkv_paged_assign", self._ref,
                 self._ints(lens, "lens", self._seqs), self._ints(table, "table", self._seqs, self._width))

    def reserve(self, n_new):
        """Room for n_new [max_seqs] (int32) more tokens of every slot."""
        _enqueue(self._at, self._lib.semkv_paged_reserve, "semkv_paged_reserve", self._ref,
                 self._ints(n_new, "n_new", self._seqs))

    def fork(self, parent):
        """Slot s takes over slot parent[s]'s contents (int32 [max_seqs]); its own number keeps it, -1 empties it."""
        _enqueue(self._at, self._lib.semkv_paged_fork, "semkv_paged_fork", self._ref,
                 self._ints(parent, "parent", self._seqs))

    def compact(self, keep, n_keep):
        """Slot s keeps tokens keep[s, :n_keep[s]] only (int32 [max_seqs, W] and [max_seqs]); -1 leaves it alone."""
        _need(keep.dim() == 2, "keep: [max_seqs, W]")
        width = keep.shape[1]
        _enqueue(self._at, self._lib.semkv_paged_compact, "semkv_paged_compact", self._ref,
                 self._ints(keep, "keep", self._seqs, width), width, self._ints(n_keep, "n_keep", self._seqs))

    # -- rows --------------------------------------------------------------
    def write(self, layer, K, V, starts):
        """Quantize K, V [n, n_kv_heads, head_dim] (layer = -1: [n_layers, n, ...]; fp16 or bf16, a unit channel
        stride) into the pages of the sequences' last tokens: sequence s has rows starts[s] .. starts[s+1]-1."""
        code = _code(K.dtype, "K")
        lead = 1 if layer < 0 else 0
        shape, st = K.shape, K.stride()
        _need(V.dtype == K.dtype and V.shape == shape and V.stride() == st
              and K.get_device() == V.get_device() == self._at
              and len(shape) == 3 + lead and shape[-2] == self._heads and shape[-1] == self._dim and st[-1] == 1
              and (not lead or shape[0] == self._layers),
              "K, V: [%sn, %d, %d] alike, with a unit channel stride, on %s",
              "%d, " % self._layers if lead else "", self._heads, self._dim, self.device)
        at, n_seqs = self._starts(starts)
        _enqueue(self._at, self._lib.semkv_paged_write, "semkv_paged_write", self._ref, layer, K.data_ptr(), V.data_ptr(),
                 code, st[0] if lead else 0, st[-3], st[-2], at, n_seqs, shape[-3])

    def read(self, layer, starts, n_rows, dtype=None, out=None):
        """The values that the pages hold for the sequences' last tokens: K, V [n_rows, n_kv_heads, head_dim] in
        `dtype` (fp16 if not given), with layer = -1 [n_layers, n_rows, ...]."""
        import torch
        shape = (n_rows, self._heads, self._dim) if layer >= 0 else (self._layers, n_rows, self._heads, self._dim)
        if out is None:
            code = _code(torch.float16 if dtype is None else dtype, "dtype", True)
            K = torch.empty(shape, dtype=torch.float16 if dtype is None else dtype, device=self.device)
            V = torch.empty_like(K)
        else:
            K, V = out
            code = _code(K.dtype, "out", True)
            _need(K.dtype == V.dtype and K.shape == V.shape == shape and K.is_contiguous() and V.is_contiguous()
                  and K.get_device() == V.get_device() == self._at and dtype in (None, K.dtype),
                  "out: two contiguous tensors of shape %s on %s", shape, self.device)
        at, n_seqs = self._starts(starts)
        _enqueue(self._at, self._lib.semkv_paged_read, "semkv_paged_read", self._ref, layer, K.data_ptr(), V.data_ptr(),
                 code, at, n_seqs, n_rows)
        return K, V

    def attn(self, layer, q, starts, scale=None, out=None, lse=None, with_lse=False, workspace=None):
        """Causal attention of the sequences' last tokens over their pages: q [n, n_q_heads, head_dim] (fp16 or bf16,
        a unit channel stride) -> out of q's shape and dtype; with_lse: (out, lse fp32 [n, n_q_heads]).  scale:
        1/sqrt(head_dim) if not given.  Calls that overlap in time need a workspace each (like cache.ws, zeroed once).
        Large chunks and single tokens of other, long sequences are faster in a call of their own each."""
        import torch
        code = _code(q.dtype, "q")
        shape, st = q.shape, q.stride()
        _need(len(shape) == 3 and shape[1] == self._q_heads and shape[2] == self._dim and st[2] == 1
              and q.get_device() == self._at,
              "q: [n, %d, %d] with a unit channel stride, on %s", self._q_heads, self._dim, self.device)
        if out is None:
            out = torch.empty(shape, dtype=q.dtype, device=self.device)
        else:
            _need(out.dtype == q.dtype and out.shape == shape and out.is_contiguous() and out.get_device() == self._at,
                  "out: contiguous, of q's shape and dtype")
        if lse is not None:
            with_lse = True
            _need(lse.dtype == torch.float32 and lse.shape == shape[:2] and lse.is_contiguous()
                  and lse.get_device() == self._at, "lse: contiguous fp32 [n, n_q_heads]")
        elif with_lse:
            lse = torch.empty(shape[:2], dtype=torch.float32, device=self.device)
        if workspace is None:
            ws = self.ws
        else:
            ws = workspace
            _need(ws.get_device() == self._at and ws.is_contiguous(), "workspace: contiguous, on %s", self.device)
        at, n_seqs = self._starts(starts)
        _enqueue(self._at, self._lib.semkv_paged_attn, "semkv_paged_attn", self._ref, layer, q.data_ptr(), code, st[0], st[1],
                 self._scale if scale is None else scale, at, n_seqs, shape[0], out.data_ptr(),
                 lse.data_ptr() if with_lse else None, ws.data_ptr(), ws.numel() * ws.element_size())
        return (out, lse) if with_lse else out

    # -- state -------------------------------------------------------------
    def status(self) -> int:
        return int(self.status_word[0].item())


@functools.lru_cache(maxsize=1024)
def _logprobs_workspace(rows, vocab, top):
    n = ctypes.c_size_t()
    check(lib().semkv_token_logprobs_workspace(rows, vocab, top, ctypes.byref(n)), "semkv_token_logprobs_workspace")
    return n.value


def _rows(t, what, shape, dtype, at):
    """Element strides of a [B, T] tensor (or [N]: one row of N)."""
    _need(t.dtype == dtype and t.shape == shape and t.get_device() == at, "%s: %s of shape %s on the logits' device",
          what, dtype, tuple(shape))
    st = t.stride()
    return st if len(shape) == 2 else (0, st[0])


def _logprobs(logits, targets, top, negate, logp, want_entropy):
    import torch
    code = _code(logits.dtype, "logits", True)
    shape, s, at, dev = logits.shape, logits.stride(), logits.get_device(), logits.device
    _need(len(shape) in (2, 3) and (s[-1] == 1 or shape[-1] == 1) and at >= 0,
          "logits: [N, V] or [B, T, V] with a unit stride over V, on a GPU")
    lead, V = shape[:-1], shape[-1]
    B, T, s_b, s_t = (lead[0], lead[1], s[0], s[1]) if len(lead) == 2 else (1, lead[0], 0, s[0])
    _need(V > 0 and 0 <= top <= 32 and top <= V, "top: 0 to 32, at most V")
    t_b, t_t = _rows(targets, "targets", lead, torch.int64, at)
    if logp is None:
        logp = torch.empty(lead, dtype=torch.float32, device=dev)
    o_b, o_t = _rows(logp, "scores", lead, torch.float32, at)
    entropy = torch.empty_like(logp) if want_entropy else None       # logp is dense then: the same strides
    top_logp = torch.empty((*lead, top), dtype=torch.float32, device=dev) if top else None
    top_ids = torch.empty((*lead, top), dtype=torch.int32, device=dev) if top else None
    n = _logprobs_workspace(B * T, V, top)
    ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    ptr = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
    _enqueue(at, lib().semkv_token_logprobs, "semkv_token_logprobs", logits.data_ptr(), code, B, T, V, s_b, s_t,
             targets.data_ptr(), t_b, t_t, negate, logp.data_ptr(), ptr(entropy), o_b, o_t, top, ptr(top_logp),
             ptr(top_ids), ptr(ws), n)
    return logp, entropy, top_logp, top_ids


def token_logprobs(logits, targets, top=0):
    """Log probabilities of given tokens: logits fp16, bf16 or fp32 [N, V] or [B, T, V] (any strides with a unit one
    over V), targets int64 [N] or [B, T] (-1: none, gives 0; another one outside [0, V): NaN) -> (logp, entropy), fp32
    of the targets' shape, and with top > 0 also (top_logp fp32, top_ids int32) [..., top]: the likeliest tokens,
    equal logits by lower index.  A row without a finite sum of exponentials gives NaN, and ids of -1."""
    logp, entropy, top_logp, top_ids = _logprobs(logits, targets, top, 0, None, True)
    return (logp, entropy, top_logp, top_ids) if top else (logp, entropy)


def score_tokens(logits, targets, scores=None):
    """Sec. 3.3 self-information -log p(target) of every token, the scores that semkv_rank takes: logits and targets as
    for token_logprobs.  scores: fp32 of the targets' shape, any strides (logits of position t predict token t+1:
    score_tokens(logits[:, :-1], ids[:, 1:], scores=s[:, 1:]))."""
    return _logprobs(logits, targets, 0, 1, scores, False)[0]
