"""Python binding of the paged 4-bit cache and of token scoring.

As the rest of the binding it only marshals arguments: torch supplies device
memory and the current stream, the library's kernels do the work.  Calls
enqueue on the current stream of the cache's device and read nothing back, so
they can be captured into graphs.
"""
import ctypes

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


def _need(ok, what):
    if not ok:
        raise ValueError(what)


class _On:
    """The device of a call made current, if it is not, and its current stream."""

    def __init__(self, device):
        import torch
        self.index = device.index if device.type == "cuda" else None
        self.back = None
        if self.index is not None and self.index != torch.cuda.current_device():
            self.back = torch.cuda.current_device()

    def __enter__(self):
        from . import _stream
        if self.back is not None:
            import torch
            torch.cuda.set_device(self.index)
        return _stream()

    def __exit__(self, *exc):
        if self.back is not None:
            import torch
            torch.cuda.set_device(self.back)


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
        self.sz = paged_sizes(cfg)
        dev = pool.device if pool is not None else torch.device(device)
        if dev.type == "cuda" and dev.index is None:
            dev = torch.device("cuda", torch.cuda.current_device())
        self.device = dev
        if pool is None:
            pool = torch.empty(self.sz.pool_bytes, dtype=torch.uint8, device=dev)
        _need(pool.dtype == torch.uint8 and pool.is_contiguous() and pool.numel() == self.sz.pool_bytes,
              "pool: contiguous uint8 of %d bytes" % self.sz.pool_bytes)
        self.pool = pool
        self.state = torch.zeros(self.sz.state_bytes // 4, dtype=torch.int32, device=dev)
        self.status_word = torch.zeros(4, dtype=torch.int32, device=dev)
        self.ws = torch.empty(self.sz.workspace_bytes // 4, dtype=torch.float32, device=dev)
        self.c = _abi.Paged()
        self._ref = ctypes.byref(self.c)
        self._lib = lib()
        with _On(dev) as stream:
            check(self._lib.semkv_paged_init(self._ref, ctypes.byref(cfg), pool.data_ptr(), self.state.data_ptr(),
                                             self.status_word.data_ptr(), stream), "semkv_paged_init")
        s, z = self.state, self.sz
        words = lambda at, *shape: s[at:at + _prod(shape)].view(shape)  # noqa: E731
        self.lens = words(z.lens_word, cfg.max_seqs)                      # tokens of each slot
        self.table = words(z.table_word, cfg.max_seqs, cfg.seq_pages)     # its pages, -1 where none
        self.refs = words(z.refs_word, cfg.n_pages)                       # table entries that name a page
        self.stalled = words(0, 1)                                        # not 0: the last reserve failed

    # -- checks ------------------------------------------------------------
    def _ints(self, t, what, *shape):
        import torch
        _need(t.dtype == torch.int32 and t.device == self.device and tuple(t.shape) == shape and t.is_contiguous(),
              "%s: contiguous int32 of shape %s on %s" % (what, list(shape), self.device))
        return t.data_ptr()

    def _starts(self, t):
        import torch
        _need(t.dtype == torch.int32 and t.device == self.device and t.dim() == 1 and t.is_contiguous()
              and 1 <= t.numel() <= self.cfg.max_seqs + 1,
              "starts: contiguous int32 of n_seqs + 1 values on %s" % self.device)
        return t.data_ptr(), t.numel() - 1

    # -- pages -------------------------------------------------------------
    def assign(self, lens, table):
        """Take over lengths [max_seqs] and page tables [max_seqs, seq_pages], int32."""
        cfg = self.cfg
        a, b = self._ints(lens, "lens", cfg.max_seqs), self._ints(table, "table", cfg.max_seqs, cfg.seq_pages)
        with _On(self.device) as stream:
            check(self._lib.semkv_paged_assign(self._ref, a, b, stream), "semkv_paged_assign")

    def reserve(self, n_new):
        """Room for n_new [max_seqs] (int32) more tokens of every slot."""
        a = self._ints(n_new, "n_new", self.cfg.max_seqs)
        with _On(self.device) as stream:
            check(self._lib.semkv_paged_reserve(self._ref, a, stream), "semkv_paged_reserve")

    def fork(self, parent):
        """Slot s takes over slot parent[s]'s contents (int32 [max_seqs]); its own number keeps it, -1 empties it."""
        a = self._ints(parent, "parent", self.cfg.max_seqs)
        with _On(self.device) as stream:
            check(self._lib.semkv_paged_fork(self._ref, a, stream), "semkv_paged_fork")

    def compact(self, keep, n_keep):
        """Slot s keeps tokens keep[s, :n_keep[s]] only (int32 [max_seqs, W] and [max_seqs]); -1 leaves it alone."""
        import torch
        _need(keep.dtype == torch.int32 and keep.device == self.device and keep.dim() == 2
              and keep.shape[0] == self.cfg.max_seqs and keep.is_contiguous(),
              "keep: contiguous int32 of shape [%d, W] on %s" % (self.cfg.max_seqs, self.device))
        a = self._ints(n_keep, "n_keep", self.cfg.max_seqs)
        with _On(self.device) as stream:
            check(self._lib.semkv_paged_compact(self._ref, keep.data_ptr(), keep.shape[1], a, stream),
                  "semkv_paged_compact")

    # -- rows --------------------------------------------------------------
    def write(self, layer, K, V, starts):
        """Quantize K, V [n, n_kv_heads, head_dim] (layer = -1: [n_layers, n, ...]; fp16 or bf16, a unit channel
        stride) into the pages of the sequences' last tokens: sequence s has rows starts[s] .. starts[s+1]-1."""
        cfg = self.cfg
        code = _code(K.dtype, "K")
        lead = 1 if layer < 0 else 0
        shape, st = K.shape, K.stride()
        _need(V.dtype == K.dtype and V.shape == shape and V.stride() == st and K.device == V.device == self.device
              and len(shape) == 3 + lead and shape[lead + 1] == cfg.n_kv_heads and shape[lead + 2] == cfg.head_dim
              and st[lead + 2] == 1 and (not lead or shape[0] == cfg.n_layers),
              "K, V: [%sn, %d, %d] alike, with a unit channel stride, on %s"
              % ("%d, " % cfg.n_layers if lead else "", cfg.n_kv_heads, cfg.head_dim, self.device))
        at, n_seqs = self._starts(starts)
        with _On(self.device) as stream:
            check(self._lib.semkv_paged_write(self._ref, layer, K.data_ptr(), V.data_ptr(), code, st[0] if lead else 0,
                                              st[lead], st[lead + 1], at, n_seqs, shape[lead], stream),
                  "semkv_paged_write")

    def read(self, layer, starts, n_rows, dtype=None, out=None):
        """The values that the pages hold for the sequences' last tokens: K, V [n_rows, n_kv_heads, head_dim] in
        `dtype` (fp16 if not given), with layer = -1 [n_layers, n_rows, ...]."""
        import torch
        cfg = self.cfg
        shape = (n_rows, cfg.n_kv_heads, cfg.head_dim)
        if layer < 0:
            shape = (cfg.n_layers,) + shape
        if out is None:
            dtype = torch.float16 if dtype is None else dtype
            K = torch.empty(shape, dtype=dtype, device=self.device)
            V = torch.empty_like(K)
        else:
            K, V = out
            _need(K.dtype == V.dtype and K.shape == V.shape == shape and K.is_contiguous() and V.is_contiguous()
                  and K.device == V.device == self.device and dtype in (None, K.dtype),
                  "out: two contiguous tensors of shape %s on %s" % (list(shape), self.device))
        at, n_seqs = self._starts(starts)
        with _On(self.device) as stream:
            check(self._lib.semkv_paged_read(self._ref, layer, K.data_ptr(), V.data_ptr(), _code(K.dtype, "out", True),
                                             at, n_seqs, n_rows, stream), "semkv_paged_read")
        return K, V

    def attn(self, layer, q, starts, scale=None, out=None, lse=None, with_lse=False, workspace=None):
        """Causal attention of the sequences' last tokens over their pages: q [n, n_q_heads, head_dim] (fp16 or bf16,
        a unit channel stride) -> out of q's shape and dtype; with_lse: (out, lse fp32 [n, n_q_heads]).  scale:
        1/sqrt(head_dim) if not given.  Calls that overlap in time need a workspace each."""
        import torch
        cfg = self.cfg
        code = _code(q.dtype, "q")
        shape, st = q.shape, q.stride()
        _need(len(shape) == 3 and shape[1] == cfg.n_q_heads and shape[2] == cfg.head_dim and st[2] == 1
              and q.device == self.device,
              "q: [n, %d, %d] with a unit channel stride, on %s" % (cfg.n_q_heads, cfg.head_dim, self.device))
        if out is None:
            out = torch.empty(shape, dtype=q.dtype, device=self.device)
        else:
            _need(out.dtype == q.dtype and out.shape == shape and out.is_contiguous() and out.device == self.device,
                  "out: contiguous, of q's shape and dtype")
        if lse is not None:
            _need(lse.dtype == torch.float32 and lse.shape == shape[:2] and lse.is_contiguous()
                  and lse.device == self.device, "lse: contiguous fp32 [n, n_q_heads]")
        elif with_lse:
            lse = torch.empty(shape[:2], dtype=torch.float32, device=self.device)
        ws = self.ws if workspace is None else workspace
        _need(ws.device == self.device and ws.is_contiguous(), "workspace: contiguous, on %s" % self.device)
        at, n_seqs = self._starts(starts)
        with _On(self.device) as stream:
            check(self._lib.semkv_paged_attn(self._ref, layer, q.data_ptr(), code, st[0], st[1],
                                             cfg.head_dim ** -0.5 if scale is None else scale, at, n_seqs, shape[0],
                                             out.data_ptr(), lse.data_ptr() if lse is not None else None, ws.data_ptr(),
                                             ws.numel() * ws.element_size(), stream), "semkv_paged_attn")
        return (out, lse) if with_lse or lse is not None else out

    # -- state -------------------------------------------------------------
    def status(self) -> int:
        return int(self.status_word[0].item())


def _prod(shape):
    n = 1
    for k in shape:
        n *= k
    return n


def _rows2(t, what, shape, dtype, device):
    """Element strides of a [B, T] tensor (or [N]: one row of N)."""
    _need(t.dtype == dtype and tuple(t.shape) == shape and t.device == device,
          "%s: %s of shape %s on %s" % (what, dtype, list(shape), device))
    return t.stride() if len(shape) == 2 else (0, t.stride(0))


def _logprobs(logits, targets, top, negate, logp, entropy, want_entropy):
    import torch
    code = _code(logits.dtype, "logits", True)
    _need(logits.dim() in (2, 3) and (logits.stride(-1) == 1 or logits.shape[-1] == 1) and logits.is_cuda,
          "logits: [N, V] or [B, T, V] with a unit stride over V, on a GPU")
    lead, V, dev = tuple(logits.shape[:-1]), logits.shape[-1], logits.device
    B, T = lead if len(lead) == 2 else (1, lead[0])
    s = logits.stride()
    s_b, s_t = (s[0], s[1]) if len(lead) == 2 else (0, s[0])
    _need(0 <= top <= 32 and top <= V and V > 0, "top: 0 to 32, at most V")
    t_b, t_t = _rows2(targets, "targets", lead, torch.int64, dev)
    if logp is None:
        logp = torch.empty(lead, dtype=torch.float32, device=dev)
    o = _rows2(logp, "scores", lead, torch.float32, dev)
    if want_entropy and entropy is None:
        entropy = torch.empty_strided(lead, logp.stride(), dtype=torch.float32, device=dev)
    top_logp = torch.empty(lead + (top,), dtype=torch.float32, device=dev) if top else None
    top_ids = torch.empty(lead + (top,), dtype=torch.int32, device=dev) if top else None
    n = ctypes.c_size_t()
    check(lib().semkv_token_logprobs_workspace(B * T, V, top, ctypes.byref(n)), "semkv_token_logprobs_workspace")
    ws = torch.empty(n.value, dtype=torch.uint8, device=dev) if n.value else None
    at = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
    with _On(dev) as stream:
        check(lib().semkv_token_logprobs(logits.data_ptr(), code, B, T, V, s_b, s_t, targets.data_ptr(), t_b, t_t,
                                         int(negate), at(logp), at(entropy), o[0], o[1], top, at(top_logp), at(top_ids),
                                         at(ws), n.value, stream), "semkv_token_logprobs")
    return logp, entropy, top_logp, top_ids


def token_logprobs(logits, targets, top=0):
    """Log probabilities of given tokens: logits fp16, bf16 or fp32 [N, V] or [B, T, V] (any strides with a unit one
    over V), targets int64 [N] or [B, T] (-1: none, gives 0; another one outside [0, V): NaN) -> (logp, entropy), fp32
    of the targets' shape, and with top > 0 also (top_logp fp32, top_ids int32) [..., top]: the likeliest tokens,
    equal logits by lower index.  A row without a finite sum of exponentials gives NaN, and ids of -1."""
    logp, entropy, top_logp, top_ids = _logprobs(logits, targets, top, False, None, None, True)
    return (logp, entropy, top_logp, top_ids) if top else (logp, entropy)


def score_tokens(logits, targets, scores=None):
    """Sec. 3.3 self-information -log p(target) of every token, the scores that semkv_rank takes: logits and targets as
    for token_logprobs.  scores: fp32 of the targets' shape, any strides (logits of position t predict token t+1:
    score_tokens(logits[:, :-1], ids[:, 1:], scores=s[:, 1:]))."""
    return _logprobs(logits, targets, 0, True, scores, None, False)[0]
