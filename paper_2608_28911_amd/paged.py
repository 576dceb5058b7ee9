"""Python binding of the paged caches (4-bit, latents), of token scoring and of
beam search's choice.

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


def _float32():
    if _torch is None:
        _setup()
    return _torch.float32


def _extent(t):
    """Bytes from a tensor's first element to the end of its last (0: it has none)."""
    if t.numel() == 0:
        return 0
    return t.element_size() * (1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride())))


def _runs(t):
    """A tensor's elements as runs of so many bytes, and the steps between them: [(bytes, number)], the longest first."""
    e = run = t.element_size()
    steps = sorted((e * s, n) for n, s in zip(t.shape, t.stride()) if n > 1 and s > 0)
    while steps and steps[0][0] <= run:
        s, n = steps.pop(0)
        run += s * (n - 1)
    return run, steps[::-1]


def _overlap(a, b):
    """Whether an element of one tensor lies in the other: slices of one buffer that interleave do not meet.  (Said to
    meet without a look at every step: ranges that do, of layouts unlike each other.)"""
    ea, eb, apart = _extent(a), _extent(b), b.data_ptr() - a.data_ptr()
    if not (ea and eb and -eb < apart < ea):
        return False
    left = 1000                                                      # steps to look at

    def meet(d, ra, sa, rb, sb):                                     # b's runs are d bytes behind a's
        nonlocal left
        if not sa and not sb:
            return -rb < d < ra
        s = max(sa[0][0] if sa else 0, sb[0][0] if sb else 0)        # the longest step: of one, or of both
        na = nb = 1
        if sa and sa[0][0] == s:
            na, sa = sa[0][1], sa[1:]
        if sb and sb[0][0] == s:
            nb, sb = sb[0][1], sb[1:]
        wa, wb = (r + sum(t * (n - 1) for t, n in rest) for r, rest in ((ra, sa), (rb, sb)))
        for k in range(max(1 - na, -((wb + d - 1) // s)), min(nb - 1, (wa - d - 1) // s) + 1):
            left -= 1
            if left < 0 or meet(d + k * s, ra, sa, rb, sb):
                return True
        return False

    return meet(apart, *_runs(a), *_runs(b))


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


def make_latent_config(n_layers, n_heads, n_pages, max_seqs, seq_pages, latent=512, rope=64, dtype=None) -> _abi.LatentConfig:
    """dtype: torch.float16 or torch.bfloat16 (the latter if not given)."""
    return _abi.LatentConfig(n_layers=n_layers, n_heads=n_heads, latent=latent, rope=rope,
                             dtype=_abi.DTYPE_BF16 if dtype is None else _code(dtype, "dtype"), n_pages=n_pages,
                             max_seqs=max_seqs, seq_pages=seq_pages)


def latent_sizes(cfg: _abi.LatentConfig) -> _abi.PagedSizes:
    s = _abi.PagedSizes()
    check(lib().semkv_latent_cache_sizes(ctypes.byref(cfg), ctypes.byref(s)), "semkv_latent_cache_sizes")
    return s


_NO_QUERIES = (None, 0, 0, None, 0, 0)


class _Paged:
    """What the paged caches have in common: their buffers, and the calls on pages.

    _NAME: the prefix of the library's calls.  z: the sizes for cfg; struct: the
    library's struct, empty."""

    def _set_up(self, cfg, z, struct, pool, device):
        import torch
        self.cfg, self.sz = cfg, z
        dev = pool.device if pool is not None else torch.device(device)
        if dev.type == "cuda" and dev.index is None:
            dev = torch.device("cuda", torch.cuda.current_device())
        self.device = dev
        self._at = dev.index if dev.type == "cuda" else -1    # as Tensor.get_device() says it
        pool = self._pool(pool)
        self.pool = pool
        self.state = s = torch.zeros(z.state_bytes // 4, dtype=torch.int32, device=dev)
        self.status_word = torch.zeros(4, dtype=torch.int32, device=dev)
        self.ws = torch.zeros(z.workspace_bytes // 4, dtype=torch.float32, device=dev)
        self.c = struct
        self._ref = ctypes.byref(self.c)
        self._lib = lib()
        # what every call reads of the configuration, as plain integers
        self._layers, self._seqs, self._width = cfg.n_layers, cfg.max_seqs, cfg.seq_pages
        self._call("init", ctypes.byref(cfg), pool.data_ptr(), s.data_ptr(), self.status_word.data_ptr())
        self.lens = s[z.lens_word:z.lens_word + self._seqs]               # tokens of each slot
        self.table = s[z.table_word:z.table_word + self._seqs * self._width].view(self._seqs, self._width)  # its pages, -1: none
        self.refs = s[z.refs_word:z.refs_word + cfg.n_pages]              # table entries that name a page
        self.stalled = s[:1]                                              # not 0: the last reserve failed

    def _call(self, name, *args):
        name = self._NAME + name
        _enqueue(self._at, getattr(self._lib, name), name, self._ref, *args)

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

    def _rotary(self, freqs, positions, interleaved, n):
        _need(freqs.dtype == _float32() and freqs.get_device() == self._at and freqs.dim() == 1 and freqs.is_contiguous(),
              "freqs: contiguous fp32 of a value for each pair, on %s", self.device)
        return _abi.Rotary(freqs.data_ptr(), None if positions is None else self._ints(positions, "positions", n),
                           2 * freqs.numel(), 1 if interleaved else 0)

    def _turned(self, q, q_out, n, heads, dim, dtype, *others):
        """Where query rows are turned to, and the addresses and strides of both; others: the call's other inputs."""
        if q is None:
            _need(q_out is None, "q_out: there is no q")
            return None, _NO_QUERIES
        shape, st = (n, heads, dim), q.stride()
        _need(q.shape == shape and (st[2] == 1 or not n) and q.dtype == dtype and q.get_device() == self._at,
              "q: [%d, %d, %d] of the rows' dtype with a unit channel stride, on %s", n, heads, dim, self.device)
        if q_out is None:
            q_out = q.new_empty(shape)
            return q_out, (q.data_ptr(), st[0], st[1], q_out.data_ptr(), heads * dim, dim)
        at, to, so = q.data_ptr(), q_out.data_ptr(), q_out.stride()
        _need(q_out.shape == shape and so[2] == 1 and q_out.dtype == dtype and q_out.get_device() == self._at,
              "q_out: of q's shape and dtype with a unit channel stride")
        # rows and heads apart from each other, and all of it from q unless it is q
        _need(so[1] >= dim and so[0] >= (heads - 1) * so[1] + dim or so[0] >= dim and so[1] >= (n - 1) * so[0] + dim
              or n == 1 and so[1] >= dim or heads == 1 and so[0] >= dim or n * heads <= 1, "q_out: rows that overlap")
        _need(to == at and so == st or not _overlap(q, q_out), "q_out: q itself, or apart from q")
        for t in others:
            _need(t is None or not _overlap(t, q_out), "q_out: apart from the call's other inputs")
        return q_out, (at, st[0], st[1], to, so[0], so[1])

    # -- pages -------------------------------------------------------------
    def assign(self, lens, table):
        """Take over lengths [max_seqs] and page tables [max_seqs, seq_pages], int32; either may be the cache's own
        (shorter lengths over self.table drop the sequences' last tokens)."""
        self._call("assign", self._ints(lens, "lens", self._seqs), self._ints(table, "table", self._seqs, self._width))

    def reserve(self, n_new):
        """Room for n_new [max_seqs] (int32) more tokens of every slot."""
        self._call("reserve", self._ints(n_new, "n_new", self._seqs))

    def fork(self, parent):
        """Slot s takes over slot parent[s]'s contents (int32 [max_seqs]); its own number keeps it, -1 empties it."""
        self._call("fork", self._ints(parent, "parent", self._seqs))

    def compact(self, keep, n_keep):
        """Slot s keeps tokens keep[s, :n_keep[s]] only (int32 [max_seqs, W] and [max_seqs]); -1 leaves it alone."""
        _need(keep.dim() == 2, "keep: [max_seqs, W]")
        width = keep.shape[1]
        self._call("compact", self._ints(keep, "keep", self._seqs, width), width, self._ints(n_keep, "n_keep", self._seqs))

    # -- state -------------------------------------------------------------
    def status(self) -> int:
        return int(self.status_word[0].item())


class PagedKV4(_Paged):
    """A KV cache held in 4 bits, in pages of 64 tokens, for sequences of their
    own lengths (include/semkv.h says what each call does).

    The pool may be given (uint8, pool_bytes of paged_sizes(cfg), any shape):
    a program then keeps its own view of the pages.  Every other buffer is the
    cache's; the workspace has its full size from the start, so that a graph
    that holds its address stays valid."""

    _NAME = "semkv_paged_"

    def __init__(self, cfg: _abi.PagedConfig, pool=None, device="cuda"):
        self._heads, self._q_heads, self._dim = cfg.n_kv_heads, cfg.n_q_heads, cfg.head_dim
        self._scale = cfg.head_dim ** -0.5
        self._set_up(cfg, paged_sizes(cfg), _abi.Paged(), pool, device)

    def _pool(self, pool):
        import torch
        if pool is None:
            pool = torch.empty(self.sz.pool_bytes, dtype=torch.uint8, device=self.device)
        _need(pool.dtype == torch.uint8 and pool.is_contiguous() and pool.numel() == self.sz.pool_bytes,
              "pool: contiguous uint8 of %d bytes" % self.sz.pool_bytes)
        return pool

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

    def append(self, layer, K, V, starts, freqs, q=None, positions=None, interleaved=False, q_out=None):
        """write of one layer with the position rotation on the way: K [n, n_kv_heads, head_dim] is turned, then
        quantized; V as it is.  Pair i of a row's first 2 len(freqs) channels (channels i and i + len(freqs), or 2i and
        2i+1: interleaved) turns by position * freqs[i] (fp32); positions: int32 [n], or None: the row's place in its
        sequence.  q [n, n_q_heads, head_dim] (a unit channel stride) is turned likewise and returned, in q_out if
        given, which may be q itself, and holds no element of another input (None without q)."""
        code = _code(K.dtype, "K")
        shape, st = K.shape, K.stride()
        _need(V.dtype == K.dtype and V.shape == shape and V.stride() == st
              and K.get_device() == V.get_device() == self._at
              and len(shape) == 3 and shape[1] == self._heads and shape[2] == self._dim and st[2] == 1,
              "K, V: [n, %d, %d] alike, with a unit channel stride, on %s", self._heads, self._dim, self.device)
        n = shape[0]
        rot = self._rotary(freqs, positions, interleaved, n)
        out, turned = self._turned(q, q_out, n, self._q_heads, self._dim, K.dtype, K, V, starts, freqs, positions)
        at, n_seqs = self._starts(starts)
        _enqueue(self._at, self._lib.semkv_paged_append, "semkv_paged_append", self._ref, layer, K.data_ptr(), V.data_ptr(),
                 code, st[0], st[1], *turned, ctypes.byref(rot), at, n_seqs, n)
        return out

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


class PagedLatent(_Paged):
    """A cache of latent vectors, one a token for all heads (key and value), and a
    rotated key part, in 16 bits, in pages of 64 tokens, for sequences of their own
    lengths (include/semkv.h says what each call does).

    The pool may be given (of the configuration's dtype, contiguous, any shape:
    [n_pages][n_layers] records of [64][latent] and [64][rope])."""

    _NAME = "semkv_latent_"

    def __init__(self, cfg: _abi.LatentConfig, pool=None, device="cuda"):
        import torch
        self._heads, self._latent, self._rope = cfg.n_heads, cfg.latent, cfg.rope
        self.dtype = torch.bfloat16 if cfg.dtype == _abi.DTYPE_BF16 else torch.float16
        self._set_up(cfg, latent_sizes(cfg), _abi.Latent(), pool, device)

    def _pool(self, pool):
        import torch
        n = self.sz.pool_bytes // 2
        if pool is None:
            pool = torch.empty(n, dtype=self.dtype, device=self.device)
        _need(pool.dtype == self.dtype and pool.is_contiguous() and pool.numel() == n,
              "pool: contiguous %s of %d values", self.dtype, n)
        return pool

    def _part(self, t, what, shape):
        _need(t.dtype == self.dtype and t.shape == shape and (t.stride()[-1] == 1 or not shape[0]) and t.get_device() == self._at,
              "%s: %s of shape %s with a unit channel stride, on %s", what, self.dtype, shape, self.device)
        return t.stride()

    # -- rows --------------------------------------------------------------
    def append(self, layer, C, R, starts, freqs, q=None, positions=None, interleaved=False, q_out=None):
        """Latents C [n, latent] as they are and key parts R [n, rope] turned by their positions (PagedKV4.append says
        how) into the pages of the sequences' last tokens.  q [n, n_heads, rope], the queries' parts that meet R, are
        turned likewise and returned (None without q)."""
        _need(C.dim() == 2, "C: [n, %d]", self._latent)
        n = C.shape[0]
        c, r = self._part(C, "C", (n, self._latent)), self._part(R, "R", (n, self._rope))
        rot = self._rotary(freqs, positions, interleaved, n)
        out, turned = self._turned(q, q_out, n, self._heads, self._rope, self.dtype, C, R, starts, freqs, positions)
        at, n_seqs = self._starts(starts)
        _enqueue(self._at, self._lib.semkv_latent_append, "semkv_latent_append", self._ref, layer, C.data_ptr(), c[0],
                 R.data_ptr(), r[0], *turned, ctypes.byref(rot), at, n_seqs, n)
        return out

    def read(self, layer, starts, n_rows, out=None):
        """What the pages hold for the sequences' last tokens: C [n_rows, latent] and R [n_rows, rope]."""
        import torch
        if out is None:
            C = torch.empty((n_rows, self._latent), dtype=self.dtype, device=self.device)
            R = torch.empty((n_rows, self._rope), dtype=self.dtype, device=self.device)
        else:
            C, R = out
            _need(C.is_contiguous() and R.is_contiguous(), "out: contiguous")
            self._part(C, "out", (n_rows, self._latent))
            self._part(R, "out", (n_rows, self._rope))
        at, n_seqs = self._starts(starts)
        _enqueue(self._at, self._lib.semkv_latent_read, "semkv_latent_read", self._ref, layer, C.data_ptr(), R.data_ptr(),
                 at, n_seqs, n_rows)
        return C, R

    def attn(self, layer, q, q_rope, starts, scale, out=None, lse=None, with_lse=False, workspace=None):
        """Causal attention of the sequences' last tokens over their pages, every head over the same latents: q
        [n, n_heads, latent] (the queries multiplied into the latent space) and q_rope [n, n_heads, rope], of any
        strides with a unit one over channels -> out [n, n_heads, latent]; with_lse: (out, lse fp32 [n, n_heads]).
        scale: of the scores.  Calls that overlap in time need a workspace each (like cache.ws)."""
        import torch
        _need(q.dim() == 3 and q_rope.dim() == 3, "q, q_rope: [n, %d, channels]", self._heads)
        n = q.shape[0]
        shape = (n, self._heads, self._latent)
        s, r = self._part(q, "q", shape), self._part(q_rope, "q_rope", (n, self._heads, self._rope))
        if out is None:
            out = q.new_empty(shape)
        else:
            _need(out.dtype == self.dtype and out.shape == shape and out.is_contiguous() and out.get_device() == self._at,
                  "out: contiguous, of q's shape and dtype")
            _need((out.data_ptr() == q.data_ptr() and q.is_contiguous() or not _overlap(out, q)) and not _overlap(out, q_rope),
                  "out: q itself where that is contiguous, or apart from q; apart from q_rope")
        if lse is not None:
            with_lse = True
            _need(lse.dtype == torch.float32 and lse.shape == shape[:2] and lse.is_contiguous()
                  and lse.get_device() == self._at, "lse: contiguous fp32 [n, n_heads]")
        elif with_lse:
            lse = torch.empty(shape[:2], dtype=torch.float32, device=self.device)
        ws = self.ws if workspace is None else workspace
        _need(ws.get_device() == self._at and ws.is_contiguous(), "workspace: contiguous, on %s", self.device)
        at, n_seqs = self._starts(starts)
        _enqueue(self._at, self._lib.semkv_latent_attn, "semkv_latent_attn", self._ref, layer, q.data_ptr(), s[0], s[1],
                 q_rope.data_ptr(), r[0], r[1], scale, at, n_seqs, n, out.data_ptr(), lse.data_ptr() if with_lse else None,
                 ws.data_ptr(), ws.numel() * ws.element_size())
        return (out, lse) if with_lse else out


@functools.lru_cache(maxsize=1024)
def _beam_workspace(groups, width, vocab, k):
    n = ctypes.c_size_t()
    check(lib().semkv_beam_select_workspace(groups, width, vocab, k, ctypes.byref(n)), "semkv_beam_select_workspace")
    return n.value


def beam_select(logits, scores, k=None, ended=None, pad=0):
    """Beam search's choice: of every group's beams and tokens the k (width if not given) of the largest score + log
    probability.  logits fp16, bf16 or fp32 [groups, width, V] (or [width, V]: one group; any strides with a unit one
    over V), scores fp32 [groups, width] (-inf: a beam not in use), ended int32 [groups, width] (not 0: the beam's one
    candidate is itself, with token `pad`) -> (scores fp32, parents int32, tokens int32) [groups, k], in descending
    order, equal ones by lower beam and token.  parents are slots (group * width + beam), as PagedKV4.fork takes them;
    include/semkv.h says what beams without candidates give."""
    import torch
    code = _code(logits.dtype, "logits", True)
    shape, s, at, dev = logits.shape, logits.stride(), logits.get_device(), logits.device
    _need(len(shape) in (2, 3) and (s[-1] == 1 or shape[-1] == 1) and at >= 0,
          "logits: [width, V] or [groups, width, V] with a unit stride over V, on a GPU")
    lead, V = shape[:-1], shape[-1]
    groups, width = (1, lead[0]) if len(lead) == 1 else lead
    k = width if k is None else k
    _need(1 <= width <= 64 and 1 <= k <= 64 and V > 0, "width and k: 1 to 64")
    _need(scores.dtype == torch.float32 and scores.shape == lead and scores.is_contiguous() and scores.get_device() == at,
          "scores: contiguous fp32 of shape %s on the logits' device", tuple(lead))
    _need(ended is None or (ended.dtype == torch.int32 and ended.shape == lead and ended.is_contiguous()
                            and ended.get_device() == at), "ended: contiguous int32 of shape %s on the logits' device", tuple(lead))
    of = (*lead[:-1], k)
    # (with the strides given an allocation takes 1.2 us, not 1.6; a call of few rows takes as long as the host does)
    along = (k, 1) if len(lead) == 2 else (1,)
    best = torch.empty_strided(of, along, dtype=torch.float32, device=dev)
    parents, tokens = torch.empty_strided((2, *of), (groups * k, *along), dtype=torch.int32, device=dev).unbind()
    n = _beam_workspace(groups, width, V, k)
    ws = torch.empty_strided((n,), (1,), dtype=torch.uint8, device=dev)
    _enqueue(at, lib().semkv_beam_select, "semkv_beam_select", logits.data_ptr(), code, groups, width, V,
             s[0] if len(lead) == 2 else 0, s[-2], scores.data_ptr(), ended.data_ptr() if ended is not None else None, pad, k,
             best.data_ptr(), parents.data_ptr(), tokens.data_ptr(), ws.data_ptr(), n)
    return best, parents, tokens


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
