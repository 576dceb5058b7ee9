"""Refusals of the paged cache and of token scoring, and the model the GPU tests
compare with: no GPU."""
import ctypes

import numpy as np
import pytest

from tests import pagedref as R


@pytest.fixture(scope="module")
def abi():
    import os
    from paper_2608_28911_amd import _abi, build
    if not os.path.exists(_abi.LIB_PATH):
        build.build()
    return _abi


GOOD = dict(n_layers=2, n_kv_heads=8, n_q_heads=32, n_pages=100, max_seqs=4, seq_pages=50, head_dim=128, group=64)


def config(**kw):
    from paper_2608_28911_amd import make_paged_config
    return make_paged_config(**{**GOOD, **kw})


@pytest.mark.parametrize("bad,status", [
    (dict(n_layers=0), -1), (dict(n_kv_heads=0), -1), (dict(n_q_heads=0), -1), (dict(n_pages=0), -1),
    (dict(max_seqs=0), -1), (dict(seq_pages=-1), -1), (dict(n_q_heads=33), -2), (dict(n_q_heads=8 * 65), -2),
    (dict(head_dim=96), -2), (dict(head_dim=256), -2), (dict(group=16), -2), (dict(group=256), -2),
    (dict(head_dim=64, group=128), -2), (dict(n_pages=(1 << 20) + 1), -2), (dict(max_seqs=1025), -2),
    (dict(seq_pages=(1 << 20) + 1), -2), (dict(max_seqs=1024, seq_pages=1 << 19), -2), (dict(n_layers=8192), -2)])
def test_config_refusals(abi, bad, status):
    s = abi.PagedSizes()
    assert abi.lib().semkv_paged_cache_sizes(ctypes.byref(config(**bad)), ctypes.byref(s)) == status


def test_sizes(abi):
    from paper_2608_28911_amd import paged_sizes
    for d, g, rec in ((128, 128, 8704), (128, 64, 9216), (128, 32, 10240), (64, 64, 4608), (64, 32, 5120)):
        s = paged_sizes(config(head_dim=d, group=g))
        assert s.record_bytes == rec and s.page_bytes == 16 * rec and s.pool_bytes == 1600 * rec
        assert all(w % 64 == 0 for w in (s.lens_word, s.table_word, s.refs_word, s.free_word, s.scratch_word))
        assert s.table_word - s.lens_word >= 4 and s.refs_word - s.table_word >= 200 and s.free_word - s.refs_word >= 100


@pytest.fixture
def cache(abi):
    c = abi.Paged()
    cfg = config()
    s = abi.PagedSizes()
    assert abi.lib().semkv_paged_cache_sizes(ctypes.byref(cfg), ctypes.byref(s)) == 0
    c.cfg, c.sz, c.pool, c.state, c.status = cfg, s, 0x1000, 0x2000, 0x3000
    return c


def test_calls_are_refused_before_the_device_is_touched(abi, cache):
    f, c, p, odd = abi.lib(), ctypes.byref(cache), ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10002)
    new, cfg = abi.Paged(), config()
    r = ctypes.byref
    assert f.semkv_paged_init(r(new), r(cfg), None, p, p, None) == -1
    assert f.semkv_paged_init(r(new), r(cfg), ctypes.c_void_p(0x10008), p, p, None) == -1
    assert f.semkv_paged_init(r(new), r(config(group=16)), p, p, p, None) == -2
    assert f.semkv_paged_assign(c, None, p, None) == f.semkv_paged_assign(c, p, odd, None) == -1
    assert f.semkv_paged_reserve(c, None, None) == f.semkv_paged_reserve(None, p, None) == -1
    assert f.semkv_paged_fork(c, odd, None) == -1
    assert f.semkv_paged_compact(c, None, 5, p, None) == f.semkv_paged_compact(c, p, -1, p, None) == -1
    write = lambda layer=0, K=p, V=p, dt=0, sT=1024, sH=128, st=p, n=4, rows=4: f.semkv_paged_write(  # noqa: E731
        c, layer, K, V, dt, 0, sT, sH, st, n, rows, None)
    assert write(layer=2) == write(layer=-2) == write(K=None) == write(V=odd) == write(dt=2) == write(sT=1025) == -1
    assert write(sH=4) == write(st=None) == write(n=5) == write(rows=-1) == -1
    assert write(rows=(1 << 28) + 1) == -2
    assert write(rows=0, K=None, V=None) == 0 and write(n=0) == 0
    read = lambda layer=0, K=p, V=p, dt=0, st=p, n=4, rows=4: f.semkv_paged_read(c, layer, K, V, dt, st, n, rows, None)  # noqa: E731
    assert read(layer=2) == read(K=None) == read(V=odd) == read(dt=3) == read(n=-1) == -1
    assert read(rows=0) == 0
    ws = cache.sz.workspace_bytes
    attn = lambda layer=0, q=p, dt=0, sT=4096, sH=128, scale=0.1, st=p, n=4, rows=4, out=p, lse=None, w=p, nb=ws: (  # noqa: E731
        f.semkv_paged_attn(c, layer, q, dt, sT, sH, scale, st, n, rows, out, lse, w, nb, None))
    assert attn(layer=-1) == attn(q=None) == attn(q=odd) == attn(dt=2) == attn(sT=4) == attn(sH=129) == -1
    assert attn(scale=0.0) == attn(scale=-1.0) == attn(scale=float("inf")) == attn(scale=float("nan")) == -1
    assert attn(out=None) == attn(out=ctypes.c_void_p(0x10008)) == attn(lse=odd) == attn(w=None) == attn(nb=ws - 1) == -1
    assert attn(rows=0) == 0
    assert attn(rows=1 << 28) == -2                      # more tiles than a grid counts


def test_token_logprobs_refusals(abi):
    f, p, odd = abi.lib(), ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10001)
    n = ctypes.c_size_t()
    size = f.semkv_token_logprobs_workspace
    assert size(4, 100, 33, ctypes.byref(n)) == size(4, 100, 101, ctypes.byref(n)) == size(-1, 100, 0, ctypes.byref(n)) == -1
    assert size(4, 0, 0, ctypes.byref(n)) == size(4, 100, 0, None) == -1
    assert size(4, 128000, 5, ctypes.byref(n)) == 0 and n.value > 0
    call = lambda x=p, dt=0, b=1, T=4, v=100, tg=p, lp=p, e=p, top=0, tl=None, ti=None, ws=None, nb=0: (  # noqa: E731
        f.semkv_token_logprobs(x, dt, b, T, v, T * v, v, tg, T, 1, 0, lp, e, T, 1, top, tl, ti, ws, nb, None))
    assert call(x=None) == call(x=odd) == call(dt=3) == call(b=-1) == call(v=0) == call(top=-1) == call(top=33) == -1
    assert call(tg=None) == call(tg=ctypes.c_void_p(0x10004)) == call(lp=odd) == call(e=odd) == -1
    assert call(top=3) == call(top=3, tl=p) == call(v=128000) == call(v=128000, ws=p, nb=8) == -1
    assert call(b=1 << 14, T=1 << 14) == call(v=1 << 31) == -2
    assert call(b=0) == call(T=0) == 0


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def bound(abi, monkeypatch):
    """The Python cache over host memory, with a recorder for the library's launches."""
    import torch
    import paper_2608_28911_amd as P
    from paper_2608_28911_amd import paged
    monkeypatch.setattr(paged, "_enqueue", lambda index, f, what, *args: f(*args, 0))
    real, rec = abi.lib(), Recorder()

    class Lib:
        def __getattr__(self, name):
            return real.semkv_paged_cache_sizes if name == "semkv_paged_cache_sizes" else getattr(rec, name)
    monkeypatch.setattr(paged, "lib", lambda: Lib())
    return P.PagedKV4(config(n_pages=8, seq_pages=4), device="cpu"), rec


def test_binding_checks_what_it_is_given(bound):
    import torch
    c, rec = bound
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    kv, q = torch.zeros((5, 8, 128), dtype=torch.float16), torch.zeros((5, 32, 128), dtype=torch.float16)
    rec.calls.clear()
    bad = [
        lambda: c.reserve(i(3)), lambda: c.reserve(i(4).long()), lambda: c.reserve(i(8)[::2]),
        lambda: c.fork(i(4, 1)), lambda: c.assign(i(4), i(4, 5)), lambda: c.assign(i(4), i(4, 4).t()),
        lambda: c.compact(i(3, 7), i(4)), lambda: c.compact(i(4, 14)[:, ::2], i(4)), lambda: c.compact(i(4, 7), i(5)),
        lambda: c.write(0, kv, kv.bfloat16(), i(3)), lambda: c.write(0, kv.float(), kv.float(), i(3)),
        lambda: c.write(0, kv[:, :7], kv[:, :7], i(3)), lambda: c.write(-1, kv, kv, i(3)),
        lambda: c.write(0, kv, kv[:4], i(3)), lambda: c.write(0, kv, kv, i(6)), lambda: c.write(0, kv, kv, i(0)),
        lambda: c.write(0, kv, kv.transpose(0, 1).contiguous().transpose(0, 1), i(3)),
        lambda: c.read(0, i(3), 5, dtype=torch.float64), lambda: c.read(0, i(3), 5, out=(kv, kv[:4])),
        lambda: c.attn(0, q[:, :31], i(3)), lambda: c.attn(0, q.float(), i(3)), lambda: c.attn(0, q, i(3), out=q.bfloat16()),
        lambda: c.attn(0, q, i(3), lse=torch.zeros((5, 31))), lambda: c.attn(0, q, i(3).long()),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
        assert not rec.calls, k
    c.write(0, kv, kv, i(3))
    c.attn(1, q, i(3))
    assert [n for n, _ in rec.calls] == ["semkv_paged_write", "semkv_paged_attn"]
    name, a = rec.calls[0]
    assert a[1] == 0 and a[4:8] == (0, 0, 1024, 128) and a[9:11] == (2, 5)


def test_a_cache_in_host_memory_is_refused(monkeypatch):
    """Its addresses must not reach a kernel."""
    import torch
    import paper_2608_28911_amd as P
    from paper_2608_28911_amd import paged
    rec = Recorder()
    sizes = P.paged_sizes(config(n_pages=8, seq_pages=4))
    monkeypatch.setattr(paged, "paged_sizes", lambda cfg: sizes)
    monkeypatch.setattr(paged, "lib", lambda: rec)
    for kw in ({"device": "cpu"}, {"device": "meta"}, {"pool": torch.empty(sizes.pool_bytes, dtype=torch.uint8)}):
        with pytest.raises(ValueError):
            P.PagedKV4(config(n_pages=8, seq_pages=4), **kw)
        assert not rec.calls, kw


def test_binding_of_logprobs_checks_what_it_is_given():
    import torch
    import paper_2608_28911_amd as P
    x, t = torch.zeros((3, 50)), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        P.token_logprobs(x, t)                           # not on a GPU


def test_model_places_every_code_once():
    for d in (64, 128):
        for word, bit in R._PLACES[d]:
            seen = set(zip(word.ravel().tolist(), bit.ravel().tolist()))
            assert len(seen) == 64 * d and max(w for w, _ in seen) == 8 * d - 1


def test_model_quantizer_keeps_rows_within_half_a_step():
    rng = np.random.default_rng(0)
    for dt, eps in ((np.float16, 2.0 ** -11), (np.float32, 2.0 ** -11)):
        x = rng.standard_normal((50, 128)).astype(dt).astype(np.float32)
        c, s, z = R.quantize(x, 32)
        v = c * np.repeat(s.astype(np.float64), 32, 1) + np.repeat(z.astype(np.float64), 32, 1)
        s64 = np.repeat(s.astype(np.float64), 32, 1)
        # half a step, and what the rounding of scale (15 steps away at most) and zero to fp16 moves
        assert np.all(np.abs(v - x) <= 0.5 * s64 * (1 + 1e-6) + 15 * eps * s64 + eps * np.abs(np.repeat(z.astype(np.float64), 32, 1)))
