"""Refusals of append with rotation, of the cache of latents and of beam search's
choice, and the models the GPU tests compare with: no GPU."""
import ctypes

import numpy as np
import pytest

from tests import stepref as S


@pytest.fixture(scope="module")
def abi():
    import os
    from paper_2608_28911_amd import _abi, build
    if not os.path.exists(_abi.LIB_PATH):
        build.build()
    return _abi


P, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10002)


def rotary(abi, freqs=0x10000, positions=None, dim=64, interleaved=0):
    return ctypes.byref(abi.Rotary(freqs, positions, dim, interleaved))


def test_append_refusals(abi):
    from paper_2608_28911_amd import make_paged_config, paged_sizes
    c = abi.Paged()
    c.cfg = make_paged_config(n_layers=2, n_kv_heads=8, n_q_heads=32, n_pages=100, max_seqs=4, seq_pages=50, head_dim=128, group=64)
    c.sz, c.pool, c.state, c.status = paged_sizes(c.cfg), 0x1000, 0x2000, 0x3000
    r = ctypes.byref(c)
    call = lambda layer=0, K=P, V=P, dt=0, sT=1024, sH=128, q=P, qT=4096, qH=128, out=P, oT=4096, oH=128, rot=None, st=P, n=4, rows=4: (  # noqa: E731
        abi.lib().semkv_paged_append(r, layer, K, V, dt, sT, sH, q, qT, qH, out, oT, oH, rot or rotary(abi), st, n, rows, None))
    assert call(layer=2) == call(layer=-1) == call(K=None) == call(V=ODD) == call(dt=2) == call(sT=1025) == call(sH=4) == -1
    assert call(q=ODD) == call(out=None) == call(out=ODD) == call(qT=4) == call(oH=12) == call(st=None) == call(st=ctypes.c_void_p(0x10001)) == -1
    assert call(n=5) == call(rows=-1) == -1
    assert call(rot=rotary(abi, freqs=None)) == call(rot=rotary(abi, freqs=0x10001)) == call(rot=rotary(abi, positions=0x10002)) == -1
    assert call(rot=rotary(abi, dim=0)) == call(rot=rotary(abi, dim=8)) == call(rot=rotary(abi, dim=24)) == call(rot=rotary(abi, dim=144)) == -2
    assert call(rows=(1 << 28) + 1) == -2
    assert call(rows=0, K=None, V=None) == call(n=0) == 0
    assert abi.lib().semkv_paged_append(r, 0, P, P, 0, 1024, 128, None, 0, 0, None, 0, 0, None, P, 4, 4, None) == -1


LATENT = dict(n_layers=2, n_heads=16, n_pages=100, max_seqs=4, seq_pages=50)


@pytest.mark.parametrize("bad,status", [
    (dict(n_layers=0), -1), (dict(n_heads=0), -1), (dict(n_pages=0), -1), (dict(max_seqs=0), -1), (dict(seq_pages=0), -1),
    (dict(n_heads=129), -2), (dict(latent=128), -2), (dict(latent=384), -2), (dict(rope=16), -2), (dict(rope=128), -2),
    (dict(n_layers=65536), -2), (dict(n_pages=(1 << 20) + 1), -2), (dict(max_seqs=1025), -2),
    (dict(max_seqs=1024, seq_pages=1 << 19), -2)])
def test_latent_config_refusals(abi, bad, status):
    from paper_2608_28911_amd import make_latent_config
    s = abi.PagedSizes()
    assert abi.lib().semkv_latent_cache_sizes(ctypes.byref(make_latent_config(**{**LATENT, **bad})), ctypes.byref(s)) == status


def test_latent_config_refuses_other_types(abi):
    import torch
    from paper_2608_28911_amd import make_latent_config
    for dt in (torch.float32, torch.int16):
        with pytest.raises(ValueError):
            make_latent_config(**LATENT, dtype=dt)
    cfg = make_latent_config(**LATENT)
    cfg.dtype = abi.DTYPE_F32
    assert abi.lib().semkv_latent_cache_sizes(ctypes.byref(cfg), ctypes.byref(abi.PagedSizes())) == -1


def test_latent_sizes(abi):
    from paper_2608_28911_amd import latent_sizes, make_latent_config
    for latent, rope in ((512, 64), (512, 32), (256, 64), (256, 32)):
        s = latent_sizes(make_latent_config(**LATENT, latent=latent, rope=rope))
        assert s.record_bytes == 128 * (latent + rope) and s.page_bytes == 2 * s.record_bytes and s.pool_bytes == 100 * s.page_bytes


@pytest.fixture
def latent(abi):
    from paper_2608_28911_amd import latent_sizes, make_latent_config
    c = abi.Latent()
    c.cfg = make_latent_config(**LATENT)
    c.sz, c.pool, c.state, c.status = latent_sizes(c.cfg), 0x1000, 0x200000, 0x3000
    return c


def test_latent_calls_are_refused_before_the_device_is_touched(abi, latent):
    f, c, new = abi.lib(), ctypes.byref(latent), abi.Latent()
    assert f.semkv_latent_init(ctypes.byref(new), ctypes.byref(latent.cfg), None, P, P, None) == -1
    assert f.semkv_latent_init(ctypes.byref(new), ctypes.byref(latent.cfg), ctypes.c_void_p(0x10008), P, P, None) == -1
    assert f.semkv_latent_assign(c, None, P, None) == f.semkv_latent_assign(c, P, ODD, None) == -1
    scratch = ctypes.c_void_p(0x200000 + 4 * latent.sz.scratch_word)
    assert f.semkv_latent_assign(c, scratch, P, None) == f.semkv_latent_reserve(c, scratch, None) == f.semkv_latent_fork(c, scratch, None) == -1
    assert f.semkv_latent_reserve(c, None, None) == f.semkv_latent_reserve(None, P, None) == f.semkv_latent_fork(c, ODD, None) == -1
    assert f.semkv_latent_compact(c, None, 5, P, None) == f.semkv_latent_compact(c, P, -1, P, None) == -1
    append = lambda layer=0, C=P, cT=576, R=P, rT=576, q=P, qT=1024, qH=64, out=P, oT=1024, oH=64, rot=None, st=P, n=4, rows=4: (  # noqa: E731
        f.semkv_latent_append(c, layer, C, cT, R, rT, q, qT, qH, out, oT, oH, rot or rotary(abi), st, n, rows, None))
    assert append(layer=2) == append(layer=-1) == append(C=None) == append(R=ODD) == append(cT=577) == append(rT=4) == -1
    assert append(out=None) == append(q=ODD) == append(qH=65) == append(st=None) == append(n=5) == append(rows=-1) == -1
    assert append(rot=rotary(abi, dim=80)) == append(rot=rotary(abi, dim=40)) == -2
    assert append(rows=0, C=None) == append(n=0) == 0
    read = lambda layer=0, C=P, R=P, st=P, n=4, rows=4: f.semkv_latent_read(c, layer, C, R, st, n, rows, None)  # noqa: E731
    assert read(layer=2) == read(C=None) == read(R=ODD) == read(n=-1) == -1
    assert read(rows=0) == 0
    ws = latent.sz.workspace_bytes
    attn = lambda layer=0, q=P, qT=8192, qH=512, r=P, rT=1024, rH=64, scale=0.1, st=P, n=4, rows=4, out=P, lse=None, w=P, nb=ws: (  # noqa: E731
        f.semkv_latent_attn(c, layer, q, qT, qH, r, rT, rH, scale, st, n, rows, out, lse, w, nb, None))
    assert attn(layer=2) == attn(q=None) == attn(r=None) == attn(q=ODD) == attn(qT=4) == attn(rH=12) == -1
    assert attn(scale=0.0) == attn(scale=-1.0) == attn(scale=float("inf")) == attn(scale=float("nan")) == -1
    assert attn(out=None) == attn(out=ODD) == attn(lse=ODD) == attn(w=None) == attn(nb=ws - 1) == -1
    assert attn(rows=1 << 28) == -2                      # more tiles than a grid counts
    assert attn(rows=0) == attn(n=0) == 0


def test_beam_select_refusals(abi):
    f, n = abi.lib(), ctypes.c_size_t()
    size = lambda g=4, w=4, v=1000, k=4, out=ctypes.byref(n): f.semkv_beam_select_workspace(g, w, v, k, out)  # noqa: E731
    assert size(g=-1) == size(w=0) == size(v=0) == size(k=0) == size(out=None) == -1
    assert size(w=65) == size(k=65) == size(v=1 << 31) == size(g=1 << 22) == -2
    assert size(g=0) == 0 and n.value == 0
    assert size() == 0 and n.value > 0
    nb = n.value
    call = lambda x=P, dt=0, g=4, w=4, v=1000, sc=P, end=None, k=4, o=P, pa=P, to=P, ws=P, b=nb: (  # noqa: E731
        f.semkv_beam_select(x, dt, g, w, v, 4000, 1000, sc, end, 0, k, o, pa, to, ws, b, None))
    assert call(x=None) == call(x=ctypes.c_void_p(0x10001)) == call(dt=3) == call(dt=2, x=ODD) == call(g=-1) == call(w=0) == -1
    assert call(sc=None) == call(sc=ODD) == call(end=ODD) == call(o=None) == call(pa=ODD) == call(to=None) == -1
    assert call(ws=None) == call(ws=ctypes.c_void_p(0x10008)) == call(b=nb - 1) == -1
    assert call(k=65) == call(w=65) == -2
    assert call(g=0) == 0


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def host(abi, monkeypatch):
    """Caches over host memory, with a recorder for the library's launches."""
    import torch
    import paper_2608_28911_amd as M
    from paper_2608_28911_amd import paged
    monkeypatch.setattr(paged, "_enqueue", lambda index, f, what, *args: f(*args, 0))
    real, rec = abi.lib(), Recorder()
    rec.semkv_paged_cache_sizes, rec.semkv_latent_cache_sizes = real.semkv_paged_cache_sizes, real.semkv_latent_cache_sizes
    monkeypatch.setattr(paged, "lib", lambda: rec)
    kv = M.PagedKV4(M.make_paged_config(n_layers=1, n_kv_heads=2, n_q_heads=8, n_pages=8, max_seqs=4, seq_pages=4), device="cpu")
    lat = M.PagedLatent(M.make_latent_config(n_layers=1, n_heads=3, n_pages=8, max_seqs=4, seq_pages=4, dtype=torch.float16), device="cpu")
    rec.calls.clear()
    return rec, kv, lat


def test_binding_of_append(host):
    import torch
    rec, kv, _ = host
    qkv = torch.zeros((5, 12, 128), dtype=torch.float16)
    q, k, v = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
    st, f, pos = torch.tensor([0, 2, 5], dtype=torch.int32), torch.ones(64), torch.arange(5, dtype=torch.int32)
    out = kv.append(0, k, v, st, f, q=q, positions=pos, interleaved=True)
    assert out.shape == q.shape and out.is_contiguous()
    name, a = rec.calls.pop()
    rot = a[13]._obj
    assert name == "semkv_paged_append" and a[1:14] == (0, k.data_ptr(), v.data_ptr(), 0, 12 * 128, 128, q.data_ptr(), 12 * 128, 128,
                                                       out.data_ptr(), 1024, 128, a[13]) and a[14:] == (st.data_ptr(), 2, 5, 0)
    assert (rot.freqs, rot.positions, rot.dim, rot.interleaved) == (f.data_ptr(), pos.data_ptr(), 128, 1)
    assert kv.append(0, k, v, st, f[:16]) is None
    name, a = rec.calls.pop()
    assert a[7:13] == (None, 0, 0, None, 0, 0) and (a[13]._obj.positions, a[13]._obj.dim) == (None, 32)
    assert kv.append(0, k, v, st, f, q=q, q_out=q) is q                  # in place
    assert rec.calls.pop()[1][7:13] == (q.data_ptr(), 1536, 128, q.data_ptr(), 1536, 128)
    for bad in (dict(q=q[:4]), dict(q=q.bfloat16()), dict(q=q[..., ::2]), dict(q_out=q), dict(q=q, q_out=torch.zeros_like(q)[:4]),
                dict(q=q, q_out=qkv[:, 1:9]), dict(q=q, q_out=torch.zeros((5, 1, 128), dtype=q.dtype).expand(5, 8, 128)),
                dict(positions=pos.long()), dict(positions=pos[:4]), dict(positions=pos[None])):
        with pytest.raises(ValueError):
            kv.append(0, k, v, st, f, **bad)
    for bad in ((k, v[:4], st, f), (k.float(), v.float(), st, f), (k, v, st.long(), f), (k, v, st, f.double()), (k, v, st, f[::2]),
                (k[:, :1], v[:, :1], st, f)):
        with pytest.raises(ValueError):
            kv.append(0, *bad)
    assert not rec.calls


def test_binding_of_latents(host):
    import torch
    rec, _, lat = host
    kv, q = torch.zeros((5, 576), dtype=torch.float16), torch.zeros((5, 3, 128), dtype=torch.float16)
    st, f = torch.tensor([0, 2, 5], dtype=torch.int32), torch.ones(32)
    out = lat.append(0, kv[:, :512], kv[:, 512:], st, f, q=q[..., 64:])
    name, a = rec.calls.pop()
    assert name == "semkv_latent_append" and a[1:12] == (0, kv.data_ptr(), 576, kv.data_ptr() + 1024, 576, q.data_ptr() + 128, 384, 128,
                                                        out.data_ptr(), 192, 64) and a[13:] == (st.data_ptr(), 2, 5, 0)
    C, R = lat.read(0, st, 5)
    assert C.shape == (5, 512) and R.shape == (5, 64) and rec.calls.pop()[1][1:4] == (0, C.data_ptr(), R.data_ptr())
    ql, qr = torch.zeros((3, 5, 512), dtype=torch.float16).transpose(0, 1), q[..., 64:]
    o, lse = lat.attn(0, ql, qr, st, 0.5, with_lse=True)
    name, a = rec.calls.pop()
    assert o.shape == ql.shape and lse.shape == (5, 3) and lse.dtype == torch.float32
    assert name == "semkv_latent_attn" and a[2:8] == (ql.data_ptr(), 512, 2560, qr.data_ptr(), 384, 128) and a[8] == 0.5
    assert a[14] == lat.ws.data_ptr() and a[15] == lat.sz.workspace_bytes
    lat.reserve(lat.lens), lat.fork(lat.lens)
    assert [c[0] for c in rec.calls] == ["semkv_latent_reserve", "semkv_latent_fork"]
    rec.calls.clear()
    for bad in (lambda: lat.append(0, kv[:, :256], kv[:, 512:], st, f), lambda: lat.append(0, kv[:, :512], kv[:4, 512:], st, f),
                lambda: lat.append(0, kv[:, :512].bfloat16(), kv[:, 512:], st, f), lambda: lat.append(0, kv[0, :512], kv[:, 512:], st, f),
                lambda: lat.attn(0, ql.bfloat16(), qr, st, 0.5), lambda: lat.attn(0, ql, qr[:4], st, 0.5),
                lambda: lat.attn(0, ql[0], qr, st, 0.5), lambda: lat.attn(0, ql, qr, st, 0.5, out=ql),
                lambda: lat.attn(0, ql, qr, st, 0.5, lse=torch.zeros((5, 3), dtype=torch.float64)),
                lambda: lat.read(0, st, 5, out=(C, R.float()))):
        with pytest.raises(ValueError):
            bad()
    assert not rec.calls


def test_output_of_latent_attention_beside_its_queries(host):
    """In place where q is contiguous; an output that meets the queries otherwise is refused."""
    import torch
    rec, _, lat = host
    st = torch.tensor([0, 3, 5], dtype=torch.int32)
    buf = torch.zeros(2 * 5 * 3 * 576, dtype=torch.float16)
    q, qr = buf[:5 * 3 * 512].view(5, 3, 512), torch.zeros((5, 3, 64), dtype=torch.float16)
    assert lat.attn(0, q, qr, st, 0.5, out=q) is q
    assert rec.calls.pop()[0] == "semkv_latent_attn"
    both = buf[:5 * 3 * 576].view(5, 3, 576)                              # q and q_rope in one row
    apart = buf[5 * 3 * 576:][:5 * 3 * 512].view(5, 3, 512)
    assert lat.attn(0, both[..., :512], both[..., 512:], st, 0.5, out=apart) is apart
    rec.calls.clear()
    shifted = buf[512:][:5 * 3 * 512].view(5, 3, 512)
    for bad in (lambda: lat.attn(0, q, qr, st, 0.5, out=shifted), lambda: lat.attn(0, both[..., :512], both[..., 512:], st, 0.5, out=q),
                lambda: lat.attn(0, apart, q[..., :64], st, 0.5, out=q)):
        with pytest.raises(ValueError):
            bad()
    assert not rec.calls


def test_pool_of_latents_is_checked(abi, monkeypatch):
    import torch
    import paper_2608_28911_amd as M
    from paper_2608_28911_amd import paged
    monkeypatch.setattr(paged, "_enqueue", lambda *a: None)
    cfg = M.make_latent_config(**LATENT)
    for bad in (torch.zeros(100 * 2 * 64 * 576, dtype=torch.float16), torch.zeros(100 * 2 * 64 * 576 - 1, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            M.PagedLatent(cfg, pool=bad)


def test_beam_select_needs_a_gpu_and_its_shapes(abi):
    import torch
    import paper_2608_28911_amd as M
    with pytest.raises(ValueError):
        M.beam_select(torch.zeros((4, 100)), torch.zeros(4))


def test_model_of_the_rotation():
    """Turning by theta and back is the row again; a turn keeps a pair's length; pairs as defined."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((7, 3, 32)).astype(np.float32)
    f, pos = S.frequencies(16), np.arange(7) * 1000003
    for il in (False, True):
        y = S.turned(x, pos, f, il)
        np.testing.assert_allclose(S.turned(y, -pos, f, il), x, atol=4e-7 * np.abs(x).max() * 4)
        assert np.array_equal(y[..., 16:], x[..., 16:])
    one = np.zeros((1, 1, 4), np.float32)
    one[..., 0] = 1
    c, s = np.float32(np.cos(1.5)), np.float32(np.sin(1.5))
    assert np.array_equal(S.turned(one, [3], [0.5, 0.25], False)[0, 0], np.float32([c, 0, s, 0]))
    assert np.array_equal(S.turned(one, [3], [0.5, 0.25], True)[0, 0], np.float32([c, s, 0, 0]))


def test_model_of_the_choice():
    x = np.log(np.array([[1, 2, 3, 2], [4, 4, 1, 1.0]]))
    t, b, v = S.choose(x, [0.0, 0.0], 5)
    assert list(zip(b, v)) == [(1, 0), (1, 1), (0, 2), (0, 1), (0, 3)]
    np.testing.assert_allclose(np.exp(t), [0.4, 0.4, 0.375, 0.25, 0.25])
    t, b, v = S.choose(x, [0.0, -1.0], 9, ended=[0, 1], pad=7)
    assert (b[2], v[2], t[2]) == (1, 7, -1.0) or (1, 7) in list(zip(b, v))
    assert list(b[5:]) == [-1] * 4 and np.all(t[5:] == -np.inf)
