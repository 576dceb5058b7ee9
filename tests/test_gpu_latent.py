"""GPU parity of the paged cache of latents with the plain models of
tests/stepref.py and tests/pagedref.py.

Stored rows and moved pages are compared bit for bit.  Attention's tolerance, from
the arithmetic (u = 2^-24 is half a step of fp32):
  - an output is rounded to its type: finfo.eps / 2 relative;
  - each weight is rounded to the type: finfo.eps / 2 of p |c| (and in fp16 2^-35
    of the largest weight where it is less than 2^-24 of that);
  - a score is a sum of latent + rope products (exact in fp32) and two more
    operations: off by at most d = (latent + rope + 8) u scale sum_j |q_j c_j|, and
    its exponent, in fp32 relative to the row's reference, by 2 u (|x| + |m|) log2 e;
    the weight by a factor e^(+-2d) with the normalisation, its exponential by 2 u;
  - fp32 sums over n tokens, in any order: n u relative to the sum of magnitudes."""
import numpy as np
import pytest

from tests import pagedref as R
from tests import stepref as S
from tests.test_gpu_paged import ints, starts_of

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def make(heads=4, latent=512, rope=64, dtype="bfloat16", n_layers=1, n_pages=32, seqs=4, seq_pages=8, fill=float("nan")):
    import torch
    import paper_2608_28911_amd as P
    dt = getattr(torch, dtype)
    cfg = P.make_latent_config(n_layers=n_layers, n_heads=heads, latent=latent, rope=rope, dtype=dt, n_pages=n_pages,
                               max_seqs=seqs, seq_pages=seq_pages)
    pool = torch.full((n_pages, n_layers, 64 * (latent + rope)), fill, dtype=dt, device="cuda")   # rows never written: NaN
    return P.PagedLatent(cfg, pool=pool)


def rows(rng, shape, dtype):
    import torch
    x = rng.standard_normal(shape).astype(np.float32)
    x[..., 3::29] *= 5.0
    x[..., 7] += 3.0
    return torch.from_numpy(x).to(getattr(torch, dtype) if isinstance(dtype, str) else dtype).cuda()


def f64(t):
    return t.detach().cpu().double().numpy()


def held(cache, s, n, layer=0):
    """c [n, latent] and r [n, rope] of a sequence's tokens, NaN rows where a page is missing."""
    L, W = cache._latent, cache._latent + cache._rope
    c, r = np.full((n, L), np.nan), np.full((n, W - L), np.nan)
    pool, table = cache.pool.view(cache.cfg.n_pages, cache.cfg.n_layers, -1), cache.table[s].tolist()
    for p in range((n + 63) // 64):
        m = min(64, n - 64 * p)
        if table[p] >= 0:
            rec = f64(pool[table[p], layer])
            c[64 * p:64 * p + m], r[64 * p:64 * p + m] = rec[:64 * L].reshape(64, L)[:m], rec[64 * L:].reshape(64, W - L)[:m]
    return c, r


def fill(cache, rng, lens):
    """Sequences of the given lengths; every layer's rows appended."""
    import torch
    lens = list(lens) + [0] * (cache.cfg.max_seqs - len(lens))
    cache.reserve(ints(lens))
    n = sum(lens)
    f = torch.from_numpy(S.frequencies(cache._rope)).cuda()
    for layer in range(cache.cfg.n_layers):
        kv = rows(rng, (n, cache._latent + cache._rope), cache.dtype)
        cache.append(layer, kv[:, :cache._latent], kv[:, cache._latent:], starts_of(lens), f)
    assert cache.status() == 0
    return lens


def check(cache, q, qr, counts, scale, got, lse, layer=0, some=None):
    """Every row (or those of `some`) against 64 bits."""
    eps = {"torch.bfloat16": 2.0 ** -8, "torch.float16": 2.0 ** -11}[str(cache.dtype)]
    L, W, H = cache._latent, cache._latent + cache._rope, cache._heads
    lens, out, lse = cache.lens.tolist(), f64(got), f64(lse)
    q, qr = f64(q), f64(qr)
    at, worst = 0, 0.0
    for s, m in enumerate(counts):
        c, r = held(cache, s, lens[s])
        there = ~np.isnan(c[:, 0]) if len(c) else np.zeros(0, bool)
        for i in range(m):
            seen = max(0, lens[s] - m + i + 1)
            ok = there[:seen]
            if some is not None and at + i not in some:
                continue
            for h in range(H):
                cs, rs = c[:seen][ok], r[:seen][ok]
                want, wl, p = S.attend(q[at + i, h], qr[at + i, h], cs, rs, scale)
                if len(p) == 0:
                    assert not out[at + i, h].any() and lse[at + i, h] == -np.inf
                    continue
                x = (cs @ q[at + i, h] + rs @ qr[at + i, h]) * scale
                mag = (np.abs(cs) @ np.abs(q[at + i, h]) + np.abs(rs) @ np.abs(qr[at + i, h])) * scale
                d = (W + 8) * U * mag + 2 * U * (np.abs(x) + np.abs(x).max() + 16) * 1.5
                n = len(p)
                tol_l = 2 * (p @ d) + (n + 4) * U + U * abs(wl)
                assert abs(lse[at + i, h] - wl) <= tol_l, (s, i, h, lse[at + i, h], wl, tol_l)
                w = p * (eps + 2 * d + (n + 4) * U)
                if eps == 2.0 ** -11:
                    w = w + np.where(p < 2.0 ** -24 * p.max(), 2.0 ** -35 * p.max(), 0.0)
                tol = w @ np.abs(cs) + (p * d).sum() * np.abs(want) + (n + 4) * U * np.abs(want) + eps * np.abs(want) + 1e-30
                e = np.abs(out[at + i, h] - want)
                worst = max(worst, (e / tol).max())
                assert np.all(e <= tol), (s, i, h, (e / tol).max())
        at += m
    return worst


# ---- rows ------------------------------------------------------------------

@pytest.mark.parametrize("latent,rope,dtype,rot,il,lens,counts,shift,heads", [
    (512, 64, "bfloat16", 64, True, [1, 65, 130], [1, 1, 1], None, 16),
    (512, 32, "float16", 32, False, [3, 200], [3, 137], None, 33),
    (256, 64, "float16", 48, False, [64, 65, 1], [64, 2, 1], 100003, 1),
    (256, 32, "bfloat16", 16, True, [129], [129], -77, 128)])
def test_rows_are_stored_and_read_bit_for_bit(latent, rope, dtype, rot, il, lens, counts, shift, heads):
    import torch
    rng = np.random.default_rng(latent + rope)
    cache = make(heads, latent, rope, dtype, n_layers=2, n_pages=16)
    cache.reserve(ints(lens + [0] * (4 - len(lens))))
    n = sum(counts)
    kv, qq = rows(rng, (n, latent + rope), dtype), rows(rng, (n, heads, 128 + rope), dtype)
    C, Rr, q = kv[:, :latent], kv[:, latent:], qq[..., 128:]
    place = np.concatenate([np.arange(a - b, a) for a, b in zip(lens, counts)])
    pos = place if shift is None else place + shift
    f, st = S.frequencies(rot), starts_of(counts)
    before = cache.pool.clone()
    out = cache.append(1, C, Rr, st, torch.from_numpy(f).cuda(), q=q, interleaved=il, positions=None if shift is None else ints(pos))
    turned = lambda t: torch.from_numpy(S.turned(t.cpu().float().numpy(), pos, f, il)).to(t.dtype)  # noqa: E731
    assert torch.equal(out.cpu(), turned(q))
    c, r = cache.read(1, st, n)
    want = turned(Rr[:, None])[:, 0]
    assert torch.equal(c, C) and torch.equal(r.cpu(), want) and cache.status() == 0
    # where the layout says, and nothing else has changed
    pool, at = before.cpu().view(16, 2, -1), 0
    table = cache.table.cpu()
    for s, (ln, m) in enumerate(zip(lens, counts)):
        for p in range(ln - m, ln):
            rec = pool[table[s, p // 64], 1]
            rec[p % 64 * latent:(p % 64 + 1) * latent] = C[at].cpu()
            rec[64 * latent + p % 64 * rope:64 * latent + (p % 64 + 1) * rope] = want[at]
            at += 1
    assert torch.equal(cache.pool.cpu().view(torch.int16), pool.view_as(cache.pool).view(torch.int16))
    same = cache.append(1, C, Rr, st, torch.from_numpy(f).cuda(), q=q, q_out=q, interleaved=il,
                        positions=None if shift is None else ints(pos))
    assert same is q and torch.equal(q, out)


def test_rows_without_a_place():
    import torch
    rng = np.random.default_rng(1)
    cache = make(heads=2, n_pages=8, seq_pages=4)
    table = torch.full((4, 4), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[2, 1] = 5, 6
    cache.assign(ints([3, 0, 70, 0]), table)
    kv, q = rows(rng, (16, 576), "bfloat16"), rows(rng, (16, 2, 64), "bfloat16")
    f, st = S.frequencies(64), ints([0, 5, 6, 14])
    before = cache.pool.clone()
    out = torch.full_like(q, 77.0)
    cache.append(0, kv[:, :512], kv[:, 512:], st, torch.from_numpy(f).cuda(), q=q, q_out=out)
    assert cache.status() == R.BAD_INDEX
    assert (out[14:] == 77).all() and not out[:2].any() and not out[5].any() and out[2:5].any() and out[6:14].any()
    c, r = cache.read(0, st, 16, out=(torch.full((16, 512), 5.0, dtype=q.dtype, device="cuda"),
                                      torch.full((16, 64), 5.0, dtype=q.dtype, device="cuda")))
    assert not c[:2].any() and not c[5].any() and not c[6:8].any() and (c[14:] == 5).all() and (r[14:] == 5).all()
    assert torch.equal(c[2:5], kv[2:5, :512]) and torch.equal(c[8:14], kv[8:14, :512])
    rest = [i for i in range(8) if i not in (5, 6)]
    assert torch.equal(cache.pool[rest].view(torch.int16), before[rest].view(torch.int16))


def test_a_token_that_is_not_finite_is_zeros():
    import torch
    rng = np.random.default_rng(2)
    cache = make(heads=1, latent=256, rope=32, dtype="float16")
    cache.reserve(ints([5, 0, 0, 0]))
    kv = rows(rng, (5, 288), "float16")
    kv[1, 3], kv[2, 287] = float("inf"), float("nan")
    kv[3, 256:] = 65504.0                                     # overflows when it is turned by an eighth
    f = torch.full((16,), np.pi / 4, device="cuda")
    cache.append(0, kv[:, :256], kv[:, 256:], starts_of([5]), f, positions=ints([1] * 5))
    c, r = cache.read(0, starts_of([5]), 5)
    assert cache.status() == R.NONFINITE
    assert not c[1:4].any() and not r[1:4].any() and torch.equal(c[[0, 4]], kv[[0, 4], :256]) and r[0].any() and r[4].any()


def test_pages_are_shared_copied_and_compacted():
    import torch
    rng = np.random.default_rng(3)
    cache = make(heads=2, n_layers=2, n_pages=20, seq_pages=4)
    lens = fill(cache, rng, [100, 64])
    old = [[held(cache, s, lens[s], l) for l in range(2)] for s in range(2)]
    cache.fork(ints([0, 1, 0, -1]))
    cache.reserve(ints([1, 0, 1, 0]))                         # the shared last page is copied
    assert cache.refs.max().item() == 2 and cache.lens.tolist() == [101, 64, 101, 0]
    for s, o in ((0, 0), (2, 0), (1, 1)):
        for l in range(2):
            for x, y in zip(held(cache, s, lens[o], l), old[o][l]):
                assert np.array_equal(x, y)
    keep = torch.zeros((4, 70), dtype=torch.int32, device="cuda")
    lists = [sorted(rng.permutation(100)[:66].tolist()), [5, 63], []]
    for s, k in enumerate(lists):
        keep[s, :len(k)] = ints(k)
    cache.compact(keep, ints([66, 2, 0, -1]))
    assert cache.lens.tolist() == [66, 2, 0, 0] and cache.status() == 0
    for s in range(2):
        for l in range(2):
            for x, y in zip(held(cache, s, len(lists[s]), l), old[s][l]):
                assert np.array_equal(x, y[lists[s]])
    assert cache.refs.sum().item() == 3


# ---- attention ---------------------------------------------------------------

def attend(cache, rng, counts, scale=None, **kw):
    import torch
    n, H = sum(counts), cache._heads
    q = rows(rng, (H, n, cache._latent), cache.dtype).transpose(0, 1)       # as a product over heads leaves it
    qr = rows(rng, (n, H, 128 + cache._rope), cache.dtype)[..., 128:]
    scale = (cache._latent + cache._rope) ** -0.5 if scale is None else scale
    out, lse = cache.attn(0, q, qr, starts_of(counts), scale, with_lse=True, **kw)
    return q, qr, scale, out, lse


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("latent,rope", [(512, 64), (512, 32), (256, 64), (256, 32)])
@pytest.mark.parametrize("heads,lens,counts", [
    (1, [1, 31, 32, 33], [1, 1, 1, 1]),
    (16, [64, 65, 200, 500], [1, 1, 1, 1]),
    (5, [3, 90, 31, 128], [3, 7, 1, 2]),
    (33, [1, 100], [1, 1]),
    (64, [130, 40], [1, 1])])
def test_attention_matches_64_bits(dtype, latent, rope, heads, lens, counts):
    rng = np.random.default_rng(heads + latent + rope)
    cache = make(heads, latent, rope, dtype, n_pages=20)
    fill(cache, rng, lens)
    q, qr, scale, out, lse = attend(cache, rng, counts)
    check(cache, q, qr, counts, scale, out, lse)
    assert cache.status() == 0


@pytest.mark.parametrize("dtype,heads,lens,counts,some", [
    ("bfloat16", 16, [5000], [1], None),                       # one token over many splits
    ("float16", 128, [3000, 700], [1, 1], (0, 1)),
    ("float16", 3, [1000, 64, 77, 2000], [40, 64, 1, 9], None),  # chunks
    ("bfloat16", 16, [700], [300], (0, 1, 137, 298, 299)),
    ("float16", 17, [300, 299], [300, 298], (0, 1, 31, 32, 63, 299, 300, 301, 597))])
def test_long_and_chunks(dtype, heads, lens, counts, some):
    rng = np.random.default_rng(heads + sum(lens))
    cache = make(heads, 512, 64, dtype, n_pages=120, seq_pages=80)
    fill(cache, rng, lens)
    q, qr, scale, out, lse = attend(cache, rng, counts)
    check(cache, q, qr, counts, scale, out, lse, some=some)


@pytest.mark.parametrize("seqs", [65, 200])
def test_many_sequences(seqs):
    """More sequences than a wave has lanes, of their own lengths, some of them empty."""
    rng = np.random.default_rng(seqs)
    cache = make(4, 256, 32, "float16", n_pages=3 * seqs, seqs=seqs, seq_pages=3)
    lens = fill(cache, rng, [int(x) for x in rng.integers(0, 150, seqs)])
    counts = [int(c) for c in rng.integers(0, 3, seqs)]
    q, qr, scale, out, lse = attend(cache, rng, counts)
    check(cache, q, qr, counts, scale, out, lse)
    assert cache.status() == 0 and len(lens) == seqs


@pytest.mark.parametrize("heads", [16, 64])
def test_empty_sequences_beside_ones_that_fill_the_chip(heads):
    """Rows of empty sequences take workgroups too: they come out as zeros, and the others whole."""
    rng = np.random.default_rng(14)
    seqs = 64
    cache = make(heads, 256, 32, "float16", n_pages=8 * 256, seqs=seqs, seq_pages=256)
    lens = [16384 if s % 8 == 3 else 0 for s in range(seqs)]
    fill(cache, rng, lens)
    counts = [1] * seqs
    q, qr, scale, out, lse = attend(cache, rng, counts)
    check(cache, q, qr, counts, scale, out, lse, some=[s for s in range(seqs) if s % 8 != 3] + [3, 35, 59])
    assert out[[s for s in range(seqs) if s % 8 == 3]].abs().sum(-1).all()


def test_rows_that_see_nothing():
    """Empty sequences, rows before the first token, missing pages, rows of nobody's."""
    import torch
    rng = np.random.default_rng(4)
    cache = make(heads=3, latent=256, rope=64, dtype="bfloat16")
    fill(cache, rng, [3, 0, 200, 100])
    table = cache.table.clone()
    table[2, 1] = -1
    table[3, 0] = -1
    table[3, 1] = -1
    cache.assign(cache.lens.clone(), table)
    cache.status_word.zero_()
    counts = [5, 2, 3, 2]
    q, qr = rows(rng, (14, 3, 256), "bfloat16"), rows(rng, (14, 3, 64), "bfloat16")
    out, lse = torch.full_like(q, 7.0), torch.full((14, 3), 7.0, device="cuda")
    got = cache.attn(0, q, qr, starts_of(counts), 0.06, out=out, lse=lse)
    assert got[0] is out and got[1] is lse
    check(cache, q, qr, counts, 0.06, out, lse)
    assert (out[12:] == 7).all() and (lse[12:] == 7).all() and not out[:2].any() and (lse[10:12] == -np.inf).all()


def test_malformed_starts_are_reported():
    import torch
    rng = np.random.default_rng(5)
    cache = make(heads=2, latent=256, rope=32)
    fill(cache, rng, [40, 50, 60])
    q, qr = rows(rng, (6, 2, 256), "bfloat16"), rows(rng, (6, 2, 32), "bfloat16")
    out, lse = torch.full_like(q, 7.0), torch.full((6, 2), 7.0, device="cuda")
    cache.attn(0, q, qr, ints([0, 2, 1, 4]), 0.1, out=out, lse=lse)         # the second descends; the third begins in the first's
    torch.cuda.synchronize()
    assert cache.status() == R.BAD_INDEX
    check(cache, q[:2], qr[:2], [2], 0.1, out[:2], lse[:2])
    assert (out[2:] == 7).all()


def test_a_query_that_is_not_finite_stays_in_its_row():
    import torch
    rng = np.random.default_rng(6)
    cache = make(heads=16, latent=512, rope=64)
    fill(cache, rng, [300, 50])
    q, qr = rows(rng, (2, 16, 512), "bfloat16"), rows(rng, (2, 16, 64), "bfloat16")
    clean = cache.attn(0, q, qr, starts_of([1, 1]), 0.04, with_lse=True)
    q[0, 3, 100], qr[1, 5, 9], q[1, 7, 0] = float("nan"), float("inf"), float("-inf")
    out, lse = cache.attn(0, q, qr, starts_of([1, 1]), 0.04, with_lse=True)
    bad = torch.zeros((2, 16), dtype=torch.bool, device="cuda")
    bad[0, 3] = bad[1, 5] = bad[1, 7] = True
    assert torch.isnan(out[bad]).all() and torch.isnan(lse[bad]).all()
    assert torch.equal(out[~bad], clean[0][~bad]) and torch.equal(lse[~bad], clean[1][~bad])


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("heads", [4, 20, 64])
def test_scores_far_apart(dtype, heads):
    """Scores that rise by hundreds along the sequence, or fall: the reference moves, or stays."""
    import torch
    rng = np.random.default_rng(7)
    for order in (1, -1):
        cache = make(heads, 256, 32, dtype)
        cache.reserve(ints([400, 0, 0, 0]))
        kv = rows(rng, (400, 288), dtype)
        rise = torch.linspace(0, 60, 400, device="cuda").to(kv.dtype)
        kv[:, 0] = rise if order > 0 else rise.flip(0)
        cache.append(0, kv[:, :256], kv[:, 256:], starts_of([400]), torch.zeros(16, device="cuda"))
        q, qr = rows(rng, (1, heads, 256), dtype), rows(rng, (1, heads, 32), dtype)
        q[..., 0] = 30.0
        out, lse = cache.attn(0, q, qr, starts_of([1]), 0.3, with_lse=True)
        check(cache, q, qr, [1], 0.3, out, lse)


def test_in_place_over_the_queries_and_repeats():
    import torch
    rng = np.random.default_rng(8)
    cache = make(heads=40, latent=512, rope=64, dtype="float16", n_pages=80, seq_pages=40)
    fill(cache, rng, [2000, 100])
    q, qr = rows(rng, (3, 40, 512), "float16"), rows(rng, (3, 40, 64), "float16")
    st = starts_of([1, 2])
    want = cache.attn(0, q, qr, st, 0.05, with_lse=True)
    for _ in range(3):
        again = cache.attn(0, q, qr, st, 0.05, with_lse=True)
        assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])
    assert cache.attn(0, q, qr, st, 0.05, out=q) is q and torch.equal(q, want[0])


def test_a_workspace_full_of_rubbish_and_no_rows():
    import torch
    rng = np.random.default_rng(15)
    cache = make(heads=16, latent=512, rope=64, n_pages=80, seq_pages=40)
    fill(cache, rng, [2000, 10])
    q, qr = rows(rng, (2, 16, 512), "bfloat16"), rows(rng, (2, 16, 64), "bfloat16")
    want = cache.attn(0, q, qr, starts_of([1, 1]), 0.05, with_lse=True)
    for fill_word in (float("nan"), 3.0, -1.0):
        cache.ws.fill_(fill_word)
        got = cache.attn(0, q, qr, starts_of([1, 1]), 0.05, with_lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    cache.ws.view(torch.int32).fill_(7)
    assert torch.equal(cache.attn(0, q, qr, starts_of([1, 1]), 0.05), want[0])
    none = cache.attn(0, q[:0], qr[:0], starts_of([0, 0]), 0.05, with_lse=True)
    assert none[0].shape == (0, 16, 512) and none[1].shape == (0, 16)
    f = torch.from_numpy(S.frequencies(64)).cuda()
    kv = rows(rng, (0, 576), "bfloat16")
    assert cache.append(0, kv[:, :512], kv[:, 512:], starts_of([0, 0]), f, q=qr[:0]).shape == (0, 16, 64)
    assert cache.status() == 0


def test_layers_are_their_own():
    rng = np.random.default_rng(9)
    cache = make(heads=2, latent=256, rope=32, n_layers=3, dtype="float16")
    fill(cache, rng, [70, 10])
    q, qr = rows(rng, (2, 2, 256), "float16"), rows(rng, (2, 2, 32), "float16")
    for layer in range(3):
        out, lse = cache.attn(layer, q, qr, starts_of([1, 1]), 0.06, with_lse=True)
        o, l = f64(out), f64(lse)
        for s in range(2):
            c, r = held(cache, s, [70, 10][s], layer)
            for h in range(2):
                want, wl, _ = S.attend(f64(q)[s, h], f64(qr)[s, h], c, r, 0.06)
                assert np.abs(o[s, h] - want).max() < 0.02 and abs(l[s, h] - wl) < 1e-4


def test_a_pool_past_4_gib():
    """Offsets of pages beyond 32 bits."""
    import torch
    rng = np.random.default_rng(10)
    cache = make(heads=2, latent=512, rope=64, dtype="float16", n_pages=62000, seq_pages=8, fill=0.0)
    assert cache.pool.numel() * 2 > 4 << 30
    table = torch.full((4, 8), -1, dtype=torch.int32, device="cuda")
    table[0, :3], table[1, 0] = ints([61999, 3, 60001]), 61000
    cache.assign(ints([150, 30, 0, 0]), table)
    kv = rows(rng, (180, 576), "float16")
    cache.append(0, kv[:, :512], kv[:, 512:], starts_of([150, 30]), torch.from_numpy(S.frequencies(64)).cuda())
    c, _ = cache.read(0, starts_of([150, 30]), 180)
    assert torch.equal(c, kv[:, :512])
    q, qr, scale, out, lse = attend(cache, rng, [2, 1])
    check(cache, q, qr, [2, 1], scale, out, lse)


def test_in_a_graph_with_growing_lengths():
    """reserve, append, attn captured once; lengths, pages and splits grow from replay to replay."""
    import torch
    rng = np.random.default_rng(11)
    a, b = (make(heads=6, latent=256, rope=32, dtype="float16", n_pages=40, seq_pages=20, fill=0.0) for _ in range(2))
    f = torch.from_numpy(S.frequencies(32)).cuda()
    one, st = ints([1, 1, 0, 1]), ints([0, 1, 2, 2, 3])
    kv, q, qr = (torch.zeros((3, *s), dtype=torch.float16, device="cuda") for s in ((288,), (6, 256), (6, 32)))
    first = rows(rng, (530, 288), "float16")
    for c in (a, b):
        c.reserve(ints([62, 447, 0, 21]))
        c.append(0, first[:, :256], first[:, 256:], starts_of([62, 447, 0, 21]), f)
    def step(c):
        c.reserve(one)
        t = c.append(0, kv[:, :256], kv[:, 256:], st, f, q=qr)
        return *c.attn(0, q, t, st, 0.06, with_lse=True), t
    step(a)
    step(b)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(a)
    for _ in range(5):
        for t in (kv, q, qr):
            t.copy_(rows(rng, tuple(t.shape), "float16"))
        want = step(b)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(a.pool, b.pool)
    check(b, q, want[2], [1, 1, 0, 1], 0.06, *want[:2])


def test_two_streams_with_a_workspace_each():
    import torch
    rng = np.random.default_rng(12)
    cache = make(heads=16, latent=512, rope=64, n_pages=200, seq_pages=100)
    fill(cache, rng, [4000, 2000])
    q, qr = rows(rng, (2, 16, 512), "bfloat16"), rows(rng, (2, 16, 64), "bfloat16")
    st = starts_of([1, 1])
    want = cache.attn(0, q, qr, st, 0.04)
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [torch.zeros_like(cache.ws) for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for stream, ws in zip(streams, spaces):
            with torch.cuda.stream(stream):
                got.append(cache.attn(0, q, qr, st, 0.04, workspace=ws))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in got)


def test_a_search_over_latents():
    """append, attn, choice, fork, reserve: lengths and tables follow the model, outputs 64 bits."""
    import torch
    import paper_2608_28911_amd as P
    rng = np.random.default_rng(13)
    n, V = 4, 97
    cache = make(heads=4, latent=256, rope=32, dtype="float16", n_pages=30, seqs=n, seq_pages=4)
    pages = R.Pages(30, n, 4)
    f = torch.from_numpy(S.frequencies(32)).cuda()
    fill(cache, rng, [63])
    pages.reserve([63, 0, 0, 0])
    cache.fork(ints([0] * n))
    pages.fork([0] * n)
    w = torch.from_numpy(rng.standard_normal((4 * 256, V)).astype(np.float32)).cuda()
    scores = torch.tensor([0.0] + [-np.inf] * (n - 1), device="cuda")
    for _ in range(4):
        cache.reserve(ints([1] * n))
        assert pages.reserve([1] * n)[0] == 0
        kv, q, qr = rows(rng, (n, 288), "float16"), rows(rng, (n, 4, 256), "float16"), rows(rng, (n, 4, 32), "float16")
        st = ints(range(n + 1))
        t = cache.append(0, kv[:, :256], kv[:, 256:], st, f, q=qr)
        out, lse = cache.attn(0, q, t, st, 0.06, with_lse=True)
        check(cache, q, t, [1] * n, 0.06, out, lse)
        logits = out.float().view(n, -1) @ w
        sc = scores.cpu().numpy()
        scores, parents, tokens = P.beam_select(logits, scores)
        t_, b_, v_ = S.choose(logits.cpu().double().numpy(), sc, n)
        assert parents.tolist() == list(b_) and tokens.tolist() == list(v_)
        cache.fork(parents)
        pages.fork(list(b_))
        assert cache.lens.tolist() == pages.lens and np.array_equal(cache.table.cpu().numpy(), pages.table())
    assert cache.status() == 0
