"""GPU parity of append with rotation, the cache of latents and beam search's choice
where they went wrong once, with the plain models of tests/stepref.py."""
import numpy as np
import pytest

from tests import stepref as S
from tests.test_gpu_paged import ints, starts_of

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


# ---- beam search's choice ----------------------------------------------------
#
# Tolerance of a score, from the arithmetic: a logit's exponential e^-y, y below its lane's maximum so far, takes y, its
# product with log2 e (0.23 u off itself) and the power of two (1 ulp: 2 u): (2.23 y + 2) u relative; up to eight of them
# are added in fp32: 3 u; the rest is in 64 bits.  Weighted by the exponentials themselves y is ln vocab on average at
# most (it is no more than the row's entropy).  So ln sum is off by (2.23 ln vocab + 5) u, and t by its rounding too.

def tolerance(t, vocab):
    return (2.23 * np.log(vocab) + 5) * U + U * np.abs(t)


def chosen(logits, scores, k):
    import torch
    import paper_2608_28911_amd as P
    out = P.beam_select(logits, torch.tensor(np.asarray(scores, np.float32), device="cuda"), k=k)
    return [t.cpu().numpy() for t in out]


def small_beside_one(dtype, vocab=160000):
    """A row in which every lane of a workgroup meets a 0 first, and then sums that are each less than half a step of
    1 in fp32 but not together."""
    import torch
    wide = 4 if dtype == "float32" else 8                  # logits of a lane at a time
    x = torch.full((vocab,), -18.25 if wide == 4 else -19.0)
    x[:256 * wide:wide] = 0.0
    return x.to(getattr(torch, dtype)).cuda()


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
def test_many_small_exponentials_beside_a_large_one(dtype):
    x = small_beside_one(dtype)
    scores = np.float32(-0.25) * np.arange(60)[None].repeat(5, 0)
    t, b, v = S.choose(x.cpu().double().numpy()[None], [0.0], 8)
    got = chosen(x.expand(5, 60, -1), scores, 8)             # 300 rows: a workgroup each
    assert (got[1] == 60 * np.arange(5)[:, None]).all() and (got[2] == v).all()
    assert np.all(np.abs(got[0] - t) <= tolerance(t, x.numel())), np.abs(got[0] - t).max()


def test_beams_that_such_sums_put_in_order():
    """ln sum of the first row is 7.4e-6 above the second's, whose score is 4.5e-6 lower: the second comes first."""
    import torch
    x = torch.stack([small_beside_one("float32"), small_beside_one("float32")])
    x[1][x[1] != 0] = -np.inf
    scores = np.float32([[0.0, -4.5e-6]]).repeat(150, 0)
    t, b, v = S.choose(x.cpu().double().numpy(), scores[0], 4)
    assert list(b) == [1] * 4 and S.choose(x.cpu().double().numpy(), scores[0], 300)[1][299] == 0
    got = chosen(x.expand(150, 2, -1), scores, 4)
    assert (got[1] == 2 * np.arange(150)[:, None] + 1).all() and (got[2] == v).all()


@pytest.mark.parametrize("rows", [1, 4, 300])
@pytest.mark.parametrize("vocab", [1000, 64000])
def test_logits_that_are_log_probabilities_already(rows, vocab):
    """ln sum is 0 but for their rounding."""
    import torch
    rng = np.random.default_rng(vocab + rows)
    x = rng.standard_normal((2, vocab)) * 2.5
    x -= np.log(np.exp(x).sum(-1, keepdims=True))
    x = x.astype(np.float32)
    got = chosen(torch.from_numpy(x).cuda().expand(rows, 2, -1), np.zeros((rows, 2)), 12)
    t, b, v = S.choose(x, [0.0, 0.0], 12)
    assert (got[1] == 2 * np.arange(rows)[:, None] + b).all() and (got[2] == v).all()
    assert np.all(np.abs(got[0] - t) <= tolerance(t, vocab)), np.abs(got[0] - t).max()


@pytest.mark.parametrize("dtype", ["float16", "float32"])
def test_logits_that_rise_and_fall(dtype):
    """A maximum that moves at every vector of a lane, or never again."""
    import torch
    vocab = 50000
    x = np.linspace(-20, 3, vocab)
    x = torch.from_numpy(np.stack([x, x[::-1]])).to(getattr(torch, dtype)).cuda()
    got = chosen(x.expand(200, 2, -1), np.float32([[0.0, -1e-3]]).repeat(200, 0), 5)
    t, b, v = S.choose(x.cpu().double().numpy(), np.float32([0.0, -1e-3]), 5)
    assert (got[1] == 2 * np.arange(200)[:, None] + b).all() and (got[2] == v).all()
    assert np.all(np.abs(got[0] - t) <= tolerance(t, vocab)), np.abs(got[0] - t).max()


# ---- rows before their sequence's first token ----------------------------------

def took(f, repeats=5):
    """The smallest of some times of f, in us."""
    import torch
    f()
    best = np.inf
    for _ in range(repeats):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        b.synchronize()
        best = min(best, 1e3 * a.elapsed_time(b))
    return best


def test_a_prompt_whose_reserve_has_failed():
    """All of its rows precede the sequence's first token: their queries, and what is read, are zeros, written by the
    whole grid (one lane for all of them took a thousand times as long as the prompt with room does)."""
    import torch
    from tests import pagedref as R
    from tests.test_gpu_paged import make
    n, h, hq = 4096, 2, 16
    caches = make(h=h, hq=hq, n_pages=4, seqs=2, seq_pages=64), make(h=h, hq=hq, n_pages=64, seqs=2, seq_pages=64)
    k, v = (torch.randn((n, h, 128), device="cuda").half() for _ in range(2))
    q = torch.randn((n, hq, 128), device="cuda").half()
    f, st = torch.from_numpy(S.frequencies(128)).cuda(), starts_of([0, n])
    us = []
    for c in caches:
        c.reserve(ints([0, n]))
        out = torch.full_like(q, 7.0)
        us.append(took(lambda: c.append(0, k, v, st, f, q=q, q_out=out)))
        back = tuple(torch.full((n, h, 128), 7.0, dtype=q.dtype, device="cuda") for _ in range(2))
        us.append(took(lambda: c.read(0, st, n, out=back)))
        if c is caches[0]:
            assert c.status() == R.NO_PAGES | R.BAD_INDEX and c.lens.tolist() == [0, 0]
            assert not out.any() and not back[0].any() and not back[1].any()
        else:
            assert c.status() == 0 and out.abs().amax(-1).all()
    assert us[0] <= 20 * us[2] and us[1] <= 20 * us[3], us


def test_a_prompt_of_latents_whose_reserve_has_failed():
    import torch
    from tests import pagedref as R
    from tests.test_gpu_latent import make
    n, heads = 4096, 16
    caches = [make(heads=heads, latent=256, rope=64, dtype="float16", n_pages=m, seqs=2, seq_pages=64, fill=0.0) for m in (4, 64)]
    kv, q = torch.randn((n, 320), device="cuda").half(), torch.randn((n, heads, 64), device="cuda").half()
    f, st = torch.from_numpy(S.frequencies(64)).cuda(), starts_of([n, 0])
    us = []
    for c in caches:
        c.reserve(ints([n, 0]))
        out = torch.full_like(q, 7.0)
        us.append(took(lambda: c.append(0, kv[:, :256], kv[:, 256:], st, f, q=q, q_out=out)))
        back = torch.full((n, 256), 7.0, dtype=q.dtype, device="cuda"), torch.full((n, 64), 7.0, dtype=q.dtype, device="cuda")
        us.append(took(lambda: c.read(0, st, n, out=back)))
        if c is caches[0]:
            assert c.status() == R.NO_PAGES | R.BAD_INDEX
            assert not out.any() and not back[0].any() and not back[1].any()
        else:
            assert c.status() == 0 and out.abs().amax(-1).all() and torch.equal(back[0], kv[:, :256])
    assert us[0] <= 20 * us[2] and us[1] <= 20 * us[3], us


@pytest.mark.parametrize("lens,counts", [
    ([0], [1]), ([1], [2]), ([0, 5, 64], [1, 1, 1]), ([64, 3], [64, 70]), ([10, 0, 130, 1], [5, 100, 130, 1]),
    ([63, 64, 65, 128], [64, 65, 66, 129]), ([0] * 70 + [9] * 70, [1] * 70 + [10, 1] * 35), ([200] * 3 + [0], [150, 1, 201, 300])])
def test_rows_before_the_first_token_beside_others(lens, counts):
    """Whoever has no page takes them: there is such a workgroup where there is such a row."""
    import torch
    from tests.test_gpu_latent import make as make_latents
    from tests.test_gpu_paged import make
    n, seqs = sum(counts), len(lens)
    st, pages = starts_of(counts), 4 * seqs
    early = np.concatenate([np.arange(m) < m - ln for ln, m in zip(lens, counts)])
    early_d = torch.from_numpy(early).cuda()
    a = make(h=3, hq=6, d=64, g=32, n_pages=pages, seqs=seqs, seq_pages=4)
    b = make_latents(heads=5, latent=256, rope=32, dtype="float16", n_pages=pages, seqs=seqs, seq_pages=4, fill=1.0)
    for c in (a, b):
        c.reserve(ints(lens))
    k, v, q = (torch.rand((n, m, 64), device="cuda").half() + 0.5 for m in (3, 3, 6))
    out = torch.full((n + 3, 6, 64), 7.0, dtype=q.dtype, device="cuda")
    a.append(0, k, v, st, torch.zeros(32, device="cuda"), q=q, q_out=out[:n])
    assert torch.equal(out[:n], q.masked_fill(early_d[:, None, None], 0.0)) and (out[n:] == 7).all()
    for x in a.read(0, st, n, out=tuple(torch.full((n, 3, 64), 7.0, device="cuda") for _ in range(2))):
        assert not x[early_d].any() and (x[~early_d] > 0.4).all() and (x[~early_d] < 1.6).all()
    kv, qr = torch.rand((n, 288), device="cuda").half() + 0.5, torch.rand((n, 5, 32), device="cuda").half() + 0.5
    out = torch.full((n + 3, 5, 32), 7.0, dtype=q.dtype, device="cuda")
    b.append(0, kv[:, :256], kv[:, 256:], st, torch.zeros(16, device="cuda"), q=qr, q_out=out[:n])
    assert torch.equal(out[:n], qr.masked_fill(early_d[:, None, None], 0.0)) and (out[n:] == 7).all()
    back = torch.full((n, 256), 7.0, dtype=q.dtype, device="cuda"), torch.full((n, 32), 7.0, dtype=q.dtype, device="cuda")
    for x, want in zip(b.read(0, st, n, out=back), (kv[:, :256], kv[:, 256:])):
        assert torch.equal(x, want.masked_fill(early_d[:, None], 0.0))


# ---- attention over latents -------------------------------------------------------

@pytest.mark.parametrize("heads", [4, 20, 64])
def test_infinite_scores(heads):
    """A score of +inf or NaN makes its row NaN, one of -inf has no weight; only such: as a row that sees nothing."""
    import torch
    from tests.test_gpu_latent import make, rows
    rng = np.random.default_rng(heads)
    n, inf = 700, float("inf")
    cache = make(heads=heads, latent=256, rope=32, dtype="bfloat16", n_pages=16, seqs=2, seq_pages=12)
    cache.reserve(ints([n, 0]))
    kv = rows(rng, (n, 288), "bfloat16")
    kv[:, 0], kv[:, 1] = 1.0, 0.0
    kv[::3, 1], kv[5, 1] = 4.0, 4.0
    cache.append(0, kv[:, :256], kv[:, 256:], starts_of([n, 0]), torch.zeros(16, device="cuda"))
    q, qr = rows(rng, (3, heads, 256), "bfloat16"), rows(rng, (3, heads, 32), "bfloat16")
    q[..., :2] = 0.0
    q[0, ::2, 0], q[1, ::2, 0], q[1, 1::2, 0], q[2, :, 1] = -inf, inf, float("nan"), -3e38      # -1.2e39 of every third token
    out, lse = cache.attn(0, q, qr, starts_of([3, 0]), 0.06, with_lse=True)
    assert cache.status() == 0
    assert not out[0, ::2].any() and (lse[0, ::2] == -inf).all()
    assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all()
    c, r = (t.cpu().double().numpy() for t in (kv[:, :256], kv[:, 256:]))
    for i, some in ((0, range(1, heads, 2)), (2, range(heads))):
        seen = np.arange(n - 2 + i)
        if i == 2:
            seen = seen[(seen % 3 != 0) & (seen != 5)]
        for h in some:
            a, b = q[i, h].cpu().double().numpy(), qr[i, h].cpu().double().numpy()
            a[1] = 0.0
            want, wl, p = S.attend(a, b, c[seen], r[seen], 0.06)
            # scores' roundings (288 products, two operations, and the exponent's), the weights', the sums', the output's
            x = 0.06 * (np.abs(c[seen]) @ np.abs(a) + np.abs(r[seen]) @ np.abs(b)).max()
            d = (296 + 3) * U * x + 48 * U
            tol = (2.0 ** -8 + 2 * d + n * U) * (p @ np.abs(c[seen])) + (2.0 ** -8 + d + n * U) * np.abs(want)
            assert np.all(np.abs(out[i, h].cpu().double().numpy() - want) <= tol)
            assert abs(lse[i, h].item() - wl) <= 2 * d + n * U + U * abs(wl)


@pytest.mark.parametrize("dtype,heads,latent,rope", [("bfloat16", 16, 512, 64), ("float16", 7, 256, 32), ("float16", 16, 512, 32)])
def test_slots_without_rows_beside_a_chunk(dtype, heads, latent, rope):
    """The height of attention's tiles goes by the rows a slot has on average: the same chunk among 1 to 64 slots takes
    tiles of 64, 32 and 16 rows, and each of them is held to 64 bits."""
    from tests.test_gpu_latent import check, fill, make, rows
    rng = np.random.default_rng(heads + latent)
    cache = make(heads=heads, latent=latent, rope=rope, dtype=dtype, n_pages=16, seqs=64, seq_pages=16)
    m, n = 60, 900
    fill(cache, rng, [n])
    q, qr = rows(rng, (m, heads, latent), dtype), rows(rng, (m, heads, rope), dtype)
    heights = set()
    for slots in (1, 40, 64):
        counts = [m] + [0] * (slots - 1)
        per = -(-m * heads // slots)
        heights.add(16 if per <= 16 else 32 if per <= 32 else 64)
        out, lse = cache.attn(0, q, qr, starts_of(counts), 0.05, with_lse=True)
        check(cache, q, qr, [m], 0.05, out, lse)
    assert len(heights) == (3 if heads == 16 else 2)
    assert cache.status() == 0


@pytest.mark.parametrize("heads,lens", [
    (16, [40000]),                                           # as many splits as a tile may have
    (40, [33000]),
    (16, [int(x) for x in np.random.default_rng(1).integers(100, 3000, 40)]),     # shares that have to grow until they suffice
    (64, [int(x) for x in np.random.default_rng(2).integers(1, 2000, 60)]),
    (20, [int(x) for x in np.random.default_rng(3).integers(1, 1500, 100)])])     # more sequences than a wave has lanes
def test_splits_of_many_lengths(heads, lens):
    from tests.test_gpu_latent import attend, check, fill, make
    rng = np.random.default_rng(heads)
    pages = sum((n + 63) // 64 for n in lens)
    cache = make(heads=heads, latent=256, rope=32, dtype="float16", n_pages=pages, seqs=len(lens), seq_pages=(max(lens) + 63) // 64)
    fill(cache, rng, lens)
    counts = [1] * len(lens)
    q, qr, scale, out, lse = attend(cache, rng, counts)
    some = None if len(lens) == 1 else set(range(0, len(lens), 7)) | {int(np.argmin(lens)), int(np.argmax(lens))}
    check(cache, q, qr, counts, scale, out, lse, some=some)
    again = cache.attn(0, q, qr, starts_of(counts), scale, with_lse=True)
    assert (again[0] == out).all() and (again[1] == lse).all() and cache.status() == 0


def test_compact_of_latents_whose_page_is_missing():
    """Tokens kept from a missing page are zeros, and reported; the others move."""
    import torch
    from tests import pagedref as R
    from tests.test_gpu_latent import make, rows
    rng = np.random.default_rng(3)
    cache = make(heads=1, latent=512, rope=32, dtype="float16", n_layers=2, n_pages=12, seqs=2, seq_pages=4)
    cache.reserve(ints([200, 30]))
    f, kv = torch.zeros(16, device="cuda"), [rows(rng, (230, 544), "float16") for _ in range(2)]
    for layer in range(2):
        cache.append(layer, kv[layer][:, :512], kv[layer][:, 512:], starts_of([200, 30]), f)
    table = cache.table.clone()
    table[0, 1] = -1                                          # tokens 64 .. 127
    cache.assign(cache.lens.clone(), table)
    cache.status_word.zero_()
    kept = sorted(rng.permutation(200)[:90].tolist())
    cache.compact(ints([kept, [0] * 90]), ints([90, -1]))
    assert cache.status() == R.BAD_INDEX and cache.lens.tolist() == [90, 30] and cache.refs.sum().item() == 3
    gone = torch.tensor([64 <= t < 128 for t in kept], device="cuda")
    for layer in range(2):
        c, r = cache.read(layer, starts_of([90, 30]), 120)
        want = torch.cat((kv[layer][kept].masked_fill(gone[:, None], 0.0), kv[layer][200:]))
        assert torch.equal(c, want[:, :512]) and torch.equal(r, want[:, 512:])
