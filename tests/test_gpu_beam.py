"""GPU parity of beam search's choice with the plain model of tests/stepref.py.

Parents and tokens are equal.  A score is off by at most 2^-24 of itself (its
rounding to fp32) and what the row's sum leaves: each exponential is off by
(|x - m| + 3) u relative, u = 2^-24, those that matter by 20 u at most, and a lane's
fp32 sum of n / 256 of them by n / 256 u: ln sum by (20 + n / 256) u in all."""
import numpy as np
import pytest

from tests import stepref as S

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def run(logits, scores, k, ended=None, pad=0):
    import torch
    import paper_2608_28911_amd as P
    e = None if ended is None else torch.tensor(ended, dtype=torch.int32, device="cuda")
    s, p, t = P.beam_select(logits, torch.tensor(scores, dtype=torch.float32, device="cuda"), k=k, ended=e, pad=pad)
    return s.cpu().numpy(), p.cpu().numpy(), t.cpu().numpy()


def check(logits, scores, k, ended=None, pad=0):
    x = logits.detach().cpu().double().numpy()
    G, W, V = x.shape
    scores = np.asarray(scores, np.float32)
    got = run(logits, scores, k, ended, pad)
    for g in range(G):
        t, b, v = S.choose(x[g], scores[g], k, None if ended is None else ended[g], pad)
        assert np.array_equal(got[1][g], np.where(b < 0, -1, b + g * W)), (g, got[1][g], b)
        assert np.array_equal(got[2][g], v), (g, got[2][g], v)
        fine = np.isfinite(t)
        assert np.array_equal(np.isnan(t), np.isnan(got[0][g])) and np.array_equal(t[~fine & ~np.isnan(t)], got[0][g][~fine & ~np.isnan(t)])
        d = np.abs(got[0][g][fine] - t[fine])
        assert np.all(d <= U * np.abs(t[fine]) + (20 + V / 256) * U), d.max()
    return got


def logits_of(rng, shape, dtype):
    import torch
    x = rng.standard_normal(shape).astype(np.float32) * 2.5
    x[..., ::97] += 6.0 * rng.random(x[..., ::97].shape, np.float32)
    return torch.from_numpy(x).to(getattr(torch, dtype)).cuda()


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("G,W,V,k", [(1, 1, 1, 1), (1, 4, 7, 4), (3, 2, 33, 5), (2, 5, 1001, 10), (16, 8, 5021, 8), (1, 4, 50021, 4),
                                    (2, 64, 130, 64), (1, 1, 64, 64), (5, 3, 20000, 6)])
def test_matches_the_model(dtype, G, W, V, k):
    rng = np.random.default_rng(V + k)
    check(logits_of(rng, (G, W, V), dtype), -10 - 3 * rng.random((G, W)), k)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
def test_a_large_vocabulary_in_splits(dtype):
    rng = np.random.default_rng(1)
    check(logits_of(rng, (1, 4, 160001), dtype), [[-3.0, -2.5, -2.0, -8.0]], 32)
    check(logits_of(rng, (2, 3, 128000), dtype), -rng.random((2, 3)), 6)


def test_one_group_without_the_leading_dimension():
    import torch
    import paper_2608_28911_amd as P
    x = logits_of(np.random.default_rng(2), (4, 3000), "float32")
    s, p, t = P.beam_select(x, torch.zeros(4, device="cuda"))
    s3, p3, t3 = P.beam_select(x[None], torch.zeros((1, 4), device="cuda"), k=4)
    assert s.shape == p.shape == t.shape == (4,) and torch.equal(s, s3[0]) and torch.equal(p, p3[0]) and torch.equal(t, t3[0])


def test_strides():
    import torch
    rng = np.random.default_rng(3)
    big = logits_of(rng, (3, 5, 2 * 4097), "bfloat16")
    for x in (big[:, :4, 1:4098], big[:, ::2, :4001], big[1:, 1:3, 4096:], big.transpose(0, 1)[:2, :, 3:1000]):
        check(x, -rng.random(x.shape[:2]), 4)


@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("V", [37, 4099, 33333])
def test_ties_go_to_the_lower_beam_and_token(dtype, V):
    """Equal logits within rows, and rows and scores that are equal, wherever they lie in memory."""
    import torch
    rng = np.random.default_rng(V)
    x = torch.from_numpy(rng.integers(-3, 3, (1, 1, V)).astype(np.float32)).to(getattr(torch, dtype)).cuda()
    same = x.expand(2, 4, V).contiguous()
    got = check(same, np.full((2, 4), -1.25), 12)
    top = np.flatnonzero(x.cpu().float().numpy()[0, 0] == 2)
    assert list(got[2][0]) == list(top[:12]) if len(top) >= 12 else True
    check(torch.zeros((1, 3, V), dtype=x.dtype, device="cuda"), [[0.0, 0.0, 0.0]], 5)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("G,W,V,k", [(1, 64, 20001, 64), (1, 2, 131073, 64), (2, 17, 17000, 40), (1, 7, 70000, 33),
                                    (1, 33, 40000, 5), (3, 3, 90000, 50)])
def test_many_candidates(dtype, G, W, V, k):
    """Lists of many beams, of many splits, of both; widths that are no powers of two; beams not in use, and ended ones."""
    rng = np.random.default_rng(W * k)
    x = logits_of(rng, (G, W, V), dtype)
    scores = -4 - 2 * rng.random((G, W)).astype(np.float32)
    check(x, scores, k)
    ended = (rng.random((G, W)) < 0.3).astype(np.int32)
    scores[rng.random((G, W)) < 0.3] = -np.inf
    check(x, scores, k, ended, pad=9)


@pytest.mark.parametrize("every", [1, 7, 1400, 2800])
def test_many_ties(every):
    """The k-th largest of 64 ties with all, with a seventh, or with some 100 or 50 of 140000 logits: a few more than k, or
    more than there is room to count."""
    import torch
    x = torch.full((1, 3, 140000), -2.0, device="cuda")
    x[..., 5::every] = 1.5
    x[0, 1, 139000:139010] = 2.0
    got = check(x, [[-1.0, -1.0, -1.0]], 64)
    assert list(got[1][0][:10]) == [1] * 10 and list(got[2][0][:10]) == list(range(139000, 139010))
    check(x[:, :1], [[-1.0]], 64)
    check(x[:, :, :20000].expand(1, 3, 20000), [[-1.0, -1.0, -1.5]], 60)


def test_first_step_ended_beams_and_empty_rows():
    rng = np.random.default_rng(5)
    x = logits_of(rng, (4, 4, 700), "float16")
    inf = float("inf")
    x[2, 1] = -inf                                        # nothing to go on with
    x[2, 2, 5:] = -inf                                    # five tokens
    x[3] = float("nan")                                   # never looked at
    scores = [[0.0, -inf, -inf, -inf], [-9.0, -2.0, -30.0, -9.5], [-1.0, -0.5, -0.25, -inf], [-3.0, -1.0, -2.0, -inf]]
    ended = [[0, 0, 0, 0], [0, 1, 1, 0], [1, 0, 0, 1], [1, 1, 1, 0]]
    got = check(x, scores, 8, ended, pad=2)
    assert list(got[1][3]) == [13, 14, 12] + [-1] * 5 and list(got[2][3]) == [2, 2, 2] + [-1] * 5
    assert list(got[0][3][:3]) == [-1.0, -2.0, -3.0] and np.all(got[0][3][3:] == -inf)
    assert np.sum(got[1][2] >= 0) == 6


def test_what_is_not_finite_is_reported():
    import torch
    rng = np.random.default_rng(6)
    x = logits_of(rng, (5, 2, 900), "float32")
    x[0, 1, 17] = float("nan")
    x[1, 0, 899] = float("inf")
    scores = np.float32([[0, 0], [0, 0], [np.nan, 0], [0, np.inf], [0, 0]])
    got = check(x, scores, 3)
    assert np.isnan(got[0][:4]).all() and (got[1][:4] == -1).all() and (got[2][:4] == -1).all() and (got[1][4] >= 0).all()


@pytest.mark.parametrize("dtype", ["float16", "float32"])
def test_masks_of_the_types_lowest_value(dtype):
    import torch
    dt = getattr(torch, dtype)
    x = torch.full((1, 2, 2050), torch.finfo(dt).min, dtype=dt, device="cuda")
    check(x, [[-1.0, -1.5]], 4)                            # all alike: a uniform distribution
    x[0, 1, 2047:] = 1.0
    check(x, [[-1.0, -1.5]], 6)
    x[0, 0, 100] = torch.finfo(dt).max
    check(x, [[-1.0, -1.5]], 4)


def test_repeats_itself_and_leaves_its_inputs():
    import torch
    import paper_2608_28911_amd as P
    x = logits_of(np.random.default_rng(7), (8, 4, 30011), "bfloat16")
    sc = -torch.rand((8, 4), device="cuda")
    keep = x.clone(), sc.clone()
    first = P.beam_select(x, sc, k=8)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, P.beam_select(x, sc, k=8)))
    assert torch.equal(x, keep[0]) and torch.equal(sc, keep[1])


def test_in_a_graph_and_on_another_stream():
    import torch
    import paper_2608_28911_amd as P
    rng = np.random.default_rng(8)
    x, sc = logits_of(rng, (2, 4, 40000), "float16"), torch.zeros((2, 4), device="cuda")
    P.beam_select(x, sc)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = P.beam_select(x, sc)
    side = torch.cuda.Stream()
    for _ in range(4):
        x.copy_(logits_of(rng, (2, 4, 40000), "float16"))
        want = P.beam_select(x, sc)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other = P.beam_select(x, sc)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(other, want))


def test_a_search_over_the_cache():
    """append, attn, choice, fork, reserve: two searches of three beams, against tables kept by hand."""
    import torch
    import paper_2608_28911_amd as P
    from tests import pagedref as R
    from tests.test_gpu_paged import ints, make, rows
    rng = np.random.default_rng(9)
    S2, W, V, D = 2, 3, 211, 128
    n = S2 * W
    cache = make(h=1, hq=2, d=D, g=128, n_pages=40, seqs=n, seq_pages=4, fill=0)
    pages = R.Pages(40, n, 4)
    f = torch.from_numpy(S.frequencies(D)).cuda()
    w = torch.from_numpy(rng.standard_normal((2 * D, V)).astype(np.float32)).cuda()
    up = [60, 0, 0, 62, 0, 0]                              # prompts in each search's first slot
    cache.reserve(ints(up))
    pages.reserve(up)
    k, v = rows(rng, (122, 1, D), torch.float16), rows(rng, (122, 1, D), torch.float16)
    cache.append(0, k, v, ints([0, 60, 60, 60, 122, 122, 122]), f)
    cache.fork(ints([0, 0, 0, 3, 3, 3]))
    pages.fork([0, 0, 0, 3, 3, 3])
    scores = torch.tensor([[0.0, -np.inf, -np.inf]] * S2, device="cuda")
    hist = [[] for _ in range(n)]
    for step in range(6):
        one = [1] * n
        cache.reserve(ints(one))
        st, _ = pages.reserve(one)
        assert st == 0
        k, v, q = (rows(rng, (n, h, D), torch.float16) for h in (1, 1, 2))
        starts = ints(range(n + 1))
        q = cache.append(0, k, v, starts, f, q=q)
        h = cache.attn(0, q, starts)
        logits = (h.float().view(n, -1) @ w).view(S2, W, V)
        x, sc = logits.cpu().double().numpy(), scores.cpu().numpy()
        scores, parents, tokens = P.beam_select(logits, scores)
        want = [S.choose(x[s], sc[s], W) for s in range(S2)]
        par = np.concatenate([wb + s * W for s, (_, wb, _) in enumerate(want)])
        assert parents.flatten().tolist() == par.tolist()
        assert tokens.flatten().tolist() == np.concatenate([t for _, _, t in want]).tolist()
        hist = [hist[p] + [t] for p, t in zip(parents.flatten().tolist(), tokens.flatten().tolist())]
        cache.fork(parents.flatten())
        assert pages.fork(par.tolist()) == 0
        assert cache.lens.tolist() == pages.lens and np.array_equal(cache.table.cpu().numpy(), pages.table())
        assert cache.refs.tolist() == pages.refs()
    assert cache.status() == 0 and all(len(t) == 6 for t in hist)
