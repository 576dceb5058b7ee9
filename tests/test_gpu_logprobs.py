"""GPU parity of token_logprobs and score_tokens with 64-bit values.

Tolerance, from the arithmetic (u = 2^-24, half a step of fp32).  Every e^(x-m)
carries the rounding of x - m and of its product with log2 e (2 u |x - m|
relative, and 2 u |x - m| e^(x-m) is below u for any x) and the exponential's
2 u; lanes' sums are chains of at most n/256 + 16 rescaled additions, so ln S
is off by at most (n/256 + 40) u, and its own rounding u |ln S|.  A log
probability x - m - ln S adds 2 u |logp| + u |x - m|.  The entropy's T is
likewise off by (n/256 + 40) u sum p |x - m|."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DT = ["float16", "bfloat16", "float32"]


def exact(x, ids, top):
    """64-bit values of rows x [N, V] (float64)."""
    n, v = x.shape
    with np.errstate(all="ignore"):
        m = x.max(1, keepdims=True)
        e = np.exp(x - m)
        S = e.sum(1)
        logp = (x[np.arange(n), np.clip(ids, 0, v - 1)] - m[:, 0]) - np.log(S)
        y = np.where(e > 0, x - m, 0.0)
        spread = (e * -y).sum(1) / S
        ent = np.log(S) + spread
        order = np.lexsort((np.broadcast_to(np.arange(v), x.shape), -x), axis=1)[:, :top]
        tl = np.take_along_axis(x, order, 1) - m - np.log(S)[:, None]
    return logp, ent, tl, order, m[:, 0], S, spread


def check(x, ids, top, got):
    import torch
    x64 = x.double().cpu().numpy()
    n, v = x64.shape
    ids = ids.cpu().numpy()
    logp, ent, tl, order, m, S, spread = exact(x64, ids, top)
    base = (v / 256 + 40) * U + U * np.abs(np.log(S))
    with np.errstate(all="ignore"):
        lim = base + 4 * U * np.abs(logp)
    g = got[0].cpu().numpy()
    fin = np.isfinite(logp)
    assert np.all(np.abs(g - logp)[fin] <= lim[fin]), float((np.abs(g - logp) / lim)[fin].max())
    assert np.array_equal(g[~fin], logp[~fin].astype(np.float32))
    assert np.all(np.abs(got[1].cpu().numpy() - ent) <= base + (v / 256 + 40) * U * spread + 2 * U * np.abs(ent))
    if top:
        assert np.array_equal(got[3].cpu().numpy(), order)
        t = got[2].cpu().numpy()
        fin = np.isfinite(tl)
        assert np.all(np.abs(t - tl)[fin] <= (base[:, None] + 4 * U * np.abs(tl))[fin])
        assert np.array_equal(t[~fin], tl[~fin].astype(np.float32))


def draw(rng, n, v, dtype, mul=3.0):
    import torch
    return torch.from_numpy((rng.standard_normal((n, v)) * mul).astype(np.float32)).to(getattr(torch, dtype)).cuda()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("v", [1, 2, 7, 8, 9, 63, 64, 65, 1000, 2049, 32003, 131072])
def test_rows_of_many_sizes(v, dtype):
    """Sizes around the vectors' and waves' ends; rows of odd sizes begin
    anywhere.  16-bit logits tie often: the lowest index comes first."""
    import torch
    import paper_2608_28911_amd as P
    rng = np.random.default_rng(v)
    for n, top in ((1, min(v, 5)), (3, 0), (37, min(v, 32))):
        x = draw(rng, n, v, dtype)
        ids = torch.from_numpy(rng.integers(0, v, n)).cuda()
        check(x, ids, top, P.token_logprobs(x, ids, top=top))


@pytest.mark.parametrize("dtype", DT)
def test_orders_and_ties(dtype):
    """Ascending, descending, constant rows, few values, a last element above."""
    import torch
    import paper_2608_28911_amd as P
    v = 20011
    up = torch.arange(v, dtype=torch.float32) / 1500
    x = torch.stack((up, -up, torch.full((v,), 2.0), (torch.arange(v) * 7919 % 4).float(), torch.zeros(v)))
    x[4, -1], x[4, 1::2] = 9.0, -0.0                     # -0 and +0 are equal
    x = x.to(getattr(torch, dtype)).cuda()
    ids = torch.tensor([0, v - 1, 5, 77, v - 1]).cuda()
    for top in (1, 20, 32):
        check(x, ids, top, P.token_logprobs(x, ids, top=top))


@pytest.mark.parametrize("dtype", DT)
def test_masked_logits(dtype):
    """-inf and the type's lowest value as masks: whole vectors of them, all but
    one, fewer left than asked for."""
    import torch
    import paper_2608_28911_amd as P
    rng = np.random.default_rng(5)
    dt = getattr(torch, dtype)
    v = 5003
    x = draw(rng, 6, v, dtype)
    low = torch.finfo(dt).min
    x[0, 100:] = -float("inf")
    x[1, 100:] = low
    x[2] = -float("inf")
    x[2, 4000] = 1.0
    x[3] = low
    x[4, ::2] = -float("inf")
    x[5, :] = -float("inf")
    x[5, [7, 4999, 12]] = 3.0
    ids = torch.tensor([50, 3, 4000, 11, 3, 8]).cuda()   # the last is masked: logp -inf
    check(x, ids, 10, P.token_logprobs(x, ids, top=10))


@pytest.mark.parametrize("dtype", DT)
def test_rows_without_a_finite_sum(dtype):
    import torch
    import paper_2608_28911_amd as P
    rng = np.random.default_rng(6)
    for v in (1001, 40000):                              # one workgroup a row, and several
        x = draw(rng, 4, v, dtype)
        x[0, 700], x[1, 3] = float("nan"), float("inf")
        x[2] = -float("inf")
        ids = torch.tensor([1, 2, 3, 4]).cuda()
        got = P.token_logprobs(x, ids, top=3)
        for g in got[:3]:
            assert torch.isnan(g[:3]).all() and torch.isfinite(g[3]).all()
        assert (got[3][:3] == -1).all() and (got[3][3] >= 0).all()
        check(x[3:], ids[3:], 3, [g[3:] for g in got])


def test_targets_that_are_none():
    import torch
    import paper_2608_28911_amd as P
    x = draw(np.random.default_rng(7), 4, 500, "float16")
    ids = torch.tensor([-1, -2, 500, 499]).cuda()
    logp, ent = P.token_logprobs(x, ids)
    assert float(logp[0]) == 0.0 and torch.isnan(logp[1:3]).all() and torch.isfinite(ent).all()
    check(x[3:], ids[3:], 0, (logp[3:], ent[3:]))
    assert float(P.score_tokens(x, ids)[0]) == 0.0


@pytest.mark.parametrize("dtype", DT)
def test_strides_and_scores_of_a_prompt(dtype):
    """[B, T, V] logits inside a wider buffer, targets a position ahead, scores
    into a slice: what the ranking takes."""
    import torch
    import paper_2608_28911_amd as P
    rng = np.random.default_rng(8)
    B, T, V = 3, 17, 777
    big = draw(rng, B * T, V + 6, dtype).view(B, T, V + 6)
    logits = big[:, :, 1:V + 1]
    ids = torch.from_numpy(rng.integers(0, V, (B, T))).cuda()
    scores = torch.full((B, T), 5.0, device="cuda")
    got = P.score_tokens(logits[:, :-1], ids[:, 1:], scores=scores[:, 1:])
    assert got.data_ptr() == scores[:, 1:].data_ptr() and torch.all(scores[:, 0] == 5.0)
    flat = logits[:, :-1].reshape(-1, V)
    lp = P.token_logprobs(logits[:, :-1], ids[:, 1:], top=4)
    assert torch.equal(-lp[0], scores[:, 1:])
    check(flat, ids[:, 1:].reshape(-1), 4, [t.reshape((-1,) + t.shape[2:]) for t in lp])
    empty = P.token_logprobs(logits[:, :0], ids[:, :0])
    assert empty[0].shape == (B, 0)


def test_extreme_logits():
    """Far apart, all near a type's ends, tiny differences on a large offset."""
    import torch
    import paper_2608_28911_amd as P
    rng = np.random.default_rng(9)
    x = torch.from_numpy(rng.standard_normal((4, 3001)).astype(np.float32)).cuda()
    x[0] *= 1e30
    x[1] += 1e4
    x[2] = 3.3e38
    x[3] = x[3] * 100 - 3e38
    ids = torch.from_numpy(rng.integers(0, 3001, 4)).cuda()
    check(x, ids, 3, P.token_logprobs(x, ids, top=3))


def test_captured_into_a_graph():
    import torch
    import paper_2608_28911_amd as P
    rng = np.random.default_rng(10)
    x, ids = draw(rng, 2, 50000, "bfloat16"), torch.tensor([3, 4]).cuda()
    P.token_logprobs(x, ids, top=5)
    torch.cuda.synchronize()
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=side):
        got = P.token_logprobs(x, ids, top=5)
    for i in range(4):
        x.copy_(draw(rng, 2, 50000, "bfloat16"))
        g.replay()
        torch.cuda.synchronize()
        want = P.token_logprobs(x, ids, top=5)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
