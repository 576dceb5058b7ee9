"""GPU parity of append with rotation, the cache of latents and beam search's choice
where they went wrong once, with the plain models of tests/stepref.py."""
import numpy as np
import pytest

from tests import stepref as S

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
