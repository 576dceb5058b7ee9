"""GPU parity of append with rotation with the plain models of tests/stepref.py and
tests/pagedref.py.

Turned queries, codes and metadata are compared bit for bit: every step is defined
to its rounding.  The one step that is not is the cosine's and sine's last place in
64 bits (2^-50 here, half a unit in numpy): a value would differ in fp32 only within
2^-50 of a rounding border, one angle in 2^25, and the inputs are fixed."""
import numpy as np
import pytest

from tests import pagedref as R
from tests import stepref as S
from tests.test_gpu_paged import ints, make, pool_of, rows, starts_of

pytestmark = pytest.mark.gpu


def np_of(t):
    return t.detach().cpu().float().numpy()


def model(cache, before, k, v, q, pos, freqs, il, lens, counts, layer=0):
    """The pool after the rows, and the turned queries."""
    c = cache.cfg
    pool, table = before.copy(), cache.table.cpu().numpy()
    ky = S.turned(np_of(k), pos, freqs, il)
    at = 0
    for s, n in enumerate(counts):
        for i in range(n):
            p = lens[s] - n + i
            for h in range(c.n_kv_heads):
                rec = pool[table[s, p // 64], layer, h]
                for kv, x in enumerate((ky[at, h], np_of(v)[at, h])):
                    cs, sc, z = R.quantize(x[None], c.group)
                    R.store(rec, p % 64, kv, cs[0], sc[0], z[0], c.head_dim, c.group)
            at += 1
    return pool, S.turned(np_of(q), pos, freqs, il)


CASES = [
    # d, g, rot, interleaved, dtype, lens, counts, kv heads, gqa, positions
    (128, 128, 128, False, "float16", [1, 65, 130], [1, 1, 1], 2, 4, None),
    (128, 32, 128, True, "bfloat16", [1, 64, 130], [1, 1, 1], 1, 1, None),
    (64, 64, 64, False, "bfloat16", [5, 200], [1, 1], 2, 7, 1 << 20),
    (64, 32, 16, True, "float16", [63, 129], [1, 1], 1, 2, -70000),
    (128, 64, 96, False, "float16", [100, 3, 140], [37, 3, 76], 2, 4, None),
    (128, 128, 64, True, "bfloat16", [129, 64], [129, 2], 1, 8, 123457),
    (64, 64, 48, False, "float16", [190, 66], [150, 3], 2, 1, 5),
    (64, 32, 32, True, "bfloat16", [70, 128], [70, 64], 1, 3, None),
]


@pytest.mark.parametrize("d,g,rot,il,dtype,lens,counts,h,gqa,shift", CASES)
def test_rows_match_the_model_bit_for_bit(d, g, rot, il, dtype, lens, counts, h, gqa, shift):
    import torch
    dt = getattr(torch, dtype)
    rng = np.random.default_rng(d + g + rot + len(lens))
    cache = make(h=h, hq=h * gqa, d=d, g=g, n_pages=24, seqs=4, seq_pages=6, fill=7)
    cache.reserve(ints(lens + [0] * (4 - len(lens))))
    before = pool_of(cache).copy()
    n = sum(counts)
    qkv = rows(rng, (n + 2, h * (gqa + 2), d), dt)[:n]         # slices of one projection's output
    q, k, v = qkv[:, :h * gqa], qkv[:, h * gqa:h * (gqa + 1)], qkv[:, h * (gqa + 1):]
    place = np.concatenate([np.arange(a - b, a) for a, b in zip(lens, counts)])
    pos = place if shift is None else place[::-1] + shift
    freqs = S.frequencies(rot)
    out = cache.append(0, k, v, starts_of(counts), torch.from_numpy(freqs).cuda(), q=q, interleaved=il,
                       positions=None if shift is None else ints(pos))
    want, wq = model(cache, before, k, v, q, pos, freqs, il, lens, counts)
    assert np.array_equal(pool_of(cache), want)
    assert torch.equal(out.cpu(), torch.from_numpy(wq).to(dt))
    assert cache.status() == 0
    # in place, over the projection's output
    same = cache.append(0, k, v, starts_of(counts), torch.from_numpy(freqs).cuda(), q=q, q_out=q, interleaved=il,
                        positions=None if shift is None else ints(pos))
    assert same is q and torch.equal(q.cpu(), torch.from_numpy(wq).to(dt)) and np.array_equal(pool_of(cache), want)


def test_without_queries_and_other_layers_stay():
    import torch
    rng = np.random.default_rng(3)
    cache = make(n_layers=3, h=2, hq=2, n_pages=8, seqs=2, seq_pages=4, fill=9)
    cache.reserve(ints([70, 0]))
    before = pool_of(cache).copy()
    k, v = rows(rng, (70, 2, 128), torch.float16), rows(rng, (70, 2, 128), torch.float16)
    f = S.frequencies(128)
    assert cache.append(1, k, v, starts_of([70]), torch.from_numpy(f).cuda()) is None
    want, _ = model(cache, before, k, v, k, np.arange(70), f, False, [70], [70], layer=1)
    assert np.array_equal(pool_of(cache), want)


def test_write_of_turned_rows_is_append_where_they_are_16_bit():
    """Quarter turns keep rows in 16 bits: append is then write of the turned rows."""
    import torch
    rng = np.random.default_rng(4)
    a, b = (make(h=2, hq=4, n_pages=8, seqs=2, seq_pages=4, fill=1) for _ in range(2))
    k, v = rows(rng, (100, 2, 128), torch.float16), rows(rng, (100, 2, 128), torch.float16)
    zero = torch.zeros(64, device="cuda")
    for c in (a, b):
        c.reserve(ints([100, 0]))
    a.append(0, k, v, starts_of([100]), zero)                  # no turn at all
    b.write(0, k, v, starts_of([100]))
    assert torch.equal(a.pool, b.pool)


@pytest.mark.parametrize("pos", [0, 1, 100003, 1 << 24, (1 << 29) - 1, (1 << 31) - 1, -(1 << 31), -12345])
def test_far_positions(pos):
    """Angles up to 2^31: cosine and sine of the 64-bit angle, as the C library reduces it."""
    import torch
    freqs = np.float32([1.0, 0.9999999, 0.7071068, 0.1, 1e-3, 3e-6, 1e-30, 0.0])
    cache = make(h=1, hq=1, d=64, g=64, n_pages=2, seqs=1, seq_pages=1)
    cache.reserve(ints([1]))
    x = torch.zeros((1, 1, 64), dtype=torch.float16, device="cuda")
    x[..., :8] = 1.0
    y = cache.append(0, x, x, starts_of([1]), torch.from_numpy(freqs).cuda(), q=x, positions=ints([pos]))
    want = torch.from_numpy(S.turned(np_of(x), [pos], freqs, False)).half()
    assert torch.equal(y.cpu(), want)


def test_padded_rows_and_early_rows_and_missing_pages():
    import torch
    rng = np.random.default_rng(5)
    cache = make(h=2, hq=4, n_pages=8, seqs=4, seq_pages=4, fill=3)
    table = torch.full((4, 4), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[2, 1] = 5, 6
    cache.assign(ints([3, 0, 70, 0]), table)                   # slot 2's first page is missing
    cache.status_word.zero_()
    before = pool_of(cache).copy()
    k, v = rows(rng, (16, 2, 128), torch.float16), rows(rng, (16, 2, 128), torch.float16)
    q = rows(rng, (16, 4, 128), torch.float16)
    out = torch.full((16, 4, 128), 77.0, dtype=torch.float16, device="cuda")
    f = S.frequencies(128)
    # 5 rows of a sequence of 3 tokens, 1 of an empty one, 8 of 70 (two of them on the missing page); 2 of nobody's
    st = ints([0, 5, 6, 14])
    got = cache.append(0, k, v, st, torch.from_numpy(f).cuda(), q=q, q_out=out)
    torch.cuda.synchronize()
    assert cache.status() == R.BAD_INDEX
    assert torch.equal(got[14:], torch.full_like(got[14:], 77.0))
    assert not got[:2].any() and not got[5].any()
    pos = np.concatenate([np.arange(3), np.arange(62, 70)])
    rest = np.r_[2:5, 6:14]
    assert torch.equal(got[rest].cpu(), torch.from_numpy(S.turned(np_of(q)[rest], pos, f, False)).half())
    want, ky = before.copy(), S.turned(np_of(k)[rest], pos, f, False)
    for i, p in enumerate(pos):
        if 3 <= i and p < 64:
            continue                                           # missing
        for h in range(2):
            rec = want[5 if i < 3 else 6, 0, h]
            for kv, x in enumerate((ky[i, h], np_of(v)[rest][i, h])):
                cs, sc, z = R.quantize(x[None], 128)
                R.store(rec, p % 64, kv, cs[0], sc[0], z[0], 128, 128)
    assert np.array_equal(pool_of(cache), want)


def test_values_that_are_not_finite():
    """A turned pair carries a NaN to both its channels: their groups are zeros, the others stay."""
    import torch
    rng = np.random.default_rng(6)
    cache = make(h=1, hq=1, d=128, g=32, n_pages=4, seqs=1, seq_pages=2)
    cache.reserve(ints([3]))
    k, v = rows(rng, (3, 1, 128), torch.bfloat16), rows(rng, (3, 1, 128), torch.bfloat16)
    k[1, 0, 5] = float("nan")
    q = k.clone()
    f = S.frequencies(128)
    out = cache.append(0, k, v, starts_of([3]), torch.from_numpy(f).cuda(), q=q)
    assert cache.status() == R.NONFINITE
    K, _ = cache.read(0, starts_of([3]), 3, dtype=torch.float32)
    assert not K[1, 0, :32].any() and not K[1, 0, 64:96].any() and K[1, 0, 32:64].any() and K[1, 0, 96:].any()
    nan = torch.isnan(out[1, 0]).nonzero().flatten().tolist()
    assert nan == [5, 69] and not torch.isnan(out[[0, 2]]).any()


def test_stalled_and_shared_pages_store_nothing():
    import torch
    rng = np.random.default_rng(7)
    cache = make(h=1, hq=2, n_pages=2, seqs=2, seq_pages=2, fill=4)
    cache.reserve(ints([10, 0]))
    cache.fork(ints([0, 0]))                                   # the page is two slots'
    before = pool_of(cache).copy()
    k, v, q = (rows(rng, (2, n, 128), torch.float16) for n in (1, 1, 2))
    f = torch.from_numpy(S.frequencies(128)).cuda()
    want = torch.from_numpy(S.turned(np_of(q), [9, 9], S.frequencies(128), False)).half()
    assert torch.equal(cache.append(0, k, v, ints([0, 1, 2]), f, q=q).cpu(), want)
    assert cache.status() == R.BAD_INDEX and np.array_equal(pool_of(cache), before)
    cache.reserve(ints([1000, 0]))                             # too many
    cache.fork(ints([0, -1]))
    cache.append(0, k[:1], v[:1], ints([0, 1]), f, q=q[:1])
    assert cache.status() == R.BAD_INDEX | R.NO_PAGES and np.array_equal(pool_of(cache), before)


def test_in_a_graph_with_growing_lengths():
    """reserve, append, attn captured once: every replay takes the next position."""
    import torch
    rng = np.random.default_rng(8)
    a, b = (make(h=2, hq=8, n_pages=16, seqs=2, seq_pages=4, fill=0) for _ in range(2))
    f = torch.from_numpy(S.frequencies(128)).cuda()
    one, st = ints([1, 1]), starts_of([1, 1])
    k, v, q = (torch.zeros((2, n, 128), dtype=torch.float16, device="cuda") for n in (2, 2, 8))
    for c in (a, b):
        c.reserve(ints([62, 5]))
    def step(c):
        c.reserve(one)
        return c.attn(0, c.append(0, k, v, st, f, q=q), st)
    step(a)
    step(b)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step(a)
    # the capture enqueued nothing: b makes the step that a's capture did not
    for i in range(5):
        for t in (k, v, q):
            t.copy_(rows(rng, tuple(t.shape), torch.float16))
        want = step(b).clone()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(a.lens, b.lens) and torch.equal(a.pool, b.pool)
    assert a.lens.tolist() == [68, 11]
