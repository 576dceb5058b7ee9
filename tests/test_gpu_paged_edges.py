"""Calls of the paged 4-bit cache at the edges of what its header allows:
arguments that are the cache's own buffers, malformed starts, missing pages,
values far apart in magnitude.
Against the plain model of tests/pagedref.py; attention's tolerance is the one
worked out in tests/test_gpu_paged.py."""
import numpy as np
import pytest

from tests import pagedref as R
from tests.test_gpu_paged import assert_tables, check_attn, fill, ints, make, rows, starts_of

pytestmark = pytest.mark.gpu


def model_of(c):
    """The plain model of the cache's present tables."""
    m = R.Pages(c.cfg.n_pages, c.cfg.max_seqs, c.cfg.seq_pages)
    m.lens = c.lens.cpu().tolist()
    m.rows = [row[:-(-n // 64)] for row, n in zip(c.table.cpu().tolist(), m.lens)]
    return m


# ------------------------------------------------- the cache's own buffers --

def test_assign_takes_the_caches_own_tables():
    """Its own lengths and tables change nothing; shorter lengths over its own
    tables drop tokens, its own lengths with another table replace pages."""
    import torch
    rng = np.random.default_rng(50)
    c = make(n_pages=20, seqs=4, seq_pages=6)
    fill(c, [200, 90, 0, 64], rng)
    c.fork(ints([0, 1, 1, 3]))                           # a page that two slots hold
    lens, m = [200, 90, 90, 64], model_of(c)
    before = c.read(0, starts_of(lens), sum(lens))
    c.assign(c.lens, c.table)
    assert_tables(c, m)
    assert all(torch.equal(a, b) for a, b in zip(before, c.read(0, starts_of(lens), sum(lens))))
    short = [130, 64, 90, 0]
    c.assign(ints(short), c.table)
    m.lens, m.rows = short, [r[:-(-n // 64)] for r, n in zip(m.rows, short)]
    assert_tables(c, m)
    other = c.table.clone()
    other[0, 1], other[3, 2] = 19, 7                     # the second is beyond its sequence's length
    c.assign(c.lens, other)
    m.rows[0][1] = 19
    assert_tables(c, m)
    assert c.status() == 0
    other[0, 0] = 20                                     # no such page
    c.assign(c.lens, other)
    m.rows[0][0] = -1
    assert_tables(c, m)
    assert c.status() == R.BAD_INDEX


def test_own_lengths_as_counts():
    """Lengths as what a call adds, keeps or takes as parents."""
    import torch
    c = make(n_pages=20, seqs=4, seq_pages=6)
    fill(c, [100, 2, 0, 3], np.random.default_rng(51))
    m = model_of(c)
    c.reserve(c.lens)
    m.reserve(list(m.lens))
    assert_tables(c, m)
    keep = torch.arange(200, dtype=torch.int32, device="cuda").repeat(4, 1)
    lens = list(m.lens)
    c.compact(keep, c.lens)
    m.compact(lens, 200)
    assert_tables(c, m)
    c.assign(ints([3, 1, 0, 2]), c.table)
    m.lens, m.rows = [3, 1, 0, 2], [r[:-(-n // 64)] for r, n in zip(m.rows, [3, 1, 0, 2])]
    c.fork(c.lens)
    m.fork([3, 1, 0, 2])
    assert_tables(c, m)
    assert c.status() == 0


# --------------------------------------------------------- malformed starts --

def accepted(starts, n_rows):
    """First row and count of every sequence, by the header's words."""
    out, reached = [], 0
    for a, b in zip(starts, starts[1:]):
        fine = 0 <= a < b <= n_rows
        out.append((a, b - a) if fine and a >= reached else (a, 0))
        reached = max(reached, b) if fine else reached
    return out


def check_accepted(c, lens, starts, q, out, lse):
    """check_attn over the rows that sequences have; the others are as they were."""
    import torch
    acc = accepted(starts, q.shape[0])
    at = [t for a, m in acc for t in range(a, a + m)]
    if at:
        check_attn(c, lens, [m for _, m in acc], q[at], out[at], lse[at], c.cfg.head_dim ** -0.5,
                   only=lambda t, h: (t + h) % 11 == 0)
    rest = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
    rest[at] = False
    assert torch.all(out[rest] == 7.0) and torch.all(lse[rest] == 7.0)


def test_attn_counters_after_malformed_starts():
    """Starts that would give two long sequences the same rows ask for more
    workgroups than there are: the workspace is whole afterwards, and the next
    call's results are those over a fresh one."""
    import torch
    rng = np.random.default_rng(60)
    lens = [3000, 3000, 10, 64, 20000]
    c = make(h=8, hq=32, n_pages=420, seqs=5, seq_pages=320)
    fill(c, lens, rng)
    q = rows(rng, (64, 32, 128), torch.float16) * 0.3
    starts = [0, 64, 0, 64, 0, 64]
    out, lse = torch.full_like(q, 7.0), torch.full((64, 32), 7.0, device="cuda")
    c.attn(0, q, ints(starts), out=out, lse=lse)
    check_accepted(c, lens, starts, q, out, lse)
    assert c.status() == R.BAD_INDEX
    assert not c.ws[:2 * 512 * 64].view(torch.int32).any()     # the counters
    c.status_word.zero_()
    good = starts_of([10, 10, 10, 10, 24])
    first = c.attn(0, q, good, with_lse=True)
    second = c.attn(0, q, good, with_lse=True, workspace=torch.zeros_like(c.ws))
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    check_attn(c, lens, [10, 10, 10, 10, 24], q, *first, 128 ** -0.5, only=lambda t, h: (t + h) % 11 == 0)
    assert c.status() == 0


@pytest.mark.parametrize("seqs", [3, 64, 130])
def test_rows_of_malformed_starts(seqs):
    """Starts that descend, pass the rows or reuse them, more sequences than a
    wave has lanes among them: write, read and attention take exactly the rows
    that the header gives a sequence, and leave the others alone."""
    import torch
    rng = np.random.default_rng(61 + seqs)
    lens = [int(x) for x in rng.integers(1, 130, seqs)]
    lens[seqs // 2] = 900
    c = make(h=1, hq=4, d=64, g=32, n_pages=500, seqs=seqs, seq_pages=16)
    fill(c, lens, rng)
    n, table = 150, c.table.cpu().numpy()
    for step in range(8):
        starts = np.sort(rng.integers(0, n + 1, seqs + 1))
        for _ in range(1 + seqs // 20):                  # some out of order, some out of range
            starts[rng.integers(0, seqs + 1)] = rng.integers(-2, n + 3)
        if step % 2:
            starts[rng.integers(0, seqs):] = rng.integers(0, n // 2)
        starts = starts.tolist()
        acc = accepted(starts, n)
        pool = c.pool.cpu().numpy().reshape(-1, c.sz.record_bytes)
        K, V = rows(rng, (n, 1, 64), torch.float16), rows(rng, (n, 1, 64), torch.float16)
        c.write(0, K, V, ints(starts))
        for s, (a, m) in enumerate(acc):
            for t in range(m):
                pos = lens[s] - m + t
                if pos < 0:
                    continue
                for kv, x in enumerate((K, V)):
                    code, sc, z = R.quantize(x[a + t].cpu().float().numpy(), 32)
                    R.store(pool[table[s, pos // 64]], pos % 64, kv, code[0], sc[0], z[0], 64, 32)
        assert np.array_equal(c.pool.cpu().numpy().reshape(-1, c.sz.record_bytes), pool), step
        back = [torch.full((n, 1, 64), 7.0, device="cuda") for _ in range(2)]
        c.read(0, ints(starts), n, out=back)
        want = [np.full((n, 64), 7.0, np.float32) for _ in range(2)]
        for s, (a, m) in enumerate(acc):
            for t in range(m):
                pos = lens[s] - m + t
                for w, v in zip(want, R.values(pool[table[s, max(pos, 0) // 64]], 64, 32)):
                    w[a + t] = v[pos % 64] if pos >= 0 else 0.0
        assert all(np.array_equal(b[:, 0].cpu().numpy(), w) for b, w in zip(back, want)), step
        q = rows(rng, (n, 4, 64), torch.float16) * 0.3
        out, lse = torch.full_like(q, 7.0), torch.full((n, 4), 7.0, device="cuda")
        c.attn(0, q, ints(starts), out=out, lse=lse)
        check_accepted(c, lens, starts, q, out, lse)
        assert not c.ws[:2 * 512 * 64].view(torch.int32).any()


# ------------------------------------------------------------ missing pages --

def test_compact_reports_tokens_of_missing_pages():
    """A kept token whose page is missing has no values: a row of zeros, as a
    position outside the sequence gives, and reported like one."""
    import torch
    c = make(n_layers=2, n_pages=16, seqs=2, seq_pages=4)
    fill(c, [150, 70], np.random.default_rng(52))
    table = c.table.clone()
    table[0, 1] = -1
    c.assign(c.lens.clone(), table)
    m = model_of(c)
    keep = ints([[3, 64, 140], [0, 69, 0]])
    before = c.read(-1, starts_of([150, 70]), 220)
    c.status_word.zero_()
    c.compact(keep, ints([3, 2]))
    m.compact([3, 2], 3)
    assert_tables(c, m)
    assert c.status() == R.BAD_INDEX
    for x, y in zip(before, c.read(-1, starts_of([3, 2]), 5)):
        assert not y[:, 1].any() and torch.equal(y[:, [0, 2, 3, 4]], x[:, [3, 140, 150, 219]])
    c.status_word.zero_()
    c.compact(ints([[0, 2], [1, 0]]), ints([2, 1]))      # every page is there now
    assert c.status() == 0


# --------------------------------------------------- values far in magnitude --

def far_apart(c, lens, rng, large):
    """Writes the sequences' tokens: small values, and where `large` says (bool
    [n, head_dim], rows of all sequences) values up to fp16's range in V, whose
    tokens are of no weight: their K lies against every q that
    far_queries makes."""
    import torch
    n, h, d = sum(lens), c.cfg.n_kv_heads, c.cfg.head_dim
    K = rng.standard_normal((n, h, d)).astype(np.float32)
    V = rng.standard_normal((n, h, d)).astype(np.float32) * 1e-4
    V = np.where(large[:, None], rng.uniform(-6e4, 6e4, V.shape).astype(np.float32), V)
    K[large.all(1)] = -8.0
    c.reserve(ints(lens + [0] * (c.cfg.max_seqs - len(lens))))
    c.write(0, torch.from_numpy(K).half().cuda(), torch.from_numpy(V).half().cuda(), starts_of(lens))


def far_queries(rng, n, heads, d, dtype):
    import torch
    q = 1.0 + 0.3 * rng.standard_normal((n, heads, d)).astype(np.float32)
    return torch.from_numpy(q).to(dtype).cuda()


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("d,g", [(128, 128), (128, 64), (128, 32), (64, 64), (64, 32)])
def test_attn_large_values_of_unseen_and_weightless_tokens(d, g, shared):
    """In every page one token's V is some 2^29 of the others'.  Its weight is
    nothing to the rows that see it (e^-60), and the rows before it do not: the
    others' weights must keep their bits for either."""
    import torch
    rng = np.random.default_rng(d + g + shared)
    h, hq = (8, 64) if shared else (2, 8)
    lens = [700, 500] if shared else [150, 90]           # 75 tiles of 8 heads
    c = make(h=h, hq=hq, d=d, g=g, n_pages=24, seqs=4, seq_pages=12)
    large = np.concatenate([np.arange(n) % 64 == 50 for n in lens])
    far_apart(c, lens, rng, np.repeat(large[:, None], d, 1))
    n = sum(lens)
    q = far_queries(rng, n, hq, d, torch.float16)
    out, lse = c.attn(0, q, starts_of(lens), with_lse=True)
    pick = (lambda t, hh: t % 13 == 0 and hh in (0, 29)) if shared else (lambda t, hh: (t + hh) % 3 == 0)
    check_attn(c, lens, lens, q, out, lse, d ** -0.5, only=pick)
    one = far_queries(rng, 2, hq, d, torch.float16)      # generation
    out, lse = c.attn(0, one, starts_of([1, 1]), with_lse=True)
    check_attn(c, lens, [1, 1], one, out, lse, d ** -0.5)
    assert c.status() == 0


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("d,g", [(128, 64), (128, 32), (64, 32)])
def test_attn_groups_far_apart(d, g, shared):
    """Channel groups of V that differ by some 2^29: each keeps its own bits."""
    import torch
    rng = np.random.default_rng(d + g + shared + 7)
    h, hq = (8, 64) if shared else (2, 8)
    lens = [700, 500] if shared else [150, 90]           # 75 tiles of 8 heads
    c = make(h=h, hq=hq, d=d, g=g, n_pages=24, seqs=4, seq_pages=12)
    n, groups = sum(lens), d // g
    large = np.zeros((n, d), bool)
    large[:, :g] = True                                  # the first group throughout
    far_apart(c, lens, rng, large)
    q = far_queries(rng, n, hq, d, torch.float16)
    out, lse = c.attn(0, q, starts_of(lens), with_lse=True)
    pick = (lambda t, hh: t % 13 == 0 and hh in (0, 29)) if shared else (lambda t, hh: (t + hh) % 3 == 0)
    check_attn(c, lens, lens, q, out, lse, d ** -0.5, only=pick)
    one = far_queries(rng, 2, hq, d, torch.float16)
    out, lse = c.attn(0, one, starts_of([1, 1]), with_lse=True)
    check_attn(c, lens, [1, 1], one, out, lse, d ** -0.5)
    assert groups > 1 and c.status() == 0


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("d,g", [(128, 128), (128, 32), (64, 64)])
def test_attn_values_of_every_magnitude(d, g, shared):
    """V rows of 2^-13 to 2^13, in random order, then in ascending and in
    descending order."""
    import torch
    rng = np.random.default_rng(d + g + shared + 9)
    h, hq = (8, 64) if shared else (2, 8)
    lens = [600, 300, 300] if shared else [150, 90, 200]
    c = make(h=h, hq=hq, d=d, g=g, n_pages=24, seqs=4, seq_pages=12)
    n = sum(lens)
    e = [rng.uniform(-13, 13, lens[0]), np.linspace(-13, 13, lens[1]), np.linspace(13, -13, lens[2])]
    K = torch.from_numpy(rng.standard_normal((n, h, d)).astype(np.float32)).half().cuda()
    V = torch.from_numpy((rng.standard_normal((n, h, d)) * 2.0 ** np.concatenate(e)[:, None, None]).astype(np.float32)).half().cuda()
    c.reserve(ints(lens + [0]))
    c.write(0, K, V, starts_of(lens))
    pick = (lambda t, hh: t % 13 == 0 and hh in (0, 29)) if shared else (lambda t, hh: (t + hh) % 3 == 0)
    for mul in (0.3, 3.0):
        q = torch.from_numpy((rng.standard_normal((n, hq, d)) * mul).astype(np.float32)).to(torch.bfloat16).cuda()
        out, lse = c.attn(0, q, starts_of(lens), with_lse=True)
        check_attn(c, lens, lens, q, out, lse, d ** -0.5, only=pick)
    assert c.status() == 0


# ------------------------------------------------------- shapes at the ends --

@pytest.mark.parametrize("h,gqa,d,g", [(1, 33, 64, 64), (2, 64, 128, 128), (2, 64, 64, 32), (8, 7, 128, 64), (150, 1, 64, 64),
                                       (256, 2, 64, 32), (300, 1, 64, 64)])
def test_attn_many_heads(h, gqa, d, g):
    """A token's rows fill several tiles, tiles begin inside a token, and so many
    kv heads that none is left a second workgroup: one token, a few, a chunk, over
    contexts long enough to be split, beside slots without a row."""
    import torch
    rng = np.random.default_rng(h + gqa + d + g)
    seqs = 6
    lens = [1500, 40, 0, 700, 64, 3]
    c = make(h=h, hq=h * gqa, d=d, g=g, n_pages=50, seqs=seqs, seq_pages=30)
    fill(c, lens, rng)
    for counts in ([1, 1, 1, 1, 1, 1], [1, 0, 0, 0, 0, 0], [3, 0, 0, 2, 0, 5], [0, 40, 0, 130, 0, 0]):
        n = sum(counts)
        q = rows(rng, (n, h * gqa, d), torch.float16) * 0.3
        out, lse = c.attn(0, q, starts_of(counts), with_lse=True)
        step = max(1, n * h * gqa // 400)
        check_attn(c, lens, counts, q, out, lse, d ** -0.5, only=lambda t, hh: (t * h * gqa + hh) % step == 0)
        again = c.attn(0, q, starts_of(counts), with_lse=True)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    assert c.status() == 0 and not c.ws[:2 * 512 * 64].view(torch.int32).any()


def test_attn_shared_decoding_with_seven_query_heads():
    """Tiles of 128 rows whose waves begin inside a token."""
    import torch
    rng = np.random.default_rng(71)
    c = make(h=8, hq=56, n_pages=40, seqs=4, seq_pages=12)
    lens, counts = [600, 310, 90, 700], [600, 300, 95, 200]
    fill(c, lens, rng)
    q = rows(rng, (sum(counts), 56, 128), torch.bfloat16) * 0.3
    out, lse = c.attn(0, q, starts_of(counts), with_lse=True)
    check_attn(c, lens, counts, q, out, lse, 128 ** -0.5, only=lambda t, h: (t * 56 + h) % 31 == 0 and t % 3 == 0)


@pytest.mark.parametrize("m", [5, 16, 20])
def test_attn_few_tokens_of_many_sequences(m):
    """64 sequences' drafts: tiles of 128 rows would be less than half full, half
    full, and more."""
    import torch
    rng = np.random.default_rng(75 + m)
    lens = [int(x) for x in rng.integers(m, 400, 64)]
    lens[10], lens[11], lens[63] = 1200, 3, 0
    c = make(h=8, hq=32, d=64, g=64, n_pages=460, seqs=64, seq_pages=20)
    fill(c, lens, rng)
    q = rows(rng, (64 * m, 32, 64), torch.bfloat16) * 0.3
    out, lse = c.attn(0, q, starts_of([m] * 64), with_lse=True)
    check_attn(c, lens, [m] * 64, q, out, lse, 64 ** -0.5, only=lambda t, h: (t * 32 + h) % 23 == 0)
    assert c.status() == 0


@pytest.mark.parametrize("counts", [[1, 1, 1], [7, 1, 20], [500, 300, 700]])
def test_attn_over_its_own_queries(counts):
    """out may be q itself."""
    import torch
    rng = np.random.default_rng(72)
    c = make(h=8, hq=32, n_pages=90, seqs=3, seq_pages=70)
    fill(c, [4000, 310, 900], rng)
    q = rows(rng, (sum(counts), 32, 128), torch.float16) * 0.3
    want = c.attn(0, q, starts_of(counts))
    assert c.attn(0, q, starts_of(counts), out=q) is q
    assert torch.equal(q, want)


def test_pool_beyond_32_bits():
    """Pages past 4 GiB of a pool: what the calls write, move, copy and read there
    is what they do in a small one."""
    import torch
    shape = dict(n_layers=8, h=8, hq=32, g=32, seqs=4)
    big, small = make(n_pages=7000, seq_pages=6980, **shape), make(n_pages=40, seq_pages=8, **shape)
    assert big.pool.numel() > 1 << 32
    got = []
    for c, first in ((big, 6980), (small, 0)):
        rng = np.random.default_rng(73)
        table = np.full((4, c.cfg.seq_pages), -1, np.int32)
        table[0, :5], table[1, :2] = first + np.array([4, 0, 19, 7, 2]), first + np.array([9, 1])
        table[3, :first] = np.arange(first)              # the last slot holds the lower pages
        c.assign(ints([300, 100, 0, 64 * first]), torch.from_numpy(table).cuda())
        K, V = (rows(rng, (8, 400, 8, 128), torch.float16) for _ in range(2))
        c.write(-1, K, V, starts_of([300, 100, 0]))
        out = list(c.read(-1, starts_of([300, 100, 0]), 400))
        q = rows(rng, (6, 32, 128), torch.float16) * 0.3
        for layer in (0, 7):
            out += c.attn(layer, q, starts_of([5, 1, 0]), with_lse=True)
        c.fork(ints([0, 1, 0, 3]))
        c.reserve(ints([1, 0, 1, 0]))
        assert int(c.table[2, 4]) == first + 3           # the copy of the shared last page
        k, v = (rows(rng, (8, 2, 8, 128), torch.float16) for _ in range(2))
        c.write(-1, k, v, starts_of([1, 0, 1]))
        keep = ints([list(range(0, 300, 3)), list(range(100)), [5] * 100, [0] * 100])
        c.compact(keep, ints([100, -1, 7, -1]))
        out += c.read(-1, starts_of([100, 100, 7]), 207)
        assert c.status() == 0
        got.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_attn_missing_pages_under_shared_decoding():
    """As the other rows, to the same tolerance: a token of a missing page is not
    there."""
    import torch
    rng = np.random.default_rng(74)
    d, h, gq = 128, 8, 8
    c = make(h=h, hq=h * gq, n_pages=60, seqs=4, seq_pages=16)
    lens, counts = [500, 1, 900, 333], [500, 1, 400, 250]
    fill(c, lens, rng)
    table = c.table.clone()
    table[0, 3], table[2, 2], table[3, 0], table[3, 5] = -1, -1, -1, -1
    c.assign(c.lens, table)
    q = rows(rng, (sum(counts), h * gq, d), torch.float16) * 0.3
    out, lse = c.attn(0, q, starts_of(counts), with_lse=True)
    pool, table = c.pool.cpu().numpy().reshape(60, 1, h, -1), table.cpu().numpy()
    u, eps, scale, at = 2.0 ** -24, 2.0 ** -11, d ** -0.5, 0
    for s, m in enumerate(counts):
        for i in range(0, m, 17):
            t, n = at + i, lens[s] - m + i + 1
            for hh in ((t * 5) % (h * gq), (t * 11 + 1) % (h * gq)):
                parts = [[], [], [], [], [], []]
                for col in range(-(-n // 64)):
                    if table[s, col] < 0:
                        continue
                    k, v = R.unpack(pool[table[s, col], 0, hh // gq], d, d)
                    for p, x in zip(parts, k + v):
                        p.append(x[:min(64, n - 64 * col)].astype(np.float64))
                qq, o, l = q[t, hh].cpu().double().numpy(), out[t, hh].cpu().double().numpy(), float(lse[t, hh])
                if not parts[0]:
                    assert not o.any() and l == -np.inf
                    continue
                kc, ks, kz, vc, vs, vz = (np.concatenate(p) for p in parts)     # scales and zeros [n, 1]
                want, wl, p = R.attend(qq, kc * ks + kz, vc * vs + vz, len(kc), scale)
                dx = (d + 8) * u * scale * (np.abs(qq) @ (15 * ks + np.abs(kz) + 0 * kc).T).max()
                lim = (eps * np.abs(want) + 2.0 ** -11 * (p @ (vs * np.abs(vc - 7.5)))
                       + (np.expm1(2 * dx) + (n + 16) * u) * (p @ (15 * vs + np.abs(vz) + 0 * vc))) * (1 + eps) + 2.0 ** -24
                assert np.all(np.abs(o - want) <= lim), (s, i, hh)
                assert abs(l - wl) <= dx + (n + 16) * u + 4 * u * abs(wl) + 2.0 ** -22, (s, i, hh)
        at += m
