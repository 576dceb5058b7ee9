"""GPU parity of the paged 4-bit cache with the plain model of tests/pagedref.py.

Codes, metadata, page tables and moved pages are compared bit for bit.

Attention's tolerance, from the arithmetic.  With p the exact weights, s, z, c a
row's scale, zero and codes (u = 2^-24 is half a step of fp32):
  - an output is rounded to its type: finfo.eps / 2 relative (fp16 2^-11, bf16
    2^-8);
  - each weight p s is rounded to fp16 (2^-11 relative), and what that takes
    from the middle 7.5 of the codes is given back: 2^-11 sum p s |c - 7.5|;
  - a score is a product sum of head_dim terms and three more fp32 operations:
    off by at most d = (head_dim + 8) u scale sum_j |q_j| (15 s + |z|), its
    weight by a factor e^(+-2d) with the normalisation, and a weight's
    exponential by 2 u;
  - fp32 sums over n tokens: n u relative to the sum of magnitudes."""
import numpy as np
import pytest

from tests import pagedref as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def np_of(t):
    return t.detach().cpu().float().numpy()


def make(n_layers=1, h=2, hq=8, d=128, g=128, n_pages=64, seqs=4, seq_pages=16, fill=None):
    import torch
    import paper_2608_28911_amd as P
    cfg = P.make_paged_config(n_layers=n_layers, n_kv_heads=h, n_q_heads=hq, n_pages=n_pages, max_seqs=seqs,
                              seq_pages=seq_pages, head_dim=d, group=g)
    pool = torch.empty(P.paged_sizes(cfg).pool_bytes, dtype=torch.uint8, device="cuda")
    pool.fill_(0xFF if fill is None else fill)           # metadata of rows never written: NaN
    return P.PagedKV4(cfg, pool=pool)


def ints(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def starts_of(counts):
    return ints([0] + list(np.cumsum(counts)))


def pool_of(cache):
    c = cache.cfg
    return cache.pool.cpu().numpy().reshape(c.n_pages, c.n_layers, c.n_kv_heads, cache.sz.record_bytes)


def rows(rng, shape, dtype):
    import torch
    x = rng.standard_normal(shape).astype(np.float32)
    x[..., 3::29] *= 10.0
    x[..., 7] += 5.0
    return torch.from_numpy(x).to(dtype).cuda()


def fill(cache, lens, rng, dtype=None, scramble=True):
    """Gives the sequences these lengths and random rows, every layer."""
    import torch
    dtype = torch.float16 if dtype is None else dtype
    c = cache.cfg
    if scramble:                                         # page numbers out of order
        order, at = rng.permutation(c.n_pages), 0
        table = np.full((c.max_seqs, c.seq_pages), -1, np.int32)
        for s, n in enumerate(lens):
            k = -(-n // 64)
            table[s, :k] = order[at:at + k]
            at += k
        cache.assign(ints(lens), torch.from_numpy(table).cuda())
    else:
        cache.reserve(ints(lens))
    n = sum(lens)
    if n:
        K, V = (rows(rng, (c.n_layers, n, c.n_kv_heads, c.head_dim), dtype) for _ in range(2))
        cache.write(-1, K, V, starts_of(lens))
    assert cache.status() == 0


def stored(pool, table, s, n, layer, head, d, g):
    """Values, and scale, zero, codes expanded per channel, of a sequence's n tokens."""
    out = [[], []]
    for t in range(-(-n // 64)):
        for kv, (c, sc, z) in enumerate(R.unpack(pool[table[s, t], layer, head], d, g)):
            out[kv].append((c.astype(np.float64), np.repeat(sc.astype(np.float64), g, 1), np.repeat(z.astype(np.float64), g, 1)))
    return [tuple(np.concatenate([p[i] for p in parts])[:n] for i in range(3)) if parts else None for parts in out]


def check_attn(cache, lens, counts, q, out, lse, scale, layer=0, only=None):
    c, pool, table = cache.cfg, pool_of(cache), cache.table.cpu().numpy()
    d, g, gq = c.head_dim, c.group, c.n_q_heads // c.n_kv_heads
    eps = {2.0 ** -10: 2.0 ** -11, 2.0 ** -7: 2.0 ** -8}[float(__import__("torch").finfo(out.dtype).eps)]
    q, out, lse = np_of(q).astype(np.float64), np_of(out).astype(np.float64), lse.cpu().numpy().astype(np.float64)
    at = 0
    for s, m in enumerate(counts):
        n = lens[s]
        for head in range(c.n_kv_heads):
            kv = stored(pool, table, s, n, layer, head, d, g)
            for i in range(m):
                seen = n - m + i + 1
                for h in range(head * gq, (head + 1) * gq):
                    if only is not None and not only(at + i, h):
                        continue
                    o, l = out[at + i, h], lse[at + i, h]
                    if seen <= 0:
                        assert not o.any() and l == -np.inf
                        continue
                    (kc, ks, kz), (vc, vs, vz) = kv
                    k, v = kc * ks + kz, vc * vs + vz
                    want, wl, p = R.attend(q[at + i, h], k, v, seen, scale)
                    dx = (d + 8) * U * scale * (np.abs(q[at + i, h]) @ (15 * ks + np.abs(kz))[:seen].T).max()
                    mag = p @ (15 * vs + np.abs(vz))[:seen]
                    lim = (eps * np.abs(want) + 2.0 ** -11 * (p @ (vs * np.abs(vc - 7.5))[:seen])
                           + (np.expm1(2 * dx) + (seen + 16) * U) * mag) * (1 + eps) + 2.0 ** -24
                    err = np.abs(o - want)
                    assert np.all(err <= lim), (s, i, h, float((err / lim).max()))
                    assert abs(l - wl) <= dx + (seen + 16) * U + 4 * U * abs(wl) + 2.0 ** -22, (s, i, h, l, wl)
        at += m


# ------------------------------------------------------------------ rows --

@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("d,g", [(128, 128), (128, 64), (128, 32), (64, 64), (64, 32)])
def test_write_and_read_rows(d, g, bf16):
    """Chunks that begin and end inside pages: every byte of the pool afterwards
    is the model's, the rows beside them among it; read gives the stored values."""
    import torch
    dt = torch.bfloat16 if bf16 else torch.float16
    rng = np.random.default_rng(d + g + bf16)
    c = make(n_layers=2, d=d, g=g, n_pages=24, seqs=5, seq_pages=8)
    fill(c, [70, 0, 130, 1, 63], rng)
    counts = [3, 0, 200, 65, 1]
    c.reserve(ints(counts))
    lens, table = c.lens.cpu().tolist(), c.table.cpu().numpy()
    n, want = sum(counts), pool_of(c).copy()
    K, V = rows(rng, (n, 2, d), dt), rows(rng, (n, 2, d), dt)
    K[5, 0], V[17, 1, :g] = 2.5, 0.0                     # constant rows: scale 0
    K[40, 1, 5], V[41, 0, d - 1] = 6e4, -6e4             # and a wide one
    c.write(1, K, V, starts_of(counts))
    at = 0
    for s, m in enumerate(counts):
        for i in range(m):
            pos = lens[s] - m + i
            for head in range(2):
                rec = want[table[s, pos // 64], 1, head]
                for kv, x in enumerate((K, V)):
                    q = R.quantize(np_of(x[at + i, head])[None], g)
                    R.store(rec, pos % 64, kv, q[0][0], q[1][0], q[2][0], d, g)
        at += m
    assert np.array_equal(pool_of(c), want)
    assert c.status() == 0
    for out in (torch.float32, torch.float16, torch.bfloat16):
        k, v = c.read(1, starts_of(counts), n, dtype=out)
        at = 0
        for s, m in enumerate(counts):
            for i in range(m):
                pos = lens[s] - m + i
                for head in range(2):
                    for got, x in zip((k, v), R.values(want[table[s, pos // 64], 1, head], d, g)):
                        # fmaf rounds the exact value once to fp32, then to the type
                        w = torch.from_numpy(x[pos % 64].astype(np.float32)).to(out)
                        assert torch.equal(got[at + i, head].cpu(), w)
            at += m


def test_write_every_layer_through_strides():
    """K and V as slices of a fused projection, all layers in one call."""
    import torch
    rng = np.random.default_rng(3)
    c = make(n_layers=3, h=2, n_pages=8, seqs=2, seq_pages=4)
    counts = [100, 29]
    c.reserve(ints(counts))
    kv = rows(rng, (3, 129, 6, 128), torch.bfloat16)     # two heads of padding
    K, V = kv[:, :, :2], kv[:, :, 2:4]
    c.write(-1, K, V, starts_of(counts))
    k, v = c.read(-1, starts_of(counts), 129, dtype=torch.float32)
    for l in range(3):
        for x, got in ((K[l], k[l]), (V[l], v[l])):
            code, s, z = R.quantize(np_of(x).reshape(-1, 128), 128)
            want = code * s.astype(np.float64) + z.astype(np.float64)
            assert np.array_equal(got.cpu().numpy().reshape(-1, 128), want.astype(np.float32))


def test_rows_not_finite_are_zeros_and_reported():
    import torch
    rng = np.random.default_rng(4)
    c = make(d=128, g=32, n_pages=4, seqs=1, seq_pages=2)
    c.reserve(ints([3]))
    K, V = rows(rng, (3, 2, 128), torch.bfloat16), rows(rng, (3, 2, 128), torch.bfloat16)
    K[1, 0, 40], V[2, 1, 127] = float("nan"), float("inf")
    c.write(0, K, V, starts_of([3]))
    assert c.status() == R.NONFINITE
    k, v = c.read(0, starts_of([3]), 3, dtype=torch.float32)
    assert not k[1, 0, 32:64].any() and not v[2, 1, 96:].any()
    for x, got in ((K, k), (V, v)):
        code, s, z = R.quantize(np_of(x).reshape(-1, 128), 32)
        want = code * np.repeat(s.astype(np.float64), 32, 1) + np.repeat(z.astype(np.float64), 32, 1)
        assert np.array_equal(got.cpu().numpy().reshape(-1, 128), want.astype(np.float32))


# -------------------------------------------------------------- attention --

LENS = [1, 2, 63, 64, 65, 0, 500, 900]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("d,g", [(128, 128), (128, 64), (128, 32), (64, 64), (64, 32)])
def test_attn_one_token(d, g, bf16):
    """One token of sequences of every kind of length, an empty one among them;
    rows of the pool that nothing was written to hold NaN."""
    import torch
    dt = torch.bfloat16 if bf16 else torch.float16
    rng = np.random.default_rng(d * g + bf16)
    c = make(d=d, g=g, n_pages=40, seqs=8, seq_pages=16)
    fill(c, LENS, rng, dt)
    q = rows(rng, (8, 8, d), dt) * 0.5
    out, lse = c.attn(0, q, starts_of([1] * 8), with_lse=True)
    check_attn(c, LENS, [1] * 8, q, out, lse, d ** -0.5)
    assert c.status() == 0


@pytest.mark.parametrize("gqa", [1, 2, 4, 7, 16])
@pytest.mark.parametrize("d,g,counts", [
    (128, 128, [1, 5, 0, 64, 65]), (128, 32, [3, 5, 2, 40, 130]), (128, 64, [1, 1, 7, 33, 257]),
    (64, 64, [2, 9, 1, 90, 300]), (64, 32, [1, 70, 4, 20, 31])])
def test_attn_several_tokens(d, g, counts, gqa):
    """Chunks of several tokens over what is cached, whole prompts among them,
    and sequences shorter than their chunk (rows that see no token)."""
    import torch
    rng = np.random.default_rng(d + g + gqa + len(counts))
    c = make(h=2, hq=2 * gqa, d=d, g=g, n_pages=40, seqs=5, seq_pages=12)
    lens = [3, counts[1], 100, 200, 301]
    fill(c, lens, rng)
    n = sum(counts)
    q = rows(rng, (n, 2 * gqa, d), torch.float16) * 0.3
    out, lse = c.attn(0, q, starts_of(counts), with_lse=True, scale=0.2)
    check_attn(c, lens, counts, q, out, lse, 0.2)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("d,g", [(128, 128), (128, 64), (128, 32), (64, 64), (64, 32)])
def test_attn_prompts_that_fill_the_chip(d, g, bf16):
    """Tiles of 128 rows, whose waves decode pages for each other: ragged prompts
    and chunks, among them one token, an empty sequence, one shorter than its
    chunk, and pages that are missing; checked at every 37th (row, head) and at
    the ends."""
    import torch
    rng = np.random.default_rng(d + g)
    h, gq = 8, 8
    c = make(h=h, hq=h * gq, d=d, g=g, n_pages=60, seqs=6, seq_pages=16)
    lens, counts = [500, 1, 0, 900, 30, 333], [500, 1, 0, 300, 70, 200]
    fill(c, lens, rng)
    n = sum(counts)
    q = (rows(rng, (n, h * gq, d), torch.float32) * 0.3).to(torch.bfloat16 if bf16 else torch.float16)
    out, lse = c.attn(0, q, starts_of(counts), with_lse=True)
    ends = {0, 499, 500, 501, 801 - 1, 801, 840, 841, 870, 871, n - 1}
    check_attn(c, lens, counts, q, out, lse, d ** -0.5, only=lambda t, hh: (t * h * gq + hh) % 37 == 0 and t % 5 == 0 or t in ends and hh in (0, 63))
    table = c.table.clone()
    table[3, 2], table[5, 0] = -1, -1                    # 64 tokens of one, the first 64 of another
    c.assign(c.lens.clone(), table)
    got, gl = c.attn(0, q, starts_of(counts), with_lse=True)
    assert torch.equal(got[:501], out[:501])
    pool, table = pool_of(c), table.cpu().numpy()
    for t, s, pos in ((501, 3, 600), (800, 3, 899), (871, 5, 133), (n - 1, 5, 332)):
        k, v = [], []
        for i in range(pos // 64 + 1):
            if table[s, i] >= 0:
                a, b = R.values(pool[table[s, i], 0, 3], d, g)
                m = min(64, pos + 1 - 64 * i)
                k.append(a[:m])
                v.append(b[:m])
        k, v = np.concatenate(k), np.concatenate(v)
        want, wl, _ = R.attend(np_of(q[t, 8 * 3 + 5]).astype(np.float64), k, v, len(k), d ** -0.5)
        # the tolerance of a row above, with everything at its largest
        assert np.abs(np_of(got[t, 29]) - want).max() <= 2.0 ** -7 * np.abs(v).max() and abs(float(gl[t, 29]) - wl) <= 1e-2


def test_attn_rows_before_the_first_token():
    """More rows than the sequence has tokens: the first see nothing."""
    import torch
    rng = np.random.default_rng(8)
    c = make(n_pages=8, seqs=3, seq_pages=4)
    fill(c, [2, 0, 70], rng)
    counts = [5, 3, 80]
    q = rows(rng, (88, 8, 128), torch.bfloat16)
    out, lse = c.attn(0, q, starts_of(counts), with_lse=True)
    check_attn(c, [2, 0, 70], counts, q, out, lse, 128 ** -0.5)
    k, v = c.read(0, starts_of(counts), 88)
    assert not k[:3].any() and not v[5:8].any() and not k[8:18].any() and v[18:].any()
    assert c.status() == R.BAD_INDEX                     # read reports them


@pytest.mark.parametrize("vmul", [1e-5, 1.0, 3e3])
@pytest.mark.parametrize("qmul", [1e-3, 1.0, 30.0])
def test_attn_magnitudes(qmul, vmul):
    """Weights are fp16 whatever the values' scale: tiny, ordinary and large
    values, flat and sharp maps, and scales that grow along the sequence."""
    import torch
    rng = np.random.default_rng(9)
    c = make(n_pages=16, seqs=1, seq_pages=16, g=64)
    c.reserve(ints([800]))
    K, V = rows(rng, (800, 2, 128), torch.float16), rows(rng, (800, 2, 128), torch.float32) * vmul * 0.2
    V *= torch.logspace(-2, 0, 800, device="cuda")[:, None, None]
    c.write(0, K, V.half(), starts_of([800]))
    q = (rows(rng, (3, 8, 128), torch.float32) * qmul).bfloat16()
    out, lse = c.attn(0, q, starts_of([3]), with_lse=True)
    check_attn(c, [800], [3], q, out, lse, 128 ** -0.5)


def test_attn_pads_strides_and_missing_pages():
    """Rows past the last sequence's stay as they were; q through strides; pages
    that are missing are not seen."""
    import torch
    rng = np.random.default_rng(10)
    c = make(n_pages=20, seqs=2, seq_pages=8)
    fill(c, [300, 200], rng)
    wide = rows(rng, (9, 12, 128), torch.float16)
    q = wide[:, 2:10]
    out = torch.full((9, 8, 128), 7.0, dtype=torch.float16, device="cuda")
    lse = torch.full((9, 8), 7.0, device="cuda")
    c.attn(0, q, starts_of([4, 2]), out=out, lse=lse)
    check_attn(c, [300, 200], [4, 2], q, out, lse, 128 ** -0.5)
    assert torch.all(out[6:] == 7.0) and torch.all(lse[6:] == 7.0)
    table = c.table.cpu()
    table[0, 1] = -1                                     # tokens 64 .. 127 are gone
    c.assign(c.lens.clone(), table.cuda())
    assert c.status() == R.BAD_INDEX
    got, _ = c.attn(0, q[:1].contiguous(), starts_of([1, 0]), with_lse=True)
    pool = pool_of(c)
    for head in range(2):
        k, v = [], []
        for t in (0, 2, 3, 4):
            a, b = R.values(pool[table[0, t], 0, head], 128, 128)
            m = 64 if t < 4 else 300 - 256
            k.append(a[:m])
            v.append(b[:m])
        k, v = np.concatenate(k), np.concatenate(v)
        for h in range(4 * head, 4 * head + 4):
            want, _, _ = R.attend(np_of(q[0, h]).astype(np.float64), k, v, len(k), 128 ** -0.5)
            assert np.abs(np_of(got[0, h]) - want).max() <= 2e-2


def test_attn_long_sequence_and_many_splits():
    """20000 tokens of one sequence beside short ones: the work is split over
    workgroups and joined."""
    import torch
    rng = np.random.default_rng(12)
    c = make(h=1, hq=4, n_pages=340, seqs=3, seq_pages=320, g=32)
    lens = [20000, 5, 700]
    fill(c, lens, rng)
    for counts in ([1, 1, 1], [7, 1, 20]):
        q = rows(rng, (sum(counts), 4, 128), torch.float16) * 0.2
        out, lse = c.attn(0, q, starts_of(counts), with_lse=True)
        check_attn(c, lens, counts, q, out, lse, 128 ** -0.5)


def test_many_sequences():
    """More sequences than a wave has lanes, some empty, some without a row in
    the call: writes, reads and attention of one and of several tokens."""
    import torch
    rng = np.random.default_rng(13)
    n = 150
    lens = [int(x) for x in rng.integers(0, 200, n)]
    lens[70], lens[149] = 1500, 700
    c = make(h=1, hq=4, d=64, g=32, n_pages=700, seqs=n, seq_pages=24)
    fill(c, lens, rng)
    back = c.read(0, starts_of(lens), sum(lens), dtype=torch.float32)[0]
    pool, table = pool_of(c), c.table.cpu().numpy()
    at = 0
    for s, m in enumerate(lens):
        for t in {0, m // 2, m - 1} if m else ():
            want = R.values(pool[table[s, t // 64], 0, 0], 64, 32)[0][t % 64]
            assert np.array_equal(back[at + t, 0].cpu().numpy(), want.astype(np.float32))
        at += m
    for counts in ([1] * n, [int(rng.integers(0, 2)) for _ in lens], [int(rng.integers(0, min(m, 40) + 1)) for m in lens]):
        q = rows(rng, (sum(counts), 4, 64), torch.float16) * 0.3
        out, lse = c.attn(0, q, starts_of(counts), with_lse=True)
        check_attn(c, lens, counts, q, out, lse, 64 ** -0.5, only=lambda t, h: (t + h) % 7 == 0)
    assert c.status() == 0


# ------------------------------------------------------------------ pages --

def assert_tables(c, m):
    assert c.lens.cpu().tolist() == m.lens
    assert np.array_equal(c.table.cpu().numpy(), m.table())
    refs = m.refs()
    assert c.refs.cpu().tolist() == refs
    words = c.state[c.sz.free_word:c.sz.free_word + (c.cfg.n_pages + 31) // 32].cpu().numpy()
    bits = np.unpackbits(words.view(np.uint8), bitorder="little")
    assert np.array_equal(bits[:c.cfg.n_pages], np.array(refs) == 0) and not bits[c.cfg.n_pages:].any()
    assert int(c.stalled) == m.stalled


@pytest.mark.parametrize("n_pages,seqs,seq_pages,seed", [(40, 6, 8, 0), (33, 17, 5, 1), (200, 64, 9, 2), (3000, 3, 900, 3)])
def test_random_page_calls(n_pages, seqs, seq_pages, seed):
    """Random reserve, fork and compact calls: tables, counts, free pages and
    every page's bytes after each are the model's; some find no pages."""
    import torch
    rng = np.random.default_rng(seed)
    c = make(n_layers=2, h=1, hq=1, d=64, g=64, n_pages=n_pages, seqs=seqs, seq_pages=seq_pages)
    m = R.Pages(n_pages, seqs, seq_pages)
    want = pool_of(c).copy()
    failed = 0
    for step in range(30):
        kind = rng.choice(["reserve", "fork", "compact"], p=[0.5, 0.3, 0.2])
        if kind == "reserve":
            n = rng.integers(0, max(2, n_pages * 64 // seqs // 4), seqs) * (rng.random(seqs) < 0.6)
            if rng.random() < 0.3:
                n = np.minimum(n, 1)
            c.reserve(ints(n.tolist()))
            st, copies = m.reserve(n.tolist())
            failed += st != 0
            for a, b in copies:
                want[b] = want[a]
            # fill the new rows, unless there are none
            if not st and n.sum():
                counts = n.tolist()
                K, V = (rows(rng, (2, int(n.sum()), 1, 64), torch.float16) for _ in range(2))
                c.write(-1, K, V, starts_of(counts))
                got = pool_of(c)                         # the rows' own parity is tested above: take them over
                table = m.table()
                for s, k in enumerate(counts):
                    for p in {table[s, t // 64] for t in range(m.lens[s] - k, m.lens[s])}:
                        want[p] = got[p]
        elif kind == "fork":
            p = rng.integers(-1, seqs, seqs)
            p = np.where(rng.random(seqs) < 0.5, np.arange(seqs), p)
            c.fork(ints(p.tolist()))
            assert m.fork(p.tolist()) == 0
        else:
            w = max(m.lens) + 3
            keep, n_keep = np.zeros((seqs, w), np.int32), []
            for s, k in enumerate(m.lens):
                n = -1 if rng.random() < 0.4 else int(rng.integers(0, k + 1))
                n_keep.append(n)
                if n > 0:
                    keep[s, :n] = np.sort(rng.choice(k, n, replace=False))
            old = [list(r) for r in m.rows]
            c.compact(torch.from_numpy(keep).cuda(), ints(n_keep))
            st, moved = m.compact(n_keep, w)
            failed += st != 0
            for s, (_, fresh) in moved.items():
                for i, p in enumerate(fresh):
                    for l in range(2):
                        new = np.zeros_like(want[p, l, 0])
                        for t in range(min(64, n_keep[s] - 64 * i)):
                            pos = keep[s, 64 * i + t]
                            src = R.unpack(want[old[s][pos // 64], l, 0], 64, 64)
                            for kv in range(2):
                                R.store(new, t, kv, *(x[pos % 64] for x in src[kv]), 64, 64)
                        want[p, l, 0] = new
        assert_tables(c, m)
        assert np.array_equal(pool_of(c)[np.array(m.refs()) > 0], want[np.array(m.refs()) > 0]), (step, kind)
        live = np.array(m.refs()) == 0
        want[live] = pool_of(c)[live]
        assert c.status() == (R.NO_PAGES if failed else 0)


@pytest.mark.parametrize("n_pages,seqs,seq_pages", [(70001, 3, 30000), (5000, 1024, 9)])
def test_page_calls_at_the_limits(n_pages, seqs, seq_pages):
    """Bitmaps of more words than a workgroup has threads; every slot in use."""
    rng = np.random.default_rng(n_pages)
    c = make(h=1, hq=1, d=64, g=64, n_pages=n_pages, seqs=seqs, seq_pages=seq_pages)
    m = R.Pages(n_pages, seqs, seq_pages)
    for most in (seq_pages * 40, 1, 1):
        n = rng.integers(0, most + 1, seqs).tolist()
        c.reserve(ints(n))
        assert m.reserve(n)[0] == 0
        p = rng.permutation(seqs)
        p[rng.random(seqs) < 0.3] = -1
        c.fork(ints(p.tolist()))
        m.fork(p.tolist())
        assert_tables(c, m)
    n = [min(k, 70) for k in m.lens]
    c.compact(ints([list(range(70))] * seqs), ints(n))
    m.compact(n, 70)
    assert_tables(c, m)
    c.reserve(ints([seq_pages * 64 - k for k in m.lens]))      # more than there is, unless the slots hold it all
    m.reserve([seq_pages * 64 - k for k in m.lens])
    assert_tables(c, m)
    assert c.status() in (0, R.NO_PAGES)


def test_shared_last_page_is_copied_before_it_grows():
    """A forked sequence and its origin grow apart; the lowest of the growing
    holders keeps the page, and a holder that does not grow keeps its rows."""
    import torch
    rng = np.random.default_rng(20)
    c = make(n_pages=12, seqs=4, seq_pages=4)
    fill(c, [70, 0, 0, 0], rng)
    m = R.Pages(12, 4, 4)
    m.lens, m.rows = [70, 0, 0, 0], [c.table[0, :2].cpu().tolist(), [], [], []]
    c.fork(ints([0, 0, 0, 3]))
    m.fork([0, 0, 0, 3])
    assert_tables(c, m)
    before = c.read(0, starts_of([70]), 70)
    c.reserve(ints([0, 1, 1, 0]))                        # slot 0 holds the page and stays
    m.reserve([0, 1, 1, 0])
    assert_tables(c, m)
    K, V = rows(rng, (2, 2, 128), torch.float16), rows(rng, (2, 2, 128), torch.float16)
    c.write(0, K, V, starts_of([0, 1, 1, 0]))
    assert c.status() == 0
    assert all(torch.equal(a, b) for a, b in zip(before, c.read(0, starts_of([70]), 70)))
    k, _ = c.read(0, starts_of([0, 71, 71]), 142)
    assert torch.equal(k[:70], before[0]) and torch.equal(k[71:141], before[0]) and not torch.equal(k[70], k[141])
    c.fork(ints([1, 1, -1, 3]))                          # both holders grow now: slot 0 keeps the page
    m.fork([1, 1, -1, 3])
    c.reserve(ints([2, 1, 0, 0]))
    m.reserve([2, 1, 0, 0])
    assert_tables(c, m)


def test_write_spares_shared_and_missing_pages():
    """Rows of a page that another slot holds too are not stored, nor rows of a
    missing one, nor any while a reserve has failed; each is reported."""
    import torch
    rng = np.random.default_rng(21)
    c = make(n_pages=6, seqs=2, seq_pages=4)
    fill(c, [70, 0], rng)
    c.fork(ints([0, 0]))
    before = pool_of(c).copy()
    K, V = rows(rng, (6, 2, 128), torch.float16), rows(rng, (6, 2, 128), torch.float16)
    c.write(0, K, V, starts_of([0, 6]))
    assert np.array_equal(pool_of(c), before) and c.status() == R.BAD_INDEX
    c.status_word.zero_()
    c.reserve(ints([0, 4 * 64]))                         # more than seq_pages hold
    assert c.status() == R.NO_PAGES and int(c.stalled) == 1 and c.lens.cpu().tolist() == [70, 70]
    c.fork(ints([0, -1]))
    c.write(0, K, V, starts_of([6]))
    assert np.array_equal(pool_of(c), before)
    c.status_word.zero_()
    c.reserve(ints([6, 0]))
    c.write(0, K, V, starts_of([6]))
    assert c.status() == 0 and not np.array_equal(pool_of(c), before)
    table = c.table.clone()
    table[0, 1] = 99
    c.assign(c.lens.clone(), table)
    assert c.status() == R.BAD_INDEX and int(c.table[0, 1]) == -1
    after = pool_of(c).copy()
    c.write(0, K, V, starts_of([6]))
    assert np.array_equal(pool_of(c), after)


def test_bad_indexes_are_reported_and_harmless():
    import torch
    rng = np.random.default_rng(22)
    c = make(n_pages=12, seqs=3, seq_pages=4)
    fill(c, [100, 30, 0], rng)
    q = rows(rng, (4, 8, 128), torch.float16)
    m = R.Pages(12, 3, 4)
    m.lens, m.rows = [100, 30, 0], [[p for p in r if p >= 0] for r in c.table.cpu().tolist()]
    calls = [
        lambda: (c.reserve(ints([1, -5, 0])), m.reserve([1, -5, 0])),
        lambda: (c.fork(ints([7, 0, -2])), m.fork([7, 0, -2])),
        lambda: (c.compact(ints([[0, 1]] * 3), ints([3, -2, -1])), m.compact([3, -2, -1], 2)),
        lambda: (c.compact(ints([[0, 400], [5, -1], [0, 0]]), ints([2, 2, -1])), m.compact([2, 2, -1], 2)),
        lambda: c.assign(ints([-3, 4 * 64 + 1, 5]), ints([[0, 1, 2, 3], [4, 5, 6, 7], [12, -1, 2, 3]])),
    ]
    for i, call in enumerate(calls):
        c.status_word.zero_()
        call()
        assert c.status() == R.BAD_INDEX, i
        if i < 4:
            assert_tables(c, m)
        if i == 3:                                       # positions that are none give zeros
            k, v = c.read(0, starts_of([2, 2]), 4)
            assert not k[1].any() and not v[1].any() and not k[3].any() and k[0].any()
    assert c.lens.cpu().tolist() == [0, 256, 5] and c.table.cpu().tolist() == [[-1] * 4, [4, 5, 6, 7], [-1] * 4]
    for bad in ([0, 3, 1, 4], [0, 2, 9, 9], [-1, 2, 3, 4]):
        for call in (lambda s: c.write(0, q[:, :2].contiguous(), q[:, 2:4].contiguous(), s), lambda s: c.attn(0, q, s),
                     lambda s: c.read(0, s, 4)):
            c.status_word.zero_()
            call(ints(bad))
            assert c.status() & R.BAD_INDEX


# ---------------------------------------------------- graphs, other streams --

def test_generation_captured_into_a_graph():
    """reserve, write and attention of two layers as one graph, replayed with new
    inputs: tables, pages and outputs are those of the eager calls, page borders
    and a fork between the replays included."""
    import torch
    rng = np.random.default_rng(30)
    caches = []
    for _ in range(2):
        r = np.random.default_rng(31)
        c = make(n_layers=2, n_pages=30, seqs=3, seq_pages=8)
        fill(c, [60, 127, 5], r)
        caches.append(c)
    eager, graph = caches
    one, starts = ints([1, 1, 1]), starts_of([1, 1, 1])
    q, k, v = (torch.zeros(s, dtype=torch.float16, device="cuda") for s in ((2, 3, 8, 128), (2, 3, 2, 128), (2, 3, 2, 128)))
    outs = torch.zeros((2, 3, 8, 128), dtype=torch.float16, device="cuda")

    def step(c, outs):
        c.reserve(one)
        for l in range(2):
            c.write(l, k[l], v[l], starts)
            c.attn(l, q[l], starts, out=outs[l])

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            step(graph, outs)
    torch.cuda.synchronize()
    want = torch.zeros_like(outs)
    for i in range(8):
        for t in (q, k, v):
            t.copy_(rows(rng, tuple(t.shape), torch.float16))
        g.replay()
        torch.cuda.synchronize()
        step(eager, want)
        torch.cuda.synchronize()
        assert torch.equal(outs, want)
        assert torch.equal(eager.state, graph.state) and torch.equal(eager.pool, graph.pool)
        if i == 3:
            for c in (eager, graph):
                c.fork(ints([0, 0, 2]))
    assert eager.status() == graph.status() == 0


def test_calls_follow_the_current_stream():
    import torch
    rng = np.random.default_rng(33)
    c = make(n_pages=12, seqs=2, seq_pages=8)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        fill(c, [200, 90], rng)
        q = rows(rng, (2, 8, 128), torch.float16)
        out, lse = c.attn(0, q, starts_of([1, 1]), with_lse=True)
    s.synchronize()
    check_attn(c, [200, 90], [1, 1], q, out, lse, 128 ** -0.5)


def test_two_calls_at_once_with_a_workspace_each():
    import torch
    rng = np.random.default_rng(34)
    c = make(n_pages=200, seqs=1, seq_pages=200)
    fill(c, [12000], rng)
    q = [rows(rng, (1, 8, 128), torch.float16) for _ in range(2)]
    ws = [torch.zeros_like(c.ws) for _ in range(2)]
    st = starts_of([1])
    want = [c.attn(0, x, st).clone() for x in q]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [torch.zeros_like(w) for w in want]
    for _ in range(20):
        for x, w, s, o in zip(q, ws, streams, got):
            with torch.cuda.stream(s):
                c.attn(0, x, st, out=o, workspace=w)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


# ------------------------------------------------------------- all together --

def test_prompt_scored_ranked_compacted_and_continued():
    """A prompt's chunks are written and attended to, its tokens scored by
    self-information and ranked, the top quarter kept; generation goes on over
    what is kept, on a fork of it too."""
    import torch
    import paper_2608_28911_amd as P
    rng = np.random.default_rng(40)
    B, T, vocab = 2, 700, 1003
    c = make(n_layers=2, n_pages=60, seqs=4, seq_pages=16)
    at = 0
    for m in (300, 399, 1):
        counts = [m, m, 0, 0]
        c.reserve(ints(counts))
        at += m
        st = starts_of(counts)
        for l in range(2):
            K, V = rows(rng, (2 * m, 2, 128), torch.bfloat16), rows(rng, (2 * m, 2, 128), torch.bfloat16)
            c.write(l, K, V, st)
            q = rows(rng, (2 * m, 8, 128), torch.bfloat16) * 0.3
            out, lse = c.attn(l, q, st, with_lse=True)
    check_attn(c, [T, T], [1, 1], q, out, lse, 128 ** -0.5, layer=1)
    logits = torch.randn((B, T, vocab), device="cuda", dtype=torch.bfloat16) * 3
    ids = torch.randint(0, vocab, (B, T), device="cuda")
    scores = torch.zeros((B, T), device="cuda")
    P.score_tokens(logits[:, :-1], ids[:, 1:], scores=scores[:, 1:])
    ranker = P.SemKVCache(P.make_config(n_layers=1, n_kv_heads=2, batch=B, base=0, L_hi=6, L_lo=5, group=128, r_num=25,
                                        r_den=100, max_prompt=T, max_new=0))
    hi, _ = ranker.rank(scores)
    assert ranker.status() == 0 and hi.shape == (B, 175)
    before = [x.view(2, B, T, 2, 128) for x in c.read(-1, starts_of([T, T]), 2 * T)]
    keep = torch.zeros((4, 175), dtype=torch.int32, device="cuda")
    keep[:B] = hi
    c.compact(keep, ints([175, 175, -1, -1]))
    kept = [x.view(2, B, 175, 2, 128) for x in c.read(-1, starts_of([175, 175]), 350)]
    for b in range(B):
        for x, y in zip(before, kept):
            assert torch.equal(x[:, b, hi[b].long()], y[:, b])
    assert int((c.refs > 0).sum()) == 6
    c.fork(ints([0, 1, 0, -1]))
    c.reserve(ints([1, 1, 1, 0]))
    st = starts_of([1, 1, 1, 0])
    c.write(-1, rows(rng, (2, 3, 2, 128), torch.bfloat16), rows(rng, (2, 3, 2, 128), torch.bfloat16), st)
    q = rows(rng, (3, 8, 128), torch.bfloat16) * 0.3
    out, lse = c.attn(1, q, st, with_lse=True)
    check_attn(c, [176] * 3, [1, 1, 1], q, out, lse, 128 ** -0.5, layer=1)
    assert c.status() == 0
