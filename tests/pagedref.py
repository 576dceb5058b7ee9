"""Plain model of the paged 4-bit cache for the tests (numpy, 64 bits, loops):
the record layout from its definition, the quantizer's steps, the page tables
as Python lists, attention over the stored values."""
import numpy as np

PAGE = 64
NO_PAGES, BAD_INDEX, NONFINITE = 8, 4, 2


def places(d):
    """(word, shift) of (token, channel) in K and in V, by the definition."""
    kw, ks, vw, vs = (np.zeros((PAGE, d), np.int64) for _ in range(4))
    for w in range(8 * d):                       # word of K or V: piece, lane, position
        p, lane, x = w // 256, w // 4 % 64, 4 * (w // 256) + w % 4
        for j in range(8):
            bit = 4 * (j // 2 + 4 * (j % 2))
            t, c = 16 * (x // (d // 32)) + lane % 16, 32 * (x % (d // 32)) + 8 * (lane // 16) + j
            kw[t, c], ks[t, c] = w, bit
            t, c = 32 * (x % 2) + 16 * (j // 4) + 4 * (lane // 16) + j % 4, 16 * (x // 2) + lane % 16
            vw[t, c], vs[t, c] = w, bit
    return (kw, ks), (vw, vs)


_PLACES = {d: places(d) for d in (64, 128)}


def unpack(rec, d, group):
    """One record's bytes -> [(codes [64, d], scale, zero [64, d/group] fp16) of K, of V]."""
    n, m, out = 32 * d, 256 * (d // group), []
    for kv in range(2):
        w = rec[kv * n:(kv + 1) * n].view(np.uint32).astype(np.int64)
        word, bit = _PLACES[d][kv]
        meta = rec[2 * n + kv * m:2 * n + (kv + 1) * m].view(np.float16).reshape(d // group, PAGE, 2)
        out.append(((w[word] >> bit) & 15, meta[..., 0].T, meta[..., 1].T))
    return out


def values(rec, d, group):
    """Stored K and V values of a record, 64 bits."""
    return [c * np.repeat(s.astype(np.float64), group, 1) + np.repeat(z.astype(np.float64), group, 1)
            for c, s, z in unpack(rec, d, group)]


def quantize(x, group):
    """Rows x (float32 of fp16 or bf16 values) -> codes, scale, zero; every step as defined."""
    f = np.float32
    g = np.asarray(x, f).reshape(x.shape[0], -1, group)
    with np.errstate(all="ignore"):
        bad = ~np.isfinite(g).all(-1)
        mn = np.clip(g.min(-1), f(-65504), f(65504)).astype(np.float16) + np.float16(0)
        z = mn.astype(f)
        s16 = np.clip((g.max(-1) - z) / f(15), f(0), f(65504)).astype(np.float16)
        s = s16.astype(f)
        inv = np.where(s > 0, f(1) / np.where(s > 0, s, f(1)), f(0)).astype(f)
        c = np.clip(np.rint((g - z[..., None]) * inv[..., None]), 0, 15)
        c = np.where(bad[..., None], 0, np.nan_to_num(c)).astype(np.int64)
        s16, mn = np.where(bad, np.float16(0), s16), np.where(bad, np.float16(0), mn)
    return c.reshape(x.shape), s16, mn


def store(rec, t, kv, codes, scale, zero, d, group):
    """Row t of a record's K (kv = 0) or V."""
    n, m = 32 * d, 256 * (d // group)
    w = rec[kv * n:(kv + 1) * n].view(np.uint32)
    word, bit = _PLACES[d][kv]
    for c in range(d):
        i, b = word[t, c], np.uint32(bit[t, c])
        w[i] = (w[i] & ~(np.uint32(15) << b)) | (np.uint32(codes[c]) << b)
    meta = rec[2 * n + kv * m:2 * n + (kv + 1) * m].view(np.float16).reshape(d // group, PAGE, 2)
    meta[:, t, 0], meta[:, t, 1] = scale, zero


class Pages:
    """Page tables as the calls are defined, one sequence after another."""

    def __init__(self, n_pages, max_seqs, seq_pages):
        self.n_pages, self.seq_pages = n_pages, seq_pages
        self.lens, self.rows = [0] * max_seqs, [[] for _ in range(max_seqs)]
        self.stalled = 0

    def refs(self):
        r = [0] * self.n_pages
        for row in self.rows:
            for p in row:
                if p >= 0:
                    r[p] += 1
        return r

    def free(self):
        return [p for p, n in enumerate(self.refs()) if n == 0]

    def table(self):
        return np.array([r + [-1] * (self.seq_pages - len(r)) for r in self.rows], np.int32)

    def reserve(self, n_new):
        """Returns (status, copies [(page, copy)])."""
        refs, free, copies, lens, rows = self.refs(), self.free(), [], list(self.lens), [list(r) for r in self.rows]
        st = BAD_INDEX if any(n < 0 for n in n_new) else 0
        grows = {}
        for s, n in enumerate(n_new):
            if n > 0 and lens[s] % PAGE and rows[s][-1] >= 0:
                grows.setdefault(rows[s][-1], []).append(s)
        try:
            for s, n in enumerate(max(n, 0) for n in n_new):
                if lens[s] + n > self.seq_pages * PAGE:
                    raise IndexError
                if n > 0 and lens[s] % PAGE and rows[s][-1] >= 0:
                    p = rows[s][-1]
                    if refs[p] > 1 and (len(grows[p]) != refs[p] or s != min(grows[p])):
                        rows[s][-1] = free.pop(0)
                        copies.append((p, rows[s][-1]))
                lens[s] += n
                while len(rows[s]) * PAGE < lens[s]:
                    rows[s].append(free.pop(0))
        except IndexError:
            self.stalled = 1
            return st | NO_PAGES, []
        self.lens, self.rows, self.stalled = lens, rows, 0
        return st, copies

    def fork(self, parent):
        bad = [not -1 <= p < len(self.lens) for p in parent]
        parent = [s if b else p for s, (p, b) in enumerate(zip(parent, bad))]
        old = [(n, list(r)) for n, r in zip(self.lens, self.rows)] + [(0, [])]
        self.lens, self.rows = [old[p][0] for p in parent], [list(old[p][1]) for p in parent]
        return BAD_INDEX if any(bad) else 0

    def compact(self, n_keep, ld):
        """Returns (status, {slot: (its former pages, fresh pages)})."""
        ok = [-1 <= n <= min(ld, PAGE * self.seq_pages) for n in n_keep]
        st, free, moved = 0 if all(ok) else BAD_INDEX, self.free(), {}
        n_keep = [n if o else -1 for n, o in zip(n_keep, ok)]
        if sum(-(-n // PAGE) for n in n_keep if n > 0) > len(free):
            return st | NO_PAGES, {}
        for s, n in enumerate(n_keep):
            if n >= 0:
                fresh = [free.pop(0) for _ in range(-(-n // PAGE))]
                moved[s] = (self.rows[s], fresh)
                self.rows[s], self.lens[s] = fresh, n
        return st, moved


def attend(q, k, v, seen, scale):
    """One row: out, lse over the first `seen` tokens; and the p."""
    if seen <= 0:
        return np.zeros(v.shape[1]), -np.inf, np.zeros(0)
    x = (k[:seen] @ q) * scale
    m = x.max()
    e = np.exp(x - m)
    p = e / e.sum()
    return p @ v[:seen], m + np.log(e.sum()), p
