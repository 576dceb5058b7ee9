"""Append with rotation, the cache of latents and beam search's choice where they went
wrong once: no GPU."""
import os
import re
import subprocess

import pytest

from tests.test_step import abi, host  # noqa: F401


def assembly(source, tmp_path):
    """The gfx950 assembly of one of the library's sources: {kernel: its lines}."""
    from paper_2608_28911_amd import build as B
    out = str(tmp_path / "a.s")
    cmd = [B.HIPCC, "--cuda-device-only", "-S", os.path.join(B.CSRC, source), "-o", out] + B.COMMON + B.SOURCES[source]
    subprocess.run(cmd, check=True, capture_output=True)
    kernels, lines = {}, None
    with open(out) as f:
        for line in f:
            line = line.split(";")[0].strip()
            name = re.match(r"(_Z\w+):$", line)
            if name:
                lines = kernels.setdefault(name.group(1), [])
            elif line.startswith(".Lfunc_end"):
                lines = None
            elif line and lines is not None:
                lines.append(line)
    return kernels


def ends_without_loading(lines):
    """Whether a wave can reach the kernel's end before any vector load.  (A branch that skips lanes that are masked
    off counts as not taken: some lane has what is behind it to do.)"""
    at = {line[:-1]: i for i, line in enumerate(lines) if line.endswith(":")}
    todo, been = [0], set()
    while todo:
        i = todo.pop()
        while i < len(lines) and i not in been:
            been.add(i)
            op = lines[i].split()[0]
            if re.match(r"(global|flat|buffer)_load", op):
                break
            if op == "s_endpgm":
                return True
            if op == "s_branch":
                i = at[lines[i].split()[1]]
                continue
            if op.startswith("s_cbranch") and op != "s_cbranch_execz":
                todo.append(at[lines[i].split()[1]])
            i += 1
    return False


def test_logits_of_a_beam_without_candidates_are_not_loaded(tmp_path):
    """A beam that is not in use, or has ended, may have no logits in memory: its row's workgroups end before the first
    load of them (the score and whether it has ended come by scalar loads)."""
    rows = {k: v for k, v in assembly("beam.hip", tmp_path).items() if "beam_rows_kernel" in k}
    assert len(rows) == 3
    for name, lines in rows.items():
        assert ends_without_loading(lines), name


def bytes_of(t):
    """Addresses of every byte of a small tensor's elements."""
    import itertools
    at = {t.data_ptr() + t.element_size() * sum(i * s for i, s in zip(index, t.stride()))
          for index in itertools.product(*map(range, t.shape))}
    return {a + b for a in at for b in range(t.element_size())}


def test_overlap_is_that_of_elements():
    """Views of one buffer, of any strides: whether an element of one lies in the other."""
    import random
    import torch
    from paper_2608_28911_amd.paged import _overlap
    rng, found = random.Random(5), [0, 0]
    buf = torch.zeros(600, dtype=torch.int16)
    for _ in range(4000):
        pair = []
        for _ in range(2):
            n, h, d = rng.randint(1, 5), rng.randint(1, 4), rng.choice((1, 2, 4, 8))
            pitch = rng.choice((d, d + 4, 8, 24))
            strides = rng.choice(((h * pitch, pitch, 1), (rng.choice((24, 48, 64)), pitch, 1), (d, n * d, 1), (0, pitch, 1)))
            pair.append(buf.as_strided((n, h, d), strides, rng.randint(0, 100)))
        a, b = pair
        if rng.random() < 0.2:
            b = b.reshape(-1)[:0] if rng.random() < 0.3 else b[0, 0]
        meet = bool(bytes_of(a) & bytes_of(b))
        assert _overlap(a, b) == _overlap(b, a) == meet, (a.stride(), a.shape, a.storage_offset(), b.stride(), b.shape, b.storage_offset())
        found[meet] += 1
    assert min(found) > 500


def test_overlap_of_large_views():
    import torch
    from paper_2608_28911_amd.paged import _overlap
    buf = torch.empty((40000, 48, 64), dtype=torch.int16)                 # (never touched)
    assert not _overlap(buf[:, :32], buf[:, 32:40]) and _overlap(buf[:, :33], buf[:, 32:40])
    assert not _overlap(buf[..., :32], buf[..., 32:]) and _overlap(buf[..., :33], buf[..., 32:])
    assert not _overlap(buf[:20000], buf[20000:]) and _overlap(buf[:20001], buf[20000:])


def test_where_queries_are_turned_to(host):  # noqa: F811
    """Another slice of the projection's buffer will do; what holds an input of the call will not, q itself but for."""
    import torch
    rec, kv, lat = host
    n = 5
    st, f, pos = torch.tensor([0, 2, n], dtype=torch.int32), torch.ones(64), torch.arange(n, dtype=torch.int32)
    qkv = torch.zeros((n, 20, 128), dtype=torch.float16)
    q, k, v, more = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:12], qkv[:, 12:]
    for out in (q, more, torch.zeros_like(q)):
        assert kv.append(0, k, v, st, f, q=q, positions=pos, q_out=out) is out
        assert rec.calls.pop()[0] == "semkv_paged_append"
    halves = torch.zeros((n, 8, 256), dtype=torch.float16)               # every head's other half
    assert kv.append(0, k, v, st, f, q=halves[..., :128], q_out=halves[..., 128:]).data_ptr() == halves.data_ptr() + 256
    tight = torch.zeros(n * (7 * 256 + 128), dtype=torch.float16).as_strided((n, 8, 128), (7 * 256 + 128, 256, 1))
    assert kv.append(0, k, v, st, f, q=q, q_out=tight) is tight
    rec.calls.clear()
    small = torch.zeros(n * 8 * 128, dtype=torch.float16)
    over = small.view(n, 8, 128)
    starts, places, turns = small[:6].view(torch.int32), small[64:64 + 2 * n].view(torch.int32), small[128:256].view(torch.float32)
    for bad in (lambda: kv.append(0, k, v, st, f, q=q, q_out=qkv[:, 2:10]), lambda: kv.append(0, k, v, st, f, q=q, q_out=qkv[:, 11:19]),
                lambda: kv.append(0, q[:, 6:], v, st, f, q=q, q_out=q),
                lambda: kv.append(0, k, v, starts, f, q=q, q_out=over), lambda: kv.append(0, k, v, st, turns, q=q, q_out=over),
                lambda: kv.append(0, k, v, st, f, q=q, positions=places, q_out=over)):
        with pytest.raises(ValueError):
            bad()
    f = f[:32]
    rows, ql = torch.zeros((n, 576 + 3 * 64), dtype=torch.float16), torch.zeros((n, 3, 64), dtype=torch.float16)
    C, R, beside = rows[:, :512], rows[:, 512:576], rows[:, 576:].unflatten(1, (3, 64))
    assert lat.append(0, C, R, st, f, q=ql, q_out=beside) is beside and lat.append(0, C, R, st, f, q=beside, q_out=beside) is beside
    rec.calls.clear()
    for out in (rows[:, 512:704].unflatten(1, (3, 64)), rows[:, 320:512].unflatten(1, (3, 64))):
        with pytest.raises(ValueError):
            lat.append(0, C, R, st, f, q=ql, q_out=out)
    assert not rec.calls
