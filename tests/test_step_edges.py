"""Append with rotation, the cache of latents and beam search's choice where they went
wrong once: no GPU."""
import os
import re
import subprocess


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
