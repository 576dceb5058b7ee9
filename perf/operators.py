"""Operators of the paged 4-bit cache and of token scoring, as a user's program
calls them, beside their plain forms.

Kinds of pass:

  write    K and V rows of one layer (a prompt, a chunk that starts inside a
           page, one token a sequence) quantized to 16 levels into the pages of
           their sequences, and the values that the pages then hold for them
  attn     causal attention of every sequence's last tokens over its pages: one
           token (generation), a few (verification of a draft), a prompt chunk
  beam     a step of a search over sequences: slots take over other slots'
           contents (fork), every slot gets room for its next token (reserve,
           which copies a last page that is shared), whose rows are written
  compact  every sequence keeps the listed tokens only, and its pages are freed
  logprob  log probability of given tokens, entropy, top alternatives

The plain forms are elementary torch operations in 32 bits on the same pages.

A page holds 64 tokens of every (layer, kv head); one (page, layer, kv head) is
a record: K codes, V codes, K metadata, V metadata.  Codes are 4 bits, 8 to a
32-bit word, kept in the order in which the 64 lanes of a wave load them:

  K word (piece p, lane, w): x = 4 p + w, token tile tt = x div (D/32), channel
    block i = x mod (D/32); slot j of the word is token 16 tt + lane mod 16,
    channel 32 i + 8 (lane div 16) + j
  V word (piece p, lane, w): x = 4 p + w, channel tile ct = x div 2, half st =
    x mod 2; slot j is channel 16 ct + lane mod 16, token 32 st + 16 (j div 4) +
    4 (lane div 16) + j mod 4
  slot j sits at bits 4 (j div 2 + 4 (j mod 2)) of its word
  metadata: fp16 {scale, zero} of (channel group, token) at [group][token]
"""
import math

import torch

own = False

PAGE = 64
DTYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}


def _pages(kind, name, **k):
    c = dict(kind=kind, layers=1, kv_heads=8, gqa=4, dim=128, group=128, seqs=1, ctx=2048, ragged=0, new=1, dtype="fp16")
    c.update(k)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one generated token of 16 conversations: a launch
        _pages("write", "write_token_b16", seqs=16, ctx=4000, ragged=60),
        # a short prompt of one layer, fine metadata
        _pages("write", "write_prompt_2k_g32", ctx=2048, new=2048, group=32, dtype="bf16"),
        # ragged prompts' last chunks, which start inside pages
        _pages("write", "write_chunks_b6", seqs=6, ctx=20011, ragged=50, new=16001),
        # one generated token over a short context: latency
        _pages("attn", "attn_token_2k_g32", ctx=2048, group=32, dtype="bf16"),
        # one generated token over a long context
        _pages("attn", "attn_token_32k", ctx=32768),
        # batched serving, every sequence of its own length
        _pages("attn", "attn_token_b16_16k", seqs=16, ctx=16384, ragged=50, dtype="bf16"),
        # verification of a draft of five tokens, 64-channel heads
        _pages("attn", "attn_verify5_b4_32k_d64", seqs=4, ctx=32771, ragged=20, new=5, dim=64, group=64),
        # a prompt chunk over what is cached already
        _pages("attn", "attn_chunk_2k_over_16k", ctx=18432, new=2048, dtype="bf16"),
        # a search step over 16 slots, every layer's pages
        _pages("beam", "beam_b16_2k", seqs=16, ctx=2021, ragged=0, layers=8),
        # a quarter of every sequence's tokens is kept
        _pages("compact", "compact_b4_16k", seqs=4, ctx=16384, ragged=10, layers=4, keep=25),
        # scoring of one generated token of 4 conversations, with alternatives
        dict(kind="logprob", name="logprob_token_b4", rows=4, vocab=128000, dtype="bf16", top=5),
        # self-information and entropy of a prompt
        dict(kind="logprob", name="logprob_prompt_4k", rows=4096, vocab=128000, dtype="fp16", top=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(("write", "attn", "beam", "compact", "logprob"), (3, 5, 2, 2, 3))[0]
    if kind == "logprob":
        vocab = _log(rng, 1000, 160000)
        return dict(kind=kind, rows=_log(rng, 1, max(1, min(8192, 300_000_000 // vocab))), vocab=vocab,
                    dtype=rng.choice(("bf16", "fp16", "fp32")), top=rng.choice((0, 1, 5, rng.randint(2, 20))))
    dim = rng.choice((128, 128, 64))
    c = _pages(kind, None, kv_heads=rng.choice((8, 8, 4, 2)), gqa=rng.choice((4, 4, 1, 2, 7, 8)), dim=dim,
               group=rng.choice((32, 64, dim, dim)), seqs=rng.choice((1, 2, 3, 4, 8, 16)), ragged=rng.choice((0, 20, 50, 90)),
               dtype=rng.choice(("fp16", "bf16")))
    if kind == "write":
        c["ctx"] = _log(rng, 100, 65536 // c["seqs"])
        c["new"] = rng.choice((1, c["ctx"], _log(rng, 1, c["ctx"])))
    elif kind == "attn":
        c["ctx"] = _log(rng, 100, min(65536, 262144 // c["seqs"]))
        c["new"] = rng.choice((1, 1, 1, rng.randint(2, 8), _log(rng, 8, 2048)))
        c["new"] = max(1, min(c["new"], c["ctx"], (1 << 30) // (c["ctx"] * c["seqs"] * c["kv_heads"] * c["gqa"])))
    elif kind == "beam":
        c.update(ctx=_log(rng, 100, 4000), layers=_log(rng, 1, 8))
    else:
        c.update(ctx=_log(rng, 100, 65536 // c["seqs"]), layers=_log(rng, 1, 4), keep=rng.randint(5, 90))
    return c


# ------------------------------------------------------------------ inputs --

def _lens(case):
    """Tokens of every sequence, the last call's new ones included, and how many of them are new."""
    s = case["seqs"]
    lens = [max(1, case["ctx"] - i * case["ctx"] * case["ragged"] // (100 * s)) for i in range(s)]
    new = [min(n, max(1, case["new"] - i * case["new"] * case["ragged"] // (100 * s))) for i, n in enumerate(lens)]
    return lens, new


def _gen(seed, key):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + key * 7919 + 12345) % (1 << 62))
    return g


def _rows(g, shape, dtype, keys):
    """K or V rows: normal values; in keys, a few channels of larger magnitude."""
    x = torch.randn(shape, generator=g, device="cuda")
    if keys:
        x[..., 5::37] *= 8.0
        x[..., 11::53] += 4.0
    return x.to(dtype)


def prepare(case, seed):
    g = _gen(seed, 1)
    if case["kind"] == "logprob":
        n, v = case["rows"], case["vocab"]
        x = torch.randn((n, v), generator=g, device="cuda", dtype=torch.float32 if case["dtype"] == "fp32" else torch.float16)
        x *= 2.5
        x = x.to(DTYPES[case["dtype"]])
        # most of the text's tokens are among the likelier ones
        ids = torch.randint(0, v, (n,), generator=g, device="cuda")
        x[torch.arange(n, device="cuda"), ids] += 9.0 * torch.rand((n,), generator=g, device="cuda").to(x.dtype)
        return dict(case=case, logits=x, ids=ids)
    dt, d, h, layers, seqs = DTYPES[case["dtype"]], case["dim"], case["kv_heads"], case["layers"], case["seqs"]
    lens, new = _lens(case)
    width = (max(lens) + 1 + PAGE - 1) // PAGE
    held = [(n + PAGE - 1) // PAGE for n in lens]
    total = sum(held)
    n_pages = total + (total if case["kind"] == "compact" else 2 * seqs) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((seqs, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(held):
        table[s, :n] = order[at:at + n]
        at += n
    k = _rows(g, (layers * n_pages * h * PAGE, d), torch.float16, True)
    v = _rows(g, (layers * n_pages * h * PAGE, d), torch.float16, False)
    pool = _record(*_quantize(k, case["group"]), *_quantize(v, case["group"]), (n_pages, layers, h), d, case["group"])
    state = dict(case=case, pool=pool, table=table, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    starts = torch.tensor([sum(new[:i]) for i in range(seqs + 1)], dtype=torch.int32, device="cuda")
    n = sum(new)
    if case["kind"] == "write":
        # K and V as slices of a fused projection's output
        kv = torch.cat((_rows(g, (n, h, d), dt, True), _rows(g, (n, h, d), dt, False)), dim=1)
        state.update(k=kv[:, :h], v=kv[:, h:], starts=starts, ends=starts, tokens=n, most=max(new))
    elif case["kind"] == "attn":
        q = torch.randn((n, h * case["gqa"], d), generator=g, device="cuda").to(dt)
        state.update(q=q, starts=starts, tokens=n, most=max(new))
    elif case["kind"] == "beam":
        # a third of the slots keeps its content, the rest takes another slot's; one ends
        parent = torch.randint(0, seqs, (seqs,), generator=g, device="cuda").to(torch.int32)
        keep = torch.rand((seqs,), generator=g, device="cuda") < 0.3
        parent = torch.where(keep, torch.arange(seqs, dtype=torch.int32, device="cuda"), parent)
        if seqs > 2:
            parent[1] = -1
        up = torch.where(parent < 0, 0, 1).to(torch.int32)
        n, most = int(up.sum()), min(lens) % PAGE + 1      # new tokens; rows of a last page, the new one among them
        ends = torch.cat((torch.zeros_like(up[:1]), up.cumsum(0).to(torch.int32)))
        state.update(parent=parent, up=up, ends=ends, starts=ends * most, tokens=n * most, most=most,
                     k=_rows(g, (layers, n, h, d), dt, True), v=_rows(g, (layers, n, h, d), dt, False))
    else:
        kept = [max(1, n * case["keep"] // 100) for n in lens]
        lists = torch.zeros((seqs, max(kept)), dtype=torch.int32, device="cuda")
        for s, (n, m) in enumerate(zip(lens, kept)):
            lists[s, :m] = torch.randperm(n, generator=g, device="cuda")[:m].sort().values.to(torch.int32)
        starts = torch.tensor([sum(kept[:i]) for i in range(seqs + 1)], dtype=torch.int32, device="cuda")
        state.update(keep=lists, n_keep=torch.tensor(kept, dtype=torch.int32, device="cuda"), starts=starts, tokens=sum(kept),
                     most=max(kept))
    return state


# ------------------------------------------------------- the pages, plainly --

def _quantize(x, group):
    """16 levels a group of channels: codes [n, d], fp16 scale and zero [n, d/group]."""
    x = x.float().view(x.shape[0], -1, group)
    zero = x.amin(-1).clamp(-65504.0, 65504.0).half() + 0.0
    scale = ((x.amax(-1) - zero.float()) / 15.0).clamp(0.0, 65504.0).half()
    s = scale.float()
    inv = torch.where(s > 0, 1.0 / s, torch.zeros_like(s))
    codes = torch.round((x - zero.float()[..., None]) * inv[..., None]).clamp(0.0, 15.0).to(torch.int32)
    return codes.flatten(1), scale, zero


def _shifts(device):
    j = torch.arange(8, device=device, dtype=torch.int32)
    return 4 * (j // 2 + 4 * (j % 2))


def _words(codes):
    """Codes [..., 8] in slot order as 32-bit words."""
    return (codes << _shifts(codes.device)).sum(-1, dtype=torch.int32)


def _record(kc, ks, kz, vc, vs, vz, shape, d, group):
    """Codes and metadata of whole pages (rows in order of token) as records: uint8 [*shape, record]."""
    n, i, t = math.prod(shape), d // 32, d // 16
    k = kc.view(n, 4, 16, i, 4, 8).permute(0, 4, 2, 1, 3, 5)               # kg, token, tile, block, slot
    k = _words(k).reshape(n, 4, 16, i, 4).permute(0, 3, 1, 2, 4)           # piece, kg, token, w
    v = vc.view(n, 2, 2, 4, 4, t, 16).permute(0, 3, 6, 5, 1, 2, 4)         # kg, channel, tile, half, slot (2, 4)
    v = _words(v.reshape(n, 4, 16, t, 2, 8)).reshape(n, 4, 16, t // 2, 4).permute(0, 3, 1, 2, 4)
    km = torch.stack((ks, kz), -1).view(n, PAGE, d // group, 2).transpose(1, 2)
    vm = torch.stack((vs, vz), -1).view(n, PAGE, d // group, 2).transpose(1, 2)
    parts = [p.contiguous().view(n, -1).view(torch.uint8) for p in (k, v, km, vm)]
    return torch.cat(parts, 1).view(*shape, -1)


def _codes(records, d, group):
    """The inverse of _record: codes [n, 64, d] and metadata [n, 64, d/group] of K and V."""
    r = records.reshape(-1, records.shape[-1])
    n, i, t, c, m = r.shape[0], d // 32, d // 16, 32 * d, d // group * 256
    sh = _shifts(r.device)
    k = r[:, :c].contiguous().view(torch.int32).view(n, i, 4, 16, 4).permute(0, 2, 3, 1, 4).reshape(n, 4, 16, 4, i)
    k = (k[..., None] >> sh) & 15
    k = k.permute(0, 3, 2, 4, 1, 5).reshape(n, PAGE, d)
    v = r[:, c:2 * c].contiguous().view(torch.int32).view(n, t // 2, 4, 16, 4).permute(0, 2, 3, 1, 4).reshape(n, 4, 16, t, 2)
    v = ((v[..., None] >> sh) & 15).view(n, 4, 16, t, 2, 2, 4)
    v = v.permute(0, 4, 5, 1, 6, 3, 2).reshape(n, PAGE, d)
    km = r[:, 2 * c:2 * c + m].contiguous().view(torch.float16).view(n, d // group, PAGE, 2).transpose(1, 2)
    vm = r[:, 2 * c + m:].contiguous().view(torch.float16).view(n, d // group, PAGE, 2).transpose(1, 2)
    return k, km[..., 0], km[..., 1], v, vm[..., 0], vm[..., 1]


def _values(records, d, group):
    """K and V of whole pages in 32 bits: [n, 64, d] each."""
    kc, ks, kz, vc, vs, vz = _codes(records, d, group)
    spread = lambda m: m.float().repeat_interleave(group, -1)  # noqa: E731
    return kc * spread(ks) + spread(kz), vc * spread(vs) + spread(vz)


def _last(lens, starts, most):
    """Positions of every sequence's last tokens, [seqs, most], and which of them are there."""
    n = (starts[1:] - starts[:-1])[:, None].long()
    i = torch.arange(most, device=n.device)[None]
    return (lens[:, None].long() - n + i).clamp_min(0), i < n


def _read(state, pool, table, lens):
    """Values of every sequence's last tokens, every layer: K and V [layers, tokens, kv heads, d] as stored types."""
    c = state["case"]
    pos, there = _last(lens, state["starts"], state["most"])
    seq = torch.arange(c["seqs"], device=pos.device)[:, None].expand_as(pos)[there]
    pos = pos[there]
    first = (lens.long() - (state["starts"][1:] - state["starts"][:-1]).long()).clamp_min(0) // PAGE
    span = int(state["most"] + PAGE - 1) // PAGE + 1
    cols = (first[:, None] + torch.arange(span, device=pos.device)).clamp_max(table.shape[1] - 1)
    page = table.gather(1, cols).clamp_min(0).long()
    k, v = _values(pool[page.flatten()], c["dim"], c["group"])             # [seqs * span * layers * heads, 64, d]
    shape = (c["seqs"], span, c["layers"], c["kv_heads"], PAGE, c["dim"])
    at = pos // PAGE - first[seq]
    pick = lambda x: x.view(shape).permute(0, 1, 4, 2, 3, 5)[seq, at, pos % PAGE].transpose(0, 1).to(DTYPES[c["dtype"]])  # noqa: E731
    return pick(k).contiguous(), pick(v).contiguous()


def _write(state, table, lens, most):
    """Quantizes the rows k, v ([layers, tokens, kv heads, d], or of the one layer) of the sequences' last tokens."""
    c, pool = state["case"], state["pool"]
    d, h, grp, layers = c["dim"], c["kv_heads"], c["group"], c["layers"]
    fresh = [x.view(layers, -1, h, x.shape[-1]).transpose(0, 1)
             for y in (state["k"], state["v"]) for x in _quantize(y.reshape(-1, d), grp)]
    pos, there = _last(lens, state["ends"], most)
    seq = torch.arange(c["seqs"], device=pos.device)[:, None].expand_as(pos)[there]
    page, slot = table[seq, pos[there] // PAGE].long(), pos[there] % PAGE
    pages, at = torch.unique(page, return_inverse=True)
    held = [x.view(-1, layers, h, PAGE, x.shape[-1]) for x in _codes(pool[pages], d, grp)]
    for old, row in zip(held, fresh):
        old.permute(0, 3, 1, 2, 4)[at, slot] = row.to(old.dtype)
    pool[pages] = _record(*(x.reshape(-1, x.shape[-1]) for x in held), (len(pages), layers, h), d, grp)


def _attn(state):
    c, lens = state["case"], state["lens"]
    s, h, d, q = c["seqs"], c["kv_heads"], c["dim"], c["gqa"]
    pages = state["table"].clamp_min(0).long()
    span = pages.shape[1] * PAGE
    k, v = (x.view(s, -1, h, PAGE, d).permute(0, 2, 1, 3, 4).reshape(s * h, span, d)
            for x in _values(state["pool"][pages.flatten(), 0], d, c["group"]))
    pos, there = _last(lens, state["starts"], state["most"])
    rows = torch.zeros((s, state["most"], h, q, d), device=k.device)
    rows[there] = state["q"].float().view(-1, h, q, d)
    rows = rows.permute(0, 2, 1, 3, 4).reshape(s * h, -1, d)
    t = torch.arange(span, device=k.device)
    seen = (t <= pos[:, :, None]) & (t < lens[:, None, None]) & there[:, :, None]
    x = torch.bmm(rows, k.transpose(1, 2).contiguous()).mul_(d ** -0.5).view(s, h, -1, q, span)
    x = x.masked_fill_(~seen[:, None, :, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min(-1e30)
    p = x.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.bmm(p.view(s * h, -1, span), v).view(s, h, -1, q, d) / total.clamp_min(1e-30)
    lse = (m + total.log()).squeeze(-1)
    back = lambda y: y.transpose(1, 2)[there].flatten(1, 2)  # noqa: E731
    return back(out).to(state["q"].dtype), back(lse)


def _free(refs):
    """The free pages in ascending order, then rubbish."""
    free = refs == 0
    at = torch.where(free, free.cumsum(0) - 1, refs.numel())
    out = torch.zeros(refs.numel() + 1, dtype=torch.int32, device=refs.device)
    out[at] = torch.arange(refs.numel(), dtype=torch.int32, device=refs.device)
    return out[:-1]


def _refs(table, n_pages):
    refs = torch.zeros(n_pages + 1, dtype=torch.int32, device=table.device)
    at = torch.where(table < 0, n_pages, table).long().flatten()
    return refs.index_add_(0, at, torch.ones_like(at, dtype=torch.int32))[:-1]


def _beam(state):
    pool, parent, up = state["pool"], state["parent"].long(), state["up"]
    src = parent.clamp_min(0)
    ended = parent < 0
    table = torch.where(ended[:, None], -1, state["table"][src])
    lens = torch.where(ended, 0, state["lens"][src])
    refs = _refs(table, pool.shape[0])
    # room for the new tokens: fresh pages, and copies of last pages that others hold too
    held, want = (lens + PAGE - 1) // PAGE, (lens + up + PAGE - 1) // PAGE
    last = table.gather(1, (held.long() - 1).clamp_min(0)[:, None]).squeeze(1)
    grows = (up > 0) & (lens % PAGE != 0)
    same = (last[:, None] == last[None, :]) & grows[:, None] & grows[None, :]
    lowest = ~torch.tril(same, -1).any(1)
    copy = grows & (refs[last.clamp_min(0).long()] > 1) & ~((same.sum(1) == refs[last.clamp_min(0).long()]) & lowest)
    need = (want - held) + copy.int()
    base = (need.cumsum(0) - need).long()
    free = _free(refs)
    col = torch.arange(table.shape[1], device=table.device)[None]
    fresh = (col >= held[:, None]) & (col < want[:, None])
    rank = base[:, None] + copy[:, None].int() + col - held[:, None]
    table = torch.where(fresh, free[rank.clamp(0, free.numel() - 1)], table)
    to = torch.where(copy, free[base], last)
    pool[to[copy].long()] = pool[last[copy].long()]
    table = torch.where((col == held[:, None] - 1) & copy[:, None], to[:, None], table)
    lens = (lens + up).to(torch.int32)
    _write(state, table, lens, 1)
    return lens, table, _refs(table, pool.shape[0]), *_read(state, pool, table, lens)


def _compact(state):
    c, pool, keep, n = state["case"], state["pool"], state["keep"].long(), state["n_keep"]
    need = (n + PAGE - 1) // PAGE
    base = need.cumsum(0) - need
    col = torch.arange(state["table"].shape[1], device=n.device)[None]
    free = _free(_refs(state["table"], pool.shape[0]))
    rank = (base[:, None] + col).clamp(0, free.numel() - 1).long()
    table = torch.where(col < need[:, None], free[rank], -1)
    i = torch.arange(keep.shape[1], device=n.device)[None]
    there = i < n[:, None]
    seq = torch.arange(c["seqs"], device=n.device)[:, None].expand_as(keep)[there]
    src, dst = keep[there], i.expand_as(keep)[there]
    shape = (-1, c["layers"] * c["kv_heads"], PAGE)
    old, at = torch.unique(state["table"][seq, src // PAGE], return_inverse=True)
    new, to = torch.unique(table[seq, dst // PAGE], return_inverse=True)
    held = _codes(pool[new.long()], c["dim"], c["group"])
    for x, y in zip(held, _codes(pool[old.long()], c["dim"], c["group"])):
        x.view(*shape, x.shape[-1]).transpose(1, 2)[to, dst % PAGE] = y.view(*shape, y.shape[-1]).transpose(1, 2)[at, src % PAGE]
    whole = (len(new), c["layers"], c["kv_heads"])
    pool[new.long()] = _record(*(x.reshape(-1, x.shape[-1]) for x in held), whole, c["dim"], c["group"])
    return n.clone(), table, _refs(table, pool.shape[0]), *_read(state, pool, table, n)


def _logprob(state):
    c, x = state["case"], state["logits"].float()
    m = x.amax(-1, keepdim=True)
    e = (x - m).exp_()
    total = e.sum(-1)
    lse = m.squeeze(-1) + total.log()
    out = [x.gather(1, state["ids"][:, None]).squeeze(1) - lse, total.log() - (e * (x - m)).sum(-1) / total]
    if c["top"]:
        # ties to the lowest index: a stable descending sort
        y, at = torch.sort(x, dim=-1, descending=True, stable=True)
        out += [y[:, :c["top"]] - lse[:, None], at[:, :c["top"]].to(torch.int32)]
    return tuple(out)


def _prompt(state):
    _write(state, state["table"], state["lens"], state["most"])
    return _read(state, state["pool"], state["table"], state["lens"])


def _plain(state):
    return {"write": _prompt, "attn": _attn, "beam": _beam, "compact": _compact, "logprob": _logprob}[state["case"]["kind"]](state)


# ------------------------------------------------------------ the framework --

def _handle(state):
    """The cache object that a program keeps, over its own pool and page tables."""
    import paper_2608_28911_amd as P
    if "cache" not in state:
        c = state["case"]
        cfg = P.make_paged_config(n_layers=c["layers"], n_kv_heads=c["kv_heads"], n_q_heads=c["kv_heads"] * c["gqa"],
                                  head_dim=c["dim"], group=c["group"], n_pages=state["pool"].shape[0], max_seqs=c["seqs"],
                                  seq_pages=state["table"].shape[1])
        state["cache"] = P.PagedKV4(cfg, pool=state["pool"])
        state["cache"].assign(state["lens"], state["table"])
    return state["cache"]


def _own(state):
    import paper_2608_28911_amd as P
    c = state["case"]
    if c["kind"] == "logprob":
        return P.token_logprobs(state["logits"], state["ids"], top=c["top"])
    cache = _handle(state)
    if c["kind"] == "write":
        cache.write(0, state["k"], state["v"], state["starts"])
        return cache.read(-1, state["starts"], state["tokens"], dtype=DTYPES[c["dtype"]])
    if c["kind"] == "attn":
        return cache.attn(0, state["q"], state["starts"], with_lse=True)
    # the pass starts from the same tables each time
    cache.assign(state["lens"], state["table"])
    if c["kind"] == "beam":
        cache.fork(state["parent"])
        cache.reserve(state["up"])
        cache.write(-1, state["k"], state["v"], state["ends"])
    else:
        cache.compact(state["keep"], state["n_keep"])
    return cache.lens, cache.table, cache.refs, *cache.read(-1, state["starts"], state["tokens"], dtype=DTYPES[c["dtype"]])


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    if case["kind"] == "logprob":
        n, v = case["rows"], case["vocab"]
        size = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": n * v * size + n * 8 + n * 8 + n * case["top"] * 8, "flops": 5 * n * v}
    d, h, q = case["dim"], case["kv_heads"], case["gqa"]
    lens, new = _lens(case)
    row = d + 8 * (d // case["group"])                       # K and V of one token and kv head
    if case["kind"] == "write":
        n = sum(new) * h
        return {"bytes": n * (4 * d + 2 * row + 4 * d), "flops": n * 2 * d * 6}
    if case["kind"] == "attn":
        seen = sum(a * n - n * (n - 1) // 2 for a, n in zip(lens, new))
        return {"bytes": sum(lens) * h * row + sum(new) * h * q * (4 * d + 4), "flops": 4 * d * h * q * seen}
    if case["kind"] == "beam":
        last = min(lens) % PAGE + 1
        n = case["seqs"] * case["layers"] * h
        return {"bytes": n * last * (2 * row + 4 * d), "flops": n * last * 2 * d}
    kept = sum(max(1, n * case["keep"] // 100) for n in lens) * case["layers"] * h
    return {"bytes": kept * (3 * row + 4 * d), "flops": kept * 2 * d}


# ------------------------------------------------------------ 64-bit values --

def _place(d):
    """Where (token, channel) of a record sits: word and shift in K, then in V."""
    t = torch.arange(PAGE)[:, None]
    e = torch.arange(d)[None, :]
    x = (t // 16) * (d // 32) + e // 32
    kw = (x // 4 * 64 + (e % 32) // 8 * 16 + t % 16) * 4 + x % 4
    kj = (e % 8).expand(PAGE, d)
    y = (e // 16) * 2 + t // 32
    vw = (y // 4 * 64 + (t % 16) // 4 * 16 + e % 16) * 4 + y % 4
    vj = ((t % 32) // 16 * 4 + t % 4).expand(PAGE, d)
    place = lambda w, j: (w.expand(PAGE, d).cuda(), (4 * (j // 2) + 16 * (j % 2)).cuda())  # noqa: E731
    return place(kw, kj), place(vw, vj)


def _exact_rows(pool, table, seq, layer, head, lo, hi, d, group):
    """K and V of positions lo .. hi-1 of one sequence, one layer and kv head, in 64 bits."""
    pages = table[seq, lo // PAGE:(hi + PAGE - 1) // PAGE].long()
    rec = pool[pages, layer, head]
    out = []
    for (word, shift), codes, meta in zip(_place(d), (0, 32 * d), (64 * d, 64 * d + 256 * (d // group))):
        w = rec[:, codes:codes + 32 * d].contiguous().view(torch.int32).long()
        m = rec[:, meta:meta + 256 * (d // group)].contiguous().view(torch.float16).double().view(len(pages), d // group, PAGE, 2)
        c = ((w[:, word] >> shift) & 15).double().view(len(pages), PAGE, d // group, group)
        x = c * m[..., 0].transpose(1, 2)[..., None] + m[..., 1].transpose(1, 2)[..., None]
        out.append(x.reshape(-1, d)[lo % PAGE:lo % PAGE + hi - lo])
    return out


def _exact_stored(x, group):
    """What 16 levels keep of the rows x: the definition's steps, of which the reciprocal, the difference and the
    product are rounded to 32 bits."""
    x = x.double().unflatten(-1, (-1, group))
    to16, to32 = lambda y: y.to(torch.float16).double(), lambda y: y.to(torch.float32).double()  # noqa: E731
    z = to16(x.min(-1, keepdim=True).values.clamp(-65504, 65504))
    s = to16(to32(to32(x.max(-1, keepdim=True).values - z) / 15).clamp(0, 65504))
    t = to32(to32(x - z) * to32(1 / torch.where(s > 0, s, torch.ones_like(s))))
    c = torch.where(s > 0, t.round().clamp(0, 15), torch.zeros_like(t))
    return (c * s + z).flatten(-2)


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "logprob":
        parts = []
        for i in range(0, case["rows"], 64):
            x = state["logits"][i:i + 64].double()
            lse = torch.logsumexp(x, -1)
            p = (x - lse[:, None]).exp()
            part = [x[torch.arange(len(x)), state["ids"][i:i + 64]] - lse, -(p * (x - lse[:, None])).sum(-1)]
            if case["top"]:
                part.append(x.topk(case["top"], -1).values - lse[:, None])
            parts.append(part)
        out = [torch.cat(p) for p in zip(*parts)]
        return (*out, None) if case["top"] else tuple(out)
    d, h, q, grp = case["dim"], case["kv_heads"], case["gqa"], case["group"]
    if case["kind"] == "write":
        return _exact_stored(state["k"], grp)[None], _exact_stored(state["v"], grp)[None]
    lens, new = _lens(case)
    if case["kind"] == "attn":
        out = torch.zeros((sum(new), h * q, d), dtype=torch.float64, device="cuda")
        lse = torch.zeros((sum(new), h * q), dtype=torch.float64, device="cuda")
        for s, (n, m) in enumerate(zip(lens, new)):
            at = sum(new[:s])
            for j in range(h):
                k, v = _exact_rows(state["pool"], state["table"], s, 0, j, 0, n, d, grp)
                for g in range(j * q, (j + 1) * q):
                    x = state["q"][at:at + m, g].double() @ k.t() / math.sqrt(d)
                    if m > 1:
                        x += torch.triu(torch.full_like(x, -math.inf), n - m + 1)
                    lse[at:at + m, g] = torch.logsumexp(x, -1)
                    out[at:at + m, g] = (x - lse[at:at + m, g, None]).exp_() @ v
        return out, lse
    beam = case["kind"] == "beam"
    if beam:     # the last rows of the parent, then the slot's own new one
        most = state["most"]
        rows = [(p, torch.arange(lens[p] + 1 - most, lens[p], device="cuda")) for p in state["parent"].tolist() if p >= 0]
        fresh = [_exact_stored(state[x], grp) for x in ("k", "v")]
    else:
        rows = [(s, state["keep"][s, :n].long()) for s, n in enumerate(state["n_keep"].tolist())]
    values = []
    for layer in range(case["layers"]):
        per = []
        for i, (s, at) in enumerate(rows):
            heads = [_exact_rows(state["pool"], state["table"], s, layer, j, 0, lens[s], d, grp) for j in range(h)]
            per.append([torch.stack([x[kv][at] for x in heads], 1) for kv in range(2)])
            if beam:
                per[-1] = [torch.cat((x, fresh[kv][layer, i:i + 1])) for kv, x in enumerate(per[-1])]
        values.append([torch.cat([p[kv] for p in per]) for kv in range(2)])
    return None, None, None, torch.stack([x[0] for x in values]), torch.stack([x[1] for x in values])
