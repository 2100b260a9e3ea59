"""Operators of a serving loop whose paged key/value cache is held in 8 bits: what each computes, from one user's token to a full batch.

Kinds:

  append   n new K/V rows per sequence rounded to 8 bits (e4m3 or int8) into the pages that the sequence's table names, with a scale, a power of
           two, for each block of tokens and head; a block that older rows have begun keeps its scale, or is rounded again under a larger one
  attend   attention of the newest n tokens of every sequence (n = 1, or drafted tokens with the causal mask) over such pages
  fork     continuations of prompts begin: those of the last turn give their pages back, new ones share their prompt's pages, get pages of their own for
           the next n tokens, and a copy of the page that the prompt has begun
  compact  the pages in use move to the front of the pool, and the tables name their new places
  adjust   logits of the next token (and behind drafted tokens) with penalties for repeated tokens, biases, and the tokens that a grammar leaves

Sizes are those of the repository's workloads (h=8, k=v=128; the long-context probe b=64, m=8192, h=32; the ragged batch b=512,
h=64, lengths 1..4096; vocabulary 32768) and the ranges around them.

`run` computes an operator in its plain form from torch's elementary operations, or, with `own` set, through the package.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1, "int8": 1}
LARGEST = {"e4m3": 448.0, "int8": 127.0}


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a decoding step's new rows: one per sequence, 128 sequences
        dict(name="append_tokens_b128", kind="append", b=128, n=1, ragged=False, h_kv=0, kv=128, m=255, page=16, block=16, dtype="e4m3"),
        # a padded batch of prompts taken into the cache
        dict(name="append_prompts_b64", kind="append", b=64, n=1024, ragged=True, h_kv=0, kv=128, m=0, page=16, block=16, dtype="int8"),
        # one user: latency
        dict(name="attend_b1", kind="attend", b=1, n=1, h=8, h_kv=0, kv=128, m=128, page=16, block=16, dtype="int8", ragged=False),
        # drafted tokens under verification, mixed lengths; a K/V head for each of 8 heads of 64
        dict(name="attend_drafts_b32", kind="attend", b=32, n=5, h=8, h_kv=8, kv=64, m=2048, page=32, block=8, dtype="int8", ragged=True),
        # long contexts, all full, large pages
        dict(name="attend_long", kind="attend", b=64, n=1, h=32, h_kv=0, kv=128, m=8192, page=64, block=64, dtype="e4m3", ragged=False),
        # a large serving batch of mixed lengths with many heads
        dict(name="attend_ragged_b512", kind="attend", b=512, n=1, h=64, h_kv=0, kv=128, m=4096, page=16, block=16, dtype="e4m3", ragged=True),
        # one prompt, four continuations
        dict(name="fork_b1", kind="fork", b=1, children=4, n=1, h_kv=0, kv=128, m=200, page=16, block=16, dtype="e4m3", spare=64),
        # many prompts of mixed lengths, eight continuations each, K/V heads, tokens to be drafted
        dict(name="fork_b64", kind="fork", b=64, children=8, n=5, h_kv=8, kv=128, m=4096, page=16, block=16, dtype="e4m3", spare=4096),
        # a small pool after a few sequences have ended, and a large one, half of it free
        dict(name="compact_small", kind="compact", b=8, h_kv=0, kv=128, m=256, page=16, block=16, dtype="bf16", pages=256),
        dict(name="compact_large", kind="compact", b=128, h_kv=0, kv=128, m=4096, page=16, block=16, dtype="bf16", pages=65536),
        # one user's next token, and drafted tokens of a batch with long histories
        dict(name="adjust_b1", kind="adjust", b=1, n=0, vocab=32768, history=500, biases=0, masked=True, ragged=False),
        dict(name="adjust_b64", kind="adjust", b=64, n=4, vocab=32768, history=8192, biases=100, masked=True, ragged=True),
    ]


def _log(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "attend", "fork", "compact", "adjust"])
    if kind == "adjust":
        vocab, n = _log(rng, 100, 65536), rng.choice([0, 0, rng.randint(1, 8)])
        return dict(kind=kind, b=_log(rng, 1, max(1, min(256, (1 << 23) // (vocab * (n + 1))))), n=n, vocab=vocab, history=_log(rng, 1, 8192),
                    biases=rng.choice([0, 0, rng.randint(1, 300)]), masked=rng.random() < 0.5, ragged=rng.random() < 0.5)
    block = rng.choice([16, 16, 32, 64, 8, 1, rng.randint(1, 40)])
    page = block * rng.choice([1, 1, 2, 4, rng.randint(1, 5)])
    kv = rng.choice([128, 128, 128, 64, 16 * rng.randint(1, 16)])
    dtype = rng.choice(["e4m3", "e4m3", "int8"])
    h_kv = rng.choice([0, 0, 0, rng.randint(1, 8)])
    heads = max(1, h_kv)
    ragged = rng.random() < 0.5
    if kind == "append":
        n = rng.choice([1, rng.randint(2, 8), _log(rng, 2, 1024)])
        b = _log(rng, 1, max(1, min(512, 65536 // (n * heads))))
        return dict(kind=kind, b=b, n=n, ragged=ragged, h_kv=h_kv, kv=kv, m=rng.randint(0, 512), page=page, block=block, dtype=dtype)
    if kind == "attend":
        m = _log(rng, 1, 8192)
        n = min(m, rng.choice([1, 1, 1, rng.randint(2, 8)]))
        h = heads * rng.randint(1, max(1, 64 // heads // n))
        b = _log(rng, 1, max(1, min(512, (1 << 18) // (m * heads), (1 << 25) // (m * h * n))))
        return dict(kind=kind, b=b, n=n, h=h, h_kv=h_kv, kv=kv, m=m, page=page, block=block, dtype=dtype, ragged=ragged)
    dtype = rng.choice(["e4m3", "int8", "bf16", "f32"])
    if kind == "fork":
        m, children = _log(rng, 1, 4096), rng.randint(1, 8)
        n = rng.choice([1, 1, rng.randint(2, 40)])
        b = _log(rng, 1, max(1, min(64, (1 << 18) // (m * heads), (1 << 24) // (children * page * heads * kv * BYTES[dtype]))))
        # now and then fewer pages than everybody needs
        most = b * children * (n // page + 2)
        return dict(kind=kind, b=b, children=children, n=n, h_kv=h_kv, kv=kv, m=m, page=page, block=block, dtype=dtype,
                    spare=rng.choice([most, most, rng.randint(1, most)]))
    m = _log(rng, 1, 4096)
    b = _log(rng, 1, max(1, min(128, (1 << 16) // (m * heads))))
    return dict(kind=kind, b=b, h_kv=h_kv, kv=kv, m=m, page=page, block=block, dtype=dtype, pages=b * (-(-m // page) + 1) + rng.randint(0, (1 << 16) // (page * heads)))


# ------------------------------------------------------------------------------------------ inputs
def _lengths(c):
    """The lengths of a case, shortest to longest (`prepare` deals them out by its seed)."""
    lo, hi, b = min(c["m"], max(1, c.get("n", 1))), c["m"], c["b"]
    return [hi] * b if not c.get("ragged", True) or b == 1 else [lo + (hi - lo) * i // (b - 1) for i in range(b)]


def _counts(c):
    n, b = c["n"], c["b"]
    return [n] * b if not c["ragged"] or b == 1 else [max(1, n * i // (b - 1)) for i in range(b)]


def _deal(values, g):
    t = torch.tensor(values, dtype=torch.int32, device=DEV)
    return t[torch.randperm(len(values), generator=g, device=DEV)].contiguous()


def _scale_of(largest, dtype):
    """The smallest power of two, 2^-126 at least, under which `largest` is no more than the type holds."""
    m, e = torch.frexp(largest.double() / LARGEST[dtype])                                  # m in [0.5, 1)
    e = torch.where(m == 0.5, e - 1, e).clamp(min=-126)
    return torch.where(largest > 0, torch.ldexp(torch.ones_like(m), e), torch.full_like(m, 2.0 ** -126)).float()


def _to_8_bits(x, dtype):
    """Float values of the type's range, rounded to the nearest (the even one of two)."""
    top = LARGEST[dtype]
    return x.clamp(-top, top).to(torch.float8_e4m3fn) if dtype == "e4m3" else x.clamp(-top, top).round().to(torch.int8)


def _pool(c, pages, g):
    """A pool of pages, [pages, page, kv] or [pages, h_kv, page, kv] with a K/V head for several heads; one of 8 bits with its scales, else (pool, None)."""
    heads, page, kv, dtype = max(1, c["h_kv"]), c["page"], c["kv"], c["dtype"]
    one = c["h_kv"] == 0
    x = torch.randn((pages, heads, page, kv), generator=g, device=DEV)
    if dtype not in LARGEST:
        x = x.to(DTYPES[dtype])
        return (x[:, 0] if one else x).contiguous(), None
    # blocks of unlike sizes, as layers and positions give them
    x = x.view(pages, heads, page // c["block"], c["block"], kv) * torch.exp(0.5 * torch.randn((pages, heads, page // c["block"], 1, 1), generator=g, device=DEV))
    s = _scale_of(x.abs().amax((3, 4)), dtype)
    q = _to_8_bits(x / s[..., None, None], dtype).view(pages, heads, page, kv)
    return (q[:, 0].contiguous(), s[:, 0].contiguous()) if one else (q.contiguous(), s.contiguous())


def _table(b, pages_each, first, g):
    """Pages first .. first + b * pages_each - 1 in no order, pages_each to a sequence."""
    return (first + torch.randperm(b * pages_each, generator=g, device=DEV)).to(torch.int32).view(b, pages_each).contiguous()


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case=c)
    b = c["b"]
    if c["kind"] == "adjust":
        n, vocab, length = c["n"], c["vocab"], c["history"]
        s["logits"] = 3.0 * torch.randn((b, n + 1, vocab), generator=g, device=DEV)
        # texts come back to some tokens again and again
        s["history"] = (vocab * torch.rand((b, length), generator=g, device=DEV) ** 4).to(torch.int32).clamp(max=vocab - 1)
        lens = [length] * b if not c["ragged"] or b == 1 else [length * i // (b - 1) for i in range(b)]
        s["lens"] = _deal(lens, g)
        s["prompts"] = torch.div(s["lens"], 2, rounding_mode="floor")
        s["drafts"] = (vocab * torch.rand((b, n), generator=g, device=DEV) ** 4).to(torch.int32).clamp(max=vocab - 1) if n else None
        s["repetition"] = 1.0 + torch.rand((b,), generator=g, device=DEV)
        s["frequency"], s["presence"] = (torch.rand((b,), generator=g, device=DEV) for _ in range(2))
        s["bias_tokens"] = s["biases"] = s["allowed"] = None
        if c["biases"]:
            s["bias_tokens"] = torch.randint(0, vocab, (b, c["biases"]), generator=g, device=DEV, dtype=torch.int32)
            s["biases"] = 4.0 * torch.randn((b, c["biases"]), generator=g, device=DEV)
        if c["masked"]:
            s["allowed"] = torch.randint(-(2 ** 31), 2 ** 31, (b, n + 1, (vocab + 31) // 32), generator=g, device=DEV, dtype=torch.int64).to(torch.int32)
        s["out"] = torch.empty_like(s["logits"])
        return s
    kv, page, heads = c["kv"], c["page"], max(1, c["h_kv"])
    per_head = () if c["h_kv"] == 0 else (heads,)
    if c["kind"] == "append":
        pages_each = -(-(c["m"] + c["n"]) // page) + 1
        (s["K"], s["K_scales"]), (s["V"], s["V_scales"]) = (_pool(c, b * pages_each, g) for _ in range(2))
        s["table"] = _table(b, pages_each, 0, g)
        s["lens"] = torch.randint(0, c["m"] + 1, (b,), generator=g, device=DEV, dtype=torch.int32)
        s["lens_out"] = torch.zeros_like(s["lens"])
        s["counts"] = _deal(_counts(c), g) if c["ragged"] else None
        # now and then a row that stands out
        size = torch.exp(0.5 * torch.randn((b, c["n"], *per_head, 1), generator=g, device=DEV))
        s["k_new"], s["v_new"] = (torch.randn((b, c["n"], *per_head, kv), generator=g, device=DEV) * size for _ in range(2))
        return s
    pages_each = -(-c["m"] // page) + 2
    if c["kind"] == "attend":
        s["lens"] = _deal(_lengths(c), g)
        s["table"] = _table(b, pages_each, 0, g)
        (s["K"], s["K_scales"]), (s["V"], s["V_scales"]) = (_pool(c, b * pages_each, g) for _ in range(2))
        # logits of a few units: some positions stand out, as in a trained model
        s["q"] = torch.randn((b, c["n"], c["h"], kv), generator=g, device=DEV)
        s["scale"] = 2.0 / math.sqrt(kv)
        return s
    used_each = -(-c["m"] // page)
    if c["kind"] == "fork":
        n, children = c["n"], c["children"]
        each, own_pages = -(-(c["m"] + n) // page), b * used_each
        pages = own_pages + c["spare"]
        (s["K"], s["K_scales"]), (s["V"], s["V_scales"]) = (_pool(c, pages, g) for _ in range(2))
        s["lens"] = _deal(_lengths(c), g)
        place = torch.randperm(pages, generator=g, device=DEV)[:own_pages].to(torch.int32).view(b, used_each)
        x = torch.arange(each, device=DEV)
        s["table"] = torch.full((b, each), -1, dtype=torch.int32, device=DEV)
        s["table"][:, :used_each] = place
        held = x < ((s["lens"] + page - 1) // page)[:, None]
        s["table"].masked_fill_(~held, -1)
        s["parents"] = torch.arange(b, device=DEV, dtype=torch.int32).repeat_interleave(children).contiguous()
        # the continuations of the turn before: they share their prompt's whole pages
        s["child"] = s["table"][s["parents"].long()].masked_fill(x >= (s["lens"] // page)[s["parents"].long()][:, None], -1).contiguous()
        s["refs"] = torch.zeros((pages,), dtype=torch.int32, device=DEV)
        for t in (s["table"], s["child"]):
            s["refs"].scatter_add_(0, t.clamp(min=0).view(-1).long(), (t >= 0).view(-1).to(torch.int32))
        s["child_lens"] = torch.zeros((b * children,), dtype=torch.int32, device=DEV)
        s["none"] = torch.zeros((b * children,), dtype=torch.int32, device=DEV)
        s["granted"] = torch.zeros((b * children,), dtype=torch.int32, device=DEV)
        s["moves"] = torch.zeros((b * children, 2), dtype=torch.int32, device=DEV)
        return s
    pages = c["pages"]
    (s["K"], s["K_scales"]), (s["V"], s["V_scales"]) = (_pool(c, pages, g) for _ in range(2))
    lens = _deal(_lengths(c), g)
    s["table"] = torch.randperm(pages, generator=g, device=DEV)[:b * used_each].to(torch.int32).view(b, used_each)
    s["table"] = s["table"].masked_fill(torch.arange(used_each, device=DEV) >= ((lens + page - 1) // page)[:, None], -1).contiguous()
    s["refs"] = torch.zeros((pages,), dtype=torch.int32, device=DEV)
    s["refs"].scatter_add_(0, s["table"].clamp(min=0).view(-1).long(), (s["table"] >= 0).view(-1).to(torch.int32))
    s["table_out"], s["refs_out"] = torch.zeros_like(s["table"]), torch.zeros_like(s["refs"])
    s["moves"] = torch.zeros((max(1, pages // 2), 2), dtype=torch.int32, device=DEV)
    s["used"] = torch.zeros((1,), dtype=torch.int32, device=DEV)
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _whole(t, c):
    """A pool as [pages, heads, page, width] (scales: [pages, heads, blocks]), 8-bit floats as bytes."""
    t = t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
    return t.unsqueeze(1) if c["h_kv"] == 0 else t


def _plain_append(s):
    c, lens = s["case"], s["lens"].long()
    b, n, block, page, kv, dtype, heads = c["b"], c["n"], c["block"], c["page"], c["kv"], c["dtype"], max(1, c["h_kv"])
    new = torch.full_like(lens, n) if s["counts"] is None else s["counts"].long()
    blocks = (n + block - 1) // block + 1
    # positions from the beginning of the block that the first new row is in
    local = torch.arange(blocks * block, device=DEV)
    pos = (lens // block * block)[:, None] + local                                          # [b, local]
    fresh = (pos >= lens[:, None]) & (pos < (lens + new)[:, None])
    older = pos < lens[:, None]
    touched = fresh.view(b, blocks, block).any(2)
    entry = s["table"].gather(1, (pos // page).clamp(max=s["table"].shape[1] - 1)).long()
    which = (pos - lens[:, None]).clamp(0, n - 1)
    write = touched.repeat_interleave(block, 1) & (fresh | older)
    for name, rows in (("K", s["k_new"]), ("V", s["v_new"])):
        pool, scales = _whole(s[name], c), _whole(s[name + "_scales"], c)
        x = rows.view(b, n, heads * kv).gather(1, which[:, :, None].expand(b, -1, heads * kv)).view(b, blocks, block, heads, kv)
        x = x.masked_fill(~fresh.view(b, blocks, block, 1, 1), 0)
        wanted = _scale_of(x.abs().amax((2, 4)), dtype)                                      # [b, blocks, heads]
        at_block = entry.view(b, blocks, block)[:, :, 0], (pos % page // block).view(b, blocks, block)[:, :, 0]
        had = scales[at_block[0], :, at_block[1]]
        begun = older.view(b, blocks, block)[:, :, :1]
        scale = torch.where(begun, torch.maximum(had, wanted), wanted)
        held = pool[entry, :, pos % page].view(b, blocks, block, heads, kv)
        held = (held.view(torch.float8_e4m3fn) if dtype == "e4m3" else held).float() * (had / scale)[:, :, None, :, None]
        x = torch.where(older.view(b, blocks, block, 1, 1), held, x / scale[:, :, None, :, None])
        x = _to_8_bits(x, dtype).view(b, blocks * block, heads, kv)
        x = x.view(torch.uint8) if dtype == "e4m3" else x
        pool[entry[write], :, (pos % page)[write]] = x[write]
        scales[at_block[0][touched], :, at_block[1][touched]] = scale[touched]
    s["lens_out"].copy_(s["lens"] + new.to(torch.int32))
    return s["K"], s["K_scales"], s["V"], s["V_scales"], s["lens_out"]


def _rows_of(s, name, c):
    """[b, heads, positions, width] in float32 of what the table names."""
    pool, scales = _whole(s[name], c), _whole(s[name + "_scales"], c)
    at = s["table"].long()
    x = pool[at]
    x = (x.view(torch.float8_e4m3fn) if c["dtype"] == "e4m3" else x).float()                # [b, pages, heads, page, width]
    x = x.view(*x.shape[:3], -1, c["block"], x.shape[-1]) * scales[at][..., None, None]
    return x.permute(0, 2, 1, 3, 4, 5).reshape(c["b"], max(1, c["h_kv"]), -1, c["kv"])


def _plain_attend(s):
    c, heads = s["case"], max(1, s["case"]["h_kv"])
    b, n, h = c["b"], c["n"], c["h"]
    K, V = (_rows_of(s, x, c) for x in "KV")
    q = s["q"].view(b, n, heads, h // heads, -1).transpose(1, 2).reshape(b, heads, n * (h // heads), -1)
    logits = torch.matmul(q, K.transpose(2, 3).contiguous()) * s["scale"]                    # [b,heads,rows,positions]
    lens, pos = s["lens"].view(b, 1, 1, 1), torch.arange(K.shape[2], device=DEV)
    query = torch.arange(n, device=DEV).repeat_interleave(h // heads).view(1, 1, -1, 1)
    logits = logits.masked_fill(pos >= lens - (n - 1 - query), -math.inf)
    w = torch.exp(logits - logits.amax(-1, keepdim=True))
    w = w / w.sum(-1, keepdim=True)
    o = torch.matmul(w, V.masked_fill((pos >= lens.view(b, 1, 1)).unsqueeze(-1), 0))
    return o.view(b, heads, n, h // heads, -1).transpose(1, 2).reshape(b, n, h, -1)


def _pools(s):
    return [s[x] for x in ("K", "V", "K_scales", "V_scales") if s[x] is not None]


def _plain_copy(s):
    moves = s["moves"].long()
    moves = moves[moves[:, 0] >= 0]
    for t in _pools(s):
        t = t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
        t[moves[:, 1]] = t[moves[:, 0]]


def _named(refs, entries, by):
    refs.scatter_add_(0, entries.clamp(min=0).view(-1).long(), torch.where(entries >= 0, by, 0).to(torch.int32).view(-1))


def _plain_fork(s):
    c, refs, page, parents = s["case"], s["refs"], s["case"]["page"], s["parents"].long()
    # the last turn's continuations end
    _named(refs, s["child"], -1)
    # new ones share their prompt's pages
    lens = s["lens"][parents].long()
    x = torch.arange(s["child"].shape[1], device=DEV)
    table = s["table"][parents].masked_fill(x >= ((lens + page - 1) // page)[:, None], -1).long()
    _named(refs, table, 1)
    # pages for the next n tokens: in place of those that are not there, and of the begun page where others share it (the last of those who are about to write
    # to it keeps it where nobody else has it)
    first, last = (lens // page)[:, None], ((lens + c["n"] + page - 1) // page)[:, None]
    within = (x >= first) & (x < last)
    begun = within & (x == first) & (lens % page != 0)[:, None]
    count = refs[table.clamp(min=0)]
    shared = (table >= 0) & (count > 1)
    me = torch.arange(len(lens), device=DEV)[:, None].expand_as(table)
    writers, latest = torch.zeros_like(refs), torch.full((len(refs),), -1, dtype=torch.long, device=DEV)
    _named(writers, torch.where(begun, table, -1), 1)
    latest.scatter_reduce_(0, table.clamp(min=0).view(-1), torch.where(begun & (table >= 0), me, -1).reshape(-1), "amax")
    keeps = begun & shared & (writers[table.clamp(min=0)] == count) & (latest[table.clamp(min=0)] == me)
    needs = torch.where(begun, shared & ~keeps, within & ((table < 0) | shared))
    order = needs.view(-1).long().cumsum(0).view_as(table)
    free = torch.where(refs <= 0, torch.arange(len(refs), device=DEV), len(refs)).sort().values
    there = (refs <= 0).sum()
    granted = (order[:, -1] <= there) | ~(needs | keeps).any(1)
    takes = needs & granted[:, None]
    page_of = free[(order - 1).clamp(0, len(refs) - 1)]
    _named(refs, torch.where(takes, table, -1), -1)
    _named(refs, torch.where(takes, page_of, -1), 1)
    copies = (takes & begun).any(1)
    at = first.clamp(max=table.shape[1] - 1)
    s["moves"].copy_(torch.where(copies[:, None], torch.cat([table.gather(1, at), page_of.gather(1, at)], 1), -1))
    s["child"].copy_(torch.where(takes, page_of, table))
    s["child_lens"].copy_(lens)
    s["granted"].copy_(torch.where(granted, c["n"], 0))
    _plain_copy(s)
    return (s["child"], s["child_lens"], refs, s["granted"], s["moves"], *_pools(s))


def _plain_compact(s):
    refs, table = s["refs"], s["table"].long()
    pages = len(refs)
    used, at = refs > 0, torch.arange(pages, device=DEV)
    total = used.sum()
    hole, tail = ~used & (at < total), used & (at >= total)
    holes, tails = (torch.where(t, at, pages).sort().values for t in (hole, tail))
    to = torch.where(tail, holes[(tail.long().cumsum(0) - 1).clamp(min=0)], at).masked_fill(~used, -1)
    pairs = torch.stack([tails, holes], 1)[:len(s["moves"])]
    s["moves"].copy_(torch.where(torch.arange(len(s["moves"]), device=DEV)[:, None] < tail.sum(), pairs, -1) if pages > 1 else torch.full_like(s["moves"], -1))
    s["refs_out"].zero_().scatter_add_(0, to.clamp(min=0), torch.where(used, refs, 0))
    s["table_out"].copy_(torch.where(table >= 0, to[table.clamp(min=0)], -1))
    s["used"].copy_(total.view(1))
    _plain_copy(s)
    return (s["table_out"], s["refs_out"], s["moves"], s["used"], *_pools(s))


def _plain_adjust(s):
    c = s["case"]
    b, n, vocab = c["b"], c["n"], c["vocab"]
    at, token = torch.arange(c["history"], device=DEV), s["history"].long()
    there = at < s["lens"][:, None]
    count = torch.zeros((b, vocab), dtype=torch.int32, device=DEV)
    seen = count.clone().scatter_add_(1, token, there.to(torch.int32))
    count.scatter_add_(1, token, (there & (at >= s["prompts"][:, None])).to(torch.int32))
    count, seen = count[:, None], seen[:, None]
    if n:
        drafted = torch.zeros((b, n + 1, vocab), dtype=torch.int32, device=DEV)
        drafted[:, 1:].scatter_(2, s["drafts"].long()[:, :, None], 1)
        drafted = drafted.cumsum(1, dtype=torch.int32)                                       # row j: of the drafts before it
        count, seen = count + drafted, seen + drafted
    repetition, frequency, presence = (s[x].view(b, 1, 1) for x in ("repetition", "frequency", "presence"))
    x = s["logits"]
    x = torch.where(seen > 0, torch.where(x > 0, x / repetition, x * repetition), x)
    x = x - (frequency * count + torch.where(count > 0, presence, 0.0))
    if s["biases"] is not None:
        m = s["biases"].shape[1]
        latest = torch.full((b, vocab), -1, dtype=torch.long, device=DEV)                    # (the last of a token's biases)
        latest.scatter_reduce_(1, s["bias_tokens"].long(), torch.arange(m, device=DEV).expand(b, m), "amax")
        x = x + torch.where(latest >= 0, s["biases"].gather(1, latest.clamp(min=0)), 0.0)[:, None]
    if s["allowed"] is not None:
        t = torch.arange(vocab, device=DEV)
        x = x.masked_fill((s["allowed"][:, :, t // 32] >> (t % 32).to(torch.int32)) & 1 == 0, -math.inf)
    return x


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        import paper_1911_02150_amd as mqa
        if kind == "append":
            mqa.mqa_paged_scaled_append_kv_rows(s["K"], s["K_scales"], s["V"], s["V_scales"], s["table"], s["k_new"], s["v_new"], s["lens"], s["lens_out"],
                                                counts=s["counts"])
            return s["K"], s["K_scales"], s["V"], s["V_scales"], s["lens_out"]
        if kind == "attend":
            return mqa.mqa_paged_scaled_decode_step(s["q"], s["K"], s["K_scales"], s["V"], s["V_scales"], s["table"], s["lens"], scale=s["scale"])
        if kind == "fork":
            mqa.mqa_paged_free_pages(s["child"], s["none"], s["refs"], s["case"]["page"])
            mqa.mqa_paged_fork_pages(s["table"], s["lens"], s["parents"], s["child"], s["child_lens"], s["refs"], s["case"]["page"])
            mqa.mqa_paged_reserve_pages(s["child"], s["child_lens"], s["refs"], s["case"]["page"], s["case"]["n"], granted=s["granted"], moves=s["moves"])
            mqa.mqa_paged_copy_pages(_pools(s), s["moves"])
            return (s["child"], s["child_lens"], s["refs"], s["granted"], s["moves"], *_pools(s))
        if kind == "compact":
            mqa.mqa_paged_compact_pages(s["table"], s["refs"], s["table_out"], s["refs_out"], s["moves"], s["used"])
            mqa.mqa_paged_copy_pages(_pools(s), s["moves"])
            return (s["table_out"], s["refs_out"], s["moves"], s["used"], *_pools(s))
        return mqa.mqa_stack_adjust_logits(s["logits"], s["history"], s["lens"], drafts=s["drafts"], prompts=s["prompts"], repetition=s["repetition"],
                                           frequency=s["frequency"], presence=s["presence"], bias_tokens=s["bias_tokens"], biases=s["biases"],
                                           allowed=s["allowed"], out=s["out"])
    return dict(append=_plain_append, attend=_plain_attend, fork=_plain_fork, compact=_plain_compact, adjust=_plain_adjust)[kind](s)


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c, b = case, case["b"]
    if c["kind"] == "adjust":
        n, vocab = c["n"], c["vocab"]
        read = b * c["history"] if not c["ragged"] or b == 1 else sum(c["history"] * i // (b - 1) for i in range(b))
        rows = b * (n + 1)
        return dict(bytes=8 * rows * vocab + (4 * rows * ((vocab + 31) // 32) if c["masked"] else 0) + 4 * read + 8 * b * c["biases"] + 4 * b * (n + 5),
                    flops=5 * rows * vocab)
    kv, heads, page, block = c["kv"], max(1, c["h_kv"]), c["page"], c["block"]
    e = BYTES[c["dtype"]]
    whole_page = heads * page * 2 * kv * e + (8 * heads * (page // block) if c["dtype"] in LARGEST else 0)      # K, V and their scales
    if c["kind"] == "append":
        rows = sum(_counts(c)) * heads
        return dict(bytes=rows * 2 * kv * 5 + 8 * sum(-(-x // block) for x in _counts(c)) * heads + 12 * b, flops=rows * 4 * kv)
    lens = _lengths(c)
    named = sum(-(-x // page) for x in lens)                                                 # entries of the tables
    if c["kind"] == "attend":
        rows = c["n"] * c["h"]
        scales = heads * sum(-(-x // block) for x in lens) * 8
        return dict(bytes=heads * sum(lens) * 2 * kv + scales + 2 * b * rows * kv * 4 + 4 * named, flops=4 * rows * kv * sum(lens))
    if c["kind"] == "fork":
        each, children = -(-(c["m"] + c["n"]) // page), c["children"]
        pages = b * -(-c["m"] // page) + c["spare"]
        copied, left = 0, c["spare"]
        for x in lens:
            for _ in range(children):
                needs = (-(-(x + c["n"]) // page) - (-(-x // page))) + (x % page != 0)
                if needs <= left:
                    left -= needs
                    copied += x % page != 0
        # the prompts' tables read, the continuations' read (the last turn's) and written, the counts of the pages read and written
        return dict(bytes=copied * 2 * whole_page + 4 * named + 8 * b * children * each + 8 * pages + 16 * b * children, flops=8 * b * children * each)
    in_use = named
    moves = in_use * max(0, c["pages"] - in_use) // c["pages"]                                # (of pages in use in no order)
    return dict(bytes=moves * 2 * whole_page + 8 * c["pages"] + 8 * (c["pages"] // 2) + 8 * b * -(-c["m"] // page), flops=4 * c["pages"])


# ------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    return dict(append=_exact_append, attend=_exact_attend, fork=_exact_fork, compact=_exact_compact, adjust=_exact_adjust)[c["kind"]](c, s)


def _values(t):
    """A pool's or scales' numbers in float64 on the host."""
    return t.float().cpu().double().numpy()


def _nearest(x, dtype):
    """The type's number next to x, the even one of two."""
    if dtype == "int8":
        return np.clip(np.rint(x), -127, 127)
    a = np.minimum(np.abs(x), 448.0)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(a, 2.0 ** -20))), -6.0) - 3.0)      # three bits behind the first; below 2^-6 as there
    return np.copysign(np.minimum(np.rint(a / step) * step, 448.0), x)


def _exact_append(c, s):
    heads, page, block, dtype = max(1, c["h_kv"]), c["page"], c["block"], c["dtype"]
    table, lens = s["table"].cpu().numpy(), s["lens"].cpu().numpy()
    counts = [c["n"]] * c["b"] if s["counts"] is None else s["counts"].cpu().numpy()
    out = []
    for name, new in (("K", s["k_new"]), ("V", s["v_new"])):
        pool, scales = _values(s[name]), _values(s[name + "_scales"])
        rows, factor = pool.reshape(-1, heads, page, c["kv"]), scales.reshape(-1, heads, page // block)
        new = _values(new).reshape(c["b"], c["n"], heads, c["kv"])
        for i in range(c["b"]):
            begin, end = int(lens[i]), int(lens[i]) + int(counts[i])
            while begin < end:
                first = begin // block * block
                upto = min(end, first + block)
                at, row, piece = table[i, first // page], first % page, first % page // block
                x = new[i, begin - lens[i]:upto - lens[i]]                                    # [rows, heads, kv]
                with np.errstate(divide="ignore"):
                    wanted = 2.0 ** np.maximum(np.ceil(np.log2(np.abs(x).max((0, 2)) / LARGEST[dtype])), -126)
                had, older = factor[at, :, piece].copy(), begin - first
                scale = np.maximum(had, wanted) if older else wanted
                factor[at, :, piece] = scale
                rows[at, :, row:row + older] = _nearest(rows[at, :, row:row + older] * (had / scale)[:, None, None], dtype)
                rows[at, :, row + older:row + upto - first] = _nearest(x.transpose(1, 0, 2) / scale[:, None, None], dtype)
                begin = upto
        out += [torch.from_numpy(pool) if dtype == "e4m3" else None, torch.from_numpy(scales)]
    return (*out, None)


def _exact_attend(c, s):
    heads, n, page, group = max(1, c["h_kv"]), c["n"], c["page"], c["h"] // max(1, c["h_kv"])
    out = torch.zeros((c["b"], n, c["h"], c["kv"]), dtype=torch.float64, device=DEV)
    for i, length in enumerate(s["lens"].tolist()):
        used = s["table"][i, :-(-length // page)].long()
        rows = []
        for name in "KV":
            x = s[name].view(torch.uint8)[used].view(s[name].dtype).double()
            f = s[name + "_scales"][used].double().view(len(used), heads, -1, 1).expand(-1, -1, -1, c["block"]).reshape(len(used), heads, page, 1)
            rows.append((x.view(len(used), heads, page, c["kv"]) * f).transpose(0, 1).reshape(heads, -1, c["kv"])[:, :length])
        for j in range(n):
            seen = length - (n - 1 - j)
            if seen <= 0:
                continue
            z = (s["q"][i, j].double().view(heads, group, c["kv"]) @ rows[0][:, :seen].transpose(1, 2)) * s["scale"]
            out[i, j] = (torch.softmax(z, dim=-1) @ rows[1][:, :seen]).reshape(c["h"], c["kv"])
    return out


def _moved(s, moves):
    """The pools' numbers after pages have been copied (whole numbers: none)."""
    out = []
    for t in _pools(s):
        if t.dtype == torch.int8:
            out.append(None)
            continue
        x = t.double()
        for a, z in moves:
            x[z] = x[a].clone()
        out.append(x)
    return out


def _exact_fork(c, s):
    page, refs = c["page"], s["refs"].tolist()
    for row in s["child"].tolist():
        for x in row:
            if x >= 0:
                refs[x] -= 1
    prompts, lens, tables = s["table"].tolist(), s["lens"].tolist(), []
    for parent in s["parents"].tolist():
        used = -(-lens[parent] // page)
        tables.append((parent, prompts[parent][:used]))
        for x in prompts[parent][:used]:
            refs[x] += 1
    free = [x for x, count in enumerate(refs) if count <= 0]
    # the prompt itself has its begun page too, so that every continuation gets a copy; once the pages do not suffice for one, none that wants any gets them
    moves, at = [], 0
    for p, t in tables:
        begun, wants = lens[p] % page != 0, -(-(lens[p] + c["n"]) // page) - len(t)
        if begun and at + wants < len(free):
            moves.append((t[-1], free[at]))
        at += wants + begun
    return (None, None, None, None, None, *_moved(s, moves))


def _exact_compact(c, s):
    refs = s["refs"].cpu().numpy()
    used = int((refs > 0).sum())
    holes, tails = [x for x in range(used) if refs[x] <= 0], [x for x in range(used, len(refs)) if refs[x] > 0]
    if len(tails) > 4096:
        moves = torch.tensor([tails, holes], device=DEV)
        return (None, None, None, None, *(None if t.dtype == torch.int8 else t.double().index_copy_(0, moves[1], t.double()[moves[0]]) for t in _pools(s)))
    return (None, None, None, None, *_moved(s, list(zip(tails, holes))))


def _exact_adjust(c, s):
    x = s["logits"].double().cpu().numpy()
    history, lens, prompts = (s[name].cpu().numpy() for name in ("history", "lens", "prompts"))
    factor, often, once = (s[name].double().cpu().numpy() for name in ("repetition", "frequency", "presence"))
    for i in range(c["b"]):
        seen = np.bincount(history[i, :lens[i]], minlength=c["vocab"])
        count = np.bincount(history[i, prompts[i]:lens[i]], minlength=c["vocab"])
        bias = np.zeros(c["vocab"])
        if s["biases"] is not None:
            for t, y in zip(s["bias_tokens"][i].tolist(), s["biases"][i].tolist()):
                bias[t] = y
        for j in range(c["n"] + 1):
            if j:
                t = int(s["drafts"][i, j - 1])
                seen[t] += 1
                count[t] += 1
            row = x[i, j]
            again = seen > 0
            row[again] = np.where(row[again] > 0, row[again] / factor[i], row[again] * factor[i])
            row -= often[i] * count + once[i] * (count > 0)
            row += bias
            if s["allowed"] is not None:
                bits = np.unpackbits(s["allowed"][i, j].cpu().numpy().view(np.uint8), bitorder="little")[:c["vocab"]]
                row[bits == 0] = -np.inf
    return torch.from_numpy(x)
