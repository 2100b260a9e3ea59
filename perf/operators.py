"""Operators of a serving loop over a paged key/value cache: what each computes, at sizes from one user's token to a full batch.

Kinds:

  append   n new K/V rows per sequence rounded into the pages that the sequence's table names
  decode   attention of the newest n tokens of every sequence (n = 1, or drafted tokens with the causal mask) over its pages
  scored   the same, which also adds up for every position the attention weight that it has received
  evict    the positions that have received most, and the latest ones, copied to other pages; the rest is left behind
  verify   drafted tokens accepted or refused against the target's probabilities from given random numbers, and the token
           that follows them

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
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a decoding step's new rows: one per sequence, 128 sequences
        dict(name="append_tokens_b128", kind="append", b=128, n=1, ragged=False, h_kv=0, kv=128, m=255, page=16, dtype="bf16"),
        # a padded batch of prompts taken into the cache
        dict(name="append_prompts_b64", kind="append", b=64, n=1024, ragged=True, h_kv=0, kv=128, m=0, page=16, dtype="bf16"),
        # one user, a short float32 cache: latency
        dict(name="decode_b1_f32", kind="decode", b=1, n=1, h=8, h_kv=0, kv=128, m=128, page=16, dtype="f32", ragged=False),
        # drafted tokens under verification: five queries per sequence, mixed lengths
        dict(name="decode_drafts_b32", kind="decode", b=32, n=5, h=8, h_kv=0, kv=128, m=2048, page=16, dtype="bf16", ragged=True),
        # long contexts, all full, large pages
        dict(name="decode_long", kind="decode", b=64, n=1, h=32, h_kv=0, kv=128, m=8192, page=64, dtype="bf16", ragged=False),
        # a large serving batch of mixed lengths with many heads
        dict(name="decode_ragged_b512", kind="decode", b=512, n=1, h=64, h_kv=0, kv=128, m=4096, page=16, dtype="bf16", ragged=True),
        # a few users, whose caches are kept to a budget by what is looked at; a K/V head for each of 8 heads
        dict(name="scored_b4_multihead", kind="scored", b=4, n=1, h=8, h_kv=8, kv=64, m=700, page=16, dtype="f32", ragged=True),
        # the same for a batch of long contexts
        dict(name="scored_long", kind="scored", b=32, n=1, h=32, h_kv=0, kv=128, m=8192, page=64, dtype="bf16", ragged=False),
        # one user's cache brought to its budget
        dict(name="evict_b1", kind="evict", b=1, h_kv=8, kv=64, m=701, budget=512, recent=64, page=16, dtype="f32", ragged=False),
        # a batch of long contexts brought to a quarter
        dict(name="evict_b32", kind="evict", b=32, h_kv=0, kv=128, m=8192, budget=2048, recent=256, page=16, dtype="bf16", ragged=True),
        # one user's drafts, and a batch's
        dict(name="verify_b1", kind="verify", b=1, n=4, vocab=32768, temperature=0.8, draft="logits", ragged=False),
        dict(name="verify_b64", kind="verify", b=64, n=4, vocab=32768, temperature=1.0, draft="logits", ragged=True),
    ]


def _log(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append", "decode", "decode", "scored", "evict", "verify"])
    page = rng.choice([16, 16, 32, 64, 8, rng.randint(1, 100)])
    kv = rng.choice([128, 128, 128, 64, 8 * rng.randint(1, 32)])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    h_kv = rng.choice([0, 0, 0, rng.randint(1, 8)])
    heads = max(1, h_kv)
    if kind == "append":
        n = rng.choice([1, rng.randint(2, 8), _log(rng, 2, 1024)])
        b = _log(rng, 1, max(1, min(512, 65536 // (n * heads))))
        return dict(kind=kind, b=b, n=n, ragged=rng.random() < 0.5, h_kv=h_kv, kv=kv, m=rng.randint(0, 512), page=page, dtype=dtype)
    if kind in ("decode", "scored"):
        m = _log(rng, 1, 8192)
        n = min(m, rng.choice([1, 1, 1, rng.randint(2, 8)]))
        h = heads * rng.randint(1, max(1, 64 // heads // n))
        b = _log(rng, 1, max(1, min(512, (1 << 18) // (m * heads), (1 << 25) // (m * h * n))))
        return dict(kind=kind, b=b, n=n, h=h, h_kv=h_kv, kv=kv, m=m, page=page, dtype=dtype, ragged=rng.random() < 0.5)
    if kind == "evict":
        m = _log(rng, 2, 8192)
        budget = rng.randint(1, m)
        b = _log(rng, 1, max(1, min(256, (1 << 17) // (m * heads))))
        return dict(kind=kind, b=b, h_kv=h_kv, kv=kv, m=m, budget=budget, recent=rng.randint(0, budget), page=page, dtype=dtype,
                    ragged=rng.random() < 0.5)
    vocab, n = _log(rng, 100, 65536), rng.randint(1, 8)
    return dict(kind="verify", b=_log(rng, 1, max(1, min(256, (1 << 24) // (vocab * (2 * n + 1))))), n=n, vocab=vocab,
                temperature=rng.choice([1.0, 1.0, 0.6, 1.5, 0.0]), draft=rng.choice(["logits", "logits", "none"]), ragged=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------ inputs
def _lengths(c):
    """The lengths of a case, shortest to longest (`prepare` deals them out by its seed)."""
    lo, hi, b = min(c["m"], max(1, c.get("n", 1))), c["m"], c["b"]
    return [hi] * b if not c["ragged"] or b == 1 else [lo + (hi - lo) * i // (b - 1) for i in range(b)]


def _counts(c):
    n, b = c["n"], c["b"]
    return [n] * b if not c["ragged"] or b == 1 else [max(1, n * i // (b - 1)) for i in range(b)]


def _deal(values, g):
    t = torch.tensor(values, dtype=torch.int32, device=DEV)
    return t[torch.randperm(len(values), generator=g, device=DEV)].contiguous()


def _pool(c, pages, g):
    """K and V pages: [pages, page, kv], or [pages, h_kv, page, kv] with a K/V head for several heads."""
    shape = (pages, c["page"], c["kv"]) if c["h_kv"] == 0 else (pages, c["h_kv"], c["page"], c["kv"])
    return [torch.randn(shape, generator=g, device=DEV).to(DTYPES[c["dtype"]]) for _ in range(2)]


def _table(b, pages_each, first, g):
    """Pages first .. first + b * pages_each - 1 in no order, pages_each to a sequence."""
    return (first + torch.randperm(b * pages_each, generator=g, device=DEV)).to(torch.int32).view(b, pages_each).contiguous()


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case=c)
    if c["kind"] == "verify":
        b, n, vocab = c["b"], c["n"], c["vocab"]
        s["logits"] = 3.0 * torch.randn((b, n + 1, vocab), generator=g, device=DEV)
        s["draft_logits"] = s["logits"][:, :n] + 0.7 * torch.randn((b, n, vocab), generator=g, device=DEV)
        t = c["temperature"] or 0.25
        # tokens as the draft model draws them: the largest of logits and Gumbel noise
        noise = -torch.log(-torch.log(torch.rand((b, n, vocab), generator=g, device=DEV).clamp(1e-6, 1 - 1e-6)))
        s["drafts"] = (s["draft_logits"] / t + noise).argmax(-1).to(torch.int32)
        s["counts"] = _deal(_counts(c), g) if c["ragged"] else None
        s["u"] = torch.rand((b, n + 1), generator=g, device=DEV)
        if c["draft"] == "none":
            s["draft_logits"] = None
        return s
    b, kv, page, heads = c["b"], c["kv"], c["page"], max(1, c["h_kv"])
    per_head = () if c["h_kv"] == 0 else (heads,)
    if c["kind"] == "append":
        pages_each = -(-(c["m"] + c["n"]) // page) + 1
        s["K"], s["V"] = _pool(c, b * pages_each, g)
        s["table"] = _table(b, pages_each, 0, g)
        s["lens"] = torch.randint(0, c["m"] + 1, (b,), generator=g, device=DEV, dtype=torch.int32)
        s["lens_out"] = torch.zeros_like(s["lens"])
        s["counts"] = _deal(_counts(c), g) if c["ragged"] else None
        s["k_new"], s["v_new"] = (torch.randn((b, c["n"], *per_head, kv), generator=g, device=DEV) for _ in range(2))
        return s
    pages_each = -(-c["m"] // page) + 2
    s["lens"] = _deal(_lengths(c), g)
    s["table"] = _table(b, pages_each, 0, g)
    positions = pages_each * page
    if c["kind"] == "evict":
        out_each = -(-c["budget"] // page)
        s["K"], s["V"] = _pool(c, b * (pages_each + out_each), g)
        s["table_out"] = _table(b, out_each, b * pages_each, g)
        s["lens_out"] = torch.zeros_like(s["lens"])
        # a few positions are looked at much, many hardly, some never
        w = torch.rand((b, *per_head, positions), generator=g, device=DEV)
        s["scores"] = torch.where(w < 0.1, torch.zeros_like(w), w ** 8)
        s["scores_out"] = torch.zeros((b, *per_head, out_each * page), device=DEV)
        s["kept"] = torch.zeros((b, *per_head, c["budget"]), dtype=torch.int32, device=DEV)
        return s
    s["K"], s["V"] = _pool(c, b * pages_each, g)
    # logits of a few units: some positions stand out, as in a trained model
    s["q"] = torch.randn((b, c["n"], c["h"], kv), generator=g, device=DEV)
    s["scale"] = 2.0 / math.sqrt(kv)
    if c["kind"] == "scored":
        s["scores"] = torch.rand((b, *per_head, positions), generator=g, device=DEV)
        s["scores_out"] = torch.zeros_like(s["scores"])
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _plain_append(s, heads):
    c, table, lens = s["case"], s["table"], s["lens"]
    b, n = c["b"], c["n"]
    K, V = (t.view(t.shape[0], heads, c["page"], -1) for t in (s["K"], s["V"]))
    i = torch.arange(n, device=DEV)
    new = torch.full_like(lens, n) if s["counts"] is None else s["counts"]
    pos = lens[:, None] + i                                                              # [b,n]
    valid = i < new[:, None]
    at = table.gather(1, (pos // c["page"]).clamp(max=table.shape[1] - 1).long())
    rows, cols = at[valid].long(), (pos % c["page"])[valid].long()
    K[rows, :, cols] = s["k_new"].view(b, n, heads, -1)[valid].to(K.dtype)
    V[rows, :, cols] = s["v_new"].view(b, n, heads, -1)[valid].to(V.dtype)
    s["lens_out"].copy_(lens + new)
    return s["K"], s["V"], s["lens_out"]


def _rows_of(pages, table, heads, page):
    """[b, heads, positions, width] in float32 of what a table names."""
    t = pages.view(pages.shape[0], heads, page, -1)[table.long()]
    return t.permute(0, 2, 1, 3, 4).reshape(table.shape[0], heads, -1, t.shape[-1]).float()


def _plain_decode(s, heads):
    c = s["case"]
    b, n, h = c["b"], c["n"], c["h"]
    K, V = (_rows_of(s[x], s["table"], heads, c["page"]) for x in "KV")
    q = s["q"].view(b, n, heads, h // heads, -1).transpose(1, 2).reshape(b, heads, n * (h // heads), -1)
    logits = torch.matmul(q, K.transpose(2, 3).contiguous()) * s["scale"]                                  # [b,heads,rows,positions]
    lens, pos = s["lens"].view(b, 1, 1, 1), torch.arange(K.shape[2], device=DEV)
    query = torch.arange(n, device=DEV).repeat_interleave(h // heads).view(1, 1, -1, 1)
    logits = logits.masked_fill(pos >= lens - (n - 1 - query), -math.inf)
    w = torch.exp(logits - logits.amax(-1, keepdim=True))
    w = w / w.sum(-1, keepdim=True)
    o = torch.matmul(w, V.masked_fill((pos >= lens.view(b, 1, 1)).unsqueeze(-1), 0))
    o = o.view(b, heads, n, h // heads, -1).transpose(1, 2).reshape(b, n, h, -1)
    if c["kind"] == "decode":
        return o
    before = s["scores"].view(b, heads, -1).masked_fill(pos >= lens.view(b, 1, 1) - n, 0)      # (the newest have received nothing yet)
    after = torch.where(pos < lens.view(b, 1, 1), before + w.sum(2), s["scores_out"].view(b, heads, -1))
    s["scores_out"].copy_(after.view_as(s["scores_out"]))
    return o, s["scores_out"]


def _plain_evict(s, heads):
    c = s["case"]
    b, budget, page = c["b"], c["budget"], c["page"]
    scores, lens = s["scores"].view(b, heads, -1), s["lens"].view(b, 1, 1)
    pos = torch.arange(scores.shape[2], device=DEV)
    key = scores.masked_fill(pos >= lens - c["recent"], math.inf).masked_fill(pos >= lens, -math.inf)
    best = key.sort(dim=2, descending=True, stable=True).indices[:, :, :budget]
    count = lens.clamp(max=budget)
    slot = torch.arange(budget, device=DEV)
    kept = best.masked_fill(slot >= count, scores.shape[2]).sort(dim=2).values
    there = slot < count                                                                   # [b,1,budget], the same for every head
    kept_or_0 = kept.masked_fill(~there, 0)
    K, V = (t.view(t.shape[0], heads, page, -1) for t in (s["K"], s["V"]))
    from_page = s["table"].gather(1, (kept_or_0 // page).view(b, -1)).view(b, heads, budget).long()
    to_page = s["table_out"][:, slot // page].view(b, 1, budget).expand(b, heads, budget).long()
    head = torch.arange(heads, device=DEV).view(1, heads, 1).expand(b, heads, budget)
    all_there = there.expand(b, heads, budget)
    source = from_page[all_there], head[all_there], (kept_or_0 % page)[all_there]
    target = to_page[all_there], head[all_there], (slot % page).expand(b, heads, budget)[all_there]
    K[target] = K[source]
    V[target] = V[source]
    s["kept"].copy_(torch.where(there, kept, -1).view_as(s["kept"]))
    out = s["scores_out"].view(b, heads, -1)
    out[:, :, :budget] = torch.where(there, scores.gather(2, kept_or_0), out[:, :, :budget])
    s["lens_out"].copy_(count.view(b))
    return s["K"], s["V"], s["lens_out"], s["scores_out"], s["kept"]


def _probabilities(logits, temperature):
    x = logits.double() / temperature
    x = torch.exp(x - x.amax(-1, keepdim=True))
    return x / x.sum(-1, keepdim=True)


def _plain_verify(s):
    c, drafts, u = s["case"], s["drafts"].long(), s["u"].double()
    b, n, vocab = c["b"], c["n"], c["vocab"]
    counts = torch.full((b,), n, dtype=torch.int32, device=DEV) if s["counts"] is None else s["counts"]
    if c["temperature"] == 0:
        best = s["logits"].argmax(-1)
        accept = best[:, :n] == drafts
    else:
        p = _probabilities(s["logits"], float(np.float32(c["temperature"])))
        if s["draft_logits"] is None:
            q = torch.zeros_like(p[:, :n]).scatter_(2, drafts[:, :, None], 1.0)
        else:
            q = _probabilities(s["draft_logits"], float(np.float32(c["temperature"])))
        accept = u[:, :n] * q.gather(2, drafts[:, :, None])[:, :, 0] < p[:, :n].gather(2, drafts[:, :, None])[:, :, 0]
    slot = torch.arange(n + 1, device=DEV)
    accept = accept & (slot[:n] < counts[:, None])
    accepted = accept.long().cumprod(1).sum(1)
    if c["temperature"] == 0:
        last = best.gather(1, accepted[:, None])
    else:
        at = accepted[:, None, None].expand(b, 1, vocab)
        rest = torch.cat([q, torch.zeros_like(p[:, :1])], 1).gather(1, at)[:, 0]
        rest = rest.masked_fill((accepted == counts)[:, None], 0)                           # (behind the last draft nothing is taken off)
        total = (p.gather(1, at)[:, 0] - rest).clamp(min=0).cumsum(1)
        last = (total <= u[:, n:] * total[:, -1:]).sum(1, keepdim=True)
    padded = torch.cat([drafts, torch.zeros_like(drafts[:, :1])], 1)
    tokens = torch.where(slot < accepted[:, None], padded, torch.where(slot == accepted[:, None], last, -1))
    return tokens.to(torch.int32), accepted.to(torch.int32)


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    s, kind = state, state["case"]["kind"]
    if own:
        import paper_1911_02150_amd as mqa
        if kind == "append":
            mqa.mqa_paged_append_kv_rows(s["K"], s["V"], s["table"], s["k_new"], s["v_new"], s["lens"], s["lens_out"], counts=s["counts"])
            return s["K"], s["V"], s["lens_out"]
        if kind == "decode":
            return mqa.mqa_paged_decode_step(s["q"], s["K"], s["V"], s["table"], s["lens"], scale=s["scale"])
        if kind == "scored":
            return mqa.mqa_paged_decode_step(s["q"], s["K"], s["V"], s["table"], s["lens"], scale=s["scale"], scores=s["scores"],
                                             scores_out=s["scores_out"]), s["scores_out"]
        if kind == "evict":
            mqa.mqa_paged_evict_kv(s["K"], s["V"], s["table"], s["lens"], s["scores"], s["table_out"], s["lens_out"], s["scores_out"],
                                   s["kept"], s["case"]["recent"])
            return s["K"], s["V"], s["lens_out"], s["scores_out"], s["kept"]
        return mqa.mqa_stack_verify_drafts(s["logits"], s["drafts"], s["u"], draft_logits=s["draft_logits"], counts=s["counts"],
                                           temperature=s["case"]["temperature"])
    heads = max(1, s["case"].get("h_kv", 0))
    if kind == "append":
        return _plain_append(s, heads)
    if kind in ("decode", "scored"):
        return _plain_decode(s, heads)
    if kind == "evict":
        return _plain_evict(s, heads)
    return _plain_verify(s)


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    if c["kind"] == "verify":
        b, n, vocab = c["b"], c["n"], c["vocab"]
        drafted = sum(_counts(c))
        rows = drafted + b + (drafted if c["draft"] == "logits" and c["temperature"] else 0)
        return dict(bytes=4 * rows * vocab + 4 * b * (3 * n + 4), flops=4 * rows * vocab)
    e = {"f32": 4, "bf16": 2}[c["dtype"]]
    b, kv, heads = c["b"], c["kv"], max(1, c["h_kv"])
    if c["kind"] == "append":
        rows = sum(_counts(c)) * heads
        return dict(bytes=rows * 2 * kv * (4 + e) + 12 * b, flops=rows * 2 * kv)
    lens = _lengths(c)
    named = sum(-(-x // c["page"]) for x in lens)                                          # entries of the tables
    if c["kind"] == "evict":
        kept = heads * sum(min(x, c["budget"]) for x in lens)
        return dict(bytes=kept * (4 * kv * e + 8) + 4 * heads * sum(lens) + 4 * named, flops=heads * sum(lens))
    rows = c["n"] * c["h"]
    out = dict(bytes=heads * sum(lens) * 2 * kv * e + 2 * b * rows * kv * 4 + 4 * named, flops=4 * rows * kv * sum(lens))
    if c["kind"] == "scored":
        out["bytes"] += 8 * heads * sum(lens)
        out["flops"] += rows * sum(lens)
    return out


# ------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "verify":
        return None                                                                       # (whole numbers alone)
    if c["kind"] == "append":
        return _exact_append(c, s)
    if c["kind"] == "evict":
        return _exact_evict(c, s)
    return _exact_decode(c, s)


def _exact_append(c, s):
    K, V = s["K"].double().cpu(), s["V"].double().cpu()
    table, lens, heads = s["table"].cpu().numpy(), s["lens"].cpu().numpy(), max(1, c["h_kv"])
    counts = [c["n"]] * c["b"] if s["counts"] is None else s["counts"].cpu().numpy()
    for pages, new in ((K, s["k_new"]), (V, s["v_new"])):
        held = pages.view(pages.shape[0], heads, c["page"], c["kv"])
        new = new.to(DTYPES[c["dtype"]]).double().cpu().view(c["b"], c["n"], heads, c["kv"])      # (the cache's own rounding is the definition's)
        for i in range(c["b"]):
            pos = np.arange(lens[i], lens[i] + counts[i])
            held[torch.from_numpy(table[i, pos // c["page"]].astype(np.int64)), :, torch.from_numpy(pos % c["page"]).long()] = new[i, :counts[i]]
    return K, V, None


def _sequence(s, x, i, length, c):
    """The first `length` rows of sequence i in float64: [heads, length, kv]."""
    heads, page = max(1, c["h_kv"]), c["page"]
    used = s["table"][i, :-(-length // page)].long()
    rows = s[x].view(-1, heads, page, c["kv"]).index_select(0, used).double()
    return rows.transpose(0, 1).reshape(heads, -1, c["kv"])[:, :length]


def _exact_decode(c, s):
    heads, n, group = max(1, c["h_kv"]), c["n"], c["h"] // max(1, c["h_kv"])
    out = torch.zeros((c["b"], n, c["h"], c["kv"]), dtype=torch.float64, device=DEV)
    scores = s["scores_out"].double().view(c["b"], heads, -1) if c["kind"] == "scored" else None
    lens = s["lens"].tolist()
    for i, length in enumerate(lens):
        K, V = _sequence(s, "K", i, length, c), _sequence(s, "V", i, length, c)
        total = torch.zeros((heads, length), dtype=torch.float64, device=DEV)
        for j in range(n):
            seen = length - (n - 1 - j)
            if seen <= 0:
                continue
            qs = s["q"][i, j].double().view(heads, group, c["kv"])
            z = (qs @ K[:, :seen].transpose(1, 2)) * s["scale"]
            a = torch.softmax(z, dim=-1)
            out[i, j] = (a @ V[:, :seen]).reshape(c["h"], c["kv"])
            total[:, :seen] += a.sum(1)
        if scores is not None:
            old = max(0, length - n)
            scores[i, :, :length] = total
            scores[i, :, :old] += s["scores"].view(c["b"], heads, -1)[i, :, :old].double()
    return out if scores is None else (out, scores.view_as(s["scores_out"]))


def _exact_evict(c, s):
    heads, page, b = max(1, c["h_kv"]), c["page"], c["b"]
    K, V = s["K"].double().cpu(), s["V"].double().cpu()
    Ks, Vs = (t.view(-1, heads, page, c["kv"]) for t in (K, V))
    scores, out = s["scores"].double().cpu().numpy().reshape(b, heads, -1), np.zeros((b, heads, s["scores_out"].shape[-1]))
    table, to, lens = (s[x].cpu().numpy() for x in ("table", "table_out", "lens"))
    for i in range(b):
        for e in range(heads):
            old = max(0, lens[i] - c["recent"])
            newest = np.arange(old, lens[i])
            most = sorted(range(old), key=lambda x: (-scores[i, e, x], x))[:max(0, c["budget"] - len(newest))]
            keep = np.array(sorted([*most, *newest]), dtype=np.int64)
            slot = np.arange(len(keep))
            source = torch.from_numpy(table[i, keep // page].astype(np.int64)), e, torch.from_numpy(keep % page)
            target = torch.from_numpy(to[i, slot // page].astype(np.int64)), e, torch.from_numpy(slot % page)
            Ks[target] = Ks[source]
            Vs[target] = Vs[source]
            out[i, e, :len(keep)] = scores[i, e, keep]
    return K, V, None, torch.from_numpy(out).view_as(s["scores_out"]), None
