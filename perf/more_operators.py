"""The operators of a batched verification round over a paged K/V cache, their
plain forms and the calls that are timed: the append with the position rotation
on the way, attention of the drafted rows of many requests over their pages, the
selection of pages by a cheap score and the attention over the selected ones,
and the log probabilities of the drafted tokens.

The cache of one layer is a pool of pages, k and v [n_pages][Hkv][page][D], with
the bounds [n_pages][Hkv][2][D] (smallest and largest key of each page in every
dimension).  A batch is a ragged list of sequences: sequence b owns the rows
row_start[b] .. row_start[b + 1] of the call's tensors, its row i sits at
position ctx_len[b] + i, and position p of it lies in row p % page of the page
page_table[b][p // page].  Rows behind row_start[n_seqs] belong to nobody and
their outputs stay as they were.

A case is a plain dict; "kind" names the operator, the rest its sizes:

  append   wf_paged_append: K rotated, V copied, bounds kept, q rotated too
  attn     wf_paged_verify_attn, block-causal or under a tree's masks
  select   wf_paged_select: each row's and KV head's n_top best pages (by the
           bound sum_d max(q_d lo_d, q_d hi_d), the largest over the query
           heads of the group) and its n_recent newest
  sparse   wf_paged_sparse_attn over such a selection
  logprob  wf_token_logprobs: log probability and rank of a given token,
           entropy, the n best tokens

Ragged lengths follow from the case alone ("mix" seeds them), everything else
from the seed.
"""
import math
import random

import torch

own = False

BF16, F32, F64, I32 = torch.bfloat16, torch.float32, torch.float64, torch.int32
DEV = "cuda"
STD = 0.02 * math.sqrt(4096)
ROPE_BASE = 1e6
VOCAB = 151936


# ---- the cases ---------------------------------------------------------------

def _batch(name, kind, seqs, rows, ctx, page, heads, dt="bf16", mix=1, pad=0, **more):
    """seqs sequences of up to `rows` rows behind contexts of up to `ctx`."""
    return {"name": name, "kind": kind, "seqs": seqs, "rows": rows, "ctx": ctx, "page": page,
            "hq": heads[0], "hkv": heads[1], "dh": heads[2], "dt": dt, "mix": mix, "pad": pad,
            **more}


def _logprob(name, rows, vocab, top, dt="f32"):
    return {"name": name, "kind": "logprob", "rows": rows, "vocab": vocab, "top": top, "dt": dt}


H8B, H32B, H64 = (32, 8, 128), (64, 8, 128), (8, 2, 64)


def listed():
    return [
        # one token of each of 64 chats (8B attention shapes): the append that
        # every layer of every decoding round makes
        _batch("append-decode-64", "append", 64, 1, 4000, 64, H8B, tree=False),
        # five ragged prompts, some thousand rows, in pages of 16
        _batch("append-prompts-5", "append", 5, 3000, 0, 16, H8B, mix=2, tree=False),
        # a single chat's token over about a thousand tokens: the smallest call
        _batch("attn-decode-1x1k", "attn", 1, 1, 1003, 64, H8B, tree=False),
        # blocks of up to 16 drafted tokens of 16 requests, up to 8K tokens each
        _batch("attn-block16-16x8k", "attn", 16, 16, 8192, 32, H8B, mix=3, tree=False),
        # draft trees of up to 61 nodes of 4 requests over up to 8K tokens
        _batch("attn-tree61-4x8k", "attn", 4, 61, 8192, 16, H8B, mix=4, tree=True),
        # a full decoding batch of mixed lengths, the largest attention
        _batch("attn-decode-128x16k", "attn", 128, 1, 16384, 16, H8B, mix=5, tree=False),
        # the page selection of one long document, and of a batch of them
        _batch("select-1x64k", "select", 1, 1, 65000, 64, H8B, n_top=60, n_recent=4),
        _batch("select-16x32k", "select", 16, 4, 32768, 32, H32B, mix=6, n_top=120, n_recent=2),
        # attention over the selected pages of the same two
        _batch("sparse-1x64k", "sparse", 1, 1, 65000, 64, H8B, n_top=60, n_recent=4, tree=False),
        _batch("sparse-16x32k", "sparse", 16, 4, 32768, 32, H32B, mix=6, n_top=120, n_recent=2,
               tree=False),
        # the drafted tokens of one verification block, fp32 logits
        _logprob("logprob-16", 16, VOCAB, 20),
        # scoring a prompt, bf16 logits
        _logprob("logprob-prompt-2000", 2000, VOCAB, 5, "bf16"),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, even over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("append", "attn", "attn", "attn", "select", "sparse", "sparse",
                       "logprob", "logprob"))
    if kind == "logprob":
        rows = _log(rng, 1, 2000)
        c = _logprob("", rows, _log(rng, 500, VOCAB), rng.choice((0, 1, 5, 20, 64)),
                     rng.choice(("f32", "bf16")))
        del c["name"]
        return c
    heads = rng.choice((H8B, H8B, H32B, (24, 8, 128), (16, 8, 128), (32, 8, 64), (16, 1, 128),
                        (7, 7, 64)))
    page, mix = rng.choice((16, 32, 64, 128)), rng.randrange(1 << 30)
    pad = rng.choice((0, 0, 3))
    dt = "bf16"
    if kind == "append":
        seqs, dt = _log(rng, 1, 64), rng.choice(("bf16", "bf16", "f32"))
        rows = _log(rng, 1, max(1, 6000 // seqs))
        c = _batch("", kind, seqs, rows, _log(rng, 1, 4000) - 1, page, heads, dt, mix, pad,
                   tree=rows <= 64 and rng.random() < 0.3)
    elif kind == "attn" and rng.random() < 0.15:
        c = _batch("", kind, _log(rng, 1, 8), _log(rng, 1, 16), _log(rng, 1, 1000) - 1, page,
                   rng.choice((H64, (8, 2, 128), (4, 4, 64))), "f32", mix, pad, tree=False)
    elif kind == "attn":
        seqs, rows = _log(rng, 1, 128), _log(rng, 1, 64)
        most = min(65536, 1500000 // seqs, (1 << 25) // (seqs * rows * heads[0]) + 64)
        c = _batch("", kind, seqs, rows, _log(rng, 50, most), page, heads, dt, mix, pad,
                   tree=rows > 4 and rng.random() < 0.4)
    else:
        seqs, rows, recent = _log(rng, 1, 16), _log(rng, 1, 4), rng.randint(1, 4)
        ctx = _log(rng, 12 * page, 32768)
        # a few of the pages up to half of them
        c = _batch("", kind, seqs, rows, ctx, page, heads, dt, mix, pad,
                   n_top=_log(rng, 2, min(8192 // page, (ctx // page - recent) // 2)),
                   n_recent=recent)
        if kind == "sparse":
            c["tree"] = rows > 2 and rng.random() < 0.3
    del c["name"]
    return c


def _lengths(c):
    """(rows, context) of every sequence, from the case alone."""
    if c["seqs"] == 1:
        return [(c["rows"], c["ctx"])]
    rng = random.Random(c["mix"])
    out = []
    for _ in range(c["seqs"]):
        # up to the most, from a third on; one sequence in twenty is idle
        rows = rng.randint((c["rows"] + 2) // 3, c["rows"])
        ctx = _log(rng, 1 + c["ctx"] // 16, 1 + c["ctx"]) - 1
        out.append((0 if rng.random() < 0.05 else rows, ctx))
    out[-1] = (c["rows"], c["ctx"])
    return out


def _pages(c, rows, ctx):
    return (ctx + rows + c["page"] - 1) // c["page"]


def _dtype(name):
    return BF16 if name == "bf16" else F32


# ---- inputs, from the seed alone ------------------------------------------------

class _Rand:
    def __init__(self, seed):
        self.gen = torch.Generator(device=DEV)
        self.gen.manual_seed(int(seed) % (1 << 62))

    def normal(self, *shape, std=1.0, dtype=BF16):
        return torch.empty(shape, device=DEV, dtype=dtype).normal_(0.0, std, generator=self.gen)

    def unit(self, *shape):
        return torch.rand(shape, generator=self.gen, device=DEV)

    def below(self, n, *shape):
        return torch.randint(0, n, shape, generator=self.gen, device=DEV)


def _tree(rng, n):
    """Depths and ancestor masks of a random draft tree: every node's parent
    is one of the ten or so nodes before it, as in a top-k expansion."""
    depth, mask = [0], [1]
    for i in range(1, n):
        p = max(0, i - 1 - int(rng.random() * min(i, 10)))
        depth.append(depth[p] + 1)
        mask.append(mask[p] | (1 << i))
    return depth, [m - (1 << 64) if m >> 63 else m for m in mask]


def _ints(values, dtype=I32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def prepare(case, seed):
    """A case's state: what a serving loop has in hand before the call."""
    c, r = case, _Rand(seed)
    s = dict(case=dict(c))
    if c["kind"] == "logprob":
        # logits of a language model: a broad bulk and some likely tokens
        x = r.normal(c["rows"], c["vocab"], std=2.0, dtype=_dtype(c["dt"]))
        some = (r.below(c["vocab"], c["rows"], 1)
                + torch.arange(40, device=DEV) * (c["vocab"] // 40)) % c["vocab"]
        x.scatter_(1, some, r.normal(c["rows"], 40, std=4.0, dtype=x.dtype) + 8.0)
        s["logits"] = x
        # a drafted token is usually a likely one
        pick = torch.where(r.unit(c["rows"]) < 0.8, some[:, 0], r.below(c["vocab"], c["rows"]))
        s["tokens"] = pick.to(I32)
        n = c["rows"]
        s["out"] = [torch.empty(n, device=DEV), torch.empty(n, device=DEV),
                    torch.empty(n, dtype=I32, device=DEV),
                    torch.empty(n, c["top"], dtype=I32, device=DEV),
                    torch.empty(n, c["top"], device=DEV)]
        if own:
            import paper_2606_07710_amd as wf
            s["wf"] = wf
            s["ws"] = wf.alloc_workspace(wf.wf_token_logprobs_workspace_bytes(
                x.dtype, n, c["vocab"], c["top"]), DEV)
        return s
    lens = s["lens"] = _lengths(c)
    dt, hq, hkv, dh, page = _dtype(c["dt"]), c["hq"], c["hkv"], c["dh"], c["page"]
    n = sum(x[0] for x in lens) + c["pad"]
    counts = [_pages(c, *x) for x in lens]
    n_pages = sum(counts) + 3
    # pages lie anywhere in the pool; entries that no sequence uses are -1
    order = torch.randperm(n_pages, generator=r.gen, device=DEV).to(I32)
    table = torch.full((c["seqs"], max(counts) + 2), -1, dtype=I32, device=DEV)
    at, start = 0, [0]
    for b, (rows, _) in enumerate(lens):
        table[b, : counts[b]] = order[at: at + counts[b]]
        at += counts[b]
        start.append(start[-1] + rows)
    s["table"], s["row_start"] = table, _ints(start)
    s["ctx_len"] = _ints([x[1] for x in lens])
    s["start"] = start
    scale = torch.ones(dh, device=DEV)
    scale[::16] = 4.0                    # some channels of keys are larger
    if c["kind"] != "select":
        s["k"] = r.normal(n_pages, hkv, page, dh, std=STD, dtype=dt)
        s["k"] *= scale.to(dt)
        s["v"] = r.normal(n_pages, hkv, page, dh, std=STD, dtype=dt)
    else:
        # the selection reads the bounds alone: those of random keys
        mid = r.normal(n_pages, hkv, 1, dh, std=STD / 2, dtype=F32)
        half = STD * (1.0 + 2.0 * r.unit(n_pages, hkv, 1, dh))
        s["k"] = s["v"] = torch.zeros(n_pages, hkv, page, dh, dtype=dt, device=DEV)
        s["bounds"] = (torch.cat([mid - half, mid + half], 2) * scale).to(dt)
    if c["kind"] == "append":
        s["bounds"] = torch.cat([s["k"].amin(2, True), s["k"].amax(2, True)], 2)
        # as one projection leaves them: q, k and v of a row side by side
        qkv = r.normal(n, (hq + 2 * hkv) * dh, std=STD, dtype=dt)
        s["q"] = qkv[:, : hq * dh].view(n, hq, dh)
        s["new_k"] = qkv[:, hq * dh: (hq + hkv) * dh].view(n, hkv, dh)
        s["new_v"] = qkv[:, (hq + hkv) * dh:].view(n, hkv, dh)
        s["out"] = torch.zeros(n, hq, dh, dtype=dt, device=DEV)
    else:
        s["q"] = r.normal(n, hq, dh, std=STD, dtype=dt)
        s["out"] = torch.zeros_like(s["q"])
    s["positions"] = s["mask"] = None
    if c.get("tree"):
        rng, depth, mask = random.Random(seed), [], []
        for rows, ctx in lens:
            if rows:
                d, m = _tree(rng, rows)
                depth += [ctx + x for x in d]
                mask += m
        s["positions"] = _ints(depth + [0] * c["pad"])
        s["mask"] = _ints(mask + [0] * c["pad"], torch.int64)
    if c["kind"] in ("select", "sparse"):
        s["sel"] = torch.full((n, hkv, c["n_top"] + c["n_recent"]), -7, dtype=I32, device=DEV)
    if c["kind"] == "sparse":
        for b, (rows, ctx) in enumerate(lens):
            if rows:
                score = r.unit(rows, hkv, counts[b])
                s["sel"][start[b]: start[b + 1]] = _pick(c, score, ctx, rows)
    if own:
        import paper_2606_07710_amd as wf
        s["wf"] = wf
        s["cache"] = wf.PagedCache(s["k"], s["v"], s.get("bounds"))
        s["batch"] = wf.PagedBatch(s["table"], s["row_start"], s["ctx_len"], min(c["rows"], 64))
        args = dt, n, c["seqs"], min(c["rows"], 64), hq, hkv, dh
        if c["kind"] == "attn":
            s["ws"] = wf.alloc_workspace(wf.wf_paged_verify_attn_workspace_bytes(*args), DEV)
        elif c["kind"] == "select":
            s["ws"] = wf.alloc_workspace(wf.wf_paged_select_workspace_bytes(
                n, hkv, s["table"].shape[1]), DEV)
        elif c["kind"] == "sparse":
            s["ws"] = wf.alloc_workspace(wf.wf_paged_sparse_attn_workspace_bytes(
                dt, n, hq, hkv, dh, page, s["sel"].shape[2]), DEV)
    return s


# ---- one pass -----------------------------------------------------------------------

def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    if kind == "append":
        if own:
            s["wf"].wf_paged_append(s["new_k"], s["new_v"], s["cache"], s["batch"], ROPE_BASE,
                                    q=s["q"], q_out=s["out"], positions=s["positions"])
        else:
            _plain_append(s, c)
        return {"k": s["k"], "v": s["v"], "bounds": s["bounds"], "q": s["out"]}
    if kind == "attn":
        if own:
            return s["wf"].wf_paged_verify_attn(s["q"], s["cache"], s["batch"], s["out"],
                                                tree_mask=s["mask"], workspace=s["ws"])
        return _plain_attn(s, c)
    if kind == "select":
        if own:
            return s["wf"].wf_paged_select(s["q"], s["cache"], s["batch"], s["sel"],
                                           c["n_recent"], workspace=s["ws"])
        return _plain_select(s, c)
    if kind == "sparse":
        if own:
            return s["wf"].wf_paged_sparse_attn(s["q"], s["cache"], s["batch"], s["sel"],
                                                s["out"], tree_mask=s["mask"],
                                                workspace=s["ws"])
        return _plain_sparse(s, c)
    names = ("logprob", "entropy", "rank", "top_ids", "top_logprobs")
    if own:
        s["wf"].wf_token_logprobs(s["logits"], s["tokens"], *s["out"][:3],
                                  *(s["out"][3:] if c["top"] else (None, None)),
                                  workspace=s["ws"])
    else:
        _plain_logprob(s, c)
    return dict(zip(names, s["out"]))


# ---- plain forms: elementary torch operations in 32 bits -------------------------------

def _rotated(x, pos):
    """x [n][heads][D] turned by its positions [n]: the pair (i, i + D/2) by
    pos * base^(-2i/D) radians, angles in 64 bits."""
    half = x.shape[-1] // 2
    i = torch.arange(half, device=DEV, dtype=F64)
    a = pos.to(F64)[:, None] * ROPE_BASE ** (-2.0 * i / (2 * half))
    cos, sin = torch.cos(a).to(F32)[:, None], torch.sin(a).to(F32)[:, None]
    lo, hi = x[..., :half].to(F32), x[..., half:].to(F32)
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)


def _plain_append(s, c):
    page, n = c["page"], s["start"][-1]
    seq = torch.repeat_interleave(torch.arange(c["seqs"], device=DEV),
                                  (s["row_start"][1:] - s["row_start"][:-1]).long(),
                                  output_size=n)
    slot = s["ctx_len"][seq] + torch.arange(n, device=DEV) - s["row_start"][seq]
    pos = slot if s["positions"] is None else s["positions"][:n]
    phys = s["table"][seq, slot // page].long()
    at = slot % page
    dt = s["k"].dtype
    s["k"][phys, :, at] = _rotated(s["new_k"][:n], pos).to(dt)
    s["v"][phys, :, at] = s["new_v"][:n]
    s["out"][:n] = _rotated(s["q"][:n], pos).to(dt)
    # bounds of every page that got a row, over its rows up to the newest
    for b, (rows, ctx) in enumerate(s["lens"]):
        if rows:
            p0, p1 = ctx // page, (ctx + rows - 1) // page + 1
            ids = s["table"][b, p0:p1].long()
            x = s["k"][ids].to(F32)
            row = torch.arange(p0 * page, p1 * page, device=DEV).view(-1, 1, page, 1)
            out = row >= ctx + rows
            lo = x.masked_fill(out, math.inf).amin(2)
            hi = x.masked_fill(out, -math.inf).amax(2)
            s["bounds"][ids] = torch.stack([lo, hi], 2).to(dt)


def _seen(s, c, b, rows, ctx, pos):
    """Whether row i of a sequence sees the keys at pos (any shape that ends in
    keys and broadcasts with [rows, ...])."""
    i = torch.arange(rows, device=DEV).view(-1, *([1] * (pos.dim() - 1)))
    if s["mask"] is None:
        return pos <= ctx + i
    m = s["mask"][s["start"][b]: s["start"][b + 1]].view(i.shape)
    j = pos - ctx
    return (j < 0) | (j == i) | ((j < rows) & (((m >> j.clamp(0, 63)) & 1) == 1))


def _softmax_v(z, v):
    p = torch.exp(z - z.amax(-1, keepdim=True))
    return torch.matmul(p, v) / p.sum(-1, keepdim=True)


def _plain_attn(s, c):
    hkv, dh, grp = c["hkv"], c["dh"], c["hq"] // c["hkv"]
    for b, (rows, ctx) in enumerate(s["lens"]):
        if not rows:
            continue
        ids = s["table"][b, : _pages(c, rows, ctx)].long()
        k = s["k"][ids].transpose(0, 1).flatten(1, 2)[:, : ctx + rows].to(F32)
        v = s["v"][ids].transpose(0, 1).flatten(1, 2)[:, : ctx + rows].to(F32)
        at = slice(s["start"][b], s["start"][b + 1])
        q = s["q"][at].to(F32).view(rows, hkv, grp, dh).permute(1, 0, 2, 3).flatten(1, 2)
        z = torch.matmul(q.contiguous(), k.transpose(1, 2).contiguous()) * dh ** -0.5
        seen = _seen(s, c, b, rows, ctx, torch.arange(ctx + rows, device=DEV)[None])
        z = z.view(hkv, rows, grp, -1).masked_fill_(~seen[None, :, None], -math.inf)
        o = _softmax_v(z.flatten(1, 2), v.contiguous()).view(hkv, rows, grp, dh)
        s["out"][at] = o.permute(1, 0, 2, 3).reshape(rows, c["hq"], dh).to(s["out"].dtype)
    return s["out"]


def _pick(c, score, ctx, rows):
    """The selection [rows][Hkv][n_top + n_recent] from scores [rows][Hkv]
    [pages]: ascending pages, -1 behind them."""
    most, n = c["n_top"] + c["n_recent"], score.shape[2]
    page = torch.arange(n, device=DEV)
    newest = (ctx + torch.arange(rows, device=DEV)).view(-1, 1, 1) // c["page"]
    recent = (page > newest - c["n_recent"]) & (page <= newest)
    old = page <= newest - c["n_recent"]
    rank = torch.sort(score.masked_fill(~old, -math.inf), dim=-1, descending=True,
                      stable=True).indices
    top = torch.zeros(score.shape, dtype=torch.bool, device=DEV)
    top.scatter_(2, rank[..., : c["n_top"]], True)
    ids = torch.where((top & old) | recent, page, torch.full_like(page, 1 << 30))
    ids = torch.sort(ids, dim=-1).values[..., :most]
    out = torch.full((*score.shape[:2], most), -1, dtype=I32, device=DEV)
    out[..., : ids.shape[2]] = torch.where(ids < 1 << 30, ids, torch.full_like(ids, -1)).to(I32)
    return out


def _plain_select(s, c):
    # scores in 64 bits: two pages next to the border must not change places
    hkv, dh, grp = c["hkv"], c["dh"], c["hq"] // c["hkv"]
    for b, (rows, ctx) in enumerate(s["lens"]):
        if not rows:
            continue
        ids = s["table"][b, : _pages(c, rows, ctx)].long()
        lo, hi = s["bounds"][ids].to(F64).permute(2, 1, 3, 0).contiguous()
        at = slice(s["start"][b], s["start"][b + 1])
        q = s["q"][at].to(F64).view(rows, hkv, grp, dh).permute(1, 0, 2, 3).reshape(hkv, -1, dh)
        z = torch.matmul(q.clamp(min=0), hi) + torch.matmul(q.clamp(max=0), lo)
        z = z.view(hkv, rows, grp, -1).amax(2).transpose(0, 1)
        s["sel"][at] = _pick(c, z, ctx, rows)
    return s["sel"]


def _plain_sparse(s, c):
    hkv, dh, grp, page = c["hkv"], c["dh"], c["hq"] // c["hkv"], c["page"]
    head = torch.arange(hkv, device=DEV)[None, :, None]
    off = torch.arange(page, device=DEV)
    for b, (rows, ctx) in enumerate(s["lens"]):
        if not rows:
            continue
        at = slice(s["start"][b], s["start"][b + 1])
        sel = s["sel"][at].long()
        phys = s["table"][b][sel.clamp(min=0)].long()
        k = s["k"][phys, head].flatten(2, 3).to(F32)
        v = s["v"][phys, head].flatten(2, 3).to(F32)
        pos = (sel[..., None] * page + off).flatten(2)
        seen = _seen(s, c, b, rows, ctx, pos) & (pos >= 0)
        # keys that no row sees may hold anything
        v = v.masked_fill(~seen[..., None], 0.0)
        q = s["q"][at].to(F32).view(rows, hkv, grp, dh)
        z = torch.matmul(q, k.transpose(2, 3).contiguous()) * dh ** -0.5
        z = z.masked_fill(~seen[:, :, None], -math.inf)
        s["out"][at] = _softmax_v(z, v).reshape(rows, c["hq"], dh).to(s["out"].dtype)
    return s["out"]


def _order_keys(x):
    """64-bit keys that order fp32 values, the lower index first among equals."""
    bits = (x + 0.0).view(torch.int32).long()         # (-0 counts as 0)
    bits = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
    return bits * (1 << 32) - torch.arange(x.shape[-1], device=DEV)


def _plain_logprob(s, c):
    lp, ent, rank, ids, tops = s["out"]
    for r0 in range(0, c["rows"], 256):
        at = slice(r0, min(r0 + 256, c["rows"]))
        x, t = s["logits"][at].to(F32), s["tokens"][at].long()[:, None]
        m = x.amax(1, keepdim=True)
        d = x - m
        e = torch.exp(d)
        total = e.sum(1, keepdim=True)
        logz = torch.log(total)
        mine = x.gather(1, t)
        lp[at] = (mine - m - logz)[:, 0]
        ent[at] = (logz - (e * d).sum(1, keepdim=True) / total)[:, 0]
        index = torch.arange(c["vocab"], device=DEV)
        rank[at] = ((x > mine) | ((x == mine) & (index < t))).sum(1).to(I32)
        if c["top"]:
            best = torch.topk(_order_keys(x), c["top"], dim=1).indices
            ids[at] = best.to(I32)
            tops[at] = x.gather(1, best) - m - logz


# ---- what a pass cannot do without ------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "logprob":
        e = 2 if c["dt"] == "bf16" else 4
        return {"bytes": c["rows"] * (c["vocab"] * e + 16 + 8 * c["top"]),
                "flops": 4 * c["rows"] * c["vocab"]}
    lens, page = _lengths(c), c["page"]
    hq, hkv, dh, e = c["hq"], c["hkv"], c["dh"], 2 if c["dt"] == "bf16" else 4
    n = sum(x[0] for x in lens)
    nbytes = flops = 0
    for rows, ctx in lens:
        if not rows:
            continue
        if c["kind"] == "append":
            # every row in and out, the open pages' older keys, the bounds
            pages = (ctx + rows - 1) // page - ctx // page + 1
            nbytes += rows * (2 * hkv + hq) * 2 * dh * e + hkv * dh * e * (ctx % page + 2 * pages)
            flops += rows * (hq + hkv) * dh * 3
        elif c["kind"] == "attn":
            nbytes += 2 * hkv * (ctx + rows) * dh * e + 2 * rows * hq * dh * e
            nbytes += 4 * _pages(c, rows, ctx) + (8 * rows if c["tree"] else 0)
            flops += 4 * rows * hq * dh * (ctx + rows)
        elif c["kind"] == "select":
            pages = _pages(c, rows, ctx)
            nbytes += pages * (2 * hkv * dh * e + 4) + rows * hq * dh * e
            nbytes += 4 * rows * hkv * (c["n_top"] + c["n_recent"])
            flops += 2 * rows * hq * dh * pages
        else:
            keys = min(_pages(c, rows, ctx), c["n_top"] + c["n_recent"]) * page
            # rows of one sequence may share pages: as many as there are at most
            seen = min(rows * keys, ctx + rows)
            nbytes += 2 * hkv * seen * dh * e + 2 * rows * hq * dh * e
            nbytes += 4 * rows * hkv * (c["n_top"] + c["n_recent"])
            flops += 4 * rows * hq * dh * keys
    return {"bytes": nbytes + 4 * (2 * c["seqs"] + 1), "flops": flops}


# ---- the definitions in 64 bits -----------------------------------------------------------

def _visible(s, b, i, ctx, rows, pos):
    """Row i's view of the positions pos, by the definition."""
    if s["mask"] is None:
        return pos <= ctx + i
    word = int(s["mask"][s["start"][b] + i])
    bits = _ints([(word >> j) & 1 for j in range(rows)], torch.bool)
    bits[i] = True
    block = (pos - ctx).clamp(0, rows - 1)
    return (pos < ctx) | ((pos < ctx + rows) & bits[block])


def _turn64(x, pos):
    """x [heads][D] (64 bits) as complex numbers, turned by one position."""
    half = x.shape[-1] // 2
    z = torch.complex(x[:, :half], x[:, half:])
    angle = pos * torch.exp(torch.arange(half, device=DEV, dtype=F64)
                            * (-math.log(ROPE_BASE) / half))
    z = z * torch.polar(torch.ones_like(angle), angle)
    return torch.cat([z.real, z.imag], -1)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "logprob":
        return _exact_logprob(s, c)
    hkv, dh, page, grp = c["hkv"], c["dh"], c["page"], c["hq"] // c["hkv"]
    out = s["out"].double()
    if c["kind"] == "append":
        k, v, bounds = s["k"].double(), s["v"].double(), s["bounds"].double()
        ids = s["table"].tolist()
        for b, (rows, ctx) in enumerate(s["lens"]):
            for i in range(rows):
                r, slot = s["start"][b] + i, ctx + i
                pos = slot if s["positions"] is None else int(s["positions"][r])
                p = ids[b][slot // page]
                k[p, :, slot % page] = _turn64(s["new_k"][r].double(), pos)
                v[p, :, slot % page] = s["new_v"][r].double()
                out[r] = _turn64(s["q"][r].double(), pos)
            for slot in range(ctx - ctx % page, ctx + rows if rows else 0, page):
                x = k[ids[b][slot // page], :, : min(page, ctx + rows - slot)]
                bounds[ids[b][slot // page], :, 0] = x.min(1).values
                bounds[ids[b][slot // page], :, 1] = x.max(1).values
        return {"k": k, "v": v, "bounds": bounds, "q": out}
    if c["kind"] == "select":
        sel = s["sel"].clone()
        for b, (rows, ctx) in enumerate(s["lens"]):
            for i in range(rows):
                newest = (ctx + i) // page
                old = max(0, newest + 1 - c["n_recent"])
                box = s["bounds"][s["table"][b, :old].long()].double()
                for g in range(hkv):
                    q = s["q"][s["start"][b] + i, g * grp:(g + 1) * grp].double()[:, None]
                    score = torch.maximum(q * box[:, g, 0], q * box[:, g, 1]).sum(-1).amax(0)
                    best = sorted(range(old), key=lambda p, z=score.tolist(): (-z[p], p))
                    got = sorted(best[: c["n_top"]]) + list(range(old, newest + 1))
                    got += [-1] * (sel.shape[2] - len(got))
                    sel[s["start"][b] + i, g] = _ints(got)
        return sel
    for b, (rows, ctx) in enumerate(s["lens"]):
        n = _pages(c, rows, ctx)
        for g in range(hkv) if rows else ():
            mine = s["table"][b, :n].long()
            k, v = s["k"][mine, g].double().flatten(0, 1), s["v"][mine, g].double().flatten(0, 1)
            for i in range(rows):
                r = s["start"][b] + i
                pos = torch.arange(ctx + rows, device=DEV)
                if c["kind"] == "sparse":
                    sel = s["sel"][r, g].long()
                    sel = sel[sel >= 0]
                    pos = (sel[:, None] * page + torch.arange(page, device=DEV)).flatten()
                pos = pos[_visible(s, b, i, ctx, rows, pos)]
                q = s["q"][r, g * grp:(g + 1) * grp].double()
                p = torch.softmax(q @ k[pos].t() / math.sqrt(dh), -1)
                out[r, g * grp:(g + 1) * grp] = p @ v[pos]
    return out


def _exact_logprob(s, c):
    n = c["rows"]
    lp, ent = torch.empty(2, n, dtype=F64, device=DEV)
    rank = torch.empty(n, dtype=I32, device=DEV)
    ids = torch.empty(n, c["top"], dtype=I32, device=DEV)
    tops = torch.empty(n, c["top"], dtype=F64, device=DEV)
    for r in range(n):
        x, t = s["logits"][r].double(), int(s["tokens"][r])
        logp = x - torch.logsumexp(x, 0)
        lp[r], ent[r] = logp[t], -(logp.exp() * logp).sum()
        order = torch.sort(x, descending=True, stable=True).indices
        rank[r] = torch.nonzero(order == t)[0, 0]
        ids[r] = order[: c["top"]]
        tops[r] = logp[order[: c["top"]]]
    return {"logprob": lp, "entropy": ent, "rank": rank, "top_ids": ids, "top_logprobs": tops}
