"""Plain 64-bit definitions of the paged-cache operators and of the token log
probabilities (numpy), the reference of their tests, with the error that each
allows: a rounding to bf16 is off by at most 2^-8 of the value, one to fp32 by
at most 2^-24."""
import numpy as np
import torch

import paper_2606_07710_amd as wf

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def f64(t):
    return t.detach().double().cpu().numpy()


class Round:
    """A paged cache filled with random keys, a batch over it, and q: lens is
    [(rows, context)], the last `pad` rows belong to no sequence."""

    def __init__(self, lens, page=16, hq=8, hkv=2, dh=64, dt="bf16", pad=0, seed=0, std=1.3,
                 spare=2, device="cuda", max_rows=None):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.page, self.hq, self.hkv, self.dh, self.dt = lens, page, hq, hkv, dh, dt
        counts = [-(-(r + c) // page) for r, c in lens]
        n_pages = sum(counts) + 3
        order = torch.randperm(n_pages, generator=g)
        self.table = torch.full((len(lens), max(counts) + spare), -1, dtype=torch.int32)
        at, self.start = 0, [0]
        for b, (rows, _) in enumerate(lens):
            self.table[b, : counts[b]] = order[at: at + counts[b]].int()
            at += counts[b]
            self.start.append(self.start[-1] + rows)
        self.n = self.start[-1] + pad
        shape = (n_pages, hkv, page, dh)
        rnd = lambda *s: (torch.randn(*s, generator=g) * std).to(DT[dt])  # noqa: E731
        self.k, self.v = rnd(*shape), rnd(*shape)
        self.bounds = torch.cat([self.k.amin(2, True), self.k.amax(2, True)], 2)
        self.q = rnd(self.n, hq, dh)
        self.new_k, self.new_v = rnd(self.n, hkv, dh), rnd(self.n, hkv, dh)
        self.ctx = torch.tensor([c for _, c in lens], dtype=torch.int32)
        self.max_rows = max_rows or max(1, min(64, max(r for r, _ in lens)))
        self.device = device

    def on_gpu(self, with_bounds=True):
        d = self.device
        self.dk, self.dv = self.k.to(d), self.v.to(d)
        self.db = self.bounds.to(d) if with_bounds else None
        self.cache = wf.PagedCache(self.dk, self.dv, self.db)
        self.batch = wf.PagedBatch(self.table.to(d), torch.tensor(self.start, dtype=torch.int32,
                                                                  device=d),
                                   self.ctx.to(d), self.max_rows)
        self.dq = self.q.to(d)
        return self


def rotate(x, pos, base):
    """x [..., D] in 64 bits, turned by pos."""
    half = x.shape[-1] // 2
    a = pos * base ** (-2.0 * np.arange(half) / (2 * half))
    lo, hi = x[..., :half], x[..., half:]
    return np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], -1)


def rotation_error(x, ref, dt):
    """Two products with factors good to 2^-21 (a reduced angle of at most pi in
    fp32, its sine and cosine), then the stored rounding."""
    half = x.shape[-1] // 2
    mag = np.abs(x[..., :half]) + np.abs(x[..., half:])
    return np.concatenate([mag, mag], -1) * 2.0 ** -21 + np.abs(ref) * HALF_STEP[dt]


def visible(rnd, b, i, tree):
    """Positions that row i of sequence b sees."""
    rows, ctx = rnd.lens[b]
    if tree is None:
        return np.arange(ctx + i + 1)
    word = int(tree[rnd.start[b] + i]) & (2 ** 64 - 1)
    block = [j for j in range(rows) if j == i or (word >> j) & 1]
    return np.concatenate([np.arange(ctx), ctx + np.array(block)]).astype(int)


def attention(rnd, tree=None, sel=None, scale=None):
    """(out, error) [n][Hq][D] of the attention; rows of no sequence are NaN.
    The error: bf16 rounds each weight and the result; the scores are fp32 sums
    of D products, an exponential takes a few steps of 2^-23 and 2^-24 of its
    exponent, the sums over the keys 2^-24 a term."""
    scale = rnd.dh ** -0.5 if scale is None else scale
    k, v, q = f64(rnd.k), f64(rnd.v), f64(rnd.q)
    out = np.full(q.shape, np.nan)
    err = np.zeros(q.shape)
    grp, n_pool = rnd.hq // rnd.hkv, rnd.k.shape[0]
    for b, (rows, ctx) in enumerate(rnd.lens):
        for i in range(rows):
            r = rnd.start[b] + i
            seen = visible(rnd, b, i, tree)
            for g in range(rnd.hkv):
                at = seen
                if sel is not None:
                    pages = [p for p in sel[r, g].tolist() if 0 <= p <= (ctx + i) // rnd.page]
                    at = np.concatenate([np.arange(p * rnd.page, (p + 1) * rnd.page)
                                         for p in pages] + [np.zeros(0, int)]).astype(int)
                    at = at[np.isin(at, seen) & (at <= ctx + i)]
                ids = rnd.table[b].numpy()[at // rnd.page]
                ok = (ids >= 0) & (ids < n_pool)
                at, ids = at[ok], ids[ok]
                kk, vv = k[ids, g, at % rnd.page], v[ids, g, at % rnd.page]
                for h in range(g * grp, (g + 1) * grp):
                    if not len(at):
                        out[r, h] = 0.0
                        continue
                    z = kk @ q[r, h] * scale
                    w = np.exp(z - z.max())
                    w /= w.sum()
                    out[r, h] = w @ vv
                    mag = w @ np.abs(vv)
                    dz = (rnd.dh + 8) * 2.0 ** -24 * (np.abs(kk) @ np.abs(q[r, h])).max() * scale
                    rel = 2 * dz + 2.0 ** -21 + 2.0 ** -24 * (2 * (z.max() - z.min()) + len(at))
                    if rnd.dt == "bf16":
                        rel += HALF_STEP["bf16"]
                    err[r, h] = mag * rel + np.abs(out[r, h]) * (HALF_STEP[rnd.dt] + 2.0 ** -22)
    return out, err


def select(rnd, n_sel, n_recent):
    """The selection [n][Hkv][n_sel]; rows of no sequence hold -7."""
    bounds, q = f64(rnd.bounds), f64(rnd.q)
    grp, n_pool = rnd.hq // rnd.hkv, rnd.k.shape[0]
    out = np.full((rnd.n, rnd.hkv, n_sel), -7, np.int32)
    for b, (rows, ctx) in enumerate(rnd.lens):
        for i in range(rows):
            r, newest = rnd.start[b] + i, (ctx + i) // rnd.page
            n_old = max(0, newest + 1 - n_recent)
            for g in range(rnd.hkv):
                score = []
                for p in range(n_old):
                    t = int(rnd.table[b, p])
                    if not 0 <= t < n_pool:
                        continue
                    lo, hi = bounds[t, g]
                    qq = q[r, g * grp:(g + 1) * grp]
                    odd = not (np.isfinite(bounds[t, g]).all() and np.isfinite(qq).all())
                    with np.errstate(invalid="ignore"):
                        s = (qq * np.where(qq >= 0, hi, lo)).sum(-1).max()
                    score.append((0, 0.0, p) if odd else (1, -s, p))
                top = sorted(p for _, _, p in sorted(score)[: n_sel - n_recent])
                got = top + list(range(n_old, newest + 1))
                out[r, g] = got + [-1] * (n_sel - len(got))
    return out


def logprobs(logits, tokens, n_top):
    """(logprob, entropy, rank, top ids, top log probabilities) in 64 bits."""
    n, vocab = logits.shape
    lp, ent, rank = np.zeros(n), np.zeros(n), np.zeros(n, np.int64)
    ids, tops = np.zeros((n, n_top), np.int64), np.zeros((n, n_top))
    for r in range(n):
        z = logits[r]
        nan = np.isnan(z)
        key = np.where(nan, np.inf, z)
        # NaN before everything, then by value, the lower index first
        order = np.lexsort((np.arange(vocab), -key, ~nan))
        with np.errstate(all="ignore"):
            m = z.max() if not nan.any() else np.nan
            w = np.exp(z - m)
            logp = z - m - np.log(w.sum())
            ent[r] = -(np.where(w > 0, logp, 0.0) * w).sum() / w.sum()
        t = int(tokens[r])
        if 0 <= t < vocab:
            lp[r], rank[r] = logp[t], np.nonzero(order == t)[0][0]
        else:
            lp[r], rank[r] = 0.0, -1
        ids[r], tops[r] = order[:n_top], logp[order[:n_top]]
    return lp, ent, rank, ids, tops


def random_tree(rng, rows):
    mask = [1]
    for i in range(1, rows):
        mask.append(mask[int(rng.integers(max(0, i - 10), i))] | (1 << i))
    return mask


def masks64(words, device="cuda"):
    """Unsigned 64-bit words as an int64 tensor."""
    return torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64,
                        device=device)
