"""wf_token_logprobs on the GPU against its 64-bit definition.  Allowed errors:
the differences z - m are exact to 2^-24 of the logits' spread, exponentials to
2^-22, and the sums join at most a few thousand fp32 terms a lane and 2^8 lanes:
2^-24 * 2^10 for their common rounding at the very most, 2^-13 in units of the
entropy's terms; observed errors are some hundred times smaller."""
import numpy as np
import pytest
import torch

import paged_ref as R

wf = pytest.importorskip("paper_2606_07710_amd")
pytestmark = pytest.mark.gpu


def run(x, tokens, n_top, ws=None, **kw):
    n = x.shape[0]
    d = dict(device="cuda")
    lp, ent = torch.full((n,), 9.0, **d), torch.full((n,), 9.0, **d)
    rank = torch.full((n,), -9, dtype=torch.int32, **d)
    ids = torch.full((n, n_top), -9, dtype=torch.int32, **d) if n_top else None
    tops = torch.full((n, n_top), 9.0, **d) if n_top else None
    wf.wf_token_logprobs(x, tokens, lp, ent, rank, ids, tops, workspace=ws, **kw)
    return lp, ent, rank, ids, tops


def compare(x, tokens, n_top, got=None):
    lp, ent, rank, ids, tops = got or run(x, tokens, n_top)
    z = R.f64(x)
    rlp, rent, rrank, rids, rtops = R.logprobs(z, tokens.cpu().numpy(), n_top)
    fin = z[np.isfinite(z)]
    spread = float(fin.max() - fin.min()) if fin.size else 0.0
    tol = 2.0 ** -13 + 2.0 ** -22 * spread

    def close(a, b, scale=1.0):
        a = R.f64(a)
        same = (np.isnan(a) & np.isnan(b)) | (a == b)
        with np.errstate(invalid="ignore"):
            near = np.abs(a - b) <= tol * scale
        assert (same | near).all(), (a[~(same | near)][:4], b[~(same | near)][:4])

    close(lp, rlp)
    close(ent, rent, 16.0)                    # sums of up to log(vocab) times p
    assert np.array_equal(rank.cpu().numpy(), rrank)
    if n_top:
        assert np.array_equal(ids.cpu().numpy(), rids)
        close(tops, rtops)


def logits(n, vocab, dt, seed, std=3.0):
    g = torch.Generator("cuda").manual_seed(seed)
    return (torch.randn(n, vocab, generator=g, device="cuda") * std).to(R.DT[dt])


def tokens(n, vocab, seed):
    g = torch.Generator("cuda").manual_seed(seed + 1000)
    return torch.randint(0, vocab, (n,), generator=g, device="cuda").int()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,top", [
    (1, 1, 1), (1, 1, 0), (3, 2, 2), (2, 63, 5), (2, 64, 64), (5, 65, 20), (1, 1000, 64),
    (4, 2047, 7), (4, 2049, 1), (16, 151936, 20), (1, 128256, 64), (3, 50257, 0), (700, 999, 8),
    (1100, 4099, 3), (1, 1 << 20, 5), (3, 30011, 33), (2, 5000, 48), (600, 9001, 40),
])
def test_sizes(dt, n, vocab, top):
    print("logprobs", dt, n, vocab, top, flush=True)
    compare(logits(n, vocab, dt, n + vocab), tokens(n, vocab, n), top)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1, 3, 5])
def test_strides_and_alignment(dt, shift):
    big = logits(5, 5003, dt, 3)
    x = big[:, shift: shift + 4001]
    t = tokens(5, 4001, 4)
    compare(x, t, 9)
    one = big.flatten()[shift: shift + 3001].unsqueeze(0)
    compare(one, t[:1].clamp(max=3000), 4)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("top", [1, 64])
def test_orders_that_fill_the_lists(dt, top):
    """Ascending rows (every value enters), equal rows (ties go to the lowest
    index), few distinct values, descending rows."""
    v = 9000
    ramp = torch.linspace(-20, 20, v, device="cuda")
    rows = [ramp, ramp.flip(0), torch.zeros(v, device="cuda"),
            (torch.arange(v, device="cuda") % 3).float(), -torch.zeros(v, device="cuda"),
            torch.where(torch.arange(v, device="cuda") % 7 == 0, 1.0, 0.0),
            torch.where(torch.arange(v, device="cuda") % 2 == 0, 0.0, -0.0)]
    x = torch.stack(rows).to(R.DT[dt])
    compare(x, tokens(len(rows), v, 5), top)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [70, 20000])
def test_masked_infinite_and_nan_logits(dt, vocab):
    inf, nan = float("inf"), float("nan")
    x = logits(9, vocab, dt, 7)
    x[0, 3:] = -inf                           # three tokens left
    x[1] = -inf                               # none
    x[2, 5] = inf
    x[3, 6] = nan
    x[4, :] = nan
    x[5, 1:] = -inf                           # one: entropy 0
    x[6, 8], x[6, 9] = nan, inf
    x[7] = torch.where(torch.arange(vocab, device="cuda") % 2 == 0, x[7].float(),
                       -inf).to(x.dtype)
    x[8, 60] = nan
    t = torch.tensor([4, 2, 5, 7, 3, 0, 9, 1, 60], dtype=torch.int32, device="cuda")
    compare(x, t, 20)
    t = torch.tensor([1, 69, 4, 6, 0, 5, 8, 2, 3], dtype=torch.int32, device="cuda")
    compare(x, t, 64)


def test_padding_tokens_and_left_out_outputs():
    x = logits(4, 3000, "f32", 11)
    t = torch.tensor([-1, 3000, -100, 5], dtype=torch.int32, device="cuda")
    lp, ent, rank, ids, tops = run(x, t, 3)
    assert lp[:3].tolist() == [0, 0, 0] and rank[:3].tolist() == [-1, -1, -1]
    compare(x, t, 3, (lp, ent, rank, ids, tops))
    # parts of the outputs alone
    only = torch.empty(4, device="cuda")
    wf.wf_token_logprobs(x, t, only)
    assert torch.equal(only, lp)
    e2 = torch.empty(4, device="cuda")
    wf.wf_token_logprobs(x, None, None, entropy=e2)
    assert torch.equal(e2, ent)
    i2, l2 = torch.empty_like(ids), torch.empty_like(tops)
    wf.wf_token_logprobs(x, None, None, top_ids=i2, top_logprobs=l2)
    assert torch.equal(i2, ids) and torch.equal(l2, tops)
    wf.wf_token_logprobs(x[:0], t[:0], only[:0])             # no rows


@pytest.mark.parametrize("big", [1e4, 1e30])
def test_large_logits(big):
    x = logits(3, 5000, "f32", 13)
    x[0] += big if big < 1e6 else 0
    x[1, 7], x[1, 8] = big, -big
    x[2, ::2] = -big
    t = torch.tensor([3, 7, 1], dtype=torch.int32, device="cuda")
    lp, ent, rank, ids, tops = run(x, t, 5)
    rlp, rent, rrank, rids, rtops = R.logprobs(R.f64(x), t.cpu().numpy(), 5)
    # the differences to the row's maximum are exact to 2^-24 of themselves
    assert np.allclose(R.f64(lp), rlp, rtol=2.0 ** -22, atol=2.0 ** -12)
    assert np.allclose(R.f64(ent), rent, rtol=2.0 ** -10, atol=2.0 ** -9)
    assert np.array_equal(rank.cpu().numpy(), rrank) and np.array_equal(ids.cpu().numpy(), rids)
    assert np.allclose(R.f64(tops), rtops, rtol=2.0 ** -22, atol=2.0 ** -12)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [70, 5000, 60000])
def test_logits_masked_with_the_lowest_number(dt, vocab):
    """A mask of the type's lowest value, before, between and behind what is
    left, and beside its largest: weights of exactly 0, so the rows' results are
    those of the same rows with -inf there."""
    low, high = torch.finfo(R.DT[dt]).min, torch.finfo(R.DT[dt]).max
    x = logits(8, vocab, dt, 41)
    at = torch.arange(vocab, device="cuda")
    keep = torch.stack([at >= vocab - 3, at < 3, at % 9 == 4, at == vocab // 2, at % 2 == 1,
                        at < 0, at == 5, (at >= vocab // 4) & (at < vocab // 2)])
    x = torch.where(keep, x.float(), low).to(x.dtype)
    x[6, 5] = high
    t = torch.stack([k.nonzero()[0, 0] if k.any() else at[7] for k in keep]).int()
    lp, ent, rank, ids, tops = run(x, t, 3)
    rlp, rent, rrank, rids, rtops = R.logprobs(R.f64(x), t.cpu().numpy(), 3)
    # as `compare` has it, the spread that of the values left (under 2^5)
    assert np.allclose(R.f64(lp), rlp, rtol=0, atol=2.0 ** -13 + 2.0 ** -17)
    assert np.allclose(R.f64(ent), rent, rtol=0, atol=16 * (2.0 ** -13 + 2.0 ** -17))
    assert np.array_equal(rank.cpu().numpy(), rrank) and np.array_equal(ids.cpu().numpy(), rids)
    # (differences of 2^128 and more are -inf in fp32; 2^-22 of the larger ones)
    with np.errstate(over="ignore"):
        assert np.allclose(R.f64(tops), rtops.astype(np.float32), rtol=2.0 ** -22,
                           atol=2.0 ** -13 + 2.0 ** -17)


def test_captured_call_replays_and_the_workspace_stays_clean():
    x, t = logits(16, 30000, "f32", 17), tokens(16, 30000, 18)
    ws = wf.alloc_workspace(wf.wf_token_logprobs_workspace_bytes(x.dtype, 16, 30000, 20), "cuda")
    out = [torch.empty(16, device="cuda"), torch.empty(16, device="cuda"),
           torch.empty(16, dtype=torch.int32, device="cuda"),
           torch.empty(16, 20, dtype=torch.int32, device="cuda"),
           torch.empty(16, 20, device="cuda")]
    wf.wf_token_logprobs(x, t, *out, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        wf.wf_token_logprobs(x, t, *out, workspace=ws)
    for i in range(3):
        x.copy_(logits(16, 30000, "f32", 20 + i))
        for o in out:
            o.fill_(-3)
        g.replay()
        torch.cuda.synchronize()
        replayed = [o.clone() for o in out]
        compare(x, t, 20, tuple(replayed))
        wf.wf_token_logprobs(x, t, *out, workspace=ws)
        for a, b in zip(out, replayed):
            assert torch.equal(a, b)
    assert not ws[: 4 << 20].any()


def test_of_the_4_bit_products_logits_beside_the_acceptance_call():
    """The logits that the 4-bit LM head writes: the same argmax and entropy as
    the acceptance call reads from them."""
    g = torch.Generator("cuda").manual_seed(23)
    w = torch.randn(5000, 512, generator=g, device="cuda").to(torch.bfloat16)
    h = torch.randn(16, 512, generator=g, device="cuda").to(torch.bfloat16)
    z = torch.empty(16, 5000, device="cuda")
    wf.wf_linear_w4(h, wf.W4Weight(*wf.wf_w4_quantize(w)), z)
    draft = tokens(15, 5000, 24)
    am = torch.empty(16, dtype=torch.int32, device="cuda")
    ent = torch.empty(16, device="cuda")
    acc = torch.empty(3, dtype=torch.int32, device="cuda")
    wf.wf_lmhead_accept_entropy(None, None, z, draft, 0.5, am, ent, acc)
    t = torch.cat([draft, am[-1:]])
    lp, e2, rank, ids, tops = run(z, t, 4)
    compare(z, t, 4, (lp, e2, rank, ids, tops))
    assert torch.equal(ids[:, 0], am)
    assert torch.allclose(ent, e2, rtol=2e-4, atol=2e-4)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("top", [1, 5, 64])
@pytest.mark.parametrize("vocab,shift", [(1023, 0), (1027, 0), (4098, 1), (9007, 3), (20013, 5)])
def test_a_zero_above_negative_logits_at_the_ends_of_the_runs(dt, top, vocab, shift):
    """Rows whose best values are zeros (of either sign) next to the unaligned
    ends of the rows and of the parts that a row is read in: the elements there
    go one to a lane, and a zero is also what is left in such a lane."""
    print("zeros", dt, top, vocab, shift, flush=True)
    g = torch.Generator("cuda").manual_seed(vocab + top)
    at = sorted({p for e in (0, 1024, 2048, 4096, 8192, vocab) for p in range(e - 8, e + 8)
                 if 0 <= p < vocab})
    n = len(at) + 3
    x = torch.full((n, vocab + 8), 50.0, dtype=R.DT[dt], device="cuda")[:, shift: shift + vocab]
    x.copy_(-1.0 - torch.randn(n, vocab, generator=g, device="cuda").abs())
    for r, p in enumerate(at):
        x[r, p] = 0.0 if r % 3 else -0.0
    x[-3, -3:] = torch.tensor([0.0, -0.0, 0.0])           # several of them
    x[-2, at] = 0.0
    x[-1, ::2] = -0.0
    t = torch.tensor(at + [vocab - 1, at[-1], 1], dtype=torch.int32, device="cuda")
    compare(x, t, top)
    ids = run(x, t, top)[3]
    assert torch.equal(ids[: len(at), 0], t[: len(at)])


def test_sums_of_long_rows():
    """The longest row there can be, in few parts: 2^28 times the logits 1/4, 0, 0,
    0.  A lane has 52428 pieces of four, whose sum 3.336 is no multiple of the
    steps of a large fp32 number: added one after the other they would be off by
    the same amount each time, by 4.5e-4 in all.  Allowed, as for short rows, are
    1100 terms' roundings, 6.6e-5, which the entropy has 1.3 times (its second
    sum is 0.18 of the first), and 2^-20 for the logarithm of about 21."""
    vocab, top = 1 << 30, 64
    print("long row", flush=True)
    x = torch.zeros((1, vocab), device="cuda")
    x[0, ::4] = 0.25
    t = torch.tensor([(1 << 29) + 4], dtype=torch.int32, device="cuda")
    lp, ent, rank, ids, tops = run(x, t, top)
    total = vocab / 4 * (np.exp(0.25) + 3.0)
    p = np.array([np.exp(0.25), 1.0]) / total
    entropy = -vocab / 4 * (p[0] * np.log(p[0]) + 3 * p[1] * np.log(p[1]))
    assert abs(float(lp[0]) - np.log(p[0])) <= 2.0 ** -13
    assert np.abs(R.f64(tops) - np.log(p[0])).max() <= 2.0 ** -13
    assert abs(float(ent[0]) - entropy) <= 2.0 ** -13
    assert int(rank[0]) == (1 << 27) + 1
    assert torch.equal(ids[0].cpu(), torch.arange(0, 4 * top, 4, dtype=torch.int32))
    # a token of the lower ones, at the end
    t.fill_(vocab - 1)
    lp, _, rank, _, _ = run(x, t, 0)
    assert abs(float(lp[0]) - np.log(p[1])) <= 2.0 ** -13
    assert int(rank[0]) == vocab - 1


U = 2.0 ** -24


def chain(vocab, dt):
    """Terms that a value passes on its way into a row's sum, at most: a lane's
    pieces (the fewest lanes: one part), the values of a piece, the sums over
    lanes, waves and parts."""
    per = 4 if dt == "f32" else 8
    return -(-vocab // (256 * per)) + 3 + per + 6 + 2 + 6


def bounds(z, tokens, dt):
    """Errors of a row's log probabilities (at z, an array) and entropy.  A lane's
    reference lies at most 8 below its largest value, so exponents are at most d + 8,
    d = max - z.  A weight e^(z - m): the difference and the product with log2 e
    (a constant with an error of its own) round by U of the exponent each, the
    exponential is good to 2 U, and the moves and joins, of d + 8 together and at most
    d / 8 + 5 of them, do the same again: 6 d + 64 units."""
    n, vocab = z.shape
    m = z.max(1, keepdims=True)
    d = m - z
    w = np.exp(-d)
    total = w.sum(1, keepdims=True)
    p = w / total
    c = chain(vocab, dt)
    a = (p * d).sum(1)
    in_l = 6 * a + 64 + c
    in_t = (p * (d + 8) * (6 * d + 65 + c)).sum(1) + 6 * (a + 16)
    log_l = 2 * (8 + np.log(vocab))                     # 2 U of the logarithm

    def of(zt):
        return U * (in_l + log_l + (m[:, 0] - zt + 8) + np.abs(zt - m[:, 0] - np.log(total[:, 0])))

    return of, U * (in_l * (1 + a + 8) + in_t + log_l + a + 8 + np.log(vocab))


def compare_closely(x, tokens, n_top, dt):
    z = R.f64(x)
    lp, ent, rank, ids, tops = run(x, tokens, n_top)
    rlp, rent, rrank, rids, rtops = R.logprobs(z, tokens.cpu().numpy(), n_top)
    of, entropy = bounds(z, tokens, dt)
    assert np.array_equal(rank.cpu().numpy(), rrank) and np.array_equal(ids.cpu().numpy(), rids)
    at = np.arange(len(z))
    assert (np.abs(R.f64(lp) - rlp) <= of(z[at, tokens.cpu().numpy()])).all()
    for i in range(n_top):
        assert (np.abs(R.f64(tops)[:, i] - rtops[:, i]) <= of(z[at, rids[:, i]])).all()
    assert (np.abs(R.f64(ent) - rent) <= entropy).all(), (R.f64(ent) - rent, entropy)
    assert (lp <= 0).all() and (tops <= 0).all() and (ent >= 0).all()
    return R.f64(lp) - rlp, R.f64(tops) - rtops, R.f64(ent) - rent


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab,top", [
    (16, 151936, 20), (511, 700, 3), (512, 5000, 5), (513, 5000, 5), (600, 9001, 20), (1, 50257, 64)])
def test_errors_of_ordinary_rows(dt, n, vocab, top):
    """Each value within its bound, and, where there are many, in the mean square:
    log l, the difference and the result round to a step of at most 2^-20 (values
    of 8 to 16), half of it at most, a third of that squared on the average, and a
    chain of up to 100 roundings of a sum is off by sqrt(100 / 3) U at random: 4e-7
    together; the exponential's own 2 U may be the same for all values."""
    print("ordinary", dt, n, vocab, top, flush=True)
    lp, tops, ent = compare_closely(logits(n, vocab, dt, n + vocab), tokens(n, vocab, n), top, dt)
    if n > 500:
        assert np.sqrt((lp ** 2).mean()) <= 2.0 ** -20
        assert np.sqrt((tops ** 2).mean()) <= 2.0 ** -20
        # t / l is up to 16 from a reference, its two sums as above
        assert np.sqrt((ent ** 2).mean()) <= 2.0 ** -18


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [4999, 151936])
@pytest.mark.parametrize("where", ["first", "middle", "last"])
def test_errors_of_rows_with_one_likely_token(dt, vocab, where):
    """One token 4 to 30 above the rest.  From 12 on the rest is more than 8 below
    it, so the row's reference is that token, its weight is 1 without an error, and
    the entropy, log(1 + s) + sum p d, is a sum of terms above 0: within (6 d + 64
    + chain) U of itself, twice (weights and their sums), but that s is lost in
    1 + s where it lies below the roundings of the sums of which 1 is a term."""
    print("likely", dt, vocab, where, flush=True)
    gaps = [4, 5, 6, 7, 8, 9, 10, 12, 13, 14, 16, 18, 20, 24, 30]
    g = torch.Generator("cuda").manual_seed(vocab)
    x = (-2.0 - torch.rand(len(gaps), vocab, generator=g, device="cuda")).to(R.DT[dt])
    at = {"first": 0, "middle": vocab // 2, "last": vocab - 1}[where]
    x[:, at] = torch.tensor(gaps, device="cuda").to(x.dtype) - 2.0
    t = torch.full((len(gaps),), at, dtype=torch.int32, device="cuda")
    t[::3] = 7 if at != 7 else 8
    _, _, ent = compare_closely(x, t, 5, dt)
    z, c = R.f64(x), chain(vocab, dt)
    ref = R.logprobs(z, t.cpu().numpy(), 0)[1]
    for i, gap in enumerate(gaps):
        if gap >= 12:
            rest = np.exp(np.delete(z[i], at) - z[i, at]).sum()
            allowed = 2 * U * (6 * (gap + 1) + 64 + c) * ref[i] + min(rest, (c + 16) * U)
            assert abs(ent[i]) <= allowed, (gap, ent[i], ref[i], allowed)
