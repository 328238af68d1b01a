"""The paged-cache calls on the GPU -- append, attention over all pages and over
selected ones, selection -- against their 64-bit definitions, at the sizes,
masks and lists where they can go wrong."""
import copy

import numpy as np
import pytest
import torch

import paged_ref as R

wf = pytest.importorskip("paper_2606_07710_amd")
pytestmark = pytest.mark.gpu

BASE = 1e6


def say(*a):
    print(*a, flush=True)


def check(got, ref, err, what=""):
    got = R.f64(got)
    nan = np.isnan(ref)
    bad = ~(np.abs(got - ref) <= err) & ~nan
    assert not bad.any(), (what, np.argwhere(bad)[:4].tolist(), got[bad][:4], ref[bad][:4],
                           err[bad][:4])


# ---- append ------------------------------------------------------------------

def expected_append(rnd, positions, k0, v0, b0, q):
    k, v, bounds = R.f64(k0), R.f64(v0), R.f64(b0)
    ek = np.zeros(k.shape)
    out = np.full(q.shape, np.nan)
    eq = np.zeros(q.shape)
    touched = []
    for b, (rows, ctx) in enumerate(rnd.lens):
        for i in range(rows):
            r, slot = rnd.start[b] + i, ctx + i
            pos = slot if positions is None else int(positions[r])
            out[r] = R.rotate(R.f64(q[r]), pos, BASE)
            eq[r] = R.rotation_error(R.f64(q[r]), out[r], rnd.dt)
            p = int(rnd.table[b, slot // rnd.page])
            if not 0 <= p < k.shape[0]:
                continue
            x = R.f64(rnd.new_k[r])
            k[p, :, slot % rnd.page] = R.rotate(x, pos, BASE)
            ek[p, :, slot % rnd.page] = R.rotation_error(x, k[p, :, slot % rnd.page], rnd.dt)
            v[p, :, slot % rnd.page] = R.f64(rnd.new_v[r])
            touched.append((p, slot // rnd.page, b))
    return k, ek, v, out, eq, sorted(set(touched))


APPENDS = [
    # lens, page, hq, hkv, dh, dt, tree positions, pad
    ([(1, 0)], 16, 8, 2, 64, "bf16", False, 0),
    ([(1, 15), (1, 16), (1, 17), (0, 9)], 16, 8, 2, 128, "bf16", False, 1),
    ([(5, 30), (0, 0), (40, 3), (64, 100)], 32, 16, 2, 128, "bf16", True, 3),
    ([(333, 0), (7, 61)], 64, 4, 4, 64, "bf16", False, 0),
    ([(130, 127), (1, 500)], 128, 6, 2, 128, "f32", False, 2),
    ([(3, 40), (70, 5)], 16, 3, 1, 64, "f32", True, 0),
    ([(2, 100000), (1, 65535)], 64, 8, 1, 128, "f32", False, 0),
    ([(1, i) for i in range(300)], 16, 2, 1, 64, "bf16", False, 0),
    ([(128, 256), (5, 250), (100, 77)], 128, 8, 4, 128, "bf16", False, 0),
    ([(2, 33)], 32, 80, 1, 128, "bf16", False, 0),
    ([(1, 7 * i % 50) if i % 9 == 4 else (0, 3) for i in range(1024)], 16, 2, 2, 64, "f32", False, 0),
]


@pytest.mark.parametrize("case", range(len(APPENDS)))
def test_append(case):
    lens, page, hq, hkv, dh, dt, tree, pad = APPENDS[case]
    say("append", APPENDS[case][1:], len(lens))
    rnd = R.Round(lens, page, hq, hkv, dh, dt, pad, seed=case).on_gpu()
    g = torch.Generator().manual_seed(case)
    positions = torch.randint(0, 200000, (rnd.n,), generator=g).int() if tree else None
    # one fused projection: rows strided alike
    qkv = torch.cat([rnd.q.flatten(1), rnd.new_k.flatten(1), rnd.new_v.flatten(1)], 1).cuda()
    q = qkv[:, : hq * dh].view(rnd.n, hq, dh)
    nk = qkv[:, hq * dh: (hq + hkv) * dh].view(rnd.n, hkv, dh)
    nv = qkv[:, (hq + hkv) * dh:].view(rnd.n, hkv, dh)
    out = torch.full((rnd.n, hq, dh), 7.0, dtype=R.DT[dt], device="cuda")
    wf.wf_paged_append(nk, nv, rnd.cache, rnd.batch, BASE, q=q, q_out=out,
                       positions=None if positions is None else positions.cuda())
    torch.cuda.synchronize()
    k, ek, v, qo, eq, touched = expected_append(rnd, positions, rnd.k, rnd.v, rnd.bounds, rnd.q)
    check(rnd.dk, k, ek, "k")
    assert np.array_equal(R.f64(rnd.dv), v)
    check(out, qo, eq, "q")
    assert (R.f64(out)[np.isnan(qo)] == 7.0).all()          # rows of no sequence
    # the bounds are those of the stored keys, other pages' stay
    ref = rnd.bounds.clone()
    stored = rnd.dk.cpu()
    for p, lp, b in touched:
        rows, ctx = lens[b]
        x = stored[p, :, : min(page, ctx + rows - lp * page)]
        ref[p, :, 0], ref[p, :, 1] = x.amin(1), x.amax(1)
    assert torch.equal(rnd.db.cpu(), ref)


def test_append_without_q_or_bounds_in_place_and_missing_pages():
    rnd = R.Round([(20, 10), (3, 50), (2, 0)], 16, 4, 2, 64, seed=3).on_gpu(with_bounds=False)
    rnd.table[0, 1] = -1                       # positions 16 .. 31 of sequence 0
    rnd.table[1, 3] = rnd.k.shape[0]           # and those of sequence 1's new rows
    rnd.batch.page_table.copy_(rnd.table)
    wf.wf_paged_append(rnd.new_k.cuda(), rnd.new_v.cuda(), rnd.cache, rnd.batch, BASE)
    k, ek, v, _, _, _ = expected_append(rnd, None, rnd.k, rnd.v, rnd.bounds, rnd.q)
    check(rnd.dk, k, ek)
    assert np.array_equal(R.f64(rnd.dv), v)
    # q in place
    q = rnd.q.cuda()
    wf.wf_paged_append(rnd.new_k.cuda(), rnd.new_v.cuda(), rnd.cache, rnd.batch, BASE, q=q, q_out=q)
    _, _, _, qo, eq, _ = expected_append(rnd, None, rnd.k, rnd.v, rnd.bounds, rnd.q)
    check(q, qo, eq)


def test_append_bounds_follow_a_rollback_and_keep_nan():
    rnd = R.Round([(4, 20)], 16, 4, 2, 64, seed=5).on_gpu()
    big = rnd.new_k.clone()
    big *= 100
    wf.wf_paged_append(big.cuda(), rnd.new_v.cuda(), rnd.cache, rnd.batch, BASE)
    p = int(rnd.table[0, 1])
    wide = rnd.db[p].clone()
    # two of the four rows stay, other two come: the large ones leave no trace
    small = rnd.new_k.clone()
    small[:, 0, 3] = float("nan")
    wf.wf_paged_append(small.cuda(), rnd.new_v.cuda(), rnd.cache, rnd.batch, BASE)
    x = rnd.dk.cpu()[p, :, :8]
    ref = torch.stack([x.amin(1), x.amax(1)], 1)
    assert torch.equal(rnd.db[p].cpu().isnan(), ref.isnan()) and ref.isnan().any()
    assert torch.equal(rnd.db[p].cpu().nan_to_num(0.0), ref.nan_to_num(0.0))
    assert (wide[:, 1] > rnd.db[p][:, 1].nan_to_num(-1e9)).any()


# ---- attention -----------------------------------------------------------------

ATTN = [
    # lens, page, hq, hkv, dh, dt, tree, pad
    ([(1, 0)], 16, 8, 2, 64, "bf16", False, 0),
    ([(1, 1003)], 64, 32, 8, 128, "bf16", False, 0),
    ([(1, 127), (1, 128), (1, 129), (0, 50), (1, 0), (1, 63)], 16, 8, 2, 128, "bf16", False, 2),
    ([(4, 31), (3, 32), (4, 33), (2, 700)], 32, 8, 2, 128, "bf16", False, 0),
    ([(8, 200), (5, 0), (8, 511)], 16, 8, 2, 128, "bf16", False, 1),
    ([(16, 300), (9, 1000), (0, 0), (16, 5)], 64, 16, 4, 128, "bf16", False, 3),
    ([(64, 90), (33, 400), (1, 1)], 16, 8, 1, 64, "bf16", False, 0),
    ([(61, 500), (20, 33)], 16, 8, 2, 128, "bf16", True, 0),
    ([(64, 0), (3, 200)], 128, 4, 2, 64, "bf16", True, 1),
    ([(7, 60), (2, 17)], 16, 4, 2, 128, "bf16", True, 0),
    ([(1, 300)], 16, 40, 1, 128, "bf16", False, 0),
    ([(2, 3000)], 16, 7, 7, 64, "bf16", False, 0),
    ([(1, 5 * i) for i in range(90)], 16, 4, 2, 64, "bf16", False, 0),
    ([(8, 256)], 16, 8, 2, 64, "f32", False, 0),
    ([(5, 40), (1, 0), (16, 200)], 32, 8, 2, 128, "f32", False, 1),
    ([(30, 100), (7, 15)], 16, 4, 1, 64, "f32", True, 0),
    ([(1 if i % 3 else 2, i % 40) for i in range(700)], 16, 2, 1, 64, "bf16", False, 0),
    ([(3, 20) if i in (0, 500, 1023) else (0, i) for i in range(1024)], 32, 8, 2, 128, "bf16", True, 5),
    ([(40, 700), (1, 3)], 128, 24, 8, 128, "bf16", False, 0),
    ([(64, 64), (2, 500)], 64, 64, 2, 64, "bf16", False, 0),
]


def trees(rnd, seed):
    rng = np.random.default_rng(seed)
    words = []
    for rows, _ in rnd.lens:
        if rows:
            words += R.random_tree(rng, rows)
    return words + [0] * (rnd.n - len(words))


@pytest.mark.parametrize("case", range(len(ATTN)))
def test_attention(case):
    lens, page, hq, hkv, dh, dt, tree, pad = ATTN[case]
    say("attention", ATTN[case][1:], len(lens))
    rnd = R.Round(lens, page, hq, hkv, dh, dt, pad, seed=100 + case).on_gpu()
    words = trees(rnd, case) if tree else None
    out = torch.full_like(rnd.dq, 7.0)
    wf.wf_paged_verify_attn(rnd.dq, rnd.cache, rnd.batch, out,
                            tree_mask=R.masks64(words) if tree else None)
    torch.cuda.synchronize()
    ref, err = R.attention(rnd, words)
    check(out, ref, err)
    assert (R.f64(out)[np.isnan(ref)] == 7.0).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_attention_of_missing_pages_and_broken_lists(dt):
    rnd = R.Round([(2, 100), (3, 40), (2, 16), (1, 200), (2, 5)], 16, 8, 2, 64, dt, seed=7).on_gpu()
    rnd.table[0, 2] = -1
    rnd.table[1, 1] = 1 << 30
    rnd.table[2, :] = -5                       # nothing to see: zeros
    rnd.table[3, 12] = -1                      # the row's own page
    rnd.batch.page_table.copy_(rnd.table)
    out = torch.full_like(rnd.dq, 7.0)
    ws = wf.alloc_workspace(wf.wf_paged_verify_attn_workspace_bytes(
        rnd.dq.dtype, rnd.n, 5, rnd.max_rows, 8, 2, 64), "cuda")
    wf.wf_paged_verify_attn(rnd.dq, rnd.cache, rnd.batch, out, workspace=ws)
    ref, err = R.attention(rnd)
    check(out, ref, err)
    assert (R.f64(out)[rnd.start[2]:rnd.start[3]] == 0).all()
    # a context that does not fit, a negative one, too many rows: skipped, the
    # others as before
    for b, c in ((0, 2000), (1, -1), (3, 1 << 30)):
        ctx = rnd.ctx.clone()
        ctx[b] = c
        rnd.batch.ctx_len.copy_(ctx)
        part = torch.full_like(rnd.dq, 7.0)
        wf.wf_paged_verify_attn(rnd.dq, rnd.cache, rnd.batch, part, workspace=ws)
        mine = slice(rnd.start[b], rnd.start[b + 1])
        assert (part[mine] == 7.0).all()
        keep = torch.ones(rnd.n, dtype=torch.bool)
        keep[mine] = False
        assert torch.equal(part[keep.cuda()], out[keep.cuda()])
    rnd.batch.ctx_len.copy_(rnd.ctx)
    for start in ([0, 2, 5, 4, 8, 10], [0, 2, 5, 7, 8, 11], [-1, 2, 5, 7, 8, 10],
                  [0, 2, 6, 7, 8, 10]):
        rnd.batch.row_start.copy_(torch.tensor(start, dtype=torch.int32))
        part = torch.full_like(rnd.dq, 7.0)
        wf.wf_paged_verify_attn(rnd.dq, rnd.cache, rnd.batch, part, workspace=ws)
        torch.cuda.synchronize()
        assert part.isfinite().all()
    assert not ws[: 4 << 20].any()


def test_attention_large_scores_and_infinities():
    rnd = R.Round([(4, 70), (2, 33)], 16, 4, 2, 64, seed=9, std=1.0)
    rnd.q *= 2.0 ** 20                         # scores of 2^20 and more
    rnd.on_gpu()
    out = torch.empty_like(rnd.dq)
    wf.wf_paged_verify_attn(rnd.dq, rnd.cache, rnd.batch, out)
    ref, err = R.attention(rnd)
    # weights are one-hot but where scores are close: compare by the allowed error
    check(out, ref, np.minimum(err, 8.0))
    # a NaN key reaches every row that sees it, and no other sequence
    p = int(rnd.table[0, 0])
    rnd.dk[p, 1, 3, 5] = float("nan")
    wf.wf_paged_verify_attn(rnd.dq, rnd.cache, rnd.batch, out)
    assert out[:4, 2:].isnan().all() and out[:4, :2].isfinite().all() and out[4:].isfinite().all()


def test_keys_behind_the_batch_are_not_read():
    """Whatever lies behind the newest position of a page stays out of it."""
    rnd = R.Round([(3, 70), (1, 17)], 16, 8, 2, 64, seed=11).on_gpu()
    out = torch.empty_like(rnd.dq)
    wf.wf_paged_verify_attn(rnd.dq, rnd.cache, rnd.batch, out)
    sel = torch.tensor([[[0, 4, 1, 2, 3, -1]] * 2] * 3 + [[[0, 1, -1, -1, -1, -1]] * 2],
                       dtype=torch.int32, device="cuda")
    some = torch.empty_like(rnd.dq)
    wf.wf_paged_sparse_attn(rnd.dq, rnd.cache, rnd.batch, sel, some)
    for b, (rows, ctx) in enumerate(rnd.lens):
        p = int(rnd.table[b, (ctx + rows - 1) // 16])
        rnd.dk[p, :, (ctx + rows - 1) % 16 + 1:] = float("nan")
        rnd.dv[p, :, (ctx + rows - 1) % 16 + 1:] = float("inf")
    used = [p for b, (r, c) in enumerate(rnd.lens) for p in rnd.table[b, : -(-(r + c) // 16)].tolist()]
    for p in set(range(rnd.k.shape[0])) - set(used):
        rnd.dk[p], rnd.dv[p] = float("nan"), float("nan")
    again = torch.empty_like(rnd.dq)
    wf.wf_paged_verify_attn(rnd.dq, rnd.cache, rnd.batch, again)
    assert torch.equal(out, again)
    wf.wf_paged_sparse_attn(rnd.dq, rnd.cache, rnd.batch, sel, again)
    assert torch.equal(some, again)


# ---- selection ------------------------------------------------------------------

SELECTS = [
    # lens, page, hq, hkv, dh, dt, n_sel, n_recent, spare, pad
    ([(1, 1000)], 16, 8, 2, 64, "bf16", 12, 2, 0, 0),
    ([(3, 700), (0, 90), (2, 40), (1, 0), (4, 15)], 16, 8, 2, 128, "bf16", 9, 1, 500, 2),
    ([(4, 3000), (2, 2900)], 32, 16, 2, 64, "f32", 40, 4, 0, 0),
    ([(1, 500), (2, 260)], 64, 4, 1, 128, "f32", 3, 3, 3, 1),
    ([(2, 800)], 128, 7, 7, 64, "bf16", 1024, 1, 0, 0),
    ([(1, 40000)], 16, 4, 2, 64, "bf16", 700, 1, 0, 0),
    ([(1, 20 * i) for i in range(70)], 16, 40, 1, 64, "bf16", 5, 2, 0, 0),
]


@pytest.mark.parametrize("case", range(len(SELECTS)))
def test_select(case):
    lens, page, hq, hkv, dh, dt, n_sel, n_recent, spare, pad = SELECTS[case]
    say("select", SELECTS[case][1:], len(lens))
    rnd = R.Round(lens, page, hq, hkv, dh, dt, pad, seed=200 + case, spare=spare).on_gpu()
    sel = torch.full((rnd.n, hkv, n_sel), -7, dtype=torch.int32, device="cuda")
    ws = wf.alloc_workspace(wf.wf_paged_select_workspace_bytes(rnd.n, hkv, rnd.table.shape[1]),
                            "cuda")
    for _ in range(2):
        wf.wf_paged_select(rnd.dq, rnd.cache, rnd.batch, sel, n_recent, workspace=ws)
        assert np.array_equal(sel.cpu().numpy(), R.select(rnd, n_sel, n_recent))
    assert not ws[: 4 << 20].any()


def test_select_ties_missing_pages_and_nan():
    rnd = R.Round([(2, 640)], 16, 4, 2, 64, seed=31)
    rnd.bounds[:] = rnd.bounds[:1]             # all scores equal
    rnd.table[0, 3] = -1
    rnd.table[0, 5] = rnd.k.shape[0]
    rnd.on_gpu()
    sel = torch.empty((2, 2, 9), dtype=torch.int32, device="cuda")
    wf.wf_paged_select(rnd.dq, rnd.cache, rnd.batch, sel, 2)
    assert np.array_equal(sel.cpu().numpy(), R.select(rnd, 9, 2))
    assert sel[0, 0].tolist() == [0, 1, 2, 4, 6, 7, 8, 39, 40]
    # NaN first; infinite bounds; a zero q against them
    rnd.bounds[int(rnd.table[0, 30]), :, 1, 4] = float("nan")
    rnd.bounds[int(rnd.table[0, 30]), :, 0, 4] = float("nan")
    rnd.bounds[int(rnd.table[0, 20]), :, 1] = float("inf")
    rnd.bounds[int(rnd.table[0, 20]), :, 0] = -float("inf")
    rnd.db.copy_(rnd.bounds)
    wf.wf_paged_select(rnd.dq, rnd.cache, rnd.batch, sel, 2)
    assert np.array_equal(sel.cpu().numpy(), R.select(rnd, 9, 2))
    assert 30 in sel[0, 0].tolist() and 20 in sel[0, 0].tolist()
    # fewer pages with an entry than there are places
    rnd.table[0, 6:39] = -1
    rnd.batch.page_table.copy_(rnd.table)
    wf.wf_paged_select(rnd.dq, rnd.cache, rnd.batch, sel, 2)
    assert sel[1, 1].tolist() == [0, 1, 2, 4, 39, 40, -1, -1, -1]


@pytest.mark.parametrize("dt,dh", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_select_of_queries_that_are_not_finite(dt, dh):
    """Such a query makes every page's score of its own row and group odd (the
    first pages are chosen), and nobody else's; signed zeros and the type's
    largest numbers are scores like others."""
    rnd = R.Round([(6, 900), (1, 400)], 16, 8, 2, dh, dt, seed=67)
    inf, nan, big = float("inf"), float("nan"), torch.finfo(rnd.q.dtype).max
    rnd.q[0, 1, 3] = inf
    rnd.q[1, 6, dh - 1] = -inf
    rnd.q[2, 0, 0], rnd.q[2, 7, 9] = nan, -nan
    rnd.q[3, :, ::2] = -0.0
    rnd.q[4, 2, 5], rnd.q[4, 5, 6] = big, -big
    rnd.q[5] = 0.0
    rnd.on_gpu()
    sel = torch.empty((rnd.n, 2, 11), dtype=torch.int32, device="cuda")
    wf.wf_paged_select(rnd.dq, rnd.cache, rnd.batch, sel, 2)
    got = sel.cpu().numpy()
    assert np.array_equal(got, R.select(rnd, 11, 2))
    assert got[0, 0, :9].tolist() == list(range(9)) == got[1, 1, :9].tolist()
    assert got[0, 1, :9].tolist() != list(range(9)) != got[6, 0, :9].tolist()


# ---- attention over selected pages -------------------------------------------------

SPARSES = [
    # lens, page, hq, hkv, dh, dt, n_sel, n_recent, tree, pad
    ([(1, 1000)], 16, 8, 2, 64, "bf16", 12, 2, False, 0),
    ([(3, 700), (0, 90), (2, 40), (1, 0), (4, 15)], 16, 8, 2, 128, "bf16", 9, 1, False, 2),
    ([(4, 600), (9, 130)], 32, 16, 2, 64, "f32", 7, 2, True, 0),
    ([(1, 500), (2, 260)], 64, 4, 1, 128, "f32", 3, 3, False, 1),
    ([(2, 800)], 128, 7, 7, 64, "bf16", 20, 1, False, 0),
    ([(12, 300)], 16, 40, 1, 128, "bf16", 6, 2, True, 0),
]


@pytest.mark.parametrize("case", range(len(SPARSES)))
def test_sparse_attention(case):
    lens, page, hq, hkv, dh, dt, n_sel, n_recent, tree, pad = SPARSES[case]
    say("sparse", SPARSES[case][1:], len(lens))
    rnd = R.Round(lens, page, hq, hkv, dh, dt, pad, seed=300 + case).on_gpu()
    sel = R.select(rnd, n_sel, n_recent)
    words = trees(rnd, case) if tree else None
    out = torch.full_like(rnd.dq, 7.0)
    wf.wf_paged_sparse_attn(rnd.dq, rnd.cache, rnd.batch, torch.tensor(sel).cuda(), out,
                            tree_mask=R.masks64(words) if tree else None)
    ref, err = R.attention(rnd, words, sel)
    check(out, ref, err)
    assert (R.f64(out)[np.isnan(ref)] == 7.0).all()


def test_sparse_attention_of_any_list():
    """Lists out of order, with holes, pages past the row's own, pages without
    an entry; a page listed twice counts twice; nothing listed gives zeros."""
    rnd = R.Round([(3, 100), (1, 60)], 16, 8, 2, 64, seed=41)
    rnd.table[0, 2] = -1
    rnd.on_gpu()
    sel = torch.full((4, 2, 7), -1, dtype=torch.int32)
    sel[0, 0] = torch.tensor([6, -1, 0, 1 << 30, 3, 2, -9])
    sel[0, 1] = torch.tensor([5, 4, 3, 2, 1, 0, 6])
    sel[1, 0] = torch.tensor([1, 1, -1, -1, -1, -1, 1])
    sel[3, 0] = torch.tensor([3, 4, 5, 6, 1, 0, -1])
    out = torch.empty_like(rnd.dq)
    wf.wf_paged_sparse_attn(rnd.dq, rnd.cache, rnd.batch, sel.cuda(), out)
    ref, err = R.attention(rnd, None, sel)
    check(out, ref, err)
    assert (out[1, 4:] == 0).all() and (out[2] == 0).all()


def test_sparse_of_all_pages_is_the_dense_attention():
    rnd = R.Round([(2, 100), (5, 30)], 16, 8, 2, 128, "f32", seed=43).on_gpu()
    sel = torch.empty((rnd.n, 2, 10), dtype=torch.int32, device="cuda")
    wf.wf_paged_select(rnd.dq, rnd.cache, rnd.batch, sel, 3)
    a, b = torch.empty_like(rnd.dq), torch.empty_like(rnd.dq)
    wf.wf_paged_verify_attn(rnd.dq, rnd.cache, rnd.batch, a)
    wf.wf_paged_sparse_attn(rnd.dq, rnd.cache, rnd.batch, sel, b)
    ref, err = R.attention(rnd)
    check(a, ref, err)
    check(b, ref, err)


# ---- how the calls are used ---------------------------------------------------------

def one_round(rnd, k, v, q, out, sel, some, ws, stream=None):
    rot = ws["rot"]
    wf.wf_paged_append(k, v, rnd.cache, rnd.batch, BASE, q=q, q_out=rot, stream=stream)
    wf.wf_paged_verify_attn(rot, rnd.cache, rnd.batch, out, workspace=ws["a"], stream=stream)
    wf.wf_paged_select(rot, rnd.cache, rnd.batch, sel, 2, workspace=ws["s"], stream=stream)
    wf.wf_paged_sparse_attn(rot, rnd.cache, rnd.batch, sel, some, workspace=ws["a"], stream=stream)


def setup_round(lens, dt="bf16", page=16, seed=0):
    rnd = R.Round(lens, page, 8, 2, 64, dt, seed=seed, spare=40, max_rows=16).on_gpu()
    n = rnd.n
    size = max(wf.wf_paged_verify_attn_workspace_bytes(rnd.dq.dtype, n, len(lens), 16, 8, 2, 64),
               wf.wf_paged_sparse_attn_workspace_bytes(rnd.dq.dtype, n, 8, 2, 64, page, 6))
    ws = dict(a=wf.alloc_workspace(size, "cuda"), rot=torch.zeros_like(rnd.dq),
              s=wf.alloc_workspace(wf.wf_paged_select_workspace_bytes(n, 2, rnd.table.shape[1]),
                                   "cuda"))
    io = dict(k=rnd.new_k.cuda(), v=rnd.new_v.cuda(), q=rnd.q.cuda(),
              out=torch.full_like(rnd.dq, 7.0), some=torch.full_like(rnd.dq, 7.0),
              sel=torch.full((n, 2, 6), -7, dtype=torch.int32, device="cuda"))
    return rnd, io, ws


def after(rnd, io):
    """The round's results against the definitions, from what is stored."""
    host = copy.copy(rnd)
    host.k, host.v, host.bounds = rnd.dk.cpu(), rnd.dv.cpu(), rnd.db.cpu()
    host.q = io["rot"].cpu()
    ref, err = R.attention(host)
    check(io["out"], ref, err, "dense")
    sel = R.select(host, 6, 2)
    assert np.array_equal(io["sel"].cpu().numpy(), sel)
    ref, err = R.attention(host, None, sel)
    check(io["some"], ref, err, "sparse")


def run_round(rnd, io, ws, stream=None):
    one_round(rnd, io["k"], io["v"], io["q"], io["out"], io["sel"], io["some"], ws, stream)
    io["rot"] = ws["rot"]


def test_a_round_together_and_on_a_side_stream():
    rnd, io, ws = setup_round([(4, 300), (16, 10), (1, 130), (9, 0)], seed=51)
    run_round(rnd, io, ws)
    after(rnd, io)
    first = {n: io[n].clone() for n in ("out", "sel", "some")}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for n in ("out", "sel", "some"):
        io[n].fill_(3)
    torch.cuda.synchronize()
    run_round(rnd, io, ws, stream=side)
    side.synchronize()
    for n, t in first.items():
        assert torch.equal(io[n], t), n


def test_captured_round_replays_with_other_lengths_and_pages():
    lens = [(4, 300), (16, 10), (1, 130)]
    rnd, io, ws = setup_round(lens, seed=53)
    run_round(rnd, io, ws)                     # first use outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run_round(rnd, io, ws)
    # the same buffers for later rounds: contexts move on, a sequence goes idle,
    # pages are handed out anew
    free = [p for p in range(rnd.k.shape[0]) if p not in rnd.table]
    for step, (new, starts) in enumerate([
            ([(4, 304), (16, 26), (1, 131)], None), ([(4, 290), (0, 42), (1, 5)], [0, 4, 4, 5]),
            ([(4, 308), (16, 0), (1, 132)], None)]):
        rnd.lens = new
        rnd.start = starts or [0, 4, 20, 21]
        rnd.ctx = torch.tensor([c for _, c in new], dtype=torch.int32)
        for b, (r, c) in enumerate(new):
            for p in range(-(-(r + c) // 16)):
                if int(rnd.table[b, p]) < 0 and free:
                    rnd.table[b, p] = free.pop()
        rnd.batch.ctx_len.copy_(rnd.ctx)
        rnd.batch.row_start.copy_(torch.tensor(rnd.start, dtype=torch.int32))
        rnd.batch.page_table.copy_(rnd.table)
        io["q"].normal_(generator=torch.Generator("cuda").manual_seed(step))
        for n in ("out", "some"):
            io[n].fill_(7.0)
        io["sel"].fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        after(rnd, io)
        got = {n: io[n].clone() for n in ("out", "sel", "some")}
        run_round(rnd, io, ws)                 # eager work between the replays
        torch.cuda.synchronize()
        for n, t in got.items():
            assert torch.equal(io[n], t), n


def test_results_repeat_and_stay_in_their_buffers():
    rnd, io, ws = setup_round([(16, 900), (3, 77), (8, 1200)], seed=57)
    n = rnd.n
    guard = torch.full((n + 2, 8, 64), 5.0, dtype=rnd.dq.dtype, device="cuda")
    need = wf.wf_paged_verify_attn_workspace_bytes(rnd.dq.dtype, n, 3, 16, 8, 2, 64)
    big = torch.zeros(need + 4096, dtype=torch.uint8, device="cuda")
    big[need:] = 0xa5
    runs = []
    for _ in range(3):
        wf.wf_paged_verify_attn(rnd.dq, rnd.cache, rnd.batch, guard[1:-1], workspace=big[:need])
        runs.append(guard.clone())
    assert torch.equal(runs[0], runs[1]) and torch.equal(runs[0], runs[2])
    assert (guard[0] == 5).all() and (guard[-1] == 5).all() and (big[need:] == 0xa5).all()
    assert not big[: 4 << 20].any()


def test_two_rounds_at_once_on_two_streams():
    """Two batches with workspaces of their own, launched side by side."""
    sets = [setup_round([(4, 900), (16, 300), (1, 130)], seed=71),
            setup_round([(9, 500), (2, 1000), (16, 44), (1, 2)], seed=72)]
    alone = []
    for rnd, io, ws in sets:
        run_round(rnd, io, ws)
        torch.cuda.synchronize()
        alone.append({n: io[n].clone() for n in ("out", "sel", "some")})
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for (rnd, io, ws), st in zip(sets, streams):
            run_round(rnd, io, ws, stream=st)
        torch.cuda.synchronize()
        for (rnd, io, ws), ref in zip(sets, alone):
            for n, t in ref.items():
                assert torch.equal(io[n], t), n


def test_select_of_broken_lists_stays_in_range():
    rnd = R.Round([(2, 640), (3, 900), (1, 320)], 16, 4, 2, 64, seed=73, max_rows=4).on_gpu()
    for start, ctx in (([0, 4, 2, 6], None), ([0, 2, 5, 9], None), ([0, 2, 5, 6], [640, -3, 1 << 29]),
                       ([3, 2, 1, 0], None)):
        rnd.batch.row_start.copy_(torch.tensor(start, dtype=torch.int32))
        rnd.batch.ctx_len.copy_(torch.tensor(ctx, dtype=torch.int32) if ctx else rnd.ctx)
        sel = torch.full((rnd.n, 2, 8), -7, dtype=torch.int32, device="cuda")
        wf.wf_paged_select(rnd.dq, rnd.cache, rnd.batch, sel, 2)
        assert ((sel >= -7) & (sel < rnd.table.shape[1])).all()
    # the sequences whose numbers hold are served as ever
    rnd.batch.row_start.copy_(torch.tensor([0, 2, 5, 6], dtype=torch.int32))
    rnd.batch.ctx_len.copy_(torch.tensor([640, -3, 320], dtype=torch.int32))
    wf.wf_paged_select(rnd.dq, rnd.cache, rnd.batch, sel.fill_(-7), 2)
    want = R.select(rnd, 8, 2)
    assert np.array_equal(sel.cpu().numpy()[[0, 1, 5]], want[[0, 1, 5]])
    assert (sel[2:5] == -7).all()


def test_copies_of_a_cache_have_their_own_memory():
    rnd = R.Round([(1, 20)], 16, 4, 2, 64, seed=61).on_gpu()
    other = copy.deepcopy(rnd.cache)
    wf.wf_paged_append(rnd.new_k.cuda(), rnd.new_v.cuda(), other, rnd.batch, BASE)
    assert torch.equal(rnd.dk.cpu(), rnd.k) and not torch.equal(other.k.cpu(), rnd.k)


def test_pages_past_32_bits():
    """A pool whose keys lie past 2^32 bytes, and past 2^31 elements."""
    n_pages = 16500                            # 128 x 8 x 128 x 2 bytes each: 4.3 GB
    k = torch.zeros((n_pages, 8, 128, 128), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    rnd = R.Round([(2, 300)], 128, 16, 8, 128, seed=63)
    for i, p in enumerate(rnd.table[0, :3].tolist()):
        k[n_pages - 1 - 40 * i], v[n_pages - 1 - 40 * i] = rnd.k[p].cuda(), rnd.v[p].cuda()
    far = torch.tensor([[n_pages - 1, n_pages - 41, n_pages - 81]], dtype=torch.int32)
    batch = wf.PagedBatch(far.cuda(), torch.tensor([0, 2], dtype=torch.int32).cuda(),
                          rnd.ctx.cuda(), 2)
    cache = wf.PagedCache(k, v)
    out = torch.empty_like(rnd.q, device="cuda")
    wf.wf_paged_verify_attn(rnd.q.cuda(), cache, batch, out)
    ref, err = R.attention(rnd)
    check(out, ref, err)
    sel = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda").repeat(2, 8, 1)
    wf.wf_paged_sparse_attn(rnd.q.cuda(), cache, batch, sel, out)
    check(out, ref, err)
    wf.wf_paged_append(rnd.new_k.cuda(), rnd.new_v.cuda(), cache, batch, BASE)
    want = R.rotate(R.f64(rnd.new_k), np.array([300, 301])[:, None, None], BASE)
    got = k[n_pages - 81, :, 300 - 256: 302 - 256].transpose(0, 1)
    check(got, want, R.rotation_error(R.f64(rnd.new_k), want, "bf16"))


def test_a_round_without_rows():
    """Every request idle: no tensor has a row, and every call of the round
    returns."""
    rnd = R.Round([(0, 30), (0, 0)], 16, 8, 2, 64, seed=99, max_rows=4).on_gpu()
    assert rnd.n == 0
    q, out = rnd.dq, torch.empty_like(rnd.dq)
    sel = torch.empty((0, 2, 5), dtype=torch.int32, device="cuda")
    kv = rnd.new_k.cuda()
    wf.wf_paged_append(kv, kv, rnd.cache, rnd.batch, BASE, q=q, q_out=out)
    wf.wf_paged_append(kv, kv, rnd.cache, rnd.batch, BASE)
    wf.wf_paged_verify_attn(q, rnd.cache, rnd.batch, out)
    wf.wf_paged_select(q, rnd.cache, rnd.batch, sel, 2)
    wf.wf_paged_sparse_attn(q, rnd.cache, rnd.batch, sel, out)
    torch.cuda.synchronize()
    assert torch.equal(rnd.dk.cpu(), rnd.k) and torch.equal(rnd.db.cpu(), rnd.bounds)


def test_append_of_lists_that_give_rows_twice():
    """Sequences whose own numbers hold are served, each in its pages, also where a
    decreasing row_start between them gives them the same rows; the others leave
    everything as it was."""
    say("append, rows given twice")
    n, ctx = 200, 5
    rnd = R.Round([(n, ctx)] * 8, 16, 4, 2, 64, seed=81).on_gpu()
    starts = [0, n] * 4 + [0]
    rnd.batch.row_start.copy_(torch.tensor(starts, dtype=torch.int32))
    q, new_k, new_v = (x[:n] for x in (rnd.q, rnd.new_k, rnd.new_v))
    out = torch.full((n, 4, 64), 7.0, dtype=q.dtype, device="cuda")
    wf.wf_paged_append(new_k.cuda(), new_v.cuda(), rnd.cache, rnd.batch, BASE, q=q.cuda(),
                       q_out=out)
    rnd.start, rnd.q = starts[:-1], q
    rnd.lens = [(n if b % 2 == 0 else 0, ctx) for b in range(8)]
    k, ek, v, qo, eq, touched = expected_append(rnd, None, rnd.k, rnd.v, rnd.bounds, q)
    assert len(touched) == 4 * 13
    check(rnd.dk, k, ek, "k")
    assert np.array_equal(R.f64(rnd.dv), v)
    check(out, qo, eq, "q")                    # (their rows are at the same positions)
    ref, stored = rnd.bounds.clone(), rnd.dk.cpu()
    for p, lp, b in touched:
        x = stored[p, :, : min(16, ctx + n - lp * 16)]
        ref[p, :, 0], ref[p, :, 1] = x.amin(1), x.amax(1)
    assert torch.equal(rnd.db.cpu(), ref)


@pytest.mark.parametrize("start,ctx,served", [
    ([0, 3, 7, 9], [30, -1, 40], [0, 2]), ([0, 3, 7, 9], [1 << 30, 20, 2000], [1]),
    ([-1, 3, 7, 9], None, [1, 2]), ([0, 3, 7, 10], None, [0, 1]), ([0, 3, 2, 9], None, [0, 2]),
    ([9, 7, 3, 0], None, []), ([0, 1 << 30, 7, 9], None, [2])])
def test_append_of_broken_lists(start, ctx, served):
    """Sequences whose numbers do not hold leave pages, bounds and q_out alone."""
    rnd = R.Round([(3, 30), (4, 20), (2, 40)], 16, 4, 2, 64, seed=83).on_gpu()
    rnd.batch.row_start.copy_(torch.tensor(start, dtype=torch.int32))
    if ctx:
        rnd.batch.ctx_len.copy_(torch.tensor(ctx, dtype=torch.int32))
    out = torch.full_like(rnd.dq, 7.0)
    # (rows that two sequences have are rotated by either's positions: without q)
    twice = start == [0, 3, 2, 9]
    wf.wf_paged_append(rnd.new_k.cuda(), rnd.new_v.cuda(), rnd.cache, rnd.batch, BASE,
                       **({} if twice else dict(q=rnd.dq, q_out=out)))
    torch.cuda.synchronize()
    lens = rnd.lens
    rnd.start = start[:-1]
    rnd.lens = [(start[b + 1] - start[b] if b in served else 0, c) for b, (_, c) in enumerate(lens)]
    if twice:
        # five rows more than its pages were made for fit them all the same
        assert rnd.lens[2] == (7, 40)
    k, ek, v, qo, eq, touched = expected_append(rnd, None, rnd.k, rnd.v, rnd.bounds, rnd.q)
    check(rnd.dk, k, ek, "k")
    assert np.array_equal(R.f64(rnd.dv), v)
    if not twice:
        check(out, qo, eq, "q")
        assert (R.f64(out)[np.isnan(qo)] == 7.0).all()
    pages = {p for p, _, _ in touched}
    rest = [p for p in range(rnd.k.shape[0]) if p not in pages]
    assert torch.equal(rnd.db.cpu()[rest], rnd.bounds[rest])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("lens,tree", [
    ([(4, 70), (2, 33)], False), ([(61, 300), (1, 1500)], True), ([(16, 900), (1, 40)], False),
    ([(1, 2000)], False), ([(2, 2000)], False)])
def test_attention_of_large_whole_numbers(dt, lens, tree):
    """Scores of up to 2^27, of whole numbers: every sum of products is exact, two
    scores are equal or at least 2^17 apart, so the weights are 1 for the largest
    score's keys and 0 for the others, and the output is the mean of those keys'
    values, off by its fp32 sum and its own rounding."""
    say("large whole numbers", dt, lens, tree)
    rnd = R.Round(lens, 16, 8, 2, 64, dt, seed=91)
    g = torch.Generator().manual_seed(92)
    whole = lambda t: torch.randint(-3, 4, t.shape, generator=g).to(t.dtype)  # noqa: E731
    rnd.k, rnd.q = whole(rnd.k), whole(rnd.q) * 2.0 ** 20
    rnd.q[0] = 0.0                             # every key alike
    rnd.on_gpu()
    words = trees(rnd, 93) if tree else None
    mask = R.masks64(words) if tree else None
    out = torch.full_like(rnd.dq, 7.0)
    wf.wf_paged_verify_attn(rnd.dq, rnd.cache, rnd.batch, out, tree_mask=mask)
    keys = max(r + c for r, c in lens)
    sums = (keys + 8) * 2.0 ** -24 * float(rnd.v.abs().max())
    ref, _ = R.attention(rnd, words)
    check(out, ref, np.abs(ref) * (R.HALF_STEP[dt] + 2.0 ** -22) + sums, "dense")
    assert rnd.n == 1 or np.abs(ref).max() > 1
    # every second page
    n_pages = -(-keys // 16)
    sel = torch.full((rnd.n, 2, n_pages), -1, dtype=torch.int32)
    sel[:, :, ::2] = torch.arange(0, n_pages, 2, dtype=torch.int32)
    some = torch.full_like(rnd.dq, 7.0)
    wf.wf_paged_sparse_attn(rnd.dq, rnd.cache, rnd.batch, sel.cuda(), some, tree_mask=mask)
    ref, _ = R.attention(rnd, words, sel)
    check(some, ref, np.abs(ref) * (R.HALF_STEP[dt] + 2.0 ** -22) + sums, "selected")


@pytest.mark.parametrize("lens,tree", [
    ([(1, 3000)] * 4, False), ([(16, 900), (16, 1500)], False), ([(61, 1200)], True)])
def test_attention_error_in_the_mean_square(lens, tree):
    """bf16: a rounding at random to 8 bits is off by 2^-8 / sqrt(3) at the foot of
    a binade and by sqrt(3 / (8 ln 2)) = 0.7355 of that over numbers spread evenly
    over their logarithm: 0.00166.  The output has one such rounding, and every
    weight one before its product with V; nothing else is held in 16 bits.  A
    tenth for distributions that are not quite that; partial rows in bf16, one
    rounding more, would be a sixth above."""
    say("mean square", lens, tree)
    rnd = R.Round(lens, 32, 8, 2, 128, "bf16", seed=95, std=1.1).on_gpu()
    words = trees(rnd, 96) if tree else None
    mask = R.masks64(words) if tree else None
    ref, _ = R.attention(rnd, words)
    # what the weights' roundings come to: sqrt(sum (p v)^2), element by element
    parts = np.zeros_like(ref)
    k, v, q = R.f64(rnd.k), R.f64(rnd.v), R.f64(rnd.q)
    for b, (rows, ctx) in enumerate(lens):
        for i in range(rows):
            at = R.visible(rnd, b, i, words)
            ids = rnd.table[b].numpy()[at // 32]
            for h in range(8):
                kk, vv = k[ids, h // 4, at % 32], v[ids, h // 4, at % 32]
                z = kk @ q[rnd.start[b] + i, h] * 128 ** -0.5
                w = np.exp(z - z.max())
                w /= w.sum()
                parts[rnd.start[b] + i, h] = np.sqrt((w * w) @ (vv * vv))
    step = 2.0 ** -8 / 3 ** 0.5 * 0.7355
    allowed = 1.1 * step * np.sqrt((ref ** 2).mean() + (parts ** 2).mean())
    n_pages = rnd.table.shape[1]
    every = torch.arange(n_pages, dtype=torch.int32).repeat(rnd.n, 2, 1).cuda()
    for what in ("dense", "selected"):
        out = torch.full_like(rnd.dq, 7.0)
        if what == "dense":
            wf.wf_paged_verify_attn(rnd.dq, rnd.cache, rnd.batch, out, tree_mask=mask)
        else:
            wf.wf_paged_sparse_attn(rnd.dq, rnd.cache, rnd.batch, every, out, tree_mask=mask)
        error = np.sqrt(((R.f64(out) - ref) ** 2).mean())
        say(what, error / np.sqrt((ref ** 2).mean()), allowed / np.sqrt((ref ** 2).mean()))
        assert error <= allowed, (what, error, allowed)


def test_an_accepted_tree_path_is_appended_again():
    """A draft tree's rows lie in their order in the tree.  The path that is
    accepted becomes the cache by being appended from the old context on: pages,
    bounds and what later rows see of them are those of a cache that never held
    the rest of the tree."""
    say("accepted path")
    ctx, rows, path = 57, 12, [0, 3, 4, 8, 11, 6, 9]      # over the end of a page of 16
    rnd = R.Round([(rows, ctx)], 16, 4, 2, 64, seed=97).on_gpu()
    alone = R.Round([(rows, ctx)], 16, 4, 2, 64, seed=97).on_gpu()
    one = dict(dtype=torch.int32, device="cuda")
    depth = torch.arange(rows, **one) // 2 + ctx
    k, v = rnd.new_k.cuda(), rnd.new_v.cuda()
    wf.wf_paged_append(k, v, rnd.cache, rnd.batch, BASE, positions=depth)
    n = len(path)
    for r in (rnd, alone):
        again = wf.PagedBatch(r.batch.page_table, torch.tensor([0, n], **one),
                              torch.tensor([ctx], **one), 64)
        wf.wf_paged_append(k[path], v[path], r.cache, again, BASE)
    new = ctx + n                              # positions up to there count
    pages = rnd.table[0, : -(-new // 16)].tolist()
    assert new % 16 == 0 and torch.equal(rnd.db[pages], alone.db[pages])
    assert torch.equal(rnd.dk[pages], alone.dk[pages]) and torch.equal(rnd.dv[pages], alone.dv[pages])
    out, sel = [], []
    for r in (rnd, alone):
        later = wf.PagedBatch(r.batch.page_table, torch.tensor([0, 2], **one),
                              torch.tensor([new], **one), 2)
        wf.wf_paged_append(k[:2], v[:2], r.cache, later, BASE)
        sel.append(torch.empty((2, 2, 3), **one))
        wf.wf_paged_select(rnd.dq[:2], r.cache, later, sel[-1], 1)
        out.append(torch.empty_like(rnd.dq[:2]))
        wf.wf_paged_verify_attn(rnd.dq[:2], r.cache, later, out[-1])
    assert torch.equal(*out) and torch.equal(*sel)
