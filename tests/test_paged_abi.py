"""What the paged-cache calls and the token log probabilities refuse, on the
CPU: no call here reaches the GPU (pointers are never dereferenced by the
checks), and what their Python wrappers refuse before the library is called."""
import copy
import ctypes

import pytest
import torch

wf = pytest.importorskip("paper_2606_07710_amd")

FAKE, ODD, ODD4 = 1 << 20, (1 << 20) + 8, (1 << 20) + 2
BIG = 1 << 40


def _cache(**kw):
    a = dict(k=FAKE, v=FAKE, bounds=FAKE, n=100, page=64, hkv=8, dh=128)
    a.update(kw)
    if a.get("none"):
        return None
    return ctypes.byref(wf.PagedCacheStruct(a["k"], a["v"], a["bounds"], a["n"], a["page"],
                                            a["hkv"], a["dh"]))


def _batch(**kw):
    a = dict(table=FAKE, start=FAKE, ctx=FAKE, n=4, pages=20, rows=16)
    a.update(kw)
    if a.get("none"):
        return None
    return ctypes.byref(wf.PagedBatchStruct(a["table"], a["start"], a["ctx"], a["n"], a["pages"],
                                            a["rows"]))


def _append(cache={}, batch={}, **kw):
    a = dict(dt=1, k=FAKE, v=FAKE, ks=1024, q=FAKE, qs=4096, qo=FAKE, hq=32, pos=None, base=1e6,
             n=8)
    a.update(kw)
    return wf.lib.wf_paged_append(a["dt"], _cache(**cache), _batch(**batch), a["k"], a["v"],
                                  a["ks"], a["q"], a["qs"], a["qo"], a["hq"], a["pos"], a["base"],
                                  a["n"], None)


def _attn(cache={}, batch={}, **kw):
    a = dict(dt=1, q=FAKE, out=FAKE, mask=None, n=8, hq=32, scale=0.1, ws=FAKE, wsb=BIG)
    a.update(kw)
    return wf.lib.wf_paged_verify_attn(a["dt"], a["q"], _cache(**cache), _batch(**batch), a["out"],
                                       a["mask"], a["n"], a["hq"], a["scale"], a["ws"], a["wsb"],
                                       None)


def _select(cache={}, batch={}, **kw):
    a = dict(dt=1, q=FAKE, sel=FAKE, ns=10, nr=2, n=8, hq=32, ws=FAKE, wsb=BIG)
    a.update(kw)
    return wf.lib.wf_paged_select(a["dt"], a["q"], _cache(**cache), _batch(**batch), a["sel"],
                                  a["ns"], a["nr"], a["n"], a["hq"], a["ws"], a["wsb"], None)


def _sparse(cache={}, batch={}, **kw):
    a = dict(dt=1, q=FAKE, sel=FAKE, ns=10, out=FAKE, mask=None, n=8, hq=32, scale=0.1, ws=FAKE,
             wsb=BIG)
    a.update(kw)
    return wf.lib.wf_paged_sparse_attn(a["dt"], a["q"], _cache(**cache), _batch(**batch),
                                       a["sel"], a["ns"], a["out"], a["mask"], a["n"], a["hq"],
                                       a["scale"], a["ws"], a["wsb"], None)


CALLS = [_append, _attn, _select, _sparse]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("cache,status", [
    (dict(none=True), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(k=ODD), 1), (dict(v=ODD), 1),
    (dict(bounds=ODD), 1), (dict(n=0), 1), (dict(hkv=0), 1), (dict(hkv=257), 1), (dict(page=0), 1),
    (dict(page=48), 1), (dict(page=256), 1), (dict(page=8), 1), (dict(dh=96), 2),
    (dict(dh=256), 2), (dict(dh=0), 2), (dict(hkv=5), 1),
])
def test_the_cache_is_checked_by_every_call(call, cache, status):
    assert call(cache) == status


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("batch", [
    dict(none=True), dict(table=None), dict(start=None), dict(ctx=None), dict(table=ODD4),
    dict(start=ODD4), dict(ctx=ODD4), dict(n=0), dict(n=1025), dict(n=-1), dict(pages=0),
    dict(pages=(1 << 20) + 1), dict(pages=2**31 - 1)])
def test_the_batch_is_checked_by_every_call(call, batch):
    assert call({}, batch) == 1


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("kw", [dict(dt=2), dict(dt=7), dict(dt=-1), dict(n=-1),
                                dict(n=(1 << 20) + 1), dict(q=ODD)])
def test_shared_refusals(call, kw):
    assert call(**kw) == 1


@pytest.mark.parametrize("call", CALLS)
def test_no_rows_are_a_no_op(call):
    assert call(n=0) == 0


@pytest.mark.parametrize("call", CALLS[1:])
@pytest.mark.parametrize("rows", [0, 65, -3])
def test_row_limit(call, rows):
    assert call({}, dict(rows=rows)) == 1
    assert _append({}, dict(rows=rows), n=0) == 0        # the append takes any number


@pytest.mark.parametrize("call", CALLS[1:])
@pytest.mark.parametrize("kw,status", [
    (dict(q=None), 1), (dict(hq=30), 1), (dict(hq=0), 1), (dict(hq=264), 1), (dict(ws=None), 3),
    (dict(ws=ODD), 3), (dict(wsb=64), 3), (dict(wsb=(4 << 20)), 3)])
def test_query_and_workspace_refusals(call, kw, status):
    assert call(**kw) == status


@pytest.mark.parametrize("kw", [
    dict(k=None), dict(v=None), dict(k=ODD), dict(v=ODD), dict(ks=1020), dict(ks=1016),
    dict(ks=1 << 41), dict(qs=4090), dict(qs=4088), dict(qo=None), dict(qo=ODD), dict(hq=30),
    dict(hq=0), dict(hq=512), dict(base=0.0), dict(base=-2.0), dict(base=float("inf")),
    dict(base=float("nan")), dict(pos=ODD4)])
def test_append_refuses(kw):
    assert _append(**kw) == 1


@pytest.mark.parametrize("call", [_attn, _sparse])
@pytest.mark.parametrize("kw", [
    dict(out=None), dict(out=ODD), dict(mask=ODD), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=float("nan")), dict(scale=float("inf")), dict(n=(1 << 17) + 1)])
def test_attention_refuses(call, kw):
    assert call(**kw) == 1


@pytest.mark.parametrize("kw", [
    dict(sel=None), dict(sel=ODD4), dict(ns=0), dict(ns=1025)])
def test_selections_are_checked(kw):
    assert _sparse(**kw) == 1
    assert _select(**kw) == 1


def test_sparse_work_is_counted_in_32_bits():
    assert _sparse(dict(hkv=32, page=128), n=1 << 17, ns=1024) == 1
    assert _sparse(dict(hkv=32, page=128), n=1 << 16, ns=1024) == 1
    assert _sparse(dict(hkv=32, page=128), n=(1 << 16) - 1, ns=1024, ws=None) == 3


@pytest.mark.parametrize("cache,batch,kw", [
    (dict(bounds=None), {}, {}), ({}, {}, dict(nr=0)), ({}, {}, dict(nr=11)),
    (dict(page=16), dict(pages=65537), {}), ({}, {}, dict(n=(1 << 16) + 1))])
def test_select_refuses(cache, batch, kw):
    assert _select(cache, batch, **kw) == 1


def _logprobs(**kw):
    a = dict(dt=0, z=FAKE, stride=1000, t=FAKE, n=4, vocab=1000, top=5, lp=FAKE, ent=FAKE,
             rank=FAKE, ids=FAKE, tops=FAKE, ws=FAKE, wsb=BIG)
    a.update(kw)
    return wf.lib.wf_token_logprobs(a["dt"], a["z"], a["stride"], a["t"], a["n"], a["vocab"],
                                    a["top"], a["lp"], a["ent"], a["rank"], a["ids"], a["tops"],
                                    a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(dt=2), 1), (dict(dt=9), 1), (dict(z=None), 1), (dict(z=ODD4), 1),
    (dict(dt=1, z=(1 << 20) + 1), 1), (dict(stride=999), 1), (dict(stride=1 << 41), 1),
    (dict(n=-1), 1), (dict(n=(1 << 20) + 1), 1), (dict(vocab=0), 1),
    (dict(vocab=(1 << 30) + 1, stride=1 << 31), 1), (dict(top=65), 1), (dict(top=-1), 1),
    (dict(vocab=3, top=4), 1), (dict(lp=None), 1), (dict(t=None), 1),
    (dict(t=None, lp=None), 1), (dict(ids=None), 1), (dict(tops=None), 1), (dict(top=0), 1),
    (dict(t=ODD4), 1), (dict(rank=ODD4), 1), (dict(tops=ODD4), 1), (dict(ent=ODD4), 1),
    (dict(ws=None), 3), (dict(ws=ODD), 3), (dict(wsb=4096), 3), (dict(n=0), 0),
    (dict(n=0, z=None, t=None, ws=None), 0)])
def test_logprobs_refuse(kw, status):
    assert _logprobs(**kw) == status


def test_workspace_queries():
    q = wf.wf_paged_verify_attn_workspace_bytes
    assert q(torch.bfloat16, 8, 4, 16, 32, 8, 128) > 4 << 20
    for bad in ((8, 0, 16, 32, 8, 128), (8, 4, 65, 32, 8, 128), (8, 4, 0, 32, 8, 128),
                (8, 4, 16, 30, 8, 128), (8, 4, 16, 32, 8, 96), (-1, 4, 16, 32, 8, 128),
                (1 << 20, 4, 16, 32, 8, 128), (8, 1025, 16, 32, 8, 128)):
        assert q(torch.bfloat16, *bad) == 0
    q = wf.wf_paged_sparse_attn_workspace_bytes
    assert q(torch.float32, 8, 32, 8, 128, 64, 10) > 4 << 20
    for bad in ((8, 32, 8, 128, 48, 10), (8, 32, 8, 128, 64, 0), (8, 32, 8, 128, 64, 1025),
                (8, 32, 0, 128, 64, 10)):
        assert q(torch.float32, *bad) == 0
    assert wf.wf_paged_select_workspace_bytes(8, 8, 100) == (4 << 20) + 8 * 8 * 100 * 8
    for bad in ((-1, 8, 100), (8, 0, 100), (8, 8, 0), (8, 8, 65537), (1 << 19, 8, 100)):
        assert wf.wf_paged_select_workspace_bytes(*bad) == 0
    assert wf.wf_token_logprobs_workspace_bytes(torch.float32, 16, 151936, 20) > 4 << 20
    for bad in ((-1, 100, 0), (1, 0, 0), (1, 100, 65), (1, 3, 4)):
        assert wf.wf_token_logprobs_workspace_bytes(torch.float32, *bad) == 0


def test_handles_refuse_what_does_not_fit():
    k = torch.zeros(3, 2, 16, 64)
    with pytest.raises(ValueError):
        wf.PagedCache(k, k)                                  # host memory
    with pytest.raises(ValueError):
        wf.PagedCache(k, k[:2])
    with pytest.raises(ValueError):
        wf.PagedCache(k, k.bfloat16())
    with pytest.raises(ValueError):
        wf.PagedCache(k, k, torch.zeros(3, 2, 64))
    with pytest.raises(ValueError):
        wf.PagedCache(k[0], k[0])
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)        # noqa: E731
    with pytest.raises(ValueError):
        wf.PagedBatch(i(2, 3), i(3), i(2))                   # host memory
    with pytest.raises(ValueError):
        wf.PagedBatch(i(2, 3), i(2), i(2))
    with pytest.raises(TypeError):
        wf.PagedBatch(i(2, 3), i(3).long(), i(2))


@pytest.mark.parametrize("call,tensors", [
    (_append, ("k", "v", "q", "qo")), (_append, ("k", "v")), (_attn, ("q", "out", "ws")),
    (_select, ("q", "sel", "ws")), (_sparse, ("q", "sel", "out", "ws"))])
def test_no_rows_are_a_no_op_with_empty_tensors(call, tensors):
    """An empty tensor's pointer is null."""
    assert call(n=0, **{t: None for t in tensors}) == 0


def test_selections_are_needed_where_there_are_rows():
    assert _sparse(sel=None, ws=None) == 1 and _select(sel=None, ws=None) == 1
    assert _sparse(n=0, sel=None, ns=0) == 1 and _sparse(n=0, sel=None, ns=1025) == 1


@pytest.mark.parametrize("query,sizes", [
    (wf.wf_paged_verify_attn_workspace_bytes, (8, 4, 16, 32, 8, 128)),
    (wf.wf_paged_sparse_attn_workspace_bytes, (8, 32, 8, 128, 64, 10)),
    (wf.wf_token_logprobs_workspace_bytes, (16, 1000, 5))])
def test_workspace_queries_refuse_other_types(query, sizes):
    assert query(torch.float32, *sizes) == query(wf.WF_F32, *sizes) >= 4 << 20
    assert query(torch.bfloat16, *sizes) == query(wf.WF_BF16, *sizes) >= 4 << 20
    for dtype in (torch.float16, torch.float64, torch.int32, torch.float8_e4m3fn, None, "bf16"):
        with pytest.raises(TypeError):
            query(dtype, *sizes)


class _Device:
    """As much of a device tensor as the handles look at."""

    def __init__(self, shape, dtype):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device("cuda", 0)

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return FAKE


def test_handles_keep_what_the_calls_hold():
    """The calls read a handle's struct: its numbers cannot be changed beside it."""
    kv = _Device((3, 2, 16, 64), torch.bfloat16)
    cache = wf.PagedCache(kv, kv, _Device((3, 2, 2, 64), torch.bfloat16))
    i32 = [_Device(s, torch.int32) for s in ((4, 9), (5,), (4,))]
    batch = wf.PagedBatch(*i32, max_rows=8)
    assert batch.max_rows == batch.struct.max_rows == 8 and cache.head_dim == 64
    for handle, names in ((batch, ("max_rows", "n_seqs", "max_pages", "dev", "struct", "ref",
                                   "page_table", "row_start", "ctx_len", "_tensors")),
                          (cache, ("head_dim", "page_size", "n_pages", "n_kv_heads", "code", "dtype",
                                   "device", "dev", "struct", "ref", "k", "v", "bounds"))):
        for name in names:
            before = getattr(handle, name)
            with pytest.raises(AttributeError):
                setattr(handle, name, 16)
            assert getattr(handle, name) is before
        handle.note = 1                        # the caller's own names are the caller's
        handle.note = 2
    again = copy.copy(batch)
    assert again.struct.max_rows == 8 and again.row_start is batch.row_start
