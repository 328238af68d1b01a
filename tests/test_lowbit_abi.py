"""What the 8-bit cache and 4-bit weight calls refuse, on the CPU: no call
here reaches the GPU (pointers are never dereferenced by the checks)."""
import contextlib
import copy
import ctypes

import numpy as np
import pytest
import torch

import lowbit_ref as R

wf = pytest.importorskip("paper_2606_07710_amd")

FAKE, ODD = 1 << 20, (1 << 20) + 8
COUNTER_BLOCK = 4 << 20


def _cache(**kw):
    a = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, hkv=8, cap=200, dh=128)
    a.update(kw)
    if a.get("none"):
        return None
    return ctypes.byref(wf.Kv8CacheStruct(a["k"], a["v"], a["k_scale"], a["v_scale"], a["hkv"],
                                          a["cap"], a["dh"]))


CACHE_FAULTS = [(dict(none=True), 1), (dict(k=None), 1), (dict(v=None), 1),
                (dict(k_scale=None), 1), (dict(v_scale=None), 1), (dict(k=ODD), 1),
                (dict(v=ODD), 1), (dict(hkv=0), 1), (dict(hkv=257), 1), (dict(cap=0), 1),
                (dict(cap=1 << 30), 1), (dict(dh=96), 2), (dict(dh=256), 2)]


def _append(cache={}, **kw):
    a = dict(dt=1, k=FAKE, v=FAKE, n=16, start=100, ts=1024, hs=128)
    a.update(kw)
    return wf.lib.wf_kv8_append(a["dt"], _cache(**cache), a["k"], a["v"], a["n"], a["start"],
                                a["ts"], a["hs"], None)


@pytest.mark.parametrize("cache,status", CACHE_FAULTS)
def test_cache_is_checked_by_every_call(cache, status):
    assert _append(cache) == status
    assert _attn(cache) == status
    assert _attn(cache, mask=FAKE) == status
    assert _compact(cache) == status
    assert _prefill(cache) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dt=2), 1), (dict(dt=7), 1), (dict(n=-1), 1), (dict(start=-1), 1), (dict(n=101), 1),
    (dict(start=185), 1), (dict(n=2**31 - 1, start=2**31 - 1), 1), (dict(k=None), 1),
    (dict(v=None), 1), (dict(k=ODD), 1), (dict(v=ODD), 1), (dict(ts=1028), 1), (dict(hs=4), 1),
    (dict(dt=0, ts=1026), 1), (dict(n=0), 0), (dict(n=0, k=None, v=None), 0),
])
def test_append_refuses(kw, status):
    assert _append(**kw) == status


def _attn(cache={}, **kw):
    a = dict(dt=1, q=FAKE, out=FAKE, mask=None, gamma=16, ctx=100, hq=32, scale=0.088, splits=0,
             ws=FAKE, wsb=1 << 30)
    a.update(kw)
    rest = (a["gamma"], a["ctx"], a["hq"], a["scale"], a["splits"], a["ws"], a["wsb"], None)
    if "mask" in kw:
        return wf.lib.wf_kv8_verify_attn_tree(a["dt"], a["q"], _cache(**cache), a["out"],
                                              a["mask"], *rest)
    return wf.lib.wf_kv8_verify_attn(a["dt"], a["q"], _cache(**cache), a["out"], *rest)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), 1), (dict(out=None), 1), (dict(q=ODD), 1), (dict(out=ODD), 1),
    (dict(gamma=0), 1), (dict(gamma=65), 1), (dict(ctx=-1), 1), (dict(ctx=185), 1),
    (dict(hq=30), 1), (dict(hq=264), 1), (dict(hq=0), 1), (dict(scale=0.0), 1),
    (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(splits=-1), 1),
    (dict(splits=1025), 1), (dict(dt=2), 1), (dict(dt=7), 1), (dict(ws=None), 3),
    (dict(wsb=64), 3), (dict(ws=ODD), 3), (dict(mask=None), 1), (dict(mask=ODD), 1),
])
def test_attention_refuses(kw, status):
    assert _attn(**kw) == status


def test_attention_workspace_query():
    f = wf.wf_kv8_verify_attn_workspace_bytes
    for dt, eb in ((1, 2), (0, 4)):
        assert f(dt, 16, 4000, 32, 8, 128, 7) >= COUNTER_BLOCK + 7 * 16 * 32 * (128 * eb + 8)
        assert f(dt, 1, 0, 8, 8, 64) > COUNTER_BLOCK
    assert f(2, 16, 4000, 32, 8, 128) == f(1, 0, 4000, 32, 8, 128) == 0
    assert f(1, 16, 4000, 32, 8, 96) == f(1, 16, -1, 32, 8, 128) == 0


def _compact(cache={}, **kw):
    a = dict(acc=FAKE, path=FAKE, gamma=61, ctx=100, layers=1, cs=0, ss=0)
    a.update(kw)
    return wf.lib.wf_kv8_compact_path(_cache(**cache), a["acc"], a["path"], a["gamma"], a["ctx"],
                                      a["layers"], a["cs"], a["ss"], None)


CODES, SCALES = 8 * 7 * 32 * 128, 8 * 7


@pytest.mark.parametrize("kw,status", [
    (dict(acc=None), 1), (dict(path=None), 1), (dict(gamma=0), 1), (dict(gamma=65), 1),
    (dict(ctx=-1), 1), (dict(ctx=140), 1), (dict(layers=0), 1),
    (dict(layers=1025, cs=CODES, ss=SCALES), 1), (dict(layers=2, cs=CODES - 16, ss=SCALES), 1),
    (dict(layers=2, cs=CODES, ss=SCALES - 1), 1), (dict(layers=2, cs=CODES + 8, ss=SCALES), 1),
])
def test_compact_refuses(kw, status):
    assert _compact(**kw) == status


def test_cache_sizes():
    assert wf.lib.wf_kv8_code_bytes(8, 200, 128) == CODES
    assert wf.lib.wf_kv8_scale_bytes(8, 200) == SCALES
    assert wf.lib.wf_kv8_code_bytes(8, 1, 64) == 8 * 32 * 64
    assert wf.lib.wf_kv8_code_bytes(256, 1 << 29, 128) == 256 * (1 << 29) * 128
    assert wf.lib.wf_kv8_code_bytes(8, 0, 128) == wf.lib.wf_kv8_code_bytes(8, 200, 96) == 0
    assert wf.lib.wf_kv8_scale_bytes(0, 200) == wf.lib.wf_kv8_scale_bytes(8, -1) == 0


def _prefill(cache={}, **kw):
    a = dict(dt=1, x=FAKE, wk=FAKE, wv=FAKE, n=16, start=100, d=4096, base=1e6, ws=FAKE,
             wsb=1 << 30)
    a.update(kw)
    return wf.lib.wf_kv8_only_prefill(a["dt"], a["x"], a["wk"], a["wv"], _cache(**cache), a["n"],
                                      a["start"], a["d"], a["base"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), 1), (dict(wk=None), 1), (dict(wv=ODD), 1), (dict(n=-1), 1), (dict(n=101), 1),
    (dict(start=-1), 1), (dict(d=0), 1), (dict(d=100), 2), (dict(base=0.0), 1), (dict(dt=7), 1),
    (dict(ws=None), 3), (dict(wsb=COUNTER_BLOCK), 3), (dict(ws=ODD), 3), (dict(n=0), 0),
    (dict(dt=0, ws=None), 3),
])
def test_prefill_refuses(kw, status):
    assert _prefill(**kw) == status


def test_prefill_workspace_query():
    f = wf.wf_kv8_only_prefill_workspace_bytes
    assert f(1, 16, 4096, 8, 128) == COUNTER_BLOCK + 2 * 16 * 8 * 128 * 2
    assert f(0, 16, 4096, 8, 128) == 2 * 16 * 8 * 128 * 4
    assert f(1, 0, 4096, 8, 128) == f(1, 16, 100, 8, 128) == f(1, 5000, 4096, 8, 128) == 0


def _linear(**kw):
    a = dict(x=FAKE, packed=FAKE, res=None, dt=1, y=FAKE, rows=16, n_out=4096, k_in=4096,
             ws=FAKE, wsb=1 << 30)
    a.update(kw)
    return wf.lib.wf_linear_w4(a["x"], a["packed"], a["res"], a["dt"], a["y"], a["rows"],
                               a["n_out"], a["k_in"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), 1), (dict(packed=None), 1), (dict(y=None), 1),
    (dict(x=ODD), 1), (dict(packed=ODD), 1), (dict(rows=0), 1), (dict(rows=65), 1),
    (dict(n_out=0), 1), (dict(n_out=(1 << 30) + 1), 1), (dict(k_in=0), 1), (dict(k_in=48), 1),
    (dict(k_in=(1 << 20) + 32), 1), (dict(dt=2), 1), (dict(dt=9), 1),
    (dict(n_out=1 << 30, k_in=1 << 20), 1),
])
def test_linear_refuses(kw, status):
    assert _linear(**kw) == status


@pytest.mark.parametrize("args,status", [
    ((None, 16, 64, FAKE, FAKE), 1), ((FAKE, 16, 64, None, FAKE), 1),
    ((FAKE, 16, 64, FAKE, None), 1), ((ODD, 16, 64, FAKE, FAKE), 1),
    ((FAKE, 16, 64, ODD, FAKE), 1), ((FAKE, 0, 64, FAKE, FAKE), 1),
    ((FAKE, 16, 0, FAKE, FAKE), 1), ((FAKE, 16, 48, FAKE, FAKE), 1),
])
def test_quantize_refuses(args, status):
    assert wf.lib.wf_w4_quantize(*args, None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(codes=None), 1), (dict(scales=None), 1), (dict(packed=None), 1), (dict(codes=ODD), 1),
    (dict(packed=ODD), 1), (dict(rows=0), 1), (dict(cols=0), 1), (dict(cols=48), 1),
    (dict(nbytes=2 * 1088 - 1), 3),
])
def test_pack_refuses(kw, status):
    a = dict(codes=FAKE, scales=FAKE, rows=16, cols=160, packed=FAKE, nbytes=2 * 1088)
    a.update(kw)
    assert wf.lib.wf_w4_pack(a["codes"], a["scales"], a["rows"], a["cols"], a["packed"],
                             a["nbytes"], None) == status


def test_packed_sizes():
    f = wf.lib.wf_w4_packed_bytes
    assert f(1, 32) == 1088 and f(16, 128) == 1088 and f(17, 160) == 4 * 1088
    assert f(151936, 2560) == 9496 * 20 * 1088
    assert f(0, 32) == f(16, 0) == f(16, 48) == f(1 << 30, 1 << 20) == 0


# ---- the Python layer -------------------------------------------------------------

class Fake:
    """A stand-in for a device tensor whose pointer the C side refuses."""
    device = "cuda"

    def __init__(self, *shape, dtype=torch.bfloat16, stride=None, ptr=8, on=0):
        self.shape, self.dtype, self.ptr, self.on = torch.Size(shape), dtype, ptr, on
        self.strides = stride or torch.empty(shape, device="meta").stride()

    def data_ptr(self):
        return self.ptr

    def get_device(self):
        return self.on

    def is_contiguous(self):
        return True

    def stride(self, d=None):
        return self.strides if d is None else self.strides[d]

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return torch.empty((), dtype=self.dtype).element_size()


class FakeStream:
    cuda_stream = 0


@pytest.fixture(autouse=True)
def _device_zero(monkeypatch):
    monkeypatch.setattr(wf, "_current", lambda: (0, 0))


def _bytes(*shape, **kw):
    return Fake(*shape, dtype=torch.uint8, **kw)


def _kv8(hkv=2, cap=70, dh=64, layers=None, **kw):
    b, lead = (cap + 31) // 32, () if layers is None else (layers,)
    t = dict(k=_bytes(*lead, hkv, b, 32, dh), v=_bytes(*lead, hkv, b, dh, 32),
             k_scale=_bytes(*lead, hkv, b), v_scale=_bytes(*lead, hkv, b))
    t.update(kw)
    return wf.Kv8Cache(t["k"], t["v"], t["k_scale"], t["v_scale"], cap)


def _w4(dev=0):
    w = wf.W4Weight.__new__(wf.W4Weight)
    w.packed, w.shape = _bytes(1088, on=dev), (16, 64)
    return w


@pytest.mark.parametrize("kw", [
    dict(v=_bytes(2, 3, 32, 64)), dict(k_scale=_bytes(2, 2)), dict(k=_bytes(2, 4, 32, 64)),
    dict(k=_bytes(2, 3, 16, 64)), dict(k=Fake(2, 3, 32, 64)), dict(cap=64), dict(cap=0),
])
def test_python_cache_shapes(kw):
    ok = _kv8()
    with pytest.raises(ValueError):
        t = dict(k=ok.k, v=ok.v, k_scale=ok.k_scale, v_scale=ok.v_scale, cap=70)
        t.update(kw)
        wf.Kv8Cache(**t)


def test_python_cache_takes_whole_capacities_only():
    with pytest.raises(TypeError):
        ok = _kv8()
        wf.Kv8Cache(ok.k, ok.v, ok.k_scale, ok.v_scale, 70.0)


def test_python_cache_keeps_its_tensors():
    """The calls hold the tensors' addresses: others cannot take their place, and a
    deep copy holds those of its own."""
    c = _kv8(layers=3)
    for name in ("k", "v", "k_scale", "v_scale"):
        with pytest.raises(AttributeError):
            setattr(c, name, getattr(c, name))
    for t, at in zip((c.k, c.v, c.k_scale, c.v_scale), (16, 32, 48, 64)):
        t.ptr = at
    mine = copy.deepcopy(c)
    assert mine.k is not c.k and (mine.n_layers, mine.cap, mine.head_dim) == (3, 70, 64)
    assert [getattr(mine.struct, n) for n in ("k", "v", "k_scale", "v_scale")] == [16, 32, 48, 64]
    assert copy.copy(c).k is c.k and c.struct.k == 8


def test_python_one_layer_calls_refuse_a_stack():
    q = Fake(4, 8, 64)
    with pytest.raises(ValueError):
        wf.wf_kv8_verify_attn(q, _kv8(layers=3), q, 5, workspace=_bytes(64), stream=FakeStream)
    with pytest.raises(ValueError):
        wf.wf_kv8_append(Fake(4, 2, 64), Fake(4, 2, 64), _kv8(layers=3), 0, stream=FakeStream)


@pytest.mark.parametrize("k,v", [
    (Fake(4, 2, 64), Fake(5, 2, 64)), (Fake(4, 3, 64), Fake(4, 3, 64)),
    (Fake(4, 2, 128), Fake(4, 2, 128)), (Fake(4, 2, 64), Fake(4, 2, 64, dtype=torch.float32)),
    (Fake(4, 2, 64, stride=(128, 64, 1)), Fake(4, 2, 64, stride=(64, 256, 1))),
    (Fake(4, 2, 64, stride=(256, 128, 2)), Fake(4, 2, 64, stride=(256, 128, 2))),
])
def test_python_append_refuses(k, v):
    with pytest.raises(ValueError):
        wf.wf_kv8_append(k, v, _kv8(), 0, stream=FakeStream)


def test_python_calls_refuse_other_devices():
    """Every tensor lies on the current device, whatever stream is given."""
    q, x, far = Fake(4, 8, 64), Fake(4, 64), dict(on=1)
    ws, path = _bytes(64), Fake(4, dtype=torch.int32)
    for call in (
            lambda: wf.wf_kv8_verify_attn(Fake(4, 8, 64, **far), _kv8(), q, 5, workspace=ws),
            lambda: wf.wf_kv8_verify_attn(q, _kv8(), Fake(4, 8, 64, **far), 5, workspace=ws),
            lambda: wf.wf_kv8_verify_attn(q, _kv8(), q, 5, workspace=_bytes(64, on=-1)),
            lambda: wf.wf_kv8_verify_attn(q, _far_cache(), q, 5, workspace=ws,
                                          stream=FakeStream),
            lambda: wf.wf_kv8_append(Fake(4, 2, 64, **far), Fake(4, 2, 64), _kv8(), 0),
            lambda: wf.wf_kv8_append(Fake(4, 2, 64), Fake(4, 2, 64, on=-1), _kv8(), 0),
            lambda: wf.wf_kv8_compact_path(_far_cache(), path, path, 0),
            lambda: wf.wf_kv8_compact_path(_kv8(), Fake(4, dtype=torch.int32, on=1), path, 0),
            lambda: wf.wf_linear_w4(Fake(4, 64, **far), _w4(), Fake(4, 16)),
            lambda: wf.wf_linear_w4(x, _w4(dev=1), Fake(4, 16)),
            lambda: wf.W4Weight(_bytes(16, 32, on=1), _bytes(16, 2)),
            lambda: wf.wf_w4_quantize(Fake(16, 64, **far)),
            lambda: _kv8(v=_bytes(2, 3, 64, 32, on=1)), lambda: _kv8(k=_bytes(2, 3, 32, 64, on=-1))):
        with pytest.raises(ValueError):
            call()


def test_python_calls_refuse_other_devices_streams():
    class Far:
        cuda_stream, device_index = 0, 1
    with pytest.raises(ValueError):
        wf.wf_kv8_append(Fake(4, 2, 64), Fake(4, 2, 64), _kv8(), 0, stream=Far)
    with pytest.raises(ValueError):
        wf.wf_linear_w4(Fake(4, 64), _w4(), Fake(4, 16), stream=Far)


def _far_cache():
    far = [_bytes(*s, on=1) for s in ((2, 3, 32, 64), (2, 3, 64, 32), (2, 3), (2, 3))]
    return wf.Kv8Cache(*far, 70)


@pytest.mark.parametrize("ctx", [5.5, "5"])
def test_python_takes_whole_numbers_only(ctx):
    q = Fake(4, 8, 64)
    with pytest.raises((ctypes.ArgumentError, TypeError)):
        wf.wf_kv8_verify_attn(q, _kv8(), q, ctx, workspace=_bytes(64), stream=FakeStream)
    with pytest.raises((ctypes.ArgumentError, TypeError)):
        wf.wf_kv8_append(Fake(4, 2, 64), Fake(4, 2, 64), _kv8(), ctx, stream=FakeStream)


def test_python_calls_reach_the_library():
    q, x = Fake(4, 8, 64), Fake(4, 64)
    path = Fake(4, dtype=torch.int32)
    w = _w4()
    for call in (lambda: wf.wf_kv8_verify_attn(q, _kv8(), q, 5, workspace=_bytes(64),
                                               stream=FakeStream),
                 lambda: wf.wf_kv8_append(Fake(4, 2, 64), Fake(4, 2, 64), _kv8(), 0,
                                          stream=FakeStream),
                 lambda: wf.wf_kv8_compact_path(_kv8(), path, path, 0, stream=FakeStream),
                 lambda: wf.wf_linear_w4(x, w, Fake(4, 16), stream=FakeStream)):
        with pytest.raises(wf.WfError) as e:
            call()
        assert e.value.status == wf.WF_ERR_INVALID_ARG


@pytest.mark.parametrize("codes,scales", [
    (_bytes(16, 24), _bytes(16, 1)), (_bytes(16, 32), _bytes(16, 1)),
    (_bytes(16, 32), _bytes(15, 2)), (Fake(16, 32), _bytes(16, 2)),
])
def test_python_weight_shapes(codes, scales):
    with pytest.raises(ValueError):
        wf.W4Weight(codes, scales)


@pytest.mark.parametrize("x,out,res", [
    (Fake(4, 96), Fake(4, 16), None), (Fake(4, 64), Fake(4, 17), None),
    (Fake(4, 64), Fake(4, 16), Fake(4, 17)),
    (Fake(4, 64, dtype=torch.float32), Fake(4, 16), None),
    (Fake(4, 64), Fake(4, 16, dtype=torch.float16), None),
    (Fake(4, 64), Fake(4, 16), Fake(4, 16, dtype=torch.float32)),
])
def test_python_linear_refuses(x, out, res):
    w = _w4()
    with pytest.raises((ValueError, TypeError)):
        wf.wf_linear_w4(x, w, out, res, stream=FakeStream)


@pytest.mark.parametrize("dtype", [torch.float64, torch.complex64, torch.int32])
def test_python_tree_masks_are_whole_words(dtype):
    q = Fake(4, 8, 64)
    with pytest.raises(ValueError):
        wf.wf_kv8_verify_attn_tree(q, _kv8(), q, 5, Fake(4, dtype=dtype), workspace=_bytes(64),
                                   stream=FakeStream)


@pytest.mark.parametrize("dtype", [torch.int64, torch.uint64])
def test_python_tree_masks_reach_the_library(dtype):
    q = Fake(4, 8, 64)
    with pytest.raises(wf.WfError):
        wf.wf_kv8_verify_attn_tree(q, _kv8(), q, 5, Fake(4, dtype=dtype), workspace=_bytes(64),
                                   stream=FakeStream)


@pytest.mark.parametrize("name,shape,good", [
    ("k", (2, 3, 32, 64), "e4m3fn"), ("v", (2, 3, 64, 32), "e4m3fn"),
    ("k_scale", (2, 3), "e8m0fnu"), ("v_scale", (2, 3), "e8m0fnu"),
])
def test_python_cache_types(name, shape, good):
    """Bytes, or the format that they are in; no other one-byte type."""
    for dtype in (torch.int8, torch.bool, torch.float8_e5m2, torch.float8_e4m3fnuz,
                  torch.float8_e8m0fnu, torch.float8_e4m3fn, torch.uint8):
        t = Fake(*shape, dtype=dtype)
        if dtype == torch.uint8 or good in str(dtype).split("_")[-1:]:
            assert getattr(_kv8(**{name: t}), name) is t
        else:
            with pytest.raises(ValueError):
                _kv8(**{name: t})


@pytest.mark.parametrize("codes,scales", [
    (torch.int8, torch.uint8), (torch.float8_e4m3fn, torch.uint8), (torch.bool, torch.uint8),
    (torch.uint8, torch.int8), (torch.uint8, torch.float8_e4m3fn),
])
def test_python_weight_types(codes, scales):
    with pytest.raises(ValueError):
        wf.W4Weight(Fake(16, 32, dtype=codes), Fake(16, 2, dtype=scales))


def test_python_weights_hold_what_a_side_stream_still_reads(monkeypatch):
    """codes, scales and w may be temporaries: memory that another stream still
    reads must not be given out again."""
    order = []

    class Held(Fake):
        device = "cpu"

        def record_stream(self, stream):
            order.append((self, stream))

    def launch(*args):
        order.append("launch")
        return 0
    monkeypatch.setattr(wf.lib, "wf_w4_pack", launch)
    monkeypatch.setattr(wf.lib, "wf_w4_quantize", launch)
    monkeypatch.setattr(wf, "_on", lambda stream: contextlib.nullcontext())
    codes, scales = Held(16, 32, dtype=torch.uint8), Held(16, 2, dtype=torch.uint8)
    wf.W4Weight(codes, scales, stream=FakeStream)
    assert order == ["launch", (codes, FakeStream), (scales, FakeStream)]
    order.clear()
    w = Held(16, 64)
    wf.wf_w4_quantize(w, stream=FakeStream)
    assert order == ["launch", (w, FakeStream)]
    order.clear()
    wf.W4Weight(codes, scales)           # (their own stream: nothing to hold)
    wf.wf_w4_quantize(w)
    assert order == ["launch", "launch"]


# ---- the reference itself -----------------------------------------------------------

def test_reference_formats():
    """The tables against torch's own conversions, and the scale rule."""
    codes = torch.arange(256, dtype=torch.uint8)
    np.testing.assert_array_equal(R.E4M3, codes.view(torch.float8_e4m3fn).double().numpy())
    assert R.E2M1[:8].tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    x = torch.randn(20000, generator=torch.Generator().manual_seed(1)) * 30
    got = R._nearest(x.double().numpy(), R.E4M3[:127]) + 128 * np.signbit(x.numpy())
    np.testing.assert_array_equal(got, x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert R.exponent(448.0, 448.0) == 0 and R.exponent(449.0, 448.0) == 1
    assert R.exponent(224.0, 448.0) == -1 and R.exponent(0.0, 448.0) == 0
    assert R.exponent(1e-45, 448.0) == -100 and R.exponent(3.3e38, 448.0) == 120
