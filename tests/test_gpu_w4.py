"""4-bit weights on the GPU against plain 64-bit definitions: the quantiser
exactly, the product within the roundings it makes."""
import copy

import numpy as np
import pytest
import torch

import lowbit_ref as R

pytestmark = pytest.mark.gpu

wf = pytest.importorskip("paper_2606_07710_amd")
DEV = "cuda"


def _normal(seed, *shape, std=1.0, dtype=torch.bfloat16):
    g = torch.Generator()
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(dtype)


@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 64), (17, 96), (5, 1056), (130, 512)])
def test_quantize(rows, cols):
    w = _normal(rows, rows, cols, std=0.02)
    w[0, :8] = torch.tensor([0.0, -0.0, 1e-30, 6.0, 5.0, -0.25, 3.5, 2.5])
    got = wf.wf_w4_quantize(w.to(DEV))
    torch.cuda.synchronize()
    codes, scales = R.encode_e2m1(w.double().numpy())
    np.testing.assert_array_equal(got[1].cpu().numpy(), scales)
    np.testing.assert_array_equal(got[0].cpu().numpy(), codes)


def test_quantize_borders():
    """Every rounding border of the format, both signs, groups of zeros, out of
    range and not finite."""
    mid = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    row = torch.tensor(mid + [-m for m in mid] + [6.0] + [0.0] * 17)
    w = torch.stack([row, row * (1 + 2.0 ** -7), row * (1 - 2.0 ** -7), row * 2.0 ** -118,
                     torch.zeros(32), row * 2.0 ** 119, row * 2.0 ** 125, row, row])
    w[7, 3], w[8, 4] = float("nan"), float("-inf")
    w = w.to(torch.bfloat16)
    got = wf.wf_w4_quantize(w.to(DEV))
    torch.cuda.synchronize()
    codes, scales = R.encode_e2m1(w.double().numpy())
    np.testing.assert_array_equal(got[1].cpu().numpy(), scales)
    fine = scales[:, 0] != 255
    assert fine.sum() == 7
    np.testing.assert_array_equal(got[0].cpu().numpy()[fine], codes[fine])


@pytest.mark.parametrize("rows,cols", [(1, 32), (16, 128), (17, 160), (40, 2880)])
def test_pack(rows, cols):
    """Every byte of the packed tiles, padding included."""
    codes, scales = _weight(rows, rows, cols)
    got = wf.W4Weight(codes.to(DEV), scales.to(DEV)).packed
    torch.cuda.synchronize()
    nb, nc = (rows + 15) // 16, (cols + 127) // 128
    c = np.zeros((nb * 16, nc * 64), np.uint8)
    c[:rows, :cols // 2] = codes.numpy()
    s = np.full((nb * 16, nc * 4), 127, np.uint8)
    s[:rows, :cols // 32] = scales.numpy()
    # [block][row][chunk][group][quarter][4 bytes] -> a lane's quarter of each group
    c = c.reshape(nb, 16, nc, 4, 4, 4).transpose(0, 2, 4, 1, 3, 5).reshape(nb, nc, 1024)
    s = s.reshape(nb, 16, nc, 4).transpose(0, 2, 1, 3).reshape(nb, nc, 64)
    np.testing.assert_array_equal(got.cpu().numpy(), np.concatenate([c, s], 2).ravel())


def _weight(seed, n_out, k_in):
    g = torch.Generator()
    g.manual_seed(seed)
    codes = torch.randint(0, 256, (n_out, k_in // 2), generator=g, dtype=torch.uint8)
    scales = torch.randint(112, 128, (n_out, k_in // 32), generator=g, dtype=torch.uint8)
    return codes, scales


SHAPES = [
    # rows, n_out, k_in
    (1, 1, 32), (1, 16, 128), (1, 4096, 4096), (2, 17, 96), (3, 1000, 2880), (5, 33, 160),
    (11, 2560, 9728), (16, 1024, 4096), (17, 130, 1024), (31, 48, 64), (32, 257, 2560),
    (33, 4096, 512), (47, 100, 4096), (61, 3001, 2560), (64, 512, 12288), (64, 5, 32),
    (48, 24576, 544), (12, 16384, 1056), (1, 40, 40960),
    # (few features and much x: slices)
    (16, 300, 12352), (13, 1001, 12000), (4, 17, 40992),
]


def _check(x, codes, scales, got, res=None, out="bf16"):
    """fp32 sums of exact products: k_in terms and the waves' sums, off by
    (k_in + 64) 2^-24 of sum |x w| at the worst; the residual's addition by
    2^-24 and a bf16 result by 2^-8 of the value."""
    w = torch.from_numpy(R.decode_e2m1(codes.numpy(), scales.numpy()))
    ref = x.double() @ w.t()
    mass = x.double().abs() @ w.abs().t()
    if res is not None:
        ref, mass = ref + res.double(), mass + res.double().abs()
    tol = mass * (x.shape[1] + 64) * 2.0 ** -24
    if out == "bf16":
        tol = tol + (ref.abs() + tol) * 2.0 ** -8
    err = (got.double().cpu() - ref).abs()
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("rows,n_out,k_in", SHAPES)
@pytest.mark.parametrize("out,res", [("bf16", False), ("bf16", True), ("f32", False),
                                     ("f32", True)])
def test_linear(rows, n_out, k_in, out, res):
    print("linear", rows, n_out, k_in, out, res, flush=True)
    codes, scales = _weight(rows + n_out, n_out, k_in)
    x = _normal(k_in, rows, k_in)
    r = _normal(7, rows, n_out) if res else None
    dt = torch.bfloat16 if out == "bf16" else torch.float32
    pad = torch.full((rows * n_out + 64,), float("nan"), dtype=dt, device=DEV)
    y = pad[:rows * n_out].view(rows, n_out)
    w = wf.W4Weight(codes.to(DEV), scales.to(DEV))
    ret = wf.wf_linear_w4(x.to(DEV), w, y, r.to(DEV) if res else None)
    torch.cuda.synchronize()
    assert ret is y
    _check(x, codes, scales, y, r, out)
    assert pad[rows * n_out:].isnan().all()          # nothing behind the output
    again = torch.empty_like(y)
    wf.wf_linear_w4(x.to(DEV), w, again, r.to(DEV) if res else None)
    torch.cuda.synchronize()
    assert torch.equal(again, y)


# Many features: the feature split of up to 16 rows, from eight waves to a feature
# group to one, several rounds of workgroups, blocks that do not divide evenly.
@pytest.mark.parametrize("rows,n_out,k_in", [
    (5, 30000, 96), (12, 82000, 64), (16, 200000, 32), (33, 40000, 160), (17, 66004, 96),
    (50, 36002, 288), (61, 90001, 64), (20, 140000, 32), (64, 170000, 32),
    (7, 20400, 1312), (16, 45000, 544), (2, 70000, 96), (10, 100000, 64), (13, 24000, 2080),
])
def test_linear_many_features(rows, n_out, k_in):
    print("many features", rows, n_out, k_in, flush=True)
    codes, scales = _weight(rows + n_out, n_out, k_in)
    x = _normal(k_in, rows, k_in)
    y = torch.full((rows, n_out), float("nan"), device=DEV)
    wf.wf_linear_w4(x.to(DEV), wf.W4Weight(codes.to(DEV), scales.to(DEV)), y)
    torch.cuda.synchronize()
    _check(x, codes, scales, y, out="f32")


# At the lines between four, two and one wave to a feature group, on both sides, for
# each number of 16-row blocks.
@pytest.mark.parametrize("n_out", [12289, 20480, 40950, 40970, 81920, 81921])
@pytest.mark.parametrize("rows,k_in", [(1, 1056), (16, 544), (20, 544), (47, 288), (64, 1312)])
def test_linear_wave_counts(rows, k_in, n_out):
    print("wave counts", rows, n_out, k_in, flush=True)
    codes, scales = _weight(rows + n_out, n_out, k_in)
    x, r = _normal(k_in, rows, k_in), _normal(3, rows, n_out)
    y = torch.full((rows, n_out), float("nan"), dtype=torch.bfloat16, device=DEV)
    wf.wf_linear_w4(x.to(DEV), wf.W4Weight(codes.to(DEV), scales.to(DEV)), y, r.to(DEV))
    torch.cuda.synchronize()
    _check(x, codes, scales, y, r)


@pytest.mark.parametrize("rows,n_out,k_in", [(3, 40, 64), (20, 1000, 512), (40, 33000, 64)])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_linear_odd_addresses(rows, n_out, k_in, out):
    """Output and residual that start at any element."""
    print("odd addresses", rows, n_out, k_in, out, flush=True)
    codes, scales = _weight(n_out, n_out, k_in)
    x, r = _normal(1, rows, k_in), _normal(2, rows, n_out)
    dt = torch.bfloat16 if out == "bf16" else torch.float32
    w = wf.W4Weight(codes.to(DEV), scales.to(DEV))
    for at in (1, 2, 3):
        buf = torch.full((rows * n_out + 8,), float("nan"), dtype=dt, device=DEV)
        rb = torch.empty(rows * n_out + 8, dtype=torch.bfloat16, device=DEV)
        y, rd = (t[at:at + rows * n_out].view(rows, n_out) for t in (buf, rb))
        rd.copy_(r)
        wf.wf_linear_w4(x.to(DEV), w, y, rd)
        torch.cuda.synchronize()
        _check(x, codes, scales, y, r, out)
        assert buf[:at].isnan().all() and buf[at + rows * n_out:].isnan().all()


@pytest.mark.parametrize("rows,n_out,k_in", [(3, 40, 96), (20, 300, 160), (18, 33000, 64), (16, 40, 10016),
                                             (5, 30000, 32)])
def test_linear_infinite_inputs(rows, n_out, k_in):
    """An infinity, also among the last inputs: infinities of the weight's sign
    in its row, and nothing in the others."""
    print("infinite inputs", rows, n_out, k_in, flush=True)
    codes, scales = _weight(n_out, n_out, k_in)
    codes = codes | 0x11                             # (no zero weight)
    x = _normal(1, rows, k_in)
    x[0, 1], x[1, k_in - 1], x[2, k_in - 2] = float("inf"), float("-inf"), float("nan")
    y = torch.empty(rows, n_out, device=DEV)
    wf.wf_linear_w4(x.to(DEV), wf.W4Weight(codes.to(DEV), scales.to(DEV)), y)
    torch.cuda.synchronize()
    w = torch.from_numpy(R.decode_e2m1(codes.numpy(), scales.numpy()))
    y = y.cpu()
    assert torch.equal(y[0].double(), float("inf") * w[:, 1].sign())
    assert torch.equal(y[1].double(), float("-inf") * w[:, -1].sign())
    assert y[2].isnan().all()
    _check(x[3:], codes, scales, y[3:], out="f32")


def test_linear_residual_in_place_and_workspace_reuse():
    """The residual may be the output; calls of several sizes share one
    workspace, also from a captured graph."""
    ws = wf.alloc_workspace(max([wf.wf_linear_w4_workspace_bytes(*s) for s in SHAPES] + [16]), DEV)
    calls = []
    for rows, n_out, k_in in SHAPES[2:14]:
        codes, scales = _weight(rows, n_out, k_in)
        calls.append((_normal(1, rows, k_in), codes, scales, _normal(2, rows, n_out),
                      wf.W4Weight(codes.to(DEV), scales.to(DEV))))
    ys = [c[3].to(DEV) for c in calls]
    xs = [c[0].to(DEV) for c in calls]
    first = [c[3].to(DEV) for c in calls]

    def step():
        for x, c, y, f in zip(xs, calls, ys, first):
            y.copy_(f)
            wf.wf_linear_w4(x, c[4], y, y, workspace=ws)

    step()
    torch.cuda.synchronize()
    ref = [y.clone() for y in ys]
    for c, y in zip(calls, ys):
        _check(c[0], c[1], c[2], y, c[3])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for y in ys:
            y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, ys))
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, ys))
    assert ws.numel() < (4 << 20) or not bool(ws[:4 << 20].any().item())


def test_linear_extreme_scales_and_nan():
    """Scales at both ends of the range, and the NaN scale: only its feature."""
    codes, scales = _weight(1, 48, 256)
    scales[3], scales[4], scales[5, 2] = 27, 240, 255
    x = _normal(2, 5, 256)
    y = torch.empty(5, 48, device=DEV)
    wf.wf_linear_w4(x.to(DEV), wf.W4Weight(codes.to(DEV), scales.to(DEV)), y)
    torch.cuda.synchronize()
    assert y[:, 5].isnan().all()
    keep = [i for i in range(48) if i != 5]
    _check(x, codes[keep], scales[keep], y[:, keep], out="f32")


@pytest.mark.parametrize("rows,n_out,k_in", [(17, 130, 1024), (61, 500, 4096), (16, 33, 12000),
                                             (33, 200, 2080)])
def test_linear_writes_its_output_and_workspace_only(rows, n_out, k_in):
    print("bounds", rows, n_out, k_in, flush=True)
    codes, scales = _weight(5, n_out, k_in)
    x = _normal(6, rows, k_in)
    w = wf.W4Weight(codes.to(DEV), scales.to(DEV))
    need = wf.wf_linear_w4_workspace_bytes(rows, n_out, k_in)
    room = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device=DEV)
    buf = torch.full((rows * n_out + 32,), 7.0, device=DEV)
    y = buf[16:16 + rows * n_out].view(rows, n_out)
    wf.wf_linear_w4(x.to(DEV), w, y, workspace=room[:need])
    torch.cuda.synchronize()
    assert (room[need:] == 0x5a).all() and (room[:4 << 20] == 0x5a).all()
    assert (buf[:16] == 7).all() and (buf[16 + rows * n_out:] == 7).all()
    _check(x, codes, scales, y, out="f32")


def test_weight_copies_stand_alone():
    """A deep copy of a packed weight holds its own memory."""
    codes, scales = _weight(3, 48, 256)
    x = _normal(2, 5, 256).to(DEV)
    w = wf.W4Weight(codes.to(DEV), scales.to(DEV))
    mine = copy.deepcopy(w)
    w.packed.zero_()
    del w
    y = torch.empty(5, 48, device=DEV)
    wf.wf_linear_w4(x, mine, y)
    torch.cuda.synchronize()
    _check(x.cpu(), codes, scales, y, out="f32")


def test_weight_on_a_side_stream():
    """Quantised, packed and used on a stream of its own, workspaces included."""
    side = torch.cuda.Stream()
    w16 = _normal(4, 130, 12352).to(DEV)
    x = _normal(5, 16, 12352).to(DEV)
    codes, scales = wf.wf_w4_quantize(w16)
    here = torch.empty(16, 130, device=DEV)
    wf.wf_linear_w4(x, wf.W4Weight(codes, scales), here)
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        there = torch.zeros(16, 130, device=DEV)
        side.wait_stream(torch.cuda.current_stream())
        w = wf.W4Weight(*wf.wf_w4_quantize(w16, stream=side), stream=side)
        wf.wf_linear_w4(x, w, there, stream=side)
        side.synchronize()
        assert torch.equal(there, here)


def test_weight_from_temporaries_on_a_side_stream():
    """Sources that nothing holds any more while a side stream, busy with other
    work, has still to read them, and whose memory is asked for again."""
    codes, scales = _weight(3, 512, 4096)
    w16 = _normal(4, 512, 4096)
    x = _normal(5, 3, 4096).to(DEV)
    side = torch.cuda.Stream()
    busy = torch.ones(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            busy = busy @ busy * 2.0 ** -12
    w = wf.W4Weight(codes.to(DEV), scales.to(DEV), stream=side)
    again = [torch.full(t.shape, 255, dtype=torch.uint8, device=DEV) for t in (codes, scales)]
    got = wf.wf_w4_quantize(w16.to(DEV), stream=side)
    again.append(torch.full((512, 4096), float("nan"), dtype=torch.bfloat16, device=DEV))
    torch.cuda.synchronize()
    y = torch.empty(3, 512, device=DEV)
    wf.wf_linear_w4(x, w, y)
    want = wf.wf_w4_quantize(w16.to(DEV))
    torch.cuda.synchronize()
    _check(x.cpu(), codes, scales, y, out="f32")
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    del again


def test_quantised_layer_of_its_own():
    """Quantise, then multiply: the product of what the codes hold."""
    w = _normal(1, 300, 768, std=0.02)
    x = _normal(2, 9, 768)
    held4, scales4 = wf.wf_w4_quantize(w.to(DEV))
    w4 = wf.W4Weight(held4, scales4)
    y = torch.empty(9, 300, dtype=torch.bfloat16, device=DEV)
    wf.wf_linear_w4(x.to(DEV), w4, y)
    torch.cuda.synchronize()
    _check(x, held4.cpu(), scales4.cpu(), y)
    # e2m1 holds a weight to half a step, at most a sixth of the group's largest
    held = R.decode_e2m1(held4.cpu().numpy(), scales4.cpu().numpy())
    big = w.double().abs().view(300, 24, 32).amax(2).repeat_interleave(32, 1).numpy()
    assert (np.abs(held - w.double().numpy()) <= big / 3).all()


def test_logits_feed_the_acceptance():
    """fp32 logits of a 4-bit LM head through the logits mode of the LM-head
    call: the argmax of the plain product where it is clear."""
    g, d, vocab = 16, 512, 5000
    codes, scales = _weight(3, vocab, d)
    h = _normal(4, g, d)
    logits = torch.empty(g, vocab, device=DEV)
    wf.wf_linear_w4(h.to(DEV), wf.W4Weight(codes.to(DEV), scales.to(DEV)), logits)
    am = torch.empty(g, dtype=torch.int32, device=DEV)
    ent, acc = torch.empty(g, device=DEV), torch.empty(3, dtype=torch.int32, device=DEV)
    ref = h.double() @ torch.from_numpy(R.decode_e2m1(codes.numpy(), scales.numpy())).t()
    draft = ref.argmax(1).to(torch.int32)[:g - 1].to(DEV)
    wf.wf_lmhead_accept_entropy(None, None, logits, draft, 1.0, am, ent, acc)
    torch.cuda.synchronize()
    assert am.cpu().tolist() == ref.argmax(1).tolist()
    assert acc[0].item() == g - 1
