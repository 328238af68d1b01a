"""Python binding of libwf, the MI355X verification-step library for WhiFlash
cross-paradigm speculative decoding (arXiv 2606.07710).

Argument marshalling only: every function passes torch tensors' device
pointers and the current HIP stream to the C ABI declared in include/wf.h,
and raises WfError on a non-OK status.  All computation runs in the HIP
kernels of libwf.so; there is no fallback path.  If the library has not been
built, importing this package raises ImportError.
"""
import contextlib
import ctypes
import operator
import os

import torch  # loaded first so libwf binds to the same HIP runtime as torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# WF_LIB names another build of the library (the host-sanitizer CPU run)
LIB_PATH = os.environ.get("WF_LIB") or os.path.join(_HERE, "libwf.so")

WF_OK, WF_ERR_INVALID_ARG, WF_ERR_UNSUPPORTED, WF_ERR_WORKSPACE, WF_ERR_HIP = range(5)
WF_F32, WF_BF16, WF_BF16_TILED = 0, 1, 2

EXPORTED_SYMBOLS = (
    "wf_abi_version", "wf_status_string", "wf_verify_attn",
    "wf_verify_attn_workspace_bytes", "wf_kv_only_prefill",
    "wf_lmhead_accept_entropy", "wf_lmhead_workspace_bytes",
    "wf_kv_only_prefill_workspace_bytes", "wf_verify_attn_tree",
    "wf_lmhead_accept_tree", "wf_kv_compact_path", "wf_router_neural",
    "wf_router_workspace_bytes", "wf_drafter_forward",
    "wf_drafter_forward_workspace_bytes", "wf_drafter_catchup",
    "wf_drafter_catchup_workspace_bytes", "wf_switch_init", "wf_switch_commit",
    "wf_kv_only_prefill_layers", "wf_kv_only_prefill_layers_workspace_bytes",
    "wf_tiled_weight_bytes", "wf_tile_weights", "wf_verify_attn_noalloc",
    "wf_read_probe", "wf_read_probe_series", "wf_lmhead_accept_route_neural",
    "wf_lmhead_route_neural_workspace_bytes",
    "wf_kv8_code_bytes", "wf_kv8_scale_bytes", "wf_kv8_append", "wf_kv8_only_prefill",
    "wf_kv8_only_prefill_workspace_bytes", "wf_kv8_verify_attn", "wf_kv8_verify_attn_tree",
    "wf_kv8_verify_attn_workspace_bytes", "wf_kv8_compact_path", "wf_w4_quantize",
    "wf_w4_packed_bytes", "wf_w4_pack", "wf_linear_w4", "wf_linear_w4_workspace_bytes",
    "wf_paged_append", "wf_paged_verify_attn", "wf_paged_verify_attn_workspace_bytes",
    "wf_paged_select", "wf_paged_select_workspace_bytes", "wf_paged_sparse_attn",
    "wf_paged_sparse_attn_workspace_bytes", "wf_token_logprobs",
    "wf_token_logprobs_workspace_bytes",
)
KV8_BLOCK = 32                       # WF_KV8_BLOCK
# what the low-bit calls take as e4m3 elements, power-of-two scales, e2m1 pairs
E4M3_BYTES = (torch.uint8, torch.float8_e4m3fn)
E8M0_BYTES = (torch.uint8, torch.float8_e8m0fnu)
E2M1_BYTES = (torch.uint8, torch.float4_e2m1fn_x2)
NOALLOC_SCRATCH_BYTES = 32 << 20     # WF_NOALLOC_SCRATCH_BYTES
WF_DRAFTER_AR, WF_DRAFTER_DIFFUSION = 0, 1

DECODER_WEIGHTS = ("attn_norm", "w_q", "w_k", "w_v", "w_o", "mlp_norm",
                   "w_gate", "w_up", "w_down")


class DecoderLayer(ctypes.Structure):
    """wf_decoder_layer_t: device pointers of a drafter layer's weights and
    its shape."""
    _fields_ = [(n, ctypes.c_void_p) for n in DECODER_WEIGHTS] + [
        ("hidden", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
        ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("inter", ctypes.c_int32), ("rms_eps", ctypes.c_float),
        ("rope_base", ctypes.c_double)]


class Kv8CacheStruct(ctypes.Structure):
    """wf_kv8_cache_t: device pointers of one layer's 8-bit KV cache and its
    shape."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n_kv_heads", ctypes.c_int32), ("cap", ctypes.c_int32),
                ("head_dim", ctypes.c_int32)]


class PagedCacheStruct(ctypes.Structure):
    """wf_paged_cache_t: device pointers of one layer's pool of pages and its
    shape."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("bounds", ctypes.c_void_p),
                ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class PagedBatchStruct(ctypes.Structure):
    """wf_paged_batch_t: device pointers of a batch's lists and their sizes."""
    _fields_ = [("page_table", ctypes.c_void_p), ("row_start", ctypes.c_void_p),
                ("ctx_len", ctypes.c_void_p), ("n_seqs", ctypes.c_int32),
                ("max_pages", ctypes.c_int32), ("max_rows", ctypes.c_int32)]


class SwitchState(ctypes.Structure):
    """wf_switch_state_t: host-side lazy catch-up bookkeeping."""
    _fields_ = [("active", ctypes.c_int32), ("lazy", ctypes.c_int32),
                ("committed", ctypes.c_int32), ("ar_cache_len", ctypes.c_int32),
                ("switches", ctypes.c_int32), ("max_backlog", ctypes.c_int32),
                ("caught_up", ctypes.c_int64), ("catchups", ctypes.c_int64)]


class WfError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} (status {status})")


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with "
            "`python -c 'import __graft_entry__ as g; g.build()'`")
    lib = ctypes.CDLL(LIB_PATH)
    p, i32, sz, f32, f64 = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t,
                            ctypes.c_float, ctypes.c_double)
    lib.wf_abi_version.restype = i32
    lib.wf_status_string.argtypes = [i32]
    lib.wf_status_string.restype = ctypes.c_char_p
    lib.wf_verify_attn.argtypes = [i32, p, p, p, p, i32, i32, i32, i32, i32,
                                   i32, f32, i32, p, sz, p]
    lib.wf_verify_attn.restype = i32
    lib.wf_verify_attn_noalloc.argtypes = [i32, p, p, p, p, i32, i32, i32, i32, i32,
                                           i32, f32, i32, p]
    lib.wf_verify_attn_noalloc.restype = i32
    lib.wf_verify_attn_workspace_bytes.argtypes = [i32, i32, i32, i32, i32,
                                                   i32, i32]
    lib.wf_verify_attn_workspace_bytes.restype = sz
    lib.wf_kv_only_prefill.argtypes = [i32, p, p, p, p, p, i32, i32, i32, i32,
                                       i32, i32, f64, p, sz, p]
    lib.wf_kv_only_prefill.restype = i32
    lib.wf_kv_only_prefill_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
    lib.wf_kv_only_prefill_workspace_bytes.restype = sz
    lib.wf_lmhead_accept_entropy.argtypes = [i32, p, p, p, p, i32, i32, i32,
                                             f32, p, p, p, p, sz, p]
    lib.wf_lmhead_accept_entropy.restype = i32
    lib.wf_lmhead_workspace_bytes.argtypes = [i32, i32]
    lib.wf_lmhead_workspace_bytes.restype = sz
    lib.wf_verify_attn_tree.argtypes = [i32, p, p, p, p, p, i32, i32, i32,
                                        i32, i32, i32, f32, i32, p, sz, p]
    lib.wf_verify_attn_tree.restype = i32
    lib.wf_lmhead_accept_tree.argtypes = [i32, p, p, p, p, p, i32, i32, i32,
                                          f32, p, p, p, p, p, sz, p]
    lib.wf_lmhead_accept_tree.restype = i32
    lib.wf_kv_compact_path.argtypes = [i32, p, p, p, p, i32, i32, i32, i32,
                                       i32, i32, sz, p]
    lib.wf_kv_compact_path.restype = i32
    lib.wf_router_neural.argtypes = [i32, p, p, p, p, p, p, i32, i32, i32, f32,
                                     p, p, p, sz, p]
    lib.wf_router_neural.restype = i32
    lib.wf_router_workspace_bytes.argtypes = [i32, i32, i32, i32]
    lib.wf_router_workspace_bytes.restype = sz
    for name in ("wf_drafter_forward", "wf_drafter_catchup"):
        fn = getattr(lib, name)
        fn.argtypes = [i32, p, p, i32, i32, p, p, i32, p, p, sz, p]
        fn.restype = i32
        q = getattr(lib, name + "_workspace_bytes")
        q.argtypes = [i32, p, i32, i32]
        q.restype = sz
    lib.wf_kv_only_prefill_layers.argtypes = [i32, p, p, p, p, p, i32, i32, i32, i32,
                                              i32, i32, f64, i32, sz, sz, sz, p, sz, p]
    lib.wf_kv_only_prefill_layers.restype = i32
    lib.wf_kv_only_prefill_layers_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32]
    lib.wf_kv_only_prefill_layers_workspace_bytes.restype = sz
    lib.wf_tiled_weight_bytes.argtypes = [i32, i32]
    lib.wf_tiled_weight_bytes.restype = sz
    lib.wf_tile_weights.argtypes = [p, i32, i32, p, sz, p]
    lib.wf_tile_weights.restype = i32
    lib.wf_lmhead_accept_route_neural.argtypes = [i32, p, p, p, i32, i32, i32, p, p, p, p,
                                                  i32, f32, p, p, p, p, p, sz, p]
    lib.wf_lmhead_accept_route_neural.restype = i32
    lib.wf_lmhead_route_neural_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
    lib.wf_lmhead_route_neural_workspace_bytes.restype = sz
    lib.wf_kv8_code_bytes.argtypes = [i32, i32, i32]
    lib.wf_kv8_code_bytes.restype = sz
    lib.wf_kv8_scale_bytes.argtypes = [i32, i32]
    lib.wf_kv8_scale_bytes.restype = sz
    lib.wf_kv8_append.argtypes = [i32, p, p, p, i32, i32, sz, sz, p]
    lib.wf_kv8_append.restype = i32
    lib.wf_kv8_only_prefill.argtypes = [i32, p, p, p, p, i32, i32, i32, f64, p, sz, p]
    lib.wf_kv8_only_prefill.restype = i32
    lib.wf_kv8_only_prefill_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
    lib.wf_kv8_only_prefill_workspace_bytes.restype = sz
    lib.wf_kv8_verify_attn.argtypes = [i32, p, p, p, i32, i32, i32, f32, i32, p, sz, p]
    lib.wf_kv8_verify_attn.restype = i32
    lib.wf_kv8_verify_attn_tree.argtypes = [i32, p, p, p, p, i32, i32, i32, f32, i32, p, sz, p]
    lib.wf_kv8_verify_attn_tree.restype = i32
    lib.wf_kv8_verify_attn_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32, i32]
    lib.wf_kv8_verify_attn_workspace_bytes.restype = sz
    lib.wf_kv8_compact_path.argtypes = [p, p, p, i32, i32, i32, sz, sz, p]
    lib.wf_kv8_compact_path.restype = i32
    lib.wf_w4_quantize.argtypes = [p, i32, i32, p, p, p]
    lib.wf_w4_quantize.restype = i32
    lib.wf_w4_packed_bytes.argtypes = [i32, i32]
    lib.wf_w4_packed_bytes.restype = sz
    lib.wf_w4_pack.argtypes = [p, p, i32, i32, p, sz, p]
    lib.wf_w4_pack.restype = i32
    lib.wf_linear_w4.argtypes = [p, p, p, i32, p, i32, i32, i32, p, sz, p]
    lib.wf_linear_w4.restype = i32
    lib.wf_linear_w4_workspace_bytes.argtypes = [i32, i32, i32]
    lib.wf_linear_w4_workspace_bytes.restype = sz
    lib.wf_paged_append.argtypes = [i32, p, p, p, p, sz, p, sz, p, i32, p, f64, i32, p]
    lib.wf_paged_append.restype = i32
    lib.wf_paged_verify_attn.argtypes = [i32, p, p, p, p, p, i32, i32, f32, p, sz, p]
    lib.wf_paged_verify_attn.restype = i32
    lib.wf_paged_verify_attn_workspace_bytes.argtypes = [i32] * 7
    lib.wf_paged_verify_attn_workspace_bytes.restype = sz
    lib.wf_paged_select.argtypes = [i32, p, p, p, p, i32, i32, i32, i32, p, sz, p]
    lib.wf_paged_select.restype = i32
    lib.wf_paged_select_workspace_bytes.argtypes = [i32] * 3
    lib.wf_paged_select_workspace_bytes.restype = sz
    lib.wf_paged_sparse_attn.argtypes = [i32, p, p, p, p, i32, p, p, i32, i32, f32, p, sz, p]
    lib.wf_paged_sparse_attn.restype = i32
    lib.wf_paged_sparse_attn_workspace_bytes.argtypes = [i32] * 7
    lib.wf_paged_sparse_attn_workspace_bytes.restype = sz
    lib.wf_token_logprobs.argtypes = [i32, p, sz, p, i32, i32, i32, p, p, p, p, p, p, sz, p]
    lib.wf_token_logprobs.restype = i32
    lib.wf_token_logprobs_workspace_bytes.argtypes = [i32] * 4
    lib.wf_token_logprobs_workspace_bytes.restype = sz
    lib.wf_read_probe.argtypes = [p, sz, p, sz, i32, p]
    lib.wf_read_probe.restype = i32
    lib.wf_read_probe_series.argtypes = [p, sz, sz, i32, i32, p, sz, i32, i32, p]
    lib.wf_read_probe_series.restype = i32
    lib.wf_switch_init.argtypes = [p, i32, i32, i32]
    lib.wf_switch_init.restype = i32
    lib.wf_switch_commit.argtypes = [p, i32, i32, p, p]
    lib.wf_switch_commit.restype = i32
    return lib


lib = _load()


def status_string(status: int) -> str:
    return lib.wf_status_string(int(status)).decode()


def abi_version() -> int:
    return int(lib.wf_abi_version())


class TiledWeight:
    """A bf16 weight (or a [L] stack of them) in the tiled layout that
    wf_tile_weights writes: `data` [L?][n] holds the tiles, `shape` is the
    logical [L?][rows][cols].  Passed wherever a weight is, it selects
    WF_BF16_TILED."""

    def __init__(self, data, shape):
        self.data, self.shape = data, tuple(shape)
        self.dtype, self.device, self.is_cuda = data.dtype, data.device, data.is_cuda

    def data_ptr(self):
        return self.data.data_ptr()

    def is_contiguous(self):
        return self.data.is_contiguous()

    def stride(self, dim):
        if dim != 0 or len(self.shape) != 3:
            raise ValueError("layer stride of a tiled stack only")
        return self.data.stride(0)


def wf_tiled_weight_bytes(rows, cols) -> int:
    return int(lib.wf_tiled_weight_bytes(int(rows), int(cols)))


def tile_weights(w, stream=None) -> TiledWeight:
    """Tiled copy of a bf16 weight [rows][cols] or stack [L][rows][cols]."""
    if w.dtype != torch.bfloat16:
        raise TypeError("tiled weights are bf16")
    rows, cols = w.shape[-2:]
    n = wf_tiled_weight_bytes(rows, cols) // 2
    if n == 0:
        raise ValueError(f"cannot tile a [{rows}][{cols}] weight (cols % 32 != 0)")
    layers = w.shape[0] if w.dim() == 3 else None
    out = torch.empty((layers, n) if layers else (n,), dtype=torch.bfloat16, device=w.device)
    for l in range(layers or 1):
        src, dst = (w[l], out[l]) if layers else (w, out)
        _check(lib.wf_tile_weights(_dev(src, "w"), rows, cols, _dev(dst, "tiled"), 2 * n,
                                   _stream(stream)), "wf_tile_weights")
    return TiledWeight(out, w.shape)


def _weight_code(x, *ws) -> int:
    """dtype code of a call whose activations are x and weights ws."""
    tiled = n = 0
    for w in ws:
        if w is not None:
            n += 1
            tiled += isinstance(w, TiledWeight)
    if tiled:
        if tiled != n or x.dtype != torch.bfloat16:
            raise TypeError("tiled weights: all weights tiled, bf16 activations")
        return WF_BF16_TILED
    return _dtype_code(x)


_DTYPE_CODES = {torch.float32: WF_F32, torch.bfloat16: WF_BF16}


def _dtype_code(t: torch.Tensor) -> int:
    code = _DTYPE_CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {t.dtype}; use float32 or bfloat16")
    return code


def _dev(t, name):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


# The current device's current stream as a raw handle: torch.cuda's own
# current_stream() builds a Stream object around it, 2.7 us of a call that
# takes about 3 on the host besides its kernel launches.  The getters are
# private to torch: a torch without them takes the public way.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)
if _raw_stream is None or _device is None:
    def _raw_stream(_):
        return torch.cuda.current_stream().cuda_stream

    def _device():
        return None


def _stream(stream):
    return stream.cuda_stream if stream is not None else _raw_stream(_device())


def _current():
    """The current device's index, and its current stream as a raw handle."""
    dev = _device()
    if dev is None:
        dev = torch.cuda.current_device()
    return dev, _raw_stream(dev)


def _at(stream):
    """(device index, raw stream) of a low-bit call: its tensors lie on the
    current device, the stream is the one given or that device's current one."""
    dev, raw = _current()
    if stream is None:
        return dev, raw
    if getattr(stream, "device_index", dev) != dev:
        raise ValueError("the stream must be one of the current device")
    return dev, stream.cuda_stream


def _on(stream):
    """Where a low-bit call allocates: on the stream that it launches on, so
    that memory freed there before is not written too early."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _hold(stream, *tensors):
    """Keeps the memory of tensors that the caller may drop at once from being
    given out again before `stream`, on which a low-bit call reads them, gets
    there (their own allocations follow the stream they were made on)."""
    if stream is not None:
        for t in tensors:
            t.record_stream(stream)


def _ptr(t, dev, name):
    """Pointer of a dense tensor of device `dev` (None: null)."""
    if t is None:
        return None
    if t.get_device() != dev:
        raise ValueError(f"{name} must be a tensor on the current device")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _check(status, what):
    if status != WF_OK:
        raise WfError(status, what)


def wf_verify_attn_workspace_bytes(dtype, gamma, ctx_len, n_q_heads,
                                   n_kv_heads, head_dim, num_splits=0) -> int:
    code = dtype if isinstance(dtype, int) else (
        WF_F32 if dtype == torch.float32 else WF_BF16)
    return int(lib.wf_verify_attn_workspace_bytes(
        code, gamma, ctx_len, n_q_heads, n_kv_heads, head_dim, num_splits))


def wf_lmhead_workspace_bytes(gamma, vocab) -> int:
    return int(lib.wf_lmhead_workspace_bytes(gamma, vocab))


def alloc_workspace(nbytes: int, device) -> torch.Tensor:
    """Caller-owned scratch for the workspace arguments: 16-byte aligned and
    zero-filled, as the calls require before a workspace's first use (each
    call leaves its arrival counters at zero again, so one workspace serves
    any number of calls that do not overlap in time)."""
    return torch.zeros(max(16, (nbytes + 15) // 16 * 16), dtype=torch.uint8,
                       device=device)


def _attn_shapes(q, k_cache, v_cache, out):
    shape = q.shape
    gamma, hq, dh = shape
    kshape = k_cache.shape
    hkv, cap, dh2 = kshape
    if dh2 != dh or v_cache.shape != kshape:
        raise ValueError("cache shapes do not match q")
    if out.shape != shape or out.dtype != q.dtype:
        raise ValueError("out must match q in shape and dtype")
    return gamma, hq, dh, hkv, cap


def wf_verify_attn(q, k_cache, v_cache, out, ctx_len, softmax_scale=None,
                   num_splits=0, workspace=None, stream=None):
    """q [gamma][Hq][D]; k_cache, v_cache [Hkv][cap][D]; out like q."""
    gamma, hq, dh, hkv, cap = _attn_shapes(q, k_cache, v_cache, out)
    code = _dtype_code(q)
    if softmax_scale is None:
        softmax_scale = dh ** -0.5
    if workspace is None:
        workspace = alloc_workspace(wf_verify_attn_workspace_bytes(
            code, gamma, ctx_len, hq, hkv, dh, num_splits), q.device)
    st = lib.wf_verify_attn(code, _dev(q, "q"), _dev(k_cache, "k_cache"),
                            _dev(v_cache, "v_cache"), _dev(out, "out"), gamma,
                            ctx_len, cap, hq, hkv, dh,
                            float(softmax_scale), num_splits,
                            _dev(workspace, "workspace"), workspace.numel(),
                            _stream(stream))
    _check(st, "wf_verify_attn")
    return out


def wf_verify_attn_noalloc(q, k_cache, v_cache, out, ctx_len, softmax_scale=None,
                           num_splits=0, stream=None):
    """wf_verify_attn with the library's static device scratch instead of a
    workspace: nothing is allocated (for graph capture and callers that
    cannot allocate).  Calls that overlap in time on one GPU race."""
    gamma, hq, dh, hkv, cap = _attn_shapes(q, k_cache, v_cache, out)
    if softmax_scale is None:
        softmax_scale = dh ** -0.5
    st = lib.wf_verify_attn_noalloc(_dtype_code(q), _dev(q, "q"), _dev(k_cache, "k_cache"),
                                    _dev(v_cache, "v_cache"), _dev(out, "out"), gamma,
                                    int(ctx_len), cap, hq, hkv, dh, float(softmax_scale),
                                    int(num_splits), _stream(stream))
    _check(st, "wf_verify_attn_noalloc")
    return out


def wf_kv_only_prefill_workspace_bytes(dtype, n_tok, d_in, n_kv_heads,
                                       head_dim) -> int:
    code = dtype if isinstance(dtype, int) else (
        WF_F32 if dtype == torch.float32 else WF_BF16)
    return int(lib.wf_kv_only_prefill_workspace_bytes(code, n_tok, d_in,
                                                      n_kv_heads, head_dim))


def wf_kv_only_prefill(x, w_k, w_v, k_cache, v_cache, start_pos, rope_base,
                       workspace=None, stream=None):
    """x [n][d_in]; w_k, w_v [Hkv*D][d_in]; caches [Hkv][cap][D]."""
    n_tok, d_in = x.shape
    hkv, cap, dh = k_cache.shape
    code = _weight_code(x, w_k, w_v)
    if workspace is None:
        need = wf_kv_only_prefill_workspace_bytes(code, n_tok, d_in, hkv, dh)
        workspace = alloc_workspace(need, x.device) if need else None
    st = lib.wf_kv_only_prefill(code, _dev(x, "x"), _dev(w_k, "w_k"),
                                _dev(w_v, "w_v"), _dev(k_cache, "k_cache"),
                                _dev(v_cache, "v_cache"), n_tok,
                                int(start_pos), cap, d_in, hkv, dh,
                                float(rope_base), _dev(workspace, "workspace"),
                                workspace.numel() if workspace is not None else 0,
                                _stream(stream))
    _check(st, "wf_kv_only_prefill")


def wf_kv_only_prefill_layers_workspace_bytes(dtype, n_tok, d_in, n_kv_heads, head_dim,
                                              n_layers) -> int:
    code = dtype if isinstance(dtype, int) else (
        WF_F32 if dtype == torch.float32 else WF_BF16)
    return int(lib.wf_kv_only_prefill_layers_workspace_bytes(code, n_tok, d_in, n_kv_heads,
                                                             head_dim, n_layers))


def wf_kv_only_prefill_layers(x, w_k, w_v, k_cache, v_cache, start_pos, rope_base,
                              workspace=None, stream=None):
    """x [L][n][d_in]; w_k, w_v [L][Hkv*D][d_in]; caches [L][Hkv][cap][D]
    (each a dense stack, so the layer strides are those of dim 0)."""
    n_layers, n_tok, d_in = x.shape
    _, hkv, cap, dh = k_cache.shape
    if w_k.shape[0] != n_layers or v_cache.stride(0) != k_cache.stride(0) or \
            w_v.stride(0) != w_k.stride(0) or k_cache.shape[0] != n_layers:
        raise ValueError("layer stacks must match")
    code = _weight_code(x, w_k, w_v)
    if workspace is None:
        need = wf_kv_only_prefill_layers_workspace_bytes(code, n_tok, d_in, hkv, dh, n_layers)
        workspace = alloc_workspace(need, x.device) if need else None
    st = lib.wf_kv_only_prefill_layers(
        code, _dev(x, "x"), _dev(w_k, "w_k"), _dev(w_v, "w_v"), _dev(k_cache, "k_cache"),
        _dev(v_cache, "v_cache"), n_tok, int(start_pos), cap, d_in, hkv, dh,
        float(rope_base), n_layers, x.stride(0), w_k.stride(0), k_cache.stride(0),
        _dev(workspace, "workspace"), workspace.numel() if workspace is not None else 0,
        _stream(stream))
    _check(st, "wf_kv_only_prefill_layers")


def wf_lmhead_accept_entropy(h, w_lm, logits, draft, tau, argmax_out,
                             entropy_out, accept_out, workspace=None,
                             stream=None, gamma=None, vocab=None):
    """Either (h [gamma][d], w_lm [vocab][d]) or logits [gamma][vocab] fp32.
    draft [gamma-1] int32 (None when gamma == 1); outputs int32 [gamma],
    fp32 [gamma], int32 [3]."""
    if logits is not None:
        gamma, vocab = logits.shape
        d, code = 0, WF_F32
    else:
        gamma, d = h.shape
        vocab = w_lm.shape[0]
        code = _weight_code(h, w_lm)
    if workspace is None:
        workspace = alloc_workspace(wf_lmhead_workspace_bytes(gamma, vocab),
                                    (logits if logits is not None else h).device)
    st = lib.wf_lmhead_accept_entropy(
        code, _dev(h, "h"), _dev(w_lm, "w_lm"), _dev(logits, "logits"),
        _dev(draft, "draft"), gamma, d, vocab, float(tau),
        _dev(argmax_out, "argmax_out"), _dev(entropy_out, "entropy_out"),
        _dev(accept_out, "accept_out"), _dev(workspace, "workspace"),
        workspace.numel(), _stream(stream))
    _check(st, "wf_lmhead_accept_entropy")


def wf_verify_attn_tree(q, k_cache, v_cache, out, ctx_len, tree_mask,
                        softmax_scale=None, num_splits=0, workspace=None,
                        stream=None):
    """Tree verification attention: tree_mask [gamma] int64/uint64 device
    tensor (bit j of row i: row i sees block row j); else as wf_verify_attn."""
    gamma, hq, dh, hkv, cap = _attn_shapes(q, k_cache, v_cache, out)
    if tree_mask.numel() != gamma or tree_mask.element_size() != 8:
        raise ValueError("tree_mask must hold gamma 64-bit words")
    code = _dtype_code(q)
    if softmax_scale is None:
        softmax_scale = dh ** -0.5
    if workspace is None:
        workspace = alloc_workspace(wf_verify_attn_workspace_bytes(
            code, gamma, ctx_len, hq, hkv, dh, num_splits), q.device)
    st = lib.wf_verify_attn_tree(code, _dev(q, "q"), _dev(k_cache, "k_cache"),
                                 _dev(v_cache, "v_cache"), _dev(out, "out"),
                                 _dev(tree_mask, "tree_mask"), gamma,
                                 ctx_len, cap, hq, hkv, dh,
                                 float(softmax_scale), num_splits,
                                 _dev(workspace, "workspace"),
                                 workspace.numel(), _stream(stream))
    _check(st, "wf_verify_attn_tree")
    return out


def wf_lmhead_accept_route_neural(h, w_lm, draft, w1, b1, w2, b2, tau_neural, argmax_out,
                                  entropy_out, accept_out, delta_out, workspace=None,
                                  stream=None):
    """h [gamma][d]; w_lm [vocab][d] and w1 [m][d] (both tiled or both
    row-major); b1, w2 [m], b2 [1]; draft [gamma-1] int32 (None when gamma
    == 1); outputs int32 [gamma], fp32 [gamma], int32 [3] (route: the neural
    policy), fp32 [gamma] (predicted gain per row)."""
    gamma, d = h.shape
    vocab = w_lm.shape[0]
    m = w1.shape[0]
    code = _weight_code(h, w_lm, w1)
    if workspace is None:
        workspace = alloc_workspace(int(lib.wf_lmhead_route_neural_workspace_bytes(
            code, gamma, vocab, d, m)), h.device)
    st = lib.wf_lmhead_accept_route_neural(
        code, _dev(h, "h"), _dev(w_lm, "w_lm"), _dev(draft, "draft"), gamma, d, vocab,
        _dev(w1, "w1"), _dev(b1, "b1"), _dev(w2, "w2"), _dev(b2, "b2"), m, float(tau_neural),
        _dev(argmax_out, "argmax_out"), _dev(entropy_out, "entropy_out"),
        _dev(accept_out, "accept_out"), _dev(delta_out, "delta_out"),
        _dev(workspace, "workspace"), workspace.numel(), _stream(stream))
    _check(st, "wf_lmhead_accept_route_neural")


def wf_lmhead_accept_tree(h, w_lm, logits, tokens, parents, tau, argmax_out,
                          entropy_out, accept_out, path_out, workspace=None,
                          stream=None):
    """Either (h [gamma][d], w_lm [vocab][d]) or logits [gamma][vocab] fp32;
    tokens, parents [gamma] int32; outputs int32 [gamma], fp32 [gamma],
    int32 [4], int32 [gamma]."""
    if logits is not None:
        gamma, vocab = logits.shape
        d, code = 0, WF_F32
    else:
        gamma, d = h.shape
        vocab = w_lm.shape[0]
        code = _weight_code(h, w_lm)
    if workspace is None:
        workspace = alloc_workspace(wf_lmhead_workspace_bytes(gamma, vocab),
                                    (logits if logits is not None else h).device)
    st = lib.wf_lmhead_accept_tree(
        code, _dev(h, "h"), _dev(w_lm, "w_lm"), _dev(logits, "logits"),
        _dev(tokens, "tokens"), _dev(parents, "parents"), gamma, d, vocab,
        float(tau), _dev(argmax_out, "argmax_out"),
        _dev(entropy_out, "entropy_out"), _dev(accept_out, "accept_out"),
        _dev(path_out, "path_out"), _dev(workspace, "workspace"),
        workspace.numel(), _stream(stream))
    _check(st, "wf_lmhead_accept_tree")


def wf_kv_compact_path(k_cache, v_cache, accept, path, ctx_len, stream=None):
    """Caches [Hkv][cap][D] (one layer) or [L][Hkv][cap][D] (all layers);
    accept (n at [0]) and path [gamma] int32 device tensors, as written by
    wf_lmhead_accept_tree."""
    if tuple(v_cache.shape) != tuple(k_cache.shape) or v_cache.dtype != k_cache.dtype:
        raise ValueError("k_cache and v_cache must match")
    if k_cache.dim() == 4:
        n_layers, hkv, cap, dh = k_cache.shape
        stride = hkv * cap * dh
    else:
        (hkv, cap, dh), n_layers, stride = k_cache.shape, 1, 0
    gamma = path.numel()
    st = lib.wf_kv_compact_path(_dtype_code(k_cache), _dev(k_cache, "k_cache"),
                                _dev(v_cache, "v_cache"), _dev(accept, "accept"),
                                _dev(path, "path"), gamma, int(ctx_len), cap,
                                hkv, dh, n_layers, stride, _stream(stream))
    _check(st, "wf_kv_compact_path")


def wf_router_neural(h, w1, b1, w2, b2, row, tau, delta_out, route_out,
                     workspace=None, stream=None):
    """h [gamma][d]; w1 [m][d]; b1, w2 [m]; b2 [1] (one dtype); row: int32
    device tensor holding the row to route on; outputs fp32 [gamma] and
    int32 [1]."""
    gamma, d = h.shape
    m = w1.shape[0]
    code = _dtype_code(h)
    if workspace is None:
        workspace = alloc_workspace(int(lib.wf_router_workspace_bytes(code, gamma, d, m)),
                                    h.device)
    st = lib.wf_router_neural(code, _dev(h, "h"), _dev(w1, "w1"), _dev(b1, "b1"),
                              _dev(w2, "w2"), _dev(b2, "b2"), _dev(row, "row"),
                              gamma, d, m, float(tau), _dev(delta_out, "delta_out"),
                              _dev(route_out, "route_out"),
                              _dev(workspace, "workspace"), workspace.numel(),
                              _stream(stream))
    _check(st, "wf_router_neural")


def decoder_layer(weights, n_q_heads, n_kv_heads, rms_eps, rope_base):
    """DecoderLayer from a dict of DECODER_WEIGHTS device tensors (bf16)."""
    w_q, w_k, w_gate = weights["w_q"], weights["w_k"], weights["w_gate"]
    head_dim = w_q.shape[0] // n_q_heads
    if w_k.shape[0] != n_kv_heads * head_dim:
        raise ValueError("w_k rows must be n_kv_heads * head_dim")
    for n in DECODER_WEIGHTS:
        if weights[n] is None:
            raise ValueError(f"{n} is missing")
    layer = DecoderLayer(*[_dev(weights[n], n) for n in DECODER_WEIGHTS],
                         w_q.shape[1], n_q_heads, n_kv_heads, head_dim,
                         w_gate.shape[0], float(rms_eps), float(rope_base))
    # the struct holds raw device pointers: keep the tensors alive with it
    layer.keepalive = dict(weights)
    # projections tiled (wf_tile_weights) -> the calls pass WF_BF16_TILED
    mats = [weights[n] for n in DECODER_WEIGHTS if not n.endswith("norm")]
    layer.tiled = all(isinstance(m, TiledWeight) for m in mats)
    if not layer.tiled and any(isinstance(m, TiledWeight) for m in mats):
        raise TypeError("tile all seven projections or none")
    return layer


def wf_drafter_forward_workspace_bytes(layer, n_tok, pos) -> int:
    """Workspace of a bf16 wf_drafter_forward call (0: shapes rejected)."""
    code = WF_BF16_TILED if getattr(layer, "tiled", False) else WF_BF16
    return int(lib.wf_drafter_forward_workspace_bytes(code, ctypes.byref(layer),
                                                      int(n_tok), int(pos)))


def wf_drafter_catchup_workspace_bytes(layer, n_backlog, pos) -> int:
    """Workspace of a bf16 wf_drafter_catchup call (0: shapes rejected)."""
    code = WF_BF16_TILED if getattr(layer, "tiled", False) else WF_BF16
    return int(lib.wf_drafter_catchup_workspace_bytes(code, ctypes.byref(layer),
                                                      int(n_backlog), int(pos)))


def wf_drafter_forward(layer, r, pos, k_cache, v_cache, out, workspace=None,
                       stream=None):
    """layer: DecoderLayer; r, out [n_tok][hidden]; caches [Hkv][cap][D]."""
    n_tok = r.shape[0]
    code = WF_BF16_TILED if getattr(layer, "tiled", False) else _dtype_code(r)
    if workspace is None:
        workspace = alloc_workspace(int(lib.wf_drafter_forward_workspace_bytes(
            code, ctypes.byref(layer), n_tok, int(pos))), r.device)
    st = lib.wf_drafter_forward(code, ctypes.byref(layer), _dev(r, "r"), n_tok, int(pos),
                                _dev(k_cache, "k_cache"), _dev(v_cache, "v_cache"),
                                k_cache.shape[1], _dev(out, "out"),
                                _dev(workspace, "workspace"), workspace.numel(),
                                _stream(stream))
    _check(st, "wf_drafter_forward")
    return out


def wf_drafter_catchup(layer, r, pos, k_cache, v_cache, out, workspace=None,
                       stream=None):
    """layer: DecoderLayer; r [n_backlog][hidden]; out [hidden]."""
    n = r.shape[0]
    code = WF_BF16_TILED if getattr(layer, "tiled", False) else _dtype_code(r)
    if workspace is None:
        workspace = alloc_workspace(int(lib.wf_drafter_catchup_workspace_bytes(
            code, ctypes.byref(layer), n, int(pos))), r.device)
    st = lib.wf_drafter_catchup(code, ctypes.byref(layer), _dev(r, "r"), n, int(pos),
                                _dev(k_cache, "k_cache"), _dev(v_cache, "v_cache"),
                                k_cache.shape[1], _dev(out, "out"),
                                _dev(workspace, "workspace"), workspace.numel(),
                                _stream(stream))
    _check(st, "wf_drafter_catchup")
    return out


class Kv8Cache:
    """An 8-bit KV cache of one layer, or of a stack of layers (wf.h: e4m3
    codes, one power-of-two scale byte per 32 tokens and KV head).

    k        [L?][Hkv][blocks][32][D] uint8 (or float8_e4m3fn) codes
    v        [L?][Hkv][blocks][D][32], each block transposed
    k_scale, v_scale  [L?][Hkv][blocks] uint8 (or float8_e8m0fnu)
    cap      rows per head; blocks = ceil(cap / 32)

    The calls on one layer take a cache without L; layer(l) is one layer of a
    stack (a view of its memory).  The tensors stay the ones it was made of (the
    calls hold their addresses); a deep copy has its own."""

    def __init__(self, k, v, k_scale, v_scale, cap):
        cap = operator.index(cap)
        shape, blocks = tuple(k.shape), (cap + KV8_BLOCK - 1) // KV8_BLOCK
        if len(shape) not in (4, 5) or cap < 1:
            raise ValueError("k must be [L?][Hkv][blocks][32][D]")
        lead, (b, rows, dh) = shape[:-3], shape[-3:]
        if b != blocks or rows != KV8_BLOCK or tuple(v.shape) != lead + (b, dh, rows) or \
                tuple(k_scale.shape) != lead + (b,) or tuple(v_scale.shape) != lead + (b,):
            raise ValueError("cache shapes do not match each other and cap")
        if k.dtype not in E4M3_BYTES or v.dtype not in E4M3_BYTES:
            raise ValueError("k and v are uint8 or float8_e4m3fn")
        if k_scale.dtype not in E8M0_BYTES or v_scale.dtype not in E8M0_BYTES:
            raise ValueError("scales are uint8 or float8_e8m0fnu")
        dev = k.get_device()
        if dev < 0:
            raise ValueError("the cache must be device memory")
        self._tensors = k, v, k_scale, v_scale
        self.n_layers = lead[0] if len(lead) == 2 else None
        self.n_kv_heads, self.cap, self.head_dim, self.device = lead[-1], cap, dh, k.device
        self.struct = Kv8CacheStruct(_ptr(k, dev, "k"), _ptr(v, dev, "v"),
                                     _ptr(k_scale, dev, "k_scale"),
                                     _ptr(v_scale, dev, "v_scale"), lead[-1], cap, dh)
        self.ref, self.dev = ctypes.byref(self.struct), dev

    k = property(lambda self: self._tensors[0])
    v = property(lambda self: self._tensors[1])
    k_scale = property(lambda self: self._tensors[2])
    v_scale = property(lambda self: self._tensors[3])

    def __reduce__(self):
        return Kv8Cache, (*self._tensors, self.cap)

    def layer(self, l):
        if self.n_layers is None:
            raise ValueError("one layer only")
        return Kv8Cache(self.k[l], self.v[l], self.k_scale[l], self.v_scale[l], self.cap)


def alloc_kv8_cache(n_kv_heads, cap, head_dim, device, n_layers=None) -> Kv8Cache:
    """An empty 8-bit KV cache (zeros) of one layer or of n_layers."""
    blocks = (cap + KV8_BLOCK - 1) // KV8_BLOCK
    lead = (n_kv_heads,) if n_layers is None else (n_layers, n_kv_heads)
    z = [torch.zeros(lead + s, dtype=torch.uint8, device=device)
         for s in ((blocks, KV8_BLOCK, head_dim), (blocks, head_dim, KV8_BLOCK), (blocks,),
                   (blocks,))]
    z[2].fill_(127)
    z[3].fill_(127)
    return Kv8Cache(*z, cap)


def _one_layer(cache, dev):
    if cache.n_layers is not None:
        raise ValueError("the call takes one layer of the cache: cache.layer(l)")
    if cache.dev != dev:
        raise ValueError("the cache must be on the current device")
    return cache.ref


def wf_kv8_append(k, v, cache, start_pos, stream=None):
    """k, v [n][Hkv][D] (bf16 or fp32) into cache rows start_pos .. of every
    head.  The last dimension is dense; the others may be strided (alike for
    k and v, in multiples of 16 bytes), as in a transposed [Hkv][n][D]."""
    dev, raw = _at(stream)
    shape = k.shape
    n, hkv, dh = shape
    code = _dtype_code(k)
    if v.shape != shape or v.dtype != k.dtype or hkv != cache.n_kv_heads or \
            dh != cache.head_dim:
        raise ValueError("k and v must match each other and the cache")
    ks, vs = k.stride(), v.stride()
    # (the stride of a dimension of one entry, or of nothing, says nothing)
    if n <= 1 or hkv == 1:
        live = (n > 1, hkv > 1 and n > 0, n > 0)
        ks = tuple(s if on else i // 2 for i, (s, on) in enumerate(zip(ks, live)))
        vs = tuple(s if on else i // 2 for i, (s, on) in enumerate(zip(vs, live)))
    if ks != vs or ks[2] != 1:
        raise ValueError("k and v must have the same strides, the last one 1")
    if k.get_device() != dev or v.get_device() != dev:
        raise ValueError("k and v must be tensors on the current device")
    _check(lib.wf_kv8_append(code, _one_layer(cache, dev), k.data_ptr(), v.data_ptr(), n,
                             start_pos, ks[0], ks[1], raw), "wf_kv8_append")


def wf_kv8_only_prefill_workspace_bytes(dtype, n_tok, d_in, n_kv_heads, head_dim) -> int:
    code = dtype if isinstance(dtype, int) else (
        WF_F32 if dtype == torch.float32 else WF_BF16)
    return int(lib.wf_kv8_only_prefill_workspace_bytes(code, n_tok, d_in, n_kv_heads, head_dim))


def wf_kv8_only_prefill(x, w_k, w_v, cache, start_pos, rope_base, workspace=None, stream=None):
    """wf_kv_only_prefill into an 8-bit cache: x [n][d_in]; w_k, w_v
    [Hkv*D][d_in]."""
    dev, raw = _at(stream)
    n_tok, d_in = x.shape
    hkv, dh = cache.n_kv_heads, cache.head_dim
    for w in (w_k, w_v):
        if tuple(w.shape) != (hkv * dh, d_in) or w.dtype != x.dtype:
            raise ValueError("weights must be [n_kv_heads * head_dim][d_in], of x's type")
    code = _weight_code(x, w_k, w_v)
    if workspace is None:
        with _on(stream):
            workspace = alloc_workspace(wf_kv8_only_prefill_workspace_bytes(
                code, n_tok, d_in, hkv, dh), x.device)
    wk, wv = (w.data if isinstance(w, TiledWeight) else w for w in (w_k, w_v))
    _check(lib.wf_kv8_only_prefill(code, _ptr(x, dev, "x"), _ptr(wk, dev, "w_k"),
                                   _ptr(wv, dev, "w_v"), _one_layer(cache, dev), n_tok,
                                   start_pos, d_in, float(rope_base),
                                   _ptr(workspace, dev, "workspace"), workspace.numel(), raw),
           "wf_kv8_only_prefill")


def wf_kv8_verify_attn_workspace_bytes(dtype, gamma, ctx_len, n_q_heads, n_kv_heads, head_dim,
                                       num_splits=0) -> int:
    code = dtype if isinstance(dtype, int) else (
        WF_F32 if dtype == torch.float32 else WF_BF16)
    return int(lib.wf_kv8_verify_attn_workspace_bytes(
        code, gamma, ctx_len, n_q_heads, n_kv_heads, head_dim, num_splits))


def _kv8_attn(q, cache, out, ctx_len, tree_mask, softmax_scale, num_splits, workspace, stream):
    dev, raw = _at(stream)
    shape = q.shape
    gamma, hq, dh = shape
    if dh != cache.head_dim or out.shape != shape or out.dtype != q.dtype:
        raise ValueError("q, out and the cache do not match")
    code = _dtype_code(q)
    if softmax_scale is None:
        softmax_scale = dh ** -0.5
    if workspace is None:
        with _on(stream):
            workspace = alloc_workspace(wf_kv8_verify_attn_workspace_bytes(
                code, gamma, ctx_len, hq, cache.n_kv_heads, dh, num_splits), q.device)
    head = (code, _ptr(q, dev, "q"), _one_layer(cache, dev), _ptr(out, dev, "out"))
    tail = (gamma, ctx_len, hq, softmax_scale, num_splits, _ptr(workspace, dev, "workspace"),
            workspace.numel(), raw)
    if tree_mask is None:
        _check(lib.wf_kv8_verify_attn(*head, *tail), "wf_kv8_verify_attn")
    else:
        _check(lib.wf_kv8_verify_attn_tree(*head, _ptr(tree_mask, dev, "tree_mask"), *tail),
               "wf_kv8_verify_attn_tree")
    return out


def wf_kv8_verify_attn(q, cache, out, ctx_len, softmax_scale=None, num_splits=0,
                       workspace=None, stream=None):
    """wf_verify_attn over an 8-bit cache: q, out [gamma][Hq][D] (bf16 or
    fp32), cache rows [0, ctx_len + gamma) valid."""
    return _kv8_attn(q, cache, out, ctx_len, None, softmax_scale, num_splits, workspace, stream)


def wf_kv8_verify_attn_tree(q, cache, out, ctx_len, tree_mask, softmax_scale=None,
                            num_splits=0, workspace=None, stream=None):
    """wf_verify_attn_tree over an 8-bit cache; tree_mask as there."""
    if tree_mask.numel() != q.shape[0] or tree_mask.dtype not in (torch.int64, torch.uint64):
        raise ValueError("tree_mask must hold gamma 64-bit words (int64 or uint64)")
    return _kv8_attn(q, cache, out, ctx_len, tree_mask, softmax_scale, num_splits, workspace,
                     stream)


def wf_kv8_compact_path(cache, accept, path, ctx_len, stream=None):
    """wf_kv_compact_path for an 8-bit cache (one layer or the whole stack):
    accept (n at [0]) and path [gamma] int32 device tensors, as written by
    wf_lmhead_accept_tree."""
    dev, raw = _at(stream)
    layers, codes, scales = 1, 0, 0
    if cache.n_layers is not None:
        layers, codes, scales = cache.n_layers, cache.k.stride(0), cache.k_scale.stride(0)
    if accept.dtype != torch.int32 or path.dtype != torch.int32:
        raise TypeError("accept and path are int32")
    if cache.dev != dev:
        raise ValueError("the cache must be on the current device")
    _check(lib.wf_kv8_compact_path(cache.ref, _ptr(accept, dev, "accept"),
                                   _ptr(path, dev, "path"), path.numel(), ctx_len, layers,
                                   codes, scales, raw), "wf_kv8_compact_path")


class W4Weight:
    """A 4-bit weight [rows][cols] in the packed tiles that wf_linear_w4
    streams (wf.h: e2m1 codes, one power-of-two scale byte per 32 columns),
    made once from its row-major form: codes [rows][cols / 2] uint8 (or
    float4_e2m1fn_x2), low nibble first, and scales [rows][cols / 32] uint8 (or float8_e8m0fnu),
    which are not kept and may be dropped at once."""

    def __init__(self, codes, scales, stream=None):
        rows, half = codes.shape
        if half % 16 or tuple(scales.shape) != (rows, half // 16):
            raise ValueError("codes [rows][cols / 2] and scales [rows][cols / 32] do not match")
        if codes.dtype not in E2M1_BYTES or scales.dtype not in E8M0_BYTES:
            raise ValueError("codes are uint8 (or float4_e2m1fn_x2), scales uint8 (or "
                             "float8_e8m0fnu)")
        dev, raw = _at(stream)
        n = int(lib.wf_w4_packed_bytes(rows, 2 * half))
        self.shape, self.device = (rows, 2 * half), codes.device
        src = _ptr(codes, dev, "codes"), _ptr(scales, dev, "scales")
        with _on(stream):
            self.packed = torch.empty(n, dtype=torch.uint8, device=codes.device)
        _check(lib.wf_w4_pack(*src, rows, 2 * half, self.packed.data_ptr(), n, raw), "wf_w4_pack")
        _hold(stream, codes, scales)


def wf_w4_quantize(w, stream=None):
    """The 4-bit form (codes, scales) of a bf16 weight [rows][cols], cols % 32
    == 0; W4Weight(codes, scales) packs it for the products."""
    if w.dtype != torch.bfloat16:
        raise TypeError("4-bit weights are made from bf16")
    dev, raw = _at(stream)
    rows, cols = w.shape
    if cols % 32:
        raise ValueError("the columns of a 4-bit weight come in groups of 32")
    src = _ptr(w, dev, "w")
    with _on(stream):
        codes = torch.empty((rows, cols // 2), dtype=torch.uint8, device=w.device)
        scales = torch.empty((rows, cols // 32), dtype=torch.uint8, device=w.device)
    _check(lib.wf_w4_quantize(src, rows, cols, codes.data_ptr(), scales.data_ptr(), raw),
           "wf_w4_quantize")
    _hold(stream, w)
    return codes, scales


def wf_linear_w4_workspace_bytes(n_rows, n_out, k_in) -> int:
    return int(lib.wf_linear_w4_workspace_bytes(n_rows, n_out, k_in))


def wf_linear_w4(x, weight, out, residual=None, workspace=None, stream=None):
    """out = x W^T (+ residual): x [n][k_in] bf16 (n <= 64), weight a W4Weight
    [n_out][k_in], residual [n][n_out] bf16, out [n][n_out] bf16 or fp32."""
    dev, raw = _at(stream)
    n, k_in = x.shape
    n_out, cols = weight.shape
    shape = out.shape
    packed = weight.packed
    if cols != k_in or shape != (n, n_out) or packed.get_device() != dev:
        raise ValueError("x, weight and out do not match")
    if x.dtype != torch.bfloat16:
        raise TypeError("x is bf16")
    if residual is not None and (residual.shape != shape or residual.dtype != torch.bfloat16):
        raise ValueError("residual must be bf16, in out's shape")
    if workspace is None:
        need = wf_linear_w4_workspace_bytes(n, n_out, k_in)
        with _on(stream):
            workspace = alloc_workspace(need, x.device) if need else None
    st = lib.wf_linear_w4(_ptr(x, dev, "x"), packed.data_ptr(), _ptr(residual, dev, "residual"),
                          _dtype_code(out), _ptr(out, dev, "out"), n, n_out, k_in,
                          _ptr(workspace, dev, "workspace"),
                          0 if workspace is None else workspace.numel(), raw)
    _check(st, "wf_linear_w4")
    return out


class _Fixed:
    """A handle whose numbers and tensors stay those that the calls hold: once it
    is made, none of them can be assigned."""
    _held = frozenset()

    def __setattr__(self, name, value):
        if name in self._held:
            raise AttributeError(f"{name} of a {type(self).__name__} cannot change: make another")
        super().__setattr__(name, value)

    def _hold(self):
        self.__dict__["_held"] = frozenset(self.__dict__) | {"_held"}


class PagedCache(_Fixed):
    """One layer's paged K/V cache (wf.h): a pool of pages that the sequences of
    a batch share.

    k, v     [n_pages][Hkv][page][D] bf16 or fp32, page 16, 32, 64 or 128
    bounds   [n_pages][Hkv][2][D] of the same type, each page's smallest and
             largest key per dimension (kept by wf_paged_append, read by
             wf_paged_select), or None

    The tensors and sizes stay the ones it was made of (the calls hold them); a
    deep copy has its own."""

    def __init__(self, k, v, bounds=None):
        shape = tuple(k.shape)
        if len(shape) != 4 or tuple(v.shape) != shape or v.dtype != k.dtype:
            raise ValueError("k and v must be [n_pages][Hkv][page][D], of one type")
        n, hkv, page, dh = shape
        if bounds is not None and (tuple(bounds.shape) != (n, hkv, 2, dh)
                                   or bounds.dtype != k.dtype):
            raise ValueError("bounds must be [n_pages][Hkv][2][D], of k's type")
        dev = k.get_device()
        if dev < 0:
            raise ValueError("the cache must be device memory")
        self._tensors = k, v, bounds
        self.code, self.dtype, self.device, self.dev = _dtype_code(k), k.dtype, k.device, dev
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = shape
        self.struct = PagedCacheStruct(_ptr(k, dev, "k"), _ptr(v, dev, "v"),
                                       _ptr(bounds, dev, "bounds"), n, page, hkv, dh)
        self.ref = ctypes.byref(self.struct)
        self._hold()

    k = property(lambda self: self._tensors[0])
    v = property(lambda self: self._tensors[1])
    bounds = property(lambda self: self._tensors[2])

    def __reduce__(self):
        return PagedCache, self._tensors


def alloc_paged_cache(n_pages, page_size, n_kv_heads, head_dim, dtype, device,
                      bounds=True) -> PagedCache:
    """An empty paged cache (zeros) of one layer."""
    k, v = (torch.zeros((n_pages, n_kv_heads, page_size, head_dim), dtype=dtype, device=device)
            for _ in range(2))
    b = torch.zeros((n_pages, n_kv_heads, 2, head_dim), dtype=dtype,
                    device=device) if bounds else None
    return PagedCache(k, v, b)


class PagedBatch(_Fixed):
    """A ragged batch over paged caches (wf.h): int32 device tensors page_table
    [n_seqs][max_pages], row_start [n_seqs + 1] and ctx_len [n_seqs], which the
    caller may refill between calls (and between a captured graph's replays), and
    the most rows that a sequence has in an attention or selection call, which the
    attention's tiles are made for.  The tensors and sizes, max_rows among them, stay
    the ones it was made of."""

    def __init__(self, page_table, row_start, ctx_len, max_rows=64):
        n, max_pages = page_table.shape
        if tuple(row_start.shape) != (n + 1,) or tuple(ctx_len.shape) != (n,):
            raise ValueError("page_table [n][max_pages], row_start [n + 1], ctx_len [n]")
        for t in (page_table, row_start, ctx_len):
            if t.dtype != torch.int32:
                raise TypeError("page_table, row_start and ctx_len are int32")
        dev = page_table.get_device()
        if dev < 0:
            raise ValueError("the batch's lists must be device memory")
        self._tensors = page_table, row_start, ctx_len
        self.n_seqs, self.max_pages, self.dev = n, max_pages, dev
        self.max_rows = operator.index(max_rows)
        self.struct = PagedBatchStruct(_ptr(page_table, dev, "page_table"),
                                       _ptr(row_start, dev, "row_start"),
                                       _ptr(ctx_len, dev, "ctx_len"), n, max_pages,
                                       self.max_rows)
        self.ref = ctypes.byref(self.struct)
        self._hold()

    page_table = property(lambda self: self._tensors[0])
    row_start = property(lambda self: self._tensors[1])
    ctx_len = property(lambda self: self._tensors[2])

    def __reduce__(self):
        return PagedBatch, (*self._tensors, self.max_rows)


def _paged(cache, batch, dev):
    if cache.dev != dev or batch.dev != dev:
        raise ValueError("the cache and the batch must be on the current device")
    return cache.ref, batch.ref


def _row_stride(t, n, heads, dh, name):
    """The distance of t's rows [n][heads][dh] in elements; the rest is dense."""
    s = t.stride()
    if n and ((dh > 1 and s[2] != 1) or (heads > 1 and s[1] != dh)):
        raise ValueError(f"the heads of a row of {name} must lie side by side")
    return s[0] if n > 1 else heads * dh


def wf_paged_append(k, v, cache, batch, rope_base, q=None, q_out=None, positions=None,
                    stream=None):
    """k, v [n][Hkv][D], not yet rotated, into the batch's pages, K rotated;
    with q [n][Hq][D], q_out [n][Hq][D] receives it rotated.  A row's heads lie
    side by side, rows may be strided (alike for k and v), as in views of one
    fused projection.  positions [n] int32: what to rotate by, where that is not
    the row's position (draft trees)."""
    dev, raw = _at(stream)
    shape, dtype = k.shape, cache.dtype
    n, hkv, dh = shape
    if v.shape != shape or k.dtype != dtype or v.dtype != dtype or \
            hkv != cache.n_kv_heads or dh != cache.head_dim:
        raise ValueError("k and v must match each other and the cache")
    stride = _row_stride(k, n, hkv, dh, "k")
    if _row_stride(v, n, hkv, dh, "v") != stride:
        raise ValueError("k and v must have the same strides")
    if k.get_device() != dev or v.get_device() != dev:
        raise ValueError("k and v must be tensors on the current device")
    qs, hq, qp, qo = 0, 0, None, None
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out come together")
    if q is not None:
        qshape = q.shape
        if len(qshape) != 3 or qshape[0] != n or qshape[2] != dh or q_out.shape != qshape or \
                q.dtype != dtype or q_out.dtype != dtype:
            raise ValueError("q and q_out must be [n][Hq][D], of the cache's type")
        if q.get_device() != dev:
            raise ValueError("q must be a tensor on the current device")
        hq = qshape[1]
        qs, qp, qo = _row_stride(q, n, hq, dh, "q"), q.data_ptr(), _ptr(q_out, dev, "q_out")
    if positions is not None and (positions.shape != (n,) or positions.dtype != torch.int32):
        raise ValueError("positions must be [n] int32")
    _check(lib.wf_paged_append(cache.code, *_paged(cache, batch, dev), k.data_ptr(), v.data_ptr(),
                               stride, qp, qs, qo, hq, _ptr(positions, dev, "positions"),
                               rope_base, n, raw), "wf_paged_append")


def _code_of(dtype):
    """The code of a torch dtype, or the code itself."""
    code = dtype if isinstance(dtype, int) else _DTYPE_CODES.get(dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {dtype}; use float32 or bfloat16")
    return code


def wf_paged_verify_attn_workspace_bytes(dtype, n_rows, n_seqs, max_rows, n_q_heads, n_kv_heads,
                                         head_dim) -> int:
    return int(lib.wf_paged_verify_attn_workspace_bytes(_code_of(dtype), n_rows, n_seqs, max_rows,
                                                        n_q_heads, n_kv_heads, head_dim))


def _tree_ptr(tree_mask, n, dev):
    if tree_mask is None:
        return None
    if tree_mask.numel() != n or tree_mask.dtype not in (torch.int64, torch.uint64):
        raise ValueError("tree_mask must hold a 64-bit word (int64 or uint64) for every row")
    return _ptr(tree_mask, dev, "tree_mask")


def wf_paged_verify_attn(q, cache, batch, out, tree_mask=None, softmax_scale=None,
                         workspace=None, stream=None):
    """Attention of the batch's rows over their pages: q, out [n][Hq][D] of the
    cache's type; tree_mask [n] 64-bit words, or None for chains and blocks.
    Rows that belong to no sequence are left as they were."""
    dev, raw = _at(stream)
    shape = tuple(q.shape)
    n, hq, dh = shape
    if dh != cache.head_dim or tuple(out.shape) != shape or q.dtype != cache.dtype or \
            out.dtype != cache.dtype:
        raise ValueError("q, out and the cache do not match")
    if workspace is None:
        with _on(stream):
            workspace = alloc_workspace(wf_paged_verify_attn_workspace_bytes(
                cache.code, n, batch.n_seqs, batch.max_rows, hq, cache.n_kv_heads, dh), q.device)
    _check(lib.wf_paged_verify_attn(
        cache.code, _ptr(q, dev, "q"), *_paged(cache, batch, dev), _ptr(out, dev, "out"),
        _tree_ptr(tree_mask, n, dev), n, hq, dh ** -0.5 if softmax_scale is None else softmax_scale,
        _ptr(workspace, dev, "workspace"), workspace.numel(), raw), "wf_paged_verify_attn")
    return out


def wf_paged_select_workspace_bytes(n_rows, n_kv_heads, max_pages) -> int:
    return int(lib.wf_paged_select_workspace_bytes(n_rows, n_kv_heads, max_pages))


def wf_paged_select(q, cache, batch, sel, n_recent, workspace=None, stream=None):
    """sel [n][Hkv][n_sel] int32 receives, for every row and KV head, the
    n_sel - n_recent old pages whose bounds promise the largest scores and the
    n_recent newest ones, ascending, then -1."""
    dev, raw = _at(stream)
    n, hq, dh = q.shape
    if dh != cache.head_dim or q.dtype != cache.dtype or sel.dim() != 3 or \
            tuple(sel.shape[:2]) != (n, cache.n_kv_heads) or sel.dtype != torch.int32:
        raise ValueError("q [n][Hq][D] of the cache's type, sel [n][Hkv][n_sel] int32")
    if workspace is None:
        with _on(stream):
            workspace = alloc_workspace(wf_paged_select_workspace_bytes(
                n, cache.n_kv_heads, batch.max_pages), q.device)
    _check(lib.wf_paged_select(cache.code, _ptr(q, dev, "q"), *_paged(cache, batch, dev),
                               _ptr(sel, dev, "sel"), sel.shape[2], n_recent, n, hq,
                               _ptr(workspace, dev, "workspace"), workspace.numel(), raw),
           "wf_paged_select")
    return sel


def wf_paged_sparse_attn_workspace_bytes(dtype, n_rows, n_q_heads, n_kv_heads, head_dim,
                                         page_size, n_sel) -> int:
    return int(lib.wf_paged_sparse_attn_workspace_bytes(_code_of(dtype), n_rows, n_q_heads,
                                                        n_kv_heads, head_dim, page_size, n_sel))


def wf_paged_sparse_attn(q, cache, batch, sel, out, tree_mask=None, softmax_scale=None,
                         workspace=None, stream=None):
    """wf_paged_verify_attn over the pages sel [n][Hkv][n_sel] (int32 logical
    page numbers, as wf_paged_select writes them)."""
    dev, raw = _at(stream)
    shape = tuple(q.shape)
    n, hq, dh = shape
    if dh != cache.head_dim or tuple(out.shape) != shape or q.dtype != cache.dtype or \
            out.dtype != cache.dtype:
        raise ValueError("q, out and the cache do not match")
    if sel.dim() != 3 or tuple(sel.shape[:2]) != (n, cache.n_kv_heads) or \
            sel.dtype != torch.int32:
        raise ValueError("sel must be [n][Hkv][n_sel] int32")
    if workspace is None:
        with _on(stream):
            workspace = alloc_workspace(wf_paged_sparse_attn_workspace_bytes(
                cache.code, n, hq, cache.n_kv_heads, dh, cache.page_size, sel.shape[2]), q.device)
    _check(lib.wf_paged_sparse_attn(
        cache.code, _ptr(q, dev, "q"), *_paged(cache, batch, dev), _ptr(sel, dev, "sel"),
        sel.shape[2], _ptr(out, dev, "out"), _tree_ptr(tree_mask, n, dev), n, hq,
        dh ** -0.5 if softmax_scale is None else softmax_scale, _ptr(workspace, dev, "workspace"),
        workspace.numel(), raw), "wf_paged_sparse_attn")
    return out


def wf_token_logprobs_workspace_bytes(dtype, n_rows, vocab, n_top) -> int:
    return int(lib.wf_token_logprobs_workspace_bytes(_code_of(dtype), n_rows, vocab, n_top))


def wf_token_logprobs(logits, tokens, logprob, entropy=None, rank=None, top_ids=None,
                      top_logprobs=None, workspace=None, stream=None):
    """logits [n][vocab] fp32 or bf16 (rows may be strided), tokens [n] int32
    -> logprob [n] fp32, entropy [n] fp32, rank [n] int32, and the n_top best
    tokens of every row, top_ids [n][n_top] int32 and top_logprobs [n][n_top]
    fp32, each where it is given; tokens and logprob may be None together."""
    dev, raw = _at(stream)
    n, vocab = logits.shape
    code = _dtype_code(logits)
    ls = logits.stride()
    if logits.get_device() != dev or (vocab > 1 and ls[1] != 1):
        raise ValueError("logits must be rows of consecutive values on the current device")
    stride = ls[0] if n > 1 else vocab
    top = 0 if top_ids is None else top_ids.shape[-1]
    for t, dt, want in ((tokens, torch.int32, (n,)), (logprob, torch.float32, (n,)),
                        (entropy, torch.float32, (n,)), (rank, torch.int32, (n,)),
                        (top_ids, torch.int32, (n, top)),
                        (top_logprobs, torch.float32, (n, top))):
        if t is not None and (tuple(t.shape) != want or t.dtype != dt):
            raise ValueError("tokens, rank [n] and top_ids [n][n_top] are int32, logprob, "
                             "entropy [n] and top_logprobs [n][n_top] fp32")
    if top == 0 and n and (top_ids is not None or top_logprobs is not None):
        raise ValueError("leave top_ids and top_logprobs out where no alternatives are wanted")
    if workspace is None:
        with _on(stream):
            workspace = alloc_workspace(wf_token_logprobs_workspace_bytes(code, n, vocab, top),
                                        logits.device)
    _check(lib.wf_token_logprobs(
        code, logits.data_ptr(), stride, _ptr(tokens, dev, "tokens"), n, vocab, top,
        _ptr(logprob, dev, "logprob"), _ptr(entropy, dev, "entropy"), _ptr(rank, dev, "rank"),
        _ptr(top_ids, dev, "top_ids"), _ptr(top_logprobs, dev, "top_logprobs"),
        _ptr(workspace, dev, "workspace"), workspace.numel(), raw), "wf_token_logprobs")


def wf_read_probe(src, sink, workgroups, stream=None):
    """Measurement support: one plain streaming read of the whole device
    tensor src (sink: device tensor of at least workgroups * 4 KB)."""
    _check(lib.wf_read_probe(_dev(src, "src"), src.numel() * src.element_size(),
                             _dev(sink, "sink"), sink.numel() * sink.element_size(),
                             int(workgroups), _stream(stream)), "wf_read_probe")


def wf_read_probe_series(buf, nbytes, n_bufs, reps, sink, workgroups, depth, stream=None):
    """Measurement support: reps rounds of plain reads of the n_bufs
    consecutive nbytes-long pieces of the device tensor buf, launched back
    to back by the library."""
    if n_bufs * nbytes > buf.numel() * buf.element_size():
        raise ValueError("wf_read_probe_series: buf holds fewer than n_bufs pieces")
    _check(lib.wf_read_probe_series(_dev(buf, "buf"), int(nbytes), int(nbytes), int(n_bufs),
                                    int(reps), _dev(sink, "sink"),
                                    sink.numel() * sink.element_size(), int(workgroups),
                                    int(depth), _stream(stream)), "wf_read_probe_series")


def wf_switch_init(active, lazy, prompt_len) -> SwitchState:
    s = SwitchState()
    _check(lib.wf_switch_init(ctypes.byref(s), int(active), int(lazy), int(prompt_len)),
           "wf_switch_init")
    return s


def wf_switch_commit(state, n_new, next_drafter):
    """-> (start, count) of the backlog now due (count 0: none)."""
    start, count = ctypes.c_int32(), ctypes.c_int32()
    _check(lib.wf_switch_commit(ctypes.byref(state), int(n_new), int(next_drafter),
                                ctypes.byref(start), ctypes.byref(count)),
           "wf_switch_commit")
    return start.value, count.value
