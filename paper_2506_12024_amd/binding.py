"""ctypes binding of the C ABI in ``include/flexq.h`` -- argument marshalling only.

Function names and argument order follow the header.  Tensor arguments are
``torch`` CUDA(HIP) tensors (or raw integer device pointers); the stream is
torch's current stream unless given.  No arithmetic happens here.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libflexq.so")

FQ_GROUP = 128
FQ_MAX_DECODE_M = 32
FQ_MAX_LM_HEAD_M = 4
FQ_STATIC_MAX_ENTRIES = 512
FQ_SCRATCH_BANKS = 16
FQ_F16, FQ_BF16 = 0, 1
FQ_ROPE_PLAIN, FQ_ROPE_LINEAR, FQ_ROPE_BASE, FQ_ROPE_WAVELENGTH, FQ_ROPE_RAMP = 0, 1, 2, 3, 4
FQ_MAX_HEAD_DIM = 256
FQ_MAX_Q_HEADS = 4096
FQ_MAX_SEQS = 65535
FQ_MAX_SAMPLE_V = 1 << 24
FQ_MAX_ADAPTERS = 16384
FQ_MAX_ADAPTER_RANK = 256
FQ_MAX_ADAPTER_ROWS = 1 << 20
FQ_MAX_GIVEN = 65536
FQ_MAX_ALTERNATIVES = 64
FQ_OK, FQ_ERR_NULL, FQ_ERR_BITS, FQ_ERR_SHAPE, FQ_ERR_NOT_ATTACHED, FQ_ERR_ALIGN, FQ_ERR_HIP = \
    0, -1, -2, -3, -4, -5, -6

EXPORTS = [
    "fq_last_error", "fq_packed_sizes", "fq_quantize", "fq_layer_create", "fq_layer_attach",
    "fq_layer_destroy", "fq_linear", "fq_plan_workspace_bytes", "fq_plan_create", "fq_plan_run",
    "fq_plan_destroy", "fq_entropy_kl", "fq_sched_state_bytes", "fq_sched_init",
    "fq_sched_threshold_from_prefill", "fq_sched_step", "fq_sched_peek",
    "fq_entropy_kl_f16", "fq_rank_ascending", "fq_quantize_act", "fq_linear_w8a8",
    "fq_quantize_sym", "fq_fake_quantize", "fq_lm_head_entropy", "fq_linears_static",
    "fq_plan_staged_workspace_bytes", "fq_plan_create_staged", "fq_plan_set_wait_limit", "fq_plan_status",
    "fq_stream_read",
    "fq_rope_freqs", "fq_kv_create", "fq_kv_destroy", "fq_seqs_create", "fq_seqs_destroy", "fq_kv_append",
    "fq_attend_workspace_bytes", "fq_attend", "fq_sample_workspace_bytes", "fq_sample", "fq_sample_f16",
    "fq_adapters_create", "fq_adapters_destroy", "fq_adapters_workspace_bytes", "fq_adapters_add", "fq_kv_append_normed",
    "fq_logprobs_workspace_bytes", "fq_logprobs", "fq_logprobs_f16",
]


class FlexqError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__("flexq error %d: %s" % (code, message))
        self.code = code


def lib_path() -> str:
    return _LIB_PATH


def _load() -> ctypes.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            "libflexq.so is not built: run `python -m paper_2506_12024_amd.build` "
            "(there is no fallback path)")
    try:
        # PyTorch-ROCm carries its own HIP runtime; loaded first, the library binds to that one
        # instead of bringing a second runtime (with no devices set up) into the process
        import torch  # noqa: F401
    except ImportError:
        pass
    L = ctypes.CDLL(_LIB_PATH)
    vp, ci, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    L.fq_last_error.restype = ctypes.c_char_p
    L.fq_last_error.argtypes = []
    L.fq_packed_sizes.restype = ci
    L.fq_packed_sizes.argtypes = [ci, ci, ci, ci, ctypes.POINTER(sz), ctypes.POINTER(sz), ctypes.POINTER(sz)]
    L.fq_quantize.restype = ci
    L.fq_quantize.argtypes = [vp, ci, ci, ci, ci, vp, vp, vp, vp]
    L.fq_layer_create.restype = ci
    L.fq_layer_create.argtypes = [ctypes.POINTER(vp), ci, ci, ci]
    L.fq_layer_attach.restype = ci
    L.fq_layer_attach.argtypes = [vp, ci, vp, vp, vp]
    L.fq_layer_destroy.restype = ci
    L.fq_layer_destroy.argtypes = [vp]
    L.fq_linear.restype = ci
    L.fq_linear.argtypes = [vp, ci, vp, ci, vp, vp]
    L.fq_plan_workspace_bytes.restype = sz
    L.fq_plan_workspace_bytes.argtypes = [ci]
    L.fq_plan_create.restype = ci
    L.fq_plan_create.argtypes = [ctypes.POINTER(vp), ci, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                 ctypes.POINTER(vp), ci, vp, sz, vp]
    L.fq_plan_run.restype = ci
    L.fq_plan_run.argtypes = [vp, vp, vp]
    L.fq_plan_destroy.restype = ci
    L.fq_plan_destroy.argtypes = [vp]
    L.fq_plan_staged_workspace_bytes.restype = sz
    L.fq_plan_staged_workspace_bytes.argtypes = [ci, ci]
    L.fq_plan_create_staged.restype = ci
    L.fq_plan_create_staged.argtypes = [ctypes.POINTER(vp), ci, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                        ctypes.POINTER(vp), ctypes.POINTER(ctypes.c_int32), ci, vp, sz, vp]
    L.fq_plan_set_wait_limit.restype = ci
    L.fq_plan_set_wait_limit.argtypes = [vp, ctypes.c_longlong]
    L.fq_plan_status.restype = ci
    L.fq_plan_status.argtypes = [vp, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32), vp]
    L.fq_stream_read.restype = ci
    L.fq_stream_read.argtypes = [vp, sz, vp, vp]
    L.fq_linears_static.restype = ci
    L.fq_linears_static.argtypes = [ci, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp), ci, vp, vp]
    L.fq_entropy_kl.restype = ci
    L.fq_entropy_kl.argtypes = [vp, vp, ci, ci, vp, vp, vp]
    L.fq_entropy_kl_f16.restype = ci
    L.fq_entropy_kl_f16.argtypes = [vp, vp, ci, ci, vp, vp, vp]
    L.fq_rank_ascending.restype = ci
    L.fq_rank_ascending.argtypes = [vp, ci, ci, vp, vp]
    L.fq_quantize_sym.restype = ci
    L.fq_quantize_sym.argtypes = [vp, ci, ci, ci, ci, vp, vp, vp, vp]
    L.fq_fake_quantize.restype = ci
    L.fq_fake_quantize.argtypes = [vp, ci, ci, ci, ci, ci, vp, vp]
    L.fq_lm_head_entropy.restype = ci
    L.fq_lm_head_entropy.argtypes = [vp, vp, ci, ci, ci, vp, vp, vp, vp]
    L.fq_quantize_act.restype = ci
    L.fq_quantize_act.argtypes = [vp, ci, ci, vp, vp, vp, vp]
    L.fq_linear_w8a8.restype = ci
    L.fq_linear_w8a8.argtypes = [vp, vp, vp, vp, ci, vp, vp]
    L.fq_sched_state_bytes.restype = sz
    L.fq_sched_state_bytes.argtypes = [ci]
    L.fq_sched_init.restype = ci
    L.fq_sched_init.argtypes = [vp, ci, ctypes.c_double, ci, vp, vp, ci, vp, ci, vp, vp]
    L.fq_sched_threshold_from_prefill.restype = ci
    L.fq_sched_threshold_from_prefill.argtypes = [vp, vp, ci, ci, vp]
    L.fq_sched_step.restype = ci
    L.fq_sched_step.argtypes = [vp, vp, vp]
    L.fq_sched_peek.restype = ci
    L.fq_sched_peek.argtypes = [vp, ctypes.POINTER(ci), ctypes.POINTER(ci), ctypes.POINTER(ctypes.c_double),
                                ctypes.POINTER(ctypes.c_double), vp]
    ll, cd, cf = ctypes.c_longlong, ctypes.c_double, ctypes.c_float
    L.fq_rope_freqs.restype = ci
    L.fq_rope_freqs.argtypes = [ci, cd, ci, cd, cd, cd, cd, ctypes.POINTER(cd)]
    L.fq_kv_create.restype = ci
    L.fq_kv_create.argtypes = [ctypes.POINTER(vp), ci, ci, ci, ci, ci, vp, vp, ll, ll, ll]
    L.fq_kv_destroy.restype = ci
    L.fq_kv_destroy.argtypes = [vp]
    L.fq_seqs_create.restype = ci
    L.fq_seqs_create.argtypes = [ctypes.POINTER(vp), ci, vp, vp, vp, ci, vp, ci]
    L.fq_seqs_destroy.restype = ci
    L.fq_seqs_destroy.argtypes = [vp]
    L.fq_kv_append.restype = ci
    L.fq_kv_append.argtypes = [vp, vp, ci, vp, ll, ci, vp, ll, vp, ll, vp, ll, vp, ci, ci, cf, vp, vp]
    L.fq_attend_workspace_bytes.restype = sz
    L.fq_attend_workspace_bytes.argtypes = [vp, vp, ci, ci, ci, ci]
    L.fq_attend.restype = ci
    L.fq_attend.argtypes = [vp, vp, ci, vp, ll, ci, cf, vp, ll, vp, ci, ci, vp, sz, vp]
    L.fq_sample_workspace_bytes.restype = sz
    L.fq_sample_workspace_bytes.argtypes = [ci, ci]
    for name in ("fq_sample", "fq_sample_f16"):
        getattr(L, name).restype = ci
        getattr(L, name).argtypes = [vp, ci, ci, ll, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    L.fq_adapters_create.restype = ci
    L.fq_adapters_create.argtypes = [ctypes.POINTER(vp), ci, ci, ci, ci, ci, vp, ll, vp, ll, vp, vp]
    L.fq_adapters_destroy.restype = ci
    L.fq_adapters_destroy.argtypes = [vp]
    L.fq_adapters_workspace_bytes.restype = sz
    L.fq_adapters_workspace_bytes.argtypes = [vp, ci]
    L.fq_adapters_add.restype = ci
    L.fq_adapters_add.argtypes = [vp, ci, vp, ll, vp, vp, ll, vp, ll, vp, sz, vp]
    L.fq_kv_append_normed.restype = ci
    L.fq_kv_append_normed.argtypes = [vp, vp, ci, vp, ll, ci, vp, ll, vp, ll, vp, ll, vp, vp, ll, cf, cf, vp, ci, ci, cf, vp, vp]
    L.fq_logprobs_workspace_bytes.restype = sz
    L.fq_logprobs_workspace_bytes.argtypes = [ci, ci]
    for name in ("fq_logprobs", "fq_logprobs_f16"):
        getattr(L, name).restype = ci
        getattr(L, name).argtypes = [vp, ci, ci, ll, vp, ci, vp, ci, vp, vp, vp, vp, sz, vp]
    return L


lib = _load()


def fq_last_error() -> str:
    return lib.fq_last_error().decode()


def _check(rc: int) -> None:
    if rc != FQ_OK:
        raise FlexqError(rc, fq_last_error())


def _ptr(t):
    """Device pointer of a torch tensor (must be contiguous), an int, or None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        # The current stream's handle without a Stream object around it, which took 2.9 us of a call (a 1 x 4096 -> 4096
        # linear: 8.1 us a call with it, 5.4 without).  The two functions are not public: a torch without them takes the public way.
        if torch.cuda.is_initialized():
            raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
            if raw and device:
                return raw(device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def fq_packed_sizes(N: int, K: int, bits: int, group: int = FQ_GROUP):
    c, s, z = ctypes.c_size_t(), ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib.fq_packed_sizes(N, K, bits, group, ctypes.byref(c), ctypes.byref(s), ctypes.byref(z)))
    return c.value, s.value, z.value


def fq_quantize(w_fp16, N: int, K: int, bits: int, group: int, codes, scales, zeros, stream=None):
    _check(lib.fq_quantize(_ptr(w_fp16), N, K, bits, group, _ptr(codes), _ptr(scales), _ptr(zeros),
                           _stream(stream)))


def fq_quantize_sym(w_fp16, N: int, K: int, bits: int, group: int, codes, scales, zeros, stream=None):
    _check(lib.fq_quantize_sym(_ptr(w_fp16), N, K, bits, group, _ptr(codes), _ptr(scales), _ptr(zeros),
                               _stream(stream)))


def fq_fake_quantize(w_fp16, N: int, K: int, bits: int, group: int, symmetric: bool, w_hat_fp16, stream=None):
    _check(lib.fq_fake_quantize(_ptr(w_fp16), N, K, bits, group, 1 if symmetric else 0, _ptr(w_hat_fp16),
                                _stream(stream)))


class Layer:
    """Owns an ``fq_layer`` handle and keeps the attached tensors alive."""

    def __init__(self, N: int, K: int, group: int = FQ_GROUP):
        h = ctypes.c_void_p()
        _check(lib.fq_layer_create(ctypes.byref(h), N, K, group))
        self.handle = h
        self.N, self.K, self.group = N, K, group
        self._keep = {}

    def attach(self, bits: int, codes, scales=None, zeros=None):
        _check(lib.fq_layer_attach(self.handle, bits, _ptr(codes), _ptr(scales), _ptr(zeros)))
        self._keep[bits] = (codes, scales, zeros)
        return self

    def destroy(self):
        if self.handle is not None:
            _check(lib.fq_layer_destroy(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def fq_linear(layer: Layer, bits: int, x_fp16, M: int, y_fp16, stream=None):
    _check(lib.fq_linear(layer.handle, bits, _ptr(x_fp16), M, _ptr(y_fp16), _stream(stream)))


class Plan:
    """Owns an ``fq_plan``: ``count`` independent linears run by one launch, the
    bit-width of each read from a device int32 array at run time."""

    def __init__(self, layers, xs, ys, M: int, workspace, stream=None):
        n = len(layers)
        arr = ctypes.c_void_p * max(n, 1)
        self._keep = (list(layers), list(xs), list(ys), workspace)
        h = ctypes.c_void_p()
        ws_bytes = workspace.numel() * workspace.element_size() if hasattr(workspace, "numel") else 0
        _check(lib.fq_plan_create(
            ctypes.byref(h), n, arr(*[l.handle for l in layers]), arr(*[_ptr(x) for x in xs]),
            arr(*[_ptr(y) for y in ys]), M, _ptr(workspace), ws_bytes, _stream(stream)))
        self.handle = h
        self.count = n

    @staticmethod
    def workspace_bytes(count: int) -> int:
        return int(lib.fq_plan_workspace_bytes(count))

    def run(self, bits_dev, stream=None):
        _check(lib.fq_plan_run(self.handle, _ptr(bits_dev), _stream(stream)))

    def status(self, stream=None):
        """Waits for ``stream``; returns (launches that gave up, flags) -- flags bit 0: in some run an
        entry's bit-width could not be served (not attached, or no kernel for it at this M)."""
        g, f = ctypes.c_int32(0), ctypes.c_int32(0)
        _check(lib.fq_plan_status(self.handle, ctypes.byref(g), ctypes.byref(f), _stream(stream)))
        return int(g.value), int(f.value)

    def destroy(self):
        if self.handle is not None:
            _check(lib.fq_plan_destroy(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class StagedPlan(Plan):
    """Owns a stage-ordered ``fq_plan``: entry i belongs to stage ``stage[i]`` (host ints, never
    decreasing); one launch runs the stages in order."""

    def __init__(self, layers, xs, ys, stage, M: int, workspace, stream=None):
        n = len(layers)
        arr = ctypes.c_void_p * max(n, 1)
        st = (ctypes.c_int32 * max(n, 1))(*[int(v) for v in stage])
        self._keep = (list(layers), list(xs), list(ys), workspace)
        h = ctypes.c_void_p()
        ws_bytes = workspace.numel() * workspace.element_size() if hasattr(workspace, "numel") else 0
        _check(lib.fq_plan_create_staged(
            ctypes.byref(h), n, arr(*[l.handle for l in layers]), arr(*[_ptr(x) for x in xs]),
            arr(*[_ptr(y) for y in ys]), st, M, _ptr(workspace), ws_bytes, _stream(stream)))
        self.handle = h
        self.count = n

    @staticmethod
    def workspace_bytes(count: int, n_stages: int) -> int:
        return int(lib.fq_plan_staged_workspace_bytes(count, n_stages))

    def set_wait_limit(self, polls: int):
        _check(lib.fq_plan_set_wait_limit(self.handle, polls))


def fq_stream_read(src, nbytes: int, sink, stream=None):
    _check(lib.fq_stream_read(_ptr(src), nbytes, _ptr(sink), _stream(stream)))


def fq_linears_static(layers, xs, ys, M: int, bits_dev, stream=None):
    n = len(layers)
    arr = ctypes.c_void_p * max(n, 1)
    _check(lib.fq_linears_static(n, arr(*[l.handle for l in layers]), arr(*[_ptr(x) for x in xs]),
                                 arr(*[_ptr(y) for y in ys]), M, _ptr(bits_dev), _stream(stream)))


def fq_entropy_kl(logits_p, logits_q, R: int, V: int, entropy_out, kl_out, stream=None):
    _check(lib.fq_entropy_kl(_ptr(logits_p), _ptr(logits_q), R, V, _ptr(entropy_out), _ptr(kl_out),
                             _stream(stream)))


def fq_entropy_kl_f16(logits_p, logits_q, R: int, V: int, entropy_out, kl_out, stream=None):
    _check(lib.fq_entropy_kl_f16(_ptr(logits_p), _ptr(logits_q), R, V, _ptr(entropy_out), _ptr(kl_out),
                                 _stream(stream)))


def fq_rank_ascending(values, n: int, m: int, order, stream=None):
    _check(lib.fq_rank_ascending(_ptr(values), n, m, _ptr(order), _stream(stream)))


def fq_lm_head_entropy(x, w, M: int, V: int, K: int, logits, H, argmax=None, stream=None):
    _check(lib.fq_lm_head_entropy(_ptr(x), _ptr(w), M, V, K, _ptr(logits), _ptr(H), _ptr(argmax), _stream(stream)))


def fq_quantize_act(x, M: int, K: int, xq, sx, xsum, stream=None):
    _check(lib.fq_quantize_act(_ptr(x), M, K, _ptr(xq), _ptr(sx), _ptr(xsum), _stream(stream)))


def fq_linear_w8a8(layer, xq, sx, xsum, M: int, y, stream=None):
    _check(lib.fq_linear_w8a8(layer.handle, _ptr(xq), _ptr(sx), _ptr(xsum), M, _ptr(y), _stream(stream)))


def fq_sched_state_bytes(window: int) -> int:
    return int(lib.fq_sched_state_bytes(window))


def fq_sched_init(state, window: int, thre: float, per_trigger: int, ev_entry, ev_bits, n_events: int,
                  bits, ev_token=None, stream=None, entries: int | None = None):
    """`entries` defaults to the length of the `bits` tensor."""
    if entries is None:
        entries = bits.numel()
    _check(lib.fq_sched_init(_ptr(state), window, thre, per_trigger, _ptr(ev_entry), _ptr(ev_bits),
                             n_events, _ptr(bits), entries, _ptr(ev_token), _stream(stream)))


def fq_sched_threshold_from_prefill(state, entropy, R: int, last_n: int, stream=None):
    _check(lib.fq_sched_threshold_from_prefill(_ptr(state), _ptr(entropy), R, last_n, _stream(stream)))


def fq_sched_step(state, entropy, stream=None):
    _check(lib.fq_sched_step(_ptr(state), _ptr(entropy), _stream(stream)))


def fq_sched_peek(state, stream=None):
    """Returns (next_event, tokens, thre, last_mean) after waiting for the stream."""
    ne, tk = ctypes.c_int(), ctypes.c_int()
    th, lm = ctypes.c_double(), ctypes.c_double()
    _check(lib.fq_sched_peek(_ptr(state), ctypes.byref(ne), ctypes.byref(tk), ctypes.byref(th),
                             ctypes.byref(lm), _stream(stream)))
    return ne.value, tk.value, th.value, lm.value


def fq_rope_freqs(rot_dim: int, base: float, kind: int = FQ_ROPE_PLAIN, factor: float = 1.0, low: float = 0.0,
                  high: float = 0.0, original: float = 0.0):
    """The frequencies as a list of ``rot_dim // 2`` floats; a float64 tensor of them on the device is what
    ``fq_kv_append`` takes."""
    out = (ctypes.c_double * max(rot_dim // 2, 1))()
    _check(lib.fq_rope_freqs(rot_dim, base, kind, factor, low, high, original, out))
    return list(out)


try:
    import torch as _torch
    _F16, _BF16, _F32, _F64, _I32 = _torch.float16, _torch.bfloat16, _torch.float32, _torch.float64, _torch.int32
    _RAW = hasattr(_torch._C, "_cuda_getDevice") and hasattr(_torch._C, "_cuda_getCurrentRawStream")  # (not public, see _stream)
except ImportError:  # the host-only calls above work without
    _F16 = _BF16 = _F32 = _F64 = _I32 = None
    _RAW = False


# The calls of a decode step are short: what a small one costs is launch and marshalling, so each argument is looked at once, in
# one call (one token of 32 heads appended: 9.0 us of marshalling with a check to a call, 5.0 with these).
def _vector(t, dtype, n, name):
    """Device pointer of a contiguous tensor of at least n elements of the type the call assumes, an int, or None."""
    if t is None or isinstance(t, int):
        return t
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of at least %d elements" % (name, dtype, n))
    return t.data_ptr()


def _rows(t, name, dtype, tokens, heads, dim):
    """(pointer, row stride) of a [tokens][heads][dim] tensor: a row is one piece, rows may lie apart."""
    if t.dtype is not dtype or t.shape != (tokens, heads, dim):
        raise ValueError("%s must be [%d][%d][%d] of %s (got %s of %s)" % (name, tokens, heads, dim, dtype, tuple(t.shape), t.dtype))
    row, head, one = t.stride()
    if one != 1 or (head != dim and heads > 1):
        raise ValueError("the heads of a row of %s must lie side by side" % name)
    return t.data_ptr(), row if tokens > 1 else heads * dim


class KVCache:
    """Owns an ``fq_kv`` handle and keeps the tensors alive: ``k`` and ``v`` are [page][head][token][dim] views of
    equal strides over fp16 or bf16 storage, values of a head side by side (a pool laid out token by token is
    ``pool.permute(0, 2, 1, 3)``)."""

    def __init__(self, k, v):
        if k.dim() != 4 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype:
            raise ValueError("k and v must be [page][head][token][dim] of one shape, layout and type")
        if k.dtype not in (_F16, _BF16):
            raise ValueError("k and v must be float16 or bfloat16 (got %s)" % k.dtype)
        if k.stride(3) != 1:
            raise ValueError("the values of a head must lie side by side")
        self.handle = None
        self._keep = (k, v)
        self.dtype = k.dtype
        self.n_pages, self.kv_heads, self.page_tokens, self.head_dim = k.shape
        h = ctypes.c_void_p()
        _check(lib.fq_kv_create(ctypes.byref(h), FQ_F16 if k.dtype is _F16 else FQ_BF16, self.kv_heads, self.head_dim,
                                self.page_tokens, self.n_pages, k.data_ptr(), v.data_ptr(), k.stride(0), k.stride(1),
                                k.stride(2)))
        self.handle = h

    def destroy(self):
        if self.handle is not None:
            _check(lib.fq_kv_destroy(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class Sequences:
    """Owns an ``fq_seqs`` handle and keeps its int32 device tables alive: ``q_start`` [seqs + 1], ``kv_len`` [seqs],
    ``table`` [seqs][pages], ``prefix_table`` [pages of the shared prefix] or None."""

    def __init__(self, q_start, kv_len, table, prefix_table=None, prefix_len: int = 0):
        self.handle = None
        if table.dim() != 2 or q_start.numel() != table.shape[0] + 1 or kv_len.numel() != table.shape[0]:
            raise ValueError("need q_start [seqs + 1], kv_len [seqs] and table [seqs][pages]")
        self._keep = (q_start, kv_len, table, prefix_table)
        self.prefix_len = prefix_len
        self.prefix_pages = 0 if prefix_table is None else prefix_table.numel()
        h = ctypes.c_void_p()
        _check(lib.fq_seqs_create(ctypes.byref(h), table.shape[0], _vector(q_start, _I32, 1, "q_start"),
                                  _vector(kv_len, _I32, 1, "kv_len"), _vector(table, _I32, 1, "table"), table.shape[1],
                                  _vector(prefix_table, _I32, 0, "prefix_table"), prefix_len))
        self.handle = h

    def covers(self, cache) -> None:
        """The prefix's table must hold every page of the prefix."""
        if self.prefix_pages * cache.page_tokens < self.prefix_len:
            raise ValueError("prefix_table has %d pages of %d tokens, the prefix %d tokens" % (
                self.prefix_pages, cache.page_tokens, self.prefix_len))

    def destroy(self):
        if self.handle is not None:
            _check(lib.fq_seqs_destroy(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def fq_kv_append(cache: KVCache, seqs: Sequences, q, k, v, q_out, freqs, interleaved: bool = False, amplitude: float = 1.0,
                 positions=None, stream=None):
    """q, k, v, q_out: [tokens][heads][dim] (rows may lie apart); q and q_out may be None.  ``freqs``: float64 on the device,
    one for each rotating pair, or None: nothing is turned."""
    T, dtype, dim = k.shape[0], cache.dtype, cache.head_dim
    kp, ks = _rows(k, "k", dtype, T, cache.kv_heads, dim)
    vp, vs = _rows(v, "v", dtype, T, cache.kv_heads, dim)
    qp = op = None
    heads = qs = os_ = 0
    if q is not None:
        heads = q.shape[1]
        qp, qs = _rows(q, "q", dtype, T, heads, dim)
        op, os_ = _rows(q_out, "q_out", dtype, T, heads, dim)
    _check(lib.fq_kv_append(cache.handle, seqs.handle, T, qp, qs, heads, op, os_, kp, ks, vp, vs, _vector(freqs, _F64, 0, "freqs"),
                            0 if freqs is None else 2 * freqs.numel(), 1 if interleaved else 0, amplitude,
                            _vector(positions, _I32, T, "positions"), _stream(stream)))


def fq_attend_workspace_bytes(cache: KVCache, seqs: Sequences, tokens: int, q_heads: int, max_q: int, max_kv: int) -> int:
    n = int(lib.fq_attend_workspace_bytes(cache.handle, seqs.handle, tokens, q_heads, max_q, max_kv))
    if n == 0:
        raise FlexqError(FQ_ERR_SHAPE, fq_last_error())
    return n


def fq_attend(cache: KVCache, seqs: Sequences, q, out, scale: float, max_q: int, max_kv: int, workspace, lse=None, stream=None):
    """q, out: [tokens][q_heads][dim] (rows may lie apart); lse: float32 [tokens][q_heads] or None."""
    seqs.covers(cache)
    T, heads, dim = q.shape
    qp, qs = _rows(q, "q", cache.dtype, T, heads, cache.head_dim)
    op, os_ = _rows(out, "out", cache.dtype, T, heads, dim)
    _check(lib.fq_attend(cache.handle, seqs.handle, T, qp, qs, heads, scale, op, os_, _vector(lse, _F32, T * heads, "lse"), max_q,
                         max_kv, _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))


def fq_sample_workspace_bytes(R: int, V: int) -> int:
    n = int(lib.fq_sample_workspace_bytes(R, V))
    if n == 0:
        raise FlexqError(FQ_ERR_SHAPE, fq_last_error())
    return n


def _sample(call, dtype, logits, R, V, u, token, workspace, temperature, top_k, top_p, min_p, prob, stream):
    rows, width = logits.shape
    row, one = logits.stride()
    if logits.dtype is not dtype or rows < R or width != V or one != 1:
        raise ValueError("logits must be %s [R][V], the logits of a row side by side" % dtype)
    _check(call(logits.data_ptr(), R, V, row if R > 1 else V, _vector(u, _F32, R, "u"), _vector(temperature, _F32, R, "temperature"),
                _vector(top_k, _I32, R, "top_k"), _vector(top_p, _F32, R, "top_p"), _vector(min_p, _F32, R, "min_p"),
                _vector(token, _I32, R, "token"), _vector(prob, _F32, R, "prob"), _ptr(workspace),
                workspace.numel() * workspace.element_size(), _stream(stream)))


def fq_sample(logits, R: int, V: int, u, token, workspace, temperature=None, top_k=None, top_p=None, min_p=None, prob=None,
              stream=None):
    """logits: float32 [R][V], rows may lie apart."""
    _sample(lib.fq_sample, _F32, logits, R, V, u, token, workspace, temperature, top_k, top_p, min_p, prob, stream)


def fq_sample_f16(logits, R: int, V: int, u, token, workspace, temperature=None, top_k=None, top_p=None, min_p=None, prob=None,
                  stream=None):
    """logits: float16 [R][V], rows may lie apart."""
    _sample(lib.fq_sample_f16, _F16, logits, R, V, u, token, workspace, temperature, top_k, top_p, min_p, prob, stream)


def _place(stream, first, *others):
    """The call's stream.  Its tensors (``first`` is one; the others may be None or raw pointers) have to lie on the current device, whose
    streams a kernel runs on."""
    import torch
    device = first.get_device()
    for t in others:
        if t is not None and t.__class__ is not int and t.get_device() != device:
            raise ValueError("tensors lie on %s and %s" % (first.device, t.device))
    if device < 0:
        raise ValueError("a tensor lies on %s" % first.device)
    current = torch._C._cuda_getDevice() if _RAW else torch.cuda.current_device()
    if device != current:
        raise ValueError("the tensors lie on cuda:%d, the current device is cuda:%d" % (device, current))
    if stream is None and _RAW:
        return torch._C._cuda_getCurrentRawStream(device)
    return _stream(stream)


def _flat(t, name):
    """(pointer, bytes) of a workspace."""
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t.data_ptr(), t.nbytes


def fq_kv_append_normed(cache: KVCache, seqs: Sequences, q, k, v, q_out, freqs, q_weight, k_weight, eps: float = 1e-6,
                        offset: float = 0.0, interleaved: bool = False, amplitude: float = 1.0, positions=None, stream=None):
    """As ``fq_kv_append``, every head of q and k divided by its root mean square and multiplied by weight + offset before it is
    turned.  q_weight, k_weight: of the cache's type, both [dim] (for all heads) or both [heads][dim]."""
    T, dtype, dim = k.shape[0], cache.dtype, cache.head_dim
    kp, ks = _rows(k, "k", dtype, T, cache.kv_heads, dim)
    vp, vs = _rows(v, "v", dtype, T, cache.kv_heads, dim)
    qp = op = wp = None
    heads = qs = os_ = 0
    each = k_weight.dim() == 2
    if q is not None:
        heads = q.shape[1]
        qp, qs = _rows(q, "q", dtype, T, heads, dim)
        op, os_ = _rows(q_out, "q_out", dtype, T, heads, dim)
        wp = _weights(q_weight, "q_weight", dtype, heads, dim, each)
    stream = _place(stream, k, v, q, q_out, freqs, q_weight if q is not None else None, k_weight, positions, cache._keep[0],
                    seqs._keep[2])
    _check(lib.fq_kv_append_normed(cache.handle, seqs.handle, T, qp, qs, heads, op, os_, kp, ks, vp, vs, wp,
                                   _weights(k_weight, "k_weight", dtype, cache.kv_heads, dim, each), dim if each else 0, eps, offset,
                                   _vector(freqs, _F64, 0, "freqs"), 0 if freqs is None else 2 * freqs.numel(),
                                   1 if interleaved else 0, amplitude, _vector(positions, _I32, T, "positions"), stream))


def _weights(t, name, dtype, heads, dim, each):
    if t.dtype is not dtype or t.shape != ((heads, dim) if each else (dim,)) or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of %s" % (name, dtype, "[%d][%d]" % (heads, dim) if each else "[%d]" % dim))
    return t.data_ptr()


class Adapters:
    """Owns an ``fq_adapters`` handle and keeps its tensors alive: ``a`` [slots][rank][K] and ``b`` [slots][N][rank] in fp16 or bf16,
    each slot contiguous; ``ranks`` int32 [slots] and ``scales`` float32 [slots] on the device, or None."""

    def __init__(self, a, b, ranks=None, scales=None):
        self.handle = None
        if a.dim() != 3 or b.dim() != 3 or a.shape[0] != b.shape[0] or a.shape[1] != b.shape[2]:
            raise ValueError("need a [slots][rank][K] and b [slots][N][rank]")
        if a.dtype not in (_F16, _BF16) or b.dtype is not a.dtype:
            raise ValueError("a and b must both be float16 or bfloat16 (got %s and %s)" % (a.dtype, b.dtype))
        self.slots, self.rank, self.K = a.shape
        self.N, self.dtype = b.shape[1], a.dtype
        if a.numel() and (not a[0].is_contiguous() or not b[0].is_contiguous()):
            raise ValueError("the values of a slot of a and b must be contiguous")
        if any(t is not None and t.device != a.device for t in (b, ranks, scales)):
            raise ValueError("a, b, ranks and scales must lie on one device")
        self._keep = (a, b, ranks, scales)
        h = ctypes.c_void_p()
        _check(lib.fq_adapters_create(ctypes.byref(h), FQ_F16 if a.dtype is _F16 else FQ_BF16, self.slots, self.rank, self.K, self.N,
                                      a.data_ptr(), a.stride(0), b.data_ptr(), b.stride(0),
                                      _vector(ranks, _I32, self.slots, "ranks"), _vector(scales, _F32, self.slots, "scales")))
        self.handle = h

    def destroy(self):
        if self.handle is not None:
            _check(lib.fq_adapters_destroy(self.handle))
            self.handle = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def fq_adapters_workspace_bytes(adapters: Adapters, M: int) -> int:
    n = int(lib.fq_adapters_workspace_bytes(adapters.handle, M))
    if n == 0:
        raise FlexqError(FQ_ERR_SHAPE, fq_last_error())
    return n


def _matrix(t, name, dtype, M, width):
    """(pointer, row stride) of [M][width], the values of a row side by side."""
    if t.dtype is not dtype or t.shape != (M, width):
        raise ValueError("%s must be [%d][%d] of %s (got %s of %s)" % (name, M, width, dtype, tuple(t.shape), t.dtype))
    row, one = t.stride()
    if one != 1 and width > 1:
        raise ValueError("the values of a row of %s must lie side by side" % name)
    return t.data_ptr(), row if M > 1 else width


def fq_adapters_add(adapters: Adapters, x, adapter, y, out, workspace, stream=None):
    """out = y + scale * (x A^T) B^T, each row by its own adapter (int32 [M], -1: none).  x: [M][K]; y, out: [M][N] (rows may lie
    apart), out may be y."""
    M, dtype = x.shape[0], adapters.dtype
    xp, xs = _matrix(x, "x", dtype, M, adapters.K)
    yp, ys = _matrix(y, "y", dtype, M, adapters.N)
    op, os_ = _matrix(out, "out", dtype, M, adapters.N)
    stream = _place(stream, x, adapter, y, out, workspace, adapters._keep[0])
    wp, n = _flat(workspace, "workspace")
    _check(lib.fq_adapters_add(adapters.handle, M, xp, xs, _vector(adapter, _I32, M, "adapter"), yp, ys, op, os_, wp, n,
                               stream))


def fq_logprobs_workspace_bytes(R: int, V: int) -> int:
    n = int(lib.fq_logprobs_workspace_bytes(R, V))
    if n == 0:
        raise FlexqError(FQ_ERR_SHAPE, fq_last_error())
    return n


def _columns(t, dtype, R, name):
    """(pointer, columns) of a contiguous [R] or [R][n] tensor, or nothing."""
    if t is None:
        return None, 0
    if t.dtype is not dtype or t.dim() not in (1, 2) or t.shape[0] != R or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of [%d] or [%d][n]" % (name, dtype, R, R))
    return t.data_ptr(), 1 if t.dim() == 1 else t.shape[1]


def _logprobs(call, dtype, logits, R, V, workspace, given, given_logprob, top_token, top_logprob, entropy, stream):
    rows, width = logits.shape
    row, one = logits.stride()
    if logits.dtype is not dtype or rows < R or width != V or (one != 1 and V > 1):
        raise ValueError("logits must be %s [R][V], the logits of a row side by side" % dtype)
    gp, n = _columns(given, _I32, R, "given")
    lp, n2 = _columns(given_logprob, _F32, R, "given_logprob")
    tp, m = _columns(top_token, _I32, R, "top_token")
    pp, m2 = _columns(top_logprob, _F32, R, "top_logprob")
    if n != n2 or m != m2:
        raise ValueError("given and given_logprob, and top_token and top_logprob, must have one shape")
    stream = _place(stream, logits, workspace, given, given_logprob, top_token, top_logprob, entropy)
    wp, bytes_ = _flat(workspace, "workspace")
    _check(call(logits.data_ptr(), R, V, row if R > 1 else V, gp, n, lp, m, tp, pp, _vector(entropy, _F32, R, "entropy"), wp, bytes_,
                stream))


def fq_logprobs(logits, R: int, V: int, workspace, given=None, given_logprob=None, top_token=None, top_logprob=None, entropy=None,
                stream=None):
    """logits: float32 [R][V], rows may lie apart.  given (int32) and given_logprob: [R] or [R][n]; top_token (int32) and
    top_logprob: [R][n], the n likeliest; entropy: [R]."""
    _logprobs(lib.fq_logprobs, _F32, logits, R, V, workspace, given, given_logprob, top_token, top_logprob, entropy, stream)


def fq_logprobs_f16(logits, R: int, V: int, workspace, given=None, given_logprob=None, top_token=None, top_logprob=None, entropy=None,
                    stream=None):
    """logits: float16 [R][V], rows may lie apart; everything else as ``fq_logprobs``."""
    _logprobs(lib.fq_logprobs_f16, _F16, logits, R, V, workspace, given, given_logprob, top_token, top_logprob, entropy, stream)
