"""Thin binding of libpab.so: argument marshalling only, by ctypes and, for the calls of a denoising loop, natively.

Every function here has the name and meaning of the C entry point it calls
(``include/pab.h``); tensors are torch CUDA tensors used purely as device
memory, the stream is torch's current stream unless one is passed.  There is no
fallback of any kind: if the library has not been built this module raises on
import, and every step of the path runs in the library's HIP kernels.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import warnings

import torch

from .build import binding_path

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpab.so")

SPATIAL, TEMPORAL, CROSS = 0, 1, 2
COMPUTE, REUSE = 0, 1
OK, EINVAL, ESTATE, ENOMEM, EDEVICE = 0, -1, -2, -3, -4
BF16, F32 = 0, 1
NONE, GELU = 0, 1                              # activations
NORM_NONE, NORM_LAYER, NORM_RMS = 0, 1, 2

EXPORTS = (
    "pab_schedule", "pab_source_step", "pab_window_from_timesteps", "pab_preset", "pab_workspace_bytes", "pab_create", "pab_reset", "pab_attention",
    "pab_attention_compute", "pab_linear", "pab_module_scratch_bytes", "pab_module_compute", "pab_module_attention",
    "pab_module_static_scratch_bytes", "pab_module_compute_static",
    "pab_mlp_schedule", "pab_mlp_source_step", "pab_steps_from_timesteps", "pab_mlp_scratch_bytes", "pab_mlp_compute",
    "pab_mlp_workspace_bytes", "pab_mlp_create", "pab_mlp_reset", "pab_mlp", "pab_mlp_launch_count", "pab_mlp_slot_ptr",
    "pab_mlp_destroy",
    "pab_quantized_bytes", "pab_quantized_layout", "pab_quantize", "pab_dequantize", "pab_linear_quantized",
    "pab_mlp_scratch_bytes_quantized", "pab_mlp_compute_quantized",
    "pab_workspace_bytes_quantized", "pab_create_quantized", "pab_attention_quantized", "pab_module_attention_quantized",
    "pab_slot_quantized", "pab_qk_norm_rope", "pab_rope_factors_count", "pab_rope_factors",
    "pab_launch_count", "pab_slot_ptr", "pab_destroy", "pab_last_error",
)


class PabError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("libpab status %d: %s" % (status, message))
        self.status = status


class pab_config(ctypes.Structure):
    _fields_ = [("n_blocks", ctypes.c_int), ("T", ctypes.c_int), ("S", ctypes.c_int), ("L", ctypes.c_int),
                ("heads", ctypes.c_int), ("head_dim", ctypes.c_int), ("dtype", ctypes.c_int),
                ("n_steps", ctypes.c_int), ("interval", ctypes.c_int * 3),
                ("range_lo", ctypes.c_int), ("range_hi", ctypes.c_int),
                ("block_kinds", ctypes.POINTER(ctypes.c_ubyte))]


class pab_module_weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("shift", "scale", "w_qkv", "b_qkv", "gamma_q", "beta_q", "gamma_k",
                                               "beta_k", "w_kv", "b_kv", "w_o", "b_o")]


class pab_mlp_weights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("shift", "scale", "w1", "b1", "w2", "b2")]


class pab_mlp_config(ctypes.Structure):
    _fields_ = [("n_blocks", ctypes.c_int), ("n_steps", ctypes.c_int), ("n_tok", ctypes.c_longlong),
                ("hidden", ctypes.c_int), ("inner", ctypes.c_int), ("n_starts", ctypes.c_int), ("range", ctypes.c_int),
                ("block_lo", ctypes.c_int), ("block_hi", ctypes.c_int)]


class pab_q8(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("ld", ctypes.c_longlong), ("ld_scale", ctypes.c_longlong)]


class pab_mlp_weights_quantized(ctypes.Structure):
    _fields_ = [("shift", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("w1", pab_q8), ("b1", ctypes.c_void_p), ("w2", pab_q8),
                ("b2", ctypes.c_void_p)]


class pab_qk_norm(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int) for n in ("dtype", "norm", "n_batch", "heads_q", "heads_k", "head_dim")]
                + [("places", ctypes.c_int * 3), ("axis_dim", ctypes.c_int * 3), ("eps", ctypes.c_float)]
                + [(n, ctypes.c_void_p) for n in ("q", "k", "q_out", "k_out")]
                + [(n, ctypes.c_longlong) for n in ("ld_q", "ld_k", "ld_q_out", "ld_k_out")]
                + [(n, ctypes.c_void_p) for n in ("gamma_q", "beta_q", "gamma_k", "beta_k", "factors")])


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            "libpab.so is not built (%s missing): run `python -m paper_2408_12588_amd.build` "
            "or __graft_entry__.build(); there is no fallback path" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    vp, ci = ctypes.c_void_p, ctypes.c_int
    lib.pab_schedule.restype = ci
    lib.pab_schedule.argtypes = [ci] * 5
    lib.pab_source_step.restype = ci
    lib.pab_source_step.argtypes = [ci] * 5
    lib.pab_window_from_timesteps.restype = ci
    lib.pab_window_from_timesteps.argtypes = [ctypes.POINTER(ctypes.c_double), ci, ctypes.c_double, ctypes.c_double,
                                              ctypes.POINTER(ci), ctypes.POINTER(ci)]
    lib.pab_preset.restype = ci
    lib.pab_preset.argtypes = [ci, ci, ctypes.POINTER(ci), ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    lib.pab_workspace_bytes.restype = ctypes.c_size_t
    lib.pab_workspace_bytes.argtypes = [ctypes.POINTER(pab_config)]
    lib.pab_create.restype = ci
    lib.pab_create.argtypes = [ctypes.POINTER(pab_config), vp, ctypes.c_size_t, ctypes.POINTER(vp)]
    lib.pab_reset.restype = ci
    lib.pab_reset.argtypes = [vp]
    lib.pab_attention.restype = ci
    lib.pab_attention.argtypes = [vp, ci, ci, ci, vp, vp, vp, vp, ctypes.POINTER(vp)]
    lib.pab_attention_compute.restype = ci
    lib.pab_attention_compute.argtypes = [ci] * 7 + [vp] * 5
    lib.pab_linear.restype = ci
    lib.pab_linear.argtypes = [ci, ci, ci, vp, vp, vp, vp, ctypes.c_longlong, vp]
    lib.pab_module_scratch_bytes.restype = ctypes.c_size_t
    lib.pab_module_scratch_bytes.argtypes = [ctypes.POINTER(pab_config)]
    lib.pab_module_compute.restype = ci
    lib.pab_module_compute.argtypes = [ci] * 6 + [vp, vp, ctypes.POINTER(pab_module_weights), vp, ctypes.c_size_t, vp, vp]
    lib.pab_module_static_scratch_bytes.restype = ctypes.c_size_t
    lib.pab_module_static_scratch_bytes.argtypes = []
    lib.pab_module_compute_static.restype = ci
    lib.pab_module_compute_static.argtypes = [ci] * 6 + [vp, vp, ctypes.POINTER(pab_module_weights), vp, vp]
    lib.pab_module_attention.restype = ci
    lib.pab_module_attention.argtypes = [vp, ci, ci, ci, vp, vp, ctypes.POINTER(pab_module_weights), vp,
                                         ctypes.c_size_t, vp, ctypes.POINTER(vp)]
    ip, dp = ctypes.POINTER(ci), ctypes.POINTER(ctypes.c_double)
    lib.pab_mlp_schedule.restype = ci
    lib.pab_mlp_schedule.argtypes = [ci, ci, ip, ci, ci, ci, ci]
    lib.pab_mlp_source_step.restype = ci
    lib.pab_mlp_source_step.argtypes = [ci, ci, ip, ci, ci, ci, ci]
    lib.pab_steps_from_timesteps.restype = ci
    lib.pab_steps_from_timesteps.argtypes = [dp, ci, dp, ci, ip]
    lib.pab_mlp_scratch_bytes.restype = ctypes.c_size_t
    lib.pab_mlp_scratch_bytes.argtypes = [ctypes.c_longlong, ci, ci]
    lib.pab_mlp_compute.restype = ci
    lib.pab_mlp_compute.argtypes = [ctypes.c_longlong, ci, ci, vp, ctypes.POINTER(pab_mlp_weights), vp, ctypes.c_size_t, vp, vp]
    lib.pab_mlp_workspace_bytes.restype = ctypes.c_size_t
    lib.pab_mlp_workspace_bytes.argtypes = [ctypes.POINTER(pab_mlp_config)]
    lib.pab_mlp_create.restype = ci
    lib.pab_mlp_create.argtypes = [ctypes.POINTER(pab_mlp_config), ip, vp, ctypes.c_size_t, ctypes.POINTER(vp)]
    lib.pab_mlp_reset.restype = ci
    lib.pab_mlp_reset.argtypes = [vp]
    lib.pab_mlp.restype = ci
    lib.pab_mlp.argtypes = [vp, ci, ci, vp, ctypes.POINTER(pab_mlp_weights), vp, ctypes.c_size_t, vp, vp, ctypes.POINTER(vp)]
    lib.pab_mlp_launch_count.restype = ctypes.c_longlong
    lib.pab_mlp_launch_count.argtypes = [vp]
    lib.pab_mlp_slot_ptr.restype = vp
    lib.pab_mlp_slot_ptr.argtypes = [vp, ci]
    lib.pab_mlp_destroy.restype = ci
    lib.pab_mlp_destroy.argtypes = [vp]
    q8p, ll, sz, cfgp = ctypes.POINTER(pab_q8), ctypes.c_longlong, ctypes.c_size_t, ctypes.POINTER(pab_config)
    for name, restype, argtypes in (
            ("pab_quantized_bytes", sz, [ll, ci]),
            ("pab_quantized_layout", ci, [ll, ci, vp, sz, q8p]),
            ("pab_quantize", ci, [ll, ci, ci, vp, ll, q8p, vp]),
            ("pab_dequantize", ci, [ll, ci, ci, q8p, vp, ll, vp, vp, ll, vp]),
            ("pab_linear_quantized", ci, [ci, ci, ci, q8p, q8p, vp, ci, vp, ll, q8p, vp]),
            ("pab_mlp_scratch_bytes_quantized", sz, [ll, ci, ci]),
            ("pab_mlp_compute_quantized", ci, [ll, ci, ci, vp, ctypes.POINTER(pab_mlp_weights_quantized), vp, sz, vp, vp]),
            ("pab_workspace_bytes_quantized", sz, [cfgp]),
            ("pab_create_quantized", ci, [cfgp, vp, sz, ctypes.POINTER(vp)]),
            ("pab_attention_quantized", ci, [vp, ci, ci, ci, vp, vp, vp, vp, sz, vp, q8p]),
            ("pab_module_attention_quantized", ci, [vp, ci, ci, ci, vp, vp, ctypes.POINTER(pab_module_weights), vp, sz, vp, q8p]),
            ("pab_slot_quantized", ci, [vp, ci, ci, q8p]),
            ("pab_qk_norm_rope", ci, [ctypes.POINTER(pab_qk_norm), vp]),
            ("pab_rope_factors_count", ll, [ip, ip]),
            ("pab_rope_factors", ci, [ip, ip, dp, dp, ctypes.c_double, vp, vp])):
        getattr(lib, name).restype = restype
        getattr(lib, name).argtypes = argtypes
    lib.pab_launch_count.restype = ctypes.c_longlong
    lib.pab_launch_count.argtypes = [vp]
    lib.pab_slot_ptr.restype = vp
    lib.pab_slot_ptr.argtypes = [vp, ci, ci]
    lib.pab_destroy.restype = ci
    lib.pab_destroy.argtypes = [vp]
    lib.pab_last_error.restype = ctypes.c_char_p
    lib.pab_last_error.argtypes = []
    return lib


lib = _load()


def pab_last_error() -> str:
    return lib.pab_last_error().decode()


def _check(status: int) -> int:
    if status < 0:
        raise PabError(status, pab_last_error())
    return status


def pab_schedule(kind: int, step: int, range_lo: int, range_hi: int, interval: int) -> int:
    return _check(lib.pab_schedule(kind, step, range_lo, range_hi, interval))


def pab_source_step(kind: int, step: int, range_lo: int, range_hi: int, interval: int) -> int:
    return _check(lib.pab_source_step(kind, step, range_lo, range_hi, interval))


OPEN_SORA, OPEN_SORA_PLAN, LATTE = 0, 1, 2


def pab_window_from_timesteps(timesteps, t_start: float, t_end: float):
    """(range_lo, range_hi) of the timestep window on this sampler's steps, or None if no step is inside."""
    n = len(timesteps)
    arr = (ctypes.c_double * n)(*[float(t) for t in timesteps])
    lo, hi = ctypes.c_int(-1), ctypes.c_int(-1)
    r = _check(lib.pab_window_from_timesteps(arr, n, float(t_start), float(t_end), ctypes.byref(lo), ctypes.byref(hi)))
    return None if r == 0 else (lo.value, hi.value)


def pab_preset(model: int, level: int):
    """((spatial, temporal, cross) broadcast ranges, t_start, t_end) of one of the paper's settings."""
    iv = (ctypes.c_int * 3)()
    a, b = ctypes.c_double(), ctypes.c_double()
    _check(lib.pab_preset(model, level, iv, ctypes.byref(a), ctypes.byref(b)))
    return tuple(iv), a.value, b.value


def make_config(n_blocks, T, S, L, heads, head_dim, dtype, n_steps, interval, range_lo, range_hi,
                block_kinds=None) -> pab_config:
    """``block_kinds``: optional sequence of n_blocks bit masks (bit k = the block has attention of kind k)."""
    cfg = pab_config(n_blocks, T, S, L, heads, head_dim, dtype, n_steps, (ctypes.c_int * 3)(*interval),
                     range_lo, range_hi, None)
    if block_kinds is not None:
        if len(block_kinds) != n_blocks:
            raise ValueError("block_kinds needs one entry per block")
        mask = (ctypes.c_ubyte * n_blocks)(*block_kinds)
        cfg.block_kinds = ctypes.cast(mask, ctypes.POINTER(ctypes.c_ubyte))
        cfg._mask = mask   # keeps the array alive as long as the struct
    return cfg


def config_of(wl, intervals=None) -> pab_config:
    """pab_config of a ``workloads.Workload`` (optionally with other broadcast ranges,
    e.g. (1, 1, 1) masked to the present kinds for the no-broadcast baseline)."""
    iv = tuple(wl.intervals if intervals is None else intervals)
    iv = tuple(i if w > 0 else 0 for i, w in zip(iv, wl.intervals))
    mask = None
    if wl.alternating:   # blocks that hold one kind each get one slot each
        mask = [sum(1 << k for k in wl.kinds_of_block(b)) for b in range(wl.n_blocks)]
    return make_config(wl.n_blocks, wl.T, wl.S, wl.L, wl.heads, wl.head_dim,
                       BF16 if wl.dtype == "bf16" else F32, wl.n_steps, iv, wl.lo, wl.hi, mask)


def pab_workspace_bytes(cfg: pab_config) -> int:
    n = lib.pab_workspace_bytes(ctypes.byref(cfg))
    if n == 0:
        raise PabError(EINVAL, pab_last_error())
    return n


class _NoBinding:
    """In the place of the native binding: hands every call back to the Python code."""

    @staticmethod
    def attention(*args):
        return NotImplemented

    attention_compute = q8_ok = quantize = dequantize = linear_quantized = qk_norm_rope = attention

    @staticmethod
    def bind_q8(q8_type):
        pass


def _load_binding():
    """csrc/pab_binding.cpp as built for this Python and this torch; without it the same calls are marshalled here, by ctypes."""
    path = binding_path(torch.__version__)
    if not os.path.exists(path):
        return _NoBinding
    try:
        spec = importlib.util.spec_from_file_location(__package__ + "._binding", path)
        binding = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(binding)
        if not hasattr(binding, "bind_q8"):
            raise ImportError("built from an earlier source")
    except ImportError as e:
        warnings.warn("%s does not load: calls go through ctypes (%s)" % (os.path.basename(path), e))
        return _NoBinding
    binding.bind(_check, getattr(torch._C, "_cuda_getDevice", None), getattr(torch._C, "_cuda_getCurrentRawStream", None))
    return binding


_binding = _load_binding()


def _stream(stream) -> int:
    if stream is None:
        # The current stream's handle without a Stream object around it: 0.3 us instead of 2.7, of 4.2 us that a reused
        # call took in all.  These two functions are not part of torch's public interface: a build without them takes the
        # public way below.
        try:
            if torch.cuda.is_initialized():
                return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except AttributeError:
            pass
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _ptr(t) -> int:
    if t is None:
        return 0
    if isinstance(t, int):
        return t
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("libpab takes dense device tensors")
    return t.data_ptr()


_TORCH_DTYPE = {BF16: torch.bfloat16, F32: torch.float32}


class PabContext:
    """pab_create / pab_attention / pab_reset / pab_destroy over a workspace
    tensor that this object keeps alive (the C library only borrows it)."""

    def __init__(self, cfg: pab_config, device="cuda:0", workspace: torch.Tensor | None = None):
        self.cfg = cfg
        need = pab_workspace_bytes(cfg)
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=device)
        self.workspace = workspace
        handle = ctypes.c_void_p()
        _check(lib.pab_create(ctypes.byref(cfg), workspace.data_ptr(), workspace.numel(), ctypes.byref(handle)))
        self._h = handle
        self._address = handle.value
        self.shape = (cfg.T, cfg.S, cfg.heads, cfg.head_dim)
        self.dtype = _TORCH_DTYPE[cfg.dtype]
        self._numel = cfg.T * cfg.S * cfg.heads * cfg.head_dim

    def pab_attention(self, block: int, kind: int, step: int, q, k, v, stream=None):
        """-> (decision, device pointer of the slot)."""
        done = _binding.attention(self._address, block, kind, step, q, k, v, stream)
        if done is not NotImplemented:
            return done
        out = ctypes.c_void_p()
        dec = _check(lib.pab_attention(self._h, block, kind, step, _ptr(q), _ptr(k), _ptr(v), _stream(stream),
                                       ctypes.byref(out)))
        return dec, out.value

    def pab_module_attention(self, block: int, kind: int, step: int, x, text, w, scratch, stream=None):
        """Module-level call -> (decision, device pointer of the slot holding the module output [T, S, C])."""
        out = ctypes.c_void_p()
        dec = _check(lib.pab_module_attention(
            self._h, block, kind, step, _ptr(x), _ptr(text), ctypes.byref(w) if w is not None else None,
            _ptr(scratch), scratch.numel() if scratch is not None else 0, _stream(stream), ctypes.byref(out)))
        return dec, out.value

    def slot_tensor(self, block: int, kind: int) -> torch.Tensor:
        """View of cache slot (block, kind) inside the workspace tensor (no copy)."""
        p = lib.pab_slot_ptr(self._h, block, kind)
        if not p:
            raise PabError(EINVAL, "no such slot")
        off = p - self.workspace.data_ptr()
        nbytes = self._numel * self.workspace.new_empty(0, dtype=self.dtype).element_size()
        return self.workspace[off:off + nbytes].view(self.dtype).view(self.shape)

    def pab_slot_ptr(self, block: int, kind: int) -> int:
        return lib.pab_slot_ptr(self._h, block, kind) or 0

    def pab_reset(self):
        _check(lib.pab_reset(self._h))

    def pab_launch_count(self) -> int:
        return lib.pab_launch_count(self._h)

    def pab_destroy(self):
        if self._h:
            self._address = None
            _check(lib.pab_destroy(self._h))
            self._h = None

    def __del__(self):
        try:
            self.pab_destroy()
        except Exception:
            pass


def pab_attention_compute(kind: int, q, k, v, out=None, L: int | None = None, stream=None):
    """One attention launch without schedule or cache.  q ``[T, S, H, D]``;
    k, v ``[T, S, H, D]`` (spatial, temporal) or ``[L, H, D]`` (cross)."""
    if out is not None and _binding.attention_compute(kind, q, k, v, out, stream) is None:
        return out
    T, S, H, D = q.shape
    dtype = BF16 if q.dtype == torch.bfloat16 else F32
    if q.dtype not in (torch.bfloat16, torch.float32) or k.dtype != q.dtype or v.dtype != q.dtype:
        raise ValueError("q, k, v must share dtype bf16 or f32")
    if kind == CROSS:
        if k.dim() != 3 or tuple(k.shape[1:]) != (H, D) or v.shape != k.shape:
            raise ValueError("cross attention wants k, v of shape [L, H, D]")
        L = k.shape[0]
    else:
        if k.shape != q.shape or v.shape != q.shape:
            raise ValueError("k, v must have the shape of q")
        L = 0
    if out is None:
        out = torch.empty_like(q)
    _check(lib.pab_attention_compute(kind, dtype, T, S, L, H, D, _ptr(q), _ptr(k), _ptr(v), _ptr(out),
                                     _stream(stream)))
    return out


def pab_linear(a, w, bias=None, out=None, stream=None):
    """out = a @ w.T + bias (bf16).  a ``[..., K]`` dense, w ``[N, K]``, bias ``[N]`` or None.  ``out`` may be a
    view whose last axis is dense and whose rows are ``out.stride(-2)`` apart (several projections side by side)."""
    if a.dtype != torch.bfloat16 or w.dtype != torch.bfloat16 or (bias is not None and bias.dtype != torch.bfloat16):
        raise ValueError("pab_linear takes bf16 tensors")
    if not a.is_contiguous() or not w.is_contiguous():
        raise ValueError("a and w must be contiguous")
    K = a.shape[-1]
    N = w.shape[0]
    M = a.numel() // K
    if w.shape[1] != K:
        raise ValueError("w must be [N, K]")
    if out is None:
        out = torch.empty(a.shape[:-1] + (N,), device=a.device, dtype=torch.bfloat16)
    if out.stride(-1) != 1 or out.shape[-1] != N or out.numel() != M * N:
        raise ValueError("out must be [..., N] with a dense last axis")
    if not out.is_cuda:
        raise ValueError("libpab takes device tensors")
    ldc = out.stride(-2) if out.dim() >= 2 else N
    if out.dim() > 2 and any(out.stride(i) != out.stride(i + 1) * out.shape[i + 1] for i in range(out.dim() - 2)):
        raise ValueError("the leading axes of out must collapse into one row index")
    _check(lib.pab_linear(M, N, K, _ptr(a), _ptr(w), _ptr(bias) if bias is not None else None, out.data_ptr(), ldc,
                          _stream(stream)))
    return out


def module_weights(**tensors):
    """pab_module_weights from bf16 device tensors given by field name; keeps them alive on the result."""
    w = pab_module_weights()
    for name, t in tensors.items():
        if t is None:
            continue
        if t.dtype != torch.bfloat16:
            raise ValueError("module weights are bf16")
        setattr(w, name, _ptr(t))
    w._keep = tensors
    return w


def pab_module_scratch_bytes(cfg: pab_config) -> int:
    n = lib.pab_module_scratch_bytes(ctypes.byref(cfg))
    if n == 0:
        raise PabError(EINVAL, pab_last_error())
    return n


def module_scratch(T, S, L, heads, head_dim, device):
    """A scratch tensor (uint8, 256-byte aligned by the allocator) for module calls of this shape."""
    cfg = make_config(1, T, S, max(L, 1), heads, head_dim, BF16, 1, (1, 1, 1), 0, 0)
    return torch.empty(pab_module_scratch_bytes(cfg), dtype=torch.uint8, device=device)


def pab_module_compute(kind: int, x, text, w: pab_module_weights, heads: int, scratch=None, out=None, stream=None):
    """One attention module without schedule or cache: x ``[T, S, C]`` (text ``[L, C]`` for cross) -> ``[T, S, C]``."""
    T, S, C = x.shape
    D = C // heads
    L = text.shape[0] if text is not None else 0
    if scratch is None:
        scratch = module_scratch(T, S, L, heads, D, x.device)
    if out is None:
        out = torch.empty_like(x)
    _check(lib.pab_module_compute(kind, T, S, L, heads, D, _ptr(x), _ptr(text) if text is not None else None,
                                  ctypes.byref(w), _ptr(scratch), scratch.numel(), _ptr(out), _stream(stream)))
    return out


def pab_module_static_scratch_bytes() -> int:
    return lib.pab_module_static_scratch_bytes()


def pab_module_compute_static(kind: int, x, text, w: pab_module_weights, heads: int, out, stream=None):
    """pab_module_compute with the library's built-in scratch: nothing is allocated, ``out`` is the caller's."""
    T, S, C = x.shape
    D = C // heads
    L = text.shape[0] if text is not None else 0
    _check(lib.pab_module_compute_static(kind, T, S, L, heads, D, _ptr(x), _ptr(text) if text is not None else None,
                                         ctypes.byref(w), _ptr(out), _stream(stream)))
    return out


# ---- MLP broadcast ----------------------------------------------------------------------------
def _int_array(values):
    return (ctypes.c_int * max(len(values), 1))(*values)


def pab_mlp_schedule(step, block, start_steps, rng, block_lo, block_hi) -> int:
    return _check(lib.pab_mlp_schedule(step, block, _int_array(start_steps), len(start_steps), rng, block_lo, block_hi))


def pab_mlp_source_step(step, block, start_steps, rng, block_lo, block_hi) -> int:
    return _check(lib.pab_mlp_source_step(step, block, _int_array(start_steps), len(start_steps), rng, block_lo, block_hi))


def pab_steps_from_timesteps(timesteps, start_timesteps):
    """Step index of each starting timestep on the sampler's list (None where no step qualifies)."""
    ts = (ctypes.c_double * len(timesteps))(*[float(t) for t in timesteps])
    st = (ctypes.c_double * max(len(start_timesteps), 1))(*[float(t) for t in start_timesteps])
    out = (ctypes.c_int * max(len(start_timesteps), 1))()
    _check(lib.pab_steps_from_timesteps(ts, len(timesteps), st, len(start_timesteps), out))
    return [None if out[i] < 0 else out[i] for i in range(len(start_timesteps))]


def mlp_weights(**tensors):
    w = pab_mlp_weights()
    for name, t in tensors.items():
        if t is None:
            continue
        if t.dtype != torch.bfloat16:
            raise ValueError("MLP weights are bf16")
        setattr(w, name, _ptr(t))
    w._keep = tensors
    return w


def mlp_scratch(n_tok, hidden, inner, device):
    return torch.empty(lib.pab_mlp_scratch_bytes(n_tok, hidden, inner), dtype=torch.uint8, device=device)


def pab_mlp_compute(x, w: pab_mlp_weights, inner: int, scratch=None, out=None, stream=None):
    """One MLP module without schedule or cache: x ``[..., C]`` bf16 -> same shape."""
    C = x.shape[-1]
    n_tok = x.numel() // C
    if scratch is None:
        scratch = mlp_scratch(n_tok, C, inner, x.device)
    if out is None:
        out = torch.empty_like(x)
    _check(lib.pab_mlp_compute(n_tok, C, inner, _ptr(x), ctypes.byref(w), _ptr(scratch), scratch.numel(), _ptr(out),
                               _stream(stream)))
    return out


class MlpContext:
    """Owns the cache slab (a torch uint8 tensor) and the library context of one MLP-broadcast run."""

    def __init__(self, n_blocks, n_steps, n_tok, hidden, inner, start_steps, rng, block_lo, block_hi, device="cuda:0"):
        self.cfg = pab_mlp_config(n_blocks, n_steps, n_tok, hidden, inner, len(start_steps), rng, block_lo, block_hi)
        nbytes = lib.pab_mlp_workspace_bytes(ctypes.byref(self.cfg))
        self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        handle = ctypes.c_void_p()
        _check(lib.pab_mlp_create(ctypes.byref(self.cfg), _int_array(start_steps), _ptr(self.workspace), nbytes,
                                  ctypes.byref(handle)))
        self._h = handle
        self.shape = (n_tok, hidden)

    def pab_mlp(self, block, step, x, w, scratch, y=None, stream=None):
        """-> (decision, device pointer of the output)."""
        out = ctypes.c_void_p()
        dec = _check(lib.pab_mlp(self._h, block, step, _ptr(x), ctypes.byref(w) if w is not None else None, _ptr(scratch),
                                 scratch.numel() if scratch is not None else 0, _ptr(y), _stream(stream), ctypes.byref(out)))
        return dec, out.value

    def slot_tensor(self, block):
        """View of the cache slot of a participating block inside the workspace tensor (no copy)."""
        p = lib.pab_mlp_slot_ptr(self._h, block)
        if not p:
            raise PabError(EINVAL, "block %d has no MLP cache slot" % block)
        off = p - self.workspace.data_ptr()
        return self.workspace[off:off + self.shape[0] * self.shape[1] * 2].view(torch.bfloat16).view(self.shape)

    def pab_mlp_reset(self):
        _check(lib.pab_mlp_reset(self._h))

    def pab_mlp_launch_count(self) -> int:
        return lib.pab_mlp_launch_count(self._h)

    def pab_mlp_destroy(self):
        if self._h:
            lib.pab_mlp_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.pab_mlp_destroy()
        except Exception:
            pass


# ---- 8-bit rows -------------------------------------------------------------------------------
def _rows_of(t, name):
    """(rows, columns, row pitch in elements) of a device tensor whose last axis is dense and whose leading axes collapse."""
    if not t.is_cuda:
        raise ValueError("libpab takes device tensors (%s)" % name)
    if t.dim() == 0 or t.stride(-1) != 1 and t.shape[-1] != 1:
        raise ValueError("%s needs a dense last axis" % name)
    K = t.shape[-1]
    if t.is_contiguous():
        return (t.numel() // K if K else 0), K, K
    lead = [(n, st) for n, st in zip(t.shape[:-1], t.stride()[:-1]) if n != 1]
    if any(a[1] != b[1] * b[0] for a, b in zip(lead, lead[1:])):
        raise ValueError("the leading axes of %s must collapse into one row index" % name)
    rows = 1
    for n, _ in lead:
        rows *= n
    return rows, K, (lead[-1][1] if lead else K)


def _float_type(t, name):
    if t.dtype is torch.bfloat16:
        return BF16
    if t.dtype is torch.float32:
        return F32
    raise ValueError("%s must be bf16 or f32" % name)


def _same_device(first, *others):
    """All on the current device: launches go to its current stream."""
    i = first.get_device()
    if any(t is not None and t.get_device() != i for t in others):
        raise ValueError("the tensors are on different devices")
    if i != torch.cuda.current_device():
        raise ValueError("the tensors are on device %d, the current device is %d" % (i, torch.cuda.current_device()))


def _new(shape, dtype, device, stream):
    """A tensor that belongs to the stream on which the launch will write it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


class Q8:
    """8-bit rows: ``data`` [rows, >= K rounded up to 128] (uint8 or e4m3), ``scale`` [rows, ...] exponent bytes (uint8 or e8m0), device
    tensors that this object keeps; ``K`` columns of values."""
    __slots__ = ("data", "scale", "K")

    def __init__(self, data, scale, K: int):
        self.data, self.scale, self.K = data, scale, K
        if _binding.q8_ok(data, scale, K) is True:
            return
        if data.dtype not in (torch.uint8, torch.float8_e4m3fn) or scale.dtype not in (torch.uint8, torch.float8_e8m0fnu):
            raise ValueError("data must be uint8 or e4m3, scale uint8 or e8m0, not %s and %s" % (data.dtype, scale.dtype))
        if data.dim() != 2 or scale.dim() != 2:
            raise ValueError("data and scale are matrices of bytes")
        if not data.is_cuda or not scale.is_cuda:
            raise ValueError("libpab takes device tensors")
        if data.get_device() != scale.get_device():
            raise ValueError("data and scale are on different devices")
        if data.shape[0] != scale.shape[0]:
            raise ValueError("data has %d rows, scale %d" % (data.shape[0], scale.shape[0]))
        nb = (K + 127) // 128
        if K < 1 or data.shape[1] < 128 * nb or scale.shape[1] < nb or data.stride(1) != 1 or scale.stride(1) != 1:
            raise ValueError("K=%d wants dense rows of at least %d bytes and %d scales" % (K, 128 * nb, nb))

    @property
    def struct(self) -> pab_q8:
        return pab_q8(self.data.data_ptr(), self.scale.data_ptr(), self.data.stride(0), self.scale.stride(0))

    @property
    def rows(self) -> int:
        return self.data.shape[0]


_binding.bind_q8(Q8)


def _q8_of(data, scale, K: int) -> Q8:
    """Rows whose tensors are known to fit."""
    y = Q8.__new__(Q8)
    y.data, y.scale, y.K = data, scale, K
    return y


def q8_empty(rows: int, K: int, device="cuda:0", stream=None) -> Q8:
    """Uninitialised 8-bit rows."""
    nb = (K + 127) // 128
    return Q8(_new((rows, 128 * nb), torch.uint8, device, stream), _new((rows, (nb + 3) // 4 * 4), torch.uint8, device, stream), K)


def pab_quantized_bytes(rows: int, K: int) -> int:
    return lib.pab_quantized_bytes(rows, K)


def q8_view(buffer, rows: int, K: int) -> Q8:
    """8-bit rows in one uint8 tensor of pab_quantized_bytes, as pab_quantized_layout places them."""
    s = pab_q8()
    _check(lib.pab_quantized_layout(rows, K, _ptr(buffer), buffer.numel(), ctypes.byref(s)))
    return _q8_inside(buffer, s, rows, K)


def _q8_inside(buffer, s: pab_q8, rows: int, K: int) -> Q8:
    a, b = s.data - buffer.data_ptr(), s.scale - buffer.data_ptr()
    return Q8(buffer[a:a + rows * s.ld].view(rows, s.ld), buffer[b:b + rows * s.ld_scale].view(rows, s.ld_scale), K)


def pab_quantize(x, out: Q8 | None = None, stream=None) -> Q8:
    """x ``[..., K]`` bf16 or f32 (dense last axis) -> 8-bit rows."""
    if out is None:
        done = _binding.quantize(x, stream)
        if done is not NotImplemented:
            return _q8_of(*done)
    dtype = _float_type(x, "x")
    rows, K, ldx = _rows_of(x, "x")
    if out is None:
        out = q8_empty(rows, K, x.device, stream)
    elif out.rows != rows or out.K != K:
        raise ValueError("out holds [%d, %d], x is [%d, %d]" % (out.rows, out.K, rows, K))
    _same_device(x, out.data)
    _check(lib.pab_quantize(rows, K, dtype, x.data_ptr(), ldx, out.struct, _stream(stream)))
    return out


def pab_dequantize(y: Q8, x=None, gate=None, dtype=None, out=None, stream=None):
    """out = x + gate * y: x ``[..., K]`` or None (0), gate ``[K]`` or None (1); type and shape of x, else ``dtype`` (bf16) and [rows, K]."""
    done = _binding.dequantize(y, x, gate, dtype, out, stream)
    if done is not NotImplemented:
        return done
    if dtype is None:
        dtype = x.dtype if x is not None else out.dtype if out is not None else torch.bfloat16
    ldx = 0
    if x is not None:
        rows, K, ldx = _rows_of(x, "x")
        if (rows, K) != (y.rows, y.K) or x.dtype != dtype:
            raise ValueError("x must be [%d, %d] of %s" % (y.rows, y.K, dtype))
    if gate is not None and (gate.dtype != dtype or gate.numel() != y.K or not gate.is_contiguous()):
        raise ValueError("gate must be a dense [%d] of %s" % (y.K, dtype))
    if out is None:
        out = _new(x.shape if x is not None else (y.rows, y.K), dtype, y.data.device, stream)
    rows, K, ldo = _rows_of(out, "out")
    if (rows, K) != (y.rows, y.K) or out.dtype != dtype:
        raise ValueError("out must be [%d, %d] of %s" % (y.rows, y.K, dtype))
    _same_device(y.data, x, gate, out)
    _check(lib.pab_dequantize(rows, K, _float_type(out, "out"), y.struct, 0 if x is None else x.data_ptr(), ldx,
                              0 if gate is None else gate.data_ptr(), out.data_ptr(), ldo, _stream(stream)))
    return out


def pab_linear_quantized(a: Q8, w: Q8, bias=None, act: int = NONE, out=None, stream=None):
    """act(a @ w.T + bias) of 8-bit rows a [M, K], w [N, K]; bias ``[N]`` bf16 or None.  ``out``: a bf16 tensor ``[..., N]`` (new if None),
    or a ``Q8`` [M, N] that the result is quantised into."""
    done = _binding.linear_quantized(a, w, bias, act, out, stream)
    if done is not NotImplemented:
        return done
    M, N, K = a.rows, w.rows, a.K
    if w.K != K:
        raise ValueError("a has %d columns, w %d" % (K, w.K))
    if bias is not None and (bias.dtype is not torch.bfloat16 or bias.numel() != N or not bias.is_contiguous()):
        raise ValueError("bias must be a dense [%d] of bf16" % N)
    if out is None:
        out = _new((M, N), torch.bfloat16, a.data.device, stream)
    if isinstance(out, Q8):
        if out.rows != M or out.K != N:
            raise ValueError("out holds [%d, %d], the product is [%d, %d]" % (out.rows, out.K, M, N))
        c, ldc, c8, where = 0, 0, out.struct, out.data
    else:
        rows, cols, ldc = _rows_of(out, "out")
        if (rows, cols) != (M, N) or out.dtype is not torch.bfloat16:
            raise ValueError("out must be [%d, %d] of bf16" % (M, N))
        c, c8, where = out.data_ptr(), None, out
    _same_device(a.data, w.data, bias, where)
    _check(lib.pab_linear_quantized(M, N, K, a.struct, w.struct, 0 if bias is None else bias.data_ptr(), act, c, ldc, c8, _stream(stream)))
    return out


def mlp_weights_quantized(shift, scale, w1: Q8, b1, w2: Q8, b2) -> pab_mlp_weights_quantized:
    """Weights of pab_mlp_compute_quantized: shift, scale ``[hidden]``, b1 ``[inner]``, b2 ``[hidden]`` bf16 (b1, b2 may be None), w1, w2 8-bit
    rows; kept alive on the result."""
    hidden, inner = w1.K, w1.rows
    if w2.rows != hidden or w2.K != inner:
        raise ValueError("w1 is [%d, %d], w2 [%d, %d]" % (inner, hidden, w2.rows, w2.K))
    for name, t, n in (("shift", shift, hidden), ("scale", scale, hidden), ("b1", b1, inner), ("b2", b2, hidden)):
        if t is None and name in ("b1", "b2"):
            continue
        if t.dtype is not torch.bfloat16 or t.numel() != n:
            raise ValueError("%s must be [%d] of bf16" % (name, n))
    if any(t is not None and t.get_device() != w1.data.get_device() for t in (shift, scale, b1, w2.data, b2)):
        raise ValueError("the weights are on different devices")
    w = pab_mlp_weights_quantized(_ptr(shift), _ptr(scale), w1.struct, _ptr(b1), w2.struct, _ptr(b2))
    w._keep = (shift, scale, w1, b1, w2, b2)
    w._shape = (hidden, inner)
    return w


def pab_mlp_scratch_bytes_quantized(n_tok: int, hidden: int, inner: int) -> int:
    return lib.pab_mlp_scratch_bytes_quantized(n_tok, hidden, inner)


def pab_mlp_compute_quantized(x, w: pab_mlp_weights_quantized, scratch=None, out=None, stream=None):
    """One MLP module on 8-bit rows, without schedule or cache: x ``[..., hidden]`` bf16 -> same shape."""
    hidden, inner = w._shape
    if x.dtype is not torch.bfloat16 or x.shape[-1] != hidden:
        raise ValueError("x must be [..., %d] of bf16" % hidden)
    n_tok = x.numel() // hidden
    if scratch is None:
        scratch = _new((lib.pab_mlp_scratch_bytes_quantized(n_tok, hidden, inner),), torch.uint8, x.device, stream)
    if out is None:
        out = _new(x.shape, torch.bfloat16, x.device, stream)
    if out.dtype is not torch.bfloat16 or out.shape != x.shape:
        raise ValueError("out must have the shape and type of x")
    _same_device(x, w._keep[2].data, scratch, out)
    _check(lib.pab_mlp_compute_quantized(n_tok, hidden, inner, _ptr(x), ctypes.byref(w), _ptr(scratch), scratch.numel(), _ptr(out),
                                         _stream(stream)))
    return out


class QuantizedContext(PabContext):
    """A broadcast cache of 8-bit rows: pab_create_quantized and the calls that go with it."""

    def __init__(self, cfg: pab_config, device="cuda:0", workspace: torch.Tensor | None = None):
        self.cfg, self._h, self._address = cfg, None, None
        need = lib.pab_workspace_bytes_quantized(ctypes.byref(cfg))
        if need == 0:
            raise PabError(EINVAL, pab_last_error())
        if workspace is None:
            workspace = torch.empty(need, dtype=torch.uint8, device=device)
        self.workspace = workspace
        handle = ctypes.c_void_p()
        _check(lib.pab_create_quantized(ctypes.byref(cfg), workspace.data_ptr(), workspace.numel(), ctypes.byref(handle)))
        self._h = handle
        self._address = handle.value
        self.shape = (cfg.T, cfg.S, cfg.heads, cfg.head_dim)
        self.dtype = _TORCH_DTYPE[cfg.dtype]
        self._numel = cfg.T * cfg.S * cfg.heads * cfg.head_dim

    def slot_tensor(self, block: int, kind: int) -> Q8:
        """Cache slot (block, kind) inside the workspace tensor (no copy)."""
        s = pab_q8()
        _check(lib.pab_slot_quantized(self._h, block, kind, ctypes.byref(s)))
        return _q8_inside(self.workspace, s, self.cfg.T * self.cfg.S, self.cfg.heads * self.cfg.head_dim)

    def pab_attention_quantized(self, block: int, kind: int, step: int, q, k, v, scratch, stream=None):
        """-> (decision, the slot as 8-bit rows).  scratch: uint8, the bytes of one output tensor (computed steps)."""
        s = pab_q8()
        dec = _check(lib.pab_attention_quantized(self._h, block, kind, step, _ptr(q), _ptr(k), _ptr(v), _ptr(scratch),
                                                 scratch.numel() if scratch is not None else 0, _stream(stream), ctypes.byref(s)))
        return dec, _q8_inside(self.workspace, s, self.cfg.T * self.cfg.S, self.cfg.heads * self.cfg.head_dim)

    def pab_module_attention_quantized(self, block: int, kind: int, step: int, x, text, w, scratch, stream=None):
        """Module-level call -> (decision, the slot as 8-bit rows); scratch as for pab_module_attention."""
        s = pab_q8()
        dec = _check(lib.pab_module_attention_quantized(
            self._h, block, kind, step, _ptr(x), _ptr(text), ctypes.byref(w) if w is not None else None, _ptr(scratch),
            scratch.numel() if scratch is not None else 0, _stream(stream), ctypes.byref(s)))
        return dec, _q8_inside(self.workspace, s, self.cfg.T * self.cfg.S, self.cfg.heads * self.cfg.head_dim)


# ---- query / key norm with rotation over several axes -----------------------------------------
def pab_rope_factors_count(places, axis_dim) -> int:
    return _check(lib.pab_rope_factors_count(_int_array(places), _int_array(axis_dim)))


def pab_rope_factors(places, axis_dim, origin=(0.0, 0.0, 0.0), step=(1.0, 1.0, 1.0), theta: float = 10000.0, device="cuda:0", stream=None):
    """The table of pab_qk_norm_rope, fp32 ``[count, 2]``: built once for a video's shape."""
    if not len(places) == len(axis_dim) == len(origin) == len(step) == 3:
        raise ValueError("three axes (one place and no features for an axis that a model lacks)")
    n = pab_rope_factors_count(places, axis_dim)
    out = _new((n, 2), torch.float32, device, stream)
    three = ctypes.c_double * 3
    if n:
        _same_device(out)
    _check(lib.pab_rope_factors(_int_array(places), _int_array(axis_dim), three(*origin), three(*step), theta, out.data_ptr(), _stream(stream)))
    return out


def _heads_of(t, name):
    """(tokens, heads, head dim, token pitch) of ``[..., H, D]`` whose heads are dense."""
    if t.dim() < 3 or not t.is_cuda:
        raise ValueError("%s must be a device tensor [..., heads, head_dim]" % name)
    H, D = t.shape[-2:]
    if t.is_contiguous():
        return t.numel() // max(H * D, 1), H, D, H * D
    if t.stride(-1) != 1 or (H > 1 and t.stride(-2) != D):
        raise ValueError("the heads of %s must be dense" % name)
    lead = [(n, st) for n, st in zip(t.shape[:-2], t.stride()[:-2]) if n != 1]
    if any(a[1] != b[1] * b[0] for a, b in zip(lead, lead[1:])):
        raise ValueError("the leading axes of %s must collapse into one token index" % name)
    n = 1
    for m, _ in lead:
        n *= m
    return n, H, D, (lead[-1][1] if lead else H * D)


def pab_qk_norm_rope(q, k, places, axis_dim, factors=None, norm: int = NORM_LAYER, gamma_q=None, beta_q=None, gamma_k=None, beta_k=None,
                     eps: float = 1e-6, q_out=None, k_out=None, stream=None):
    """Norm per head and rotation of q ``[..., Hq, D]`` and k ``[..., Hk, D]`` (or None), tokens in the order of the grid ``places`` (times a
    batch); ``factors`` from pab_rope_factors (None: no rotation).  -> (q_out, k_out); they may be q and k."""
    done = _binding.qk_norm_rope(q, k, places, axis_dim, factors, norm, gamma_q, beta_q, gamma_k, beta_k, eps, q_out, k_out, stream)
    if done is not NotImplemented:
        return done
    n, Hq, D, ld_q = _heads_of(q, "q")
    dtype = _float_type(q, "q")
    grid = places[0] * places[1] * places[2]
    if grid < 1 or n % grid or n == 0:
        raise ValueError("%d tokens are no batch of grids of %s" % (n, tuple(places)))
    if factors is not None and (factors.dtype is not torch.float32 or not factors.is_contiguous()
                                or factors.numel() != 2 * sum(p * (a // 2) for p, a in zip(places, axis_dim))):
        raise ValueError("factors must be the dense f32 table of these places and sections")
    for name, t in (("gamma_q", gamma_q), ("beta_q", beta_q), ("gamma_k", gamma_k), ("beta_k", beta_k)):
        if t is not None and (t.dtype != q.dtype or t.numel() != D or not t.is_contiguous()):
            raise ValueError("%s must be a dense [%d] of the type of q" % (name, D))
    q_out = _new(q.shape, q.dtype, q.device, stream) if q_out is None else q_out
    if q_out.shape != q.shape or q_out.dtype != q.dtype:
        raise ValueError("q_out must have the shape and type of q")
    d = pab_qk_norm(dtype, norm, n // grid, Hq, 0, D, tuple(places), tuple(axis_dim), eps, q.data_ptr(), 0, q_out.data_ptr(), 0,
                    ld_q, 0, _heads_of(q_out, "q_out")[3], 0, *(0 if t is None else t.data_ptr() for t in (gamma_q, beta_q, gamma_k, beta_k, factors)))
    if k is not None:
        m, Hk, Dk, d.ld_k = _heads_of(k, "k")
        if (m, Dk) != (n, D) or k.dtype != q.dtype:
            raise ValueError("k must have the tokens, head dim and type of q")
        k_out = _new(k.shape, k.dtype, k.device, stream) if k_out is None else k_out
        if k_out.shape != k.shape or k_out.dtype != k.dtype:
            raise ValueError("k_out must have the shape and type of k")
        d.heads_k, d.k, d.k_out, d.ld_k_out = Hk, k.data_ptr(), k_out.data_ptr(), _heads_of(k_out, "k_out")[3]
    _same_device(q, k, q_out, k_out, factors, gamma_q, beta_q, gamma_k, beta_k)
    _check(lib.pab_qk_norm_rope(ctypes.byref(d), _stream(stream)))
    return q_out, k_out
