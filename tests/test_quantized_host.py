"""Refusals and host logic of the 8-bit rows and of the query / key norm; nothing here reaches a GPU: every call fails its checks
before a launch, and the pointers are numbers that nobody follows."""
import ctypes
import subprocess
import sys

import pytest

from paper_2408_12588_amd import pab

OK = 1 << 20            # an aligned address


def q8(data=OK, scale=OK, ld=1152, ld_scale=12):
    return pab.pab_q8(data, scale, ld, ld_scale)


def status(name, *args):
    return getattr(pab.lib, name)(*args)


def test_buffer_layout():
    assert pab.pab_quantized_bytes(1, 1) == 512
    assert pab.pab_quantized_bytes(3, 1152) == 3584 + 256        # 3456 -> 3584, 36 -> 256
    assert pab.pab_quantized_bytes(100, 4608) == 100 * 4608 + 3840   # 3600 -> 3840
    for bad in ((0, 8), (-1, 8), (8, 0), (2**40 + 1, 128), (2**40, 2**31 - 1)):
        assert pab.pab_quantized_bytes(*bad) == 0
    s = pab.pab_q8()
    assert status("pab_quantized_layout", 3, 1152, OK, 3840, ctypes.byref(s)) == pab.OK
    assert (s.data, s.scale, s.ld, s.ld_scale) == (OK, OK + 3584, 1152, 12)
    assert status("pab_quantized_layout", 3, 1152, OK, 3839, ctypes.byref(s)) == pab.ENOMEM
    assert status("pab_quantized_layout", 3, 1152, OK + 16, 3840, ctypes.byref(s)) == pab.EINVAL
    assert status("pab_quantized_layout", 3, 1152, 0, 3840, ctypes.byref(s)) == pab.EINVAL
    assert status("pab_quantized_layout", 0, 1152, OK, 3840, ctypes.byref(s)) == pab.EINVAL
    assert status("pab_quantized_layout", 3, 1152, OK, 3840, None) == pab.EINVAL


BAD_ROWS = [q8(data=0), q8(scale=0), q8(data=OK + 8), q8(scale=OK + 2), q8(ld=1024), q8(ld=1160), q8(ld=(1 << 24) + 128), q8(ld=-1152),
            q8(ld_scale=8), q8(ld_scale=13), q8(ld_scale=(1 << 24) + 4)]


@pytest.mark.parametrize("bad", BAD_ROWS)
def test_bad_rows_are_refused(bad):
    assert status("pab_quantize", 4, 1152, pab.BF16, OK, 1152, bad, None) == pab.EINVAL
    assert status("pab_dequantize", 4, 1152, pab.BF16, bad, 0, 0, 0, OK, 1152, None) == pab.EINVAL
    good = q8()
    assert status("pab_linear_quantized", 4, 1152, 1152, bad, good, 0, 0, OK, 1152, None, None) == pab.EINVAL
    assert status("pab_linear_quantized", 4, 1152, 1152, good, bad, 0, 0, OK, 1152, None, None) == pab.EINVAL
    assert status("pab_linear_quantized", 4, 1152, 1152, good, good, 0, 0, 0, 0, bad, None) == pab.EINVAL
    w = pab.pab_mlp_weights_quantized(OK, OK, bad, 0, q8(ld=1152), 0)
    assert status("pab_mlp_compute_quantized", 4, 1152, 1152, OK, w, OK, 1 << 30, OK, None) == pab.EINVAL
    assert pab.pab_last_error()


@pytest.mark.parametrize("rows,K,dtype,x,ldx", [
    (0, 1152, 0, OK, 1152), (-1, 1152, 0, OK, 1152), (4, 0, 0, OK, 1152), (4, 1148, 0, OK, 1152), (4, -8, 0, OK, 1152), (4, 1152, 2, OK, 1152),
    (4, 1152, -1, OK, 1152), (4, 1152, 0, 0, 1152), (4, 1152, 0, OK + 8, 1152), (4, 1152, 0, OK, 1144), (4, 1152, 0, OK, 1156),
    (4, 1152, 1, OK, 1154), (2**31, 1152, 0, OK, 1152), (2**62, 8, 0, OK, 8)])
def test_quantize_and_dequantize_refuse(rows, K, dtype, x, ldx):
    assert status("pab_quantize", rows, K, dtype, x, ldx, q8(), None) == pab.EINVAL
    assert status("pab_dequantize", rows, K, dtype, q8(), 0, 0, 0, x, ldx, None) == pab.EINVAL
    if x:
        assert status("pab_dequantize", rows, K, dtype, q8(), x, ldx, 0, OK, 1152, None) == pab.EINVAL


def test_quantize_refuses_more_threads_than_a_grid_holds():
    """2^28 blocks of 16 threads each are 2^32."""
    y = q8(ld=256, ld_scale=4)
    assert status("pab_quantize", 1 << 28, 128, 0, OK, 128, y, None) == pab.EINVAL
    assert status("pab_quantize", 1 << 27, 256, 1, OK, 256, y, None) == pab.EINVAL
    assert "too many" in pab.pab_last_error()


def test_dequantize_refuses_more_than_its_index_holds():
    """2^31 chunks of 8 columns: the launch splits a chunk's number into row and column by a high product that is exact below that."""
    y = q8(ld=4096, ld_scale=32)
    assert status("pab_dequantize", 1 << 22, 4096, 0, y, 0, 0, 0, OK, 4096, None) == pab.EINVAL
    assert "too many" in pab.pab_last_error()


def test_dequantize_refuses_gate():
    assert status("pab_dequantize", 4, 1152, 0, q8(), 0, 0, OK + 4, OK, 1152, None) == pab.EINVAL


@pytest.mark.parametrize("M,N,K,bias,act,C,ldc,out8", [
    (0, 1152, 1152, 0, 0, OK, 1152, None), (4, 0, 1152, 0, 0, OK, 1152, None), (4, 1148, 1152, 0, 0, OK, 1152, None),
    (4, 1152, 1148, 0, 0, OK, 1152, None), (260, 9120, 1100, 0, 0, OK, 9120, None), (4, 1152, 0, 0, 0, OK, 1152, None), (4, 1152, 1152, OK + 8, 0, OK, 1152, None),
    (4, 1152, 1152, 0, 2, OK, 1152, None), (4, 1152, 1152, 0, -1, OK, 1152, None), (4, 1152, 1152, 0, 0, 0, 1152, None),
    (4, 1152, 1152, 0, 0, OK, 1152, q8()), (4, 1152, 1152, 0, 0, OK + 8, 1152, None), (4, 1152, 1152, 0, 0, OK, 1144, None),
    (4, 1152, 1152, 0, 0, OK, 1156, None), (2**31 - 1, 1152, 1152, 0, 0, OK, 1152, None)])
def test_linear_refuses(M, N, K, bias, act, C, ldc, out8):
    assert status("pab_linear_quantized", M, N, K, q8(), q8(), bias, act, C, ldc, out8, None) == pab.EINVAL


@pytest.mark.parametrize("M,N", [(1, 2**31 - 8), (64, 2**31 - 256), (2**31 - 1, 8)])
def test_linear_refuses_what_its_indexes_do_not_hold(M, N):
    y = q8(ld=128, ld_scale=4)
    assert status("pab_linear_quantized", M, N, 8, y, y, 0, 0, OK, N, None, None) == pab.EINVAL
    assert "too large" in pab.pab_last_error()


def test_linear_refuses_null_operands():
    assert status("pab_linear_quantized", 4, 1152, 1152, None, q8(), 0, 0, OK, 1152, None, None) == pab.EINVAL
    assert status("pab_linear_quantized", 4, 1152, 1152, q8(), None, 0, 0, OK, 1152, None, None) == pab.EINVAL


def test_mlp_refuses():
    good = pab.pab_mlp_weights_quantized(OK, OK, q8(), 0, q8(ld=4608, ld_scale=36), 0)
    need = pab.pab_mlp_scratch_bytes_quantized(4, 1152, 4608)
    assert need == pab.pab_quantized_bytes(4, 1152) + pab.pab_quantized_bytes(4, 4608)

    def call(n=4, C=1152, F=4608, x=OK, w=good, scratch=OK, nbytes=need, out=OK):
        return status("pab_mlp_compute_quantized", n, C, F, x, w, scratch, nbytes, out, None)

    for kw in (dict(n=0), dict(n=2**25 + 1), dict(C=1148), dict(C=2080), dict(F=0), dict(F=4600 + 4), dict(x=0), dict(x=OK + 2), dict(w=None),
               dict(scratch=0), dict(scratch=OK + 16), dict(out=0), dict(out=OK + 8)):
        assert call(**kw) == pab.EINVAL, kw
    assert call(nbytes=need - 1) == pab.ENOMEM
    for kw in (dict(shift=0), dict(scale=0), dict(shift=OK + 2), dict(scale=OK + 2), dict(b1=OK + 2), dict(b2=OK + 2)):
        w = pab.pab_mlp_weights_quantized(kw.get("shift", OK), kw.get("scale", OK), q8(), kw.get("b1", 0), q8(ld=4608, ld_scale=36), kw.get("b2", 0))
        assert call(w=w) == pab.EINVAL, kw


def test_mlp_refuses_products_that_no_launch_holds():
    """... before its layernorm is launched: the status is a refusal also where there is no device."""
    n, C, F = 2**25, 1152, 2**20 + 32
    w = pab.pab_mlp_weights_quantized(OK, OK, q8(), 0, q8(ld=2**20 + 128, ld_scale=8196), 0)
    need = pab.pab_mlp_scratch_bytes_quantized(n, C, F)
    assert need
    assert status("pab_mlp_compute_quantized", n, C, F, OK, w, OK, need, OK, None) == pab.EINVAL
    assert "too large" in pab.pab_last_error()


def config(dtype=pab.BF16, interval=(2, 2, 2)):
    return pab.make_config(2, 4, 8, 16, 4, 32, dtype, 6, interval, 1, 4)


def context(create, cfg):
    h = ctypes.c_void_p()
    assert create(ctypes.byref(cfg), OK, 1 << 30, ctypes.byref(h)) == pab.OK
    return h


def test_contexts_do_not_mix():
    cfg, s, out = config(), pab.pab_q8(), ctypes.c_void_p()
    need = pab.lib.pab_workspace_bytes_quantized(ctypes.byref(cfg))
    assert need == 6 * pab.pab_quantized_bytes(32, 128)
    h = ctypes.c_void_p()
    assert status("pab_create_quantized", ctypes.byref(cfg), OK, need - 1, ctypes.byref(h)) == pab.ENOMEM and not h.value
    assert status("pab_create_quantized", ctypes.byref(cfg), OK + 16, need, ctypes.byref(h)) == pab.EINVAL
    assert status("pab_create_quantized", ctypes.byref(cfg), 0, need, ctypes.byref(h)) == pab.EINVAL
    assert status("pab_create_quantized", None, OK, need, ctypes.byref(h)) == pab.EINVAL
    assert status("pab_create_quantized", ctypes.byref(cfg), OK, need, None) == pab.EINVAL
    a, b = context(pab.lib.pab_create_quantized, cfg), context(pab.lib.pab_create, cfg)
    scratch = pab.pab_module_scratch_bytes(cfg)
    assert status("pab_attention", a, 0, 0, 0, OK, OK, OK, None, ctypes.byref(out)) == pab.EINVAL
    assert status("pab_module_attention", a, 0, 0, 0, OK, OK, None, OK, scratch, None, ctypes.byref(out)) == pab.EINVAL
    assert status("pab_attention_quantized", b, 0, 0, 0, OK, OK, OK, OK, 1 << 20, None, s) == pab.EINVAL
    assert status("pab_module_attention_quantized", b, 0, 0, 0, OK, OK, None, OK, scratch, None, s) == pab.EINVAL
    assert status("pab_slot_quantized", b, 0, 0, s) == pab.EINVAL
    assert status("pab_slot_quantized", a, 1, 2, s) == pab.OK
    assert (s.data, s.ld, s.ld_scale) == (OK + 5 * pab.pab_quantized_bytes(32, 128), 128, 4)
    assert status("pab_slot_quantized", a, 2, 0, s) == pab.EINVAL
    for h in (a, b):
        pab.lib.pab_destroy(h)


def test_quantized_slots_are_what_a_launch_fills():
    """A slot that the quantiser refuses is refused when the context is made, not behind the attention of its first computed step."""
    big = pab.make_config(1, 1 << 14, 1 << 14, 0, 4, 32, pab.BF16, 6, (2, 0, 0), 1, 4)        # 2^28 rows of one block
    fits = pab.make_config(1, 1 << 14, (1 << 14) - 1, 0, 4, 32, pab.BF16, 6, (2, 0, 0), 1, 4)
    h = ctypes.c_void_p()
    assert pab.lib.pab_workspace_bytes_quantized(ctypes.byref(big)) == 0 and "2^28" in pab.pab_last_error()
    assert status("pab_create_quantized", ctypes.byref(big), OK, 1 << 50, ctypes.byref(h)) == pab.EINVAL and not h.value
    with pytest.raises(pab.PabError):
        pab.QuantizedContext(big)
    need = pab.lib.pab_workspace_bytes_quantized(ctypes.byref(fits))
    assert need == pab.pab_quantized_bytes(2**28 - 2**14, 128)
    assert status("pab_create_quantized", ctypes.byref(fits), OK, need, ctypes.byref(h)) == pab.OK
    pab.lib.pab_destroy(h)


OUT_OF_MEMORY = """
import ctypes, resource, sys
lib = ctypes.CDLL(sys.argv[1])
class Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int) for n in ("n_blocks", "T", "S", "L", "heads", "head_dim", "dtype", "n_steps")] + [
        ("interval", ctypes.c_int * 3), ("range_lo", ctypes.c_int), ("range_hi", ctypes.c_int), ("block_kinds", ctypes.c_void_p)]
used = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
resource.setrlimit(resource.RLIMIT_AS, (used + (1 << 30),) * 2)
cfg = Config(2**31 - 1, 1, 1, 0, 4, 32, 0, 4, (2, 0, 0), 0, 3, None)
out = ctypes.c_void_p()
for name in ("pab_create", "pab_create_quantized"):
    f = getattr(lib, name)
    f.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
    assert f(ctypes.byref(cfg), 1 << 20, 1 << 62, ctypes.byref(out)) == -3 and not out.value, name
class MlpConfig(ctypes.Structure):
    _fields_ = [("n_blocks", ctypes.c_int), ("n_steps", ctypes.c_int), ("n_tok", ctypes.c_longlong)] + [
        (n, ctypes.c_int) for n in ("hidden", "inner", "n_starts", "range", "block_lo", "block_hi")]
cfg, start = MlpConfig(2**31 - 1, 4, 8, 32, 32, 1, 2, 0, 1), ctypes.c_int(1)
lib.pab_mlp_create.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
assert lib.pab_mlp_create(ctypes.byref(cfg), ctypes.byref(start), 1 << 20, 1 << 62, ctypes.byref(out)) == -3 and not out.value
"""


def test_contexts_without_host_memory(tmp_path):
    """More blocks than the host has memory for are an error, no exception through the C boundary (which would end the process)."""
    script = tmp_path / "oom.py"
    script.write_text(OUT_OF_MEMORY)
    done = subprocess.run([sys.executable, str(script), pab.LIB_PATH], capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stderr[-2000:]


def test_quantized_context_refuses():
    cfg, s = config(), pab.pab_q8()
    h = context(pab.lib.pab_create_quantized, cfg)
    need = 4 * 8 * 4 * 32 * 2

    def call(block=0, kind=0, step=0, q=OK, scratch=OK, nbytes=need, out=s):
        return status("pab_attention_quantized", h, block, kind, step, q, OK, OK, scratch, nbytes, None, out)

    for kw in (dict(block=2), dict(kind=3), dict(step=6), dict(step=-1), dict(q=0), dict(q=OK + 2), dict(scratch=0), dict(scratch=OK + 2), dict(out=None)):
        assert call(**kw) == pab.EINVAL, kw
    assert call(nbytes=need - 1) == pab.ENOMEM
    assert call(step=2) == pab.ESTATE          # reuse of a slot that holds nothing
    assert s.data is None
    assert status("pab_module_attention_quantized", h, 0, 0, 0, 0, 0, None, OK, 1 << 30, None, s) == pab.EINVAL
    assert status("pab_module_attention_quantized", h, 0, 0, 0, OK, 0, None, 0, 0, None, s) == pab.EINVAL
    pab.lib.pab_destroy(h)
    f = context(pab.lib.pab_create_quantized, config(dtype=pab.F32))
    assert status("pab_module_attention_quantized", f, 0, 0, 0, OK, 0, None, OK, 1 << 30, None, s) == pab.EINVAL
    pab.lib.pab_destroy(f)


def three(*v):
    return (ctypes.c_int * 3)(*v)


def test_rope_factors_refuse():
    assert pab.pab_rope_factors_count((16, 30, 53), (24, 24, 24)) == 12 * 99
    assert pab.pab_rope_factors_count((16, 1, 1), (0, 0, 0)) == 0
    for places, dims in (((0, 1, 1), (8, 8, 8)), ((1, 1, -1), (8, 8, 8)), ((1, 1, 1), (7, 8, 8)), ((1, 1, 1), (-2, 8, 8)),
                         ((2**31 - 1, 1, 1), (8, 0, 0))):
        assert pab.lib.pab_rope_factors_count(three(*places), three(*dims)) == pab.EINVAL
        assert status("pab_rope_factors", three(*places), three(*dims), None, None, 1e4, OK, None) == pab.EINVAL
    dbl = ctypes.c_double * 3
    inf, nan = float("inf"), float("nan")
    for origin, step, theta, out in ((None, None, 0.0, OK), (None, None, -1.0, OK), (None, None, nan, OK), (None, None, inf, OK),
                                     (dbl(0, nan, 0), None, 1e4, OK), (None, dbl(1, 1, inf), 1e4, OK), (None, None, 1e4, 0), (None, None, 1e4, OK + 8)):
        assert status("pab_rope_factors", three(2, 2, 2), three(8, 8, 8), origin, step, theta, out, None) == pab.EINVAL
    assert status("pab_rope_factors", three(2, 2, 2), three(0, 0, 0), None, None, 1e4, 0, None) == pab.OK   # nothing to write
    assert status("pab_rope_factors", None, three(0, 0, 0), None, None, 1e4, 0, None) == pab.EINVAL


def qk(**kw):
    d = pab.pab_qk_norm(pab.BF16, pab.NORM_LAYER, 1, 16, 16, 72, (16, 30, 53), (24, 24, 24), 1e-6, OK, OK, OK, OK, 1152, 1152, 1152, 1152,
                        OK, OK, OK, OK, OK)
    for name, v in kw.items():
        setattr(d, name, v)
    return d


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(norm=3), dict(norm=-1), dict(n_batch=0), dict(heads_q=0), dict(heads_k=-1), dict(head_dim=48), dict(head_dim=0),
    dict(places=(0, 30, 53)), dict(axis_dim=(24, 24, 26)), dict(axis_dim=(23, 24, 24)), dict(axis_dim=(-2, 24, 24)), dict(eps=-1.0),
    dict(eps=float("nan")), dict(q=0), dict(k=0), dict(q_out=0), dict(k_out=0), dict(q=OK + 8), dict(k_out=OK + 2), dict(ld_q=1144),
    dict(ld_k=1156), dict(ld_q_out=1144), dict(ld_k_out=0), dict(gamma_q=OK + 2), dict(beta_k=OK + 2), dict(factors=OK + 8),
    dict(n_batch=2**20), dict(places=(2**20, 2**20, 1))])
def test_qk_norm_refuses(kw):
    assert status("pab_qk_norm_rope", qk(**kw), None) == pab.EINVAL
    assert pab.pab_last_error()


def test_qk_norm_refuses_null():
    assert status("pab_qk_norm_rope", None, None) == pab.EINVAL


def test_python_checks_its_tensors():
    import torch
    x = torch.zeros(4, 128, dtype=torch.bfloat16)
    b = torch.zeros(4, 128, dtype=torch.uint8)
    s = torch.zeros(4, 4, dtype=torch.uint8)
    for f in (lambda: pab.pab_quantize(x), lambda: pab.pab_quantize(x.half()), lambda: pab.Q8(b, s, 128),
              lambda: pab.pab_qk_norm_rope(x.view(4, 4, 32), None, (1, 2, 2), (8, 8, 8)),
              lambda: pab.pab_rope_factors((1, 1), (2, 2))):
        with pytest.raises(ValueError):
            f()


@pytest.mark.parametrize("data,scale", [("float8_e5m2", "uint8"), ("float8_e4m3fnuz", "uint8"), ("float8_e8m0fnu", "uint8"), ("int8", "uint8"),
                                        ("bool", "uint8"), ("uint8", "int8"), ("uint8", "float8_e4m3fn"), ("float32", "uint8")])
def test_other_bytes_are_no_rows(data, scale):
    """Bytes of another meaning would be read as e4m3 values and powers of two."""
    import torch
    with pytest.raises(ValueError, match="uint8 or e4m3"):
        pab.Q8(torch.zeros(4, 128, dtype=torch.uint8).to(getattr(torch, data)), torch.zeros(4, 4, dtype=torch.uint8).view(getattr(torch, scale)), 128)


def test_mlp_weights_are_on_one_device():
    import torch

    class Stub:
        """What the check looks at of a device tensor."""
        dtype = torch.bfloat16

        def __init__(self, n, device):
            self.n, self.device = n, device

        def numel(self):
            return self.n

        def get_device(self):
            return self.device

    def rows(n, K, device):
        return pab._q8_of(type("data", (), {"shape": (n, K), "get_device": lambda self: device})(), None, K)

    devices = [0] * 6
    for i in range(6):
        d = list(devices)
        d[i] = 1
        with pytest.raises(ValueError, match="different devices"):
            pab.mlp_weights_quantized(Stub(64, d[0]), Stub(64, d[1]), rows(128, 64, d[2]), Stub(128, d[3]), rows(64, 128, d[4]), Stub(64, d[5]))
