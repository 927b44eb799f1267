"""Cases for the 8-bit operators and for query / key norm with rotation over several axes.

Five operators, as a program around the attention calls them through ``paper_2408_12588_amd.pab``:

  quantize   rows of bf16 or fp32 values -> 8-bit rows: activations before a product, a broadcast slot as it is written
  read       8-bit rows -> values, added to the residual stream with a gate: a broadcast slot read back
  linear     C = act(A W^T + bias) of 8-bit rows
  qk         norm of queries and keys per head and rotation by frame, row and column, one pass
  mlp        layernorm + modulate, product with GELU, product, everything between them in 8-bit rows

8-bit rows of a matrix [R, K]: e4m3 bytes [R, 128 ceil(K / 128)], zero behind column K, and one scale for 128 columns of a
row, 2^(byte - 127), bytes [R, 4 ceil(K / 512)].  The scale of a block is the smallest power of two, 2^-127 at least,
for which its largest value stays within 448.

``own`` false: plain torch operations in fp32.  ``own`` true: the library's kernels.  ``exact``: the definitions in fp64.
Values are N(0,1) and weight rows have about unit norm, as everywhere in this repository.
"""
import math

import torch

own = False

DEV = "cuda:0"
FLOAT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ---------------------------------------------------------------------------------------------------------


def listed():
    return [
        # One token through a quantiser: the embedding of the timestep before its product, the smallest call there is.
        dict(name="quantize_one", form="quantize", dtype="bf16", rows=1, K=1152),
        # The output of a computed attention module of the 480p configuration, written into its broadcast slot.
        dict(name="quantize_480p", form="quantize", dtype="bf16", rows=25440, K=1152),
        # A slot of a tiny fp32 model read back, ...
        dict(name="read_tiny", form="read", dtype="f32", rows=256, K=128, residual=False),
        # ... and one of the 480p configuration, with the gated residual that follows every module.
        dict(name="read_480p", form="read", dtype="bf16", rows=25440, K=1152, residual=True),
        # Modulation vectors from the embedding of a timestep: one token, six times the hidden size.
        dict(name="linear_one", form="linear", M=1, N=6912, K=1152, act="none"),
        # A small clip: five frames of 252 tokens, hidden size 576 into an MLP, far too few tiles for the chip.
        dict(name="linear_small_gelu", form="linear", M=1260, N=2304, K=576, act="gelu"),
        # The query / key / value projection of the 480p configuration ...
        dict(name="linear_qkv_480p", form="linear", M=25440, N=3456, K=1152, act="none"),
        # ... and the MLP's second product at 720p, the longest.
        dict(name="linear_720p", form="linear", M=57600, N=1152, K=4608, act="none"),
        # Queries and keys of the tiny fp32 model, heads of 32, ...
        dict(name="qk_tiny", form="qk", dtype="f32", batch=1, T=4, Y=8, X=8, heads_q=4, heads_k=4, head_dim=32, norm="layer",
             axes="8,12,12"),
        # ... and of the 480p configuration: 16 frames of 30 x 53 tokens, 16 heads of 72 in three equal sections.
        dict(name="qk_480p", form="qk", dtype="bf16", batch=1, T=16, Y=30, X=53, heads_q=16, heads_k=16, head_dim=72, norm="layer",
             axes="24,24,24"),
        # The MLP of a block of the small clip and of the 480p configuration.
        dict(name="mlp_small", form="mlp", rows=1260, hidden=576, inner=2304),
        dict(name="mlp_480p", form="mlp", rows=25440, hidden=1152, inner=4608),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    form = rng.choice(["quantize", "read", "linear", "linear", "linear", "qk", "qk", "mlp"])
    if form in ("quantize", "read"):
        K = 8 * _log_int(rng, 1, 576)
        rows = _log_int(rng, 1, min(57600, 25440 * 1152 // K))
        case = dict(form=form, dtype=rng.choice(["bf16", "bf16", "f32"]), rows=rows, K=K)
        if form == "read":
            case["residual"] = rng.random() < 0.7
        return case
    if form == "linear":
        K, N = 8 * _log_int(rng, 4, 576), 8 * _log_int(rng, 4, 864)
        return dict(form=form, M=_log_int(rng, 1, 57600 * 1152 * 4608 // max(N * K, 1152 * 4608)), N=N, K=K, act=rng.choice(["none", "gelu"]))
    if form == "qk":
        D = rng.choice([32, 64, 72, 96, 128])
        t = 2 * rng.randint(0, D // 8)
        y = 2 * rng.randint(0, (D - t) // 4)
        x = y if rng.random() < 0.7 else 2 * rng.randint(0, (D - t - y) // 2)
        heads_q = rng.randint(1, 1152 // D)
        return dict(form=form, dtype=rng.choice(["bf16", "bf16", "f32"]), batch=rng.randint(1, 2), T=rng.randint(1, 17), Y=_log_int(rng, 1, 32),
                    X=_log_int(rng, 1, 40), heads_q=heads_q, heads_k=heads_q if rng.random() < 0.6 else rng.randint(1, heads_q), head_dim=D,
                    norm=rng.choice(["none", "layer", "rms"]), axes="%d,%d,%d" % (t, y, x))
    hidden = 32 * rng.randint(4, 36)
    return dict(form=form, rows=_log_int(rng, 1, 25440), hidden=hidden, inner=rng.choice([2, 3, 4]) * hidden)


# ---- the format, in plain operations -------------------------------------------------------------------------------


def _blocks(K):
    return -(-K // 128)


def _two_to(e):
    """2^e of whole numbers, exactly, in fp64."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _quantise(x):
    """fp32 [R, K] -> e4m3 bytes [R, 128 b] and scale bytes [R, 4 ceil(b / 4)], both uint8."""
    R, K = x.shape
    nb = _blocks(K)
    x = torch.nn.functional.pad(x, (0, 128 * nb - K)).view(R, nb, 128)
    big = x.abs().amax(-1)
    m, e = torch.frexp(big)                                        # big = m 2^e, 1/2 <= m < 1; 448 = 0.875 * 2^9
    e = torch.where(big > 0, e - 9 + (m > 0.875).int(), -127).clamp(min=-127)
    inv = _two_to(-e).float()
    data = (x * inv[..., None]).to(torch.float8_e4m3fn).view(torch.uint8).view(R, 128 * nb)
    scale = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -nb % 4))
    return data, scale


def _values(data, scale, K):
    """fp32 [R, K] that 8-bit rows stand for."""
    R, nb = data.shape[0], _blocks(K)
    s = _two_to(scale[:, :nb].int() - 127).float()
    return (data[:, :128 * nb].view(torch.float8_e4m3fn).float().view(R, nb, 128) * s[..., None]).reshape(R, 128 * nb)[:, :K]


def _gelu(x):
    return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))


def _as_out(data, scale, K):
    return data[:, :K].view(torch.float8_e4m3fn), scale[:, :_blocks(K)].view(torch.float8_e8m0fnu)


# ---- states --------------------------------------------------------------------------------------------------------


def _axes(case):
    return tuple(int(a) for a in case["axes"].split(","))


def _factors(case):
    """(cos, sin) of every position of every axis, fp32 [n, 2]: what a program builds once for a video's shape."""
    parts = []
    for n, d in zip((case["T"], case["Y"], case["X"]), _axes(case)):
        if d:
            i = torch.arange(0, d, 2, dtype=torch.float64, device=DEV)
            a = torch.arange(n, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (-i / d)
            parts.append(torch.stack([a.cos(), a.sin()], -1).reshape(-1, 2))
    return torch.cat(parts).float() if parts else None


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    form = case["form"]
    s = dict(case=case)
    if form == "quantize":
        s["x"] = normal(case["rows"], case["K"]).to(FLOAT[case["dtype"]])
    elif form == "read":
        s["data"], s["scale"] = _quantise(normal(case["rows"], case["K"]))
        if case["residual"]:
            s["x"] = normal(case["rows"], case["K"]).to(FLOAT[case["dtype"]])
            s["gate"] = normal(case["K"]).to(FLOAT[case["dtype"]])
    elif form == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        s["a"] = _quantise(normal(M, K))
        s["w"] = _quantise(normal(N, K) / math.sqrt(K))
        s["bias"] = normal(N).bfloat16()
    elif form == "qk":
        t = FLOAT[case["dtype"]]
        n, D = case["batch"] * case["T"] * case["Y"] * case["X"], case["head_dim"]
        s["q"], s["k"] = normal(n, case["heads_q"], D).to(t), normal(n, case["heads_k"], D).to(t)
        s["weights"] = [(1 + 0.1 * normal(D)).to(t), (0.1 * normal(D)).to(t), (1 + 0.1 * normal(D)).to(t), (0.1 * normal(D)).to(t)]
        s["factors"] = _factors(case)
        s["axes"] = _axes(case)
    else:
        C, F = case["hidden"], case["inner"]
        s["x"] = normal(case["rows"], C).bfloat16()
        s["shift"], s["mod"] = (0.1 * normal(C)).bfloat16(), (0.1 * normal(C)).bfloat16()
        s["w1"], s["w2"] = _quantise(normal(F, C) / math.sqrt(C)), _quantise(normal(C, F) / math.sqrt(F))
        s["b1"], s["b2"] = normal(F).bfloat16(), normal(C).bfloat16()
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------


def _run_own(s):
    from paper_2408_12588_amd import pab
    case = s["case"]
    form = case["form"]
    if form == "quantize":
        y = pab.pab_quantize(s["x"])
        return _as_out(y.data, y.scale, case["K"])
    if form == "read":
        return pab.pab_dequantize(pab.Q8(s["data"], s["scale"], case["K"]), s.get("x"), s.get("gate"), dtype=FLOAT[case["dtype"]])
    if form == "linear":
        a, w = pab.Q8(*s["a"], case["K"]), pab.Q8(*s["w"], case["K"])
        return pab.pab_linear_quantized(a, w, s["bias"], act=pab.GELU if case["act"] == "gelu" else pab.NONE)
    if form == "qk":
        norm = {"none": pab.NORM_NONE, "layer": pab.NORM_LAYER, "rms": pab.NORM_RMS}[case["norm"]]
        return pab.pab_qk_norm_rope(s["q"], s["k"], (case["T"], case["Y"], case["X"]), s["axes"], s["factors"], norm, *s["weights"], eps=1e-6)
    w = pab.mlp_weights_quantized(s["shift"], s["mod"], pab.Q8(*s["w1"], case["hidden"]), s["b1"], pab.Q8(*s["w2"], case["inner"]), s["b2"])
    return pab.pab_mlp_compute_quantized(s["x"], w)


def _norm(v, norm, gamma, beta, eps):
    if norm == "layer":
        v = v - v.mean(-1, keepdim=True)
    if norm != "none":
        v = v * torch.rsqrt((v * v).mean(-1, keepdim=True) + eps)
    return v * gamma + beta


def _rotate(v, case, factors, axes):
    """fp32 [n, H, D]: neighbouring pairs of each axis's section turned by the token's place on that axis."""
    T, Y, X = case["T"], case["Y"], case["X"]
    token = torch.arange(v.shape[0], device=v.device) % (T * Y * X)
    places = (token // (Y * X), token // X % Y, token % X)
    columns, first = [], 0
    for place, n, d in zip(places, (T, Y, X), axes):
        if d:
            columns.append(factors[first:first + n * (d // 2)].view(n, d // 2, 2)[place])
            first += n * (d // 2)
    if not columns:
        return v
    f = torch.cat(columns, 1)[:, None]
    r = 2 * f.shape[2]
    a, b = v[..., 0:r:2], v[..., 1:r:2]
    turned = torch.stack([a * f[..., 0] - b * f[..., 1], a * f[..., 1] + b * f[..., 0]], -1).flatten(-2)
    return torch.cat([turned, v[..., r:]], -1)


def run(state):
    if own:
        return _run_own(state)
    s = state
    case = s["case"]
    form = case["form"]
    if form == "quantize":
        return _as_out(*_quantise(s["x"].float()), case["K"])
    if form == "read":
        y = _values(s["data"], s["scale"], case["K"])
        if case["residual"]:
            y = s["x"].float() + s["gate"].float() * y
        return y.to(FLOAT[case["dtype"]])
    if form == "linear":
        y = _values(*s["a"], case["K"]) @ _values(*s["w"], case["K"]).T + s["bias"].float()
        return (_gelu(y) if case["act"] == "gelu" else y).bfloat16()
    if form == "qk":
        gq, bq, gk, bk = (w.float() for w in s["weights"])
        q = _rotate(_norm(s["q"].float(), case["norm"], gq, bq, 1e-6), case, s["factors"], s["axes"])
        k = _rotate(_norm(s["k"].float(), case["norm"], gk, bk, 1e-6), case, s["factors"], s["axes"])
        return q.to(s["q"].dtype), k.to(s["k"].dtype)
    C, F = case["hidden"], case["inner"]
    h = _norm(s["x"].float(), "layer", 1 + s["mod"].float(), s["shift"].float(), 1e-6)
    h = _values(*_quantise(h), C)
    u = _gelu(h @ _values(*s["w1"], C).T + s["b1"].float())
    u = _values(*_quantise(u), F)
    return (u @ _values(*s["w2"], F).T + s["b2"].float()).bfloat16()


def work(case):
    form = case["form"]
    if form in ("quantize", "read"):
        wide = case["rows"] * case["K"] * FLOAT[case["dtype"]].itemsize
        eight = case["rows"] * (case["K"] + _blocks(case["K"]))
        return {"bytes": eight + wide * (2 if case.get("residual") else 1), "flops": 0}
    if form == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": (M + N) * (K + _blocks(K)) + 2 * N + 2 * M * N, "flops": 2.0 * M * N * K}
    if form == "qk":
        n = case["batch"] * case["T"] * case["Y"] * case["X"]
        return {"bytes": 2 * n * (case["heads_q"] + case["heads_k"]) * case["head_dim"] * FLOAT[case["dtype"]].itemsize, "flops": 0}
    R, C, F = case["rows"], case["hidden"], case["inner"]
    return {"bytes": 4 * R * C + 2 * F * C, "flops": 4.0 * R * C * F}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------


def _exact_round(x):
    """fp64 [R, K] -> the e4m3 values and the scales of its 8-bit rows, as fp64 numbers."""
    R, K = x.shape
    nb = _blocks(K)
    z = torch.zeros(R, 128 * nb, dtype=torch.float64, device=x.device)
    z[:, :K] = x
    z = z.view(R, nb, 128)
    m, e = torch.frexp(z.abs().amax(-1) / 448)
    e = torch.where(m > 0.5, e, e - 1)
    s = _two_to(torch.where(m > 0, e, torch.full_like(e, -127)).clamp(min=-127))
    v = z / s[..., None]
    _, f = torch.frexp(v)
    step = _two_to((f - 1).clamp(min=-6) - 3)                      # three bits behind the leading one
    return (torch.round(v / step) * step).view(R, 128 * nb)[:, :K], s


def _exact_value(data, scale, K):
    """fp64 values of stored 8-bit rows, decoded bit by bit."""
    d = data[:, :K].int()
    sign = 1.0 - 2.0 * (d >> 7).double()
    e, m = (d >> 3) & 15, (d & 7).double()
    v = sign * torch.where(e > 0, (1 + m / 8) * _two_to(e - 7), m / 512)
    s = _two_to(scale.int() - 127)
    return v * torch.repeat_interleave(s, 128, 1)[:, :K]


def exact(case, seed):
    s = prepare(case, seed)
    form = case["form"]
    if form == "quantize":
        return _exact_round(s["x"].double())
    if form == "read":
        y = _exact_value(s["data"], s["scale"], case["K"])
        return s["x"].double() + s["gate"].double() * y if case["residual"] else y

    def gelu(x):
        return x / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))

    if form == "linear":
        y = _exact_value(*s["a"], case["K"]) @ _exact_value(*s["w"], case["K"]).T.contiguous() + s["bias"].double()
        return gelu(y) if case["act"] == "gelu" else y
    if form == "qk":
        out = []
        T, Y, X = case["T"], case["Y"], case["X"]
        for x, gamma, beta in ((s["q"], *s["weights"][:2]), (s["k"], *s["weights"][2:])):
            v = x.double()
            if case["norm"] == "layer":
                v = (v - v.mean(-1, keepdim=True)) / torch.sqrt(v.var(-1, unbiased=False, keepdim=True) + 1e-6)
            elif case["norm"] == "rms":
                v = v / torch.sqrt(v.square().mean(-1, keepdim=True) + 1e-6)
            v = v * gamma.double() + beta.double()
            grid = torch.cartesian_prod(*(torch.arange(n, dtype=torch.float64, device=DEV) for n in (T, Y, X))).view(-1, 3).repeat(case["batch"], 1)
            first = 0
            for a, d in enumerate(s["axes"]):
                if d:
                    c = torch.view_as_complex(v[..., first:first + d].reshape(*v.shape[:2], d // 2, 2).contiguous())
                    angle = grid[:, a, None] * 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64, device=DEV) / d)
                    c = c * torch.polar(torch.ones_like(angle), angle)[:, None]
                    v[..., first:first + d] = torch.view_as_real(c).flatten(-2)
                    first += d
            out.append(v)
        return tuple(out)
    C, F = case["hidden"], case["inner"]

    def rounded(x):
        v, e = _exact_round(x)
        return v * torch.repeat_interleave(e, 128, 1)[:, :x.shape[1]]

    x = s["x"].double()
    h = (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, unbiased=False, keepdim=True) + 1e-6)
    h = rounded(h * (1 + s["mod"].double()) + s["shift"].double())
    u = rounded(gelu(h @ _exact_value(*s["w1"], C).T.contiguous() + s["b1"].double()))
    return u @ _exact_value(*s["w2"], F).T.contiguous() + s["b2"].double()
