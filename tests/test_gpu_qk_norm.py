"""Query / key norm with rotation over several axes against the fp64 definition.

Tolerance of an element: one rounding of the output type (2^-8 or 2^-24 of it), and fp32 arithmetic before: sums over the head dimension D are at
most D 2^-24 of their terms off, a handful of products follow, all relative to the largest normed value of its row (a rotation mixes pairs):
(D + 16) 2^-23 of that, and of what the mean takes away times 1 / sigma."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as qo
from paper_2408_12588_amd import pab

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
NORMS = {"none": pab.NORM_NONE, "layer": pab.NORM_LAYER, "rms": pab.NORM_RMS}


def normal(seed, *shape):
    return torch.from_numpy(np.random.Generator(np.random.Philox(seed)).standard_normal(shape, dtype=np.float32))


def check(got, x, places, dims, norm, gamma, beta, eps, rotate=True, **angles):
    D = x.shape[-1]
    f64 = lambda t: None if t is None else t.double().numpy()   # noqa: E731
    flat = f64(x).reshape(-1, *x.shape[-2:])
    args = (norm, f64(gamma), f64(beta), eps)
    want = qo.qk_norm_rope(flat, places, dims, *args, rotate, **angles)
    straight = qo.qk_norm_rope(flat, places, dims, *args, False)
    sigma = np.sqrt(flat.var(-1, keepdims=True) + eps) if norm == "layer" else np.inf
    big = np.abs(straight).max(-1, keepdims=True) + np.abs(flat.mean(-1, keepdims=True)) / sigma
    if gamma is not None:
        big = big * (1 + np.abs(f64(gamma)).max())
    tol = HALF[x.dtype] * np.abs(want) + (D + 16) * 2.0 ** -23 * big
    err = np.abs(got.cpu().double().numpy().reshape(want.shape) - want)
    assert np.all(err <= tol), float((err / tol).max())


def weights(D, dtype, seed):
    return tuple((base + 0.3 * normal(seed + i, D)).to(dtype) for i, base in enumerate((1, 0, 1, 0)))


CASES = [
    (32, (4, 8, 8), (8, 12, 12), 4, 4, 1), (72, (3, 5, 7), (24, 24, 24), 16, 16, 2), (72, (1, 1, 1), (24, 24, 24), 16, 16, 1),
    (64, (2, 3, 5), (16, 24, 24), 9, 3, 1), (96, (5, 1, 6), (32, 0, 64), 12, 1, 3), (128, (3, 4, 2), (16, 56, 56), 8, 2, 2),
    (128, (7, 1, 1), (128, 0, 0), 1, 1, 1), (72, (17, 2, 1), (72, 0, 0), 5, 5, 1), (32, (1, 13, 1), (0, 30, 0), 3, 7, 1),
    (72, (2, 2, 11), (2, 14, 6), 2, 1, 1), (64, (6, 1, 1), (0, 0, 0), 2, 2, 1)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("norm", ["none", "layer", "rms"])
@pytest.mark.parametrize("D,places,dims,Hq,Hk,batch", CASES)
def test_against_definition(D, places, dims, Hq, Hk, batch, norm, dtype):
    n = batch * places[0] * places[1] * places[2]
    q, k = (normal(D + n, n, Hq, D) * 3 + 1).to(dtype), normal(D + n + 1, n, Hk, D).to(dtype)
    gq, bq, gk, bk = weights(D, dtype, 50)
    f = pab.pab_rope_factors(places, dims, device=DEV)
    dev = [t.to(DEV) for t in (gq, bq, gk, bk)]
    qd, kd = q.to(DEV), k.to(DEV)
    qo_, ko_ = pab.pab_qk_norm_rope(qd, kd, places, dims, f, NORMS[norm], *dev, eps=1e-6)
    check(qo_, q, places, dims, norm, gq, bq, 1e-6)
    check(ko_, k, places, dims, norm, gk, bk, 1e-6)
    assert torch.equal(qd.cpu(), q) and torch.equal(kd.cpu(), k)
    q2, k2 = pab.pab_qk_norm_rope(qd, kd, places, dims, f, NORMS[norm], *dev, eps=1e-6, q_out=qd, k_out=kd)   # in place
    assert q2 is qd and torch.equal(qd, qo_) and torch.equal(kd, ko_)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [32, 64, 72, 96, 128])
def test_without_weights_factors_or_keys(D, dtype):
    q, k = normal(1, 11, 3, D).to(dtype), normal(2, 11, 2, D).to(dtype)
    for norm in NORMS:
        a, b = pab.pab_qk_norm_rope(q.to(DEV), k.to(DEV), (1, 1, 11), (0, 0, 0), None, NORMS[norm], eps=1e-5)
        check(a, q, (1, 1, 11), (0, 0, 0), norm, None, None, 1e-5, False)
        check(b, k, (1, 1, 11), (0, 0, 0), norm, None, None, 1e-5, False)
        c, none = pab.pab_qk_norm_rope(q.to(DEV), None, (1, 1, 11), (0, 0, 0), None, NORMS[norm], eps=1e-5)
        assert none is None and torch.equal(a, c)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [32, 72, 128])
def test_parts_of_one_buffer(D, dtype):
    """q, k, v side by side as a projection leaves them, rotated in place; v and what lies around stay as they are."""
    H, places, dims = 4, (2, 3, 4), (8, 8, 16)
    buf = normal(3, 24 + 2, 3 * H * D + 16).to(dtype).to(DEV)
    kept = buf.clone()
    body = buf[1:25, 8:8 + 3 * H * D].view(24, 3, H, D)
    q, k = body[:, 0], body[:, 1]
    q0, k0 = q.cpu().clone(), k.cpu().clone()
    f = pab.pab_rope_factors(places, dims, device=DEV)
    gq, bq, gk, bk = weights(D, dtype, 9)
    pab.pab_qk_norm_rope(q, k, places, dims, f, pab.NORM_RMS, gq.to(DEV), bq.to(DEV), gk.to(DEV), bk.to(DEV), q_out=q, k_out=k)
    check(q, q0, places, dims, "rms", gq, bq, 1e-6)
    check(k, k0, places, dims, "rms", gk, bk, 1e-6)
    q.copy_(q0), k.copy_(k0)
    assert torch.equal(buf, kept)


def test_rows_without_spread_or_finite_values():
    """A constant row has no variance: eps keeps it finite.  A row with a NaN or infinity stays alone with it."""
    q = normal(4, 6, 2, 72)
    q[1, 0], q[2, 1] = 5.0, 0.0
    q[3, 0, 7], q[4, 1, 0] = float("nan"), float("inf")
    f = pab.pab_rope_factors((6, 1, 1), (24, 24, 24), device=DEV)
    for norm in ("layer", "rms"):
        out, _ = pab.pab_qk_norm_rope(q.to(DEV), None, (6, 1, 1), (24, 24, 24), f, NORMS[norm], eps=1e-6)
        out = out.cpu()
        assert bool(out[3, 0].isnan().all()) and not bool(out[4, 1].isfinite().all())
        bad = torch.zeros(6, 2, dtype=torch.bool)
        bad[3, 0] = bad[4, 1] = True
        assert bool(out[~bad].isfinite().all())
        if norm == "layer":
            assert float(out[1, 0].abs().max()) <= 2e-3 and float(out[2, 1].abs().max()) == 0.0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,dims", [(72, (8, 8, 8)), (72, (2, 14, 6)), (32, (0, 10, 0)), (128, (56, 0, 16)), (64, (0, 0, 0))])
def test_what_is_not_turned_keeps_its_value(D, dims, dtype):
    """Behind the last section nothing meets its neighbour: infinities and NaNs stay where they are, and the bits are those of a call
    without a table."""
    end, inf = sum(dims), float("inf")
    q = normal(5, 6, 3, D).to(dtype)
    q[0, 0, end], q[1, 1, end + 1], q[2, 2, D - 1], q[3, 0, D - 2] = inf, -inf, inf, float("nan")
    q[4, 1, end:] = -0.0
    places = (1, 3, 2)
    f = pab.pab_rope_factors(places, dims, device=DEV)
    out, _ = pab.pab_qk_norm_rope(q.to(DEV), None, places, dims, f, pab.NORM_NONE)
    plain, _ = pab.pab_qk_norm_rope(q.to(DEV), None, places, dims, None, pab.NORM_NONE)
    bits = torch.int16 if dtype == torch.bfloat16 else torch.int32
    out, plain = out.cpu(), plain.cpu()
    finite = q.isfinite()
    assert torch.equal(out.isfinite(), finite)
    same = finite[..., end:]
    assert torch.equal(out[..., end:].contiguous().view(bits)[same], plain[..., end:].contiguous().view(bits)[same])
    assert torch.equal(out[..., end:][~same & ~q[..., end:].isnan()], q[..., end:][~same & ~q[..., end:].isnan()])
    gamma = torch.full((D,), 3e38).to(dtype)                  # products that overflow behind the section
    gamma[:end] = 1.0
    q = normal(6, 6, 3, D).to(dtype)
    q[..., end::2], q[..., end + 1::2] = 4.0, 0.25
    out, _ = pab.pab_qk_norm_rope(q.to(DEV), None, places, dims, f, pab.NORM_NONE, gamma_q=gamma.to(DEV))
    out = out.cpu()
    assert bool(out[..., end::2].isinf().all()) and bool(out[..., end + 1::2].isfinite().all()) and bool(out[..., :end].isfinite().all())


def test_factors_of_far_and_stretched_places():
    """fp64 until the last rounding: 2^-24 of at most 1, and 10^-9 for an angle of 10^6 whose frequency is 10^-15 off."""
    places, dims = (300, 5, 64), (24, 32, 72)
    for origin, step, theta in (((0, 0, 0), (1, 1, 1), 10000.0), ((1e6, 3.5, 0), (1, 0.25, 1.7), 500.0), ((-50, 0, 10), (2, 1, 0.5), 1e6)):
        got = pab.pab_rope_factors(places, dims, origin, step, theta, device=DEV).cpu().double().numpy()
        want = qo.rope_factors(places, dims, origin, step, theta)
        assert got.shape == want.shape and np.all(np.abs(got - want) <= 2.0 ** -24 + 1e-8)


@pytest.mark.parametrize("D,dims", [(72, (24, 24, 24)), (128, (16, 56, 56))])
def test_stretched_places_reach_the_rotation(D, dims):
    places, origin, step = (3, 4, 5), (16, 0, 0.5), (1, 0.5, 0.25)
    q = normal(6, 60, 2, D)
    f = pab.pab_rope_factors(places, dims, origin, step, 5000.0, device=DEV)
    out, _ = pab.pab_qk_norm_rope(q.to(DEV), None, places, dims, f, pab.NORM_NONE)
    check(out, q, places, dims, "none", None, None, 0.0, origin=origin, step=step, theta=5000.0)


def test_many_tokens_in_order():
    """Places of tokens far down the list: every token is its own frame, row and column."""
    places, dims, D = (40, 45, 80), (8, 12, 12), 32
    n = 40 * 45 * 80
    q = torch.zeros(n, 1, D)
    q[:, :, 0::2] = 1.0                                       # each pair (1, 0) turns into its (cos, sin)
    f = pab.pab_rope_factors(places, dims, device=DEV)
    out, _ = pab.pab_qk_norm_rope(q.to(DEV), None, places, dims, f, pab.NORM_NONE)
    t = torch.arange(n)
    table = f.cpu()
    parts, first = [], 0
    for place, m, d in zip((t // 3600, t // 80 % 45, t % 80), places, dims):
        parts.append(table[first:first + m * (d // 2)].view(m, d)[place])
        first += m * (d // 2)
    assert torch.equal(out.cpu()[:, 0], torch.cat(parts, 1))


@pytest.mark.parametrize("dtype,groups", [(torch.bfloat16, 1536), (torch.float32, 8192)])
@pytest.mark.parametrize("D,dims", [(32, (8, 12, 12)), (64, (16, 24, 24)), (72, (24, 24, 24)), (96, (32, 32, 20)), (128, (16, 56, 56))])
def test_wavefronts_take_several_groups_of_rows(D, dims, dtype, groups):
    """More (token, head) rows than `groups` workgroups of four wavefronts hold at 64 / (D / 8) rows each, up to which every wavefront has one group: each takes
    two, some a third, the last one part of a group.  Every element against the definition in fp64 (vectorised, on the device), with check's tolerance."""
    places, batch, Hq, Hk = (3, 7, 11), 2, 4, 3
    at_once = groups * 4 * (64 // (D // 8))
    T = -(-(2 * at_once + 4 * 64) // (batch * 77 * Hq))
    places = (T, 7, 11)
    n = batch * T * 77
    assert 2 * at_once < n * Hq < 3 * at_once
    gen = torch.Generator(device=DEV).manual_seed(D)
    g = [t.to(DEV) for t in weights(D, dtype, 70)]
    f = pab.pab_rope_factors(places, dims, device=DEV)
    q, k = ((torch.randn(n, h, D, generator=gen, device=DEV) * 2 + 0.5).to(dtype) for h in (Hq, Hk))
    got = pab.pab_qk_norm_rope(q, k, places, dims, f, pab.NORM_LAYER, *g, eps=1e-6)
    table = torch.from_numpy(qo.rope_factors(places, dims)).to(DEV)
    token = torch.arange(n, device=DEV) % (T * 77)
    columns, first = [], 0
    for place, m, d in zip((token // 77, token // 11 % 7, token % 11), places, dims):
        columns.append(table[first:first + m * (d // 2)].view(m, d // 2, 2)[place])
        first += m * (d // 2)
    turn = torch.cat(columns, 1)[:, None]
    r = 2 * turn.shape[2]
    for out, x, gamma, beta in ((got[0], q, *g[:2]), (got[1], k, *g[2:])):
        v = x.double()
        mean = v.mean(-1, keepdim=True)
        sigma = torch.sqrt(v.var(-1, unbiased=False, keepdim=True) + 1e-6)
        v = (v - mean) / sigma * gamma.double() + beta.double()
        big = (v.abs().amax(-1, keepdim=True) + mean.abs() / sigma) * (1 + gamma.double().abs().max())
        a, b = v[..., 0:r:2], v[..., 1:r:2]
        want = torch.cat([torch.stack([a * turn[..., 0] - b * turn[..., 1], a * turn[..., 1] + b * turn[..., 0]], -1).flatten(-2), v[..., r:]], -1)
        over = (out.double() - want).abs() - HALF[dtype] * want.abs() - (D + 16) * 2.0 ** -23 * big
        assert bool((over <= 0).all()), float(over.max())


def test_streams_and_graphs():
    places, dims = (4, 5, 6), (24, 24, 24)
    q, k = normal(7, 120, 16, 72).bfloat16().to(DEV), normal(8, 120, 16, 72).bfloat16().to(DEV)
    f = pab.pab_rope_factors(places, dims, device=DEV)
    g = [t.to(DEV) for t in weights(72, torch.bfloat16, 1)]
    a, b = torch.empty_like(q), torch.empty_like(k)
    run = lambda **kw: pab.pab_qk_norm_rope(q, k, places, dims, f, pab.NORM_LAYER, *g, **kw)   # noqa: E731
    run(q_out=a, k_out=b)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    c, d = run(stream=side)
    side.synchronize()
    assert torch.equal(a, c) and torch.equal(b, d)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(q_out=a, k_out=b)
    for seed in range(3):
        q.copy_(normal(20 + seed, 120, 16, 72).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        c, d = run()
        assert torch.equal(a, c) and torch.equal(b, d)


def test_whole_clip_attention_behind_it():
    """The operators together as a model that attends over the whole clip in 8 bits uses them: 8-bit projections, norm and rotation, attention
    into an 8-bit slot, output projection from the slot, gated residual.  Against the same chain in fp64 with the GPU's own roundings to
    8 bits left out: every 8-bit rounding is worth at most 2^-4 of a value, of independent signs, so the norm of the relative error stays
    below 2^-4 a stage (four roundings on the way to the output: 2^-2)."""
    places, dims, H, D = (3, 6, 8), (24, 24, 24), 4, 72
    n, C = 144, 288
    x = normal(30, n, C).bfloat16()
    ws = [normal(31 + i, C, C) / C ** 0.5 for i in range(4)]
    gate = normal(40, C).bfloat16()
    g = weights(D, torch.bfloat16, 41)
    w8 = [pab.pab_quantize(w.to(DEV)) for w in ws]
    f = pab.pab_rope_factors(places, dims, device=DEV)
    xd = x.to(DEV)
    a = pab.pab_quantize(xd)
    q, k, v = (pab.pab_linear_quantized(a, w).view(1, n, H, D) for w in w8[:3])
    pab.pab_qk_norm_rope(q, k, places, dims, f, pab.NORM_LAYER, *(t.to(DEV) for t in g), q_out=q, k_out=k)
    cfg = pab.make_config(1, 1, n, 0, H, D, pab.BF16, 4, (2, 0, 0), 0, 3)
    ctx = pab.QuantizedContext(cfg, DEV)
    scratch = torch.empty(n * C * 2, dtype=torch.uint8, device=DEV)
    assert ctx.pab_attention_quantized(0, pab.SPATIAL, 0, q, k, v, scratch)[0] == pab.COMPUTE
    dec, slot = ctx.pab_attention_quantized(0, pab.SPATIAL, 1, None, None, None, None)
    assert dec == pab.REUSE
    y = pab.pab_linear_quantized(slot, w8[3], out=pab.q8_empty(n, C, DEV))
    out = pab.pab_dequantize(y, xd, gate.to(DEV)).cpu().double().numpy()

    xf = x.double().numpy()
    qf, kf, vf = ((xf @ w.double().numpy().T).reshape(n, H, D) for w in ws[:3])
    qf, kf = (qo.qk_norm_rope(t, places, dims, "layer", g[2 * i].double().numpy(), g[2 * i + 1].double().numpy(), 1e-6) for i, t in enumerate((qf, kf)))
    s = np.einsum("qhd,khd->hqk", qf, kf) / np.sqrt(D)
    p = np.exp(s - s.max(-1, keepdims=True))
    o = np.einsum("hqk,khd->qhd", p / p.sum(-1, keepdims=True), vf).reshape(n, C)
    want = gate.double().numpy() * (o @ ws[3].double().numpy().T)
    got = out - xf
    assert np.linalg.norm(got - want) <= 0.25 * np.linalg.norm(want)
