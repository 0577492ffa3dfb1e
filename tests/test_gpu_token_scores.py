"""Token scores on the GPU (log probabilities, log-sum-exp, entropy, alternatives)
and their gradient, against the oracle.

Tolerances. With y = scale z, each y is off by 3 2^-24 |y| (two factors and the
subtraction of the maximum, in units of log 2), a sum of V exponentials taken as
running sums of at most V / 64 + 64 terms by 2^-24 of itself for each, and by
what its arguments are off. So with Y the largest finite |y| that has any
probability, t = (V / 64 + 64 + 8 Y) 2^-24 bounds the relative error of the sum and the
absolute one of its logarithm; a log probability is off by 2 t + 8 |y| 2^-24, the
entropy by 4 t (1 + H). Probabilities in the gradient are off by the error of their
logarithm, and bf16 stores round by 2^-8. Alternatives are exact: the order is that
of the stored logits.
"""
import numpy as np
import pytest

import oracle
import paper_1711_03016_amd as dl
from helpers import device, quant, to_dev, to_np, torch_dtype

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
ROUND = {"f32": 0.0, "bf16": 2.0 ** -8}


def _rng(*key):
    return np.random.default_rng([707, *key])


def _logits(r, R, V, how):
    z = (r.standard_normal((R, V)) * 3).astype(np.float32)
    if how == "ties":
        z = np.round(z)
    elif how == "same":
        z[:] = 1.25
    elif how == "rising":
        z = np.sort(z, axis=1)
    elif how == "falling":
        z = -np.sort(-z, axis=1)
    elif how == "masked":                   # rows of which few, one and no classes are left
        keep = r.random((R, V)) < 0.1
        z[~keep] = -np.inf
        z[0] = -np.inf
        if R > 1:
            z[1] = -np.inf
            z[1, V // 2] = 0.5
        if R > 2:
            z[2, : V - 1] = np.finfo(np.float32).min if V > 1 else z[2, : V - 1]
    elif how == "large":
        z *= 1000
    elif how == "zeros":
        z = np.where(r.random((R, V)) < 0.5, np.float32(0.0), np.float32(-0.0))
    return z


def _stored(z, dtype, ld):
    import torch
    R, V = z.shape
    t = torch.full((R, ld), float("nan"), dtype=torch_dtype(dtype), device=device())
    t[:, :V] = to_dev(z, dtype)
    return t


def _run(z, dtype, tokens, scale, top, pad=0, use_ws=True, td=None):
    import torch
    R, V = z.shape
    zd = _stored(z, dtype, V + pad) if td is None else td
    tk = None if tokens is None else torch.from_numpy(np.asarray(tokens, np.int32)).to(device())
    logp, lse, ent = (torch.full((R + 4,), 7.0, device=device()) for _ in range(3))
    ids = torch.full((R * top + 4,), 7, dtype=torch.int32, device=device()) if top else None
    tlp = torch.full((R * top + 4,), 7.0, device=device()) if top else None
    ws = None
    if use_ws:
        n = dl.token_logprobs_ws_bytes(R, V, top)
        assert n > 0
        ws = torch.full((n,), 255, dtype=torch.uint8, device=device())
    dl.token_logprobs(dtype, R, V, zd, V + pad, scale, tk, None if tk is None else logp, lse, ent, top,
                      ids, tlp, ws)
    out = {"logp": logp, "lse": lse, "entropy": ent}
    out = {k: to_np(v) for k, v in out.items()}
    for v in out.values():
        assert (v[R:] == 7.0).all()
    out = {k: v[:R] for k, v in out.items()}
    if top:
        assert (ids[R * top:] == 7).all() and (tlp[R * top:] == 7).all()
        out["top_ids"] = ids[:R * top].cpu().numpy().reshape(R, top)
        out["top_logp"] = to_np(tlp[:R * top]).reshape(R, top)
    return out, (zd, tk, lse, ent)


def _tol(z, scale, ref):
    V = z.shape[1]
    y = np.abs(scale * np.where(np.isfinite(z) & (np.abs(z) < 1e30), z, 0.0))
    m = (scale * np.where(np.isnan(z), -np.inf, z)).max(axis=1)
    near = np.abs(np.where(np.isfinite(m), m, 0.0)) + 110   # below that, 2^(y - m) is zero
    Y = np.minimum(y.max(axis=1), near)
    return (V / 64 + 64 + 8 * Y) * U32


def _same(got, ref, tol, what):
    special = ~np.isfinite(ref)
    same = np.where(np.isnan(ref), np.isnan(got), got == ref)
    assert same[special].all(), (what, got[special][:4], ref[special][:4])
    err = np.abs(got[~special] - ref[~special])
    assert (err <= np.broadcast_to(tol, ref.shape)[~special]).all(), (what, err.max())


def _check(got, z, tokens, scale, top):
    ref = oracle.token_scores(z, tokens, scale, top)
    t = _tol(z, scale, ref)
    if tokens is not None:
        _same(got["logp"], ref["logp"], 2 * t + 8 * U32 * np.abs(np.nan_to_num(ref["logp"], posinf=0, neginf=0)), "logp")
    _same(got["lse"], ref["lse"], 2 * t, "lse")
    _same(got["entropy"], ref["entropy"], 4 * t * (1 + np.nan_to_num(ref["entropy"])), "entropy")
    if top:
        assert (got["top_ids"] == ref["top_ids"]).all()
        lp = ref["top_logp"]
        _same(got["top_logp"], lp, 2 * t[:, None] + 8 * U32 * np.abs(np.nan_to_num(lp, posinf=0, neginf=0)), "top_logp")
    return ref


SIZES = [(1, 1), (3, 2), (5, 10), (9, 64), (7, 65), (300, 1000), (130, 257), (4, 2049), (3, 4097),
         (2, 9001), (600, 5003), (1, 32768), (2, 50001), (5, 131072)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("top", [0, 1, 5, 32])
def test_scores(dtype, size, top):
    R, V = size
    top = min(top, V)
    r = _rng(1, R, V)
    z = _logits(r, R, V, "plain")
    tokens = r.integers(0, V, R).astype(np.int32)
    if R > 3:
        tokens[0], tokens[1], tokens[2] = -1, V, -7
    got, _ = _run(z, dtype, tokens, 1.25, top)
    _check(got, quant(z, dtype), tokens, 1.25, top)
    other, _ = _run(z, dtype, tokens, 1.25, top, pad=3, use_ws=False)
    _check(other, quant(z, dtype), tokens, 1.25, top)
    again, _ = _run(z, dtype, tokens, 1.25, top)
    assert all(np.array_equal(again[k], got[k], equal_nan=True) for k in got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["ties", "same", "rising", "falling", "masked", "large", "zeros"])
@pytest.mark.parametrize("size", [(6, 40), (9, 1000), (3, 3000), (3, 20000), (2, 131072), (300, 4100)])
def test_orders_and_masks(dtype, how, size):
    R, V = size
    z = _logits(_rng(2, R, V), R, V, how)
    tokens = _rng(3, R, V).integers(0, V, R).astype(np.int32)
    for top in (1, 20):
        for use_ws in (True, False):
            got, _ = _run(z, dtype, tokens, 0.5, top, pad=1, use_ws=use_ws)
            _check(got, quant(z, dtype), tokens, 0.5, top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [7, 1000, 6000, 70000])
def test_rows_with_nan_and_infinity(dtype, V):
    z = _logits(_rng(4, V), 7, V, "plain")
    z[0, V // 2] = np.nan
    z[1, :] = np.nan
    z[2, V - 1] = np.inf
    z[3, :] = np.inf
    z[4, : V // 2] = np.nan
    z[4, V // 2:] = -np.inf
    z[5, 0] = np.nan
    z[5, 1] = np.inf
    tokens = np.zeros(7, np.int32)
    for use_ws in (True, False):
        got, _ = _run(z, dtype, tokens, 1.0, 7, use_ws=use_ws)
        _check(got, quant(z, dtype), tokens, 1.0, 7)


def _grad(zd, R, V, ld, dtype, out_dtype, scale, tk, lse, ent, dlogp, dent, pad=2, in_place=False):
    import torch
    if in_place:
        out, ldo = zd, ld
    else:
        ldo = V + pad
        out = torch.full((R, ldo), 7.0, dtype=torch_dtype(out_dtype), device=device())
    dev = lambda v: None if v is None else to_dev(v)  # noqa: E731
    dl.token_logprobs_backward(dtype, out_dtype, R, V, zd, ld, scale, tk, lse, ent, dev(dlogp),
                               dev(dent), out, ldo)
    got = to_np(out)
    assert in_place or (got[:, V:] == 7.0).all()
    return got[:, :V]


def _grad_tol(z, tokens, scale, dlogp, dent, out_dtype, ref):
    s = oracle.token_scores(z, None, scale, 0)
    t = _tol(z, scale, s)[:, None]
    with np.errstate(invalid="ignore"):
        lp = np.where(np.isfinite(s["lse"])[:, None], scale * z - s["lse"][:, None], -np.inf)
    p = np.exp(lp)
    lp = np.where(p > 0, lp, 0.0)
    el = 4 * t + 16 * U32 * np.abs(lp)                  # of log p, and so of p relative
    gl = 0.0 if dlogp is None else np.abs(dlogp)[:, None]
    ge = 0.0 if dent is None else np.abs(dent)[:, None]
    H = s["entropy"][:, None]
    tol = gl * (p * el + 4 * U32) + ge * p * (el * (np.abs(lp + H) + 1) + 4 * t * (1 + H) + 8 * U32 * np.abs(lp + H))
    return scale * tol * 1.01 + (ROUND[out_dtype] + 4 * U32) * np.abs(np.nan_to_num(ref)) + 1e-37


@pytest.mark.parametrize("types", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("size", [(1, 1), (3, 2), (5, 10), (300, 1000), (7, 65), (4, 2049), (2, 50001), (33, 4096)])
@pytest.mark.parametrize("which", ["both", "logp", "entropy"])
def test_gradient(types, size, which):
    dtype, out_dtype = types
    R, V = size
    r = _rng(5, R, V)
    z = _logits(r, R, V, "plain")
    tokens = r.integers(0, V, R).astype(np.int32)
    if R > 3:
        tokens[0], tokens[1] = -1, V
    dlogp = None if which == "entropy" else r.standard_normal(R).astype(np.float32)
    dent = None if which == "logp" else r.standard_normal(R).astype(np.float32)
    _, (zd, tk, lse, ent) = _run(z, dtype, tokens, 0.8, 0, pad=1)
    q = quant(z, dtype)
    scale = float(np.float32(0.8))
    ref = oracle.token_scores_vjp(q, tokens, scale, dlogp, dent)
    tol = _grad_tol(q, tokens, scale, dlogp, dent, out_dtype, ref)
    got = _grad(zd, R, V, V + 1, dtype, out_dtype, 0.8, tk, lse, ent, dlogp, dent)
    _same(got, ref, tol, "dlogits")
    if dtype == out_dtype:
        there = _grad(zd, R, V, V + 1, dtype, out_dtype, 0.8, tk, lse, ent, dlogp, dent, in_place=True)
        assert np.array_equal(there, got, equal_nan=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(5, 100), (4, 5000)])
def test_gradient_of_masked_rows(dtype, size):
    R, V = size
    r = _rng(6, R, V)
    z = _logits(r, R, V, "masked")
    tokens = np.array([int(np.argmax(row)) for row in z], np.int32)
    dlogp, dent = r.standard_normal(R).astype(np.float32), r.standard_normal(R).astype(np.float32)
    _, (zd, tk, lse, ent) = _run(z, dtype, tokens, 1.0, 0)
    q = quant(z, dtype)
    ref = oracle.token_scores_vjp(q, tokens, 1.0, dlogp, dent)
    got = _grad(zd, R, V, V, dtype, dtype, 1.0, tk, lse, ent, dlogp, dent)
    assert (got[0] == 0).all()                          # every class masked
    _same(got, ref, _grad_tol(q, tokens, 1.0, dlogp, dent, dtype, ref), "dlogits")


def test_cross_entropy_is_the_mean_of_minus_logp():
    """The same loss and adjoint as the softmax cross-entropy call on the same logits."""
    import torch
    R, V = 200, 333
    r = _rng(8)
    z = _logits(r, R, V, "plain")
    tokens = r.integers(0, V, R).astype(np.int32)
    got, (zd, tk, lse, ent) = _run(z, "f32", tokens, 1.0, 0)
    d = torch.empty((R, V), device=device())
    loss = torch.empty(1, device=device())
    ws = torch.empty(dl.softmax_xent_ws_bytes(R), dtype=torch.uint8, device=device())
    dl.softmax_xent("f32", R, V, zd, tk, 1.0 / R, d, loss, ws)
    t = (V / 64 + 64 + 8 * np.abs(z).max()) * U32
    assert abs(loss.item() + got["logp"].mean()) <= 8 * t * abs(loss.item()) + 8 * t
    g = _grad(zd, R, V, V, "f32", "f32", 1.0, tk, lse, ent, np.full(R, -1.0 / R, np.float32), None)
    assert np.abs(g - to_np(d)).max() <= 8 * t / R


@pytest.mark.parametrize("types", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("V", [5, 1001, 9000])
@pytest.mark.parametrize("entropy", [False, True])
def test_gradient_of_padding_is_zero(types, V, entropy):
    """Rows of padding hold anything; with an adjoint of the entropy they are not padding."""
    dtype, out = types
    R = 6
    r = _rng(9, V)
    z = _logits(r, R, V, "plain")
    tokens = np.array([0, -1, V - 1, -1, -1, 2], np.int32)
    z[1], z[3, 0], z[4] = np.nan, np.inf, 1e30
    dlogp = r.standard_normal(R).astype(np.float32)
    dent = np.zeros(R, np.float32) if entropy else None
    if entropy:
        dent[3], dent[5] = 0.5, -2.0
    _, (zd, tk, lse, ent) = _run(z, dtype, tokens, 1.0, 0)
    got = _grad(zd, R, V, V, dtype, out, 1.0, tk, lse, ent, dlogp, dent)
    assert (got[[1, 4]] == 0).all()
    assert np.isnan(got[3]).all() if entropy else (got[3] == 0).all()
    keep = [0, 2, 5]
    q = quant(z, dtype)[keep]
    sub = lambda v: None if v is None else v[keep]  # noqa: E731
    ref = oracle.token_scores_vjp(q, tokens[keep], 1.0, dlogp[keep], sub(dent))
    _same(got[keep], ref, _grad_tol(q, tokens[keep], 1.0, dlogp[keep], sub(dent), out, ref), "dlogits")


@pytest.mark.parametrize("top", [0, 5])
def test_offsets_beyond_32_bits(top):
    """More than 2^31 logits: the last rows' scores and gradient as those of a call of them alone."""
    import torch
    R, V = 53_000, 41_000
    assert R * V > 1 << 31
    g = torch.Generator(device=device()).manual_seed(11)
    z = torch.zeros((R, V), dtype=torch.bfloat16, device=device())
    z[-8:] = torch.randn((8, V), generator=g, device=device()).to(torch.bfloat16)
    tokens = torch.arange(R, dtype=torch.int32, device=device()) % V
    dlogp = torch.randn(R, generator=g, device=device())

    def scores(z, tokens, dlogp, out):
        n = z.shape[0]
        o = [torch.empty(n, device=device()) for _ in range(3)]
        ids = torch.empty((n, top), dtype=torch.int32, device=device()) if top else None
        tlp = torch.empty((n, top), device=device()) if top else None
        dl.token_logprobs("bf16", n, V, z, V, 1.0, tokens, *o, top, ids, tlp)
        dl.token_logprobs_backward("bf16", "bf16", n, V, z, V, 1.0, tokens, o[1], o[2], dlogp, None, out, V)
        return o + ([ids, tlp] if top else []) + [out]

    few = z[-8:].clone()
    want = scores(few, tokens[-8:].clone(), dlogp[-8:].clone(), torch.empty_like(few))
    got = scores(z, tokens, dlogp, z)                       # in place
    t = (V / 64 + 64 + 8 * 6) * U32                         # |y| of a normal of these rows below 6
    for a, b in zip(got[:3], want[:3]):
        assert (a[-8:] - b).abs().max() <= 4 * t * (1 + np.log(V))
        assert a.isfinite().all()
    assert (got[1][:-8] - np.log(V)).abs().max() <= 4 * t
    if top:
        assert torch.equal(got[3][-8:], want[3])
        assert (got[3][0].cpu() == torch.arange(top)).all()
    d, ref = got[-1][-8:].float(), want[-1].float()
    assert ((d - ref).abs() <= 2 * (2.0 ** -8 + 8 * t) * ref.abs() + 1e-37).all()
