"""Token scores by how many waves share a row: one through several tiles of it (rows of up to 2048
classes, or many rows), four, and a gradient in several stretches of a wave, with ties, masks,
NaN and rising logits. Against the oracle within the bounds derived in test_gpu_token_scores.py;
of many rows a sample.
"""
import numpy as np
import pytest

import oracle
from helpers import quant
from test_gpu_token_scores import U32, _grad, _grad_tol, _logits, _rng, _run, _same, _tol

pytestmark = pytest.mark.gpu


def _check_rows(got, z, dtype, tokens, scale, top, rows):
    q = quant(z[rows], dtype)
    ref = oracle.token_scores(q, tokens[rows], scale, top)
    t = _tol(q, scale, ref)
    finite = lambda v: np.abs(np.nan_to_num(v, posinf=0, neginf=0))  # noqa: E731
    _same(got["logp"][rows], ref["logp"], 2 * t + 8 * U32 * finite(ref["logp"]), "logp")
    _same(got["lse"][rows], ref["lse"], 2 * t, "lse")
    _same(got["entropy"][rows], ref["entropy"], 4 * t * (1 + np.nan_to_num(ref["entropy"])), "entropy")
    if top:
        assert (got["top_ids"][rows] == ref["top_ids"]).all()
        lp = ref["top_logp"]
        _same(got["top_logp"][rows], lp, 2 * t[:, None] + 8 * U32 * finite(lp), "top_logp")


# One wave to a row: exactly one tile, more, the longest such row, many rows; four waves.
SIZES = [(5, 1024), (5, 1500), (5, 2048), (4097, 2500), (4100, 16384), (800, 3000), (769, 20000)]

HOW = ["plain", "ties", "same", "rising", "falling", "masked", "large"]


def _sample(R):
    return np.unique(np.concatenate((np.arange(min(R, 8)), np.arange(0, R, max(1, R // 16)), [R - 1])))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size,how", [(s, h) for s in SIZES for h in HOW if s[0] * s[1] < 1 << 25 or h in ("plain", "falling")])
def test_rows(dtype, size, how):
    R, V = size
    few = min(R, 16)                        # distinct rows, then the same again
    z = np.tile(_logits(_rng(30, V), few, V, how), (-(-R // few), 1))[:R]
    tokens = _rng(31, R, V).integers(0, V, R).astype(np.int32)
    tokens[1], tokens[-1] = -1, V
    for top in (0, 1, 20, 32):
        got, _ = _run(z, dtype, tokens, 0.75, top, pad=top % 2)
        _check_rows(got, z, dtype, tokens, 0.75, top, _sample(R))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(8, 1024), (8, 2048), (4100, 2500), (800, 3000)])
def test_rows_with_nan_and_infinity(dtype, size):
    R, V = size
    z = np.tile(_logits(_rng(32, V), 8, V, "plain"), (-(-R // 8), 1))[:R]
    z[0, V // 2] = np.nan
    z[1, :] = np.nan
    z[2, V - 1] = np.inf
    z[3, :] = np.inf
    z[4, : V // 2] = np.nan
    z[4, V // 2:] = -np.inf
    z[5, 0], z[5, 1] = np.nan, np.inf
    z[6, 3::2] = np.nan                     # more than a list of alternatives holds
    tokens = np.zeros(R, np.int32)
    got, _ = _run(z, dtype, tokens, 1.0, 7)
    _check_rows(got, z, dtype, tokens, 1.0, 7, _sample(R))


@pytest.mark.parametrize("types", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("size", [(5, 1025), (5, 1500), (5, 2048), (5, 2049)])
def test_gradient_in_stretches(types, size):
    dtype, out_dtype = types
    R, V = size
    r = _rng(33, R, V)
    z = _logits(r, R, V, "plain")
    tokens = np.array([0, V - 1, V // 2, -1, 1024], np.int32)
    dlogp, dent = r.standard_normal(R).astype(np.float32), r.standard_normal(R).astype(np.float32)
    _, (zd, tk, lse, ent) = _run(z, dtype, tokens, 0.8, 0, pad=1)
    q, scale = quant(z, dtype), float(np.float32(0.8))
    ref = oracle.token_scores_vjp(q, tokens, scale, dlogp, dent)
    got = _grad(zd, R, V, V + 1, dtype, out_dtype, 0.8, tk, lse, ent, dlogp, dent)
    _same(got, ref, _grad_tol(q, tokens, scale, dlogp, dent, out_dtype, ref), "dlogits")
