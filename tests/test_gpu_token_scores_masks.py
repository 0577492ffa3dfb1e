"""Token scores of rows whose masked classes hold the type's lowest value, or other values so low
that their scaled differences overflow: alone in a thread, in a wave, in a tile, in a whole part
of a row, before and behind the live classes. Scores and gradient against the oracle within
the bounds derived in test_gpu_token_scores.py (a masked class adds no term to any sum).
"""
import numpy as np
import pytest

import oracle
import paper_1711_03016_amd as dl
from helpers import quant
from test_gpu_token_scores import _grad, _grad_tol, _rng, _run, _same, _tol

pytestmark = pytest.mark.gpu

FMAX = float(np.finfo(np.float32).max)
LOWEST = {"f32": -FMAX, "bf16": -(2.0 - 2.0 ** -7) * 2.0 ** 127}
HOW = ["front", "back", "one_left", "one_in_ten", "halves", "threads"]


def _masked(R, V, how, mask, r):
    z = (r.standard_normal((R, V)) * 3).astype(np.float32)
    c = np.arange(V)
    live = {"front": c >= V - max(1, V // 7), "back": c < max(1, V // 7), "halves": c % (V // 2 + 1) < V // 4 + 1,
            "threads": c // 8 % 5 == 3 if V > 32 else c == V - 1}.get(how)
    if live is None:
        live = r.random((R, V)) < (0.1 if how == "one_in_ten" else 0.0)
        live[np.arange(R), r.integers(0, V, R)] = True
    z[~np.broadcast_to(live, (R, V))] = mask
    if R > 2:
        z[2] = mask                         # masked everywhere
    return z


def _stored(z, dtype, mask):
    """What the oracle sees; the mask as the type holds it."""
    q = quant(z, dtype)
    assert np.isfinite(q).all() and (q[z == np.float32(mask)] < 0).all()
    return q


def _check_rows(got, q, tokens, scale, top, rows):
    """Rows against the oracle; a y below float32's range is -infinity."""
    q = np.where(scale * q < -FMAX, -np.inf, q)[rows]
    ref = oracle.token_scores(q, tokens[rows], scale, top)
    t = _tol(q, scale, ref)
    finite = lambda v: np.abs(np.nan_to_num(v, posinf=0, neginf=0))  # noqa: E731
    _same(got["logp"][rows], ref["logp"], 2 * t + 8 * 2.0 ** -24 * finite(ref["logp"]), "logp")
    _same(got["lse"][rows], ref["lse"], 2 * t, "lse")
    _same(got["entropy"][rows], ref["entropy"], 4 * t * (1 + finite(ref["entropy"])), "entropy")
    if top:
        assert (got["top_ids"][rows] == ref["top_ids"]).all()
        lp = ref["top_logp"]
        _same(got["top_logp"][rows], lp, 2 * t[:, None] + 8 * 2.0 ** -24 * finite(lp), "top_logp")


# One wave to a row (less than a tile, several), four, eight, parts and their join.
SIZES = [(5, 7), (6, 100), (5, 1500), (4100, 2500), (800, 3000), (5, 3000), (3, 20000), (4, 40000), (3, 131072)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("scale", [1.0, 0.5, 1.25])
def test_scores_under_masks(dtype, size, scale):
    R, V = size
    rows = np.unique(np.concatenate((np.arange(min(R, 4)), np.arange(0, R, max(1, R // 8)), [R - 1])))
    for i, how in enumerate(HOW if R < 100 else HOW[:2]):
        for mask in (LOWEST[dtype], -3e37, -1e32)[: 3 if R < 100 else 1]:
            z = _masked(R, V, how, mask, _rng(20, R, V, i))
            tokens = np.argmax(z, axis=1).astype(np.int32)
            tokens[::3] = V // 2
            q = _stored(z, dtype, mask)
            for top, use_ws in ((0, True), (min(6, V), True), (min(6, V), False)):
                got, _ = _run(z, dtype, tokens, scale, top, pad=i % 2, use_ws=use_ws)
                _check_rows(got, q, tokens, scale, top, rows)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(5, 100), (4, 1500), (4, 5000), (3, 131072)])
@pytest.mark.parametrize("scale", [1.0, 0.5])
def test_gradient_under_masks(dtype, size, scale):
    R, V = size
    for i, how in enumerate(HOW):
        r = _rng(21, R, V, i)
        z = _masked(R, V, how, LOWEST[dtype], r)
        tokens = np.argmax(z, axis=1).astype(np.int32)
        dlogp, dent = r.standard_normal(R).astype(np.float32), r.standard_normal(R).astype(np.float32)
        _, (zd, tk, lse, ent) = _run(z, dtype, tokens, scale, 0)
        q = _stored(z, dtype, LOWEST[dtype])
        ref = oracle.token_scores_vjp(q, tokens, scale, dlogp, dent)
        got = _grad(zd, R, V, V, dtype, dtype, scale, tk, lse, ent, dlogp, dent)
        _same(got, ref, _grad_tol(q, tokens, scale, dlogp, dent, dtype, ref), "dlogits")
        assert (got[z == np.float32(LOWEST[dtype])] == 0).all()
