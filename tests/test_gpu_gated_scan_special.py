"""Infinite and NaN values in the gated recurrence: what they reach is infinite or NaN, in every
variant alike, and nothing else changes; and strides whose offsets pass 32 bits, forwards and
backwards.

Where the oracle is finite the bounds are those of test_gpu_gated_scan.py for the same inputs with
zeros in the place of the values that are not: nothing finite depends on them.
"""
import numpy as np
import pytest

import oracle
import paper_1711_03016_amd as dl
from helpers import device, quant, to_dev, to_np
from test_gpu_gated_scan import _bounds, _case, _reference, _run

pytestmark = pytest.mark.gpu


def _finite(v):
    return np.where(np.isfinite(v), v, 0.0)


# One thread through all steps, eight waves, chained and in segments (with a workspace).
SIZES = [(16, 4, 40), (40, 4, 40), (200, 2, 72), (600, 2, 40), (1100, 3, 33)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mode", ["free", "coupled"])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("shut", [False, True])
def test_infinite_and_nan_values(dtype, mode, size, shut):
    """Also where the product of the gates since then is below float32's range (`shut`)."""
    T, B, H = size
    z, x, h0, dhs, dhT, _ = _case(T, B, H, dtype, False, False, 11)
    if shut:
        z = (z * 0.1 - 4.0).astype(np.float32)
    h0[0, 0], h0[1, 3] = np.inf, -np.inf
    x[T // 2, 0, 5], x[T // 3, 1, 6], x[0, 0, 7] = np.inf, -np.inf, np.nan
    z[T // 2, 0, 9] = np.nan
    dhs[T // 2, 1, 11], dhs[T - 1, 0, 12], dhT[1, 13] = np.inf, np.nan, -np.inf
    q = [quant(np.nan_to_num(v, nan=0, posinf=0, neginf=0), dtype) for v in (z, x, dhs)]
    for clean, v in zip(q, (z, x, dhs)):
        clean[~np.isfinite(v)] = v[~np.isfinite(v)]
    coupled = mode == "coupled"
    with np.errstate(invalid="ignore", over="ignore"):
        ref = _reference(q[0], q[1], h0, None, coupled, q[2], dhT)
    tol = _bounds(_finite(q[0]), _finite(q[1]), _finite(h0), None, coupled, _finite(q[2]), _finite(dhT), dtype)
    for use_ws in (True, False):
        got = _run(T, B, H, dtype, mode, z, x, h0, None, dhs, dhT, use_ws=use_ws)
        for name, want in ref.items():
            ok = np.isfinite(want)
            assert (np.isfinite(got[name]) == ok).all(), (name, np.argwhere(np.isfinite(got[name]) != ok)[:3])
            assert (np.abs(got[name][ok] - want[ok]) <= tol[name][ok]).all(), name
    assert not np.isfinite(ref["hT"][0, 0]) and not np.isfinite(ref["dz"][T - 1, 0, 0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [9, 40])
def test_strides_beyond_32_bits_backwards(dtype, T):
    """All rows, inputs and gradients, lie in one buffer of more than 2^32 bytes."""
    import torch
    B, H = 2, 24
    ld = ((1 << 32) // (4 if dtype == "f32" else 2) // (T * B - 2)) // 8 * 8 + 8
    z, x, h0, dhs, dhT, _ = _case(T, B, H, dtype, False, False, 12)
    buf = torch.zeros((T * B - 1) * ld + 6 * H, dtype=torch.float32 if dtype == "f32" else torch.bfloat16,
                      device=device())
    rows = buf.as_strided((T * B, 6 * H), (ld, 1))
    cols = [buf[i * H:] for i in range(6)]                  # z, x, dhs, hs, dz, dx
    for i, v in enumerate((z, x, dhs)):
        rows[:, i * H:(i + 1) * H] = to_dev(v.reshape(-1, H), dtype)
    assert (T * B - 1) * ld * buf.element_size() > 1 << 32
    hT, dh0 = torch.empty((B, H), device=device()), torch.empty((B, H), device=device())
    h0d, dTd = to_dev(h0), to_dev(dhT)
    dl.gated_scan_forward(dtype, "coupled", T, B, H, cols[0], ld, cols[1], ld, h0d, None, cols[3], ld, hT)
    dl.gated_scan_backward(dtype, "coupled", T, B, H, cols[0], ld, cols[1], ld, h0d, None, cols[3], ld, cols[2], ld,
                           dTd, cols[4], ld, cols[5], ld, dh0)
    q = [quant(v, dtype) for v in (z, x, dhs)]
    ref = _reference(q[0], q[1], h0, None, True, q[2], dhT)
    tol = _bounds(q[0], q[1], h0, None, True, q[2], dhT, dtype)
    got = {"hT": to_np(hT), "dh0": to_np(dh0)}
    for i, name in ((3, "hs"), (4, "dz"), (5, "dx")):
        got[name] = to_np(rows[:, i * H:(i + 1) * H]).reshape(T, B, H)
    for name in ref:
        assert (np.abs(got[name] - ref[name]) <= tol[name]).all(), name
    # nothing between the rows was written
    assert (rows[:, :3 * H].float().abs().sum() > 0) and (buf[6 * H:ld] == 0).all()
