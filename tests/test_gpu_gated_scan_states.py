"""The states that the gradient of the gated recurrence works with are float32 whatever the
storage type: dz against the oracle where the state follows the input, so that h - x is
far smaller than either.

Tolerances, entry by entry, with the errors k of a gate and e of a state that the
recurrence's other tests derive (k = (|z| + 16) 2^-23, e_t = a e_{t-1} + 2 k (a A_{t-1} +
|u_t|), A the state of absolute terms) and the adjoint's alike (L of absolute terms, f its
error): dz = a c lam D with D = h - x (coupled) or h is a product of four factors, D off by e
and by its own rounding, so it is off by a c (f (|D| + e) + L e + 6 k L (|D| + e)), and what is
stored by at most half a step (bf16: 2^-8 relative). Nothing in it grows with the sizes of h and
x beyond e.
"""
import numpy as np
import pytest

import oracle
import paper_1711_03016_amd as dl
from helpers import device, quant, to_dev, to_np, torch_dtype

pytestmark = pytest.mark.gpu

ROUND = {"f32": 0.0, "bf16": 2.0 ** -8}
TINY = 1e-35


def _case(T, B, H, how, seed):
    r = np.random.default_rng([616, T, B, H, seed])
    z = (r.standard_normal((T, B, H)) * 0.5 + 1.0).astype(np.float32)
    phase = r.uniform(0, 6.28, (1, B, H))
    x = 2.0 + np.sin(phase + 0.002 * np.arange(T)[:, None, None])
    if how == "steps":                      # the input stays, then changes: the state catches up
        x = np.where(np.arange(T)[:, None, None] % 40 < 25, x[:1], -x[:1])
    x = x.astype(np.float32)
    h0 = (quant(x[0], "bf16") * (1 + 1e-3 * r.standard_normal((B, H)))).astype(np.float32)
    dhs = (r.standard_normal((T, B, H)) * 0.3).astype(np.float32)
    dhT = r.standard_normal((B, H)).astype(np.float32)
    return z, x, h0, dhs, dhT


def _bounds(z, x, h0, lens, coupled, dhs, dhT, dtype, ref):
    """Tolerances of dz, dx and dh0 (see above)."""
    T, B, H = z.shape
    n = np.full(B, T) if lens is None else np.clip(lens.astype(np.int64), 0, T)
    live = (np.arange(T)[:, None] < n)[..., None]
    zz, xx = np.where(live, z, 0.0), np.where(live, x, 0.0)
    a, c = oracle.sigmoid(zz), oracle.sigmoid(-zz)
    u = np.abs(c * xx if coupled else xx)
    k = (np.abs(zz) + 16) * 2.0 ** -23
    h, _ = oracle.gated_scan(z, x, h0, lens, coupled)
    A, e = np.zeros((T + 1, B, H)), np.zeros((T + 1, B, H))
    A[0] = np.abs(h0)
    for t in range(T):
        A[t + 1] = np.where(live[t], a[t] * A[t] + u[t], A[t])
        e[t + 1] = np.where(live[t], a[t] * e[t] + 2 * k[t] * (a[t] * A[t] + u[t]), e[t])
    q = ROUND[dtype]
    L, f = np.abs(dhT).astype(np.float64), np.zeros((B, H))
    tol = {"dz": np.zeros((T, B, H)), "dx": np.zeros((T, B, H))}
    for t in range(T - 1, -1, -1):
        on = live[t]
        lam = L + np.where(on, np.abs(dhs[t]), 0.0)
        fl = f + 2.0 ** -23 * lam
        D = np.abs(h[t] - xx[t] if coupled else h[t]) + e[t]
        g = c[t] if coupled else 1.0
        tol["dz"][t] = np.where(on, a[t] * c[t] * (fl * D + lam * e[t] + 6 * k[t] * lam * D), 0.0)
        tol["dx"][t] = np.where(on, g * (fl + 2 * k[t] * lam), 0.0)
        f = np.where(on, a[t] * (fl + 2 * k[t] * lam), f)
        L = np.where(on, a[t] * lam, L)
    for name in tol:
        tol[name] = tol[name] * (1 + q) + q * np.abs(ref[name]) + TINY
    return tol | {"dh0": f + TINY}


def _gradient(T, B, H, dtype, mode, z, x, h0, lens, dhs, dhT, halves, use_ws, pad=0):
    import torch
    new = lambda *s, t=torch_dtype(dtype): torch.full(s, float("nan"), dtype=t, device=device())  # noqa: E731
    if halves:                              # inputs and gradients are the halves of one product
        both, grads = torch.cat((to_dev(z, dtype), to_dev(x, dtype)), dim=2).contiguous(), new(T, B, 2 * H)
        zd, xd, dz, dx, ld = both[..., :H], both[..., H:], grads[..., :H], grads[..., H:], 2 * H
    else:
        ld = H + pad
        zd, xd, dz, dx = (new(T, B, ld) for _ in range(4))
        zd[..., :H], xd[..., :H] = to_dev(z, dtype), to_dev(x, dtype)
    hs, hT, dh0 = new(T, B, H), new(B, H, t=torch.float32), new(B, H, t=torch.float32)
    n = dl.gated_scan_ws_bytes(dtype, T, B, H)
    ws = torch.full((n,), 255, dtype=torch.uint8, device=device()) if use_ws else None
    ln = None if lens is None else torch.from_numpy(lens).to(device())
    h0d, dd, dTd = to_dev(h0), to_dev(dhs, dtype), to_dev(dhT)
    dl.gated_scan_forward(dtype, mode, T, B, H, zd, ld, xd, ld, h0d, ln, hs, H, hT, ws)
    if use_ws:
        ws.fill_(127)
    dl.gated_scan_backward(dtype, mode, T, B, H, zd, ld, xd, ld, h0d, ln, hs, H, dd, H, dTd, dz, ld, dx, ld,
                           dh0, ws)
    if pad:
        assert dz[..., H:].isnan().all() and dx[..., H:].isnan().all()
    return {"dz": dz[..., :H], "dx": dx[..., :H], "dh0": dh0}


def _compare(got, z, x, h0, lens, dhs, dhT, dtype, mode, keep):
    """The batch entries `keep` against the oracle."""
    q = [quant(v, dtype)[:, keep] for v in (z, x, dhs)]
    ln = None if lens is None else lens[keep]
    args = (q[0], q[1], h0[keep], ln, mode == "coupled", q[2], dhT[keep])
    dz, dx, dh0 = oracle.gated_scan_vjp(*args)
    ref = {"dz": dz, "dx": dx, "dh0": dh0}
    tol = _bounds(*args, dtype, ref)
    for name, want in ref.items():
        t = got[name][:, keep] if want.ndim == 3 else got[name][keep]
        err = np.abs(to_np(t) - want)
        assert (err <= tol[name]).all(), (name, np.nanmax(err / tol[name]), np.isnan(err).sum())


# About the eight steps of a thread and the 64 of a workgroup, a thread through many steps, one
# workgroup through many rounds, segments.
SIZES = [(8, 2, 64), (9, 5, 63), (16, 2, 130), (17, 3, 64), (32, 64, 1024), (33, 40, 96), (64, 300, 64),
         (65, 2, 24), (129, 1, 40), (300, 2, 257), (383, 2, 72), (384, 2, 72), (1000, 1, 96), (1025, 3, 33),
         (2100, 3, 40)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mode", ["free", "coupled"])
@pytest.mark.parametrize("size", SIZES)
def test_gradient_where_the_state_follows_the_input(dtype, mode, size):
    T, B, H = size
    keep = np.arange(0, B, max(1, B // 8))
    for how, use_ws, pad in (("smooth", True, 0), ("steps", True, 3), ("smooth", False, 5)):
        case = _case(T, B, H, how, 1)
        z, x, h0, dhs, dhT = case
        got = _gradient(T, B, H, dtype, mode, z, x, h0, None, dhs, dhT, False, use_ws, pad)
        _compare(got, z, x, h0, None, dhs, dhT, dtype, mode, keep)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(13, 6, 64), (40, 4100, 64), (130, 5, 40), (300, 200, 64), (700, 9, 72),
                                  (400, 200, 64), (520, 257, 64)])
def test_padded_gradient_where_the_state_follows_the_input(dtype, size):
    """Lengths of zero, one, about a round and all; what dead steps hold is not used. A thread
    through many rounds, and a gradient that is cut only because sequences have lengths."""
    T, B, H = size
    z, x, h0, dhs, dhT = _case(T, B, H, "smooth", 2)
    lens = np.random.default_rng([617, T]).integers(0, T + 1, B).astype(np.int32)
    lens[:6] = (0, 1, T, T + 9, min(T, 8), -2) if B > 5 else (0, 1, T, T + 9, min(T, 8))
    keep = np.unique(np.concatenate((np.arange(5), np.arange(0, B, max(1, B // 8)), [B - 1])))
    dead = np.arange(T)[:, None] >= np.clip(lens, 0, T)
    good = [v.copy() for v in (z, x, dhs)]
    for v, bad in ((z, np.nan), (x, np.inf), (dhs, -np.inf)):
        v[dead] = bad
    for use_ws, halves in ((True, False), (False, True)):
        got = _gradient(T, B, H, dtype, "coupled", z, x, h0, lens, dhs, dhT, halves, use_ws)
        _compare(got, good[0], good[1], h0, lens, good[2], dhT, dtype, "coupled", keep)
        import torch
        off = torch.from_numpy(dead).to(device())
        assert (got["dz"][off] == 0).all() and (got["dx"][off] == 0).all()


def test_steps_of_a_wide_batch():
    """A thread through many steps of its own without lengths: 72 steps of 4097 x 64 states."""
    T, B, H = 72, 4097, 64
    z, x, h0, dhs, dhT = _case(T, B, H, "smooth", 3)
    keep = np.array([0, 1, 2, 2048, 4095, 4096])
    for dtype in ("f32", "bf16"):
        got = _gradient(T, B, H, dtype, "coupled", z, x, h0, None, dhs, dhT, False, True)
        _compare(got, z, x, h0, None, dhs, dhT, dtype, "coupled", keep)
