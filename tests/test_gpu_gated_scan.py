"""The gated linear recurrence on the GPU, forward and gradient, against the oracle.

Tolerances, entry by entry. A gate computed in float32 from its preactivation z is
off by at most k = (|z| + 16) 2^-23 of itself (the exponent's argument is rounded,
|z| 2^-24 relative to the exponential; the exponential, sum and quotient take a few
units in the last place). Each step multiplies and adds once, so with absolute
values in the place of all terms (A_t = a A_{t-1} + |u_t|) the error of a state
obeys e_t = a e_{t-1} + 2 k (a A_{t-1} + |u_t|), in whatever order the steps' maps
are joined. The adjoints obey the same recurrence backwards. Storage in bf16 rounds
by 2^-8 relative; the states that the gradient starts from have been rounded so.
"""
import numpy as np
import pytest

import oracle
import paper_1711_03016_amd as dl
from helpers import device, quant, to_dev, to_np, torch_dtype

pytestmark = pytest.mark.gpu

ROUND = {"f32": 0.0, "bf16": 2.0 ** -8}
TINY = 1e-35      # results below the normal range of float32 may be flushed


def _rng(*key):
    return np.random.default_rng([606, *key])


# (T, B, H): one step, one column, lengths about the steps that a thread, a group of
# threads and a workgroup take, few columns with many steps, many columns with few.
SIZES = [(1, 1, 1), (1, 64, 1024), (2, 3, 5), (3, 1, 2048), (8, 2, 64), (7, 2, 130), (9, 5, 63),
         (33, 40, 96), (64, 300, 64), (128, 4, 64), (129, 1, 40), (257, 2, 100), (300, 2, 257),
         (1000, 1, 96), (1025, 3, 33), (5000, 1, 17)]


def _case(T, B, H, dtype, ragged, halves, seed):
    r = _rng(T, B, H, seed)
    z = (r.standard_normal((T, B, H)) * 1.5 + 1.5).astype(np.float32)
    x = r.standard_normal((T, B, H)).astype(np.float32)
    h0 = r.standard_normal((B, H)).astype(np.float32)
    dhs = (r.standard_normal((T, B, H)) * 0.3).astype(np.float32)
    dhT = r.standard_normal((B, H)).astype(np.float32)
    lens = None
    if ragged:
        lens = r.integers(0, T + 1, B).astype(np.int32)
        lens[0] = (0, T, T + 7, -3)[(T + B + H) % 4]
    return z, x, h0, dhs, dhT, lens


def _bounds(z, x, h0, lens, coupled, dhs, dhT, dtype):
    """Tolerances of hs, hT, dz, dx, dh0 (see above) in float64."""
    T, B, H = z.shape
    n = np.full(B, T) if lens is None else np.clip(lens.astype(np.int64), 0, T)
    live = (np.arange(T)[:, None] < n)[..., None]
    zz, xx = np.where(live, z, 0.0), np.where(live, x, 0.0)
    a, c = oracle.sigmoid(zz), oracle.sigmoid(-zz)
    u = np.abs(c * xx if coupled else xx)
    k = (np.abs(zz) + 16) * 2.0 ** -23
    A, e = np.zeros((T + 1, B, H)), np.zeros((T + 1, B, H))
    A[0] = 0.0 if h0 is None else np.abs(h0)
    for t in range(T):
        on = live[t]
        A[t + 1] = np.where(on, a[t] * A[t] + u[t], A[t])
        e[t + 1] = np.where(on, a[t] * e[t] + 2 * k[t] * (a[t] * A[t] + u[t]), e[t])
    q = ROUND[dtype]
    out = {"hs": np.where(live, e[1:] + q * (A[1:] + e[1:]), 0.0) + TINY, "hT": e[T] + TINY}
    L = np.zeros((B, H)) if dhT is None else np.abs(dhT).astype(np.float64)
    f = np.zeros((B, H))
    dz, dx = np.zeros((T, B, H)), np.zeros((T, B, H))
    for t in range(T - 1, -1, -1):
        on = live[t]
        lam = L + (0.0 if dhs is None else np.where(on, np.abs(dhs[t]), 0.0))
        fl = f + 2.0 ** -23 * lam
        eh = e[t] + q * A[t]                                # the state before, rounded when stored
        big = A[t] + (np.abs(xx[t]) if coupled else 0.0)
        ac = a[t] * c[t]
        dz[t] = np.where(on, ac * (fl * big + lam * eh + 6 * k[t] * lam * big) + q * ac * lam * big, 0.0)
        g = c[t] if coupled else 1.0
        dx[t] = np.where(on, g * (fl + 2 * k[t] * lam) + q * g * lam, 0.0)
        f = np.where(on, a[t] * (fl + 2 * k[t] * lam), f)
        L = np.where(on, a[t] * lam, L)
    out |= {"dz": dz * (1 + q) + TINY, "dx": dx * (1 + q) + TINY, "dh0": f + TINY}
    return out


def _strided(a, dtype, ld, fill):
    """`a` [T, B, H] on the device in rows of stride ld, `fill` between."""
    import torch
    T, B, H = a.shape
    t = torch.full((T, B, ld), fill, dtype=torch_dtype(dtype), device=device())
    t[..., :H] = to_dev(a, dtype)
    return t


def _run(T, B, H, dtype, mode, z, x, h0, lens, dhs, dhT, pad=0, halves=False, use_ws=True):
    """All outputs of a forward and a backward call as float64, guards checked."""
    import torch
    ld = H + pad
    dev = lambda v: None if v is None else to_dev(v)  # noqa: E731
    if halves:
        both = torch.cat((to_dev(z, dtype), to_dev(x, dtype)), dim=2).contiguous()
        zd, xd, ldi = both[..., :H], both[..., H:], 2 * H
    else:
        zd, xd, ldi = _strided(z, dtype, ld, float("nan")), _strided(x, dtype, ld, float("nan")), ld
    nan = torch.full((T, B, H), float("nan"))
    hs, dz, dx = (_strided(nan.numpy(), dtype, ld, 7.0) for _ in range(3))
    hT, dh0 = torch.full((B, H), float("nan"), device=device()), torch.full((B, H), float("nan"), device=device())
    n = dl.gated_scan_ws_bytes(dtype, T, B, H)
    assert n > 0
    ws = torch.full((n,), 255, dtype=torch.uint8, device=device()) if use_ws else None
    ln = None if lens is None else torch.from_numpy(lens).to(device())
    dl.gated_scan_forward(dtype, mode, T, B, H, zd, ldi, xd, ldi, dev(h0), ln, hs, ld, hT, ws)
    if use_ws:
        ws.fill_(127)
    dd = None if dhs is None else _strided(dhs, dtype, ld, float("nan"))
    dl.gated_scan_backward(dtype, mode, T, B, H, zd, ldi, xd, ldi, dev(h0), ln, hs, ld, dd, ld,
                           dev(dhT), dz, ld, dx, ld, dh0, ws)
    out = {"hT": to_np(hT), "dh0": to_np(dh0)}
    for name, t in (("hs", hs), ("dz", dz), ("dx", dx)):
        v = to_np(t)
        assert (v[..., H:] == 7.0).all(), name
        out[name] = v[..., :H]
    return out


def _reference(z, x, h0, lens, coupled, dhs, dhT):
    h, hs = oracle.gated_scan(z, x, h0, lens, coupled)
    dz, dx, dh0 = oracle.gated_scan_vjp(z, x, h0, lens, coupled, dhs, dhT)
    return {"hs": hs, "hT": h[-1], "dz": dz, "dx": dx, "dh0": dh0}


def _compare(got, ref, tol):
    for name in ref:
        err = np.abs(got[name] - ref[name])
        worst = np.nanmax(err / tol[name])
        assert (err <= tol[name]).all(), (name, worst, np.isnan(got[name]).sum())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mode", ["free", "coupled"])
@pytest.mark.parametrize("size", SIZES)
def test_scan(dtype, mode, size):
    T, B, H = size
    z, x, h0, dhs, dhT, lens = _case(T, B, H, dtype, False, False, 1)
    q = [quant(v, dtype) for v in (z, x, dhs)]
    ref = _reference(q[0], q[1], h0, None, mode == "coupled", q[2], dhT)
    tol = _bounds(q[0], q[1], h0, None, mode == "coupled", q[2], dhT, dtype)
    got = _run(T, B, H, dtype, mode, z, x, h0, None, dhs, dhT)
    _compare(got, ref, tol)
    # without a workspace, in rows of another stride
    _compare(_run(T, B, H, dtype, mode, z, x, h0, None, dhs, dhT, pad=3, use_ws=False), ref, tol)
    # again: the same bits
    again = _run(T, B, H, dtype, mode, z, x, h0, None, dhs, dhT)
    assert all((again[k] == got[k]).all() for k in got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mode", ["free", "coupled"])
@pytest.mark.parametrize("size", [s for s in SIZES if s[1] > 1] + [(1, 5, 8), (500, 6, 130), (2100, 3, 40)])
def test_padded_batch(dtype, mode, size):
    """Lengths of zero, one, all and beyond; what padded steps hold is not used."""
    T, B, H = size
    z, x, h0, dhs, dhT, lens = _case(T, B, H, dtype, True, False, 2)
    if B > 4:
        lens[1], lens[2], lens[3], lens[4] = 0, 1, T, T + 1000
    dead = np.arange(T)[:, None] >= np.clip(lens, 0, T)
    q = [quant(v, dtype) for v in (z, x, dhs)]
    ref = _reference(q[0], q[1], h0, lens, mode == "coupled", q[2], dhT)
    tol = _bounds(q[0], q[1], h0, lens, mode == "coupled", q[2], dhT, dtype)
    for k, v in enumerate((z, x, dhs)):
        v[dead] = (np.nan, np.inf, -np.inf)[k]
    got = _run(T, B, H, dtype, mode, z, x, h0, lens, dhs, dhT, pad=5)
    _compare(got, ref, tol)
    for name in ("hs", "dz", "dx"):
        assert (got[name][dead] == 0).all(), name
    if H % 8 == 0:
        _compare(_run(T, B, H, dtype, mode, z, x, h0, lens, dhs, dhT, halves=True), ref, tol)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(5, 2, 24), (700, 2, 40), (260, 9, 33)])
@pytest.mark.parametrize("which", ["no_h0", "dhs_only", "dhT_only"])
def test_optional_arguments(dtype, size, which):
    T, B, H = size
    z, x, h0, dhs, dhT, _ = _case(T, B, H, dtype, False, False, 3)
    h0 = None if which == "no_h0" else h0
    dhT = None if which == "dhs_only" else dhT
    dhs = None if which == "dhT_only" else dhs
    qz, qx, qd = quant(z, dtype), quant(x, dtype), None if dhs is None else quant(dhs, dtype)
    ref = _reference(qz, qx, h0, None, True, qd, dhT)
    tol = _bounds(qz, qx, h0, None, True, qd, dhT, dtype)
    _compare(_run(T, B, H, dtype, "coupled", z, x, h0, None, dhs, dhT), ref, tol)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mode", ["free", "coupled"])
@pytest.mark.parametrize("size,ragged", [((40000, 1, 70), False), ((20011, 3, 64), True), ((1024, 190, 64), False)])
def test_long_sequences(dtype, mode, size, ragged):
    """More blocks of time than a workgroup looks at once, and the same bits every time."""
    T, B, H = size
    z, x, h0, dhs, dhT, lens = _case(T, B, H, dtype, ragged, False, 9)
    z += 3.0                                            # gates so open that states reach far
    q = [quant(v, dtype) for v in (z, x, dhs)]
    h, _ = oracle.gated_scan(q[0], q[1], h0, lens, mode == "coupled")
    tol = _bounds(q[0], q[1], h0, lens, mode == "coupled", q[2], dhT, dtype)
    got = _run(T, B, H, dtype, mode, z, x, h0, lens, dhs, dhT)
    live = np.arange(T)[:, None] < (np.full(B, T) if lens is None else np.clip(lens, 0, T))
    _compare(got, {"hs": np.where(live[..., None], h[1:], 0.0), "hT": h[-1]}, tol)
    whole = _run(T, B, H, dtype, mode, z, x, h0, lens, dhs, dhT, use_ws=False)
    # a gradient in one piece is within the bound of the oracle's (above): this one of it
    _compare(got, {k: whole[k] for k in ("dz", "dx", "dh0")}, {k: 2 * v for k, v in tol.items()})
    for _ in range(3):
        again = _run(T, B, H, dtype, mode, z, x, h0, lens, dhs, dhT)
        assert all((again[k] == got[k]).all() for k in got)


@pytest.mark.parametrize("T", [1, 40, 900, 1500])
def test_state_in_place_and_in_pieces(T):
    """hT may be h0 and dh0 may be dhT: a sequence fed in pieces through one state."""
    import torch
    B, H = 2, 72
    z, x, h0, dhs, dhT, _ = _case(3 * T, B, H, "f32", False, False, 4)
    ref = _reference(z, x, h0, None, True, dhs, dhT)
    tol = _bounds(z, x, h0, None, True, dhs, dhT, "f32")
    state = to_dev(h0)
    starts, hs = [], []
    ws = torch.empty(dl.gated_scan_ws_bytes("f32", T, B, H), dtype=torch.uint8, device=device())
    zd, xd, dd = to_dev(z), to_dev(x), to_dev(dhs)
    for i in range(3):
        starts.append(state.clone())
        out = torch.empty((T, B, H), device=device())
        dl.gated_scan_forward("f32", "coupled", T, B, H, zd[i * T:(i + 1) * T], H,
                              xd[i * T:(i + 1) * T], H, state, None, out, H, state, ws)
        hs.append(out)
    got = {"hs": np.concatenate([to_np(v) for v in hs]), "hT": to_np(state)}
    mu = to_dev(dhT)
    dz, dx = torch.empty_like(zd), torch.empty_like(zd)
    for i in (2, 1, 0):
        s = slice(i * T, (i + 1) * T)
        dl.gated_scan_backward("f32", "coupled", T, B, H, zd[s], H, xd[s], H, starts[i], None,
                               hs[i], H, dd[s], H, mu, dz[s], H, dx[s], H, mu, ws)
    got |= {"dz": to_np(dz), "dx": to_np(dx), "dh0": to_np(mu)}
    # each join of two pieces rounds a state that the bound counts as one more step
    _compare(got, ref, {k: 2 * v for k, v in tol.items()})


@pytest.mark.parametrize("size", [(1, 1, 8), (6, 3, 64), (400, 1, 64)])
@pytest.mark.parametrize("mode", ["free", "coupled"])
def test_gates_open_and_shut(size, mode):
    """Preactivations of +-infinity and of the type's largest values: a is 0 or 1."""
    T, B, H = size
    z, x, h0, dhs, dhT, _ = _case(T, B, H, "f32", False, False, 5)
    big = np.finfo(np.float32).max
    z = _rng(6, T).choice(np.array([np.inf, -np.inf, big, -big, 0, 120, -120], np.float32), z.shape)
    ref = _reference(z, x, h0, None, mode == "coupled", dhs, dhT)
    tol = _bounds(np.clip(z, -200, 200), x, h0, None, mode == "coupled", dhs, dhT, "f32")
    _compare(_run(T, B, H, "f32", mode, z, x, h0, None, dhs, dhT), ref, tol)


def test_offsets_beyond_32_bits():
    """More than 2^32 bytes and 2^31 elements between the first and the last row."""
    import torch
    T, B, H, ld = 9, 3, 24, (1 << 31) // 26 // 8 * 8
    r = _rng(7)
    z, x = r.standard_normal((T, B, H)).astype(np.float32), r.standard_normal((T, B, H)).astype(np.float32)
    buf = torch.zeros((T * B - 1) * ld + 2 * H, dtype=torch.bfloat16, device=device())
    rows = buf.as_strided((T * B, 2 * H), (ld, 1))
    rows[:, :H], rows[:, H:] = to_dev(z.reshape(-1, H), "bf16"), to_dev(x.reshape(-1, H), "bf16")
    hs = torch.empty((T, B, H), dtype=torch.bfloat16, device=device())
    hT = torch.empty((B, H), device=device())
    assert T * B * ld > 1 << 31
    dl.gated_scan_forward("bf16", "free", T, B, H, buf, ld, buf[H:], ld, None, None, hs, H, hT)
    qz, qx = quant(z, "bf16"), quant(x, "bf16")
    h, _ = oracle.gated_scan(qz, qx, None, None, False)
    tol = _bounds(qz, qx, None, None, False, None, np.ones((B, H)), "bf16")
    assert (np.abs(to_np(hT) - h[-1]) <= tol["hT"]).all()
