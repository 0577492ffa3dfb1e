"""Token embeddings on the GPU, lookup and gradient of the table, against the oracle.

Tolerances. The lookup rounds scale * value to float32 (half a step of 2^-24
relative) and then to the storage type (2^-8 for bf16). A row of the gradient is
a float32 sum of n products in some fixed order: each of at most n additions and
one multiplication by scale is off by at most 2^-24 of the sum of the absolute
terms.
"""
import numpy as np
import pytest

import oracle
import paper_1711_03016_amd as dl
from helpers import device, quant, to_dev, to_np, torch_dtype

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
ROUND = {"f32": 0.0, "bf16": 2.0 ** -8}
GUARD = 64


def _rng(*key):
    return np.random.default_rng([505, *key])


def _ids(r, V, N, how):
    if how == "uniform":
        ids = r.integers(0, V, N)
    elif how == "zipf":
        ids = np.minimum((np.exp(r.random(N) * np.log(V + 1)) - 1).astype(np.int64), V - 1)
    elif how == "one":
        ids = np.full(N, V // 2)
    elif how == "few":                       # two rows take turns, the last row at the end
        ids = np.where(np.arange(N) % 2 == 0, 0, V // 3)
        ids[-1] = V - 1
    elif how == "stride":                    # rows a power of two apart
        ids = (r.integers(0, max(1, V // 512), N) * 512) % V
    else:
        ids = np.full(N, -1)
    ids = ids.astype(np.int32)
    if how in ("uniform", "zipf") and N > 4:
        ids[N // 2], ids[N // 3] = -1, -1
    return ids


def _dev_ids(ids):
    import torch
    return torch.from_numpy(ids).to(device())


SIZES = [(1, 1, 1), (7, 3, 5), (50, 64, 33), (1000, 130, 257), (32003, 1001, 300), (4099, 96, 9000),
         (300, 2048, 700), (513, 8, 3000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_lookup(dtype, size):
    import torch
    V, E, N = size
    r = _rng(1, *size)
    table = r.standard_normal((V, E)).astype(np.float32)
    ids = _ids(r, V, N, "uniform")
    if N > 8:
        ids[1], ids[2], ids[3] = V, -2, np.iinfo(np.int32).min
    scale = np.float32(1.7)
    out = torch.full((N * E + GUARD,), 7.0, dtype=torch_dtype(dtype), device=device())
    dl.embedding_forward(dtype, V, E, N, to_dev(table, dtype), _dev_ids(ids), float(scale), out)
    got = to_np(out)
    assert (got[N * E:] == 7.0).all()
    ref = oracle.embedding(quant(table, dtype), ids, float(scale))
    got = got[:N * E].reshape(N, E)
    bad = np.isnan(ref)
    assert (np.isnan(got) == bad).all()
    tol = np.abs(ref) * (ROUND[dtype] + 2 * U32)
    assert (np.abs(got - ref)[~bad] <= tol[~bad]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["uniform", "zipf", "one", "few", "stride", "none"])
@pytest.mark.parametrize("size", SIZES)
def test_gradient(dtype, how, size):
    import torch
    V, E, N = size
    r = _rng(2, *size)
    ids = _ids(r, V, N, how)
    if N > 8 and how == "uniform":
        ids[1], ids[2], ids[3] = V, -2, np.iinfo(np.int32).max
    dout = r.standard_normal((N, E)).astype(np.float32)
    scale = np.float32(0.3)
    dd, di = to_dev(dout, dtype), _dev_ids(ids)
    ref, mag, cnt = oracle.embedding_grad(quant(dout, dtype), ids, V, float(scale))
    tol = (cnt[:, None] + 2) * U32 * mag
    first = None
    for fill in (0, 255):                    # whatever the workspace held before
        ws = torch.full((dl.embedding_backward_ws_bytes(V, E, N),), fill, dtype=torch.uint8,
                        device=device())
        d = torch.full((V * E + GUARD,), float("nan"), device=device())
        dl.embedding_backward(dtype, V, E, N, di, dd, float(scale), False, d, ws)
        got = to_np(d)
        assert np.isnan(got[V * E:]).all()
        got = got[:V * E].reshape(V, E)
        assert (np.abs(got - ref) <= tol).all(), np.abs(got - ref).max()
        assert first is None or (got == first).all()
        first = got
    base = r.standard_normal((V, E)).astype(np.float32)
    d = to_dev(base)
    dl.embedding_backward(dtype, V, E, N, di, dd, float(scale), True, d, ws)
    got = to_np(d)
    assert (np.abs(got - (base + ref)) <= tol + (cnt[:, None] > 0) * 2 * U32 * (np.abs(base) + mag)).all()
    assert (got[cnt == 0] == base[cnt == 0]).all()


@pytest.mark.parametrize("V,E,N", [(1021, 16, 300001), (131072, 8, 70000), (300000, 4, 5000)])
def test_gradient_of_many_tokens(V, E, N):
    """Tokens beyond one sorting launch, vocabularies of several sorting groups a row."""
    import torch
    r = _rng(3, V, E, N)
    ids = _ids(r, V, N, "zipf")
    dout = r.standard_normal((N, E)).astype(np.float32)
    have = ids >= 0
    ref, mag = np.zeros((V, E)), np.zeros((V, E))
    np.add.at(ref, ids[have], dout[have].astype(np.float64))
    np.add.at(mag, ids[have], np.abs(dout[have]).astype(np.float64))
    cnt = np.bincount(ids[have], minlength=V)
    ws = torch.full((dl.embedding_backward_ws_bytes(V, E, N),), 255, dtype=torch.uint8, device=device())
    d = torch.full((V, E), float("nan"), device=device())
    dl.embedding_backward("f32", V, E, N, _dev_ids(ids), to_dev(dout), 1.0, False, d, ws)
    assert (np.abs(to_np(d) - ref) <= (cnt[:, None] + 2) * U32 * mag).all()


def test_gradient_takes_differences():
    """The directional derivative of a loss of the lookup, by differences of the lookup."""
    import torch
    V, E, N = 40, 24, 100
    r = _rng(4)
    ids = _dev_ids(_ids(r, V, N, "zipf"))
    table, g = to_dev(r.standard_normal((V, E))), to_dev(r.standard_normal((V, E)))
    w = to_dev(r.standard_normal((N, E)))
    outs = []
    for sign in (1.0, -1.0):
        out = torch.empty((N, E), device=device())
        dl.embedding_forward("f32", V, E, N, table + sign * 0.5 * g, ids, 1.5, out)
        outs.append((out.double() * w.double()).sum().item())
    ws = torch.empty(dl.embedding_backward_ws_bytes(V, E, N), dtype=torch.uint8, device=device())
    d = torch.empty((V, E), device=device())
    dl.embedding_backward("f32", V, E, N, ids, w, 1.5, False, d, ws)
    want = (d.double() * g.double()).sum().item()
    # linear: the difference is exact but for the roundings of N * E terms of about 3
    assert abs(outs[0] - outs[1] - want) <= N * E * 4 * 4 * U32


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["zipf", "one", "few"])
@pytest.mark.parametrize("V,E,N", [(700, 20, 8193), (70001, 6, 32769), (1025, 12, 131073), (3000, 9, 270000)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_each_sort(dtype, how, V, E, N, accumulate):
    """About the numbers of tokens at which the sort changes, rows of thousands of pieces; sums
    of small whole numbers, which float32 holds exactly in any order."""
    import torch
    r = _rng(5, V, E, N)
    ids = _ids(r, V, N, how)
    dout = r.integers(-2, 3, (N, E)).astype(np.float32)
    base = r.integers(-9, 10, (V, E)).astype(np.float32)
    ref = np.stack([np.bincount(ids[ids >= 0], weights=dout[ids >= 0, c], minlength=V) for c in range(E)], axis=1)
    ws = torch.full((dl.embedding_backward_ws_bytes(V, E, N),), 255, dtype=torch.uint8, device=device())
    d = to_dev(base) if accumulate else torch.full((V, E), float("nan"), device=device())
    dl.embedding_backward(dtype, V, E, N, _dev_ids(ids), to_dev(dout, dtype), 2.0, accumulate, d, ws)
    assert (to_np(d) == 2 * ref + (base if accumulate else 0)).all()


def test_offsets_beyond_32_bits():
    """Tables of more than 2^31 elements: rows at their ends looked up, and summed."""
    import torch
    V, E = 1_060_000, 2048
    assert V * E > 1 << 31
    r = _rng(6)
    rows = np.array([0, 1, V // 2, 1048576, V - 2, V - 1], np.int32)
    ids = np.concatenate([rows, rows[::-1], [-1, V]]).astype(np.int32)
    values = quant(r.standard_normal((len(rows), E)).astype(np.float32), "bf16")
    table = torch.zeros((V, E), dtype=torch.bfloat16, device=device())
    table[torch.from_numpy(rows.astype(np.int64)).to(device())] = to_dev(values.astype(np.float32), "bf16")
    out = torch.empty((len(ids), E), dtype=torch.bfloat16, device=device())
    dl.embedding_forward("bf16", V, E, len(ids), table, _dev_ids(ids), 2.0, out)
    got = to_np(out)
    assert (got[:6] == 2 * values).all() and (got[6:12] == 2 * values[::-1]).all()
    assert (got[12] == 0).all() and np.isnan(got[13]).all()
    del table
    d = torch.full((V, E), float("nan"), device=device())
    ws = torch.empty(dl.embedding_backward_ws_bytes(V, E, len(ids)), dtype=torch.uint8, device=device())
    dl.embedding_backward("bf16", V, E, len(ids), _dev_ids(ids), out, 1.0, False, d, ws)
    at = torch.from_numpy(rows.astype(np.int64)).to(device())
    assert (to_np(d[at]) == 4 * values).all()
    d[at] = 0.0
    assert not d.any()


@pytest.mark.parametrize("V,E,N", [(70001, 1000, 9001), (131072, 513, 20000), (40000, 333, 8193), (131071, 513, 77)])
def test_gradient_of_large_tables(V, E, N):
    """Tables zeroed beside the sort and beside the sums; sums of whole numbers, exact in any order."""
    import torch
    r = _rng(8, V, E, N)
    ids = _ids(r, V, N, "zipf")
    ids[::50] = -1
    ids[-1] = V - 1
    dout = torch.from_numpy(r.integers(-2, 3, (N, E)).astype(np.float32)).to(device())
    have = torch.from_numpy((ids >= 0).astype(np.int64).nonzero()[0]).to(device())
    ref = torch.zeros((V, E), device=device())
    ref.index_add_(0, torch.from_numpy(ids[ids >= 0].astype(np.int64)).to(device()), dout[have])
    ws = torch.full((dl.embedding_backward_ws_bytes(V, E, N),), 255, dtype=torch.uint8, device=device())
    d = torch.full((V * E + GUARD,), 7.0, device=device())
    dl.embedding_backward("f32", V, E, N, _dev_ids(ids), dout, 1.0, False, d, ws)
    assert torch.equal(d[:V * E].view(V, E), ref)
    assert (d[V * E:] == 7.0).all()
