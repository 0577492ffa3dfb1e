"""Tensors of the sequence operators whose rows lie between each other's in one buffer share no
memory: such calls run and give the bits of calls on buffers of their own."""
import pytest

import paper_1711_03016_amd as dl
from helpers import device, torch_dtype

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(12, 3, 64), (300, 2, 72)])
def test_recurrence_in_one_buffer(dtype, size):
    import torch
    T, B, H = size
    td = torch_dtype(dtype)
    g = torch.Generator(device=device()).manual_seed(5)
    z, x, dhs = (torch.randn((T, B, H), generator=g, device=device()).to(td) for _ in range(3))
    h0 = torch.randn((B, H), generator=g, device=device())
    ws = torch.empty(dl.gated_scan_ws_bytes(dtype, T, B, H), dtype=torch.uint8, device=device())
    new = lambda n: torch.full((T, B, n * H), 7.0, dtype=td, device=device())  # noqa: E731

    def run(z, x, hs, dz, dx, dhs, ld):
        hT, dh0 = torch.empty((B, H), device=device()), torch.empty((B, H), device=device())
        dl.gated_scan_forward(dtype, "coupled", T, B, H, z, ld, x, ld, h0, None, hs, ld, hT, ws)
        dl.gated_scan_backward(dtype, "coupled", T, B, H, z, ld, x, ld, h0, None, hs, ld, dhs, ld, None, dz, ld, dx,
                               ld, dh0, ws)
        return [v.clone() for v in (hs, dz, dx, hT, dh0)]

    want = run(z, x, new(1), new(1), new(1), dhs, H)
    all_of = new(6)
    cols = [all_of[..., i * H:(i + 1) * H] for i in range(6)]
    cols[0][:], cols[1][:], cols[5][:] = z, x, dhs
    got = run(*cols, 6 * H)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert torch.equal(cols[0], z) and torch.equal(cols[1], x) and torch.equal(cols[5], dhs)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_and_gradient_in_one_buffer(dtype):
    import torch
    R, V = 40, 1000
    td = torch_dtype(dtype)
    g = torch.Generator(device=device()).manual_seed(6)
    z = torch.randn((R, V), generator=g, device=device()).to(td)
    tokens = torch.arange(R, dtype=torch.int32, device=device())
    dlogp = torch.randn(R, generator=g, device=device())

    def run(z, d, ld):
        lse, ent, logp = (torch.empty(R, device=device()) for _ in range(3))
        dl.token_logprobs(dtype, R, V, z, ld, 1.0, tokens, logp, lse, ent, 0, None, None)
        dl.token_logprobs_backward(dtype, dtype, R, V, z, ld, 1.0, tokens, lse, ent, dlogp, None, d, ld)
        return d.clone()

    want = run(z, torch.empty_like(z), V)
    both = torch.full((R, 2 * V), 7.0, dtype=td, device=device())
    both[:, :V] = z
    assert torch.equal(run(both[:, :V], both[:, V:], 2 * V), want)
    assert torch.equal(both[:, :V], z)
