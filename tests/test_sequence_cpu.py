"""Refusals of the sequence operators' calls: every one fails on the host, before any
device call, with its status and a message. Device pointers are made-up addresses."""
import math

import pytest

import paper_1711_03016_amd as dl

A = 1 << 20          # 16-byte aligned
ODD = A + 4
I32 = (1 << 31) - 1


@pytest.fixture(scope="module", autouse=True)
def built_library():
    import os
    if not os.path.exists(dl.LIB_PATH):
        from paper_1711_03016_amd import build
        build.build()


def _call(name, defaults, changes):
    args = {**defaults, **changes}
    assert set(args) == set(defaults), set(changes) - set(defaults)
    status = getattr(dl.lib(), name)(*args.values())
    if status != dl.OK:
        assert dl.lib().dlvm_last_error()
    return status


INV, MIS, WS, UNS = dl.ERR_INVALID_ARG, dl.ERR_MISALIGNED, dl.ERR_WORKSPACE, dl.ERR_UNSUPPORTED

LOOKUP = dict(dtype=0, vocab=10, width=4, tokens=3, table=A, ids=A, scale=1.0, out=A, stream=None)


@pytest.mark.parametrize("changes,status", [
    (dict(dtype=2), INV), (dict(dtype=-1), INV), (dict(vocab=0), INV), (dict(width=0), INV),
    (dict(tokens=0), INV), (dict(tokens=-1), INV), (dict(scale=math.nan), INV),
    (dict(scale=math.inf), INV), (dict(table=None), INV), (dict(ids=None), INV), (dict(out=None), INV),
    (dict(table=ODD), MIS), (dict(ids=ODD), MIS), (dict(out=ODD), MIS),
    (dict(vocab=(1 << 24) + 1), UNS), (dict(width=(1 << 20) + 1), UNS), (dict(tokens=(1 << 30) + 1), UNS),
])
def test_embedding_forward_refuses(changes, status):
    assert _call("dlvm_embedding_forward", LOOKUP, changes) == status


GRAD = dict(dtype=0, vocab=10, width=4, tokens=3, ids=A, dout=A, scale=1.0, accumulate=0, dtable=A,
            ws=A, ws_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("changes,status", [
    (dict(dtype=9), INV), (dict(vocab=0), INV), (dict(width=-2), INV), (dict(tokens=0), INV),
    (dict(scale=-math.inf), INV), (dict(accumulate=2), INV), (dict(accumulate=-1), INV),
    (dict(ids=None), INV), (dict(dout=None), INV), (dict(dtable=None), INV), (dict(ws=None), WS),
    (dict(ws_bytes=0), WS), (dict(ids=ODD), MIS), (dict(dout=ODD), MIS), (dict(dtable=ODD), MIS),
    (dict(ws=ODD), MIS), (dict(vocab=1 << 25), UNS), (dict(tokens=1 << 31), UNS),
])
def test_embedding_backward_refuses(changes, status):
    assert _call("dlvm_embedding_backward", GRAD, changes) == status


def test_embedding_backward_wants_its_whole_workspace():
    for v, e, n in ((10, 4, 3), (131072, 1024, 65536), (1 << 24, 8, 1 << 20)):
        need = dl.embedding_backward_ws_bytes(v, e, n)
        assert need > 0
        assert _call("dlvm_embedding_backward", GRAD, dict(vocab=v, width=e, tokens=n, ws_bytes=need - 1)) == WS
    for bad in ((0, 4, 3), (10, 0, 3), (10, 4, 0), (1 << 25, 4, 3), (10, 1 << 25, 3), (10, 4, 1 << 31)):
        assert dl.embedding_backward_ws_bytes(*bad) == 0


SCAN = dict(dtype=0, mode=0, steps=5, batch=2, width=8, z=A, ldz=8, x=A, ldx=8, h0=A, lens=A, hs=A,
            ldh=8, hT=A, ws=A, ws_bytes=1 << 40, stream=None)
SCAN_SIZES = [
    (dict(dtype=3), INV), (dict(mode=2), INV), (dict(mode=-1), INV), (dict(steps=0), INV),
    (dict(batch=0), INV), (dict(width=0), INV), (dict(ldz=7), INV), (dict(ldx=7), INV),
    (dict(ldh=7), INV), (dict(z=None), INV), (dict(x=None), INV), (dict(hs=None), INV),
    (dict(ws_bytes=0), WS), (dict(z=ODD), MIS), (dict(x=ODD), MIS), (dict(h0=ODD), MIS),
    (dict(lens=ODD), MIS), (dict(hs=ODD), MIS), (dict(ws=ODD), MIS),
    (dict(steps=I32 + 1), UNS), (dict(batch=1 << 16, width=1 << 15, ldz=1 << 15, ldx=1 << 15, ldh=1 << 15), UNS),
    (dict(steps=1 << 16, batch=1 << 15), UNS), (dict(ldz=(1 << 31) + 8), UNS),
]


@pytest.mark.parametrize("changes,status", SCAN_SIZES + [(dict(hT=ODD), MIS)])
def test_gated_scan_forward_refuses(changes, status):
    assert _call("dlvm_gated_scan_forward", SCAN, changes) == status


SCANB = dict(dtype=0, mode=0, steps=5, batch=2, width=8, z=A, ldz=8, x=A, ldx=8, h0=A, lens=A, hs=A,
             ldh=8, dhs=A, lddh=8, dhT=A, dz=A, lddz=8, dx=A, lddx=8, dh0=A, ws=A, ws_bytes=1 << 40,
             stream=None)


@pytest.mark.parametrize("changes,status", SCAN_SIZES + [
    (dict(lddh=7), INV), (dict(lddz=7), INV), (dict(lddx=7), INV), (dict(dz=None), INV),
    (dict(dx=None), INV), (dict(dhs=None, dhT=None), INV), (dict(dhs=ODD), MIS), (dict(dhT=ODD), MIS),
    (dict(dz=ODD), MIS), (dict(dx=ODD), MIS), (dict(dh0=ODD), MIS), (dict(lddh=1 << 40), UNS),
])
def test_gated_scan_backward_refuses(changes, status):
    assert _call("dlvm_gated_scan_backward", SCANB, changes) == status


B, C, D, E, F = (A + 4096 * i for i in range(1, 6))


@pytest.mark.parametrize("call,args,changes", [
    ("dlvm_embedding_forward", LOOKUP, dict(ids=B)),
    ("dlvm_embedding_backward", GRAD, dict(ids=B)),
    ("dlvm_gated_scan_forward", SCAN, dict(x=B)), ("dlvm_gated_scan_forward", SCAN, dict(z=B)),
    ("dlvm_gated_scan_backward", SCANB, dict(z=B, x=C, hs=D, dhs=E, dx=E)),
    ("dlvm_gated_scan_backward", SCANB, dict(z=B, x=C, hs=D, dhs=E, dx=F, dz=B)),
    ("dlvm_gated_scan_backward", SCANB, dict(z=B, x=C, hs=D, dhs=E, dx=F, dz=F)),
])
def test_outputs_in_place_of_inputs_are_refused(call, args, changes):
    assert _call(call, args, changes) == INV


def test_gated_scan_workspace():
    for dtype in ("f32", "bf16"):
        for t, b, h in ((1, 1, 1), (100000, 1, 64), (77, 1000, 1000)):
            need = dl.gated_scan_ws_bytes(dtype, t, b, h)
            assert need > 0
            ld = dict(steps=t, batch=b, width=h, ldz=h, ldx=h, ldh=h, ws_bytes=need - 1)
            assert _call("dlvm_gated_scan_forward", SCAN, {**ld, "dtype": dl.DTYPES[dtype]}) == WS
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1 << 31, 1, 1), (1, 1 << 16, 1 << 16)):
        assert dl.gated_scan_ws_bytes("f32", *bad) == 0
    assert dl.lib().dlvm_gated_scan_ws_bytes(5, 1, 1, 1) == 0


SCORES = dict(dtype=0, rows=3, classes=50, logits=A, ld=50, scale=1.0, tokens=A, logp=A, lse=A,
              entropy=A, top=4, top_ids=A, top_logp=A, ws=A, ws_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("changes,status", [
    (dict(dtype=4), INV), (dict(rows=0), INV), (dict(classes=0), INV), (dict(ld=49), INV),
    (dict(scale=0.0), INV), (dict(scale=-1.0), INV), (dict(scale=math.nan), INV), (dict(scale=math.inf), INV),
    (dict(logits=None), INV), (dict(tokens=None), INV), (dict(logp=None), INV), (dict(top=-1), INV),
    (dict(top=33), INV), (dict(classes=3, ld=3), INV), (dict(top=0), INV), (dict(top_ids=None), INV),
    (dict(top_logp=None), INV),
    (dict(tokens=None, logp=None, lse=None, entropy=None, top=0, top_ids=None, top_logp=None), INV),
    (dict(ws_bytes=0), WS), (dict(logits=ODD), MIS), (dict(tokens=ODD), MIS), (dict(logp=ODD), MIS),
    (dict(lse=ODD), MIS), (dict(entropy=ODD), MIS), (dict(top_ids=ODD), MIS), (dict(top_logp=ODD), MIS),
    (dict(ws=ODD), MIS), (dict(rows=1 << 31), UNS), (dict(classes=(1 << 30) + 1, ld=1 << 31), UNS),
    (dict(ld=(1 << 31) + 1), UNS),
])
def test_token_logprobs_refuses(changes, status):
    assert _call("dlvm_token_logprobs", SCORES, changes) == status


SCORESB = dict(dtype=0, out_dtype=0, rows=3, classes=50, logits=A, ld=50, scale=1.0, tokens=A, lse=A,
               entropy=A, dlogp=A, dentropy=A, dlogits=A + 4096, ld_out=50, stream=None)


@pytest.mark.parametrize("changes,status", [
    (dict(dtype=4), INV), (dict(out_dtype=4), INV), (dict(rows=0), INV), (dict(classes=-1), INV),
    (dict(ld=49), INV), (dict(ld_out=49), INV), (dict(scale=0.0), INV), (dict(dtype=1), UNS),
    (dict(logits=None), INV), (dict(lse=None), INV), (dict(dlogits=None), INV),
    (dict(dlogp=None, dentropy=None), INV), (dict(tokens=None), INV), (dict(entropy=None), INV),
    (dict(dlogits=A, out_dtype=1), INV), (dict(dlogits=A, ld_out=51), INV),
    (dict(logits=ODD), MIS), (dict(tokens=ODD), MIS), (dict(lse=ODD), MIS), (dict(entropy=ODD), MIS),
    (dict(dlogp=ODD), MIS), (dict(dentropy=ODD), MIS), (dict(dlogits=ODD), MIS), (dict(rows=1 << 31), UNS),
])
def test_token_logprobs_backward_refuses(changes, status):
    assert _call("dlvm_token_logprobs_backward", SCORESB, changes) == status


def test_token_logprobs_workspace():
    for r, v, k in ((1, 1, 0), (1, 131072, 32), (8, 50001, 20), (4096, 131072, 5)):
        need = dl.token_logprobs_ws_bytes(r, v, k)
        assert need > 0
        assert _call("dlvm_token_logprobs", SCORES,
                     dict(rows=r, classes=v, ld=v, top=k, ws_bytes=need - 1, top_ids=A if k else None,
                          top_logp=A if k else None)) == WS
    for bad in ((0, 5, 0), (5, 0, 0), (5, 5, 6), (5, 50, 33), (5, 50, -1), (1 << 31, 5, 0)):
        assert dl.token_logprobs_ws_bytes(*bad) == 0


def test_binding_refuses_tensors_of_another_type_or_on_the_host():
    import torch
    f, b, i = torch.zeros(64), torch.zeros(64, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.int32)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    calls = [
        lambda t, n, o: dl.embedding_forward("f32", 8, 4, 2, t, n, 1.0, o, stream=0),
        lambda t, n, o: dl.embedding_backward("f32", 8, 4, 2, n, t, 1.0, False, o, ws, stream=0),
        lambda t, n, o: dl.gated_scan_forward("f32", "free", 2, 2, 4, t, 4, o, 4, None, n, o, 4, None, stream=0),
        lambda t, n, o: dl.gated_scan_backward("f32", "free", 2, 2, 4, t, 4, o, 4, None, n, o, 4, o, 4,
                                               None, o, 4, o, 4, None, stream=0),
        lambda t, n, o: dl.token_logprobs("f32", 2, 8, t, 8, 1.0, n, o, o, o, 0, None, None, stream=0),
        lambda t, n, o: dl.token_logprobs_backward("f32", "f32", 2, 8, t, 8, 1.0, n, o, o, o, o, o, 8, stream=0),
    ]
    for call in calls:
        for args in ((f, i, f), (b, i, f), (f, i.long(), f), (f, i, f.double())):
            with pytest.raises(dl.DlvmError) as e:
                call(*args)
            assert e.value.status == dl.ERR_INVALID_ARG
