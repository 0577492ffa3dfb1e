"""What the sequence operators are timed on: token embeddings, the gated linear
recurrence, and the scoring of tokens, each in the calls that a program training or
serving a recurrent language model makes, from one token to the largest batch.

A case is a plain dict; its "op" says which operator a pass goes through:

  embed   embedding_forward, then embedding_backward if "train"
  scan    gated_scan_forward, then gated_scan_backward if "train"
  score   token_logprobs, then token_logprobs_backward if "train"

`run` computes them in their plain form with elementary torch operations, or, where
`own` is true, through the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

_TD = {"f32": torch.float32, "bf16": torch.bfloat16}
_ES = {"f32": 4, "bf16": 2}
_DEV = "cuda"


def listed():
    return [
        # Serving: the rows of one batch's next tokens, what a lookup costs beside its bytes.
        _embed("embed_lookup_bf16", "bf16", 64, 32768, 1024, False),
        # A training batch of 32 x 2048 tokens against a large vocabulary: the lookup, and
        # the gradient of the whole table, most of whose rows no token of the batch touches.
        _embed("embed_train_bf16", "bf16", 65536, 131072, 1024, True),
        # A small float32 model: odd width, odd vocabulary, a batch that fills nothing.
        _embed("embed_train_odd_f32", "f32", 4099, 32003, 1001, True),
        # Characters or bytes as tokens: a short narrow table and many tokens to each row.
        _embed("embed_train_narrow_bf16", "bf16", 200001, 1021, 160, True),
        # Serving: one step of 64 sequences, the state carried in float32.
        _scan("scan_step_bf16", "bf16", "coupled", 1, 64, 1024, False, False, 1),
        # The recurrent workload's sizes (32 steps, batch 1024, 1024 wide), a training step.
        _scan("scan_train_short_bf16", "bf16", "coupled", 32, 1024, 1024, True, False, 1),
        # A training step over long sequences: gate and input are the two halves of one product.
        _scan("scan_train_long_bf16", "bf16", "coupled", 4096, 4, 2048, True, False, 2),
        # One very long sequence read by a narrow model in float32.
        _scan("scan_prefill_f32", "f32", "free", 65536, 1, 512, False, False, 1),
        # A padded batch of sequences of unequal lengths, no size a multiple of anything.
        _scan("scan_train_ragged_f32", "f32", "free", 777, 13, 1001, True, True, 1),
        # Serving: the choices of 8 sequences' next token with twenty alternatives each.
        _score("score_step_bf16", "bf16", 8, 131072, 20, False),
        # Scoring a batch of texts under a large vocabulary with a few alternatives.
        _score("score_large_bf16", "bf16", 4096, 131072, 5, False),
        # A policy's training step: log probabilities, entropy and the gradient of both.
        _score("score_train_odd_f32", "f32", 2048, 50001, 0, True),
    ]


def _embed(name, dtype, tokens, vocab, width, train):
    return dict(name=name, op="embed", dtype=dtype, tokens=tokens, vocab=vocab, width=width,
                train=train)


def _scan(name, dtype, mode, steps, batch, width, train, ragged, halves):
    return dict(name=name, op="scan", dtype=dtype, mode=mode, steps=steps, batch=batch,
                width=width, train=train, ragged=ragged, halves=halves)


def _score(name, dtype, rows, classes, top, train):
    return dict(name=name, op="score", dtype=dtype, rows=rows, classes=classes, top=top,
                train=train)


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _rounded(rng, n, to):
    """n, rounded up to a multiple of `to` two times in three (odd sizes otherwise)."""
    return n if rng.random() < 1 / 3 else -(-n // to) * to


def draw(rng):
    op = rng.choice(("embed", "scan", "score"))
    dtype = rng.choice(("f32", "bf16"))
    train = rng.random() < 0.6
    while True:
        if op == "embed":
            c = _embed("", dtype, _log_uniform(rng, 1, 200000), _log_uniform(rng, 256, 131072),
                       _rounded(rng, _log_uniform(rng, 64, 2048), 64), train)
        elif op == "scan":
            c = _scan("", dtype, rng.choice(("free", "coupled")), _log_uniform(rng, 1, 65536),
                      _log_uniform(rng, 1, 1024), _rounded(rng, _log_uniform(rng, 64, 2048), 64),
                      train, rng.random() < 0.3, 1)
            # halves of one product start on 16 bytes only where the width allows it
            c["halves"] = 2 if c["width"] % 8 == 0 and rng.random() < 0.4 else 1
        else:
            c = _score("", dtype, _log_uniform(rng, 1, 16384),
                       _rounded(rng, _log_uniform(rng, 1000, 131072), 64),
                       rng.choice((0, 1, 5, 20)), train)
        # the plain scan makes log2(steps) passes over float32 copies: a third of the bytes
        if work(c)["bytes"] <= (0.35e9 if op == "scan" else 0.9e9):
            break
    del c["name"]
    return c


def work(case):
    es = _ES[case["dtype"]]
    if case["op"] == "embed":
        n, v, e = case["tokens"], case["vocab"], case["width"]
        rows = min(n, v)  # the table's rows that are read: at most one for each token
        b, f = (rows + n) * e * es + 4 * n, n * e
        if case["train"]:
            b, f = b + n * e * es + 4 * v * e, f + 2 * n * e
    elif case["op"] == "scan":
        n, r = case["steps"] * case["batch"] * case["width"], case["batch"] * case["width"]
        b, f = 3 * n * es + 8 * r, 10 * n
        if case["train"]:
            b, f = b + 3 * n * es + 8 * r, f + 20 * n
    else:
        n, r = case["rows"] * case["classes"], case["rows"]
        b, f = n * es + r * (16 + 8 * case["top"]), 6 * n
        if case["train"]:
            b, f = b + n * es + 8 * r, f + 10 * n
    return {"bytes": b, "flops": f}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device=_DEV).manual_seed(int(seed))
    td = _TD[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=_DEV, dtype=torch.float32)

    def uniform(*shape):
        return torch.rand(shape, generator=g, device=_DEV, dtype=torch.float32)

    s = dict(case=dict(case), kept={})
    if case["op"] == "embed":
        n, v, e = case["tokens"], case["vocab"], case["width"]
        s["table"] = (normal(v, e) * 0.02).to(td)
        # frequencies of tokens fall as one over their rank; one position in fifty is padding
        ids = (torch.exp(uniform(n) * math.log(v + 1)) - 1).to(torch.int32).clamp_(0, v - 1)
        s["ids"] = torch.where(uniform(n) < 0.02, torch.full_like(ids, -1), ids)
        s["scale"] = math.sqrt(e)
        if case["train"]:
            s["dout"] = (normal(n, e) * 0.1).to(td)
    elif case["op"] == "scan":
        t, b, h = case["steps"], case["batch"], case["width"]
        if case["halves"] == 2:
            zx = normal(t, b, 2 * h)
            zx[..., :h].mul_(1.5).add_(2.0)
            zx = zx.to(td)
            s["z"], s["x"] = zx[..., :h], zx[..., h:]
        else:
            s["z"], s["x"] = (normal(t, b, h) * 1.5 + 2.0).to(td), normal(t, b, h).to(td)
        s["h0"] = normal(b, h) * 0.5
        s["lens"] = None
        if case["ragged"]:
            s["lens"] = (uniform(b) * (t + 1)).to(torch.int32).clamp_(0, t)
        if case["train"]:
            s["dhs"] = (normal(t, b, h) * 0.1).to(td)
            s["dhT"] = normal(b, h) * 0.1
    else:
        r, v = case["rows"], case["classes"]
        z = normal(r, v)
        z *= 0.5 + 3.0 * uniform(r, 1)  # from nearly even rows to ones with a clear favourite
        s["logits"] = z.to(td)
        s["tokens"] = (uniform(r) * v).to(torch.int32).clamp_(0, v - 1)
        s["scale"] = 1.25
        if case["train"]:
            s["dlogp"] = normal(r) / r
            s["dentropy"] = torch.full((r,), -0.01 / r, device=_DEV)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    op = s["case"]["op"]
    if own:
        return {"embed": _own_embed, "scan": _own_scan, "score": _own_score}[op](s)
    return {"embed": _plain_embed, "scan": _plain_scan, "score": _plain_score}[op](s)


def _plain_embed(s):
    ids, td = s["ids"].long(), s["table"].dtype
    have = (ids >= 0)[:, None]
    row = ids.clamp(min=0)
    out = {"out": torch.where(have, s["table"][row].float() * s["scale"], 0.0).to(td)}
    if s["case"]["train"]:
        g = torch.where(have, s["dout"].float() * s["scale"], 0.0)
        out["dtable"] = torch.zeros(s["table"].shape, device=g.device).index_add_(0, row, g)
    return out


def _compose(a, b):
    """h_t = a_t h_{t-1} + b_t from h_{-1} = 0 along the first axis: each pass joins every
    step's map with that of the step `k` before it, k = 1, 2, 4, ..."""
    k = 1
    while k < a.shape[0]:
        b = torch.cat((b[:k], b[k:] + a[k:] * b[:-k]))
        a = torch.cat((a[:k], a[k:] * a[:-k]))
        k *= 2
    return b


def _plain_scan(s):
    case, td = s["case"], s["z"].dtype
    t = case["steps"]
    z, x = s["z"].float(), s["x"].float()
    live = None
    if s["lens"] is not None:
        live = (torch.arange(t, device=z.device)[:, None] < s["lens"][None, :])[..., None]
    a = torch.sigmoid(z)
    u = torch.sigmoid(-z) * x if case["mode"] == "coupled" else x
    if live is not None:
        a, u = torch.where(live, a, 1.0), torch.where(live, u, 0.0)
    u = torch.cat((u[:1] + a[:1] * s["h0"], u[1:]))
    h = _compose(a, u)
    out = {"hs": (h if live is None else torch.where(live, h, 0.0)).to(td), "hT": h[-1]}
    if case["train"]:
        prev = torch.cat((s["h0"][None], h[:-1]))
        dhs = s["dhs"].float()
        if live is not None:
            dhs = torch.where(live, dhs, 0.0)
        d = torch.cat((dhs[:-1], dhs[-1:] + s["dhT"]))
        # lam_t = d_t + a_{t+1} lam_{t+1}: the same recurrence from the last step backwards
        lam = _compose(torch.cat((torch.ones_like(a[:1]), a.flip(0)[:-1])), d.flip(0)).flip(0)
        c = torch.sigmoid(-z)
        if case["mode"] == "coupled":
            dx, dz = c * lam, lam * (prev - x) * a * c
        else:
            dx, dz = lam, lam * prev * a * c
        if live is not None:
            dx, dz = torch.where(live, dx, 0.0), torch.where(live, dz, 0.0)
        out |= {"dz": dz.to(td), "dx": dx.to(td), "dh0": a[0] * lam[0]}
    return out


def _plain_score(s):
    case, z = s["case"], s["logits"].float()
    y = z * s["scale"]
    m = y.amax(1, keepdim=True)
    y -= m
    p = torch.exp(y)
    total = p.sum(1, keepdim=True)
    lt = torch.log(total)
    p /= total
    entropy = (lt - (p * y).sum(1, keepdim=True))
    at = s["tokens"].long()[:, None]
    out = {"logp": (y.gather(1, at) - lt)[:, 0], "lse": (m + lt)[:, 0], "entropy": entropy[:, 0]}
    if case["top"]:
        # whole numbers in the order of the logits, the lowest index first among equals
        key = (z + 0.0).view(torch.int32)
        key = torch.where(key < 0, key ^ 0x7FFFFFFF, key).long() << 32
        key += 0xFFFFFFFF - torch.arange(z.shape[1], device=z.device)
        idx = 0xFFFFFFFF - (key.topk(case["top"], dim=1).values & 0xFFFFFFFF)
        out |= {"top_ids": idx.int(), "top_logp": y.gather(1, idx) - lt}
    if case["train"]:
        d = -s["dlogp"][:, None] * p
        d.scatter_add_(1, at, s["dlogp"][:, None])
        d -= s["dentropy"][:, None] * p * (y - lt + entropy)
        out["dlogits"] = (d * s["scale"]).to(s["logits"].dtype)
    return out


def _buffer(s, name, shape, dtype):
    """An output or workspace of the library's calls, made on the state's first pass."""
    if name not in s["kept"]:
        s["kept"][name] = torch.empty(shape, dtype=dtype, device=_DEV)
    return s["kept"][name]


def _own_embed(s):
    import paper_1711_03016_amd as dl

    c = s["case"]
    n, v, e, td = c["tokens"], c["vocab"], c["width"], _TD[c["dtype"]]
    out = {"out": _buffer(s, "out", (n, e), td)}
    dl.embedding_forward(c["dtype"], v, e, n, s["table"], s["ids"], s["scale"], out["out"])
    if c["train"]:
        out["dtable"] = _buffer(s, "dtable", (v, e), torch.float32)
        if "ws" not in s["kept"]:
            _buffer(s, "ws", (dl.embedding_backward_ws_bytes(v, e, n),), torch.uint8)
        dl.embedding_backward(c["dtype"], v, e, n, s["ids"], s["dout"], s["scale"], False,
                              out["dtable"], s["kept"]["ws"])
    return out


def _own_scan(s):
    import paper_1711_03016_amd as dl

    c = s["case"]
    t, b, h, td = c["steps"], c["batch"], c["width"], _TD[c["dtype"]]
    ld = h * c["halves"]
    if "ws" not in s["kept"]:
        _buffer(s, "ws", (dl.gated_scan_ws_bytes(c["dtype"], t, b, h),), torch.uint8)
    ws = s["kept"]["ws"]
    out = {"hs": _buffer(s, "hs", (t, b, h), td), "hT": _buffer(s, "hT", (b, h), torch.float32)}
    dl.gated_scan_forward(c["dtype"], c["mode"], t, b, h, s["z"], ld, s["x"], ld, s["h0"],
                          s["lens"], out["hs"], h, out["hT"], ws)
    if c["train"]:
        out["dz"], out["dx"] = _buffer(s, "dz", (t, b, h), td), _buffer(s, "dx", (t, b, h), td)
        out["dh0"] = _buffer(s, "dh0", (b, h), torch.float32)
        dl.gated_scan_backward(c["dtype"], c["mode"], t, b, h, s["z"], ld, s["x"], ld, s["h0"],
                               s["lens"], out["hs"], h, s["dhs"], h, s["dhT"], out["dz"], h,
                               out["dx"], h, out["dh0"], ws)
    return out


def _own_score(s):
    import paper_1711_03016_amd as dl

    c = s["case"]
    r, v, k, td = c["rows"], c["classes"], c["top"], _TD[c["dtype"]]
    f32 = torch.float32
    out = {m: _buffer(s, m, (r,), f32) for m in ("logp", "lse", "entropy")}
    if k:
        out["top_ids"] = _buffer(s, "top_ids", (r, k), torch.int32)
        out["top_logp"] = _buffer(s, "top_logp", (r, k), f32)
    if "ws" not in s["kept"]:
        _buffer(s, "ws", (dl.token_logprobs_ws_bytes(r, v, k),), torch.uint8)
    dl.token_logprobs(c["dtype"], r, v, s["logits"], v, s["scale"], s["tokens"], out["logp"],
                      out["lse"], out["entropy"], k, out.get("top_ids"), out.get("top_logp"),
                      s["kept"]["ws"])
    if c["train"]:
        out["dlogits"] = _buffer(s, "dlogits", (r, v), td)
        dl.token_logprobs_backward(c["dtype"], c["dtype"], r, v, s["logits"], v, s["scale"],
                                   s["tokens"], out["lse"], out["entropy"], s["dlogp"],
                                   s["dentropy"], out["dlogits"], v)
    return out


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "scan": _exact_scan, "score": _exact_score}[case["op"]](s)


def _exact_embed(s):
    ids = s["ids"].long()
    at = ids.clamp(min=0)
    out = {"out": s["table"].double()[at] * s["scale"] * (ids >= 0).double()[:, None]}
    if s["case"]["train"]:
        # tokens sorted by row: rows of at most 16 tokens take them one rank at a time (the
        # tokens of one rank have distinct rows), rows of more are summed one by one
        have = torch.nonzero(ids >= 0)[:, 0]
        rows, order = ids[have].sort(stable=True)
        d = torch.zeros(s["table"].shape, dtype=torch.float64, device=ids.device)
        uniq, counts = torch.unique_consecutive(rows, return_counts=True)
        begin = counts.cumsum(0) - counts
        begins, sizes, names = begin.tolist(), counts.tolist(), uniq.tolist()
        short = counts <= 16
        for k in range(16):
            m = short & (counts > k)
            if bool(m.any()):
                d[uniq[m]] += s["dout"][have[order[begin[m] + k]]].double()
        for b, n, v in zip(begins, sizes, names):
            if n > 16:
                d[v] = s["dout"][have[order[b:b + n]]].double().sum(0)
        out["dtable"] = d * s["scale"]
    return out


def _exact_scan(s):
    case = s["case"]
    t, coupled = case["steps"], case["mode"] == "coupled"
    n = None if s["lens"] is None else s["lens"].long()[:, None]
    h = s["h0"].double()
    hs = torch.zeros((t + 1, *h.shape), dtype=torch.float64, device=h.device)
    hs[0] = h
    for i in range(t):
        z, x = s["z"][i].double(), s["x"][i].double()
        a = 1 / (1 + torch.exp(-z))
        new = a * h + ((1 - a) * x if coupled else x)
        h = new if n is None else torch.where(n > i, new, h)
        hs[i + 1] = h
    shown = hs[1:]
    if n is not None:
        shown = shown * (torch.arange(t, device=h.device)[:, None, None] < n[None]).double()
    out = {"hs": shown, "hT": h}
    if case["train"]:
        dz, dx = torch.zeros_like(hs[1:]), torch.zeros_like(hs[1:])
        mu = s["dhT"].double()
        for i in range(t - 1, -1, -1):
            z, x = s["z"][i].double(), s["x"][i].double()
            a = 1 / (1 + torch.exp(-z))
            lam = mu + s["dhs"][i].double()
            gx = lam * (1 - a) if coupled else lam
            gz = lam * (hs[i] - x if coupled else hs[i]) * a * (1 - a)
            on = torch.ones_like(lam) if n is None else (n > i).double().expand_as(lam)
            dz[i], dx[i] = gz * on, gx * on
            mu = a * lam * on + mu * (1 - on)
        out |= {"dz": dz, "dx": dx, "dh0": mu}
    return out


def _exact_score(s):
    case = s["case"]
    r, v = s["logits"].shape
    new = {m: [] for m in ("logp", "lse", "entropy", "top_logp", "dlogits")}
    step = max(1, (1 << 26) // v)
    for b in range(0, r, step):
        y = s["logits"][b:b + step].double() * s["scale"]
        lse = torch.logsumexp(y, 1)
        lp = y - lse[:, None]
        p = torch.exp(lp)
        ent = -(p * lp).sum(1)
        hot = torch.zeros_like(p)
        hot[torch.arange(len(p), device=p.device), s["tokens"][b:b + step].long()] = 1
        new["logp"].append((lp * hot).sum(1))
        new["lse"].append(lse)
        new["entropy"].append(ent)
        if case["top"]:
            new["top_logp"].append(lp.topk(case["top"], dim=1).values)
        if case["train"]:
            gl, ge = s["dlogp"][b:b + step].double(), s["dentropy"][b:b + step].double()
            d = gl[:, None] * (hot - p) - ge[:, None] * p * (lp + ent[:, None])
            new["dlogits"].append(d * s["scale"])
    out = {k: torch.cat(x) for k, x in new.items() if x}
    if case["top"]:
        out["top_ids"] = None
    return out
