"""Timed operators of the generator's blocks, in their plain form and as calls of ``paper_2602_04789_amd.lf``.

Finetuning a video generator, and running it over prompts and videos of different lengths, needs these beside the sparse attention:

  norm   what stands between two blocks: the first one's output, normalised or not, gated and added to the residual stream, and the
         norm before the next one with its scale and shift, which belong to a frame or a sequence; with ``train`` the gradients too
  attn   attention over packed sequences of different lengths with heads that share keys and values: every row sees its whole sequence
         (a text), the tokens up to its own, or the chunks up to its own; prompts, training, and single rows over a long cache
  clip   the norm over the gradients of all parameters and their scaling to a largest norm

Sequence lengths follow from the numbers of a case alone; inputs follow from the seed.
"""
import math

import torch

own = False

EPS = 1e-6


def _norm(name, rows, width, kind, stream, block, post, groups, ragged, pad, train):
    c = dict(op="norm", rows=rows, width=width, kind=kind, stream=stream, block=block, post=post, groups=groups, ragged=ragged, pad=pad,
             train=train)
    return dict(c, name=name) if name else c


def _attn(name, heads, kv_heads, head_dim, seqs, rows, tokens, same, unit, mix, pad, train):
    c = dict(op="attn", heads=heads, kv_heads=kv_heads, head_dim=head_dim, seqs=seqs, rows=rows, tokens=tokens, same=same, unit=unit, mix=mix,
             pad=pad, train=train)
    return dict(c, name=name) if name else c


def _clip(name, layers, width, dtype, apart, most):
    c = dict(op="clip", layers=layers, width=width, dtype=dtype, apart=apart, most=most)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token between two blocks: latency alone counts
        _norm("norm_one_token", 1, 1536, "layer", "bf16", True, False, 1, False, 0, False),
        # a chunk of the benchmark's rollout, a modulation for each of its three frames
        _norm("norm_chunk", 4680, 1536, "layer", "bf16", True, False, 3, False, 0, False),
        # finetuning, packed clips of odd lengths in a narrow model with norms before and after its blocks, float32 stream, padding behind
        _norm("norm_train_ragged", 1333, 320, "rms", "f32", True, True, 6, True, 11, True),
        # finetuning, a whole video of the 40-head model, a modulation for each of its 21 frames
        _norm("norm_train_video", 32760, 5120, "layer", "bf16", True, False, 21, False, 0, True),
        # one row over the tokens of a short text
        _attn("attn_one_row", 12, 12, 128, 1, 1, 77, False, 0, 0, 0, False),
        # serving: one row of each of 16 requests over its own past, five heads to a shared one
        _attn("attn_rows", 40, 8, 128, 16, 16, 120003, False, 1, 3, 0, False),
        # a chunk's rows over the 512 tokens of its text
        _attn("attn_text", 12, 12, 128, 1, 4680, 512, False, 0, 0, 0, False),
        # whole prompts of different lengths, token by token causal, five heads to a shared one
        _attn("attn_prompts", 40, 8, 128, 7, 16384, 16384, True, 1, 5, 0, False),
        # finetuning, packed clips of odd lengths, narrow heads, three to a shared one, padding behind
        _attn("attn_train_ragged", 6, 2, 64, 9, 1333, 1333, True, 1, 7, 19, True),
        # finetuning, a whole video of seven chunks, every chunk seeing itself and those before it
        _attn("attn_train_video", 12, 12, 128, 1, 32760, 32760, True, 4680, 0, 0, True),
        # a small model's gradients in place, their norm below the largest one
        _clip("clip_small", 2, 320, "f32", False, 1e9),
        # the gradients of a model of 30 layers, clipped into the optimizer's buffers
        _clip("clip_model", 30, 1536, "bf16", True, 1.0),
    ]


_MOST = {}


def _kind(c):
    return c["op"], c.get("train", False)


def _most():
    if not _MOST:
        for c in listed():
            w = work(c)
            most = _MOST.setdefault(_kind(c), w)
            _MOST[_kind(c)] = {k: max(v, most[k]) for k, v in w.items()}
    return _MOST


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["norm", "norm", "norm", "attn", "attn", "attn", "attn", "clip"])
        if op == "norm":
            rows = _log(rng, 1, 32760)
            block = rng.random() < 0.85
            width = rng.choice([8 * _log(rng, 1, 2048), 64 * _log(rng, 1, 120), 128 * rng.randint(1, 40)])
            ragged = rng.random() < 0.5
            c = _norm(None, rows, width, rng.choice(["layer", "rms"]), rng.choice(["bf16", "bf16", "f32"]), block,
                      block and rng.random() < 0.5, min(rows, _log(rng, 1, 64)), ragged, rng.choice([0, rng.randint(1, 70)]) if ragged else 0,
                      rng.random() < 0.6)
        elif op == "attn":
            shared, kv_heads = rng.choice([1, 1, 2, 3, 5, 8]), _log(rng, 1, 16)
            seqs, head_dim, train = _log(rng, 1, 40), rng.choice([64, 128, 128]), False
            unit, pad, mix = rng.choice([0, 1, 1, _log(rng, 2, 5000)]), rng.choice([0, rng.randint(1, 200)]), rng.randint(0, 99)
            if rng.random() < 0.4:      # serving: few rows of each sequence over its past
                rows, tokens, same = seqs * _log(rng, 1, 16), _log(rng, 1, 130000), False
            else:
                rows, same, train = _log(rng, 1, 33000), rng.random() < 0.7, rng.random() < 0.6
                tokens = rows if same else _log(rng, 1, 33000)
            c = _attn(None, shared * kv_heads, kv_heads, head_dim, seqs, rows, tokens, same, unit, mix, pad, train)
        else:
            c = _clip(None, _log(rng, 1, 40), 8 * _log(rng, 1, 250) + rng.choice([0, 0, 1, 3]), rng.choice(["bf16", "f32", "mixed"]), True,
                      rng.choice([0.01, 1.0, 1e9]))
        most, w = _most()[_kind(c)], work(c)
        if all(w[k] <= most[k] for k in w):
            return c


def _shares(total, parts, mix):
    """`total` as `parts` whole numbers: about equal ones for mix = 0, else from nothing to several times the mean."""
    if mix == 0:
        return [total * (i + 1) // parts - total * i // parts for i in range(parts)]
    x, weight = 12345 + 7919 * mix, []
    for _ in range(parts):
        x = (1103515245 * x + 12345) % (1 << 31)
        u = x / (1 << 31)
        weight.append(0.0 if u < 0.06 and parts > 2 else math.exp(2.5 * u))
    if sum(weight) == 0.0:
        weight[0] = 1.0
    edges, run = [0], 0.0
    for w in weight:
        run += w
        edges.append(int(round(total * run / sum(weight))))
    return [b - a for a, b in zip(edges, edges[1:])]


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _row_groups(c):
    """Lengths of the row groups that share a modulation."""
    if c["ragged"]:
        return _shares(c["rows"], c["groups"], 1)
    n = -(-c["rows"] // c["groups"])
    return [min(n, c["rows"] - at) for at in range(0, c["rows"], n)]


def _lengths(c):
    q = _shares(c["rows"], c["seqs"], c["mix"])
    if c["same"]:
        return q, q
    if c["rows"] <= 16 * c["seqs"]:
        q = _shares(c["rows"], c["seqs"], 0)
    return q, _shares(c["tokens"], c["seqs"], c["mix"])


def _seen(c, nq, nk, i):
    """How many of its sequence's nk tokens row i of nq sees."""
    if c["unit"] == 0:
        return nk
    return max(0, min(nk, ((nk - nq + i) // c["unit"] + 1) * c["unit"]))


def _pairs(c):
    """(row, token) pairs of one head."""
    total = 0
    for nq, nk in zip(*_lengths(c)):
        if c["unit"] == 0:
            total += nq * nk
            continue
        if c["unit"] == 1:      # n + (n + 1) + .. from the first row that sees a token on
            rows = min(nq, nk)
            total += rows * max(1, nk - nq + 1) + rows * (rows - 1) // 2
            continue
        i = 0
        while i < nq:           # rows that see the same tokens, together
            last = min(nq, max(i + 1, ((nk - nq + i) // c["unit"] + 1) * c["unit"] - (nk - nq)))
            total += (last - i) * _seen(c, nq, nk, i)
            i = last
    return total


def _tensors(c):
    """Shapes of a model's parameters: for every layer four square projections, two wide ones, two norms and a modulation."""
    w = c["width"]
    return c["layers"] * [(w, w)] * 4 + c["layers"] * [(4 * w, w)] * 2 + c["layers"] * [(w,)] * 2 + c["layers"] * [(6, w)]


def _bytes(c, i):
    return 2 if c["dtype"] == "bf16" or (c["dtype"] == "mixed" and i % 2) else 4


def work(case):
    c = case
    if c["op"] == "norm":
        n, C, s = float(c["rows"]) * c["width"], c["width"], 2 if c["stream"] == "bf16" else 4
        G = len(_row_groups(c))
        tables = 4.0 * G * C * (3 if c["block"] else 2) + 4.0 * C * ((c["kind"] == "rms") + c["post"])
        fwd = n * (s + 2 + ((2 + s) if c["block"] else 0)) + tables
        if not c["train"]:
            return {"bytes": fwd, "flops": 12.0 * n}
        # the stream, the block's output and the two upstream gradients in; the forward's outputs, two gradients and the tables' out
        return {"bytes": fwd + n * (2 + s + s + (2 if c["block"] else 0)) + tables, "flops": 40.0 * n}
    if c["op"] == "attn":
        H, Hk, d, pairs = c["heads"], c["kv_heads"], c["head_dim"], _pairs(c)
        q, kv = 2.0 * c["rows"] * H * d, 2.0 * c["tokens"] * Hk * d
        if not c["train"]:
            return {"bytes": 2 * q + 2 * kv, "flops": 4.0 * d * H * pairs}
        return {"bytes": 4 * q + 4 * kv, "flops": 14.0 * d * H * pairs}
    each = [math.prod(s) for s in _tensors(c)]
    size = float(sum(n * _bytes(c, i) for i, n in enumerate(each)))
    return {"bytes": (2.0 if c["apart"] else 1.0) * size, "flops": 3.0 * sum(each)}


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if c["op"] == "norm":
        return _prepare_norm(c, g)
    if c["op"] == "attn":
        H, Hk, d = c["heads"], c["kv_heads"], c["head_dim"]
        (nq, nk), pad = _lengths(c), c["pad"]
        rows, tokens = c["rows"] + pad, c["tokens"] + pad
        bf = torch.bfloat16
        # a few channels of the keys are larger, as projections leave them
        wide = 1.0 + 2.0 * (torch.rand((Hk, 1, d), generator=g, device="cuda") < 0.04).float()
        s = dict(case=dict(c), lengths=(nq, nk), Q=_randn(g, H, rows, d).to(bf), K=(_randn(g, Hk, tokens, d) * wide).to(bf),
                 V=_randn(g, Hk, tokens, d).to(bf), q_start=torch.tensor(_starts(nq), dtype=torch.int32, device="cuda"),
                 kv_start=torch.tensor(_starts(nk), dtype=torch.int32, device="cuda"), O=torch.zeros((H, rows, d), dtype=bf, device="cuda"))
        if c["train"]:
            s["dO"] = _randn(g, H, rows, d).to(bf)
            s["grads"] = tuple(torch.zeros_like(s[k]) for k in ("Q", "K", "V"))
        return s
    # gradients are views of one buffer for each type, one behind the other, and so is what the clipped ones are written to
    shapes, flat, out = _tensors(c), {}, {}
    for size, dt in ((2, torch.bfloat16), (4, torch.float32)):
        n = sum(math.prod(shape) for i, shape in enumerate(shapes) if _bytes(c, i) == size)
        if n:
            flat[size] = torch.empty(n, dtype=dt, device="cuda")
            out[size] = torch.empty_like(flat[size]) if c["apart"] else flat[size]
    s, at = dict(case=dict(c), flat=out, grads=[], out=[] if c["apart"] else None), {2: 0, 4: 0}
    for i, shape in enumerate(shapes):
        size, n = _bytes(c, i), math.prod(shape)
        x = flat[size][at[size]:at[size] + n].view(shape)
        x.copy_(_randn(g, *shape) * (0.02 * (1 + i % 7)))
        s["grads"].append(x)
        if c["apart"]:
            s["out"].append(out[size][at[size]:at[size] + n].view(shape))
        at[size] += n
    return s


def _prepare_norm(c, g):
    C, rows, lengths = c["width"], c["rows"] + c["pad"], _row_groups(c)
    dt = torch.bfloat16 if c["stream"] == "bf16" else torch.float32
    G = len(lengths)
    # the stream has a few channels far larger than the others, and a mean
    tall = 1.0 + 12.0 * (torch.rand((1, C), generator=g, device="cuda") < 0.01).float()
    s = dict(case=dict(c), lengths=lengths, X=(_randn(g, rows, C) * tall + 0.3).to(dt), B=None, gate=None, post=None, weight=None,
             starts=None, group_len=0)
    tables = 0.2 * _randn(g, G, 6, C)      # shift, scale and gate of a frame lie side by side
    s["shift"], s["scale"] = tables[:, 0], tables[:, 1]
    if c["block"]:
        s["B"], s["gate"] = _randn(g, rows, C).to(torch.bfloat16), tables[:, 2]
    if c["post"]:
        s["post"] = 1.0 + 0.1 * _randn(g, C)
    if c["kind"] == "rms":
        s["weight"] = 1.0 + 0.1 * _randn(g, C)
    if c["ragged"]:
        s["starts"] = torch.tensor(_starts(lengths), dtype=torch.int32, device="cuda")
    else:
        s["group_len"] = lengths[0]
    s["Xout"] = torch.zeros_like(s["X"]) if c["block"] else None
    s["Y"] = torch.zeros((rows, C), dtype=torch.bfloat16, device="cuda")
    if c["train"]:
        s["dY"], s["dXout"] = _randn(g, rows, C).to(torch.bfloat16), _randn(g, rows, C).to(dt)
        s["dX"], s["dB"] = torch.zeros_like(s["X"]), torch.zeros_like(s["Y"]) if c["block"] else None
    return s


def _plain_norm(s):
    c = s["case"]
    n = c["rows"]
    group = torch.repeat_interleave(torch.arange(len(s["lengths"]), device="cuda"), torch.tensor(s["lengths"], device="cuda"),
                                    output_size=n)
    X = s["X"]
    out = {}
    if c["block"]:
        b = s["B"][:n].float()
        rb = 1.0 / torch.sqrt((b * b).mean(1, keepdim=True) + EPS) if c["post"] else 1.0
        bn = b * rb
        p = bn * s["post"] if c["post"] else bn
        X = torch.zeros_like(X)
        X[:n] = (s["X"][:n].float() + s["gate"][group] * p).to(X.dtype)
        out["Xout"] = X
    x = X[:n].float()
    if c["kind"] == "layer":
        x = x - x.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    z = x * r
    f = 1.0 + s["scale"][group]
    if s["weight"] is not None:
        f = f * s["weight"]
    out["Y"] = torch.zeros_like(s["Y"])
    out["Y"][:n] = (z * f + s["shift"][group]).to(torch.bfloat16)
    if not c["train"]:
        return out
    dy = s["dY"][:n].float()
    u = dy * f
    u -= z * (u * z).mean(1, keepdim=True)
    if c["kind"] == "layer":
        u -= u.mean(1, keepdim=True)
    D = s["dXout"][:n].float() + r * u
    del u, f
    out["dX"] = torch.zeros_like(X)
    out["dX"][:n] = D.to(X.dtype)

    def sums(t):
        return torch.stack([part.sum(0) for part in t.split(s["lengths"])])

    zy = sums(dy * z)
    out["dshift"], out["dscale"] = sums(dy), zy if s["weight"] is None else zy * s["weight"]
    if s["weight"] is not None:
        out["dweight"] = (zy * (1.0 + s["scale"])).sum(0)
    if c["block"]:
        e = s["gate"][group] * D
        t = sums(bn * D)
        out["dgate"] = t * s["post"] if c["post"] else t
        if c["post"]:
            out["dpost"] = (t * s["gate"]).sum(0)
            e = e * s["post"]
            e = rb * (e - bn * (e * bn).mean(1, keepdim=True))
        out["dB"] = torch.zeros_like(s["dB"])
        out["dB"][:n] = e.to(torch.bfloat16)
    return out


def _plain_attn(s):
    c = s["case"]
    H, Hk, d, train = c["heads"], c["kv_heads"], c["head_dim"], c["train"]
    out = {"O": torch.zeros_like(s["O"])}
    if train:
        out["dQ"] = torch.zeros_like(s["Q"])
        out["dK"], out["dV"] = (torch.zeros(s[k].shape, device="cuda") for k in ("K", "V"))
    G, scale, q0, k0 = H // Hk, 1.0 / math.sqrt(d), 0, 0
    for nq, nk in zip(*s["lengths"]):
        K, V = (s[k][:, k0:k0 + nk].float().repeat_interleave(G, 0) for k in ("K", "V"))
        step = max(1, (1 << 28) // (H * max(nk, 1)))
        for at in range(0, nq, step):
            rows = slice(q0 + at, q0 + min(nq, at + step))
            n = rows.stop - rows.start
            if nk == 0:
                continue
            Q = s["Q"][:, rows].float()
            p = torch.matmul(Q, K.transpose(1, 2).contiguous())
            p *= scale
            if c["unit"]:
                pos = nk - nq + at + torch.arange(n, device="cuda")
                seen = (torch.div(pos, c["unit"], rounding_mode="floor") + 1) * c["unit"]
                p.masked_fill_(torch.arange(nk, device="cuda") >= seen[:, None], -math.inf)
            top = p.amax(-1, keepdim=True)
            p -= torch.where(top == -math.inf, torch.zeros_like(top), top)
            p.exp_()
            total = p.sum(-1, keepdim=True)
            p /= torch.where(total == 0.0, torch.ones_like(total), total)
            out["O"][:, rows] = torch.matmul(p, V).to(torch.bfloat16)
            if not train:
                continue
            dO = s["dO"][:, rows].float()
            dp = torch.matmul(dO, V.transpose(1, 2).contiguous())
            dp -= (dp * p).sum(-1, keepdim=True)
            dv = torch.matmul(p.transpose(1, 2).contiguous(), dO)
            dp *= p
            del p
            out["dQ"][:, rows] = (torch.matmul(dp, K) * scale).to(torch.bfloat16)
            dk = torch.matmul(dp.transpose(1, 2).contiguous(), Q) * scale
            for name, t in (("dK", dk), ("dV", dv)):
                out[name][:, k0:k0 + nk] += t.view(Hk, G, nk, d).sum(1)
        q0, k0 = q0 + nq, k0 + nk
    if train:
        out["dK"], out["dV"] = out["dK"].to(torch.bfloat16), out["dV"].to(torch.bfloat16)
    return out


def _plain_clip(s):
    c = s["case"]
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for x in s["grads"]:
        f = x.float()
        total += (f * f).sum(dtype=torch.float64)
    norm = torch.sqrt(total)
    by = torch.where(torch.isfinite(norm), (c["most"] / (norm + EPS)).clamp(max=1.0), torch.ones_like(norm)).float()
    to = s["grads"] if s["out"] is None else s["out"]
    for x, y in zip(s["grads"], to):
        y.copy_((x.float() * by).to(y.dtype))
    return {"norm": norm.float().view(1), "grads": list(s["flat"].values())}


def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(s, c)
    return {"norm": _plain_norm, "attn": _plain_attn, "clip": _plain_clip}[c["op"]](s)


def _run_own(s, c):
    from paper_2602_04789_amd import lf

    def buffer(name, need):   # what a program keeps between its calls
        if name not in s:
            s[name] = torch.empty(max(need(), 256), dtype=torch.uint8, device="cuda")
        return s[name]

    if c["op"] == "clip":
        ws = buffer("ws", lambda: lf.lf_grad_workspace_bytes(len(s["grads"]), sum(x.numel() for x in s["grads"])))
        norm = lf.lf_grad_clip(s["grads"], c["most"], out=s["out"], eps=EPS, workspace=ws)
        return {"norm": norm, "grads": list(s["flat"].values())}
    if c["op"] == "norm":
        how = dict(B=s["B"], gate=s["gate"], post_weight=s["post"], weight=s["weight"], scale=s["scale"], group_len=s["group_len"],
                   starts=s["starts"], kind=lf.LF_NORM_LAYER if c["kind"] == "layer" else lf.LF_NORM_RMS, eps=EPS)
        X, Y = lf.lf_gate_norm(s["X"], shift=s["shift"], Xout=s["Xout"], Y=s["Y"], **how)
        out = {"Xout": X, "Y": Y} if c["block"] else {"Y": Y}
        if c["train"]:
            rows, G = s["X"].shape[0], len(s["lengths"])
            ws = buffer("ws", lambda: lf.lf_gate_norm_bwd_workspace_bytes(rows, c["width"], G, s["group_len"]))
            got = lf.lf_gate_norm_bwd(X, s["dY"], dXout=s["dXout"], dX=s["dX"], dB=s["dB"], workspace=ws, **how)
            names = ("dX", "dB", "dgate", "dpost", "dweight", "dscale", "dshift")
            out.update((k, t) for k, t in zip(names, got) if t is not None)
        return out
    how = dict(causal=c["unit"])
    shape = (c["heads"], c["kv_heads"], c["head_dim"], c["seqs"], s["Q"].shape[1], s["K"].shape[1], c["unit"])
    ws = buffer("ws", lambda: lf.lf_packed_attn_workspace_bytes(*shape))
    if not c["train"]:
        return {"O": lf.lf_packed_attn(s["Q"], s["K"], s["V"], s["q_start"], s["kv_start"], O=s["O"], workspace=ws, **how)}
    O, lse2 = lf.lf_packed_attn_fwd(s["Q"], s["K"], s["V"], s["q_start"], s["kv_start"], O=s["O"], workspace=ws, **how)
    wsb = buffer("wsb", lambda: lf.lf_packed_attn_bwd_workspace_bytes(*shape))
    dQ, dK, dV = lf.lf_packed_attn_bwd(s["Q"], s["K"], s["V"], O, s["dO"], lse2, s["q_start"], s["kv_start"], grads=s["grads"],
                                       workspace=wsb, **how)
    return {"O": O, "dQ": dQ, "dK": dK, "dV": dV}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "attn": _exact_attn, "clip": _exact_clip}[case["op"]](s, case)


def _exact_norm(s, c):
    """Group by group, the gradients by differentiation in 64 bits."""
    keys = ["Y"] + (["Xout"] if c["block"] else [])
    out = {k: torch.zeros(s["X"].shape, dtype=torch.float64, device="cuda") for k in keys}
    G, C, train = len(s["lengths"]), c["width"], c["train"]
    if train:
        out["dX"] = torch.zeros_like(out["Y"])
        for k in ("dscale", "dshift") + (("dgate",) if c["block"] else ()):
            out[k] = torch.zeros((G, C), dtype=torch.float64, device="cuda")
        for k, there in (("dweight", s["weight"] is not None), ("dpost", c["post"])):
            if there:
                out[k] = torch.zeros(C, dtype=torch.float64, device="cuda")
        if c["block"]:
            out["dB"] = torch.zeros_like(out["Y"])
    first = 0
    for g, length in enumerate(s["lengths"]):
        for at in range(first, first + length, 4096):
            r = slice(at, min(at + 4096, first + length))

            def leaf(t):
                return t.double().requires_grad_(train) if t is not None else None

            x, sc, sh = leaf(s["X"][r]), leaf(s["scale"][g]), leaf(s["shift"][g])
            b, gate = (leaf(s["B"][r]), leaf(s["gate"][g])) if c["block"] else (None, None)
            w, post = leaf(s["weight"]), leaf(s["post"])
            with torch.set_grad_enabled(train):
                xo = x
                if b is not None:
                    p = b
                    if post is not None:
                        p = b * torch.rsqrt(b.square().sum(1, keepdim=True) / C + EPS) * post
                    xo = x + p * gate
                    # the norm is that of the stream as it is written
                    xo = xo + (xo.detach().to(s["X"].dtype).double() - xo.detach())
                if c["kind"] == "layer":
                    var, mean = torch.var_mean(xo, 1, unbiased=False, keepdim=True)
                    n = (xo - mean) / (var + EPS).sqrt()
                else:
                    n = xo / (xo.square().sum(1, keepdim=True) / C + EPS).sqrt()
                y = n * ((1 + sc) if w is None else (1 + sc) * w) + sh
            out["Y"][r] = y.detach()
            if b is not None:
                out["Xout"][r] = xo.detach()
            if not train:
                continue
            leaves = [(k, t) for k, t in (("dX", x), ("dscale", sc), ("dshift", sh), ("dB", b), ("dgate", gate), ("dweight", w),
                                          ("dpost", post)) if t is not None]
            got = torch.autograd.grad((y, xo), [t for _, t in leaves], (s["dY"][r].double(), s["dXout"][r].double()))
            for (k, _), t in zip(leaves, got):
                if k in ("dX", "dB"):
                    out[k][r] = t
                elif k in ("dweight", "dpost"):
                    out[k] += t
                else:
                    out[k][g] += t
        first += length
    return out


def _exact_attn(s, c):
    H, Hk, d, train = c["heads"], c["kv_heads"], c["head_dim"], c["train"]
    out = {"O": torch.zeros(s["O"].shape, dtype=torch.float64, device="cuda")}
    if train:
        out.update((name, torch.zeros(s[k].shape, dtype=torch.float64, device="cuda")) for name, k in (("dQ", "Q"), ("dK", "K"), ("dV", "V")))
    q_at, k_at = _starts(s["lengths"][0]), _starts(s["lengths"][1])
    for h in range(H):
        hk = h * Hk // H
        for b in range(c["seqs"]):
            nq, nk = q_at[b + 1] - q_at[b], k_at[b + 1] - k_at[b]
            i = 0
            while i < nq:        # rows that see the same tokens, or a square of rows and tokens
                many = max(1, min(nq - i, (1 << 26) // max(nk, 1)))
                sees = [_seen(c, nq, nk, i + j) for j in (0, many - 1)]
                n = sees[1]
                rows, cols = slice(q_at[b] + i, q_at[b] + i + many), slice(k_at[b], k_at[b] + n)
                first, i = i, i + many
                if n == 0:
                    continue
                leaf = [t.double().requires_grad_(train) for t in (s["Q"][h, rows], s["K"][hk, cols], s["V"][hk, cols])]
                with torch.set_grad_enabled(train):
                    z = leaf[0] @ leaf[1].T / d ** 0.5
                    if sees[0] != sees[1]:
                        limit = torch.tensor([_seen(c, nq, nk, first + j) for j in range(many)], device="cuda")
                        z = z.masked_fill(torch.arange(n, device="cuda")[None] >= limit[:, None], -1e300)
                        o = (torch.softmax(z, -1) @ leaf[2]) * (limit > 0).double()[:, None]
                    else:
                        o = torch.softmax(z, -1) @ leaf[2]
                out["O"][h, rows] = o.detach()
                if train:
                    gq, gk, gv = torch.autograd.grad(o, leaf, s["dO"][h, rows].double())
                    out["dQ"][h, rows] = gq
                    out["dK"][hk, cols] += gk
                    out["dV"][hk, cols] += gv
    return out


def _exact_clip(s, c):
    squares = [torch.linalg.vector_norm(x.double()).square() for x in s["grads"]]
    norm = torch.stack(squares).sum().sqrt()
    by = min(1.0, c["most"] / (norm.item() + EPS)) if math.isfinite(norm.item()) else 1.0
    grads = [torch.cat([x.flatten() for x in s["grads"] if x.element_size() == size]).double() * by for size in s["flat"]]
    return {"norm": norm.view(1), "grads": grads}
