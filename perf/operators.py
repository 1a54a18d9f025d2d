"""Timed operators of a long rollout, in their plain form and as calls of ``paper_2602_04789_amd.lf``.

A video generator that keeps a long history makes, beside the sparse attention itself, these calls:

  rope   RMSNorm and rotary positions over three axes (time, height, width) of a projection's output, written
         head-major as the attention reads it; with ``train`` the gradients too
  store  keys and values of finished frames go into the cache in 4 bits (e2m1 values, one power of two for 32 channels of
         a token) and come back from it in bfloat16
  chunk  blockwise sparse attention of one chunk over that cache
  token  attention of a few query rows over every token of that cache

The cache is one buffer: codes of K [H][capacity][d/2], codes of V, scales of K [H][capacity][d/32], scales of V, each part
padded to 256 bytes.  Channel 2i is in the low half of byte i.
"""
import math

import torch

own = False

BLOCK = 64
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
# a value next to a border goes to the code that is even
BORDERS = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))


def _rope(name, tokens, heads, head_dim, across, pairing, far, train):
    c = dict(op="rope", tokens=tokens, heads=heads, head_dim=head_dim, across=across, pairing=pairing, far=far, train=train)
    return dict(c, name=name) if name else c


def _store(name, tokens, heads, head_dim, capacity, first):
    c = dict(op="store", tokens=tokens, heads=heads, head_dim=head_dim, capacity=capacity, first=first)
    return dict(c, name=name) if name else c


def _chunk(name, heads, head_dim, frame_len, per_chunk, chunk, kept, own_tokens):
    c = dict(op="chunk", heads=heads, head_dim=head_dim, frame_len=frame_len, per_chunk=per_chunk, chunk=chunk, kept=kept,
             own_tokens=own_tokens)
    return dict(c, name=name) if name else c


def _token(name, heads, head_dim, rows, cached, extra):
    c = dict(op="token", heads=heads, head_dim=head_dim, rows=rows, cached=cached, extra=extra)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token's queries: latency alone counts
        _rope("rope_one_token", 1, 12, 128, False, 0, 1 << 20, False),
        # the queries of one chunk of the benchmark's rollout: three frames of 30 x 52 tokens
        _rope("rope_chunk", 4680, 12, 128, True, 0, 21, False),
        # finetuning, a packed batch of images of odd sizes with few heads, positions far out
        _rope("rope_train_ragged", 1333, 5, 64, False, 1, 100000, True),
        # finetuning, one chunk of the 12-head model
        _rope("rope_train_chunk", 4680, 12, 128, True, 0, 21, True),
        # finetuning, a whole video of the 40-head model at once
        _rope("rope_train_video", 32760, 40, 128, True, 0, 21, True),
        # one token goes into the cache
        _store("store_one_token", 1, 12, 128, 32760, 4681),
        # a finished chunk goes into the cache
        _store("store_chunk", 4680, 12, 128, 32760, 28080),
        # a small rollout, everything in the cache: few query blocks
        _chunk("chunk_small", 2, 64, 256, 1, 5, 0.5, False),
        # the last chunk of the benchmark's rollout, its own tokens still in bfloat16
        _chunk("chunk_last", 12, 128, 1560, 3, 7, 0.25, True),
        # one query row over a short cache
        _token("token_short", 12, 128, 1, 77, 1),
        # one query row over a long one
        _token("token_long", 12, 128, 1, 131075, 1),
        # a block of query rows, 40 narrow heads, over a cache of a rollout's length
        _token("token_rows", 40, 64, 64, 32760, 64),
    ]


_MOST = {}


def _pairs(c):
    """Scores that the plain form of the attention lays out."""
    if c["op"] == "token":
        return c["heads"] * c["rows"] * (c["cached"] + c["extra"])
    if c["op"] == "chunk":
        q = c["frame_len"] * c["per_chunk"]
        return c["heads"] * q * q * c["chunk"]
    return 0


def _most():
    if not _MOST:
        for c in listed():
            w = dict(work(c), pairs=_pairs(c))
            most = _MOST.setdefault(c["op"], w)
            _MOST[c["op"]] = {k: max(v, most[k]) for k, v in w.items()}
    return _MOST


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["rope", "rope", "store", "chunk", "chunk", "token", "token"])
        heads, head_dim = _log(rng, 1, 40), rng.choice([64, 128, 128])
        if op == "rope":
            c = _rope(None, _log(rng, 1, 32760), heads, head_dim, rng.random() < 0.5, rng.randint(0, 1),
                      _log(rng, 8, 1 << 20), rng.random() < 0.6)
        elif op == "store":
            tokens = _log(rng, 1, 6000)
            first = rng.choice([0, _log(rng, 1, 40000)])
            c = _store(None, tokens, heads, head_dim, first + tokens + _log(rng, 1, 3000) - 1, first)
        elif op == "chunk":
            frame_len = rng.choice([_log(rng, 1, 1600), _log(rng, 48, 1600), 1560, 64 * _log(rng, 1, 24)])
            c = _chunk(None, heads, head_dim, frame_len, rng.randint(1, 3), rng.randint(1, 7), round(rng.uniform(0.1, 1.0), 3),
                       rng.random() < 0.6)
        else:
            rows, extra = _log(rng, 1, 64), rng.choice([0, 1, rng.randint(1, 100)])
            c = _token(None, heads, head_dim, rows, _log(rng, 1, 131075), extra)
        most, w = _most()[op], dict(work(c), pairs=_pairs(c))
        if all(w[k] <= most[k] for k in w):
            return c


def _part(n):
    return -(-n // 256) * 256


def _parts(heads, capacity, d):
    """Where the four parts of a cache begin, and its size."""
    codes, scales = _part(heads * capacity * d // 2), _part(heads * capacity * d // 32)
    return (0, codes, 2 * codes, 2 * codes + scales), 2 * (codes + scales)


def _lists(c):
    """Query blocks, KV blocks of the history, all KV blocks and the length of a list."""
    nb = -(-c["frame_len"] // BLOCK)
    n_q, n_h = c["per_chunk"] * nb, (c["chunk"] - 1) * c["per_chunk"] * nb
    keep = max(1, math.ceil(c["kept"] * n_h)) if n_h else 0
    return n_q, n_h, n_h + n_q, keep + n_q


def work(case):
    c, H, d = case, case["heads"], case["head_dim"]
    if c["op"] == "rope":
        n = c["tokens"] * H * d
        small = 4.0 * H * d + 12.0 * c["tokens"] + 4.0 * d
        if c["train"]:   # X and dY are read, Y and dX written, and the norm's weight has a gradient
            return {"bytes": 8.0 * n + small + 4.0 * H * d, "flops": 30.0 * n}
        return {"bytes": 4.0 * n + small, "flops": 10.0 * n}
    bits = d / 2 + d / 32    # bytes of a token's keys or values in the cache
    if c["op"] == "store":
        rows = 2.0 * c["tokens"] * H
        return {"bytes": rows * (4 * d + bits), "flops": 4 * rows * d}
    if c["op"] == "token":
        rows, cached, extra = c["rows"], c["cached"], c["extra"]
        return {"bytes": H * (4.0 * rows * d + 2 * cached * bits + 4.0 * extra * d), "flops": 4.0 * H * rows * (cached + extra) * d}
    n, f, chunk = c["frame_len"], c["per_chunk"], c["chunk"]
    n_q, n_h, n_k, kept = _lists(c)
    q, hist = f * n, (chunk - 1) * f * n
    held = hist if c["own_tokens"] else hist + q
    pairs = H * q * kept * (n / (n_q / f))
    return {"bytes": H * (4.0 * q * d + 2 * held * bits + (4.0 * q * d if c["own_tokens"] else 0.0)) + 4.0 * H * n_q * kept,
            "flops": 4.0 * pairs * d}


def _quantise(x):
    """Codes [.., d/2] and scales [.., d/32] of bfloat16 values: per 32 channels the smallest power of two by which the
    largest value is at most 7 (which goes to 6, the largest code), at least 2^-126; byte 255 where a value is not finite."""
    v = x.float().unflatten(-1, (-1, 32))
    top = v.abs().amax(-1, keepdim=True)
    fine = torch.isfinite(top)
    m, e = torch.frexp(torch.where(fine, top, torch.zeros_like(top)))
    e = torch.where(m > 0.875, e - 2, e - 3).clamp(min=-126)
    v = torch.where(fine, torch.ldexp(v, -e), torch.zeros_like(v))
    a = v.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    for at, up in BORDERS:
        code += (a >= at) if up else (a > at)
    code += 8 * torch.signbit(v).to(torch.uint8)
    code = code.flatten(-2)
    scale = torch.where(fine, e + 127, torch.full_like(e, 255)).to(torch.uint8).squeeze(-1)
    return code[..., 0::2] | (code[..., 1::2] << 4), scale


def _write(cache, heads, capacity, d, first, K, V):
    """Lays K and V [H, L, d] into the cache at the tokens from `first` on."""
    at, _ = _parts(heads, capacity, d)
    last = first + K.shape[1]
    for i, x in enumerate((K, V)):
        code, scale = _quantise(x)
        cache[at[i]:at[i] + heads * capacity * d // 2].view(heads, capacity, d // 2)[:, first:last] = code
        cache[at[2 + i]:at[2 + i] + heads * capacity * d // 32].view(heads, capacity, d // 32)[:, first:last] = scale


def _read(cache, heads, capacity, d, first, last):
    """K and V [H, last - first, d] in float32, as the cache holds them."""
    at, _ = _parts(heads, capacity, d)
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=cache.device)
    got = []
    for i in range(2):
        code = cache[at[i]:at[i] + heads * capacity * d // 2].view(heads, capacity, d // 2)[:, first:last]
        scale = cache[at[2 + i]:at[2 + i] + heads * capacity * d // 32].view(heads, capacity, d // 32)[:, first:last]
        v = grid[torch.stack((code & 15, code >> 4), -1).flatten(-2).int()].unflatten(-1, (-1, 32))
        v = torch.ldexp(v, scale.int().unsqueeze(-1) - 127)
        got.append(torch.where((scale == 255).unsqueeze(-1), torch.full_like(v, math.nan), v).flatten(-2))
    return got


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _keys(g, heads, tokens, d):
    """Unit normal keys; a few channels of every head are larger, as projections leave them."""
    wide = 1.0 + 3.0 * (torch.rand((heads, 1, d), generator=g, device="cuda") < 0.04).float()
    return (_randn(g, heads, tokens, d) * wide).to(torch.bfloat16)


def _axes(d):
    side = 2 * (d // 6)
    return (d - 2 * side) // 2, side // 2, side // 2


def prepare(case, seed):
    c, H, d = case, case["heads"], case["head_dim"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if c["op"] == "rope":
        L = c["tokens"]
        axes = _axes(d)
        freq = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64) / n) for n in axes]).cuda()
        # frames of 30 x 52 tokens, from a frame on that the seed gives
        l = torch.arange(L, device="cuda")
        t0 = torch.randint(0, c["far"], (1,), generator=g, device="cuda")
        pos = torch.stack((t0 + l // 1560, l // 52 % 30, l % 52), 1).to(torch.int32).contiguous()
        s = dict(X=_randn(g, L, H * d).to(torch.bfloat16), g=1.0 + 0.1 * _randn(g, H * d), pos=pos, freq=freq, axes=axes,
                 Y=torch.empty((H, L, d), dtype=torch.bfloat16, device="cuda"))
        if c["train"]:
            s["dY"] = _randn(g, H, L, d).to(torch.bfloat16)
        return dict(s, case=dict(c))
    if c["op"] == "store":
        L, cap = c["tokens"], c["capacity"]
        return dict(K=_keys(g, H, L, d), V=_randn(g, H, L, d).to(torch.bfloat16), case=dict(c),
                    cache=torch.zeros(_parts(H, cap, d)[1], dtype=torch.uint8, device="cuda"))
    if c["op"] == "token":
        held, more, q = c["cached"], c["extra"], c["rows"]
    else:
        q = c["frame_len"] * c["per_chunk"]
        hist = (c["chunk"] - 1) * q
        held, more = (hist, q) if c["own_tokens"] else (hist + q, 0)
    capacity = held + 5
    cache = torch.zeros(_parts(H, capacity, d)[1], dtype=torch.uint8, device="cuda")
    if held:
        step = max(1, (1 << 26) // (H * d))
        for at in range(0, held, step):
            n = min(step, held - at)
            _write(cache, H, capacity, d, at, _keys(g, H, n, d), _randn(g, H, n, d).to(torch.bfloat16))
    s = dict(Q=_randn(g, H, q, d).to(torch.bfloat16), cache=cache, capacity=capacity, held=held, case=dict(c), K=None, V=None,
             O=torch.empty((H, q, d), dtype=torch.bfloat16, device="cuda"))
    if more:
        s.update(K=_keys(g, H, more, d), V=_randn(g, H, more, d).to(torch.bfloat16))
    if c["op"] == "chunk":
        n_q, n_h, n_k, kept = _lists(c)
        own_blocks = torch.arange(n_h, n_k, device="cuda", dtype=torch.int32).expand(H, n_q, n_q)
        if n_h:   # history blocks by a score that leans to some frames, as the mask selection's do
            score = _randn(g, H, n_q, n_h) + _randn(g, H, 1, n_h // (n_q // c["per_chunk"])).repeat_interleave(n_q // c["per_chunk"], -1)
            picked = score.topk(kept - n_q, dim=-1).indices.sort(-1).values.to(torch.int32)
            s["lists"] = torch.cat((picked, own_blocks), -1).contiguous()
        else:
            s["lists"] = own_blocks.contiguous()
    return s


def _turn(y, cos, sin, pairing):
    """Channel pairs of y [L, H, d] turned by the angles of their token."""
    half = y.shape[-1] // 2
    a, b = (y[..., 0::2], y[..., 1::2]) if pairing == 0 else (y[..., :half], y[..., half:])
    p, q = a * cos - b * sin, a * sin + b * cos
    return torch.stack((p, q), -1).flatten(-2) if pairing == 0 else torch.cat((p, q), -1)


def _plain_rope(s):
    c = s["case"]
    H, d, L = c["heads"], c["head_dim"], c["tokens"]
    axis = torch.repeat_interleave(torch.arange(3, device="cuda"), torch.tensor(s["axes"], device="cuda"), output_size=d // 2)
    angle = s["pos"].double()[:, axis] * s["freq"]
    cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    over = (1, 2) if c["across"] else (2,)
    x, g = s["X"].float().view(L, H, d), s["g"].view(H, d)
    inv = 1.0 / torch.sqrt((x * x).mean(over, keepdim=True) + 1e-6)
    n = x * inv
    y = _turn(n * g, cos, sin, c["pairing"]).transpose(0, 1).to(torch.bfloat16).contiguous()
    if not c["train"]:
        return y
    back = _turn(s["dY"].transpose(0, 1).float(), cos, -sin, c["pairing"])
    u = back * g
    dX = inv * (u - n * (u * n).mean(over, keepdim=True))
    return {"Y": y, "dX": dX.to(torch.bfloat16).view(L, H * d), "dg": (back * n).sum(0).view(H * d)}


def _plain_attention(s, seen):
    """Rows of softmax(Q K^T / sqrt(d)) V over the tokens of the cache and those after it; `seen`: [H, q, tokens] or None."""
    c = s["case"]
    K, V = _read(s["cache"], c["heads"], s["capacity"], c["head_dim"], 0, s["held"])
    if s["K"] is not None:
        K, V = torch.cat((K, s["K"].float()), 1), torch.cat((V, s["V"].float()), 1)
    p = torch.matmul(s["Q"].float(), K.transpose(1, 2).contiguous())
    p *= 1.0 / math.sqrt(c["head_dim"])
    if seen is not None:
        p.masked_fill_(~seen, -math.inf)
    p -= p.amax(-1, keepdim=True)
    p.exp_()
    return (torch.matmul(p, V) / p.sum(-1, keepdim=True)).to(torch.bfloat16)


def _seen(s):
    """Which token a query row sees, from the lists: [H, q, tokens]."""
    c = s["case"]
    n, nb = c["frame_len"], -(-c["frame_len"] // BLOCK)
    n_q, _, n_k, _ = _lists(c)
    kept = torch.zeros((c["heads"], n_q, n_k), dtype=torch.bool, device="cuda").scatter_(2, s["lists"].long(), True)
    token = torch.arange(n, device="cuda") // BLOCK
    rows = (torch.arange(n_q // nb, device="cuda")[:, None] * nb + token).flatten()
    cols = (torch.arange(n_k // nb, device="cuda")[:, None] * nb + token).flatten()
    return kept[:, rows][:, :, cols]


def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(s, c)
    if c["op"] == "rope":
        return _plain_rope(s)
    if c["op"] == "store":
        H, d = c["heads"], c["head_dim"]
        _write(s["cache"], H, c["capacity"], d, c["first"], s["K"], s["V"])
        K, V = _read(s["cache"], H, c["capacity"], d, c["first"], c["first"] + c["tokens"])
        return {"K": K.to(torch.bfloat16), "V": V.to(torch.bfloat16)}
    return _plain_attention(s, _seen(s) if c["op"] == "chunk" else None)


def _run_own(s, c):
    from paper_2602_04789_amd import lf

    def buffer(name, need):   # what a program keeps between its calls
        if name not in s:
            s[name] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
        return s[name]

    H, d = c["heads"], c["head_dim"]
    if c["op"] == "rope":
        how = dict(across_heads=c["across"], pairing=c["pairing"])
        Y = lf.lf_qk_norm_rope_axes(s["X"], s["g"], s["pos"], s["freq"], s["axes"], H, s["Y"], **how)
        if not c["train"]:
            return Y
        if "ws" not in s:
            buffer("ws", lf.lf_qk_norm_rope_axes_bwd_workspace_bytes(H, d, c["tokens"]))
        dX, dg = lf.lf_qk_norm_rope_axes_bwd(s["X"], s["g"], s["pos"], s["freq"], s["axes"], H, s["dY"], workspace=s["ws"], **how)
        return {"Y": Y, "dX": dX, "dg": dg}
    if c["op"] == "store":
        lf.lf_kvq_append(s["K"], s["V"], s["cache"], c["capacity"], c["first"])
        K, V = lf.lf_kvq_read(s["cache"], H, d, c["capacity"], c["first"], c["tokens"])
        return {"K": K, "V": V}
    if c["op"] == "token":
        if "ws" not in s:
            buffer("ws", lf.lf_token_attn_kvq_workspace_bytes(H, d, c["rows"], c["cached"], c["extra"]))
        return lf.lf_token_attn_kvq(s["Q"], s["cache"], s["capacity"], s["held"], K=s["K"], V=s["V"], O=s["O"], workspace=s["ws"])
    kv_len = c["frame_len"] * c["per_chunk"] * c["chunk"]
    if "ws" not in s:
        buffer("ws", lf.lf_sparse_attn_kvq_workspace_bytes(H, d, c["frame_len"], BLOCK, s["Q"].shape[1], kv_len, s["lists"].shape[2]))
    return lf.lf_sparse_attn_kvq(s["Q"], s["cache"], s["capacity"], kv_len, s["lists"], c["frame_len"], BLOCK, K=s["K"], V=s["V"],
                                 O=s["O"], workspace=s["ws"])


def exact(case, seed):
    s, c = prepare(case, seed), case
    H, d = c["heads"], c["head_dim"]
    if c["op"] == "rope":
        return _exact_rope(s, c)
    if c["op"] == "store":
        got = {}
        for name in ("K", "V"):   # every group of 32 on the grid of its own step
            x = s[name].double().reshape(-1, 32)
            top = x.abs().max(1, keepdim=True).values
            e = torch.ceil(torch.log2(top / 7.0 + 2.0 ** -200)).clamp(min=-126.0)
            e = torch.where(top <= 7.0 * 2.0 ** (e - 1), (e - 1).clamp(min=-126.0), e)
            z = x / 2.0 ** e
            a = z.abs()
            step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
            got[name] = (torch.copysign(torch.clamp(torch.round(a / step) * step, max=6.0), z) * 2.0 ** e).reshape(H, c["tokens"], d)
        return got
    out = torch.empty_like(s["Q"], dtype=torch.float64)
    at, _ = _parts(H, s["capacity"], d)
    for h in range(H):
        K, V = (_exact_held(s, c, h, at[i], at[2 + i]) for i in range(2))
        if s["K"] is not None:
            K, V = torch.cat((K, s["K"][h].double())), torch.cat((V, s["V"][h].double()))
        if c["op"] == "token":
            out[h] = torch.softmax(s["Q"][h].double() @ K.T / d ** 0.5, -1) @ V
            continue
        n, nb = c["frame_len"], -(-c["frame_len"] // BLOCK)
        for r in range(s["lists"].shape[1]):
            first, last = r // nb * n + r % nb * BLOCK, r // nb * n + min(n, (r % nb + 1) * BLOCK)
            ids = s["lists"][h, r].long()
            begin = ids // nb * n + ids % nb * BLOCK
            at_token = begin[:, None] + torch.arange(BLOCK, device="cuda")
            there = (ids % nb * BLOCK)[:, None] + torch.arange(BLOCK, device="cuda") < n
            t = at_token[there]
            out[h, first:last] = torch.softmax(s["Q"][h, first:last].double() @ K[t].T / d ** 0.5, -1) @ V[t]
    return out


def _exact_held(s, c, h, code_at, scale_at):
    """What the cache holds for head h, [held, d] in float64."""
    d, cap, held = c["head_dim"], s["capacity"], s["held"]
    b = s["cache"][code_at + h * cap * d // 2:][:held * d // 2].int()
    nibble = torch.empty(held * d, dtype=torch.int32, device="cuda")
    nibble[0::2], nibble[1::2] = b % 16, b // 16
    sign, ee, m = 1.0 - 2.0 * (nibble // 8).double(), (nibble // 2 % 4).double(), (nibble % 2).double()
    v = sign * torch.where(ee == 0, 0.5 * m, (1.0 + 0.5 * m) * 2.0 ** (ee - 1))
    e = s["cache"][scale_at + h * cap * d // 32:][:held * d // 32].double() - 127.0
    return (v.view(-1, 32) * 2.0 ** e[:, None]).view(held, d)


def _exact_rope(s, c):
    H, d, L = c["heads"], c["head_dim"], c["tokens"]
    dX = torch.empty((L, H * d), dtype=torch.float64, device="cuda")
    Y = torch.empty((H, L, d), dtype=torch.float64, device="cuda")
    dg = torch.zeros(H * d, dtype=torch.float64, device="cuda")
    where = [a for a in range(3) for _ in range(s["axes"][a])]
    for first in range(0, L, 2048):
        l = slice(first, min(L, first + 2048))
        theta = s["pos"][l].double()[:, where] * s["freq"]
        turn = torch.polar(torch.ones_like(theta), theta)[:, None]
        x = s["X"][l].double()
        rows = x if c["across"] else x.reshape(-1, d)
        r = torch.sqrt(rows.square().sum(1) / rows.shape[1] + 1e-6).view(len(x), -1)
        r = r.expand(-1, H) if c["across"] else r
        n = x.view(-1, H, d) / r[..., None]
        w = s["g"].double().view(H, d)

        def pairs(v):
            return torch.complex(v[..., 0::2], v[..., 1::2]) if c["pairing"] == 0 else torch.complex(v[..., :d // 2], v[..., d // 2:])

        def channels(z):
            return torch.view_as_real(z).flatten(-2) if c["pairing"] == 0 else torch.cat((z.real, z.imag), -1)

        Y[:, l] = channels(pairs(n * w) * turn).transpose(0, 1)
        if c["train"]:
            back = channels(pairs(s["dY"][:, l].transpose(0, 1).double()) * turn.conj())
            dg += (back * n).sum(0).flatten()
            u = back * w
            # the gradient of x / r at a fixed r, and through r
            dot = (u * x.view(-1, H, d)).sum(-1)
            dot, N = (dot.sum(1, keepdim=True), H * d) if c["across"] else (dot, d)
            dX[l] = (u / r[..., None] - x.view(-1, H, d) * (dot / (N * r ** 3))[..., None]).flatten(1)
    return {"Y": Y, "dX": dX, "dg": dg} if c["train"] else Y
