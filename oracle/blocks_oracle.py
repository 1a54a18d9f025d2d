"""Binary64 definitions of the calls around the attention: the norm between two blocks with its gradients, attention over packed sequences with its
gradients, clipping to a largest norm.  Test infrastructure only; numpy, no code of the package."""
import numpy as np


def groups_of(tokens, group_len=0, starts=None):
    """Group of every token, -1 for tokens of none."""
    at = np.arange(tokens)
    if group_len > 0:
        return at // group_len
    g = np.searchsorted(np.asarray(starts), at, side="right") - 1
    # an empty group before the token's own does not hold it; tokens behind the last group belong to none
    return np.where((at < starts[0]) | (at >= starts[-1]), -1, g)


def _norm(x, eps, layer):
    mean = x.mean(1, keepdims=True) if layer else np.zeros((len(x), 1))
    z = x - mean
    inv = 1.0 / np.sqrt((z * z).mean(1, keepdims=True) + eps)
    return z * inv, mean, inv


def _factor(C, groups, weight, scale, g):
    f = np.ones((1, C)) if scale is None else 1.0 + scale[g]
    return f if weight is None else f * weight


def gate(X, B, g, gate, post_weight, eps, rs):
    """The stream behind a block, before it is rounded."""
    p = B
    if post_weight is not None:
        p = B / np.sqrt((B * B).mean(1, keepdims=True) + eps) * post_weight
    return X + rs * (1.0 if gate is None else gate[g]) * p


def norm(Xout, g, weight, scale, shift, eps, layer):
    n, _, _ = _norm(Xout, eps, layer)
    y = n * _factor(Xout.shape[1], None, weight, scale, g)
    return y if shift is None else y + shift[g]


def gate_norm_backward(Xout, B, g, groups, gate, post_weight, weight, scale, eps, rs, layer, dY, dXout):
    """{name: gradient} and {name: size of the terms that its float32 form adds up}, the latter for error bars."""
    L, C = Xout.shape
    n, mean, inv = _norm(Xout, eps, layer)
    f = _factor(C, groups, weight, scale, g)
    u = dY * f
    mu = u.mean(1, keepdims=True) if layer else 0.0
    D = dXout + inv * (u - mu - n * (u * n).mean(1, keepdims=True))
    sn = (np.abs(Xout) + np.abs(mean) + np.abs(Xout).mean(1, keepdims=True)) * inv + np.abs(n)
    au = np.abs(u)
    sD = np.abs(dXout) + inv * (au + au.mean(1, keepdims=True) + sn * (au * np.abs(n)).mean(1, keepdims=True)
                                + np.abs(n) * (au * sn).mean(1, keepdims=True))
    one = np.zeros((groups, L))
    one[g[g >= 0], np.nonzero(g >= 0)[0]] = 1.0
    w = np.ones(C) if weight is None else weight
    sc = np.ones((groups, C)) if scale is None else 1.0 + scale
    S, sS = one @ (dY * n), one @ (np.abs(dY) * sn)
    out = dict(dX=D, dscale=S * w, dshift=one @ dY, dweight=(sc * S).sum(0))
    size = dict(dX=sD, dscale=sS * np.abs(w), dshift=one @ np.abs(dY), dweight=(np.abs(sc) * sS).sum(0))
    if B is not None:
        ga = rs * (np.ones((L, 1)) if gate is None else gate[g])
        rb = 1.0 / np.sqrt((B * B).mean(1, keepdims=True) + eps) if post_weight is not None else 1.0
        bn = B * rb
        pw = np.ones(C) if post_weight is None else post_weight
        e, se = ga * D * pw, np.abs(ga) * sD * np.abs(pw)
        if post_weight is not None:
            out["dB"] = rb * (e - bn * (e * bn).mean(1, keepdims=True))
            size["dB"] = rb * (se + np.abs(bn) * (se * np.abs(bn)).mean(1, keepdims=True))
        else:
            out["dB"], size["dB"] = e, se
        T, sT = rs * (one @ (bn * D)), abs(rs) * (one @ (np.abs(bn) * sD))
        gt = np.ones((groups, C)) if gate is None else gate
        out.update(dgate=T * pw, dpost_weight=(gt * T).sum(0))
        size.update(dgate=sT * np.abs(pw), dpost_weight=(np.abs(gt) * sT).sum(0))
    return out, size


def seen(nq, nk, causal, i):
    """How many of its sequence's nk tokens row i of nq sees."""
    if causal == 0:
        return nk
    return max(0, min(nk, ((nk - nq + i) // causal + 1) * causal))


def packed_attention(Q, K, V, q_start, kv_start, causal, scale, dO=None):
    """O [H, L, d] and lse2 [H, L] (log2 of the sum of exponentials, +inf for a row that sees nothing); rows of no sequence are NaN.  With dO also dQ, dK
    and dV and, for each of the four, the size that its error is measured against: sums of absolute values, with a dS that is off by P times
    what the rounding of O leaves in delta and by its own rounding, in units of 2^-8."""
    H, Hk, d = Q.shape[0], K.shape[0], Q.shape[2]
    G = H // Hk
    O, lse2 = np.full(Q.shape, np.nan), np.full(Q.shape[:2], np.nan)
    sO = np.full(Q.shape, np.nan)
    dQ, sQ = np.full(Q.shape, np.nan), np.full(Q.shape, np.nan)
    dK, sK, dV, sV = (np.full(K.shape, np.nan) for _ in range(4))
    for b in range(len(q_start) - 1):
        q, k = slice(q_start[b], q_start[b + 1]), slice(kv_start[b], kv_start[b + 1])
        nq, nk = q.stop - q.start, k.stop - k.start
        for t in (dK, sK, dV, sV):
            t[:, k] = 0.0
        if nq == 0:
            continue
        mask = np.arange(nk)[None, :] < np.array([seen(nq, nk, causal, i) for i in range(nq)])[:, None]
        for h in range(H):
            hk = h // G
            s = np.where(mask, Q[h, q] @ K[hk, k].T * scale, -np.inf)
            top = np.max(s, 1, initial=-np.inf, keepdims=True)
            p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
            total = p.sum(1, keepdims=True)
            some = total > 0.0
            p = p / np.where(some, total, 1.0)
            with np.errstate(divide="ignore"):
                lse2[h, q] = np.where(some, (np.log(total) + top) / np.log(2.0), np.inf)[:, 0]
            O[h, q], sO[h, q] = p @ V[hk, k], p @ np.abs(V[hk, k])
            if dO is None:
                continue
            g = dO[h, q]
            dp = g @ V[hk, k].T
            ds = p * (dp - (p * dp).sum(1, keepdims=True))
            left = (np.abs(g) * 3.2 * sO[h, q]).sum(1, keepdims=True)
            e = p * left * (mask.sum(1, keepdims=True) > 1) + 2.2 * np.abs(ds)
            dQ[h, q], sQ[h, q] = scale * ds @ K[hk, k], scale * e @ np.abs(K[hk, k])
            dK[hk, k] += scale * ds.T @ Q[h, q]
            sK[hk, k] += scale * e.T @ np.abs(Q[h, q])
            dV[hk, k] += p.T @ g
            sV[hk, k] += p.T @ np.abs(g)
    if dO is None:
        return O, lse2, sO
    return O, lse2, sO, (dQ, dK, dV), (sQ, sK, sV)


def clip(grads, max_norm, eps):
    """(norm, factor) of a list of arrays."""
    n = np.sqrt(sum(float(np.sum(np.square(x, dtype=np.float64))) for x in grads))
    return n, (min(1.0, max_norm / (n + eps)) if np.isfinite(n) else 1.0)
