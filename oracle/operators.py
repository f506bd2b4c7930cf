"""Plain definitions, in double precision on the CPU, of the operators around and beside the local attention: group norm with an
activation, dropout from a counter-based generator, block-sparse attention.  Test infrastructure only; slow and literal."""
from __future__ import annotations

import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])


def activation(z, act):
    """act(z) and its derivative; act: "none", "silu", "gelu"."""
    if act == "silu":
        g = 1.0 / (1.0 + np.exp(-z))
        return z * g, g + z * g * (1.0 - g)
    if act == "gelu":
        cdf = 0.5 * (1.0 + _erf(z / math.sqrt(2.0)))
        return z * cdf, cdf + z * np.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
    return z, np.ones_like(z)


def group_norm(x, gamma, beta, groups, eps, act, dy=None):
    """x: [B, H, W, C]; gamma, beta: [C] or None.  Returns a dict of y, mean, rstd [B, groups] and, with dy, dx, dgamma, dbeta and the sums
    of the absolute values of what dgamma and dbeta add up."""
    x = np.asarray(x, np.float64)
    B, H, W, C = x.shape
    per = C // groups
    gamma = np.ones(C) if gamma is None else np.asarray(gamma, np.float64)
    beta = np.zeros(C) if beta is None else np.asarray(beta, np.float64)
    y, dx = np.empty_like(x), np.empty_like(x)
    mean, rstd = np.empty((B, groups)), np.empty((B, groups))
    sums = {n: np.zeros(C) for n in ("dgamma", "dbeta", "dgamma_abs", "dbeta_abs")}
    for b in range(B):
        for g in range(groups):
            c = slice(g * per, (g + 1) * per)
            part = x[b, :, :, c]
            m = part.mean()
            r = 1.0 / math.sqrt(((part - m) ** 2).mean() + eps)
            mean[b, g], rstd[b, g] = m, r
            u = (part - m) * r
            y[b, :, :, c], slope = activation(u * gamma[c] + beta[c], act)
            if dy is not None:
                dz = np.asarray(dy[b, :, :, c], np.float64) * slope
                du = dz * gamma[c]
                dx[b, :, :, c] = r * (du - du.mean() - u * (du * u).mean())
                for n, t in (("dgamma", dz * u), ("dbeta", dz)):
                    sums[n][c] += t.sum((0, 1))
                    sums[n + "_abs"][c] += np.abs(t).sum((0, 1))
    out = {"y": y, "mean": mean, "rstd": rstd}
    return out if dy is None else {**out, "dx": dx, **sums}


def philox(counter, key):
    """Ten rounds of Philox4x32 of one counter (four 32-bit words) under one key (two), in Python's integers."""
    a, b, c, d = counter
    k0, k1 = key
    low = 0xFFFFFFFF
    for _ in range(10):
        p, q = 0xD2511F53 * a, 0xCD9E8D57 * c
        a, b, c, d = (q >> 32) ^ b ^ k0, q & low, (p >> 32) ^ d ^ k1, p & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return a, b, c, d


def kept(n, p, seed, offset, first=0):
    """Which of the units first .. first + n - 1 are kept."""
    low = 0xFFFFFFFF
    words, at = {}, np.empty(n, bool)
    limit = math.floor(float(np.float32(p)) * 2 ** 32)
    for i, e in enumerate(range(first, first + n)):
        if e // 4 not in words:
            q = e // 4
            words = {q: philox((q & low, q >> 32, offset & low, offset >> 32), (seed & low, seed >> 32))}
        at[i] = words[e // 4][e % 4] >= limit
    return at


def dropout(x, residual, p, images, seed, offset):
    """residual + (kept ? x / (1 - p) : 0); x: images first."""
    x = np.asarray(x, np.float64)
    mask = kept(x.shape[0], p, seed, offset).reshape((-1,) + (1,) * (x.ndim - 1)) if images else kept(x.size, p, seed, offset).reshape(x.shape)
    p = float(np.float32(p))
    y = np.where(mask, x / (1.0 - p) if p < 1.0 else 0.0, 0.0)
    return y if residual is None else y + np.asarray(residual, np.float64)


def block_pixels(H, W, block):
    """The pixels (y * W + x) of every block, row by row."""
    bh, bw = block
    return [[y * W + x for y in range(y0, min(H, y0 + bh)) for x in range(x0, min(W, x0 + bw))] for y0 in range(0, H, bh) for x0 in range(0, W, bw)]


def scores(q, k, block):
    """[B, heads, blocks, blocks]: the sum of q over a block times the mean of k over a block."""
    B, H, W, heads, d = q.shape
    pix = block_pixels(H, W, block)
    q, k = (np.asarray(t, np.float64).reshape(B, H * W, heads, d) for t in (q, k))
    qs = np.stack([q[:, p].sum(1) for p in pix], 1)
    ks = np.stack([k[:, p].sum(1) / len(p) for p in pix], 1)
    return np.einsum("brhd,bshd->bhrs", qs, ks)


def select(q, k, block, top):
    s = scores(q, k, block)
    s = np.where(np.isnan(s), -np.inf, s)
    return np.argsort(-s, axis=-1, kind="stable")[..., :top].astype(np.int32)


def sparse(q, k, v, idx, block, dout=None, out=None):
    """Attention over the listed blocks: a dict of out, lse and, with dout (and the out that was stored), dq, dk, dv.  "*_abs": the same sums
    with every term's absolute value, which is what rounding errors are relative to."""
    B, H, W, heads, d = q.shape
    pix = block_pixels(H, W, block)
    flat = lambda t: np.asarray(t, np.float64).reshape(B, H * W, heads, d)  # noqa: E731
    shape = q.shape
    q, k, v = flat(q), flat(k), flat(v)
    names = ["out", "out_abs"] + (["dq", "dk", "dv", "dq_abs", "dk_abs", "dv_abs"] if dout is not None else [])
    r = {n: np.zeros((B, H * W, heads, d)) for n in names}
    lse = np.full((B, H * W, heads), -np.inf)
    g = flat(dout) if dout is not None else None
    for b in range(B):
        for h in range(heads):
            for i, rows in enumerate(pix):
                cols = [p for s in idx[b, h, i] if 0 <= s < len(pix) for p in pix[s]]
                if not cols:
                    continue
                logits = q[b, rows, h] @ k[b, cols, h].T / math.sqrt(d)
                most = logits.max(1, keepdims=True)
                most = np.where(np.isneginf(most), 0.0, most)
                e = np.exp(logits - most)
                total = e.sum(1, keepdims=True)
                w = e / np.where(total == 0.0, 1.0, total)
                with np.errstate(divide="ignore"):
                    lse[b, rows, h] = (most + np.log(total))[:, 0]
                r["out"][b, rows, h] = w @ v[b, cols, h]
                r["out_abs"][b, rows, h] = w @ np.abs(v[b, cols, h])
                if dout is None:
                    continue
                gi = g[b, rows, h]
                stored = r["out"][b, rows, h] if out is None else np.asarray(out, np.float64).reshape(B, H * W, heads, d)[b, rows, h]
                ds = w * (gi @ v[b, cols, h].T - (gi * stored).sum(1, keepdims=True)) / math.sqrt(d)
                da = w * (np.abs(gi) @ np.abs(v[b, cols, h]).T + (np.abs(gi * stored)).sum(1, keepdims=True)) / math.sqrt(d)
                r["dq"][b, rows, h] = ds @ k[b, cols, h]
                r["dq_abs"][b, rows, h] = da @ np.abs(k[b, cols, h])
                for n, t in (("dk", ds.T @ q[b, rows, h]), ("dv", w.T @ gi), ("dk_abs", da.T @ np.abs(q[b, rows, h])), ("dv_abs", w.T @ np.abs(gi))):
                    np.add.at(r[n][b, :, h], cols, t)
    return {**{n: t.reshape(shape) for n, t in r.items()}, "lse": lse.reshape(shape[:4])}
