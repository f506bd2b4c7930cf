"""The operators around and beside the local attention, as cases to time and to compare: each as a plain form in elementary torch
operations (`own` false) and as the calls that a user of this library makes (`own` true).

    op  "norm"          group norm with an activation, channels last: slide_attn_group_norm_forward
        "norm_train"    that, and slide_attn_group_norm_backward of its output's gradient
        "drop"          residual + dropout(x) from a counter-based generator: slide_attn_dropout_forward
        "drop_train"    that, and slide_attn_dropout_backward
        "select"        the blocks of keys that each block of queries is to see: slide_attn_select_blocks
        "sparse"        attention over given blocks: slide_attn_sparse_forward
        "routed"        slide_attn_select_blocks, then slide_attn_sparse_forward over what it chose
        "sparse_train"  slide_attn_sparse_forward and slide_attn_sparse_backward
    B, H, W, heads, head_dim, dtype ("f32" / "bf16"): the maps, [B, H, W, heads, head_dim], or [B, H, W, C] with C = heads * head_dim
    groups, act ("none" / "silu" / "gelu"), affine       group norm
    p, images (whole images are dropped, not elements)   dropout
    block (edge of a block in pixels), top (blocks that a block of queries sees), holes (some of them are left out)   block-sparse attention
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5

# Philox4x32 with ten rounds (J. K. Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", SC11): multipliers and key increments
MULTIPLIERS = (0xD2511F53, 0xCD9E8D57)
INCREMENTS = (0x9E3779B9, 0xBB67AE85)


def _maps(name, op, B, H, W, heads, head_dim, dtype, **more):
    return dict(name=name, op=op, B=B, H=H, W=W, heads=heads, head_dim=head_dim, dtype=dtype, **more)


def listed():
    return [
        # the norm of one small map of one image: the smallest call, where latency and launches count
        _maps("norm_tiny_f32", "norm", 1, 14, 14, 1, 32, "f32", groups=8, act="none", affine=True),
        # training with the norm ahead of a first stage's block, a batch of 64 images, three channels in a group
        _maps("norm_train_bf16", "norm_train", 64, 56, 56, 3, 32, "bf16", groups=32, act="gelu", affine=True),
        # the same in a dense-prediction network at full precision: few images, large maps
        _maps("norm_train_crop_f32", "norm_train", 2, 128, 128, 3, 32, "f32", groups=8, act="silu", affine=True),
        # dropout after the output projection of a first stage's block, and its gradient
        _maps("drop_train_bf16", "drop_train", 64, 56, 56, 3, 32, "bf16", p=0.1, images=False),
        # stochastic depth: the residual branch of whole images left out, maps that are not square
        _maps("drop_images_f32", "drop", 32, 28, 42, 6, 32, "f32", p=0.2, images=True),
        # choosing four of 64 blocks of 7 x 7 pixels on a whole batch of first-stage maps
        _maps("select_bf16", "select", 64, 56, 56, 2, 32, "bf16", block=7, top=4),
        # one small image, two of four blocks: choosing and attention where latency counts
        _maps("routed_tiny_f32", "routed", 1, 14, 14, 1, 32, "f32", block=7, top=2),
        # a dense-prediction crop at full precision: eight of 256 blocks
        _maps("routed_crop_f32", "routed", 2, 128, 128, 3, 32, "f32", block=8, top=8),
        # inference of a first stage over blocks that are known
        _maps("sparse_bf16", "sparse", 64, 56, 56, 2, 32, "bf16", block=7, top=4, holes=False),
        # training on crops: each block of queries sees 1024 keys
        _maps("sparse_train_crop_bf16", "sparse_train", 2, 128, 128, 3, 32, "bf16", block=8, top=16, holes=False),
        # heads twice as wide, maps that no block divides, lists with holes
        _maps("sparse_train_ragged_bf16", "sparse_train", 32, 28, 42, 3, 64, "bf16", block=8, top=4, holes=True),
        # training at full precision
        _maps("sparse_train_f32", "sparse_train", 8, 56, 56, 3, 32, "f32", block=7, top=4, holes=False),
    ]


# What the largest listed cases work on: elements of one map, and elements times keys per query (a quarter of that at full precision).
MOST_ELEMENTS = 64 * 56 * 56 * 96
MOST_KEYS = 2 * 128 * 128 * 96 * 1024


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _elements(c):
    return c["B"] * c["H"] * c["W"] * c["heads"] * c["head_dim"]


def draw(rng):
    op = rng.choice(["norm", "norm_train", "drop", "drop_train", "select", "sparse", "routed", "sparse_train"])
    c = dict(op=op, B=_log_int(rng, 1, 64), H=_log_int(rng, 7, 128), W=_log_int(rng, 7, 128), dtype=rng.choice(["f32", "bf16"]))
    if op in ("norm", "norm_train", "drop", "drop_train"):
        c.update(heads=rng.randint(1, 8), head_dim=rng.choice([8, 16, 24, 32, 40, 64]))
    else:
        c.update(heads=rng.randint(1, 6), head_dim=rng.choice([16, 32, 32, 64]))
    if op in ("norm", "norm_train"):
        C = c["heads"] * c["head_dim"]
        c.update(groups=rng.choice([g for g in range(1, C + 1) if C % g == 0]), act=rng.choice(["none", "silu", "gelu"]), affine=rng.random() < 0.8)
    elif op in ("drop", "drop_train"):
        c.update(p=rng.choice([0.0, 0.05, 0.1, 0.3, 0.5, 0.9]), images=rng.random() < 0.3)
    else:
        edge = rng.choice([4, 5, 7, 8, 8, 12, 16])
        blocks = -(-c["H"] // edge) * -(-c["W"] // edge)
        c.update(block=edge, top=min(blocks, rng.choice([1, 2, 3, 4, 8, 16])))
        if op in ("sparse", "sparse_train"):
            c["holes"] = rng.random() < 0.4
    most = MOST_ELEMENTS // 2 if c["dtype"] == "f32" else MOST_ELEMENTS
    while c["B"] > 1 and (_elements(c) > most or ("top" in c and _elements(c) * c["top"] * c["block"] ** 2 > (MOST_KEYS // 4 if c["dtype"] == "f32" else MOST_KEYS))):
        c["B"] -= 1
    while "top" in c and c["top"] > 1 and _elements(c) * c["top"] * c["block"] ** 2 > (MOST_KEYS // 4 if c["dtype"] == "f32" else MOST_KEYS):
        c["top"] //= 2
    return c


def _blocks(c):
    return -(-c["H"] // c["block"]) * -(-c["W"] // c["block"])


class _State:
    """What the user's program keeps: its tensors, outputs among them."""

    def __init__(self, case):
        self.case = case


def prepare(case, seed):
    c, s = case, _State(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    td = DTYPES[c["dtype"]]
    B, H, W, heads, d = (c[n] for n in ("B", "H", "W", "heads", "head_dim"))
    C = heads * d
    if c["op"] in ("norm", "norm_train"):
        # features as a residual stream has them: each channel with an offset and a spread of its own
        spread = 0.5 + torch.rand(C, device="cuda", generator=gen)
        s.x = (normal(B, H, W, C) * spread + 0.5 * normal(C)).to(td)
        s.gamma = 1 + 0.2 * normal(C) if c["affine"] else None
        s.beta = 0.2 * normal(C) if c["affine"] else None
        s.y = torch.empty_like(s.x)
        s.mean, s.rstd = (torch.empty(B, c["groups"], device="cuda") for _ in range(2))
        if c["op"] == "norm_train":
            s.dy, s.dx = normal(B, H, W, C).to(td), torch.empty_like(s.x)
            s.dgamma, s.dbeta = ((torch.empty(C, device="cuda") for _ in range(2)) if c["affine"] else (None, None))
        return s
    if c["op"] in ("drop", "drop_train"):
        s.x, s.residual = (normal(B, H, W, C).to(td) for _ in range(2))
        s.y = torch.empty_like(s.x)
        s.rng = torch.randint(0, 2 ** 62, (2,), device="cuda", generator=gen)      # seed and offset of the generator
        if c["op"] == "drop_train":
            s.dy, s.dx = normal(B, H, W, C).to(td), torch.empty_like(s.x)
        return s
    s.q, s.k = (normal(B, H, W, heads, d).to(td) for _ in range(2))
    R = _blocks(c)
    if c["op"] in ("select", "routed"):
        s.idx = torch.empty(B, heads, R, c["top"], device="cuda", dtype=torch.int32)
    else:
        # distinct blocks in any order; with holes, a tenth of the entries are -1, and the first row of each list of rows is empty
        s.idx = torch.rand(B, heads, R, R, device="cuda", generator=gen).argsort(-1)[..., :c["top"]].to(torch.int32).contiguous()
        if c["holes"]:
            s.idx[torch.rand(s.idx.shape, device="cuda", generator=gen) < 0.1] = -1
            s.idx[:, :, 0] = -1
    if c["op"] != "select":
        s.v = normal(B, H, W, heads, d).to(td)
        s.out = torch.empty_like(s.q)
        s.lse = torch.empty(B, H, W, heads, device="cuda")
    if c["op"] == "sparse_train":
        s.dout = normal(B, H, W, heads, d).to(td)
        s.dq, s.dk, s.dv = (torch.empty_like(s.q) for _ in range(3))
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------------------------

def _activation(z, act):
    """act(z) and its derivative."""
    if act == "silu":
        g = 1 / (1 + torch.exp(-z))
        return z * g, g * (1 + z * (1 - g))
    if act == "gelu":
        g = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * g, g + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    return z, torch.ones_like(z)


def _plain_norm(s):
    c = s.case
    B, H, W, C = s.x.shape
    G = c["groups"]
    x = s.x.float().view(B, H * W, G, C // G)
    mean = x.mean((1, 3), keepdim=True)
    centred = x - mean
    rstd = 1 / torch.sqrt((centred * centred).mean((1, 3), keepdim=True) + EPS)
    xhat = centred * rstd
    gamma = s.gamma.view(G, C // G) if c["affine"] else 1.0
    beta = s.beta.view(G, C // G) if c["affine"] else 0.0
    y, slope = _activation(xhat * gamma + beta, c["act"])
    out = {"y": y.view(s.x.shape).to(s.x.dtype), "mean": mean.view(B, G), "rstd": rstd.view(B, G)}
    if c["op"] == "norm_train":
        dz = s.dy.float().view(x.shape) * slope
        dxhat = dz * gamma
        dx = rstd * (dxhat - dxhat.mean((1, 3), keepdim=True) - xhat * (dxhat * xhat).mean((1, 3), keepdim=True))
        out["dx"] = dx.view(s.x.shape).to(s.x.dtype)
        if c["affine"]:
            out["dgamma"] = (dz * xhat).sum((0, 1)).view(C)
            out["dbeta"] = dz.sum((0, 1)).view(C)
    return out


def _philox(n, rng):
    """n 32-bit words: word e is lane e % 4 of the block cipher of counter (e // 4, offset) under the key (seed)."""
    low = 0xFFFFFFFF
    i = torch.arange((n + 3) // 4, device=rng.device)
    a, b = i & low, i >> 32
    c, d = (rng[1] & low).expand_as(i), ((rng[1] >> 32) & low).expand_as(i)
    k0, k1 = rng[0] & low, (rng[0] >> 32) & low
    for _ in range(10):
        p, q = a * MULTIPLIERS[0], c * MULTIPLIERS[1]
        a, b, c, d = ((q >> 32) & low) ^ b ^ k0, q & low, ((p >> 32) & low) ^ d ^ k1, p & low
        k0, k1 = (k0 + INCREMENTS[0]) & low, (k1 + INCREMENTS[1]) & low
    return torch.stack([a, b, c, d], -1).view(-1)[:n]


def _threshold(p):
    """Words below it are dropped; p as the 32-bit number that the call takes."""
    return int(math.floor(float(np.float32(p)) * 2.0 ** 32))


def _plain_drop(s):
    c = s.case
    words = _philox(s.x.shape[0] if c["images"] else s.x.numel(), s.rng)
    kept = (words >= _threshold(c["p"])).view((-1, 1, 1, 1) if c["images"] else s.x.shape)
    scale = 1 / (1 - float(np.float32(c["p"])))
    zero = torch.zeros((), device=s.x.device)
    y = (s.residual.float() + torch.where(kept, s.x.float() * scale, zero)).to(s.x.dtype)
    if c["op"] == "drop":
        return y
    return {"y": y, "dx": torch.where(kept, s.dy.float() * scale, zero).to(s.x.dtype)}


def _pixels(c, device):
    """[blocks, block^2] the pixels of each block in row-major order, -1 where the map ends inside it."""
    e, H, W = c["block"], c["H"], c["W"]
    bh, bw = -(-H // e), -(-W // e)
    y = torch.arange(bh * e, device=device).view(bh, 1, e, 1)
    x = torch.arange(bw * e, device=device).view(1, bw, 1, e)
    return torch.where((y < H) & (x < W), y * W + x, -1).reshape(bh * bw, e * e)


def _by_block(t, pix):
    """[B, H, W, heads, d] as [B, heads, blocks, pixels of a block, d] in 32 bits; zero where there is none."""
    B, H, W, heads, d = t.shape
    t = t.reshape(B, H * W, heads, d)[:, pix.clamp(min=0)].float()
    return (t * (pix >= 0)[:, :, None, None]).permute(0, 3, 1, 2, 4)


def _by_pixel(t, pix, like):
    """The inverse of _by_block, rounded to the map's type."""
    B, H, W, heads, d = like.shape
    out = torch.empty(B, H * W, heads, d, device=t.device, dtype=like.dtype)
    out[:, pix[pix >= 0]] = t.permute(0, 2, 3, 1, 4)[:, pix >= 0].to(like.dtype)
    return out.view(like.shape)


def _plain_select(s):
    """Scores in 64 bits: neighbours in rank are not to change places by rounding."""
    c = s.case
    pix = _pixels(c, s.q.device)
    q, k = (_by_block(t, pix).double().sum(3) for t in (s.q, s.k))
    k = k / (pix >= 0).sum(1).double()[:, None]
    score = q @ k.transpose(-1, -2)
    return torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :c["top"]].to(torch.int32)


def _plain_sparse(s, idx):
    c = s.case
    B, H, W, heads, d = s.q.shape
    pix = _pixels(c, s.q.device)
    R, T = pix.shape
    keys = idx.shape[-1] * T
    q, k, v = (_by_block(t, pix) for t in (s.q, s.k, s.v))
    chosen = idx.clamp(min=0).long()
    there = ((idx >= 0)[..., None] & (pix >= 0)[chosen]).view(B, heads, R, 1, keys)

    def gathered(t):
        at = chosen.view(B, heads, -1, 1, 1).expand(-1, -1, -1, T, d)
        return torch.gather(t, 2, at).view(B, heads, R, keys, d)

    k, v = gathered(k), gathered(v)
    scale = 1 / math.sqrt(d)
    logits = (q @ k.transpose(-1, -2) * scale).masked_fill(~there, -math.inf)
    top = logits.amax(-1, keepdim=True)
    e = torch.exp(logits - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    weights = e / torch.where(total == 0, torch.ones_like(total), total)
    o = weights @ v
    lse = torch.empty(B, H * W, heads, device=q.device)
    lse[:, pix[pix >= 0]] = (top + torch.log(total)).squeeze(-1).permute(0, 2, 3, 1)[:, pix >= 0]
    out = {"out": _by_pixel(o, pix, s.q), "lse": lse.view(B, H, W, heads)}
    if c["op"] == "sparse_train":
        # of the output as it was stored
        stored, g = _by_block(out["out"], pix), _by_block(s.dout, pix)
        dl = weights * (g @ v.transpose(-1, -2) - (g * stored).sum(-1, keepdim=True)) * scale

        def spread(t):
            at = chosen.view(B, heads, -1, 1, 1).expand(-1, -1, -1, T, d)
            return torch.zeros(B, heads, R, T, d, device=t.device).scatter_add_(2, at, t.reshape(B, heads, -1, T, d))

        out["dq"] = _by_pixel(dl @ k, pix, s.q)
        out["dk"] = _by_pixel(spread(dl.transpose(-1, -2) @ q), pix, s.q)
        out["dv"] = _by_pixel(spread(weights.transpose(-1, -2) @ g), pix, s.q)
    return out


# ---- the calls ------------------------------------------------------------------------------------------------------------------------

def _own(s):
    import paper_2304_04237_b200 as sa
    c, op = s.case, s.case["op"]
    if op in ("norm", "norm_train"):
        act = {"none": sa.ACT_NONE, "silu": sa.ACT_SILU, "gelu": sa.ACT_GELU}[c["act"]]
        sa.slide_attn_group_norm_forward(s.x, s.gamma, s.beta, c["groups"], EPS, act, s.y, s.mean, s.rstd)
        out = {"y": s.y, "mean": s.mean, "rstd": s.rstd}
        if op == "norm_train":
            sa.slide_attn_group_norm_backward(s.x, s.gamma, s.beta, c["groups"], act, s.mean, s.rstd, s.dy, s.dx, s.dgamma, s.dbeta)
            out["dx"] = s.dx
            if c["affine"]:
                out.update(dgamma=s.dgamma, dbeta=s.dbeta)
        return out
    if op in ("drop", "drop_train"):
        unit = sa.DROP_IMAGES if c["images"] else sa.DROP_ELEMENTS
        sa.slide_attn_dropout_forward(s.x, s.residual, c["p"], unit, s.rng, s.y)
        if op == "drop":
            return s.y
        sa.slide_attn_dropout_backward(s.dy, c["p"], unit, s.rng, s.dx)
        return {"y": s.y, "dx": s.dx}
    block = (c["block"], c["block"])
    if op in ("select", "routed"):
        sa.slide_attn_select_blocks(s.q, s.k, block, s.idx)
        if op == "select":
            return s.idx
    sa.slide_attn_sparse_forward(s.q, s.k, s.v, s.idx, block, s.out, s.lse)
    out = {"out": s.out, "lse": s.lse}
    if op == "routed":
        out["idx"] = s.idx
    elif op == "sparse_train":
        sa.slide_attn_sparse_backward(s.q, s.k, s.v, s.idx, block, s.out, s.lse, s.dout, s.dq, s.dk, s.dv)
        out.update(dq=s.dq, dk=s.dk, dv=s.dv)
    return out


def run(s):
    if own:
        return _own(s)
    op = s.case["op"]
    if op in ("norm", "norm_train"):
        return _plain_norm(s)
    if op in ("drop", "drop_train"):
        return _plain_drop(s)
    if op == "select":
        return _plain_select(s)
    if op == "routed":
        idx = _plain_select(s)
        return {**_plain_sparse(s, idx), "idx": idx}
    return _plain_sparse(s, s.idx)


def work(case):
    """Every input read and every output written once, and the operations of the products (two for a multiply and add)."""
    c = case
    n = _elements(c)
    size = 4 if c["dtype"] == "f32" else 2
    C = c["heads"] * c["head_dim"]
    if c["op"] in ("norm", "norm_train"):
        # forward 2 maps; backward x again (the forward's result is not what it needs), dy and dx
        small = 8 * c["B"] * c["groups"] + (8 * C if c["affine"] else 0)
        train = c["op"] == "norm_train"
        return {"bytes": (5 if train else 2) * n * size + (2 if train else 1) * small, "flops": (25 if train else 10) * n}
    if c["op"] in ("drop", "drop_train"):
        return {"bytes": (5 if c["op"] == "drop_train" else 3) * n * size, "flops": 3 * n}
    R = _blocks(c)
    idx = 4 * c["B"] * c["heads"] * R * c["top"]
    lse = 4 * c["B"] * c["H"] * c["W"] * c["heads"]
    choose = 2 * c["B"] * R * R * C + 2 * n
    if c["op"] == "select":
        return {"bytes": 2 * n * size + idx, "flops": choose}
    keys = c["top"] * c["block"] ** 2
    forward = 4 * n * keys
    if c["op"] == "sparse_train":
        # the forward's maps, then q, k, v, out, dout in and dq, dk, dv out; five products beside the forward's two
        return {"bytes": 12 * n * size + 2 * idx + 2 * lse, "flops": forward + 10 * n * keys}
    return {"bytes": 4 * n * size + idx + lse, "flops": forward + (choose if c["op"] == "routed" else 0)}


# ---- the definitions in 64 bits, written apart from the plain forms ---------------------------------------------------------------------

def _exact_norm(s):
    """Group by group: sums over [images, pixels] of one group's channels, the gradient as J^T dy of (x - m) / sigma."""
    c = s.case
    B, H, W, C = s.x.shape
    G, n = c["groups"], H * W * (C // c["groups"])
    wide = lambda t: t.double().reshape(B, H * W, C)  # noqa: E731
    x, train = wide(s.x), c["op"] == "norm_train"
    member = torch.arange(C, device=x.device) // (C // G)
    fold = torch.nn.functional.one_hot(member, G).double()                    # [C, G]
    m = (x.sum(1) @ fold) / n
    var = ((x - m[:, member][:, None]).pow(2).sum(1) @ fold) / n
    sigma = (var + EPS).sqrt()
    u = (x - m[:, member][:, None]) / sigma[:, member][:, None]
    w = s.gamma.double() if c["affine"] else torch.ones(C, device=x.device, dtype=torch.double)
    b = s.beta.double() if c["affine"] else torch.zeros(C, device=x.device, dtype=torch.double)
    z = u * w + b
    if c["act"] == "silu":
        y, dact = z * torch.sigmoid(z), torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
    elif c["act"] == "gelu":
        cdf = 0.5 * torch.erfc(-z / math.sqrt(2))
        y, dact = z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    else:
        y, dact = z, torch.ones_like(z)
    out = {"y": y.view(s.x.shape), "mean": m, "rstd": 1 / sigma}
    if train:
        dz = wide(s.dy) * dact
        du = dz * w
        first = (du.sum(1) @ fold) / n
        second = ((du * u).sum(1) @ fold) / n
        out["dx"] = ((du - first[:, member][:, None] - u * second[:, member][:, None]) / sigma[:, member][:, None]).view(s.x.shape)
        if c["affine"]:
            out.update(dgamma=(dz * u).sum((0, 1)), dbeta=dz.sum((0, 1)))
    return out


def _exact_words(n, seed, offset):
    """The generator's words with the products of 32-bit numbers put together from 16-bit halves."""
    u = np.uint64
    half, low = u(0xFFFF), u(0xFFFFFFFF)

    def product(x, m):
        m0, m1 = u(m & 0xFFFF), u(m >> 16)
        x0, x1 = x & half, x >> u(16)
        middle = x1 * m0 + ((x0 * m0) >> u(16))
        other = x0 * m1 + (middle & half)
        return x1 * m1 + (middle >> u(16)) + (other >> u(16)), ((other & half) << u(16)) | ((x0 * m0) & half)

    i = np.arange((n + 3) // 4, dtype=np.uint64)
    ctr = [i & low, i >> u(32), np.full_like(i, offset & 0xFFFFFFFF), np.full_like(i, offset >> 32)]
    for r in range(10):
        key = [u(((seed >> (32 * j)) + r * INCREMENTS[j]) & 0xFFFFFFFF) for j in range(2)]
        (h0, l0), (h1, l1) = product(ctr[0], MULTIPLIERS[0]), product(ctr[2], MULTIPLIERS[1])
        ctr = [h1 ^ ctr[1] ^ key[0], l1, h0 ^ ctr[3] ^ key[1], l0]
    return np.stack(ctr, 1).reshape(-1)[:n]


def _exact_drop(s):
    c = s.case
    seed, offset = (int(v) for v in s.rng.cpu())
    words = _exact_words(s.x.shape[0] if c["images"] else s.x.numel(), seed, offset)
    p = float(np.float32(c["p"]))
    gain = np.where(words.astype(np.float64) < math.floor(p * 2.0 ** 32), 0.0, 1 / (1 - p))
    gain = torch.from_numpy(gain).to(s.x.device).view((-1, 1, 1, 1) if c["images"] else s.x.shape)
    y = s.residual.double() + s.x.double() * gain
    return y if c["op"] == "drop" else {"y": y, "dx": s.dy.double() * gain}


def _exact_sparse(s, idx):
    """Dense attention, image by image and head by head: the weight of key j for query i counts as often as j's block is in the list of i's."""
    c = s.case
    B, H, W, heads, d = s.q.shape
    n, e = H * W, c["block"]
    across = -(-W // e)
    at = torch.arange(n, device=s.q.device)
    block = (at // W // e) * across + at % W // e
    R = _blocks(c)
    train = c["op"] == "sparse_train"
    out = {name: torch.empty(B, n, heads, d, device=s.q.device, dtype=torch.double) for name in (("out", "dq", "dk", "dv") if train else ("out",))}
    out["lse"] = torch.empty(B, n, heads, device=s.q.device, dtype=torch.double)
    for b in range(B):
        for h in range(heads):
            q, k, v = (t[b].reshape(n, heads, d)[:, h].double() for t in (s.q, s.k, s.v))
            rows = idx[b, h].long()
            count = torch.zeros(R, R + 1, device=q.device, dtype=torch.double).scatter_add_(1, torch.where(rows < 0, R, rows), torch.ones_like(rows, dtype=torch.double))
            w = torch.exp(q @ k.T / math.sqrt(d)) * count[:, :R][block][:, block]
            total = w.sum(1, keepdim=True)
            out["lse"][b, :, h] = total.squeeze(1).log()
            w = w / total.clamp(min=1e-300)
            o = w @ v
            out["out"][b, :, h] = o
            if train:
                g = s.dout[b].reshape(n, heads, d)[:, h].double()
                dw = g @ v.T
                dl = w * (dw - (w * dw).sum(1, keepdim=True)) / math.sqrt(d)
                out["dq"][b, :, h], out["dk"][b, :, h], out["dv"][b, :, h] = dl @ k, dl.T @ q, w.T @ g
    return {name: t.view(B, H, W, heads, *t.shape[3:]) for name, t in out.items()}


def _exact_select(s):
    """Pooling as a product with the matrix of which pixel is in which block; equal scores stay in the order of their indexes."""
    c = s.case
    B, H, W, heads, d = s.q.shape
    n, e = H * W, c["block"]
    at = torch.arange(n, device=s.q.device)
    pool = torch.nn.functional.one_hot((at // W // e) * -(-W // e) + at % W // e, _blocks(c)).double()
    size = pool.sum(0)
    mean = [torch.einsum("nr,bnhd->bhrd", pool, t.reshape(B, n, heads, d).double()) / size[:, None] for t in (s.q, s.k)]
    score = torch.einsum("bhrd,bhsd->bhrs", *mean)
    return (-score).argsort(stable=True, dim=-1)[..., :c["top"]].to(torch.int32)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("norm", "norm_train"):
        return _exact_norm(s)
    if case["op"] in ("drop", "drop_train"):
        return _exact_drop(s)
    if case["op"] == "select":
        return _exact_select(s)
    if case["op"] == "routed":
        idx = _exact_select(s)
        return {**_exact_sparse(s, idx), "idx": idx}
    return _exact_sparse(s, s.idx)
