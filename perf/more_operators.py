"""Operators of a prompt's way into a 4-bit cache and of decoding from it, each in its plain form and as the library's own call.

  norm    RMS norms of every head of the queries and keys and their rotary positions, of a tree's nodes or of a prompt, in one pass
  prompt  causal attention of whole prompts (or the next chunk of them) with grouped heads, sequences of different lengths
  append  new K/V rows into the 4-bit block cache: the open block of 64 tokens stays in bf16, full blocks become E2M1 codes
  attend  tree attention (or plain decoding) over that cache; the tree's own K/V are bf16

A case is a dict of plain values; listed() names the fixed ones, draw() gives more of the same ranges.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
BLOCK = 64
GROUP = 32           # values of the 4-bit cache to a scale
LOWEST = -100        # exponent of the smallest scale


def _norm(name, batch, heads, head_dim, depth, width, prefix, rotary_dim=0, interleaved=False, dtype="bf16", fused=False, prompt=0,
          per_head=False):
    """prompt: that many explicit positions per sequence instead of a tree; fused: q and k are parts of one QKV projection;
    per_head: norm weights of each head's own."""
    return dict(name=name, kind="norm", batch=batch, q_heads=heads[0], kv_heads=heads[1], head_dim=head_dim, depth=depth, width=width,
                prefix=prefix, rotary_dim=rotary_dim or head_dim, interleaved=interleaved, dtype=dtype, fused=fused, prompt=prompt,
                per_head=per_head)


def _prompt(name, batch, heads, head_dim, tokens, shortest=0, past=0, dtype="bf16", lse=False):
    """Sequences of `shortest` to `tokens` new tokens, evenly spread; past > 0: the next chunk of longer prompts whose keys and values
    lie in a cache of one slab per sequence, that many of the longest's before it; else packed, straight out of the QKV projection."""
    return dict(name=name, kind="prompt", batch=batch, q_heads=heads[0], kv_heads=heads[1], head_dim=head_dim, tokens=tokens,
                shortest=shortest or tokens, past=past, dtype=dtype, lse=lse)


def _append(name, batch, kv_heads, head_dim, depth, width, prefix, layers, new=0):
    """new: a prompt's tokens, all of them, behind an empty cache (0: the accepted path of a tree of depth x width nodes behind `prefix`)."""
    return dict(name=name, kind="append", batch=batch, kv_heads=kv_heads, head_dim=head_dim, depth=depth, width=width, prefix=prefix,
                layers=layers, new=new)


def _attend(name, batch, heads, head_dim, depth, width, prefix, shortest=0, lse=False):
    """Confirmed lengths are spread evenly over shortest .. prefix (0: all `prefix`)."""
    return dict(name=name, kind="attend", batch=batch, q_heads=heads[0], kv_heads=heads[1], head_dim=head_dim, depth=depth, width=width,
                prefix=prefix, shortest=shortest or prefix, lse=lse)


def listed():
    return [
        # one decoding step of a small fp32 model: one token, launch latency
        _norm("norm one token", 1, (4, 4), 64, 0, 1, 128, dtype="f32"),
        # the trees of sixteen requests to a 70B-shaped model, straight out of the QKV projection
        _norm("norm tree 70B batch 16", 16, (64, 8), 128, 6, 8, 8192, fused=True),
        # two prompts of an 8B-shaped model, half of each head rotated, interleaved pairs, weights of each head's own
        _norm("norm prompt 8B", 2, (32, 8), 128, 0, 1, 131072, rotary_dim=64, interleaved=True, prompt=6000, per_head=True),
        # a short prompt of a small fp32 model
        _prompt("prompt tiny fp32", 1, (4, 4), 64, 37, dtype="f32", lse=True),
        # the drafter reads the prompts of eight requests
        _prompt("prompt drafter batch 8", 8, (12, 12), 64, 2047, shortest=90),
        # a whole prompt of an 8B-shaped model: the matrix cores
        _prompt("prompt 8B", 1, (32, 8), 128, 8192),
        # the next 500 tokens of two long prompts of a 70B-shaped model: few rows, many keys
        _prompt("prompt chunk 70B", 2, (64, 8), 128, 500, shortest=333, past=30000, lse=True),
        # the accepted path of each of sixteen requests into the caches of 32 layers; a few fill their block
        _append("append accepted 8B", 16, 8, 128, 6, 8, 511, 32),
        # a prompt of 8191 tokens into the caches of four layers
        _append("append prompt 8B", 1, 8, 128, 0, 1, 0, 4, new=8191),
        # plain decoding, one token each, sixteen ragged requests: the stream of the cache
        _attend("attend one token batch 16", 16, (32, 8), 128, 0, 1, 8192, shortest=512),
        # the drafter's own attention over its tree, ragged, log-sum-exps wanted
        _attend("attend drafter batch 3", 3, (12, 12), 64, 8, 8, 2047, shortest=301, lse=True),
        # verification of 49 nodes behind eight long prefixes, grouped heads
        _attend("attend 8B batch 8", 8, (32, 8), 128, 6, 8, 16384),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_HEADS = [((32, 32), 128), ((40, 40), 128), ((32, 8), 128), ((64, 8), 128), ((12, 12), 64), ((32, 8), 64)]


def draw(rng):
    kind = rng.choice(["norm", "prompt", "prompt", "append", "attend", "attend"])
    batch = 1 if rng.random() < 0.4 else _log_int(rng, 2, 16)
    depth, width = rng.randint(2, 10), _log_int(rng, 2, 32)
    if rng.random() < 0.25:
        depth, width = 0, 1
    prefix = _log_int(rng, 64, 32768)
    heads, head_dim = rng.choice(_HEADS)
    if kind == "norm":
        rotary_dim = rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4])
        prompt = _log_int(rng, 2, 16384 // batch) if rng.random() < 0.4 else 0
        case = _norm("", batch, heads, head_dim, depth, width, prefix + prompt, rotary_dim, rng.random() < 0.5,
                     rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.5, prompt, rng.random() < 0.3)
    elif kind == "prompt":
        dtype = rng.choice(["bf16", "bf16", "bf16", "bf16", "f32"])
        tokens = _log_int(rng, 1, 8192 if dtype == "bf16" else 512)
        past = _log_int(rng, 1, 30000) if rng.random() < 0.3 else 0
        case = _prompt("", batch, heads, head_dim, tokens, rng.choice([0, max(1, tokens // 20)]), past, dtype, rng.random() < 0.3)
    elif kind == "append":
        layers = rng.choice([1, 4, 32])
        if rng.random() < 0.5:
            case = _append("", batch, heads[1], head_dim, depth, width, min(prefix, 2000), layers)
        else:
            case = _append("", batch, heads[1], head_dim, 0, 1, 0, layers, new=min(_log_int(rng, 2, 16384), 2048 if layers > 4 else 16384))
    else:
        case = _attend("", batch, heads, head_dim, depth, width, prefix, rng.choice([0, max(1, prefix // 16)]), rng.random() < 0.3)
    limit = max(_cost(c) for c in listed())
    while _cost(case) > limit or _plain_bytes(case) > 24e9:        # stay below the largest listed cases
        for key in ("layers", "batch", "past", "prompt", "new", "tokens", "prefix"):
            if case.get(key, 0) > 1:
                case[key] //= 2
                if "shortest" in case:
                    case["shortest"] = max(1, min(case["shortest"], case.get("tokens", case.get("prefix", 1))))
                break
    del case["name"]
    return case


def _cost(case):
    w = work(case)
    rate = 1e15 if case.get("dtype", "bf16") == "bf16" else 1e14
    return max(w["bytes"] / 5e12, w["flops"] / rate)


def _plain_bytes(case):
    """Of the scores that the plain form holds."""
    if case["kind"] == "prompt":
        return 4.0 * case["batch"] * case["q_heads"] * case["tokens"] * (case["tokens"] + case["past"])
    if case["kind"] == "attend":
        return 4.0 * case["batch"] * case["q_heads"] * (1 + case["depth"] * case["width"]) * (case["prefix"] + 1200)
    return 0.0


def _elem(case):
    return 4 if case["dtype"] == "f32" else 2


def _spread(longest, shortest, batch):
    """The batch's lengths, evenly spread from the longest to the shortest (their order comes from the seed)."""
    return np.rint(np.linspace(longest, shortest, batch)).astype(np.int64)


def _lens(case):
    """Confirmed lengths in front of a tree."""
    if case["kind"] == "attend":
        return _spread(case["prefix"], case["shortest"], case["batch"])
    return np.maximum(case["prefix"] - np.arange(case["batch"], dtype=np.int64), 0)


def _rows(case):
    """(new tokens, tokens before them) of a batch of prompts."""
    new = _spread(case["tokens"], case["shortest"], case["batch"])
    return new, _spread(case["past"], (case["past"] + 1) // 2, case["batch"])


def _accepted(case):
    """Accepted tokens of each sequence: the whole prompt, or one to depth + 1 tokens of a tree."""
    if case["new"]:
        return np.full(case["batch"], case["new"], np.int64)
    return 1 + np.arange(case["batch"], dtype=np.int64) % (case["depth"] + 1)


def _stored(head_dim, tokens):
    """Bytes of so many tokens of one head in whole blocks: codes and scales, K and V."""
    return 2.0 * tokens * head_dim * (0.5 + 1.0 / GROUP)


def work(case):
    if case["kind"] == "norm":
        tokens = case["batch"] * (case["prompt"] or 1 + case["depth"] * case["width"])
        values = float(tokens) * (case["q_heads"] + case["kv_heads"])
        return {"bytes": 2.0 * values * case["head_dim"] * _elem(case), "flops": values * (4.0 * case["head_dim"] + 3.0 * case["rotary_dim"])}
    if case["kind"] == "prompt":
        new, past = (x.astype(float) for x in _rows(case))
        pairs = float((new * past + new * (new + 1) / 2).sum())
        row = case["head_dim"] * _elem(case)
        nbytes = 2.0 * row * (case["q_heads"] * float(new.sum()) + case["kv_heads"] * float((new + past).sum()))
        return {"bytes": nbytes + 4.0 * case["lse"] * case["q_heads"] * float(new.sum()), "flops": 4.0 * case["q_heads"] * case["head_dim"] * pairs}
    if case["kind"] == "append":
        old, new = _lens(case), _accepted(case)
        full = ((old + new) // BLOCK - old // BLOCK) * BLOCK                                  # tokens that become codes
        tail = np.where(full > 0, (old + new) % BLOCK, new)                                   # rows that are left open
        reread = np.where(full > 0, old % BLOCK, 0)
        row = 2.0 * case["layers"] * case["kv_heads"] * case["head_dim"]
        nbytes = row * float((2 * new + 2 * reread + 2 * tail).sum()) + case["layers"] * case["kv_heads"] * _stored(case["head_dim"], float(full.sum()))
        return {"bytes": nbytes, "flops": 3.0 * row * float(full.sum())}
    B, D, W = case["batch"], case["depth"], case["width"]
    N = 1 + D * W
    lens = _lens(case).astype(float)
    full = lens // BLOCK * BLOCK
    row = case["kv_heads"] * case["head_dim"]
    nbytes = case["kv_heads"] * _stored(case["head_dim"], float(full.sum())) + 4.0 * row * float((lens - full).sum() + B * N)
    nbytes += 4.0 * B * N * case["q_heads"] * case["head_dim"] + 4.0 * case["lse"] * B * N * case["q_heads"]
    keys = N * float(lens.sum()) + B * (1 + W * D * (D + 3) / 2)
    return {"bytes": nbytes, "flops": 4.0 * case["q_heads"] * case["head_dim"] * keys}


# ---------------------------------------------------------------- what a program has in hand

def _ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _normal(gen, shape, dtype):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=gen)


def _tree(host, D, W):
    """A level-structured tree with skewed child counts."""
    parent = np.full(1 + D * W, -1, np.int64)
    for d in range(1, D + 1):
        at = 1 + (d - 1) * W
        parent[at:at + W] = 0 if d == 1 else at - W + host.choice(W, size=W, p=host.dirichlet(np.full(W, 0.5)))
    return parent


def _path(parent, length, host):
    """`length` nodes from the root downwards where the tree has such a path, else as many as it has."""
    path = [0]
    while len(path) < length:
        kids = np.nonzero(parent == path[-1])[0]
        if not len(kids):
            break
        path.append(int(host.choice(kids)))
    return path


def _cache(case, lead, nblk, gen, fill):
    """Codes (two to a byte), scales (powers of two: their exponents + 127) and open blocks of a cache."""
    Hkv, Dh = case["kv_heads"], case["head_dim"]
    s = {}
    for x, encode in (("k", _encode_k), ("v", _encode_v)):
        if fill:
            s[x + "_codes"], s[x + "_scale"] = encode(_normal(gen, (*lead, Hkv, nblk, BLOCK, Dh), torch.float32))
        else:
            s[x + "_codes"] = torch.zeros((*lead, Hkv, nblk, BLOCK * Dh // 2), dtype=torch.uint8, device=DEV)
            s[x + "_scale"] = torch.full((*lead, Hkv, nblk, BLOCK * Dh // GROUP), 127, dtype=torch.uint8, device=DEV)
        s[x + "_tail"] = _normal(gen, (*lead, 2 * BLOCK, Hkv, Dh), torch.bfloat16)
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    host = np.random.default_rng(seed)
    B, kind = case["batch"], case["kind"]
    s = dict(case=case)
    if kind != "prompt":
        D, W = case["depth"], case["width"]
        N = 1 + D * W
        parent = np.stack([_tree(host, D, W) for _ in range(B)])
        s["parent"] = _ints(parent)

    if kind == "norm":
        T = case["prompt"] or N
        Hq, Hkv, Dh = case["q_heads"], case["kv_heads"], case["head_dim"]
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        # projections' magnitudes differ from token to token: that is what the norm is for
        size = torch.exp(_normal(gen, (B, T, 1, 1), torch.float32))
        if case["fused"]:
            qkv = (_normal(gen, (B, T, Hq + 2 * Hkv, Dh), torch.float32) * size).to(dt)
            s["q"], s["k"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]
        else:
            s["q"], s["k"] = ((_normal(gen, (B, T, h, Dh), torch.float32) * size).to(dt) for h in (Hq, Hkv))
        s["q_out"], s["k_out"] = (torch.empty((B, T, h, Dh), dtype=dt, device=DEV) for h in (Hq, Hkv))
        s["q_weight"], s["k_weight"] = (1 + 0.3 * _normal(gen, (h, Dh) if case["per_head"] else (Dh,), torch.float32) for h in (Hq, Hkv))
        s["eps"] = 1e-6
        pairs = case["rotary_dim"] // 2
        s["frequencies"] = torch.from_numpy(500000.0 ** (-np.arange(pairs) / pairs)).to(DEV)
        s["lens"] = _ints(host.permutation(_lens(case)))
        # a prompt is the last part of a context as long as `prefix`
        s["positions"] = _ints(np.maximum(_lens(case)[:, None] - T + np.arange(T)[None], 0)) if case["prompt"] else None

    if kind == "prompt":
        Hq, Hkv, Dh = case["q_heads"], case["kv_heads"], case["head_dim"]
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        new, past = _rows(case)
        order = host.permutation(B)
        new, past = new[order], past[order]
        T = int(new.sum())
        s["longest"] = int((new + past).max())
        s["q_first"], s["q_len"] = _ints(np.cumsum(new) - new), _ints(new)
        s["k_len"] = _ints(new + past)
        if case["past"]:
            cap = -(-(case["past"] + case["tokens"]) // 64) * 64
            s["q"] = _normal(gen, (T, Hq, Dh), dt)
            s["k"], s["v"] = (_normal(gen, (B * cap, Hkv, Dh), dt) for _ in range(2))
            s["k_first"] = _ints(np.arange(B) * cap)
        else:
            qkv = _normal(gen, (T, Hq + 2 * Hkv, Dh), dt)
            s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
            s["k_first"] = s["q_first"]
        s["out"] = torch.empty((T, Hq, Dh), dtype=dt, device=DEV)
        s["lse"] = torch.empty((T, Hq), dtype=torch.float32, device=DEV) if case["lse"] else None

    if kind == "append":
        old, new = host.permutation(_lens(case)), host.permutation(_accepted(case))
        T, L = case["new"] or N, case["layers"]
        rows = np.full((B, D + 1), -1, np.int64)
        if not case["new"]:
            for b in range(B):
                path = _path(parent[b], new[b], host)
                rows[b, :len(path)] = path
                new[b] = len(path)
            s["rows"] = _ints(rows)
        s["lens"], s["new"] = _ints(old + new), _ints(new)
        s |= _cache(case, (L, B), -(-(case["prefix"] + (case["new"] or D + 1)) // BLOCK), gen, fill=False)
        for x in "kv":
            s[x + "_new"] = _normal(gen, (L, B, T, case["kv_heads"], case["head_dim"]), torch.bfloat16)

    if kind == "attend":
        Hq, Hkv, Dh = case["q_heads"], case["kv_heads"], case["head_dim"]
        s["lens"] = _ints(host.permutation(_lens(case)))
        s |= _cache(case, (B,), -(-(case["prefix"] + D + 1) // BLOCK), gen, fill=True)
        s["q"] = _normal(gen, (B, N, Hq, Dh), torch.bfloat16)
        for x in "kv":
            s[x + "_tree"] = _normal(gen, (B, N, Hkv, Dh), torch.bfloat16)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((B, N, Hq), dtype=torch.float32, device=DEV) if case["lse"] else None
    return s


# ---------------------------------------------------------------- one pass, in its plain form

def _ancestors(parent, D):
    """[B, N, N] truth values: column j is on the path from the root to row i, i included."""
    B, N = parent.shape
    node = torch.arange(N, device=DEV).expand(B, N)
    on = torch.zeros((B, N, N + 1), dtype=torch.bool, device=DEV)
    up = parent.long()
    for _ in range(D + 1):
        on.scatter_(2, node[..., None], True)                                   # (column N: beyond the root)
        node = torch.where(node < N, torch.gather(up, 1, node.clamp(max=N - 1)), node)
        node = torch.where(node < 0, N, node)
    return on[..., :N]


def _plain_norm(s):
    c = s["case"]
    if s["positions"] is not None:
        position = s["positions"].double()
    else:
        position = s["lens"][:, None].double() + _ancestors(s["parent"], c["depth"]).sum(-1) - 1
    angle = position[..., None] * s["frequencies"]
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    r = c["rotary_dim"]

    def turned(x, weight):
        y = x.float()
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + s["eps"]) * weight
        part, rest = y[..., :r], y[..., r:]
        a, b = (part[..., ::2], part[..., 1::2]) if c["interleaved"] else (part[..., :r // 2], part[..., r // 2:])
        a, b = a * cos - b * sin, b * cos + a * sin
        part = torch.stack((a, b), -1).flatten(-2) if c["interleaved"] else torch.cat((a, b), -1)
        return torch.cat((part, rest), -1).to(x.dtype)
    return {"q": turned(s["q"], s["q_weight"]), "k": turned(s["k"], s["k_weight"])}


def _plain_prompt(s):
    c = s["case"]
    T, Hq, Dh = s["q"].shape
    Hkv, B = s["k"].shape[1], c["batch"]
    G = Hq // Hkv
    q_len, k_len = s["q_len"].long()[:, None], s["k_len"].long()[:, None]
    i, j = torch.arange(c["tokens"], device=DEV)[None], torch.arange(s["longest"], device=DEV)[None]
    q_row = torch.minimum(s["q_first"].long()[:, None] + i, torch.tensor(T - 1, device=DEV))
    k_row = torch.where(j < k_len, s["k_first"].long()[:, None] + j, s["k_first"].long()[:, None])
    q = s["q"][q_row].float().view(B, -1, Hkv, G, Dh).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, Dh)
    k, v = (s[x][k_row].float().transpose(1, 2).contiguous() for x in "kv")                    # [B, Hkv, keys, Dh]
    seen = j[:, None] <= (i + k_len - q_len)[..., None]                                        # [B, rows, keys]
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(Dh)).view(B, Hkv, G, -1, s["longest"])
    score.masked_fill_(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = score.sub_(top).exp_()
    total = weight.sum(-1, keepdim=True)
    out = torch.matmul(weight.view(B, Hkv, -1, s["longest"]), v).view(B, Hkv, G, -1, Dh) / total
    there = i < q_len                                                                          # [B, rows]
    out = out.permute(0, 3, 1, 2, 4).reshape(B, -1, Hq, Dh)[there].to(s["q"].dtype)            # the batch's rows lie in order
    got = {"out": torch.empty_like(out).index_copy_(0, q_row[there], out)}
    if c["lse"]:
        lse = (top + total.log())[..., 0].permute(0, 3, 1, 2).reshape(B, -1, Hq)[there]
        got["lse"] = torch.empty_like(lse).index_copy_(0, q_row[there], lse)
    return got


def _e2m1(y, negative):
    """Codes of values in scale: nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code, sign above."""
    a = y.abs()
    code = negative.to(torch.uint8) * 8
    for bound, up in ((0.25, a.gt), (0.75, a.ge), (1.25, a.gt), (1.75, a.ge), (2.5, a.gt), (3.5, a.ge), (5.0, a.gt)):
        code += up(bound)
    return code


def _exponent(amax):
    """The least whole number e >= LOWEST with amax <= 7 * 2^e."""
    part, e = torch.frexp(amax)                                                                # amax = part * 2^e, part in [0.5, 1)
    return torch.where(amax > 0, e - 3 + (part > 0.875).int(), LOWEST).clamp(min=LOWEST)


def _pairs(code):
    return code[..., ::2] | code[..., 1::2] << 4


def _encode(x):
    """[.., 32] values to a group -> codes [.., 16] (two to a byte), exponents [..]."""
    e = _exponent(x.abs().amax(-1))
    return _pairs(_e2m1(torch.ldexp(x, -e[..., None]), torch.signbit(x))), (e + 127).to(torch.uint8)


def _encode_k(x):
    """K of whole blocks [.., 64 tokens, Dh] in fp32 -> (codes, scales) in storage order: 32 tokens by 64 dimensions after another, each as
    the operand of a matrix instruction (64 lanes: token and half of the dimensions, 32 dimensions to a lane)."""
    Dh = x.shape[-1]
    x = x.reshape(*x.shape[:-2], 2, 32, Dh // 64, 2, 32)                                       # tokens: t r   dimensions: j h i
    n = x.dim() - 5
    codes, scale = _encode(x.permute(*range(n), n, n + 2, n + 3, n + 1, n + 4))                # t j h r i
    return codes.reshape(*x.shape[:n], 32 * Dh), scale.permute(*range(n), n + 2, n + 3, n, n + 1).reshape(*x.shape[:n], 2 * Dh)


def _encode_v(x):
    """V of whole blocks: 32 dimensions after another, 32 tokens to a lane in the order in which a matrix instruction meets the scores of
    another one's accumulator."""
    Dh = x.shape[-1]
    x = x.reshape(*x.shape[:-2], 2, 4, 2, 4, Dh // 32, 32)                                     # tokens: u e4 h e1   dimensions: d r
    n = x.dim() - 6
    x = x.permute(*range(n), n + 4, n, n + 5, n + 2, n + 1, n + 3)                             # d u r, h e4 e1
    codes, scale = _encode(x.reshape(*x.shape[:n + 3], 32))
    return codes.reshape(*x.shape[:n], 32 * Dh), scale.permute(*range(n), n + 1, n + 2, n).reshape(*x.shape[:n], 2 * Dh)


def _plain_append(s):
    c = s["case"]
    L, B, T, Hkv, Dh = s["k_new"].shape
    most = c["new"] or c["depth"] + 1
    new, end = s["new"].long(), s["lens"].long()
    old = end - new
    blocks = (most + 2 * BLOCK - 2) // BLOCK
    token = (old // BLOCK * BLOCK)[:, None] + torch.arange(blocks * BLOCK, device=DEV)         # [B, tokens of the touched blocks]
    k = (token - old[:, None]).clamp(0, most - 1)
    row = torch.gather(s["rows"].long(), 1, k).clamp(min=0) if "rows" in s else k
    seq = torch.arange(B, device=DEV)[:, None]
    is_old, is_new = token < old[:, None], (token >= old[:, None]) & (token < end[:, None])
    whole = (token[:, ::BLOCK] + BLOCK <= end[:, None])                                        # [B, touched blocks]
    b, j = whole.nonzero(as_tuple=True)
    at = token[b, j * BLOCK] // BLOCK
    b2, t2 = (is_new & (token >= (end // BLOCK * BLOCK)[:, None])).nonzero(as_tuple=True)      # rows that stay open
    for x, encode in (("k", _encode_k), ("v", _encode_v)):
        tail = s[x + "_tail"]
        rows = torch.where(is_old[None, :, :, None, None], tail[:, seq, token % (2 * BLOCK)], s[x + "_new"][:, seq, row])
        full = rows.view(L, B, blocks, BLOCK, Hkv, Dh)[:, b, j].transpose(2, 3).float()        # [L, blocks, Hkv, 64, Dh]
        codes, scale = encode(full)
        s[x + "_codes"][:, b, :, at] = codes.transpose(0, 1)
        s[x + "_scale"][:, b, :, at] = scale.transpose(0, 1)
        tail[:, b2, token[b2, t2] % (2 * BLOCK)] = rows[:, b2, t2]
    return _cache_outputs(s)


def _cache_outputs(s):
    """(Codes as they are stored, two to a byte: scales are powers of two, so every rounding is decided and equal values are equal bytes.)"""
    return {x + y: s[x + y] for x in "kv" for y in ("_codes", "_scale", "_tail")}


def _decoded(codes, scale):
    """Codes [.., 16] and their groups' scales [..] -> values [.., 32]."""
    value = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=DEV)
    x = value[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return torch.ldexp(x, (scale.int() - 127)[..., None])


def _plain_attend(s):
    c = s["case"]
    B, N, Hq, Dh = s["q"].shape
    Hkv, nblk = s["k_scale"].shape[1:3]
    G, J = Hq // Hkv, Dh // 64
    lens = s["lens"].long()
    full = lens // BLOCK * BLOCK
    K = _decoded(s["k_codes"].view(B, Hkv, nblk, 2, J, 2, 32, 16), s["k_scale"].view(B, Hkv, nblk, 2, 32, 2, J).permute(0, 1, 2, 5, 6, 3, 4))
    K = K.permute(0, 1, 2, 3, 6, 4, 5, 7).reshape(B, Hkv, -1, Dh)                              # t r, j h i
    V = _decoded(s["v_codes"].view(B, Hkv, nblk, Dh // 32, 2, 32, 16), s["v_scale"].view(B, Hkv, nblk, 2, 32, Dh // 32).permute(0, 1, 2, 5, 3, 4))
    V = V.view(B, Hkv, nblk, Dh // 32, 2, 32, 2, 4, 4).permute(0, 1, 2, 4, 7, 6, 8, 3, 5).reshape(B, Hkv, -1, Dh)      # u e4 h e1, d r
    seq, r = torch.arange(B, device=DEV)[:, None], torch.arange(BLOCK, device=DEV)
    half = (full % (2 * BLOCK))[:, None] + r
    K = torch.cat((K, s["k_tail"][seq, half].float().transpose(1, 2), s["k_tree"].float().transpose(1, 2)), 2)
    V = torch.cat((V, s["v_tail"][seq, half].float().transpose(1, 2), s["v_tree"].float().transpose(1, 2)), 2)
    seen = torch.cat((torch.arange(nblk * BLOCK, device=DEV) < full[:, None], full[:, None] + r < lens[:, None]), 1)
    seen = torch.cat((seen[:, None].expand(B, N, -1), _ancestors(s["parent"], c["depth"])), 2)
    q = s["q"].float().view(B, N, Hkv, G, Dh).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, Dh)
    score = torch.matmul(q, K.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(Dh)).view(B, Hkv, N, G, -1)
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = score.sub_(top).exp_()
    total = weight.sum(-1, keepdim=True)
    # keys that no row sees may hold anything: their values must not meet a weight of zero
    V = torch.where(seen.any(1)[:, None, :, None], V, 0.0)
    out = torch.matmul(weight.view(B, Hkv, N * G, -1), V).view(B, Hkv, N, G, Dh) / total
    got = {"out": out.permute(0, 2, 1, 3, 4).reshape(B, N, Hq, Dh).to(torch.bfloat16)}
    if c["lse"]:
        got["lse"] = (top + total.log())[..., 0].permute(0, 2, 1, 3).reshape(B, N, Hq)
    return got


# ---------------------------------------------------------------- one pass, as a user's program calls it

def _handle(s):
    """Shape, cache and workspace: what such a program makes once."""
    import paper_2512_23858_amd as ygg
    if "handle" in s:
        return ygg, s["handle"]
    c = s["case"]
    kind = c["kind"]
    depth, width = c.get("depth", 0), c.get("width", 1)
    prefix = c.get("prefix", 0) + c.get("new", 0)
    shape = ygg.Shape(batch=c["batch"], n_q_heads=c.get("q_heads", c.get("kv_heads", 1)), n_kv_heads=c.get("kv_heads", 1),
                      head_dim=c["head_dim"], depth=depth, width=width, n_nodes=c.get("prompt") or 1 + depth * width, vocab=1,
                      kv_dtype=ygg.F32 if c.get("dtype") == "f32" else ygg.BF16, softmax_scale=1.0 / math.sqrt(c["head_dim"]),
                      kv_capacity=prefix + depth + 1, max_seq_len=prefix)
    s["workspace"] = None
    if kind == "prompt":       # rows of q, rows of k and v, and the longest sequence's keys
        shape.n_nodes, shape.kv_capacity, shape.max_seq_len = s["q"].shape[0], s["k"].shape[0], s["longest"]
        if ygg.workspace_bytes(shape, ygg.OP_PROMPT_ATTENTION):
            s["workspace"] = ygg.new_workspace(shape, ygg.OP_PROMPT_ATTENTION)
    if kind in ("append", "attend"):
        shape.kv_dtype = ygg.FP4_BLOCK
        shape.kv_capacity = s["k_scale"].shape[-2] * BLOCK
        shape.max_seq_len = min(prefix, shape.kv_capacity - depth - 1)
        s["cache"] = ygg.Block4Cache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["k_tail"], s["v_tail"])
    if kind == "attend":
        s["workspace"] = ygg.new_workspace(shape, ygg.OP_ATTENTION_BLOCK4)
    s["handle"] = shape
    return ygg, shape


def _own_pass(s):
    ygg, shape = _handle(s)
    c = s["case"]
    if c["kind"] == "norm":
        where = dict(positions=s["positions"]) if c["prompt"] else dict(seq_lens=s["lens"], parent_idx=s["parent"])
        ygg.tree_norm_rotary(shape, s["q"], s["k"], s["q_out"], s["k_out"], s["q_weight"], s["k_weight"], s["frequencies"],
                             interleaved=c["interleaved"], eps=s["eps"], **where)
        return {"q": s["q_out"], "k": s["k_out"]}
    if c["kind"] == "prompt":
        ygg.prompt_attention(shape, s["q"], s["k"], s["v"], s["q_first"], s["q_len"], s["k_first"], s["k_len"], s["out"], s["lse"], s["workspace"])
    elif c["kind"] == "append":
        ygg.block4_append(shape, c["layers"], s["k_new"], s["v_new"], s["cache"], s["lens"], s["new"], rows=s.get("rows"))
        return _cache_outputs(s)
    else:
        ygg.tree_attention_block4(shape, s["q"], s["cache"], s["lens"], s["k_tree"], s["v_tree"], s["parent"], s["out"], s["lse"], s["workspace"])
    return {"out": s["out"], "lse": s["lse"]} if c["lse"] else {"out": s["out"]}


def run(state):
    if own:
        return _own_pass(state)
    return {"norm": _plain_norm, "prompt": _plain_prompt, "append": _plain_append, "attend": _plain_attend}[state["case"]["kind"]](state)


# ---------------------------------------------------------------- the definitions in 64 bits

def _walk(parent, i):
    """Node i and its ancestors, the root last."""
    out = []
    while i >= 0:
        out.append(i)
        i = int(parent[i])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "prompt": _exact_prompt, "append": _exact_append, "attend": _exact_attend}[case["kind"]](s, case)


def _exact_norm(s, case):
    parent, lens = s["parent"].cpu().numpy(), s["lens"].cpu().numpy()
    if case["prompt"]:
        position = s["positions"].cpu().numpy()
    else:
        position = np.array([[lens[b] + len(_walk(parent[b], i)) - 1 for i in range(parent.shape[1])] for b in range(case["batch"])])
    turn = torch.from_numpy(position.astype(np.float64)).to(DEV)[..., None] * s["frequencies"]
    turn = torch.polar(torch.ones_like(turn), turn)[:, :, None]                                # unit complex numbers
    r = case["rotary_dim"]

    def turned(x, weight):
        out = x.double()
        out = out / torch.sqrt((out * out).sum(-1, keepdim=True) / out.shape[-1] + s["eps"]) * weight.double()
        first = slice(0, r, 2) if case["interleaved"] else slice(0, r // 2)
        second = slice(1, r, 2) if case["interleaved"] else slice(r // 2, r)
        z = torch.complex(out[..., first], out[..., second]) * turn
        out[..., first], out[..., second] = z.real, z.imag
        return out
    return {"q": turned(s["q"], s["q_weight"]), "k": turned(s["k"], s["k_weight"])}


def _exact_prompt(s, case):
    T, Hq, Dh = s["q"].shape
    G = Hq // case["kv_heads"]
    out = torch.empty((T, Hq, Dh), dtype=torch.float64, device=DEV)
    lse = torch.empty((T, Hq), dtype=torch.float64, device=DEV)
    for q0, n, k0, m in zip(*(s[x].tolist() for x in ("q_first", "q_len", "k_first", "k_len"))):
        hidden = torch.ones((n, m), dtype=torch.bool, device=DEV).triu(m - n + 1)
        for h in range(Hq):
            q, k, v = s["q"][q0:q0 + n, h].double(), s["k"][k0:k0 + m, h // G].double(), s["v"][k0:k0 + m, h // G].double()
            score = (q @ k.T / math.sqrt(Dh)).masked_fill_(hidden, -math.inf)
            lse[q0:q0 + n, h] = torch.logsumexp(score, 1)
            out[q0:q0 + n, h] = torch.exp(score - lse[q0:q0 + n, h, None]) @ v
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def _stored_at(case, which):
    """[64, Dh]: (index of the 4-bit code, low half of a byte first; index of the scale) at which token t and dimension d are stored."""
    Dh = case["head_dim"]
    t, d = np.meshgrid(np.arange(64), np.arange(Dh), indexing="ij")
    if which == "k":
        chunk, lane, i = t // 32 * (Dh // 64) + d // 64, d // 32 % 2 * 32 + t % 32, d % 32
    else:
        chunk, lane, i = d // 32, t // 32 * 32 + d % 32, t // 4 % 2 * 16 + t % 32 // 8 * 4 + t % 4
    return torch.from_numpy(chunk * 2048 + lane * 32 + i).to(DEV), torch.from_numpy(lane * (Dh // 32) + chunk).to(DEV)


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_append(s, case):
    new, end = s["new"].tolist(), s["lens"].tolist()
    got = {x + y: s[x + y].double() if y == "_tail" else s[x + y].clone() for x in "kv" for y in ("_codes", "_scale", "_tail")}
    levels = torch.tensor(_E2M1, dtype=torch.float64, device=DEV)
    for b in range(case["batch"]):
        old = end[b] - new[b]
        row = s["rows"][b, :new[b]].long() if "rows" in s else torch.arange(new[b], device=DEV)
        for x in "kv":
            code_at, scale_at = _stored_at(case, x)
            first = old // BLOCK * BLOCK
            rows = torch.cat((s[x + "_tail"][:, b, first % 128:first % 128 + old - first], s[x + "_new"][:, b, row]), 1)     # tokens first .. end - 1
            for at in range(first, end[b] // BLOCK * BLOCK, BLOCK):
                block = rows[:, at - first:at - first + BLOCK].transpose(1, 2).double()        # [L, Hkv, 64, Dh]
                lead = block.shape[:2]
                amax = torch.zeros((*lead, 2 * case["head_dim"]), dtype=torch.float64, device=DEV)
                amax.scatter_reduce_(-1, scale_at.flatten().expand(*lead, -1), block.abs().flatten(-2), "amax")
                scale = torch.ceil(torch.log2((amax / 7).clamp(min=2.0 ** LOWEST)) - 1e-12)
                y = block / torch.exp2(scale[..., scale_at])
                away = (y.abs()[..., None] - levels).abs()
                near = away.argmin(-1)                                                         # (the first of equals: the lower code)
                tie = (near < 7) & (away.gather(-1, near[..., None])[..., 0] == away.gather(-1, (near + 1).clamp(max=7)[..., None])[..., 0])
                nibble = near + (tie & (near % 2 == 1)).long() + 8 * torch.signbit(y).long()
                flat = torch.empty((*lead, 64 * case["head_dim"]), dtype=torch.long, device=DEV)
                flat[..., code_at.flatten()] = nibble.flatten(-2)
                got[x + "_codes"][:, b, :, at // BLOCK] = (flat[..., ::2] + 16 * flat[..., 1::2]).to(torch.uint8)
                got[x + "_scale"][:, b, :, at // BLOCK] = (scale + 127).to(torch.uint8)
            at = max(end[b] // BLOCK * BLOCK, old)
            here = torch.arange(at, end[b], device=DEV)
            got[x + "_tail"][:, b, here % 128] = rows[:, here - first].double()
    return got


def _exact_attend(s, case):
    B, N, Hq, Dh = s["q"].shape
    Hkv = case["kv_heads"]
    G = Hq // Hkv
    parent, lens = s["parent"].cpu().numpy(), s["lens"].tolist()
    out = torch.empty((B, N, Hq, Dh), dtype=torch.float64, device=DEV)
    lse = torch.empty((B, N, Hq), dtype=torch.float64, device=DEV)
    value = torch.tensor(_E2M1 + tuple(-x for x in _E2M1), dtype=torch.float64, device=DEV)
    where = {x: _stored_at(case, x) for x in "kv"}
    for b in range(B):
        n_full, first = lens[b] // BLOCK, lens[b] // BLOCK * BLOCK
        hidden = torch.ones((N, N), dtype=torch.bool)
        for i in range(N):
            hidden[i, _walk(parent[b], i)] = False
        hidden = torch.cat((torch.zeros((N, lens[b]), dtype=torch.bool), hidden), 1).to(DEV).repeat_interleave(G, 0)
        for g in range(Hkv):
            kv = []
            for x in "kv":
                code_at, scale_at = where[x]
                byte = s[x + "_codes"][b, g, :n_full][:, code_at // 2].long()
                blocks = value[torch.where(code_at % 2 == 0, byte % 16, byte // 16)] * torch.exp2(s[x + "_scale"][b, g, :n_full][:, scale_at].double() - 127)
                tail = s[x + "_tail"][b, first % 128:first % 128 + lens[b] - first, g].double()
                kv.append(torch.cat((blocks.reshape(-1, Dh), tail, s[x + "_tree"][b, :, g].double())))
            q = s["q"][b, :, g * G:(g + 1) * G].double().reshape(N * G, Dh)
            score = (q @ kv[0].T / math.sqrt(Dh)).masked_fill(hidden, -math.inf)
            norm = torch.logsumexp(score, 1)
            out[b, :, g * G:(g + 1) * G] = (torch.exp(score - norm[:, None]) @ kv[1]).view(N, G, Dh)
            lse[b, :, g * G:(g + 1) * G] = norm.view(N, G)
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}
