"""Operators around the tree-verification calls, each in its plain form and as the library's own call.

  rotary  rotary positions of the queries and keys of a tree's nodes (position = confirmed length + depth) or of a prompt
  append  new K/V rows into the 8-bit block cache: the open block of 64 tokens stays in bf16, full blocks become E4M3 codes
  attend  tree attention over that cache; the tree's own K/V are bf16
  logits  penalties, biases and grammar masks on the verifier's logits, node by node, with the first maximum of each row

A case is a dict of plain values; listed() names the fixed ones, draw() gives more of the same ranges.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEV = "cuda:0"
BLOCK = 64
PROMPT = -2**31      # the sign bit of a token's count: it occurs in the prompt


def _rotary(name, batch, heads, head_dim, depth, width, prefix, rotary_dim=0, interleaved=False, dtype="bf16", scaling="none",
            fused=False, prompt=0):
    """prompt: that many explicit positions per sequence instead of a tree; fused: q and k are parts of one QKV projection."""
    return dict(name=name, kind="rotary", batch=batch, q_heads=heads[0], kv_heads=heads[1], head_dim=head_dim, depth=depth, width=width,
                prefix=prefix, rotary_dim=rotary_dim or head_dim, interleaved=interleaved, dtype=dtype, scaling=scaling, fused=fused,
                prompt=prompt)


def _append(name, batch, kv_heads, head_dim, depth, width, prefix, layers, new=0):
    """new: a prompt's tokens, all of them, behind an empty cache (0: the accepted path of a tree of depth x width nodes behind `prefix`)."""
    return dict(name=name, kind="append", batch=batch, kv_heads=kv_heads, head_dim=head_dim, depth=depth, width=width, prefix=prefix,
                layers=layers, new=new)


def _attend(name, batch, heads, head_dim, depth, width, prefix, shortest=0, lse=False):
    return dict(name=name, kind="attend", batch=batch, q_heads=heads[0], kv_heads=heads[1], head_dim=head_dim, depth=depth, width=width,
                prefix=prefix, shortest=shortest or prefix, lse=lse)


def _logits(name, batch, depth, width, vocab, history, dtype="bf16", masks=0, bias=False, write=True, best=True, fresh=False):
    """history: confirmed tokens per sequence, half of them the prompt's; fresh: they are counted within the pass (a request's first step)."""
    return dict(name=name, kind="logits", batch=batch, depth=depth, width=width, vocab=vocab, history=history, dtype=dtype, masks=masks,
                bias=bias, write=write, best=best, fresh=fresh)


def listed():
    return [
        # one decoding step of a small fp32 model: one token, launch latency
        _rotary("rotary one token", 1, (4, 4), 64, 0, 1, 128, dtype="f32"),
        # the tree of a 70B-shaped serving batch, interleaved pairs, long-context frequencies, straight out of the QKV projection
        _rotary("rotary 70B batch 16", 16, (64, 8), 128, 6, 8, 8192, interleaved=True, scaling="bands", fused=True),
        # a prompt of two requests, half of each head rotated
        _rotary("rotary prompt 8B", 2, (32, 8), 128, 0, 1, 131072, rotary_dim=64, scaling="linear", prompt=8191),
        # the accepted path of each of sixteen requests into the caches of 32 layers; a few fill their block
        _append("append accepted 8B", 16, 8, 128, 6, 8, 511, 32),
        # a prompt of 8191 tokens into the caches of four layers
        _append("append prompt 8B", 1, 8, 128, 0, 1, 0, 4, new=8191),
        # plain decoding, one token each, sixteen ragged requests: the stream of the cache
        _attend("attend one token batch 16", 16, (32, 8), 128, 0, 1, 8192, shortest=512),
        # the drafter's own attention over its tree, ragged, log-sum-exps wanted
        _attend("attend drafter batch 3", 3, (12, 12), 64, 8, 8, 2047, shortest=301, lse=True),
        # verification behind eight long prefixes, one query head per K/V head
        _attend("attend 7B batch 8", 8, (32, 32), 128, 6, 8, 4096),
        # long context, widest tree: the matrix cores
        _attend("attend long context", 1, (32, 8), 128, 10, 32, 32768),
        # a small vocabulary, a request's first step: counting included
        _logits("logits first step", 1, 3, 4, 1000, 128, dtype="f32", fresh=True),
        # an 8B verifier's rows of 128k logits in bf16, everything on, constrained logits and their maxima wanted
        _logits("logits 8B", 1, 8, 16, 128256, 4096, masks=16, bias=True),
        # sixteen requests, only the tokens wanted (acceptance), a vocabulary that fits no alignment
        _logits("logits batch 16", 16, 6, 8, 32003, 2048, dtype="f32", masks=64, write=False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


_HEADS = [((32, 32), 128), ((40, 40), 128), ((32, 8), 128), ((64, 8), 128), ((12, 12), 64), ((32, 8), 64)]


def draw(rng):
    kind = rng.choice(["rotary", "append", "attend", "attend", "logits"])
    batch = 1 if rng.random() < 0.4 else _log_int(rng, 2, 16)
    depth, width = rng.randint(2, 10), _log_int(rng, 2, 32)
    if rng.random() < 0.25:
        depth, width = 0, 1
    prefix = _log_int(rng, 64, 32768)
    heads, head_dim = rng.choice(_HEADS)
    n = 1 + depth * width
    if kind == "rotary":
        rotary_dim = rng.choice([head_dim, head_dim, head_dim // 2, head_dim // 4])
        prompt = _log_int(rng, 2, 16384 // batch) if rng.random() < 0.4 else 0
        case = _rotary("", batch, heads, head_dim, depth, width, prefix + prompt, rotary_dim, rng.random() < 0.5,
                       rng.choice(["bf16", "bf16", "f32"]), rng.choice(["none", "linear", "bands"]), rng.random() < 0.5, prompt)
    elif kind == "append":
        layers = rng.choice([1, 4, 32])
        if rng.random() < 0.5:
            case = _append("", batch, heads[1], head_dim, depth, width, min(prefix, 2000), layers)
        else:
            case = _append("", batch, heads[1], head_dim, 0, 1, 0, layers, new=min(_log_int(rng, 2, 16384), 2048 if layers > 4 else 16384))
    elif kind == "attend":
        case = _attend("", batch, heads, head_dim, depth, width, prefix, rng.choice([0, max(1, prefix // 16)]), rng.random() < 0.3)
    else:
        vocab = _log_int(rng, 1000, 128256)
        if batch * n * vocab > 32 << 20:
            batch = max(1, (32 << 20) // (n * vocab))
        write = rng.random() < 0.6
        case = _logits("", batch, depth, width, vocab, min(prefix, 8192), rng.choice(["bf16", "f32"]), rng.choice([0, batch, 8 * batch]),
                       rng.random() < 0.5, write, not write or rng.random() < 0.5, rng.random() < 0.2)
    while _cost(case) > 1.6e-4:        # stay below the largest listed cases
        for key in ("layers", "batch", "prompt", "new", "prefix"):
            if case.get(key, 0) > 1:
                case[key] //= 2
                case["shortest"] = min(case.get("shortest", 0), case.get("prefix", 0))
                break
        if case["kind"] != "attend":
            case.pop("shortest", None)
    del case["name"]
    return case


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15)


def _elem(case):
    return 4 if case["dtype"] == "f32" else 2


def _lens(case):
    """The batch's confirmed lengths, evenly spread from the shortest to the longest (their order comes from the seed)."""
    if case["kind"] == "attend":
        return np.rint(np.linspace(case["prefix"], case["shortest"], case["batch"])).astype(np.int64)
    return np.maximum(case["prefix"] - np.arange(case["batch"], dtype=np.int64), 0)


def _accepted(case):
    """Accepted tokens of each sequence: the whole prompt, or one to depth + 1 tokens of a tree."""
    if case["new"]:
        return np.full(case["batch"], case["new"], np.int64)
    return 1 + np.arange(case["batch"], dtype=np.int64) % (case["depth"] + 1)


def work(case):
    B, D, W = case["batch"], case["depth"], case["width"]
    N = 1 + D * W
    if case["kind"] == "rotary":
        tokens = B * (case["prompt"] or N)
        values = tokens * (case["q_heads"] + case["kv_heads"])
        return {"bytes": 2.0 * values * case["head_dim"] * _elem(case), "flops": 3.0 * values * case["rotary_dim"]}
    if case["kind"] == "append":
        old, new = _lens(case), _accepted(case)
        full = ((old + new) // BLOCK - old // BLOCK) * BLOCK                                  # tokens that become codes
        tail = np.where(full > 0, (old + new) % BLOCK, new)                                   # rows that are left open
        reread = np.where(full > 0, old % BLOCK, 0)
        row = 2.0 * case["layers"] * case["kv_heads"] * case["head_dim"]
        return {"bytes": row * float((2 * new + 2 * reread + full + 2 * tail).sum()), "flops": 3.0 * row * float(full.sum())}
    if case["kind"] == "attend":
        lens = _lens(case).astype(float)
        full = lens // BLOCK * BLOCK
        row = case["kv_heads"] * case["head_dim"]
        nbytes = 2.0 * row * float(full.sum() + 2 * (lens - full).sum() + 2 * B * N) + 4.0 * B * N * case["q_heads"] * case["head_dim"]
        keys = N * float(lens.sum()) + B * (1 + W * D * (D + 3) / 2)
        return {"bytes": nbytes, "flops": 4.0 * case["q_heads"] * case["head_dim"] * keys}
    rows, V = B * N, case["vocab"]
    nbytes = float(rows) * V * (_elem(case) + (4 if case["write"] else 0)) + 4.0 * B * V * (1 + case["bias"]) + case["masks"] * V / 8
    return {"bytes": nbytes + case["fresh"] * 4.0 * B * (V + case["history"]), "flops": 6.0 * rows * V}


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


def _frequencies(case):
    """Radians per position of each rotated pair, in 64 bits; scaled for contexts longer than the model was trained on."""
    pairs = case["rotary_dim"] // 2
    f = 10000.0 ** (-np.arange(pairs) / pairs)
    if case["scaling"] == "linear":
        f = f / 4.0
    if case["scaling"] == "bands":       # short wavelengths stay, long ones are stretched eightfold, a ramp between
        turns = 8192 * f / (2 * np.pi)
        keep = np.clip((turns - 1.0) / 3.0, 0.0, 1.0)
        f = f * keep + f / 8.0 * (1 - keep)
    return f


def _k_order(x):
    """[.., 64 tokens, Dh] -> the order in which a block of K is stored, [.., 64 * Dh]: 32 tokens by 64 dimensions after another, each
    as the operand of a matrix instruction (16 bytes of 64 lanes: token and half of the dimensions)."""
    Dh = x.shape[-1]
    x = x.reshape(*x.shape[:-2], 2, 32, Dh // 64, 2, 2, 16)                  # tokens: t r   dimensions: j h part e
    n = x.dim() - 6
    return x.permute(*range(n), n, n + 2, n + 4, n + 3, n + 1, n + 5).reshape(*x.shape[:n], 64 * Dh)


def _v_order(x):
    """[.., 64 tokens, Dh] -> the order in which a block of V is stored: 32 dimensions after another, tokens in the order in which the
    scores of a 32 x 32 matrix instruction lie in its accumulator."""
    Dh = x.shape[-1]
    x = x.reshape(*x.shape[:-2], 2, 4, 2, 4, Dh // 32, 32)                   # tokens: part e4 h e1   dimensions: d r
    n = x.dim() - 6
    return x.permute(*range(n), n + 4, n, n + 2, n + 5, n + 1, n + 3).reshape(*x.shape[:n], 64 * Dh)


def _encode(x, order):
    """Blocks [.., 64, Dh] in fp32 -> (codes in storage order, scales)."""
    amax = x.abs().amax(dim=(-2, -1))
    scale = torch.where(amax > 0, amax / 448.0, torch.ones_like(amax))
    return order((x / scale[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)), scale


def _cache(case, lead, nblk, gen, fill):
    """Codes, scales and open blocks of a cache: [*lead, Hkv, nblk, 64 * Dh], [*lead, Hkv, nblk], [*lead, 128, Hkv, Dh]."""
    Hkv, Dh = case["kv_heads"], case["head_dim"]
    s = {}
    for x, order in (("k", _k_order), ("v", _v_order)):
        if fill:
            s[x + "_codes"], s[x + "_scale"] = _encode(_normal(gen, (*lead, Hkv, nblk, BLOCK, Dh), torch.float32), order)
        else:
            s[x + "_codes"] = torch.zeros((*lead, Hkv, nblk, BLOCK * Dh), dtype=torch.uint8, device=DEV)
            s[x + "_scale"] = torch.ones((*lead, Hkv, nblk), dtype=torch.float32, device=DEV)
        s[x + "_tail"] = _normal(gen, (*lead, 2 * BLOCK, Hkv, Dh), torch.bfloat16)
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    host = np.random.default_rng(seed)
    B, D, W = case["batch"], case["depth"], case["width"]
    N = 1 + D * W
    kind = case["kind"]
    s = dict(case=case)
    parent = np.stack([_tree(host, D, W) for _ in range(B)])
    s["parent"] = _ints(parent)

    if kind == "rotary":
        T = case["prompt"] or N
        Hq, Hkv, Dh = case["q_heads"], case["kv_heads"], case["head_dim"]
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        if case["fused"]:
            qkv = _normal(gen, (B, T, Hq + 2 * Hkv, Dh), dt)
            s["q"], s["k"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]
        else:
            s["q"], s["k"] = _normal(gen, (B, T, Hq, Dh), dt), _normal(gen, (B, T, Hkv, Dh), dt)
        s["q_out"], s["k_out"] = (torch.empty((B, T, h, Dh), dtype=dt, device=DEV) for h in (Hq, Hkv))
        s["frequencies"] = torch.from_numpy(_frequencies(case)).to(DEV)
        s["lens"] = _ints(host.permutation(_lens(case)))
        # a prompt is the last part of a context as long as `prefix`
        s["positions"] = _ints(_lens(case)[:, None] - T + np.arange(T)[None]).clamp_(min=0) if case["prompt"] else None

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
        nblk = -(-(case["prefix"] + (case["new"] or D + 1)) // BLOCK)
        s |= _cache(case, (L, B), nblk, gen, fill=False)
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

    if kind == "logits":
        V, H = case["vocab"], case["history"]
        s["logits"] = _normal(gen, (B, N, V), torch.float32).mul_(3.0).to(torch.float32 if case["dtype"] == "f32" else torch.bfloat16)
        # text repeats itself: half of a sequence's tokens come from a small part of the vocabulary
        text = np.where(host.random((B, H + N)) < 0.5, host.integers(0, max(V // 50, 1), (B, H + N)), host.integers(0, V, (B, H + N)))
        s["token"] = _ints(text[:, H:])
        s["history"] = _ints(text[:, :H])
        s["prompt_len"], s["reply_len"] = _ints(np.full(B, H // 2)), _ints(np.full(B, H - H // 2))
        counts = np.zeros((B, V), np.int64)
        if not case["fresh"]:
            for b in range(B):
                counts[b] = np.bincount(text[b, H // 2:H], minlength=V)
                counts[b, text[b, :H // 2]] += PROMPT
        s["counts"] = _ints(counts)
        s["repetition"] = torch.from_numpy(host.uniform(1.0, 1.3, B).astype(np.float32)).to(DEV)
        s["presence"], s["frequency"] = (torch.from_numpy(host.uniform(0.0, 0.5, B).astype(np.float32)).to(DEV) for _ in range(2))
        s["bias"] = None
        if case["bias"]:
            bias = torch.zeros((B, V), device=DEV)
            at = torch.rand((B, V), device=DEV, generator=gen).topk(300).indices      # 300 different tokens each
            s["bias"] = bias.scatter_(1, at, _normal(gen, (B, 300), torch.float32))
        s["masks"] = s["mask_index"] = None
        if case["masks"]:
            s["masks"] = torch.randint(-2**31, 2**31, (case["masks"], (V + 31) // 32), dtype=torch.int32, device=DEV, generator=gen)
            s["mask_index"] = _ints(host.integers(-1, case["masks"], (B, N)))      # -1: that node is free
        s["out"] = torch.empty((B, N, V), dtype=torch.float32, device=DEV) if case["write"] else None
        s["best"] = torch.empty((B, N), dtype=torch.int32, device=DEV) if case["best"] else None
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


def _plain_rotary(s):
    c = s["case"]
    if s["positions"] is not None:
        position = s["positions"].double()
    else:
        position = s["lens"][:, None].double() + _ancestors(s["parent"], c["depth"]).sum(-1) - 1
    angle = position[..., None] * s["frequencies"]
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    r = c["rotary_dim"]

    def rotate(x):
        turned, rest = x[..., :r].float(), x[..., r:]
        a, b = (turned[..., ::2], turned[..., 1::2]) if c["interleaved"] else (turned[..., :r // 2], turned[..., r // 2:])
        a, b = a * cos - b * sin, b * cos + a * sin
        turned = torch.stack((a, b), -1).flatten(-2) if c["interleaved"] else torch.cat((a, b), -1)
        return torch.cat((turned.to(x.dtype), rest), -1)
    return {"q": rotate(s["q"]), "k": rotate(s["k"])}


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
    for x, order in (("k", _k_order), ("v", _v_order)):
        tail = s[x + "_tail"]
        rows = torch.where(is_old[None, :, :, None, None], tail[:, seq, token % (2 * BLOCK)], s[x + "_new"][:, seq, row])
        full = rows.view(L, B, blocks, BLOCK, Hkv, Dh)[:, b, j].transpose(2, 3).float()        # [L, blocks, Hkv, 64, Dh]
        codes, scale = _encode(full, order)
        s[x + "_codes"][:, b, :, at] = codes.transpose(0, 1)
        s[x + "_scale"][:, b, :, at] = scale.transpose(0, 1)
        tail[:, b2, token[b2, t2] % (2 * BLOCK)] = rows[:, b2, t2]
    return _cache_outputs(s)


def _cache_outputs(s):
    return {x + y: s[x + y].view(torch.float8_e4m3fn) if y == "_codes" else s[x + y] for x in "kv" for y in ("_codes", "_scale", "_tail")}


def _plain_attend(s):
    c = s["case"]
    B, N, Hq, Dh = s["q"].shape
    Hkv, nblk = s["k_scale"].shape[1:]
    G, J = Hq // Hkv, Dh // 64
    lens = s["lens"].long()
    full = lens // BLOCK * BLOCK
    K = s["k_codes"].view(torch.float8_e4m3fn).view(B, Hkv, nblk, 2, J, 2, 2, 32, 16).float().permute(0, 1, 2, 3, 7, 4, 6, 5, 8)
    V = s["v_codes"].view(torch.float8_e4m3fn).view(B, Hkv, nblk, Dh // 32, 2, 2, 32, 4, 4).float().permute(0, 1, 2, 4, 7, 5, 8, 3, 6)
    K = K.reshape(B, Hkv, nblk, BLOCK, Dh) * s["k_scale"][..., None, None]
    V = V.reshape(B, Hkv, nblk, BLOCK, Dh) * s["v_scale"][..., None, None]
    seq, r = torch.arange(B, device=DEV)[:, None], torch.arange(BLOCK, device=DEV)
    half = (full % (2 * BLOCK))[:, None] + r
    K = torch.cat((K.reshape(B, Hkv, -1, Dh), s["k_tail"][seq, half].float().transpose(1, 2), s["k_tree"].float().transpose(1, 2)), 2)
    V = torch.cat((V.reshape(B, Hkv, -1, Dh), s["v_tail"][seq, half].float().transpose(1, 2), s["v_tree"].float().transpose(1, 2)), 2)
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


def _plain_logits(s):
    c = s["case"]
    B, N, V = s["logits"].shape
    counts = s["counts"]
    if c["fresh"]:
        h = c["history"]
        counts = torch.zeros((B, V), dtype=torch.int32, device=DEV)
        counts.scatter_add_(1, s["history"][:, h // 2:].long(), torch.ones_like(s["history"][:, h // 2:]))
        given = torch.zeros((B, V), dtype=torch.bool, device=DEV).scatter_(1, s["history"][:, :h // 2].long(), True)
        counts = torch.where(given, counts + PROMPT, counts)
    on = _ancestors(s["parent"], c["depth"])                                                   # [B, N, N]
    path = torch.zeros((B, N, V), dtype=torch.float32, device=DEV)
    path.scatter_add_(2, s["token"].long()[:, None].expand(B, N, N), on.float())
    times = path + (counts & 0x7fffffff).float()[:, None]
    seen = (path > 0) | (counts != 0)[:, None]
    x = s["logits"].float()
    factor, presence, frequency = (s[y][:, None, None] for y in ("repetition", "presence", "frequency"))
    x = torch.where(seen, torch.where(x > 0, x / factor, x * factor), x)
    x = x - frequency * times
    x = x - presence * (times > 0)
    if s["bias"] is not None:
        x = x + s["bias"][:, None]
    if s["masks"] is not None:
        bits = (s["masks"][:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
        allowed = bits.flatten(1)[:, :V].bool()[s["mask_index"].long().clamp(min=0)] | (s["mask_index"] < 0)[..., None]
        x = torch.where(allowed, x, -math.inf)
    got = {}
    if c["write"]:
        got["logits"] = x
    if c["best"]:
        token = torch.arange(V, device=DEV, dtype=torch.int32)
        got["best"] = torch.where(x == x.amax(-1, keepdim=True), token, V).amin(-1).int()
    if c["fresh"]:
        got["counts"] = counts
    return got


# ---------------------------------------------------------------- one pass, as a user's program calls it

def _handle(s):
    """Shape, cache and workspace: what such a program makes once."""
    import paper_2512_23858_amd as ygg
    if "handle" in s:
        return ygg, s["handle"]
    c = s["case"]
    kind = c["kind"]
    prefix = c.get("prefix", 0) + c.get("new", 0)
    tree = 1 + c["depth"] * c["width"]
    shape = ygg.Shape(batch=c["batch"], n_q_heads=c.get("q_heads", c.get("kv_heads", 1)), n_kv_heads=c.get("kv_heads", 1),
                      head_dim=c.get("head_dim", 64), depth=c["depth"], width=c["width"], n_nodes=c.get("prompt") or tree,
                      vocab=c.get("vocab", 1), kv_dtype=ygg.F32 if c.get("dtype") == "f32" else ygg.BF16,
                      softmax_scale=1.0 / math.sqrt(c.get("head_dim", 64)), kv_capacity=prefix + c["depth"] + 1, max_seq_len=prefix)
    if kind in ("append", "attend"):
        shape.kv_dtype = ygg.FP8_BLOCK
        shape.kv_capacity = s["k_scale"].shape[-1] * BLOCK
        shape.max_seq_len = min(prefix, shape.kv_capacity - c["depth"] - 1)
        s["cache"] = ygg.BlockCache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["k_tail"], s["v_tail"])
    s["workspace"] = None
    if kind == "attend":
        s["workspace"] = ygg.new_workspace(shape, ygg.OP_ATTENTION_BLOCK8)
    if kind == "logits" and c["best"]:
        s["workspace"] = ygg.new_workspace(shape, ygg.OP_CONSTRAIN)
    s["handle"] = shape
    return ygg, shape


def _own_pass(s):
    ygg, shape = _handle(s)
    c = s["case"]
    if c["kind"] == "rotary":
        where = dict(positions=s["positions"]) if c["prompt"] else dict(seq_lens=s["lens"], parent_idx=s["parent"])
        ygg.tree_rotary(shape, s["q"], s["k"], s["q_out"], s["k_out"], s["frequencies"], interleaved=c["interleaved"], **where)
        return {"q": s["q_out"], "k": s["k_out"]}
    if c["kind"] == "append":
        ygg.block8_append(shape, c["layers"], s["k_new"], s["v_new"], s["cache"], s["lens"], s["new"], rows=s.get("rows"))
        return _cache_outputs(s)
    if c["kind"] == "attend":
        ygg.tree_attention_block8(shape, s["q"], s["cache"], s["lens"], s["k_tree"], s["v_tree"], s["parent"], s["out"], s["lse"], s["workspace"])
        return {"out": s["out"], "lse": s["lse"]} if c["lse"] else {"out": s["out"]}
    if c["fresh"]:
        h = c["history"]
        s["counts"].zero_()
        ygg.count_tokens(shape, s["history"], s["prompt_len"], s["counts"], prompt=True)
        ygg.count_tokens(shape, s["history"], s["reply_len"], s["counts"], first=h // 2)
    ygg.constrain_logits(shape, s["logits"], s["parent"], s["token"], out=s["out"], best=s["best"], counts=s["counts"],
                         repetition=s["repetition"], presence=s["presence"], frequency=s["frequency"], bias=s["bias"], masks=s["masks"],
                         mask_index=s["mask_index"], workspace=s["workspace"])
    got = {}
    if c["write"]:
        got["logits"] = s["out"]
    if c["best"]:
        got["best"] = s["best"]
    if c["fresh"]:
        got["counts"] = s["counts"]
    return got


def run(state):
    if own:
        return _own_pass(state)
    return {"rotary": _plain_rotary, "append": _plain_append, "attend": _plain_attend, "logits": _plain_logits}[state["case"]["kind"]](state)


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
    return {"rotary": _exact_rotary, "append": _exact_append, "attend": _exact_attend, "logits": _exact_logits}[case["kind"]](s, case)


def _exact_rotary(s, case):
    parent, lens = s["parent"].cpu().numpy(), s["lens"].cpu().numpy()
    if case["prompt"]:
        position = s["positions"].cpu().numpy()
    else:
        position = np.array([[lens[b] + len(_walk(parent[b], i)) - 1 for i in range(parent.shape[1])] for b in range(case["batch"])])
    turn = torch.from_numpy(position.astype(np.float64)).to(DEV)[..., None] * s["frequencies"]
    turn = torch.polar(torch.ones_like(turn), turn)[:, :, None]                                # unit complex numbers
    r = case["rotary_dim"]

    def rotate(x):
        out = x.double()
        first = slice(0, r, 2) if case["interleaved"] else slice(0, r // 2)
        second = slice(1, r, 2) if case["interleaved"] else slice(r // 2, r)
        z = torch.complex(out[..., first], out[..., second]) * turn
        out[..., first], out[..., second] = z.real, z.imag
        return out
    return {"q": rotate(s["q"]), "k": rotate(s["k"])}


def _nearest_e4m3(x):
    """The nearest E4M3 value (ties to even, magnitudes up to 448) of 64-bit numbers."""
    exponent = torch.frexp(x.abs())[1].clamp(min=-5) - 1
    step = torch.ldexp(torch.ones_like(x), exponent - 3)
    return (x / step).round() * step


def _stored_at(case, which):
    """Byte of a block at which (token, dimension) is stored, [64, Dh]."""
    Dh = case["head_dim"]
    t, d = np.meshgrid(np.arange(64), np.arange(Dh), indexing="ij")
    if which == "k":
        chunk = (t // 32 * (Dh // 64) + d // 64) * 2 + d // 16 % 2
        lane = d // 32 % 2 * 32 + t % 32
        byte = d % 16
    else:
        chunk = d // 32 * 2 + t // 32
        lane = t // 4 % 2 * 32 + d % 32
        byte = t % 32 // 8 * 4 + t % 4
    return torch.from_numpy(chunk * 1024 + lane * 16 + byte).to(DEV)


def _exact_append(s, case):
    new, end = s["new"].tolist(), s["lens"].tolist()
    got = {x + y: s[x + y].view(torch.float8_e4m3fn).double() if y == "_codes" else s[x + y].double()
           for x in "kv" for y in ("_codes", "_scale", "_tail")}
    for b in range(case["batch"]):
        old = end[b] - new[b]
        row = s["rows"][b, :new[b]].long() if "rows" in s else torch.arange(new[b], device=DEV)
        for x in "kv":
            tail, fresh = s[x + "_tail"][:, b].double(), s[x + "_new"][:, b, row].double()
            first = old // BLOCK * BLOCK
            rows = torch.cat((tail[:, first % 128:first % 128 + old - first], fresh), 1)       # tokens first .. end - 1
            where = _stored_at(case, x).flatten()
            for at in range(first, end[b] // BLOCK * BLOCK, BLOCK):
                block = rows[:, at - first:at - first + BLOCK].transpose(1, 2)                 # [L, Hkv, 64, Dh]
                scale = block.abs().amax((-2, -1)) / 448
                got[x + "_scale"][:, b, :, at // BLOCK] = scale
                got[x + "_codes"][:, b, :, at // BLOCK, where] = _nearest_e4m3(block / scale[..., None, None]).flatten(-2)
            at = max(end[b] // BLOCK * BLOCK, old)
            here = torch.arange(at, end[b], device=DEV)
            got[x + "_tail"][:, b, here % 128] = rows[:, here - first]
    return got


def _exact_attend(s, case):
    B, N, Hq, Dh = s["q"].shape
    Hkv = case["kv_heads"]
    G = Hq // Hkv
    parent, lens = s["parent"].cpu().numpy(), s["lens"].tolist()
    out = torch.empty((B, N, Hq, Dh), dtype=torch.float64, device=DEV)
    lse = torch.empty((B, N, Hq), dtype=torch.float64, device=DEV)
    at = {x: _stored_at(case, x) for x in "kv"}
    for b in range(B):
        n_full, first = lens[b] // BLOCK, lens[b] // BLOCK * BLOCK
        hidden = torch.ones((N, N), dtype=torch.bool)
        for i in range(N):
            hidden[i, _walk(parent[b], i)] = False
        hidden = torch.cat((torch.zeros((N, lens[b]), dtype=torch.bool), hidden), 1).to(DEV).repeat_interleave(G, 0)
        for g in range(Hkv):
            kv = []
            for x in "kv":
                blocks = s[x + "_codes"][b, g, :n_full].view(torch.float8_e4m3fn).double()[:, at[x]] * s[x + "_scale"][b, g, :n_full, None, None].double()
                tail = s[x + "_tail"][b, first % 128:first % 128 + lens[b] - first, g].double()
                kv.append(torch.cat((blocks.reshape(-1, Dh), tail, s[x + "_tree"][b, :, g].double())))
            q = s["q"][b, :, g * G:(g + 1) * G].double().reshape(N * G, Dh)
            score = (q @ kv[0].T / math.sqrt(Dh)).masked_fill(hidden, -math.inf)
            norm = torch.logsumexp(score, 1)
            out[b, :, g * G:(g + 1) * G] = (torch.exp(score - norm[:, None]) @ kv[1]).view(N, G, Dh)
            lse[b, :, g * G:(g + 1) * G] = norm.view(N, G)
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def _exact_logits(s, case):
    if not case["write"]:
        return None
    B, N, V = s["logits"].shape
    parent, token, history = (s[x].cpu().numpy() for x in ("parent", "token", "history"))
    out = s["logits"].double()
    masks = None if s["masks"] is None else np.unpackbits(s["masks"].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :V]
    half = case["history"] // 2
    for b in range(B):
        prompt, reply = set(history[b, :half].tolist()), history[b, half:].tolist()
        factor, presence, frequency = (float(s[x][b]) for x in ("repetition", "presence", "frequency"))
        for i in range(N):
            times = np.bincount(reply + [int(token[b, j]) for j in _walk(parent[b], i)], minlength=V)
            seen = times > 0
            seen[list(prompt)] = True
            seen, times = torch.from_numpy(seen).to(DEV), torch.from_numpy(times).to(DEV)
            x = out[b, i]
            x = torch.where(seen, torch.where(x > 0, x / factor, x * factor), x) - frequency * times - presence * (times > 0)
            if s["bias"] is not None:
                x = x + s["bias"][b].double()
            which = -1 if masks is None else int(s["mask_index"][b, i])
            if which >= 0:
                x = x.masked_fill(torch.from_numpy(masks[which] == 0).to(DEV), -math.inf)
            out[b, i] = x
    return {"logits": out, "best": None, "counts": None}
