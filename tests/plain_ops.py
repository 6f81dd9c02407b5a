"""The definitions of the operators around the verification calls, in numpy and 64 bits (include/ygg.h states them): rotary positions,
the 8-bit block cache, tree attention over it, constrained logits.  TEST INFRASTRUCTURE ONLY; nothing here comes from the library."""
from __future__ import annotations

import numpy as np

BLOCK = 64


def path_of(parent, i):
    """Node i and its ancestors, root last."""
    out = []
    while i >= 0:
        out.append(i)
        i = int(parent[i])
    return out


def positions(parent_idx, seq_lens):
    return np.array([[seq_lens[b] + len(path_of(parent_idx[b], i)) - 1 for i in range(parent_idx.shape[1])] for b in range(len(seq_lens))])


def rotary(x, pos, freq, interleaved, scale):
    """x [B,N,H,Dh] float64 -> (rotated, sum of the magnitudes that enter each element)."""
    r = 2 * len(freq)
    a = pos[..., None, None] * freq
    c, s = np.cos(a) * scale, np.sin(a) * scale
    i, j = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    out, size = x.copy(), np.abs(x)
    out[..., i], out[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    size[..., i] = size[..., j] = (np.abs(x[..., i]) + np.abs(x[..., j])) * abs(scale)
    return out, size


def stored_at(which, Dh):
    """Byte of a block at which token t and dimension d are stored, [64, Dh] (the formula of include/ygg.h)."""
    t, d = np.meshgrid(np.arange(BLOCK), np.arange(Dh), indexing="ij")
    if which == "k":
        chunk, lane, e = 2 * ((t // 32) * (Dh // 64) + d // 64) + d // 16 % 2, 32 * (d // 32 % 2) + t % 32, d % 16
    else:
        chunk, lane, e = 2 * (d // 32) + t // 32, 32 * (t // 4 % 2) + d % 32, 4 * (t % 32 // 8) + t % 4
    return 1024 * chunk + 16 * lane + e


def e4m3_values():
    """Values of the 256 codes (1 sign, 4 exponent bits of bias 7, 3 of significand; 0x7f and 0xff are NaN)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[(c & 127) == 127] = np.nan
    return np.where(c & 128, -v, v)


def decode(codes, scale, which):
    """codes [.., 64*Dh] uint8, scale [..] -> [.., 64, Dh] float64."""
    Dh = codes.shape[-1] // BLOCK
    return e4m3_values()[codes[..., stored_at(which, Dh)]] * scale[..., None, None].astype(np.float64)


def block_scale(x):
    """fp32 scale of rows x [.., 64, Dh]."""
    amax = np.abs(x).max(axis=(-2, -1)).astype(np.float32)
    return np.where(amax > 0, np.maximum(amax / np.float32(448), np.float32(2.0 ** -100)), np.float32(1)).astype(np.float32)


def tree_attention(q, keys, values, prefix, parent, scale):
    """One sequence and kv head: q [N,G,Dh]; keys, values [prefix + N, Dh].  -> out, lse, sum of weight * |value|."""
    N = q.shape[0]
    seen = np.zeros((N, prefix + N), bool)
    seen[:, :prefix] = True
    for i in range(N):
        seen[i, prefix + np.array(path_of(parent, i))] = True
    score = np.where(seen[:, None], np.einsum("ngd,kd->ngk", q, keys) * scale, -np.inf)
    top = score.max(-1, keepdims=True)
    w = np.exp(score - top)
    total = w.sum(-1, keepdims=True)
    w /= total
    return np.einsum("ngk,kd->ngd", w, values), (top + np.log(total))[..., 0], np.einsum("ngk,kd->ngd", w, np.abs(values))


def constrain(logits, parent, token, counts, repetition, presence, frequency, bias, masks, mask_index):
    """One sequence, logits [N,V] float32, in fp32 and in the order of the definition; scalars per sequence."""
    out = logits.astype(np.float32).copy()
    V = out.shape[1]
    confirmed = (counts.astype(np.int64) & 0x7fffffff) if counts is not None else np.zeros(V, np.int64)
    known = counts != 0 if counts is not None else np.zeros(V, bool)
    f32 = np.float32
    with np.errstate(invalid="ignore", over="ignore"):
        for i in range(out.shape[0]):
            on_path = [int(token[j]) for j in path_of(parent, i)]
            c = confirmed + np.bincount([t for t in on_path if 0 <= t < V], minlength=V)
            seen = known | (c > 0)
            x = out[i]
            x = np.where(seen, np.where(x > 0, x / f32(repetition), x * f32(repetition)), x).astype(f32)
            x = x - f32(frequency) * c.astype(f32)
            x = x - np.where(c > 0, f32(presence), f32(0))
            if bias is not None:
                x = x + bias
            if masks is not None and mask_index[i] >= 0:
                words = masks[min(mask_index[i], len(masks) - 1)].view(np.uint32)
                v = np.arange(V)
                x = np.where((words[v // 32] >> (v % 32).astype(np.uint32)) & 1, x, f32(-np.inf))
            out[i] = x
    return out


def encode(x, scale, which):
    """Bytes of a block in storage order, [.., 64*Dh] uint8, of rows x [.., 64, Dh] at fp32 scales [..]: the E4M3 value nearest to
    x * (1 / scale) in fp32, ties to even."""
    y = x.astype(np.float32) * (np.float32(1) / scale.astype(np.float32))[..., None, None]
    size = np.abs(y).astype(np.float64)
    step = np.exp2(np.maximum(np.frexp(size)[1] - 1, -6) - 3.0)
    code = np.searchsorted(e4m3_values()[:127], np.minimum(np.rint(size / step) * step, 448.0))      # (rint: ties to even)
    code = (code | np.where(np.signbit(y), 128, 0)).astype(np.uint8)
    out = np.empty((*x.shape[:-2], 64 * x.shape[-1]), np.uint8)
    out[..., stored_at(which, x.shape[-1])] = code
    return out
