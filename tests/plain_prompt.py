"""The definitions of the operators of a prompt's way into the 4-bit cache, in numpy and 64 bits (include/ygg.h states them): norms with
rotary positions, attention of prompts, the 4-bit block cache.  TEST INFRASTRUCTURE ONLY; nothing here comes from the library."""
from __future__ import annotations

import numpy as np

import plain_ops as plain

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = np.concatenate((LEVELS, -LEVELS))


def norm_rotary(x, weight, eps, pos, freq, interleaved, scale):
    """x [B,N,H,Dh] float64, weight [Dh] or [H,Dh] -> (normed and rotated, sum of the magnitudes that enter each element)."""
    mean = (x * x).mean(-1, keepdims=True) + eps
    return plain.rotary(x * weight / np.sqrt(np.where(mean > 0, mean, 1.0)), pos, freq, interleaved, scale)


def prompt_attention(q, k, v, scale):
    """One sequence: q [n,H,Dh], k and v [m,Hkv,Dh] float64; the last query sees every key.  -> out, lse, sum of weight * |value|."""
    n, H, Dh = q.shape
    m, Hkv, _ = k.shape
    seen = np.arange(m)[None] <= np.arange(n)[:, None] + m - n
    out, size, lse = np.zeros((n, H, Dh)), np.zeros((n, H, Dh)), np.full((n, H), -np.inf)
    some = seen.any(1)
    for h in range(H):
        g = h // (H // Hkv)
        score = np.where(seen, q[:, h] @ k[:, g].T * scale, -np.inf)[some]
        if not len(score):
            continue
        top = score.max(-1, keepdims=True)
        w = np.exp(score - top)
        total = w.sum(-1, keepdims=True)
        out[some, h], size[some, h] = w / total @ v[:, g], w / total @ np.abs(v[:, g])
        lse[some, h] = (top + np.log(total))[:, 0]
    return out, lse, size


def stored_at(which, Dh):
    """([64, Dh] number of the code, [64, Dh] byte of the scale) of a block at which token t and dimension d are stored."""
    t, d = np.meshgrid(np.arange(64), np.arange(Dh), indexing="ij")
    if which == "k":
        chunk, lane, e = t // 32 * (Dh // 64) + d // 64, 32 * (d // 32 % 2) + t % 32, d % 32
    else:
        chunk, lane, e = d // 32, 32 * (t // 32) + d % 32, 16 * (t // 4 % 2) + 4 * (t % 32 // 8) + t % 4
    return 2048 * chunk + 32 * lane + e, lane * (Dh // 32) + chunk


def decode(codes, scale, which):
    """codes [.., 32*Dh] and scales [.., 2*Dh], bytes -> [.., 64, Dh] float64."""
    code_at, scale_at = stored_at(which, codes.shape[-1] // 32)
    byte = codes[..., code_at // 2]
    return VALUES[np.where(code_at % 2 == 0, byte & 15, byte >> 4)] * np.exp2(scale[..., scale_at].astype(np.float64) - 127)


def encode(x, which):
    """Rows x [.., 64, Dh] of whole blocks -> (codes [.., 32*Dh], scales [.., 2*Dh]), bytes."""
    Dh = x.shape[-1]
    code_at, scale_at = stored_at(which, Dh)
    amax = np.zeros((*x.shape[:-2], 2 * Dh))
    for i in np.ndindex(64, Dh):
        amax[..., scale_at[i]] = np.maximum(amax[..., scale_at[i]], np.abs(x[(..., *i)]))
    e = np.full(amax.shape, -100)
    while (over := amax > 7 * np.exp2(e.astype(np.float64))).any():
        e += over
    y = np.abs(x) / np.exp2(e[..., scale_at].astype(np.float64))
    bounds = (LEVELS[1:] + LEVELS[:-1]) / 2                     # at a bound the even code wins
    code = sum((y >= b) if i % 2 else (y > b) for i, b in enumerate(bounds)) | np.where(np.signbit(x), 8, 0)
    nibbles = np.empty((*x.shape[:-2], 64 * Dh), np.uint8)
    nibbles[..., code_at] = code
    return nibbles[..., ::2] | nibbles[..., 1::2] << 4, (e + 127).astype(np.uint8)
