"""ygg_tree_attention_block8 where scores are far from zero: keys with a component in common, as models with large key biases have."""
import numpy as np
import pytest
import torch

import plain_ops as plain
from gpu_util import DEV
from test_gpu_block8 import _attend, _bf16, _check, _problem

pytestmark = pytest.mark.gpu


def _read_back(p):
    """The keys and values that the cache and the tree's rows stand for now, as _problem forms them."""
    Hkv, Dh = p["shape"].n_kv_heads, p["shape"].head_dim
    for x in "kv":
        codes, scale, tail = (getattr(p["cache"], f"{x}_{y}").cpu() for y in ("codes", "scale", "tail"))
        tree = p["dense"][x + "_tree"].cpu()
        p["dense"][x] = []
        for b, L in enumerate(p["lens"]):
            full, at = int(L) // 64, int(L) // 64 % 2 * 64
            blocks = plain.decode(codes[b, :, :full].numpy(), scale[b, :, :full].numpy(), x).reshape(Hkv, full * 64, Dh)
            rows = torch.cat((tail[b, at:at + int(L) - full * 64], tree[b])).double().numpy().transpose(1, 0, 2)
            p["dense"][x].append(np.concatenate((blocks, rows), 1))


def _common_component(B, Hq, Hkv, Dh, N, lens, seed):
    """Every key is about 2 in magnitude with the same signs, every row of q the opposite of them: row r's largest score lies near
    -(60 .. 700), evenly over the rows, in base 2."""
    p = _problem(B, Hq, Hkv, Dh, N, lens, seed)
    g = np.random.default_rng(seed)
    sign = np.where(g.random(Dh) < 0.5, -1.0, 1.0)
    codes = g.integers(0x3C, 0x44, (*p["cache"].k_codes.shape[:3], 64, Dh)).astype(np.uint8)      # 1.5, 1.625 .. 2.75
    codes |= np.where(sign < 0, 0x80, 0).astype(np.uint8)
    stored = np.empty((*codes.shape[:3], 64 * Dh), np.uint8)
    stored[..., plain.stored_at("k", Dh)] = codes
    for b, L in enumerate(lens):
        full, c = int(L) // 64, p["cache"]
        c.k_codes[b, :, :full] = torch.from_numpy(stored[b, :, :full]).to(DEV)
        c.k_scale[b, :, :full] = 1.0
        rows = lambda *s: _bf16(sign * (2 + 0.25 * g.standard_normal(s))).to(DEV)
        at, open_rows = full % 2 * 64, int(L) - full * 64
        c.k_tail[b, at:at + open_rows] = rows(open_rows, Hkv, Dh)
        p["dense"]["k_tree"][b] = rows(N, Hkv, Dh)
    level = np.linspace(60, 700, B * N * Hq).reshape(B, N, Hq, 1) * np.log(2) / (2 * Dh)
    p["q"].copy_(_bf16(-level * sign * (1 + 0.05 * g.standard_normal((B, N, Hq, Dh)))))
    p["shape"].softmax_scale = 1.0
    _read_back(p)
    return p


@pytest.mark.parametrize("B,Hq,Hkv,Dh,N,lens", [
    (1, 8, 2, 128, 161, [700]), (1, 8, 4, 64, 321, [1000]), (4, 16, 4, 128, 17, [640, 64, 0, 201]), (16, 32, 8, 64, 1, [64 + 70 * b for b in range(16)]),
    (3, 8, 2, 128, 33, [64, 128, 65]), (8, 32, 8, 128, 3, [4096] + [64 * b for b in range(1, 8)]),
])
def test_scores_far_below_zero(B, Hq, Hkv, Dh, N, lens):
    """The reference of a run's first block is any whole number, whatever exponent it leaves for the weights of no block before it."""
    p = _common_component(B, Hq, Hkv, Dh, N, lens, seed=N)
    out, lse = _attend(p)
    assert not torch.isnan(out).any() and not torch.isnan(lse).any()
    _check(p, out, lse)
