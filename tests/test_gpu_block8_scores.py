"""ygg_tree_attention_block8 where scores are far from zero: keys with a component in common, as models with large key biases have."""
import numpy as np
import pytest
import torch

import plain_ops as plain
from gpu_util import DEV, to_f64
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


@pytest.mark.parametrize("Dh", [64, 128])
@pytest.mark.parametrize("score", [-2.0 ** 21, -2.0 ** 22, 2.0 ** 22])
@pytest.mark.parametrize("Hq,Hkv,N,lens", [(4, 1, 65, [0]), (2, 2, 65, [130]), (4, 4, 33, [1000, 5]), (8, 1, 200, [64, 0, 300]), (2, 1, 40, [4000])])
def test_equal_scores_of_any_magnitude(Dh, score, Hq, Hkv, N, lens):
    """All scores are the same power of two, exactly: every row is the mean of the values that it sees.  A node's own keys begin with tiles
    that it sees and end with tiles that it does not, and another wavefront or run has those alone."""
    p = _problem(len(lens), Hq, Hkv, Dh, N, lens, seed=N)
    p["q"].zero_()
    p["q"][..., 0] = score / 1024
    c = p["cache"]
    codes = np.zeros((64, Dh), np.uint8)
    codes[:, 0] = 0x58                                                      # 16, times a scale of 64
    stored = np.empty(64 * Dh, np.uint8)
    stored[plain.stored_at("k", Dh)] = codes
    row = torch.zeros(Dh, dtype=torch.bfloat16, device=DEV)
    row[0] = 1024
    for b, L in enumerate(lens):
        full = L // 64
        c.k_codes[b, :, :full] = torch.from_numpy(stored).to(DEV)
        c.k_scale[b, :, :full] = 64.0
        c.v_scale[b, :, :full] = 2.0 ** -8                                  # (another significand would join a block's scores, rounded)
        c.k_tail[b, full % 2 * 64:full % 2 * 64 + L % 64] = row
        p["dense"]["k_tree"][b] = row
    p["shape"].softmax_scale = 1.0
    _read_back(p)
    out, lse = (to_f64(x) for x in _attend(p))
    G = Hq // Hkv
    for b, L in enumerate(lens):
        for h in range(Hkv):
            ref, ref_lse, size = plain.tree_attention(np.zeros((N, G, Dh)), p["dense"]["k"][b][h], p["dense"]["v"][b][h], L, p["parent"][b], 1.0)
            hs = slice(h * G, (h + 1) * G)
            # in base 2 a score is this power of two times log2 e in fp32, so exact, and equal over blocks and own keys.  Weights are off by
            # 2^-8, their products with V are cut by 2^-8 of the sum of magnitudes, partial rows 2^-12 of the largest, the result 2^-8
            tol = size * (2.0 ** -7 + 2.0 ** -12) + size.max(-1, keepdims=True) * 2.0 ** -12 + np.abs(ref) * 2.0 ** -8
            assert (np.abs(out[b, :, hs] - ref) <= tol).all(), (b, h)
            # m * ln 2 in fp32, from log2 e in fp32: 2^-24 of the score each, a few of them
            assert (np.abs(lse[b, :, hs] - (score + ref_lse)) <= abs(score) * 2.0 ** -22).all(), (b, h)


@pytest.mark.parametrize("Dh", [64, 128])
@pytest.mark.parametrize("q_power,v_power", [(57, 56), (-57, 56), (57, -57)])
def test_magnitudes_at_the_ends_of_the_stated_range(Dh, q_power, v_power):
    """q near 2^60 with keys near 2^-57 and the other way round, values near 2^60 and 2^-57: the scores stay ordinary."""
    p = _problem(2, 8, 2, Dh, 37, [700, 90], seed=Dh)
    c, d = p["cache"], p["dense"]
    for t, power in ((p["q"], q_power), (c.k_scale, -q_power), (c.k_tail, -q_power), (d["k_tree"], -q_power), (c.v_scale, v_power),
                     (c.v_tail, v_power), (d["v_tree"], v_power)):
        t.copy_((t.double() * 2.0 ** power).to(t.dtype))
    _read_back(p)
    _check(p, *_attend(p))
