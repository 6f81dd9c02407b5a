"""ygg_prompt_attention at the ends of the range of values that the header states, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2512_23858_amd as ygg
import plain_prompt as plain
from gpu_util import DEV, to_f64
from test_gpu_prompt_attention import _attend, _problem

pytestmark = pytest.mark.gpu

# heads, head_dim, queries, keys, (rows of a workgroup, keys in parts); fp32 has one kind
KINDS = [((2, 2), 64, 300, 300, (128, False)), ((64, 8), 128, 600, 1600, (256, False)), ((4, 2), 64, 9, 3000, (128, True)), ((40, 8), 128, 500, 3000, (256, True))]


def _kind(heads, Dh, nq, nk, plan, dtype, seed):
    p = _problem(heads, Dh, [nq], [nk], dtype=dtype, seed=seed)
    if dtype == ygg.BF16:
        got = ygg.prompt_plan(p["shape"])
        assert (got["rows"], got["splits"] > 1) == plan, got
    return p


def _out_tolerance(dtype, ref, size, n, split):
    """Weights that are equal: in bf16 half a step, 2^-8, against a sum in fp32; n / 2 additions of 2^-23 to either sum; a partial row in fp16,
    2^-12 of its largest, twice that for what of it is left in the sum; the result's own half step and a division."""
    f32 = dtype == ygg.F32
    row = np.maximum(size.max(-1, keepdims=True), np.abs(ref).max(-1, keepdims=True))
    return size * ((0 if f32 else 2.0 ** -8) + n * 2.0 ** -23) + (2.0 ** -11 * row if split and not f32 else 0) + np.abs(ref) * (2.0 ** -22 if f32 else 2.0 ** -8 + 2.0 ** -20)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [ygg.BF16, ygg.F32])
@pytest.mark.parametrize("power", [10, 24, 32, 45, 56])
def test_equal_scores_of_any_size_weigh_the_same(kind, dtype, power):
    """All keys are one vector times 1 or 2, and the queries' magnitudes run from 1 to 2^(power): a row's scores are s and 2 s, exactly, from
    ordinary ones to beyond 2^110, of either sign and in one wavefront.  Where s and 2 s lie more than 200 apart a row is the mean of the keys
    of the larger; the others are left out here."""
    heads, Dh, nq, nk, plan = kind
    p = _kind(*kind, dtype, seed=power)
    g = np.random.default_rng(power)
    # (a base of few bits: a score's products and sums are exact, so s and 2 s are, whatever their order)
    base = torch.from_numpy(g.integers(1, 4, (1, heads[1], Dh)) * 2.0 ** power)
    twice = torch.from_numpy(1 + (g.random(nk) < 0.3))[:, None, None]
    twice[:40] = 1        # (the larger ones of a row may come late)
    p["k"] = (base * twice).to(p["k"].dtype).to(DEV)
    size = np.exp2(g.integers(0, power + 1, (nq, heads[0], 1))) * g.choice([-1.0, 1.0], (nq, heads[0], 1))
    p["q"] = torch.from_numpy(size * g.integers(1, 4, (nq, heads[0], Dh))).to(p["q"].dtype).to(DEV)
    out, lse = (to_f64(x) for x in _attend(p))
    q, k, v = to_f64(p["q"]), to_f64(p["k"]), to_f64(p["v"])
    scale, tw = p["shape"].softmax_scale, twice[:, 0, 0].numpy()
    seen_rows = 0
    for h in range(heads[0]):
        kv = h // (heads[0] // heads[1])
        s = q[:, h] @ k[0, kv] * scale                           # (key 0 is the vector itself)
        seen = np.arange(nk)[None] <= np.arange(nq)[:, None] + nk - nq
        has2 = (seen & (tw == 2)).any(1)
        most = np.where((s > 0) & has2, 2, 1)                    # the multiple whose score is the row's largest (multiple 1 is always seen)
        w = (seen & (tw[None] == most[:, None])).astype(np.float64)
        count = w.sum(1)
        ref, mag = w @ v[:, kv] / count[:, None], w @ np.abs(v[:, kv]) / count[:, None]
        good = np.abs(s) > 200
        seen_rows += good.sum()
        err = np.abs(out[:, h] - ref)
        assert (err <= _out_tolerance(dtype, ref, mag, nk, plan[1]))[good].all(), (h, err[good].max())
        want = s * most + np.log(count)
        # the score, its product with the scale and log2(e), and that with ln(2): 2^-24 each of the scores, the scales' own rounding likewise
        assert (np.abs(lse[:, h] - want) <= np.abs(s * most) * 2.0 ** -21 + nk * 2.0 ** -24 + 2.0 ** -20 * (1 + np.log(nk)))[good].all(), h
    assert seen_rows > 0.5 * nq * heads[0]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [ygg.BF16, ygg.F32])
@pytest.mark.parametrize("power", [-60, -100, -119])
def test_small_values_keep_their_bits(kind, dtype, power):
    """Rows whose softmax is one key or a few, values of 2^power: as exact, relative to themselves, as values of 1, with keys in parts too."""
    heads, Dh, nq, nk, plan = kind
    p = _kind(*kind, dtype, seed=5)
    p["q"] = p["q"] * 30
    p["v"] = p["v"] * 2.0 ** power
    out, _ = (to_f64(x) for x in _attend(p))
    q, k, v = to_f64(p["q"]), to_f64(p["k"]), to_f64(p["v"])
    scale = p["shape"].softmax_scale
    seen = np.arange(nk)[None] <= np.arange(nq)[:, None] + nk - nq
    for h in range(0, heads[0], max(heads[0] // 2, 1)):
        kv = h // (heads[0] // heads[1])
        s = np.where(seen, q[:, h] @ k[:, kv].T * scale, -np.inf)
        w = np.exp(s - s.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        ref, mag = w @ v[:, kv], w @ np.abs(v[:, kv])
        # Scores: Dh rounded additions (bf16: sixteen products to an instruction, Dh / 16 + 4) of 2^-23 of the terms' magnitudes, the base-2
        # score once more, the exponential to 2^-22; on either side of the quotient
        terms = scale * np.abs(q[:, h]).sum(-1).max() * np.abs(k[:, kv]).max()
        score = terms * ((Dh if dtype == ygg.F32 else Dh / 16 + 4) * 2.0 ** -23 + 2.0 ** -22) + 2.0 ** -22
        # a product of a weight and a value, or a value of a partial row, below the smallest normal number may count as zero
        lost = np.minimum(w * np.abs(v[:, kv]).max(), 2.0 ** -126).sum(1, keepdims=True) + 2.0 ** -126
        tol = _out_tolerance(dtype, ref, mag, nk, plan[1]) + mag * 2 * score + lost
        err = np.abs(out[:, h] - ref)
        assert (err <= tol).all(), (h, (err / tol).max())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [ygg.BF16, ygg.F32])
def test_values_near_2_to_the_60_under_rising_scores(kind, dtype):
    """Every key's score is a little above the one before, by 29 base-2 units from the first to the last of a block, so that a reference lags
    as far as it may; values all of one sign, up to 2^60."""
    heads, Dh, nq, nk, plan = kind
    p = _kind(*kind, dtype, seed=3)
    t = p["k"].dtype
    g = np.random.default_rng(4)
    # one dimension carries the score: base-2 units (k rises by whole units and falls back every 30 keys, by 8 further units every 300)
    j = np.arange(nk)
    units = j % 30 + 8.0 * (j // 300 % 8)
    k = torch.zeros((nk, heads[1], Dh), dtype=torch.float64)
    k[:, :, 0] = torch.from_numpy(units)[:, None]
    q = torch.zeros((nq, heads[0], Dh), dtype=torch.float64)
    q[:, :, 0] = 1
    p["shape"].softmax_scale = float(np.float32(np.log(2.0)))
    p["q"], p["k"] = q.to(t).to(DEV), k.to(t).to(DEV)
    p["v"] = torch.from_numpy((0.5 + 0.498 * g.random((nk, heads[1], Dh))) * 2.0 ** 60).to(t).to(DEV)
    out, lse = (to_f64(x) for x in _attend(p))
    ref, ref_lse, size = plain.prompt_attention(to_f64(p["q"]), to_f64(p["k"]), to_f64(p["v"]), p["shape"].softmax_scale)
    # scores to 93 units, rounded with their scale to 2^-23 each: 2^-15 of a weight, on either side of the quotient
    tol = _out_tolerance(dtype, ref, size, nk, plan[1]) + size * 2.0 ** -14
    assert (np.abs(out - ref) <= tol).all(), (np.abs(out - ref) / tol).max()
    assert (np.abs(lse - ref_lse) <= 2.0 ** -15 + nk * 2.0 ** -24 + 2.0 ** -20 * (1 + np.abs(ref_lse))).all()
