"""ygg_tree_norm_rotary against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2512_23858_amd as ygg
import plain_ops
import plain_prompt as plain
import ygg_workloads as wl
from gpu_util import DEV, to_dev, to_f64

pytestmark = pytest.mark.gpu


def _shape(B, N, Hq, Hkv, Dh, dtype, cap=1 << 22):
    return ygg.Shape(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=Dh, depth=0, width=1, n_nodes=N, vocab=1, kv_dtype=dtype,
                     softmax_scale=1.0, kv_capacity=cap, max_seq_len=cap - 1)


def _check(got, x, weight, eps, pos, freq, interleaved, scale, bf16):
    ref, size = plain.norm_rotary(x, weight, eps, pos, freq, interleaved, scale)
    # The mean of the squares: sixteen additions of a lane, three between lanes, the division and eps, 2^-24 each, halved by the root; the
    # root, its reciprocal and the two products 2^-24 each: 15 * 2^-24, below 2^-20.  Sine and cosine are off by at most 2^-21, the rotation's
    # products and sum by 2^-24 each of what enters; a bf16 result by half a step, 2^-8.
    tol = size * (2.0 ** -20 + 2.0 ** -21 + 3 * 2.0 ** -24) + (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(ref) + 1e-37
    assert (np.abs(got - ref) <= tol).all(), np.abs(got - ref).max()


CASES = [  # B, N, Hq, Hkv, Dh, rotary_dim, interleaved, dtype, scale, farthest length, per head
    (1, 1, 4, 4, 64, 64, False, ygg.F32, 1.0, 5, False), (1, 1, 32, 8, 128, 128, True, ygg.BF16, 1.0, 4_000_000, False),
    (3, 13, 5, 1, 64, 16, False, ygg.BF16, 1.0, 100, True), (2, 49, 8, 2, 128, 64, True, ygg.F32, 0.75, 4_000_000, True),
    (2, 321, 32, 8, 128, 128, False, ygg.BF16, 1.25, 131072, False), (1, 1024, 2, 1, 64, 48, False, ygg.BF16, 1.0, 0, True),
    (70, 7, 12, 12, 64, 32, True, ygg.FP8_BLOCK, 1.0, 999, False), (16, 49, 64, 8, 128, 112, True, ygg.FP4_BLOCK, 1.0, 8192, True),
    (1, 3, 1, 1, 128, 128, False, ygg.F32, 1.0, 64, False),
]


def _inputs(g, B, N, h, Dh, dt):
    """Tokens of very different magnitudes."""
    return torch.from_numpy(g.standard_normal((B, N, h, Dh)) * np.exp2(g.integers(-12, 12, (B, N, 1, 1)))).to(dt).to(DEV)


@pytest.mark.parametrize("B,N,Hq,Hkv,Dh,rd,inter,dtype,scale,far,per_head", CASES)
def test_tree_positions(B, N, Hq, Hkv, Dh, rd, inter, dtype, scale, far, per_head):
    g = np.random.default_rng(N * 7 + Hq)
    parent = np.stack([wl.random_topological_tree(B * N, N, sub=b) for b in range(B)])
    lens = g.integers(0, far + 1, B).astype(np.int32)
    lens[0] = far
    f32 = dtype == ygg.F32
    q, k = (_inputs(g, B, N, h, Dh, torch.float32 if f32 else torch.bfloat16) for h in (Hq, Hkv))
    qw, kw = (torch.from_numpy(1 + 0.5 * g.standard_normal((h, Dh) if per_head else (Dh,))).float().to(DEV) for h in (Hq, Hkv))
    freq = ygg.rotary_frequencies(rd, 10000.0)
    q0, k0 = q.clone(), k.clone()
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    shape = _shape(B, N, Hq, Hkv, Dh, dtype)
    kw_ = dict(seq_lens=to_dev(lens), parent_idx=to_dev(parent), interleaved=inter, scale=scale, eps=1e-5)
    ygg.tree_norm_rotary(shape, q, k, qo, ko, qw, kw, freq.to(DEV), **kw_)
    pos = plain_ops.positions(parent, lens)
    for got, x, w in ((qo, q, qw), (ko, k, kw)):
        _check(to_f64(got), to_f64(x), to_f64(w), 1e-5, pos, freq.numpy(), inter, scale, not f32)
    assert torch.equal(q, q0) and torch.equal(k, k0)
    # in place, and one tensor alone: the same bits
    ygg.tree_norm_rotary(shape, q, None, q, None, qw, None, freq.to(DEV), **kw_)
    ygg.tree_norm_rotary(shape, None, k, None, k, None, kw, freq.to(DEV), **kw_)
    assert torch.equal(q, qo) and torch.equal(k, ko)


@pytest.mark.parametrize("T", [1, 5, 2049])
@pytest.mark.parametrize("inter", [False, True])
def test_explicit_positions_of_a_fused_projection(T, inter):
    B, Hq, Hkv, Dh, rd = 2, 8, 2, 128, 96
    g = np.random.default_rng(T)
    qkv = _inputs(g, B, T, Hq + 2 * Hkv, Dh, torch.bfloat16)
    before = qkv.clone()
    pos = g.integers(-1000, 1_000_000, (B, T)).astype(np.int32)
    freq = ygg.rotary_frequencies(rd, 500000.0, factor=8.0, original_len=8192)
    w = torch.from_numpy(g.standard_normal(Dh)).float().to(DEV)
    q, k = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]
    qo, ko = torch.empty((B, T, Hq, Dh), dtype=torch.bfloat16, device=DEV), torch.empty((B, T, Hkv, Dh), dtype=torch.bfloat16, device=DEV)
    ygg.tree_norm_rotary(_shape(B, T, Hq, Hkv, Dh, ygg.BF16), q, k, qo, ko, w, w, freq.to(DEV), positions=to_dev(pos), interleaved=inter)
    _check(to_f64(qo), to_f64(q), to_f64(w), 1e-6, pos, freq.numpy(), inter, 1.0, True)
    _check(to_f64(ko), to_f64(k), to_f64(w), 1e-6, pos, freq.numpy(), inter, 1.0, True)
    assert torch.equal(qkv, before)


@pytest.mark.parametrize("dtype", [ygg.F32, ygg.BF16])
def test_heads_of_zeros_and_of_any_magnitude(dtype):
    """A head of zeros stays zero, with and without eps; others' magnitudes come out, down to where eps outweighs them."""
    dt = torch.float32 if dtype == ygg.F32 else torch.bfloat16
    q = torch.randn((1, 6, 3, 64), device=DEV).to(dt)
    q[0, 0] = 0
    for i, power in enumerate((-40, -10, 10, 40)):
        q[0, 1 + i] *= 2.0 ** power
    w = torch.ones(64, device=DEV)
    freq, pos = ygg.rotary_frequencies(32), np.arange(6)[None]
    for eps in (0.0, 1e-6):
        out = torch.full_like(q, float("nan"))
        ygg.tree_norm_rotary(_shape(1, 6, 3, 3, 64, dtype), q, None, out, None, w, None, freq.to(DEV), positions=to_dev(pos.astype(np.int32)), eps=eps)
        _check(to_f64(out), to_f64(q), to_f64(w), eps, pos, freq.numpy(), False, 1.0, dtype == ygg.BF16)
        assert (out[0, 0] == 0).all()


def test_a_head_whose_squares_are_subnormal_counts_as_zeros():
    q = torch.ones((1, 4, 2, 128), device=DEV)
    q[0, 0], q[0, 1], q[0, 2] = 2.0 ** -62, 2.0 ** -64, 1e-45
    out = torch.full_like(q, float("nan"))
    w = torch.ones(128, device=DEV)
    pos = torch.zeros((1, 4), dtype=torch.int32, device=DEV)
    ygg.tree_norm_rotary(_shape(1, 4, 2, 2, 128, ygg.F32), q, None, out, None, w, None, ygg.rotary_frequencies(64).to(DEV), positions=pos, eps=0.0)
    assert (out[0, [0, 3]] == 1).all() and (out[0, [1, 2]] == 0).all()


@pytest.mark.parametrize("dtype", [ygg.F32, ygg.BF16])
@pytest.mark.parametrize("inter", [False, True])
def test_a_head_with_a_nan_is_nan_and_its_neighbours_are_not(dtype, inter):
    """x / sqrt(mean(x^2)) of a head with a NaN is NaN throughout.  Everything else comes out as without it, bit for bit."""
    dt = torch.float32 if dtype == ygg.F32 else torch.bfloat16
    for Dh, rd in ((64, 32), (128, 128)):
        shape = _shape(1, 9, 3, 3, Dh, dtype)
        x = torch.randn((1, 9, 3, Dh), device=DEV).to(dt)
        f, w = ygg.rotary_frequencies(rd).to(DEV), torch.rand(Dh, device=DEV) + 0.5
        pos = torch.arange(9, dtype=torch.int32, device=DEV)[None]
        run = lambda x, out: ygg.tree_norm_rotary(shape, x, None, out, None, w, None, f, positions=pos, interleaved=inter)
        clean = torch.empty_like(x)
        run(x, clean)
        for at in (0, rd - 1, Dh - 1):
            y, out = x.clone(), torch.empty_like(x)
            y[0, 4, 1, at] = float("nan")
            run(y, out)
            assert out[0, 4, 1].isnan().all()
            out[0, 4, 1] = clean[0, 4, 1]
            assert torch.equal(out, clean)


def test_the_norm_of_ones_is_the_rotation_alone():
    shape = _shape(2, 9, 4, 2, 128, ygg.F32)
    q = torch.sign(torch.randn((2, 9, 4, 128), device=DEV))        # every head's mean square is 1
    f, pos, w = ygg.rotary_frequencies(128).to(DEV), torch.arange(18, dtype=torch.int32, device=DEV).view(2, 9), torch.ones(128, device=DEV)
    a, b = torch.empty_like(q), torch.empty_like(q)
    ygg.tree_norm_rotary(shape, q, None, a, None, w, None, f, positions=pos, eps=0.0)
    ygg.tree_rotary(shape, q, None, b, None, f, positions=pos)
    assert torch.equal(a, b)


def test_refusals_on_the_gpu_binding():
    shape = _shape(1, 4, 2, 1, 64, ygg.BF16)
    q, k = (torch.zeros((1, 4, h, 64), dtype=torch.bfloat16, device=DEV) for h in (2, 1))
    f, pos, w = ygg.rotary_frequencies(64).to(DEV), torch.zeros((1, 4), dtype=torch.int32, device=DEV), torch.ones(64, device=DEV)
    good = dict(q=q, k=k, q_out=q.clone(), k_out=k.clone(), q_weight=w, k_weight=w, frequencies=f, positions=pos)
    ygg.tree_norm_rotary(shape, **good)
    own = dict(q_weight=torch.ones((2, 64), device=DEV), k_weight=torch.ones((1, 64), device=DEV))
    ygg.tree_norm_rotary(shape, **{**good, **own})
    for kw, error, match in ((dict(q_weight=w.double()), TypeError, "q_weight"), (dict(k_weight=w[:32]), ValueError, "k_weight"),
                             (dict(q_weight=own["q_weight"]), ValueError, "k_weight"), (dict(k_weight=torch.ones((2, 64), device=DEV)), ValueError, "q_weight"),
                             ({**own, "k_weight": torch.ones((2, 64), device=DEV)}, ValueError, "k_weight"), (dict(q_weight=w.cpu()), ValueError, "GPU"),
                             (dict(q_weight=None), RuntimeError, "null"), (dict(eps=-1.0), RuntimeError, "inconsistent"), (dict(q=q.cpu()), ValueError, "GPU"),
                             (dict(frequencies=f.float()), TypeError, "frequencies"), (dict(q=q[:, :3]), ValueError, "q"),
                             (dict(k_out=k[:, :3].contiguous()), ValueError, "k_out"), (dict(positions=pos[:, :2].contiguous()), ValueError, "positions"),
                             (dict(q=q[:, :1].expand(1, 4, 2, 64)), ValueError, "rows must be dense"), (dict(positions=None), RuntimeError, "null")):
        with pytest.raises(error, match=match):
            ygg.tree_norm_rotary(shape, **{**good, **kw})
