"""ygg_tree_rotary against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2512_23858_amd as ygg
import plain_ops as plain
import ygg_workloads as wl
from gpu_util import DEV, to_dev, to_f64

pytestmark = pytest.mark.gpu


def _shape(B, N, Hq, Hkv, Dh, dtype, cap=1 << 22):
    return ygg.Shape(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=Dh, depth=0, width=1, n_nodes=N, vocab=1, kv_dtype=dtype,
                     softmax_scale=1.0, kv_capacity=cap, max_seq_len=cap - 1)


def _check(got, x, pos, freq, interleaved, scale, bf16):
    ref, size = plain.rotary(x, pos, freq, interleaved, scale)
    # sine and cosine are off by at most 2^-21 (the fp32 fraction of a turn 2^-25 * 2 pi, their own rounding, that of `scale`), the two
    # products and the sum by 2^-24 each of what enters; a bf16 result by half a step, 2^-8
    tol = size * (2.0 ** -21 + 3 * 2.0 ** -24) + (2.0 ** -8 if bf16 else 2.0 ** -24) * np.abs(ref) + 1e-30
    assert (np.abs(got - ref) <= tol).all(), np.abs(got - ref).max()


CASES = [  # B, N, Hq, Hkv, Dh, rotary_dim, interleaved, dtype, scale, farthest length
    (1, 1, 4, 4, 64, 64, False, ygg.F32, 1.0, 5), (1, 1, 32, 8, 128, 128, True, ygg.BF16, 1.0, 4_000_000),
    (3, 13, 5, 1, 64, 16, False, ygg.BF16, 1.0, 100), (2, 49, 8, 2, 128, 64, True, ygg.F32, 0.75, 4_000_000),
    (2, 321, 32, 8, 128, 128, False, ygg.BF16, 1.25, 131072), (1, 1024, 2, 1, 64, 48, False, ygg.BF16, 1.0, 0),
    (70, 7, 12, 12, 64, 32, True, ygg.BF16, 1.0, 999), (16, 49, 64, 8, 128, 112, True, ygg.FP8_BLOCK, 1.0, 8192),
]


@pytest.mark.parametrize("B,N,Hq,Hkv,Dh,rd,inter,dtype,scale,far", CASES)
def test_tree_positions(B, N, Hq, Hkv, Dh, rd, inter, dtype, scale, far):
    g = np.random.default_rng(N * 7 + Hq)
    parent = np.stack([wl.random_topological_tree(B * N, N, sub=b) for b in range(B)])
    lens = g.integers(0, far + 1, B).astype(np.int32)
    lens[0] = far
    f32 = dtype == ygg.F32
    dt = torch.float32 if f32 else torch.bfloat16
    q, k = (torch.from_numpy(g.standard_normal((B, N, h, Dh))).to(dt).to(DEV) for h in (Hq, Hkv))
    freq = ygg.rotary_frequencies(rd, 10000.0)
    q0, k0 = q.clone(), k.clone()
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    shape = _shape(B, N, Hq, Hkv, Dh, dtype)
    ygg.tree_rotary(shape, q, k, qo, ko, freq.to(DEV), seq_lens=to_dev(lens), parent_idx=to_dev(parent), interleaved=inter, scale=scale)
    pos = plain.positions(parent, lens)
    for got, x in ((qo, q), (ko, k)):
        _check(to_f64(got), to_f64(x), pos, freq.numpy(), inter, scale, not f32)
    assert torch.equal(q, q0) and torch.equal(k, k0)
    # in place, and one tensor alone: the same bits
    ygg.tree_rotary(shape, q, None, q, None, freq.to(DEV), seq_lens=to_dev(lens), parent_idx=to_dev(parent), interleaved=inter, scale=scale)
    ygg.tree_rotary(shape, None, k, None, k, freq.to(DEV), seq_lens=to_dev(lens), parent_idx=to_dev(parent), interleaved=inter, scale=scale)
    assert torch.equal(q, qo) and torch.equal(k, ko)


@pytest.mark.parametrize("T", [1, 5, 2049])
@pytest.mark.parametrize("inter", [False, True])
def test_explicit_positions_of_a_fused_projection(T, inter):
    B, Hq, Hkv, Dh, rd = 2, 8, 2, 128, 96
    g = np.random.default_rng(T)
    qkv = torch.from_numpy(g.standard_normal((B, T, Hq + 2 * Hkv, Dh))).to(torch.bfloat16).to(DEV)
    before = qkv.clone()
    pos = g.integers(-1000, 1_000_000, (B, T)).astype(np.int32)
    freq = ygg.rotary_frequencies(rd, 500000.0, factor=8.0, original_len=8192)
    q, k = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv]
    qo, ko = torch.empty((B, T, Hq, Dh), dtype=torch.bfloat16, device=DEV), torch.empty((B, T, Hkv, Dh), dtype=torch.bfloat16, device=DEV)
    ygg.tree_rotary(_shape(B, T, Hq, Hkv, Dh, ygg.BF16), q, k, qo, ko, freq.to(DEV), positions=to_dev(pos), interleaved=inter)
    _check(to_f64(qo), to_f64(q), pos, freq.numpy(), inter, 1.0, True)
    _check(to_f64(ko), to_f64(k), pos, freq.numpy(), inter, 1.0, True)
    assert torch.equal(qkv, before)


def test_a_length_beyond_the_bound_counts_as_the_bound_and_a_bad_parent_ends_the_walk():
    parent = np.array([[-1, 0, 7, 2]], np.int32)      # node 2's parent is no earlier node: depth 0, node 3 below it depth 1
    freq = ygg.rotary_frequencies(64)
    q = torch.randn((1, 4, 1, 64), device=DEV)
    out = torch.empty_like(q)
    ygg.tree_rotary(_shape(1, 4, 1, 1, 64, ygg.F32, cap=101), q, None, out, None, freq.to(DEV), seq_lens=to_dev(np.array([500], np.int32)),
                    parent_idx=to_dev(parent))
    _check(to_f64(out), to_f64(q), np.array([[100, 101, 100, 101]]), freq.numpy(), False, 1.0, False)


def test_refusals_on_the_gpu_binding():
    shape = _shape(1, 4, 2, 2, 64, ygg.BF16)
    q = torch.zeros((1, 4, 2, 64), dtype=torch.bfloat16, device=DEV)
    f = ygg.rotary_frequencies(64).to(DEV)
    pos = torch.zeros((1, 4), dtype=torch.int32, device=DEV)
    with pytest.raises(TypeError, match="frequencies"):
        ygg.tree_rotary(shape, q, None, q, None, f.float(), positions=pos)
    with pytest.raises(ValueError, match="GPU"):
        ygg.tree_rotary(shape, q.cpu(), None, q, None, f, positions=pos)
    with pytest.raises(ValueError, match="rows"):
        ygg.tree_rotary(shape, torch.zeros((1, 4, 64, 2), dtype=torch.bfloat16, device=DEV).transpose(2, 3), None, q, None, f, positions=pos)
    with pytest.raises(RuntimeError, match="null"):
        ygg.tree_rotary(shape, q, None, q, None, f)
    wide = torch.zeros((1, 4, 3, 64), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(RuntimeError, match="inconsistent"):      # in place needs dense tokens
        ygg.tree_rotary(shape, wide[:, :, :2], None, wide, None, f, positions=pos)
    for kw in (dict(q=q[:, :3]), dict(q_out=q[:, :3].contiguous()), dict(positions=pos[:, :2].contiguous())):
        with pytest.raises(ValueError, match=next(iter(kw))):
            ygg.tree_rotary(shape, **{**dict(q=q, k=None, q_out=q.clone(), k_out=None, frequencies=f, positions=pos), **kw})


@pytest.mark.parametrize("B,N", [(1, 5), (4, 1), (4, 5)])
def test_expanded_rows_are_refused(B, N):
    """One token's memory under several tokens: a stride of 0 is no dense tensor."""
    shape = _shape(B, N, 2, 2, 64, ygg.BF16)
    one = torch.ones((1, 1, 2, 64), dtype=torch.bfloat16, device=DEV).expand(B, N, 2, 64)
    full, f, pos = one.contiguous(), ygg.rotary_frequencies(64).to(DEV), torch.zeros((B, N), dtype=torch.int32, device=DEV)
    out = torch.zeros_like(full)
    for q, k in ((one, full), (full, one)):
        with pytest.raises(ValueError, match="rows must be dense"):
            ygg.tree_rotary(shape, q, k, out, out.clone(), f, positions=pos)
    assert (out == 0).all()
    ygg.tree_rotary(shape, full, full, out, out.clone(), f, positions=pos)
    assert torch.equal(out, full)                                  # position 0
