"""ygg_block8_append and ygg_tree_attention_block8 against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2512_23858_amd as ygg
import plain_ops as plain
import ygg_workloads as wl
from gpu_util import DEV, to_dev, to_f64, workspace

pytestmark = pytest.mark.gpu
NAN_CODE, NAN_ROW = 0x7F, float("nan")


def _shape(B, Hq, Hkv, Dh, N, cap, D=0, most=None, scale=None):
    return ygg.Shape(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=Dh, depth=D, width=1, n_nodes=N, vocab=1, kv_dtype=ygg.FP8_BLOCK,
                     softmax_scale=scale or Dh ** -0.5, kv_capacity=cap, max_seq_len=cap - D - 1 if most is None else most)


def _bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16)


# ---------------------------------------------------------------- append

def _poisoned(shape, layers):
    c = ygg.new_block_cache(shape, layers, device=DEV)
    for t, v in zip(c.tensors(), (NAN_CODE, NAN_CODE, NAN_ROW, NAN_ROW, NAN_ROW, NAN_ROW)):
        t.fill_(v)
    return c


def _check_cache(cache, rows, written, ends, Dh):
    """rows: {(layer, b): {"k"/"v": [end, Hkv, Dh] float64}}: every token ever appended; written: {(l, b): encoded blocks};
    ends: tokens whose tail rows must hold their values."""
    for x in "kv":
        codes, scale, tail = (getattr(cache, f"{x}_{y}").cpu() for y in ("codes", "scale", "tail"))
        codes, scale, tail = codes.numpy(), scale.numpy(), tail.double().numpy()
        L, B, Hkv, nblk = scale.shape
        for l in range(L):
            for b in range(B):
                r = rows[l, b][x]
                for k in range(nblk):
                    if k not in written[l, b]:
                        assert np.isnan(scale[l, b, :, k]).all() and (codes[l, b, :, k] == NAN_CODE).all(), (x, l, b, k)
                        continue
                    block = r[64 * k:64 * k + 64].transpose(1, 0, 2)                      # [Hkv, 64, Dh]
                    want = plain.block_scale(block)
                    assert np.array_equal(scale[l, b, :, k], want), (x, l, b, k)
                    value = plain.decode(codes[l, b, :, k], want, x)
                    # the nearest value: half a step of its binade (E4M3: 3 bits of significand, steps of 2^-9 below 2^-6), and 2^-22
                    # of the quotient, which is formed in fp32
                    q = np.abs(block) / want[:, None, None].astype(np.float64)
                    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(q, 1e-30))), -6) - 3)
                    assert (np.abs(value - block) <= want[:, None, None] * (step / 2 + q * 2.0 ** -22)).all(), (x, l, b, k)
                for t in ends[l, b]:
                    assert np.array_equal(tail[l, b, t % 128], r[t]), (x, l, b, t)


@pytest.mark.parametrize("Dh", [64, 128])
@pytest.mark.parametrize("steps", [[1], [63, 1], [64], [65, 62, 1, 128], [1, 200, 0, 7, 56, 64], [300, 5, 400]])
def test_append_in_steps(Dh, steps):
    L, B, Hkv, cap = 2, 3, 3, 900
    g = np.random.default_rng(Dh + len(steps))
    shape = _shape(B, 6, Hkv, Dh, 1, cap)
    cache = _poisoned(shape, L)
    rows = {(l, b): {x: np.zeros((0, Hkv, Dh)) for x in "kv"} for l in range(L) for b in range(B)}
    written = {(l, b): set() for l in range(L) for b in range(B)}
    length = np.zeros(B, np.int64)
    for step, n in enumerate(steps):
        new = np.maximum(n - np.arange(B) * (step % 2), 0)               # ragged every other time
        T = max(int(new.max()), 1) + 2
        k, v = (_bf16(g.standard_normal((L, B, T, Hkv, Dh)) * np.exp2(g.integers(-9, 9, (L, B, 1, Hkv, 1)))) for _ in range(2))
        picked = None
        if step % 3 == 1:                                                # rows picked from anywhere, some of them nowhere
            picked = g.integers(0, T, (B, T)).astype(np.int32)
            picked[0, 0], picked[1, 0] = -1, T
        length += new
        ygg.block8_append(shape, L, k.to(DEV), v.to(DEV), cache, to_dev(length.astype(np.int32)), to_dev(new.astype(np.int32)),
                          rows=None if picked is None else to_dev(picked))
        for (l, b), r in rows.items():
            which = np.arange(new[b]) if picked is None else picked[b, :new[b]]
            ok = (which >= 0) & (which < T)
            for x, t in (("k", k), ("v", v)):
                got = np.where(ok[:, None, None], t[l, b].double().numpy()[np.where(ok, which, 0)], 0.0)
                r[x] = np.concatenate((r[x], got))
            written[l, b] = set(range(int(length[b]) // 64))
        ends = {(l, b): range(int(length[b]) // 64 * 64, int(length[b])) for l in range(L) for b in range(B)}
        _check_cache(cache, rows, written, ends, Dh)


def test_append_twice_gives_the_same_and_a_length_may_be_taken_back():
    shape = _shape(1, 2, 2, 128, 1, 256)
    cache = _poisoned(shape, 1)
    g = np.random.default_rng(1)
    k, v = (_bf16(g.standard_normal((1, 1, 100, 2, 128))).to(DEV) for _ in range(2))
    i32 = lambda x: torch.tensor([x], dtype=torch.int32, device=DEV)
    ygg.block8_append(shape, 1, k, v, cache, i32(62), i32(62))
    ygg.block8_append(shape, 1, k[:, :, 62:70].contiguous(), v[:, :, 62:70].contiguous(), cache, i32(70), i32(8))
    first = [t.clone() for t in cache.tensors()]
    ygg.block8_append(shape, 1, k[:, :, 62:70].contiguous(), v[:, :, 62:70].contiguous(), cache, i32(70), i32(8))   # block 0 again, from its tail
    bits = lambda t: t.view(torch.int16) if t.dtype == torch.bfloat16 else t.view(torch.int32) if t.dtype == torch.float32 else t
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip(first, cache.tensors()))
    # back to 60 tokens, four others behind them
    ygg.block8_append(shape, 1, k[:, :, 90:94].contiguous(), v[:, :, 90:94].contiguous(), cache, i32(64), i32(4))
    want = torch.cat((k[0, 0, :60], k[0, 0, 90:94])).double().cpu().numpy().transpose(1, 0, 2)
    scale = plain.block_scale(want)
    assert np.array_equal(cache.k_scale[0, 0, :, 0].cpu().numpy(), scale)
    value = plain.decode(cache.k_codes[0, 0, :, 0].cpu().numpy(), scale, "k")
    assert (np.abs(value - want) <= np.abs(want) * 2.0 ** -4 + scale[:, None, None] * 2.0 ** -10).all()


def test_append_of_zeros_tiny_and_huge_values():
    shape = _shape(1, 3, 3, 64, 1, 128)
    cache = _poisoned(shape, 1)
    x = torch.zeros((1, 1, 64, 3, 64), dtype=torch.bfloat16)
    x[0, 0, 5, 1, 7] = 1e-38
    x[0, 0, 6, 2] = 3e38
    n = torch.tensor([64], dtype=torch.int32, device=DEV)
    ygg.block8_append(shape, 1, x.to(DEV), x.to(DEV), cache, n, n)
    for t in (cache.k_scale, cache.v_scale):
        s = t[0, 0, :, 0].cpu().numpy()
        assert s[0] == 1 and s[1] == np.float32(2.0 ** -100) and s[2] == np.float32(x[0, 0, 6, 2, 0].item()) / np.float32(448)
    for codes, which in ((cache.k_codes, "k"), (cache.v_codes, "v")):
        c = plain.decode(codes[0, 0, :, 0].cpu().numpy(), np.ones(3, np.float32), which)
        assert (c[:2] == 0).all() and (c[2, 6] == 448).all()


def test_contract_violations_stay_inside():
    """Lengths and counts out of range are clamped: nothing is written behind the capacity, nothing for no new tokens."""
    shape = _shape(3, 1, 1, 64, 1, 100)
    cache = _poisoned(shape, 1)
    k = torch.ones((1, 3, 80, 1, 64), dtype=torch.bfloat16, device=DEV)
    ygg.block8_append(shape, 1, k, k, cache, to_dev(np.array([1 << 30, -5, 64], np.int32)), to_dev(np.array([1 << 30, 7, -1], np.int32)))
    assert not torch.isnan(cache.k_scale[0, 0, :, 0]).any() and torch.isnan(cache.k_scale[0, 0, :, 1]).all()     # tokens 20 .. 99
    assert torch.isnan(cache.k_scale[0, 1:]).all() and torch.isnan(cache.k_tail[0, 1:]).all()


# ---------------------------------------------------------------- attention

def _problem(B, Hq, Hkv, Dh, N, lens, seed, cap=None, tree="random", q_gain=1.0, k_gain=None, v_gain=None):
    """A cache whose unused parts are poisoned, and what it stands for in float64."""
    g = np.random.default_rng(seed)
    parent = np.stack([wl.chain_tree(N) if tree == "chain" else wl.random_topological_tree(seed, N, sub=b) for b in range(B)])
    D = max(len(plain.path_of(p, i)) for p in parent for i in range(N)) - 1
    lens = np.asarray(lens)
    shape = _shape(B, Hq, Hkv, Dh, N, (int(lens.max()) if cap is None else cap) + D + 1, D=D)
    shape.max_seq_len = int(lens.max()) if cap is None else cap
    cache = _poisoned(shape, 1).layer(0)
    dense = {}
    nblk = cache.k_scale.shape[-1]
    for x, gain in (("k", k_gain), ("v", v_gain)):
        codes = g.integers(0, 256, (B, Hkv, nblk, 64 * Dh)).astype(np.uint8)
        codes[(codes & 127) == 127] = 0x30
        size = (2.0 ** -8 if gain is None else gain(g, (B, Hkv, nblk))) * np.exp2(g.uniform(-1, 1, (B, Hkv, nblk)))
        scale = np.broadcast_to(size, (B, Hkv, nblk)).astype(np.float32).copy()
        tail, tree_rows = _bf16(g.standard_normal((B, 128, Hkv, Dh))), _bf16(g.standard_normal((B, N, Hkv, Dh)))
        dense[x] = []
        for b in range(B):
            full = int(lens[b]) // 64
            blocks = plain.decode(codes[b, :, :full], scale[b, :, :full], x).reshape(Hkv, full * 64, Dh)
            at = full % 2 * 64
            rows = tail[b, at:at + int(lens[b]) - full * 64].double().numpy().transpose(1, 0, 2)
            dense[x].append(np.concatenate((blocks, rows, tree_rows[b].double().numpy().transpose(1, 0, 2)), 1))
            codes[b, :, full:], scale[b, :, full:] = NAN_CODE, np.nan
            keep = tail[b, at:at + int(lens[b]) - full * 64].clone()
            tail[b] = NAN_ROW
            tail[b, at:at + int(lens[b]) - full * 64] = keep
        getattr(cache, x + "_codes").copy_(torch.from_numpy(codes))
        getattr(cache, x + "_scale").copy_(torch.from_numpy(scale))
        getattr(cache, x + "_tail").copy_(tail)
        dense[x + "_tree"] = tree_rows.to(DEV)
    q = _bf16(g.standard_normal((B, N, Hq, Dh)) * q_gain).to(DEV)
    return dict(shape=shape, cache=cache, lens=lens, parent=parent, q=q, dense=dense)


def _attend(p, want_lse=True, stream=None):
    s = p["shape"]
    out = torch.full_like(p["q"], float("nan"))
    lse = torch.full(p["q"].shape[:3], float("nan"), dtype=torch.float32, device=DEV) if want_lse else None
    ws = workspace(s, ygg.OP_ATTENTION_BLOCK8, poison=0xFF)
    ygg.tree_attention_block8(s, p["q"], p["cache"], to_dev(p["lens"].astype(np.int32)), p["dense"]["k_tree"], p["dense"]["v_tree"],
                              to_dev(p["parent"]), out, lse, ws)
    torch.cuda.synchronize()
    return out, lse


def _check(p, out, lse, sequences=None):
    s = p["shape"]
    G, Dh = s.n_q_heads // s.n_kv_heads, s.head_dim
    out, lse, q = to_f64(out), to_f64(lse), to_f64(p["q"])
    for b in sequences or range(s.batch):
        for h in range(s.n_kv_heads):
            keys, values = p["dense"]["k"][b][h], p["dense"]["v"][b][h]
            hs = slice(h * G, (h + 1) * G)
            ref, ref_lse, size = plain.tree_attention(q[b, :, hs], keys, values, int(p["lens"][b]), p["parent"][b], s.softmax_scale)
            # Scores.  q as hi + lo: scaled to a largest magnitude in [128, 256), the remainder's step below 2^-6 is 2^-9, so an element is off
            # by 2^-10 at most, 2^-17 of the largest.  The matrix instruction cuts each of a sum's products to a multiple of 2^-13 of the
            # largest (measured: 2^16 + 31 * 4 gives 2^16 + 96), Dh of them at most; adding up in fp32: 2^-22 of the terms.
            kd, qd = np.abs(keys), np.abs(q[b, :, hs]).max()
            score = s.softmax_scale * qd * (kd.sum(-1).max() * (2.0 ** -17 + 2.0 ** -22) + kd.max() * Dh * 2.0 ** -13)
            # Weights: by 2^-8 (bf16, or twice 2^-4), by the scores' error on both sides of the quotient.  Their products with V are cut
            # likewise: 32 of them by 2^-13 of the largest, 2^-8 of the sum of their magnitudes at most.  Sums over the keys in fp32:
            # 2^-12; a partial row in fp16: 2^-12 of its largest; the bf16 result: half a step.
            row = np.maximum(size.max(-1, keepdims=True), np.abs(ref).max(-1, keepdims=True))
            tol = size * (2.0 ** -7 + 2 * score + 2.0 ** -12) + row * 2.0 ** -12 + np.abs(ref) * 2.0 ** -8
            err = np.abs(out[b, :, hs] - ref)
            assert (err <= tol).all(), (b, h, float((err / tol).max()))
            assert np.sqrt((err ** 2).mean()) <= 0.01 * np.sqrt((ref ** 2).mean()), (b, h)      # a lost key or a wrong mask bit shows here
            off = np.abs(lse[b, :, hs] - ref_lse)
            assert (off <= score + 2.0 ** -18 * (1 + np.abs(ref_lse))).all(), (b, h)
            # the cuts have the products' signs, which are independent: sqrt(Dh) of them, not Dh
            assert np.sqrt((off ** 2).mean()) <= score / 4 + 2.0 ** -18 * (1 + np.abs(ref_lse).max()), (b, h)


SHAPES = [  # B, Hq, Hkv, Dh, N, lens
    (1, 1, 1, 64, 1, [0]), (1, 4, 1, 128, 1, [1]), (1, 8, 2, 128, 1, [63]), (2, 8, 2, 128, 1, [64, 0]), (3, 8, 8, 64, 1, [65, 127, 128]),
    (1, 4, 4, 64, 2, [129]), (2, 8, 2, 128, 8, [1000, 3]), (1, 4, 4, 128, 33, [700]), (2, 12, 12, 64, 49, [64, 321]), (1, 32, 8, 128, 16, [640]),
    (1, 8, 2, 128, 17, [1919]), (1, 8, 2, 64, 32, [2048]), (3, 6, 2, 128, 43, [77, 500, 0]), (1, 8, 2, 128, 65, [256]), (2, 16, 1, 64, 21, [130, 1]),
    (1, 4, 1, 128, 129, [1500]), (1, 2, 2, 64, 300, [200]), (1, 16, 2, 128, 49, [4095]), (5, 4, 2, 128, 13, [10, 2000, 64, 128, 129]),
    (70, 2, 1, 128, 3, [(37 * b) % 200 for b in range(70)]), (16, 8, 1, 64, 1, [512 + 100 * b for b in range(16)]),
    (1, 64, 1, 128, 1, [9999]), (300, 1, 1, 64, 1, [b % 130 for b in range(300)]),
]


@pytest.mark.parametrize("B,Hq,Hkv,Dh,N,lens", SHAPES)
def test_attention_shapes(B, Hq, Hkv, Dh, N, lens):
    p = _problem(B, Hq, Hkv, Dh, N, lens, seed=N * 31 + B)
    _check(p, *_attend(p))


@pytest.mark.parametrize("Dh", [64, 128])
@pytest.mark.parametrize("G,N", [(4, 1), (1, 32), (4, 9), (1, 64), (4, 17), (2, 61)])
@pytest.mark.parametrize("lens", [[256], [700, 0, 319], [5, 1, 255, 64]])
def test_attention_with_a_compute_unit_to_each_sequence(Dh, G, N, lens):
    """Bounds from four blocks on with few sequences: the keys of one are dealt out to many wavefronts, some of which get none."""
    p = _problem(len(lens), 2 * G, 2, Dh, N, lens, seed=N + len(lens), cap=max(max(lens), 256))
    _check(p, *_attend(p))


def test_attention_widest_tree_and_longest_chain():
    for tree in ("random", "chain"):
        p = _problem(1, 2, 1, 128, 1024, [100], seed=6, tree=tree)
        _check(p, *_attend(p))


def test_attention_where_the_bound_is_far_above_the_lengths():
    p = _problem(4, 8, 2, 128, 9, [0, 70, 1, 640], seed=8, cap=20000)
    _check(p, *_attend(p))


@pytest.mark.parametrize("Dh", [64, 128])
def test_attention_scores_and_scales_over_a_wide_range(Dh):
    """Rows whose softmax is one key, whose maximum comes late, whose blocks' scales span many powers of two."""
    spread = lambda lo, hi: lambda g, s: np.exp2(g.uniform(lo, hi, s) - 8)
    rising = lambda g, s: np.broadcast_to(np.exp2(np.linspace(-8, 3, s[-1]) - 8), s)
    falling = lambda g, s: np.broadcast_to(np.exp2(np.linspace(3, -8, s[-1]) - 8), s)
    for seed, (kg, vg, qg) in enumerate([(spread(-6, 4), spread(-20, 20), 1.0), (rising, spread(-3, 3), 4.0), (falling, rising, 4.0),
                                         (spread(-40, -30), spread(-60, -50), 1.0), (None, spread(30, 40), 1e-3)]):
        p = _problem(2, 8, 2, Dh, 11, [1700, 333], seed=seed, k_gain=kg, v_gain=vg, q_gain=qg)
        _check(p, *_attend(p))


def test_attention_rows_of_q_of_any_magnitude():
    p = _problem(1, 4, 2, 128, 7, [300], seed=3)
    q = p["q"]
    q[0, 0] = 0
    q[0, 1] *= 1e-30
    q[0, 2] *= 1e-39                      # subnormal
    q[0, 3, :, :64] *= 1e-6
    _check(p, *_attend(p))


def test_attention_without_lse_on_another_stream_and_again():
    p = _problem(2, 8, 2, 128, 20, [500, 64], seed=4)
    out, _ = _attend(p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again, none = _attend(p, want_lse=False)
    assert torch.equal(out, again) and none is None


def test_attention_at_an_offset_beyond_32_bits():
    """Two sequences whose code slabs are 4.3 GB each: the second's first block lies behind 32-bit offsets."""
    B, Hkv, Dh, nblk = 2, 4, 128, 131073
    shape = _shape(B, 4, Hkv, Dh, 1, nblk * 64, most=200)
    cache = ygg.BlockCache(*(torch.empty((B, Hkv, nblk, 64 * Dh), dtype=torch.uint8, device=DEV) for _ in range(2)),
                           *(torch.ones((B, Hkv, nblk), dtype=torch.float32, device=DEV) for _ in range(2)),
                           *(torch.zeros((B, 128, Hkv, Dh), dtype=torch.bfloat16, device=DEV) for _ in range(2)))
    g = np.random.default_rng(0)
    k, v = (_bf16(g.standard_normal((1, B, 200, Hkv, Dh))).to(DEV) for _ in range(2))
    n = torch.tensor([130, 200], dtype=torch.int32, device=DEV)
    ygg.block8_append(shape, 1, k, v, cache, n, n)
    small = _shape(B, 4, Hkv, Dh, 1, 300, most=200)
    near = ygg.new_block_cache(small, 1, device=DEV)
    ygg.block8_append(small, 1, k, v, near, n, n)
    got = []
    for s, c in ((shape, cache), (small, near.layer(0))):
        out = torch.empty((B, 1, 4, Dh), dtype=torch.bfloat16, device=DEV)
        ygg.tree_attention_block8(s, k[0, :, :1].contiguous(), c, n, k[0, :, 1:2].contiguous(), v[0, :, 1:2].contiguous(),
                                  torch.full((B, 1), -1, dtype=torch.int32, device=DEV), out, None, workspace(s, ygg.OP_ATTENTION_BLOCK8))
        got.append(out)
    assert torch.equal(*got) and not torch.isnan(got[0]).any()


def test_refusals_on_the_gpu_binding():
    p = _problem(1, 4, 2, 128, 3, [10], seed=1)
    s, c = p["shape"], p["cache"]
    args = [p["q"], c, torch.tensor([10], dtype=torch.int32, device=DEV), p["dense"]["k_tree"], p["dense"]["v_tree"], to_dev(p["parent"]),
            torch.empty_like(p["q"])]
    ws = workspace(s, ygg.OP_ATTENTION_BLOCK8)
    with pytest.raises(RuntimeError, match="workspace"):
        ygg.tree_attention_block8(s, *args)
    with pytest.raises(TypeError, match="k_codes"):
        bad = ygg.BlockCache(*c.tensors())
        bad.k_codes = c.k_codes.view(torch.int8)
        ygg.tree_attention_block8(s, args[0], bad, *args[2:], workspace=ws)
    with pytest.raises(TypeError, match="q:"):
        ygg.tree_attention_block8(s, args[0].float(), *args[1:], workspace=ws)
    with pytest.raises(ValueError, match="k_tree"):
        ygg.tree_attention_block8(s, *args[:3], args[3].transpose(1, 2), *args[4:], workspace=ws)
    with pytest.raises(RuntimeError, match="unsupported"):
        plain_shape = ygg.Shape(**{**s.__dict__, "kv_dtype": ygg.BF16})
        ygg.tree_attention_block8(plain_shape, *args, workspace=ws)
    with pytest.raises(RuntimeError, match="unsupported"):      # and the other calls do not take the block type
        ygg.tree_attention(s, args[0], args[3], args[4], args[2], args[3], args[4], args[5], args[6], workspace=ws)


def test_tensors_smaller_than_the_shape_are_refused():
    p = _problem(2, 4, 2, 64, 3, [70, 10], seed=1)
    s, c, i32 = p["shape"], p["cache"], dict(dtype=torch.int32, device=DEV)
    ws = workspace(s, ygg.OP_ATTENTION_BLOCK8)
    lens = torch.tensor([70, 10], **i32)
    good = dict(q=p["q"], cache=c, seq_lens=lens, k_tree=p["dense"]["k_tree"], v_tree=p["dense"]["v_tree"], parent_idx=to_dev(p["parent"]),
                out=torch.empty_like(p["q"]), lse=torch.empty((2, 3, 4), device=DEV), workspace=ws)
    ygg.tree_attention_block8(s, **good)
    for name in ("q", "seq_lens", "k_tree", "v_tree", "parent_idx", "out", "lse"):
        with pytest.raises(ValueError, match=name):
            ygg.tree_attention_block8(s, **{**good, name: good[name][:1]})
    for name in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail"):
        bad = ygg.BlockCache(*c.tensors())
        setattr(bad, name, getattr(c, name)[:1])
        with pytest.raises(ValueError, match=name):
            ygg.tree_attention_block8(s, **{**good, "cache": bad})
    k = torch.zeros((1, 2, 5, 2, 64), dtype=torch.bfloat16, device=DEV)
    n = torch.tensor([1, 1], **i32)
    one = ygg.BlockCache(*(t[None] for t in c.tensors()))
    for kw in (dict(v_new=k[:, :1]), dict(n_new=n[:1]), dict(seq_lens=n[:1]), dict(rows=torch.zeros((1, 3), **i32)), dict(n_layers=2)):
        with pytest.raises(ValueError, match=next(iter(kw)) if "n_layers" not in kw else "k_new"):
            ygg.block8_append(s, **{**dict(n_layers=1, k_new=k, v_new=k, cache=one, seq_lens=n, n_new=n), **kw})


# ---------------------------------------------------------------- lengths taken back

def _stands_for(cache, b, rows, L, Dh):
    """Sequence b of a one-layer cache holds the L tokens of rows {"k"/"v": [>= L, Hkv, Dh] float64}."""
    for x in "kv":
        codes, scale, tail = (getattr(cache, f"{x}_{y}")[0, b].cpu() for y in ("codes", "scale", "tail"))
        for k in range(L // 64):
            block = rows[x][64 * k:64 * k + 64].transpose(1, 0, 2)
            want = plain.block_scale(block)
            assert np.array_equal(scale[:, k].numpy(), want), (x, b, L, k)
            value = plain.decode(codes[:, k].numpy(), want, x)
            assert (np.abs(value - block) <= np.abs(block) * 2.0 ** -4 + want[:, None, None] * 2.0 ** -10).all(), (x, b, L, k)    # half a step
        for t in range(L // 64 * 64, L):
            assert np.array_equal(tail[t % 128].double().numpy(), rows[x][t]), (x, b, L, t)


@pytest.mark.parametrize("n", [1, 8, 64, 100, 200])
def test_lengths_that_may_be_taken_back_to(n):
    """The open block's tokens, multiples of 64, and in the block before up to where the append that completed it began: attention at each
    of these lengths, and an append behind it."""
    Dh, G = 64, 2
    end = -(-300 // n) * n
    before = end // 64 - 1                                       # the block before the open one
    began = (64 * before + 63) // n * n
    lengths = sorted({*range(64 * (end // 64), end + 1), *range(0, end + 1, 64), *range(64 * before, began + 1)})
    B = len(lengths)
    g = np.random.default_rng(n)
    shape = _shape(B, G, 1, Dh, 1, end + 80)
    cache = _poisoned(shape, 1)
    k, v = (_bf16(np.broadcast_to(g.standard_normal((1, 1, end, 1, Dh)), (1, B, end, 1, Dh))) for _ in range(2))
    i32 = lambda x: torch.full((B,), x, dtype=torch.int32, device=DEV)
    for at in range(0, end, n):
        ygg.block8_append(shape, 1, k[:, :, at:at + n].contiguous().to(DEV), v[:, :, at:at + n].contiguous().to(DEV), cache, i32(at + n), i32(n))
    lens = to_dev(np.array(lengths, np.int32))
    q, kt, vt = (_bf16(g.standard_normal((B, 1, h, Dh))) for h in (G, 1, 1))
    out = torch.full((B, 1, G, Dh), float("nan"), dtype=torch.bfloat16, device=DEV)
    ygg.tree_attention_block8(shape, q.to(DEV), cache.layer(0), lens, kt.to(DEV), vt.to(DEV), i32(-1)[:, None], out, None,
                              workspace(shape, ygg.OP_ATTENTION_BLOCK8, poison=0xFF))
    out = to_f64(out)
    for b, L in enumerate(lengths):
        _stands_for(cache, b, {"k": k[0, b].double().numpy(), "v": v[0, b].double().numpy()}, L, Dh)
        dense = {}
        for x, rows, tree in (("k", k, kt), ("v", v, vt)):
            blocks = plain.decode(getattr(cache, x + "_codes")[0, b, :, :L // 64].cpu().numpy(), getattr(cache, x + "_scale")[0, b, :, :L // 64].cpu().numpy(), x)
            dense[x] = np.concatenate((blocks.reshape(-1, Dh), rows[0, b, L // 64 * 64:L, 0].double().numpy(), tree[b, :, 0].double().numpy()))
        ref, _, size = plain.tree_attention(q[b].double().numpy(), dense["k"], dense["v"], L, np.array([-1]), shape.softmax_scale)
        # as in _check, with |q|, |k| and |v| below 6: scores off by at most 6 * 6 * 64 * 2^-13 / 8 = 2^-4.8, on both sides of the quotient
        assert (np.abs(out[b] - ref) <= size * 2 * 2.0 ** -4.8 + 6 * 2.0 ** -12 + np.abs(ref) * 2.0 ** -6).all(), (b, L)
    more = 70
    k2, v2 = (_bf16(g.standard_normal((1, B, more, 1, Dh))) for _ in range(2))
    ygg.block8_append(shape, 1, k2.to(DEV), v2.to(DEV), cache, lens + more, i32(more))
    for b, L in enumerate(lengths):
        rows = {x: np.concatenate((old[0, b, :L].double().numpy(), new[0, b].double().numpy())) for x, old, new in (("k", k, k2), ("v", v, v2))}
        _stands_for(cache, b, rows, L + more, Dh)


def test_new_rows_of_another_form_than_the_cache_are_refused():
    """Rows without a layer dimension, and K and V of different row counts, hold enough elements but lie differently."""
    shape = _shape(2, 4, 2, 64, 1, 200)
    cache, n = _poisoned(shape, 1), torch.tensor([5, 3], dtype=torch.int32, device=DEV)
    k = torch.ones((1, 2, 5, 2, 64), dtype=torch.bfloat16, device=DEV)
    call = lambda k_new, v_new, **kw: ygg.block8_append(shape, 1, k_new, v_new, cache, n, n, **kw)
    for bad in (k[0], k.flatten(3), k.view(1, 2, 5, 1, 128), torch.cat((k, k), 1), torch.cat((k, k), 4)):
        with pytest.raises(ValueError, match="k_new"):
            call(bad, bad)
    for bad in (torch.cat((k, k), 2), k[0], torch.cat((k, k), 1)):
        with pytest.raises(ValueError, match="v_new"):
            call(k, bad)
    assert torch.isnan(cache.k_tail).all() and torch.isnan(cache.v_tail).all()      # nothing was written
    call(k, k)
    call(torch.cat((k, k)), k)                                                     # (layers that the call leaves out)


def test_a_cache_of_another_size_is_refused():
    """Several layers given to the attention of one, a capacity other than the shape's, another batch in several layers."""
    p = _problem(2, 4, 2, 64, 3, [70, 10], seed=1)
    s, i32 = p["shape"], dict(dtype=torch.int32, device=DEV)
    lens = torch.tensor([70, 10], **i32)
    args = dict(seq_lens=lens, k_tree=p["dense"]["k_tree"], v_tree=p["dense"]["v_tree"], parent_idx=to_dev(p["parent"]), out=torch.empty_like(p["q"]),
                workspace=workspace(s, ygg.OP_ATTENTION_BLOCK8))
    wider = ygg.Shape(**{**s.__dict__, "kv_capacity": s.kv_capacity + 128})
    more = ygg.Shape(**{**s.__dict__, "batch": 4})
    k, n = torch.zeros((1, 2, 5, 2, 64), dtype=torch.bfloat16, device=DEV), torch.tensor([1, 1], **i32)
    for cache in (ygg.new_block_cache(s, 2, device=DEV), ygg.new_block_cache(wider, 1, device=DEV), ygg.new_block_cache(more, 2, device=DEV)):
        with pytest.raises(ValueError, match="k_codes"):
            ygg.tree_attention_block8(s, p["q"], cache, **args)
    for cache in (ygg.new_block_cache(wider, 2, device=DEV), ygg.new_block_cache(more, 2, device=DEV), ygg.new_block_cache(s, 1, device=DEV)):
        with pytest.raises(ValueError, match="k_codes"):
            ygg.block8_append(s, 2, torch.cat((k, k)), torch.cat((k, k)), cache, n, n)
    for cache in (ygg.new_block_cache(s, 1, device=DEV), ygg.new_block_cache(more, 1, device=DEV)):     # (further sequences may follow one layer)
        ygg.tree_attention_block8(s, p["q"], cache, **args)
        ygg.tree_attention_block8(s, p["q"], cache.layer(0), **args)
        ygg.block8_append(s, 1, k, k, cache, n, n)
    ygg.block8_append(s, 1, k, k, ygg.new_block_cache(s, 2, device=DEV), n, n)                          # (and further layers the call's)


def test_longer_trees_than_the_shape_are_refused_in_a_batch():
    p = _problem(2, 4, 2, 64, 3, [70, 10], seed=1)
    s = p["shape"]
    good = dict(q=p["q"], seq_lens=torch.tensor([70, 10], dtype=torch.int32, device=DEV), k_tree=p["dense"]["k_tree"], v_tree=p["dense"]["v_tree"],
                parent_idx=to_dev(p["parent"]), out=torch.empty_like(p["q"]), lse=torch.empty((2, 3, 4), device=DEV))
    ws = workspace(s, ygg.OP_ATTENTION_BLOCK8)
    for name in ("q", "k_tree", "v_tree", "parent_idx", "out", "lse"):
        with pytest.raises(ValueError, match=name):
            ygg.tree_attention_block8(s, cache=p["cache"], workspace=ws, **{**good, name: torch.cat((good[name], good[name]), 1)})
    # one sequence: the first nodes of a longer tree
    first = ygg.Shape(**{**s.__dict__, "n_nodes": 2, "batch": 1})
    out = torch.full_like(p["q"], float("nan"))
    ygg.tree_attention_block8(first, cache=p["cache"], workspace=ws, **{**good, "out": out[:1], "lse": None, **{x: good[x][:1] for x in (
        "q", "k_tree", "v_tree", "parent_idx")}})
    assert not torch.isnan(out[0, :2]).any() and torch.isnan(out[0, 2:]).all() and torch.isnan(out[1]).all()


@pytest.mark.parametrize("Dh", [64, 128])
def test_codes_are_the_ones_of_the_definition_byte_for_byte(Dh):
    """Random blocks of many sizes, values half way between two codes at a scale of a power of two (ties), zeros of both signs, steps
    below the smallest normal code, and largest magnitudes whose quotient rounds above 448."""
    Hkv, blocks = 3, 40
    g = np.random.default_rng(Dh)
    shape = _shape(1, Hkv, Hkv, Dh, 1, 64 * blocks)
    cache = _poisoned(shape, 1)
    x = g.standard_normal((2, blocks, 64, Hkv, Dh)) * np.exp2(g.integers(-12, 12, (2, blocks, 1, Hkv, 1)))
    values = plain.e4m3_values()[:127]
    ties = np.concatenate(((values[1:] + values[:-1]) / 2, values))
    x[:, 3:9] = g.choice(np.concatenate((ties, -ties)), (2, 6, 64, Hkv, Dh))
    x[:, 3:9, 0, :, 0] = 448.0
    x[:, 5] *= 2.0 ** -7
    x[:, 6] *= 2.0 ** 30
    x[:, 9:12, ::3] = -0.0
    x[:, 10, 1::3] *= 1e-4
    rows = _bf16(x.reshape(2, 1, 1, blocks * 64, Hkv, Dh))
    n = torch.tensor([64 * blocks], dtype=torch.int32, device=DEV)
    ygg.block8_append(shape, 1, rows[0].to(DEV), rows[1].to(DEV), cache, n, n)
    for i, which in enumerate("kv"):
        block = rows[i].double().numpy().reshape(blocks, 64, Hkv, Dh).transpose(2, 0, 1, 3)          # [Hkv, blocks, 64, Dh]
        scale = plain.block_scale(block)
        assert np.array_equal(getattr(cache, which + "_scale")[0, 0].cpu().numpy(), scale)
        got, want = getattr(cache, which + "_codes")[0, 0].cpu().numpy(), plain.encode(block, scale, which)
        assert np.array_equal(got, want), (which, np.argwhere(got != want)[:5])
        # the test does reach ties, and they go both ways
        tied = np.isin(np.abs(block[:, 3]), (values[1:] + values[:-1]) / 2)
        kept = np.abs(plain.decode(want[:, 3], np.ones(Hkv, np.float32), which)) > np.abs(block[:, 3])
        assert (tied & kept).any() and (tied & ~kept).any() and (scale[:, 3] == 1).all()
