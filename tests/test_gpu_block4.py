"""ygg_block4_append and ygg_tree_attention_block4 against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2512_23858_amd as ygg
import plain_ops
import plain_prompt as plain
import ygg_workloads as wl
from gpu_util import DEV, to_dev, to_f64, workspace
from test_gpu_block8 import _bf16, _check
from test_gpu_block8 import _shape as _block8_shape

gpu = pytest.mark.gpu
NAN_SCALE, NAN_ROW = 255, float("nan")      # 255 is the scale format's NaN


def _shape(*args, **kw):
    s = _block8_shape(*args, **kw)
    s.kv_dtype = ygg.FP4_BLOCK
    return s


# ---------------------------------------------------------------- append

def _poisoned(shape, layers):
    c = ygg.new_block4_cache(shape, layers, device=DEV)
    for t, v in zip(c.tensors(), (0x7F, 0x7F, NAN_SCALE, NAN_SCALE, NAN_ROW, NAN_ROW)):
        t.fill_(v)
    return c


def _check_cache(cache, rows, length):
    """rows: {(layer, b): {"k"/"v": [length, Hkv, Dh] float64}}: every token ever appended.  Whole blocks are compared byte for byte."""
    for x in "kv":
        codes, scale, tail = (getattr(cache, f"{x}_{y}").cpu() for y in ("codes", "scale", "tail"))
        codes, scale, tail = codes.numpy(), scale.numpy(), tail.double().numpy()
        nblk = scale.shape[3]
        for (l, b), r in rows.items():
            full = int(length[b]) // 64
            want = plain.encode(r[x][:64 * full].reshape(full, 64, *r[x].shape[1:]).transpose(2, 0, 1, 3), x)
            assert np.array_equal(scale[l, b, :, :full], want[1]), (x, l, b)
            assert np.array_equal(codes[l, b, :, :full], want[0]), (x, l, b)
            assert (scale[l, b, :, full:nblk] == NAN_SCALE).all() and (codes[l, b, :, full:nblk] == 0x7F).all(), (x, l, b)
            for t in range(64 * full, int(length[b])):
                assert np.array_equal(tail[l, b, t % 128], r[x][t]), (x, l, b, t)


@gpu
@pytest.mark.parametrize("Dh", [64, 128])
@pytest.mark.parametrize("steps", [[1], [63, 1], [64], [65, 62, 1, 128], [1, 200, 0, 7, 56, 64], [300, 5, 400]])
def test_append_in_steps(Dh, steps):
    L, B, Hkv, cap = 2, 3, 3, 900
    g = np.random.default_rng(Dh + len(steps))
    shape = _shape(B, 6, Hkv, Dh, 1, cap)
    cache = _poisoned(shape, L)
    rows = {(l, b): {x: np.zeros((0, Hkv, Dh)) for x in "kv"} for l in range(L) for b in range(B)}
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
        ygg.block4_append(shape, L, k.to(DEV), v.to(DEV), cache, to_dev(length.astype(np.int32)), to_dev(new.astype(np.int32)),
                          rows=None if picked is None else to_dev(picked))
        for (l, b), r in rows.items():
            which = np.arange(new[b]) if picked is None else picked[b, :new[b]]
            ok = (which >= 0) & (which < T)
            for x, t in (("k", k), ("v", v)):
                got = np.where(ok[:, None, None], t[l, b].double().numpy()[np.where(ok, which, 0)], 0.0)
                r[x] = np.concatenate((r[x], got))
        _check_cache(cache, rows, length)


@gpu
@pytest.mark.parametrize("Dh", [64, 128])
def test_codes_are_the_ones_of_the_definition_byte_for_byte(Dh):
    """Random blocks of many sizes, sizes that differ within a group's neighbours, values half way between two codes (ties), largest
    magnitudes between 6 and 7 and above, zeros of both signs, subnormal values, values near the ends of the type."""
    Hkv, blocks = 3, 30
    g = np.random.default_rng(Dh)
    shape = _shape(1, Hkv, Hkv, Dh, 1, 64 * blocks)
    cache = _poisoned(shape, 1)
    x = g.standard_normal((2, blocks, 64, Hkv, Dh)) * np.exp2(g.integers(-12, 12, (2, blocks, 1, Hkv, 1)))
    x[:, 3:6] *= np.exp2(g.integers(-6, 6, (2, 3, 64, Hkv, Dh)))
    mids = (plain.LEVELS[1:] + plain.LEVELS[:-1]) / 2
    ties = np.concatenate((mids, plain.LEVELS))
    x[:, 6:12] = g.choice(np.concatenate((ties, -ties)), (2, 6, 64, Hkv, Dh))
    x[:, 6:8, 0, :, ::32] = 6.0
    x[0, 6:8, :, :, ::32] = 6.0
    x[1, 6:8, ::32] = -6.0
    x[:, 8] = g.choice([6.5, 7.0, 7.03125, -6.96875, 3.5, 3.515625, 0.25, -0.75], (2, 64, Hkv, Dh))
    x[:, 9] *= 2.0 ** -7
    x[:, 10] *= 2.0 ** 30
    x[:, 12:15, ::3] = -0.0
    x[:, 13, 1::3] *= 1e-4
    x[:, 15] = 0
    x[:, 16] *= 2.0 ** -126                     # below the smallest scale: zeros that keep their signs
    x[:, 17] *= 2.0 ** -104 / np.abs(x[:, 17]).max()
    x[:, 18] *= 3e38 / np.abs(x[:, 18]).max()
    x[:, 19, 5, 1, 7] = 1e-38
    rows = _bf16(x.reshape(2, 1, 1, blocks * 64, Hkv, Dh))
    n = torch.tensor([64 * blocks], dtype=torch.int32, device=DEV)
    ygg.block4_append(shape, 1, rows[0].to(DEV), rows[1].to(DEV), cache, n, n)
    for i, which in enumerate("kv"):
        block = rows[i].double().numpy().reshape(blocks, 64, Hkv, Dh).transpose(2, 0, 1, 3)          # [Hkv, blocks, 64, Dh]
        codes, scale = plain.encode(block, which)
        assert np.array_equal(getattr(cache, which + "_scale")[0, 0].cpu().numpy(), scale), which
        got = getattr(cache, which + "_codes")[0, 0].cpu().numpy()
        assert np.array_equal(got, codes), (which, np.argwhere(got != codes)[:5])
        # the test does reach ties at a scale of 1, and they go both ways
        tied = np.isin(np.abs(block[:, 6]), mids)
        value = np.abs(plain.decode(codes[:, 6], scale[:, 6], which))
        assert (scale[:, 6] == 127).all() and (tied & (value > np.abs(block[:, 6]))).any() and (tied & (value < np.abs(block[:, 6]))).any()


@gpu
def test_append_twice_gives_the_same_and_a_length_may_be_taken_back():
    shape = _shape(1, 2, 2, 128, 1, 256)
    cache = _poisoned(shape, 1)
    g = np.random.default_rng(1)
    k, v = (_bf16(g.standard_normal((1, 1, 100, 2, 128))).to(DEV) for _ in range(2))
    i32 = lambda x: torch.tensor([x], dtype=torch.int32, device=DEV)
    part = lambda a, b: (k[:, :, a:b].contiguous(), v[:, :, a:b].contiguous())
    ygg.block4_append(shape, 1, k, v, cache, i32(62), i32(62))
    ygg.block4_append(shape, 1, *part(62, 70), cache, i32(70), i32(8))
    first = [t.clone() for t in cache.tensors()]
    ygg.block4_append(shape, 1, *part(62, 70), cache, i32(70), i32(8))                               # block 0 again, from its tail
    bits = lambda t: t.view(torch.int16) if t.dtype == torch.bfloat16 else t
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip(first, cache.tensors()))
    ygg.block4_append(shape, 1, *part(90, 94), cache, i32(64), i32(4))                               # back to 60 tokens, four others behind them
    for x, rows in (("k", k), ("v", v)):
        want = torch.cat((rows[0, 0, :60], rows[0, 0, 90:94])).double().cpu().numpy().transpose(1, 0, 2)
        codes, scale = plain.encode(want, x)
        assert np.array_equal(getattr(cache, x + "_codes")[0, 0, :, 0].cpu().numpy(), codes)
        assert np.array_equal(getattr(cache, x + "_scale")[0, 0, :, 0].cpu().numpy(), scale)


@gpu
def test_contract_violations_stay_inside():
    """Lengths and counts out of range are clamped: nothing is written behind the capacity, nothing for no new tokens."""
    shape = _shape(3, 1, 1, 64, 1, 100)
    cache = _poisoned(shape, 1)
    k = torch.ones((1, 3, 80, 1, 64), dtype=torch.bfloat16, device=DEV)
    ygg.block4_append(shape, 1, k, k, cache, to_dev(np.array([1 << 30, -5, 64], np.int32)), to_dev(np.array([1 << 30, 7, -1], np.int32)))
    assert (cache.k_scale[0, 0, :, 0] != NAN_SCALE).all() and (cache.k_scale[0, 0, :, 1] == NAN_SCALE).all()     # tokens 20 .. 99
    assert (cache.k_scale[0, 1:] == NAN_SCALE).all() and torch.isnan(cache.k_tail[0, 1:]).all()


# ---------------------------------------------------------------- attention

def _problem(B, Hq, Hkv, Dh, N, lens, seed, cap=None, tree="random", q_gain=1.0, spread=(2, 2)):
    """A cache of random codes whose unused parts are poisoned, and what it stands for in float64.  spread: K's and V's scales are
    2^-spread .. 2^0 times a quarter, group by group."""
    g = np.random.default_rng(seed)
    parent = np.stack([wl.chain_tree(N) if tree == "chain" else wl.random_topological_tree(seed, N, sub=b) for b in range(B)])
    D = max(len(plain_ops.path_of(p, i)) for p in parent for i in range(N)) - 1
    lens = np.asarray(lens)
    bound = int(lens.max()) if cap is None else cap
    shape = _shape(B, Hq, Hkv, Dh, N, bound + D + 1, D=D)
    shape.max_seq_len = bound
    cache = _poisoned(shape, 1).layer(0)
    nblk = cache.k_scale.shape[2]
    p = dict(shape=shape, cache=cache, lens=lens, parent=parent, dense={})
    for x, powers in zip("kv", spread):
        codes = g.integers(0, 256, (B, Hkv, nblk, 32 * Dh)).astype(np.uint8)
        scale = (125 - g.integers(0, powers + 1, (B, Hkv, nblk, 2 * Dh))).astype(np.uint8)
        tail, tree_rows = _bf16(g.standard_normal((B, 128, Hkv, Dh))), _bf16(g.standard_normal((B, N, Hkv, Dh)))
        for b in range(B):
            full = int(lens[b]) // 64
            codes[b, :, full:], scale[b, :, full:] = 0x7F, NAN_SCALE
            at, n = full % 2 * 64, int(lens[b]) - full * 64
            keep = tail[b, at:at + n].clone()
            tail[b] = NAN_ROW
            tail[b, at:at + n] = keep
        for y, t in (("codes", torch.from_numpy(codes)), ("scale", torch.from_numpy(scale)), ("tail", tail)):
            getattr(cache, f"{x}_{y}").copy_(t)
        p["dense"][x + "_tree"] = tree_rows.to(DEV)
    p["q"] = _bf16(g.standard_normal((B, N, Hq, Dh)) * q_gain).to(DEV)
    _read_back(p)
    return p


def _read_back(p):
    """The keys and values that the cache and the tree's rows stand for now."""
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


def _attend(p, want_lse=True):
    s = p["shape"]
    out = torch.full_like(p["q"], float("nan"))
    lse = torch.full(p["q"].shape[:3], float("nan"), dtype=torch.float32, device=DEV) if want_lse else None
    ygg.tree_attention_block4(s, p["q"], p["cache"], to_dev(p["lens"].astype(np.int32)), p["dense"]["k_tree"], p["dense"]["v_tree"],
                              to_dev(p["parent"]), out, lse, workspace(s, ygg.OP_ATTENTION_BLOCK4, poison=0xFF))
    torch.cuda.synchronize()
    return out, lse


SHAPES = [  # B, Hq, Hkv, Dh, N, lens
    (1, 1, 1, 64, 1, [0]), (1, 4, 1, 128, 1, [1]), (1, 8, 2, 128, 1, [63]), (2, 8, 2, 128, 1, [64, 0]), (3, 8, 8, 64, 1, [65, 127, 128]),
    (1, 4, 4, 64, 2, [129]), (2, 8, 2, 128, 8, [1000, 3]), (1, 4, 4, 128, 33, [700]), (2, 12, 12, 64, 49, [64, 321]), (1, 32, 8, 128, 16, [640]),
    (1, 8, 2, 128, 17, [1919]), (1, 8, 2, 64, 32, [2048]), (3, 6, 2, 128, 43, [77, 500, 0]), (1, 8, 2, 128, 65, [256]), (2, 16, 1, 64, 21, [130, 1]),
    (1, 4, 1, 128, 129, [1500]), (1, 2, 2, 64, 300, [200]), (1, 16, 2, 128, 49, [4095]), (5, 4, 2, 128, 13, [10, 2000, 64, 128, 129]),
    (70, 2, 1, 128, 3, [(37 * b) % 200 for b in range(70)]), (16, 8, 1, 64, 1, [512 + 100 * b for b in range(16)]),
    (1, 64, 1, 128, 1, [9999]), (300, 1, 1, 64, 1, [b % 130 for b in range(300)]),
]


@gpu
@pytest.mark.parametrize("B,Hq,Hkv,Dh,N,lens", SHAPES)
def test_attention_shapes(B, Hq, Hkv, Dh, N, lens):
    p = _problem(B, Hq, Hkv, Dh, N, lens, seed=N * 31 + B)
    _check(p, *_attend(p))


@gpu
@pytest.mark.parametrize("Dh", [64, 128])
@pytest.mark.parametrize("G,N", [(4, 1), (1, 32), (4, 9), (1, 64), (4, 17), (2, 61)])
@pytest.mark.parametrize("lens", [[256], [700, 0, 319], [5, 1, 255, 64]])
def test_attention_with_a_compute_unit_to_each_sequence(Dh, G, N, lens):
    """Bounds from four blocks on with few sequences: the keys of one are dealt out to many wavefronts, some of which get none."""
    p = _problem(len(lens), 2 * G, 2, Dh, N, lens, seed=N + len(lens), cap=max(max(lens), 256))
    _check(p, *_attend(p))


@gpu
def test_attention_widest_tree_and_longest_chain():
    for tree in ("random", "chain"):
        p = _problem(1, 2, 1, 128, 1024, [100], seed=6, tree=tree)
        _check(p, *_attend(p))


@gpu
def test_attention_where_the_bound_is_far_above_the_lengths():
    p = _problem(4, 8, 2, 128, 9, [0, 70, 1, 640], seed=8, cap=20000)
    _check(p, *_attend(p))


@gpu
@pytest.mark.parametrize("Dh", [64, 128])
@pytest.mark.parametrize("spread,q_gain", [((0, 0), 1.0), ((8, 12), 1.0), ((3, 40), 6.0), ((30, 3), 1.0)])
def test_attention_scales_over_a_wide_range(Dh, spread, q_gain):
    """Groups whose scales differ by many powers of two, in one key and from key to key."""
    p = _problem(2, 8, 2, Dh, 11, [1700, 333], seed=Dh, spread=spread, q_gain=q_gain)
    _check(p, *_attend(p))


@gpu
@pytest.mark.parametrize("Dh", [64, 128])
def test_every_code_and_scale_has_its_place(Dh):
    """One value of one token at a time: K's through the score that it alone makes large, V's through the output that it alone is."""
    g = np.random.default_rng(Dh)
    B = 64
    p = _problem(B, 1, 1, Dh, 1, [128] * B, seed=1)
    c, d = p["cache"], p["dense"]
    token, dim = g.integers(0, 128, B), g.integers(0, Dh, B)
    token[:4], dim[:4] = (0, 31, 32, 127), (0, 31, 32, Dh - 1)
    for x in "kv":
        getattr(c, x + "_codes").zero_()
        getattr(c, x + "_scale").fill_(127)
        d[x + "_tree"].zero_()
        code_at, scale_at = plain.stored_at(x, Dh)
        for b in range(B):
            t, k = token[b] % 64, token[b] // 64
            at = int(code_at[t, dim[b]])
            getattr(c, x + "_codes")[b, 0, k, at // 2] = 7 << 4 * (at % 2)                     # 6
            getattr(c, x + "_scale")[b, 0, k, int(scale_at[t, dim[b]])] = 130 if x == "k" else 122
    p["q"].zero_()
    for b in range(B):
        p["q"][b, 0, 0, dim[b]] = 2.0
    p["shape"].softmax_scale = 1.0
    _read_back(p)
    out, lse = _attend(p)
    _check(p, out, lse)
    want = torch.zeros_like(out)
    for b in range(B):
        want[b, 0, 0, dim[b]] = 6 / 32                                                        # its weight is 1: the score is 96 above the others
    assert torch.equal(out, want)


@gpu
def test_attention_rows_of_q_of_any_magnitude():
    p = _problem(1, 4, 2, 128, 7, [300], seed=3)
    q = p["q"]
    q[0, 0] = 0
    q[0, 1] *= 1e-30
    q[0, 2] *= 1e-39                      # subnormal
    q[0, 3, :, :64] *= 1e-6
    _check(p, *_attend(p))


@gpu
def test_attention_without_lse_on_another_stream_and_again():
    p = _problem(2, 8, 2, 128, 20, [500, 64], seed=4)
    out, _ = _attend(p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again, none = _attend(p, want_lse=False)
    assert torch.equal(out, again) and none is None


@gpu
def test_attention_at_an_offset_beyond_32_bits():
    """Two sequences whose code slabs are 4.3 GB each: the second's first block lies behind 32-bit offsets."""
    B, Hkv, Dh, nblk = 2, 8, 128, 131073
    shape = _shape(B, 8, Hkv, Dh, 1, nblk * 64, most=200)
    cache = ygg.Block4Cache(*(torch.empty((B, Hkv, nblk, 32 * Dh), dtype=torch.uint8, device=DEV) for _ in range(2)),
                            *(torch.empty((B, Hkv, nblk, 2 * Dh), dtype=torch.uint8, device=DEV) for _ in range(2)),
                            *(torch.zeros((B, 128, Hkv, Dh), dtype=torch.bfloat16, device=DEV) for _ in range(2)))
    g = np.random.default_rng(0)
    k, v = (_bf16(g.standard_normal((1, B, 200, Hkv, Dh))).to(DEV) for _ in range(2))
    n = torch.tensor([130, 200], dtype=torch.int32, device=DEV)
    ygg.block4_append(shape, 1, k, v, cache, n, n)
    small = _shape(B, 8, Hkv, Dh, 1, 300, most=200)
    near = ygg.new_block4_cache(small, 1, device=DEV)
    ygg.block4_append(small, 1, k, v, near, n, n)
    got = []
    for s, c in ((shape, cache), (small, near.layer(0))):
        out = torch.empty((B, 1, 8, Dh), dtype=torch.bfloat16, device=DEV)
        ygg.tree_attention_block4(s, k[0, :, :1].contiguous(), c, n, k[0, :, 1:2].contiguous(), v[0, :, 1:2].contiguous(),
                                  torch.full((B, 1), -1, dtype=torch.int32, device=DEV), out, None, workspace(s, ygg.OP_ATTENTION_BLOCK4))
        got.append(out)
    assert torch.equal(*got) and not torch.isnan(got[0]).any()


# ---------------------------------------------------------------- scores far from zero

@gpu
@pytest.mark.parametrize("B,Hq,Hkv,Dh,N,lens", [
    (1, 8, 2, 128, 161, [700]), (1, 8, 4, 64, 321, [1000]), (4, 16, 4, 128, 17, [640, 64, 0, 201]), (16, 32, 8, 64, 1, [64 + 70 * b for b in range(16)]),
    (3, 8, 2, 128, 33, [64, 128, 65]), (8, 32, 8, 128, 3, [4096] + [64 * b for b in range(1, 8)]),
])
def test_scores_far_below_zero(B, Hq, Hkv, Dh, N, lens):
    """Every key is about 2 in magnitude with the same signs, every row of q the opposite of them: row r's largest score lies near
    -(60 .. 700), evenly over the rows, in base 2."""
    p = _problem(B, Hq, Hkv, Dh, N, lens, seed=N)
    g = np.random.default_rng(N)
    sign = np.where(g.random(Dh) < 0.5, -1.0, 1.0)
    code_at, _ = plain.stored_at("k", Dh)
    c = p["cache"]
    for b, L in enumerate(lens):
        full = int(L) // 64
        nibble = g.integers(3, 6, (Hkv, full, 64, Dh)) | np.where(sign < 0, 8, 0)                # 1.5, 2, 3
        stored = np.empty((Hkv, full, 64 * Dh), np.uint8)
        stored[..., code_at] = nibble
        c.k_codes[b, :, :full] = torch.from_numpy(stored[..., ::2] | stored[..., 1::2] << 4).to(DEV)
        c.k_scale[b, :, :full] = 127
        rows = lambda *s: _bf16(sign * (2 + 0.25 * g.standard_normal(s))).to(DEV)
        at, open_rows = full % 2 * 64, int(L) - full * 64
        c.k_tail[b, at:at + open_rows] = rows(open_rows, Hkv, Dh)
        p["dense"]["k_tree"][b] = rows(N, Hkv, Dh)
    level = np.linspace(60, 700, B * N * Hq).reshape(B, N, Hq, 1) * np.log(2) / (2 * Dh)
    p["q"].copy_(_bf16(-level * sign * (1 + 0.05 * g.standard_normal((B, N, Hq, Dh)))))
    p["shape"].softmax_scale = 1.0
    _read_back(p)
    out, lse = _attend(p)
    assert not torch.isnan(out).any() and not torch.isnan(lse).any()
    _check(p, out, lse)


@gpu
@pytest.mark.parametrize("Dh", [64, 128])
@pytest.mark.parametrize("score", [-2.0 ** 21, -2.0 ** 22, 2.0 ** 22])
@pytest.mark.parametrize("Hq,Hkv,N,lens", [(4, 1, 65, [0]), (2, 2, 65, [130]), (4, 4, 33, [1000, 5]), (8, 1, 200, [64, 0, 300]), (2, 1, 40, [4000])])
def test_equal_scores_of_any_magnitude(Dh, score, Hq, Hkv, N, lens):
    """All scores are the same power of two, exactly: every row is the mean of the values that it sees."""
    p = _problem(len(lens), Hq, Hkv, Dh, N, lens, seed=N)
    p["q"].zero_()
    p["q"][..., 0] = score / 1024
    c = p["cache"]
    code_at, scale_at = plain.stored_at("k", Dh)
    nibble = np.zeros(64 * Dh, np.uint8)
    nibble[code_at[:, 0]] = 6                                               # 4, times a scale of 256
    byte = np.full(2 * Dh, 127, np.uint8)
    byte[scale_at[:, 0]] = 135
    row = torch.zeros(Dh, dtype=torch.bfloat16, device=DEV)
    row[0] = 1024
    for b, L in enumerate(lens):
        full = L // 64
        c.k_codes[b, :, :full] = torch.from_numpy(nibble[::2] | nibble[1::2] << 4).to(DEV)
        c.k_scale[b, :, :full] = torch.from_numpy(byte).to(DEV)
        c.k_tail[b, full % 2 * 64:full % 2 * 64 + L % 64] = row
        p["dense"]["k_tree"][b] = row
    p["shape"].softmax_scale = 1.0
    _read_back(p)
    out, lse = (to_f64(x) for x in _attend(p))
    G = Hq // Hkv
    for b, L in enumerate(lens):
        for h in range(Hkv):
            ref, ref_lse, size = plain_ops.tree_attention(np.zeros((N, G, Dh)), p["dense"]["k"][b][h], p["dense"]["v"][b][h], L, p["parent"][b], 1.0)
            hs = slice(h * G, (h + 1) * G)
            # in base 2 a score is this power of two times log2 e in fp32, so exact, and equal over blocks and own keys.  Weights are off by
            # 2^-8, their products with V are cut by 2^-8 of the sum of magnitudes, partial rows 2^-12 of the largest, the result 2^-8
            tol = size * (2.0 ** -7 + 2.0 ** -12) + size.max(-1, keepdims=True) * 2.0 ** -12 + np.abs(ref) * 2.0 ** -8
            assert (np.abs(out[b, :, hs] - ref) <= tol).all(), (b, h)
            # m * ln 2 in fp32, from log2 e in fp32: 2^-24 of the score each, a few of them
            assert (np.abs(lse[b, :, hs] - (score + ref_lse)) <= abs(score) * 2.0 ** -22).all(), (b, h)


@gpu
@pytest.mark.parametrize("Dh", [64, 128])
@pytest.mark.parametrize("q_power,v_power", [(57, 56), (-57, 56), (57, -57)])
def test_magnitudes_at_the_ends_of_the_stated_range(Dh, q_power, v_power):
    """q near 2^60 with keys near 2^-57 and the other way round, values near 2^60 and 2^-57: the scores stay ordinary."""
    p = _problem(2, 8, 2, Dh, 37, [700, 90], seed=Dh)
    c, d = p["cache"], p["dense"]
    for t, power in ((p["q"], q_power), (c.k_tail, -q_power), (d["k_tree"], -q_power), (c.v_tail, v_power), (d["v_tree"], v_power)):
        t.copy_((t.double() * 2.0 ** power).to(t.dtype))
    for t, power in ((c.k_scale, -q_power), (c.v_scale, v_power)):
        t.copy_(torch.where(t == NAN_SCALE, t.int(), t.int() + power).to(torch.uint8))
    _read_back(p)
    _check(p, *_attend(p))


# ---------------------------------------------------------------- refusals

@gpu
def test_refusals_on_the_gpu_binding():
    p = _problem(2, 4, 2, 64, 3, [70, 10], seed=1)
    s, c, i32 = p["shape"], p["cache"], dict(dtype=torch.int32, device=DEV)
    good = dict(q=p["q"], cache=c, seq_lens=torch.tensor([70, 10], **i32), k_tree=p["dense"]["k_tree"], v_tree=p["dense"]["v_tree"],
                parent_idx=to_dev(p["parent"]), out=torch.empty_like(p["q"]), lse=torch.empty((2, 3, 4), device=DEV), workspace=workspace(s, ygg.OP_ATTENTION_BLOCK4))
    ygg.tree_attention_block4(s, **good)
    with pytest.raises(RuntimeError, match="workspace"):
        ygg.tree_attention_block4(s, **{**good, "workspace": None})
    with pytest.raises(TypeError, match="q:"):
        ygg.tree_attention_block4(s, **{**good, "q": p["q"].float()})
    for dtype in (ygg.BF16, ygg.FP8_BLOCK):
        with pytest.raises(RuntimeError, match="unsupported"):
            ygg.tree_attention_block4(ygg.Shape(**{**s.__dict__, "kv_dtype": dtype}), **good)
    for name in ("q", "seq_lens", "k_tree", "v_tree", "parent_idx", "out", "lse"):
        with pytest.raises(ValueError, match=name):
            ygg.tree_attention_block4(s, **{**good, name: good[name][:1]})
    for name in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail"):
        bad = ygg.Block4Cache(*c.tensors())
        setattr(bad, name, getattr(c, name)[:1])
        with pytest.raises(ValueError, match=name):
            ygg.tree_attention_block4(s, **{**good, "cache": bad})
    with pytest.raises(TypeError, match="k_scale"):
        bad = ygg.Block4Cache(*c.tensors())
        bad.k_scale = c.k_scale.float()
        ygg.tree_attention_block4(s, **{**good, "cache": bad})
    # an 8-bit cache is no 4-bit one, nor the other way round
    eight = ygg.Shape(**{**s.__dict__, "kv_dtype": ygg.FP8_BLOCK})
    with pytest.raises((TypeError, ValueError)):
        ygg.tree_attention_block4(s, **{**good, "cache": ygg.new_block_cache(eight, 1, device=DEV).layer(0)})
    with pytest.raises((TypeError, ValueError)):
        ygg.tree_attention_block8(eight, **{**good, "workspace": workspace(eight, ygg.OP_ATTENTION_BLOCK8)})
    wider = ygg.Shape(**{**s.__dict__, "kv_capacity": s.kv_capacity + 128})
    k = torch.zeros((1, 2, 5, 2, 64), dtype=torch.bfloat16, device=DEV)
    n = torch.tensor([1, 1], **i32)
    for cache in (ygg.new_block4_cache(s, 2, device=DEV), ygg.new_block4_cache(wider, 1, device=DEV)):
        with pytest.raises(ValueError, match="k_codes"):
            ygg.tree_attention_block4(s, **{**good, "cache": cache})
    one = ygg.Block4Cache(*(t[None] for t in c.tensors()))
    for kw in (dict(v_new=k[:, :1]), dict(n_new=n[:1]), dict(seq_lens=n[:1]), dict(rows=torch.zeros((1, 3), **i32)), dict(n_layers=2)):
        with pytest.raises(ValueError, match=next(iter(kw)) if "n_layers" not in kw else "k_new"):
            ygg.block4_append(s, **{**dict(n_layers=1, k_new=k, v_new=k, cache=one, seq_lens=n, n_new=n), **kw})
    ygg.block4_append(s, 1, k, k, ygg.new_block4_cache(s, 2, device=DEV), n, n)                          # (further layers that the call leaves out)
