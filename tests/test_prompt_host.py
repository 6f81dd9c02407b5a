"""Host-side checks, without a GPU, of the operators of a prompt's way into the 4-bit cache: refusals, sizes, plans, the storage order."""
import os
import re

import numpy as np
import pytest
import torch

import paper_2512_23858_amd as ygg
import plain_prompt as plain
from test_serving_host import BIG, FAKE, NULL, OK, ROOT, SHAPE, UNSUPPORTED, WORKSPACE, _cache, _Cache, _call, _replaced
from test_serving_host import _shape as _block8_shape


def _shape(**kw):
    return _block8_shape(**{"kv_dtype": ygg.FP4_BLOCK, **kw})


def test_block4_attention_refuses():
    call = lambda shape, args: _call("ygg_tree_attention_block4", shape, args)
    good = [FAKE, _cache(), FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, BIG]
    assert call(None, good) == NULL
    for i in (0, 1, 2, 3, 4, 5, 6):
        assert call(_shape(), _replaced(good, i, None)) == NULL
    for x, _ in _Cache._fields_:
        assert call(_shape(), _replaced(good, 1, _cache(**{x: None}))) == NULL
        assert call(_shape(), _replaced(good, 1, _cache(**{x: FAKE + 8}))) == UNSUPPORTED      # (scales too are read 16 bytes at a time)
    for i in (0, 3, 4, 6):
        assert call(_shape(), _replaced(good, i, FAKE + 8)) == UNSUPPORTED
    for kw, rc in ((dict(kv_dtype=ygg.BF16), UNSUPPORTED), (dict(kv_dtype=ygg.FP8_BLOCK), UNSUPPORTED), (dict(kv_dtype=4), UNSUPPORTED),
                   (dict(head_dim=96), UNSUPPORTED), (dict(n_nodes=1025), UNSUPPORTED), (dict(n_q_heads=7), SHAPE), (dict(batch=0), SHAPE),
                   (dict(kv_capacity=131), SHAPE), (dict(softmax_scale=0.0), SHAPE), (dict(softmax_scale=float("nan")), SHAPE)):
        assert call(_shape(**kw), good) == rc, kw
    need = ygg.workspace_bytes(_shape(), ygg.OP_ATTENTION_BLOCK4)
    assert need > 0 and need % 256 == 0
    assert call(_shape(), _replaced(good, 8, None)) == WORKSPACE
    assert call(_shape(), _replaced(good, 8, FAKE + 16)) == WORKSPACE
    assert call(_shape(), _replaced(good, 9, need - 1)) == WORKSPACE
    big = dict(batch=65535, n_q_heads=512, n_kv_heads=512, max_seq_len=0, kv_capacity=4)       # a workgroup to each sequence and head
    assert call(_shape(**big), good) == UNSUPPORTED


def test_the_calls_of_other_caches_refuse_the_type():
    s = _shape()
    assert ygg.workspace_bytes(s, ygg.OP_ATTENTION) == ygg.workspace_bytes(s, ygg.OP_ATTENTION_BLOCK8) == 0
    assert ygg.workspace_bytes(_block8_shape(), ygg.OP_ATTENTION_BLOCK4) == 0
    assert _call("ygg_tree_attention", s, [FAKE] * 8 + [None, FAKE, BIG]) == UNSUPPORTED
    assert _call("ygg_tree_attention_fp8kv", s, [FAKE] * 10 + [None, FAKE, BIG]) == UNSUPPORTED
    assert _call("ygg_tree_attention_block8", s, [FAKE, _cache(), FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, BIG]) == UNSUPPORTED
    assert _call("ygg_block8_append", s, [2, FAKE, FAKE, 13, FAKE, 4, FAKE, FAKE, _cache()]) == UNSUPPORTED
    assert _call("ygg_accept_and_compact", s, [1, FAKE, None, *[FAKE] * 10, FAKE, BIG]) == UNSUPPORTED


def test_block4_append_refuses():
    call = lambda shape, args: _call("ygg_block4_append", shape, args)
    good = [2, FAKE, FAKE, 13, FAKE, 4, FAKE, FAKE, _cache()]     # layers, k, v, n_rows, rows, max_new, n_new, lens, cache
    for i in (1, 2, 6, 7, 8):
        assert call(_shape(), _replaced(good, i, None)) == NULL
    for i, value in ((0, 0), (0, 65536), (3, 0), (5, 0), (5, -1)):
        assert call(_shape(), _replaced(good, i, value)) == SHAPE
    assert call(_shape(), [2, FAKE, FAKE, 13, None, 14, FAKE, FAKE, _cache()]) == SHAPE      # more tokens than rows
    for i in (1, 2):
        assert call(_shape(), _replaced(good, i, FAKE + 2)) == UNSUPPORTED
    for x, _ in _Cache._fields_:
        assert call(_shape(), _replaced(good, 8, _cache(**{x: FAKE + 4}))) == UNSUPPORTED
    assert call(_shape(kv_dtype=ygg.FP8_BLOCK), good) == UNSUPPORTED
    assert call(_shape(batch=65535), _replaced(_replaced(good, 0, 65535), 5, 1 << 30)) == UNSUPPORTED      # the launch grid


def test_norm_rotary_refuses():
    call = lambda shape, args: _call("ygg_tree_norm_rotary", shape, args)
    # q, stride, k, stride, q_out, k_out, q_weight, k_weight, per_head, eps, frequencies, rotary_dim, interleaved, scale, lens, parent, positions
    good = [FAKE, 0, FAKE, 0, FAKE, FAKE, FAKE, FAKE, 0, 1e-6, FAKE, 128, 0, 1.0, FAKE, FAKE, None]
    assert call(None, good) == NULL
    for i in (4, 5, 6, 7, 10, 14, 15):
        assert call(_shape(), _replaced(good, i, None)) == NULL
    for i in (6, 7):
        assert call(_shape(), _replaced(good, i, FAKE + 4)) == UNSUPPORTED
    for eps in (-1e-6, float("nan"), float("inf")):
        assert call(_shape(), _replaced(good, 9, eps)) == SHAPE
    for dim, rc in ((0, SHAPE), (8, SHAPE), (24, UNSUPPORTED), (130, SHAPE), (144, SHAPE)):
        assert call(_shape(), _replaced(good, 11, dim)) == rc, dim
    assert call(_shape(), _replaced(good, 13, float("inf"))) == SHAPE
    assert call(_shape(), _replaced(good, 1, 2048)) == SHAPE                                 # in place, but not dense
    assert call(_shape(), _replaced(good, 1, 1023)) == SHAPE                                 # tokens would overlap
    assert call(_shape(n_nodes=1025), good) == UNSUPPORTED                                   # as a tree; positions may be more
    assert call(_shape(kv_dtype=4), good) == UNSUPPORTED
    assert call(_shape(n_nodes=(1 << 25) + 1), _replaced(good, 16, FAKE)) == UNSUPPORTED     # the launch grid
    # one tensor alone needs its own weights only
    assert call(_shape(), [None, 0, FAKE, 0, None, FAKE, None, None, *good[8:]]) == NULL


def _prompt(**kw):
    return _shape(**{"kv_dtype": ygg.BF16, "n_nodes": 300, "kv_capacity": 500, "max_seq_len": 400, **kw})


def test_prompt_attention_refuses():
    call = lambda shape, args: _call("ygg_prompt_attention", shape, args)
    # q, stride, k, stride, v, stride, q_first, q_len, k_first, k_len, out, lse, workspace, bytes
    good = [FAKE, 0, FAKE, 0, FAKE, 0, FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, BIG]
    assert call(None, good) == NULL
    for i in (0, 2, 4, 6, 7, 8, 9, 10):
        assert call(_prompt(), _replaced(good, i, None)) == NULL
    for i in (0, 2, 4, 10):
        assert call(_prompt(), _replaced(good, i, FAKE + 8)) == UNSUPPORTED
    for i, dense in ((1, 1024), (3, 256), (5, 256)):
        assert call(_prompt(), _replaced(good, i, dense - 1)) == SHAPE
        assert call(_prompt(), _replaced(good, i, dense + 4)) == UNSUPPORTED                 # rows off 16 bytes
        assert call(_prompt(), _replaced(good, i, -dense)) == SHAPE
    for i in (3, 5):
        assert call(_prompt(), _replaced(good, i, (1 << 24) + 8)) == UNSUPPORTED
    for kw, rc in ((dict(kv_dtype=ygg.FP8_E4M3), UNSUPPORTED), (dict(kv_dtype=ygg.FP4_BLOCK), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED),
                   (dict(n_q_heads=7), SHAPE), (dict(batch=0), SHAPE), (dict(batch=65536), SHAPE), (dict(n_nodes=0), SHAPE), (dict(kv_capacity=0, max_seq_len=0), SHAPE),
                   (dict(max_seq_len=501), SHAPE), (dict(max_seq_len=-1), SHAPE), (dict(softmax_scale=0.0), SHAPE), (dict(softmax_scale=float("inf")), SHAPE),
                   (dict(n_nodes=(1 << 25) + 1), UNSUPPORTED), (dict(kv_capacity=1 << 31), UNSUPPORTED), (dict(n_q_heads=512, n_kv_heads=512, n_nodes=1 << 24), UNSUPPORTED)):
        assert call(_prompt(**kw), good) == rc, kw
        assert ygg.workspace_bytes(_prompt(**kw), ygg.OP_PROMPT_ATTENTION) == 0
    few = _prompt(n_nodes=16, batch=1, kv_capacity=40000, max_seq_len=40000)                 # few rows, many keys: the keys are split
    need = ygg.workspace_bytes(few, ygg.OP_PROMPT_ATTENTION)
    assert need > 0 and need % 256 == 0 and ygg.prompt_plan(few)["splits"] > 1
    assert call(few, _replaced(good, 12, None)) == WORKSPACE
    assert call(few, _replaced(good, 12, FAKE + 16)) == WORKSPACE
    assert call(few, _replaced(good, 13, need - 1)) == WORKSPACE
    with pytest.raises(RuntimeError, match="inconsistent"):
        ygg.prompt_plan(_prompt(batch=0))


def test_scratch_of_the_longest_prefix_serves_the_shorter_ones():
    for B in (1, 3, 16, 64):
        for heads in ((32, 32), (32, 8), (12, 12), (64, 8)):
            for N in (1, 17, 49, 321):
                for op, kw in ((ygg.OP_ATTENTION_BLOCK4, {}), (ygg.OP_PROMPT_ATTENTION, dict(kv_dtype=ygg.BF16, kv_capacity=32768))):
                    sizes = [ygg.workspace_bytes(_shape(**{**dict(batch=B, n_q_heads=heads[0], n_kv_heads=heads[1], n_nodes=N, max_seq_len=L, kv_capacity=L + 4), **kw}), op)
                             for L in (0, 64, 100, 640, 4096, 32768)]
                    assert sizes == sorted(sizes) and (op == ygg.OP_PROMPT_ATTENTION or sizes[0] > 0)


def test_prompt_plan_has_a_tile_for_every_row():
    """Row tiles are counted for the worst that sequences which share no rows can be: one row beyond a tile each."""
    for heads in ((8, 8), (64, 8), (12, 12), (5, 1)):
        for B in (1, 2, 7, 300):
            for n in (1, 2, 300, 4096, 20000):
                p = ygg.prompt_plan(_prompt(batch=B, n_q_heads=heads[0], n_kv_heads=heads[1], n_nodes=n, kv_capacity=30000, max_seq_len=30000))
                G, rows = heads[0] // heads[1], p["rows"]
                g = np.random.default_rng(n + B)
                for cuts in ([], g.integers(0, n + 1, B - 1), np.minimum(np.arange(1, B) * (rows // G + 1), n), np.minimum(np.arange(1, B), n)):
                    lens = np.diff(np.sort(np.concatenate(([0], cuts, [n]))).astype(np.int64))[:B]
                    assert (-(-lens * G // rows)).sum() <= p["tiles"], (heads, B, n)


def test_prompts_up_to_the_stated_size_are_accepted_and_larger_ones_refused():
    """The launch grid: row tiles of all kv heads, in as many parts as their keys have, up to 2^22."""
    g = np.random.default_rng(0)
    for _ in range(3000):
        kv = int(np.exp2(g.uniform(0, 7)))
        hq, B = kv * int(g.integers(1, 9)), int(min(np.exp2(g.uniform(0, 16)), 65535, (1 << 28) // (128 * kv)))
        most = ((1 << 29) - 128 * B * kv) // hq
        n = min(most, 1 << 25, int(np.exp2(g.uniform(0, 25)))) if g.random() < 0.7 else min(most, 1 << 25)
        L = int(np.exp2(g.uniform(0, 30)))
        s = _prompt(batch=B, n_q_heads=hq, n_kv_heads=kv, n_nodes=n, kv_capacity=L, max_seq_len=L, head_dim=int(g.choice([64, 128])),
                    kv_dtype=int(g.choice([ygg.BF16, ygg.F32])))
        p = ygg.prompt_plan(s)
        assert p["tiles"] * kv * p["splits"] <= 1 << 22, (s, p)
    good = [FAKE, 0, FAKE, 0, FAKE, 0, FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, BIG]
    for kw in (dict(n_nodes=1 << 25, n_q_heads=32, n_kv_heads=32), dict(batch=65535, n_q_heads=512, n_kv_heads=512, n_nodes=1 << 20)):
        assert _call("ygg_prompt_attention", _prompt(**kw), good) == UNSUPPORTED, kw


def test_cache_tensors_and_storage_order():
    c = ygg.new_block4_cache(_shape(head_dim=64, kv_capacity=201), 3, device="cpu")
    assert isinstance(c, ygg.Block4Cache) and isinstance(c.layer(0), ygg.Block4Cache)
    assert [tuple(t.shape) for t in c.tensors()] == [(3, 2, 2, 4, 2048)] * 2 + [(3, 2, 2, 4, 128)] * 2 + [(3, 2, 128, 2, 64)] * 2
    with pytest.raises(ValueError):
        ygg.new_block4_cache(_block8_shape(), 1, device="cpu")
    for which in "kv":
        for Dh in (64, 128):       # every code is some token's and dimension's, every scale 32 of them
            code, scale = plain.stored_at(which, Dh)
            assert np.array_equal(np.sort(code.ravel()), np.arange(64 * Dh))
            assert np.array_equal(np.bincount(scale.ravel()), np.full(2 * Dh, 32))
            for s in np.unique(scale):
                t, d = np.nonzero(scale == s)
                assert (len(set(t)) == 1 and set(d) == set(range(min(d), min(d) + 32)) and min(d) % 32 == 0) if which == "k" else (
                    len(set(d)) == 1 and set(t) == set(range(min(t), min(t) + 32)) and min(t) % 32 == 0)


def test_the_definition_of_the_codes_is_the_nearest_value():
    g = np.random.default_rng(0)
    mids = (plain.LEVELS[1:] + plain.LEVELS[:-1]) / 2
    x = g.standard_normal((3, 64, 64)) * np.exp2(g.integers(-8, 8, (3, 64, 1)))
    x[0, :4, :14] = np.concatenate((mids, plain.LEVELS[1:]))
    x[0, :4, 14:32] = 0
    x[0, :4, 14] = 7
    for which in "kv":
        code, scale = plain.encode(x, which)
        got = plain.decode(code, scale, which)
        size = np.exp2(scale[..., plain.stored_at(which, 64)[1]].astype(float) - 127)
        near = np.abs(np.abs(x)[..., None] / size[..., None] - plain.LEVELS).min(-1)
        assert np.allclose(np.abs(got - x) / size, near, rtol=0, atol=1e-12) and (near <= 1).all()
        again, s2 = plain.encode(got, which)
        assert np.array_equal(plain.decode(again, s2, which), got)
    code, scale = plain.encode(x, "k")
    assert scale[0, plain.stored_at("k", 64)[1][0, 0]] == 127                       # 7 is still within a scale of 1, as 6
    assert np.array_equal(plain.decode(code, scale, "k")[0, 0, :15], [0, 1, 1, 2, 2, 4, 4, .5, 1, 1.5, 2, 3, 4, 6, 6])


def test_python_binding_refuses_host_tensors():
    s = _shape()
    c = ygg.new_block4_cache(s, 1, device="cpu")
    i, n = torch.zeros((2, 13), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    q, k = torch.zeros((2, 13, 8, 128), dtype=torch.bfloat16), torch.zeros((2, 13, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q must be a GPU tensor"):
        ygg.tree_attention_block4(s, q, c.layer(0), n, k, k, i, q.clone())
    with pytest.raises(ValueError, match="k_new must be a GPU tensor"):
        ygg.block4_append(s, 1, k[None], k[None], c, n, n)
    with pytest.raises(ValueError, match="q must be a GPU tensor"):
        ygg.tree_norm_rotary(s, q, None, q, None, torch.ones(128), None, ygg.rotary_frequencies(128), positions=i)
    with pytest.raises(ValueError, match="q must be a GPU tensor"):
        ygg.prompt_attention(_prompt(n_nodes=26), q.flatten(0, 1), k.flatten(0, 1), k.flatten(0, 1), n, n, n, n, q.flatten(0, 1).clone())


def test_public_names_of_the_header_are_in_the_package():
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ygg.h")).read(), flags=re.S)
    for name in ("ygg_tree_norm_rotary", "ygg_prompt_attention", "ygg_block4_append", "ygg_tree_attention_block4"):
        assert re.search(rf"\b{name}\s*\(", header) and hasattr(ygg.load_library(), name) and callable(getattr(ygg, name[4:]))
    assert ygg.workspace_bytes(_shape(), ygg.OP_ATTENTION_BLOCK4) > 0 and OK == 0
