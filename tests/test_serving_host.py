"""Host-side checks, without a GPU, of the operators around the verification calls: refusals, sizes, tables, the storage order."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

import paper_2512_23858_amd as ygg
import plain_ops as plain

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = range(5)
FAKE, BIG = 0x100000, 1 << 40      # never dereferenced: every call below fails validation first
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _shape(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, depth=3, width=4, n_nodes=13, vocab=1000, kv_dtype=ygg.FP8_BLOCK,
                softmax_scale=0.09, kv_capacity=200, max_seq_len=128)
    base.update(kw)
    return ygg.Shape(**base)


class _Cache(ctypes.Structure):
    _fields_ = [(x, ctypes.c_void_p) for x in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail")]


class _Rules(ctypes.Structure):
    _fields_ = [(x, ctypes.c_void_p) for x in ("counts", "repetition", "presence", "frequency", "bias")] + [
        ("bias_shared", ctypes.c_int32), ("n_masks", ctypes.c_int32), ("masks", ctypes.c_void_p), ("mask_index", ctypes.c_void_p)]


def _ptr(x):
    return ctypes.cast(ctypes.pointer(x), ctypes.c_void_p) if isinstance(x, ctypes.Structure) else x


def _cache(**kw):
    return _Cache(**{**{x: FAKE for x, _ in _Cache._fields_}, **kw})


def _call(name, shape, args):
    return getattr(ygg.load_library(), name)(ctypes.byref(shape.c()) if shape is not None else None, *(_ptr(a) for a in args), None)


def _replaced(args, i, value):
    return [value if j == i else a for j, a in enumerate(args)]


def test_block_attention_refuses():
    call = lambda shape, args: _call("ygg_tree_attention_block8", shape, args)
    good = [FAKE, _cache(), FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, BIG]
    assert call(None, good) == NULL
    for i in (0, 1, 2, 3, 4, 5, 6):
        assert call(_shape(), _replaced(good, i, None)) == NULL
    for x, _ in _Cache._fields_:
        assert call(_shape(), _replaced(good, 1, _cache(**{x: None}))) == NULL
    for x in ("k_codes", "v_codes", "k_tail", "v_tail"):
        assert call(_shape(), _replaced(good, 1, _cache(**{x: FAKE + 8}))) == UNSUPPORTED
    for i in (0, 3, 4, 6):
        assert call(_shape(), _replaced(good, i, FAKE + 8)) == UNSUPPORTED
    for kw, rc in ((dict(kv_dtype=ygg.BF16), UNSUPPORTED), (dict(kv_dtype=ygg.FP8_E4M3), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED),
                   (dict(n_nodes=1025), UNSUPPORTED), (dict(n_q_heads=7), SHAPE), (dict(batch=0), SHAPE), (dict(kv_capacity=131), SHAPE),
                   (dict(softmax_scale=0.0), SHAPE), (dict(softmax_scale=float("nan")), SHAPE)):
        assert call(_shape(**kw), good) == rc, kw
    need = ygg.workspace_bytes(_shape(), ygg.OP_ATTENTION_BLOCK8)
    assert need > 0 and need % 256 == 0
    assert call(_shape(), _replaced(good, 8, None)) == WORKSPACE
    assert call(_shape(), _replaced(good, 8, FAKE + 16)) == WORKSPACE
    assert call(_shape(), _replaced(good, 9, need - 1)) == WORKSPACE


def test_the_other_calls_refuse_the_block_type():
    """A block cache's shape is no plain K/V shape: no call reads codes it was not given."""
    s = _shape()
    assert ygg.workspace_bytes(s, ygg.OP_ATTENTION) == 0
    assert _call("ygg_tree_attention", s, [FAKE] * 8 + [None, FAKE, BIG]) == UNSUPPORTED
    assert _call("ygg_tree_attention_fp8kv", s, [FAKE] * 10 + [None, FAKE, BIG]) == UNSUPPORTED
    assert ygg.load_library().ygg_accept_and_compact(ctypes.byref(s.c()), 1, FAKE, *[None], *[FAKE] * 10, FAKE, BIG, None) == UNSUPPORTED


def test_append_refuses():
    call = lambda shape, args: _call("ygg_block8_append", shape, args)
    good = [2, FAKE, FAKE, 13, FAKE, 4, FAKE, FAKE, _cache()]     # layers, k, v, n_rows, rows, max_new, n_new, lens, cache
    for i in (1, 2, 6, 7, 8):
        assert call(_shape(), _replaced(good, i, None)) == NULL
    for i, value in ((0, 0), (0, 65536), (3, 0), (5, 0), (5, -1)):
        assert call(_shape(), _replaced(good, i, value)) == SHAPE
    assert call(_shape(), [2, FAKE, FAKE, 13, None, 14, FAKE, FAKE, _cache()]) == SHAPE      # more tokens than rows
    for i in (1, 2):
        assert call(_shape(), _replaced(good, i, FAKE + 2)) == UNSUPPORTED
    assert call(_shape(kv_dtype=ygg.BF16), good) == UNSUPPORTED
    huge = _replaced(_replaced(good, 0, 65535), 5, 1 << 30)
    assert call(_shape(batch=65535), huge) == UNSUPPORTED                                    # the launch grid


def test_rotary_refuses():
    call = lambda shape, args: _call("ygg_tree_rotary", shape, args)
    # q, stride, k, stride, q_out, k_out, frequencies, rotary_dim, interleaved, scale, lens, parent, positions
    good = [FAKE, 0, FAKE, 0, FAKE, FAKE, FAKE, 128, 0, 1.0, FAKE, FAKE, None]
    assert call(None, good) == NULL
    for i in (4, 5, 6, 10, 11):
        assert call(_shape(), _replaced(good, i, None)) == NULL
    assert call(_shape(), _replaced(_replaced(good, 0, None), 2, None)) == NULL
    for dim, rc in ((0, SHAPE), (8, SHAPE), (24, UNSUPPORTED), (130, SHAPE), (144, SHAPE)):
        assert call(_shape(), _replaced(good, 7, dim)) == rc, dim
    assert call(_shape(), _replaced(good, 9, float("inf"))) == SHAPE
    assert call(_shape(), _replaced(good, 1, 1023)) == SHAPE                                 # tokens would overlap
    assert call(_shape(), _replaced(_replaced(good, 4, 2 * FAKE), 1, 1028)) == UNSUPPORTED   # rows off 16 bytes
    assert call(_shape(), _replaced(good, 1, 2048)) == SHAPE                                 # in place, but not dense
    assert call(_shape(), _replaced(good, 0, FAKE + 2)) == UNSUPPORTED
    assert call(_shape(n_nodes=1025), good) == UNSUPPORTED                                   # as a tree; positions may be more
    assert call(_shape(head_dim=256), good) == UNSUPPORTED
    assert call(_shape(kv_dtype=4), good) == UNSUPPORTED
    assert call(_shape(n_kv_heads=3), good) == SHAPE


def test_constrain_and_count_refuse():
    call = lambda shape, args: _call("ygg_constrain_logits", shape, args)
    # logits, dtype, stride, parent, token, rules, out, best, workspace, bytes
    good = [FAKE, ygg.F32, 0, FAKE, FAKE, _Rules(), FAKE, FAKE, FAKE, BIG]
    for i in (0, 3, 4, 5):
        assert call(_shape(), _replaced(good, i, None)) == NULL
    assert call(_shape(), _replaced(_replaced(good, 6, None), 7, None)) == NULL
    for dtype in (ygg.FP8_E4M3, ygg.FP8_BLOCK, -1):
        assert call(_shape(), _replaced(good, 1, dtype)) == UNSUPPORTED
    assert call(_shape(), _replaced(good, 2, 999)) == SHAPE
    assert call(_shape(), _replaced(good, 2, 1024)) == SHAPE                                 # in place, but not dense
    assert call(_shape(), _replaced(good, 1, ygg.BF16)) == SHAPE                             # in place, but not fp32
    assert call(_shape(), _replaced(good, 5, _Rules(masks=FAKE, n_masks=1))) == NULL
    assert call(_shape(), _replaced(good, 5, _Rules(masks=FAKE, mask_index=FAKE))) == SHAPE
    assert call(_shape(vocab=0), good) == SHAPE
    need = ygg.workspace_bytes(_shape(), ygg.OP_CONSTRAIN)
    assert need > 0 and call(_shape(), _replaced(good, 9, need - 1)) == WORKSPACE and call(_shape(), _replaced(good, 8, None)) == WORKSPACE

    count = lambda args: _call("ygg_count_tokens", _shape(), args)
    ok = [FAKE, 13, FAKE, 0, 4, FAKE, 0, FAKE]                                               # tokens, n, rows, first, max_new, n_new, prompt, counts
    for i in (0, 5, 7):
        assert count(_replaced(ok, i, None)) == NULL
    for i, value in ((1, 0), (3, -1), (4, 0)):
        assert count(_replaced(ok, i, value)) == SHAPE


def test_scratch_of_the_longest_prefix_serves_the_shorter_ones():
    for B in (1, 3, 16, 64):
        for heads in ((32, 32), (32, 8), (12, 12), (64, 8)):
            for N in (1, 17, 49, 321):
                sizes = [ygg.workspace_bytes(_shape(batch=B, n_q_heads=heads[0], n_kv_heads=heads[1], n_nodes=N, max_seq_len=L, kv_capacity=L + 4),
                                             ygg.OP_ATTENTION_BLOCK8) for L in (0, 64, 100, 640, 4096, 32768)]
                assert sizes[0] > 0 and sizes == sorted(sizes)


def test_launches_beyond_the_grid_are_refused():
    big = dict(batch=65535, n_q_heads=512, n_kv_heads=512, max_seq_len=0, kv_capacity=4)     # a workgroup to each sequence and head
    assert _call("ygg_tree_attention_block8", _shape(**big), [FAKE, _cache(), FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, BIG]) == UNSUPPORTED
    assert _call("ygg_block8_append", _shape(batch=65535), [64, FAKE, FAKE, 13, FAKE, 65, FAKE, FAKE, _cache()]) == UNSUPPORTED
    assert _call("ygg_tree_rotary", _shape(n_nodes=(1 << 25) + 1), [FAKE, 0, FAKE, 0, FAKE, FAKE, FAKE, 128, 0, 1.0, None, None, FAKE]) == UNSUPPORTED
    assert _call("ygg_constrain_logits", _shape(batch=65535, n_nodes=1000),
                 [FAKE, ygg.F32, 0, FAKE, FAKE, _Rules(), FAKE, FAKE, FAKE, BIG]) == UNSUPPORTED


def test_frequencies():
    f = ygg.rotary_frequencies(128)
    assert f.dtype == torch.float64 and f.shape == (64,) and f[0] == 1 and math.isclose(f[63], 10000 ** (-126 / 128))
    assert torch.allclose(ygg.rotary_frequencies(64, 500000.0, factor=4.0), ygg.rotary_frequencies(64, 500000.0) / 4, rtol=1e-15)
    f, s = ygg.rotary_frequencies(128, 500000.0), ygg.rotary_frequencies(128, 500000.0, factor=8.0, original_len=8192)
    turns = 8192 * f / (2 * math.pi)
    assert torch.equal(s[turns >= 4], f[turns >= 4]) and torch.allclose(s[turns <= 1], f[turns <= 1] / 8, rtol=1e-15)
    between = (turns > 1) & (turns < 4)
    assert between.any() and ((s < f) & (s > f / 8))[between].all()
    for bad in (dict(rotary_dim=0), dict(rotary_dim=15), dict(rotary_dim=64, base=0.0), dict(rotary_dim=64, factor=-1.0),
                dict(rotary_dim=64, original_len=-1), dict(rotary_dim=64, low_turns=4.0)):
        with pytest.raises(ValueError):
            ygg.rotary_frequencies(**bad)


def test_block_cache_tensors_and_storage_order():
    c = ygg.new_block_cache(_shape(head_dim=64, kv_capacity=201), 3, device="cpu")
    assert [tuple(t.shape) for t in c.tensors()] == [(3, 2, 2, 4, 4096)] * 2 + [(3, 2, 2, 4)] * 2 + [(3, 2, 128, 2, 64)] * 2
    assert c.layer(1).k_tail.data_ptr() == c.k_tail[1].data_ptr() and c.layer(1).k_codes.is_contiguous()
    with pytest.raises(ValueError):
        ygg.new_block_cache(_shape(kv_dtype=ygg.BF16), 1, device="cpu")
    for which in "kv":
        for Dh in (64, 128):       # every byte of a block is some token's and dimension's
            assert np.array_equal(np.sort(plain.stored_at(which, Dh).ravel()), np.arange(64 * Dh))
    v = plain.e4m3_values()
    ref = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, ref, equal_nan=True)


def test_python_binding_refuses_host_tensors():
    s = _shape()
    c = ygg.new_block_cache(s, 1, device="cpu")
    i = torch.zeros((2, 13), dtype=torch.int32)
    n = torch.zeros(2, dtype=torch.int32)
    q = torch.zeros((2, 13, 8, 128), dtype=torch.bfloat16)
    k = torch.zeros((2, 13, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q must be a GPU tensor"):
        ygg.tree_attention_block8(s, q, c.layer(0), n, k, k, i, q.clone())
    with pytest.raises(ValueError, match="k_new must be a GPU tensor"):
        ygg.block8_append(s, 1, k[None], k[None], c, n, n)
    with pytest.raises(ValueError, match="q must be a GPU tensor"):
        ygg.tree_rotary(s, q, None, q, None, ygg.rotary_frequencies(128), positions=i)
    with pytest.raises(ValueError, match="tokens must be a GPU tensor"):
        ygg.count_tokens(s, i, n, torch.zeros((2, 1000), dtype=torch.int32))
    with pytest.raises(ValueError, match="logits must be a GPU tensor"):
        ygg.constrain_logits(s, torch.zeros((2, 13, 1000)), i, i, best=i.clone())


def test_public_names_of_the_header_are_in_the_package():
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ygg.h")).read(), flags=re.S)
    for name in ("ygg_tree_attention_block8", "ygg_block8_append", "ygg_tree_rotary", "ygg_count_tokens", "ygg_constrain_logits"):
        assert re.search(rf"\b{name}\s*\(", header) and hasattr(ygg.load_library(), name) and callable(getattr(ygg, name[4:]))


def test_the_definition_of_the_codes_is_the_nearest_value():
    """plain_ops.encode against torch's rounding to E4M3, and back through the storage order."""
    g = np.random.default_rng(0)
    values = plain.e4m3_values()[:127]
    x = np.concatenate((values, (values[1:] + values[:-1]) / 2, g.standard_normal(64 * 128 - 253) * np.exp2(g.integers(-12, 8, 64 * 128 - 253))))
    x = np.clip(np.where(g.random(x.size) < 0.5, x, -x), -448, 448).astype(np.float32).reshape(1, 64, 128)
    for which in "kv":
        code = plain.encode(x, np.ones(1, np.float32), which)[:, plain.stored_at(which, 128)]
        assert np.array_equal(code, torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
