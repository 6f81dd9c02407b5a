"""ygg_constrain_logits and ygg_count_tokens against the definition, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2512_23858_amd as ygg
import plain_ops as plain
import ygg_workloads as wl
from gpu_util import DEV, to_dev, workspace

pytestmark = pytest.mark.gpu


def _shape(B, N, V):
    return ygg.Shape(batch=B, n_q_heads=1, n_kv_heads=1, head_dim=64, depth=0, width=1, n_nodes=N, vocab=V, kv_dtype=ygg.BF16,
                     softmax_scale=1.0, kv_capacity=1, max_seq_len=0)


def _case(B, N, V, seed, dtype, counts=True, bias="full", masks=3):
    g = np.random.default_rng(seed)
    h = dict(parent=np.stack([wl.random_topological_tree(seed, N, sub=b) for b in range(B)]))
    h["token"] = g.integers(0, max(V // 3, 1), (B, N)).astype(np.int32)
    x = torch.from_numpy(g.standard_normal((B, N, V)).astype(np.float32) * 3).to(dtype)
    x[:, :, ::7] = -x[:, :, ::7].abs()
    h["logits"] = x
    c = g.integers(0, 5, (B, V)) * (g.random((B, V)) < 0.3)
    h["counts"] = np.where(g.random((B, V)) < 0.2, c - 2 ** 31, c).astype(np.int32) if counts else None
    for name, lo, hi in (("repetition", 0.8, 1.5), ("presence", -0.3, 0.7), ("frequency", -0.3, 0.7)):
        h[name] = g.uniform(lo, hi, B).astype(np.float32)
    b = g.standard_normal((B, V)).astype(np.float32)
    b[g.random((B, V)) < 0.05] = -np.inf
    h["bias"] = {"full": b, "shared": b[0], None: None}[bias]
    h["masks"] = g.integers(-2 ** 31, 2 ** 31, (masks, (V + 31) // 32)).astype(np.int32) if masks else None
    h["mask_index"] = g.integers(-1, max(masks, 1), (B, N)).astype(np.int32)
    return h


def _ref(h):
    x = h["logits"].float().numpy()
    return np.stack([plain.constrain(x[b], h["parent"][b], h["token"][b], None if h["counts"] is None else h["counts"][b], h["repetition"][b],
                                     h["presence"][b], h["frequency"][b],
                                     None if h["bias"] is None else h["bias"] if h["bias"].ndim == 1 else h["bias"][b],
                                     h["masks"], h["mask_index"][b]) for b in range(x.shape[0])])


def _up(a):
    return None if a is None else to_dev(np.ascontiguousarray(a)) if isinstance(a, np.ndarray) else a.to(DEV)


def _run(h, write=True, best=True, logits=None, out=None):
    B, N, V = h["logits"].shape
    shape = _shape(B, N, V)
    logits = h["logits"].to(DEV) if logits is None else logits
    if write and out is None:
        out = torch.full((B, N, V), float("nan"), device=DEV)
    tokens = torch.full((B, N), -7, dtype=torch.int32, device=DEV) if best else None
    ws = workspace(shape, ygg.OP_CONSTRAIN, poison=0xFF) if best else None
    ygg.constrain_logits(shape, logits, _up(h["parent"]), _up(h["token"]), out=out if write else None, best=tokens, counts=_up(h["counts"]),
                         repetition=_up(h["repetition"]), presence=_up(h["presence"]), frequency=_up(h["frequency"]), bias=_up(h["bias"]),
                         masks=_up(h["masks"]), mask_index=_up(h["mask_index"]), workspace=ws)
    return None if out is None or not write else out.cpu().numpy(), None if tokens is None else tokens.cpu().numpy()


def _same(a, b):
    return np.array_equal(a.view(np.int32), b.view(np.int32)) or (np.array_equal(a, b) and not np.isnan(a).any())


@pytest.mark.parametrize("B,N,V", [(1, 1, 1), (1, 1, 31), (2, 5, 1000), (3, 13, 4096), (1, 49, 4097), (2, 7, 8191), (1, 33, 32003),
                                   (1, 129, 12345), (1, 1024, 77), (70, 2, 515), (1, 2, 128256)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_everything_on(B, N, V, dtype):
    h = _case(B, N, V, seed=B + N + V, dtype=dtype)
    ref = _ref(h)
    out, best = _run(h)
    assert _same(out, ref)
    assert np.array_equal(best, ref.argmax(-1))
    assert np.array_equal(_run(h, write=False)[1], best)
    assert _same(_run(h, best=False)[0], ref)


@pytest.mark.parametrize("counts", [False, True])
@pytest.mark.parametrize("bias", [None, "shared"])
@pytest.mark.parametrize("masks", [0, 1])
def test_parts_left_out(counts, bias, masks):
    h = _case(2, 13, 5003, seed=5, dtype=torch.float32, counts=counts, bias=bias, masks=masks)
    ref = _ref(h)
    out, best = _run(h)
    assert _same(out, ref) and np.array_equal(best, ref.argmax(-1))


def test_no_rules_at_all_is_the_plain_argmax_and_ties_go_to_the_lowest_token():
    B, N, V = 2, 3, 9000
    x = torch.zeros((B, N, V))
    x[0, 1, 4095:4098] = 2.0
    x[1, 2, 8999] = 1.0
    x[1, 0] = -float("inf")                 # nothing left: the lowest token
    x[0, 2] = torch.finfo(torch.float32).min
    h = dict(logits=x, parent=np.array([[-1, 0, 1]] * B, np.int32), token=np.zeros((B, N), np.int32), counts=None, repetition=None,
             presence=None, frequency=None, bias=None, masks=None, mask_index=None)
    out, best = _run(h)
    assert _same(out, x.numpy()) and np.array_equal(best, [[0, 4095, 0], [0, 0, 8999]])


def test_a_mask_that_leaves_nothing_and_one_that_leaves_one_token():
    h = _case(1, 4, 6001, seed=2, dtype=torch.bfloat16, masks=3)
    h["masks"][:] = 0
    h["masks"][1, 5000 // 32] = 1 << (5000 % 32)
    h["mask_index"] = np.array([[0, 1, -1, 99]], np.int32)      # beyond the last mask: the last
    h["bias"][:] = np.where(np.isinf(h["bias"]), 0, h["bias"])
    ref = _ref(h)
    out, best = _run(h)
    assert _same(out, ref) and np.isinf(out[0, 0]).all() and best[0, 0] == 0 and best[0, 1] == 5000 and best[0, 3] == 0


def test_chain_of_one_token_counts_up_along_the_path():
    N, V = 40, 300
    h = _case(1, N, V, seed=9, dtype=torch.float32)
    h["parent"], h["token"] = wl.chain_tree(N)[None], np.full((1, N), 17, np.int32)
    h["token"][0, 3], h["token"][0, 4] = -5, V + 3              # tokens outside the vocabulary are nobody's
    assert _same(_run(h)[0], _ref(h))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_padded_rows_and_in_place(dtype):
    h = _case(3, 5, 4999, seed=4, dtype=dtype)
    ref = _ref(h)
    wide = torch.full((3, 5, 5057), float("inf"), dtype=dtype, device=DEV)
    wide[..., :4999] = h["logits"].to(DEV)
    out, best = _run(h, logits=wide[..., :4999])
    assert _same(out, ref) and np.array_equal(best, ref.argmax(-1)) and torch.isinf(wide[..., 4999:]).all()
    if dtype == torch.float32:
        x = h["logits"].to(DEV)
        assert _same(_run(h, logits=x, out=x)[0], ref)


def test_counts_of_prompt_reply_and_accepted_path():
    g = np.random.default_rng(3)
    B, T, V = 5, 3000, 700
    tokens = g.integers(-3, V + 3, (B, T)).astype(np.int32)
    shape = _shape(B, 4, V)
    counts = torch.zeros((B, V), dtype=torch.int32, device=DEV)
    n_prompt, n_reply = np.array([0, 1, 1500, 1499, 9999], np.int32), np.array([1500, 0, 7, 1500, 64], np.int32)
    rows = np.array([[0, 2, -1, 5], [3, 3, 3, 3], [4000, 1, 1, 0], [9, 8, 7, 6], [1, 1, 2, 2]], np.int32)
    n_rows = np.array([2, 4, 3, 0, -2], np.int32)
    ygg.count_tokens(shape, to_dev(tokens), to_dev(n_prompt), counts, prompt=True)
    ygg.count_tokens(shape, to_dev(tokens), to_dev(n_reply), counts, first=1500)
    ygg.count_tokens(shape, to_dev(tokens), to_dev(n_rows), counts, rows=to_dev(rows))
    ref = np.zeros((B, V), np.int64)
    for b in range(B):
        picked = [tokens[b, r] for r in rows[b, :max(n_rows[b], 0)] if 0 <= r < T]
        for t in [*tokens[b, 1500:1500 + n_reply[b]], *picked]:
            if 0 <= t < V:
                ref[b, t] += 1
        for t in tokens[b, :n_prompt[b]]:
            if 0 <= t < V:
                ref[b, t] -= 2 ** 31 * (ref[b, t] >= 0)
    assert np.array_equal(counts.cpu().numpy(), ref)


def test_refusals_on_the_gpu_binding():
    shape = _shape(1, 2, 100)
    x = torch.zeros((1, 2, 100), device=DEV)
    i = torch.zeros((1, 2), dtype=torch.int32, device=DEV)
    ws = workspace(shape, ygg.OP_CONSTRAIN)
    with pytest.raises(RuntimeError, match="null"):
        ygg.constrain_logits(shape, x, i, i)
    with pytest.raises(RuntimeError, match="workspace"):
        ygg.constrain_logits(shape, x, i, i, best=i.clone())
    with pytest.raises(TypeError, match="logits"):
        ygg.constrain_logits(shape, x.half(), i, i, best=i.clone(), workspace=ws)
    with pytest.raises(RuntimeError, match="null"):
        ygg.constrain_logits(shape, x, i, i, out=x.clone(), masks=torch.zeros((1, 4), dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError, match="rows"):
        ygg.constrain_logits(shape, torch.zeros((1, 100, 2), device=DEV).transpose(1, 2), i, i, out=x.clone())
    wide = torch.zeros((1, 2, 128), device=DEV)
    with pytest.raises(ValueError, match="out"):
        ygg.constrain_logits(shape, wide[..., :100], i, i, out=wide[..., :100])
    with pytest.raises(TypeError, match="counts"):
        ygg.count_tokens(shape, i, torch.ones(1, dtype=torch.int32, device=DEV), x)


def test_tensors_smaller_than_the_shape_are_refused():
    shape = _shape(2, 3, 100)
    i32 = dict(dtype=torch.int32, device=DEV)
    good = dict(logits=torch.zeros((2, 3, 100), device=DEV), parent_idx=torch.full((2, 3), -1, **i32), token_ids=torch.zeros((2, 3), **i32),
                out=torch.zeros((2, 3, 100), device=DEV), best=torch.zeros((2, 3), **i32), counts=torch.zeros((2, 100), **i32),
                repetition=torch.ones(2, device=DEV), presence=torch.ones(2, device=DEV), frequency=torch.ones(2, device=DEV),
                bias=torch.zeros((2, 100), device=DEV), masks=torch.zeros((2, 4), **i32), mask_index=torch.zeros((2, 3), **i32),
                workspace=workspace(shape, ygg.OP_CONSTRAIN))
    ygg.constrain_logits(shape, **good)
    for name in good:
        if name not in ("workspace", "masks"):
            with pytest.raises(ValueError, match=name):
                ygg.constrain_logits(shape, **{**good, name: good[name][:1]})
    with pytest.raises(ValueError, match="masks"):
        ygg.constrain_logits(shape, **{**good, "masks": torch.zeros((2, 3), **i32)})
    t, n = torch.zeros((2, 7), **i32), torch.ones(2, **i32)
    for args, kw, name in (((t[:1], n, good["counts"]), {}, "tokens"), ((t, n[:1], good["counts"]), {}, "n_new"),
                           ((t, n, good["counts"][:1]), {}, "counts"), ((t, n, good["counts"]), dict(rows=t[:1]), "rows")):
        with pytest.raises(ValueError, match=name):
            ygg.count_tokens(shape, *args, **kw)


def test_zeros_of_both_signs_are_equal_and_a_nan_is_the_largest():
    x = torch.full((1, 5, 9000), -1.0)
    x[0, 0, 4000], x[0, 0, 4500], x[0, 0, 8800] = -0.0, 0.0, 0.0
    x[0, 1, 3], x[0, 1, 100], x[0, 1, 8999] = 0.0, -0.0, 0.0
    x[0, 2, 5], x[0, 2, 7000], x[0, 2, 7001], x[0, 2, 8500] = float("inf"), float("nan"), 9.0, -float("nan")
    x[0, 3, 0], x[0, 3, 1], x[0, 3, 8999] = float("nan"), float("nan"), 3.0
    x[0, 4, 600], x[0, 4, 8704], x[0, 4, 8705] = float("nan"), -float("nan"), 0.5
    masks = np.full((1, 282), -1, np.int32)
    masks[0, 600 // 32] &= ~(1 << (600 % 32))
    masks[0, 8704 // 32] &= ~(1 << (8704 % 32))
    h = dict(logits=x, parent=np.array([[-1, 0, 1, 2, 3]], np.int32), token=np.zeros((1, 5), np.int32), counts=None, repetition=None,
             presence=None, frequency=None, bias=None, masks=masks, mask_index=np.array([[-1, -1, -1, -1, 0]], np.int32))
    out, best = _run(h)
    assert np.array_equal(out, _ref({**h, "repetition": np.ones(1, np.float32), "presence": np.zeros(1, np.float32),
                                     "frequency": np.zeros(1, np.float32)}), equal_nan=True)
    assert np.array_equal(best, [[4000, 3, 7000, 0, 8705]])


def test_quotients_at_the_ends_of_the_range_are_the_rounded_ones():
    """The division by the repetition penalty, bit for bit, where the quotient or the remainder leaves the range of normal numbers."""
    V = 4003
    g = np.random.default_rng(8)
    repetition = np.array([1e-40, 1e-3, 0.5, 0.7, 1.3, 3.0, 1e30, 1.7e38, 3.4e38], np.float32)
    B = len(repetition)
    x = np.exp2(g.uniform(-149, 128, (B, 1, V))).astype(np.float32)
    x[:, 0, :5] = [np.inf, 0.0, 1e-45, np.finfo(np.float32).max, np.finfo(np.float32).tiny]
    h = dict(logits=torch.from_numpy(x), parent=np.full((B, 1), -1, np.int32), token=np.full((B, 1), -1, np.int32),
             counts=np.full((B, V), -2 ** 31, np.int32), repetition=repetition, presence=np.zeros(B, np.float32),
             frequency=np.zeros(B, np.float32), bias=None, masks=None, mask_index=np.full((B, 1), -1, np.int32))
    with np.errstate(over="ignore"):
        ref = _ref(h)
    out, best = _run(h)
    assert _same(out, ref) and np.array_equal(best, ref.argmax(-1))


@pytest.mark.parametrize("B,N", [(1, 4), (3, 1), (3, 4)])
def test_expanded_and_overlapping_logits_are_refused(B, N):
    """One row's memory under several rows: a stride of 0 is no dense tensor."""
    V = 4096
    shape, i = _shape(B, N, V), torch.zeros((B, N), dtype=torch.int32, device=DEV)
    best, ws = torch.full_like(i, -7), workspace(shape, ygg.OP_CONSTRAIN)
    row = torch.zeros(B * N * V, device=DEV)
    for x in (row[:V].expand(B, N, V), row.as_strided((B, N, V), (N * (V - 8), V - 8, 1))):
        with pytest.raises(ValueError, match="rows must be dense"):
            ygg.constrain_logits(shape, x, i, i, best=best, workspace=ws)
    assert (best == -7).all()
    ygg.constrain_logits(shape, row.view(B, N, V), i, i, best=best, workspace=ws)
    assert (best == 0).all()


def test_tensors_with_longer_rows_than_the_shape_are_refused():
    """Counts, biases, masks or an output of a padded vocabulary have enough elements, but the second row lies elsewhere."""
    shape = _shape(2, 3, 100)
    i32 = dict(dtype=torch.int32, device=DEV)
    good = dict(logits=torch.zeros((2, 3, 100), device=DEV), parent_idx=torch.full((2, 3), -1, **i32), token_ids=torch.zeros((2, 3), **i32),
                out=torch.zeros((2, 3, 100), device=DEV), best=torch.zeros((2, 3), **i32), counts=torch.zeros((2, 100), **i32),
                bias=torch.zeros((2, 100), device=DEV), masks=torch.full((2, 4), -1, **i32), mask_index=torch.zeros((2, 3), **i32),
                workspace=workspace(shape, ygg.OP_CONSTRAIN))
    ygg.constrain_logits(shape, **good)
    for name in ("parent_idx", "token_ids", "out", "best", "counts", "bias", "masks", "mask_index"):
        t = good[name]
        with pytest.raises(ValueError, match=name):
            ygg.constrain_logits(shape, **{**good, name: torch.cat((t, t), -1)})
        if name != "masks":                                        # further sequences may follow, and further masks
            ygg.constrain_logits(shape, **{**good, name: torch.cat((t, t), 0)})
    t, n = torch.zeros((2, 7), **i32), torch.ones(2, **i32)
    wide = torch.zeros((2, 128), **i32)
    with pytest.raises(ValueError, match="counts"):
        ygg.count_tokens(shape, t, n, wide)
    assert not wide.any()
    # a single sequence may be the first part of a longer one
    one = _shape(1, 3, 100)
    ygg.constrain_logits(one, good["logits"][:1], torch.full((1, 9), -1, **i32), torch.zeros((1, 9), **i32), best=good["best"], counts=wide[:1],
                         workspace=good["workspace"])
