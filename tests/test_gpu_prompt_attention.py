"""ygg_prompt_attention against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2512_23858_amd as ygg
import plain_prompt as plain
from gpu_util import DEV, to_dev, to_f64

pytestmark = pytest.mark.gpu


def _shape(B, Hq, Hkv, Dh, q_rows, k_rows, most, dtype=ygg.BF16, scale=None):
    return ygg.Shape(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=Dh, depth=0, width=1, n_nodes=q_rows, vocab=1, kv_dtype=dtype,
                     softmax_scale=scale or Dh ** -0.5, kv_capacity=k_rows, max_seq_len=most)


def _problem(heads, Dh, q_lens, k_lens=None, dtype=ygg.BF16, seed=0, gap=0, k_gap=None, fused=False, most=None, gain=1.0, scale=None):
    """Sequences with `gap` (of keys k_gap) rows of NaN in front of each and behind the last (k_lens None: keys are the queries' own tokens)."""
    g = np.random.default_rng(seed)
    Hq, Hkv = heads
    dt = torch.float32 if dtype == ygg.F32 else torch.bfloat16
    own = k_lens is None
    q_lens, k_lens = np.asarray(q_lens), np.asarray(q_lens if own else k_lens)
    k_gap = gap if k_gap is None else k_gap
    first = lambda lens, gap: np.cumsum(lens + gap) - lens
    rows = lambda lens, gap: max(int(lens.sum()) + gap * (len(lens) + 1), 1)
    q_first, k_first, q_rows, k_rows = first(q_lens, gap), first(k_lens, k_gap), rows(q_lens, gap), rows(k_lens, k_gap)
    used = lambda lens, firsts, n: np.isin(np.arange(n), np.concatenate([np.arange(f, f + l) for f, l in zip(firsts, lens)] + [[]]))
    hole = lambda x, mask: torch.where(torch.from_numpy(mask)[:, None, None], x, float("nan"))
    q, k, v = (torch.from_numpy(g.standard_normal((n, h, Dh)) * a).to(dt) for n, h, a in ((q_rows, Hq, gain), (k_rows, Hkv, 1.0), (k_rows, Hkv, 1.0)))
    qm, km = used(q_lens, q_first, q_rows), used(k_lens, k_first, k_rows)
    q, k, v = hole(q, qm), hole(k, km), hole(v, km)
    if fused and own:
        qkv = torch.cat((q, k, v), 1).to(DEV)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    else:
        q, k, v = q.to(DEV), k.to(DEV), v.to(DEV)
    most = max(int(k_lens.max()), 0) if most is None else most
    return dict(shape=_shape(len(q_lens), Hq, Hkv, Dh, q_rows, max(k_rows, most), most, dtype, scale) if most <= k_rows else None, q=q, k=k, v=v, q_first=q_first, q_lens=q_lens,
                k_first=k_first, k_lens=k_lens, used=qm)


def _attend(p, want_lse=True):
    s = p["shape"]
    out = torch.full((s.n_nodes, s.n_q_heads, s.head_dim), 77.0, dtype=p["q"].dtype, device=DEV)
    lse = torch.full((s.n_nodes, s.n_q_heads), 77.0, device=DEV) if want_lse else None
    n = ygg.workspace_bytes(s, ygg.OP_PROMPT_ATTENTION)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) if n else None
    i32 = lambda x: to_dev(np.asarray(x, np.int32))
    ygg.prompt_attention(s, p["q"], p["k"], p["v"], i32(p["q_first"]), i32(p["q_lens"]), i32(p["k_first"]), i32(p["k_lens"]), out, lse, ws)
    torch.cuda.synchronize()
    return out, lse


def _check(p, out, lse, sequences=None, rms=True):
    s = p["shape"]
    Dh, f32 = s.head_dim, s.kv_dtype == ygg.F32
    split = ygg.prompt_plan(s)["splits"] > 1
    out, lse = to_f64(out), to_f64(lse)
    assert (out[~p["used"]] == 77).all() and (lse[~p["used"]] == 77).all()        # rows of no sequence stay as they were
    for b in sequences if sequences is not None else range(s.batch):
        rows, keys = (slice(f, f + n) for f, n in ((p["q_first"][b], p["q_lens"][b]), (p["k_first"][b], p["k_lens"][b])))
        q, k, v = to_f64(p["q"][rows]), to_f64(p["k"][keys]), to_f64(p["v"][keys])
        ref, ref_lse, size = plain.prompt_attention(q, k, v, s.softmax_scale)
        empty = np.isneginf(ref_lse)
        assert (out[rows][empty] == 0).all() and np.isneginf(lse[rows][empty]).all()
        if not len(k) or empty.all():
            continue
        n = len(k)
        # Scores: the sum of Dh products in fp32, at most Dh rounded additions (fp32) or, sixteen products to an instruction, Dh / 16 + 4 (bf16)
        # of 2^-23 of the terms' magnitudes.  In base 2 they are rounded once more, 2^-23 of the largest; the exponential is good to 2^-22.
        terms = s.softmax_scale * np.abs(q).sum(-1).max() * np.abs(k).max()
        top = np.abs(ref_lse[~empty]).max() + terms
        score = terms * (Dh if f32 else Dh / 16 + 4) * 2.0 ** -23 + top * 2.0 ** -22 + 2.0 ** -22
        # Weights: that on both sides of the quotient; in bf16 half a step, 2^-8.  Sums over the keys in fp32, n / 2 additions of 2^-24 each
        # (the weights') and n / 2 or n / 16 + 4 of 2^-23 (the values').  A partial row in fp16: 2^-12 of its largest, twice that for what of it is
        # left in the sum.  The result: half a step, 2^-8 or 2^-24, and a division.
        row = np.maximum(size.max(-1, keepdims=True), np.abs(ref).max(-1, keepdims=True))
        tol = size * ((0 if f32 else 2.0 ** -8) + 2 * score + n * 2.0 ** -23) + (2.0 ** -11 * row if split else 0) + np.abs(ref) * (2.0 ** -22 if f32 else 2.0 ** -8 + 2.0 ** -20)
        err = np.abs(out[rows] - ref)
        assert (err <= tol).all(), (b, float((err / np.maximum(tol, 1e-30)).max()))
        if rms:    # a lost key or a wrong mask bit shows here
            assert np.sqrt((err ** 2).mean()) <= (2e-5 if f32 else 0.006) * np.sqrt((ref ** 2).mean()), b
        off = np.abs(lse[rows][~empty] - ref_lse[~empty])
        assert (off <= score + n * 2.0 ** -24 + 2.0 ** -22 * (1 + top)).all(), (b, off.max())


EDGES = [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 320, 511]


@pytest.mark.parametrize("dtype", [ygg.BF16, ygg.F32])
@pytest.mark.parametrize("Dh", [64, 128])
@pytest.mark.parametrize("heads", [(1, 1), (4, 2), (3, 1), (8, 1), (16, 1)])
def test_lengths_around_the_tiles_edges(dtype, Dh, heads):
    """All in one batch, and each alone."""
    p = _problem(heads, Dh, EDGES, dtype=dtype, seed=Dh + heads[0], gap=1)
    _check(p, *_attend(p))
    for n in EDGES[::3]:
        p = _problem(heads, Dh, [n], dtype=dtype, seed=n)
        _check(p, *_attend(p))


@pytest.mark.parametrize("dtype", [ygg.BF16, ygg.F32])
@pytest.mark.parametrize("Dh", [64, 128])
@pytest.mark.parametrize("heads", [(2, 2), (8, 2)])
def test_chunks_behind_cached_keys_and_queries_that_see_nothing(dtype, Dh, heads):
    """More keys than queries: the next chunk of a prompt.  Fewer: the first queries see no key.  None on either side."""
    q_lens = [1, 5, 64, 70, 130, 40, 0, 9, 300, 65]
    k_lens = [700, 64, 65, 3, 129, 0, 50, 9, 280, 1000]
    p = _problem(heads, Dh, q_lens, k_lens, dtype=dtype, seed=3, gap=2)
    _check(p, *_attend(p))


PLANS = [  # heads, Dh, q_lens, k_lens, (rows of a workgroup, key splits > 1)
    ((32, 8), 128, [1500, 1, 300], None, (256, False)), ((40, 8), 128, [600], [9000], (256, True)),
    ((12, 12), 128, [150, 140, 160], [5150, 5000, 300], (256, True)), ((12, 12), 64, [700] * 8, [2700] + [700] * 7, (256, False)),
    ((8, 1), 64, [300], [30300], (256, True)), ((40, 40), 128, [1000, 700], None, (128, False)), ((8, 8), 128, [4100], None, (128, False)),
    ((32, 32), 64, [700, 699], None, (128, False)), ((8, 8), 128, [40] * 20, None, (128, False)), ((2, 2), 64, [600, 300], None, (128, False)),
    ((32, 8), 128, [990], None, (128, False)), ((32, 8), 128, [990], [1900], (128, True)), ((64, 8), 128, [30, 77], [3000, 2500], (128, True)),
    ((8, 8), 64, [4100], None, (128, True)), ((12, 12), 64, [1990], None, (128, True)), ((8, 1), 128, [600], None, (128, True)),
    ((12, 12), 64, [150, 149, 140, 100], [2150, 2000, 1900, 300], (128, True)), ((8, 1), 128, [16], [5000], (128, True)),
    ((4, 4), 64, [3, 1], [5000, 70], (128, True)), ((1, 1), 128, [1], [9999], (128, True)), ((12, 12), 64, [100, 200], [4000, 30], (128, True)),
]


@pytest.mark.parametrize("heads,Dh,q_lens,k_lens,plan", PLANS)
def test_every_kind_of_plan(heads, Dh, q_lens, k_lens, plan):
    p = _problem(heads, Dh, q_lens, k_lens, seed=len(q_lens) + Dh, gap=3)
    got = ygg.prompt_plan(p["shape"])
    assert (got["rows"], got["splits"] > 1) == plan, got
    _check(p, *_attend(p))


def test_the_bound_may_be_far_above_the_lengths():
    p = _problem((8, 2), 128, [20, 3], [100, 40], seed=1, k_gap=9000, most=18000)
    assert ygg.prompt_plan(p["shape"])["splits"] > 1
    _check(p, *_attend(p))
    # rows of no sequence count too: tiles of 256 rows
    for lens in ([700], [200, 70]):
        p = _problem((40, 40), 128, lens, seed=2, gap=(3000 - sum(lens)) // (len(lens) + 1), most=3000 // len(lens) - 20)
        if len(lens) == 1:
            assert (ygg.prompt_plan(p["shape"])["rows"], ygg.prompt_plan(p["shape"])["splits"]) == (256, 1)
        _check(p, *_attend(p))


@pytest.mark.parametrize("dtype", [ygg.BF16, ygg.F32])
def test_parts_of_a_fused_projection_and_many_short_sequences(dtype):
    lens = [(37 * b) % 90 for b in range(150)]
    p = _problem((6, 2), 64, lens, dtype=dtype, seed=5, fused=True, gap=1)
    assert not p["q"].is_contiguous()
    out, lse = _attend(p)
    _check(p, out, lse)
    dense = {**p, **{x: p[x].contiguous() for x in "qkv"}}
    again, lse2 = _attend(dense)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_padded_batch_and_slabs_of_a_cache():
    """The same sequences packed, padded to the longest, and with keys in slabs of a cache whose rest is garbage: the same bits."""
    B, T, cap, heads, Dh = 3, 90, 128, (8, 2), 128
    lens = np.array([90, 17, 64])
    p = _problem(heads, Dh, lens, seed=9)
    want = _attend(p)
    pad = {x: torch.full((B * (T if x == "q" else cap), *p[x].shape[1:]), float("nan"), dtype=torch.bfloat16, device=DEV) for x in "qkv"}
    for b, n in enumerate(lens):
        for x in "qkv":
            at = b * (T if x == "q" else cap)
            pad[x][at:at + n] = p[x][p["q_first"][b]:p["q_first"][b] + n]
    padded = dict(p, **pad, q_first=np.arange(B) * T, k_first=np.arange(B) * cap, used=(np.arange(B * T) % T) < np.repeat(lens, T),
                  shape=_shape(B, *heads, Dh, B * T, B * cap, 90))
    got = _attend(padded)
    for b, n in enumerate(lens):
        for x, y in zip(want, got):
            assert torch.equal(x[p["q_first"][b]:p["q_first"][b] + n], y[b * T:b * T + n])
    _check(padded, *got)


@pytest.mark.parametrize("Dh", [64, 128])
def test_scores_over_a_wide_range(Dh):
    """Rows whose softmax is one key, scores hundreds above and below zero, rising and falling along the keys."""
    for seed, gain in enumerate((8.0, 30.0)):
        p = _problem((4, 2), Dh, [700, 130, 300], seed=seed, gain=gain)
        _check(p, *_attend(p), rms=False)
    for sign in (1.0, -1.0):
        p = _problem((4, 2), Dh, [900, 65], seed=7)
        ramp = torch.cat([torch.linspace(0.1, 2, int(n)) for n in p["q_lens"]]).to(DEV)[:, None, None]
        p["k"] = (p["k"].float() * 0.2 + ramp).to(torch.bfloat16)
        p["q"] = (p["q"].float() * 0.2 + sign * 3).to(torch.bfloat16)
        _check(p, *_attend(p), rms=False)


def test_a_prompt_in_one_piece_and_in_chunks():
    """The chunks' rows agree with the whole prompt's: both are the definition's."""
    n, heads, Dh = 900, (8, 2), 128
    p = _problem(heads, Dh, [n], seed=2)
    for cuts in ([0, 300, 301, 556, 900], [0, 899, 900]):
        for a, b in zip(cuts, cuts[1:]):
            c = dict(p, shape=_shape(1, *heads, Dh, b - a, n, n), q=p["q"][a:b], q_first=np.array([0]), q_lens=np.array([b - a]), k_lens=np.array([b]),
                     used=np.ones(b - a, bool))
            _check(c, *_attend(c))


def test_without_lse_on_another_stream_and_again():
    p = _problem((8, 2), 128, [500, 64], seed=4)
    out, _ = _attend(p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again, none = _attend(p, want_lse=False)
    assert torch.equal(out, again) and none is None


def test_lengths_and_rows_that_do_not_fit_are_cut():
    """Starts outside the rows make a sequence empty, lengths end with the rows, k_len with the bound; nothing else is touched."""
    T, heads, Dh = 200, (4, 2), 64
    p = _problem(heads, Dh, [T], seed=6)
    p["shape"] = _shape(4, *heads, Dh, T, T, 150)
    p |= dict(q_first=np.array([0, 100, -3, 500]), q_lens=np.array([90, 1 << 30, 5, 4]), k_first=np.array([50, 190, 0, 0]), k_lens=np.array([1 << 30, 40, 5, 5]),
              used=(np.arange(T) < 90) | (np.arange(T) >= 100))
    out, lse = _attend(p)
    cut = dict(p, q_lens=np.array([90, 100, 0, 0]), k_lens=np.array([150, 10, 5, 5]), q_first=np.array([0, 100, 0, 0]))
    _check(cut, out, lse)
    p |= dict(q_lens=np.array([-1, 10, 0, 0]), k_first=np.array([0, 200, 0, 0]), k_lens=np.array([4, 4, -7, 0]), used=(np.arange(T) >= 100) & (np.arange(T) < 110))
    out, lse = _attend(p)
    assert (out[100:110] == 0).all() and torch.isneginf(lse[100:110]).all() and (out[:100] == 77).all() and (out[110:] == 77).all()


def test_keys_behind_an_offset_beyond_32_bits():
    """K and V of 4.4 GB each; the sequence's rows are the last ones."""
    rows, heads, Dh = (1 << 21) + 100, (8, 8), 128
    k, v = (torch.empty((rows, heads[1], Dh), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    p = _problem(heads, Dh, [70], [90], seed=8)
    k[-90:], v[-90:] = p["k"], p["v"]
    far = dict(p, k=k, v=v, k_first=np.array([rows - 90]), shape=_shape(1, *heads, Dh, 70, rows, 90))
    for x, y in zip(_attend(p), _attend(far)):
        assert torch.equal(x, y)


def test_a_captured_call_replays_like_the_eager_one():
    """Both kinds (one launch, and two with a workspace), captured together, replayed on new inputs with eager work between."""
    problems = [_problem((8, 2), 128, [300, 33], seed=1), _problem((8, 2), 128, [16], [5000], seed=2)]
    i32 = lambda x: to_dev(np.asarray(x, np.int32))
    calls = []
    for p in problems:
        n = ygg.workspace_bytes(p["shape"], ygg.OP_PROMPT_ATTENTION)
        calls.append([p["shape"], p["q"], p["k"], p["v"], *(i32(p[x]) for x in ("q_first", "q_lens", "k_first", "k_lens")),
                      torch.zeros((p["shape"].n_nodes, 8, 128), dtype=torch.bfloat16, device=DEV), None, torch.empty(n, dtype=torch.uint8, device=DEV) if n else None])
        ygg.prompt_attention(*calls[-1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for c in calls:
            ygg.prompt_attention(*c)
    for round_ in range(4):
        for c in calls:
            c[1].normal_()
            c[8].zero_()
        calls[0][5].copy_(i32([300 - round_, 33 - 5 * round_]))       # lengths are the device's: shorter ones
        graph.replay()
        torch.cuda.synchronize()
        got = [c[8].clone() for c in calls]
        for c, g in zip(calls, got):
            c[8].zero_()
            ygg.prompt_attention(*c)
            torch.cuda.synchronize()
            assert torch.equal(c[8], g) and (g != 0).any()


def test_refusals_on_the_gpu_binding():
    p = _problem((4, 2), 64, [20, 10], seed=1)
    s = p["shape"]
    i32 = lambda x: to_dev(np.asarray(x, np.int32))
    good = dict(q=p["q"], k=p["k"], v=p["v"], q_first=i32(p["q_first"]), q_len=i32(p["q_lens"]), k_first=i32(p["k_first"]), k_len=i32(p["k_lens"]),
                out=torch.empty_like(p["q"]), lse=torch.empty((30, 4), device=DEV))
    ygg.prompt_attention(s, **good)
    for x in "qkv":
        for kw, error in ((good[x].float(), TypeError), (good[x].cpu(), ValueError), (good[x][:29], ValueError), (good[x].transpose(1, 2), ValueError),
                          (good[x][:1].expand_as(good[x]), ValueError), (good[x][:, :1], ValueError)):
            with pytest.raises(error, match=x):
                ygg.prompt_attention(s, **{**good, x: kw})
    for x in ("q_first", "q_len", "k_first", "k_len"):
        with pytest.raises(TypeError, match=x):
            ygg.prompt_attention(s, **{**good, x: good[x].long()})
        with pytest.raises(ValueError, match=x):
            ygg.prompt_attention(s, **{**good, x: good[x][:1]})
    for x in ("out", "lse"):
        with pytest.raises(ValueError, match=x):
            ygg.prompt_attention(s, **{**good, x: good[x][:29]})
    with pytest.raises(TypeError, match="out"):
        ygg.prompt_attention(s, **{**good, "out": good["out"].float()})
    with pytest.raises(RuntimeError, match="null"):
        ygg.prompt_attention(s, **{**good, "v": None})
    few = _problem((4, 2), 64, [3], [4000], seed=1)
    with pytest.raises(RuntimeError, match="workspace"):
        ygg.prompt_attention(few["shape"], few["q"], few["k"], few["v"], *(i32(few[x]) for x in ("q_first", "q_lens", "k_first", "k_lens")), torch.empty_like(few["q"]))
