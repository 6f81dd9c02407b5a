"""The operators around the verification calls in a row, as a decode step uses them: rotary positions, attention over the 8-bit block
cache, constrained acceptance, append and count -- eagerly, and captured once and replayed with other work between the replays."""
import numpy as np
import pytest
import torch

import paper_2512_23858_amd as ygg
import plain_ops as plain
import ygg_workloads as wl
from gpu_util import DEV, to_dev, workspace

pytestmark = pytest.mark.gpu

B, D, W, V, HQ, HKV, DH, LAYERS = 3, 4, 5, 1999, 8, 2, 64, 2
N = 1 + D * W


class Step:
    """One static decode step: the buffers that a program keeps, and the calls."""

    def __init__(self, seed):
        g = np.random.default_rng(seed)
        self.shape = ygg.Shape(batch=B, n_q_heads=HQ, n_kv_heads=HKV, head_dim=DH, depth=D, width=W, n_nodes=N, vocab=V,
                               kv_dtype=ygg.FP8_BLOCK, softmax_scale=DH ** -0.5, kv_capacity=700, max_seq_len=600)
        self.cache = ygg.new_block_cache(self.shape, LAYERS, device=DEV)
        self.prompt = np.array([190, 61, 0], np.int32)
        bf = lambda *s: torch.from_numpy(g.standard_normal(s)).to(torch.bfloat16).to(DEV)
        self.k_prompt, self.v_prompt = bf(LAYERS, B, 190, HKV, DH), bf(LAYERS, B, 190, HKV, DH)
        self.qkv = bf(LAYERS, B, N, HQ + 2 * HKV, DH)
        self.q = torch.empty((LAYERS, B, N, HQ, DH), dtype=torch.bfloat16, device=DEV)
        self.k = torch.empty((LAYERS, B, N, HKV, DH), dtype=torch.bfloat16, device=DEV)
        self.v = self.qkv[:, :, :, HQ + HKV:].contiguous()
        self.out = torch.empty_like(self.q)
        self.freq = ygg.rotary_frequencies(DH).to(DEV)
        self.parent = to_dev(np.stack([wl.level_tree(seed, D, W, "uniform", 0.0, sub=b) for b in range(B)]))
        self.token = to_dev(np.stack([wl.node_tokens(seed, self.parent[b].cpu().numpy(), V, sub=b) for b in range(B)]))
        self.logits = torch.from_numpy(np.stack([wl.target_logits(seed, self.parent[b].cpu().numpy(), self.token[b].cpu().numpy(), V, 0.9, sub=b)
                                                 for b in range(B)])).to(DEV)
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
        self.lens, self.counts, self.best = i32(B), i32(B, V), i32(B, N)
        self.alen, self.path, self.bonus = i32(B), i32(B, D + 1), i32(B)
        self.factor = torch.full((B,), 1.05, device=DEV)
        self.ws = [workspace(self.shape, op) for op in (ygg.OP_ATTENTION_BLOCK8, ygg.OP_CONSTRAIN, ygg.OP_ACCEPT)]

    def begin(self):
        self.lens.copy_(to_dev(self.prompt))
        self.counts.zero_()
        for t in self.cache.tensors():
            t.zero_()
        ygg.block8_append(self.shape, LAYERS, self.k_prompt, self.v_prompt, self.cache, self.lens, self.lens)

    def run(self):
        s = self.shape
        for l in range(LAYERS):
            x = self.qkv[l]
            ygg.tree_rotary(s, x[:, :, :HQ], x[:, :, HQ:HQ + HKV], self.q[l], self.k[l], self.freq, seq_lens=self.lens, parent_idx=self.parent)
            ygg.tree_attention_block8(s, self.q[l], self.cache.layer(l), self.lens, self.k[l], self.v[l], self.parent, self.out[l], None, self.ws[0])
        ygg.constrain_logits(s, self.logits, self.parent, self.token, best=self.best, counts=self.counts, repetition=self.factor,
                             workspace=self.ws[1])
        ygg.accept_and_compact(s, 0, self.parent, self.token, None, None, None, None, self.lens, self.alen, self.path, self.bonus,
                               target_tokens=self.best, workspace=self.ws[2])
        ygg.block8_append(s, LAYERS, self.k, self.v, self.cache, self.lens, self.alen, rows=self.path)
        ygg.count_tokens(s, self.token, self.alen, self.counts, rows=self.path)

    def state(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.out, self.best, self.alen, self.path, self.bonus, self.lens, self.counts, *self.cache.tensors())]


def _equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_steps_follow_from_each_other():
    s = Step(11)
    s.begin()
    tokens = {(l, b): s.k_prompt[l, b, :s.prompt[b]] for l in range(LAYERS) for b in range(B)}
    counts = np.zeros((B, V), np.int64)
    for _ in range(20):
        before = s.lens.cpu().numpy()
        s.run()
        torch.cuda.synchronize()
        alen, path, best = s.alen.cpu().numpy(), s.path.cpu().numpy(), s.best.cpu().numpy()
        assert (alen >= 1).all() and np.array_equal(s.lens.cpu().numpy(), before + alen)
        for b in range(B):
            token = s.token[b].cpu().numpy()
            x = plain.constrain(s.logits[b].cpu().numpy(), s.parent[b].cpu().numpy(), token, counts[b].astype(np.int32), 1.05, 0, 0, None, None, None)
            assert np.array_equal(best[b], x.argmax(-1))
            rows = path[b, :alen[b]]
            assert s.bonus[b].item() == best[b, rows[-1]]
            np.add.at(counts[b], token[rows], 1)
            for l in range(LAYERS):
                tokens[l, b] = torch.cat((tokens[l, b], s.k[l, b, torch.from_numpy(rows).long().to(DEV)]))
        assert np.array_equal(s.counts.cpu().numpy(), counts)
    for (l, b), k in tokens.items():          # the cache stands for every confirmed key
        L = int(s.lens[b])
        assert len(k) == L
        k = k.double().cpu().numpy().transpose(1, 0, 2)
        full = L // 64
        scale = s.cache.k_scale[l, b, :, :full].cpu().numpy()
        got = plain.decode(s.cache.k_codes[l, b, :, :full].cpu().numpy(), scale, "k").reshape(HKV, full * 64, DH)
        room = np.repeat(scale, 64, axis=1)[..., None] * 2.0 ** -10 + np.abs(k[:, :full * 64]) * 2.0 ** -4     # half a step, E4M3
        assert (np.abs(got - k[:, :full * 64]) <= room).all()
        tail = s.cache.k_tail[l, b].double().cpu().numpy()
        for t in range(full * 64, L):
            assert np.array_equal(tail[t % 128], k[:, t])


def test_a_captured_step_replays_like_the_eager_one():
    eager, graphed = Step(12), Step(12)
    eager.begin()
    graphed.begin()
    want = []
    for _ in range(6):
        eager.run()
        want.append(eager.state())
    graphed.run()                              # warm
    graphed.begin()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        graphed.run()
    other = Step(13)                           # a second capture with workspaces of its own
    other.begin()
    g2 = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g2):
        other.run()
    graphed.begin()
    other.begin()
    for i in range(6):
        g.replay()
        g2.replay()
        assert _equal(graphed.state(), want[i]), i
        eager.run()                            # the program's own work between the replays
        torch.cuda.synchronize()
