"""The operators of a prompt's way in a row, as a program uses them: norms and rotary positions, attention of the prompts, their keys and
values into the 4-bit cache, then decode steps of trees over it -- eagerly, and captured once and replayed with other work between."""
import numpy as np
import pytest
import torch

import paper_2512_23858_amd as ygg
import plain_ops
import plain_prompt as plain
import ygg_workloads as wl
from gpu_util import DEV, to_dev, to_f64, workspace
from test_gpu_block8 import _check as check_tree_attention

pytestmark = pytest.mark.gpu

B, D, W, V, HQ, HKV, DH, LAYERS, T = 3, 3, 4, 997, 8, 2, 64, 2, 150
N = 1 + D * W
PROMPT = np.array([150, 61, 0], np.int32)


class Program:
    """A model's attention layers with random projections: the buffers that a program keeps, and the calls."""

    def __init__(self, seed):
        g = np.random.default_rng(seed)
        base = dict(batch=B, n_q_heads=HQ, n_kv_heads=HKV, head_dim=DH, vocab=V, softmax_scale=DH ** -0.5, kv_capacity=500, max_seq_len=400)
        self.step_shape = ygg.Shape(depth=D, width=W, n_nodes=N, kv_dtype=ygg.FP4_BLOCK, **base)
        self.prompt_shape = ygg.Shape(depth=0, width=1, n_nodes=T, kv_dtype=ygg.FP4_BLOCK, **base)                # T tokens of each sequence
        self.rows_shape = ygg.Shape(depth=0, width=1, n_nodes=B * T, kv_dtype=ygg.BF16, **{**base, "kv_capacity": B * T, "max_seq_len": T})
        self.cache = ygg.new_block4_cache(self.step_shape, LAYERS, device=DEV)
        bf = lambda *s: torch.from_numpy(g.standard_normal(s)).to(torch.bfloat16).to(DEV)
        self.weights = [torch.from_numpy(1 + 0.2 * g.standard_normal(DH)).float().to(DEV) for _ in range(2)]
        self.freq = ygg.rotary_frequencies(DH).to(DEV)
        self.prompt_qkv, self.tree_qkv = bf(LAYERS, B, T, HQ + 2 * HKV, DH) * 3, bf(LAYERS, B, N, HQ + 2 * HKV, DH) * 3
        empty = lambda n, h: torch.zeros((LAYERS, B, n, h, DH), dtype=torch.bfloat16, device=DEV)
        self.pq, self.pk, self.pout, self.q, self.k, self.out = empty(T, HQ), empty(T, HKV), empty(T, HQ), empty(N, HQ), empty(N, HKV), empty(N, HQ)
        self.pv, self.v = (x[:, :, :, HQ + HKV:].contiguous() for x in (self.prompt_qkv, self.tree_qkv))
        self.lse = torch.zeros((LAYERS, B, N, HQ), device=DEV)
        self.positions = torch.arange(T, dtype=torch.int32, device=DEV).expand(B, T).contiguous()
        self.first, self.n = to_dev(np.arange(B, dtype=np.int32) * T), to_dev(PROMPT)
        self.parent = to_dev(np.stack([wl.level_tree(seed, D, W, "uniform", 0.0, sub=b) for b in range(B)]))
        self.token = to_dev(np.stack([wl.node_tokens(seed, self.parent[b].cpu().numpy(), V, sub=b) for b in range(B)]))
        self.logits = torch.from_numpy(np.stack([wl.target_logits(seed, self.parent[b].cpu().numpy(), self.token[b].cpu().numpy(), V, 0.9, sub=b)
                                                 for b in range(B)])).to(DEV)
        i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
        self.lens, self.alen, self.path, self.bonus = i32(B), i32(B), i32(B, D + 1), i32(B)
        need = ygg.workspace_bytes(self.rows_shape, ygg.OP_PROMPT_ATTENTION)
        self.prompt_ws = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
        self.ws = [workspace(self.step_shape, op) for op in (ygg.OP_ATTENTION_BLOCK4, ygg.OP_ACCEPT)]

    def prompt(self):
        self.lens.copy_(self.n)
        for l in range(LAYERS):
            x = self.prompt_qkv[l]
            ygg.tree_norm_rotary(self.prompt_shape, x[:, :, :HQ], x[:, :, HQ:HQ + HKV], self.pq[l], self.pk[l], *self.weights, self.freq,
                                 positions=self.positions)
            ygg.prompt_attention(self.rows_shape, self.pq[l].flatten(0, 1), self.pk[l].flatten(0, 1), x.flatten(0, 1)[:, HQ + HKV:], self.first, self.n,
                                 self.first, self.n, self.pout[l].flatten(0, 1), None, self.prompt_ws)
        ygg.block4_append(self.step_shape, LAYERS, self.pk, self.pv, self.cache, self.lens, self.n)

    def step(self):
        s = self.step_shape
        for l in range(LAYERS):
            x = self.tree_qkv[l]
            ygg.tree_norm_rotary(s, x[:, :, :HQ], x[:, :, HQ:HQ + HKV], self.q[l], self.k[l], *self.weights, self.freq, seq_lens=self.lens,
                                 parent_idx=self.parent)
            ygg.tree_attention_block4(s, self.q[l], self.cache.layer(l), self.lens, self.k[l], self.v[l], self.parent, self.out[l], self.lse[l], self.ws[0])
        ygg.accept_and_compact(s, 0, self.parent, self.token, None, None, None, None, self.lens, self.alen, self.path, self.bonus,
                               target_logits=self.logits, workspace=self.ws[1])
        ygg.block4_append(s, LAYERS, self.k, self.v, self.cache, self.lens, self.alen, rows=self.path)

    def state(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.pout, self.out, self.lse, self.alen, self.path, self.bonus, self.lens, *self.cache.tensors())]


def _equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def _stored(program, confirmed):
    """Every confirmed token of (layer, sequence) as the cache has to hold it: codes of whole blocks byte for byte, the rest as rows."""
    for (l, b), rows in confirmed.items():
        L = int(program.lens[b])
        for x in "kv":
            assert len(rows[x]) == L
            full = L // 64
            codes, scale = plain.encode(rows[x][:64 * full].reshape(full, 64, HKV, DH).transpose(2, 0, 1, 3), x)
            assert np.array_equal(getattr(program.cache, x + "_codes")[l, b, :, :full].cpu().numpy(), codes)
            assert np.array_equal(getattr(program.cache, x + "_scale")[l, b, :, :full].cpu().numpy(), scale)
            tail = to_f64(getattr(program.cache, x + "_tail")[l, b])
            for t in range(64 * full, L):
                assert np.array_equal(tail[t % 128], rows[x][t])


def test_a_prompt_and_the_steps_behind_it():
    p = Program(21)
    p.prompt()
    torch.cuda.synchronize()
    for l in range(LAYERS):
        x = to_f64(p.prompt_qkv[l])
        q, size = plain.norm_rotary(x[:, :, :HQ], to_f64(p.weights[0]), 1e-6, np.arange(T)[None], to_f64(p.freq), False, 1.0)
        assert (np.abs(to_f64(p.pq[l]) - q) <= np.abs(q) * 2.0 ** -8 + size * 2.0 ** -19).all()
        for b in range(B):
            n = PROMPT[b]
            ref, _, size = plain.prompt_attention(*(to_f64(y[l, b, :n]) for y in (p.pq, p.pk, p.pv)), DH ** -0.5)
            # scores of at most 8 * 4 * 4 / 8 .. in fp32 add little to the weights' half step and the result's, 2^-8 each
            assert (np.abs(to_f64(p.pout[l, b, :n]) - ref) <= size * 2.0 ** -7 + np.abs(ref) * 2.0 ** -8).all()
            assert (p.pout[l, b, n:] == 0).all()                                # rows of no sequence stay as they were
    confirmed = {(l, b): {"k": to_f64(p.pk[l, b, :PROMPT[b]]), "v": to_f64(p.pv[l, b, :PROMPT[b]])} for l in range(LAYERS) for b in range(B)}
    _stored(p, confirmed)
    for _ in range(25):
        before = p.lens.cpu().numpy().copy()
        cache = [t.clone() for t in p.cache.tensors()]
        p.step()
        torch.cuda.synchronize()
        alen, path = p.alen.cpu().numpy(), p.path.cpu().numpy()
        assert (alen >= 1).all() and np.array_equal(p.lens.cpu().numpy(), before + alen)
        position = plain_ops.positions(p.parent.cpu().numpy(), before)
        for l in range(LAYERS):
            x = to_f64(p.tree_qkv[l])
            k, size = plain.norm_rotary(x[:, :, HQ:HQ + HKV], to_f64(p.weights[1]), 1e-6, position, to_f64(p.freq), False, 1.0)
            assert (np.abs(to_f64(p.k[l]) - k) <= np.abs(k) * 2.0 ** -8 + size * 2.0 ** -19).all()
            dense = {"k": [], "v": []}
            for b in range(B):
                full, at = before[b] // 64, before[b] // 64 % 2 * 64
                for i, (y, tree) in enumerate((("k", p.k), ("v", p.v))):
                    blocks = plain.decode(cache[i][l, b, :, :full].cpu().numpy(), cache[2 + i][l, b, :, :full].cpu().numpy(), y).reshape(HKV, full * 64, DH)
                    rows = torch.cat((cache[4 + i][l, b, at:at + before[b] - full * 64], tree[l, b])).double().cpu().numpy().transpose(1, 0, 2)
                    dense[y].append(np.concatenate((blocks, rows), 1))
                confirmed[l, b]["k"] = np.concatenate((confirmed[l, b]["k"], to_f64(p.k[l, b])[path[b, :alen[b]]]))
                confirmed[l, b]["v"] = np.concatenate((confirmed[l, b]["v"], to_f64(p.v[l, b])[path[b, :alen[b]]]))
            check_tree_attention(dict(shape=p.step_shape, q=p.q[l], lens=before, parent=p.parent.cpu().numpy(), dense=dense), p.out[l], p.lse[l])
    _stored(p, confirmed)


def test_captured_prompt_and_steps_replay_like_the_eager_ones():
    eager, graphed = Program(22), Program(22)
    eager.prompt()
    want = [eager.state()]
    for _ in range(6):
        eager.step()
        want.append(eager.state())
    graphed.prompt()                          # warm
    graphed.step()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph, call in zip(graphs, (graphed.prompt, graphed.step)):
        with torch.cuda.graph(graph):
            call()
    for _ in range(2):                        # the whole run twice, over the same buffers
        for t in (graphed.pout, graphed.out, graphed.lse, graphed.alen, graphed.path, graphed.bonus):
            t.zero_()
        for t, fill in zip(graphed.cache.tensors(), (0, 0, 127, 127, 0, 0)):
            t.fill_(fill)
        graphs[0].replay()
        for i in range(7):
            got = graphed.state()
            assert _equal(got[:1] + got[3:] if i == 0 else got, want[i][:1] + want[i][3:] if i == 0 else want[i]), i
            eager.step()                      # the program's own work between the replays
            graphs[1].replay()
        torch.cuda.synchronize()
