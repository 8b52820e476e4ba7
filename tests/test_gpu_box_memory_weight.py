"""Frames through a relation head whose memory forgets by weight, against the definition in 64 bits: the weights
that decide, which boxes they leave, and what every layer holds of each of them afterwards.

Tolerances, u = 2^-23: a logit is off by u ((8 + 2 sqrt dim) sum |q k| + |bias| + 2 |s|) (test_gpu_evict.py has
why), a row's log sum by the largest of its logits' and 4 u |lse| for the two sums and their joining, and a
weight's exponent by both and by 2 u |lse| + u (2 + 1.5 |s - lse|); a place's sum over n terms by (8 + 2 sqrt n) u of
itself, and each layer's addition to the old weight by u of the sum.
"""
import math

import numpy as np
import pytest
import torch

import paper_1906_07155_amd as rex
import relation_oracle as O
from paper_1906_07155_amd import relation_head as RH
from test_gpu_evict import U, plain_evict
from test_gpu_relation_attn import draw_boxes

pytestmark = pytest.mark.gpu
HEADS, KV, DIM, LAYERS, NB = 4, 2, 16, 2, 15


def shares(q, k, tables, boxes, layer, pages, used):
    """A stream's places: the attention of q [rows, heads, dim] that they receive beside the frame's own keys
    k [rows, kv heads, dim], and how far a binary32 result may be off."""
    rows, scale = len(q), float(np.float32(DIM ** -0.5))
    far8, far_scale, far_boxes = layer
    far = (far8[pages].astype(np.float64) * far_scale[pages].astype(np.float64)[..., None]).transpose(1, 0, 2, 3).reshape(KV, -1, DIM)[:, :used]
    at = O.buckets(boxes, np.concatenate([boxes, far_boxes[pages].reshape(-1, 4)[:used]]), NB, -4, 1)
    total, tol = np.zeros(used), np.zeros(used)
    for h in range(HEADS):
        keys = np.concatenate([k[:, h // (HEADS // KV)], far[h // (HEADS // KV)]])
        add = tables[h].reshape(-1)[at]
        s = scale * (q[:, h] @ keys.T) + add
        off = U * ((8 + 2 * math.sqrt(DIM)) * scale * (np.abs(q[:, h]) @ np.abs(keys).T) + np.abs(add) + 2 * np.abs(s))
        top = s.max(1, keepdims=True)
        lse = top + np.log(np.exp(s - top).sum(1, keepdims=True))
        off_lse = off.max(1, keepdims=True) + 4 * U * np.abs(lse)
        p = np.exp(s - lse)[:, rows:]
        total += p.sum(0)
        tol += (p * (off[:, rows:] + off_lse + U * (2 * np.abs(lse) + 2 + 1.5 * np.abs(s - lse)[:, rows:]))).sum(0)
    return total, tol + U * (8 + 2 * math.sqrt(HEADS * rows)) * total


def test_what_is_kept_has_received_the_most(monkeypatch):
    torch.manual_seed(5)
    head = rex.RelationHead(HEADS * DIM, heads=HEADS, kv_heads=KV, layers=LAYERS).cuda()
    with torch.no_grad():
        for layer in head.layers:
            layer.bias.copy_(torch.randn(HEADS, NB, NB))
    memory = head.memory(num_pages=8, streams=2, max_pages=3, evict="weight", decay=0.5)
    seen, evicted = [], []
    attend, evict = RH.relation.box_attn_fwd, RH.evict.box_memory_evict
    monkeypatch.setattr(RH.relation, "box_attn_fwd", lambda q, k, v, **kw: (seen.append((q.clone(), k.clone())), attend(q, k, v, **kw))[1])
    monkeypatch.setattr(RH.evict, "box_memory_evict",
                        lambda m, p, n, w, keep: (evicted.append((n.tolist(), w.clone(), keep.tolist())), evict(m, p, n, w, keep))[1])
    rng = np.random.default_rng(2)
    moved = 0
    for frame, counts in enumerate(([40, 17], [30, 40], [40, 40], [33, 1], [0, 40], [40, 0], [40, 40])):
        boxes = draw_boxes(rng, (2, 40))
        gen = torch.Generator(device="cuda")
        gen.manual_seed(frame)
        x = torch.randn(2, 40, HEADS * DIM, generator=gen, device="cuda")
        used, table = list(memory.used), [list(p) for p in memory.table]
        before = [[t.cpu().numpy() for t in m] for m in memory.layers]
        weight = memory.weight.double().cpu().numpy()
        seen.clear()
        evicted.clear()
        with torch.no_grad():
            head(x, torch.from_numpy(boxes).cuda(), counts, memory)
        assert len(seen) == LAYERS
        keep = [min(u, 96 - c) for u, c in zip(used, counts)]
        decided = memory.weight if keep == used else evicted[0][1]
        assert len(evicted) == (keep != used) and all(e[0] == used and e[2] == keep for e in evicted)
        for s, c in enumerate(counts):
            want, tol = 0.5 * weight[s, :used[s]], 0.0
            for i, (q, k) in enumerate(seen):
                q64, k64 = (t[s, :c].double().cpu().numpy() for t in (q, k))
                if c and used[s]:
                    tables = head.layers[i].bias.detach().double().cpu().numpy()
                    add, off = shares(q64, k64, tables, boxes[s, :c], (before[i][0], before[i][2], before[i][4]), table[s], used[s])
                    want = want + add
                    tol = tol + off + U * np.abs(want)
            got = decided[s].double().cpu().numpy()
            assert (np.abs(got[:used[s]] - want) <= tol + U * np.abs(want) + 1e-37).all(), (frame, s)
            assert not got[used[s]:].any()
            # who stays, by these weights, and where; everything that a layer holds of a box goes with it
            k, origin = plain_evict(decided[s].tolist(), used[s], keep[s])
            moved += sum(t != o for t, o in enumerate(origin))
            assert memory.used[s] == k + c
            assert memory.weight[s, :k].tolist() == decided[s][origin].tolist() and not memory.weight[s, k:].any()
            for i, m in enumerate(memory.layers):
                now = [t.cpu().numpy() for t in m]
                for t, o in enumerate(origin):
                    p, a, q, b = memory.table[s][t // 32], t % 32, table[s][o // 32], o % 32
                    assert np.array_equal(now[0][p, :, a], before[i][0][q, :, b]) and np.array_equal(now[1][p, :, :, a], before[i][1][q, :, :, b])
                    assert all(np.array_equal(now[j][p, :, a], before[i][j][q, :, b]) for j in (2, 3))
                    assert np.array_equal(now[4][p, a], before[i][4][q, b])
                fresh = [now[4][memory.table[s][t // 32], t % 32] for t in range(k, k + c)]
                assert np.array_equal(np.array(fresh).reshape(-1, 4), boxes[s, :c])
    assert moved > 20


@pytest.mark.parametrize("kv,dim", [(2, 32), (5, 40)])
def test_several_memories_with_one_table(kv, dim):
    """All of them moved as each alone would be, and nothing where one of them does not belong."""
    rng = np.random.default_rng(dim)

    def fill(shape, dtype):
        if dtype == torch.int8:
            return torch.from_numpy(rng.integers(-127, 128, shape).astype(np.int8)).cuda()
        return torch.from_numpy(rng.uniform(0.5, 2.0, shape).astype(np.float32)).cuda()
    memories = [tuple(fill(tuple(t.shape), t.dtype) for t in rex.box_memory(8, kv, dim)) for _ in range(3)]
    pages = torch.from_numpy(rng.permutation(8)[:6].reshape(2, 3).astype(np.int32)).cuda()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    lengths, keep = i32(96, 50), i32(60, 33)
    weight = torch.from_numpy(rng.exponential(size=(2, 96)).astype(np.float32)).cuda()
    alone = [[t.clone() for t in m] for m in memories]
    want = [rex.box_memory_evict(m, pages, lengths, weight, keep) for m in alone]
    kept = [[t.clone() for t in m] for m in memories]
    for bad in ([*memories[:2], rex.box_memory(9, kv, dim)], [memories[0], memories[1][:4]],
                [memories[0], tuple(t.cpu() for t in memories[1])], [*memories[:2], ()]):
        with pytest.raises((ValueError, TypeError)):
            rex.box_memory_evict(bad, pages, lengths, weight, keep)
    with pytest.raises(rex.RoIExtractError):
        rex.box_memory_evict(memories, pages, lengths, weight, keep,
                             workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert all(torch.equal(a, b) for m, n in zip(memories, kept) for a, b in zip(m, n))
    got = rex.box_memory_evict(memories, pages, lengths, weight, keep)
    assert all(torch.equal(a, b) for w in want for a, b in zip(got, w))
    assert all(torch.equal(a, b) for m, n in zip(memories, alone) for a, b in zip(m, n))
