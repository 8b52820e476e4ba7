"""The attention that remembered boxes have received, and eviction, against the definitions in
64 bits and place by place.

Tolerances of box_memory_weigh, with u = 2^-23: a logit is a binary32 sum of dim products, each of a
query and a code (exact for bf16 queries), times scale and code scale, plus bias, less lse: off by
u ((8 + 2 sqrt dim) sum |q k| + |bias| + 2 |s| + 2 |lse|).  exp2 and its argument add u (2 + 1.5 |s - lse|);
the sum over heads and rows stays below (8 + 2 sqrt n) u of itself, and the old weight and the new
share are each rounded once.  What eviction returns and moves is equal, bit for bit.
"""
import math

import numpy as np
import pytest
import torch

import paper_1906_07155_amd as rex
import relation_oracle as O
from test_gpu_relation_attn import draw_boxes

pytestmark = pytest.mark.gpu
U = 2.0 ** -23
F32, BF16 = torch.float32, torch.bfloat16


def fill(rng, pages, hkv, D):
    m = rex.box_memory(pages, hkv, D)
    for t in m[:2]:
        t.copy_(torch.from_numpy(rng.integers(-127, 128, t.shape).astype(np.int8)))
    for t in m[2:4]:
        t.copy_(torch.from_numpy((rng.uniform(0.5, 2.0, t.shape) / 127).astype(np.float32)))
    m[4].copy_(torch.from_numpy(draw_boxes(rng, tuple(m[4].shape[:2]))))
    return m


def table(rng, streams, max_pages, pages):
    return torch.from_numpy(rng.permutation(pages)[:streams * max_pages].reshape(streams, max_pages).astype(np.int32)).cuda()


def check_weigh(seed, streams, nq, heads, hkv, D, dtype, max_pages, lengths, nb=0, q_len=None, decay=0.5, change=None,
                weighted=True, lse_up=0.0):
    rng = np.random.default_rng(seed)
    pages = streams * max_pages + 2
    m = fill(rng, pages, hkv, D)
    tab = table(rng, streams, max_pages, pages)
    q = torch.from_numpy(rng.standard_normal((streams, nq, heads, D)).astype(np.float32)).to(dtype).cuda()
    boxes = torch.from_numpy(draw_boxes(rng, (streams, nq))).cuda()
    bias = torch.from_numpy(rng.standard_normal((heads, nb, nb)).astype(np.float32)).cuda() if nb else None
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    ql = None if q_len is None else torch.tensor(q_len, dtype=torch.int32, device="cuda")
    if change:
        change(q, tab, bias, ql)
    geo = dict(q_boxes=boxes, bias=bias, octave_steps=2, q_len=ql)
    _, lse = rex.box_memory_attn_fwd(q, m, tab, lens, save=True, **geo)
    lse = lse + lse_up
    w = torch.from_numpy(rng.exponential(size=(streams, 32 * max_pages)).astype(np.float32)).cuda()
    got = rex.box_memory_weigh(q, m, tab, lens, lse, weight=w if weighted else None, decay=decay, **geo)
    scale = float(np.float32(D ** -0.5))
    want, tol = np.zeros(w.shape), np.zeros(w.shape)
    tabn, wn, lsen, qn = tab.cpu().numpy(), w.cpu().numpy().astype(np.float64), lse.double().cpu().numpy(), q.double().cpu().numpy()
    k8, ks, mb = m[0].cpu().numpy(), m[2].cpu().numpy(), m[4].cpu().numpy()
    for b in range(streams):
        t = int(np.clip(lengths[b], 0, 32 * max_pages))
        rows = nq if q_len is None else int(np.clip(q_len[b], 0, nq))
        ok = np.repeat((tabn[b] >= 0) & (tabn[b] < pages), 32)[:t]
        safe = np.clip(tabn[b], 0, pages - 1)
        k = (k8[safe].astype(np.float64) * ks[safe].astype(np.float64)[..., None]).transpose(1, 0, 2, 3).reshape(hkv, -1, D)[:, :t]
        at = O.buckets(boxes[b, :rows].cpu().numpy(), mb[safe].reshape(-1, 4)[:t], nb, -4, 2) if nb else None
        new, new_tol, terms = np.zeros(t), np.zeros(t), 0
        for h in range(heads):
            kh = k[h // (heads // hkv)]
            dots = scale * (qn[b, :rows, h] @ kh.T)
            size = scale * (np.abs(qn[b, :rows, h]) @ np.abs(kh).T)
            add = np.zeros_like(dots)
            if nb:
                add = bias[h].double().cpu().numpy().reshape(-1)[at]
                add = np.where(add <= -1e30, -np.inf, add)
            s, l = dots + add, lsen[b, h, :rows, None]
            on = np.isfinite(l) & np.ones_like(s, dtype=bool)
            with np.errstate(all="ignore"):
                p = np.where(on, np.exp(np.minimum(s - l, 0)), 0.0)
                gap = np.where(p > 0, np.abs(s - l), 0.0)
                off = U * ((8 + 2 * math.sqrt(D)) * size + np.where(np.isfinite(add), np.abs(add), 0) + 2 * np.where(np.isfinite(s), np.abs(s), 0) + 2 * np.where(on, np.abs(l), 0) + 2 + 1.5 * gap)
            new += p.sum(0)
            new_tol += np.where(p > 0, p * off, 0.0).sum(0)
            terms += rows
        new_tol += U * (8 + 2 * math.sqrt(max(terms, 1))) * new
        old = float(np.float32(decay)) * wn[b, :t] if weighted else 0.0
        want[b, :t] = np.where(ok, old + new, 0.0)
        tol[b, :t] = np.where(ok, new_tol + U * np.abs(want[b, :t]) + 1e-37, 0.0)
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol).all(), "%d of %d, worst %s" % ((err > tol).sum(), err.size, np.max(err / np.maximum(tol, 1e-300)))
    return m, q, tab, lens, lse, w, geo


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("nq", [1, 5, 16, 17, 100, 300])
@pytest.mark.parametrize("heads,hkv,D,nb", [(1, 1, 8, 0), (8, 8, 32, 15), (6, 2, 40, 7), (16, 4, 64, 31), (3, 3, 96, 1), (8, 1, 128, 15)])
def test_weigh(dtype, nq, heads, hkv, D, nb):
    check_weigh(nq + D, 2, nq, heads, hkv, D, dtype, 4, [128, 70], nb)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("nq,heads,hkv", [(2, 3, 3), (3, 2, 2), (4, 2, 2), (1, 4, 2), (2, 4, 2), (1, 8, 2), (2, 6, 2)])
def test_weigh_rows_that_share_keys(dtype, nq, heads, hkv):
    check_weigh(nq * heads, 3, nq, heads, hkv, 40, dtype, 9, [288, 150, 31], 15, q_len=[nq, nq - 1, nq])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_weigh_many_pages(dtype, D):
    """So many of them that a workgroup has fewer waves."""
    check_weigh(D, 3, 20, 4, 2, D, dtype, 200, [6400, 5000, 33], 7)


@pytest.mark.parametrize("nq", [3, 40])
def test_weigh_lengths(nq):
    """No box, one, pages that end inside a tile, lengths and rows outside their range; in place."""
    lengths = [0, 1, 32, 33, 95, 96, 500, -7]
    check_weigh(nq, 8, nq, 4, 2, 32, BF16, 3, lengths, 15, q_len=[nq, 1, 0, 2, nq + 9, -1, nq, nq])
    m, q, tab, lens, lse, w, geo = check_weigh(nq, 8, nq, 4, 2, 32, F32, 3, lengths, 15)
    want = rex.box_memory_weigh(q, m, tab, lens, lse, weight=w, **geo)
    got = rex.box_memory_weigh(q, m, tab, lens, lse, weight=w, out=w, **geo)
    assert got is w and torch.equal(got, want)


@pytest.mark.parametrize("nq", [2, 50])
def test_weigh_masks_and_bad_pages(nq):
    def change(q, tab, bias, ql):
        tab[0, 1], tab[1, 0] = -1, 10 ** 6
        bias[0] = torch.finfo(F32).min            # a head that sees nothing
        bias[1, :4] = -math.inf
        q[1, 1] = math.nan                        # a row that is none adds nothing
    check_weigh(nq, 2, nq, 4, 2, 32, BF16, 4, [128, 100], 15, change=change)
    check_weigh(nq, 2, nq, 4, 2, 32, F32, 4, [128, 100], 15, change=change, weighted=False)


def test_weigh_a_softmax_over_more_keys():
    check_weigh(3, 2, 20, 4, 4, 32, BF16, 4, [128, 100], 0, lse_up=1.5)


def test_weigh_nothing():
    m = rex.box_memory(4, 2, 32)
    q = torch.zeros((2, 0, 4, 32), device="cuda")
    tab, lens = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda"), torch.tensor([64, 10], dtype=torch.int32, device="cuda")
    w = torch.rand((2, 64), device="cuda")
    got = rex.box_memory_weigh(q, m, tab, lens, torch.zeros((2, 4, 0), device="cuda"), weight=w, decay=0.25)
    want = 0.25 * w
    want[1, 10:] = 0
    assert torch.equal(got, want)
    none = rex.box_memory_weigh(q[:0], m, tab[:0], lens[:0], torch.zeros((0, 4, 0), device="cuda"))
    assert none.shape == (0, 64)


def plain_evict(weight, length, keep):
    """(new length, origin) of one stream, place by place."""
    order = sorted(range(length), key=lambda t: (not math.isnan(weight[t]), -weight[t] if weight[t] == weight[t] else 0, t))
    chosen = set(order[:keep])
    late = iter(t for t in range(keep, length) if t in chosen)
    return keep, [t if t in chosen else next(late) for t in range(keep)]


def check_evict(seed, hkv, D, max_pages, lengths, keep, weights=None, bad=()):
    rng = np.random.default_rng(seed)
    B = len(lengths)
    pages = B * max_pages + 3
    m = fill(rng, pages, hkv, D)
    tab = table(rng, B, max_pages, pages)
    for b, p, v in bad:
        tab[b, p] = v
    places = 32 * max_pages
    w = rng.exponential(size=(B, places)).astype(np.float32) if weights is None else weights(rng, B, places)
    wt = torch.from_numpy(w).cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    before = [t.clone() for t in m]
    left, held, origin = rex.box_memory_evict(m, tab, i32(lengths), wt, i32(keep))
    want = [t.clone() for t in before]
    tabn = tab.cpu().numpy()
    for b in range(B):
        length = int(np.clip(lengths[b], 0, places))
        used = tabn[b, :(length + 31) // 32]
        k = length if ((used < 0) | (used >= pages)).any() else int(np.clip(keep[b], 0, length))
        k, places_of = plain_evict(w[b].tolist(), length, k)
        assert int(left[b]) == k
        assert origin[b].tolist() == places_of + [-1] * (places - k)
        same = held[b].cpu().numpy()
        wanted = np.concatenate([w[b][places_of], np.zeros(places - k, np.float32)]).astype(np.float32)
        assert np.array_equal(same, wanted, equal_nan=True)
        for t, o in enumerate(places_of):
            if t != o:
                p, a, op, oa = tabn[b, t // 32], t % 32, tabn[b, o // 32], o % 32
                want[0][p, :, a] = before[0][op, :, oa]
                want[1][p, :, :, a] = before[1][op, :, :, oa]
                want[2][p, :, a], want[3][p, :, a] = before[2][op, :, oa], before[3][op, :, oa]
                want[4][p, a] = before[4][op, oa]
    assert all(torch.equal(g, x) for g, x in zip(m, want))


@pytest.mark.parametrize("hkv,D", [(1, 8), (2, 32), (5, 40), (8, 64), (3, 128)])
def test_evict(hkv, D):
    check_evict(D, hkv, D, 9, [288, 200, 33, 1], [200, 150, 20, 1])


def test_evict_lengths():
    """Nothing to keep, all of it, one, and numbers outside their range."""
    check_evict(1, 2, 32, 3, [0, 1, 96, 96, 96, 96, 50, 40, 1000, -5], [0, 0, 0, 96, 1, 95, 100, -3, 64, 7])


def test_evict_equal_weights():
    def levels(rng, B, places):
        return rng.integers(0, 3, (B, places)).astype(np.float32)
    check_evict(2, 2, 32, 8, [256] * 4, [100, 1, 255, 128], levels)
    check_evict(3, 2, 32, 8, [256] * 2, [100, 13], lambda rng, B, places: np.zeros((B, places), np.float32))
    def signed(rng, B, places):
        return np.where(rng.random((B, places)) < 0.5, np.float32(-0.0), np.float32(0.0))
    check_evict(4, 2, 32, 8, [256], [100], signed)


def test_evict_numbers():
    """NaN is kept before all, infinities and negative weights by their order."""
    def odd(rng, B, places):
        w = rng.standard_normal((B, places)).astype(np.float32)
        w[rng.random((B, places)) < 0.1] = np.nan
        w[rng.random((B, places)) < 0.1] = np.inf
        w[rng.random((B, places)) < 0.1] = -np.inf
        return w
    check_evict(5, 2, 32, 8, [256, 256, 200], [10, 128, 190], odd)


def test_evict_long():
    check_evict(6, 1, 32, 300, [9600, 5000], [7000, 4990])


def test_evict_bad_pages():
    """A stream with a page outside the memory is left as it is, one behind its boxes does not matter."""
    check_evict(7, 2, 32, 4, [128, 128, 60], [50, 50, 30], bad=((0, 2, -1), (1, 3, 10 ** 6), (2, 3, -1)))


def test_evict_no_stream():
    m = rex.box_memory(4, 2, 32)
    none = torch.zeros((0,), dtype=torch.int32, device="cuda")
    left, held, origin = rex.box_memory_evict(m, none.view(0, 2), none, torch.zeros((0, 64), device="cuda"), none)
    assert left.shape == (0,) and held.shape == (0, 64)
    empty = torch.zeros((3, 0), dtype=torch.int32, device="cuda")
    zero = torch.zeros((3,), dtype=torch.int32, device="cuda")
    left, held, origin = rex.box_memory_evict(m, empty, zero + 5, torch.zeros((3, 0), device="cuda"), zero + 2)
    assert left.tolist() == [0, 0, 0]


def test_streams_graphs_and_the_attention():
    """Weighed, evicted, asked again, eagerly, on another stream and in a graph."""
    rng = np.random.default_rng(8)
    m = fill(rng, 20, 2, 32)
    tab = table(rng, 2, 8, 20)
    lens, keep = torch.tensor([256, 200], dtype=torch.int32, device="cuda"), torch.tensor([100, 150], dtype=torch.int32, device="cuda")
    q = torch.from_numpy(rng.standard_normal((2, 30, 4, 32)).astype(np.float32)).cuda()
    start = [t.clone() for t in m]

    def step():
        for t, s in zip(m, start):
            t.copy_(s)
        _, lse = rex.box_memory_attn_fwd(q, m, tab, lens, save=True)
        w = rex.box_memory_weigh(q, m, tab, lens, lse)
        left, held, origin = rex.box_memory_evict(m, tab, lens, w, keep)
        out, _ = rex.box_memory_attn_fwd(q, m, tab, left)
        return w, left, held, origin, out
    want = [t.clone() for t in step()]
    # the weights are shares: over the places they are the rows times the heads
    assert torch.allclose(want[0].sum(1), torch.full((2,), 120.0, device="cuda"), rtol=1e-5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for seed in range(3):
        q.copy_(torch.from_numpy(np.random.default_rng(seed).standard_normal((2, 30, 4, 32)).astype(np.float32)))
        want = [t.clone() for t in step()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, want))
