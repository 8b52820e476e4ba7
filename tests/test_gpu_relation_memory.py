"""The 8-bit memory of boxes: what is written and read back is decided in binary32 and has to
be equal bit for bit; the attention over it is held to the bounds of the attention over dense
keys (test_gpu_relation_attn.py), the keys being the values held."""
import numpy as np
import pytest

import paper_1906_07155_amd as rex
import relation_oracle as O
from gpu_helpers import log
from test_gpu_relation_attn import DT, draw_boxes, f64

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rex.lib()


def values(x, dt):
    """[N, Hkv, D] tensor -> what the memory holds of it, in dt."""
    code, scale = O.encode(x.float().cpu().numpy())
    held = code.astype(np.float32) * scale[..., None]
    return torch.from_numpy(held).to(dt)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,hkv,D,layout", [(1, 1, 8, "dense"), (33, 4, 32, "dense"), (300, 8, 32, "packed"),
                                            (70, 3, 40, "rows"), (65, 2, 128, "heads"), (64, 1, 96, "odd")])
def test_append_and_read(dtype, n, hkv, D, layout):
    log("memory %s %d %d %d %s" % (dtype, n, hkv, D, layout))
    dt = DT[dtype]
    rng = np.random.default_rng([n, D])

    def make(shape):
        x = torch.from_numpy(rng.standard_normal(shape).astype(np.float32) * np.exp(rng.uniform(-8, 8, shape[:1] + (1,) * (len(shape) - 1))).astype(np.float32))
        return x.to(dt).cuda()

    if layout == "packed":
        x = make((n, 2 * hkv, D))
        k, v = x[:, :hkv], x[:, hkv:]
    elif layout == "rows":
        k, v = make((2 * n, hkv, D))[::2], make((n, hkv, D))
    elif layout == "heads":
        k, v = make((hkv, n, D)).transpose(0, 1), make((hkv, n, D)).transpose(0, 1)
    elif layout == "odd":               # rows that start at no multiple of 16 bytes
        k, v = make((n, hkv, D + 1))[..., 1:], make((n, hkv, D + 3))[..., :D]
    else:
        k, v = make((n, hkv, D)), make((n, hkv, D))
    boxes = torch.from_numpy(draw_boxes(rng, (n,))).cuda()
    pages = (n + 31) // 32 + 2
    m = rex.box_memory(pages, hkv, D)
    slots = torch.from_numpy(rng.permutation(pages * 32)[:n].astype(np.int64)).cuda()
    rex.box_memory_append(m, slots, k, v, boxes)
    gk, gv, gb = rex.box_memory_read(m, slots, dt)
    assert torch.equal(gk.cpu(), values(k, dt)) and torch.equal(gv.cpu(), values(v, dt))
    assert torch.equal(gb, boxes)
    # the layout that the header documents
    code, scale = O.encode(k.float().cpu().numpy())
    p, at = slots.cpu().numpy() // 32, slots.cpu().numpy() % 32
    assert np.array_equal(m[0].cpu().numpy()[p, :, at], code)
    assert np.array_equal(m[2].cpu().numpy()[p, :, at], scale)
    code, scale = O.encode(v.float().cpu().numpy())
    assert np.array_equal(m[1].cpu().numpy()[p, :, :, at], code)
    assert np.array_equal(m[3].cpu().numpy()[p, :, at], scale)
    # nothing else was written
    rest = torch.from_numpy(np.setdiff1d(np.arange(pages * 32), slots.cpu().numpy())).cuda()
    assert all(float(t.abs().sum()) == 0.0 for t in rex.box_memory_read(m, rest))


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pages,hkv,D,n", [(64, 32, 128, 2048),      # every page full
                                           (530, 32, 128, 2120),     # workgroups with two pages
                                           (75, 112, 40, 2000)])
def test_many_boxes(dt, pages, hkv, D, n):
    """Calls with so many boxes that workgroups share them out by pages; what the call does not
    name keeps what it held."""
    log("memory many %d %d %d %d" % (pages, hkv, D, n))
    rng = np.random.default_rng(n)
    make = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dt).cuda()
    k, v = make(n, hkv, D), make(n, hkv, D)
    boxes = torch.from_numpy(draw_boxes(rng, (n,))).cuda()
    m = rex.box_memory(pages, hkv, D)
    for t in m:
        t.fill_(7)
    want = [t.cpu().numpy().copy() for t in m]
    slots = rng.permutation(pages * 32)[:n].astype(np.int64)
    out = slots.copy()
    out[::97] = [-5, pages * 32, 1 << 40][n % 3]           # some outside the memory
    rex.box_memory_append(m, torch.from_numpy(out).cuda(), k, v, boxes)
    inside = np.flatnonzero((out >= 0) & (out < pages * 32))
    p, at = out[inside] // 32, out[inside] % 32
    (kc, ks), (vc, vs) = O.encode(k.float().cpu().numpy()), O.encode(v.float().cpu().numpy())
    want[0][p, :, at], want[2][p, :, at] = kc[inside], ks[inside]
    want[1][p, :, :, at], want[3][p, :, at] = vc[inside], vs[inside]
    want[4][p, at] = boxes.cpu().numpy()[inside]
    for got, w in zip(m, want):
        assert np.array_equal(got.cpu().numpy(), w)
    # read back in another order, some slots several times and some outside
    ask = rng.choice(out, n + 8)
    gk, gv, gb = rex.box_memory_read(m, torch.from_numpy(ask).cuda(), dt)
    there = (ask >= 0) & (ask < pages * 32)
    p, at = np.where(there, ask, 0) // 32, np.where(there, ask, 0) % 32
    mask = there[:, None, None]
    product = lambda code, scale: torch.from_numpy(
        np.where(mask, code.astype(np.float32) * scale[..., None], np.float32(0))).to(dt)
    assert torch.equal(gk.cpu(), product(want[0][p, :, at], want[2][p, :, at]))
    assert torch.equal(gv.cpu(), product(want[1][p, :, :, at], want[3][p, :, at]))
    assert np.array_equal(gb.cpu().numpy(), np.where(there[:, None], want[4][p, at], np.float32(0)))


def test_many_reads_of_few_slots():
    """One page's boxes asked for more often than a workgroup's list holds."""
    log("memory many reads")
    rng = np.random.default_rng(3)
    hkv, D, n = 32, 64, 9000
    m = rex.box_memory(2, hkv, D)
    slots = torch.arange(64, device="cuda")
    k = torch.from_numpy(rng.standard_normal((64, hkv, D)).astype(np.float32)).cuda()
    boxes = torch.from_numpy(draw_boxes(rng, (64,))).cuda()
    rex.box_memory_append(m, slots, k, k.flip(0), boxes)
    ask = torch.from_numpy(rng.choice([3, 40, 5, -1], n, p=[0.8, 0.1, 0.05, 0.05])).cuda()
    one = rex.box_memory_read(m, slots)
    got = rex.box_memory_read(m, ask)
    for g, w in zip(got, one):
        w = torch.where((ask >= 0).view(-1, *[1] * (w.dim() - 1)), w[ask.clamp(min=0)], torch.zeros_like(w[:1]))
        assert torch.equal(g, w)


def test_slots_outside_and_values_that_are_no_numbers():
    log("memory slots")
    m = rex.box_memory(2, 2, 16)
    x = torch.randn((5, 2, 16), device="cuda")
    x[0, 0, 3], x[0, 0, 4], x[0, 1] = float("inf"), float("nan"), 0.0
    x[1, 0] = float("nan")
    x[1, 1] = float("-inf")
    x[2, 0] = 1e-44
    boxes = torch.rand((5, 4), device="cuda")
    slots = torch.tensor([0, 63, 31, -1, 64], device="cuda")
    rex.box_memory_append(m, slots, x, x.clone(), boxes)
    for got in rex.box_memory_read(m, slots)[:2]:
        want = values(x, torch.float32)
        want[3:] = 0.0
        assert torch.equal(got.cpu(), want)
    assert float(rex.box_memory_read(m, slots)[2][3:].abs().sum()) == 0.0
    # halves go to the even code, the largest magnitude to 127 exactly
    row = torch.arange(16, device="cuda").float() * 0.5 + 120.0
    x = row.clamp(max=127.0).expand(1, 2, 16).contiguous()
    rex.box_memory_append(m, slots[:1], x, x, boxes[:1])
    got = rex.box_memory_read(m, slots[:1])[0][0, 0].cpu().numpy()
    assert np.array_equal(got, np.rint(x[0, 0].cpu().numpy()))
    rex.box_memory_append(m, slots[:0], x[:0], x[:0], boxes[:0])
    assert rex.box_memory_read(m, slots[:0])[0].shape == (0, 2, 16)


class Recall:
    def __init__(self, dtype, streams, nq, tokens, H, hkv, D, nb=0, lengths=None, seed=0, spare=2):
        rng = np.random.default_rng([seed, streams, nq, tokens, D])
        dt = DT[dtype]
        per = (tokens + 31) // 32
        pages = streams * per + spare
        self.memory = rex.box_memory(pages, hkv, D)
        n = pages * 32
        k, v = (torch.from_numpy(rng.standard_normal((n, hkv, D)).astype(np.float32)).cuda() for _ in range(2))
        boxes = draw_boxes(rng, (n,))
        rex.box_memory_append(self.memory, torch.arange(n, device="cuda"), k, v, torch.from_numpy(boxes).cuda())
        held = [x.cpu().numpy() for x in rex.box_memory_read(self.memory, torch.arange(n, device="cuda"))]
        self.pages = rng.permutation(pages)[:streams * per].reshape(streams, per).astype(np.int32)
        self.lengths = [tokens] * streams if lengths is None else lengths
        self.q = torch.from_numpy(rng.standard_normal((streams, nq, H, D)).astype(np.float32)).to(dt).cuda()
        slot = (self.pages[:, :, None] * 32 + np.arange(32)).reshape(streams, per * 32)
        self.k, self.v, self.kb = (np.asarray(x, np.float64)[slot] for x in held)
        self.nb, self.geo, self.idx, self.bias = nb, {}, None, None
        if nb:
            qb = draw_boxes(rng, (streams, nq))
            bias = rng.standard_normal((H, nb, nb)).astype(np.float32)
            self.geo = dict(q_boxes=torch.from_numpy(qb).cuda(), bias=torch.from_numpy(bias).cuda())
            self.idx = np.stack([O.buckets(qb[b], self.kb[b].astype(np.float32), nb, -4, 1) for b in range(streams)])
            self.bias = bias.reshape(H, -1).astype(np.float64)
        self.dtype, self.D = dtype, D

    def run(self, **kw):
        return rex.box_memory_attn_fwd(self.q, self.memory, torch.from_numpy(self.pages).cuda(),
                                       torch.tensor(self.lengths, dtype=torch.int32).cuda(), **self.geo, **kw)

    def check(self, got, lse, name, keep=None, q_len=None):
        ref = O.attn(f64(self.q), self.k, self.v, self.D ** -0.5, self.idx, self.bias, q_len, self.lengths, keep)
        e = 2 * (self.D + 8) * 2.0 ** -24 * max(ref["logit"], 1.0) + 2.0 ** -21 + (self.k.shape[1] + 64) * 2.0 ** -24
        tol = e * ref["out_abs"] + 1e-30
        if self.dtype == "bf16":
            tol = tol + 2.0 ** -7 * ref["out_abs"]
        have = f64(got)
        bad = np.abs(have - ref["out"]) > tol
        assert not bad.any(), "%s: %d off, worst %g" % (name, int(bad.sum()), float((np.abs(have - ref["out"]) / tol).max()))
        few = 3e-3 if self.dtype == "bf16" else 1e-5
        assert np.linalg.norm(have - ref["out"]) <= few * np.linalg.norm(ref["out"]) + 1e-30, name
        if lse is not None:
            have, want = f64(lse), ref["lse"]
            assert np.array_equal(np.isinf(have), np.isinf(want)), name
            fin = np.isfinite(want)
            assert np.all(np.abs(have[fin] - want[fin]) <= 2 * e + 2.0 ** -22 * np.abs(want[fin])), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 1, 8, 0), (2, 1, 33, 8, 8, 32, 15), (3, 1, 1000, 8, 2, 64, 15),
                                   (1, 17, 95, 4, 4, 40, 7), (2, 40, 64, 6, 3, 96, 31), (1, 33, 700, 16, 16, 64, 15),
                                   (1, 3, 260, 2, 1, 128, 31), (1, 1, 5000, 8, 8, 32, 0)], ids=str)
def test_recall_shapes(dtype, shape):
    log("recall %s %s" % (dtype, shape))
    r = Recall(dtype, *shape)
    r.check(*r.run(save=True), str(shape))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_recall_lengths_and_pages_that_are_not_there(dtype):
    log("recall lengths %s" % dtype)
    r = Recall(dtype, 5, 9, 200, 8, 4, 32, 15, lengths=[200, 0, 1, 33, 500])
    # what no length reaches and no page names must not matter
    for t in r.memory[2:]:
        used = torch.from_numpy(np.unique(r.pages)).cuda()
        spare = torch.ones(t.shape[0], dtype=torch.bool, device="cuda")
        spare[used.long()] = False
        t[spare] = float("nan")
    last = int(r.pages[2, 0])
    r.memory[2][last, :, 1:], r.memory[3][last, :, 1:] = float("nan"), float("inf")
    r.memory[4][last, 1:] = float("nan")
    r.lengths[4] = 200
    r.check(*r.run(save=True), "lengths")
    r.lengths[4] = 500                          # clamped to what the pages hold: 7 * 32 places
    got = r.run()[0]
    r.lengths[4] = 224
    r.check(got, None, "clamped")
    keep = np.ones((5, 224), bool)
    r.pages[0, 2], r.pages[3, 0] = -1, 10 ** 6
    keep[0, 64:96] = False
    keep[3, :32] = False
    r.check(*r.run(save=True), "pages", keep)


def test_recall_splits_repeat_bit_for_bit():
    log("recall repeats")
    r = Recall("bf16", 2, 1, 3000, 4, 4, 64, 15)
    a = r.run(save=True)
    for _ in range(3):
        b = r.run(save=True)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_recall_of_many_pages_by_one_wave(dtype):
    """So many streams that a wave takes all of its stream's pages, more than it reads numbers of at
    once: every stream remembers the same boxes in another order of pages."""
    log("recall many pages %s" % dtype)
    rng = np.random.default_rng(8)
    streams, pages, H, D, nb = 512, 131, 8, 32, 15
    m = rex.box_memory(pages, H, D)
    n = pages * 32
    k, v = (torch.from_numpy(rng.standard_normal((n, H, D)).astype(np.float32)).cuda() for _ in range(2))
    kb, qb = draw_boxes(rng, (n,)), draw_boxes(rng, (streams, 1))
    everything = torch.arange(n, device="cuda")
    rex.box_memory_append(m, everything, k, v, torch.from_numpy(kb).cuda())
    gk, gv, _ = rex.box_memory_read(m, everything)
    bias = rng.standard_normal((H, nb, nb)).astype(np.float32)
    q = torch.from_numpy(rng.standard_normal((streams, 1, H, D)).astype(np.float32)).to(DT[dtype]).cuda()
    table = torch.from_numpy(np.stack([rng.permutation(pages) for _ in range(streams)]).astype(np.int32)).cuda()
    out, lse = rex.box_memory_attn_fwd(q, m, table, torch.full((streams,), n, dtype=torch.int32, device="cuda"),
                                       q_boxes=torch.from_numpy(qb).cuda(), bias=torch.from_numpy(bias).cuda(), save=True)
    idx = O.buckets(qb[:, 0], kb, nb, -4, 1)[None]
    ref = O.attn(f64(q).reshape(1, streams, H, D), f64(gk)[None], f64(gv)[None], D ** -0.5, idx,
                 bias.reshape(H, -1).astype(np.float64))
    e = 2 * (D + 8) * 2.0 ** -24 * max(ref["logit"], 1.0) + 2.0 ** -21 + (n + 64) * 2.0 ** -24
    tol = (e + (2.0 ** -7 if dtype == "bf16" else 0.0)) * ref["out_abs"] + 1e-30
    assert (np.abs(f64(out)[:, 0] - ref["out"][0]) <= tol[0]).all()
    few = 3e-3 if dtype == "bf16" else 1e-5
    assert np.linalg.norm(f64(out)[:, 0] - ref["out"][0]) <= few * np.linalg.norm(ref["out"])
    assert np.all(np.abs(f64(lse)[:, :, 0].T - ref["lse"][0]) <= 2 * e + 2.0 ** -22 * np.abs(ref["lse"][0]))


def test_memory_in_a_graph_and_on_another_stream():
    """Append (both forms), read and recall recorded and replayed, with eager work between."""
    log("memory graph")
    rng = np.random.default_rng(12)
    for pages, hkv, D, n in ((8, 4, 32, 100), (64, 32, 128, 2048)):
        m = rex.box_memory(pages, hkv, D)
        make = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda()
        k, v, q = make(n, hkv, D), make(n, hkv, D), make(2, 1, hkv, D)
        boxes = torch.from_numpy(draw_boxes(rng, (n,))).cuda()
        slots = torch.from_numpy(rng.permutation(pages * 32)[:n].astype(np.int64)).cuda()
        table = torch.arange(pages, dtype=torch.int32, device="cuda").expand(2, -1).contiguous()
        lengths = torch.tensor([pages * 32, 40], dtype=torch.int32, device="cuda")

        def run():
            rex.box_memory_append(m, slots, k, v, boxes)
            return (*rex.box_memory_read(m, slots), rex.box_memory_attn_fwd(q, m, table, lengths)[0])

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = run()
        for _ in range(4):
            k.copy_(make(n, hkv, D))
            v.copy_(make(n, hkv, D))
            rex.box_memory_append(m, torch.arange(pages * 32, device="cuda"), *(make(pages * 32, hkv, D) for _ in range(2)),
                                  torch.zeros(pages * 32, 4, device="cuda"))
            rest = [t.clone() for t in m]
            want = [t.clone() for t in run()]
            for t, r in zip(m, rest):
                t.copy_(r)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        # on a given stream, with the current one busy elsewhere
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        rex.box_memory_append(m, slots, k, v, boxes, stream=other)
        far = rex.box_memory_read(m, slots, stream=other)
        out, _ = rex.box_memory_attn_fwd(q, m, table, lengths, stream=other)
        torch.cuda.current_stream().wait_stream(other)
        assert all(torch.equal(a, b) for a, b in zip((*far, out), want))


def test_recall_query_lengths():
    log("recall q_len")
    r = Recall("f32", 3, 20, 100, 4, 4, 32, 7)
    r.q[1, 7:] = float("nan")
    got, lse = r.run(save=True, q_len=torch.tensor([20, 7, 0], dtype=torch.int32).cuda())
    r.q[1, 7:] = 0.0
    r.check(got, lse, "q_len", q_len=[20, 7, 0])


def test_memory_past_four_gigabytes():
    """Pages whose bytes lie past 2^32 in both arrays."""
    log("memory past 4 GiB")
    pages, hkv, D = 140000, 8, 128              # 4.6 GB of keys and as much of values
    m = tuple(torch.empty_like(t, device="meta") for t in rex.box_memory(1, hkv, D, device="cpu"))
    m = tuple(torch.zeros((pages, *t.shape[1:]), dtype=t.dtype, device="cuda") for t in m)
    rng = np.random.default_rng(0)
    k, v = (torch.from_numpy(rng.standard_normal((64, hkv, D)).astype(np.float32)).cuda() for _ in range(2))
    boxes = torch.from_numpy(draw_boxes(rng, (64,))).cuda()
    far = torch.cat([torch.arange(32), (pages - 1) * 32 + torch.arange(32)]).cuda()
    rex.box_memory_append(m, far, k, v, boxes)
    gk, gv, gb = rex.box_memory_read(m, far)
    assert torch.equal(gk.cpu(), values(k, torch.float32)) and torch.equal(gv.cpu(), values(v, torch.float32))
    assert torch.equal(gb, boxes)
    q = torch.from_numpy(rng.standard_normal((1, 2, hkv, D)).astype(np.float32)).cuda()
    out, _ = rex.box_memory_attn_fwd(q, m, torch.tensor([[pages - 1, 0]], dtype=torch.int32).cuda(),
                                     torch.tensor([50], dtype=torch.int32).cuda())
    order = torch.cat([torch.arange(32, 64), torch.arange(18)]).cuda()
    ref = O.attn(f64(q), f64(gk[order])[None], f64(gv[order])[None], D ** -0.5)
    assert np.linalg.norm(f64(out) - ref["out"]) <= 1e-5 * np.linalg.norm(ref["out"])
