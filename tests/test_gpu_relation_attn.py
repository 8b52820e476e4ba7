"""Attention among boxes (box_attn_fwd, box_attn_bwd) against the definition in 64 bits.

How far a result may be off, element by element, from how it is computed:
  weights   p = exp(s - lse): an error of s is a relative error of p.  s is a binary32 sum
            of D products (D * 2^-24 of the sum of their absolute values, at most `logit`),
            lse has the same error again, exp and the scaling add a few roundings of |s|:
            e = 2 * (D + 8) * 2^-24 * max(logit, 1) + 2^-21
  sums      of n terms in binary32: n * 2^-24 of the absolute sum; results whose terms are
            differences (ds) carry e and these roundings on what they are differences of
            (the "_big" sums)
  bf16      has 8 significant bits, so rounding to nearest takes up to 2^-8: of each weight and
            of the result, 2^-7 of the absolute sum
Norm-wise the roundings are independent: two of bf16, rms 2^-8 / sqrt(3) at the bottom and half
of that at the top of an octave, stay under 3e-3, binary32 under 1e-5; to which comes 2^-21 of what
differences are taken of (with a single visible key every ds is 0 and that is all there is).
"""
import numpy as np
import pytest

import paper_1906_07155_amd as rex
import relation_oracle as O
from gpu_helpers import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rex.lib()


DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def f64(t):
    return t.detach().double().cpu().numpy()


def draw_boxes(rng, shape):
    c = rng.uniform(0, 600, (*shape, 2))
    s = np.exp(rng.uniform(np.log(8), np.log(400), (*shape, 2)))
    return np.concatenate([c - s / 2, c + s / 2], -1).astype(np.float32)


class Case:
    """Inputs of one call on the GPU and what the definition makes of them."""

    def __init__(self, dtype, B, nq, nk, H, hkv, D, nb=0, steps=1, first_exp=-4, q_len=None, k_len=None,
                 masked=0.0, layout="dense", seed=0, scale=None, spoil=False):
        rng = np.random.default_rng([seed, B, nq, nk, H, D])
        self.dtype, self.D, self.nk, self.nq = dtype, D, nk, nq
        dt = DT[dtype]

        def dev(x):
            return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(dt).cuda()

        if layout == "packed":                      # one projection's output, cut into q, k, v
            x = dev(rng.standard_normal((B, nq, H + 2 * hkv, D)))
            self.q, self.k, self.v = x[:, :, :H], x[:, :, H:H + hkv], x[:, :, H + hkv:]
        elif layout == "heads":                     # [B, H, N, D] in memory
            self.q, self.k, self.v = (dev(rng.standard_normal((B, h, n, D))).transpose(1, 2)
                                      for h, n in ((H, nq), (hkv, nk), (hkv, nk)))
        elif layout == "shared":                    # every image sees the same keys
            self.q = dev(rng.standard_normal((B, nq, H, D)))
            self.k, self.v = (dev(rng.standard_normal((1, nk, hkv, D))).expand(B, -1, -1, -1)
                              for _ in range(2))
        else:
            self.q = dev(rng.standard_normal((B, nq, H, D)))
            self.k, self.v = (dev(rng.standard_normal((B, nk, hkv, D))) for _ in range(2))
        self.g = dev(rng.standard_normal((B, nq, H, D)))
        self.q_len = None if q_len is None else torch.tensor(q_len, dtype=torch.int32).cuda()
        self.k_len = None if k_len is None else torch.tensor(k_len, dtype=torch.int32).cuda()
        self.mask = None
        if masked:
            self.mask = torch.from_numpy(rng.random((B, nk)) >= masked).cuda()
        self.geo = {}
        idx = bias = None
        if nb:
            qb, kb = draw_boxes(rng, (B, nq)), draw_boxes(rng, (B, nk))
            bias = rng.standard_normal((H, nb, nb)).astype(np.float32)
            rois = np.concatenate([np.zeros((B, nq, 1), np.float32), qb], -1)
            self.geo = dict(q_boxes=torch.from_numpy(rois).cuda()[..., 1:],     # RoIs' columns
                            k_boxes=torch.from_numpy(kb).cuda(), bias=torch.from_numpy(bias).cuda(),
                            first_exp=first_exp, octave_steps=steps)
            idx = np.zeros((B, nq, nk), np.int64)
            for b in range(B):
                idx[b] = O.buckets(qb[b], kb[b], nb, first_exp, steps)
            bias = bias.reshape(H, -1).astype(np.float64)
        self.nb = nb
        self.scale = D ** -0.5 if scale is None else scale
        np_mask = None if self.mask is None else self.mask.cpu().numpy()
        q, k, v, g = (f64(t) for t in (self.q, self.k, self.v, self.g))
        self.ref = O.attn(q, k, v, self.scale, idx, bias, q_len, k_len, np_mask, g)
        if spoil:                                    # what must not matter
            for b in range(B):
                if q_len is not None:
                    self.q[b, max(q_len[b], 0):] = float("nan")
                    self.g[b, max(q_len[b], 0):] = float("inf")
                if k_len is not None:
                    self.k[b, max(k_len[b], 0):] = float("inf")
                    self.v[b, max(k_len[b], 0):] = float("nan")
                if np_mask is not None:
                    off = torch.from_numpy(np.nonzero(~np_mask[b])[0]).cuda()
                    self.k[b, off] = float("nan")
                    self.v[b, off] = float("-inf")

    def args(self):
        return dict(scale=self.scale, q_len=self.q_len, k_len=self.k_len, k_mask=self.mask, **self.geo)

    def fwd(self, **kw):
        return rex.box_attn_fwd(self.q, self.k, self.v, **self.args(), **kw)

    def both(self):
        out, lse, full = self.fwd(save=True)
        grads = rex.box_attn_bwd(self.g, self.q, self.k, self.v, out, lse, full, **self.args())
        return dict(zip(("out", "grad_q", "grad_k", "grad_v", "grad_bias"), (out, *grads)), lse=lse)

    def check(self, got, name):
        e = 2 * (self.D + 8) * 2.0 ** -24 * max(self.ref["logit"], 1.0) + 2.0 ** -21
        e += (max(self.nk, self.nq) + 64) * 2.0 ** -24
        for key in ("out", "grad_q", "grad_k", "grad_v", "grad_bias"):
            if got.get(key) is None:
                continue
            ref, have = self.ref[key], f64(got[key]).reshape(self.ref[key].shape)
            tol = e * self.ref[key + "_big"] + 1e-30
            if self.dtype == "bf16" and key != "grad_bias":
                assert got[key].dtype == torch.bfloat16
                tol = tol + 2.0 ** -7 * self.ref[key + "_abs"]
            assert np.isfinite(have).all(), (name, key)
            bad = np.abs(have - ref) > tol
            assert not bad.any(), "%s %s: %d off, worst %g of its bound" % (
                name, key, int(bad.sum()), float((np.abs(have - ref) / tol).max()))
            few = 3e-3 if self.dtype == "bf16" and key != "grad_bias" else 1e-5
            big = 2.0 ** -21 * np.linalg.norm(self.ref[key + "_big"])
            assert np.linalg.norm(have - ref) <= few * np.linalg.norm(ref) + big, (name, key)
        if got.get("lse") is not None:
            have = f64(got["lse"])
            ref = self.ref["lse"]
            assert np.array_equal(np.isinf(have), np.isinf(ref)), name
            fin = np.isfinite(ref)
            assert np.all(np.abs(have[fin] - ref[fin]) <= e * 2 + 2.0 ** -22 * np.abs(ref[fin])), name


SHAPES = [
    # B, nq, nk, H, hkv, D, nb
    (1, 1, 1, 1, 1, 8, 0), (1, 1, 1, 8, 8, 32, 15), (2, 3, 5, 2, 2, 16, 3), (1, 16, 32, 4, 4, 32, 7),
    (1, 17, 31, 4, 2, 24, 15), (2, 33, 33, 8, 8, 32, 15), (1, 64, 65, 16, 16, 64, 15), (1, 100, 100, 8, 8, 32, 15),
    (3, 49, 49, 6, 2, 48, 15), (1, 40, 70, 3, 1, 40, 31), (2, 20, 129, 8, 1, 72, 31), (1, 130, 20, 4, 4, 96, 15),
    (1, 35, 67, 2, 2, 128, 31), (1, 5, 300, 5, 5, 64, 1), (1, 300, 5, 7, 7, 64, 15), (1, 1, 700, 8, 8, 64, 15),
    (2, 9, 33, 32, 4, 32, 15), (1, 33, 9, 64, 2, 16, 31),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_shapes(dtype, shape):
    log("attn %s %s" % (dtype, shape))
    B, nq, nk, H, hkv, D, nb = shape
    c = Case(dtype, B, nq, nk, H, hkv, D, nb)
    c.check(c.both(), str(shape))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["packed", "heads", "shared"])
def test_layouts(dtype, layout):
    log("attn layout %s %s" % (dtype, layout))
    c = Case(dtype, 2, 45, 45, 8, 2 if layout != "heads" else 8, 32, 15, layout=layout, seed=3)
    c.check(c.both(), layout)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nb", [0, 15])
def test_lengths_and_masks_hide_what_they_leave_out(dtype, nb):
    """Images without boxes, without keys, lengths past the end; NaN and infinities in what
    is left out."""
    log("attn masks %s %d" % (dtype, nb))
    c = Case(dtype, 6, 40, 50, 8, 4, 32, nb, q_len=[40, 0, 33, 5, 99, -3], k_len=[50, 50, 0, 33, 70, 1],
             masked=0.3, spoil=True, seed=5)
    c.check(c.both(), "masks")
    c = Case(dtype, 2, 33, 37, 4, 4, 64, nb, masked=1.0, spoil=True, seed=6)     # no key at all
    got = c.both()
    c.check(got, "no key")
    assert all(float(got[k].abs().max()) == 0.0 for k in ("out", "grad_q", "grad_k", "grad_v"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bias_of_minus_infinity_and_of_the_lowest_value(dtype):
    log("attn -inf bias %s" % dtype)
    c = Case(dtype, 1, 40, 40, 4, 4, 32, 7, seed=8)
    bias = c.geo["bias"]
    q, k, v, g = (f64(t) for t in (c.q, c.k, c.v, c.g))
    idx = np.stack([O.buckets(c.geo["q_boxes"][0].cpu().numpy(), c.geo["k_boxes"][0].cpu().numpy(), 7, -4, 1)])
    bias[0] = float("-inf")                          # head 0: every row is left without a key
    bias[1, 3:] = float("-inf")
    bias[2, :4] = torch.finfo(torch.float32).min     # counts as -inf
    bias[3] = torch.finfo(torch.bfloat16).min
    bias[3, 2, 2] = -30.0
    ref = torch.where(bias < -1e30, -float("inf"), bias.double())
    c.ref = O.attn(q, k, v, c.scale, idx, f64(ref).reshape(4, -1), g=g)
    got = c.both()
    assert float(got["out"][:, :, 0].abs().max()) == 0.0 and bool((got["lse"][:, 0] == float("-inf")).all())
    assert float(got["grad_bias"][0].abs().max()) == 0.0
    c.check(got, "-inf bias")


def test_boxes_at_the_edges_of_the_buckets():
    """Distances that lie on an edge, one binary32 number below and above it, zero, negative,
    infinite and not a number: the buckets are seen through one-hot tables."""
    log("attn buckets")
    for nb, steps, first in ((15, 1, -4), (15, 2, -2), (31, 4, -3), (3, 1, 0), (1, 1, 0)):
        n = (nb - 1) // 2
        edges = [2.0 ** (first + i // steps) * (1 + (i % steps) / steps) for i in range(max(n, 1))]
        d = np.array([x for e in edges for x in (np.nextafter(F32(e), F32(0)), F32(e), np.nextafter(F32(e), F32(9e9)))])
        d = np.concatenate([d, -d, [0.0, -0.0, 1e-30, 3e38, np.inf, -np.inf, np.nan]]).astype(np.float32)
        nk = d.size
        qb = np.array([[-0.5, -0.5, 0.5, 0.5], [-2, -1, 2, 1], [0, 0, 0, 0], [np.nan, 0, 1, 1]], np.float32)
        with np.errstate(all="ignore"):
            kb = np.stack([d, d[::-1], d, d[::-1]], -1)      # centre (d, d reversed)
        idx = O.buckets(qb, kb, nb, first, steps)
        for start in range(0, nb * nb, 64):                  # 64 buckets at a time, one head each
            H = min(64, nb * nb - start)
            bias = torch.zeros((H, nb * nb), device="cuda")
            bias[torch.arange(H), start + torch.arange(H)] = 8.0
            z = torch.zeros((1, 4, H, 8), device="cuda")
            eye = torch.zeros((1, nk, 1, 8), device="cuda")
            for lo in range(0, nk, 8):                       # which keys got the bonus, 8 at a time
                v = eye.clone()
                m = min(8, nk - lo)
                v[0, lo + torch.arange(m), 0, torch.arange(m)] = 1.0
                out, _, _ = rex.box_attn_fwd(z, eye, v, bias=bias.view(H, nb, nb), first_exp=first, octave_steps=steps,
                                             q_boxes=torch.from_numpy(qb)[None].cuda(),
                                             k_boxes=torch.from_numpy(kb)[None].cuda())
                p = out[0, :, :, :m].cpu().numpy()           # [4, H, m]
                hit = idx[:, None, lo:lo + m] == (start + np.arange(H))[None, :, None]
                count = (idx[:, None, :] == (start + np.arange(H))[None, :, None]).sum(-1, keepdims=True)
                w = np.where(hit, np.exp(8.0), 1.0) / (count * np.exp(8.0) + (nk - count))
                assert np.allclose(p, w, rtol=1e-4, atol=0), (nb, steps, first)


F32 = np.float32


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeats_bit_for_bit(dtype):
    log("attn repeats %s" % dtype)
    c = Case(dtype, 3, 150, 150, 8, 4, 32, 15, q_len=[150, 90, 1], k_len=[150, 90, 1], masked=0.1)
    a = c.both()
    for _ in range(3):
        b = c.both()
        assert all(torch.equal(a[k], b[k]) for k in a)


def test_gradient_against_differences():
    """The loss of the 64-bit forward moved along random directions, against the GPU's gradient."""
    log("attn differences")
    c = Case("f32", 1, 20, 37, 4, 2, 24, 7, masked=0.2, seed=12)
    got = {k: f64(v) for k, v in c.both().items()}
    rng = np.random.default_rng(1)
    q, k, v, g = (f64(t) for t in (c.q, c.k, c.v, c.g))
    bias = f64(c.geo["bias"]).reshape(4, -1)
    idx = np.stack([O.buckets(c.geo["q_boxes"][0].cpu().numpy(), c.geo["k_boxes"][0].cpu().numpy(), 7, -4, 1)])
    mask = c.mask.cpu().numpy()

    def loss(q, k, v, bias):
        return float((O.attn(q, k, v, c.scale, idx, bias, k_mask=mask)["out"] * g).sum())

    for i, key in enumerate(("grad_q", "grad_k", "grad_v", "grad_bias")):
        args = [q, k, v, bias]
        d = rng.standard_normal(args[i].shape)
        eps = 1e-4
        hi, lo = list(args), list(args)
        hi[i], lo[i] = args[i] + eps * d, args[i] - eps * d
        diff = (loss(*hi) - loss(*lo)) / (2 * eps)
        here = float((got[key].reshape(d.shape) * d).sum())
        # central differences: eps^2 times third derivatives, 1e-8 of sums of order 10
        assert abs(diff - here) <= 1e-5 * (1 + np.abs(got[key].reshape(d.shape) * d).sum()), key


def test_without_out_f32_the_gradients_are_those_of_the_rounded_output():
    log("attn without out_f32")
    c = Case("bf16", 1, 60, 60, 4, 4, 32, 15, seed=4)
    out, lse, full = c.fwd(save=True)
    assert full.dtype == torch.float32 and torch.equal(full.to(torch.bfloat16), out)
    grads = rex.box_attn_bwd(c.g, c.q, c.k, c.v, out, lse, **c.args())
    d = abs(f64(grads[3]).reshape(c.ref["grad_bias"].shape) - c.ref["grad_bias"])
    assert np.all(d <= 2.0 ** -8 * c.ref["grad_bias_big"] + 1e-6)


def test_on_another_stream_and_into_given_buffers():
    log("attn stream")
    c = Case("bf16", 1, 1, 2000, 8, 8, 64, 15, seed=2)
    need = rex.box_attn_workspace_size(c.q, c.k, c.v, True, q_boxes=c.geo["q_boxes"],
                                       k_boxes=c.geo["k_boxes"], bias=c.geo["bias"])
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = torch.full_like(c.q, 7.0)
    lse = torch.empty((1, 8, 1), device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = c.fwd(out=out, lse=lse, workspace=ws, stream=s)
    assert got[0] is out and got[1] is lse and got[2] is None
    also = c.fwd(stream=s)[0]
    s.synchronize()
    assert torch.equal(also, out)
    c.check({"out": out, "lse": lse}, "stream")


def test_inside_a_graph():
    log("attn graph")
    c = Case("bf16", 2, 70, 70, 8, 8, 32, 15, q_len=[70, 41], k_len=[70, 41])
    eager = {k: v.clone() for k, v in c.both().items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = c.both()
    for r in range(3):
        for t in got.values():
            t.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], eager[k]) for k in eager), r
        c.both()
        torch.cuda.synchronize()


def test_empty_sides():
    log("attn empty")
    for B, nq, nk in ((0, 5, 5), (2, 0, 5), (2, 5, 0)):
        c = Case("f32", B, nq, nk, 4, 4, 16, 3)
        got = c.both()
        for k in ("out", "grad_q", "grad_k", "grad_v", "grad_bias"):
            assert float(got[k].abs().sum()) == 0.0, (B, nq, nk, k)


def test_many_tiles_share_a_histogram():
    """More query tiles than partial tables: a workgroup adds several of them up."""
    log("attn many tiles")
    c = Case("f32", 90, 24 * 32, 3, 1, 1, 8, 3, seed=9)
    c.check(c.both(), "many tiles")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_largest_tables_of_eight_heads_in_one_workgroup(dtype, D):
    """One step of keys (and of queries): a workgroup takes eight heads, whose tables and tiles come
    near to all of its LDS; heads that share keys, four at a time with small tables."""
    log("attn tables %s %d" % (dtype, D))
    for shape in ((2, 31, 30, 16, 8, D, 31), (2, 30, 32, 8, 8, D, 31), (3, 32, 17, 8, 1, D, 15), (1, 70, 33, 16, 16, D, 31)):
        c = Case(dtype, *shape, seed=13)
        c.check(c.both(), str(shape))


def test_tensors_on_the_host_are_refused():
    log("attn host tensors")
    c = Case("f32", 1, 4, 4, 2, 2, 8, 3)
    for name, bad in (("bias", c.geo["bias"].cpu()), ("q_boxes", c.geo["q_boxes"].cpu()),
                      ("k_len", torch.zeros(1, dtype=torch.int32))):
        with pytest.raises(ValueError, match=name):
            rex.box_attn_fwd(c.q, c.k, c.v, **dict(c.args(), **{name: bad}))
    with pytest.raises(ValueError, match="v must be"):
        rex.box_attn_fwd(c.q, c.k, c.v.cpu())
    out, lse, _ = c.fwd(save=True)
    with pytest.raises(ValueError, match="lse"):
        rex.box_attn_bwd(c.g, c.q, c.k, c.v, out, lse.cpu(), **c.args())
    with pytest.raises(ValueError, match="grad_out"):
        rex.box_attn_bwd(c.g[:, :3], c.q, c.k, c.v, out, lse, **c.args())
    m = rex.box_memory(2, 2, 8)
    with pytest.raises(ValueError, match="slots"):
        rex.box_memory_read(m, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="pages"):
        rex.box_memory_attn_fwd(c.q, m, torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32).cuda())
    with pytest.raises(ValueError, match="post_weight"):
        rex.gated_norm_fwd(c.q[0, :, 0], c.k[0, :, 0], post_weight=torch.ones(8))
    with pytest.raises(rex.RoIExtractError):
        rex.box_attn_fwd(c.q, c.k, c.v, scale=0.0)
