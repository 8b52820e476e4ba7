"""The gated norms (gated_norm_fwd, gated_norm_bwd) against the formulas in 64 bits.

Rows are computed in binary32 from their one read on: a result is a chain of about twenty
roundings and two sums over C channels (sums of C terms in a tree: log2 C + 8 roundings), so
it is off by up to 64 * 2^-24 of what its terms add up to in absolute value, here bounded by the
largest value of the row and column sums; column sums over R rows add (R + 64) * 2^-24 of the
absolute sum.  A bf16 result is rounded once: 2^-8 of itself, and 2.5e-3 in the mean over a
thousand values or more.
"""
import numpy as np
import pytest

import paper_1906_07155_amd as rex
import relation_oracle as O
from gpu_helpers import log
from test_gpu_relation_attn import DT, f64

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

NAMES = ("x", "branch", "gate", "post_weight", "post_bias", "pre_weight", "pre_bias")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rex.lib()


class Case:
    def __init__(self, dtype, rows, C, norm, gates=0, branch=True, params=True, stride=0, seed=0, alpha=0.7):
        rng = np.random.default_rng([seed, rows, C, gates])
        dt = DT[dtype]

        def make(*s):
            return torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()

        def data(scale=1.0):
            t = (make(rows, C + stride) * scale + 0.3).to(dt)
            return t[:, stride:] if stride else t
        self.x, self.branch = data(), data(2.0) if branch else None
        self.gy, self.gu = (data().contiguous() for _ in range(2))
        self.args = dict(alpha=alpha, norm=norm, eps=1e-5, gate=make(gates, C) if gates else None)
        for n in ("post_weight", "post_bias", "pre_weight", "pre_bias"):
            on = params and (branch or n.startswith("pre")) and (norm == "layer" or n.endswith("weight"))
            self.args[n] = make(C) * 0.2 + (1.0 if n.endswith("weight") else 0.0) if on else None
        self.dtype, self.rows, self.C, self.gates = dtype, rows, C, gates

    def reference(self, gy=True, gu=True):
        a = {k: f64(v) if torch.is_tensor(v) else v for k, v in self.args.items()}
        gate = None
        if self.gates:
            gate = np.repeat(a["gate"], self.rows // self.gates, 0)
        r = O.norm(f64(self.x), None if self.branch is None else f64(self.branch), gate, a["alpha"], a["post_weight"],
                   a["post_bias"], a["pre_weight"], a["pre_bias"], a["norm"] == "layer", a["eps"],
                   f64(self.gy) if gy else None, f64(self.gu) if gu else None)
        if self.gates:
            r["gate"] = r["gate"].reshape(self.gates, -1, self.C).sum(1)
        return r

    def check(self, got, ref, name, scale=8.0):
        """scale: the largest value that the terms of a result reach."""
        for key, t in got.items():
            if t is None:
                continue
            have, want = f64(t), ref[key]
            assert have.shape == want.shape and np.isfinite(have).all(), (name, key)
            wide = key in ("y", "u", "x", "branch")
            rows = 1 if wide or (key == "gate" and self.gates == self.rows) else self.rows
            tol = (64 + rows) * 2.0 ** -24 * scale * (1 if wide else np.sqrt(rows) * 8 + 8) + 64 * 2.0 ** -24 * np.abs(want)
            if wide and self.dtype == "bf16":
                tol = tol + 2.0 ** -8 * np.abs(want)
            bad = np.abs(have - want) > tol
            assert not bad.any(), "%s %s: %d off, worst %g of its bound" % (
                name, key, int(bad.sum()), float((np.abs(have - want) / tol).max()))
            few = 2.5e-3 if wide and self.dtype == "bf16" else 2e-6
            if have.size < 1000:
                continue                         # the mean is one over many roundings
            assert np.linalg.norm(have - want) <= few * np.linalg.norm(want) + 1e-5 * few * np.sqrt(have.size), (name, key)

    def both(self):
        y, u, stats = rex.gated_norm_fwd(self.x, self.branch, save=True, **self.args)
        grads = rex.gated_norm_bwd(self.gy, self.gu, self.x, self.branch, stats, **self.args)
        return dict(zip(NAMES, grads), y=y, u=u)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("rows,C,gates", [(1, 8, 1), (1, 1024, 0), (7, 77, 7), (33, 96, 1), (100, 250, 4), (64, 256, 64),
                                          (513, 250, 1), (300, 1024, 3), (40, 1025, 2), (9, 2048, 1), (5, 4096, 1),
                                          (3, 5000, 1), (2, 8192, 2), (2000, 128, 1000)])
def test_shapes(dtype, norm, rows, C, gates):
    log("norm %s %s %d %d %d" % (dtype, norm, rows, C, gates))
    c = Case(dtype, rows, C, norm, gates)
    c.check(c.both(), c.reference(), "shape", 30.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parts_left_out(dtype):
    log("norm parts %s" % dtype)
    c = Case(dtype, 50, 256, "layer", 0, params=False)         # no weights: 1 and 0
    got = c.both()
    assert got["gate"] is None and got["pre_weight"] is None
    c.check(got, c.reference(), "bare")
    c = Case(dtype, 50, 256, "rms", 0, branch=False)            # only the second norm
    y, u, stats = rex.gated_norm_fwd(c.x, save=True, **c.args)
    assert y is c.x
    grads = rex.gated_norm_bwd(c.gy, c.gu, c.x, None, stats, **c.args)
    assert grads[1] is None and grads[2] is None and grads[3] is None
    c.check(dict(zip(NAMES, grads), u=u), c.reference(), "second only")
    c = Case(dtype, 50, 256, "layer", 5)                        # only the first
    y, u, stats = rex.gated_norm_fwd(c.x, c.branch, second=False, save=True, **c.args)
    assert u is None
    grads = dict(zip(NAMES, rex.gated_norm_bwd(c.gy, None, c.x, c.branch, stats, **c.args)))
    assert float(grads["pre_weight"].abs().sum()) == 0.0
    c.check(dict(grads, y=y), c.reference(gu=False), "first only", 30.0)
    grads = dict(zip(NAMES, rex.gated_norm_bwd(None, None, c.x, c.branch, stats, **c.args)))
    assert all(float(t.abs().sum()) == 0.0 for t in grads.values())
    y, u, stats = rex.gated_norm_fwd(c.x, c.branch, save=True, **c.args)
    grads = rex.gated_norm_bwd(None, c.gu, c.x, c.branch, stats, **c.args)
    c.check(dict(zip(NAMES, grads), y=y, u=u), c.reference(gy=False), "no grad_y", 30.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [256, 77])
def test_strides_and_alignment(dtype, C):
    log("norm strides %s %d" % (dtype, C))
    for stride in (1, 3, 8, 16):
        c = Case(dtype, 37, C, "rms", 1, stride=stride)
        c.check(c.both(), c.reference(), "stride %d" % stride, 30.0)
    # one row seen many times
    c = Case(dtype, 12, C, "layer", 1)
    c.x = c.x[:1].expand(12, C)
    c.check(c.both(), c.reference(), "expanded", 30.0)


def test_a_row_that_is_no_number_stays_alone():
    log("norm nan")
    c = Case("f32", 20, 128, "rms", 0)
    want = c.both()
    c.x[3, 5], c.branch[7] = float("nan"), float("inf")
    got = c.both()
    keep = torch.ones(20, dtype=torch.bool, device="cuda")
    keep[3] = keep[7] = False
    for k in ("y", "u", "x", "branch"):
        assert torch.equal(got[k][keep], want[k][keep]), k
    assert bool(torch.isnan(got["u"][3]).all()) and bool(torch.isnan(got["u"][7]).all())


def test_rows_of_zeros_and_of_one_value():
    log("norm zeros")
    for norm in ("rms", "layer"):
        c = Case("f32", 8, 256, norm, 0)
        c.x[:], c.branch[:] = 0.0, 0.0
        c.branch[4:] = 5.0                       # no variance
        c.check(c.both(), c.reference(), "zeros", 2e3)
    c = Case("f32", 0, 64, "rms", 3)
    got = c.both()
    assert all(float(got[k].abs().sum()) == 0.0 for k in ("gate", "post_weight", "pre_weight"))
    assert got["y"].shape == (0, 64)


def test_repeats_bit_for_bit_on_another_stream_and_in_a_graph():
    log("norm repeats")
    c = Case("bf16", 3000, 256, "layer", 3)
    want = c.both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y, u, stats = rex.gated_norm_fwd(c.x, c.branch, save=True, stream=s, **c.args)
    grads = rex.gated_norm_bwd(c.gy, c.gu, c.x, c.branch, stats, stream=s, **c.args)
    s.synchronize()
    got = dict(zip(NAMES, grads), y=y, u=u)
    assert all(torch.equal(got[k], want[k]) for k in want)
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
        assert all(torch.equal(got[k], want[k]) for k in want), r
        c.both()
        torch.cuda.synchronize()


def test_gradient_against_differences():
    log("norm differences")
    c = Case("f32", 12, 40, "layer", 3, seed=2)
    got = {k: f64(v) for k, v in c.both().items()}
    a = {k: f64(v) if torch.is_tensor(v) else v for k, v in c.args.items()}
    args = dict(x=f64(c.x), branch=f64(c.branch), gate=a["gate"], post_weight=a["post_weight"], post_bias=a["post_bias"],
                pre_weight=a["pre_weight"], pre_bias=a["pre_bias"])
    gy, gu = f64(c.gy), f64(c.gu)

    def loss(p):
        r = O.norm(p["x"], p["branch"], np.repeat(p["gate"], 4, 0), 0.7, p["post_weight"], p["post_bias"],
                   p["pre_weight"], p["pre_bias"], True, 1e-5)
        return float((r["y"] * gy).sum() + (r["u"] * gu).sum())

    rng = np.random.default_rng(1)
    for key in NAMES:
        d = rng.standard_normal(args[key].shape)
        hi, lo = dict(args), dict(args)
        hi[key], lo[key] = args[key] + 1e-4 * d, args[key] - 1e-4 * d
        diff = (loss(hi) - loss(lo)) / 2e-4
        here = float((got[key] * d).sum())
        # central differences: 1e-8 of third derivatives, the gradient itself to binary32
        assert abs(diff - here) <= 1e-5 * (1 + np.abs(got[key] * d).sum()), key
