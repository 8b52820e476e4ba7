"""Dense layers with their epilogue against the definition in 64 bits.

Tolerances.  A binary32 sum of n products is off by less than u = 2^-23 times (8 + 2 sqrt n) times
the sum S of the products' magnitudes (each of n roundings is off by at most 2^-24 of a partial
sum, signs are random, and 4 deviations of that walk stay below it; 8 for short sums).  The activations
change such an error by a factor of at most 1.13, and are off by 2^-17 of their value at most (of
that x^2 / 2 * 2^-23 for |x| <= 8 from the exponent's argument).  A result is off by half a step of
its type more.  The gradient g = grad_y * slope of bf16 data has slopes off by 2^-23 and, where the
slope is not 0 or 1, is rounded to bf16 (2^-8): both enter the products with the other operand's
magnitude.
"""
import math

import pytest
import torch

import paper_1906_07155_amd as rex
from paper_1906_07155_amd import head

pytestmark = pytest.mark.gpu

U = 2.0 ** -23
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # half a step, relative to the value


def short(n):
    return U * (8 + 2 * math.sqrt(n))


def act64(name, t):
    return {"none": lambda: t, "relu": lambda: t.clamp(min=0), "silu": lambda: t * torch.sigmoid(t),
            "gelu": lambda: t * torch.special.ndtr(t)}[name]()


def slope64(name, t):
    if name == "none":
        return torch.ones_like(t)
    if name == "relu":
        return (t > 0).double()
    if name == "silu":
        s = torch.sigmoid(t)
        return s * (1 + t * (1 - s))
    return torch.special.ndtr(t) + t * torch.exp(-t * t / 2) / math.sqrt(2 * math.pi)


def make(seed, m, n, k, dtype, bias, residual, wide=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    randn = lambda *s, dt=dtype: torch.randn(s, generator=gen, device="cuda").to(dt)
    x, w = randn(m, k + wide)[:, :k], (randn(n, k + wide) * k ** -0.5)[:, :k]
    b = None if bias is None else 0.5 * randn(n, dt=bias)
    r = randn(m, n + wide)[:, :n] if residual else None
    return x, w, b, r, randn(m, n)


def within(got, want, tolerance, what):
    err = (got.double() - want).abs()
    tolerance = tolerance + HALF[got.dtype] * want.abs() + 1e-38
    bad = err > tolerance
    assert not bad.any(), "%s: %d of %d, worst %.3g of the tolerance" % (
        what, int(bad.sum()), bad.numel(), float((err / tolerance).max()))


def kept(saved, dtype, m, n):
    """What the backward takes the slopes (or relu's result) from, as numbers."""
    if dtype == torch.float32 or saved.dtype == dtype:
        return saved.double()
    upper = saved[:2 * m * n].view(torch.int16).int() & 0xffff
    return ((upper << 8 | saved[2 * m * n:].int()).double() * 2.0 ** -23 - 0.25).view(m, n)


def check(seed, m, n, k, dtype, act="none", bias=torch.float32, residual=False, wide=0, backward=True):
    x, w, b, r, gy = make(seed, m, n, k, dtype, bias, residual, wide)
    y, saved = rex.linear_act_fwd(x, w, b, act=act, residual=r, save=True)
    xd, wd = x.double(), w.double()
    t, size = xd @ wd.t(), xd.abs() @ wd.abs().t()
    if b is not None:
        t, size = t + b.double(), size + b.double().abs()
    tol_t = short(k) * size
    a = act64(act, t)
    want = a if r is None else a + r.double()
    within(y, want, 1.13 * tol_t + 2.0 ** -17 * a.abs() + U * want.abs(), "y")
    assert (saved is None) == (act == "none")
    if not backward:
        return
    if act in ("gelu", "silu"):
        slope = slope64(act, t)
        err = (kept(saved, dtype, m, n) - slope).abs()
        assert bool((err <= 0.8 * tol_t + 2.0 ** -17 * slope.abs() + 2.0 ** -22).all())
    grads = rex.linear_act_bwd(gy, x, w, saved, bias=b, act=act)
    g64 = gy.double()
    if act == "relu":           # (a sum next to 0 may fall to either side)
        on = kept(saved, dtype, m, n) > 0
        assert bool((on == (t > 0))[t.abs() > tol_t].all())
        g, g_tol = g64 * on, torch.zeros_like(g64)
    else:
        g = g64 * slope64(act, t)
        # (the second derivatives are below 0.8)
        g_tol = g64.abs() * (0.8 * tol_t + 2.0 ** -17) if act != "none" else torch.zeros_like(g64)
    col_tol = g_tol + (g64.abs() * 2.0 ** -23 if dtype == torch.bfloat16 and act in ("gelu", "silu") else 0)
    if dtype == torch.bfloat16 and act in ("gelu", "silu"):
        g_tol = col_tol + 2.0 ** -8 * g.abs()
    within(grads[0], g @ wd, short(n) * (g.abs() @ wd.abs()) + g_tol @ wd.abs(), "grad_x")
    within(grads[1], g.t() @ xd, short(m) * (g.abs().t() @ xd.abs()) + g_tol.t() @ xd.abs(), "grad_weight")
    if b is None:
        assert grads[2] is None
    else:
        assert grads[2].dtype == b.dtype
        within(grads[2], g.sum(0), short(m) * g.abs().sum(0) + col_tol.sum(0), "grad_bias")


F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("residual", [False, True])
def test_activations(dtype, act, residual):
    check(1, 70, 48, 96, dtype, act, residual=residual)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 5, 3), (2, 1, 129), (3, 77, 250), (65, 63, 65), (64, 64, 64),
                                   (130, 17, 1000), (513, 77, 250), (129, 257, 31), (1, 1024, 1024),
                                   (17, 1000, 264), (33, 16, 4104), (64, 24, 12544), (300, 81, 1024)])
def test_sizes(dtype, m, n, k):
    check(m * 7 + n, m, n, k, dtype, "silu", bias=F32, residual=True)
    check(m * 7 + n + 1, m, n, k, dtype, "none", bias=None)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(16, 40, 8192), (17, 40, 1024), (64, 300, 512), (300, 16, 4104), (1001, 5, 264), (400, 33, 256),
                                   (2000, 1, 8192), (9000, 16, 2048), (9000, 12, 64), (130, 64, 512), (15, 15, 15 * 8)])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_few_rows_or_outputs(dtype, m, n, k, act):
    check(m + n + k, m, n, k, dtype, act, residual=act == "gelu")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(1000, 1024, 2048), (2048, 1536, 512), (4000, 520, 264), (256, 256, 8200)])
def test_large(dtype, m, n, k):
    check(3, m, n, k, dtype, "relu")
    check(4, m, n, k, dtype, "gelu", residual=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(1000, 1001, 2049), (777, 401, 1027), (4001, 131, 513), (257, 255, 8199), (1500, 1300, 70)])
def test_large_and_odd(dtype, m, n, k):
    check(5, m, n, k, dtype, "none", bias=None)
    check(6, m, n, k, dtype, "gelu", residual=True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("wide", [1, 4, 8, 24])
@pytest.mark.parametrize("m", [5, 200])
def test_strides(dtype, wide, m):
    """Rows that are parts of wider ones, at odd strides and at multiples of 16 bytes."""
    check(5, m, 72, 136, dtype, "gelu", residual=True, wide=wide)


def test_bias_of_the_data_type():
    check(6, 200, 120, 64, BF16, "relu", bias=BF16)
    check(7, 9, 120, 64, BF16, "silu", bias=BF16)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_base_off_16_bytes(dtype):
    x, w, b, r, gy = make(8, 90, 40, 64, dtype, F32, False)
    flat = torch.empty(gy.numel() + 1, dtype=dtype, device="cuda")
    shifted = flat[1:].view(gy.shape).copy_(gy)
    got = rex.linear_act_bwd(shifted, x, w, None, bias=b)
    want = rex.linear_act_bwd(gy, x, w, None, bias=b)
    size = gy.double().abs() @ w.double().abs()
    within(got[0], want[0].double(), 2 * short(40) * size + HALF[dtype] * want[0].double().abs(), "grad_x")
    size = gy.double().abs().t() @ x.double().abs()
    within(got[1], want[1].double(), 2 * short(90) * size + HALF[dtype] * want[1].double().abs(), "grad_weight")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
def test_no_rows(dtype, act):
    x, w, b, r, gy = make(9, 0, 24, 40, dtype, F32, True)
    y, saved = rex.linear_act_fwd(x, w, b, act=act, residual=r, save=True)
    assert y.shape == (0, 24)
    gx, gw, gb = rex.linear_act_bwd(gy, x, w, saved, bias=b, act=act)
    assert gx.shape == (0, 40) and not gw.any() and not gb.any()


def test_what_lies_outside_has_no_effect():
    """NaN beside, behind and between the rows; padded outputs keep what they held."""
    for dtype in (F32, BF16):
        for m, n, k in ((70, 40, 72), (5, 40, 72), (300, 130, 520)):
            x, w, b, r, gy = make(10, m, n, k, dtype, F32, False)
            want = rex.linear_act_fwd(x, w, b)[0]
            full = lambda t: torch.full((t.shape[0] + 9, t.shape[1] + 16), math.nan, dtype=dtype, device="cuda")
            xs, wss = full(x), full(w)
            xs[:m, 8:8 + k], wss[:n, 8:8 + k] = x, w
            got = rex.linear_act_fwd(xs[:m, 8:8 + k], wss[:n, 8:8 + k], b)[0]
            assert torch.equal(got, want)
            gx, gw, _ = rex.linear_act_bwd(gy, x, w, None)
            gx2, gw2, _ = rex.linear_act_bwd(gy, xs[:m, 8:8 + k], wss[:n, 8:8 + k], None)
            assert torch.equal(gx, gx2) and torch.equal(gw, gw2)


def test_numbers_that_are_none():
    """A NaN or an infinity stays in its row, and relu lets NaN through."""
    for dtype in (F32, BF16):
        for m in (4, 100):
            x, w, b, r, gy = make(11, m, 32, 64, dtype, F32, False)
            x[2, 5] = math.nan
            for act in ("none", "relu", "gelu", "silu"):
                y = rex.linear_act_fwd(x, w, b, act=act)[0]
                assert bool(y[2].isnan().all()) and not bool(y[3].isnan().any()) and not bool(y[:2].isnan().any())
            w[7] = 0.0
            b[7] = 3e38
            y = rex.linear_act_fwd(x, w, b, act="gelu")[0]
            assert bool((y[3, 7].float() > 2.9e38))


def test_same_bits():
    for dtype in (F32, BF16):
        x, w, b, r, gy = make(12, 300, 200, 4096, dtype, F32, True)
        first = rex.linear_act_fwd(x, w, b, act="gelu", residual=r, save=True)
        grads = rex.linear_act_bwd(gy, x, w, first[1], bias=b, act="gelu")
        for _ in range(3):
            again = rex.linear_act_fwd(x, w, b, act="gelu", residual=r, save=True)
            assert all(torch.equal(p, q) for p, q in zip(first, again))
            assert all(torch.equal(p, q) for p, q in
                       zip(grads, rex.linear_act_bwd(gy, x, w, first[1], bias=b, act="gelu")))


def test_only_what_is_wanted():
    x, w, b, r, gy = make(13, 100, 64, 72, BF16, F32, False)
    y, saved = rex.linear_act_fwd(x, w, b, act="silu", save=True)
    full = rex.linear_act_bwd(gy, x, w, saved, bias=b, act="silu")
    for i in range(3):
        want = [j == i for j in range(3)]
        got = rex.linear_act_bwd(gy, x, w, saved, bias=b, act="silu", want_x=want[0], want_weight=want[1],
                                 want_bias=want[2])
        assert [t is not None for t in got] == want and torch.equal(got[i], full[i])


def test_buffers_and_streams():
    x, w, b, r, gy = make(14, 64, 40, 8192, BF16, F32, False)
    need = rex.linear_act_workspace_size(x, w, b)
    assert need > 0
    want = rex.linear_act_fwd(x, w, b)[0]
    ws, out = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty_like(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = rex.linear_act_fwd(x, w, b, out=out, workspace=ws, stream=side)[0]
    side.synchronize()
    assert got is out and torch.equal(out, want)
    with pytest.raises(rex.RoIExtractError):
        rex.linear_act_fwd(x, w, b, workspace=ws[:need - 256])


def test_graph_replays():
    for dtype in (F32, BF16):
        x, w, b, r, gy = make(15, 200, 96, 1024, dtype, F32, True)

        def step():
            y, saved = rex.linear_act_fwd(x, w, b, act="gelu", residual=r, save=True)
            return (y, *rex.linear_act_bwd(gy, x, w, saved, bias=b, act="gelu"))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step()
        for seed in range(3):
            x.copy_(make(20 + seed, 200, 96, 1024, dtype, F32, True)[0])
            want = step()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(held, want))
