"""Log probabilities of classes, entropy, top classes and the gradient against the definition in
64 bits.

Tolerances, with u = 2^-23 and d_c = x_c - max x: x is rounded once (u/2 |x|, nothing with scale 1), d
once; a term of the sum has the relative error of its exponent's argument and of exp2, u (2 + 1.5 |d|);
sums of terms of one sign over up to 2^12 registers and lanes stay below 8 u.  So the log sum is off by
u (16 + sum p (2 |d| + |x|)), the entropy's second sum by the same times |d|, and a result by half a
step of its type more.
"""
import math

import pytest
import torch

import paper_1906_07155_amd as rex

pytestmark = pytest.mark.gpu

U = 2.0 ** -23
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
F32, BF16 = torch.float32, torch.bfloat16


def make(seed, m, c, dtype, wide=0, spread=2.0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = (torch.randn((m, c + wide), generator=gen, device="cuda") * spread).to(dtype)[:, :c]
    labels = torch.randint(0, c, (m,), generator=gen, device="cuda")
    return x, labels, torch.randn((m,), generator=gen, device="cuda"), torch.randn((m,), generator=gen, device="cuda")


def within(got, want, tolerance, what):
    got = got.double()
    same = (got == want) | (got.isnan() & want.isnan())
    bad = ~same & ~((got - want).abs() <= tolerance)
    assert not bad.any(), "%s: %d of %d, first %s: got %s want %s" % (
        what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), got[bad][0].item(), want[bad][0].item())


def check(x, labels, gl, gh, scale=1.0, top=0):
    m, c = x.shape
    logp, entropy, stats, top_logp, top_index = rex.class_logprob_fwd(x, labels, scale=scale, top=top)
    f32 = lambda v: torch.tensor(v, dtype=torch.float32).double().item()
    fin = lambda t: torch.where(t.isfinite(), t, torch.zeros_like(t))
    xs = x.double() * f32(scale)
    largest = xs.amax(-1)
    dead = largest == -math.inf
    d = xs - torch.where(dead, torch.zeros_like(largest), largest)[:, None]
    log_sum = torch.where(dead, torch.zeros_like(largest), d.exp().sum(-1).log())     # (NaN with +inf)
    logs = d - log_sum[:, None]
    p = logs.exp()
    far, ax = fin(d).abs(), fin(xs).abs() * (scale != 1.0)
    want_h = torch.where(log_sum.isnan(), log_sum, -fin(p * fin(logs)).sum(-1))
    part = lambda t: torch.where(p == 0, torch.zeros_like(t), p * t).sum(-1)
    tol_log = U * (16 + part(2 * far + ax))
    tol_h = U * (16 + part((1 + far) * (4 * far + ax)) + want_h)
    x_tol = U * fin(largest).abs() * (scale != 1.0)
    nan = log_sum.isnan()
    within(stats[:, 0][~nan], largest[~nan], x_tol[~nan], "largest")
    within(stats[:, 1], log_sum, tol_log, "log sum")
    within(entropy, want_h, tol_h, "entropy")
    counted = (labels >= 0) & (labels < c)
    at = torch.where(counted, labels, torch.zeros_like(labels))
    want = logs.gather(1, at[:, None])[:, 0]
    want = torch.where(counted, want, torch.zeros_like(want))
    log_tol = tol_log[:, None] + U * (2 * ax + far + fin(logs).abs())
    within(logp, want, log_tol.gather(1, at[:, None])[:, 0], "logp")
    if top:
        key = torch.where(x.isnan(), torch.full_like(xs, math.inf), x.double())
        key, odd = key.cpu(), x.isnan().cpu()
        for i in range(min(m, 64)):
            order = sorted(range(c), key=lambda j: (not bool(odd[i, j]), -float(key[i, j]), j))[:top]
            assert top_index[i].tolist() == order, (i, top_index[i].tolist(), order)
        within(top_logp, logs.gather(1, top_index), log_tol.gather(1, top_index), "top_logp")
    grad = rex.class_logprob_bwd(gl, gh, x, labels, stats, entropy, scale=scale)
    zero = torch.zeros_like(log_sum)
    g_l = zero if gl is None else torch.where(counted, gl.double(), zero)
    g_h = zero if gh is None else gh.double()
    inner = g_l[:, None] + g_h[:, None] * (fin(logs) + want_h[:, None])
    inner = torch.where(p == 0, torch.zeros_like(inner), inner)
    hot = torch.zeros_like(p).scatter_(1, at[:, None], g_l[:, None])
    g = f32(scale) * (hot - p * inner)
    size = g_l[:, None].abs() + g_h[:, None].abs() * (fin(logs).abs() + want_h[:, None])
    tol = p * (size * (U * (6 + 2 * fin(logs).abs()) + log_tol) + g_h[:, None].abs() * (log_tol + tol_h[:, None]))
    # (a probability below the smallest normal number, 2^-126, may be taken as 0)
    tol = torch.where(p == 0, torch.zeros_like(tol), tol) + 2.0 ** -126 * size
    tol = f32(scale) * (tol + 2 * U * hot.abs())
    g = torch.where(dead[:, None], torch.zeros_like(g), g)
    g = torch.where(nan[:, None], log_sum[:, None].expand_as(g), g)
    within(grad, g, tol + HALF[x.dtype] * g.abs() + 1e-37, "grad")
    assert grad.dtype == x.dtype and grad.is_contiguous()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,c", [(1, 1), (3, 2), (100, 81), (17, 64), (9, 127), (33, 128), (5, 129), (20, 513), (7, 1025),
                                 (64, 1231), (3, 2047), (3, 2049), (2, 4088), (3, 4089), (2, 4096), (5, 4097), (2, 8192), (3, 100003), (1, 300001)])
def test_sizes(dtype, m, c):
    x, labels, gl, gh = make(m + c, m, c, dtype)
    check(x, labels, gl, gh, top=min(c, 5))
    check(x, labels, gl, None, scale=0.7)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("c", [16, 81, 700, 1500, 5000])
def test_most_alternatives(dtype, c):
    """Sixteen of them, with many ties: the lower class first."""
    x, labels, gl, gh = make(c, 12, c, dtype)
    check((x * 2).round() / 2, labels, gl, gh, top=16)
    check(torch.zeros_like(x), labels, gl, gh, top=16)
    signed = torch.zeros_like(x)
    signed[:, ::2] = -0.0
    check(signed, labels, gl, gh, top=16)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("wide", [1, 3, 8])
@pytest.mark.parametrize("c", [81, 1000, 4500])
def test_strides(dtype, wide, c):
    x, labels, gl, gh = make(wide, 10, c, dtype, wide)
    check(x, labels, gl, gh, top=3)
    full = x._base if x._base is not None else x
    check(full[:, wide:], labels, gl, gh, top=3)            # bases off their alignment too


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("c", [7, 81, 1231, 9000])
def test_masks(dtype, c):
    x, labels, gl, gh = make(c, 12, c, dtype)
    x[0] = -math.inf                                        # nothing is left
    x[1, 1:] = -math.inf                                    # one class, which is not the label
    labels[1] = 2
    x[2, :3] = -math.inf
    x[3] = torch.finfo(dtype).min                           # masks of the type's lowest value
    x[4, 1:] = torch.finfo(dtype).min
    x[5] = -1e9
    x[5, 2] = -1e9 + 1024
    labels[6], labels[7], labels[8] = -1, c, -(2 ** 40)     # not counted
    x[9, 3] = math.nan
    x[10, 4] = math.inf
    check(x, labels, gl, gh, top=min(c, 5))
    assert not rex.class_logprob_bwd(gl, gh, x, labels, *rex.class_logprob_fwd(x, labels)[2:0:-1])[0].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("c", [1, 81, 1231, 9000])
def test_rows_of_nothing_but_nan(dtype, c):
    x, labels, gl, gh = make(c, 8, c, dtype)
    x[0] = math.nan
    x[1, :-1] = -math.inf                                   # and one NaN
    x[1, -1] = math.nan
    x[2] = math.inf
    x[3, :-1] = -math.inf
    x[3, -1] = math.inf
    labels[4] = -1
    x[4] = math.nan
    check(x, labels, gl, gh, top=min(c, 5))
    logp, entropy, stats, _, _ = rex.class_logprob_fwd(x, labels)
    assert logp[:4].isnan().all() and float(logp[4]) == 0.0 and entropy[:5].isnan().all() and stats[:5].sum(1).isnan().all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_logits(dtype):
    for spread in (50.0, 1000.0, 1e30):
        x, labels, gl, gh = make(5, 30, 333, dtype, spread=spread)
        check(x, labels, gl, gh, top=4)


def test_no_rows():
    x, labels, gl, gh = make(1, 0, 81, F32)
    logp, entropy, stats, top_logp, top_index = rex.class_logprob_fwd(x, labels, top=5)
    assert logp.shape == (0,) and top_index.shape == (0, 5)
    assert rex.class_logprob_bwd(gl, gh, x, labels, stats, entropy).shape == (0, 81)


def test_upstream_gradients_left_out():
    x, labels, gl, gh = make(2, 20, 300, F32)
    check(x, labels, None, gh)
    check(x, labels, gl, None)
    check(x, labels, None, None)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradient_against_differences(dtype):
    """Central differences of the results themselves, in binary32 for both types' values."""
    x, labels, gl, gh = make(3, 1, 40, dtype, spread=1.0)
    def value(z):
        logp, entropy, *_ = rex.class_logprob_fwd(z, labels.expand(z.shape[0]).contiguous())
        return gl.double() * logp.double() + gh.double() * entropy.double()
    _, entropy, stats, _, _ = rex.class_logprob_fwd(x, labels)
    grad = rex.class_logprob_bwd(gl, gh, x, labels, stats, entropy)[0].double()
    step = 2.0 ** -6
    eye = torch.eye(40, device="cuda") * step
    up, down = value((x.float() + eye).contiguous()), value((x.float() - eye).contiguous())
    # results off by 32 u at most, third derivatives below 8: both of (|gl| + |gh|)
    size = float(gl.abs() + gh.abs())
    tol = size * (32 * U / step + 8 * step * step) + HALF[dtype] * grad.abs()
    assert bool(((up - down) / (2 * step) - grad).abs().le(tol).all())


def test_same_bits_streams_graphs():
    for c in (81, 1231, 20000):
        x, labels, gl, gh = make(c, 50, c, BF16)
        def step():
            out = rex.class_logprob_fwd(x, labels, top=3)
            return (*out, rex.class_logprob_bwd(gl, gh, x, labels, out[2], out[1]))
        want = step()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = rex.class_logprob_fwd(x, labels, top=3, stream=side)
        with torch.cuda.stream(side):
            step()
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step()
        for seed in range(3):
            x.copy_(make(seed, 50, c, BF16)[0])
            want = step()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(held, want))
