"""The dense layers' results where whatever they allocate, results and workspaces, is NaN beforehand, and no NaN passes
for a number: an element that a kernel leaves out, or a sum that takes in what nobody wrote, is found.

The checks and their tolerances are those of test_gpu_linear.py, in which a NaN result would compare as within
any tolerance; the cases reach each of its kernels: few rows and few outputs, whole and in parts, tiles of every
size, of whole chunks and through registers, whole and in parts, and what joins the parts.
"""
import contextlib

import pytest
import torch

import paper_1906_07155_amd as rex
import test_gpu_linear as T

pytestmark = pytest.mark.gpu
F32, BF16 = T.F32, T.BF16


def within(got, want, tolerance, what):
    err = (got.double() - want).abs()
    tolerance = tolerance + T.HALF[got.dtype] * want.abs() + 1e-38
    bad = ~(err <= tolerance)
    assert not bad.any(), "%s: %d of %d, %d of them NaN" % (what, int(bad.sum()), bad.numel(), int(got.isnan().sum()))


@contextlib.contextmanager
def filled():
    """New tensors hold NaN (bytes: 255, NaN in every type)."""
    assert torch.utils.deterministic.fill_uninitialized_memory
    before = torch.are_deterministic_algorithms_enabled()
    torch.use_deterministic_algorithms(True)
    try:
        assert bool(torch.empty(8, device="cuda").isnan().all()) and int(torch.empty(8, dtype=torch.uint8, device="cuda").min()) == 255
        yield
    finally:
        torch.use_deterministic_algorithms(before)


@pytest.fixture(autouse=True)
def strict(monkeypatch):
    def wrap(f):
        def call(*args, **kw):
            with filled():
                return f(*args, **kw)
        return call
    monkeypatch.setattr(T, "within", within)
    for name in ("linear_act_fwd", "linear_act_bwd"):
        monkeypatch.setattr(rex, name, wrap(getattr(rex, name)))


def test_nan_is_no_number():
    with pytest.raises(AssertionError, match="1 of them NaN"):
        within(torch.tensor([1.0, float("nan")]), torch.ones(2, dtype=torch.float64), 1.0, "y")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [
    (1, 1, 1), (1, 1024, 1024), (17, 40, 1024), (64, 300, 512), (16, 40, 8192), (64, 24, 12544),      # few rows
    (1001, 5, 264), (400, 33, 256), (300, 16, 4104), (2000, 1, 8192), (9000, 12, 64),                 # few outputs
    (70, 48, 96), (300, 81, 1024), (1000, 1024, 2048), (2048, 1536, 512), (4000, 520, 264),           # whole chunks
    (256, 256, 8200), (4096, 4096, 512),
    (3, 77, 250), (129, 257, 31), (513, 77, 250), (777, 401, 1027), (4001, 131, 513), (257, 255, 8199),   # through registers
    (1500, 1300, 70), (2100, 2050, 130)])
@pytest.mark.parametrize("act,bias,residual", [("none", None, False), ("gelu", F32, True), ("relu", F32, False)])
def test_every_element_is_written(dtype, m, n, k, act, bias, residual):
    T.check(m + 3 * n + k, m, n, k, dtype, act, bias=bias, residual=residual)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("wide", [1, 8])
@pytest.mark.parametrize("m,n,k", [(5, 72, 136), (200, 72, 136), (700, 300, 264)])
def test_rows_that_are_parts_of_wider_ones(dtype, wide, m, n, k):
    T.check(wide, m, n, k, dtype, "silu", residual=True, wide=wide)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_no_rows(dtype):
    x, w, b, r, gy = T.make(9, 0, 24, 40, dtype, F32, False)
    gx, gw, gb = rex.linear_act_bwd(gy, x, w, None, bias=b)
    assert gx.shape == (0, 40) and bool((gw == 0).all()) and bool((gb == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(5, 72, 136), (16, 40, 8192), (9000, 12, 64), (300, 81, 1024), (1000, 1024, 2048), (513, 77, 250),
                                   (257, 255, 8199)])
def test_a_residual_that_is_written_to(dtype, m, n, k):
    x, w, b, r, _ = T.make(m, m, n, k, dtype, F32, True)
    want = rex.linear_act_fwd(x, w, b, act="gelu", residual=r)[0]
    got = rex.linear_act_fwd(x, w, b, act="gelu", residual=r, out=r)[0]
    assert got is r and torch.equal(got, want)
