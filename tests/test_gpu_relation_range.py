"""The attention over the whole range of biases and logits: rows whose visible keys all carry one
large offset (a mask written as -1e9, say) have the weights that they have without it.

A softmax does not change when a row's logits are moved by one number, so the oracle is given the
table less its offset, and the bounds are those of test_gpu_relation_attn.py for the logits that are
left.  Differences of two entries are exact in the oracle and in binary32 alike: both are numbers of
the table, and those of one row here lie within a factor of two of each other.  `lse` is the
offset and what is left, rounded once more to binary32.
"""
import numpy as np
import pytest

import paper_1906_07155_amd as rex
import relation_oracle as O
from gpu_helpers import log
from test_gpu_relation_attn import Case, f64
from test_gpu_relation_memory import Recall

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rex.lib()


# (binary32 numbers, so that taking them off a table is exact)
OFFSETS = [float(np.float32(x)) for x in (-300.0, -1e5, -1e7, -1e9, -1e15, -9e29, 300.0, 1e5, 1e9, 1e29)]


def oracle(c, bias, idx, lens=None, keep=None):
    """The reference for a table (64 bits) that stands for the one on the GPU."""
    q, k, v, g = (f64(t) for t in (c.q, c.k, c.v, c.g))
    return O.attn(q, k, v, c.scale, idx, bias, None, lens, keep, g)


def buckets(c):
    qb, kb = (c.geo[n].cpu().numpy() for n in ("q_boxes", "k_boxes"))
    return np.stack([O.buckets(a, b, c.nb, -4, 1) for a, b in zip(qb, kb)])


def check(c, got, offset, name):
    """As Case.check, with lse compared as offset + what the oracle has."""
    lse = f64(got.pop("lse"))
    c.check(got, name)
    want = c.ref["lse"] + offset
    assert np.array_equal(np.isfinite(lse), np.isfinite(want)), name
    fin = np.isfinite(want)
    e = 2 * (c.D + 8) * 2.0 ** -24 * max(c.ref["logit"], 1.0) + 2.0 ** -20
    assert np.all(np.abs(lse - want)[fin] <= 2 * e + 2.0 ** -22 * np.abs(want[fin])), name


@pytest.mark.parametrize("offset", OFFSETS)
@pytest.mark.parametrize("dtype,shape", [("f32", (1, 70, 45, 4, 2, 32, 7)), ("bf16", (1, 70, 45, 4, 2, 32, 7)),
                                         ("bf16", (1, 40, 200, 8, 8, 64, 15)), ("f32", (2, 20, 130, 2, 1, 128, 7)),
                                         ("bf16", (1, 1, 900, 8, 8, 64, 15)), ("bf16", (1, 33, 70, 2, 2, 96, 7))], ids=str)
def test_rows_that_are_all_at_one_offset(dtype, shape, offset):
    log("range %s %s %g" % (dtype, shape, offset))
    c = Case(dtype, *shape, seed=21)
    step = max(float(np.spacing(np.float32(abs(offset)))), 2.0 ** -10)
    bias = c.geo["bias"]
    # steps of whole spacings near the offset: every entry is a binary32 number, one head is flat
    near = torch.round(bias / step).clamp(-3, 3) * step
    near[0] = 0.0
    bias.copy_(near.double() + offset)
    left = f64(bias) - offset
    c.ref = oracle(c, left.reshape(bias.shape[0], -1), buckets(c))
    if step > 1e3:
        # entries that differ do so by a thousand and more: the weights of all but the largest are 0,
        # and those of one entry are told apart by the products alone
        c.ref["logit"] = oracle(c, np.zeros((bias.shape[0], c.nb ** 2)), buckets(c))["logit"]
    check(c, c.both(), offset, "%g" % offset)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [-1e4, -1e6, -1e9])
def test_rows_with_and_without_keys_near_by(dtype, offset):
    """Buckets far away are masked by a large number: rows with a near key see the near ones, rows
    without one see all of theirs, masked keys count for neither."""
    log("range mixed %s %g" % (dtype, offset))
    c = Case(dtype, 2, 60, 90, 4, 2, 32, 15, k_len=[90, 61], masked=0.2, seed=22)
    bias = c.geo["bias"]
    far = torch.ones(15, 15, dtype=torch.bool, device="cuda")
    far[5:10, 5:10] = False
    bias[:, far] = offset
    idx = buckets(c)
    keep = c.mask.cpu().numpy()
    ref = oracle(c, f64(bias).reshape(4, -1), idx, [90, 61], keep)
    flat = f64(torch.where(far, torch.zeros_like(bias), bias)).reshape(4, -1)
    ref["logit"] = oracle(c, flat, idx, [90, 61], keep)["logit"]
    c.ref = ref
    near = (~far).cpu().numpy().reshape(-1)[idx] & keep[:, None, :]
    near[1, :, 61:] = False
    assert near.any(-1).any() and not near.any(-1).all()
    # 64-bit logits of -1e9 are 2^-24 apart: nothing beside the bounds
    check(c, c.both(), 0.0, "mixed")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", OFFSETS)
def test_memory_whose_boxes_are_all_at_one_offset(dtype, offset):
    log("range memory %s %g" % (dtype, offset))
    for shape in ((2, 1, 700, 8, 2, 32, 7), (1, 40, 300, 4, 4, 64, 7)):
        r = Recall(dtype, *shape, seed=23)
        r.geo["bias"].fill_(offset)
        r.bias[:] = 0.0
        got, lse = r.run(save=True)
        r.check(got, None, "%g" % offset)
        ref = O.attn(f64(r.q), r.k, r.v, r.D ** -0.5, r.idx, r.bias, None, r.lengths)
        e = 2 * (r.D + 8) * 2.0 ** -24 * max(ref["logit"], 1.0) + 2.0 ** -20 + (r.k.shape[1] + 64) * 2.0 ** -24
        want = ref["lse"] + offset
        assert np.all(np.abs(f64(lse) - want) <= 2 * e + 2.0 ** -22 * np.abs(want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nb", [0, 7])
def test_logits_that_are_large_by_themselves(dtype, nb):
    """Queries and keys of 1e5 and 1e8: the largest logit takes everything; its weight is 1, and what
    follows from a weight of 1 is right."""
    log("range logits %s %d" % (dtype, nb))
    for size in (1e3, 1e5, 1e8):
        c = Case(dtype, 1, 50, 66, 4, 2, 32, nb, seed=24)
        c.q.mul_(size)
        c.k.mul_(size)
        bias = f64(c.geo["bias"]).reshape(4, -1) if nb else None
        ref = oracle(c, bias, buckets(c) if nb else None)
        got = c.both()
        s = np.einsum("bqhd,bkhd->bhqk", f64(c.q), np.repeat(f64(c.k), 2, 2)) * c.scale
        if nb:
            s = s + bias[:, buckets(c)].transpose(1, 0, 2, 3)
        top = np.sort(s, -1)
        # rows whose largest logit leads by more than binary32 sums of this size can be off
        sure = top[..., -1] - top[..., -2] > 2 * (c.D + 8) * 2.0 ** -24 * ref["logit"] + 30.0
        assert sure.mean() > 0.9
        rows = sure.transpose(0, 2, 1)
        low = 2.0 ** -7 if dtype == "bf16" else 1e-5
        assert np.isfinite(f64(got["out"])).all()
        assert np.all(np.abs(f64(got["out"]) - ref["out"])[rows] <= low * ref["out_abs"][rows] + 1e-6)
        lse = f64(got["lse"])
        assert np.all(np.abs(lse - ref["lse"])[sure] <= 2 * (c.D + 8) * 2.0 ** -24 * ref["logit"] + 1e-5 * np.abs(ref["lse"][sure]))
        # grad_v: every sure row adds its whole upstream gradient to one key's
        assert all(np.isfinite(f64(got[k])).all() for k in got if got[k] is not None and k != "lse")
        if sure.all():
            assert np.all(np.abs(f64(got["grad_v"]) - ref["grad_v"]) <= (low + 50 * 2.0 ** -8 * (dtype == "bf16")) * ref["grad_v_abs"] + 1e-5)


def test_the_smallest_scales():
    """Logits that are their biases: scales of 1e-8 and 1e-20, biases of ordinary size and large."""
    log("range scale")
    for scale in (1e-8, 1e-20):
        for offset in (0.0, -1e3, -1e9, OFFSETS[5]):
            c = Case("f32", 1, 30, 50, 2, 2, 16, 5, scale=scale, seed=25)
            bias = c.geo["bias"]
            step = max(float(np.spacing(np.float32(abs(offset)))), 2.0 ** -10) if offset else 2.0 ** -10
            bias.copy_((torch.round(bias / step).clamp(-2000, 2000) * step).double() + offset)
            c.ref = oracle(c, (f64(bias) - offset).reshape(2, -1), buckets(c))
            # grad_q and grad_k carry the scale: held against what their terms add up to
            got = c.both()
            assert float(got["grad_bias"].abs().max()) > 0.0
            e = 2 * (c.D + 8) * 2.0 ** -24 * max(c.ref["logit"] if step < 1 else 1.0, 1.0) + 2.0 ** -20
            for key in ("out", "grad_q", "grad_k", "grad_v", "grad_bias"):
                have, ref = f64(got[key]).reshape(c.ref[key].shape), c.ref[key]
                assert np.isfinite(have).all(), (scale, offset, key)
                assert np.all(np.abs(have - ref) <= (e + 150 * 2.0 ** -24) * c.ref[key + "_big"] + 1e-37), (scale, offset, key)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_of_one_image_leave_the_others_alone(dtype):
    """Results of rows that see no large bias are the bits they are in a call of their own."""
    log("range alone %s" % dtype)
    c = Case(dtype, 1, 64, 80, 4, 4, 32, 7, seed=26)
    bias = c.geo["bias"]
    for h in (1, 3):
        bias[h] = -1e9
    got = c.both()
    c.geo["bias"] = torch.where(bias < -1e8, torch.zeros_like(bias), bias)
    want = c.both()
    for k in ("out", "grad_q", "grad_k", "grad_v"):
        for h in (0, 2):
            assert torch.equal(got[k][:, :, h], want[k][:, :, h]), k
