"""What adds nothing to the weights of remembered boxes: rows whose log sum is not finite, rows past a
stream's count, and logits that are NaN, wherever the NaN or infinity comes from.

The reference and its tolerances are those of test_gpu_evict.py.
"""
import math

import numpy as np
import pytest
import torch

import paper_1906_07155_amd as rex
from test_gpu_evict import BF16, F32, U, check_weigh, fill, table

pytestmark = [pytest.mark.gpu, pytest.mark.filterwarnings("ignore:invalid value:RuntimeWarning")]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [32, 64])
@pytest.mark.parametrize("hkv,group", [(1, 1), (2, 1), (3, 2)])
@pytest.mark.parametrize("nq", [1, 2, 5, 16, 40])
def test_queries_that_are_nan_or_infinite(dtype, D, hkv, group, nq):
    """Key heads in numbers that are no multiple of those whose codes are on their way together."""
    def change(q, tab, bias, ql):
        q[0, 0] = math.nan
        q[1, nq - 1] = math.inf
        if nq > 2:
            q[1, 1, 0, 3] = -math.inf
    check_weigh(nq + D + hkv, 3, nq, hkv * group, hkv, D, dtype, 3, [96, 70, 33], change=change)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("poison", [math.nan, math.inf])
@pytest.mark.parametrize("heads,hkv", [(2, 2), (3, 1), (8, 2)])
@pytest.mark.parametrize("nq", [1, 2, 5, 16, 17, 40, 300])
def test_biases_that_are_nan_or_infinite(dtype, poison, heads, hkv, nq):
    """Every other row of the tables, and all of one head's: rows that meet one, and rows and columns that
    are none, add nothing."""
    def change(q, tab, bias, ql):
        bias[0, ::2] = poison
        bias[heads - 1] = poison
    check_weigh(nq, 3, nq, heads, hkv, 40, dtype, 3, [96, 50, 7], 7, q_len=[nq, (nq + 1) // 2, max(nq - 1, 0)], change=change)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("nq", [1, 4, 9, 33])
def test_a_nan_logit_of_a_finite_row(dtype, nq):
    """The log sum is of other keys: what is NaN adds nothing, the box's other heads do."""
    rng = np.random.default_rng(nq)
    m = fill(rng, 4, 2, 32)
    tab, lens = table(rng, 1, 3, 4), torch.tensor([90], dtype=torch.int32, device="cuda")
    q = torch.from_numpy(rng.standard_normal((1, nq, 2, 32)).astype(np.float32)).to(dtype).cuda()
    _, lse = rex.box_memory_attn_fwd(q, m, tab, lens, save=True)
    page = int(tab[0, 1])
    m[2][page, 1, 5] = math.nan                       # the scale of a key of the second head
    got = rex.box_memory_weigh(q, m, tab, lens, lse)[0].double().cpu().numpy()
    want, tol = np.zeros(96), np.zeros(96)
    for h in range(2):
        k = np.concatenate([m[0][p, h].double().cpu().numpy() * m[2][p, h].double().cpu().numpy()[:, None] for p in tab[0].tolist()])
        scale, x, l = float(np.float32(32 ** -0.5)), q[0, :, h].double().cpu().numpy(), lse[0, h].double().cpu().numpy()[:, None]
        s, size = scale * (x @ k.T), scale * (np.abs(x) @ np.abs(k).T)
        p = np.where(np.isnan(s), 0.0, np.exp(np.minimum(np.nan_to_num(s) - l, 0)))
        want += p.sum(0)
        off = U * ((8 + 2 * math.sqrt(32)) * size + 2 * np.abs(s) + 2 * np.abs(l) + 2 + 1.5 * np.abs(s - l))
        tol += np.where(np.isnan(s), 0.0, p * off).sum(0)
    want[90:] = tol[90:] = 0
    tol += U * (10 + 2 * math.sqrt(2 * nq)) * want
    assert (np.abs(got - want) <= tol).all()
