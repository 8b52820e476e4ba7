"""How many bits the attention's results have, whatever the size of a call.  The bounds are those of
test_gpu_relation_attn.py."""
import numpy as np
import pytest

import paper_1906_07155_amd as rex
import relation_oracle as O
from gpu_helpers import log
from test_gpu_relation_attn import Case, f64

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rex.lib()


@pytest.mark.parametrize("shape", [(2, 60, 90, 4, 2, 32, 15), (1, 40, 300, 4, 4, 64, 15)], ids=str)
def test_grad_q_where_few_of_many_keys_count(shape):
    """grad_q is a difference of two terms that nearly cancel where one or two keys have nearly all
    of a row's weight: the second one, sum_c grad_out * out, may not come from the rounded out."""
    log("precision grad_q %s" % (shape,))
    c = Case("bf16", *shape, k_len=[shape[2] - 9 * i for i in range(shape[0])], masked=0.2, seed=22)
    bias = c.geo["bias"]
    far = torch.ones(15, 15, dtype=torch.bool, device="cuda")
    far[5:10, 5:10] = False
    bias[:, far] = -40.0
    idx = np.stack([O.buckets(a, b, 15, -4, 1) for a, b in
                    zip(c.geo["q_boxes"].cpu().numpy(), c.geo["k_boxes"].cpu().numpy())])
    q, k, v, g = (f64(t) for t in (c.q, c.k, c.v, c.g))
    lens, mask = c.k_len.cpu().numpy(), c.mask.cpu().numpy()
    flat = f64(torch.where(far, torch.zeros_like(bias), bias)).reshape(bias.shape[0], -1)
    small = O.attn(q, k, v, c.scale, idx, flat, None, lens, mask)["logit"]
    c.ref = O.attn(q, k, v, c.scale, idx, f64(bias).reshape(bias.shape[0], -1), None, lens, mask, g)
    # rows without a near key have logits near -40, whose binary32 sums are 2^-24 of that off
    c.ref["logit"] = small + 40.0
    c.check(c.both(), "few of many")


def test_saved_results_are_there_for_any_number_of_keys():
    log("precision out_f32")
    for nk in (5, 64, 65, 500):
        c = Case("bf16", 1, 7, nk, 2, 2, 16, 3, seed=2)
        out, lse, full = c.fwd(save=True)
        assert full.dtype == torch.float32 and torch.equal(full.to(torch.bfloat16), out)
        assert c.fwd()[1] is None and c.fwd()[2] is None
        # without gradients nothing is kept for them
        with torch.no_grad():
            got, far = rex.box_attention(c.q, c.k, c.v, **c.args())
        assert not got.requires_grad and torch.allclose(far, lse, rtol=1e-6, atol=1e-6)
        q = c.q.clone().requires_grad_()
        rex.box_attention(q, c.k, c.v, **c.args())[0].backward(c.g)
        assert torch.equal(q.grad, c.both()["grad_q"])
