"""What rows past an image's count hold has no effect on the head's results and gradients."""
import numpy as np
import pytest

import paper_1906_07155_amd as rex
from gpu_helpers import log
from test_gpu_relation_attn import draw_boxes
from test_gpu_relation_head import make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rex.lib()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_padding_reaches_no_gradient(dtype, norm):
    log("padding %s %s" % (dtype, norm))
    rng = np.random.default_rng(6)
    counts, n = [33, 0, 50, 7], 50
    boxes = torch.from_numpy(draw_boxes(rng, (4, n))).cuda()
    x = torch.from_numpy(rng.standard_normal((4, n, 64))).to(dtype).cuda()
    g = torch.from_numpy(rng.standard_normal((4, n, 64))).to(dtype).cuda()
    pad = torch.arange(n)[None] >= torch.tensor(counts)[:, None]
    found = []
    for fill in (0.0, 3.0, float("nan"), float("inf")):
        head = make(2, 2, norm).to(dtype)
        xi, bi = x.clone(), boxes.clone()
        xi[pad.cuda()] = fill
        bi[pad.cuda()] = fill
        xi.requires_grad_()
        y = head(xi, bi, counts)
        (y * g).sum().backward()                # the padding's upstream gradient is no less than the others'
        assert float(y[pad.cuda()].abs().max()) == 0.0 and float(xi.grad[pad.cuda()].abs().max()) == 0.0
        found.append((fill, y.detach(), {"x": xi.grad, **{k: p.grad for k, p in head.named_parameters()}}))
    _, y0, grads0 = found[0]
    assert all(bool(torch.isfinite(t).all()) for t in grads0.values())
    for fill, y, grads in found[1:]:
        assert torch.equal(y, y0), fill
        for k in grads0:
            assert torch.equal(grads[k], grads0[k]), (fill, k)
