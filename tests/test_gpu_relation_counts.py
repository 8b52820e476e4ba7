"""The numbers of boxes that RelationHead is given: tensors, and no images at all."""
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


def test_counts_on_the_device_are_read_at_once(monkeypatch):
    log("counts device")
    rng = np.random.default_rng(1)
    head = make(1)
    boxes = torch.from_numpy(draw_boxes(rng, (3, 20))).cuda()
    x = torch.randn(3, 20, 64, device="cuda")
    counts = torch.tensor([20, 0, 7], dtype=torch.int32, device="cuda")
    with torch.no_grad():
        want = head(x, boxes, [20, 0, 7])

        def one_by_one(self):
            raise AssertionError("a tensor read element by element")
        monkeypatch.setattr(torch.Tensor, "__iter__", one_by_one)
        assert torch.equal(head(x, boxes, counts), want)
        with pytest.raises(ValueError, match="counts"):
            head(x, boxes, counts + 1)
