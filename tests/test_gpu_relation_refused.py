"""What a call that fails leaves behind: the memory's table, its free pages and what it holds stay as they
were, so that the next frame does not attend to places that were never written."""
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


def state(m):
    return ([list(p) for p in m.table], list(m.used), list(m.free)), [t.clone() for layer in m.layers for t in layer]


def same(a, b):
    return a[0] == b[0] and all(torch.equal(x, y) for x, y in zip(a[1], b[1]))


def test_a_call_that_fails_changes_nothing():
    log("refused memory")
    rng = np.random.default_rng(3)
    head = make(2, 2)
    memory = head.memory(num_pages=7, streams=2, max_pages=3)
    frame = lambda: (torch.from_numpy(rng.standard_normal((2, 40, 64)).astype(np.float32)).cuda(),
                     torch.from_numpy(draw_boxes(rng, (2, 40))).cuda())
    with torch.no_grad():
        for _ in range(3):                          # the oldest pages have been given back already
            head(*frame(), [40, 33], memory)
        before = state(memory)
        x, boxes = frame()
        other = make(2, 4).memory(num_pages=7, streams=2, max_pages=3)
        calls = [lambda: head(x, boxes.double(), [40, 33], memory),
                 lambda: head(x, boxes[:, :39], [40, 33], memory),
                 lambda: head(x, boxes.cpu(), [40, 33], memory),
                 lambda: head(x.double(), boxes, [40, 33], memory),
                 lambda: head(x[..., :63], boxes, [40, 33], memory),
                 lambda: head(x, boxes, [40], memory),
                 lambda: head(x, boxes, [40, 41], memory),
                 lambda: head(x.repeat(1, 2, 1), boxes.repeat(1, 2, 1), [80, 3], memory),
                 lambda: make(1, 2)(x, boxes, [40, 33], memory),
                 lambda: head(x, boxes, [40, 33], other)]
        for i, call in enumerate(calls):
            with pytest.raises((ValueError, TypeError, RuntimeError)):
                call()
            assert same(state(memory), before), i
        assert other.used == [0, 0] and len(other.free) == 7

        # a failure in the second layer, after the first has recalled
        def fail(*args):
            raise MemoryError("second layer")
        kept, head.layers[1].forward = head.layers[1].forward, fail
        with pytest.raises(MemoryError):
            head(x, boxes, [40, 33], memory)
        assert same(state(memory), before)
        head.layers[1].forward = kept

        small = head.memory(num_pages=3, streams=2, max_pages=3)
        head(x, boxes, [40, 20], small)
        before = state(small)
        with pytest.raises(RuntimeError, match="free pages"):
            head(x, boxes, [40, 20], small)
        assert same(state(small), before)
