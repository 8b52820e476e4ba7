"""Box attention with heads that share few keys: a key's gradients go over the heads with few products
between two of them.  Each result against 64 bits, and the same bits at every call."""
import pytest

import paper_1906_07155_amd as rex
from gpu_helpers import log
from test_gpu_relation_attn import Case

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rex.lib()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [8, 32, 40, 64, 128])
@pytest.mark.parametrize("shape", [(1, 304, 3, 32, 8, 7), (2, 97, 16, 12, 2, 5), (1, 64, 1, 8, 8, 3), (1, 130, 17, 16, 4, 5),
                                   (2, 33, 40, 6, 3, 0)], ids=str)
def test_few_keys_many_heads(dtype, D, shape):
    B, nq, nk, H, hkv, nb = shape
    log("shared %s D%d %s" % (dtype, D, shape))
    c = Case(dtype, B, nq, nk, H, hkv, D, nb, seed=21)
    first = c.both()
    c.check(first, "shared")
    for _ in range(3):
        again = c.both()
        for key, x in first.items():
            assert again[key] is x is None or torch.equal(again[key], x), key
