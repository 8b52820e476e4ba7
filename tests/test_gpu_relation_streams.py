"""Calls on a given stream: what they allocate is not memory that the current stream has just given
back, which kernels enqueued there may still be using."""
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


def given_back(like):
    """Addresses of blocks of these tensors' sizes that the current stream gives back."""
    blocks = [torch.empty_like(t) for t in like for _ in range(4)]
    found = {t.data_ptr() for t in blocks}
    del blocks
    return found


def test_results_on_another_stream_have_memory_of_their_own():
    log("streams memory")
    c = Case("bf16", 2, 40, 50, 4, 2, 32, 7)
    m = rex.box_memory(4, 2, 32)
    slots = torch.arange(64, device="cuda")
    rex.box_memory_append(m, slots, torch.randn(64, 2, 32, device="cuda"), torch.randn(64, 2, 32, device="cuda"),
                          torch.rand(64, 4, device="cuda"))
    pages, lengths = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2), torch.tensor([64, 5], dtype=torch.int32, device="cuda")
    x, gate = torch.randn(64, 96, device="cuda"), torch.randn(4, 96, device="cuda")
    w = torch.ones(96, device="cuda")
    norm = dict(gate=gate, post_weight=w, pre_weight=w)
    out, lse, full = c.fwd(save=True)
    y, u, stats = rex.gated_norm_fwd(x, x, save=True, **norm)
    calls = [lambda **kw: c.fwd(save=True, **kw),
             lambda **kw: rex.box_attn_bwd(c.g, c.q, c.k, c.v, out, lse, full, **c.args(), **kw),
             lambda **kw: rex.box_memory_read(m, slots, **kw),
             lambda **kw: rex.box_memory_attn_fwd(c.q, m, pages, lengths, save=True, **kw),
             lambda **kw: rex.gated_norm_fwd(x, x, save=True, **norm, **kw),
             lambda **kw: [t for t in rex.gated_norm_bwd(y, u, x, x, stats, **norm, **kw) if t is not None]]
    other = torch.cuda.Stream()
    for i, call in enumerate(calls):
        want = [t.clone() for t in call()]
        torch.cuda.synchronize()
        freed = given_back(want)
        got = call(stream=other)
        assert not freed & {t.data_ptr() for t in got}, i
        torch.cuda.current_stream().wait_stream(other)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
