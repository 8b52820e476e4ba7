"""Calls with many boxes that workgroups share out by pages, at 128 pages and more, and memories of so
few pages that each box goes by itself."""
import numpy as np
import pytest

import paper_1906_07155_amd as rex
import relation_oracle as O
from gpu_helpers import log
from test_gpu_relation_attn import draw_boxes

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rex.lib()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pages,hkv,D,n", [(128, 16, 128, 4096),     # every page full
                                           (127, 24, 96, 4000),      # one page too few
                                           (130, 72, 40, 3000), (600, 30, 64, 5000)])
def test_both_forms_write_and_read_the_same(dt, pages, hkv, D, n):
    log("pages %d %d %d %d" % (pages, hkv, D, n))
    assert n * hkv * D >= 1 << 23 and n >= 4 * pages
    rng = np.random.default_rng(n)
    make = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(dt).cuda()
    k, v = make(n, hkv, D), make(n, hkv, D)
    boxes = torch.from_numpy(draw_boxes(rng, (n,))).cuda()
    m = rex.box_memory(pages, hkv, D)
    for t in m:
        t.fill_(7)
    want = [t.cpu().numpy().copy() for t in m]
    slots = rng.permutation(pages * 32)[:n].astype(np.int64)
    rex.box_memory_append(m, torch.from_numpy(slots).cuda(), k, v, boxes)
    p, at = slots // 32, slots % 32
    (kc, ks), (vc, vs) = O.encode(k.float().cpu().numpy()), O.encode(v.float().cpu().numpy())
    want[0][p, :, at], want[2][p, :, at], want[1][p, :, :, at], want[3][p, :, at] = kc, ks, vc, vs
    want[4][p, at] = boxes.cpu().numpy()
    for got, w in zip(m, want):
        assert np.array_equal(got.cpu().numpy(), w)
    # all of it, and as often again two slots of one page and two outside: more than a list holds
    ask = np.concatenate([slots, rng.choice([int(slots[0]), int(slots[0]) // 32 * 32, -1, pages * 32], 2 * n, p=[0.6, 0.2, 0.1, 0.1])])
    there = (ask >= 0) & (ask < pages * 32)
    p, at = np.where(there, ask, 0) // 32, np.where(there, ask, 0) % 32
    gk, gv, gb = rex.box_memory_read(m, torch.from_numpy(ask).cuda(), dt)
    product = lambda code, scale: torch.from_numpy(np.where(
        there[:, None, None], code.astype(np.float32) * scale[..., None], np.float32(0))).to(dt)
    assert torch.equal(gk.cpu(), product(want[0][p, :, at], want[2][p, :, at]))
    assert torch.equal(gv.cpu(), product(want[1][p, :, :, at], want[3][p, :, at]))
    assert np.array_equal(gb.cpu().numpy(), np.where(there[:, None], want[4][p, at], np.float32(0)))


def test_reading_few_pages_takes_no_longer_than_many():
    """A workgroup owns a page: one page's boxes asked for 16000 times would all be one workgroup's work
    (76 times as long as from 512 pages; by boxes it is as long)."""
    log("pages few")
    took = []
    for pages in (1, 512):
        m = rex.box_memory(pages, 8, 128)
        ask = torch.arange(16000, device="cuda") * 37 % (pages * 32)
        best = 1e9
        for _ in range(6):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            rex.box_memory_read(m, ask)
            end.record()
            torch.cuda.synchronize()
            best = min(best, start.elapsed_time(end))
        took.append(best)
    assert took[0] < 8 * took[1], took
