"""The C ABI of box_head.h and box_evict.h on the host: what is exported, how its structs are laid
out, what its functions refuse before anything is enqueued, and the sizes of workspaces; then the
Python binding's refusals of mis-shaped, mistyped and misplaced tensors.

No call reaches a kernel launch, so these run without a GPU.  Device pointers are stand-in addresses.
"""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_1906_07155_amd as rex
from paper_1906_07155_amd import binding as B
from paper_1906_07155_amd import evict as E
from paper_1906_07155_amd import head as H
from paper_1906_07155_amd import relation as R
from test_relation_abi_cpu import memory, recall

OK, INVALID, UNSUPPORTED, WORKSPACE, DEVICE = range(5)
FAKE = 1 << 20
INF, NAN = float("inf"), float("nan")
BIG = 1 << 62


@pytest.fixture(scope="module")
def L():
    E.lib()
    return H.lib()


def linear(**kw):
    f = dict(x=FAKE, weight=FAKE, bias=FAKE, residual=0, x_stride=64, weight_stride=64, residual_stride=48, rows=100,
             ins=64, outs=48, dtype=0, bias_dtype=0, act=1)
    f.update(kw)
    return H._LINEAR.pack(*f.values())


def logprob(**kw):
    f = dict(logits=FAKE, labels=FAKE, stride=81, rows=10, classes=81, dtype=0, top=0, scale=1.0)
    f.update(kw)
    return H._LOGPROB.pack(*f.values())


def eviction(**kw):
    f = dict(batch=2, max_pages=3, pages=FAKE, lengths=FAKE, keep=FAKE, weight=FAKE)
    f.update(kw)
    return E._EVICT.pack(*f.values())


def size_of(fn, *args):
    n = ctypes.c_size_t(1)
    assert fn(*args, ctypes.byref(n)) == OK
    return n.value


BAD_LINEAR = [
    (dict(dtype=2), INVALID), (dict(dtype=-1), INVALID), (dict(act=-1), INVALID), (dict(act=4), INVALID),
    (dict(rows=-1), INVALID), (dict(ins=0), INVALID), (dict(outs=0), INVALID), (dict(x=0), INVALID),
    (dict(weight=0), INVALID), (dict(x=FAKE + 2), INVALID), (dict(weight=FAKE + 1), INVALID),
    (dict(residual=FAKE + 2), INVALID), (dict(bias=FAKE + 2), INVALID), (dict(bias_dtype=2), INVALID),
    (dict(bias_dtype=1), INVALID), (dict(x_stride=-1), INVALID), (dict(weight_stride=-64), INVALID),
    (dict(residual=FAKE, residual_stride=-1), INVALID), (dict(x_stride=BIG), INVALID),
    (dict(rows=1 << 31), UNSUPPORTED), (dict(ins=(1 << 24) + 1), UNSUPPORTED), (dict(outs=(1 << 24) + 1), UNSUPPORTED),
    (dict(x_stride=1 << 20), UNSUPPORTED), (dict(weight_stride=1 << 20), UNSUPPORTED),      # 256 rows past a buffer's reach
    (dict(ins=1 << 20, x_stride=1 << 20, weight_stride=1 << 20), UNSUPPORTED), (dict(outs=1 << 20), UNSUPPORTED),
    (dict(rows=1 << 30, outs=64), UNSUPPORTED),                 # more workgroups than a launch has
]


@pytest.mark.parametrize("change,status", BAD_LINEAR, ids=[str(c) for c, _ in BAD_LINEAR])
def test_linear_refuses(L, change, status):
    d, n = linear(**change), ctypes.c_size_t(0)
    for backward in (0, 1):
        assert L.linear_act_workspace_size(d, backward, ctypes.byref(n)) == status
    assert L.linear_act_fwd(d, FAKE, 0, FAKE, 1 << 40, 0) == status
    assert L.linear_act_bwd(d, FAKE, FAKE, 0, FAKE, FAKE, FAKE, FAKE, 1 << 40, 0) == status


def test_linear_refuses_buffers(L):
    d, plain, bf16 = linear(), linear(act=0), linear(dtype=1)
    assert L.linear_act_workspace_size(None, 0, ctypes.byref(ctypes.c_size_t(0))) == INVALID
    assert L.linear_act_workspace_size(d, 0, None) == INVALID
    for y, slope in ((0, 0), (FAKE + 2, 0), (FAKE, FAKE + 2)):
        assert L.linear_act_fwd(d, y, slope, FAKE, 1 << 30, 0) == INVALID
    assert L.linear_act_fwd(plain, FAKE, FAKE, FAKE, 1 << 30, 0) == INVALID           # no slope without an activation
    assert L.linear_act_fwd(bf16, FAKE, FAKE + 8, FAKE, 1 << 30, 0) == INVALID
    bwd = lambda d, gy=FAKE, slope=0, y=FAKE, gx=FAKE, gw=FAKE, gb=FAKE, ws=FAKE, n=1 << 30: \
        L.linear_act_bwd(d, gy, slope, y, gx, gw, gb, ws, n, 0)
    for kw in (dict(gy=0), dict(gy=FAKE + 2), dict(y=0), dict(slope=FAKE), dict(y=FAKE + 1), dict(gx=FAKE + 2),
               dict(gw=FAKE + 2), dict(gb=FAKE + 2)):
        assert bwd(d, **kw) == INVALID, kw
    assert bwd(linear(act=2)) == INVALID                                              # gelu's slope is not in y
    assert bwd(plain) == INVALID and bwd(plain, y=0, slope=FAKE) == INVALID
    assert bwd(linear(bias=0)) == INVALID                                             # a gradient of no bias
    need = size_of(L.linear_act_workspace_size, d, 1)
    assert need > 0
    for ws, n in ((0, need), (FAKE, need - 1), (FAKE + 128, need)):
        assert bwd(d, ws=ws, n=n) == WORKSPACE
    few = linear(rows=64, ins=65536, x_stride=65536, weight_stride=65536, act=0)
    need = size_of(L.linear_act_workspace_size, few, 0)
    assert need > 0 and L.linear_act_fwd(few, FAKE, 0, FAKE, need - 1, 0) == WORKSPACE


def test_linear_workspaces(L):
    size = lambda backward, **kw: size_of(L.linear_act_workspace_size, linear(**kw), backward)
    assert size(0, rows=0) == 0 and size(0, rows=1, ins=64) == 0
    assert size(1, rows=0) == 0
    # the gradient of the sums, and column sums
    assert size(1, rows=1000, outs=48) >= 1000 * 48 * 4
    assert size(1, rows=1000, outs=48) > size(1, rows=1000, outs=48, bias=0) >= size(1, rows=1000, outs=48, bias=0, act=0)
    # a single output row or column, strides of one row are not looked at
    assert size(0, rows=1, x_stride=-5) == 0
    # many results: nothing to join; few with long sums: parts of them
    assert size(0, rows=8192, ins=512, outs=8192, x_stride=512, weight_stride=512) == 0
    assert size(0, rows=256, ins=8192, outs=256, x_stride=8192, weight_stride=8192) >= 2 * 256 * 256 * 4


BAD_LOGPROB = [
    (dict(dtype=2), INVALID), (dict(rows=-1), INVALID), (dict(classes=0), INVALID), (dict(top=-1), INVALID),
    (dict(top=17), INVALID), (dict(classes=4, top=5), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=NAN), INVALID), (dict(scale=INF), INVALID), (dict(logits=0), INVALID), (dict(labels=0), INVALID),
    (dict(logits=FAKE + 2), INVALID), (dict(labels=FAKE + 4), INVALID), (dict(stride=-1), INVALID),
    (dict(stride=BIG), INVALID), (dict(classes=(1 << 24) + 1), UNSUPPORTED), (dict(rows=(1 << 23) + 1), UNSUPPORTED),
    (dict(rows=1 << 22, classes=20000), UNSUPPORTED),
]


@pytest.mark.parametrize("change,status", BAD_LOGPROB, ids=[str(c) for c, _ in BAD_LOGPROB])
def test_logprob_refuses(L, change, status):
    d, n = logprob(**change), ctypes.c_size_t(0)
    assert L.class_logprob_workspace_size(d, ctypes.byref(n)) == status
    assert L.class_logprob_fwd(d, *[FAKE] * 5, FAKE, 1 << 40, 0) == status
    assert L.class_logprob_bwd(d, *[FAKE] * 5, 0) == status


def test_logprob_refuses_buffers(L):
    d = logprob(top=3)
    assert L.class_logprob_workspace_size(None, ctypes.byref(ctypes.c_size_t(0))) == INVALID
    assert L.class_logprob_workspace_size(d, None) == INVALID
    for i in range(5):
        for bad in (0, FAKE + 2):
            args = [FAKE] * 5
            args[i] = bad
            assert L.class_logprob_fwd(d, *args, 0, 0, 0) == INVALID
    assert L.class_logprob_fwd(d, FAKE, FAKE, FAKE + 4, FAKE, FAKE, 0, 0, 0) == INVALID
    for i in range(2, 5):                   # the upstream gradients may be left out, nothing else
        args = [FAKE] * 5
        args[i] = 0
        assert L.class_logprob_bwd(d, *args, 0) == INVALID
    for i in range(5):
        args = [FAKE] * 5
        args[i] = FAKE + 2
        assert L.class_logprob_bwd(d, *args, 0) == INVALID
    assert size_of(L.class_logprob_workspace_size, d) == 0
    long = logprob(classes=50000, stride=50000, top=3)
    need = size_of(L.class_logprob_workspace_size, long)
    assert need >= 10 * 13 * (12 + 3 * 8) and need % 256 == 0
    for ws, n in ((0, need), (FAKE, need - 1), (FAKE + 8, need)):
        assert L.class_logprob_fwd(long, *[FAKE] * 5, ws, n, 0) == WORKSPACE
    assert H.LOGPROB_SPAN == 4088
    assert size_of(L.class_logprob_workspace_size, logprob(classes=4088, stride=4088)) == 0
    assert size_of(L.class_logprob_workspace_size, logprob(classes=4089, stride=4089)) > 0


def test_weigh_refuses(L):
    m = memory()
    call = lambda m=m, r=recall(), lse=FAKE, weight=FAKE, decay=1.0, out=FAKE: \
        L.box_memory_weigh(m, r, lse, weight, decay, out, 0)
    for kw in (dict(lse=0), dict(lse=FAKE + 2), dict(weight=FAKE + 2), dict(out=0), dict(out=FAKE + 1), dict(decay=NAN),
               dict(decay=INF), dict(m=memory(k=0)), dict(m=memory(dim=12)), dict(r=recall(dtype=2)),
               dict(r=recall(heads=3)), dict(r=recall(scale=0.0)), dict(r=recall(pages=0)), dict(r=recall(lengths=0)),
               dict(r=recall(bias=0)), dict(r=recall(buckets=4)), dict(r=recall(q=0)), dict(r=None), dict(m=None)):
        assert call(**kw) == INVALID, kw
    assert call(r=recall(batch=1 << 22, num_q=1)) == UNSUPPORTED
    assert call(r=recall(batch=0), out=0, lse=0) == OK           # nothing to do


def test_evict_refuses(L):
    m, n = memory(), ctypes.c_size_t(0)
    need = size_of(L.box_memory_evict_workspace_size, m, eviction())
    call = lambda m=m, e=eviction(), left=FAKE, out=FAKE << 1, origin=FAKE, ws=FAKE, size=need: \
        L.box_memory_evict(m, e, left, out, origin, ws, size, 0)
    for kw in (dict(batch=-1), dict(max_pages=-1), dict(pages=0), dict(lengths=0), dict(keep=0), dict(weight=0),
               dict(pages=FAKE + 2), dict(lengths=FAKE + 1), dict(keep=FAKE + 2), dict(weight=FAKE + 2)):
        assert L.box_memory_evict_workspace_size(m, eviction(**kw), ctypes.byref(n)) == INVALID, kw
        assert call(e=eviction(**kw)) == INVALID, kw
    for kw in (dict(max_pages=1 << 20), dict(batch=1 << 22), dict(batch=1 << 20, max_pages=32)):
        assert call(e=eviction(**kw)) == UNSUPPORTED, kw
    for kw in (dict(m=memory(v=0)), dict(m=None), dict(e=None), dict(left=0), dict(left=FAKE + 2), dict(out=0),
               dict(out=FAKE + 2), dict(origin=FAKE + 2), dict(out=FAKE)):       # (the last: the weights themselves)
        assert call(**kw) == INVALID, kw
    assert need >= 3 * 2 * 96 * 4
    for ws, size in ((0, need), (FAKE, need - 1), (FAKE + 64, need)):
        assert call(ws=ws, size=size) == WORKSPACE
    assert call(e=eviction(batch=0), left=0, out=0, origin=0, ws=0, size=0) == OK


@pytest.mark.skipif(not os.environ.get("REX_LIBRARY", "").endswith("_host.so"),
                    reason="needs a build whose launchers do nothing")
@pytest.mark.parametrize("dtype", [0, 1])
def test_valid_calls(L, dtype):
    sizes = (1, 3, 16, 17, 63, 64, 65, 255, 256, 257, 1000, 4096, 12544, 16001)
    shapes = [(m, n, k) for m in (0,) + sizes for n in sizes for k in sizes]
    shapes += [(64 * ((1 << 24) - 16), 1, 8), ((1 << 24) - 16, 64, 64), ((1 << 25) - 64, 6, 2048),
               (1 << 29, 16, 64), (1, 1 << 19, 2048), (1 << 20, 128, 256)]
    for m, n, k in shapes:
        for act, aligned in ((0, True), (1, True), (2, False)) if m < 300 else ((3, True), (0, False)):
            stride = k if m < 1 << 24 else 0
            d = linear(rows=m, outs=n, ins=k, dtype=dtype, bias_dtype=dtype, act=act, x=FAKE + (0 if aligned else 4),
                       x_stride=stride, weight_stride=k, residual_stride=n, residual=FAKE if aligned else 0)
            size = size_of(L.linear_act_workspace_size, d, 0)
            assert L.linear_act_fwd(d, FAKE, FAKE if act else 0, FAKE if size else 0, size, 0) == OK, (m, n, k, act)
            size = size_of(L.linear_act_workspace_size, d, 1)
            y = FAKE if act == 1 else 0
            gy = FAKE if aligned else FAKE + 4
            for gx, gw, gb in ((FAKE, FAKE, FAKE), (FAKE, 0, 0), (0, FAKE, 0), (0, 0, FAKE), (0, 0, 0)):
                assert L.linear_act_bwd(d, gy, 0 if act < 2 else FAKE, y, gx, gw, gb, FAKE, size, 0) == OK, (m, n, k, act)
    for rows in (0, 1, 100, 1000):
        for classes in (1, 7, 81, 4088, 4089, 8177, 100003, 1 << 24):
            for top in (0, min(classes, 16)):
                d = logprob(rows=rows, classes=classes, stride=classes, top=top, dtype=dtype)
                size = size_of(L.class_logprob_workspace_size, d)
                assert L.class_logprob_fwd(d, *[FAKE] * 5, FAKE, size, 0) == OK
                assert L.class_logprob_bwd(d, *[FAKE] * 5, 0) == OK
    for kw in (dict(), dict(batch=0), dict(num_q=0), dict(max_pages=0, pages=0), dict(batch=3, num_q=1, max_pages=1 << 19)):
        assert L.box_memory_weigh(memory(), recall(dtype=dtype, **kw), FAKE, FAKE, 0.5, FAKE << 1, 0) == OK
    for kw in (dict(), dict(batch=0), dict(max_pages=0, pages=0, weight=0), dict(batch=16, max_pages=1 << 18),
               dict(batch=1 << 21, max_pages=1)):
        size = size_of(L.box_memory_evict_workspace_size, memory(), eviction(**kw))
        for origin in (0, FAKE):
            assert L.box_memory_evict(memory(), eviction(**kw), FAKE, FAKE << 1, origin, FAKE, size, 0) == OK


def test_headers_and_binding_agree(L, tmp_path):
    assert sorted(H.header_functions()) == sorted(H.SIGNATURES) and len(H.SIGNATURES) == 6
    assert sorted(E.header_functions()) == sorted(E.SIGNATURES) and len(E.SIGNATURES) == 3
    text = """#include <stdio.h>
#include <stddef.h>
#include "box_head.h"
#include "box_evict.h"
int main(void) {
    printf("%zu %zu %zu %zu %zu %zu %d %d\\n", sizeof(linear_act_t), offsetof(linear_act_t, rows), offsetof(linear_act_t, act),
           sizeof(class_logprob_t), offsetof(class_logprob_t, scale), sizeof(box_evict_t), RE_LOGPROB_MAX_TOP, RE_ACT_SILU);
    return 0;
}"""
    (tmp_path / "a.c").write_text(text)
    exe = str(tmp_path / "a.out")
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.dirname(H.HEADER), str(tmp_path / "a.c"), "-o", exe])
    got = [int(v) for v in subprocess.check_output([exe], text=True).split()]
    assert got == [H._LINEAR.size, 56, 88, H._LOGPROB.size, 48, E._EVICT.size, H.MAX_TOP, H.ACTS["silu"]]


def test_binding_refuses(monkeypatch):
    x, w, b = torch.zeros(5, 8), torch.zeros(6, 8), torch.zeros(6)
    for kw in (dict(act="tanh"), dict(x=x[0]), dict(weight=w[0]), dict(weight=torch.zeros(6, 7)), dict(weight=w.bfloat16()),
               dict(bias=torch.zeros(5)), dict(bias=b.double()), dict(bias=b.bfloat16()), dict(bias=torch.zeros(12)[::2]),
               dict(residual=torch.zeros(5, 5)), dict(residual=torch.zeros(5, 6).bfloat16()), dict(x=torch.zeros(8, 5).t()),
               dict(weight=torch.zeros(8, 6).t()), dict(residual=torch.zeros(6, 5).t())):
        a = dict(x=x, weight=w, bias=b)
        a.update(kw)
        with pytest.raises(ValueError):
            rex.linear_act_fwd(**a)
    with pytest.raises(TypeError):
        rex.linear_act_fwd(x.double(), w.double())
    with pytest.raises((ValueError, RuntimeError)):         # a CPU tensor
        rex.linear_act_fwd(x, w, b)
    logits, labels = torch.zeros(5, 7), torch.zeros(5, dtype=torch.int64)
    for kw in (dict(logits=logits[0]), dict(logits=torch.zeros(5, 0)), dict(labels=labels[:4]), dict(labels=labels.int()),
               dict(top=-1), dict(top=8), dict(logits=torch.zeros(7, 5).t())):
        a = dict(logits=logits, labels=labels)
        a.update(kw)
        with pytest.raises(ValueError):
            rex.class_logprob_fwd(**a)
    with pytest.raises(TypeError):
        rex.class_logprob_fwd(logits.half(), labels)
    with pytest.raises(ValueError):
        rex.class_logprob_fwd(torch.zeros(5, 40), labels, top=17)


def test_binding_refuses_memories(monkeypatch):
    for module in (R, E):
        monkeypatch.setattr(module, "_need_cuda", lambda *a: None)
    m = rex.box_memory(4, 2, 32, device="cpu")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    q, lse = torch.zeros(2, 3, 4, 32), torch.zeros(2, 4, 3)
    good = dict(q=q, memory=m, pages=i32(2, 2), lengths=i32(2), lse=lse)
    for kw in (dict(q=torch.zeros(2, 3, 4, 40)), dict(q=torch.zeros(2, 3, 3, 32)), dict(q=q[0]), dict(pages=i32(3, 2)),
               dict(pages=i32(2)), dict(pages=torch.zeros(2, 2)), dict(lengths=i32(3)), dict(lse=torch.zeros(2, 3, 4)),
               dict(lse=lse.double()), dict(weight=torch.zeros(2, 63)), dict(out=torch.zeros(2, 64).double()),
               dict(q_len=i32(3)), dict(bias=torch.zeros(4, 4, 4)), dict(bias=torch.zeros(4, 5, 5)),
               dict(memory=m[:4])):
        with pytest.raises(ValueError):
            rex.box_memory_weigh(**{**good, **kw})
    good = dict(memory=m, pages=i32(2, 2), lengths=i32(2), weight=torch.zeros(2, 64), keep=i32(2))
    for kw in (dict(pages=i32(2)), dict(lengths=i32(1)), dict(weight=torch.zeros(2, 32)), dict(weight=torch.zeros(2, 64).double()),
               dict(keep=i32(3)), dict(keep=torch.zeros(2, dtype=torch.int64)), dict(memory=m[1:])):
        with pytest.raises(ValueError):
            rex.box_memory_evict(**{**good, **kw})


def test_box_memory_by_weight(monkeypatch):
    """Places and room of a memory that forgets by weight, the kernels' part played by a plain one."""
    from paper_1906_07155_amd import relation_head as RH

    def plain(memory, pages, lengths, weight, keep):
        left, held = keep.clone(), torch.zeros_like(weight)
        for s in range(len(keep)):
            n, k = int(lengths[s]), int(keep[s])
            order = sorted(range(n), key=lambda t: (-float(weight[s, t]), t))[:k]
            late = iter(sorted(t for t in order if t >= k))
            held[s, :k] = torch.tensor([float(weight[s, t if t in order else next(late)]) for t in range(k)])
        return left, held, None
    monkeypatch.setattr(RH.evict, "box_memory_evict", plain)
    with pytest.raises(ValueError):
        RH.BoxMemory(8, 2, 3, 2, 32, device="cpu", evict="least")
    memory = RH.BoxMemory(6, 2, 3, 2, 32, layers=2, device="cpu", evict="weight")
    assert len(memory.take([60, 0])) == 60 and memory.used == [60, 0]
    memory.weight[0, :60] = torch.arange(60.0)
    taken = memory.take([50, 40])
    assert memory.used == [96, 40] and len(memory.table[0]) == 3 and len(memory.table[1]) == 2
    # the fourteen lightest made room; what was left is in the first 46 places, the new ones behind
    assert sorted(memory.weight[0, :46].tolist()) == list(range(14, 60)) and not memory.weight[0, 46:].any()
    pages = memory.table[0]
    assert taken[:50].tolist() == [pages[t // 32] * 32 + t % 32 for t in range(46, 96)]
    memory.take([64, 0])
    assert memory.used == [96, 40]
    with pytest.raises(ValueError):
        memory.take([65, 0])
    memory.forget(0)
    assert memory.used == [0, 40] and not memory.weight[0].any() and len(memory.free) == 4
    assert len(memory.take([10, 0])) == 10


def test_box_memory_forgets_outside_inference_mode():
    from paper_1906_07155_amd import relation_head as RH
    memory = RH.BoxMemory(6, 2, 3, 2, 32, device="cpu", evict="weight")
    memory.take([10, 10])
    with torch.inference_mode():                # as a frame does
        memory.weight = memory.weight + 1
    memory.forget(0)
    assert memory.used == [0, 10] and not memory.weight[0].any() and (memory.weight[1] == 1).all()
