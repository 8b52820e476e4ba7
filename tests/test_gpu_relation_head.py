"""RelationHead, which runs the operators together, against the same layers written out in 64
bits with torch's own gradients.

A binary32 stage of n-term sums is off by at most (n + 16) 2^-24 of its norm, 128-term ones here by
8.6e-6; a layer has eight of them (two norms, the attention's two, four linear ones) and the gate,
its backward twice as many, and errors add: 2 layers forward 1.6e-4, with the backward 5e-4.
"""
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


def make(layers, kv_heads=None, norm="rms", channels=64, heads=4):
    torch.manual_seed(5)
    head = rex.RelationHead(channels, heads, kv_heads, layers, norm=norm).cuda()
    with torch.no_grad():
        for layer in head.layers:
            layer.bias.normal_()
            for p in (*layer.post, *layer.pre):
                p.uniform_(0.5, 1.5)
    return head


def normed(x, w, norm):
    if norm == "layer":
        x = x - x.mean(-1, keepdim=True)
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w


def plain(p, x, boxes, counts, heads, kv_heads, layers, norm, held=None):
    """The head of parameters `p` (64 bits, by name), one image at a time; held[i][layer]: keys,
    values and boxes that image i's stream remembers."""
    out = []
    for i, n in enumerate(counts):
        xi, bi = x[i, :n], boxes[i, :n]
        linear = lambda name, t: t @ p[name + ".weight"].T + p[name + ".bias"]
        mean = xi.sum(0) / max(n, 1)
        for j in range(layers):
            at = "layers.%d." % j
            u = normed(xi, p[at + "pre.0"], norm)
            d = xi.shape[1] // heads
            q, k, v = linear(at + "qkv", u).view(n, heads + 2 * kv_heads, d).split([heads, kv_heads, kv_heads], 1)
            kb = bi
            if held is not None:
                k, v = torch.cat([k, held[i][j][0]]), torch.cat([v, held[i][j][1]])
                kb = np.concatenate([bi, held[i][j][2]])
            idx = torch.from_numpy(O.buckets(bi, kb, 15, -4, 1))
            rep = heads // kv_heads
            s = torch.einsum("qhd,khd->hqk", q, k.repeat_interleave(rep, 1)) * d ** -0.5
            s = s + p[at + "bias"].reshape(heads, -1)[:, idx]
            o = torch.einsum("hqk,khd->qhd", s.softmax(-1), v.repeat_interleave(rep, 1)).reshape(n, heads * d)
            gate = torch.sigmoid(linear(at + "gate", mean))
            xi = xi + gate * normed(linear(at + "proj", o), p[at + "post.0"], norm)
            u = normed(xi, p[at + "pre.1"], norm)
            branch = linear(at + "fc2", torch.relu(linear(at + "fc1", u)))
            xi = xi + gate * normed(branch, p[at + "post.1"], norm)
        out.append(xi)
    return out


def close(got, want, tol, what):
    got, want = got.detach().double().cpu(), want.detach()
    err = float((got - want).norm() / want.norm())
    assert err <= tol, (what, err)


@pytest.mark.parametrize("kv_heads,norm,counts", [(4, "rms", [50, 33]), (2, "layer", [50, 1]), (1, "rms", [7, 50])])
def test_head_and_its_gradients(kv_heads, norm, counts):
    log("head %d %s" % (kv_heads, norm))
    rng = np.random.default_rng(kv_heads)
    head = make(2, kv_heads, norm)
    boxes = draw_boxes(rng, (2, 50))
    x0, g0 = (torch.from_numpy(rng.standard_normal((2, 50, 64))) for _ in range(2))
    x = x0.float().cuda().requires_grad_()
    y = head(x, torch.from_numpy(boxes).cuda(), counts)
    live = torch.arange(50)[None] < torch.tensor(counts)[:, None]
    (y * (g0 * live[..., None]).float().cuda()).sum().backward()

    p = {k: v.detach().double().cpu().requires_grad_() for k, v in head.named_parameters()}
    xr = x.detach().double().cpu().requires_grad_()
    want = plain(p, xr, boxes, counts, 4, kv_heads, 2, norm)
    sum((w * g0[i, :n].float().double()).sum() for i, (w, n) in enumerate(zip(want, counts))).backward()
    for i, n in enumerate(counts):
        close(y[i, :n], want[i], 1.6e-4, "y")
        close(x.grad[i, :n], xr.grad[i, :n], 5e-4, "grad x")
    for name, t in head.named_parameters():
        if name.endswith("qkv.bias"):       # a key's bias shifts a row of logits: its gradient is 0
            d, h = 16, 4
            keep = torch.cat([torch.arange(h * d), torch.arange((h + kv_heads) * d, (h + 2 * kv_heads) * d)])
            close(t.grad[keep.cuda()], p[name].grad[keep], 5e-4, name)
        else:
            close(t.grad, p[name].grad, 5e-4, name)


def test_head_in_bf16_follows_binary32():
    log("head bf16")
    rng = np.random.default_rng(9)
    head = make(2)
    boxes = torch.from_numpy(draw_boxes(rng, (2, 300))).cuda()
    x = torch.from_numpy(rng.standard_normal((2, 300, 64)).astype(np.float32)).cuda()
    with torch.no_grad():
        want = head(x.bfloat16().float(), boxes, [300, 211])
        low = make(2).bfloat16()
        assert low.layers[0].bias.dtype == torch.float32
        got = low(x.bfloat16(), boxes, [300, 211])
    # some twenty roundings to bf16, each at most 2^-8 of its stage
    close(got[0], want[0].double().cpu(), 20 * 2.0 ** -8, "bf16")
    assert got.dtype == torch.bfloat16


def test_video_recalls_what_it_was_shown():
    """Three frames of two streams: each frame's boxes attend to their own and to the boxes of the
    frames before, as the memory holds them."""
    log("head video")
    rng = np.random.default_rng(4)
    head = make(2, 2)
    memory = head.memory(num_pages=40, streams=2, max_pages=12)
    p = {k: v.detach().double().cpu() for k, v in head.named_parameters()}
    for counts in ([40, 17], [0, 40], [31, 32]):
        boxes = draw_boxes(rng, (2, 40))
        x = torch.from_numpy(rng.standard_normal((2, 40, 64)).astype(np.float32)).cuda()
        pages, lengths = (t.cpu() for t in memory.pages_and_lengths())
        held = []
        for s in range(2):
            t = torch.arange(int(lengths[s]))
            slots = (pages[s][t // 32].long() * 32 + t % 32).cuda()
            held.append([tuple(r.double().cpu() if r.dim() == 3 else r.cpu().numpy()
                               for r in rex.box_memory_read(m, slots)) for m in memory.layers])
        with torch.no_grad():
            y = head(x, torch.from_numpy(boxes).cuda(), counts, memory)
            want = plain(p, x.double().cpu(), boxes, counts, 4, 2, 2, "rms", held)
        for i, n in enumerate(counts):
            if n:
                close(y[i, :n], want[i], 1.6e-4, "frame %s" % counts)
    assert memory.used == [71, 89]


def test_refusals():
    head = make(1)
    x, boxes = torch.zeros(2, 3, 64, device="cuda"), torch.zeros(2, 3, 4, device="cuda")
    memory = head.memory(8, 2, 2)
    with pytest.raises(RuntimeError, match="no_grad"):
        head(x, boxes, memory=memory)
    with pytest.raises(ValueError, match="counts"):
        head(x, boxes, [4, 1])
    with torch.no_grad(), pytest.raises(ValueError, match="streams"):
        head(x[:1], boxes[:1], memory=memory)
    with pytest.raises(ValueError, match="nothing to do"):
        rex.gated_norm(x[0], second=False)
