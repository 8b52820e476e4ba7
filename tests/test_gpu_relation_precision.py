"""How many bits the attention's results have, whatever the size of a call.  The bounds are those of
test_gpu_relation_attn.py."""
import numpy as np
import pytest

import paper_1906_07155_amd as rex
import relation_oracle as O
from gpu_helpers import log
from test_gpu_relation_attn import Case, draw_boxes, f64
from test_gpu_relation_memory import Recall

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


def rounded_only(name, have, ref, share):
    """`have` is bf16 and as far from the 64-bit `ref` as rounding alone takes it.

    What is rounded is off by 2^-17 of the weights and binary32 sums, `share` of them in all: norm-wise
    2^-16 of the sums of absolute values is a bound with room.  The roundings themselves are as large as
    those of the reference, up to which of two neighbours a value near the middle goes to (a
    twentieth of them is more than that can make of thousands of values)."""
    have, ref, share = f64(have), np.asarray(ref), np.asarray(share)
    own = np.linalg.norm(f64(torch.from_numpy(ref).to(torch.bfloat16)) - ref)
    err = np.linalg.norm(have - ref)
    assert err <= 1.05 * own + 2.0 ** -16 * np.linalg.norm(share), (name, err / np.linalg.norm(ref), own / np.linalg.norm(ref))


@pytest.mark.parametrize("shape", [(1, 100, 100, 8, 8, 32, 15), (2, 100, 100, 8, 8, 32, 15), (1, 300, 300, 8, 2, 64, 15),
                                   (1, 200, 333, 4, 4, 128, 7), (4, 150, 150, 8, 8, 48, 0)], ids=str)
def test_bf16_results_are_rounded_once(shape):
    """In small calls and in large ones."""
    log("precision bf16 %s" % (shape,))
    c = Case("bf16", *shape, seed=31)
    for got in (c.both(), {"out": c.fwd()[0]}):
        for key in ("out", "grad_q", "grad_k", "grad_v"):
            if key in got:
                rounded_only(key, got[key], c.ref[key], c.ref[key + "_big"])


@pytest.mark.parametrize("shape", [(1, 1, 500, 8, 8, 32, 15), (2, 200, 400, 8, 4, 64, 15), (1, 150, 200, 2, 2, 128, 0)], ids=str)
def test_bf16_results_of_the_memory_are_rounded_once(shape):
    log("precision memory %s" % (shape,))
    r = Recall("bf16", *shape, seed=32)
    ref = O.attn(f64(r.q), r.k, r.v, r.D ** -0.5, r.idx, r.bias, None, r.lengths)
    rounded_only("out", r.run()[0], ref["out"], ref["out_abs"])


@pytest.mark.parametrize("n", [257, 771, 999])
def test_the_gate_sees_the_mean_of_an_image(n):
    """The mean over the counted boxes, rounded once to the features' type: at most 2^-8 of it (half a
    spacing at the bottom of an octave), and binary32 sums of n terms."""
    log("precision gate %d" % n)
    torch.manual_seed(n)
    head = rex.RelationHead(64, 4, layers=1).cuda().bfloat16()
    x = (torch.randn(2, 1000, 64, device="cuda") + 1.0).bfloat16()
    boxes = torch.rand(2, 1000, 4, device="cuda") * 100.0
    seen = []
    head.layers[0].gate.register_forward_hook(lambda module, args, out: seen.append(args[0].detach()))
    with torch.no_grad():
        head(x, boxes, [n, 1000])
    for i, m in enumerate((n, 1000)):
        want = f64(x[i, :m]).mean(0)
        bound = 2.0 ** -8 * np.abs(want) + (m + 8) * 2.0 ** -24 * np.abs(f64(x[i, :m])).mean(0)
        assert np.all(np.abs(f64(seen[0][i]) - want) <= bound), (m, (np.abs(f64(seen[0][i]) - want) / bound).max())


def test_a_frame_and_its_memory_are_joined_before_they_are_rounded():
    """The layer's attention over a frame's own boxes and the remembered ones is one softmax."""
    log("precision join")
    torch.manual_seed(3)
    rng = np.random.default_rng(3)
    head = rex.RelationHead(256, 8, layers=1).cuda().bfloat16()
    with torch.no_grad():
        head.layers[0].bias.normal_()
    memory = head.memory(num_pages=64, streams=2, max_pages=30)
    seen = []
    head.layers[0].qkv.register_forward_hook(lambda module, args, out: seen.append(out.detach()))
    head.layers[0].proj.register_forward_hook(lambda module, args, out: seen.append(args[0].detach()))
    counts = [200, 150]
    for frame in range(3):
        boxes = draw_boxes(rng, (2, 200))
        x = torch.from_numpy(rng.standard_normal((2, 200, 256))).bfloat16().cuda()
        pages, lengths = (t.cpu().numpy() for t in memory.pages_and_lengths())
        held = [rex.box_memory_read(memory.layers[0], torch.from_numpy(p[np.arange(t) // 32].astype(np.int64) * 32 + np.arange(t) % 32).cuda())
                for p, t in zip(pages, lengths)]
        seen.clear()
        with torch.no_grad():
            head(x, torch.from_numpy(boxes).cuda(), counts, memory)
        qkv, joined = seen[0].view(2, 200, 24, 32), seen[1].view(2, 200, 8, 32)
        for s, n in enumerate(counts):
            q, k, v = (f64(t)[None] for t in qkv[s, :n].split(8, 1))
            hk, hv, hb = held[s]
            kb = np.concatenate([boxes[s, :n], hb.cpu().numpy()])
            idx = O.buckets(boxes[s, :n], kb, 15, -4, 1)[None]
            ref = O.attn(q, np.concatenate([k, f64(hk)[None]], 1), np.concatenate([v, f64(hv)[None]], 1), 32 ** -0.5, idx,
                         f64(head.layers[0].bias).reshape(8, -1))
            rounded_only("frame %d" % frame, joined[s, :n][None], ref["out"], ref["out_abs"])
