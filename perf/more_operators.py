"""What the operators around a detector's heads are measured on, and their plain forms.

A box head takes what was extracted for each RoI through dense layers to scores and deltas and
trains on the log probability of each RoI's class; a relation head has the same dense layers
between its attentions, and a memory of earlier frames that is full has to forget something.

Kinds of case:
  linear   y = act(x weight^T + bias) + residual, its gradients (linear_act_fwd, linear_act_bwd)
  logprob  log probability of each row's label, entropy and the top classes (class_logprob_fwd,
           and in training class_logprob_bwd)
  weigh    the attention that each remembered box has received (box_memory_weigh)
  evict    the boxes of least weight leave the memory (box_memory_evict)

`run` computes the plain forms in binary32, or calls the library where `own` is true;
`exact` is the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 32                       # boxes of one page of the memory
STEPS, FIRST = 1, -4            # bias buckets: one per octave, the first from 2^-4 box sizes


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------

def _linear(rows, ins, outs, dtype, direction, act, **kw):
    case = {"kind": "linear", "rows": rows, "ins": ins, "outs": outs, "dtype": dtype,
            "pass": direction, "act": act, "bias": True, "residual": False}
    case.update(kw)
    return case


def _logprob(rows, classes, dtype, train, top, **kw):
    case = {"kind": "logprob", "rows": rows, "classes": classes, "dtype": dtype, "train": train,
            "top": top, "scale": 1.0}
    case.update(kw)
    return case


def listed():
    return [
        # One tracked box through a dense layer: the smallest call.
        dict(_linear(1, 1024, 1024, "bf16", "fwd", "relu"), name="linear_infer_1_bf16"),
        # Serving: the 1000 proposals of one image, 256 channels of 7 x 7, into a box head.
        dict(_linear(1000, 12544, 1024, "bf16", "fwd", "relu"), name="linear_infer_1000_bf16"),
        # The same layer's gradients over the 512 sampled boxes of each of two images.
        dict(_linear(1024, 12544, 1024, "f32", "bwd", "relu"), name="linear_bwd_1024_f32"),
        # A relation layer's wide product in a training step over 16 images: the largest.
        dict(_linear(16000, 1024, 2048, "bf16", "train", "gelu"), name="linear_train_16000_bf16"),
        # An odd number of boxes, channels and outputs, added to what came before.
        dict(_linear(513, 250, 77, "f32", "train", "silu", residual=True),
             name="linear_train_513_odd_f32"),
        # The 100 detections of an image over 80 classes and background.
        dict(_logprob(100, 81, "bf16", False, 5), name="logprob_infer_100x81_bf16"),
        # A training step over the 512 sampled boxes of 16 images and a large set of classes.
        dict(_logprob(8192, 1231, "bf16", True, 0), name="logprob_train_8192x1231_bf16"),
        # A few rows over a long list of classes, an odd number of them.
        dict(_logprob(16, 100003, "f32", False, 8, scale=0.7), name="logprob_infer_16x100003_f32"),
        # Tracking: one box in each of 64 streams looks at all that its stream remembers.
        {"kind": "weigh", "streams": 64, "queries": 1, "tokens": 8192, "heads": 8, "kv_heads": 8,
         "dim": 32, "buckets": 15, "dtype": "bf16", "ragged": True, "name": "weigh_64x1_bf16"},
        # Video detection: a frame's 300 boxes over 20 frames of one stream.
        {"kind": "weigh", "streams": 1, "queries": 300, "tokens": 6000, "heads": 16,
         "kv_heads": 16, "dim": 64, "buckets": 15, "dtype": "bf16", "ragged": False,
         "name": "weigh_1x300_bf16"},
        # One full stream makes room for the next frame's 300 boxes.
        {"kind": "evict", "streams": 1, "tokens": 992, "keep": 0.7, "kv_heads": 8, "dim": 32,
         "name": "evict_1x992"},
        # 16 long streams at once, a quarter of each.
        {"kind": "evict", "streams": 16, "tokens": 8192, "keep": 0.75, "kv_heads": 16, "dim": 64,
         "name": "evict_16x8192"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear"] * 4 + ["logprob"] * 3 + ["weigh"] * 2 + ["evict"])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "linear":
        direction = rng.choice(["fwd", "fwd", "bwd", "train"])
        # (binary32 matrix products are some eight times as slow)
        most = 2.0e10 if dtype == "bf16" else 5.0e9
        ins = rng.choice([_log_int(rng, 8, 12544), 8 * _log_int(rng, 8, 1568)])
        outs = rng.choice([_log_int(rng, 1, 4096), 8 * _log_int(rng, 4, 512)])
        rows = _log_int(rng, 1, max(1, min(16000, int(most / (ins * outs)))))
        # (what a sum that is 0 but for its rounding has for a slope is no number to compare:
        # relu's backward pass takes the forward's results as given; what the others keep is the
        # library's own, so they run forward and backward)
        act = rng.choice({"fwd": ["none", "relu", "relu", "gelu", "silu"], "bwd": ["none", "relu"],
                          "train": ["none", "gelu", "silu"]}[direction])
        return _linear(rows, ins, outs, dtype, direction, act, bias=rng.random() < 0.8,
                       residual=direction != "bwd" and rng.random() < 0.3)
    if kind == "logprob":
        classes = _log_int(rng, 2, 100003)
        rows = _log_int(rng, 1, max(1, min(16000, 8192 * 1231 // classes)))
        return _logprob(rows, classes, dtype, rng.random() < 0.5,
                        min(classes, rng.choice([0, 0, 1, 5, 8])), scale=rng.choice([1.0, 1.0, 0.7]))
    dim = rng.choice([32, 64, 64, 40, 96, 128])
    kv = rng.choice([1, 2, 4, 8])
    if kind == "evict":
        return {"kind": kind, "streams": _log_int(rng, 1, 16), "tokens": _log_int(rng, 2, 8192),
                "keep": rng.choice([0.5, 0.75, rng.random()]), "kv_heads": kv, "dim": dim}
    streams, q = rng.choice([(_log_int(rng, 1, 64), 1), (_log_int(rng, 1, 8), rng.randint(2, 30)),
                             (1, _log_int(rng, 30, 300))])
    return {"kind": kind, "streams": streams, "queries": q, "tokens": _log_int(rng, 30, 8192),
            "heads": kv * rng.choice([1, 1, 2, 4]), "kv_heads": kv, "dim": dim,
            "buckets": rng.choice([0, 7, 15, 31]), "dtype": dtype, "ragged": rng.random() < 0.6}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _boxes(gen, shape):
    """Boxes of an 800 x 1344 image: sides log-uniform in 16..512, some around one centre."""
    u = torch.rand((*shape, 4), generator=gen, device="cuda")
    side = 16.0 * torch.exp(u[..., 2:] * math.log(32.0))
    centre = u[..., :2] * torch.tensor([1344.0, 800.0], device="cuda")
    near = torch.rand(shape, generator=gen, device="cuda") < 0.3
    middle = torch.tensor([600.0, 400.0], device="cuda") + 40.0 * (u[..., :2] - 0.5)
    centre = torch.where(near[..., None], middle, centre)
    return torch.cat([centre - 0.5 * side, centre + 0.5 * side], -1).contiguous()


def _keep_count(case):
    return int(case["keep"] * case["tokens"])


def prepare(case, seed):
    st = {"case": dict(case)}
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    kind = case["kind"]

    def randn(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=gen, dtype=dtype, device="cuda")

    def rand(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    def below(n, *shape, dtype=torch.int64):
        return torch.randint(0, n, shape, generator=gen, dtype=dtype, device="cuda")

    if kind == "linear":
        dt = _dtype(case)
        m, n, k = case["rows"], case["outs"], case["ins"]
        st["x"] = randn(m, k, dtype=dt)
        st["weight"] = randn(n, k, dtype=dt) * k ** -0.5
        st["b"] = 0.1 * randn(n) if case["bias"] else None
        st["residual"] = randn(m, n, dtype=dt) if case["residual"] else None
        if case["pass"] != "fwd":
            st["gy"] = randn(m, n, dtype=dt)
        if case["pass"] == "bwd":           # what the forward pass has kept
            st["saved"] = None if case["act"] == "none" else randn(m, n, dtype=dt).clamp(min=0.0)
        return st

    if kind == "logprob":
        m, c = case["rows"], case["classes"]
        st["labels"] = below(c, m)
        x = randn(m, c) * 2.0
        x.scatter_add_(1, st["labels"][:, None], 6.0 * rand(m, 1))
        st["logits"] = x.to(_dtype(case))
        st["labels"] = torch.where(rand(m) < 0.05, torch.full_like(st["labels"], -1), st["labels"])
        if case["train"]:
            st["g_logp"], st["g_entropy"] = -rand(m) - 0.5, 0.1 * randn(m)
        return st

    # a memory that has been in use: every page holds earlier boxes
    b, t, kv, d = case["streams"], case["tokens"], case["kv_heads"], case["dim"]
    per = (t + PAGE - 1) // PAGE
    pages = b * per
    st["pages"] = torch.randperm(pages, generator=gen, device="cuda").int().view(b, per)
    st["lengths"] = torch.full((b,), t, dtype=torch.int32, device="cuda")

    def codes(*shape):
        return (below(255, *shape, dtype=torch.int16) - 127).to(torch.int8)

    def scales():
        return (1.5 + rand(pages, kv, PAGE)) / 127.0

    st["memory"] = (codes(pages, kv, PAGE, d), codes(pages, kv, d, PAGE), scales(), scales(),
                    _boxes(gen, (pages, PAGE)))
    if kind == "evict":
        # what attention leaves: a few boxes with much, many with next to nothing or nothing
        w = torch.exp(2.0 * randn(b, per * PAGE))
        st["weight"] = torch.where(rand(b, per * PAGE) < 0.2, torch.zeros_like(w), w)
        st["keep"] = torch.full((b,), _keep_count(case), dtype=torch.int32, device="cuda")
        return st
    if case["ragged"]:
        st["lengths"] -= below(t // 4 + 1, b, dtype=torch.int32)
    n = case["buckets"]
    st["q"] = randn(b, case["queries"], case["heads"], d, dtype=_dtype(case))
    st["q_boxes"] = _boxes(gen, (b, case["queries"]))
    st["scale"] = d ** -0.5
    st["bias"] = randn(case["heads"], n, n) * 0.5 if n else None
    st["weight"] = torch.exp(randn(b, per * PAGE))
    st["lse"] = torch.logsumexp(_logits(st), -1)      # as the attention over the memory gave it
    return st


# ---------------------------------------------------------------------------
# Plain forms (binary32)
# ---------------------------------------------------------------------------

def _act(name, t):
    if name == "relu":
        return torch.clamp(t, min=0.0)
    if name == "gelu":
        return 0.5 * t * (1.0 + torch.erf(t * 0.5 ** 0.5))
    if name == "silu":
        return t / (1.0 + torch.exp(-t))
    return t


def _slope(name, t):
    if name == "relu":
        return (t > 0).float()
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(t * 0.5 ** 0.5)) + t * torch.exp(-0.5 * t * t) / math.sqrt(2.0 * math.pi)
    s = 1.0 / (1.0 + torch.exp(-t))
    return s * (1.0 + t * (1.0 - s))


def _plain_linear(st):
    case, dt = st["case"], st["x"].dtype
    x, w = st["x"].float(), st["weight"].float()
    found, pre = {}, st.get("saved")
    if case["pass"] != "bwd":
        pre = torch.matmul(x, w.t())
        if case["bias"]:
            pre = pre + st["b"]
        y = _act(case["act"], pre)
        found["y"] = (y + st["residual"].float() if case["residual"] else y).to(dt)
    if case["pass"] != "fwd":
        g = st["gy"].float()
        if case["act"] != "none":
            g = g * _slope(case["act"], pre.float())
        found["grad_x"] = torch.matmul(g, w).to(dt)
        found["grad_weight"] = torch.matmul(g.t(), x).to(dt)
        if case["bias"]:
            found["grad_bias"] = g.sum(0)
    return found


def _plain_logprob(st):
    case = st["case"]
    raw = st["logits"].float()
    x = raw * case["scale"]
    top = x.amax(-1, keepdim=True)
    total = torch.exp(x - top).sum(-1, keepdim=True)
    lse = top + torch.log(total)
    logs = x - lse
    p = torch.exp(logs)
    entropy = -(p * logs).sum(-1)
    counted = st["labels"] >= 0
    at = st["labels"].clamp(min=0)[:, None]
    zero = torch.zeros_like(entropy)
    found = {"logp": torch.where(counted, logs.gather(1, at)[:, 0], zero), "entropy": entropy}
    if case["top"]:
        # unique whole numbers in the order of the logits, the lower index first among equals
        bits = (raw + 0.0).view(torch.int32)
        key = (bits ^ (bits >> 31 & 0x7fffffff)).long() << 32
        key = key + (0x7fffffff - torch.arange(raw.shape[1], device="cuda"))
        index = 0x7fffffff - (key.topk(case["top"], -1)[0] & 0xffffffff)
        found.update(top_logp=logs.gather(1, index), top_index=index)
    if case["train"]:
        g = torch.where(counted, st["g_logp"], zero)
        grad = -p * (g[:, None] + st["g_entropy"][:, None] * (logs + entropy[:, None]))
        grad.scatter_add_(1, at, g[:, None])
        found["grad_logits"] = (case["scale"] * grad).to(st["logits"].dtype)
    return found


def _bucket(q_boxes, k_boxes, n):
    """[..., Nq, Nk] index into the n x n buckets: the box centres' distance in units of the
    query box's sides, by octaves, binary32 in the written order."""
    half = n // 2
    qc, kc = ((b[..., :2] + b[..., 2:]) * 0.5 for b in (q_boxes, k_boxes))
    inv = torch.ones_like(qc) / (q_boxes[..., 2:] - q_boxes[..., :2]).clamp(min=1.0)
    r = (kc[..., None, :, :] - qc[..., :, None, :]) * inv[..., :, None, :]
    bits = r.abs().contiguous().view(torch.int32) >> (23 - int(math.log2(STEPS)))
    m = (bits - (127 + FIRST) * STEPS + 1).clamp(0, half)
    b = torch.where(r < 0, half - m, half + m).long()
    return b[..., 1] * n + b[..., 0]


def _logits(st):
    """[B, H, Nq, places] of a stream's boxes against what it remembers, -inf past its length."""
    case = st["case"]
    mk, _, sk, _, mb = st["memory"]
    h, n = case["heads"], case["buckets"]
    page = st["pages"].long()
    k = (mk[page].float() * sk[page][..., None]).permute(0, 2, 1, 3, 4).flatten(2, 3)
    k = k.repeat_interleave(h // case["kv_heads"], 1)
    q = st["q"].float().permute(0, 2, 1, 3).contiguous()
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * st["scale"]
    if n:
        idx = _bucket(st["q_boxes"], mb[page].flatten(1, 2), n)
        s = s + st["bias"].view(h, n * n)[:, idx.flatten()].view(h, *idx.shape).transpose(0, 1)
    seen = torch.arange(k.shape[2], device="cuda")[None] < st["lengths"][:, None]
    return s.masked_fill(~seen[:, None, None, :], -math.inf)


DECAY = 0.9


def _plain_weigh(st):
    p = torch.exp(_logits(st) - st["lse"][..., None])
    seen = torch.arange(p.shape[-1], device="cuda")[None] < st["lengths"][:, None]
    w = DECAY * st["weight"] + p.sum((1, 2))
    return {"weight": torch.where(seen, w, torch.zeros_like(w))}


def _plain_evict(st):
    """The kept boxes that lie past the new length go to the places there that are free, both
    in the order of places."""
    weight, pages = st["weight"], st["pages"].long()
    b, places = weight.shape
    at = torch.arange(places, device="cuda").expand(b, places)
    keep = torch.minimum(st["keep"], st["lengths"]).clamp(min=0)
    seen = at < st["lengths"][:, None]
    order = weight.masked_fill(~seen, -math.inf).sort(dim=-1, descending=True, stable=True)[1]
    rank = torch.empty_like(order).scatter_(1, order, at)
    kept = rank < keep[:, None]
    inside = at < keep[:, None]
    free, late = inside & ~kept, kept & ~inside
    # the i-th of the late ones, by its number (the others go to a column of their own)
    late_at = torch.full((b, places + 1), 0, device="cuda")
    late_at.scatter_(1, torch.where(late, late.cumsum(1) - 1, places), at)
    origin = torch.where(free, late_at.gather(1, (free.cumsum(1) - 1).clamp(min=0)), at)
    own_slot = pages[:, :, None] * PAGE + torch.arange(PAGE, device="cuda")
    to = own_slot.flatten(1)
    frm = to.gather(1, origin).flatten()
    to = to.flatten()
    mk, mv, sk, sv, mb = st["memory"]
    fp, fa, tp, ta = frm // PAGE, frm % PAGE, to // PAGE, to % PAGE
    mk[tp, :, ta] = mk[fp, :, fa]
    mv[tp, :, :, ta] = mv[fp, :, :, fa]
    sk[tp, :, ta] = sk[fp, :, fa]
    sv[tp, :, ta] = sv[fp, :, fa]
    mb[tp, ta] = mb[fp, fa]
    none = torch.full_like(origin, -1)
    return {"lengths": keep, "weight": torch.where(inside, weight.gather(1, origin), torch.zeros_like(weight)),
            "origin": torch.where(inside, origin, none).int(), "k": mk, "v": mv, "k_scale": sk,
            "v_scale": sv, "boxes": mb}


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        return {"linear": _plain_linear, "logprob": _plain_logprob, "weigh": _plain_weigh,
                "evict": _plain_evict}[kind](st)
    import paper_1906_07155_amd as rex
    if kind == "linear":
        found, saved = {}, st.get("saved")
        if case["pass"] != "bwd":
            found["y"], saved = rex.linear_act_fwd(st["x"], st["weight"], st["b"], act=case["act"],
                                                   residual=st["residual"],
                                                   save=case["pass"] == "train")
        if case["pass"] != "fwd":
            gx, gw, gb = rex.linear_act_bwd(st["gy"], st["x"], st["weight"], saved, bias=st["b"],
                                            act=case["act"])
            found.update(grad_x=gx, grad_weight=gw)
            if case["bias"]:
                found["grad_bias"] = gb
        return found
    if kind == "logprob":
        logp, entropy, lse, top_logp, top_index = rex.class_logprob_fwd(
            st["logits"], st["labels"], scale=case["scale"], top=case["top"])
        found = {"logp": logp, "entropy": entropy}
        if case["top"]:
            found.update(top_logp=top_logp, top_index=top_index)
        if case["train"]:
            found["grad_logits"] = rex.class_logprob_bwd(
                st["g_logp"], st["g_entropy"], st["logits"], st["labels"], lse, entropy,
                scale=case["scale"])
        return found
    if kind == "weigh":
        geo = {}
        if case["buckets"]:
            geo = dict(q_boxes=st["q_boxes"], bias=st["bias"], first_exp=FIRST, octave_steps=STEPS)
        return {"weight": rex.box_memory_weigh(st["q"], st["memory"], st["pages"], st["lengths"],
                                               st["lse"], weight=st["weight"], decay=DECAY,
                                               scale=st["scale"], **geo)}
    lengths, weight, origin = rex.box_memory_evict(st["memory"], st["pages"], st["lengths"],
                                                   st["weight"], st["keep"])
    mk, mv, sk, sv, mb = st["memory"]
    return {"lengths": lengths, "weight": weight, "origin": origin, "k": mk, "v": mv, "k_scale": sk,
            "v_scale": sv, "boxes": mb}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    size = 2 if case.get("dtype") == "bf16" else 4
    if kind == "linear":
        m, n, k = case["rows"], case["outs"], case["ins"]
        x, w, y = m * k * size, n * k * size, m * n * size
        b = 4 * n if case["bias"] else 0
        # (one value for each of the sums is kept for the slopes; for relu that is y itself)
        kept = 0 if case["act"] == "none" else y
        fwd = x + w + y * (2 if case["residual"] else 1) + b
        bwd = 2 * x + 2 * w + y + b
        total = {"fwd": fwd, "bwd": bwd + kept, "train": fwd + 2 * (kept if case["act"] != "relu" else 0) + bwd}
        return {"bytes": total[case["pass"]],
                "flops": 2 * m * n * k * {"fwd": 1, "bwd": 2, "train": 3}[case["pass"]]}
    if kind == "logprob":
        m, c = case["rows"], case["classes"]
        row = 8 + 4 + 4 + 12 * case["top"]
        if case["train"]:                   # the logits are needed whole before their gradient
            return {"bytes": 2 * m * c * size + m * (row + 8), "flops": 12 * m * c}
        return {"bytes": m * c * size + m * row, "flops": 5 * m * c}
    kv, d, b = case["kv_heads"], case["dim"], case["streams"]
    if kind == "evict":
        keep = _keep_count(case)
        moved = keep * (1.0 - keep / case["tokens"])
        return {"bytes": b * (2 * moved * (2 * kv * (d + 4) + 16) + 4 * case["tokens"] + 8 * keep),
                "flops": b * case["tokens"]}
    t = b * case["tokens"] * (0.875 if case["ragged"] else 1.0)
    q = b * case["queries"] * case["heads"]
    return {"bytes": t * (kv * (d + 4) + 16 + 8) + q * (d * size + 4) + case["heads"] * case["buckets"] ** 2 * 4,
            "flops": 2 * t * case["queries"] * case["heads"] * d}


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------

def _exact_linear(case, st):
    """Gradients by torch.autograd in 64 bits."""
    act = {"none": lambda t: t, "relu": torch.nn.functional.relu, "gelu": torch.nn.functional.gelu,
           "silu": torch.nn.functional.silu}[case["act"]]
    with torch.enable_grad():
        x, w = (st[k].double().requires_grad_(True) for k in ("x", "weight"))
        leaves = {"grad_x": x, "grad_weight": w}
        t = torch.nn.functional.linear(x, w)
        if case["bias"]:
            leaves["grad_bias"] = b = st["b"].double().requires_grad_(True)
            t = t + b
        found = {}
        if case["pass"] != "bwd":
            y = act(t)
            found["y"] = (y + st["residual"].double() if case["residual"] else y).detach()
        if case["pass"] != "fwd":
            g = st["gy"].double()
            at = t if st.get("saved") is None else st["saved"].double().requires_grad_(True)
            if case["act"] != "none":
                g = torch.autograd.grad(act(at), at, g, retain_graph=True)[0]
            found.update(zip(leaves, torch.autograd.grad(t, list(leaves.values()), g)))
    return found


def _exact_logprob(case, st):
    with torch.enable_grad():
        leaf = st["logits"].double().requires_grad_(True)
        logs = torch.log_softmax(leaf * case["scale"], -1)
        entropy = torch.special.entr(logs.exp()).sum(-1)
        counted = (st["labels"] >= 0).double()
        logp = logs[torch.arange(len(leaf), device="cuda"), st["labels"].clamp(min=0)] * counted
        found = {"logp": logp.detach(), "entropy": entropy.detach()}
        if case["top"]:
            order = leaf.detach().sort(dim=-1, descending=True, stable=True)[1][:, :case["top"]]
            found.update(top_logp=logs.detach().gather(1, order), top_index=order)
        if case["train"]:
            loss = (logp * st["g_logp"].double()).sum() + (entropy * st["g_entropy"].double()).sum()
            found["grad_logits"] = torch.autograd.grad(loss, leaf)[0]
    return found


def _exact_buckets(qb, kb, n):
    """[Nq, Nk] buckets of one image: the distance in box sides is a binary32 number by
    definition; its bucket is the count of edges 2^(FIRST + i / STEPS ...) it has reached."""
    edges = [2.0 ** (FIRST + i // STEPS) * (1.0 + (i % STEPS) / STEPS) for i in range(n // 2)]
    edges = torch.tensor(edges, dtype=torch.float64, device=qb.device)
    found = []
    for lo in (0, 1):
        qc = (qb[:, lo] + qb[:, lo + 2]) * 0.5
        kc = (kb[:, lo] + kb[:, lo + 2]) * 0.5
        side = torch.maximum(qb[:, lo + 2] - qb[:, lo], torch.ones_like(qc))
        r = ((kc[None] - qc[:, None]) * side.reciprocal()[:, None]).double()
        m = torch.bucketize(r.abs().contiguous(), edges, right=True)
        found.append(n // 2 + torch.sign(r).long() * m)
    return found[1] * n + found[0]


def _exact_weigh(case, st):
    mk, _, sk, _, mb = st["memory"]
    n, h = case["buckets"], case["heads"]
    bias = st["bias"].double().flatten(1) if n else None
    out = torch.zeros(st["weight"].shape, dtype=torch.float64, device="cuda")
    for i in range(case["streams"]):
        t, page = int(st["lengths"][i]), st["pages"][i].long()
        k = (mk[page].double() * sk[page].double()[..., None]).transpose(1, 2).flatten(0, 1)[:t]
        idx = _exact_buckets(st["q_boxes"][i], mb[page].flatten(0, 1)[:t], n) if n else None
        total = 0.9 * st["weight"][i, :t].double()
        for j in range(h):
            s = st["q"][i, :, j].double() @ k[:, j // (h // case["kv_heads"])].T * st["scale"]
            if n:
                s = s + bias[j][idx]
            total = total + (s - st["lse"][i, j].double()[:, None]).exp().sum(0)
        out[i, :t] = total
    return {"weight": out}


def _exact_evict(case, st):
    """Stream by stream, place by place on the host; the memory's numbers stay what they are."""
    out = torch.zeros(st["weight"].shape, dtype=torch.float64)
    for i in range(case["streams"]):
        t, w = int(st["lengths"][i]), st["weight"][i].double().tolist()
        keep = min(int(st["keep"][i]), t)
        chosen = set(sorted(range(t), key=lambda j: (-w[j], j))[:keep])
        late = iter(sorted(j for j in chosen if j >= keep))
        out[i, :keep] = torch.tensor([w[j if j in chosen else next(late)] for j in range(keep)],
                                     dtype=torch.float64)
    return {"lengths": None, "weight": out, "origin": None, "k": None, "v": None, "k_scale": None,
            "v_scale": None, "boxes": None}


def exact(case, seed):
    st = prepare(case, seed)
    return {"linear": _exact_linear, "logprob": _exact_logprob, "weigh": _exact_weigh,
            "evict": _exact_evict}[case["kind"]](case, st)
