"""What the operators of a relation head are measured on, and their plain forms.

A detector's relation head lets the boxes of an image attend to each other, with a learned
bias that depends on where one box lies as seen from another, and in video lets them attend
to the boxes of earlier frames, which are kept in a paged memory of 8 bits.  Between two
such steps stand norms, a gate and the residual sum.

Kinds of case:
  attn     attention among the boxes of each image, bias by bucket (box_attn_fwd, and in
           training box_attn_bwd)
  write    boxes of a frame quantised into the memory and read back (box_memory_append,
           box_memory_read)
  recall   attention of a frame's boxes over the memory (box_memory_attn_fwd)
  norm     y = x + alpha * gate * N1(branch), u = N2(y) (gated_norm_fwd, and in training
           gated_norm_bwd)

`run` computes the plain forms in binary32, or calls the library where `own` is true;
`exact` is the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 32                       # tokens of one page of the memory
STEPS, FIRST = 1, -4            # bias buckets: one per octave, the first from 2^-4 box sizes
EPS = 1e-6


# ---------------------------------------------------------------------------
# The cases
# ---------------------------------------------------------------------------

def _attn(images, boxes, heads, dim, dtype, train, **kw):
    case = {"kind": "attn", "images": images, "queries": boxes, "keys": boxes, "heads": heads,
            "kv_heads": heads, "dim": dim, "dtype": dtype, "train": train, "buckets": 15,
            "ragged": False, "masked": 0.0}
    case.update(kw)
    return case


def _norm(rows, channels, dtype, train, **kw):
    case = {"kind": "norm", "rows": rows, "channels": channels, "dtype": dtype, "train": train,
            "norm": "rms", "gates": 1}
    case.update(kw)
    return case


def listed():
    return [
        # The 100 detections kept of one image related to each other: the smallest call.
        dict(_attn(1, 100, 8, 32, "bf16", False), name="attn_infer_100_bf16"),
        # Serving: the 1000 proposals of one image, a 1024-channel head.
        dict(_attn(1, 1000, 16, 64, "bf16", False), name="attn_infer_1000_bf16"),
        # A training step on the 512 sampled boxes of each of two images, 256 channels.
        dict(_attn(2, 512, 8, 32, "f32", True), name="attn_train_2x512_f32"),
        # Heads that share keys, an odd number of boxes, some of them padding.
        dict(_attn(3, 171, 6, 48, "f32", True, kv_heads=2, ragged=True, masked=0.1),
             name="attn_train_3x171_shared_f32"),
        # A training step on the proposals NMS keeps in 16 images, up to 1000 each: the largest.
        dict(_attn(16, 1000, 16, 64, "bf16", True, ragged=True), name="attn_train_16x1000_bf16"),
        # One frame's 300 boxes into a video's memory, the last frames read back.
        {"kind": "write", "write": 300, "read": 900, "pages": 256, "kv_heads": 8, "dim": 32,
         "dtype": "bf16", "name": "write_300_bf16"},
        # The proposals of 16 streams at once, in the type their features were trained in.
        {"kind": "write", "write": 16000, "read": 16000, "pages": 2048, "kv_heads": 16, "dim": 64,
         "dtype": "f32", "name": "write_16000_f32"},
        # Tracking: one box in each of 64 streams against all its stream remembers.
        {"kind": "recall", "streams": 64, "queries": 1, "tokens": 8192, "heads": 8, "kv_heads": 8,
         "dim": 32, "buckets": 15, "dtype": "bf16", "ragged": True, "name": "recall_64x1_bf16"},
        # Video detection: a frame's 300 boxes against 20 frames of one stream.
        {"kind": "recall", "streams": 1, "queries": 300, "tokens": 6000, "heads": 16,
         "kv_heads": 16, "dim": 64, "buckets": 15, "dtype": "bf16", "ragged": False,
         "name": "recall_1x300_bf16"},
        # The norms around a block while serving 1000 proposals.
        dict(_norm(1000, 256, "bf16", False), name="norm_infer_1000_bf16"),
        # The same in a training step over 16 images, a gate for each image.
        dict(_norm(16000, 1024, "bf16", True, gates=16), name="norm_train_16000_bf16"),
        # Layer norms with their biases, an odd number of rows and of channels.
        dict(_norm(513, 250, "f32", True, norm="layer"), name="norm_train_513_layer_f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "write", "recall", "recall", "norm", "norm"])
    dtype = rng.choice(["f32", "bf16"])
    dim = rng.choice([32, 64, 64, 40, 96, 128])
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 4])
    if kind == "attn":
        images = _log_int(rng, 1, 16)
        q = _log_int(rng, 1, 800)
        train = rng.random() < 0.6
        case = _attn(images, q, heads, dim, dtype, train, kv_heads=kv,
                     buckets=rng.choice([0, 7, 15, 15, 31]), ragged=rng.random() < 0.5,
                     masked=rng.choice([0.0, 0.0, 0.2]))
        if rng.random() < 0.3:
            case["keys"] = _log_int(rng, 1, 800)
        if heads * dim > 1024:          # never more than the largest listed case
            case["images"] = min(images, 4)
        return case
    if kind == "write":
        n = _log_int(rng, 1, 16000)
        return {"kind": kind, "write": n, "read": _log_int(rng, 1, 16000),
                "pages": (n + PAGE - 1) // PAGE + rng.randint(0, 1024), "kv_heads": kv,
                "dim": dim, "dtype": dtype}
    if kind == "recall":
        streams, q = rng.choice([(_log_int(rng, 1, 64), 1), (_log_int(rng, 1, 8), rng.randint(2, 30)),
                                 (1, _log_int(rng, 30, 300))])
        return {"kind": kind, "streams": streams, "queries": q, "tokens": _log_int(rng, 30, 8192),
                "heads": heads, "kv_heads": kv, "dim": dim, "buckets": rng.choice([0, 7, 15, 31]),
                "dtype": dtype, "ragged": rng.random() < 0.6}
    gates = rng.choice([0, 1, 1, 4])
    rows = _log_int(rng, 1, 16000 if dtype == "bf16" else 8000)
    each = rng.random() < 0.2           # a gate for every row, else for every image
    return _norm(rows if each else max(1, rows // max(1, gates)) * max(1, gates),
                 rng.choice([256, 1024, 1024, 128, 96, 250, 77]), dtype, rng.random() < 0.6,
                 norm=rng.choice(["rms", "layer"]), gates=rows if each else gates)


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


def prepare(case, seed):
    st = {"case": dict(case)}
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = _dtype(case)

    def randn(*shape, dtype=dt):
        return torch.randn(shape, generator=gen, dtype=dtype, device="cuda")

    def below(n, *shape, dtype=torch.int64):
        return torch.randint(0, n, shape, generator=gen, dtype=dtype, device="cuda")

    def shuffled(n):
        return torch.randperm(n, generator=gen, device="cuda")

    kind = case["kind"]
    if kind == "norm":
        m, c = case["rows"], case["channels"]
        st["x"], st["branch"] = randn(m, c), randn(m, c) * 2.0
        one = {"generator": gen, "dtype": torch.float32, "device": "cuda"}
        st["gate"] = 0.5 * torch.randn((case["gates"], c), **one) if case["gates"] else None
        st["w1"], st["w2"] = (1.0 + 0.1 * torch.randn((2, c), **one)).unbind(0)
        st["c1"] = st["c2"] = None
        if case["norm"] == "layer":
            st["c1"], st["c2"] = (0.1 * torch.randn((2, c), **one)).unbind(0)
        if case["train"]:
            st["gy"], st["gu"] = randn(m, c), randn(m, c)
        return st

    d, kv = case["dim"], case["kv_heads"]
    if kind == "attn":
        b, nq, nk = case["images"], case["queries"], case["keys"]
        st["q"], st["k"] = randn(b, nq, case["heads"], d), randn(b, nk, kv, d)
        st["v"] = randn(b, nk, kv, d)
        st["k_boxes"] = _boxes(gen, (b, nk))
        st["q_boxes"] = st["k_boxes"] if nq == nk else _boxes(gen, (b, nq))
        st["q_len"] = st["k_len"] = st["k_mask"] = None
        if case["ragged"]:              # what NMS kept of each image, of one perhaps nothing
            share = 0.6 + 0.4 * torch.rand(b, generator=gen, device="cuda")
            if b > 4:
                share[seed % b] = 0.0
            st["q_len"], st["k_len"] = (share * nq).int(), (share * nk).int()
        if case["masked"]:
            st["k_mask"] = torch.rand((b, nk), generator=gen, device="cuda") >= case["masked"]
        if case["train"]:
            st["gout"] = randn(b, nq, case["heads"], d)
    else:
        # a memory that has been in use: every page holds earlier boxes
        if kind == "recall":
            b, t = case["streams"], case["tokens"]
            per = (t + PAGE - 1) // PAGE
            pages = b * per
            st["pages"] = shuffled(pages).int().view(b, per)
            st["lengths"] = torch.full((b,), t, dtype=torch.int32, device="cuda")
            if case["ragged"]:
                st["lengths"] -= below(t // 4 + 1, b, dtype=torch.int32)
            st["q"] = randn(b, case["queries"], case["heads"], d)
            st["q_boxes"] = _boxes(gen, (b, case["queries"]))
        else:
            n, pages = case["write"], case["pages"]
            st["k"], st["v"], st["boxes"] = randn(n, kv, d), randn(n, kv, d), _boxes(gen, (n,))
            st["slots"] = shuffled(pages * PAGE)[:n].contiguous()
            st["read"] = torch.cat([st["slots"], below(pages * PAGE, case["read"])])
            st["read"] = st["read"][:case["read"]].contiguous()
        def codes(*shape):
            return (below(255, *shape, dtype=torch.int16) - 127).to(torch.int8)

        def scales():
            return (1.5 + torch.rand((pages, kv, PAGE), generator=gen, device="cuda")) / 127.0
        st["memory"] = (codes(pages, kv, PAGE, d), codes(pages, kv, d, PAGE), scales(), scales(),
                        _boxes(gen, (pages, PAGE)))
    n = case.get("buckets", 0)
    if kind in ("attn", "recall"):
        st["scale"] = d ** -0.5
        st["bias"] = randn(case["heads"], n, n, dtype=torch.float32) * 0.5 if n else None
    return st


# ---------------------------------------------------------------------------
# Plain forms (binary32)
# ---------------------------------------------------------------------------

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


def _per_head(x, heads):
    """[B, N, Hkv, D] -> [B, H, N, D] in binary32, shared heads repeated."""
    return x.float().permute(0, 2, 1, 3).repeat_interleave(heads // x.shape[2], 1).contiguous()


def _visible(n, length, mask):
    """[B, 1, 1, Nk] or None."""
    keep = None
    if length is not None:
        keep = torch.arange(n, device="cuda")[None] < length[:, None]
    if mask is not None:
        keep = mask if keep is None else keep & mask
    return None if keep is None else keep[:, None, None, :]


def _softmax(s, keep):
    if keep is not None:
        s = s.masked_fill(~keep, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, torch.ones_like(total), total)


def _logits(q, k, st, idx):
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * st["scale"]
    return s if idx is None else s + st["bias"][:, idx.flatten(0)].view(
        st["bias"].shape[0], *idx.shape).transpose(0, 1)


def _plain_attn(st):
    case, dt = st["case"], st["q"].dtype
    h, hk, n = case["heads"], case["kv_heads"], case["buckets"]
    q, k, v = _per_head(st["q"], h), _per_head(st["k"], h), _per_head(st["v"], h)
    idx = _bucket(st["q_boxes"], st["k_boxes"], n) if n else None
    bias = None
    if n:
        st = dict(st, bias=st["bias"].view(h, n * n))
    p = _softmax(_logits(q, k, st, idx), _visible(case["keys"], st["k_len"], st["k_mask"]))
    rows = None
    if st["q_len"] is not None:
        rows = (torch.arange(case["queries"], device="cuda")[None] < st["q_len"][:, None])
        p = p * rows[:, None, :, None]
    o = torch.matmul(p, v)
    out = o.permute(0, 2, 1, 3).contiguous().to(dt)
    if not case["train"]:
        return {"out": out}
    g = _per_head(st["gout"], h)
    ds = torch.matmul(g, v.transpose(2, 3).contiguous())
    ds = (ds - (g * o).sum(-1, keepdim=True)) * p

    def back(x):                        # [B, H, N, D] -> [B, N, Hkv, D], shared heads summed
        b, _, m, d = x.shape
        return x.view(b, hk, h // hk, m, d).sum(2).permute(0, 2, 1, 3).contiguous().to(dt)

    if n:
        bias = torch.zeros((n * n, h), device="cuda")
        bias.index_add_(0, idx.flatten(), ds.permute(0, 2, 3, 1).reshape(-1, h))
        bias = bias.t().contiguous().view(h, n, n)
    gq = (torch.matmul(ds, k) * st["scale"]).permute(0, 2, 1, 3).contiguous().to(dt)
    gk = back(torch.matmul(ds.transpose(2, 3).contiguous(), q) * st["scale"])
    gv = back(torch.matmul(p.transpose(2, 3).contiguous(), g))
    return {"out": out, "grad_q": gq, "grad_k": gk, "grad_v": gv, "grad_bias": bias}


def _quantise(x):
    x = x.float()
    scale = x.abs().amax(-1) / torch.full((), 127.0, device="cuda")
    code = torch.round(x / torch.where(scale == 0, torch.ones_like(scale), scale)[..., None])
    return code.clamp(-127, 127).to(torch.int8), scale


def _plain_write(st):
    mk, mv, sk, sv, mb = st["memory"]
    dt = st["k"].dtype
    page, at = st["slots"] // PAGE, st["slots"] % PAGE
    (k8, ks), (v8, vs) = _quantise(st["k"]), _quantise(st["v"])
    mk[page, :, at], mv[page, :, :, at], mb[page, at] = k8, v8, st["boxes"]
    sk[page, :, at], sv[page, :, at] = ks, vs
    page, at = st["read"] // PAGE, st["read"] % PAGE
    return {"k": (mk[page, :, at].float() * sk[page, :, at][..., None]).to(dt),
            "v": (mv[page, :, :, at].float() * sv[page, :, at][..., None]).to(dt),
            "boxes": mb[page, at]}


def _plain_recall(st):
    case = st["case"]
    mk, mv, sk, sv, mb = st["memory"]
    b, h, d, n = case["streams"], case["heads"], case["dim"], case["buckets"]
    page = st["pages"].long()           # [B, P] -> [B, Hkv, tokens, D]
    k = (mk[page].float() * sk[page][..., None]).permute(0, 2, 1, 3, 4).flatten(2, 3)
    v = (mv[page].float() * sv[page][..., None, :]).permute(0, 2, 1, 4, 3).flatten(2, 3)
    k, v = (x.repeat_interleave(h // case["kv_heads"], 1) for x in (k, v))
    idx = _bucket(st["q_boxes"], mb[page].flatten(1, 2), n) if n else None
    if n:
        st = dict(st, bias=st["bias"].view(h, n * n))
    s = _logits(_per_head(st["q"], h), k, st, idx)
    p = _softmax(s, _visible(k.shape[2], st["lengths"], None))
    return {"out": torch.matmul(p, v).permute(0, 2, 1, 3).contiguous().to(st["q"].dtype)}


def _plain_norm(st):
    case, dt = st["case"], st["x"].dtype
    layer, train = case["norm"] == "layer", case["train"]
    rows = case["rows"]
    x, b = st["x"].float(), st["branch"].float()
    gate = 0.5
    if st["gate"] is not None:
        gate = 0.5 * st["gate"].repeat_interleave(rows // case["gates"], 0)

    def norm(t, w, c):
        t = t - t.mean(-1, keepdim=True) if layer else t
        rstd = torch.rsqrt((t * t).mean(-1, keepdim=True) + EPS)
        hat = t * rstd
        return hat, rstd, hat * w + c if layer else hat * w

    def back(g, hat, rstd, w):
        g = g * w
        t = g - hat * (g * hat).mean(-1, keepdim=True)
        return rstd * (t - g.mean(-1, keepdim=True) if layer else t)

    hat1, rstd1, z = norm(b, st["w1"], st["c1"])
    y = x + gate * z
    hat2, rstd2, u = norm(y, st["w2"], st["c2"])
    found = {"y": y.to(dt), "u": u.to(dt)}
    if not train:
        return found
    gu = st["gu"].float()
    t = st["gy"].float() + back(gu, hat2, rstd2, st["w2"])
    gz = gate * t
    found.update(grad_x=t.to(dt), grad_branch=back(gz, hat1, rstd1, st["w1"]).to(dt),
                 grad_gate=None, grad_w1=(gz * hat1).sum(0), grad_c1=gz.sum(0) if layer else None,
                 grad_w2=(gu * hat2).sum(0), grad_c2=gu.sum(0) if layer else None)
    if st["gate"] is not None:
        found["grad_gate"] = 0.5 * (t * z).view(case["gates"], -1, t.shape[1]).sum(1)
    return found


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------

def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        found = {"attn": _plain_attn, "write": _plain_write, "recall": _plain_recall,
                 "norm": _plain_norm}[kind](st)
        return {k: v for k, v in found.items() if v is not None}
    import paper_1906_07155_amd as rex
    if kind == "attn":
        geo = {}
        if case["buckets"]:
            geo = dict(q_boxes=st["q_boxes"], k_boxes=st["k_boxes"], bias=st["bias"],
                       first_exp=FIRST, octave_steps=STEPS)
        geo.update(scale=st["scale"], q_len=st["q_len"], k_len=st["k_len"], k_mask=st["k_mask"])
        out, lse, low = rex.box_attn_fwd(st["q"], st["k"], st["v"], save=case["train"], **geo)
        if not case["train"]:
            return {"out": out}
        gq, gk, gv, gb = rex.box_attn_bwd(st["gout"], st["q"], st["k"], st["v"], out, lse, low,
                                          **geo)
        found = {"out": out, "grad_q": gq, "grad_k": gk, "grad_v": gv, "grad_bias": gb}
    elif kind == "write":
        rex.box_memory_append(st["memory"], st["slots"], st["k"], st["v"], st["boxes"])
        k, v, boxes = rex.box_memory_read(st["memory"], st["read"], st["k"].dtype)
        found = {"k": k, "v": v, "boxes": boxes}
    elif kind == "recall":
        geo = {}
        if case["buckets"]:
            geo = dict(q_boxes=st["q_boxes"], bias=st["bias"], first_exp=FIRST,
                       octave_steps=STEPS)
        out, _ = rex.box_memory_attn_fwd(st["q"], st["memory"], st["pages"], st["lengths"],
                                         scale=st["scale"], **geo)
        found = {"out": out}
    else:
        args = dict(gate=st["gate"], alpha=0.5, post_weight=st["w1"], post_bias=st["c1"],
                    pre_weight=st["w2"], pre_bias=st["c2"], norm=case["norm"], eps=EPS)
        y, u, stats = rex.gated_norm_fwd(st["x"], st["branch"], save=case["train"], **args)
        found = {"y": y, "u": u}
        if case["train"]:
            names = ("grad_x", "grad_branch", "grad_gate", "grad_w1", "grad_c1", "grad_w2",
                     "grad_c2")
            found.update(zip(names, rex.gated_norm_bwd(st["gy"], st["gu"], st["x"], st["branch"],
                                                       stats, **args)))
    return {k: v for k, v in found.items() if v is not None}


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    size = 2 if case["dtype"] == "bf16" else 4
    if kind == "norm":
        n, c = case["rows"] * case["channels"], case["channels"]
        params = (case["gates"] + (4 if case["norm"] == "layer" else 2)) * c * 4
        if case["train"]:               # x, branch, y, u; their gradients, in and out
            return {"bytes": 8 * n * size + 2 * params, "flops": 45 * n}
        return {"bytes": 4 * n * size + params, "flops": 15 * n}
    d, kv = case["dim"], case["kv_heads"]
    token = 2 * kv * (d + 4) + 16       # one box in the memory: codes, scales, sides
    if kind == "write":
        n, r = case["write"], case["read"]
        return {"bytes": n * (2 * kv * d * size + 24 + token) + r * (2 * kv * d * size + 24 + token),
                "flops": 6 * n * kv * d + 2 * r * kv * d}
    table = case["heads"] * case["buckets"] ** 2 * 4
    if kind == "recall":
        t = case["streams"] * case["tokens"] * (0.875 if case["ragged"] else 1.0)
        q = case["streams"] * case["queries"] * case["heads"] * d
        return {"bytes": t * token + 2 * q * size + table,
                "flops": 4 * t * case["queries"] * case["heads"] * d}
    share = 0.8 if case["ragged"] else 1.0
    b, nq, nk = case["images"], share * case["queries"], share * case["keys"]
    q, k = b * nq * case["heads"] * d * size, b * nk * kv * d * size
    pairs = b * nq * nk * case["heads"] * d * (1.0 - case["masked"])
    boxes = b * (nq + nk) * 16
    if case["train"]:                   # q, out, both gradients; k, v, their gradients
        return {"bytes": 4 * q + 4 * k + 2 * table + boxes, "flops": 14 * pairs}
    return {"bytes": 2 * q + 2 * k + table + boxes, "flops": 4 * pairs}


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------

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


def _exact_heads(q, k, v, idx, bias, scale, keep, g=None):
    """One image in 64 bits: q [Nq, H, D], k, v [Nk, Hkv, D], keep [Nk] -> o and gradients."""
    nq, h, d = q.shape
    group = h // k.shape[1]
    o = torch.zeros(nq, h, d, dtype=torch.float64, device=q.device)
    gq, gk, gv = torch.zeros_like(o), torch.zeros_like(k), torch.zeros_like(v)
    gb = None if bias is None else torch.zeros_like(bias)
    if bool(keep.any()):
        for i in range(h):
            ki, vi = k[keep][:, i // group], v[keep][:, i // group]
            s = (q[:, i] @ ki.T) * scale
            if bias is not None:
                at = idx[:, keep]
                s = s + bias[i][at]
            p = torch.softmax(s, -1)
            o[:, i] = p @ vi
            if g is None:
                continue
            gi = g[:, i]
            dp = gi @ vi.T
            ds = p * (dp - (p * dp).sum(-1, keepdim=True))
            gq[:, i] = scale * (ds @ ki)
            gk[keep, i // group] += scale * (ds.T @ q[:, i])
            gv[keep, i // group] += p.T @ gi
            if gb is not None:
                gb[i] = torch.bincount(at.flatten(), ds.flatten(), gb.shape[1])
    return o, gq, gk, gv, gb


def _exact_attn(case, st):
    n, b = case["buckets"], case["images"]
    q, k, v = st["q"].double(), st["k"].double(), st["v"].double()
    bias = st["bias"].double().flatten(1) if n else None
    o, gq, gk, gv = (torch.zeros_like(x) for x in (q, q, k, v))
    gb = torch.zeros_like(bias) if n else None
    for i in range(b):
        nq = case["queries"] if st["q_len"] is None else int(st["q_len"][i])
        keep = torch.ones(case["keys"], dtype=torch.bool, device="cuda")
        if st["k_len"] is not None:
            keep[int(st["k_len"][i]):] = False
        if st["k_mask"] is not None:
            keep &= st["k_mask"][i]
        if nq == 0:
            continue
        idx = _exact_buckets(st["q_boxes"][i, :nq], st["k_boxes"][i], n) if n else None
        got = _exact_heads(q[i, :nq], k[i], v[i], idx, bias, st["scale"], keep,
                           st["gout"][i, :nq].double() if case["train"] else None)
        o[i, :nq] = got[0]
        gq[i, :nq], gk[i], gv[i] = got[1:4]
        if n:
            gb += got[4]
    if not case["train"]:
        return {"out": o}
    found = {"out": o, "grad_q": gq, "grad_k": gk, "grad_v": gv}
    if n:
        found["grad_bias"] = gb.view(case["heads"], n, n)
    return found


def _exact_write(case, st):
    """Token by token of what is read: the codes are decided in binary32 by definition."""
    mk, mv, sk, sv, mb = st["memory"]
    k = mk.double() * sk.double()[..., None]
    v = (mv.double() * sv.double()[:, :, None, :]).transpose(2, 3).contiguous()
    boxes = mb.clone()
    page, at = torch.div(st["slots"], PAGE, rounding_mode="floor"), st["slots"].remainder(PAGE)
    for held, new in ((k, st["k"].float()), (v, st["v"].float())):
        step = new.abs().max(-1, keepdim=True).values / torch.full((1,), 127.0, device="cuda")
        held[page, :, at] = (new / step).round().double() * step.double()
    boxes[page, at] = st["boxes"]
    page, at = torch.div(st["read"], PAGE, rounding_mode="floor"), st["read"].remainder(PAGE)
    return {"k": k[page, :, at], "v": v[page, :, at], "boxes": boxes[page, at]}


def _exact_recall(case, st):
    mk, mv, sk, sv, mb = st["memory"]
    n = case["buckets"]
    bias = st["bias"].double().flatten(1) if n else None
    outs = []
    for i in range(case["streams"]):
        t = int(st["lengths"][i])
        page = st["pages"][i].long()
        k = (mk[page].double() * sk[page].double()[..., None]).transpose(1, 2).flatten(0, 1)[:t]
        v = mv[page].double() * sv[page].double()[:, :, None, :]
        v = v.permute(0, 3, 1, 2).flatten(0, 1)[:t]
        idx = _exact_buckets(st["q_boxes"][i], mb[page].flatten(0, 1)[:t], n) if n else None
        keep = torch.ones(t, dtype=torch.bool, device="cuda")
        outs.append(_exact_heads(st["q"][i].double(), k, v, idx, bias, st["scale"], keep)[0])
    return {"out": torch.stack(outs)}


def _exact_norm(case, st):
    """Gradients by torch.autograd in 64 bits."""
    names = ("x", "branch", "gate", "w1", "c1", "w2", "c2")
    with torch.enable_grad():
        leaf = {k: st[k].double().requires_grad_(True) for k in names if st[k] is not None}

        def norm(t, w, c):
            if case["norm"] == "layer":
                dev = t - t.sum(-1, keepdim=True) / t.shape[-1]
                return dev / torch.sqrt((dev ** 2).sum(-1, keepdim=True) / t.shape[-1] + EPS) * w + c
            return t / torch.sqrt((t ** 2).sum(-1, keepdim=True) / t.shape[-1] + EPS) * w

        z = norm(leaf["branch"], leaf["w1"], leaf.get("c1"))
        if "gate" in leaf:
            g = leaf["gate"]
            z = (z.view(g.shape[0], -1, z.shape[1]) * g[:, None]).view_as(z)
        y = leaf["x"] + 0.5 * z
        u = norm(y, leaf["w2"], leaf.get("c2"))
        found = {"y": y.detach(), "u": u.detach()}
        if case["train"]:
            loss = (y * st["gy"].double()).sum() + (u * st["gu"].double()).sum()
            grads = torch.autograd.grad(loss, list(leaf.values()))
            found.update(("grad_" + k, v) for k, v in zip(leaf, grads))
    return found


def exact(case, seed):
    st = prepare(case, seed)
    return {"attn": _exact_attn, "write": _exact_write, "recall": _exact_recall,
            "norm": _exact_norm}[case["kind"]](case, st)
